"""The attention of a decoder whose cache is ESB codes, as its operators' speed is followed.

Three operators, each through its public entry point where `own` is true and in
elementary torch operations where it is false:

  headnorm  the root-mean-square norm of every head of queries and keys with the
            position rotation in the same pass; or forward and backward
  append    keys (rotated by their positions) and values of new tokens onto 4-bit
            ESB codes with a scale for each token and head, into the pages of a
            cache; the numbers that the codes stand for beside them
  attend    queries (rotated by their positions) over such a cache: one token of
            each sequence, a few (a draft that is verified), or a part of a prompt

What is held in 4 bits is also returned as the values it stands for.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 500000.0


def _norm(name, tokens, hq, hk, d, dtype, rot, inter, train):
    return dict(name=name, kind="headnorm", tokens=tokens, hq=hq, hk=hk, d=d, dtype=dtype, rot=rot, inter=inter, train=train)


def _append(name, tokens, hk, d, dtype, rot, inter, page, kk, vk, pad):
    return dict(name=name, kind="append", tokens=tokens, hk=hk, d=d, dtype=dtype, rot=rot, inter=inter, page=page, kk=kk, vk=vk, pad=pad)


def _attend(name, seqs, length, ragged, queries, hk, group, d, page, dtype, kk, vk, rot, window):
    return dict(name=name, kind="attend", seqs=seqs, length=length, ragged=ragged, queries=queries, hk=hk, group=group, d=d, page=page,
                dtype=dtype, kk=kk, vk=vk, rot=rot, window=window)


def listed():
    return [
        # a decoding step of one sequence: all latency
        _norm("headnorm_1x40x128", 1, 32, 8, 128, "bf16", 128, False, False),
        # a prompt's queries and keys
        _norm("headnorm_8192x40x128", 8192, 32, 8, 128, "bf16", 128, False, False),
        # a training step of a model with heads of 96, a quarter of them rotated in neighbouring pairs, fp32
        _norm("headnorm_train_2000x15x96_f32", 2000, 12, 3, 96, "f32", 24, True, True),
        # a training step, forward and backward
        _norm("headnorm_train_8192x20x128", 8192, 16, 4, 128, "bf16", 128, False, True),
        # a decoding step of 64 sequences, some places of the batch empty
        _append("append_64x8x128", 64, 8, 128, "bf16", 128, False, 64, 2, 2, 6),
        # a prompt's keys and values
        _append("append_8192x8x128", 8192, 8, 128, "bf16", 128, False, 64, 2, 2, 0),
        # one sequence decoding: the smallest call
        _attend("attend_1x2048", 1, 2048, False, 1, 8, 4, 128, 64, "bf16", 2, 2, 128, 0),
        # a serving step of 64 sequences of different lengths
        _attend("attend_64x8192_ragged", 64, 8192, True, 1, 8, 4, 128, 64, "bf16", 2, 2, 128, 0),
        # heads of 64 without sharing, small pages, a window over the last 1000 tokens, fp16
        _attend("attend_48x4000_window_d64", 48, 4000, True, 1, 16, 1, 64, 16, "f16", 1, 3, 64, 1000),
        # a draft of four tokens verified for each of 24 sequences, twelve queries a head
        _attend("attend_24x10000_draft4", 24, 10000, True, 4, 4, 3, 128, 32, "bf16", 2, 1, 128, 0),
        # four long contexts
        _attend("attend_4x131072", 4, 131072, False, 1, 8, 4, 128, 64, "bf16", 2, 2, 128, 0),
        # a part of each of four prompts over what is in the cache before it
        _attend("attend_4x4096_prompt512", 4, 4096, False, 512, 8, 4, 128, 64, "bf16", 2, 2, 128, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["headnorm", "append", "attend", "attend", "attend"])
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    rot = rng.choice([d, d, d, d // 2, 0])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    inter = rng.random() < 0.3
    if kind == "headnorm":
        hk = rng.choice([1, 2, 4, 5, 8])
        hq = hk * rng.choice([1, 2, 3, 4, 7, 8])
        tokens = max(1, min(_log(rng, 1, 16384), (1 << 25) // ((hq + hk) * d)))
        return _norm("", tokens, hq, hk, d, dtype, rot, inter, rng.random() < 0.5)
    kk, vk = rng.choice([2, 2, 1, 0, 3]), rng.choice([2, 2, 1, 0, 3])
    if kind == "append":
        hk = rng.choice([1, 2, 4, 5, 8, 16])
        tokens = max(1, min(_log(rng, 1, 16384), (1 << 23) // (hk * d)))
        return _append("", tokens, hk, d, dtype, rot, inter, rng.choice([16, 32, 48, 64, 128]), kk, vk, rng.choice([0, 0, 1, 5]))
    hk, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 12, 16])
    queries = rng.choice([1, 1, 1, 2, 4, 8, _log(rng, 16, 512)])
    length = max(queries, _log(rng, 1, 131072))
    most = min(1 << 26, (1 << 34) // (queries * group)) // (hk * d)          # cached places by both costs
    length = max(queries, min(length, most))
    seqs = max(1, min(_log(rng, 1, 128), most // length))
    window = 0 if rng.random() < 0.75 else _log(rng, 1, 4096)
    return _attend("", seqs, length, rng.random() < 0.6, queries, hk, group, d, rng.choice([16, 32, 48, 64, 128]), dtype, kk, vk, rot, window)


# ------------------------------------------------------------------ ESB formats

def _set(k):
    """Value of each of the 16 codes (sign | exponent | fraction) in units of the scale."""
    n = (1 << (3 - k)) - 1
    out = []
    for c in range(16):
        e, f = (c >> k) & n, c & ((1 << k) - 1)
        v = f / (1 << k) if e == n else math.ldexp(1.0 + f / (1 << k), e)
        out.append(-v if c >> 3 else v)
    return out


def _words(d):
    """32-bit words of a head's codes: eight codes each, whole sixteen bytes."""
    return -(-d // 32) * 4


def _quantise(x, k):
    """(values, scales, code words) of the rows of x (fp32; last dimension a head): the largest magnitude lands on the
    set's end, others on the nearest element, ties away from zero."""
    pos = sorted(v for v in _set(k) if v >= 0)
    top = pos[-1]
    scale = x.abs().amax(-1) / torch.full((1,), top, dtype=x.dtype, device=x.device)
    s = scale[..., None]
    v = torch.where(s > 0, x.abs() / s, torch.zeros_like(x))
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v).exponent - 1).clamp_min(0) - k)
    t = v / step
    r = torch.floor(t)
    m = torch.where(t - r >= 0.5, r + 1, r).mul(step).clamp_max(top)
    order = sorted(range(8), key=lambda c: _set(k)[c])
    mids = torch.tensor([(_set(k)[order[i]] + _set(k)[order[i + 1]]) / 2 for i in range(7)], device=x.device)
    mag = torch.tensor(order, device=x.device)[torch.bucketize(m, mids)]
    code = torch.where((x < 0) & (m > 0), mag | 8, mag)
    w = _words(x.shape[-1])
    code = torch.nn.functional.pad(code, (0, w * 8 - x.shape[-1]), value=order[0]).reshape(*x.shape[:-1], w, 8)
    word = (code << (torch.arange(8, device=x.device) * 4)).sum(-1)
    return torch.copysign(m, x) * s, scale, torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def _values(codes, scales, d, k, dtype):
    """The numbers that code words (..., words) with scales (...) stand for: (..., d)."""
    table = torch.tensor(_set(k), dtype=dtype, device=codes.device)
    sh = torch.arange(8, device=codes.device, dtype=torch.int32) * 4
    v = table[((codes[..., None] >> sh) & 15).int()].flatten(-2)[..., :d]
    return v * scales.to(dtype)[..., None]


# ------------------------------------------------------------------ rotation

def _table(rot, positions):
    """cos and sin of every position's angles, computed in 64 bits: (positions, rot) fp32."""
    f = BASE ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _pairs(x, rot, inter):
    """The two halves of the rotated part of heads (..., d)."""
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])


def _join(a, b, rest, inter):
    y = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([y, rest], -1)


def _rotate(x, rows, rot, inter, back=False):
    """Heads x (tokens, heads, d) rotated by the table's rows (tokens, rot)."""
    if rot == 0:
        return x
    a, b = _pairs(x, rot, inter)
    c, s = rows[:, None, :rot // 2].to(x.dtype), rows[:, None, rot // 2:].to(x.dtype)
    s = -s if back else s
    return _join(a * c - b * s, b * c + a * s, x[..., rot:], inter)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _normal(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _heads(tokens, heads, d, g):
    """Projected queries or keys: normal values, some channels of a head several times as large."""
    big = torch.where(torch.rand(heads * d, generator=g, device=DEV) < 0.03, 4.0, 1.0)
    return _normal((tokens, heads * d), g) * big


def _lens(c):
    """Tokens in the cache of each sequence, its queries among them."""
    if not c["ragged"]:
        return [c["length"]] * c["seqs"]
    r = random.Random(c["length"] * 1000 + c["seqs"])
    return [max(c["queries"], int(c["length"] * r.uniform(0.2, 1.0))) for _ in range(c["seqs"])]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    t, d = TYPES[c["dtype"]], c["d"]
    if c["kind"] == "headnorm":
        n, hq, hk = c["tokens"], c["hq"], c["hk"]
        s["table"] = _table(c["rot"], n + 1000)
        s["pos"] = torch.arange(n, device=DEV) + torch.randint(0, 1000, (1,), generator=g, device=DEV)
        # queries, keys and values as one projection makes them
        qkv = torch.cat([_heads(n, hq, d, g), _heads(n, hk, d, g), _normal((n, hk * d), g)], 1).to(t)
        s["q"], s["k"] = qkv[:, :hq * d], qkv[:, hq * d:(hq + hk) * d]
        s["qw"], s["kw"] = ((1.0 + 0.1 * _normal((d,), g)).to(t) for _ in range(2))
        s["qy"], s["ky"] = torch.empty((n, hq * d), dtype=t, device=DEV), torch.empty((n, hk * d), dtype=t, device=DEV)
        if c["train"]:
            s["gq"], s["gk"] = (1e-3 * _normal((n, hq * d), g)).to(t), (1e-3 * _normal((n, hk * d), g)).to(t)
            s["dq"], s["dk"] = torch.empty_like(s["qy"]), torch.empty_like(s["ky"])
        return s
    if c["kind"] == "append":
        n, hk, page = c["tokens"], c["hk"], c["page"]
        pages = -(-n // page) + 8
        s["table"] = _table(c["rot"], n + 1000)
        s["pos"] = torch.arange(n, device=DEV) + torch.randint(0, 1000, (1,), generator=g, device=DEV)
        qkv = torch.cat([_normal((n, hk * d), g), _heads(n, hk, d, g), _normal((n, hk * d), g)], 1).to(t)
        s["k"], s["v"] = qkv[:, hk * d:2 * hk * d], qkv[:, 2 * hk * d:]
        order = torch.randperm(pages, generator=g, device=DEV)
        i = torch.arange(n, device=DEV)
        s["slots"] = order[i // page] * page + i % page
        s["slots"][n - min(c["pad"], n - 1):] = -1                            # places of the batch without a sequence
        for x in ("k", "v"):
            s[x + "_codes"] = torch.zeros((pages, hk, page, _words(d)), dtype=torch.int32, device=DEV)
            s[x + "_scales"] = torch.zeros((pages, hk, page), dtype=torch.float32, device=DEV)
            s[x + "q"] = torch.zeros((n, hk * d), dtype=torch.bfloat16, device=DEV)
        return s
    lens, hk, page = _lens(c), c["hk"], c["page"]
    n, most = c["seqs"] * c["queries"], -(-max(lens) // page)
    pages = c["seqs"] * most + 4
    s["lens_host"] = lens
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["starts"] = torch.arange(c["seqs"] + 1, dtype=torch.int32, device=DEV) * c["queries"]
    s["pages"] = torch.randperm(pages, generator=g, device=DEV)[:c["seqs"] * most].reshape(c["seqs"], most).to(torch.int32)
    s["table"] = _table(c["rot"], max(lens))
    q = torch.cat([1.5 * _heads(n, hk * c["group"], d, g), _normal((n, 2 * hk * d), g)], 1).to(t)
    s["q"] = q[:, :hk * c["group"] * d]
    s["out"] = torch.empty((n, hk * c["group"] * d), dtype=t, device=DEV)
    for x, k in (("k", c["kk"]), ("v", c["vk"])):
        # cached rows out of some thousands of quantised ones, with sizes of their own
        _, scales, codes = _quantise(_heads(4000, 1, d, g) * torch.exp(0.3 * _normal((4000, 1), g)), k)
        at = torch.randint(0, 4000, (pages, hk, page), generator=g, device=DEV)
        s[x + "_codes"], s[x + "_scales"] = codes[at], scales[at]
    return s


# ------------------------------------------------------------------ one pass

def _run_own(s):
    from paper_2109_03513_gb300 import esb

    c = s["case"]
    rot = esb.Rotation(s["table"], c.get("inter", False)) if c["rot"] else None
    if c["kind"] == "headnorm":
        pos = s["pos"] if c["rot"] else None
        o = esb.esb_headnorm(s["q"], s["k"], c["d"], s["qw"], s["kw"], EPS, rotation=rot, positions=pos, qy=s["qy"], ky=s["ky"], want_rstd=c["train"])
        if not c["train"]:
            return dict(q=o.q, k=o.k)
        b = esb.esb_headnorm_backward(s["gq"], s["gk"], s["q"], s["k"], c["d"], s["qw"], s["kw"], o.q_rstd, o.k_rstd, rotation=rot, positions=pos,
                                      dq=s["dq"], dk=s["dk"])
        return dict(q=o.q, k=o.k, dq=b.dq, dk=b.dk, dqw=b.dq_weight, dkw=b.dk_weight)
    cache = esb.KvCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], c["d"], esb.Fmt(4, c["kk"]), esb.Fmt(4, c["vk"]))
    if c["kind"] == "append":
        esb.esb_cache_append(cache, s["k"], s["v"], s["slots"], rotation=rot, positions=s["pos"] if c["rot"] else None, kq=s["kq"], vq=s["vq"])
        return dict(kq=s["kq"], vq=s["vq"], k_codes=s["k_codes"], v_codes=s["v_codes"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return esb.esb_cache_attention(s["q"], cache, s["lens"], s["pages"], starts=s["starts"] if c["queries"] > 1 else None, rotation=rot,
                                   window=c["window"], out=s["out"])[0]


def _plain_headnorm(s, c):
    t, d = TYPES[c["dtype"]], c["d"]
    rows = s["table"][s["pos"]]
    out = {}
    for x in ("q", "k"):
        h = s[x].float().unflatten(1, (-1, d))
        w = s[x + "w"].float()
        rstd = 1.0 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()
        n = h * rstd
        out[x] = _rotate(n * w, rows, c["rot"], c["inter"]).flatten(1).to(t)
        if c["train"]:
            dy = _rotate(s["g" + x].float().unflatten(1, (-1, d)), rows, c["rot"], c["inter"], back=True)
            e = dy * w
            out["d" + x] = (rstd * (e - n * (e * n).mean(-1, keepdim=True))).flatten(1).to(t)
            out["d" + x + "w"] = (dy * n).sum((0, 1))
    return out


def _plain_append(s, c):
    d, hk, page = c["d"], c["hk"], c["page"]
    on = s["slots"] >= 0
    at = s["slots"][on]
    for x, k in (("k", c["kk"]), ("v", c["vk"])):
        h = s[x][on].unflatten(1, (hk, d))
        if x == "k":                                          # in 64 bits: rotated keys may lie next to a border of the set
            h = _rotate(h.double(), s["table"][s["pos"][on]], c["rot"], c["inter"])
        values, scales, codes = _quantise(h.float(), k)
        s[x + "_codes"][at // page, :, at % page] = codes
        s[x + "_scales"][at // page, :, at % page] = scales
        s[x + "q"][on] = values.flatten(1).to(torch.bfloat16)
    return {x + y: s[x + y] for x in ("k", "v") for y in ("q", "_codes", "_scales")}


def _cached(s, c, i, n, x, dtype):
    """Keys or values of the first n places of sequence i: (kv heads, n, d)."""
    at = s["pages"][i, :-(-n // c["page"])].long()
    codes = s[x + "_codes"][at].transpose(0, 1).flatten(1, 2)[:, :n]
    scales = s[x + "_scales"][at].transpose(0, 1).flatten(1, 2)[:, :n]
    return _values(codes, scales, c["d"], c[x + "k"], dtype)


def _plain_attend(s, c):
    d, hk, g, m = c["d"], c["hk"], c["group"], c["queries"]
    out = torch.empty_like(s["out"])
    for i, n in enumerate(s["lens_host"]):
        at = torch.arange(n - m, n, device=DEV)
        q = _rotate(s["q"][i * m:(i + 1) * m].float().unflatten(1, (hk * g, d)), s["table"][at], c["rot"], False)
        q = q.unflatten(1, (hk, g)).permute(1, 0, 2, 3).flatten(1, 2)          # (hk, m g, d)
        k, v = (_cached(s, c, i, n, x, torch.float32) for x in ("k", "v"))
        sc = (q @ k.transpose(1, 2)) / math.sqrt(d)
        p = torch.arange(n, device=DEV)
        seen = p[None] <= at[:, None]
        if c["window"]:
            seen &= p[None] > at[:, None] - c["window"]
        sc = torch.where(seen.repeat_interleave(g, 0)[None], sc, torch.full_like(sc, -math.inf))
        e = (sc - sc.amax(-1, keepdim=True)).exp()
        y = (e @ v) / e.sum(-1, keepdim=True)
        out[i * m:(i + 1) * m] = y.unflatten(1, (m, g)).permute(1, 0, 2, 3).reshape(m, -1).to(out.dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return dict(headnorm=_plain_headnorm, append=_plain_append, attend=_plain_attend)[c["kind"]](state, c)


# ------------------------------------------------------------------ what a pass cannot do without

def _seen(c):
    """(cached places that some query sees, pairs of a query and a place) over the sequences."""
    places = pairs = 0
    for n in _lens(c):
        m, w = c["queries"], c["window"] or n
        places += min(n, w + m - 1)
        pairs += sum(min(n - m + 1 + i, w) for i in range(m))
    return places, pairs


def work(case):
    c = case
    t, d = {"f32": 4, "f16": 2, "bf16": 2}[c["dtype"]], c["d"]
    if c["kind"] == "headnorm":
        n = c["tokens"] * (c["hq"] + c["hk"]) * d
        # x in, y out; the backward pass reads x and dy and writes dx
        return dict(bytes=n * t * (5.0 if c["train"] else 2.0) + c["tokens"] * c["rot"] * 4, flops=0.0)
    row = d / 2 + 4                                                           # codes and scale of a head
    if c["kind"] == "append":
        n = (c["tokens"] - min(c["pad"], c["tokens"] - 1)) * c["hk"] * 2
        return dict(bytes=n * (d * (t + 2) + row) + c["tokens"] * c["rot"] * 4, flops=0.0)
    places, pairs = _seen(c)
    q = c["seqs"] * c["queries"] * c["hk"] * c["group"] * d
    return dict(bytes=2.0 * places * c["hk"] * row + 2.0 * q * t + c["seqs"] * c["queries"] * c["rot"] * 4, flops=4.0 * d * c["hk"] * c["group"] * pairs)


# ------------------------------------------------------------------ 64-bit results

def _turn(x, pos, table, rot, inter):
    """Heads (tokens, heads, d) in 64 bits, turned by complex multiplication."""
    if rot == 0:
        return x
    z = torch.complex(table[pos, :rot // 2].double(), table[pos, rot // 2:].double())[:, None]
    if inter:
        p = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * z
        r = torch.view_as_real(p).flatten(-2)
    else:
        p = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * z
        r = torch.cat([p.real, p.imag], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _exact_headnorm(s, c):
    d, out = c["d"], {}
    for x in ("q", "k"):
        h, w = s[x].double().unflatten(1, (-1, d)), s[x + "w"].double()
        rms = torch.sqrt((h * h).sum(-1, keepdim=True) / d + EPS)
        out[x] = _turn(h / rms * w, s["pos"], s["table"], c["rot"], c["inter"]).flatten(1)
        if c["train"]:
            back = s["table"].clone()
            back[:, c["rot"] // 2:] *= -1
            dy = _turn(s["g" + x].double().unflatten(1, (-1, d)), s["pos"], back, c["rot"], c["inter"])
            dot = (dy * w * h).sum(-1, keepdim=True)
            out["d" + x] = (dy * w / rms - h * dot / (d * rms ** 3)).flatten(1)
            out["d" + x + "w"] = (dy * h / rms).sum((0, 1))
    return out


def _exact_append(s, c):
    d, hk, page, out = c["d"], c["hk"], c["page"], {}
    on = torch.nonzero(s["slots"] >= 0)[:, 0]
    for x, k in (("k", c["kk"]), ("v", c["vk"])):
        h = s[x].double().unflatten(1, (hk, d))
        if x == "k":
            h = _turn(h, s["pos"], s["table"], c["rot"], c["inter"])
        pos = torch.tensor(sorted(v for v in _set(k) if v > 0 or (v == 0 and math.copysign(1, v) > 0)), dtype=torch.float64, device=DEV)
        # a projection takes fp32 numbers, and its scale and quotients are such numbers: ties are those of the rounded quotient
        h = h.float().double()
        scale = (h.abs().amax(-1, keepdim=True) / pos[-1]).float().double()
        ratio = torch.where(scale > 0, h.abs() / scale, torch.zeros_like(h)).float().double()
        near = pos[torch.bucketize(ratio, (pos[1:] + pos[:-1]) / 2, right=True)]
        values = torch.zeros((c["tokens"], hk * d), dtype=torch.float64, device=DEV)
        values[on] = (torch.sign(h) * near * scale).flatten(1)[on]
        scales = s[x + "_scales"].double()
        for head in range(hk):
            scales[s["slots"][on] // page, head, s["slots"][on] % page] = scale[on, head, 0]
        out.update({x + "q": values, x + "_codes": None, x + "_scales": scales})
    return out


def _exact_attend(s, c):
    d, g, m, page = c["d"], c["group"], c["queries"], c["page"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lens(c)):
        pos = torch.arange(n - m, n, device=DEV)
        q = _turn(s["q"][i * m:(i + 1) * m].double().unflatten(1, (-1, d)), pos, s["table"], c["rot"], False)
        p = torch.arange(n, device=DEV)
        page_of, place = s["pages"][i].long()[p // page], p % page
        behind = pos[:, None] - p[None]
        hidden = (behind < 0) | ((behind >= c["window"]) if c["window"] else torch.zeros_like(behind, dtype=torch.bool))
        for h in range(c["hk"]):
            kv = []
            for x in ("k", "v"):
                w = s[x + "_codes"][page_of, h, place].long()
                code = torch.stack([(w >> (4 * j)) & 15 for j in range(8)], -1).flatten(1)[:, :d]
                kv.append(torch.tensor(_set(c[x + "k"]), dtype=torch.float64, device=DEV)[code] * s[x + "_scales"][page_of, h, place].double()[:, None])
            for j in range(h * g, (h + 1) * g):
                sc = torch.einsum("md,nd->mn", q[:, j], kv[0]).div(d ** 0.5).masked_fill(hidden, -math.inf)
                lse = torch.log(torch.exp(sc - sc.amax(1, keepdim=True)).sum(1, keepdim=True)) + sc.amax(1, keepdim=True)
                out[i * m:(i + 1) * m, j * d:(j + 1) * d] = torch.exp(sc - lse) @ kv[1]
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    return dict(headnorm=_exact_headnorm, append=_exact_append, attend=_exact_attend)[c["kind"]](s, c)
