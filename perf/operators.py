"""The operators of a language model built on ESB codes, as their speed is followed.

Four operators, each through its public entry point where `own` is true and in
elementary torch operations where it is false:

  project   a matrix onto ESB codes with one scale for every `group` values of
            a row (weights laid out for serving; fake-quantised values for
            training)
  matvec    a few rows times a 4-bit group-scaled matrix; the rows are plain
            numbers or 8-bit ESB codes with a scale for each row
  norm      the residual's addition and the root-mean-square norm, its output
            plain, or in 8-bit ESB codes with scales; or forward and backward
  logprobs  log probabilities of given tokens, the entropy and the most likely
            alternatives from a row of logits; or forward and backward

Codes are returned as the values they stand for.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # one small projection of fp32 weights (a 3x3x64 filter bank read as a matrix): all latency
        dict(name="project_512x576_g64_f32", kind="project", rows=512, cols=576, group=64, b=4, k=2, dtype="f32"),
        # the feed-forward weights of a layer converted for serving
        dict(name="project_16384x4096_g128", kind="project", rows=16384, cols=4096, group=128, b=4, k=2, dtype="bf16"),
        # one token through a square projection: the smallest product of a decoding step
        dict(name="matvec_1x4096x4096_g128", kind="matvec", m=1, n=4096, k=4096, group=128, fk=2, x="bf16"),
        # four sequences' 8-bit activations through AlexNet's first classifier layer (9216 -> 4096), small groups
        dict(name="matvec_4x4096x9216_g64_c8", kind="matvec", m=4, n=4096, k=9216, group=64, fk=1, x="codes"),
        # sixteen sequences decoding together through a feed-forward matrix
        dict(name="matvec_16x16384x4096_g128", kind="matvec", m=16, n=16384, k=4096, group=128, fk=2, x="f16"),
        # one token through the output head, the largest matrix of a decoding step
        dict(name="matvec_1x65536x4096_g128", kind="matvec", m=1, n=65536, k=4096, group=128, fk=2, x="bf16"),
        # a decoding step's norm: one row, residual added, 8-bit codes with one scale for the row
        dict(name="norm_1x4096_row", kind="norm", rows=1, cols=4096, dtype="bf16", group=0, b=8, k=6, train=False),
        # a prompt's norm: residual added, 8-bit codes with a scale for every 128 values
        dict(name="norm_8192x4096_g128", kind="norm", rows=8192, cols=4096, dtype="bf16", group=128, b=8, k=6, train=False),
        # a training step's norm, forward and backward
        dict(name="norm_train_8192x4096", kind="norm", rows=8192, cols=4096, dtype="bf16", group=0, b=0, k=0, train=True),
        # one sampled token's log probability with eight alternatives
        dict(name="logprobs_1x131072_top8", kind="logprobs", rows=1, cols=131072, dtype="bf16", top=8, train=False),
        # a scored batch of answers over an odd vocabulary, fp32 logits
        dict(name="logprobs_256x65537_top5", kind="logprobs", rows=256, cols=65537, dtype="f32", top=5, train=False),
        # a training step's loss and its gradient with an entropy term
        dict(name="logprobs_train_4096x49999", kind="logprobs", rows=4096, cols=49999, dtype="bf16", top=0, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd(rng, n, step):
    """n as it is, or on the next multiple of `step`: model widths are mostly round, some are not."""
    n = n if rng.random() < 0.4 else -(-n // step) * step
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["project", "matvec", "matvec", "norm", "norm", "logprobs", "logprobs"])
    if kind == "project":
        cols = _odd(rng, _log(rng, 32, 16384), 128)
        rows = max(1, min(_log(rng, 16, 65536), (1 << 26) // cols))
        b, k = rng.choice([(4, 2), (4, 2), (4, 1), (4, 0), (8, 6), (8, 3)])
        return dict(kind=kind, rows=rows, cols=cols, group=rng.choice([32, 64, 128]), b=b, k=k, dtype=rng.choice(["f32", "f16", "bf16"]))
    if kind == "matvec":
        k = _odd(rng, _log(rng, 64, 16384), 128)
        n = max(16, min(_odd(rng, _log(rng, 64, 65536), 64), (1 << 28) // k))
        return dict(kind=kind, m=_log(rng, 1, 32), n=n, k=k, group=rng.choice([32, 64, 128, 128]), fk=rng.choice([0, 1, 2, 2, 3]),
                    x=rng.choice(["bf16", "bf16", "f16", "f32", "codes"]))
    if kind == "norm":
        cols = _odd(rng, _log(rng, 64, 16384), 128)
        rows = max(1, min(_log(rng, 1, 16384), (1 << 25) // cols))
        train = rng.random() < 0.4
        b, k = (0, 0) if train or rng.random() < 0.25 else rng.choice([(8, 6), (8, 6), (8, 3), (8, 4)])
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), group=rng.choice([0, 64, 128]), b=b, k=k, train=train)
    cols = _odd(rng, _log(rng, 100, 200000), 64)
    rows = max(1, min(_log(rng, 1, 4096), (1 << 27) // cols))
    return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["bf16", "f16", "f32"]), top=min(cols, rng.choice([0, 1, 5, 8, 20])), train=rng.random() < 0.4)


# ------------------------------------------------------------------ ESB formats

def _set(b, k):
    """Value of each of the 2^b codes (sign | exponent | fraction) in units of the scale."""
    n = (1 << (b - k - 1)) - 1
    out = []
    for c in range(1 << b):
        e, f = (c >> k) & n, c & ((1 << k) - 1)
        v = f / (1 << k) if e == n else math.ldexp(1.0 + f / (1 << k), e)
        out.append(-v if c >> (b - 1) else v)
    return out


def _top_value(b, k):
    return max(_set(b, k))


def _nearest(v, b, k):
    """|v| (in units of the scale, any float type) rounded onto the set, ties away from zero, clipped."""
    c = _top_value(b, k)
    e = torch.frexp(v).exponent - 1
    step = torch.ldexp(torch.ones_like(v), e.clamp_min(0) - k)
    t = v / step
    r = torch.floor(t)
    return torch.where(t - r >= 0.5, r + 1, r).mul(step).clamp_max(c)


def _quantise(x, group, b, k):
    """(values, scales) of the rows of x, one scale (the largest magnitude lands on the set's end) per group."""
    rows, cols = x.shape
    g = cols if group == 0 else group
    n = -(-cols // g)
    xp = torch.nn.functional.pad(x, (0, n * g - cols)).reshape(rows, n, g)
    c = torch.full((1,), _top_value(b, k), dtype=x.dtype, device=x.device)
    scale = xp.abs().amax(-1) / c
    s = scale[..., None]
    v = torch.where(s > 0, xp.abs() / s, torch.zeros_like(xp))
    q = torch.copysign(_nearest(v, b, k), xp) * s
    return q.reshape(rows, n * g)[:, :cols], scale


def _pack(values, scale, group, b, k):
    """Code words (rows, words of a multiple of four) of quantised values, as the library lays them out."""
    rows, cols = values.shape
    g = cols if group == 0 else group
    s = scale.repeat_interleave(g, 1)[:, :cols]
    v = torch.where(s > 0, values / s, torch.zeros_like(values))
    pos = _set(b, k)[: 1 << (b - 1)]
    order = sorted(range(len(pos)), key=lambda c: pos[c])
    mids = torch.tensor([(pos[order[i]] + pos[order[i + 1]]) / 2 for i in range(len(order) - 1)], device=DEV, dtype=torch.float32)
    mag = torch.tensor(order, device=DEV)[torch.bucketize(v.abs(), mids)]
    zero = order[0]
    code = torch.where((v < 0) & (mag != zero), mag | (1 << (b - 1)), mag)
    cpw = 32 // b
    words = -(-cols // cpw)
    ld = -(-words // 4) * 4
    code = torch.nn.functional.pad(code, (0, ld * cpw - cols), value=zero).reshape(rows, ld, cpw)
    w = (code << (torch.arange(cpw, device=DEV) * b)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _values(codes, scale, cols, group, b, k, dtype):
    """The numbers that packed codes stand for."""
    table = torch.tensor(_set(b, k), dtype=dtype, device=codes.device)
    sh = torch.arange(32 // b, device=codes.device, dtype=torch.int32) * b
    v = table[((codes[..., None] >> sh) & ((1 << b) - 1)).long()].reshape(codes.shape[0], -1)[:, :cols]
    g = cols if group == 0 else group
    return v * scale.to(dtype).repeat_interleave(g, 1)[:, :cols]


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _normal(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _activations(rows, cols, g):
    """A hidden state: normal values, with a few channels several times as large."""
    big = torch.where(torch.rand(cols, generator=g, device=DEV) < 0.01, 4.0, 1.0)
    return _normal((rows, cols), g) * big


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    if c["kind"] == "project":
        # weights with the spread of a trained matrix: rows of different size
        x = _normal((c["rows"], c["cols"]), g) * (0.5 + torch.rand((c["rows"], 1), generator=g, device=DEV)) / math.sqrt(c["cols"])
        s["x"] = x.to(TYPES[c["dtype"]])
        s["xq"] = torch.empty_like(s["x"])
    elif c["kind"] == "matvec":
        q, s["ws"] = _quantise(_normal((c["n"], c["k"]), g) / math.sqrt(c["k"]), c["group"], 4, c["fk"])
        s["wc"] = _pack(q, s["ws"], c["group"], 4, c["fk"])
        x = _activations(c["m"], c["k"], g)
        if c["x"] == "codes":
            q, s["xs"] = _quantise(x, 0, 8, 6)
            s["xc"] = _pack(q, s["xs"], 0, 8, 6)
        else:
            s["x"] = x.to(TYPES[c["x"]])
        s["y"] = torch.empty((c["m"], c["n"]), dtype=TYPES.get(c["x"], torch.bfloat16), device=DEV)
    elif c["kind"] == "norm":
        t, shape = TYPES[c["dtype"]], (c["rows"], c["cols"])
        s["x"] = _activations(*shape, g).to(t)
        s["r"] = (2.0 * _normal(shape, g)).to(t)
        s["w"] = (1.0 + 0.1 * _normal((c["cols"],), g)).to(t)
        s["h"] = torch.empty_like(s["x"])
        # what the norm hands on: codes stand for values of the model's 16-bit type
        s["y"] = torch.empty(shape, dtype=torch.bfloat16 if c["b"] and c["dtype"] == "f32" else t, device=DEV)
        if c["train"]:
            s["dy"] = (1e-3 * _normal(shape, g)).to(t)
            s["dh"] = (1e-3 * _normal(shape, g)).to(t)
    else:
        t = TYPES[c["dtype"]]
        x = 2.5 * _normal((c["rows"], c["cols"]), g)
        ids = torch.randint(0, max(1, c["cols"] - c["cols"] // 64), (c["rows"],), generator=g, device=DEV)
        # the given token is likely, as an answer's tokens are, and the padded end of the vocabulary is masked
        x.scatter_add_(1, ids[:, None], 6.0 * torch.rand((c["rows"], 1), generator=g, device=DEV))
        x[:, c["cols"] - c["cols"] // 64:] = -math.inf
        s["x"] = x.to(t)
        s["ids"] = ids
        if c["train"]:
            s["ids"] = torch.where(torch.rand(c["rows"], generator=g, device=DEV) < 0.1, -100, ids)  # positions of the prompt
            s["dlogp"] = -torch.rand(c["rows"], generator=g, device=DEV) / c["rows"]
            s["dent"] = -0.01 * torch.rand(c["rows"], generator=g, device=DEV) / c["rows"]
            s["dx"] = torch.empty_like(s["x"])
    return s


# ------------------------------------------------------------------ one pass

def _run_own(s):
    from paper_2109_03513_gb300 import esb

    c = s["case"]
    if c["kind"] == "project":
        coded, xq = esb.esb_project_groups(s["x"], esb.Fmt(c["b"], c["k"]), c["group"], xq=s["xq"])
        return dict(values=xq, scales=coded.scales)
    if c["kind"] == "matvec":
        w = esb.Coded(s["wc"], s["ws"], esb.Fmt(4, c["fk"]), c["k"], c["group"])
        x = esb.Coded(s["xc"], s["xs"], esb.Fmt(8, 6), c["k"], 0) if c["x"] == "codes" else s["x"]
        return esb.esb_matvec_groups(x, w, y=s["y"])
    if c["kind"] == "norm":
        if c["train"]:
            o = esb.esb_rmsnorm(s["x"], s["w"], EPS, residual=s["r"], h=s["h"], y=s["y"], want_rstd=True)
            dx, dw = esb.esb_rmsnorm_backward(s["dy"], o.h, s["w"], o.rstd, dh=s["dh"])
            return dict(h=o.h, y=o.y, dx=dx, dw=dw)
        if c["b"]:
            o = esb.esb_rmsnorm(s["x"], s["w"], EPS, residual=s["r"], h=s["h"], fmt=esb.Fmt(c["b"], c["k"]), group=c["group"], yq=s["y"])
            return dict(h=o.h, values=o.yq, scales=o.coded.scales)
        o = esb.esb_rmsnorm(s["x"], s["w"], EPS, residual=s["r"], h=s["h"], y=s["y"])
        return dict(h=o.h, y=o.y)
    o = esb.esb_logprobs(s["x"], s["ids"], top=c["top"])
    out = dict(logp=o.logp, entropy=o.entropy, lse=o.lse)
    if c["top"]:
        out.update(top_logp=o.top_logp, top_ids=o.top_ids)
    if c["train"]:
        out["dx"] = esb.esb_logprobs_backward(s["x"], s["ids"], o.lse, o.entropy, s["dlogp"], s["dent"], dlogits=s["dx"])
    return out


def _top(x, n):
    """The n largest of each row and their places, the lower place first among equals."""
    bits = x.float().add(0.0).view(torch.int32).long()       # -0 becomes +0
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) + ((1 << 20) - 1 - torch.arange(x.shape[1], device=x.device))
    best = key.topk(n, dim=1).values
    ids = (1 << 20) - 1 - (best & ((1 << 20) - 1))
    return x.gather(1, ids), ids


def run(state):
    s = state
    if own:
        return _run_own(s)
    c = s["case"]
    if c["kind"] == "project":
        q, scales = _quantise(s["x"].float(), c["group"], c["b"], c["k"])
        return dict(values=q.to(s["x"].dtype), scales=scales)
    if c["kind"] == "matvec":
        w = _values(s["wc"], s["ws"], c["k"], c["group"], 4, c["fk"], torch.float32)
        x = _values(s["xc"], s["xs"], c["k"], 0, 8, 6, torch.float32) if c["x"] == "codes" else s["x"].float()
        return (x @ w.t()).to(s["y"].dtype)
    if c["kind"] == "norm":
        t = s["x"].dtype
        z, w = s["x"].float() + s["r"].float(), s["w"].float()
        rstd = 1.0 / (z.square().mean(-1, keepdim=True) + EPS).sqrt()
        y = z * rstd * w
        h = z.to(t)
        if c["train"]:
            dy, hf = s["dy"].float(), h.float()
            n, d = hf * rstd, dy * w
            dx = rstd * (d - n * (d * n).mean(-1, keepdim=True)) + s["dh"].float()
            return dict(h=h, y=y.to(t), dx=dx.to(t), dw=(dy * n).sum(0))
        if c["b"]:
            q, scales = _quantise(y, c["group"], c["b"], c["k"])
            return dict(h=h, values=q.to(s["y"].dtype), scales=scales)
        return dict(h=h, y=y.to(t))
    x, ids = s["x"].float(), s["ids"]
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = d.exp()
    z = e.sum(-1, keepdim=True)
    lz = z.log()
    p = e / z
    lp = d - lz                                               # log probabilities
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    ent = -plp.sum(-1)
    has = ids >= 0
    at = ids.clamp_min(0)[:, None]
    out = dict(logp=torch.where(has, lp.gather(1, at)[:, 0], torch.zeros_like(ent)), entropy=ent, lse=(m + lz)[:, 0])
    if c["top"]:
        best, out["top_ids"] = _top(s["x"], c["top"])
        out["top_logp"] = best.float() - out["lse"][:, None]
    if c["train"]:
        gl = torch.where(has, s["dlogp"], torch.zeros_like(s["dlogp"]))[:, None]
        dx = -gl * p - s["dent"][:, None] * (plp + p * ent[:, None])
        out["dx"] = dx.scatter_add(1, at, gl).to(s["x"].dtype)
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def _size(dtype):
    return {"f32": 4, "f16": 2, "bf16": 2}[dtype]


def work(case):
    c = case
    if c["kind"] == "project":
        n, groups = c["rows"] * c["cols"], c["rows"] * -(-c["cols"] // c["group"])
        return dict(bytes=n * (2 * _size(c["dtype"]) + c["b"] / 8) + 4 * groups, flops=0.0)
    if c["kind"] == "matvec":
        xb, yb = (1, 2) if c["x"] == "codes" else (_size(c["x"]),) * 2
        return dict(bytes=c["n"] * (c["k"] / 2 + 4 * -(-c["k"] // c["group"])) + c["m"] * (c["k"] * xb + c["n"] * yb), flops=2.0 * c["m"] * c["n"] * c["k"])
    if c["kind"] == "norm":
        n, t = c["rows"] * c["cols"], _size(c["dtype"])
        if c["train"]:                                       # x, r, dy, dh in; h, y, dx out; h read again by the backward pass
            return dict(bytes=8.0 * n * t, flops=0.0)
        if c["b"]:
            return dict(bytes=n * (3 * t + 3) + 4 * c["rows"] * (-(-c["cols"] // c["group"]) if c["group"] else 1), flops=0.0)
        return dict(bytes=4.0 * n * t, flops=0.0)
    n, t = c["rows"] * c["cols"], _size(c["dtype"])
    return dict(bytes=n * t * (3.0 if c["train"] else 1.0), flops=0.0)


# ------------------------------------------------------------------ 64-bit results

def _exact_quantise(x, group, b, k):
    """Values and scales by the nearest element of the whole set, half-open cells."""
    rows, cols = x.shape
    g = group or cols
    pos = torch.tensor(sorted(v for v in _set(b, k) if v >= 0 and math.copysign(1.0, v) > 0), dtype=torch.float64, device=x.device)
    mids = (pos[1:] + pos[:-1]) / 2
    scale = torch.stack([x[:, i:i + g].abs().amax(-1) / pos[-1] for i in range(0, cols, g)], 1)
    per = scale[:, torch.arange(cols, device=x.device) // g]
    v = torch.where(per > 0, x.abs() / per, torch.zeros_like(x))
    return torch.sign(x) * pos[torch.bucketize(v, mids, right=True)] * per, scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "project":
        q, scales = _exact_quantise(s["x"].to(f64), c["group"], c["b"], c["k"])
        return dict(values=q, scales=scales)
    if c["kind"] == "matvec":
        x = _values(s["xc"], s["xs"], c["k"], 0, 8, 6, f64) if c["x"] == "codes" else s["x"].to(f64)
        y = torch.empty((c["m"], c["n"]), dtype=f64, device=DEV)
        for i in range(0, c["n"], 4096):                      # a block of the matrix at a time
            w = _values(s["wc"][i:i + 4096], s["ws"][i:i + 4096], c["k"], c["group"], 4, c["fk"], f64)
            y[:, i:i + 4096] = (w[None] * x[:, None]).sum(-1) if c["m"] * w.numel() < 1 << 27 else x @ w.t()
        return y
    if c["kind"] == "norm":
        z = s["x"].to(f64) + s["r"].to(f64)
        h = z.to(s["x"].dtype)
        rms = torch.sqrt((z * z).sum(-1, keepdim=True) / c["cols"] + EPS)
        y = z / rms * s["w"].to(f64)
        if c["train"]:
            n, d = h.to(f64) / rms, s["dy"].to(f64) * s["w"].to(f64)
            dx = (d - n * (d * n).sum(-1, keepdim=True) / c["cols"]) / rms + s["dh"].to(f64)
            return dict(h=z, y=y, dx=dx, dw=(s["dy"].to(f64) * n).sum(0))
        if c["b"]:
            q, scales = _exact_quantise(y, c["group"], c["b"], c["k"])
            return dict(h=z, values=q, scales=scales)
        return dict(h=z, y=y)
    x, ids = s["x"].to(f64), s["ids"]
    lse = torch.log(torch.exp(x - x.amax(-1, keepdim=True)).sum(-1)) + x.amax(-1)
    logp = x - lse[:, None]
    p = torch.exp(logp)
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(-1)
    here = torch.arange(c["cols"], device=DEV)[None] == ids[:, None]
    out = dict(logp=torch.where(here, logp, torch.zeros_like(p)).sum(-1), entropy=ent, lse=lse)
    if c["top"]:
        best, idx = torch.sort(x, dim=1, descending=True, stable=True)
        out.update(top_logp=best[:, :c["top"]] - lse[:, None], top_ids=idx[:, :c["top"]])
    if c["train"]:
        gl = torch.where(ids >= 0, s["dlogp"], torch.zeros_like(s["dlogp"])).to(f64)[:, None]
        neg = torch.where(p > 0, p * (logp + ent[:, None]), torch.zeros_like(p))
        out["dx"] = gl * (here.to(f64) - p) - s["dent"].to(f64)[:, None] * neg
    return out
