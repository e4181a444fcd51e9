"""The operators of a decoder's attention together, as a serving step calls
them: prompts and single tokens of several sequences against a dense pass."""
import pytest
import torch

import oracle as o
from paper_2109_03513_gb300 import esb, lmrun

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def dense(coded):
    """The numbers of a coded matrix in 64 bits."""
    w = coded.codes
    table = torch.tensor([o.decode(c, 4, coded.fmt.k) for c in range(16)], dtype=torch.float64, device="cuda")
    v = table[torch.stack([(w >> (4 * i)) & 15 for i in range(8)], -1).flatten(1)[:, :coded.cols].long()]
    return v * coded.scales.double().repeat_interleave(coded.group or coded.cols, 1)[:, :coded.cols]


def quantised(x, f):
    """Rows of heads (tokens, heads, d) as the cache holds them."""
    n, h, d = x.shape
    return esb.esb_project_groups(x.float().reshape(n * h, d), f, 0, want_xq=True)[1].double().reshape(n, h, d)


def dense_logits(m, tokens):
    """All tokens of one sequence in 64 bits, with the quantisation of keys and values only."""
    c, d, h, kv = m.cfg, m.head_dim, m.heads, m.kv_heads
    n = tokens.numel()
    x, out = m.ffn.embed[tokens].double(), 0.0
    t = m.rotation.table[:n].double()
    cos, sin = t[:, None, :d // 2], t[:, None, d // 2:]

    def norm(v, w):
        return v / (v.square().mean(-1, keepdim=True) + c.eps).sqrt() * w.double()

    def turn(v):
        a, b = v[..., :d // 2], v[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    for i in range(c.layers):
        wx, wq, wk = m.norms[i]
        x = x + out
        qkv = (norm(x, wx) @ dense(m.qkv[i]).t()).unflatten(1, (-1, d))
        q, k, v = turn(norm(qkv[:, :h], wq)), turn(norm(qkv[:, h:h + kv], wk)), qkv[:, h + kv:]
        k, v = quantised(k, m.caches[i].k_fmt), quantised(v, m.caches[i].v_fmt)
        k, v = k.repeat_interleave(h // kv, 1), v.repeat_interleave(h // kv, 1)
        s = torch.einsum("mhd,nhd->hmn", q, k) / d ** 0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
        a = torch.einsum("hmn,nhd->mhd", torch.softmax(s, -1), v).flatten(1)
        x = x + a @ dense(m.out[i]).t()
        y = norm(x, m.ffn.norms[f"norm{i}"])
        out = torch.relu(y @ dense(m.ffn.w[f"up{i}"]).t()) @ dense(m.ffn.w[f"down{i}"]).t()
    return norm(x + out, m.ffn.norms["norm"]) @ dense(m.ffn.w["head"]).t()


def test_prompts_and_single_tokens_match_a_dense_pass():
    cfg = lmrun.Config(vocab=333, width=128, hidden=192, layers=2)
    m = lmrun.Decoder(cfg, heads=6, kv_heads=2, head_dim=64, pages=40)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    sizes = [40, 1, 23, 100]
    text = [torch.randint(0, cfg.vocab, (n,), generator=g, device="cuda") for n in sizes]
    order = torch.randperm(40, generator=g, device="cuda").to(torch.int32)
    pages = order[:32].reshape(4, 8)
    got = [[] for _ in sizes]
    # the prompt but for its last tokens (in two parts, the sequences out of step), then token by token
    parts = [(30, 0, 0, 17), (33, 0, 0, 17), (33, 0, 10, 94)] + [(min(33 + i, 40), 0, 0, 94 + i) for i in range(1, 7)]
    done = [0] * 4
    for part in parts + [(40, 1, 23, 100)]:
        upto = [max(p, q) for p, q in zip(done, part)]
        new = [text[i][done[i]:upto[i]] for i in range(4)]
        starts = torch.tensor([0] + [sum(len(t) for t in new[:i + 1]) for i in range(4)], dtype=torch.int32, device="cuda")
        logits = m.step(torch.cat(new), starts, torch.tensor(upto, dtype=torch.int32, device="cuda"), pages)
        for i in range(4):
            got[i].append(logits[int(starts[i]):int(starts[i + 1])])
        done = upto
    assert done == sizes
    for i, n in enumerate(sizes):
        y, want = torch.cat(got[i]).double(), dense_logits(m, text[i])
        assert y.shape == want.shape
        # Activations are 8-bit codes (half a step of 1/127 of a row's largest value, itself some 4 times the spread: 0.016
        # of the spread), five times a layer, and bf16; now and then one moves a 4-bit key or value by a step, a seventh of
        # its head's largest.  Logits have a spread of 1: ten such errors of 0.016, added in squares, are 0.05; a single
        # logit may be off by five of those.
        assert (y - want).square().mean().sqrt() < 0.1
        assert (y - want).abs().max() < 0.5
