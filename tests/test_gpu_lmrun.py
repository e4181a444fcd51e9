"""The language-model operators together: the example model's answers against
a plain 64-bit forward pass of the values that its codes stand for, and a
short training run."""
import pytest
import torch

from paper_2109_03513_gb300 import esb, lmrun

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def test_answers_match_a_dense_pass():
    cfg = lmrun.Config(vocab=333, width=96, hidden=160, layers=2)
    m = lmrun.Model(cfg, seed=3)
    t = torch.randint(0, cfg.vocab, (5,), device="cuda")
    a = m.serving().answer(t, t, top=4)
    # the same pass from dequantised weights in 64 bits; activations are rounded to 8-bit codes and to bf16 on the
    # way (half a step of 1/127 of a row's largest value for codes, 2^-9 for bf16), each of about relative size 0.01 to
    # the layer's output, so logits of spread 1 agree to a few hundredths: 0.15 is over five of these together
    wq = {n: esb.esb_project_groups(m.p[n], lmrun.W_FMT, lmrun.GROUP, want_xq=True)[1].double() for n in m.matrices()}
    x, out = m.p["embed"][t].double(), 0.0
    for i in range(cfg.layers):
        x = x + out
        y = x / (x.square().mean(1, keepdim=True) + cfg.eps).sqrt() * m.p[f"norm{i}"].double()
        out = torch.relu(y @ wq[f"up{i}"].t()) @ wq[f"down{i}"].t()
    x = x + out
    logits = (x / (x.square().mean(1, keepdim=True) + cfg.eps).sqrt()) @ wq["head"].t()
    want = torch.log_softmax(logits, 1)
    assert (a.logp.double() - want.gather(1, t[:, None])[:, 0]).abs().max() < 0.15
    assert (a.top_logp.double() - want.gather(1, a.top_ids)).abs().max() < 0.15


def test_training_learns_and_the_coded_model_answers():
    # a rule over 1000 tokens from 512 examples a step; an untrained answer is right once in 1000
    assert lmrun.main(steps=150) >= 0.9
