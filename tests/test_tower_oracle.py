"""The 64-bit definitions of the text tower's operators against differences and
closed forms (CPU)."""

import math

import pytest
import torch

from oracle import tower


def _rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_against_differences(causal):
    cu_q, cu_k = [0, 3, 3, 7, 9], [0, 5, 7, 9, 9]  # more and fewer queries than keys, none of either
    q, k, v, do = _rand(9, 4, 8, seed=1), _rand(9, 2, 8, seed=2), _rand(9, 2, 8, seed=3), _rand(9, 4, 8, seed=4)
    r = tower.attention(q, k, v, cu_q, cu_k, causal, 0.4, do)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        step = _rand(*x.shape, seed=5)
        f = []
        for h in (1e-5, -1e-5):
            y = {"dq": q, "dk": k, "dv": v} | {name: x + h * step}
            f.append(float((tower.attention(y["dq"], y["dk"], y["dv"], cu_q, cu_k, causal, 0.4)["out"] * do).sum()))
        # central difference: the third derivative's h^2 (1e-10) and the cancellation (1e-16 / 1e-5), over sums of order 10
        assert abs((f[0] - f[1]) / 2e-5 - float((r[name] * step).sum())) < 1e-7


def test_attention_sees_what_it_should():
    q, k, v = _rand(3, 1, 8), _rand(2, 1, 8, seed=1), _rand(2, 1, 8, seed=2)
    r = tower.attention(q, k, v, [0, 3], [0, 2], True, 1.0)
    assert (r["out"][0] == 0).all() and r["lse"][0, 0] == -math.inf  # one query more than keys: the first sees none
    assert torch.allclose(r["out"][1], v[0], atol=1e-14)             # ... the second the first key only
    assert abs(float(r["lse"][0, 1]) - float(q[1, 0] @ k[0, 0])) < 1e-12


def test_embedding_gradient_is_the_transpose():
    t = torch.tensor([3, 0, 3, -1, 7, 2])
    w, do = _rand(5, 4, seed=1), _rand(6, 4, seed=2)
    g, _, c = tower.embedding_grad(t, do, 5, 2.0)
    assert c.tolist() == [1, 0, 1, 2, 0]
    assert abs(float((tower.embedding(t, w, 2.0) * do).sum()) - float((w * g).sum())) < 1e-12


def test_checkpoint_bounds():
    x = _rand(5, 70, seed=3).float() * torch.exp2(torch.arange(70.0) - 35)
    q, e = tower.kept(x)
    assert q.abs().max() <= 127 and e.min() >= 1
    step = torch.exp2(e.repeat_interleave(32, 1)[:, :70].double() - 127)
    assert ((tower.unkept(q, e) - x.double()).abs() <= 0.5 * step).all()


@pytest.mark.parametrize("name", ["gelu", "quick_gelu"])
def test_slopes_against_differences(name):
    x = torch.linspace(-9, 9, 721, dtype=torch.float64)
    d = (tower.act(x + 1e-5, name) - tower.act(x - 1e-5, name)) / 2e-5
    assert (d - tower.act_slope(x, name)).abs().max() < 1e-9
