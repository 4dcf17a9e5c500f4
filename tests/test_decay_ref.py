"""The tests' plain forms of attention with a decaying bias (CPU): against the oracle's Eq. (10) with
b_t = rate t, against differences and against each other."""
import numpy as np
import pytest
import torch

import decay_ref as ref
import oracle


def _inputs(n, d, m, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k, v, dz = (torch.randn(n, d, generator=g, dtype=torch.float64) * s for s in (0.5, 0.5, 1, 1))
    return q, k, v, dz, torch.randn(m, d, generator=g, dtype=torch.float64)


def _bias(n, rate):
    t = np.arange(-(n - 1), n)
    return np.where(t <= 0, rate * t, -np.inf)[None]


@pytest.mark.parametrize("nprf", [False, True])
@pytest.mark.parametrize("features", ["prf", "elu"])
def test_prompt_is_the_oracles(nprf, features):
    n, d, m, rate = 37, 6, 6, 0.07
    q, k, v, _, W = _inputs(n, d, m)
    z, _, _, _ = ref.prompt(q, k, v, rate, W, nprf=nprf, features=features)
    want, _ = oracle.attention(*(x[None, None].numpy() for x in (q, k, v)), _bias(n, rate), W[None].numpy(), nprf=nprf,
                               kind=features)
    np.testing.assert_allclose(z.numpy(), want[0, 0], rtol=1e-12, atol=1e-13)


def test_a_state_carries_a_prompt_on():
    q, k, v, _, W = _inputs(30, 5, 7)
    z, _, last, _ = ref.prompt(q, k, v, 0.2, W)
    za, _, mid, _ = ref.prompt(q[:11], k[:11], v[:11], 0.2, W)
    zb, _, end, _ = ref.prompt(q[11:], k[11:], v[11:], 0.2, W, state=mid)
    torch.testing.assert_close(torch.cat([za, zb]), z, rtol=1e-12, atol=1e-13)
    torch.testing.assert_close(end, last, rtol=1e-12, atol=1e-13)
    chain, _ = ref.tree(q[11:], k[11:], v[11:], range(-1, 18), 0.2, W, state=mid)
    torch.testing.assert_close(chain, zb, rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("nprf", [False, True])
@pytest.mark.parametrize("features", ["prf", "elu"])
def test_gradients_are_the_differences(nprf, features):
    n, d, rate, h = 9, 4, 0.3, 1e-6
    q, k, v, dz, W = _inputs(n, d, 4, seed=3)
    got = ref.gradients(q, k, v, rate, W, dz, nprf=nprf, features=features)
    for name, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        want = torch.zeros_like(q)
        for e in range(n * d):
            ends = []
            for s in (h, -h):
                x = [q.clone(), k.clone(), v.clone()]
                x[i].view(-1)[e] += s
                ends.append((ref.prompt(*x, rate, W, nprf=nprf, features=features)[0] * dz).sum())
            want.view(-1)[e] = (ends[0] - ends[1]) / (2 * h)
        # differences of 64-bit sums: roundings 1e-16 / h, curvature h^2
        torch.testing.assert_close(got[name][0], want, rtol=1e-6, atol=2e-8)


def test_gradients_are_the_oracles():
    n, d, m, rate = 40, 5, 8, 0.1
    q, k, v, dz, W = _inputs(n, d, m, seed=4)
    got = ref.gradients(q, k, v, rate, W, dz)
    want = oracle.attention_grad(*(x[None, None].numpy() for x in (q, k, v)), _bias(n, rate), W[None].numpy(),
                                 dz[None, None].numpy())
    for name, w in zip(("dq", "dk", "dv"), want):
        np.testing.assert_allclose(got[name][0].numpy(), w[0, 0], rtol=1e-10, atol=1e-12)
