"""Attention with a decaying bias on the GPU (krpe_decay_*): prompts, gradients, single tokens, drafted
trees and copies of states against the plain 64-bit forms of decay_ref.py, elementwise, in units of
what its docstring derives; then what the calls promise about masks, slots, streams and graphs."""
import numpy as np
import pytest
import torch

import decay_ref as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


def _say(*a):
    print(*a, flush=True)


class Case:
    """Seeded inputs of B sequences and H heads."""

    def __init__(self, B, H, n, d, m, dtype="f32", features="prf", nprf=False, rates=None, seed=0, slots=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(1000 * seed + 7 * n + d + m)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.B, self.H, self.n, self.d, self.m = B, H, n, d, m
        self.q, self.k = ((r(B, H, n, d) * d ** -0.25).to(DT[dtype]) for _ in range(2))
        self.v, self.dz = (r(B, H, n, d).to(DT[dtype]) for _ in range(2))
        self.W = None if features == "elu" else r(H, m, d)
        self.rate = torch.tensor(rates, device="cuda") if rates is not None else 0.3 * torch.rand(H, generator=g, device="cuda") ** 4
        self.opt = {"nprf": nprf, "features": features}
        den = 0.1 + torch.rand((slots or B, H, 1, m), generator=g, device="cuda")
        self.state = torch.cat([den * r(slots or B, H, d, m), den], dim=2).contiguous()

    def head(self, b, h, n=None):
        W = None if self.W is None else self.W[h]
        return [x[b, h, :n] for x in (self.q, self.k, self.v)] + [float(self.rate[h]), W]


PROMPTS = [
    # B, H, n, d, m, dtype, features, nprf, state
    (1, 1, 1, 1, 1, "f32", "prf", False, False),
    (2, 2, 1, 64, 64, "bf16", "prf", False, True),
    (1, 2, 2, 3, 5, "f32", "prf", False, True),
    (1, 2, 31, 8, 33, "bf16", "prf", False, False),
    (2, 1, 127, 64, 64, "f32", "prf", False, True),
    (1, 2, 128, 32, 32, "bf16", "prf", True, False),
    (1, 2, 129, 64, 100, "bf16", "prf", False, True),
    (1, 1, 300, 128, 256, "f32", "prf", True, True),
    (1, 1, 300, 100, 130, "bf16", "prf", False, False),
    (1, 1, 257, 128, 1024, "bf16", "prf", False, True),
    (1, 1, 200, 128, 1024, "f32", "prf", False, False),
    (2, 2, 260, 65, 65, "f32", "elu", False, True),
    (2, 2, 130, 64, 64, "bf16", "elu", True, True),
    (1, 3, 2000, 64, 64, "f32", "prf", False, True),
    (1, 2, 4001, 64, 128, "bf16", "prf", True, False),
    (3, 2, 700, 40, 48, "f32", "prf", False, False),
    (40, 3, 300, 16, 24, "f32", "prf", False, True),   # more chunks than CUs
    (40, 3, 300, 16, 24, "bf16", "prf", False, False),
    (32, 4, 40, 16, 24, "bf16", "prf", False, False),  # one chunk from empty states: one launch,
    (65, 3, 40, 16, 24, "bf16", "prf", False, False),  # and two
    (43, 3, 128, 33, 160, "f32", "prf", False, False),
    (2, 2, 100, 72, 90, "bf16", "prf", True, False),
    (1, 2, 390, 96, 300, "f32", "prf", False, True),
]


@pytest.mark.parametrize("B,H,n,d,m,dt,features,nprf,with_state", PROMPTS)
def test_prompt(gpu_lib, B, H, n, d, m, dt, features, nprf, with_state):
    _say(f"prompt B={B} H={H} n={n} d={d} m={m} {dt} {features} nprf={nprf}")
    c = Case(B, H, n, d, m, dt, features, nprf)
    before = c.state.clone()
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, fresh=not with_state, **c.opt)
    alone = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, **c.opt)
    assert z.dtype == c.q.dtype
    worst = [0.0, 0.0]
    for b in range(B):
        for h in range(H):
            first = before[b, h] if with_state else None
            want, scale, last, lscale = ref.prompt(*c.head(b, h), state=first, **c.opt)
            worst[0] = max(worst[0], ref.excess(z[b, h], want, scale, z.dtype))
            worst[1] = max(worst[1], ref.excess(c.state[b, h], last, lscale, torch.float32, ref.STATE_DELTA))
    _say(f"  z {worst[0]:.3f}, state {worst[1]:.3f} of what is allowed")
    assert max(worst) <= 1.0
    if not with_state:
        assert torch.equal(alone, z)      # the state that is kept changes nothing


@pytest.mark.parametrize("rates", [[0.0, 1e-4], [INF, 50.0], [0.02, 3.0], [-0.01, 0.0], [24.0, 41.0]])
def test_rates(gpu_lib, rates):
    _say("rates", rates)
    c = Case(1, 2, 400, 16, 24, rates=rates)
    before = c.state.clone()
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state)
    for h in range(2):
        want, scale, last, lscale = ref.prompt(*c.head(0, h), state=before[0, h])
        assert ref.excess(z[0, h], want, scale, z.dtype) <= 1.0
        assert ref.excess(c.state[0, h], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0


def test_next_positions_of_little_weight(gpu_lib):
    """Keys that match a query badly beside one that does, three positions before at 32 bits each."""
    _say("little weight")
    n, d = 128, 16
    c = Case(1, 1, n, d, 8, rates=[32 * float(np.log(2.0))])
    x = torch.zeros(n, d, device="cuda")
    x[:, 0] = torch.tensor([-7.0, -7.0, -7.0, 7.0], device="cuda").repeat(n // 4)
    c.k[0, 0], c.q[0, 0] = x, x[3]
    c.W.fill_(0.0)
    c.W[0, :, 0] = 7.0        # phi(q) . phi(k): 1 or, for the others, e^-98 = 2^-141 of it
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    # a matching key and the three rows after it, which it weighs 2^-32, 2^-64 and 2^-96: the others 2^-45 of that at most
    want = c.v[0, 0, 3:127].double().view(31, 4, d)[:, :1]
    assert float((z[0, 0, 3:127].view(31, 4, d) - want).abs().max()) <= 4e-5 * float(want.abs().max())


@pytest.mark.parametrize("size", [3e-7, 3e-5])
def test_small_projections(gpu_lib, size):
    """W below what its operands' type holds without loss: phi is as near as elsewhere."""
    _say("small W", size)
    c = Case(1, 2, 200, 64, 64, rates=[3.0, 2.0])
    c.W.mul_(size)
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, fresh=True)
    for h in range(2):
        want, scale, last, lscale = ref.prompt(*c.head(0, h))
        assert ref.excess(z[0, h], want, scale, z.dtype) <= 1.0
        assert ref.excess(c.state[0, h], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0


def test_is_eq10_with_that_bias(gpu_lib):
    """The framework's own attention, given the bias explicitly."""
    _say("against attention_fwd")
    c = Case(2, 2, 500, 64, 64)
    t = torch.arange(-499, 500, device="cuda", dtype=torch.float32)
    b = torch.where(t <= 0, c.rate[:, None] * t, torch.full_like(t, -INF))
    want = gpu_lib.attention_fwd(c.q, c.k, c.v, b, c.W, causal=True)
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    # attention_fwd's own bar against 64 bits is 2e-4 of a row's largest element
    assert float(((z - want).abs().amax(-1) / want.abs().amax(-1)).max()) <= 2e-4


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_lens(gpu_lib, dt):
    _say("lens", dt)
    n, lens = 300, [0, 1, 128, 129, 300, 999, -4]
    c = Case(len(lens), 2, n, 24, 40, dt)
    real = [min(max(x, 0), n) for x in lens]
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    before = c.state.clone()
    for b, x in enumerate(real):  # what lies behind a sequence is not looked at
        for t in (c.q, c.k, c.v, c.dz):
            t[b, :, x:] = NAN
    out = torch.full_like(c.q, 7.0)
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, lens=ln, out=out)
    zeros = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, lens=ln)
    grads = gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz, lens=ln)
    assert z is out
    for b, x in enumerate(real):
        assert bool((z[b, :, x:] == 7).all()) and bool((zeros[b, :, x:] == 0).all())
        assert all(bool((g[b, :, x:] == 0).all()) for g in grads)
        for h in range(2):
            if x == 0:
                assert torch.equal(c.state[b, h], before[b, h])
                continue
            want, scale, last, lscale = ref.prompt(*c.head(b, h, x), state=before[b, h])
            assert ref.excess(z[b, h, :x], want, scale, z.dtype) <= 1.0
            assert ref.excess(c.state[b, h], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0
            g = ref.gradients(*c.head(b, h, x), c.dz[b, h, :x])
            for name, got in zip(("dq", "dk", "dv"), grads):
                assert ref.excess(got[b, h, :x], *g[name], got.dtype, ref.GRAD_DELTA[got.dtype]) <= 1.0, name


@pytest.mark.parametrize("n,d", [(40, 7), (300, 24), (513, 72)])
def test_rows_behind_lens_are_cleared(gpu_lib, n, d):
    """Outputs in memory that held something else, one chunk or more, with and without a state."""
    _say("cleared rows", n, d)
    lens = [0, 1, n // 2, n]
    c = Case(4, 3, n, d, 33, "bf16")
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for with_state in (False, True):
        for _ in range(2):
            junk = [torch.full_like(c.q, 7.0) for _ in range(6)]
            del junk
            outs = [gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, lens=ln, state=c.state if with_state else None),
                    *gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz, lens=ln)]
            for b, x in enumerate(lens):
                assert all(bool((o[b, :, x:] == 0).all()) and bool(o[b].isfinite().all()) for o in outs)


def test_empty_prompts(gpu_lib):
    _say("n = 0")
    c = Case(2, 2, 0, 8, 16, slots=4)
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    before = c.state.clone()
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, slots=slots)
    assert z.shape == (2, 2, 0, 8) and torch.equal(c.state, before)
    gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, slots=slots, fresh=True)
    assert bool((c.state[[1, 3]] == 0).all()) and torch.equal(c.state[[0, 2]], before[[0, 2]])
    assert gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.q)[2].numel() == 0


GRADS = [
    (1, 1, 1, 4, 4, "f32", "prf", False),
    (1, 2, 2, 3, 5, "f32", "prf", True),
    (2, 2, 33, 16, 20, "bf16", "prf", False),
    (1, 2, 128, 64, 64, "f32", "prf", False),
    (1, 2, 129, 64, 32, "bf16", "prf", True),
    (1, 1, 300, 128, 256, "f32", "prf", False),
    (1, 1, 257, 100, 130, "bf16", "prf", False),
    (1, 1, 140, 128, 1024, "f32", "prf", False),
    (2, 2, 260, 65, 65, "f32", "elu", False),
    (1, 2, 300, 64, 64, "bf16", "elu", True),
    (1, 2, 1500, 32, 64, "f32", "prf", False),
    (1, 1, 2600, 64, 64, "bf16", "prf", False),
    (40, 3, 300, 16, 24, "f32", "prf", False),         # more chunks than CUs
    (40, 3, 300, 16, 24, "bf16", "prf", False),
    (1, 2, 270, 72, 90, "bf16", "prf", True),
    (1, 1, 200, 96, 300, "f32", "prf", False),
]


@pytest.mark.parametrize("B,H,n,d,m,dt,features,nprf", GRADS)
def test_gradients(gpu_lib, B, H, n, d, m, dt, features, nprf):
    _say(f"gradients B={B} H={H} n={n} d={d} m={m} {dt} {features} nprf={nprf}")
    c = Case(B, H, n, d, m, dt, features, nprf)
    got = gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz, **c.opt)
    again = gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz, **c.opt)
    worst = {}
    for b in range(B):
        for h in range(H):
            want = ref.gradients(*c.head(b, h), c.dz[b, h], **c.opt)
            for name, x in zip(("dq", "dk", "dv"), got):
                worst[name] = max(worst.get(name, 0.0), ref.excess(x[b, h], *want[name], x.dtype, ref.GRAD_DELTA[x.dtype]))
    _say("  ", {k: round(v, 3) for k, v in worst.items()}, "of what is allowed")
    assert max(worst.values()) <= 1.0
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("features", ["prf", "elu"])
def test_gradients_are_the_differences(gpu_lib, features):
    """Along one direction of all inputs, differences of the forward pass on the GPU."""
    _say("differences", features)
    c = Case(1, 1, 150, 16, 16, features=features)
    g = gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz, **c.opt)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    u = [torch.randn(x.shape, generator=gen, device="cuda") for x in (c.q, c.k, c.v)]
    h = 2e-3
    ends = []
    for s in (h, -h):
        z = gpu_lib.decay_attention_fwd(*(x + s * y for x, y in zip((c.q, c.k, c.v), u)), c.rate, c.W, **c.opt)
        ends.append(float((z.double() * c.dz.double()).sum()))
    got, want = sum(float((x.double() * y.double()).sum()) for x, y in zip(g, u)), (ends[0] - ends[1]) / (2 * h)
    # the 2400 values of z are off by 1e-6 at random (sum 5e-5, over 2 h: 0.02); the third
    # derivative along a direction of norm sqrt(7200) adds h^2 / 6 of about norm^3: below 0.5
    norm = sum(float((x.double() ** 2).sum()) for x in g) ** 0.5
    assert abs(got - want) <= 0.52 + 0.01 * norm, (got, want, norm)


STEPS = [
    (1, 1, 1, 1, "f32", "prf", False),
    (3, 2, 64, 64, "bf16", "prf", False),
    (2, 2, 3, 5, "f32", "prf", True),
    (5, 3, 128, 256, "bf16", "prf", False),
    (2, 1, 128, 1024, "f32", "prf", False),
    (2, 2, 30, 77, "bf16", "prf", True),
    (2, 2, 20, 300, "f32", "prf", False),     # features past 256 that do not fill a wave
    (1, 2, 64, 513, "bf16", "prf", False),
    (4, 2, 65, 65, "f32", "elu", False),
    (40, 2, 64, 128, "bf16", "prf", False),
]


@pytest.mark.parametrize("B,H,d,m,dt,features,nprf", STEPS)
def test_step(gpu_lib, B, H, d, m, dt, features, nprf):
    _say(f"step B={B} H={H} d={d} m={m} {dt} {features}")
    c = Case(B, H, 1, d, m, dt, features, nprf, slots=B + 3)
    slots = torch.randperm(B + 3, generator=torch.Generator().manual_seed(1))[:B].to(torch.int32).cuda()
    before = c.state.clone()
    z = gpu_lib.decay_attention_step(c.q[:, :, 0], c.k[:, :, 0], c.v[:, :, 0], c.rate, c.W, c.state, slots=slots, **c.opt)
    others = [s for s in range(B + 3) if s not in slots.tolist()]
    assert torch.equal(c.state[others], before[others])
    for b in range(B):
        for h in range(H):
            s = int(slots[b])
            want, scale, last, lscale = ref.prompt(*c.head(b, h), state=before[s, h], **c.opt)
            assert ref.excess(z[b, h][None], want, scale, z.dtype) <= 1.0
            assert ref.excess(c.state[s, h], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0


def test_step_of_states_past_the_cache(gpu_lib):
    """More than 256 MiB of states, beside the same in two halves."""
    _say("step past the cache")
    for d, m, B in ((64, 256, 260), (30, 77, 1900)):
        c = Case(B, 16, 1, d, m, "bf16")
        token = [x[:, :, 0].contiguous() for x in (c.q, c.k, c.v)]
        halves = c.state.clone()
        z = gpu_lib.decay_attention_step(*token, c.rate, c.W, c.state)
        at = B // 2
        for part in (slice(0, at), slice(at, B)):
            y = gpu_lib.decay_attention_step(*(x[part] for x in token), c.rate, c.W, halves[part])
            assert torch.equal(y, z[part])
        assert torch.equal(halves, c.state)


def _random_tree(rng, T):
    return [-1] + [int(rng.integers(-1, t)) for t in range(1, T)]


TREES = [
    (1, 1, 1, 4, 4, "f32", "prf", False),
    (2, 2, 2, 64, 64, "bf16", "prf", False),
    (1, 2, 12, 64, 128, "bf16", "prf", False),
    (2, 1, 31, 3, 5, "f32", "prf", True),
    (1, 2, 32, 64, 100, "f32", "prf", False),
    (2, 2, 33, 128, 256, "bf16", "prf", False),
    (1, 2, 64, 64, 64, "f32", "prf", False),
    (1, 1, 64, 128, 1024, "f32", "prf", False),
    (1, 2, 50, 65, 65, "bf16", "elu", True),
    (1, 2, 64, 100, 130, "bf16", "prf", False),
    (1, 2, 40, 72, 90, "f32", "prf", True),
    (1, 1, 20, 96, 300, "bf16", "prf", False),
]


@pytest.mark.parametrize("B,H,T,d,m,dt,features,nprf", TREES)
def test_tree(gpu_lib, B, H, T, d, m, dt, features, nprf):
    _say(f"tree B={B} H={H} T={T} d={d} m={m} {dt} {features}")
    c = Case(B, H, T, d, m, dt, features, nprf, slots=B + 2)
    rng = np.random.default_rng(T)
    parent = torch.tensor([_random_tree(rng, T) for _ in range(B)], dtype=torch.int32, device="cuda")
    slots = torch.tensor([B + 1 - b for b in range(B)], dtype=torch.int32, device="cuda")
    before = c.state.clone()
    z = gpu_lib.decay_attention_tree(c.q, c.k, c.v, parent, c.rate, c.W, c.state, slots=slots, **c.opt)
    assert torch.equal(c.state, before)
    for b in range(B):
        for h in range(H):
            want, scale = ref.tree(*c.head(b, h)[:3], parent[b].tolist(), *c.head(b, h)[3:], state=before[int(slots[b]), h],
                                   **c.opt)
            assert ref.excess(z[b, h], want, scale, z.dtype) <= 1.0
    # a path taken in is the prompt of its tokens
    path = []
    for b in range(B):
        node, p = T - 1, []
        while node >= 0:
            p.append(node)
            node = int(parent[b, node])
        path.append(p[::-1])
    pt = torch.full((B, T + 1), -1, dtype=torch.int32)
    for b, p in enumerate(path):
        pt[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    gpu_lib.decay_attention_commit(c.k, c.v, pt.cuda(), c.rate, c.W, c.state, slots=slots, **c.opt)
    for b, p in enumerate(path):
        for h in range(H):
            q, k, v, rate, W = c.head(b, h)
            s = int(slots[b])
            _, _, last, lscale = ref.prompt(q[p], k[p], v[p], rate, W, state=before[s, h], **c.opt)
            assert ref.excess(c.state[s, h], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0
    others = [s for s in range(B + 2) if s not in slots.tolist()]
    assert torch.equal(c.state[others], before[others])


@pytest.mark.parametrize("T", [20, 45])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_tree_masks(gpu_lib, T, dt):
    """Nodes without valid parents give zeros, and what a node does not see does not reach it."""
    _say("tree masks", T, dt)
    c = Case(1, 1, T, 16, 40, dt)
    parent = _random_tree(np.random.default_rng(3), T)
    parent[4], parent[9] = -7, 9          # padding: no parent, its own parent
    want, scale = ref.tree(*c.head(0, 0)[:3], parent, *c.head(0, 0)[3:], state=c.state[0, 0])
    pt = torch.tensor([parent], dtype=torch.int32, device="cuda")
    z = gpu_lib.decay_attention_tree(c.q, c.k, c.v, pt, c.rate, c.W, c.state)
    dead = [t for t in range(T) if float(scale[t].abs().max()) == 0]
    assert {4, 9} <= set(dead) and bool((z[0, 0, dead] == 0).all())
    assert ref.excess(z[0, 0], want, scale, z.dtype) <= 1.0
    # a value and a key that are not finite, at two nodes: only what is below them changes
    below = {2: {2}, T - 3: {T - 3}}
    for t in range(T):
        for s in below.values():
            if parent[t] in s and 0 <= parent[t] < t:
                s.add(t)
    c.v[0, 0, 2, 5], c.k[0, 0, T - 3, 1] = INF, NAN
    y = gpu_lib.decay_attention_tree(c.q, c.k, c.v, pt, c.rate, c.W, c.state)
    for t in range(T):
        if t in dead:
            assert bool((y[0, 0, t] == 0).all())
        elif t in below[T - 3]:
            assert bool(y[0, 0, t].isnan().all())
        else:
            keep = torch.ones(16, dtype=torch.bool)
            keep[5] = t not in below[2]
            assert torch.equal(y[0, 0, t][keep], z[0, 0, t][keep])
            assert keep[5] or not bool(y[0, 0, t, 5].isfinite())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_prompt_values_that_are_not_finite(gpu_lib, dt):
    """They reach the rows from theirs on, in their column (a key's: in all), and nothing before."""
    _say("not finite", dt)
    c = Case(1, 2, 300, 16, 40, dt)
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    c.v[0, 0, 70, 3], c.v[0, 0, 200, 9], c.k[0, 1, 150, 0] = NAN, -INF, NAN
    y = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    assert torch.equal(y[0, 1, :150], z[0, 1, :150]) and bool(y[0, 1, 150:].isnan().all())
    cols = [x for x in range(16) if x not in (3, 9)]
    assert torch.equal(y[0, 0][:, cols], z[0, 0][:, cols])
    for col, at in ((3, 70), (9, 200)):
        assert torch.equal(y[0, 0, :at, col], z[0, 0, :at, col]) and not bool(y[0, 0, at:, col].isfinite().any())


def test_slots_that_are_refused(gpu_lib):
    """-1: nothing before, nothing kept.  Outside the pool, or named twice: NaN, the pool as it was."""
    _say("slots")
    B, H, n, d, m = 7, 2, 140, 16, 32
    c = Case(B, H, n, d, m, slots=5)
    slots = torch.tensor([2, -1, 5, 3, 0, 3, -2], dtype=torch.int32, device="cuda")
    bad, good = [2, 3, 5, 6], [0, 1, 4]
    parent = torch.tensor([list(range(-1, 19))] * B, dtype=torch.int32, device="cuda")
    path = parent[:, 1:].contiguous()
    before = c.state.clone()

    def check(z, n):
        assert bool(z[bad].isnan().all()) and bool(z[good].isfinite().all())
        for b in good:
            for h in range(H):
                first = before[int(slots[b]), h] if int(slots[b]) >= 0 else None
                want, scale, _, _ = ref.prompt(*c.head(b, h, n), state=first)
                assert ref.excess(z[b, h], want, scale, z.dtype) <= 1.0

    check(gpu_lib.decay_attention_tree(c.q[:, :, :20], c.k[:, :, :20], c.v[:, :, :20], parent, c.rate, c.W, c.state,
                                       slots=slots), 20)
    assert torch.equal(c.state, before)
    for call in ("fwd", "step", "commit"):
        c.state.copy_(before)
        if call == "fwd":
            check(gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, slots=slots), n)
        elif call == "step":
            check(gpu_lib.decay_attention_step(c.q[:, :, 0], c.k[:, :, 0], c.v[:, :, 0], c.rate, c.W, c.state,
                                               slots=slots)[:, :, None], 1)
        else:
            gpu_lib.decay_attention_commit(c.k[:, :, :20], c.v[:, :, :20], path, c.rate, c.W, c.state, slots=slots)
        assert torch.equal(c.state[[1, 3, 4]], before[[1, 3, 4]]), call
        assert not torch.equal(c.state[0], before[0]) and not torch.equal(c.state[2], before[2])


def test_commit_stops_at_what_is_no_node(gpu_lib):
    _say("commit paths")
    c = Case(4, 1, 6, 8, 16)
    path = torch.tensor([[0, 1, 6, 2], [-1, 0, 0, 0], [3, 3, 5, -9], [5, 4, 3, 2]], dtype=torch.int32, device="cuda")
    taken = [[0, 1], [], [3, 3, 5], [5, 4, 3, 2]]
    before = c.state.clone()
    gpu_lib.decay_attention_commit(c.k, c.v, path, c.rate, c.W, c.state)
    for b, p in enumerate(taken):
        if not p:
            assert torch.equal(c.state[b], before[b])
            continue
        q, k, v, rate, W = c.head(b, 0)
        _, _, last, lscale = ref.prompt(q[p], k[p], v[p], rate, W, state=before[b, 0])
        assert ref.excess(c.state[b, 0], last, lscale, torch.float32, ref.STATE_DELTA) <= 1.0


@pytest.mark.parametrize("count,nslots,H,d,m", [(1, 1, 1, 1, 1), (5, 4, 3, 3, 5), (32, 16, 2, 64, 64), (64, 200, 1, 8, 12),
                                                (65, 70, 2, 8, 12), (256, 40, 1, 7, 9), (256, 300, 2, 64, 64)])
def test_state_copy(gpu_lib, count, nslots, H, d, m):
    """Forks, cycles, clears, repeated targets and moves outside the pool, against moves on a snapshot."""
    _say(f"copy count={count} nslots={nslots}")
    rng = np.random.default_rng(count)
    state = torch.from_numpy(rng.standard_normal((nslots, H, d + 1, m)).astype(np.float32)).cuda()
    src, dst = rng.integers(-3, nslots + 2, count), rng.integers(-2, nslots + 2, count)
    want = state.clone()
    for s, t in zip(src, dst):
        if -1 <= s < nslots and 0 <= t < nslots:
            want[t] = state[int(s)] if s >= 0 else 0.0
    gpu_lib.decay_state_copy(state, *(torch.from_numpy(x.astype(np.int32)).cuda() for x in (src, dst)))
    assert torch.equal(state, want)


def test_serving_run(gpu_lib):
    """Prompts, tokens, drafted trees, forks and further tokens through one pool are the whole sequences."""
    _say("serving")
    B, H, d, m = 3, 2, 32, 64
    c = Case(B, H, 420, d, m, "bf16")
    pool = gpu_lib.decay_state(6, H, d, m)
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    whole = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    row = lambda x, i: x[:, :, i].contiguous()
    z = [gpu_lib.decay_attention_fwd(*(x[:, :, :200].contiguous() for x in (c.q, c.k, c.v)), c.rate, c.W, state=pool,
                                     slots=slots)]
    for i in range(200, 210):
        z.append(gpu_lib.decay_attention_step(row(c.q, i), row(c.k, i), row(c.v, i), c.rate, c.W, pool, slots=slots)[:, :, None])
    # 20 drafts, the next 12 tokens among them as a chain at every other node or so
    chain = [0, 1, 3, 4, 6, 8, 9, 11, 13, 14, 16, 18]
    parent = [-1] * 20
    for a, b in zip(chain, chain[1:]):
        parent[b] = a
    draft = [torch.randn(B, H, 20, d, device="cuda").to(torch.bfloat16) for _ in range(3)]
    for x, y in zip(draft, (c.q, c.k, c.v)):
        x[:, :, chain] = y[:, :, 210:222]
    pt = torch.tensor([parent] * B, dtype=torch.int32, device="cuda")
    z.append(gpu_lib.decay_attention_tree(*draft, pt, c.rate, c.W, pool, slots=slots)[:, :, chain])
    path = torch.tensor([chain] * B, dtype=torch.int32, device="cuda")
    gpu_lib.decay_attention_commit(draft[1], draft[2], path, c.rate, c.W, pool, slots=slots)
    # the sequences move to other slots; a fork goes on from the first
    gpu_lib.decay_state_copy(pool, torch.tensor([4, 0, 2, 4], dtype=torch.int32, device="cuda"),
                             torch.tensor([0, 2, 5, 1], dtype=torch.int32, device="cuda"))
    moved = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    rest = [x[:, :, 222:].contiguous() for x in (c.q, c.k, c.v)]
    z.append(gpu_lib.decay_attention_fwd(*rest, c.rate, c.W, state=pool, slots=moved))
    fork = gpu_lib.decay_attention_fwd(*(x[:1].contiguous() for x in rest), c.rate, c.W, state=pool,
                                       slots=torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert torch.equal(fork, z[-1][:1])
    z = torch.cat(z, dim=2)
    for b in range(B):
        for h in range(H):
            want, scale, last, lscale = ref.prompt(*c.head(b, h))
            assert ref.excess(whole[b, h], want, scale, z.dtype) <= 1.0
            assert ref.excess(z[b, h], want, scale, z.dtype) <= 1.0
            # each of the calls behind a state adds its own roundings
            assert ref.excess(pool[int(moved[b]), h], last, lscale, torch.float32, 2 * ref.STATE_DELTA) <= 1.0


def test_views_streams_and_surroundings(gpu_lib):
    """Strided inputs, a stream of one's own, and NaN behind every array and in the workspace."""
    _say("views")
    B, H, n, d, m = 2, 3, 333, 48, 33
    c = Case(B, H, n, d, m)
    want = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W)
    packed = torch.stack([x.transpose(1, 2) for x in (c.q, c.k, c.v)], dim=3)  # [B, n, H, 3, d], as a projection leaves them
    views = [packed[:, :, :, i].transpose(1, 2) for i in range(3)]
    assert torch.equal(gpu_lib.decay_attention_fwd(*views, c.rate, c.W), want)

    def lonely(x):
        flat = torch.full((x.numel() + 4096,), NAN, dtype=x.dtype, device="cuda")
        flat[:x.numel()].copy_(x.reshape(-1))
        return flat[:x.numel()].view(x.shape)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        args = [lonely(x) for x in (c.q, c.k, c.v, c.rate, c.W)]
        ws = torch.full((gpu_lib.decay_attention_bwd_workspace(B, H, n, d, m),), 0xFF, dtype=torch.uint8, device="cuda")
        z = gpu_lib.decay_attention_fwd(*args, workspace=ws)
        ws.fill_(0xFF)
        g = gpu_lib.decay_attention_bwd(*args, lonely(c.dz), workspace=ws)
    stream.synchronize()
    assert torch.equal(z, want)
    for a, b in zip(g, gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz)):
        assert torch.equal(a, b)
    bad = torch.zeros(B, H, m, d + 1, device="cuda").transpose(2, 3)
    with pytest.raises(gpu_lib.KrpeError, match="contiguous"):
        gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=bad)
    with pytest.raises(gpu_lib.KrpeError):
        gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, slots=torch.zeros(B, dtype=torch.int32, device="cuda"))
    with pytest.raises(gpu_lib.KrpeError, match="int32"):
        gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, lens=torch.zeros(B, dtype=torch.int64, device="cuda"))
    with pytest.raises(gpu_lib.KrpeError):
        gpu_lib.decay_attention_fwd(c.q, c.k, c.v.bfloat16(), c.rate, c.W)


def test_two_streams_at_once(gpu_lib):
    """Prompts, tokens and gradients of two streams side by side are those one after the other."""
    _say("two streams")
    cases = [Case(2, 6, 900, 64, 128, "bf16", seed=s) for s in (1, 2)]
    token = lambda c: [x[:, :, 5].contiguous() for x in (c.q, c.k, c.v)]

    def work(c, state):
        return [gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=state),
                gpu_lib.decay_attention_step(*token(c), c.rate, c.W, state),
                *gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz)]

    alone = []
    for c in cases:
        state = c.state.clone()
        alone.append(work(c, state) + [state])
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        states = [c.state.clone() for c in cases]
        torch.cuda.synchronize()
        got = []
        for c, state, stream in zip(cases, states, streams):
            with torch.cuda.stream(stream):
                got.append(work(c, state) + [state])
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_graph(gpu_lib):
    """Tokens, trees, prompts and gradients captured and replayed, the program's own calls between."""
    _say("graph")
    B, H, n, d, m = 2, 2, 150, 32, 48
    c = Case(B, H, n, d, m)
    slots = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    parent = torch.tensor([list(range(-1, 39))] * B, dtype=torch.int32, device="cuda")
    first = c.state.clone()
    tok = [x[:, :, 0].contiguous() for x in (c.q, c.k, c.v)]
    drafts = [x[:, :, :40].contiguous() for x in (c.q, c.k, c.v)]

    def work(state):
        a = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=state, slots=slots)
        b = gpu_lib.decay_attention_step(*tok, c.rate, c.W, state, slots=slots)
        t = gpu_lib.decay_attention_tree(*drafts, parent, c.rate, c.W, state, slots=slots)
        gpu_lib.decay_attention_commit(drafts[1], drafts[2], parent[:, 1:].contiguous(), c.rate, c.W, state, slots=slots)
        gpu_lib.decay_state_copy(state, slots, slots.flip(0))
        return [a, b, t, *gpu_lib.decay_attention_bwd(c.q, c.k, c.v, c.rate, c.W, c.dz)]

    work(c.state)  # (first use outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = work(c.state)
    eager = first.clone()
    c.state.copy_(first)
    for i in range(4):
        want = work(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.state, eager), i
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), i
        c.v.add_(0.25)  # the program's own work between the replays


def test_pool_beyond_32_bits(gpu_lib):
    """Slots whose cells lie past 2^31 floats."""
    H, d, m = 16, 64, 256
    cells = H * (d + 1) * m
    nslots = (1 << 31) // cells + 3
    _say(f"pool of {nslots} slots, {nslots * cells * 4 / 2**30:.1f} GiB")
    c = Case(2, H, 130, d, m, slots=2)
    pool = gpu_lib.decay_state(nslots, H, d, m)
    slots = torch.tensor([nslots - 1, nslots - 2], dtype=torch.int32, device="cuda")
    pool[slots.long()] = c.state
    want = c.state.clone()
    token = [x[:, :, 0].contiguous() for x in (c.q, c.k, c.v)]
    for st, sl in ((pool, slots), (want, None)):
        a = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=st, slots=sl)
        b = gpu_lib.decay_attention_step(*token, c.rate, c.W, st, slots=sl)
        if sl is not None:
            za, zb = a, b
    assert torch.equal(za, a) and torch.equal(zb, b) and torch.equal(pool[slots.long()], want)
    gpu_lib.decay_state_copy(pool, slots, torch.tensor([0, nslots - 3], dtype=torch.int32, device="cuda"))
    assert torch.equal(pool[0], want[0]) and torch.equal(pool[nslots - 3], want[1])


def test_long_prompt(gpu_lib):
    """40000 positions at a rate that remembers thousands, through 313 chunks: sampled rows in 64 bits."""
    _say("n = 40000")
    c = Case(1, 1, 40000, 16, 32, rates=[2.0 ** -12])
    z = gpu_lib.decay_attention_fwd(c.q, c.k, c.v, c.rate, c.W, state=c.state, fresh=True)
    q, k, v, rate, W = c.head(0, 0)
    fq, fk, vh = ref.phi(q, W)[0], ref.phi(k, W)[0], torch.cat([v.double(), torch.ones_like(v[:, :1]).double()], 1)
    for i in (0, 127, 128, 5000, 20001, 39999):
        w = torch.exp(-rate * torch.arange(i, -1, -1, device="cuda", dtype=torch.float64)) * (fk[:i + 1] @ fq[i])
        num, mag = w @ vh[:i + 1], w @ vh[:i + 1].abs()
        want = num[:-1] / num[-1]
        assert ref.excess(z[0, 0, i], want, mag[:-1] / num[-1] + want.abs(), z.dtype) <= 1.0, i
