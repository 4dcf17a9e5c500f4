"""Refusals of the decaying bias's entry points, all on the host and before any HIP call (CPU).

The addresses are never dereferenced: each call below is rejected by validation or is empty."""
import os

import pytest
import torch

from paper_2106_12566_amd import krpe

OK, NULL, SHAPE, UNSUP, DTYPE, WS, ALIAS, HIP, ALIGN = range(9)
BASE = 1 << 40
Q, K, V, W, Z, S, WSP, DQ, DK, DV, DZ = (BASE + i * (1 << 36) for i in range(11))
R, I, J = BASE - 4096, BASE - 8192, BASE - 16384


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(krpe.lib_path()):
        from paper_2106_12566_amd import build
        build.build()
    return krpe.load()


def test_fwd(lib):
    need = lib.krpe_decay_fwd_workspace(2, 3, 300, 8, 16, 0)
    assert need > 0

    def call(q=Q, k=K, v=V, dt=0, r=R, w=W, z=Z, s=S, slots=I, ns=4, lens=J, B=2, H=3, n=300, d=8, m=16, flags=0, ws=WSP,
             wb=need):
        return lib.krpe_decay_fwd(q, k, v, dt, r, w, z, s, slots, ns, lens, B, H, n, d, m, flags, ws, wb, None)

    for name in "qkvrwz":
        assert call(**{name: None}) == NULL
    for name in ("q", "k", "v", "w", "z", "s", "ws"):
        assert call(**{name: {"q": Q, "k": K, "v": V, "w": W, "z": Z, "s": S, "ws": WSP}[name] + 8}) == ALIGN
    assert call(r=R + 2) == ALIGN and call(slots=I + 1) == ALIGN and call(lens=J + 2) == ALIGN
    assert call(B=-1) == SHAPE and call(n=-1) == SHAPE and call(d=0) == SHAPE and call(m=0) == SHAPE
    assert call(d=129) == UNSUP and call(m=1025) == UNSUP and call(n=1 << 30) == UNSUP
    assert call(B=1 << 12, H=1 << 12, n=1) == UNSUP    # more chunks than a grid has groups
    assert call(B=1, H=1, n=(1 << 31) - 1) == UNSUP and call(B=1, H=1, n=(1 << 31) - 129, wb=0) == WS
    assert call(flags=2) == UNSUP and call(flags=8) == UNSUP and call(flags=16) == UNSUP and call(flags=256) == UNSUP
    assert call(flags=4) == SHAPE                      # elu + 1 needs m == d
    assert call(dt=2) == DTYPE
    assert call(ws=None) == WS and call(wb=need - 1) == WS
    assert call(slots=None, ns=1) == SHAPE             # a slot for each sequence
    assert call(ns=-1) == SHAPE
    assert call(s=None) == NULL                        # slots without a pool
    assert call(s=None, slots=None, ns=0, flags=64) == NULL
    assert call(z=Q) == ALIAS and call(s=Q) == ALIAS and call(ws=V) == ALIAS and call(ws=S) == ALIAS and call(z=S) == ALIAS
    assert call(s=I - 256) == ALIAS                    # the pool over its slots
    assert call(B=0) == OK and call(H=0) == OK
    assert call(n=0, s=None, slots=None, ns=0, q=None, k=None, v=None, z=None) == OK
    assert b"" == lib.krpe_last_error()
    assert lib.krpe_decay_fwd_workspace(2, 3, 300, 129, 16, 0) == 0
    assert lib.krpe_decay_fwd_workspace(2, 3, 300, 8, 16, 2) == 0


def test_bwd(lib):
    need = lib.krpe_decay_bwd_workspace(2, 3, 300, 8, 16, 0)
    assert need > lib.krpe_decay_fwd_workspace(2, 3, 300, 8, 16, 0)

    def call(q=Q, k=K, v=V, dt=0, r=R, w=W, dz=DZ, dq=DQ, dk=DK, dv=DV, lens=J, B=2, H=3, n=300, d=8, m=16, flags=0,
             ws=WSP, wb=need):
        return lib.krpe_decay_bwd(q, k, v, dt, r, w, dz, dq, dk, dv, lens, B, H, n, d, m, flags, ws, wb, None)

    for name in ("q", "k", "v", "r", "w", "dz", "dq", "dk", "dv"):
        assert call(**{name: None}) == NULL
    assert call(dq=DQ + 4) == ALIGN and call(lens=J + 3) == ALIGN
    assert call(flags=64) == UNSUP and call(flags=2) == UNSUP and call(d=129) == UNSUP
    assert call(wb=need - 1) == WS and call(ws=None) == WS
    assert call(dq=DK) == ALIAS and call(dv=V) == ALIAS and call(ws=DZ) == ALIAS
    assert call(dt=5) == DTYPE
    assert call(n=0) == OK and call(B=0) == OK


def test_pool_calls(lib):
    def step(q=Q, k=K, v=V, dt=0, r=R, w=W, z=Z, s=S, slots=I, ns=4, B=2, H=3, d=8, m=16, flags=0):
        return lib.krpe_decay_step(q, k, v, dt, r, w, z, s, slots, ns, B, H, d, m, flags, None)

    def tree(q=Q, k=K, v=V, dt=0, r=R, w=W, z=Z, s=S, slots=I, ns=4, B=2, H=3, d=8, m=16, flags=0, par=J, T=7):
        return lib.krpe_decay_tree(q, k, v, dt, par, r, w, z, s, slots, ns, B, H, T, d, m, flags, None)

    def commit(k=K, v=V, dt=0, r=R, w=W, s=S, slots=I, ns=4, B=2, H=3, d=8, m=16, flags=0, path=J, T=7, P=3):
        return lib.krpe_decay_commit(k, v, dt, path, r, w, s, slots, ns, B, H, T, P, d, m, flags, None)

    for call in (step, tree, commit):
        for name in "kvrws":
            assert call(**{name: None}) == NULL, name
        assert call(dt=9) == DTYPE
        assert call(flags=2) == UNSUP and call(flags=64) == UNSUP
        assert call(flags=4) == SHAPE
        assert call(d=129) == UNSUP and call(m=0) == SHAPE and call(B=-2) == SHAPE
        assert call(slots=None, ns=1) == SHAPE
        assert call(s=S + 4) == ALIGN and call(k=K + 2) == ALIGN and call(slots=I + 2) == ALIGN
        assert call(B=0) == OK
    assert step(s=K) == ALIAS and commit(s=K) == ALIAS
    for call in (step, tree):
        assert call(q=None) == NULL and call(z=None) == NULL
        assert call(z=Q) == ALIAS and call(z=S) == ALIAS
    assert tree(T=65) == UNSUP and tree(T=-1) == SHAPE and tree(T=0) == OK and tree(par=None) == NULL
    assert commit(P=-1) == SHAPE and commit(P=0) == OK and commit(path=None) == NULL
    assert commit(P=1 << 30) == UNSUP and commit(T=65537) == UNSUP


def test_state_copy(lib):
    def call(s=S, src=I, dst=J, count=3, ns=4, H=3, d=8, m=16):
        return lib.krpe_decay_state_copy(s, src, dst, count, ns, H, d, m, None)

    assert call(s=None) == NULL and call(src=None) == NULL and call(dst=None) == NULL
    assert call(s=S + 4) == ALIGN and call(src=I + 1) == ALIGN
    assert call(count=-1) == SHAPE and call(ns=-1) == SHAPE
    assert call(count=krpe.COPY_MAX + 1) == UNSUP and call(d=200) == UNSUP
    assert call(H=1 << 24, d=128, m=1024) == UNSUP     # a slot of 2^31 elements
    assert call(s=I - 256) == ALIAS
    assert call(count=0) == OK and call(ns=0) == OK
    assert call(ns=1 << 20, H=16, count=0) == OK


def test_binding_refuses(lib):
    x, r, W = torch.zeros(1, 2, 8, 4), torch.zeros(2), torch.zeros(2, 4, 4)
    for f in (lambda: krpe.decay_attention_fwd(x, x, x, r, W),
              lambda: krpe.decay_attention_bwd(x, x, x, r, W, x),
              lambda: krpe.decay_attention_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], r, W, torch.zeros(1, 2, 5, 4)),
              lambda: krpe.decay_state_copy(torch.zeros(1, 2, 5, 4), torch.zeros(1, dtype=torch.int32),
                                            torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(krpe.KrpeError):
            f()
    with pytest.raises(krpe.KrpeError, match="features"):
        krpe.decay_attention_fwd(x, x, x, r, W, features="trf")
