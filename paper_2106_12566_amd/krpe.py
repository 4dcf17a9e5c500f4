"""Python binding of libkrpe.so: argument marshalling only.

Every function takes torch tensors that live on a GPU, checks that their shapes
agree with each other, allocates the output (and workspace) with torch, and
calls the C entry point of the same name on the current torch stream.  All
arithmetic happens in the library's HIP kernels; there is no CPU path: calling
any of these without the built library or without a GPU raises.

Names and layouts follow the C header ``include/krpe.h``:
  q, k, v : [B, H, n, d]  float32 or bfloat16      W : [H, m, d] float32
  b       : [H, 2n-1] float32, b[h, s] = b_{s-(n-1)} (Algorithm 1's ordering)

The decay_* functions are Eq. (10) with the bias b_t = rate t (t <= 0, -inf after)
over a state of constant size: prompts, their gradients, single tokens, trees of
drafted tokens, and copies within a pool of states.  Their outputs have q's type.
  rate    : [H] float32         state : [slots, H, d + 1, M] float32, changed in place
  slots   : [B] int32, the pool's row of each sequence (None: row b; -1: none)
"""
from __future__ import annotations

import ctypes
import os

import torch

__all__ = ["KrpeError", "load", "lib_path", "feature_map", "toeplitz_conv", "toeplitz_conv_noalloc",
           "attention_fwd", "attention_bwd",
           "attention_fwd_route",
           "attention_fwd_workspace", "attention_bwd_workspace", "toeplitz_conv_workspace",
           "attention_fwd_fixed_rows", "decay_state", "decay_attention_fwd", "decay_attention_bwd",
           "decay_attention_step", "decay_attention_tree", "decay_attention_commit", "decay_state_copy",
           "decay_attention_fwd_workspace", "decay_attention_bwd_workspace", "DTYPES"]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libkrpe.so")
_lib = None

DTYPES = {torch.float32: 0, torch.bfloat16: 1}
STAGE_EVENTS = 5
NPRF = 1  # option bit: l2-normalise the rows of q and k (x) before the feature map
FEAT_TRF = 2  # option bit: trigonometric random features (2m signed features)
FEAT_ELU = 4  # option bit: elu(x) + 1 (d features, W not read)
FEATURES = {"prf": 0, "trf": FEAT_TRF, "elu": FEAT_ELU}
ROUTE_DIRECT = 8  # option bit: evaluate Eq. (10) directly (quadratic, MFMA)
ROUTE_FFT = 16  # option bit: the FFT route of Section 3.2
ROUTES = {"auto": 0, "direct": ROUTE_DIRECT, "fft": ROUTE_FFT}
HINT_CAUSAL = 32  # option bit: b is -inf for every t > 0 (read by the route choice only)
STATE_FRESH = 64  # option bit of decay_attention_fwd: sequences start from zeros
ZERO_TAIL = 128  # option bit of decay_attention_fwd and _bwd: rows behind lens are zeros
TREE_MAX, COPY_MAX = 64, 256  # nodes of a tree, moves of a copy


class KrpeError(RuntimeError):
    """A non-OK status returned by the library, or a missing library/GPU."""


def lib_path() -> str:
    """The library this binding loads: $KRPE_LIBRARY if set (e.g. a build with host-side
    sanitizers), else libkrpe.so next to this file."""
    return os.environ.get("KRPE_LIBRARY") or _LIB_PATH


def load(path: str | None = None) -> ctypes.CDLL:
    """Load the library (once).  Raises KrpeError if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or lib_path()
    if not os.path.exists(p):
        raise KrpeError(f"{p} is missing: build it with `python -m paper_2106_12566_amd.build`")
    lib = ctypes.CDLL(p)
    vp, i, sz, fp = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p
    lib.krpe_abi_version.restype = i
    lib.krpe_abi_version.argtypes = []
    lib.krpe_status_str.restype = ctypes.c_char_p
    lib.krpe_status_str.argtypes = [i]
    lib.krpe_last_error.restype = ctypes.c_char_p
    lib.krpe_last_error.argtypes = []
    lib.krpe_feature_map.restype = i
    lib.krpe_feature_map.argtypes = [vp, i, fp, fp, i, i, i, i, i, vp]
    lib.krpe_feature_map_ex.restype = i
    lib.krpe_feature_map_ex.argtypes = [vp, i, fp, fp, i, i, i, i, i, ctypes.c_uint, vp]
    lib.krpe_toeplitz_conv_workspace.restype = sz
    lib.krpe_toeplitz_conv_workspace.argtypes = [i, i, i, i]
    lib.krpe_toeplitz_conv.restype = i
    lib.krpe_toeplitz_conv.argtypes = [fp, fp, fp, i, i, i, i, vp, sz, vp]
    lib.krpe_toeplitz_conv_noalloc.restype = i
    lib.krpe_toeplitz_conv_noalloc.argtypes = [fp, fp, fp, i, i, i, i, vp]
    lib.krpe_attention_fwd_workspace.restype = sz
    lib.krpe_attention_fwd_workspace.argtypes = [i, i, i, i, i]
    lib.krpe_attention_fwd_workspace_ex.restype = sz
    lib.krpe_attention_fwd_workspace_ex.argtypes = [i, i, i, i, i, ctypes.c_uint]
    lib.krpe_attention_fwd.restype = i
    lib.krpe_attention_fwd.argtypes = [vp, vp, vp, i, fp, fp, fp, i, i, i, i, i, vp, sz, vp]
    lib.krpe_attention_fwd_ex.restype = i
    lib.krpe_attention_fwd_ex.argtypes = [vp, vp, vp, i, fp, fp, fp, i, i, i, i, i, ctypes.c_uint, vp, sz, vp]
    lib.krpe_attention_fwd_profiled.restype = i
    lib.krpe_attention_fwd_profiled.argtypes = [vp, vp, vp, i, fp, fp, fp, i, i, i, i, i, ctypes.c_uint, vp, sz,
                                                vp, ctypes.POINTER(ctypes.c_void_p)]
    lib.krpe_attention_fwd_route.restype = i
    lib.krpe_attention_fwd_route.argtypes = [i, i, i, i, i, ctypes.c_uint]
    lib.krpe_attention_bwd_workspace.restype = sz
    lib.krpe_attention_bwd_workspace.argtypes = [i, i, i, i, i, ctypes.c_uint]
    lib.krpe_attention_bwd.restype = i
    lib.krpe_attention_bwd.argtypes = [vp, vp, vp, i, fp, fp, fp, fp, fp, fp, fp, i, i, i, i, i, ctypes.c_uint, vp,
                                       sz, vp]
    lib.krpe_attention_fwd_stats.restype = i
    lib.krpe_attention_fwd_stats.argtypes = [vp, sz, i, i, i, i, i, ctypes.POINTER(ctypes.c_uint), vp]
    u = ctypes.c_uint
    for name, res, args in (
            ("krpe_decay_fwd_workspace", sz, [i, i, i, i, i, u]),
            ("krpe_decay_fwd", i, [vp, vp, vp, i, vp, vp, vp, vp, vp, i, vp, i, i, i, i, i, u, vp, sz, vp]),
            ("krpe_decay_bwd_workspace", sz, [i, i, i, i, i, u]),
            ("krpe_decay_bwd", i, [vp, vp, vp, i, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, u, vp, sz, vp]),
            ("krpe_decay_step", i, [vp, vp, vp, i, vp, vp, vp, vp, vp, i, i, i, i, i, u, vp]),
            ("krpe_decay_tree", i, [vp, vp, vp, i, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, u, vp]),
            ("krpe_decay_commit", i, [vp, vp, i, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, u, vp]),
            ("krpe_decay_state_copy", i, [vp, vp, vp, i, i, i, i, i, vp])):
        getattr(lib, name).restype = res
        getattr(lib, name).argtypes = args
    if path is None:
        _lib = lib
    return lib


def _check(status: int, what: str) -> None:
    if status != 0:
        lib = load()
        msg = lib.krpe_status_str(status).decode()
        detail = lib.krpe_last_error().decode()
        raise KrpeError(f"{what}: {msg} ({detail})")


def _gpu(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise KrpeError(f"{name} must be on a GPU (libkrpe has no CPU path)")
    return t.contiguous()


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _stream(device: torch.device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _dtype_code(t: torch.Tensor, name: str) -> int:
    if t.dtype not in DTYPES:
        raise KrpeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return DTYPES[t.dtype]


def _flags(nprf: bool, features: str, route: str = "auto", causal: bool = False) -> int:
    if features not in FEATURES:
        raise KrpeError(f"features must be one of {sorted(FEATURES)}, got {features!r}")
    if route not in ROUTES:
        raise KrpeError(f"route must be one of {sorted(ROUTES)}, got {route!r}")
    return (NPRF if nprf else 0) | FEATURES[features] | ROUTES[route] | (HINT_CAUSAL if causal else 0)


def _proj(W: torch.Tensor | None, H: int, d: int, features: str) -> tuple[torch.Tensor | None, int]:
    """W (None allowed for elu + 1) and the m the C call takes."""
    if features == "elu":
        return None, d
    if W is None:
        raise KrpeError("W is required for the prf and trf feature maps")
    W = _gpu(W, "W")
    if W.dim() != 3 or W.shape[0] != H or W.shape[2] != d or W.dtype != torch.float32:
        raise KrpeError("W must be float32 [H, m, d]")
    return W, W.shape[1]


def feature_map(x: torch.Tensor, W: torch.Tensor | None, nprf: bool = False, features: str = "prf") -> torch.Tensor:
    """phi of x [B,H,n,d] -> [B,H,n,M] fp32 with the projections W [H,m,d].

    features: "prf" (Eq. (5), M = m), "trf" (sin then cos features, M = 2m),
    "elu" (elu(x) + 1, M = d, W unused).  nprf: phi of x / ||x|| (Algorithm 1)."""
    lib = load()
    x = _gpu(x, "x")
    if x.dim() != 4:
        raise KrpeError("x must be [B,H,n,d]")
    B, H, n, d = x.shape
    flags = _flags(nprf, features)
    W, m = _proj(W, H, d, features)
    M = 2 * m if features == "trf" else m
    phi = torch.empty((B, H, n, M), dtype=torch.float32, device=x.device)
    st = lib.krpe_feature_map_ex(_ptr(x), _dtype_code(x, "x"), _ptr(W), _ptr(phi), B, H, n, d, m, flags,
                                 _stream(x.device))
    _check(st, "krpe_feature_map_ex")
    return phi


def toeplitz_conv_workspace(B: int, H: int, C: int, n: int) -> int:
    return int(load().krpe_toeplitz_conv_workspace(B, H, C, n))


def toeplitz_conv(b: torch.Tensor, a: torch.Tensor) -> torch.Tensor:
    """y[beta,h,c,i] = sum_j exp(b[h, j-i+n-1]) a[beta,h,c,j]; b [H,2n-1], a [B,H,C,n] fp32."""
    lib = load()
    b = _gpu(b, "b")
    a = _gpu(a, "a")
    if a.dim() != 4 or b.dim() != 2:
        raise KrpeError("a must be [B,H,C,n] and b [H,2n-1]")
    B, H, C, n = a.shape
    if b.shape != (H, 2 * n - 1) or b.dtype != torch.float32 or a.dtype != torch.float32:
        raise KrpeError("b must be float32 [H, 2n-1] and a float32 [B,H,C,n]")
    y = torch.empty_like(a)
    wsb = lib.krpe_toeplitz_conv_workspace(B, H, C, n)
    ws = torch.empty(max(int(wsb), 1), dtype=torch.uint8, device=a.device)
    st = lib.krpe_toeplitz_conv(_ptr(b), _ptr(a), _ptr(y), B, H, C, n, ws.data_ptr(), ws.numel(),
                                _stream(a.device))
    _check(st, "krpe_toeplitz_conv")
    return y


def toeplitz_conv_noalloc(b: torch.Tensor, a: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """toeplitz_conv through krpe_toeplitz_conv_noalloc: no workspace, the library's static scratch instead.

    Only the output is allocated here (or passed as ``out``); the call itself allocates nothing.  Calls
    that overlap on one GPU share that scratch and race.
    """
    lib = load()
    b = _gpu(b, "b")
    a = _gpu(a, "a")
    if a.dim() != 4 or b.dim() != 2:
        raise KrpeError("a must be [B,H,C,n] and b [H,2n-1]")
    B, H, C, n = a.shape
    if b.shape != (H, 2 * n - 1) or b.dtype != torch.float32 or a.dtype != torch.float32:
        raise KrpeError("b must be float32 [H, 2n-1] and a float32 [B,H,C,n]")
    if out is None:
        out = torch.empty_like(a)
    elif out.shape != a.shape or out.dtype != torch.float32 or not out.is_contiguous():
        raise KrpeError("out must be a contiguous float32 tensor shaped like a")
    st = lib.krpe_toeplitz_conv_noalloc(_ptr(b), _ptr(a), _ptr(out), B, H, C, n, _stream(a.device))
    _check(st, "krpe_toeplitz_conv_noalloc")
    return out


def attention_fwd_workspace(B: int, H: int, n: int, d: int, m: int, nprf: bool = False,
                            features: str = "prf", route: str = "auto", causal: bool = False) -> int:
    return int(load().krpe_attention_fwd_workspace_ex(B, H, n, d, m, _flags(nprf, features, route, causal)))


def attention_fwd_fixed_rows(workspace: torch.Tensor, B: int, H: int, n: int, d: int, m: int) -> int:
    """Rows of the last attention_fwd call on `workspace` that were evaluated exactly (waits for the stream)."""
    lib = load()
    out = ctypes.c_uint(0)
    st = lib.krpe_attention_fwd_stats(workspace.data_ptr(), workspace.numel(), B, H, n, d, m,
                                      ctypes.byref(out), _stream(workspace.device))
    _check(st, "krpe_attention_fwd_stats")
    return int(out.value)


def attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, b: torch.Tensor, W: torch.Tensor | None,
                  out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                  events=None, nprf: bool = False, features: str = "prf", route: str = "auto",
                  causal: bool = False) -> torch.Tensor:
    """Eq. (10): z [B,H,n,d] fp32 from q, k, v [B,H,n,d] (fp32 or bf16), b [H,2n-1], W [H,m,d].

    ``nprf``: normalise the rows of q and k first (Algorithm 1's NPRF attention).
    ``features``: "prf" (Eq. (5)), "trf" (trigonometric, 2m features) or "elu"
    (elu + 1, W unused and may be None).
    ``route``: "fft" (Section 3.2), "direct" (Eq. (10) evaluated directly on
    MFMA, faster for short sequences) or "auto" (by sequence length).
    ``causal``: the caller states that b is -inf for every t > 0; only the
    "auto" route choice reads it (the direct route then costs half the pairs).

    ``out`` and ``workspace`` may be passed to reuse allocations (a uint8 tensor
    of at least attention_fwd_workspace() bytes).  ``events``: optional list of
    5 raw hipEvent_t handles recorded around the stages (see the C header).
    """
    lib = load()
    q, k, v = _gpu(q, "q"), _gpu(k, "k"), _gpu(v, "v")
    b = _gpu(b, "b")
    if q.dim() != 4:
        raise KrpeError("q must be [B,H,n,d]")
    B, H, n, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise KrpeError("q, k, v must share shape and dtype")
    flags = _flags(nprf, features, route, causal)
    W, m = _proj(W, H, d, features)
    if b.shape != (H, 2 * n - 1) or b.dtype != torch.float32:
        raise KrpeError("b must be float32 [H, 2n-1]")
    if out is None:
        out = torch.empty((B, H, n, d), dtype=torch.float32, device=q.device)
    elif out.shape != (B, H, n, d) or out.dtype != torch.float32 or not out.is_contiguous():
        raise KrpeError("out must be a contiguous float32 [B,H,n,d] tensor")
    wsb = int(lib.krpe_attention_fwd_workspace_ex(B, H, n, d, m, flags))
    if workspace is None:
        workspace = torch.empty(max(wsb, 1), dtype=torch.uint8, device=q.device)
    dt = _dtype_code(q, "q")
    if workspace.numel() < wsb:
        raise KrpeError(f"workspace must hold at least {wsb} bytes")
    args = (_ptr(q), _ptr(k), _ptr(v), dt, _ptr(b), _ptr(W), _ptr(out), B, H, n, d, m, flags,
            workspace.data_ptr(), workspace.numel(), _stream(q.device))
    if events is None:
        st = lib.krpe_attention_fwd_ex(*args)
    else:
        if len(events) != STAGE_EVENTS:
            raise KrpeError(f"events must hold {STAGE_EVENTS} hipEvent_t handles")
        arr = (ctypes.c_void_p * STAGE_EVENTS)(*events)
        st = lib.krpe_attention_fwd_profiled(*args, arr)
    _check(st, "krpe_attention_fwd")
    return out


def attention_fwd_route(B: int, H: int, n: int, d: int, m: int, nprf: bool = False, features: str = "prf",
                        route: str = "auto", causal: bool = False) -> str:
    """The route ("direct" or "fft") attention_fwd takes for these sizes and options."""
    r = int(load().krpe_attention_fwd_route(B, H, n, d, m, _flags(nprf, features, route, causal)))
    if r == 0:
        raise KrpeError("invalid sizes or options")
    return "direct" if r == ROUTE_DIRECT else "fft"


def attention_bwd_workspace(B: int, H: int, n: int, d: int, m: int, nprf: bool = False) -> int:
    return int(load().krpe_attention_bwd_workspace(B, H, n, d, m, NPRF if nprf else 0))



def attention_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, b: torch.Tensor, W: torch.Tensor,
                  dz: torch.Tensor, workspace: torch.Tensor | None = None, nprf: bool = False,
                  with_db: bool = False, route: str = "auto", causal: bool = False) -> tuple:
    """Gradients (dq, dk, dv) [B,H,n,d] fp32 of sum(dz * z), z = attention_fwd(q, k, v, b, W, nprf=nprf)
    with PRF features and W fixed (the C header states the formulas); with_db adds db [H, 2n-1]."""
    lib = load()
    q, k, v = _gpu(q, "q"), _gpu(k, "k"), _gpu(v, "v")
    b, W, dz = _gpu(b, "b"), _gpu(W, "W"), _gpu(dz, "dz")
    if q.dim() != 4:
        raise KrpeError("q must be [B,H,n,d]")
    B, H, n, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise KrpeError("q, k, v must share shape and dtype")
    if dz.shape != q.shape or dz.dtype != torch.float32:
        raise KrpeError("dz must be float32 [B,H,n,d]")
    if W.dim() != 3 or W.shape[0] != H or W.shape[2] != d or W.dtype != torch.float32:
        raise KrpeError("W must be float32 [H, m, d]")
    if b.shape != (H, 2 * n - 1) or b.dtype != torch.float32:
        raise KrpeError("b must be float32 [H, 2n-1]")
    m = W.shape[1]
    flags = _flags(nprf, "prf", route, causal)
    if workspace is None:
        # (one given is checked by the call: sized for the transforms, it has them)
        wsb = int(lib.krpe_attention_bwd_workspace(B, H, n, d, m, flags))
        workspace = torch.empty(max(wsb, 1), dtype=torch.uint8, device=q.device)
    dq = torch.empty((B, H, n, d), dtype=torch.float32, device=q.device)
    dk = torch.empty_like(dq)
    dv = torch.empty_like(dq)
    db = torch.empty((H, 2 * n - 1), dtype=torch.float32, device=q.device) if with_db else None
    st = lib.krpe_attention_bwd(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q, "q"), _ptr(b), _ptr(W), _ptr(dz), _ptr(dq),
                                _ptr(dk), _ptr(dv), _ptr(db), B, H, n, d, m, flags, workspace.data_ptr(),
                                workspace.numel(), _stream(q.device))
    _check(st, "krpe_attention_bwd")
    return (dq, dk, dv, db) if with_db else (dq, dk, dv)


# ---- attention with a decaying bias -------------------------------------------------

def _decay_flags(nprf: bool, features: str) -> int:
    if features not in ("prf", "elu"):
        raise KrpeError(f"features must be one of ['elu', 'prf'] here, got {features!r}")
    return (NPRF if nprf else 0) | FEATURES[features]


def _enqueue(name: str, device: torch.device, *args) -> None:
    """The C call `name` on the current stream of `device`, with that device the current one."""
    index = device.index
    fn = getattr(_lib or load(), name)
    if torch.cuda.current_device() == index:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(device):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != 0:
        _check(st, name)


def _decay_inputs(names: tuple, tensors: tuple, rate: torch.Tensor, W: torch.Tensor | None, features: str, dims: int):
    """Checked, contiguous inputs of one shape [B, H, (rows,) d] and type; rate, W, m and that shape.

    (A token's call is a few microseconds: every attribute is read once.)"""
    out = []
    shape = dtype = device = None
    for name, t in zip(names, tensors):
        t = _gpu(t, name)
        if shape is None:
            shape, dtype, device = t.shape, t.dtype, t.device
            if len(shape) != dims:
                raise KrpeError(f"{name} must have {dims} dimensions")
            if dtype not in DTYPES:
                raise KrpeError(f"{name} must be float32 or bfloat16, got {dtype}")
        elif t.shape != shape or t.dtype != dtype:
            raise KrpeError(f"{', '.join(names)} must share shape and dtype")
        elif t.device != device:
            _elsewhere(t, device)
        out.append(t)
    H, d = shape[1], shape[-1]
    rate = _gpu(rate, "rate")
    if rate.shape != (H,) or rate.dtype != torch.float32:
        raise KrpeError("rate must be float32 [H]")
    W, m = _proj(W, H, d, features)
    if rate.device != device or (W is not None and W.device != device):
        _elsewhere(rate if rate.device != device else W, device)
    return out, rate, W, m, shape, device


def _elsewhere(t: torch.Tensor, device: torch.device) -> None:
    raise KrpeError(f"all tensors must be on one GPU: {t.device} and {device}")


def _ints(t: torch.Tensor | None, name: str, shape: tuple, device: torch.device) -> torch.Tensor | None:
    if t is None:
        return None
    t = _gpu(t, name)
    if t.dtype != torch.int32 or t.shape != shape:
        raise KrpeError(f"{name} must be int32 {list(shape)}")
    if t.device != device:
        _elsewhere(t, device)
    return t


def _pool(state: torch.Tensor, H: int, d: int, m: int, device: torch.device) -> int:
    """The number of slots of a pool, which has to be contiguous (it is changed in place)."""
    if not isinstance(state, torch.Tensor) or not state.is_cuda:
        raise KrpeError("state must be on a GPU (libkrpe has no CPU path)")
    shape = state.shape
    if len(shape) != 4 or shape != (shape[0], H, d + 1, m) or state.dtype != torch.float32:
        raise KrpeError(f"state must be float32 [slots, {H}, {d + 1}, {m}]")
    if not state.is_contiguous():
        raise KrpeError("state must be contiguous")
    if state.device != device:
        _elsewhere(state, device)
    return shape[0]


def _at(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _like(out: torch.Tensor | None, x: torch.Tensor) -> torch.Tensor:
    """The output beside input x: the one given, checked, or a new one."""
    if out is None:
        return torch.empty_like(x)
    if not isinstance(out, torch.Tensor) or out.shape != x.shape or out.dtype != x.dtype or not out.is_contiguous():
        raise KrpeError("out must be a contiguous tensor of q's shape and dtype")
    if out.device != x.device:
        _elsewhere(out, x.device)
    return out


def _space(workspace: torch.Tensor | None, need: int, device: torch.device) -> torch.Tensor:
    if workspace is None:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or workspace.numel() < need or not workspace.is_contiguous():
        raise KrpeError(f"workspace must hold at least {need} bytes (uint8)")
    if workspace.device != device:
        _elsewhere(workspace, device)
    return workspace


def decay_state(slots: int, H: int, d: int, m: int, device="cuda") -> torch.Tensor:
    """A pool of empty states [slots, H, d + 1, m] (m: the features; d with features="elu")."""
    return torch.zeros((slots, H, d + 1, m), dtype=torch.float32, device=device)


def decay_attention_fwd_workspace(B: int, H: int, n: int, d: int, m: int) -> int:
    return int(load().krpe_decay_fwd_workspace(B, H, n, d, m, 0))


def decay_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rate: torch.Tensor, W: torch.Tensor | None,
                        state: torch.Tensor | None = None, slots: torch.Tensor | None = None,
                        lens: torch.Tensor | None = None, fresh: bool = False, out: torch.Tensor | None = None,
                        workspace: torch.Tensor | None = None, nprf: bool = False,
                        features: str = "prf") -> torch.Tensor:
    """Eq. (10) with b_t = rate t (t <= 0): z [B,H,n,d] in q's type, O(n).

    ``state``: the pool whose rows are the states before the sequences (zeros with
    ``fresh``, whatever the rows hold) and, after the call, those behind them.
    ``lens``: int32 [B], the positions of each sequence; rows of q, k, v behind them are
    not read and rows of ``out`` stay as they were (zeros without ``out``)."""
    flags = _decay_flags(nprf, features)
    (q, k, v), rate, W, m, shape, dev = _decay_inputs(("q", "k", "v"), (q, k, v), rate, W, features, 4)
    B, H, n, d = shape
    nslots = 0
    if state is not None:
        nslots = _pool(state, H, d, m, dev)
        flags |= STATE_FRESH if fresh else 0
    elif slots is not None or fresh:
        raise KrpeError("slots and fresh need a state")
    slots, lens = _ints(slots, "slots", (B,), dev), _ints(lens, "lens", (B,), dev)
    flags |= ZERO_TAIL if out is None and lens is not None else 0
    z = _like(out, q)
    ws = _space(workspace, int(load().krpe_decay_fwd_workspace(B, H, n, d, m, flags)), dev)
    _enqueue("krpe_decay_fwd", dev, _at(q), _at(k), _at(v), DTYPES[q.dtype], _at(rate), _at(W), _at(z),
             _at(state), _at(slots), nslots, _at(lens), B, H, n, d, m, flags, ws.data_ptr(), ws.numel())
    return z


def decay_attention_bwd_workspace(B: int, H: int, n: int, d: int, m: int) -> int:
    return int(load().krpe_decay_bwd_workspace(B, H, n, d, m, 0))


def decay_attention_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rate: torch.Tensor, W: torch.Tensor | None,
                        dz: torch.Tensor, lens: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                        nprf: bool = False, features: str = "prf") -> tuple:
    """Gradients (dq, dk, dv) [B,H,n,d] in q's type of sum(dz * z), z = decay_attention_fwd(q, k, v, rate, W)
    from empty states, rate and W fixed.  Rows behind ``lens`` are zero."""
    flags = _decay_flags(nprf, features)
    (q, k, v, dz), rate, W, m, shape, dev = _decay_inputs(("q", "k", "v", "dz"), (q, k, v, dz), rate, W, features, 4)
    B, H, n, d = shape
    lens = _ints(lens, "lens", (B,), dev)
    flags |= ZERO_TAIL if lens is not None else 0
    dq, dk, dv = (torch.empty_like(q) for _ in range(3))
    ws = _space(workspace, int(load().krpe_decay_bwd_workspace(B, H, n, d, m, flags)), dev)
    _enqueue("krpe_decay_bwd", dev, _at(q), _at(k), _at(v), DTYPES[q.dtype], _at(rate), _at(W), _at(dz),
             _at(dq), _at(dk), _at(dv), _at(lens), B, H, n, d, m, flags, ws.data_ptr(), ws.numel())
    return dq, dk, dv


def decay_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rate: torch.Tensor, W: torch.Tensor | None,
                         state: torch.Tensor, slots: torch.Tensor | None = None, out: torch.Tensor | None = None,
                         nprf: bool = False, features: str = "prf") -> torch.Tensor:
    """One token of every sequence: its k, v [B,H,d] go into the states, z [B,H,d] is its output.
    Allocates nothing with ``out`` (a captured graph may replay it)."""
    flags = _decay_flags(nprf, features)
    (q, k, v), rate, W, m, shape, dev = _decay_inputs(("q", "k", "v"), (q, k, v), rate, W, features, 3)
    B, H, d = shape
    nslots = _pool(state, H, d, m, dev)
    slots = _ints(slots, "slots", (B,), dev)
    z = _like(out, q)
    _enqueue("krpe_decay_step", dev, _at(q), _at(k), _at(v), DTYPES[q.dtype], _at(rate), _at(W), _at(z),
             _at(state), _at(slots), nslots, B, H, d, m, flags)
    return z


def decay_attention_tree(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, parent: torch.Tensor, rate: torch.Tensor,
                         W: torch.Tensor | None, state: torch.Tensor, slots: torch.Tensor | None = None,
                         out: torch.Tensor | None = None, nprf: bool = False, features: str = "prf") -> torch.Tensor:
    """Trees of drafted tokens q, k, v [B,H,T,d] (T <= 64) behind every sequence: z of each node from
    the state, its ancestors and itself.  ``parent``: int32 [B,T], parent[b,t] < t, -1 for the children
    of the sequence's last token; a node with any other parent, and what is below it, gets zeros.
    The states stay as they are: decay_attention_commit takes the accepted nodes in."""
    flags = _decay_flags(nprf, features)
    (q, k, v), rate, W, m, shape, dev = _decay_inputs(("q", "k", "v"), (q, k, v), rate, W, features, 4)
    B, H, T, d = shape
    nslots = _pool(state, H, d, m, dev)
    if parent is None:
        raise KrpeError("parent must be int32 [B, T]")
    parent, slots = _ints(parent, "parent", (B, T), dev), _ints(slots, "slots", (B,), dev)
    z = _like(out, q)
    _enqueue("krpe_decay_tree", dev, _at(q), _at(k), _at(v), DTYPES[q.dtype], _at(parent), _at(rate), _at(W),
             _at(z), _at(state), _at(slots), nslots, B, H, T, d, m, flags)
    return z


def decay_attention_commit(k: torch.Tensor, v: torch.Tensor, path: torch.Tensor, rate: torch.Tensor,
                           W: torch.Tensor | None, state: torch.Tensor, slots: torch.Tensor | None = None,
                           nprf: bool = False, features: str = "prf") -> None:
    """Takes tokens path[b, 0], path[b, 1], .. of k, v [B,H,T,d] into the states, up to the first entry
    outside [0, T).  ``path``: int32 [B,P]."""
    flags = _decay_flags(nprf, features)
    (k, v), rate, W, m, shape, dev = _decay_inputs(("k", "v"), (k, v), rate, W, features, 4)
    B, H, T, d = shape
    nslots = _pool(state, H, d, m, dev)
    if not isinstance(path, torch.Tensor) or path.dim() != 2:
        raise KrpeError("path must be int32 [B, P]")
    path = _ints(path, "path", (B, path.shape[1]), dev)
    slots = _ints(slots, "slots", (B,), dev)
    _enqueue("krpe_decay_commit", dev, _at(k), _at(v), DTYPES[k.dtype], _at(path), _at(rate), _at(W),
             _at(state), _at(slots), nslots, B, H, T, path.shape[1], d, m, flags)


def decay_state_copy(state: torch.Tensor, src: torch.Tensor, dst: torch.Tensor) -> None:
    """state[dst[i]] = state[src[i]] for all i at once (src -1: cleared): forks, reorders, compacts and
    frees the states of a pool.  ``src``, ``dst``: int32 [count], count <= 256.  Of moves to one slot the
    last holds; moves with a slot outside the pool are left out."""
    if not isinstance(state, torch.Tensor) or state.dim() != 4:
        raise KrpeError("state must be float32 [slots, H, d + 1, m]")
    nslots, H, rows, m = state.shape
    _pool(state, H, rows - 1, m, state.device)
    if not isinstance(src, torch.Tensor) or src.dim() != 1:
        raise KrpeError("src must be int32 [count]")
    src, dst = _ints(src, "src", (src.shape[0],), state.device), _ints(dst, "dst", (src.shape[0],), state.device)
    if dst is None:
        raise KrpeError("dst must be int32 [count]")
    _enqueue("krpe_decay_state_copy", state.device, _at(state), _at(src), _at(dst), src.shape[0], nslots, H, rows - 1,
             m)
