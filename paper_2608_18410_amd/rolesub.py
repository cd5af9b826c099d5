"""ctypes binding of librolesub.

Argument marshalling only: every step of the hot path runs in the library's
HIP kernels. torch tensors supply device memory (data_ptr) and the current
HIP stream. Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librolesub.so")

F32, BF16 = 0, 1
VIS, LANG, PROP, ACT = 0, 1, 2, 3
TOPK, THRESHOLD = 0, 1
MLP2, ADDITIVE = 0, 1

EXPORTS = (
    "rolesub_status_str", "rolesub_last_error", "rolesub_version",
    "rolesub_rotate_values", "rolesub_route_workspace_size", "rolesub_route",
    "rolesub_pack_kv", "rolesub_rotate_pack", "rolesub_attend_workspace_size", "rolesub_attend",
    "rolesub_attend_causal", "rolesub_retain_tokens", "rolesub_gather_tokens",
    "rolesub_allocate_groups", "rolesub_route_allocate_workspace_size", "rolesub_route_allocate",
    "rolesub_full_workspace_size", "rolesub_full_transpose", "rolesub_full_rotate_pack", "rolesub_full_values",
    "rolesub_attend_values", "rolesub_route_noalloc",
    "rolesub_rotary", "rolesub_cache_append", "rolesub_attend_paged_workspace_size", "rolesub_attend_paged",
    "rolesub_evict_workspace_size", "rolesub_evict_tokens", "rolesub_cache_compact",
    "rolesub_norm_rotary", "rolesub_append_rotary", "rolesub_tree_masks", "rolesub_attend_tree_workspace_size",
    "rolesub_attend_tree", "rolesub_cache_accept", "rolesub_page_bounds", "rolesub_select_pages_workspace_size",
    "rolesub_select_pages", "rolesub_attend_selected_workspace_size", "rolesub_attend_selected",
)
ROUTE_NOALLOC_MAX_BYTES = 8 << 20


class RolesubError(RuntimeError):
    def __init__(self, fn: str, status: int, message: str):
        super().__init__(f"{fn} -> {status_name(status)}: {message}")
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "H", "dh", "G", "d")]


class Budget(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("k_by_type", ctypes.c_int32 * 4), ("tau", ctypes.c_float),
                ("kmin", ctypes.c_int32), ("kmax", ctypes.c_int32)]


class RouterDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("C", ctypes.c_int32), ("d_e", ctypes.c_int32),
                ("Hr", ctypes.c_int32), ("alpha_role", ctypes.c_float), ("alpha_lang", ctypes.c_float)] + \
               [(n, ctypes.c_void_p) for n in ("W_r", "b_r", "E", "W1", "b1", "W2", "b2",
                                               "W_tok", "b_tok", "W_role", "W_lang", "b_lang")]


class PagesDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page", "vcap", "H", "dh", "G")] + \
               [(n, ctypes.c_void_p) for n in ("K", "V", "mask", "slot")]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load librolesub.so (built in-tree by paper_2608_18410_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"librolesub is not built ({path} is missing); "
                          "run `python -m paper_2608_18410_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.rolesub_status_str.argtypes = [ctypes.c_int]
    lib.rolesub_status_str.restype = ctypes.c_char_p
    lib.rolesub_last_error.argtypes = []
    lib.rolesub_last_error.restype = ctypes.c_char_p
    lib.rolesub_version.argtypes = []
    lib.rolesub_version.restype = I32
    lib.rolesub_rotate_values.argtypes = [P, ctypes.c_int, P, P, P, P]
    lib.rolesub_route_workspace_size.argtypes = [P, P]
    lib.rolesub_route_workspace_size.restype = SZ
    lib.rolesub_route.argtypes = [P, ctypes.c_int, P, P, P, P, P, P, P, P, P, P, SZ, P]
    lib.rolesub_route_noalloc.argtypes = [P, ctypes.c_int, P, P, P, P, P, P, P, P, P, P]
    lib.rolesub_pack_kv.argtypes = [P, ctypes.c_int, P, P, P, P, P, P, I64, P]
    lib.rolesub_rotate_pack.argtypes = [P, ctypes.c_int, P, P, P, P, P, P, P, I64, P]
    lib.rolesub_attend_workspace_size.argtypes = [P, I32]
    lib.rolesub_attend_workspace_size.restype = SZ
    lib.rolesub_attend.argtypes = [P, ctypes.c_int, I32, P, P, P, P, P, I64, P, ctypes.c_float, P,
                                   ctypes.c_int, P, SZ, P]
    lib.rolesub_attend_causal.argtypes = [P, ctypes.c_int, P, P, P, P, P, I64, P, ctypes.c_float, P,
                                          ctypes.c_int, P, SZ, P]
    lib.rolesub_retain_tokens.argtypes = [I32, I32, I32, P, P, P, P, P]
    lib.rolesub_gather_tokens.argtypes = [I32, I32, I32, I64, P, P, P, P]
    lib.rolesub_allocate_groups.argtypes = [I32, I32, I32, P, P, P, P, P, P, P, P, P]
    lib.rolesub_route_allocate_workspace_size.argtypes = [P, P]
    lib.rolesub_route_allocate.argtypes = [P, ctypes.c_int, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P]
    lib.rolesub_full_workspace_size.argtypes = [I32, I32, I32]
    lib.rolesub_full_workspace_size.restype = SZ
    lib.rolesub_full_transpose.argtypes = [I32, ctypes.c_int, P, P, P]
    lib.rolesub_full_rotate_pack.argtypes = [P, ctypes.c_int, P, P, P, P, P, I64, P, P, P, SZ, P]
    lib.rolesub_full_values.argtypes = [P, ctypes.c_int, P, P, P, P, I64, P, P, SZ, P]
    lib.rolesub_attend_values.argtypes = [P, ctypes.c_int, I32, P, P, P, ctypes.c_float, P, ctypes.c_int, P]
    F, C = ctypes.c_float, ctypes.c_int
    lib.rolesub_rotary.argtypes = [I32, I32, I32, I32, I32, C, P, I64, P, I64, P, I32, P, P, I32, I32, I32, P, P, P]
    lib.rolesub_cache_append.argtypes = [P, C, I32, I32, P, I64, P, I64, P, P, I32, P, P, P]
    lib.rolesub_attend_paged_workspace_size.argtypes = [P, I32, I32, I32, I32, I32]
    lib.rolesub_attend_paged_workspace_size.restype = SZ
    lib.rolesub_attend_paged.argtypes = [P, C, I32, I32, I32, P, I64, P, I32, P, P, I32, P, F, P, C, P, F, P, I64, P, SZ, P]
    lib.rolesub_evict_workspace_size.argtypes = [I32, I32]
    lib.rolesub_evict_workspace_size.restype = SZ
    lib.rolesub_evict_tokens.argtypes = [I32, I32, P, I64, P, I32, I32, I32, P, P, P, SZ, P]
    lib.rolesub_cache_compact.argtypes = [P, P, C, I32, P, I32, P, P, I32, P, I32, P, I64, P, I64, P]
    lib.rolesub_norm_rotary.argtypes = [I32, I32, I32, I32, I32, C, P, I64, P, I64, P, P, F, P, I32, P, P, I32, I32, P, P, P]
    lib.rolesub_append_rotary.argtypes = [P, C, I32, I32, I32, P, I64, P, I64, P, I64, P, P, P, P, F, P, I32, P, P, I32, I32,
                                          P, I32, P, P, P, P]
    lib.rolesub_tree_masks.argtypes = [I32, I32, P, P, P, P]
    lib.rolesub_attend_tree_workspace_size.argtypes = [P, I32, I32, I32, I32]
    lib.rolesub_attend_tree_workspace_size.restype = SZ
    lib.rolesub_attend_tree.argtypes = [P, C, I32, I32, I32, P, I64, P, I32, P, P, P, I32, I32, P, F, P, C, P, SZ, P]
    lib.rolesub_cache_accept.argtypes = [P, C, I32, I32, P, I32, P, P, I32, P, P, P]
    lib.rolesub_page_bounds.argtypes = [P, C, I32, I32, P, I32, P, P, P]
    lib.rolesub_select_pages_workspace_size.argtypes = [P, I32, I32, I32]
    lib.rolesub_select_pages_workspace_size.restype = SZ
    lib.rolesub_select_pages.argtypes = [P, C, I32, I32, I32, P, I64, P, P, I32, P, P, I32, I32, I32, I32, P, P, SZ, P]
    lib.rolesub_attend_selected_workspace_size.argtypes = [P, I32, I32, I32, I32]
    lib.rolesub_attend_selected_workspace_size.restype = SZ
    lib.rolesub_attend_selected.argtypes = [P, C, I32, I32, I32, P, I64, P, I32, P, P, P, I32, P, F, P, C, P, SZ, P]
    for fn in ("rolesub_rotate_values", "rolesub_route", "rolesub_route_noalloc", "rolesub_pack_kv",
               "rolesub_rotate_pack", "rolesub_attend"):
        getattr(lib, fn).restype = ctypes.c_int
    _lib = lib
    return lib


def status_name(status: int) -> str:
    return load().rolesub_status_str(status).decode()


# A layer at small batches is bound by the host work of its calls, so the checks
# below take a short way when everything is in order (shapes compared as whole
# tuples, raw addresses and stream handles, one constructor per struct); what fails
# it is looked at in detail.
_Tensor = torch.Tensor
_I32x4 = ctypes.c_int32 * 4


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise RolesubError(fn, status, load().rolesub_last_error().decode())


_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _code(t: torch.Tensor) -> int:
    c = _CODES.get(t.dtype)
    if c is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return c


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not isinstance(t, _Tensor):
        raise TypeError("expected a torch tensor")
    if not t.is_cuda:
        raise ValueError("librolesub takes device tensors only")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _fmt(shape):
    return "[" + ", ".join("*" if x is None else str(int(x)) for x in shape) + "]"


def _need(name, t, shape, dtype=None):
    """Check a tensor argument's shape (None: any extent) and dtype on the host,
    before anything is launched: the library receives bare pointers and would
    otherwise read or write past a wrongly sized buffer."""
    if t is None:
        return
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.shape == shape and (dtype is None or t.dtype is dtype):
        return
    got = t.shape
    ok = len(got) == len(shape)
    if ok:
        for want, x in zip(shape, got):
            if want is not None and want != x and int(want) != int(x):
                ok = False
                break
    if not ok:
        raise ValueError(f"{name}: expected shape {_fmt(shape)}, got {list(got)}")
    if dtype is not None:
        ok = dtype if isinstance(dtype, tuple) else (dtype,)
        if t.dtype not in ok:
            raise TypeError(f"{name}: expected dtype {' or '.join(str(d) for d in ok)}, got {t.dtype}")


_MASK = (torch.int32, torch.uint32)


def _same_device(*ts):
    first = None
    for t in ts:
        if isinstance(t, _Tensor):
            d = t.device
            if first is None:
                first = d
            elif d != first:
                devs = {t.device for t in ts if isinstance(t, _Tensor)}
                raise ValueError(f"tensors on different devices: {sorted(str(d) for d in devs)}")


def _need_workspace(t):
    if t is not None:
        _need("workspace", t, (None,), torch.uint8)


# torch.cuda.current_stream().cuda_stream without the Stream object, where this
# torch has the two calls it takes
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _empty(shape, dtype, device, stream, output=True):
    """A new tensor for a call on `stream` (None: the current one). It comes out of that
    stream's memory: a block of the current stream's could still be in use by what is
    pending there, which `stream` does not wait for. An output is the current
    stream's as well, where the caller goes on with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if output and t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def make_budget(mode=TOPK, k_by_type=(0, 0, 0, 0), tau=0.0, kmin=0, kmax=0) -> Budget:
    b = Budget()
    b.mode = mode
    for i, k in enumerate(k_by_type):
        b.k_by_type[i] = int(k)
    b.tau, b.kmin, b.kmax = float(tau), int(kmin), int(kmax)
    return b


@dataclass
class Router:
    """Router weights as device tensors (kept alive while calls are in flight)."""
    kind: int
    C: int
    tensors: dict
    d_e: int = 0
    Hr: int = 0
    alpha_role: float = 0.1
    alpha_lang: float = 0.1

    def desc(self) -> RouterDesc:
        return RouterDesc(self.kind, self.C, self.d_e, self.Hr, self.alpha_role, self.alpha_lang,
                          **{name: _ptr(t) for name, t in self.tensors.items()})

    def check(self, d: int, G: int, dtype) -> None:
        """Weight shapes against the hidden size d and G groups (row-major [out][in])."""
        t, C = self.tensors, self.C
        if self.kind == MLP2:
            shapes = dict(W_r=(C, d), b_r=(C,), E=(C, self.d_e), W1=(self.Hr, 2 * d + self.d_e), b1=(self.Hr,),
                          W2=(G, self.Hr), b2=(G,))
        else:
            shapes = dict(W_tok=(G, d), b_tok=(G,), W_r=(C, d), b_r=(C,), W_role=(G, C), W_lang=(G, d),
                          b_lang=(G,))
        for name, shape in shapes.items():
            if name not in t:
                raise ValueError(f"router: missing {name}")
            w = t[name]
            if not isinstance(w, _Tensor) or w.shape != shape or w.dtype is not dtype:
                _need(f"router.{name}", w, shape, dtype)

    @staticmethod
    def mlp2(W_r, b_r, E, W1, b1, W2, b2) -> "Router":
        return Router(MLP2, W_r.shape[0], dict(W_r=W_r, b_r=b_r, E=E, W1=W1, b1=b1, W2=W2, b2=b2),
                      d_e=E.shape[1], Hr=W1.shape[0])

    @staticmethod
    def additive(W_tok, b_tok, W_r, b_r, W_role, W_lang, b_lang, alpha_role=0.1, alpha_lang=0.1):
        return Router(ADDITIVE, W_r.shape[0], dict(W_tok=W_tok, b_tok=b_tok, W_r=W_r, b_r=b_r,
                                                   W_role=W_role, W_lang=W_lang, b_lang=b_lang),
                      alpha_role=alpha_role, alpha_lang=alpha_lang)


# ----------------------------------------------------------------------------
# The four calls
# ----------------------------------------------------------------------------

def rotate_values(v: torch.Tensor, R: torch.Tensor, out: torch.Tensor | None = None, stream=None):
    """z = R_h^T v per head. v [B,T,H,dh], R [H,dh,dh]."""
    _need("v", v, (None, None, None, None))
    B, T, H, dh = v.shape
    _need("R", R, (H, dh, dh), v.dtype)
    _need("out", out, (B, T, H, dh), v.dtype)
    _same_device(v, R, out)
    z = _empty(v.shape, v.dtype, v.device, stream) if out is None else out
    dims = Dims(B, T, H, dh, 1, 0)
    _check("rolesub_rotate_values", load().rolesub_rotate_values(
        ctypes.byref(dims), _code(v), _ptr(v), _ptr(R, v.dtype), _ptr(z, v.dtype), _stream(stream)))
    return z


def route_workspace_size(B, T, G, d, router: Router) -> int:
    dims = Dims(B, T, 1, 64, G, d)
    desc = router.desc()
    return load().rolesub_route_workspace_size(ctypes.byref(dims), ctypes.byref(desc))


def route(token_type: torch.Tensor, budget: Budget, G: int, h: torch.Tensor | None = None,
          router: Router | None = None, scores_in: torch.Tensor | None = None, *,
          want_scores=True, want_idx=True, want_count=True, workspace=None, out=None, stream=None):
    """Routing scores and group selection. Returns dict(mask, idx, count, scores)."""
    _need("token_type", token_type, (None, None), torch.uint8)
    B, T = token_type.shape
    dev = token_type.device
    _need("h", h, (B, T, None), (torch.float32, torch.bfloat16))
    d = 0 if h is None else h.shape[2]
    dtype = torch.float32 if h is None else h.dtype
    _need("scores_in", scores_in, (B, T, G), torch.float32)
    if router is not None and h is not None:
        router.check(d, G, dtype)
    o = out or {}
    for name, shape, dt in (("mask", (B, T), _MASK), ("idx", (B, T, G), torch.uint8),
                            ("count", (B, T), torch.uint8), ("scores", (B, T, G), torch.float32)):
        x = o.get(name)
        if x is not None and (not isinstance(x, _Tensor) or x.shape != shape or x.dtype is not dt):
            _need(f"out[{name!r}]", x, shape, dt)
    _need_workspace(workspace)
    _same_device(token_type, h, scores_in, workspace, *o.values())

    def buf(name, shape, dtype, want=True):
        if not want:
            return None
        return o[name] if name in o else _empty(shape, dtype, dev, stream)

    mask = buf("mask", (B, T), torch.int32)
    idx = buf("idx", (B, T, G), torch.uint8, want_idx)
    cnt = buf("count", (B, T), torch.uint8, want_count)
    sco = buf("scores", (B, T, G), torch.float32, want_scores)
    dims = Dims(B, T, 1, 64, G, d)
    desc = router.desc() if router is not None else None
    ws_ptr, ws_bytes = None, 0
    if scores_in is None and router is not None:
        if workspace is None:
            ws_bytes = load().rolesub_route_workspace_size(ctypes.byref(dims), ctypes.byref(desc))
            workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, output=False)
        ws_ptr, ws_bytes = _ptr(workspace), workspace.numel()
    _check("rolesub_route", load().rolesub_route(
        ctypes.byref(dims), F32 if dtype == torch.float32 else BF16,
        ctypes.byref(desc) if desc is not None else None, ctypes.byref(budget),
        _ptr(h), _ptr(token_type, torch.uint8), _ptr(scores_in, torch.float32), _ptr(sco),
        _ptr(mask), _ptr(idx), _ptr(cnt), ws_ptr, ws_bytes, _stream(stream)))
    return {"mask": mask, "idx": idx, "count": cnt, "scores": sco}


def route_noalloc(token_type: torch.Tensor, budget: Budget, G: int, h: torch.Tensor | None = None,
                  router: Router | None = None, scores_in: torch.Tensor | None = None, *, out, stream=None):
    """rolesub_route with the library's own fixed device scratch as workspace:
    the call allocates nothing. Every output buffer comes from the caller
    (out: dict with mask [B,T] int32 and optionally idx, count, scores)."""
    _need("token_type", token_type, (None, None), torch.uint8)
    B, T = token_type.shape
    _need("h", h, (B, T, None), (torch.float32, torch.bfloat16))
    d = 0 if h is None else h.shape[2]
    dtype = torch.float32 if h is None else h.dtype
    _need("scores_in", scores_in, (B, T, G), torch.float32)
    if router is not None and h is not None:
        router.check(d, G, dtype)
    if "mask" not in out:
        raise ValueError("out['mask'] is required")
    for name, shape, dt in (("mask", (B, T), _MASK), ("idx", (B, T, G), torch.uint8),
                            ("count", (B, T), torch.uint8), ("scores", (B, T, G), torch.float32)):
        x = out.get(name)
        if x is not None and (not isinstance(x, _Tensor) or x.shape != shape or x.dtype is not dt):
            _need(f"out[{name!r}]", x, shape, dt)
    _same_device(token_type, h, scores_in, *out.values())
    dims = Dims(B, T, 1, 64, G, d)
    desc = router.desc() if router is not None else None
    _check("rolesub_route_noalloc", load().rolesub_route_noalloc(
        ctypes.byref(dims), F32 if dtype == torch.float32 else BF16,
        ctypes.byref(desc) if desc is not None else None, ctypes.byref(budget),
        _ptr(h), _ptr(token_type, torch.uint8), _ptr(scores_in, torch.float32), _ptr(out.get("scores")),
        _ptr(out["mask"]), _ptr(out.get("idx")), _ptr(out.get("count")), _stream(stream)))
    return out


def pack_kv(z: torch.Tensor, mask: torch.Tensor, G: int, cap: int, budget: Budget | None = None,
            type_counts=None, out=None, stream=None):
    """Compact group-indexed cache. Returns (offsets [B,T+1] int32, Vp [B,H,cap,ds])."""
    _need("z", z, (None, None, None, None))
    B, T, H, dh = z.shape
    ds = dh // G
    _need("mask", mask, (B, T), _MASK)
    if out is not None:
        _need("offsets", out[0], (B, T + 1), torch.int32)
        _need("Vp", out[1], (B, H, cap, ds), z.dtype)
    _same_device(z, mask, *(out or ()))
    offsets = _empty((B, T + 1), torch.int32, z.device, stream) if out is None else out[0]
    Vp = _empty((B, H, cap, ds), z.dtype, z.device, stream) if out is None else out[1]
    dims = Dims(B, T, H, dh, G, 0)
    tc = _I32x4(*type_counts) if type_counts is not None else None
    _check("rolesub_pack_kv", load().rolesub_pack_kv(
        ctypes.byref(dims), _code(z), ctypes.byref(budget) if budget is not None else None, tc,
        _ptr(z), _ptr(mask), _ptr(offsets, torch.int32), _ptr(Vp, z.dtype), int(cap), _stream(stream)))
    return offsets, Vp


def rotate_pack(v: torch.Tensor, R: torch.Tensor, mask: torch.Tensor, G: int, cap: int,
                budget: Budget | None = None, type_counts=None, out=None, stream=None):
    """Rotation and pack in one pass (z is not materialised). Returns (offsets, Vp)."""
    _need("v", v, (None, None, None, None))
    B, T, H, dh = v.shape
    ds = dh // G
    _need("R", R, (H, dh, dh), v.dtype)
    _need("mask", mask, (B, T), _MASK)
    if out is not None:
        _need("offsets", out[0], (B, T + 1), torch.int32)
        _need("Vp", out[1], (B, H, cap, ds), v.dtype)
    _same_device(v, R, mask, *(out or ()))
    offsets = _empty((B, T + 1), torch.int32, v.device, stream) if out is None else out[0]
    Vp = _empty((B, H, cap, ds), v.dtype, v.device, stream) if out is None else out[1]
    dims = Dims(B, T, H, dh, G, 0)
    tc = _I32x4(*type_counts) if type_counts is not None else None
    _check("rolesub_rotate_pack", load().rolesub_rotate_pack(
        ctypes.byref(dims), _code(v), ctypes.byref(budget) if budget is not None else None, tc,
        _ptr(v), _ptr(R, v.dtype), _ptr(mask), _ptr(offsets, torch.int32), _ptr(Vp, v.dtype), int(cap),
        _stream(stream)))
    return offsets, Vp


def attend(q, k, mask, offsets, Vp, R, G: int, scale: float = 0.0, out_dtype=None, out=None, stream=None):
    """Attention with full q, k over the packed routed values; returns [B,Tq,H,dh]."""
    _need("q", q, (None, None, None, None))
    B, Tq, H, dh = q.shape
    _need("k", k, (B, None, H, dh), q.dtype)
    T = k.shape[1]
    _need("Vp", Vp, (B, H, None, dh // max(G, 1)), q.dtype)
    cap = Vp.shape[2]
    _need("mask", mask, (B, T), _MASK)
    _need("offsets", offsets, (B, T + 1), torch.int32)
    _need("R", R, (H, dh, dh), q.dtype)
    _need("out", out, (B, Tq, H, dh), (torch.float32, torch.bfloat16))
    _same_device(q, k, mask, offsets, Vp, R, out)
    odt = q.dtype if out_dtype is None else out_dtype
    o = _empty((B, Tq, H, dh), odt, q.device, stream) if out is None else out
    dims = Dims(B, T, H, dh, G, 0)
    _check("rolesub_attend", load().rolesub_attend(
        ctypes.byref(dims), _code(q), Tq, _ptr(q), _ptr(k, q.dtype), _ptr(mask), _ptr(offsets, torch.int32),
        _ptr(Vp, q.dtype), int(cap), _ptr(R, q.dtype), float(scale), _ptr(o), _code(o), None, 0,
        _stream(stream)))
    return o


def attend_causal(q, k, mask, offsets, Vp, R, G: int, scale: float = 0.0, out_dtype=None, out=None, stream=None):
    """Prefix self-attention over the packed routed values (query t sees keys
    0..t); q and k are [B,T,H,dh]; returns [B,T,H,dh]."""
    _need("q", q, (None, None, None, None))
    B, T, H, dh = q.shape
    _need("k", k, (B, T, H, dh), q.dtype)
    _need("Vp", Vp, (B, H, None, dh // max(G, 1)), q.dtype)
    cap = Vp.shape[2]
    _need("mask", mask, (B, T), _MASK)
    _need("offsets", offsets, (B, T + 1), torch.int32)
    _need("R", R, (H, dh, dh), q.dtype)
    _need("out", out, (B, T, H, dh), (torch.float32, torch.bfloat16))
    _same_device(q, k, mask, offsets, Vp, R, out)
    odt = q.dtype if out_dtype is None else out_dtype
    o = _empty((B, T, H, dh), odt, q.device, stream) if out is None else out
    dims = Dims(B, T, H, dh, G, 0)
    _check("rolesub_attend_causal", load().rolesub_attend_causal(
        ctypes.byref(dims), _code(q), _ptr(q), _ptr(k, q.dtype), _ptr(mask), _ptr(offsets, torch.int32),
        _ptr(Vp, q.dtype), int(cap), _ptr(R, q.dtype), float(scale), _ptr(o), _code(o), None, 0,
        _stream(stream)))
    return o


def retain_tokens(scores, seg_len, seg_keep, out=None, stream=None):
    """Per sample and per segment of consecutive tokens, the indices of the
    seg_keep highest-scoring tokens (int32 [B, sum(seg_keep)])."""
    _need("scores", scores, (None, None), torch.float32)
    B, N = scores.shape
    n = len(seg_len)
    if len(seg_keep) != n:
        raise ValueError(f"seg_keep has {len(seg_keep)} entries for {n} segments")
    _need("out", out, (B, int(sum(seg_keep))), torch.int32)
    _same_device(scores, out)
    lens = (ctypes.c_int32 * n)(*[int(x) for x in seg_len])
    keeps = (ctypes.c_int32 * n)(*[int(x) for x in seg_keep])
    K = int(sum(seg_keep))
    o = _empty((B, K), torch.int32, scores.device, stream) if out is None else out
    _check("rolesub_retain_tokens", load().rolesub_retain_tokens(
        B, N, n, lens, keeps, _ptr(scores, torch.float32), _ptr(o, torch.int32), _stream(stream)))
    return o


def gather_tokens(x, idx, out=None, stream=None):
    """Rows x[b, idx[b, j]] of a [B, N, ...] tensor (the retained prefix)."""
    if not isinstance(x, torch.Tensor) or x.dim() < 2:
        raise ValueError("x: expected a [B, N, ...] tensor")
    B, N = x.shape[:2]
    _need("idx", idx, (B, None), torch.int32)
    K = idx.shape[1]
    _need("out", out, (B, K) + tuple(x.shape[2:]), x.dtype)
    _same_device(x, idx, out)
    o = _empty((B, K) + tuple(x.shape[2:]), x.dtype, x.device, stream) if out is None else out
    row_bytes = x[0, 0].numel() * x.element_size() if N else 0
    _check("rolesub_gather_tokens", load().rolesub_gather_tokens(
        B, N, K, row_bytes, _ptr(idx, torch.int32), _ptr(x), _ptr(o), _stream(stream)))
    return o


def allocate_groups(priority, token_type, k_by_type, G: int, scores=None, *, want_k=True, want_idx=True,
                    want_count=True, out=None, stream=None):
    """Role-driven within-type group budgets K_i from token priorities, and with
    scores the Top-K_i selection on them. Returns dict(k, mask, idx, count)."""
    _need("token_type", token_type, (None, None), torch.uint8)
    B, T = token_type.shape
    dev = token_type.device
    _need("priority", priority, (B, T), torch.float32)
    _need("scores", scores, (B, T, G), torch.float32)
    o = out or {}
    for name, shape, dt in (("k", (B, T), torch.uint8), ("mask", (B, T), _MASK), ("idx", (B, T, G), torch.uint8),
                            ("count", (B, T), torch.uint8)):
        x = o.get(name)
        if x is not None and (not isinstance(x, _Tensor) or x.shape != shape or x.dtype is not dt):
            _need(f"out[{name!r}]", x, shape, dt)
    _same_device(token_type, priority, scores, *o.values())

    def buf(name, shape, dtype, want=True):
        if not want:
            return None
        return o[name] if name in o else _empty(shape, dtype, dev, stream)

    sel = scores is not None
    kk = buf("k", (B, T), torch.uint8, want_k)
    mask = buf("mask", (B, T), torch.int32, sel)
    idx = buf("idx", (B, T, G), torch.uint8, sel and want_idx)
    cnt = buf("count", (B, T), torch.uint8, sel and want_count)
    kby = _I32x4(*[int(x) for x in k_by_type])
    _check("rolesub_allocate_groups", load().rolesub_allocate_groups(
        B, T, G, kby, _ptr(priority, torch.float32), _ptr(token_type, torch.uint8), _ptr(scores, torch.float32),
        _ptr(kk), _ptr(mask), _ptr(idx), _ptr(cnt), _stream(stream)))
    return {"k": kk, "mask": mask, "idx": idx, "count": cnt}


def route_allocate_workspace_size(B, T, G, d, router: Router) -> int:
    dims = Dims(B, T, 1, 64, G, d)
    desc = router.desc()
    return load().rolesub_route_allocate_workspace_size(ctypes.byref(dims), ctypes.byref(desc))


def route_allocate(token_type, k_by_type, G: int, h, router: Router, w_pri, *, want_priority=True,
                   want_scores=True, want_k=True, want_idx=True, want_count=True, workspace=None, out=None,
                   stream=None):
    """Routing with role-driven budgets: scores, priorities p = w_pri^T a, the
    allocated K_i and the Top-K_i selection. Returns dict(mask, idx, count, k,
    scores, priority)."""
    _need("token_type", token_type, (None, None), torch.uint8)
    B, T = token_type.shape
    dev = token_type.device
    _need("h", h, (B, T, None), (torch.float32, torch.bfloat16))
    d = h.shape[2]
    router.check(d, G, h.dtype)
    _need("w_pri", w_pri, (router.C,), h.dtype)
    o = out or {}
    for name, shape, dt in (("mask", (B, T), _MASK), ("idx", (B, T, G), torch.uint8), ("count", (B, T), torch.uint8),
                            ("k", (B, T), torch.uint8), ("scores", (B, T, G), torch.float32),
                            ("priority", (B, T), torch.float32)):
        x = o.get(name)
        if x is not None and (not isinstance(x, _Tensor) or x.shape != shape or x.dtype is not dt):
            _need(f"out[{name!r}]", x, shape, dt)
    _need_workspace(workspace)
    _same_device(token_type, h, w_pri, workspace, *o.values())

    def buf(name, shape, dtype, want=True):
        if not want:
            return None
        return o[name] if name in o else _empty(shape, dtype, dev, stream)

    mask = buf("mask", (B, T), torch.int32)
    idx = buf("idx", (B, T, G), torch.uint8, want_idx)
    cnt = buf("count", (B, T), torch.uint8, want_count)
    kk = buf("k", (B, T), torch.uint8, want_k)
    sco = buf("scores", (B, T, G), torch.float32, want_scores)
    pri = buf("priority", (B, T), torch.float32, want_priority)
    dims = Dims(B, T, 1, 64, G, d)
    desc = router.desc()
    if workspace is None:
        ws_bytes = load().rolesub_route_allocate_workspace_size(ctypes.byref(dims), ctypes.byref(desc))
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, output=False)
    kby = _I32x4(*[int(x) for x in k_by_type])
    _check("rolesub_route_allocate", load().rolesub_route_allocate(
        ctypes.byref(dims), F32 if h.dtype == torch.float32 else BF16, ctypes.byref(desc), _ptr(w_pri, h.dtype),
        kby, _ptr(h), _ptr(token_type, torch.uint8), _ptr(pri), _ptr(sco), _ptr(kk), _ptr(mask), _ptr(idx),
        _ptr(cnt), _ptr(workspace), workspace.numel(), _stream(stream)))
    return {"mask": mask, "idx": idx, "count": cnt, "k": kk, "scores": sco, "priority": pri}


# ----------------------------------------------------------------------------
# Full-width routing space (one R over all H*dh value dims, S groups)
# ----------------------------------------------------------------------------

def full_workspace_size(B, T, S) -> int:
    return load().rolesub_full_workspace_size(B, T, S)


def full_transpose(R, out=None, stream=None):
    """R^T of a frozen [d_v, d_v] rotation (the layout full_rotate_pack takes)."""
    _need("R", R, (None, None))
    n = R.shape[0]
    _need("R", R, (n, n))
    _need("out", out, (n, n), R.dtype)
    _same_device(R, out)
    Rt = _empty(R.shape, R.dtype, R.device, stream) if out is None else out
    _check("rolesub_full_transpose", load().rolesub_full_transpose(n, _code(R), _ptr(R), _ptr(Rt, R.dtype),
                                                                   _stream(stream)))
    return Rt


def full_rotate_pack(v, Rt, mask, S: int, cap: int, budget: Budget | None = None, type_counts=None,
                     workspace=None, out=None, stream=None):
    """Full-width cache: (offsets [B,T+1] int32, Vp [B,cap,d_v/S])."""
    _need("v", v, (None, None, None, None))
    B, T, H, dh = v.shape
    dv = H * dh
    _need("Rt", Rt, (dv, dv), v.dtype)
    _need("mask", mask, (B, T), _MASK)
    if out is not None:
        _need("offsets", out[0], (B, T + 1), torch.int32)
        _need("Vp", out[1], (B, cap, dv // max(S, 1)), v.dtype)
    _need_workspace(workspace)
    _same_device(v, Rt, mask, workspace, *(out or ()))
    if out is None:
        out = (_empty((B, T + 1), torch.int32, v.device, stream),
               _empty((B, cap, dv // S), v.dtype, v.device, stream))
    offsets, Vp = out
    if workspace is None:
        workspace = _empty(max(full_workspace_size(B, T, S), 1), torch.uint8, v.device, stream, output=False)
    tc = _I32x4(*[int(x) for x in type_counts]) if type_counts is not None else None
    dims = Dims(B, T, H, dh, S, 0)
    _check("rolesub_full_rotate_pack", load().rolesub_full_rotate_pack(
        ctypes.byref(dims), _code(v), _ptr(Rt, v.dtype), _ptr(v), _ptr(mask), _ptr(offsets, torch.int32),
        _ptr(Vp, v.dtype), cap, ctypes.byref(budget) if budget is not None else None, tc, _ptr(workspace),
        workspace.numel(), _stream(stream)))
    return offsets, Vp


def full_values(R, mask, offsets, Vp, S: int, H: int, workspace=None, out=None, stream=None):
    """Routed values [B,H,T,dh] (head-major) from the full-width cache."""
    _need("Vp", Vp, (None, None, None))
    B, cap, ds = Vp.shape
    _need("offsets", offsets, (B, None), torch.int32)
    T = offsets.shape[1] - 1
    if H < 1 or (ds * S) % H:
        raise ValueError(f"d_v = {ds * S} does not split into {H} heads")
    dh = ds * S // H
    _need("R", R, (ds * S, ds * S), Vp.dtype)
    _need("mask", mask, (B, T), _MASK)
    _need("out", out, (B, H, T, dh), Vp.dtype)
    _need_workspace(workspace)
    _same_device(Vp, offsets, R, mask, out, workspace)
    Vh = _empty((B, H, T, dh), Vp.dtype, Vp.device, stream) if out is None else out
    if workspace is None:
        workspace = _empty(max(full_workspace_size(B, T, S), 1), torch.uint8, Vp.device, stream, output=False)
    dims = Dims(B, T, H, dh, S, 0)
    _check("rolesub_full_values", load().rolesub_full_values(
        ctypes.byref(dims), _code(Vp), _ptr(R, Vp.dtype), _ptr(mask), _ptr(offsets, torch.int32), _ptr(Vp),
        cap, _ptr(Vh, Vp.dtype), _ptr(workspace), workspace.numel(), _stream(stream)))
    return Vh


def attend_values(q, k, V, scale: float = 0.0, out_dtype=None, out=None, stream=None):
    """Attention over plain head-major values V [B,H,T,dh] (the full-width
    routing space's rebuilt values). Returns [B,Tq,H,dh]."""
    _need("q", q, (None, None, None, None))
    B, Tq, H, dh = q.shape
    _need("k", k, (B, None, H, dh), q.dtype)
    T = k.shape[1]
    _need("V", V, (B, H, T, dh), q.dtype)
    _need("out", out, (B, Tq, H, dh), (torch.float32, torch.bfloat16))
    _same_device(q, k, V, out)
    od = out.dtype if out is not None else (out_dtype or q.dtype)
    o = _empty((B, Tq, H, dh), od, q.device, stream) if out is None else out
    dims = Dims(B, T, H, dh, 1, 0)
    _check("rolesub_attend_values", load().rolesub_attend_values(
        ctypes.byref(dims), _code(q), Tq, _ptr(q), _ptr(k, q.dtype), _ptr(V, q.dtype), ctypes.c_float(scale),
        _ptr(o), _code(o), _stream(stream)))
    return o


# ----------------------------------------------------------------------------
# Paged routed cache: positions, append, attention of new tokens, eviction
# ----------------------------------------------------------------------------

def _current():
    """The current device's index (-1 without one)."""
    try:
        return torch.cuda.current_device() if _raw_device is None else _raw_device()
    except (RuntimeError, AssertionError):
        return -1


def _args(stream, spec, *caches):
    """Addresses of the tensors of spec, (name, tensor or None, shape, dtype) each, and
    the stream's handle. All lie dense on the current device (the library launches
    there), the caches too; shape None is an operand whose layout _rows has checked.
    What fails the short way is looked at in detail, shapes before devices."""
    cur, out, n = _current(), [], len(spec)
    for c in caches:
        if c._ready != cur:
            spec = c.spec() + tuple(spec)
    for _, t, shape, dtype in spec:
        if t is None:
            out.append(None)
        elif isinstance(t, _Tensor) and t.dtype is dtype and t.get_device() == cur and (
                shape is None or (t.shape == shape and t.is_contiguous())):
            out.append(t.data_ptr())
        else:
            break
    else:
        if cur >= 0 and (stream is None or stream.device_index == cur):
            for c in caches:
                if c._ready != cur:
                    object.__setattr__(c, "_ready", cur)
            return out[len(out) - n:], _stream(stream)
    spec = [(n, t[0, 0, 0], (t.shape[3],), d) if t is not None and x is None else (n, t, x, d) for n, t, x, d in spec]
    for name, t, shape, dtype in spec:
        _need(name, t, shape, dtype)
    out = [_ptr(t) for _, t, _, _ in spec]
    _on_current(cur, stream, [t for _, t, _, _ in spec])
    for c in caches:
        object.__setattr__(c, "_ready", cur)
    return out[len(out) - n:], _stream(stream)


def _on_current(cur, stream, ts):
    _same_device(*ts)
    for t in ts:
        if t is not None and t.get_device() != cur:
            raise ValueError(f"tensors on {t.device}, but the current device is cuda:{cur}")
    if stream is not None and stream.device_index != cur:
        raise ValueError(f"the stream is on cuda:{stream.device_index}, but the current device is cuda:{cur}")


def _rows(name, t):
    """Token stride of a [B, T, H, dh] operand whose tokens lie at one stride (dense,
    or a view of a fused projection), and its shape for _args: None where it is not
    dense, and checked here (a rotation of two such views takes the host 15 us; 21 with
    a dense row of each as its stand-in)."""
    if t.is_contiguous():
        return t.shape[2] * t.shape[3], t.shape
    B, T, H, dh = t.shape
    sb, st, sh, sd = t.stride()
    if T == 1:
        st = sb if B > 1 else H * dh
    # (a stride of 0, an expanded operand, would be taken for dense rows)
    if (sd != 1 and dh > 1) or (sh != dh and H > 1) or (B > 1 and sb != T * st) or st < H * dh:
        raise ValueError(f"{name}: heads and dims must be dense and tokens at one stride, got strides {list(t.stride())}")
    return st, None


def _operand(name, t, H, dh, dtype):
    """Shape, token stride and shape for _args of a [B, T, H (None: any), dh] operand."""
    shape = t.shape if isinstance(t, _Tensor) and t.dtype is dtype else ()
    if len(shape) != 4 or shape[3] != dh or (H is not None and shape[2] != H):
        _need(name, t, (None, None, H, dh), dtype)
    if t.is_contiguous():
        return shape, shape[2] * dh, shape
    return shape, *_rows(name, t)


_FLOATS = (torch.float32, torch.bfloat16)


@dataclass(frozen=True, eq=False)
class PagedCache:
    """Pages of a growing routed cache (kept alive while calls are in flight):
    K [n_pages,H,page,dh], V [n_pages,H,vcap,dh/G], mask and slot [n_pages,page]
    int32. A sequence is a row of page numbers and a length, kept by the caller."""
    K: torch.Tensor
    V: torch.Tensor
    mask: torch.Tensor
    slot: torch.Tensor

    def __post_init__(self):
        _need("K", self.K, (None, None, None, None), _FLOATS)
        n, H, page, dh = self.K.shape
        _need("V", self.V, (n, H, None, None), self.K.dtype)
        ds = self.V.shape[3]
        if ds < 1 or dh % ds:
            raise ValueError(f"V: groups of {ds} dims do not divide heads of {dh}")
        _need("mask", self.mask, (n, page), _MASK)
        _need("slot", self.slot, (n, page), torch.int32)
        put = object.__setattr__
        for name, x in (("G", dh // ds), ("H", H), ("dh", dh), ("page", page), ("dtype", self.K.dtype)):
            put(self, name, x)
        # the library's description of the cache, made once
        put(self, "_desc", PagesDesc(n, page, self.V.shape[2], H, dh, dh // ds, None, None, None, None))
        put(self, "_at", None)
        put(self, "_ready", None)  # the device its arrays were found dense on

    @staticmethod
    def allocate(n_pages, page, H, dh, G, vcap, dtype, device="cuda") -> "PagedCache":
        """vcap: group slots of a page and head; page times the most groups a
        token keeps holds every page."""
        return PagedCache(K=torch.empty((n_pages, H, page, dh), dtype=dtype, device=device),
                          V=torch.empty((n_pages, H, vcap, dh // G), dtype=dtype, device=device),
                          mask=torch.empty((n_pages, page), dtype=torch.int32, device=device),
                          slot=torch.empty((n_pages, page), dtype=torch.int32, device=device))

    def spec(self):
        return tuple((n, t, t.shape, t.dtype) for n, t in zip(("K", "V", "mask", "slot"), self.tensors()))

    def desc(self):
        """The description with the arrays' present addresses."""
        d, at = self._desc, (self.K.data_ptr(), self.V.data_ptr(), self.mask.data_ptr(), self.slot.data_ptr())
        if at != self._at:
            d.K, d.V, d.mask, d.slot = at
            object.__setattr__(self, "_at", at)
        return ctypes.byref(d)

    def tensors(self):
        return self.K, self.V, self.mask, self.slot


def _width(t):
    """Columns of a matrix argument for its spec (None sends it to the detailed check)."""
    return t.shape[1] if isinstance(t, _Tensor) and t.dim() == 2 else None


def rotary(q, k, positions, inv_freq, axis=None, interleaved=False, inverse=False, out=None, stream=None):
    """q [B,T,H,dh] and k [B,T,Hkv,dh] (either may be None) turned by their
    positions ([B,T], or [B,T,axes] with axis [pairs] uint8 naming each pair's).
    out: (q_out, k_out); an input itself turns it in place. Returns (q_out, k_out)."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("q and k are both None")
    shape = some.shape if isinstance(some, _Tensor) else ()
    if len(shape) != 4 or some.dtype not in _FLOATS:
        _need("q" if q is not None else "k", some, (None, None, None, None), _FLOATS)
    B, T, H, dh = shape
    dt = some.dtype
    spec, A, n = [], 1, None
    if isinstance(positions, _Tensor) and positions.dim() == 3:
        A = positions.shape[2]
        spec.append(("positions", positions, (B, T, A), torch.int32))
    else:
        spec.append(("positions", positions, (B, T), torch.int32))
    if isinstance(inv_freq, _Tensor) and inv_freq.dim() == 1:
        n = inv_freq.shape[0]
    spec.append(("inv_freq", inv_freq, (n,), torch.float32))
    spec.append(("axis", axis, (n,), torch.uint8))
    qo, ko = (None, None) if out is None else out
    heads, strides, outs = [0, 0], [0, 0], [qo, ko]
    for i, (name, x) in enumerate((("q", q), ("k", k))):
        o = outs[i]
        if x is None:
            outs[i] = None
            spec += [(name, None, None, None)] * 2
            continue
        if x is some:
            xs = shape
            strides[i], dense = _rows(name, x)
        else:
            xs, strides[i], dense = _operand(name, x, None, dh, dt)
            if xs[0] != B or xs[1] != T:
                _need(name, x, (B, T, None, dh), dt)
        heads[i] = xs[2]
        if o is None:
            o = outs[i] = torch.empty_like(x) if dense and stream is None else _empty(xs, dt, x.device, stream)
            odense = xs
        else:
            _need(f"{name}_out", o, xs, dt)
            so, odense = _rows(f"{name}_out", o)
            if odense is None and (so != strides[i] or o.data_ptr() != x.data_ptr()):
                raise ValueError(f"{name}_out: must be {name} itself or contiguous")
            if odense is not None and o.data_ptr() == x.data_ptr() and dense is None and o.numel():
                raise ValueError(f"{name}_out: must be {name} itself or lie apart from it")
        spec += [(name, x, dense, dt), (f"{name}_out", o, odense, dt)]
    (pp, pf, pa, pq, pqo, pk, pko), s = _args(stream, spec)
    _check("rolesub_rotary", load().rolesub_rotary(
        B, T, heads[0], heads[1], dh, _code(some), pq, strides[0], pk, strides[1], pp, A, pf, pa, n,
        1 if interleaved else 0, 1 if inverse else 0, pqo, pko, s))
    return outs[0], outs[1]


def cache_append(cache: PagedCache, k, z, mask, table, lens, n_new=None, stream=None) -> PagedCache:
    """Token j of sequence b (j < n_new[b], or all) becomes token lens[b] + j of its
    pages: k and z [B,T,H,dh], mask [B,T]; table [B,max_pages], lens [B] int32."""
    dt = cache.dtype
    shape, sk, dk = _operand("k", k, cache.H, cache.dh, dt)
    B, T = shape[:2]
    _need("z", z, shape, dt)
    sz, dz = _rows("z", z)
    W = _width(table)
    (pk, pz, pmask, pt, pl, pn), s = _args(stream, (
        ("k", k, dk, dt), ("z", z, dz, dt),
        ("mask", mask, (B, T), mask.dtype if getattr(mask, "dtype", None) in _MASK else _MASK),
        ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32), ("n_new", n_new, (B,), torch.int32)), cache)
    _check("rolesub_cache_append", load().rolesub_cache_append(
        cache.desc(), _CODES[dt], B, T, pk, sk, pz, sz, pmask, pt, W, pl, pn, s))
    return cache


def attend_paged_workspace_size(cache: PagedCache, B, Hq, Tq, max_len, mass=False) -> int:
    return load().rolesub_attend_paged_workspace_size(ctypes.byref(cache._desc), B, Hq, Tq, max_len, 1 if mass else 0)


def attend_paged(q, cache: PagedCache, table, lens, R=None, scale: float = 0.0, visible=None, max_len: int = 0,
                 mass=None, decay: float = 1.0, mass_out=None, workspace=None, out_dtype=None, out=None, stream=None):
    """Attention of new tokens q [B,Tq,Hq,dh] over the cached ones; returns
    [B,Tq,Hq,dh]. visible [B,Tq] int32: the tokens each query sees. mass [B,>=max_len]
    f32: the tokens' accumulated weight, in place or into mass_out (which alone
    starts from zero): decay * mass + the weight of this call's queries, for every
    token below lens, so entries of tokens that are new must hold zeros."""
    H, dh, dt = cache.H, cache.dh, cache.dtype
    shape, sq, dq = _operand("q", q, None, dh, dt)
    B, Tq, Hq, _ = shape
    W, ld = _width(table), 0
    if mass_out is None:
        mass_out = mass
    if mass_out is not None:
        ld = _width(mass_out) if mass is None else _width(mass)
    o = _empty(shape, out_dtype or dt, q.device, stream) if out is None else out
    odt = o.dtype if isinstance(o, _Tensor) and o.dtype in _CODES else _FLOATS
    if workspace is None:
        whole = (W or 0) * cache.page
        need = attend_paged_workspace_size(cache, B, Hq, Tq, min(int(max_len), whole) if max_len else whole,
                                           mass_out is not None)
        workspace = _empty(max(need, 1), torch.uint8, q.device, stream, output=False)
    ws = workspace.numel() if isinstance(workspace, _Tensor) else 0
    (pq, pt, pl, pR, pv, pmi, pmo, po, pw), s = _args(stream, (
        ("q", q, dq, dt), ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32),
        ("R", R, (H, dh, dh), dt), ("visible", visible, (B, Tq), torch.int32), ("mass", mass, (B, ld), torch.float32),
        ("mass_out", mass_out, (B, ld), torch.float32), ("out", o, shape, odt), ("workspace", workspace, (ws,), torch.uint8)), cache)
    _check("rolesub_attend_paged", load().rolesub_attend_paged(
        cache.desc(), _CODES[dt], B, Hq, Tq, pq, sq, pt, W, pl, pv, int(max_len), pR, float(scale), po,
        _CODES[odt], pmi, float(decay), pmo, ld, pw, ws, s))
    return o


def evict_workspace_size(B, max_len) -> int:
    return load().rolesub_evict_workspace_size(B, max_len)


def evict_tokens(mass, lens, keep: int, first: int = 0, recent: int = 0, max_len: int = 0, workspace=None, out=None,
                 stream=None):
    """Which `keep` tokens of every sequence stay: the first, the recent, and of the
    others those with the most mass [B,>=max_len]. Returns (keep_idx [B,keep] int32,
    ascending, then -1; n_keep [B] int32). max_len 0: mass.shape[1]."""
    shape = mass.shape if isinstance(mass, _Tensor) else ()
    if len(shape) != 2:
        _need("mass", mass, (None, None), torch.float32)
    B, ld = shape
    if out is None:
        if keep < 1:
            raise ValueError(f"keep: expected at least 1, got {keep}")
        out = (_empty((B, keep), torch.int32, mass.device, stream), _empty((B,), torch.int32, mass.device, stream))
    idx, n = out
    ml = int(max_len) if max_len else ld
    if workspace is None:
        workspace = _empty(max(evict_workspace_size(B, ml), 1), torch.uint8, mass.device, stream, output=False)
    ws = workspace.numel() if isinstance(workspace, _Tensor) else 0
    (pm, pl, pi, pn, pw), s = _args(stream, (
        ("mass", mass, (B, ld), torch.float32), ("lens", lens, (B,), torch.int32), ("keep_idx", idx, (B, keep), torch.int32),
        ("n_keep", n, (B,), torch.int32), ("workspace", workspace, (ws,), torch.uint8)))
    _check("rolesub_evict_tokens", load().rolesub_evict_tokens(
        B, ml, pm, ld, pl, int(keep), int(first), int(recent), pi, pn, pw, ws, s))
    return idx, n


def cache_compact(src: PagedCache, table, keep_idx, n_keep, dst: PagedCache, dst_table, mass=None, mass_out=None,
                  stream=None):
    """Token j < n_keep[b] of the pages dst_table[b] of dst becomes token
    keep_idx[b, j] of the pages table[b] of src; mass_out[b, j] = mass[b, keep_idx[b, j]]
    (a new [B, keep] tensor when mass comes alone). Returns mass_out (or None)."""
    shape = keep_idx.shape if isinstance(keep_idx, _Tensor) else ()
    if len(shape) != 2:
        _need("keep_idx", keep_idx, (None, None), torch.int32)
    B, keep = shape
    dt = src.dtype
    if dst.dtype is not dt:
        _need("dst.K", dst.K, (None, None, None, None), dt)
    if mass is None and mass_out is not None:
        raise ValueError("mass_out without mass")
    if mass is not None and mass_out is None:
        mass_out = _empty((B, keep), torch.float32, mass.device, stream)
    W, D, L, M = _width(table), _width(dst_table), _width(mass), _width(mass_out)
    (pi, pn, pt, pd, pm, pmo), s = _args(stream, (
        ("keep_idx", keep_idx, (B, keep), torch.int32), ("n_keep", n_keep, (B,), torch.int32),
        ("table", table, (B, W), torch.int32), ("dst_table", dst_table, (B, D), torch.int32),
        ("mass", mass, (B, L), torch.float32), ("mass_out", mass_out, (B, M), torch.float32)), src, dst)
    _check("rolesub_cache_compact", load().rolesub_cache_compact(
        src.desc(), dst.desc(), _CODES[dt], B, pt, W, pi, pn, keep, pd, D, pm, L or 0, pmo, M or 0, s))
    return mass_out


# ----------------------------------------------------------------------------
# Paged routed cache: normed heads, drafted tokens, few pages of a long history
# ----------------------------------------------------------------------------

def _positions(positions, B, T, inv_freq, axis, spec):
    """Positions, frequencies and axes of a call that turns heads, into its spec: (axes, pairs)."""
    A, n = 1, None
    if isinstance(positions, _Tensor) and positions.dim() == 3:
        A = positions.shape[2]
        spec.append(("positions", positions, (B, T, A), torch.int32))
    else:
        spec.append(("positions", positions, (B, T), torch.int32))
    if isinstance(inv_freq, _Tensor) and inv_freq.dim() == 1:
        n = inv_freq.shape[0]
    spec += [("inv_freq", inv_freq, (n,), torch.float32), ("axis", axis, (n,), torch.uint8)]
    return A, n


def _turned(name, x, xs, stride, dense, o, dt, stream):
    """The output of a call that turns x (new where o is None), and its shape for _args."""
    if o is None:
        return (torch.empty_like(x) if dense and stream is None else _empty(xs, dt, x.device, stream)), xs
    _need(f"{name}_out", o, xs, dt)
    so, odense = _rows(f"{name}_out", o)
    if odense is None and (so != stride or o.data_ptr() != x.data_ptr()):
        raise ValueError(f"{name}_out: must be {name} itself or contiguous")
    if odense is not None and o.data_ptr() == x.data_ptr() and dense is None and o.numel():
        raise ValueError(f"{name}_out: must be {name} itself or lie apart from it")
    return o, odense


def norm_rotary(q, k, q_weight, k_weight, eps: float, positions, inv_freq, axis=None, interleaved=False, out=None,
                stream=None):
    """rotary of q and k (either may be None) whose heads are first divided by their root
    mean square and weighted: q_weight and k_weight [dh], None for a tensor that is
    turned only. out: (q_out, k_out); an input itself is written in place. Returns
    (q_out, k_out)."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("q and k are both None")
    shape = some.shape if isinstance(some, _Tensor) else ()
    if len(shape) != 4 or some.dtype not in _FLOATS:
        _need("q" if q is not None else "k", some, (None, None, None, None), _FLOATS)
    B, T, _, dh = shape
    dt = some.dtype
    spec = []
    A, n = _positions(positions, B, T, inv_freq, axis, spec)
    outs, heads, strides = [None, None] if out is None else list(out), [0, 0], [0, 0]
    for i, (name, x, w) in enumerate((("q", q, q_weight), ("k", k, k_weight))):
        if x is None:
            outs[i] = None
            spec += [(name, None, None, None)] * 3
            continue
        xs, strides[i], dense = _operand(name, x, None, dh, dt)
        if xs[0] != B or xs[1] != T:
            _need(name, x, (B, T, None, dh), dt)
        heads[i] = xs[2]
        outs[i], odense = _turned(name, x, xs, strides[i], dense, outs[i], dt, stream)
        spec += [(name, x, dense, dt), (f"{name}_weight", w, (dh,), dt), (f"{name}_out", outs[i], odense, dt)]
    (pp, pf, pa, pq, pqw, pqo, pk, pkw, pko), s = _args(stream, spec)
    _check("rolesub_norm_rotary", load().rolesub_norm_rotary(
        B, T, heads[0], heads[1], dh, _CODES[dt], pq, strides[0], pk, strides[1], pqw, pkw, float(eps), pp, A, pf, pa, n,
        1 if interleaved else 0, pqo, pko, s))
    return outs[0], outs[1]


def append_rotary(cache: PagedCache, k, v, mask, table, lens, positions, inv_freq, axis=None, R=None, q=None,
                  q_weight=None, k_weight=None, eps: float = 1e-6, interleaved=False, n_new=None, q_out=None, stream=None):
    """cache_append of new tokens straight from their projections: keys k [B,T,H,dh]
    normed (with k_weight [dh]) and turned by their positions, values v [B,T,H,dh]
    rotated by R [H,dh,dh] (None: kept as they are). Returns the queries q [B,T,Hq,dh],
    normed (with q_weight) and turned, or None without them."""
    dt, dh = cache.dtype, cache.dh
    shape, sk, dk = _operand("k", k, cache.H, dh, dt)
    B, T = shape[:2]
    _need("v", v, shape, dt)
    sv, dv = _rows("v", v)
    W, Hq, sq = _width(table), 0, 0
    spec = []
    A, n = _positions(positions, B, T, inv_freq, axis, spec)
    if q is None:
        if q_weight is not None or q_out is not None:
            raise ValueError("q_weight and q_out need q")
        spec += [("q", None, None, None)] * 3
    else:
        qs, sq, dq = _operand("q", q, None, dh, dt)
        if qs[0] != B or qs[1] != T:
            _need("q", q, (B, T, None, dh), dt)
        Hq = qs[2]
        q_out, odense = _turned("q", q, qs, sq, dq, q_out, dt, stream)
        spec += [("q", q, dq, dt), ("q_weight", q_weight, (dh,), dt), ("q_out", q_out, odense, dt)]
    spec += [("k", k, dk, dt), ("v", v, dv, dt), ("k_weight", k_weight, (dh,), dt), ("R", R, (cache.H, dh, dh), dt),
             ("mask", mask, (B, T), mask.dtype if getattr(mask, "dtype", None) in _MASK else _MASK),
             ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32), ("n_new", n_new, (B,), torch.int32)]
    (pp, pf, pa, pq, pqw, pqo, pk, pv, pkw, pR, pm, pt, pl, pn), s = _args(stream, spec, cache)
    _check("rolesub_append_rotary", load().rolesub_append_rotary(
        cache.desc(), _CODES[dt], B, T, Hq, pq, sq, pk, sk, pv, sv, pR, pm, pqw, pkw, float(eps), pp, A, pf, pa, n,
        1 if interleaved else 0, pt, W, pl, pn, pqo, s))
    return q_out


def tree_masks(parents, out=None, stream=None):
    """Ancestors of drafted tokens from their parents [B,T] int32 (negative: a child of the
    cached tokens). Returns (tree [B,T,ceil(T/32)] int32 bits, themselves among them; depth
    [B,T] int32, how many ancestors)."""
    shape = parents.shape if isinstance(parents, _Tensor) else ()
    if len(shape) != 2:
        _need("parents", parents, (None, None), torch.int32)
    B, T = shape
    words = (B, T, (T + 31) // 32)
    if out is None:
        out = (_empty(words, torch.int32, parents.device, stream), _empty((B, T), torch.int32, parents.device, stream))
    tree, depth = out
    (pp, pt, pd), s = _args(stream, (
        ("parents", parents, (B, T), torch.int32),
        ("tree", tree, words, tree.dtype if getattr(tree, "dtype", None) in _MASK else _MASK),
        ("depth", depth, (B, T), torch.int32)))
    _check("rolesub_tree_masks", load().rolesub_tree_masks(B, T, pp, pt, pd, s))
    return tree, depth


def _tree(tree, B, T):
    """A tree's bits for _args, and how many trees there are."""
    n = tree.shape[0] if isinstance(tree, _Tensor) and tree.dim() == 3 and tree.shape[0] == 1 else B
    return ("tree", tree, (n, T, (T + 31) // 32), tree.dtype if getattr(tree, "dtype", None) in _MASK else _MASK), n


def attend_tree_workspace_size(cache: PagedCache, B, Hq, Tq, max_len) -> int:
    return load().rolesub_attend_tree_workspace_size(ctypes.byref(cache._desc), B, Hq, Tq, max_len)


def attend_tree(q, cache: PagedCache, table, lens, tree, R=None, n_new=None, scale: float = 0.0, max_len: int = 0,
                workspace=None, out_dtype=None, out=None, stream=None):
    """Attention of drafted tokens q [B,Tq,Hq,dh], cached from lens [B] on, each over the
    cached tokens before them and its own bits of tree [B or 1,Tq,ceil(Tq/32)]; rows past
    n_new [B] (None: Tq) give zeros. Returns [B,Tq,Hq,dh]."""
    H, dh, dt = cache.H, cache.dh, cache.dtype
    shape, sq, dq = _operand("q", q, None, dh, dt)
    B, Tq, Hq, _ = shape
    W = _width(table)
    o = _empty(shape, out_dtype or dt, q.device, stream) if out is None else out
    odt = o.dtype if isinstance(o, _Tensor) and o.dtype in _CODES else _FLOATS
    if workspace is None:
        whole = (W or 0) * cache.page
        need = attend_tree_workspace_size(cache, B, Hq, Tq, min(int(max_len), whole) if max_len else whole)
        workspace = _empty(max(need, 1), torch.uint8, q.device, stream, output=False)
    ws = workspace.numel() if isinstance(workspace, _Tensor) else 0
    bits, trees = _tree(tree, B, Tq)
    (pq, pt, pl, pn, pb, pR, po, pw), s = _args(stream, (
        ("q", q, dq, dt), ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32),
        ("n_new", n_new, (B,), torch.int32), bits, ("R", R, (H, dh, dh), dt), ("out", o, shape, odt),
        ("workspace", workspace, (ws,), torch.uint8)), cache)
    _check("rolesub_attend_tree", load().rolesub_attend_tree(
        cache.desc(), _CODES[dt], B, Hq, Tq, pq, sq, pt, W, pl, pn, pb, trees, int(max_len), pR, float(scale), po,
        _CODES[odt], pw, ws, s))
    return o


def cache_accept(cache: PagedCache, table, lens, tree, leaf, new_lens=None, stream=None):
    """Of the drafted tokens cached from lens [B] on, those on the path of token leaf [B]
    (its bits of tree [B or 1,T,ceil(T/32)]; -1: none) move behind the cached ones.
    Returns the new lengths [B]."""
    T = tree.shape[1] if isinstance(tree, _Tensor) and tree.dim() == 3 else 0
    B = leaf.shape[0] if isinstance(leaf, _Tensor) and leaf.dim() == 1 else None
    if B is None:
        _need("leaf", leaf, (None,), torch.int32)
        raise TypeError("leaf: expected a torch tensor, got None")
    if new_lens is None:
        new_lens = _empty((B,), torch.int32, leaf.device, stream)
    W = _width(table)
    bits, trees = _tree(tree, B, T)
    (pl, pt, pn, pb, po), s = _args(stream, (
        ("leaf", leaf, (B,), torch.int32), ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32), bits,
        ("new_lens", new_lens, (B,), torch.int32)), cache)
    _check("rolesub_cache_accept", load().rolesub_cache_accept(
        cache.desc(), _CODES[cache.dtype], B, T, pt, W, pn, pb, trees, pl, po, s))
    return new_lens


def page_bounds(cache: PagedCache, table, lens, bounds, T: int, stream=None):
    """Bounds [n_pages,H,2,dh] of the keys in the pages that hold each sequence's last T
    tokens (lens [B] counts them), written over what was there. Returns bounds."""
    B = lens.shape[0] if isinstance(lens, _Tensor) and lens.dim() == 1 else None
    W = _width(table)
    (pt, pl, pb), s = _args(stream, (
        ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32),
        ("bounds", bounds, (cache.K.shape[0], cache.H, 2, cache.dh), cache.dtype)), cache)
    _check("rolesub_page_bounds", load().rolesub_page_bounds(
        cache.desc(), _CODES[cache.dtype], B, int(T), pt, W, pl, pb, s))
    return bounds


def select_pages_workspace_size(cache: PagedCache, B, Tq, max_len) -> int:
    return load().rolesub_select_pages_workspace_size(ctypes.byref(cache._desc), B, Tq, max_len)


def select_pages(q, cache: PagedCache, bounds, table, lens, n_sel: int, first: int = 0, recent: int = 0, visible=None,
                 max_len: int = 0, workspace=None, out=None, stream=None):
    """The n_sel pages that each query q [B,Tq,Hq,dh] and key head attends to: the first, the
    recent, and of the others those whose bounds promise the highest scores. Returns
    [B,Tq,H,n_sel] int32, ascending, then -1."""
    dh, dt, H = cache.dh, cache.dtype, cache.H
    shape, sq, dq = _operand("q", q, None, dh, dt)
    B, Tq, Hq, _ = shape
    W = _width(table)
    if out is None:
        if n_sel < 1:
            raise ValueError(f"n_sel: expected at least 1, got {n_sel}")
        out = _empty((B, Tq, H, int(n_sel)), torch.int32, q.device, stream)
    if workspace is None:
        whole = (W or 0) * cache.page
        need = select_pages_workspace_size(cache, B, Tq, min(int(max_len), whole) if max_len else whole)
        workspace = _empty(max(need, 1), torch.uint8, q.device, stream, output=False)
    ws = workspace.numel() if isinstance(workspace, _Tensor) else 0
    (pq, pb, pt, pl, pv, po, pw), s = _args(stream, (
        ("q", q, dq, dt), ("bounds", bounds, (cache.K.shape[0], H, 2, dh), dt), ("table", table, (B, W), torch.int32),
        ("lens", lens, (B,), torch.int32), ("visible", visible, (B, Tq), torch.int32),
        ("sel", out, (B, Tq, H, int(n_sel)), torch.int32), ("workspace", workspace, (ws,), torch.uint8)), cache)
    _check("rolesub_select_pages", load().rolesub_select_pages(
        cache.desc(), _CODES[dt], B, Hq, Tq, pq, sq, pb, pt, W, pl, pv, int(max_len), int(n_sel), int(first), int(recent), po,
        pw, ws, s))
    return out


def attend_selected_workspace_size(cache: PagedCache, B, Hq, Tq, n_sel) -> int:
    return load().rolesub_attend_selected_workspace_size(ctypes.byref(cache._desc), B, Hq, Tq, n_sel)


def attend_selected(q, cache: PagedCache, table, lens, sel, R=None, scale: float = 0.0, visible=None, workspace=None,
                    out_dtype=None, out=None, stream=None):
    """attend_paged over the tokens of the listed pages only: sel [B,Tq,H,n_sel] int32 for
    each query and key head, in any order, -1 for none. Returns [B,Tq,Hq,dh]."""
    H, dh, dt = cache.H, cache.dh, cache.dtype
    shape, sq, dq = _operand("q", q, None, dh, dt)
    B, Tq, Hq, _ = shape
    W = _width(table)
    n = sel.shape[3] if isinstance(sel, _Tensor) and sel.dim() == 4 else None
    if n is None:
        _need("sel", sel, (B, Tq, H, None), torch.int32)
        raise TypeError("sel: expected a torch tensor, got None")
    o = _empty(shape, out_dtype or dt, q.device, stream) if out is None else out
    odt = o.dtype if isinstance(o, _Tensor) and o.dtype in _CODES else _FLOATS
    if workspace is None:
        need = attend_selected_workspace_size(cache, B, Hq, Tq, n)
        workspace = _empty(max(need, 1), torch.uint8, q.device, stream, output=False)
    ws = workspace.numel() if isinstance(workspace, _Tensor) else 0
    (pq, pt, pl, ps, pR, pv, po, pw), s = _args(stream, (
        ("q", q, dq, dt), ("table", table, (B, W), torch.int32), ("lens", lens, (B,), torch.int32),
        ("sel", sel, (B, Tq, H, n), torch.int32), ("R", R, (H, dh, dh), dt), ("visible", visible, (B, Tq), torch.int32),
        ("out", o, shape, odt), ("workspace", workspace, (ws,), torch.uint8)), cache)
    _check("rolesub_attend_selected", load().rolesub_attend_selected(
        cache.desc(), _CODES[dt], B, Hq, Tq, pq, sq, pt, W, pl, pv, ps, n, pR, float(scale), po, _CODES[odt], pw, ws, s))
    return o
