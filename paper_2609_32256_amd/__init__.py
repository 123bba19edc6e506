"""Python binding of liblam (include/lam.h) -- argument marshalling only.

Every step of the hot path runs in the HIP library; this module only turns
torch tensors into device pointers and sizes, calls the C ABI through ctypes,
and turns status codes into exceptions.  torch provides device memory and the
current stream; nothing here computes on the CPU.  If the library has not been
built (``python paper_2609_32256_amd/build.py``) importing this module fails.

    import torch, paper_2609_32256_amd as lam
    codes, p = lam.quantize(x, eps=1e-3)            # Q_eps, packed b-bit codes
    xh = lam.dequantize(codes, p)
    s = lam.Store(dim=768, tau=0.95, capacity=1 << 20)
    rep, stats = s.ingest(x_batch)                 # greedy near-duplicate test
    s.quantize(eps=1e-3)
    scores, ids, bound = s.score_topk(q, k=10)
    s.score_topk_certified(q, k=10)                # + rank-invariance flags
    s.block_encode(); s.score_topk_blocks(q, 10)   # per-block codec of the codes
    lam.removal_ceiling(x, tau=0.95)               # greedy at delta and at 2 delta
    b = lam.Store(768, 0.95, 1 << 20, eps_band=0.2 / 768 ** 0.5, band_width=4)
                                                   # banded candidates over Q_eps codes
    pages = lam.kv_pages(4096, kv_heads=8, head_dim=128)   # the model's key/value cache, in 4 bits
    lam.kv_append(k, v, pages, table, lengths)     # rows quantized into it
    o = lam.kv_attend(q, pages, table, lengths, weights=w)  # attention; what each token received
    lam.kv_evict(pages, table, lengths, w, budget, 128)     # back to the budget
    f, amplitude = lam.rotary_frequencies(128)     # rotation by position, with a norm of each head where gains are given
    q, k = lam.kv_rotate(q, f, positions, k=k)
    q = lam.kv_rotate_append(q, k, v, pages, table, lengths, f, q_norm=gq, k_norm=gk)   # and into the cache
"""
from __future__ import annotations

import ctypes
import os
import struct
import torch  # noqa: F401  (loads the HIP runtime that liblam then shares)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblam.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2609_32256_amd/build.py`")

_lib = ctypes.CDLL(LIB_PATH)

STATUS = {0: "LAM_OK", 1: "LAM_EINVAL", 2: "LAM_ERANGE", 3: "LAM_ENOMEM", 4: "LAM_ECAPACITY",
          5: "LAM_EDEVICE", 6: "LAM_ESTATE"}
PACK_BITS, PACK_BYTES = 0, 1
_MODES = {"bits": PACK_BITS, "bytes": PACK_BYTES}


class LamError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status
        self.name = STATUS.get(status, str(status))


class QParams(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_double), ("step", ctypes.c_double), ("absmax", ctypes.c_float),
                ("bits", ctypes.c_int32), ("mode", ctypes.c_int32), ("max_code", ctypes.c_int32),
                ("n", ctypes.c_int64), ("code_bytes", ctypes.c_uint64)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


class IngestStats(ctypes.Structure):
    _fields_ = [("n_in", ctypes.c_int64), ("n_kept", ctypes.c_int64), ("n_dropped", ctypes.c_int64),
                ("store_size", ctypes.c_int64), ("n_ambiguous_pairs", ctypes.c_int64),
                ("n_exact_escalations", ctypes.c_int64), ("delta_hat_call", ctypes.c_double),
                ("delta_hat_run", ctypes.c_double), ("min_margin_d2", ctypes.c_double)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


class StoreInfo(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int64), ("capacity", ctypes.c_int64), ("n_seen", ctypes.c_int64),
                ("dim", ctypes.c_int32), ("quantized", ctypes.c_int32), ("tau", ctypes.c_double),
                ("delta_hat_run", ctypes.c_double), ("q", QParams)]


_P = ctypes.c_void_p
_I64 = ctypes.c_int64
class BlockStats(ctypes.Structure):
    _fields_ = [("rows", _I64), ("blocks", _I64), ("data_bytes", ctypes.c_uint64), ("meta_bytes", ctypes.c_uint64),
                ("total_bytes", ctypes.c_uint64), ("bits_per_code", ctypes.c_double), ("plain_bits", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("codec_ratio", ctypes.c_double), ("composite_ratio", ctypes.c_double)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_ if f != "pad"}


# lam_kv_view and lam_kv_slots as the bytes of the C structs: packing them takes a
# third of the time that filling a ctypes.Structure does, on calls of some microseconds.
_KV_VIEW = struct.Struct("@PqPqPPqiiiiii")
_KV_SLOTS = struct.Struct("@Pqqi4x")
# lam_rotary and lam_heads
_ROTARY = struct.Struct("@Piid")
_HEADS = struct.Struct("@PqqPqqPii")


class CeilingStats(ctypes.Structure):
    _fields_ = [("n", _I64), ("kept", _I64), ("kept_2delta", _I64), ("tau", ctypes.c_double),
                ("tau_2delta", ctypes.c_double), ("removal", ctypes.c_double), ("ceiling", ctypes.c_double),
                ("frac_of_ceiling", ctypes.c_double), ("bits_lo", ctypes.c_double), ("bits_hi", ctypes.c_double),
                ("delta_hat", ctypes.c_double), ("delta_hat_2delta", ctypes.c_double)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


_SIGS = {
    "lam_abi_version": ([], ctypes.c_int),
    "lam_status_name": ([ctypes.c_int], ctypes.c_char_p),
    "lam_last_error": ([], ctypes.c_char_p),
    "lam_ctx_create": ([ctypes.c_int, _P, ctypes.POINTER(_P)], ctypes.c_int),
    "lam_ctx_destroy": ([_P], None),
    "lam_ctx_synchronize": ([_P], ctypes.c_int),
    "lam_ctx_profile": ([_P, ctypes.c_int], ctypes.c_int),
    "lam_ctx_profile_only": ([_P, ctypes.c_char_p], ctypes.c_int),
    "lam_ctx_set_screen_tile": ([_P, ctypes.c_int], ctypes.c_int),
    "lam_ctx_profile_reset": ([_P], ctypes.c_int),
    "lam_ctx_profile_read": ([_P, ctypes.c_char_p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_I64)],
                             ctypes.c_int),
    "lam_qeps_plan": ([ctypes.c_double, ctypes.c_float, ctypes.c_int, _I64, ctypes.POINTER(QParams)], ctypes.c_int),
    "lam_quantize": ([_P, _P, _I64, ctypes.c_double, ctypes.c_float, ctypes.c_int, _P, ctypes.c_uint64,
                      ctypes.POINTER(QParams)], ctypes.c_int),
    "lam_quantize_async": ([_P, _P, _I64, ctypes.c_double, ctypes.c_float, ctypes.c_int, _P, ctypes.c_uint64, _P,
                            ctypes.POINTER(QParams)], ctypes.c_int),
    "lam_dequantize": ([_P, _P, ctypes.POINTER(QParams), _P], ctypes.c_int),
    "lam_store_create": ([_P, ctypes.c_int32, ctypes.c_double, _I64, ctypes.POINTER(_P)], ctypes.c_int),
    "lam_store_create_banded": ([_P, ctypes.c_int32, ctypes.c_double, _I64, ctypes.c_double, ctypes.c_int32,
                                 ctypes.POINTER(_P)], ctypes.c_int),
    "lam_store_destroy": ([_P], None),
    "lam_store_get_info": ([_P, ctypes.POINTER(StoreInfo)], ctypes.c_int),
    "lam_dedup_ingest": ([_P, _P, _P, _I64, _P, _P, ctypes.POINTER(IngestStats)], ctypes.c_int),
    "lam_store_quantize": ([_P, _P, ctypes.c_double, ctypes.c_float, ctypes.c_int, ctypes.POINTER(QParams)],
                           ctypes.c_int),
    "lam_store_clear": ([_P, _P], ctypes.c_int),
    "lam_store_dequantize": ([_P, _P, _P], ctypes.c_int),
    "lam_store_export": ([_P, _P, _P, _P, ctypes.c_uint64], ctypes.c_int),
    "lam_score_topk_certified": ([_P, _P, _P, _I64, ctypes.c_int32, _P, _P, _P, _P, _P], ctypes.c_int),
    "lam_store_block_encode": ([_P, _P, ctypes.POINTER(BlockStats)], ctypes.c_int),
    "lam_store_block_decode": ([_P, _P, _P], ctypes.c_int),
    "lam_store_block_export": ([_P, _P, _P, _P, _P, ctypes.c_uint64], ctypes.c_int),
    "lam_score_topk_blocks": ([_P, _P, _P, _I64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "lam_removal_ceiling": ([_P, _P, _I64, ctypes.c_int32, ctypes.c_double, _I64, ctypes.POINTER(CeilingStats)],
                            ctypes.c_int),
    "lam_score_topk": ([_P, _P, _P, _I64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "lam_score_topk_noalloc": ([_P, _P, _P, _I64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "lam_kv_page_bytes": ([ctypes.c_int32, ctypes.c_int32], _I64),
    "lam_kv_append": ([_P, _P, _P, _I64, _I64, _P, _I64, _I64, _P,
                       _P, _P, _P], ctypes.c_int),
    "lam_rotary_frequencies": ([ctypes.c_int32, ctypes.c_double, ctypes.c_int, ctypes.c_double, ctypes.c_double,
                                ctypes.c_double, ctypes.c_double, _P, _P], ctypes.c_int),
    "lam_kv_rotate": ([_P, _P, _P, _P, _I64, ctypes.c_int32, ctypes.c_int32, _P, ctypes.c_double, ctypes.c_int32],
                      ctypes.c_int),
    "lam_kv_rotate_append": ([_P, _P, _P, _P, _P, _P, _I64, _I64, _P, _P, _P, ctypes.c_double, ctypes.c_int32, _P],
                             ctypes.c_int),
    "lam_kv_read": ([_P, _P, _P, _P], ctypes.c_int),
    "lam_kv_attend": ([_P, _P, _P, _I64, _I64, ctypes.c_int32, ctypes.c_double, ctypes.c_int, _I64,
                       _P, _P, _P, _P], ctypes.c_int),
    "lam_kv_attend_window": ([_P, _P, _P, _I64, _I64, ctypes.c_int32, ctypes.c_double, ctypes.c_int, _I64, _I64, _I64,
                              _P, _P, _P, _P], ctypes.c_int),
    "lam_kv_evict": ([_P, _P, _P, _P, ctypes.c_int32,
                      ctypes.c_int32, ctypes.c_int32, _P, _P, _P, _P],
                     ctypes.c_int),
    "lam_triad": ([_P, _P, _P, _P, _I64, ctypes.c_float], ctypes.c_int),
}
for _name, (_args, _res) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res

EXPORTED = tuple(_SIGS)


def _check(status: int):
    if status != 0:
        raise LamError(status, _lib.lam_last_error().decode(errors="replace"))


def abi_version() -> int:
    return _lib.lam_abi_version()


def removal_ceiling(x: torch.Tensor, tau: float, batch: int = 4096, ctx: Context | None = None) -> dict:
    """Theorem "removal ceiling" / Corollary "measured bracket": greedy over the
    rows of x at tau and at 4 tau - 3 (radius 2 delta).  Returns the counts,
    the attained removal, the ceiling and the bracket log2|R(2 delta)| <=
    H_delta <= log2|R(delta)|."""
    ctx = ctx or default_context()
    x = _dev_tensor(x, torch.float32, "x")
    if x.dim() != 2:
        raise ValueError("x must be (n, dim)")
    out = CeilingStats()
    _check(_lib.lam_removal_ceiling(ctx.handle, _ptr(x), x.shape[0], x.shape[1], float(tau), int(batch),
                                    ctypes.byref(out)))
    return out.as_dict()


def qeps_plan(eps: float, absmax: float, mode: str = "bits", n: int = 0) -> QParams:
    """Width plan of Q_eps (host only)."""
    p = QParams()
    _check(_lib.lam_qeps_plan(float(eps), float(absmax), _MODES[mode], int(n), ctypes.byref(p)))
    return p


# ---------------------------------------------------------------- contexts
class Context:
    """A liblam context bound to one device and one HIP stream."""

    def __init__(self, device: int | None = None, stream: "torch.cuda.Stream | None" = None):
        if not torch.cuda.is_available():
            raise RuntimeError("liblam needs a GPU (torch.cuda.is_available() is False)")
        self.device = torch.cuda.current_device() if device is None else int(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = _P()
        _check(_lib.lam_ctx_create(self.device, _P(self.stream.cuda_stream), ctypes.byref(h)))
        self._h = h

    @property
    def handle(self):
        return self._h

    def synchronize(self):
        _check(_lib.lam_ctx_synchronize(self._h))

    def profile(self, enable: bool = True):
        _check(_lib.lam_ctx_profile(self._h, 1 if enable else 0))

    def profile_only(self, kernel: str | None):
        """Time only the launches of the kernel names in a comma-separated list
        (None: every kernel)."""
        _check(_lib.lam_ctx_profile_only(self._h, (kernel or "").encode()))

    def profile_reset(self):
        _check(_lib.lam_ctx_profile_reset(self._h))

    def set_screen_tile(self, policy):
        """The screen's tile: "auto" (by launch size), "small" (128 x 128) or
        "large" (256 x 256).  Decisions are the same."""
        code = {"auto": 0, "small": 1, "large": 2}.get(policy, policy)
        _check(_lib.lam_ctx_set_screen_tile(self._h, int(code)))

    def profile_read(self, kernel: str):
        ms, n = ctypes.c_double(), _I64()
        _check(_lib.lam_ctx_profile_read(self._h, kernel.encode(), ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def close(self):
        if getattr(self, "_h", None):
            _lib.lam_ctx_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_default_ctx: dict = {}


def default_context() -> Context:
    # (current_device() without its test that the GPU is initialised, which the first context did)
    dev = torch._C._cuda_getDevice() if _default_ctx else torch.cuda.current_device()
    key = (dev, torch._C._cuda_getCurrentRawStream(dev))   # the handle of current_stream(dev), without the object
    c = _default_ctx.get(key)
    if c is None:
        c = _default_ctx[key] = Context(dev)
    return c


def _ptr(t: torch.Tensor | None):
    return _P(t.data_ptr()) if t is not None else _P(None)


def _dev_tensor(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return t.contiguous()


# ---------------------------------------------------------------- Q_eps
def quantize(x: torch.Tensor, eps: float, absmax: float | None = None, mode: str = "bits",
             out: torch.Tensor | None = None, ctx: Context | None = None):
    """Q_eps of a float32 tensor: returns (codes uint32-words tensor viewed as
    int32, QParams).  absmax=None measures max|x| on the device."""
    ctx = ctx or default_context()
    x = _dev_tensor(x, torch.float32, "x").reshape(-1)
    n = x.numel()
    a = 0.0 if absmax is None else float(absmax)
    if out is None:
        plan_a = a if absmax is not None else 0.0
        # capacity for the widest code the plan could pick (32 bits) if absmax is measured
        words = (n * 32 + 31) // 32 if absmax is None else (n * qeps_plan(eps, plan_a, mode, n).bits + 31) // 32
        out = torch.empty(max(1, words), dtype=torch.int32, device=x.device)
    p = QParams()
    _check(_lib.lam_quantize(ctx.handle, _ptr(x), n, float(eps), a, _MODES[mode], _ptr(out),
                             out.numel() * 4, ctypes.byref(p)))
    return out[: p.code_bytes // 4], p


def quantize_async(x: torch.Tensor, eps: float, absmax: float, status: torch.Tensor, mode: str = "bits",
                   out: torch.Tensor | None = None, ctx: Context | None = None):
    """Q_eps that does not wait for the device (lam_quantize_async): returns
    (codes, QParams) once the encode is queued; the encode adds a positive
    count to status[0] if any element is NaN/Inf and to status[1] if any is
    above absmax (status: a contiguous int32 device tensor of at least 2
    entries that the caller clears)."""
    ctx = ctx or default_context()
    x = _dev_tensor(x, torch.float32, "x").reshape(-1)
    if not isinstance(status, torch.Tensor) or not status.is_cuda or status.dtype != torch.int32 \
            or not status.is_contiguous() or status.numel() < 2:
        raise ValueError("status must be a contiguous int32 device tensor of at least 2 entries")
    n = x.numel()
    if out is None:
        out = torch.empty(max(1, (n * qeps_plan(eps, absmax, mode, n).bits + 31) // 32), dtype=torch.int32,
                          device=x.device)
    p = QParams()
    _check(_lib.lam_quantize_async(ctx.handle, _ptr(x), n, float(eps), float(absmax), _MODES[mode], _ptr(out),
                                   out.numel() * 4, _ptr(status), ctypes.byref(p)))
    return out[: p.code_bytes // 4], p


def dequantize(codes: torch.Tensor, p: QParams, out: torch.Tensor | None = None,
               ctx: Context | None = None) -> torch.Tensor:
    ctx = ctx or default_context()
    codes = _dev_tensor(codes, torch.int32, "codes")
    if codes.numel() * 4 < p.code_bytes:
        raise ValueError("codes tensor shorter than params.code_bytes")
    if out is None:
        out = torch.empty(p.n, dtype=torch.float32, device=codes.device)
    _check(_lib.lam_dequantize(ctx.handle, _ptr(codes), ctypes.byref(p), _ptr(out)))
    return out


def triad(a: torch.Tensor, b: torch.Tensor, c: torch.Tensor, s: float = 3.0, ctx: Context | None = None):
    """The bandwidth anchor c = a + s * b over float32 device tensors of equal
    size (lam_triad; 12 bytes moved per element)."""
    ctx = ctx or default_context()
    a = _dev_tensor(a, torch.float32, "a")
    b = _dev_tensor(b, torch.float32, "b")
    c = _dev_tensor(c, torch.float32, "c")
    if not (a.numel() == b.numel() == c.numel()):
        raise ValueError("a, b and c must have the same size")
    _check(_lib.lam_triad(ctx.handle, _ptr(a), _ptr(b), _ptr(c), a.numel(), float(s)))
    return c


# ---------------------------------------------------------------- 4-bit key/value cache
_KV_DTYPES = {torch.float16: 0, torch.bfloat16: 1}
_KV_HEADS = (64, 128, 256)
_KV_PAGES = (32, 64, 128, 256, 512, 1024)


def _kv_int(x, name):
    """A Python integer as a C int32, of which ctypes would take the low 32 bits."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} must be a 32-bit integer, got {x}")
    return x


def kv_pages(n_pages: int, kv_heads: int, head_dim: int, page_size: int = 64, device=None) -> torch.Tensor:
    """An empty pool of cache pages: uint8 (n_pages, kv_heads, bytes of a head's
    page).  head_dim 64, 128 or 256; page_size a power of two, 32 to 1024."""
    size = _lib.lam_kv_page_bytes(_kv_int(head_dim, "head_dim"), _kv_int(page_size, "page_size"))
    if size < 0:
        raise ValueError("head_dim must be 64, 128 or 256 and page_size a power of two from 32 to 1024")
    return torch.zeros((int(n_pages), int(kv_heads), size), dtype=torch.uint8, device="cuda" if device is None else device)


def _kv_tensor(t, dtype, dims, name, dev):
    """Checks of a tensor argument (dev: the device's index)."""
    if isinstance(t, torch.Tensor) and t.get_device() == dev and t.dtype is dtype and t.dim() == dims:
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the context on cuda:{dev}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must have {dims} dimensions")


def _kv_view(dev, pages, table, lengths, starts, rows, head_dim, dtype):
    """(lam_kv_view, sequences, kv_heads, tensors to hold until the launch is queued)
    of a call.  Index tensors whose last axis is not contiguous are copied."""
    if not (isinstance(pages, torch.Tensor) and isinstance(table, torch.Tensor) and isinstance(lengths, torch.Tensor)
            and pages.get_device() == dev and table.get_device() == dev and lengths.get_device() == dev
            and pages.dtype is torch.uint8 and table.dtype is torch.int32 and lengths.dtype is torch.int32
            and pages.dim() == 3 and table.dim() == 2 and lengths.dim() == 1):
        _kv_tensor(pages, torch.uint8, 3, "pages", dev)
        _kv_tensor(table, torch.int32, 2, "table", dev)
        _kv_tensor(lengths, torch.int32, 1, "lengths", dev)
    if not pages.is_contiguous():
        raise ValueError("pages must be contiguous")
    n_pages, heads, size = pages.shape
    page_size, rest = divmod(size, head_dim + head_dim // 16) if head_dim > 0 else (0, 1)
    if rest or head_dim not in _KV_HEADS or page_size not in _KV_PAGES:
        raise ValueError(f"pages of {size} bytes a head do not hold heads of {head_dim} channels")
    (n, cols), (stride, step) = table.shape, table.stride()
    if step != 1 and cols > 1 or stride < cols:
        table = table.contiguous()
        stride = table.stride(0)
    lengths = lengths.contiguous()
    if lengths.numel() != n:
        raise ValueError("table and lengths must have a row for each sequence")
    if starts is not None:
        _kv_tensor(starts, torch.int32, 1, "starts", dev)
        starts = starts.contiguous()
        if starts.numel() != n + 1:
            raise ValueError("starts must have an entry for each sequence and one more")
    elif rows and (n == 0 or rows % n):
        raise ValueError("without starts every sequence has the same number of rows")
    v = _KV_VIEW.pack(pages.data_ptr(), n_pages, table.data_ptr(), stride, lengths.data_ptr(),
                      0 if starts is None else starts.data_ptr(), rows, n, cols, heads, head_dim, page_size,
                      _KV_DTYPES[dtype])
    return v, n, heads, (table, lengths, starts)


def _kv_graphless(t, name):
    """Refuses a tensor whose gradient the call would drop: the cache's operators have none."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which the 4-bit cache's operators do not have: "
                         "call them under torch.no_grad() or with a detached tensor")


def _kv_elsewhere(ctx):
    """Whether a context's stream is not the current one: copies and outputs of its
    calls are then made on its own."""
    return ctx.stream.cuda_stream != torch._C._cuda_getCurrentRawStream(ctx.device)


def _kv_rows(t, heads, name, dev):
    """(rows, heads, head_dim) in float16 or bfloat16, channels contiguous."""
    if isinstance(t, torch.Tensor) and t.get_device() == dev and t.dtype in _KV_DTYPES and not t.requires_grad \
            and t.dim() == 3 and (heads is None or t.shape[1] == heads):
        row, head, step = t.stride()
        return t if step == 1 and row > 0 and head > 0 else t.contiguous()
    if not isinstance(t, torch.Tensor) or t.dtype not in _KV_DTYPES:
        raise TypeError(f"{name} must be a float16 or bfloat16 tensor")
    _kv_tensor(t, t.dtype, 3, name, dev)
    if heads is not None and t.shape[1] != heads:
        raise ValueError(f"{name} must have {heads} heads")
    if t.requires_grad:
        _kv_graphless(t, name)
    row, head, step = t.stride()
    return t if step == 1 and row > 0 and head > 0 else t.contiguous()


def _kv_slots(t, dtype, n, heads, name, dev, shared=False, copy=False):
    """(lam_kv_slots, tensor to hold) of a value per cached token: (sequences, heads or
    1 where shared, slots).  A tensor whose slots are not contiguous is copied where
    the library only reads it."""
    if t is None:
        return None, None
    _kv_tensor(t, dtype, 3, name, dev)
    seqs, own, cols = t.shape
    if seqs != n or not (own == heads or (shared and own == 1)):
        raise ValueError(f"{name} must be (sequences, heads, slots)")
    if t.requires_grad:
        _kv_graphless(t, name)
    if cols > 1 and t.stride(2) != 1:
        if not copy:
            raise ValueError(f"the slots of {name} must be contiguous")
        t = t.contiguous()
    seq, head, _ = t.stride()
    return _KV_SLOTS.pack(t.data_ptr(), seq, 0 if own == 1 else head, cols), t


def _kv_first(first, n, dev):
    if first is None:
        return None
    _kv_tensor(first, torch.int32, 1, "first", dev)
    if first.numel() != n:
        raise ValueError("first must have an entry for each sequence")
    return first.contiguous()


def _kv_status(status, dev):
    if status is None:
        return
    _kv_tensor(status, torch.int32, 1, "status", dev)
    if not status.is_contiguous() or status.numel() < 3:
        raise ValueError("status must be a contiguous int32 tensor of at least 3 entries")


def kv_append(k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
              starts: torch.Tensor | None = None, weights: torch.Tensor | None = None,
              positions: torch.Tensor | None = None, first: torch.Tensor | None = None,
              status: torch.Tensor | None = None, ctx: Context | None = None) -> None:
    """Quantize rows of keys and values (rows, kv_heads, head_dim) into the last
    tokens of their sequences (lam_kv_append).  lengths counts the new tokens in;
    starts gives each sequence's rows, None: equally many each.  weights of the
    new tokens become 0, positions first[s], first[s] + 1, ...; status: int32
    tensor of 3, counts of non-finite, out-of-range and misplaced input."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_append(k, v, pages, table, lengths, starts, weights, positions, first, status, ctx)
    dev = ctx.device
    k = _kv_rows(k, None, "k", dev)
    v = _kv_rows(v, k.shape[1], "v", dev)
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("k and v must have the same shape and dtype")
    rows, own, head_dim = k.shape
    view, n, heads, hold = _kv_view(dev, pages, table, lengths, starts, rows, head_dim, k.dtype)
    if own != heads:
        raise ValueError(f"k must have {heads} heads")
    w, _ = _kv_slots(weights, torch.float32, n, heads, "weights", dev)
    p, _ = _kv_slots(positions, torch.int32, n, heads, "positions", dev)
    first = _kv_first(first, n, dev)
    _kv_status(status, dev)
    _check(_lib.lam_kv_append(ctx.handle, view, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0),
                              v.stride(1), w, p, None if first is None else first.data_ptr(),
                              None if status is None else status.data_ptr()))


_ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
_ROTARY_SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}
_CONTIGUOUS = torch.contiguous_format


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                       length: float = 0.0, low: float = 1.0, high: float = 32.0, device=None):
    """(frequencies, amplitude) of a rotation of the first rotary_dim channels (lam_rotary_frequencies):
    float64 (rotary_dim / 2,), radians a position, on `device` (the current GPU by default).  scaling,
    for contexts `factor` times the trained `length`: "linear", "base" or "parts" (pairs of `high` or more
    turns over `length` as they are, of `low` or fewer slower by factor; the amplitude is then 0.1 ln(factor) + 1)."""
    pairs, rest = divmod(_kv_int(rotary_dim, "rotary_dim"), 2)
    if rest or pairs < 0:
        raise ValueError("rotary_dim must be even and not negative")
    if scaling not in _ROTARY_SCALINGS:
        raise ValueError(f"scaling must be one of {list(_ROTARY_SCALINGS)}")
    out, amplitude = (ctypes.c_double * max(pairs, 1))(), ctypes.c_double()
    _check(_lib.lam_rotary_frequencies(pairs, float(base), _ROTARY_SCALINGS[scaling], float(factor), float(length),
                                       float(low), float(high), out, ctypes.addressof(amplitude)))
    return torch.tensor(out[:pairs], dtype=torch.float64, device="cuda" if device is None else device), amplitude.value


def _kv_rotary(frequencies, layout, amplitude, dev):
    """(lam_rotary, tensor to hold) of a call."""
    if layout not in _ROTARY_LAYOUTS:
        raise ValueError(f"layout must be one of {list(_ROTARY_LAYOUTS)}")
    if frequencies is None:
        return _ROTARY.pack(0, 0, 0, 1.0), None
    _kv_tensor(frequencies, torch.float64, 1, "frequencies", dev)
    if frequencies.requires_grad:
        _kv_graphless(frequencies, "frequencies")
    f = frequencies.contiguous()
    return _ROTARY.pack(f.data_ptr(), f.numel(), _ROTARY_LAYOUTS[layout], float(amplitude)), f


def _kv_heads(x, gain, out, name, dev):
    """(lam_heads, the rows as they are taken, result, tensor to hold) of rows that are normed and
    turned; out: True for a new result, False for none."""
    if not (isinstance(x, torch.Tensor) and x.get_device() == dev and x.dtype in _KV_DTYPES and x.dim() == 3
            and not x.requires_grad):
        x = _kv_rows(x, None, name, dev)
    row, head, step = x.stride()
    if step != 1 or row <= 0 or head <= 0:
        x = x.contiguous()
        row, head, _ = x.stride()
    rows, heads, head_dim = x.shape
    dtype = x.dtype
    g, g_type = 0, 2
    if gain is not None:
        own = gain.dtype if isinstance(gain, torch.Tensor) else None
        if own is dtype:
            g_type = _KV_DTYPES[own]
        elif own is not torch.float32:
            raise TypeError(f"{name}_norm must be a tensor of float32 or of {name}'s type")
        if gain.get_device() != dev or gain.dim() != 1 or gain.numel() != head_dim:
            _kv_tensor(gain, own, 1, name + "_norm", dev)
            raise ValueError(f"{name}_norm must have an entry for each of the {head_dim} channels")
        if gain.requires_grad:
            _kv_graphless(gain, name + "_norm")
        gain = gain.contiguous()
        g = gain.data_ptr()
    if out is True:
        out = torch.empty_like(x, memory_format=_CONTIGUOUS)
        return _HEADS.pack(x.data_ptr(), row, head, out.data_ptr(), heads * head_dim, head_dim, g, g_type, heads), x, out, gain
    if out is False:
        return _HEADS.pack(x.data_ptr(), row, head, 0, 0, 0, g, g_type, heads), x, None, gain
    _kv_tensor(out, dtype, 3, name + "'s out", dev)
    y_row, y_head, step = out.stride()
    if out.shape != x.shape or step != 1:
        raise ValueError(f"{name}'s out must be of {name}'s shape with its channels contiguous")
    if out.requires_grad:
        _kv_graphless(out, name + "'s out")
    return _HEADS.pack(x.data_ptr(), row, head, out.data_ptr(), y_row, y_head, g, g_type, heads), x, out, gain


def kv_rotate(q: torch.Tensor, frequencies: torch.Tensor | None, positions: torch.Tensor | None = None,
              k: torch.Tensor | None = None, layout: str = "half", amplitude: float = 1.0,
              q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6,
              norm_dim: int | None = None, out=None, ctx: Context | None = None):
    """Norm the heads of rows of queries (rows, heads, head_dim), and of keys, and turn their channel
    pairs by position times frequency (lam_kv_rotate): layout "half" (channels i and i + pairs) or
    "interleaved" (2 i and 2 i + 1); frequencies (float64, radians a position) of up to head_dim / 2
    pairs, None: none is turned.  positions: int32, of each row.  q_norm, k_norm: gains of an RMS norm
    (float32 or q's type: head_dim), None: no norm; norm_dim: the channels of the mean, head_dim by default.
    Returns q's result, with k (q's, k's).  out: q's result or (q's, k's) to write to, which may be q
    and k themselves.  There is no gradient: tensors that require one are refused outside
    torch.no_grad()."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_rotate(q, frequencies, positions, k, layout, amplitude, q_norm, k_norm, eps, norm_dim, out, ctx)
    dev = ctx.device
    if k is None:
        if isinstance(out, (tuple, list)):
            out, = out
        k_out = None
    elif out is None:
        k_out = None
    elif not isinstance(out, (tuple, list)):
        raise TypeError("out must be (q's result, k's result)")
    else:
        out, k_out = out
    qh, q, out, hold_q = _kv_heads(q, q_norm, True if out is None else out, "q", dev)
    rows, _, head_dim = q.shape
    r, hold = _kv_rotary(frequencies, layout, amplitude, dev)
    if positions is not None:
        _kv_tensor(positions, torch.int32, 1, "positions", dev)
        positions = positions.contiguous()
        if positions.numel() != rows:
            raise ValueError("positions must have an entry for each row")
    elif hold is not None and hold.numel() and rows:
        raise ValueError("a rotation needs positions")
    kh = None
    if k is not None:
        kh, k, k_out, hold_k = _kv_heads(k, k_norm, True if k_out is None else k_out, "k", dev)
        if k.dtype != q.dtype or k.shape[0] != rows or k.shape[2] != head_dim:
            raise ValueError("k must have q's rows, channels and type")
    _check(_lib.lam_kv_rotate(ctx.handle, r, qh, kh, rows, head_dim, _KV_DTYPES[q.dtype],
                              None if positions is None else positions.data_ptr(), float(eps),
                              0 if norm_dim is None else _kv_norm_dim(norm_dim)))
    return out if k is None else (out, k_out)


def _kv_norm_dim(n):
    n = _kv_int(n, "norm_dim")
    if n < 1:
        raise ValueError("norm_dim must be at least 1")
    return n


def kv_rotate_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, table: torch.Tensor,
                     lengths: torch.Tensor, frequencies: torch.Tensor | None, starts: torch.Tensor | None = None,
                     first: torch.Tensor | None = None, layout: str = "half", amplitude: float = 1.0,
                     q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6,
                     norm_dim: int | None = None, weights: torch.Tensor | None = None,
                     positions: torch.Tensor | None = None, status: torch.Tensor | None = None,
                     out: torch.Tensor | None = None, ctx: Context | None = None):
    """kv_append with the norm and the rotation of kv_rotate on the way (lam_kv_rotate_append): keys
    are normed, turned and quantized, values quantized, and q (rows, q_heads, head_dim; or None), normed and
    turned, is returned (in out, which may be q itself).  Row i of sequence s has the position
    first[s] + i, without first its token's slot; positions (a value per cached token) get it."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_rotate_append(q, k, v, pages, table, lengths, frequencies, starts, first, layout, amplitude,
                                    q_norm, k_norm, eps, norm_dim, weights, positions, status, out, ctx)
    dev = ctx.device
    kh, k, _, hold_k = _kv_heads(k, k_norm, False, "k", dev)
    rows, own, head_dim = k.shape
    v = _kv_rows(v, own, "v", dev)
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("k and v must have the same shape and dtype")
    view, n, heads, hold = _kv_view(dev, pages, table, lengths, starts, rows, head_dim, k.dtype)
    if own != heads:
        raise ValueError(f"k must have {heads} heads")
    r, hold_f = _kv_rotary(frequencies, layout, amplitude, dev)
    qh = None
    if q is not None:
        qh, q, out, hold_q = _kv_heads(q, q_norm, True if out is None else out, "q", dev)
        if q.dtype != k.dtype or q.shape[0] != rows or q.shape[2] != head_dim:
            raise ValueError("q must have k's rows, channels and type")
    elif out is not None:
        raise ValueError("out without q")
    w, _ = _kv_slots(weights, torch.float32, n, heads, "weights", dev)
    p, _ = _kv_slots(positions, torch.int32, n, heads, "positions", dev)
    first = _kv_first(first, n, dev)
    _kv_status(status, dev)
    _check(_lib.lam_kv_rotate_append(ctx.handle, view, r, qh, kh, v.data_ptr(), v.stride(0), v.stride(1), w, p,
                                     None if first is None else first.data_ptr(), float(eps),
                                     0 if norm_dim is None else _kv_norm_dim(norm_dim),
                                     None if status is None else status.data_ptr()))
    return out


def kv_read(pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, rows: int, head_dim: int,
            dtype: torch.dtype = torch.bfloat16, starts: torch.Tensor | None = None, ctx: Context | None = None):
    """The values the cache holds for the last tokens of the sequences, addressed
    as by kv_append: (k, v), each (rows, kv_heads, head_dim) (lam_kv_read)."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_read(pages, table, lengths, rows, head_dim, dtype, starts, ctx)
    if dtype not in _KV_DTYPES:
        raise TypeError("dtype must be float16 or bfloat16")
    view, _, heads, hold = _kv_view(ctx.device, pages, table, lengths, starts, int(rows), int(head_dim), dtype)
    k = pages.new_empty((int(rows), heads, int(head_dim)), dtype=dtype)
    v = torch.empty_like(k)
    _check(_lib.lam_kv_read(ctx.handle, view, k.data_ptr(), v.data_ptr()))
    return k, v


def _kv_count(x, name, least):
    """A Python integer as a C int64 of at least `least`."""
    x = int(x)
    if not least <= x < 1 << 63:
        raise ValueError(f"{name} must be a 64-bit integer of at least {least}, got {x}")
    return x


def kv_attend(q: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
              starts: torch.Tensor | None = None, causal: bool = True, scale: float | None = None,
              mask: torch.Tensor | None = None, weights: torch.Tensor | None = None, max_length: int | None = None,
              out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
              ctx: Context | None = None, window: int | None = None, sinks: int = 0) -> torch.Tensor:
    """Attention of the sequences' last tokens over the cache (lam_kv_attend): q
    and the result (rows, q_heads, head_dim).  scale: 1 / sqrt(head_dim) by
    default.  mask (bool or uint8: sequences, kv_heads or 1, slots) leaves cached
    tokens out; weights (float32: sequences, kv_heads, slots) is added to what
    each token received; lse (float32: rows, q_heads) receives the scores' log
    sums.  Rows that see no token, those of no sequence among them, get 0 (lse -inf).
    max_length, where the caller knows a bound of lengths, sizes the launch.  With a window a row
    sees, of those tokens, the last `window` up to its own and the first `sinks` (lam_kv_attend_window);
    pages that no row sees need not be there.  out may be q
    itself, if contiguous (but for chunks with weights, which read q twice).  There is
    no gradient: tensors that require one are refused outside torch.no_grad()."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_attend(q, pages, table, lengths, starts, causal, scale, mask, weights, max_length, out, lse, ctx,
                             window, sinks)
    dev = ctx.device
    q = _kv_rows(q, None, "q", dev)
    rows, q_heads, head_dim = q.shape
    view, n, heads, hold = _kv_view(dev, pages, table, lengths, starts, rows, head_dim, q.dtype)
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    m, hold_mask = _kv_slots(mask, torch.uint8, n, heads, "mask", dev, shared=True, copy=True)
    w, _ = _kv_slots(weights, torch.float32, n, heads, "weights", dev)
    if out is None:
        out = torch.empty_like(q) if q.is_contiguous() else torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _kv_tensor(out, q.dtype, 3, "out", dev)
        if out.shape != q.shape or not out.is_contiguous():
            raise ValueError("out must be contiguous and of q's shape")
        _kv_graphless(out, "out")
    if lse is not None:
        _kv_tensor(lse, torch.float32, 2, "lse", dev)
        if lse.shape != q.shape[:2] or not lse.is_contiguous():
            raise ValueError("lse must be contiguous and (rows, q_heads)")
        _kv_graphless(lse, "lse")
    if window is not None:
        window, sinks = _kv_count(window, "window", 1), _kv_count(sinks, "sinks", 0)
    elif sinks:
        raise ValueError("sinks need a window")
    else:
        window = sinks = 0
    _check(_lib.lam_kv_attend_window(ctx.handle, view, q.data_ptr(), q.stride(0), q.stride(1), q_heads,
                                     head_dim ** -0.5 if scale is None else float(scale), 1 if causal else 0,
                                     0 if max_length is None else max(1, _kv_count(max_length, "max_length", -(1 << 63))), window, sinks, m, w,
                                     out.data_ptr(), None if lse is None else lse.data_ptr()))
    return out


def kv_evict(pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, scores: torch.Tensor, budget: int,
             head_dim: int, recent: int = 0, sinks: int = 0, positions: torch.Tensor | None = None, out=None,
             ctx: Context | None = None):
    """Bring sequences of more than `budget` tokens back to budget tokens
    (lam_kv_evict): those of the largest scores stay, the `recent` newest (by position,
    whichever slots hold them) and the `sinks` first positions whatever their scores.  Returns (kept, scores,
    positions, lengths): the old slot of each new one (sequences, kv_heads,
    budget), the new slots' scores and positions, and the new lengths.  out:
    (scores, positions or None, lengths) to write to, which may be the inputs
    (only their first budget slots are written)."""
    if ctx is None:
        ctx = default_context()
    elif _kv_elsewhere(ctx):
        with torch.cuda.stream(ctx.stream):
            return kv_evict(pages, table, lengths, scores, budget, head_dim, recent, sinks, positions, out, ctx)
    dev = ctx.device
    view, n, heads, hold = _kv_view(dev, pages, table, lengths, None, 0, int(head_dim), torch.float16)
    s, hold_s = _kv_slots(scores, torch.float32, n, heads, "scores", dev, copy=True)
    p, hold_p = _kv_slots(positions, torch.int32, n, heads, "positions", dev, copy=True)
    if s is None:
        raise TypeError("scores must be a CUDA (HIP) tensor")
    budget, recent, sinks = int(budget), int(recent), int(sinks)
    if max(budget, recent, sinks) >= 1 << 31 or min(budget, recent, sinks) < -(1 << 31):
        raise ValueError(f"budget, recent and sinks must be 32-bit integers, got {budget}, {recent}, {sinks}")
    kept = lengths.new_empty((n, heads, max(budget, 0)))
    if out is None:
        out = (torch.empty_like(kept, dtype=torch.float32), torch.empty_like(kept), torch.empty_like(hold[1]))
        so, po = (_KV_SLOTS.pack(t.data_ptr(), heads * budget, budget, budget) for t in out[:2])
    else:
        so, _ = _kv_slots(out[0], torch.float32, n, heads, "out scores", dev)
        po, _ = _kv_slots(out[1], torch.int32, n, heads, "out positions", dev)
        _kv_tensor(out[2], torch.int32, 1, "out lengths", dev)
        if out[2].numel() != n or not out[2].is_contiguous():
            raise ValueError("out lengths must be contiguous, an entry for each sequence")
    _check(_lib.lam_kv_evict(ctx.handle, view, s, p, budget, recent, sinks, kept.data_ptr(), so, po,
                             out[2].data_ptr()))
    return kept, out[0], out[1], out[2]


# ---------------------------------------------------------------- store
class Store:
    """The retained set of the greedy near-duplicate test, on one device."""

    def __init__(self, dim: int, tau: float, capacity: int, ctx: Context | None = None,
                 eps_band: float | None = None, band_width: int | None = None):
        """With eps_band and band_width the store takes its candidates from a
        band index over Q_eps codes (lam_store_create_banded); otherwise every
        retained row is screened."""
        self.ctx = ctx or default_context()
        h = _P()
        if (eps_band is None) != (band_width is None):
            raise ValueError("give both eps_band and band_width, or neither")
        if band_width is None:
            _check(_lib.lam_store_create(self.ctx.handle, int(dim), float(tau), int(capacity), ctypes.byref(h)))
        else:
            _check(_lib.lam_store_create_banded(self.ctx.handle, int(dim), float(tau), int(capacity),
                                                float(eps_band), int(band_width), ctypes.byref(h)))
        self._h = h
        self.banded = band_width is not None
        self.dim = int(dim)
        self.tau = float(tau)

    def info(self) -> StoreInfo:
        i = StoreInfo()
        _check(_lib.lam_store_get_info(self._h, ctypes.byref(i)))
        return i

    @property
    def size(self) -> int:
        return self.info().size

    def ingest(self, x: torch.Tensor, max_cos: bool = False, rep: torch.Tensor | None = None, sync: bool = True):
        """Algorithm "admit" over the rows of x (n x dim float32).  Returns
        (rep int64[n], stats dict[, max_cos float32[n]]).  With sync=False the
        call may return before the device has finished (stats is then None);
        invalid input of such a call is raised by the next call that waits
        (size, info, quantize, scoring or a synchronous ingest)."""
        x = _dev_tensor(x, torch.float32, "x")
        if x.dim() != 2 or x.shape[1] != self.dim:
            raise ValueError(f"x must be (n, {self.dim})")
        n = x.shape[0]
        if rep is None:
            rep = torch.empty(n, dtype=torch.int64, device=x.device)
        mc = torch.empty(n, dtype=torch.float32, device=x.device) if max_cos else None
        st = IngestStats() if sync else None
        _check(_lib.lam_dedup_ingest(self.ctx.handle, self._h, _ptr(x), n, _ptr(rep), _ptr(mc),
                                     ctypes.byref(st) if st is not None else None))
        stats = st.as_dict() if st is not None else None
        return (rep, stats, mc) if max_cos else (rep, stats)

    def quantize(self, eps: float, absmax: float | None = None, mode: str = "bits") -> QParams:
        p = QParams()
        _check(_lib.lam_store_quantize(self.ctx.handle, self._h, float(eps),
                                       0.0 if absmax is None else float(absmax), _MODES[mode], ctypes.byref(p)))
        return p

    def clear(self):
        """Empty the store, keeping its device memory."""
        _check(_lib.lam_store_clear(self.ctx.handle, self._h))

    def dequantize(self, out: torch.Tensor | None = None) -> torch.Tensor:
        """The reconstruction x_hat of every retained row (size x dim float32)."""
        n = self.size
        if out is None:
            out = torch.empty((max(1, n), self.dim), dtype=torch.float32, device=f"cuda:{self.ctx.device}")
        _check(_lib.lam_store_dequantize(self.ctx.handle, self._h, _ptr(out)))
        return out[:n]

    def ids(self) -> torch.Tensor:
        n = self.size
        out = torch.empty(max(1, n), dtype=torch.int64, device=f"cuda:{self.ctx.device}")
        _check(_lib.lam_store_export(self.ctx.handle, self._h, _ptr(out), _P(None), 0))
        return out[:n]

    def codes(self) -> torch.Tensor:
        p = self.info().q
        out = torch.empty(max(1, p.code_bytes // 4), dtype=torch.int32, device=f"cuda:{self.ctx.device}")
        _check(_lib.lam_store_export(self.ctx.handle, self._h, _P(None), _ptr(out), out.numel() * 4))
        return out[: p.code_bytes // 4]

    def block_encode(self) -> dict:
        """Per-block codec of the current codes (lam_store_block_encode)."""
        st = BlockStats()
        _check(_lib.lam_store_block_encode(self.ctx.handle, self._h, ctypes.byref(st)))
        self._blocks = st.as_dict()
        return self._blocks

    def block_decode(self, out: torch.Tensor | None = None) -> torch.Tensor:
        n = self.size
        if out is None:
            out = torch.empty((max(1, n), self.dim), dtype=torch.float32, device=f"cuda:{self.ctx.device}")
        _check(_lib.lam_store_block_decode(self.ctx.handle, self._h, _ptr(out)))
        return out[:n]

    def block_export(self):
        """(widths uint8[size, dim/32], row_off int64[size + 1], data int32[words])."""
        n = self.size
        dev = f"cuda:{self.ctx.device}"
        words = int(self._blocks["data_bytes"] // 4)
        w = torch.empty((max(1, n), self.dim // 32), dtype=torch.uint8, device=dev)
        ro = torch.empty(n + 1, dtype=torch.int64, device=dev)
        d = torch.empty(max(1, words), dtype=torch.int32, device=dev)
        _check(_lib.lam_store_block_export(self.ctx.handle, self._h, _ptr(w), _ptr(ro), _ptr(d), d.numel() * 4))
        return w[:n], ro, d[:words]

    def score_topk_blocks(self, q: torch.Tensor, k: int):
        """lam_score_topk over the block encoding."""
        q = _dev_tensor(q, torch.float32, "q")
        nq = q.shape[0]
        scores = torch.empty((nq, k), dtype=torch.float32, device=q.device)
        ids = torch.empty((nq, k), dtype=torch.int64, device=q.device)
        bound = torch.empty(nq, dtype=torch.float32, device=q.device)
        _check(_lib.lam_score_topk_blocks(self.ctx.handle, self._h, _ptr(q), nq, int(k), _ptr(scores), _ptr(ids),
                                          _ptr(bound)))
        return scores, ids, bound

    def score_topk_certified(self, q: torch.Tensor, k: int):
        """Top-k plus the rank-invariance certificate: (scores, ids, bound,
        certified bool[nq], margin float32[nq]); see lam_score_topk_certified."""
        q = _dev_tensor(q, torch.float32, "q")
        if q.dim() != 2 or q.shape[1] != self.dim:
            raise ValueError(f"q must be (nq, {self.dim})")
        nq = q.shape[0]
        dev = q.device
        scores = torch.empty((nq, k), dtype=torch.float32, device=dev)
        ids = torch.empty((nq, k), dtype=torch.int64, device=dev)
        bound = torch.empty(nq, dtype=torch.float32, device=dev)
        cert = torch.empty(nq, dtype=torch.uint8, device=dev)
        margin = torch.empty(nq, dtype=torch.float32, device=dev)
        _check(_lib.lam_score_topk_certified(self.ctx.handle, self._h, _ptr(q), nq, int(k), _ptr(scores), _ptr(ids),
                                             _ptr(bound), _ptr(cert), _ptr(margin)))
        return scores, ids, bound, cert.bool(), margin

    def score_topk(self, q: torch.Tensor, k: int, out=None):
        """Top-k (scores float32[nq, k], ids int64[nq, k], bound float32[nq])."""
        q = _dev_tensor(q, torch.float32, "q")
        if q.dim() != 2 or q.shape[1] != self.dim:
            raise ValueError(f"q must be (nq, {self.dim})")
        nq = q.shape[0]
        if out is None:
            out = (torch.empty((nq, k), dtype=torch.float32, device=q.device),
                   torch.empty((nq, k), dtype=torch.int64, device=q.device),
                   torch.empty(nq, dtype=torch.float32, device=q.device))
        s, i, b = out
        _check(_lib.lam_score_topk(self.ctx.handle, self._h, _ptr(q), nq, int(k), _ptr(s), _ptr(i), _ptr(b)))
        return s, i, b

    def score_topk_noalloc(self, q: torch.Tensor, k: int, out):
        """score_topk through the allocation-free entry point (lam_score_topk_noalloc):
        the library takes its scratch from a fixed per-device array; the caller
        passes every output, out = (scores float32[nq, k], ids int64[nq, k],
        bound float32[nq]).  nq <= 256; the store must be settled (info())."""
        q = _dev_tensor(q, torch.float32, "q")
        if q.dim() != 2 or q.shape[1] != self.dim:
            raise ValueError(f"q must be (nq, {self.dim})")
        s, i, b = out
        _check(_lib.lam_score_topk_noalloc(self.ctx.handle, self._h, _ptr(q), q.shape[0], int(k), _ptr(s), _ptr(i),
                                           _ptr(b)))
        return s, i, b

    def close(self):
        if getattr(self, "_h", None):
            _lib.lam_store_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


__all__ = ["LamError", "QParams", "IngestStats", "StoreInfo", "Context", "default_context", "quantize",
           "dequantize", "triad", "Store", "qeps_plan", "removal_ceiling", "CeilingStats", "kv_pages", "kv_append", "kv_read", "kv_attend",
           "kv_evict", "rotary_frequencies", "kv_rotate", "kv_rotate_append", "abi_version", "EXPORTED", "LIB_PATH"]
