"""LVSA block-sparse video attention for MI355X (gfx950): Python binding.

A thin ctypes layer over ``liblvsa.so`` (C ABI in ``include/lvsa.h``).  It only
marshals arguments: every mask and attention computation runs in the native
library (host C++ builder, HIP kernels).  torch is used for device memory and
streams only.  If the library is missing every call raises; there is no
fallback.

    import paper_2605_31057_amd as lvsa
    p = lvsa.Params(window=6, budget_frames=21)
    csr = lvsa.build_mask(T=121, P=1560, B=128, step=10, params=p)
    csr.upload()
    lvsa.attention(q, k, v, csr.device_mask(), out)      # q,k,v,out: [H,N,128] bf16
    ex = lvsa.build_mask(T=121, P=1560, B=128, step=10, params=p, exact=True)
    ex.upload()
    lvsa.attention_exact(q, k, v, ex.exact_mask(), out)  # Eq. 2 token for token
    m = lvsa.csr_mask(row_ptr, col_idx, n_tokens, block)  # any block CSR on the device
    lvsa.attention(q, k, v, m, out)
    r = lvsa.Rope(121, 30, 52)                            # positions of a 121 x 30 x 52 grid
    cache = lvsa.KvCache(heads=12, capacity=121 * 1560)   # 8-bit keys and values
    q = lvsa.rope(q, r, start=n0)                         # new tokens n0, n0 + 1, ..
    lvsa.kv_write(cache, k, v, start=n0, rope=r)          # keys rotated on the way
    lvsa.attention_cache(q, cache)                        # over every token so far
"""
import ctypes
import os

__all__ = [
    "LvsaError", "Params", "Csr", "BlockMask", "ExactMask", "lib",
    "params_default", "frame_sets", "frame_window", "build_mask", "build_mask_device",
    "build_exact_mask_device", "csr_mask", "attention", "attention_noalloc",
    "attention_exact",
    "dense_attention", "WINDOW_BASIC", "WINDOW_ADAPTIVE", "WINDOW_EXPANDED",
    "MAX_FRAMES", "Rope", "rope", "rope_backward", "KvCache", "kv_write", "kv_read",
    "attention_cache", "ROPE_PAIRS", "ROPE_HALVES",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblvsa.so")

WINDOW_BASIC, WINDOW_ADAPTIVE, WINDOW_EXPANDED = 0, 1, 2
MAX_FRAMES = 4096
ROPE_PAIRS, ROPE_HALVES = 0, 1
OK, EINVAL, ENOMEM, EDEVICE, EUNSUPPORTED = 0, -1, -2, -3, -4

_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_p = ctypes.c_void_p
_pi32 = ctypes.POINTER(ctypes.c_int32)
_byref = ctypes.byref


class LvsaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().lvsa_status_str(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


class Params(ctypes.Structure):
    """lvsa_params: C, W, T_per override, window rule, rotation, tie rule,
    dedicated initial anchors, text tokens after the video tokens."""
    _fields_ = [("budget_frames", _i32), ("window", _i32), ("tper", _i32),
                ("window_mode", _i32), ("rotate", _i32), ("tie_high", _i32),
                ("extra_anchors", _i32), ("text_tokens", _i32)]

    def __init__(self, **kw):
        d = dict(budget_frames=21, window=6, tper=0,
                 window_mode=WINDOW_EXPANDED, rotate=1, tie_high=0,
                 extra_anchors=0, text_tokens=0)
        d.update(kw)
        super().__init__(**{k: int(v) for k, v in d.items()})


class BlockMask(ctypes.Structure):
    """lvsa_block_mask: a block CSR in device memory."""
    _fields_ = [("n_tokens", _i32), ("block", _i32), ("n_q_blocks", _i32),
                ("n_kv_blocks", _i32), ("row_ptr", _p), ("col_idx", _p)]


class ExactMask(ctypes.Structure):
    """lvsa_exact_mask: device-resident token-exact form (row_ptr and entry
    words)."""
    _fields_ = [("n_tokens", _i32), ("block", _i32), ("n_q_blocks", _i32),
                ("frame_tokens", _i32), ("row_ptr", _p), ("entry", _p)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", _p), ("heads", _i32), ("n_tokens", _i32),
                ("head_dim", _i32), ("stride_head", _i64),
                ("stride_token", _i64)]


class _Rope(ctypes.Structure):
    _fields_ = [("frames", _i32), ("height", _i32), ("width", _i32), ("pairs", _i32 * 3),
                ("layout", _i32), ("table", _p)]


class _KvCache(ctypes.Structure):
    _fields_ = [("heads", _i32), ("capacity", _i32), ("block", _i32), ("n_tokens", _i32),
                ("k", _p), ("v", _p), ("k_scale", _p), ("v_scale", _p)]


_LIB = None


def lib():
    """The loaded native library (raises if it was not built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2605_31057_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        sig = {
            "lvsa_status_str": (ctypes.c_char_p, [_i32]),
            "lvsa_version": (_i32, []),
            "lvsa_params_default": (None, [ctypes.POINTER(Params)]),
            "lvsa_frame_sets": (_i32, [_i32, _i32, ctypes.POINTER(Params), _pi32,
                                       _pi32, _pi32, _pi32, _pi32, _pi32]),
            "lvsa_frame_window": (_i32, [_i32, _i32, ctypes.POINTER(Params), _i32,
                                         _pi32, _pi32, _pi32]),
            "lvsa_build_mask": (_i32, [_i32, _i32, _i32, _i32, _i32,
                                       ctypes.POINTER(Params), ctypes.POINTER(_p)]),
            "lvsa_csr_info": (_i32, [_p, _pi32, _pi32, ctypes.POINTER(_i64),
                                     ctypes.POINTER(_pi32), ctypes.POINTER(_pi32)]),
            "lvsa_csr_shape": (_i32, [_p, _pi32, _pi32]),
            "lvsa_csr_upload": (_i32, [_p, _p]),
            "lvsa_csr_free": (None, [_p]),
            "lvsa_csr_device_view": (_i32, [_p, ctypes.POINTER(BlockMask)]),
            "lvsa_build_mask_device": (_i32, [_i32, _i32, _i32, _i32, _i32,
                                              ctypes.POINTER(Params), _p, _p, _i64, _p]),
            "lvsa_build_exact_mask": (_i32, [_i32, _i32, _i32, _i32, _i32,
                                             ctypes.POINTER(Params),
                                             ctypes.POINTER(_p)]),
            "lvsa_csr_entries": (_i32, [_p, _pi32,
                                        ctypes.POINTER(ctypes.POINTER(ctypes.c_uint32))]),
            "lvsa_csr_exact_view": (_i32, [_p, ctypes.POINTER(ExactMask)]),
            "lvsa_build_exact_mask_device": (_i32, [_i32, _i32, _i32, _i32, _i32,
                                                    ctypes.POINTER(Params), _p, _p,
                                                    _i64, _p]),
            "lvsa_attention_exact": (_i32, [ctypes.POINTER(_Tensor)] * 3 +
                                     [ctypes.POINTER(ExactMask),
                                      ctypes.POINTER(_Tensor), _p]),
            "lvsa_attention": (_i32, [ctypes.POINTER(_Tensor)] * 3 +
                               [ctypes.POINTER(BlockMask), ctypes.POINTER(_Tensor), _p]),
            "lvsa_attention_noalloc": (_i32, [ctypes.POINTER(_Tensor)] * 3 +
                                       [ctypes.POINTER(BlockMask), ctypes.POINTER(_Tensor),
                                        _p]),
            "lvsa_dense_attention": (_i32, [ctypes.POINTER(_Tensor)] * 3 +
                                     [_i32, ctypes.POINTER(_Tensor), _p]),
            "lvsa_rope_table_size": (_i32, [ctypes.POINTER(_Rope), ctypes.POINTER(_i64)]),
            "lvsa_rope_table": (_i32, [ctypes.POINTER(_Rope), ctypes.c_double, _p, _i64]),
            "lvsa_rope_forward": (_i32, [ctypes.POINTER(_Tensor), _i32, _i32,
                                         ctypes.POINTER(_Rope), ctypes.POINTER(_Tensor), _p]),
            "lvsa_rope_backward": (_i32, [ctypes.POINTER(_Tensor), _i32, _i32,
                                          ctypes.POINTER(_Rope), ctypes.POINTER(_Tensor), _p]),
            "lvsa_kv_write": (_i32, [ctypes.POINTER(_KvCache), ctypes.POINTER(_Tensor),
                                     ctypes.POINTER(_Tensor), _i32, _i32,
                                     ctypes.POINTER(_Rope), _p]),
            "lvsa_kv_read": (_i32, [ctypes.POINTER(_KvCache), _i32, ctypes.POINTER(_Tensor),
                                    ctypes.POINTER(_Tensor), _i32, _p]),
            "lvsa_attention_cache": (_i32, [ctypes.POINTER(_Tensor), _i32,
                                            ctypes.POINTER(_KvCache),
                                            ctypes.POINTER(BlockMask),
                                            ctypes.POINTER(_Tensor), _p, _i64, _p]),
            "lvsa_attention_cache_workspace": (_i32, [ctypes.POINTER(_Tensor), _i32,
                                                      ctypes.POINTER(_KvCache),
                                                      ctypes.POINTER(BlockMask),
                                                      ctypes.POINTER(_i64)]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


def _check(status, where):
    if status != OK:
        raise LvsaError(status, where)


def params_default():
    p = Params()
    lib().lvsa_params_default(ctypes.byref(p))
    return p


def frame_sets(T, step, params=None, growth=False):
    """(T_per, anchors, win_lo, win_hi) for one step (lists of ints), plus the
    Alg. 1 growth steps per frame when ``growth`` is set."""
    params = params or Params()
    tper, n = _i32(), _i32()
    anchors = (_i32 * T)()
    lo = (_i32 * T)()
    hi = (_i32 * T)()
    grow = (_i32 * T)()
    _check(lib().lvsa_frame_sets(T, step, ctypes.byref(params), ctypes.byref(tper),
                                 anchors, ctypes.byref(n), lo, hi, grow), "lvsa_frame_sets")
    res = (tper.value, list(anchors[:n.value]), list(lo), list(hi))
    return res + (list(grow),) if growth else res


def frame_window(T, step, t, params=None):
    """(lo, hi, growth) of query frame t (lvsa_frame_window)."""
    params = params or Params()
    lo, hi, g = _i32(), _i32(), _i32()
    _check(lib().lvsa_frame_window(T, step, ctypes.byref(params), t, ctypes.byref(lo),
                                   ctypes.byref(hi), ctypes.byref(g)), "lvsa_frame_window")
    return lo.value, hi.value, g.value


def _stream_ptr(stream):
    if stream is None:
        import torch
        return _p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return _p(stream)
    return _p(stream.cuda_stream)


class Csr:
    """Host-built block CSR (lvsa_csr handle)."""

    def __init__(self, handle):
        self._h = _p(handle)

    def __del__(self):
        self.free()

    def free(self):
        if getattr(self, "_h", None) and self._h.value and _LIB is not None:
            _LIB.lvsa_csr_free(self._h)
            self._h = _p()

    def info(self):
        """(n_q_blocks, n_kv_blocks, nnz, row_ptr, col_idx) as lvsa_csr_info
        returns them (the arrays as ctypes pointers)."""
        nq, nk, nnz = _i32(), _i32(), _i64()
        rp, ci = _pi32(), _pi32()
        _check(lib().lvsa_csr_info(self._h, ctypes.byref(nq), ctypes.byref(nk),
                                   ctypes.byref(nnz), ctypes.byref(rp), ctypes.byref(ci)),
               "lvsa_csr_info")
        return nq.value, nk.value, nnz.value, rp, ci

    def shape(self):
        """(n_tokens, block) of the handle (lvsa_csr_shape)."""
        n, b = _i32(), _i32()
        _check(lib().lvsa_csr_shape(self._h, ctypes.byref(n), ctypes.byref(b)),
               "lvsa_csr_shape")
        return n.value, b.value

    @property
    def n_tokens(self):
        return self.shape()[0]

    @property
    def block(self):
        return self.shape()[1]

    @property
    def n_blocks(self):
        return self.info()[0]

    @property
    def nnz(self):
        return self.info()[2]

    def arrays(self):
        """(row_ptr, col_idx) as numpy int32 copies."""
        import numpy as np
        nb, _, nnz, rp, ci = self.info()
        row_ptr = np.ctypeslib.as_array(rp, shape=(nb + 1,)).copy()
        col_idx = (np.ctypeslib.as_array(ci, shape=(nnz,)).copy() if nnz
                   else np.zeros(0, dtype=np.int32))
        return row_ptr, col_idx

    def entries(self):
        """Token-exact entry words as a numpy uint32 copy (raises LvsaError
        with EUNSUPPORTED for a handle built without them)."""
        import numpy as np
        nnz = self.nnz
        P = _i32()
        e = ctypes.POINTER(ctypes.c_uint32)()
        _check(lib().lvsa_csr_entries(self._h, ctypes.byref(P), ctypes.byref(e)),
               "lvsa_csr_entries")
        return (np.ctypeslib.as_array(e, shape=(nnz,)).copy() if nnz
                else np.zeros(0, dtype=np.uint32))

    def upload(self, stream=None):
        _check(lib().lvsa_csr_upload(self._h, _stream_ptr(stream)), "lvsa_csr_upload")
        return self

    def device_mask(self):
        m = BlockMask()
        _check(lib().lvsa_csr_device_view(self._h, ctypes.byref(m)),
               "lvsa_csr_device_view")
        return m

    def exact_mask(self):
        m = ExactMask()
        _check(lib().lvsa_csr_exact_view(self._h, ctypes.byref(m)),
               "lvsa_csr_exact_view")
        return m


def build_mask(T, P, B, step, params=None, layer=0, exact=False):
    """Host LVSA mask builder -> Csr.  ``exact=True`` also builds the
    token-exact entry words (lvsa_build_exact_mask)."""
    params = params or Params()
    h = _p()
    fn, name = ((lib().lvsa_build_exact_mask, "lvsa_build_exact_mask") if exact
                else (lib().lvsa_build_mask, "lvsa_build_mask"))
    _check(fn(T, P, B, step, layer, ctypes.byref(params), ctypes.byref(h)), name)
    return Csr(h.value)


def _mask_keep(mask, tensors):
    mask._keep = tensors   # keep the device buffers alive with the view
    return mask


def build_mask_device(T, P, B, step, row_ptr, col_idx, params=None, layer=0,
                      stream=None):
    """Device LVSA mask builder into int32 device tensors row_ptr [nb+1] and
    col_idx [>= nb*nb]; returns a BlockMask over them."""
    params = params or Params()
    _check(lib().lvsa_build_mask_device(T, P, B, step, layer, ctypes.byref(params),
                                        _p(row_ptr.data_ptr()), _p(col_idx.data_ptr()),
                                        col_idx.numel(), _stream_ptr(stream)),
           "lvsa_build_mask_device")
    N = T * P + params.text_tokens
    nb = (N + B - 1) // B
    m = BlockMask(N, B, nb, nb, row_ptr.data_ptr(), col_idx.data_ptr())
    return _mask_keep(m, (row_ptr, col_idx))


def build_exact_mask_device(T, P, B, step, row_ptr, entry, params=None, layer=0,
                            stream=None):
    """Device builder of the token-exact form into device tensors (row_ptr
    int32 [nb+1], entry int32/uint32 [>= nb*nb]); returns an ExactMask."""
    params = params or Params()
    _check(lib().lvsa_build_exact_mask_device(
        T, P, B, step, layer, ctypes.byref(params), _p(row_ptr.data_ptr()),
        _p(entry.data_ptr()), entry.numel(), _stream_ptr(stream)),
        "lvsa_build_exact_mask_device")
    N = T * P + params.text_tokens
    nb = (N + B - 1) // B
    m = ExactMask(N, B, nb, P, row_ptr.data_ptr(), entry.data_ptr())
    return _mask_keep(m, (row_ptr, entry))


def csr_mask(row_ptr, col_idx, n_tokens, block):
    """A BlockMask over a caller-built block CSR in device int32 tensors
    (row_ptr [nb+1], col_idx [nnz], nb = ceil(n_tokens / block))."""
    nb = (n_tokens + block - 1) // block
    if row_ptr.numel() != nb + 1:
        raise LvsaError(EINVAL, f"row_ptr holds {row_ptr.numel()} offsets, the mask has "
                        f"{nb} query blocks")
    m = BlockMask(n_tokens, block, nb, nb, row_ptr.data_ptr(), col_idx.data_ptr())
    return _mask_keep(m, (row_ptr, col_idx))


def exact_csr_mask(row_ptr, entry, n_tokens, block, frame_tokens):
    """An ExactMask over caller-built token-exact entry words in device
    tensors (row_ptr int32 [nb+1], entry int32/uint32 [nnz])."""
    nb = (n_tokens + block - 1) // block
    m = ExactMask(n_tokens, block, nb, frame_tokens, row_ptr.data_ptr(), entry.data_ptr())
    return _mask_keep(m, (row_ptr, entry))


def _tensor(t):
    if t.dim() != 3:
        raise ValueError("expected a [heads, n_tokens, head_dim] tensor")
    if t.stride(2) != 1:
        raise ValueError("head_dim must be contiguous")
    import torch
    if t.dtype != torch.bfloat16 or not t.is_cuda:
        raise ValueError("expected a bfloat16 device tensor")
    return _Tensor(t.data_ptr(), t.shape[0], t.shape[1], t.shape[2],
                   t.stride(0), t.stride(1))


def attention(q, k, v, mask, out=None, stream=None):
    """Block-sparse attention (lvsa_attention); returns out."""
    import torch
    if out is None:
        out = torch.empty_like(q)
    tq, tk, tv, to = (_tensor(x) for x in (q, k, v, out))
    _check(lib().lvsa_attention(ctypes.byref(tq), ctypes.byref(tk), ctypes.byref(tv),
                                ctypes.byref(mask), ctypes.byref(to),
                                _stream_ptr(stream)), "lvsa_attention")
    return out


def attention_noalloc(q, k, v, mask, out, stream=None):
    """lvsa_attention_noalloc: block-sparse attention that allocates nothing
    (the caller passes `out`); calls overlapping on one device race."""
    tq, tk, tv, to = (_tensor(x) for x in (q, k, v, out))
    _check(lib().lvsa_attention_noalloc(ctypes.byref(tq), ctypes.byref(tk),
                                        ctypes.byref(tv), ctypes.byref(mask),
                                        ctypes.byref(to), _stream_ptr(stream)),
           "lvsa_attention_noalloc")
    return out


def attention_exact(q, k, v, mask, out=None, stream=None):
    """Token-exact attention (lvsa_attention_exact): Eq. 2 token for token."""
    import torch
    if out is None:
        out = torch.empty_like(q)
    tq, tk, tv, to = (_tensor(x) for x in (q, k, v, out))
    _check(lib().lvsa_attention_exact(ctypes.byref(tq), ctypes.byref(tk),
                                      ctypes.byref(tv), ctypes.byref(mask),
                                      ctypes.byref(to), _stream_ptr(stream)),
           "lvsa_attention_exact")
    return out


def dense_attention(q, k, v, block=128, out=None, stream=None):
    """Dense attention of the same kernel design (lvsa_dense_attention)."""
    import torch
    if out is None:
        out = torch.empty_like(q)
    tq, tk, tv, to = (_tensor(x) for x in (q, k, v, out))
    _check(lib().lvsa_dense_attention(ctypes.byref(tq), ctypes.byref(tk),
                                      ctypes.byref(tv), block, ctypes.byref(to),
                                      _stream_ptr(stream)), "lvsa_dense_attention")
    return out


# ------------------------------------------- rotary positions, 8-bit cache

# A call of one of these on a few tokens takes a few microseconds on the GPU, so the
# marshalling keeps to what it needs: plain integers, no context managers without a
# stream, and nothing looked up twice (``_fast``).

_FAST = None


class _Fast:
    """What the calls below use of torch and the library."""

    def __init__(self):
        import torch
        L = lib()
        self.torch = torch
        self.codes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
        self.bf16 = torch.bfloat16
        self.empty, self.empty_like = torch.empty, torch.empty_like
        self.device = torch.cuda.current_device
        # The current stream of a device, as an address.
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        self.turns = ((L.lvsa_rope_forward, "lvsa_rope_forward"),
                      (L.lvsa_rope_backward, "lvsa_rope_backward"))
        self.grad_enabled = torch.is_grad_enabled
        self.written = torch.autograd.graph.increment_version
        self.turn = _turn_function(torch)
        self.write, self.read = L.lvsa_kv_write, L.lvsa_kv_read
        self.attend = L.lvsa_attention_cache
        self.attend_workspace = L.lvsa_attention_cache_workspace


def _fast():
    global _FAST
    if _FAST is None:
        _FAST = _Fast()
    return _FAST


def _rows(t, device):
    """A [heads, n_tokens, head_dim] tensor on device number ``device``; the strides
    of axes of one element are put right, torch leaves them open."""
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("expected a [heads, n_tokens, head_dim] tensor")
    sh, st, sd = t.stride()
    if sd != 1:
        raise ValueError("head_dim must be contiguous")
    if t.get_device() != device:
        raise ValueError("expected a tensor on the current device")
    H, n, d = shape
    if (H | n | d) >> 31:      # ctypes would cut them down without a word
        raise LvsaError(EUNSUPPORTED, f"a tensor of shape {tuple(shape)}")
    if n <= 1:
        st = d
    return _byref(_Tensor(t.data_ptr(), H, n, d, sh if H > 1 else n * st, st))


def _type_code(first, second):
    if first.dtype != second.dtype:
        raise ValueError("expected tensors of one type")
    code = _FAST.codes.get(first.dtype)
    if code is None:
        raise ValueError("expected bfloat16, float16 or float32")
    return code


def _place(at):
    """A token's place, within what the library's 32-bit arguments hold (ctypes would
    cut it down without a word)."""
    if not 0 <= at < 2 ** 31:
        raise LvsaError(EINVAL, f"token {at}")
    return at


def _with_stream(fn, stream, *args):
    """fn(*args) with ``stream`` current: torch allocates for it then."""
    torch = _fast().torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return fn(*args)


class Rope:
    """Rotary positions over a latent grid of ``frames`` x ``height`` x ``width``
    tokens (lvsa_rope): ``pairs`` of the 64 pairs of a row turn with the frame,
    the row and the column.  ``table``: a float32 device tensor [entries, 2] of
    (cos, sin), frames first, then rows, then columns; built from ``theta``
    (lvsa_rope_table) and put on ``device`` if not given."""

    def __init__(self, frames, height, width, pairs=(22, 21, 21), theta=10000.0,
                 layout=ROPE_PAIRS, table=None, device="cuda"):
        import torch
        if not all(0 <= n < 2 ** 31 for n in (frames, height, width, layout, *pairs)):
            raise LvsaError(EINVAL, "Rope")
        self._c = _Rope(frames, height, width, (_i32 * 3)(*pairs), layout, None)
        n = _i64()
        _check(lib().lvsa_rope_table_size(ctypes.byref(self._c), ctypes.byref(n)),
               "lvsa_rope_table_size")
        if table is None:
            host = torch.empty(n.value, 2, dtype=torch.float32)
            _check(lib().lvsa_rope_table(ctypes.byref(self._c), theta, _p(host.data_ptr()),
                                         n.value), "lvsa_rope_table")
            table = host.to(device)
        if (table.dtype != torch.float32 or not table.is_contiguous()
                or table.numel() != 2 * n.value):
            raise ValueError(f"expected a contiguous float32 table of {n.value} (cos, sin)")
        self.table = table
        self._c.table = table.data_ptr()
        self._device, self._ref = table.get_device(), ctypes.byref(self._c)


def _rope_ref(r, device):
    if r is None:
        return None
    if r._device != device:
        raise ValueError("expected a table on the current device")
    return r._ref


def _turn_function(torch):
    class Turn(torch.autograd.Function):
        """``rope`` (back False) or ``rope_backward`` (True): each is the other's
        gradient."""

        @staticmethod
        def forward(ctx, x, out, r, start, back):
            ctx.turn = r, start, back
            if out is not None:
                ctx.mark_dirty(out)
            return _launch_turn(x, r, start, out, back)

        @staticmethod
        def backward(ctx, grad):
            r, start, back = ctx.turn
            return _rotate(_readable(grad), r, start, None, not back), None, None, None, None

    return Turn


def _readable(grad):
    """A gradient as autograd hands it on (expanded, say) with rows that the library
    takes."""
    sh, st, sd = grad.stride()
    H, n, _ = grad.shape
    if (sd == 1 and (n == 1 or (st > 0 and st % 8 == 0)) and (H == 1 or sh % 8 == 0)
            and grad.data_ptr() % 16 == 0):
        return grad
    return grad.clone(memory_format=_FAST.torch.contiguous_format)


def _launch_turn(x, r, start, out, back):
    f = _FAST
    dev = f.device()
    if out is None:
        out = f.empty_like(x)
    call, name = f.turns[back]
    status = call(_rows(x, dev), _type_code(x, out), _place(start), _rope_ref(r, dev),
                  _rows(out, dev), f.stream(dev))
    if status:
        raise LvsaError(status, name)
    return out


def _rotate(x, r, start, out, back):
    f = _fast()
    if (x.requires_grad or (out is not None and out.requires_grad)) and f.grad_enabled():
        return f.turn.apply(x, out, r, start, back)
    if out is None:
        return _launch_turn(x, r, start, out, back)
    _launch_turn(x, r, start, out, back)
    f.written(out)       # a graph that has saved it notices
    return out


def rope(x, r, start=0, out=None, stream=None):
    """x [heads, n, 128] (bfloat16, float16, float32), token i of which is token
    start + i of the grid, rotated by ``r`` (lvsa_rope_forward); out may be x.
    Differentiable in x (the table is data)."""
    if stream is not None:
        return _with_stream(rope, stream, x, r, start, out)
    return _rotate(x, r, start, out, False)


def rope_backward(grad, r, start=0, out=None, stream=None):
    """Gradient of ``rope``: of its input, from that of its output
    (lvsa_rope_backward); out may be grad.  What autograd calls, for programs that
    have no graph."""
    if stream is not None:
        return _with_stream(rope_backward, stream, grad, r, start, out)
    return _rotate(grad, r, start, out, True)


class KvCache:
    """Keys and values of a sequence held in 8 bits (lvsa_kv_cache): room for
    ``capacity`` tokens (rounded up to 128) of ``heads`` key heads, one scale a
    head and ``block`` tokens.  ``n_tokens`` are held; setting it lower drops the
    last ones.  ``buffers``: the caller's own (k, v, k_scale, v_scale), as
    lvsa_kv_cache lays them out; allocated if not given."""

    def __init__(self, heads, capacity, block=128, n_tokens=0, buffers=None, device="cuda"):
        import torch
        capacity = -(-capacity // 128) * 128
        if block not in (64, 128) or not 0 < capacity <= 1 << 24 or not 0 < heads < 65536:
            raise LvsaError(EUNSUPPORTED, f"KvCache of {heads} heads, {capacity} tokens, "
                            f"blocks of {block}")
        f8, f32 = torch.float8_e4m3fn, torch.float32
        shapes = [((heads, capacity, 128), f8), ((heads, capacity // 64, 128, 64), f8),
                  ((heads, capacity // block), f32), ((heads, capacity // block), f32)]
        if buffers is None:
            buffers = [torch.empty(s, dtype=t, device=device) for s, t in shapes]
        for b, (s, t) in zip(buffers, shapes, strict=True):
            if tuple(b.shape) != s or b.dtype != t or not b.is_contiguous():
                raise ValueError(f"expected a contiguous {t} buffer of shape {s}")
            if b.device != buffers[0].device:
                raise ValueError("expected buffers on one device")
        self.k, self.v, self.k_scale, self.v_scale = buffers
        self._c = _KvCache(heads, capacity, block, 0, *(b.data_ptr() for b in buffers))
        self._device, self._ref = self.k.get_device(), ctypes.byref(self._c)
        self.n_tokens = n_tokens

    @property
    def heads(self):
        return self._c.heads

    @property
    def capacity(self):
        return self._c.capacity

    @property
    def block(self):
        return self._c.block

    @property
    def n_tokens(self):
        return self._c.n_tokens

    @n_tokens.setter
    def n_tokens(self, n):
        if not 0 <= n <= self._c.capacity:
            raise ValueError(f"n_tokens must lie in 0 .. {self._c.capacity}")
        self._c.n_tokens = n


def _cache_ref(c, device):
    if c._device != device:
        raise ValueError("expected a cache on the current device")
    return c._ref


def kv_write(cache, k, v, start=None, rope=None, stream=None):
    """Quantises k and v [heads, n, 128] (bfloat16, float16, float32) into tokens
    start, start + 1, .. of the cache (by default behind its last), the keys
    rotated by ``rope`` on the way (lvsa_kv_write); returns the cache.  It has no
    gradient."""
    if stream is not None:
        return _with_stream(kv_write, stream, cache, k, v, start, rope)
    f = _fast()
    dev = f.device()
    _check(f.write(_cache_ref(cache, dev), _rows(k, dev), _rows(v, dev), _type_code(k, v),
                   cache._c.n_tokens if start is None else _place(start),
                   _rope_ref(rope, dev), f.stream(dev)), "lvsa_kv_write")
    return cache


def kv_read(cache, start=0, n=None, dtype=None, out=None, stream=None):
    """Keys and values [heads, n, 128] of tokens start .. start + n - 1 (by default
    to the last) in ``dtype`` (bfloat16 by default), or into ``out`` = (k, v)
    (lvsa_kv_read); returns (k, v)."""
    if stream is not None:
        return _with_stream(kv_read, stream, cache, start, n, dtype, out)
    f = _fast()
    dev = f.device()
    given = out is not None
    _place(start)
    if out is None:
        n = cache.n_tokens - start if n is None else n
        if n < 1:
            raise LvsaError(EINVAL, f"{n} tokens to read")
        if start + n > cache.n_tokens:
            raise LvsaError(EINVAL, f"tokens {start} .. {start + n - 1} of {cache.n_tokens}")
        out = f.empty((2, cache._c.heads, n, 128), dtype=dtype or f.bf16,
                      device=cache.k.device).unbind(0)
    k, v = out
    if v.shape != k.shape or (n is not None and k.shape[1] != n):
        raise ValueError("expected out tensors of n tokens")
    if dtype is not None and k.dtype != dtype:
        raise ValueError("expected out tensors of the given type")
    _check(f.read(_cache_ref(cache, dev), start, _rows(k, dev), _rows(v, dev), _type_code(k, v),
                  f.stream(dev)), "lvsa_kv_read")
    if given:
        f.written([k, v])
    return out


def attention_cache(q, cache, mask=None, q_start=0, out=None, stream=None):
    """Attention of q [heads, n, 128] (bfloat16; heads a multiple of the cache's)
    over every held token, or over the blocks that ``mask`` (a BlockMask over the
    cache's tokens) keeps for queries q_start, q_start + 1, ..
    (lvsa_attention_cache); returns out.  It has no gradient."""
    if stream is not None:
        return _with_stream(attention_cache, stream, q, cache, mask, q_start, out)
    f = _fast()
    dev = f.device()
    given = out is not None
    if out is None:
        out = f.empty_like(q)
    if q.dtype != f.bf16 or out.dtype != f.bf16:
        raise ValueError("expected bfloat16 tensors")
    tq, to, c = _rows(q, dev), _rows(out, dev), _cache_ref(cache, dev)
    m = None if mask is None else _byref(mask)
    _place(q_start)
    need = _i64()
    _check(f.attend_workspace(tq, q_start, c, m, _byref(need)), "lvsa_attention_cache_workspace")
    size, work = need.value, None
    if size:
        work = f.empty(size, dtype=f.torch.uint8, device=q.device)
    _check(f.attend(tq, q_start, c, m, to, work.data_ptr() if size else None, size,
                    f.stream(dev)), "lvsa_attention_cache")
    if given:
        f.written(out)
    return out
