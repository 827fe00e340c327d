"""Python binding of libdejavu.so (argument marshalling only).

The functions named like the C entry points (``dv_create``, ``dv_encode``, ...) take
plain integers for device pointers and streams and raise ``DejaVuError`` on a
non-zero status.  ``Encoder`` wraps them for torch tensors: torch supplies device
memory and the current HIP stream; every step of the computation runs in the
library's HIP kernels.  Importing this module never falls back to anything: if
the library is missing, ``load()`` raises.
"""
import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib", "libdejavu.so")

DV_OK, DV_EINVAL, DV_ENOMEM, DV_EHIP, DV_EUNSUPPORTED = 0, -1, -2, -3, -4
DV_F32, DV_BF16 = 0, 1
STAGES = ["patch", "gate", "compact", "ln1", "qkv", "attn", "oproj", "ln2", "fc1", "fc2",
          "merge", "final", "restore", "cls"]
DV_FLAG_RESTORE = 1
DV_FLAG_DECISION = 2
DV_FLAG_REORDER = 4
DV_FLAG_ROTARY = 16
DV_FLAG_CACHE8 = 32
DV_ROTARY_HALVES, DV_ROTARY_PAIRS = 0, 1


class DejaVuError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"dejavu error {code}: {msg}")
        self.code = code


class dv_rotary_plan(ctypes.Structure):
    _fields_ = [("dim", ctypes.c_int), ("section", ctypes.c_int * 3), ("layout", ctypes.c_int),
                ("turn", ctypes.c_uint64 * 64)]


class dv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("pages", ctypes.c_int),
                ("page_tokens", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


class dv_config(ctypes.Structure):
    _fields_ = [("image_size", ctypes.c_int), ("patch", ctypes.c_int), ("depth", ctypes.c_int),
                ("width", ctypes.c_int), ("heads", ctypes.c_int), ("mlp", ctypes.c_int),
                ("dtype", ctypes.c_int), ("max_batch_frames", ctypes.c_int),
                ("flags", ctypes.c_uint)]


_lib = None
_P = ctypes.c_void_p
_I64 = ctypes.c_longlong


def load(path=None):
    """Load libdejavu.so (built by ``paper_2506_14107_amd.build``); raises if it is absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(f"{p} is missing: build it with python -m paper_2506_14107_amd.build")
    lib = ctypes.CDLL(p)
    sig = {
        "dv_weights_floats": (ctypes.c_size_t, [ctypes.POINTER(dv_config)]),
        "dv_create": (ctypes.c_int, [ctypes.POINTER(dv_config), _P, ctypes.c_size_t,
                                     ctypes.POINTER(_P)]),
        "dv_destroy": (ctypes.c_int, [_P]),
        "dv_last_error": (ctypes.c_char_p, []),
        "dv_workspace_bytes": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_size_t)]),
        "dv_encode": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_float, _P, _P,
                                     _P]),
        "dv_encode_noalloc": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                             _P, _P, _P]),
        "dv_encode_masked": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P]),
        "dv_encode_tokens": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                            _P, _P, _P, _P, _P]),
        "dv_compact": (ctypes.c_int, [_P, ctypes.c_int, ctypes.c_int, ctypes.c_int, _P, _P, _P,
                                      _P, _P]),
        "dv_stream_encode": (ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                            _P, _P, _P, _P, _P]),
        "dv_stream_reset": (ctypes.c_int, [_P]),
        "dv_stream_held": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_int)]),
        "dv_stream_flush": (ctypes.c_int, [_P, _P, _P, _P, _P]),
        "dv_rotary_init": (ctypes.c_int, [ctypes.POINTER(dv_rotary_plan),
                                          ctypes.POINTER(ctypes.c_int * 3), ctypes.c_int,
                                          ctypes.c_int, ctypes.c_double]),
        "dv_rotary": (ctypes.c_int, [_P, ctypes.c_int, _P, _I64, ctypes.c_int, ctypes.c_int,
                                     ctypes.c_int, _P, _P, _I64, _P]),
        "dv_cache_write": (ctypes.c_int, [_P, ctypes.c_int, _P, ctypes.c_int, _P, _P, ctypes.c_int,
                                          _P, _I64, _P, _I64, ctypes.c_int, _P, _P, _P, _I64,
                                          ctypes.c_int, _P, _I64, _P]),
        "dv_cache_read": (ctypes.c_int, [_P, ctypes.c_int, _P, ctypes.c_int, _P, _P, ctypes.c_int,
                                         _P, _I64, _P, _I64, ctypes.c_int, _P]),
        "dv_cache_attention_workspace": (ctypes.c_int, [_P, ctypes.c_int, ctypes.c_int,
                                                        ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                        ctypes.c_int, ctypes.c_int,
                                                        ctypes.POINTER(ctypes.c_size_t)]),
        "dv_cache_attention": (ctypes.c_int, [_P, ctypes.c_int, _P, ctypes.c_int, _P, _P,
                                              ctypes.c_int, _P, _I64, ctypes.c_int, ctypes.c_int,
                                              ctypes.c_int, ctypes.c_float, ctypes.c_int, _P, _I64,
                                              _P, ctypes.c_size_t, _P]),
        "dv_mfma_probe": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, _P,
                                         ctypes.POINTER(ctypes.c_double), _P]),
        "dv_profile": (ctypes.c_int, [_P, ctypes.c_uint]),
        "dv_profile_read": (ctypes.c_int, [_P, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_longlong)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    if path is None:
        _lib = lib
    return lib


def _check(rc):
    if rc != DV_OK:
        raise DejaVuError(rc, load().dv_last_error().decode())


def make_config(image_size, patch, depth, width, heads, mlp, dtype, max_batch_frames, flags=0):
    dt = {"f32": DV_F32, "bf16": DV_BF16}.get(dtype, dtype)
    return dv_config(image_size, patch, depth, width, heads, mlp, dt, max_batch_frames, flags)


# ---- the C entry points, one to one -----------------------------------------------------------
def dv_weights_floats(cfg):
    return load().dv_weights_floats(ctypes.byref(cfg))


def dv_create(cfg, weights):
    """weights: host float32 array (the blob).  Returns the handle (an int)."""
    w = np.ascontiguousarray(weights, dtype=np.float32)
    h = _P()
    _check(load().dv_create(ctypes.byref(cfg), w.ctypes.data, w.nbytes, ctypes.byref(h)))
    return h.value


def dv_destroy(handle):
    _check(load().dv_destroy(handle))


def dv_last_error():
    return load().dv_last_error().decode()


def dv_workspace_bytes(handle):
    n = ctypes.c_size_t()
    _check(load().dv_workspace_bytes(handle, ctypes.byref(n)))
    return n.value


def dv_encode(handle, frames, n_frames, group_size, tau, out_embeddings, out_masks, stream):
    _check(load().dv_encode(handle, frames, n_frames, group_size, tau, out_embeddings,
                            out_masks, stream))


def dv_encode_noalloc(handle, frames, n_frames, group_size, tau, out_embeddings, out_masks,
                      stream):
    _check(load().dv_encode_noalloc(handle, frames, n_frames, group_size, tau, out_embeddings,
                                    out_masks, stream))


DV_SCRATCH_BYTES = 128 << 20   # the static scratch array of dv_encode_noalloc


def dv_encode_masked(handle, frames, n_frames, group_size, masks, out_embeddings, out_masks,
                     stream):
    _check(load().dv_encode_masked(handle, frames, n_frames, group_size, masks, out_embeddings,
                                   out_masks, stream))


def dv_encode_tokens(handle, frames, n_frames, group_size, tau, masks, out_embeddings, out_masks,
                     out_tokens, stream):
    _check(load().dv_encode_tokens(handle, frames, n_frames, group_size, tau, masks,
                                   out_embeddings, out_masks, out_tokens, stream))


def dv_stream_encode(handle, frames, n_frames, group_size, tau, masks, out_embeddings, out_masks,
                     out_tokens, stream):
    _check(load().dv_stream_encode(handle, frames, n_frames, group_size, tau, masks,
                                   out_embeddings, out_masks, out_tokens, stream))


def dv_stream_reset(handle):
    _check(load().dv_stream_reset(handle))


def dv_stream_held(handle):
    n = ctypes.c_int(0)
    _check(load().dv_stream_held(handle, ctypes.byref(n)))
    return n.value


def dv_stream_flush(handle, out_embeddings, out_masks, out_tokens, stream):
    _check(load().dv_stream_flush(handle, out_embeddings, out_masks, out_tokens, stream))


def dv_compact(masks, n_frames, n_tokens, group_size, idx, pos, qoff, count, stream):
    _check(load().dv_compact(masks, n_frames, n_tokens, group_size, idx, pos, qoff, count,
                             stream))


def dv_rotary_init(section, layout, per_axis, base):
    """Returns the filled dv_rotary_plan."""
    plan = dv_rotary_plan()
    sec = (ctypes.c_int * 3)(*section)
    _check(load().dv_rotary_init(ctypes.byref(plan), ctypes.byref(sec), layout, int(per_axis),
                                 float(base)))
    return plan


# In the calls below `plan` and `cache` are addresses (ctypes.addressof) of the structures.
def dv_rotary(plan, dtype, x, x_stride, rows, heads, head_dim, positions, out, out_stride, stream):
    _check(load().dv_rotary(plan, dtype, x, x_stride, rows, heads, head_dim, positions, out,
                            out_stride, stream))


def dv_cache_write(cache, n_seqs, table, table_pages, offsets, starts, dtype, k, k_stride, v,
                   v_stride, rows, plan, positions, q, q_stride, q_heads, q_out, q_out_stride,
                   stream):
    _check(load().dv_cache_write(cache, n_seqs, table, table_pages, offsets, starts, dtype, k,
                                 k_stride, v, v_stride, rows, plan, positions, q, q_stride,
                                 q_heads, q_out, q_out_stride, stream))


def dv_cache_read(cache, n_seqs, table, table_pages, offsets, starts, dtype, k, k_stride, v,
                  v_stride, rows, stream):
    _check(load().dv_cache_read(cache, n_seqs, table, table_pages, offsets, starts, dtype, k,
                                k_stride, v, v_stride, rows, stream))


def dv_cache_attention_workspace(cache, n_seqs, table_pages, with_offsets, dtype, rows, q_heads,
                                 max_rows):
    n = ctypes.c_size_t()
    _check(load().dv_cache_attention_workspace(cache, n_seqs, table_pages, int(with_offsets), dtype,
                                               rows, q_heads, max_rows, ctypes.byref(n)))
    return n.value


def dv_cache_attention(cache, n_seqs, table, table_pages, offsets, lengths, dtype, q, q_stride,
                       rows, q_heads, max_rows, scale, causal, out, out_stride, workspace,
                       workspace_bytes, stream):
    _check(load().dv_cache_attention(cache, n_seqs, table, table_pages, offsets, lengths, dtype, q,
                                     q_stride, rows, q_heads, max_rows, scale, int(causal), out,
                                     out_stride, workspace, workspace_bytes, stream))


def dv_mfma_probe(blocks, iters, sink, stream):
    """Enqueues the MFMA-loop probe; returns the FLOPs of the launch."""
    fl = ctypes.c_double()
    _check(load().dv_mfma_probe(blocks, iters, sink, ctypes.byref(fl), stream))
    return fl.value


DV_PROFILE_ALL = 0x3FFF


def dv_profile(handle, stage_mask):
    _check(load().dv_profile(handle, int(stage_mask)))


def dv_profile_read(handle, stage):
    ms, n = ctypes.c_double(), ctypes.c_longlong()
    _check(load().dv_profile_read(handle, stage, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


# ---- torch convenience wrapper ----------------------------------------------------------------
def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _stream(stream):
    import torch
    return (stream or torch.cuda.current_stream()).cuda_stream


class Encoder:
    """A handle bound to one model.  Tensors must live on the current HIP device."""

    def __init__(self, model, weights, max_batch_frames):
        m = model
        self.model = m
        flags = (DV_FLAG_RESTORE if getattr(m, "restore", False) else 0) | \
            (DV_FLAG_DECISION if getattr(m, "decision", False) else 0) | \
            (DV_FLAG_REORDER if getattr(m, "reorder", False) else 0) | \
            (DV_FLAG_ROTARY if getattr(m, "rotary", False) else 0) | \
            (DV_FLAG_CACHE8 if getattr(m, "cache8", False) else 0)
        self.cfg = make_config(m.image_size, m.patch, m.depth, m.width, m.heads, m.mlp, m.dtype,
                               max_batch_frames, flags)
        self.handle = dv_create(self.cfg, weights)

    def close(self):
        if self.handle:
            dv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _outs(self, n, want_masks, want_tokens):
        import torch
        m = self.model
        emb = torch.empty((n, m.width), dtype=torch.float32, device="cuda")
        masks = (torch.empty((n, m.depth, m.n_tokens), dtype=torch.uint8, device="cuda")
                 if want_masks else None)
        toks = (torch.empty((n, m.n_tokens, m.width), dtype=torch.float32, device="cuda")
                if want_tokens else None)
        return emb, masks, toks

    def _check_frames(self, frames):
        m = self.model
        if (not frames.is_cuda or frames.dtype.itemsize != 4 or not frames.is_contiguous()
                or tuple(frames.shape[1:]) != (3, m.image_size, m.image_size)):
            raise ValueError("frames must be a contiguous fp32 CUDA tensor [n, 3, S, S]")

    def encode(self, frames, group_size, tau, want_masks=True, want_tokens=False, stream=None):
        """Gate mode; returns (embeddings, masks or None, tokens or None)."""
        self._check_frames(frames)
        n = frames.shape[0]
        emb, masks, toks = self._outs(n, want_masks, want_tokens)
        if want_tokens:
            dv_encode_tokens(self.handle, _ptr(frames), n, group_size, float(tau), 0, _ptr(emb),
                             _ptr(masks), _ptr(toks), _stream(stream))
        else:
            dv_encode(self.handle, _ptr(frames), n, group_size, float(tau), _ptr(emb),
                      _ptr(masks), _stream(stream))
        return emb, masks, toks

    def encode_noalloc(self, frames, group_size, tau, out_embeddings, out_masks=None, stream=None):
        """Gate mode through dv_encode_noalloc, into caller-allocated outputs (embeddings
        [n, D] fp32, masks [n, depth, N] uint8 or None); the library allocates nothing."""
        self._check_frames(frames)
        n = frames.shape[0]
        dv_encode_noalloc(self.handle, _ptr(frames), n, group_size, float(tau),
                          _ptr(out_embeddings), _ptr(out_masks), _stream(stream))
        return out_embeddings, out_masks

    def encode_masked(self, frames, group_size, masks_in, want_masks=True, want_tokens=False,
                      stream=None):
        """Mask-injection mode; masks_in: uint8 CUDA tensor [n, depth, N]."""
        self._check_frames(frames)
        n = frames.shape[0]
        m = self.model
        if (not masks_in.is_cuda or masks_in.dtype.itemsize != 1 or not masks_in.is_contiguous()
                or tuple(masks_in.shape) != (n, m.depth, m.n_tokens)):
            raise ValueError("masks must be a contiguous uint8 CUDA tensor [n, depth, N]")
        emb, masks, toks = self._outs(n, want_masks, want_tokens)
        if want_tokens:
            dv_encode_tokens(self.handle, _ptr(frames), n, group_size, 0.0, _ptr(masks_in),
                             _ptr(emb), _ptr(masks), _ptr(toks), _stream(stream))
        else:
            dv_encode_masked(self.handle, _ptr(frames), n, group_size, _ptr(masks_in), _ptr(emb),
                             _ptr(masks), _stream(stream))
        return emb, masks, toks

    def stream_encode(self, frames, group_size, tau=0.0, masks_in=None, want_masks=True,
                      want_tokens=False, stream=None):
        """The next frames of a stream (gate mode with tau, or injected masks_in).  Returns the
        outputs of the frames the call completes: its own frames, except that a reordered
        stream first completes the frames it held and then holds back those after its last
        anchor."""
        self._check_frames(frames)
        n = frames.shape[0]
        held = dv_stream_held(self.handle)
        emb, masks, toks = self._outs(n + held, want_masks, want_tokens)
        dv_stream_encode(self.handle, _ptr(frames), n, group_size, float(tau),
                         _ptr(masks_in) if masks_in is not None else 0, _ptr(emb), _ptr(masks),
                         _ptr(toks), _stream(stream))
        k = n + held - dv_stream_held(self.handle)
        return tuple(o[:k] if o is not None else None for o in (emb, masks, toks))

    def stream_flush(self, want_masks=True, want_tokens=False, stream=None):
        """End the stream: the outputs of the frames it still held (none without reordering)."""
        held = dv_stream_held(self.handle)
        emb, masks, toks = self._outs(held, want_masks, want_tokens)
        dv_stream_flush(self.handle, _ptr(emb) if held else 0, _ptr(masks) if held else 0,
                        _ptr(toks) if held else 0, _stream(stream))
        return emb, masks, toks

    def stream_reset(self):
        dv_stream_reset(self.handle)

    def profile(self, stages=True):
        """stages: True (all), False (off), or an iterable of stage names."""
        if stages is True:
            mask = DV_PROFILE_ALL
        elif not stages:
            mask = 0
        else:
            mask = sum(1 << STAGES.index(s) for s in stages)
        dv_profile(self.handle, mask)

    def profile_read(self):
        return {name: dv_profile_read(self.handle, i) for i, name in enumerate(STAGES)}


def compact(masks, group_size, stream=None):
    """Stream compaction of a [n_frames, n_tokens] uint8 CUDA map; returns (idx, pos, qoff, count)."""
    import torch
    F, N = masks.shape
    idx = torch.empty(F * N, dtype=torch.int32, device="cuda")
    pos = torch.empty(F * N, dtype=torch.int32, device="cuda")
    qoff = torch.empty(F + 1, dtype=torch.int32, device="cuda")
    cnt = torch.empty(1, dtype=torch.int32, device="cuda")
    dv_compact(_ptr(masks.contiguous()), F, N, group_size, _ptr(idx), _ptr(pos), _ptr(qoff),
               _ptr(cnt), _stream(stream))
    return idx, pos, qoff, cnt


# ---- token rows and their 8-bit cache -----------------------------------------------------------
# Small calls are bound by what the host does: the checks below read few attributes, and torch is
# looked up once (by the first Rotary or TokenCache).
torch = None


def _need_torch():
    global torch
    if torch is None:
        import torch as t
        torch = t


def _dtype(t):
    d = t.dtype
    if d is torch.bfloat16:
        return DV_BF16
    if d is torch.float32:
        return DV_F32
    raise ValueError(f"rows must be bf16 or fp32 (got {d})")


def _misfit(name, t):
    raise ValueError(f"{name} has shape {tuple(t.shape)}, type {t.dtype} and device {t.device}, which "
                     "do not fit the other arguments")


_INT_MAX = 2 ** 31 - 1   # counts are C ints, to which ctypes cuts what is larger


def _stride(name, t):
    """Row stride of a tensor [rows, heads, head_dim] whose heads lie side by side."""
    n, h, d = t.shape
    if n > _INT_MAX:
        raise ValueError(f"{name} has {n} rows: too many for one call")
    sr, sh, sd = t.stride()
    if (sd != 1 and d > 1) or (sh != d and h > 1):
        raise ValueError(f"the heads of a row of {name} must lie side by side")
    return sr if n > 1 else max(sr, h * d)


def _rows(name, t, shape, dtype, index):
    """Checks a row tensor against what it has to be; returns its row stride."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        _misfit(name, t)
    return _stride(name, t)


def _like(t, stride, wide):
    """New rows like those of t, side by side."""
    if stride == wide:
        return torch.empty_like(t)   # the cheaper call
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _ints(name, t, index, shape):
    if (t.dtype is not torch.int32 or t.get_device() != index or t.shape != shape
            or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on device {index}")
    return t.data_ptr()


def _elsewhere(index, stream):
    """Whether a call on device `index` and `stream` (None: the device's current one) needs another
    device or stream current, so that what it allocates belongs there (_Away)."""
    if index < 0:
        raise ValueError("tensors must be on a HIP device")
    if stream is None:
        return torch.cuda.current_device() != index
    if stream.device.index != index:
        raise ValueError(f"a stream of {stream.device} for tensors on device {index}")
    return True


class _Away:
    def __init__(self, index, stream):
        self.stack = [torch.cuda.device(index)] + ([torch.cuda.stream(stream)] if stream else [])

    def __enter__(self):
        for c in self.stack:
            c.__enter__()

    def __exit__(self, *e):
        for c in reversed(self.stack):
            c.__exit__(*e)


def _raw_stream(index):
    return torch._C._cuda_getCurrentRawStream(index)


class Rotary:
    """Rates of rotary positions with a time, a height and a width axis: `sections` pairs of channels
    turn with each.  layout "halves" (channels i and i + dim/2) or "pairs" (2i and 2i + 1); per_axis:
    every axis takes the whole range of rates."""

    def __init__(self, sections, layout="halves", per_axis=False, base=10000.0):
        _need_torch()
        code = {"halves": DV_ROTARY_HALVES, "pairs": DV_ROTARY_PAIRS}.get(layout)
        if code is None:
            raise ValueError(f"unknown rotary layout {layout!r}")
        if len(sections) != 3:
            raise ValueError("sections are the pairs of three axes")
        self.plan = dv_rotary_init(sections, code, per_axis, base)
        self.dim = self.plan.dim
        self.address = ctypes.addressof(self.plan)


def rotary(x, positions, rot, out=None, stream=None):
    """Rows x [rows, heads, head_dim] with their heads turned by `positions` (int32 [rows, 3]) at the
    rates of `rot` (Rotary), into `out` (which may be x) or a new tensor."""
    index = x.get_device()
    if _elsewhere(index, stream):
        with _Away(index, stream):
            return rotary(x, positions, rot, out)
    shape = x.shape
    if len(shape) != 3:
        _misfit("x", x)
    n, h, d = shape
    dtype = _dtype(x)
    xs = _stride("x", x)
    if out is None:
        os = h * d
        out = _like(x, xs, os)
    else:
        os = xs if out is x else _rows("out", out, shape, x.dtype, index)
    dv_rotary(rot.address, dtype, x.data_ptr(), xs, n, h, d,
              _ints("positions", positions, index, (n, 3)), out.data_ptr(), os, _raw_stream(index))
    return out


class TokenCache:
    """A paged cache of keys and values in 8 bits (float8_e4m3fn codes, a power-of-two scale for each
    page and head): `pages` pages of `page_tokens` tokens of `kv_heads` heads.

    A sequence's places lie in the pages of its row of `table` (int32 [n_seqs, table_pages]; None:
    sequence s has the table_pages = pages // n_seqs pages from s * table_pages on).  `offsets`
    (int32 [n_seqs + 1]) cuts a call's rows into sequences; None: one row each.

    buffers: (k, v, k_scale, v_scale) to use instead of new ones: float8_e4m3fn [pages, kv_heads,
    page_tokens, head_dim] and [pages, kv_heads, head_dim, page_tokens], fp32 [pages, kv_heads].
    """

    def __init__(self, pages, kv_heads, head_dim, page_tokens=64, device=None, buffers=None):
        _need_torch()
        shapes = [(pages, kv_heads, page_tokens, head_dim), (pages, kv_heads, head_dim, page_tokens),
                  (pages, kv_heads), (pages, kv_heads)]
        types = [torch.float8_e4m3fn, torch.float8_e4m3fn, torch.float32, torch.float32]
        if buffers is None:
            if device is None:
                device = torch.device("cuda", torch.cuda.current_device())
            buffers = [torch.empty(s, dtype=t, device=device) for s, t in zip(shapes, types)]
        for b, s, t in zip(buffers, shapes, types):
            if (tuple(b.shape) != s or b.dtype is not t or not b.is_contiguous()
                    or b.device != buffers[0].device):
                raise ValueError(f"a cache buffer must be a contiguous {t} tensor {list(s)}")
        self.k, self.v, self.k_scale, self.v_scale = buffers
        self.device, self.index = self.k.device, self.k.get_device()
        self.pages, self.kv_heads = pages, kv_heads
        self.head_dim, self.page_tokens = head_dim, page_tokens
        self.desc = dv_cache(*(b.data_ptr() for b in buffers), pages, page_tokens, kv_heads,
                             head_dim)
        self.address = ctypes.addressof(self.desc)
        self.scratch = {}   # workspace bytes by the sizes they depend on

    def _seqs(self, at, name, offsets, table):
        """(n_seqs, table, table_pages, offsets, at) as the entry points take them."""
        index = self.index
        n = at.shape[0] if at.dim() == 1 else -1
        if n > _INT_MAX:
            raise ValueError(f"{name} has {n} sequences: too many for one call")
        if table is None:
            t, tp = 0, self.pages // max(n, 1)
        else:
            tp = table.shape[1] if table.dim() == 2 else -1
            t = _ints("table", table, index, (n, tp))
        o = 0 if offsets is None else _ints("offsets", offsets, index, (n + 1,))
        return n, t, tp, o, _ints(name, at, index, (n,))

    def write(self, k, v, starts, offsets=None, table=None, rotary=None, positions=None, q=None,
              q_out=None, stream=None):
        """Quantises rows k and v [rows, kv_heads, head_dim] into places starts[s] .. of each
        sequence.  With `rotary` and `positions` the keys are turned first, and the rows of q
        [rows, heads, head_dim] into `q_out` (which may be q) or a new tensor, which is returned."""
        index = self.index
        if _elsewhere(index, stream):
            with _Away(index, stream):
                return self.write(k, v, starts, offsets, table, rotary, positions, q, q_out)
        n, t, tp, o, at = self._seqs(starts, "starts", offsets, table)
        rows, dt = k.shape[0], k.dtype
        dtype = _dtype(k)
        shape = (rows, self.kv_heads, self.head_dim)
        ks = _rows("k", k, shape, dt, index)
        vs = _rows("v", v, shape, dt, index)
        plan = pos = qp = qs = qop = qos = heads = 0
        if rotary is not None and positions is not None:
            plan, pos = rotary.address, _ints("positions", positions, index, (rows, 3))
        elif rotary is not None or positions is not None:
            raise ValueError("rotary and positions come together")
        if q is not None:
            if q.dim() != 3:
                _misfit("q", q)
            heads = q.shape[1]
            shape = (rows, heads, self.head_dim)
            qs = _rows("q", q, shape, dt, index)
            if q_out is None:
                q_out = _like(q, qs, heads * self.head_dim)
            qos = _rows("q_out", q_out, shape, dt, index)
            qp, qop = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise ValueError("q_out without q")
        dv_cache_write(self.address, n, t, tp, o, at, dtype, k.data_ptr(), ks, v.data_ptr(), vs, rows,
                       plan, pos, qp, qs, heads, qop, qos, _raw_stream(index))
        return q_out

    def read(self, starts, offsets=None, table=None, rows=None, dtype=None, out=None, stream=None):
        """Keys and values [rows, kv_heads, head_dim] of places starts[s] .. of each sequence, into
        `out` (a pair of tensors) or new tensors of `rows` rows and `dtype` (bf16)."""
        index = self.index
        if _elsewhere(index, stream):
            with _Away(index, stream):
                return self.read(starts, offsets, table, rows, dtype, out)
        n, t, tp, o, at = self._seqs(starts, "starts", offsets, table)
        if out is None:
            shape = (n if rows is None else rows, self.kv_heads, self.head_dim)
            out = [torch.empty(shape, dtype=dtype or torch.bfloat16, device=self.device)
                   for _ in range(2)]
        k, v = out
        rows, dt = k.shape[0], k.dtype
        shape = (rows, self.kv_heads, self.head_dim)
        ks = _rows("k", k, shape, dt, index)
        vs = _rows("v", v, shape, dt, index)
        dv_cache_read(self.address, n, t, tp, o, at, _dtype(k), k.data_ptr(), ks, v.data_ptr(), vs,
                      rows, _raw_stream(index))
        return out

    def attention(self, q, lengths, offsets=None, table=None, causal=True, scale=None, max_rows=0,
                  out=None, workspace=None, stream=None):
        """Attention of rows q [rows, heads, head_dim] over the first lengths[s] places of their
        sequences, into `out` or a new tensor.  causal: the rows are the sequence's last places and
        see no later ones.  max_rows: an upper bound of any sequence's rows, if known.  workspace: a
        uint8 tensor to use (see attention_workspace) instead of one of the call's own."""
        index = self.index
        if _elsewhere(index, stream):
            with _Away(index, stream):
                return self.attention(q, lengths, offsets, table, causal, scale, max_rows, out,
                                      workspace)
        n, t, tp, o, at = self._seqs(lengths, "lengths", offsets, table)
        if q.dim() != 3:
            _misfit("q", q)
        rows, heads, d = q.shape
        shape = (rows, heads, self.head_dim)
        qs = _rows("q", q, shape, q.dtype, index)
        dtype = _dtype(q)
        if out is None:
            os = heads * d
            out = _like(q, qs, os)
        else:
            os = _rows("out", out, shape, q.dtype, index)
        ws = size = 0
        if workspace is None:
            key = (n, tp, o != 0, dtype, rows, heads, max_rows)
            size = self.scratch.get(key)
            if size is None:
                size = dv_cache_attention_workspace(self.address, *key)
                if len(self.scratch) >= 1024:
                    self.scratch.clear()
                self.scratch[key] = size
            if size:
                workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
                ws = workspace.data_ptr()
        else:
            if (workspace.get_device() != index or workspace.dtype is not torch.uint8
                    or not workspace.is_contiguous()):
                _misfit("workspace", workspace)
            ws, size = workspace.data_ptr(), workspace.numel()
        dv_cache_attention(self.address, n, t, tp, o, at, dtype, q.data_ptr(), qs, rows, heads,
                           max_rows, d ** -0.5 if scale is None else scale, causal, out.data_ptr(), os,
                           ws, size, _raw_stream(index))
        return out

    def attention_workspace(self, n_seqs, rows, heads, table_pages=None, with_offsets=True,
                            max_rows=0, dtype=None):
        """Bytes of scratch that `attention` needs for such a call (of rows of `dtype`; bf16)."""
        tp = self.pages // max(n_seqs, 1) if table_pages is None else table_pages
        return dv_cache_attention_workspace(self.address, n_seqs, tp, with_offsets,
                                            DV_F32 if dtype is torch.float32 else DV_BF16, rows,
                                            heads, max_rows)
