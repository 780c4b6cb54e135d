"""Thin ctypes binding over libfdkv.so: argument marshalling only, every step runs in the CUDA kernels.

torch is used for device memory and streams.  Importing this module loads the shared library and raises if
it is missing; there is no CPU or eager fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("FDKV_LIB_PATH", os.path.join(_HERE, "libfdkv.so"))  # override: A/B runs of two builds

F32, BF16 = 0, 1
SHARED, RESIDUAL, EXACT = 0, 1, 2
RESIDUAL_ENTRIES, RESIDUAL_TOKENS = 0, 1
_STATUS = ["ok", "invalid argument", "unsupported", "arena full", "workspace too small", "state", "cuda error",
           "device timeout", "device check failed", "too large for the built-in scratch"]
NOALLOC_MAX_ELEMS = 1 << 20


class FdkvError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        name = _STATUS[code] if 0 <= code < len(_STATUS) else str(code)
        super().__init__(f"{where}: fdkv status {code} ({name})")


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "max_batch", "max_prefill",
                                         "max_tail", "dtype", "keep_num", "keep_den", "residual_rule", "block_size", "max_fold", "row_format")]


class _Rotary(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "rotary_dim", "interleaved", "n_axes")] + \
               [("eps", C.c_float), ("scale", C.c_float)] + [(n, C.c_void_p) for n in ("inv_freq", "axis_of", "q_weight", "k_weight")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_06519_b200.build` "
                          "(nvcc, sm_100a); this package has no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER
    sig = {
        "fdkv_sizes": [P(_Config), P(sz), P(sz)],
        "fdkv_sizes_prompts": [P(_Config), i32, P(sz), P(sz)],
        "fdkv_create": [P(_Config), vp, sz, vp, sz, P(vp)],
        "fdkv_reset": [vp],
        "fdkv_compress_prefill": [vp, i32, i32, i32, i32, P(vp), P(vp), i64, i64, vp],
        "fdkv_probe": [vp, i32, i32, i32, P(vp), P(i32), i32, C.c_double, vp, vp, vp],
        "fdkv_set_modes": [vp, i32, P(i32)],
        "fdkv_route_budget": [vp, i32, sz, P(C.c_double), vp, vp],
        "fdkv_commit": [vp, i32, vp],
        "fdkv_decode_attn": [vp, i32, i32, vp, vp, vp, vp, i32, vp],
        "fdkv_decode_attn_host": [vp, i32, i32, vp, vp, vp, vp, i32, vp],
        "fdkv_decode_step_host": [vp, i32, vp, vp, vp, vp, i32, vp],
        "fdkv_decode_attn_shared": [vp, i32, i32, vp, i32, vp, vp, vp, vp, i32, vp],
        "fdkv_append_tail": [vp, i32, i32, i32, vp, vp, i64, i64, vp],
        "fdkv_qk_norm_rope": [P(_Rotary), i64, vp, i64, i64, vp, i64, i64, vp, i64, vp, i64, i64, vp, i64, i64, vp],
        "fdkv_decode_qkv": [vp, i32, i32, vp, i32, P(_Rotary), vp, i64, vp, vp, i32, vp],
        "fdkv_set_tail_len": [vp, i32, i32, vp],
        "fdkv_fold_tail": [vp, i32, i32, vp],
        "fdkv_get_rows_e4m3": [vp, i32, i32, i32, i32, vp, vp, vp],
        "fdkv_get_shared": [vp, i32, i32, i32, i32, vp, vp],
        "fdkv_get_residual": [vp, i32, i32, i32, i32, vp, vp, P(i32), vp],
        "fdkv_get_modes": [vp, i32, P(i32)],
        "fdkv_get_token_set": [vp, i32, i32, i32, vp, vp, P(i32), vp],
        "fdkv_footprint": [vp, i32, P(sz), P(sz)],
        "fdkv_decode_bytes": [vp, i32, i32, P(sz)],
        "fdkv_plan_decode": [i32, i32, P(i32), P(i32), i32, i32, i32, i32, i32, P(C.c_uint32), P(i32), P(i32)],
        "fdkv_device_status": [vp],
        "fdkv_compress_unit_noalloc": [vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, P(i32), vp],
        "fdkv_test_wait_expiry": [vp, i32, vp],
        "fdkv_test_count_expiry": [vp, i32, vp],
        "fdkv_test_plan_shared": [i32] * 6 + [vp] + [i32] * 5 + [vp, vp],
        "fdkv_test_clear_device_status": [vp, vp],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.fdkv_destroy.argtypes = [vp]
    lib.fdkv_destroy.restype = None
    lib.fdkv_last_cuda_error.restype = C.c_int32
    lib.fdkv_status_str.argtypes = [C.c_int]
    lib.fdkv_status_str.restype = C.c_char_p
    lib.fdkv_launch_count.restype = C.c_int64
    lib.fdkv_kernel_launch_count.argtypes = [C.c_int32]
    lib.fdkv_kernel_launch_count.restype = C.c_int64
    return lib


_lib = _load()
_decode_attn = _lib.fdkv_decode_attn
_decode_attn_shared = _lib.fdkv_decode_attn_shared
_qk_norm_rope = _lib.fdkv_qk_norm_rope


def launch_count() -> int:
    return int(_lib.fdkv_launch_count())


KERNEL_PROBE_TC, KERNEL_PROBE_PORTABLE, KERNEL_DECODE_FAST, KERNEL_DECODE_PORTABLE, KERNEL_TOKEN_SCORE, KERNEL_SHARED_TC, KERNEL_SHARED_PORTABLE = range(7)


def kernel_launch_count(kernel: int) -> int:
    """Launches of one of the kernels that exist in a portable and an sm_100a form (fdkv_kernel_id)."""
    return int(_lib.fdkv_kernel_launch_count(kernel))


def last_cuda_error() -> int:
    return int(_lib.fdkv_last_cuda_error())


@dataclass
class Config:
    n_layers: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    max_batch: int
    max_prefill: int
    max_tail: int
    dtype: int
    keep_num: int
    keep_den: int
    residual_rule: int = 0  # 0: largest-magnitude entries; 1: the paper's probe-scored tokens
    block_size: int = 2  # layers per depth block (B of Eq. 1): 2 or 4; "pair" arguments then index blocks
    max_fold: int = 0  # generated tokens fold_tail may move into the compressed form per sequence
    row_format: int = 0  # 0: committed rows keep the storage type; 1: e4m3 codes with per-channel scales

    def c(self) -> _Config:
        return _Config(*(int(getattr(self, f[0])) for f in _Config._fields_))


def sizes(cfg: Config, prompts: int | None = None):
    """(arena, workspace) bytes; prompts: slots that hold a committed prompt at a time (None: all)."""
    a, w = C.c_size_t(0), C.c_size_t(0)
    if prompts is None:
        st = _lib.fdkv_sizes(C.byref(cfg.c()), C.byref(a), C.byref(w))
    else:
        st = _lib.fdkv_sizes_prompts(C.byref(cfg.c()), prompts, C.byref(a), C.byref(w))
    if st:
        raise FdkvError(st, "fdkv_sizes")
    return a.value, w.value


def _check(st: int, where: str):
    if st:
        raise FdkvError(st, where)


def _stream(stream) -> int:
    # (the raw handle: building a torch.cuda.Stream object per call costs a microsecond)
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def plan_decode(T, modes, n_kv_heads: int, keep_num: int, keep_den: int, n_ctas: int, residual_rule: int = 0, row_format: int = 0):
    """fdkv_plan_decode (host only): T = prefill length per sequence, modes = [batch][n_kv_heads] of the layer's units.
    Returns (ranges, parts): ranges[c] = ((unit, slice) begin, (unit, slice) end) of thread block c, parts[u] = split-K
    parts of unit u."""
    batch = len(T)
    t_arr = (C.c_int32 * batch)(*[int(t) for t in T])
    flat = [int(m) for row in modes for m in row]
    if len(flat) != batch * n_kv_heads:
        raise ValueError("modes must be [batch][n_kv_heads]")
    m_arr = (C.c_int32 * len(flat))(*flat)
    start = (C.c_uint32 * (n_ctas + 1))()
    used = C.c_int32(0)
    parts = (C.c_int32 * len(flat))()
    _check(_lib.fdkv_plan_decode(batch, n_kv_heads, t_arr, m_arr, keep_num, keep_den, residual_rule, row_format, n_ctas, start,
                                 C.byref(used), parts), "fdkv_plan_decode")
    pts = [(int(v) >> 20, int(v) & 0xFFFFF) for v in start[:used.value + 1]]
    return [(pts[c], pts[c + 1]) for c in range(used.value)], list(parts)


def compress_unit_noalloc(x0, x1, keep_num: int, keep_den: int, z0_out, idx_out, val_out, stream=None) -> int:
    """Allocation-free compression of one [T, d] pair into caller-owned outputs (no context, no workspace).

    For callers that may not allocate device memory: the scratch is a static array inside the library.  The
    outputs must already exist (z0_out [T, d], idx_out int32 [k], val_out [k]); returns k.  Calls on one device
    share the scratch, so do not overlap them on different streams.
    """
    T, d = x0.shape
    dtype = BF16 if x0.dtype == torch.bfloat16 else F32
    cnt = C.c_int32(0)
    _check(_lib.fdkv_compress_unit_noalloc(_ptr(x0), _ptr(x1), x0.stride(0), T, d, dtype, keep_num, keep_den, _ptr(z0_out),
                                           _ptr(idx_out), _ptr(val_out), C.byref(cnt), _stream(stream)),
           "fdkv_compress_unit_noalloc")
    return int(cnt.value)


class Rotary:
    """What fdkv_qk_norm_rope does to a layer's queries and keys (fdkv_rotary): kept by the caller beside the layer's weights.

    inv_freq: one frequency per rotating pair of channels; axis_of: the position axis that turns it (None: axis 0 for all);
    q_weight / k_weight: RMS norm weights [head_dim] on the device (None: no norm).
    """

    def __init__(self, inv_freq, axis_of=None, n_axes=1, interleaved=False, q_weight=None, k_weight=None, eps=1e-6, scale=1.0):
        m = len(inv_freq)
        if axis_of is not None and len(axis_of) != m:
            raise ValueError("axis_of needs one entry per frequency")
        self._inv = (C.c_float * max(m, 1))(*[float(f) for f in inv_freq])
        self._axis = None if axis_of is None else (C.c_int32 * max(m, 1))(*[int(a) for a in axis_of])
        self.n_axes, self.q_weight, self.k_weight = n_axes, q_weight, k_weight
        self._rest = (2 * m, int(interleaved), n_axes, eps, scale, C.addressof(self._inv), None if self._axis is None else C.addressof(self._axis))
        self._c = {}  # sizes -> (what the weights are, struct): one for each (a call reads it while other threads may make calls of other sizes)
        for w in (q_weight, k_weight):
            if w is not None and (w.dim() != 1 or w.stride(0) != 1):
                raise ValueError("norm weights must be dense [head_dim] tensors")
        if q_weight is not None and k_weight is not None and q_weight.get_device() != k_weight.get_device():
            raise ValueError("norm weights must be on one device")

    @property
    def device(self):
        """The weights' device (None without weights)."""
        w = self.k_weight if self.q_weight is None else self.q_weight
        return None if w is None else w.get_device()

    def c(self, n_q_heads: int, n_kv_heads: int, head_dim: int, tdtype) -> _Rotary:
        rows, q, k = (n_q_heads, n_kv_heads, head_dim, tdtype), self.q_weight, self.k_weight
        # (as they are now: a module may have given its parameters new memory)
        weights = (None if q is None else (q.data_ptr(), q.dtype, q.shape, q.stride()), None if k is None else (k.data_ptr(), k.dtype, k.shape, k.stride()))
        kept = self._c.get(rows)
        if kept is None or kept[0] != weights:
            for w in weights:
                if w is not None and w[1:] != (tdtype, (head_dim,), (1,)):
                    raise ValueError("norm weights must be dense [head_dim] tensors of the rows' dtype")
            if q is not None and k is not None and q.get_device() != k.get_device():
                raise ValueError("norm weights must be on one device")
            kept = self._c[rows] = (weights, _Rotary(*rows[:3], _dtype_code(tdtype), *self._rest, *[w and w[0] for w in weights]))
        return kept[1]


def _dtype_code(tdtype) -> int:
    if tdtype is torch.bfloat16:
        return BF16
    if tdtype is torch.float32:
        return F32
    raise ValueError("rows must be bfloat16 or float32")


def _positions(positions, n_axes: int, n: int) -> int:
    """The distance between the axes of positions [n_axes, n], or [n] for one axis."""
    shape, strides = positions.shape, positions.stride()
    if positions.dtype is not torch.int32 or (shape != (n_axes, n) and not (n_axes == 1 and shape == (n,))) or (n > 1 and strides[-1] != 1):
        raise ValueError("positions must be int32 [n_axes, n], dense along n")
    return strides[0] if n_axes > 1 else n


def qk_norm_rope(rotary: Rotary, q, k, positions, q_out=None, k_out=None, stream=None):
    """Norm and rotation of queries [n, n_q_heads, d] and keys [n, n_kv_heads, d] (either may be None); returns (q_out, k_out).
    Tensors may be strided (a slice of the fused projection, a layer's rows); an output may be its own input."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("queries or keys are needed")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("an output needs its input")
    n, _, d = x.shape
    dtype, device = x.dtype, x.get_device()
    qp = kp = qop = kop = None
    qn = qh = kn = kh = qon = qoh = kon = koh = 0
    hq = hk = 1
    if q is not None:
        if q_out is None:
            q_out = _empty(q.shape, dtype, q.device, stream)
        qp, qn, qh, hq = _rows(q, n, d, dtype, device)
        qop, qon, qoh, ho = _rows(q_out, n, d, dtype, device)
        if ho != hq:
            raise ValueError("q_out must have the shape of q")
    if k is not None:
        if k_out is None:
            k_out = _empty(k.shape, dtype, k.device, stream)
        kp, kn, kh, hk = _rows(k, n, d, dtype, device)
        kop, kon, koh, ho = _rows(k_out, n, d, dtype, device)
        if ho != hk:
            raise ValueError("k_out must have the shape of k")
    pos, step = None, 0
    if positions is not None:
        pos, step = positions.data_ptr(), _positions(positions, rotary.n_axes, n)
        if positions.get_device() != device:
            raise ValueError("all tensors must be on one CUDA device")
    r = rotary.c(hq, hk, d, dtype)
    if device < 0 or rotary.device not in (None, device):
        raise ValueError("all tensors must be on one CUDA device")
    if device != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return qk_norm_rope(rotary, q, k, positions, q_out, k_out, stream)
    st = _qk_norm_rope(r, n, qp, qn, qh, kp, kn, kh, pos, step, qop, qon, qoh, kop, kon, koh, _stream(stream))
    if st:
        raise FdkvError(st, "fdkv_qk_norm_rope")
    return q_out, k_out


def _empty(shape, dtype, device, stream):
    """A new output; it belongs to the stream that writes it, so that its memory is not handed out on another one while that does."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _on_device(device: int, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on one CUDA device")
    if device < 0:
        raise ValueError("all tensors must be on one CUDA device")


def _rows(t, n: int, d: int, dtype, device: int):
    """Address, strides (token, head) and heads of rows [n, heads, d]; a stride that nothing is reached by counts as d."""
    tn, th, td = t.shape
    st, sh, sc = t.stride()
    if sc != 1 or tn != n or td != d or t.dtype is not dtype or t.get_device() != device:
        raise ValueError("rows must be [n, heads, d] of one dtype on one device, dense along d")
    return t.data_ptr(), st if n > 1 else d, sh if th > 1 else d, th


def _slots(seqs):
    """Sequence slots as a HOST int32 array: (address, count, what keeps it alive).  An int32 CPU tensor is passed as it is."""
    if isinstance(seqs, torch.Tensor) and seqs.dtype is torch.int32 and seqs.device.type == "cpu" and seqs.is_contiguous():
        return seqs.data_ptr(), seqs.numel(), seqs
    arr = (C.c_int32 * max(len(seqs), 1))(*[int(x) for x in seqs])
    return C.addressof(arr), len(seqs), arr


class Context:
    """One fdkv context over torch-owned device memory; prompts: slots that hold a committed prompt at a time (None: all), which sizes the arena
    unless arena_bytes does."""

    def __init__(self, cfg: Config, device="cuda:0", arena_bytes: int | None = None, prompts: int | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("fdkv needs a CUDA device; there is no CPU path")
        self.cfg = cfg
        self.device = torch.device(device)
        self.tdtype = torch.bfloat16 if cfg.dtype == BF16 else torch.float32
        worst, work = sizes(cfg) if prompts is None else sizes(cfg, prompts)
        self.arena_bytes = int(arena_bytes if arena_bytes is not None else worst)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(self.arena_bytes, dtype=torch.uint8, device=self.device)
            self.work = torch.empty(work, dtype=torch.uint8, device=self.device)
            h = C.c_void_p()
            torch.cuda.synchronize()
            _check(_lib.fdkv_create(C.byref(cfg.c()), self.arena.data_ptr(), self.arena_bytes, self.work.data_ptr(), work,
                                    C.byref(h)), "fdkv_create")
        self.h = h
        self.block_size = cfg.block_size or 2
        self.n_pairs = cfg.n_layers // self.block_size  # depth blocks (pairs when the block size is 2)

    def close(self):
        if getattr(self, "h", None):
            _lib.fdkv_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self):
        _check(_lib.fdkv_reset(self.h), "fdkv_reset")

    def compress_prefill(self, seq, pair_begin, pair_end, T, k_layers, v_layers, stream=None):
        """k_layers / v_layers: per-layer tensors [T, n_kv_heads, head_dim] (None outside the pair range)."""
        L = self.cfg.n_layers
        layout, dtype = k_layers[2 * pair_begin].stride(), self.tdtype
        kp = (C.c_void_p * L)(*[None if t is None else t.data_ptr() for t in k_layers])
        vp = (C.c_void_p * L)(*[None if t is None else t.data_ptr() for t in v_layers])
        for layers in (k_layers, v_layers):
            for t in layers:
                if t is not None and (t.stride() != layout or t.dtype is not dtype):
                    raise ValueError("all K/V layers must share one [T, Hkv, d] strided layout and the context dtype")
        if layout[2] != 1:
            raise ValueError("all K/V layers must share one [T, Hkv, d] strided layout and the context dtype")
        _check(_lib.fdkv_compress_prefill(self.h, seq, pair_begin, pair_end, T, kp, vp, layout[0], layout[1],
                                          _stream(stream)), "fdkv_compress_prefill")

    def probe(self, seq, pair_begin, pair_end, q_layers, probe_pos, lam, stream=None):
        """q_layers: per-layer contiguous [W, n_q_heads, head_dim]; returns (modes int32 [pairs, Hkv], scores f32 [pairs, Hkv, 2])."""
        L = self.cfg.n_layers
        W = len(probe_pos)
        qp = (C.c_void_p * L)(*[None if t is None else t.data_ptr() for t in q_layers])
        pos = (C.c_int32 * W)(*[int(p) for p in probe_pos])
        n = (pair_end - pair_begin) * self.cfg.n_kv_heads
        modes = torch.empty(n, dtype=torch.int32, device=self.device)
        scores = torch.empty(n * 2, dtype=torch.float32, device=self.device)
        _check(_lib.fdkv_probe(self.h, seq, pair_begin, pair_end, qp, pos, W, float(lam), _ptr(modes), _ptr(scores),
                               _stream(stream)), "fdkv_probe")
        return modes.view(pair_end - pair_begin, -1), scores.view(pair_end - pair_begin, -1, 2)

    def set_modes(self, seq, modes):
        flat = [int(m) for m in torch.as_tensor(modes).reshape(-1).tolist()]
        arr = (C.c_int32 * len(flat))(*flat)
        if len(flat) != self.n_pairs * self.cfg.n_kv_heads:
            raise ValueError("modes must have n_pairs * n_kv_heads entries")
        _check(_lib.fdkv_set_modes(self.h, seq, arr), "fdkv_set_modes")

    def route_budget(self, seq, budget_bytes, stream=None):
        """Smallest lambda whose routing fits the byte budget: (fits, lambda, modes int32 [pairs, Hkv]); sets the modes."""
        n = self.n_pairs * self.cfg.n_kv_heads
        lam = C.c_double(0.0)
        modes = torch.zeros(n, dtype=torch.int32)
        st = _lib.fdkv_route_budget(self.h, seq, int(budget_bytes), C.byref(lam), modes.data_ptr(), _stream(stream))
        if st not in (0, 3):
            raise FdkvError(st, "fdkv_route_budget")
        return st == 0, float(lam.value), modes.view(self.n_pairs, -1)

    def commit(self, seq, stream=None):
        _check(_lib.fdkv_commit(self.h, seq, _stream(stream)), "fdkv_commit")

    def decode_attn(self, layer, q, k_new=None, v_new=None, out=None, out_dtype=None, stream=None):
        """q: [batch, n_q_heads, d]; returns out [batch, n_q_heads, d]."""
        od = self.cfg.dtype if out_dtype is None else out_dtype
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16 if od == BF16 else torch.float32, device=self.device)
        # one call per layer and token: plain integers, no wrapper objects
        st = _decode_attn(self.h, layer, len(q), q.data_ptr(), None if k_new is None else k_new.data_ptr(),
                          None if v_new is None else v_new.data_ptr(), out.data_ptr(), od, _stream(stream))
        if st:
            raise FdkvError(st, "fdkv_decode_attn")
        return out

    def decode_attn_shared(self, layer, prompt_seq, seqs, q, k_new=None, v_new=None, out=None, out_dtype=None, stream=None):
        """Decode attention of sequences that continue the prompt of slot `prompt_seq`: q [len(seqs), n_q_heads, d], row b for slot
        seqs[b]; returns out [len(seqs), n_q_heads, d]."""
        od = self.cfg.dtype if out_dtype is None else out_dtype
        slots, n, _keep = _slots(seqs)
        c = self.cfg
        if q.shape != (n, c.n_q_heads, c.head_dim) or q.dtype is not self.tdtype or not q.is_contiguous():
            raise ValueError("q must be a contiguous [len(seqs), n_q_heads, head_dim] tensor of the context dtype")
        for t in (k_new, v_new):
            if t is not None and (t.shape != (n, c.n_kv_heads, c.head_dim) or t.dtype is not self.tdtype or not t.is_contiguous()):
                raise ValueError("k_new and v_new must be contiguous [len(seqs), n_kv_heads, head_dim] tensors of the context dtype")
        _on_device(self.arena.get_device(), q, k_new, v_new, out)
        if self.arena.get_device() != torch._C._cuda_getDevice():
            with torch.cuda.device(self.device):
                return self.decode_attn_shared(layer, prompt_seq, seqs, q, k_new, v_new, out, out_dtype, stream)
        out = self._out(out, n, od, stream)
        st = _decode_attn_shared(self.h, layer, prompt_seq, slots, n, q.data_ptr(), None if k_new is None else k_new.data_ptr(),
                                 None if v_new is None else v_new.data_ptr(), out.data_ptr(), od, _stream(stream))
        if st:
            raise FdkvError(st, "fdkv_decode_attn_shared")
        return out

    def decode_qkv(self, layer, rotary: Rotary, qkv, positions, prompt_seq=-1, seqs=None, out=None, out_dtype=None, stream=None):
        """A decode step of one layer from its fused projection rows [batch, (n_q_heads + 2 n_kv_heads) * d]: norm, rotation, append
        and attention, each sequence on its own prompt, or (prompt_seq, seqs) all on one."""
        od = self.cfg.dtype if out_dtype is None else out_dtype
        c = self.cfg
        n = len(qkv)
        if qkv.dim() != 2 or qkv.dtype is not self.tdtype or qkv.shape[1] != (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim or qkv.stride(1) != 1:
            raise ValueError("qkv must be [batch, (n_q_heads + 2 n_kv_heads) * head_dim] of the context dtype")
        if positions is not None and _positions(positions, rotary.n_axes, n) != n:
            raise ValueError("positions must be dense")
        slots, ns, _keep = (None, n, None) if seqs is None else _slots(seqs)
        if ns != n:
            raise ValueError("qkv needs one row per sequence")
        _on_device(self.arena.get_device(), qkv, positions, rotary.q_weight, rotary.k_weight, out)
        if self.arena.get_device() != torch._C._cuda_getDevice():
            with torch.cuda.device(self.device):
                return self.decode_qkv(layer, rotary, qkv, positions, prompt_seq, seqs, out, out_dtype, stream)
        out = self._out(out, n, od, stream)
        _check(_lib.fdkv_decode_qkv(self.h, layer, prompt_seq, slots, n, rotary.c(c.n_q_heads, c.n_kv_heads, c.head_dim, self.tdtype), qkv.data_ptr(),
                                    qkv.stride(0) if n > 1 else qkv.shape[1], _ptr(positions), out.data_ptr(), od, _stream(stream)), "fdkv_decode_qkv")
        return out

    def append_tail(self, layer, seq, k, v, stream=None):
        """Appends rows k, v [n, n_kv_heads, d] (one strided layout) to a layer's tail of a sequence slot."""
        n, d = len(k), self.cfg.head_dim
        if k.shape != v.shape or tuple(k.shape[1:]) != (self.cfg.n_kv_heads, d):
            raise ValueError("k and v must be [n, Hkv, d]")
        kp, st, sh, _ = _rows(k, n, d, self.tdtype, self.arena.get_device())
        vp, vt, vh, _ = _rows(v, n, d, self.tdtype, self.arena.get_device())
        if (st, sh) != (vt, vh):
            raise ValueError("k and v must share one strided layout")
        with torch.cuda.device(self.device):
            _check(_lib.fdkv_append_tail(self.h, layer, seq, n, kp, vp, st, sh, _stream(stream)), "fdkv_append_tail")

    def _out(self, out, n, out_dtype, stream):
        """The attention's output tensor, or a new one; a caller's is checked."""
        tdtype = torch.bfloat16 if out_dtype == BF16 else torch.float32
        shape = (n, self.cfg.n_q_heads, self.cfg.head_dim)
        if out is None:
            return _empty(shape, tdtype, self.device, stream)
        if out.dtype is not tdtype or out.numel() != n * shape[1] * shape[2] or not out.is_contiguous():
            raise ValueError("out must be a contiguous [len(seqs), n_q_heads, head_dim] tensor of the output type")
        return out

    def decode_attn_host(self, layer, q, k_new, v_new, out, out_dtype, stream=None):
        """Same with host (ideally pinned) tensors; synchronous."""
        _check(_lib.fdkv_decode_attn_host(self.h, layer, q.shape[0], _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                          out_dtype, _stream(stream)), "fdkv_decode_attn_host")
        return out

    def decode_step_host(self, q, k_new, v_new, out, out_dtype, stream=None):
        """All layers of one step with host (ideally pinned) tensors: q, out [L, batch, Hq, d]; k_new, v_new
        [L, batch, Hkv, d] or None.  One copy in, L layer calls, one copy out; synchronous."""
        _check(_lib.fdkv_decode_step_host(self.h, q.shape[1], _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), out_dtype,
                                          _stream(stream)), "fdkv_decode_step_host")
        return out

    def set_tail_len(self, seq, n, stream=None):
        _check(_lib.fdkv_set_tail_len(self.h, seq, n, _stream(stream)), "fdkv_set_tail_len")

    def fold_tail(self, seq, n, stream=None):
        """Moves the first n generated tokens of every layer from the exact tails into the compressed form."""
        _check(_lib.fdkv_fold_tail(self.h, seq, n, _stream(stream)), "fdkv_fold_tail")

    def get_rows_e4m3(self, seq, layer, kv_head, is_v, T, stream=None):
        """8-bit row streams: (codes uint8 [T, d], scales float32 [d]) of a committed layer's K or V rows."""
        codes = torch.empty((T, self.cfg.head_dim), dtype=torch.uint8, device=self.device)
        scale = torch.empty(self.cfg.head_dim, dtype=torch.float32, device=self.device)
        _check(_lib.fdkv_get_rows_e4m3(self.h, seq, layer, kv_head, int(is_v), _ptr(codes), _ptr(scale), _stream(stream)),
               "fdkv_get_rows_e4m3")
        return codes, scale

    def get_shared(self, seq, pair, kv_head, is_v, T, stream=None):
        out = torch.empty((T, self.cfg.head_dim), dtype=self.tdtype, device=self.device)
        _check(_lib.fdkv_get_shared(self.h, seq, pair, kv_head, int(is_v), _ptr(out), _stream(stream)), "fdkv_get_shared")
        return out

    def get_residual(self, seq, pair, kv_head, is_v, stream=None):
        cnt = C.c_int32(0)
        _check(_lib.fdkv_get_residual(self.h, seq, pair, kv_head, int(is_v), None, None, C.byref(cnt), _stream(stream)),
               "fdkv_get_residual")
        k = cnt.value
        idx = torch.empty(k, dtype=torch.int32, device=self.device)
        # a block of four layers keeps four values per position: [4, k]
        val = torch.empty((4, k) if self.block_size == 4 else (k,), dtype=self.tdtype, device=self.device)
        _check(_lib.fdkv_get_residual(self.h, seq, pair, kv_head, int(is_v), _ptr(idx), _ptr(val), C.byref(cnt),
                                      _stream(stream)), "fdkv_get_residual")
        return idx, val

    def get_token_set(self, seq, pair, kv_head, T, stream=None):
        """Token rule: (selected tokens int32 [k_tok] ascending, scores float32 [T]) of a staged, probed unit."""
        cnt = C.c_int32(0)
        _check(_lib.fdkv_get_token_set(self.h, seq, pair, kv_head, None, None, C.byref(cnt), _stream(stream)), "fdkv_get_token_set")
        tok = torch.empty(cnt.value, dtype=torch.int32, device=self.device)
        score = torch.empty(T, dtype=torch.float32, device=self.device)
        _check(_lib.fdkv_get_token_set(self.h, seq, pair, kv_head, _ptr(tok), _ptr(score), C.byref(cnt), _stream(stream)),
               "fdkv_get_token_set")
        return tok, score

    def get_modes(self, seq):
        n = self.n_pairs * self.cfg.n_kv_heads
        arr = (C.c_int32 * n)()
        _check(_lib.fdkv_get_modes(self.h, seq, arr), "fdkv_get_modes")
        return torch.tensor(list(arr), dtype=torch.int32).view(self.n_pairs, -1)

    def footprint(self, seq):
        by = (C.c_size_t * 3)()
        ex = C.c_size_t(0)
        _check(_lib.fdkv_footprint(self.h, seq, by, C.byref(ex)), "fdkv_footprint")
        return list(by), ex.value

    def decode_bytes(self, layer, batch):
        b = C.c_size_t(0)
        _check(_lib.fdkv_decode_bytes(self.h, layer, batch, C.byref(b)), "fdkv_decode_bytes")
        return b.value

    def device_status(self):
        return int(_lib.fdkv_device_status(self.h))

    # ---- test hooks (include/fdkv_testing.h) ----
    def test_wait_expiry(self, poll_cap: int, stream=None):
        """Runs a bounded device-side wait that nobody satisfies; device_status() then reports the timeout (7)."""
        _check(_lib.fdkv_test_wait_expiry(self.h, int(poll_cap), _stream(stream)), "fdkv_test_wait_expiry")

    def test_count_expiry(self, poll_cap: int, stream=None):
        """The same for the wait for a counter."""
        _check(_lib.fdkv_test_count_expiry(self.h, int(poll_cap), _stream(stream)), "fdkv_test_count_expiry")

    def test_clear_device_status(self, stream=None):
        _check(_lib.fdkv_test_clear_device_status(self.h, _stream(stream)), "fdkv_test_clear_device_status")
