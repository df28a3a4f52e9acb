"""Python binding of librheo.so (the C ABI in include/rheo.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  torch supplies device buffers (``data_ptr``) and the HIP stream
(``torch.cuda.current_stream().cuda_stream``).  Importing this module fails
loudly when the library has not been built.
"""

import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librheo.so")

RHEO_OK, RHEO_EINVAL, RHEO_ENOMEM, RHEO_EHIP, RHEO_ESTATE = 0, -1, -2, -3, -4
RHEO_F32, RHEO_BF16, RHEO_F16 = 0, 1, 2
RHEO_METHOD_RHEO, RHEO_METHOD_RRSW, RHEO_METHOD_TOPK = 0, 1, 2
METHODS = {"rheo": RHEO_METHOD_RHEO, "rrsw": RHEO_METHOD_RRSW, "topk": RHEO_METHOD_TOPK}
ERROR_NAMES = {RHEO_EINVAL: "EINVAL", RHEO_ENOMEM: "ENOMEM", RHEO_EHIP: "EHIP",
               RHEO_ESTATE: "ESTATE"}

# every symbol the header declares
EXPORTS = ["rheo_create", "rheo_create_static", "rheo_destroy", "rheo_begin_step", "rheo_expand_level",
           "rheo_frontier", "rheo_frontier_view", "rheo_prune", "rheo_pruned_view",
           "rheo_tree_mask", "rheo_verify",
           "rheo_read_nodes", "rheo_device_error", "rheo_node_count",
           "rheo_cache_create", "rheo_cache_destroy", "rheo_cache_error", "rheo_cache_plan",
           "rheo_cache_write", "rheo_tree_attention", "rheo_cache_commit",
           "rheo_cache_commit_served",
           "rheo_scorer_create", "rheo_scorer_destroy", "rheo_token_logprobs",
           "rheo_last_error"]


class RheoConfig(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("pool", ctypes.c_int32), ("leads", ctypes.c_int32),
                ("depth", ctypes.c_int32), ("n_expand", ctypes.c_int32),
                ("support", ctypes.c_int32), ("construct_tempered", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("method", ctypes.c_int32),
                ("construct_full", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("eps_m0", ctypes.c_double)]


class CacheConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "heads", "kv_heads", "head_dim", "page_size", "pages", "table_width",
        "layers", "dtype")] + [("page_stride", ctypes.c_int64), ("layer_stride", ctypes.c_int64)]


_VP, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class WriteArgs(ctypes.Structure):
    _fields_ = [("n", _I32), ("rot_dim", _I32), ("max_position", _I32), ("interleaved", _I32),
                ("q", _VP), ("k", _VP), ("v", _VP), ("q_out", _VP), ("q_stride", _I64),
                ("k_stride", _I64), ("v_stride", _I64), ("q_out_stride", _I64), ("slots", _VP),
                ("positions", _VP), ("rotation", _VP), ("q_weight", _VP), ("k_weight", _VP),
                ("eps", _F32), ("k_cache", _VP), ("v_cache", _VP)]


class AttentionArgs(ctypes.Structure):
    _fields_ = [("n", _I32), ("tail", _I32), ("q", _VP), ("q_stride", _I64),
                ("out_stride", _I64), ("k_cache", _VP), ("v_cache", _VP), ("table", _VP),
                ("lens", _VP), ("count", _VP), ("mask", _VP), ("scale", _F32), ("out", _VP),
                ("lse", _VP), ("status", _VP)]


class RheoError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {msg}")
        self.code = code


_LIB = None


def load_library(path=LIB_PATH):
    """Loads librheo.so (raises if it is missing) and declares signatures."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with "
                          "`python -m paper_2609_21827_amd.build` first")
    lib = ctypes.CDLL(path)
    vp, i32, u64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_float
    sig = {
        "rheo_create": ([ctypes.POINTER(RheoConfig), ctypes.POINTER(vp)], ctypes.c_int),
        "rheo_create_static": ([ctypes.POINTER(RheoConfig), ctypes.POINTER(vp)], ctypes.c_int),
        "rheo_destroy": ([vp], ctypes.c_int),
        "rheo_begin_step": ([vp], ctypes.c_int),
        "rheo_expand_level": ([vp, vp, f32, u64, vp], ctypes.c_int),
        "rheo_frontier": ([vp, vp, vp, vp], ctypes.c_int),
        "rheo_frontier_view": ([vp, ctypes.POINTER(vp), ctypes.POINTER(vp)], ctypes.c_int),
        "rheo_prune": ([vp, i32, vp], ctypes.c_int),
        "rheo_pruned_view": ([vp, vp, vp, vp], ctypes.c_int),
        "rheo_tree_mask": ([vp, vp, vp, vp], ctypes.c_int),
        "rheo_verify": ([vp, vp, f32, u64, vp, vp, vp, vp], ctypes.c_int),
        "rheo_read_nodes": ([vp] * 10, ctypes.c_int),
        "rheo_device_error": ([vp, ctypes.POINTER(ctypes.c_int32)], ctypes.c_int),
        "rheo_node_count": ([vp], ctypes.c_int32),
        "rheo_cache_create": ([ctypes.POINTER(CacheConfig), ctypes.POINTER(vp)], ctypes.c_int),
        "rheo_cache_destroy": ([vp], ctypes.c_int),
        "rheo_cache_error": ([vp, ctypes.POINTER(ctypes.c_int32)], ctypes.c_int),
        "rheo_cache_plan": ([vp, i32] + [vp] * 11, ctypes.c_int),
        "rheo_cache_write": ([vp, ctypes.POINTER(WriteArgs), vp], ctypes.c_int),
        "rheo_tree_attention": ([vp, ctypes.POINTER(AttentionArgs), vp], ctypes.c_int),
        "rheo_cache_commit": ([vp, i32, i32] + [vp] * 11, ctypes.c_int),
        "rheo_cache_commit_served": ([vp, i32, i32] + [vp] * 12, ctypes.c_int),
        "rheo_scorer_create": ([i32, i32, ctypes.c_int64, ctypes.POINTER(vp)], ctypes.c_int),
        "rheo_scorer_destroy": ([vp], ctypes.c_int),
        "rheo_token_logprobs": ([vp, vp, i32, i32, vp, vp, i32, i32, f32] + [vp] * 6, ctypes.c_int),
        "rheo_last_error": ([], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _LIB = lib
    return lib


def _check(code):
    if code != RHEO_OK:
        raise RheoError(code, _LIB.rheo_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _output(shape, dtype, device, stream, make=torch.empty):
    """A new output of a call on `stream` (None: torch's current one).

    Memory comes back to the allocator while the stream that it was made on has still
    work on it to do, and a fill is work of its own: both are in order only for calls
    on that very stream.  So the output is made on the call's stream, and torch's
    current stream, where the caller reads it, is noted with it."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    reader = torch.cuda.current_stream(device)
    if stream.cuda_stream == reader.cuda_stream:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = make(shape, dtype=dtype, device=device)
    t.record_stream(reader)
    return t


def _current_stream(index):
    """The address of torch's current stream on a device."""
    return _RAW_STREAM(index) if _RAW_STREAM else torch.cuda.current_stream(index).cuda_stream


_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


class _CudaArray:
    """A device int32 array exposed through __cuda_array_interface__."""

    def __init__(self, ptr, shape):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": "<i4",
                                         "data": (int(ptr), False), "version": 3,
                                         "strides": None}


def _device_view(ptr, shape, device):
    return torch.as_tensor(_CudaArray(ptr, shape), device=device)


class Tree:
    """One tree handle: B sequences, fixed shape, reused step after step."""

    def __init__(self, batch, vocab, pool, leads, depth, support, dtype,
                 n_expand=0, construct_tempered=False, row_stride=None,
                 eps_m0=0.0, method="rheo", construct_full=False, device="cuda",
                 static=False):
        lib = load_library()
        self.device = torch.device(device)
        self.B, self.V, self.K, self.m, self.D = batch, vocab, pool, leads, depth
        self.NE = n_expand or pool
        self.dtype = dtype
        self.row_stride = row_stride or vocab
        cfg = RheoConfig(batch, vocab, pool, leads, depth, n_expand, support,
                         int(construct_tempered),
                         RHEO_BF16 if dtype == torch.bfloat16 else RHEO_F32,
                         METHODS[method] if isinstance(method, str) else int(method),
                         int(construct_full), self.row_stride, eps_m0)
        h = ctypes.c_void_p()
        # static: the device state in the library's static scratch array
        create = lib.rheo_create_static if static else lib.rheo_create
        _check(create(ctypes.byref(cfg), ctypes.byref(h)))
        self._h = h
        self.N = lib.rheo_node_count(h)
        self.R = None

    def close(self):
        if getattr(self, "_h", None):
            _LIB.rheo_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def begin_step(self):
        _check(_LIB.rheo_begin_step(self._h))

    def expand_level(self, draft_logits, T, rng_key, stream=None):
        _check(_LIB.rheo_expand_level(self._h, _ptr(draft_logits), float(T),
                                      int(rng_key) & (2 ** 64 - 1), _stream(stream)))

    def frontier(self, out=None, stream=None):
        if out is None:
            out = tuple(_output((self.B, self.NE), torch.int32, self.device, stream)
                        for _ in range(2))
        par, tok = out
        _check(_LIB.rheo_frontier(self._h, _ptr(par), _ptr(tok), _stream(stream)))
        return par, tok

    def frontier_view(self):
        """The tree-owned frontier arrays as int32 [B, n_expand] tensors
        (zero-copy views; contents change with every expand below the last
        level)."""
        par, tok = ctypes.c_void_p(), ctypes.c_void_p()
        _check(_LIB.rheo_frontier_view(self._h, ctypes.byref(par), ctypes.byref(tok)))
        return (_device_view(par.value, (self.B, self.NE), self.device),
                _device_view(tok.value, (self.B, self.NE), self.device))

    def prune(self, budget, stream=None):
        _check(_LIB.rheo_prune(self._h, int(budget), _stream(stream)))
        self.R = int(budget)

    def pruned_view(self, out=None, stream=None):
        if out is None:
            out = tuple(_output((self.B, self.R + 1), torch.int32, self.device, stream)
                        for _ in range(2))
        par, tok = out
        _check(_LIB.rheo_pruned_view(self._h, _ptr(par), _ptr(tok), _stream(stream)))
        return par, tok

    def tree_mask(self, out=None, stream=None):
        """(mask [B][R+1][R+1] uint8, depth [B][R+1] int32) of the pruned tree."""
        n = self.R + 1
        if out is None:
            out = (_output((self.B, n, n), torch.uint8, self.device, stream),
                   _output((self.B, n), torch.int32, self.device, stream))
        mask, depth = out
        _check(_LIB.rheo_tree_mask(self._h, _ptr(mask), _ptr(depth), _stream(stream)))
        return mask, depth

    def verify(self, target_logits, T, rng_key, out=None, stream=None):
        if out is None:
            out = tuple(_output(shape, torch.int32, self.device, stream)
                        for shape in ((self.B, self.D), (self.B,), (self.B,)))
        acc, alen, fin = out
        _check(_LIB.rheo_verify(self._h, _ptr(target_logits), float(T),
                                int(rng_key) & (2 ** 64 - 1), _ptr(acc), _ptr(alen),
                                _ptr(fin), _stream(stream)))
        return acc, alen, fin

    def read_nodes(self, stream=None):
        shape = (self.B, self.N)
        dev = self.device
        out = {k: _output(shape, torch.int32, dev, stream)
               for k in ("token", "parent", "depth", "slot", "kind")}
        out.update({k: _output(shape, torch.float64, dev, stream)
                    for k in ("proxy", "qtrue", "score")})
        _check(_LIB.rheo_read_nodes(self._h, *[_ptr(out[k]) for k in (
            "token", "parent", "depth", "slot", "kind", "proxy", "qtrue", "score")],
            _stream(stream)))
        return out

    def device_error(self):
        flag = ctypes.c_int32(0)
        _check(_LIB.rheo_device_error(self._h, ctypes.byref(flag)))
        return flag.value


_DTYPES = {torch.float32: RHEO_F32, torch.bfloat16: RHEO_BF16, torch.float16: RHEO_F16}


def _dtype_code(dtype):
    if dtype not in _DTYPES:
        raise RheoError(RHEO_EINVAL, f"unknown dtype {dtype}")
    return _DTYPES[dtype]


def _refuse(msg):
    raise RheoError(RHEO_EINVAL, msg)


class _OnDevice:
    """What the handles below share: tensors are checked for place, type, shape and
    layout (nothing is copied or converted), outputs are allocated on the handle's
    device, in the order of the stream that the call runs on, and a stream given by
    the caller is noted with the allocator.

    A call is some 5 us of checks and marshalling beside kernels of 4 us, so the
    checks are few and plain: get_device() and `is` instead of device and dtype
    objects compared, addresses as plain numbers."""

    def _set_device(self, device):
        device = torch.device(device)
        if device.type != "cuda":
            _refuse(f"device must be a GPU, got {device}")
        self._index = torch.cuda.current_device() if device.index is None else device.index
        self.device = torch.device("cuda", self._index)

    def _dense(self, t, dtype, shape, name):
        """The address of a contiguous tensor of exactly this type and shape."""
        if not isinstance(t, torch.Tensor):
            _refuse(f"{name} must be a tensor, got {type(t).__name__}")
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index:
            _refuse(f"{name} must be {dtype} {tuple(shape)} on {self.device}, got {t.dtype} "
                    f"{tuple(t.shape)} on {t.device}")
        if not t.is_contiguous():
            _refuse(f"{name} must be contiguous")
        return t.data_ptr()

    def _aside(self, stream):
        """Whether a stream is another than torch's current one; it has to be of the
        handle's device, since its outputs are made and its kernels run there."""
        if stream.device_index != self._index:
            _refuse(f"stream must be of {self.device}, got one of device {stream.device_index}")
        return stream.cuda_stream != _current_stream(self._index)

    def _new(self, dtype, shape, stream, make=torch.empty):
        """A new output of a call on `stream`, which is of the handle's device."""
        if stream is not None:
            self._aside(stream)
        return _output(shape, dtype, self.device, stream, make)

    def _made(self, t, dtype, shape, name, stream):
        """(tensor, address) of an output, allocated unless given."""
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=self.device) if stream is None else \
                self._new(dtype, shape, stream)
            return t, t.data_ptr()
        return t, self._dense(t, dtype, shape, name)

    def _stream(self, stream, tensors):
        """The stream to launch on; one that is not torch's current is noted for the
        tensors, so that their memory is not used again before its work has run."""
        if stream is None:
            return _current_stream(self._index)
        if self._aside(stream):
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
        return stream.cuda_stream

    def _open(self, create):
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(create(ctypes.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache(_OnDevice):
    """The paged key/value cache of B sequences (see "The key/value cache around a
    drafted tree" in rheo.h).  The caller owns the tensors:

    k_cache, v_cache  one layer's pages [pages, page_size, kv_heads, head_dim], or
                      for ``commit`` all layers' [layers, pages, ...]
    table             [B, table_width] int32, lens, held [B] int32
    free_list         [pages] int32, free_count [1] int32
    """

    def __init__(self, batch, heads, kv_heads, head_dim, page_size, pages, table_width,
                 layers=1, dtype=torch.bfloat16, page_stride=0, layer_stride=0, device="cuda"):
        lib = load_library()
        cfg = CacheConfig(batch, heads, kv_heads, head_dim, page_size, pages, table_width, layers,
                          _dtype_code(dtype), page_stride, layer_stride)
        self._set_device(device)
        self._destroy = lib.rheo_cache_destroy
        self._open(lambda h: lib.rheo_cache_create(ctypes.byref(cfg), h))
        self.B, self.H, self.K, self.D = batch, heads, kv_heads, head_dim
        self.page_size, self.pages, self.width = page_size, pages, table_width
        self.layers, self.dtype = layers, dtype
        self.page_stride = page_stride or page_size * kv_heads * head_dim
        self.layer_stride = layer_stride or pages * self.page_stride
        self._page_shape = (pages, page_size, kv_heads, head_dim)
        self._page_strides = (self.page_stride, kv_heads * head_dim, head_dim, 1)

    def _i32(self, t, shape, name):
        return None if t is None else self._dense(t, torch.int32, shape, name)

    def _rows(self, t, n, heads, name):
        """(address, elements between rows) of [B, n, heads, head_dim] with dense heads."""
        B, D, shape = self.B, self.D, (self.B, n, heads, self.D)
        if not isinstance(t, torch.Tensor) or t.dtype is not self.dtype or t.shape != shape \
                or t.get_device() != self._index:
            _refuse(f"{name} must be {self.dtype} {shape} on {self.device}")
        s0, s1, s2, s3 = t.stride()
        row = s1 if n > 1 else s0 if B > 1 else heads * D
        if n and (s3 != 1 or (heads > 1 and s2 != D) or (B > 1 and s0 != n * row)
                  or row < heads * D):
            _refuse(f"{name}: a row's heads must be dense and rows evenly apart over the batch")
        return t.data_ptr(), row

    def _pages(self, t, name, layers=None):
        shape, want = self._page_shape, self._page_strides
        if layers is not None:
            shape, want = (layers,) + shape, (self.layer_stride,) + want
        if not isinstance(t, torch.Tensor) or t.dtype is not self.dtype or t.shape != shape \
                or t.get_device() != self._index:
            _refuse(f"{name} must be {self.dtype} {shape} on {self.device}")
        if t.stride() != want and any(s != w for s, w, k in zip(t.stride(), want, shape) if k > 1):
            _refuse(f"{name} must have strides {want}, got {t.stride()}")
        return t.data_ptr()

    def plan(self, lens, held, table, free_list, free_count, n, count=None, depth=None, out=None,
             stream=None):
        """Pages and slots for the next n rows of each sequence; (slots [B, n] int64,
        positions [B, n] int32, status [B] int32).  held, table, free_list and
        free_count are updated in place.  A sequence of status not 0 has no place for its
        rows; attention and commit are given the status, or they meet pages of others."""
        B, i32 = self.B, self._i32
        one, rows = (B,), (B, n)
        slots, positions, status = out or (None, None, None)
        slots, p_slots = self._made(slots, torch.int64, rows, "slots", stream)
        positions, p_positions = self._made(positions, torch.int32, rows, "positions", stream)
        status, p_status = self._made(status, torch.int32, one, "status", stream)
        _check(_LIB.rheo_cache_plan(
            self._h, n, i32(lens, one, "lens"), i32(count, one, "count"), i32(depth, rows, "depth"),
            i32(held, one, "held"), i32(table, (B, self.width), "table"),
            i32(free_list, (self.pages,), "free_list"), i32(free_count, (1,), "free_count"),
            p_slots, p_positions, p_status,
            self._stream(stream, (lens, count, depth, held, table, free_list, free_count, slots,
                                  positions, status))))
        return slots, positions, status

    def write(self, q, k, v, slots, k_cache, v_cache, positions=None, rotation=None,
              interleaved=False, q_weight=None, k_weight=None, eps=1e-6, out=None, stream=None):
        """Head norms (where a weight is given), rotation (where a table is: [max_position,
        rot_dim] float32, cosines then sines) and store; returns the rotated q
        (``out``, which may be q itself), or None if q is None."""
        B, n, dim = self.B, k.shape[1], (self.D,)
        p_k, k_row = self._rows(k, n, self.K, "k")
        p_v, v_row = self._rows(v, n, self.K, "v")
        p_q = p_out = q_row = out_row = 0
        if q is not None:
            p_q, q_row = self._rows(q, n, self.H, "q")
            if out is None:
                out = self._new(self.dtype, (B, n, self.H, self.D), stream)
            p_out, out_row = self._rows(out, n, self.H, "out")
        elif out is not None:
            _refuse("out without q")
        rot_dim = most = 0
        p_rotation = None
        if rotation is not None:
            if rotation.dim() != 2:
                _refuse("rotation must be [max_position, rot_dim]")
            p_rotation = self._dense(rotation, torch.float32, rotation.shape, "rotation")
            most, rot_dim = rotation.shape
            if positions is None:
                _refuse("rotation without positions")
        a = WriteArgs(
            n, rot_dim, most, int(interleaved), p_q or None, p_k, p_v, p_out or None, q_row, k_row,
            v_row, out_row, self._dense(slots, torch.int64, (B, n), "slots"),
            self._i32(positions, (B, n), "positions"), p_rotation,
            None if q_weight is None else self._dense(q_weight, self.dtype, dim, "q_weight"),
            None if k_weight is None else self._dense(k_weight, self.dtype, dim, "k_weight"),
            float(eps), self._pages(k_cache, "k_cache"), self._pages(v_cache, "v_cache"))
        _check(_LIB.rheo_cache_write(
            self._h, ctypes.byref(a),
            self._stream(stream, (q, k, v, out, slots, positions, rotation, q_weight, k_weight,
                                  k_cache, v_cache))))
        return out

    def attention(self, q, k_cache, v_cache, table, lens, mask=None, tail=None, count=None,
                  scale=None, out=None, lse=None, status=None, stream=None):
        """Attention of q [B, n, heads, head_dim] over each sequence's prefix (lens) and the
        ``tail`` entries behind it (by default the mask's columns, or n) that mask [B, n,
        tail] uint8 names; without a mask, causal.  Returns out, or (out, lse) where lse is
        True or a tensor [B, n, heads] float32.  scale: 1 / sqrt(head_dim) by default.
        status: the plan's; sequences that it did not serve are left out."""
        B, n = self.B, q.shape[1]
        p_q, q_row = self._rows(q, n, self.H, "q")
        if tail is None:
            tail = n if mask is None else mask.shape[-1]
        p_table = self._i32(table, (B, self.width), "table")
        p_mask = None
        if mask is not None:         # (one without columns has no address, but names nothing)
            p_mask = self._dense(mask, torch.uint8, (B, n, tail), "mask") or p_table
        if out is None:
            out = self._new(self.dtype, (B, n, self.H, self.D), stream)
        p_out, out_row = self._rows(out, n, self.H, "out")
        both, p_lse = lse is not None and lse is not False, None
        if both:
            lse, p_lse = self._made(None if lse is True else lse, torch.float32, (B, n, self.H),
                                    "lse", stream)
        a = AttentionArgs(
            n, tail, p_q, q_row, out_row, self._pages(k_cache, "k_cache"),
            self._pages(v_cache, "v_cache"), p_table, self._i32(lens, (B,), "lens"),
            self._i32(count, (B,), "count"), p_mask,
            float(self.D ** -0.5 if scale is None else scale), p_out, p_lse,
            self._i32(status, (B,), "status"))
        _check(_LIB.rheo_tree_attention(
            self._h, ctypes.byref(a),
            self._stream(stream, (q, k_cache, v_cache, table, lens, count, mask, out,
                                  lse if both else None, status))))
        return (out, lse) if both else out

    def commit(self, parent, token, accepted, accept_len, lens, table, k_cache, v_cache,
               out=None, status=None, stream=None):
        """Moves the entries of the accepted path together in all layers; (path [B, depth +
        1] int32, new lens [B] int32).  ``out``'s second tensor may be lens itself.
        status: the plan's; sequences that it did not serve keep entries and length."""
        B, n, depth, i32 = self.B, parent.shape[-1], accepted.shape[-1], self._i32
        one, rows = (B,), (B, n)
        path, new_lens = out or (None, None)
        path, p_path = self._made(path, torch.int32, (B, depth + 1), "path", stream)
        new_lens, p_new = self._made(new_lens, torch.int32, one, "new_lens", stream)
        _check(_LIB.rheo_cache_commit_served(
            self._h, n, depth, i32(parent, rows, "parent"), i32(token, rows, "token"),
            i32(accepted, (B, depth), "accepted"), i32(accept_len, one, "accept_len"),
            i32(lens, one, "lens"), i32(table, (B, self.width), "table"), i32(status, one, "status"),
            self._pages(k_cache, "k_cache", self.layers),
            self._pages(v_cache, "v_cache", self.layers), p_path, p_new,
            self._stream(stream, (parent, token, accepted, accept_len, lens, table, status, k_cache,
                                  v_cache, path, new_lens))))
        return path, new_lens

    def device_error(self):
        flag = ctypes.c_int32(0)
        _check(_LIB.rheo_cache_error(self._h, ctypes.byref(flag)))
        return flag.value


class Scorer(_OnDevice):
    """Log probabilities of given tokens in rows of ``vocab`` logits (rheo_token_logprobs)."""

    def __init__(self, vocab, dtype, row_stride=None, device="cuda"):
        lib = load_library()
        code = _dtype_code(dtype)
        self._set_device(device)
        self._destroy = lib.rheo_scorer_destroy
        self.V, self.dtype, self.row_stride = vocab, dtype, row_stride or vocab
        self._open(lambda h: lib.rheo_scorer_create(vocab, code, self.row_stride, h))

    def logprobs(self, logits, tokens, path=None, top=0, T=1.0, out=None, stream=None):
        """Of tokens [B, m] int32 in rows path [B, m] (or 0..m-1) of logits [B, n, row_stride]:
        (logprob, entropy [B, m] float32, rank [B, m] int32, top_token [B, m, top] int32,
        top_logprob [B, m, top] float32).  Entries with a path or token out of range, as -1,
        are left as they were (new outputs: zeros)."""
        if not isinstance(logits, torch.Tensor) or logits.dim() != 3:
            _refuse("logits must be a tensor [B, n, row_stride]")
        if not 0 <= top <= 32:
            _refuse("top must be in [0, 32]")
        B, n = logits.shape[:2]
        m = tokens.shape[-1]
        one, best = (B, m), (B, m, top)
        want = (("logprob", torch.float32, one), ("entropy", torch.float32, one),
                ("rank", torch.int32, one), ("top_token", torch.int32, best),
                ("top_logprob", torch.float32, best))
        if out is None:
            out = tuple(self._new(d, s, stream, torch.zeros) for _, d, s in want)
        if len(out) != len(want):
            _refuse(f"out must be {len(want)} tensors")
        _check(_LIB.rheo_token_logprobs(
            self._h, self._dense(logits, self.dtype, (B, n, self.row_stride), "logits"), B, n,
            None if path is None else self._dense(path, torch.int32, one, "path"),
            self._dense(tokens, torch.int32, one, "tokens"), m, top, float(T),
            *[self._dense(t, d, s, name) for t, (name, d, s) in zip(out, want)],
            self._stream(stream, (logits, path, tokens, *out))))
        return tuple(out)
