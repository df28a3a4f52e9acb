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
                ("lse", _VP)]


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
            out = (torch.empty((self.B, self.NE), dtype=torch.int32, device=self.device),
                   torch.empty((self.B, self.NE), dtype=torch.int32, device=self.device))
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
            out = (torch.empty((self.B, self.R + 1), dtype=torch.int32, device=self.device),
                   torch.empty((self.B, self.R + 1), dtype=torch.int32, device=self.device))
        par, tok = out
        _check(_LIB.rheo_pruned_view(self._h, _ptr(par), _ptr(tok), _stream(stream)))
        return par, tok

    def tree_mask(self, out=None, stream=None):
        """(mask [B][R+1][R+1] uint8, depth [B][R+1] int32) of the pruned tree."""
        n = self.R + 1
        if out is None:
            out = (torch.empty((self.B, n, n), dtype=torch.uint8, device=self.device),
                   torch.empty((self.B, n), dtype=torch.int32, device=self.device))
        mask, depth = out
        _check(_LIB.rheo_tree_mask(self._h, _ptr(mask), _ptr(depth), _stream(stream)))
        return mask, depth

    def verify(self, target_logits, T, rng_key, out=None, stream=None):
        if out is None:
            out = (torch.empty((self.B, self.D), dtype=torch.int32, device=self.device),
                   torch.empty((self.B,), dtype=torch.int32, device=self.device),
                   torch.empty((self.B,), dtype=torch.int32, device=self.device))
        acc, alen, fin = out
        _check(_LIB.rheo_verify(self._h, _ptr(target_logits), float(T),
                                int(rng_key) & (2 ** 64 - 1), _ptr(acc), _ptr(alen),
                                _ptr(fin), _stream(stream)))
        return acc, alen, fin

    def read_nodes(self, stream=None):
        shape = (self.B, self.N)
        dev = self.device
        out = {k: torch.empty(shape, dtype=torch.int32, device=dev)
               for k in ("token", "parent", "depth", "slot", "kind")}
        out.update({k: torch.empty(shape, dtype=torch.float64, device=dev)
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
    device, and a stream given by the caller is noted with the allocator."""

    def _device_of(self, device):
        device = torch.device(device)
        if device.type != "cuda":
            _refuse(f"device must be a GPU, got {device}")
        return torch.device("cuda", torch.cuda.current_device() if device.index is None
                            else device.index)

    def _dense(self, t, dtype, shape, name):
        """A contiguous tensor of exactly this type and shape."""
        if not isinstance(t, torch.Tensor):
            _refuse(f"{name} must be a tensor, got {type(t).__name__}")
        if t.device != self.device or t.dtype != dtype or tuple(t.shape) != tuple(shape):
            _refuse(f"{name} must be {dtype} {tuple(shape)} on {self.device}, got {t.dtype} "
                    f"{tuple(t.shape)} on {t.device}")
        if not t.is_contiguous():
            _refuse(f"{name} must be contiguous")
        return t

    def _launch(self, stream, tensors, call):
        """``call`` with the stream, noted for every tensor if it is not torch's own."""
        own = torch.cuda.current_stream(self.device)
        if stream is not None and stream != own:
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
        _check(call(ctypes.c_void_p((stream or own).cuda_stream)))

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
        self.device = self._device_of(device)
        self._destroy = lib.rheo_cache_destroy
        self._open(lambda h: lib.rheo_cache_create(ctypes.byref(cfg), h))
        self.B, self.H, self.K, self.D = batch, heads, kv_heads, head_dim
        self.page_size, self.pages, self.width = page_size, pages, table_width
        self.layers, self.dtype = layers, dtype
        self.page_stride = page_stride or page_size * kv_heads * head_dim
        self.layer_stride = layer_stride or pages * self.page_stride

    def _i32(self, t, shape, name):
        return None if t is None else self._dense(t, torch.int32, shape, name)

    def _out(self, t, dtype, shape, name):
        if t is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        return self._dense(t, dtype, shape, name)

    def _rows(self, t, n, heads, name):
        """[B, n, heads, head_dim] with dense heads; returns the stride of a row."""
        shape = (self.B, n, heads, self.D)
        if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype != self.dtype \
                or tuple(t.shape) != shape:
            _refuse(f"{name} must be {self.dtype} {shape} on {self.device}")
        row = t.stride(1) if n > 1 else t.stride(0) if self.B > 1 else heads * self.D
        if t.numel() and ((self.D > 1 and t.stride(3) != 1) or (heads > 1 and t.stride(2) != self.D)
                          or (self.B > 1 and t.stride(0) != n * row) or row < heads * self.D):
            _refuse(f"{name}: a row's heads must be dense and rows evenly apart over the batch")
        return row

    def _pages(self, t, name, layers=None):
        lead = () if layers is None else (layers,)
        shape = lead + (self.pages, self.page_size, self.K, self.D)
        if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype != self.dtype \
                or tuple(t.shape) != shape:
            _refuse(f"{name} must be {self.dtype} {shape} on {self.device}")
        want = (self.layer_stride,) if layers is not None else ()
        want += (self.page_stride, self.K * self.D, self.D, 1)
        if any(s != w for s, w, k in zip(t.stride(), want, shape) if k > 1):
            _refuse(f"{name} must have strides {want}, got {t.stride()}")
        return t

    def plan(self, lens, held, table, free_list, free_count, n, count=None, depth=None, out=None,
             stream=None):
        """Pages and slots for the next n rows of each sequence; (slots [B, n] int64,
        positions [B, n] int32, status [B] int32).  held, table, free_list and
        free_count are updated in place."""
        B = self.B
        self._i32(lens, (B,), "lens"), self._i32(held, (B,), "held")
        self._i32(table, (B, self.width), "table")
        self._i32(free_list, (self.pages,), "free_list")
        self._i32(free_count, (1,), "free_count")
        self._i32(count, (B,), "count"), self._i32(depth, (B, n), "depth")
        slots, positions, status = out or (None, None, None)
        slots = self._out(slots, torch.int64, (B, n), "slots")
        positions = self._out(positions, torch.int32, (B, n), "positions")
        status = self._out(status, torch.int32, (B,), "status")
        ts = (lens, count, depth, held, table, free_list, free_count, slots, positions, status)
        self._launch(stream, ts, lambda s: _LIB.rheo_cache_plan(
            self._h, n, *[_ptr(t) for t in ts], s))
        return slots, positions, status

    def write(self, q, k, v, slots, k_cache, v_cache, positions=None, rotation=None,
              interleaved=False, q_weight=None, k_weight=None, eps=1e-6, out=None, stream=None):
        """Head norms (where a weight is given), rotation (where a table is: [max_position,
        rot_dim] float32, cosines then sines) and store; returns the rotated q
        (``out``, which may be q itself), or None if q is None."""
        B, n = self.B, k.shape[1]
        a = WriteArgs(n=n, interleaved=int(interleaved), eps=float(eps))
        a.k_stride, a.v_stride = self._rows(k, n, self.K, "k"), self._rows(v, n, self.K, "v")
        if q is not None:
            a.q_stride = self._rows(q, n, self.H, "q")
            if out is None:
                out = torch.empty((B, n, self.H, self.D), dtype=self.dtype, device=self.device)
            a.q_out_stride = self._rows(out, n, self.H, "out")
        elif out is not None:
            _refuse("out without q")
        self._dense(slots, torch.int64, (B, n), "slots")
        if rotation is not None:
            if rotation.dim() != 2:
                _refuse("rotation must be [max_position, rot_dim]")
            self._dense(rotation, torch.float32, rotation.shape, "rotation")
            a.max_position, a.rot_dim = rotation.shape
            if positions is None:
                _refuse("rotation without positions")
        self._i32(positions, (B, n), "positions")
        for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if w is not None:
                self._dense(w, self.dtype, (self.D,), name)
        self._pages(k_cache, "k_cache"), self._pages(v_cache, "v_cache")
        ts = dict(q=q, k=k, v=v, q_out=out, slots=slots, positions=positions, rotation=rotation,
                  q_weight=q_weight, k_weight=k_weight, k_cache=k_cache, v_cache=v_cache)
        for name, t in ts.items():
            setattr(a, name, None if t is None else t.data_ptr())
        self._launch(stream, ts.values(),
                     lambda s: _LIB.rheo_cache_write(self._h, ctypes.byref(a), s))
        return out

    def attention(self, q, k_cache, v_cache, table, lens, mask=None, tail=None, count=None,
                  scale=None, out=None, lse=None, stream=None):
        """Attention of q [B, n, heads, head_dim] over each sequence's prefix (lens) and the
        ``tail`` entries behind it (by default the mask's columns, or n) that mask [B, n,
        tail] uint8 names; without a mask, causal.  Returns out, or (out, lse) where lse is
        True or a tensor [B, n, heads] float32.  scale: 1 / sqrt(head_dim) by default."""
        B, n = self.B, q.shape[1]
        a = AttentionArgs(n=n, scale=float(self.D ** -0.5 if scale is None else scale))
        a.q_stride = self._rows(q, n, self.H, "q")
        if mask is not None:
            a.tail = mask.shape[-1] if tail is None else tail
            self._dense(mask, torch.uint8, (B, n, a.tail), "mask")
        else:
            a.tail = n if tail is None else tail
        self._pages(k_cache, "k_cache"), self._pages(v_cache, "v_cache")
        self._i32(table, (B, self.width), "table")
        self._i32(lens, (B,), "lens"), self._i32(count, (B,), "count")
        if out is None:
            out = torch.empty((B, n, self.H, self.D), dtype=self.dtype, device=self.device)
        a.out_stride = self._rows(out, n, self.H, "out")
        both = lse is not None and lse is not False
        lse = self._out(None if lse is True else lse, torch.float32, (B, n, self.H), "lse") \
            if both else None
        # (an empty mask stands for one that names nothing)
        ts = dict(q=q, k_cache=k_cache, v_cache=v_cache, table=table, lens=lens, count=count,
                  out=out, lse=lse)
        for name, t in ts.items():
            setattr(a, name, None if t is None else t.data_ptr())
        if mask is not None:
            a.mask = mask.data_ptr() or table.data_ptr()
        self._launch(stream, list(ts.values()) + [mask],
                     lambda s: _LIB.rheo_tree_attention(self._h, ctypes.byref(a), s))
        return (out, lse) if both else out

    def commit(self, parent, token, accepted, accept_len, lens, table, k_cache, v_cache,
               out=None, stream=None):
        """Moves the entries of the accepted path together in all layers; (path [B, depth +
        1] int32, new lens [B] int32).  ``out``'s second tensor may be lens itself."""
        B, n, depth = self.B, parent.shape[-1], accepted.shape[-1]
        self._i32(parent, (B, n), "parent"), self._i32(token, (B, n), "token")
        self._i32(accepted, (B, depth), "accepted"), self._i32(accept_len, (B,), "accept_len")
        self._i32(lens, (B,), "lens"), self._i32(table, (B, self.width), "table")
        self._pages(k_cache, "k_cache", self.layers), self._pages(v_cache, "v_cache", self.layers)
        path, new_lens = out or (None, None)
        path = self._out(path, torch.int32, (B, depth + 1), "path")
        new_lens = self._out(new_lens, torch.int32, (B,), "new_lens")
        ts = (parent, token, accepted, accept_len, lens, table, k_cache, v_cache, path, new_lens)
        self._launch(stream, ts, lambda s: _LIB.rheo_cache_commit(
            self._h, n, depth, *[_ptr(t) for t in ts], s))
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
        self.device = self._device_of(device)
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
        B, n = logits.shape[:2]
        m = tokens.shape[-1]
        self._dense(logits, self.dtype, (B, n, self.row_stride), "logits")
        self._dense(tokens, torch.int32, (B, m), "tokens")
        if path is not None:
            self._dense(path, torch.int32, (B, m), "path")
        if not 0 <= top <= 32:
            _refuse("top must be in [0, 32]")
        want = [("logprob", torch.float32, (B, m)), ("entropy", torch.float32, (B, m)),
                ("rank", torch.int32, (B, m)), ("top_token", torch.int32, (B, m, top)),
                ("top_logprob", torch.float32, (B, m, top))]
        if out is None:
            out = [torch.zeros(s, dtype=d, device=self.device) for _, d, s in want]
        out = tuple(self._dense(t, d, s, name) for t, (name, d, s) in zip(out, want))
        self._launch(stream, (logits, path, tokens) + out, lambda s: _LIB.rheo_token_logprobs(
            self._h, _ptr(logits), B, n, _ptr(path), _ptr(tokens), m, top, float(T),
            *[_ptr(t) for t in out], s))
        return out
