"""Plain rows beside the clustered index: norm and rotary embedding of heads, a paged row cache, attention over it.

Argument marshalling only, like the rest of the binding: every method is one C call (two to four launches for attention) on
the stream that is current on the tensors' device.  Nothing synchronises, results and scratch come from torch's caching
allocator (so calls on several streams, and calls captured into several CUDA graphs, never share scratch).  The calls
compute no gradients and refuse, unless gradients are off, tensors that would need one: inputs, weights and cache rows alike.
"""
from __future__ import annotations

import ctypes as C
import math

from .binding import BF16, F32, FP8, DynaKVError, load_library

PAGE = 32          # rows per cache page
MAX_TREE = 256     # drafted tokens per sequence and call
MAX_CHUNK = 1 << 24


class _RowCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p), ("n_pages", C.c_int64),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("kv_dtype", C.c_int32)]


class _HeadRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("dtype", C.c_int32)]


class _Rotary(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("rotary_dim", C.c_int32),
                ("interleaved", C.c_int32), ("eps", C.c_float), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p),
                ("inv_freq", C.c_void_p)]


class _Scores(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p), ("rows_from", C.c_void_p),
                ("rows_to", C.c_void_p)]


_vp, _i32, _i64 = C.c_void_p, C.c_int32, C.c_int64
SIGNATURES = {
    "dynakv_norm_rope": (C.c_int, [_vp, _vp, _vp, _vp, _i64, _vp, _i32, _vp, _i32, _vp]),
    "dynakv_norm_rope_store": (C.c_int, [_vp, _vp, _vp, _vp, _vp, _i64, _vp, _i32, _vp, _vp, _vp, _vp]),
    "dynakv_rows_write": (C.c_int, [_vp, _vp, _vp, _vp, _i64, _vp, _vp]),
    "dynakv_rows_read": (C.c_int, [_vp, _vp, _i32, _vp, _i32, _i64, _i64, _vp, _vp, _vp, _vp]),
}
SIGNATURES["dynakv_attend_tree"] = (C.c_int, [_vp, _vp, _i32, _i64, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _i32, C.c_float, _vp, _vp, _vp, _i64, _vp, _vp])
SIGNATURES["dynakv_attend_tree_workspace"] = (_i64, [_vp, _i32, _i32])
SIGNATURES["dynakv_attend_chunk"] = (C.c_int, [_vp, _vp, _i32, _i64, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp])
SIGNATURES["dynakv_attend_chunk_workspace"] = (_i64, [_vp, _i32, _i64, _i32, _i32, _i32])
SIGNATURES["dynakv_rows_keep"] = (C.c_int, [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _vp])
SIGNATURES["dynakv_pages_extend"] = (C.c_int, [_vp, _vp, _i32, _vp, _vp, _i32, _i64, _vp, _vp, _vp, _vp, _vp])
SIGNATURES["dynakv_pages_trim"] = (C.c_int, [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp])
SIGNATURES["dynakv_verify_drafts"] = (C.c_int, [_vp, _i64, _i32, _i64, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp])
SIGNATURES["dynakv_verify_drafts_workspace"] = (_i64, [_i32, _i64, _i32, _i32, _i32])


class _Env:
    """What every call looks up, found once: the library's functions, torch's types, and torch's raw accessors of the current
    device and stream, which make no Python objects (some 2 us of a call that takes ten)."""

    def __init__(self):
        import torch
        L = load_library()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
            setattr(self, name, fn)
        self.library, self.torch = L, torch
        self.empty, self.i32, self.f32, self.bf16, self.i64, self.byte = torch.empty, torch.int32, torch.float32, torch.bfloat16, torch.int64, torch.uint8
        self.types = {torch.float32: F32, torch.bfloat16: BF16}
        self.grad = torch.is_grad_enabled
        stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.stream = stream if stream is not None else lambda device: torch.cuda.current_stream(device).cuda_stream
        self.device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_env_made = None


def _env() -> _Env:
    global _env_made
    if _env_made is None:
        _env_made = _Env()
    return _env_made


def _library():
    return _env().library


def _torch():
    import torch
    return torch


def _float_type(E, dtype, what: str) -> int:
    code = E.types.get(dtype)
    if code is None:
        raise DynaKVError(f"{what} is {dtype}: expected torch.float32 or torch.bfloat16")
    return code


def _index(E, t, shape: tuple, device: int, what: str) -> int:
    """A contiguous int32 tensor of `shape` on CUDA device `device`; its address."""
    if t.dtype is not E.i32 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise DynaKVError(f"expected {what} as a contiguous int32 tensor of shape {shape} on cuda:{device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(E, t, shape: tuple, device: int, dtype, code: int, what: str) -> _HeadRows:
    """A [n, heads, d] tensor whose last dimension is contiguous; the other strides are free."""
    stride = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or stride[2] != 1:
        raise DynaKVError(f"expected {what} as a {dtype} tensor of shape {shape} on cuda:{device} with a contiguous last dimension, "
                          f"got {t.dtype} {tuple(t.shape)} on {t.device}, strides {stride}")
    if t.requires_grad and E.grad():
        _no_gradient()
    return _HeadRows(t.data_ptr(), stride[0], stride[1], code)


def _no_gradient() -> None:
    raise DynaKVError("this call computes no gradients: detach its inputs or run it under torch.no_grad()")


def _overlap(a, b) -> bool:
    """Whether two contiguous tensors share memory."""
    x, y = a.data_ptr(), b.data_ptr()
    return x < y + b.numel() * b.element_size() and y < x + a.numel() * a.element_size()


class _Held:
    """The tensors that an object was made around, and what its calls check of them: their memory is where it was (not replaced by
    ``.data =`` or a resize of the storage) and none of them wants a gradient."""
    __slots__ = ("where", "leaves")

    def __init__(self, *tensors):
        tensors = [t for t in tensors if t is not None]
        self.where = tuple((t.data_ptr, t.data_ptr()) for t in tensors)         # bound methods: half the time of looking them up
        self.leaves = tuple(t for t in tensors if t.is_floating_point())

    def check(self, E) -> None:
        for now, then in self.where:
            if now() != then:
                raise DynaKVError("a tensor of this object has got other memory since the object was made: make a new one")
        for t in self.leaves:
            if t.requires_grad and E.grad():
                _no_gradient()


def _call(E, device: int, fn, *args) -> None:
    """One C call on the device's current stream (its last argument), with the device made current when it is not."""
    if E.device() == device:
        rc = fn(*args, E.stream(device))
    else:
        with E.torch.cuda.device(device):
            rc = fn(*args, E.stream(device))
    if rc != 0:
        raise DynaKVError(f"{fn.__name__} returned {rc}")


def _on_cuda(t, what: str):
    if not t.is_cuda:
        raise DynaKVError(f"{what} is on {t.device}: expected a CUDA tensor (there is no CPU fallback)")
    return t.device


class HeadRotary:
    """Norm and rotary embedding of a model's heads (``dynakv_norm_rope``).

    ``inv_freq`` [rotary_dim / 2] fp32: the angle of pair i at position p is p * inv_freq[i], taken in 64 bits;
    ``q_weight``, ``k_weight`` [head_dim] fp32: RMS norm of every head before the rotation (None: no norm).  Pairs are
    (i, i + rotary_dim / 2), or (2 i, 2 i + 1) with ``interleaved``; elements past rotary_dim are only normed."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, inv_freq, q_weight=None, k_weight=None, eps: float = 1e-6,
                 interleaved: bool = False):
        torch = _torch()
        self.n_heads, self.n_kv_heads, self.head_dim = int(n_heads), int(n_kv_heads), int(head_dim)
        if self.n_heads < 1 or self.n_kv_heads < 1 or self.head_dim not in (64, 128):
            raise DynaKVError(f"expected at least one query and KV head of 64 or 128 elements, got {n_heads}, {n_kv_heads}, {head_dim}")
        if not (eps >= 0.0 and math.isfinite(eps)):
            raise DynaKVError(f"eps is {eps}: expected a number >= 0")
        rotary_dim = 2 * inv_freq.numel()
        if rotary_dim > self.head_dim or rotary_dim % 16 != 0:
            raise DynaKVError(f"inv_freq has {inv_freq.numel()} elements: rotary_dim = {rotary_dim} has to be a multiple of 16 up to head_dim")
        self.device = _on_cuda(inv_freq, "inv_freq")
        self._device = inv_freq.get_device()
        for name, w, numel in (("inv_freq", inv_freq, rotary_dim // 2), ("q_weight", q_weight, self.head_dim), ("k_weight", k_weight, self.head_dim)):
            if w is not None and (w.dtype != torch.float32 or tuple(w.shape) != (numel,) or not w.is_contiguous() or w.device != self.device):
                raise DynaKVError(f"expected {name} as a contiguous float32 tensor of {numel} elements on {self.device}, got {w.dtype} {tuple(w.shape)} on {w.device}")
        self._held = _Held(inv_freq, q_weight, k_weight)
        self._c = _Rotary(self.n_heads, self.n_kv_heads, self.head_dim, rotary_dim, 1 if interleaved else 0, eps,
                          q_weight.data_ptr() if q_weight is not None else None,
                          k_weight.data_ptr() if k_weight is not None else None,
                          inv_freq.data_ptr() if rotary_dim else None)
        self._ref = C.byref(self._c)

    def _q_k(self, E, q, k):
        shape = q.shape
        if len(shape) != 3:
            raise DynaKVError(f"expected q of three dimensions, got {tuple(shape)}")
        self._held.check(E)
        n, dtype = shape[0], q.dtype
        code = _float_type(E, dtype, "q")
        return n, dtype, code, _heads(E, q, (n, self.n_heads, self.head_dim), self._device, dtype, code, "q"), \
            _heads(E, k, (n, self.n_kv_heads, self.head_dim), self._device, dtype, code, "k")

    def apply(self, q, k, positions, q_dtype=None, k_dtype=None):
        """q [n, heads, d], k [n, KV heads, d] (fp32 or bf16, any token and head strides), positions [n] int32 ->
        (q, k) normed and rotated, contiguous, of ``q_dtype`` and ``k_dtype`` (default: the input's).  With one token per
        sequence an fp32 q is what ``DynaKV.decode_step`` takes and k what ``DynaKV.append`` takes, as [U, G, d] and
        [U, d] views."""
        E, device = _env_made or _env(), self.device
        n, dtype, code, qr, kr = self._q_k(E, q, k)
        q_dtype, k_dtype = q_dtype or dtype, k_dtype or dtype
        qt = code if q_dtype is dtype else _float_type(E, q_dtype, "q_dtype")
        kt = code if k_dtype is dtype else _float_type(E, k_dtype, "k_dtype")
        place = _index(E, positions, (n,), self._device, "positions")
        q_out = E.empty((n, self.n_heads, self.head_dim), dtype=q_dtype, device=device)
        k_out = E.empty((n, self.n_kv_heads, self.head_dim), dtype=k_dtype, device=device)
        _call(E, self._device, E.dynakv_norm_rope, self._ref, C.byref(qr), C.byref(kr), place, n, q_out.data_ptr(), qt, k_out.data_ptr(), kt)
        return q_out, k_out

    def store(self, q, k, v, positions, cache: "RowCache", slots, q_dtype=None):
        """As ``apply``, with the keys and the values v [n, KV heads, d] going into ``slots`` [n] int32 of ``cache``
        (``RowCache.write``'s rules) in the same launch.  Returns q."""
        E = _env_made or _env()
        n, dtype, code, qr, kr = self._q_k(E, q, k)
        vr = _heads(E, v, (n, self.n_kv_heads, self.head_dim), self._device, dtype, code, "v")
        cache._held.check(E)
        if cache._device != self._device or cache.head_dim != self.head_dim or cache.n_kv_heads != self.n_kv_heads:
            raise DynaKVError(f"the cache holds {cache.n_kv_heads} heads of {cache.head_dim} on {cache.device}, the embedding has "
                              f"{self.n_kv_heads} of {self.head_dim} on {self.device}")
        q_dtype = q_dtype or dtype
        qt = code if q_dtype is dtype else _float_type(E, q_dtype, "q_dtype")
        place, slot = _index(E, positions, (n,), self._device, "positions"), _index(E, slots, (n,), self._device, "slots")
        q_out = E.empty((n, self.n_heads, self.head_dim), dtype=q_dtype, device=self.device)
        _call(E, self._device, E.dynakv_norm_rope_store, self._ref, C.byref(qr), C.byref(kr), C.byref(vr), place, n, q_out.data_ptr(), qt,
              cache._ref, slot, cache._status_at)
        return q_out


class RowCache:
    """A paged cache of K/V rows in fp32, bf16 or FP8 (``dynakv_row_cache``) around tensors the caller owns.

    k, v: [pages, KV heads, 32, head_dim], contiguous; float32, bfloat16, or for FP8 float8_e4m3fn (or uint8) with
    ``k_exp``, ``v_exp`` [pages, KV heads, 32] int8, the rows' power-of-two scales.  A slot is 32 * page + row.  What only
    the device can see (a page id, slot or length out of range) is skipped and sets a bit that ``get_status`` reads."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        torch = _torch()
        self.device = _on_cuda(k, "k")
        self._device = k.get_device()
        if k.dim() != 4 or k.shape[2] != PAGE or k.shape[3] not in (64, 128) or k.numel() == 0:
            raise DynaKVError(f"expected k of shape [pages, KV heads, {PAGE}, 64 or 128], got {tuple(k.shape)}")
        types = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8, torch.uint8: FP8}
        if k.dtype not in types:
            raise DynaKVError(f"k is {k.dtype}: expected float32, bfloat16 or float8_e4m3fn")
        if v.dtype != k.dtype or v.shape != k.shape or v.device != k.device or not (k.is_contiguous() and v.is_contiguous()):
            raise DynaKVError("expected k and v contiguous, of one type and shape on one device")
        self.kv_dtype = types[k.dtype]
        self.n_pages, self.n_kv_heads, _, self.head_dim = (int(x) for x in k.shape)
        for name, e in (("k_exp", k_exp), ("v_exp", v_exp)):
            if (e is None) != (self.kv_dtype != FP8):
                raise DynaKVError(f"{name} goes with FP8 rows, and only with them")
            if e is not None and (e.dtype != torch.int8 or tuple(e.shape) != tuple(k.shape[:3]) or not e.is_contiguous() or e.device != self.device):
                raise DynaKVError(f"expected {name} as a contiguous int8 tensor of shape {tuple(k.shape[:3])} on {self.device}")
        if self.n_pages * self.n_kv_heads >= 1 << 26:
            raise DynaKVError(f"{self.n_pages} pages x {self.n_kv_heads} heads: a cache holds fewer than 2^26 of them")
        if any(t is not None and t.data_ptr() % 16 for t in (k, v, k_exp, v_exp)):
            raise DynaKVError("the cache's tensors have to be 16-byte aligned")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self._held = _Held(k, v, k_exp, v_exp)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._status_at = self._status.data_ptr()
        self._c = _RowCache(k.data_ptr(), v.data_ptr(), k_exp.data_ptr() if k_exp is not None else None,
                            v_exp.data_ptr() if v_exp is not None else None, self.n_pages, self.n_kv_heads, self.head_dim, self.kv_dtype)
        self._ref = C.byref(self._c)
        self._io = torch.float32 if self.kv_dtype == F32 else torch.bfloat16      # type of q, of the results and of rows read
        self._byte, self._scale = torch.uint8, self.head_dim ** -0.5
        self._workspace = {}           # bytes attend_tree needs, by (heads, max_tree), and attend_chunk

    @classmethod
    def allocate(cls, n_pages: int, n_kv_heads: int, head_dim: int, kv_dtype: int = BF16, device="cuda") -> "RowCache":
        """A cache with tensors of its own, contents unspecified."""
        torch = _torch()
        if kv_dtype not in (F32, BF16, FP8):
            raise DynaKVError(f"kv_dtype is {kv_dtype}: expected F32, BF16 or FP8")
        shape = (n_pages, n_kv_heads, PAGE, head_dim)
        dtype = {F32: torch.float32, BF16: torch.bfloat16, FP8: torch.float8_e4m3fn}[kv_dtype]
        pools = [torch.empty(shape, dtype=dtype, device=device) for _ in range(2)]
        exps = [torch.empty(shape[:3], dtype=torch.int8, device=device) for _ in range(2)] if kv_dtype == FP8 else []
        return cls(*pools, *exps)

    def get_status(self) -> int:
        """The status bits set since the cache was made (``ST_BOUNDS``, ``ST_INTERNAL``).  Synchronises."""
        return int(self._status.item())

    def write(self, k, v, slots) -> None:
        """Rows k, v [n, KV heads, d] (fp32 or bf16, any token and head strides) into ``slots`` [n] int32, rounded to the
        cache's type.  A negative slot skips its token; slots >= 0 must differ."""
        shape = k.shape
        if len(shape) != 3:
            raise DynaKVError(f"expected k of three dimensions, got {tuple(shape)}")
        E, device = _env_made or _env(), self._device
        self._held.check(E)
        n, dtype = shape[0], k.dtype
        shape, code = (n, self.n_kv_heads, self.head_dim), _float_type(E, dtype, "k")
        kr, vr = _heads(E, k, shape, device, dtype, code, "k"), _heads(E, v, shape, device, dtype, code, "v")
        _call(E, device, E.dynakv_rows_write, self._ref, C.byref(kr), C.byref(vr), _index(E, slots, (n,), device, "slots"), n, self._status_at)

    def read(self, page_table, lengths, n: int, first: int = 0):
        """Rows [first, first + n) of every sequence in order, (K, V) of shape [sequences, KV heads, n, d], fp32 for an
        fp32 cache, else bf16; zeros at and past ``lengths`` [sequences] int32.  ``page_table`` [sequences, pages per
        sequence] int32.  As [U, n, d] views these are the K, V of ``DynaKV.build_index``."""
        E, device = _env_made or _env(), self._device
        self._held.check(E)
        rows = page_table.shape
        if len(rows) != 2 or n < 0 or first < 0:
            raise DynaKVError(f"expected page_table of two dimensions, n >= 0 and first >= 0, got {tuple(rows)}, {n}, {first}")
        b, per = rows
        table, lens = _index(E, page_table, (b, per), device, "page_table"), _index(E, lengths, (b,), device, "lengths")
        shape = (b, self.n_kv_heads, n, self.head_dim)
        K, V = E.empty(shape, dtype=self._io, device=self.device), E.empty(shape, dtype=self._io, device=self.device)
        _call(E, device, E.dynakv_rows_read, self._ref, table, per, lens, b, first, n, K.data_ptr(), V.data_ptr(), self._status_at)
        return K, V

    def keep(self, page_table, kv_len, q_start, path, kept) -> None:
        """Rows of accepted drafts moved together (``dynakv_rows_keep``): of every sequence's last q_start[b + 1] - q_start[b] rows, its
        tree's, row ``path`` [sequences, width] int32 [b, i] goes to row i for i < ``kept`` [sequences] int32.  Paths go upward from 0, as
        ``verify_drafts`` returns them."""
        E, device = _env_made or _env(), self._device
        self._held.check(E)
        rows, wide = page_table.shape, path.shape
        if len(rows) != 2 or len(wide) != 2:
            raise DynaKVError(f"expected page_table and path of two dimensions, got {tuple(rows)}, {tuple(wide)}")
        b, per = rows
        _call(E, device, E.dynakv_rows_keep, self._ref, _index(E, page_table, (b, per), device, "page_table"), per, _index(E, kv_len, (b,), device, "kv_len"),
              _index(E, q_start, (b + 1,), device, "q_start"), b, _index(E, path, (b, wide[1]), device, "path"), wide[1],
              _index(E, kept, (b,), device, "kept"), self._status_at)

    def attend_tree(self, q, page_table, kv_len, q_start, max_tree: int, tree_mask=None, scale=None, out=None, lse=None):
        """Attention of drafted tokens over the cache (``dynakv_attend_tree``): (out, lse).

        q [tokens, heads, d] (fp32 for an fp32 cache, else bf16), the tokens of all sequences one after the other:
        sequence b has tokens q_start[b] .. q_start[b + 1] - 1 (``q_start`` [sequences + 1] int32), at most ``max_tree`` of
        them; the last as many of its ``kv_len`` [sequences] int32 rows in ``page_table`` [sequences, pages] int32 are their own, the others the
        context, which every token sees.  ``tree_mask`` [tokens, words] int64: bit j of a token's words says that it
        sees row j of its tree (None: a chain, j <= i).  ``scale`` defaults to 1 / sqrt(d).  lse [tokens, heads]
        fp32 is the natural logarithm of the weights' sum, for merging with other calls of this kind.  A token that sees
        nothing gets zeros and -inf.  Tokens of no sequence (before q_start[0], behind the last sequence: a padded batch) are left as
        they are in ``out`` and ``lse``, so what they hold is unspecified in one that is not passed in.  Neither may share memory with
        the other or with anything that is read."""
        E, device = _env_made or _env(), self._device
        n, heads, b, per = self._queries(E, q, page_table, out, lse)
        size = self._workspace.get((heads, max_tree))
        if size is None:
            size = self._workspace_bytes(E, heads, max_tree)
        mask, words = None, 0
        if tree_mask is not None:
            words = tree_mask.shape[-1]
            if tree_mask.dtype is not E.i64 or tree_mask.shape != (n, words) or not 1 <= words <= MAX_TREE // 64 or \
                    not tree_mask.is_contiguous() or tree_mask.get_device() != device:
                raise DynaKVError(f"expected tree_mask as a contiguous int64 tensor [{n}, 1 to {MAX_TREE // 64}] on {self.device}, "
                                  f"got {tree_mask.dtype} {tuple(tree_mask.shape)} on {tree_mask.device}")
            mask = tree_mask.data_ptr()
        if scale is None:
            scale = self._scale
        elif not math.isfinite(scale):
            raise DynaKVError(f"scale is {scale}: expected a finite number")
        out, lse = self._results(E, q, out, lse)
        table, lens, start = _index(E, page_table, (b, per), device, "page_table"), _index(E, kv_len, (b,), device, "kv_len"), \
            _index(E, q_start, (b + 1,), device, "q_start")
        space = E.empty(size, dtype=self._byte, device=self.device)
        _call(E, device, E.dynakv_attend_tree, self._ref, q.data_ptr(), heads, n, start, b, max_tree, table, per, lens, mask, words, scale,
              out.data_ptr(), lse.data_ptr(), space.data_ptr(), size, self._status_at)
        return out, lse

    def attend_chunk(self, q, page_table, kv_len, q_start, max_chunk: int, scale=None, softcap: float = 0.0, window: int = 0, slopes=None,
                     rows_from=None, rows_to=None, out=None, lse=None):
        """Attention of a chunk of new tokens per sequence over the cache (``dynakv_attend_chunk``): (out, lse).

        q, ``q_start``, ``kv_len``, ``page_table``, ``scale``, ``out`` and ``lse`` as in ``attend_tree``, for chunks of any length up to
        ``max_chunk``: the last rows of a sequence are its tokens' own, token i's at P = kv_len - T + i.  It sees the rows before and
        at P, or with ``rows_to`` [tokens] int32 those before rows_to; of these with ``rows_from`` [tokens] int32 those from
        rows_from on, and with ``window`` the last so many up to P.  (Documents in one sequence: rows_from is the first row of the token's
        document; a prefix that all tokens see: rows_to = max(P + 1, prefix length).)  ``softcap``: logits s become
        softcap * tanh(s / softcap); ``slopes`` [heads] float32: then s - slope * |P - j| for row j.  A token that sees nothing gets
        zeros and -inf.  Over bf16 and FP8 rows, with more than 32 query rows per KV head (``max_chunk`` * heads / KV heads; rows of 64: 64), results
        are a little coarser than ``attend_tree``'s: weights enter the products with V as bf16, each off by 2^-8 of itself at most."""
        E, device = _env_made or _env(), self._device
        n, heads, b, per = self._queries(E, q, page_table, out, lse)
        size = self._workspace.get((heads, max_chunk, n, b, per))
        if size is None:
            size = self._chunk_workspace_bytes(E, heads, max_chunk, n, b, per)
        if scale is None:
            scale = self._scale
        if not (math.isfinite(scale) and (softcap == 0.0 or 2.0 ** -100 <= softcap <= 2.0 ** 100 and abs(scale / softcap) < 2.0 ** 127) and 0 <= window < 1 << 31):
            raise DynaKVError(f"scale is {scale}, softcap {softcap}, window {window}: expected finite numbers, softcap 0 or 2^-100 to 2^100, scale / softcap below 2^127, "
                              "window not negative")
        at_slopes = None
        if slopes is not None:
            if slopes.dtype is not E.f32 or slopes.shape != (heads,) or slopes.get_device() != device or not slopes.is_contiguous():
                raise DynaKVError(f"expected slopes as a contiguous float32 tensor of {heads} elements on {self.device}, got {slopes.dtype} {tuple(slopes.shape)} on {slopes.device}")
            if slopes.requires_grad and E.grad():
                _no_gradient()
            at_slopes = slopes.data_ptr()
        first = _index(E, rows_from, (n,), device, "rows_from") if rows_from is not None else None
        end = _index(E, rows_to, (n,), device, "rows_to") if rows_to is not None else None
        out, lse = self._results(E, q, out, lse)
        table, lens, start = _index(E, page_table, (b, per), device, "page_table"), _index(E, kv_len, (b,), device, "kv_len"), \
            _index(E, q_start, (b + 1,), device, "q_start")
        space = E.empty(size, dtype=self._byte, device=self.device)
        _call(E, device, E.dynakv_attend_chunk, self._ref, q.data_ptr(), heads, n, start, b, max_chunk, table, per, lens,
              C.byref(_Scores(scale, softcap, window, at_slopes, first, end)), out.data_ptr(), lse.data_ptr(), space.data_ptr(), size, self._status_at)
        return out, lse

    def _queries(self, E, q, page_table, out, lse):
        """What both kinds of attention check first: (tokens, heads, sequences, pages per sequence)."""
        shape = q.shape
        if len(shape) != 3 or shape[2] != self.head_dim or q.dtype is not self._io or not q.is_contiguous() or q.get_device() != self._device or q.data_ptr() % 16:
            raise DynaKVError(f"expected q as a contiguous, 16-byte aligned {self._io} tensor [tokens, heads, {self.head_dim}] on {self.device}, "
                              f"got {q.dtype} {tuple(q.shape)} on {q.device}")
        self._held.check(E)
        if E.grad() and (q.requires_grad or out is not None and out.requires_grad or lse is not None and lse.requires_grad):
            _no_gradient()
        rows = page_table.shape
        if len(rows) != 2:
            raise DynaKVError(f"expected page_table of two dimensions, got {tuple(rows)}")
        return shape[0], shape[1], rows[0], rows[1]

    def _results(self, E, q, out, lse):
        """(out, lse), checked or made."""
        n, heads, d = q.shape
        device, dtype = self._device, self._io
        if out is None:
            out = E.empty((n, heads, d), dtype=dtype, device=self.device)
        elif out.dtype is not dtype or out.shape != q.shape or not out.is_contiguous() or out.get_device() != device or out.data_ptr() % 16:
            raise DynaKVError(f"expected out as a contiguous, 16-byte aligned {dtype} tensor {tuple(q.shape)} on {self.device}")
        elif _overlap(out, q):
            raise DynaKVError("out shares memory with q")
        if lse is None:
            lse = E.empty((n, heads), dtype=E.f32, device=self.device)
        elif lse.dtype is not E.f32 or lse.shape != (n, heads) or not lse.is_contiguous() or lse.get_device() != device:
            raise DynaKVError(f"expected lse as a contiguous float32 tensor {(n, heads)} on {self.device}, got {lse.dtype} {tuple(lse.shape)} on {lse.device}")
        elif _overlap(lse, q) or _overlap(lse, out):
            raise DynaKVError("lse shares memory with q or out")
        return out, lse

    def _chunk_workspace_bytes(self, E, heads: int, max_chunk: int, n: int, b: int, per: int) -> int:
        if heads == 0 or heads % self.n_kv_heads != 0 or heads // self.n_kv_heads > 8:
            raise DynaKVError(f"{heads} query heads over {self.n_kv_heads} KV heads: expected 1 to 8 per KV head")
        if not 1 <= max_chunk <= MAX_CHUNK:
            raise DynaKVError(f"max_chunk is {max_chunk}: expected 1 to {MAX_CHUNK}")
        with E.torch.cuda.device(self._device):
            size = E.dynakv_attend_chunk_workspace(self._ref, heads, n, b, max_chunk, per)
        if size < 0:
            raise DynaKVError(f"dynakv_attend_chunk_workspace returned {size}")
        if len(self._workspace) >= 4096:       # lengths of prompts differ without end
            self._workspace.clear()
        self._workspace[heads, max_chunk, n, b, per] = size
        return size

    def _workspace_bytes(self, E, heads: int, max_tree: int) -> int:
        """Checks the two numbers that choose the kernel, and keeps the bytes of scratch that they come to."""
        if heads == 0 or heads % self.n_kv_heads != 0 or heads // self.n_kv_heads > 8:
            raise DynaKVError(f"{heads} query heads over {self.n_kv_heads} KV heads: expected 1 to 8 per KV head")
        if not 1 <= max_tree <= MAX_TREE:
            raise DynaKVError(f"max_tree is {max_tree}: expected 1 to {MAX_TREE}")
        with E.torch.cuda.device(self._device):
            size = E.dynakv_attend_tree_workspace(self._ref, heads, max_tree)
        if size < 0:
            raise DynaKVError(f"dynakv_attend_tree_workspace returned {size}")
        self._workspace[heads, max_tree] = size
        return size
