"""Around the paged row cache's attention: pages and slots for new tokens, and which drafted tokens are kept.

Argument marshalling only: every call is one C call on the stream that is current on the tensors' device, and nothing synchronises.
"""
from __future__ import annotations

import ctypes as C

from . import rows as _rows
from .binding import DynaKVError
from .rows import MAX_TREE, _call, _Held, _index, _no_gradient, _on_cuda, _torch


class _Pool(C.Structure):
    _fields_ = [("free_pages", C.c_void_p), ("count", C.c_void_p), ("n_pages", C.c_int64)]


class PagePool:
    """The free pages of a ``RowCache`` (``dynakv_page_pool``) around tensors the caller owns: the first ``count`` [1] int32 entries
    of ``free`` [pages] int32, taken and given back at the end.  What only the device can see (lengths out of range, too few pages) leaves the sequences
    concerned as they are and sets a bit that ``get_status`` reads."""

    def __init__(self, free, count):
        torch = _torch()
        self.device = _on_cuda(free, "free")
        self._device = free.get_device()
        if free.dim() != 1 or not 1 <= free.numel() < 1 << 26 or free.dtype != torch.int32 or not free.is_contiguous():
            raise DynaKVError(f"expected free as a contiguous int32 tensor of 1 to 2^26 - 1 pages, got {free.dtype} {tuple(free.shape)}")
        if count.dtype != torch.int32 or tuple(count.shape) != (1,) or count.device != self.device:
            raise DynaKVError(f"expected count as an int32 tensor of one element on {self.device}, got {count.dtype} {tuple(count.shape)} on {count.device}")
        self.free, self.count, self.n_pages = free, count, free.numel()
        self._held = _Held(free, count)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._status_at = self._status.data_ptr()
        self._c = _Pool(free.data_ptr(), count.data_ptr(), self.n_pages)
        self._ref = C.byref(self._c)

    @classmethod
    def allocate(cls, n_pages: int, device="cuda") -> "PagePool":
        """A pool in which pages 0 .. n_pages - 1 are free, page 0 the first to be taken."""
        torch = _torch()
        return cls(torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device), torch.full((1,), n_pages, dtype=torch.int32, device=device))

    def get_status(self) -> int:
        """The status bits set since the pool was made (``ST_PAGE_POOL``, ``ST_BOUNDS``).  Synchronises."""
        return int(self._status.item())

    def _tables(self, E, page_table, kv_len, change, what):
        self._held.check(E)
        shape = page_table.shape
        if len(shape) != 2:
            raise DynaKVError(f"expected page_table of two dimensions, got {tuple(shape)}")
        b, per = shape
        device = self._device
        return b, per, _index(E, page_table, (b, per), device, "page_table"), _index(E, kv_len, (b,), device, "kv_len"), _index(E, change, (b,), device, what)

    def extend(self, page_table, kv_len, new_len, n_tokens: int):
        """Rows for ``new_len`` [sequences] int32 new tokens behind every sequence: ``page_table`` [sequences, pages] and ``kv_len``
        [sequences] int32 are brought up to date, and (q_start [sequences + 1], positions [n_tokens], slots [n_tokens]), all int32, are
        what ``HeadRotary.store``, ``RowCache.write`` and the attention calls take; drafts of a tree are rotated by their depth in it, ``positions`` minus
        their place in the tree plus their depth.  ``n_tokens``: places in the packed batch; those that are left over get
        position 0 and slot -1.  Sequences are served in order until pages or places run out."""
        E = _rows._env_made or _rows._env()
        b, per, table, lens, add = self._tables(E, page_table, kv_len, new_len, "new_len")
        if not 0 <= n_tokens < 1 << 31:
            raise DynaKVError(f"n_tokens is {n_tokens}: expected 0 to 2^31 - 1")
        results = E.empty(2 * n_tokens + b + 1, dtype=E.i32, device=self.device)         # an allocation costs more than a view
        to = results.data_ptr()
        _call(E, self._device, E.dynakv_pages_extend, self._ref, table, per, lens, add, b, n_tokens, to + 8 * n_tokens, to, to + 4 * n_tokens, self._status_at)
        positions, slots, q_start = results.split_with_sizes((n_tokens, n_tokens, b + 1))
        return q_start, positions, slots

    def trim(self, page_table, kv_len, drop) -> None:
        """The last ``drop`` [sequences] int32 rows of every sequence given up, with the pages that then hold none (drop = kv_len
        ends a sequence).  ``drop`` must not be ``kv_len`` itself."""
        E = _rows._env_made or _rows._env()
        b, per, table, lens, less = self._tables(E, page_table, kv_len, drop, "drop")
        if b and less == lens:
            raise DynaKVError("drop is kv_len itself, which this call writes: pass a copy")
        _call(E, self._device, E.dynakv_pages_trim, self._ref, table, per, lens, less, b, self._status_at)


_workspace = {}            # bytes of scratch, by device and shapes


def _floats(E, t, shape: tuple, device: int, what: str) -> int:
    if t.dtype is not E.f32 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise DynaKVError(f"expected {what} as a contiguous float32 tensor of shape {shape} on cuda:{device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.requires_grad and E.grad():
        _no_gradient()
    return t.data_ptr()


def _matrix(E, t, shape: tuple, device: int, types, what: str) -> int:
    """A [n, vocabulary] tensor whose rows are contiguous; the stride between them is free."""
    if t.shape != shape or t.dtype not in types or t.get_device() != device or (shape[1] > 1 and t.stride(1) != 1):
        raise DynaKVError(f"expected {what} as a {' or '.join(map(str, types))} tensor of shape {tuple(shape)} on cuda:{device} with contiguous rows, "
                          f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.requires_grad and E.grad():
        _no_gradient()
    return t.data_ptr()


def verify_drafts(logits, tokens, q_start, max_tree: int, uniform, temperature, parent=None, draft_probs=None):
    """Which drafted tokens the target model accepts, and the token behind them (``dynakv_verify_drafts``): (kept, dropped, path, next).

    ``tokens`` [n] int32: the trees of all sequences as ``RowCache.attend_tree`` takes them, sequence b's from ``q_start`` [sequences + 1]
    int32 [b] on, the first its last certain token, the others drafts; ``parent`` [n] int32: a draft's parent's place in its tree
    (None: chains).  ``logits`` [n, vocabulary] (fp32 or bf16): the target's behind each token.  ``draft_probs`` [n, vocabulary] fp32: what each draft was drawn from
    (None: drafts that were not drawn but looked up).  ``uniform`` [n] fp32 in [0, 1): a draft's number decides on it, the root's draws
    the next token.  ``temperature`` [sequences] fp32, 0: always the first largest logit.
    kept [sequences]: tokens on the accepted path with the root; dropped: the others; path [sequences, max_tree]: the kept tokens' places, then
    -1 (``RowCache.keep`` takes both); next [sequences].  All int32."""
    E = _rows._env_made or _rows._env()
    if logits.dim() != 2:
        raise DynaKVError(f"expected logits of two dimensions, got {tuple(logits.shape)}")
    if not logits.is_cuda:
        raise DynaKVError(f"logits is on {logits.device}: expected a CUDA tensor (there is no CPU fallback)")
    n, vocab = logits.shape
    device, where = logits.get_device(), logits.device
    b = q_start.shape[0] - 1 if q_start.dim() == 1 else -1
    if b < 0:
        raise DynaKVError(f"expected q_start of sequences + 1 elements, got {tuple(q_start.shape)}")
    if not 1 <= max_tree <= MAX_TREE or not 1 <= vocab <= 1 << 26 or n >= 1 << 24 or b > 65535:
        raise DynaKVError(f"max_tree is {max_tree}, {n} tokens of a vocabulary of {vocab}, {b} sequences: expected 1 to {MAX_TREE}, fewer than 2^24, 1 to 2^26, at most 65535")
    at = _matrix(E, logits, (n, vocab), device, (E.f32, E.bf16), "logits")
    if parent is not None and draft_probs is not None:
        raise DynaKVError("draft_probs goes with chains (parent=None): drafts of a tree are taken as looked up")
    draft = _matrix(E, draft_probs, (n, vocab), device, (E.f32,), "draft_probs") if draft_probs is not None else None
    code = E.types[logits.dtype]
    key = (device, code, n, vocab, b, max_tree)
    size = _workspace.get(key)
    if size is None:
        with E.torch.cuda.device(device):
            size = E.dynakv_verify_drafts_workspace(code, n, vocab, b, max_tree)
        if size < 0:
            raise DynaKVError(f"dynakv_verify_drafts_workspace returned {size}")
        if len(_workspace) >= 4096:
            _workspace.clear()
        _workspace[key] = size
    words, start = _index(E, tokens, (n,), device, "tokens"), _index(E, q_start, (b + 1,), device, "q_start")
    above = _index(E, parent, (n,), device, "parent") if parent is not None else None
    chance, heat = _floats(E, uniform, (n,), device, "uniform"), _floats(E, temperature, (b,), device, "temperature")
    results, space = E.empty(b * (3 + max_tree), dtype=E.i32, device=where), E.empty(size, dtype=E.byte, device=where)      # an allocation costs more than a view
    to = results.data_ptr()
    _call(E, device, E.dynakv_verify_drafts, at, logits.stride(0), code, n, vocab, words, start, b, max_tree, chance, heat, above,
          draft, draft_probs.stride(0) if draft is not None else 0, to, to + 4 * b, to + 12 * b, to + 8 * b, space.data_ptr(), size)
    kept, dropped, following, path = results.split_with_sizes((b, b, b, b * max_tree))
    return kept, dropped, path.view(b, max_tree), following
