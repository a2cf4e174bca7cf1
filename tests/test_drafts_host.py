"""CPU checks of the calls around drafted tokens: what the C entries and the binding refuse, before anything touches a device."""
import ctypes as C

import pytest
import torch

import paper_2511_07427_b200 as P
from paper_2511_07427_b200 import drafts as D
from paper_2511_07427_b200 import rows as R

BUF = C.create_string_buffer(4096 + 64)
ADDR = (C.addressof(BUF) + 63) // 64 * 64        # an aligned host address: never read, every call below is refused or empty


def _cache(**kw):
    base = dict(k=ADDR, v=ADDR, k_exp=None, v_exp=None, n_pages=4, n_kv_heads=2, head_dim=128, kv_dtype=P.BF16)
    base.update(kw)
    return R._RowCache(**base)


def _chunk(cache=None, q=ADDR, n_heads=4, n_tokens=3, q_start=ADDR, n_seqs=1, max_chunk=3, table=ADDR, per=2, kv_len=ADDR, scale=0.1, softcap=0.0, window=0,
           no_scores=False, out=ADDR, lse=None, space=ADDR, size=1 << 40):
    s = R._Scores(scale, softcap, window, None, None, None)
    return R._library().dynakv_attend_chunk(C.byref(cache or _cache()), q, n_heads, n_tokens, q_start, n_seqs, max_chunk, table, per, kv_len,
                                            None if no_scores else C.byref(s), out, lse, space, size, None, None)


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=3), dict(n_heads=18), dict(max_chunk=0), dict(max_chunk=(1 << 24) + 1), dict(n_tokens=-1), dict(n_tokens=1 << 31),
                                 dict(n_seqs=-1), dict(per=-1), dict(per=1 << 26), dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0),
                                 dict(softcap=float("inf")), dict(softcap=float("nan")), dict(softcap=1e-40), dict(softcap=1e38), dict(softcap=1e-10, scale=1e30), dict(window=-1), dict(no_scores=True), dict(q=None), dict(q_start=None),
                                 dict(table=None), dict(kv_len=None), dict(out=None), dict(space=None), dict(q=ADDR + 8), dict(out=ADDR + 2), dict(space=ADDR + 4),
                                 dict(cache=_cache(head_dim=32)), dict(cache=_cache(kv_dtype=P.FP8)), dict(cache=_cache(k=None))])
def test_attend_chunk_refuses_bad_arguments(bad):
    assert _chunk(**bad) == -1


def test_attend_chunk_without_tokens_or_sequences_needs_nothing():
    assert _chunk(n_tokens=0, q=None, out=None, space=None) == 0
    assert _chunk(n_seqs=0, q=None, out=None, space=None) == 0
    for bad in (dict(n_heads=5), dict(max_chunk=0), dict(n_tokens=-1), dict(n_seqs=-1), dict(per=-1)):
        a = dict(n_heads=4, n_tokens=3, n_seqs=1, max_chunk=3, per=2)
        a.update(bad)
        assert R._library().dynakv_attend_chunk_workspace(C.byref(_cache()), a["n_heads"], a["n_tokens"], a["n_seqs"], a["max_chunk"], a["per"]) == -1


def _pool(**kw):
    base = dict(free_pages=ADDR, count=ADDR, n_pages=8)
    base.update(kw)
    return D._Pool(**base)


def _extend(pool=None, table=ADDR, per=2, lens=ADDR, add=ADDR, n_seqs=1, n_tokens=4, q_start=ADDR, positions=ADDR, slots=ADDR):
    return R._library().dynakv_pages_extend(C.byref(pool or _pool()), table, per, lens, add, n_seqs, n_tokens, q_start, positions, slots, None, None)


@pytest.mark.parametrize("bad", [dict(pool=_pool(free_pages=None)), dict(pool=_pool(count=None)), dict(pool=_pool(n_pages=0)), dict(pool=_pool(n_pages=1 << 26)), dict(table=None),
                                 dict(per=-1), dict(per=1 << 26), dict(lens=None), dict(add=None), dict(n_seqs=-1), dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(q_start=None),
                                 dict(positions=None), dict(slots=None)])
def test_pages_extend_refuses_bad_arguments(bad):
    assert _extend(**bad) == -1


def test_pages_trim_refuses_bad_arguments_and_takes_none():
    L = R._library()
    for pool, table, per, lens, drop, n in ((_pool(n_pages=0), ADDR, 2, ADDR, ADDR, 1), (_pool(), None, 2, ADDR, ADDR, 1), (_pool(), ADDR, 2, None, ADDR, 1),
                                            (_pool(), ADDR, 2, ADDR, None, 1), (_pool(), ADDR, 2, ADDR, ADDR, -1), (_pool(), ADDR, -1, ADDR, ADDR, 1)):
        assert L.dynakv_pages_trim(C.byref(pool), table, per, lens, drop, n, None, None) == -1
    assert L.dynakv_pages_trim(C.byref(_pool()), None, 0, None, None, 0, None, None) == 0
    assert L.dynakv_pages_trim(None, ADDR, 2, ADDR, ADDR, 1, None, None) == -1


def _verify(**kw):
    a = dict(logits=ADDR, stride=100, dtype=P.F32, n=3, vocab=100, tokens=ADDR, q_start=ADDR, n_seqs=1, most=3, uniform=ADDR, heat=ADDR, parent=None, draft=None, draft_stride=0,
             kept=ADDR, dropped=ADDR, path=ADDR, following=ADDR, space=ADDR, size=1 << 40)
    a.update(kw)
    return R._library().dynakv_verify_drafts(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(dtype=P.FP8), dict(dtype=7), dict(n=-1), dict(n=1 << 24), dict(vocab=0), dict(vocab=(1 << 26) + 1), dict(n_seqs=-1), dict(n_seqs=65536),
                                 dict(most=0), dict(most=257), dict(parent=ADDR, draft=ADDR), dict(q_start=None), dict(heat=None), dict(kept=None), dict(dropped=None),
                                 dict(path=None), dict(following=None), dict(space=None), dict(space=ADDR + 8), dict(logits=None), dict(tokens=None), dict(uniform=None),
                                 dict(logits=ADDR + 2), dict(draft=ADDR + 2), dict(stride=-1), dict(draft=ADDR, draft_stride=-1)])
def test_verify_drafts_refuses_bad_arguments(bad):
    assert _verify(**bad) == -1


def test_verify_drafts_without_sequences_needs_nothing():
    assert _verify(n_seqs=0, q_start=None, heat=None, kept=None, space=None) == 0
    for bad in ((P.FP8, 3, 100, 1, 3), (P.F32, -1, 100, 1, 3), (P.F32, 3, 0, 1, 3), (P.F32, 3, 100, 1, 0)):
        assert R._library().dynakv_verify_drafts_workspace(*bad) == -1


def test_rows_keep_refuses_bad_arguments():
    L = R._library()
    ok = dict(cache=_cache(), table=ADDR, per=2, lens=ADDR, q_start=ADDR, n=1, path=ADDR, width=2, kept=ADDR)
    for bad in (dict(cache=_cache(head_dim=96)), dict(table=None), dict(per=-1), dict(per=1 << 26), dict(lens=None), dict(q_start=None), dict(n=-1), dict(path=None), dict(width=-1),
                dict(kept=None), dict(cache=_cache(n_kv_heads=65536, n_pages=1))):
        a = {**ok, **bad}
        assert L.dynakv_rows_keep(C.byref(a["cache"]), a["table"], a["per"], a["lens"], a["q_start"], a["n"], a["path"], a["width"], a["kept"], None, None) == -1, bad
    assert L.dynakv_rows_keep(C.byref(_cache()), None, 0, None, None, 0, None, 2, None, None, None) == 0
    assert L.dynakv_rows_keep(C.byref(_cache()), ADDR, 2, ADDR, ADDR, 3, None, 0, None, None, None) == 0


def test_binding_refuses_cpu_tensors():
    with pytest.raises(P.DynaKVError, match="CUDA"):
        P.PagePool(torch.zeros(4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(P.DynaKVError, match="CUDA"):
        P.verify_drafts(torch.zeros(2, 5), torch.zeros(2, dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), 2, torch.zeros(2), torch.ones(1))
    with pytest.raises(P.DynaKVError, match="dimensions"):
        P.verify_drafts(torch.zeros(5), torch.zeros(2, dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), 2, torch.zeros(2), torch.ones(1))
