"""CPU checks of the calls on plain rows: what the C entries and the binding refuse, before anything touches a device."""
import ctypes as C

import pytest
import torch

import paper_2511_07427_b200 as P
from paper_2511_07427_b200 import rows as R

BUF = C.create_string_buffer(4096 + 64)
ADDR = (C.addressof(BUF) + 63) // 64 * 64        # an aligned host address: never read, every call below is refused or empty


def _cache(**kw):
    base = dict(k=ADDR, v=ADDR, k_exp=None, v_exp=None, n_pages=4, n_kv_heads=2, head_dim=128, kv_dtype=P.BF16)
    base.update(kw)
    return R._RowCache(**base)


def _rows(**kw):
    base = dict(data=ADDR, token_stride=256, head_stride=128, dtype=P.BF16)
    base.update(kw)
    return R._HeadRows(**base)


def _rotary(**kw):
    base = dict(n_heads=4, n_kv_heads=2, head_dim=128, rotary_dim=128, interleaved=0, eps=1e-6, q_weight=None, k_weight=None, inv_freq=ADDR)
    base.update(kw)
    return R._Rotary(**base)


def _norm_rope(ro=None, q=None, k=None, positions=ADDR, n=1, q_out=ADDR, q_dtype=P.BF16, k_out=ADDR, k_dtype=P.BF16):
    return R._library().dynakv_norm_rope(C.byref(ro or _rotary()), C.byref(q or _rows()), C.byref(k or _rows()), positions, n, q_out, q_dtype, k_out, k_dtype, None)


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_kv_heads=0), dict(head_dim=96), dict(rotary_dim=136), dict(rotary_dim=24), dict(rotary_dim=-16),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(inv_freq=None)])
def test_norm_rope_refuses_a_bad_embedding(bad):
    assert _norm_rope(ro=_rotary(**bad)) == -1


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=1 << 31), dict(positions=None), dict(q_out=None), dict(k_out=None), dict(q_out=ADDR + 8), dict(k_out=ADDR + 4),
                                 dict(q_dtype=P.FP8), dict(k_dtype=7), dict(q=_rows(data=None)), dict(k=_rows(dtype=P.F32)), dict(q=_rows(dtype=P.FP8), k=_rows(dtype=P.FP8)),
                                 dict(q=_rows(data=ADDR + 1))])
def test_norm_rope_refuses_bad_arrays(bad):
    assert _norm_rope(**bad) == -1


def test_empty_calls_are_fine_without_a_device():
    L = R._library()
    assert _norm_rope(n=0, q_out=None, k_out=None, positions=None) == 0
    none = _rows(data=None)
    assert L.dynakv_rows_write(C.byref(_cache()), C.byref(none), C.byref(none), None, 0, None, None) == 0
    assert L.dynakv_rows_read(C.byref(_cache()), None, 0, None, 0, 0, 5, None, None, None, None) == 0
    assert L.dynakv_rows_read(C.byref(_cache()), ADDR, 2, ADDR, 3, 0, 0, None, None, None, None) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k=ADDR + 8), dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=80), dict(kv_dtype=3),
                                 dict(kv_dtype=P.FP8), dict(kv_dtype=P.FP8, k_exp=ADDR, v_exp=ADDR + 4), dict(n_pages=1 << 31), dict(n_pages=1 << 26, n_kv_heads=1)])
def test_every_cache_call_refuses_a_bad_cache(bad):
    L, c, x = R._library(), _cache(**bad), _rows()
    assert L.dynakv_rows_write(C.byref(c), C.byref(x), C.byref(x), ADDR, 1, None, None) == -1
    assert L.dynakv_rows_read(C.byref(c), ADDR, 2, ADDR, 1, 0, 5, ADDR, ADDR, None, None) == -1
    assert L.dynakv_norm_rope_store(C.byref(_rotary(head_dim=c.head_dim, n_kv_heads=c.n_kv_heads)), C.byref(x), C.byref(x), C.byref(x), ADDR, 1, ADDR, P.BF16,
                                    C.byref(c), ADDR, None, None) == -1


def test_store_refuses_a_cache_of_other_heads():
    L, x = R._library(), _rows()
    for c in (_cache(n_kv_heads=3), _cache(head_dim=64)):
        assert L.dynakv_norm_rope_store(C.byref(_rotary()), C.byref(x), C.byref(x), C.byref(x), ADDR, 1, ADDR, P.BF16, C.byref(c), ADDR, None, None) == -1
    assert L.dynakv_norm_rope_store(C.byref(_rotary()), C.byref(x), C.byref(x), C.byref(x), ADDR, 1, ADDR, P.BF16, C.byref(_cache()), None, None, None) == -1
    assert L.dynakv_norm_rope_store(C.byref(_rotary()), C.byref(x), C.byref(x), None, ADDR, 1, ADDR, P.BF16, C.byref(_cache()), ADDR, None, None) == -1


def test_write_and_read_refuse_bad_arrays():
    L, c, x = R._library(), _cache(), _rows()
    for k, v, slots, n in ((_rows(dtype=P.FP8), x, ADDR, 1), (x, _rows(dtype=P.F32), ADDR, 1), (x, x, None, 1), (x, x, ADDR, -1), (x, _rows(data=None), ADDR, 1)):
        assert L.dynakv_rows_write(C.byref(c), C.byref(k), C.byref(v), slots, n, None, None) == -1
    ok = dict(table=ADDR, per=2, lens=ADDR, b=1, first=0, n=5, K=ADDR, V=ADDR)
    for bad in (dict(table=None), dict(per=-1), dict(lens=None), dict(b=-1), dict(b=65536), dict(first=-1), dict(n=-1), dict(n=1 << 31), dict(K=None), dict(V=ADDR + 8)):
        a = {**ok, **bad}
        assert L.dynakv_rows_read(C.byref(c), a["table"], a["per"], a["lens"], a["b"], a["first"], a["n"], a["K"], a["V"], None, None) == -1, bad


def test_binding_refuses_cpu_tensors():
    z = torch.zeros(4, 2, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(P.DynaKVError, match="CUDA"):
        P.RowCache(z, z.clone())
    with pytest.raises(P.DynaKVError, match="CUDA"):
        P.HeadRotary(4, 2, 128, torch.ones(64))
    with pytest.raises(P.DynaKVError, match="rotary_dim"):
        P.HeadRotary(4, 2, 64, torch.ones(40))
    with pytest.raises(P.DynaKVError, match="eps"):
        P.HeadRotary(4, 2, 128, torch.ones(64), eps=-1.0)
    with pytest.raises(P.DynaKVError, match="heads|head"):
        P.HeadRotary(0, 2, 128, torch.ones(64))


def _attend(cache=None, q=ADDR, n_heads=4, n_tokens=3, q_start=ADDR, n_seqs=1, max_tree=3, table=ADDR, per=2, kv_len=ADDR, mask=None, words=0, scale=0.1,
            out=ADDR, lse=None, space=ADDR, size=1 << 40):
    return R._library().dynakv_attend_tree(C.byref(cache or _cache()), q, n_heads, n_tokens, q_start, n_seqs, max_tree, table, per, kv_len, mask, words, scale,
                                           out, lse, space, size, None, None)


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_heads=3), dict(n_heads=18), dict(max_tree=0), dict(max_tree=257), dict(n_tokens=-1), dict(n_tokens=1 << 31),
                                 dict(n_seqs=-1), dict(per=-1), dict(per=1 << 26), dict(scale=float("nan")), dict(scale=float("inf")), dict(mask=ADDR, words=0),
                                 dict(mask=ADDR, words=5), dict(q=None), dict(q_start=None), dict(table=None), dict(kv_len=None), dict(out=None), dict(space=None),
                                 dict(q=ADDR + 8), dict(out=ADDR + 2), dict(space=ADDR + 4), dict(cache=_cache(head_dim=32)), dict(cache=_cache(kv_dtype=P.FP8))])
def test_attend_tree_refuses_bad_arguments(bad):
    assert _attend(**bad) == -1


def test_attend_tree_without_tokens_or_sequences_needs_nothing():
    assert _attend(n_tokens=0, q=None, out=None, space=None) == 0
    assert _attend(n_seqs=0, q=None, out=None, space=None) == 0
    for bad in (dict(n_heads=5), dict(max_tree=0), dict(max_tree=1000)):
        a = dict(n_heads=4, max_tree=3)
        a.update(bad)
        assert R._library().dynakv_attend_tree_workspace(C.byref(_cache()), a["n_heads"], a["max_tree"]) == -1
