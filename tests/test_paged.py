"""Paged-cache operators without a GPU: the oracle against closed forms, and what the entry points refuse (nothing is launched)."""
import ctypes as C
import math

import numpy as np
import pytest

import workloads as wl
from oracle import paged
from oracle.tree_attention import tree_verify_attention
from paper_2406_17276_amd import api

F = C.c_void_p(0x1000)


# ---- oracle pins --------------------------------------------------------------------------------------------------
def test_rotation_keeps_lengths_and_relative_angles():
    g = np.random.default_rng(0)
    inv = 10000.0 ** (-np.arange(0, 32, 2) / 32)
    for inter in (False, True):
        q, k = g.standard_normal(64), g.standard_normal(64)
        a = paged.turn(q, 1000, inv, inter) @ paged.turn(k, 990, inv, inter)
        b = paged.turn(q, 10, inv, inter) @ paged.turn(k, 0, inv, inter)
        assert abs(a - b) < 1e-10
        assert abs(np.linalg.norm(paged.turn(q, 12345, inv, inter)) - np.linalg.norm(q)) < 1e-12
        np.testing.assert_array_equal(paged.turn(q, 7, inv, inter)[32:], q[32:])
    one = paged.turn(np.eye(64)[0], 1, np.array([math.pi / 2]), True)
    np.testing.assert_allclose(one[:2], [0, 1], atol=1e-15)


def test_norm_gives_unit_mean_square():
    g = np.random.default_rng(1)
    x = g.standard_normal((2, 3, 4, 64)) * 7
    y = paged.norm_rope(x, np.zeros((2, 4)), np.zeros(0), np.ones(64), 0.0)
    np.testing.assert_allclose((y * y).mean(-1), 1.0, rtol=1e-12)


def test_exponent_is_the_smallest_that_holds_the_largest():
    for top in (1e-30, 0.9, 448.0, 448.0001, 1.0, 3e38, 2.0 ** -126 * 448):
        e = paged.needed_exponent(top)
        assert top <= 448 * 2.0 ** (e - 127) and (e == 1 or top > 448 * 2.0 ** (e - 128))
    assert paged.needed_exponent(0.0) == 1


def test_paged_attention_equals_the_contiguous_one():
    g = np.random.default_rng(2)
    B, Hq, H, n, D, ps = 2, 4, 2, 5, 64, 16
    table = np.array([[3, 0, 5], [1, 4, 2]])
    pools = [g.standard_normal((6, H, ps, D)) for _ in range(2)]
    lens = np.array([40, 7])
    Q, Kt, Vt = g.standard_normal((B, Hq, n, D)), g.standard_normal((B, H, n, D)), g.standard_normal((B, H, n, D))
    mask = np.tril(np.ones((n, n), dtype=np.uint64)) @ (np.uint64(1) << np.arange(n, dtype=np.uint64))
    mask = np.broadcast_to(mask[None, :, None], (B, n, 1)).copy()
    Kp = np.stack([np.concatenate([pools[0][p] for p in t], 1) for t in table])
    Vp = np.stack([np.concatenate([pools[1][p] for p in t], 1) for t in table])
    want = tree_verify_attention(Q, Kp, Vp, Kt, Vt, lens, mask)
    got, A, _ = paged.attention(Q, pools, (None, None), table, lens, Kt, Vt, mask)
    np.testing.assert_allclose(got, want, atol=1e-12)
    assert np.all(A >= np.abs(got) - 1e-12)


def test_append_then_gather_returns_the_rows():
    g = np.random.default_rng(3)
    pool = g.standard_normal((5, 2, 16, 64))
    K = g.standard_normal((1, 2, 20, 64))
    table = np.array([[4, -1, 2], [0, 3, 1]])
    want, _, new = paged.append(pool, None, K, table[1:], [9], [20])
    assert list(new) == [29]
    pool2 = np.where(np.isnan(want), pool, want)
    rows, there = paged.gather(pool2, None, table[1], 29)
    assert there.all()
    np.testing.assert_array_equal(rows[:, 9:], K[0])
    assert paged.stored_rows(9, 20, table[0], 16, 5) == (9, 7)          # its second page is none
    assert paged.stored_rows(16, 20, table[0], 16, 5) == (16, 0)
    assert paged.stored_rows(40, 20, table[1], 16, 5) == (40, 8)        # capacity


def test_eight_bit_rows_follow_a_larger_exponent():
    pool = np.zeros((1, 1, 16, 64), dtype=np.uint8)
    pool[0, 0, 0] = wl.f32_to_e4m3_bits(np.full(64, 300.0))
    want, exps, _ = paged.append(pool, np.array([[127]], dtype=np.uint8), np.full((1, 1, 1, 64), 2000.0), [[0]], [1], [1],
                                 decode=lambda q: wl.e4m3_bits_to_f32(q).astype(np.float64))
    assert exps[0, 0] == 130                                               # 2000 <= 448 * 8
    decoded = wl.e4m3_bits_to_f32(pool[0, 0, 0])[0]                        # 300 is stored as 288
    assert want[0, 0, 0, 0] == decoded / 8 and want[0, 0, 1, 0] == 250.0 and np.isnan(want[0, 0, 2, 0])


# ---- refusals -----------------------------------------------------------------------------------------------------
s3 = C.c_int64 * 3


def _qk(**kw):
    d = dict(batch=1, q_heads=4, kv_heads=2, head_dim=64, n=3, dtype=1, rotary_dim=64, interleaved=0, shift=0, eps=1e-6)
    for k in ("q_strides", "k_strides", "qo_strides", "ko_strides"):
        d[k] = s3(768, 192, 64)
    d.update(kw)
    return api.QkParams(**d)


@pytest.mark.parametrize("bad, status", [
    (dict(batch=0), -1), (dict(n=0), -1), (dict(q_heads=-1), -1), (dict(q_heads=0, kv_heads=0), -1), (dict(dtype=2), -1),
    (dict(interleaved=2), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1), (dict(rotary_dim=-16), -1),
    (dict(rotary_dim=80), -1), (dict(rotary_dim=24), -2), (dict(head_dim=96), -2), (dict(batch=1 << 20, n=1 << 12), -2),
    (dict(q_heads=60000, kv_heads=6000), -2), (dict(q_strides=s3(768, 192, 60)), -1), (dict(ko_strides=s3(768, -192, 64)), -1)])
def test_norm_rope_refuses(bad, status):
    assert api.lib().ot_qk_norm_rope(C.byref(_qk(**bad)), *([F] * 9), None) == status


@pytest.mark.parametrize("stride", [(0, 192, 64), (768, 0, 64), (768, 192, 0)])
def test_broadcast_rows_are_not_written(stride):
    """Two rows of an output at one address would be a race; on an axis of one row a stride says nothing."""
    L, far = api.lib(), C.c_void_p(0x900000)
    for name in ("qo_strides", "ko_strides"):
        assert L.ot_qk_norm_rope(C.byref(_qk(batch=2, **{name: s3(*stride)})), *([F] * 9), None) == -1, name
    assert L.ot_tree_verify_attention_paged(C.byref(_pp(batch=2, o_strides=s3(*stride))), C.byref(_cache()), *([F] * 7), 1 << 30, None) == -1
    assert L.ot_paged_attn_workspace_bytes(C.byref(_pp(batch=1, n=1, o_strides=s3(0, 64, 0))), C.byref(_cache())) > 0
    for name in ("k_strides", "v_strides"):
        for pool in ((0, 1024, 64), (2048, 0, 64)):
            c = _cache(**{name: s3(*pool)})
            assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(c), F, F, F, F, F, F, far, None) == -1, (name, pool)
            assert L.ot_paged_attn_workspace_bytes(C.byref(_pp()), C.byref(c)) > 0                       # is read


def test_norm_rope_refuses_pointers():
    L, p = api.lib(), _qk()
    for i in (0, 1, 4, 5, 7, 8):                                           # Q, K, inv_freq, first, Q_out, K_out
        args = [F] * 9
        args[i] = None
        assert L.ot_qk_norm_rope(C.byref(p), *args, None) == -1, i
    for i, off in ((0, 8), (1, 8), (2, 8), (3, 8), (4, 4), (5, 2), (6, 2), (7, 8), (8, 8)):
        args = [F] * 9
        args[i] = C.c_void_p(0x1000 + off)
        assert L.ot_qk_norm_rope(C.byref(p), *args, None) == -1, i
    assert L.ot_qk_norm_rope(None, *([F] * 9), None) == -1


def _cache(**kw):
    d = dict(num_pages=8, page_size=16, kv_heads=2, head_dim=64, dtype=2, max_pages=4, k_strides=s3(2048, 1024, 64),
             v_strides=s3(2048, 1024, 64), k_pages=0x1000, v_pages=0x1000, k_exp=0x1000, v_exp=0x1000, page_table=0x1000)
    d.update(kw)
    return api.PagedCacheParams(**d)


def _ap(**kw):
    d = dict(batch=1, n=3, dtype=1, rotary_dim=64, interleaved=0, shift=0, count_shift=0, k_strides=s3(384, 192, 64),
             v_strides=s3(384, 192, 64))
    d.update(kw)
    return api.AppendParams(**d)


def _pp(**kw):
    d = dict(batch=1, q_heads=4, n=3, tree_keys=3, softmax_scale=0.0, q_strides=s3(768, 192, 64), kt_strides=s3(384, 192, 64),
             vt_strides=s3(384, 192, 64), o_strides=s3(768, 192, 64))
    d.update(kw)
    return api.PagedAttnParams(**d)


BAD_CACHES = [(dict(num_pages=0), -1), (dict(page_size=0), -1), (dict(page_size=24), -2), (dict(page_size=512), -2), (dict(page_size=8), -2),
              (dict(kv_heads=0), -1), (dict(head_dim=96), -2), (dict(dtype=0), -1), (dict(max_pages=0), -1), (dict(max_pages=1 << 27), -2),
              (dict(k_strides=s3(2048, 1024, 72)), -1), (dict(v_strides=s3(2048, 1024, 48)), -1), (dict(k_pages=0x1008), -1),
              (dict(v_pages=None), -1), (dict(page_table=0x1002), -1), (dict(page_table=None), -1), (dict(k_exp=None), -1), (dict(v_exp=None), -1)]


@pytest.mark.parametrize("bad, status", BAD_CACHES)
def test_bad_caches_are_refused(bad, status):
    L, c = api.lib(), _cache(**bad)
    far = C.c_void_p(0x9000)
    assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(c), F, F, F, F, F, F, far, None) == status
    assert L.ot_tree_verify_attention_paged(C.byref(_pp()), C.byref(c), *([F] * 7), 1 << 30, None) == status


@pytest.mark.parametrize("bad, status", [
    (dict(batch=0), -1), (dict(n=0), -1), (dict(n=(1 << 24) + 1), -2), (dict(dtype=2), -1), (dict(rotary_dim=80), -1), (dict(rotary_dim=8), -2),
    (dict(interleaved=-1), -1), (dict(batch=1 << 16, n=1 << 15), -2), (dict(k_strides=s3(384, 192, 60)), -1), (dict(v_strides=s3(-8, 192, 64)), -1)])
def test_append_refuses(bad, status):
    far = C.c_void_p(0x900000)
    assert api.lib().ot_kv_append_paged(C.byref(_ap(**bad)), C.byref(_cache()), F, F, F, F, F, F, far, None) == status


def test_append_refuses_pointers():
    L, far = api.lib(), C.c_void_p(0x9000)
    ok = [F, F, F, F, F, F, far]                                           # K, V, inv_freq, cache_len, count, rows, new_len
    for i in (0, 1, 2, 3, 6):
        args = list(ok)
        args[i] = None
        assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(_cache()), *args, None) == -1, i
    for i, off in ((0, 8), (1, 8), (2, 4), (3, 1), (4, 1), (5, 1), (6, 1)):
        args = list(ok)
        args[i] = C.c_void_p((args[i].value or 0) + off)
        assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(_cache()), *args, None) == -1, i
    for i in (3, 4, 5):                                                    # new_len on one of the arrays that are still read
        args = list(ok)
        args[6] = args[i]
        assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(_cache()), *args, None) == -1, i
    assert L.ot_kv_append_paged(None, C.byref(_cache()), *ok, None) == -1
    assert L.ot_kv_append_paged(C.byref(_ap()), None, *ok, None) == -1


@pytest.mark.parametrize("bad, status", [
    (dict(batch=0), -1), (dict(n=0), -1), (dict(n=257), -2), (dict(q_heads=5), -1), (dict(q_heads=0), -1), (dict(tree_keys=-1), -1),
    (dict(tree_keys=8193), -2), (dict(softmax_scale=-1.0), -1), (dict(softmax_scale=math.nan), -1), (dict(softmax_scale=math.inf), -1),
    (dict(batch=20000), -2), (dict(q_strides=s3(768, 192, 60)), -1), (dict(o_strides=s3(768, 4, 64)), -1), (dict(kt_strides=s3(384, 192, 4)), -1)])
def test_paged_attention_refuses(bad, status):
    L = api.lib()
    assert L.ot_tree_verify_attention_paged(C.byref(_pp(**bad)), C.byref(_cache()), *([F] * 7), 1 << 30, None) == status
    assert L.ot_paged_attn_workspace_bytes(C.byref(_pp(**bad)), C.byref(_cache())) == 0


def test_paged_attention_refuses_pointers_and_small_workspaces():
    L, p, c = api.lib(), _pp(), _cache()
    need = L.ot_paged_attn_workspace_bytes(C.byref(p), C.byref(c))
    assert need >= 65536
    assert L.ot_tree_verify_attention_paged(C.byref(p), C.byref(c), *([F] * 7), need - 1, None) == -3
    for i in range(7):                                                     # Q, K_tree, V_tree, prefix_len, mask, O, workspace
        args = [F] * 7
        args[i] = None
        assert L.ot_tree_verify_attention_paged(C.byref(p), C.byref(c), *args, need, None) == -1, i
        args[i] = C.c_void_p(0x1000 + (2 if i == 3 else 4 if i == 4 else 8))
        assert L.ot_tree_verify_attention_paged(C.byref(p), C.byref(c), *args, need, None) == -1, i
    assert L.ot_paged_attn_workspace_prepare(None, need, None) == -1
    assert L.ot_paged_attn_workspace_prepare(F, 65535, None) == -3
    assert L.ot_paged_attn_workspace_prepare(C.c_void_p(0x1008), need, None) == -1


def test_binding_refuses_tensors_on_the_host():
    import torch
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = api.alloc_paged_cache(4, 2, 16, 64, 1, 2, device="cpu")
    with pytest.raises(ValueError):
        api.qk_norm_rope(bf(1, 4, 3, 64), bf(1, 2, 3, 64), i(1))
    with pytest.raises(ValueError):
        api.qk_norm_rope(None, None, i(1))
    with pytest.raises(ValueError):
        api.kv_append_paged(cache, bf(1, 2, 3, 64), bf(1, 2, 3, 64), i(1))
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(bf(1, 4, 1, 64), cache, i(1), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(TypeError):
        api.kv_append_paged(cache, 3, bf(1, 2, 3, 64), i(1))
