"""Seeded sweeps of the paged-cache operators over random small shapes that straddle the kernels' own boundaries (rows per
workgroup, pages within and across tiles, ranges and their joins), against the 64-bit oracle."""
import numpy as np
import pytest

import workloads as wl
from oracle import paged
from tests import test_gpu_paged as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(40))
def test_attention(seed):
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(1000 + seed)
    pick = lambda *a: a[int(g.integers(len(a)))]
    B, Hkv, gq, D, ps = int(g.integers(1, 5)), int(g.integers(1, 4)), int(pick(1, 1, 2, 3, 4, 8)), pick(64, 128), pick(16, 32, 64, 128, 256)
    n = int(pick(1, 2, 8, 9, 16, 17, 31, 33, 64, 65, 100, 129, 256) if gq < 3 else pick(1, 3, 5, 11, 16, 32, 43, 85))
    keys = pick(0, n, n, int(g.integers(1, 200)))
    kind = "tree" if keys == n else "random"
    most = int(pick(40, 300, 1500, 4000) if n * gq * B * Hkv < 700 else pick(40, 300, 900))
    lens = [int(x) for x in g.integers(0, most, B)]
    pages = max(1, max(-(-l // ps) for l in lens)) + int(g.integers(0, 3))
    table = P.random_table(g, B, pages, B * pages + 2)
    eight = bool(seed % 3)
    print("case", seed, B, Hkv, gq, D, n, keys, ps, lens, eight, flush=True)
    host, exps, cache = P.make_cache(g, B * pages + 2, Hkv, ps, D, eight, table, token_major=bool(seed & 1))
    Q = wl.store((g.standard_normal((B, Hkv * gq, n, D)) * pick(0.5, 1, 3)).astype(np.float32), "bf16")
    Kt = Vt = mask = None
    if keys:
        Kt, Vt = (wl.store(g.standard_normal((B, Hkv, keys, D)).astype(np.float32), "bf16") for _ in range(2))
        mask = P.tree_masks(g, B, n, keys, kind)
    put = lambda a: None if a is None else P.dev(a, "bf16")
    got = api.tree_verify_attention_paged(put(Q), cache, P.i32(lens), put(Kt), put(Vt), None if mask is None else P.U.mask_to_device(mask))
    torch.cuda.synchronize()
    P.check_attention(got, Q, host, exps, table, lens, Kt, Vt, mask)


@pytest.mark.parametrize("seed", range(30))
def test_append(seed):
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(2000 + seed)
    pick = lambda *a: a[int(g.integers(len(a)))]
    B, H, D, ps = int(g.integers(1, 6)), int(g.integers(1, 9)), pick(64, 128), pick(16, 32, 64, 128, 256)
    n = int(pick(1, 2, 15, 16, 17, 40, 100, 300))
    lens = [int(x) for x in g.integers(0, 3 * ps, B)]
    pages = max(1, max(-(-(l + n) // ps) for l in lens) - int(g.integers(0, 2)))         # now and then too few
    table = P.random_table(g, B, pages, B * pages + 2)
    rotary, inter, dtype, eight = int(pick(0, 16, D // 2, D)), bool(g.integers(2)), pick("bf16", "f32"), bool(g.integers(3))
    print("case", seed, B, H, D, ps, n, lens, rotary, inter, dtype, eight, flush=True)
    host, exps, cache = P.make_cache(g, B * pages + 2, H, ps, D, eight, table, token_major=bool(seed & 1))
    scale = np.exp(2 * g.standard_normal((B, H, 1, 1)))
    K, V = (wl.store((g.standard_normal((B, H, n, D)) * scale).astype(np.float32), dtype) for _ in range(2))
    count = None if seed % 3 else [int(x) for x in g.integers(0, n + 1, B)]
    rows = None if seed % 4 else g.permuted(np.tile(np.arange(n), (B, 1)), axis=1)
    f, f_dev = P.inv_freq(rotary)
    new = api.kv_append_paged(cache, P.dev(K, dtype), P.dev(V, dtype), P.i32(lens), count=None if count is None else P.i32(count),
                              rows=None if rows is None else P.i32(rows), inv_freq=f_dev, interleaved=inter, shift=int(seed) - 3)
    torch.cuda.synchronize()
    P.check_append(host, exps, cache, K, V, dtype, lens, [n] * B if count is None else count, rows, f, inter, int(seed) - 3, new)


@pytest.mark.parametrize("seed", range(20))
def test_norm_rope(seed):
    from paper_2406_17276_amd import api
    g = np.random.default_rng(3000 + seed)
    pick = lambda *a: a[int(g.integers(len(a)))]
    B, n, Hq, Hkv, D = int(g.integers(1, 5)), int(pick(1, 2, 7, 33, 130)), int(g.integers(1, 40)), int(g.integers(1, 12)), pick(64, 128)
    rotary, inter, dtype, norm = int(pick(0, 16, D // 2, D - 16, D)), bool(g.integers(2)), pick("bf16", "f32"), bool(g.integers(2))
    q, k = (wl.store((g.standard_normal((B, h, n, D)) * 2).astype(np.float32), dtype) for h in (Hq, Hkv))
    w = wl.store((1 + 0.3 * g.standard_normal(D)).astype(np.float32), dtype)
    f, f_dev = P.inv_freq(rotary, 500000.0)
    first = g.integers(0, 200000, B)
    got = api.qk_norm_rope(P.dev(q, dtype), P.dev(k, dtype), P.i32(first), f_dev, q_weight=P.dev(w, dtype) if norm else None, interleaved=inter)
    u = P.UBF if dtype == "bf16" else P.U32
    for x, weight, y in ((q, w if norm else None, got[0]), (k, None, got[1])):
        want = paged.norm_rope(wl.to_f64(x, dtype), first[:, None] + np.arange(n), f, None if weight is None else wl.to_f64(weight, dtype), 1e-6, inter)
        tol = u * np.abs(want) + 32 * P.U32 * P.pair_length(want, rotary, inter) * (1 + u)
        assert np.all(np.abs(P.U.from_device_f64(y) - want) <= tol)
