"""Operators around a paged cache on the GPU against the 64-bit oracle.

Tolerances count roundings.  Half a step: u = 2^-8 (bf16), 2^-24 (fp32), 2^-4 (E4M3), relative to the value.
  norm_rope   one rounding of the result, and fp32 errors of the norm (a sum of 128 squares in a tree of depth < 24: 24 u32), of
              cosine, sine, three products and a sum: below 32 u32 of the pair's length
  append      one rounding (E4M3 below 2^-6 of the page's factor: half a step of 2^-9), the same fp32 errors before it
  attention   probabilities and the output are rounded once each to bf16 (2 * 2^-8 of sum w |v|); a score of D products is off by
              (D + 4) u32 of sum |q k| at most, which moves a weight and the sum of weights by that each; exponentials,
              sums and merges in fp32: 2^-14 covers a hundred of their steps
"""
import numpy as np
import pytest

import workloads as wl
from oracle import paged
from tests import _util as U

pytestmark = pytest.mark.gpu
U32, UBF, U8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4


def decode(q):
    return wl.e4m3_bits_to_f32(np.asarray(q)).astype(np.float64)


def dev(a, dtype):
    import torch
    if dtype == "u8":
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return U.to_device(a, dtype)


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def inv_freq(rotary, base=10000.0):
    import torch
    f = base ** (-np.arange(0, rotary, 2) / rotary)
    return f, (torch.from_numpy(f).cuda() if rotary else None)


# ---------------------------------------------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------------------------------------------
def pair_length(y, rotary, interleaved):
    """Length of the pair that each column belongs to."""
    out, half = np.abs(y), rotary // 2
    if interleaved:
        l = np.hypot(y[..., 0:rotary:2], y[..., 1:rotary:2])
        out[..., :rotary] = np.repeat(l, 2, -1)
    else:
        l = np.hypot(y[..., :half], y[..., half:rotary])
        out[..., :rotary] = np.concatenate([l, l], -1)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B, n, Hq, Hkv, D, rotary, interleaved, norm, tree", [
    (1, 1, 32, 8, 128, 128, False, True, False), (3, 7, 5, 1, 64, 64, True, True, True), (2, 50, 8, 8, 128, 64, False, True, True),
    (2, 33, 3, 3, 128, 96, False, False, False), (1, 5, 7, 2, 64, 16, True, True, False), (2, 3, 4, 2, 128, 0, False, True, False),
    (1, 700, 6, 2, 64, 48, False, True, False), (1, 2, 71, 9, 128, 128, True, False, False), (5, 600, 2, 1, 128, 128, False, True, False)])
def test_norm_rope(dtype, B, n, Hq, Hkv, D, rotary, interleaved, norm, tree):
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(n + Hq)
    store = lambda x: wl.store(x.astype(np.float32), dtype)
    q, k = store(g.standard_normal((B, Hq, n, D)) * 3), store(g.standard_normal((B, Hkv, n, D)) * 3)
    qw, kw = store(1 + 0.3 * g.standard_normal(D)), store(1 + 0.3 * g.standard_normal(D))
    f, f_dev = inv_freq(rotary)
    first = g.integers(0, 1 << 20, B)
    offset = np.sort(g.integers(1, 12, (B, n)), 1) if tree else None
    shift = -1 if tree else 0
    pos = first[:, None] + (offset if tree else np.arange(n)) + shift
    got = api.qk_norm_rope(dev(q, dtype), dev(k, dtype), i32(first), f_dev, offset=None if offset is None else i32(offset), shift=shift,
                           q_weight=dev(qw, dtype) if norm else None, k_weight=dev(kw, dtype) if norm else None, interleaved=interleaved)
    torch.cuda.synchronize()
    u = UBF if dtype == "bf16" else U32
    for x, w, y in ((q, qw, got[0]), (k, kw, got[1])):
        want = paged.norm_rope(wl.to_f64(x, dtype), pos, f, wl.to_f64(w, dtype) if norm else None, 1e-6, interleaved)
        tol = u * np.abs(want) + 32 * U32 * pair_length(want, rotary, interleaved) * (1 + u)
        assert np.all(np.abs(U.from_device_f64(y) - want) <= tol)


def test_norm_rope_in_place_strided_one_sided():
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(0)
    B, n, H, D = 2, 9, 6, 128
    f, f_dev = inv_freq(D)
    fused = torch.randn(B, n, 3 * H, D, device="cuda").to(torch.bfloat16)          # q, k, v of a fused projection, token major
    q, k = fused[:, :, :H].transpose(1, 2), fused[:, :, H:2 * H].transpose(1, 2)
    first = i32([3, 100000])
    want_q, want_k = api.qk_norm_rope(q.contiguous(), k.contiguous(), first, f_dev)
    only_q, none = api.qk_norm_rope(q, None, first, f_dev)
    none2, only_k = api.qk_norm_rope(None, k, first, f_dev)
    assert none is None and none2 is None
    v = fused[:, :, 2 * H:].clone()
    q2, k2 = api.qk_norm_rope(q, k, first, f_dev, q_out=q, k_out=k)
    torch.cuda.synchronize()
    for x in (only_q, q2, q):
        assert torch.equal(x, want_q)
    for x in (only_k, k2, k):
        assert torch.equal(x, want_k)
    assert torch.equal(fused[:, :, 2 * H:], v)
    one = q[:, :1].expand(B, H, n, D)                                              # a broadcast input
    a, _ = api.qk_norm_rope(one, None, first, f_dev, q_out=torch.empty(B, H, n, D, dtype=torch.bfloat16, device="cuda"))
    b, _ = api.qk_norm_rope(one.contiguous(), None, first, f_dev)
    assert torch.equal(a, b)


def test_norm_rope_edges():
    """A zero row stays zero, an infinity stays in its own row, positions may be negative and far."""
    import torch
    from paper_2406_17276_amd import api
    x = torch.randn(1, 2, 3, 64, device="cuda")
    x[0, 0, 1] = 0
    x[0, 1, 2, 5] = float("inf")
    f, f_dev = inv_freq(64)
    w = torch.ones(64, device="cuda")
    y, _ = api.qk_norm_rope(x, None, i32([2147483640]), f_dev, offset=i32([[0, 7, 7]]), shift=2147483647, q_weight=w)
    assert not y[0, 0, 1].any() and torch.isfinite(y[0, 0]).all() and torch.isfinite(y[0, 1, :2]).all()
    want = paged.norm_rope(U.from_device_f64(x)[:, :1], np.array([[4294967287, 4294967294, 4294967294]]), f, np.ones(64))
    np.testing.assert_allclose(U.from_device_f64(y)[:, :1], want, atol=32 * U32 * 8)          # |pair| < 8 after the norm
    z, _ = api.qk_norm_rope(x[:, :1], None, i32([-5]), f_dev, shift=-3)
    want = paged.norm_rope(U.from_device_f64(x)[:, :1], np.array([[-8, -7, -6]]), f)
    np.testing.assert_allclose(U.from_device_f64(z), want, atol=32 * U32 * 8)


# ---------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------
def make_cache(g, P, H, ps, D, eight, table, token_major=False):
    """Random pages; (host pools k and v as stored, host exponents, api.PagedCache)."""
    from paper_2406_17276_amd import api
    shape = (P, H, ps, D)
    if eight:
        host = [wl.f32_to_e4m3_bits((g.standard_normal(shape) * 90).astype(np.float32)) for _ in range(2)]
        exps = [g.integers(117, 123, (P, H)).astype(np.uint8) for _ in range(2)]
    else:
        host = [wl.store(g.standard_normal(shape).astype(np.float32), "bf16") for _ in range(2)]
        exps = [None, None]
    put = lambda a: dev(a, "u8" if eight else "bf16")
    if token_major:                                       # [page][row][head][D] in memory
        k, v = (put(a.transpose(0, 2, 1, 3).copy()).transpose(1, 2) for a in host)
    else:
        k, v = (put(a) for a in host)
    return host, exps, api.PagedCache(k, v, i32(table), *[None if e is None else dev(e, "u8") for e in exps])


def random_table(g, B, most, P):
    return g.permutation(P)[:B * most].reshape(B, most)


def check_append(host, exps, cache, K, V, dtype, lens, count, rows, f, interleaved, shift, new):
    eight = exps[0] is not None
    for m, (x, pool, e, got, got_e) in enumerate(((K, host[0], exps[0], cache.k, cache.k_exp), (V, host[1], exps[1], cache.v, cache.v_exp))):
        x64 = wl.to_f64(x, dtype)
        rot = f if m == 0 and len(f) else None
        want, want_e, want_len = paged.append(pool if eight else wl.to_f64(pool, "bf16"), e, x64, np.asarray(cache.table.cpu()), lens,
                                              count, rows, rot, interleaved, shift, decode)
        np.testing.assert_array_equal(new.cpu().numpy(), want_len)
        raw = got.contiguous().cpu()
        if eight:
            np.testing.assert_array_equal(got_e.cpu().numpy(), want_e)
            bytes_ = raw.numpy()
            value = decode(bytes_)
            untouched = np.isnan(want) & ~np.isnan(value)
            np.testing.assert_array_equal(bytes_[untouched], pool[untouched])
            fresh = ~np.isnan(want)
            tol = np.maximum(U8 * np.abs(want), 2.0 ** -10) + 64 * U32 * 448        # a pair is no longer than sqrt(2) * 448 of a page's units
            assert np.all(np.abs(value - want)[fresh] <= tol[fresh])
        else:
            value = U.from_device_f64(raw)
            untouched = np.isnan(want)
            np.testing.assert_array_equal(value[untouched], wl.to_f64(pool, "bf16")[untouched])
            tol = UBF * np.abs(want) + 64 * U32 * np.nanmax(np.abs(np.where(np.isfinite(want), want, np.nan)))
            assert np.all(np.abs(value - want)[~untouched] <= tol[~untouched])


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B, H, D, ps, n, lens, count, rotary, interleaved, token_major", [
    (1, 2, 128, 16, 1, [0], None, 128, False, False), (3, 3, 64, 16, 1, [5, 16, 47], None, 64, True, True),
    (2, 2, 128, 32, 40, [31, 0], [40, 17], 64, False, True), (2, 5, 64, 64, 130, [100, 64], [130, 1], 0, False, False),
    (1, 1, 128, 128, 300, [77], None, 128, True, False), (2, 1, 128, 256, 280, [250, 3], [280, 0], 32, False, True),
    (1, 2, 64, 256, 200, [100], None, 64, False, False), (4, 2, 64, 16, 33, [0, 15, 16, 17], [0, 33, 16, 15], 16, True, False)])
def test_append(eight, dtype, B, H, D, ps, n, lens, count, rotary, interleaved, token_major):
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(ps + n + B)
    most = max(-(-(l + n) // ps) for l in lens)
    table = random_table(g, B, most, B * most + 2)
    host, exps, cache = make_cache(g, B * most + 2, H, ps, D, eight, table, token_major)
    K, V = (wl.store((g.standard_normal((B, H, n, D)) * np.exp(g.standard_normal((H, 1, 1)))).astype(np.float32), dtype) for _ in range(2))
    to = (lambda a: dev(a.transpose(0, 2, 1, 3).copy(), dtype).transpose(1, 2)) if token_major else (lambda a: dev(a, dtype))
    f, f_dev = inv_freq(rotary)
    new = api.kv_append_paged(cache, to(K), to(V), i32(lens), count=None if count is None else i32(count), inv_freq=f_dev,
                              interleaved=interleaved, shift=2)
    torch.cuda.synchronize()
    check_append(host, exps, cache, K, V, dtype, lens, [n] * B if count is None else count, None, f, interleaved, 2, new)


@pytest.mark.parametrize("eight", [True, False])
def test_append_of_branches_bad_rows_and_pages(eight):
    """accept_len / accept_node as verification leaves them, row indices that are none, pages that are none, full and clamped
    sequences, counts that are too large or negative."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(5)
    B, H, D, ps, n, most, P = 8, 2, 64, 16, 20, 3, 30
    table = random_table(g, B, most, P)
    table[2, 1], table[3, 0], table[7, 2] = -1, P, 2 ** 31 - 1
    lens = [14, 30, 10, 3, 48, 60, -7, 32]
    accept_len = [4, 21, 20, 5, 9, 3, 12, 2]
    rows = g.permuted(np.tile(np.arange(n), (B, 1)), axis=1)
    rows[0, 1], rows[6, 0], rows[6, 3] = -1, n, 2 ** 31 - 1
    host, exps, cache = make_cache(g, P, H, ps, D, eight, table)
    K, V = (wl.store(g.standard_normal((B, H, n, D)).astype(np.float32), "bf16") for _ in range(2))
    new = api.kv_append_paged(cache, dev(K, "bf16"), dev(V, "bf16"), i32(lens), count=i32(accept_len), count_shift=-1, rows=i32(rows))
    torch.cuda.synchronize()
    check_append(host, exps, cache, K, V, "bf16", lens, [a - 1 for a in accept_len], rows, np.zeros(0), False, 0, new)
    assert new.tolist()[3] == 3 and new.tolist()[4:6] == [48, 48]
    for counts, want in (([0] * B, [14, 30, 10, 3, 48, 48, 0, 32]), ([-2 ** 31] * B, [14, 30, 10, 3, 48, 48, 0, 32]),
                         ([2 ** 31 - 1] * B, [34, 48, 16, 3, 48, 48, 20, 32])):
        before = [t.clone() for t in (cache.k, cache.v)]
        new = api.kv_append_paged(cache, dev(K, "bf16"), dev(V, "bf16"), i32(lens), count=i32(counts), count_shift=-1)
        assert new.tolist() == want
        if max(counts) <= 0:
            assert torch.equal(before[0], cache.k) and torch.equal(before[1], cache.v)


def test_append_of_zeros_infinities_and_nans():
    """They stay in their own rows; the exponent is that of the finite values; NaN pages stay NaN when their exponent rises."""
    import torch
    from paper_2406_17276_amd import api
    cache = api.alloc_paged_cache(2, 1, 16, 64, 1, 2)
    cache.table.copy_(i32([[1, 0]]))
    x = torch.zeros(1, 1, 4, 64, device="cuda")
    new = api.kv_append_paged(cache, x, x, i32([0]))
    assert cache.k_exp[1, 0].item() == 1 and not cache.k[1, 0, :4].any()
    x[0, 0, 0] = 3.0
    x[0, 0, 1, 7], x[0, 0, 1, 8], x[0, 0, 2, 9] = float("inf"), float("-inf"), float("nan")
    api.kv_append_paged(cache, x, x, new)
    y = cache.k[1, 0, :8].view(torch.float8_e4m3fn).float()
    assert cache.k_exp[1, 0].item() == paged.needed_exponent(3.0)
    f = 2.0 ** (cache.k_exp[1, 0].item() - 127)
    assert (y[4] * f == 3.0).all() and y[5, 7] == 448 and y[5, 8] == -448 and torch.isnan(y[6, 9])
    assert torch.isnan(y).sum() == 1 and (y[7] == 0).all()
    big = torch.full((1, 1, 1, 64), 3e38, device="cuda")
    api.kv_append_paged(cache, big, big, i32([8]))
    y = cache.k[1, 0, :9].view(torch.float8_e4m3fn).float()
    assert cache.k_exp[1, 0].item() == paged.needed_exponent(float(np.float32(3e38)))
    assert torch.isnan(y[6, 9]) and (y[4] == 0).all() and abs(y[8, 0].item() * 2.0 ** (cache.k_exp[1, 0].item() - 127) / 3e38 - 1) <= U8


def test_appends_one_by_one_agree_with_one():
    """16-bit pages: token by token is the same as all at once; with rotation on the way the same as rotating first."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(1)
    K, V = (torch.randn(2, 2, 21, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = i32([[0, 1, 2], [5, 4, 3]])
    f, f_dev = inv_freq(128)
    caches = [api.alloc_paged_cache(6, 2, 16, 128, 2, 3, eight_bit=False) for _ in range(3)]
    for c in caches:
        c.k.zero_(); c.v.zero_(); c.table.copy_(table)
    lens = i32([9, 20])
    api.kv_append_paged(caches[0], K, V, lens, inv_freq=f_dev)
    at = lens
    for j in range(21):
        at = api.kv_append_paged(caches[1], K[:, :, j:j + 1], V[:, :, j:j + 1], at, inv_freq=f_dev)
    assert at.tolist() == [30, 41]
    _, turned = api.qk_norm_rope(None, K, lens, f_dev)
    api.kv_append_paged(caches[2], turned, V, lens)
    for c in caches[1:]:
        assert torch.equal(c.k, caches[0].k) and torch.equal(c.v, caches[0].v)


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------
def tree_masks(g, B, n, keys, kind):
    bits = np.zeros((B, n, (keys + 63) // 64 * 64), dtype=np.uint8)
    if kind == "tree":
        for b in range(B):
            for i in range(n):
                p = int(g.integers(-1, min(i, keys))) if i else -1
                if p >= 0:
                    bits[b, i] = bits[b, p]
                if i < keys:
                    bits[b, i, i] = 1
    elif kind == "random":
        bits[..., :keys] = g.random((B, n, keys)) < 0.2
        bits[:, 0] = 0                                       # a query that sees no tree key
    return np.packbits(bits, axis=-1, bitorder="little").view(np.uint64)


def check_attention(got, Q, host, exps, table, lens, Kt=None, Vt=None, mask=None, scale=None):
    eight = exps[0] is not None
    pools = host if eight else [wl.to_f64(p, "bf16") for p in host]
    f64 = lambda a: None if a is None else wl.to_f64(a, "bf16")
    D = Q.shape[-1]
    O, A, S = paged.attention(f64(Q), pools, exps, table, lens, f64(Kt), f64(Vt), mask, decode if eight else None, scale)
    tol = A * (2 * UBF + 2.0 ** -14 + 2 * (D + 4) * U32 * S[..., None])
    err = np.abs(U.from_device_f64(got) - O)
    assert np.all(err <= tol), (err.max(), (err / np.maximum(tol, 1e-30)).max())


CASES = [  # B, Hq, Hkv, D, n, keys, kind, ps, lens
    (1, 4, 1, 128, 1, 0, None, 16, [1]), (1, 8, 2, 128, 1, 0, None, 64, [300]), (2, 8, 8, 64, 1, 0, None, 16, [0, 77]),
    (2, 4, 4, 128, 5, 5, "tree", 32, [33, 500]), (1, 2, 2, 128, 50, 50, "tree", 64, [129]), (3, 2, 1, 64, 31, 31, "tree", 16, [0, 64, 65]),
    (2, 8, 2, 128, 20, 20, "tree", 16, [200, 15]), (1, 16, 2, 128, 60, 60, "tree", 64, [700]), (2, 6, 2, 64, 50, 50, "tree", 128, [260, 31]),
    (1, 2, 1, 128, 256, 256, "tree", 256, [400]), (1, 5, 5, 64, 7, 70, "random", 32, [40]), (2, 4, 2, 128, 64, 200, "random", 16, [90, 0]),
    (2, 3, 1, 64, 120, 300, "random", 64, [0, 1]), (1, 4, 1, 128, 3, 0, None, 16, [2100]), (65, 2, 2, 64, 2, 2, "tree", 16, None),
    (1, 1, 1, 128, 200, 1, "random", 16, [17])]


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}/{c[2]}x{c[3]} n{c[4]} keys{c[5]} page{c[7]}" for c in CASES])
def test_attention(eight, case):
    import torch
    from paper_2406_17276_amd import api
    B, Hq, Hkv, D, n, keys, kind, ps, lens = case
    g = np.random.default_rng(n + ps + B)
    lens = [int(x) for x in g.integers(0, 200, B)] if lens is None else lens
    most = max(1, max(-(-l // ps) for l in lens)) + 1
    table = random_table(g, B, most, B * most + 1)
    host, exps, cache = make_cache(g, B * most + 1, Hkv, ps, D, eight, table, token_major=n % 2 == 1)
    Q = wl.store(g.standard_normal((B, Hq, n, D)).astype(np.float32), "bf16")
    Kt = Vt = mask = None
    if keys:
        Kt, Vt = (wl.store(g.standard_normal((B, Hkv, keys, D)).astype(np.float32), "bf16") for _ in range(2))
        mask = tree_masks(g, B, n, keys, kind)
    got = api.tree_verify_attention_paged(dev(Q, "bf16"), cache, i32(lens), None if Kt is None else dev(Kt, "bf16"),
                                          None if Vt is None else dev(Vt, "bf16"), None if mask is None else U.mask_to_device(mask))
    torch.cuda.synchronize()
    check_attention(got, Q, host, exps, table, lens, Kt, Vt, mask)


@pytest.mark.parametrize("n, g_", [(1, 4), (40, 1), (40, 3), (64, 8)])
@pytest.mark.parametrize("eight", [True, False])
def test_attention_ignores_what_nobody_sees(eight, n, g_):
    """NaNs and infinities behind the last row, in tree rows that no query sees and in pages that are none change nothing;
    lengths beyond the table are clamped; both are reported."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(n)
    B, Hkv, D, ps, most = 3, 2, 128, 16, 8
    table = random_table(g, B, most, 30)
    table[1, 2], table[1, 6], table[2, 0] = -1, 30, -2 ** 31
    lens = [37, 128, 5]
    host, exps, cache = make_cache(g, 30, Hkv, ps, D, eight, table)
    bad8 = np.array([0x7f, 0xff], dtype=np.uint8)
    bad16 = np.array([0x7f80, 0xff80, 0x7fc0], dtype=np.uint16)
    for pool in host:
        for b in range(B):
            for r in range(lens[b], most * ps):
                if 0 <= table[b, r // ps] < 30:
                    pool[table[b, r // ps], :, r % ps] = g.choice(bad8 if eight else bad16, (Hkv, D))
    for name, pool in zip(("k", "v"), host):
        getattr(cache, name).copy_(dev(pool, "u8" if eight else "bf16"))
    keys = n + 30
    Q = wl.store(g.standard_normal((B, Hkv * g_, n, D)).astype(np.float32), "bf16")
    Kt, Vt = (wl.store(g.standard_normal((B, Hkv, keys, D)).astype(np.float32), "bf16") for _ in range(2))
    mask = tree_masks(g, B, n, n, "tree")
    mask = np.concatenate([mask, np.zeros((B, n, (keys + 63) // 64 - mask.shape[2]), dtype=np.uint64)], -1)
    clean = [a.copy() for a in (Kt, Vt)]
    for a in (Kt, Vt):
        a[:, :, n:] = g.choice(bad16, a[:, :, n:].shape)
    q = dev(Q, "bf16")
    ws = api.paged_attn_workspace(q, cache, dev(Kt, "bf16"))
    got = api.tree_verify_attention_paged(q, cache, i32(lens), dev(Kt, "bf16"), dev(Vt, "bf16"), U.mask_to_device(mask), workspace=ws)
    assert api.attn_status(ws) == api.OT_ATTN_STATUS_BAD_PAGE
    check_attention(got, Q, host, exps, table, lens, clean[0], clean[1], mask)
    again = api.tree_verify_attention_paged(q, cache, i32([37, 1000, -4]), dev(Kt, "bf16"), dev(Vt, "bf16"), U.mask_to_device(mask), workspace=ws)
    assert api.attn_status(ws) == api.OT_ATTN_STATUS_BAD_PAGE | api.OT_ATTN_STATUS_PREFIX_CLAMPED
    check_attention(again, Q, host, exps, table, [37, 128, 0], clean[0], clean[1], mask)
    assert not ws[4096:65536].any()                              # tickets are left as they were


def test_attention_strides_scales_and_empty_queries():
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(9)
    B, Hq, Hkv, D, n, ps = 2, 4, 2, 64, 40, 32
    table = random_table(g, B, 4, 9)
    lens = [0, 100]
    host, exps, cache = make_cache(g, 9, Hkv, ps, D, True, table)
    Q = wl.store(g.standard_normal((B, Hq, n, D)).astype(np.float32), "bf16")
    Kt, Vt = (wl.store(g.standard_normal((B, Hkv, n, D)).astype(np.float32), "bf16") for _ in range(2))
    mask = tree_masks(g, B, n, n, "tree")
    mask[0, 7] = 0                                               # sequence 0 has no cache: this query sees nothing
    turn = lambda a: dev(a.transpose(0, 2, 1, 3).copy(), "bf16").transpose(1, 2)
    out = torch.full((B, n, Hq, 2 * D), 9.0, dtype=torch.bfloat16, device="cuda")
    o = out[..., :D].transpose(1, 2)
    api.tree_verify_attention_paged(turn(Q), cache, i32(lens), turn(Kt), turn(Vt), U.mask_to_device(mask), out=o, softmax_scale=0.37)
    torch.cuda.synchronize()
    check_attention(o, Q, host, exps, table, lens, Kt, Vt, mask, 0.37)
    assert not o[0, :, 7].any() and (out[..., D:] == 9.0).all()


@pytest.mark.parametrize("eight, Hq, Hkv, D, n, ps", [(True, 8, 1, 128, 1, 16), (False, 4, 4, 128, 40, 64), (True, 8, 2, 64, 60, 128),
                                                      (True, 16, 2, 128, 100, 64)])
def test_attention_over_long_contexts(eight, Hq, Hkv, D, n, ps):
    """Contexts that are cut into ranges, of very different lengths; scores that grow along the context move the reference."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(ps)
    lens = [9001, 3, 2500]
    most = -(-max(lens) // ps)
    table = random_table(g, 3, most, 3 * most)
    host, exps, cache = make_cache(g, 3 * most, Hkv, ps, D, eight, table)
    Q = wl.store((g.standard_normal((3, Hq, n, D)) * 2).astype(np.float32), "bf16")
    if eight:                                                    # page by page larger keys
        for b in range(3):
            for p in range(most):
                exps[0][table[b, p]] = 110 + 12 * p // most
        cache.k_exp.copy_(dev(exps[0], "u8"))
    Kt, Vt = (wl.store(g.standard_normal((3, Hkv, n, D)).astype(np.float32), "bf16") for _ in range(2))
    mask = tree_masks(g, 3, n, n, "tree")
    args = (dev(Q, "bf16"), cache, i32(lens), dev(Kt, "bf16"), dev(Vt, "bf16"), U.mask_to_device(mask))
    ws = api.paged_attn_workspace(args[0], cache, args[3])
    got = api.tree_verify_attention_paged(*args, workspace=ws)
    check_attention(got, Q, host, exps, table, lens, Kt, Vt, mask)
    for _ in range(3):
        assert torch.equal(api.tree_verify_attention_paged(*args, workspace=ws), got)          # joins in a fixed order


def test_two_streams_and_shapes_share_nothing_but_the_pool():
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(3)
    cache = api.alloc_paged_cache(64, 2, 64, 128, 1, 64)
    cache.table.copy_(torch.randperm(64, device="cuda", dtype=torch.int32)[None])
    x = torch.randn(1, 2, 4000, 128, device="cuda").to(torch.bfloat16)
    new = api.kv_append_paged(cache, x, x, i32([0]))
    q = [torch.randn(1, 4, k, 128, device="cuda").to(torch.bfloat16) for k in (1, 60)]
    ws = [api.paged_attn_workspace(t, cache) for t in q]
    want = [api.tree_verify_attention_paged(t, cache, new, workspace=w) for t, w in zip(q, ws)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, t, w in zip(streams, q, ws):
            with torch.cuda.stream(s):
                got.append(api.tree_verify_attention_paged(t, cache, new, workspace=w))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for t in q:                                                   # one workspace, sizes in turn
        assert torch.equal(api.tree_verify_attention_paged(t, cache, new, workspace=max(ws, key=lambda w: w.numel())),
                           want[0 if t is q[0] else 1])


# ---------------------------------------------------------------------------------------------------------------
# together: prompt, draft tree, verification, accepted branch, generated token
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("eight", [True, False])
def test_a_decoding_step_over_a_paged_cache(eight):
    """The layer's own arithmetic around the framework's tree: rows that the cache has at the end attend as the same rows of a
    contiguous cache do (ot_tree_verify_attention), graph replays equal the eager calls."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(7)
    B, Hq, Hkv, D, V, n, depth, k, ps, cap = 2, 8, 2, 128, 1000, 24, 5, 4, 16, 512
    bf = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    cache = api.alloc_paged_cache(B * cap // ps, Hkv, ps, D, B, cap // ps, eight_bit=eight)
    cache.table.copy_(torch.randperm(B * cap // ps, device="cuda", dtype=torch.int32).view(B, -1))
    f, f_dev = inv_freq(D)
    w = bf(D)
    # prompt: norm, rotation on the way into the cache
    K, Vv = bf(B, Hkv, 200, D), bf(B, Hkv, 200, D)
    _, Kn = api.qk_norm_rope(None, K, i32([0, 0]), None, k_weight=w)
    length = api.kv_append_paged(cache, Kn, Vv, i32([0, 0]), count=i32([200, 131]), inv_freq=f_dev)
    assert length.tolist() == [200, 131]
    draft, target = bf(B, depth, n, V) * 3, bf(B, n + 1, V) * 4
    Qt, Kt, Vt = bf(B, Hq, n, D), bf(B, Hkv, n, D), bf(B, Hkv, n, D)
    q1, k1, v1 = bf(B, Hq, 1, D), bf(B, Hkv, 1, D), bf(B, Hkv, 1, D)
    ws = api.paged_attn_workspace(Qt, cache, Kt)
    ws1 = api.paged_attn_workspace(q1, cache)
    tree = api.alloc_tree(B, n)

    def step():
        api.build_tree(draft, k, n, depth, out=tree)
        q, kk = api.qk_norm_rope(Qt, Kt, length, f_dev, offset=tree.depth, shift=-1, q_weight=w, k_weight=w)
        out = api.tree_verify_attention_paged(q, cache, length, kk, Vt, tree.mask, workspace=ws)
        # accept the branch that the target agrees with: force agreement with the first nodes of the tree
        alen, anode, _ = api.verify_greedy(target, tree)
        after = api.kv_append_paged(cache, kk, Vt, length, count=alen, count_shift=-1, rows=anode)
        qq, _ = api.qk_norm_rope(q1, None, after, f_dev, q_weight=w)
        after1 = api.kv_append_paged(cache, k1, v1, after, inv_freq=f_dev)
        out1 = api.tree_verify_attention_paged(qq, cache, after1, workspace=ws1)
        return q, kk, out, alen, anode, after, qq, after1, out1

    # make the target agree with a child of the root and one of its children
    api.build_tree(draft, k, n, depth, out=tree)
    tok, par = tree.token.cpu(), tree.parent.cpu()
    for b in range(B):
        i = int((par[b] == -1).nonzero()[0])
        target[b, 0, tok[b, i]] = 100.0
        kids = (par[b] == i).nonzero()
        if len(kids):
            target[b, 1 + i, tok[b, int(kids[0])]] = 100.0
    q, kk, out, alen, anode, after, qq, after1, out1 = step()
    torch.cuda.synchronize()
    assert (alen >= 2).all() and torch.equal(after, length + alen - 1) and torch.equal(after1, after + 1)

    def contiguous(name):
        pages = getattr(cache, name)[cache.table.long()]                  # [B, pages, H, ps, D]
        x = pages.float() if not eight else pages.view(torch.float8_e4m3fn).float() * torch.exp2(
            getattr(cache, name + "_exp")[cache.table.long()].float() - 127)[..., None, None]
        return x.transpose(1, 2).reshape(B, Hkv, cap, D)
    Kc, Vc = contiguous("k"), contiguous("v")
    rows = [(Kc[b, :, :int(after[b])], Vc[b, :, :int(after[b])]) for b in range(B)]
    for b in range(B):                                                    # the accepted rows are where they belong
        for j in range(int(alen[b]) - 1):
            at, node = int(length[b]) + j, int(anode[b, j])
            unit = rows[b][0].abs().amax()
            assert ((rows[b][0][:, at] - kk[b, :, node].float()).abs() <= kk[b, :, node].float().abs() * (U8 if eight else 0) + (unit * 2.0 ** -17 if eight else 0)).all()
    # bf16 holds every value of either cache, so the contiguous attention reads the same numbers
    plain = api.tree_verify_attention(q, Kc.to(torch.bfloat16), Vc.to(torch.bfloat16), kk, Vt, length, tree.mask)
    # (rows behind a sequence's last one were never written: only those that are attended to say how large V is)
    scale = max(float(r[1].abs().amax()) for r in rows + [(None, Vt.float())])
    assert ((plain.float() - out.float()).abs() <= 4 * UBF * scale).all()    # two roundings of weights and two of results

    g_cache = [t.clone() for t in (cache.k, cache.v) + ((cache.k_exp, cache.v_exp) if eight else ())]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            recorded = step()
    for replay in range(3):
        draft.copy_(bf(B, depth, n, V) * 3); Qt.copy_(bf(B, Hq, n, D)); Kt.copy_(bf(B, Hkv, n, D)); k1.copy_(bf(B, Hkv, 1, D))
        for t, saved in zip((cache.k, cache.v) + ((cache.k_exp, cache.v_exp) if eight else ()), g_cache):
            t.copy_(saved)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in recorded] + [cache.k.clone(), cache.v.clone()]
        for t, saved in zip((cache.k, cache.v) + ((cache.k_exp, cache.v_exp) if eight else ()), g_cache):
            t.copy_(saved)
        want = list(step()) + [cache.k, cache.v]
        torch.cuda.synchronize()
        # bit by bit: rows that nothing has written may be NaNs
        assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(got, want)), replay


# ---------------------------------------------------------------------------------------------------------------
# calls that the documentation allows and the cases above do not make
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("eight", [True, False])
def test_pools_of_more_than_4_gib(eight):
    """Pages behind 2^32 bytes: what an append writes there is what an attention reads, and equals the same rows in a small pool."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(11)
    H, ps, D, n = 8, 64, 128, 150
    pages = (5 << 30) // (H * ps * D * (1 if eight else 2))
    big = api.alloc_paged_cache(pages, H, ps, D, 1, 4, eight_bit=eight)
    small = api.alloc_paged_cache(4, H, ps, D, 1, 4, eight_bit=eight)
    ids = [pages - 1, 3, pages // 2 + 7, pages - 2]
    big.table.copy_(i32([ids]))
    small.table.copy_(i32([[2, 0, 3, 1]]))
    K, V = (torch.randn(1, H, n, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    f, f_dev = inv_freq(D)
    for q_rows in (1, 40, 200):
        Q = torch.randn(1, H, q_rows, D, device="cuda").to(torch.bfloat16)
        out = []
        for c in (big, small):
            new = api.kv_append_paged(c, K, V, i32([0]), inv_freq=f_dev)
            new = api.kv_append_paged(c, K[:, :, :30], V[:, :, :30], new, inv_freq=f_dev)
            assert new.tolist() == [180]
            out.append(api.tree_verify_attention_paged(Q, c, new))
        assert torch.equal(out[0], out[1]) and torch.isfinite(out[0]).all()
    for a, b in ((ids[0], 2), (ids[1], 0)):
        assert torch.equal(big.k[a].view(torch.uint8), small.k[b].view(torch.uint8)) and torch.equal(big.v[a].view(torch.uint8), small.v[b].view(torch.uint8))


@pytest.mark.parametrize("B, Hq, Hkv, n", [(300, 2, 1, 1), (130, 2, 2, 3), (300, 4, 2, 40)])
def test_attention_of_large_batches(B, Hq, Hkv, n):
    """More sequences than lanes, and more than are cut into ranges; one of them is long."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(B + n)
    D, ps = 64, 16
    lens = g.integers(0, 40, B).tolist()
    lens[B - 2] = 700
    counts = [-(-l // ps) for l in lens]
    order = g.permutation(sum(counts))
    table = np.full((B, max(counts)), -1)
    at = 0
    for b, c in enumerate(counts):                               # entries behind a sequence's pages are no pages, and not read
        table[b, :c] = order[at:at + c]
        at += c
    host, exps, cache = make_cache(g, sum(counts), Hkv, ps, D, True, table)
    Q = wl.store(g.standard_normal((B, Hq, n, D)).astype(np.float32), "bf16")
    q = dev(Q, "bf16")
    ws = api.paged_attn_workspace(q, cache)
    got = api.tree_verify_attention_paged(q, cache, i32(lens), workspace=ws)
    assert api.attn_status(ws) == 0
    check_attention(got, Q, host, exps, table, lens)


def test_padded_pools_and_fused_projections():
    """Pools that are slices of larger ones (pages, heads and rows further apart than they are long), rows of a fused projection."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(5)
    B, H, ps, D, n = 2, 3, 32, 64, 50
    for eight in (True, False):
        t = torch.uint8 if eight else torch.bfloat16
        store = [torch.full((9, 4, ps + 3, D + 16), 7, dtype=t, device="cuda") for _ in range(2)]
        views = [x[1:, :H, 1:ps + 1, 16:] for x in store]
        exps = [torch.full((8, H), 120, dtype=torch.uint8, device="cuda") for _ in range(2)] if eight else [None, None]
        table = i32([[7, 0, 3], [2, 6, 4]])
        slices, plain = api.PagedCache(*views, table, *exps), api.alloc_paged_cache(8, H, ps, D, B, 3, eight_bit=eight)
        plain.table.copy_(table)
        fused = torch.randn(B, n, 5 * H, D, device="cuda").to(torch.bfloat16)
        K, V = fused[:, :, H:2 * H].transpose(1, 2), fused[:, :, 4 * H:].transpose(1, 2)
        for c in (slices, plain):
            new = api.kv_append_paged(c, K, V, i32([0, 20]), count=i32([50, 44]))
        assert new.tolist() == [50, 64]
        Q = torch.randn(B, 2 * H, 9, D, device="cuda").to(torch.bfloat16)
        lens = i32([50, 20])                                     # (rows 0..19 of the second are not the same in both pools)
        a, b = (api.tree_verify_attention_paged(Q[:1], api.PagedCache(c.k, c.v, c.table[:1], c.k_exp, c.v_exp), lens[:1]) for c in (slices, plain))
        assert torch.equal(a, b)
        for x, v in zip(store, views):                           # nothing between the rows was touched
            v.fill_(7)
            assert (x == 7).all()


def test_refusals_leave_the_device_alone():
    import torch
    from paper_2406_17276_amd import api
    cache = api.alloc_paged_cache(4, 2, 16, 64, 1, 2)
    q = torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(api.OptTreeError) as e:
        api.tree_verify_attention_paged(q, cache, i32([0]), workspace=torch.zeros(65536, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q, cache, torch.zeros(1, dtype=torch.int32))                     # lengths on the host
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q, cache, torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q.float(), cache, i32([0]))
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q, cache, i32([0]), k, k)                                        # a tree without its mask
    with pytest.raises(ValueError):
        api.kv_append_paged(cache, k, k[:, :, :2], i32([0]))
    with pytest.raises(ValueError):
        api.kv_append_paged(cache, k, k, i32([0]), rows=i32([[0, 1]]))
    with pytest.raises(ValueError):
        api.kv_append_paged(cache, k.transpose(2, 3).contiguous().transpose(2, 3), k, i32([0]))          # last dimension apart
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda"), i32([0]))
    with pytest.raises(ValueError):
        api.qk_norm_rope(q, None, i32([0]), torch.zeros(32, device="cuda"))                              # inv_freq is float64
    with pytest.raises(api.OptTreeError):
        api.qk_norm_rope(q, None, i32([0]), torch.zeros(40, dtype=torch.float64, device="cuda"))         # more than head_dim
    lens = i32([3])
    with pytest.raises(api.OptTreeError):
        api.kv_append_paged(cache, k, k, lens, new_len=lens)                                             # in place
    cache.k_exp = None
    with pytest.raises(TypeError):
        api.kv_append_paged(cache, k, k, lens)
    torch.cuda.synchronize()


def test_prompt_in_chunks_equals_the_prompt_at_once():
    """A prompt of 300 tokens attends in chunks of 64 under a causal mask over what earlier chunks left in 16-bit pages; every
    output row is what plain causal attention gives."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(21)
    Hq, H, D, ps, n, chunk = 6, 2, 128, 32, 300, 64
    f, f_dev = inv_freq(D)
    cache = api.alloc_paged_cache(10, H, ps, D, 1, 10, eight_bit=False)
    cache.table.copy_(torch.randperm(10, device="cuda", dtype=torch.int32)[None])
    Q, K, V = (wl.store(g.standard_normal((1, h, n, D)).astype(np.float32), "bf16") for h in (Hq, H, H))
    q, k, v = (dev(x, "bf16") for x in (Q, K, V))
    length, outs = i32([0]), []
    for c0 in range(0, n, chunk):
        m = min(chunk, n - c0)
        tri = torch.tensor([-1 if i == 63 else (2 << i) - 1 for i in range(m)], dtype=torch.int64, device="cuda").view(1, m, 1)
        qq, kk = api.qk_norm_rope(q[:, :, c0:c0 + m], k[:, :, c0:c0 + m], length, f_dev)
        outs.append(api.tree_verify_attention_paged(qq, cache, length, kk, v[:, :, c0:c0 + m], tri))
        length = api.kv_append_paged(cache, kk, v[:, :, c0:c0 + m], length)
    got = U.from_device_f64(torch.cat(outs, 2))
    qr, kr = api.qk_norm_rope(q, k, i32([0]), f_dev)                      # the same rotated rows, all at once
    qr, kr, v64 = U.from_device_f64(qr), U.from_device_f64(kr), wl.to_f64(V, "bf16")
    for h in range(Hq):
        s = qr[0, h] @ kr[0, h // 3].T / np.sqrt(D)
        s[np.triu_indices(n, 1)] = -np.inf
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        S = np.abs(qr[0, h]) @ np.abs(kr[0, h // 3]).T / np.sqrt(D)
        tol = (w @ np.abs(v64[0, h // 3])) * (2 * UBF + 2.0 ** -14 + 2 * (D + 4) * U32 * S.max())
        assert np.all(np.abs(got[0, h] - w @ v64[0, h // 3]) <= tol)


def test_broadcast_inputs_are_read_and_broadcast_outputs_refused():
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(33)
    B, Hq, H, D, ps, n = 2, 4, 2, 64, 16, 5
    _, f_dev = inv_freq(D)
    new = lambda *s: dev(wl.store(g.standard_normal(s).astype(np.float32), "bf16"), "bf16")
    q, k, v, page = new(1, Hq, n, D).expand(B, -1, -1, -1), new(B, 1, n, D).expand(-1, H, -1, -1), new(B, H, 1, D).expand(-1, -1, n, -1), new(6, 1, ps, D)
    first, lens = i32([30, 7]), i32([30, 16])
    for a, b in zip(api.qk_norm_rope(q, k, first, f_dev), api.qk_norm_rope(q.contiguous(), k.contiguous(), first, f_dev)):
        assert torch.equal(a, b)
    table = i32([[4, 1, 3], [0, 5, 2]])
    one = api.PagedCache(page.expand(-1, H, -1, -1), page.expand(-1, H, -1, -1), table)          # the heads share their keys
    many = api.PagedCache(one.k.contiguous(), one.v.contiguous(), table)
    mask = torch.full((B, n, 1), 31, dtype=torch.int64, device="cuda")
    want = api.tree_verify_attention_paged(q.contiguous(), many, lens, k.contiguous(), v.contiguous(), mask)
    assert torch.equal(api.tree_verify_attention_paged(q, one, lens, k, v, mask), want)
    with pytest.raises(api.OptTreeError):
        api.kv_append_paged(one, k, v, lens)
    with pytest.raises(api.OptTreeError):
        api.qk_norm_rope(q, None, first, f_dev, q_out=q)
    other = api.PagedCache(many.k.clone(), many.v.clone(), table)
    assert torch.equal(api.kv_append_paged(many, k, v, lens, inv_freq=f_dev), i32([35, 21]))
    api.kv_append_paged(other, k.contiguous(), v.contiguous(), lens, inv_freq=f_dev)
    assert torch.equal(many.k, other.k) and torch.equal(many.v, other.v)
