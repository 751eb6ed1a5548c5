"""Corners of the operators around a paged cache on the GPU: what must hold exactly, or whatever lies where nobody looks."""
import numpy as np
import pytest

import workloads as wl
from tests import test_gpu_paged as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("Hq, Hkv, D, n, keys, ps, lens", [
    (256, 256, 64, 1, 0, 16, [700, 300]), (8, 2, 64, 8, 8, 32, [400, 300]), (4, 4, 128, 40, 40, 64, [500, 129]), (6, 2, 128, 30, 30, 16, [600, 90]),
    (128, 128, 64, 70, 70, 64, [333, 500]), (128, 128, 64, 200, 200, 64, [500, 333]), (256, 128, 128, 100, 100, 128, [300, 200])])
def test_an_average_of_equal_rows_is_that_row(eight, Hq, Hkv, D, n, keys, ps, lens):
    """Weights that divide by their own sum average a value to itself.  Rows of V that are all the same: products are exact in fp32, sums of N
    positive terms and the merges are off by less than 2 N 2^-24 + 2^-14 < 2^-12 (N <= 1000), and a bf16 value stays itself under errors below
    2^-9, so the output is V to the last bit.  (A sum of weights that are not those of the products is off by up to 2^-8.)"""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(n + D)
    B = len(lens)
    most = max(-(-l // ps) for l in lens)
    table = P.random_table(g, B, most, B * most)
    host, exps, cache = P.make_cache(g, B * most, Hkv, ps, D, eight, table)
    row = wl.store((1 + g.random(D)).astype(np.float32), "bf16")
    row[:4] = wl.store(np.float32([1, 1.9921875, 1.0078125, 1.5]), "bf16")
    if eight:
        q = wl.f32_to_e4m3_bits(wl.to_f64(row, "bf16").astype(np.float32) * 64)
        row = wl.store(wl.e4m3_bits_to_f32(q) / 64, "bf16")              # 2^(121 - 127)
        cache.v.copy_(P.dev(np.broadcast_to(q, host[1].shape), "u8"))
        cache.v_exp.fill_(121)
    else:
        cache.v.copy_(P.dev(np.broadcast_to(row, host[1].shape), "bf16"))
    Q = P.dev(wl.store((g.standard_normal((B, Hq, n, D)) * 3).astype(np.float32), "bf16"), "bf16")
    Kt = Vt = mask = None
    if keys:
        Kt = P.dev(wl.store(g.standard_normal((B, Hkv, keys, D)).astype(np.float32), "bf16"), "bf16")
        Vt = P.dev(np.broadcast_to(row, (B, Hkv, keys, D)), "bf16")
        mask = P.U.mask_to_device(P.tree_masks(g, B, n, keys, "tree"))
    if eight:
        cache.k_exp.fill_(120)                                           # keys of about 0.7: scores some 3 apart
    got = api.tree_verify_attention_paged(Q, cache, P.i32(lens), Kt, Vt, mask)
    want = P.dev(np.broadcast_to(row, got.shape), "bf16")
    assert torch.equal(got, want), (int((got != want).sum()), got.numel())


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("Hq, Hkv, D, n, keys", [(2, 2, 128, 1, 37), (2, 1, 64, 20, 20), (2, 2, 128, 40, 90), (2, 1, 128, 50, 100), (2, 1, 128, 120, 120)])
def test_mask_bits_behind_the_last_tree_row_mean_nothing(eight, Hq, Hkv, D, n, keys):
    """Every bit of the last word from tree_keys on is set; the last tree row, which no query sees, is NaNs and infinities."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(keys)
    table = P.random_table(g, 2, 6, 12)
    lens = [70, 0]
    host, exps, cache = P.make_cache(g, 12, Hkv, 16, D, eight, table)
    Q, Kt, Vt = (wl.store(g.standard_normal((2, h, r, D)).astype(np.float32), "bf16") for h, r in ((Hq, n), (Hkv, keys), (Hkv, keys)))
    mask = P.tree_masks(g, 2, n, keys, "random")
    mask[:, :, -1] &= ~np.uint64(1 << (keys - 1) % 64)
    mask[:, 0, 0] |= np.uint64(1)
    Kt[:, :, -1] = Vt[:, :, -1] = 0
    run = lambda k, v, m: api.tree_verify_attention_paged(P.dev(Q, "bf16"), cache, P.i32(lens), P.dev(k, "bf16"), P.dev(v, "bf16"), P.U.mask_to_device(m))
    want = run(Kt, Vt, mask)
    P.check_attention(want, Q, host, exps, table, lens, Kt, Vt, mask)
    Kt[:, :, -1], Vt[:, :, -1] = 0x7fc0, 0x7f80
    Vt[:, :, -1, ::2] = 0x7fc0
    mask[:, :, -1] |= np.uint64(-(1 << keys % 64) & (1 << 64) - 1)
    assert torch.equal(run(Kt, Vt, mask), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D, ps, rotary", [(128, 16, 0), (64, 64, 0), (128, 256, 64), (64, 16, 32)])
def test_signalling_nans_hide_no_value(dtype, D, ps, rotary):
    """NaNs whose quiet bit is clear reach the maxima of V, and of key columns that are not turned, as they are: behind larger values
    of their lane, in either run of its columns, in the last place.  They are stored as NaNs and change nothing else."""
    import torch
    from paper_2406_17276_amd import api
    g = np.random.default_rng(D + ps)
    H, n = 2, 20
    pages = -(-(n + 3) // ps)
    table = np.arange(pages)[None]
    host, exps, cache = P.make_cache(g, pages, H, ps, D, True, table)
    for e in exps:
        e[:] = 100                                                       # the older rows' exponent: well below what comes
    cache.k_exp.fill_(100)
    cache.v_exp.fill_(100)
    bits = np.uint16 if dtype == "bf16" else np.uint32
    nans = np.array([0x7f81, 0xffbf] if dtype == "bf16" else [0x7f800001, 0xffbfffff], dtype=bits)
    stored = []
    for turned in (rotary, 0):                                           # K, V
        x = wl.store((g.standard_normal((1, H, n, D)) * 0.1).astype(np.float32), dtype)
        raw = x.view(bits)
        x64 = wl.to_f64(x, dtype)
        for h in range(H):                                               # per head: a large value, then the NaN in its lane
            for i, (big, at) in enumerate(((0, 3), (8, 11), (1, 15), (9, 7), (0, 8))):
                r, c = 4 * i + h, turned + 16 * (i % ((D - turned) // 16))
                raw[0, h, r, c + big] = wl.store(np.float32([200.0 + 10 * i + h]), dtype).view(bits)[0]
                raw[0, h, r, c + at] = nans[i % 2]
        stored.append(x)
    K, V = stored
    f, f_dev = P.inv_freq(rotary)
    new = api.kv_append_paged(cache, P.dev(K, dtype), P.dev(V, dtype), P.i32([3]), inv_freq=f_dev)
    P.check_append(host, exps, cache, K, V, dtype, [3], [n], None, f, False, 0, new)
    for x, pool in ((K, cache.k), (V, cache.v)):
        rows = P.decode(pool.cpu().numpy()).transpose(1, 0, 2, 3).reshape(H, -1, D)[:, 3:3 + n]
        np.testing.assert_array_equal(np.isnan(rows), np.isnan(wl.to_f64(x, dtype)[0]))


def test_sizes_that_32_bits_do_not_hold_are_refused():
    """An axis of 2^32 + 3 rows, broadcast from one, is not one of 3."""
    import torch
    from paper_2406_17276_amd import api
    cache = api.alloc_paged_cache(4, 2, 16, 64, 1, 2)
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    far, q, mask = (1 << 32) + 3, new(1, 2, 3, 64), torch.zeros(1, 3, 1, dtype=torch.int64, device="cuda")
    ws = api.paged_attn_workspace(q, cache)
    long = new(1, 2, 1, 64).expand(-1, -1, far, -1)
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q, cache, P.i32([0]), long, long, mask, workspace=ws)
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(long, cache, P.i32([0]), out=long, workspace=ws)
    many = new(1, 1, 3, 64).expand(-1, (1 << 32) + 2, -1, -1)
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(many, cache, P.i32([0]), out=many, workspace=ws)
    with pytest.raises(ValueError):
        api.qk_norm_rope(many, None, P.i32([0]), q_out=many)
    heads = cache.k[:, :1].expand(-1, (1 << 32) + 2, -1, -1)
    with pytest.raises(ValueError):
        api.tree_verify_attention_paged(q, api.PagedCache(heads, heads, cache.table, cache.k_exp, cache.v_exp), P.i32([0]), workspace=ws)
    with pytest.raises(ValueError):
        api.kv_append_paged(cache, long, long, P.i32([0]))


@pytest.mark.parametrize("eight", [True, False])
def test_an_append_of_very_many_pages_equals_its_pieces(eight):
    """Sequences of up to 80000 pages in one call and in calls of 2000 pages each; one of them meets a table entry that is no page, one
    its capacity, one is nearly empty."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(2)
    H, D, ps, B, most = 1, 64, 16, 4, 80000
    lens, n = [0, 5, 16 * 70000, 3], 16 * 79000
    count = [n, n, n, 7]
    caches = [api.alloc_paged_cache(B * most, H, ps, D, B, most, eight_bit=eight) for _ in range(2)]
    table = torch.randperm(B * most, device="cuda", dtype=torch.int32).view(B, most)
    table[1, 41234], table[1, 60000] = -1, B * most
    for c in caches:
        c.k.zero_(), c.v.zero_(), c.table.copy_(table)
    K, V = (torch.randn(1, H, n, D, device="cuda").to(torch.bfloat16).expand(B, -1, -1, -1) for _ in range(2))
    new = api.kv_append_paged(caches[0], K, V, P.i32(lens), count=P.i32(count))
    want = [n, 16 * 41234, 16 * 80000, 10]
    assert new.tolist() == want
    at = P.i32(lens)
    step = 16 * 2000
    for j in range(0, n, step):
        for b in range(B):
            skew = 11 if b == 1 else 0                                   # row 5 + 11 begins a page: later pieces begin with theirs
            lo, hi = (j + skew if j else 0), min(n, j + step + skew)
            m = max(0, min(hi, count[b]) - lo)
            if m:
                one = api.PagedCache(caches[1].k, caches[1].v, table[b:b + 1], caches[1].k_exp, caches[1].v_exp)
                at[b:b + 1] = api.kv_append_paged(one, K[:1, :, lo:lo + m], V[:1, :, lo:lo + m], at[b:b + 1].clone())
                if int(at[b]) == want[b]:
                    count[b] = 0                                         # what comes after a missing page is dropped, not moved up
    assert at.tolist() == want
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
    if eight:
        assert torch.equal(caches[0].k_exp, caches[1].k_exp) and torch.equal(caches[0].v_exp, caches[1].v_exp)


def test_a_long_append_costs_what_its_pieces_cost():
    """1048576 rows into pages of 16 at once, and 65536 at a time: a cost per row that grows with the length would show as 16 times."""
    import torch
    from paper_2406_17276_amd import api
    H, D, ps, n, parts = 2, 64, 16, 1 << 20, 16
    cache = api.alloc_paged_cache(n // ps, H, ps, D, 1, n // ps, eight_bit=False)
    cache.table.copy_(torch.randperm(n // ps, device="cuda", dtype=torch.int32)[None])
    K = torch.randn(1, H, n, D, device="cuda").to(torch.bfloat16)
    at = [P.i32([i * (n // parts)]) for i in range(parts)]
    rows = [K[:, :, i * (n // parts):(i + 1) * (n // parts)] for i in range(parts)]
    calls = (lambda: api.kv_append_paged(cache, K, K, at[0]), lambda: [api.kv_append_paged(cache, r, r, a) for r, a in zip(rows, at)])

    def best(f):
        times = []
        for _ in range(7):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record(), f(), e[1].record()
            torch.cuda.synchronize()
            times.append(e[0].elapsed_time(e[1]))
        return min(times)
    assert best(calls[0]) < 2 * best(calls[1])


def test_long_appends_in_a_graph():
    """The two launches of a long append, captured once and replayed over other lengths, counts and table entries."""
    import torch
    from paper_2406_17276_amd import api
    torch.manual_seed(4)
    H, D, ps, B, most = 1, 64, 16, 2, 1700
    n = 16 * 1600
    caches = [api.alloc_paged_cache(B * most, H, ps, D, B, most) for _ in range(2)]
    table = torch.randperm(B * most, device="cuda", dtype=torch.int32).view(B, most)
    for c in caches:
        c.k.zero_(), c.v.zero_()
    K, V = (torch.randn(B, H, n, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    lens, count, new = P.i32([0, 0]), P.i32([n, n]), P.i32([0, 0])
    call = lambda c, out: api.kv_append_paged(c, K, V, lens, count=count, new_len=out)
    caches[0].table.copy_(table)
    call(caches[0], new)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call(caches[0], new)
    for c in caches:
        c.k.zero_(), c.v.zero_(), c.k_exp.fill_(127), c.v_exp.fill_(127)
    for at, many, gap in (([0, 5], [n, n], None), ([1, 16 * 1690], [n, n], 1500), ([100, 0], [0, 3], None), ([7, 1600], [n, n - 1], 3), ([0, 0], [n, n], None)):
        lens.copy_(P.i32(at)), count.copy_(P.i32(many))
        for c in caches:
            c.table.copy_(table)
            if gap is not None:
                c.table[0, gap] = -1
        K.mul_(-0.75)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = call(caches[1], P.i32([-1, -1]))
        assert torch.equal(new, eager), (at, many, gap)
        for name in ("k", "v", "k_exp", "v_exp"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), (name, at)
    assert new.tolist() == [n, n]
