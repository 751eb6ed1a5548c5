"""The operators around a paged key/value cache, as timed cases: what a serving decoder does between a layer's projections
and its output projection.

  rope    queries and keys of new tokens: norm of every head, rotation by the token's position, in one pass
  append  keys and values of new tokens (a prompt, a generated token, an accepted branch of a draft tree) into the pages of
          a cache, keys rotated on the way where they come straight from the projection; pages hold bfloat16, or E4M3 bytes
          with a power of two for every page and head
  attn    attention of a draft tree (or of a single new token) over such a cache and the tree's own keys

With `own` false, run() computes them in elementary torch operations in 32 bits; with `own` true through
`paper_2406_17276_amd.api`.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one generated token of one user, grouped-query model with head norms: launch latency is all there is
        dict(name="rope_token", kind="rope", dtype="bf16", batch=1, n=1, q_heads=32, kv_heads=8, head_dim=128, rotary=128,
             interleaved=False, norm=True, tree=False, token_major=True, first=20000),
        # the draft trees of a serving batch, positions by depth
        dict(name="rope_tree_70b", kind="rope", dtype="bf16", batch=16, n=60, q_heads=64, kv_heads=8, head_dim=128, rotary=128,
             interleaved=False, norm=True, tree=True, token_major=False, first=4096),
        # a long prompt in 32 bits, half of each head rotated in neighbouring pairs
        dict(name="rope_prompt_f32", kind="rope", dtype="f32", batch=3, n=5003, q_heads=32, kv_heads=8, head_dim=128, rotary=64,
             interleaved=True, norm=False, tree=False, token_major=True, first=100000),
        # the accepted branch of one sequence's draft tree joins a cache kept in 8 bits
        dict(name="append_branch_8bit", kind="append", dtype="bf16", cache="e4m3", batch=1, n=50, mode="branch", kv_heads=32,
             head_dim=128, page=64, prefix=1024, ragged=0.0, rotary=0, interleaved=False, token_major=False),
        # one generated token for every sequence of a batch, key rotated on the way into 8 bits
        dict(name="append_token_8bit", kind="append", dtype="bf16", cache="e4m3", batch=64, n=1, mode="rows", kv_heads=8,
             head_dim=128, page=16, prefix=2500, ragged=0.5, rotary=128, interleaved=False, token_major=True),
        # prompts of unequal length, 16-bit pages, heads of 64
        dict(name="append_prompt", kind="append", dtype="bf16", cache="bf16", batch=7, n=1777, mode="rows", kv_heads=5,
             head_dim=64, page=32, prefix=100, ragged=0.5, rotary=64, interleaved=True, token_major=True),
        # long prompts into 8 bits
        dict(name="append_prompt_8bit", kind="append", dtype="bf16", cache="e4m3", batch=8, n=8192, mode="rows", kv_heads=8,
             head_dim=128, page=64, prefix=0, ragged=0.0, rotary=128, interleaved=False, token_major=True),
        # one token of one user over a middling context
        dict(name="attn_token", kind="attn", cache="e4m3", batch=1, n=1, tree=0, q_heads=32, kv_heads=8, head_dim=128, page=64,
             prefix=1500, ragged=0.0),
        # the draft tree of one sequence, multi-head target, 16-bit pages
        dict(name="attn_tree_7b", kind="attn", cache="bf16", batch=1, n=50, tree=1, q_heads=32, kv_heads=32, head_dim=128,
             page=64, prefix=1024, ragged=0.0),
        # single tokens over long contexts: the cache streams past
        dict(name="attn_token_long", kind="attn", cache="e4m3", batch=4, n=1, tree=0, q_heads=64, kv_heads=8, head_dim=128,
             page=16, prefix=100000, ragged=0.25),
        # the draft trees of a serving batch
        dict(name="attn_tree_70b", kind="attn", cache="e4m3", batch=16, n=60, tree=1, q_heads=64, kv_heads=8, head_dim=128,
             page=64, prefix=4096, ragged=0.25),
        # the large node budget: bound by the matrix cores
        dict(name="attn_tree_large", kind="attn", cache="e4m3", batch=16, n=256, tree=1, q_heads=32, kv_heads=8, head_dim=128,
             page=64, prefix=8192, ragged=0.0),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 150)


def draw(rng):
    kind = rng.choice(("rope", "append", "append", "attn", "attn", "attn"))
    c = dict(kind=kind)
    most = max(_cost(x) for x in listed() if x["kind"] == kind)
    if kind != "attn":
        c["dtype"] = rng.choice(("bf16", "bf16", "bf16", "f32"))
    c["batch"] = _log(rng, 1, 64)
    c["kv_heads"] = _log(rng, 1, 40)
    g = rng.choice((1, 1, 2, 4, 5, 8))
    if kind != "append":
        c["q_heads"] = g * c["kv_heads"]
    while c.get("q_heads", 0) > 64:
        c["kv_heads"] -= 1
        c["q_heads"] = g * c["kv_heads"]
    c["head_dim"] = rng.choice((64, 128, 128))
    if kind != "rope":
        c["cache"] = rng.choice(("bf16", "e4m3", "e4m3"))
        c["page"] = rng.choice((16, 32, 64, 64, 128, 256))
        c["ragged"] = rng.choice((0.0, 0.25, 0.5))
    if kind != "attn":
        c["rotary"] = rng.choice((c["head_dim"], c["head_dim"], c["head_dim"] // 2, 0 if kind == "append" else c["head_dim"]))
        c["interleaved"] = rng.random() < 0.3
        c["token_major"] = rng.random() < 0.6
    if kind == "rope":
        c["norm"] = rng.random() < 0.7
        c["tree"] = rng.random() < 0.4
        c["first"] = _log(rng, 1, 1000000)
        c["n"] = _log(rng, 1, 256 if c["tree"] else 8192)
    if kind == "append":
        c["mode"] = rng.choice(("rows", "rows", "branch"))
        c["prefix"] = rng.choice((0, _log(rng, 1, 20000), _log(rng, 1, 20000)))
        c["n"] = _log(rng, 4, 256) if c["mode"] == "branch" else _log(rng, 1, 8192)
    if kind == "attn":
        c["tree"] = rng.choice((0, 1, 1, rng.randint(2, 10)))
        c["n"] = rng.choice((1, 1, _log(rng, 2, 8))) if c["tree"] == 0 else _log(rng, 1, 256)
        c["prefix"] = _log(rng, 1, 131072)
    while _cost(c) > most or kind != "rope" and _pool_bytes(c) > 4e9:
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 3 // 4
        elif kind == "attn" and c["prefix"] > 1:
            c["prefix"] = c["prefix"] * 3 // 4
        elif kind == "append" and c["prefix"] > 64:
            c["prefix"] //= 2
        else:
            c["n"] = c["n"] * 3 // 4
    return c


def _pool_bytes(c):
    rows = (c["prefix"] * (1 + c["ragged"]) + c["n"] * (c["kind"] == "append") + c["page"]) * c["batch"]
    return rows * c["kv_heads"] * c["head_dim"] * 2 * 4


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once, products of the cached rows."""
    c = case
    if c["kind"] == "rope":
        elements = c["batch"] * c["n"] * (c["q_heads"] + c["kv_heads"]) * c["head_dim"]
        return dict(bytes=2 * elements * (4 if c["dtype"] == "f32" else 2), flops=6 * elements)
    esz = 1 if c["cache"] == "e4m3" else 2
    if c["kind"] == "append":
        per_seq = c["n"] if c["mode"] == "rows" else min(c["n"], 5)
        elements = c["batch"] * per_seq * c["kv_heads"] * c["head_dim"] * 2
        return dict(bytes=elements * ((4 if c["dtype"] == "f32" else 2) + esz) + c["batch"] * 16, flops=4 * elements)
    keys = c["n"] * c["tree"]
    rows = c["batch"] * c["q_heads"] * c["n"]
    kv = c["batch"] * c["kv_heads"] * (c["prefix"] * esz + keys * 2) * c["head_dim"] * 2
    return dict(bytes=kv + rows * c["head_dim"] * 4 + c["batch"] * c["n"] * keys / 8, flops=4 * rows * c["prefix"] * c["head_dim"])


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _e4m3_table():
    """The values of the 256 bytes, from the format's definition: 4 exponent bits with bias 7, 3 mantissa bits."""
    b = torch.arange(256, dtype=torch.int32)
    e, m = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2((e - 7).double()))
    mag = torch.where((e == 15) & (m == 7), torch.full_like(mag, float("nan")), mag)
    return torch.where(b >= 128, -mag, mag).to(DEV)


def _inverse_frequencies(rotary):
    return 500000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device=DEV) / rotary)


def _lengths(c, gen):
    """Rows that each sequence has in the cache."""
    u = torch.rand(c["batch"], generator=gen, dtype=torch.float64, device=DEV) * 2 - 1
    return torch.round(c["prefix"] * (1 + c["ragged"] * u)).to(torch.int32)


def _heads(c, gen, heads, dtype):
    """Projections of new tokens [batch, heads, n, head_dim]: a few loud channels, as keys and queries have them."""
    D = c["head_dim"]
    shape = (c["batch"], c["n"], heads, D) if c.get("token_major") else (c["batch"], heads, c["n"], D)
    loud = torch.exp(0.5 * torch.randn(heads, D, generator=gen, device=DEV))
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= loud if c.get("token_major") else loud[:, None]
    x = x.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    return x.transpose(1, 2) if c.get("token_major") else x


def _pages(c, gen, count):
    """A pool of `count` pages: what earlier appends have left there, garbage behind a sequence's last row included."""
    shape = (count, c["kv_heads"], c["page"], c["head_dim"])
    if c["cache"] == "bf16":
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16), None
    # values between 2^-6 and 448 of either sign, largest most often near 1/4 of the range, as quantised keys are
    data = (torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16) * 90).clamp_(-E4M3_MAX, E4M3_MAX)
    exponent = torch.randint(118, 121, shape[:2], generator=gen, device=DEV, dtype=torch.int32).to(torch.uint8)
    return data.to(torch.float8_e4m3fn).view(torch.uint8), exponent


def _cache(c, gen, rows_most):
    """Pages scattered over a pool, some of them nobody's: (k, v, k_exp, v_exp, table [batch, pages of the longest])."""
    per_seq = max(1, -(-rows_most // c["page"]))
    used = c["batch"] * per_seq
    count = used + 3
    order = torch.randperm(count, generator=gen, device=DEV, dtype=torch.int32)
    table = order[:used].view(c["batch"], per_seq).contiguous()
    k, k_exp = _pages(c, gen, count)
    v, v_exp = _pages(c, gen, count)
    return k, v, k_exp, v_exp, table


def _tree_mask(c, seed):
    """Ancestor masks [batch, n, words]: `tree` layers of n keys, a query in the last one, a parent drawn for every node
    (one layer: a tree in parents-first order, as the tree builder numbers it)."""
    n, layers = c["n"], c["tree"]
    g = np.random.default_rng(seed)
    words = (n * layers + 63) // 64
    bits = np.zeros((c["batch"], n, words * 64), dtype=np.uint8)
    for b in range(c["batch"]):
        if layers == 1:
            for i in range(n):
                p = int(g.integers(-1, i)) if i else -1
                if p >= 0:
                    bits[b, i] = bits[b, p]
                bits[b, i, i] = 1
        else:
            slot = np.arange(n)
            for t in range(layers - 1, -1, -1):
                bits[b, np.arange(n), t * n + slot] = 1
                slot = g.integers(0, n, n)[slot]
    packed = np.packbits(bits, axis=-1, bitorder="little").view(np.int64)
    return torch.from_numpy(packed.copy()).to(DEV)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(c=c)
    if c["kind"] == "rope":
        s["Q"], s["K"] = _heads(c, gen, c["q_heads"], c["dtype"]), _heads(c, gen, c["kv_heads"], c["dtype"])
        t = s["Q"].dtype
        s["q_weight"] = s["k_weight"] = None
        if c["norm"]:
            s["q_weight"] = (1 + 0.2 * torch.randn(c["head_dim"], generator=gen, device=DEV)).to(t)
            s["k_weight"] = (1 + 0.2 * torch.randn(c["head_dim"], generator=gen, device=DEV)).to(t)
        s["inv_freq"] = _inverse_frequencies(c["rotary"])
        s["first"] = torch.randint(c["first"] // 2, c["first"] + 1, (c["batch"],), generator=gen, device=DEV, dtype=torch.int32)
        s["offset"], s["shift"] = None, 0
        if c["tree"]:       # depths of the nodes, the root being the last row of the cache
            s["offset"] = torch.randint(1, 11, (c["batch"], c["n"]), generator=gen, device=DEV, dtype=torch.int32).sort(1)[0].contiguous()
            s["shift"] = -1
        return s
    lengths = _lengths(c, gen)
    if c["kind"] == "append":
        s["K"], s["V"] = _heads(c, gen, c["kv_heads"], c["dtype"]), _heads(c, gen, c["kv_heads"], c["dtype"])
        most = int(c["prefix"] * (1 + c["ragged"]) + 1 + c["n"])
        s["rows"] = None
        if c["mode"] == "branch":      # what verification leaves: tokens produced, and the accepted nodes root side first
            depth = min(c["n"], 10)
            s["count"] = torch.randint(1, depth + 1, (c["batch"],), generator=gen, device=DEV, dtype=torch.int32)
            pick = torch.rand(c["batch"], c["n"], generator=gen, device=DEV).argsort(1)[:, :depth].sort(1)[0].to(torch.int32)
            s["rows"] = torch.full((c["batch"], c["n"]), -1, device=DEV, dtype=torch.int32)
            kept = torch.arange(depth, device=DEV)[None] < s["count"][:, None] - 1
            s["rows"][:, :depth] = torch.where(kept, pick, s["rows"][:, :depth])
            s["count_shift"] = -1
        else:
            s["count"], s["count_shift"] = None, 0
            if c["n"] > 1:             # padded prompts of unequal length
                s["count"] = torch.randint(max(1, c["n"] * 3 // 4), c["n"] + 1, (c["batch"],), generator=gen, device=DEV, dtype=torch.int32)
        s["inv_freq"] = _inverse_frequencies(c["rotary"]) if c["rotary"] else None
    else:
        most = int(c["prefix"] * (1 + c["ragged"]) + 1)
        n, D = c["n"], c["head_dim"]
        s["Q"] = torch.randn(c["batch"], c["q_heads"], n, D, generator=gen, device=DEV).to(torch.bfloat16)
        s["K_tree"] = s["V_tree"] = s["mask"] = None
        if c["tree"]:
            shape = (c["batch"], c["kv_heads"], n * c["tree"], D)
            s["K_tree"] = torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)
            s["V_tree"] = torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)
            s["mask"] = _tree_mask(c, seed)
    s["lengths"] = lengths
    s["k"], s["v"], s["k_exp"], s["v_exp"], s["table"] = _cache(c, gen, most)
    return s


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2406_17276_amd import api
    c = s["c"]
    if c["kind"] == "rope":
        return api.qk_norm_rope(s["Q"], s["K"], s["first"], s["inv_freq"], offset=s["offset"], shift=s["shift"], q_weight=s["q_weight"],
                                k_weight=s["k_weight"], eps=1e-6, interleaved=c["interleaved"])
    if "cache" not in s:               # the decoder's cache object, and the workspace it keeps
        s["cache"] = api.PagedCache(s["k"], s["v"], s["table"], s["k_exp"], s["v_exp"])
        if c["kind"] == "attn":
            s["workspace"] = api.paged_attn_workspace(s["Q"], s["cache"], s["K_tree"])
    if c["kind"] == "append":
        new = api.kv_append_paged(s["cache"], s["K"], s["V"], s["lengths"], count=s["count"], count_shift=s["count_shift"],
                                  rows=s["rows"], inv_freq=s["inv_freq"], interleaved=c["interleaved"])
        return _appended(s, new)
    return api.tree_verify_attention_paged(s["Q"], s["cache"], s["lengths"], s["K_tree"], s["V_tree"], s["mask"],
                                           workspace=s["workspace"])


def _appended(s, new_lengths):
    """The updated state; bytes of an 8-bit pool as the E4M3 numbers that they are, beside their exponents."""
    if s["k_exp"] is None:
        return new_lengths, s["k"], s["v"]
    return new_lengths, s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["k_exp"], s["v_exp"]


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _rotate(x, positions, inv_freq, interleaved):
    """x float32 [batch, heads, n, D], positions [batch, n]: the first 2 len(inv_freq) columns rotated."""
    angle = positions.double()[:, None, :, None] * inv_freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    half = inv_freq.numel()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_rope(s):
    c = s["c"]
    steps = s["offset"] if s["offset"] is not None else torch.arange(c["n"], device=DEV, dtype=torch.int32)[None]
    positions = s["first"][:, None] + steps + s["shift"]
    out = []
    for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        out.append(_rotate(y, positions, s["inv_freq"], c["interleaved"]).to(x.dtype))
    return tuple(out)


def _power(exponent):
    """2^(e - 127) of exponent bytes, as float32."""
    return (exponent.to(torch.int32) << 23).view(torch.float32)


def _plain_append(s):
    c = s["c"]
    B, H, n, D, ps = c["batch"], c["kv_heads"], c["n"], c["head_dim"], c["page"]
    table, lengths = s["table"].long(), s["lengths"].long()
    capacity = table.shape[1] * ps
    count = torch.full_like(lengths, n) if s["count"] is None else (s["count"].long() + s["count_shift"]).clamp(0, n)
    new = torch.minimum(lengths + count, torch.full_like(lengths, capacity))
    # the pages that an append may touch: slots of the page grid from the one that holds row `length` on
    slots = min(-(-(n + ps - 1) // ps), table.shape[1])
    first = torch.minimum(lengths // ps, torch.full_like(lengths, table.shape[1] - slots))
    slot = first[:, None] + torch.arange(slots, device=DEV)
    ids = table.gather(1, slot)
    position = (slot[:, :, None] * ps + torch.arange(ps, device=DEV)).view(B, -1)              # of every row of these pages
    fresh = (position >= lengths[:, None]) & (position < new[:, None])
    step = (position - lengths[:, None]).clamp(0, n - 1)
    source = step if s["rows"] is None else s["rows"].long().gather(1, step).clamp(0, n - 1)
    fresh = fresh.view(B, slots, 1, ps, 1)
    for name, x in (("k", s["K"]), ("v", s["V"])):
        rows = x.float().gather(2, source[:, None, :, None].expand(B, H, slots * ps, D))
        if name == "k" and s["inv_freq"] is not None:
            rows = _rotate(rows, position, s["inv_freq"], c["interleaved"])
        rows = rows.view(B, H, slots, ps, D).transpose(1, 2)
        pages = s[name]
        old = pages[ids]
        if c["cache"] == "bf16":
            pages[ids] = torch.where(fresh, rows.to(torch.bfloat16), old)
            continue
        exps = s[name + "_exp"]
        e_old = exps[ids].to(torch.int32)
        touched = fresh.any(3).view(B, slots, 1)
        top = torch.where(fresh, rows.abs(), torch.zeros_like(rows)).amax((-1, -2))
        # smallest power of two that brings the largest magnitude to 448 or below
        mantissa, power = torch.frexp(top)
        e_new = (power + 118 + (mantissa > 0.875).int()).clamp(1, 254)       # 448 = 0.875 * 2^9
        e_new = torch.where(top == 0, torch.ones_like(e_new), e_new)
        older = ((slot * ps) < lengths[:, None])[:, :, None]
        e = torch.where(touched, torch.where(older, torch.maximum(e_old, e_new), e_new), e_old)
        kept = (position < lengths[:, None]).view(B, slots, 1, ps, 1)
        again = (old.view(torch.float8_e4m3fn).float() * torch.exp2((e_old - e).float())[..., None, None]).to(torch.float8_e4m3fn)
        quantised = (rows * _power(254 - e)[..., None, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        data = torch.where(fresh, quantised.view(torch.uint8), torch.where(kept & touched[..., None, None], again.view(torch.uint8), old))
        pages[ids] = data
        exps[ids] = e.to(torch.uint8)
    return _appended(s, new.to(torch.int32))


def _gathered(s, name):
    """The cache of every sequence as float32 [batch, heads, rows, D]."""
    table = s["table"].long()
    pages = s[name][table]                                       # [batch, pages, heads, page, D]
    if s["k_exp"] is not None:
        x = pages.view(torch.float8_e4m3fn).float() * _power(s[name + "_exp"][table])[..., None, None]
    else:
        x = pages.float()
    B, P, H, ps, D = x.shape
    return x.transpose(1, 2).reshape(B, H, P * ps, D)


def _plain_attn(s):
    c = s["c"]
    B, Hq, Hkv, n, D = c["batch"], c["q_heads"], c["kv_heads"], c["n"], c["head_dim"]
    g = Hq // Hkv
    q = (s["Q"].float() / math.sqrt(D)).reshape(B, Hkv, g * n, D)
    k = _gathered(s, "k")
    seen = (torch.arange(k.shape[2], device=DEV) < s["lengths"][:, None])[:, None, None, :]
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(B, Hq, n, -1)
    del k
    scores.masked_fill_(~seen, float("-inf"))
    if c["tree"]:
        keys = s["K_tree"].shape[2]
        at = torch.arange(keys, device=DEV)
        seen = ((s["mask"][..., at // 64] >> (at % 64)) & 1).bool()[:, None]
        tree = torch.matmul(q, s["K_tree"].float().transpose(-1, -2).contiguous()).view(B, Hq, n, keys)
        scores = torch.cat((scores, tree.masked_fill_(~seen, float("-inf"))), -1)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.view(B, Hkv, g * n, -1)
    v = _gathered(s, "v")
    rows = v.shape[2]
    v.masked_fill_((torch.arange(rows, device=DEV) >= s["lengths"][:, None])[:, None, :, None], 0)
    out = torch.matmul(p[..., :rows].contiguous(), v)
    if c["tree"]:
        out += torch.matmul(p[..., rows:].contiguous(), s["V_tree"].float())
    out = out.view(B, Hq, n, D)
    return torch.where(total > 0, out / total, torch.zeros_like(out)).to(torch.bfloat16)


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn}[state["c"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turned(x, pos, inv_freq, interleaved):
    """Rows of one sequence, float64 [heads, n, D], turned as complex numbers."""
    half = inv_freq.numel()
    pair = x[..., :2 * half].reshape(*x.shape[:-1], half, 2) if interleaved else torch.stack((x[..., :half], x[..., half:2 * half]), -1)
    z = torch.view_as_complex(pair.contiguous()) * torch.polar(torch.ones(pos.numel(), half, dtype=torch.float64, device=DEV),
                                                               pos.double()[:, None] * inv_freq)
    z = torch.view_as_real(z)
    y = x.clone()
    y[..., :2 * half] = z.flatten(-2) if interleaved else torch.cat((z[..., 0], z[..., 1]), -1)
    return y


def _to_e4m3(x):
    """float64 -> the nearest E4M3 value, ties to the even one, as float64."""
    size = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -30))).clamp(min=-6)
    step = torch.exp2(size - 3)
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_rope(s):
    c = s["c"]
    out = []
    for x, w in ((s["Q"], s["q_weight"]), (s["K"], s["k_weight"])):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["head_dim"] + 1e-6) * w.double()
        for b in range(c["batch"]):
            at = torch.arange(c["n"], device=DEV) if s["offset"] is None else s["offset"][b].long()
            y[b] = _turned(y[b], int(s["first"][b]) + at + s["shift"], s["inv_freq"], c["interleaved"])
        out.append(y)
    return tuple(out)


def _exact_append(s):
    c = s["c"]
    ps, eight = c["page"], c["cache"] == "e4m3"
    values = _e4m3_table()
    pools = {m: values[s[m].long()] if eight else s[m].double() for m in "kv"}
    for b in range(c["batch"]):
        length = int(s["lengths"][b])
        count = c["n"] if s["count"] is None else max(0, min(c["n"], int(s["count"][b]) + s["count_shift"]))
        count = min(count, s["table"].shape[1] * ps - length)
        if count <= 0:
            continue
        source = torch.arange(count, device=DEV) if s["rows"] is None else s["rows"][b, :count].long()
        ids = s["table"][b].tolist()
        for m, x in (("k", s["K"]), ("v", s["V"])):
            y = x[b][:, source].double()
            if m == "k" and s["inv_freq"] is not None:
                y = _turned(y, length + torch.arange(count, device=DEV), s["inv_freq"], c["interleaved"])
            for page in range(length // ps, (length + count - 1) // ps + 1):
                lo, hi = max(length, page * ps), min(length + count, page * ps + ps)
                rows, pool = y[:, lo - length:hi - length], pools[m][ids[page]]
                at = slice(lo - page * ps, hi - page * ps)
                if not eight:
                    pool[:, at] = rows
                    continue
                old = s[m + "_exp"][ids[page]].double() - 127
                e = torch.ceil(torch.log2(rows.abs().amax((1, 2)) / E4M3_MAX)).clamp(min=-126)
                if lo > page * ps:
                    e = torch.maximum(e, old)
                    kept = slice(0, lo - page * ps)
                    pool[:, kept] = _to_e4m3(pool[:, kept] * torch.exp2(old - e)[:, None, None])
                pool[:, at] = _to_e4m3(rows / torch.exp2(e)[:, None, None])
    return (None, pools["k"], pools["v"], None, None) if eight else (None, pools["k"], pools["v"])


def _exact_attn(s):
    c = s["c"]
    values = _e4m3_table()
    g, ps, D = c["q_heads"] // c["kv_heads"], c["page"], c["head_dim"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        length = int(s["lengths"][b])
        ids = s["table"][b, :-(-length // ps)].long()
        for h in range(c["kv_heads"]):
            kv = []
            for m in "kv":
                x = s[m][ids, h]
                if s["k_exp"] is not None:
                    x = values[x.long()] * torch.exp2(s[m + "_exp"][ids, h].double() - 127)[:, None, None]
                x = x.double().reshape(-1, D)[:length]
                kv.append(torch.cat((x, s["K_tree" if m == "k" else "V_tree"][b, h].double())) if c["tree"] else x)
            z = s["Q"][b, h * g:(h + 1) * g].double() @ kv[0].T / math.sqrt(D)
            if c["tree"]:
                at = torch.arange(s["K_tree"].shape[2], device=DEV)
                z[..., length:][:, ((s["mask"][b][:, at // 64] >> (at % 64)) & 1) == 0] = float("-inf")
            w = torch.softmax(z, -1)
            out[b, h * g:(h + 1) * g] = torch.nan_to_num(w, nan=0.0) @ kv[1]
    return out


def exact(case, seed):
    return {"rope": _exact_rope, "append": _exact_append, "attn": _exact_attn}[case["kind"]](prepare(case, seed))
