"""Which strides the paged-cache operators take for what they write, without a GPU (nothing is launched): rows that lie over one
another are refused, every layout that slicing and transposing a tensor gives is taken."""
import ctypes as C
import itertools

import pytest

from paper_2406_17276_amd import api
from tests.test_paged import F, _ap, _cache, _pp, _qk, s3

FAR = C.c_void_p(0x900000)
# of (batch, head, row) for 3 sequences x 4 heads x 3 rows of 64; each has an axis that does not step over what the smaller ones span
OVERLAPPING = [(768, 8, 64), (768, 192, 56), (768, 184, 64), (760, 192, 64), (64, 192, 64), (64, 128, 512), (8, 8, 8), (768, 64, 248),
               (192, 384, 64), (1 << 62, 1 << 62, 1 << 62)]
APART = [(768, 192, 64), (768, 64, 256), (192, 576, 64), (64, 192, 768), (1536, 192, 64), (776, 192, 64), (4096, 72, 1024), (1 << 60, 192, 64)]


@pytest.mark.parametrize("strides", OVERLAPPING)
def test_overlapping_rows_are_not_written(strides):
    L = api.lib()
    for name in ("qo_strides", "ko_strides"):
        p = _qk(batch=3, n=3, q_heads=4, kv_heads=4, **{name: s3(*strides)})
        assert L.ot_qk_norm_rope(C.byref(p), *([F] * 9), None) == -1, name
    p = _pp(batch=3, n=3, q_heads=4, o_strides=s3(*strides))
    assert L.ot_paged_attn_workspace_bytes(C.byref(p), C.byref(_cache())) == 0
    assert L.ot_tree_verify_attention_paged(C.byref(p), C.byref(_cache()), *([F] * 7), 1 << 30, None) == -1


@pytest.mark.parametrize("strides", APART)
def test_rows_apart_are_taken_in_every_order(strides):
    p = _pp(batch=3, n=3, q_heads=4, o_strides=s3(*strides))
    assert api.lib().ot_paged_attn_workspace_bytes(C.byref(p), C.byref(_cache())) > 0


def test_layouts_of_tensors_are_taken():
    """Slices, steps, selections and diagonals of a tensor, transposed every way."""
    import torch
    t = torch.empty(6, 5, 4, 128)
    views = [t, t[1:], t[:, ::2], t[:, :, 1:3], t[..., 64:], t.view(6, 5, 2, 2, 128).select(3, 1), torch.empty(6, 5, 4, 3, 128)[:, :, :, 2],
             torch.empty(5, 6, 4, 7, 128).diagonal(0, 0, 1).permute(3, 0, 1, 2), t[:, :1], t[None, 2]]
    for v in views:
        for order in itertools.permutations(range(3)):
            x = v.permute(*order, 3)[..., :64]
            p = _pp(batch=x.shape[0], q_heads=x.shape[1], n=x.shape[2], o_strides=s3(*x.stride()[:3]))
            assert api.lib().ot_paged_attn_workspace_bytes(C.byref(p), C.byref(_cache(kv_heads=1))) > 0, (x.shape, x.stride())
    one = _pp(batch=1, q_heads=2, n=1, o_strides=s3(8, 64, 16))             # axes of one row say nothing
    assert api.lib().ot_paged_attn_workspace_bytes(C.byref(one), C.byref(_cache())) > 0


@pytest.mark.parametrize("pool", [(2048, 1024, 72), (2032, 1024, 64), (2048, 64, 64), (64, 1024, 64), (1024, 1024, 64), (2048, 512, 64), (2048, 48, 128)])
@pytest.mark.parametrize("name", ["k_strides", "v_strides"])
@pytest.mark.parametrize("dtype", [api.OT_BF16, api.OT_E4M3])
def test_overlapping_pages_are_read_but_not_written(dtype, name, pool):
    L = api.lib()
    if pool[2] == 72 and dtype == api.OT_E4M3:
        pool = (2048, 1024, 80)
    c = _cache(dtype=dtype, v_pages=0x100000, v_exp=0x2000, **{name: s3(*pool)})
    assert L.ot_kv_append_paged(C.byref(_ap()), C.byref(c), F, F, F, F, F, F, FAR, None) == -1
    assert L.ot_paged_attn_workspace_bytes(C.byref(_pp()), C.byref(c)) > 0


def test_two_outputs_at_one_address_are_not_written():
    """Pointers that no GPU has: a call that is not refused fails at its launch (no GPU) with another status."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch if it were not refused")
    L = api.lib()
    apart = dict(v_pages=0x100000, v_exp=0x2000)
    call = lambda c: L.ot_kv_append_paged(C.byref(_ap()), C.byref(c), F, F, F, F, F, F, FAR, None)
    assert call(_cache(**apart)) == -4                                      # nothing wrong with it but the missing GPU
    assert call(_cache(v_exp=0x2000)) == -1 and call(_cache(v_pages=0x100000)) == -1
    assert call(_cache(**{**apart, "dtype": api.OT_BF16, "v_exp": 0x1000})) == -4        # exponents that are not used
    qk = lambda q, k, **kw: L.ot_qk_norm_rope(C.byref(_qk(**kw)), F, F, F, F, F, F, F, C.c_void_p(q), C.c_void_p(k), None)
    assert qk(0x10000, 0x10000) == -1 and qk(0x10000, 0x20000) == -4
    assert qk(0x10000, 0x10000, kv_heads=0) == -4 and qk(0x10000, 0x10000, q_heads=0) == -4
