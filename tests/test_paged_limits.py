"""The sizes at which the paged cache's calls have to be refused, or not: host-side, with made-up addresses, nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2503_01330_amd import binding as wkv
from test_paged_boundary import cache, evict, prefill, rows


# Units whose moves make 2^32 threads, by their rows' bytes: (bytes / 32 + 1) x 1024 threads each, units in eights.
@pytest.mark.parametrize("head_dim,dtype,most", [(64, wkv.WKV_FP16, 838856), (128, wkv.WKV_FP16, 466032), (64, wkv.WKV_FP32, 466032),
                                                 (256, wkv.WKV_BF16, 246720), (128, wkv.WKV_FP32, 246720)])
def test_evictions_of_as_many_units_as_a_launch_holds(head_dim, dtype, most):
    def code(units):
        c = cache(batch=units, heads=1, kv_heads=1, head_dim=head_dim, dtype=dtype)
        return evict(c), wkv.wkv_last_error()
    assert code(most)[0] == wkv.WKV_ESIZE and "workspace" in code(most)[1]          # (sound but for its workspace of 0 bytes)
    for units in (most + 1, most + 2, most + 7, most + 8, most + 9, 1 << 22):
        assert code(units)[0] == wkv.WKV_ESIZE and "threads" in code(units)[1], units


# ---------------------------------------------------------------- prefills of one long chunk among many short ones
MIXED = [
    # batch, heads, kv_heads, dtype, head_dim, n_tokens, max_new: tokens that fit, though batch x the longest chunk would be too many workgroups
    (256, 32, 8, wkv.WKV_FP16, 128, 40000, 32768),
    (4096, 32, 8, wkv.WKV_BF16, 128, 40000, 32768),
    (1024, 8, 8, wkv.WKV_FP32, 64, 60000, 50000),
    (1 << 16, 8, 2, wkv.WKV_FP16, 64, 100000, 30000),
]


def taken(c, r, n, most):
    """Whether a call is refused for no other reason than that there is no GPU (where there is one, it is not made)."""
    code = prefill(c, r, n=n, most=most, size=1 << 62)
    return code == wkv.WKV_EHIP or (code, wkv.wkv_last_error())


without_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")


@without_gpu
@pytest.mark.parametrize("batch,heads,kv_heads,dtype,head_dim,n,most", MIXED)
def test_mixed_chunks_are_taken(batch, heads, kv_heads, dtype, head_dim, n, most):
    c = cache(batch=batch, heads=heads, kv_heads=kv_heads, dtype=dtype, head_dim=head_dim, page_size=256, max_pages=256, table_stride=256)
    assert taken(c, rows(out_stride=1 << 14), n, most) is True
    need = wkv._lib.wkv_paged_workspace_bytes(C.byref(c), n, most)
    assert need >= n * heads * 4
    # fewer tokens with the same longest chunk want no more
    assert most == n or wkv._lib.wkv_paged_workspace_bytes(C.byref(c), most, most) <= need


def test_no_workspace_for_prefills_that_are_refused():
    c = cache(batch=1 << 12, heads=1 << 10, kv_heads=1 << 10, max_pages=1 << 10, table_stride=1 << 10)
    r = rows(q_stride=1 << 17, k_stride=1 << 17, v_stride=1 << 17, out_stride=1 << 17)
    assert prefill(c, r, n=1 << 20, most=1 << 12, work=None) == wkv.WKV_ESIZE and "threads" in wkv.wkv_last_error()
    assert wkv._lib.wkv_paged_workspace_bytes(C.byref(c), 1 << 20, 1 << 12) == 0 and "threads" in wkv.wkv_last_error()
    assert wkv._lib.wkv_paged_workspace_bytes(C.byref(c), 0, 0) > 0


@without_gpu
def test_tiles_are_counted_as_they_are_launched():
    """Chunks of the same length, more than 2^24 tiles of 16 rows but not of 128, which the kernel for long chunks takes."""
    c = cache(batch=1 << 8, heads=64, kv_heads=64, max_pages=1 << 11, table_stride=1 << 11)
    r = rows(q_stride=1 << 13, k_stride=1 << 13, v_stride=1 << 13, out_stride=1 << 13)
    assert taken(c, r, 1 << 22, 1 << 14) is True
