"""The sizes at which the paged cache's calls have to be refused, or not: host-side, with made-up addresses, nothing is launched."""
import pytest

from paper_2503_01330_amd import binding as wkv
from test_paged_boundary import cache, evict


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
