"""What the paged cache's calls report: their own launches' errors, not those of the program's calls before."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paged
    from paged import Paged
    from paper_2503_01330_amd import binding as wkv


@pytest.fixture
def left_behind():
    """Leaves an error behind in the HIP runtime (a device that does not exist is asked for), and takes it away at the end."""
    hip = wkv._lib                                           # (the runtime that the library is linked to)
    yield lambda: hip.hipSetDevice(1 << 20)
    hip.hipGetLastError()


@pytest.mark.parametrize("lens,new,scores", [([2000, 30], None, False), ([2000, 30], None, True), ([90, 30], [80, 30], True), ([2000, 700], [300, 2], True)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_an_error_of_an_earlier_call_is_not_ours(left_behind, lens, new, scores, dtype):
    p = Paged(121, lens, new, heads=4, kv_heads=2, d=64, dtype=dtype, page=64, scores=scores)
    x = p.device()
    c = x["cache"] = wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 4, scores=x["scores"], max_tokens=p.rows, max_new=max(p.new))
    torch.cuda.synchronize()
    assert left_behind() != 0
    if p.step:
        c.step(x["q"], x["k_new"], x["v_new"], x["out"])
    else:
        c.prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], max(p.new))
    wkv._lib.hipGetLastError()
    torch.cuda.synchronize()
    paged.check(p, x)


def test_nor_an_evictions(left_behind):
    p = Paged(122, [200, 30], heads=2, kv_heads=2, d=64, scores=True)
    p.k, p.v = p.appended()
    x = p.device()
    torch.cuda.synchronize()
    assert left_behind() != 0
    x["cache"].evict(50, 5, x["lens"], x["scores"])
    wkv._lib.hipGetLastError()
    torch.cuda.synchronize()
    _, lens, scores, k, v = paged.evicted(p, 50, 5)
    assert x["lens"].tolist() == lens and paged.same(x["scores"].cpu(), scores) and paged.same(x["k"].cpu(), k) and paged.same(x["v"].cpu(), v)
