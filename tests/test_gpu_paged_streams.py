"""PagedCache's calls on a stream that is not the current one: their workspace is theirs until they have run."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paged
    from paged import Paged
    from paper_2503_01330_amd import binding as wkv


def _cases():
    yield Paged(101, [3000, 130], heads=8, kv_heads=2, page=64, scores=True)                     # parts, logits and sums in the workspace
    yield Paged(102, [1500, 130], [70, 60], heads=8, kv_heads=2, page=64, scores=True)           # (and a workspace that grows with the call)


@pytest.mark.parametrize("which", [0, 1])
def test_a_call_on_another_stream_whose_object_is_dropped(which):
    """The stream is still busy when the call returns; what the current stream takes and fills meanwhile is not the workspace."""
    p = list(_cases())[which]
    x = p.device()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(40):
            big = (big @ big).clamp_(-1, 1)                  # some milliseconds of work before the call's turn comes
    c = x.pop("cache")
    if p.step:
        c.step(x["q"], x["k_new"], x["v_new"], x["out"], stream=side.cuda_stream)
    else:
        c.prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], max(p.new), stream=side.cuda_stream)
    size = c._bytes
    del c
    other = [torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    paged.check(p, x)
    del other


def test_one_object_on_several_streams_in_turn():
    p = Paged(103, [1500, 40], heads=8, kv_heads=2, page=64, scores=True, max_pages=40)
    x, y = p.device(), p.device()
    streams = [torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.default_stream()]
    for t in range(8):
        s = streams[t % 4]
        torch.cuda.synchronize()
        x["cache"].step(x["q"], x["k_new"], x["v_new"], x["out"], stream=s.cuda_stream)
        if t == 5:
            x["cache"].evict(900, 10, x["lens"], x["scores"], stream=s.cuda_stream)
        torch.cuda.synchronize()
        y["cache"].step(y["q"], y["k_new"], y["v_new"], y["out"])
        if t == 5:
            y["cache"].evict(900, 10, y["lens"], y["scores"])
        torch.cuda.synchronize()
        for n in ("out", "k", "v", "scores", "lens"):
            assert paged.same(x[n].cpu(), y[n].cpu()), (t, n)
        for z in (x, y):
            z["lens"].add_(1)


def test_no_workspace_is_taken_while_a_graph_is_recorded():
    """A recorded call that would want a larger workspace is refused, on the stream that is recorded and from beside it; calls of sizes that are
    there already are recorded."""
    p = Paged(104, [1500, 130], [70, 60], heads=8, kv_heads=2, page=64, scores=True)
    x = p.device()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(wkv.WkvError, match="recorded"):
            x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 70)
        with pytest.raises(wkv.WkvError, match="recorded"):
            wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 8, scores=x["scores"])
        x["out"].add_(0)
    cache = wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 8, scores=x["scores"], max_tokens=130, max_new=70)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cache.prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 70)
    old = p.scores.cuda()
    for _ in range(3):
        x["scores"].copy_(old)
        x["out"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        paged.check(p, x)
