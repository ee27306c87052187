"""Prefills of a few long chunks among many short and empty ones: workgroups for the tiles that there are, not for every sequence's longest chunk."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paged
    from paged import Paged, run

FORMS = [("fp16", 128, 32, 8), ("bf16", 64, 12, 4), ("fp16", 256, 12, 3), ("fp32", 64, 8, 8), ("bf16", 128, 7, 1)]


def _chunks(seed, batch, longest):
    """Lengths and chunks: `longest` once at the front, once near the end, nothing or little elsewhere."""
    g = torch.Generator().manual_seed(seed)
    new = torch.randint(0, 4, (batch,), generator=g).tolist()
    old = torch.randint(0, 30, (batch,), generator=g).tolist()
    new[1], new[batch - 2], new[batch // 2] = longest, longest - 37, longest // 3
    return [a + b for a, b in zip(old, new)], new


@pytest.mark.parametrize("dtype,d,heads,kv_heads", FORMS)
def test_mixed_chunks(dtype, d, heads, kv_heads):
    """The longest chunk has 11 to 15 tiles of 128 rows (fp32: 27 of 16); so many for every sequence are more than 8 (2) times the room that all tokens want,
    and enough that no tile's keys are cut into parts."""
    batch = 100 if kv_heads > 2 else 200
    lens, new = _chunks(3, batch, {1: 420, 3: 560, 4: 420, 7: 260}[heads // kv_heads])
    run(Paged(111, lens, new, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, page=32, scores=True, extra_rows=5))
    run(Paged(112, lens, new, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, page=32, window=90, sink=3, max_pages=40, missing=[(1, 2), (1, 7)]))


def test_mixed_chunks_of_many_sequences():
    """More sequences than a wave looks through at once, most of them without a token, in front of, between and behind those with some."""
    lens, new = [0] * 4300, [0] * 4300
    for b, n in ((5, 300), (63, 1), (64, 2), (65, 40), (2000, 130), (4095, 7), (4096, 300), (4290, 3)):
        lens[b], new[b] = n + b % 20, n
    run(Paged(113, lens, new, heads=8, kv_heads=1, d=64, dtype="bf16", max_pages=20, scores=True))
    run(Paged(114, lens, new, heads=2, kv_heads=2, d=64, dtype="fp32", max_pages=20))


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_mixed_starts_that_do_not_fit(dtype):
    """Chunks longer than max_new and than their sequence; rows before the first and behind the last chunk are left as they are."""
    lens, new = _chunks(5, 80, 500)
    p = Paged(115, lens, new, heads=32, kv_heads=8, d=64, dtype=dtype, page=32, extra_rows=30)
    x = p.device()
    most = 450                                               # the two longest are cut to it
    x["starts"].add_(11)                                     # eleven rows belong to nobody
    p.starts = [s + 11 for s in p.starts]
    p.new = [min(n, most) for n in new]
    short = next(b for b in range(80) if p.new[b] == 3)
    p.lens[short] = 1                                        # two of its tokens have no slot
    x["lens"].copy_(torch.tensor(p.lens, dtype=torch.int32))
    x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], most)
    torch.cuda.synchronize()
    paged.check(p, x)
