"""The paged cache (wkv_paged_step, wkv_paged_prefill, wkv_paged_evict) against attention and eviction in 64 bits on the CPU."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paged
    from paged import Paged, run
    from paper_2503_01330_amd import binding as wkv

TYPES = [("fp32", 64), ("fp32", 128), ("fp16", 64), ("fp16", 128), ("fp16", 256), ("bf16", 64), ("bf16", 128), ("bf16", 256)]
LENS = [1, 0, 15, 16, 17, 31, 33, 64, 127, 129, 300]


# ---------------------------------------------------------------- one token
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (16, 1), (17, 1), (40, 2)])
def test_step(dtype, d, heads, kv_heads):
    run(Paged(1, LENS, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, scores=True))


@pytest.mark.parametrize("dtype,d", [("fp32", 128), ("fp16", 128), ("bf16", 64), ("bf16", 256)])
@pytest.mark.parametrize("window,sink", [(1, 0), (16, 4), (33, 0), (100, 7), (64, 33), (64, 300), (1000, 4)])
def test_step_with_a_window(dtype, d, window, sink):
    for scores in (False, True):
        run(Paged(2, LENS + [777], heads=6, kv_heads=2, d=d, dtype=dtype, window=window, sink=sink, scores=scores))


@pytest.mark.parametrize("layout", ["slots", "heads", "padded"])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_step_layouts_and_pages(layout, page):
    run(Paged(3, LENS, d=128, page=page, layout=layout, scores=True, score_slack=5))
    run(Paged(4, [5, 400], d=64, dtype="bf16", page=page, layout=layout, max_pages=40))


def test_step_long_sequences_are_split_and_joined():
    for dtype, d in (("fp16", 128), ("bf16", 64), ("fp32", 64)):
        run(Paged(5, [3000], heads=2, kv_heads=1, d=d, dtype=dtype, page=64, scores=True))
        run(Paged(6, [1, 2077, 130], heads=4, kv_heads=2, d=d, dtype=dtype, page=16, window=1500, sink=20, scores=True))


def test_step_without_rows_to_append():
    p = Paged(7, [40, 1, 200], scores=True)
    p.k, p.v = p.appended()
    run(p, append=False)


def test_step_pages_that_are_not_there():
    """Given back behind the window, or never given: nothing of them is seen; a new row without a page is dropped."""
    run(Paged(8, [200, 100, 48, 17], missing=[(0, 1), (0, 2), (1, 0), (2, 0), (2, 1), (2, 2), (3, 1)], scores=True))
    run(Paged(9, [400], window=64, sink=4, missing=[(0, i) for i in range(1, 20)], scores=True))


# ---------------------------------------------------------------- a chunk of tokens
CHUNKS = [([1, 7, 16, 17, 40], [1, 7, 16, 17, 40]), ([100, 5, 64, 200], [1, 0, 33, 60]), ([129, 300], [128, 129])]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (7, 1)])
def test_prefill(dtype, d, heads, kv_heads):
    for lens, new in CHUNKS:
        run(Paged(11, lens, new, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, scores=True, extra_rows=3))


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("fp16", 128), ("bf16", 64), ("bf16", 256)])
@pytest.mark.parametrize("window,sink", [(1, 0), (16, 4), (50, 0), (100, 7), (64, 40)])
def test_prefill_with_a_window(dtype, d, window, sink):
    for scores in (False, True):
        run(Paged(12, [300, 31, 260], [300, 31, 50], heads=4, kv_heads=2, d=d, dtype=dtype, window=window, sink=sink, scores=scores))


@pytest.mark.parametrize("layout", ["slots", "heads", "padded"])
@pytest.mark.parametrize("page", [16, 64])
def test_prefill_layouts_and_pages(layout, page):
    run(Paged(13, [200, 77], [150, 77], page=page, layout=layout, scores=True, score_slack=3))


def test_prefill_without_rows_to_append_and_missing_pages():
    p = Paged(14, [140, 100], [70, 100], scores=True)
    p.k, p.v = p.appended()
    run(p, append=False)
    run(Paged(15, [140, 100, 30], [70, 100, 5], missing=[(0, 0), (0, 5), (1, 6), (2, 0), (2, 1)], scores=True))


# ---------------------------------------------------------------- eviction
def _evict(p, budget, recent, in_place=False):
    x = p.device()
    new_lens = x["lens"] if in_place else torch.full_like(x["lens"], -5)
    new_scores = x["scores"] if in_place else x["scores"].clone()
    kept = torch.full((len(p.lens), p.kv_heads, budget), -9, dtype=torch.int32, device="cuda")
    x["cache"].evict(budget, recent, new_lens, new_scores, None if in_place else kept)
    torch.cuda.synchronize()
    want = paged.evicted(p, budget, recent)
    if not in_place:
        assert (kept.cpu().numpy() == want[0]).all()
    assert new_lens.tolist() == want[1]
    assert paged.same(new_scores.cpu(), want[2])
    assert paged.same(x["k"].cpu(), want[3]) and paged.same(x["v"].cpu(), want[4])


def _full(p):
    p.k, p.v = p.appended()
    return p


@pytest.mark.parametrize("dtype,d,layout", [("fp32", 64, "slots"), ("fp16", 128, "heads"), ("bf16", 256, "padded"), ("bf16", 64, "slots")])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(dtype, d, layout, in_place):
    for budget, recent, sink in ((1, 1, 0), (40, 7, 4), (64, 60, 4), (129, 1, 0), (500, 10, 0)):
        _evict(_full(Paged(21, LENS + [1100], kv_heads=3, heads=3, d=d, dtype=dtype, layout=layout, sink=sink, scores=True, score_slack=9)),
               budget, recent, in_place)


def test_evict_ties_and_numbers_that_are_none():
    """Equal scores: the oldest leave first.  NaN counts as +inf, -0 as 0, negative scores are ordered."""
    for sink, fill in ((0, None), (3, None), (0, "equal"), (2, "odd"), (0, "bits")):
        p = _full(Paged(22, [700, 64, 65, 2, 333], heads=2, kv_heads=2, d=64, scores=True, sink=sink))
        if fill is None:
            p.scores = (p.scores * 3).floor()
        elif fill == "equal":
            p.scores.fill_(0.25)
        elif fill == "odd":
            g = torch.Generator().manual_seed(1)
            odd = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, -1.5, 1e-42, -1e-42, 3e38])
            p.scores = odd[torch.randint(0, len(odd), p.scores.shape, generator=g)]
        else:                                                # differ in the last bits only
            p.scores = (p.scores * 0 + 1.0).view(torch.int32).add(torch.arange(p.scores.shape[2], dtype=torch.int32).flip(0) % 37).view(torch.float32)
        _evict(p, 64, 5)


def test_evict_leaves_sequences_that_miss_a_page():
    p = _full(Paged(23, [200, 200, 90, 16], scores=True, missing=[(1, 5), (2, 0)]))
    _evict(p, 50, 7)


def test_evict_long():
    p = Paged(24, [9000, 5], heads=1, kv_heads=1, d=64, page=128, scores=True)
    _evict(p, 4000, 100)


# ---------------------------------------------------------------- numbers that are none, and large ones
@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("fp16", 128), ("bf16", 64), ("bf16", 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_has_no_effect(dtype, d, bad):
    """Values and keys that are not finite, at slots that some rows of a tile see and others do not."""
    for window, sink in ((0, 0), (20, 3)):
        p = Paged(31, [90, 40], [60, 40], heads=4, kv_heads=2, d=d, dtype=dtype, window=window, sink=sink, scores=True)
        for row in (7, 20, 33, 59, 61, 99):
            p.v_new[row, row % 2, :: 7] = bad
        p.k_new[45, 0, 3] = bad
        run(p)
        p = Paged(32, [90, 40], heads=4, kv_heads=2, d=d, dtype=dtype, window=window, sink=sink)
        p.v_new[0, 0, 5] = bad
        p.k_new[1, 1, 5] = bad
        run(p)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_values_near_the_largest(dtype):
    """Outputs are means: finite wherever the values are."""
    for new in (None, [300]):
        p = Paged(33, [300], new, heads=2, kv_heads=1, d=64, dtype=dtype)
        p.q.mul_(0.01)
        largest = torch.finfo(p.v_new.dtype).max
        p.v_new[..., ::2] = largest
        p.v[:, :, :, ::2] = torch.where(torch.isnan(p.v[:, :, :, ::2]), p.v[:, :, :, ::2], largest)
        x = p.device()
        if new is None:
            x["cache"].step(x["q"], x["k_new"], x["v_new"], x["out"])
        else:
            x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 300)
        torch.cuda.synchronize()
        got = x["out"][..., ::2].double().cpu()
        # a mean of equal numbers: off by the weights' own roundings (2^-8 in bf16, and as derived there for the sums) and the output's
        assert torch.isfinite(got).all() and ((got / largest - 1).abs() <= 2 * paged.HALF_STEP[dtype] + 2 * 310 * paged.U).all()


@pytest.mark.parametrize("dtype,gain", [("fp16", 60.0), ("bf16", 300.0), ("fp32", 300.0)])
def test_sharp_attention(dtype, gain):
    """Logits of hundreds: one key takes nearly all of a row."""
    run(Paged(34, [300, 90], heads=4, kv_heads=2, d=64, dtype=dtype, gain=gain, scores=True))
    run(Paged(35, [300, 90], [300, 20], heads=4, kv_heads=2, d=64, dtype=dtype, gain=gain, scores=True))


def test_logits_of_minus_infinity():
    """A row whose visible logits are all -inf is one that sees nothing."""
    p = Paged(36, [40], heads=2, kv_heads=1, d=64, dtype="fp32", scores=True)
    p.q = p.q.abs()
    p.k[~torch.isnan(p.k)] = -3e38
    p.k_new.fill_(-3e38)
    p.q.mul_(1e3)
    x = p.device()
    x["cache"].step(x["q"], x["k_new"], x["v_new"], x["out"])
    torch.cuda.synchronize()
    assert not x["out"].any() and torch.equal(x["scores"].cpu()[..., :39], p.scores[..., :39]) and not x["scores"][0, 0, 39]


# ---------------------------------------------------------------- how calls come
def test_calls_on_a_stream_and_in_a_graph():
    """A step, a prefill and an eviction recorded once and replayed, lengths and rows changed in between; every replay against the
    same calls made directly."""
    def make():
        p = Paged(41, [150, 40, 0, 97], heads=4, kv_heads=2, d=64, dtype="bf16", scores=True, max_pages=12)
        x = p.device()
        x["new_lens"], x["new_scores"] = torch.zeros_like(x["lens"]), torch.zeros_like(x["scores"])
        return p, x
    p, x = make()
    _, y = make()
    g = torch.Generator().manual_seed(3)

    def calls(z):
        z["cache"].step(z["q"], z["k_new"], z["v_new"], z["out"])
        z["cache"].evict(90, 10, z["lens"], z["scores"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    before = {n: x[n].clone() for n in ("k", "v", "scores", "lens", "out")}
    with torch.cuda.stream(s):
        calls(x)                                             # warm, then put back
        torch.cuda.synchronize()
        for n, t in before.items():
            x[n].copy_(t)
        with torch.cuda.graph(graph, stream=s):
            calls(x)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        calls(y)
        torch.cuda.synchronize()
        for n in ("k", "v", "scores", "lens", "out"):
            assert paged.same(x[n].cpu(), y[n].cpu()), n
        for z in (x, y):
            z["lens"].add_(torch.tensor([1, 1, 0, 1], dtype=torch.int32, device="cuda"))
        new = torch.randn(p.q.shape, generator=g).to(p.q.dtype)
        for z in (x, y):
            z["q"].copy_(new)
    with torch.cuda.stream(s):
        run(Paged(42, [100, 7], heads=4, kv_heads=2, scores=True))
        run(Paged(43, [100, 7], [50, 7], heads=4, kv_heads=2, scores=True))


def test_prefill_in_a_graph():
    p = Paged(44, [150, 40], [100, 40], heads=4, kv_heads=2, scores=True)
    x = p.device()
    old = x["scores"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 100)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 100)
    for _ in range(3):
        x["scores"].copy_(old)
        x["out"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        paged.check(p, x)


def test_generation_from_prompt_to_eviction():
    """As a program uses them together: prompts, steps whose weights are kept, an eviction, steps on what is left; against the same
    kept in 64 bits."""
    B, kvh, group, d, page, budget, recent = 3, 2, 2, 64, 16, 48, 8
    heads, g = kvh * group, torch.Generator().manual_seed(7)
    lens = [37, 60, 5]
    width, pages = 8, 8 * B
    k, v = (torch.full((pages, page, kvh, d), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.randperm(pages, generator=g).to(torch.int32).reshape(B, width).cuda()
    tl, scores = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.full((B, kvh, width * page), 99.0, device="cuda")
    cache = wkv.PagedCache(k, v, table, tl, heads, n_sink=2, scores=scores, max_tokens=sum(lens), max_new=max(lens))
    made = lambda n, h: torch.randn(n, h, d, generator=g).half()  # noqa: E731
    K = [[torch.zeros(0, d).double() for _ in range(kvh)] for _ in range(B)]
    V = [[torch.zeros(0, d).double() for _ in range(kvh)] for _ in range(B)]
    A = [[torch.zeros(0).double() for _ in range(kvh)] for _ in range(B)]

    def one(b, q, kn, vn):
        out = torch.zeros(heads, d).double()
        for h in range(kvh):
            K[b][h], V[b][h] = torch.cat([K[b][h], kn[h: h + 1].double()]), torch.cat([V[b][h], vn[h: h + 1].double()])
            A[b][h] = torch.cat([A[b][h], torch.zeros(1).double()])
            for i in range(group):
                w = torch.softmax(K[b][h] @ q[h * group + i].double() / d ** 0.5, 0)
                out[h * group + i] = w @ V[b][h]
                A[b][h] += w
        return out

    def near(got, want):
        # fp16 output and, for a chunk, fp16 weights; logits below 8 from 64 products in fp32
        assert ((got.double().cpu() - want).abs() <= 2 * 2.0 ** -11 * 4 + 1e-4).all()

    n = sum(lens)
    q, kn, vn = made(n, heads), made(n, kvh), made(n, kvh)
    out, starts = torch.empty(n, heads, d, dtype=torch.float16, device="cuda"), torch.tensor([0, 37, 97, 102], dtype=torch.int32, device="cuda")
    cache.prefill(q.cuda(), kn.cuda(), vn.cuda(), out, starts, max(lens))
    want = torch.stack([one(b, q[r], kn[r], vn[r]) for b in range(B) for r in range(int(starts[b]), int(starts[b + 1]))])
    near(out, want)
    out = torch.empty(B, heads, d, dtype=torch.float16, device="cuda")
    for t in range(40):
        if t in (20, 35):
            kept = torch.empty(B, kvh, budget, dtype=torch.int32, device="cuda")
            cache.evict(budget, recent, tl, scores, kept)
            for b in range(B):
                for h in range(kvh):
                    L = len(A[b][h])
                    stay = kept[b, h][kept[b, h] >= 0].long().cpu()
                    assert len(stay) == min(L, budget)
                    if L > budget:                           # what left scored no more than what stayed (to the sums' roundings)
                        mid = torch.zeros(L, dtype=torch.bool)
                        mid[2: L - recent] = True
                        gone = mid.clone()
                        gone[stay] = False
                        mid &= ~gone
                        assert not gone[:2].any() and A[b][h][gone].max() <= A[b][h][mid].min() + 1e-4
                    K[b][h], V[b][h], A[b][h] = K[b][h][stay], V[b][h][stay], A[b][h][stay]
        tl += 1
        q, kn, vn = made(B, heads), made(B, kvh), made(B, kvh)
        cache.step(q.cuda(), kn.cuda(), vn.cuda(), out)
        near(out, torch.stack([one(b, q[b], kn[b], vn[b]) for b in range(B)]))
    for b in range(B):
        for h in range(kvh):
            assert tl[b] == len(A[b][h]) and ((scores[b, h, : tl[b]].double().cpu() - A[b][h]).abs() < 1e-4).all()


def test_the_binding_refuses_rows_of_another_kind():
    p = Paged(45, [20, 30], heads=4, kv_heads=2, d=64, scores=True)
    x = p.device()
    q, k, v, o, c = x["q"], x["k_new"], x["v_new"], x["out"], x["cache"]
    wide = torch.zeros(2, 4, 128, dtype=q.dtype, device="cuda")
    for bad in ((q.float(), k, v, o), (q[:1], k, v, o), (q, k, None, o), (q, None, v, o), (q.cpu(), k, v, o), (q, q, v, o),
                (wide[..., ::2], k, v, o), (q, k, v, q.double())):
        with pytest.raises(wkv.WkvError):
            c.step(*bad)
    for starts, most in ((x["starts"].long(), 1), (x["starts"][:2], 1), (x["starts"].cpu(), 1), (x["starts"], 0), (x["starts"], 3)):
        with pytest.raises(wkv.WkvError):
            c.prefill(q, k, v, o, starts, most)
    for args in ((0, 1, x["lens"], x["scores"]), (8, 9, x["lens"], x["scores"]), (8, 1, x["lens"].float(), x["scores"]),
                 (8, 1, x["lens"], x["scores"][:1]), (8, 1, x["lens"], x["scores"], x["lens"])):
        with pytest.raises(wkv.WkvError):
            c.evict(*args)
    with pytest.raises(wkv.WkvError):
        wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 4).evict(8, 1, x["lens"], x["scores"])
    torch.cuda.synchronize()
    assert (o == 7.0).all()


# ---------------------------------------------------------------- every way that a call's size leads
@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("dtype,d", [("fp16", 128), ("fp32", 64)])
def test_steps_of_many_sequences(dtype, d, scores):
    """More workgroups than run at once (longest sequences first), and more sequences than are put in order together."""
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 70, (100,), generator=g).tolist()
    run(Paged(51, lens, heads=8, kv_heads=8, d=d, dtype=dtype, scores=scores))
    lens = torch.randint(0, 40, (300,), generator=g).tolist()
    run(Paged(52, lens, heads=4, kv_heads=4, d=64, dtype=dtype, scores=scores, window=17, sink=2))
    run(Paged(53, lens, heads=3, kv_heads=3, d=64, dtype=dtype, scores=scores))


def test_lengths_below_zero_among_many_sequences():
    """Sequences in order of their lengths, their number no multiple of 4: lengths below 0 count as 0."""
    p = Paged(67, [n % 50 for n in range(129)] + [0], heads=8, kv_heads=8, d=64, scores=True)
    x = p.device()
    x["lens"].copy_(torch.tensor([n if n else -2 ** 31 + b for b, n in enumerate(p.lens)], dtype=torch.int32))
    run(p, x=x)


def test_many_heads_to_a_kv_head():
    run(Paged(54, [70, 3], heads=300, kv_heads=1, d=64, scores=True))
    run(Paged(55, [70, 3], [5, 3], heads=300, kv_heads=1, d=64, scores=True))


@pytest.mark.parametrize("dtype,d,heads,kv_heads", [("fp16", 64, 71, 1), ("bf16", 128, 66, 2), ("bf16", 256, 33, 1), ("fp32", 128, 48, 1)])
@pytest.mark.parametrize("scores", [False, True])
def test_steps_of_many_heads_to_a_kv_head(dtype, d, heads, kv_heads, scores):
    """More rows a unit than short chunks have, onto sequences long enough for the kernel that takes longer chunks."""
    run(Paged(56, [700, 3, 0, 290], heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, page=32, scores=scores))
    run(Paged(57, [700, 3, 0, 290], heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, window=99, sink=5, scores=scores))


@pytest.mark.parametrize("dtype,d", [("fp16", 64), ("bf16", 128), ("bf16", 256), ("fp32", 128)])
def test_short_chunks_onto_long_sequences(dtype, d):
    """The keys are cut into parts, few and many, for both kernels."""
    for lens, new, heads in (([1200, 90], [3, 2], 4), ([1200, 90], [30, 2], 8), ([2700], [2], 1), ([2700], [40], 4)):
        run(Paged(56, lens, new, heads=heads, kv_heads=1, d=d, dtype=dtype, page=64, scores=True))
        run(Paged(57, lens, new, heads=heads, kv_heads=1, d=d, dtype=dtype, page=32, window=900, sink=5))


@pytest.mark.parametrize("dtype,d", [("fp16", 128), ("bf16", 64)])
def test_chunks_of_many_sequences(dtype, d):
    """More than 512 tiles of rows."""
    g = torch.Generator().manual_seed(6)
    lens = torch.randint(33, 60, (70,), generator=g).tolist()
    run(Paged(58, lens, [min(n, 35) for n in lens], heads=8, kv_heads=8, d=d, dtype=dtype, max_pages=20, scores=True))


def test_evict_more_slots_than_a_workgroup_holds():
    g = torch.Generator().manual_seed(8)
    n, page, kvh, d = 40000, 4096, 2, 64
    k = torch.randn(11, page, kvh, d, generator=g).half()
    p = Paged(59, [1], heads=2, kv_heads=kvh, d=d, page=page, sink=3, scores=True, spare=0, max_pages=10)
    p.lens, p.k, p.v = [n], k, k.flip(0).contiguous()
    p.table = torch.randperm(11, generator=g)[:10].to(torch.int32)[None]
    p.scores = (torch.rand(1, kvh, 10 * page, generator=g) * 5000).floor()
    _evict(p, 39000, 100)
    _evict(p, 500, 100, in_place=True)


def test_offsets_beyond_32_bits():
    """A pool whose pages are 2 GiB apart, rows of calls far apart: step, chunk and eviction."""
    big = torch.empty(5 << 30, dtype=torch.float16, device="cuda")
    for new in (None, [45, 20]):
        p = Paged(60, [70, 20], new, heads=4, kv_heads=2, d=64, spare=0, scores=True)
        x = p.device()
        n = p.k.shape[0]
        assert n <= 8
        view = {"k": big[: 4 << 30], "v": big[1 << 12:]}
        for w in ("k", "v"):
            y = view[w].as_strided((n, p.page, p.kv_heads, p.d), ((1 << 29) + 8, 64 * p.kv_heads, 64, 1))
            y.copy_(x[w])
            x[w] = y
        x["cache"] = wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], p.heads, scores=x["scores"])
        run(p, x=x)
    p = _full(Paged(61, [70, 20], heads=2, kv_heads=2, d=64, spare=0, scores=True))
    x = p.device()
    for w in ("k", "v"):
        y = view[w].as_strided((p.k.shape[0], p.page, 2, 64), ((1 << 29) + 8, 128, 64, 1))
        y.copy_(x[w])
        x[w] = y
    cache = wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 2, scores=x["scores"])
    cache.evict(30, 3, x["lens"], x["scores"])
    torch.cuda.synchronize()
    _, lens, scores, k, v = paged.evicted(p, 30, 3)
    assert x["lens"].tolist() == lens and paged.same(x["scores"].cpu(), scores) and paged.same(x["k"].cpu(), k) and paged.same(x["v"].cpu(), v)


def test_shared_pages_and_broadcast_rows():
    """Two sequences with the same first pages; one row for all tokens, by strides of 0."""
    p = Paged(62, [100, 100], heads=4, kv_heads=2, d=64, page=16, scores=True)
    p.table[1, :6] = p.table[0, :6]
    for b in (0, 1):
        for j in range(96, 99):
            at = p.where(b, j)
            p.k[at], p.v[at] = p.k[p.where(0, j)], p.v[p.where(0, j)]
    run(p)
    p = Paged(63, [50, 20], [50, 20], heads=4, kv_heads=2, d=64, scores=True)
    x = p.device()
    for n in ("q", "k_new", "v_new"):
        setattr(p, n, getattr(p, n)[:1].expand(p.rows, -1, -1).contiguous())
        x[n] = x[n][:1].expand(p.rows, -1, -1)
    x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 50)
    torch.cuda.synchronize()
    paged.check(p, x)


def test_lengths_and_starts_that_do_not_fit():
    """Lengths below 0 and beyond the table, chunks longer than max_new or than their sequence, starts that decrease or lie
    outside: all are cut to what is there."""
    p = Paged(64, [64, 48, 33], heads=4, kv_heads=2, d=64, max_pages=4, scores=True)
    p.lens[0] = 64
    x = p.device()
    x["lens"].copy_(torch.tensor([1 << 20, 48, -7], dtype=torch.int32))
    p.lens, p.new = [64, 48, 0], [1, 1, 0]
    p.k_new[2], p.v_new[2] = 0, 0
    run(p, x=x)
    p = Paged(65, [40, 30, 20], [5, 30, 20], heads=4, kv_heads=2, d=64, extra_rows=9, scores=True)
    x = p.device()
    before = {n: x[n].clone() for n in ("k", "v", "scores")}
    x["starts"].copy_(torch.tensor([3, 1, -50, 1 << 30], dtype=torch.int32))
    # sequence 0: from 3 to max(1, 3), none; 1: from 1 to 1, none; 2: from 0 to the end of 64 rows, cut to 25, five more than its 20 slots
    x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 25)
    torch.cuda.synchronize()
    p.starts, p.new = [0, 0, 0], [0, 0, 25]
    p.starts[2] = 0
    out, tol, sums, stol = p.reference()
    out[25:] = 7.0
    paged.close(x["out"], out, tol, "out")
    paged.close(x["scores"], sums, stol, "scores")
    k, v = p.appended()
    assert paged.same(x["k"].cpu(), k) and paged.same(x["v"].cpu(), v) and not paged.same(x["k"], before["k"])


def test_the_same_call_gives_the_same_bits():
    for new in (None, [300, 90]):
        got = []
        for _ in range(2):
            p = Paged(66, [1500, 90], new, heads=8, kv_heads=2, d=128, dtype="bf16", page=64, scores=True)
            x = p.device()
            if new is None:
                x["cache"].step(x["q"], x["k_new"], x["v_new"], x["out"])
            else:
                x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 300)
            torch.cuda.synchronize()
            got.append((x["out"], x["scores"], x["k"]))
        assert all(paged.same(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_the_largest_window(dtype):
    """A window of 2^31 - 1 is none, also for tokens that have no slot (a chunk longer than its sequence)."""
    p = Paged(68, [20, 300], [20, 260], heads=4, kv_heads=2, d=64, dtype=dtype, window=2 ** 31 - 1, sink=2, scores=True, extra_rows=5)
    x = p.device()
    p.lens, p.new = [13, 300], [20, 260]                     # seven rows of the first sequence before its slot 0
    x["lens"].copy_(torch.tensor(p.lens, dtype=torch.int32))
    run(p, x=x)
    p = Paged(69, [20, 300], heads=4, kv_heads=2, d=64, dtype=dtype, window=2 ** 31 - 1, sink=2 ** 31 - 1, scores=True)
    run(p)


def test_the_workspace_grows_by_steps():
    """A chunk longer by one token every time does not want a new workspace every time, and all of them stay within a small multiple
    of what the longest wants."""
    p = Paged(70, [200], [200], heads=4, kv_heads=2, d=64, scores=True)
    x = p.device()
    seen = set()
    for n in range(1, 201):
        x["lens"].fill_(n)
        x["starts"][1] = n
        x["cache"].prefill(x["q"][:n], x["k_new"][:n], x["v_new"][:n], x["out"][:n], x["starts"], n)
        seen.add(x["cache"]._at)
    torch.cuda.synchronize()
    most = max(wkv._lib.wkv_paged_workspace_bytes(ctypes.byref(x["cache"].c), n, n) for n in range(1, 201))
    assert len(seen) < 20 and x["cache"]._bytes <= 1.5 * most
    with pytest.raises(wkv.WkvError, match="32-bit"):
        x["cache"].evict(2 ** 32 + 9, 1, x["lens"], x["scores"])


def test_many_rows_of_more_than_a_few_parts():
    """Rows that are joined from five and more parts, as many as fill the chip."""
    run(Paged(71, [2100], [260], heads=8, kv_heads=1, d=128, dtype="bf16", page=64, scores=True))
    run(Paged(72, [2100, 2000], [130, 130], heads=8, kv_heads=1, d=64, window=1900, sink=3, missing=[(0, 5)]))
    run(Paged(73, [700, 5100], heads=1024, kv_heads=1, d=64, page=256, scores=True))


def test_tiles_that_share_keys():
    """More heads to a K/V head than a tile has rows, in numbers of workgroups that are multiples of the chip's partitions and that are not."""
    for batch, group, kvh in ((8, 40, 1), (4, 17, 4), (3, 64, 1), (1, 96, 2), (8, 9, 3)):
        lens = [(37 * i + 41) % 300 for i in range(batch)]
        run(Paged(74, lens, heads=group * kvh, kv_heads=kvh, d=64, scores=True))
        run(Paged(75, lens, [min(n, 3) for n in lens], heads=group * kvh, kv_heads=kvh, d=64, scores=True))
