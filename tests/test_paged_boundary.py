"""Host-side checks of the paged cache's entry points that need no GPU: what is refused, with which code, and the size arithmetic.
Addresses are made up: nothing may be launched with them."""
import ctypes as C

import pytest
import torch

from paper_2503_01330_amd import binding as wkv

P = 1 << 20          # a made-up address, 16-byte aligned


def cache(**kw):
    x = dict(k=P, v=P, page_stride=16 * 2 * 128, slot_stride=2 * 128, head_stride=128, table=P, table_stride=8, lens=P, scores=P,
             score_stride=None, batch=3, heads=8, kv_heads=2, head_dim=128, dtype=wkv.WKV_FP16, page_size=16, n_pages=20, max_pages=8,
             window=0, n_sink=0)
    x.update(kw)
    if x["score_stride"] is None:
        x["score_stride"] = x["max_pages"] * x["page_size"]
    return wkv.wkv_paged(**x)


def rows(**kw):
    x = dict(q=P, k=P, v=P, out=P, q_stride=1024, q_head_stride=128, k_stride=256, k_head_stride=128, v_stride=256, v_head_stride=128,
             out_stride=1024, out_head_stride=128)
    x.update(kw)
    return wkv.wkv_paged_rows(**x)


def step(c, r, work=P, size=0):
    return wkv._lib.wkv_paged_step(C.addressof(c) if c else None, C.addressof(r) if r else None, work, size, None)


def prefill(c, r, starts=P, n=10, most=5, work=P, size=0):
    return wkv._lib.wkv_paged_prefill(C.addressof(c), C.addressof(r), starts, n, most, work, size, None)


def evict(c, budget=50, recent=5, new_lens=P, new_scores=P, kept=None, work=P, size=0):
    return wkv._lib.wkv_paged_evict(C.addressof(c), budget, recent, new_lens, new_scores, kept, work, size, None)


# With a workspace of 0 bytes a call that is otherwise sound ends with this (sums of weights always need some: nothing is launched).
SOUND = wkv.WKV_ESIZE


def test_structures_have_the_layout_of_the_header():
    assert C.sizeof(wkv.wkv_paged) == 8 * 10 + 4 * 14 and C.sizeof(wkv.wkv_paged_rows) == 8 * 12


def test_sound_calls_reach_the_workspace_check():
    c = cache(scores=P, score_stride=128)
    assert step(c, rows()) == SOUND and "workspace" in wkv.wkv_last_error()
    assert prefill(c, rows()) == SOUND and "workspace" in wkv.wkv_last_error()
    assert evict(c) == SOUND and "workspace" in wkv.wkv_last_error()


SHAPES = [
    (dict(batch=0), wkv.WKV_EINVAL), (dict(heads=0), wkv.WKV_EINVAL), (dict(kv_heads=-2), wkv.WKV_EINVAL), (dict(kv_heads=3), wkv.WKV_EINVAL),
    (dict(batch=1 << 22), wkv.WKV_ESIZE), (dict(head_dim=96), wkv.WKV_EINVAL), (dict(head_dim=256, dtype=wkv.WKV_FP32), wkv.WKV_EINVAL),
    (dict(dtype=3), wkv.WKV_EINVAL), (dict(page_size=8), wkv.WKV_EINVAL), (dict(page_size=48), wkv.WKV_EINVAL),
    (dict(page_size=8192), wkv.WKV_EINVAL), (dict(n_pages=0), wkv.WKV_EINVAL), (dict(max_pages=0), wkv.WKV_EINVAL),
    (dict(max_pages=(1 << 20) + 1, table_stride=1 << 21), wkv.WKV_ESIZE), (dict(window=-1), wkv.WKV_EINVAL), (dict(n_sink=-1), wkv.WKV_EINVAL),
    (dict(scores=P, score_stride=112), wkv.WKV_EINVAL), (dict(scores=P, score_stride=129), wkv.WKV_EINVAL),
]


@pytest.mark.parametrize("kw,code", SHAPES + [
    (dict(k=None), wkv.WKV_EINVAL), (dict(v=None), wkv.WKV_EINVAL), (dict(table=None), wkv.WKV_EINVAL), (dict(lens=None), wkv.WKV_EINVAL),
    (dict(k=P + 8), wkv.WKV_EINVAL), (dict(v=P + 2), wkv.WKV_EINVAL), (dict(table=P + 2), wkv.WKV_EINVAL), (dict(lens=P + 1), wkv.WKV_EINVAL),
    (dict(scores=P + 2, score_stride=128), wkv.WKV_EINVAL), (dict(page_stride=4), wkv.WKV_EINVAL), (dict(slot_stride=132), wkv.WKV_EINVAL),
    (dict(head_stride=-128), wkv.WKV_EINVAL), (dict(table_stride=7), wkv.WKV_EINVAL),
])
def test_descriptions_that_are_refused(kw, code):
    c = cache(**kw)
    assert step(c, rows()) == code and wkv.wkv_last_error()
    assert prefill(c, rows()) == code
    assert evict(c) == code


@pytest.mark.parametrize("kw,code", SHAPES)
def test_no_workspace_for_a_description_that_is_refused(kw, code):
    assert wkv._lib.wkv_paged_workspace_bytes(C.byref(cache(**kw)), 0, 0) == 0


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(q=P + 8), dict(k=P + 4), dict(v=P + 2), dict(out=P + 8), dict(q_stride=1028),
    dict(k_head_stride=4), dict(v_stride=-256), dict(q_head_stride=-128), dict(out_stride=64), dict(out_head_stride=0), dict(out_head_stride=64),
])
def test_rows_that_are_refused(kw):
    assert step(cache(), rows(**kw)) == wkv.WKV_EINVAL
    assert prefill(cache(), rows(**kw)) == wkv.WKV_EINVAL


def test_strides_that_32_bits_do_not_hold():
    assert step(cache(slot_stride=(1 << 25) + 8), rows()) == wkv.WKV_ESIZE
    assert step(cache(), rows(k_stride=(1 << 25) + 8)) == wkv.WKV_ESIZE and prefill(cache(), rows(v_stride=1 << 30)) == wkv.WKV_ESIZE
    assert step(cache(page_stride=1 << 40, head_stride=1 << 40), rows(q_stride=1 << 40, k_head_stride=1 << 40, out_stride=1 << 40)) == SOUND


def test_rows_that_are_not_used_are_not_looked_at():
    work = wkv._lib.wkv_paged_workspace_bytes(C.byref(cache()), 0, 0)
    assert work > 0
    assert step(cache(), rows(k=None, v=None, k_stride=3, v_head_stride=-1)) == SOUND
    assert step(cache(), rows(q_stride=0, q_head_stride=0, k_stride=0)) == SOUND             # one row for all tokens or heads
    assert step(cache(batch=1, heads=1, kv_heads=1), rows(out_stride=0, out_head_stride=0)) == SOUND


def test_null_arguments():
    assert step(None, rows()) == wkv.WKV_EINVAL and step(cache(), None) == wkv.WKV_EINVAL
    assert prefill(cache(), rows(), starts=None) == wkv.WKV_EINVAL and prefill(cache(), rows(), starts=P + 2) == wkv.WKV_EINVAL
    assert wkv._lib.wkv_paged_workspace_bytes(None, 0, 0) == 0


@pytest.mark.parametrize("n,most", [(0, 1), (10, 0), (10, 11), (-1, -1)])
def test_chunk_sizes_that_are_refused(n, most):
    assert prefill(cache(), rows(), n=n, most=most) == wkv.WKV_EINVAL
    if (n, most) != (10, 0):                               # (no chunk at all is what a cache without prefills asks for)
        assert wkv._lib.wkv_paged_workspace_bytes(C.byref(cache()), n, most) == 0


def test_evictions_that_are_refused():
    c = dict(scores=P, score_stride=128)
    assert evict(cache(scores=None)) == wkv.WKV_EINVAL
    assert evict(cache(**c, window=64)) == wkv.WKV_EINVAL
    assert evict(cache(**c), new_lens=None) == wkv.WKV_EINVAL and evict(cache(**c), new_scores=None) == wkv.WKV_EINVAL
    assert evict(cache(**c), new_lens=P + 2) == wkv.WKV_EINVAL and evict(cache(**c), kept=P + 2) == wkv.WKV_EINVAL
    for budget, recent, sink in ((0, 1, 0), (10, 0, 0), (10, 11, 0), (10, 7, 4), (-5, 1, 0)):
        assert evict(cache(**c, n_sink=sink), budget, recent) == wkv.WKV_EINVAL
    assert evict(cache(**c, n_sink=4), 10, 6) == SOUND


def test_workspaces_that_are_refused():
    c = cache(scores=P, score_stride=128)
    need = wkv._lib.wkv_paged_workspace_bytes(C.byref(c), 10, 5)
    assert step(c, rows(), work=None, size=need) == wkv.WKV_EINVAL and step(c, rows(), work=P + 8, size=need) == wkv.WKV_EINVAL
    assert evict(c, work=None, size=need) == wkv.WKV_EINVAL and prefill(c, rows(), work=P + 4, size=need) == wkv.WKV_EINVAL


def test_workspace_arithmetic():
    """Logits of a step whose weights are summed: a float a slot and query head; of a prefill: a float a token and head; the list of an
    eviction: an int a slot and K/V head."""
    def need(n=0, most=0, **kw):
        return wkv._lib.wkv_paged_workspace_bytes(C.byref(cache(**kw)), n, most)
    s = dict(scores=P, score_stride=128)
    assert 0 < need(scores=None) < need(**s) <= need(1000, 10, **s)
    assert need(**s) >= 3 * 8 * 128 * 4
    assert need(100000, 10, **s) >= 100000 * 8 * 4
    long = dict(batch=1, heads=1, kv_heads=1, max_pages=1 << 12, table_stride=1 << 12, scores=P, score_stride=1 << 16)
    assert need(**long) >= (1 << 16) * 4


def test_chunks_that_32_bits_do_not_count():
    small = dict(heads=1, kv_heads=1, batch=1)
    assert prefill(cache(**small), rows(), n=1 << 30, most=1 << 24) == SOUND and "workspace" in wkv.wkv_last_error()
    assert prefill(cache(**small), rows(), n=1 << 30, most=(1 << 24) + 1) == wkv.WKV_ESIZE and "max_new" in wkv.wkv_last_error()
    assert prefill(cache(), rows(), n=(1 << 27) + 1, most=5) == wkv.WKV_ESIZE and "n_tokens" in wkv.wkv_last_error()
    assert wkv._lib.wkv_paged_workspace_bytes(C.byref(cache()), (1 << 27) + 1, 5) == 0
    assert wkv._lib.wkv_paged_workspace_bytes(C.byref(cache(**small)), 1 << 30, (1 << 24) + 1) == 0


def test_evictions_of_too_many_units_are_refused():
    c = cache(batch=1 << 10, heads=1 << 9, kv_heads=1 << 9, n_sink=1)
    assert evict(c, size=1 << 62) == wkv.WKV_ESIZE and "threads" in wkv.wkv_last_error()


def test_launches_of_too_many_threads_are_refused():
    c = cache(batch=1 << 12, heads=1 << 10, kv_heads=1 << 10, page_stride=16 << 17, slot_stride=1 << 17, max_pages=1 << 10, table_stride=1 << 10)
    r = rows(q_stride=1 << 17, k_stride=1 << 17, v_stride=1 << 17, out_stride=1 << 17)
    assert prefill(c, r, n=1 << 20, most=1 << 12, size=1 << 62) == wkv.WKV_ESIZE and "threads" in wkv.wkv_last_error()


def test_binding_refuses_what_it_cannot_describe():
    k = torch.zeros(4, 16, 2, 64, dtype=torch.float16)
    table, lens = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for bad in (dict(k=k[0]), dict(v=k.float()), dict(v=k[:3]), dict(table=table.long()), dict(lens=lens[:1]), dict(lens=lens.float()),
                dict(scores=torch.zeros(2, 3, 32)), dict(scores=torch.zeros(2, 2, 32).half()), dict(k=k.double(), v=k.double()),
                dict(k=k.transpose(0, 3), v=k.transpose(0, 3)), dict()):            # (the last: sound, but not on a GPU)
        x = dict(k=k, v=k, table=table, lens=lens, scores=None)
        x.update(bad)
        with pytest.raises(wkv.WkvError) as e:
            wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], 4, scores=x["scores"])
        assert e.value.code == wkv.WKV_EINVAL


@pytest.mark.parametrize("kw", [dict(heads=2 ** 32 + 4), dict(window=2 ** 32), dict(n_sink=2 ** 31), dict(max_tokens=2 ** 32, max_new=1)])
def test_binding_refuses_numbers_of_more_than_32_bits(kw):
    k = torch.zeros(4, 16, 2, 64, dtype=torch.float16)
    table, lens = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(wkv.WkvError, match="32-bit"):
        wkv.PagedCache(k, k, table, lens, **{**dict(heads=4), **kw})
