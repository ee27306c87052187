"""The paged cache's operators, as cases that can be timed: one pass through an operator, as a program calls it.

Three kinds, all through paper_2503_01330_amd.binding.PagedCache:

  step     one new token for every sequence: its K and V rows go into the sequence's last slot, its
           query attends over the pages (all of them, or a sliding window and a few first tokens);
           with scores, the weights are added to the running sum of every slot;
  prefill  a chunk of new tokens for every sequence, the last ones of what the cache then holds;
  evict    every sequence cut down to a budget: the slots of lowest running sum outside the first
           and the newest tokens leave, the rest move up in order.

With `own` false the same is computed in plain torch, in 32 bits, over the rows gathered from the
pages.  Shapes are those of the library's configurations (32 heads x 128, lengths of 4096 and 32768,
budgets of 819 and 2048, narrow heads of 64, a tiny fp32 cache) and generic ones between them.
"""
import math

import torch

own = False

TORCH = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}

# new: tokens of the longest chunk; ragged: lengths differ, down to a small part of `length`; window, sink: what is visible
# (0: everything); scores: the weights are summed a slot; budget, recent: of an eviction; slots_first: a page is laid out
# [slot][head][d], otherwise [head][slot][d]
_PLAIN = dict(new=1, ragged=False, window=0, sink=0, scores=False, budget=0, recent=0, slots_first=True)


def _case(name, kind, batch, heads, kv_heads, head_dim, dtype, page, length, **kw):
    return dict(name=name, kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, page=page,
                length=length, **{**_PLAIN, **kw})


def listed():
    return [
        # the smallest call: a tiny fp32 cache, where only latency counts
        _case("step tiny fp32", "step", 1, 4, 4, 64, "fp32", 16, 64),
        # one user, a context of 4096 tokens, four query heads to a K/V head
        _case("step one sequence", "step", 1, 32, 8, 128, "fp16", 16, 4096),
        # few long documents
        _case("step long", "step", 4, 32, 8, 128, "fp16", 64, 32768),
        # a serving batch with sequences of every length, whose weights are kept for an eviction to come
        _case("step batch 64 ragged", "step", 64, 32, 8, 128, "bf16", 16, 4096, ragged=True, scores=True),
        # a small model with narrow heads and a sliding window, far into its sequences
        _case("step window narrow", "step", 5, 12, 12, 64, "bf16", 32, 5003, window=333, sink=4),
        # wide heads, sixteen query heads to a K/V head
        _case("step wide heads", "step", 16, 32, 2, 256, "fp16", 32, 2047, ragged=True, slots_first=False),
        # a short question, every head with K and V of its own
        _case("prefill 77", "prefill", 1, 32, 32, 128, "fp16", 16, 77, new=77),
        # the next turn of a few conversations, whose weights are kept
        _case("prefill turn", "prefill", 3, 32, 8, 128, "bf16", 64, 6001, new=333, ragged=True, scores=True),
        # long documents under a sliding window
        _case("prefill window", "prefill", 2, 32, 8, 128, "bf16", 64, 8192, new=8192, window=1024, sink=4),
        # the largest: prompts as long as the model's context
        _case("prefill 4096", "prefill", 4, 32, 8, 128, "fp16", 16, 4096, new=4096),
        # a narrow cache of sequences of odd lengths, cut to a fifth
        _case("evict narrow ragged", "evict", 5, 12, 12, 64, "bf16", 16, 1237, ragged=True, budget=255, recent=17, sink=4),
        # long contexts, cut to 2048 slots
        _case("evict long", "evict", 4, 32, 8, 128, "fp16", 64, 32768, budget=2048, recent=128, sink=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "prefill", "prefill", "evict"])
    dtype = rng.choice(["fp16", "bf16", "fp16", "bf16", "fp32"] if kind != "prefill" else ["fp16", "bf16"])
    head_dim = rng.choice([64, 128, 128] if dtype == "fp32" else [64, 128, 128, 256])
    heads, kv_heads = rng.choice([(4, 4), (12, 12), (32, 8), (32, 8), (32, 2), (32, 32), (20, 4), (7, 1)])
    c = _case("", kind, 1, heads, kv_heads, head_dim, dtype, rng.choice([16, 32, 64]), 1, ragged=rng.random() < 0.6,
              slots_first=rng.random() < 0.7)
    del c["name"]
    row = 2 * kv_heads * head_dim * BYTES[dtype]
    c["batch"] = _log(rng, 1, 64 if kind == "step" else 6)
    if kind == "prefill":
        c["length"] = _log(rng, 16, 8192)
        c["new"] = c["length"] if rng.random() < 0.5 else max(1, int(c["length"] * rng.uniform(0.02, 1)))
        while c["batch"] > 1 and c["batch"] * heads * c["new"] * c["length"] > 4 * 32 * 4096 ** 2 // 2:
            c["batch"] -= 1
        while c["batch"] * heads * c["new"] * c["length"] > 4 * 32 * 4096 ** 2 // 2:
            c["new"] -= c["new"] // 2
    else:
        c["length"] = _log(rng, 64, 32768)
        while c["batch"] > 1 and c["batch"] * c["length"] * row > 4 * 32768 * 2 * 8 * 128 * 2:
            c["batch"] //= 2
        while c["batch"] * c["length"] * row > 4 * 32768 * 2 * 8 * 128 * 2:
            c["length"] //= 2
    if kind == "evict":
        c["budget"] = max(16, int(c["length"] * rng.uniform(0.05, 0.6)))
        c["recent"] = max(1, int(c["budget"] * rng.uniform(0.03, 0.3)))
        c["sink"] = rng.choice([0, 4])
    elif rng.random() < 0.3:
        c["window"] = _log(rng, 16, max(17, c["length"] // 2))
        c["sink"] = rng.choice([0, 4])
    else:
        c["scores"] = rng.random() < 0.4
    return c


def _lens(case):
    """Tokens that each sequence holds when the call is over, and how many of them are new."""
    n = range(case["batch"])
    share = [1.0 - (0.618 * b % 1.0) * (0.97 if case["ragged"] else 0.0) for b in n]
    lens = [max(1, int(case["length"] * s)) for s in share]
    new = [min(lens[b], max(1, int(case["new"] * share[b]))) for b in n]
    return lens, new


def _sees(case, position):
    """How many slots the query at `position` attends over."""
    w = case["window"]
    return position + 1 if not w else min(position + 1, w + min(case["sink"], max(0, position + 1 - w)))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t, d, kvh, page, B = TORCH[case["dtype"]], case["head_dim"], case["kv_heads"], case["page"], case["batch"]
    lens, new = _lens(case)
    wide = -(-case["length"] // page)
    pages = sum(-(-n // page) for n in lens)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    # the pool's pages go to the sequences in any order; keys are of low rank, as a model's are
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    used = 0
    for b, n in enumerate(lens):
        table[b, : -(-n // page)] = order[used: used - (-n // page)]
        used -= -n // page
    mix = normal(kvh, 16, d) / 4.0
    shape = (pages, page, kvh) if case["slots_first"] else (pages, kvh, page)

    def keys(*lead):
        """[*lead, kvh, d]"""
        z = normal(kvh, math.prod(lead), 16)
        return torch.matmul(z, mix).transpose(0, 1).reshape(*lead, kvh, d).to(t)

    k = torch.empty(*shape, d, dtype=t, device="cuda")
    v = torch.empty(*shape, d, dtype=t, device="cuda")
    for lo in range(0, pages, 1024):
        part = keys(min(1024, pages - lo), page)
        k[lo: lo + 1024] = part if case["slots_first"] else part.transpose(1, 2)
        v[lo: lo + 1024] = normal(min(1024, pages - lo), *shape[1:], d).to(t)
    if not case["slots_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)         # always seen as [page][slot][head][d]
    state = {"case": case, "k": k, "v": v, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "scores": None}
    if case["scores"] or case["kind"] == "evict":
        # running sums as attention leaves them: most slots got little, a few much; old ones never attended again hold equal sums
        state["scores"] = torch.empty(B, kvh, case["length"], device="cuda").exponential_(generator=gen).pow_(2)
        state["scores"].mul_(torch.rand(B, kvh, case["length"], generator=gen, device="cuda") > 0.05)
    if case["kind"] == "evict":
        # (the sums of what is left go to a buffer of their own: a program keeps two and takes them in turn)
        state["new_lens"], state["new_scores"] = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros_like(state["scores"])
        state["kept"] = torch.zeros(B, kvh, case["budget"], dtype=torch.int32, device="cuda")
    else:
        n = B if case["kind"] == "step" else sum(new)
        state["q"] = normal(n, case["heads"], d).to(t)
        state["k_new"], state["v_new"] = keys(n), normal(n, kvh, d).to(t)
        state["out"] = torch.empty_like(state["q"])
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        state["starts"], state["max_new"] = torch.tensor(starts, dtype=torch.int32, device="cuda"), max(new)
    if own:
        from paper_2503_01330_amd import binding as wkv
        state["cache"] = wkv.PagedCache(k, v, table, state["lens"], case["heads"], window=case["window"], n_sink=case["sink"],
                                        scores=state["scores"])
    return state


def run(state):
    case = state["case"]
    if case["kind"] == "evict":
        if own:
            state["cache"].evict(case["budget"], case["recent"], state["new_lens"], state["new_scores"], state["kept"])
        else:
            _evict(state)
        return {n: state[n] for n in ("k", "v", "new_scores", "new_lens", "kept")}
    if own and case["kind"] == "step":
        state["cache"].step(state["q"], state["k_new"], state["v_new"], state["out"])
    elif own:
        state["cache"].prefill(state["q"], state["k_new"], state["v_new"], state["out"], state["starts"], state["max_new"])
    else:
        _attend(state)
    return {n: state[n] for n in ("out", "k", "v", "scores")}


# ---------------------------------------------------------------- plain forms
def _rows(state, pool, length):
    """The sequences' rows, [batch, kv_heads, length, d] in 32 bits; slots without a page get those of page 0."""
    x = pool[state["table"].clamp(min=0).long()].float()
    B, n, page, kvh, d = x.shape
    return x.reshape(B, n * page, kvh, d)[:, :length].transpose(1, 2).contiguous()


def _place(state, slot):
    """Page and place within the page of slot[b, i] of sequence b."""
    page = state["case"]["page"]
    return state["table"].long().gather(1, slot // page), slot % page


def _attend(state):
    case, lens, starts = state["case"], state["lens"].long(), state["starts"].long()
    B, H, kvh, d, N, L = case["batch"], case["heads"], case["kv_heads"], case["head_dim"], state["max_new"], case["length"]
    new = starts[1:] - starts[:-1]
    i = torch.arange(N, device="cuda")
    real = i < new[:, None]
    position = lens[:, None] - new[:, None] + i                                  # [B, N]
    row = (starts[:-1, None] + i).clamp(max=state["q"].shape[0] - 1)
    page, place = _place(state, torch.where(real, position, 0))
    state["k"][page[real], place[real]] = state["k_new"]
    state["v"][page[real], place[real]] = state["v_new"]
    K, V = _rows(state, state["k"], L), _rows(state, state["v"], L)              # [B, kvh, L, d]
    q = state["q"].float()[row].reshape(B, N, kvh, H // kvh, d).permute(0, 2, 3, 1, 4).reshape(B * kvh, -1, d)
    s = torch.matmul(q, K.reshape(B * kvh, L, d).transpose(1, 2).contiguous()).mul_(1 / math.sqrt(d)).reshape(B, kvh, H // kvh, N, L)
    j = torch.arange(L, device="cuda")
    seen = (j <= position[:, :, None]) & real[:, :, None]
    if case["window"]:
        seen &= (j > position[:, :, None] - case["window"]) | (j < case["sink"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    w = s.sub_(top).exp_()
    w /= w.sum(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).tiny)
    o = torch.matmul(w.reshape(B * kvh, -1, L), V.reshape(B * kvh, L, d)).reshape(B, kvh, H // kvh, N, d)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, N, H, d)
    state["out"][row[real]] = o[real].to(state["out"].dtype)
    if case["scores"]:
        mine = (j >= (lens - new)[:, None]) & (j < lens[:, None])                # appended by this call: their sums start here
        state["scores"].masked_fill_(mine[:, None], 0.0)
        state["scores"] += w.sum((2, 3))


def _evict(state):
    case, lens = state["case"], state["lens"].long()
    L, m, kvh = case["length"], case["budget"], case["kv_heads"]
    j = torch.arange(L, device="cuda")
    live = j < lens[:, None]
    free = (j >= case["sink"]) & (j < lens[:, None] - case["recent"])
    score = state["scores"].masked_fill(~free[:, None], math.inf)
    order = score.sort(dim=-1, stable=True).indices                                # ties: the oldest first
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order))
    keep = (rank >= (lens - m).clamp(min=0)[:, None, None]) & live[:, None]
    n = torch.minimum(lens, torch.full_like(lens, m))
    src = (~keep).int().sort(dim=-1, stable=True).indices[..., :m]               # kept slots, ascending
    i = torch.arange(src.shape[-1], device="cuda")
    real = i < n[:, None]
    state["kept"].fill_(-1)[..., : src.shape[-1]] = torch.where(real[:, None], src, -1).int()
    page, place = _place(state, torch.where(real, i, 0))
    for name in ("k", "v"):
        rows = _pool_rows(state, state[name], src)
        state[name][page[real], place[real]] = rows[real]
    state["new_scores"].masked_fill_(live[:, None], 0.0)
    had = state["new_scores"][..., : src.shape[-1]]
    had.copy_(torch.where(real[:, None], state["scores"].gather(-1, src), had))
    state["new_lens"].copy_(n)


def _pool_rows(state, pool, src):
    """Rows src[b, h, i] of every sequence and head, [B, i, kvh, d]."""
    page, place = _place(state, src.flatten(1))
    head = torch.arange(src.shape[1], device="cuda")[:, None].expand(src.shape[1:]).flatten()
    return pool[page.clamp(min=0), place, head].reshape(*src.shape, -1).transpose(1, 2)


def work(case):
    """Rows of K and V that some query sees, read once; queries, new rows, outputs; scores read and written."""
    lens, new = _lens(case)
    d, H, kvh, e = case["head_dim"], case["heads"], case["kv_heads"], BYTES[case["dtype"]]
    row = 2 * kvh * d * e
    if case["kind"] == "evict":
        moved = sum(min(n, case["budget"]) for n in lens if n > case["budget"])
        return {"bytes": moved * 2 * row + sum(lens) * kvh * 4 + sum(min(n, case["budget"]) for n in lens) * kvh * 8, "flops": sum(lens) * kvh}
    pairs = sum(_sees(case, p) for n, m in zip(lens, new) for p in range(n - m, n))
    rows = sum(min(n, m + _sees(case, n - m)) for n, m in zip(lens, new))
    scored = sum(lens) * kvh * 8 if case["scores"] else 0
    return {"bytes": rows * row + sum(new) * (2 * H * d * e + row) + scored, "flops": pairs * H * 4 * d}


# ---------------------------------------------------------------- the definition, in 64 bits, sequence by sequence
def exact(case, seed):
    state = prepare(case, seed)
    lens, new = _lens(case)
    d, kvh, page = case["head_dim"], case["kv_heads"], case["page"]
    group = case["heads"] // kvh
    if case["kind"] == "evict":
        K, V, A = (state[n].double() for n in ("k", "v", "scores"))
        left = torch.zeros_like(A)
        for b, n in enumerate(lens):
            where = [int(p) for p in state["table"][b, : -(-n // page)]]
            rows = [x[where].reshape(-1, kvh, d)[:n].clone() for x in (K, V)]
            m = min(n, case["budget"])
            for h in range(kvh):
                a = A[b, h, :n].tolist()
                able = sorted((a[j], j) for j in range(case["sink"], n - case["recent"]))
                gone = {j for _, j in able[: n - m]}
                kept = torch.tensor([j for j in range(n) if j not in gone], device="cuda")
                left[b, h, :m] = A[b, h, kept]
                at = torch.arange(m, device="cuda")
                place = torch.tensor(where, device="cuda")[at // page]
                K[place, at % page, h], V[place, at % page, h] = rows[0][kept, h], rows[1][kept, h]
        return {"k": K, "v": V, "new_scores": left, "new_lens": None, "kept": None}
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    sums = state["scores"].double() if case["scores"] else None
    lo = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        where = state["table"][b, : -(-n // page)].long()
        K, V = (state[x][where].reshape(-1, kvh, d)[:n].double() for x in ("k", "v"))
        K[n - m:], V[n - m:] = state["k_new"][lo: lo + m].double(), state["v_new"][lo: lo + m].double()
        at, j = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        hidden = j > at
        if case["window"]:
            hidden |= (j <= at - case["window"]) & (j >= case["sink"])
        if sums is not None:
            sums[b, :, n - m: n] = 0.0
        for h in range(case["heads"]):
            q = state["q"][lo: lo + m, h].double()
            w = torch.softmax((q @ K[:, h // group].t().contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf), -1)
            out[lo: lo + m, h] = w @ V[:, h // group]
            if sums is not None:
                sums[b, h // group, :n] += w.sum(0)
        lo += m
    return {"out": out, "k": None, "v": None, "scores": sums}
