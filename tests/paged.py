"""Paged caches for the tests: made from a seed, and what a call on them has to give, in 64 bits on the CPU.

Everything that no sequence holds (slots behind a length, pages of nobody) is NaN, so that whatever leaks shows.  The reference
takes, for every query, the slots that it sees and nothing else."""
import math

import numpy as np
import torch

from paper_2503_01330_amd import binding as wkv

TORCH = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {t: torch.finfo(x).eps / 2 for t, x in TORCH.items()}
U = 2.0 ** -24
BAD = float("nan")


class Paged:
    def __init__(self, seed, lens, new=None, heads=8, kv_heads=2, d=128, dtype="fp16", page=16, layout="slots", window=0, sink=0,
                 scores=False, max_pages=None, spare=3, missing=(), gain=1.0, extra_rows=0, score_slack=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.kv_heads, self.d, self.dtype, self.page = list(lens), heads, kv_heads, d, dtype, page
        self.new = [min(n, 1) for n in lens] if new is None else list(new)
        self.window, self.sink, self.step = window, sink, new is None
        B = len(lens)
        used = [-(-n // page) for n in lens]
        self.max_pages = max_pages or max(1, max(used))
        n_pages = sum(used) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((B, self.max_pages), -1, dtype=torch.int32)
        for b in range(B):
            for i in range(used[b]):
                self.table[b, i] = order.pop()
            for i in range(used[b], self.max_pages):         # entries that nothing should look at
                self.table[b, i] = [-1, n_pages, 2 ** 30, order[0] if order else -7][(b + i) % 4]
        for b, i in missing:
            self.table[b, i] = -1 if (b + i) % 2 else n_pages + 5
        t = TORCH[dtype]
        self.k, self.v = (torch.full((n_pages, page, kv_heads, d), BAD, dtype=t) for _ in range(2))
        self.rows = sum(self.new) + extra_rows if new is not None else B
        self.q = torch.randn(self.rows, heads, d, generator=g).mul(gain).to(t)
        self.k_new, self.v_new = (torch.randn(self.rows, kv_heads, d, generator=g).to(t) for _ in range(2))
        self.starts = [0]
        for n in self.new:
            self.starts.append(self.starts[-1] + n)
        for b in range(B):
            for j in range(max(0, lens[b] - self.new[b])):
                at = self.where(b, j)
                if at:
                    self.k[at], self.v[at] = (torch.randn(kv_heads, d, generator=g).to(t) for _ in range(2))
        n = max(self.max_pages * page - score_slack, *lens)
        self.scores = torch.rand(B, kv_heads, n, generator=g) * 3 if scores else None
        self.layout = layout

    def where(self, b, j):
        p = int(self.table[b, j // self.page])
        return (p, j % self.page) if 0 <= p < self.k.shape[0] else None

    def row(self, b, i):
        return b if self.step else self.starts[b] + i

    def device(self, dev="cuda"):
        """The tensors on the GPU and a cache over them."""
        x = {}
        for n in ("k", "v"):
            y = getattr(self, n)
            if self.layout == "heads":                       # [page][head][slot][d]
                y = y.transpose(1, 2).contiguous().to(dev).transpose(1, 2)
            elif self.layout == "padded":                    # rows and pages further apart than they are long
                z = torch.full((y.shape[0], y.shape[1] + 1, y.shape[2] + 1, y.shape[3] + 16), BAD, dtype=y.dtype, device=dev)
                z[:, : y.shape[1], : y.shape[2], : y.shape[3]] = y.to(dev)
                y = z[:, : y.shape[1], : y.shape[2], : y.shape[3]]
            else:
                y = y.to(dev)
            x[n] = y
        for n in ("table", "q", "k_new", "v_new", "scores"):
            y = getattr(self, n)
            x[n] = None if y is None else y.to(dev)
        if self.layout == "heads":                           # rows of a call by head, too
            for n in ("q", "k_new", "v_new"):
                x[n] = x[n].transpose(0, 1).contiguous().transpose(0, 1)
        x["lens"] = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        x["starts"] = torch.tensor(self.starts, dtype=torch.int32, device=dev)
        x["out"] = torch.full_like(x["q"], 7.0)
        x["cache"] = wkv.PagedCache(x["k"], x["v"], x["table"], x["lens"], self.heads, window=self.window, n_sink=self.sink, scores=x["scores"])
        return x

    def appended(self):
        """The pools with the new rows in them."""
        k, v = self.k.clone(), self.v.clone()
        for b, n in enumerate(self.new):
            for i in range(n):
                j = self.lens[b] - n + i
                at = self.where(b, j) if j >= 0 else None
                if at:
                    k[at], v[at] = self.k_new[self.row(b, i)], self.v_new[self.row(b, i)]
        return k, v

    def sees(self, b, p):
        return [j for j in range(p + 1) if (not self.window or j > p - self.window or j < self.sink) and self.where(b, j)]

    def reference(self, append=True):
        """out, its tolerance, scores, their tolerance.

        Tolerances count roundings.  A logit is a sum of d products in fp32, each addition and product off by at most a unit of
        2^-23 (the matrix instructions need not round to nearest): |ds| <= 2 (d + 2) U sum |q_i k_i| / sqrt(d), plus 3 roundings of
        size |s| on the way to the exponent; so a weight is off by e = 2 max |ds| relative, the factor 2 for the reference that is
        subtracted, and by 4 U more for the exponential and the sum.  As operands of the second product weights of 16-bit caches are
        rounded: w below.  The second product's sum over n keys adds 2 (n + 8) U."""
        k, v = self.appended() if append else (self.k, self.v)
        out = torch.full((self.rows, self.heads, self.d), 7.0, dtype=torch.float64)
        tol = torch.zeros_like(out)
        sums = self.scores.double().clone() if self.scores is not None else None
        stol = torch.zeros_like(sums) if sums is not None else None
        group = self.heads // self.kv_heads
        if self.step:
            rounds = [(b, 0, n - 1) for b, n in enumerate(self.lens)]
        else:
            rounds = [(b, i, self.lens[b] - n + i) for b, n in enumerate(self.new) for i in range(n)]
        if sums is not None and append:
            for b, n in enumerate(self.new):
                lo = max(0, self.lens[b] - n)
                sums[b, :, lo: self.lens[b]] = 0
        weight = HALF_STEP[self.dtype] if self.dtype != "fp32" else 0.0
        for b, i, p in rounds:
            r, js = self.row(b, i), self.sees(b, p) if p >= 0 else []
            if not js:
                out[r] = 0
                continue
            at = [self.where(b, j) for j in js]
            K = torch.stack([k[a] for a in at]).double()             # [n, kvh, d]
            V = torch.stack([v[a] for a in at]).double()
            q = self.q[r].double().reshape(self.kv_heads, group, self.d)
            s = torch.einsum("hgd,nhd->hgn", q, K) / math.sqrt(self.d)
            mag = torch.einsum("hgd,nhd->hgn", q.abs(), K.abs()) / math.sqrt(self.d)
            top = s.amax(-1, keepdim=True)
            w = torch.where(torch.isneginf(top), 0.0, torch.exp(s - torch.where(torch.isneginf(top), 0.0, top)))
            w = w / w.sum(-1, keepdim=True).clamp(min=1e-300)
            o = torch.stack([torch.stack([(w[h, g][:, None] * V[:, h]).sum(0) for g in range(group)]) for h in range(self.kv_heads)])
            a = torch.stack([w[h] @ V[:, h].abs() for h in range(self.kv_heads)])
            e = 2 * (2 * (self.d + 2) * U * mag.nan_to_num(0, 0, 0).amax(-1) + 3 * U * s.abs().nan_to_num(0, 0, 0).amax(-1)) + 4 * U
            n = len(js)
            rel = (e + 2 * (n + 8) * U + weight)[..., None]
            out[r] = o.reshape(self.heads, self.d)
            tol[r] = (HALF_STEP[self.dtype] * o.abs() * (1 + rel) + rel * a + 1e-38 * n
                      + (2.0 ** -25 if self.dtype == "fp16" else 0)).reshape(self.heads, self.d)
            if sums is not None:
                for h in range(self.kv_heads):
                    sums[b, h, js] += w[h].sum(0)
                    stol[b, h, js] += (w[h] * (e[h][:, None] + 2 * (n + 8) * U)).sum(0) + 1e-30
        if sums is not None:
            stol += 2 * U * (sum(self.new) * group + 2) * sums.abs()
        return out, tol, sums, stol


def same(a, b):
    """Bit for bit, NaNs included."""
    bits = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


def close(got, want, tol, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaNs elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine]
    assert torch.isfinite(got[fine]).all() and bool((off <= tol[fine]).all()), \
        f"{what}: {float((off / tol[fine].clamp(min=1e-300)).max()):.3g} times the tolerance, {float(off.max()):.3g} off"


def run(p, append=True, stream=None, x=None):
    """One call on p, checked whole: outputs, pools, sums."""
    x = x or p.device()
    k, v = (x["k_new"], x["v_new"]) if append else (None, None)
    if p.step:
        x["cache"].step(x["q"], k, v, x["out"], stream=stream)
    else:
        x["cache"].prefill(x["q"], k, v, x["out"], x["starts"], max(1, max(p.new)), stream=stream)
    torch.cuda.synchronize()
    check(p, x, append)
    return x


def check(p, x, append=True):
    out, tol, sums, stol = p.reference(append)
    close(x["out"], out, tol, "out")
    k, v = p.appended() if append else (p.k, p.v)
    assert same(x["k"].cpu(), k) and same(x["v"].cpu(), v), "the pools are not what they should be"
    if sums is not None:
        close(x["scores"], sums, stol, "scores")


def evicted(p, budget, recent):
    """kept, new lengths, sums and pools after an eviction, in plain Python."""
    B = len(p.lens)
    kept = np.full((B, p.kv_heads, budget), -1, np.int32)
    lens, k, v = list(p.lens), p.k.clone(), p.v.clone()
    scores = p.scores.clone()
    for b, n in enumerate(p.lens):
        if not all(p.where(b, j) for j in range(n)):
            continue
        for h in range(p.kv_heads):
            a = [math.inf if math.isnan(x) else x for x in p.scores[b, h, :n].tolist()]
            able = sorted((a[j], j) for j in range(p.sink, n - recent))
            gone = {j for _, j in able[: max(0, n - budget)]}
            stay = [j for j in range(n) if j not in gone]
            kept[b, h, : len(stay)] = stay
            if n > budget:
                for i, j in enumerate(stay):
                    to, src = p.where(b, i), p.where(b, j)
                    k[to[0], to[1], h], v[to[0], to[1], h] = p.k[src[0], src[1], h], p.v[src[0], src[1], h]
                scores[b, h, :n] = 0
                scores[b, h, : len(stay)] = p.scores[b, h, stay]
        lens[b] = min(n, budget)
    return kept, lens, scores, k, v
