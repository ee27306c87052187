"""What the paged cache's kernels keep of the weights: those far below a row's largest, and both halves of a step's."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paged
    from paged import HALF_STEP, U, Paged

# Roundings of a weight as an operand of the second product: two 16-bit numbers (steps, short chunks), or one.
TWO = 2.0 ** -16


def attend(p, weight, terms):
    """out of p's call in 64 bits, and its tolerance: as in paged.py, with `weight` relative to every weight, 2^-60 of a row's largest
    (below what either kernel keeps; it sees at most 2^13 slots here), and `terms` products of a logit that are not exact in 32 bits."""
    k, v = p.appended()
    out = torch.full((p.rows, p.heads, p.d), 7.0, dtype=torch.float64)
    tol = torch.zeros_like(out)
    group = p.heads // p.kv_heads
    for b, n in enumerate(p.lens):
        at = [p.where(b, j) for j in range(n)]
        K, V = (torch.stack([x[a] for a in at]).double() for x in (k, v))                 # [n, kvh, d]
        rows = [b] if p.step else list(range(p.starts[b], p.starts[b] + p.new[b]))
        hidden = torch.arange(n) > torch.arange(n - len(rows), n)[:, None]
        for h in range(p.heads):
            q, x, y = p.q[rows, h].double(), K[:, h // group], V[:, h // group]
            s = (q @ x.T / math.sqrt(p.d)).masked_fill(hidden, -math.inf)
            w = torch.softmax(s, -1)
            o, a = w @ y, w @ y.abs()
            mag = (q.abs() @ x.abs().T / math.sqrt(p.d)).masked_fill(hidden, 0).amax(-1, keepdim=True)
            e = 2 * (2 * (terms + 2) * U * mag * (terms > 0) + 3 * U * s.masked_fill(hidden, 0).abs().amax(-1, keepdim=True)) + 4 * U
            rel = e + 2 * (n + 8) * U + weight
            out[rows, h] = o
            half = HALF_STEP[p.dtype]
            tol[rows, h] = half * o.abs() * (1 + rel) + rel * a + 2.0 ** -60 * y.abs().sum(0) + (2.0 ** -25 if p.dtype == "fp16" else 0)
    return out, tol


def check(p, weight, terms):
    x = p.device()
    if p.step:
        x["cache"].step(x["q"], x["k_new"], x["v_new"], x["out"])
    else:
        x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], max(p.new))
    torch.cuda.synchronize()
    paged.close(x["out"], *attend(p, weight, terms), "out")


@pytest.mark.parametrize("new", [None, [3, 2], [300, 60]])
@pytest.mark.parametrize("dtype,d", [("fp16", 64), ("fp16", 128), ("fp16", 256), ("bf16", 128)])
def test_one_key_that_takes_nearly_all(dtype, d, new):
    """A key that lies `gap` above all others, with a value of 0, first and in the middle: the output is what the others sum to."""
    for gap in (10.0, 14.0, 18.0, 22.0, 26.0, 34.0):
        for top in (0, 60):
            p = Paged(81, [1500, 130], new, heads=8, kv_heads=2, d=d, dtype=dtype, page=64)
            p.q[..., 0] = 4.0
            p.k[..., 0] = torch.where(torch.isnan(p.k[..., 0]), p.k[..., 0], 0.0)
            p.k_new[..., 0] = 0.0
            for b in (0, 1):
                at = p.where(b, top)
                p.k[at], p.v[at] = 0.0, 0.0
                p.k[at[0], at[1], :, 0] = gap * math.sqrt(d) / 4.0
            p.q[..., 1:] *= 0.25
            p.v, p.v_new = ((x * 500.0 + 1000.0).to(x.dtype) for x in (p.v, p.v_new))
            for b in (0, 1):
                p.v[p.where(b, top)] = 0.0
            check(p, HALF_STEP[dtype] if new and max(new) > 8 else TWO, d)


@pytest.mark.parametrize("dtype,d", [("fp16", 64), ("fp16", 256), ("bf16", 128)])
def test_steps_and_short_chunks_keep_two_numbers_of_a_weight(dtype, d):
    """Values that cancel, so that the output's rounding is small beside one of a weight; logits that are exact in 32 bits: q and k are
    multiples of 1/8 up to 4, products of 1/64, and sums of 256 of them below 2^18 of these."""
    for lens, new in (([2, 3, 4, 20, 100], None), ([2, 3, 4, 20], [2, 1, 3, 4])):
        p = Paged(82, lens, new, heads=16, kv_heads=4, d=d, dtype=dtype)
        quarter = lambda x: (x * 4).round().clamp(-16, 16) / 8  # noqa: E731
        p.q, p.k, p.k_new = quarter(p.q), quarter(p.k), quarter(p.k_new)
        k, v = p.appended()
        for b, n in enumerate(lens):                         # every second value is minus the one before
            for j in range(1, n, 2):
                x = -v[p.where(b, j - 1)]
                first = n - p.new[b]
                if j >= first:
                    p.v_new[p.row(b, j - first)] = x
                else:
                    p.v[p.where(b, j)] = x
        check(p, TWO, 0)


def test_one_key_that_takes_nearly_all_in_a_large_launch():
    """The kernel for long chunks with blocks of 32 keys, which launches of more than 512 workgroups take; the key in front of the chunk and within it,
    where some of a tile's rows see it and others do not."""
    lens, new = [420, 350, 400, 351, 410, 420], [350] * 6
    for gap in (14.0, 20.0, 26.0):
        for top in (0, 200):
            p = Paged(83, lens, new, heads=32, kv_heads=32, d=128, page=64)
            p.q[..., 0] = 4.0
            p.q[..., 1:] *= 0.25
            p.k[..., 0] = torch.where(torch.isnan(p.k[..., 0]), p.k[..., 0], 0.0)
            p.k_new[..., 0] = 0.0
            p.v, p.v_new = ((x * 500.0 + 1000.0).to(x.dtype) for x in (p.v, p.v_new))
            for b, (n, m) in enumerate(zip(lens, new)):
                for k, v, at in ((p.k_new, p.v_new, p.row(b, top - n + m)),) if top >= n - m else ((p.k, p.v, p.where(b, top)),):
                    k[at], v[at] = 0.0, 0.0
                    k[at][:, 0] = gap * math.sqrt(128) / 4.0
            check(p, HALF_STEP["fp16"], 128)


@pytest.mark.parametrize("d", [64, 128])
def test_one_key_with_values_of_0_in_some_elements(d):
    """Where a row's largest output is not small, what the long chunks' kernel may lose of the others is below a 64th of half a step of that."""
    for gap in (18.0, 24.0, 30.0):
        p = Paged(84, [1500, 130], [300, 60], heads=8, kv_heads=2, d=d, page=64)
        p.q[..., 0] = 4.0
        p.q[..., 1:] *= 0.25
        p.k[..., 0] = torch.where(torch.isnan(p.k[..., 0]), p.k[..., 0], 0.0)
        p.k_new[..., 0] = 0.0
        p.v, p.v_new = ((x * 500.0 + 1000.0).to(x.dtype) for x in (p.v, p.v_new))
        for b in (0, 1):
            at = p.where(b, 7)
            p.k[at] = 0.0
            p.k[at][:, 0] = gap * math.sqrt(d) / 4.0
            p.v[at][:, ::2] = 0.0
        x = p.device()
        x["cache"].prefill(x["q"], x["k_new"], x["v_new"], x["out"], x["starts"], 300)
        torch.cuda.synchronize()
        out, tol = attend(p, HALF_STEP["fp16"], d)
        paged.close(x["out"], out, tol + 2.0 ** -18 * out.abs().amax(-1, keepdim=True), "out")
