"""Sums of weights where a row has no finite ones: they reach the slots that the row sees, and no others."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paged import Paged, run

GONE = [(0, 1), (0, 3), (1, 0), (2, 2)]


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("fp16", 128), ("bf16", 64), ("bf16", 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("window,sink,missing", [(0, 0, GONE), (21, 3, ()), (21, 3, GONE), (50, 0, GONE)])
def test_slots_that_a_row_without_finite_weights_does_not_see(dtype, d, bad, window, sink, missing):
    for lens, new in (([90, 40, 150], None), ([90, 40, 150], [1, 2, 1]), ([90, 40, 150], [60, 40, 70])):
        p = Paged(95, lens, new, heads=4, kv_heads=2, d=d, dtype=dtype, window=window, sink=sink, scores=True, missing=missing)
        last = p.row(0, p.new[0] - 1)
        p.q[last, 1] = bad
        p.q[p.row(2, 0), 2, 5] = bad
        run(p)
