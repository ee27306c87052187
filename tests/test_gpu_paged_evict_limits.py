"""wkv_paged_evict at the largest sizes that its documentation allows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paged import Paged


@pytest.mark.parametrize("missing", [(), [(0, 1)]])
def test_the_largest_budget(missing):
    """2^31 - 1 entries of `kept`, of which the sequence fills the first: all others are -1."""
    budget = 2 ** 31 - 1
    p = Paged(91, [40], heads=1, kv_heads=1, d=64, scores=True, missing=missing)
    x = p.device()
    kept = torch.full((1, 1, budget), 5, dtype=torch.int32, device="cuda")
    new_lens = torch.zeros_like(x["lens"])
    x["cache"].evict(budget, 7, new_lens, x["scores"], kept)
    torch.cuda.synchronize()
    n = 0 if missing else 40
    assert new_lens.tolist() == [40] and torch.equal(kept[0, 0, :n].cpu(), torch.arange(n, dtype=torch.int32))
    for lo in range(n, budget, 1 << 28):
        assert bool((kept[0, 0, lo: lo + (1 << 28)] == -1).all())
    assert torch.equal(x["scores"].cpu(), p.scores)
