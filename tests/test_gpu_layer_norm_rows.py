"""Layer norm's rows in full: statistics of rows with Inf and NaN."""
import pytest
import torch

from paper_2112_10769_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [5, 64, 300, 1000, 1024, 4096, 9001, 40000])
def test_the_statistics_of_rows_with_inf_and_nan_are_the_formulas(ctx, cols, dtype):
    # mean: Inf with its sign, NaN for NaN or for both infinities; rstd: NaN, for the variance is
    x = torch.randn(7, cols, device="cuda").to(dtype)
    clean = ctx.layer_norm(x)
    x[1, 2], x[3, cols - 1], x[4, 0], x[5, 1], x[5, cols - 1] = float("inf"), float("nan"), -float("inf"), float("inf"), -float("inf")
    y, mean, rstd = ctx.layer_norm(x)
    for got, before in zip((y, mean, rstd), clean):
        assert torch.equal(got[[0, 2, 6]], before[[0, 2, 6]])
    bad = [1, 3, 4, 5]
    assert torch.isnan(y[bad]).all() and torch.isnan(rstd[bad]).all()
    assert mean[1] == float("inf") and mean[4] == -float("inf") and torch.isnan(mean[[3, 5]]).all()
