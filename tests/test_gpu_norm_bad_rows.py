"""Statistics of layer norm for rows that hold an infinity or a NaN."""
import pytest
import torch

from paper_2407_15452_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("columns", [24, 33, 128, 512, 777, 1024, 4096, 8192, 9000, 16383])
def test_both_statistics_of_a_bad_row_are_nan(columns, dtype):
    gen = torch.Generator("cuda").manual_seed(columns)
    x = torch.randn((2, 20, columns), generator=gen, device="cuda").to(dtype)
    clean, clean_stats = B.gs_layer_norm_forward(x)
    bad = {(0, 7): (3, float("inf")), (0, 12): (columns - 1, float("nan")), (1, 0): (columns // 2, float("-inf"))}
    hit = torch.zeros((2, 20), dtype=torch.bool, device="cuda")
    for (b, t), (c, value) in bad.items():
        x[b, t, c] = value
        hit[b, t] = True
    for checkpoint in (False, True):
        y, stats = B.gs_layer_norm_forward(x, checkpoint=checkpoint)[:2]
        # 1 / sqrt(NaN + eps); the mean of an infinity is infinite, and what differs from it NaN
        assert torch.isnan(stats[..., 1][hit]).all() and not torch.isfinite(stats[..., 0][hit]).any() and torch.isnan(y[hit]).all()
        assert torch.equal(y[~hit], clean[~hit]) and torch.equal(stats[~hit], clean_stats[~hit])
