"""Merging of gathered partials: a log-sum-exp that is no number makes its row NaN, whatever values stand beside it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 5])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_partial_without_a_weight_makes_its_row_nan(n, bad):
    from paper_2509_21081_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(n)
    B, H = 6, 16
    o = torch.randn(n, B, H, 128, generator=g, device="cuda")
    lse = torch.randn(n, B, H, generator=g, device="cuda")
    clean, clean_lse = torch.empty(B, H, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, device="cuda")
    b.typhoon_mla_combine_partials(o, lse, clean, clean_lse)
    hit = torch.zeros(B, H, dtype=torch.bool, device="cuda")
    for i, (r, h) in enumerate([(0, 0), (2, 15), (5, 7)]):
        lse[i % n, r, h] = bad
        hit[r, h] = True
    if n > 1:
        lse[1, 5, 7], lse[0, 5, 7] = bad, float("-inf")        # beside an empty partial
    out, got_lse = torch.empty_like(clean), torch.empty_like(clean_lse)
    b.typhoon_mla_combine_partials(o, lse, out, got_lse)
    assert torch.isnan(out[hit]).all() and torch.isnan(got_lse[hit]).all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(got_lse[~hit], clean_lse[~hit])
