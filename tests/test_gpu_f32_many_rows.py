"""The fp32 weight side over many rows: chains of 1024, added up in order.

Every addend is 1 + 2^-10.  1024 of them are 1025, and every sum on the way below 2048 has a last place of 2^-13 or less: exact.  Sums of 1025 are whole numbers below 2^24: exact.  So the
result is off by the rounding of what the last, partial chain adds: half a last place.  (One chain over all rows loses 2^-10 with every row past 2^15.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

ONE = 1 + 2.0 ** -10


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


def weight(spa, d, x, M, total=None, d_idx=None, x_idx=None, gate=None):
    dW, db = torch.full((d.shape[1], x.shape[1]), float("nan"), device="cuda"), torch.full((d.shape[1],), float("nan"), device="cuda")
    spa.spa_linear_packed_bwd_weight(d, d_idx, x, x_idx, gate, total, M, dW, db)
    return dW, db


@pytest.mark.parametrize("M", [1023, 1024, 1025, 2048, 33000, 66745, 200000])
@pytest.mark.parametrize("n_out,K", [(8, 40), (1000, 900)])
def test_sums_that_are_exact(spa, M, n_out, K):
    d, x = torch.full((M, n_out), ONE, device="cuda"), torch.ones(M, K, device="cuda")
    dW, db = weight(spa, d, x, M)
    want = M * ONE
    half = 2.0 ** -24 * want
    assert float((dW.double() - want).abs().max()) <= half and float((db.double() - want).abs().max()) <= half
    # (through indices, the live rows counted on the device)
    live = M - 1
    idx = torch.randperm(M, generator=torch.Generator().manual_seed(M)).to(torch.int32).cuda()
    dW, db = weight(spa, d, x, M, torch.tensor([live], dtype=torch.int32, device="cuda"), idx, idx)
    want = live * ONE
    assert float((dW.double() - want).abs().max()) <= half and float((db.double() - want).abs().max()) <= half


@pytest.mark.parametrize("M", [700, 1024, 1100, 5000])
@pytest.mark.parametrize("gated", [False, True])
def test_the_same_bits_in_any_tile(spa, M, gated):
    """A few rows and columns alone, in small tiles, and inside a result that takes the large ones."""
    g = torch.Generator(device="cuda").manual_seed(M)
    d, x = torch.randn(M, 1000, generator=g, device="cuda"), torch.randn(M, 900, generator=g, device="cuda")
    idx = torch.arange(M, dtype=torch.int32, device="cuda")
    gate = torch.randn(M, generator=g, device="cuda") if gated else None
    large = weight(spa, d, x, M, None, idx, idx, gate)
    small = weight(spa, d[:, :70], x[:, :33].contiguous(), M, None, idx, idx, gate)
    assert torch.equal(small[0].view(torch.int32), large[0][:70, :33].contiguous().view(torch.int32))
    assert torch.equal(small[1].view(torch.int32), large[1][:70].view(torch.int32))


def test_one_chain_up_to_1024_rows(spa):
    """With 2^24 in the first row every one of the others is lost, as in one chain; past 1024 rows those behind them are kept together."""
    for M, kept in ((1024, 0), (1025, 0), (2048, 1024), (3000, 1976)):
        d = torch.ones(M, 40, device="cuda")
        d[0] = 2.0 ** 24
        dW, db = weight(spa, d, torch.ones(M, 50, device="cuda"), M)
        assert bool((dW == 2.0 ** 24 + kept).all()) and bool((db == 2.0 ** 24 + kept).all()), M
