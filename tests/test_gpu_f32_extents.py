"""fp32 projections of as many rows and columns as an int counts: every element is there, and nothing past the live rows.

A row is one of seven given through an index, so its result is known from a call on those seven: the same bits (an element is one chain over the contraction, whatever its tile).
Other operands hold small whole numbers, whose sums are exact in any order."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1
CHUNK = 1 << 27


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    yield mod
    torch.cuda.empty_cache()


@pytest.fixture(scope="module")
def seven():
    """Row j is row j % 7 of seven."""
    return torch.arange(MOST, dtype=torch.int32, device="cuda").remainder_(7)


def _rows(out, idx, table, live):
    for a in range(0, live, CHUNK):
        b = min(a + CHUNK, live)
        assert torch.equal(out[a:b], table[idx[a:b].long()]), (a, b)
    assert bool(torch.isnan(out[live:]).all())


@pytest.mark.parametrize("live", [MOST, MOST - 40])
def test_forward_rows(spa, seven, live):
    g = torch.Generator(device="cuda").manual_seed(0)
    x, W, b = (torch.randn(*s, generator=g, device="cuda") for s in ((7, 64), (2, 64), (2,)))
    table, out = torch.empty(7, 2, device="cuda"), torch.full((MOST, 2), float("nan"), device="cuda")
    spa.spa_linear_packed(x, None, None, None, W, b, table)
    total = None if live == MOST else torch.tensor([live], dtype=torch.int32, device="cuda")
    spa.spa_linear_packed(x, seven, None, total, W, b, out)
    _rows(out, seven, table, live)


@pytest.mark.parametrize("live", [MOST, MOST - 40])
def test_input_side_rows(spa, seven, live):
    g = torch.Generator(device="cuda").manual_seed(1)
    d, W = (torch.randn(*s, generator=g, device="cuda") for s in ((7, 64), (64, 2)))
    table, dx = torch.empty(7, 2, device="cuda"), torch.full((MOST, 2), float("nan"), device="cuda")
    spa.spa_linear_packed_bwd_input(d, None, None, W, 7, None, None, table)
    total = None if live == MOST else torch.tensor([live], dtype=torch.int32, device="cuda")
    spa.spa_linear_packed_bwd_input(d, seven, total, W, MOST, None, None, dx)
    _rows(dx, seven, table, live)


def _whole(shape, n, seed):
    return (torch.arange(n, dtype=torch.int32, device="cuda").add_(seed).remainder_(5)).view(shape).float()


def test_columns(spa):
    """Forward and weight side with as many columns of the result."""
    x = torch.tensor([[1.0, -2.0, 3.0]], device="cuda")
    row = _whole((MOST, 1), MOST, 0)
    W = torch.cat((row, row + 1, row - 2), 1)
    out = torch.full((1, MOST), float("nan"), device="cuda")
    spa.spa_linear_packed(x, None, None, None, W, None, out)
    for a in range(0, MOST, CHUNK):
        w = W[a:a + CHUNK]
        assert torch.equal(out[0, a:a + CHUNK], w[:, 0] - 2 * w[:, 1] + 3 * w[:, 2]), a
    del W, row
    d = torch.stack((_whole(MOST, MOST, 1), _whole(MOST, MOST, 3)))
    xr = torch.tensor([[2.0], [-1.0]], device="cuda")
    dW, db = torch.full((MOST, 1), float("nan"), device="cuda"), torch.full((MOST,), float("nan"), device="cuda")
    spa.spa_linear_packed_bwd_weight(d, None, xr, None, None, None, 2, dW, db)
    for a in range(0, MOST, CHUNK):
        b = min(a + CHUNK, MOST)
        assert torch.equal(dW[a:b, 0], 2 * d[0, a:b] - d[1, a:b]) and torch.equal(db[a:b], d[0, a:b] + d[1, a:b]), a
