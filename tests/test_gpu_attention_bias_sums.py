"""The sums of dS by offset where they are longest."""
import pytest
import torch

from test_gpu_attention_bias import U, spa  # noqa: F401 (spa: the fixture)

pytestmark = pytest.mark.gpu


def test_many_pairs_at_one_offset(spa):  # noqa: F811
    """16 images of 4096 rows, all at the first two places of the map, half at either: 2^23 pairs of an image at offset 0, whose dS are
    equal.  q and the table are 0, v is +1.875 for rows at the first place and -1.875 at the other, dout +1 and -1: P = 1/n, out = 0,
    dP = +-60, dS = +-60 / n.  With E = U (16 + n / 8) P is off by E of itself (as in test_gpu_attention_bias.py), each dS by 2 E, and
    what its row's then add up to is taken off again: 2 E more."""
    H, Dh, n, B, grid = 64, 32, 4096, 16, (64, 64)
    C, T, nb = H * Dh, n * B, 127 * 127
    first = (torch.arange(n, device="cuda") < n // 2).repeat(B)
    sign = torch.where(first, 1.0, -1.0).bfloat16()[:, None]
    qkv = torch.zeros(T, 3 * C, dtype=torch.bfloat16, device="cuda")
    qkv[:, 2 * C:] = 1.875 * sign
    q, k, v = (qkv[:, i * C:(i + 1) * C] for i in range(3))
    dout = sign.expand(T, C).contiguous()
    cu = torch.arange(0, T + 1, n, dtype=torch.int32, device="cuda")
    at = ((~first).int() + grid[0] * grid[1] * torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(n)).int()
    table = torch.zeros(H, nb, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty(T, C, dtype=torch.bfloat16, device="cuda"), torch.empty(H, T, device="cuda")
    args = (cu, at, table, None, grid, B, n, H, Dh)
    spa.spa_packed_attention_bias(q, k, v, *args, out, lse)
    dqkv, d_table = torch.empty_like(qkv), torch.empty(H, nb, device="cuda")
    dq, dk, dv = (dqkv[:, i * C:(i + 1) * C] for i in range(3))
    ws = torch.empty(spa.spa_attention_bias_bwd_workspace_bytes(B, n, H, Dh, *grid, spa.SPA_BF16), dtype=torch.uint8, device="cuda")
    spa.spa_packed_attention_bias_bwd(q, k, v, out, dout, lse, *args, dq, dk, dv, d_table, ws)
    want = torch.zeros(nb, dtype=torch.float64)
    centre = 63 * 127 + 63
    want[centre], want[centre - 1], want[centre + 1] = B * n / 2 * 60, -B * n / 4 * 60, -B * n / 4 * 60
    off = (d_table.cpu().double() - want).abs()
    tol = 4 * U * (16 + n / 8) * want.abs()
    assert bool((off <= tol).all()), (float(off.max()), d_table[0, centre - 1:centre + 2].tolist())
