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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_next_to_the_largest_number(spa, dtype):  # noqa: F811
    """Two rows, q = k = 0, v = +1 and -1 and dout = 1.25 x 2^127 in one column: P = 1/2 (off by U (16 + 2 / 8) of itself), out = D = 0, and
    dS = +-1.25 x 2^126 is finite: +- that at the offsets of the one row from the other, 0 at the middle."""
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    Dh, x = 32, 1.25 * 2.0 ** 126
    qkv = torch.zeros(2, 3 * Dh, dtype=td, device="cuda")
    qkv[0, 2 * Dh], qkv[1, 2 * Dh] = 1, -1
    q, k, v = (qkv[:, i * Dh:(i + 1) * Dh] for i in range(3))
    dout = torch.zeros(2, Dh, dtype=td, device="cuda")
    dout[:, 0] = 2 * x
    args = (torch.tensor([0, 2], dtype=torch.int32, device="cuda"), None, torch.zeros(1, 3, dtype=td, device="cuda"), None, (1, 2), 1, 2, 1, Dh)
    out, lse, dqkv = torch.empty_like(dout), torch.empty(1, 2, device="cuda"), torch.empty_like(qkv)
    spa.spa_packed_attention_bias(q, k, v, *args, out, lse)
    d_table = torch.empty(1, 3, device="cuda")
    code = spa.SPA_BF16 if dtype == "bf16" else spa.SPA_F32
    ws = torch.empty(spa.spa_attention_bias_bwd_workspace_bytes(1, 2, 1, Dh, 1, 2, code), dtype=torch.uint8, device="cuda")
    spa.spa_packed_attention_bias_bwd(q, k, v, out, dout, lse, *args, *(dqkv[:, i * Dh:(i + 1) * Dh] for i in range(3)), d_table, ws)
    # o = column of the query - column of the key + 1: query 0 and key 1 (dS = P (dP - D) = -x), one and the same, query 1 and key 0
    want = torch.tensor([-x, 0.0, x], dtype=torch.float64)
    assert bool(((d_table[0].cpu().double() - want).abs() <= 4 * U * 17 * x).all()), d_table.tolist()
