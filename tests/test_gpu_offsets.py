"""Norms and attention with a position bias where elements lie past 2^31: tokens and packed rows by the million, the last ones looked at.

Against plain fp32 arithmetic on the device, rounded to bf16: both sides are off by half a step (2^-8) and by what the sums in fp32 are, far
below a step: 2^-7 of the value and 2^-9 of the row's largest beside it for values that cancel."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


def near(got, want):
    got, want = got.float(), want.float()
    tol = 2.0 ** -7 * want.abs() + 2.0 ** -9 * want.abs().amax(1, keepdim=True) + 1e-30
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


def test_norms_past_2_31_elements(spa):
    C, rows = 1024, 2 ** 21 + 777                             # 2^31 elements and some
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, da = torch.randn(rows, C, generator=g, **bf), torch.randn(rows, C, generator=g, **bf)
    gamma, beta = (torch.randn(C, generator=g, **bf) for _ in range(2))
    scores = torch.randn(rows, generator=g, device="cuda")
    index = torch.arange(rows, dtype=torch.int32, device="cuda")
    total = torch.tensor([rows], dtype=torch.int32, device="cuda")
    packed, stats = torch.empty(rows, C, **bf), torch.empty(2, rows, device="cuda")
    spa.spa_norm_packed(x, index, total, gamma, beta, spa.SPA_NORM_LAYER, 1e-6, packed, stats)
    some = torch.cat([torch.arange(5), torch.arange(rows - 900, rows)]).cuda()
    xs, ds, gm, bt = x[some].float(), da[some].float(), gamma.float(), beta.float()
    mu = xs.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((xs - mu) ** 2).mean(1, keepdim=True) + 1e-6)
    xh = (xs - mu) * r
    near(packed[some], xh * gm + bt)
    dx = packed                                                # (written anew)
    ws = torch.empty(spa.spa_norm_bwd_workspace_bytes(rows, C, spa.SPA_BF16), dtype=torch.uint8, device="cuda")
    spa.spa_norm_packed_bwd(da, x, index, total, gamma, spa.SPA_NORM_LAYER, stats, None, dx, None, None, ws)
    gg = ds * gm
    near(dx[some], r * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True)))
    y = dx
    spa.spa_norm_residual_unpack(x, index, da, gamma, beta, None, scores, spa.SPA_NORM_LAYER, 1e-6, y, stats)
    p = torch.sigmoid(scores[some])[:, None]
    near(y[some], ds + p * (xh * gm + bt))
    dz = y
    spa.spa_norm_residual_unpack_bwd(da, x, index, index, total, gamma, beta, None, scores, spa.SPA_NORM_LAYER, stats, dz, None, None, None,
                                     None, ws)
    near(dz[some], p * r * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True)))


def test_attention_past_2_31_elements(spa):
    """Segments of 40 rows, the last ones past 2^31 elements of a buffer of q | k | v rows."""
    H, Dh, n, grid = 8, 64, 40, (8, 8)
    C, B = H * Dh, 36000
    rows = B * n                                               # x 3 C: 2.2e9 elements
    g = torch.Generator(device="cuda").manual_seed(2)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    qkv, dout = torch.randn(rows, 3 * C, generator=g, **bf), torch.randn(rows, C, generator=g, **bf)
    q, k, v = (qkv[:, i * C:(i + 1) * C] for i in range(3))
    table = torch.randn(H, 225, generator=g, **bf)
    cu = torch.arange(0, rows + 1, n, dtype=torch.int32, device="cuda")
    place = torch.randperm(64, generator=g, device="cuda")[:n].sort()[0].int()
    at = (place + 64 * torch.arange(B, dtype=torch.int32, device="cuda")[:, None]).view(-1)
    out, lse = torch.empty(rows, C, **bf), torch.empty(H, rows, device="cuda")
    args = (cu, at, table, None, grid, B, n, H, Dh)
    spa.spa_packed_attention_bias(q, k, v, *args, out, lse)
    dqkv, d_table = torch.empty_like(qkv), torch.empty(H, 225, device="cuda")
    dq, dk, dv = (dqkv[:, i * C:(i + 1) * C] for i in range(3))
    ws = torch.empty(spa.spa_attention_bias_bwd_workspace_bytes(B, n, H, Dh, *grid, spa.SPA_BF16), dtype=torch.uint8, device="cuda")
    spa.spa_packed_attention_bias_bwd(q, k, v, out, dout, lse, *args, dq, dk, dv, d_table, ws)
    r, c = place.long() // 8, place.long() % 8
    bias = table.float()[:, (r[:, None] - r[None] + 7) * 15 + c[:, None] - c[None] + 7]
    for b in (0, 1, B - 2, B - 1):
        j = slice(b * n, (b + 1) * n)
        heads = lambda t: t[j].float().view(n, H, Dh).transpose(0, 1).contiguous()
        Q, K, V, dO = heads(q), heads(k), heads(v), heads(dout)
        P = torch.softmax(torch.matmul(Q, K.transpose(1, 2).contiguous()) / math.sqrt(Dh) + bias, -1)
        dP = torch.matmul(dO, V.transpose(1, 2).contiguous())
        dS = P * (dP - (P * dP).sum(-1, keepdim=True))
        flat = lambda t: t.transpose(0, 1).reshape(n, C)
        want = dict(out=torch.matmul(P, V), dq=torch.matmul(dS, K) / math.sqrt(Dh), dk=torch.matmul(dS.transpose(1, 2).contiguous(), Q) / math.sqrt(Dh),
                    dv=torch.matmul(P.transpose(1, 2).contiguous(), dO))
        for name, t in dict(out=out, dq=dq, dk=dk, dv=dv).items():
            got, ref = t[j].float(), flat(want[name])
            # (P, dS and the result rounded to bf16, D from the rounded out: four roundings of 2^-8 at most, added up without cancelling)
            assert float((got - ref).norm()) <= 4 * 2.0 ** -8 * float(ref.norm()), (name, b)
    assert bool(torch.isfinite(d_table).all())
