"""The query gradient of short segments, where D from the rounded out would show most.

v of a segment's rows is one row up to a few steps of bf16, so that dP_ij - D_i is as small as the rounding of out, and k one row up to noise
of a quarter, so that sum_j P_ij k_j, which an error of D is multiplied by, is not.  Tolerance of dq: each dS is off by 2 E of itself (E as in
test_gpu_attention_bias.py), by P times what dP and D are off by as sums in fp32, (Dh + 4 + n) U of their magnitudes, and in bf16 by
half a step as an operand; and half a step of the result.  Nothing of the rounding of out."""
import math

import pytest
import torch

from test_gpu_attention_bias import HALF, U, Case, spa  # noqa: F401 (spa: the fixture)


def alike(lens, Dh, dtype, seed=0):
    c = Case(lens, (9, 10), 2, Dh, dtype, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    C, td, at = c.C, c.qkv.dtype, 0
    for n in c.lens:
        base = 1 + torch.rand(2 * C, generator=g)
        k = base[:C] + 0.25 * torch.randn(n, C, generator=g)
        v = base[C:] + 2.0 ** -7 * torch.randint(-2, 3, (n, C), generator=g)
        c.qkv[at:at + n, C:] = torch.cat([k, v], 1).to(td)
        at += n
    return c


def dq_of(c):
    H, Dh, C, (gh, gw) = c.H, c.Dh, c.C, c.grid
    half = HALF[c.dtype]
    hp, scale, at = half if c.dtype == "bf16" else 0.0, 1 / math.sqrt(Dh), 0
    want, tol = torch.zeros(c.T, C, dtype=torch.float64), torch.zeros(c.T, C, dtype=torch.float64)
    for n in c.lens:
        j = slice(at, at + n)
        at += n
        r, x = c.pos[j] // gw, c.pos[j] % gw
        o = (r[:, None] - r[None] + gh - 1) * (2 * gw - 1) + x[:, None] - x[None] + gw - 1
        for h in range(H):
            col = slice(h * Dh, (h + 1) * Dh)
            q, k, v = (c.qkv[j, i * C:(i + 1) * C][:, col].double() for i in range(3))
            dO, bias = c.dout[j, col].double(), c.table[h].double()[o]
            P = torch.softmax(q @ k.T * scale + bias, 1)
            E = U * (2 * (Dh + 4) * (q.abs() @ k.abs().T * scale + bias.abs()).amax(1, keepdim=True) + 16 + n / 8)
            dP, mag = dO @ v.T, dO.abs() @ v.abs().T
            dS = P * (dP - (P * dP).sum(1, keepdim=True))
            off = (Dh + 4 + n) * U * (mag + (P * mag).sum(1, keepdim=True)) + 2 * E * (dP.abs() + (P * dP.abs()).sum(1, keepdim=True))
            want[j, col] = dS @ k * scale
            tol[j, col] = ((hp + 2 * E) * dS.abs() + P * off) @ k.abs() * scale + half * want[j, col].abs() + 1e-30
    return want, tol


LENS = {"few": [1, 2, 3, 4, 5, 7, 8], "more": [9, 13, 16, 17, 24], "most": [31, 32, 30, 1]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("name", list(LENS))
def test_dq_of_short_segments(spa, name, Dh, dtype):  # noqa: F811
    c = alike(LENS[name], Dh, dtype)
    want, tol = dq_of(c)
    off = (c.run(spa)["dq"][:c.T].cpu().double() - want).abs()
    assert bool((off <= tol).all()), f"worst {float((off / tol).max()):.3g} of the tolerance"
