"""Attention to another sequence where scores are -inf: such keys weigh nothing, and a row that has no others gives 0 and lse = -inf, forward and backward, in every way through
the kernels (a unit in one workgroup, two launches, keys split and joined, rows split and added).

Tolerances.  A row's weights P may be off by eP = 2 eS + 2^-15 of themselves (eS = 36 x 2^-24 x 0.18 x sum |q||k| <= 1.5e-5: rows of 32 normal numbers, sum |q||k| below 40; 2^-15: the
other form of the exponent, which a wave takes where one of its rows has no score yet), so out by 2 eP max |v| <= 6e-4 on each of the two sides compared (|v| below 5), lse by eS + eP;
dS is at most P times 30 and |k| below 5, so dq is off by 0.18 x 30 x 5 eP <= 1.7e-3.  bf16 rounds P and out, and dS and dq, half a step of 2^-8 each: 2 x 2^-8 x 5 = 0.04 and
2^-8 (27 + 27) = 0.2 more."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


def run(spa, q, k, v, dout, dtype):
    nq, nk, H, Hk, Dh = q.shape[0], k.shape[0], q.shape[1] // 32, k.shape[1] // 32, 32
    code = spa.SPA_BF16 if dtype == "bf16" else spa.SPA_F32
    sizes, i32 = (1, nq, nk, H, Hk, Dh), lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    ws = [torch.empty(max(f(*sizes, code), 256), dtype=torch.uint8, device="cuda") for f in (spa.spa_cross_attention_workspace_bytes, spa.spa_cross_attention_bwd_workspace_bytes)]
    out, lse = torch.full_like(q, float("nan")), torch.full((H, nq), float("nan"), device="cuda")
    dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, k, v))
    spa.spa_cross_attention(q, k, v, i32(0, nq), i32(0, nk), None, *sizes, out, lse, ws[0])
    spa.spa_cross_attention_bwd(q, k, v, out, dout, lse, i32(0, nq), i32(0, nk), None, *sizes, dq, dk, dv, ws[1])
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(30, 20), (80, 75), (300, 150), (1200, 150), (40, 1500), (3, 5000)])
def test_scores_of_minus_infinity(spa, nq, nk, dtype):
    """Elements 0 and 1 of a row of q are 1 where it meets the lowest numbers of k (two of which overflow a score), else 0.  The first half of the keys holds these: rows that meet them see
    the others alone; with all keys so, those rows see none."""
    g = torch.Generator(device="cuda").manual_seed(nk)
    td = TD[dtype]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k, v, dout = rnd(nq, 64), rnd(nk, 32), rnd(nk, 32), rnd(nq, 64)
    meets = torch.arange(nq, device="cuda") % 3 == 0
    low = -3e38
    q[:, 0:2] = q[:, 32:34] = meets.float()[:, None]                          # (two products of -3e38: past the smallest float)
    k[:, 0:2] = 0
    q, k, v, dout = (t.to(td) for t in (q, k, v, dout))
    half = nk // 2
    masked = k.clone()
    masked[:half, 0:2] = low
    have, all_keys, others = run(spa, q, masked, v, dout, dtype), run(spa, q, k, v, dout, dtype), run(spa, q, k[half:].contiguous(), v[half:].contiguous(), dout, dtype)
    out, lse, dq, dk, dv = have
    bf16 = dtype == "bf16"
    near = lambda a, b, tol: float((a.float() - b.float()).abs().max()) <= tol
    out_tol, lse_tol, dq_tol = 1.2e-3 + 0.04 * bf16, 1e-4, 3.4e-3 + 0.2 * bf16
    # (the same terms, added beside others of 0)
    assert near(out[meets], others[0][meets], out_tol) and near(lse[:, meets], others[1][:, meets], lse_tol)
    assert near(out[~meets], all_keys[0][~meets], out_tol) and near(lse[:, ~meets], all_keys[1][:, ~meets], lse_tol)
    # (in elements 0 and 1 the gradient of the other rows, which do weigh these keys, is a sum of dS times -3e38)
    columns = torch.tensor([c not in (0, 1) for c in range(32)] * 2, device="cuda")
    finite = lambda *ts: all(bool(torch.isfinite(t).all()) for t in ts)
    assert finite(dk, dv, dq[:, columns], dq[meets])
    assert near(dq[meets][:, columns], others[2][meets][:, columns], dq_tol)
    # ---- no key left
    none = k.clone()
    none[:, 0:2] = low
    out, lse, dq, dk, dv = run(spa, q, none, v, dout, dtype)
    assert bool((out[meets] == 0).all()) and bool((lse[:, meets] == float("-inf")).all()) and bool((dq[meets] == 0).all())
    assert near(out[~meets], all_keys[0][~meets], out_tol)
    assert finite(dk, dv, dq[:, columns])
