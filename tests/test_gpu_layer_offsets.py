"""The operators of a layer on rows whose last ones lie past 2^31 elements, every tensor with a row stride of its own: the bits of the same call on rows close together.

Of the attention each way through the kernels: a unit in one workgroup, two launches, keys split and joined, rows split and added, bf16 and fp32."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    yield mod
    torch.cuda.empty_cache()


def wide(t):
    """t's rows so far apart that the last lies past 2^31 elements."""
    rows, width = t.shape
    stride = max(width, (2 ** 31 // (rows - 1) + 64) // 64 * 64)
    out = torch.empty(rows * stride, dtype=t.dtype, device="cuda").view(rows, stride)[:, :width]
    assert (rows - 1) * stride >= 2 ** 31 and stride < 2 ** 31
    out.copy_(t)
    return out


def far(t):
    return wide(torch.full_like(t, float("nan")))


def i32(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,G", [(80, 75, 1), (90, 60, 2), (300, 150, 2), (600, 150, 2), (40, 1500, 3), (3, 5000, 4)])
def test_attention(spa, nq, nk, G, dtype):
    g = torch.Generator(device="cuda").manual_seed(nq)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TD[dtype])
    Hk, Dh = 1, 32
    H, code = G * Hk, spa.SPA_BF16 if dtype == "bf16" else spa.SPA_F32
    sizes = (1, nq, nk, H, Hk, Dh)
    cu_q, cu_k = i32(0, nq), i32(0, nk)
    bytes_of = lambda f: torch.empty(max(f(*sizes, code), 256), dtype=torch.uint8, device="cuda")
    ws, ws_bwd = bytes_of(spa.spa_cross_attention_workspace_bytes), bytes_of(spa.spa_cross_attention_bwd_workspace_bytes)
    q, kv, dout = rnd(nq, H * Dh), rnd(nk, 2 * Hk * Dh), rnd(nq, H * Dh)
    split = lambda t: (t[:, :Hk * Dh], t[:, Hk * Dh:])
    results = []
    for q_, kv_, dq, dkv in ((q, kv, torch.empty_like(q), torch.empty_like(kv)), (wide(q), wide(kv), far(q), far(kv))):
        out, lse = torch.full_like(q, float("nan")), torch.full((H, nq), float("nan"), device="cuda")
        spa.spa_cross_attention(q_, *split(kv_), cu_q, cu_k, None, *sizes, out, lse, ws)
        spa.spa_cross_attention_bwd(q_, *split(kv_), out, dout, lse, cu_q, cu_k, None, *sizes, dq, *split(dkv), ws_bwd)
        results.append([t.contiguous().clone() for t in (out, lse, dq, dkv)])
    for close, apart in zip(*results):
        assert bool(torch.isfinite(close).all()) and torch.equal(close, apart)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
def test_rotation(spa, layout, dtype):
    g = torch.Generator(device="cuda").manual_seed(layout)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TD[dtype])
    M, H, Hk, Dh, grid, pairs = 130, 3, 1, 32, (1, 15, 12), (0, 8)
    code = spa.SPA_BF16 if dtype == "bf16" else spa.SPA_F32
    idx = torch.randperm(180, generator=g, device="cuda")[:M].int()
    table, total = spa.rotary_table(grid, Dh, pairs).cuda(), i32(M)
    gammas = [rnd(Dh) for _ in range(4)]
    q, k, dqo, dko = rnd(M, H * Dh), rnd(M, Hk * Dh), rnd(M, H * Dh), rnd(M, Hk * Dh)
    ws = torch.empty(spa.spa_qk_norm_rotary_bwd_workspace_bytes(M, H, Hk, Dh, code), dtype=torch.uint8, device="cuda")
    results = []
    for place, empty in ((lambda t: t, torch.empty_like), (wide, far)):
        qo, ko, dq, dk = empty(q), empty(k), empty(q), empty(k)
        grads = [torch.empty(Dh, device="cuda") for _ in range(4)]
        q_, k_ = place(q), place(k)
        spa.spa_qk_norm_rotary(q_, k_, idx, total, *gammas, spa.SPA_NORM_LAYER, 1e-6, table, pairs, grid, H, Hk, Dh, qo, ko, layout)
        spa.spa_qk_norm_rotary_bwd(place(dqo), place(dko), q_, k_, idx, total, gammas[0], gammas[2], spa.SPA_NORM_LAYER, 1e-6, table, pairs, grid, H, Hk, Dh, dq, dk,
                                   *grads, ws, layout)
        results.append([t.contiguous().clone() for t in (qo, ko, dq, dk, *grads)])
    for close, apart in zip(*results):
        assert bool(torch.isfinite(close).all()) and torch.equal(close, apart)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("indexed", [False, True])
def test_gated_block_backward(spa, indexed, dtype):
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TD[dtype])
    M, N_out, F = 150, 64, 96
    dy, W_down, pre = rnd(M, N_out), rnd(N_out, F), rnd(M, 2 * F)
    idx = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda") if indexed else None
    results = []
    for dy_ in (dy, wide(dy)):
        d_pre = torch.full_like(pre, float("nan"))
        spa.spa_gated_linear_packed_bwd(dy_, idx, None, W_down, pre, spa.SPA_ACT_SILU, d_pre)
        results.append(d_pre)
    assert bool(torch.isfinite(results[0]).all()) and torch.equal(*results)
