"""The gated feed-forward block: both projections, the activation and their product in one kernel, and its backward, against a plain 64-bit form.

Tolerances.  half: half a step of the tensors' type, relative (2^-8 bf16, 2^-24 fp32).  A projection is off by eg = (K + 4) 2^-24 sum |x||w|, |act'| <= 1.13; the activation and its slope
themselves by 2^-20 (1 + |g|) of 1 + |g| where they are formed with the fast exponential and reciprocal (a few 2^-23 each; its argument is off by 2^-24 |g|), and Phi by 7.5e-8 (bf16) beside it.
  pre: eg + half |pre|;   h: |u| (1.13 eg + e_act) + |act| eu + half |h|
  dh: eh = (N_out + 4) 2^-24 sum |dy||W_down|;   d_g: |u| (|slope| eh + |dh| e_slope) + half |d_g|;   d_u: |act| eh + |dh| e_act + half |d_u|"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


def act64(g, act):
    if act == 0:
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = torch.special.ndtr(g)
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / (2 * np.pi) ** 0.5


class Case:
    def __init__(self, M, K, F, act=0, dtype="bf16", live=None, index=False, counted=True, bias=True, N_out=None, seed=0, size=1.0, tokens=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        self.M, self.K, self.F, self.act, self.live = M, K, F, act, M if live is None else live
        self.N_out, tokens = N_out or K, tokens or (2 * M if index else M)
        self.idx = torch.randperm(tokens, generator=g, device="cuda")[:M].int() if index else None
        self.total = torch.tensor([self.live], dtype=torch.int32, device="cuda") if counted else None
        self.x, self.dy = (size * rnd(tokens, K)).to(self.td), rnd(tokens, self.N_out).to(self.td)
        self.W, self.W_down = (rnd(2 * F, K) / K ** 0.5).to(self.td), (rnd(self.N_out, F) / F ** 0.5).to(self.td)
        self.b = (0.3 * rnd(2 * F)).to(self.td) if bias else None

    def run(self, spa, keep=True):
        nan = lambda *s: torch.full(s, float("nan"), dtype=self.td, device="cuda")
        h, pre = nan(self.M, self.F), nan(self.M, 2 * self.F) if keep else None
        spa.spa_gated_linear_packed(self.x, self.idx, self.total, self.W, self.b, self.act, h, pre)
        res = dict(h=h)
        if keep:
            d_pre = nan(self.M, 2 * self.F)
            spa.spa_gated_linear_packed_bwd(self.dy, self.idx, self.total, self.W_down, pre, self.act, d_pre)
            res.update(pre=pre, d_pre=d_pre)
        return res

    def check(self, res):
        T, F, half = self.live, self.F, self.half
        rows = lambda t: (t if self.idx is None else t[self.idx.long()])[:T].double()
        mul = lambda a, b: torch.matmul(a, b.contiguous())

        def near(name, have, want, tol):
            err = (have[:T].double() - want).abs()
            assert bool((err <= tol).all()), (name, float((err - tol).max()))
            assert bool(torch.isnan(have[T:].float()).all()), name

        x, W = rows(self.x), self.W.double()
        pre = mul(x, W.T)
        eg = (self.K + 4) * U * mul(x.abs(), W.abs().T)
        if self.b is not None:
            pre = pre + self.b.double()
            eg = eg + 2 * U * (self.b.double().abs() + pre.abs())
        g, u = pre[:, :F], pre[:, F:]
        a, _ = act64(g, self.act)
        e_act = lambda v: 2.0 ** -20 * (1 + v.abs()) ** 2 + (7.5e-8 * (1 + v.abs()) if self.act else 0.0)
        want = a * u
        near("h", res["h"], want, u.abs() * (1.13 * eg[:, :F] + e_act(g)) + a.abs() * eg[:, F:] + 2 * eg[:, :F] * eg[:, F:] + half * want.abs())
        if "pre" not in res:
            return
        near("pre", res["pre"], pre, eg + half * pre.abs())
        g, u = res["pre"][:T, :F].double(), res["pre"][:T, F:].double()
        a, slope = act64(g, self.act)
        dy, Wd = rows(self.dy), self.W_down.double()
        dh, eh = mul(dy, Wd), (self.N_out + 4) * U * mul(dy.abs(), Wd.abs())
        want = dh * u * slope
        near("d_g", res["d_pre"][:, :F], want, u.abs() * (slope.abs() * eh + (dh.abs() + eh) * e_act(g)) + half * want.abs())
        want = dh * a
        near("d_u", res["d_pre"][:, F:], want, a.abs() * eh + (dh.abs() + eh) * e_act(g) + half * want.abs())


BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
ACTS = pytest.mark.parametrize("act", [0, 1])


@BOTH
@ACTS
@pytest.mark.parametrize("M,K,F", [(1, 8, 8), (1, 384, 200), (3, 64, 176), (31, 72, 8), (33, 40, 56), (127, 64, 64), (128, 128, 128), (129, 136, 136), (200, 384, 200), (257, 520, 72)])
def test_small(spa, dtype, act, M, K, F):
    c = Case(M, K, F, act, dtype, seed=M)
    c.check(c.run(spa))


# (rows, contraction, F) of every shape of tile, of the forward (2 F columns) and of the backward (F): eight waves and four steps, two workgroups a unit, 192 x 192, 256 x 256 with
# 256 x 192 behind it, either alone
SHAPES = [(200, 384, 200), (3000, 512, 1000), (1600, 256, 1904), (3000, 512, 1504), (6272, 768, 2048), (2000, 512, 3000), (6272, 768, 1024), (3000, 512, 2000), (6272, 768, 4096),
          (2000, 512, 6000), (9000, 64, 504)]


@ACTS
@pytest.mark.parametrize("M,K,F", SHAPES)
def test_shapes(spa, act, M, K, F):
    c = Case(M, K, F, act, seed=F)
    c.check(c.run(spa))


@pytest.mark.parametrize("tiles", ["2", "14"])
@pytest.mark.parametrize("M,K,F", [(40, 64, 72), (700, 200, 328), (6272, 128, 1024)])
def test_tiles_by_option(spa, tiles, M, K, F):
    """The option of the projections' tiles holds here too: 128 x 128, or the large ones, where the rule would not take them."""
    c = Case(M, K, F, seed=3)
    spa.spa_set_option("gemm_tm", tiles)
    try:
        c.check(c.run(spa))
    finally:
        spa.spa_set_option("gemm_tm")


@pytest.mark.parametrize("M,K,F,live", [(1, 64, 72, 1), (98, 384, 1024, 98), (196, 1024, 384, 101), (300, 72, 520, 300), (900, 200, 104, 640)])
def test_small_tiles_keep_the_bits(spa, M, K, F, live):
    """Few rows take small tiles: the block, and the projection of its result back onto the residual stream, with the bits of the 128 x 128 tiles."""
    c = Case(M, K, F, live=live, index=True, tokens=M + 60)

    def run():
        res = c.run(spa)
        inv = torch.full((M + 60,), -1, dtype=torch.int32, device="cuda")
        inv[c.idx[:live].long()] = torch.arange(live, dtype=torch.int32, device="cuda")
        y = torch.full((1, M + 60, K), float("nan"), dtype=torch.bfloat16, device="cuda")
        spa.spa_linear_packed_unpack(res["h"], c.total, c.W_down, None, c.idx, inv, c.x.view(1, M + 60, K), y)
        return dict(res, y=y)

    got = run()
    c.check({n: got[n] for n in ("h", "pre", "d_pre")})
    spa.spa_set_option("gemm_tm", "2")
    try:
        want = run()
    finally:
        spa.spa_set_option("gemm_tm")
    for n in got:
        rows = slice(None) if n == "y" else slice(0, live)
        assert torch.equal(got[n][rows], want[n][rows]), n
    assert bool(torch.isfinite(got["y"].float()).all())


@BOTH
@pytest.mark.parametrize("M,live", [(700, 700), (700, 0), (700, 1), (700, 129), (9000, 4100)])
def test_counted_and_gathered(spa, dtype, M, live):
    c = Case(M, 96, 264 if dtype == "bf16" else 40, 0, dtype, live=live, index=True, N_out=104)
    c.check(c.run(spa))


@BOTH
def test_optional_arguments(spa, dtype):
    for over in (dict(bias=False), dict(counted=False), dict(index=True, counted=False)):
        c = Case(150, 64, 88, 1, dtype, **over)
        c.check(c.run(spa))
        assert torch.equal(c.run(spa, keep=False)["h"], c.run(spa)["h"])


def test_odd_sizes_in_fp32(spa):
    c = Case(37, 13, 7, 1, "f32", N_out=5)
    c.check(c.run(spa))


@pytest.mark.parametrize("K,F", [(7, 1030), (130, 1024), (64, 1000)])
def test_an_fp32_element_has_its_bits_in_any_tile(spa, K, F):
    """Every element is one chain over the contraction: the same alone, in a small tile and in a large one, whatever the tail of the contraction; and -0 stays -0."""
    c = Case(900, K, F, 0, "f32", bias=False)
    c.x[3] = -0.0
    c.W[:, :] = c.W.abs()
    big = c.run(spa)
    for rows in (1, 40):
        few = Case(rows, K, F, 0, "f32", bias=False)
        few.x, few.dy, few.W, few.W_down = c.x[3:3 + rows].contiguous(), c.dy[3:3 + rows].contiguous(), c.W, c.W_down
        got = few.run(spa)
        for n in got:
            assert torch.equal(got[n].view(torch.int32), big[n][3:3 + rows].view(torch.int32)), n
    dx = lambda d, M: spa.spa_linear_packed_bwd_input(d, None, None, c.W, M, None, None, (o := torch.empty(M, K, device="cuda"))) or o
    assert torch.equal(dx(big["d_pre"], 900)[3:43].view(torch.int32), dx(big["d_pre"][3:43].contiguous(), 40).view(torch.int32))


@BOTH
@ACTS
@pytest.mark.parametrize("size", [0.01, 8.0, 100.0])
def test_far_activations(spa, dtype, act, size):
    c = Case(90, 64, 136, act, dtype, size=size)
    c.check(c.run(spa))


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("M,F", [(200, 72), (6272, 1024)])
def test_the_tails_are_rounded_once(spa, act, M, F):
    """Far below 0 the activation and its slope are small, not lost: g is one element of x times 1, u = 1, dh = 1, so that h = act(g), d_g = slope, d_u = act(g).  GELU: Phi is off by 2^-12
    relative; the slope Phi + g phi of g <= -3 is at least 2/3 |g| phi > 2 Phi, so off by 2^-12; the fast exponential by (|g| or g^2 / 2) 2^-23 <= 2^-16.  SiLU: s and its slope by 2^-16."""
    td = torch.bfloat16
    x, W, W_down = torch.zeros(M, 16, dtype=td, device="cuda"), torch.zeros(2 * F, 16, dtype=td, device="cuda"), torch.zeros(8, F, dtype=td, device="cuda")
    x[:, 0] = -torch.linspace(3, 12 if act else 80, M, device="cuda").to(td)
    x[:, 1] = 1
    W[:F, 0] = 1
    W[F:, 1] = 1
    W_down[0] = 1
    dy = torch.zeros(M, 8, dtype=td, device="cuda")
    dy[:, 0] = 1
    h, pre, d_pre = (torch.empty(M, n * F, dtype=td, device="cuda") for n in (1, 2, 2))
    spa.spa_gated_linear_packed(x, None, None, W, None, act, h, pre)
    spa.spa_gated_linear_packed_bwd(dy, None, None, W_down, pre, act, d_pre)
    g = x[:, :1].double()
    value, slope = act64(g, act)
    if act:                                     # (ndtr subtracts from 1 here and is 0 at -12)
        cdf = 0.5 * torch.special.erfc(-g / 2 ** 0.5)
        value, slope = g * cdf, cdf + g * torch.exp(-g * g / 2) / (2 * np.pi) ** 0.5
    assert torch.equal(pre[:, :F].double(), g.expand(M, F)) and bool((pre[:, F:] == 1).all())
    for have, want in ((h, value), (d_pre[:, :F], slope), (d_pre[:, F:], value)):
        assert bool(((have.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -11) * want.abs()).all())


def test_more_live_rows_than_there_are(spa):
    c = Case(300, 64, 72)
    want = c.run(spa)
    c.total.fill_(5000)
    got = c.run(spa)
    assert all(torch.equal(got[n], want[n]) for n in got)


def test_the_same_row_twice_and_a_column_slice(spa):
    """Rows may repeat in an index; dy may be a slice of wider rows."""
    c = Case(256, 64, 72, index=True)
    c.idx = torch.randint(0, 60, (256,), dtype=torch.int32, device="cuda")
    c.check(c.run(spa))
    wide = torch.full((512, 64 + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:72] = c.dy
    want, pre = c.run(spa), c.run(spa)["pre"]
    d_pre = torch.empty_like(pre)
    spa.spa_gated_linear_packed_bwd(wide[:, 8:72], c.idx, c.total, c.W_down, pre, 0, d_pre)
    assert torch.equal(d_pre, want["d_pre"])


@BOTH
def test_the_gradient_over_its_input(spa, dtype):
    """d_pre may be pre itself."""
    for M, K, F in ((300, 64, 136), (6272, 64, 1024) if dtype == "bf16" else (2100, 40, 1024)):
        c = Case(M, K, F, 1, dtype, live=M - 7)
        want = c.run(spa)
        pre = want["pre"].clone()
        spa.spa_gated_linear_packed_bwd(c.dy, c.idx, c.total, c.W_down, pre, 1, pre)
        assert torch.equal(pre[:M - 7], want["d_pre"][:M - 7])


def test_values_that_are_not_finite_stay_in_their_rows(spa):
    for M, K, F in ((200, 128, 72), (6272, 256, 1024)):
        c = Case(M, K, F)
        clean = c.run(spa)
        c.x[5, 3] = float("nan")
        c.dy[9, 4] = float("inf")
        got = c.run(spa)
        assert bool(torch.isnan(got["h"][5]).all()) and not bool(torch.isfinite(got["d_pre"][9].float()).all())
        for n in got:
            rows = torch.ones(M, dtype=torch.bool, device="cuda")
            rows[5] = rows[9] = False
            assert torch.equal(got[n][rows], clean[n][rows]), n


def test_gradient_against_differences(spa):
    """The fp32 block's gradients (this kernel's d_pre through the projections' backward) along random directions against central differences of the 64-bit form."""
    c = Case(23, 24, 16, 1, "f32", N_out=8)
    res = c.run(spa)
    f32 = lambda *s: torch.empty(*s, device="cuda")
    dx, dW, db, dWd = f32(23, 24), f32(32, 24), f32(32), f32(8, 16)
    spa.spa_linear_packed_bwd_input(res["d_pre"], None, c.total, c.W, 23, None, None, dx)
    work = lambda K, N: torch.empty(max(spa.spa_linear_bwd_weight_workspace_bytes(23, K, N, "f32"), 256), dtype=torch.uint8, device="cuda")
    spa.spa_linear_packed_bwd_weight(res["d_pre"], None, c.x, None, None, c.total, 23, dW, db, work(24, 32))
    spa.spa_linear_packed_bwd_weight(c.dy, None, res["h"], None, None, c.total, 23, dWd, None, work(16, 8))

    def value(x, W, b, Wd):
        pre = x @ W.T + b
        return float(((act64(pre[:, :16], 1)[0] * pre[:, 16:]) @ Wd.T * c.dy.double()).sum())

    at = [t.double() for t in (c.x, c.W, c.b, c.W_down)]
    g, h = torch.Generator(device="cuda").manual_seed(2), 1e-4
    for i, d in enumerate((dx, dW, db, dWd)):
        for _ in range(3):
            v = torch.randn(d.shape, generator=g, device="cuda", dtype=torch.float64)
            move = lambda s: value(*[t + s * v if k == i else t for k, t in enumerate(at)])
            num, have, size = (move(h) - move(-h)) / (2 * h), float((d * v).sum()), float((d * v).abs().sum())
            assert abs(num - have) <= 2e-5 * size, i


@pytest.mark.parametrize("M,K,F", [(300, 64, 72), (6272, 128, 1024)])
def test_replayed_and_repeated(spa, M, K, F):
    c = Case(M, K, F)
    x0, x1 = c.x.clone(), Case(M, K, F, seed=8).x
    h, pre, d_pre = (torch.zeros(M, n * F, dtype=torch.bfloat16, device="cuda") for n in (1, 2, 2))

    def calls():
        spa.spa_gated_linear_packed(c.x, None, c.total, c.W, c.b, 0, h, pre)
        spa.spa_gated_linear_packed_bwd(c.dy, None, c.total, c.W_down, pre, 0, d_pre)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for rep in range(4):
        c.x.copy_((x0, x1)[rep % 2])
        c.total.fill_((M, M // 2)[rep // 2])
        h.zero_(), pre.zero_(), d_pre.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.live = (M, M // 2)[rep // 2]
        want = c.run(spa)
        torch.cuda.synchronize()
        for got, name in ((h, "h"), (pre, "pre"), (d_pre, "d_pre")):
            assert torch.equal(got[:c.live], want[name][:c.live]), (rep, name)
            assert bool((got[c.live:] == 0).all())
