"""Norm of the heads of q and k with the rotation by place: forward and backward against a plain 64-bit form, at the sizes, types and
layouts where it can go wrong.

Tolerances.  A result is rounded once to its type (half a step: 2^-8 of the value in bf16, 2^-24 in fp32).  In front of that stand fp32 steps:
a sum of Dh values (at most 16 added in a lane, 3 exchanges, one division each for mean and variance, a square root), the affine step
and one rotation: fewer than 64 roundings, each of at most 2^-24 of a quantity no larger than A below; 2^-24 * 64 * A covers them.
Sums over rows and heads add at most as many terms in a chain as there are rows, then 512 partial rows in chains of 8 + 16 + 6: 2^-24 * (rows + 96)
times the sum of magnitudes."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
KINDS = {"layer": 0, "rms": 1, "none": 2}
EPS = 1e-6


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


class Case:
    def __init__(self, rows=37, live=None, H=3, Hk=2, Dh=64, dtype="bf16", kind="rms", layout=0, grid=(1, 5, 9), pairs=(0, 16), affine=True,
                 seed=0, pad=0, index=True, counted=True, table=True, images=4):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.live = rows, rows if live is None else live
        self.H, self.Hk, self.Dh, self.kind, self.layout, self.grid, self.pairs = H, Hk, Dh, kind, layout, grid, pairs
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        rnd = lambda *s: torch.randn(*s, generator=g)
        N = grid[0] * grid[1] * grid[2]
        self.gather = torch.randint(0, images * N, (rows,), generator=g, dtype=torch.int32) if index else None      # (any order, repeats)
        self.counted = counted
        width = (H + 2 * Hk) * Dh + pad
        self.qkv = (1.5 * rnd(rows, width) + 0.3).to(self.td)
        self.grad = rnd(rows, width).to(self.td)
        norm = kind != "none" and affine
        self.gamma = [(1 + 0.3 * rnd(Dh)).to(self.td) if norm else None for _ in range(2)]
        self.beta = [(0.3 * rnd(Dh)).to(self.td) if norm and kind == "layer" else None for _ in range(2)]
        self.base = 100.0
        self.with_table = table

    def slices(self, t):
        a, b = self.H * self.Dh, (self.H + self.Hk) * self.Dh
        return t[:, :a], t[:, a:b] if self.Hk else None

    # ---- 64 bits
    def angles(self):
        j = np.arange(self.live) if self.gather is None else self.gather[:self.live].numpy().astype(np.int64)
        gt, gh, gw = self.grid
        n = j % (gt * gh * gw)
        places = (n // (gh * gw), n // gw % gh, n % gw)
        counts = (self.pairs[0], self.pairs[1], self.Dh // 2 - sum(self.pairs))
        out = [np.outer(p, self.base ** (-np.arange(c) / max(c, 1))) for p, c in zip(places, counts)]
        a = np.concatenate(out, 1)[:, None] if self.with_table else np.zeros((self.live, 1, self.Dh // 2))
        return torch.from_numpy(np.cos(a)), torch.from_numpy(np.sin(a))

    def turn(self, x, sign=1):
        c, s = self.angles()
        s = sign * s
        if self.layout == 0:
            a, b = x[..., 0::2], x[..., 1::2]
            return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
        h = self.Dh // 2
        a, b = x[..., :h], x[..., h:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)

    def forward64(self, side, x):
        """(result, A) of the live heads of one tensor, x [live, heads, Dh] in 64 bits"""
        mu = x.mean(-1, keepdim=True) if self.kind == "layer" else torch.zeros_like(x[..., :1])
        r = 1 / torch.sqrt(((x - mu) ** 2).mean(-1, keepdim=True) + EPS) if self.kind != "none" else torch.ones_like(x[..., :1])
        xh = (x - mu) * r
        gamma = 1.0 if self.gamma[side] is None else self.gamma[side].double()
        beta = 0.0 if self.beta[side] is None else self.beta[side].double()
        size = (xh.abs().amax(-1, keepdim=True) + x.abs().mean(-1, keepdim=True) * r) * (gamma.abs().max() if torch.is_tensor(gamma) else 1.0)
        size = size + (beta.abs().max() if torch.is_tensor(beta) else 0.0)
        return self.turn(xh * gamma + beta), 2 * size, xh, r, gamma

    def backward64(self, side, x, dy):
        _, _, xh, r, gamma = self.forward64(side, x)
        du = self.turn(dy, -1)
        g = du * gamma
        if self.kind == "none":
            return du, 2 * du.abs().amax(-1, keepdim=True), None, None
        m1 = g.mean(-1, keepdim=True) if self.kind == "layer" else 0.0
        m2 = (g * xh).mean(-1, keepdim=True)
        size = r * (2 * g.abs().amax(-1, keepdim=True) + (1 + xh.abs().amax(-1, keepdim=True)) * (g * xh).abs().mean(-1, keepdim=True)
                    + g.abs().mean(-1, keepdim=True))
        # (xh itself is off by a share of x's mean: it multiplies m2, and the sums)
        return r * (g - m1 - xh * m2), 2 * size * (1 + x.abs().mean(-1, keepdim=True) * r), (du * xh, du), xh

    # ---- the calls
    def run(self, spa, back=True, in_place=False, inputs=None):
        cu = lambda t: None if t is None else t.cuda()
        nan = lambda t: torch.full_like(t, float("nan"))
        qkv, grad = (self.qkv.cuda(), self.grad.cuda()) if inputs is None else inputs
        gather, total = cu(self.gather), torch.tensor([self.live], dtype=torch.int32).cuda() if self.counted else None
        gamma, beta = [cu(t) for t in self.gamma], [cu(t) for t in self.beta]
        table = spa.rotary_table(self.grid, self.Dh, self.pairs, self.base).cuda() if self.with_table else None
        out = qkv if in_place else nan(qkv)
        (q, k), (qo, ko) = self.slices(qkv), self.slices(out)
        res = dict(out=out)
        if back:
            din = nan(qkv)
            (dqo, dko), (dq, dk) = self.slices(grad), self.slices(din)
            f32 = lambda: torch.full((self.Dh,), float("nan"), device="cuda")
            sums = [f32() if self.kind != "none" and (i < 2 or self.Hk) else None for i in range(4)]
            code = spa.dtype_code(q)
            ws = torch.full((spa.spa_qk_norm_rotary_bwd_workspace_bytes(self.rows, self.H, self.Hk, self.Dh, code),), 255, dtype=torch.uint8, device="cuda")
            spa.spa_qk_norm_rotary_bwd(dqo, dko, q, k, gather, total, gamma[0], gamma[1], KINDS[self.kind], EPS, table, self.pairs, self.grid,
                                       self.H, self.Hk, self.Dh, dq, dk, *sums, ws, self.layout)
            res.update(din=din, sums=sums)
        spa.spa_qk_norm_rotary(q, k, gather, total, gamma[0], beta[0], gamma[1], beta[1], KINDS[self.kind], EPS, table, self.pairs, self.grid,
                               self.H, self.Hk, self.Dh, qo, ko, self.layout)
        return res

    def check(self, res, in_place=False):
        T, half = self.live, HALF[self.td]
        heads = lambda t, n: t[:T].cpu().double().reshape(T, n, self.Dh)
        out, before = res["out"].cpu(), self.qkv
        for side, (n, got) in enumerate(zip((self.H, self.Hk), self.slices(out))):
            if n == 0 or T == 0:
                continue
            x = heads(self.slices(self.qkv)[side], n)
            want, size, *_ = self.forward64(side, x)
            err = (heads(got, n) - want).abs()
            tol = half * want.abs() + U * 64 * size
            assert bool((err <= tol).all()), (side, float((err - tol).max()))
            if "din" in res:
                dy = heads(self.slices(self.grad)[side], n)
                want, size, terms, _ = self.backward64(side, x, dy)
                err = (heads(self.slices(res["din"].cpu())[side], n) - want).abs()
                tol = half * want.abs() + U * 96 * size
                assert bool((err <= tol).all()), ("d", side, float((err - tol).max()))
                if terms is not None:
                    r = 1 / torch.sqrt((x ** 2).mean(-1, keepdim=True))
                    for i, t in enumerate(terms):
                        s = res["sums"][2 * side + i].cpu().double()
                        # (a term of dgamma is off as xh is: by U * 64 * (|xh| + mean |x| r) |du|)
                        more = (terms[1].abs() * (terms[0].abs() / terms[1].abs().clamp_min(1e-30) + 2)).sum((0, 1)) if i == 0 else t.abs().sum((0, 1))
                        assert bool(((s - t.sum((0, 1))).abs() <= U * (T + 160) * more).all()), (side, i)
        # nothing else is written
        keep = out[T:] if self.Hk else torch.cat((out[T:, :self.H * self.Dh].flatten(), out[:, self.H * self.Dh:].flatten()))
        assert bool(torch.isnan(keep.float()).all()) or in_place
        if in_place:
            assert torch.equal(out[T:], before[T:]) and torch.equal(out[:, (self.H + self.Hk) * self.Dh:], before[:, (self.H + self.Hk) * self.Dh:])
        else:
            assert bool(torch.isnan(out[:, (self.H + self.Hk) * self.Dh:].float()).all())
        if "din" in res:
            din = res["din"].cpu().float()
            assert bool(torch.isnan(din[T:]).all()) and bool(torch.isnan(din[:, (self.H + self.Hk) * self.Dh:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("kind", ["layer", "rms", "none"])
@pytest.mark.parametrize("layout", [0, 1])
def test_forms(spa, dtype, Dh, kind, layout):
    c = Case(rows=53, live=41, Dh=Dh, dtype=dtype, kind=kind, layout=layout, pairs=(0, Dh // 4), pad=8, seed=Dh + layout)
    c.check(c.run(spa))


@pytest.mark.parametrize("H,Hk", [(1, 0), (1, 1), (5, 5), (6, 1), (12, 4), (16, 16), (33, 7), (100, 3), (256, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads(spa, H, Hk, dtype):
    c = Case(rows=29, H=H, Hk=Hk, Dh=32, dtype=dtype, pairs=(0, 8), seed=H)
    c.check(c.run(spa))


@pytest.mark.parametrize("rows,live", [(1, 1), (1, 0), (2, 1), (300, 0), (64, 64), (1000, 777), (9001, 9001)])
def test_lengths(spa, rows, live):
    c = Case(rows=rows, live=live, seed=rows)
    c.check(c.run(spa))


@pytest.mark.parametrize("grid,pairs", [((1, 1, 1), (0, 0)), ((1, 1, 5000), (0, 0)), ((7, 6, 5), (10, 11)), ((3, 4, 2), (32, 0)), ((3, 400, 2), (0, 32)),
                                        ((3, 4, 50), (1, 2)), ((2, 9, 3), (5, 3))])
@pytest.mark.parametrize("layout", [0, 1])
def test_axes(spa, grid, pairs, layout):
    """Axes of any share of the pairs, odd ones among them, and far places."""
    for dtype in ("bf16", "f32"):
        c = Case(rows=61, grid=grid, pairs=pairs, dtype=dtype, layout=layout, seed=sum(pairs))
        c.check(c.run(spa))


def test_optional_arguments(spa):
    for over in (dict(index=False), dict(counted=False), dict(table=False), dict(affine=False), dict(affine=False, kind="layer"),
                 dict(index=False, counted=False, table=False, kind="layer")):
        c = Case(rows=90, **over)
        c.check(c.run(spa))


def test_more_live_rows_than_there_are(spa):
    c = Case(rows=40)
    c.live = 40
    total = torch.tensor([4000], dtype=torch.int32).cuda()
    qkv = c.qkv.cuda()
    out = torch.empty_like(qkv)
    (q, k), (qo, ko) = c.slices(qkv), c.slices(out)
    table = spa.rotary_table(c.grid, c.Dh, c.pairs, c.base).cuda()
    spa.spa_qk_norm_rotary(q, k, c.gather.cuda(), total, c.gamma[0].cuda(), None, c.gamma[1].cuda(), None, 1, EPS, table, c.pairs, c.grid, c.H, c.Hk,
                           c.Dh, qo, ko)
    want = c.run(spa, back=False)["out"]
    cols = (c.H + c.Hk) * c.Dh
    assert torch.equal(out[:, :cols], want[:, :cols])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(spa, dtype):
    c = Case(rows=47, live=33, dtype=dtype, pad=16, layout=1)
    res = c.run(spa, back=False, in_place=True)
    c.check(res, in_place=True)
    want = c.run(spa)
    # dq over the gradient, and over q
    (q, k), g = c.slices(c.qkv.cuda()), c.grad.cuda()
    for over in (g, c.qkv.cuda()):
        dq, dk = c.slices(over)
        qq, kk = (dq, dk) if over is not g else (q, k)
        gq, gk = c.slices(g) if over is g else c.slices(c.grad.cuda())
        ws = torch.empty(spa.spa_qk_norm_rotary_bwd_workspace_bytes(c.rows, c.H, c.Hk, c.Dh, spa.dtype_code(q)), dtype=torch.uint8, device="cuda")
        table = spa.rotary_table(c.grid, c.Dh, c.pairs, c.base).cuda()
        spa.spa_qk_norm_rotary_bwd(gq, gk, qq, kk, c.gather.cuda(), torch.tensor([c.live], dtype=torch.int32).cuda(), c.gamma[0].cuda(),
                                   c.gamma[1].cuda(), 1, EPS, table, c.pairs, c.grid, c.H, c.Hk, c.Dh, dq, dk, None, None, None, None, ws, 1)
        cols = (c.H + c.Hk) * c.Dh
        assert torch.equal(over[:c.live, :cols], want["din"][:c.live, :cols])


def test_values_that_are_not_finite_stay_in_their_head(spa):
    """A NaN makes its head NaN.  An infinity makes r = 1 / sqrt(inf) = 0: its own pair is inf * 0 = NaN, the head's others are 0."""
    c = Case(rows=20, H=4, Hk=4)
    clean = c.run(spa)["out"]
    c.qkv[3, 70] = float("nan")                      # row 3, head 1 of q
    c.qkv[9, 4 * 64 + 2 * 64] = float("inf")         # row 9, head 2 of k, its first pair
    got = c.run(spa)["out"]
    assert bool(torch.isnan(got[3, 64:128].float()).all())
    assert bool(torch.isnan(got[9, 384:386].float()).all()) and bool((got[9, 386:448] == 0).all())
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[3, 64:128] = bad[9, 384:448] = True
    cols = 8 * 64
    assert torch.equal(got[:, :cols][~bad[:, :cols]], clean[:, :cols][~bad[:, :cols]])


def test_gradient_against_differences(spa):
    """The fp32 gradient along random directions against central differences of the 64-bit form: error h^2 times the third
    derivative (here below 1e3 of the value's scale) plus the gradient's own."""
    c = Case(rows=11, H=2, Hk=1, Dh=32, dtype="f32", kind="layer", pairs=(0, 8))
    res = c.run(spa)
    g = torch.Generator().manual_seed(5)
    h = 1e-4
    for side, n in enumerate((2, 1)):
        x = c.slices(c.qkv)[side].double().reshape(11, n, 32)
        dy = c.slices(c.grad)[side].double().reshape(11, n, 32)
        d = c.slices(res["din"].cpu())[side].double().reshape(11, n, 32)
        for _ in range(4):
            v = torch.randn(x.shape, generator=g, dtype=torch.float64)
            num = ((c.forward64(side, x + h * v)[0] - c.forward64(side, x - h * v)[0]) * dy).sum() / (2 * h)
            assert abs(float(num - (d * v).sum())) <= 1e-5 * float((d.abs() * v.abs()).sum())
        for i, param in enumerate((c.gamma, c.beta)):
            v = torch.randn(32, generator=g, dtype=torch.float64)
            keep, s = param[side], res["sums"][2 * side + i].cpu().double()
            param[side] = keep.double() + h * v
            up = (c.forward64(side, x)[0] * dy).sum()
            param[side] = keep.double() - h * v
            down = (c.forward64(side, x)[0] * dy).sum()
            param[side] = keep
            assert abs(float((up - down) / (2 * h) - (s * v).sum())) <= 1e-5 * float((s.abs() * v.abs()).sum() + 1)


def test_replayed_on_streams_and_repeated(spa):
    """Captured forward and backward, replayed with other inputs and eager work between, on two streams at once: bit for bit the eager results."""
    c = Case(rows=700, live=611, H=6, Hk=2)
    other = Case(rows=700, live=611, H=6, Hk=2, seed=9)
    flat = lambda r: [r["out"], r["din"], *r["sums"]]
    cols = (c.H + c.Hk) * c.Dh
    same = lambda a, b: all(torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float())) for x, y in zip(flat(a), flat(b)))
    inputs = (c.qkv.cuda(), c.grad.cuda())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = c.run(spa, inputs=inputs)
    torch.cuda.synchronize()
    gather, total = c.gather.cuda(), torch.tensor([c.live], dtype=torch.int32).cuda()
    table = spa.rotary_table(c.grid, c.Dh, c.pairs, c.base).cuda()
    gq, gk = c.gamma[0].cuda(), c.gamma[1].cuda()
    out, din, sums = torch.full_like(inputs[0], float("nan")), torch.full_like(inputs[0], float("nan")), [torch.zeros(64, device="cuda") for _ in range(4)]
    ws = torch.empty(spa.spa_qk_norm_rotary_bwd_workspace_bytes(700, 6, 2, 64, 1), dtype=torch.uint8, device="cuda")
    (q, k), (qo, ko), (dqo, dko), (dq, dk) = (c.slices(t) for t in (inputs[0], out, inputs[1], din))

    def calls():
        spa.spa_qk_norm_rotary_bwd(dqo, dko, q, k, gather, total, gq, gk, 1, EPS, table, c.pairs, c.grid, 6, 2, 64, dq, dk, *sums, ws)
        spa.spa_qk_norm_rotary(q, k, gather, total, gq, None, gk, None, 1, EPS, table, c.pairs, c.grid, 6, 2, 64, qo, ko)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for rep in range(4):
        src = (c, other)[rep % 2]
        inputs[0].copy_(src.qkv.cuda())
        inputs[1].copy_(src.grad.cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        keep = c.qkv, c.grad
        c.qkv, c.grad = src.qkv, src.grad
        want = c.run(spa)
        torch.cuda.synchronize()
        c.qkv, c.grad = keep
        assert same(dict(out=out, din=din, sums=sums), want), rep
    assert same(first, c.run(spa))


def test_threads(spa):
    cases = [Case(rows=400, H=h, Hk=2, seed=h, dtype="f32" if h % 2 else "bf16") for h in (2, 3, 5, 8)]
    want = [c.run(spa) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def calls(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got = cases[i].run(spa)
                    torch.cuda.current_stream().synchronize()
                    if not torch.equal(torch.nan_to_num(got["din"].float()), torch.nan_to_num(want[i]["din"].float())):
                        wrong.append(i)
        except Exception as e:
            wrong.append((i, e))

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]
