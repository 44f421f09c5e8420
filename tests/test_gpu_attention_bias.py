"""Packed attention with a relative position bias and its backward, against the formulas in 64 bits, segment by segment.

Tolerances count roundings.  H: half a step of the stored type, relative (bf16 2^-8, fp32 2^-24); U = 2^-24.  A score is a sum of
Dh products in fp32, off by at most (Dh + 4) U of the products' magnitudes, and the exponent's argument by 4 U of its own:
with A the largest magnitude of a row's scores, P is off by E = U (2 (Dh + 4) A + 16) of itself (once in the score, once in lse).
bf16: P and dS are rounded to bf16 as operands of the products, H of themselves each; D of dq comes from the rounded out,
off by H sum|dO O| and by what the rounded P put there, H sum_j P |dP|.  d_table is a sum of fp32 dS, off by E |dS| and P times what
dP and D are off by, (Dh + 4 + n) U of their magnitudes, and by half a unit of the integers each, 2^-30 of the largest possible
|dS| at most."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


class Case:
    """lens: rows of every segment.  positions: 'sorted' distinct ascending tokens, 'any' order with repeats, None: no index."""

    def __init__(self, lens, grid, H, Dh, dtype, seed=0, buckets="exact", positions="sorted", sigma=1.0, spare=5, holes=0.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.grid, self.H, self.Dh, self.dtype = list(lens), grid, H, Dh, dtype
        gh, gw = grid
        self.N, self.B, self.T, self.C = gh * gw, len(lens), sum(lens), H * Dh
        self.n_max = max(max(lens), 1)
        td = TD[dtype]
        rows = self.rows = max(self.T + spare, 1)
        self.cu = torch.tensor([0] + list(torch.tensor(self.lens).cumsum(0)), dtype=torch.int32)
        self.qkv = (sigma * torch.randn(rows, 3 * self.C, generator=g)).to(td)
        self.dout = torch.randn(rows, self.C, generator=g).to(td)
        self.pos = torch.zeros(rows, dtype=torch.int64)
        at = 0
        for b, n in enumerate(self.lens):
            p = torch.randperm(self.N, generator=g)[:n].sort()[0] if positions != "any" else torch.randint(self.N, (n,), generator=g)
            self.pos[at:at + n] = torch.arange(n) if positions is None else p
            at += n
        image = torch.repeat_interleave(torch.arange(self.B), torch.tensor(self.lens))
        self.gidx = None
        if positions is not None:
            self.gidx = torch.zeros(rows, dtype=torch.int32)
            self.gidx[:self.T] = (self.pos[:self.T] + image * self.N).int()
        offsets = (2 * gh - 1) * (2 * gw - 1)
        if buckets == "exact":
            self.buckets, self.nb = None, offsets
            self.map = torch.arange(offsets)
        else:
            if buckets == "log":
                from paper_2410_23608_amd import spa as mod
                self.buckets, self.nb = mod.relative_position_buckets(gh, gw, 2, 3)
            else:                                   # random, some of them out of range: no bias there
                self.nb = 37
                self.buckets = torch.randint(-3, self.nb + 3, (offsets,), generator=g, dtype=torch.int32)
            self.map = self.buckets.long()
        self.table = torch.randn(H, self.nb, generator=g)
        if holes:
            self.table[torch.rand(H, self.nb, generator=g) < holes] = -math.inf
        self.table = self.table.to(td)

    def exact(self):
        """Results and tolerances."""
        H, Dh, C, (gh, gw) = self.H, self.Dh, self.C, self.grid
        half = HALF[self.dtype]
        hp = half if self.dtype == "bf16" else 0.0
        f64 = lambda *s: torch.zeros(*s, dtype=torch.float64)
        res = {k: (f64(self.T, C), f64(self.T, C)) for k in ("out", "dq", "dk", "dv")}
        lse, dt = (f64(H, self.T), f64(H, self.T)), (f64(H, self.nb), f64(H, self.nb))
        scale = 1 / math.sqrt(Dh)
        big = f64(H)
        at = 0
        for n in self.lens:
            j = slice(at, at + n)
            at += n
            if n == 0:
                continue
            r, c = self.pos[j] // gw, self.pos[j] % gw
            bucket = self.map[(r[:, None] - r[None] + gh - 1) * (2 * gw - 1) + c[:, None] - c[None] + gw - 1]
            known = (bucket >= 0) & (bucket < self.nb)
            for h in range(H):
                col = slice(h * Dh, (h + 1) * Dh)
                q, k, v = (self.qkv[j, i * C:(i + 1) * C][:, col].double() for i in range(3))
                dO = self.dout[j, col].double()
                bias = torch.where(known, self.table[h].double()[bucket.clamp(0, self.nb - 1)], 0.0)
                S = q @ k.T * scale + bias
                some = (S > -math.inf).any(1, keepdim=True)
                m = torch.where(some, S.amax(1, keepdim=True), 0.0)
                e = torch.exp(S - m)
                l = e.sum(1, keepdim=True)
                P = e / torch.where(some, l, 1.0)
                O = P @ v
                L = (m + torch.log(l))[:, 0]
                A = (q.abs() @ k.abs().T * scale + torch.where(bias > -math.inf, bias.abs(), 0.0)).amax(1, keepdim=True)
                E = U * (2 * (Dh + 4) * A + 16 + n / 8)         # (n / 8: the row's sum of exponentials)
                res["out"][0][j, col] = O
                res["out"][1][j, col] = (hp + 2 * E) * (P @ v.abs()) + half * O.abs() + 1e-30
                lse[0][h, j], lse[1][h, j] = L, torch.where(L > -math.inf, E[:, 0] + 4 * U * L.abs(), 0.0)
                dP, mag = dO @ v.T, dO.abs() @ v.abs().T
                D = (P * dP).sum(1, keepdim=True)
                dS = P * (dP - D)
                off = (Dh + 4 + n) * U * (mag + (P * mag).sum(1, keepdim=True))
                off_d = off + half * (dO.abs() * O.abs()).sum(1, keepdim=True) + hp * (P * dP.abs()).sum(1, keepdim=True)
                wrong = hp * dS.abs() + 2 * E * dS.abs() + P * off_d
                res["dq"][0][j, col], res["dk"][0][j, col] = dS @ k * scale, dS.T @ q * scale
                res["dv"][0][j, col] = P.T @ dO
                res["dq"][1][j, col] = wrong @ k.abs() * scale + half * res["dq"][0][j, col].abs() + 1e-30
                res["dk"][1][j, col] = wrong.T @ q.abs() * scale + half * res["dk"][0][j, col].abs() + 1e-30
                res["dv"][1][j, col] = (P * (hp + 2 * E)).T @ dO.abs() + half * res["dv"][0][j, col].abs() + 1e-30
                dt[0][h].index_add_(0, bucket[known], dS[known])
                big[h] = torch.maximum(big[h], 8 * Dh * self.dout[:self.T, col].abs().max().double() * self.qkv[:self.T, 2 * C:][:, col].abs().max())
                dt[1][h].index_add_(0, bucket[known], (2 * E * dS.abs() + P * off)[known] + 2.0 ** -30 * big[h])
        res["lse"], res["d_table"] = lse, (dt[0], dt[1] + 4 * U * dt[0].abs())
        return res

    def run(self, spa, backward=True, want_table=True):
        H, Dh, C, B, td = self.H, self.Dh, self.C, self.B, TD[self.dtype]
        dev = lambda t: None if t is None else t.cuda()
        code = spa.SPA_BF16 if self.dtype == "bf16" else spa.SPA_F32
        qkv = self.qkv.cuda()
        q, k, v = (qkv[:, i * C:(i + 1) * C] for i in range(3))
        out = torch.full((self.rows, C), 7.0, dtype=td, device="cuda")
        lse = torch.full((H, B * self.n_max), 7.0, dtype=torch.float32, device="cuda")
        args = (dev(self.cu), dev(self.gidx), dev(self.table), dev(self.buckets), self.grid, B, self.n_max, H, Dh)
        spa.spa_packed_attention_bias(q, k, v, *args, out, lse)
        got = dict(out=out, lse=lse)
        if backward:
            dqkv = torch.full((self.rows, 3 * C), 7.0, dtype=td, device="cuda")
            dq, dk, dv = (dqkv[:, i * C:(i + 1) * C] for i in range(3))
            d_table = torch.full((H, self.nb), float("nan"), device="cuda") if want_table else None
            ws = torch.full((spa.spa_attention_bias_bwd_workspace_bytes(B, self.n_max, H, Dh, *self.grid, code),), 255, dtype=torch.uint8,
                            device="cuda")
            spa.spa_packed_attention_bias_bwd(q, k, v, out, self.dout.cuda(), lse, *args, dq, dk, dv, d_table, ws)
            got.update(dq=dq, dk=dk, dv=dv, d_table=d_table)
        return got

    def check(self, got, names=None):
        T = self.T
        for name, (want, tol) in self.exact().items():
            if name not in got or got[name] is None or (names and name not in names):
                continue
            t = got[name].cpu().double()
            live = t if name == "d_table" else t[:, :T] if name == "lse" else t[:T]
            if name != "d_table":
                rest = t[:, T:] if name == "lse" else t[T:]
                assert bool((rest == 7.0).all()), f"{name}: rows behind the last segment"
            bad = ~(((live - want).abs() <= tol) | (live == want))
            assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} off, worst "
                                   f"{float(((live - want).abs() / tol)[bad].max()):.3g} of the tolerance")


LENS = {"few": [1, 0, 2, 5], "edges": [31, 32, 33, 64, 65, 63], "one": [1], "none": [0, 0], "tile": [127, 128, 129, 1],
        "more": [190, 17, 96, 256]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("name", list(LENS))
def test_against_the_formula(spa, name, Dh, dtype):
    c = Case(LENS[name], (16, 16), 3, Dh, dtype, seed=len(name) + Dh)
    c.check(c.run(spa))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("buckets", ["exact", "log", "random"])
@pytest.mark.parametrize("grid,lens", [((1, 300), [300, 7, 150]), ((200, 1), [64, 200]), ((7, 7), [49, 3, 0, 48]), ((17, 23), [391, 200]),
                                       ((1, 1), [1, 1, 0])])
def test_maps_and_buckets(spa, grid, lens, buckets, dtype):
    c = Case(lens, grid, 2, 32, dtype, seed=grid[1], buckets=buckets)
    c.check(c.run(spa))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [32, 64])
def test_long_segments(spa, Dh, dtype):
    c = Case([1100, 3, 517, 640], (50, 84), 2, Dh, dtype, seed=3, buckets="exact" if Dh == 32 else "log")
    c.check(c.run(spa))


@pytest.mark.parametrize("positions", ["any", None])
@pytest.mark.parametrize("grid,lens", [((12, 31), [300, 64, 5]), ((40, 40), [700, 1000, 33])])
def test_rows_in_any_order_repeated_positions_and_no_index(spa, positions, grid, lens):
    c = Case(lens, grid, 2, 32, "bf16", seed=8, positions=positions)
    c.check(c.run(spa))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("holes", [0.5, 0.97, 1.0])
def test_entries_that_leave_pairs_out(spa, holes, dtype):
    """Rows without any pair left give zeros, lse -inf and no gradient."""
    c = Case([70, 1, 33, 150], (15, 15), 2, 32, dtype, seed=5, buckets="random", holes=holes)
    if holes == 1.0:
        c.buckets.clamp_(0, c.nb - 1)
        c.map = c.buckets.long()
    got = c.run(spa)
    c.check(got)
    if holes == 1.0:
        assert bool((got["out"][:c.T] == 0).all()) and bool((got["lse"][:, :c.T] == -math.inf).all())
        assert all(bool((got[n][:c.T] == 0).all()) for n in ("dq", "dk", "dv")) and bool((got["d_table"] == 0).all())


def test_steep_rows_and_zero_bias_is_the_plain_attention(spa):
    c = Case([200, 77, 1], (14, 15), 2, 64, "bf16", seed=6, sigma=3.0)
    c.check(c.run(spa))
    c.table.zero_()
    got = c.run(spa)
    C, out, lse = c.C, torch.empty_like(got["out"]), torch.empty_like(got["lse"])
    qkv = c.qkv.cuda()
    spa.spa_packed_attention(qkv[:, :C], qkv[:, C:2 * C], qkv[:, 2 * C:], c.cu.cuda(), c.B, c.n_max, c.H, c.Dh, out, lse)
    want, tol = c.exact()["out"]
    assert bool(((out[:c.T].cpu().double() - want).abs() <= tol).all())
    assert bool(((got["out"][:c.T].cpu().double() - out[:c.T].cpu().double()).abs() <= 2 * tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entries_of_the_types_lowest_value(spa, dtype):
    """A mask written with the type's lowest number: such pairs weigh nothing beside any other, and share a row that has no other."""
    c = Case([70, 1, 33, 150], (15, 15), 2, 32, dtype, seed=15, buckets="random")
    c.buckets.clamp_(0, c.nb - 1)
    c.map = c.buckets.long()
    low = torch.finfo(TD[dtype]).min
    c.table[0, ::2], c.table[1] = low, low
    c.qkv[:, :c.C] = 0                                        # (scores beside such an entry are below its last place)
    got = c.run(spa)
    c.check(got, ("out", "dq", "dk", "dv"))
    assert bool(torch.isfinite(got["d_table"]).all())


def test_without_the_table_gradient_the_rest_is_the_same(spa):
    c = Case([100, 300, 9], (20, 20), 2, 32, "bf16", seed=7)
    a, b = c.run(spa), c.run(spa, want_table=False)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(a[n], b[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("grid,lens", [((24, 25), [300, 130]), ((56, 56), [700, 65, 193]), ((64, 64), [390, 1, 64]), ((130, 130), [1500, 65])])
def test_every_size_of_map_with_and_without_the_table_gradient(spa, grid, lens, Dh, dtype):
    """Maps that LDS holds beside the sums of dS by offset, or with part of them, and larger ones."""
    c = Case(lens, grid, 2, Dh, dtype, seed=19 + Dh)
    got, without = c.run(spa), c.run(spa, want_table=False)
    c.check(got)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(got[n], without[n])


def test_results_are_the_same_in_every_run(spa):
    c = Case([700, 256, 31, 400], (30, 31), 3, 32, "bf16", seed=9, buckets="log")
    first = c.run(spa)
    for _ in range(3):
        again = c.run(spa)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_gradient_of_the_table_against_differences(spa):
    """fp32 calls: the change of sum(out * dout) along a direction of the table."""
    c = Case([40, 13], (8, 9), 2, 32, "f32", seed=10, buckets="log")
    d_table = c.run(spa)["d_table"].cpu().double()
    g = torch.Generator().manual_seed(1)
    v = torch.randn(c.H, c.nb, generator=g).double()
    base, h = c.table.double(), 1e-5

    def value(t):
        c.table = base + t * v
        return float((c.exact()["out"][0] * c.dout[:c.T].double()).sum())

    slope = (value(h) - value(-h)) / (2 * h)
    # (d_table: U n of the sums' magnitudes; differences: h^2 and 1e-16 |value| / h)
    assert abs(float((d_table * v).sum()) - slope) <= 1e-4 * (1 + abs(slope))


@pytest.mark.parametrize("where", ["q", "v", "dout", "table"])
def test_a_head_that_is_not_finite_says_so(spa, where):
    """d_table of that head is NaN, the other head's results are as without."""
    c = Case([50, 80], (10, 10), 2, 32, "bf16", seed=11, buckets="log")
    clean = c.run(spa)
    if where == "table":
        c.table[0, int(c.map[c.map.numel() // 2])] = math.nan
    elif where == "dout":
        c.dout[60, 3] = math.inf
    else:
        c.qkv[60, (0 if where == "q" else 2 * c.C) + 3] = math.nan
    got = c.run(spa)
    assert bool(got["d_table"][0].isnan().all())
    assert torch.equal(got["d_table"][1], clean["d_table"][1])
    for n in ("out", "dq", "dk", "dv"):
        assert torch.equal(got[n][:, 32:], clean[n][:, 32:])
        if where != "table":                                       # the other segment too
            assert torch.equal(got[n][:50], clean[n][:50])


def test_separate_buffers_and_wide_strides(spa):
    """q, k, v and their gradients in buffers of different widths give the bits of the fused ones."""
    c = Case([90, 33, 140], (13, 14), 2, 32, "bf16", seed=12)
    want = c.run(spa)
    C, dev = c.C, lambda t: None if t is None else t.cuda()
    wide = [torch.zeros(c.rows, C + 8 * (i + 1), dtype=torch.bfloat16, device="cuda") for i in range(6)]
    for i in range(3):
        wide[i][:, 8:8 + C] = c.qkv.cuda()[:, i * C:(i + 1) * C]
    view = [t[:, 8:8 + C] for t in wide]
    out, lse = torch.empty_like(want["out"]), torch.empty_like(want["lse"])
    args = (dev(c.cu), dev(c.gidx), dev(c.table), None, c.grid, c.B, c.n_max, c.H, c.Dh)
    spa.spa_packed_attention_bias(*view[:3], *args, out, lse)
    assert torch.equal(out[:c.T], want["out"][:c.T])
    d_table = torch.empty_like(want["d_table"])
    ws = torch.empty(spa.spa_attention_bias_bwd_workspace_bytes(c.B, c.n_max, c.H, c.Dh, *c.grid, spa.SPA_BF16), dtype=torch.uint8,
                     device="cuda")
    spa.spa_packed_attention_bias_bwd(*view[:3], out, c.dout.cuda(), lse, *args, *view[3:], d_table, ws)
    for n, t in zip(("dq", "dk", "dv"), view[3:]):
        assert torch.equal(t[:c.T], want[n][:c.T])
    assert torch.equal(d_table, want["d_table"])
    for t in wide[3:]:                                             # beside the columns and behind the rows: as they were
        assert bool((t[:, :8] == 0).all()) and bool((t[:, 8 + C:] == 0).all()) and bool((t[c.T:] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grid,Dh", [((40, 41), 32), ((60, 90), 32), ((60, 90), 64)])
def test_maps_whose_offsets_take_more_than_one_pass(spa, grid, Dh, dtype):
    c = Case([900, 70, 333, 128, 1], grid, 2, Dh, dtype, seed=16, buckets="exact" if Dh == 32 else "log")
    c.check(c.run(spa))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [70, 300])
def test_many_segments(spa, B, dtype):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 60, (B,), generator=g).tolist()
    lens[B // 2] = 130                                             # two blocks of keys
    c = Case(lens, (12, 13), 2, 32, dtype, seed=17, buckets="log")
    c.check(c.run(spa))


@pytest.mark.parametrize("Dh", [32, 64])
def test_long_and_many_short_segments_on_a_large_map(spa, Dh):
    c = Case([1200, 390, 700] + [20] * 52, (56, 56), 2, Dh, "bf16", seed=21)
    got, without = c.run(spa), c.run(spa, want_table=False)
    c.check(got)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(got[n], without[n])


@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("lens", [[700], [513, 64], [65, 1], [1024]])
def test_few_long_segments(spa, lens, Dh):
    """Few blocks of queries: the waves of a block share its keys."""
    c = Case(lens, (33, 34), 2, Dh, "bf16", seed=18)
    c.check(c.run(spa))


def test_large_and_sparse_maps(spa):
    """Few tokens far apart on a map of many offsets, and a long sequence without a second axis."""
    for grid, lens in (((300, 300), [150, 40]), ((1, 20000), [400, 90])):
        c = Case(lens, grid, 2, 32, "bf16", seed=13, buckets="log")
        c.check(c.run(spa))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grid,lens", [((9, 8), [72, 30]), ((30, 31), [400, 65]), ((60, 61), [300, 129])])
def test_a_bucket_of_its_own_for_every_offset(spa, grid, lens, dtype):
    """A map that only renames the offsets: the results are those without a map, in the renamed places.  d_table by way of a map is rounded
    once more, to a unit of 2^-40 of the power of two above the largest sum: 2^-40 of it at most, and its own last place."""
    c = Case(lens, grid, 2, 32, dtype, seed=22)
    plain = c.run(spa)
    E = c.nb
    name = torch.randperm(E, generator=torch.Generator().manual_seed(3))
    table = torch.empty_like(c.table)
    table[:, name] = c.table
    c.table, c.buckets, c.map = table, name.int(), name
    got = c.run(spa)
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(got[n], plain[n]), n
    a, b = got["d_table"].cpu().double()[:, name], plain["d_table"].cpu().double()
    tol = 2.0 ** -40 * b.abs().amax(1, keepdim=True) + 2 * U * b.abs()
    assert bool(((a - b).abs() <= tol).all())


@pytest.mark.parametrize("where", ["v", "dout"])
def test_a_head_that_is_not_finite_says_so_in_fp32(spa, where):
    c = Case([50, 80], (10, 10), 2, 32, "f32", seed=23, buckets="log")
    clean = c.run(spa)
    if where == "dout":
        c.dout[60, 3] = math.inf
    else:
        c.qkv[60, 2 * c.C + 3] = math.nan
    got = c.run(spa)
    assert bool(got["d_table"][0].isnan().all()) and torch.equal(got["d_table"][1], clean["d_table"][1])


def test_more_than_one_head_row_and_strides_of_their_own(spa):
    """q, k, v and their gradients in buffers of different widths, what lies between the rows untouched; 70 heads."""
    H, Dh, lens, grid = 70, 32, [40, 33, 1], (7, 9)
    c = Case(lens, grid, H, Dh, "bf16", seed=24)
    want = c.run(spa)
    C, B, rows = c.C, c.B, c.rows
    wide = [torch.full((rows, C + 8 * (i + 1)), 3.0, dtype=torch.bfloat16, device="cuda") for i in range(3)]
    q, k, v = (w[:, 8 * i:8 * i + C] for i, w in enumerate(wide))
    for i, t in enumerate((q, k, v)):
        t.copy_(c.qkv[:, i * C:(i + 1) * C])
    args = (c.cu.cuda(), c.gidx.cuda(), c.table.cuda(), None, grid, B, c.n_max, H, Dh)
    out, lse = torch.full((rows, C), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((H, B * c.n_max), 7.0, device="cuda")
    spa.spa_packed_attention_bias(q, k, v, *args, out, lse)
    gw = [torch.full((rows, C + 8 * (3 - i)), 5.0, dtype=torch.bfloat16, device="cuda") for i in range(3)]
    dq, dk, dv = (w[:, 8:8 + C] for w in gw)
    d_table = torch.empty(H, c.nb, device="cuda")
    ws = torch.empty(spa.spa_attention_bias_bwd_workspace_bytes(B, c.n_max, H, Dh, *grid, spa.SPA_BF16), dtype=torch.uint8, device="cuda")
    spa.spa_packed_attention_bias_bwd(q, k, v, out, c.dout.cuda(), lse, *args, dq, dk, dv, d_table, ws)
    for n, t in (("out", out), ("lse", lse), ("d_table", d_table)):
        assert torch.equal(t, want[n]), n
    for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(t[:c.T], want[n][:c.T]), n
        assert bool((t[c.T:] == 5.0).all()), n
    assert all(bool((w[:, :8] == 5.0).all()) and bool((w[:, 8 + C:] == 5.0).all()) for w in gw)
