"""Attention with a position bias where the table holds finite masks, from beyond any usual score to the type's lowest number.

Beside a key without a mask a masked one weighs nothing (the least mask here is -200, e^-200 in 64 bits); a row all of whose keys have the
same mask is the softmax of its scores alone, which are 0 here (q of such rows is 0, so that no last place of a sum with the mask matters): its
weights are equal.  Tolerances are those of test_gpu_attention_bias.py with A taken over the keys without a mask alone, 0
for a row that has none, since its scores differ by nothing."""
import math

import pytest
import torch

from test_gpu_attention_bias import HALF, TD, U, Case, spa  # noqa: F401 (spa: the fixture)


class Masked(Case):
    """Three heads.  0: only keys a quarter of the map behind the query's place are left (the first tiles of most rows are
    masked, the last rows altogether); 1: only keys within a quarter; 2: none."""

    def __init__(self, lens, grid, Dh, dtype, value, seed=0):
        super().__init__(lens, grid, 3, Dh, dtype, seed=seed)
        gh, gw = grid
        centre = (gh - 1) * (2 * gw - 1) + gw - 1
        by = torch.arange(self.nb) - centre                          # place of the query less the key's
        self.hidden = torch.stack([by > -(centre // 4), by.abs() > centre // 4, torch.ones(self.nb, dtype=torch.bool)])
        self.table[self.hidden] = torch.finfo(TD[dtype]).min if value == "lowest" else value
        at = 0
        for n in self.lens:
            j = slice(at, at + n)
            at += n
            for h in range(3):
                empty = self.hidden[h][self.offset(j)].all(1) if n else torch.zeros(0, dtype=torch.bool)
                self.qkv[j, h * Dh:(h + 1) * Dh][empty] = 0

    def offset(self, j):
        gh, gw = self.grid
        r, c = self.pos[j] // gw, self.pos[j] % gw
        return (r[:, None] - r[None] + gh - 1) * (2 * gw - 1) + c[:, None] - c[None] + gw - 1

    def exact(self):
        H, Dh, C = self.H, self.Dh, self.C
        half = HALF[self.dtype]
        hp = half if self.dtype == "bf16" else 0.0
        f64 = lambda *s: torch.zeros(*s, dtype=torch.float64)
        res = {k: (f64(self.T, C), f64(self.T, C)) for k in ("out", "dq", "dk", "dv")}
        lse, dt = (f64(H, self.T), f64(H, self.T)), (f64(H, self.nb), f64(H, self.nb))
        scale, at = 1 / math.sqrt(Dh), 0
        for n in self.lens:
            j = slice(at, at + n)
            at += n
            o = self.offset(j)
            for h in range(H):
                col = slice(h * Dh, (h + 1) * Dh)
                q, k, v = (self.qkv[j, i * C:(i + 1) * C][:, col].double() for i in range(3))
                dO, bias, seen = self.dout[j, col].double(), self.table[h].double()[o], ~self.hidden[h][o]
                S = q @ k.T * scale + bias
                m = S.amax(1, keepdim=True)
                e = torch.exp(S - m)
                l = e.sum(1, keepdim=True)
                P, L = e / l, (m + torch.log(l))[:, 0]
                O = P @ v
                A = torch.where(seen, q.abs() @ k.abs().T * scale + bias.abs(), 0.0).amax(1, keepdim=True)
                E = U * (2 * (Dh + 4) * A + 16 + n / 8)
                res["out"][0][j, col], res["out"][1][j, col] = O, (hp + 2 * E) * (P @ v.abs()) + half * O.abs() + 1e-30
                lse[0][h, j], lse[1][h, j] = L, E[:, 0] + 4 * U * L.abs()
                dP, mag = dO @ v.T, dO.abs() @ v.abs().T
                dS = P * (dP - (P * dP).sum(1, keepdim=True))
                off = (Dh + 4 + n) * U * (mag + (P * mag).sum(1, keepdim=True))
                off_d = off + half * (dO.abs() * O.abs()).sum(1, keepdim=True) + hp * (P * dP.abs()).sum(1, keepdim=True)
                wrong = hp * dS.abs() + 2 * E * dS.abs() + P * off_d
                res["dq"][0][j, col], res["dk"][0][j, col], res["dv"][0][j, col] = dS @ k * scale, dS.T @ q * scale, P.T @ dO
                res["dq"][1][j, col] = wrong @ k.abs() * scale + half * res["dq"][0][j, col].abs() + 1e-30
                res["dk"][1][j, col] = wrong.T @ q.abs() * scale + half * res["dk"][0][j, col].abs() + 1e-30
                res["dv"][1][j, col] = (P * (hp + 2 * E)).T @ dO.abs() + half * res["dv"][0][j, col].abs() + 1e-30
                big = 8 * Dh * self.dout[:self.T, col].abs().max().double() * self.qkv[:self.T, 2 * C:][:, col].abs().max()
                dt[0][h].index_put_((o,), dS, accumulate=True)
                dt[1][h].index_put_((o,), 2 * E * dS.abs() + P * off + 2.0 ** -30 * big, accumulate=True)
        res["lse"], res["d_table"] = lse, (dt[0], dt[1] + 4 * U * dt[0].abs())
        return res


VALUES = [-200.0, -1e4, -1e9, -1e10, -1e12, -1e20, -1e25, -1e30, "lowest"]
# four waves a block; eight (four blocks of 128 queries or more, few of them); a window that moves; sums of dS in slices
SHAPES = {"four": ([300, 1, 65], (18, 19), 32), "eight": ([420, 70], (21, 21), 64), "moving": ([330, 129], (150, 90), 32),
          "slices": ([400, 33], (50, 84), 64)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_the_tolerances_say_something(name, dtype):
    """Each is far below what it is for: within it nothing is left out, doubled or 0."""
    lens, grid, Dh = SHAPES[name]
    for value in (-200.0, "lowest"):
        for what, (want, tol) in Masked(lens, grid, Dh, dtype, value).exact().items():
            if what != "lse":
                assert float(tol.norm()) < (0.25 if dtype == "bf16" else 0.005) * float(want.norm()), what


@pytest.mark.gpu
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_finite_masks_forward(spa, name, dtype, value):  # noqa: F811
    lens, grid, Dh = SHAPES[name]
    c = Masked(lens, grid, Dh, dtype, value, seed=len(name))
    c.check(c.run(spa, backward=False))


@pytest.mark.gpu
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_finite_masks_backward(spa, name, dtype, value):  # noqa: F811
    lens, grid, Dh = SHAPES[name]
    c = Masked(lens, grid, Dh, dtype, value, seed=len(name))
    c.check(c.run(spa))
