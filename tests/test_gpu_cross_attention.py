"""Attention to another sequence, forward and backward, against a plain 64-bit form, at the lengths, layouts and masks where it can go wrong.

Tolerances.  half: half a step of the tensors' type, relative (2^-8 bf16, 2^-24 fp32).  A score is a sum of Dh products in fp32, off by eS = (Dh + 4) 2^-24
scale sum |q||k| at most; the exponent's argument is below 185 in size where it is formed by one multiply-add (2^-16 with the exponential's own error), beyond it the
scores' and lse's own roundings count: 2^-22 of the score's size.  So P is off by eP = 2 max eS + 2^-15 + 2^-22 max |S| of itself, and by another half step where it is rounded as an
operand (bf16).  Sums of n terms in fp32 in any order: n 2^-24 of the sum of magnitudes.
  out: sum P|v| (2 eP + [half] + n u) + half |out|
  D:   sum |dO| (out's bound), dP: (Dh + 4) u sum |dO||v|;   dS: |dS| (eP + [half]) + P (D's and dP's)
  dq, dk, dv: scale sum |k| (dS's), ..., sum |dO| P (eP + [half]), each + n u of the magnitudes + half of the value.
Weights below 2^-126 may be 0: fewer than 2^14 of them, times operands below 2^12, are less than 2^-100."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


class Case:
    """q_lens, k_lens: of every segment; held: places of a key segment (padded batch) or None; more_q, more_k: by how much max_q, max_k exceed the longest."""

    def __init__(self, q_lens, k_lens, H=2, Hk=1, Dh=64, dtype="bf16", held=None, seed=0, size=1.0, more_q=0, more_k=0, pad=0, scale=0.0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        self.q_lens, self.k_lens, self.H, self.Hk, self.Dh, self.B = list(q_lens), list(k_lens), H, Hk, Dh, len(q_lens)
        places = [held] * self.B if held is not None else self.k_lens
        self.cu_q, self.cu_k = np.concatenate(([0], np.cumsum(self.q_lens))), np.concatenate(([0], np.cumsum(places)))
        self.key_lens = torch.tensor(self.k_lens, dtype=torch.int32) if held is not None else None
        self.max_q, self.max_k = max(max(q_lens), 1) + more_q, max(max(places), 1) + more_k
        self.rows_q, self.rows_k = int(self.cu_q[-1]) + 3, int(self.cu_k[-1]) + 3            # (some behind the last segment)
        C, Ck = H * Dh, Hk * Dh
        self.softmax_scale, self.scale = scale, scale or Dh ** -0.5
        self.q = (size * rnd(self.rows_q, C + pad)).to(self.td)
        self.kv = rnd(self.rows_k, 2 * Ck + pad).to(self.td)
        self.dout = rnd(self.rows_q, C).to(self.td)
        for b in range(self.B):                              # what no row may see
            self.kv[self.cu_k[b] + self.k_lens[b]:self.cu_k[b + 1]] = float("nan")
        self.kv[self.cu_k[-1]:] = float("inf")

    def run(self, spa, back=True, inputs=None):
        C, Ck, H, Hk, Dh, B = self.H * self.Dh, self.Hk * self.Dh, self.H, self.Hk, self.Dh, self.B
        i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()
        nan = lambda *s, dt=self.td: torch.full(s, float("nan"), dtype=dt, device="cuda")
        q, kv, dout = (self.q.cuda(), self.kv.cuda(), self.dout.cuda()) if inputs is None else inputs
        cu_q, cu_k, lens = i32(self.cu_q), i32(self.cu_k), None if self.key_lens is None else self.key_lens.cuda()
        code = spa.dtype_code(q)
        work = lambda n: torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
        qs, ks, vs = q[:, :C], kv[:, :Ck], kv[:, Ck:2 * Ck]
        out, lse = nan(self.rows_q, C), nan(H, B * self.max_q, dt=torch.float32)
        spa.spa_cross_attention(qs, ks, vs, cu_q, cu_k, lens, B, self.max_q, self.max_k, H, Hk, Dh, out, lse,
                                work(spa.spa_cross_attention_workspace_bytes(B, self.max_q, self.max_k, H, Hk, Dh, code)), self.softmax_scale)
        res = dict(out=out, lse=lse)
        if back:
            dq, dkv = nan(*q.shape), nan(*kv.shape)
            spa.spa_cross_attention_bwd(qs, ks, vs, out, dout, lse, cu_q, cu_k, lens, B, self.max_q, self.max_k, H, Hk, Dh, dq[:, :C], dkv[:, :Ck],
                                        dkv[:, Ck:2 * Ck], work(spa.spa_cross_attention_bwd_workspace_bytes(B, self.max_q, self.max_k, H, Hk, Dh, code)),
                                        self.softmax_scale)
            res.update(dq=dq, dkv=dkv)
        return res

    def check(self, res, back=True):
        H, Hk, Dh, G, half = self.H, self.Hk, self.Dh, self.H // self.Hk, self.half
        C, Ck, bf = H * Dh, Hk * Dh, half if self.td == torch.bfloat16 else 0.0
        got = {n: t.cpu().double() for n, t in res.items()}
        q64, kv64, do64 = self.q.double(), self.kv.double(), self.dout.double()

        def near(name, have, want, tol):
            err = (have - want).abs()
            assert bool((err <= tol + 2.0 ** -100).all()), (name, float((err - tol).max()), float(err.max()))

        for b in range(self.B):
            i, j, n, m = slice(self.cu_q[b], self.cu_q[b + 1]), slice(self.cu_k[b], self.cu_k[b] + self.k_lens[b]), self.q_lens[b], self.k_lens[b]
            behind = slice(self.cu_k[b] + m, self.cu_k[b + 1])
            if back:
                assert bool((got["dkv"][behind, :2 * Ck] == 0).all())
            if n == 0 or m == 0:
                assert bool((got["out"][i] == 0).all()) and bool((got["lse"][:, i] == -np.inf).all())
                if back:
                    assert bool((got["dq"][i, :C] == 0).all()) and bool((got["dkv"][j, :2 * Ck] == 0).all())
                continue
            for hk in range(Hk):
                col = slice(hk * Dh, (hk + 1) * Dh)
                k, v = kv64[j, col], kv64[j, Ck + hk * Dh:Ck + (hk + 1) * Dh]
                dk, dv, tk, tv, sk, sv = (torch.zeros(m, Dh, dtype=torch.float64) for _ in range(6))
                for h in range(hk * G, (hk + 1) * G):
                    qc = slice(h * Dh, (h + 1) * Dh)
                    q, dO = q64[i, qc], do64[i, qc]
                    S = q @ k.T * self.scale
                    lse = torch.logsumexp(S, 1)
                    P = torch.exp(S - lse[:, None])
                    O = P @ v
                    eS = (Dh + 4) * U * self.scale * (q.abs() @ k.abs().T).max()
                    eP = float(2 * eS + 2.0 ** -15 + 2.0 ** -22 * S.abs().max())
                    to = (P @ v.abs()) * (2 * eP + bf + m * U) + half * O.abs()
                    near("out", got["out"][i, qc], O, to)
                    near("lse", got["lse"][h, i], lse, eS + 2.0 ** -20 * (1 + lse.abs()) + eP)
                    if not back:
                        continue
                    D, dP = (dO * O).sum(1, keepdim=True), dO @ v.T
                    dS = P * (dP - D)
                    tS = dS.abs() * (eP + bf) + P * ((dO.abs() * to).sum(1, keepdim=True) + (Dh + 4) * U * ((dO.abs() @ v.abs().T) + (dO.abs() * O.abs()).sum(1, keepdim=True)))
                    dq = dS @ k * self.scale
                    near("dq", got["dq"][i, qc], dq, self.scale * (tS @ k.abs() + m * U * (dS.abs() @ k.abs())) + half * dq.abs())
                    dk += dS.T @ q * self.scale
                    dv += P.T @ dO
                    tk += self.scale * (tS.T @ q.abs() + n * G * U * (dS.abs().T @ q.abs()))
                    tv += P.T @ dO.abs() * (eP + bf + n * G * U)
                if back:
                    near("dk", got["dkv"][j, col], dk, tk + half * dk.abs())
                    near("dv", got["dkv"][j, Ck + hk * Dh:Ck + (hk + 1) * Dh], dv, tv + half * dv.abs())
        # nothing else is written
        Tq, Tk = int(self.cu_q[-1]), int(self.cu_k[-1])
        assert bool(torch.isnan(got["out"][Tq:]).all()) and bool(torch.isnan(got["lse"][:, Tq:]).all())
        if back:
            assert bool(torch.isnan(got["dq"][Tq:]).all()) and bool(torch.isnan(got["dq"][:, C:]).all())
            assert bool(torch.isnan(got["dkv"][Tk:]).all()) and bool(torch.isnan(got["dkv"][:, 2 * Ck:]).all())


BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@BOTH
@pytest.mark.parametrize("Dh", [32, 64])
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 4), (6, 2), (8, 1), (7, 1)])
def test_heads(spa, dtype, Dh, H, Hk):
    c = Case([40, 9, 130], [77, 20, 33], H, Hk, Dh, dtype, seed=H)
    c.check(c.run(spa))


@BOTH
@pytest.mark.parametrize("nq", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
@pytest.mark.parametrize("nk", [1, 32, 65, 128, 200])
def test_edges(spa, dtype, nq, nk):
    """Every edge of the waves' and the steps' rows, on both sides."""
    c = Case([nq], [nk], 2, 2, 32, dtype, seed=nq + nk)
    c.check(c.run(spa))


@BOTH
@pytest.mark.parametrize("nq", [1, 3, 17])
@pytest.mark.parametrize("nk", [31, 33, 63, 64, 127, 129, 255, 1000])
def test_few_queries(spa, dtype, nq, nk):
    c = Case([nq] * 3, [nk, max(nk - 30, 1), 1], 4, 2, 64, dtype, seed=nk)
    c.check(c.run(spa))


@BOTH
def test_empty_segments(spa, dtype):
    for q_lens, k_lens in (([0, 5, 0, 40], [3, 0, 0, 70]), ([0], [0]), ([0], [50]), ([50], [0]), ([200, 1], [0, 1])):
        c = Case(q_lens, k_lens, 4, 2, 32, dtype)
        c.check(c.run(spa))


@BOTH
@pytest.mark.parametrize("held", [77, 128, 300])
def test_padded_states(spa, dtype, held):
    """Keys of a padded batch: what lies behind key_lens is never read, and has no gradient."""
    c = Case([100, 7, 0, 33, 64], [77, 0, 5, 64, 1], 6, 3, 64, dtype, held=held, seed=held)
    c.check(c.run(spa))


@BOTH
def test_longer_bounds_and_wider_rows(spa, dtype):
    c = Case([30, 45], [60, 100], 4, 2, 64, dtype, more_q=500, more_k=700, pad=16)
    c.check(c.run(spa))
    c = Case([3, 45], [600, 100], 2, 2, 32, dtype, more_q=3, more_k=5000, pad=8, scale=0.3)
    c.check(c.run(spa))


@BOTH
@pytest.mark.parametrize("q_lens,k_lens,H,Hk", [([1], [9001], 4, 1), ([1, 2], [5000, 513], 8, 8), ([20], [3000], 1, 1), ([40], [2049], 2, 2),
                                                ([100, 3], [4000, 1], 2, 1), ([3000], [40], 2, 2), ([2500, 1, 800], [20, 60, 0], 4, 2), ([1500], [1500], 1, 1)])
def test_split(spa, dtype, q_lens, k_lens, H, Hk):
    """Few units and long rows on one side: split over workgroups and joined."""
    c = Case(q_lens, k_lens, H, Hk, 64, dtype, seed=sum(q_lens))
    code = spa.SPA_BF16 if dtype == "bf16" else spa.SPA_F32
    sizes = (c.B, c.max_q, c.max_k, H, Hk, 64, code)
    plain = ((H * c.B * c.max_q * 4) + 255) // 256 * 256
    assert spa.spa_cross_attention_workspace_bytes(*sizes) > 0 or spa.spa_cross_attention_bwd_workspace_bytes(*sizes) > plain
    c.check(c.run(spa))


@BOTH
def test_many_segments(spa, dtype):
    g = torch.Generator().manual_seed(3)
    lens = lambda n, top: torch.randint(0, top, (n,), generator=g).tolist()
    c = Case(lens(300, 40), lens(300, 50), 2, 1, 32, dtype)
    c.check(c.run(spa))


@pytest.mark.parametrize("Dh,H,Hk,top", [(64, 4, 4, 256), (32, 8, 4, 128), (64, 32, 4, 30), (32, 4, 4, 97)])
@pytest.mark.parametrize("held", [None, 128, 77])
def test_units_of_one_workgroup(spa, Dh, H, Hk, top, held):
    """More units than compute units, of up to 256 rows and 128 keys: every number of blocks of rows beside every number of blocks of keys."""
    g = torch.Generator().manual_seed(top)
    pick = lambda most, n: [0, 1, most] + torch.randint(0, most + 1, (n - 3,), generator=g).tolist()
    c = Case(pick(top, 66), pick(held or 128, 66)[::-1], H, Hk, Dh, held=held, seed=top)
    assert c.B * Hk >= 256 and c.max_q * (H // Hk) <= 256 and c.max_k <= 128
    c.check(c.run(spa))


@pytest.mark.parametrize("size", [30.0, 3000.0])
def test_large_scores_in_one_workgroup(spa, size):
    c = Case([60, 33, 9], [90, 64, 5], 2, 1, 64, size=size)
    c.check(c.run(spa))


@BOTH
@pytest.mark.parametrize("size", [8.0, 300.0, 1e4])
def test_large_scores(spa, dtype, size):
    """Rows whose largest score is far from zero: next to one-hot rows."""
    c = Case([70, 5], [90, 300], 2, 1, 64, dtype, size=size)
    c.check(c.run(spa))


def test_gradient_against_differences(spa):
    """fp32 gradients along random directions against central differences of the 64-bit form (errors h^2 of the third derivative, and fp32's)."""
    c = Case([9, 4], [12, 30], 4, 2, 32, "f32")
    res = c.run(spa)
    C, Ck, G = 4 * 32, 2 * 32, 2

    def value(q, kv):
        total = 0.0
        for b in range(2):
            i, j = slice(c.cu_q[b], c.cu_q[b + 1]), slice(c.cu_k[b], c.cu_k[b + 1])
            for h in range(4):
                hk = h // G
                P = torch.softmax(q[i, h * 32:(h + 1) * 32] @ kv[j, hk * 32:(hk + 1) * 32].T * c.scale, 1)
                total = total + ((P @ kv[j, Ck + hk * 32:Ck + (hk + 1) * 32]) * c.dout[i, h * 32:(h + 1) * 32].double()).sum()
        return float(total)

    g, h = torch.Generator().manual_seed(1), 1e-4
    q, kv = c.q.double(), c.kv.double()
    dq, dkv = torch.nan_to_num(res["dq"].cpu().double()), torch.nan_to_num(res["dkv"].cpu().double())
    for _ in range(5):
        vq, vk = torch.randn(q.shape, generator=g, dtype=torch.float64), torch.randn(kv.shape, generator=g, dtype=torch.float64)
        vk[c.cu_k[-1]:] = 0
        num = (value(q + h * vq, kv + h * vk) - value(q - h * vq, kv - h * vk)) / (2 * h)
        have, size = float((dq * vq).sum() + (dkv * vk).sum()), float((dq * vq).abs().sum() + (dkv * vk).abs().sum())
        assert abs(num - have) <= 2e-5 * size


def test_values_that_are_not_finite_stay_in_their_rows(spa):
    """A NaN in a query makes that query's head NaN, an infinity in a value the column of the rows that see it."""
    c = Case([50, 60], [70, 90], 2, 2, 32)
    clean = c.run(spa, back=False)
    c.q[7, 3] = float("nan")
    c.kv[75, 2 * 32 + 32 + 5] = float("inf")          # a value of segment 1, head 1
    got = c.run(spa, back=False)["out"]
    want = clean["out"].clone()
    assert bool(torch.isnan(got[7, :32]).all()) and bool(torch.isinf(got[50:110, 37]).all())
    got[7, :32] = want[7, :32]
    got[50:110, 37] = want[50:110, 37]
    assert torch.equal(torch.nan_to_num(got.float()), torch.nan_to_num(want.float()))


def test_offsets_past_32_bits(spa):
    """Row strides that put the last rows past 2^31 elements, of keys, queries and gradients."""
    stride = 1 << 25
    c = Case([80], [75], 1, 1, 32)
    want = c.run(spa)
    wide = lambda rows: torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)
    kv, dkv = wide(76), wide(76)
    q = c.q.cuda()
    kv[:75, :64] = c.kv.cuda()[:75]
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32).cuda()
    out, lse, dq = torch.empty_like(want["out"]), torch.empty(1, 80, device="cuda"), torch.empty_like(want["dq"])
    spa.spa_cross_attention(q, kv[:, :32], kv[:, 32:64], i32(0, 80), i32(0, 75), None, 1, 80, 75, 1, 1, 32, out, lse)
    ws = torch.empty(spa.spa_cross_attention_bwd_workspace_bytes(1, 80, 75, 1, 1, 32, 1), dtype=torch.uint8, device="cuda")
    spa.spa_cross_attention_bwd(q, kv[:, :32], kv[:, 32:64], out, c.dout.cuda(), lse, i32(0, 80), i32(0, 75), None, 1, 80, 75, 1, 1, 32, dq, dkv[:, :32],
                                dkv[:, 32:64], ws)
    assert torch.equal(out[:80], want["out"][:80]) and torch.equal(dq[:80], want["dq"][:80])
    assert torch.equal(dkv[:75, :64], want["dkv"][:75])


def test_rows_without_a_place_are_left(spa):
    """Segments that are longer than max_q, max_k say, and rows from B max_q on: neither computed nor written."""
    c = Case([6, 4], [20, 30], 2, 2, 32)
    C, Ck, i32 = 64, 64, lambda *a: torch.tensor(a, dtype=torch.int32).cuda()
    q, kv, dout = torch.zeros(20, C, dtype=torch.bfloat16).cuda(), c.kv.cuda(), torch.zeros(20, C, dtype=torch.bfloat16).cuda()
    q[4:14], dout[4:14] = c.q[:10].cuda(), c.dout[:10].cuda()
    want = c.run(spa)
    nan = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device="cuda")
    out, lse, dq, dkv = nan(20, C), nan(2, 12 + 4, dt=torch.float32), nan(20, C), nan(*kv.shape)
    cu_q, cu_k, args = i32(4, 10, 14), i32(0, 20, 50), (None, 2, 6, 30, 2, 2, 32)                # 12 rows have a place: 4 .. 11
    spa.spa_cross_attention(q, kv[:, :Ck], kv[:, Ck:], cu_q, cu_k, *args, out, lse)
    assert torch.equal(out[4:12], want["out"][:8]) and bool(torch.isnan(out[12:]).all()) and bool(torch.isnan(out[:4]).all())
    ws = torch.zeros(spa.spa_cross_attention_bwd_workspace_bytes(2, 6, 30, 2, 2, 32, 1), dtype=torch.uint8, device="cuda")
    spa.spa_cross_attention_bwd(q, kv[:, :Ck], kv[:, Ck:], out, dout, lse, cu_q, cu_k, *args, dq, dkv[:, :Ck], dkv[:, Ck:], ws)
    assert torch.equal(dq[4:12], want["dq"][:8]) and bool(torch.isnan(dq[12:]).all())
    assert torch.equal(dkv[:20], want["dkv"][:20])                                              # (of the first segment nothing is cut)
    args = (None, 2, 5, 25, 2, 2, 32)                                                           # the first segment's sixth row, five keys of the second
    out, lse = nan(20, C), nan(2, 16, dt=torch.float32)
    spa.spa_cross_attention(c.q.cuda(), kv[:, :Ck], kv[:, Ck:], i32(0, 6, 10), cu_k, *args, out, lse)
    assert torch.equal(out[:5], want["out"][:5]) and bool(torch.isnan(out[5]).all())
    short = Case([6, 4], [20, 25], 2, 2, 32)
    short.q, short.kv = c.q, torch.cat((c.kv[:45], c.kv[50:]))
    assert torch.equal(out[6:10], short.run(spa, back=False)["out"][6:10])


def _same(a, b):
    return all(torch.equal(torch.nan_to_num(a[n].float()), torch.nan_to_num(b[n].float())) for n in a)


@pytest.mark.parametrize("q_lens,k_lens", [([300, 200], [77, 50]), ([2, 2], [3000, 700]), ([60, 40], [50, 77])])
def test_replayed_and_repeated(spa, q_lens, k_lens):
    """Captured, replayed with other inputs and eager work between: bit for bit the eager results, which are the same in every run."""
    c, other = Case(q_lens, k_lens, 4, 2, seed=1), Case(q_lens, k_lens, 4, 2, seed=2)
    inputs = (c.q.cuda(), c.kv.cuda(), c.dout.cuda())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(spa, inputs=inputs)
    torch.cuda.synchronize()
    # (what a run makes beside the calls is made before the capture)
    C, Ck, i32 = 4 * 64, 2 * 64, lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()
    cu_q, cu_k = i32(c.cu_q), i32(c.cu_k)
    out, dq, dkv = (torch.zeros_like(t) for t in (inputs[0], inputs[0], inputs[1]))
    lse = torch.zeros(4, c.B * c.max_q, device="cuda")
    sizes = (c.B, c.max_q, c.max_k, 4, 2, 64)
    ws = [torch.empty(max(f(*sizes, 1), 1), dtype=torch.uint8, device="cuda") for f in (spa.spa_cross_attention_workspace_bytes, spa.spa_cross_attention_bwd_workspace_bytes)]

    def calls():
        q, k, v = inputs[0], inputs[1][:, :Ck], inputs[1][:, Ck:]
        spa.spa_cross_attention(q, k, v, cu_q, cu_k, None, *sizes, out, lse, ws[0])
        spa.spa_cross_attention_bwd(q, k, v, out, inputs[2], lse, cu_q, cu_k, None, *sizes, dq, dkv[:, :Ck], dkv[:, Ck:], ws[1])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    Tq, Tk = int(c.cu_q[-1]), int(c.cu_k[-1])
    for rep in range(4):
        src = (c, other)[rep % 2]
        for t, s in zip(inputs, (src.q, src.kv, src.dout)):
            t.copy_(s.cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = src.run(spa)
        torch.cuda.synchronize()
        assert torch.equal(out[:Tq], want["out"][:Tq]) and torch.equal(dq[:Tq], want["dq"][:Tq]) and torch.equal(dkv[:Tk], want["dkv"][:Tk]), rep
    assert _same(c.run(spa), c.run(spa))


def test_threads(spa):
    cases = [Case([100, 30], [77, 40], 4, 2, seed=0), Case([1], [6000], 2, 1, seed=1), Case([60], [40], 2, 2, 32, "f32", seed=2), Case([500], [20], 2, 2, 32, seed=3)]
    want = [c.run(spa) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def calls(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got = cases[i].run(spa)
                    torch.cuda.current_stream().synchronize()
                    if not _same(got, want[i]):
                        wrong.append(i)
        except Exception as e:
            wrong.append((i, e))

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]
