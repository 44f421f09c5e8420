"""fp32 projections with a short contraction, a thread an element, against the tiles that longer ones and larger results take (tests/test_f32_shape.py asks the rule for
these sizes): every element is one chain over the contraction, so it has the same bits inside a call of more columns."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOKENS = 1500                                   # of which ROWS are selected
ROWS, LIVE = 1000, 930


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


class Inputs:
    def __init__(self, K, N):
        g = torch.Generator(device="cuda").manual_seed(K)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        chosen = torch.randperm(TOKENS, generator=g, device="cuda")[:ROWS].sort()[0]
        self.idx, self.inv = chosen.int(), torch.full((TOKENS,), -1, dtype=torch.int32, device="cuda")
        self.inv[chosen[:LIVE]] = torch.arange(LIVE, dtype=torch.int32, device="cuda")
        self.total = torch.tensor([LIVE], dtype=torch.int32, device="cuda")
        self.x, self.tokens, self.scores, self.W, self.b = rnd(ROWS, K), rnd(TOKENS, K), rnd(TOKENS), rnd(N, K), rnd(N)
        self.res, self.d, self.d_tokens = rnd(TOKENS, N), rnd(ROWS, K), rnd(TOKENS, K)          # (K: the contraction of the input side, too)


def nan(*shape):
    return torch.full(shape, float("nan"), device="cuda")


def same(small, large):
    assert small.shape == large.shape and torch.equal(small.contiguous().view(torch.int32), large.contiguous().view(torch.int32))


@pytest.mark.parametrize("K,few", [(1, 64), (3, 16), (4, 1), (8, 4), (8, 33), (16, 3)])
def test_forward(spa, K, few):
    i, many = Inputs(K, 512), 512
    res, b, W = i.res[:, :few].contiguous(), i.b[:few].contiguous(), i.W[:few].contiguous()
    for gather, gate, bias in ((None, None, True), (i.idx, None, False), (i.idx, i.scores, True)):
        x = i.x if gather is None else i.tokens
        out = [nan(ROWS, n) for n in (few, many)]
        spa.spa_linear_packed(x, gather, gate, i.total, W, b if bias else None, out[0])
        spa.spa_linear_packed(x, gather, gate, i.total, i.W, i.b if bias else None, out[1])
        same(out[0][:LIVE], out[1][:LIVE, :few])
        assert bool(torch.isnan(out[0][LIVE:]).all()) and not bool(torch.isnan(out[0][:LIVE]).any())
        want = (x if gather is None else x[gather.long()]).double()[:LIVE]
        want = (want * torch.sigmoid(gate[gather.long()][:LIVE].double())[:, None] if gate is not None else want) @ W.double().T + (b.double() if bias else 0)
        # (K fused steps and the bias, each rounded once, the gate's factor by 2^-22, of sums of the magnitudes; operands below 6)
        assert float((out[0][:LIVE].double() - want).abs().max()) <= (K + 6) * 2.0 ** -24 * (36 * K + 6)
    y = [nan(TOKENS, n) for n in (few, many)]
    spa.spa_linear_packed_unpack(i.x, i.total, W, b, i.idx, i.inv, res, y[0])
    spa.spa_linear_packed_unpack(i.x, i.total, i.W, i.b, i.idx, i.inv, i.res, y[1])
    same(y[0], y[1][:, :few])
    assert torch.equal(y[0][i.inv < 0], res[i.inv < 0])
    y = [nan(TOKENS, n) for n in (few, many)]
    spa.spa_linear_packed_scatter(i.x, i.total, W, None, i.idx, res, y[0])
    spa.spa_linear_packed_scatter(i.x, i.total, i.W, None, i.idx, i.res, y[1])
    on = i.inv >= 0
    same(y[0][on], y[1][on][:, :few])
    assert bool(torch.isnan(y[0][~on]).all())


@pytest.mark.parametrize("kc,few", [(1, 64), (4, 16), (8, 1), (8, 33), (16, 4)])
def test_input_side(spa, kc, few):
    i, many = Inputs(kc, 4000), 4000
    W = i.W.T.contiguous()                                                   # [kc, columns]
    part = W[:, :few].contiguous()
    out = [nan(ROWS, n) for n in (few, many)]
    for o, w in zip(out, (part, W)):
        spa.spa_linear_packed_bwd_input(i.d, None, i.total, w, ROWS, None, None, o)
    same(out[0][:LIVE], out[1][:LIVE, :few])
    assert bool(torch.isnan(out[0][LIVE:]).all())
    assert float((out[0][:LIVE].double() - i.d[:LIVE].double() @ part.double()).abs().max()) <= (kc + 2) * 2.0 ** -24 * 36 * kc
    out = [nan(TOKENS, n) for n in (few, many)]
    for o, w in zip(out, (part, W)):
        spa.spa_linear_packed_bwd_input(i.d_tokens, i.idx, i.total, w, ROWS, i.idx, i.inv, o)
    same(out[0], out[1][:, :few])
    assert bool((out[0][i.inv < 0] == 0).all()) and not bool(torch.isnan(out[0]).any())


@pytest.mark.parametrize("M,live", [(1, 1), (4, 3), (4, 0), (8, 8)])
def test_weight_side(spa, M, live):
    g = torch.Generator(device="cuda").manual_seed(M)
    d, x, scores = torch.randn(20, 1500, generator=g, device="cuda"), torch.randn(20, 1500, generator=g, device="cuda"), torch.randn(20, generator=g, device="cuda")
    idx = torch.randperm(20, generator=g, device="cuda")[:M].int()
    total = torch.tensor([live], dtype=torch.int32, device="cuda")
    for gate in (None, scores):
        sizes = ((70, 33), (1500, 1500))
        dW, db = [nan(*s) for s in sizes], [nan(s[0]) for s in sizes]
        for (n, k), w, b in zip(sizes, dW, db):
            spa.spa_linear_packed_bwd_weight(d[:, :n], idx, x[:, :k].contiguous(), idx, gate, total, M, w, b)
        if M > 1:                                                            # (one row: a thread an element for both)
            same(dW[0], dW[1][:70, :33])
            same(db[0], db[1][:70])
        rows = idx[:live].long()
        xs = x[rows, :33].double() * (1 if gate is None else torch.sigmoid(scores[rows].double())[:, None])
        assert float((dW[0].double() - d[rows, :70].double().T @ xs).abs().max()) <= (M + 6) * 2.0 ** -24 * 36 * M
        assert float((db[0].double() - d[rows, :70].double().sum(0)).abs().max()) <= M * 2.0 ** -24 * 6 * M
        w = nan(70, 33)
        spa.spa_linear_packed_bwd_weight(d[:, :70], idx, x[:, :33].contiguous(), idx, gate, total, M, w, None)
        same(w, dW[0])
