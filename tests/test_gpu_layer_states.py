"""A layer's states behind key_lens (LayerPass, LayerTrainPass): nothing reads them, whatever they hold."""
import pytest
import torch

from test_gpu_layer import Inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pipeline():
    from paper_2410_23608_amd import pipeline as mod
    return mod


def results(p):
    torch.cuda.synchronize()
    return {n: t.clone() for n, t in dict(p.grads, y=p.y, dx=p.dx, d_states=p.d_states, dw=p.dw, db=p.db, loss=p.loss).items() if t is not None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["small", "image"])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), 3e38])
def test_what_lies_behind_is_not_read(pipeline, shape, dtype, fill):
    """The same bits as with zeros there, in the run that goes call by call and in the recorded one."""
    i = Inputs(pipeline, shape, dtype)
    behind = torch.arange(i.s["L"], device="cuda") >= i.key_lens[:, None]
    assert bool(behind[1].all()) and bool(behind.any()) and not bool(behind.all())
    i.states[behind] = 0
    p = i.make(pipeline, True)
    p.run(*i.args(True))
    want = results(p)
    assert all(bool(torch.isfinite(t).all()) for t in want.values())
    y = i.make(pipeline, False).run(*i.args(False)).clone()
    i.states[behind] = fill
    q, infer = i.make(pipeline, True), i.make(pipeline, False)
    for _ in range(3):
        q.run(*i.args(True))
        have = results(q)
        assert have.keys() == want.keys()
        for name in want:
            assert torch.equal(have[name], want[name]), name
        assert torch.equal(infer.run(*i.args(False)), y) and torch.equal(y, want["y"])
    assert q._plan is not None
    assert bool((q.d_states.view(*behind.shape, -1)[behind] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_states_without_lengths(pipeline, dtype):
    """key_lens None: every state counts, as with lengths of L; sums over rows in the same order."""
    i = Inputs(pipeline, "small", dtype)
    i.key_lens = torch.full_like(i.key_lens, i.s["L"])
    p = i.make(pipeline, True)
    p.run(*i.args(True))
    want = results(p)
    i.key_lens = None
    q = i.make(pipeline, True)
    for _ in range(3):
        q.run(*i.args(True))
        have = results(q)
        for name in want:
            assert torch.equal(have[name], want[name]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_state_counts(pipeline, dtype):
    """All lengths 0 and NaN in every state: the attention adds nothing, what belongs to the states has gradients of 0."""
    i = Inputs(pipeline, "image", dtype)
    i.key_lens.zero_()
    i.states.fill_(float("nan"))
    p, infer = i.make(pipeline, True), i.make(pipeline, False)
    for _ in range(3):
        p.run(*i.args(True))
        have = results(p)
        assert all(bool(torch.isfinite(t).all()) for t in have.values())
        for name in ("gamma_cross_k", "W_cross_kv", "d_states", "gamma_cross_q", "W_cross_q", "W_cross_o"):
            assert bool((have[name] == 0).all()), name
        assert torch.equal(infer.run(*i.args(False)), have["y"])
