"""The gradients that LayerTrainPass hands out: one of every parameter that the last run had, None for the others, however that run was issued."""
import pytest
import torch

from test_gpu_layer import Inputs

pytestmark = pytest.mark.gpu

ABSENT = [(), ("b_in", "b_out"), ("b_out",), ("gamma_q", "gamma_cross_k", "gamma_ffn"), ("gamma_self", "gamma_k", "gamma_cross", "gamma_cross_q", "b_in")]


@pytest.fixture(scope="module")
def pipeline():
    from paper_2410_23608_amd import pipeline as mod
    return mod


def _without(i, names):
    return dict(i.params, **{n: None for n in names})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("absent", ABSENT)
def test_none_where_the_parameter_is(pipeline, dtype, absent):
    i = Inputs(pipeline, "small", dtype)
    i.params = _without(i, absent)
    p = i.make(pipeline, True)
    for t in p.grad_list:
        t.fill_(float("nan"))
    for _ in range(3):                                                       # call by call, then recorded
        p.run(*i.args(True))
        torch.cuda.synchronize()
        assert list(p.grads) == list(p.PARAMS)
        for name, g in p.grads.items():
            assert (g is None) == (i.params[name] is None), name
            assert g is None or bool(torch.isfinite(g).all()), name
    assert p._plan is not None


def test_the_last_run_decides(pipeline):
    """Runs with and without some of the parameters in turn, each recorded, and the launches called one by one."""
    i = Inputs(pipeline, "small", "bf16")
    p, all_params = i.make(pipeline, True), i.params
    for k in range(8):
        absent = ABSENT[(0, 1, 3)[k // 2 % 3]]
        i.params = _without(i, absent) if absent else all_params
        p.run(*i.args(True))
        assert tuple(n for n, g in p.grads.items() if g is None) == tuple(n for n in p.PARAMS if n in absent), k
        i.params = all_params
    st = p.stages(i.x, i.w, i.states, i.key_lens, *(None if n == "b_in" else all_params[n] for n in p.PARAMS), i.labels, i.dy)
    for _, fn in st:
        fn()
    torch.cuda.synchronize()
    assert [n for n, g in p.grads.items() if g is None] == ["b_in"]
