"""What the calls of the gated feed-forward block refuse before anything is launched (no GPU)."""
import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def msg():
    return lib.spa_last_error().decode()


def fwd(**k):
    a = dict(x=F, idx=F, total=F, W=F, bias=F, M=8, K=64, F=72, act=0, dtype=1, h=F, pre=F)
    a.update((n, v) for n, v in k.items() if n in a)
    return lib.spa_gated_linear_packed(*a.values(), None)


def bwd(**k):
    a = dict(x=F, idx=F, stride=64, total=F, W=F, pre=F, M=8, K=64, F=72, act=0, dtype=1, h=F)
    a.update(k)
    return lib.spa_gated_linear_packed_bwd(*a.values(), None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_refusals(call):
    for name in ("x", "W", "h"):
        assert call(**{name: None}) == -1 and "null" in msg()
        assert call(**{name: F + 8}) == -1 and "aligned" in msg()
    assert call(pre=F + 4) == -1 and "aligned" in msg()
    for name in ("M", "K", "F"):
        assert call(**{name: 0}) == -1
    assert call(F=1 << 30) == -1
    assert call(M=2 ** 31 - 1) == -1 and call(M=2 ** 31 - 600, K=8, F=8, stride=8) == -1 and "tiles" in msg()
    assert call(act=2) == -1 and "activation" in msg()
    assert call(dtype=3) == -2 and call(K=60) == -2 and call(F=76) == -2 and "multiples of 8" in msg()
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in msg()


def test_particular_refusals():
    assert bwd(pre=None) == -1 and "null" in msg()
    assert bwd(stride=63) == -1 and bwd(stride=68) == -2 and bwd(stride=1 << 31) == -1


def test_the_binding_compares_types_and_sizes():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt=bf: torch.zeros(shape, dtype=dt)
    ok = dict(x=t((20, 64)), gather_idx=t(8, i32), total=t(1, i32), W=t((144, 64)), bias=t(144), act=0, h=t((8, 72)), pre=t((8, 144)))
    call = lambda **k: spa.spa_gated_linear_packed(**{**ok, **k})
    for over, match in ((dict(W=t((144, 64), f32)), "share one dtype"), (dict(W=t((143, 64))), "W must be"), (dict(W=t((144, 72))), "W must be"), (dict(h=t((8, 80))), "h must be"),
                        (dict(pre=t((7, 144))), "pre must be"), (dict(bias=t(143)), "bias holds"), (dict(gather_idx=t(7, i32)), "gather_idx holds"),
                        (dict(gather_idx=None, x=t((7, 64))), "x holds"), (dict(h=t((8, 144))[:, :72]), "contiguous"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            call(**over)
    ok = dict(dy=t((20, 64)), dy_idx=t(8, i32), total=t(1, i32), W_down=t((64, 72)), pre=t((8, 144)), act=0, d_pre=t((8, 144)))
    call = lambda **k: spa.spa_gated_linear_packed_bwd(**{**ok, **k})
    for over, match in ((dict(dy=t((20, 72))), "dy must be"), (dict(dy=t((7, 64)), dy_idx=None), "dy must be"), (dict(pre=t((7, 144))), "pre must be"), (dict(d_pre=t((8, 72))), "d_pre must be"),
                        (dict(dy_idx=t(7, i32)), "dy_idx holds"), (dict(pre=t((8, 144), f32)), "share one dtype"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            call(**over)
