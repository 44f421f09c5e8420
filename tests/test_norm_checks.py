"""What the norms' entry points refuse, before anything is launched (no GPU): through the C-ABI and through the binding."""
import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def msg():
    return lib.spa_last_error().decode()


def front(**k):
    a = dict(x=F, idx=F, total=F, gamma=F, beta=F, kind=0, eps=1e-6, M=8, C=64, dtype=1, packed=F, stats=F)
    a.update(k)
    return lib.spa_norm_packed(*a.values(), None)


def behind(**k):
    a = dict(z=F, inv=F, res=F, gamma=F, beta=F, scale=F, gate=F, kind=1, eps=0.0, M=8, rows=16, C=64, dtype=0, y=F, stats=F)
    a.update(k)
    return lib.spa_norm_residual_unpack(*a.values(), None)


def front_bwd(**k):
    a = dict(da=F, x=F, inv=F, total=F, gamma=F, kind=0, stats=F, res=F, M=8, rows=16, C=64, dtype=1, dx=F, dgamma=F, dbeta=F, ws=F,
             bytes=lib.spa_norm_bwd_workspace_bytes(16, 64, 1))
    a.update(k)
    return lib.spa_norm_packed_bwd(*a.values(), None)


def behind_bwd(**k):
    a = dict(dy=F, z=F, idx=F, inv=F, total=F, gamma=F, beta=F, scale=F, gate=F, kind=0, stats=F, M=8, rows=16, C=64, dtype=1, dz=F,
             ds=F, dgamma=F, dbeta=F, dscale=F, ws=F, bytes=lib.spa_norm_bwd_workspace_bytes(8, 64, 1))
    a.update(k)
    return lib.spa_norm_residual_unpack_bwd(*a.values(), None)


@pytest.mark.parametrize("call,required", [(front, ("x", "packed")), (behind, ("z", "y")), (front_bwd, ("da", "x", "stats", "dx")),
                                           (behind_bwd, ("dy", "z", "stats", "dz"))])
def test_common_refusals(call, required):
    for name in required:
        assert call(**{name: None}) == -1 and "null" in msg()
    assert call(kind=2) == -1 and "kind" in msg()
    assert call(dtype=7) == -2 and "dtype" in msg()
    assert call(C=0) == -1
    assert call(C=66, dtype=0) == -1 and "multiple of 16" in msg()
    assert call(C=8200) == -2 and "8192" in msg()
    assert call(M=0) == -1 and "M_cap" in msg()
    assert call(gamma=F + 8) == -1 and "aligned" in msg()
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in msg()            # (and the group is over)


def test_particular_refusals():
    for eps in (-1e-6, float("nan"), float("inf")):
        assert front(eps=eps) == -1 and "eps" in msg()
        assert behind(eps=eps) == -1 and "eps" in msg()
    assert behind(rows=0) == -1 and behind(rows=2 ** 31) == -1
    assert front_bwd(bytes=lib.spa_norm_bwd_workspace_bytes(16, 64, 1) - 1) == -3 and "workspace" in msg()
    assert front_bwd(ws=None) == -3
    assert behind_bwd(bytes=lib.spa_norm_bwd_workspace_bytes(8, 64, 1) - 1) == -3
    assert behind_bwd(idx=None) == -1 and "together" in msg()
    assert behind_bwd(inv=None) == -1 and "together" in msg()
    assert behind_bwd(idx=None, inv=None, M=17, bytes=1 << 20) == -1 and "packed rows" in msg()
    assert behind_bwd(gate=None) == -1 and "gate_scores" in msg()
    assert lib.spa_norm_bwd_workspace_bytes(0, 64, 1) == 0 and lib.spa_norm_bwd_workspace_bytes(5, 0, 1) == 0
    a = (F, F, 0.0, F, None, F, None, F, 1.0, 1, 8, 8, 1, F, F, F, F, F, 1 << 20, None)
    assert lib.spa_gate_bwd_scores(*a) == -1 and "d_scores" in msg()
    assert lib.spa_group_begin() == 0
    assert lib.spa_gate_bwd_scores(*a) == -2 and "group" in msg()


def test_the_binding_compares_types_and_sizes():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt: torch.zeros(shape, dtype=dt)
    cap, C = 32, 64
    x, packed, idx, total, st = t((2, 16, C), bf), t((cap, C), bf), t(cap, i32), t(1, i32), t((2, cap), f32)
    with pytest.raises(ValueError, match="share one dtype"):
        spa.spa_norm_packed(x, idx, total, t(C, f32), None, 0, 1e-6, packed)
    with pytest.raises(ValueError, match="stats holds"):
        spa.spa_norm_packed(x, idx, total, None, None, 0, 1e-6, packed, t((1, cap), f32))
    with pytest.raises(ValueError, match="gather_idx holds"):
        spa.spa_norm_packed(x, t(cap - 1, i32), total, None, None, 0, 1e-6, packed)
    with pytest.raises(ValueError, match="x holds"):
        spa.spa_norm_packed(x, None, None, None, None, 0, 1e-6, t((cap + 1, C), bf))
    with pytest.raises(ValueError, match="gamma holds"):
        spa.spa_norm_packed(x, idx, total, t(C - 8, bf), None, 0, 1e-6, packed)
    with pytest.raises(ValueError, match="device tensors"):
        spa.spa_norm_packed(x, idx, total, None, None, 0, 1e-6, packed)
    with pytest.raises(ValueError, match="residual"):
        spa.spa_norm_residual_unpack(packed, idx, t((2, 15, C), bf), None, None, None, None, 0, 1e-6, x)
    with pytest.raises(ValueError, match="gate_scores must be torch.float32"):
        spa.spa_norm_residual_unpack(packed, idx, x, None, None, None, t((2, 16), bf), 0, 1e-6, x)
    with pytest.raises(ValueError, match="inv_pos holds"):
        spa.spa_norm_residual_unpack(packed, t(cap - 1, i32), x, None, None, None, None, 0, 1e-6, x)
    with pytest.raises(ValueError, match="dgamma must be torch.float32"):
        spa.spa_norm_packed_bwd(packed, x, idx, total, None, 0, st, None, x, t(C, bf), None, None)
    with pytest.raises(ValueError, match="d_scores holds"):
        spa.spa_norm_residual_unpack_bwd(x, packed, idx, idx, total, None, None, None, t((2, 16), f32), 0, st, packed,
                                         t(cap - 1, f32), None, None, None, None)
    with pytest.raises(ValueError, match="d_scores must be torch.float32"):
        spa.spa_gate_bwd_scores(x, t(C, bf), 0.0, t((2, 16), f32), None, t((2, 16), torch.uint8), t((2, 16), bf), None, 1.0, t(1, f32),
                                x, t(C, f32), t(1, f32), None)
