"""What the calls of the normed and rotated heads refuse before anything is launched (no GPU), and the table of angles."""
import math

import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def msg():
    return lib.spa_last_error().decode()


def fwd(**k):
    a = dict(q=F, k=F, qs=128, ks=64, idx=F, total=F, gq=F, bq=F, gk=F, bk=F, kind=0, eps=1e-6, table=F, pt=0, ph=8, t=1, h=4, w=5, layout=0, M=8,
             H=4, Hk=2, Dh=32, dtype=1, qo=F, ko=F, qos=128, kos=64)
    a.update(k)
    return lib.spa_qk_norm_rotary(*a.values(), None)


NEED = lib.spa_qk_norm_rotary_bwd_workspace_bytes(8, 4, 2, 32, 1)


def bwd(**k):
    a = dict(dqo=F, dko=F, dqos=128, dkos=64, q=F, k=F, qs=128, ks=64, idx=F, total=F, gq=F, gk=F, kind=0, eps=1e-6, table=F, pt=0, ph=8, t=1, h=4,
             w=5, layout=0, M=8, H=4, Hk=2, Dh=32, dtype=1, dq=F, dk=F, qos=128, kos=64, dgq=F, dbq=F, dgk=F, dbk=F, ws=F, bytes=NEED)
    a.update(k)
    return lib.spa_qk_norm_rotary_bwd(*a.values(), None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_common_refusals(call):
    for name in ("q", "k"):
        assert call(**{name: None}) == -1 and "null" in msg()
        assert call(**{name: F + 8}) == -1 and "aligned" in msg()
    assert call(kind=3) == -1 and "kind" in msg()
    assert call(kind=2) == -1 and "belong to a norm" in msg()
    assert call(dtype=2) == -2 and call(Dh=48) == -2 and call(Dh=128) == -2
    assert call(M=0) == -1 and call(H=0) == -1 and call(Hk=-1) == -1 and call(H=257, qs=1 << 20, qos=1 << 20) == -2
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(eps=eps) == -1 and "eps" in msg()
    assert call(layout=2) == -1 and "layout" in msg()
    assert call(gq=F + 4) == -1 and call(table=F + 8) == -1 and "aligned" in msg()
    assert call(t=0) == -1 and call(h=0) == -1 and call(w=0) == -1 and call(t=1 << 11, h=1 << 10, w=1 << 10) == -1
    assert call(pt=-1) == -1 and call(ph=-1) == -1 and call(pt=9, ph=8) == -1 and call(pt=2 ** 31 - 1, ph=2 ** 31 - 1) == -1
    assert call(qs=127) == -1 and call(qs=132) == -1 and "16 bytes" in msg()
    assert call(qs=1 << 31) == -1 and call(kos=63) == -1
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in msg()


def test_particular_refusals():
    assert fwd(qo=None) == -1 and fwd(ko=None) == -1 and bwd(dqo=None) == -1 and bwd(dko=None) == -1 and bwd(dq=None) == -1
    assert bwd(bytes=NEED - 1) == -3 and bwd(ws=None) == -3
    assert bwd(kind=2, gq=None, gk=None) == -1 and "belong" in msg()
    assert fwd(qs=256) == -1 and "in place" in msg() and fwd(ks=128) == -1 and "in place" in msg()
    assert bwd(qs=256) == -1 and "in place" in msg() and bwd(dkos=128) == -1 and "in place" in msg() and bwd(dqos=256) == -1 and "in place" in msg()
    assert bwd(Hk=0, bytes=NEED) == -1 and "without k" in msg()
    size = lib.spa_qk_norm_rotary_bwd_workspace_bytes
    assert size(0, 4, 2, 32, 1) == size(8, 0, 2, 32, 1) == size(8, 4, -1, 32, 1) == size(8, 4, 2, 48, 1) == size(8, 4, 2, 32, 3) == 0
    assert size(2 ** 31 - 1, 256, 256, 64, 0) == 1024 * 2 * 64 * 4


def test_the_table():
    t = spa.rotary_table((2, 7, 5), 32, (4, 5), 50.0)
    assert t.shape == (7, 16, 2) and t.dtype == torch.float32
    counts = (4, 5, 7)
    for p in (0, 1, 6):
        i = 0
        for n in counts:
            for m in range(n):
                a = p * 50.0 ** (-m / n)
                assert t[p, i, 0] == torch.tensor(math.cos(a)).float() and t[p, i, 1] == torch.tensor(math.sin(a)).float()
                i += 1
    for bad in (dict(grid=(0, 1, 1)), dict(grid=(1, 1)), dict(pairs=(9, 8)), dict(pairs=(-1, 0)), dict(base=0.0), dict(base=float("nan"))):
        with pytest.raises(ValueError):
            spa.rotary_table(**{**dict(grid=(1, 2, 2), Dh=32, pairs=(0, 8), base=10.0), **bad})


def test_the_binding_compares_types_and_sizes():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt=bf: torch.zeros(shape, dtype=dt)
    ok = dict(q=t((8, 128)), k=t((8, 64)), gather_idx=t(8, i32), total=t(1, i32), gamma_q=t(32), beta_q=None, gamma_k=t(32), beta_k=None, kind=1,
              eps=1e-6, table=t((5, 16, 2), f32), pairs=(0, 8), grid=(1, 4, 5), H=4, Hk=2, Dh=32, q_out=t((8, 128)), k_out=t((8, 64)))
    call = lambda **k: spa.spa_qk_norm_rotary(**{**ok, **k})
    for over, match in ((dict(k=t((8, 64), f32)), "share one dtype"), (dict(gamma_q=t(32, f32)), "share one dtype"), (dict(q=t((8, 96))), "q must be"),
                        (dict(k_out=None), "must be given"), (dict(Hk=0), "no k"), (dict(gather_idx=t(7, i32)), "gather_idx holds"),
                        (dict(table=t((4, 16, 2), f32)), "table holds"), (dict(table=t((5, 16, 2))), "table must be"), (dict(gamma_k=t(31)), "gamma_k holds"),
                        (dict(grid=(4, 5)), "grid must be"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            call(**over)
