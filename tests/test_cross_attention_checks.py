"""What the calls of the attention to another sequence refuse before anything is launched (no GPU)."""
import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def msg():
    return lib.spa_last_error().decode()


SIZES = dict(B=2, max_q=20, max_k=3000, H=4, Hk=2, Dh=32, dtype=1)
NEED = lib.spa_cross_attention_workspace_bytes(*SIZES.values())
NEED_BWD = lib.spa_cross_attention_bwd_workspace_bytes(*SIZES.values())


def fwd(**k):
    a = dict(q=F, k=F, v=F, qs=128, ks=64, vs=64, cuq=F, cuk=F, lens=F, **SIZES, scale=0.0, out=F, lse=F, ws=F, bytes=NEED)
    a.update((n, v) for n, v in k.items() if n in a)
    return lib.spa_cross_attention(*a.values(), None)


def bwd(**k):
    a = dict(q=F, k=F, v=F, qs=128, ks=64, vs=64, out=F, dout=F, lse=F, cuq=F, cuk=F, lens=F, **SIZES, scale=0.0, dq=F, dk=F, dv=F, dqs=128, dks=64,
             dvs=64, ws=F, bytes=NEED_BWD)
    a.update(k)
    return lib.spa_cross_attention_bwd(*a.values(), None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_common_refusals(call):
    for name in ("q", "k", "v", "cuq", "cuk", "out"):
        assert call(**{name: None}) == -1 and "null" in msg()
    for name in ("q", "k", "v", "out"):
        assert call(**{name: F + 8}) == -1 and "aligned" in msg()
    for name in ("B", "max_q", "max_k", "H", "Hk"):
        assert call(**{name: 0}) == -1
    assert call(Hk=3) == -1 and "multiple" in msg()
    assert call(B=65536) == -1 and call(B=65535, max_q=40000) == -1 and call(B=65535, max_k=40000) == -1
    assert call(max_q=2 ** 30, H=8, Hk=2, qs=512) == -1 and "max_q" in msg()
    assert call(B=60000, max_q=30000, max_k=30000, H=256, Hk=256, qs=8192, ks=8192, vs=8192, dqs=8192, dks=8192, dvs=8192) == -1 and "workgroups" in msg()
    assert call(dtype=5) == -2 and call(Dh=48) == -2
    assert call(qs=127) == -1 and call(qs=132) == -1 and call(ks=63) == -1 and call(vs=1 << 31) == -1
    for scale in (-1.0, float("nan"), float("inf")):
        assert call(scale=scale) == -1 and "softmax_scale" in msg()
    assert call(ws=None) == -3 and call(bytes=64) == -3 and "workspace" in msg()
    assert call(ws=F + 16) == -1 and "256" in msg()
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in msg()


def test_particular_refusals():
    assert NEED > 0 and NEED_BWD > 0
    for name in ("dout", "lse", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == -1 and "null" in msg()
    assert bwd(dqs=127) == -1 and bwd(dks=60) == -1 and bwd(dvs=68) == -1
    size = lib.spa_cross_attention_workspace_bytes
    assert size(2, 20, 100, 4, 2, 32, 1) == 0                   # (short keys are not split)
    for f in (size, lib.spa_cross_attention_bwd_workspace_bytes):
        assert f(0, 20, 100, 4, 2, 32, 1) == f(2, 20, 100, 4, 3, 32, 1) == f(2, 20, 100, 4, 2, 48, 1) == f(2, 20, 100, 4, 2, 32, 2) == 0


def test_the_binding_compares_types_and_sizes():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt=bf: torch.zeros(shape, dtype=dt)
    ok = dict(q=t((9, 128)), k=t((30, 64)), v=t((30, 64)), cu_seqlens_q=t(3, i32), cu_seqlens_k=t(3, i32), key_lens=t(2, i32), B=2, max_q=8, max_k=20, H=4,
              Hk=2, Dh=32, out=t((9, 128)), lse=t((4, 16), f32), workspace=None)
    call = lambda **k: spa.spa_cross_attention(**{**ok, **k})
    for over, match in ((dict(k=t((30, 64), f32)), "share one dtype"), (dict(q=t((9, 64))), "q must be"), (dict(v=t((30, 128))), "v must be"),
                        (dict(cu_seqlens_k=t(2, i32)), "cu_seqlens_k holds"), (dict(key_lens=t(1, i32)), "key_lens holds"), (dict(key_lens=t(2)), "key_lens must be"),
                        (dict(lse=t((4, 15), f32)), "lse holds"), (dict(out=t((9, 256))[:, :128]), "contiguous"), (dict(out=t((8, 128))), "out must be"), (dict(v=t((29, 64))), "v must be"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            call(**over)
    more = dict(dout=t((9, 128)), dq=t((9, 128)), dk=t((30, 64)), dv=t((30, 64)))
    back = lambda **k: spa.spa_cross_attention_bwd(**{**ok, **more, **k})
    for over, match in ((dict(dk=t((30, 128))), "dk must be"), (dict(dv=t((29, 64))), "dv must be"), (dict(dq=t((8, 128))), "dq must be"), (dict(dout=t((8, 128))), "dout must be"), (dict(dq=t((9, 128), f32)), "share one dtype"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            back(**over)
