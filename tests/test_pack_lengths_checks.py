"""What spa_pack_lengths refuses before anything is launched (no GPU)."""
import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def call(**k):
    a = dict(lens=F, B=3, N=7, cu=F, gather=F, inv=F, total=F)
    a.update(k)
    return lib.spa_pack_lengths(*a.values(), None)


def test_refusals():
    for name in ("lens", "cu", "gather", "inv", "total"):
        assert call(**{name: None}) == -1 and "null" in lib.spa_last_error().decode()
    assert call(B=0) == -1 and call(N=0) == -1 and call(B=65536, N=32768) == -1
    assert call(B=65536, N=1) == -1 and "65535" in lib.spa_last_error().decode()
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in lib.spa_last_error().decode()


def test_the_binding_compares_types_and_sizes():
    t = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    ok = dict(lens=t(3), N=7, cu_seqlens=t(4), gather_idx=t(21), inv_pos=t(21), total=t(1))
    for over, match in ((dict(lens=t(3, torch.int64)), "lens must be"), (dict(cu_seqlens=t(3)), "cu_seqlens holds"), (dict(gather_idx=t(20)), "gather_idx holds"),
                        (dict(inv_pos=t(20)), "inv_pos holds"), (dict(total=t(0)), "total holds"), (dict(lens=t(6)[::2]), "contiguous"), (dict(), "device tensors")):
        with pytest.raises(ValueError, match=match):
            spa.spa_pack_lengths(**{**ok, **over})
