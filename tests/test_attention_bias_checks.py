"""What the attention with a position bias refuses before anything is launched (no GPU), and its bucket map."""
import pytest
import torch

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read


def msg():
    return lib.spa_last_error().decode()


def fwd(**k):
    a = dict(q=F, k=F, v=F, qs=192, ks=192, vs=192, cu=F, gidx=F, table=F, buckets=F, nb=9, gh=4, gw=5, B=2, n_max=20, H=2, Dh=32, dtype=1,
             scale=0.0, out=F, lse=F)
    a.update(k)
    return lib.spa_packed_attention_bias(*a.values(), None)


NEED = lib.spa_attention_bias_bwd_workspace_bytes(2, 20, 2, 32, 4, 5, 1)


def bwd(**k):
    a = dict(q=F, k=F, v=F, qs=192, ks=192, vs=192, out=F, dout=F, lse=F, cu=F, gidx=F, table=F, buckets=F, nb=9, gh=4, gw=5, B=2, n_max=20,
             H=2, Dh=32, dtype=1, scale=0.0, dq=F, dk=F, dv=F, dqs=192, dks=192, dvs=192, d_table=F, ws=F, bytes=NEED)
    a.update(k)
    return lib.spa_packed_attention_bias_bwd(*a.values(), None)


@pytest.mark.parametrize("call,required", [(fwd, ("q", "k", "v", "cu", "table", "out")),
                                           (bwd, ("q", "k", "v", "cu", "table", "out", "dout", "lse", "dq", "dk", "dv"))])
def test_refusals(call, required):
    for name in required:
        assert call(**{name: None}) == -1 and "null" in msg()
    for name in ("B", "n_max", "H"):
        assert call(**{name: 0}) == -1
    assert call(dtype=3) == -2 and call(Dh=48) == -2 and "head dim" in msg()
    assert call(qs=32) == -1 and "row stride" in msg()
    assert call(ks=196) == -1 and "16 bytes" in msg()
    assert call(vs=1 << 24) == -1
    assert call(k=F + 8) == -1 and "aligned" in msg()
    assert call(scale=float("nan")) == -1 and call(scale=-1.0) == -1 and "softmax_scale" in msg()
    assert call(gh=0) == -1 and call(gw=-1) == -1 and call(gh=8192, gw=8192) == -1 and "grid_h" in msg()
    assert call(gh=3) == -1 and "max_seqlen exceeds" in msg()
    assert call(nb=0) == -1 and "n_buckets" in msg()
    assert call(buckets=None) == -1 and "bucket per offset" in msg()
    assert lib.spa_group_begin() == 0
    assert call() == -2 and "group" in msg()


def test_refusals_of_the_backward():
    assert bwd(dqs=32) == -1 and bwd(dks=196) == -1 and bwd(dv=F + 2) == -1
    assert bwd(ws=None) == -3 and bwd(bytes=NEED - 1) == -3 and "workspace" in msg()
    assert bwd(ws=F + 16) == -1 and "256" in msg()
    assert lib.spa_attention_bias_bwd_workspace_bytes(0, 20, 2, 32, 4, 5, 1) == 0
    assert lib.spa_attention_bias_bwd_workspace_bytes(2, 20, 2, 32, 4, 0, 1) == 0


def test_the_binding_compares_types_and_sizes():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt: torch.zeros(shape, dtype=dt)
    H, Dh, B, n, grid = 2, 32, 2, 20, (4, 5)
    q, out, cu, table, lse = t((40, 64), bf), t((40, 64), bf), t(3, i32), t((H, 63), bf), t((H, 40), f32)
    call = lambda **k: spa.spa_packed_attention_bias(*{**dict(q=q, k=q, v=q, cu=cu, gidx=None, table=table, buckets=None, grid=grid, B=B, n=n,
                                                              H=H, Dh=Dh, out=out, lse=lse), **k}.values())
    with pytest.raises(ValueError, match="device tensors"):
        call()
    with pytest.raises(ValueError, match="share one dtype"):
        call(table=t((H, 63), f32))
    with pytest.raises(ValueError, match="table must be"):
        call(table=t((3, 63), bf))
    with pytest.raises(ValueError, match="buckets must be torch.int32"):
        call(buckets=t(63, torch.int64))
    with pytest.raises(ValueError, match="buckets holds"):
        call(buckets=t(62, i32))
    with pytest.raises(ValueError, match="lse holds"):
        call(lse=t((H, 39), f32))
    with pytest.raises(ValueError, match="contiguous"):
        call(table=t((63, H), bf).t())
    args = (q, q, q, out, out, lse, cu, None, table, None, grid, B, n, H, Dh, q, q, q)
    with pytest.raises(ValueError, match="d_table must be torch.float32"):
        spa.spa_packed_attention_bias_bwd(*args, t((H, 63), bf), None)
    with pytest.raises(ValueError, match="d_table holds"):
        spa.spa_packed_attention_bias_bwd(*args, t((H, 62), f32), None)


def test_bucket_map():
    m, n = spa.relative_position_buckets(5, 9, near=2, levels=3, far=6)
    assert m.shape == ((2 * 5 - 1) * (2 * 9 - 1),) and m.dtype == torch.int32 and n == 100
    m = m.view(9, 17)
    cols = (m[4] - m[4, 8]).tolist()              # offsets -8 .. 8 along a row: 0 and 1 apart, then widening, signs apart
    assert cols[8:] == [0, 1, 2, 3, 3, 4, 4, 4, 4]
    assert cols[:8] == [b + 5 for b in cols[:8:-1]]
    rows = ((m[:, 8] - m[4, 8]) // 10).tolist()
    assert rows[4:] == [0, 1, 2, 3, 3] and rows[:4] == [b + 5 for b in rows[:4:-1]]
    assert int(m.min()) >= 0 and int(m.max()) < n
    one, n1 = spa.relative_position_buckets(1, 1)
    assert one.shape == (1,) and 0 <= int(one[0]) < n1
    for bad in ((0, 3), (3, 0), (3, 3, 0), (3, 3, 2, 0)):
        with pytest.raises(ValueError):
            spa.relative_position_buckets(*bad)
