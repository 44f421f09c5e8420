"""The shape of the table's gradient (no GPU)."""
import pytest
import torch

from paper_2410_23608_amd import spa


def test_a_table_gradient_with_other_rows_than_the_table_is_refused():
    """Its rows would be written one behind the other as the table's are, not in its own."""
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda shape, dt: torch.zeros(shape, dtype=dt)
    q, table, buckets = t((40, 64), bf), t((2, 9), bf), t(63, i32)
    args = (q, q, q, q, q, t((2, 40), f32), t(3, i32), None, table, buckets, (4, 5), 2, 20, 2, 32, q, q, q)
    with pytest.raises(ValueError, match="rows of 9 entries"):
        spa.spa_packed_attention_bias_bwd(*args, t((2, 12), f32), None)
    for fits in (t((2, 9), f32), t(18, f32), t(30, f32)):
        with pytest.raises(ValueError, match="device tensors"):
            spa.spa_packed_attention_bias_bwd(*args, fits, None)
