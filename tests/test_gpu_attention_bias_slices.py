"""The table gradient on maps taken in slices, with more rows or blocks than the slices keep lists of."""
import pytest

from test_gpu_attention_bias import Case, spa  # noqa: F401 (spa: the fixture)

pytestmark = pytest.mark.gpu


# A segment of more than 64 tiles of queries beside short ones; more blocks a workgroup than it keeps
# the tiles of (4 workgroups a head: 1.96 million offsets); more segments than are ranked
@pytest.mark.parametrize("grid,lens,H,dtype", [((50, 84), [4170, 70, 0, 9], 1, "bf16"), ((70, 60), [4161, 33], 1, "f32"),
                                               ((700, 700), [12 + i % 7 for i in range(200)], 8, "bf16"),
                                               ((700, 700), [9 + i % 5 for i in range(150)], 8, "f32"),
                                               ((50, 84), [3 + i % 61 for i in range(300)], 2, "bf16"),
                                               ((50, 84), [3 + i % 61 for i in range(300)], 2, "f32")])
def test_slices_without_lists(spa, grid, lens, H, dtype):  # noqa: F811
    c = Case(lens, grid, H, 32, dtype, seed=len(lens))
    c.check(c.run(spa))
