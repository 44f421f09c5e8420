"""bf16 products count the steps of a contraction in an int: longer ones are refused before anything is launched (no GPU)."""
import pytest

from paper_2410_23608_amd import spa

lib = spa.lib
F = 4096                                        # a pointer that is never read
LONG = 2 ** 31 - 56                             # the shortest multiple of 8 whose last step would pass 2^31


def forward(k):
    return lib.spa_linear_packed(F, None, None, None, F, None, 4, k, 8, 1, F, 8, None)


def unpack(k):
    return lib.spa_linear_packed_unpack(F, None, F, None, 4, k, 8, 1, F, F, 4, F, F, None)


def scatter(k):
    return lib.spa_linear_packed_scatter(F, None, F, None, 4, k, 8, 1, F, F, F, 8, None)


def input_side(k):
    return lib.spa_linear_packed_bwd_input(F, None, k, None, F, 4, 8, k, 1, None, None, 0, F, 8, None)


def gated(k):
    return lib.spa_gated_linear_packed(F, None, None, F, None, 4, k, 8, 0, 1, F, None, None)


def gated_bwd(k):
    return lib.spa_gated_linear_packed_bwd(F, None, k, None, F, F, 4, k, 8, 0, 1, F, None)


@pytest.mark.parametrize("call", [forward, unpack, scatter, input_side, gated, gated_bwd])
def test_refused(call):
    for k in (LONG, 2 ** 31 - 8):
        assert call(k) == -1
        assert "2^31 - 64" in lib.spa_last_error().decode()
