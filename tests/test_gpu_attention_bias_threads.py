"""Threads that call the attention with a position bias with maps of different sizes at the same time."""
import threading

import pytest
import torch

from test_gpu_attention_bias import Case, spa  # noqa: F401 (spa: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_threads_with_maps_of_their_own(spa, dtype):  # noqa: F811
    """Two and two take the same kernels with different shares of LDS, from a thread and a stream each: every result is that of
    the calls one after the other."""
    grids = ((10, 11), (24, 25), (40, 41), (44, 45))
    cases = [Case([90, 40], grid, 2, 32, dtype, seed=i) for i, grid in enumerate(grids)]
    want = [c.run(spa) for c in cases]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(len(cases))

    def calls(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(30)
                for _ in range(50):
                    got = cases[i].run(spa)
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(got[n], want[i][n]) for n in got):
                        wrong.append((i, "other results"))
        except Exception as e:                                   # (a call's error ends the thread, not the test)
            wrong.append((i, e))

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]
