"""The packing index of padded batches (spa_pack_lengths) against spa_pack of a mask of the same places, and against the definition."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spa():
    from paper_2410_23608_amd import spa as mod
    return mod


class Index:
    def __init__(self, B, N):
        full = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")
        self.cu, self.idx, self.inv, self.total = full(B + 1), full(B * N), full(B * N), full(1)

    def tensors(self):
        return self.cu, self.idx, self.inv, self.total


@pytest.mark.parametrize("B,N", [(1, 1), (1, 5000), (3, 7), (64, 77), (5, 1024), (4, 1025), (300, 130), (2000, 3), (65535, 2)])
@pytest.mark.parametrize("kind", ["random", "none", "all", "past"])
def test_index(spa, B, N, kind):
    g = torch.Generator().manual_seed(B * N)
    lens = {"random": torch.randint(0, N + 1, (B,), generator=g), "none": torch.zeros(B), "all": torch.full((B,), N),
            "past": torch.randint(-N, 3 * N + 1, (B,), generator=g)}[kind].to(torch.int32).cuda()
    have, want = Index(B, N), Index(B, N)
    spa.spa_pack_lengths(lens, N, *have.tensors())
    n = lens.clamp(0, N).long()
    mask = torch.arange(N, device="cuda") < n[:, None]
    spa.spa_pack(None, mask.to(torch.uint8), None, None, 0, None, *want.tensors())
    T = int(n.sum())
    assert torch.equal(have.cu, want.cu) and torch.equal(have.inv, want.inv) and torch.equal(have.idx, want.idx)
    assert int(have.total) == T and int(have.cu[-1]) == T
    assert torch.equal(have.idx[:T].long(), mask.view(-1).nonzero().view(-1)) and bool((have.idx[T:] == -7).all())


def test_replayed(spa):
    B, N = 9, 200
    lens, have = torch.zeros(B, dtype=torch.int32, device="cuda"), Index(B, N)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        spa.spa_pack_lengths(lens, N, *have.tensors())
    for rep in range(4):
        lens.copy_(torch.randint(0, N + 1, (B,), generator=torch.Generator().manual_seed(rep), dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = Index(B, N)
        spa.spa_pack_lengths(lens, N, *want.tensors())
        T = int(want.total)
        assert torch.equal(have.cu, want.cu) and torch.equal(have.inv, want.inv) and torch.equal(have.idx[:T], want.idx[:T]) and int(have.total) == T == int(lens.sum())
