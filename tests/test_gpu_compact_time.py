"""A pool's compaction takes no longer because the pool is a page smaller: the form in one launch, whose time grows with the pool, ends before the
form in several is faster by half.  Launches in a captured graph, the shortest of several runs."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = "cuda:0"


def microseconds(n_pages):
    refs = torch.from_numpy((np.random.default_rng(0).random(n_pages) < 0.5).astype(np.int32)).to(DEV)
    state, page_map, moves = refs.clone(), torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.zeros(2 + n_pages, dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.octopus_pages_workspace(n_pages, 1, 1), dtype=torch.uint8, device=DEV)

    def call():
        state.copy_(refs)                                       # (a kernel of 2 us, in both)
        binding.octopus_pages_compact(state, page_map, moves, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(20):
            call()
    best = float("inf")
    for _ in range(10):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        best = min(best, begin.elapsed_time(end) * 1000 / 20)
    return best


@pytest.mark.parametrize("n_pages", [4096, 16384, 32768, 65536])
def test_a_smaller_pool_takes_no_longer(n_pages):
    assert microseconds(n_pages) < 1.75 * microseconds(70000)
