"""README.md's step over pages with the library: pages that run out, slots that end, and what neither may write, eagerly and captured."""
import pytest

from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from readme_step import D, LENS, N_NEW, N_PAGES, PER, SCENES, VOCAB, Scene, code  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("name", SCENES)
def test_no_page_of_another_slot_is_written(name, captured):
    cb = binding.octopus_build_codebooks(D, 3)
    scene = Scene(name, binding, DEV, cb, cb.plan.granules)
    scene.names["ws"] = torch.empty(binding.octopus_pages_workspace(N_PAGES, len(LENS), PER), dtype=torch.uint8, device=DEV)
    scene.names["ws_verify"] = torch.empty(binding.octopus_verify_workspace(len(LENS), N_NEW - 1, VOCAB), dtype=torch.uint8, device=DEV)
    step = code()
    exec(step, scene.names)
    torch.cuda.synchronize()
    written = scene.check()
    assert (written == 0) == (name == "pages run out")
    if captured:
        scene.restore()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            exec(step, scene.names)
        for _ in range(3):
            scene.restore()
            graph.replay()
            torch.cuda.synchronize()
            assert scene.check() == written
            exec(step, scene.names)              # (an eager step between, on what the replay left)
            torch.cuda.synchronize()
