"""Without a GPU: pools and moves in the memory of several devices are refused."""
import pytest

torch = pytest.importorskip("torch")

from paper_2605_21226_amd import binding  # noqa: E402


class Reached(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def f(*_):
            raise Reached
        return f


def test_pools_and_moves_of_one_device(monkeypatch):
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    here, moves = torch.zeros((10, 4, 16), dtype=torch.uint8), torch.zeros(12, dtype=torch.int32)
    there = here.to("meta")
    for bad in ([here, there], [there, here, here]):
        with pytest.raises(AssertionError):
            binding.page_pools(bad)
    for pools in (binding.page_pools([here, here.clone()]), binding.page_pools([there])):
        for at in ("cpu", "meta"):
            with pytest.raises(Reached if at == pools.tensors[0].device.type else AssertionError):
                binding.octopus_pages_copy(pools, moves.to(at))
