"""Without a GPU: what octopus_append_paged does in Python before it reaches the library, since a single token's call waits for it."""
import sys

import pytest

torch = pytest.importorskip("torch")

from paper_2605_21226_amd import binding  # noqa: E402


def test_no_function_between_the_call_and_the_library(monkeypatch):
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *_: reached.append(name) or 0

    library, cb = Library(), binding.octopus_build_codebooks(128, 3)
    monkeypatch.setattr(binding, "load", lambda: library)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    qkv, zeros = torch.zeros((2, 1, 48, 128), dtype=torch.bfloat16), lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    q, k, v = qkv.split([32, 8, 8], dim=2)
    args = (cb, k, v, zeros(8, 4), torch.zeros(8 * 4096 * 2, dtype=torch.uint8), torch.zeros((2, 8, 64, 128), dtype=torch.bfloat16), 2, zeros(2, 1))
    rope, more = torch.zeros((9, 64, 2)), dict(start_pos=zeros(2), q=q, q_out=torch.zeros((2, 1, 32, 128), dtype=torch.bfloat16))
    calls = []
    sys.setprofile(lambda frame, event, _: calls.append(frame.f_code.co_name) if event == "call" and frame.f_code.co_filename == binding.__file__ else None)
    try:
        binding.octopus_append_paged(*args, rope=rope, **more)
    finally:
        sys.setprofile(None)
    assert reached == ["octopus_append_paged"]
    assert set(calls) == {"octopus_append_paged", "_check_pools", "_dtype_code", "_ptr"}, calls
    binding.octopus_append_paged_axes(*args, rope, bytes(64), zeros(2, 1, 3), **more)
    assert reached == ["octopus_append_paged", "octopus_append_paged_axes"]
