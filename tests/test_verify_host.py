"""Without a GPU: what octopus_verify_drafts refuses, its workspace, and the definition that its GPU tests go by."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding
from test_serve_host import EINVAL, EUNSUPPORTED, EWORKSPACE, FAKE, lib, refuses  # noqa: F401
from verify_model import verify

VERIFY = "target dtype ts tp draft qs qp draft_tokens draft_lens uniforms n_seq n_draft vocab tokens_out accepted ws ws_bytes stream"


def test_refusals(lib):  # noqa: F811
    need = lib.octopus_verify_workspace(4, 3, 1000)
    assert need > 0 and lib.octopus_verify_workspace(5, 3, 1000) >= need and lib.octopus_verify_workspace(4, 4, 10 ** 6) >= need
    good = dict(target=FAKE, dtype=0, ts=4000, tp=1000, draft=FAKE, qs=3000, qp=1000, draft_tokens=FAKE, draft_lens=FAKE, uniforms=FAKE, n_seq=4, n_draft=3,
                vocab=1000, tokens_out=FAKE, accepted=FAKE, ws=FAKE, ws_bytes=need - 1, stream=None)
    shapes = [{name: n} for name, bad in (("n_seq", (0, -1, 65536)), ("n_draft", (-1, (1 << 20) + 1)), ("vocab", (0, -1, (1 << 30) + 1))) for n in bad]
    refuses(lib.octopus_verify_drafts, VERIFY, good, [
        ({}, EWORKSPACE), ({"ws": None, "ws_bytes": need}, EWORKSPACE), ({"ws": FAKE + 128, "ws_bytes": need}, EWORKSPACE),
        ({"draft": None, "qs": -1, "draft_lens": None}, EWORKSPACE), ({"n_draft": 0, "draft_tokens": None, "draft": None}, EWORKSPACE),
        ({"dtype": 1, "target": FAKE + 2, "draft": FAKE + 2}, EWORKSPACE), ({"ts": 0, "tp": 0, "qs": 0, "qp": 0}, EWORKSPACE),
        *[({name: None}, EINVAL) for name in ("target", "draft_tokens", "uniforms", "tokens_out", "accepted")],
        *[(bad, EINVAL) for bad in shapes], *[({name: -1}, EINVAL) for name in ("ts", "tp", "qs", "qp")],
        *[({name: FAKE + 2}, EINVAL) for name in ("target", "draft", "draft_tokens", "draft_lens", "uniforms", "tokens_out", "accepted")],
        ({"dtype": 1, "target": FAKE + 1}, EINVAL), ({"dtype": 1, "draft": FAKE + 1}, EINVAL), ({"dtype": 2}, EUNSUPPORTED), ({"dtype": -1}, EUNSUPPORTED)])
    for bad in shapes:
        f = {**dict(n_seq=4, n_draft=3, vocab=1000), **bad}
        assert lib.octopus_verify_workspace(f["n_seq"], f["n_draft"], f["vocab"]) == 0


def test_what_the_python_call_refuses(monkeypatch):
    torch = pytest.importorskip("torch")

    class Reached(Exception):
        pass

    class Library:
        def octopus_verify_drafts(self, *_):
            raise Reached
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    good = dict(target=torch.zeros(2, 4, 9), draft=torch.zeros(2, 3, 9), draft_tokens=ints(2, 3), uniforms=torch.zeros(2, 4), tokens_out=ints(2, 4),
                n_accepted=ints(2), workspace=torch.zeros(8, dtype=torch.uint8), draft_lens=ints(2))
    for more in ({}, {"draft": None}, {"draft_lens": None}, {"target": torch.zeros(4, 2, 20)[:, :, 3:12].transpose(0, 1)},
                 {"target": torch.zeros(2, 1, 9), "draft": None, "draft_tokens": None, "uniforms": torch.zeros(2, 1), "tokens_out": ints(2, 1)}):
        with pytest.raises(Reached):
            binding.octopus_verify_drafts(**{**good, **more})
    for bad in ({"target": torch.zeros(2, 9, 4).transpose(1, 2)}, {"draft": torch.zeros(2, 9, 3).transpose(1, 2)}, {"draft": torch.zeros(2, 4, 9)},
                {"draft": torch.zeros(2, 3, 8)}, {"draft": torch.zeros(2, 3, 9).bfloat16()}, {"draft_tokens": ints(2, 4)}, {"draft_tokens": ints(2, 3).long()},
                {"draft_tokens": ints(3, 2).t()}, {"uniforms": torch.zeros(2, 3)}, {"uniforms": torch.zeros(2, 4).double()}, {"uniforms": torch.zeros(4, 2).t()},
                {"tokens_out": ints(2, 3)}, {"tokens_out": ints(2, 4).long()}, {"tokens_out": ints(4, 2).t()}, {"n_accepted": ints(1)}, {"n_accepted": ints(2).long()},
                {"draft_lens": ints(1)}, {"target": torch.zeros(2, 4, 9).half(), "draft": None}):
        with pytest.raises((AssertionError, TypeError)):
            binding.octopus_verify_drafts(**{**good, **bad})


def test_the_definition_keeps_the_targets_distribution():
    """Exactly, for dyadic rows: over all values of both random numbers on a grid the first token comes out p(v) of the time."""
    p, q, n = np.array([0.5, 0.125, 0.375, 0.0]), np.array([0.25, 0.5, 0.125, 0.125]), 64
    target, count = np.stack([p, p]), np.zeros(4)
    for x in range(4):
        for i in range(n):
            for j in range(n):
                tokens, _ = verify(target, q[None], [x], np.array([i / n, j / n]), 1)
                count[tokens[0]] += q[x] / n ** 2
    assert np.abs(count - p).max() <= 1.5 / n        # (borders of the grid: half a step of each number)
