"""Without a GPU: README.md's step over pages, run on models of its calls.  Where a slot did not grow, because pages ran out or it ended, its row
names no pages for new tokens, and what is appended there would go to pages of others."""
import pytest

torch = pytest.importorskip("torch")

from pages_model import TILE, Pages  # noqa: E402
from readme_step import LENS, N_NEW, SCENES, Scene, code  # noqa: E402


class Calls:
    """The library's calls, as sequential Python on tensors."""

    def page_pools(self, pools):
        return pools

    def octopus_pages_update(self, refs, table, lens, new_lens, moves, ws, source=None, keep_lens=None):
        x = Pages(refs.tolist(), table.tolist(), lens.tolist())
        x.update(new_lens.tolist(), source.tolist(), keep_lens.tolist())
        for tensor, value in ((refs, x.refs), (table, x.table), (lens, x.lens)):
            tensor.copy_(torch.from_numpy(value))
        flat = [len(x.moves), x.missing, *(p for pair in x.moves for p in pair)]
        moves[:len(flat)] = torch.tensor(flat)

    def octopus_pages_copy(self, pools, moves):
        for a, b in moves[2:2 + 2 * int(moves[0])].view(-1, 2).tolist():
            for pool in pools:
                pool[b] = pool[a]

    def octopus_append_paged_axes(self, cb, k, v, signs, k_pool, v_pool, n_pages, table, rope, axis, pos, start_pos=None, new_lens=None, q=None, q_out=None):
        for s in range(len(k)):
            for t in range(k.shape[1] if new_lens is None else min(max(int(new_lens[s]), 0), k.shape[1])):
                slot = int(start_pos[s]) + t
                q_out[s, t] = -q[s, t]
                if slot < TILE * table.shape[1]:
                    page = min(max(int(table[s, slot // TILE]), 0), n_pages - 1)
                    k_pool[page, :, :, slot % TILE] += 1
                    v_pool[page, :, slot % TILE] = v[s, t]

    def octopus_verify_drafts(self, *_, **__):
        pass


@pytest.mark.parametrize("name", SCENES)
def test_no_page_of_another_slot_is_written(name):
    scene = Scene(name, Calls(), "cpu")
    exec(code(), scene.names)
    written = scene.check()
    assert (written == 0) == (name == "pages run out") and written < N_NEW * len(LENS)
