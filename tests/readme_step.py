"""The step over pages that README.md shows, as code, with data to run it on: five slots of which one ends, one comes from another and shares a page
that both would write into, and one asks for pages that are there or are not; and what it may have written."""
import os
import re

import numpy as np
import torch

from pages_model import TILE, Pages

N_KV, N_QH, D, N_AXES, N_NEW, N_PAGES, PER, VOCAB = 2, 4, 64, 3, 3, 8, 4, 50
LENS = [70, 130, 64, 20]
# entries past a slot's pages name pages of the others: what earlier holders left there
TABLE = [[5, 2, 0, 4], [0, 1, 3, 6], [4, 1, 2, 0], [6, 5, 2, 0]]
# source, tokens kept, tokens asked for
SCENES = {"pages run out": ([0, 1, 2, 0], [70, 130, 64, 70], [73, 133, 195, 73]),
          "a slot ends": ([0, 0, 2, -1], [70, 70, 64, 20], [73, 73, 67, 0]),
          "a slot has no new tokens": ([0, 0, 2, 3], [70, 66, 64, 20], [73, 66, 65, 21]),
          "a slot is emptied": ([3, 1, 2, 3], [20, 130, 64, 20], [23, 0, 67, 23])}


def code():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        found = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "octopus_pages_update" in b]
    assert len(found) == 1
    return compile(found[0], "README.md", "exec")


class Scene:
    """The names that the step's code takes, and the state before it."""

    def __init__(self, name, oct, dev, cb=None, granules=1):
        source, keep, new = SCENES[name]
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        g = torch.Generator().manual_seed(3)
        bf16 = lambda *shape: torch.randn(shape, generator=g).bfloat16().to(dev)  # noqa: E731
        refs = np.zeros(N_PAGES, dtype=np.int32)
        for row, n in zip(TABLE, LENS):
            refs[row[:-(-n // TILE)]] += 1
        k_pools = [torch.randint(0, 256, (N_PAGES, N_KV, granules, TILE, 16), generator=g, dtype=torch.uint8).to(dev) for _ in range(2)]
        v_pools = [bf16(N_PAGES, N_KV, TILE, D) for _ in range(2)]
        angle = torch.arange(500)[:, None] * 100.0 ** (-torch.arange(D // 2) / D)
        positions = (torch.tensor(keep)[:, None, None] + torch.arange(N_NEW)[:, None] + 10 * torch.arange(N_AXES)).int().to(dev)
        self.names = dict(
            oct=oct, torch=torch, cb=cb, k_pools=k_pools, v_pools=v_pools, k_pool=k_pools[0], v_pool=v_pools[0], n_pages=N_PAGES, refs=ints(refs.tolist()),
            table=ints(TABLE), lens=ints(LENS), new_lens=ints(new), parents=ints(source), keep=ints(keep), moves=ints([0] * (2 + 2 * len(LENS))),
            k=bf16(len(LENS), N_NEW, N_KV, D), v=bf16(len(LENS), N_NEW, N_KV, D), q=bf16(len(LENS), N_NEW, N_QH, D),
            q_rot=torch.full((len(LENS), N_NEW, N_QH, D), 7.0, dtype=torch.bfloat16, device=dev), n_new=N_NEW,
            sign_bits=torch.zeros((N_KV, D // 8), dtype=torch.uint8, device=dev), cos_sin=torch.stack([angle.cos(), angle.sin()], -1).contiguous().to(dev),
            axis_of_pair=bytes(i % N_AXES for i in range(D // 2)), positions=positions, drafts=ints([[1] * (N_NEW - 1)] * len(LENS)),
            p_target=torch.full((len(LENS), N_NEW, VOCAB), 1 / VOCAB, device=dev), p_draft=torch.full((len(LENS), N_NEW - 1, VOCAB), 1 / VOCAB, device=dev),
            uniforms=torch.full((len(LENS), N_NEW), 0.5, device=dev), tokens=ints([[0] * N_NEW] * len(LENS)), n_accepted=ints([0] * len(LENS)),
            ws=None, ws_verify=None)
        self.model = Pages(refs, TABLE, LENS)
        self.changed = ("refs", "table", "lens", "moves", "q_rot")
        self.before = {name: self.names[name].clone() for name in self.changed}
        self.pools = [*k_pools, *v_pools]
        self.pools_before = [p.clone() for p in self.pools]
        self.keep, self.asked = keep, (new, source, keep)
        self.model.update(*self.asked)

    def restore(self):
        for name, value in self.before.items():
            self.names[name].copy_(value)
        for pool, value in zip(self.pools, self.pools_before):
            pool.copy_(value)

    def check(self):
        """State as the model's; of the pools only copied pages and the slots' own new tokens differ from what they were."""
        model, got = self.model, {name: self.names[name].cpu() for name in self.changed}
        assert got["lens"].tolist() == model.lens.tolist() and got["refs"].tolist() == model.refs.tolist()
        assert got["moves"][:2].tolist() == [len(model.moves), model.missing]
        own = np.zeros((N_PAGES, TILE), dtype=bool)
        new = {}
        for s, (n, keep) in enumerate(zip(model.lens, self.keep)):
            for t in range(min(max(int(n) - keep, 0), N_NEW)):
                page, at = int(model.table[s, (keep + t) // TILE]), (keep + t) % TILE
                assert model.refs[page] == 1 and not own[page, at]          # (nobody else's)
                own[page, at] = True
                new[s, t] = page, at
        for i, (pool, before) in enumerate(zip(self.pools, self.pools_before)):
            pool, want = pool.cpu(), before.cpu().clone()
            for a, b in model.moves:
                want[b] = before[a].cpu()
            layer_0, axis = i % 2 == 0, 2 if pool.dim() == 4 else 3          # (the step's code appends to the first layer)
            same = (pool == want).movedim(axis, 1).flatten(2).all(-1).numpy()          # [page, slot]
            assert np.all(same | own) if layer_0 else np.all(same), (i, np.argwhere(~same & ~own))
        for (s, t), (page, at) in new.items():
            assert torch.equal(self.names["v_pool"][page, :, at].cpu(), self.names["v"][s, t].cpu())
        rows = np.array([[(s, t) in new for t in range(N_NEW)] for s in range(len(LENS))])
        still = (got["q_rot"] == 7.0).flatten(2).all(-1).numpy()
        assert np.array_equal(still, ~rows)
        return len(new)
