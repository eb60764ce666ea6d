"""The definition of octopus_pages_update and octopus_pages_compact as sequential Python over lists."""
import numpy as np

TILE = 64


def ceil(tokens):
    return -(-tokens // TILE)


class Pages:
    """refs, table rows and lens as lists of ints (or arrays)."""

    def __init__(self, refs, table, lens):
        self.refs = np.array(refs, dtype=np.int64)
        self.table = np.array(table, dtype=np.int64)
        self.lens = np.array(lens, dtype=np.int64)
        self.moves, self.missing = [], 0

    def page(self, entry):
        return int(min(max(entry, 0), len(self.refs) - 1))

    def update(self, new_lens, source=None, keep_lens=None):
        n_seq, per = self.table.shape
        old, held = self.table.copy(), [min(max(int(n), 0), per * TILE) for n in self.lens]
        source = list(range(n_seq)) if source is None else [int(x) for x in source]
        kept, want = [], []
        for s in range(n_seq):
            w = min(max(int(new_lens[s]), 0), per * TILE)
            k = min(held[source[s]] if 0 <= source[s] < n_seq else 0, w)
            if keep_lens is not None:
                k = min(k, max(int(keep_lens[s]), 0))
            kept.append(k)
            want.append(w)
        for s in range(n_seq):
            for j in range(ceil(held[s])):
                self.refs[self.page(old[s, j])] -= 1
        rows = []
        for s in range(n_seq):
            rows.append([self.page(old[source[s], j]) for j in range(ceil(kept[s]))])
            for page in rows[s]:
                self.refs[page] += 1
        # pages that are written into
        writers = {}
        for s in range(n_seq):
            if want[s] > kept[s] and kept[s] % TILE:
                writers.setdefault(rows[s][-1], []).append(s)
        copied = set()
        for page, slots in writers.items():
            stays = min(slots, key=lambda s: (source[s] != s, s)) if self.refs[page] <= len(slots) else None
            copied |= {s for s in slots if s != stays}
        free = [page for page in range(len(self.refs)) if self.refs[page] <= 0]
        need = sum(ceil(want[s]) - ceil(kept[s]) + (s in copied) for s in range(n_seq) if want[s] > kept[s])
        self.missing, self.moves = max(0, need - len(free)), []
        if self.missing:
            want, copied = kept, set()
        free = iter(free)
        fresh = []
        for s in range(n_seq):
            if s in copied:
                to = next(free)
                self.moves.append((rows[s][-1], to))
                self.refs[rows[s][-1]] -= 1
                rows[s][-1] = to
                fresh.append(to)
            while len(rows[s]) < ceil(want[s]):
                rows[s].append(next(free))
                fresh.append(rows[s][-1])
        for page in fresh:
            self.refs[page] = 1
        for s in range(n_seq):
            new = rows[s]
            if source[s] == s:       # entries that stay are not written (a number outside the pool stays as it is)
                new = [int(old[s, j]) if j < ceil(kept[s]) - (s in copied) else page for j, page in enumerate(rows[s])]
            self.table[s, :len(new)] = new
            self.lens[s] = want[s]

    def compact(self):
        """The map of page numbers; moves and `used` are set."""
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        free = [p for p in range(len(self.refs)) if self.refs[p] <= 0]
        page_map, self.moves, self.used = list(range(len(self.refs))), [], len(used)
        for high, low in zip(reversed(used), free):
            if low > high:
                break
            self.moves.append((high, low))
            page_map[high] = low
            self.refs[low], self.refs[high] = self.refs[high], 0
        return page_map

    def rename(self, page_map):
        for s in range(len(self.table)):
            for j in range(min(ceil(max(int(self.lens[s]), 0)), self.table.shape[1])):
                self.table[s, j] = page_map[self.page(self.table[s, j])]

    def check(self, pinned=None):
        """What has to hold of a state that only these calls have made."""
        count = np.zeros(len(self.refs), dtype=np.int64) if pinned is None else np.array(pinned, dtype=np.int64)
        for s in range(len(self.table)):
            row = self.table[s, :ceil(int(self.lens[s]))]
            assert len(set(row.tolist())) == len(row)
            np.add.at(count, row, 1)
        assert np.array_equal(count, self.refs)
