"""The pool's blocks by the definition: lists, a set of free blocks and loops."""
import numpy as np

B = 16


def ceil(n, by=B):
    return -(-n // by)


class Pool:
    def __init__(self, tables, lens, num_blocks):
        self.tables, self.lens, self.nb = tables.astype(np.int64).copy(), [int(t) for t in lens], num_blocks
        self.refs = [0] * num_blocks
        for s in range(len(self.lens)):
            for e in self.held(s):
                self.refs[self.tables[s, e]] += 1

    def held(self, s):
        n = min(ceil(max(self.lens[s], 0)), self.tables.shape[1])
        return [e for e in range(n) if 0 <= self.tables[s, e] < self.nb]

    def free_blocks(self):
        return [b for b in range(self.nb) if self.refs[b] == 0]

    def free_map(self):
        words = np.zeros(ceil(self.nb, 32), np.uint32)
        for b in self.free_blocks():
            words[b // 32] |= np.uint32(1 << (b % 32))
        return words

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lens):
                for e in self.held(s):
                    self.refs[self.tables[s, e]] -= 1
                self.lens[s] = 0

    def free_outside_window(self, window, sinks):
        for s in range(len(self.lens)):
            for e in self.held(s):
                if e * B >= sinks and (e + 1) * B <= self.lens[s] - window:
                    self.refs[self.tables[s, e]] -= 1
                    self.tables[s, e] = -1

    def reserve(self, starts, num_rows, slots):
        """slots: as before the call -> (result, slots behind it)."""
        S, slots = len(self.lens), slots.copy()
        new = [int(t > 0) for t in self.lens] if starts is None else [int(starts[s + 1] - starts[s]) for s in range(S)]
        rows = S if starts is None else min(int(starts[S]), num_rows)
        row0 = list(range(S)) if starts is None else [int(x) for x in starts[:S]]
        bad = starts is not None and (starts[0] != 0 or starts[S] > num_rows or any(n < 0 for n in new))
        if bad or any(t + n > self.tables.shape[1] * B for t, n in zip(self.lens, new)):
            slots[:rows] = -1
            return -1, slots
        need = sum(ceil(t + n) - ceil(t) for t, n in zip(self.lens, new))
        free = self.free_blocks()
        if need > len(free):
            slots[:rows] = -1
            return need - len(free), slots
        if starts is None:
            slots[:rows] = -1
        for s in range(S):
            for e in range(ceil(self.lens[s]), ceil(self.lens[s] + new[s])):
                b = free.pop(0)
                self.tables[s, e] = b
                self.refs[b] = 1
            for i in range(new[s]):
                pos = self.lens[s] + i
                slots[row0[s] + i] = self.tables[s, pos // B] * B + pos % B
            self.lens[s] += new[s]
        return 0, slots

    def fork(self, parents, children):
        S, n = len(self.lens), len(parents)
        copies = np.full((n, 2), -1, np.int64)
        real = [i for i in range(n) if parents[i] >= 0 and children[i] >= 0]
        ok = all(parents[i] < S and children[i] < S and parents[i] != children[i] for i in real)
        ok = ok and all(self.lens[children[i]] == 0 for i in real) and len({int(children[i]) for i in real}) == len(real)
        if not ok:
            return -1, copies
        tokens = {i: self.lens[parents[i]] for i in real}
        partial = [i for i in real if tokens[i] % B]
        free = self.free_blocks()
        if len(partial) > len(free):
            return len(partial) - len(free), copies
        for i in partial:
            b = free.pop(0)
            e = tokens[i] // B
            copies[i] = self.tables[parents[i], e], b
            self.tables[children[i], e] = b
            self.refs[b] = 1
        for i in real:
            for e in range(tokens[i] // B):
                self.tables[children[i], e] = self.tables[parents[i], e]
                if 0 <= self.tables[parents[i], e] < self.nb:
                    self.refs[self.tables[parents[i], e]] += 1
        for i in real:
            self.lens[children[i]] = tokens[i]
        return 0, copies

    def compact(self):
        n = self.nb - len(self.free_blocks())
        src = [b for b in range(n, self.nb) if self.refs[b]]
        dst = [b for b in range(n) if not self.refs[b]]
        assert len(src) == len(dst)
        to = dict(zip(src, dst))
        for s in range(len(self.lens)):
            for e in self.held(s):
                self.tables[s, e] = to.get(self.tables[s, e], self.tables[s, e])
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        return list(zip(src, dst))
