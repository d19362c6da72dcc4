"""The pages of a cache, step by step on the CPU from what the header says.  A cache's contents are one label a block."""
BLOCK = 64


def _need(length, width):
    return -(-min(max(length, 0), width * BLOCK) // BLOCK)


def _unfinished(length, width):
    return 0 < length < width * BLOCK and length % BLOCK != 0


class Pages:
    def __init__(self, users, table, lengths, contents):
        self.users, self.table, self.lengths, self.contents = list(users), [list(r) for r in table], list(lengths), list(contents)

    def _there(self, e):
        return 0 <= e < len(self.users)

    def _deal(self, places):
        """places: (sequence, entry, block it is to be a copy of or None), in order; returns how many got none"""
        free = [b for b, n in enumerate(self.users) if n == 0]
        before = list(self.contents)
        missing = 0
        for b, j, source in places:
            if source is not None:
                self.users[source] -= 1
            if free:
                block = free.pop(0)
                self.users[block] += 1
                self.table[b][j] = block
                if source is not None:
                    self.contents[block] = before[source]
            else:
                self.table[b][j] = -1
                missing += 1
        return missing

    def resize(self, lengths):
        width = len(self.table[0])
        for row, length in zip(self.table, lengths):
            for j in range(_need(length, width), width):
                if self._there(row[j]):
                    self.users[row[j]] -= 1
                row[j] = -1
        places = []
        shared = [n > 1 for n in self.users]
        for b, length in enumerate(lengths):
            need = _need(length, width)
            for j in range(need):
                e = self.table[b][j]
                if not self._there(e):
                    places.append((b, j, None))
                elif j == need - 1 and _unfinished(length, width) and shared[e]:
                    places.append((b, j, e))
        if len(places) > sum(n == 0 for n in self.users):
            cut = {}
            for place in places:
                cut.setdefault(place[2], []).append(place)
            for e, held in cut.items():
                if e is not None and len(held) >= self.users[e]:
                    places.remove(held[0])
        return self._deal(places)

    def fork(self, parents):
        width = len(self.table[0])
        old, lengths = [list(r) for r in self.table], list(self.lengths)
        places, taken = [], set(p for b, p in enumerate(parents) if p == b)
        for b, p in enumerate(parents):
            if p == b:
                continue
            for e in old[b]:
                if self._there(e):
                    self.users[e] -= 1
            length = lengths[p] if 0 <= p < len(parents) else 0
            need = _need(length, width)
            row = [old[p][j] if j < need and self._there(old[p][j]) else -1 for j in range(width)]
            if _unfinished(length, width) and row[need - 1] >= 0:
                if p in taken:
                    places.append((b, need - 1, row[need - 1]))
                    self.users[row[need - 1]] += 1          # (taken back when the copy is dealt)
                taken.add(p)
            self.table[b], self.lengths[b] = row, length
            for j, e in enumerate(row):
                if e >= 0 and not (places and places[-1][:2] == (b, j)):
                    self.users[e] += 1
        return self._deal(places)

    def compact(self, blocks_to):
        used = [b for b, n in enumerate(self.users) if n > 0]
        kept = used[:blocks_to]
        number = {b: i for i, b in enumerate(kept)}
        table = [[number.get(e, -1) for e in row] for row in self.table]
        users = [self.users[b] for b in kept] + [0] * (blocks_to - len(kept))
        return table, users, [self.contents[b] for b in kept], len(used) - len(kept)
