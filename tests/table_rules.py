"""q4kv_resize_tables as include/q4kv.h states it, row by row: who gets blocks and places where there are too few."""
import numpy as np

from tests.table_model import PAGE, Tables, blocks_of


class Rules(Tables):
    """Tables whose rows are served by the header's rule.

    Blocks are handed out to rows in order.  A row that gets longer and finds too few blocks, or too few places in the map, stays as
    it was, and so do the growing rows behind it.  A row that does not grow and ends in a block that others list takes one block
    for its copy if there is one; if not, it loses what it has of that block if it was cut, and keeps the block if it was not."""

    def resize(self, new_len, max_tokens=0):
        rows, width = self.table.shape
        old, want = list(self.len), []
        self.refused = sum(int(n) > width * PAGE for n in new_len)
        for r in range(rows):
            want.append(old[r] if new_len[r] < 0 or new_len[r] > width * PAGE else int(new_len[r]))
        grows, cut = [r for r in range(rows) if want[r] > old[r]], [r for r in range(rows) if want[r] < old[r]]
        for r in cut:
            for j in range(blocks_of(want[r]), blocks_of(old[r])):
                self.count(self.table[r, j], -1)
                self.table[r, j] = -1
        self.at = {r: min(want[r], old[r]) for r in range(rows) if self.pools is not None or r in cut}
        shared = self.ends()
        leaves = dict(shared)                              # the block that a row has to leave, if it gets another
        stays_in = {r: int(self.table[r, n // PAGE]) for r, n in self.at.items() if n % PAGE and r not in shared}
        free = [int(i) for i in np.flatnonzero(self.refs == 0)]
        while True:
            used, tokens, stopped, served = 0, 0, False, {}
            for r in range(rows):
                copies = r in leaves and self.pools is not None
                need, more = copies + max(0, blocks_of(want[r]) - blocks_of(old[r])), max(0, want[r] - old[r])
                if r in grows:
                    stopped |= (need > 0 and used + need > len(free)) or 0 < max_tokens < tokens + more
                    served[r] = not stopped
                else:
                    served[r] = need == 0 or used + need <= len(free)
                if served[r]:
                    used, tokens = used + need, tokens + more
            # the lowest row goes on in a block only if no row that has more tokens there is left in it
            left = {}
            for r in leaves:
                if not served[r] and r not in cut:
                    left[leaves[r]] = max(left.get(leaves[r], 0), self.at[r] % PAGE)
            over = [r for r in stays_in if r in grows and served[r] and left.get(stays_in[r], 0) > self.at[r] % PAGE]
            if not over:
                break
            for r in over:
                leaves[r] = stays_in.pop(r)
        begin, made, tokens = [0], [], 0
        for r in range(rows):
            if r in leaves and (not served[r] or self.pools is None):
                if r in cut:
                    self.len[r] = want[r]
                    self.lose(r, leaves[r])
                elif r in grows:
                    self.refused += 1
            elif r in grows and not served[r]:
                self.refused += 1
            else:
                if r in leaves:
                    self.copy(r, leaves[r], free.pop(0))
                for j in range(blocks_of(old[r]), blocks_of(want[r])):
                    self.table[r, j] = free.pop(0)
                    self.refs[self.table[r, j]] = 1
                self.len[r] = want[r]
                if max_tokens:
                    made += [(r, p) for p in range(old[r], want[r])]
                    tokens = len(made)
            begin.append(tokens)
        slot = [int(self.table[r, p // PAGE]) * PAGE + p % PAGE if 0 <= self.table[r, p // PAGE] < len(self.refs) else -1 for r, p in made]
        fill = [-1] * (max_tokens - len(made))
        return begin, slot + fill, [r for r, _ in made] + fill, [p for _, p in made] + fill


def families(rng, rows, width, members=4, outside=True):
    """Rows of which up to `members` list the same blocks, up to where each of them ends: also inside one block, at different tokens.
    With `outside`, somebody else lists some of the blocks.  Returns the table, the lengths, the counts, and the number of rows' blocks;
    ids are shuffled among twice as many and eight blocks."""
    lens, lists = [], []
    while len(lens) < rows:
        n = int(rng.integers(1, width * PAGE + 1))
        low = (n - 1) // PAGE * PAGE if rng.random() < 0.7 else 0
        at = len(lists)
        for _ in range(min(int(rng.integers(1, members + 1)), rows - len(lens))):
            lens.append(int(rng.choice([n, rng.integers(low, n + 1)])))
            lists.append(at)
    first = {}
    for r, f in enumerate(lists):
        first[f] = max(first.get(f, 0), blocks_of(lens[r]))
    used = sum(first.values())
    ids = [int(i) for i in rng.permutation(2 * used + 8)]
    blocks = {f: [ids.pop() for _ in range(n)] for f, n in first.items()}
    table, refs = np.full((rows, width), -1, np.int32), np.zeros(2 * used + 8, np.int32)
    for r, f in enumerate(lists):
        mine = blocks[f][:blocks_of(lens[r])]
        table[r, :len(mine)] = mine
        refs[mine] += 1
    if outside:
        refs[rng.random(len(refs)) < 0.1] += 1
    order = rng.permutation(rows)                          # members of a family need not be neighbours
    return table[order], np.array(lens, np.int32)[order], refs


def leave_free(rng, refs, count):
    """All free blocks but `count` become somebody else's."""
    refs[rng.permutation(np.flatnonzero(refs == 0))[count:]] += 1


def lengths(rng, lens, width):
    """What a step may ask for: rows left alone, at their length, a little longer, over the end of a block, cut, emptied, too long."""
    out = []
    for n in (int(x) for x in lens):
        out.append(int(rng.choice([-1, n, n + 1, n + int(rng.integers(1, 400)), int(rng.integers(0, n + 1)), max(0, n - 3), 0, width * PAGE + 1],
                                  p=[0.2, 0.1, 0.25, 0.1, 0.15, 0.15, 0.02, 0.03])))
    return [min(n, width * PAGE) if i % 9 else n for i, n in enumerate(out)]
