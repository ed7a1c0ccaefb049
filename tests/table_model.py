"""Block tables, beam choices and slots as plain Python, row by row: what the GPU calls are compared with."""
import numpy as np

PAGE = 256


def blocks_of(n):
    return -(-n // PAGE)


class Tables:
    """table [agents][max_blocks], len [agents], refs [blocks]; pools: a list of arrays [layers][blocks][heads][256][width], or None."""

    def __init__(self, table, length, refs, pools=None):
        self.table, self.len, self.refs, self.pools = table.copy(), [int(n) for n in length], refs.copy(), pools
        self.refused = 0

    def count(self, block, by):
        if 0 <= block < len(self.refs):
            self.refs[block] += by

    def ends(self):
        """The rows' places and whether they go on in a block that others list: {row: block} of those that need a copy."""
        inside = {}
        for r, n in self.at.items():
            block = int(self.table[r, n // PAGE]) if n % PAGE else -1
            if 0 <= block < len(self.refs) and self.refs[block] > 1:
                inside.setdefault(block, []).append(r)
        out = {}
        for block, rows in inside.items():
            for r in rows:
                if not (r == min(rows) and len(rows) == self.refs[block]):
                    out[r] = block
        return out

    def free_block(self):
        free = np.flatnonzero(self.refs == 0)
        return int(free[0]) if len(free) else -1

    def copy(self, r, block, free):
        n = self.at[r]
        self.count(block, -1)
        self.refs[free] = 1
        self.table[r, n // PAGE] = free
        for pool in self.pools:
            pool[:, free, :, :n % PAGE] = pool[:, block, :, :n % PAGE]

    def lose(self, r, block):
        n = self.at[r]
        self.count(block, -1)
        self.table[r, n // PAGE] = -1
        self.len[r] = n // PAGE * PAGE
        self.refused += 1

    def resize(self, new_len, max_tokens=0):
        rows, width = self.table.shape
        self.refused = 0
        want = {}
        for r in range(rows):
            if new_len[r] > width * PAGE:
                self.refused += 1
            want[r] = self.len[r] if new_len[r] < 0 or new_len[r] > width * PAGE else int(new_len[r])
        cut = {r for r in range(rows) if want[r] < self.len[r]}
        for r in cut:
            for j in range(blocks_of(want[r]), blocks_of(self.len[r])):
                self.count(self.table[r, j], -1)
                self.table[r, j] = -1
        self.at = {r: min(want[r], self.len[r]) for r in range(rows) if self.pools is not None or r in cut}
        shared = self.ends()
        # what is free now, lowest first, goes to rows in order
        free = [int(i) for i in np.flatnonzero(self.refs == 0)]
        tokens, stopped, begin, made = 0, False, [0], []
        for r in range(rows):
            old, new = self.len[r], want[r]
            copies = r in shared and self.pools is not None
            need = copies + max(0, blocks_of(new) - blocks_of(old))
            more = max(0, new - old) if max_tokens else 0
            if r in shared and self.pools is None:
                self.lose(r, shared[r])
            elif (need or more) and not stopped and (need > len(free) or (max_tokens and tokens + more > max_tokens)):
                stopped = True
            if stopped and (need or new > old):
                if new > old:
                    self.refused += 1
                else:
                    self.lose(r, shared[r])
            elif not (r in shared and self.pools is None):
                if copies:
                    self.copy(r, shared[r], free.pop(0))
                for j in range(blocks_of(old), blocks_of(new)):
                    self.table[r, j] = free.pop(0)
                    self.refs[self.table[r, j]] = 1
                self.len[r] = new
                if max_tokens:
                    made += [(r, p) for p in range(old, new)]
                    tokens += more
            begin.append(tokens)
        slot = [int(self.table[r, p // PAGE]) * PAGE + p % PAGE if 0 <= self.table[r, p // PAGE] < len(self.refs) else -1 for r, p in made]
        fill = [-1] * (max_tokens - len(made))
        return begin, slot + fill, [r for r, _ in made] + fill, [p for _, p in made] + fill

    def reorder(self, parent):
        rows = len(self.len)
        old, lens = self.table.copy(), list(self.len)
        self.refused = 0
        for r in range(rows):
            p = int(parent[r]) if 0 <= parent[r] < rows else -1
            if p == r:
                continue
            mine, theirs = blocks_of(lens[r]), blocks_of(lens[p]) if p >= 0 else 0
            for j in range(mine):
                self.count(old[r, j], -1)
            for j in range(theirs):
                self.count(old[p, j], 1)
            self.table[r, :theirs] = old[p, :theirs]
            self.table[r, theirs:max(mine, theirs)] = -1
            self.len[r] = lens[p] if p >= 0 else 0
        self.at = dict(enumerate(self.len))
        free = [int(i) for i in np.flatnonzero(self.refs == 0)]
        for r, block in sorted(self.ends().items()):
            if free:
                self.copy(r, block, free.pop(0))
            else:
                self.lose(r, block)


def choose(logits, score, bounds, num_out, end=None):
    """logits float64 [rows][vocab] -> parents, tokens, totals (float64) and every continuation's total [groups] of dicts' arrays."""
    logits = np.where(np.isnan(logits), -np.inf, np.minimum(logits, float(np.finfo(np.float32).max)))
    rows, vocab = logits.shape
    groups = len(bounds) - 1
    parent, token = (np.full((groups, num_out), -1, np.int64) for _ in range(2))
    total = np.full((groups, num_out), -np.inf)
    every = []
    for g in range(groups):
        lo, hi = (min(max(b, 0), rows) for b in (bounds[g], bounds[g + 1]))
        t, of_row, of_token, value = [], [], [], []
        for r in range(lo, hi):
            if not score[r] > -np.inf:
                continue
            if end is not None and end[r] >= 0:
                t.append(np.array([float(score[r])])), of_row.append(np.array([r])), of_token.append(np.array([end[r]])), value.append(np.zeros(1))
                continue
            x = logits[r].astype(np.longdouble)
            on = np.flatnonzero(x > -np.inf)
            if len(on) == 0:
                continue
            top = x[on].max()
            log_sum = top + np.log(np.exp(x[on] - top).sum())
            t.append((np.longdouble(score[r]) + (x[on] - log_sum)).astype(np.float64))
            of_row.append(np.full(len(on), r)), of_token.append(on), value.append(logits[r, on])
        if t:
            t, of_row, of_token, value = (np.concatenate(v) for v in (t, of_row, of_token, value))
            best = np.lexsort((of_token, -value, of_row, -t))[:num_out]
            parent[g, :len(best)], token[g, :len(best)], total[g, :len(best)] = of_row[best], of_token[best], t[best]
            every.append({(int(a), int(c)): float(v) for a, c, v in zip(of_row, of_token, t)})
        else:
            every.append({})
    return parent, token, total, every
