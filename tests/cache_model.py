"""A plain model of the paged cache and of the attention over it, on the host: lists and float64,
written from the definitions in include/flexprefill.h and sharing no code with the library."""
import numpy as np

FULL, TOO_LONG, SHARED = 1, 2, 4


class Model:
    """Bookkeeping and contents (bf16 bit patterns) of a cache."""

    def __init__(self, layers, pages, hkv, d, slots, max_pages, page):
        self.page, self.max_pages = page, max_pages
        self.holders = [0] * pages
        self.error = 0
        self.len = [0] * slots
        self.rows = [[] for _ in range(slots)]
        self.k = np.zeros((layers, pages, hkv, page, d), np.uint16)
        self.v = np.zeros((layers, pages, hkv, page // 16, d, 16), np.uint16)

    def reserve(self, slots, counts):
        if self.error:
            return
        holders = list(self.holders)
        free = [p for p, n in enumerate(holders) if n == 0]
        plan, copies, at = [], [], 0
        for s, n in zip(slots, counts):
            if self.len[s] + n > self.max_pages * self.page:
                self.error |= TOO_LONG
                continue
            row = list(self.rows[s])
            new = -(-(self.len[s] + n) // self.page) - len(row)
            if n > 0 and self.len[s] % self.page and holders[row[-1]] > 1:
                holders[row[-1]] -= 1
                copies.append((row.pop(), at))
                new += 1
            plan.append((s, row, new, n))
            at += new
        if at > len(free):
            self.error |= FULL
        if self.error:
            return
        at = 0
        for s, row, new, n in plan:
            self.rows[s] = row + free[at:at + new]
            self.len[s] += n
            at += new
        for p in free[:at]:
            holders[p] = 1
        self.holders = holders
        for src, i in copies:
            self.k[:, free[i]] = self.k[:, src]
            self.v[:, free[i]] = self.v[:, src]

    def write(self, layer, k, v, slots, cu):
        if self.error & (FULL | TOO_LONG):
            return
        for i, s in enumerate(slots):
            n = cu[i + 1] - cu[i]
            for j in range(n):
                t = self.len[s] - n + j
                if t < 0:
                    continue
                p = self.rows[s][t // self.page]
                if self.holders[p] != 1:
                    self.error |= SHARED
                    continue
                r = t % self.page
                self.k[layer, p, :, r] = k[cu[i] + j]
                self.v[layer, p, :, r // 16, :, r % 16] = v[cu[i] + j]

    def truncate(self, slots, lens):
        if self.error:
            return
        for s, n in zip(slots, lens):
            keep = -(-n // self.page)
            for p in self.rows[s][keep:]:
                self.holders[p] -= 1
            self.rows[s] = self.rows[s][:keep]
            self.len[s] = min(self.len[s], n)

    def fork(self, src, dst):
        if self.error:
            return
        self.truncate(dst, [0] * len(dst))
        for a, b in zip(src, dst):
            self.rows[b] = list(self.rows[a])
            self.len[b] = self.len[a]
            for p in self.rows[b]:
                self.holders[p] += 1

    def compact(self):
        if self.error:
            return
        n = sum(h > 0 for h in self.holders)
        holes = [p for p in range(n) if self.holders[p] == 0]
        movers = [p for p in range(n, len(self.holders)) if self.holders[p] > 0]
        name = dict(zip(movers, holes))
        for a, b in name.items():
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
            self.holders[b], self.holders[a] = self.holders[a], 0
        self.rows = [[name.get(p, p) for p in row] for row in self.rows]

    def meta(self):
        pages = len(self.holders)
        used = np.zeros(-(-pages // 64) * 2, np.uint32)
        for p, h in enumerate(self.holders):
            if h:
                used[p // 32] |= np.uint32(1 << (p % 32))
        table = np.full((len(self.rows), self.max_pages), -1, np.int32)
        for s, row in enumerate(self.rows):
            table[s, :len(row)] = row
        state = np.zeros(8, np.int32)
        state[0], state[1] = sum(h > 0 for h in self.holders), self.error
        return np.concatenate([state, used.view(np.int32), np.asarray(self.len, np.int32),
                               np.asarray(self.holders, np.int32), table.ravel()])

    def tokens(self, layer, slot):
        """Keys and values of a slot, [len, hkv, d], bit patterns."""
        t = np.arange(self.len[slot])
        p = np.asarray(self.rows[slot], np.int64)[t // self.page] if t.size else t
        r = t % self.page
        return self.k[layer, p, :, r], self.v[layer, p, :, r // 16, :, r % 16]


def bits(x):
    """float -> bf16 bit patterns, round to nearest even."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def floats(b):
    return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def attend(q, keys, values, scale):
    """One sequence: q [nq, Hq, d], keys and values [n, Hkv, d], float64; query t sees keys
    0 .. n - nq + t.  Returns o and the sum of weight * |value| that error bounds are made of."""
    nq, hq, d = q.shape
    n, hkv = keys.shape[:2]
    G = hq // hkv
    o, mass = np.zeros((nq, hq, d)), np.zeros((nq, hq, d))
    for t in range(nq):
        m = n - nq + 1 + t
        if m <= 0:
            continue
        for h in range(hq):
            with np.errstate(invalid="ignore", over="ignore"):
                s = keys[:m, h // G] @ q[t, h] * scale
                top = s.max()
                w = np.exp(s - (top if top > -np.inf else 0.0))
                if w.sum() == 0:
                    continue
                w /= w.sum()
                o[t, h] = w @ values[:m, h // G]
                mass[t, h] = w @ np.abs(values[:m, h // G])
    return o, mass


def tolerance(o, mass):
    """Largest error allowed: the rounding of the result to bf16 is at most 2^-8 |o|, and |o| is at
    most the mass (the sum of weight * |value|); what is left, at least 2^-9 |o| and a part in 10^4
    of the mass for float32 scores and exponentials, has to hold the rounding of the weights."""
    return 2.0 ** -8 * mass + 2.0 ** -9 * np.abs(o) + 1e-4 * mass + 1e-37
