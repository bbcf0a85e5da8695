"""The serving operators from their definitions, in 64 bits, in plain numpy on the host."""
import numpy as np

E4M3 = np.array([(-1.0 if b > 127 else 1.0) * ((1 + (b & 7) / 8) * 2.0 ** (((b >> 3) & 15) - 7) if (b >> 3) & 15 else (b & 7) / 8 * 2.0 ** -6)
                 for b in range(256)])                       # 0x7f and 0xff are NaN; nothing here produces them
TOP = {"e4m3": 448.0, "int8": 127.0}


def turns(positions, frequency):
    """Exact fractions of a turn: Python integers modulo 2^64."""
    return np.array([[((int(p) * int(f)) % (1 << 64)) / 2.0 ** 64 for f in frequency] for p in positions]).reshape(len(positions), len(frequency))


def rotate(x, positions, frequency, interleaved, amplitude=1.0, inverse=False):
    """x [tokens, heads, dim] float64."""
    half = len(frequency)
    t = turns(positions, frequency)[:, None, :] * 2 * np.pi
    cos, sin = amplitude * np.cos(t), amplitude * np.sin(t) * (-1 if inverse else 1)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def values(codes, fmt):
    codes = np.asarray(codes).view(np.uint8)
    return E4M3[codes] if fmt == "e4m3" else codes.view(np.int8).astype(np.float64)


def scale_of(amax, fmt):
    """Least power of two s with amax / s <= the format's largest value, within 2^-100 .. 2^122."""
    if amax == 0:
        return 2.0 ** -100
    e = -100
    while amax / 2.0 ** e > TOP[fmt] and e < 122:
        e += 1
    return 2.0 ** e


def step_of(x, fmt):
    """Distance between neighbouring codes' values around x (in units of the scale)."""
    if fmt == "int8":
        return np.ones_like(x)
    return 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6) - 3)


def attend(q, k, v, start, scale, window):
    """One sequence: q [n, q_heads, d], k and v [length, kv_heads, d] (values).  Returns out, lse and sum of p |v|."""
    n, hq, d = q.shape
    length, h, _ = k.shape
    out, lse, weight = np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq, d))
    for t in range(n):
        pos = start + t
        lo, hi = (max(0, pos - window + 1) if window else 0), min(pos + 1, length)
        if hi <= lo:
            continue
        for j in range(hq):
            g = j // (hq // h)
            s = scale * (k[lo:hi, g] @ q[t, j])
            m = s.max()
            p = np.exp(s - m)
            out[t, j] = p @ v[lo:hi, g] / p.sum()
            weight[t, j] = p @ np.abs(v[lo:hi, g]) / p.sum()
            lse[t, j] = m + np.log(p.sum())
    return out, lse, weight


class Pages:
    """The page operations on Python lists: refs, table, length; data moves are returned as (source, destination) pairs."""

    def __init__(self, num_pages, page_tokens, max_seqs, max_pages):
        self.t, self.max_pages = page_tokens, max_pages
        self.refs, self.length = [0] * num_pages, [0] * max_seqs
        self.table = [[-1] * max_pages for _ in range(max_seqs)]

    def held(self, n):
        return -(-n // self.t)

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def reserve(self, seqs, want):
        free, asked = self.free_pages(), 0
        for s, w in zip(seqs, want):
            have, x = self.held(self.length[s]), self.held(w) - self.held(self.length[s])
            asked += x
            if x and asked > len(free):
                continue
            for e in range(x):
                p = free[asked - x + e]
                self.table[s][have + e] = p
                self.refs[p] = 1
            self.length[s] = max(self.length[s], w)

    def fork(self, parents, children):
        free, asked, moves = self.free_pages(), 0, []
        lengths = [self.length[p] for p in parents]
        for p, c, n in zip(parents, children, lengths):
            part = n % self.t != 0
            asked += part
            if part and asked > len(free):
                continue
            row = list(self.table[p][:self.held(n)])
            for e, page in enumerate(row):
                if part and e + 1 == len(row):
                    moves.append((page, free[asked - 1]))
                    row[e] = free[asked - 1]
                    self.refs[row[e]] = 1
                else:
                    self.refs[page] += 1
            self.table[c] = row + [-1] * (self.max_pages - len(row))
            self.length[c] = n
        return moves

    def free(self, seqs):
        for s in seqs:
            for e in range(self.held(self.length[s])):
                self.refs[self.table[s][e]] -= 1
                self.table[s][e] = -1
            self.length[s] = 0

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        source = [p for p, r in enumerate(self.refs) if r > 0 and p >= used]
        hole = [p for p, r in enumerate(self.refs) if r == 0 and p < used]
        to = dict(zip(source, hole))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return list(to.items()), used
