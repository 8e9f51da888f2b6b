"""Plain forms of the paged 4-bit cache, of attention over it and of rotary positions, in 64 bits on the CPU (numpy and plain
Python), for the tests."""
import math

import numpy as np
import torch

CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_values(x):
    """float64 [n, 32]: what each element of a block reads back as."""
    out = np.empty_like(x)
    for i, blk in enumerate(x):
        if not np.isfinite(blk).all():
            out[i] = np.nan
            continue
        top = np.abs(blk).max()
        e = -125
        if top > 7.0 * 2.0 ** e:
            e = max(e, math.frexp(top / 7.0)[1] - 1)          # 2^e <= top / 7 < 2^(e + 1)
            while top > 7.0 * 2.0 ** e and e < 125:
                e += 1
        e = min(e, 125)
        y = np.abs(blk) / 2.0 ** e
        dist = np.abs(y[:, None] - CODES)
        best = dist.min(1)
        code = np.array([min((c for c in range(8) if dist[j, c] == best[j]), key=lambda c: (c & 1, c)) for j in range(32)])
        out[i] = np.copysign(CODES[code] * 2.0 ** e, blk)
    return out


def cache_values(x):
    """[..., d] (any float tensor) -> float64 numpy, what the cache holds of it"""
    a = x.detach().cpu().double().numpy()
    with np.errstate(invalid="ignore"):
        return block_values(a.reshape(-1, 32)).reshape(a.shape)


def attention(Q, K, V, visible, scale):
    """One key-value head in float64: Q [R, d], K, V [n, d], visible [R, n] -> O [R, d], and E = sum of weights times |V| and
    S = the largest sum of |q k| over the visible rows, for error bounds."""
    R, d = Q.shape
    O, E, S = np.zeros((R, d)), np.zeros((R, d)), np.zeros(R)
    for r in range(R):
        rows = np.nonzero(visible[r])[0]
        if rows.size == 0:
            continue
        x = K[rows] @ Q[r] * scale
        w = np.exp(x - x.max())
        w /= w.sum()
        O[r], E[r] = w @ V[rows], w @ np.abs(V[rows])
        S[r] = (np.abs(K[rows]) @ np.abs(Q[r])).max() * scale
    return O, E, S


def attention_bound(O, E, S, n, d, dtype, one_term):
    """How far the kernel's output may be off.  Scores: sums of d products in fp32 (three-term operands leave out less than
    one more unit each), scaled once; a score off by e changes every weight by a factor within exp(+-2 e).  Weights: exp2 is
    within 2 units.  Sums of n rows in fp32.  bf16: the weights as two bf16 terms (2^-16 left out) or one (2^-8, which the
    normaliser shares), the output rounded by half a step, 2^-8."""
    u = 2.0 ** -24
    score = (d + 8) * u * S[:, None] + 4 * u
    rel = 2 * score + (n + 64) * u
    if dtype == torch.bfloat16:
        rel = rel + (2 * 2.0 ** -8 if one_term else 2 * 2.0 ** -16)
        return E * rel * 1.01 + np.abs(O) * 2.0 ** -8 + 1e-37
    return E * rel * 1.01 + np.abs(O) * 2 * u + 1e-37


def rotary(x, pos, freq, sections, adjacent, inverse):
    """x [L, B, H, T, d] float64, pos [axes, B, T] int, freq [P] -> float64"""
    y = x.clone()
    P = len(freq)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for j in range(P):
        # exact remainder of the angle: both factors are integers times powers of two
        ang = torch.tensor([[math.remainder(int(p) * float(freq[j]), 2 * math.pi) for p in row] for row in pos[axis[j]].tolist()], dtype=torch.float64)
        c, s = torch.cos(ang)[None, :, None], torch.sin(ang)[None, :, None]
        if inverse:
            s = -s
        a, b = (2 * j, 2 * j + 1) if adjacent else (j, j + P)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


class Sim:
    """The page calls in plain Python."""

    def __init__(self, B, page, n_pages, max_pages):
        self.B, self.page, self.max_pages = B, page, max_pages
        self.table, self.length, self.refs, self.status = [[-1] * max_pages for _ in range(B)], [0] * B, [0] * n_pages, 0

    def _count(self, n):
        return -(-n // self.page)

    def reserve(self, n_new):
        """Starts, and the copies (from, to, tokens)"""
        free, plan, take = [p for p, r in enumerate(self.refs) if r == 0], [], 0
        bad = [False] * self.B
        for b in range(self.B):
            n, ln = max(n_new[b], 0), self.length[b]
            need, src = 0, -1
            if ln + n > self.max_pages * self.page:
                bad[b] = True
            elif n > 0:
                need = self._count(ln + n) - self._count(ln)
                if ln % self.page:
                    p = self.table[b][ln // self.page]
                    if not 0 <= p < len(self.refs):
                        bad[b], need = True, 0
                    elif self.refs[p] > 1:
                        src, need = p, need + 1
            plan.append((need, src, n))
            take += need
        if any(bad):
            self.status |= 2
        if take > len(free):
            self.status |= 1
            return [-1] * self.B, []
        starts, copies = [], []
        free = iter(free)
        for b, (need, src, n) in enumerate(plan):
            if bad[b]:
                starts.append(-1)
                continue
            ln = self.length[b]
            if src >= 0:
                p = next(free)
                self.table[b][ln // self.page] = p
                self.refs[p], self.refs[src] = 1, self.refs[src] - 1
                copies.append((src, p, ln % self.page))
                need -= 1
            for i in range(need):
                p = next(free)
                self.table[b][self._count(ln) + i], self.refs[p] = p, 1
            self.length[b] = ln + n
            starts.append(ln)
        return starts, copies

    def fork(self, src, dst):
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= s < self.B and 0 <= d < self.B and d not in dst[:i] and s not in dst
            if not ok or self.length[d] != 0:
                self.status |= 4
                continue
            self.table[d], self.length[d] = list(self.table[s]), self.length[s]
            for p in self.table[d]:
                if p >= 0:
                    self.refs[p] += 1

    def trim(self, rows, first, keep):
        for i, b in enumerate(rows):
            if not 0 <= b < self.B:
                continue
            self.length[b] = min(self.length[b], max(keep[i], 0) if keep else self.length[b])
            begin = (min(max(first[i], 0), self.length[b]) if first else 0) // self.page
            for j in range(self.max_pages):
                if not begin <= j < self._count(self.length[b]) and self.table[b][j] >= 0:
                    self.refs[self.table[b][j]] -= 1
                    self.table[b][j] = -1
