"""Plain 64-bit forms of the paged attention operators, on the CPU: rows and pages as numpy arrays, one loop per definition."""
import numpy as np
import torch


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def per_group(dtype):
    return 8 if dtype == torch.bfloat16 else 4


def f64(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- norm and rotation
def rotate(y, pos, freq, interleaved):
    """y [T, h, d] turned by pos [T] * freq [rot / 2]."""
    half = len(freq)
    y = np.array(y, np.float64)
    if half == 0:
        return y
    a = (np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64))[:, None]
    c, s = np.cos(a), np.sin(a)
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = u * c - v * s, v * c + u * s
    return y


def heads(x, w, pos, freq, eps, interleaved=False):
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return rotate(x, pos, freq, interleaved)


def heads_backward(dy, x, w, pos, freq, eps, interleaved=False):
    """(gradient of x, gradient of w)."""
    x = np.asarray(x, np.float64)
    g = rotate(dy, pos, -np.asarray(freq, np.float64), interleaved)
    if w is None:
        return g, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, h = x * r, g * w
    return r * (h - xh * (h * xh).mean(-1, keepdims=True)), (g * xh).sum((0, 1))


# ---------------------------------------------------------------- pools
def pool_rows(k_pages, v_pages, layer, numbers):
    """Keys and values [tokens, Hkv, d] of the pages `numbers`, one after the other (CPU tensors of any type)."""
    k, v = k_pages[layer][numbers], v_pages[layer][numbers]       # [n, Hkv, d/E, page, E], [n, Hkv, page/E, d, E]
    n, Hkv, g, page, E = k.shape
    return (k.permute(0, 3, 1, 2, 4).reshape(n * page, Hkv, g * E), v.permute(0, 2, 4, 1, 3).reshape(n * page, Hkv, g * E))


class Book:
    """The bookkeeping in plain Python: what the calls do to it, one sequence and page at a time."""

    def __init__(self, seqs, pages, max_pages, page):
        self.page, self.max_pages = page, max_pages
        self.lens, self.refs = [0] * seqs, [0] * pages
        self.table = [[-1] * max_pages for _ in range(seqs)]
        self.status = [0] * 8

    def count(self, n):
        return -(-n // self.page)

    def _free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def reserve(self, seqs, add):
        bad = 0
        if len(set(seqs)) < len(seqs) or any(s < 0 or s >= len(self.lens) for s in seqs) or any(a < 0 for a in add):
            bad |= 4
        ok = [(s, a) for s, a in zip(seqs, add) if 0 <= s < len(self.lens) and a >= 0]
        if any(self.count(self.lens[s] + a) > self.max_pages for s, a in ok):
            bad |= 2
        free = self._free()
        if not bad and sum(self.count(self.lens[s] + a) - self.count(self.lens[s]) for s, a in ok) > len(free):
            bad |= 1
        if bad:
            self.status[0] |= bad
            return
        for s, a in ok:
            for j in range(self.count(self.lens[s]), self.count(self.lens[s] + a)):
                p = free.pop(0)
                self.table[s][j], self.refs[p] = p, 1
            self.lens[s] += a

    def fork(self, src, dst):
        """The (page, page, tokens) that are copied."""
        if len(set(dst)) < len(dst) or set(src) & set(dst) or any(not 0 <= s < len(self.lens) for s in src + dst):
            self.status[0] |= 4
            return []
        if any(self.lens[b] for b in dst):
            self.status[0] |= 8
            return []
        free = self._free()
        if sum(self.lens[a] % self.page > 0 for a in src) > len(free):
            self.status[0] |= 1
            return []
        copies = []
        for a, b in zip(src, dst):
            full, rest = divmod(self.lens[a], self.page)
            for j in range(full):
                self.table[b][j] = self.table[a][j]
                self.refs[self.table[a][j]] += 1
            if rest:
                p = free.pop(0)
                copies.append((self.table[a][full], p, rest))
                self.table[b][full], self.refs[p] = p, 1
            self.lens[b] = self.lens[a]
        self.status[1] = len(copies)
        return copies

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens):
                self.status[0] |= 4
                continue
            for j in range(self.count(self.lens[s])):
                self.refs[self.table[s][j]] -= 1
                self.table[s][j] = -1
            self.lens[s] = 0

    def compact(self):
        """The (page, page) that move."""
        live = sum(r > 0 for r in self.refs)
        moves = list(zip([p for p, r in enumerate(self.refs) if r > 0 and p >= live], [p for p, r in enumerate(self.refs) if r == 0 and p < live]))
        to = dict(moves)
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        self.status[1], self.status[2] = len(moves), live
        return moves

    def words(self):
        return self.status + self.lens + self.refs + [p for row in self.table for p in row]


# ---------------------------------------------------------------- attention
def attend(q, k, v, scale, window=0, there=None):
    """q [n, H, d] are the last tokens of the sequence with keys and values k, v [m, Hkv, d]; `there` [m]: tokens that exist (all).
    Keys that a row does not see are left out of its sums altogether.  Returns out [n, H, d], lse [n, H]."""
    n, H, d = q.shape
    m, Hkv = k.shape[:2]
    out, lse = np.zeros((n, H, d)), np.full((n, H), -np.inf)
    for i in range(n):
        p = m - n + i
        seen = [j for j in range(max(0, p - window + 1) if window else 0, p + 1) if there is None or there[j]]
        if not seen:
            continue
        for h in range(H):
            s = scale * (k[seen, h // (H // Hkv)] @ q[i, h])
            top = s.max()
            e = np.exp(s - top)
            with np.errstate(invalid="ignore"):
                out[i, h] = (e[:, None] * v[seen, h // (H // Hkv)]).sum(0) / e.sum()
            lse[i, h] = top + np.log(e.sum())
    return out, lse


def attend_bound(q, k, v, scale, dtype, window=0, there=None):
    """How far an element of the output may be off, [n, H, d]: half a step for each rounded weight and value's sum, half a step for the output, and the
    arithmetic of 32 bits.  With weights p_j, |error| <= sum_j p_j |v_j| (weights' rounding + scores' error) + |o| (output's rounding); the scores, sums of d
    products, are off by at most (d + 4) 2^-24 sum_c |q_c k_c| scale, and sums over m keys add m 2^-24 (a bound; what it really is grows with the
    square root)."""
    n, H, d = q.shape
    m, Hkv = k.shape[:2]
    u32, u = 2.0 ** -24, half_step(dtype)
    bound = np.zeros((n, H, d))
    for i in range(n):
        p = m - n + i
        seen = [j for j in range(max(0, p - window + 1) if window else 0, p + 1) if there is None or there[j]]
        if not seen:
            continue
        for h in range(H):
            g = h // (H // Hkv)
            s = scale * (k[seen, g] @ q[i, h])
            e = np.exp(s - s.max())
            e /= e.sum()
            score = scale * (np.abs(k[seen, g]) @ np.abs(q[i, h])) * (d + 4) * u32 + 8 * u32
            weight = (u if dtype == torch.bfloat16 else 0) + 2 * score.max() + (len(seen) + 16) * u32
            bound[i, h] = (e[:, None] * np.abs(v[seen, g])).sum(0) * (weight + u) + 1e-30
    return bound
