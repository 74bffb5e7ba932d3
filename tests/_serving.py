"""Plain 64-bit forms of the serving operators (paged attention, rotation, sampling, page bookkeeping) for the tests."""
import numpy as np


def visible(n, kv, mask_block):
    """Number of keys that each of the last n of kv positions sees."""
    if mask_block == 0:
        return np.full(n, kv)
    p = np.arange(kv - n, kv)
    return np.where(p < 0, 0, np.minimum(kv, (p // mask_block + 1) * mask_block))


def gather(pages, table, kv, page_size):
    """[n_pages, H, page_size, D], one sequence's table -> [H, kv, D]."""
    p = np.arange(kv)
    return pages[table[p // page_size], :, p % page_size].transpose(1, 0, 2)


def attend(q, k, v, lim, scale):
    """q [n, Hq, D], k, v [Hkv, kv, D], lim [n] -> (out, sum_j p_j |v_j|, largest sum |q k| scale), all [n, Hq, D] / scalar."""
    n, hq, d = q.shape
    g = hq // k.shape[0]
    out, mass, size = np.zeros((n, hq, d)), np.zeros((n, hq, d)), 0.0
    for h in range(hq):
        kk, vv = k[h // g], v[h // g]
        s = q[:, h] @ kk.T * scale
        if kk.shape[0]:
            size = max(size, float((np.abs(q[:, h]) @ np.abs(kk).T).max(initial=0) * scale))
        for i in range(n):
            m = int(lim[i])
            if m <= 0:
                continue
            w = np.exp(s[i, :m] - s[i, :m].max())
            w /= w.sum()
            out[i, h] = w @ vv[:m]
            mass[i, h] = w @ np.abs(vv[:m])
    return out, mass, size


def attend_tolerance(out, mass, size, head_dim, kv, bf16):
    """Elementwise bound of the kernels' error.

    A score is a sum of head_dim fp32 products: off by at most head_dim 2^-24 sum|q k| scale, so every weight by that factor
    (twice: numerator and sum), the exponential by 2^-21 (its argument, up to some tens, rounded to 2^-24 of itself, and
    ex2's 2^-22), sums over kv keys and the merges by (kv + 64) 2^-24.  bf16: each weight of the second product rounded
    by 2^-8, the output once more by 2^-8 of itself; fp32: the output by 2^-24."""
    rel = 2 * (head_dim * 2.0 ** -24 * size + 2.0 ** -19) + (kv + 64) * 2.0 ** -24
    last = 2.0 ** -8 if bf16 else 2.0 ** -24
    return mass * (rel + (2.0 ** -8 if bf16 else 0.0)) * 1.01 + np.abs(out) * last + 1e-30


def norm_rope(x, w, eps, pos, inv_freq, rot_dim, interleaved):
    """x [n, H, D] -> (result, |y_a| + |y_b| of the pair that an element was turned with)."""
    y = x.astype(np.float64).copy()
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w
    size = np.abs(y).copy()
    if rot_dim:
        t = pos.astype(np.float64)[:, None] * inv_freq.astype(np.float64)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        lo = slice(0, rot_dim, 2) if interleaved else slice(0, rot_dim // 2)
        hi = slice(1, rot_dim, 2) if interleaved else slice(rot_dim // 2, rot_dim)
        a, b = y[..., lo].copy(), y[..., hi].copy()
        y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
        size[..., lo] = size[..., hi] = np.abs(a) + np.abs(b)
    return y, size


def rope_tolerance(y, size, bf16):
    """The norm: 16 squares summed in a row and up to three more additions, a mean, a root and a quotient (half of the
    sum's 20 roundings, 3 more), two products: 15 x 2^-24.  Sine and cosine: sincospi's 2^-23, the angle's rest to first
    order (2^-25 pi squared: nothing), 2^-24 for putting it back.  Two products and a sum of the pair: 3 x 2^-24.  The result's
    rounding: 2^-8 or 2^-24 of it."""
    return size * 24 * 2.0 ** -24 * 1.01 + np.abs(y) * (2.0 ** -8 if bf16 else 2.0 ** -24) + 1e-37


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row in fp64: (token, probability, kept)."""
    order = np.argsort(-x.astype(np.float64), kind="stable")
    order = order[x[order] > -np.inf]
    if order.size == 0:
        return -1, 0.0, 0
    if temperature <= 0:
        return int(order[0]), 1.0, 1
    z = x[order].astype(np.float64)
    w = np.exp((z - z[0]) / np.float64(temperature))
    run = np.cumsum(w)
    n = order.size if top_k <= 0 else min(order.size, int(top_k))
    k = n
    if top_p < 1:
        k = min(k, int(np.searchsorted(run[:n], np.float64(top_p) * run[n - 1])) + 1)
    if min_p > 0:
        k = min(k, max(1, int((w >= np.float64(min_p)).sum())))
    j = min(int(np.searchsorted(run[:k], np.float64(u) * run[k - 1], side="right")), k - 1)
    return int(order[j]), float(w[j] / run[k - 1]), k


class Pages:
    """The bookkeeping with lists and loops."""

    def __init__(self, table, lens, refs, page_size):
        self.table, self.lens, self.refs, self.ps = table.copy(), lens.copy(), refs.copy(), page_size

    def used(self, b, length=None):
        return -(-int(self.lens[b] if length is None else length) // self.ps)

    def fork(self, src, dst):
        bad, lens, seen = False, self.lens.copy(), set()
        for a, b in zip(src, dst):
            ok = 0 <= a < len(lens) and 0 <= b < len(lens) and lens[b] == 0 and b not in seen
            seen.add(b)
            if not ok:
                bad = True
                continue
            n = -(-int(lens[a]) // self.ps)
            self.table[b, :n] = self.table[a, :n]
            for p in self.table[a, :n]:
                self.refs[p] += 1
            self.lens[b] = lens[a]
        return bad

    def reserve(self, write_from, new_lens, cap):
        """Pairs, or None where nothing changes."""
        before, limit = self.refs.copy(), self.table.shape[1] * self.ps
        free = [int(p) for p in np.flatnonzero(before == 0)]
        plan, at = [], 0
        for b in range(len(self.lens)):
            if new_lens[b] > limit:
                return None
            have, upto = self.used(b), -(-max(int(new_lens[b]), 0) // self.ps)
            start = max(int(write_from[b]), 0) // self.ps if max(int(write_from[b]), 0) < new_lens[b] else upto
            for e in range(start, min(have, upto)):
                if before[self.table[b, e]] > 1:
                    plan.append((b, e, True))
            for e in range(have, upto):
                plan.append((b, e, False))
        if len(plan) > len(free) or sum(c for _, _, c in plan) > cap:
            return None
        pairs = []
        for b, e, copied in plan:
            page = free[at]
            at += 1
            if copied:
                pairs.append((int(self.table[b, e]), page))
                self.refs[self.table[b, e]] -= 1
            self.table[b, e] = page
            self.refs[page] = 1
        self.lens = np.maximum(self.lens, new_lens)
        return pairs

    def release(self, keep):
        for b in range(len(self.lens)):
            k = max(int(keep[b]), 0)
            if k >= self.lens[b]:
                continue
            for e in range(-(-k // self.ps), self.used(b)):
                self.refs[self.table[b, e]] -= 1
                self.table[b, e] = -1
            self.lens[b] = k

    def compact(self):
        u = int((self.refs > 0).sum())
        dst = [p for p in range(u) if self.refs[p] == 0]
        src = [p for p in range(u, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(src, dst))
        for b in range(len(self.lens)):
            for e in range(self.used(b)):
                self.table[b, e] = to.get(int(self.table[b, e]), self.table[b, e])
        for a, b in zip(src, dst):
            self.refs[b], self.refs[a] = self.refs[a], 0
        return list(zip(src, dst))
