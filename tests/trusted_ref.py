"""What the operators of the trusted half compute, in 64 bits on the CPU, from bifrost.h alone."""
import numpy as np


def rows_of(starts, n):
    return [int(starts[i + 1] - starts[i]) for i in range(n)] if starts is not None else [1] * n


# ---- the cache's layout, place by place

def places(D, G):
    """(key nibble, key parameter half, value nibble, value parameter half): offsets of [token][channel or group] in a sub-block; nibbles
    count from the sub-block's start."""
    u, c = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    kw = u // 8 + 2 * (c // 32 % 2) + 4 * (c // 8 % 4) + 16 * (u % 8) + 128 * (c // 64)
    vw = c // 16 % 4 + 4 * (u // 2 % 4) + 16 * (c % 8) + 128 * (c // 64)
    E = D // G
    ug, e = np.meshgrid(np.arange(16), np.arange(E), indexing="ij")
    k_par, v_code, v_par = 8 * D, 8 * D + 64 * E, 16 * D + 64 * E
    kn = 8 * kw + c % 8
    vn = 2 * v_code + 8 * vw + c // 8 % 2 + 2 * (u // 8) + 4 * (u % 2)
    kp = k_par // 2 + 2 * (e + E * (ug // 8 + 2 * (ug % 8)))
    vp = v_par // 2 + ug % 2 + 2 * (ug // 8) + 8 * (ug // 2 % 4) + 32 * e
    return kn, kp, vn, vp


def quantise(x, G):
    """(codes, scale, low) of float64 [..., D]."""
    x = np.clip(x, -61440.0, 61440.0).reshape(*x.shape[:-1], -1, G)
    with np.errstate(all="ignore"):
        low, high = x.min(-1), x.max(-1)
        s = ((high - low) / 15.0).astype(np.float32).astype(np.float16)
        m = low.astype(np.float32).astype(np.float16)
        q = np.where(s[..., None] > 0, np.rint((x - m[..., None].astype(np.float64)) / s[..., None].astype(np.float64)), 0)
        q = np.nan_to_num(np.clip(q, 0, 15), nan=0.0).astype(np.uint8)
    return q.reshape(*q.shape[:-2], -1), s, m


class Cache:
    """A cache on the host: pool bytes and tables, with the operators on it."""

    def __init__(self, layers, pages, heads, D, G, T, seqs, max_pages, seed=0):
        rng = np.random.default_rng(seed)
        self.layers, self.pages, self.heads, self.D, self.G, self.T, self.seqs, self.max_pages = layers, pages, heads, D, G, T, seqs, max_pages
        self.sub = 16 * D + 128 * (D // G)
        # what nobody wrote may hold anything, NaN among the parameters
        self.pool = rng.integers(0, 256, (layers, pages, heads, T // 16, self.sub), dtype=np.uint8)
        self.pool[..., 8 * D:8 * D + 64 * (D // G)] = 0xFF
        self.pool[..., 16 * D + 64 * (D // G):] = 0xFF
        self.tables = np.full((seqs, max_pages), -1, np.int32)
        self.lengths = np.zeros(seqs, np.int32)
        self.refs = np.zeros(pages, np.int32)
        self.kn, self.kp, self.vn, self.vp = places(D, G)

    # -- elements
    def put(self, layer, seq, t, k, v):
        """k, v: float64 [heads][D]."""
        block = self.pool[layer, self.tables[seq, t // self.T]]
        for h in range(self.heads):
            sub = block[h, t % self.T // 16]
            half = sub.view(np.float16)
            for x, nib, par, low_at in ((k[h], self.kn, self.kp, 1), (v[h], self.vn, self.vp, 4)):
                q, s, m = quantise(x, self.G)
                n = nib[t % 16]
                keep = np.where(n % 2 == 0, 0xF0, 0x0F).astype(np.uint8)
                for b, kp_, qv, sh in zip(n // 2, keep, q, 4 * (n % 2)):
                    sub[b] = (sub[b] & kp_) | (int(qv) << int(sh))
                half[par[t % 16]], half[par[t % 16] + low_at] = s, m

    def get(self, layer, seq, n):
        """Keys and values of tokens 0 .. n-1: float64 [n][heads][D]."""
        out = []
        t = np.arange(n)
        blocks = self.pool[layer][self.tables[seq, t // self.T], :, t % self.T // 16]            # [n][heads][bytes]
        half = blocks.view(np.float16).astype(np.float64)
        g = np.arange(self.D) // self.G
        for nib, par, low_at in ((self.kn, self.kp, 1), (self.vn, self.vp, 4)):
            nb, pb = nib[t % 16], par[t % 16][:, g]
            idx = np.broadcast_to(nb[:, None, :] // 2, (n, self.heads, self.D))
            code = (np.take_along_axis(blocks, idx, 2) >> (4 * (nb % 2))[:, None, :].astype(np.uint8)) & 15
            pidx = np.broadcast_to(pb[:, None, :], (n, self.heads, self.D))
            out.append(code * np.take_along_axis(half, pidx, 2) + np.take_along_axis(half, pidx + low_at, 2))
        return out

    def top(self, layer, seq, n):
        """Bound of |low| + 15 scale of keys and values: float64 [n][heads][D] each."""
        out = []
        t = np.arange(n)
        blocks = self.pool[layer][self.tables[seq, t // self.T], :, t % self.T // 16]
        half = np.abs(blocks.view(np.float16).astype(np.float64))
        g = np.arange(self.D) // self.G
        for par, low_at in ((self.kp, 1), (self.vp, 4)):
            pidx = np.broadcast_to(par[t % 16][:, g][:, None, :], (n, self.heads, self.D))
            out.append(15 * np.take_along_axis(half, pidx, 2) + np.take_along_axis(half, pidx + low_at, 2))
        return out

    # -- pages
    def free_pages(self):
        return [p for p in range(self.pages) if self.refs[p] == 0]

    def grow(self, seqs, counts):
        bad = set()
        seen, free, need_so_far = set(), self.free_pages(), 0
        for a, more in zip(seqs, counts):
            if not 0 <= a < self.seqs or a in seen or more < 0 or self.lengths[a] + more > self.max_pages * self.T:
                bad.add("range")
                continue
            seen.add(a)
            have, want = -(-int(self.lengths[a]) // self.T), -(-(int(self.lengths[a]) + more) // self.T)
            if want > have:
                need_so_far += want - have
                if need_so_far > len(free):
                    bad.add("oom")
                    continue
                for i, p in enumerate(free[need_so_far - (want - have):need_so_far]):
                    self.tables[a, have + i] = p
                    self.refs[p] = 1
            self.lengths[a] += more
        return bad

    def fork(self, src, dst):
        bad, seen, free, used = set(), set(), self.free_pages(), 0
        for a, b in zip(src, dst):
            if not (0 <= a < self.seqs and 0 <= b < self.seqs) or b in seen or a in dst or self.lengths[b] != 0:
                bad.add("range")
                continue
            seen.add(b)
            n = int(self.lengths[a])
            full = n // self.T
            if n % self.T:
                used += 1
                if used > len(free):
                    bad.add("oom")
                    continue
                p = free[used - 1]
                self.pool[:, p] = self.pool[:, self.tables[a, full]]
                self.refs[p] = 1
            self.tables[b] = -1
            self.tables[b, :full] = self.tables[a, :full]
            self.refs[self.tables[a, :full]] += 1
            if n % self.T:
                self.tables[b, full] = p
            self.lengths[b] = n
        return bad

    def free(self, seqs):
        for a in seqs:
            n = -(-int(self.lengths[a]) // self.T)
            for p in self.tables[a, :n]:
                self.refs[p] -= 1
            self.tables[a, :n] = -1
            self.lengths[a] = 0

    def compact(self):
        n_live = int((self.refs > 0).sum())
        holes = [p for p in range(n_live) if self.refs[p] == 0]
        movers = [p for p in range(n_live, self.pages) if self.refs[p] > 0]
        for h, m in zip(holes, movers):
            self.pool[:, h] = self.pool[:, m]
            self.tables[self.tables == m] = h
            self.refs[h], self.refs[m] = self.refs[m], 0
        return n_live


def attention(cache, layer, seq, q, scale, window):
    """q float64 [rows][q heads][D] of one sequence -> (out, lse, tolerance of out before its own rounding, tolerance of lse).

    The tolerance counts what bifrost.h states: probabilities and values rounded to fp16 for their product, 2^-11 of each (2^-25
    where that is below the type's normal range), and sums in 32 bits.  A matrix instruction adds 16 products to an
    accumulator with an error of at most 2^-22 of the largest magnitude met, whatever the order; a score's is D/16 of those on
    sum |q| (|low| + 15 scale), and as many again for the parameters' sums; q itself is taken relative to the largest of
    its row, 2^-24 of that.  An error d of a score is a factor e^d on its probability, in numerator and denominator both."""
    n, H, D = q.shape
    L = int(cache.lengths[seq])
    k, v = cache.get(layer, seq, L)
    kt, vt = cache.top(layer, seq, L)
    per = H // cache.heads
    out, lse, tol, tol_l = np.zeros((n, H, D)), np.full((n, H), -np.inf), np.zeros((n, H, D)), np.zeros((n, H))
    for j in range(n):
        pos = L - n + j
        lo = max(0, pos - window + 1) if window else 0
        if pos < lo or pos < 0:
            continue
        for h in range(H):
            kk, vv = k[lo:pos + 1, h // per], v[lo:pos + 1, h // per]
            s = scale * (kk @ q[j, h])
            e = np.exp(s - s.max())
            p = e / e.sum()
            out[j, h], lse[j, h] = p @ vv, s.max() + np.log(e.sum())
            mag = abs(scale) * (kt[lo:pos + 1, h // per] @ (np.abs(q[j, h]) + 2.0 ** -24 * np.abs(q[j, h]).max()))
            d = 2.0 ** -22 * (2 * (D / 16) + 8) * mag.max() + 2.0 ** -22 * np.abs(s).max() + abs(scale) * kt.max() * D * 2.0 ** -24 * np.abs(q[j, h]).max()
            steps = 2.0 ** -22 * (len(s) / 16 + 16)
            tol[j, h] = (2.0 ** -11 + 2.0 ** -11 + 2 * np.expm1(d) + 2 * steps) * (p @ vt[lo:pos + 1, h // per]) + 2.0 ** -24
            tol_l[j, h] = d + 2 * steps + 2.0 ** -22 * (np.abs(lse[j, h]) + 1)
    return out, lse, tol, tol_l
