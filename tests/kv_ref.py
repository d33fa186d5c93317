"""Plain 64-bit statements of the 4-bit key/value cache (numpy): storing, reading, attention, the pool of pages."""
import numpy as np


def unpack(codes):
    out = np.empty(codes.shape[:-1] + (2 * codes.shape[-1],), np.float64)
    out[..., 0::2] = codes & 15
    out[..., 1::2] = codes >> 4
    return out


def quantize(x):
    """float32 [..., d] -> codes uint8 [..., d/2], scale, zero float32 [...]: scale and zero-point in the float32 arithmetic of the
    quantizer, x / alpha as the exact product of x with the float32 reciprocal (float64 holds it), rounded once.  Rows whose
    quotients or zero-point pass 2^21 are rounded as float32 products."""
    x = np.asarray(x, np.float32)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    alpha = np.where(hi > lo, (hi - lo) / np.float32(15), np.where(lo != 0, np.abs(lo), np.float32(1))).astype(np.float32)
    inv = np.float32(1) / alpha
    zero = -np.rint(lo * inv)
    small = (np.maximum(np.abs(lo), np.abs(hi)) * inv < 2097152) & (np.abs(zero) < 2097152)
    q = np.where(small, np.rint(x.astype(np.float64) * inv), np.rint(x * inv).astype(np.float64))
    q = np.where(small, q + zero, (q.astype(np.float32) + zero).astype(np.float64))
    q = np.clip(q, 0, 15).astype(np.uint8)
    return q[..., 0::2] | (q[..., 1::2] << 4), alpha[..., 0], zero[..., 0]


class Store:
    """Host copies of one layer's arrays: codes uint8 [pages][heads][page][d/2], param float32 [pages][heads][page][2]."""

    def __init__(self, k_codes, k_param, v_codes, v_param):
        self.kc, self.kp, self.vc, self.vp = k_codes, k_param, v_codes, v_param
        self.pages, self.heads, self.page, self.d = k_codes.shape[0], k_codes.shape[1], k_codes.shape[2], 2 * k_codes.shape[3]

    def rows(self, table_row, first, last):
        """(codes, param) x keys, values of positions first .. last - 1: [n][heads][...]"""
        pos = np.arange(first, last)
        pg, at = table_row[pos // self.page], pos % self.page
        return (unpack(self.kc[pg, :, at]), self.kp[pg, :, at].astype(np.float64),
                unpack(self.vc[pg, :, at]), self.vp[pg, :, at].astype(np.float64))


def attention(store, table, lens, starts, q, scale, causal):
    """q float64 [rows][q_heads][d].  Returns out, lse and, for tolerances, three magnitudes per output:
    spread = sum_j p_j vs_j (|cv_j| + |vz_j|) (what rounding a weight can move), and per row the largest
    |score| built without cancellation, scale ks_j (sum |q| c_j + |z_j| sum |q|), and the number of keys."""
    rows, qh, d = q.shape
    out, lse = np.zeros((rows, qh, d)), np.full((rows, qh), -np.inf)
    spread, mag, seen = np.zeros((rows, qh, d)), np.zeros((rows, qh)), np.zeros((rows, qh))
    g = qh // store.heads
    for s in range(len(lens)):
        n = starts[s + 1] - starts[s]
        if n <= 0:
            continue
        kc, kp, vc, vp = store.rows(table[s], 0, lens[s])
        for i in range(n):
            t = starts[s] + i
            keys = min(lens[s], max(0, lens[s] - n + i + 1)) if causal else lens[s]
            if keys == 0:
                continue
            for h in range(qh):
                c, p = kc[:keys, h // g], kp[:keys, h // g]
                sc = scale * p[:, 0] * (c @ q[t, h] - p[:, 1] * q[t, h].sum())
                m = sc.max()
                w = np.exp(sc - m)
                l = w.sum()
                v, z = vc[:keys, h // g], vp[:keys, h // g]
                out[t, h] = (w * z[:, 0] / l) @ (v - z[:, 1:2])
                spread[t, h] = (w * np.abs(z[:, 0]) / l) @ (v + np.abs(z[:, 1:2]))
                lse[t, h] = m + np.log(l)
                mag[t, h] = (abs(scale) * np.abs(p[:, 0]) * (c @ np.abs(q[t, h]) + np.abs(p[:, 1]) * np.abs(q[t, h]).sum())).max()
                seen[t, h] = keys
    return out, lse, spread, mag, seen


class Pool:
    """The pool's rules, one entry after the other."""

    def __init__(self, pages, seqs, width, page):
        self.refs = np.zeros(pages, np.int32)
        self.table = np.full((seqs, width), -1, np.int32)
        self.lens = np.zeros(seqs, np.int32)
        self.page = page
        self.failed = False
        self.copies = []                                    # (from, to) pages whose contents were copied, in order

    def _n(self, length):
        return -(-length // self.page)

    def extend(self, add):
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        asked = 0
        for s, more in enumerate(add):
            have, want = self._n(int(self.lens[s])), self._n(int(self.lens[s]) + int(more))
            if more < 0 or want > self.table.shape[1] or want - have > len(self.refs):
                self.failed = True
                continue
            need = want - have
            asked += need
            if need and asked > len(free):
                self.failed = True
                continue
            for j in range(need):
                p = free[asked - need + j]
                self.table[s, have + j] = p
                self.refs[p] = 1
            self.lens[s] += more

    def fork(self, parent, child):
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        n, used, fresh = len(self.lens), 0, []
        lens0 = self.lens.copy()
        for i, (a, c) in enumerate(zip(parent, child)):
            ok = 0 <= a < n and 0 <= c < n and c not in child[:i] and a not in child and lens0[c] == 0
            if not ok:
                self.failed = True
                fresh.append(-2)
                continue
            length = int(self.lens[a])
            full, rest = divmod(length, self.page)
            if rest:
                used += 1
                if used > len(free):
                    self.failed = True
                    fresh.append(-2)
                    continue
            for j in range(full):
                self.table[c, j] = self.table[a, j]
                self.refs[self.table[a, j]] += 1
            fresh.append(-1)
            if rest:
                fresh[-1] = free[used - 1]
                self.table[c, full] = fresh[-1]
                self.refs[fresh[-1]] = 1
                self.copies.append((int(self.table[a, full]), fresh[-1]))
            self.lens[c] = length
        return fresh

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens):
                self.failed = True
                continue
            for p in self.table[s][self.table[s] >= 0]:
                self.refs[p] -= 1
            self.table[s] = -1
            self.lens[s] = 0

    def compact(self):
        used = int((self.refs > 0).sum())
        holes = [p for p in range(used) if self.refs[p] == 0]
        remap = np.where(self.refs > 0, np.arange(len(self.refs)), -1).astype(np.int32)
        for p in range(used, len(self.refs)):
            if self.refs[p] > 0:
                to = holes.pop(0)
                remap[p] = to
                self.copies.append((p, to))
        refs = np.zeros_like(self.refs)
        for p, to in enumerate(remap):
            if to >= 0:
                refs[to] = self.refs[p]
        self.table = np.where(self.table >= 0, remap[np.maximum(self.table, 0)], -1).astype(np.int32)
        self.refs = refs
        return remap
