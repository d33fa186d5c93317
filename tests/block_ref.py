"""Plain statements of what stands around a quantized projection (numpy / torch): the decisions of the quantizer in float32 as they are
documented, everything else in 64 bits."""
import numpy as np
import torch


def decide(u, bits):
    """float32 rows [..., d] -> codes (float64), scale, zero (float32 [..., 1]): Eq. 2 as qllm_quantize_rows takes it.  x / alpha is the
    exact product of x with alpha's float32 reciprocal, rounded once; rows whose quotients or zero-point pass 2^21 are rounded as
    float32 products."""
    u = np.asarray(u, np.float32)
    one, top = np.float32(1), np.float32(2 ** bits - 1)
    lo, hi = u.min(-1, keepdims=True), u.max(-1, keepdims=True)
    alpha = np.where(hi > lo, (hi - lo) / top, np.where(lo != 0, np.abs(lo), one)).astype(np.float32)
    inv = one / alpha
    zero = -np.rint(lo * inv)
    small = (np.maximum(np.abs(lo), np.abs(hi)) * inv < 2097152) & (np.abs(zero) < 2097152)
    q = np.where(small, np.rint(u.astype(np.float64) * inv) + zero, (np.rint(u * inv) + zero).astype(np.float64))
    return np.clip(q, 0, float(top)), alpha, zero


def unpack(codes, bits):
    if bits != 4:
        return codes.astype(np.float64)
    out = np.empty(codes.shape[:-1] + (2 * codes.shape[-1],), np.float64)
    out[..., 0::2] = codes & 15
    out[..., 1::2] = codes >> 4
    return out


def norm(x, residual, gamma, eps, csr, bits):
    """x, residual: float32 arrays (residual may be None).  Returns h, y, factor (float64), codes, zero, alpha of u' (float32), u'."""
    x = np.asarray(x, np.float32)
    h32 = x if residual is None else (x + residual).astype(np.float32)
    h = x.astype(np.float64) + (0 if residual is None else residual)
    factor = 1.0 / np.sqrt(np.square(h).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
    u = (h32 * gamma).astype(np.float32)
    if csr is not None:
        ptr, src, coef = csr
        u = np.stack([(u[:, src[b:e]].astype(np.float64) * coef[b:e].astype(np.float64)).sum(1) for b, e in zip(ptr[:-1], ptr[1:])], 1).astype(np.float32)
    codes, alpha, zero = decide(u, bits)
    return h, h * gamma.astype(np.float64) * factor, factor, codes, zero, alpha, u


def random_map(rng, c):
    """A reassembly map with c rows: some channels split into 2 to 5 parts, as many saved by averaging sets of 2 to 12 channels."""
    order, parts, extra = list(rng.permutation(c)), np.ones(c, np.int64), max(1, c // 7)
    while extra > 0:
        n = min(extra, int(rng.randint(1, 5)))
        parts[order.pop()] += n
        extra -= n
    need, merged, gone = int(parts.sum()) - c, {}, set()
    while need > 0:
        n = min(need, int(rng.choice([1, 1, 1, 2, 3, 11])), len(order) - 1)
        into = int(order.pop())
        merged[into] = [into] + [int(order.pop()) for _ in range(n)]
        gone.update(merged[into][1:])
        need -= n
    rows, coef = [], []
    for i in range(c):
        if i in gone:
            continue
        for _ in range(parts[i]):
            r = merged.get(i, [i])
            rows.append(r)
            coef.append([1.0 / parts[i] if len(r) == 1 else 1.0 / len(r)] * len(r))
    ptr = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
    return ptr, np.concatenate(rows).astype(np.int32), np.concatenate(coef).astype(np.float32)


def adapters(A, Bm, scale, rank, x, base, start, adapter):
    """All in float64 on the tensors' device; start, adapter: lists.  Returns (out, what the sums are made of without signs: of the first
    product carried through the second, and of the second)."""
    out = base.double().clone()
    first, second = torch.zeros_like(out), torch.zeros_like(out)
    for s, a in enumerate(adapter):
        r0, r1 = start[s], start[s + 1]
        if a < 0 or r1 <= r0:
            continue
        n = int(rank[a])
        aa, bb, xx, sc = A[a, :n].double(), Bm[a, :, :n].double(), x[r0:r1].double(), float(scale[a])
        inner = xx @ aa.T
        out[r0:r1] += sc * (inner @ bb.T)
        first[r0:r1] = abs(sc) * ((xx.abs() @ aa.abs().T) @ bb.abs().T)
        second[r0:r1] = abs(sc) * (inner.abs() @ bb.abs().T)
    return out, first, second


def turned(x, cos, sin, rot_dim, interleaved, kind=np.float32):
    """Rows [t][heads][d] turned by cos, sin [t][rot_dim / 2]; in `kind`, an operation at a time."""
    x, c, s = x.astype(kind), cos.astype(kind)[:, None], sin.astype(kind)[:, None]
    out = x.copy()
    i = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if interleaved else (slice(0, rot_dim // 2), slice(rot_dim // 2, rot_dim))
    a, b = x[..., i[0]], x[..., i[1]]
    out[..., i[0]] = a * c - b * s
    out[..., i[1]] = b * c + a * s
    return out
