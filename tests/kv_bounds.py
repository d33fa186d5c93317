"""Attention over the 4-bit cache in 64 bits with the error that the tensor-core kernel's roundings leave, as a distribution.

What the kernel rounds, each to 11 bits and each once: a key's scale and its products scale (code - zero); a value's scale and its
products; a weight.  A rounding to 11 bits moves x by at most 2^-11 |x|, spread evenly over that range at worst: a standard
deviation of at most U |x|, U = 2^-11 / sqrt(3).  Roundings of different tokens (and of different channels of a product) are
independent, so variances add:

    var score_j = U^2 (score_j^2 + scale^2 sum_i (q_i k_ji)^2)
    var out_d   = sum_j p_j^2 (var score_j (v_jd - out_d)^2 + 3 U^2 v_jd^2)
    var lse     = sum_j p_j^2 var score_j

What is not independent is bounded as it adds up: sums in float32 (a score's products in groups of 16 at least, (16 + 16) 2^-23 of
their absolute sum; a sum over the keys 2^-23 for every 16 of them, and 2^-20 for exponentials and rescalings), and weights so small
that they are no normal fp16 numbers (2^-25 each, where the largest lies at 2^6).  The output's own rounding to bf16 is at most 2^-8 of
the value, 2^-8 / sqrt(3) as a deviation.  An element may be off by ten deviations, the root of the sum of squares over a head's
rows by 1.5: U is the deviation of a number just above a power of two, 1.4 times that of the mean number."""
import numpy as np
import torch

U = 2.0 ** -11 / 3 ** 0.5


def values(codes, param):
    """uint8 [..., d/2], float32 [..., 2] -> float64 [..., d]"""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    return (c - param[..., 1:2].double()) * param[..., 0:1].double()


def expect(layer, table, lens, starts, q, scale, causal):
    """layer: (k_codes, k_param, v_codes, v_param) of one layer, table numpy, q [rows][heads][d].  Returns a dict of float64 tensors on
    q's device: out, lse, and for both the deviation (sd) and what adds up (drift)."""
    kc, kp, vc, vp = layer
    rows, heads, d = q.shape
    group, page, dev = heads // kc.shape[1], kc.shape[2], q.device
    r = {n: torch.zeros(rows, heads, d, dtype=torch.float64, device=dev) for n in ("out", "sd", "drift")}
    r.update({n: torch.zeros(rows, heads, dtype=torch.float64, device=dev) for n in ("lse", "lse_sd", "lse_drift")})
    r["lse"] -= torch.inf
    for s, length in enumerate(lens):
        a, b = int(starts[s]), int(starts[s + 1])
        n = b - a
        if n <= 0 or length <= 0:
            continue
        pos = np.arange(length)
        pg, at = torch.as_tensor(np.asarray(table)[s][pos // page].astype(np.int64), device=dev), torch.as_tensor(pos % page, device=dev)
        keys, vals = values(kc[pg, :, at], kp[pg, :, at]), values(vc[pg, :, at], vp[pg, :, at])
        sees = torch.arange(length - n + 1, length + 1, device=dev).clamp(0, length) if causal else torch.full((n,), length, device=dev)
        hidden = torch.arange(length, device=dev)[None] >= sees[:, None]
        some = (sees > 0)[:, None]
        for h in range(heads):
            k, v, x = keys[:, h // group], vals[:, h // group], q[a:b, h].double()
            score = (scale * x @ k.T).masked_fill(hidden, -torch.inf)
            lse = torch.logsumexp(score, 1, keepdim=True)
            p = torch.where(some, torch.exp(score - lse), 0.0).masked_fill(hidden, 0.0)
            score = score.masked_fill(hidden, 0.0)
            var = U * U * (score ** 2 + scale ** 2 * (x ** 2) @ (k.T ** 2))
            add = 2.0 ** -18 * abs(scale) * x.abs() @ k.T.abs()
            out, pv = p @ v, p @ v.abs()
            w = p * p * var
            sums = sees[:, None].double() / 16 * 2.0 ** -23 + 2.0 ** -20
            small = sees[:, None].double() * 2.0 ** -31 * (p.amax(1, keepdim=True) * v.abs().amax())
            r["out"][a:b, h] = out
            r["sd"][a:b, h] = (w @ v ** 2 - 2 * out * (w @ v) + out ** 2 * w.sum(1, keepdim=True) + 3 * U * U * (p * p) @ v ** 2).clamp(min=0).sqrt()
            r["drift"][a:b, h] = (p * add) @ v.abs() + (p * add).sum(1, keepdim=True) * out.abs() + 2 * sums * pv + small
            r["lse"][a:b, h] = torch.where(some, lse, -torch.inf)[:, 0]
            r["lse_sd"][a:b, h] = w.sum(1).sqrt()
            r["lse_drift"][a:b, h] = (p * add).sum(1) + sums[:, 0] + torch.where(some, 2.0 ** -22 * (1 + lse.abs()), 0.0)[:, 0]
    return r


def check(got, lse, want, rows=None):
    """`rows`: the rows to look at (all by default).  lse may be None."""
    pick = (lambda t: t) if rows is None else (lambda t: t[rows])
    out, sd, drift = pick(want["out"]), pick(want["sd"]), pick(want["drift"])
    err = (pick(got).double() - out).abs()
    assert bool(torch.isfinite(err).all()), "not finite"
    tol = 2.0 ** -8 * (out.abs() + 10 * sd + drift) + 10 * sd + drift + 1e-300
    assert bool((err <= tol).all()), "an element is off by %.3g times its bound" % (err / tol).max()
    root = lambda t: t.square().sum((0, 2)).sqrt()  # noqa: E731
    most = 1.5 * (sd.square().sum((0, 2)) + (2.0 ** -16 / 3) * out.square().sum((0, 2))).sqrt() + root(drift) + 1e-300
    assert bool((root(err) <= most).all()), "a head is off by %.3g times its bound" % (root(err) / most).max()
    if lse is None:
        return
    ref, bound = pick(want["lse"]), 10 * pick(want["lse_sd"]) + pick(want["lse_drift"])
    l = pick(lse).double()
    assert torch.equal(torch.isneginf(l), torch.isneginf(ref))
    fin = torch.isfinite(ref)
    assert bool(((l - ref).abs() <= bound)[fin].all()), "a logarithm is off by %.3g times its bound" % ((l - ref).abs() / bound)[fin].max()
