"""The bounds that the tensor-core attention kernel's tests use, tried on the CPU: the kernel's roundings pass, planted mistakes do not."""
import numpy as np
import pytest
import torch

import kv_bounds


def fp16(x):
    return x.to(torch.float16).double()


def emulate(layer, table, lens, starts, q, scale, key_scale=1.0, value_scale=1.0, value_zero=0.0):
    """The tensor-core kernel's roundings on the CPU, causal: scales and products in fp16 under a tile's exponent, weights in fp16."""
    kc, kp, vc, vp = layer
    rows, heads, d = q.shape
    group, page = heads // kc.shape[1], kc.shape[2]
    out, lse = torch.zeros(rows, heads, d, dtype=torch.float64), torch.full((rows, heads), -torch.inf, dtype=torch.float64)
    for s, length in enumerate(lens):
        n = starts[s + 1] - starts[s]
        pos = np.arange(length)
        pg, at = torch.as_tensor(table[s][pos // page].astype(np.int64)), torch.as_tensor(pos % page)
        both = []
        for codes, param, f, z in ((kc, kp, key_scale, 0.0), (vc, vp, value_scale, value_zero)):
            c, p = codes[pg, :, at], param[pg, :, at].double()
            c = torch.stack([c & 15, c >> 4], -1).flatten(-2).double() - p[..., 1:2] - z
            e = 2.0 ** torch.floor(torch.log2((p[..., 0] * c.abs().amax(-1)).amax()))
            both.append(fp16(c * fp16(p[..., 0:1] * f / e)) * e)
        for h in range(heads):
            k, v = both[0][:, h // group], both[1][:, h // group]
            for i in range(n):
                m = length - n + i + 1
                t = starts[s] + i
                sc = scale * k[:m] @ q[t, h].double()
                w = torch.exp(sc - sc.max())
                out[t, h] = fp16(w * 64) @ v[:m] / (64 * w.sum())
                lse[t, h] = sc.max() + torch.log(w.sum())
    return out.to(torch.bfloat16), lse.float()


CASES = [([257], [257]), ([700, 90], [130, 90]), ([3000], [40]), ([513, 300], [70, 100])]


def case(i):
    lens, news = CASES[i]
    rng, g = np.random.RandomState(i), torch.Generator().manual_seed(i)
    heads, group, page, d = 1, 2, 64, 128
    pages = sum(-(-n // page) for n in lens)
    layer = []
    for _ in range(2):
        layer.append(torch.randint(0, 256, (pages, heads, page, d // 2), generator=g, dtype=torch.uint8))
        p = torch.empty(pages, heads, page, 2).uniform_(0.1, 0.4, generator=g)
        p[..., 1].random_(3, 13, generator=g)
        layer.append(p)
    order, table, at = rng.permutation(pages), np.zeros((len(lens), max(-(-n // page) for n in lens)), np.int32), 0
    for s, n in enumerate(lens):
        used = -(-n // page)
        table[s, :used] = order[at:at + used]
        at += used
    starts = [0] + np.cumsum(news).tolist()
    q = torch.randn(starts[-1], heads * group, d, generator=g).to(torch.bfloat16)
    args = (tuple(layer), table, lens, starts, q, d ** -0.5)
    return args, kv_bounds.expect(*args, True)


@pytest.mark.parametrize("i", range(len(CASES)))
def test_roundings_pass_and_mistakes_do_not(i):
    args, want = case(i)
    good, lse = emulate(*args)
    kv_bounds.check(good, lse, want)
    for wrong in (torch.zeros_like(good), good * 1.02, good.roll(1, 0), good.roll(1, 2)):
        with pytest.raises(AssertionError):
            kv_bounds.check(wrong, lse, want)
    with pytest.raises(AssertionError):
        kv_bounds.check(good, lse + 0.01, want)
    for mistake in (dict(key_scale=1.02), dict(value_scale=1.02), dict(value_zero=0.5)):
        with pytest.raises(AssertionError):
            kv_bounds.check(*emulate(*args, **mistake), want)
    one = good.clone()
    one[args[3][-1] // 2, 0] = 0                             # a single row
    with pytest.raises(AssertionError):
        kv_bounds.check(one, lse, want)
