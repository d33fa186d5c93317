"""What stands around a quantized projection in a decoder block: the root-mean-square norm in front of it, the low-rank
adapters beside it, and the position rotation between it and the key/value cache.

norm       h = x + residual, y = gamma h / sqrt(mean(h^2) + eps), and y (or the channels that a reassembly map makes of it) in
           4, 6 or 8 bits per token: alpha = (max - min) / (2^bits - 1), zero = -round(min / alpha), code = clamp(round(v / alpha)
           + zero).  The norm's factor r = 1 / sqrt(mean(h^2) + eps) is the same for a token's channels, so codes and zero-point
           are those of u = gamma h, and alpha is r times u's.  The codes are read back as the values they stand for.
adapters   out[m] = base[m] + scale[a] B[a] (A[a] x[m]) for the rows m of every sequence of a packed batch, a the sequence's
           adapter (-1: none); A[a] is rank[a] x K, B[a] is N x rank[a], bfloat16.
rotate     query and key channels (i, j) of a pair p are turned by their token's angle, (a cos - b sin, b cos + a sin); pairs are
           (p, p + rot_dim / 2) or (2p, 2p + 1).  Keys and values go into the paged 4-bit cache and are read back.

Each case is one call, or the two that a program makes together.  `run` computes it from elementary torch operations, or with
this package's operators where `own` is true; `exact` says what comes out, from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    norm = dict(op="norm", residual=True, y=False, map=False, dtype="bf16")
    ad = dict(op="adapters", dtype="bf16", mix="same")
    rot = dict(op="rotate", head_dim=128, rot_dim=128, interleaved=False, dtype="bf16")
    return [
        # one token of a chat: latency counts.  4096 channels, 4-bit activations
        dict(norm, name="norm_token", tokens=1, channels=4096, bits=4),
        # a decode step of 61 sequences in front of a reassembled layer, 5120 channels
        dict(norm, name="norm_map_step", tokens=61, channels=5120, bits=4, map=True),
        # a prompt of 2048 tokens in 8 bits, whose normalised rows the adapters beside the projection read too
        dict(norm, name="norm_prompt_y", tokens=2048, channels=8192, bits=8, y=True),
        # a batch of prompts in front of a reassembled layer of 4096 channels
        dict(norm, name="norm_map_prompts", tokens=6011, channels=4096, bits=8, map=True),
        # one token with one adapter beside a 4096 -> 12288 projection: latency counts
        dict(ad, name="adapters_token", seqs=1, new=1, slots=4, max_rank=16, k=4096, n=12288),
        # a serving step: 96 requests on 24 adapters of ranks up to 64, beside an 8192 -> 10240 projection
        dict(ad, name="adapters_step", seqs=96, new=1, slots=24, max_rank=64, k=8192, n=10240),
        # drafted tokens of a few requests, float32 activations
        dict(ad, name="adapters_verify_f32", seqs=7, new=5, slots=5, max_rank=32, k=5120, n=5120, dtype="f32", mix="ragged"),
        # prompts of five requests and the single tokens of others in one batch
        dict(ad, name="adapters_prompts", seqs=12, new=1500, slots=8, max_rank=32, k=8192, n=8192, mix="mixed"),
        # a decode step's tokens, 64 query heads on 8 key heads
        dict(rot, name="rotate_step", seqs=32, q_heads=64, kv_heads=8, page=64, longest=9001, new=1, mix="ragged"),
        # one token of a chat
        dict(rot, name="rotate_token", seqs=1, q_heads=32, kv_heads=32, page=16, longest=517, new=1, mix="same"),
        # float32 drafted tokens, neighbouring channels as pairs, a quarter of the channels without rotation
        dict(rot, name="rotate_verify_f32", seqs=6, q_heads=40, kv_heads=40, page=32, longest=1999, new=5, mix="ragged", dtype="f32", rot_dim=96,
             interleaved=True),
        # a batch of prompts, 32 heads
        dict(rot, name="rotate_prompts", seqs=5, q_heads=32, kv_heads=32, page=32, longest=4095, new=4095, mix="ragged"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "adapters", "rotate"])
    if op == "norm":
        channels, dtype = rng.choice([512, 1000, 2048, 4096, 5120, 6152, 8192]), rng.choice(["bf16", "bf16", "f32"])
        top = (12000000 if dtype == "bf16" else 6000000) // channels
        return dict(op="norm", tokens=_log(rng, 1, top), channels=channels, bits=rng.choice([4, 6, 8]), residual=rng.random() < 0.8,
                    y=rng.random() < 0.4, map=rng.random() < 0.3, dtype=dtype)
    if op == "adapters":
        step = rng.random() < 0.6
        seqs = _log(rng, 1, 128) if step else rng.randint(1, 12)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(op="adapters", seqs=seqs, new=1 if step else _log(rng, 2, 1200 if dtype == "bf16" else 150), slots=rng.randint(1, 24 if step else 8),
                    max_rank=rng.choice([8, 16, 16, 32, 64]), k=rng.choice([1024, 2056, 4096, 5120, 8192]), n=rng.choice([1000, 4096, 5120, 8192, 10240]),
                    dtype=dtype, mix=rng.choice(["same", "ragged", "mixed"]) if seqs < 8 or step else "mixed")
    kv_heads, group = rng.choice([(1, 8), (2, 5), (4, 7), (8, 8), (8, 4), (32, 1), (40, 1)])
    head_dim = rng.choice([64, 128, 128, 256])
    new = _log(rng, 1, 3000) if rng.random() < 0.5 else rng.choice([1, 1, 1, 4])
    return dict(op="rotate", seqs=rng.randint(1, 3) if new > 64 else _log(rng, 1, 64), q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim,
                rot_dim=rng.choice([head_dim, head_dim, head_dim // 2, 48]), interleaved=rng.random() < 0.4, page=rng.choice([16, 32, 64, 128]),
                longest=new + _log(rng, 1, 12000), new=new, mix=rng.choice(["same", "ragged", "mixed"]), dtype=rng.choice(["bf16", "bf16", "f32"]) if new < 500 else "bf16")


# ------------------------------------------------------------------------------------------------ sizes of a case
def _sizes(case):
    """(lengths, new tokens) of the sequences: from the case alone."""
    rng = random.Random(case["seqs"] * 1000003 + case.get("longest", 0) * 101 + case["new"])
    n, new, mix = case["seqs"], case["new"], case["mix"]
    top = case.get("longest", new)
    lens, news = [], []
    for s in range(n):
        length = top if s == 0 or mix == "same" else max(1, int(top ** rng.uniform(0.55, 1.0)))
        k = new if s == 0 or mix == "same" or new <= 1 else rng.randint(1, new) if mix == "ragged" else 1 if s % 2 else new
        if case["op"] == "adapters" and mix == "mixed" and 0 < s:     # as many prompts as a step of chunked prompts takes
            k = rng.randint(1, new) if s < 5 and new > 1 else 1
        lens.append(length)
        news.append(k if case["op"] == "adapters" else min(k, length))
    return lens, news


def _adapters_of(case):
    """(ranks of the slots, adapter of every sequence): from the case alone.  Some sequences have none."""
    rng = random.Random(case["seqs"] * 31 + case["slots"] * 7 + case["max_rank"])
    top = case["max_rank"]
    ranks = [top if a == 0 else rng.choice([top, top, max(8, top // 2), max(8, top // 4), max(1, top - 3)]) for a in range(case["slots"])]
    used = [rng.randrange(case["slots"]) if s == 0 or rng.random() > 0.08 else -1 for s in range(case["seqs"])]
    return ranks, used


def _starts(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int64)


def _map_sizes(case):
    """(channels that are split, merged pairs and triples) of a reassembly map: an eighth of the channels come and go."""
    extra = max(1, case["channels"] // 8)
    return extra


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        m, c = case["tokens"], case["channels"]
        codes = c // 2 if case["bits"] == 4 else c
        values = 2 + case["residual"] + case["y"]                     # x, what is read back, the residual, y
        bytes_ = m * (c * size * (values + 1) + 2 * codes + 12) + 4 * c   # and h
        return {"bytes": bytes_ + (8 * (c + _map_sizes(case)) + 4 * c if case["map"] else 0), "flops": 10 * m * c}
    if case["op"] == "adapters":
        _, news = _sizes(case)
        ranks, used = _adapters_of(case)
        rows, k, n = sum(news), case["k"], case["n"]
        weights = sum(ranks[a] for a in set(used) if a >= 0) * (k + n) * 2
        with_one = sum(x for x, a in zip(news, used) if a >= 0)
        return {"bytes": weights + with_one * k * size + 2 * rows * n * size + 8 * len(news),
                "flops": sum(2 * x * ranks[a] * (k + n) for x, a in zip(news, used) if a >= 0)}
    lens, news = _sizes(case)
    d, rows, heads = case["head_dim"], sum(news), case["kv_heads"]
    token = 2 * heads * (d // 2 + 8)
    q, kv = rows * case["q_heads"] * d * size, 2 * rows * heads * d * size
    return {"bytes": 2 * q + 2 * kv + 2 * rows * token + rows * case["rot_dim"] * 4 + 8 * len(lens), "flops": rows * (3 * d * (case["q_heads"] + heads) + 16 * d * heads)}


# ------------------------------------------------------------------------------------------------ plain forms
def _codes(u, bits):
    """float32 rows [..., d] -> codes (float64), scale, zero (float32 [..., 1]) in the quantizer's float32 arithmetic: x / alpha is x
    times the float32 reciprocal of alpha, rounded once."""
    lo, hi = u.amin(-1, keepdim=True), u.amax(-1, keepdim=True)
    top = float(2 ** bits - 1)
    alpha = (hi - lo) / torch.full_like(lo, top)                      # by a tensor: a number would be multiplied by its reciprocal
    alpha = torch.where(hi > lo, alpha, torch.where(lo != 0, lo.abs(), torch.ones_like(lo)))
    inv = 1.0 / alpha
    zero = -torch.round(lo * inv)
    q = (torch.round(u.double() * inv.double()) + zero.double()).clamp(0, top)
    return q, alpha, zero


def _plain_norm(state):
    x, bits = state["x"], state["bits"]
    h = x.float() + state["residual"].float() if state["residual"] is not None else x.float()
    r = torch.rsqrt((h.double() * h.double()).mean(-1, keepdim=True) + EPS).float()
    u = h * state["gamma"]
    y = u * r
    v = u
    if state["map"] is not None:                                      # a row's members side by side, in 64 bits: rounded once
        src, coef = state["padded"]
        v = (u.double()[:, src] * coef).sum(-1).float()
    q, alpha, zero = _codes(v, bits)
    alpha = alpha * r
    values = ((q.float() - zero) * alpha).to(x.dtype)
    out = [h.to(x.dtype), values, alpha[:, 0], zero[:, 0], q.sum(-1).to(torch.int32)]
    return out + [y.to(x.dtype)] if state["want_y"] else out


def _plain_adapters(state):
    """Every row against every adapter, all but its own taken out in the middle."""
    slots, top, k = state["A"].shape
    n = state["B"].shape[1]
    row_adapter = state["adapter"].long()[state["row_seq"]]
    live = torch.arange(top, device=DEV)[None] < state["rank"][:, None]
    a = torch.where(live[:, :, None], state["A"].float(), 0.0).reshape(slots * top, k)
    b = torch.where(live[:, None, :], state["B"].float(), 0.0).transpose(1, 2).reshape(slots * top, n)
    inner = (state["x"].float() @ a.T).reshape(-1, slots, top)
    mine = row_adapter[:, None] == torch.arange(slots, device=DEV)[None]
    inner = (inner * (mine * state["scale"][None])[:, :, None]).reshape(-1, slots * top)
    return (state["base"].float() + inner @ b).to(state["x"].dtype)


def _turn(x, cos, sin, rot_dim, interleaved):
    """float32 rows [t][heads][d] turned by cos, sin [t][1][rot_dim / 2]: each product and each sum rounded to float32."""
    part = x[..., :rot_dim]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else part.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot_dim:]], -1)


def _plain_rotate(state):
    pos = state["seq_lens"].long()[state["row_seq"]] - state["row_new"] + state["row_at"]
    cs = state["angles"][pos]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    turn = lambda x: _turn(x.float(), cos, sin, state["rot_dim"], state["interleaved"])  # noqa: E731
    q = turn(state["q"]).to(state["dtype"])
    page = state["page"]
    pages, at = state["table"][state["row_seq"], pos // page].long(), pos % page
    c, layer = state["cache"], state["layer"]
    for i, x in ((0, turn(state["k"])), (2, state["v"].float())):
        codes, alpha, zero = _codes(x, 4)
        codes = codes.to(torch.uint8)
        c[i][layer][pages, :, at] = codes[..., 0::2] | (codes[..., 1::2] << 4)
        c[i + 1][layer][pages, :, at] = torch.cat([alpha, zero], -1)
    back = []
    for i in (0, 2):
        codes, param = c[i][layer][pages, :, at], c[i + 1][layer][pages, :, at]
        v = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
        back.append(((v - param[..., 1:2]) * param[..., 0:1]).to(state["dtype"]))
    return q, back[0], back[1]


# ------------------------------------------------------------------------------------------------ inputs
def _dev(a, t):
    return torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(t)


def _loud(x, gen, share, factor):
    """Some channels several times larger, as activations have them."""
    c = x.shape[-1]
    x[..., torch.randint(0, c, (max(1, int(c * share)),), generator=gen, device=DEV)] *= factor
    return x


def _make_map(case, seed):
    """A reassembly map with exactly C rows (row starts, sources, coefficients): an eighth of the channels are added by splitting
    channels into two to five equal parts, as many rows saved by averaging two or three quiet ones."""
    c, rng = case["channels"], np.random.RandomState(seed % (2 ** 31))
    left, order, parts = _map_sizes(case), list(rng.permutation(c)), np.ones(c, np.int64)
    merged = {}
    while left > 0:
        t = min(left, int(rng.randint(1, 5)))
        parts[order.pop()] += t
        left -= t
    gone, need = set(), int(parts.sum()) - c
    while need > 0:
        t = min(need, int(rng.randint(1, 3)))
        into, members = int(order.pop()), [int(order.pop()) for _ in range(t)]
        merged[into] = [into] + members
        gone.update(members)
        need -= t
    rows = []
    for i in range(c):
        if i not in gone:
            rows += [[i]] * int(parts[i]) if parts[i] > 1 else [merged.get(i, [i])]
    coef = [1.0 / parts[r[0]] if len(r) == 1 else 1.0 / len(r) for r in rows]
    ptr = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
    most = max(len(r) for r in rows)
    pad_src = np.array([r + [r[0]] * (most - len(r)) for r in rows])
    pad_coef = np.array([[np.float32(f)] * len(r) + [0.0] * (most - len(r)) for r, f in zip(rows, coef)])
    each = np.concatenate([[f] * len(r) for r, f in zip(rows, coef)]).astype(np.float32)
    return ptr, np.concatenate(rows).astype(np.int32), each, pad_src, pad_coef


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"norm": _prepare_norm, "adapters": _prepare_adapters, "rotate": _prepare_rotate}[case["op"]](case, gen, seed)
    state["op"] = case["op"]
    if own:  # the handles that a program makes once, beside its tensors
        from paper_2310_08041_b200 import binding as B
        state["binding"] = B
        if case["op"] == "adapters":
            state["adapters"] = B.Adapters(state["A"], state["B"], state["scale"], state["rank"])
        elif case["op"] == "rotate":
            state["kv"] = B.KvCache(*state["cache"])
            state["batch"] = B.KvBatch(state["table"], state["seq_lens"], state["q_start"], state["rows"], state["most_new"])
            state["rotary"] = B.Rotary(state["angles"], interleaved=state["interleaved"])
    return state


def _prepare_norm(case, gen, seed):
    m, c, dtype = case["tokens"], case["channels"], DTYPES[case["dtype"]]
    x = torch.randn(m, c, generator=gen, device=DEV)
    stream = _loud(2.0 * torch.randn(m, c, generator=gen, device=DEV), gen, 0.01, 20.0)
    state = dict(x=(x if case["residual"] else x + stream).to(dtype), residual=stream.to(dtype) if case["residual"] else None,
                 gamma=1.0 + 0.1 * torch.randn(c, generator=gen, device=DEV), bits=case["bits"], want_y=case["y"], map=None)
    if case["map"]:
        ptr, src, coef, pad_src, pad_coef = _make_map(case, seed)
        state.update(map=(_dev(ptr, torch.int32), _dev(src, torch.int32), _dev(coef, torch.float32)),
                     padded=(_dev(pad_src, torch.int64), _dev(pad_coef, torch.float64)))
    make = lambda *s, t=dtype: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    state.update(h=make(m, c), y=make(m, c) if case["y"] else None, values=make(m, c), codes=make(m, c // 2 if case["bits"] == 4 else c, t=torch.uint8),
                 a_scale=make(m, t=torch.float32), a_zero=make(m, t=torch.float32), a_rowsum=make(m, t=torch.int32))
    return state


def _prepare_adapters(case, gen, seed):
    _, news = _sizes(case)
    ranks, used = _adapters_of(case)
    start, row_seq = _starts(news), np.repeat(np.arange(len(news)), news)
    rows, slots, top, k, n, dtype = int(start[-1]), case["slots"], case["max_rank"], case["k"], case["n"], DTYPES[case["dtype"]]
    rank = _dev(ranks, torch.int32)
    live = (torch.arange(top, device=DEV)[None] < rank[:, None]).float()       # a slot's rows beyond its rank are zero
    a = torch.randn(slots, top, k, generator=gen, device=DEV) * k ** -0.5 * live[:, :, None]
    b = torch.randn(slots, n, top, generator=gen, device=DEV) * 0.2 * live[:, None, :]
    x = _loud(torch.randn(rows, k, generator=gen, device=DEV), gen, 0.005, 10.0).to(dtype)
    base = torch.randn(rows, n, generator=gen, device=DEV).to(dtype)
    return dict(A=a.to(torch.bfloat16), B=b.to(torch.bfloat16), scale=0.25 + torch.rand(slots, generator=gen, device=DEV), rank=rank, x=x, base=base,
                out=torch.empty_like(base), q_start=_dev(start, torch.int32), adapter=_dev(used, torch.int32), row_seq=_dev(row_seq, torch.int64))


def _angles(positions, rot_dim):
    """cos and sin of position / 10000^(2 p / rot_dim), float32 [positions][rot_dim / 2][2], from angles in 64 bits."""
    p = torch.arange(rot_dim // 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-2.0 * p / rot_dim)[None]
    return torch.stack([torch.cos(angle), torch.sin(angle)], -1).float()


def _prepare_rotate(case, gen, seed):
    lens, news = _sizes(case)
    used, d = [-(-x // case["page"]) for x in lens], case["head_dim"]
    pages, start = sum(used) + 2, _starts(news)
    row_seq = np.repeat(np.arange(len(news)), news)
    rows, dtype, q_heads, kv_heads = int(start[-1]), DTYPES[case["dtype"]], case["q_heads"], case["kv_heads"]
    table = torch.full((len(lens), max(used)), -1, dtype=torch.int32)
    order, at = torch.randperm(pages, generator=gen, device=DEV).cpu().to(torch.int32), 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        at += n
    shape = (2, pages, kv_heads, case["page"])
    make = lambda last, t: torch.zeros(*shape, last, dtype=t, device=DEV)  # noqa: E731
    cache = (make(d // 2, torch.uint8), make(2, torch.float32), make(d // 2, torch.uint8), make(2, torch.float32))
    qkv = torch.randn(rows, q_heads + 2 * kv_heads, d, generator=gen, device=DEV)                  # one projection's rows
    qkv[:, :q_heads + kv_heads] = _loud(qkv[:, :q_heads + kv_heads], gen, 0.03, 4.0)
    qkv = qkv.to(dtype)
    empty = lambda heads: torch.empty(rows, heads, d, dtype=dtype, device=DEV)  # noqa: E731
    return dict(q=qkv[:, :q_heads], k=qkv[:, q_heads:q_heads + kv_heads], v=qkv[:, q_heads + kv_heads:], q_out=empty(q_heads), k_out=empty(kv_heads),
                v_out=empty(kv_heads), table=table.to(DEV), cache=cache, layer=1, dtype=dtype, page=case["page"], rot_dim=case["rot_dim"],
                interleaved=case["interleaved"], angles=_angles(max(lens), case["rot_dim"]), seq_lens=_dev(lens, torch.int32),
                q_start=_dev(start, torch.int32), row_seq=_dev(row_seq, torch.int64), row_new=_dev(np.asarray(news)[row_seq], torch.int64),
                row_at=_dev(np.arange(rows) - start[row_seq], torch.int64), rows=rows, most_new=max(news))


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "adapters": _plain_adapters, "rotate": _plain_rotate}[state["op"]](state)


def _run_own(state):
    B, s = state["binding"], state
    if s["op"] == "norm":
        B.qllm_rmsnorm_quant(s["x"], s["gamma"], s["bits"], s["codes"], s["a_scale"], s["a_zero"], s["a_rowsum"], residual=s["residual"], h=s["h"], y=s["y"],
                             map=s["map"], eps=EPS)
        B.qllm_dequantize_rows(s["codes"], s["a_scale"], s["a_zero"], s["bits"], s["values"])
        out = [s["h"], s["values"], s["a_scale"], s["a_zero"], s["a_rowsum"]]
        return out + [s["y"]] if s["want_y"] else out
    if s["op"] == "adapters":
        B.qllm_adapters_add(s["adapters"], s["x"], s["base"], s["out"], s["q_start"], s["adapter"])
        return s["out"]
    B.qllm_kv_rotate_append(s["kv"], s["layer"], s["q"], s["q_out"], s["k"], s["v"], s["rotary"], s["batch"])
    B.qllm_kv_read(s["kv"], s["layer"], s["k_out"], s["v_out"], s["batch"])
    return s["q_out"], s["k_out"], s["v_out"]


# ------------------------------------------------------------------------------------------------ what comes out
def exact(case, seed):
    """From the definitions, in 64 bits.  Which code a value gets is decided in float32, on the values that the definition names:
    those decisions are repeated here in numpy, what the codes stand for and everything else is in 64 bits."""
    global own
    kept, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = kept
    return {"norm": _exact_norm, "adapters": _exact_adapters, "rotate": _exact_rotate}[case["op"]](case, state)


def _decide(x, bits):
    """float32 numpy rows -> (codes, scale, zero) as float64."""
    one, top = np.float32(1), np.float32(2 ** bits - 1)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    alpha = ((hi - lo) / top).astype(np.float32)
    flat = np.where(lo != 0, np.abs(lo), one)
    alpha = np.where(hi > lo, alpha, flat).astype(np.float32)
    inv = one / alpha
    zero = -np.rint(lo * inv).astype(np.float64)
    codes = np.rint(x.astype(np.float64) * inv.astype(np.float64)) + zero
    return np.clip(codes, 0.0, float(top)), alpha.astype(np.float64), zero


def _host(t):
    return t.to(torch.float32).cpu().numpy()


def _exact_norm(case, state):
    x, gamma = _host(state["x"]), _host(state["gamma"])
    add = _host(state["residual"]) if case["residual"] else np.zeros((1, x.shape[1]), np.float32)
    h, stream = x.astype(np.float64) + add, (x + add).astype(np.float32)
    factor = 1.0 / np.sqrt(np.square(h).mean(-1, keepdims=True) + EPS)
    u = (stream * gamma).astype(np.float32)
    if case["map"]:
        ptr, src, coef = (t.cpu().numpy() for t in state["map"])
        u = np.add.reduceat(u[:, src].astype(np.float64) * coef.astype(np.float64), ptr[:-1], axis=1).astype(np.float32)
    codes, alpha, zero = _decide(u, case["bits"])
    out = [h, (codes - zero) * alpha * factor, (alpha * factor)[:, 0], None, None]   # zero-points and sums of codes are the decisions themselves
    if case["y"]:
        out.append(h * gamma.astype(np.float64) * factor)
    return [None if o is None else torch.from_numpy(np.ascontiguousarray(o)) for o in out]


def _exact_adapters(case, state):
    _, news = _sizes(case)
    ranks, used = _adapters_of(case)
    out, at = state["base"].double(), 0
    for n, a in zip(news, used):
        if a >= 0:
            inner = state["x"][at:at + n].double() @ state["A"][a, :ranks[a]].double().T
            out[at:at + n] += float(state["scale"][a]) * (inner @ state["B"][a, :, :ranks[a]].double().T)
        at += n
    return out


def _exact_rotate(case, state):
    lens, news = _sizes(case)
    rot, rows = case["rot_dim"], state["rows"]
    pos = np.concatenate([np.arange(length - n, length) for length, n in zip(lens, news)])
    angles = state["angles"].cpu().numpy()[pos][:, None]
    channel = np.arange(rot)
    pair = channel // 2 if case["interleaved"] else channel % (rot // 2)
    partner = channel ^ 1 if case["interleaved"] else (channel + rot // 2) % rot
    first = channel % 2 == 0 if case["interleaved"] else channel < rot // 2
    sign = np.where(first, -1.0, 1.0)

    def turned(x, kind):
        x, cs = x.astype(kind), angles.astype(kind)
        out = x.copy()
        out[..., :rot] = x[..., :rot] * cs[..., pair, 0] + sign.astype(kind) * (x[..., partner] * cs[..., pair, 1])
        return out

    k, v = _host(state["k"]), _host(state["v"])
    back = []
    for x in (turned(k, np.float32), v):
        codes, alpha, zero = _decide(x, 4)
        back.append(torch.from_numpy((codes - zero) * alpha))
    assert pos.size == rows
    return torch.from_numpy(turned(_host(state["q"]), np.float64)), back[0], back[1]
