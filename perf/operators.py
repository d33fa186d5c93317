"""The 4-bit key/value cache: attention over it, appending to it and reading it back, and its pages.

A cache holds keys and values the way the quantizer of this library stores a row: asymmetric 4-bit codes with a
float32 scale and an integer-valued float32 zero-point for each token and head,

    alpha = (max x - min x) / 15,  zero = -round(min x / alpha),  code = clamp(round(x / alpha) + zero, 0, 15),

where x / alpha is x times the float32 reciprocal of alpha, as qllm_quantize_rows takes it.  It is paged:
k_codes, v_codes uint8 [layers][pages][kv_heads][page][head_dim / 2] (channel 2i in the low nibble of byte i),
k_param, v_param float32 [layers][pages][kv_heads][page][2] (scale, zero).  table[s][j] is the page of positions
j*page .. j*page + page - 1 of sequence s, seq_lens[s] its length, and rows q_start[s] .. q_start[s+1] - 1 of a packed
batch are its newest tokens.

Each case is one call, or the few calls that a program makes together.  `run` computes it from elementary torch
operations, or with this package's operators where `own` is true; `exact` says what comes out, from the definitions in
64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    att = dict(op="attention", head_dim=128, causal=True)
    return [
        # one request at the start of a chat, 32 heads of 128 (the 4096-channel shapes of bench.py): latency counts
        dict(att, name="attention_first_token", seqs=1, q_heads=32, kv_heads=32, page=16, longest=517, new=1, mix="same", dtype="bf16"),
        # a serving step: 32 sequences of very different lengths, 64 query heads on 8 key heads (the 10240-column QKV)
        dict(att, name="attention_decode_ragged", seqs=32, q_heads=64, kv_heads=8, page=64, longest=9001, new=1, mix="ragged", dtype="bf16"),
        # one sequence with a long context: the work has to be split along it
        dict(att, name="attention_decode_long", seqs=1, q_heads=64, kv_heads=8, page=64, longest=131071, new=1, mix="same", dtype="bf16"),
        # a few drafted tokens checked at once, float32 activations, 40 heads (the 5120-channel shapes)
        dict(att, name="attention_verify_f32", seqs=6, q_heads=40, kv_heads=40, page=32, longest=1999, new=5, mix="ragged", dtype="f32"),
        # a prompt of 2048 tokens, the token count of bench.py's default workload
        dict(att, name="attention_prompt", seqs=1, q_heads=32, kv_heads=32, page=64, longest=2048, new=2048, mix="same", dtype="bf16"),
        # prompts taken in chunks: 1024 new tokens behind up to 8191 cached ones, grouped heads, odd lengths
        dict(att, name="attention_chunk_grouped", seqs=2, q_heads=64, kv_heads=8, page=64, longest=8191, new=1024, mix="ragged", dtype="bf16"),
        # the keys and values of a decode step's tokens are stored, and read back as values
        dict(op="append", name="append_step", seqs=16, kv_heads=8, head_dim=128, page=64, longest=4001, new=1, mix="ragged", dtype="bf16"),
        # those of a batch of prompts
        dict(op="append", name="append_prompts", seqs=5, kv_heads=32, head_dim=128, page=32, longest=4095, new=4095, mix="ragged", dtype="bf16"),
        # a prefix is copied page by page, all layers at once
        dict(op="copy", name="copy_prefix", seqs=4, layers=32, kv_heads=32, head_dim=128, page=16, longest=300, beams=1),
        # a beam step: every parent gets three children, whose last pages are copies
        dict(op="fork", name="fork_beams", seqs=4, layers=32, kv_heads=32, head_dim=128, page=16, longest=611, beams=3),
        # every second sequence has ended: its pages are freed and the others' pages close up; small and large
        dict(op="compact", name="compact_small", seqs=8, layers=2, kv_heads=8, head_dim=64, page=16, longest=200, beams=1),
        dict(op="compact", name="compact_large", seqs=40, layers=40, kv_heads=8, head_dim=128, page=64, longest=2900, beams=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "verify", "prompt", "prompt", "append", "append", "copy", "fork", "compact"])
    head_dim = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind in ("decode", "verify", "prompt"):
        kv_heads, group = rng.choice([(1, 8), (2, 5), (4, 7), (8, 8), (8, 4), (32, 1), (40, 1)])
        case = dict(op="attention", q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page=page,
                    causal=rng.random() < 0.8, mix=rng.choice(["same", "ragged", "mixed"]))
        if kind == "decode":
            case.update(seqs=_log(rng, 1, 40), longest=_log(rng, 1, 9000), new=1, dtype=rng.choice(["bf16", "bf16", "f32"]))
        elif kind == "verify":
            case.update(seqs=_log(rng, 1, 24), longest=_log(rng, 16, 6000), new=rng.randint(2, 12), dtype=rng.choice(["bf16", "f32"]))
        else:
            new = _log(rng, 33, 1500)
            case.update(seqs=rng.randint(1, 2), longest=new + _log(rng, 1, 4000), new=new, dtype="bf16")
        return case
    if kind == "append":
        new = _log(rng, 1, 4000)
        return dict(op="append", seqs=rng.randint(1, 5) if new > 64 else _log(rng, 1, 64), kv_heads=rng.choice([1, 4, 8, 32]), head_dim=head_dim,
                    page=page, longest=new + _log(rng, 1, 2000), new=new, mix=rng.choice(["same", "ragged", "mixed"]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    return dict(op=kind, seqs=rng.randint(2, 12), layers=_log(rng, 1, 40), kv_heads=rng.choice([1, 8, 16]), head_dim=head_dim, page=page,
                longest=_log(rng, 20, 2000), beams=rng.randint(1, 4) if kind == "fork" else 1)


# ------------------------------------------------------------------------------------------------ sizes of a case
def _sizes(case):
    """(lengths, new tokens) of the sequences: from the case alone."""
    rng = random.Random(case["seqs"] * 1000003 + case["longest"] * 101 + case.get("new", 0))
    n, top, new = case["seqs"], case["longest"], case.get("new", 0)
    mix = case.get("mix", "ragged")
    lens, news = [], []
    for s in range(n):
        length = top if s == 0 or mix == "same" else max(1, int(top ** rng.uniform(0.55, 1.0)))
        k = new if s == 0 or mix == "same" or new <= 1 else rng.randint(1, new) if mix == "ragged" else 1 if s % 2 else new
        lens.append(length)
        news.append(min(k, length))
    return lens, news


def _starts(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int64)


def _pages(lens, page):
    return [-(-x // page) for x in lens]


def _page_state(case):
    """Sizes of a page case: lengths, rows of the table, its width, pages of the cache."""
    lens, _ = _sizes(case)
    used = _pages(lens, case["page"])
    rows = case["seqs"] * (1 + (case["beams"] if case["op"] == "fork" else 0))
    total = sum(used) + (case["seqs"] * case["beams"] if case["op"] == "fork" else sum(used) if case["op"] == "copy" else 0)
    return lens, used, rows, max(used) + 1, total + total // 4 + 3


def work(case):
    d, page = case["head_dim"], case["page"]
    token = case["kv_heads"] * 2 * (d // 2 + 8)                       # a token's keys and values in one layer of the cache
    if case["op"] == "attention":
        lens, news = _sizes(case)
        pairs = sum(n * length - (n * (n - 1) // 2 if case["causal"] else 0) for length, n in zip(lens, news))
        size = 2 if case["dtype"] == "bf16" else 4
        ints = 4 * sum(_pages(lens, page)) + 8 * len(lens)
        return {"bytes": sum(lens) * token + 2 * sum(news) * case["q_heads"] * d * size + ints, "flops": 4 * d * case["q_heads"] * pairs}
    if case["op"] == "append":
        lens, news = _sizes(case)
        values = 2 * sum(news) * case["kv_heads"] * d * (2 if case["dtype"] == "bf16" else 4)
        return {"bytes": 2 * values + 2 * sum(news) * token, "flops": 8 * sum(news) * 2 * case["kv_heads"] * d}
    lens, used, rows, width, pages = _page_state(case)
    if case["op"] == "copy":
        moved, read = sum(used), sum(min(x, page) for x in lens)
    elif case["op"] == "fork":
        moved = sum(case["beams"] for x in lens if x % page)
        read = case["beams"] * sum(min(x, page) for x in lens)
    else:
        table, refs = _layout(case)
        keep = np.zeros(pages, bool)
        for s in range(1, case["seqs"], 2):
            keep[table[s, :used[s]]] = True
        moved = int(keep[keep.sum():].sum())
        read = sum(min(lens[s], page) for s in range(1, case["seqs"], 2))
    values = read * case["kv_heads"] * d * 2 * 2
    return {"bytes": 2 * moved * page * token * case["layers"] + read * token + values + 8 * (pages + rows * width), "flops": 0}


def _layout(case):
    """A page case's table and reference counts: the pages of a cache that has been in use for a while lie anywhere."""
    lens, used, rows, width, pages = _page_state(case)
    order = np.random.RandomState(case["seqs"] * 7 + case["longest"]).permutation(pages)
    table, refs, at = np.full((rows, width), -1, np.int32), np.zeros(pages, np.int32), 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        refs[order[at:at + n]] = 1
        at += n
    return table, refs


# ------------------------------------------------------------------------------------------------ the cache in torch
def _quantize(x):
    """float32 or bf16 [..., d] -> (codes uint8 [..., d/2], param float32 [..., 2])."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    alpha = (hi - lo) / torch.full_like(lo, 15.0)                     # by a tensor: a number would be multiplied by its reciprocal
    alpha = torch.where(hi > lo, alpha, torch.where(lo != 0, lo.abs(), torch.ones_like(lo)))
    inv = 1.0 / alpha
    zero = -torch.round(lo * inv)
    q = (torch.round(x.double() * inv.double()) + zero.double()).clamp(0, 15).to(torch.uint8)
    return q[..., 0::2] | (q[..., 1::2] << 4), torch.cat([alpha, zero], -1)


def _values(codes, param):
    """(codes uint8 [..., d/2], param float32 [..., 2]) -> float32 [..., d]."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    return (q - param[..., 1:2]) * param[..., 0:1]


def _slots(state):
    """Page and place in it of every packed row's token."""
    pos = state["seq_lens"][state["row_seq"]] - state["row_new"] + state["row_at"]
    return state["table"][state["row_seq"], pos // state["page"]].long(), pos % state["page"]


def _plain_read(state, layer):
    pages, at = _slots(state)
    c = state["cache"]
    k = _values(c[0][layer][pages, :, at], c[1][layer][pages, :, at])
    v = _values(c[2][layer][pages, :, at], c[3][layer][pages, :, at])
    return k.to(state["dtype"]), v.to(state["dtype"])


def _plain_attention(state):
    c, layer, page, q = state["cache"], state["layer"], state["page"], state["q"]
    seqs, width = state["table"].shape
    rows, q_heads, d = q.shape
    kv_heads = c[0].shape[2]
    most, new = width * page, state["most_new"]
    at = state["table"].clamp(min=0).long()
    keys = _values(c[0][layer][at], c[1][layer][at]).transpose(2, 3).reshape(seqs, most, kv_heads, d).transpose(1, 2)
    vals = _values(c[2][layer][at], c[3][layer][at]).transpose(2, 3).reshape(seqs, most, kv_heads, d).transpose(1, 2)
    group = q_heads // kv_heads
    padded = torch.zeros(seqs, new, q_heads, d, device=q.device)
    padded[state["row_seq"], state["row_at"]] = q.float()
    padded = padded.reshape(seqs, new, kv_heads, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, new * group, d)
    s = torch.matmul(padded, keys.transpose(2, 3)) * state["scale"]
    j = torch.arange(most, device=q.device)
    lens, n = state["seq_lens"].long(), state["seq_new"].long()
    if state["causal"]:
        sees = (lens - n)[:, None] + torch.arange(new, device=q.device)[None] + 1
    else:
        sees = lens[:, None].expand(seqs, new)
    hidden = j >= sees.repeat_interleave(group, 1)[:, None, :, None]
    s = s.masked_fill(hidden, float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p, vals) / p.sum(-1, keepdim=True)
    o = o.reshape(seqs, kv_heads, new, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, new, q_heads, d)
    return o[state["row_seq"], state["row_at"]].to(q.dtype)


# ------------------------------------------------------------------------------------------------ inputs
def _packed(case, lens, news):
    """A packed batch's integers on the device."""
    start = _starts(news)
    row_seq = np.repeat(np.arange(len(news)), news)
    dev = lambda a, t: torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(t)  # noqa: E731
    return dict(seq_lens=dev(lens, torch.int32), q_start=dev(start, torch.int32), seq_new=dev(news, torch.int32),
                row_seq=dev(row_seq, torch.int64), row_new=dev(np.asarray(news)[row_seq], torch.int64),
                row_at=dev(np.arange(start[-1]) - start[row_seq], torch.int64), rows=int(start[-1]), most_new=max(news),
                page=case["page"])


def _heads(gen, tokens, heads, d, loud):
    """Rows of normal values in which some channels are several times larger, as keys have them."""
    x = torch.randn(tokens, heads, d, generator=gen, device=DEV)
    if loud:
        x[:, :, torch.randint(0, d, (max(1, d // 32),), generator=gen, device=DEV)] *= 4.0
    return x


def _empty_cache(layers, pages, case):
    shape = (layers, pages, case["kv_heads"], case["page"])
    make = lambda last, t: torch.empty(*shape, last, dtype=t, device=DEV)  # noqa: E731
    return (make(case["head_dim"] // 2, torch.uint8), make(2, torch.float32), make(case["head_dim"] // 2, torch.uint8), make(2, torch.float32))


def _random_cache(gen, layers, pages, case):
    c = _empty_cache(layers, pages, case)
    for i in (0, 2):
        c[i].random_(0, 256, generator=gen)
        c[i + 1].uniform_(0.05, 0.5, generator=gen)
        c[i + 1][..., 1].random_(3, 13, generator=gen)
    return c


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["op"] in ("attention", "append"):
        state = _prepare_tokens(case, gen)
    else:
        state = _prepare_pages(case, gen)
    state["op"] = case["op"]
    if own:  # the handles that a program makes once, beside its tensors
        from paper_2310_08041_b200 import binding as B
        state["B"] = B
        state["kv"] = B.KvCache(*state["cache"])
        if case["op"] in ("attention", "append"):
            state["batch"] = B.KvBatch(state["table"], state["seq_lens"], state["q_start"], state["rows"], state["most_new"])
        else:
            state["pool"] = B.KvPool(state["refs"], state["table"], state["seq_lens"])
            r = state["reader"]
            r["batch"] = B.KvBatch(r["table"], r["seq_lens"], r["q_start"], r["rows"], r["most_new"])
        if case["op"] == "attention":
            n = B.qllm_kv_attention_workspace(state["kv"], case["q_heads"], state["q"], state["batch"])
            state["workspace"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    return state


def _prepare_tokens(case, gen):
    lens, news = _sizes(case)
    used, page, d = _pages(lens, case["page"]), case["page"], case["head_dim"]
    pages = sum(used) + 2
    layers, layer = (1, 0) if case["op"] == "attention" else (2, 1)
    state = _packed(case, lens, news)
    dtype = DTYPES[case["dtype"]]
    table = torch.full((len(lens), max(used)), -1, dtype=torch.int32)
    order, at = torch.randperm(pages, generator=gen, device=DEV).cpu().to(torch.int32), 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        at += n
    state.update(table=table.to(DEV), cache=_random_cache(gen, layers, pages, case), layer=layer, dtype=dtype)
    if case["op"] == "append":
        n = state["rows"]
        qkv = torch.cat([_heads(gen, n, case["kv_heads"], d, True), _heads(gen, n, case["kv_heads"], d, False)], 1).to(dtype)
        state.update(k=qkv[:, :case["kv_heads"]], v=qkv[:, case["kv_heads"]:])   # the two ends of one projection's rows
        state.update(k_out=torch.empty(n, case["kv_heads"], d, dtype=dtype, device=DEV), v_out=torch.empty(n, case["kv_heads"], d, dtype=dtype, device=DEV))
        return state
    for i, loud in ((0, True), (2, False)):                           # every page holds quantized rows, page by page
        for p in range(0, pages, 512):
            n = min(512, pages - p)
            codes, param = _quantize(_heads(gen, n * case["kv_heads"], page, d, loud).reshape(n, case["kv_heads"], page, d))
            state["cache"][i][0, p:p + n] = codes
            state["cache"][i + 1][0, p:p + n] = param
    rows, h = state["rows"], case["q_heads"]
    qkv = _heads(gen, rows, h + 2 * case["kv_heads"], d, False).to(dtype)
    state.update(q=qkv[:, :h], out=torch.empty(rows, h, d, dtype=dtype, device=DEV), scale=d ** -0.5, causal=case["causal"])
    return state


def _prepare_pages(case, gen):
    lens, used, rows, width, pages = _page_state(case)
    table, refs = _layout(case)
    n = case["seqs"]
    state = dict(cache=_random_cache(gen, case["layers"], pages, case), page=case["page"], layer=case["layers"] - 1, dtype=torch.bfloat16)
    # one buffer of integers: counts, table, lengths; `saved` puts it back before every pass
    ints = torch.zeros(pages + rows * width + rows, dtype=torch.int32)
    ints[:pages] = torch.from_numpy(refs)
    ints[pages:pages + rows * width] = torch.from_numpy(table).reshape(-1)
    ints[pages + rows * width:pages + rows * width + n] = torch.tensor(lens, dtype=torch.int32)
    state["saved"] = ints.to(DEV)
    state["ints"] = state["saved"].clone()
    state["refs"] = state["ints"][:pages]
    state["table"] = state["ints"][pages:pages + rows * width].view(rows, width)
    state["seq_lens"] = state["ints"][pages + rows * width:]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["op"] == "copy":
        spare = np.nonzero(refs == 0)[0][:sum(used)]
        taken = np.concatenate([table[s, :u] for s, u in enumerate(used)])
        perm = torch.randperm(len(taken), generator=gen, device=DEV).cpu().numpy()
        state.update(src=dev(taken), dst=dev(spare[perm[:len(taken)]]))
        other = np.full((n, width), -1, np.int32)
        at = 0
        for s, u in enumerate(used):
            other[s, :u] = spare[perm[at:at + u]]
            at += u
        look, look_lens, look_table = list(range(n)), lens, dev(other)
    elif case["op"] == "fork":
        parents = [s for s in range(n) for _ in range(case["beams"])]
        state.update(parent=dev(parents), child=dev(list(range(n, n + len(parents)))))
        look, look_lens, look_table = list(range(n, n + len(parents))), [lens[s] for s in parents], None
    else:
        state.update(ended=dev(list(range(0, n, 2))), remap=torch.empty(pages, dtype=torch.int32, device=DEV))
        look = list(range(1, n, 2))
        look_lens, look_table = [lens[s] for s in look], None
    # the last tokens of the sequences that came out of it are read back
    reader = _packed(case, look_lens, [min(x, case["page"]) for x in look_lens])
    reader.update(cache=state["cache"], dtype=torch.bfloat16, layer=state["layer"])
    if case["op"] == "copy":
        reader["table"] = look_table
    elif case["op"] == "fork":
        reader["table"], reader["seq_lens"] = state["table"][n:], state["seq_lens"][n:]
    else:
        reader["look"] = torch.tensor(look, device=DEV)
        reader["table"] = torch.empty(len(look), width, dtype=torch.int32, device=DEV)
    shape = (reader["rows"], case["kv_heads"], case["head_dim"])
    reader.update(k_out=torch.empty(shape, dtype=torch.bfloat16, device=DEV), v_out=torch.empty(shape, dtype=torch.bfloat16, device=DEV))
    state["reader"] = reader
    return state


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    B, op = state["B"], state["op"]
    if op == "attention":
        B.qllm_kv_attention(state["kv"], state["layer"], state["q"], state["out"], state["scale"], state["batch"], state["workspace"], causal=state["causal"])
        return state["out"]
    if op == "append":
        B.qllm_kv_append(state["kv"], state["layer"], state["k"], state["v"], state["batch"])
        B.qllm_kv_read(state["kv"], state["layer"], state["k_out"], state["v_out"], state["batch"])
        return state["k_out"], state["v_out"]
    r = state["reader"]
    state["ints"].copy_(state["saved"])
    if op == "copy":
        B.qllm_kv_pages_copy(state["kv"], state["src"], state["dst"])
    elif op == "fork":
        B.qllm_kv_pages_fork(state["kv"], state["pool"], state["parent"], state["child"])
    else:
        B.qllm_kv_pages_free(state["pool"], state["ended"])
        B.qllm_kv_pages_compact(state["kv"], state["pool"], state["remap"])
        torch.index_select(state["table"], 0, r["look"], out=r["table"])
    B.qllm_kv_read(state["kv"], r["layer"], r["k_out"], r["v_out"], r["batch"])
    return state["refs"], state["table"], state["seq_lens"], r["k_out"], r["v_out"]


def _run_plain(state):
    op = state["op"]
    if op == "attention":
        return _plain_attention(state)
    if op == "append":
        pages, at = _slots(state)
        for i, x in ((0, state["k"]), (2, state["v"])):
            codes, param = _quantize(x)
            state["cache"][i][state["layer"]][pages, :, at] = codes
            state["cache"][i + 1][state["layer"]][pages, :, at] = param
        return _plain_read(state, state["layer"])
    r = state["reader"]
    state["ints"].copy_(state["saved"])
    refs, table, lens = state["refs"], state["table"], state["seq_lens"]
    if op == "copy":
        _plain_copy(state["cache"], state["src"].long(), state["dst"].long())
    elif op == "fork":
        parent, child, page = state["parent"].long(), state["child"].long(), state["page"]
        length = lens[parent].long()
        rest, full = length % page != 0, length // page
        shared = table[parent].clone()
        j = torch.arange(table.shape[1], device=refs.device)
        refs.index_add_(0, shared[j < full[:, None]].long(), torch.ones(1, dtype=torch.int32, device=refs.device).expand(int(full.sum())))
        fresh = torch.nonzero(refs == 0)[:, 0][:int(rest.sum())]
        refs[fresh] = 1
        last = shared[rest, full[rest]].long()
        shared[rest, full[rest]] = fresh.to(torch.int32)
        table[child] = shared
        lens[child] = length.to(torch.int32)
        _plain_copy(state["cache"], last, fresh)
    else:
        ended = state["ended"].long()
        gone = table[ended]
        gone = gone[gone >= 0].long()
        refs.index_add_(0, gone, torch.full((1,), -1, dtype=torch.int32, device=refs.device).expand(gone.numel()))
        table[ended] = -1
        lens[ended] = 0
        live = refs > 0
        index = torch.arange(refs.numel(), device=refs.device)
        count = live.sum()
        src, dst = torch.nonzero(live & (index >= count))[:, 0], torch.nonzero(~live & (index < count))[:, 0]
        _plain_copy(state["cache"], src, dst)
        to = index.clone()
        to[src] = dst
        refs[dst] = refs[src]
        refs[src] = 0
        table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
        torch.index_select(table, 0, r["look"], out=r["table"])
    return (refs, table, lens) + _plain_read(r, r["layer"])


def _plain_copy(cache, src, dst):
    for t in cache:
        t[:, dst] = t[:, src]


# ------------------------------------------------------------------------------------------------ what comes out
def exact(case, seed):
    """From the definitions, in 64 bits: one sequence after the other, a token's place found from its position."""
    global own
    kept, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "attention":
        return _exact_attention(case, state)
    if case["op"] == "append":
        return tuple(_exact_values(*_exact_codes(state[x].to(torch.float64).cpu().numpy())) for x in ("k", "v"))
    return _exact_pages(case, state)


def _nibbles(codes):
    """uint8 [..., d/2] -> the codes in channel order, as float64."""
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    out[..., ::2] = codes.remainder(16).double()
    out[..., 1::2] = codes.div(16, rounding_mode="floor").double()
    return out


def _stored(cache, layer, pages, page, count):
    """Keys or values of the first `count` positions that `pages` hold, float64 [count][kv_heads][d]."""
    pos = torch.arange(count, device=DEV)
    where = pages.long()[pos // page]
    codes, param = cache[0][layer][where, :, pos % page], cache[1][layer][where, :, pos % page].double()
    return (_nibbles(codes) - param[..., 1].unsqueeze(-1)) * param[..., 0].unsqueeze(-1)


def _exact_attention(case, state):
    lens, news = _sizes(case)
    start, h, hk, d = _starts(news), case["q_heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty(state["rows"], h, d, dtype=torch.float64, device=DEV)
    for s, (length, n) in enumerate(zip(lens, news)):
        k = _stored(state["cache"][:2], 0, state["table"][s], case["page"], length)
        v = _stored(state["cache"][2:], 0, state["table"][s], case["page"], length)
        q = state["q"][start[s]:start[s + 1]].double()
        for head in range(h):
            a = q[:, head] @ k[:, head // (h // hk)].T / math.sqrt(d)
            if case["causal"]:
                a = a + torch.full((n, length), -torch.inf, dtype=torch.float64, device=DEV).triu(length - n + 1)
            out[start[s]:start[s + 1], head] = torch.softmax(a, 1) @ v[:, head // (h // hk)]
    return out


def _exact_codes(x):
    """Rows [..., d] (float64 numpy) -> codes, scale, zero: the quantizer with its float32 parameters."""
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    alpha = ((hi.astype(np.float32) - lo.astype(np.float32)) / np.float32(15)).astype(np.float32)
    alpha = np.where(hi > lo, alpha, np.where(lo != 0, np.abs(lo), 1.0)).astype(np.float32)
    inv = (np.float32(1) / alpha).astype(np.float32)
    zero = -np.rint((lo.astype(np.float32) * inv).astype(np.float32)).astype(np.float64)
    return np.clip(np.rint(x * inv.astype(np.float64)) + zero, 0, 15), alpha.astype(np.float64), zero


def _exact_values(codes, alpha, zero):
    return torch.from_numpy((codes - zero) * alpha)


def _exact_pages(case, state):
    lens, used, rows, width, pages = _page_state(case)
    table, refs = _layout(case)
    lens = lens + [0] * (rows - len(lens))
    n = case["seqs"]
    source = {}                                                       # page -> the page whose contents it has now
    if case["op"] == "copy":
        looked = list(range(n))
    elif case["op"] == "fork":
        looked = list(range(n, rows))
        spare = [int(p) for p in np.nonzero(refs == 0)[0]]
        for i, c in enumerate(looked):
            p = i // case["beams"]
            lens[c] = lens[p]
            for j in range(used[p]):
                if (j + 1) * case["page"] <= lens[p]:
                    table[c, j] = table[p, j]
                    refs[table[p, j]] += 1
                else:
                    table[c, j] = spare.pop(0)
                    refs[table[c, j]] = 1
                    source[int(table[c, j])] = int(table[p, j])
    else:
        looked = list(range(1, n, 2))
        for s in range(0, n, 2):
            refs[table[s, :used[s]]] -= 1
            table[s], lens[s] = -1, 0
        count = int((refs > 0).sum())
        holes = [p for p in range(count) if refs[p] == 0]
        for p in range(count, pages):
            if refs[p] > 0:
                to = holes.pop(0)
                refs[to], refs[p] = refs[p], 0
                table[table == p] = to
                source[to] = p
    k, v = [], []
    for s in looked:
        row = torch.tensor([source.get(int(p), int(p)) for p in table[s]], device=DEV).clamp(min=0)
        last = min(lens[s], case["page"])
        k.append(_stored(state["cache"][:2], state["layer"], row, case["page"], lens[s])[-last:])
        v.append(_stored(state["cache"][2:], state["layer"], row, case["page"], lens[s])[-last:])
    ints = [torch.tensor(np.ascontiguousarray(x).astype(np.int32)) for x in (refs, table, np.asarray(lens))]
    return ints[0], ints[1], ints[2], torch.cat(k), torch.cat(v)
