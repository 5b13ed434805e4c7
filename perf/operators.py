"""Measured cases of the paged key/value cache and the attention that reads it.

A cache holds the keys and values of many sequences in pages of a fixed number of tokens, as fp16, as bf16 or in 4 bits.
Its operators are timed on the calls a serving program makes of them:

    hypotheses   sequences forked (full pages shared, the last one copied) and handed out in token order;
    move         sequences copied, the originals freed, the pool compacted, the copies forked back and freed;
    token        attention of one new token of each sequence over its cache, with or without a sliding window whose first
                 tokens stay visible;
    prompt       many new tokens of each sequence, written to the cache (rounded to 4 bits, where it holds 4) and attended.

Without `own` the same is computed in elementary torch operations on a pool of plain tensors with a page table.

Four bits: each 32 consecutive values of a head's vector share a scale, the smallest number with 3 significant bits and an
exponent from -14 to 13, at most 10240, that is at least a sixth of the largest magnitude; a value is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, the nearest, halves to the even code; beyond 61440 it saturates.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_CASE = dict(op="token", cache="f16", io="f16", seqs=1, shortest=1, longest=1, new_shortest=0, new_longest=0, q_heads=8, kv_heads=8,
             width=64, page=64, window=0, sinks=0, layers=1, copies=1)


def listed():
    return [
        # a batch of 12 short translations whose hypotheses are forked four ways: one head as wide as the model, nothing but latency
        dict(_CASE, name="hypotheses, short", op="hypotheses", seqs=12, shortest=8, longest=60, q_heads=1, kv_heads=1, width=512, page=32, copies=4),
        # samples of a few long prompts: 2 layers, shared heads
        dict(_CASE, name="hypotheses, long", op="hypotheses", cache="bf16", io="bf16", seqs=6, shortest=700, longest=5000, q_heads=32, width=128,
             layers=2, copies=8),
        # a pool tidied between two bursts: everything copied, freed and moved down, 4 layers of 4-bit pages
        dict(_CASE, name="move, 4 bits", op="move", cache="q4", seqs=24, shortest=300, longest=9000, q_heads=32, width=128, layers=4),
        # one sentence of an interactive session, the eight heads of the ablation student
        dict(_CASE, name="token, one sentence", seqs=1, shortest=41, longest=41),
        # a decoder step of a translation batch: one head as wide as the model, fp32 activations
        dict(_CASE, name="token, translation batch", io="f32", seqs=300, shortest=1, longest=240, q_heads=1, kv_heads=1, width=512, page=32),
        # a serving batch with shared heads, no window
        dict(_CASE, name="token, serving batch", cache="bf16", io="bf16", seqs=64, shortest=500, longest=16000, q_heads=32, width=128),
        # long streams that keep a window and four first tokens
        dict(_CASE, name="token, window of long streams", cache="bf16", io="bf16", seqs=10, shortest=5000, longest=100000, q_heads=32, width=128,
             window=4096, sinks=4),
        # ragged prompts behind cached prefixes, with a window that is shorter than most
        dict(_CASE, name="prompt, window", op="prompt", seqs=13, shortest=1, longest=700, new_shortest=1, new_longest=2900, q_heads=16, width=64,
             window=777, sinks=5),
        # two long prompts
        dict(_CASE, name="prompt, long", op="prompt", cache="bf16", io="bf16", seqs=2, shortest=1, longest=2, new_shortest=8000, new_longest=8400,
             q_heads=32, width=128),
        # 4 bits: a few conversations
        dict(_CASE, name="token, 4 bits, few", cache="q4", seqs=3, shortest=300, longest=2500, q_heads=32, width=128),
        # 4 bits: four times the serving batch in the same memory
        dict(_CASE, name="token, 4 bits, many", cache="q4", io="bf16", seqs=256, shortest=500, longest=16000, q_heads=32, width=128),
        # 4 bits: prompts written to the cache and attended
        dict(_CASE, name="prompt, 4 bits", op="prompt", cache="q4", seqs=9, shortest=1, longest=1500, new_shortest=90, new_longest=3000, q_heads=32,
             width=128, window=2000, sinks=4),
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["hypotheses", "move", "token", "token", "token", "prompt", "prompt"])
    cache = rng.choice(["f16", "bf16", "q4", "q4"])
    kv_heads, group, width = rng.choice([(8, 4, 128), (8, 1, 64), (1, 1, 512), (4, 8, 128), (2, 3, 256), (8, 2, 64), (1, 12, 64)])
    io = {"bf16": ["bf16"], "f16": ["f16", "f32"], "q4": ["f16", "bf16", "f32"]}[cache]
    c = dict(_CASE, op=op, cache=cache, io=rng.choice(io), q_heads=kv_heads * group, kv_heads=kv_heads, width=width, page=rng.choice([32, 64, 128]))
    if rng.random() < 0.5:
        c["window"], c["sinks"] = between(30, 5000), rng.choice([0, 1, 4, 37])
    room = 64 * 4000 * 8 * 128 // (kv_heads * width)  # tokens in all
    if op == "token":
        c["seqs"] = between(1, 300)
        c["shortest"], c["longest"] = between(1, 400), between(400, max(401, min(50000, room // c["seqs"])))
    elif op == "prompt":
        c["seqs"] = between(1, 16)
        c["shortest"], c["longest"] = between(1, 30), between(30, 1500)
        c["new_shortest"] = between(1, 300)
        c["new_longest"] = between(300, max(301, min(6000, 24000 // c["seqs"])))
    else:
        c["seqs"], c["layers"], c["copies"] = between(1, 24), rng.choice([1, 2, 4]), rng.choice([1, 2, 4])
        c["shortest"], c["longest"] = between(1, 200), between(200, max(201, min(9000, room // (c["seqs"] * c["layers"] * c["copies"]))))
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n lengths from lo to hi, even over their logarithm: every seed gives the same amount of work."""
    return [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]


def _lengths(case, seed):
    """(tokens in the cache before the call, new tokens of the call) per sequence"""
    n = case["seqs"]
    past, new = np.array(_spread(case["shortest"], case["longest"], n)), np.zeros(n, dtype=np.int64)
    if case["op"] == "prompt":  # a long prefix does not go with a long prompt
        new = np.array(_spread(case["new_shortest"], case["new_longest"], n))[np.random.default_rng(0).permutation(n)]
    order = np.random.default_rng(seed).permutation(n)
    return past[order], new[order]


def _first(counts):
    return np.concatenate([[0], np.cumsum(counts)])


def _values(case, seed):
    """What both forms are given: lengths, and keys, values [layers][tokens, kv_heads, width] of the cached and the new tokens and queries."""
    past, new = _lengths(case, seed)
    g = torch.Generator("cuda").manual_seed(seed)
    kv, w, t = case["kv_heads"], case["width"], _TYPES[case["io"]]
    # keys have columns that are large in every token, as trained models' keys do
    column = torch.exp(0.5 * torch.randn(kv, w, device="cuda", generator=g))

    def rows(n, scale=1.0):
        return (torch.randn(n, kv, w, device="cuda", generator=g) * scale).to(t)

    d = dict(case=case, past=past, new=new)
    d["old_k"] = [rows(int(past.sum()), column) for _ in range(case["layers"])]
    d["old_v"] = [rows(int(past.sum())) for _ in range(case["layers"])]
    if case["op"] == "prompt":
        d["k"], d["v"] = rows(int(new.sum()), column), rows(int(new.sum()))
    if case["op"] in ("prompt", "token"):
        n = int(new.sum()) if case["op"] == "prompt" else case["seqs"]
        d["q"] = torch.randn(n, case["q_heads"], w, device="cuda", generator=g).to(t)
    return d


def _ints(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _targets(case):
    """Sequence ids that the sequences are copied to, and their sources."""
    n, c = case["seqs"], case["copies"]
    return list(range(n, n + n * c)), [i // c for i in range(n * c)]


def _kept(case):
    """Type in which cached values are handed out."""
    return _TYPES[case["io"]] if case["cache"] == "q4" else _TYPES[case["cache"]]


def prepare(case, seed):
    d = _values(case, seed)
    past, new, n = d["past"], d["new"], case["seqs"]
    total, page = past + new, case["page"]
    longest = int(total.max())
    dst, src = _targets(case)
    many = n + len(dst)
    pages = sum(-(-int(t) // page) for t in total) * (1 + case["copies"]) + len(dst) + 2
    s = dict(case=case, past=past, new=new, longest=longest, dst=dst, most_new=int(new.max()))
    kv, w = case["kv_heads"], case["width"]
    if "q" in d:
        s["q"], s["out"] = d["q"], torch.zeros_like(d["q"])
    if "k" in d:
        s["k"], s["v"] = d["k"], d["v"]
    if case["op"] != "token":
        rows = len(dst) if case["op"] == "hypotheses" else n
        for name in ("out_k", "out_v"):
            s[name] = [torch.zeros((rows, longest, kv, w), dtype=_kept(case), device="cuda") for _ in range(case["layers"])]
    if own:
        import paper_2109_08003_amd as nt
        cache = nt.Cache(case["cache"], n_layers=case["layers"], n_q_heads=case["q_heads"], n_kv_heads=kv, d_head=w, page_tokens=page, n_pages=pages,
                         max_seqs=many, max_len=longest)
        at = _ints(_first(past))
        cache.reserve(n, first=at)
        for l in range(case["layers"]):
            cache.write(d["old_k"][l], d["old_v"][l], n, first=at, max_new=int(past.max()), layer=l)
        if case["op"] == "prompt":
            s["first"] = _ints(_first(new))
            cache.reserve(n, first=s["first"])
        s.update(cache=cache, d_src=_ints(src), d_dst=_ints(dst), d_all=_ints(range(n)))
        return s
    # the plain form's pool: [pages, page, heads, width] and a page table
    shape = (pages, page, kv, w)
    s["pool"] = [_plain_pool(case, shape) for _ in range(2 * case["layers"])]
    g = torch.Generator().manual_seed(seed)
    free = torch.randperm(pages, generator=g).tolist()
    table = torch.zeros((many, -(-longest // page)), dtype=torch.int64)
    for i in range(n):
        for p in range(-(-int(total[i]) // page)):
            table[i, p] = free.pop()
    s["table"], s["free"] = table.cuda(), torch.tensor(free, device="cuda")
    s["lens"] = torch.as_tensor(total, device="cuda")
    s["everything"], s["plain_src"], s["plain_dst"] = (torch.tensor(list(a), device="cuda") for a in (range(n), src, dst))
    s["old_at"] = _slots(s["table"], page, past, np.zeros_like(past))
    for l in range(case["layers"]):
        _plain_put(s["pool"][2 * l], s["old_at"], d["old_k"][l])
        _plain_put(s["pool"][2 * l + 1], s["old_at"], d["old_v"][l])
    if case["op"] == "prompt":
        s["new_at"] = _slots(s["table"], page, new, past)
    return s


# ---- the plain form ----------------------------------------------------------------------------------------------

_SCALES = [m / 4 * 2.0 ** e for e in range(-14, 14) for m in (4, 5, 6, 7) if m / 4 * 2.0 ** e <= 10240]


def _to_four_bits(x):
    """(codes uint8 [..., width], scales float32 [..., width / 32]); compared with the borders in 64 bits"""
    b = x.double().unflatten(-1, (-1, 32))
    table = torch.tensor(_SCALES, dtype=torch.float64, device=x.device)
    s = table[torch.searchsorted(table * 6, b.abs().amax(-1)).clamp_(max=len(_SCALES) - 1)]
    a = b.abs() / s[..., None]
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5).byte()
            + 8 * (b < 0).byte())
    return code.flatten(-2), s.float()


def _from_four_bits(code, s):
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return (v[code.int()].unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _plain_pool(case, shape):
    if case["cache"] == "q4":
        return [torch.zeros(shape, dtype=torch.uint8, device="cuda"), torch.ones(shape[:-1] + (shape[-1] // 32,), device="cuda")]
    return [torch.zeros(shape, dtype=_TYPES[case["cache"]], device="cuda")]


def _slots(table, page, counts, start):
    """Flat places in the pool of the tokens start .. start + counts of every sequence."""
    seq = torch.repeat_interleave(torch.arange(len(counts)), torch.as_tensor(counts)).cuda()
    at = torch.cat([torch.arange(int(c)) + int(b) for c, b in zip(counts, start)]).cuda()
    return table[seq, at // page] * page + at % page


def _plain_put(pool, at, rows):
    parts = _to_four_bits(rows) if len(pool) == 2 else (rows.to(pool[0].dtype),)
    for t, r in zip(pool, parts):
        t.flatten(0, 1)[at] = r


def _plain_get(pool, at):
    """float32 values of the tokens at flat places"""
    rows = [t.flatten(0, 1)[at] for t in pool]
    return _from_four_bits(*rows) if len(rows) == 2 else rows[0].float()


def _plain_read(s, seqs, tables, kept):
    """[rows, longest, heads, width] of the sequences, zero behind their ends"""
    page, longest = s["case"]["page"], s["longest"]
    pos = torch.arange(longest, device="cuda")
    at = tables[seqs][:, pos // page] * page + pos % page
    real = (pos[None, :] < s["lens"][seqs][:, None])[..., None, None]
    return [torch.where(real, _plain_get(pool, at), 0.0).to(kept) for pool in s["pool"]]


def _plain_copy(s, table, lens, src, dst, share):
    """The page table after dst became src: full pages shared or, like the last one, copied to free pages."""
    page = s["case"]["page"]
    table, width = table.clone(), table.shape[1]
    rows, n = table[src], lens[src]
    col = torch.arange(width, device="cuda")[None, :]
    there = col < (n[:, None] + page - 1) // page
    copied = there & ((col >= n[:, None] // page) | (not share))
    fresh = s["free"][:int(there.numel())][copied.flatten().cumsum(0).sub(1).clamp_(min=0, max=len(s["free"]) - 1)].view(rows.shape)
    a, b = rows[copied], fresh[copied]
    for pool in s["pool"]:
        for t in pool:
            t[b] = t[a]
    table[dst] = torch.where(copied, fresh, rows)
    return table


def _softmax_product(scores, seen, v):
    """Weights of the seen keys and their mean of v; rows that see nothing give zero."""
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(scores - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / torch.where(total == 0, 1.0, total)


def _plain_token(s):
    case = s["case"]
    kv, page, window, sinks, L = case["kv_heads"], case["page"], case["window"], case["sinks"], s["longest"]
    n, group = case["seqs"], case["q_heads"] // case["kv_heads"]
    lens = s["lens"][:, None]
    if window and sinks + window < L:  # the sinks, then the window
        pos = torch.cat([torch.arange(sinks, device="cuda").expand(n, -1), lens - window + torch.arange(window, device="cuda")], 1)
        seen = (pos >= 0) & (pos < lens) & ((torch.arange(sinks + window, device="cuda") < sinks) | (pos >= sinks))
        pos = pos.clamp(0, L - 1)
    else:
        pos = torch.arange(L, device="cuda").expand(n, -1)
        seen = pos < lens
    out = torch.empty(s["q"].shape, device="cuda")
    step = max(1, int(3e9 // (pos.shape[1] * kv * case["width"] * 4)))  # so many sequences at a time
    for i in range(0, n, step):
        at = s["table"][:n][i:i + step].gather(1, pos[i:i + step] // page) * page + pos[i:i + step] % page
        k, v = (_plain_get(pool, at).transpose(1, 2) for pool in s["pool"])
        q = s["q"][i:i + step].float().unflatten(1, (kv, group)) * case["width"] ** -0.5
        out[i:i + step] = _softmax_product(torch.matmul(q, k.transpose(2, 3).contiguous()), seen[i:i + step, None, None, :], v).flatten(1, 2)
    return out.to(s["q"].dtype)


def _plain_prompt(s):
    case = s["case"]
    kv, page, window, sinks = case["kv_heads"], case["page"], case["window"], case["sinks"]
    group, w = case["q_heads"] // kv, case["width"]
    _plain_put(s["pool"][0], s["new_at"], s["k"])
    _plain_put(s["pool"][1], s["new_at"], s["v"])
    out, first = torch.empty(s["q"].shape, device="cuda"), _first(s["new"])
    for i in range(case["seqs"]):
        p, m = int(s["past"][i]), int(s["new"][i])
        j = torch.arange(p + m, device="cuda")
        at = s["table"][i][j // page] * page + j % page
        k, v = (_plain_get(pool, at).transpose(0, 1).contiguous() for pool in s["pool"])  # [heads, keys, width]
        q = (s["q"][first[i]:first[i + 1]].float() * w ** -0.5).unflatten(1, (kv, group)).permute(1, 2, 0, 3)
        step = max(1, int(5e8 // (case["q_heads"] * (p + m))))
        for a in range(0, m, step):
            b = min(m, a + step)
            at_q = p + torch.arange(a, b, device="cuda")[:, None]
            seen = j[None, :] <= at_q
            if window:
                seen &= (at_q - j[None, :] < window) | (j[None, :] < sinks)
            o = _softmax_product(torch.matmul(q[:, :, a:b].flatten(1, 2), k.transpose(1, 2).contiguous()).unflatten(1, (group, b - a)), seen, v[:, None])
            out[first[i] + a:first[i] + b] = o.permute(2, 0, 1, 3).flatten(1, 2)
    return out.to(s["q"].dtype)


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s)
    n, op = case["seqs"], case["op"]
    everything, src, dst = s["everything"], s["plain_src"], s["plain_dst"]
    if op == "token":
        return _plain_token(s)
    if op == "prompt":
        return [_plain_prompt(s)] + _plain_read(s, everything, s["table"], _kept(case))
    if op == "hypotheses":
        table = _plain_copy(s, s["table"], s["lens"], src, dst, True)
        lens = torch.zeros(len(table), dtype=s["lens"].dtype, device="cuda")
        lens[:n] = s["lens"]
        lens[dst] = s["lens"][src]
        return _plain_read(dict(s, lens=lens), dst, table, _kept(case))
    # move: copied to free pages, then back to the first ones
    there = _plain_copy(s, s["table"], s["lens"], everything, everything + n, False)
    for pool in s["pool"]:
        for t in pool:
            for i in range(n):
                used = -(-int(s["past"][i]) // case["page"])
                t[s["table"][i, :used]] = t[there[n + i, :used]]
    return _plain_read(s, everything, s["table"], _kept(case))


def _run_own(s):
    case, cache, n = s["case"], s["cache"], s["case"]["seqs"]
    scale = case["width"] ** -0.5
    if case["op"] == "token":
        cache.attend(s["q"], s["out"], n, max_keys=s["longest"], window=case["window"], sinks=case["sinks"], scale=scale)
        return s["out"]
    if case["op"] == "prompt":
        cache.attend(s["q"], s["out"], n, k=s["k"], v=s["v"], first=s["first"], max_new=s["most_new"], max_keys=s["longest"], window=case["window"],
                     sinks=case["sinks"], scale=scale)
        cache.read(s["out_k"][0], s["out_v"][0], n)
        return [s["out"], s["out_k"][0], s["out_v"][0]]
    if case["op"] == "hypotheses":
        cache.fork(s["d_src"], s["d_dst"])
        for l in range(case["layers"]):
            cache.read(s["out_k"][l], s["out_v"][l], len(s["dst"]), seqs=s["d_dst"], layer=l)
    else:
        moved = s["d_dst"][:n]
        cache.copy(s["d_all"], moved)
        cache.truncate(n)
        cache.compact()
        cache.fork(moved, s["d_all"])
        cache.truncate(n, seqs=moved)
        for l in range(case["layers"]):
            cache.read(s["out_k"][l], s["out_v"][l], n, layer=l)
    return [t for l in range(case["layers"]) for t in (s["out_k"][l], s["out_v"][l])]


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def _seen(case, past, new):
    """(keys that some query of a sequence sees, pairs of a query and a key that it sees)"""
    if not case["window"]:
        return past + new, sum(range(past + 1, past + new + 1)) if new else past
    w, s = case["window"], case["sinks"]
    at = np.arange(past, past + new) if new else np.array([past - 1])
    low = np.maximum(at - w + 1, 0)
    pairs = int((at - low + 1 + np.minimum(low, s)).sum())
    return int(at[-1] - low[0] + 1 + min(low[0], s)), pairs


def work(case):
    """Bytes: cached keys and values that are seen, in the cache's form, queries and outputs, what is written and handed out.
    Flops: the two products of every query with the keys it sees."""
    past, new = _lengths(case, 0)
    io, kv, w = _TYPES[case["io"]].itemsize, case["kv_heads"], case["width"]
    token = 2 * kv * (w // 2 + w // 32 if case["cache"] == "q4" else 2 * w)  # bytes of a cached token and layer
    handed = 2 * kv * w * _kept(case).itemsize
    if case["op"] == "hypotheses":
        return {"bytes": float(case["layers"] * past.sum() * (token + case["copies"] * handed)), "flops": 0.0}
    if case["op"] == "move":  # read and written for the copy and for the move, read and handed out
        return {"bytes": float(case["layers"] * past.sum() * (5 * token + handed)), "flops": 0.0}
    counted = [_seen(case, int(p), int(n)) for p, n in zip(past, new)]
    rows = int(new.sum()) if case["op"] == "prompt" else case["seqs"]
    total = sum(k for k, _ in counted) * token + 2 * rows * case["q_heads"] * w * io
    if case["op"] == "prompt":
        total += int(new.sum()) * (2 * kv * w * io + token) + int((past + new).sum()) * handed
    return {"bytes": float(total), "flops": float(4 * case["q_heads"] * w * sum(p for _, p in counted))}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------

def _held(case, rows):
    """What the cache stands for after it has been given these rows."""
    if case["cache"] != "q4":
        return rows.to(_TYPES[case["cache"]]).double()
    x = rows.double()
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = blocks.abs().amax(-1)
    sixth = (top / 6).clamp(min=2.0 ** -14)
    quarter = ((torch.frexp(sixth).exponent.long() - 3 + 1023) << 52).view(torch.float64)  # of the power of two below it: one step
    scale = torch.floor(sixth / quarter) * quarter
    scale = torch.where(scale * 6 < top, scale + quarter, scale).clamp(max=10240.0)
    y = (blocks / scale[..., None]).clamp(-6, 6)
    # steps of 1/2 up to 2, of 1 up to 4, of 2 above; round() takes halves to the even multiple, which is the even code
    size = y.abs()
    step = torch.where(size <= 2, 0.5, torch.where(size <= 4, 1.0, 2.0))
    return (torch.round(y / step) * step * scale[..., None]).reshape(x.shape)


def exact(case, seed):
    d = _values(case, seed)
    past, new, n, w = d["past"], d["new"], case["seqs"], case["width"]
    total, kv, group = past + new, case["kv_heads"], case["q_heads"] // case["kv_heads"]
    at, first, longest = _first(past), _first(new), int((past + new).max())
    if case["op"] in ("hypotheses", "move"):
        order = _targets(case)[1] if case["op"] == "hypotheses" else list(range(n))
        out = []
        for l in range(case["layers"]):
            for rows in (d["old_k"][l], d["old_v"][l]):
                held = _held(case, rows)
                o = torch.zeros((len(order), longest, kv, w), dtype=torch.float64, device="cuda")
                for r, i in enumerate(order):
                    o[r, :past[i]] = held[at[i]:at[i + 1]]
                out.append(o)
        return out
    old_k, old_v = _held(case, d["old_k"][0]), _held(case, d["old_v"][0])
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "prompt":
        new_k, new_v = _held(case, d["k"]), _held(case, d["v"])
        kept = [torch.zeros((n, longest, kv, w), dtype=torch.float64, device="cuda") for _ in range(2)]
    for i in range(n):
        k, v = old_k[at[i]:at[i + 1]], old_v[at[i]:at[i + 1]]
        start, rows = int(past[i]) - 1, slice(i, i + 1)
        if case["op"] == "prompt":
            k, v = torch.cat([k, new_k[first[i]:first[i + 1]]]), torch.cat([v, new_v[first[i]:first[i + 1]]])
            kept[0][i, :total[i]], kept[1][i, :total[i]] = k, v
            start, rows = int(past[i]), slice(int(first[i]), int(first[i + 1]))
        q = d["q"][rows].double()
        where = torch.arange(start, start + len(q), device="cuda")[:, None]
        j = torch.arange(len(k), device="cuda")[None, :]
        hidden = (j > where) | ((where - j >= case["window"]) & (j >= case["sinks"]) if case["window"] else torch.zeros_like(j > where))
        for h in range(case["q_heads"]):
            scores = (q[:, h] @ k[:, h // group].T / math.sqrt(w)).masked_fill_(hidden, -math.inf)
            out[rows, h] = torch.softmax(scores, -1) @ v[:, h // group]
    return [out] + kept if case["op"] == "prompt" else out
