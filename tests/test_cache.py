"""Paged key/value caches (nt_cache_*) on the GPU against a plain model of them in 64 bits.

Reading back is exact: the cache's own rounding is part of its definition.  Tolerances of the attention are derived, not
measured (`allowed`): half a step of the type for each rounding that the documentation names, and sums of n fp32 terms within n
half steps."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

KINDS = ["f16", "bf16", "q4"]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


@pytest.fixture(scope="module")
def nt():
    import paper_2109_08003_amd as nt
    nt.load_library()
    return nt


# ---- the plain model -----------------------------------------------------------------------------------------------

def four_bits(x):
    """What 4-bit pages hold for x float64 [..., width]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    scales = np.array([m / 4 * 2.0 ** e for e in range(-14, 14) for m in (4, 5, 6, 7) if m / 4 * 2.0 ** e <= 10240])
    nan = np.isnan(b).any(-1)
    top = np.where(np.isnan(b), 0, np.abs(b)).max(-1)
    s = scales[np.minimum(np.searchsorted(scales * 6, top), len(scales) - 1)][..., None]
    with np.errstate(invalid="ignore"):
        a = np.abs(b) / s
        code = sum([a > 0.25, a >= 0.75, a > 1.25, a >= 1.75, a > 2.5, a >= 3.5, a > 5], np.zeros(a.shape, int))
    out = np.copysign(np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])[code] * s, b)
    return np.where(nan[..., None], np.nan, out).reshape(x.shape)


def held(torch, kind, x):
    """float64 values of a cache of this kind that was given the tensor x"""
    if kind == "q4":
        return four_bits(x.double().cpu().numpy())
    return x.to({"f16": torch.float16, "bf16": torch.bfloat16}[kind]).double().cpu().numpy()


def attention(q, k, v, first_pos, window, sinks, scale, present=None):
    """q [rows, Hq, w] at positions first_pos .., k, v [keys, Hkv, w]: (out, largest sum of |q k|, most keys seen), float64"""
    rows, hq, w = q.shape
    group = hq // k.shape[1] if k.shape[1] else 1
    out, biggest, most = np.zeros(q.shape), 0.0, 0
    for r in range(rows):
        p = first_pos + r
        j = np.arange(len(k))
        seen = j <= p
        if window:
            seen &= (p - j < window) | (j < sinks)
        if present is not None:
            seen &= present
        if not seen.any():
            continue
        most = max(most, int(seen.sum()))
        for h in range(hq):
            ks, vs = k[seen, h // group], v[seen, h // group]
            s = ks @ q[r, h] * scale
            biggest = max(biggest, float((np.abs(ks) @ np.abs(q[r, h])).max()) * abs(scale))
            e = np.exp(s - s.max())
            out[r, h] = (e / e.sum()) @ vs
    return out, biggest, most


STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def allowed(kind, io, width, biggest, most, top, out, tokens):
    """How far an output may be off.  Scores: the query rounded to the cache's type (to twice its bits for single tokens), the
    sum of `width` products in fp32, and the exponent's argument; a weight is off by twice a score's error, relative,
    twice more after the division, and rounded like the query; the sum over the keys in fp32; the output's own rounding."""
    step = STEP["f16" if kind == "q4" else kind]
    exact_query = io == {"f16": "f16", "bf16": "bf16", "q4": "f16"}[kind]
    fine = 2 * step * step if tokens else step  # the tail is formed against the head: half a step of half a step, and the sum of both
    score = biggest * ((0 if exact_query else fine) + (width + 4) * 2.0 ** -24)
    weight = 4 * score + 2 * fine + most * 2.0 ** -24
    if kind != "bf16":
        weight += most * 2.0 ** -25  # weights below fp16's normal numbers
    return top * weight * 1.01 + STEP[io] * np.abs(out) + 2.0 ** -25 * (io == "f16")


def types(torch):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def ints(torch, a):
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


def rows_of(counts):
    return np.concatenate([[0], np.cumsum(counts)])


def compare(got, want, tol):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all() or not np.isfinite(want).all()
    worst = (np.abs(got - want) - tol).max()
    assert worst <= 0, f"off by {np.abs(got - want).max()}, {worst} too much"


class Filled:
    """A cache and what it ought to hold."""

    def __init__(self, torch, nt, kind, io, lens, heads=(4, 2), width=64, page=64, layers=1, seed=0, spare=8, max_len=None, max_seqs=None, k_scale=1.0):
        self.torch, self.kind, self.io, self.width, self.heads, self.lens = torch, kind, io, width, heads, list(lens)
        self.g = torch.Generator("cuda").manual_seed(seed)
        n = len(lens)
        pages = sum(-(-l // page) for l in lens) + spare
        self.cache = nt.Cache(kind, layers, heads[0], heads[1], width, pages, max_seqs or n + 4, max_len or max(max(lens), 1) + 300, page)
        first = ints(torch, rows_of(lens))
        self.cache.reserve(n, first=first)
        self.k, self.v = [], []
        for l in range(layers):
            k, v = self.random(sum(lens), heads[1], k_scale), self.random(sum(lens), heads[1])
            self.cache.write(k, v, n, first=first, max_new=max(max(lens), 1), layer=l)
            hk, hv = held(torch, kind, k), held(torch, kind, v)
            r = rows_of(lens)
            self.k.append([hk[r[i]:r[i + 1]] for i in range(n)])
            self.v.append([hv[r[i]:r[i + 1]] for i in range(n)])
        self.cache.check()

    def random(self, n, heads, scale=1.0):
        return (self.torch.randn(n, heads, self.width, device="cuda", generator=self.g) * scale).to(types(self.torch)[self.io])

    def expect(self, q, counts, seqs, window, sinks, layer=0, scale=None, tokens=False):
        """(out, tolerance) for queries q (tensor) of `counts` rows per sequence"""
        scale = self.width ** -0.5 if scale is None else scale
        qs, r = q.double().cpu().numpy(), rows_of(counts)
        want, tol = np.zeros(qs.shape), np.zeros(qs.shape)
        for i, s in enumerate(seqs):
            k, v = self.k[layer][s], self.v[layer][s]
            o, biggest, most = attention(qs[r[i]:r[i + 1]], k, v, len(k) - counts[i], window, sinks, scale)
            want[r[i]:r[i + 1]] = o
            top = np.abs(v).max() if len(v) else 0
            tol[r[i]:r[i + 1]] = allowed(self.kind, self.io, self.width, biggest, most, top, o, tokens)
        return want, tol


# ---- single tokens -------------------------------------------------------------------------------------------------

EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 511]


@pytest.mark.parametrize("kind,io", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("q4", "f16"), ("q4", "bf16"), ("q4", "f32")])
@pytest.mark.parametrize("heads,width,page", [((4, 2), 64, 32), ((8, 1), 128, 64), ((9, 1), 64, 128), ((1, 1), 512, 32), ((3, 3), 256, 256)])
def test_tokens(torch, nt, kind, io, heads, width, page):
    f = Filled(torch, nt, kind, io, EDGES, heads, width, page, seed=width + page)
    n = len(EDGES)
    q, out = f.random(n, heads[0]), torch.full((n, heads[0], width), float("nan"), dtype=types(torch)[io], device="cuda")
    for window, sinks in [(0, 0), (1, 0), (40, 0), (64, 3), (33, 70), (100, 200), (600, 5)]:
        out.fill_(float("nan"))
        f.cache.attend(q, out, n, window=window, sinks=sinks)
        want, tol = f.expect(q, [1] * n, range(n), window, sinks, tokens=True)
        compare(out, want, tol)
    f.cache.check()


@pytest.mark.parametrize("kind,io", [("bf16", "bf16"), ("q4", "f32")])
@pytest.mark.parametrize("lens,max_keys", [([20011], 0), ([20011], 1), ([5000, 1, 16000, 0, 333], 16000), ([700] * 60, 700)])
def test_tokens_over_many_keys(torch, nt, kind, io, lens, max_keys):
    """Keys shared by workgroups, also where max_keys says too little."""
    f = Filled(torch, nt, kind, io, lens, (4, 2), 128, 64, seed=3, k_scale=2.0)
    seqs = [i for i, l in enumerate(lens) if l]
    q, out = f.random(len(seqs), 4), torch.empty((len(seqs), 4, 128), dtype=types(torch)[io], device="cuda")
    for window, sinks in [(0, 0), (3000, 4)]:
        for _ in range(3):
            out.fill_(7)
            f.cache.attend(q, out, seqs=ints(torch, seqs), max_keys=max_keys, window=window, sinks=sinks)
            want, tol = f.expect(q, [1] * len(seqs), seqs, window, sinks, tokens=True)
            compare(out, want, tol)
    again = torch.empty_like(out)
    f.cache.attend(q, again, seqs=ints(torch, seqs), max_keys=max_keys, window=3000, sinks=4)
    assert torch.equal(out, again)   # the order of the shares is fixed
    f.cache.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,width", [((4, 2), 64), ((6, 2), 128), ((2, 2), 256), ((1, 1), 512)])
def test_prompts_of_fp32_keep_twice_the_bits(torch, nt, kind, heads, width):
    """Within the tolerance of single tokens, also where the keys are shared by workgroups and where infinities are among the values."""
    past, new = [0, 33, 2500], [150, 70, 41]
    f = Filled(torch, nt, kind, "f32", past, heads, width, 64, seed=width, spare=12)
    first, r = ints(torch, rows_of(new)), rows_of(new)
    f.cache.reserve(3, first=first)
    k, v, q = f.random(sum(new), heads[1]), f.random(sum(new), heads[1]), f.random(sum(new), heads[0])
    hk, hv = held(torch, kind, k), held(torch, kind, v)
    for i in range(3):
        f.k[0][i], f.v[0][i] = np.concatenate([f.k[0][i], hk[r[i]:r[i + 1]]]), np.concatenate([f.v[0][i], hv[r[i]:r[i + 1]]])
    for window, sinks in [(0, 0), (100, 3)]:
        out = torch.empty_like(q)
        f.cache.attend(q, out, 3, first=first, k=k, v=v, max_new=150, window=window, sinks=sinks)
        want, tol = f.expect(q, new, range(3), window, sinks, tokens=True)
        compare(out, want, tol)
    if kind != "q4":
        again, v[100] = torch.empty_like(out), float("-inf")
        f.cache.attend(q, again, 3, first=first, k=k, v=v, max_new=150, window=100, sinks=3)
        assert torch.equal(again[:100], out[:100]) and torch.equal(again[150:], out[150:])
        assert (again[100:150] == float("-inf")).all()
    f.cache.check()


@pytest.mark.parametrize("kind,io", [("bf16", "f32"), ("f16", "bf16"), ("bf16", "f16")])
def test_other_pairs_of_types(torch, nt, kind, io):
    f = Filled(torch, nt, kind, io, [1, 40, 300], (4, 2), 128, 64, seed=2)
    q = f.random(3, 4)
    out = torch.empty_like(q)
    f.cache.attend(q, out, 3, window=100, sinks=3)
    want, tol = f.expect(q, [1, 1, 1], range(3), 100, 3, tokens=True)
    compare(out, want, tol)
    new, first = [1, 30, 100], ints(torch, [0, 1, 31, 131])
    f.cache.truncate(3, lengths=ints(torch, [1, 40, 300]))
    f.cache.reserve(3, first=first)
    k, v, q = f.random(131, 2), f.random(131, 2), f.random(131, 4)
    hk, hv, r = held(torch, kind, k), held(torch, kind, v), rows_of(new)
    for i in range(3):
        f.k[0][i], f.v[0][i] = np.concatenate([f.k[0][i], hk[r[i]:r[i + 1]]]), np.concatenate([f.v[0][i], hv[r[i]:r[i + 1]]])
    out = torch.empty_like(q)
    f.cache.attend(q, out, 3, first=first, k=k, v=v, max_new=100)
    want, tol = f.expect(q, new, range(3), 0, 0)
    compare(out, want, tol)
    f.cache.check()


def test_negative_and_zero_scale(torch, nt):
    for kind, new in (("f16", 1), ("q4", 1), ("f16", 70), ("bf16", 70)):
        io = "bf16" if kind == "bf16" else "f16"
        f = Filled(torch, nt, kind, io, [100], (4, 2), 64, 64, seed=2)
        q = f.random(new, 4)
        for scale in (-0.2, 0.0):
            out = torch.empty_like(q)
            f.cache.attend(q, out, 1, first=ints(torch, [0, new]) if new > 1 else None, max_new=new, scale=scale)
            want, tol = f.expect(q, [new], [0], 0, 0, scale=scale, tokens=new == 1)
            compare(out, want, tol)


def test_one_step_of_many_sequences(torch, nt):
    """More sequences than workgroups that share keys, ids in any order, twelve query heads to a key/value head."""
    n = 1500
    lens = [1 + i % 90 for i in range(n)]
    f = Filled(torch, nt, "q4", "bf16", lens, (12, 1), 64, 32, seed=5, spare=40)  # 34 of them are 32 or 64 long: the step takes as many pages
    order = np.random.default_rng(1).permutation(n)
    d = ints(torch, order)
    f.cache.reserve(seqs=d)
    k, v, q = f.random(n, 1), f.random(n, 1), f.random(n, 12)
    out = torch.empty_like(q)
    f.cache.attend(q, out, seqs=d, k=k, v=v, window=60, sinks=1)
    hk, hv = held(torch, "q4", k), held(torch, "q4", v)
    for i, s in enumerate(order):
        f.k[0][s], f.v[0][s] = np.concatenate([f.k[0][s], hk[i:i + 1]]), np.concatenate([f.v[0][s], hv[i:i + 1]])
    want, tol = f.expect(q, [1] * n, order, 60, 1, tokens=True)
    compare(out, want, tol)
    f.cache.check()


def test_large_and_tiny_numbers(torch, nt):
    """Queries beyond fp16 with small keys, tiny queries with large keys.  (Without the scale of 1e-3 the first kind's scores were
    sums of 64 products of about 1e6 * 3e-3 * 0.6, and fp32 sums of 1e5 decide no weight: 68 half steps of them are 0.5.)"""
    for kind, io in [("q4", "f32"), ("f16", "f32"), ("q4", "bf16"), ("bf16", "bf16")]:
        for size in (1e6, 1e-6):
            f = Filled(torch, nt, kind, io, [70, 300], (2, 1), 64, 64, seed=9, k_scale=3e-3 if size > 1 else 1e4 if kind != "q4" else 1e3)
            q = (f.random(2, 2).float() * size).to(types(torch)[io])
            out = torch.empty_like(q)
            scale = 1e-3 if size > 1 else 1.0
            f.cache.attend(q, out, 2, scale=scale)
            want, tol = f.expect(q, [1, 1], range(2), 0, 0, scale=scale, tokens=True)
            assert tol.max() < 0.1
            compare(out, want, tol)


# ---- many rows -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind,io", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("q4", "f16"), ("q4", "bf16")])
@pytest.mark.parametrize("heads,width,page", [((4, 2), 64, 32), ((6, 2), 128, 64), ((1, 1), 512, 128), ((2, 2), 256, 64), ((12, 1), 64, 256)])
def test_prompts(torch, nt, kind, io, heads, width, page):
    """New tokens behind cached ones, written and attended in one call; lengths around tiles, and a sequence without new ones."""
    past, new = [0, 5, 31, 64, 100, 0, 77], [1, 27, 1, 65, 130, 33, 0]
    f = Filled(torch, nt, kind, io, past, heads, width, page, seed=width, spare=40)
    n, first = len(past), ints(torch, rows_of(new))
    f.cache.reserve(n, first=first)
    k, v, q = f.random(sum(new), heads[1]), f.random(sum(new), heads[1]), f.random(sum(new), heads[0])
    hk, hv, r = held(torch, kind, k), held(torch, kind, v), rows_of(new)
    for i in range(n):
        f.k[0][i] = np.concatenate([f.k[0][i], hk[r[i]:r[i + 1]]])
        f.v[0][i] = np.concatenate([f.v[0][i], hv[r[i]:r[i + 1]]])
    for window, sinks in [(0, 0), (1, 0), (50, 3), (20, 40), (64, 0)]:
        out = torch.full((sum(new) + 1, heads[0], width), 5.0, dtype=types(torch)[io], device="cuda")
        f.cache.attend(q, out[:-1], n, first=first, k=k, v=v, max_new=130, window=window, sinks=sinks)
        want, tol = f.expect(q, new, range(n), window, sinks)
        compare(out[:-1], want, tol)
        assert (out[-1] == 5).all()  # rows behind the last sequence
    f.cache.check()


@pytest.mark.parametrize("kind,io", [("f16", "f32"), ("bf16", "bf16"), ("q4", "f16")])
@pytest.mark.parametrize("new", [[2, 1, 0], [9, 16, 3], [17, 5, 16], [40, 0, 33], [130, 64, 1]])
@pytest.mark.parametrize("heads,width", [((8, 2), 128), ((1, 1), 512), ((2, 2), 64)])
def test_new_tokens_over_many_keys(torch, nt, kind, io, new, heads, width):
    """Rows of several tokens whose keys are shared by workgroups: both kernels, and rows of sequences that are much shorter."""
    f = Filled(torch, nt, kind, io, [5000, 70, 1], heads, width, 64, seed=sum(new), spare=20)
    first, r = ints(torch, rows_of(new)), rows_of(new)
    f.cache.reserve(3, first=first)
    k, v, q = f.random(sum(new), heads[1]), f.random(sum(new), heads[1]), f.random(sum(new), heads[0])
    hk, hv = held(torch, kind, k), held(torch, kind, v)
    for i in range(3):
        f.k[0][i], f.v[0][i] = np.concatenate([f.k[0][i], hk[r[i]:r[i + 1]]]), np.concatenate([f.v[0][i], hv[r[i]:r[i + 1]]])
    for window, sinks in [(0, 0), (1500, 7)]:
        out = torch.full((sum(new) + 1, heads[0], width), 5.0, dtype=types(torch)[io], device="cuda")
        f.cache.attend(q, out[:-1], 3, first=first, k=k, v=v, max_new=max(new), window=window, sinks=sinks)
        want, tol = f.expect(q, new, range(3), window, sinks)
        compare(out[:-1], want, tol)
        assert (out[-1] == 5).all()
    # a value that is no number, seen by the later half of the longest's rows: no trace in the earlier ones
    if new[0] > 1 and kind != "q4":
        half, plain = new[0] // 2, out.clone()
        v[half] = float("inf")
        f.cache.attend(q, out[:-1], 3, first=first, k=k, v=v, max_new=max(new), window=1500, sinks=7)
        assert torch.equal(out[:half], plain[:half]) and torch.equal(out[new[0]:], plain[new[0]:])
        assert not torch.isfinite(out[half:new[0]]).any()
    f.cache.check()


@pytest.mark.parametrize("kind,io", [("f16", "f16"), ("bf16", "bf16"), ("q4", "f16")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_values_have_no_influence(torch, nt, kind, io, bad):
    """Keys and values that are no numbers reach the queries that see them and no others: later tokens, tokens before the window."""
    f = Filled(torch, nt, kind, io, [40, 3], (4, 2), 64, 32, spare=20, seed=1)
    new = [90, 50]
    n, first, r = 2, ints(torch, rows_of(new)), rows_of(new)
    f.cache.reserve(n, first=first)
    k, v, q = f.random(sum(new), 2), f.random(sum(new), 2), f.random(sum(new), 4)
    plain_k, plain_v = k.clone(), v.clone()
    spot = [r[0] + 20, r[1] + 31]          # positions 60 and 34
    for row in spot:
        k[row, 0], v[row, 1] = bad, bad
    for window, sinks in [(0, 0), (30, 2)]:
        out, clean = torch.empty_like(q), torch.empty_like(q)
        f.cache.attend(q, out, n, first=first, k=k, v=v, max_new=90, window=window, sinks=sinks)
        f.cache.attend(q, clean, n, first=first, k=plain_k, v=plain_v, max_new=90, window=window, sinks=sinks)
        for i, row in enumerate(spot):
            for t in range(new[i]):
                sees = t >= row - r[i] and (not window or t - (row - r[i]) < window)
                if not sees:
                    assert torch.equal(out[r[i] + t], clean[r[i] + t]), (i, t)
                elif math.isnan(bad) or kind != "q4":
                    assert not torch.isfinite(out[r[i] + t, 2:]).all()
    # the newest token alone does not see them through the window either
    f.cache.write(k, v, n, first=first, max_new=90)
    q1, out1, clean1 = q[:2].contiguous(), torch.empty_like(q[:2]), torch.empty_like(q[:2])
    f.cache.attend(q1, out1, n, window=15, sinks=1)
    f.cache.write(plain_k, plain_v, n, first=first, max_new=90)
    f.cache.attend(q1, clean1, n, window=15, sinks=1)
    assert torch.equal(out1, clean1) and torch.isfinite(out1).all()


def test_pages_with_old_contents_that_are_no_numbers(torch, nt):
    """A freed page keeps what it held; the unfilled part of a page has no influence when it is handed out again."""
    for kind in KINDS:
        io = "bf16" if kind == "bf16" else "f16"
        f = Filled(torch, nt, kind, io, [64], (2, 1), 64, 64, spare=0, max_seqs=2)
        nan = torch.full((64, 1, 64), float("nan"), dtype=types(torch)[io], device="cuda")
        f.cache.truncate(1)
        first = ints(torch, [0, 64])
        f.cache.reserve(1, first=first)
        f.cache.write(nan, nan, 1, first=first, max_new=64)
        f.cache.truncate(1)
        k, v, q = f.random(5, 1), f.random(5, 1), f.random(5, 2)
        first = ints(torch, [0, 5])
        f.cache.reserve(1, first=first)
        out = torch.empty_like(q)
        f.cache.attend(q, out, 1, first=first, k=k, v=v, max_new=5)
        f.k[0][0], f.v[0][0] = held(torch, kind, k), held(torch, kind, v)
        want, tol = f.expect(q, [5], [0], 0, 0)
        compare(out, want, tol)
        one = torch.empty_like(q[:1])
        f.cache.attend(q[4:], one, 1)
        want, tol = f.expect(q[4:], [1], [0], 0, 0, tokens=True)
        compare(one, want, tol)


# ---- rounding ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_read_returns_what_is_held(torch, nt, kind, io):
    """Borders between codes and scales, numbers beyond the range, zeros of both signs, tiny ones; all lengths of a tile."""
    rng = np.random.default_rng(5)
    lens = list(range(0, 70, 3))
    rows = sum(lens)
    x = rng.normal(0, 1, (rows, 2, 64)) * np.exp(rng.normal(0, 4, (rows, 2, 1)))
    grid = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6])
    for r in range(0, rows, 3):  # a block on the borders of its codes, a power of two away from 1
        x[r, 0, :32] = rng.permutation(np.concatenate([grid, -grid, [6, 0]])) * 2.0 ** rng.integers(-8, 8)
        x[r, 1, 32:] = rng.choice([1.25, 1.5, 1.75]) * rng.permutation(np.concatenate([grid, -grid, [6, -0.0]])) * 2.0 ** rng.integers(-6, 6)
    x[1], x[2, 0], x[4, 1] = 0, 1e5 * rng.normal(0, 1, 64), 1e-6
    if io == "f16":
        x = np.clip(x, -65504, 65504)
    k = torch.tensor(x, device="cuda").to(types(torch)[io])
    v = -k.flip(0)
    n, first = len(lens), ints(torch, rows_of(lens))
    cache = nt.Cache(kind, 2, 2, 2, 64, 60, n, 100, 32)
    cache.reserve(n, first=first)
    cache.write(k, v, n, first=first, max_new=max(lens), layer=1)
    gk, gv = (torch.full((n, 80, 2, 64), 9.0, dtype=torch.float32, device="cuda") for _ in range(2))
    cache.read(gk, gv, n, layer=1)
    hk, hv, r = held(torch, kind, k), held(torch, kind, v), rows_of(lens)
    for i in range(n):
        for got, want in ((gk, hk), (gv, hv)):
            assert np.array_equal(got[i, :lens[i]].double().cpu().numpy(), want[r[i]:r[i + 1]]), i
            assert (got[i, lens[i]:] == 0).all()
    cache.check()


def test_read_of_numbers_that_are_none(torch, nt):
    for kind in KINDS:
        k = torch.randn(3, 1, 64, device="cuda")
        k[0, 0, 3], k[1, 0, 40], k[2, 0, 5], k[2, 0, 6] = float("nan"), float("inf"), -float("inf"), 1.0
        cache = nt.Cache(kind, 1, 1, 1, 64, 2, 1, 64, 32)
        first = ints(torch, [0, 3])
        cache.reserve(1, first=first)
        cache.write(k, k, 1, first=first, max_new=3)
        gk, gv = torch.empty(1, 3, 1, 64, device="cuda"), torch.empty(1, 3, 1, 64, device="cuda")
        cache.read(gk, gv, 1)
        want = held(torch, kind, k)
        for g in (gk, gv):
            assert np.array_equal(g[0].double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("kind", KINDS)
def test_tokens_written_one_by_one(torch, nt, kind):
    """Equal to the same tokens written at once, whatever the pages held before."""
    io = "bf16" if kind == "bf16" else "f32"
    f = Filled(torch, nt, kind, io, [3, 37], (2, 2), 64, 32, spare=20)
    k, v = f.random(2 * 70, 2), f.random(2 * 70, 2)
    for t in range(70):
        f.cache.reserve(2)
        f.cache.write(k[2 * t:2 * t + 2], v[2 * t:2 * t + 2], 2)
    gk, gv = (torch.empty(2, 107, 2, 64, dtype=types(torch)[io], device="cuda") for _ in range(2))
    f.cache.read(gk, gv, 2)
    hk, hv = held(torch, kind, k), held(torch, kind, v)
    for i, p in enumerate([3, 37]):
        assert np.array_equal(gk[i, :p + 70].double().cpu().numpy(), np.concatenate([f.k[0][i], hk[i::2]]))
        assert np.array_equal(gv[i, :p + 70].double().cpu().numpy(), np.concatenate([f.v[0][i], hv[i::2]]))
    f.cache.check()


# ---- pages ---------------------------------------------------------------------------------------------------------

class Pool:
    """Sequences, their pages and holders."""

    def __init__(self, pages, page, seqs, layers):
        self.page, self.ref = page, [0] * pages
        self.rows = [[] for _ in range(seqs)]                       # pages, None = trimmed
        self.values = [[np.zeros((2, 0))] * layers for _ in range(seqs)]   # (key, value) marks per token

    def take(self):
        p = self.ref.index(0)
        self.ref[p] = 1
        return p

    def drop(self, p):
        if p is not None:
            self.ref[p] -= 1

    def used(self):
        return sum(r > 0 for r in self.ref), max([i + 1 for i, r in enumerate(self.ref) if r > 0], default=0)


@pytest.mark.parametrize("kind,page,layers", [("f16", 32, 2), ("q4", 64, 1), ("bf16", 32, 1)])
def test_page_calls_at_random(torch, nt, kind, page, layers):
    """Reserve, write, fork (permutations, one source several times, itself), copy, truncate, trim, compact in any order: contents, lengths
    and pages in use after every call."""
    rng = np.random.default_rng(page + layers)
    seqs, pages, longest = 9, 90, 300
    cache = nt.Cache(kind, layers, 1, 1, 64, pages, seqs, longest, page)
    pool = Pool(pages, page, seqs, layers)
    # a token is one value in all dims, exact in every kind: in 4 bits its scale is a sixth of it, which has to have 3 bits (2 would be
    # held as 2.25)
    values = 6 * np.array([0.125, 0.25, 0.5, 1, 1.25, 1.5, 1.75])
    gk, gv = (torch.empty(seqs, longest, 1, 64, device="cuda") for _ in range(2))
    for step in range(120):
        call = rng.choice(["add", "add", "add", "fork", "fork", "copy", "cut", "end", "trim", "compact"])
        if call == "add":
            ids = rng.permutation(seqs)[:rng.integers(1, seqs + 1)]
            counts = [int(min(rng.integers(0, 50), longest - pool.values[s][0].shape[1])) for s in ids]
            need = [-(-(pool.values[s][0].shape[1] + c) // page) - len(pool.rows[s]) for s, c in zip(ids, counts)]
            if sum(need) > pool.ref.count(0):
                continue
            first, d = ints(torch, rows_of(counts)), ints(torch, ids)
            cache.reserve(seqs=d, first=first)
            for s, k in zip(ids, need):
                pool.rows[s] = pool.rows[s] + [pool.take() for _ in range(k)]
            for l in range(layers):
                kv = rng.choice(values, (2, sum(counts)))
                k, v = (torch.tensor(x, device="cuda", dtype=torch.float32).reshape(-1, 1, 1).expand(-1, 1, 64).contiguous() for x in kv)
                cache.write(k, v, seqs=d, first=first, max_new=max(max(counts), 1), layer=l)
                r = rows_of(counts)
                for i, s in enumerate(ids):
                    pool.values[s] = list(pool.values[s])
                    pool.values[s][l] = np.concatenate([pool.values[s][l], kv[:, r[i]:r[i + 1]]], 1)
        elif call in ("fork", "copy"):
            n = int(rng.integers(1, seqs + 1))
            dst, src = rng.permutation(seqs)[:n], rng.integers(0, seqs, n)
            if rng.random() < 0.3:
                src = rng.permutation(dst)
            rows = [list(pool.rows[s]) for s in src]
            vals = [list(pool.values[s]) for s in src]
            copied = [[p for p in range(len(r)) if r[p] is not None and (call == "copy" or (p + 1) * page > v[0].shape[1])] if s != t else []
                      for r, v, s, t in zip(rows, vals, src, dst)]
            if sum(map(len, copied)) > pool.ref.count(0):
                continue
            cache.fork(ints(torch, src), ints(torch, dst)) if call == "fork" else cache.copy(ints(torch, src), ints(torch, dst))
            for r, which, s, t in zip(rows, copied, src, dst):
                if s == t:
                    continue
                for p in which:
                    r[p] = pool.take()
                for p in range(len(r)):
                    if p not in which and r[p] is not None:
                        pool.ref[r[p]] += 1
            for r, v, s, t in zip(rows, vals, src, dst):
                if s != t:
                    for p in pool.rows[t]:
                        pool.drop(p)
            for r, v, t in zip(rows, vals, dst):
                pool.rows[t], pool.values[t] = r, v
        elif call == "cut":
            ids = rng.permutation(seqs)[:rng.integers(1, seqs + 1)]
            keep = []
            for s in ids:
                l = pool.values[s][0].shape[1]
                k = int(rng.integers(0, l + 1))
                keep.append(l if k % page and pool.rows[s][k // page] is None else k)
            shared = sum(1 for s, k in zip(ids, keep) if k % page and k < pool.values[s][0].shape[1] and pool.ref[pool.rows[s][k // page]] > 1)
            if shared > pool.ref.count(0):
                continue
            cache.truncate(seqs=ints(torch, ids), lengths=ints(torch, keep))
            split = [k % page and k < pool.values[s][0].shape[1] and pool.ref[pool.rows[s][k // page]] > 1 for s, k in zip(ids, keep)]
            fresh = [pool.take() if x else None for x in split]
            for s, k, x, p in zip(ids, keep, split, fresh):
                n = -(-k // page)
                for q in pool.rows[s][n:]:
                    pool.drop(q)
                pool.rows[s] = pool.rows[s][:n]
                if x:
                    pool.drop(pool.rows[s][-1])
                    pool.rows[s][-1] = p
                pool.values[s] = [v[:, :k] for v in pool.values[s]]
        elif call == "end":
            ids = rng.permutation(seqs)[:2]
            cache.truncate(seqs=ints(torch, ids))
            for s in ids:
                for p in pool.rows[s]:
                    pool.drop(p)
                pool.rows[s], pool.values[s] = [], [np.zeros((2, 0))] * layers
        elif call == "trim":
            ids, window, sinks = rng.permutation(seqs)[:3], int(rng.integers(1, 120)), int(rng.integers(0, 70))
            cache.trim(window, sinks, seqs=ints(torch, ids))
            for s in ids:
                l = pool.values[s][0].shape[1]
                for p in range(len(pool.rows[s])):
                    if p * page >= sinks and (p + 1) * page <= l - window:
                        pool.drop(pool.rows[s][p])
                        pool.rows[s][p] = None
        else:
            cache.compact()
            n = pool.used()[0]
            moved = dict(zip([p for p in range(n, pages) if pool.ref[p]], [p for p in range(n) if not pool.ref[p]]))
            for a, b in moved.items():
                pool.ref[b], pool.ref[a] = pool.ref[a], 0
            pool.rows = [[moved.get(p, p) for p in r] for r in pool.rows]
        lens, used = cache.lengths()
        assert lens.tolist() == [v[0].shape[1] for v in pool.values], (step, call)
        assert tuple(used.tolist()) == pool.used(), (step, call)
        for l in range(layers):
            cache.read(gk, gv, seqs, layer=l)
            for x, side in ((gk, 0), (gv, 1)):
                got = x[:, :, 0].cpu().numpy()
                assert (got == got[..., :1]).all()
                for s in range(seqs):
                    want = np.zeros(longest)
                    for t, val in enumerate(pool.values[s][l][side]):
                        want[t] = val if pool.rows[s][t // page] is not None else 0
                    assert np.array_equal(got[s, :, 0], want), (step, call, s)
    cache.check()


def test_attention_after_trim(torch, nt):
    """Freed pages are not seen, and what the window shows is still there."""
    for kind, io in [("f16", "f16"), ("q4", "bf16")]:
        f = Filled(torch, nt, kind, io, [500, 130], (2, 1), 64, 32, seed=4)
        q = f.random(2, 2)
        before, after, wide = (torch.empty_like(q) for _ in range(3))
        f.cache.attend(q, before, 2, window=100, sinks=5)
        f.cache.trim(100, 5, n=2)
        f.cache.attend(q, after, 2, window=100, sinks=5)
        assert torch.equal(before, after)
        f.cache.attend(q, wide, 2)
        for i, l in enumerate([500, 130]):
            page = np.arange(l) // 32
            present = (page * 32 < 5) | ((page + 1) * 32 > l - 100)
            want, biggest, most = attention(q[i:i + 1].double().cpu().numpy(), f.k[0][i], f.v[0][i], l - 1, 0, 0, 64 ** -0.5, present)
            compare(wide[i:i + 1], want, allowed(kind, io, 64, biggest, most, np.abs(f.v[0][i]).max(), want, True))
        f.cache.check()


def test_what_does_not_fit_is_skipped_and_reported(torch, nt):
    def code(f):
        with pytest.raises(nt.NtError) as e:
            f()
        return e.value.code

    cache = nt.Cache("f16", 1, 1, 1, 64, 6, 4, 200, 32)
    k = torch.randn(200, 1, 64, device="cuda").half()
    state = lambda: (cache.lengths()[0].tolist(), cache.lengths()[1].tolist())
    cache.reserve(seqs=ints(torch, [0, 1]), first=ints(torch, [0, 33, 73]))
    cache.write(k, k, seqs=ints(torch, [0, 1]), first=ints(torch, [0, 33, 73]), max_new=40)
    assert state() == ([33, 40, 0, 0], [4, 4])
    # ids that are none, the second of two equal ones, more than max_len, a negative count
    cache.reserve(seqs=ints(torch, [-1, 4, 2, 2]), first=ints(torch, [0, 1, 2, 7, 9]))
    cache.reserve(seqs=ints(torch, [3, 1]), first=ints(torch, [0, 201, 196]))
    assert state() == ([33, 40, 5, 0], [5, 5]) and code(cache.check) == -6
    cache.check()
    # no pages: those before it in the call are served, what needs none is served too
    cache.reserve(seqs=ints(torch, [0, 3, 2, 1]), first=ints(torch, [0, 40, 60, 61, 100]))
    assert state() == ([73, 40, 6, 0], [6, 6]) and code(cache.check) == -4
    # rows of a sequence that got no room are not written
    cache.write(k, k, seqs=ints(torch, [0, 3, 2, 1]), first=ints(torch, [0, 40, 60, 61, 100]), max_new=40)
    assert code(cache.check) == -6
    got = [torch.empty(4, 80, 1, 64, device="cuda").half() for _ in range(2)]
    cache.read(*got, 4)
    assert torch.equal(got[0][0, :33], k[:33]) and torch.equal(got[0][0, 33:73], k[:40]) and torch.equal(got[0][1, :40], k[33:73])
    # copies and forks without room, of ids that are none, to one target twice
    cache.copy(ints(torch, [1]), ints(torch, [3]))
    assert state() == ([73, 40, 6, 0], [6, 6]) and code(cache.check) == -4
    cache.fork(ints(torch, [1, 5, 2, 0]), ints(torch, [1, 0, -1, 1]))
    assert state() == ([73, 40, 6, 0], [6, 6]) and code(cache.check) == -6
    # lengths that a sequence does not have
    cache.truncate(seqs=ints(torch, [0, 1, 9, 2]), lengths=ints(torch, [74, -1, 0, 6]))
    assert state() == ([73, 40, 6, 0], [6, 6]) and code(cache.check) == -6
    # queries beyond a length, and of ids that are none: zeros
    q, out = torch.randn(5, 1, 64, device="cuda").half(), torch.ones(5, 1, 64, device="cuda").half()
    cache.attend(q, out, seqs=ints(torch, [3, 7, 1]), first=ints(torch, [0, 2, 4, 5]), max_new=2)
    assert (out[:4] == 0).all() and (out[4] != 0).any() and code(cache.check) == -6
    cache.trim(1, 0, seqs=ints(torch, [9]))
    assert code(cache.check) == -6
    # trimmed inside: cannot be cut there
    cache.trim(1, 0, seqs=ints(torch, [0]))
    cache.truncate(seqs=ints(torch, [0]), lengths=ints(torch, [40]))
    assert state()[0][0] == 73 and code(cache.check) == -6
    cache.truncate(seqs=ints(torch, [0, 1, 2, 0]))
    assert state() == ([0, 0, 0, 0], [0, 0]) and code(cache.check) == -6


# ---- how it is called ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind,io", [("f16", "f16"), ("q4", "f32"), ("bf16", "bf16")])
def test_strides_and_alignment(torch, nt, kind, io):
    """Rows of a fused projection, at odd offsets; outputs among other columns."""
    f = Filled(torch, nt, kind, io, [37, 64], (4, 2), 64, 32, spare=8)
    new, first = [3, 40], ints(torch, [0, 3, 43])
    f.cache.reserve(2, first=first)
    for shift in (0, 1):
        wide = f.random(43, 1)[:, 0, :1].expand(43, 8 * 64 + 3).clone().normal_(generator=f.g)
        parts = [wide[:, shift + a * 64:shift + b * 64].unflatten(1, (-1, 64)) for a, b in ((0, 4), (4, 6), (6, 8))]
        holder = torch.full((43, 300), 3.0, dtype=wide.dtype, device="cuda")
        out = holder[:, shift:shift + 256].unflatten(1, (4, 64))
        f.cache.attend(parts[0], out, 2, first=first, k=parts[1], v=parts[2], max_new=40, window=30, sinks=1)
        dense = torch.empty(43, 4, 64, dtype=wide.dtype, device="cuda")
        f.cache.attend(parts[0].contiguous(), dense, 2, first=first, k=parts[1].contiguous(), v=parts[2].contiguous(), max_new=40, window=30, sinks=1)
        assert torch.equal(out, dense) and (holder[:, shift + 256:] == 3).all() and (holder[:, :shift] == 3).all()
        one, one_dense = holder[:2, 1:257].unflatten(1, (4, 64)), dense[:2].clone()
        f.cache.attend(parts[0][:2], one, 2)
        f.cache.attend(parts[0][:2].contiguous(), one_dense, 2)
        assert torch.equal(one, one_dense)
    f.cache.check()


def test_pool_beyond_32_bit_offsets(torch, nt):
    """Pages behind the first 4 GiB of a pool, in a second layer too."""
    for kind in ("bf16", "q4"):
        pages = 20000 if kind == "bf16" else 70000
        cache = nt.Cache(kind, 2, 8, 8, 128, pages, 4, 64 * pages, 64)
        assert nt.Cache.bytes(kind, 2, 8, 8, 128, pages, 4, 64 * pages, 64) > 2 * 2 ** 32
        cache.reserve(seqs=ints(torch, [0]), first=ints(torch, [0, 64 * (pages - 6)]))
        first = ints(torch, [0, 100, 180])
        d = ints(torch, [1, 2])
        cache.reserve(seqs=d, first=first)
        g = torch.Generator("cuda").manual_seed(1)
        k, v, q = (torch.randn(180, 8, 128, device="cuda", generator=g).bfloat16() for _ in range(3))
        out = torch.empty_like(q)
        cache.attend(q, out, seqs=d, first=first, k=k, v=v, max_new=100, layer=1)
        small = nt.Cache(kind, 1, 8, 8, 128, 4, 3, 200, 64)
        small.reserve(seqs=d, first=first)
        want = torch.empty_like(q)
        small.attend(q, want, seqs=d, first=first, k=k, v=v, max_new=100)
        assert torch.equal(out, want)
        one, want_one = torch.empty_like(q[:2]), torch.empty_like(q[:2])
        cache.attend(q[:2], one, seqs=d, layer=1, max_keys=100)
        small.attend(q[:2], want_one, seqs=d, max_keys=100)
        assert torch.equal(one, want_one)
        cache.check()
        del cache


def test_captured_decoding(torch, nt):
    """A step (room, new token, attention, trim) captured into a graph and replayed, with eager steps and reads between the replays."""
    for kind, io in [("f16", "f16"), ("q4", "f16")]:
        runs = []
        for captured in (False, True):
            f = Filled(torch, nt, kind, io, [3, 70], (4, 2), 64, 32, spare=30, seed=6)
            k, v, q = f.random(2, 2), f.random(2, 2), f.random(2, 4)
            out, outs = torch.empty_like(q), []

            def step():
                f.cache.reserve(2)
                f.cache.attend(q, out, 2, k=k, v=v, window=60, sinks=2, max_keys=200)
                f.cache.trim(60, 2, n=2)

            if captured:
                torch.cuda.synchronize()
                stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    step()
            for t in range(40):
                for x in (k, v, q):
                    x.copy_(f.random(2, x.shape[1]))
                graph.replay() if captured and t % 3 else step()
                outs.append(out.clone())
                if t % 5 == 0:
                    torch.cuda.synchronize()
            f.cache.check()
            lens, pages = f.cache.lengths()
            runs.append((torch.stack(outs), lens, pages))
        for a, b in zip(*runs):
            assert torch.equal(a, b)


def test_on_another_stream(torch, nt):
    f = Filled(torch, nt, "f16", "f16", [300, 20], (4, 2), 64, 32)
    q, a, b = f.random(2, 4), *(torch.empty(2, 4, 64, device="cuda").half() for _ in range(2))
    f.cache.attend(q, a, 2)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    f.cache.attend(q, b, 2, stream=other)
    other.synchronize()
    assert torch.equal(a, b)


def test_beam_of_hypotheses(torch, nt):
    """The calls as they are used together: a prompt, then steps whose hypotheses are permuted and forked, against sequences that
    are kept whole."""
    rng = np.random.default_rng(8)
    for kind, io in [("f16", "f32"), ("q4", "f16")]:
        beams, steps, heads, width = 5, 45, (4, 1), 64
        f = Filled(torch, nt, kind, io, [41], heads, width, 32, spare=60, max_seqs=beams)
        f.cache.fork(ints(torch, [0] * (beams - 1)), ints(torch, range(1, beams)))
        f.k[0], f.v[0] = [[f.k[0][0]] * beams], [[f.v[0][0]] * beams]
        f.k, f.v = f.k[0], f.v[0]
        everyone = ints(torch, range(beams))
        for t in range(steps):
            parent = rng.integers(0, beams, beams)
            f.cache.fork(ints(torch, parent), everyone)
            k, v, q = f.random(beams, 1), f.random(beams, 1), f.random(beams, 4)
            out = torch.empty_like(q)
            f.cache.reserve(beams)
            f.cache.attend(q, out, beams, k=k, v=v, window=50, sinks=3)
            hk, hv = held(torch, kind, k), held(torch, kind, v)
            f.k[0] = [np.concatenate([f.k[0][p], hk[i:i + 1]]) for i, p in enumerate(parent)]
            f.v[0] = [np.concatenate([f.v[0][p], hv[i:i + 1]]) for i, p in enumerate(parent)]
            if t % 9 == 0:
                f.cache.compact()
            want, tol = f.expect(q, [1] * beams, range(beams), 50, 3, tokens=True)
            compare(out, want, tol)
        f.cache.truncate(beams)
        assert f.cache.lengths()[1].tolist() == [0, 0]
        f.cache.check()
