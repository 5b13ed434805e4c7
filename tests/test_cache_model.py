"""Models whose decoder keeps its self-attention's keys and values in a paged cache (nt_config.self_cache, self_window,
self_sinks), against the oracle and against an independent decoder with a window and rounded keys and values."""
import numpy as np
import pytest

import nt_synth
from oracle import nt_oracle_np as onp
from test_cache import four_bits
from test_gpu_parity import audit_mismatches, nt, pad, rel_l2, split, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = {"one head": ("C0", dict(vocab=600)), "eight heads, FFN, two layers": ("C3", dict(vocab=700, n_enc=2, n_dec=2)),
          "width 320": ("C0", dict(vocab=500, d_model=320, n_heads=5, d_ffn=128, n_enc=2))}


def held(kind, x):
    """What a cache of this kind holds of x [..., heads, d_head], given as fp32"""
    if kind == "q4":
        return four_bits(x.astype(np.float32).astype(np.float64))
    if kind == "f16":
        return x.astype(np.float32).astype(np.float16).astype(np.float64)
    b = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)).view(np.float32).astype(np.float64)


def decoder_logits(cfg, blob, src, tgt_in, kind, window, sinks):
    """Teacher-forced logits, each self-attention with rounded keys and values and a window.  list of [T, V]"""
    W = onp.Weights(cfg, blob)
    d, eps, H = cfg["d_model"], cfg["ln_eps"], nt_synth.dec_heads(cfg)
    enc, lens = onp.encode(cfg, blob, src)
    tid, tlens = onp.pad_batch(tgt_in, cfg["pad_id"])
    B, T = tid.shape
    z = np.sqrt(d) * W["E"][tid] + onp.positions(T, d)[None]
    t = np.arange(T)
    seen = t[None, :] <= t[:, None]
    if window:
        seen &= (t[:, None] - t[None, :] < window) | (t[None, :] < sinks)
    cross = np.broadcast_to((np.arange(enc.shape[1])[None, :] < lens[:, None])[:, None, :], (B, T, enc.shape[1]))
    for l in range(cfg["n_dec"]):
        a = onp.layer_norm(z, W[f"dec{l}.ln1.g"], W[f"dec{l}.ln1.b"], eps)
        q, k, v = ((a @ W[f"dec{l}.self.W{n}"] + W[f"dec{l}.self.b{n}"]).reshape(B, T, H, d // H) for n in "qkv")
        k, v = held(kind, k), held(kind, v)
        s = np.einsum("bqhd,bkhd->bhqk", q / np.sqrt(d // H), k)
        o = np.einsum("bhqk,bkhd->bqhd", onp.masked_softmax(s, seen[None, None]), v).reshape(B, T, d)
        z = z + o @ W[f"dec{l}.self.Wo"] + W[f"dec{l}.self.bo"]
        a = onp.layer_norm(z, W[f"dec{l}.ln2.g"], W[f"dec{l}.ln2.b"], eps)
        z = z + onp.attention(W, f"dec{l}.cross", a, enc, cross, False, H)[0]
        if nt_synth.dec_ffn(cfg):
            z = onp.ffn(W, f"dec{l}.ln3", f"dec{l}.ffn", z)
    h = onp.layer_norm(z, W["dec_final.g"], W["dec_final.b"], eps)
    return [(h @ (W["E"] if cfg["tie_output"] else W["W_out"]).T)[i, :tlens[i]] for i in range(B)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind,window,sinks", [("f16", 0, 0), ("f16", 7, 2), ("bf16", 40, 0), ("q4", 0, 0), ("q4", 33, 1)])
def test_teacher_forced_logits(torch_cuda, nt, shape, kind, window, sinks):  # noqa: F811
    """The tolerances of the other logits (rel-L2 2e-3): the rounding is on both sides, and a key or value that the two sides compute
    on different sides of a border is one in about 2^20 of them."""
    torch = torch_cuda
    name, kw = SHAPES[shape]
    cfg = nt_synth.model_config(name, **kw)
    blob = nt_synth.make_weights(cfg, seed=3, random_affine=True)
    rng = np.random.default_rng(4)
    src = [rng.integers(4, cfg["vocab"], n) for n in (5, 17, 30, 1)]
    T = 70
    tgt = [np.concatenate([[cfg["bos_id"]], rng.integers(4, cfg["vocab"], T - 1)]) for _ in src]
    ids, lens = pad(src, cfg["pad_id"])
    gm = nt.Model(dict(cfg, self_cache=kind, self_window=window, self_sinks=sinks), blob, max_batch_tokens=2048, pipeline_lanes=1)
    logits = torch.empty((len(src), T, cfg["vocab"]), dtype=torch.float32, device="cuda")
    want = decoder_logits(cfg, blob, src, tgt, kind, window, sinks)
    for _ in range(2):  # the second decode finds the first one's pages
        gm.encode(torch.from_numpy(ids).cuda(), torch.from_numpy(lens).cuda())
        logits.fill_(float("nan"))
        gm.debug_teacher_forced_logits(torch.from_numpy(np.stack(tgt).astype(np.int32)).cuda(), logits)
        for g, w in zip(logits.cpu().numpy(), want):
            assert rel_l2(g, w) <= 2e-3, rel_l2(g, w)
    gm.check_device_flags()
    gm.close()


@pytest.mark.parametrize("shape", SHAPES)
def test_greedy_against_oracle(torch_cuda, nt, oracle, shape):  # noqa: F811
    """fp16 pages, no window: the oracle's tokens, but for near-ties, in every call that decodes."""
    name, kw = SHAPES[shape]
    cfg = nt_synth.model_config(name, **kw)
    blob = nt_synth.make_weights(cfg, seed=1)
    tokens, offsets = _sentences(cfg, 60)
    om = oracle.Model(cfg, blob)
    ref, ro, _ = om.translate(tokens, offsets)
    gm = nt.Model(dict(cfg, self_cache="f16"), blob, max_batch_tokens=4096)
    src = split(tokens, offsets)
    whole, oo = gm.translate_batch(tokens, offsets, token_budget=4096)
    assert np.array_equal(oo, ro)
    bad, _ = audit_mismatches(om, src, split(whole, oo), split(ref, ro), cfg)
    assert bad <= 2, bad
    # small batches on all lanes, and the mode that ends sentences (no sentence emits this id before its cap or all of them do)
    small, _ = gm.translate_batch(tokens, offsets, token_budget=300)
    assert (small != whole).mean() <= 0.02
    eos = int(np.bincount(whole).argmax())
    out, o2, length = gm.translate_batch_eos(tokens, offsets, 4096, eos)
    assert np.array_equal(o2, oo)
    cut = 0
    for i in range(len(oo) - 1):
        w, g = whole[oo[i]:oo[i + 1]], out[oo[i]:oo[i + 1]]
        end = np.nonzero(w == eos)[0]
        n = int(end[0]) + 1 if len(end) else len(w)
        if length[i] != n or not np.array_equal(g[:n], w[:n]):
            cut += 1
        assert (g[length[i]:] == cfg["pad_id"]).all()
    assert cut <= 1, cut
    gm.check_device_flags()
    gm.close()


def _sentences(cfg, n):
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 30, n)
    return rng.integers(4, cfg["vocab"], lens.sum()).astype(np.int32), np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def test_pages_of_a_long_batch(torch_cuda, nt):  # noqa: F811
    """The largest batch the arena takes, twice, with steps per row: no page is missing."""
    torch = torch_cuda
    cfg = nt_synth.model_config("C0", vocab=300, n_enc=1, max_len=128)
    blob = nt_synth.make_weights(cfg, seed=0)
    gm = nt.Model(dict(cfg, self_cache="q4", self_window=30), blob, max_batch_tokens=1000, pipeline_lanes=1)
    for rows, length in ((1000, 1), (10, 100), (31, 32), (1000, 1)):
        steps = min(nt.n_steps(length), cfg["max_len"])
        ids = torch.randint(4, 300, (rows, length), dtype=torch.int32, device="cuda")
        gm.encode(ids, torch.full((rows,), length, dtype=torch.int32, device="cuda"))
        out = torch.full((rows, steps), -1, dtype=torch.int32, device="cuda")
        gm.decode_greedy(rows, steps, out)
        again = torch.full_like(out, -1)
        gm.decode_greedy(rows, steps, again)
        assert torch.equal(out, again) and int(out.min()) >= 0
    gm.check_device_flags()
    gm.close()
