"""Host side of the paged caches on a HIP runtime that runs nothing: what is refused, with which code, and that a refused call launches
nothing; sizes; which kernels the calls launch."""
import pytest
from test_host_launches import host  # noqa: F401  (a fixture)

CACHE = """
from paper_2109_08003_amd.binding import NtCacheConfig, NtAttendArgs, lib
L = lib()

def config(kind=1, n_layers=2, n_q_heads=4, n_kv_heads=2, d_head=64, page_tokens=64, n_pages=8, max_seqs=4, max_len=200):
    return NtCacheConfig(C.sizeof(NtCacheConfig), kind, n_layers, n_q_heads, n_kv_heads, d_head, page_tokens, n_pages, max_seqs, max_len)

def create(**kw):
    h = C.c_void_p(1)
    return L.nt_cache_create(C.byref(config(**kw)), None, C.byref(h)), h

x = np.zeros(1 << 16, dtype=np.float32).ctypes.data   # stands for any device buffer
def attend(h, **kw):
    a = NtAttendArgs(C.sizeof(NtAttendArgs), 0, 2, 1, 0, 0, 0, 0, 1.0)
    a.q = a.out = x
    a.ld_q = a.ld_out = 256
    for k, v in kw.items():
        setattr(a, k, v)
    return L.nt_cache_attend(h, C.byref(a), None)
"""


def test_configurations(host):  # noqa: F811
    bad, good, null = host(CACHE + """
bad = [(kw, create(**kw)[0], create(**kw)[1].value, int(L.nt_cache_bytes(C.byref(config(**kw))))) for kw in (
    dict(kind=0), dict(kind=4), dict(n_layers=0), dict(n_q_heads=3), dict(n_q_heads=1), dict(n_kv_heads=0), dict(d_head=96), dict(d_head=1024),
    dict(page_tokens=16), dict(page_tokens=48), dict(page_tokens=512), dict(n_pages=0), dict(n_pages=1 << 25), dict(max_seqs=0), dict(max_seqs=1 << 21),
    dict(max_len=0), dict(max_len=1 << 25), dict(n_pages=1 << 24, page_tokens=256, n_layers=1024, n_kv_heads=4))]
good = [(k, d, p, create(kind=k, d_head=d, page_tokens=p)[0], int(L.nt_cache_bytes(C.byref(config(kind=k, d_head=d, page_tokens=p)))))
        for k in (1, 2, 3) for d in (64, 128, 256, 512) for p in (32, 64, 128, 256)]
c = config(); c.struct_size = 8
h = C.c_void_p()
null = [L.nt_cache_create(None, None, C.byref(h)), L.nt_cache_create(C.byref(config()), None, None), L.nt_cache_create(C.byref(c), None, C.byref(h)),
        L.nt_cache_reserve(None, 1, None, None, None), L.nt_cache_attend(None, None, None), L.nt_cache_compact(None, None), L.nt_cache_check(None, None),
        int(L.nt_cache_bytes(None))]
L.nt_cache_destroy(None)
print(json.dumps((bad, good, null)))
""")
    for kw, rc, handle, size in bad:
        assert rc == (-1 if "kind" in kw else -2) and handle is None and size == 0, kw
    for kind, width, page, rc, size in good:
        token = 2 * 2 * (width * 2 if kind < 3 else width // 2 + width // 32)   # two heads, keys and values
        pool = 2 * 8 * page * token                                            # two layers of eight pages
        split = min(16 << 20, max(4 * 4 * 64 * (width + 2), pool // 4)) // 4 * 16  # four sequences, four query heads, 64 shares; or the pool
        assert rc == 0 and pool + split <= size <= pool + split + 32768, (kind, width, page, size - pool - split)
    assert null == [-1, -1, -1, -1, -1, -1, -1, 0]


def test_refusals_launch_nothing(host):  # noqa: F811
    rcs, launched, empty, launched_empty = host(CACHE + """
_, h = create()
stub.stub_clear()
rcs = {
  "negative n": L.nt_cache_reserve(h, -1, None, None, None),
  "too many": L.nt_cache_reserve(h, 5, None, None, None),
  "layer": L.nt_cache_write(h, 2, 1, None, None, 1, x, x, 128, 0, None),
  "negative layer": L.nt_cache_write(h, -1, 1, None, None, 1, x, x, 128, 0, None),
  "type": L.nt_cache_write(h, 0, 1, None, None, 1, x, x, 128, 3, None),
  "stride": L.nt_cache_write(h, 0, 1, None, None, 1, x, x, 127, 0, None),
  "max_new": L.nt_cache_write(h, 0, 1, None, None, 201, x, x, 128, 0, None),
  "no keys": L.nt_cache_write(h, 0, 1, None, None, 1, None, x, 128, 0, None),
  "struct_size": attend(h, struct_size=7),
  "window": attend(h, window=-1), "sinks": attend(h, sinks=-1), "max_keys": attend(h, max_keys=-1),
  "scale": attend(h, scale=float("nan")), "infinite scale": attend(h, scale=float("inf")),
  "q stride": attend(h, ld_q=255), "out stride": attend(h, ld_out=255), "kv stride": attend(h, k=x, v=x, ld_kv=127),
  "k alone": attend(h, k=x, ld_kv=128), "no q": attend(h, q=None), "no out": attend(h, out=None),
  "rows without d_first": attend(h, max_new=2), "attend layer": attend(h, layer=2), "attend type": attend(h, type=9), "attend n": attend(h, n=5),
  "read": L.nt_cache_read(h, 0, 1, None, 5, None, x, 0, None), "read max_keys": L.nt_cache_read(h, 0, 1, None, -1, x, x, 0, None),
  "fork": L.nt_cache_fork(h, 1, None, x, None), "copy": L.nt_cache_copy(h, 1, x, None, None),
  "trim window": L.nt_cache_trim(h, 1, None, 0, 0, None), "trim sinks": L.nt_cache_trim(h, 1, None, 1, -1, None),
}
launched = stub.stub_n_launches()
empty = [L.nt_cache_reserve(h, 0, None, None, None), L.nt_cache_write(h, 0, 0, None, None, 1, None, None, 0, 0, None), attend(h, n=0, q=None, out=None),
         attend(h, max_new=0, d_first=x), L.nt_cache_read(h, 0, 0, None, 5, None, None, 0, None), L.nt_cache_fork(h, 0, None, None, None),
         L.nt_cache_truncate(h, 0, None, None, None), L.nt_cache_trim(h, 0, None, 1, 0, None)]
print(json.dumps((rcs, launched, empty, stub.stub_n_launches())))
""")
    want = {"too many": -2, "attend n": -2, "layer": -6, "negative layer": -6, "max_new": -6, "attend layer": -6, "read max_keys": -6}
    assert {k: v for k, v in rcs.items() if v != want.get(k, -1)} == {}
    assert launched == 0 and empty == [0] * 8 and launched_empty == 0


@pytest.mark.parametrize("kind", [1, 2, 3])
def test_grids(host, kind):  # noqa: F811
    """No grid is empty or beyond what the kernels index, from one token to a million."""
    out = host(CACHE + f"""
_, h = create(kind={kind}, n_pages=1 << 14, max_len=1 << 20, max_seqs=4)
out = []
for n, new, keys in ((1, 1, 1), (4, 1, 0), (1, 1, 1 << 20), (4, 5000, 0), (2, 1 << 20, 0), (3, 2, 100)):
    stub.stub_clear()
    rc = attend(h, n=n, max_new=new, max_keys=keys, d_first=x if new > 1 else None, k=x, v=x, ld_kv=128)
    out.append((n, new, rc, launches()))
print(json.dumps(out))
""")
    for n, new, rc, launches in out:
        assert rc == 0
        for name, blocks in launches:
            assert 0 < blocks < 2 ** 31, (name, blocks)
        write = [b for name, b in launches if "cache_write" in name]
        assert write == ([((new + 30) // 32 + 1) * 2 * n] if new > 1 else [])  # a single token is written by the attention


def test_models_with_a_paged_self_cache(host):  # noqa: F811
    """Refusals, the configuration without the three fields (an older caller), device memory, and which launches a step makes."""
    codes, older, sizes, steps = host("""
from paper_2109_08003_amd.binding import NtConfig, lib, make_config
def rc(**kw):
    c, h = make_config(config(**kw), 4096), C.c_void_p()
    blob = np.zeros(int(lib().nt_param_count(C.byref(make_config(config(), 4096)))), dtype=np.float16)
    return lib().nt_load_weights(C.byref(c), blob.ctypes.data, blob.nbytes, None, C.byref(h))
codes = [rc(self_cache=4), rc(self_cache=-1), rc(self_window=5), rc(self_sinks=1), rc(self_cache="q4", self_window=-1), rc(self_cache="f16", self_sinks=-1)]
try:
    codes.append(load(config(self_cache="f16", rpr_clip=4)))
except nt.NtError as e:
    codes.append(e.code)
except AssertionError:
    codes.append("no blob")
c, h = make_config(config(), 4096), C.c_void_p()
c.struct_size = NtConfig.self_cache.offset
c.self_cache = 77                        # behind the caller's struct
blob = np.zeros(int(lib().nt_param_count(C.byref(c))), dtype=np.float16)
older = [lib().nt_load_weights(C.byref(c), blob.ctypes.data, blob.nbytes, None, C.byref(h)), c.self_cache, blob.size == nt.param_count(config())]
sizes = [load(config(self_cache=k, self_window=20), tokens=2048).device_bytes() for k in ("f16", "bf16", "q4")]
model = load(config(self_cache="q4", self_window=9, self_sinks=2, n_dec=2))
encode(model, 3, 10)
out = np.zeros((3, 5), dtype=np.int32)
steps = []
for _ in range(2):
    stub.stub_clear()
    nt.binding._check(lib().nt_decode_greedy(model._h, 3, 5, None, out.ctypes.data, None))
    names = [n for n, b in launches()]
    steps.append([sum(w in n for n in names) for w in ("cache_end", "cache_reserve", "cache_token", "cache_join", "dec1_kernel")])
print(json.dumps((codes, older, sizes, steps)))
""")
    assert codes == [-1, -1, -1, -1, -1, -1, -2]
    assert older == [0, 77, True]
    positions = (6 * 2048 + 4) // 5 + 3 * 2048 + 8
    pages = positions // 32 + 2048
    assert sizes[0] == sizes[1] and sizes[0] - sizes[2] == pages * 32 * 2 * (512 * 2 - 512 // 2 - 512 // 32)
    assert steps == [[0, 5, 10, 0, 0], [1, 5, 10, 0, 0]]


def test_binding_refuses_tensors_that_do_not_fit(host):  # noqa: F811
    """Host tensors, other devices, types, shapes and strides; nothing is launched."""
    kinds, launched = host("""
import torch
class Dev:  # a host tensor that says it is on a device
    def __init__(self, t, device=0):
        self.t, self.device = t, device
    def get_device(self):
        return self.device
    def __getattr__(self, name):
        return getattr(self.t, name)
c = nt.Cache("f16", 1, 4, 2, 64, 8, 4, 200, stream=Stream)
def t(*shape, dtype=torch.float16, device=0):
    return Dev(torch.zeros(shape, dtype=dtype), device)
q, out, k = t(3, 4, 64), t(3, 4, 64), t(3, 2, 64)
ids = t(3, dtype=torch.int32)
wide = Dev(torch.zeros(3, 4, 128, dtype=torch.float16)[:, :, ::2])
stub.stub_clear()
def kind(f):
    try:
        f()
        return "none"
    except (TypeError, nt.NtError) as e:
        return type(e).__name__
s = dict(stream=Stream)
kinds = [kind(f) for f in (
    lambda: c.attend(torch.zeros(3, 4, 64).half(), out, 3, **s), lambda: c.attend(t(3, 4, 64, device=1), out, 3, **s),
    lambda: c.attend(q, t(3, 4, 64, dtype=torch.float32), 3, **s), lambda: c.attend(t(3, 4, 64, dtype=torch.float64), t(3, 4, 64, dtype=torch.float64), 3, **s),
    lambda: c.attend(t(3, 5, 64), t(3, 5, 64), 3, **s), lambda: c.attend(wide, out, 3, **s), lambda: c.attend(q, t(2, 4, 64), 3, **s),
    lambda: c.attend(q, out, 4, **s), lambda: c.attend(q, out, **s), lambda: c.attend(q, out, 3, k=k, **s), lambda: c.attend(q, out, 3, k=k, v=t(2, 2, 64), **s),
    lambda: c.attend(q, out, seqs=t(3, dtype=torch.int64), **s), lambda: c.attend(q, out, 3, seqs=t(2, dtype=torch.int32), **s),
    lambda: c.attend(q, out, 3, first=ids, **s), lambda: c.write(k, t(3, 2, 64, dtype=torch.float32), 3, **s), lambda: c.write(k, k, 4, **s),
    lambda: c.read(t(3, 9, 2, 64), t(3, 8, 2, 64), 3, **s), lambda: c.read(t(2, 9, 2, 64), t(2, 9, 2, 64), 3, **s),
    lambda: c.fork(ids, t(2, dtype=torch.int32), **s), lambda: c.reserve(seqs=t(3, dtype=torch.int32, device=1), **s),
    lambda: c.attend(q, out, 3, window=-1, **s), lambda: c.reserve(5, **s))]
launched = stub.stub_n_launches()
c.attend(q, out, 3, k=k, v=k, **s)
print(json.dumps((kinds, (launched, stub.stub_n_launches()))))
""")
    assert kinds == ["TypeError"] * 20 + ["NtError"] * 2
    assert launched[0] == 0 < launched[1]
