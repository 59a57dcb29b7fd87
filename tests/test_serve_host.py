"""Rotary positions, the paged cache and the attention over it: what is refused on the host before anything touches the
device, the frequencies, and the oracle's pins (against the attention oracle, and by differences).  CPU only."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import oracle
from oracle import serve


@pytest.fixture(scope="module")
def lib():
    from paper_2508_04711_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2508_04711_amd import build
        build.build()
    return binding.load_library()


FAKE = 0x1000  # never dereferenced: every call below fails validation first


def _cache(**kw):
    from paper_2508_04711_amd import binding
    v = dict(batch=2, num_kv_heads=2, d_qk=64, d_v=32, page_size=16, pages_per_seq=4, dtype=0, reserved=0, num_pages=8,
             k_page_stride=2 * 16 * 64, v_page_stride=2 * 16 * 32, table_stride=4, k_pages=FAKE, v_pages=FAKE, ts_pages=None,
             page_table=FAKE, seq_lens=FAKE)
    v.update(kw)
    return binding._PagedCache(*[v[n] for n, _ in binding._PagedCache._fields_])


def _rotary(freq=FAKE, dim=32, inter=0, scale=1.0, reserved=0):
    from paper_2508_04711_amd import binding
    return binding._RotaryDesc(freq, dim, inter, scale, reserved)


def _tensor(src=FAKE, dst=FAKE, ss=128, ds=128, heads=2, dim=64):
    from paper_2508_04711_amd import binding
    return binding._RotaryTensor(src, dst, ss, ds, heads, dim)


BAD_CACHES = [
    (dict(batch=-1), -2), (dict(num_kv_heads=0), -2), (dict(num_kv_heads=1 << 20), -2), (dict(pages_per_seq=-1), -2),
    (dict(num_pages=-1), -2), (dict(num_pages=1 << 31), -2), (dict(table_stride=3), -2), (dict(d_qk=48), -3),
    (dict(d_v=96), -3), (dict(dtype=5), -3), (dict(reserved=1), -3), (dict(page_size=8), -3), (dict(page_size=24), -3),
    (dict(page_size=65536), -3), (dict(k_page_stride=2 * 16 * 64 - 8), -2), (dict(k_page_stride=2 * 16 * 64 + 4), -2),
    (dict(v_page_stride=8), -2),
]
BAD_CACHE_POINTERS = [(dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(page_table=None), -1),
                      (dict(seq_lens=None), -1), (dict(k_pages=FAKE + 8), -7), (dict(v_pages=FAKE + 4), -7)]


def test_rotary_refusals(lib):
    def call(r=None, tensors=(None,), dtype=0, batch=2, rows=10, n=None, pos=None, off=FAKE):
        from paper_2508_04711_amd import binding
        r = _rotary() if r is None else r
        ts = [_tensor() if t is None else t for t in tensors]
        arr = (binding._RotaryTensor * 8)(*ts)
        return lib.hstu_rotary(ctypes.byref(r), 0, dtype, batch, rows, len(ts) if n is None else n, arr, pos, off, None)
    assert lib.hstu_rotary(None, 0, 0, 2, 10, 1, ctypes.byref(_tensor()), None, FAKE, None) == -1
    assert lib.hstu_rotary(ctypes.byref(_rotary()), 0, 0, 2, 10, 1, None, None, FAKE, None) == -1
    assert call(batch=-1) == -2 and call(rows=-1) == -2 and call(rows=1 << 31) == -2
    assert call(n=0) == -2 and call(tensors=(None,) * 5) == -2
    assert call(dtype=2) == -3
    for dim in (0, 8, 24, -16, 80):
        assert call(r=_rotary(dim=dim)) == -2, dim
    assert call(r=_rotary(scale=math.inf)) == -2 and call(r=_rotary(reserved=1)) == -3
    assert call(r=_rotary(freq=None)) == -1 and call(r=_rotary(freq=FAKE + 4)) == -7
    assert call(tensors=(_tensor(heads=0),)) == -2 and call(tensors=(_tensor(dim=40),)) == -3
    assert call(tensors=(_tensor(ss=120),)) == -2            # rows overlap
    assert call(tensors=(_tensor(ds=132),)) == -2            # rows not on 16 bytes
    assert call(tensors=(_tensor(ss=256),)) == -2            # in place with two strides
    assert call(tensors=(_tensor(src=None),)) == -1 and call(tensors=(_tensor(dst=None),)) == -1
    assert call(tensors=(_tensor(src=FAKE + 8),)) == -7
    assert call(tensors=(None, _tensor(dst=FAKE + 2))) == -7
    assert call(off=None) == -1
    x, y = 0x100000, 0x200000                                # one tensor into the other's place
    assert call(tensors=(_tensor(src=x, dst=y), _tensor(src=y, dst=x))) == -2
    assert call(tensors=(_tensor(src=x, dst=y), _tensor(src=0x300000, dst=y))) == -2
    assert call(rows=0, off=None) == 0 and call(batch=0) == 0   # nothing to do


def test_append_refusals(lib):
    def call(c=None, r=None, rows=10, q=None, k=FAKE, ks=128, v=FAKE, vs=64, ts=None, off=FAKE):
        c = _cache() if c is None else c
        return lib.hstu_cache_append(ctypes.byref(c), ctypes.byref(r) if r is not None else None, rows,
                                     ctypes.byref(q) if q is not None else None, k, ks, v, vs, ts, off, None)
    assert lib.hstu_cache_append(None, None, 10, None, FAKE, 128, FAKE, 64, None, FAKE, None) == -1
    for kw, status in BAD_CACHES + BAD_CACHE_POINTERS:
        assert call(c=_cache(**kw)) == status, kw
    assert call(rows=-1) == -2 and call(rows=1 << 31) == -2
    assert call(ks=120) == -2 and call(vs=68) == -2
    assert call(r=_rotary(dim=80)) == -2 and call(r=_rotary(freq=None)) == -1
    assert call(q=_tensor(dim=32)) == -2 and call(q=_tensor(src=None)) == -1 and call(q=_tensor(dst=FAKE + 8)) == -7
    assert call(k=None) == -1 and call(v=None) == -1 and call(off=None) == -1 and call(k=FAKE + 4) == -7
    assert call(ts=FAKE) == -1                                   # timestamps that the cache has no room for
    assert call(c=_cache(ts_pages=FAKE)) == -1                   # ... and a cache whose timestamps are not given
    assert call(rows=0, k=None) == 0 and call(c=_cache(batch=0), k=None) == 0
    for kw in (dict(k=0x200000), dict(v=0x200000)):              # q's output over rows that are still read
        assert call(q=_tensor(src=0x100000, dst=0x200000, ss=128, ds=128), **kw) == -2


def test_attention_refusals(lib):
    from paper_2508_04711_amd import binding

    def params(heads=4, max_len=16, alpha=0.1, causal=1, out=0, max_kv=0, rows=10):
        return binding._PagedParams(heads, max_len, alpha, causal, out, max_kv, rows)

    def call(p=None, c=None, bias=None, q=FAKE, qs=256, off=FAKE, o=FAKE, ws=FAKE, size=1 << 30):
        p, c = params() if p is None else p, _cache() if c is None else c
        return lib.hstu_paged_attn_fwd(ctypes.byref(p), ctypes.byref(c), ctypes.byref(bias) if bias is not None else None,
                                       q, qs, off, o, ws, size, None)
    need = lambda p, c: lib.hstu_paged_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(c))
    assert lib.hstu_paged_attn_fwd(None, ctypes.byref(_cache()), None, FAKE, 256, FAKE, FAKE, FAKE, 1, None) == -1
    assert lib.hstu_paged_attn_fwd(ctypes.byref(params()), None, None, FAKE, 256, FAKE, FAKE, FAKE, 1, None) == -1
    for kw, status in BAD_CACHES + BAD_CACHE_POINTERS:
        assert call(c=_cache(**kw)) == status, kw
    for kw, _ in BAD_CACHES:
        assert need(params(), _cache(**kw)) == 0, kw
    for kw, status in [(dict(heads=0), -2), (dict(heads=3), -2), (dict(max_len=0), -2), (dict(alpha=math.nan), -2),
                       (dict(max_kv=-1), -2), (dict(rows=-1), -2), (dict(rows=1 << 31), -2), (dict(rows=(1 << 30) - 100), -2),
                       (dict(out=2), -3)]:
        assert call(p=params(**kw)) == status, kw
        assert need(params(**kw), _cache()) == 0, kw
    assert call(p=params(out=0), c=_cache(dtype=1)) == -3       # fp32 in, bf16 out
    assert call(qs=248) == -2 and call(qs=260) == -2
    assert call(q=None) == -1 and call(o=None) == -1 and call(ws=None) == -1 and call(off=None) == -1
    assert call(q=FAKE + 8) == -7 and call(o=FAKE + 8) == -7 and call(ws=FAKE + 8) == -7
    # long histories are cut: the call needs room for the parts
    big = _cache(pages_per_seq=1 << 10, table_stride=1 << 10)
    assert need(params(), big) > 256
    assert call(c=big, size=need(params(), big) - 1) == -4
    # a bound on the lengths that says they are short: nothing is cut
    assert need(params(max_kv=100), big) == 256
    bias = lambda ts=FAKE, w=FAKE, nb=16, f=2: binding._TsBias(ts, w, None, nb, f)
    with_ts = _cache(ts_pages=FAKE)
    assert call(c=with_ts, bias=bias(nb=0)) == -2 and call(c=with_ts, bias=bias(nb=513)) == -2
    assert call(c=with_ts, bias=bias(f=-1)) == -2 and call(c=with_ts, bias=bias(f=9)) == -2
    assert call(c=with_ts, bias=bias(ts=None)) == -1 and call(c=with_ts, bias=bias(w=None)) == -1
    assert call(bias=bias()) == -1                               # the cache holds no timestamps
    assert call(p=params(rows=0), q=None) == 0 and call(c=_cache(batch=0), q=None) == 0


def test_binding_refusals():
    import paper_2508_04711_amd as hstu
    x = torch.zeros((4, 2, 32))
    with pytest.raises(ValueError):
        hstu.hstu_rotary_fwd([x], torch.zeros(8, dtype=torch.float64), seq_offsets=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        hstu.hstu_rotary_fwd([], torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        hstu.HstuPagedCache(torch.zeros((2, 2, 16, 32)), torch.zeros((2, 2, 16, 32)), torch.zeros((1, 2), dtype=torch.int32),
                            torch.zeros(1, dtype=torch.int32))


def test_frequencies():
    import paper_2508_04711_amd as hstu
    f = lambda *a, **k: hstu.hstu_rotary_frequencies(*a, device="cpu", **k).numpy()
    j = np.arange(32)
    plain = 10000.0 ** (-2.0 * j / 64)
    assert np.allclose(f(64), plain, rtol=1e-15)
    assert np.allclose(f(64, scaling="linear", factor=8.0), plain / 8, rtol=1e-15)
    raised = f(64, scaling="base", factor=8.0)
    assert raised[0] == 1.0 and math.isclose(raised[-1], plain[-1] / 8, rel_tol=1e-12)
    parts = f(64, scaling="by_parts", factor=8.0, trained_len=4096)
    turns = 4096 * plain / (2 * math.pi)
    assert np.all(parts[turns >= 32] == plain[turns >= 32])
    assert np.allclose(parts[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and np.all((parts[mid] < plain[mid]) & (parts[mid] > plain[mid] / 8))
    for bad in (dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=32, scaling="other"),
                dict(rotary_dim=32, factor=0.0), dict(rotary_dim=32, scaling="by_parts")):
        with pytest.raises(ValueError):
            hstu.hstu_rotary_frequencies(device="cpu", **bad)


def test_oracle_rotation():
    rng = np.random.default_rng(0)
    freq = 100.0 ** (-2.0 * np.arange(4) / 8)
    for inter in (False, True):
        x, g = rng.standard_normal((5, 2, 12)), rng.standard_normal((5, 2, 12))
        pos = np.array([0, 1, 7, 100, 5])
        y = serve.rotate(x, pos, freq, inter, 1.5)
        assert np.allclose(y[0, :, :8], 1.5 * x[0, :, :8]) and np.all(y[:, :, 8:] == x[:, :, 8:])
        # lengths of pairs, and products of two rows, depend on the distance of their positions alone
        assert np.allclose((y[:, :, :8] ** 2).sum(-1), 2.25 * (x[:, :, :8] ** 2).sum(-1))
        z = serve.rotate(x, pos + 13, freq, inter, 1.5)
        assert np.allclose((y[2, :, :8] * y[3, :, :8]).sum(-1), (z[2, :, :8] * z[3, :, :8]).sum(-1))
        # the gradient of sum(y g), by differences (the map is linear: exact up to rounding)
        grad = serve.rotate(g, pos, freq, inter, 1.5, backward=True)
        for idx in [(0, 0, 0), (2, 1, 3), (3, 0, 6), (4, 1, 10)]:
            d = np.zeros_like(x)
            d[idx] = 1.0
            diff = ((serve.rotate(x + d, pos, freq, inter, 1.5) - serve.rotate(x - d, pos, freq, inter, 1.5)) * g).sum() / 2
            assert math.isclose(diff, grad[idx], rel_tol=1e-9, abs_tol=1e-9)


@pytest.mark.parametrize("causal", [True, False])
def test_oracle_attention_over_whole_histories_is_the_attention_oracle(causal):
    """All rows new: the paged attention is the jagged one."""
    rng = np.random.default_rng(1)
    lens, ps, heads, d = [5, 0, 33, 16], 16, 2, 8
    rows, off = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (rng.standard_normal((rows, heads, d)) for _ in range(3))
    table = rng.permutation(12).reshape(4, 3)
    kp, vp = np.full((12, heads, ps, d), np.nan), np.full((12, heads, ps, d), np.nan)
    for b, n in enumerate(lens):
        for p in range(n):
            g, s = serve.place(table, 12, ps, b, p)
            kp[g, :, s], vp[g, :, s] = k[off[b] + p], v[off[b] + p]
    o, _ = serve.attention(q, kp, vp, table, lens, off, 40, 0.3, causal)
    want = oracle.fwd(q, k, v, off.astype(np.int32), 40, 0.3, causal)
    assert np.allclose(o, want, rtol=1e-12, atol=1e-14)
    ts = np.sort(rng.integers(0, 100000, size=rows)).astype(np.int32)
    w = rng.standard_normal(24)
    tp = np.zeros((12, ps), dtype=np.int32)
    for b, n in enumerate(lens):
        for p in range(n):
            g, s = serve.place(table, 12, ps, b, p)
            tp[g, s] = ts[off[b] + p]
    o, _ = serve.attention(q, kp, vp, table, lens, off, 40, 0.3, causal, ts, tp, w, 2)
    want = oracle.bias_attention(q, k, v, v, off.astype(np.int32), ts, w, 2, 40, 0.3, causal)[0]
    assert np.allclose(o, want, rtol=1e-12, atol=1e-14)
