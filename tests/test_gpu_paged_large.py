"""Caches and rotations of the sizes from which on loads and stores are nontemporal: more than 128 MB of keys and values, more than
256 MB written."""
import pytest
import torch

import paper_2508_04711_amd as hstu
from test_gpu_paged import DT, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,buckets,new", [("bf16", 0, 1), ("f32", 0, 2), ("bf16", 64, 1), ("f32", 64, 1), ("bf16", 0, 12), ("bf16", 64, 10)])
def test_caches_that_memory_side_caches_do_not_hold(dtype, buckets, new):
    """Few rows (1, 2), and many (10 and 12 a sequence: tiles of 128 pairs)."""
    rows = 16500 if dtype == "bf16" else 8300
    lens = [rows, rows - 1, rows + 17, 5, rows - 4000, rows + 3000, rows, rows, rows + 1]
    pr = Problem(dtype, lens, [new] * 4 + [0] + [new] * 4, 4, 4, 64, 64, 64, seed=new, buckets=buckets)
    assert 2 * pr.kp.numel() * pr.kp.element_size() > 128 << 20
    cache = pr.cache()
    need = hstu.hstu_paged_attn_workspace_bytes(cache, 4, pr.rows)
    assert (need >= 2 * 512 * 128 * 64 * 4) == (new > 8) and need > 256
    got = pr.call(cache, out_dtype=torch.float32)
    pr.check(got, one_term=None if new > 8 else False)
    assert torch.equal(got, pr.call(cache, out_dtype=torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_rotations_that_memory_side_caches_do_not_hold(dtype, inter):
    """Bit for bit what calls of fewer rows give, rows outside every sequence left alone."""
    heads, d, rotary = 9, 128, 96
    rows = (1 << 28) // (heads * d * (2 if dtype == "bf16" else 4)) + 1001
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, heads, d), generator=g, device="cuda").to(DT[dtype])
    assert x.numel() * x.element_size() > 256 << 20
    cuts = [0, 3, 3, 20000, 20001, rows - 30000, rows - 7]
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(b - a) for a, b in zip(cuts, cuts[1:])]).to(torch.int32).cuda()
    freq = hstu.hstu_rotary_frequencies(rotary, 1000.0)
    out = torch.full_like(x, 7.0)
    for fn in (hstu.hstu_rotary_fwd, hstu.hstu_rotary_bwd):
        fn([x], freq, seq_offsets=off, interleaved=inter, out=[out])
        assert (out[rows - 7:] == 7.0).all()
        for a in range(0, rows - 7, 20011):
            b = min(a + 20011, rows - 7)
            part, = fn([x[a:b]], freq, positions=pos[a:b].contiguous(), interleaved=inter)
            assert torch.equal(part, out[a:b])


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("f32", 1), ("bf16", 40)])
def test_pages_beyond_four_gigabytes(dtype, new):
    """Pages whose offsets pass 32 bits, K and V as halves of one buffer: the append and the attention of few and of many rows give what they
    give over a cache of the same pages alone."""
    ps, heads, d = 64, 4, 128
    pr = Problem(dtype, [1500, 64, 700], [new, new, new], heads, heads, d, d, ps, seed=new, fill=0.0)
    size = 2 if dtype == "bf16" else 4
    first = (5 << 30) // (2 * heads * ps * d * size)
    buf = torch.empty((first + pr.pages, 2, heads, ps, d), dtype=DT[dtype], device="cuda")
    buf[first:, 0], buf[first:, 1] = pr.kp.cuda(), pr.vp.cuda()
    small = pr.cache()
    large = hstu.HstuPagedCache(buf[:, 0], buf[:, 1], small.page_table + first, small.seq_lens)
    off, freq = torch.from_numpy(pr.off).cuda(), hstu.hstu_rotary_frequencies(d)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((pr.rows, heads, d), generator=g).to(DT[dtype]).cuda() for _ in range(2))
    qs = [hstu.hstu_cache_append(c, k, v, off, q=pr.q.cuda(), inv_freq=freq) for c in (small, large)]
    assert torch.equal(qs[0], qs[1])
    assert torch.equal(buf[first:, 0], small.k_pages) and torch.equal(buf[first:, 1], small.v_pages)
    # (the same division of the work: a hint that both caches are bounded by)
    want = hstu.hstu_paged_attn_fwd(qs[0], small, off, 1500, 0.1, max_kv=1500)
    got = hstu.hstu_paged_attn_fwd(qs[0], large, off, 1500, 0.1, max_kv=1500)
    assert torch.equal(got, want)
    pr.q, pr.kp, pr.vp, pr.alpha, pr.max_len = qs[0].cpu(), small.k_pages.cpu(), small.v_pages.cpu(), 0.1, 1500
    pr.check(got)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("f32", 3), ("bf16", 40)])
@pytest.mark.parametrize("ps", [4096, 32768])
def test_large_pages(dtype, new, ps):
    """The largest pages there are, histories that end anywhere in them."""
    pr = Problem(dtype, [ps + 77, 5, ps], [new, 2, new], 2, 2, 32, 64, ps, seed=ps, spare=1)
    cache = pr.cache()
    for causal in (True, False):
        pr.check(pr.call(cache, causal=causal), causal)
    off = torch.from_numpy(pr.off).cuda()
    k, v = torch.randn((pr.rows, 2, 32)).to(DT[dtype]).cuda(), torch.randn((pr.rows, 2, 64)).to(DT[dtype]).cuda()
    before = cache.k_pages.clone()
    hstu.hstu_cache_append(cache, k, v, off)
    at = 0
    for b, (n, m) in enumerate(zip(pr.lens, pr.new)):
        for p in range(n - m, n):
            pg, sl = int(pr.table[b, p // ps]), p % ps
            assert torch.equal(cache.k_pages[pg, :, sl], k[at]) and torch.equal(cache.v_pages[pg, :, sl], v[at])
            before[pg, :, sl] = k[at]
            at += 1
    assert torch.equal(torch.nan_to_num(before), torch.nan_to_num(cache.k_pages))
