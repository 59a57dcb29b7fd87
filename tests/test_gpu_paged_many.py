"""The kernel of many new rows (tiles of 128 pairs, bf16) at every pair of head dimensions, with pages smaller than a tile of keys, as
large and larger, causal or not, with the timestamp bias, and with infinities and NaN among the values.  Every call here is
asserted to be that kernel's, with its tiles cut along the keys."""
import numpy as np
import pytest
import torch

import paper_2508_04711_amd as hstu
from test_gpu_paged import NAN, Problem
from test_gpu_paged_special import INF, _check, _row

pytestmark = pytest.mark.gpu

DIMS = [(a, b) for a in (32, 64, 128) for b in (32, 64, 128)]
HEADS, KV_HEADS = 4, 2


def _problem(dqk, dv, ps, causal, buckets=0, seed=0, new0=150, **kw):
    """A history of more keys than 64 small pages hold, one that ends inside a tile, two of a few rows; tables with room for so many keys that
    no tile is a single worker's."""
    pr = Problem("bf16", [1301, 300, 3, 0, 64], [new0, 41, 3, 0, 64] if causal else [41, 150, 1, 2, 64], HEADS, KV_HEADS, dqk, dv, ps,
                 seed=seed, fill=NAN, buckets=buckets, **kw)
    room = -(-(1 << 19) // ((dqk + dv) * 2 * ps)) + 1
    wide = np.random.default_rng(seed).integers(0, pr.pages, size=(5, max(room, pr.width))).astype(np.int32)
    wide[:, :pr.width] = pr.table
    pr.table, pr.width = wide, wide.shape[1]
    return pr


def _many(pr, cache, **kw):
    """The call, after making sure that it is the kernel's: its partial results are tiles of 128 pairs, two of each of 512 workgroups or more."""
    need = hstu.hstu_paged_attn_workspace_bytes(cache, HEADS, pr.rows)
    assert need >= 2 * 512 * 128 * pr.vp.shape[3] * 4
    return pr.call(cache, **kw)


@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("ps", [16, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_against_the_definition(dqk, dv, ps, causal):
    pr = _problem(dqk, dv, ps, causal, seed=ps + dqk + dv)
    cache = pr.cache()
    got = _many(pr, cache, causal=causal, out_dtype=torch.float32)
    pr.check(got, causal)
    assert torch.equal(got, _many(pr, cache, causal=causal, out_dtype=torch.float32))
    ws = torch.empty(hstu.hstu_paged_attn_workspace_bytes(cache, HEADS, pr.rows), dtype=torch.uint8, device="cuda")
    ws.fill_(0xff)
    assert torch.equal(pr.call(cache, causal=causal, out_dtype=torch.float32, workspace=ws), got)


@pytest.mark.parametrize("dqk,dv", DIMS)
@pytest.mark.parametrize("ps", [16, 64])
def test_bias(dqk, dv, ps):
    for causal, buckets in ((True, 64), (False, 512)):
        pr = _problem(dqk, dv, ps, causal, buckets, seed=ps + 2 * dqk + dv)
        pr.check(_many(pr, pr.cache(), causal=causal), causal)


@pytest.mark.parametrize("ps", [16, 64, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_that_do_not_exist(ps, causal):
    """Wrong ids inside a history and at its end: their rows count as zeros, the tiles around them as they are."""
    pr = _problem(64, 64, ps, causal, seed=ps)
    pr.table[0, 1], pr.table[0, 1300 // ps] = -1, pr.pages
    pr.table[1, 299 // ps] = -(1 << 31)
    pr.check(_many(pr, pr.cache(), causal=causal), causal)


@pytest.mark.parametrize("dqk,dv", [(32, 32), (128, 128), (64, 128), (128, 32)])
@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("causal", [True, False])
def test_infinities_and_nan(dqk, dv, ps, causal):
    """In rows that all new rows see and, causal, in rows that only some of a tile's see: they reach those that see them, as what the
    definition makes of them."""
    pr = _problem(dqk, dv, ps, causal, seed=5)
    n, m = pr.lens[0], pr.new[0]
    for p, element, value in ((7, 0, INF), (700, 1, -INF), (n - 1, 2, INF), (n - 40, 3, -INF), (n - 41, 30, NAN), (n - 3, 4, NAN)):
        _row(pr, pr.vp, 0, p)[:, element] = value
    _row(pr, pr.vp, 1, 299)[0, 5] = -INF
    pr.q[:m, :, 6] = pr.q[:m, :, 6].abs() + 0.125
    _row(pr, pr.kp, 0, n - 2)[:, 6] = INF       # an infinite probability of the last two new rows
    pr.q[m - 1, 0, 6] = -1.0
    finite, o = _check(pr, _many(pr, pr.cache(), causal=causal), causal)
    if causal:
        assert finite[:m - 41, :, [2, 3, 4, 30]].all() and not finite[m - 40:m, :, 30].any()
        assert np.isnan(o[m - 1, 0]).all() and (o == INF).any() and (o == -INF).any()


@pytest.mark.parametrize("batch", [40, 300])
def test_offsets_that_do_not_ascend(batch):
    """Every second sequence says that all rows are its own, with the sums over the batch worked out by every workgroup or once: the call ends,
    nothing is written outside o, and the next call is right."""
    rows = 2600
    pr = _problem(64, 64, 16, True)
    cache = pr.cache()
    table = torch.from_numpy(np.resize(pr.table, (batch, pr.width))).cuda()
    wrong = hstu.HstuPagedCache(cache.k_pages, cache.v_pages, table, torch.full((batch,), 300, dtype=torch.int32, device="cuda"))
    assert hstu.hstu_paged_attn_workspace_bytes(wrong, HEADS, rows) >= 2 * 512 * 128 * 64 * 4
    off = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    off[1::2] = rows
    buf = torch.full((rows + 128, HEADS, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((rows, HEADS, 64), dtype=torch.bfloat16, device="cuda")
    for causal in (True, False):
        hstu.hstu_paged_attn_fwd(q, wrong, off, 300, 0.1, causal, out=buf[64:64 + rows])
    assert (buf[:64] == 7).all() and (buf[64 + rows:] == 7).all()
    pr.check(_many(pr, cache))


@pytest.mark.parametrize("batch", [5, 140])
def test_captured(batch):
    """Captured once and replayed while lengths change, the sums over the batch worked out by every workgroup or once, with eager work and
    another workspace's calls in between."""
    lens, new = [1301, 300, 64, 700, 40] + [30] * (batch - 5), [150, 41, 64, 12, 40] + [11] * (batch - 5)
    pr = Problem("bf16", lens, new, HEADS, KV_HEADS, 64, 64, 16, seed=batch, fill=0.0)
    pr.table = np.pad(pr.table, ((0, 0), (0, 200)), constant_values=-1)
    pr.width = pr.table.shape[1]
    cache, off, q = pr.cache(), torch.from_numpy(pr.off).cuda(), pr.q.cuda()
    need = hstu.hstu_paged_attn_workspace_bytes(cache, HEADS, pr.rows)
    assert need >= 2 * 512 * 128 * 64 * 4
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    hstu.hstu_paged_attn_fwd(q, cache, off, pr.max_len, pr.alpha)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hstu.hstu_paged_attn_fwd(q, cache, off, pr.max_len, pr.alpha, out=out, workspace=ws)
    for i in range(4):
        now = torch.tensor([max(n - 37 * i, 0) for n in lens], dtype=torch.int32)
        cache.seq_lens.copy_(now)
        q.normal_()
        out.fill_(NAN)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(hstu.hstu_paged_attn_fwd(q, cache, off, pr.max_len, pr.alpha), got)
        ws.fill_(0xff)
        pr.lens, pr.q = [int(n) for n in now], q.cpu()
        pr.check(got)


def test_two_streams_at_once():
    prs = [_problem(64, 64, 16, True, seed=s) for s in (1, 2)]
    caches, qs = [p.cache() for p in prs], [p.q.cuda() for p in prs]
    off = torch.from_numpy(prs[0].off).cuda()
    want = [hstu.hstu_paged_attn_fwd(q, c, off, p.max_len, p.alpha) for q, c, p in zip(qs, caches, prs)]
    streams = [torch.cuda.Stream() for _ in prs]
    torch.cuda.synchronize()
    got = [[hstu.hstu_paged_attn_fwd(qs[i], caches[i], off, prs[i].max_len, prs[i].alpha, stream=s) for i, s in enumerate(streams)]
           for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(w, g) for pair in got for w, g in zip(want, pair))
