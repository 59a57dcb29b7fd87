"""Appends and the attention read the same wrong length or offset alike: lengths count as at least 0 and at most the table's room,
sequences end at the last row of the call."""
import numpy as np
import pytest
import torch

import paper_2508_04711_amd as hstu
from oracle import serve
from test_gpu_paged import DT, Problem, _f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_lengths_beyond_the_room(dtype, inter):
    """Histories that outgrow their tables by some rows, by very many, and a negative length: every row that has a place is
    written where the attention takes it to be, turned by that position."""
    ps, d, rotary = 16, 64, 64
    pr = Problem(dtype, [48, 48, 48, 40, 48, 48], [2, 1, 5, 2, 1, 3], 2, 2, d, d, ps, seed=9, fill=0.0)
    pr.width = 3
    pr.table = np.ascontiguousarray(pr.table[:, :3])                     # room for 48 rows
    pr.lens = [49, 1000, 48 + 5, -7, 2 ** 31 - 1, 47]
    cache, off = pr.cache(), torch.from_numpy(pr.off).cuda()
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((pr.rows, 2, d), generator=g).to(DT[dtype]) for _ in range(2))
    freq = hstu.hstu_rotary_frequencies(rotary, 100.0)
    before = [t.cpu().clone() for t in (cache.k_pages, cache.v_pages)]
    q = hstu.hstu_cache_append(cache, k.cuda(), v.cuda(), off, q=pr.q.cuda(), inv_freq=freq, interleaved=inter)
    lens = [min(max(n, 0), 48) for n in pr.lens]
    seq, pos = serve.positions(pr.off, pr.rows, lens)
    f = freq.cpu().numpy()
    want = serve.rotate(_f64(pr.q), pos, f, inter)
    tol = serve.rotation_tolerance(_f64(pr.q), want, rotary, inter, 1.0, dtype == "bf16")
    assert (np.abs(_f64(q) - want) <= tol).all()
    kw = serve.rotate(_f64(k), pos, f, inter)
    tol = serve.rotation_tolerance(_f64(k), kw, rotary, inter, 1.0, dtype == "bf16")
    kp, vp = cache.k_pages.cpu(), cache.v_pages.cpu()
    written = np.zeros((pr.pages, ps), dtype=bool)
    for r in range(pr.rows):
        at = serve.place(pr.table, pr.pages, ps, seq[r], int(pos[r]))
        assert (at is None) == (seq[r] == 3)
        if at is None:
            continue
        written[at] = True
        assert (np.abs(_f64(kp[at[0], :, at[1]]) - kw[r]) <= tol[r]).all() and torch.equal(vp[at[0], :, at[1]], v[r])
    rest = torch.from_numpy(~written)
    for old, new in zip(before, (kp, vp)):
        assert torch.equal(old.permute(0, 2, 1, 3)[rest], new.permute(0, 2, 1, 3)[rest])
    # the attention over what was written
    pr.kp, pr.vp, pr.q, pr.alpha, pr.max_len = kp, vp, q.cpu(), 0.125, 48
    pr.check(pr.call(cache, q))


def test_offsets_beyond_the_rows():
    """The last sequence says that it has more rows than the call: it has those that there are, for the append as for the attention."""
    pr = Problem("f32", [40, 33], [2, 3], 2, 2, 32, 32, 16, fill=0.0)
    cache, off = pr.cache(), torch.from_numpy(pr.off).cuda()
    other = pr.cache()
    far = off.clone()
    far[-1] += 7
    k, v = (torch.randn((pr.rows, 2, 32)).cuda() for _ in range(2))
    freq = hstu.hstu_rotary_frequencies(32)
    qs = [hstu.hstu_cache_append(c, k, v, o, q=pr.q.cuda(), inv_freq=freq) for c, o in ((cache, off), (other, far))]
    assert torch.equal(qs[0], qs[1]) and torch.equal(cache.k_pages, other.k_pages) and torch.equal(cache.v_pages, other.v_pages)
    outs = [hstu.hstu_paged_attn_fwd(qs[0], c, o, 40, 0.2) for c, o in ((cache, off), (other, far))]
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_with_timestamps_and_without_pages(dtype):
    """Rows have no places: queries are turned, keys and timestamps are dropped, and the attention with the bias gives zeros."""
    none = torch.empty((0, 2, 16, 64), dtype=DT[dtype], device="cuda")
    table = torch.zeros((3, 40), dtype=torch.int32, device="cuda")
    lens, off = torch.tensor([20, 500, 9], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 101, 102], dtype=torch.int32, device="cuda")
    cache = hstu.HstuPagedCache(none, none.clone(), table, lens, torch.empty((0, 16), dtype=torch.int32, device="cuda"))
    x = torch.ones((102, 2, 64), dtype=DT[dtype], device="cuda")
    ts = torch.arange(102, dtype=torch.int32, device="cuda")
    freq = hstu.hstu_rotary_frequencies(64)
    q = hstu.hstu_cache_append(cache, x, x, off, q=x, inv_freq=freq, timestamps=ts)
    pos = torch.cat((torch.tensor([19]), torch.arange(400, 500), torch.tensor([8]))).to(torch.int32).cuda()
    assert torch.equal(q, hstu.hstu_rotary_fwd([x], freq, positions=pos)[0])
    w = torch.randn(16, device="cuda")
    for causal in (True, False):
        assert (hstu.hstu_paged_attn_bias_fwd(q, cache, off, ts, w, 2, 500, 0.1, causal) == 0).all()
        assert (hstu.hstu_paged_attn_bias_fwd(q, cache, off, ts, w, 2, 500, 0.1, causal, max_kv=500) == 0).all()
