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
