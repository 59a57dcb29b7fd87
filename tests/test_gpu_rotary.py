"""Rotary positions on the device against the definition in float64 (oracle/serve.py): both layouts, parts of heads, types,
strides, positions near and far, empty sequences, in place, the gradient, streams and captured calls."""
import numpy as np
import pytest
import torch

import paper_2508_04711_amd as hstu
from oracle import serve

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _values(shape, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype])


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _check(got, x, pos, freq, inter, scale, dtype, backward=False, rows=None):
    want = serve.rotate(_f64(x), pos, freq, inter, scale, backward)
    angle = float(np.abs(np.asarray(pos, dtype=np.float64)).max(initial=0.0) * np.abs(freq).max())
    tol = serve.rotation_tolerance(_f64(x), want, 2 * len(freq), inter, scale, dtype == "bf16", angle * 2.0 ** -51)
    err = np.abs(_f64(got) - want)
    rows = slice(None) if rows is None else rows
    assert (err[rows] <= tol[rows]).all(), float((err[rows] / np.maximum(tol[rows], 1e-300)).max())


LENGTHS = [[1], [3, 0, 0, 5, 1], [0, 0], [70, 1, 0, 300, 64], [1] * 130 + [0] * 70 + [2] * 3]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rotary", [(32, 16), (32, 32), (64, 48), (128, 128), (128, 16)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=[str(i) for i in range(len(LENGTHS))])
def test_forward_and_backward(dtype, inter, d, rotary, lengths):
    rows, off = sum(lengths), np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    freq = hstu.hstu_rotary_frequencies(rotary, 500.0, "linear", 2.0)
    f = freq.cpu().numpy()
    _, pos = serve.positions(off, rows)
    # two tensors with different numbers of heads, one of them more than a thread does at once
    x = [_values((rows, h, d), dtype, h) for h in (2, 9)]
    dev = [t.cuda() for t in x]
    do = torch.from_numpy(off).cuda()
    for backward, fn in ((False, hstu.hstu_rotary_fwd), (True, hstu.hstu_rotary_bwd)):
        out = fn(dev, freq, seq_offsets=do, interleaved=inter, scale=1.25)
        for t, g in zip(x, out):
            _check(g, t, pos, f, inter, 1.25, dtype, backward)
            assert torch.equal(g[:, :, rotary:].cpu(), t[:, :, rotary:])
    again = hstu.hstu_rotary_fwd(dev, freq, seq_offsets=do, interleaved=inter, scale=1.25)
    first = hstu.hstu_rotary_fwd(dev, freq, positions=torch.from_numpy(pos.astype(np.int32)).cuda(), interleaved=inter, scale=1.25)
    assert all(torch.equal(a, b) for a, b in zip(again, first))
    hstu.hstu_rotary_fwd(dev, freq, seq_offsets=do, interleaved=inter, scale=1.25, out=dev)  # in place
    assert all(torch.equal(a, b) for a, b in zip(again, dev))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    pos = np.array([0, -1, 1, 1 << 20, (1 << 31) - 1, -(1 << 31), 123456789, -77777], dtype=np.int32)
    freq = hstu.hstu_rotary_frequencies(128)
    x = _values((len(pos), 3, 128), dtype)
    for inter in (False, True):
        got, = hstu.hstu_rotary_fwd([x.cuda()], freq, positions=torch.from_numpy(pos).cuda(), interleaved=inter)
        for i in range(len(pos)):  # (each position with the tolerance of its own angle)
            _check(got[i:i + 1], x[i:i + 1], pos[i:i + 1], freq.cpu().numpy(), inter, 1.0, dtype)


def test_gradient_is_the_transpose():
    """sum(g * fwd(x)) = sum(bwd(g) * x): both calls in fp32, against the sums' own rounding."""
    x, g = (_values((50, 4, 64), "f32", s).cuda() for s in (1, 2))
    off = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    freq = hstu.hstu_rotary_frequencies(64)
    for inter in (False, True):
        y, = hstu.hstu_rotary_fwd([x], freq, seq_offsets=off, interleaved=inter, scale=0.7)
        b, = hstu.hstu_rotary_bwd([g], freq, seq_offsets=off, interleaved=inter, scale=0.7)
        left, right = (y.double() * g.double()).sum(), (b.double() * x.double()).sum()
        # every y, b is off by at most 4 u (|x_a| + |x_b|) 0.7
        bound = 2 * 4 * serve.U32 * 0.7 * 2 * (x.abs().double().max() * g.abs().double().sum()).item()
        assert abs(left - right).item() <= bound


def test_slices_of_a_projection_and_rows_outside():
    """q and k as slices of one fused buffer; rows behind the last sequence stay as they were."""
    rows, h, d = 40, 3, 64
    fused = _values((rows, 4 * h * d), "bf16").cuda()
    q, k = (fused[:, i * h * d:(i + 1) * h * d].view(rows, h, d) for i in (1, 3))
    off = torch.tensor([0, 7, 7, 33], dtype=torch.int32, device="cuda")
    freq = hstu.hstu_rotary_frequencies(32)
    want = hstu.hstu_rotary_fwd([q.contiguous(), k.contiguous()], freq, seq_offsets=off)
    before = fused.clone()
    out = [torch.full((rows, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    hstu.hstu_rotary_fwd([q, k], freq, seq_offsets=off, out=out)
    assert torch.equal(fused, before)
    for o, w in zip(out, want):
        assert torch.equal(o[:33], w[:33]) and (o[33:] == 7.0).all()
    hstu.hstu_rotary_fwd([q, k], freq, seq_offsets=off, out=[q, k])  # in place in the fused buffer
    assert torch.equal(q[:33], want[0][:33]) and torch.equal(k[:33], want[1][:33])
    after, old = fused.view(rows, 4, h, d), before.view(rows, 4, h, d)
    assert torch.equal(after[:, 0], old[:, 0]) and torch.equal(after[:, 2], old[:, 2]) and torch.equal(after[33:], old[33:])


def test_many_sequences():
    """More sequences than one and two steps of the search see."""
    rng = np.random.default_rng(3)
    lengths = rng.choice([0, 0, 1, 2, 5], size=9000)
    rows, off = int(lengths.sum()), np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    _, pos = serve.positions(off, rows)
    x = _values((rows, 1, 32), "f32")
    freq = hstu.hstu_rotary_frequencies(32)
    got, = hstu.hstu_rotary_fwd([x.cuda()], freq, seq_offsets=torch.from_numpy(off).cuda())
    _check(got, x, pos, freq.cpu().numpy(), False, 1.0, "f32")


def test_streams_and_captured_calls():
    x = _values((100, 4, 128), "bf16").cuda()
    off = torch.tensor([0, 60, 100], dtype=torch.int32, device="cuda")
    freq = hstu.hstu_rotary_frequencies(128)
    want = hstu.hstu_rotary_fwd([x], freq, seq_offsets=off)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hstu.hstu_rotary_fwd([x], freq, seq_offsets=off, stream=s)[0]
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    out = torch.empty_like(x)
    with torch.cuda.graph(g):
        hstu.hstu_rotary_fwd([x], freq, seq_offsets=off, out=[out])
    for new in ([0, 60, 100], [0, 10, 100], [0, 0, 100]):  # (the offsets are read when the graph runs)
        off.copy_(torch.tensor(new, dtype=torch.int32))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, hstu.hstu_rotary_fwd([x], freq, seq_offsets=off)[0])


def test_refusals():
    x = torch.zeros((4, 2, 32), device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    freq = hstu.hstu_rotary_frequencies(32)
    for bad in (dict(tensors=[x.half()]), dict(tensors=[x, x[:3]]), dict(tensors=[x, x.bfloat16()]), dict(tensors=[x] * 5),
                dict(inv_freq=freq.float()), dict(inv_freq=freq.cpu()), dict(seq_offsets=None), dict(seq_offsets=off.long()),
                dict(positions=torch.zeros(4, dtype=torch.int32, device="cuda")), dict(out=[x[:, :1]]), dict(out=[x, x]),
                dict(tensors=[x.transpose(0, 1)]), dict(tensors=[x.cpu()]), dict(seq_offsets=off.cpu())):
        kw = dict(tensors=[x], inv_freq=freq, seq_offsets=off)
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hstu.hstu_rotary_fwd(kw.pop("tensors"), kw.pop("inv_freq"), **kw)
    with pytest.raises(hstu.HstuError):
        hstu.hstu_rotary_fwd([x], hstu.hstu_rotary_frequencies(64), seq_offsets=off)  # more than the head has
