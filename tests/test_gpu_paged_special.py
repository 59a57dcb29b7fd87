"""Infinities, NaN and probabilities at the end of the range in the attention over a paged cache: every output is what the definition
in float64 gives (oracle/serve.py), infinite with its sign, NaN or finite."""
import numpy as np
import pytest
import torch

from oracle import serve
from test_gpu_paged import Problem, _f64

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")

# One worker of several waves per tile; a wave per tile, uncut; tiles cut along the keys.
DIVISIONS = {
    "team": dict(lens=[90, 33], new=[5, 1], heads=2, kv_heads=1),
    "uncut": dict(lens=[90, 33] + [20] * 300, new=[5, 1] + [1] * 300, heads=2, kv_heads=2),
    "cut": dict(lens=[5000, 90], new=[5, 1], heads=2, kv_heads=1),
}


def _row(pr, pages, b, p):
    """Row p of sequence b in k_pages or v_pages: [kv_heads, d]."""
    return pages[pr.table[b, p // pr.ps], :, p % pr.ps]


def _check(pr, got, causal=True, one_term=None):
    with np.errstate(all="ignore"):
        o, sums = pr.want(causal)
        bf16 = pr.dtype == "bf16"
        tol = serve.attention_tolerance(o, sums, pr.q.shape[2], max(pr.lens), bf16, got.dtype == torch.bfloat16,
                                        bf16 if one_term is None else one_term)
        g = _f64(got)
        assert (np.isnan(g) == np.isnan(o)).all(), "NaN where there is none, or the other way round"
        assert ((g == INF) == (o == INF)).all() and ((g == -INF) == (o == -INF)).all()
        finite = np.isfinite(o)
        assert (np.abs(g - o)[finite] <= tol[finite]).all()
        return finite, o


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("division", list(DIVISIONS))
@pytest.mark.parametrize("out", [torch.float32, None])
def test_infinite_values(dtype, division, out):
    """Infinite values in rows that every new row sees and in rows that only some see: each output they reach is infinite, with the sign of
    the probability times the value's."""
    kw = DIVISIONS[division]
    for causal in (True, False):
        pr = Problem(dtype, dqk=64, dv=128, ps=16, seed=7, fill=NAN, **kw)
        n, m = pr.lens[0], pr.new[0]
        for p, element, value in ((3, 0, INF), (20, 1, -INF), (n - 40, 9, INF), (n - m + 2, 77, -INF), (n - 1, 127, INF)):
            _row(pr, pr.vp, 0, p)[:, element] = value
        _row(pr, pr.vp, 1, 32)[:, 5] = INF
        finite, o = _check(pr, pr.call(causal=causal, out_dtype=out), causal)
        assert (o == INF).any() and (o == -INF).any() and finite.any()
        if causal:  # (rows before the infinity stay finite in that element)
            assert finite[:2, :, 77].all() and not finite[2:m, :, 77].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("division", list(DIVISIONS))
def test_infinite_keys(dtype, division):
    """An infinite key makes an infinite probability where the query's element is positive (NaN where it is negative), and an infinite
    or finite value of its row an infinite output."""
    kw = DIVISIONS[division]
    pr = Problem(dtype, dqk=64, dv=64, ps=16, seed=11, fill=NAN, **kw)
    n, m = pr.lens[0], pr.new[0]
    pr.q[:m, :, 3] = pr.q[:m, :, 3].abs() + 0.125
    pr.q[0, -1, 3] = -1.0
    _row(pr, pr.kp, 0, 5)[:, 3] = INF
    _row(pr, pr.vp, 0, 5)[:, 8] = -INF
    _row(pr, pr.kp, 0, n - m + 3)[:, 3] = INF
    finite, o = _check(pr, pr.call(out_dtype=torch.float32))
    assert (o[:m] == INF).any() and (o[:m] == -INF).any() and np.isnan(o[0, -1]).all() and finite[m:].all()


@pytest.mark.parametrize("division", list(DIVISIONS))
def test_probabilities_that_only_round_to_infinity(division):
    """A finite probability beyond the largest bf16: two bf16 terms hold it all the same."""
    kw = DIVISIONS[division]
    pr = Problem("bf16", dqk=32, dv=32, ps=16, seed=3, fill=NAN, **kw)
    # (2 - 2^-7) 2^127 + 1.5 2^119 = 1.998 2^127, in fp32 finite
    pr.q[0, :, :] = 0.0
    pr.q[0, :, 0], pr.q[0, :, 1] = (2 - 2.0 ** -7) * 2.0 ** 63, 1.5 * 2.0 ** 59
    key, value = _row(pr, pr.kp, 0, 17), _row(pr, pr.vp, 0, 17)
    key[:] = 0.0
    key[:, 0], key[:, 1] = 2.0 ** 64, 2.0 ** 60
    value *= 2.0 ** -20
    finite, o = _check(pr, pr.call(out_dtype=torch.float32), one_term=False)
    assert finite.all() and np.abs(o[0]).max() > 1e24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("division", list(DIVISIONS))
def test_nan_values_reach_those_who_see_them(dtype, division):
    kw = DIVISIONS[division]
    pr = Problem(dtype, dqk=64, dv=64, ps=16, seed=5, fill=NAN, **kw)
    n, m = pr.lens[0], pr.new[0]
    clean, _ = pr.want()
    _row(pr, pr.vp, 0, n - m + 1)[:, 2] = NAN
    _row(pr, pr.kp, 0, n - m + 3)[:, 2] = NAN
    _check(pr, pr.call(out_dtype=torch.float32))
    _, o = _check(pr, pr.call())
    assert np.isnan(o[1:m, :, 2]).all() and np.isnan(o[3:m]).all() and not np.isnan(o[:3, :, 3]).any() and not np.isnan(clean).any()
