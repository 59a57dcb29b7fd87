"""Few new rows in bf16 keep their probabilities in two bf16 terms: before the output's rounding, results are off by 2^-16 of
the sum of |p| |v| and by the rounding of fp32 sums (serve.attention_tolerance without its one term).  In every division of the work,
with and without the timestamp bias; a dropped second term is some 2^-10 of the sum and fails."""
import numpy as np
import pytest
import torch

import paper_2508_04711_amd as hstu
from oracle import serve
from test_gpu_paged import NAN, Problem, _f64
from test_gpu_paged_special import DIVISIONS, INF, _check, _row

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dqk,dv", [(32, 32), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("division", list(DIVISIONS))
@pytest.mark.parametrize("buckets", [0, 64])
def test_two_terms(dtype, dqk, dv, division, buckets):
    for ps, causal in ((16, True), (64, False)):
        pr = Problem(dtype, dqk=dqk, dv=dv, ps=ps, seed=dqk + ps, buckets=buckets, **DIVISIONS[division])
        cache = pr.cache()
        need = hstu.hstu_paged_attn_workspace_bytes(cache, pr.q.shape[1], pr.rows)
        assert (need > 256) == (division == "cut")
        pr.check(pr.call(cache, causal=causal, out_dtype=torch.float32), causal, one_term=False)


@pytest.mark.parametrize("division", list(DIVISIONS))
def test_two_terms_beside_an_infinity(division):
    """Elements that an infinity does not reach keep both terms."""
    pr = Problem("bf16", dqk=64, dv=64, ps=16, seed=2, fill=NAN, **DIVISIONS[division])
    n, m = pr.lens[0], pr.new[0]
    _row(pr, pr.vp, 0, n - m + 1)[:, 3] = INF
    _row(pr, pr.vp, 0, 4)[:, 60] = -INF
    finite, _ = _check(pr, pr.call(out_dtype=torch.float32), one_term=False)
    assert finite.any() and not finite[1:m, :, 3].any()


def test_the_tolerance_sees_a_dropped_term():
    """The same check on the definition with probabilities rounded to one bf16 term (on the host): it fails."""
    pr = Problem("bf16", dqk=64, dv=64, ps=16, seed=80, **DIVISIONS["team"])
    o, sums = pr.want()
    tol = serve.attention_tolerance(o, sums, 64, max(pr.lens), True, False, False)
    one = np.zeros_like(o)
    q, kp, vp = _f64(pr.q), _f64(pr.kp), _f64(pr.vp)
    for b, (n, m) in enumerate(zip(pr.lens, pr.new)):
        pg, sl = pr.table[b, np.arange(n) // 16], np.arange(n) % 16
        for i in range(m):
            r, seen = int(pr.off[b]) + i, slice(0, n - m + i + 1)
            for h in range(2):
                x = pr.alpha * (kp[pg, 0, sl][seen] @ q[r, h])
                s = torch.from_numpy(x / (1.0 + np.exp(-x)) / pr.alpha).to(torch.bfloat16)
                one[r, h] = pr.alpha * (_f64(s) @ vp[pg, 0, sl][seen]) / pr.max_len
    assert (np.abs(one - o) > tol).mean() > 0.1
