"""Infinities in V in attention over a paged cache: what the sum of products gives.  (A weight that multiplies V as two values must not make inf - inf or 0 inf of one.)
And scales of an e4m3 cache's rows of zeros that are not numbers: what is left out of a reference is not left out of the result."""
import numpy as np
import pytest

from test_gpu_answer import Paged, check_attention, host, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
PLANS = {"block": (40, 3), "clusters": (700, 44), "shares": (3000, 1063)}


def attend(mtf, p, group, d_v, change):  # noqa: F811
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, group, p.k.shape[-1], d_v)
    change()
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    p.guard.check()
    return q, o


@pytest.mark.parametrize("group", [None, 11])
@pytest.mark.parametrize("d_v", [64, 128, 256])
@pytest.mark.parametrize("plan", PLANS)
def test_infinities_in_rows_of_v(mtf, plan, d_v, group):  # noqa: F811
    n, per = PLANS[plan]
    p = Paged(mtf, "bf16", [n, n], 2, 64, d_v, 16, per=per, seed=5)
    inf = float("inf")

    def change():
        # first and last positions, weights of every kind: logits 0, whose weights are a power of two, and others
        for m, d, x in ((0, 3, inf), (n - 1, 5, -inf), (n // 2, 9, inf), (n // 3, 9, inf), (1, 12, inf), (n - 2, 12, -inf), (7, 20, -inf)):
            p.v[p.table_host[0, m // 16], m % 16, 0, d] = x
        for m in range(n):                                            # equal weights, all of them 1
            p.k[p.table_host[1, m // 16], m % 16, 1] = 0.0
        p.v[p.table_host[1, 0], 2, 1, 33] = -inf
        p.v[p.table_host[1, 2], 1, 1, 34] = inf
    q, o = attend(mtf, p, group, d_v, change)
    got = host(o).reshape(2, 2, -1, d_v)
    for d, x in ((3, inf), (5, -inf), (9, inf), (20, -inf)):
        assert (got[0, 0, :, d] == x).all(), d
    assert np.isnan(got[0, 0, :, 12]).all()
    assert (got[1, 1, :, 33] == -inf).all() and (got[1, 1, :, 34] == inf).all()
    odd = np.zeros(got.shape, bool)
    odd[0, 0, :, [3, 5, 9, 12, 20]] = True
    odd[1, 1, :, [33, 34]] = True
    assert np.isfinite(got[~odd]).all()
    # the other columns are those of the same rows without them
    p.v.copy_(p.v.nan_to_num(nan=float("nan"), posinf=1.0, neginf=1.0))
    q, o = attend(mtf, p, group, d_v, lambda: None)
    again = host(o).reshape(got.shape)
    assert np.array_equal(again[~odd], got[~odd])
    check_attention(p, q, o, 0.125)


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_rows_of_zeros_with_scales_that_are_not_numbers(mtf, scale, plan):  # noqa: F811
    n, per = PLANS[plan]
    p = Paged(mtf, "e4m3", [n], 2, 64, 64, 16, per=per, seed=5)

    def change():
        import torch
        p.v.view(torch.uint8)[p.table_host[0, 1], 4, 0] = 0
        p.v_scale[p.table_host[0, 1], 4, 0] = scale
    q, o = attend(mtf, p, 3, 64, change)
    assert np.isnan(host(o)[0, 0]).all() and np.isfinite(host(o)[0, 1]).all()
