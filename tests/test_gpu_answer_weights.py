"""Attention over a paged cache keeps its weights' digits: rows of V that all but cancel leave the error of the weights alone.

Pairs of positions hold x and -x with logits one step of 2^-7 apart, exact in every product: the result is P = sum p |v| times some 2^-9, and a weight rounded once, off by up to 2^-8 (bf16) or
2^-11 (f16) of itself and by another amount in each of a pair, would show as some 2^-11 or 2^-14 P.  Tolerances count the roundings as those of test_gpu_answer do.  With a bf16 cache a weight is
two pieces, of which the second rounds what the first leaves: w = (2^-8)^2; with an e4m3 cache it is one f16, w = 2^-11.  The positions that have a value have logits z below 2: theirs is off by delta = (2 d_k u) |z| + 6 u |z| (one product is
not 0), and a weight by 2 delta + 2^-20; in e4m3 the exponent of V's scale and the lift add three roundings of numbers below 16, 2^-21 each.  The other positions lie 2^17 e lower and have no
value.  The sums take (n / 32 + 64) 2 u.  So
    |o - o*| <= 2^-8 |o*| + (P + |o*|) (w + 2 delta + 2^-20 + (n / 32 + 64) 2 u [+ 3 2^-21]) [+ n 2^-33 max |v|]    with e4m3's terms in brackets."""
import numpy as np
import pytest

from oracle import answer as oa
from test_gpu_answer import U, Paged, check_attention, host, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
CAP = 17000

# positions, pages of a sequence of 16: a block an item, clusters, the even cut
PLANS = {"block": ([40, 17], 3), "clusters": ([700, 333], 44), "shares": ([3000, 40], -(-CAP // 16))}


@pytest.mark.parametrize("group", [None, 3, 11])
@pytest.mark.parametrize("d_v", [64, 128, 256])
@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_weights_keep_their_digits(mtf, dtype, plan, d_v, group):  # noqa: F811
    import torch
    lengths, per = PLANS[plan]
    r, d_k, eight = np.random.RandomState(d_v + len(plan)), 16, dtype == "e4m3"
    p = Paged(mtf, dtype, lengths, 2, d_k, d_v, 16, per=per, seed=1)
    for s, n in enumerate(lengths):
        z, v = np.full((n, 2), -16.0), np.zeros((n, 2, d_v))
        for m in range(0, n - 1, 2 * max(1, n // 40)):
            z[m] = 1 + r.randint(0, 127, 2) / 128                      # (one step below 2 left for the other)
            z[m + 1] = z[m] + 2.0 ** -7
            v[m] = r.randint(-15, 16, (2, d_v)) / 4.0                  # (four digits)
            v[m + 1] = -v[m]
        k = np.zeros((n, 2, d_k))
        k[:, :, 0] = z
        page, slot = p.table_host[s, np.arange(n) // 16], np.arange(n) % 16
        if eight:                                                      # (a key's value is its scale's, and negative ones its sign's)
            p.k_scale[page, slot] = torch.tensor(np.abs(z), dtype=torch.float32, device="cuda")
            p.v_scale[page, slot] = 1.0
            for pool, x in ((p.k, k / np.abs(z)[..., None]), (p.v, v)):
                pool.view(torch.uint8)[page, slot] = torch.tensor(oa.to_e4m3(x), device="cuda")
        else:
            p.k[page, slot], p.v[page, slot] = (torch.tensor(x, dtype=torch.bfloat16, device="cuda") for x in (k, v))
        assert np.array_equal(p.rows("k", s), k) and np.array_equal(p.rows("v", s), v)
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, group, d_k, d_v)
    q.zero_()
    q[..., 0] = 1.0
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 1.0, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    p.guard.check()
    got = host(o).reshape(len(lengths), 2, -1, d_v)
    delta = (2 * d_k + 6) * U * 2
    for s, n in enumerate(lengths):
        v = p.rows("v", s)
        want, size, _ = oa.decode(host(q)[s].reshape(2, -1, d_k), p.rows("k", s), v, 1.0)
        off = (2.0 ** -11 + 3 * 2.0 ** -21 if eight else 2.0 ** -16) + 2 * delta + 2.0 ** -20 + (n / 32 + 64) * 2 * U
        tol = 2.0 ** -8 * np.abs(want) + (size + np.abs(want)) * off + (n * 2.0 ** -33 * np.abs(v).max() if eight else 0.0)
        err = np.abs(got[s] - want)
        assert (err <= tol).all(), (s, n, float((err / np.maximum(tol, 1e-300)).max()))


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("far", [-110, -117, -120, -126])
@pytest.mark.parametrize("some_zero", [False, True])
def test_rows_of_v_with_the_smallest_scales(mtf, some_zero, far, plan):  # noqa: F811
    """Scales of V down to the smallest normal float, all of them or all but every fifth, which is 0: results that a bf16 still holds."""
    lengths, per = PLANS[plan]
    p = Paged(mtf, "e4m3", lengths, 2, 64, 64, 16, per=per, seed=far + 200)
    for s, n in enumerate(lengths):
        page, slot = p.table_host[s, np.arange(n) // 16], np.arange(n) % 16
        p.v_scale[page, slot] = 2.0 ** far
        if some_zero:
            p.v_scale[page[::5], slot[::5]] = 0.0
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, 3, 64, 64)
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    p.guard.check()
    got = host(o)
    for s, n in enumerate(lengths):
        k, v, qs = p.rows("k", s), p.rows("v", s), host(q)[s]
        want, size, z = oa.decode(qs, k, v, 0.125)
        assert np.abs(want).max() > 2.0 ** (far + 2)
        A = 0.125 * np.einsum("hgd,mhd->hgm", np.abs(qs), np.abs(k)).max(-1)
        delta = (2 * 64 * U * A + 6 * U * np.abs(z).max(-1))[..., None]
        # the tolerance of test_gpu_answer; a weight as small as 2^-34 of the largest that a scale goes with; and half of the smallest step of bf16
        tol = 2.0 ** -8 * np.abs(want) + size * (2.0 ** -11 + 4 * delta + 2.0 ** -20 + (n / 32 + 64) * 4 * U) + n * 2.0 ** -33 * np.abs(v).max() + 2.0 ** -134
        assert (np.abs(got[s] - want) <= tol).all(), (s, float((np.abs(got[s] - want) / tol).max()))


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("size", [1.0, 1e-4, 1e-6, 1e-12, 1e-30])
@pytest.mark.parametrize("order", ["first", "last", "between"])
def test_rows_of_zeros_leave_the_others_their_digits(mtf, order, size, plan):  # noqa: F811
    """A row of zeros of V is stored with the scale 1: beside rows of small values that must not take the range of the weights, whether it comes before them, behind them or among them."""
    import torch
    lengths, per = PLANS[plan]
    p = Paged(mtf, "e4m3", lengths, 2, 64, 128, 16, per=per, seed=3)
    lay, n0 = layout(mtf), max(lengths)
    g = torch.Generator(device="cuda").manual_seed(7)
    kk, vv = (torch.randn(len(lengths), n0, 2, d, generator=g, device="cuda") for d in (64, 128))
    vv *= size
    for s, n in enumerate(lengths):
        zero = {"first": np.arange(n) < n // 4, "last": np.arange(n) >= n - n // 4, "between": np.arange(n) % 7 == 3}[order]
        vv[s, :n][torch.tensor(zero, device="cuda")] = 0.0
        vv[s, 1 if order == "first" else n - 2, :, ::2] *= -0.0        # (zeros of both signs)
    dims = ["batch", "length", "heads"]
    mtf.mtf_cache_write(lay, mtf.named(kk, dims + ["d_k"]), mtf.named(vv, dims + ["d_v"]), None, p.lengths, p.cache)
    q, o, nq, no = queries(mtf, p, 3, 64, 128)
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    p.guard.check()
    for s, n in enumerate(lengths):
        scales = oa.gather(host(p.v_scale), p.table_host[s], n, 16, True)
        zero = ~p.rows("v", s).any(-1)
        assert zero.any() and (scales[zero] == 1).all()
    check_attention(p, q, o, 0.125)
