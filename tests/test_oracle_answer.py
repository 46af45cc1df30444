"""Pins of oracle/answer.py: e4m3 against torch's type, scales by their definition, attention against a softmax written out, selection against all offers sorted."""
import numpy as np
import pytest
import torch

from oracle import answer as oa


def test_e4m3_is_the_type():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oa.E4M3, want, equal_nan=True)
    # every value, every midpoint between neighbours and the numbers on either side of it
    size = oa.E4M3[:127]
    mid = (size[1:] + size[:-1]) / 2
    x = np.concatenate([size, mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    x = np.concatenate([x, -x])
    got = oa.E4M3[oa.to_e4m3(x)]
    assert np.array_equal(got, torch.tensor(x).float().to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("top", [448.0, 449.0, 447.9, 1.0, 3.5, 1.75, 1.7500001, 2.0 ** -100, 2.0 ** -140, 3e38])
def test_scale_is_the_smallest_power_of_two(top):
    b, s = oa.quantise(np.array([[top, -top / 3, 0.0, top / 1000]]))
    assert np.log2(s[0]) == np.round(np.log2(s[0])) and top <= 448 * s[0]
    assert top > 224 * s[0] or s[0] == 2.0 ** -126
    back = oa.E4M3[b[0]] * s[0]
    assert abs(back[0] - top) <= top * 2.0 ** -4 or s[0] == 2.0 ** -126
    z, s = oa.quantise(np.zeros((2, 4)))
    assert (s == 1).all() and not z.any()
    n, s = oa.quantise(np.array([[np.nan, np.inf, 7.0, -np.inf]]))
    assert s[0] == 2.0 ** -6 and np.isnan(oa.E4M3[n[0]][[0, 1, 3]]).all() and oa.E4M3[n[0]][2] * s[0] == 7.0


def test_attention_by_hand():
    r = np.random.RandomState(0)
    q, k, v = r.randn(2, 3, 8), r.randn(5, 2, 8), r.randn(5, 2, 4)
    o, size, _ = oa.decode(q, k, v, 0.5)
    w = np.exp(0.5 * np.einsum("hgd,mhd->hgm", q, k))
    assert np.allclose(o, np.einsum("hgm,mhd->hgd", w, v) / w.sum(-1)[..., None])
    assert (size >= np.abs(o) - 1e-12).all()
    assert not oa.decode(q, k[:0], v[:0], 0.5)[0].any()


def test_selection_is_the_head_of_all_offers():
    r = np.random.RandomState(1)
    z, s = r.randn(3, 11), np.array([-1.0, -1.5, -np.inf])
    fin = [0, 1, 0]
    p, t, best, f = oa.beam_select(z, s, fin, 4, 6)
    logp = z[0] - np.log(np.exp(z[0]).sum())
    all_offers = sorted([(-(s[0] + logp[v]), 0, v) for v in range(11)] + [(1.5, 1, 4)])[:6]
    assert [(int(a), int(b)) for a, b in zip(p, t)] == [(i, v) for _, i, v in all_offers]
    assert np.allclose(best, [-x for x, _, _ in all_offers])
    assert [int(x) for x in f] == [int(v == 4) for _, _, v in all_offers]
    # equal rows: the lower beam, then the lower word; too few offers: the rest is empty
    p, t, best, f = oa.beam_select(np.zeros((2, 3)), [0.0, 0.0], None, 0, 6)
    assert p.tolist() == [0, 0, 0, 1, 1, 1] and t.tolist() == [0, 1, 2, 0, 1, 2]
    p, t, best, f = oa.beam_select(np.array([[0.0, -np.inf, -np.inf]]), [0.0], None, 2, 3)
    assert p.tolist() == [0, 0, 0] and t.tolist() == [0, 2, 2] and best.tolist() == [0.0, -np.inf, -np.inf] and f.tolist() == [0, 1, 1]
