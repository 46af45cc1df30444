"""Caches of beams reordered where a last page, a fresh page or a length is none: what is left out goes on being left out, and nothing that a page held before takes its place."""
import numpy as np
import pytest

from test_gpu_answer import Paged, check_attention, host, ints, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
S, K, SLOTS, LENGTH = 2, 3, 16, 37                                    # sentences, beams, slots of a page, positions: two whole pages and 5 more


def reported(mtf):  # noqa: F811
    with pytest.raises(mtf.MtfError) as e:
        mtf.mtf_device_status()
    assert e.value.code == "MTF_ERR_INVALID_ARG"
    mtf.mtf_device_status()                                           # (once)


def setting(mtf, dtype, slot_first, per=4):  # noqa: F811
    p = Paged(mtf, dtype, [LENGTH] * (S * K), 2, 64, 64, SLOTS, slot_first, per=per, seed=4, spare=S * K + 1)
    pools = [n for n in ("k", "v", "k_scale", "v_scale") if getattr(p, n) is not None]
    fresh = p.spare[:S * K].reshape(S, K)
    return p, pools, fresh, ints(np.full((S, K, per), -3)), ints(np.full((S, K), -3))


def raw(t):
    import torch
    return t.detach().view(torch.uint8).clone()


def cache(mtf, p, table):  # noqa: F811
    return mtf.Cache(p.named["k"], p.named["v"], table, p.named["k_scale"], p.named["v_scale"])


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("which", ["behind", "below", "far"])
def test_a_last_page_outside_the_pool_stays_outside(mtf, which, dtype, slot_first):  # noqa: F811
    import torch
    p, pools, fresh, new_table, new_lengths = setting(mtf, dtype, slot_first)
    bad = {"behind": p.pages, "below": -1, "far": 1 << 30}[which]
    table = p.table_host.copy().reshape(S, K, -1)
    table[1, 2, LENGTH // SLOTS] = bad                                # the last page of one beam, of which two answers go on
    parents = np.array([[0, 1, 2], [2, 0, 2]])
    before = {n: raw(getattr(p, n)) for n in pools}
    lay = layout(mtf)
    mtf.mtf_cache_reorder(lay, cache(mtf, p, ints(table)), ints(parents), p.lengths.view(S, K), ints(fresh), new_table, new_lengths)
    reported(mtf)
    p.guard.check()
    nt = host(new_table).astype(int)
    for s in range(S):
        for i in range(K):
            want = table[s, parents[s, i]].copy()
            if parents[s, i] != 2 or s != 1:
                want[LENGTH // SLOTS] = fresh[s, i]
            assert nt[s, i].tolist() == want.tolist(), (s, i)
    assert (host(new_lengths) == LENGTH).all()
    # the fresh pages of the two are as they were
    for n in pools:
        now, was = raw(getattr(p, n)), before[n]
        for page in fresh[1, [0, 2]]:
            assert torch.equal(now[page], was[page])
    # and what follows leaves the positions of that page out: attention, and reading
    q, o, nq, no = queries(mtf, p, 3, 64, 64)
    c = cache(mtf, p, new_table.view(S * K, -1))
    mtf.mtf_attention_decode(lay, nq, c, new_lengths.view(-1), 0.125, no, workspace(mtf, lay, nq, p))
    reported(mtf)
    without = (K, K + 2)                                              # sequences of those two

    def rows(j):
        n = 2 * SLOTS if j in without else LENGTH
        return p.rows("k", j, n, nt[j // K, j % K]), p.rows("v", j, n, nt[j // K, j % K])
    check_attention(p, q, o, 0.125, rows=rows)
    back = [torch.full((S * K, LENGTH, 2, 64), 7.0, device="cuda") for _ in range(2)]
    mtf.mtf_cache_read(lay, c, None, None, *[mtf.named(x, ["batch", "length", "heads", d]) for x, d in zip(back, ("d_k", "d_v"))])
    reported(mtf)
    for j in without:
        assert all(not x[j, 2 * SLOTS:].any() and not x[j, :2 * SLOTS].isnan().any() for x in back)
    # another reordering hands the id on
    lengths, again = np.full((S, K), 2 * SLOTS), torch.empty_like(new_table)
    lengths[1, [0, 2]] = LENGTH
    mtf.mtf_cache_reorder(lay, cache(mtf, p, new_table), ints([[0, 1, 2], [2, 1, 0]]), ints(lengths), ints(np.full((S, K), p.spare[-1])), again, torch.empty_like(new_lengths))
    reported(mtf)
    assert host(again)[1, [0, 2], LENGTH // SLOTS].tolist() == [bad, bad]


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_lengths_below_0_and_beyond_the_table_become_what_the_table_has(mtf, dtype, slot_first):  # noqa: F811
    import torch
    p, pools, fresh, new_table, new_lengths = setting(mtf, dtype, slot_first, per=3)
    room = 3 * SLOTS
    lengths = np.array([[-1, room + 1, LENGTH], [-2 ** 31, 2 ** 31 - 1, 0]])
    parents = np.array([[0, 1, 2], [0, 1, 2]])
    before = {n: raw(getattr(p, n)) for n in pools}
    mtf.mtf_cache_reorder(layout(mtf), cache(mtf, p, p.table.view(S, K, -1)), ints(parents), ints(lengths), ints(fresh), new_table, new_lengths)
    reported(mtf)
    p.guard.check()
    assert host(new_lengths).tolist() == [[0, room, LENGTH], [0, room, 0]]
    want = p.table_host.reshape(S, K, -1).copy()
    want[0, 2, LENGTH // SLOTS] = fresh[0, 2]                         # (the one that goes on)
    assert np.array_equal(host(new_table).astype(int), want)
    for n in pools:
        now = raw(getattr(p, n))
        now[fresh[0, 2]] = before[n][fresh[0, 2]]
        assert torch.equal(now, before[n])
