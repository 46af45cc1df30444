"""GPU parity of attention over a paged cache where the keys of all sequences are shared out evenly over the GPU's blocks and the parts joined: tables that could hold long sequences,
whatever the sequences have.  Tolerances: those of test_gpu_answer."""
import threading

import numpy as np
import pytest

from test_gpu_answer import Paged, check_attention, decode, host, ints, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
CAP = 17000                                                          # positions of a table's pages: more than the widest rule asks for

#     heads group d_k  d_v slots  lengths
SHAPES = [
    (2, 4, 64, 64, 16, [0, 1, 15, 3000, 129, 700]),
    (1, None, 64, 64, 16, [CAP - 3, 0, 17]),                           # one long sequence beside nearly nothing
    (1, 8, 128, 128, 16, [5000, 1, 64, 65, 0, 0, 63]),
    (3, 9, 128, 72, 7, [2000, 129, 0]),                                # two tiles of heads, one of them nearly empty
    (1, 40, 64, 128, 24, [4500, 2]),                                   # more heads than a block takes at once
    (2, 3, 256, 256, 16, [4200, 31]),
    (1, 17, 256, 136, 50, [1500]),
    (1, 1, 8, 16, 1, [3001]),                                          # pages of one position
    (6, 2, 64, 64, 64, [(37 * i * i) % 900 for i in range(40)]),       # more items than blocks
    (2, 2, 32, 64, 100, [0, 0, 0]),                                    # no position at all
    (2, 2, 32, 64, 100, [0, 1, 0, 0, 1]),                              # hardly one
    (1, 5, 128, 128, 32, [30000]),                                     # more parts of a sequence than are joined at a time
]


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(mtf, dtype, shape, slot_first):  # noqa: F811
    heads, group, dk, dv, slots, lengths = SHAPES[shape]
    if dtype == "e4m3":
        dk, dv = -(-dk // 16) * 16, -(-dv // 16) * 16
    p = Paged(mtf, dtype, lengths, heads, dk, dv, slots, slot_first, max(-(-CAP // slots), -(-max(lengths) // slots)), seed=shape)
    q, o, nq, no = queries(mtf, p, group, dk, dv)
    w = workspace(mtf, layout(mtf), nq, p)
    assert w is not None                                             # (shared out, not a block or cluster an item)
    mtf.mtf_attention_decode(layout(mtf), nq, p.cache, p.lengths, dk ** -0.5, no, w)
    mtf.mtf_device_status()
    p.guard.check()
    check_attention(p, q, o, dk ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n_seq,shared", [(1024, True), (1025, False)])
def test_as_many_sequences_as_a_block_adds_up(mtf, dtype, n_seq, shared):  # noqa: F811
    """The most sequences that are shared out, and one more, which get a block each; few of them have positions, one of them many."""
    lengths = [0] * n_seq
    for i in (0, 7, 1000, 1020, n_seq - 1):
        lengths[i] = 1 + i % 400
    lengths[512] = 2500
    p = Paged(mtf, dtype, lengths, 1, 64, 64, 16, per=200, seed=5)
    assert (mtf.mtf_attention_decode_workspace_bytes(layout(mtf), queries(mtf, p, 2, 64, 64)[2], p.cache) > 0) == shared
    q, o = decode(mtf, p, 2, 64, 64, 0.125)
    got = host(o)
    for i in range(n_seq):
        assert lengths[i] or not got[i].any()
    live = [i for i in range(n_seq) if lengths[i]]
    check_attention(p, q[live], o[live], 0.125, rows=lambda s: (p.rows("k", live[s]), p.rows("v", live[s])))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_peaks_and_far_scales(mtf, dtype):  # noqa: F811
    """Logits of some hundreds and of none, so that parts differ by all of a float's range or not at all."""
    for scale, qscale in ((3.0, 4.0), (-0.3, 1.0), (0.0, 1.0), (1e4, 1e-4)):
        p = Paged(mtf, dtype, [2700, 33], 2, 64, 64, 16, per=-(-CAP // 16), seed=3)
        q, o = decode(mtf, p, 4, 64, 64, scale, qscale=qscale)
        check_attention(p, q, o, scale)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_not_numbers(mtf, dtype):  # noqa: F811
    """A NaN in a key takes its head's results, one in a value its column's; keys of -infinity (bf16) are left out, a head of such keys alone is 0."""
    import torch
    n = 3000
    p = Paged(mtf, dtype, [n, n], 3, 64, 64, 16, per=-(-CAP // 16), seed=6)
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, 2, 64, 64)
    q.abs_()
    w = workspace(mtf, lay, nq, p)
    assert w is not None
    nan = torch.tensor(float("nan"), device="cuda").to(p.k.dtype)

    def put(pool, s, m, h, d, x):
        pool[p.table_host[s, m // 16], m % 16, h, d] = x
    put(p.k, 0, 2900, 0, 5, nan)
    put(p.v, 0, 17, 1, 9, nan)
    if dtype == "bf16":
        pages = torch.tensor(p.table_host[1, :-(-n // 16)], device="cuda")
        p.k[pages[:100], :, 0, 0] = float("-inf")                    # the first 1600 positions of head 0, all of head 1
        p.k[pages, :, 1, 0] = float("-inf")
        put(p.k, 1, 1700, 2, 0, float("inf"))
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, w)
    mtf.mtf_device_status()
    p.guard.check()
    got = host(o)
    assert np.isnan(got[0, 0]).all()
    column = np.zeros((2, 64), bool)
    column[:, 9] = True
    assert np.array_equal(np.isnan(got[0, 1]), column) and np.isfinite(got[0, 2]).all()
    if dtype == "bf16":
        assert not got[1, 1].any() and np.isnan(got[1, 2]).all()
        k, v = p.rows("k", 1)[1600:, :1], p.rows("v", 1)[1600:, :1]
        one = Paged.__new__(Paged)
        one.dtype = dtype
        check_attention(one, q[1:, :1], o[1:, :1], 0.125, rows=lambda s: (k, v))


def test_bad_pages_and_lengths(mtf):  # noqa: F811
    """Pages outside the pool and lengths beyond the table: reported, and as if their positions were not there."""
    per = 1100
    lay = layout(mtf)
    p = Paged(mtf, "bf16", [2000, 100, 100], 2, 64, 64, 16, per=per, seed=2)
    table = p.table_host.copy()
    table[0, 100:110], table[1, 2], table[2, :7] = p.pages, -1, 1 << 30
    p.table.copy_(ints(table))
    q, o, nq, no = queries(mtf, p, 2, 64, 64)
    w = workspace(mtf, lay, nq, p)
    assert w is not None
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, w)
    with pytest.raises(mtf.MtfError) as e:
        mtf.mtf_device_status()
    assert e.value.code == "MTF_ERR_INVALID_ARG"
    mtf.mtf_device_status()                                        # (said once)
    p.guard.check()
    out = {0: range(1600, 1760), 1: range(32, 48), 2: range(100)}

    def rows(s):
        keep = [m for m in range(p.lengths_host[s]) if m not in out[s]]
        return p.rows("k", s)[keep], p.rows("v", s)[keep]
    check_attention(p, q, o, 0.125, rows=rows)
    full = Paged(mtf, "bf16", [per * 16, 1, 100], 1, 64, 64, 16, per=per, seed=9)
    full.lengths.copy_(ints([per * 16 + 1, -5, 100]))
    q, o, nq, no = queries(mtf, full, 2, 64, 64)
    mtf.mtf_attention_decode(lay, nq, full.cache, full.lengths, 0.125, no, workspace(mtf, lay, nq, full))
    with pytest.raises(mtf.MtfError):
        mtf.mtf_device_status()
    full.lengths_host = [per * 16, 0, 100]
    full.guard.check()
    check_attention(full, q, o, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_one_workspace_for_calls_in_turn_graphs_and_threads(mtf, dtype):  # noqa: F811
    """Two calls of different lengths that take turns in one workspace, eagerly, captured and replayed, with lengths that change between replays; and with a workspace each, at
    once: the bits of the first call each time."""
    import torch
    lay, n = layout(mtf), 3
    p = Paged(mtf, dtype, [3000, 1200, 5], 2, 64, 64, 16, per=-(-CAP // 16), seed=11)
    q, o, nq, no = queries(mtf, p, 4, 64, 64)
    o2 = torch.zeros_like(o)
    no2 = mtf.named(o2, no.names)
    lengths = [p.lengths.clone(), ints([700, 1, 0])]
    w = [workspace(mtf, lay, nq, p) for _ in range(2)]
    outs, refs = [(o, no), (o2, no2)], []

    def one(i, of=0):
        mtf.mtf_attention_decode(lay, nq, p.cache, lengths[i], 0.125, outs[i][1], w[of])
    for i in range(2):
        one(i)
        refs.append(outs[i][0].clone())
    mtf.mtf_device_status()
    check_attention(p, q, o, 0.125)
    side = torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gr, stream=side):
        one(0)
        one(1)
    for _ in range(3):
        o.zero_(), o2.zero_()
        gr.replay()
        one(1)
        assert torch.equal(o, refs[0]) and torch.equal(o2, refs[1])
    # the same graph, with other lengths in the same places
    keep = [x.clone() for x in lengths]
    lengths[0].copy_(keep[1]), lengths[1].copy_(keep[0])
    gr.replay()
    assert torch.equal(o, refs[1]) and torch.equal(o2, refs[0])
    lengths[0].copy_(keep[0]), lengths[1].copy_(keep[1])
    torch.cuda.synchronize()

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(n):
                one(i, i)
        s.synchronize()
    o.zero_(), o2.zero_()
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    mtf.mtf_device_status()
    p.guard.check()
    assert torch.equal(o, refs[0]) and torch.equal(o2, refs[1])
