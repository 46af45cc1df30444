"""Pages outside the pool and lengths outside the table in attention over a paged cache, in both types: reported once, and as if their positions were not there.  With an e4m3 cache places in the
scales, the mask of a chunk's keys (up to 64) and the zeros written over rows of V that are none have ways of their own.  Tolerances: those of test_gpu_answer."""
import numpy as np
import pytest

from test_gpu_answer import Paged, check_attention, ints, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
CAP = 17000


def attend(mtf, p, q, o, nq, no, scale):  # noqa: F811
    lay = layout(mtf)
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, scale, no, workspace(mtf, lay, nq, p))
    with pytest.raises(mtf.MtfError) as e:
        mtf.mtf_device_status()
    assert e.value.code == "MTF_ERR_INVALID_ARG"
    mtf.mtf_device_status()                                           # (said once)
    p.guard.check()


#     positions of the longest, positions that a table has room for: a block an item, clusters, the even cut
PLANS = {"block": (100, 112), "clusters": (700, 704), "shares": (2000, CAP)}


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("slots", [2, 7, 16, 64])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("plan", PLANS)
def test_pages_outside_the_pool(mtf, plan, dtype, d, slots, slot_first):  # noqa: F811
    most, room = PLANS[plan]
    lengths = [most, 97, 64, 33]
    p = Paged(mtf, dtype, lengths, 2, d, d, slots, slot_first, per=-(-room // slots), seed=slots + d)
    table, gone = p.table_host.copy(), [set() for _ in lengths]

    def lose(s, page, to):
        if page * slots < lengths[s]:
            table[s, page] = to
            gone[s] |= set(range(page * slots, min(lengths[s], (page + 1) * slots)))
    # pages in the first and in the second half of a 64-key chunk, in either order of who is there, and the last one
    lose(0, 16 // slots, p.pages)
    lose(0, 48 // slots, -1)
    lose(0, 80 // slots, 1 << 30)
    lose(0, (most - 1) // slots, -2 ** 31)
    for page in range(0, 32 // slots + 1):                            # the whole first half
        lose(1, page, p.pages + 5)
    for page in range(-(-64 // slots)):                               # all of a sequence
        lose(2, page, -1)
    lose(3, 32 // slots, 2 ** 31 - 1)                                 # the one position behind 32
    p.table.copy_(ints(table))
    q, o, nq, no = queries(mtf, p, 3, d, d)
    attend(mtf, p, q, o, nq, no, d ** -0.5)

    def rows(s):
        keep = [m for m in range(lengths[s]) if m not in gone[s]]
        return p.rows("k", s)[keep], p.rows("v", s)[keep]
    check_attention(p, q, o, d ** -0.5, rows=rows)


@pytest.mark.parametrize("slots", [7, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("per", [6, 40, -(-CAP // 7)])
def test_lengths_outside_the_table(mtf, per, dtype, d, slots):  # noqa: F811
    room = per * slots
    p = Paged(mtf, dtype, [min(room, 4000), 1, 50 if room > 50 else room - 1], 1, d, d, slots, per=per, seed=9)
    if room <= 4000:
        p.lengths.copy_(ints([room + 1, -5, p.lengths_host[2]]))
        p.lengths_host = [room, 0, p.lengths_host[2]]
    else:
        p.lengths.copy_(ints([4000, -2 ** 31, p.lengths_host[2]]))
        p.lengths_host = [4000, 0, p.lengths_host[2]]
    q, o, nq, no = queries(mtf, p, 2, d, d)
    attend(mtf, p, q, o, nq, no, 0.125)
    check_attention(p, q, o, 0.125)
    if room <= 4000:
        # as far beyond as a number goes
        p.lengths[0] = 2 ** 31 - 1
        attend(mtf, p, q, o, nq, no, 0.125)
        check_attention(p, q, o, 0.125)
