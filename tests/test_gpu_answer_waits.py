"""The failure path of the bounded waits of attention over a cache and of beam selection, without faulting anything: the testing hook shortens the limit to about a millisecond and has
each warp's first wait ask for a copy that nobody has sent.  The call ends, the host reads MTF_ERR_TIMEOUT, nothing outside the outputs is written, and the next call is correct."""
import pytest

from helpers import Guarded
from test_gpu_answer import Paged, ints, layout, mtf, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
LIMIT = 2_000_000                                                     # cycles, about 1 ms; a call below takes some 20 us


def attention(m, dtype, lengths, per, d):
    p = Paged(m, dtype, lengths, 2, d, d, 16, per=per, seed=1)
    q, o, nq, no = queries(m, p, 4, d, d)
    lay = layout(m)
    w = workspace(m, lay, nq, p)
    return lambda: m.mtf_attention_decode(lay, nq, p.cache, p.lengths, d ** -0.5, no, w), [o], p.guard


def selection(m, dtype, V):
    import torch
    g, guard, lay = torch.Generator(device="cuda").manual_seed(V), Guarded(), layout(m)
    z = torch.randn(2, 4, V, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    scores = torch.randn(2, 4, generator=g, device="cuda")
    nz, ns = m.named(z, ["sentence", "beam", "vocab"]), m.named(scores, ["sentence", "beam"])
    outs = [guard.empty((2, 4), torch.int32, fill=0) for _ in range(3)] + [guard.empty((2, 4), "f32")]
    nnew = m.named(outs[3], ["sentence", "out"])
    w = guard.empty((m.mtf_beam_select_workspace_bytes(lay, nz, 4),), "u8")
    return lambda: m.mtf_beam_select(lay, nz, ns, None, 1, outs[0], outs[1], nnew, outs[2], w), outs, guard


# attention: a block an item, clusters, the even cut; selection: copies of whole runs, at and off 16 bytes, in two launches and in one
CALLS = {
    "block": lambda m, t: attention(m, t, [100, 30], 7, 64),
    "clusters": lambda m, t: attention(m, t, [700, 300], 44, 64),
    "wide": lambda m, t: attention(m, t, [700, 300], 44, 256),
    "shares": lambda m, t: attention(m, t, [3000, 300, 0], 1100, 64),
    "aligned": lambda m, t: selection(m, t, 32768),
    "odd": lambda m, t: selection(m, t, 40001),
    "few": lambda m, t: selection(m, t, 8000),
    "few odd": lambda m, t: selection(m, t, 8001),
}


@pytest.mark.parametrize("what,dtype,code", [(w, t, "0xb01") for w in ("block", "clusters", "wide", "shares") for t in ("bf16", "e4m3")]
                         + [(w, t, "0xb11") for w in ("aligned", "odd", "few", "few odd") for t in ("bf16", "f32")])
def test_a_wait_runs_out_and_the_next_call_is_correct(mtf, what, dtype, code):  # noqa: F811
    import torch
    call, outs, guard = CALLS[what](mtf, dtype)
    call()
    mtf.mtf_device_status()
    want = [t.clone() for t in outs]
    try:
        mtf.mtf_debug_wait_test(LIMIT, 0)                             # the limit alone changes nothing
        call()
        mtf.mtf_device_status()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        mtf.mtf_debug_wait_test(LIMIT, 1)
        call()
        with pytest.raises(mtf.MtfError, match=code) as e:
            mtf.mtf_device_status()
        assert e.value.code == "MTF_ERR_TIMEOUT"
    finally:
        mtf.mtf_debug_wait_test(0, 0)
    mtf.mtf_device_status()                                           # reported once
    guard.check()
    for t in outs:
        t.zero_()
    for _ in range(2):
        call()
    mtf.mtf_device_status()
    guard.check()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
