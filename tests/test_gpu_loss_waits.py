"""The failure path of the streamed losses' bounded waits, without faulting anything: the testing hook shortens the limit to about a millisecond and has a wait ask for a signal that
does not come, of a row's numbers within a block or of the sums within a cluster.  The call ends, the host reads MTF_ERR_TIMEOUT, nothing outside the outputs is written, and the next call is correct."""
import pytest

from helpers import Guarded
from test_gpu_losses import TOK, bits, layout, mtf, t_dtype  # noqa: F401

pytestmark = pytest.mark.gpu
LIMIT = 2_000_000                                                     # cycles, about 1 ms; a step below takes some 40 us


def prepared(m, op, dtype, T, V):
    import torch
    g = torch.Generator(device="cuda").manual_seed(T + V)
    z = (2 * torch.randn(1, T, V, generator=g, device="cuda")).to(t_dtype(dtype))
    y = torch.randint(0, V, (1, T), generator=g, device="cuda").int()
    guard, N, lay = Guarded(), m.named, layout(m)
    loss, logp, dz = guard.empty([1, T], "f32"), guard.empty([1, T], "f32"), guard.empty([1, T, V], dtype)
    n_z, n_dz, n_loss = N(z, TOK + ["vocab"]), N(dz, TOK + ["vocab"]), N(loss, TOK)
    if op == "policy":
        old, adv = N(torch.full((1, T), -9.0, device="cuda"), TOK), N(torch.randn(1, T, generator=g, device="cuda"), TOK)
        return lambda: m.mtf_policy_step(lay, n_z, y, old, None, adv, None, 0.2, 0.25, 0.0, N(logp, TOK), n_loss, n_dz), [loss, logp, dz], guard
    ids, teacher = torch.randint(0, V, (1, T, 40), generator=g, device="cuda").int(), N(torch.randn(1, T, 40, generator=g, device="cuda"), TOK + ["slot"])
    return lambda: m.mtf_distill_step(lay, n_z, ids, teacher, y, None, 2.0, 0.5, 0.5, n_loss, n_dz), [loss, dz], guard


# rows of one block, and of clusters of 2, 4 and 8
@pytest.mark.parametrize("dtype,T,V,withhold", [("bf16", 1300, 20000, 1), ("bf16", 220, 131072, 1), ("f32", 60, 270000, 1), ("bf16", 220, 131072, 2), ("f32", 110, 131072, 2), ("f32", 60, 270000, 2)])
@pytest.mark.parametrize("op", ["policy", "distill"])
def test_a_wait_runs_out_and_the_next_call_is_correct(mtf, op, dtype, T, V, withhold):  # noqa: F811
    import torch
    call, outs, guard = prepared(mtf, op, dtype, T, V)
    call()
    mtf.mtf_device_status()
    want = bits(outs)
    try:
        mtf.mtf_debug_wait_test(LIMIT, 0)                             # the limit alone changes nothing
        call()
        mtf.mtf_device_status()
        assert all(torch.equal(a, b) for a, b in zip(bits(outs), want))
        mtf.mtf_debug_wait_test(LIMIT, withhold)
        call()
        with pytest.raises(mtf.MtfError, match="0xa[01]") as e:
            mtf.mtf_device_status()
        assert e.value.code == "MTF_ERR_TIMEOUT"
    finally:
        mtf.mtf_debug_wait_test(0, 0)
    mtf.mtf_device_status()                                           # reported once
    guard.check()
    for t in outs:
        t.fill_(float("nan"))
    for _ in range(2):
        call()
    mtf.mtf_device_status()
    guard.check()
    assert all(torch.equal(a, b) for a, b in zip(bits(outs), want))
