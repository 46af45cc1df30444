"""GPU tests of the losses on stored logits (distillation, policy, preference) where one row, one entry of it, or one call beside another decides."""
import ctypes
import threading

import numpy as np
import pytest

from helpers import Guarded
from test_gpu_losses import TOK, U, bits, layout, mtf, t_dtype  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- calls of host threads beside each other ----------------------------------------------------------------------------------------------------

def test_streamed_distillation_in_threads_with_lists_of_different_sizes(mtf):  # noqa: F811
    """Rows that are streamed through shared memory, whose size goes by the slots of a list: every call of every thread is taken, and leaves the bits that it leaves alone.
    (The library's calls themselves, their arguments made beforehand, so that the threads are in the library for most of the time, and rows that are mostly skipped.)"""
    import torch
    from paper_1811_02084_b200 import binding
    V, T = 20000, 1300                                                # 52 MB in bf16, 40 KB a row
    N, lay = mtf.named, layout(mtf)

    def prepared(slots, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        z = (2 * torch.randn(1, T, V, generator=g, device="cuda")).bfloat16()
        ids = torch.randint(0, V, (1, T, slots), generator=g, device="cuda").int()
        teacher, y = torch.randn(1, T, slots, generator=g, device="cuda"), torch.randint(0, V, (1, T), generator=g, device="cuda").int()
        loss, dz = torch.full((1, T), 7.0, device="cuda"), torch.full_like(z, 7.0)
        w = torch.zeros(1, T, device="cuda")
        w[0, ::100] = 1.0
        stream, hp = torch.cuda.Stream(), mtf.mtf_distill_params(2.0, 0.5, 0.5)
        keep = [N(z, TOK + ["vocab"]), N(teacher, TOK + ["slot"]), N(w, TOK), N(loss, TOK), N(dz, TOK + ["vocab"]), ids, y, hp, stream, lay]
        n_z, n_teacher, n_w, n_loss, n_dz = (n.ref for n in keep[:5])
        args = (lay.handle, n_z, ids.data_ptr(), n_teacher, y.data_ptr(), n_w, ctypes.byref(hp), n_loss, n_dz, stream.cuda_stream)
        return args, [loss, dz], keep

    work = [prepared(slots, 50 + i) for i, slots in enumerate((4, 64, 512, 1))]
    step, want = binding._lib.mtf_distill_step, []
    torch.cuda.synchronize()
    for args, outs, _ in work:
        assert step(*args) == 0
        torch.cuda.synchronize()
        want.append(bits(outs))
        for t in outs:
            t.fill_(7.0)
    mtf.mtf_device_status()
    codes, start = [[] for _ in work], threading.Barrier(len(work))

    def run(args, into):
        start.wait()
        for _ in range(4000):
            into.append(step(*args))

    threads = [threading.Thread(target=run, args=(args, into)) for (args, _, _), into in zip(work, codes)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert [sum(c != 0 for c in into) for into in codes] == [0] * len(work)
    mtf.mtf_device_status()
    for (_, outs, _), w in zip(work, want):
        assert all(torch.equal(a, b) for a, b in zip(bits(outs), w))


# ---- rows that are not finite -------------------------------------------------------------------------------------------------------------------

def distill_forward(m, z, tau, soft=0.5, hard=0.5):
    """(stats, loss, gradient of the step) of rows z with a list of three words and the label 0"""
    import torch
    T, V = z.shape
    N, lay = m.named, layout(m)
    ids = (torch.arange(3, device="cuda") % V).expand(1, T, 3).contiguous().int()
    teacher, y = torch.zeros(1, T, 3, device="cuda"), torch.zeros(1, T, dtype=torch.int32, device="cuda")
    guard = Guarded()
    stats, loss, step_loss, dz = guard.empty([1, T, 2], "f32"), guard.empty([1, T], "f32"), guard.empty([1, T], "f32"), guard.empty([1, T, V], "bf16" if z.dtype == torch.bfloat16 else "f32")
    args = (N(z.view(1, T, V), TOK + ["vocab"]), ids, N(teacher, TOK + ["slot"]), y, None, tau, soft, hard)
    m.mtf_distill_forward(lay, *args, N(stats, TOK + ["stat"]), N(loss, TOK))
    m.mtf_distill_step(lay, *args, N(step_loss, TOK), N(dz, TOK + ["vocab"]))
    m.mtf_device_status()
    guard.check()
    return stats[0], loss[0], step_loss[0], dz[0]


# (a row to a block, few long rows in clusters, and rows beside which a step streams)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 4099, 150001])
@pytest.mark.parametrize("tau", [1.0, 1.5, 2.0, 2.5, 0.7])
def test_a_nan_anywhere_in_a_row_shows_in_all_its_results(mtf, V, dtype, tau):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(V)
    near = min(V, 40)
    at = sorted({*range(near), *range(V - near, V), *np.random.RandomState(V).randint(0, V, 24).tolist()})
    z = (2 * torch.randn(len(at) + 1, V, generator=g, device="cuda")).to(t_dtype(dtype))
    z[torch.arange(len(at), device="cuda"), torch.tensor(at, device="cuda")] = float("nan")
    stats, loss, step_loss, dz = distill_forward(mtf, z, tau)
    assert bool(stats[:-1].isnan().all()), ("stats", [at[i] for i in (~stats[:-1].isnan()).any(-1).nonzero()[:8, 0].tolist()])
    assert bool(loss[:-1].isnan().all()) and bool(step_loss[:-1].isnan().all()) and bool(dz[:-1].isnan().all())
    assert bool(stats[-1].isfinite().all()) and bool(loss[-1].isfinite()) and bool(step_loss[-1].isfinite()) and bool(dz[-1].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 40, 4099, 150001])
def test_rows_without_a_finite_logit_have_nan_statistics(mtf, V, dtype):  # noqa: F811
    import torch
    T, inf = 4, float("inf")
    z = torch.zeros(T, V, device="cuda").to(t_dtype(dtype))
    z[0] = -inf                                                       # row 1 has one word left, row 2 a word of infinite weight, row 3 is ordinary
    z[1], z[2, V - 1] = -inf, inf
    z[1, V // 2] = -3.0
    for tau in (1.0, 1.5, 2.0, 2.5, 0.7):
        stats, loss, step_loss, _ = distill_forward(mtf, z, tau)
        assert bool(stats[[0, 2]].isnan().all()) and bool(loss[[0, 2]].isnan().all()) and bool(step_loss[[0, 2]].isnan().all())
        assert bool(stats[[1, 3]].isfinite().all())
        # (the one exponential, of an argument of 0 or its rounding, is 1 but for 2^-22, and so are its powers up to the third but for three times that and their roundings)
        t = float(np.float32(tau))
        assert abs(float(stats[1, 0]) + 3.0 / t) <= (16 + 3.0 / t) * U and abs(float(stats[1, 1]) + 3.0) <= (16 + 3) * U
    N, lay = mtf.named, layout(mtf)
    guard = Guarded()
    y = torch.full((1, T), V // 2, dtype=torch.int32, device="cuda")
    zero, tok2 = torch.zeros(1, T, device="cuda"), ["branch", "batch", "length"]
    room = [guard.empty([1, T], "f32") for _ in range(4)]
    mtf.mtf_policy_forward(lay, N(z.view(1, T, V), TOK + ["vocab"]), y, N(zero, TOK), None, N(zero, TOK), None, 0.2, 0.2, 0.0, *[N(t, TOK) for t in room])
    lse, logp = room[0][0], room[1][0]
    assert bool(lse[[0, 2]].isnan().all()) and bool(logp[[0, 2]].isnan().all())
    assert abs(float(lse[1]) + 3.0) <= (16 + 3) * U and abs(float(logp[1])) <= 16 * U and bool(lse[3].isfinite())
    lse, logp, seq, dseq, loss = (guard.empty(s, "f32") for s in ([2, 2, 1], [2, 2, 1], [2, 2], [2, 2], [2]))
    ref = torch.zeros(2, 2, device="cuda")
    mtf.mtf_preference_forward(lay, N(z.view(2, 2, 1, V), tok2 + ["vocab"]), y.view(2, 2, 1), None, N(ref, tok2[:2]), "sigmoid", 0.1, 0.0, N(lse, tok2), N(logp, tok2), N(seq, tok2[:2]),
                               N(dseq, tok2[:2]), N(loss, ["batch"]))
    mtf.mtf_device_status()
    guard.check()
    lse = lse.view(-1)
    assert bool(lse[[0, 2]].isnan().all()) and abs(float(lse[1]) + 3.0) <= (16 + 3) * U and bool(lse[3].isfinite())
