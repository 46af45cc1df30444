"""GPU tests of the losses on stored logits (distillation, policy, preference) where one row, one entry of it, or one call beside another decides."""
import ctypes
import threading

import numpy as np
import pytest

from helpers import Guarded
from test_gpu_losses import TOK, bits, layout, mtf, t_dtype  # noqa: F401

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
