"""GPU tests of the losses on stored logits (distillation, policy, preference) where one row, one entry of it, or one call beside another decides."""
import ctypes
import threading

import numpy as np
import pytest

from helpers import Guarded
from test_gpu_losses import STEP, TOK, U, all_within, bits, layout, mtf, t_dtype  # noqa: F401

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


# ---- rows whose weight lies in a few entries ----------------------------------------------------------------------------------------------------

def delta(V):
    """A sum's relative error, as in test_gpu_losses.py (additions, and the errors of the exponentials), but with the additions that a launch makes: rows of 40 000 entries
    and more are walked by 128 threads at least, each with two partial sums, so that a chain has V / 256 of them at most; the joins of a warp's lanes, of warps and of a
    row's parts are 5 + 4 + 3 more and as many rescalings, for which 32 stands.  At V = 270001 that is 6.8e-5, where an average entry
    of those that hold a row's sum below is 1 / 1700 of it or more."""
    return (V / 256 + 32 + 3 * (np.log(V) + 1) + 8) * U


def rows_of_few_entries(dtype, T, V, seed):
    """Logits near -13 but for a few near 0, which hold nearly all of a row's sum: its first entries (row t % 4 == 0), its last ones (1), those around the places at which a
    row is cut into up to 8 parts (2), a few anywhere (3).  An entry left out or counted twice there moves the sum by far more than the bounds."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = 0.1 * torch.randn(T, V, generator=g, device="cuda") - 13.0
    few = torch.randn(T, V, generator=g, device="cuda")
    kind = torch.arange(T, device="cuda")[:, None] % 4
    at = torch.arange(V, device="cuda")[None]
    eighth = (at - at * 8 // V * V // 8).minimum((V - at * 8 % V) // 8)      # how far from a multiple of V / 8
    some = torch.zeros(T, V, dtype=torch.bool, device="cuda")
    some.scatter_(1, torch.randint(0, V, (T, 12), generator=g, device="cuda"), True)
    chosen = torch.where(kind == 0, at < 15, torch.where(kind == 1, at >= V - 15, torch.where(kind == 2, (eighth < 72) & (at >= 72) & (at < V - 72), some)))
    return g, torch.where(chosen, few, z).to(t_dtype(dtype))


# few rows (blocks, clusters and independent parts of the rows' kernel) and rows that are streamed, by one block and by clusters
@pytest.mark.parametrize("dtype,T,V", [("bf16", 5, 70001), ("f32", 8, 70001), ("bf16", 360, 70001), ("f32", 180, 70001), ("bf16", 9, 140001), ("bf16", 182, 140001), ("f32", 91, 140001),
                                       ("bf16", 94, 270000), ("f32", 49, 270001), ("f32", 600, 40003), ("bf16", 700, 50007)])
def test_no_entry_is_left_out_or_counted_twice(mtf, dtype, T, V):  # noqa: F811
    import torch
    g, z = rows_of_few_entries(dtype, T, V, T + V)
    z64, d = z.double(), delta(V)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    p1 = torch.log_softmax(z64, -1)
    logp = p1.gather(-1, y[:, None])[:, 0]
    lse = torch.logsumexp(z64, -1)
    old, adv = (logp - 0.1).float(), torch.ones(T, device="cuda")
    guard, N, lay = Guarded(), mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, V), TOK + ["vocab"])
    y32 = y.int().view(1, T)
    x = z64.amax(-1, keepdim=True) - z64
    # policy: in one call, and its two directions
    out = {k: guard.empty([1, T], "f32") for k in ("logp", "loss", "lse", "logp2", "dlogp", "loss2")}
    dz, dz2 = guard.empty([1, T, V], dtype), guard.empty([1, T, V], dtype)
    args = (mat(z), y32, row(old), None, row(adv), None, 0.2, 0.25, 0.0)
    mtf.mtf_policy_step(lay, *args, row(out["logp"]), row(out["loss"]), mat(dz))
    mtf.mtf_policy_forward(lay, *args, *[row(out[k]) for k in ("lse", "logp2", "dlogp", "loss2")])
    mtf.mtf_policy_backward(lay, mat(z), y32, row(out["lse"]), row(out["dlogp"]), None, mat(dz2))
    mtf.mtf_device_status()
    guard.check()
    ratio = (logp - old.double()).exp()
    for k, want, tol in (("logp", logp, d + U * logp.abs()), ("logp2", logp, d + U * logp.abs()), ("lse", lse, d + U * lse.abs()), ("loss", -ratio, ratio * (d + 2 * U)),
                         ("loss2", -ratio, ratio * (d + 2 * U)), ("dlogp", -ratio, ratio * (d + 2 * U))):
        all_within(out[k][0], want, tol, k)
    p = p1.exp()
    # (the derivative's coefficient is off by d, too; the backward call's log-sum-exp, and so its exponentials, by a rounding to f32)
    want = (ratio[:, None] * p).scatter_add_(1, y[:, None], -ratio[:, None])
    tol = ratio[:, None] * p * (2 * d + (3 * x + 8) * U) + (d + STEP[dtype] + 4 * U) * want.abs()
    all_within(dz[0], want, tol, "dlogits of the step")
    all_within(dz2[0], want, tol + ratio[:, None] * p * 2 * U * lse.abs()[:, None], "dlogits")
    del want, tol, dz, dz2
    # distillation: powers of one exponential, two of them, one
    K = 4
    ids = torch.randint(0, V, (T, K), generator=g, device="cuda")
    teacher = torch.randn(T, K, generator=g, device="cuda")
    for tau in (2.0, 2.5, 1.0):
        p2 = torch.log_softmax(z64 / tau, -1)
        q = torch.softmax(teacher.double() / tau, -1)
        want_loss = 0.5 * tau ** 2 * (q * (q.log() - p2.gather(-1, ids))).sum(-1) - 0.5 * logp
        lses = torch.stack([torch.logsumexp(z64 / tau, -1), lse], -1)
        want = 0.5 * tau * p2.exp() + 0.5 * p
        tol = 0.5 * tau * p2.exp() * (d + (3 * x / tau + 8) * U) + 0.5 * p * (d + (3 * x + 8) * U)
        off = 0.5 * tau * p2.exp() * 2 * U * lses[:, :1].abs() + 0.5 * p * 2 * U * lses[:, 1:].abs()
        del p2
        want.scatter_add_(-1, ids, -0.5 * tau * q)
        want.scatter_add_(-1, y[:, None], torch.full((T, 1), -0.5, dtype=torch.float64, device="cuda"))
        stats, loss, loss2 = guard.empty([1, T, 2], "f32"), guard.empty([1, T], "f32"), guard.empty([1, T], "f32")
        dz, dz2 = guard.empty([1, T, V], dtype), guard.empty([1, T, V], dtype)
        args = (ids.int().view(1, T, K), N(teacher.view(1, T, K), TOK + ["slot"]), y32, None, tau, 0.5, 0.5)
        mtf.mtf_distill_step(lay, mat(z), *args, row(loss), mat(dz))
        mtf.mtf_distill_forward(lay, mat(z), *args, N(stats, TOK + ["stat"]), row(loss2))
        mtf.mtf_distill_backward(lay, mat(z), *args, N(stats, TOK + ["stat"]), None, mat(dz2))
        mtf.mtf_device_status()
        guard.check()
        for got in (loss, loss2):
            all_within(got[0], want_loss, (0.5 * tau * tau + 0.5) * d + 2 * U * want_loss.abs(), ("loss", tau))
        all_within(stats[0], lses, d + U * lses.abs(), ("stats", tau))
        tol += (STEP[dtype] + 4 * U) * want.abs()
        all_within(dz[0], want, tol, ("dlogits of the step", tau))
        all_within(dz2[0], want, tol + off, ("dlogits", tau))
        del want, tol, off, dz, dz2


# ---- one tensor in two parts of a call ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 33, 512])
def test_logits_that_teach_themselves_and_each_other(mtf, V, dtype):  # noqa: F811
    """All words are the list: against the logits themselves the softened term is 0, against another student's it is the divergence."""
    import torch
    T, tau = 40, 2.0
    g = torch.Generator(device="cuda").manual_seed(V)
    a, b = ((2 * torch.randn(1, T, V, generator=g, device="cuda")).to(t_dtype(dtype)) for _ in range(2))
    N, lay, guard = mtf.named, layout(mtf), Guarded()
    n = {"a": N(a, TOK + ["vocab"]), "b": N(b, TOK + ["vocab"])}
    z = {"a": a[0].double(), "b": b[0].double()}
    as_list = {k: N(t, TOK + ["slot"]) for k, t in (("a", a), ("b", b))}
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda") for _ in range(T)]).int().view(1, T, V)
    in_order = torch.arange(V, device="cuda").expand(1, T, V).contiguous().int()
    d = (V / 32 + 32 + 3 * (np.log(V) + 1) + 8) * U                    # (test_gpu_losses.py's)
    for student, teacher, words in (("a", "a", in_order), ("a", "b", in_order), ("b", "a", ids), ("b", "b", in_order)):
        for desc in (n, as_list):                                      # the very descriptor of the logits, or one of its own
            loss, dz = guard.empty([1, T], "f32"), guard.empty([1, T, V], dtype)
            mtf.mtf_distill_step(lay, n[student], words, desc[teacher], None, None, tau, 1.0, 0.0, N(loss, TOK), N(dz, TOK + ["vocab"]))
            mtf.mtf_device_status()
            guard.check()
            p = torch.log_softmax(z[student] / tau, -1)
            q = torch.zeros(T, V, dtype=torch.float64, device="cuda").scatter_(1, words[0].long(), torch.softmax(z[teacher] / tau, -1))
            want_loss = tau ** 2 * (q * (q.log() - p)).sum(-1)
            all_within(loss[0], want_loss, tau ** 2 * d + U * want_loss.abs(), "loss")
            want = tau * (p.exp() - q)
            x = z[student].amax(-1, keepdim=True) - z[student]
            all_within(dz[0], want, tau * p.exp() * (d + (3 * x / tau + 8) * U) + (STEP[dtype] + 4 * U) * want.abs(), "dlogits")
