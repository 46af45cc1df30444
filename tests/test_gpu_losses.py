"""GPU parity of the losses on stored logits (distillation, policy, preference) against the oracle in 64 bits: every direction and type, vocabularies
that no vector width divides, rows that are masked, empty, infinite or NaN, teachers' lists with empty slots and repeated words, and the calls in a row
as a training step makes them.

Tolerances.  u = 2^-24 is f32's half step.  A row's sum of exponentials adds at most N = V / 32 + 32 positive f32 numbers one after the other (a warp's
lanes share the shortest rows), each exact to the 3 roundings of its argument (z - m, times a rounded factor: 3 u X at an exponent of X) and the 2^-22 of the
exponential: with weights p the arguments' part is 3 u sum p X <= 3 u (log V + 1), so the sum is off by at most
    delta = (N + 3 (log V + 1) + 8) u   relative, and log-sum-exp and logp by delta, absolute.
A gradient's entry k exp2((z - m) a) is off by delta (in k) + (3 X + 8) u of itself.  What is worked out from these in 64 bits and rounded once adds u (f32)
or 2^-8 (bf16) of the value."""
import gc
import itertools
import threading

import numpy as np
import pytest

from helpers import Guarded
from oracle import losses as ol

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
STEP = {"bf16": 2.0 ** -8, "f32": U}
TOK = ["batch", "length"]


@pytest.fixture(scope="module")
def mtf():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1811_02084_b200 as m
    return m


def layout(mtf, mesh=(("all", 1),), rules=()):
    return mtf.mtf_layout(mtf.mtf_mesh_create(list(mesh)), list(rules))


def delta(V):
    return (V / 32 + 32 + 3 * (np.log(V) + 1) + 8) * U


def t_dtype(dtype):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def host(t):
    return t.detach().cpu().double().numpy()


class Case:
    """Seeded inputs of one operator on the GPU and in 64 bits, and room for its results between guard bands."""

    def __init__(self, op, dtype, V, B=3, L=5, K=6, seed=0, masked=True, logits=None):
        import torch
        self.op, self.dtype, self.V, self.B, self.L, self.K = op, dtype, V, B, L, K
        self.lead = ([2] if op == "preference" else []) + [B, L]
        self.tok = (["branch"] if op == "preference" else []) + TOK
        T = int(np.prod(self.lead))
        r = np.random.RandomState(1000 + seed)
        z = 2.0 * r.randn(T, V) if logits is None else logits
        y = r.randint(0, V, T)
        if logits is None:
            z[np.arange(T), y] += 3.0 * r.randn(T) + 2.0
        self.y = y
        self.z_t = torch.from_numpy(z).to(t_dtype(dtype)).cuda().view(*self.lead, V)
        self.z = host(self.z_t).reshape(T, V)
        self.targets = torch.from_numpy(y.astype(np.int32)).cuda().view(self.lead)
        self.w = r.rand(T).astype(np.float32) + 0.5
        if masked:
            self.w[r.rand(T) < 0.25] = 0.0
        self.put("weight", self.w)
        self.dl = (r.randn(B if op == "preference" else T) + 0.1).astype(np.float32)
        with np.errstate(all="ignore"):
            self.logp64 = np.array([ol.token_logp(self.z[t], y[t])[0] for t in range(T)])
        # ratios on both sides of the limits 0.8 and 1.25 and between them, none near a limit
        self.ratio = r.choice([0.4, 0.7, 0.9, 1.0, 1.1, 1.4, 2.5], T)
        self.old, self.ref = (self.logp64 - np.log(self.ratio)).astype(np.float32), (self.logp64 + 0.3 * r.randn(T)).astype(np.float32)
        self.adv = r.randn(T).astype(np.float32)
        self.ids = np.stack([r.permutation(max(V, K))[:K] % V for _ in range(T)]).astype(np.int32)
        self.teacher_t = torch.from_numpy(2.0 * r.randn(T, K)).to(t_dtype(dtype)).cuda()
        if K > 2:
            self.ids[::2, K // 2] = -1                                    # an empty slot
            self.ids[1::3, 1] = self.ids[1::3, 0]                         # a word twice
            self.ids[2::3, 2] = y[2::3]                                   # the label among the words
        self.seq_ref = (0.3 * r.randn(2, B)).astype(np.float32)
        self.guard = Guarded()

    def put(self, name, a, names=None):
        import torch
        import paper_1811_02084_b200 as mtf
        t = torch.from_numpy(np.ascontiguousarray(a)).cuda().view(*self.lead[:len(names) if names else None])
        n = mtf.named(t, names or self.tok)
        setattr(self, "n_" + name, n)
        return n

    def room(self, names, shape, dtype="f32"):
        import paper_1811_02084_b200 as mtf
        t = self.guard.empty(list(shape), dtype)
        return t, mtf.named(t, names)

    @property
    def logits(self):
        import paper_1811_02084_b200 as mtf
        return mtf.named(self.z_t, self.tok + ["vocab"])

    def gradient(self, in_place):
        import paper_1811_02084_b200 as mtf
        t, n = self.room(self.tok + ["vocab"], self.lead + [self.V], self.dtype)
        if in_place:
            t.copy_(self.z_t)
            return t, n, n
        return t, n, self.logits


def close(got, want, tol, what):
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.asarray(tol, np.float64) + 1e-37
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = np.isfinite(want)
    off = np.abs(got - want)[ok] / np.broadcast_to(tol, want.shape)[ok]
    assert off.size == 0 or off.max() <= 1.0, (what, float(off.max()))


def entry_error(z, tau, d):
    """Relative error of k exp((z - m) / tau)."""
    with np.errstate(all="ignore"):
        x = np.where(np.isfinite(z), (np.max(z) - z) / tau, 0.0)
    return d + (3 * np.abs(x) + 8) * U


def policy_reference(c, hp, dl=None):
    d = delta(c.V)
    rows = []
    for t in range(len(c.y)):
        w = float(c.w[t])
        if w == 0:
            rows.append((0.0, 0.0, 0.0, 0.0, 0.0, np.zeros(c.V), np.zeros(c.V), 0.0))
            continue
        logp, lse, g = ol.token_logp(c.z[t], c.y[t])
        loss, dlogp = ol.policy_of_logp(logp, float(c.old[t]), float(c.ref[t]), float(c.adv[t]), *hp)
        ratio, e = np.exp(logp - float(c.old[t])), np.exp(float(c.ref[t]) - logp)
        slope = w * (abs(c.adv[t]) * ratio + hp[2] * e)                    # how fast loss and dlogp move with logp
        coef = w * dlogp * (1.0 if dl is None else float(dl[t]))
        p = np.exp(c.z[t] - lse)
        rows.append((w * loss, logp, lse, w * dlogp, slope, coef * g, abs(coef) * p * entry_error(c.z[t], 1.0, d), coef))
    return rows, d


VOCABS = [1, 2, 3, 7, 8, 9, 15, 17, 100, 1000, 2050, 4099, 8192, 32768, 50001]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("in_place", [False, True])
def test_policy_step(mtf, V, dtype, in_place):
    c = Case("policy", dtype, V, seed=V)
    hp = (0.2, 0.25, 0.05)
    logp, n_logp = c.room(TOK, c.lead)
    loss, n_loss = c.room(TOK, c.lead)
    dz, n_dz, n_z = c.gradient(in_place)
    mtf.mtf_policy_step(layout(mtf), n_z, c.targets, c.put("old", c.old), c.put("ref", c.ref), c.put("adv", c.adv), c.n_weight, *hp, n_logp, n_loss, n_dz)
    mtf.mtf_device_status()
    c.guard.check()
    rows, d = policy_reference(c, hp)
    close(host(logp).ravel(), [r[1] for r in rows], [d + U * abs(r[1]) for r in rows], "logp")
    close(host(loss).ravel(), [r[0] for r in rows], [r[4] * d + U * abs(r[0]) for r in rows], "loss")
    close(host(dz).reshape(-1, V), [r[5] for r in rows], [r[4] * d * np.abs(r[5] / r[7] if r[7] else 0.0) + r[6] + (STEP[dtype] + 2 * U) * np.abs(r[5]) for r in rows], "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 9, 1000, 4099, 32768])
@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_forward_and_backward(mtf, V, dtype, kl):
    c = Case("policy", dtype, V, seed=V + 1)
    hp = (0.2, float("inf"), kl)
    room = {k: c.room(TOK, c.lead) for k in ("lse", "logp", "dlogp", "loss")}
    lay = layout(mtf, [("rows", 1)], [])
    mtf.mtf_policy_forward(lay, c.logits, c.targets, c.put("old", c.old), c.put("ref", c.ref) if kl else None, c.put("adv", c.adv), c.n_weight, *hp, room["lse"][1],
                           room["logp"][1], room["dlogp"][1], room["loss"][1])
    dz, n_dz, _ = c.gradient(False)
    mtf.mtf_policy_backward(lay, c.logits, c.targets, room["lse"][1], room["dlogp"][1], c.put("dloss", c.dl), n_dz)
    dz1, n_dz1, _ = c.gradient(False)
    mtf.mtf_policy_backward(lay, c.logits, c.targets, room["lse"][1], room["dlogp"][1], None, n_dz1)
    mtf.mtf_device_status()
    c.guard.check()
    rows, d = policy_reference(c, hp)
    got = {k: host(t).ravel() for k, (t, _) in room.items()}
    close(got["lse"], [r[2] for r in rows], [d + U * abs(r[2]) for r in rows], "lse")
    close(got["logp"], [r[1] for r in rows], [d + U * abs(r[1]) for r in rows], "logp")
    close(got["dlogp"], [r[3] for r in rows], [r[4] * d + U * abs(r[3]) for r in rows], "dlogp")
    close(got["loss"], [r[0] for r in rows], [r[4] * d + U * abs(r[0]) for r in rows], "loss")
    for dz, dl in ((dz, c.dl.astype(np.float64)), (dz1, np.ones(len(c.y)))):
        # from the values that the forward call stored
        coef = got["dlogp"] * dl
        p = np.where(c.w[:, None] != 0, np.exp(c.z - got["lse"][:, None]), 0.0)
        g = (np.arange(V) == c.y[:, None]) - p
        err = np.stack([entry_error(z, 1.0, 2 * U) for z in c.z]) + 2 * U * np.abs(got["lse"])[:, None]
        close(host(dz).reshape(-1, V), coef[:, None] * g, np.abs(coef)[:, None] * (p * err + (STEP[dtype] + 2 * U) * np.abs(g)), "dlogits")


def distill_reference(c, tau, soft, hard, dl=None):
    rows = []
    teacher = host(c.teacher_t)
    for t in range(len(c.y)):
        w = float(c.w[t])
        if w == 0:
            rows.append((0.0, 0.0, 0.0, np.zeros(c.V), np.zeros(c.V)))
            continue
        loss, g, l0, l1 = ol.distill_row(c.z[t], c.ids[t], teacher[t], int(c.y[t]), tau, soft, hard)
        s = w * (1.0 if dl is None else float(dl[t]))
        d = delta(c.V) + U * (abs(l0) + abs(l1))
        part = np.zeros(c.V)
        if soft and l0:
            part += soft * tau * np.exp(c.z[t] / tau - l0) * entry_error(c.z[t], tau, d)
        if hard:
            part += hard * np.exp(c.z[t] - l1) * entry_error(c.z[t], 1.0, d)
        rows.append((w * loss, l0, l1, s * g, abs(s) * part))
    return rows


MIXES = [(1.0, 1.0, 0.0), (2.0, 0.75, 0.25), (1.5, 1.0, 0.0), (1.0, 0.5, 0.5), (2.0, 0.0, 1.0), (0.5, 0.5, 0.5)]


def run_distill(mtf, c, tau, soft, hard, targets="given", lay=None):
    """Step, forward and backward; results in 64 bits."""
    lay = lay or layout(mtf)
    teacher = (__import__("torch").from_numpy(c.ids).cuda().view(*c.lead, c.K), mtf.named(c.teacher_t.view(*c.lead, c.K), TOK + ["slot"]),
               c.targets if targets == "given" else None, c.n_weight, tau, soft, hard)
    loss, n_loss = c.room(TOK, c.lead)
    dz, n_dz, n_z = c.gradient(True)
    mtf.mtf_distill_step(lay, n_z, *teacher, n_loss, n_dz)
    loss2, n_loss2 = c.room(TOK, c.lead)
    stats, n_stats = c.room(TOK + ["stat"], c.lead + [2])
    mtf.mtf_distill_forward(lay, c.logits, *teacher, n_stats, n_loss2)
    dz2, n_dz2, _ = c.gradient(False)
    mtf.mtf_distill_backward(lay, c.logits, *teacher, n_stats, c.put("dloss", c.dl), n_dz2)
    return [host(t) for t in (loss, dz, loss2, stats, dz2)]


def check_distill(mtf, c, tau, soft, hard, **kw):
    loss, dz, loss2, stats, dz2 = run_distill(mtf, c, tau, soft, hard, **kw)
    mtf.mtf_device_status()
    c.guard.check()
    V, d = c.V, delta(c.V)
    rows = distill_reference(c, tau, soft, hard)
    tol = [abs(float(w)) * (soft * tau * tau + hard) * d + U * abs(r[0]) for w, r in zip(c.w, rows)]
    close(loss.ravel(), [r[0] for r in rows], tol, "loss of the step")
    close(loss2.ravel(), [r[0] for r in rows], tol, "loss")
    for i in (0, 1):
        close(stats.reshape(-1, 2)[:, i], [r[1 + i] for r in rows], [d + U * abs(r[1 + i]) for r in rows], "stats")
    close(dz.reshape(-1, V), [r[3] for r in rows], [r[4] + (STEP[c.dtype] + 4 * U) * np.abs(r[3]) for r in rows], "dlogits of the step")
    rows = distill_reference(c, tau, soft, hard, c.dl)
    close(dz2.reshape(-1, V), [r[3] for r in rows], [r[4] + (STEP[c.dtype] + 4 * U) * np.abs(r[3]) for r in rows], "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 3, 8, 17, 1000, 4099, 32768, 50001])
@pytest.mark.parametrize("mix", MIXES, ids=str)
def test_distillation(mtf, V, dtype, mix):
    check_distill(mtf, Case("distill", dtype, V, K=min(6, V), seed=V), *mix, targets="given" if mix[2] else None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 9, 1003, 40000])
@pytest.mark.parametrize("mix", [(1.5, 0.25, 0.75), (3.0, 0.5, 0.5), (4.0, 0.75, 0.25), (2.5, 0.5, 0.5), (100.0, 0.5, 0.5)], ids=str)
def test_distillation_at_other_temperatures(mtf, V, dtype, mix):
    check_distill(mtf, Case("distill", dtype, V, K=min(6, V), seed=V + 2), *mix)


@pytest.mark.parametrize("tau", [1.5, 2.0, 3.0, 4.0, 2.5])
def test_a_term_of_little_weight_keeps_its_rows(mtf, tau):
    """Rows whose words lie far apart, and one of the two terms alone but for a weight of 2^-30 of the other."""
    for soft, hard in ((1.0, 2.0 ** -30), (2.0 ** -30, 1.0)):
        c = Case("distill", "f32", 5000, K=6, seed=17, masked=False, logits=8.0 * np.random.RandomState(17).randn(15, 5000))
        check_distill(mtf, c, tau, soft, hard)


@pytest.mark.parametrize("K", [1, 2, 31, 32, 33, 100, 256, 257, 512])
def test_distillation_lists(mtf, K):
    c = Case("distill", "f32", 2000, K=K, seed=K, B=2, L=3)
    c.ids[-1] = -1 if K > 1 else c.ids[-1]                                  # no word at all
    if K > 30:
        c.ids[0, :] = c.ids[0, 0]                                           # one word in all slots
        c.ids[1, 20:] = c.ids[1, :K - 20][::-1][:K - 20]                    # many words more than once
    check_distill(mtf, c, 2.0, 0.6, 0.4)


def preference_reference(c, kind, beta, smoothing, dl):
    d = delta(c.V)
    T = len(c.y)
    logp, lse, g = np.zeros(T), np.zeros(T), np.zeros((T, c.V))
    for t in range(T):
        if c.w[t]:
            logp[t], lse[t], g[t] = ol.token_logp(c.z[t], c.y[t])
    w = c.w.astype(np.float64).reshape(2, c.B, c.L)
    lp = logp.reshape(w.shape)
    seq, off = (w * lp).sum(-1), (np.abs(w) * (d + U * np.abs(lp))).sum(-1)
    margin, moff = (seq[0] - c.seq_ref[0]) - (seq[1] - c.seq_ref[1]), off[0] + off[1]
    out = [ol.preference_of_margin(float(m), kind, beta, smoothing) for m in margin]
    return logp, lse, g, seq, off, np.array([o[0] for o in out]), np.array([o[1] for o in out]), moff


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 9, 1000, 4099, 32768])
@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.2), ("hinge", 0.0), ("squared", 0.0)])
def test_preference(mtf, V, dtype, kind, smoothing):
    c = Case("preference", dtype, V, B=3, L=7, seed=V)
    c.w[:7] = 0.0                                                            # an answer without any token that counts
    c.put("weight", c.w)
    beta, lay = float(np.float32(0.3)), layout(mtf)
    smoothing = float(np.float32(smoothing))
    pair, room = ["branch", "batch"], {}
    for k, names, shape in (("lse", c.tok, c.lead), ("logp", c.tok, c.lead), ("seq", pair, [2, 3]), ("dseq", pair, [2, 3]), ("loss", ["batch"], [3])):
        room[k] = c.room(names, shape)
    mtf.mtf_preference_forward(lay, c.logits, c.targets, c.n_weight, c.put("seq_ref", c.seq_ref, pair), kind, beta, smoothing, *[room[k][1] for k in ("lse", "logp", "seq", "dseq", "loss")])
    import torch
    dl = torch.from_numpy(c.dl).cuda()
    got = {k: host(t) for k, (t, _) in room.items()}
    grads = []
    for in_place, n_dl in ((False, mtf.named(dl, ["batch"])), (True, None)):
        dz, n_dz, n_z = c.gradient(in_place)
        mtf.mtf_preference_backward(lay, n_z, c.targets, c.n_weight, room["lse"][1], room["dseq"][1], n_dl, n_dz)
        grads.append(host(dz).reshape(-1, V))
    mtf.mtf_device_status()
    c.guard.check()
    logp, lse, g, seq, off, loss, dm, moff = preference_reference(c, kind, beta, smoothing, None)
    d = delta(V)
    close(got["lse"].ravel(), lse, d + U * np.abs(lse), "lse")
    close(got["logp"].ravel(), logp, d + U * np.abs(logp), "logp")
    close(got["seq"], seq, off + U * np.abs(seq), "seq_logp")
    bend = {"sigmoid": beta * beta / 4, "hinge": 0.0, "squared": 2.0}[kind]
    close(got["loss"], loss, np.abs(dm) * moff + bend * moff ** 2 + U * np.abs(loss), "loss")
    close(got["dseq"], np.stack([dm, -dm]), bend * moff + U * np.abs(dm), "dseq")
    # the gradient from the values that the forward call stored
    for got_dz, dl in zip(grads, (c.dl.astype(np.float64), np.ones(3))):
        coef = (c.w.astype(np.float64).reshape(2, 3, 7) * (got["dseq"] * dl)[:, :, None]).ravel()
        p = np.where(c.w[:, None] != 0, np.exp(c.z - got["lse"].reshape(-1, 1)), 0.0)
        gg = (np.arange(V) == c.y[:, None]) - p
        err = np.stack([entry_error(z, 1.0, 2 * U) for z in c.z]) + 2 * U * np.abs(got["lse"].reshape(-1, 1))
        close(got_dz, coef[:, None] * gg, np.abs(coef)[:, None] * (p * err + (STEP[dtype] + 4 * U) * np.abs(gg)), "dlogits")


def test_one_pair_without_pair_dimensions(mtf):
    import torch
    c = Case("preference", "bf16", 100, B=1, L=4, seed=5)
    c.lead, c.tok = [2, 4], ["branch", "length"]
    n = lambda a, names: mtf.named(torch.from_numpy(np.ascontiguousarray(a)).cuda(), names)     # noqa: E731
    z, y, w, ref = mtf.named(c.z_t.view(2, 4, 100), ["branch", "length", "vocab"]), c.targets.view(2, 4), n(c.w.reshape(2, 4), c.tok), n(c.seq_ref[:, 0], ["branch"])
    room = {k: c.room(names, shape) for k, names, shape in (("lse", c.tok, [2, 4]), ("logp", c.tok, [2, 4]), ("seq", ["branch"], [2]), ("dseq", ["branch"], [2]), ("loss", ["one"], [1]))}
    mtf.mtf_preference_forward(layout(mtf), z, y, w, ref, mtf.MTF_PREFERENCE_SIGMOID, 0.5, 0.0, *[v[1] for v in room.values()])
    mtf.mtf_device_status()
    c.guard.check()
    _, _, _, seq, off, loss, dm, moff = preference_reference(c, "sigmoid", 0.5, 0.0, None)
    close(host(room["seq"][0]), seq[:, 0], off[:, 0] + U * np.abs(seq[:, 0]), "seq_logp")
    close(host(room["loss"][0]), loss, np.abs(dm) * moff + moff ** 2 / 16 + U * np.abs(loss), "loss")


# ---- values that rows are masked with, and rows that are not finite -----------------------------------------------------------------------------

def special_logits(V, dtype):
    low = {"bf16": -3.3895313892515355e38, "f32": -3.4028234663852886e38}[dtype]
    r = np.random.RandomState(9)
    z = 2.0 * r.randn(10, V)
    z[0, V // 2:] = -np.inf                       # words that are masked, by infinity and by the type's lowest value
    z[1, V // 2:] = low
    z[2, :] = low                                 # ... all of them
    z[3, :] = -np.inf
    z[4, 3] = np.nan
    z[5, 5] = np.inf
    z[6, :] += 3.0e4                              # far from zero
    z[7, :] *= 1.0e30                             # one word far above the rest
    z[8, :] = np.nan                              # weight 0 (below): not looked at
    z[9, :] = 0.0                                 # all the same
    return z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 1003, 20000])
def test_special_rows(mtf, V, dtype):
    hp = (0.2, 0.25, 0.0)
    c = Case("policy", dtype, V, B=2, L=5, seed=3, masked=False, logits=special_logits(V, dtype))
    c.w[8] = 0.0
    c.put("weight", c.w)
    c.y[:] = 1
    c.y[7] = int(c.z[7].argmax())
    c.targets.copy_(__import__("torch").from_numpy(c.y).view(2, 5))
    with np.errstate(all="ignore"):
        logp = np.array([ol.token_logp(z, y)[0] for z, y in zip(c.z, c.y)])
    c.old = np.where(np.isfinite(logp), logp, 0.0).astype(np.float32)
    out, n_logp = c.room(TOK, c.lead)
    loss, n_loss = c.room(TOK, c.lead)
    dz, n_dz, n_z = c.gradient(True)
    mtf.mtf_policy_step(layout(mtf), n_z, c.targets, c.put("old", c.old), None, c.put("adv", c.adv), c.n_weight, *hp, n_logp, n_loss, n_dz)
    mtf.mtf_device_status()
    c.guard.check()
    got, g = host(out).ravel(), host(dz).reshape(10, V)
    bad = [3, 4, 5]
    assert np.isnan(got[bad]).all() and np.isnan(host(loss).ravel()[bad]).all() and np.isnan(g[bad]).all()
    assert got[8] == 0 and host(loss).ravel()[8] == 0 and not g[8].any()
    fine = [0, 1, 2, 6, 7, 9]
    d = delta(V)
    # (row 2's words are all alike, 3.4e38 below zero: logp is a difference there as everywhere)
    want = logp.copy()
    want[2] = -np.log(V)
    close(got[fine], want[fine], d + U * np.abs(want[fine]) + U * 8, "logp")
    for t in fine:
        p = ol.softmax(c.z[t]) if t != 2 else np.full(V, 1.0 / V)
        # the derivative's coefficient from the kernel's own logp, which the old one's rounding stands against
        ratio = np.exp(want[t] - float(c.old[t])) if t != 2 else np.exp(got[t] - float(c.old[t]))
        if not 0.81 < ratio < 1.24:
            continue
        coef = -float(c.w[t]) * float(c.adv[t]) * ratio
        want_g = coef * ((np.arange(V) == c.y[t]) - p)
        close(g[t], want_g, abs(coef) * p * entry_error(c.z[t] if t not in (1, 2) else np.zeros(V), 1.0, 3 * d + 4 * U) + (STEP[dtype] + 4 * U + 2 * d) * np.abs(want_g), ("dlogits", t))


def test_special_teachers(mtf):
    V, K = 50, 4
    c = Case("distill", "f32", V, B=2, L=5, K=K, seed=11, masked=False)
    t = host(c.teacher_t)
    c.ids[:] = np.arange(K) + 3
    c.ids[:, 3] = -1
    t[:, 3] = np.nan                                   # an empty slot's value is not looked at
    t[1, 1] = -np.inf                                  # a word that the teacher rules out
    t[2, :3] = -np.inf                                 # ... all of them: no list
    t[3, 0] = np.nan
    t[4, 0] = 1.0e30                                   # all its weight on one word
    c.z[5, 3] = -np.inf                                # the student rules out what the teacher does not
    c.z[6, 4], t[6, 1] = -np.inf, -np.inf              # both rule it out
    c.ids[7, :] = -1
    import torch
    c.teacher_t = torch.from_numpy(t).float().cuda()
    c.z_t.view(-1, V).copy_(torch.from_numpy(c.z))
    c.y[:] = 20
    c.targets.fill_(20)
    tau, soft, hard = 2.0, 0.5, 0.5
    with np.errstate(all="ignore"):
        loss, dz, loss2, stats, dz2 = run_distill(mtf, c, tau, soft, hard)
        mtf.mtf_device_status()
        c.guard.check()
        rows = distill_reference(c, tau, soft, hard)
    loss, loss2, dz = loss.ravel(), loss2.ravel(), dz.reshape(-1, V)
    assert np.isnan(loss[3]) and np.isnan(loss2[3]) and np.isnan(dz[3, 3:6]).all()
    assert loss[5] == np.inf and loss2[5] == np.inf
    ok = [0, 1, 2, 4, 6, 7, 8, 9]
    tol = np.array([float(w) * (soft * tau * tau + hard) * delta(V) + U * abs(r[0]) for w, r in zip(c.w, rows)])
    close(loss[ok], [rows[t][0] for t in ok], tol[ok], "loss")
    close(loss2[ok], [rows[t][0] for t in ok], tol[ok], "loss")
    for t in ok + [5]:
        close(dz[t], rows[t][3], rows[t][4] + 4 * U * np.abs(rows[t][3]), ("dlogits", t))


@pytest.mark.parametrize("op", ["policy", "distill"])
def test_ids_out_of_range_are_reported(mtf, op):
    import torch
    V = 70
    c = Case(op, "f32", V, B=1, L=4, K=3, seed=12, masked=False)
    c.w[3] = 0.0
    c.put("weight", c.w)
    targets = c.targets.clone()
    targets[0, 1], targets[0, 3] = V, -7                       # the second one belongs to a row that is not looked at
    for bad in (targets, c.targets):
        loss, n_loss = c.room(TOK, c.lead)
        logp, n_logp = c.room(TOK, c.lead)
        dz, n_dz, _ = c.gradient(False)
        if op == "policy":
            mtf.mtf_policy_step(layout(mtf), c.logits, bad, c.put("old", c.old), None, c.put("adv", c.adv), c.n_weight, 0.2, 0.25, 0.0, n_logp, n_loss, n_dz)
        else:
            ids = torch.from_numpy(c.ids).cuda().view(1, 4, 3)
            ids[0, 2, 0] = V + 5 if bad is c.targets else 4    # ... or a teacher's word
            mtf.mtf_distill_step(layout(mtf), c.logits, ids, mtf.named(c.teacher_t.view(1, 4, 3), TOK + ["slot"]), bad, c.n_weight, 2.0, 0.5, 0.5, n_loss, n_dz)
        if bad is targets or op == "distill":
            with pytest.raises(mtf.MtfError) as e:
                mtf.mtf_device_status()
            assert e.value.code == "MTF_ERR_INVALID_ARG"
        mtf.mtf_device_status()
        c.guard.check()
        if bad is targets:
            # (a row of the policy's whose ratio is cut off has a gradient of 0 of its own)
            moves = [r[7] != 0 for r in policy_reference(c, (0.2, 0.25, 0.0))[0]] if op == "policy" else [True] * 4
            assert float(loss[0, 1]) == 0 and not dz[0, 1].any() and bool(dz[0, 0].any()) == moves[0] and bool(dz[0, 2].any()) == moves[2]
        assert float(loss[0, 3]) == 0 and not dz[0, 3].any()


# ---- shapes of a launch: few rows, many rows, one launch behind another ---------------------------------------------------------------------------

@pytest.mark.parametrize("B,L,V", [(1, 1, 200000), (1, 2, 131072), (1, 9, 70001), (1, 40, 50000), (1, 75, 40000), (4, 90, 1111), (9, 333, 515), (2, 100, 120000), (148, 64, 2100), (66, 148, 1030), (33, 63, 70001)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_vocabularies_in_bulk(mtf, B, L, V, dtype):
    """Against torch in 64 bits on the GPU: numbers of rows on both sides of what fills the GPU, rows on both sides of what an SM keeps."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(B * L + V)
    z = (2 * torch.randn(B, L, V, generator=g, device="cuda")).to(t_dtype(dtype))
    y = torch.randint(0, V, (B, L), generator=g, device="cuda")
    w = (torch.rand(B, L, generator=g, device="cuda") > 0.2).float()
    w[0, 0] = 1.0
    teacher_ids = torch.randint(0, V, (B, L, 5), generator=g, device="cuda")
    teacher = torch.randn(B, L, 5, generator=g, device="cuda")
    z64, live = z.double(), w[..., None] != 0
    guard = Guarded()
    N, lay, d = mtf.named, layout(mtf), delta(V)
    loss, dz = guard.empty([B, L], "f32"), guard.empty([B, L, V], dtype)
    tau = 2.0
    p1, p2 = torch.log_softmax(z64, -1), torch.log_softmax(z64 / tau, -1)
    q = torch.softmax(teacher.double() / tau, -1)
    want_loss = w * (0.5 * tau ** 2 * (q * (q.log() - p2.gather(-1, teacher_ids))).sum(-1) - 0.5 * p1.gather(-1, y[..., None])[..., 0])
    want = 0.5 * tau * p2.exp() + 0.5 * p1.exp()
    tol = want * (d + U * 8 + 3 * U * (z64.amax(-1, keepdim=True) - z64))
    want.scatter_add_(-1, teacher_ids, -0.5 * tau * q)
    want.scatter_add_(-1, y[..., None], torch.full_like(y[..., None], -0.5, dtype=torch.float64))
    want = torch.where(live, want, 0.0)
    mtf.mtf_distill_step(lay, N(z, TOK + ["vocab"]), teacher_ids.int(), N(teacher, TOK + ["slot"]), y.int(), N(w, TOK), tau, 0.5, 0.5, N(loss, TOK), N(dz, TOK + ["vocab"]))
    mtf.mtf_device_status()
    assert bool(((loss.double() - want_loss).abs() <= 2.5 * d * w + U * want_loss.abs()).all())
    assert bool(((dz.double() - want).abs() <= tol + (STEP[dtype] + 4 * U) * want.abs()).all())
    # the two directions one after the other agree with the step to the same bounds
    stats, dz2 = guard.empty([B, L, 2], "f32"), guard.empty([B, L, V], dtype)
    args = (teacher_ids.int(), N(teacher, TOK + ["slot"]), y.int(), N(w, TOK), tau, 0.5, 0.5)
    mtf.mtf_distill_forward(lay, N(z, TOK + ["vocab"]), *args, N(stats, TOK + ["stat"]), N(loss, TOK))
    mtf.mtf_distill_backward(lay, N(z, TOK + ["vocab"]), *args, N(stats, TOK + ["stat"]), None, N(dz2, TOK + ["vocab"]))
    lse = torch.where(live, torch.stack([torch.logsumexp(z64 / tau, -1), torch.logsumexp(z64, -1)], -1), 0.0)
    assert bool(((stats.double() - lse).abs() <= d + U * lse.abs()).all())
    assert bool(((loss.double() - want_loss).abs() <= 2.5 * d * w + U * want_loss.abs()).all())
    assert bool(((dz2.double() - want).abs() <= tol + U * 30 * (tol > 0) * want.abs() + (STEP[dtype] + 34 * U) * want.abs() + 30 * U * (0.5 * tau * p2.exp() + 0.5 * p1.exp())).all())
    guard.check()


def rows_of_every_kind(dtype, T, V, seed, skipped):
    """Logits on the GPU, row t of kind t * 7 % 16: masked by infinity (1) and by the type's lowest value (2), all lowest (3), all -infinity (4), with a NaN (5)
    and an infinity (6), far from zero (7), one word far above the rest (8), all alike (9), and ordinary ones; targets among the words that are not masked;
    weights, a share of them 0 (those rows hold NaN)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (2 * torch.randn(T, V, generator=g, device="cuda")).to(t_dtype(dtype))
    kind = torch.arange(T, device="cuda") * 7 % 16
    low = torch.finfo(z.dtype).min
    half = V // 2
    z[kind == 1, half:] = float("-inf")
    z[kind == 2, half:] = low
    z[kind == 3] = low
    z[kind == 4] = float("-inf")
    z[kind == 5, V // 3] = float("nan")
    z[kind == 6, V - 1] = float("inf")
    z[kind == 7] += 3.0e4
    z[kind == 8] *= 1.0e30
    z[kind == 9] = 1.5
    y = torch.randint(0, half, (T,), generator=g, device="cuda")
    y[kind == 8] = z[kind == 8].argmax(-1)
    w = 0.5 + torch.rand(T, generator=g, device="cuda")
    w[torch.rand(T, generator=g, device="cuda") < skipped] = 0.0
    z[w == 0, V // 2] = float("nan")
    return g, z, kind, y, w


# few rows and short ones (blocks and clusters of the rows' kernel), and numbers of rows and words for which rows are streamed: one block a row
# and clusters of 2 to 8, whole pieces and ragged ones, more than 32 and 64 rows a block
KINDS = [("f32", 30, 5003), ("bf16", 40, 40000), ("bf16", 300, 2000), ("f32", 1600, 9000), ("bf16", 1600, 17001), ("bf16", 9600, 16411), ("f32", 700, 20480),
         ("f32", 400, 36001), ("bf16", 250, 140001), ("f32", 90, 150000), ("f32", 60, 270000)]


def in_guard(guard, t, dtype, in_place):
    d = guard.empty(list(t.shape), dtype)
    if not in_place:
        return t, d
    d.copy_(t)
    return d, d


def all_within(got, want, tol, what):
    """Entries alike, or NaN in both."""
    off = (got.double() - want).abs() > tol.nan_to_num(nan=0.0) + 1e-37
    off &= ~(got.isnan() & want.isnan())
    off |= got.isnan() != want.isnan()
    off &= ~((got.double() == want) & want.isinf())
    assert not bool(off.any()), (what, off.nonzero()[:5].tolist())


@pytest.mark.parametrize("dtype,T,V", KINDS)
@pytest.mark.parametrize("skipped", [0.1, 0.95])
def test_policy_rows_of_every_kind(mtf, dtype, T, V, skipped):
    """Every fifth row's gradient is 0 by a cut ratio.  Against torch in 64 bits on the GPU."""
    import torch
    g, z, kind, y, w = rows_of_every_kind(dtype, T, V, T + V, skipped)
    z64, d = z.double(), delta(V)
    lp = torch.log_softmax(z64, -1)
    logp = lp.gather(-1, y[:, None])[:, 0]
    ratio = torch.tensor([0.4, 0.7, 0.9, 1.1, 2.5], dtype=torch.float64, device="cuda")[torch.randint(0, 5, (T,), generator=g, device="cuda")]
    old = torch.where(logp.isnan(), 0.0, logp - ratio.log()).float()
    adv = torch.randn(T, generator=g, device="cuda")
    adv[::5], old[::5] = adv[::5].abs(), torch.where(logp.isnan(), 0.0, logp - 1.0)[::5].float()      # ratio e, cut at 1.25
    guard = Guarded()
    zin, dz = in_guard(guard, z, dtype, T % 3 == 0)
    out_logp, loss = guard.empty([1, T], "f32"), guard.empty([1, T], "f32")
    N, lay = mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, V), TOK + ["vocab"])
    mtf.mtf_policy_step(lay, mat(zin), y.int().view(1, T), row(old), None, row(adv), row(w), 0.2, 0.25, 0.0, row(out_logp), row(loss), mat(dz))
    mtf.mtf_device_status()
    guard.check()
    rat = (logp - old.double()).exp()
    plain, clipped = rat * adv, rat.clamp(0.8, 1.25) * adv
    cut = plain > clipped
    live = w != 0
    slope = w * adv.abs() * rat
    want_loss = torch.where(live, -w * torch.where(cut, clipped, plain), 0.0)
    coef = torch.where(cut, 0.0, -w * plain)
    all_within(out_logp[0], torch.where(live, logp, 0.0), d + U * logp.abs(), "logp")
    all_within(loss[0], want_loss, slope * d + 2 * U * want_loss.abs(), "loss")
    p = lp.exp()
    x = torch.where(z64.isfinite(), z64.amax(-1, keepdim=True) - z64, 0.0)
    want = -coef[:, None] * p
    tol = coef.abs()[:, None] * p * (d + (3 * x + 8) * U)
    want.scatter_add_(-1, y[:, None], coef[:, None])
    want = torch.where((live & ~cut)[:, None], want, 0.0)
    # (the label's entry is the difference c - c p: where p is 1 it is 0 with the error of c p, |c| p (d + ...), which a bound on its own size would leave out)
    all_within(dz, want, torch.where((live & ~cut)[:, None], tol + (d + STEP[dtype] + 4 * U) * want.abs(), 0.0), "dlogits")


@pytest.mark.parametrize("dtype,T,V", KINDS)
@pytest.mark.parametrize("mix,K", [((1.0, 0.5, 0.5), 3), ((2.0, 0.75, 0.25), 40), ((1.5, 0.5, 0.5), 130), ((0.7, 1.0, 0.0), 512)], ids=str)
def test_distillation_rows_of_every_kind(mtf, dtype, T, V, mix, K):
    """Lists with empty slots, words more than once, the label among the words, and no word at all.  Against torch in 64 bits on the GPU."""
    import torch
    tau, soft, hard = (float(np.float32(v)) for v in mix)            # (as the call takes them)
    g, z, kind, y, w = rows_of_every_kind(dtype, T, V, T + V + K, 0.15)
    ids = torch.randint(0, V // 2, (T, K), generator=g, device="cuda")
    ids[::3, K // 2:] = ids[::3, :K - K // 2]                        # words twice
    ids[1::4, 0] = y[1::4]
    ids[torch.rand(T, K, generator=g, device="cuda") < 0.1] = -1
    ids[5::11] = -1
    teacher = (2 * torch.randn(T, K, generator=g, device="cuda")).to(t_dtype(dtype))
    teacher[ids < 0] = float("nan")                                  # (not looked at)
    z64, d = z.double(), delta(V)
    p1, p2 = torch.log_softmax(z64, -1), torch.log_softmax(z64 / tau, -1)
    used = ids >= 0
    at, some = ids.clamp(min=0), used.any(-1, keepdim=True)
    q = torch.softmax(torch.where(used, teacher.double() / tau, float("-inf")), -1)
    q = torch.where(used, q, 0.0)
    term = torch.where(used & (q > 0), q * (q.log() - p2.gather(-1, at)), 0.0)
    live = w != 0
    want_loss = torch.where(live, w * (soft * tau ** 2 * term.sum(-1) - (hard * p1.gather(-1, y[:, None])[:, 0] if hard else 0.0)), 0.0)
    s = soft * some
    x = torch.where(z64.isfinite(), z64.amax(-1, keepdim=True) - z64, 0.0)
    want, tol = s * tau * p2.exp(), s * tau * p2.exp() * (d + (3 * x / tau + 8) * U)
    if hard:
        want, tol = want + hard * p1.exp(), tol + hard * p1.exp() * (d + (3 * x + 8) * U)
    del x, p1, p2
    want.scatter_add_(-1, at, -s * tau * q)
    want.scatter_add_(-1, y[:, None], torch.full((T, 1), -hard, dtype=torch.float64, device="cuda"))
    want, tol = want * w[:, None], tol * w[:, None]
    want = torch.where(live[:, None], want, 0.0)
    nothing = ~(some[:, 0] | bool(hard)) | ~live
    want[nothing], want_loss[nothing] = 0.0, 0.0
    guard = Guarded()
    zin, dz = in_guard(guard, z, dtype, T % 3 == 0)
    loss = guard.empty([1, T], "f32")
    N, lay = mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, -1), TOK + ["vocab"])
    mtf.mtf_distill_step(lay, mat(zin), ids.int().view(1, T, K), N(teacher.view(1, T, K), TOK + ["slot"]), y.int().view(1, T), row(w), tau, soft, hard, row(loss), mat(dz))
    mtf.mtf_device_status()
    guard.check()
    all_within(loss[0], want_loss, w * (soft * tau * tau + hard) * d + 2 * U * want_loss.abs(), "loss")
    all_within(dz, want, torch.where(live[:, None], tol + (STEP[dtype] + 4 * U) * want.abs(), 0.0), "dlogits")


def gradient_of_stored(z64, y, lse, coef, dtype):
    """(gradient, tolerance) of coef * (onehot(y) - exp(z - lse)) from the f32 lse that a forward call stored"""
    import torch
    x = torch.where(z64.isfinite(), (z64.amax(-1, keepdim=True) - z64).abs(), 0.0)
    part = coef[:, None] * (z64 - lse.double()[:, None]).exp()
    want = -part
    want.scatter_add_(-1, y[:, None], coef[:, None])
    return want, part.abs() * ((3 * x + 8) * U + 2 * U * lse.double().abs()[:, None].clamp(max=1e6)) + (STEP[dtype] + 4 * U) * want.abs()


@pytest.mark.parametrize("dtype,T,V", [("f32", 30, 5003), ("bf16", 40, 140001), ("bf16", 300, 2000), ("f32", 700, 20480)])
def test_policy_directions_on_rows_of_every_kind(mtf, dtype, T, V):
    import torch
    g, z, kind, y, w = rows_of_every_kind(dtype, T, V, T + V, 0.2)
    z64, d = z.double(), delta(V)
    lse = torch.logsumexp(z64, -1)
    logp = torch.log_softmax(z64, -1).gather(-1, y[:, None])[:, 0]
    old = torch.where(logp.isnan(), 0.0, logp - 0.1).float()
    adv = torch.randn(T, generator=g, device="cuda")
    live = w != 0
    bad = logp.isnan() & live
    assert bool(bad.any()) and bool((~bad & live).any())
    guard = Guarded()
    N, lay = mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, V), TOK + ["vocab"])
    out = {k: guard.empty([1, T], "f32") for k in ("lse", "logp", "dlogp", "loss")}
    mtf.mtf_policy_forward(lay, mat(z), y.int().view(1, T), row(old), None, row(adv), row(w), 0.2, 0.25, 0.0, *[row(out[k]) for k in ("lse", "logp", "dlogp", "loss")])
    zin, dz = in_guard(guard, z, dtype, T % 3 == 0)
    mtf.mtf_policy_backward(lay, mat(zin), y.int().view(1, T), row(out["lse"]), row(out["dlogp"]), None, mat(dz))
    mtf.mtf_device_status()
    guard.check()
    ratio = (logp - old.double()).exp()
    slope = w * adv.abs() * ratio
    for k, want, tol in (("lse", torch.where(bad, float("nan"), lse), d + U * lse.abs()), ("logp", logp, d + U * logp.abs()),
                         ("dlogp", -w * adv * ratio, slope * d + 2 * U * slope), ("loss", -w * adv * ratio, slope * d + 2 * U * slope)):
        got = out[k][0]
        fine = live & ~bad
        all_within(got, torch.where(live, torch.where(bad & got.isnan(), float("nan"), want), 0.0), torch.where(fine, tol, 0.0), k) if k != "lse" else \
            all_within(got[fine], want[fine], tol[fine], k)
    want, tol = gradient_of_stored(z64, y, out["lse"][0], out["dlogp"][0].double(), dtype)
    off = out["dlogp"][0] == 0
    want, tol = torch.where(off[:, None], 0.0, want), torch.where(off[:, None], 0.0, tol)
    want = torch.where(bad[:, None], float("nan"), want)
    all_within(dz, want, tol, "dlogits")


@pytest.mark.parametrize("dtype,T,V", [("f32", 30, 5003), ("bf16", 40, 140001), ("bf16", 300, 2000), ("f32", 700, 20480)])
@pytest.mark.parametrize("mix", [(1.0, 0.5, 0.5), (2.0, 0.75, 0.25), (1.5, 0.5, 0.5), (4.0, 0.5, 0.5), (0.75, 0.5, 0.5)], ids=str)
def test_distillation_directions_on_rows_of_every_kind(mtf, dtype, T, V, mix):
    import torch
    tau, soft, hard = mix
    K = 9
    g, z, kind, y, w = rows_of_every_kind(dtype, T, V, T + V, 0.2)
    ids = torch.stack([torch.randperm(V // 2, generator=g, device="cuda")[:K] for _ in range(T)])
    teacher = torch.randn(T, K, generator=g, device="cuda")
    z64, d = z.double(), delta(V)
    live = w != 0
    lses = torch.stack([torch.logsumexp(z64 / tau, -1), torch.logsumexp(z64, -1)], -1)
    lp, lp2 = torch.log_softmax(z64, -1), torch.log_softmax(z64 / tau, -1)
    bad = live & lp[:, 0].isnan()
    q = torch.softmax(teacher.double() / tau, -1)
    want_loss = w * (soft * tau ** 2 * (q * (q.log() - lp2.gather(-1, ids))).sum(-1) - hard * lp.gather(-1, y[:, None])[:, 0])
    del lp, lp2
    guard = Guarded()
    N, lay = mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, -1), TOK + ["vocab"])
    stats, loss = guard.empty([1, T, 2], "f32"), guard.empty([1, T], "f32")
    args = (ids.int().view(1, T, K), N(teacher.view(1, T, K), TOK + ["slot"]), y.int().view(1, T), row(w), tau, soft, hard)
    mtf.mtf_distill_forward(lay, mat(z), *args, N(stats, TOK + ["stat"]), row(loss))
    zin, dz = in_guard(guard, z, dtype, T % 3 == 0)
    mtf.mtf_distill_backward(lay, mat(zin), *args, N(stats, TOK + ["stat"]), None, mat(dz))
    mtf.mtf_device_status()
    guard.check()
    fine = live & ~bad
    all_within(loss[0], torch.where(live, want_loss, 0.0), w * (soft * tau * tau + hard) * d + 2 * U * want_loss.abs(), "loss")
    in_f32 = lses.float().double()                                     # (all lowest, divided by a temperature below 1: infinity)
    all_within(stats[0][fine], torch.where(in_f32.isinf(), in_f32, lses)[fine], (d + U * lses.abs())[fine], "stats")
    if tau not in (1.0, 2.0, 4.0):
        # An f32 log-sum-exp of 1e30 / tau is off by up to half a step, 2^-24 of it, 4e22: no digit is left of an exponential of the difference, and
        # the formula on the stored number says nothing.  (Powers of two divide without a rounding.)
        lost = live & ((kind == 3) | (kind == 8))
        assert bool(dz[lost].isfinite().all()) and bool((dz[lost].double().abs() <= w[lost, None] * (2 * soft * tau + 2 * hard) * (1 + STEP[dtype])).all())
        live = live & ~lost
        dz = torch.where(lost[:, None], torch.zeros_like(dz), dz)
    l0, l1 = stats[0].double().unbind(-1)
    x = torch.where(z64.isfinite(), z64.amax(-1, keepdim=True) - z64, 0.0)
    part0, part1 = soft * tau * (z64 / tau - l0[:, None]).exp(), hard * (z64 - l1[:, None]).exp()
    want = part0 + part1
    far = torch.minimum(torch.maximum(l0.abs() * tau, l1.abs()), torch.tensor(1e6, dtype=torch.float64, device="cuda"))[:, None]
    tol = part0 * ((3 * x + 4 * far) / tau * U + 8 * U) + part1 * ((3 * x + 4 * far) * U + 8 * U)
    want.scatter_add_(-1, ids, -soft * tau * q)
    want.scatter_add_(-1, y[:, None], torch.full((T, 1), -hard, dtype=torch.float64, device="cuda"))
    want, tol = w[:, None] * want, w[:, None] * tol
    want = torch.where(live[:, None], torch.where(bad[:, None], float("nan"), want), 0.0)
    all_within(dz, want, torch.where(live[:, None], tol + (STEP[dtype] + 4 * U) * want.abs(), 0.0), "dlogits")


@pytest.mark.parametrize("dtype,B,L,V", [("f32", 16, 1, 5003), ("bf16", 24, 1, 2000), ("bf16", 8, 3, 140001), ("f32", 2, 1111, 800)])
def test_preference_on_rows_of_every_kind(mtf, dtype, B, L, V):
    """A pair with a row that is not finite is NaN, and no other; answers longer than a block has threads."""
    import torch
    T = 2 * B * L
    g, z, kind, y, w = rows_of_every_kind(dtype, T, V, T + V, 0.2)
    if L > 1000:                                                       # (one pair without rows that are not finite)
        t = torch.arange(T, device="cuda") % (B * L)
        w[(t < L) & ((kind == 4) | (kind == 5) | (kind == 6))] = 0.0
    z64, d = z.double(), delta(V)
    live = w != 0
    logp = torch.where(live, torch.log_softmax(z64, -1).gather(-1, y[:, None])[:, 0], 0.0)
    seq = (w * logp).view(2, B, L).sum(-1)
    off = (w * (d + U * logp.abs())).view(2, B, L).sum(-1)
    ref = torch.zeros(2, B, device="cuda")
    beta = 0.25
    margin = seq[0] - seq[1]
    want_loss = torch.nn.functional.softplus(-beta * margin)
    want_d = -beta * torch.sigmoid(-beta * margin)
    moff = off[0] + off[1]
    nan = margin.isnan()
    assert bool(nan.any()) and bool((~nan).any())
    guard = Guarded()
    N, lay, tok = mtf.named, layout(mtf), ["branch", "batch", "length"]
    row, mat = lambda t: N(t.view(2, B, L), tok), lambda t: N(t.view(2, B, L, V), tok + ["vocab"])
    lse, got_logp = guard.empty([2, B, L], "f32"), guard.empty([2, B, L], "f32")
    got_seq, dseq, loss = guard.empty([2, B], "f32"), guard.empty([2, B], "f32"), guard.empty([B], "f32")
    pair = lambda t: N(t, ["branch", "batch"])
    y32 = y.int().view(2, B, L)
    mtf.mtf_preference_forward(lay, mat(z), y32, row(w), pair(ref), "sigmoid", beta, 0.0, row(lse), row(got_logp), pair(got_seq), pair(dseq), N(loss, ["batch"]))
    zin, dz = in_guard(guard, z, dtype, True)
    mtf.mtf_preference_backward(lay, mat(zin), y32, row(w), row(lse), pair(dseq), None, mat(dz))
    mtf.mtf_device_status()
    guard.check()
    all_within(got_logp.view(-1), logp, d + U * logp.abs(), "logp")
    all_within(got_seq, seq, off + U * seq.abs(), "seq_logp")
    all_within(loss, want_loss, beta * moff + U * want_loss.abs(), "loss")
    all_within(dseq, torch.stack([want_d, -want_d]), beta * beta / 4 * moff + U * want_d.abs(), "dseq")
    fine = live & ~logp.isnan()
    want_lse = torch.logsumexp(z64, -1)
    all_within(lse.view(-1)[fine], want_lse[fine], (d + U * want_lse.abs())[fine], "lse")
    coef = (w.view(2, B, L) * dseq[:, :, None]).double().view(-1)
    want, tol = gradient_of_stored(z64, y, lse.view(-1), coef, dtype)
    tol = tol + U * (want.abs() + coef.abs()[:, None] * (z64 - lse.view(-1).double()[:, None]).exp())
    want = torch.where(live[:, None], torch.where((logp.isnan() | nan.repeat(2)[:, None].expand(2 * B, L).reshape(-1))[:, None], float("nan"), want), 0.0)
    all_within(dz.view(T, V), want, torch.where(live[:, None], tol, 0.0), "dlogits")


@pytest.mark.parametrize("op", ["policy", "distill"])
@pytest.mark.parametrize("V", [20001, 150000])
def test_streamed_rows_repeat_captured_and_side_by_side(mtf, op, V):
    """Rows of which two launches on two streams share the GPU, a captured launch, and targets out of range among them: the same bits each time."""
    import torch
    T = -(-(52 << 20) // (2 * V))
    g, z, kind, y, w = rows_of_every_kind("bf16", T, V, V, 0.1)
    w[3], y[3] = 1.0, V                                               # reported, its row 0
    N, lay = mtf.named, layout(mtf)
    row, mat = lambda t: N(t.view(1, T), TOK), lambda t: N(t.view(1, T, -1), TOK + ["vocab"])
    old, adv = torch.full((T,), -9.0, device="cuda"), torch.randn(T, generator=g, device="cuda")
    ids, teacher = torch.randint(0, V, (1, T, 16), generator=g, device="cuda").int(), torch.randn(1, T, 16, generator=g, device="cuda")
    y32 = y.int().view(1, T)

    def call():
        loss, logp, dz = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda"), torch.full_like(z, 7.0)

        def run():
            if op == "policy":
                mtf.mtf_policy_step(lay, mat(z), y32, row(old), row(old), row(adv), row(w), 0.2, 0.25, 0.1, row(logp), row(loss), mat(dz))
            else:
                mtf.mtf_distill_step(lay, mat(z), ids, N(teacher, TOK + ["slot"]), y32, row(w), 1.5, 0.5, 0.5, row(loss), mat(dz))
        return run, [loss, logp, dz]

    run, outs = call()
    run()
    with pytest.raises(mtf.MtfError, match="MTF_ERR_INVALID_ARG"):
        mtf.mtf_device_status()
    want = bits(outs)
    assert float(outs[0][3]) == 0 and not outs[2][3].any()
    for t in outs:
        t.fill_(7.0)
    gc.collect()                                                      # (an older graph that is collected during a capture ends it)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bits(outs), want))
    both = [call() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(3):
        for (r, _), st in zip(both, streams):
            with torch.cuda.stream(st):
                r()
    torch.cuda.synchronize()
    for _, o in both:
        assert all(torch.equal(a, b) for a, b in zip(bits(o), want))
    with pytest.raises(mtf.MtfError):
        mtf.mtf_device_status()


def test_offsets_behind_two_to_the_31(mtf):
    """Rows whose elements lie behind 2^31 elements and 2^32 bytes."""
    import torch
    V, T = 131101, 16500                                          # 2.16e9 elements
    z = torch.zeros(1, T, V, dtype=torch.bfloat16, device="cuda")
    dz = torch.empty_like(z)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [0, 8191, 16379, 16380, 16381, T - 1]
    for r in rows:
        z[0, r] = (2 * torch.randn(V, generator=g, device="cuda")).to(z.dtype)
    w = torch.zeros(1, T, device="cuda")
    w[0, rows] = 1.0
    y = torch.full((1, T), 77, dtype=torch.int32, device="cuda")
    adv, old = torch.ones(1, T, device="cuda"), torch.full((1, T), -12.0, device="cuda")
    logp, loss = torch.empty(1, T, device="cuda"), torch.empty(1, T, device="cuda")
    N = mtf.named
    mtf.mtf_policy_step(layout(mtf), N(z, TOK + ["vocab"]), y, N(old, TOK), None, N(adv, TOK), N(w, TOK), 1.0, float("inf"), 0.0, N(logp, TOK), N(loss, TOK), N(dz, TOK + ["vocab"]))
    mtf.mtf_device_status()
    for r in rows:
        lp = torch.log_softmax(z[0, r].double(), -1)
        assert abs(float(logp[0, r]) - float(lp[77])) <= delta(V) + 16 * U
        coef = -torch.exp(lp[77] + 12.0)
        want = -coef * lp.exp()
        want[77] += coef
        assert bool(((dz[0, r].double() - want).abs() <= (STEP["bf16"] + 2 * delta(V) + 60 * U) * want.abs()).all()), r
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[rows] = False
    for k in range(0, T, 1500):
        assert not bool(dz[0, k:k + 1500][others[k:k + 1500]].any())


def step_of(mtf, op, dtype, V, seed, lay=None):
    """(step, outputs) on tensors of its own"""
    import torch
    c = Case(op, dtype, V, B=4, L=6, seed=seed)
    lay = lay or layout(mtf)
    outs = []

    def room(names, shape, dt="f32"):
        t = torch.full(list(shape), float("nan"), dtype=t_dtype(dt), device="cuda")
        outs.append(t)
        return mtf.named(t, names)

    loss, dz = room(TOK if op != "preference" else ["batch"], c.lead if op != "preference" else [4]), room(c.tok + ["vocab"], c.lead + [V], dtype)
    if op == "policy":
        old, ref, adv, logp = c.put("old", c.old), c.put("ref", c.ref), c.put("adv", c.adv), room(TOK, c.lead)
        return lambda: mtf.mtf_policy_step(lay, c.logits, c.targets, old, ref, adv, c.n_weight, 0.2, 0.25, 0.05, logp, loss, dz), outs
    if op == "distill":
        args = (torch.from_numpy(c.ids).cuda().view(*c.lead, c.K), mtf.named(c.teacher_t.view(*c.lead, c.K), TOK + ["slot"]), c.targets, c.n_weight, 2.0, 0.5, 0.5)
        return lambda: mtf.mtf_distill_step(lay, c.logits, *args, loss, dz), outs
    pair = ["branch", "batch"]
    ref, lse, logp, seq, dseq = c.put("seq_ref", c.seq_ref, pair), room(c.tok, c.lead), room(c.tok, c.lead), room(pair, [2, 4]), room(pair, [2, 4])

    def step():
        mtf.mtf_preference_forward(lay, c.logits, c.targets, c.n_weight, ref, "sigmoid", 0.1, 0.0, lse, logp, seq, dseq, loss)
        mtf.mtf_preference_backward(lay, c.logits, c.targets, c.n_weight, lse, dseq, None, dz)
    return step, outs


def bits(outs):
    import torch
    return [t.view(torch.int16 if t.element_size() == 2 else torch.int32).clone() for t in outs]


@pytest.mark.parametrize("op,dtype,V", [(o, d, v) for o in ("policy", "distill", "preference") for d, v in (("bf16", 5003), ("f32", 40000))])
def test_repeats_captured_on_a_stream_and_in_threads(mtf, op, dtype, V):
    import torch
    lay = layout(mtf, [("all", 1)], [])
    step, outs = step_of(mtf, op, dtype, V, 21, lay)
    step()
    mtf.mtf_device_status()
    want = bits(outs)

    def same():
        torch.cuda.synchronize()
        ok = all(torch.equal(a, b) for a, b in zip(bits(outs), want))
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        return ok

    assert same()
    for _ in range(3):
        step()
    assert same()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    graph.replay()
    graph.replay()
    assert same()
    with torch.cuda.stream(side):
        step()
    assert same()
    step2, outs2 = step_of(mtf, op, dtype, V, 21, lay)
    fails = []

    def work(s):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    s()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                           # noqa: BLE001
            fails.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in (step, step2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails
    assert all(torch.equal(a, b) for a, b in zip(bits(outs2), want)) and same()
    mtf.mtf_device_status()


def test_layouts_do_not_change_a_bit(mtf):
    import torch
    got = []
    for mesh, rules in (([("all", 1)], []), ([("all", 4)], [("vocab", "all")]), ([("rows", 2), ("cols", 4)], [("batch", "rows"), ("vocab", "cols")])):
        for op in ("policy", "distill", "preference"):
            step, outs = step_of(mtf, op, "bf16", 1000, 22, layout(mtf, mesh, rules))
            step()
            got.append((op, bits(outs)))
    for (op, a), (op2, b) in itertools.product(got, got):
        if op == op2:
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- as a training step uses them ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("op", ["policy", "distill", "preference"])
def test_training_step_from_hidden_states_to_weights(mtf, op):
    """h . wout -> logits, the loss and its gradient over the logits in place, dh and dwout, and the update of wout: each launch against
    64 bits on what the launch before it left."""
    import torch
    c = Case(op, "bf16", 512, B=2, L=8, seed=31)
    D, V = 64, 512
    lay = layout(mtf, [("rows", 2), ("cols", 4)], [("batch", "rows"), ("vocab", "cols")])
    r = np.random.RandomState(5)
    h = torch.from_numpy(r.randn(*c.lead, D)).to(torch.bfloat16).cuda()
    master = torch.from_numpy(r.randn(D, V) / 8).float().cuda()
    wout = master.to(torch.bfloat16)
    N, ht = mtf.named, c.tok + ["d_model"]
    z, n_z = c.room(c.tok + ["vocab"], c.lead + [V], "bf16")
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    mtf.mtf_einsum(lay, None, [N(h, ht), N(wout, ["d_model", "vocab"])], n_z, None, ws)
    c.z_t = z
    c.z = host(z).reshape(-1, V)
    with torch.no_grad():
        want_z = h.double() @ wout.double()
    assert float((z.double() - want_z).abs().max()) <= 2.0 ** -8 * float(want_z.abs().max()) + 1e-4
    loss, n_loss = c.room(TOK if op != "preference" else ["batch"], c.lead if op != "preference" else [2])
    if op == "policy":
        c.logp64 = np.array([ol.token_logp(zz, y)[0] for zz, y in zip(c.z, c.y)])
        c.old, c.ref = (c.logp64 - np.log(c.ratio)).astype(np.float32), (c.logp64 + 0.2).astype(np.float32)
        _, n_logp = c.room(TOK, c.lead)
        mtf.mtf_policy_step(lay, n_z, c.targets, c.put("old", c.old), c.put("ref", c.ref), c.put("adv", c.adv), c.n_weight, 0.2, 0.25, 0.05, n_logp, n_loss, n_z)
        rows = [x[5] for x in policy_reference(c, (0.2, 0.25, 0.05))[0]]
    elif op == "distill":
        mtf.mtf_distill_step(lay, n_z, torch.from_numpy(c.ids).cuda().view(*c.lead, c.K), N(c.teacher_t.view(*c.lead, c.K), TOK + ["slot"]), c.targets, c.n_weight, 2.0, 0.5, 0.5,
                             n_loss, n_z)
        rows = [x[3] for x in distill_reference(c, 2.0, 0.5, 0.5)]
    else:
        pair = ["branch", "batch"]
        room = {k: c.room(names, shape) for k, names, shape in (("lse", c.tok, c.lead), ("logp", c.tok, c.lead), ("seq", pair, [2, 2]), ("dseq", pair, [2, 2]))}
        mtf.mtf_preference_forward(lay, n_z, c.targets, c.n_weight, c.put("seq_ref", c.seq_ref, pair), "sigmoid", 0.5, 0.0, *[v[1] for v in room.values()], n_loss)
        mtf.mtf_preference_backward(lay, n_z, c.targets, c.n_weight, room["lse"][1], room["dseq"][1], None, n_z)
        _, _, g, _, _, _, dm, _ = preference_reference(c, "sigmoid", 0.5, 0.0, None)
        rows = (c.w.reshape(2, 2, 8) * np.stack([dm, -dm])[:, :, None]).reshape(-1, 1) * g
    dz = host(z).reshape(-1, V)
    rows = np.stack(list(rows))
    assert np.abs(dz - rows).max() <= 2.0 ** -8 * np.abs(rows).max() + 1e-5
    dh, n_dh = c.room(ht, c.lead + [D], "bf16")
    dw, n_dw = c.room(["d_model", "vocab"], [D, V])
    mtf.mtf_einsum(lay, None, [n_z, N(wout, ["d_model", "vocab"])], n_dh, None, ws)
    mtf.mtf_einsum(lay, None, [N(h, ht), n_z], n_dw, None, ws)
    before = master.clone()
    mtf.mtf_update(lay, n_dw, N(master, ["d_model", "vocab"]), None, N(wout, ["d_model", "vocab"]), 0.1)
    mtf.mtf_device_status()
    c.guard.check()
    want_dw = host(h).reshape(-1, D).T @ dz
    assert np.abs(host(dw) - want_dw).max() <= 1e-4 * np.abs(want_dw).max()
    want_dh = dz @ host(before.to(torch.bfloat16)).T
    assert np.abs(host(dh).reshape(-1, D) - want_dh).max() <= 2.0 ** -8 * np.abs(want_dh).max() + 1e-4 * np.abs(want_dh).max()
    assert float((master - (before - 0.1 * dw)).abs().max()) <= 4 * U * float(before.abs().max())
