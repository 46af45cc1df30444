"""GPU parity of answering - paged caches, attention of one new token, beam selection, reordering - against the oracle in 64 bits, and a run of them together
behind the attention block that trains them.

Tolerances of attention, per element of o.  u = 2^-24.  A weight p is rounded to bf16 (2^-8 of it; with an e4m3 cache to f16, 2^-11, or a step of its
subnormals, 2^-25 of a largest weight held as 2^9 or more: 2^-34 each), the result to bf16 (2^-8).  A logit z adds d_k products of magnitudes A = scale sum |q k| in f32, each addition off by at
most 2 u of the sum of magnitudes so far (the tensor cores cut off instead of rounding), and takes three more roundings: it is off by
    delta = (2 d_k u) A + 6 u |z|,   and a weight by 2 delta + 2^-21 (the exponential and its argument's rounding up to 2^3 log2 e u |z - max|, part of 6 u |z| twice).
The sums over n positions add n / 64 terms a lane and join some tens: (n / 32 + 64) 2 u relative to the sum of magnitudes P = sum p |v|.  Hence
    |o - o*| <= 2^-8 |o*| + P (w + 4 delta + 2^-20 + (n / 32 + 64) 4 u) + n 2^-33 max |v|   with w = 2^-8 (bf16: times 1 + 2^-8) or 2^-11, the last term for e4m3 alone."""
import threading

import numpy as np
import pytest

from helpers import Guarded
from oracle import answer as oa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mtf():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1811_02084_b200 as m
    return m


def layout(mtf, mesh=(("all", 1),), rules=()):
    return mtf.mtf_layout(mtf.mtf_mesh_create(list(mesh)), list(rules))


def host(t):
    import torch
    if t.dtype == torch.float8_e4m3fn:
        return oa.E4M3[t.detach().cpu().view(torch.uint8).numpy()]
    return t.detach().cpu().double().numpy()


def ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Paged:
    """A pool of pages with tables in no order; slots that no sequence has reached hold NaN."""

    def __init__(self, mtf, dtype, lengths, heads, dk, dv, slots, slot_first=True, per=None, seed=0, guard=None, spare=3, values=None):
        import torch
        self.mtf, self.dtype, self.slots, self.slot_first, self.heads = mtf, dtype, slots, slot_first, heads
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = np.random.RandomState(seed)
        n_seq = len(lengths)
        self.per = per or max(1, -(-max(lengths) // slots))
        need = [-(-n // slots) for n in lengths]
        self.pages = sum(need) + spare
        order = r.permutation(self.pages)
        table = np.full((n_seq, self.per), -7)                     # (entries behind the pages in use are not read)
        at = 0
        for s, k in enumerate(need):
            table[s, :k] = order[at:at + k]
            at += k
        self.spare = order[at:]
        self.table_host, self.lengths_host = table, list(lengths)
        self.table, self.lengths = ints(table), ints(lengths)
        inner, shape = (["slot", "heads"], (self.pages, slots, heads)) if slot_first else (["heads", "slot"], (self.pages, heads, slots))
        used = np.zeros((self.pages, slots), bool)
        for s, n in enumerate(lengths):
            for m in range(n):
                used[table[s, m // slots], m % slots] = True
        mask = torch.tensor(used, device="cuda")
        mask = mask[:, :, None] if slot_first else mask[:, None, :]
        guard = guard or Guarded()
        self.guard = guard
        names, self.named = ["page"] + inner, {}
        for name, d in (("k", dk), ("v", dv)):
            x = torch.randn(shape + (d,), generator=g, device="cuda") if values is None else values(name, shape + (d,), g)
            if dtype == "e4m3":
                # scales of any kind, not powers of two alone
                s = torch.exp(torch.randn(shape, generator=g, device="cuda")) * 0.01
                q = (x / x.abs().amax(-1, keepdim=True).clamp(min=1e-9) * 400).to(torch.float8_e4m3fn)
                pool = guard.empty(shape + (d,), "u8").view(torch.float8_e4m3fn)
                q = torch.where(mask[..., None], q.view(torch.uint8), torch.full_like(q.view(torch.uint8), 127))
                pool.view(torch.uint8).copy_(q)
                scale = guard.empty(shape, "f32")
                scale.copy_(torch.where(mask, s, float("nan")))
                setattr(self, name + "_scale", scale)
                self.named[name + "_scale"] = mtf.named(scale, names)
            else:
                pool = guard.empty(shape + (d,), "bf16")
                pool.copy_(torch.where(mask[..., None], x, float("nan")))
                setattr(self, name + "_scale", None)
                self.named[name + "_scale"] = None
            setattr(self, name, pool)
            self.named[name] = mtf.named(pool, names + ["d_" + name])
        self.cache = mtf.Cache(self.named["k"], self.named["v"], self.table, self.named["k_scale"], self.named["v_scale"])

    def rows(self, name, s, n=None, table=None):
        """Positions of a sequence in 64 bits, [n, heads, d]."""
        n = self.lengths_host[s] if n is None else n
        table = self.table_host[s] if table is None else table
        x = oa.gather(host(getattr(self, name)), table, n, self.slots, self.slot_first)
        if self.dtype == "e4m3":
            x = x * oa.gather(host(getattr(self, name + "_scale")), table, n, self.slots, self.slot_first)[..., None]
        return x


def queries(mtf, p, group, dk, dv, seed=1, scale=1.0, n_seq=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = n_seq or len(p.lengths_host)
    lead, dims = ((n, p.heads), ["batch", "heads"]) if group is None else ((n, p.heads, group), ["batch", "heads", "group"])
    q = (torch.randn(lead + (dk,), generator=g, device="cuda") * scale).to(torch.bfloat16)
    o = p.guard.empty(lead + (dv,), "bf16")
    return q, o, mtf.named(q, dims + ["d_k"]), mtf.named(o, dims + ["d_v"])


def workspace(mtf, lay, nq, p):
    import torch
    n = mtf.mtf_attention_decode_workspace_bytes(lay, nq, p.cache)
    if n == 0:
        return None
    w = p.guard.empty((n,), "u8")
    w.fill_(255)                                                   # (NaN as numbers, -1 as places)
    return w


def decode(mtf, p, group, dk, dv, scale, seed=1, qscale=1.0, lay=None):
    lay = lay or layout(mtf)
    q, o, nq, no = queries(mtf, p, group, dk, dv, seed, qscale)
    w = workspace(mtf, lay, nq, p)
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, scale, no, w)
    mtf.mtf_device_status()
    p.guard.check()
    return q, o


def check_attention(p, q, o, scale, rows=None, lengths=None):
    """Every element of o within the tolerance above; returns the largest share of it that was used."""
    qq, got = host(q), host(o)
    if qq.ndim == 3:
        qq, got = qq[:, :, None], got[:, :, None]
    worst = 0.0
    for s in range(qq.shape[0]):
        k, v = rows(s) if rows else (p.rows("k", s), p.rows("v", s))
        want, size, z = oa.decode(qq[s], k, v, scale)
        n = k.shape[0]
        if n == 0:
            assert not got[s].any()
            continue
        A = abs(scale) * np.einsum("hgd,mhd->hgm", np.abs(qq[s]), np.abs(k)).max(-1)
        delta = (2 * k.shape[-1] * U * A + 6 * U * np.abs(z).max(-1))[..., None]
        w = 2.0 ** -11 if p.dtype == "e4m3" else 2.0 ** -8 * (1 + 2.0 ** -8)
        tol = 2.0 ** -8 * np.abs(want) + size * (w + 4 * delta + 2.0 ** -20 + (n / 32 + 64) * 4 * U)
        if p.dtype == "e4m3":
            tol = tol + n * 2.0 ** -33 * np.abs(v).max()
        ok = np.abs(got[s] - want) <= tol
        assert ok.all(), (s, n, float((np.abs(got[s] - want) / tol).max()))
        worst = max(worst, float((np.abs(got[s] - want) / np.maximum(tol, 1e-300)).max()))
    return worst


#     heads group d_k  d_v slots  lengths                                     pages of a sequence
SHAPES = [
    (4, 1, 64, 64, 16, [0, 1, 15, 16, 17, 100], None),                        # not cut
    (2, None, 64, 64, 16, [512, 3, 0, 300], None),                            # cut, no group
    (3, 5, 72, 40, 24, [777, 0, 1, 24, 25, 300], None),                       # widths of their own, pages that end inside a tile
    (1, 8, 128, 128, 16, [2000, 1, 64, 65], None),
    (2, 9, 128, 128, 7, [1500, 129], 400),                                    # two tiles of heads, one of them nearly empty; a table longer than any sequence
    (1, 16, 64, 128, 64, [900], None),
    (2, 40, 128, 64, 33, [700, 2], None),                                     # more heads than a block takes at once
    (2, 3, 256, 256, 16, [600, 31], None),
    (1, 17, 256, 136, 50, [500], None),
    (2, 2, 8, 16, 1, [300, 5], None),                                         # pages of one position
    (5, 1, 32, 32, 100, [90, 1000, 100, 101, 99, 1, 0, 0, 640], None),
]


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(mtf, dtype, shape, slot_first):
    heads, group, dk, dv, slots, lengths, per = SHAPES[shape]
    if dtype == "e4m3":
        dk, dv = -(-dk // 16) * 16, -(-dv // 16) * 16
    p = Paged(mtf, dtype, lengths, heads, dk, dv, slots, slot_first, per, seed=shape)
    q, o = decode(mtf, p, group, dk, dv, dk ** -0.5)
    check_attention(p, q, o, dk ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_many_sequences(mtf, dtype):
    """More sequences than a block's plan, and just as many as it takes; few of them have positions."""
    for n_seq in (2049, 1025, 1024):
        lengths = [0] * n_seq
        for i in (0, 7, 1000, 1020, n_seq - 1):
            lengths[i] = 1 + i % 400
        p = Paged(mtf, dtype, lengths, 1, 64, 64, 16, per=30, seed=5)
        q, o = decode(mtf, p, 2, 64, 64, 0.125)
        got = host(o)
        for i in range(n_seq):
            if not lengths[i]:
                assert not got[i].any()
        live = [i for i in range(n_seq) if lengths[i]]
        sub = q[live], o[live]
        check_attention(p, *sub, 0.125, rows=lambda s: (p.rows("k", live[s]), p.rows("v", live[s])))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_scales_and_peaks(mtf, dtype):
    """Logits of some hundreds, one position that takes all of the weight, negative and zero scales, and queries far from 1."""
    import torch
    for scale, qscale in ((3.0, 4.0), (-0.3, 1.0), (0.0, 1.0), (1e-4, 1e4), (1e4, 1e-4), (2.0 ** 60, 2.0 ** -64), (2.0 ** -60, 2.0 ** 62)):
        p = Paged(mtf, dtype, [700, 33], 2, 64, 64, 16, seed=3)
        q, o = decode(mtf, p, 4, 64, 64, scale, qscale=qscale)
        check_attention(p, q, o, scale)
    # rising and falling logits: the running maximum moves at every chunk, or never
    for sign in (1.0, -1.0):
        def ramp(name, shape, g):
            x = torch.randn(shape, generator=g, device="cuda")
            return x
        p = Paged(mtf, dtype, [640], 1, 64, 64, 16, seed=4, values=ramp)
        for m in range(640):
            page, slot = p.table_host[0, m // 16], m % 16
            if dtype == "bf16":
                p.k[page, slot] = sign * m / 64.0
            else:
                p.k[page, slot] = torch.tensor(sign, device="cuda").to(torch.float8_e4m3fn)
                p.k_scale[page, slot] = m / 64.0
        lay = layout(mtf)
        q, o, nq, no = queries(mtf, p, 2, 64, 64)
        q.fill_(0.5)
        mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.25, no, workspace(mtf, lay, nq, p))
        mtf.mtf_device_status()
        check_attention(p, q, o, 0.25)


def test_attention_v_scales_far_apart(mtf):
    """Rows of v whose scales differ by 2^40 and whose weights make up for it, and rows of scale 0."""
    import torch
    p = Paged(mtf, "e4m3", [600], 1, 64, 64, 16, seed=8)
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, 3, 64, 64)
    q.fill_(1.0)
    p.k.copy_(torch.ones(p.k.shape, device="cuda").to(torch.float8_e4m3fn))
    for m in range(600):
        page, slot = p.table_host[0, m // 16], m % 16
        p.k_scale[page, slot] = -0.0 if m % 3 == 0 else (20.0 if m % 3 == 1 else 7.0)       # logits of 0, 20 log 2.. and some between
        p.v_scale[page, slot] = 2.0 ** 40 if m % 3 == 0 else (1.0 if m % 3 == 1 else 0.0)
    scale = 2 * np.log(2.0) / 64
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, scale, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    check_attention(p, q, o, scale)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_not_numbers(mtf, dtype):
    """A NaN in a key takes its head's results, one in a value its column's; a key of -infinity (bf16) is left out, a head of such keys alone is 0."""
    import torch
    dims = dict(heads=3, dk=64, dv=64, slots=16)
    p = Paged(mtf, dtype, [400, 400], seed=6, **dims)
    lay = layout(mtf)
    q, o, nq, no = queries(mtf, p, 2, 64, 64)
    q.abs_()
    nan = torch.tensor(float("nan"), device="cuda").to(p.k.dtype)

    def put(pool, s, m, h, d, x):
        pool[p.table_host[s, m // 16], m % 16, h, d] = x
    put(p.k, 0, 300, 0, 5, nan)
    put(p.v, 0, 17, 1, 9, nan)
    if dtype == "bf16":
        put(p.k, 1, 3, 0, 0, float("-inf"))
        for m in range(400):
            put(p.k, 1, m, 1, 0, float("-inf"))
        put(p.k, 1, 5, 2, 0, float("inf"))
    mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, workspace(mtf, lay, nq, p))
    mtf.mtf_device_status()
    got = host(o)
    assert np.isnan(got[0, 0]).all()
    column = np.zeros((2, 64), bool)
    column[:, 9] = True
    assert np.array_equal(np.isnan(got[0, 1]), column) and np.isfinite(got[0, 2]).all()
    if dtype == "bf16":
        assert not got[1, 1].any() and np.isnan(got[1, 2]).all()
        keep = [m for m in range(400) if m != 3]
        k, v = p.rows("k", 1)[keep][:, :1], p.rows("v", 1)[keep][:, :1]
        one = Paged.__new__(Paged)
        one.dtype = dtype
        check_attention(one, q[1:, :1], o[1:, :1], 0.125, rows=lambda s: (k, v))


def test_bad_pages_and_lengths_are_left_out(mtf):
    """Pages outside the pool and lengths beyond the table: reported, and as if their positions were not there."""
    for per in (8, 40):                                            # not cut, cut
        p = Paged(mtf, "bf16", [100, 100, 100], 2, 64, 64, 16, per=per, seed=2)
        table = p.table_host.copy()
        table[0, 1], table[1, 2], table[2, :7] = p.pages, -1, 1 << 30
        p.table.copy_(ints(table))
        lay = layout(mtf)
        q, o, nq, no = queries(mtf, p, 2, 64, 64)
        mtf.mtf_attention_decode(lay, nq, p.cache, p.lengths, 0.125, no, workspace(mtf, lay, nq, p))
        with pytest.raises(mtf.MtfError) as e:
            mtf.mtf_device_status()
        assert e.value.code == "MTF_ERR_INVALID_ARG"
        mtf.mtf_device_status()                                    # (said once)
        p.guard.check()
        out = {0: range(16, 32), 1: range(32, 48), 2: range(100)}

        def rows(s):
            keep = [m for m in range(100) if m not in out[s]]
            return p.rows("k", s)[keep], p.rows("v", s)[keep]
        check_attention(p, q, o, 0.125, rows=rows)
        # a length beyond the table's pages, and one below 0
        p.table.copy_(ints(p.table_host))
        n = [per * 16 + 1, -5, 100]
        full = Paged(mtf, "bf16", [per * 16, 1, 100], 2, 64, 64, 16, per=per, seed=9)
        full.lengths.copy_(ints(n))
        q, o, nq, no = queries(mtf, full, 2, 64, 64)
        mtf.mtf_attention_decode(lay, nq, full.cache, full.lengths, 0.125, no, workspace(mtf, lay, nq, full))
        with pytest.raises(mtf.MtfError):
            mtf.mtf_device_status()
        full.lengths_host = [per * 16, 0, 100]
        check_attention(full, q, o, 0.125)


# ---- the cache's rows ------------------------------------------------------------------------------------------------

def special_rows(shape, seed):
    """Rows in f32 with zeros, tiny and huge ones, values at the borders of e4m3's steps, NaN and infinities among them."""
    r = np.random.RandomState(seed)
    x = r.randn(*shape).astype(np.float32)
    flat = x.reshape(-1, shape[-1])
    flat[0] = 0.0
    flat[1 % len(flat)] *= 1e-42
    flat[2 % len(flat)] *= 3e37
    size = oa.E4M3[:127]
    mids = ((size[1:] + size[:-1]) / 2).astype(np.float32)
    for i in range(3, len(flat)):
        if i % 3 == 0:
            pick = r.choice(np.concatenate([size, mids]).astype(np.float32), shape[-1])
            flat[i] = pick * r.choice([-1, 1], shape[-1]) * np.float32(2.0 ** r.randint(-30, 30))
            flat[i, 0] = 448.0 * 2.0 ** r.randint(-3, 3)
    if len(flat) > 6:
        flat[5, 1], flat[5, 2], flat[5, 3] = np.nan, np.inf, -np.inf
    return x


def bf16_of(x):
    import torch
    return torch.tensor(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("source", ["bf16", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,dk,dv,slots,length", [(1, 64, 64, 16, 1), (3, 80, 48, 20, 13), (2, 256, 144, 5, 37), (5, 128, 16, 64, 70), (1, 16, 256, 1, 3), (9, 64, 48, 16, 21)])
def test_rows_there_and_back(mtf, dtype, source, heads, dk, dv, slots, length, slot_first):
    import torch
    lay, guard = layout(mtf), Guarded()
    starts, counts = [0, 3, slots - 1, 2 * slots, 7], [length, 0, max(1, length - 3), length, -2]
    B = len(starts)
    ends = [s + length for s in starts]
    p = Paged(mtf, dtype, ends, heads, dk, dv, slots, slot_first, seed=1, guard=guard)
    before = {n: host(getattr(p, n)).copy() for n in ("k", "v")}
    tdt = torch.bfloat16 if source == "bf16" else torch.float32
    new = {}
    for name, d in (("k", dk), ("v", dv)):
        x = special_rows((B, length, heads, d), 3 if name == "k" else 4)
        new[name] = torch.tensor(x).to(tdt).cuda()
    dims = ["batch", "memory_length", "heads"]
    mtf.mtf_cache_write(lay, mtf.named(new["k"], dims + ["d_k"]), mtf.named(new["v"], dims + ["d_v"]), ints(starts), ints(counts), p.cache)
    mtf.mtf_device_status()
    guard.check()
    for name in ("k", "v"):
        want, scales = before[name].copy(), None
        x = host(new[name])
        if dtype == "e4m3":
            bytes_, scale = oa.quantise(x)
            rows = oa.E4M3[bytes_]
            scales = host(getattr(p, name + "_scale"))
        else:
            rows = bf16_of(x)
        for b in range(B):
            for i in range(max(0, counts[b])):
                m = starts[b] + i
                page, slot = p.table_host[b, m // slots], m % slots
                for h in range(heads):
                    at = (page, slot, h) if slot_first else (page, h, slot)
                    want[at] = rows[b, i, h]
                    if scales is not None:
                        assert scales[at] == scale[b, i, h]
        assert np.array_equal(host(getattr(p, name)), want, equal_nan=True)          # (and everything else as it was)
    # back, in both types
    for back in ("bf16", "f32"):
        kk, vv = guard.empty((B, length, heads, dk), back), guard.empty((B, length, heads, dv), back)
        mtf.mtf_cache_read(lay, p.cache, ints(starts), ints(counts), mtf.named(kk, dims + ["d_k"]), mtf.named(vv, dims + ["d_v"]))
        mtf.mtf_device_status()
        guard.check()
        for name, t in (("k", kk), ("v", vv)):
            x = host(new[name])
            if dtype == "e4m3":
                bytes_, scale = oa.quantise(x)
                want = oa.E4M3[bytes_] * scale[..., None]
            else:
                want = bf16_of(x)
            for b in range(B):
                want[b, max(0, counts[b]):] = 0.0
            if back == "bf16":
                want = bf16_of(want)
            assert np.array_equal(host(t), want, equal_nan=True)


def test_rows_without_starts_and_counts_and_bad_places(mtf):
    import torch
    lay, dims = layout(mtf), ["batch", "length", "heads"]
    p = Paged(mtf, "bf16", [20, 20], 2, 64, 64, 8, per=4, seed=1)
    x = torch.randn(2, 20, 2, 64, device="cuda").to(torch.bfloat16)
    n = [mtf.named(x, dims + [d]) for d in ("d_k", "d_v")]
    mtf.mtf_cache_write(lay, *n, None, None, p.cache)
    y, z = torch.empty_like(x), torch.empty_like(x)
    mtf.mtf_cache_read(lay, p.cache, None, None, mtf.named(y, dims + ["d_k"]), mtf.named(z, dims + ["d_v"]))
    mtf.mtf_device_status()
    assert torch.equal(x, y) and torch.equal(x, z)
    # no place: positions below 0 and behind the table, pages outside the pool
    table = p.table_host.copy()
    table[1, 1] = p.pages
    p.table.copy_(ints(table))
    before = p.k.clone()
    mtf.mtf_cache_write(lay, *n, ints([-3, 1 << 30]), ints([3, 20]), p.cache)
    with pytest.raises(mtf.MtfError):
        mtf.mtf_device_status()
    p.guard.check()
    assert torch.equal(before.nan_to_num(7.0), p.k.nan_to_num(7.0))
    mtf.mtf_cache_read(lay, p.cache, ints([2, 4]), None, mtf.named(y, dims + ["d_k"]), mtf.named(z, dims + ["d_v"]))
    with pytest.raises(mtf.MtfError):
        mtf.mtf_device_status()
    mtf.mtf_device_status()
    assert torch.equal(y[0, :18], x[0, 2:]) and torch.equal(y[1, :4], x[1, 4:8]) and not y[1, 4:12].any()


# ---- beam search -------------------------------------------------------------------------------------------------------

def select(mtf, z, scores, finished, end_id, slots, dtype):
    import torch
    lay, guard = layout(mtf), Guarded()
    S, K, V = z.shape
    t = guard.empty((S, K, V), dtype)
    t.copy_(torch.tensor(z))
    sc = torch.tensor(np.asarray(scores, dtype=np.float32), device="cuda")
    fin = None if finished is None else ints(finished)
    out = {n: ints(np.full((S, slots), -9)) for n in ("parents", "tokens", "finished")}
    new = guard.empty((S, slots), "f32")
    nl = mtf.named(t, ["sentence", "beam", "vocab"])
    w = guard.empty((mtf.mtf_beam_select_workspace_bytes(lay, nl, slots),), "u8")
    w.fill_(255)
    mtf.mtf_beam_select(lay, nl, mtf.named(sc, ["sentence", "beam"]), fin, end_id, out["parents"], out["tokens"], mtf.named(new, ["sentence", "out"]), out["finished"], w)
    mtf.mtf_device_status()
    guard.check()
    zz, ss = host(t), host(sc)
    for s in range(S):
        p, v, best, f = oa.beam_select(zz[s], ss[s], None if finished is None else finished[s], end_id, slots)
        assert host(out["parents"])[s].tolist() == p.tolist(), s
        assert host(out["tokens"])[s].tolist() == v.tolist(), s
        assert host(out["finished"])[s].tolist() == f.tolist(), s
        got = host(new)[s]
        # a sum of exponentials of V / 256 + 16 f32 additions a thread and their roundings (3 u X + 2^-22 at an exponent of X, with weights: log V + 1), and the rounding of the result
        tol = (V / 256 + 16 + 3 * (np.log(V) + 1) + 8) * U + 2 * U * np.abs(np.where(np.isfinite(best), best, 0.0))
        is_one = np.isfinite(best)
        assert (np.isfinite(got) == is_one).all() and (np.abs(got[is_one] - best[is_one]) <= tol[is_one]).all()


def logits(S, K, V, seed, spread=2.0):
    r = np.random.RandomState(seed)
    z = r.randn(S, K, V) * spread
    z[:, :, r.randint(0, V, 12)] += 6.0
    return z, -20.0 + 3.0 * r.randn(S, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,K,V,slots", [(1, 4, 32768, 4), (3, 5, 50001, 10), (2, 1, 7, 7), (2, 12, 1003, 24), (5, 8, 4096, 8), (1, 64, 515, 64), (40, 3, 2050, 6), (2, 2, 131072, 1),
                                         (1, 1, 200001, 64), (2, 3, 1, 3)])
def test_selection(mtf, dtype, S, K, V, slots):
    z, sc = logits(S, K, V, seed=S + K + V)
    select(mtf, z, sc, None, 0, slots, dtype)
    fin = np.random.RandomState(3).rand(S, K) < 0.3
    fin[0, 0] = True
    select(mtf, z, sc, fin.astype(np.int32), min(2, V - 1), slots, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,K,V,slots", [(9, 4, 8192, 4), (10, 4, 8192, 4), (2, 4, 16384, 4), (2, 4, 32768, 4), (2, 4, 32776, 4), (1, 64, 2049, 33), (9, 3, 4099, 32)])
def test_selection_where_one_launch_becomes_two(mtf, dtype, S, K, V, slots):
    """Numbers of sentences and of runs on both sides of what a cluster a sentence takes, some beams not there, some finished."""
    z, sc = logits(S, K, V, seed=S * V)
    sc[0, -1], sc[-1, 0] = -np.inf, np.nan
    fin = np.random.RandomState(7).rand(S, K) < 0.2
    select(mtf, z, sc, fin.astype(np.int32), 3, slots, dtype)


@pytest.mark.parametrize("V", [4096, 9001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_ties_masks_and_empty_beams(mtf, dtype, V):
    low = -3.38e38 if dtype == "bf16" else -3.4028235e38
    r = np.random.RandomState(0)
    K, slots = 4, 8
    z, sc = logits(1, K, V, 5)
    # equal rows, equal scores: to the bit, whatever their place in memory
    z[0, 1:] = z[0, 0]
    select(mtf, z, np.zeros((1, K)), None, 0, slots, dtype)
    # all words alike, in one beam and in all; zeros of both signs
    select(mtf, np.zeros((1, K, V)), sc, None, 0, slots, dtype)
    signed = np.where(r.rand(1, K, V) < 0.5, -0.0, 0.0)
    select(mtf, signed, np.zeros((1, K)), None, 0, slots, dtype)
    # few words allowed: the others -infinity, or the type's lowest value
    for mask in (-np.inf, low):
        for allowed in (1, 3, 20):
            m = np.full((1, K, V), mask)
            at = r.choice(V, allowed, replace=False)
            m[:, :, at] = z[:, :, at] + r.randn(1, K, allowed)
            select(mtf, m, sc, None, 0, slots, dtype)
    m = np.full((1, K, V), low)
    m[0, 1:] = z[0, 1:]
    select(mtf, m, sc, None, 0, slots, dtype)
    # few different values: many equal ones above and at the threshold
    select(mtf, np.round(r.randn(2, K, V) * 1.5), np.zeros((2, K)), None, 0, 16, dtype)
    # many large words that one thread of a part may hold, rising and falling rows
    for z2 in (np.linspace(-5, 5, V), np.linspace(5, -5, V), np.arange(V) % 2048 / 100.0, np.arange(V) // 8 % 256 / 10.0):
        select(mtf, np.broadcast_to(z2, (1, 2, V)).copy(), [[-1.0, -1.5]], None, 0, 16, dtype)
    # beams that are none yet, all but one finished, not numbers
    z, sc = logits(3, K, V, 6)
    sc[0, 1:] = -np.inf
    sc[1, 0], sc[1, 1] = np.nan, np.inf
    z[2, 0, 17], z[2, 1, 5] = np.nan, np.inf
    z[2, 2] = -np.inf
    select(mtf, z, sc, None, 3, slots, dtype)
    select(mtf, z, sc, np.array([[0, 0, 0, 0], [0, 1, 1, 1], [1, 1, 1, 1]], np.int32), 3, slots, dtype)
    # fewer offers than slots: all beams finished
    select(mtf, z[:1], np.array([[-1.0, -2.0, -1.0, -np.inf]]), np.ones((1, K), np.int32), 3, slots, dtype)
    # scores far apart, and far from 0
    select(mtf, z[1:2], np.array([[-1e30, 1e5, -1e5, 1e30]]), None, 3, slots, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("lead,beams,slots,rest", [((2,), 3, 4, (5, 8)), ((), 4, 2, (16, 16)), ((3, 2), 1, 3, (7,)), ((2,), 5, 5, ()), ((1,), 2, 9, (3, 1001)), ((4,), 4, 4, (64, 128))])
def test_states(mtf, dtype, lead, beams, slots, rest):
    import torch
    lay, guard = layout(mtf), Guarded()
    r = np.random.RandomState(0)
    names = ["g%d" % i for i in range(len(lead))] + ["beam"] + ["x%d" % i for i in range(len(rest))]
    raw = torch.randn(lead + (beams,) + rest, device="cuda")
    tdt = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[dtype]
    x = raw.to(tdt)
    width = x.element_size()
    out = guard.empty((int(np.prod(lead + (slots,) + rest)) * width,), "u8").view(tdt).view(lead + (slots,) + rest)
    parents = r.randint(0, beams, lead + (slots,))
    mtf.mtf_beam_reorder(lay, "beam", ints(parents), mtf.named(x, names), mtf.named(out, names))
    mtf.mtf_device_status()
    guard.check()
    xs, got = host(x).reshape((-1, beams) + rest), host(out).reshape((-1, slots) + rest)
    for g, row in enumerate(parents.reshape(-1, slots)):
        for i, p in enumerate(row):
            assert np.array_equal(got[g, i], xs[g, p])
    # a parent outside the beams: zeros, and said
    parents.reshape(-1)[-1] = beams
    mtf.mtf_beam_reorder(lay, "beam", ints(parents), mtf.named(x, names), mtf.named(out, names))
    with pytest.raises(mtf.MtfError):
        mtf.mtf_device_status()
    assert not host(out).reshape((-1, slots) + rest)[-1, -1].any()


@pytest.mark.parametrize("slot_first", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("slots,length", [(16, 37), (16, 32), (5, 3), (1, 4), (40, 0), (130, 100)])
def test_caches_of_beams(mtf, dtype, slots, length, slot_first):
    """Tables change hands, pages that go on are copied as far as they are used, whole ones are shared, nothing else is touched."""
    import torch
    S, K, out, heads = 2, 3, 4, 2
    lengths = [length] * (S * K)
    lengths[1] = max(0, length - 1)
    p = Paged(mtf, dtype, lengths, heads, 64, 32, slots, slot_first, per=length // slots + 2, seed=3, spare=S * out + 1)
    table = p.table.view(S, K, -1)
    cache = mtf.Cache(p.named["k"], p.named["v"], table, p.named["k_scale"], p.named["v_scale"])
    parents = np.array([[1, 1, 0, 2], [2, 0, 0, 0]])
    fresh = p.spare[:S * out].reshape(S, out)
    new_table, new_lengths = ints(np.full((S, out, p.per), -3)), ints(np.full((S, out), -3))
    pools = [n for n in ("k", "v", "k_scale", "v_scale") if getattr(p, n) is not None]
    before = {n: host(getattr(p, n)).copy() for n in pools}
    lay = layout(mtf)
    mtf.mtf_cache_reorder(lay, cache, ints(parents), p.lengths.view(S, K), ints(fresh), new_table, new_lengths)
    mtf.mtf_device_status()
    p.guard.check()
    nt, nl = host(new_table).astype(int), host(new_lengths).astype(int)
    want = {n: before[n].copy() for n in pools}
    for s in range(S):
        for i in range(out):
            q = s * K + parents[s, i]
            n, old = lengths[q], p.table_host[q].copy()
            assert nl[s, i] == n
            if n % slots:
                page, to, used = old[n // slots], fresh[s, i], n % slots
                for name in pools:
                    if slot_first:
                        want[name][to, :used] = before[name][page, :used]
                    else:
                        want[name][to, :, :used] = before[name][page, :, :used]
                old[n // slots] = to
            assert nt[s, i].tolist() == old.tolist()
    for name in pools:
        assert np.array_equal(host(getattr(p, name)), want[name], equal_nan=True)
    if length:
        # a parent, a length and a fresh page that are none
        bad = parents.copy()
        bad[0, 0] = K
        mtf.mtf_cache_reorder(lay, cache, ints(bad), p.lengths.view(S, K), ints(np.full((S, out), p.pages)), new_table, new_lengths)
        with pytest.raises(mtf.MtfError):
            mtf.mtf_device_status()
        assert host(new_lengths)[0, 0] == 0 and (host(new_table)[0, 0] == -1).all()
        for name in pools:
            assert np.array_equal(host(getattr(p, name)), want[name], equal_nan=True)


# ---- together ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_answers_go_on_from_the_attention_block(mtf, dtype):
    """A prompt through the attention block, its keys and values into a cache, then token by token: each new position's projections by einsums, its row into the cache,
    attention over it, the output projection.  What the block computes for the whole sequence at once, causal, is what the tokens get one by one."""
    import torch
    B, L, D, H, K, prompt, slots = 2, 128, 128, 2, 64, 100, 16
    g = torch.Generator(device="cuda").manual_seed(0)
    lay = layout(mtf, (("m", 2),), [("heads", "m")])
    bf = torch.bfloat16
    rnd = lambda shape, s: (torch.randn(shape, generator=g, device="cuda") * s).to(bf)                                   # noqa: E731
    act, N = ["batch", "length", "d_model"], mtf.named
    x, wq, wk, wv = rnd((B, L, D), 1.0), rnd((D, H, K), D ** -0.5), rnd((D, H, K), D ** -0.5), rnd((D, H, K), D ** -0.5)
    wo = rnd((H, K, D), (H * K) ** -0.5)
    q, kk, vv, o = (torch.empty(B, L, H, K, dtype=bf, device="cuda") for _ in range(4))
    weights, y = torch.empty(B, H, L, L, dtype=bf, device="cuda"), torch.empty(B, L, D, dtype=bf, device="cuda")
    w = {"wq": N(wq, ["d_model", "heads", "d_k"]), "wk": N(wk, ["d_model", "heads", "d_k"]), "wv": N(wv, ["d_model", "heads", "d_v"]), "wo": N(wo, ["heads", "d_v", "d_model"])}
    ws = torch.empty(mtf.mtf_attention_workspace_bytes(lay, N(x, act), w["wq"], w["wv"]), dtype=torch.uint8, device="cuda")
    mtf.mtf_attention_forward(lay, N(x, act), w["wq"], w["wk"], w["wv"], w["wo"], True, None, N(q, ["batch", "length", "heads", "d_k"]), N(kk, ["batch", "memory_length", "heads", "d_k"]),
                              N(vv, ["batch", "memory_length", "heads", "d_v"]), N(weights, ["batch", "heads", "length", "memory_length"]), N(o, ["batch", "length", "heads", "d_v"]),
                              N(y, act), ws)
    per = L // slots
    pools = [torch.zeros(B * per, slots, H, K, device="cuda").to(bf if dtype == "bf16" else torch.float8_e4m3fn) for _ in range(2)]
    inner = ["page", "slot", "heads"]
    scales = [None, None] if dtype == "bf16" else [N(torch.zeros(B * per, slots, H, device="cuda"), inner) for _ in range(2)]
    table = torch.randperm(B * per, generator=torch.Generator().manual_seed(1)).int().view(B, per).cuda()
    cache = mtf.Cache(N(pools[0], inner + ["d_k"]), N(pools[1], inner + ["d_v"]), table, *scales)
    mem = ["batch", "memory_length", "heads"]
    mtf.mtf_cache_write(lay, N(kk, mem + ["d_k"]), N(vv, mem + ["d_v"]), None, ints([prompt] * B), cache)
    lengths = ints([prompt] * B)
    # what one new token needs, made once
    x1 = torch.empty(B, D, dtype=bf, device="cuda")
    q1, k1, v1, o1 = (torch.empty(B, H, K, dtype=bf, device="cuda") for _ in range(4))
    y1 = torch.empty(B, D, dtype=bf, device="cuda")
    nx, nq, nk, nv, no = N(x1, ["batch", "d_model"]), N(q1, ["batch", "heads", "d_k"]), N(k1, ["batch", "heads", "d_k"]), N(v1, ["batch", "heads", "d_v"]), N(o1, ["batch", "heads", "d_v"])
    krow, vrow = N(k1.view(B, 1, H, K), mem + ["d_k"]), N(v1.view(B, 1, H, K), mem + ["d_v"])
    n = mtf.mtf_attention_decode_workspace_bytes(lay, nq, cache)
    wd = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    we = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    worst = 0.0
    for m in range(prompt, L):
        x1.copy_(x[:, m])
        for name, out in (("wq", nq), ("wk", nk), ("wv", nv)):
            mtf.mtf_einsum(lay, None, [nx, w[name]], out, None, we)
        mtf.mtf_cache_write(lay, krow, vrow, lengths, None, cache)
        lengths += 1
        mtf.mtf_attention_decode(lay, nq, cache, lengths, K ** -0.5, no, wd)
        mtf.mtf_einsum(lay, None, [no, w["wo"]], N(y1, ["batch", "d_model"]), None, we)
        # against 64 bits on the rows that the block has, in the cache's type; each side rounds weights (2^-8) and the result (2^-8), and the
        # projections of a token may round another way (2^-8 of a value) than those of the whole sequence
        k, v = host(kk)[:, :m + 1], host(vv)[:, :m + 1]
        if dtype == "e4m3":
            k, v = (oa.E4M3[b] * s[..., None] for b, s in (oa.quantise(t) for t in (k, v)))
        for b in range(B):
            want, size, z = oa.decode(host(q)[b, m][:, None], k[b], v[b], K ** -0.5)
            A = K ** -0.5 * np.einsum("hd,mhd->hm", np.abs(host(q)[b, m]), np.abs(k[b])).max(-1)[:, None]
            # (a value of the newest row, and of q, one rounding apart: 2^-8 of A in a logit; in e4m3 the newest row may be a step, 2^-3, apart)
            step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -8
            p_new = np.exp(z[:, 0, -1] - z.max(-1)[:, 0]) / np.exp(z - z.max(-1, keepdims=True)).sum(-1)[:, 0]
            new = 0.0 if dtype == "bf16" else (p_new[:, None] * 2.0 ** -3 * (np.abs(v[b, -1]) + (np.abs(want[:, 0]) + size[:, 0]) * A))
            tol = size[:, 0] * (2 * 2.0 ** -8 + 2 * 2 * step * A) + 2 * 2.0 ** -8 * np.abs(want[:, 0]) + new + 1e-6
            err = np.abs(host(o1)[b] - want[:, 0])
            assert (err <= tol).all(), (m, b, float((err / tol).max()))
            worst = max(worst, float((err / tol).max()))
        if dtype == "bf16":
            # the block itself: two results with the roundings above each
            d = np.abs(host(y1) - host(y)[:, m])
            assert d.max() <= 0.05 * np.abs(host(y)[:, m]).max() + 1e-3
    mtf.mtf_device_status()
    assert worst > 0.0


def test_beams_share_pages_and_part(mtf):
    """Three steps of beam search over caches: selection, reordering, a new row for each beam, attention; every beam attends to its own history."""
    import torch
    S, K, H, D, slots, V = 2, 3, 2, 64, 4, 1000
    lay = layout(mtf)
    g = torch.Generator(device="cuda").manual_seed(3)
    bf = torch.bfloat16
    start, steps = 6, 5
    per = (start + steps) // slots + 1
    pages = S * K * per * 3
    pool = [torch.full((pages, slots, H, D), float("nan"), dtype=bf, device="cuda") for _ in range(2)]
    inner, seq = ["page", "slot", "heads"], ["sentence", "beam"]
    used = 0
    table = torch.arange(S * K * per, dtype=torch.int32, device="cuda").view(S, K, per)
    used = S * K * per
    lengths = torch.full((S, K), start, dtype=torch.int32, device="cuda")
    N = mtf.named
    rows = lambda n: [torch.randn(S, K, n, H, D, generator=g, device="cuda").to(bf) for _ in range(2)]                  # noqa: E731
    cache_of = lambda t: mtf.Cache(N(pool[0], inner + ["d_k"]), N(pool[1], inner + ["d_v"]), t)                         # noqa: E731
    first = rows(start)
    mtf.mtf_cache_write(lay, N(first[0], seq + ["length", "heads", "d_k"]), N(first[1], seq + ["length", "heads", "d_v"]), None, None, cache_of(table))
    history = [[(host(first[0])[s, b], host(first[1])[s, b]) for b in range(K)] for s in range(S)]
    scores = torch.randn(S, K, generator=g, device="cuda")
    finished = torch.zeros(S, K, dtype=torch.int32, device="cuda")
    for _ in range(steps):
        z = torch.randn(S, K, V, generator=g, device="cuda") * 3
        parents, tokens, fin = (torch.empty(S, K, dtype=torch.int32, device="cuda") for _ in range(3))
        new_scores = torch.empty(S, K, device="cuda")
        nl = N(z, seq + ["vocab"])
        w = torch.empty(mtf.mtf_beam_select_workspace_bytes(lay, nl, K), dtype=torch.uint8, device="cuda")
        mtf.mtf_beam_select(lay, nl, N(scores, seq), finished, 0, parents, tokens, N(new_scores, seq), fin, w)
        for s in range(S):
            p, v, best, f = oa.beam_select(host(z)[s], host(scores)[s], host(finished)[s], 0, K)
            assert host(parents)[s].tolist() == p.tolist() and host(tokens)[s].tolist() == v.tolist()
        fresh = torch.arange(used, used + S * K, dtype=torch.int32, device="cuda").view(S, K)
        used += S * K
        new_table, new_lengths = torch.empty_like(table), torch.empty_like(lengths)
        mtf.mtf_cache_reorder(lay, cache_of(table), parents, lengths, fresh, new_table, new_lengths)
        # a page that is full: the table's own next one of the beam is another beam's too after a few steps, so a new one is given
        n = int(new_lengths[0, 0])
        if n % slots == 0:
            new_table[:, :, n // slots] = fresh
        history = [[history[s][int(parents[s, b])] for b in range(K)] for s in range(S)]
        new = rows(1)
        mtf.mtf_cache_write(lay, N(new[0], seq + ["length", "heads", "d_k"]), N(new[1], seq + ["length", "heads", "d_v"]), new_lengths, None, cache_of(new_table))
        new_lengths += 1
        history = [[tuple(np.concatenate([history[s][b][i], host(new[i])[s, b]]) for i in range(2)) for b in range(K)] for s in range(S)]
        q, o = rows(1)[0][:, :, 0].contiguous(), torch.empty(S, K, H, D, dtype=bf, device="cuda")
        mtf.mtf_attention_decode(lay, N(q, seq + ["heads", "d_k"]), cache_of(new_table), new_lengths, 0.125, N(o, seq + ["heads", "d_v"]))
        mtf.mtf_device_status()
        p = Paged.__new__(Paged)
        p.dtype = "bf16"
        check_attention(p, q.view(S * K, H, D), o.view(S * K, H, D), 0.125, rows=lambda i: history[i // K][i % K])
        states = torch.randn(S, K, 7, generator=g, device="cuda")
        out = torch.empty_like(states)
        mtf.mtf_beam_reorder(lay, "beam", parents, N(states, seq + ["x"]), N(out, seq + ["x"]))
        assert torch.equal(out, states[torch.arange(S, device="cuda")[:, None], parents.long()])
        table, lengths, scores, finished = new_table, new_lengths, new_scores, fin


def step_of(mtf, seed):
    """One step of answering on tensors of its own: selection, reordering, writing, attention; and what it leaves."""
    import torch
    lay, S, K = layout(mtf), 2, 4
    p = Paged(mtf, "e4m3", [300] * (S * K), 2, 64, 64, 16, per=24, seed=seed, spare=S * K)
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(S, K, 20000, generator=g, device="cuda").to(torch.bfloat16)
    scores = torch.randn(S, K, generator=g, device="cuda")
    seq = ["sentence", "beam"]
    outs = [torch.zeros(S, K, dtype=torch.int32, device="cuda") for _ in range(3)] + [torch.zeros(S, K, device="cuda")]
    nl, nsc, nnew = mtf.named(z, seq + ["vocab"]), mtf.named(scores, seq), mtf.named(outs[3], seq)
    w1 = torch.empty(mtf.mtf_beam_select_workspace_bytes(lay, nl, K), dtype=torch.uint8, device="cuda")
    table, fresh = p.table.view(S, K, -1), ints(p.spare[:S * K].reshape(S, K))
    new_table, new_lengths = torch.zeros_like(table), torch.zeros(S, K, dtype=torch.int32, device="cuda")
    old = mtf.Cache(p.named["k"], p.named["v"], table, p.named["k_scale"], p.named["v_scale"])
    new = mtf.Cache(p.named["k"], p.named["v"], new_table, p.named["k_scale"], p.named["v_scale"])
    rows = [torch.randn(S, K, 1, 2, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    q = torch.randn(S, K, 2, 3, 64, generator=g, device="cuda").to(torch.bfloat16)
    o = torch.zeros_like(q)
    nq, no = mtf.named(q, seq + ["heads", "group", "d_k"]), mtf.named(o, seq + ["heads", "group", "d_v"])
    w2 = torch.empty(mtf.mtf_attention_decode_workspace_bytes(lay, nq, new), dtype=torch.uint8, device="cuda")
    kk, vv = (mtf.named(r, seq + ["length", "heads", d]) for r, d in zip(rows, ("d_k", "d_v")))
    lengths, grown = p.lengths.view(S, K), torch.zeros(S, K, dtype=torch.int32, device="cuda")

    def step():
        mtf.mtf_beam_select(lay, nl, nsc, None, 1, outs[0], outs[1], nnew, outs[2], w1)
        mtf.mtf_cache_reorder(lay, old, outs[0], lengths, fresh, new_table, new_lengths)
        mtf.mtf_cache_write(lay, kk, vv, new_lengths, None, new)
        torch.add(new_lengths, 1, out=grown)
        mtf.mtf_attention_decode(lay, nq, new, grown, 0.125, no, w2)
    return step, outs + [new_table, new_lengths, o]


def test_graphs_streams_and_threads(mtf):
    """Captured and replayed, on another stream, by two threads at once, eagerly between replays: the bits of the serial call each time."""
    import torch
    step, outs = step_of(mtf, 1)
    other, other_outs = step_of(mtf, 2)
    step(), other()
    mtf.mtf_device_status()
    want, other_want = [t.clone() for t in outs], [t.clone() for t in other_outs]

    def same(got, ref):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    side = torch.cuda.Stream()
    graphs = []
    for f in (step, other):
        with torch.cuda.stream(side):
            f()
        side.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            f()
        graphs.append(gr)
    for t in outs + other_outs:
        t.zero_()
    for _ in range(3):
        graphs[0].replay()
        graphs[1].replay()
        step()
    torch.cuda.synchronize()
    same(outs, want)
    same(other_outs, other_want)
    for t in outs + other_outs:
        t.zero_()
    torch.cuda.synchronize()

    def work(f):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                f()
        s.synchronize()
    threads = [threading.Thread(target=work, args=(f,)) for f in (step, other)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    mtf.mtf_device_status()
    same(outs, want)
    same(other_outs, other_want)


def test_offsets_beyond_32_bits(mtf):
    """A pool of more than 2^32 bytes a side: rows written, attended to and read back at its far end."""
    import torch
    pages, slots, H, D = 36000, 64, 8, 128                         # 4.7 GB a side in bf16
    lay, bf = layout(mtf), torch.bfloat16
    pool = [torch.empty(pages, slots, H, D, dtype=bf, device="cuda") for _ in range(2)]
    inner, mem = ["page", "slot", "heads"], ["batch", "length", "heads"]
    table = torch.arange(pages - 10, pages, dtype=torch.int32, device="cuda").view(2, 5)
    cache = mtf.Cache(mtf.named(pool[0], inner + ["d_k"]), mtf.named(pool[1], inner + ["d_v"]), table)
    g = torch.Generator(device="cuda").manual_seed(0)
    rows = [torch.randn(2, 300, H, D, generator=g, device="cuda").to(bf) for _ in range(2)]
    mtf.mtf_cache_write(lay, mtf.named(rows[0], mem + ["d_k"]), mtf.named(rows[1], mem + ["d_v"]), None, None, cache)
    back = [torch.zeros_like(r) for r in rows]
    mtf.mtf_cache_read(lay, cache, None, None, mtf.named(back[0], mem + ["d_k"]), mtf.named(back[1], mem + ["d_v"]))
    assert torch.equal(rows[0], back[0]) and torch.equal(rows[1], back[1])
    q = torch.randn(2, H, 2, D, generator=g, device="cuda").to(bf)
    o = torch.empty_like(q)
    nq = mtf.named(q, ["batch", "heads", "group", "d_k"])
    w = torch.empty(mtf.mtf_attention_decode_workspace_bytes(lay, nq, cache), dtype=torch.uint8, device="cuda")
    mtf.mtf_attention_decode(lay, nq, cache, ints([300, 257]), D ** -0.5, mtf.named(o, ["batch", "heads", "group", "d_v"]), w)
    mtf.mtf_device_status()
    p = Paged.__new__(Paged)
    p.dtype = "bf16"
    n = [300, 257]
    check_attention(p, q, o, D ** -0.5, rows=lambda s: (host(rows[0][s, :n[s]]), host(rows[1][s, :n[s]])))
