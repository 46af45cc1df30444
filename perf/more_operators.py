"""What a model answers with as timed cases: attention of one new token over a paged cache of keys and values, the cache's writing (8-bit with a scale a row, or as
it comes) and reading back, beam search's selection over beams and vocabulary, and the reordering of states and caches behind it."""
import math

import torch

own = False

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32, "e4m3": E4M3}


def _case(name, op, **sizes):
    c = {"op": op, **sizes}
    return {"name": name, **c} if name else c


def decode(name, dtype, batch, low, high, heads, group, d_k, d_v, page, slot_first=False):
    """One new token of each of `batch` sequences against `low` to `high` cached positions; every head of the cache serves `group` heads of the queries."""
    return _case(name, "decode", dtype=dtype, batch=batch, low=low, high=high, heads=heads, group=group, d_k=d_k, d_v=d_v, page=page, slot_first=slot_first)


def write(name, dtype, batch, length, low, high, heads, d_k, d_v, page, slot_first=False):
    """`length` new rows of each sequence behind `low` to `high` positions that are there; an 8-bit cache gives the new rows back as what it holds of them."""
    return _case(name, "write", dtype=dtype, batch=batch, length=length, low=low, high=high, heads=heads, d_k=d_k, d_v=d_v, page=page, slot_first=slot_first)


def read(name, dtype, batch, low, high, heads, d_k, d_v, page, slot_first=False):
    """All of the `low` to `high` positions that each sequence has, as dense rows in bf16."""
    return _case(name, "read", dtype=dtype, batch=batch, low=low, high=high, heads=heads, d_k=d_k, d_v=d_v, page=page, slot_first=slot_first)


def select(name, dtype, batch, beams, slots, vocab, finished=0.0):
    return _case(name, "select", dtype=dtype, batch=batch, beams=beams, slots=slots, vocab=vocab, finished=finished)


def reorder_cache(name, dtype, batch, beams, low, high, heads, d_k, d_v, page, slot_first=False):
    return _case(name, "reorder_cache", dtype=dtype, batch=batch, beams=beams, low=low, high=high, heads=heads, d_k=d_k, d_v=d_v, page=page, slot_first=slot_first)


def reorder_states(name, dtype, batch, beams, length, width):
    return _case(name, "reorder_states", dtype=dtype, batch=batch, beams=beams, length=length, width=width)


def listed():
    return [
        # one sequence of some hundred words, heads as the attention block trains them: a reader waits for each word, all latency
        decode("decode one", "bf16", 1, 300, 512, 16, 1, 64, 64, 16),
        # a served batch whose sequences have got unequally far, as many heads in the cache as in the queries
        decode("decode", "bf16", 64, 100, 4096, 16, 1, 128, 128, 16),
        # a few long documents in an 8-bit cache, eight heads of queries to a head of the cache
        decode("decode long e4m3", "e4m3", 4, 30000, 65536, 8, 8, 128, 128, 64),
        # sizes that no tile divides, heads of keys and values of unlike width, some sequences only begun, rows of a position beside each other
        decode("decode ragged", "bf16", 37, 0, 777, 5, 3, 72, 40, 24, slot_first=True),
        # the token that a served batch has just made
        write("write tokens", "bf16", 64, 1, 100, 700, 16, 128, 128, 16),
        # prompts of a batch into an 8-bit cache, and what their attention reads of them
        write("write prompts e4m3", "e4m3", 32, 512, 0, 0, 16, 64, 64, 64),
        # the cached prefix of a prompt that goes on, for attention over all of it
        read("read e4m3", "e4m3", 8, 1000, 16384, 8, 128, 128, 64),
        # odd sizes and few rows, as they come
        read("read ragged", "bf16", 5, 1, 333, 6, 80, 48, 20, slot_first=True),
        # four beams of one sentence over the benchmark's vocabulary
        select("select one", "bf16", 1, 4, 4, 32768),
        # eight beams each of a batch of sentences, a wide vocabulary, some of them finished
        select("select wide", "bf16", 64, 8, 8, 131072, finished=0.1),
        # the caches of a batch's beams: tables change hands, pages that go on are copied
        reorder_cache("reorder cache", "bf16", 32, 8, 40, 400, 16, 64, 64, 16),
        # a state that is kept densely, a row a beam
        reorder_states("reorder states", "bf16", 16, 4, 256, 1024),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(low * (high / low) ** rng.random()))))


def draw(rng):
    op = rng.choice(["decode", "decode", "decode", "write", "read", "select", "select", "reorder_cache", "reorder_states"])
    dtype = rng.choice(["bf16", "e4m3"])
    step = 8 if dtype == "bf16" else 16
    d_k = rng.choice([64, 128, 64, 128, 32, 96, 256, step * rng.randint(1, 256 // step)])
    d_v = rng.choice([d_k, d_k, d_k, step * rng.randint(1, 256 // step)])
    page, slot_first = rng.choice([16, 16, 32, 64, 128, rng.randint(1, 100)]), rng.random() < 0.4
    heads, batch = _log(rng, 1, 32), _log(rng, 1, 128)

    def positions(high, rows, budget):
        """As many positions as the budget of bytes lets `rows` sequences have."""
        each = heads * (d_k + d_v) * (2 if dtype == "bf16" else 1) * rows
        return max(1, min(high, budget // each))

    if op == "decode":
        high = positions(_log(rng, 16, 65536), batch, 500 << 20)
        return decode("", dtype, batch, rng.choice([0, 1, high // 2, high]), high, heads, rng.choice([1, 1, 2, 4, 8, 16, rng.randint(1, 20)]), d_k, d_v, page, slot_first)
    if op == "write":
        length = positions(rng.choice([1, _log(rng, 2, 1024)]), batch, 60 << 20)
        return write("", dtype, batch, length, 0, positions(_log(rng, 1, 2048), batch, 200 << 20), heads, d_k, d_v, page, slot_first)
    if op == "read":
        high = positions(_log(rng, 4, 16384), batch, 120 << 20)
        return read("", dtype, batch, high // 3, high, heads, d_k, d_v, page, slot_first)
    if op == "reorder_cache":
        batch, beams = _log(rng, 1, 32), rng.randint(2, 12)
        high = positions(_log(rng, 2, 2000), batch * beams, 400 << 20)
        return reorder_cache("", "bf16", batch, beams, high // 4, high, heads, d_k, d_v, page, slot_first)
    if op == "reorder_states":
        batch, beams, width = _log(rng, 1, 32), rng.randint(2, 12), _log(rng, 5, 2000)
        return reorder_states("", rng.choice(["bf16", "f32"]), batch, beams, max(1, min(_log(rng, 1, 500), (8 << 20) // (batch * beams * width))), width)
    vocab, beams = _log(rng, 1000, 131072), rng.randint(1, 12)
    if rng.random() < 0.5:
        vocab = vocab // 8 * 8
    dtype = rng.choice(["bf16", "f32"])
    batch = max(1, min(_log(rng, 1, 64), (60 << 20) // (vocab * beams * (2 if dtype == "bf16" else 4))))
    return select("", dtype, batch, beams, rng.choice([beams, beams, 2 * beams]), vocab, rng.choice([0.0, 0.2]))


# ---- inputs ---------------------------------------------------------------------------------------------------

def _lengths(case, rows):
    """Positions that each sequence has: spread over the range, fixed by the case's sizes.  (A range from 0 has a sequence without any and one of one position.)"""
    low, high = case["low"], case["high"]
    n = [low + (high - low) * (61 * i % 97) // 96 for i in range(rows)]
    if rows > 1:
        n[-1] = high
    return n


class _State:
    pass


def _pool(s, c, rows, capacity, normal, g):
    """A pool of pages with a little more than `rows` sequences of `capacity` positions take, and the pages that each has, in an order that an allocator leaves."""
    heads, page = c["heads"], c["page"]
    each = -(-max(1, capacity) // page)
    s.pages = rows * each + (2 * rows if c["op"] == "reorder_cache" else 3)

    def side(d):
        shape = (s.pages, page, heads, d) if c["slot_first"] else (s.pages, heads, page, d)
        x = torch.empty(shape, dtype=BF16, device="cuda")
        flat = x.view(-1)
        flat.copy_(normal(1 << 16).to(BF16).repeat(-(-flat.numel() // (1 << 16)) + 1)[17:17 + flat.numel()])
        # rows differ by position, so that attention has something to weigh
        x.mul_((0.5 + torch.rand(shape[:3], generator=g, device="cuda")).to(BF16)[..., None])
        if c["dtype"] == "bf16":
            return x, None
        return _quantise(x.float())

    s.k, s.k_scale = side(c["d_k"])
    s.v, s.v_scale = side(c["d_v"])
    order = torch.randperm(s.pages, generator=g, device="cuda").to(torch.int32)
    s.table = order[:rows * each].view(rows, each).contiguous()
    s.spare = order[rows * each:].contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s, c = _State(), case
    s.case, s.handles, op, batch = case, None, case["op"], case["batch"]
    if op in ("decode", "write", "read"):
        lengths = _lengths(c, batch)
        _pool(s, c, batch, max(lengths) + c.get("length", 0), normal, g)
        s.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if op == "decode":
        s.q = (normal(batch, c["heads"], c["group"], c["d_k"]) * 1.5).to(BF16)
    elif op == "write":
        length = c["length"]
        # (a batch of prompts is padded to its longest)
        s.counts = torch.tensor([max(1, length - 29 * i % max(1, length // 2 + 1)) for i in range(batch)], dtype=torch.int32, device="cuda")
        s.kk = normal(batch, length, c["heads"], c["d_k"]).to(BF16)
        s.vv = (normal(batch, length, c["heads"], c["d_v"]) * 0.3).to(BF16)
    elif op == "select":
        beams, vocab = c["beams"], c["vocab"]
        z = normal(batch * beams, vocab).mul_(2.0)
        # some words stand out, others beams' words among them
        z.scatter_add_(1, (torch.rand((batch * beams, 64), generator=g, device="cuda") * vocab).long().clamp_(max=vocab - 1), 4.0 + 3.0 * normal(batch * beams, 64))
        s.logits = z.to(TYPES[c["dtype"]]).view(batch, beams, vocab)
        del z
        s.scores = (-20.0 + 3.0 * normal(batch, beams)).contiguous()
        s.finished = (torch.rand((batch, beams), generator=g, device="cuda") < c["finished"]).to(torch.int32)
        s.end_id = 1
    elif op == "reorder_cache":
        beams = c["beams"]
        _pool(s, c, batch * beams, c["high"], normal, g)
        n = torch.tensor(_lengths(c, batch), dtype=torch.int32, device="cuda")
        s.lengths = n[:, None].expand(batch, beams).contiguous()                     # (a sentence's beams are of one length)
        s.table = s.table.view(batch, beams, -1)
        s.fresh = s.spare[:batch * beams].view(batch, beams).contiguous()
    elif op == "reorder_states":
        s.states = normal(batch, c["beams"], c["length"], c["width"]).to(TYPES[c["dtype"]])
    if op.startswith("reorder"):
        s.parents = (torch.rand((batch, c["beams"]), generator=g, device="cuda") * c["beams"]).int().clamp_(max=c["beams"] - 1)
    torch.cuda.empty_cache()
    return s


# ---- one pass -------------------------------------------------------------------------------------------------

def run(s):
    call = _own if own else _plain
    return call(s, s.case)


def _handles(s, c):
    """The library's handles, descriptors and the tensors that it writes, as a program keeps them from step to step."""
    import paper_1811_02084_b200 as mtf
    h, op = _State(), c["op"]
    h.mtf, h.layout = mtf, mtf.mtf_layout(mtf.mtf_mesh_create([("all", 1)]), [])
    seq = ["batch", "beam"] if op == "reorder_cache" else ["batch"]

    def room(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if "page" in c:
        inner = ["slot", "heads"] if c["slot_first"] else ["heads", "slot"]
        scales = [None, None] if s.k_scale is None else [mtf.named(x, ["page"] + inner) for x in (s.k_scale, s.v_scale)]
        h.cache = mtf.Cache(mtf.named(s.k, ["page"] + inner + ["d_k"]), mtf.named(s.v, ["page"] + inner + ["d_v"]), s.table, *scales)
    if op == "decode":
        h.out = room((c["batch"], c["heads"], c["group"], c["d_v"]), BF16)
        h.q, h.o = mtf.named(s.q, seq + ["heads", "group", "d_k"]), mtf.named(h.out, seq + ["heads", "group", "d_v"])
        h.workspace = room((max(16, mtf.mtf_attention_decode_workspace_bytes(h.layout, h.q, h.cache)),), torch.uint8)
    elif op in ("write", "read"):
        dense, n = seq + ["memory_length", "heads"], c["length"] if op == "write" else c["high"]
        h.kk_out, h.vv_out = (room((c["batch"], n, c["heads"], d), BF16) for d in (c["d_k"], c["d_v"]))
        h.kk_back, h.vv_back = mtf.named(h.kk_out, dense + ["d_k"]), mtf.named(h.vv_out, dense + ["d_v"])
        if op == "write":
            h.kk, h.vv = mtf.named(s.kk, dense + ["d_k"]), mtf.named(s.vv, dense + ["d_v"])
    elif op == "select":
        shape = (c["batch"], c["slots"])
        h.parents, h.tokens, h.finished, h.new_scores = room(shape, torch.int32), room(shape, torch.int32), room(shape, torch.int32), room(shape, F32)
        h.logits, h.scores, h.n_new = mtf.named(s.logits, ["batch", "beam", "vocab"]), mtf.named(s.scores, ["batch", "beam"]), mtf.named(h.new_scores, ["batch", "beam_out"])
        h.workspace = room((max(16, mtf.mtf_beam_select_workspace_bytes(h.layout, h.logits, c["slots"])),), torch.uint8)
    elif op == "reorder_cache":
        h.table, h.lengths = torch.empty_like(s.table), torch.empty_like(s.lengths)
    else:
        dims = ["batch", "beam", "length", "width"]
        h.new_states = torch.empty_like(s.states)
        h.states, h.out = mtf.named(s.states, dims), mtf.named(h.new_states, dims)
    return h


def _own(s, c):
    if s.handles is None:
        s.handles = _handles(s, c)
    h, op = s.handles, c["op"]
    mtf = h.mtf
    if op == "decode":
        mtf.mtf_attention_decode(h.layout, h.q, h.cache, s.lengths, c["d_k"] ** -0.5, h.o, h.workspace)
        return h.out
    if op == "write":
        mtf.mtf_cache_write(h.layout, h.kk, h.vv, s.lengths, s.counts, h.cache)
        if c["dtype"] == "bf16":
            return {"k": s.k, "v": s.v}
        mtf.mtf_cache_read(h.layout, h.cache, s.lengths, s.counts, h.kk_back, h.vv_back)
        return {"kk": h.kk_out, "vv": h.vv_out}
    if op == "read":
        mtf.mtf_cache_read(h.layout, h.cache, None, s.lengths, h.kk_back, h.vv_back)
        return {"kk": h.kk_out, "vv": h.vv_out}
    if op == "select":
        mtf.mtf_beam_select(h.layout, h.logits, h.scores, s.finished, s.end_id, h.parents, h.tokens, h.n_new, h.finished, h.workspace)
        return {"parents": h.parents, "tokens": h.tokens, "scores": h.new_scores, "finished": h.finished}
    if op == "reorder_cache":
        mtf.mtf_cache_reorder(h.layout, h.cache, s.parents, s.lengths, s.fresh, h.table, h.lengths)
        return {"table": h.table, "lengths": h.lengths, "k": s.k, "v": s.v}
    mtf.mtf_beam_reorder(h.layout, "beam", s.parents, h.states, h.out)
    return h.new_states


def _quantise(x):
    """Rows of e4m3 and their scale: the smallest power of two by which the row's largest value is at most 448, e4m3's largest (1 for a row of zeros)."""
    m, e = torch.frexp(x.abs().amax(-1))                                             # = m 2^e, m from 1/2 up to 1; 448 = 7/8 2^9
    e = torch.where(m > 0, e - 9 + (m > 0.875).to(e.dtype), 0)
    scale = torch.ldexp(torch.ones_like(m), e)
    return (x / scale[..., None]).to(E4M3), scale


def _rows(c, pool, page, slot):
    """Rows of a pool's pages, [..., heads, d] (scales: [..., heads])."""
    raw = pool.view(torch.uint8) if pool.dtype == E4M3 else pool
    got = raw[page, slot] if c["slot_first"] else raw[page, :, slot]
    return got.view(E4M3) if pool.dtype == E4M3 else got


def _dense(s, c, first, n):
    """Positions first .. first + n - 1 of each sequence as f32 rows [sequence, n, heads, d], keys and values."""
    at = (first[:, None] + torch.arange(n, device="cuda")).long()
    index = (at // c["page"]).clamp(max=s.table.shape[-1] - 1)
    page, slot = s.table.gather(1, index).long(), at % c["page"]
    got = [_rows(c, x, page, slot).float() for x in (s.k, s.v)]
    if s.k_scale is not None:
        got = [x * _rows(c, y, page, slot)[..., None] for x, y in zip(got, (s.k_scale, s.v_scale))]
    return got


def _plain(s, c):
    return {"decode": _plain_decode, "write": _plain_write, "read": _plain_read, "select": _plain_select, "reorder_cache": _plain_reorder_cache,
            "reorder_states": _plain_reorder_states}[c["op"]](s, c)


def _plain_decode(s, c):
    n = s.lengths.long()
    k, v = _dense(s, c, torch.zeros_like(n), c["high"])
    z = torch.einsum("bhgd,blhd->bhgl", s.q.float(), k) * c["d_k"] ** -0.5
    there = (torch.arange(c["high"], device="cuda") < n[:, None])[:, None, None]
    z = torch.where(there, z, -torch.inf)
    p = torch.where(there, (z - z.amax(-1, keepdim=True)).exp(), 0.0)
    o = torch.einsum("bhgl,blhd->bhgd", p, v) / p.sum(-1, keepdim=True)
    return torch.where(n[:, None, None, None] > 0, o, 0.0).to(BF16)


def _plain_write(s, c):
    i = torch.arange(c["length"], device="cuda")
    real = i < s.counts[:, None]
    at = (s.lengths[:, None] + i).long()
    page, slot = s.table.gather(1, at // c["page"]).long()[real], (at % c["page"])[real]
    for new, pool, scales in ((s.kk, s.k, s.k_scale), (s.vv, s.v, s.v_scale)):
        new = new[real]
        if scales is not None:
            new, scale = _quantise(new.float())
            _put(c, scales, page, slot, scale)
        _put(c, pool, page, slot, new)
    if c["dtype"] == "bf16":
        return {"k": s.k, "v": s.v}
    kk, vv = (torch.where(real[..., None, None], x, 0.0).to(BF16) for x in _dense(s, c, s.lengths, c["length"]))
    return {"kk": kk, "vv": vv}


def _put(c, pool, page, slot, rows):
    to = pool.view(torch.uint8) if pool.dtype == E4M3 else pool
    (to if c["slot_first"] else to.transpose(1, 2))[page, slot] = rows.view(torch.uint8) if pool.dtype == E4M3 else rows


def _plain_read(s, c):
    n = s.lengths.long()
    there = (torch.arange(c["high"], device="cuda") < n[:, None])[..., None, None]
    kk, vv = (torch.where(there, x, 0.0).to(BF16) for x in _dense(s, c, torch.zeros_like(n), c["high"]))
    return {"kk": kk, "vv": vv}


def _plain_select(s, c):
    batch, beams, vocab, slots = c["batch"], c["beams"], c["vocab"], c["slots"]
    z = s.logits.float()
    top = z.amax(-1, keepdim=True)
    lse = top[..., 0].double() + (z - top).exp().sum(-1, dtype=torch.float64).log()
    # a key of 64 bits that orders a beam's words: the logit's bits in rising order in front, and behind them the lower index first
    bits = (z + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits) * (1 << 32) + (vocab - 1 - torch.arange(vocab, device="cuda"))
    words = vocab - 1 - (key.topk(min(slots, vocab), -1).values & 0xffffffff)
    done = s.finished[..., None] != 0
    # a beam's best words, a finished beam's end and nothing else; then the best over the beams
    first = torch.arange(words.shape[-1], device="cuda") == 0
    value = s.scores[..., None].double() + torch.where(done, torch.where(first, 0.0, -torch.inf), z.gather(-1, words).double() - lse[..., None])
    words = torch.where(done, s.end_id, words)
    best, which = value.view(batch, -1).sort(dim=-1, descending=True, stable=True)
    best, which = best[:, :slots], which[:, :slots]
    parents, tokens = which // words.shape[-1], words.view(batch, -1).gather(1, which)
    ended = (tokens == s.end_id) | (s.finished.gather(1, parents) != 0)
    return {"parents": parents.int(), "tokens": tokens.int(), "scores": best.float(), "finished": ended.int()}


def _plain_reorder_cache(s, c):
    page, each = c["page"], s.table.shape[-1]
    parents = s.parents.long()
    n = s.lengths.gather(1, parents)
    table = s.table.gather(1, parents[..., None].expand(-1, -1, each))
    whole = (n // page).long()
    goes_on = (n % page != 0) & (whole < each)
    last = table.gather(2, whole.clamp(max=each - 1)[..., None])[..., 0]
    # the rows in use of a page that goes on, into the beam's own page
    slot = torch.arange(page, device="cuda")
    used = goes_on[..., None] & (slot < (n % page)[..., None])
    row, column = last[..., None].expand(used.shape)[used].long(), slot.expand(used.shape)[used]
    to = s.fresh[..., None].expand(used.shape)[used].long()
    for x in (s.k, s.v):
        _put(c, x, to, column, _rows(c, x, row, column))
    table = torch.where((torch.arange(each, device="cuda") == whole[..., None]) & goes_on[..., None], s.fresh[..., None], table)
    return {"table": table, "lengths": n, "k": s.k, "v": s.v}


def _plain_reorder_states(s, c):
    b, p = torch.arange(c["batch"], device="cuda")[:, None], s.parents.long()
    return s.states[b, p]


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    c, op = case, case["op"]
    size = {"bf16": 2, "f32": 4, "e4m3": 1}[c["dtype"]]
    if "page" in c:
        widths = c["d_k"] + c["d_v"]
        row = c["heads"] * (widths * size + (8 if c["dtype"] == "e4m3" else 0))         # a position in the cache, its scales too
        dense = c["heads"] * widths * 2
        positions = sum(_lengths(c, c["batch"]))
    if op == "decode":
        return {"bytes": positions * row + 4 * c["batch"] * (1 + c["high"] // c["page"]) + c["batch"] * c["group"] * dense,
                "flops": 2 * positions * c["heads"] * c["group"] * widths}
    if op == "write":
        length = c["length"]
        new = sum(max(1, length - 29 * i % max(1, length // 2 + 1)) for i in range(c["batch"]))
        if c["dtype"] == "bf16":
            return {"bytes": new * (dense + row), "flops": 0}
        return {"bytes": new * (dense + 2 * row) + c["batch"] * length * dense, "flops": 2 * new * c["heads"] * widths}
    if op == "read":
        return {"bytes": positions * row + c["batch"] * c["high"] * dense, "flops": positions * c["heads"] * widths}
    if op == "select":
        n = c["batch"] * c["beams"] * c["vocab"]
        return {"bytes": n * size * (1 - c["finished"]) + c["batch"] * (8 * c["beams"] + 16 * c["slots"]), "flops": 3 * n * (1 - c["finished"])}
    if op == "reorder_cache":
        tails = c["beams"] * sum(n % c["page"] for n in _lengths(c, c["batch"]))
        return {"bytes": 2 * tails * row + 8 * c["batch"] * c["beams"] * -(-c["high"] // c["page"]), "flops": 0}
    return {"bytes": 2 * c["batch"] * c["beams"] * c["length"] * c["width"] * size, "flops": 0}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _values(c, pool, scales, pages, n):
    """The first n rows of a list of pages, position by position, in 64 bits."""
    def of(x):
        raw = x.view(torch.uint8) if x.dtype == E4M3 else x
        y = raw.index_select(0, pages)
        y = (y if c["slot_first"] else y.transpose(1, 2)).flatten(0, 1)[:n].contiguous()
        return (y.view(E4M3).float() if x.dtype == E4M3 else y).double()
    return of(pool) if scales is None else of(pool) * of(scales)[..., None]


def exact(case, seed):
    s, c, op = prepare(case, seed), case, case["op"]
    if op == "decode":
        out = torch.zeros(c["batch"], c["heads"], c["group"], c["d_v"], dtype=torch.float64, device="cuda")
        for b, n in enumerate(s.lengths.tolist()):
            if n:
                pages = s.table[b, :-(-n // c["page"])].long()
                k, v = _values(c, s.k, s.k_scale, pages, n), _values(c, s.v, s.v_scale, pages, n)
                for h in range(c["heads"]):
                    z = s.q[b, h].double() @ k[:, h].T / math.sqrt(c["d_k"])
                    out[b, h] = torch.softmax(z, -1) @ v[:, h]
        return out
    if op == "write":
        if c["dtype"] == "bf16":
            for b, (n, m) in enumerate(zip(s.lengths.tolist(), s.counts.tolist())):
                for new, pool in ((s.kk, s.k), (s.vv, s.v)):
                    at = torch.arange(n, n + m, device="cuda")
                    page, slot = s.table[b].long()[at // c["page"]], at % c["page"]
                    if c["slot_first"]:
                        pool[page, slot] = new[b, :m]
                    else:
                        pool[page, :, slot] = new[b, :m]
            return {"k": s.k.double(), "v": s.v.double()}
        real = (torch.arange(c["length"], device="cuda") < s.counts[:, None])[..., None, None]
        return {name: _nearest(x.double()).where(real, 0.0) for name, x in (("kk", s.kk), ("vv", s.vv))}
    if op == "read":
        out = {}
        for name, pool, scales, d in (("kk", s.k, s.k_scale, c["d_k"]), ("vv", s.v, s.v_scale, c["d_v"])):
            out[name] = torch.zeros(c["batch"], c["high"], c["heads"], d, dtype=torch.float64, device="cuda")
            for b, n in enumerate(s.lengths.tolist()):
                out[name][b, :n] = _values(c, pool, scales, s.table[b].long(), n)
        return out
    if op == "select":
        got = []
        for b in range(c["batch"]):
            value = s.scores[b].double()[:, None] + torch.log_softmax(s.logits[b].double(), -1)
            alone = torch.full_like(value, -math.inf)
            alone[:, s.end_id] = s.scores[b].double()
            got.append(torch.where(s.finished[b][:, None] != 0, alone, value).flatten().topk(c["slots"]).values)
        return {"parents": None, "tokens": None, "scores": torch.stack(got), "finished": None}
    if op == "reorder_states":
        return torch.stack([torch.stack([s.states[b, p] for p in row]) for b, row in enumerate(s.parents.tolist())]).double()
    for b, row in enumerate(s.parents.tolist()):
        n = int(s.lengths[b, 0])                                                     # (one for all beams of a sentence)
        for i, p in enumerate(row):
            if n % c["page"]:
                of, to = int(s.table[b, p, n // c["page"]]), int(s.fresh[b, i])
                rows = (slice(None), slice(0, n % c["page"]))[c["slot_first"]:] + (slice(None),)
                for pool in (s.k, s.v):
                    pool[(to,) + rows] = pool[(of,) + rows]
    return {"table": None, "lengths": None, "k": s.k.double(), "v": s.v.double()}


def _nearest(x):
    """Each value as an 8-bit row holds it: to 4 significant bits, or to a step of 2^-9, of the row's scale; halves to the even neighbour."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)))
    y = x / torch.where(top > 0, scale, 1.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.where(top > 0, scale, 1.0)
