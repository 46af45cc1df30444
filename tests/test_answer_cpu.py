"""The calls of answering refuse what they do not take, before anything is launched (no GPU: tensors in host memory)."""
import pytest
import torch

import paper_1811_02084_b200 as mtf

B, L, H, G, P, S, D, N = 2, 3, 2, 3, 7, 4, 16, 5          # sequences, rows, heads, group, pages, slots, width, pages of a sequence
SENT, BEAMS, OUT, V = 2, 3, 4, 20


def lay(mesh=(("all", 1),), rules=()):
    return mtf.mtf_layout(mtf.mtf_mesh_create(list(mesh)), list(rules))


def ranks(rules):
    return mtf.mtf_layout_bind_ranks(lay((("r", 2), ("all", 1)), rules), "r", 2, 0)


def room(nbytes):
    """16-byte aligned bytes."""
    raw = torch.zeros(nbytes + 16, dtype=torch.uint8)
    return raw[-raw.data_ptr() % 16:][:nbytes]


def tensor(shape, dtype):
    n = 1
    for s in shape:
        n *= s
    return room(n * torch.empty(0, dtype=dtype).element_size()).view(dtype).view(*shape)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def things(e4m3=False, slot_first=True):
    t = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    inner, shape = (["slot", "heads"], (P, S, H)) if slot_first else (["heads", "slot"], (P, H, S))
    n = {"layout": lay(), "k": mtf.named(tensor(shape + (D,), t), ["page"] + inner + ["d_k"]), "v": mtf.named(tensor(shape + (2 * D,), t), ["page"] + inner + ["d_v"]),
         "k_scale": None, "v_scale": None, "table": ints(B, N), "slot": "slot"}
    if e4m3:
        n["k_scale"], n["v_scale"] = (mtf.named(tensor(shape, torch.float32), ["page"] + inner) for _ in range(2))
    n["kk"] = mtf.named(tensor((B, L, H, D), torch.bfloat16), ["batch", "length", "heads", "d_k"])
    n["vv"] = mtf.named(tensor((B, L, H, 2 * D), torch.bfloat16), ["batch", "length", "heads", "d_v"])
    n["starts"], n["counts"], n["lengths"] = ints(B), ints(B), ints(B)
    n["q"] = mtf.named(tensor((B, H, G, D), torch.bfloat16), ["batch", "heads", "group", "d_k"])
    n["o"] = mtf.named(tensor((B, H, G, 2 * D), torch.bfloat16), ["batch", "heads", "group", "d_v"])
    n["scale"], n["workspace"] = 0.25, None
    # beam search
    n["logits"] = mtf.named(tensor((SENT, BEAMS, V), torch.float32), ["sentence", "beam", "vocab"])
    n["scores"] = mtf.named(tensor((SENT, BEAMS), torch.float32), ["sentence", "beam"])
    n["new_scores"] = mtf.named(tensor((SENT, OUT), torch.float32), ["sentence", "out"])
    n["finished"], n["end_id"], n["parents"], n["tokens"], n["new_finished"] = ints(SENT, BEAMS), 1, ints(SENT, OUT), ints(SENT, OUT), ints(SENT, OUT)
    n["beam_ws"] = room(1 << 16)
    n["beam"] = "beam"
    n["states"] = mtf.named(tensor((SENT, BEAMS, 5), torch.float32), ["sentence", "beam", "x"])
    n["out"] = mtf.named(tensor((SENT, OUT, 5), torch.float32), ["sentence", "beam", "x"])
    n["beam_table"], n["beam_lengths"], n["fresh"] = ints(SENT, BEAMS, N), ints(SENT, BEAMS), ints(SENT, OUT)
    n["new_table"], n["new_lengths"] = ints(SENT, OUT, N), ints(SENT, OUT)
    return n


def call(op, n):
    l = n["layout"]
    cache = lambda table: mtf.Cache(n["k"], n["v"], table, n["k_scale"], n["v_scale"], n["slot"])                  # noqa: E731
    if op == "write":
        return mtf.mtf_cache_write(l, n["kk"], n["vv"], n["starts"], n["counts"], cache(n["table"]))
    if op == "read":
        return mtf.mtf_cache_read(l, cache(n["table"]), n["starts"], n["counts"], n["kk"], n["vv"])
    if op == "decode":
        return mtf.mtf_attention_decode(l, n["q"], cache(n["table"]), n["lengths"], n["scale"], n["o"], n["workspace"])
    if op == "select":
        return mtf.mtf_beam_select(l, n["logits"], n["scores"], n["finished"], n["end_id"], n["parents"], n["tokens"], n["new_scores"], n["new_finished"], n["beam_ws"])
    if op == "reorder":
        return mtf.mtf_beam_reorder(l, n["beam"], n["parents"], n["states"], n["out"])
    return mtf.mtf_cache_reorder(l, cache(n["beam_table"]), n["parents"], n["beam_lengths"], n["fresh"], n["new_table"], n["new_lengths"])


def refused(op, change, code="MTF_ERR_INVALID_ARG", **kind):
    n = things(**kind)
    n.update(change(n) if callable(change) else change)
    n0 = mtf.mtf_launch_count()
    with pytest.raises(mtf.MtfError) as e:
        call(op, n)
    assert e.value.code == code, e.value
    assert mtf.mtf_launch_count() == n0


READS = {"write": ["kk", "vv", "k", "v"], "read": ["kk", "vv", "k", "v"], "decode": ["q", "o", "k", "v"], "select": ["logits", "scores", "new_scores"],
         "reorder": ["states", "out"], "cache_reorder": ["k", "v"]}
IDS = {"write": ["starts", "counts"], "read": ["starts", "counts"], "decode": ["lengths"], "select": ["finished", "parents", "tokens", "new_finished"], "reorder": ["parents"],
       "cache_reorder": ["parents", "beam_lengths", "fresh", "new_table", "new_lengths"]}
MAY_BE_NONE = {"starts", "counts", "finished", "new_finished"}
PAGED = ["write", "read", "decode", "cache_reorder"]


def as_type(t, dtype):
    return mtf.named(tensor(t.owner.shape, dtype), t.names)


def renamed(t, of, to):
    return mtf.named(t.owner, [to if x == of else x for x in t.names])


@pytest.mark.parametrize("op", READS)
def test_missing_tensors_and_descriptors_without_data(op):
    for name in READS[op]:
        refused(op, {name: None})
        refused(op, lambda n: {name: mtf.Named(n[name].dims, n[name].dtype)})
    for name in IDS[op]:
        if name not in MAY_BE_NONE:
            refused(op, {name: None})
        refused(op, lambda n: {name: n[name].long()})
        refused(op, lambda n: {name: torch.cat([n[name], n[name]], -1)[..., ::2]})
        refused(op, lambda n: {name: torch.cat([n[name], n[name]])}, "MTF_ERR_SIZE_MISMATCH")


@pytest.mark.parametrize("op", PAGED)
@pytest.mark.parametrize("slot_first", [True, False])
def test_caches_that_are_none(op, slot_first):
    kind = {"slot_first": slot_first}
    table = "beam_table" if op == "cache_reorder" else "table"
    refused(op, {table: None}, **kind)
    refused(op, lambda n: {table: n[table].long()}, **kind)
    refused(op, lambda n: {table: n[table][:1].contiguous()}, "MTF_ERR_SIZE_MISMATCH", **kind)
    refused(op, lambda n: {"k": as_type(n["k"], torch.float32), "v": as_type(n["v"], torch.float32)}, "MTF_ERR_UNSUPPORTED", **kind)
    refused(op, lambda n: {"v": as_type(n["v"], torch.float8_e4m3fn)}, **kind)
    refused(op, {"slot": "place"}, "MTF_ERR_UNKNOWN_DIM", **kind)
    refused(op, lambda n: {"k": renamed(n["k"], "page", "leaf")}, "MTF_ERR_SIZE_MISMATCH", **kind)
    refused(op, lambda n: {"k": mtf.named(n["k"].owner[:-1], n["k"].names)}, "MTF_ERR_SIZE_MISMATCH", **kind)
    # scales where there is none to have, and none where there is
    refused(op, lambda n: {"k_scale": things(True, slot_first)["k_scale"]}, **kind)
    for s in ("k_scale", "v_scale"):
        refused(op, {s: None}, e4m3=True, **kind)
        refused(op, lambda n: {s: as_type(n[s], torch.bfloat16)}, "MTF_ERR_UNSUPPORTED", e4m3=True, **kind)
        refused(op, lambda n: {s: mtf.named(n[s].owner[:-1].contiguous(), n[s].names)}, "MTF_ERR_SIZE_MISMATCH", e4m3=True, **kind)
    # widths that no 16-byte piece divides, or beyond the kernels'
    for d in (12, 264):
        def narrow(n):
            return {"k": mtf.named(tensor(n["k"].owner.shape[:3] + (d,), torch.bfloat16), n["k"].names), "q": mtf.named(tensor((B, H, G, d), torch.bfloat16), n["q"].names),
                    "kk": mtf.named(tensor((B, L, H, d), torch.bfloat16), n["kk"].names)}
        refused(op, narrow, "MTF_ERR_UNSUPPORTED", **kind)
    # memory
    for name in ("k", "v"):
        refused(op, lambda n: {name: mtf.Named(n[name].dims, n[name].dtype, n[name].ptr + 2, n[name].owner)}, "MTF_ERR_UNSUPPORTED", **kind)
    if op in ("write", "cache_reorder"):
        refused(op, lambda n: {"v": mtf.Named(n["v"].dims, n["v"].dtype, n["k"].ptr, n["k"].owner)}, **kind)
    # layouts
    for dim in ("page", "slot", "d_k", "d_v"):
        sizes = dict(page=P, slot=S, d_k=D, d_v=2 * D)
        if sizes[dim] % 2 == 0:
            refused(op, {"layout": ranks([(dim, "r")])}, "MTF_ERR_UNSUPPORTED", **kind)
    refused(op, {"layout": lay((("m", 2),), [("heads", "m"), ("slot", "m")])}, "MTF_ERR_ILLEGAL_LAYOUT", **kind)
    refused(op, {"layout": lay((("m", 5),), [("heads", "m")])}, "MTF_ERR_NOT_DIVISIBLE", **kind)


@pytest.mark.parametrize("op", ["write", "read"])
def test_dense_rows(op):
    for name in ("kk", "vv"):
        refused(op, lambda n: {name: mtf.named(n[name].owner[0], n[name].names[1:])}, "MTF_ERR_SIZE_MISMATCH")
        refused(op, lambda n: {name: mtf.named(tensor((B, L, H, 64), torch.bfloat16), n[name].names)}, "MTF_ERR_SIZE_MISMATCH")
        refused(op, lambda n: {name: mtf.Named(n[name].dims, n[name].dtype, n[name].ptr + 8, n[name].owner)}, "MTF_ERR_UNSUPPORTED")
    refused(op, lambda n: {"vv": as_type(n["vv"], torch.float32)})
    refused(op, lambda n: {"kk": as_type(n["kk"], torch.float8_e4m3fn), "vv": as_type(n["vv"], torch.float8_e4m3fn)}, "MTF_ERR_UNSUPPORTED")
    refused(op, lambda n: {"kk": renamed(n["kk"], "heads", "h"), "vv": renamed(n["vv"], "heads", "h")}, "MTF_ERR_SIZE_MISMATCH")
    refused(op, lambda n: {"vv": renamed(n["vv"], "length", "other")}, "MTF_ERR_SIZE_MISMATCH")
    refused(op, lambda n: {"vv": mtf.Named(n["vv"].dims, n["vv"].dtype, n["v"].ptr, n["v"].owner)})
    # heads and sequences on one mesh dimension: two dims of one tensor
    refused(op, {"layout": lay((("m", 2),), [("heads", "m"), ("batch", "m")])}, "MTF_ERR_ILLEGAL_LAYOUT")
    # ... and dims of two tensors of the call
    refused(op, {"layout": lay((("m", 2),), [("slot", "m"), ("batch", "m")])}, "MTF_ERR_ILLEGAL_LAYOUT")


def test_attention():
    refused("decode", lambda n: {"q": as_type(n["q"], torch.float32)}, "MTF_ERR_UNSUPPORTED")
    refused("decode", lambda n: {"o": as_type(n["o"], torch.float32)}, "MTF_ERR_UNSUPPORTED")
    refused("decode", lambda n: {"q": renamed(n["q"], "heads", "h")}, "MTF_ERR_SIZE_MISMATCH")
    refused("decode", lambda n: {"o": renamed(n["o"], "group", "g")}, "MTF_ERR_SIZE_MISMATCH")
    refused("decode", lambda n: {"o": mtf.named(tensor((B, H, G, D), torch.bfloat16), n["o"].names)}, "MTF_ERR_SIZE_MISMATCH")
    for x in (float("nan"), float("inf"), -3e38):
        refused("decode", {"scale": x})
    for name in ("q", "o"):
        refused("decode", lambda n: {name: mtf.Named(n[name].dims, n[name].dtype, n[name].ptr + 8, n[name].owner)}, "MTF_ERR_UNSUPPORTED")
    refused("decode", lambda n: {"o": mtf.Named(n["o"].dims, n["o"].dtype, n["q"].ptr, n["q"].owner)})
    refused("decode", lambda n: {"o": mtf.Named(n["o"].dims, n["o"].dtype, n["v"].ptr, n["v"].owner)})
    # a workspace is asked for where an item may be cut
    n = things()
    n["table"] = ints(B, 1 << 14)
    cache = mtf.Cache(n["k"], n["v"], n["table"])
    need = mtf.mtf_attention_decode_workspace_bytes(n["layout"], n["q"], cache)
    assert need > 0
    refused("decode", {"table": n["table"]}, "MTF_ERR_WORKSPACE_TOO_SMALL")
    refused("decode", {"table": n["table"], "workspace": room(need - 1)}, "MTF_ERR_WORKSPACE_TOO_SMALL")
    refused("decode", {"table": n["table"], "workspace": room(need + 16)[8:]}, "MTF_ERR_UNSUPPORTED")
    both = room(need)
    refused("decode", {"table": n["table"], "workspace": both, "o": mtf.Named(n["o"].dims, "bf16", both.data_ptr(), both)})
    assert mtf.mtf_attention_decode_workspace_bytes(n["layout"], n["q"], mtf.Cache(n["k"], n["v"], ints(B, 8))) == 0
    # descriptors without data are enough to ask
    q = mtf.desc(n["q"].dims, "bf16")
    assert mtf.mtf_attention_decode_workspace_bytes(n["layout"], q, cache) == need


def test_selection():
    refused("select", lambda n: {"logits": as_type(n["logits"], torch.float8_e4m3fn)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"scores": as_type(n["scores"], torch.bfloat16)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"new_scores": as_type(n["new_scores"], torch.bfloat16)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"scores": renamed(n["scores"], "beam", "b")}, "MTF_ERR_SIZE_MISMATCH")
    refused("select", lambda n: {"new_scores": mtf.named(tensor((SENT + 1, OUT), torch.float32), n["new_scores"].names), "parents": ints(SENT + 1, OUT), "tokens": ints(SENT + 1, OUT),
                                 "new_finished": ints(SENT + 1, OUT)}, "MTF_ERR_SIZE_MISMATCH")
    for e in (-1, V):
        refused("select", {"end_id": e})
    for slots in (65, 61):                                     # beyond the kernels', beyond the words of all beams
        refused("select", lambda n: {"new_scores": mtf.named(tensor((SENT, slots), torch.float32), n["new_scores"].names), "parents": ints(SENT, slots), "tokens": ints(SENT, slots),
                                     "new_finished": ints(SENT, slots)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"logits": mtf.named(tensor((1, 65, V), torch.float32), n["logits"].names), "scores": mtf.named(tensor((1, 65), torch.float32), n["scores"].names),
                                 "finished": ints(1, 65)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"logits": mtf.Named(n["logits"].dims, "f32", n["logits"].ptr + 4, n["logits"].owner)}, "MTF_ERR_UNSUPPORTED")
    refused("select", lambda n: {"new_scores": mtf.Named(n["new_scores"].dims, "f32", n["logits"].ptr, n["logits"].owner)})
    refused("select", lambda n: {"tokens": n["parents"]})
    n = things()
    need = mtf.mtf_beam_select_workspace_bytes(n["layout"], n["logits"], OUT)
    refused("select", {"beam_ws": None}, "MTF_ERR_WORKSPACE_TOO_SMALL")
    refused("select", {"beam_ws": room(need - 1)}, "MTF_ERR_WORKSPACE_TOO_SMALL")
    refused("select", {"beam_ws": room(need + 16)[4:]}, "MTF_ERR_UNSUPPORTED")
    for dim in ("vocab", "beam"):
        x = {"logits": mtf.named(tensor((SENT, 2, V), torch.float32), n["logits"].names), "scores": mtf.named(tensor((SENT, 2), torch.float32), n["scores"].names), "finished": ints(SENT, 2)}
        refused("select", {"layout": ranks([(dim, "r")]), **x}, "MTF_ERR_UNSUPPORTED")
    for slots in (0, 65):
        with pytest.raises(mtf.MtfError):
            mtf.mtf_beam_select_workspace_bytes(n["layout"], n["logits"], slots)


def test_reorderings():
    refused("reorder", lambda n: {"out": as_type(n["out"], torch.bfloat16)})
    refused("reorder", {"beam": "y"}, "MTF_ERR_UNKNOWN_DIM")
    refused("reorder", lambda n: {"states": renamed(n["states"], "x", "y")}, "MTF_ERR_SIZE_MISMATCH")
    refused("reorder", lambda n: {"states": mtf.named(tensor((SENT, BEAMS, 6), torch.float32), n["states"].names)}, "MTF_ERR_SIZE_MISMATCH")
    refused("reorder", lambda n: {"out": mtf.Named(n["out"].dims, "f32", n["states"].ptr, n["states"].owner)})
    refused("reorder", lambda n: {"states": mtf.Named(n["states"].dims, "f32", n["states"].ptr + 2, n["states"].owner)})
    refused("reorder", {"layout": ranks([("beam", "r")]), "states": mtf.named(tensor((SENT, 2, 5), torch.float32), ["sentence", "beam", "x"])}, "MTF_ERR_UNSUPPORTED")
    refused("cache_reorder", lambda n: {"new_table": n["beam_table"], "parents": ints(SENT, BEAMS), "fresh": ints(SENT, BEAMS), "new_lengths": ints(SENT, BEAMS)})
    refused("cache_reorder", lambda n: {"new_lengths": n["fresh"]})
    refused("cache_reorder", {"parents": ints(SENT + 1, OUT)}, "MTF_ERR_SIZE_MISMATCH")


def sized(t, **sizes):
    """The same memory with other sizes of some dims: refused before anything looks at it."""
    return mtf.Named([(n, sizes.get(n, s)) for n, s in t.dims], {0: "f32", 1: "bf16", 2: "e4m3"}[t.dtype], t.ptr, t.owner)


@pytest.mark.parametrize("op", PAGED)
def test_caches_beyond_the_kernels_numbers(op):
    # rows of a page, rows of a pool, and products that wrap around 64 bits
    for sizes in (dict(slot=(1 << 23) + 1), dict(page=1 << 28), dict(page=1 << 40, slot=1 << 30), dict(page=1 << 62)):
        refused(op, lambda n: {name: sized(n[name], **sizes) for name in ("k", "v")}, "MTF_ERR_UNSUPPORTED")
    for sizes in (dict(length=1 << 31), dict(length=1 << 62)):
        if op in ("write", "read"):
            refused(op, lambda n: {name: sized(n[name], **sizes) for name in ("kk", "vv")}, "MTF_ERR_UNSUPPORTED")
    if op == "decode":
        for group in (4097, 1 << 61):
            refused(op, lambda n: {name: sized(n[name], group=group) for name in ("q", "o")}, "MTF_ERR_UNSUPPORTED")


def test_selections_and_states_beyond_the_kernels_numbers():
    for vocab in (1 << 30, 1 << 62):                           # (of three beams)
        refused("select", lambda n: {"logits": sized(n["logits"], vocab=vocab)}, "MTF_ERR_UNSUPPORTED")
        n = things()
        with pytest.raises(mtf.MtfError) as e:
            mtf.mtf_beam_select_workspace_bytes(n["layout"], sized(n["logits"], vocab=vocab), 4)
        assert e.value.code == "MTF_ERR_UNSUPPORTED"
    refused("reorder", lambda n: {name: sized(n[name], x=1 << 62) for name in ("states", "out")}, "MTF_ERR_UNSUPPORTED")


def test_other_calls_refuse_8_bits():
    """A type that only caches and their reordering have: what took f32 and bf16 does not take it for one of them."""
    x = mtf.named(tensor((4, 16), torch.float8_e4m3fn), ["a", "b"])
    y = mtf.named(tensor((16, 4), torch.float8_e4m3fn), ["b", "a"])
    f = mtf.named(tensor((4, 16), torch.float32), ["a", "b"])
    ids, l = ints(4), lay()
    calls = [lambda: mtf.mtf_transpose(l, x, y), lambda: mtf.mtf_slice_scatter(l, tensor((4, 16), torch.float8_e4m3fn), 0, x),
             lambda: mtf.mtf_slice_gather(l, x, 0, tensor((4, 16), torch.float8_e4m3fn)), lambda: mtf.mtf_embedding_forward(l, ids, x, x),
             lambda: mtf.mtf_embedding_backward(l, ids, x, f), lambda: mtf.mtf_reduce_sum(l, x, mtf.named(tensor((4,), torch.float32), ["a"])),
             lambda: mtf.mtf_einsum_plan(l, [x, y], mtf.named(tensor((4, 4), torch.float32), ["a", "c"])), lambda: mtf.mtf_softmax_forward(l, x, 0, x),
             lambda: mtf.mtf_update(l, x, f, None, None, 0.1, 0.0, 0.0)]
    n0 = mtf.mtf_launch_count()
    for c in calls:
        with pytest.raises((mtf.MtfError, TypeError)):
            c()
    assert mtf.mtf_launch_count() == n0
