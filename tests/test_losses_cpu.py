"""The losses on stored logits refuse what they do not take, before anything is launched (no GPU: tensors in host memory)."""
import pytest
import torch

import paper_1811_02084_b200 as mtf

B, L, V, K = 2, 3, 24, 4
TOK = ["batch", "length"]


def lay(mesh=(("all", 1),), rules=()):
    return mtf.mtf_layout(mtf.mtf_mesh_create(list(mesh)), list(rules))


def tensors(op="policy", dtype=torch.bfloat16):
    tok, lead = (["branch"] + TOK, (2, B, L)) if op == "preference" else (TOK, (B, L))
    n = {"logits": mtf.named(torch.zeros(*lead, V, dtype=dtype), tok + ["vocab"]), "dlogits": mtf.named(torch.zeros(*lead, V, dtype=dtype), tok + ["vocab"]),
         "targets": torch.zeros(lead, dtype=torch.int32)}
    for k in ("old", "ref", "adv", "weight", "lse", "logp", "dlogp", "loss", "dloss"):
        n[k] = mtf.named(torch.zeros(lead), tok)
    n["ids"], n["teacher"] = torch.zeros(*lead, K, dtype=torch.int32), mtf.named(torch.zeros(*lead, K), tok + ["slot"])
    n["stats"] = mtf.named(torch.zeros(*lead, 2), tok + ["stat"])
    if op == "preference":
        for k in ("ref", "seq", "dseq"):
            n[k] = mtf.named(torch.zeros(2, B), ["branch", "batch"])
        for k in ("loss", "dloss"):
            n[k] = mtf.named(torch.zeros(B), ["batch"])
    n["hp"] = {"policy": (0.2, 0.2, 0.1), "distill": (2.0, 1.0, 1.0), "preference": ("sigmoid", 0.1, 0.0)}[op]
    n["layout"] = lay()
    return n


def calls(op, n):
    l, hp = n["layout"], n["hp"]
    if op == "policy":
        return {"forward": lambda: mtf.mtf_policy_forward(l, n["logits"], n["targets"], n["old"], n["ref"], n["adv"], n["weight"], *hp, n["lse"], n["logp"], n["dlogp"], n["loss"]),
                "backward": lambda: mtf.mtf_policy_backward(l, n["logits"], n["targets"], n["lse"], n["dlogp"], n["dloss"], n["dlogits"]),
                "step": lambda: mtf.mtf_policy_step(l, n["logits"], n["targets"], n["old"], n["ref"], n["adv"], n["weight"], *hp, n["logp"], n["loss"], n["dlogits"])}
    if op == "distill":
        t = lambda: (n["ids"], n["teacher"], n["targets"], n["weight"], *hp)      # noqa: E731
        return {"forward": lambda: mtf.mtf_distill_forward(l, n["logits"], *t(), n["stats"], n["loss"]),
                "backward": lambda: mtf.mtf_distill_backward(l, n["logits"], *t(), n["stats"], n["dloss"], n["dlogits"]),
                "step": lambda: mtf.mtf_distill_step(l, n["logits"], *t(), n["loss"], n["dlogits"])}
    return {"forward": lambda: mtf.mtf_preference_forward(l, n["logits"], n["targets"], n["weight"], n["ref"], *hp, n["lse"], n["logp"], n["seq"], n["dseq"], n["loss"]),
            "backward": lambda: mtf.mtf_preference_backward(l, n["logits"], n["targets"], n["weight"], n["lse"], n["dseq"], n["dloss"], n["dlogits"])}


def refused(op, call, change, code="MTF_ERR_INVALID_ARG"):
    n = tensors(op)
    n.update(change(n) if callable(change) else change)
    n0 = mtf.mtf_launch_count()
    with pytest.raises(mtf.MtfError) as e:
        calls(op, n)[call]()
    assert e.value.code == code, e.value
    assert mtf.mtf_launch_count() == n0


ALL = [("policy", "forward"), ("policy", "backward"), ("policy", "step"), ("distill", "forward"), ("distill", "backward"), ("distill", "step"),
       ("preference", "forward"), ("preference", "backward")]
READS = {"policy": {"forward": ["logits", "old", "adv", "lse", "logp", "dlogp", "loss"], "backward": ["logits", "lse", "dlogp", "dlogits"],
                    "step": ["logits", "old", "adv", "logp", "loss", "dlogits"]},
         "distill": {"forward": ["logits", "teacher", "stats", "loss"], "backward": ["logits", "teacher", "stats", "dlogits"], "step": ["logits", "teacher", "loss", "dlogits"]},
         "preference": {"forward": ["logits", "ref", "lse", "logp", "seq", "dseq", "loss"], "backward": ["logits", "lse", "dseq", "dlogits"]}}
TOKENWISE = {"old", "adv", "lse", "logp", "dlogp", "weight", "dloss"}


@pytest.mark.parametrize("op,call", ALL)
def test_missing_tensors_types_and_sizes(op, call):
    for name in READS[op][call]:
        refused(op, call, {name: None})
        refused(op, call, lambda n: {name: mtf.Named(n[name].dims, n[name].dtype)})                          # a descriptor without data
        # other dims (a preference's logits want at least three of them)
        refused(op, call, lambda n: {name: mtf.named(torch.zeros(5, 7, dtype=n[name].owner.dtype), ["a", "b"])},
                "MTF_ERR_INVALID_ARG" if name == "logits" and call == "forward" and op == "preference" else "MTF_ERR_SIZE_MISMATCH")
        if name not in ("logits", "dlogits", "teacher"):
            refused(op, call, lambda n: {name: mtf.named(n[name].owner.bfloat16(), n[name].names)}, "MTF_ERR_UNSUPPORTED")
    refused(op, call, {"targets": None})
    if "dlogits" in READS[op][call]:
        refused(op, call, lambda n: {"dlogits": mtf.named(n["dlogits"].owner.float(), n["dlogits"].names)})
    # a permutation of the token dimensions has as many values and is another tensor
    n = tensors(op)
    for name in set(READS[op][call]) & TOKENWISE:
        t = n[name].owner.transpose(-1, -2).contiguous()
        if n[name].names[-2:] == TOK:
            refused(op, call, {name: mtf.named(t, n[name].names[:-2] + ["length", "batch"])}, "MTF_ERR_SIZE_MISMATCH")


@pytest.mark.parametrize("op,call", ALL)
def test_ids_of_another_number_or_type(op, call):
    for name in ["targets"] + (["ids"] if op == "distill" else []):
        refused(op, call, lambda n: {name: n[name][:1].contiguous()}, "MTF_ERR_SIZE_MISMATCH")
        refused(op, call, lambda n: {name: torch.cat([n[name], n[name]])}, "MTF_ERR_SIZE_MISMATCH")
        refused(op, call, lambda n: {name: n[name].long()})
        refused(op, call, lambda n: {name: n[name].transpose(0, 1)})


@pytest.mark.parametrize("op,call", ALL)
def test_alignment_and_overlap(op, call):
    for name in READS[op][call]:
        t = tensors(op)[name]
        raw = torch.zeros(t.owner.numel() * t.owner.element_size() + 64, dtype=torch.uint8)
        by = 2 if name in ("logits", "dlogits") else 1
        refused(op, call, {name: mtf.Named(t.dims, t.dtype, raw.data_ptr() + -raw.data_ptr() % 16 + by, raw)},
                "MTF_ERR_UNSUPPORTED" if name in ("logits", "dlogits") else "MTF_ERR_INVALID_ARG")
    if "dlogits" in READS[op][call]:
        # over the logits as a whole is allowed; over a part of them, or over another tensor, is not
        big = torch.zeros(4 * V * 2 * B * L, dtype=torch.bfloat16)
        n = tensors(op)
        refused(op, call, {"logits": mtf.Named(n["logits"].dims, "bf16", big.data_ptr(), big), "dlogits": mtf.Named(n["logits"].dims, "bf16", big.data_ptr() + 16, big)})
        other = next(k for k in READS[op][call] if k not in ("logits", "dlogits"))
        refused(op, call, {"dlogits": mtf.Named(n["logits"].dims, "bf16", big.data_ptr(), big), other: mtf.Named(n[other].dims, n[other].dtype, big.data_ptr() + 32, big)})
    if call == "forward":
        for k in READS[op][call]:
            if k in ("lse", "logp", "loss", "dlogp") and tensors(op)[k].dims == tensors(op)["weight"].dims:
                refused(op, call, lambda n: {"weight": mtf.Named(n["weight"].dims, "f32", n[k].ptr, n[k].owner)})


def test_parameters():
    nan, inf = float("nan"), float("inf")
    for hp in [(0.0, 1, 1), (-1.0, 1, 1), (nan, 1, 1), (inf, 1, 1), (1.0, -0.1, 1), (1.0, nan, 1), (1.0, inf, 1), (1.0, 1, -1), (1.0, 1, nan)]:
        for call in ("forward", "backward", "step"):
            refused("distill", call, {"hp": hp})
    refused("distill", "step", {"hp": (1e-5, 1, 1)}, "MTF_ERR_UNSUPPORTED")
    for hp in [(-0.1, 0.2, 0), (1.1, 0.2, 0), (nan, 0.2, 0), (0.2, -0.1, 0), (0.2, nan, 0), (0.2, 0.2, -1), (0.2, 0.2, inf), (0.2, 0.2, nan)]:
        for call in ("forward", "step"):
            refused("policy", call, {"hp": hp})
    refused("policy", "step", {"ref": None})                                        # kl_weight 0.1 needs it
    for hp in [(3, 0.1, 0.0), (-1, 0.1, 0.0), ("sigmoid", 0.0, 0.0), ("sigmoid", nan, 0.0), ("sigmoid", inf, 0.0), ("sigmoid", 0.1, 0.6), ("sigmoid", 0.1, -0.1),
               ("hinge", 0.1, 0.1), ("squared", 0.1, nan)]:
        refused("preference", "forward", {"hp": hp})
    slots = torch.zeros(B, L, 513)
    refused("distill", "step", {"teacher": mtf.named(slots, TOK + ["slot"]), "ids": torch.zeros(B, L, 513, dtype=torch.int32)}, "MTF_ERR_UNSUPPORTED")
    refused("distill", "forward", {"stats": mtf.named(torch.zeros(B, L, 3), TOK + ["stat"])}, "MTF_ERR_SIZE_MISMATCH")
    refused("preference", "forward", {"logits": mtf.named(torch.zeros(3, B, L, V), ["branch"] + TOK + ["vocab"])})


def test_ids_are_contiguous_int32():
    n = tensors("policy")
    for bad in (n["targets"].long(), torch.zeros(L, B, dtype=torch.int32).t()):
        with pytest.raises(mtf.MtfError):
            mtf.mtf_policy_backward(n["layout"], n["logits"], bad, n["lse"], n["dlogp"], None, n["dlogits"])


@pytest.mark.parametrize("op,call", ALL)
def test_layouts(op, call):
    # two dimensions of the logits on one mesh dimension
    refused(op, call, {"layout": lay([("all", 1)], [("vocab", "all"), ("length", "all")])}, "MTF_ERR_ILLEGAL_LAYOUT")
    refused(op, call, {"layout": lay([("all", 5)], [("vocab", "all")])}, "MTF_ERR_NOT_DIVISIBLE")
    # a dimension that is taken as a whole may not be split across ranks
    whole = ["vocab"] + {"policy": [], "distill": ["slot"], "preference": ["length", "branch"]}[op]
    for dim in whole:
        size = {"length": 3}.get(dim, 2)
        refused(op, call, {"layout": mtf.mtf_layout_bind_ranks(lay([("all", size)], [(dim, "all")]), "all", size, 0)}, "MTF_ERR_UNSUPPORTED")
