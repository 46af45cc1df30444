"""The number of ids that a loss call takes goes by what a descriptor is in that call: one tensor may be the logits of one call and the teacher's of another (two
students that teach each other).  No GPU: the library refuses the calls for a tensor that is missing, behind the check of the ids."""
import itertools

import pytest
import torch

import paper_1811_02084_b200 as mtf

B, L, V = 2, 3, 24
TOK = ["batch", "length"]


def tensors():
    return {"z": mtf.named(torch.zeros(B, L, V), TOK + ["vocab"]), "other": mtf.named(torch.zeros(B, L, V), TOK + ["vocab"]), "per_word": torch.zeros(B, L, V, dtype=torch.int32),
            "per_token": torch.zeros(B, L, dtype=torch.int32), "layout": mtf.mtf_layout(mtf.mtf_mesh_create([("all", 1)]), [])}


def code(f):
    """The error of a call that has no loss tensor: MTF_ERR_INVALID_ARG where the ids are in order."""
    n0 = mtf.mtf_launch_count()
    with pytest.raises(mtf.MtfError) as e:
        f()
    assert mtf.mtf_launch_count() == n0
    return e.value.code


def distill(t, logits, teacher, ids, targets):
    stats = mtf.named(torch.zeros(B, L, 2), TOK + ["stat"])
    return lambda: mtf.mtf_distill_forward(t["layout"], logits, ids, teacher, targets, None, 2.0, 0.5, 0.5, stats, None)


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))), ids=str)
def test_one_descriptor_as_logits_and_as_teacher(order):
    t = tensors()
    z, other, word, token = t["z"], t["other"], t["per_word"], t["per_token"]
    roles = [(z, other), (other, z), (z, z)]                    # z teaches, learns, and both
    for logits, teacher in (roles[i] for i in order):
        assert code(distill(t, logits, teacher, word, token)) == "MTF_ERR_INVALID_ARG"
        assert code(distill(t, logits, teacher, token, token)) == "MTF_ERR_SIZE_MISMATCH"      # too few: the kernel would read past their end
        assert code(distill(t, logits, teacher, word, word)) == "MTF_ERR_SIZE_MISMATCH"
        assert code(distill(t, logits, teacher, token, word)) == "MTF_ERR_SIZE_MISMATCH"


def test_a_descriptor_of_other_calls_as_teacher():
    """... as logits of the calls that take no list."""
    t = tensors()
    z, token = t["z"], t["per_token"]
    value = mtf.named(torch.zeros(B, L), TOK)
    policy = lambda: mtf.mtf_policy_backward(t["layout"], z, token, value, value, None, None)      # noqa: E731
    assert code(policy) == "MTF_ERR_INVALID_ARG"
    assert code(distill(t, t["other"], z, t["per_word"], token)) == "MTF_ERR_INVALID_ARG"
    assert code(distill(t, t["other"], z, token, token)) == "MTF_ERR_SIZE_MISMATCH"
    assert code(policy) == "MTF_ERR_INVALID_ARG"


@pytest.mark.parametrize("kind", ["other", "", None, 1.5, 3, -1, [0]], ids=str)
def test_a_kind_that_is_none_is_refused_as_other_arguments_are(kind):
    lay = tensors()["layout"]
    tok = ["branch"] + TOK
    z, value = mtf.named(torch.zeros(2, B, L, V), tok + ["vocab"]), [mtf.named(torch.zeros(2, B, L), tok) for _ in range(2)]
    pair = [mtf.named(torch.zeros(2, B), tok[:2]) for _ in range(3)]
    ids, loss = torch.zeros(2, B, L, dtype=torch.int32), mtf.named(torch.zeros(B), ["batch"])
    assert code(lambda: mtf.mtf_preference_forward(lay, z, ids, None, pair[0], kind, 0.1, 0.0, *value, *pair[1:], loss)) == "MTF_ERR_INVALID_ARG"
