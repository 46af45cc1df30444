"""The losses on stored logits beyond cross-entropy as timed cases: distillation from a teacher's top logits, the clipped policy loss with a KL term and
the preference loss on pairs of sequences, each on logits [batch, length, vocab] (the preference loss: [2, batch, length, vocab])."""
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TOK = ["batch", "length"]


def _case(name, op, call, dtype, batch, length, vocab, prompt, **more):
    c = {"op": op, "call": call, "dtype": dtype, "batch": batch, "length": length, "vocab": vocab, "prompt": prompt, **more}
    return {"name": name, **c} if name else c


def policy(name, call, dtype, batch, length, vocab, prompt=0.2, kl_weight=0.05, clip_high=0.25):
    return _case(name, "policy", call, dtype, batch, length, vocab, prompt, clip_low=0.2, clip_high=clip_high, kl_weight=kl_weight)


def distill(name, call, dtype, batch, length, vocab, teacher, temperature, soft=0.75, hard=0.25, prompt=0.0):
    return _case(name, "distill", call, dtype, batch, length, vocab, prompt, teacher=teacher, temperature=temperature, soft=soft, hard=hard)


def preference(name, call, dtype, batch, length, vocab, kind="sigmoid", beta=0.1, smoothing=0.0, prompt=0.3):
    return _case(name, "preference", call, dtype, batch, length, vocab, prompt, kind=kind, beta=beta, smoothing=smoothing)


def listed():
    return [
        # the last tokens of a few short answers: one optimizer step of a policy on a handful of rows; all latency
        policy("policy step few", "step", "bf16", 2, 8, 32768, prompt=0.0),
        # eight answers of up to 1024 tokens behind their prompts, loss and gradient in one call: a step of policy training at the benchmark's vocabulary
        policy("policy step", "step", "bf16", 8, 1024, 32768),
        # a multilingual vocabulary in 16 bits, one row longer than an SM's shared memory
        policy("policy step wide", "step", "bf16", 4, 512, 131072, kl_weight=0.0),
        # a vocabulary that no vector width divides, logits in 32 bits, the two directions called one after the other as an autograd engine does
        policy("policy f32 ragged", "both", "f32", 3, 259, 50001),
        # a few positions of a student against sixteen words of its teacher
        distill("distill step few", "step", "bf16", 1, 24, 32768, 16, 2.0),
        # the benchmark's 32 sequences of 256 tokens, a teacher's 64 best words and the label, softened by 2
        distill("distill step", "step", "bf16", 32, 256, 32768, 64, 2.0),
        # the teacher alone at its own temperature, 32 bits, odd sizes, one direction after the other
        distill("distill f32 ragged", "both", "f32", 2, 411, 32001, 100, 1.0, soft=1.0, hard=0.0),
        # evaluation of a student on a wide vocabulary: the loss alone
        distill("distill forward wide", "forward", "bf16", 4, 500, 131072, 32, 1.5, prompt=0.1),
        # one pair of short answers
        preference("preference few", "both", "bf16", 1, 20, 32768),
        # four pairs of answers of up to 1024 tokens behind their prompts
        preference("preference", "both", "bf16", 4, 1024, 32768),
        # pairs of odd length over an odd vocabulary, squared form
        preference("preference ragged", "both", "bf16", 3, 333, 50001, kind="squared"),
        # the loss of held-out pairs, smoothed labels, 32 bits
        preference("preference forward f32", "forward", "f32", 5, 200, 32768, smoothing=0.1),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(low * (high / low) ** rng.random()))))


def draw(rng):
    op, dtype = rng.choice(["policy", "distill", "preference"]), rng.choice(["bf16", "bf16", "f32"])
    call = rng.choice(["step", "step", "both", "forward"]) if op != "preference" else rng.choice(["both", "both", "forward"])
    vocab = _log(rng, 2000, 131072)
    if rng.random() < 0.5:
        vocab = max(2048, vocab // 256 * 256)
    batch, length = _log(rng, 1, 16), _log(rng, 8, 1024)
    while batch * length * vocab * (2 if op == "preference" else 1) * (4 if dtype == "f32" else 2) > 8192 * 32768 * 2:
        length = max(1, length // 2)
        batch = max(1, batch - 1)
    prompt = rng.choice([0.0, 0.1, 0.2, 0.4])
    if op == "policy":
        return policy("", call, dtype, batch, length, vocab, prompt, rng.choice([0.0, 0.02, 0.05]), rng.choice([0.2, 0.28]))
    if op == "distill":
        hard = rng.choice([0.0, 0.1, 0.5])
        return distill("", call, dtype, batch, length, vocab, _log(rng, 4, 256), rng.choice([1.0, 1.5, 2.0, 4.0]), 1.0 - hard, hard, prompt)
    kind = rng.choice(["sigmoid", "sigmoid", "hinge", "squared"])
    return preference("", call, dtype, batch, length, vocab, kind, rng.choice([0.05, 0.1, 0.3]), rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0, prompt)


def _spans(case):
    """Per sequence the positions [first, end) that the loss counts: behind a prompt, in front of the padding of a ragged batch.  Fixed by the case's sizes."""
    L, n = case["length"], case["batch"] * (2 if case["op"] == "preference" else 1)
    # (the two answers of a pair lie behind the same prompt)
    starts = [int(case["prompt"] * L * (1 + 37 * (i % case["batch"]) % 10 / 10)) for i in range(n)]
    return [(s, max(s + 1, L - (53 * i % 16) * L // 100)) for i, s in enumerate(starts)]


def _rows(case):
    return case["batch"] * case["length"] * (2 if case["op"] == "preference" else 1)


class _State:
    pass


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = _State()
    s.case, V, T, dtype = case, case["vocab"], _rows(case), TYPES[case["dtype"]]
    shape = ([2] if case["op"] == "preference" else []) + [case["batch"], case["length"]]
    # a head's logits: a spread of 2, and the word at hand often well above the rest
    z = normal(T, V).mul_(2.0)
    targets = (uniform(T) * V).long().clamp_(max=V - 1)
    z.scatter_add_(1, targets[:, None], 4.0 + 4.0 * normal(T)[:, None])
    s.logits = z.to(dtype).view(*shape, V)
    del z
    s.targets = targets.to(torch.int32).view(shape)
    spans = torch.tensor(_spans(case), device="cuda").view(*shape[:-1], 2)
    at = torch.arange(case["length"], device="cuda")
    s.weight = ((at >= spans[..., :1]) & (at < spans[..., 1:])).float()
    picked = _logp(s.logits.view(T, V), targets).view(shape) if case["op"] != "distill" else None
    if case["op"] == "policy":
        s.weight = s.weight / s.weight.sum(-1, keepdim=True) / case["batch"]
        # the policy has moved a little since the answers were sampled, and more since the reference
        s.old_logp = (picked + 0.2 * normal(*shape)).float()
        s.ref_logp = (picked + 0.4 * normal(*shape)).float() if case["kl_weight"] else None
        s.advantage = normal(case["batch"], 1).expand(shape).contiguous()
    elif case["op"] == "distill":
        s.weight = s.weight / s.weight.sum()
        # the teacher's best words: near the student's own, with some of the slots empty where it gave fewer
        noisy = s.logits.view(T, V).float() + normal(T, V)
        top = noisy.topk(case["teacher"], -1)
        s.teacher_logits = top.values.add_(normal(T, case["teacher"])).to(dtype).view(*shape, -1)
        kept = (case["teacher"] * (0.5 + 0.5 * uniform(T, 1))).long().clamp_(min=1)
        s.teacher_ids = torch.where(torch.arange(case["teacher"], device="cuda") < kept, top.indices, -1).to(torch.int32).view(*shape, -1)
        del noisy, top
    else:
        s.ref_logp = ((picked + 0.2 * normal(*shape)) * s.weight).sum(-1).float()
    s.dloss = (1.0 + 0.1 * normal(*shape[-2:] if case["op"] != "preference" else (case["batch"],))).contiguous()
    if own:
        _own_state(s)
    torch.cuda.empty_cache()
    return s


def _logp(z, targets):
    z = z.float()
    m = z.amax(-1, keepdim=True)
    return z.gather(1, targets[:, None])[:, 0].double() - m[:, 0].double() - torch.exp(z - m).sum(-1, dtype=torch.float64).log()


def _own_state(s):
    """The library's handles, descriptors and the tensors it writes, as a program keeps them from step to step."""
    import paper_1811_02084_b200 as mtf
    s.mtf, op = mtf, s.case["op"]
    s.layout = mtf.mtf_layout(mtf.mtf_mesh_create([("all", 1)]), [])
    tok = (["branch"] if op == "preference" else []) + TOK
    shape = list(s.targets.shape)

    def put(name, names, t):
        setattr(s, "n_" + name, mtf.named(t, names))
        return t

    def room(name, names, shape):
        setattr(s, name, put(name, names, torch.empty(shape, dtype=torch.float32, device="cuda")))

    put("logits", tok + ["vocab"], s.logits)
    put("weight", tok, s.weight)
    room("loss", TOK if op != "preference" else ["batch"], shape if op != "preference" else shape[1:2])
    put("dloss", TOK if op != "preference" else ["batch"], s.dloss)
    if s.case["call"] != "forward":
        s.dlogits = put("dlogits", tok + ["vocab"], torch.empty_like(s.logits))
    if op == "distill":
        put("teacher_logits", tok + ["teacher"], s.teacher_logits)
        room("stats", tok + ["stat"], shape + [2])
        s.hard_targets = s.targets if s.case["hard"] else None
        return
    s.n_ref_logp = None
    room("logp", tok, shape)
    room("lse", tok, shape)
    if op == "policy":
        put("old_logp", tok, s.old_logp)
        put("advantage", tok, s.advantage)
        if s.ref_logp is not None:
            put("ref_logp", tok, s.ref_logp)
        room("dlogp", tok, shape)
        return
    put("ref_logp", ["branch", "batch"], s.ref_logp)
    room("seq_logp", ["branch", "batch"], shape[:2])
    room("dseq", ["branch", "batch"], shape[:2])


def run(s):
    call = _own if own else _plain
    return call(s, s.case)


def _own(s, c):
    mtf, lay, call = s.mtf, s.layout, c["call"]
    if c["op"] == "policy":
        if call == "step":
            mtf.mtf_policy_step(lay, s.n_logits, s.targets, s.n_old_logp, s.n_ref_logp, s.n_advantage, s.n_weight, c["clip_low"], c["clip_high"], c["kl_weight"],
                                s.n_logp, s.n_loss, s.n_dlogits)
            return {"loss": s.loss, "logp": s.logp, "dlogits": s.dlogits}
        mtf.mtf_policy_forward(lay, s.n_logits, s.targets, s.n_old_logp, s.n_ref_logp, s.n_advantage, s.n_weight, c["clip_low"], c["clip_high"], c["kl_weight"],
                               s.n_lse, s.n_logp, s.n_dlogp, s.n_loss)
        if call == "forward":
            return {"loss": s.loss, "lse": s.lse, "logp": s.logp, "dlogp": s.dlogp}
        mtf.mtf_policy_backward(lay, s.n_logits, s.targets, s.n_lse, s.n_dlogp, s.n_dloss, s.n_dlogits)
        return {"loss": s.loss, "lse": s.lse, "logp": s.logp, "dlogp": s.dlogp, "dlogits": s.dlogits}
    if c["op"] == "distill":
        teacher = (s.teacher_ids, s.n_teacher_logits, s.hard_targets, s.n_weight, c["temperature"], c["soft"], c["hard"])
        if call == "step":
            mtf.mtf_distill_step(lay, s.n_logits, *teacher, s.n_loss, s.n_dlogits)
            return {"loss": s.loss, "dlogits": s.dlogits}
        mtf.mtf_distill_forward(lay, s.n_logits, *teacher, s.n_stats, s.n_loss)
        if call == "forward":
            return {"loss": s.loss, "stats": s.stats}
        mtf.mtf_distill_backward(lay, s.n_logits, *teacher, s.n_stats, s.n_dloss, s.n_dlogits)
        return {"loss": s.loss, "stats": s.stats, "dlogits": s.dlogits}
    mtf.mtf_preference_forward(lay, s.n_logits, s.targets, s.n_weight, s.n_ref_logp, c["kind"], c["beta"], c["smoothing"], s.n_lse, s.n_logp, s.n_seq_logp, s.n_dseq,
                               s.n_loss)
    if call == "forward":
        return {"loss": s.loss, "lse": s.lse, "logp": s.logp, "seq_logp": s.seq_logp, "dseq": s.dseq}
    mtf.mtf_preference_backward(lay, s.n_logits, s.targets, s.n_weight, s.n_lse, s.n_dseq, s.n_dloss, s.n_dlogits)
    return {"loss": s.loss, "lse": s.lse, "logp": s.logp, "seq_logp": s.seq_logp, "dseq": s.dseq, "dlogits": s.dlogits}


def _rows_lse(z, scale=1.0):
    """log sum exp of each row of scale * z, its sum in 64 bits: the scalars of a row are differences of numbers near each other."""
    m = z.amax(-1, keepdim=True)
    return m[..., 0].double() * scale + ((z - m) * scale).exp().sum(-1, dtype=torch.float64).log()


def _plain(s, c):
    z, w, live = s.logits.float(), s.weight, s.weight != 0
    lse = _rows_lse(z)
    targets = s.targets.long()[..., None]
    picked = z.gather(-1, targets)[..., 0].double()
    logp = torch.where(live, picked - lse, 0.0)
    if c["op"] == "distill":
        return _plain_distill(s, c, z, w, live, lse, targets, logp)
    if c["op"] == "policy":
        ratio = (logp - s.old_logp).exp()
        plain, clipped = ratio * s.advantage, ratio.clamp(1 - c["clip_low"], 1 + c["clip_high"]) * s.advantage
        loss = -torch.minimum(plain, clipped)
        dlogp = torch.where(plain <= clipped, -plain, 0.0)
        if c["kl_weight"]:
            e = s.ref_logp - logp
            loss = loss + c["kl_weight"] * (torch.expm1(e) - e)
            dlogp = dlogp - c["kl_weight"] * torch.expm1(e)
        out = {"loss": (w * loss).float(), "logp": logp.float()}
        if c["call"] != "step":
            out.update(lse=torch.where(live, lse, 0.0).float(), dlogp=(w * dlogp).float())
        rows = w * dlogp * (1.0 if c["call"] == "step" else s.dloss)
    else:
        seq = (w * logp).sum(-1)
        margin = (seq[0] - s.ref_logp[0]) - (seq[1] - s.ref_logp[1])
        h, eps = c["beta"] * margin, c["smoothing"]
        if c["kind"] == "sigmoid":
            # log(1 + exp(x)) = max(x, 0) + log1p(exp(-|x|))
            tail = torch.log1p((-h.abs()).exp())
            loss = (1 - eps) * ((-h).clamp(min=0) + tail) + eps * (h.clamp(min=0) + tail)
            d = c["beta"] * (eps - 1 / (1 + h.exp()))
        elif c["kind"] == "hinge":
            loss, d = (1 - h).clamp(min=0), torch.where(h < 1, -c["beta"], 0.0).double()
        else:
            loss, d = (margin - 0.5 / c["beta"]).square(), 2 * (margin - 0.5 / c["beta"])
        dseq = torch.stack([d, -d])
        out = {"loss": loss.float(), "lse": torch.where(live, lse, 0.0).float(), "logp": logp.float(), "seq_logp": seq.float(), "dseq": dseq.float()}
        rows = w * (dseq * s.dloss)[..., None]
    if c["call"] == "forward":
        return out
    p = (z - lse.float()[..., None]).exp_()
    hit = torch.arange(c["vocab"], device=z.device) == targets
    out["dlogits"] = torch.where(live[..., None], (hit.float() - p) * rows.float()[..., None], 0.0).to(s.logits.dtype)
    return out


def _plain_distill(s, c, z, w, live, lse, targets, logp):
    tau = c["temperature"]
    used, ids = s.teacher_ids >= 0, s.teacher_ids.long().clamp(min=0)
    t = torch.where(used, s.teacher_logits.double() / tau, -torch.inf)
    t = t - t.amax(-1, keepdim=True)
    logq = t - t.exp().sum(-1, keepdim=True).log()
    q = logq.exp()
    lse_tau = _rows_lse(z, 1 / tau)
    logp_tau = z.gather(-1, ids).double() / tau - lse_tau[..., None]
    soft = torch.where(used, q * (logq - logp_tau), 0.0).sum(-1)
    loss = w * (c["soft"] * tau * tau * soft - c["hard"] * logp)
    out = {"loss": torch.where(live, loss, 0.0).float()}
    if c["call"] != "step":
        out["stats"] = torch.where(live[..., None], torch.stack([lse_tau, lse if c["hard"] else torch.zeros_like(lse)], -1), 0.0).float()
    if c["call"] == "forward":
        return out
    d = (z / tau - lse_tau.float()[..., None]).exp_()
    d.scatter_add_(-1, ids, -q.float())
    d *= c["soft"] * tau
    if c["hard"]:
        d += c["hard"] * (z - lse.float()[..., None]).exp_()
        d.scatter_add_(-1, targets, torch.full_like(targets, -c["hard"], dtype=torch.float32))
    rows = w * (1.0 if c["call"] == "step" else s.dloss)
    out["dlogits"] = torch.where(live[..., None], d * rows[..., None], 0.0).to(s.logits.dtype)
    return out


def work(case):
    T, V, e = _rows(case), case["vocab"], 4 if case["dtype"] == "f32" else 2
    n = sum(end - first for first, end in _spans(case))
    size = n * V * e + (0 if case["call"] == "forward" else T * V * e) + 4 * T * 6
    if case["op"] == "distill":
        size += n * case["teacher"] * (4 + e)
    temperatures = 2 if case["op"] == "distill" and case["hard"] and case["temperature"] != 1.0 else 1
    return {"bytes": size, "flops": n * V * temperatures * (4.0 if case["call"] == "forward" else 8.0)}


def exact(case, seed):
    """What `run` returns, from the losses' definitions in 64 bits; the gradients by differentiating the losses."""
    global own
    asked, own = own, False
    s, c = prepare(case, seed), case
    own = asked
    z = s.logits.double().requires_grad_(c["call"] != "forward")
    w, live = s.weight.double(), s.weight != 0
    logp_all = torch.log_softmax(z, -1)
    token = torch.where(live, logp_all.gather(-1, s.targets.long()[..., None])[..., 0], 0.0)
    r = {} if c["call"] == "step" else {"lse": torch.where(live, torch.logsumexp(z, -1), 0.0)}
    if c["op"] == "distill":
        tau = c["temperature"]
        used = s.teacher_ids >= 0
        teacher = torch.log_softmax(torch.where(used, s.teacher_logits.double() / tau, -torch.inf), -1)
        student = torch.log_softmax(z / tau, -1).gather(-1, torch.where(used, s.teacher_ids, 0).long())
        kl = torch.where(used, teacher.exp() * (torch.where(used, teacher, 0.0) - student), 0.0).sum(-1)
        loss = torch.where(live, w * (c["soft"] * tau ** 2 * kl - c["hard"] * token), 0.0)
        r["loss"] = loss
        if c["call"] != "step":
            # (the second sum belongs to the label's part alone)
            r["stats"] = torch.stack([torch.where(live, torch.logsumexp(z / tau, -1), 0.0), r.pop("lse") * (c["hard"] != 0)], -1)
    elif c["op"] == "policy":
        x = token.detach().requires_grad_()
        ratio = torch.exp(x - s.old_logp.double())
        a = s.advantage.double()
        low, high = 1 - c["clip_low"], 1 + c["clip_high"]
        # where the clipped side is the smaller one the loss does not move with the ratio
        outside = ((a > 0) & (ratio > high)) | ((a < 0) & (ratio < low))
        each = -a * torch.where(outside, torch.where(a > 0, high, low), ratio)
        if c["kl_weight"]:
            e = s.ref_logp.double() - x
            each = each + c["kl_weight"] * (torch.exp(e) - 1 - e)
        each = w * each
        dlogp, = torch.autograd.grad(each.sum(), x)
        r["loss"], r["logp"] = each, token
        if c["call"] != "step":
            r["dlogp"] = dlogp
        loss = dlogp * token
    else:
        seq = (w * token).sum(-1)
        x = seq.detach().requires_grad_()
        ref = s.ref_logp.double()
        margin = x[0] - x[1] - (ref[0] - ref[1])
        if c["kind"] == "sigmoid":
            eps = c["smoothing"]
            each = -(1 - eps) * torch.nn.functional.logsigmoid(c["beta"] * margin) - eps * torch.nn.functional.logsigmoid(-c["beta"] * margin)
        elif c["kind"] == "hinge":
            each = torch.relu(1 - c["beta"] * margin)
        else:
            each = (margin - 1 / (2 * c["beta"])) ** 2
        dseq, = torch.autograd.grad(each.sum(), x)
        r["loss"], r["logp"], r["seq_logp"], r["dseq"] = each, token, seq, dseq
        loss = dseq * seq
    if c["call"] != "forward":
        scale = s.dloss.double() if c["call"] == "both" else torch.ones((), dtype=torch.float64, device=z.device)
        r["dlogits"], = torch.autograd.grad((loss * scale).sum(), z)
    return {k: v.detach() for k, v in r.items()}
