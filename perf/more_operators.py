"""What the losses over a vocabulary's classes are measured on: the log-likelihood of a many-class logistic model, and what is learned
through it from preferences, from rewards and from a teacher.

The operators and what a user's program does with them:

``logp`` / ``logp_grad``   log-probability of every row's target under softmax(scale * logits), with the row's log-sum-exp, as a
                           program scores the answers of a policy, of its older self or of a reference; and the gradient of any
                           function of those log-probabilities back to the logits
``policy``                 the clipped policy loss of rewarded answers with a KL term against a reference, and its gradient
``pref``                   the logistic loss of preferred against rejected answers (paired log ratios), and its gradient
``distill``                the divergence from a teacher of whom the top logits are known, and its gradient

Each case is one pass through one of them.  ``own`` false: plain torch in 32 bits (64 for the few numbers of a row that are next to a
border or differences of large ones); true: the library's entry points.
"""
import math

import torch

own = False


def listed():
    return [
        # four sequences that are decoded together: the tokens that came out are scored
        {"name": "logp-step", "op": "logp", "T": 4, "V": 32000, "scale": 1.0, "live": 1.0, "dtype": "bfloat16", "ids": "int64"},
        # the answers of a rollout scored by a reference that gives fp32 logits, prompts left out
        {"name": "logp-rollout", "op": "logp", "T": 6000, "V": 100000, "scale": 1.0, "live": 0.8, "dtype": "float32", "ids": "int64"},
        # one short sequence of a loss that the user wrote, a vocabulary of odd size
        {"name": "logp-grad-ragged", "op": "logp_grad", "T": 509, "V": 32003, "scale": 1.0, "live": 0.7, "dtype": "bfloat16",
         "ids": "int64"},
        # a micro-batch of the same, every row counted
        {"name": "logp-grad-train", "op": "logp_grad", "T": 8192, "V": 65536, "scale": 1.0, "live": 1.0, "dtype": "bfloat16",
         "ids": "int32"},
        # a small model's policy step: few rows, few classes, temperature 0.8, no reference
        {"name": "policy-small", "op": "policy", "T": 64, "V": 1003, "scale": 1.25, "live": 1.0, "kl": 0.0, "norm": None,
         "dtype": "float32", "ids": "int64"},
        # one answer of a policy step, divided by the tokens of the whole batch
        {"name": "policy-micro", "op": "policy", "T": 1000, "V": 32000, "scale": 1.0, "live": 0.9, "kl": 0.05, "norm": 16000.0,
         "dtype": "bfloat16", "ids": "int64"},
        # a policy step over a large vocabulary, prompts and padding left out
        {"name": "policy-train", "op": "policy", "T": 8192, "V": 128000, "scale": 1.0, "live": 0.75, "kl": 0.02, "norm": None,
         "dtype": "bfloat16", "ids": "int64"},
        # a single pair of short answers
        {"name": "pref-pair", "op": "pref", "P": 1, "T": 301, "V": 32000, "live": 0.8, "average": False, "dtype": "bfloat16",
         "ids": "int64"},
        # a step over eight pairs of ragged answers
        {"name": "pref-train", "op": "pref", "P": 8, "T": 6101, "V": 100000, "live": 0.7, "average": False, "dtype": "bfloat16",
         "ids": "int64"},
        # a few positions of a teacher with eight logits each, an odd vocabulary
        {"name": "distill-few", "op": "distill", "T": 16, "V": 50021, "K": 8, "scale": 0.5, "part": False, "live": 1.0,
         "teacher": "float32", "dtype": "float32", "ids": "int32"},
        # a training step with 64 of the teacher's logits
        {"name": "distill-train", "op": "distill", "T": 4096, "V": 128000, "K": 64, "scale": 1.0, "part": False, "live": 1.0,
         "teacher": "bfloat16", "dtype": "bfloat16", "ids": "int32"},
        # fp32 logits, 256 of the teacher's with the mass that they have in its whole vocabulary, padding left out
        {"name": "distill-part", "op": "distill", "T": 2048, "V": 100000, "K": 256, "scale": 0.5, "part": True, "live": 0.9,
         "teacher": "float32", "dtype": "float32", "ids": "int64"},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "logp_grad", "policy", "pref", "distill"])
    dtype = rng.choice(["float32", "bfloat16"])
    V = _spread(rng, 500, 160000)
    V = V // 8 * 8 if rng.random() < 0.6 else V
    most = (4500 if op == "pref" else 7000) * 128000 // V
    T = _spread(rng, 1 if op == "logp" else 4, min(32768, most if dtype == "bfloat16" else most // 2))
    case = {"op": op, "T": T, "V": V, "live": rng.choice([1.0, 0.9, 0.7, 0.5]), "dtype": dtype, "ids": rng.choice(["int32", "int64"])}
    if op != "pref":
        case["scale"] = rng.choice([1.0, 1.0, 0.5, 1.25])
    if op == "policy":
        case.update(kl=rng.choice([0.0, 0.01, 0.1]), norm=rng.choice([None, None, 4096.0]))
    if op == "pref":
        case.update(P=max(1, min(T // 2, rng.choice([1, 2, 3, 5, 8, 16]))), average=rng.random() < 0.4)
    if op == "distill":
        case.update(K=_spread(rng, 1, 256), part=rng.random() < 0.4, teacher=rng.choice(["float32", "bfloat16"]))
    return case


def _rows(V):
    """Rows of a matrix of V columns that are worked on at a time where a whole copy in 64 bits would be too much."""
    return max(1, (1 << 26) // V)


def _lse(logits, scale):
    """Row-wise log-sum-exp of scale * logits in fp32, for the inputs that a user has from an earlier pass."""
    return torch.cat([torch.logsumexp(x.float() * scale, 1) for x in logits.split(_rows(logits.shape[1]))])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    c, dt, ids = dict(case), getattr(torch, case["dtype"]), getattr(torch, case["ids"])
    T, V, op = c["T"], c["V"], c["op"]
    scale = c.setdefault("scale", 1.0)
    logits = torch.empty(T, V, dtype=dt, device="cuda")
    for part in logits.split(_rows(V)):
        part.copy_(2.5 * randn(*part.shape))
    # what stands in a text mostly has one of the larger logits
    at = torch.arange(T, device="cuda")
    target = torch.randint(0, V, (T,), generator=gen, device="cuda")
    logits[at, target] += (7.0 + 4.0 * randn(T)).to(dt)
    c["logits"] = logits
    live = rand(T) < c["live"]
    live[T // 2] = True                             # (a batch in which nothing counts would be no step)
    if op != "distill":
        c["targets"] = torch.where(live, target, -100).to(ids)
    if op in ("logp_grad", "policy"):
        lse = _lse(logits, scale)
        logp = logits[at, target].float() * scale - lse
        if op == "logp_grad":
            c["lse"] = lse
            c["dlogp"] = randn(T) / T
        else:
            c["advantages"] = randn(T)
            c["old"] = torch.clamp(logp + 0.15 * randn(T), max=0.0)
            c["ref"] = torch.clamp(logp + 0.3 * randn(T), max=0.0) if c["kl"] > 0 else None
    elif op == "pref":
        P = c["P"]
        length = 0.2 + rand(2 * P)
        edges = torch.cumsum(length / length.sum(), 0)
        c["offsets"] = torch.cat([torch.zeros(1, device="cuda"), edges * T]).round().clamp(0, T).to(torch.int32)
        c["offsets"][-1] = T
        logp = torch.where(live, logits[at, target].double() - _lse(logits, 1.0), 0.0)
        o, size = c["offsets"].tolist(), live.double()
        sums = torch.stack([logp[a:z].sum() / (size[a:z].sum().clamp(min=1.0) if c["average"] else 1.0) for a, z in zip(o, o[1:])]).float()
        c["ref"] = sums + (0.1 if c["average"] else 5.0) * randn(2 * P)
        c["beta"], c["margin"], c["smoothing"] = (2.0, 0.5, 0.0) if c["average"] else (0.1, 0.0, 0.1)
    elif op == "distill":
        K = c["K"]
        # different classes for every row, the student's better ones more often than others
        step = 1 + torch.randint(0, max(1, (V - 1) // K), (T, 1), generator=gen, device="cuda")
        c["top"] = ((target[:, None] + step * torch.arange(K, device="cuda")) % V).to(ids)
        c["values"] = (4.0 * rand(T, K).sort(1, descending=True)[0] + 2.0 * randn(T, 1)).to(getattr(torch, c["teacher"]))
        c["teacher_lse"] = torch.logsumexp(c["values"].float() * scale, 1) + 0.3 * rand(T) if c["part"] else None
        c["weights"] = live.float() if c["live"] < 1.0 else None
    return c


def run(state):
    return (_own if own else _plain)[state["op"]](state)


# ---- the library's entry points ------------------------------------------------------------------------

def _own_logp(c):
    from paper_2308_10037_b200 import lr_logp
    return lr_logp(c["logits"], c["targets"], scale=c["scale"])


def _own_logp_grad(c):
    from paper_2308_10037_b200 import lr_logp_grad
    return lr_logp_grad(c["logits"], c["targets"], c["lse"], c["dlogp"], scale=c["scale"])


def _own_policy(c):
    from paper_2308_10037_b200 import lr_policy_loss
    return lr_policy_loss(c["logits"], c["targets"], c["advantages"], old_logp=c["old"], ref_logp=c["ref"], scale=c["scale"],
                          clip_low=0.2, clip_high=0.25, kl_coef=c["kl"], norm=c["norm"])


def _own_pref(c):
    from paper_2308_10037_b200 import lr_pref_loss
    return lr_pref_loss(c["logits"], c["targets"], c["offsets"], ref_logp=c["ref"], beta=c["beta"], margin=c["margin"],
                        smoothing=c["smoothing"], average=c["average"])


def _own_distill(c):
    from paper_2308_10037_b200 import lr_distill_loss
    return lr_distill_loss(c["logits"], c["top"], c["values"], teacher_lse=c["teacher_lse"], weights=c["weights"], scale=c["scale"],
                           factor=1.0 / c["scale"] ** 2)


_own = {"logp": _own_logp, "logp_grad": _own_logp_grad, "policy": _own_policy, "pref": _own_pref, "distill": _own_distill}


# ---- the same in plain torch ---------------------------------------------------------------------------

def _plain_rows(c):
    """(e = exp(x - largest x), largest x, sum of e) for the rows x of scale * logits."""
    x = c["logits"].float() * c["scale"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    return e, top[:, 0].double(), e.sum(1)


def _plain_targets(c):
    """(which rows count, their targets; 0 for the others)"""
    live = c["targets"] != -100
    return live, torch.where(live, c["targets"], 0).long()


def _plain_picked(c, target):
    return c["logits"].gather(1, target[:, None])[:, 0].double() * c["scale"]


def _plain_back(c, e, total, live, target, g):
    """dlogits of sum g * logp: scale * g * (1 at the target - softmax)."""
    g = torch.where(live, g * c["scale"], 0.0).float()
    d = e * (-g / total)[:, None]
    d = torch.where(live[:, None], d, 0.0)
    d.scatter_add_(1, target[:, None], g[:, None])
    return d.to(c["logits"].dtype)


def _plain_logp(c):
    e, top, total = _plain_rows(c)
    live, target = _plain_targets(c)
    lse = top + torch.log(total.double())
    logp = _plain_picked(c, target) - lse
    return torch.where(live, logp, 0.0).float(), torch.where(live, lse, 0.0).float()


def _plain_logp_grad(c):
    live, target = _plain_targets(c)
    x = c["logits"].float() * c["scale"]
    p = torch.exp(x - c["lse"][:, None])
    g = torch.where(live, c["dlogp"] * c["scale"], 0.0)
    d = torch.where(live[:, None], p * -g[:, None], 0.0)
    d.scatter_add_(1, target[:, None], g[:, None])
    return d.to(c["logits"].dtype)


def _plain_policy(c):
    e, top, total = _plain_rows(c)
    live, target = _plain_targets(c)
    logp = _plain_picked(c, target) - top - torch.log(total.double())
    adv = c["advantages"].double()
    ratio = torch.exp(logp - c["old"].double())
    low, high = 1.0 - float(torch.tensor(0.2)), 1.0 + float(torch.tensor(0.25))
    free, bound = ratio * adv, ratio.clamp(low, high) * adv
    clipped = free > bound
    gain = torch.where(clipped, bound, free)
    dlogp = torch.where(clipped, 0.0, -free)
    kl = torch.zeros_like(logp)
    if c["ref"] is not None:
        d = c["ref"].double() - logp
        kl = torch.exp(d) - d - 1.0
        dlogp = dlogp + c["kl"] * (1.0 - torch.exp(d))
    count = live.double()
    norm = c["norm"] if c["norm"] is not None else count.sum()
    parts = [(-gain * count).sum() / norm, (kl * count).sum() / norm, (clipped.double() * count).sum() / norm]
    stats = torch.stack([parts[0] + c["kl"] * parts[1], *parts]).float()
    return stats, torch.where(live, logp, 0.0).float(), _plain_back(c, e, total, live, target, dlogp / norm)


def _plain_pref(c):
    e, top, total = _plain_rows(c)
    live, target = _plain_targets(c)
    P, T = c["P"], c["T"]
    logp = torch.where(live, _plain_picked(c, target) - top - torch.log(total.double()), 0.0)
    owner = torch.searchsorted(c["offsets"].long(), torch.arange(T, device=logp.device), right=True) - 1
    score = torch.zeros(2 * P, dtype=torch.float64, device=logp.device).index_add_(0, owner, logp)
    size = torch.ones_like(score)
    if c["average"]:
        size = torch.zeros_like(score).index_add_(0, owner, live.double()).clamp(min=1.0)
        score = score / size
    ratio = score - c["ref"].double()
    h = c["beta"] * (ratio[:P] - ratio[P:]) - c["margin"]
    right, wrong = 1.0 / (1.0 + torch.exp(-h)), 1.0 / (1.0 + torch.exp(h))
    loss = (-(1.0 - c["smoothing"]) * torch.log(right) - c["smoothing"] * torch.log(wrong)).sum() / P
    dh = (c["smoothing"] * right - (1.0 - c["smoothing"]) * wrong) * c["beta"] / P
    g = (torch.cat([dh, -dh]) / size)[owner]
    return loss.float().view(1), h.float(), score.float(), _plain_back(c, e, total, live, target, g)


def _plain_distill(c):
    e, top, total = _plain_rows(c)
    ids, t = c["top"].long(), c["values"].double() * c["scale"]
    if c["teacher_lse"] is not None:
        logq = t - c["teacher_lse"].double()[:, None]
    else:
        largest = t.amax(1, keepdim=True)
        logq = t - largest - torch.log(torch.exp(t - largest).sum(1, keepdim=True))
    q = torch.exp(logq)
    logp = c["logits"].gather(1, ids).double() * c["scale"] - (top + torch.log(total.double()))[:, None]
    w = c["weights"] if c["weights"] is not None else torch.ones(c["T"], device=e.device)
    live = w != 0
    rows = torch.where(live, (q * (logq - logp)).sum(1), 0.0)
    factor = 1.0 / c["scale"] ** 2
    norm = w.double().sum()
    loss = factor * (rows * w).sum() / norm
    g = torch.where(live, w * (factor * c["scale"] / norm), 0.0)
    d = e * (g * q.sum(1) / total).float()[:, None]
    d.scatter_add_(1, ids, (-g[:, None] * q).float())
    return loss.float().view(1), rows.float(), d.to(c["logits"].dtype)


_plain = {"logp": _plain_logp, "logp_grad": _plain_logp_grad, "policy": _plain_policy, "pref": _plain_pref, "distill": _plain_distill}


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    c, T, V = case, case["T"], case["V"]
    b = 4 if c["dtype"] == "float32" else 2
    ib = 4 if c["ids"] == "int32" else 8
    seen = c["live"] * (T - 1) + 1                  # rows that count: the logits of the others are not needed
    per_row = {"logp": ib + 8, "logp_grad": ib + 8, "policy": ib + 16, "pref": ib, "distill": 4}[c["op"]]
    if c["op"] == "distill":
        per_row += c["K"] * (ib + (4 if c["teacher"] == "float32" else 2)) + 4
    written = 0 if c["op"] == "logp" else T * V * b
    return {"bytes": int(seen * V * b + written + T * per_row), "flops": int(seen * V * (4 if c["op"] == "logp" else 7))}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    c = prepare(case, seed)
    x, T, V, op, scale = c["logits"], c["T"], c["V"], c["op"], c["scale"]
    if op == "distill":
        used = torch.ones(T, dtype=torch.bool, device="cuda") if c["weights"] is None else c["weights"] > 0
        pick = c["top"].long()
    else:
        used = c["targets"] >= 0
        pick = c["targets"].long().clamp(min=0).unsqueeze(1)
    cuts = list(range(0, T, _rows(V)))
    lse = torch.empty(T, dtype=torch.float64, device="cuda")
    for a in cuts:
        lse[a:a + _rows(V)] = torch.logsumexp(x[a:a + _rows(V)].double().mul_(scale), dim=1)
    picked = (torch.gather(x, 1, pick).double() * scale - lse[:, None]).requires_grad_(op != "logp")
    if op == "logp":
        return picked[:, 0] * used, lse * used
    first = ()
    if op == "logp_grad":
        lse = c["lse"].double()
        value = (picked[:, 0] * c["dlogp"].double())[used].sum()
    elif op == "policy":
        lp, adv = picked[:, 0][used], c["advantages"].double()[used]
        ratio = (lp - c["old"].double()[used]).exp()
        hi, lo = 1 + torch.tensor(0.25).double().item(), 1 - torch.tensor(0.2).double().item()
        held = ((adv > 0) & (ratio > hi)) | ((adv < 0) & (ratio < lo))
        edge = torch.where(adv > 0, hi, lo)
        gain = adv * torch.where(held, edge, ratio)
        n = float(used.sum()) if c["norm"] is None else c["norm"]
        gap = c["ref"].double()[used] - lp if c["ref"] is not None else torch.zeros_like(lp)
        kl = torch.expm1(gap) - gap
        value = (c["kl"] * kl - gain).sum() / n
        stats = torch.stack([value, -gain.sum() / n, kl.sum() / n, held.sum().double() / n]).detach()
        first = (stats, (picked[:, 0] * used).detach())
    elif op == "pref":
        P, o = c["P"], c["offsets"].tolist()
        lp = picked[:, 0] * used
        s = torch.stack([lp[a:z].sum() for a, z in zip(o, o[1:])])
        if c["average"]:
            s = s / torch.stack([used[a:z].sum().clamp(min=1) for a, z in zip(o, o[1:])])
        better, worse = (s - c["ref"].double()).view(2, P)
        h = c["beta"] * (better - worse) - c["margin"]
        sm = c["smoothing"]
        value = ((1 - sm) * torch.nn.functional.softplus(-h, threshold=1e9) + sm * torch.nn.functional.softplus(h, threshold=1e9)).mean()
        first = (value.detach().view(1), h.detach(), s.detach())
    else:
        z = c["values"].double() * scale
        logq = torch.log_softmax(z, 1) if c["teacher_lse"] is None else z - c["teacher_lse"].double().unsqueeze(1)
        kl = (logq.exp() * (logq - picked)).sum(1) * used
        value = kl.sum() / used.sum() / scale ** 2
        first = (value.detach().view(1), kl.detach())
    (dpicked,) = torch.autograd.grad(value, picked)
    out = torch.empty(T, V, dtype=torch.float64, device="cuda")
    for a in cuts:
        part = slice(a, a + _rows(V))
        p = torch.exp(x[part].double().mul_(scale).sub_(lse[part, None]))
        out[part] = p.mul_(-scale * dpicked[part].sum(1, keepdim=True)).scatter_add_(1, pick[part], scale * dpicked[part])
    return (*first, out) if first else out
