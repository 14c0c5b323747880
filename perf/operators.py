"""What the token-gate operators are measured on: a many-class logistic gate learned over tokens.

The operators and what a user's program does with them:

``embed`` / ``embed_grad``   rows of a token table, scaled, as the rows X that a logistic model reads; and the table's
                             gradient, summed over all places where a token stands
``route`` / ``route_grad``   a gate's logits to the k experts of every token with their weights, and how many tokens each
                             expert got; and the gradient of the weights back to the logits
``ckpt8`` / ``ckpt8_grad``   the rows kept between forward and backward in 8 bits (one scale for 128 columns of a row), read
                             back; and the gradient of a C-class logistic layer taken from the 8-bit rows

Each case is one pass through one of them.  ``own`` false: plain torch in 32 bits; true: the library's entry points.
"""
import math

import torch

own = False

GROUP = 128                                     # columns that share a scale in the 8-bit form


def listed():
    return [
        # a decoding step: eight sequences, one token each; the gate of a 64-expert layer
        {"name": "route-decode", "op": "route", "T": 8, "E": 64, "k": 6, "groups": 1, "top": 1, "score": "softmax",
         "renorm": True, "dtype": "bfloat16"},
        # a prompt's or a training step's 16384 tokens, 256 experts in 8 groups of which 4 are kept
        {"name": "route-prefill", "op": "route", "T": 16384, "E": 256, "k": 8, "groups": 8, "top": 4, "score": "sigmoid",
         "renorm": True, "dtype": "float32"},
        # a small ragged micro-batch, an expert count that is no power of two, weights as they come out of the softmax
        {"name": "route-grad-ragged", "op": "route_grad", "T": 1001, "E": 100, "k": 2, "score": "softmax", "renorm": False,
         "dtype": "bfloat16"},
        # a large training step
        {"name": "route-grad-train", "op": "route_grad", "T": 32768, "E": 128, "k": 8, "score": "sigmoid", "renorm": True,
         "dtype": "float32"},
        # a decoding step's lookup
        {"name": "embed-decode", "op": "embed", "T": 16, "V": 32000, "n": 4096, "dtype": "bfloat16", "ids": "int64"},
        # a training step's lookup, tokens past a whole number of tiles
        {"name": "embed-train", "op": "embed", "T": 40009, "V": 100000, "n": 1024, "dtype": "float32", "ids": "int32"},
        # a small table with rows of odd length, one token marked as padding
        {"name": "embed-grad-odd", "op": "embed_grad", "T": 2003, "V": 10007, "n": 257, "dtype": "float32", "ids": "int64",
         "accumulate": False, "pad": True},
        # a training step of a large vocabulary, a whole gradient written
        {"name": "embed-grad-train", "op": "embed_grad", "T": 32768, "V": 65536, "n": 1024, "dtype": "bfloat16",
         "ids": "int32", "accumulate": False, "pad": False},
        # the rows of a few sequences, a row length that ends inside a group
        {"name": "ckpt8-short", "op": "ckpt8", "T": 100, "n": 1000, "dtype": "float32"},
        # a layer's activations of a training step
        {"name": "ckpt8-train", "op": "ckpt8", "T": 16384, "n": 4096, "dtype": "bfloat16"},
        # the gradient of one logistic unit (a reward or a probe) over the rows of a training step
        {"name": "ckpt8-grad-unit", "op": "ckpt8_grad", "T": 65536, "n": 256, "C": 1, "dtype": "float32"},
        # the gradient of a 64-expert gate
        {"name": "ckpt8-grad-gate", "op": "ckpt8_grad", "T": 16384, "n": 4096, "C": 64, "dtype": "float32"},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "route_grad", "embed", "embed_grad", "ckpt8", "ckpt8_grad"])
    dtype = rng.choice(["float32", "bfloat16"])
    if op in ("route", "route_grad"):
        E = rng.choice([8, 16, 60, 64, 100, 128, 160, 256, 384, 512])
        T = _spread(rng, 1 if op == "route" else 64, 16384 * 256 // E)
        k = rng.choice([1, 2, 4, 6, 8])
        case = {"op": op, "T": T, "E": E, "k": k, "score": rng.choice(["sigmoid", "softmax"]),
                "renorm": rng.random() < 0.7, "dtype": dtype}
        if op == "route":
            groups = rng.choice([1, 1, 2, 4])
            top = rng.randint(max(1, -(-k * groups // E)), groups)
            case.update(groups=groups, top=top)
        return case
    if op in ("embed", "embed_grad"):
        n = _spread(rng, 64, 8192)
        n = n // 8 * 8 if rng.random() < 0.6 else n
        V = _spread(rng, 1000, 65536 * 1024 // n if op == "embed_grad" else min(131072, 100000 * 2048 // n))
        T = _spread(rng, 1 if op == "embed" else 64, min(131072, 32768 * 1024 // n))
        case = {"op": op, "T": T, "V": V, "n": n, "dtype": dtype, "ids": rng.choice(["int32", "int64"])}
        if op == "embed_grad":
            case.update(accumulate=rng.random() < 0.4, pad=rng.random() < 0.3)
        return case
    if op == "ckpt8":
        n = _spread(rng, 64, 16384)
        n = n // 8 * 8 if rng.random() < 0.6 else n
        return {"op": op, "T": _spread(rng, 1, 16384 * 4096 // n), "n": n, "dtype": dtype}
    n = _spread(rng, 64, 8192)
    n = n // 16 * 16 if rng.random() < 0.6 else n
    C = rng.choice([1, 2, 5, 8, 16, 40, 64, 100, 128])
    return {"op": op, "T": _spread(rng, 64, min(65536, 16384 * 4096 * 64 // (n * max(C, 64)))), "n": n, "C": C, "dtype": dtype}


def _tokens(T, V, gen, dtype):
    """Token numbers with the frequencies of text (the r-th most frequent one about 1/r as often), spread over the table."""
    rank = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64).mul_(math.log(V)).exp_().long().clamp_(1, V) - 1
    return torch.randperm(V, generator=gen, device="cuda")[rank].to(dtype)


def _logits(T, E, gen, dtype):
    """What a gate gives: a part that all tokens share and a part of each token's own."""
    return (0.5 * torch.randn(E, generator=gen, device="cuda") + 1.5 * torch.randn(T, E, generator=gen, device="cuda")).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    c, dt = dict(case), getattr(torch, case["dtype"])
    T = c["T"]
    if c["op"] == "route":
        c["logits"] = _logits(T, c["E"], gen, dt)
        c["bias"] = 0.05 * torch.randn(c["E"], generator=gen, device="cuda")
    elif c["op"] == "route_grad":
        c["logits"] = _logits(T, c["E"], gen, dt)
        c["ids"] = c["logits"].float().sort(dim=1, descending=True, stable=True)[1][:, :c["k"]].to(torch.int32).contiguous()
        c["dweights"] = torch.randn(T, c["k"], generator=gen, device="cuda")
    elif c["op"] == "embed":
        c["table"] = (torch.randn(c["V"], c["n"], generator=gen, device="cuda") / math.sqrt(c["n"])).to(dt)
        c["tokens"] = _tokens(T, c["V"], gen, getattr(torch, c["ids"]))
        c["scale"] = math.sqrt(c["n"])
    elif c["op"] == "embed_grad":
        c["tokens"] = _tokens(T, c["V"], gen, getattr(torch, c["ids"]))
        c["dout"] = (torch.randn(T, c["n"], generator=gen, device="cuda") / T).to(dt)
        c["scale"] = math.sqrt(c["n"])
        c["padding"] = int(c["tokens"][T // 2]) if c["pad"] else -1
        # the sum of the micro-batches so far, where this one is added to it
        c["grad"] = torch.randn(c["V"], c["n"], generator=gen, device="cuda") / T if c["accumulate"] else None
    elif c["op"] == "ckpt8":
        # a layer's activations: most columns alike, a few much larger than the others
        wide = torch.ones(c["n"], device="cuda")
        wide[torch.rand(c["n"], generator=gen, device="cuda") < 0.01] = 20.0
        c["x"] = (torch.randn(T, c["n"], generator=gen, device="cuda") * wide).to(dt)
    else:
        n, C = c["n"], c["C"]
        ng = -(-n // GROUP)
        c["q"] = torch.randn(T, n, generator=gen, device="cuda").mul_(40).round_().clamp_(-127, 127).to(torch.int8)
        c["s"] = 0.02 + 0.02 * torch.rand(T, ng, generator=gen, device="cuda")
        z = torch.randn(T, C, generator=gen, device="cuda")
        if C == 1:                              # one unit: sigmoid minus a 0/1 target
            dz = torch.sigmoid(z) - torch.randint(0, 2, (T, 1), generator=gen, device="cuda")
        else:                                   # C classes: softmax minus the one that is right
            dz = torch.softmax(z, 1)
            dz[torch.arange(T, device="cuda"), torch.randint(0, C, (T,), generator=gen, device="cuda")] -= 1
        c["dz"] = (dz / T).to(dt)
    return c


def run(state):
    return (_own if own else _plain)[state["op"]](state)


# ---- the library's entry points ------------------------------------------------------------------------

def _own_route(c):
    from paper_2308_10037_b200 import lr_route
    return lr_route(c["logits"], c["k"], bias=c["bias"], groups=c["groups"], top_groups=c["top"], score=c["score"],
                    renorm=c["renorm"], factor=2.5)


def _own_route_grad(c):
    from paper_2308_10037_b200 import lr_route_grad
    return lr_route_grad(c["logits"], c["ids"], c["dweights"], score=c["score"], renorm=c["renorm"], factor=2.5)


def _own_embed(c):
    from paper_2308_10037_b200 import lr_embed
    return lr_embed(c["table"], c["tokens"], scale=c["scale"])


def _own_embed_grad(c):
    from paper_2308_10037_b200 import lr_embed_grad
    # a pass adds to a copy, so that every pass gives the same sum
    into = c["grad"].clone() if c["accumulate"] else None
    return lr_embed_grad(c["tokens"], c["dout"], c["V"], scale=c["scale"], padding_id=c["padding"], out=into,
                         accumulate=c["accumulate"])


def _own_ckpt8(c):
    from paper_2308_10037_b200 import lr_ckpt8_load, lr_ckpt8_save
    q, s = lr_ckpt8_save(c["x"])
    return lr_ckpt8_load(q, s, dtype=c["x"].dtype), s


def _own_ckpt8_grad(c):
    from paper_2308_10037_b200 import lr_ckpt8_grad
    return lr_ckpt8_grad(c["q"], c["s"], c["dz"])


_own = {"route": _own_route, "route_grad": _own_route_grad, "embed": _own_embed, "embed_grad": _own_embed_grad,
        "ckpt8": _own_ckpt8, "ckpt8_grad": _own_ckpt8_grad}


# ---- the same in plain torch ---------------------------------------------------------------------------

def _probabilities(x, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    e = torch.exp(x - x.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(c):
    x = c["logits"].float()
    T, E = x.shape
    p = _probabilities(x, c["score"])
    # what is chosen by: the sigmoid with the balance bias added, or the logit with it (softmax keeps the order of the logits)
    choice = (p if c["score"] == "sigmoid" else x) + c["bias"]
    if c["groups"] > 1:
        by_group = choice.view(T, c["groups"], E // c["groups"])
        top = by_group.sort(dim=2, descending=True)[0]
        worth = top[:, :, :2].sum(2) if c["score"] == "sigmoid" else top[:, :, 0]
        kept = worth.sort(dim=1, descending=True, stable=True)[1][:, :c["top"]]
        keep = torch.zeros(T, c["groups"], dtype=torch.bool, device=x.device).scatter_(1, kept, True)
        choice = torch.where(keep[:, :, None], by_group, -math.inf).view(T, E)
    ids = choice.sort(dim=1, descending=True, stable=True)[1][:, :c["k"]]
    w = p.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    counts = torch.zeros(E, dtype=torch.int32, device=x.device)
    counts.index_add_(0, ids.reshape(-1), torch.ones(ids.numel(), dtype=torch.int32, device=x.device))
    return ids.to(torch.int32), w * 2.5, counts


def _plain_route_grad(c):
    x, ids, g = c["logits"].float(), c["ids"].long(), c["dweights"]
    p = _probabilities(x, c["score"])
    chosen = p.gather(1, ids)
    if c["renorm"]:
        total = chosen.sum(1, keepdim=True)
        w = chosen / total
        dchosen = (g - (g * w).sum(1, keepdim=True)) * (2.5 / total)
    else:
        dchosen = g * 2.5
    dp = torch.zeros_like(p).scatter_(1, ids, dchosen)
    if c["score"] == "sigmoid":
        dx = dp * p * (1.0 - p)
    else:
        dx = p * (dp - (dp * p).sum(1, keepdim=True))
    return dx.to(c["logits"].dtype)


def _plain_embed(c):
    return (c["table"][c["tokens"].long()].float() * c["scale"]).to(c["table"].dtype)


def _plain_embed_grad(c):
    ids = c["tokens"].long()
    rows = torch.where((ids != c["padding"])[:, None], c["dout"].float() * c["scale"], 0.0)
    into = c["grad"].clone() if c["accumulate"] else torch.zeros(c["V"], c["n"], device=ids.device)
    return into.index_add_(0, ids, rows)


def _grouped(x):
    T, n = x.shape
    ng = -(-n // GROUP)
    full = torch.zeros(T, ng * GROUP, dtype=x.dtype, device=x.device)
    full[:, :n] = x
    return full.view(T, ng, GROUP)


def _plain_ckpt8(c):
    x = c["x"].float()
    T, n = x.shape
    g = _grouped(x)
    top = g.abs().amax(2)
    s = top / 127.0
    q = (g * (127.0 / top)[:, :, None]).round().clamp(-127, 127).to(torch.int8)
    back = (q.float() * s[:, :, None]).view(T, -1)[:, :n]
    return back.to(c["x"].dtype).contiguous(), s


def _plain_ckpt8_grad(c):
    T, n = c["q"].shape
    dz = c["dz"].float()
    x = (_grouped(c["q"]).float() * c["s"][:, :, None]).view(T, -1)[:, :n]
    return dz.t() @ x, dz.sum(0)


_plain = {"route": _plain_route, "route_grad": _plain_route_grad, "embed": _plain_embed, "embed_grad": _plain_embed_grad,
          "ckpt8": _plain_ckpt8, "ckpt8_grad": _plain_ckpt8_grad}


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    c, T = case, case["T"]
    b = 4 if c["dtype"] == "float32" else 2
    if c["op"] == "route":
        return {"bytes": T * c["E"] * b + T * c["k"] * 8 + c["E"] * 8, "flops": T * c["E"] * 4}
    if c["op"] == "route_grad":
        # the sigmoid's gradient needs the chosen logits alone, the softmax's all of them
        read = T * c["k"] * b if c["score"] == "sigmoid" else T * c["E"] * b
        return {"bytes": read + T * c["k"] * 8 + T * c["E"] * b, "flops": T * c["E"] * 4}
    if c["op"] in ("embed", "embed_grad"):
        tb = 4 if c["ids"] == "int32" else 8
        # different tokens among T drawn with frequencies 1/r: one for each r, less those that did not come up
        seen = sum((1.0 - (1.0 - math.log1p(1.0 / r) / math.log(c["V"])) ** T) * w for r, w in _ranks(c["V"]))
        if c["op"] == "embed":
            return {"bytes": int(seen * c["n"] * b + T * c["n"] * b + T * tb), "flops": T * c["n"]}
        # a whole gradient written; added to another, that one is copied first and the rows of the tokens read and written again
        out = 2 * c["V"] * c["n"] * 4 + 2 * seen * c["n"] * 4 if c["accumulate"] else c["V"] * c["n"] * 4
        return {"bytes": int(T * c["n"] * b + T * tb + out), "flops": 2 * T * c["n"]}
    ng = -(-c["n"] // GROUP)
    if c["op"] == "ckpt8":                      # kept: one byte a value and the scales, written and read; values in and out
        return {"bytes": T * c["n"] * (2 * b + 2) + 2 * T * ng * 4, "flops": 3 * T * c["n"]}
    return {"bytes": T * c["n"] + T * ng * 4 + T * c["C"] * b + c["C"] * c["n"] * 4, "flops": 2 * T * c["n"] * c["C"]}


def _ranks(V):
    """Ranks 1..V in steps that grow with the rank, each with the number of ranks it stands for."""
    r = 1
    while r < V:
        step = max(1, r // 64)
        yield r + (step - 1) / 2, min(step, V - r)
        r += step


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    c = prepare(case, seed)
    op = c["op"]
    if op in ("route", "route_grad"):
        x = c["logits"].double()
        p = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, dim=1)
        if op == "route":
            v = (p if c["score"] == "sigmoid" else x) + c["bias"].double()
            T, E = v.shape
            if c["groups"] > 1:
                g = v.reshape(T, c["groups"], -1)
                two = g.topk(min(2, g.shape[2]) if c["score"] == "sigmoid" else 1, dim=2)[0].sum(2)
                last = two.topk(c["top"], dim=1)[0][:, -1:]
                v = v.masked_fill((two < last).repeat_interleave(g.shape[2], dim=1), -math.inf)
            order = torch.argsort(v, dim=1, descending=True, stable=True)[:, :c["k"]]
            w = torch.gather(p, 1, order)
            if c["renorm"]:
                w = w / w.sum(1, keepdim=True)
            return None, 2.5 * w, None
        x.requires_grad_(True)
        p = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, dim=1)
        w = torch.gather(p, 1, c["ids"].long())
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        (2.5 * w * c["dweights"].double()).sum().backward()
        return x.grad
    if op == "embed":
        return c["table"].double().index_select(0, c["tokens"].long()) * c["scale"]
    if op == "embed_grad":
        got = torch.zeros(c["V"], c["n"], dtype=torch.float64, device="cuda") if c["grad"] is None else c["grad"].double()
        keep = torch.nonzero(c["tokens"] != c["padding"]).squeeze(1)
        return got.index_add_(0, c["tokens"][keep].long(), c["scale"] * c["dout"][keep].double())
    if op == "ckpt8":
        x = torch.nn.functional.pad(c["x"].double(), (0, -c["n"] % GROUP)).unflatten(1, (-1, GROUP))
        step = x.abs().max(dim=2)[0] / 127.0
        back = torch.round(x / step.unsqueeze(2)).mul(step.unsqueeze(2))
        return back.flatten(1)[:, :c["n"]], step
    q = torch.nn.functional.pad(c["q"].double(), (0, -c["n"] % GROUP)).unflatten(1, (-1, GROUP))
    x = (q * c["s"].double().unsqueeze(2)).flatten(1)[:, :c["n"]]
    dz = c["dz"].double()
    return torch.einsum("tc,tn->cn", dz, x), dz.sum(0)
