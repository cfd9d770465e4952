"""Performance cases of the operators behind the decode attention: routing to experts, products in 8-bit integers
(dense and by expert), and sampling of tokens.

Every case runs in two forms.  The plain form (`own = False`) spells the operator out in elementary torch operations;
the other form makes the calls of `paper_2609_07008_b200.binding` that a program makes.

Routing.  s = softmax(logits) or sigmoid(logits), c = s + bias.  A group's rank is the sum of its `group_top` largest c;
experts of the `top_groups` best groups take part; the k largest c are chosen (ties: the lower index), in descending
order; weights are the chosen s, divided by their sum where asked for, times `scale`.  The (token, slot) pairs t * k + s
are then listed by expert, ascending inside an expert.
8-bit products.  A row of n values has the scale fp32(max|x| / 127) and the codes round(x / scale), half to even.
y[t][o] = scale_x[t] * scale_w[o] * sum_j X[t][j] W[o][j]; by expert, row i of expert e's list is a pair p, and
y[p] = W[e] x[p / per].
Sampling.  p_i = exp((l_i - max l) / T).  In the order of falling logits (ties: the lower index first), a token stays
if its rank is below top_k, if the p in front of it sum to less than top_p times the sum over the top_k, and if
p >= min_p; the first one always stays.  The token is the first of those that stayed, by index, whose cumulated p exceeds
u times their sum.  T = 0 takes the largest logit.
"""
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one layer of a decode step: 64 running requests, grouped sigmoid routing with a balance bias
        dict(name="route_decode_64", op="route", n=64, experts=256, k=6, groups=8, top_groups=4, group_top=2,
             score="sigmoid", bias=1, renorm=1, scale=2.5, dtype="f32"),
        # a short prompt, softmax scores in bf16, the best expert stands for its group
        dict(name="route_prompt_777", op="route", n=777, experts=160, k=6, groups=8, top_groups=3, group_top=1,
             score="softmax", bias=0, renorm=0, scale=1.0, dtype="bf16"),
        # the tokens of a long prompt, no groups
        dict(name="route_prompt_32768", op="route", n=32768, experts=256, k=8, groups=1, top_groups=1, group_top=1,
             score="sigmoid", bias=1, renorm=1, scale=1.0, dtype="f32"),
        # W_b of the 64-head shape for five tokens, fp32 out: the weights' bytes count
        dict(name="product_decode_5", op="product", n=5, n_out=4096, k=8192, out="f32"),
        # nothing a multiple of anything
        dict(name="product_odd_333", op="product", n=333, n_out=1001, k=777, out="bf16"),
        # W_b of the 128-head shape for a prompt of 8192 tokens
        dict(name="product_prompt_8192", op="product", n=8192, n_out=7168, k=16384, out="bf16"),
        # first products of the experts in a decode step: 64 tokens, one or two rows for most experts
        dict(name="experts_decode_64", op="experts", n=64, experts=128, slots=6, per=6, n_out=2048, k=4096, out="bf16",
             skew=0.5, drop=0.2, geo=1),
        # second products for a short prompt: every pair has a row of its own; ragged, some experts without rows
        dict(name="experts_down_1000", op="experts", n=1000, experts=64, slots=6, per=1, n_out=4096, k=1024, out="f32",
             skew=1.5, drop=0.3, geo=2),
        # first products for a long prompt
        dict(name="experts_prompt_8192", op="experts", n=8192, experts=128, slots=6, per=6, n_out=2048, k=4096, out="bf16",
             skew=0.7, drop=0.2, geo=3),
        # one request with every filter on
        dict(name="sample_1", op="sample", n=1, vocab=32001, dtype="f32", top_k=50, top_p=0.9, min_p=0.02, greedy=0.0, spread=2.5),
        # a running batch: each request has its own temperature and filters, some are greedy
        dict(name="sample_batch_64", op="sample", n=64, vocab=131072, dtype="f32", top_k=-1, top_p=-1.0, min_p=-1.0, greedy=0.1,
             spread=2.5),
        # many drafted tokens, plain sampling by nucleus, logits in bf16 (many ties)
        dict(name="sample_drafts_256", op="sample", n=256, vocab=65537, dtype="bf16", top_k=0, top_p=0.95, min_p=0.0, greedy=0.0,
             spread=2.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "product", "experts", "sample"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log_int(rng, 4, 256 // groups)
        top = rng.randrange(1, groups + 1)
        k = rng.randrange(1, min(8, top * (experts // groups)) + 1)
        score = rng.choice(["softmax", "sigmoid"])
        return dict(op=op, n=_log_int(rng, 1, 32768), experts=experts, k=k, groups=groups, top_groups=top,
                    group_top=rng.choice([1, 2]), score=score, bias=rng.randrange(2), renorm=rng.randrange(2),
                    scale=rng.choice([1.0, 2.5]), dtype=rng.choice(["f32", "bf16"]))
    if op == "product":
        n, n_out, k = _log_int(rng, 1, 8192), _log_int(rng, 16, 7168), _log_int(rng, 32, 16384)
        return dict(op=op, n=n, n_out=n_out, k=k, out=rng.choice(["bf16", "f32"]))
    if op == "experts":
        slots = rng.choice([1, 2, 4, 6, 8])
        experts = _log_int(rng, max(8, slots), 128)
        return dict(op=op, n=_log_int(rng, 1, 8192 * 6 // slots), experts=experts, slots=slots, per=rng.choice([1, slots]),
                    n_out=_log_int(rng, 64, 2048), k=_log_int(rng, 128, 4096), out=rng.choice(["bf16", "f32"]),
                    skew=rng.uniform(0.0, 1.0), drop=rng.choice([0.0, 0.2, 0.4]), geo=rng.randrange(1, 1 << 20))
    vocab = _log_int(rng, 1000, 150000)
    return dict(op=op, n=_log_int(rng, 1, max(1, 16_000_000 // vocab)), vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                top_k=rng.choice([-1, 0, 1, 40, 1000]), top_p=rng.choice([-1.0, 1.0, 0.3, 0.9, 0.99]),
                min_p=rng.choice([-1.0, 0.0, 0.05]), greedy=rng.choice([0.0, 0.1]), spread=rng.uniform(1.0, 4.0))


def _pairs(case):
    """The expert of every (token, slot) pair, -1 where the fan-out dropped it: from the case alone."""
    r = np.random.default_rng(np.random.PCG64(case["geo"]))
    popular = r.standard_normal(case["experts"]) * case["skew"]
    score = r.gumbel(size=(case["n"], case["experts"])) + popular
    ids = np.argpartition(-score, case["slots"] - 1, axis=1)[:, :case["slots"]]
    ids[r.random((case["n"], case["slots"])) < case["drop"]] = -1
    return ids.reshape(-1)


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "route":
        n, e, k = case["n"], case["experts"], case["k"]
        return {"bytes": n * e * size[case["dtype"]] + case["bias"] * e * 4 + n * k * 12 + (e + 1) * 4, "flops": 8 * n * e}
    if case["op"] == "product":
        n, o, k = case["n"], case["n_out"], case["k"]
        return {"bytes": n * k * 2 + o * (k + 4) + n * o * size[case["out"]], "flops": 2 * n * o * k}
    if case["op"] == "experts":
        ids = _pairs(case)
        used = ids[ids >= 0]
        x_rows = case["n"] * case["slots"] // case["per"]
        o, k = case["n_out"], case["k"]
        return {"bytes": x_rows * k * 2 + len(np.unique(used)) * o * (k + 4) + len(used) * (o * size[case["out"]] + 4),
                "flops": 2 * len(used) * o * k}
    return {"bytes": case["n"] * (case["vocab"] * size[case["dtype"]] + 28), "flops": 4 * case["n"] * case["vocab"]}


# ------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7907 + 13)
    return g


def _quantise(x):
    """Rows of x (bf16) -> codes (float64 whole numbers), scales (float32).  The quotients are taken in 64 bits: in 32 a value
    next to the middle between two codes may fall on it.  Divisions are by tensors: by a number they may become products."""
    top = x.abs().amax(-1, keepdim=True).float()
    scale = top / torch.full_like(top, 127.0)
    return torch.nan_to_num(torch.round(x.double() / scale.double())).clamp(-127, 127), scale


def _weights(g, mats, n_out, k):
    """8-bit weights as a program keeps them: codes [mats, n_out, k rounded up to 16] int8, scales [mats, n_out] float32."""
    codes = torch.zeros((mats, n_out, (k + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    scales = torch.empty((mats, n_out), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 27) // (n_out * k))
    for lo in range(0, mats, step):
        w = (torch.randn((min(step, mats - lo), n_out, k), generator=g, device="cuda") * 0.02).to(torch.bfloat16)
        c, s = _quantise(w)
        codes[lo:lo + step, :, :k], scales[lo:lo + step] = c.to(torch.int8), s[..., 0]
    return codes, scales


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "route":
        x = torch.randn((case["n"], case["experts"]), generator=g, device="cuda") * 1.5
        s["logits"] = x.to(torch.bfloat16) if case["dtype"] == "bf16" else x
        s["bias"] = torch.randn(case["experts"], generator=g, device="cuda") * 0.1 if case["bias"] else None
    elif case["op"] in ("product", "experts"):
        experts = case["op"] == "experts"
        s["codes"], s["scales"] = _weights(g, case["experts"] if experts else 1, case["n_out"], case["k"])
        rows = case["n"] * case["slots"] // case["per"] if experts else case["n"]
        # activations: a few channels are much larger than the rest
        x = torch.randn((rows, case["k"]), generator=g, device="cuda")
        x *= 1.0 + 15.0 * (torch.rand(case["k"], generator=g, device="cuda") < 0.01)
        s["x"] = x.to(torch.bfloat16)
        s["out"] = torch.bfloat16 if case["out"] == "bf16" else torch.float32
        if experts:
            ids = _pairs(case)
            order = np.argsort(np.where(ids < 0, case["experts"], ids), kind="stable")
            count = np.bincount(ids[ids >= 0], minlength=case["experts"])
            off = np.concatenate([[0], np.cumsum(count)])
            order[off[-1]:] = -1
            s["row_off"] = torch.tensor(off, dtype=torch.int32, device="cuda")
            s["rows"] = torch.tensor(order, dtype=torch.int32, device="cuda")
            s["longest"] = int(count.max())
            s["y"] = torch.zeros((len(ids), case["n_out"]), dtype=s["out"], device="cuda")   # rows of dropped pairs stay 0
    else:
        n, v = case["n"], case["vocab"]
        x = torch.randn((n, v), generator=g, device="cuda") * case["spread"]
        s["logits"] = x.to(torch.bfloat16) if case["dtype"] == "bf16" else x
        pick = lambda given, choices: (torch.full((n,), float(given), device="cuda") if given >= 0 else  # noqa: E731
                                       torch.tensor(choices, device="cuda")[torch.randint(len(choices), (n,), generator=g, device="cuda")])
        greedy = torch.rand(n, generator=g, device="cuda") < case["greedy"]
        s["temperature"] = (0.5 + torch.rand(n, generator=g, device="cuda")).masked_fill(greedy, 0.0)
        s["top_k"] = pick(case["top_k"], [0.0, 1.0, 20.0, 50.0, 1000.0]).to(torch.int32)
        s["top_p"] = pick(case["top_p"], [1.0, 0.95, 0.9, 0.5])
        s["min_p"] = pick(case["min_p"], [0.0, 0.0, 0.02, 0.1])
        s["u"] = torch.rand(n, generator=g, device="cuda")
    if own:
        from paper_2609_07008_b200 import binding as rk
        s["ctx"] = rk.Context(64, 8, 256, 1024, [8 * i for i in range(8)], 1.0 / math.sqrt(192.0))
        if "codes" in s:
            s["w8"] = rk.Q8(s["codes"], s["scales"], case["k"])
    return s


# ------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------
def _plain_route(s):
    case = s["case"]
    n, e, k, groups = case["n"], case["experts"], case["k"], case["groups"]
    x = s["logits"].double()                    # 64 bits: neighbours in the order are often closer than 32 bits tell apart
    if case["score"] == "softmax":
        p = torch.exp(x - x.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-x))
    c = p if s["bias"] is None else p + s["bias"].double()
    if groups > 1:
        by = c.view(n, groups, e // groups)
        rank = torch.sort(by, dim=2, descending=True).values[..., :case["group_top"]].sum(2)
        best = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        open_ = torch.zeros((n, groups), dtype=torch.bool, device="cuda").scatter_(1, best, True)
        c = torch.where(open_[..., None], by, torch.full_like(by, float("-inf"))).view(n, e)
    ids = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    w = torch.gather(p, 1, ids)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True)
    flat = ids.reshape(-1)
    rows = torch.sort(flat, stable=True).indices
    ends = torch.cumsum((flat[None, :] == torch.arange(e, device="cuda")[:, None]).sum(1), 0)
    row_off = torch.cat([torch.zeros_like(ends[:1]), ends])
    return ids.to(torch.int32), (w * case["scale"]).float(), row_off.to(torch.int32), rows.to(torch.int32)


def _plain_product(s):
    x, sx = _quantise(s["x"])
    acc = torch.matmul(x, s["codes"][0, :, :s["case"]["k"]].double().t())           # 64 bits: the sums need up to 31
    return (acc * sx.double() * s["scales"][0].double()).to(s["out"])


def _plain_experts(s):
    case = s["case"]
    # every expert's rows side by side, padded to the longest list, so that one batched product does them all
    lane = torch.arange(s["longest"], device="cuda")
    at = s["row_off"][:-1, None].long() + lane
    used = at < s["row_off"][1:, None]
    pair = s["rows"].long()[torch.where(used, at, torch.zeros_like(at))]
    pair = torch.where(used, pair, torch.zeros_like(pair))
    x, sx = _quantise(s["x"])
    acc = torch.matmul(x[pair // case["per"]], s["codes"][..., :case["k"]].double().transpose(1, 2))
    acc = acc * sx[pair // case["per"]].double() * s["scales"][:, None].double()
    y = torch.zeros_like(s["y"])
    y[pair[used]] = acc[used].to(s["out"])
    return y


def _plain_sample(s):
    x = s["logits"].double()                    # 64 bits: long sums, and borders in them
    n, v = x.shape
    temp = s["temperature"].double()[:, None]
    greedy = temp <= 0
    p = torch.exp((x - x.amax(1, keepdim=True)) / torch.where(greedy, torch.ones_like(temp), temp))
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    sp = torch.gather(p, 1, order)
    rank = torch.arange(v, device="cuda")[None]
    top_k = torch.where(s["top_k"] > 0, s["top_k"], torch.full_like(s["top_k"], v))[:, None]
    sp = torch.where(rank < top_k, sp, torch.zeros_like(sp))
    run = torch.cumsum(sp, 1)
    before = torch.cat([torch.zeros_like(run[:, :1]), run[:, :-1]], 1)
    top_p = s["top_p"].double()[:, None]
    keep = (rank < top_k) & ((before < top_p * run[:, -1:]) | (top_p >= 1)) & (sp >= s["min_p"].double()[:, None])
    keep = (keep & ~greedy) | (rank == 0)
    kept = torch.zeros_like(p).scatter_(1, order, torch.where(keep, sp, torch.zeros_like(sp)))
    cdf = torch.cumsum(kept, 1)
    # rounding may leave the last sum at u * total: then it is the last token that stayed
    beyond = cdf > torch.minimum(s["u"].double()[:, None] * cdf[:, -1:], cdf[:, -1:] * (1 - 2.0 ** -50))
    token = torch.argmax(beyond.to(torch.int8), 1, keepdim=True)
    return token[:, 0].to(torch.int32), (torch.gather(kept, 1, token)[:, 0] / cdf[:, -1]).float()


def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        return {"route": _plain_route, "product": _plain_product, "experts": _plain_experts, "sample": _plain_sample}[op](s)
    ctx = s["ctx"]
    if op == "route":
        ids, w = ctx.rk_moe_route(s["logits"], case["k"], bias=s["bias"], score=case["score"], n_groups=case["groups"],
                                  top_groups=case["top_groups"], group_top=case["group_top"], renorm=bool(case["renorm"]),
                                  scale=case["scale"])
        row_off, rows = ctx.rk_moe_group(ids, case["experts"])
        return ids, w, row_off, rows
    if op == "product":
        return ctx.rk_matmul8(s["w8"], ctx.rk_quant8(s["x"]), out_dtype=s["out"])
    if op == "experts":
        return ctx.rk_matmul8_experts(s["w8"], ctx.rk_quant8(s["x"]), s["row_off"], s["rows"], case["per"], y=s["y"])
    return ctx.rk_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


# ------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------
def _exact_route(case, s):
    """On the host, token by token in lexicographic order of (-score, index)."""
    x = s["logits"].double().cpu().numpy()
    n, e = x.shape
    if n * e > 12_000_000:
        return None
    if case["score"] == "softmax":
        z = np.exp(x - x.max(axis=1, keepdims=True))
        p = z / z.sum(axis=1, keepdims=True)
    else:
        p = 1.0 / (1.0 + np.exp(-x))
    c = p + (0.0 if s["bias"] is None else s["bias"].double().cpu().numpy()[None])
    size = e // case["groups"]
    if case["groups"] > 1:
        g = -np.sort(-c.reshape(n, case["groups"], size), axis=2)[:, :, :case["group_top"]].sum(axis=2)
        place = np.argsort(np.argsort(-g, axis=1, kind="stable"), axis=1, kind="stable")     # the place of every group
        c = np.where(np.repeat(place < case["top_groups"], size, axis=1), c, -np.inf)
    ids = np.argsort(-c, axis=1, kind="stable")[:, :case["k"]]
    w = np.take_along_axis(p, ids, axis=1)
    w = w * case["scale"] / (w.sum(axis=1, keepdims=True) if case["renorm"] else 1.0)
    flat = ids.reshape(-1)
    return ids, w, np.searchsorted(np.sort(flat), np.arange(e + 1)), np.lexsort((np.arange(flat.size), flat))


def _codes64(x):
    step = (x.double().abs().max(dim=1).values / 127.0).float().double()
    q = x.double() / step[:, None]
    low = torch.floor(q)
    up = (q - low > 0.5) | ((q - low == 0.5) & (torch.remainder(low, 2) == 1))
    return low + up, step


def _exact_product(s, codes, scales, x):
    q, step = _codes64(x)
    y = torch.einsum("tk,ok->to", q, codes[:, :x.shape[1]].double())
    return y * (step[:, None] * scales.double()[None])


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    if case["op"] == "route":
        out = _exact_route(case, s)
        return None if out is None else tuple(torch.from_numpy(np.ascontiguousarray(o)) for o in out)
    if case["op"] == "product":
        return _exact_product(s, s["codes"][0], s["scales"][0], s["x"])
    if case["op"] == "experts":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        off = s["row_off"].tolist()
        for e in range(case["experts"]):
            pair = s["rows"][off[e]:off[e + 1]].long()
            if len(pair):
                y[pair] = _exact_product(s, s["codes"][e], s["scales"][e], s["x"][torch.div(pair, case["per"], rounding_mode="floor")])
        return y
    x = s["logits"].double().cpu().numpy()
    if x.size > 20_000_000:
        return None
    temp, top_p, min_p, u = (s[k].double().cpu().numpy() for k in ("temperature", "top_p", "min_p", "u"))
    tokens, probs = np.zeros(len(x), dtype=np.int64), np.ones(len(x))
    for r, row in enumerate(x):
        top = np.argmax(row)
        tokens[r] = top
        if temp[r] > 0:
            p = np.exp((row - row[top]) / temp[r])
            order = np.lexsort((np.arange(len(row)), -row))
            k = int(s["top_k"][r])
            order = order[:k] if k > 0 else order
            front = np.concatenate([[0.0], np.cumsum(p[order])])
            if top_p[r] < 1:
                order = order[:max(1, int(np.searchsorted(front[:-1], top_p[r] * front[-1], side="left")))]
            order = order[:max(1, int((p[order] >= min_p[r]).sum()))]
            stay = np.sort(order)
            total = np.cumsum(p[stay])
            at = min(int(np.searchsorted(total, u[r] * total[-1], side="right")), len(stay) - 1)
            tokens[r], probs[r] = stay[at], p[stay[at]] / total[-1]
    return torch.from_numpy(tokens), torch.from_numpy(probs)
