"""What a user of the routed 4-bit products has them do, as measured cases.

A layer of experts sends every row of its input to a few experts (``route_topk``), groups the rows of an expert
(``route_plan``), multiplies each group by that expert's matrix, which is kept in 4 bits (``Q4.mm_routed``), and sums the
results of a row with the router's weights (``route_combine``).  A plain layer is one matrix in 4 bits times the rows in hand
(``Q4.mm``).  Training a router takes the gradients of its weights and of the sum.  Accordingly a case has an ``op``:

  topk       the router's choice from its scores; with ``train`` the gradient of its weights as well
  plan       the grouping of the chosen pairs
  mm         rows times one 4-bit matrix
  experts    rows times their experts' matrices, the gated first half of a layer
  combine    the weighted sum and its gradients
  layer      all of it in turn, as a layer of a model calls it

``T`` rows, ``E`` experts, ``k`` of them for each row, ``K`` inputs and ``N`` outputs of a matrix (``F`` gated ones), ``g`` inputs to
a scale.  The plain forms dequantise and multiply in fp32; choices are made on the scores themselves where that decides, and in 64 bits
where scores and biases are added.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # The router of one new token: a launch and its latency.
        dict(name="topk_token", op="topk", T=1, E=64, k=4, dtype="bf16", score="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0,
             masked=0.0, train=False),
        # A long prompt through a router with balancing biases and groups of experts, scores in fp32.
        dict(name="topk_groups", op="topk", T=16384, E=256, k=8, dtype="f32", score="sigmoid", bias=True, groups=8, top_groups=4, renorm=True, scale=2.5,
             masked=0.0, train=False),
        # A training step's router: choice, weights and the gradient to the scores, some rows padding and some experts closed.
        dict(name="topk_train", op="topk", T=8192, E=128, k=8, dtype="bf16", score="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0,
             masked=0.02, train=True),
        # The pairs of one serving step ...
        dict(name="plan_step", op="plan", T=32, E=64, k=4),
        # ... and of a long prompt.
        dict(name="plan_prompt", op="plan", T=16384, E=256, k=8),
        # One new token through a plain layer: the matrix is read once, for one row.
        dict(name="mm_token", op="mm", T=1, K=4096, N=4096, g=128, dtype="bf16", out="bf16", zeros=False),
        # A few rows, odd sizes, small groups with zero points, results kept in fp32.
        dict(name="mm_few_odd", op="mm", T=5, K=4064, N=10999, g=32, dtype="f16", out="f32", zeros=True),
        # A serving batch through a wide layer.
        dict(name="mm_batch", op="mm", T=192, K=4096, N=14336, g=128, dtype="bf16", out="bf16", zeros=True),
        # A serving step's rows through the gated half of their experts: about one row for each matrix.
        dict(name="experts_step", op="experts", T=16, E=64, k=4, K=2048, F=1408, g=64, dtype="f16", zeros=True),
        # The weighted sum behind the experts and its gradients, of a training step.
        dict(name="combine_train", op="combine", T=4096, k=8, D=2048, dtype="bf16"),
        # A whole layer of experts for one new token ...
        dict(name="layer_token", op="layer", T=1, E=128, k=8, K=2048, F=768, g=128, dtype="bf16", zeros=False, score="softmax", bias=False, groups=1,
             top_groups=1, renorm=True, scale=1.0),
        # ... and for a prompt: the largest.
        dict(name="layer_prompt", op="layer", T=2048, E=64, k=4, K=2048, F=1408, g=128, dtype="bf16", zeros=True, score="sigmoid", bias=True, groups=8,
             top_groups=4, renorm=True, scale=1.5),
    ]


def draw(rng):
    def between(lo, hi, q=1):                      # over the logarithm, a multiple of q
        return max(q, int(math.exp(rng.uniform(math.log(lo), math.log(hi))) / q + 0.5) * q)

    def router(T):
        groups = rng.choice([1, 1, 4, 8])
        E = groups * between(max(2, 16 // groups), 256 // groups)
        top = 1 if groups == 1 else rng.randint(groups // 2, groups)
        k = rng.randint(1, min(10, E // groups * top))
        return dict(T=T, E=E, k=k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, top_groups=top,
                    renorm=rng.random() < 0.7, scale=rng.choice([1.0, 1.5, 2.5]))

    op = rng.choice(["topk", "topk", "plan", "mm", "mm", "mm", "experts", "experts", "combine", "layer", "layer"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    g, zeros = rng.choice([32, 64, 128, 128, 256]), rng.random() < 0.5
    if op == "topk":
        return dict(router(between(1, 16384)), op=op, dtype=rng.choice(["f32", "bf16", "f16"]), masked=rng.choice([0.0, 0.02]), train=rng.random() < 0.5)
    if op == "plan":
        c = router(between(1, 16384))
        return dict(op=op, T=c["T"], E=c["E"], k=c["k"])
    if op == "mm":
        return dict(op=op, T=between(1, 256), K=between(256, 8192, 32), N=between(64, 14336), g=g, dtype=dtype, out=rng.choice([dtype, "f32"]), zeros=zeros)
    if op == "combine":
        return dict(op=op, T=between(1, 4096), k=rng.randint(1, 8), D=between(64, 4096, 8), dtype=dtype)
    E, k = between(4, 64), rng.randint(1, 4)
    c = dict(op=op, T=between(1, 1024), E=E, k=k, K=between(256, 2048, 32), F=between(64, 1408, 32), g=g, dtype=dtype, zeros=zeros)
    if op == "layer":
        c.update(score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=1, top_groups=1, renorm=rng.random() < 0.7,
                 scale=rng.choice([1.0, 2.5]))
    return c


# ------------------------------------------------------------------------------------------- the inputs
def _matrices(gen, count, rows, cols, g, dtype, zeros):
    """Codes, scales and zero points of `count` matrices, as a quantiser leaves them: rows of weights with standard deviation near 1 / sqrt(cols)."""
    n_groups = -(-cols // g)
    codes = torch.randint(0, 256, (count, rows, cols // 2), generator=gen, device=DEV, dtype=torch.uint8)
    scales = ((torch.rand((count, rows, n_groups), generator=gen, device=DEV) + 0.5) / (4.6 * math.sqrt(cols))).to(TYPES[dtype])
    z = torch.randint(4, 12, (count, rows, n_groups), generator=gen, device=DEV, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def _scores(gen, T, E, dtype, masked):
    """A router's raw scores: some experts are liked better than others; `masked` of the rows are padding and of the experts closed."""
    l = 1.5 * torch.randn((T, E), generator=gen, device=DEV) + 0.5 * torch.randn((E,), generator=gen, device=DEV)
    if masked:
        rows = torch.rand((T, 1), generator=gen, device=DEV) < masked
        experts = torch.rand((1, E), generator=gen, device=DEV) < masked
        l = l.masked_fill(rows | experts, -math.inf)
    return l.to(TYPES[dtype])


def _data(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    op, T = case["op"], case["T"]
    d = {}
    if op in ("topk", "layer"):
        d["logits"] = _scores(gen, T, case["E"], case["dtype"] if op == "topk" else "f32", case.get("masked", 0.0))
        d["bias"] = 0.1 * normal(case["E"]) if case["bias"] else None
    if op == "topk":
        d["dweights"] = normal(T, case["k"])
    if op in ("plan", "experts"):
        d["ids"] = torch.topk(_scores(gen, T, case["E"], "f32", 0.0), case["k"], dim=1).indices.to(torch.int32)
    if op == "mm":
        d["x"] = normal(T, case["K"]).to(TYPES[case["dtype"]])
        d["up"] = _matrices(gen, 1, case["N"], case["K"], case["g"], case["dtype"], case["zeros"])
    if op in ("experts", "layer"):
        d["x"] = normal(T, case["K"]).to(TYPES[case["dtype"]])
        d["up"] = _matrices(gen, case["E"], 2 * case["F"], case["K"], case["g"], case["dtype"], case["zeros"])
    if op == "layer":
        d["down"] = _matrices(gen, case["E"], case["K"], case["F"], case["g"], case["dtype"], case["zeros"])
    if op == "combine":
        t = TYPES[case["dtype"]]
        d["y"], d["dout"] = normal(T * case["k"], case["D"]).to(t), normal(T, case["D"]).to(t)
        d["weights"] = torch.softmax(normal(T, case["k"]), dim=1)
        d["ids"] = torch.randint(0, 64, (T, case["k"]), generator=gen, device=DEV, dtype=torch.int32)
    return d


def prepare(case, seed):
    """Inputs, and the matrices as a program keeps them between calls."""
    s = dict(_data(case, seed), case=case)
    if own:
        from paper_2202_05868_amd import routed
        if "up" in s:
            s["up"] = routed.Q4(*s["up"], group=case["g"], gated=case["op"] != "mm").upload()
        if "down" in s:
            s["down"] = routed.Q4(*s["down"], group=case["g"]).upload()
        if case["op"] == "experts":
            s["plan"] = routed.route_plan(s["ids"], case["E"])
    return s


# ------------------------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2202_05868_amd import routed
    c, op = s["case"], s["case"]["op"]
    if op in ("topk", "layer"):
        how = dict(score=c["score"], renormalise=c["renorm"], scale=c["scale"])
        ids, weights = routed.route_topk(s["logits"], c["k"], bias=s["bias"], n_groups=c["groups"], top_groups=c["top_groups"], **how)
        if op == "layer":
            return dict(out=routed.experts_forward(s["x"], ids, weights, s["up"], s["down"]), ids=ids)
        r = dict(ids=ids, weights=weights)
        if c["train"]:
            r["dlogits"] = routed.route_topk_grad(s["logits"], ids, s["dweights"], **how)
        return r
    if op == "plan":
        p = routed.route_plan(s["ids"], c["E"])
        return dict(order=p.order, offsets=p.offsets)
    if op == "mm":
        return s["up"].mm(s["x"], y_dtype=TYPES[c["out"]])
    if op == "experts":
        return s["up"].mm_routed(s["x"], s["plan"])
    out = routed.route_combine(s["y"], s["ids"], s["weights"])
    dy, dweights = routed.route_combine_grad(s["dout"], s["y"], s["ids"], s["weights"])
    return dict(out=out, dy=dy, dweights=dweights)


# ------------------------------------------------------------------------------------------- the plain forms
def _plain_matrices(q, g):
    """[count, rows, cols] in fp32 from codes, scales and zero points."""
    codes, scales, zeros = q
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).float()
    cols = c.shape[-1]
    wide = scales.float().repeat_interleave(g, dim=-1)[..., :cols]
    z = 8.0 if zeros is None else zeros.float().repeat_interleave(g, dim=-1)[..., :cols]
    return (c - z) * wide


def _of_experts(q, used):
    return tuple(None if t is None else t[used] for t in q)


def _plain_scores(l, score):
    """Scores of every expert from raw scores in which -inf closes one; rows without an open one are zeros."""
    if score == "sigmoid":
        return torch.where(l == -math.inf, 0.0, 1 / (1 + torch.exp(-l)))
    m = l.amax(dim=1, keepdim=True)
    e = torch.exp(l - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(dim=1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total)


def _plain_topk(c, logits, bias):
    l = logits.float()
    closed = l == -math.inf
    key = l
    if bias is not None or c["groups"] > 1:
        key = _plain_scores(l.double(), c["score"]) + (0.0 if bias is None else bias.double())
    if c["groups"] > 1:
        by = key.masked_fill(closed, -math.inf).view(len(l), c["groups"], -1)
        best = torch.sort(by, dim=2, descending=True).values[..., :2]
        group_key = best[..., 0] + torch.where(best[..., 1:] == -math.inf, 0.0, best[..., 1:]).sum(-1)
        chosen = torch.sort(group_key, dim=1, descending=True, stable=True).indices[:, : c["top_groups"]]
        stays = torch.zeros_like(group_key, dtype=torch.bool).scatter_(1, chosen, True)
        closed = closed | ~stays.repeat_interleave(by.shape[2], dim=1)
    if bias is None:
        key = l                                    # the same order as the scores', which rises with them
    ids = torch.sort(key.masked_fill(closed, -math.inf), dim=1, descending=True, stable=True).indices[:, : c["k"]]
    there = ~closed.gather(1, ids)
    p = _plain_scores(l, c["score"]).gather(1, ids) * there
    total = p.sum(dim=1, keepdim=True)
    weights = c["scale"] * (p / torch.where(total == 0, 1.0, total) if c["renorm"] else p)
    return torch.where(there, ids, -1).to(torch.int32), weights


def _plain_topk_grad(c, logits, ids, dweights):
    l = logits.float()
    p = _plain_scores(l, c["score"])
    there = ids >= 0
    at = ids.clamp(min=0).long()
    dw = c["scale"] * dweights * there
    sel = p.gather(1, at) * there
    total = sel.sum(dim=1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    dsel = (dw - (dw * sel).sum(dim=1, keepdim=True) / total) / total * there if c["renorm"] else dw
    dp = torch.zeros_like(p).scatter_add_(1, at, dsel)
    dl = dp * p * (1 - p) if c["score"] == "sigmoid" else p * (dp - (dp * p).sum(dim=1, keepdim=True))
    return dl.to(logits.dtype)


def _plain_plan(ids, E):
    order = torch.sort(ids.reshape(-1), stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, ids.reshape(-1).long() + 1, torch.ones_like(order))
    return order, counts.cumsum(0)


def _plain_experts(x, order, offsets, of_pair, w):
    """Row x[of_pair[p]] times the matrix of pair p's expert, for every pair p: the rows of each expert in a slab of their own."""
    counts = offsets[1:] - offsets[:-1]
    expert = torch.repeat_interleave(torch.arange(len(counts), device=x.device), counts)
    place = torch.arange(len(order), device=x.device) - offsets[expert]
    slabs = torch.zeros((len(counts), int(counts.max()), x.shape[1]), device=x.device)
    slabs[expert, place] = x[of_pair[order]]
    y = torch.empty((len(order), w.shape[1]), device=x.device)
    y[order] = torch.bmm(slabs, w.transpose(1, 2).contiguous())[expert, place]
    return y


def _plain_gated(y):
    gate, up = y.chunk(2, dim=1)
    return gate / (1 + torch.exp(-gate)) * up


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    op = c["op"]
    if op in ("topk", "layer"):
        ids, weights = _plain_topk(c, s["logits"], s["bias"])
    if op == "topk":
        r = dict(ids=ids, weights=weights)
        if c["train"]:
            r["dlogits"] = _plain_topk_grad(c, s["logits"], ids, s["dweights"])
        return r
    if op == "plan":
        order, offsets = _plain_plan(s["ids"], c["E"])
        return dict(order=order.to(torch.int32), offsets=offsets.to(torch.int32))
    if op == "mm":
        return (s["x"].float() @ _plain_matrices(s["up"], c["g"])[0].t()).to(TYPES[c["out"]])
    if op == "combine":
        y, dout, w = s["y"].float().view(c["T"], c["k"], -1), s["dout"].float(), s["weights"]
        return dict(out=(w[..., None] * y).sum(1).to(s["y"].dtype), dy=(w[..., None] * dout[:, None]).flatten(0, 1).to(s["y"].dtype),
                    dweights=(y * dout[:, None]).sum(2))
    if op == "experts":
        ids = s["ids"]
    used, of_used = torch.unique(ids, return_inverse=True)       # only the matrices that a row goes to
    order, offsets = _plain_plan(of_used, len(used))
    pairs = torch.arange(c["T"] * c["k"], device=DEV)
    h = _plain_gated(_plain_experts(s["x"].float(), order, offsets, pairs // c["k"], _plain_matrices(_of_experts(s["up"], used), c["g"])))
    if op == "experts":
        return h.to(s["x"].dtype)
    y = _plain_experts(h, order, offsets, pairs, _plain_matrices(_of_experts(s["down"], used), c["g"]))
    out = (weights[..., None] * y.view(c["T"], c["k"], -1)).sum(1)
    return dict(out=out.to(s["x"].dtype), ids=ids)


# ------------------------------------------------------------------------------------------- what a pass cannot do without
def _touched(T, E, k):
    """Experts that T rows with k of E each reach, about."""
    return min(E, max(k, round(E * (1 - (1 - k / E) ** T))))


def _matrix_bytes(rows, cols, g, zeros):
    return rows * cols / 2 + rows * -(-cols // g) * (3 if zeros else 2)


def work(case):
    c, op, T = case, case["op"], case["T"]
    if op == "topk":
        size = 4 if c["dtype"] == "f32" else 2
        again = 2 * size * T * c["E"] + 8 * T * c["k"] if c["train"] else 0            # the gradient's pass: scores in, gradient out
        return dict(bytes=size * T * c["E"] + 8 * T * c["k"] + again, flops=(20 if c["train"] else 10) * T * c["E"])
    if op == "plan":
        return dict(bytes=8 * T * c["k"] + 4 * c["E"] + 4, flops=T * c["k"])
    if op == "mm":
        return dict(bytes=_matrix_bytes(c["N"], c["K"], c["g"], c["zeros"]) + 2 * T * c["K"] + (4 if c["out"] == "f32" else 2) * T * c["N"],
                    flops=2 * T * c["N"] * c["K"])
    if op == "combine":
        return dict(bytes=T * c["D"] * (2 * c["k"] + 2) + T * c["D"] * (4 * c["k"] + 2) + 16 * T * c["k"], flops=5 * T * c["k"] * c["D"])
    P = T * c["k"]
    up = dict(bytes=_touched(T, c["E"], c["k"]) * _matrix_bytes(2 * c["F"], c["K"], c["g"], c["zeros"]) + 2 * T * c["K"] + 2 * P * c["F"],
              flops=4 * P * c["K"] * c["F"])
    if op == "experts":
        return up
    return dict(bytes=up["bytes"] - 2 * P * c["F"] + _touched(T, c["E"], c["k"]) * _matrix_bytes(c["K"], c["F"], c["g"], c["zeros"]) + 2 * T * c["K"]
                + 4 * T * c["E"] + 8 * P, flops=up["flops"] + 2 * P * c["K"] * c["F"])


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_matrix(q, e, g):
    codes, scales, zeros = (None if t is None else t[e].cpu().numpy() if t.dtype == torch.uint8 else t[e].double().cpu().numpy() for t in q)
    w = np.empty((codes.shape[0], 2 * codes.shape[1]))
    w[:, 0::2], w[:, 1::2] = codes % 16, codes // 16
    group = np.arange(w.shape[1]) // g
    w -= 8 if zeros is None else zeros.astype(np.float64)[:, group]
    return torch.from_numpy(w * scales[:, group]).to(DEV)


def _exact_choice(c, logits, bias):
    """Ids, weights and the Jacobians' ingredients, row by row."""
    L, T, k = logits.double().cpu().numpy(), c["T"], c["k"]
    b = np.zeros(c["E"]) if bias is None else bias.double().cpu().numpy()
    ids, weights, scores = np.full((T, k), -1, np.int32), np.zeros((T, k)), np.zeros((T, c["E"]))
    size = c["E"] // c["groups"]
    for t in range(T):
        l = L[t]
        open_ = np.nonzero(l > -np.inf)[0]
        if not len(open_):
            continue
        if c["score"] == "softmax":
            e = np.exp(l[open_] - l[open_].max())
            scores[t, open_] = e / e.sum()
        else:
            scores[t, open_] = 1 / (1 + np.exp(-l[open_]))
        key = scores[t] + b
        if c["groups"] > 1:
            of_group = [np.sort(key[open_[open_ // size == j]])[::-1][:2] for j in range(c["groups"])]
            best = sorted((j for j in range(c["groups"]) if len(of_group[j])), key=lambda j: (-of_group[j].sum(), j))[: c["top_groups"]]
            open_ = open_[np.isin(open_ // size, best)]
        order = l if bias is None else key
        mine = open_[np.argsort(-order[open_], kind="stable")][:k]
        ids[t, : len(mine)] = mine
        weights[t, : len(mine)] = c["scale"] * scores[t, mine] / (scores[t, mine].sum() if c["renorm"] else 1)
    return ids, weights, scores


def _exact_choice_grad(c, ids, scores, dweights):
    d = dweights.double().cpu().numpy()
    out = np.zeros_like(scores)
    for t in range(c["T"]):
        mine = ids[t][ids[t] >= 0]
        if not len(mine):
            continue
        s, ds = scores[t], c["scale"] * d[t, : len(mine)]
        if c["renorm"]:
            ds = ds / s[mine].sum() - (ds @ s[mine]) / s[mine].sum() ** 2
        wide = np.zeros_like(s)
        wide[mine] = ds
        out[t] = wide * s * (1 - s) if c["score"] == "sigmoid" else s * wide - s * (s @ wide)
    return out


def exact(case, seed):
    c, s = case, _data(case, seed)
    op = c["op"]
    if op in ("topk", "layer"):
        ids, weights, scores = _exact_choice(c, s["logits"], s["bias"])
        if op == "topk":
            r = dict(ids=ids, weights=weights)
            if c["train"]:
                r["dlogits"] = _exact_choice_grad(c, ids, scores, s["dweights"])
            return r
    if op == "plan":
        flat = s["ids"].cpu().numpy().reshape(-1)
        return dict(order=np.argsort(flat, kind="stable").astype(np.int32), offsets=np.searchsorted(np.sort(flat), np.arange(c["E"] + 1)).astype(np.int32))
    if op == "mm":
        return s["x"].double() @ _exact_matrix(s["up"], 0, c["g"]).t()
    if op == "combine":
        y, w, dout = s["y"].double().view(c["T"], c["k"], -1), s["weights"].double(), s["dout"].double()
        out = torch.zeros_like(dout)
        dy, dw = torch.empty_like(y), torch.empty_like(w)
        for j in range(c["k"]):
            out += w[:, j, None] * y[:, j]
            dy[:, j] = w[:, j, None] * dout
            dw[:, j] = torch.linalg.vecdot(y[:, j], dout)
        return dict(out=out, dy=dy.flatten(0, 1), dweights=dw)
    if op == "experts":
        ids = s["ids"].cpu().numpy()
    x = s["x"].double()
    h = torch.zeros((c["T"] * c["k"], c["F"]), dtype=torch.float64, device=DEV)
    out = torch.zeros_like(x)
    for e in range(c["E"]):
        t, j = (torch.from_numpy(v).to(DEV) for v in np.nonzero(ids == e))
        if not len(t):
            continue
        y = x[t] @ _exact_matrix(s["up"], e, c["g"]).t()
        mine = torch.sigmoid(y[:, : c["F"]]) * y[:, : c["F"]] * y[:, c["F"]:]
        if op == "experts":
            h[t * c["k"] + j] = mine
        else:
            out.index_add_(0, t, (mine @ _exact_matrix(s["down"], e, c["g"]).t()) * torch.from_numpy(weights).to(DEV)[t, j, None])
    return h if op == "experts" else dict(out=out, ids=ids)
