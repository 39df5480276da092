"""Routed products and products with matrices in 4 bits, against their definitions in 64 bits.

Tolerances count roundings.  U = 2^-24 is half a step of fp32; a result kept in type t is off by half a step of t more.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2202_05868_amd import binding, routed

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(t):
    return torch.finfo(t).eps / 2


def np64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------- definitions, in 64 bits
def choice(l, k, score, bias, n_groups, top_groups, renorm, scale):
    """ids, weights and scores of raw scores `l` [T, E] (float64 numpy; NaN and -inf close an expert)."""
    T, E = l.shape
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, float(np.finfo(np.float32).max)))
    ids, weights, scores = np.full((T, k), -1, np.int64), np.zeros((T, k)), np.zeros((T, E))
    size = E // n_groups
    for t in range(T):
        open_ = [e for e in range(E) if l[t, e] > -np.inf and (bias is None or bias[e] > -np.inf)]
        closed = l[t] == -np.inf
        if closed.all():
            continue
        with np.errstate(under="ignore", over="ignore"):
            if score == "softmax":
                x = np.exp(l[t] - l[t].max())
                scores[t] = x / x.sum()
            else:
                scores[t] = np.where(closed, 0.0, 1 / (1 + np.exp(-l[t])))
        key = scores[t] + (0 if bias is None else bias)
        if n_groups > 1:
            best = {}
            for e in open_:
                best.setdefault(e // size, []).append(key[e])
            stays = sorted(best, key=lambda g: (-sum(sorted(best[g])[-2:]), g))[:top_groups]
            open_ = [e for e in open_ if e // size in stays]
        order = l[t] if bias is None else key
        mine = sorted(open_, key=lambda e: (-order[e], e))[:k]
        ids[t, : len(mine)] = mine
        weights[t] = weights_of(l[t], scores[t], ids[t], score, renorm, scale)
    return ids, weights, scores


def weights_of(l, s, ids, score, renorm, scale):
    """scale * score, or scale * score / sum of the scores: from their logarithms, so that the quotient has a value where the scores have none."""
    there = ids >= 0
    w = np.zeros(len(ids))
    if there.any():
        mine = ids[there]
        if renorm:
            log_s = l[mine] if score == "softmax" else np.minimum(l[mine], 0) - np.log1p(np.exp(-np.abs(l[mine])))
            x = np.exp(log_s - log_s.max())
            w[there] = scale * x / x.sum()
        else:
            w[there] = scale * s[mine]
    return w


def choice_grad(l, ids, dw, score, renorm, scale):
    """The gradient of sum(dw * weights) to l, by the formulas' Jacobians; ids may repeat."""
    T, E = l.shape
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, float(np.finfo(np.float32).max)))
    out = np.zeros((T, E))
    for t in range(T):
        place = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E and l[t, ids[t, j]] > -np.inf]
        if not place:
            continue
        e, d = ids[t, place], dw[t, place] * scale
        x = np.exp(l[t] - l[t].max())
        s = x / x.sum() if score == "softmax" else np.where(l[t] == -np.inf, 0.0, 1 / (1 + np.exp(-l[t])))
        ds = np.zeros(E)
        if renorm:
            total = s[e].sum()
            np.add.at(ds, e, d / total - (d * s[e]).sum() / total ** 2)
        else:
            np.add.at(ds, e, d)
        common = 0.0 if renorm else (s * ds).sum()                          # renormalised, the sum is zero: d_j - sum d s / total, times s_j / total, over j
        out[t] = s * (ds - common) if score == "softmax" else ds * s * (1 - s)
    return out


def matrices(gen, M, N, K, group, dtype, zeros):
    G = -(-K // group)
    codes = torch.randint(0, 256, (M, N, K // 2), generator=gen, dtype=torch.uint8)
    scales = ((torch.rand((M, N, G), generator=gen) + 0.5) * torch.where(torch.rand((M, N, G), generator=gen) < 0.1, -0.02, 0.02)).to(dtype)
    z = torch.randint(0, 16, (M, N, G), generator=gen, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def product(x, q, m, group):
    """x W^T of matrix m, and its bound: what the fp32 sums of a group of at most 128 columns (4 steps of 32 products, each product exact, the sum of x
    likewise) and the sums over such groups can be off by, at two half steps an addition."""
    codes, scales, zeros = q
    c = np.empty((codes.shape[1], 2 * codes.shape[2]))
    raw = codes[m].numpy()
    c[:, 0::2], c[:, 1::2] = raw & 15, raw >> 4
    K = c.shape[1]
    at = np.arange(K) // group
    s, z = np64(scales[m])[:, at], (np.full(c.shape, 8.0) if zeros is None else zeros[m].numpy().astype(np.float64)[:, at])
    w = s * (c - z)
    y = x @ w.T
    piece = min(group, 128)
    inside = np.abs(x) @ (np.abs(s) * (32 + c + z)).T
    outside = sum(np.abs(x[:, b: b + piece] @ w[:, b: b + piece].T) for b in range(0, K, piece))
    steps = -(-K // piece) + 8
    return y, 2 * U * (40 * inside + steps * outside)


def gated(y, tol):
    F = y.shape[1] // 2
    g, u, tg, tu = y[:, :F], y[:, F:], tol[:, :F], tol[:, F:]
    silu = g / (1 + np.exp(-g))
    return silu * u, 1.1 * tg * (np.abs(u) + tu) + np.abs(silu) * tu + 8 * U * np.abs(silu * u)      # |silu'| < 1.1; exp, sum, quotient, product


def assert_close(got, want, tol, dtype):
    got = np64(got)
    limit = tol + half_step(dtype) * (np.abs(want) + tol) + (2.0 ** -25 if dtype is torch.float16 else 0)        # below fp16's normal numbers steps are 2^-24
    bad = ~(np.abs(got - want) <= limit)
    assert not bad.any(), "%d of %d off, worst by %g of the limit" % (bad.sum(), bad.size, np.nanmax(np.abs(got - want) / limit))


# ------------------------------------------------------------------------------------------- the choice
CHOICES = [
    # T, E, k, type, score, bias, groups, top_groups, renorm, scale
    (1, 1, 1, "f32", "softmax", False, 1, 1, True, 1.0),
    (3, 5, 5, "bf16", "softmax", False, 1, 1, False, 2.5),
    (1, 64, 4, "bf16", "softmax", False, 1, 1, True, 1.0),
    (7, 60, 6, "f16", "sigmoid", True, 4, 2, True, 2.5),
    (33, 65, 8, "f32", "softmax", True, 1, 1, False, 1.0),
    (130, 128, 8, "bf16", "sigmoid", False, 8, 3, False, 1.5),
    (65, 160, 6, "f32", "softmax", False, 8, 4, True, 1.0),
    (257, 256, 8, "f32", "sigmoid", True, 8, 4, True, 2.5),
    (20, 300, 10, "bf16", "softmax", True, 1, 1, True, 1.0),
    (9, 1024, 64, "f32", "sigmoid", True, 64, 9, True, 1.0),
    (5, 515, 33, "f16", "softmax", False, 1, 1, False, 1.0),
    (11, 16, 16, "f32", "sigmoid", False, 16, 16, True, 1.0),
]


def raw_scores(seed, T, E, dtype):
    """Scores with ties, closed experts, rows without any, the lowest finite number, infinities and NaN in some rows."""
    gen = torch.Generator().manual_seed(seed)
    l = 2 * torch.randn((T, E), generator=gen)
    l = torch.where(torch.rand((T, E), generator=gen) < 0.3, (l * 2).round() / 2, l).to(TYPES[dtype])          # ties
    kind = torch.randint(0, 8, (T, 1), generator=gen)
    some = torch.rand((T, E), generator=gen) < 0.4
    l = torch.where((kind == 1) & some, torch.tensor(-math.inf, dtype=l.dtype), l)
    l = torch.where((kind == 2) & some, torch.tensor(torch.finfo(l.dtype).min, dtype=l.dtype), l)
    l = torch.where((kind == 3) & some, torch.tensor(math.nan, dtype=l.dtype), l)
    if T > 4:
        l[2] = -math.inf
        l[3] = torch.finfo(l.dtype).min
        l[4, 0] = math.inf
    return l


@pytest.mark.gpu
@pytest.mark.parametrize("case", CHOICES, ids=lambda c: "T%d-E%d-k%d-%s-%s" % c[:5])
def test_choice_and_weights(case):
    T, E, k, dtype, score, with_bias, n_groups, top_groups, renorm, scale = case
    l = raw_scores(T + E, T, E, dtype)
    bias = 0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E)) if with_bias else None
    if with_bias and E > 70:
        bias[3], bias[64] = -math.inf, math.nan
    want_ids, want, _ = choice(np64(l), k, score, None if bias is None else np.nan_to_num(np64(bias), nan=-math.inf, neginf=-math.inf), n_groups, top_groups, renorm, scale)
    wide = torch.full((T, E + 3), 7.0, dtype=l.dtype, device=DEV)           # rows behind each other with a gap
    wide[:, :E] = l.to(DEV)
    for on in (l.to(DEV), wide[:, :E]):
        ids, weights = routed.route_topk(on, k, score=score, bias=None if bias is None else bias.to(DEV), n_groups=n_groups, top_groups=top_groups, renormalise=renorm,
                                         scale=scale)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        got = np64(weights)
        # exp's argument is off by a step of its size (below 90, or the exponential is nothing), sums of E positive numbers by 80 additions in a row at most
        spread = np.minimum(90, np.nan_to_num(np.abs(np64(l)), nan=0, posinf=0, neginf=0).max(axis=1, keepdims=True) * 2)
        assert np.all(np.abs(got - want) <= U * (2 * spread + 80) * want + 1e-37)


def many_rows(seed, T, E, dtype):
    """Scores of many rows, some so near each other that 32 bits do not tell their sums with a bias apart, some rows with closed experts or without any."""
    gen = torch.Generator().manual_seed(seed)
    l = 1.5 * torch.randn((T, E), generator=gen)
    near = torch.rand((T, 1), generator=gen) < 0.2
    l = torch.where(near, l[:, :1] * (1 + 1e-7 * torch.randint(-3, 4, (T, E), generator=gen)), l)
    l = torch.where(torch.rand((T, E), generator=gen) < 0.05, torch.tensor(-math.inf), l)
    l[T // 3: T // 3 + 3] = -math.inf
    return l.to(TYPES[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4095, 4096, 5001])
@pytest.mark.parametrize("E,k,dtype,score,bias_step,groups,top_groups,renorm", [
    (256, 8, "f32", "sigmoid", 2.0 ** -24, 8, 4, True), (256, 8, "f32", "softmax", 2.0 ** -26, 8, 3, False), (128, 8, "bf16", "softmax", None, 1, 1, True),
    (240, 10, "f16", "sigmoid", 0.1, 8, 5, True), (16, 3, "f32", "softmax", None, 4, 2, False), (100, 16, "bf16", "sigmoid", 0.0, 1, 1, False), (60, 1, "f32", "sigmoid", None, 1, 1, True),
    (33, 5, "f16", "softmax", 2.0 ** -20, 3, 2, True), (256, 4, "bf16", "sigmoid", 0.1, 16, 16, True)])
def test_choice_of_many_rows(T, E, k, dtype, score, bias_step, groups, top_groups, renorm):
    l = many_rows(E, T, E, dtype)
    bias = None if bias_step is None else bias_step * torch.randn(E, generator=torch.Generator().manual_seed(E))
    ids, weights = routed.route_topk(l.to(DEV), k, score=score, bias=None if bias is None else bias.to(DEV), n_groups=groups, top_groups=top_groups, renormalise=renorm, scale=1.5)
    # the definition, all rows at once
    x = np64(l)
    closed = x == -np.inf
    if score == "softmax":
        most = x.max(1, keepdims=True)
        e = np.exp(x - np.where(most == -np.inf, 0, most))
        s = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
    else:
        s = np.where(closed, 0, 1 / (1 + np.exp(-x)))
    key = s + (0 if bias is None else np64(bias))
    out = closed.copy()
    if groups > 1:
        by = -np.sort(-np.where(closed, -np.inf, key).reshape(T, groups, -1), 2)[:, :, :2]
        total = by[:, :, 0] + np.where(by[:, :, -1] == -np.inf, 0, by[:, :, -1]) * (by.shape[2] > 1)
        stays = np.argsort(-total, 1, kind="stable")[:, :top_groups]
        mask = np.zeros((T, groups), bool)
        np.put_along_axis(mask, stays, True, 1)
        out |= ~np.repeat(mask, E // groups, 1)
    order = x if bias is None else key
    want = np.argsort(-np.where(out, -np.inf, order), 1, kind="stable")[:, :k]
    want = np.where(np.take_along_axis(out, want, 1), -1, want)
    assert np.array_equal(ids.cpu().numpy(), want)
    w = np.where(want >= 0, np.take_along_axis(s, np.maximum(want, 0), 1), 0)
    if renorm:
        w = w / np.maximum(w.sum(1, keepdims=True), 1e-300)
    spread = np.where(closed, 0, np.abs(x)).max(1, keepdims=True) * 2
    assert np.all(np.abs(np64(weights) - 1.5 * w) <= U * (2 * spread + 80) * 1.5 * w)


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k,dtype,score,renorm", [(4096, 128, 8, "bf16", "softmax", True), (5001, 256, 16, "f32", "sigmoid", True), (4500, 60, 3, "f16", "softmax", False), (4099, 130, 2, "f32", "sigmoid", False)])
def test_gradient_of_many_rows(T, E, k, dtype, score, renorm):
    l = many_rows(E, T, E, dtype)
    gen = torch.Generator().manual_seed(2)
    ids = torch.randint(-1, E + 1, (T, k), generator=gen, dtype=torch.int32)
    dw = torch.randn((T, k), generator=gen)
    got = np64(routed.route_topk_grad(l.to(DEV), ids.to(DEV), dw.to(DEV), score=score, renormalise=renorm, scale=1.5))
    rows = np.r_[0:40, T // 3 - 2: T // 3 + 6, T - 40: T]
    l64, i64, d64 = np64(l)[rows], ids.numpy().astype(np.int64)[rows], np64(dw)[rows]
    want = choice_grad(l64, i64, d64, score, renorm, 1.5)
    # every term of the gradient is at most 1.5 |dw| (weights and their derivatives are at most 1)
    limit = U * 400 * 1.5 * np.abs(d64).sum(1, keepdims=True)
    assert np.all(np.abs(got[rows] - want) <= limit + half_step(l.dtype) * (np.abs(want) + limit) + (2.0 ** -25 if dtype == "f16" else 0))
    other = torch.from_numpy(rows)
    few = routed.route_topk_grad(l[other].to(DEV), ids[other].to(DEV), dw[other].to(DEV), score=score, renormalise=renorm, scale=1.5)
    assert np.all(np.abs(np64(few) - got[rows]) <= 2 * (limit + half_step(l.dtype) * (np.abs(want) + limit) + (2.0 ** -25 if dtype == "f16" else 0)))


def test_gradient_of_the_choice_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    for score in ("softmax", "sigmoid"):
        for renorm in (False, True):
            l, dw = rng.normal(size=(4, 9)), rng.normal(size=(4, 3))
            ids = np.stack([rng.permutation(9)[:3] for _ in range(4)])
            ids[1, 2] = -1
            ids[2, 1] = ids[2, 0]

            def total(l):
                s = np.exp(l) / np.exp(l).sum(1, keepdims=True) if score == "softmax" else 1 / (1 + np.exp(-l))
                return sum((dw[t] * weights_of(l[t], s[t], ids[t], score, renorm, 1.5)).sum() for t in range(4))

            g, h = choice_grad(l, ids, dw, score, renorm, 1.5), 1e-6
            for t in range(4):
                for e in range(9):
                    d = np.zeros_like(l)
                    d[t, e] = h
                    assert abs((total(l + d) - total(l - d)) / (2 * h) - g[t, e]) < 1e-8


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 64, 4, "f32"), (70, 128, 8, "bf16"), (37, 37, 5, "f16"), (6, 1000, 64, "f32"), (9, 300, 3, "bf16"), (2, 1, 1, "f32")])
def test_gradient_of_the_choice(T, E, k, dtype, score, renorm):
    l = raw_scores(T * E, T, E, dtype)
    if T > 4:
        l[4, 0] = 9.0                                                      # (an infinite score has no difference quotient)
        l[3] = -2.0
        l = torch.where(l == torch.finfo(l.dtype).min, torch.tensor(-20.0, dtype=l.dtype), l)
    gen = torch.Generator().manual_seed(1)
    ids = torch.stack([torch.randperm(E, generator=gen)[:k] for _ in range(T)]).to(torch.int32)
    if T > 6 and k > 2:
        ids[5, 1], ids[6, 0], ids[6, 2], ids[1, 0] = -1, ids[6, 1], E, 2 ** 30      # none, twice, out of range
    dw = torch.randn((T, k), generator=gen)
    got = routed.route_topk_grad(l.to(DEV), ids.to(DEV), dw.to(DEV), score=score, renormalise=renorm, scale=1.5)
    assert got.dtype is l.dtype
    l64, i64, d64 = np64(l), ids.numpy().astype(np.int64), np64(dw)
    want = choice_grad(l64, i64, d64, score, renorm, 1.5)
    size = np.zeros((T, E))                                                # of the terms that the gradient is a difference of
    for t in range(T):
        lt = np.where(np.isnan(l64[t]), -np.inf, l64[t])
        place = [j for j in range(k) if 0 <= i64[t, j] < E and lt[i64[t, j]] > -np.inf]
        if not place:
            continue
        e, d = i64[t, place], np.abs(d64[t, place]) * 1.5
        x = np.exp(lt - lt.max())
        s = x / x.sum() if score == "softmax" else np.where(lt == -np.inf, 0.0, 1 / (1 + np.exp(-lt)))
        total = s[e].sum() if renorm else 1.0
        r = s / total
        common = (d * r[e]).sum()
        np.add.at(size[t], e, r[e] * (d + (common if renorm else 0.0)))
        if score == "softmax" and not renorm:
            size[t] += s * common
    spread = np.nan_to_num(np.abs(l64), nan=0, posinf=0, neginf=0).max(axis=1, keepdims=True) * 2
    assert_close(got, want, U * (4 * spread + 200) * size, l.dtype)


# ------------------------------------------------------------------------------------------- the grouping
PLANS = [(1, 1, 1), (4097, 2, 1000), (70000, 2, 17), (1023, 4, 3), (1, 4, 7), (5, 3, 64), (64, 1, 1), (100, 8, 256), (257, 6, 60), (4096, 2, 1024), (3000, 8, 5), (0, 2, 8), (20000, 4, 300)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,E", PLANS)
@pytest.mark.parametrize("kind", ["spread", "one", "holes"])
def test_plan_is_the_stable_sort(T, k, E, kind):
    rng = np.random.default_rng(T + E)
    ids = rng.integers(0, E, size=(T, k))
    if kind == "one":
        ids[:] = E - 1
    if kind == "holes":
        ids = np.where(rng.random((T, k)) < 0.3, rng.choice([-1, E, -(2 ** 31), 2 ** 31 - 1], size=(T, k)), ids)
        ids[T // 2:] = -1
    plan = routed.route_plan(torch.from_numpy(ids.astype(np.int32)).to(DEV), E)
    flat = ids.reshape(-1)
    pairs = np.nonzero((flat >= 0) & (flat < E))[0]
    order = pairs[np.argsort(flat[pairs], kind="stable")]
    offsets = np.searchsorted(flat[order], np.arange(E + 1))
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    got = plan.order.cpu().numpy()
    assert np.array_equal(got[: len(order)], order) and np.all(got[len(order):] == -1)


# ------------------------------------------------------------------------------------------- products
MM = [
    # T, N, K, group, type, zeros, gated
    (1, 64, 128, 128, "bf16", False, False),
    (1, 1, 32, 32, "f16", True, False),
    (5, 17, 96, 32, "bf16", True, False),
    (16, 40, 160, 64, "f16", False, False),
    (17, 130, 416, 128, "bf16", True, False),
    (33, 2, 1056, 256, "f16", True, True),
    (3, 70, 1024, 32, "bf16", False, True),
    (70, 96, 800, 64, "bf16", True, True),
    (64, 48, 2048, 2048, "f16", False, False),
    (2, 4098, 4096, 128, "bf16", True, True),
    (130, 515, 640, 384, "f16", True, False),
    (200, 258, 320, 32, "f16", True, True),
    (300, 272, 2080, 128, "bf16", False, False),
    (257, 64, 8192, 64, "bf16", True, False),
]


# as many rows and outputs as fill the GPU
MM_FULL = [
    (1000, 3600, 32, 32, "f16", True, False),
    (900, 4098, 160, 64, "bf16", False, True),
    (961, 3700, 288, 128, "bf16", True, False),
    (1024, 3585, 416, 256, "f16", False, False),
    (31, 57400, 96, 32, "bf16", False, False),
    (20, 57360, 320, 64, "f16", True, True),
    (32, 57344, 640, 128, "bf16", True, False),
    (700, 6000, 256, 32, "bf16", True, True),
    (16, 20000, 1100 // 32 * 32, 128, "f16", True, False),
    (10, 12000, 2304, 64, "bf16", True, True),
    (3, 33000, 576, 32, "bf16", False, False),
    (64, 16384, 2048, 128, "f16", False, False),
    (100, 9000, 160, 64, "bf16", True, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", MM + MM_FULL, ids=lambda c: "T%d-N%d-K%d-g%d-%s-z%d-gated%d" % c)
@pytest.mark.parametrize("out", ["same", "f32"])
def test_products_with_one_matrix(case, out):
    T, N, K, group, dtype, zeros, gate = case
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(T + N)
    q = matrices(gen, 1, N, K, group, t, zeros)
    x = torch.randn((T, K), generator=gen).to(t)
    want, tol = product(np64(x), q, 0, group)
    if gate:
        want, tol = gated(want, tol)
    y_type = t if out == "same" else torch.float32
    m = routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=gate).upload()
    assert_close(m.mm(x.to(DEV), y_dtype=y_type), want, tol, y_type)
    # rows with gaps, and what lies between and behind them stays
    wide = torch.full((T, K + 24), math.nan, dtype=t, device=DEV)
    wide[:, 8: 8 + K] = x.to(DEV)
    y = torch.full((T + 2, m.n_out + 5), 7.0, dtype=y_type, device=DEV)
    m.mm(wide[:, 8: 8 + K], y[1: T + 1, 3: 3 + m.n_out])
    assert_close(y[1: T + 1, 3: 3 + m.n_out], want, tol, y_type)
    assert bool((y[0] == 7).all()) and bool((y[T + 1] == 7).all()) and bool((y[:, :3] == 7).all()) and bool((y[:, 3 + m.n_out:] == 7).all())


# on both sides of where tiles of 16, 32 and 64 rows begin
@pytest.mark.gpu
@pytest.mark.parametrize("T,N,K,group,dtype,zeros,gate", [
    (17, 520, 96, 32, "bf16", True, False), (33, 8176, 160, 64, "f16", False, False), (48, 5456, 288, 128, "bf16", True, True), (64, 4097, 416, 32, "f16", True, False),
    (1024, 256, 1056, 128, "bf16", True, False), (1025, 256, 96, 64, "f16", True, True), (40, 16384, 224, 128, "bf16", False, False), (40, 16400, 224, 32, "bf16", True, False),
    (96, 11000, 160, 64, "bf16", True, True), (97, 11000, 160, 64, "f16", True, False), (65, 20000, 64, 32, "f16", False, False), (512, 2048, 2080, 256, "bf16", True, False),
    (513, 2048, 544, 128, "f16", False, True), (160, 6144, 640, 128, "bf16", True, False), (48, 4000, 288, 32, "bf16", True, False),
    (33, 4180, 416, 32, "f16", False, True), (12, 12000, 288, 32, "f16", True, True)])
def test_products_where_tiles_change(T, N, K, group, dtype, zeros, gate):
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(T + N)
    q = matrices(gen, 1, N, K, group, t, zeros)
    x = torch.randn((T, K), generator=gen).to(t)
    want, tol = product(np64(x), q, 0, group)
    if gate:
        want, tol = gated(want, tol)
    m = routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=gate).upload()
    y = torch.full((T + 1, m.n_out), 7.0, dtype=torch.float32, device=DEV)
    m.mm(x.to(DEV), y[:T])
    assert_close(y[:T], want, tol, torch.float32)
    assert bool((y[T] == 7).all())


ROUTED = [
    # T, k, E, N, K, group, type, zeros, gated
    (1, 1, 1, 16, 32, 32, "f16", False, False),
    (1, 4, 9, 66, 256, 64, "bf16", True, True),
    (16, 4, 64, 34, 160, 32, "bf16", False, True),
    (7, 2, 3, 50, 416, 128, "f16", True, False),
    (100, 3, 5, 130, 640, 256, "bf16", True, True),
    (300, 2, 4, 96, 288, 128, "f16", False, False),
    (513, 1, 2, 32, 1024, 32, "bf16", True, False),
    (40, 8, 130, 20, 96, 32, "f16", True, False),
    (600, 4, 8, 258, 544, 128, "bf16", True, True),
    (400, 4, 64, 1026, 160, 32, "f16", True, True),
    (2000, 4, 64, 514, 288, 128, "bf16", True, False),
    (2000, 4, 64, 514, 224, 64, "f16", False, True),
    (250, 4, 60, 700, 160, 64, "bf16", False, False),
    (60, 4, 40, 2064, 800, 64, "bf16", False, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", ROUTED, ids=lambda c: "T%d-k%d-E%d-N%d-K%d-g%d-%s-z%d-gated%d" % c)
@pytest.mark.parametrize("a_pair", [False, True])
@pytest.mark.parametrize("kind", ["spread", "one", "holes"])
def test_routed_products(case, a_pair, kind):
    T, k, E, N, K, group, dtype, zeros, gate = case
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(T + N)
    q = matrices(gen, E, N, K, group, t, zeros)
    x = torch.randn((T * k if a_pair else T, K), generator=gen).to(t)
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    if kind == "one":
        ids[:] = E - 1
    if kind == "holes":
        ids = torch.where(torch.rand((T, k), generator=gen) < 0.4, torch.tensor(-1 if T % 2 else E, dtype=torch.int32), ids)
    m = routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=gate).upload()
    plan = routed.route_plan(ids.to(DEV), E)
    y_type = torch.float32 if a_pair else t
    y = torch.full((T * k, m.n_out), 7.0, dtype=y_type, device=DEV)
    m.mm_routed(x.to(DEV), plan, y)
    flat = ids.reshape(-1).numpy()
    x64 = np64(x)
    if not a_pair:
        x64 = np.repeat(x64, k, axis=0)
    want, tol = np.full((T * k, m.n_out), 7.0), np.zeros((T * k, m.n_out))
    for e in range(E):
        at = np.nonzero(flat == e)[0]
        if len(at):
            a, b = product(x64[at], q, e, group)
            want[at], tol[at] = gated(a, b) if gate else (a, b)
    assert_close(y, want, tol, y_type)


# as many tiles and columns as fill the GPU: experts of many tiles and of few, tiles that most of the plan's places are not needed for
@pytest.mark.gpu
@pytest.mark.parametrize("T,k,E,N,K,group,dtype,zeros,gate", [
    (2400, 1, 3, 3000, 64, 32, "f16", True, False), (2000, 4, 100, 2100, 96, 64, "bf16", False, True), (800, 4, 200, 1500, 160, 128, "bf16", True, False),
    (300, 4, 24, 4100, 1056, 128, "f16", False, True), (100, 4, 24, 4100, 288, 32, "bf16", True, False),
    # tiles of the plan that the product takes whole, in halves and in quarters
    (400, 2, 4, 1280, 160, 64, "f16", True, False), (700, 2, 7, 1300, 1056, 128, "bf16", True, True), (700, 2, 7, 700, 160, 32, "bf16", False, False),
    (200, 2, 4, 320, 288, 128, "bf16", True, True), (60, 2, 4, 320, 2080, 256, "f16", False, False)])
@pytest.mark.parametrize("kind", ["spread", "few", "none"])
def test_routed_products_that_fill(T, k, E, N, K, group, dtype, zeros, gate, kind):
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(T + N)
    q = matrices(gen, E, N, K, group, t, zeros)
    x = torch.randn((T, K), generator=gen).to(t)
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    if kind == "few":
        ids = torch.where(ids % 3 == 1, ids, torch.tensor(E, dtype=torch.int32))
    if kind == "none":
        ids[:] = -1
    m = routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=gate).upload()
    y = torch.full((T * k, m.n_out), 7.0, dtype=t, device=DEV)
    m.mm_routed(x.to(DEV), routed.route_plan(ids.to(DEV), E), y)
    flat, x64 = ids.reshape(-1).numpy(), np.repeat(np64(x), k, axis=0)
    want, tol = np.full((T * k, m.n_out), 7.0), np.zeros((T * k, m.n_out))
    for e in range(E):
        at = np.nonzero(flat == e)[0]
        if len(at):
            a, b = product(x64[at], q, e, group)
            want[at], tol[at] = gated(a, b) if gate else (a, b)
    assert_close(y, want, tol, t)


@pytest.mark.gpu
def test_a_row_with_nan_stays_alone():
    gen = torch.Generator().manual_seed(5)
    q = [a.to(DEV) for a in matrices(gen, 1, 40, 256, 64, torch.bfloat16, True)]
    x = torch.randn((70, 256), generator=gen).to(torch.bfloat16).to(DEV)
    m = routed.Q4(*q, group=64).upload()
    clean = m.mm(x)
    x[3, 7], x[40, 100] = math.nan, math.inf
    y = m.mm(x)
    others = [r for r in range(70) if r not in (3, 40)]
    assert torch.equal(y[others], clean[others]) and bool(y[3].isnan().all()) and not bool(y[40].isfinite().any())


@pytest.mark.gpu
@pytest.mark.parametrize("count", [1, 3])
def test_matrices_beyond_4_gib(count):
    # codes of 4.5 GiB, in one matrix or in three: the last rows are behind 32-bit offsets
    K, group = 8192, 128
    N = (9 * 2 ** 29 // (K // 2) // count // 2 * 2) + 2
    gen = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randint(0, 256, (count, N, K // 2), generator=gen, device=DEV, dtype=torch.uint8)
    scales = torch.full((count, N, K // group), 0.01, dtype=torch.bfloat16, device=DEV)
    m = routed.Q4(codes, scales, group=group).upload()
    x = torch.randn((2, K), generator=gen, device=DEV).to(torch.bfloat16)
    ids = torch.tensor([[count - 1], [0]], dtype=torch.int32, device=DEV)
    y = m.mm_routed(x, routed.route_plan(ids, count), y_dtype=torch.float32)
    rows = [0, 1, N // 2, N - 18, N - 1]
    for r, e in ((0, count - 1), (1, 0)):
        q = (codes[e, rows].cpu()[None], scales[e, rows].cpu()[None], None)
        want, tol = product(np64(x[r: r + 1]), q, 0, group)
        assert_close(y[r: r + 1, rows], want, tol, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 20])
def test_rows_of_x_beyond_4_gib(T):
    K, N, ld = 256, 40, 2 ** 31 // T // 8 * 8 + 64                           # T rows that span more than 2^31 elements
    gen = torch.Generator().manual_seed(T)
    q = matrices(gen, 3, N, K, 64, torch.bfloat16, True)
    far = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV).as_strided((T, K), (ld, 1))
    x = torch.randn((T, K), generator=gen).to(torch.bfloat16)
    far.copy_(x.to(DEV))
    m = routed.Q4(*[a.to(DEV) for a in q], group=64).upload()
    ids = torch.arange(T, dtype=torch.int32).view(T, 1) % 3
    y = m.mm_routed(far, routed.route_plan(ids.to(DEV), 3), y_dtype=torch.float32)
    one = routed.Q4(*[a[0].to(DEV) for a in q], group=64).upload()
    y0 = one.mm(far, y_dtype=torch.float32)
    for r in range(T):
        want, tol = product(np64(x[r: r + 1]), q, r % 3, 64)
        assert_close(y[r: r + 1], want, tol, torch.float32)
    want, tol = product(np64(x), q, 0, 64)
    assert_close(y0, want, tol, torch.float32)


@pytest.mark.gpu
def test_a_layer_for_rows_beyond_4_gib():
    T, k, E, K, F, t = 3, 2, 5, 64, 32, torch.bfloat16
    ld = 2 ** 31 // T // 8 * 8 + 64
    gen = torch.Generator().manual_seed(2)
    up, down = matrices(gen, E, 2 * F, K, 32, t, True), matrices(gen, E, K, F, 32, t, True)
    on = [routed.Q4(*[a.to(DEV) for a in q], group=32, gated=g).upload() for q, g in ((up, True), (down, False))]
    x, w = torch.randn((T, K), generator=gen).to(t), torch.randn((T, k), generator=gen)
    far = torch.empty(T * ld, dtype=t, device=DEV).as_strided((T, K), (ld, 1))
    far.copy_(x.to(DEV))
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    want, tol = layer_of(np64(x), ids.numpy(), np64(w), up, down, 32, t)
    assert_close(routed.experts_forward(far, ids.to(DEV), w.to(DEV), *on), want, tol, t)


@pytest.mark.gpu
def test_codes_that_begin_between_words():
    gen = torch.Generator().manual_seed(8)
    q = matrices(gen, 1, 50, 160, 32, torch.float16, True)
    raw = torch.zeros(50 * 80 + 16, dtype=torch.uint8, device=DEV)
    x = torch.randn((4, 160), generator=gen).half()
    want, tol = product(np64(x), q, 0, 32)
    for shift in (0, 1, 4, 8):
        codes = raw[shift: shift + 50 * 80].view(50, 80)
        codes.copy_(q[0][0].to(DEV))
        m = routed.Q4(codes, q[1][0].to(DEV), q[2][0].to(DEV), group=32).upload()
        assert_close(m.mm(x.to(DEV), y_dtype=torch.float32), want, tol, torch.float32)


# ------------------------------------------------------------------------------------------- the sum
SUMS = [(1, 1, 8, "f32", "f32"), (3, 4, 72, "bf16", "bf16"), (33, 8, 520, "f16", "f16"), (7, 2, 4096, "f32", "bf16"), (5, 3, 1000, "f32", "f16"), (130, 6, 64, "bf16", "f32"),
        (2, 64, 256, "bf16", "bf16"), (1000, 5, 24, "f16", "f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,D,y_type,out_type", SUMS)
@pytest.mark.parametrize("holes", [False, True])
def test_sum_and_its_gradients(T, k, D, y_type, out_type, holes):
    gen = torch.Generator().manual_seed(T + D)
    ty, to = TYPES[y_type], TYPES[out_type]
    y = torch.randn((T * k, D), generator=gen).to(ty)
    dout = torch.randn((T, D), generator=gen).to(to)
    w = torch.randn((T, k), generator=gen)
    ids = torch.randint(0, 9, (T, k), generator=gen, dtype=torch.int32)
    if holes:
        ids = torch.where(torch.rand((T, k), generator=gen) < 0.5, torch.tensor(-3 if T % 2 else 9, dtype=torch.int32), ids)
    there = ((ids >= 0) & (ids < 9)).numpy()
    y64, w64, g64 = np64(y).reshape(T, k, D), np64(w) * there, np64(dout)
    y[~there.reshape(-1)] = math.nan                                        # rows that nobody may read
    on = [a.to(DEV) for a in (y, ids, w, dout)]
    out = routed.route_combine(on[0], on[1], on[2], out_dtype=to, n_experts=9)
    terms = np.abs(w64[..., None] * y64).sum(1)
    assert_close(out, (w64[..., None] * y64).sum(1), k * U * terms, to)
    dy, dw = routed.route_combine_grad(on[3], on[0], on[1], on[2], n_experts=9)
    want = w64[..., None] * g64[:, None]
    assert_close(dy.view(T, k, D), want, U * np.abs(want), ty)
    want = (y64 * g64[:, None]).sum(2) * there
    assert_close(dw, want, U * (D / 64 + 16) * np.abs(y64 * g64[:, None]).sum(2) * there, torch.float32)
    wide = torch.full((T, D + 16), 7.0, dtype=to, device=DEV)
    routed.route_combine(on[0], on[1], on[2], wide[:, 8: 8 + D], n_experts=9)
    assert torch.equal(wide[:, 8: 8 + D], out) and bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + D:] == 7).all())


# ------------------------------------------------------------------------------------------- together
def layer(seed, E, K, F, group, dtype):
    gen = torch.Generator().manual_seed(seed)
    up, down = matrices(gen, E, 2 * F, K, group, dtype, True), matrices(gen, E, K, F, group, dtype, False)
    on = [routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=g).upload() for q, g in ((up, True), (down, False))]
    return up, down, on[0], on[1]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 64, 400])
def test_a_layer_of_experts(T):
    E, k, K, F, group, t = 12, 3, 288, 160, 32, torch.bfloat16
    up, down, on_up, on_down = layer(T, E, K, F, group, t)
    gen = torch.Generator().manual_seed(T + 1)
    x, l = torch.randn((T, K), generator=gen).to(t), torch.randn((T, E), generator=gen)
    l[T // 2] = -math.inf                                                   # a padding row
    ids, weights = routed.route_topk(l.to(DEV), k, score="sigmoid", renormalise=True, scale=1.5)
    out = routed.experts_forward(x.to(DEV), ids, weights, on_up, on_down)
    i64, w64, x64 = ids.cpu().numpy(), np64(weights), np64(x)
    want, tol = np.zeros((T, K)), np.zeros((T, K))
    for e in range(E):
        at, place = np.nonzero(i64 == e)
        if not len(at):
            continue
        h, th = gated(*product(x64[at], up, e, group))
        th = th + half_step(t) * (np.abs(h) + th)                           # kept in bf16
        y, ty = product(h, down, e, group)
        w = np64(down[1][e])[:, np.arange(F) // group]
        c = down[0][e].numpy()
        codes = np.empty((K, F))
        codes[:, 0::2], codes[:, 1::2] = c & 15, c >> 4
        ty = 1.01 * ty + th @ np.abs(w * (codes - 8)).T
        np.add.at(want, at, w64[at, place][:, None] * y)
        np.add.at(tol, at, np.abs(w64[at, place][:, None]) * (ty + 4 * U * np.abs(y)))
    assert_close(out, want, tol, t)
    assert bool((out[T // 2] == 0).all())


def numbers(m, e, group):
    """|s (c - z)| of matrix e"""
    c = m[0][e].numpy()
    codes = np.empty((c.shape[0], 2 * c.shape[1]))
    codes[:, 0::2], codes[:, 1::2] = c & 15, c >> 4
    by = np.arange(codes.shape[1]) // group
    return np.abs(np64(m[1][e])[:, by] * (codes - (8 if m[2] is None else np64(m[2][e])[:, by])))


def layer_of(x, ids, weights, up, down, group, dtype):
    """What a layer gives, and its bound."""
    T, k, K = len(x), ids.shape[1], down[0].shape[1]
    want, tol = np.zeros((T, K)), np.zeros((T, K))
    for e in range(up[0].shape[0]):
        at, place = np.nonzero(ids == e)
        if len(at):
            h, th = gated(*product(x[at], up, e, group))
            th = th + half_step(dtype) * (np.abs(h) + th) + (2.0 ** -25 if dtype is torch.float16 else 0)        # kept in the matrices' type
            y, ty = product(h, down, e, group)
            ty = 1.01 * ty + th @ numbers(down, e, group).T
            # the sum: a product with the weight and at most k additions, each rounded, of terms no larger than all together
            np.add.at(want, at, weights[at, place][:, None] * y)
            np.add.at(tol, at, np.abs(weights[at, place][:, None]) * (ty + (k + 8) * U * (np.abs(y) + ty)))
    return want, tol


# few pairs, which are not grouped: one to many of a row, parts of columns and waves without any, odd sizes, the last two on both sides of where they are
@pytest.mark.gpu
@pytest.mark.parametrize("T,k,E,K,F,group,dtype,zeros,out_type", [
    (1, 1, 1, 32, 32, 32, "bf16", True, "bf16"), (1, 8, 16, 256, 160, 64, "f16", True, "f32"), (1, 2, 3, 96, 1056, 128, "bf16", False, "f32"),
    (1, 64, 64, 64, 32, 32, "f16", False, "f16"), (2, 3, 40, 288, 416, 32, "f16", True, "bf16"), (3, 2, 30, 544, 96, 256, "bf16", True, "f16"),
    (1, 4, 9, 64, 4128, 64, "bf16", False, "bf16"), (13, 10, 200, 64, 64, 64, "bf16", True, "f32"), (51, 5, 1024, 32, 32, 32, "f16", False, "f16"),
    (52, 5, 1024, 32, 32, 32, "f16", False, "f16")])
def test_a_layer_for_few_rows(T, k, E, K, F, group, dtype, zeros, out_type):
    t, to = TYPES[dtype], TYPES[out_type]
    gen = torch.Generator().manual_seed(T * k + E)
    up, down = matrices(gen, E, 2 * F, K, group, t, zeros), matrices(gen, E, K, F, group, t, zeros)
    on_up, on_down = [routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=g).upload() for q, g in ((up, True), (down, False))]
    x, weights = torch.randn((T, K), generator=gen).to(t), torch.randn((T, k), generator=gen)
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)             # the same one twice, too
    ids = torch.where(torch.rand((T, k), generator=gen) < 0.2, torch.tensor(-1 if T % 2 else E, dtype=torch.int32), ids)
    if T > 2:
        ids[1] = E + 5                                                              # a row of none
    wide = torch.full((T, K + 16), 7.0, dtype=to, device=DEV)
    out = routed.experts_forward(x.to(DEV), ids.to(DEV), weights.to(DEV), on_up, on_down, wide[:, 8: 8 + K])
    i64, w64, x64 = ids.numpy(), np64(weights), np64(x)
    want, tol = layer_of(x64, i64, w64, up, down, group, t)
    assert_close(out, want, tol, to)
    assert bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + K:] == 7).all())
    # in a graph, twice, with other work between
    static = [a.to(DEV) for a in (x, ids, weights)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        routed.experts_forward(*static, on_up, on_down)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = routed.experts_forward(*static, on_up, on_down)
    for _ in range(2):
        again.fill_(3.0)
        graph.replay()
        assert torch.equal(again, routed.experts_forward(*static, on_up, on_down))


@pytest.mark.gpu
def test_a_layer_in_a_graph_and_on_other_streams():
    E, k, K, F, group, t, T = 16, 4, 256, 128, 64, torch.float16, 37
    _, _, up, down = layer(7, E, K, F, group, t)
    x, l, bias = torch.zeros((T, K), dtype=t, device=DEV), torch.zeros((T, E), device=DEV), torch.zeros(E, device=DEV)
    dout = torch.zeros((T, K), dtype=t, device=DEV)

    def step():
        ids, weights = routed.route_topk(l, k, score="sigmoid", bias=bias, n_groups=4, top_groups=2)
        plan = routed.route_plan(ids, E)
        h = up.mm_routed(x, plan)
        y = down.mm_routed(h, plan)
        out = routed.route_combine(y, ids, weights)
        dy, dw = routed.route_combine_grad(dout, y, ids, weights)
        return out, ids, dy, dw, routed.route_topk_grad(l, ids, dw, score="sigmoid"), routed.experts_forward(x, ids, weights, up, down)

    def fill(seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        for a in (x, l, bias, dout):
            a.normal_(generator=gen)

    side = torch.cuda.Stream()
    fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graphs = []
    for _ in range(2):                                                      # two of them, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = step()
        graphs.append((g, r))
    for seed in range(1, 6):
        fill(seed)
        want = [a.clone() for a in step()]
        for g, r in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, r))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, again))


# ------------------------------------------------------------------------------------------- refusals
def test_choice_refuses_on_the_host():
    l = torch.zeros((4, 12))
    with pytest.raises(ValueError, match="on the GPU"):
        routed.route_topk(l, 2)
    for bad in (torch.zeros(12), torch.zeros((4, 12), dtype=torch.float64), torch.zeros((12, 4)).t(), torch.zeros((1, 12)).expand(4, 12)):
        with pytest.raises(ValueError):
            routed.route_topk(bad, 2)
    for kw in (dict(bias=torch.zeros(11)), dict(bias=torch.zeros(12, dtype=torch.float16)), dict(ids=torch.zeros((4, 2))), dict(weights=torch.zeros((4, 3))), dict(score="tanh")):
        with pytest.raises(ValueError):
            routed.route_topk(l, 2, **kw)
    for ids, dw in ((torch.zeros((4, 2)), torch.zeros((4, 2))), (torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2))), (torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 3)))):
        with pytest.raises(ValueError):
            routed.route_topk_grad(l, ids, dw)
    one = ctypes.c_void_p(4096)                                             # never read: every call below is refused
    ok = dict(n_experts=12, top_k=2, score=0, n_groups=1, top_groups=1, renormalise=1, scale=1.0)
    for change in (dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=13), dict(score=2), dict(n_groups=5), dict(n_groups=0), dict(top_groups=2),
                   dict(n_groups=12, top_groups=1), dict(scale=math.inf), dict(scale=math.nan), dict(n_experts=130, n_groups=65, top_groups=65), dict(n_experts=200, top_k=65)):
        how = binding._Route(**{**ok, **change})
        assert binding._lib.route_topk(ctypes.byref(how), one, 2000, 2, None, 4, one, one, None) == -1
        assert binding._lib.route_topk_grad(ctypes.byref(how), one, 2000, 2, one, one, 4, one, 2000, None) == -1
    how = ctypes.byref(binding._Route(**ok))
    f = binding._lib.route_topk
    assert f(how, one, 11, 2, None, 4, one, one, None) == -1 and f(how, one, 12, 3, None, 4, one, one, None) == -1 and f(how, None, 12, 2, None, 4, one, one, None) == -1
    assert f(how, one, 12, 2, None, -1, one, one, None) == -1 and f(how, ctypes.c_void_p(4098), 12, 2, None, 4, one, one, None) == -1
    assert f(None, one, 12, 2, None, 4, one, one, None) == -1 and f(how, one, 12, 2, None, 2 ** 30, one, one, None) == -5
    assert f(how, None, 12, 2, None, 0, None, None, None) == 0


def test_plan_and_sum_refuse_on_the_host():
    ids = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        routed.route_plan(ids, 8)
    for bad in (torch.zeros(8, dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int64), torch.zeros((2, 4), dtype=torch.int32).t()):
        with pytest.raises(ValueError):
            routed.route_plan(bad, 8)
    for E in (0, -1, 1025):
        with pytest.raises(binding.VbrError):
            routed.route_plan(ids, E)
    lib, one = binding._lib, ctypes.c_void_p(4096)
    assert lib.route_plan_bytes(-1, 8) == 0 and lib.route_plan_bytes(2 ** 30 + 1, 8) == 0 and lib.route_plan_bytes(8, 0) == 0
    assert lib.route_plan(one, 8, 8, None, None) == -1 and lib.route_plan(None, 8, 8, one, None) == -1 and lib.route_plan(one, 8, 8, ctypes.c_void_p(4096 + 128), None) == -1
    y, w = torch.zeros((8, 16)), torch.zeros((4, 2))
    with pytest.raises(ValueError, match="on the GPU"):
        routed.route_combine(y, ids, w)
    for args in ((y[:7], ids, w), (y.double(), ids, w), (y, ids.long(), w), (y, ids, w.half()), (y, ids, w[:3]), (y, ids, w, torch.zeros((4, 15)))):
        with pytest.raises(ValueError):
            routed.route_combine(*args)
    with pytest.raises(ValueError):
        routed.route_combine_grad(torch.zeros((4, 15)), y, ids, w)
    with pytest.raises(ValueError):
        routed.route_combine_grad(torch.zeros((4, 16)), y, ids, w, dy=torch.zeros((8, 16), dtype=torch.float16))
    f = lib.route_combine
    assert f(one, 16, 2, one, one, 4, 2, 8, 12, one, 16, 2, None) == -1       # columns that are no multiple of 8
    assert f(one, 12, 2, one, one, 4, 2, 8, 16, one, 16, 2, None) == -1 and f(one, 16, 2, one, one, 4, 0, 8, 16, one, 16, 2, None) == -1
    assert f(one, 16, 2, one, one, 4, 2, 0, 16, one, 16, 2, None) == -1 and f(ctypes.c_void_p(4104), 16, 2, one, one, 4, 2, 8, 16, one, 16, 2, None) == -1
    assert f(one, 16, 2, None, one, 4, 2, 8, 16, one, 16, 2, None) == -1 and f(None, 16, 2, None, None, 0, 2, 8, 16, None, 16, 2, None) == 0


def test_matrices_and_products_refuse_on_the_host():
    codes, scales = torch.zeros((2, 6, 64), dtype=torch.uint8), torch.zeros((2, 6, 2), dtype=torch.float16)
    ok = routed.Q4(codes, scales, group=64)
    with pytest.raises(ValueError, match="on the GPU"):
        ok.upload()
    with pytest.raises(binding.VbrError):                                   # not uploaded
        ok.mm(torch.zeros((1, 128), dtype=torch.float16))
    for args, kw in (((codes.int(), scales), dict(group=64)), ((codes, scales.float()), dict(group=64)), ((codes, scales[:, :5]), dict(group=64)), ((codes, scales[0]), dict(group=64)),
                     ((codes, scales, scales), dict(group=64)), ((codes, scales, torch.zeros((2, 6, 1), dtype=torch.uint8)), dict(group=64)), ((codes, scales), dict(group=0))):
        with pytest.raises(ValueError):
            routed.Q4(*args, **kw)
    for shape, group, gate in (((2, 6, 64), 96, False), ((2, 6, 40), 32, False), ((2, 5, 64), 64, True), ((2, 6, 64), 48, False), ((2, 6, 64), 16, False)):
        g = -(-2 * shape[2] // group)
        with pytest.raises(binding.VbrError):
            routed.Q4(torch.zeros(shape, dtype=torch.uint8), torch.zeros(shape[:2] + (g,), dtype=torch.float16), group=group, gated=gate)
    for x in (torch.zeros((1, 64), dtype=torch.float16), torch.zeros((1, 128)), torch.zeros(128, dtype=torch.float16)):
        with pytest.raises(ValueError):
            ok.mm(x)
    x = torch.zeros((3, 128), dtype=torch.float16)
    for y in (torch.zeros((3, 5), dtype=torch.float16), torch.zeros((2, 6), dtype=torch.float16), torch.zeros((3, 6), dtype=torch.bfloat16), torch.zeros((1, 6)).expand(3, 6)):
        with pytest.raises(ValueError):
            ok.mm(x, y)
    lib, h, one = binding._lib, ctypes.c_void_p(), ctypes.c_void_p(4096)
    for args in ((0, 6, 128, 64, 0), (1, 0, 128, 64, 0), (1, 6, 0, 64, 0), (1, 6, 120, 64, 0), (1, 6, 128, 64, 2)):
        assert lib.q4_create(*args, 0, 0, ctypes.byref(h)) == -1 and not h
    assert lib.q4_create(1025, 6, 128, 64, 0, 0, 0, ctypes.byref(h)) == -5 and lib.q4_create(1, 6, 128, 64, 0, 0, 0, None) == -1
    assert lib.q4_create(2, 6, 128, 64, 0, 1, 0, ctypes.byref(h)) == 0
    assert lib.q4_mm(h, one, 128, one, 6, 0, 4, None) == -4 and lib.q4_mm(None, one, 128, one, 6, 0, 4, None) == -1 and lib.q4_mm(h, one, 128, one, 6, 1, 4, None) == -1
    assert lib.q4_upload(h, one, one, None, one, None) == -1 and lib.q4_upload(h, one, one, one, ctypes.c_void_p(4160), None) == -1 and lib.q4_upload(h, None, one, one, one, None) == -1
    lib.q4_free(h)


def test_types_of_results_are_refused_on_the_host():
    ids, w, y = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), torch.zeros((8, 16))
    for kw in (dict(out_dtype=torch.float64), dict(out_dtype=torch.float16, out=torch.zeros((4, 16))), dict(out=torch.zeros((4, 16), dtype=torch.float64))):
        with pytest.raises(ValueError):
            routed.route_combine(y, ids, w, **kw)
    m = routed.Q4(torch.zeros((6, 64), dtype=torch.uint8), torch.zeros((6, 2), dtype=torch.float16), group=64)
    x = torch.zeros((3, 128), dtype=torch.float16)
    for kw in (dict(y_dtype=torch.bfloat16), dict(y_dtype=torch.float64), dict(y_dtype=torch.float32, y=torch.zeros((3, 6), dtype=torch.float16))):
        with pytest.raises(ValueError):
            m.mm(x, **kw)


@pytest.mark.gpu
def test_products_refuse_on_the_gpu():
    codes, scales = torch.zeros((2, 6, 64), dtype=torch.uint8, device=DEV), torch.zeros((2, 6, 2), dtype=torch.float16, device=DEV)
    m = routed.Q4(codes, scales, group=64).upload()
    x = torch.zeros((3, 128), dtype=torch.float16, device=DEV)
    ids = torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(binding.VbrError):                                   # two matrices
        m.mm(x)
    with pytest.raises(ValueError):
        m.mm_routed(x, routed.route_plan(ids, 3))
    with pytest.raises(ValueError):
        m.mm_routed(x[:2], routed.route_plan(ids, 2))
    with pytest.raises(ValueError):
        m.mm_routed(x.cpu(), routed.route_plan(ids, 2))
    with pytest.raises(binding.VbrError):                                   # a row stride that is no multiple of 8, an address that is none of 16
        m.mm_routed(torch.zeros((3, 132), dtype=torch.float16, device=DEV)[:, :128], routed.route_plan(ids, 2))
    with pytest.raises(binding.VbrError):
        m.mm_routed(torch.zeros((3, 136), dtype=torch.float16, device=DEV)[:, 4:132], routed.route_plan(ids, 2))
    with pytest.raises(ValueError):
        routed.route_topk(torch.zeros((3, 4), device=DEV), 2, bias=torch.zeros(4))
    with pytest.raises(ValueError):
        routed.experts_forward(x, ids, torch.zeros((3, 2), device=DEV), m, m)
