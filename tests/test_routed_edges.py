"""Routed products where numbers are far apart or near each other, against the definitions in 64 bits of test_routed."""
import math

import numpy as np
import pytest
import torch

from paper_2202_05868_amd import binding, routed
from test_routed import DEV, TYPES, U, assert_close, choice, choice_grad, gated, layer_of, matrices, np64, product

LOWEST = torch.finfo(torch.float32).min


# ------------------------------------------------------------------------------------------- gates
def far_matrices(gen, M, N, K, group, dtype, zeros):
    """Gated matrices whose gates' rows are of very different size, so that with x of deviation 1 gates have deviations of 4 .. 4000 and every
    tenth lies between -89 and -2000; what they gate has a deviation near 0.1, so that results stay in fp16's range."""
    G, F = -(-K // group), N // 2
    codes = torch.randint(0, 256, (M, N, K // 2), generator=gen, dtype=torch.uint8)
    size = torch.full((M, N, 1), 0.1)
    size[:, :F] = 4 * 1000 ** torch.rand((M, F, 1), generator=gen)
    scales = ((torch.rand((M, N, G), generator=gen) + 0.5) * size / (4.6 * math.sqrt(K))).to(dtype)
    z = torch.randint(6, 10, (M, N, G), generator=gen, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def gated_of(x, q, m, group):
    with np.errstate(over="ignore"):                                        # (1 + an infinite exponential divides to zero)
        return gated(*product(x, q, m, group))


def on_gpu(q, group, gate=True):
    return routed.Q4(*[None if a is None else a.to(DEV) for a in q], group=group, gated=gate).upload()


# products of 16, 32 and 64 rows, in few workgroups and in many
@pytest.mark.gpu
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("T,F,K,group,dtype,zeros", [
    (1, 66, 160, 64, "bf16", False), (5, 300, 288, 32, "f16", True), (16, 12000, 160, 64, "bf16", True), (48, 5456, 288, 128, "bf16", True), (40, 16384, 96, 128, "f16", False),
    (130, 16384, 64, 32, "bf16", True), (300, 8192, 160, 128, "f16", True), (70, 24000, 64, 64, "bf16", False), (961, 8200, 96, 128, "bf16", True), (1024, 8200, 64, 32, "f16", False)])
def test_gates_far_from_zero(T, F, K, group, dtype, zeros, out):
    t = TYPES[dtype]
    y_type = t if out == "same" else torch.float32
    gen = torch.Generator().manual_seed(T + F)
    q = far_matrices(gen, 1, 2 * F, K, group, t, zeros)
    x = torch.randn((T, K), generator=gen).to(t)
    want, tol = gated_of(np64(x), q, 0, group)
    y = on_gpu(q, group).mm(x.to(DEV), y_dtype=y_type)
    assert bool(y.isfinite().all())
    assert_close(y, want, tol, y_type)


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,E,F,K,group,dtype,zeros", [(16, 4, 64, 34, 160, 32, "bf16", True), (600, 4, 8, 129, 544, 128, "bf16", True), (400, 4, 64, 513, 160, 32, "f16", True),
                                                         (2000, 4, 64, 257, 224, 64, "f16", False)])
def test_routed_gates_far_from_zero(T, k, E, F, K, group, dtype, zeros):
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(T + F)
    q = far_matrices(gen, E, 2 * F, K, group, t, zeros)
    x = torch.randn((T, K), generator=gen).to(t)
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    y = on_gpu(q, group).mm_routed(x.to(DEV), routed.route_plan(ids.to(DEV), E))
    flat, x64 = ids.reshape(-1).numpy(), np.repeat(np64(x), k, axis=0)
    want, tol = np.zeros((T * k, F)), np.zeros((T * k, F))
    for e in range(E):
        at = np.nonzero(flat == e)[0]
        want[at], tol[at] = gated_of(x64[at], q, e, group)
    assert bool(y.isfinite().all())
    assert_close(y, want, tol, t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 4, 400])
def test_a_layer_with_gates_far_from_zero(T, dtype):
    E, k, K, F, group, t = 12, 3, 288, 160, 32, TYPES[dtype]
    gen = torch.Generator().manual_seed(T)
    up = far_matrices(gen, E, 2 * F, K, group, t, True)
    down = matrices(gen, E, K, F, group, t, False)
    x, w = torch.randn((T, K), generator=gen).to(t), torch.rand((T, k), generator=gen)
    ids = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    with np.errstate(over="ignore"):
        want, tol = layer_of(np64(x), ids.numpy(), np64(w), up, down, group, t)
    out = routed.experts_forward(x.to(DEV), ids.to(DEV), w.to(DEV), on_gpu(up, group), on_gpu(down, group, False))
    assert bool(out.isfinite().all())
    assert_close(out, want, tol, t)


# ------------------------------------------------------------------------------------------- biases of the lowest number
def lowest_biases(kind, E, groups):
    size = E // groups
    b = torch.full((E,), LOWEST)
    if kind == "one open":                     # and the others of its group closed for good
        b[size: 2 * size] = -math.inf
        b[size + 1 if size > 1 else size] = 0.25
    if kind == "few":
        b = torch.full((E,), -math.inf)
        b[::3] = LOWEST
        b[1] = 0.5
    if kind == "high":                         # sums of two are beyond fp32
        b = 3e38 - 1e37 * torch.arange(E, dtype=torch.float32).flip(0) % 7e37
    if kind == "infinite":
        b = torch.full((E,), 0.1)
        b[size - 1::size] = math.inf
        b[E // 2] = torch.finfo(torch.float32).max
    return b


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["all", "one open", "few", "high", "infinite"])
@pytest.mark.parametrize("T", [5, 2048])
@pytest.mark.parametrize("E,groups,top_groups,k", [(32, 16, 3, 4), (16, 8, 2, 3), (60, 4, 2, 20), (256, 8, 3, 8), (12, 12, 5, 4), (64, 32, 4, 7), (576, 64, 5, 6)])
def test_groups_of_biases_at_the_ends_of_the_range(kind, T, E, groups, top_groups, k):
    gen = torch.Generator().manual_seed(E)
    l = torch.randn((T, E), generator=gen)
    b = lowest_biases(kind, E, groups)
    for score in ("sigmoid", "softmax"):
        ids, weights = routed.route_topk(l.to(DEV), k, score=score, bias=b.to(DEV), n_groups=groups, top_groups=top_groups, renormalise=False)
        some = slice(0, 40)
        want, w, _ = choice(np64(l)[some], k, score, np64(b), groups, top_groups, False, 1.0)
        assert np.array_equal(ids[some].cpu().numpy(), want)
        assert np.allclose(np64(weights)[some], w, rtol=2.0 ** -17, atol=0)     # scores of |l| < 8 in fp32: 2 * 8 + 80 roundings, and more


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 2048])
@pytest.mark.parametrize("E,groups,top_groups,k", [(32, 16, 3, 4), (60, 4, 1, 5), (60, 4, 2, 9), (256, 8, 3, 8), (256, 8, 1, 3), (12, 12, 5, 4), (64, 32, 4, 7), (576, 64, 5, 6)])
@pytest.mark.parametrize("infinite", [1, 2, 4])
def test_groups_with_infinite_biases_come_first(T, E, groups, top_groups, k, infinite):
    """The other groups have two biases that are larger than half of the largest number, those with an infinite one have low ones beside it."""
    size = E // groups
    l = torch.randn((T, E), generator=torch.Generator().manual_seed(E))
    b = 3e38 * (1 - 0.3 * torch.arange(E) / E)
    for g in range(infinite):
        at = (groups - 1 - 2 * g) % groups * size
        b[at: at + size] = -1e30
        b[at + size // 2] = math.inf
    ids, _ = routed.route_topk(l.to(DEV), k, score="sigmoid", bias=b.to(DEV), n_groups=groups, top_groups=top_groups)
    want, _, _ = choice(np64(l)[:40], k, "sigmoid", np64(b), groups, top_groups, True, 1.0)
    assert np.array_equal(ids[:40].cpu().numpy(), want)


# ------------------------------------------------------------------------------------------- sums near each other
def choice_of_all(l, k, score, bias, groups, top_groups):
    """ids [T, k] of all rows at once; -inf closes."""
    T, E = l.shape
    closed = l == -np.inf
    if score == "softmax":
        most = l.max(1, keepdims=True)
        e = np.exp(l - np.where(most == -np.inf, 0, most))
        s = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
    else:
        s = np.where(closed, 0, 1 / (1 + np.exp(-l)))
    key = s + (0 if bias is None else bias)
    out = closed | (key == -np.inf)
    if groups > 1:
        by = -np.sort(-np.where(out, -np.inf, key).reshape(T, groups, -1), 2)[:, :, :2]
        total = by[:, :, 0] + np.where(by[:, :, -1] == -np.inf, 0, by[:, :, -1]) * (by.shape[2] > 1)
        stays = np.argsort(-total, 1, kind="stable")[:, :top_groups]
        mask = np.zeros((T, groups), bool)
        np.put_along_axis(mask, stays, True, 1)
        out |= ~np.repeat(mask, E // groups, 1)
    order = l if bias is None else key
    want = np.argsort(-np.where(out, -np.inf, order), 1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(out, want, 1), -1, want)


def near_scores(seed, T, E):
    """Rows of scores that 32 bits tell apart, and rows of scores that they do not, once a bias is added; some closed."""
    gen = torch.Generator().manual_seed(seed)
    l = 1.5 * torch.randn((T, E), generator=gen)
    near = torch.rand((T, 1), generator=gen) < 0.5
    l = torch.where(near, l[:, :1] * (1 + 1e-7 * torch.randint(-3, 4, (T, E), generator=gen)), l)
    l = torch.where(torch.rand((T, E), generator=gen) < 0.05, torch.tensor(-math.inf), l)
    l[T // 3: T // 3 + 3] = -math.inf
    return l


# on both sides of where a row has 64 lanes, and of more experts, places and groups than 16 lanes take
@pytest.mark.gpu
@pytest.mark.parametrize("far", [None, -1e4, -1e9, LOWEST, -math.inf, 100.0])
@pytest.mark.parametrize("T,E,k,score,step,groups,top_groups", [
    (700, 256, 8, "sigmoid", 2.0 ** -24, 8, 4), (2047, 256, 8, "softmax", 2.0 ** -26, 8, 3), (2048, 256, 8, "sigmoid", 2.0 ** -24, 8, 4), (2048, 96, 6, "softmax", 2.0 ** -26, 12, 5),
    (2500, 100, 5, "sigmoid", 2.0 ** -24, 5, 2), (900, 512, 8, "sigmoid", 2.0 ** -24, 16, 4), (900, 1024, 8, "softmax", 2.0 ** -28, 32, 5), (800, 128, 33, "sigmoid", 2.0 ** -24, 1, 1),
    (800, 1024, 12, "sigmoid", 2.0 ** -24, 1, 1), (700, 160, 6, "softmax", 2.0 ** -26, 32, 7), (700, 300, 9, "sigmoid", 2.0 ** -24, 20, 6), (600, 64, 4, "softmax", 2.0 ** -24, 32, 3)])
def test_choices_of_sums_near_each_other(T, E, k, score, step, groups, top_groups, far):
    l = near_scores(E + T, T, E)
    gen = torch.Generator().manual_seed(E)
    bias = step * torch.randn(E, generator=gen)
    if far is not None:                                    # a third of the experts
        bias = torch.where(torch.rand(E, generator=gen) < 0.33, torch.tensor(far), bias)
    want = choice_of_all(np64(l), k, score, np64(bias), groups, top_groups)
    ids, _ = routed.route_topk(l.to(DEV), k, score=score, bias=bias.to(DEV), n_groups=groups, top_groups=top_groups)
    assert np.array_equal(ids.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------- results of pairs without an expert
@pytest.mark.gpu
@pytest.mark.parametrize("T,k,D,type_", [(1, 1, 8, "f32"), (40, 3, 72, "bf16"), (300, 8, 264, "f16"), (7, 13, 1032, "f32"), (5, 64, 24, "bf16")])
@pytest.mark.parametrize("kind", ["first", "last", "one", "none"])
def test_sums_of_rows_with_few_results(T, k, D, type_, kind):
    """The kernel reads zeros in the place of results that do not count; these are NaN here, so that one that got into a sum would show."""
    t = TYPES[type_]
    gen = torch.Generator().manual_seed(T + k)
    y, w = torch.randn((T * k, D), generator=gen).to(t), torch.randn((T, k), generator=gen)
    ids = torch.randint(0, 5, (T, k), generator=gen, dtype=torch.int32)
    keep = dict(first=torch.arange(k) == 0, last=torch.arange(k) == k - 1, one=torch.arange(k) == torch.randint(0, k, (T, 1), generator=gen), none=torch.zeros(k, dtype=torch.bool))[kind]
    ids = torch.where(keep.expand(T, k), ids, torch.tensor(-1 if T % 2 else 5, dtype=torch.int32))
    ids[T // 2] = 7                                                        # a row of none among the others
    there = ((ids >= 0) & (ids < 5)).numpy()
    terms = np64(w)[..., None] * np64(y).reshape(T, k, D) * there[..., None]
    y[~there.reshape(-1)] = math.nan
    out = routed.route_combine(y.to(DEV), ids.to(DEV), w.to(DEV), n_experts=5)
    assert_close(out, terms.sum(1), U * np.abs(terms).sum(1), t)           # one term a row: its product is the one rounding
    assert bool((out[T // 2] == 0).all())


# ------------------------------------------------------------------------------------------- gradients that would be lost
def test_operands_that_require_a_gradient_are_refused():
    l, x, y = torch.zeros((4, 12)), torch.zeros((4, 128), dtype=torch.float16), torch.zeros((8, 16))
    ids, w = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2))
    up = routed.Q4(torch.zeros((3, 8, 64), dtype=torch.uint8), torch.zeros((3, 8, 2), dtype=torch.float16), group=64, gated=True)
    down = routed.Q4(torch.zeros((3, 8, 16), dtype=torch.uint8), torch.zeros((3, 8, 1), dtype=torch.float16), group=32)
    up.n_out = down.n_cols                                                  # (matrices that no call gets as far as multiplying)
    plan = routed.RoutePlan(torch.zeros(64, dtype=torch.int32), 4, 2, 3)
    bias = torch.zeros(12, requires_grad=True)
    calls = [(l, lambda l: routed.route_topk(l, 2)), (y, lambda y: routed.route_combine(y, ids, w)), (w, lambda w: routed.route_combine(y, ids, w)),
             (x, lambda x: up.mm(x)), (x, lambda x: up.mm_routed(x, plan)), (x, lambda x: routed.experts_forward(x, ids, w, up, down)),
             (w, lambda w: routed.experts_forward(x, ids, w, up, down))]
    for t, call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call(t.clone().requires_grad_())
        with torch.no_grad(), pytest.raises((ValueError, binding.VbrError)) as e:        # gets as far as the GPU that is not there
            call(t.clone().requires_grad_())
        assert "gradient" not in str(e.value)
    with pytest.raises(ValueError, match="on the GPU"):                     # no gradient reaches a bias
        routed.route_topk(l, 2, bias=bias)
    with pytest.raises(ValueError, match="on the GPU"):                     # nor is one lost of a gradient's own operands
        routed.route_topk_grad(l.requires_grad_(), ids, w)


@pytest.mark.gpu
def test_a_router_under_autograd():
    """The router's choice and its gradient inside a function of autograd's."""
    class Weights(torch.autograd.Function):
        @staticmethod
        def forward(ctx, l):
            ids, w = routed.route_topk(l, 3, scale=1.5)
            ctx.save_for_backward(l, ids)
            ctx.mark_non_differentiable(ids)
            return w, ids

        @staticmethod
        def backward(ctx, dw, _):
            l, ids = ctx.saved_tensors
            return routed.route_topk_grad(l, ids, dw.contiguous(), scale=1.5)

    gen = torch.Generator().manual_seed(1)
    l0, dw = torch.randn((30, 20), generator=gen), torch.randn((30, 3), generator=gen)
    l = l0.to(DEV).requires_grad_()
    w, ids = Weights.apply(l)
    (w * dw.to(DEV)).sum().backward()
    want = choice_grad(np64(l0), ids.cpu().numpy().astype(np.int64), np64(dw), "softmax", True, 1.5)
    # every term of the gradient is at most 1.5 |dw|
    assert np.all(np.abs(np64(l.grad) - want) <= U * 400 * 1.5 * np.abs(np64(dw)).sum(1, keepdims=True))


# ------------------------------------------------------------------------------------------- small numbers
@pytest.mark.gpu
@pytest.mark.parametrize("T,N,K,group,zeros,gate", [(1, 200, 288, 32, True, False), (13, 66, 1056, 128, False, False), (16, 12000, 160, 64, True, False), (48, 5456, 288, 128, True, True),
                                                    (130, 16384, 64, 32, True, False), (300, 8192, 160, 64, False, False), (1024, 8200, 96, 128, True, False)])
@pytest.mark.parametrize("what", ["x", "scales", "both"])
def test_products_of_numbers_below_the_normal_ones(T, N, K, group, zeros, gate, what):
    """fp16 has numbers below 2^-14 with fewer bits: they are multiplied and summed as they are, like all others, and nothing of them is lost."""
    gen = torch.Generator().manual_seed(T + N)
    codes, scales, z = matrices(gen, 1, N, K, group, torch.float16, zeros)
    x = torch.randn((T, K), generator=gen)
    if what != "x":
        scales = (scales.float() * 2.0 ** -11).half()                      # 0.02 to 1e-5
    if what != "scales":
        x = x * 2.0 ** torch.randint(-20, -14, (T, 1), generator=gen)
    x, q = x.half(), (codes, scales, z)
    want, tol = product(np64(x), q, 0, group)
    if gate:
        want, tol = gated(want, tol)
    y = on_gpu(q, group, gate).mm(x.to(DEV), y_dtype=torch.float32)
    assert_close(y, want, tol + 2.0 ** -126, torch.float32)
