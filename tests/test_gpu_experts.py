"""A mixture of experts on the GPU: the router against binary64 in numpy, the experts' products against sums in
binary64, and the steps of a decode token one behind the other.

Tolerance of a product as in test_gpu_mx4.py; one rounding more where the router's weight multiplies a slice's sum."""
import numpy as np
import pytest

import teal_inputs as ti
from test_gpu_mx4 import T, dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ---- the router ----

def route_reference(logits, bias, sigmoid, groups, top_groups, group_top, top_k, renormalise, scaling):
    z = np.where(np.isnan(logits), -np.inf, np.minimum(logits, np.finfo(np.float32).max)).astype(np.float64)
    tokens, experts = z.shape
    with np.errstate(all="ignore"):
        if sigmoid:
            score = 1 / (1 + np.exp(-z))
        else:
            top = z.max(-1, keepdims=True)
            e = np.where(z == -np.inf, 0.0, np.exp(z - top))
            score = np.where(e > 0, e / e.sum(-1, keepdims=True), 0.0)
    biased = score + (0 if bias is None else bias.astype(np.float64))
    order = z.copy() if bias is None else np.where(np.isnan(biased), -np.inf, biased)
    if groups > 1:
        size = experts // groups
        by = order if group_top == 1 or bias is not None else score
        value = np.sort(by.reshape(tokens, groups, size), -1)[..., -group_top:].sum(-1)
        first = np.argsort(-value, -1, kind="stable")[:, :top_groups]
        open_ = np.zeros((tokens, groups), bool)
        np.put_along_axis(open_, first, True, -1)
        shut = ~np.repeat(open_, size, -1)
    else:
        shut = np.zeros_like(z, bool)
    # the shut ones behind all others, also behind those of -infinity; ties by number
    idx = np.stack([np.lexsort((np.arange(experts), -o, s))[:top_k] for o, s in zip(order, shut)])
    weight = np.take_along_axis(score, idx, -1)
    if renormalise:
        total = weight.sum(-1, keepdims=True)
        weight = np.divide(weight, total, out=np.zeros_like(weight), where=total > 0)
    return idx, weight * float(np.float32(scaling))


def run_route(T, logits, bias, sigmoid, groups, top_groups, group_top, top_k, renormalise, scaling):   # noqa: F811
    tokens, experts = logits.shape
    idx = torch.full((tokens + 1, top_k), -7, dtype=torch.int32, device="cuda")
    weight = torch.full((tokens + 1, top_k), 7.0, device="cuda")
    T.check(T.teal_route_experts(dev(logits), None if bias is None else dev(bias), int(sigmoid), tokens, experts, groups,
                                 top_groups, group_top, top_k, renormalise, scaling, idx, weight))
    assert bool((idx[tokens] == -7).all()) and bool((weight[tokens] == 7.0).all())
    return idx[:tokens].cpu().numpy(), weight[:tokens].cpu().numpy().astype(np.float64)


def check_route(T, logits, bias, *how):   # noqa: F811
    idx, weight = run_route(T, logits, bias, *how)
    want_idx, want = route_reference(logits, bias, *how)
    assert np.array_equal(idx, want_idx)
    # one rounding to fp32, or to its smallest number, and what two exponential functions differ by
    assert np.all(np.abs(weight - want) <= np.abs(want) * (2.0 ** -24 + 2.0 ** -48) + 2.0 ** -149)


CASES = [(1, 1, 1, 1, 1, 1), (1, 4, 1, 1, 1, 2), (5, 8, 1, 1, 1, 8), (3, 33, 1, 1, 1, 32), (64, 60, 1, 1, 1, 4),
         (7, 64, 1, 1, 1, 6), (65, 64, 8, 3, 2, 6), (33, 65, 5, 2, 1, 4), (9, 128, 4, 1, 2, 8), (300, 256, 8, 4, 2, 8),
         (17, 256, 64, 9, 2, 8), (2, 333, 3, 2, 2, 10), (11, 512, 16, 16, 1, 8), (4, 1024, 1, 1, 1, 32), (3, 1024, 32, 5, 2, 16),
         (5, 24, 24, 7, 2, 7)]


@pytest.mark.parametrize("tokens,experts,groups,top_groups,group_top,top_k", CASES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_route_against_binary64(T, tokens, experts, groups, top_groups, group_top, top_k, sigmoid, biased):   # noqa: F811
    rng = np.random.default_rng(experts + tokens)
    logits = (1.5 * rng.standard_normal((tokens, experts))).astype(np.float32)
    bias = (0.05 * rng.standard_normal(experts)).astype(np.float32) if biased else None
    for renormalise, scaling in [(True, 1.0), (False, 2.5)]:
        check_route(T, logits, bias, sigmoid, groups, top_groups, group_top, top_k, renormalise, scaling)


@pytest.mark.parametrize("tokens,experts,groups,top_groups,group_top,top_k", CASES)
def test_route_takes_the_lowest_number_of_equal_ones(T, tokens, experts, groups, top_groups, group_top, top_k):   # noqa: F811
    rng = np.random.default_rng(experts)
    logits = rng.integers(-1, 2, (tokens, experts)).astype(np.float32)
    bias = (rng.integers(0, 2, experts) / 4).astype(np.float32)
    for b in (None, bias):
        check_route(T, logits, b, True, groups, top_groups, group_top, top_k, True, 1.0)
    logits[:] = 0.5
    check_route(T, logits, None, False, groups, top_groups, group_top, top_k, False, 1.0)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_route_of_masked_infinite_and_nan_logits(T, sigmoid, biased, groups):   # noqa: F811
    rng = np.random.default_rng(5)
    logits = rng.standard_normal((12, 48)).astype(np.float32)
    logits[0] = -np.inf                                        # nothing is left
    logits[1, 3:] = -np.inf                                    # less than top_k is left
    logits[2, ::2] = -np.inf
    logits[3, 5] = np.inf
    logits[4, [5, 40]] = np.inf
    logits[5, 7] = np.nan
    logits[6] = np.nan
    logits[7] = np.finfo(np.float32).min                       # masks of the type's lowest value
    logits[8, 4:] = np.finfo(np.float32).min
    logits[9] = 3e38
    logits[10] *= 1e4                                          # scores that underflow
    logits[11] = 0
    bias = (0.1 * rng.standard_normal(48)).astype(np.float32) if biased else None
    for top_groups, group_top in [(groups, 1), (max(1, groups // 2), 2)]:
        if not biased and group_top == 2:
            rows = [r for r in range(12) if r != 10]           # groups of scores that are zero in one library and not in the other
        else:
            rows = list(range(12))
        for renormalise in (False, True):
            check_route(T, logits[rows], bias, sigmoid, groups, top_groups, group_top, 6, renormalise, 1.0)


@pytest.mark.parametrize("tokens", [40, 8195])
@pytest.mark.parametrize("experts,groups,top_groups,group_top,top_k", [(256, 8, 4, 2, 8), (64, 1, 1, 1, 6), (128, 4, 2, 1, 15),
                                                                      (1000, 1, 1, 1, 8), (60, 5, 2, 2, 4)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_route_of_scores_next_to_each_other(T, tokens, experts, groups, top_groups, group_top, top_k, sigmoid):   # noqa: F811
    """Sums of score and bias that differ by less than an fp32 score can tell, in experts and in groups, and equal ones;
    biases much larger than the scores."""
    rng = np.random.default_rng(experts + tokens)
    z = rng.standard_normal(experts).astype(np.float32)
    score = 1 / (1 + np.exp(-z.astype(np.float64)))
    bias = (0.75 - score).astype(np.float32)                   # with sigmoid scores all sums are 0.75 to within 2^-25
    logits = np.tile(z, (tokens, 1))
    logits[1::4] += (1e-7 * rng.integers(-3, 4, (len(logits[1::4]), experts))).astype(np.float32)
    logits[2::4] += rng.standard_normal((len(logits[2::4]), experts)).astype(np.float32)
    logits[3::4] = 0.25
    for b in (bias, 1000 * bias, np.where(np.arange(experts) % 7 == 0, np.float32(1e30), bias).astype(np.float32), None):
        check_route(T, logits, b, sigmoid, groups, top_groups, group_top, top_k, True, 1.0)


@pytest.mark.parametrize("experts,groups,top_groups,group_top,top_k", [(256, 8, 4, 2, 8), (64, 4, 1, 1, 4), (48, 3, 2, 2, 15), (16, 16, 7, 1, 5),
                                                                      (32, 16, 5, 2, 6), (512, 8, 3, 2, 8)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_route_of_groups_next_to_each_other(T, experts, groups, top_groups, group_top, top_k, sigmoid):   # noqa: F811
    """Groups of the same experts in other orders, whose largest differ by less than an fp32 score can tell, next to tokens
    of ordinary groups."""
    rng = np.random.default_rng(experts + groups)
    tokens, size = 402, experts // groups
    one = np.sort(rng.standard_normal((tokens, 1, size)), -1)
    logits = rng.permuted(np.tile(one, (1, groups, 1)), axis=-1)
    logits = (logits * (1 + 2e-7 * rng.standard_normal((tokens, groups, size)))).reshape(tokens, experts).astype(np.float32)
    logits[1::3] = rng.standard_normal((len(logits[1::3]), experts))
    for bias in (None, np.full(experts, 0.125, np.float32)):
        check_route(T, logits, bias, sigmoid, groups, top_groups, group_top, top_k, True, 1.0)


@pytest.mark.parametrize("experts,groups,top_groups,group_top,top_k", [(256, 8, 4, 2, 8), (128, 1, 1, 1, 8), (64, 8, 3, 1, 15),
                                                                      (60, 1, 1, 1, 4), (256, 1, 1, 1, 17), (512, 8, 2, 2, 6)])
@pytest.mark.parametrize("sigmoid,biased", [(False, False), (False, True), (True, False), (True, True)])
def test_route_of_many_tokens(T, experts, groups, top_groups, group_top, top_k, sigmoid, biased):   # noqa: F811
    rng = np.random.default_rng(experts)
    logits = (1.5 * rng.standard_normal((8194, experts))).astype(np.float32)
    logits[100, ::3] = -np.inf
    logits[8193] = np.nan
    bias = (0.05 * rng.standard_normal(experts)).astype(np.float32) if biased else None
    check_route(T, logits, bias, sigmoid, groups, top_groups, group_top, top_k, sigmoid, 2.5)


@pytest.mark.parametrize("size,groups", [(11, 4), (11, 8), (3, 5), (1, 16), (2, 7), (17, 8), (33, 15), (128, 3), (129, 2), (32, 16), (20, 6),
                                         (33, 16), (5, 17), (255, 4)])
@pytest.mark.parametrize("sigmoid,biased", [(False, False), (False, True), (True, False), (True, True)])
def test_route_of_groups_of_any_size(T, size, groups, sigmoid, biased):   # noqa: F811
    rng = np.random.default_rng(100 * size + groups)
    experts = size * groups
    logits = rng.standard_normal((150, experts)).astype(np.float32)
    logits[3, :size] = -np.inf                                 # groups with nothing in them
    logits[4, size:] = -np.inf
    logits[5] = 0.5
    logits[6::10] = np.round(2 * logits[6::10]) / 2            # many equal ones
    bias = (0.1 * rng.standard_normal(experts)).astype(np.float32) if biased else None
    for top_groups in {1, groups // 2, groups - 1, groups}:
        for group_top in (1, 2):
            # the sum of two scores of a softmax over few equal logits is a matter of its rounding
            rows = [r for r in range(150) if sigmoid or group_top == 1 or r not in range(6, 150, 10)]
            check_route(T, logits[rows], bias, sigmoid, groups, top_groups, group_top, min(7, top_groups * size), True, 1.0)


@pytest.mark.parametrize("experts,groups", [(64, 1), (400, 1), (256, 8), (15, 1), (48, 3)])
def test_route_of_logits_that_begin_anywhere(T, experts, groups):   # noqa: F811
    rng = np.random.default_rng(experts)
    logits = rng.standard_normal((21, experts)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(experts)).astype(np.float32)
    room = torch.empty(21 * experts + experts + 8, device="cuda")
    idx, weight = torch.empty(21, 4, dtype=torch.int32, device="cuda"), torch.empty(21, 4, device="cuda")
    for shift in range(4):
        z, b = room[shift:shift + 21 * experts], room[21 * experts + 4 + shift % 2:][:experts]
        z.copy_(dev(logits.ravel()))
        b.copy_(dev(bias))
        for used in (None, b):
            T.check(T.teal_route_experts(z, used, 1, 21, experts, groups, groups, 1, 4, True, 1.0, idx, weight))
            how = (True, groups, groups, 1, 4, True, 1.0)
            assert np.array_equal(idx.cpu().numpy(), route_reference(logits, None if used is None else bias, *how)[0])


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("groups", [1, 4])
def test_route_with_a_bias_that_is_no_number(T, value, groups):   # noqa: F811
    rng = np.random.default_rng(9)
    logits = rng.standard_normal((6, 64)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(64)).astype(np.float32)
    bias[[3, 40]] = value
    idx, _ = run_route(T, logits, bias, True, groups, max(1, groups // 2), 1, 6, True, 1.0)
    assert np.array_equal(idx, route_reference(logits, bias, True, groups, max(1, groups // 2), 1, 6, True, 1.0)[0])


def test_route_in_a_graph_and_on_another_stream(T):   # noqa: F811
    rng = np.random.default_rng(8)
    first, second = rng.standard_normal((2, 8, 128)).astype(np.float32)
    logits = dev(first)
    idx, weight = torch.empty(8, 4, dtype=torch.int32, device="cuda"), torch.empty(8, 4, device="cuda")
    call = lambda **kw: T.check(T.teal_route_experts(logits, None, 0, 8, 128, 1, 1, 1, 4, True, 1.0, idx, weight, **kw))   # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a in (first, second, first, second):
        logits.copy_(dev(a))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(idx.cpu().numpy(), route_reference(a, None, False, 1, 1, 1, 4, True, 1.0)[0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    call(stream=stream)
    stream.synchronize()
    assert np.array_equal(idx.cpu().numpy(), route_reference(second, None, False, 1, 1, 1, 4, True, 1.0)[0])


# ---- the experts' products ----

class Experts:
    """count matrices of [experts][m][n] in a format: what a call takes, and their values in binary64."""

    def __init__(self, fmt, experts, m, widths, seed):
        self.fmt, self.experts, self.m, self.widths = fmt, experts, m, widths
        self.args, self.values = [], []
        for k, n in enumerate(widths):
            if fmt == "mx4":
                made = [ti.random_mx4(m, n, seed + 100 * k + e) for e in range(experts)]
                self.args.append((dev(np.stack([c for c, _ in made])), dev(np.stack([s for _, s in made]))))
                self.values.append([ti.mx4_values(c, s) for c, s in made])
            else:
                made = [ti.weights_bf16(n, m, seed + 100 * k + e) for e in range(experts)]
                self.args.append((dev(np.stack([ti.to_input_channel_major(w) for w in made])),))
                self.values.append([ti.bf16_bits_to_f32(w).T.astype(np.float64) for w in made])

    def __call__(self, T, t, ys, idx, x, ws, **kw):   # noqa: F811
        call = T.teal_sparse_experts_mx4 if self.fmt == "mx4" else T.teal_sparse_experts_bf16
        T.check(call(*map(list, zip(*self.args)), t, ys, self.widths, self.experts, idx, *idx.shape, x, self.m, ws, **kw))

    def down(self, T, t, y, idx, weight, gate, up, ws, **kw):   # noqa: F811
        call = T.teal_sparse_experts_mx4_swiglu if self.fmt == "mx4" else T.teal_sparse_experts_bf16_swiglu
        T.check(call(*self.args[0], t, y, self.experts, idx, weight, *idx.shape, gate, up, self.m, self.widths[0], ws, **kw))


def expert_workspace(T, m, n, pairs):   # noqa: F811
    return torch.zeros(T.teal_workspace_bytes_experts(m, n, pairs), dtype=torch.uint8, device="cuda")


def product(x, t, values):
    """(product, bound of its error) of one token and expert."""
    kept = np.abs(x.astype(np.float64)) > t
    xk, wk = x[kept].astype(np.float64), values[kept]
    with np.errstate(invalid="ignore"):                      # (infinite inputs)
        return xk @ wk, (kept.sum() / 8 + 65) * 2.0 ** -24 * (np.abs(xk) @ np.abs(wk))


def choose(rng, tokens, experts, top_k):
    idx = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)       # the same expert may occur again
    idx[-1, 0] = -1
    if tokens > 2:
        idx[1] = [experts, -5, 2 ** 31 - 1, -2 ** 31][:top_k] + [-1] * (top_k - 4)
    return idx


SIZES = [(1, 4, 1, 64, [32], 0.5), (1, 8, 2, 1000, [96, 352], 0.5), (3, 5, 2, 129, [64, 64], 0.0), (8, 16, 4, 513, [544, 96], 0.5),
         (2, 3, 2, 4500, [256], 0.8), (8, 4, 8, 640, [768, 768], 0.5), (4, 2, 3, 2048, [1024, 1024, 64, 32], 0.95),
         (8, 3, 32, 200, [1056], 0.5), (1, 2, 2, 2048, [4096, 4096], 0.5), (5, 6, 1, 33, [64], 1.0),
         (8, 3, 8, 4200, [1536, 1536], 0.9), (1, 2, 1, 70001, [32], 0.5), (2, 1, 1, 8200, [96, 64], 0.25)]


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,experts,top_k,m,widths,p", SIZES)
def test_experts_against_binary64(T, fmt, tokens, experts, top_k, m, widths, p):   # noqa: F811
    rng = np.random.default_rng(m + tokens)
    ex = Experts(fmt, experts, m, widths, m)
    x = rng.standard_normal((tokens, m)).astype(np.float16)
    base = ti.quantile_threshold(x.ravel(), p)
    ts = [(base * rng.uniform(0.8, 1.2, experts)).astype(np.float32) if p < 1 else np.full(experts, base, np.float32)
          for _ in widths]
    idx = choose(rng, tokens, experts, top_k)
    ws = expert_workspace(T, m, sum(widths), tokens * top_k)
    ys = [torch.full((tokens * top_k * n + 8,), 7.0, device="cuda") for n in widths]
    args = [dev(t) for t in ts], ys, dev(idx), dev(x), ws
    ex(T, *args)
    first = [y.clone() for y in ys]
    for k, n in enumerate(widths):
        got = ys[k][:-8].cpu().numpy().astype(np.float64).reshape(tokens, top_k, n)
        assert bool((ys[k][-8:] == 7.0).all())
        for b in range(tokens):
            for j in range(top_k):
                e = idx[b, j]
                if not 0 <= e < experts:
                    assert not got[b, j].any()
                    continue
                want, bound = product(x[b], ts[k][e], ex.values[k][e])
                assert np.all(np.abs(got[b, j] - want) <= bound), (b, j, k)
    for _ in range(2):
        ex(T, *args)
        assert all(torch.equal(a, b) for a, b in zip(first, ys))


DOWN = [(1, 4, 1, 64, 32, 0.5), (1, 8, 2, 1000, 96, 0.5), (3, 5, 2, 129, 544, 0.0), (8, 16, 4, 513, 1056, 0.5),
        (2, 3, 2, 4500, 256, 0.8), (8, 4, 8, 768, 2048, 0.5), (1, 2, 32, 640, 64, 0.5), (1, 3, 8, 20000, 64, 0.5),
        (4, 3, 2, 2048, 512, 0.95), (1, 2, 2, 3584, 1024, 0.5), (5, 6, 1, 33, 64, 1.0),
        (8, 3, 8, 4200, 2048, 0.9), (1, 2, 1, 70001, 32, 0.5), (8, 2, 32, 130, 1024, 0.5)]


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,experts,top_k,m,n,p", DOWN)
def test_experts_down_against_binary64(T, fmt, tokens, experts, top_k, m, n, p):   # noqa: F811
    rng = np.random.default_rng(m + n)
    ex = Experts(fmt, experts, m, [n], n)
    gate, up = (1.5 * rng.standard_normal((tokens, top_k, m))).astype(np.float32), rng.standard_normal((tokens, top_k, m)).astype(np.float32)
    gd, ud = dev(gate), dev(up)
    h = torch.empty(tokens, top_k, m, dtype=torch.float16, device="cuda")
    T.check(T.teal_swiglu_f16(gd, ud, h, h.numel()))
    h = h.cpu().numpy()
    base = ti.quantile_threshold(h.ravel(), p)
    t = (base * rng.uniform(0.8, 1.2, experts)).astype(np.float32) if p < 1 else np.full(experts, base, np.float32)
    idx = choose(rng, tokens, experts, top_k)
    weight = rng.uniform(0, 1, (tokens, top_k)).astype(np.float32)
    weight[-1, 0] = np.nan                                      # of a pair without an expert
    ws = expert_workspace(T, m, n, tokens * top_k)
    y = torch.full((tokens * n + 8,), 7.0, device="cuda")
    args = dev(t), y, dev(idx), dev(weight), gd, ud, ws
    ex.down(T, *args)
    first = y.clone()
    got = y[:-8].cpu().numpy().astype(np.float64).reshape(tokens, n)
    assert bool((y[-8:] == 7.0).all())
    slices = top_k * 16                                         # at most; added in fp32 where they are more than 32
    for b in range(tokens):
        want, bound, size = np.zeros(n), np.zeros(n), np.zeros(n)
        for j in range(top_k):
            e = idx[b, j]
            if 0 <= e < experts:
                one, off = product(h[b, j], t[e], ex.values[0][e])
                want += weight[b, j] * one
                bound += weight[b, j] * off
                size += weight[b, j] * np.abs(h[b, j].astype(np.float64)) @ np.abs(ex.values[0][e])
        assert np.all(np.abs(got[b] - want) <= bound + (slices + 1) * 2.0 ** -24 * size), b
    for _ in range(2):
        ex.down(T, *args)
        assert torch.equal(first, y)


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,m,n", [(8, 8, 4200, 1536), (1, 32, 640, 64), (1, 8, 20000, 64), (8, 32, 130, 1024), (2, 2, 2048, 512),
                                              (3, 1, 9000, 2048)])
def test_a_workspace_is_as_large_as_it_is_said_to_be(T, fmt, tokens, top_k, m, n):   # noqa: F811
    """Sums of unusual size take the way through the partial rows in every launch shape: nothing behind the workspace is
    written, and the next call, of other sizes, finds it as it should be."""
    ex, down = Experts(fmt, 2, m, [n], 3), Experts(fmt, 2, m, [n], 4)
    rng = np.random.default_rng(6)
    need = T.teal_workspace_bytes_experts(m, n, tokens * top_k)
    room = torch.full((need + 4096,), 0xEE, dtype=torch.uint8, device="cuda")
    ws = room[:need]
    ws.zero_()
    idx = dev(rng.integers(0, 2, (tokens, top_k)).astype(np.int32))
    t = torch.zeros(2, device="cuda")
    for size in (2.0 ** -14, 1.0, 2.0 ** 13):
        x = (rng.standard_normal((tokens, m)) * size).astype(np.float16)
        y = torch.empty(tokens, top_k, n, device="cuda")
        ex(T, [t], [y], idx, dev(x), ws)
        gate, up = rng.standard_normal((2, tokens, top_k, m)).astype(np.float32)
        up *= np.float32(size)
        z = torch.empty(tokens, n, device="cuda")
        weight = torch.full((tokens, top_k), 0.75, device="cuda")
        down.down(T, t, z, idx, weight, dev(gate), dev(up), ws)
        chosen = idx.cpu().numpy()
        h = torch.empty(tokens, top_k, m, dtype=torch.float16, device="cuda")
        T.check(T.teal_swiglu_f16(dev(gate), dev(up), h, h.numel()))
        h = h.cpu().numpy()
        for b in (0, tokens - 1):
            want, bound = product(x[b], 0, ex.values[0][chosen[b, 0]])
            assert np.all(np.abs(y[b, 0].cpu().numpy() - want) <= bound)
            parts = [product(h[b, j], 0, down.values[0][chosen[b, j]]) for j in range(top_k)]
            want, off = 0.75 * sum(w for w, _ in parts), sum(o for _, o in parts)
            # what more than 32 slices are added in fp32 with is, slice by slice, within a last place of sums whose
            # magnitudes the bounds of the products have too
            got = z[b].cpu().numpy()
            with np.errstate(invalid="ignore"):              # (some h are infinite: then so is what has to come out)
                assert np.all((got == want) | np.isnan(got) & np.isnan(want) | (np.abs(got - want) <= off * (1 + 16 * top_k / 65)) & np.isfinite(want))
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xEE).all())
    assert not bool(ws[:T.teal_survivors_offset()].any())           # ready for the next call


def test_experts_on_two_streams(T):   # noqa: F811
    ex = Experts("mx4", 6, 1024, [512, 512], 2)
    rng = np.random.default_rng(2)
    x, idx = dev(rng.standard_normal((4, 1024)).astype(np.float16)), dev(rng.integers(0, 6, (4, 2)).astype(np.int32))
    t = [torch.full((6,), 0.7, device="cuda")] * 2
    spaces = [expert_workspace(T, 1024, 1024, 8) for _ in range(2)]
    ys = [[torch.empty(4, 2, 512, device="cuda") for _ in range(2)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, ws, y in zip(streams, spaces, ys):
            ex(T, t, y, idx, x, ws, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*ys))
    want, bound = product(x[3].cpu().numpy(), float(t[0][0]), ex.values[1][int(idx[3, 1])])
    assert np.all(np.abs(ys[0][1][3, 1].cpu().numpy() - want) <= bound)


def test_thresholds_that_no_call_would_accept_count_as_zero(T):   # noqa: F811
    ex = Experts("bf16", 3, 70, [64], 1)
    x, idx = dev(ti.gaussian_x(70, 2)[None]), dev(np.array([[0, 1, 2]], np.int32))
    ys, ws = [[torch.empty(1, 3, 64, device="cuda")] for _ in range(2)], expert_workspace(T, 70, 64, 3)
    ex(T, [dev(np.array([-1.0, np.nan, 0.0], np.float32))], ys[0], idx, x, ws)
    ex(T, [dev(np.zeros(3, np.float32))], ys[1], idx, x, ws)
    assert torch.equal(ys[0][0], ys[1][0])


def test_expert_weights_past_32_bits(T):   # noqa: F811
    experts, m, n = 40, 4096, 14336                            # 4.7 GB of bf16 weights
    w = torch.zeros(experts, m, n, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    w[39] = 0.02 * torch.randn(m, n, generator=g, device="cuda").bfloat16()
    x = ti.gaussian_x(m, 4)
    t = ti.quantile_threshold(x, 0.5)
    y, ws = torch.empty(1, 1, n, device="cuda"), expert_workspace(T, m, n, 1)
    idx = dev(np.array([[39]], np.int32))
    T.check(T.teal_sparse_experts_bf16([w], [torch.full((experts,), t, device="cuda")], [y], [n], experts, idx, 1, 1, dev(x), m, ws))
    want, bound = product(x, t, w[39].double().cpu().numpy())
    assert np.all(np.abs(y[0, 0].cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_a_token_through_router_and_experts(T, fmt):   # noqa: F811
    """Weights laid out, a router's product, its choice, gate and up, W_down: eagerly, and captured and replayed with
    eager calls of another size on the same workspace in between."""
    rng = np.random.default_rng(31)
    d, f, experts, tokens, top_k = 1024, 416, 24, 4, 3
    pack = {"bf16": lambda w: ti.to_input_channel_major(w), "mx4": lambda w: w}[fmt]
    gate_up, down = Experts("bf16", 1, 32, [32], 1), Experts("bf16", 1, 32, [32], 1)
    for ex, m, widths in ((gate_up, d, [f, f]), (down, f, [d])):
        ex.fmt, ex.experts, ex.m, ex.widths, ex.args, ex.values = fmt, experts, m, widths, [], []
        for k, n in enumerate(widths):
            ws_ = [ti.weights_bf16(n, m, 1000 * k + e + m) for e in range(experts)]
            if fmt == "bf16":
                ex.args.append((dev(np.stack([pack(w) for w in ws_])),))
                ex.values.append([ti.bf16_bits_to_f32(w).T.astype(np.float64) for w in ws_])
                continue
            size = T.teal_mx4_scale_bytes(m, n)
            q = torch.empty(experts, m, n // 2, dtype=torch.uint8, device="cuda")
            s = torch.empty(experts, size, dtype=torch.uint8, device="cuda")
            for e, w in enumerate(ws_):
                T.check(T.teal_pack_mx4(dev(w), q[e], s[e], m, n))
            ex.args.append((q, s))
            ex.values.append([ti.mx4_values(*ti.quantize_mx4(w)) for w in ws_])
    router = ti.weights_bf16(experts, d, 77)
    router_t = dev(ti.to_input_channel_major(router))
    x = torch.empty(tokens, d, dtype=torch.float16, device="cuda")
    t = [torch.full((experts,), v, device="cuda") for v in (0.6, 0.5, 0.01)]
    logits = torch.empty(tokens, experts, device="cuda")
    idx, weight = torch.empty(tokens, top_k, dtype=torch.int32, device="cuda"), torch.empty(tokens, top_k, device="cuda")
    gu = [torch.empty(tokens, top_k, f, device="cuda") for _ in range(2)]
    y = torch.empty(tokens, d, device="cuda")
    ws = torch.zeros(max(T.teal_workspace_bytes_experts(d, 2 * f, tokens * top_k), T.teal_workspace_bytes_experts(f, d, tokens * top_k),
                         T.teal_workspace_bytes_batch(d, experts, tokens)), dtype=torch.uint8, device="cuda")

    def step():
        T.check(T.teal_sparse_gemv_bf16_batch(router_t, x, tokens, 0.0, logits, d, experts, ws))
        T.check(T.teal_route_experts(logits, None, T.TEAL_SCORE_SOFTMAX, tokens, experts, 1, 1, 1, top_k, True, 1.0, idx, weight))
        gate_up(T, t[:2], gu, idx, x, ws)
        down.down(T, t[2], y, idx, weight, gu[0], gu[1], ws)

    def compare(xn):
        chosen, w, (gate, up) = idx.cpu().numpy(), weight.cpu().numpy().astype(np.float64), (v.cpu().numpy() for v in gu)
        want_idx, want_w = route_reference(logits.cpu().numpy(), None, False, 1, 1, 1, top_k, True, 1.0)
        assert np.array_equal(chosen, want_idx) and np.allclose(w, want_w, rtol=2.0 ** -23, atol=0)
        h = torch.empty(tokens, top_k, f, dtype=torch.float16, device="cuda")
        T.check(T.teal_swiglu_f16(gu[0], gu[1], h, h.numel()))
        h = h.cpu().numpy()
        for b in range(tokens):
            total, off = np.zeros(d), np.zeros(d)
            for j in range(top_k):
                e = chosen[b, j]
                for k, got in enumerate((gate, up)):
                    want, bound = product(xn[b], float(t[k][e]), gate_up.values[k][e])
                    assert np.all(np.abs(got[b, j] - want) <= bound)
                want, bound = product(h[b, j], float(t[2][e]), down.values[0][e])
                total, off = total + w[b, j] * want, off + w[b, j] * bound
            # three products of at most 16 slices each meet in a sum; their roundings are in the products' bounds,
            # whose sums of magnitudes they are relative to
            assert np.all(np.abs(y[b].cpu().numpy() - total) <= 2 * off)

    inputs = [rng.standard_normal((tokens, d)).astype(np.float16) for _ in range(3)]
    x.copy_(dev(inputs[0]))
    step()
    compare(inputs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = Experts(fmt, 2, 96, [64], 5)
    for xn in inputs + inputs[:1]:
        x.copy_(dev(xn))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        compare(xn)
        replayed = y.clone()
        other(T, [torch.zeros(2, device="cuda")], [torch.empty(4, 2, 64, device="cuda")],
              torch.ones(4, 2, dtype=torch.int32, device="cuda"), torch.ones(4, 96, dtype=torch.float16, device="cuda"), ws)
        step()
        assert torch.equal(y, replayed)
