"""The experts' calls, the router and microscaled products at the ends of their ranges: infinite thresholds, sums of unusual
size that are finite, groups of many equal scores, sums that are no number, infinite weights, the longest inputs.

Tolerances of products as in test_gpu_mx4.py and test_gpu_experts.py."""
import numpy as np
import pytest

import teal_inputs as ti
from test_gpu_experts import Experts, check_route, expert_workspace, product
from test_gpu_mx4 import T, dev, workspace  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def whole_sum(x, t, values):
    """The product term by term, infinities and NaN included."""
    kept = np.abs(x.astype(np.float64)) > t
    with np.errstate(invalid="ignore"):
        return (x[kept].astype(np.float64)[:, None] * values[kept]).sum(0)


INFINITE = [(1, 4, 70, 64), (2, 3, 1000, 96), (8, 8, 4200, 1536)]       # slices of every way of compaction


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,m,n", INFINITE)
def test_nothing_is_above_an_infinite_threshold(T, fmt, tokens, top_k, m, n):   # noqa: F811
    """Not even an infinite input, which every finite threshold keeps, also those beyond fp16."""
    rng = np.random.default_rng(m)
    t = np.array([np.inf, 7e4, 0.5, np.inf, 3e38], np.float32)
    ex = Experts(fmt, 5, m, [n], m)
    x = rng.standard_normal((tokens, m)).astype(np.float16)
    x[0, 5], x[0, m - 1], x[0, 9], x[-1, 11] = np.inf, -np.inf, 65504, np.nan
    idx = ((np.arange(tokens)[:, None] + np.arange(top_k)) % 5).astype(np.int32)
    idx[0, -1] = 4                          # the infinite inputs with the largest finite threshold, too
    y = torch.full((tokens, top_k, n), 7.0, device="cuda")
    ex(T, [dev(t)], [y], dev(idx), dev(x), expert_workspace(T, m, n, tokens * top_k))
    got = y.cpu().numpy()
    for b in range(tokens):
        for j in range(top_k):
            e = idx[b, j]
            if t[e] == np.inf or b and t[e] > 65504:
                assert not got[b, j].any(), (b, j)
            elif b == 0:
                assert np.array_equal(got[b, j], whole_sum(x[b], t[e], ex.values[0][e]), equal_nan=True), (b, j)
            else:
                want, bound = product(x[b], t[e], ex.values[0][e])
                assert np.all(np.abs(got[b, j] - want) <= bound), (b, j)


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,m,n", INFINITE)
def test_an_expert_with_an_infinite_threshold_adds_nothing(T, fmt, tokens, top_k, m, n):   # noqa: F811
    """Also as a token's first expert, whose threshold the slices of the others are added by."""
    rng = np.random.default_rng(n)
    t = np.array([np.inf, 0.5, 0.25], np.float32)
    ex = Experts(fmt, 3, m, [n], n)
    idx = (np.arange(top_k) % 3 * np.ones((tokens, 1))).astype(np.int32)
    idx[-1] = 0 if tokens > 1 else idx[-1]
    gate, up = rng.uniform(0.5, 3, (tokens, top_k, m)).astype(np.float32), rng.standard_normal((tokens, top_k, m)).astype(np.float32)
    up[idx == 0, 3] = np.inf
    up[idx == 0, m - 1] = -np.inf
    weight = rng.uniform(0.1, 1, (tokens, top_k)).astype(np.float32)
    h = torch.empty(tokens, top_k, m, dtype=torch.float16, device="cuda")
    T.check(T.teal_swiglu_f16(dev(gate), dev(up), h, h.numel()))
    h = h.cpu().numpy()
    assert np.isinf(h[idx == 0]).any() and np.isfinite(h[idx > 0]).all()
    y = torch.full((tokens, n), 7.0, device="cuda")
    ex.down(T, dev(t), y, dev(idx), dev(weight), dev(gate), dev(up), expert_workspace(T, m, n, tokens * top_k))
    got = y.cpu().numpy().astype(np.float64)
    for b in range(tokens):
        want, bound, size = np.zeros(n), np.zeros(n), np.zeros(n)
        for j in range(top_k):
            if idx[b, j]:
                one, off = product(h[b, j], t[idx[b, j]], ex.values[0][idx[b, j]])
                want += weight[b, j] * one
                bound += weight[b, j] * off
                size += weight[b, j] * np.abs(h[b, j].astype(np.float64)) @ np.abs(ex.values[0][idx[b, j]])
        assert np.all(np.abs(got[b] - want) <= bound + (top_k * 16 + 1) * 2.0 ** -24 * size), b
    if tokens > 1:
        assert not got[-1].any()


@pytest.mark.parametrize("m,n", [(300, 96), (2048, 1024), (16384, 64)])
def test_finite_thresholds_beyond_fp16_keep_infinite_inputs(T, m, n):   # noqa: F811
    w = ti.weights_bf16(n, m, 3)
    values = ti.bf16_bits_to_f32(w).T.astype(np.float64)
    wt, x = dev(ti.to_input_channel_major(w)), ti.gaussian_x(m, 4)
    x[7], x[m // 2], x[9] = 65504, -np.inf, np.nan
    y, ws = torch.empty(n, device="cuda"), workspace(T, m, n)
    for t in (65503.9, 65504.0, 65520.0, 1e5, 3.4e38):
        T.check(T.teal_sparse_gemv_bf16(wt, dev(x), t, y, m, n, ws))
        assert np.array_equal(y.cpu().numpy(), whole_sum(x, np.float32(t), values), equal_nan=True), t


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,m,n", [(8, 8, 4200, 1536), (1, 32, 640, 64), (1, 8, 20000, 64), (8, 32, 130, 1024), (2, 2, 2048, 512),
                                              (3, 1, 9000, 2048)])
def test_finite_sums_of_unusual_size(T, fmt, tokens, top_k, m, n):   # noqa: F811
    """Every slice of every expert counts once where the sums take the way past the column words: their size is in the
    router's weights, so that nothing is infinite."""
    ex = Experts(fmt, 2, m, [n], 4)
    rng = np.random.default_rng(6)
    need = T.teal_workspace_bytes_experts(m, n, tokens * top_k)
    room = torch.full((need + 4096,), 0xEE, dtype=torch.uint8, device="cuda")
    ws = room[:need]
    ws.zero_()
    idx = rng.integers(0, 2, (tokens, top_k)).astype(np.int32)
    for scale in (2.0 ** -30, 2.0 ** -14, 1.0, 2.0 ** 13, 2.0 ** 40):
        gate, up = rng.standard_normal((2, tokens, top_k, m)).astype(np.float32)
        weight = (scale * rng.uniform(0.5, 1, (tokens, top_k))).astype(np.float32)
        h = torch.empty(tokens, top_k, m, dtype=torch.float16, device="cuda")
        T.check(T.teal_swiglu_f16(dev(gate), dev(up), h, h.numel()))
        h = h.cpu().numpy()
        y = torch.empty(tokens, n, device="cuda")
        ex.down(T, torch.zeros(2, device="cuda"), y, dev(idx), dev(weight), dev(gate), dev(up), ws)
        for b in (0, tokens - 1):
            want, bound, size = np.zeros(n), np.zeros(n), np.zeros(n)
            for j in range(top_k):
                one, off = product(h[b, j], 0, ex.values[0][idx[b, j]])
                want += weight[b, j] * one
                bound += weight[b, j] * off
                size += weight[b, j] * np.abs(h[b, j].astype(np.float64)) @ np.abs(ex.values[0][idx[b, j]])
            assert np.isfinite(want).all()
            assert np.all(np.abs(y[b].cpu().numpy() - want) <= bound + (top_k * 16 + 1) * 2.0 ** -24 * size), (scale, b)
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xEE).all())
    assert not bool(ws[:T.teal_survivors_offset()].any())


@pytest.mark.parametrize("size,groups", [(11, 4), (11, 8), (3, 5), (1, 16), (2, 7), (17, 8), (33, 15), (128, 3), (129, 2), (32, 16), (20, 6),
                                         (33, 16), (5, 17), (255, 4)])
@pytest.mark.parametrize("biased", [False, True])
def test_softmax_groups_of_many_equal_scores(T, size, groups, biased):   # noqa: F811
    """Groups valued by their two largest scores, of logits that are multiples of a half: equal logits have the same score,
    so equal groups are equal and the lower number is taken."""
    rng = np.random.default_rng(100 * size + groups)
    experts = size * groups
    logits = (np.round(2 * rng.standard_normal((60, experts))) / 2).astype(np.float32)
    logits[5] = 0.5
    bias = (0.1 * rng.standard_normal(experts)).astype(np.float32) if biased else None
    for top_groups in {1, groups // 2, groups - 1, groups}:
        for renormalise in (True, False):
            check_route(T, logits, bias, False, groups, top_groups, 2, min(7, top_groups * size), renormalise, 1.0)


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("experts,top_k", [(24, 12), (24, 24), (64, 15)])
def test_sums_that_are_no_number_rank_as_the_lowest(T, experts, top_k, groups):   # noqa: F811
    """NaN and -infinity among the biases are equal: by number, behind all others."""
    rng = np.random.default_rng(experts)
    logits = rng.standard_normal((9, experts)).astype(np.float32)
    bias = (0.1 * rng.standard_normal(experts)).astype(np.float32)
    bias[1::3], bias[2::6] = np.nan, -np.inf
    for top_groups, group_top in {(groups, 1), (max(1, groups // 2 + 1), 2)}:
        check_route(T, logits, bias, True, groups, top_groups, group_top, min(top_k, experts // groups * top_groups), True, 1.0)


@pytest.mark.parametrize("experts,top_k", [(8, 3), (64, 6), (64, 16)])
def test_sigmoid_scores_up_to_the_last_that_is_not_zero(T, experts, top_k):   # noqa: F811
    """Renormalised scores of logits down to where exp(-l) leaves binary64, fp32 number by fp32 number at the end."""
    last = np.float32(-709.78265)
    assert np.isfinite(np.exp(-np.float64(last))) and np.exp(709.0) < np.exp(-np.float64(last))
    with np.errstate(over="ignore"):
        assert np.isinf(np.exp(-np.float64(np.nextafter(last, np.float32(-800)))))
    steps = np.arange(-8, 60, dtype=np.float32) * np.float32(2.0 ** -14)
    logits = np.full((len(steps), experts), -800, np.float32)
    logits[:, ::3] = last + steps[:, None]
    logits[::2, 1] = last
    for bias in (None, np.zeros(experts, np.float32)):
        check_route(T, logits, bias, True, 1, 1, 1, top_k, True, 1.0)


@pytest.mark.parametrize("scale", [253, 254])
def test_how_far_an_infinite_weight_reaches(T, scale):   # noqa: F811
    m, n = 520, 96
    codes, scales, x = *ti.random_mx4(m, n, 1), ti.gaussian_x(m, 2)
    x[100], x[101] = 3, 0
    for channel in (100, 101):
        marked, levels = scales.copy(), codes.copy()
        marked[ti.mx4_scale_places(m, n)[channel, 1]] = scale
        levels[channel, 16:32] = 0x11                        # columns 32 to 63: a half
        levels[channel, 16 + 5] = 0x17                       # column 42: six of a scale that makes it infinite
        values = ti.mx4_values(levels, marked)
        y = torch.empty(n, device="cuda")
        T.check(T.teal_sparse_gemv_mx4(dev(levels), dev(marked), dev(x), 0.5, y, m, n, workspace(T, m, n)))
        want, bound = product(x, 0.5, values)
        beside = (np.arange(n) < 40) | (np.arange(n) >= 48) if channel == 100 else np.ones(n, bool)
        with np.errstate(invalid="ignore"):
            assert np.all(np.abs(y.cpu().numpy() - want)[beside] <= bound[beside])


@pytest.mark.parametrize("fmt,n", [("bf16", 8), ("mx4", 32)])
def test_the_longest_inputs(T, fmt, n):   # noqa: F811
    """2^24 channels, 4096 slices, of which a few survive: the sum is what their roundings leave of it."""
    m, rng = 1 << 24, np.random.default_rng(n)
    rows = np.unique(np.concatenate([[0, 1, 4095, 4096, m - 4097, m - 4096, m - 2, m - 1], rng.integers(0, m, 40)]))
    at = dev(rows)
    x = np.zeros(m, np.float16)
    x[rows] = rng.uniform(0.5, 2, len(rows))
    if fmt == "mx4":
        codes = rng.integers(0, 256, (len(rows), n // 2), dtype=np.uint8)
        q = torch.zeros(1, m, n // 2, dtype=torch.uint8, device="cuda")
        q[0, at] = dev(codes)
        s = torch.full((T.teal_mx4_scale_bytes(m, n),), 120, dtype=torch.uint8, device="cuda")
        values = ti.mx4_values(codes, np.full(ti.mx4_scale_bytes(len(rows), n), 120, np.uint8))
        args = (q, s)
    else:
        w = torch.zeros(1, m, n, dtype=torch.bfloat16, device="cuda")
        w[0, at] = dev(rng.standard_normal((len(rows), n)).astype(np.float32)).bfloat16()
        values = w[0, at].double().cpu().numpy()
        args = (w,)
    ex = Experts(fmt, 1, 32, [32], 0)                        # for its calls, not for its weights
    ex.m, ex.widths, ex.args = m, [n], [args]
    t, ws = torch.full((1,), 0.25, device="cuda"), expert_workspace(T, m, n, 2)
    idx, y = dev(np.array([[0, -1]], np.int32)), torch.full((1, 2, n), 7.0, device="cuda")
    ex(T, [t], [y], idx, dev(x[None]), ws)
    want, bound = product(x[rows], 0.25, values)
    assert np.all(np.abs(y[0, 0].cpu().numpy() - want) <= bound) and not y[0, 1].any()
    gate, up = torch.full((2, m), 80.0, device="cuda"), dev(x.astype(np.float32) / 80).repeat(2, 1)
    h = torch.empty(m, dtype=torch.float16, device="cuda")
    T.check(T.teal_swiglu_f16(gate, up, h, m))
    h, z = h.cpu().numpy(), torch.full((1, n), 7.0, device="cuda")
    ex.down(T, t, z, idx, torch.full((1, 2), 0.5, device="cuda"), gate, up, ws)
    want, bound = product(h[rows], 0.25, values)
    assert np.all(np.abs(z[0].cpu().numpy() - 0.5 * want) <= 0.5 * bound)
    if fmt == "mx4":
        y1 = torch.empty(n, device="cuda")
        T.check(T.teal_sparse_gemv_mx4(q, s, dev(x), 0.25, y1, m, n, workspace(T, m, n)))
        want, bound = product(x[rows], 0.25, values)
        assert np.all(np.abs(y1.cpu().numpy() - want) <= bound)


def test_the_most_tokens_of_a_router(T):   # noqa: F811
    tokens = 1 << 24
    logits = torch.randn(tokens, 4, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    idx, weight = torch.empty(tokens, 2, dtype=torch.int32, device="cuda"), torch.empty(tokens, 2, device="cuda")
    T.check(T.teal_route_experts(logits, None, 1, tokens, 4, 1, 1, 1, 2, False, 1.0, idx, weight))
    best = logits.sort(dim=1, descending=True, stable=True)
    assert torch.equal(idx.long(), best.indices[:, :2])
    score = torch.sigmoid(best.values[:, :2].double())
    assert bool(((weight - score).abs() <= score * (2.0 ** -24 + 2.0 ** -48)).all())
