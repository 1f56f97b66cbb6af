"""The experts' products for many tokens, on the GPU, against sums in binary64.

Tolerances.  A product of two bf16 numbers has 16 significant bits: exact in fp32.  A sum of m of them in fp32, in any order,
is off by at most m * 2^-23 * sum |x w| (an addition by half a step of its result, 2^-24; the matrix cores may cut where
they do not round, 2^-23).  Weights and joins of top_k rows add top_k + 1 roundings of 2^-24.  For H the products'
errors go through SiLU(g) * u, whose derivatives are at most 1.1 |u| and |g| in size, SiLU(g) * u itself is off by less than
2^-16 of its value, as the header says, and the rounding to bf16 by 2^-8 of it.  Where everything is a small whole number the sums
are not off at all."""
import numpy as np
import pytest

import teal_inputs as ti
from test_gpu_many_rows import FILL
from test_gpu_mx4 import T  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ---- the arrangement ----

def arranged(idx, experts):
    key = np.where((idx.reshape(-1) >= 0) & (idx.reshape(-1) < experts), idx.reshape(-1), experts)
    order = np.argsort(key, kind="stable")
    return order.astype(np.int32), np.searchsorted(key[order], np.arange(experts + 1)).astype(np.int32)


def run_arrange(T, idx, experts, workspace=None):   # noqa: F811
    tokens, top_k = idx.shape
    pairs = tokens * top_k
    order = torch.full((pairs + 1,), -7, dtype=torch.int32, device="cuda")
    start = torch.full((experts + 2,), -7, dtype=torch.int32, device="cuda")
    if workspace is None:
        workspace = torch.zeros(T.teal_workspace_bytes_arrange_experts(experts, pairs), dtype=torch.uint8, device="cuda")
    T.check(T.teal_arrange_experts(idx, tokens, top_k, experts, order, start, workspace))
    assert int(order[pairs]) == -7 and int(start[experts + 1]) == -7
    assert bool((workspace[:1 << 20] == 0).all())
    return order[:pairs], start[:experts + 1]


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (1, 6, 64), (3, 2, 8), (64, 1, 2), (65, 7, 33), (200, 8, 128),
                                                  (1000, 8, 256), (1024, 8, 1024), (1025, 8, 1023), (2000, 32, 1024),
                                                  (5000, 4, 60), (16384, 8, 256), (70000, 10, 300), (100, 32, 1)])
@pytest.mark.parametrize("kind", ["spread", "uneven", "one", "padded"])
def test_arrange(T, tokens, top_k, experts, kind):   # noqa: F811
    rng = np.random.default_rng(tokens + experts)
    idx = rng.integers(0, experts, (tokens, top_k))
    if kind == "uneven":
        idx = np.minimum(idx, rng.integers(0, experts, (tokens, top_k)))
        idx = np.minimum(idx, rng.integers(0, experts, (tokens, top_k)))
    elif kind == "one":
        idx[:] = experts - 1
    elif kind == "padded":
        idx[rng.random(idx.shape) < 0.3] = -1
        idx[rng.random(idx.shape) < 0.1] = experts
        idx[rng.random(idx.shape) < 0.1] = 2 ** 31 - 1
        idx[rng.random(idx.shape) < 0.1] = -2 ** 31
    idx = idx.astype(np.int32)
    order, start = run_arrange(T, torch.from_numpy(idx).cuda(), experts)
    want_order, want_start = arranged(idx, experts)
    assert np.array_equal(start.cpu().numpy(), want_start)
    assert np.array_equal(order.cpu().numpy(), want_order)


def test_arrange_nothing(T):   # noqa: F811
    start = torch.full((9,), -7, dtype=torch.int32, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_arrange_experts(8, 0), dtype=torch.uint8, device="cuda")
    T.check(T.teal_arrange_experts(None, 0, 4, 8, None, start, ws))
    assert bool((start == 0).all())


# ---- the products ----

class Case:
    """Experts with their weights, a router's choice, and the products in binary64."""

    def __init__(self, T, fmt, tokens, top_k, experts, m, f, n, seed=0, whole=False, padded=0, choose=None):   # noqa: F811
        gen = torch.Generator(device="cuda").manual_seed(seed + tokens + m + f + n)
        self.T, self.fmt, self.tokens, self.top_k, self.experts = T, fmt, tokens, top_k, experts
        self.m, self.f, self.n, self.pairs = m, f, n, tokens * top_k

        def weights(a, b):
            if whole:
                w = torch.randint(-2, 3, (experts, a, b), generator=gen, device="cuda").bfloat16()
            else:
                w = (torch.randn(experts, a, b, generator=gen, device="cuda") * a ** -0.5).bfloat16()
            if fmt == "bf16":
                return (w,), w.double()
            codes = torch.empty(experts, a, b // 2, dtype=torch.uint8, device="cuda")
            size = T.teal_mx4_scale_bytes(a, b)
            scales = torch.full((experts, size), 255, dtype=torch.uint8, device="cuda")
            back = torch.empty(experts, b, a, dtype=torch.bfloat16, device="cuda")
            for e in range(experts):
                T.check(T.teal_pack_mx4(w[e].t().contiguous(), codes[e], scales[e], a, b))
                T.check(T.teal_unpack_mx4(codes[e], scales[e], back[e], a, b))
            # what stands in a tile behind the last channel has no meaning
            tiles = scales.view(experts, (a + 7) // 8, -1, 8, 16)
            if a % 8:
                tiles[:, -1, :, a % 8:] = 255
            return (codes, scales), back.transpose(1, 2).double()

        self.gate, self.gate64 = weights(m, f)
        self.up, self.up64 = weights(m, f)
        self.down, self.down64 = weights(f, n)
        if choose is not None:
            idx = torch.from_numpy(choose).cuda()
        else:
            idx = torch.rand(tokens, experts, generator=gen, device="cuda").argsort(-1)[:, :top_k].int()
            idx = torch.cat([idx, torch.full((tokens, top_k - idx.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
        idx[tokens - padded:] = -1
        self.idx = idx.contiguous()
        if whole:
            self.x = torch.randint(-2, 3, (tokens, m), generator=gen, device="cuda").bfloat16()
            self.weight = torch.exp2(torch.randint(-2, 3, (tokens, top_k), generator=gen, device="cuda").float())
        else:
            self.x = torch.randn(tokens, m, generator=gen, device="cuda").bfloat16()
            self.weight = torch.rand(tokens, top_k, generator=gen, device="cuda") + 0.1
        self.order, self.start = run_arrange(T, self.idx, experts)

    def run_gate_up(self, x=None):
        h = torch.full((self.pairs + 1, self.f), FILL, dtype=torch.bfloat16, device="cuda")
        call = self.T.teal_grouped_experts_bf16_gate_up if self.fmt == "bf16" else self.T.teal_grouped_experts_mx4_gate_up
        self.T.check(call(*self.gate, *self.up, self.experts, self.order, self.start, self.tokens, self.top_k,
                          self.x if x is None else x, h, self.m, self.f))
        used = int(self.start[self.experts])
        assert bool((h[used:] == FILL).all())          # rows behind the last pair with an expert, left as they were
        return h[:self.pairs]

    def run_down(self, h, workspace=None):
        y = torch.full((self.tokens + 1, self.n), FILL, device="cuda")
        if workspace is None:
            workspace = torch.zeros(self.T.teal_workspace_bytes_grouped_experts(self.pairs, self.n), dtype=torch.uint8,
                                    device="cuda")
            workspace[1 << 20:] = 255                  # NaN where the rows of sums are: none is read that was not written
        call = self.T.teal_grouped_experts_bf16_down if self.fmt == "bf16" else self.T.teal_grouped_experts_mx4_down
        self.T.check(call(*self.down, self.experts, self.order, self.start, self.tokens, self.top_k, self.idx, self.weight, h,
                          y, self.f, self.n, workspace))
        assert bool((y[self.tokens] == FILL).all())
        assert bool((workspace[:1 << 20] == 0).all())
        return y[:self.tokens]

    def places(self):
        """(expert, its places in `order`, their pairs) for those that have any."""
        order, start = self.order.long(), self.start.tolist()
        return [(e, slice(a, b), order[a:b]) for e, (a, b) in enumerate(zip(start, start[1:])) if b > a]

    def check_gate_up(self):
        h = self.run_gate_up()
        for e, at, pairs in self.places():
            x = self.x[pairs // self.top_k].double()
            g, u = x @ self.gate64[e], x @ self.up64[e]
            off_g, off_u = (self.m * 2.0 ** -23 * (x.abs() @ w[e].abs()) for w in (self.gate64, self.up64))
            want = g * torch.sigmoid(g) * u
            off = 1.1 * off_g * (u.abs() + off_u) + off_u * g.abs() + want.abs() * (2.0 ** -8 + 2.0 ** -16) + 2.0 ** -133
            assert bool(((h[at].double() - want).abs() <= off).all()), e
        return h

    def check_down(self, h):
        y = self.run_down(h)
        want = torch.zeros(self.pairs, self.n, dtype=torch.float64, device="cuda")
        off = torch.zeros_like(want)
        weight = self.weight.flatten().double()[:, None]
        for e, at, pairs in self.places():
            v = h[at].double()
            want[pairs] = weight[pairs] * (v @ self.down64[e])
            off[pairs] = weight[pairs].abs() * (v.abs() @ self.down64[e].abs())
        want, off = (a.unflatten(0, (self.tokens, self.top_k)).sum(1) for a in (want, off))
        assert bool(((y.double() - want).abs() <= off * (self.f * 2.0 ** -23 + (self.top_k + 1) * 2.0 ** -24)).all())

    def check(self):
        self.check_down(self.check_gate_up())


SIZES = [(1, 1, 1, 64, 32, 32), (1, 6, 64, 128, 96, 64), (5, 2, 8, 72, 160, 288), (33, 2, 4, 8, 32, 64), (40, 4, 16, 200, 64, 320),
         (130, 8, 60, 136, 96, 96), (257, 2, 8, 512, 256, 160), (64, 1, 1, 1000, 384, 256), (100, 2, 2, 64, 32, 32),
         (600, 2, 4, 104, 288, 544), (1100, 4, 8, 320, 160, 256), (2000, 8, 128, 64, 64, 64), (700, 1, 2, 128, 512, 1024)]


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,experts,m,f,n", SIZES)
def test_grouped_experts(T, fmt, tokens, top_k, experts, m, f, n):   # noqa: F811
    Case(T, fmt, tokens, top_k, experts, m, f, n, padded=tokens // 7).check()


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("f,n", [(1024, 2048), (2048, 4096), (96, 160)])
def test_large_groups_whose_last_tiles_are_more_or_less_empty(T, fmt, f, n):   # noqa: F811
    """The shapes that many rows take (128 or 256 rows by 128 or 256 columns), and last tiles of few rows, about a quarter, half,
    three quarters and all of them."""
    sizes = [512 + 20, 3 * 256 + 64, 256 + 65, 2 * 256 + 128, 256 + 129, 256 + 192, 256 + 193, 1024, 7, 0]
    choose = np.repeat(np.arange(len(sizes), dtype=np.int32), sizes)
    choose = np.random.default_rng(f).permutation(choose)[:, None]
    Case(T, fmt, choose.shape[0], 1, len(sizes), 136, f, n, choose=choose).check()


@pytest.mark.parametrize("tokens,top_k,experts,m,f,n", [(3, 2, 4, 8, 8, 8), (50, 3, 5, 40, 24, 72), (300, 2, 2, 24, 136, 264)])
def test_bf16_widths_in_steps_of_eight(T, tokens, top_k, experts, m, f, n):   # noqa: F811
    Case(T, "bf16", tokens, top_k, experts, m, f, n).check()


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,experts,m,f,n", [(9, 2, 8, 72, 64, 96), (200, 2, 4, 136, 96, 320), (900, 2, 2, 264, 160, 544)])
def test_whole_numbers_come_out_exactly(T, fmt, tokens, top_k, experts, m, f, n):   # noqa: F811
    """Products and sums of small whole numbers, and weights that are powers of two: every bit of y is determined, and H lies
    between the roundings of what is 2^-16 smaller and larger."""
    c = Case(T, fmt, tokens, top_k, experts, m, f, n, whole=True)
    h = c.run_gate_up()
    for e, at, pairs in c.places():
        x = c.x[pairs // top_k].double()
        g, u = x @ c.gate64[e], x @ c.up64[e]
        want = g * torch.sigmoid(g) * u
        ends = torch.stack([(want * (1 + s)).float().bfloat16() for s in (-2.0 ** -16, 2.0 ** -16)])
        ok = (h[at] >= ends.amin(0)) & (h[at] <= ends.amax(0))
        # |SiLU(g)| <= 87 e^-87 < 1.5e-36 for g <= -87; where 1 / (1 + e^-g) is below 2^-126 = e^-87.3 it may count as zero
        ok |= (g < -87) & (h[at].double().abs() <= 1.5e-36 * u.abs())
        assert bool(ok.all()), e
    h = torch.randint(-3, 4, (c.pairs, f), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    y = c.run_down(h)
    want = torch.zeros(c.pairs, n, dtype=torch.float64, device="cuda")
    for e, at, pairs in c.places():
        want[pairs] = c.weight.flatten().double()[pairs, None] * (h[at].double() @ c.down64[e])
    assert torch.equal(y.double(), want.unflatten(0, (tokens, top_k)).sum(1))


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("kind", ["one", "none", "first_and_last", "same_twice", "ladder"])
def test_uneven_groups(T, fmt, kind):   # noqa: F811
    tokens, top_k, experts = 300, 2, 16
    choose = np.full((tokens, top_k), -1, np.int32)
    if kind == "one":
        choose[:, 0] = 5
    elif kind == "first_and_last":
        choose[:] = [0, experts - 1]
        choose[7:] = [0, -1]
    elif kind == "same_twice":
        choose[:] = 3
    elif kind == "ladder":                             # groups of 0, 1, 2 ... rows, and one of very many
        flat = np.concatenate([np.full(e, e, np.int32) for e in range(experts - 1)])
        choose.reshape(-1)[:flat.size] = flat
        choose.reshape(-1)[flat.size:] = experts - 1
    c = Case(T, fmt, tokens, top_k, experts, 136, 64, 96, choose=choose)
    c.check()
    if kind == "none":
        assert bool((c.run_down(torch.full((c.pairs, c.f), float("nan"), device="cuda").bfloat16()) == 0).all())


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens", [20, 800])
def test_one_bad_row_stays_in_its_row(T, fmt, tokens):   # noqa: F811
    """NaN and infinities in a token's row, and in an expert's weights behind other experts' columns, reach nobody else."""
    c = Case(T, fmt, tokens, 2, 4, 72, 64, 96)
    clean_h = c.run_gate_up()
    clean_y = c.run_down(clean_h)
    x = c.x.clone()
    x[3, 71], x[4, 0] = float("nan"), float("inf")
    h = c.run_gate_up(x)
    token = c.order.long() // c.top_k
    touched = (token == 3) | (token == 4)
    assert bool(torch.isnan(h[token == 3]).all())
    assert not bool(torch.isfinite(h[token == 4]).all())
    assert torch.equal(h[~touched], clean_h[~touched])
    y = c.run_down(h)
    keep = torch.arange(tokens, device="cuda")
    keep = (keep != 3) & (keep != 4)
    assert torch.equal(y[keep], clean_y[keep]) and bool(torch.isnan(y[3]).all())
    c.weight[5] = float("nan")                         # a weight is its token's own
    y = c.run_down(clean_h)
    keep[:] = True
    keep[5] = False
    assert torch.equal(y[keep], clean_y[keep]) and bool(torch.isnan(y[5]).all())


@pytest.mark.parametrize("fmt,n", [("bf16", 1032), ("mx4", 1056)])
def test_sums_of_more_pairs_than_the_workspace_has_rows_of(T, fmt, n):   # noqa: F811
    """W_down in parts of 512 columns, the last one of 8 or 32: the rows of all columns would be more than 256 MB."""
    c = Case(T, fmt, 50000, 2, 8, 32, 32, n, padded=3)
    assert T.teal_workspace_bytes_grouped_experts(c.pairs, n) < (1 << 20) + c.pairs * n * 4
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_two_mixtures_at_once(T, fmt):   # noqa: F811
    """On two streams with a workspace each."""
    sides = []
    for seed in (1, 2):
        c = Case(T, fmt, 300 * seed, 2, 8, 128, 96, 256, seed=seed)
        h = c.run_gate_up()
        sides.append((c, h, c.run_down(h), torch.cuda.Stream(), torch.empty_like(h), torch.empty(c.tokens, c.n, device="cuda"),
                      torch.zeros(T.teal_workspace_bytes_grouped_experts(c.pairs, c.n), dtype=torch.uint8, device="cuda")))
    gate_up = T.teal_grouped_experts_bf16_gate_up if fmt == "bf16" else T.teal_grouped_experts_mx4_gate_up
    down = T.teal_grouped_experts_bf16_down if fmt == "bf16" else T.teal_grouped_experts_mx4_down
    torch.cuda.synchronize()
    for _ in range(10):
        for c, _, _, stream, h, y, ws in sides:
            s = stream.cuda_stream
            T.check(T.teal_arrange_experts(c.idx, c.tokens, c.top_k, c.experts, c.order, c.start, ws, stream=s))
            T.check(gate_up(*c.gate, *c.up, c.experts, c.order, c.start, c.tokens, c.top_k, c.x, h, c.m, c.f, stream=s))
            T.check(down(*c.down, c.experts, c.order, c.start, c.tokens, c.top_k, c.idx, c.weight, h, y, c.f, c.n, ws, stream=s))
    torch.cuda.synchronize()
    for c, want_h, want, _, h, y, _ in sides:
        assert torch.equal(h, want_h) and torch.equal(y, want)


def test_the_weight_of_a_pair_without_an_expert_adds_nothing(T):   # noqa: F811
    c = Case(T, "bf16", 30, 3, 4, 64, 64, 64, choose=np.tile(np.array([[1, -1, 2]], np.int32), (30, 1)))
    h = c.run_gate_up()
    y = c.run_down(h)
    c.weight[:, 1] = float("nan")
    assert torch.equal(c.run_down(h), y)


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_numbers_out_of_range_read_and_write_nothing_else(T, fmt):   # noqa: F811
    """An order and starts that are no arrangement: the results have no meaning, and nothing outside the arrays is touched."""
    c = Case(T, fmt, 70, 2, 8, 64, 64, 64)
    c.order = torch.randint(-2 ** 31, 2 ** 31 - 1, (c.pairs,), device="cuda", dtype=torch.int64).int()
    for start in ([-5, 10, 1 << 30, 3, -(1 << 31), 50, 60, 70, (1 << 31) - 1], [140] * 9, list(range(140, 131, -1)), [0] * 8 + [140]):
        c.start = torch.tensor(start, dtype=torch.int32, device="cuda")
        h = torch.full((c.pairs + 8, c.f), FILL, dtype=torch.bfloat16, device="cuda")
        call = T.teal_grouped_experts_bf16_gate_up if fmt == "bf16" else T.teal_grouped_experts_mx4_gate_up
        T.check(call(*c.gate, *c.up, 8, c.order, c.start, 70, 2, c.x, h, 64, 64))
        assert bool((h[c.pairs:] == FILL).all())
        c.run_down(h[:c.pairs].contiguous())
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_a_mixture_of_experts_from_logits_to_its_output(T, fmt):   # noqa: F811
    """Router, arrangement, gate and up, W_down, one behind the other on another stream, then captured and replayed on new
    inputs with eager calls between the replays; some tokens against the calls of a decode step."""
    tokens, experts, top_k, m, f, n = 150, 8, 2, 256, 96, 256
    c = Case(T, fmt, tokens, top_k, experts, m, f, n)
    gen = torch.Generator(device="cuda").manual_seed(77)
    logits = torch.randn(tokens, experts, generator=gen, device="cuda")
    ws = torch.zeros(max(T.teal_workspace_bytes_grouped_experts(c.pairs, n),
                         T.teal_workspace_bytes_arrange_experts(experts, c.pairs)), dtype=torch.uint8, device="cuda")
    ws2 = torch.zeros_like(ws)
    h = torch.zeros(c.pairs, f, dtype=torch.bfloat16, device="cuda")
    gate_up = T.teal_grouped_experts_bf16_gate_up if fmt == "bf16" else T.teal_grouped_experts_mx4_gate_up
    down = T.teal_grouped_experts_bf16_down if fmt == "bf16" else T.teal_grouped_experts_mx4_down

    def step(y, ws):
        T.check(T.teal_route_experts(logits, None, T.TEAL_SCORE_SOFTMAX, tokens, experts, 1, 1, 1, top_k, True, 1.0, c.idx, c.weight))
        T.check(T.teal_arrange_experts(c.idx, tokens, top_k, experts, c.order, c.start, ws))
        T.check(gate_up(*c.gate, *c.up, experts, c.order, c.start, tokens, top_k, c.x, h, m, f))
        T.check(down(*c.down, experts, c.order, c.start, tokens, top_k, c.idx, c.weight, h, y, f, n, ws))

    y, eager = torch.empty(tokens, n, device="cuda"), torch.empty(tokens, n, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(y, ws)
    stream.synchronize()
    c.check()
    assert torch.equal(y, c.run_down(h))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(y, ws)
    for k in range(4):
        logits.copy_(torch.randn(tokens, experts, generator=gen, device="cuda") * (k + 1))
        c.x.copy_(torch.randn(tokens, m, generator=gen, device="cuda"))
        y.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        step(eager, ws2)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        c.check()

    # the same through the calls of a decode step, dense, on the rows as fp16 numbers
    few = 8
    x16 = c.x[:few].half()
    g, u = (torch.empty(few, top_k, f, device="cuda") for _ in range(2))
    zero = torch.zeros(experts, device="cuda")
    out = torch.empty(few, n, device="cuda")
    dws = torch.zeros(T.teal_workspace_bytes_experts(m, 2 * f, few * top_k) + T.teal_workspace_bytes_experts(f, n, few * top_k),
                      dtype=torch.uint8, device="cuda")
    idx, weight = c.idx[:few].contiguous(), c.weight[:few].contiguous()
    if fmt == "bf16":
        T.check(T.teal_sparse_experts_bf16([c.gate[0], c.up[0]], [zero, zero], [g, u], [f, f], experts, idx, few, top_k, x16, m, dws))
        T.check(T.teal_sparse_experts_bf16_swiglu(c.down[0], zero, out, experts, idx, weight, few, top_k, g, u, f, n, dws))
    else:
        T.check(T.teal_sparse_experts_mx4([c.gate[0], c.up[0]], [c.gate[1], c.up[1]], [zero, zero], [g, u], [f, f], experts, idx,
                                          few, top_k, x16, m, dws))
        T.check(T.teal_sparse_experts_mx4_swiglu(*c.down, zero, out, experts, idx, weight, few, top_k, g, u, f, n, dws))
    # x as fp16 (half a step, 2^-11, or 2^-25 where it is tiny) and h as fp16 or bf16 (2^-8): of the sums of sizes
    scale = float(out.abs().max())
    assert float((eager[:few] - out).abs().max()) <= scale * f * (2.0 ** -8 + 2.0 ** -9)


@pytest.mark.parametrize("tokens", [4, 60, 700])
def test_a_block_of_nan_weights_stays_in_its_columns(T, tokens):   # noqa: F811
    """The scale byte 255 makes a block of 32 outputs NaN, whatever its codes, for the rows of its expert."""
    c = Case(T, "mx4", tokens, 2, 3, 136, 320, 288)
    clean_h = c.run_gate_up()
    clean_y = c.run_down(clean_h)
    assert bool(torch.isfinite(clean_y).all())
    places = torch.from_numpy(np.asarray(ti.mx4_scale_places(c.m, c.f))).long()
    for weights in (c.gate, c.up):
        kept = weights[1].clone()
        weights[1][1, int(places[c.m - 1, 4])] = 255
        weights[0][1, c.m - 1, 4 * 16:5 * 16] = 0                  # codes of zeros: NaN none the less
        h = c.run_gate_up()
        bad = torch.zeros_like(h, dtype=torch.bool)
        a, b = int(c.start[1]), int(c.start[2])
        bad[a:b, 4 * 32:5 * 32] = True
        assert torch.equal(torch.isnan(h), bad) and torch.equal(h[~bad], clean_h[~bad])
        weights[1].copy_(kept)
        clean_h = c.run_gate_up()                                  # (those codes are zeros now)
    clean_y = c.run_down(clean_h)
    places = torch.from_numpy(np.asarray(ti.mx4_scale_places(c.f, c.n))).long()
    c.down[1][2, int(places[0, 8])] = 255
    y = c.run_down(clean_h)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[(c.idx == 2).any(1), 8 * 32:] = True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean_y[~bad])


def test_offsets_beyond_32_bits_in_the_weights(T):   # noqa: F811
    """80 experts of 8192 x 4096, more than 2^31 weights each of gate, up and W_down; the last two are chosen."""
    gen = torch.Generator(device="cuda").manual_seed(51)
    experts, m, f, tokens, top_k = 80, 8192, 4096, 20, 2
    gate, up = (torch.empty(experts, m, f, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    down = torch.empty(experts, f, m, dtype=torch.bfloat16, device="cuda")
    assert gate[:experts - 2].numel() > 2 ** 31
    for w in (gate, up, down):
        w[:experts - 2] = float("nan")
        w[experts - 2:] = torch.randint(-2, 3, w[experts - 2:].shape, generator=gen, device="cuda").bfloat16()
    idx = torch.tensor([[experts - 2, experts - 1]] * tokens, dtype=torch.int32, device="cuda")
    order, start = run_arrange(T, idx, experts)
    x = torch.randint(0, 2, (tokens, m), generator=gen, device="cuda").bfloat16()
    h = torch.empty(tokens * top_k, f, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_grouped_experts_bf16_gate_up(gate, up, experts, order, start, tokens, top_k, x, h, m, f))
    for i, e in enumerate((experts - 2, experts - 1)):
        g, u = x.double() @ gate[e].double(), x.double() @ up[e].double()       # whole numbers, exact in fp32
        want = g * torch.sigmoid(g) * u
        off = want.abs() * (2.0 ** -8 + 2.0 ** -16) + 1.5e-36 * u.abs() + 2.0 ** -133
        assert bool(((h[i * tokens:(i + 1) * tokens].double() - want).abs() <= off).all())
    ones = torch.randint(-1, 2, h.shape, generator=gen, device="cuda").bfloat16()
    weight, y = torch.ones(tokens, top_k, device="cuda"), torch.empty(tokens, m, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_grouped_experts(tokens * top_k, m), dtype=torch.uint8, device="cuda")
    T.check(T.teal_grouped_experts_bf16_down(down, experts, order, start, tokens, top_k, idx, weight, ones, y, f, m, ws))
    want = sum(ones[i * tokens:(i + 1) * tokens].double() @ down[experts - 2 + i].double() for i in range(2))
    assert torch.equal(y.double(), want)                                            # whole numbers below 2^24


def test_offsets_beyond_32_bits_in_the_rows(T):   # noqa: F811
    """2^20 pairs of 2064 columns: more than 2^31 numbers of H."""
    gen = torch.Generator(device="cuda").manual_seed(52)
    experts, m, f, n, tokens, top_k = 4, 8, 2064, 16, 1 << 19, 2
    gate, up = (torch.randint(-2, 3, (experts, m, f), generator=gen, device="cuda").bfloat16() for _ in range(2))
    down = torch.randint(-2, 3, (experts, f, n), generator=gen, device="cuda").bfloat16()
    idx = torch.rand(tokens, experts, generator=gen, device="cuda").argsort(-1)[:, :top_k].int().contiguous()
    order, start = run_arrange(T, idx, experts)
    x = torch.randint(-2, 3, (tokens, m), generator=gen, device="cuda").bfloat16()
    h = torch.full((tokens * top_k, f), FILL, dtype=torch.bfloat16, device="cuda")
    assert h.numel() > 2 ** 31
    T.check(T.teal_grouped_experts_bf16_gate_up(gate, up, experts, order, start, tokens, top_k, x, h, m, f))
    y = torch.full((tokens, n), FILL, device="cuda")
    weight = torch.rand(tokens, top_k, generator=gen, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_grouped_experts(tokens * top_k, n), dtype=torch.uint8, device="cuda")
    T.check(T.teal_grouped_experts_bf16_down(down, experts, order, start, tokens, top_k, idx, weight, h, y, f, n, ws))
    place = torch.empty(tokens * top_k, dtype=torch.long, device="cuda")
    place[order.long()] = torch.arange(tokens * top_k, device="cuda")
    for b in (0, 1, 12345, tokens // 2, tokens - 2, tokens - 1):
        total, off = 0, 0
        for j in range(top_k):
            e, at = int(idx[b, j]), int(place[b * top_k + j])
            g, u = (x[b].double() @ w[e].double() for w in (gate, up))
            want = g * torch.sigmoid(g) * u
            row = h[at].double()
            assert bool(((row - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -16) + 2.0 ** -133).all())
            total = total + float(weight[b, j]) * (row @ down[e].double())
            off = off + float(weight[b, j]) * (row.abs() @ down[e].double().abs())
        assert bool(((y[b].double() - total).abs() <= off * (f * 2.0 ** -23 + (top_k + 1) * 2.0 ** -24)).all())
