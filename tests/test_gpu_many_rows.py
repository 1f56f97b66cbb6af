"""Rows to 8-bit integers and the products of many rows with int8 weights, on the GPU.

Nothing here has a tolerance: the integers are the nearest ones to real quotients, sums of integers are exact, and the
two scales are applied in binary32 in a stated order."""
import numpy as np
import pytest

from test_gpu_mx4 import T  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FILL = -77.0


def swiglu_f32(g, u):
    """The stated binary32 operations of SiLU(g) * u: fused multiply-adds as products and sums in binary64."""
    f, d = np.float32, np.float64
    with np.errstate(all="ignore"):
        z = np.clip(-g, f(-80), f(80))
        k = np.rint(z * f(1.44269502))
        r = (d(f(-0.693145752)) * k + z).astype(f)
        r = (d(f(-1.42860677e-06)) * k + r).astype(f)
        p = np.full_like(r, f(1) / f(5040))
        for c in (720, 120, 24, 6, 2, 1, 1):
            p = (p.astype(d) * r + d(f(1) / f(c))).astype(f)
        e = np.ldexp(p, np.nan_to_num(k).astype(np.int32))
        return np.where(np.isnan(g), g, g * (f(1) / (f(1) + e)) * u).astype(f)


def quantized(x, t):
    """(integers, scales) of rows of binary64 values that are 16-bit numbers."""
    with np.errstate(all="ignore"):
        v = np.where(np.abs(x) > t, x, 0.0)
        a = np.abs(v).max(-1, keepdims=True)
        # a quotient half way between two integers is a binary64 number, and any other is further from there than its rounding
        q = np.rint(127 * v / np.where(a > 0, a, 1.0))
        q = np.where(np.isinf(a), np.where(np.isinf(v), np.copysign(127.0, v), 0.0), q)
        scale = a[:, 0].astype(np.float32) / np.float32(127)
    return q.astype(np.int8), scale


def run_quantize(T, x, t):   # noqa: F811
    """x: a tensor of 16-bit floats or a pair (gate, up); checks that nothing else is written."""
    rows, m = (x if torch.is_tensor(x) else x[0]).shape
    pitch = T.teal_quantized_pitch(m)
    q = torch.full((rows + 1, pitch), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((rows + 1,), FILL, device="cuda")
    if torch.is_tensor(x):
        T.check(T.teal_quantize_rows(x, T.TEAL_BF16 if x.dtype == torch.bfloat16 else T.TEAL_F16, rows, m, t, q, scale))
    else:
        T.check(T.teal_quantize_rows_swiglu(*x, rows, m, t, q, scale))
    assert bool((q[rows] == 99).all()) and float(scale[rows]) == FILL
    assert bool((q[:rows, m:] == 0).all())
    return q[:rows], scale[:rows]


def check_quantize(T, x, t, values=None):   # noqa: F811
    q, scale = run_quantize(T, x, t)
    values = x.double().cpu().numpy() if values is None else values
    want_q, want_scale = quantized(values, t)
    assert np.array_equal(q[:, :want_q.shape[1]].cpu().numpy(), want_q)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    return q, scale


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,m", [(1, 1), (3, 7), (2, 8), (5, 127), (4, 128), (3, 513), (2, 1024), (7, 1500), (2, 2048),
                                    (3, 4096), (2, 5001), (1, 8192), (2, 14336), (1, 16385), (2, 28672), (1, 131072)])
def test_quantize_rows(T, dtype, rows, m):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(m + rows)
    x = (torch.randn(rows, m, generator=gen, device="cuda") *
         torch.exp2(torch.randint(-12, 8, (rows, 1), generator=gen, device="cuda").float())).to(dtype)
    check_quantize(T, x, 0.0)
    check_quantize(T, x, float(x.float().abs().median()))
    check_quantize(T, x, float(x.float().abs().max()))                    # nothing is kept


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_quotients_half_way_between_integers(T, dtype):   # noqa: F811
    """Rows whose largest value is 127 * 2^e have every k + 1/2 among their quotients; and every 16-bit number there is, by
    rows of all sizes of the largest."""
    k = torch.arange(-127, 128, device="cuda").float()
    halves = torch.cat([k, (k + 0.5).clamp(max=127)])
    x = torch.stack([halves * 2.0 ** e for e in (-6, -1, 0, 5)]).to(dtype)
    check_quantize(T, x, 0.0)
    bits = torch.arange(0, 32768, dtype=torch.int32, device="cuda")
    every = bits.to(torch.int16).view(dtype)
    every = every[torch.isfinite(every.float())]
    # a window of 11 binary orders below each largest value: what is smaller has the quotient 0
    span = 11 << (10 if dtype == torch.float16 else 7)
    ends = torch.randint(1, every.numel(), (200,), generator=torch.Generator().manual_seed(1)).tolist() + [1, 2, every.numel()]
    rows = [torch.nn.functional.pad(every[max(0, e - span):e].flip(0), (0, max(0, span - e))) for e in ends]
    check_quantize(T, torch.stack(rows).contiguous(), 0.0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_infinities_nan_and_zero_rows(T, dtype):   # noqa: F811
    x = torch.randn(8, 300, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    x[0] = 0
    x[1, 5] = float("nan")
    x[2] = float("nan")
    x[3, 7], x[3, 9] = float("inf"), float("-inf")
    x[4, 299] = float("-inf")
    x[5] = torch.finfo(dtype).min
    x[6, :200] = float("nan")
    x[7] = -0.0
    for t in (0.0, 0.5, 70000.0):
        check_quantize(T, x, t)


def test_addresses_that_allow_no_wide_loads(T):   # noqa: F811
    buf = torch.randn(2 * 4 * 512 + 1, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").half()
    x = buf[1:1 + 4 * 512].view(4, 512)
    assert x.data_ptr() % 16 == 2
    check_quantize(T, x, 0.25)
    f = torch.randn(2 * 4 * 512 + 1, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    gate, up = f[1:1 + 2048].view(4, 512), f[2049:].view(4, 512)
    h = swiglu_f32(gate.cpu().numpy(), up.cpu().numpy()).astype(np.float16)
    check_quantize(T, (gate, up), 0.1, h.astype(np.float64))


@pytest.mark.parametrize("rows,m", [(1, 5), (3, 128), (2, 1000), (5, 2730), (2, 14336), (1, 40000)])
def test_quantize_swiglu(T, rows, m):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(m)
    gate, up = (torch.randn(rows, m, generator=gen, device="cuda") * s for s in (2.0, 1.0))
    if m >= 128:
        gate[0, 3], up[0, 9] = float("nan"), float("nan")
        gate[0, 10:14] = torch.tensor([-100.0, 100.0, 0.0, -0.0])
    with np.errstate(over="ignore"):
        h = swiglu_f32(gate.cpu().numpy(), up.cpu().numpy()).astype(np.float16).astype(np.float64)
    for t in (0.0, 0.3):
        check_quantize(T, (gate, up), t, h)


# ---- the product ----

def random_ints(gen, *shape, low=-127):
    return torch.randint(low, 128, shape, generator=gen, device="cuda", dtype=torch.int8)


def make_rows(T, gen, rows, m):   # noqa: F811
    q = torch.zeros(rows, T.teal_quantized_pitch(m), dtype=torch.int8, device="cuda")
    q[:, :m] = random_ints(gen, rows, m)
    return q, torch.rand(rows, generator=gen, device="cuda") * 0.02


def product(q, row_scale, W, scale):
    m = W.shape[0]
    total = q[:, :m].double() @ W.double()            # whole numbers below 2^53
    return total.float() * row_scale[:, None] * scale.float()


def check_products(T, rows, m, widths, seed=0, workspace=None):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(seed + m + rows)
    q, row_scale = make_rows(T, gen, rows, m)
    W = [random_ints(gen, m, n, low=-128) for n in widths]
    scale = [(torch.rand(n, generator=gen, device="cuda") * 0.01 + 1e-3).half() for n in widths]
    ys = [torch.full((rows + 1, n), FILL, device="cuda") for n in widths]
    if workspace is None:
        workspace = torch.zeros(T.teal_workspace_bytes_gemm_w8(rows, m, sum(widths)), dtype=torch.uint8, device="cuda")
    for again in range(2):                            # the workspace is as it was
        for y in ys:
            y.fill_(FILL)
        if len(widths) == 1 and not again:
            T.check(T.teal_gemm_w8(W[0], scale[0], q, row_scale, rows, ys[0], m, widths[0], workspace))
        else:
            T.check(T.teal_gemm_w8_multi(W, scale, ys, widths, q, row_scale, rows, m, workspace))
        for y, w, s in zip(ys, W, scale):
            assert bool((y[rows] == FILL).all())
            assert torch.equal(y[:rows], product(q, row_scale, w, s))
    assert bool((workspace[:1 << 20] == 0).all())     # the counters


@pytest.mark.parametrize("rows", [1, 2, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257])
@pytest.mark.parametrize("m,widths", [(128, [128]), (1, [16]), (129, [48, 16]), (1000, [400]), (257, [144, 256, 16, 272])])
def test_products_of_any_size(T, rows, m, widths):   # noqa: F811
    check_products(T, rows, m, widths)


@pytest.mark.parametrize("rows,m,widths", [(1, 4096, [1024]), (1, 14336, [64]), (3, 5001, [3424, 416]), (32, 8191, [1040]),
                                           (48, 2048, [4096, 512, 512]), (100, 11008, [528]), (300, 4097, [1536]),
                                           (333, 5001, [3424, 416]), (700, 1500, [2064]), (1025, 640, [1296])])
def test_products_with_a_sum_cut_into_slices(T, rows, m, widths):   # noqa: F811
    check_products(T, rows, m, widths)


@pytest.mark.parametrize("rows,m,widths", [(1024, 384, [12288]), (2050, 200, [8192 + 16, 48]), (4096, 130, [4096]),
                                           (700, 11008, [4096]), (1000, 2048, [8192])])
def test_products_of_large_tiles(T, rows, m, widths):   # noqa: F811
    check_products(T, rows, m, widths)


@pytest.mark.parametrize("tile_rows,tile_cols", [(16, 128), (32, 128), (64, 128), (128, 128), (256, 128), (256, 256)])
def test_every_launch_shape(T, tile_rows, tile_cols):   # noqa: F811
    """All tiles, with last ones of a quarter, half and three quarters of their rows, whole and cut sums, ragged columns and
    channels: the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(tile_rows + tile_cols)
    for rows, m, widths in [(1, 300, [144]), (tile_rows, 129, [256, 48]), (tile_rows // 4, 640, [272]), (tile_rows // 2 + 1, 1000, [528]),
                            (tile_rows * 2 + tile_rows * 3 // 4, 257, [400]), (tile_rows * 3 + tile_rows // 2, 1300, [112, 16, 336]),
                            (tile_rows + tile_rows // 4, 100, [512]), (9 * tile_rows + 7, 384, [1040])]:
        q, row_scale = make_rows(T, gen, rows, m)
        W = [random_ints(gen, m, n, low=-128) for n in widths]
        scale = [(torch.rand(n, generator=gen, device="cuda") * 0.01 + 1e-3).half() for n in widths]
        ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(max(rows, tile_rows), m, sum(widths)), dtype=torch.uint8, device="cuda")
        blocks = -(-rows // tile_rows) * sum(-(-n // tile_cols) for n in widths)
        for splits in (1, 2, 3, 8, 16):
            if splits > 1 and (tile_rows > 128 or blocks * splits > 512):
                continue
            ys = [torch.full((rows + 1, n), FILL, device="cuda") for n in widths]
            T.check(T.teal_gemm_w8_ex(W, scale, ys, widths, q, row_scale, rows, m, ws, tile_rows=tile_rows, tile_cols=tile_cols,
                                      splits=splits))
            for y, w, s in zip(ys, W, scale):
                assert bool((y[rows] == FILL).all())
                assert torch.equal(y[:rows], product(q, row_scale, w, s)), (rows, m, widths, splits)
            assert bool((ws[:1 << 20] == 0).all())


def test_one_workspace_for_calls_of_all_sizes(T):   # noqa: F811
    ws = torch.zeros(max(T.teal_workspace_bytes_gemm_w8(r, 8192, 16384) for r in (1, 300, 4096)), dtype=torch.uint8,
                     device="cuda")
    for rows, m, widths in [(300, 4097, [1536]), (1, 4096, [1024]), (40, 8000, [16]), (600, 300, [96, 32]), (1, 4096, [1024])]:
        check_products(T, rows, m, widths, workspace=ws)


def test_the_largest_sums(T):   # noqa: F811
    m, n = 1 << 17, 16
    q = torch.full((2, m), 127, dtype=torch.int8, device="cuda")
    q[1] = -127
    W = torch.full((m, n), -128, dtype=torch.int8, device="cuda")
    W[:, 3] = 127
    one = torch.ones(n, device="cuda").half()
    y = torch.empty(2, n, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(2, m, n), dtype=torch.uint8, device="cuda")
    T.check(T.teal_gemm_w8(W, one, q, torch.ones(2, device="cuda"), 2, y, m, n, ws))
    assert float(y[0, 0]) == -127.0 * 128 * m and float(y[1, 0]) == 127.0 * 128 * m
    assert float(y[1, 3]) == np.float32(-127.0 * 127 * m)


def test_infinite_and_nan_scales(T):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, row_scale = make_rows(T, gen, 5, 300)
    row_scale[1], row_scale[2], row_scale[3] = float("inf"), float("nan"), 0.0
    W, scale = random_ints(gen, 300, 32), torch.rand(32, generator=gen, device="cuda").half()
    W[:, 7] = 0
    scale[5], scale[6] = float("inf"), float("nan")
    y = torch.empty(5, 32, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(5, 300, 32), dtype=torch.uint8, device="cuda")
    T.check(T.teal_gemm_w8(W, scale, q, row_scale, 5, y, 300, 32, ws))
    assert torch.equal(torch.nan_to_num(y, nan=5e30), torch.nan_to_num(product(q, row_scale, W, scale), nan=5e30))


def test_no_rows(T):   # noqa: F811
    y = torch.full((4,), FILL, device="cuda")
    T.check(T.teal_quantize_rows(None, T.TEAL_F16, 0, 64, 0.0, None, None))
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(0, 64, 16), dtype=torch.uint8, device="cuda")
    W, scale = torch.zeros(64, 16, dtype=torch.int8, device="cuda"), torch.zeros(16, device="cuda").half()
    T.check(T.teal_gemm_w8(W, scale, None, None, 0, y, 64, 16, ws))
    assert bool((y == FILL).all())


def test_on_another_stream_and_captured(T):   # noqa: F811
    """Quantisation and product of a step, replayed on new inputs with eager calls between the replays."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    rows, m, n = 40, 1536, 640
    x, W = torch.randn(rows, m, generator=gen, device="cuda").half(), random_ints(gen, m, n)
    scale = (torch.rand(n, generator=gen, device="cuda") * 0.01).half()
    q = torch.empty(rows, T.teal_quantized_pitch(m), dtype=torch.int8, device="cuda")
    row_scale, y = torch.empty(rows, device="cuda"), torch.empty(rows, n, device="cuda")
    ws, ws2 = (torch.zeros(T.teal_workspace_bytes_gemm_w8(rows, m, n), dtype=torch.uint8, device="cuda") for _ in range(2))

    def step(y, ws):
        T.check(T.teal_quantize_rows(x, T.TEAL_F16, rows, m, 0.3, q, row_scale))
        T.check(T.teal_gemm_w8(W, scale, q, row_scale, rows, y, m, n, ws))

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(y, ws)
    stream.synchronize()
    assert torch.equal(y, product(q, row_scale, W, scale))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(y, ws)
    eager = torch.empty_like(y)
    for k in range(4):
        x.copy_(torch.randn(rows, m, generator=gen, device="cuda") * (k + 1))
        y.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        step(eager, ws2)
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(y, product(q, row_scale, W, scale))


def test_rows_of_a_batch_are_what_one_row_gives(T):   # noqa: F811
    """A row's outputs do not depend on the rows beside it, whatever tiles a call takes."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    m, n = 2048, 1040
    q, row_scale = make_rows(T, gen, 600, m)
    W, scale = random_ints(gen, m, n), (torch.rand(n, generator=gen, device="cuda") * 0.01).half()
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(600, m, n), dtype=torch.uint8, device="cuda")
    whole = torch.empty(600, n, device="cuda")
    T.check(T.teal_gemm_w8(W, scale, q, row_scale, 600, whole, m, n, ws))
    for a, b in [(0, 1), (17, 50), (100, 300), (599, 600)]:
        part = torch.empty(b - a, n, device="cuda")
        T.check(T.teal_gemm_w8(W, scale, q[a:b], row_scale[a:b], b - a, part, m, n, ws))
        assert torch.equal(part, whole[a:b])


def test_one_workspace_with_the_calls_of_one_row(T):   # noqa: F811
    """Calls of one row, of a few and of many in turn on one workspace: each leaves it ready for the others."""
    gen = torch.Generator(device="cuda").manual_seed(31)
    m, n = 4096, 1024
    W, scale = random_ints(gen, m, n), (torch.rand(n, generator=gen, device="cuda") * 0.01).half()
    Wt = torch.randn(m, n, generator=gen, device="cuda").bfloat16()
    x = torch.randn(40, m, generator=gen, device="cuda").half()
    q, row_scale = make_rows(T, gen, 40, m)
    fresh = [torch.empty(n, device="cuda"), torch.empty(4, n, device="cuda")]
    size = max(T.teal_workspace_bytes(m, n), T.teal_workspace_bytes_batch(4, m, n), T.teal_workspace_bytes_gemm_w8(40, m, n))

    def one(y, ws):
        T.check(T.teal_sparse_gemv_w8(W, scale, x[0], 0.5, y, m, n, ws))

    def few(y, ws):
        T.check(T.teal_sparse_gemv_bf16_batch(Wt, x[:4], 4, 0.5, y, m, n, ws))

    for call, y in zip((one, few), fresh):
        call(y, torch.zeros(size, dtype=torch.uint8, device="cuda"))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    many = torch.empty(40, n, device="cuda")
    for splits in (0, 4, 16):
        T.check(T.teal_gemm_w8_ex([W], [scale], [many], [n], q, row_scale, 40, m, ws, tile_rows=64 if splits else 0,
                                  tile_cols=128 if splits else 0, splits=splits))
        assert torch.equal(many, product(q, row_scale, W, scale))
        for call, want in zip((one, few), fresh):
            got = torch.full_like(want, FILL)
            call(got, ws)
            assert torch.equal(got, want)


def test_two_calls_at_once_and_a_recorded_one(T):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(32)
    m, n = 8192, 1024
    W, scale = random_ints(gen, m, n), (torch.rand(n, generator=gen, device="cuda") * 0.01).half()
    sides = []
    for rows in (20, 70):
        q, row_scale = make_rows(T, gen, rows, m)
        ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(rows, m, n), dtype=torch.uint8, device="cuda")
        sides.append((rows, q, row_scale, torch.empty(rows, n, device="cuda"), ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for rows, q, row_scale, y, ws, stream in sides:
            T.check(T.teal_gemm_w8_ex([W], [scale], [y], [n], q, row_scale, rows, m, ws, stream=stream.cuda_stream, tile_rows=16,
                                      tile_cols=128, splits=8))
    torch.cuda.synchronize()
    for rows, q, row_scale, y, _, _ in sides:
        assert torch.equal(y, product(q, row_scale, W, scale))

    rows, q, row_scale, y, ws, _ = sides[0]
    W2, y2 = random_ints(gen, m, 208), torch.empty(rows, 208, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(rows, m, n + 208), dtype=torch.uint8, device="cuda")
    run = T.prepare(lambda: T.teal_gemm_w8_multi([W, W2], [scale, scale], [y, y2], [n, 208], q, row_scale, rows, m, ws))
    for _ in range(3):
        q[:, :m] = random_ints(gen, rows, m)
        y.fill_(FILL)
        y2.fill_(FILL)
        T.check(run())
        assert torch.equal(y, product(q, row_scale, W, scale))
        assert torch.equal(y2, product(q, row_scale, W2, scale[:208]))


def test_offsets_beyond_32_bits(T):   # noqa: F811
    """2^20 rows of 2064: more than 2^31 numbers of X, Q and Y."""
    gen = torch.Generator(device="cuda").manual_seed(41)
    rows, m, n = T.TEAL_MAX_ROWS, 2064, 2064
    x = torch.empty(rows, m, dtype=torch.float16, device="cuda").normal_(generator=gen)
    pitch = T.teal_quantized_pitch(m)
    q, row_scale = torch.empty(rows, pitch, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    T.check(T.teal_quantize_rows(x, T.TEAL_F16, rows, m, 0.25, q, row_scale))
    assert x.numel() > 2 ** 31 and q.numel() > 2 ** 31
    for at in (0, rows // 2 - 3, rows - 40):
        want_q, want_scale = quantized(x[at:at + 40].double().cpu().numpy(), 0.25)
        assert np.array_equal(q[at:at + 40, :m].cpu().numpy(), want_q)
        assert np.array_equal(row_scale[at:at + 40].cpu().numpy(), want_scale)
    del x
    W, scale = random_ints(gen, m, n), (torch.rand(n, generator=gen, device="cuda") * 0.01).half()
    y = torch.full((rows, n), float("nan"), device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_gemm_w8(rows, m, n), dtype=torch.uint8, device="cuda")
    T.check(T.teal_gemm_w8(W, scale, q, row_scale, rows, y, m, n, ws))
    assert not bool(torch.isnan(y).any())
    for at in range(0, rows, rows // 16):
        part = slice(at + rows // 16 - 1000, at + rows // 16)
        assert torch.equal(y[part], product(q[part], row_scale[part], W, scale))
