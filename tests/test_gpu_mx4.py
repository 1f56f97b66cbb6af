"""Microscaled 4-bit weights on the GPU: the layout step bit for bit against the quantiser in numpy, the products
against sums in binary64, and the calls that stand for one another bit for bit.

Tolerance of a product: a wavefront has an eighth of a slice's survivors and rounds at most once for each of them,
and at most 64 roundings join a column's parts (pieces, wavefronts, slices), each by at most 2^-24 of a partial
sum, which is at most the sum of the magnitudes."""
import numpy as np
import pytest

import teal_inputs as ti

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import paper_2408_14690_amd as T
    assert torch.cuda.is_available(), "these tests need the GPU"
    T.load_library()
    return T


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def workspace(T, m, n):
    return torch.zeros(T.teal_workspace_bytes(m, n), dtype=torch.uint8, device="cuda")


def survivors(T, ws, count=1):
    off = T.teal_survivors_offset()
    return ws[off:off + 4 * count].view(torch.int32).tolist()


def exact(x, t, values):
    """(sum over |x_i| > t of x_i W_i, the same of magnitudes, survivors), W [m][n] in binary64."""
    kept = np.abs(x.astype(np.float64)) > t
    xk, wk = x[kept].astype(np.float64), values[kept]
    return xk @ wk, np.abs(xk) @ np.abs(wk), int(kept.sum())


def check(y, x, t, values):
    want, size, kept = exact(x, t, values)
    y = y.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(y - want) <= (kept / 8 + 64) * 2.0 ** -24 * size)
    return kept


def make(m, n, p, seed):
    codes, scales = ti.random_mx4(m, n, seed)
    x = ti.make_x(m, seed + 1, "gaussian")
    return codes, scales, ti.mx4_values(codes, scales), x, ti.quantile_threshold(x, p)


# ---- layout ----

def layout_weights(m, n, seed):
    """bf16 weights with ties, zeros of both signs, subnormal, huge, infinite and NaN entries."""
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((n, m)).astype(np.float32) * np.exp2(rng.integers(-8, 8, m)).astype(np.float32)
    b = ti.f32_to_bf16_bits(w)
    for value in (0x0000, 0x8000, 0x0001, 0x8003, 0x007F, 0x0080, 0x3F80, 0xBFC0, 0x4080):
        b[rng.integers(0, n, 1 + n // 16), rng.integers(0, m)] = value
    for value in (0x7F80, 0xFF80, 0x7FC0, 0x7F7F):
        b[rng.integers(0, n), rng.integers(0, m)] = value
    b[:, rng.integers(0, m)] = rng.choice(np.array([0x0000, 0x0001, 0x8002, 0x0013], np.uint16), n)
    if m > 4:
        b[:, 2], b[:, 3] = 0, 0x8000
    return b


@pytest.mark.parametrize("m,n", [(1, 32), (7, 32), (8, 512), (9, 544), (64, 256), (65, 1056), (200, 96), (333, 288),
                                 (130, 2080)])
def test_pack_is_the_quantiser_and_unpack_its_values(T, m, n):
    b = layout_weights(m, n, m * n)
    codes, scales = ti.quantize_mx4(b)
    w, q = dev(b), torch.full((m * n // 2 + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    s = torch.full((len(scales) + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    T.check(T.teal_pack_mx4(w, q, s, m, n))
    assert np.array_equal(q[:m * n // 2].cpu().numpy(), codes.ravel())
    assert np.array_equal(s[:len(scales)].cpu().numpy(), scales)
    assert bool((q[m * n // 2:] == 0xEE).all()) and bool((s[len(scales):] == 0xEE).all())
    back = torch.full((n * m + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_unpack_mx4(q, s, back, m, n))
    got = back[:n * m].double().cpu().numpy().reshape(n, m)
    assert np.array_equal(got, ti.mx4_values(codes, scales).T, equal_nan=True)
    assert bool((back[n * m:] == 3.0).all())
    # what has been rounded once stays as it is, up to the sign of zero
    again = torch.empty_like(q)
    finite = dev(np.where(np.isnan(got), 0, got).astype(np.float32)).bfloat16().contiguous()
    T.check(T.teal_pack_mx4(finite, again, s, m, n))
    T.check(T.teal_unpack_mx4(again, s, back, m, n))
    assert torch.equal(back[:n * m].view(n, m), finite)


@pytest.mark.parametrize("m,n", [(9, 64), (128, 128), (257, 544), (320, 96)])
def test_layout_of_weights_that_begin_anywhere(T, m, n):
    b = layout_weights(m, n, 5)
    codes, scales = ti.quantize_mx4(b)
    room = torch.zeros(n * m + 8, dtype=torch.int16, device="cuda")
    q = torch.empty(m, n // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(len(scales), dtype=torch.uint8, device="cuda")
    for shift in range(4):
        w = room[shift:shift + n * m]
        w.copy_(dev(b).flatten())
        T.check(T.teal_pack_mx4(w, q, s, m, n))
        assert np.array_equal(q.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
        room.fill_(77)
        T.check(T.teal_unpack_mx4(q, s, w, m, n))
        got = w.view(torch.bfloat16).double().cpu().numpy().reshape(n, m)
        assert np.array_equal(got, ti.mx4_values(codes, scales).T, equal_nan=True)
        assert bool((room[:shift] == 77).all()) and bool((room[shift + n * m:] == 77).all())


def test_unpack_every_scale_and_code(T):
    m, n = 256, 32
    codes = np.tile(np.arange(16, dtype=np.uint8) * 16 + np.arange(16, dtype=np.uint8)[::-1], (m, 1))
    scales = np.zeros(ti.mx4_scale_bytes(m, n), np.uint8)
    scales[ti.mx4_scale_places(m, n)[:, 0]] = np.arange(256)
    w = torch.empty(n, m, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_unpack_mx4(dev(codes), dev(scales), w, m, n))
    want = ti.mx4_values(codes, scales).T
    largest = 255 * 2.0 ** 120                              # of bf16
    big = np.abs(want) > largest
    want[big] = np.copysign(np.inf, want[big])
    assert np.array_equal(w.double().cpu().numpy(), want, equal_nan=True)


# ---- products ----

@pytest.mark.parametrize("m,n,p", [
    (1, 32, 0.0), (1, 544, 0.0), (2, 64, 1.0), (63, 64, 0.5), (64, 512, 0.0), (129, 96, 0.5), (513, 512, 0.95),
    (512, 1024, 0.5), (1000, 1056, 0.25), (1031, 4128, 0.5), (2048, 2048, 0.5), (2048, 256, 1.0), (4097, 32, 0.5),
    (4096, 4096, 0.0), (5001, 3424, 0.8), (9000, 352, 0.9), (20000, 64, 0.5), (70001, 32, 0.5), (256, 20000, 0.5)])
def test_product_against_binary64(T, m, n, p):
    codes, scales, values, x, t = make(m, n, p, 7 * m + n)
    q, s, xd, ws = dev(codes), dev(scales), dev(x), workspace(T, m, n)
    y = torch.full((n + 32,), 7.0, device="cuda")
    T.check(T.teal_sparse_gemv_mx4(q, s, xd, t, y, m, n, ws))
    kept = check(y[:n], x, t, values)
    assert survivors(T, ws) == [kept]
    assert bool((y[n:] == 7.0).all())
    if kept == 0:
        assert bool((y[:n] == 0).all())
    again = torch.empty(n, device="cuda")
    for _ in range(3):
        T.check(T.teal_sparse_gemv_mx4(q, s, xd, t, again, m, n, ws))
        assert torch.equal(again, y[:n])


@pytest.mark.parametrize("m,widths,p", [(64, [32], 0.5), (513, [96, 544], 0.5), (2048, [512, 512, 64], 0.5),
                                        (3000, [2048, 512, 512, 1056], 0.65), (4096, [14336, 14336], 0.5),
                                        (8192, [1024], 0.25), (9001, [64, 32], 0.5)])
def test_grouped_product_against_binary64(T, m, widths, p):
    made = [make(m, n, p, 11 * m + n + k) for k, n in enumerate(widths)]
    x = made[0][3]
    ts = [ti.quantile_threshold(x, p) * (1 + 0.2 * k) for k in range(len(widths))]
    ws = workspace(T, m, sum(widths))
    ys = [torch.full((n,), 7.0, device="cuda") for n in widths]
    qs, ss, xd = [dev(c[0]) for c in made], [dev(c[1]) for c in made], dev(x)
    T.check(T.teal_sparse_gemv_mx4_multi(qs, ss, ts, ys, widths, xd, m, ws))
    assert survivors(T, ws, len(widths)) == [check(y, x, t, c[2]) for y, t, c in zip(ys, ts, made)]
    again = [torch.empty_like(y) for y in ys]
    T.check(T.teal_sparse_gemv_mx4_multi(qs, ss, ts, again, widths, xd, m, ws))
    assert all(torch.equal(a, b) for a, b in zip(again, ys))
    if len(widths) == 1:
        T.check(T.teal_sparse_gemv_mx4(qs[0], ss[0], xd, ts[0], again[0], m, widths[0], ws))
        assert torch.equal(again[0], ys[0])


@pytest.mark.parametrize("m,n", [(8, 32), (520, 96), (2048, 2048), (4104, 544), (14336, 1024)])
def test_formed_inputs_are_the_producer_and_the_plain_call(T, m, n):
    codes, scales, _, _, _ = make(m, n, 0.5, m + n)
    q, s, ws = dev(codes), dev(scales), workspace(T, m, 2 * n)
    gate, up = (dev(a) for a in ti.mlp_gate_up(m, 5))
    h, normed = (torch.empty(m, dtype=torch.float16, device="cuda") for _ in range(2))
    y, z = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    T.check(T.teal_swiglu_f16(gate, up, h, m))
    for t in (0.0, 0.25):
        T.check(T.teal_sparse_gemv_mx4(q, s, h, t, y, m, n, ws))
        T.check(T.teal_sparse_gemv_mx4_swiglu(q, s, gate, up, t, z, m, n, ws))
        assert torch.equal(y, z)
        gamma = 0.5 + 0.1 * up
        T.check(T.teal_rmsnorm_f16(gate, gamma, 1e-5, normed, m))
        pairs = [[torch.empty(n, device="cuda") for _ in range(2)] for _ in range(2)]
        T.check(T.teal_sparse_gemv_mx4_multi([q, q], [s, s], [t, 0.5], pairs[0], [n, n], normed, m, ws))
        T.check(T.teal_sparse_gemv_mx4_rmsnorm_multi([q, q], [s, s], [t, 0.5], pairs[1], [n, n], gate, gamma, 1e-5, m, ws))
        assert all(torch.equal(a, b) for a, b in zip(*pairs))


@pytest.mark.parametrize("m,n", [(300, 96), (2048, 2048)])
def test_inputs_of_every_size(T, m, n):
    """Subnormal and the largest fp16 inputs beside ordinary ones; NaN is dropped."""
    codes, scales, values, x, _ = make(m, n, 0.5, 3)
    rng = np.random.default_rng(1)
    x = (x.astype(np.float64) * 2.0 ** rng.integers(-24, 14, m)).astype(np.float16)
    x[::7] = np.float16(65504)
    x[1::11] = np.float16(2.0 ** -24)
    x[2::13] = np.nan
    q, s, ws, y = dev(codes), dev(scales), workspace(T, m, n), torch.empty(n, device="cuda")
    for t in (0.0, 2.0 ** -24, 1.0, 65504.0):
        T.check(T.teal_sparse_gemv_mx4(q, s, dev(x), t, y, m, n, ws))
        assert check(y, np.nan_to_num(x), t, values) == survivors(T, ws)[0]


def test_infinite_inputs_and_nan_blocks(T):
    m, n = 1000, 1056
    codes, scales, values, x, t = make(m, n, 0.5, 9)
    q, s, ws, y = dev(codes), dev(scales), workspace(T, m, n), torch.empty(n, device="cuda")
    x[500] = np.inf
    T.check(T.teal_sparse_gemv_mx4(q, s, dev(x), t, y, m, n, ws))
    want = np.where(values[500] == 0, np.nan, np.copysign(np.inf, values[500]))
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)
    # a NaN block of a channel that is kept is NaN in its 32 columns, of one that is dropped in none
    x[500], x[17] = 3.0, 0.0
    for channel, nan in [(500, True), (17, False)]:
        marked = scales.copy()
        marked[ti.mx4_scale_places(m, n)[channel, 4]] = 255
        T.check(T.teal_sparse_gemv_mx4(q, dev(marked), dev(x), t, y, m, n, ws))
        where = np.zeros(n, bool)
        where[128:160] = nan
        assert np.array_equal(np.isnan(y.cpu().numpy()), where)


def test_scales_of_every_size(T):
    """Blocks from 2^-110 to 2^110; what is below a column's last place goes with it."""
    m, n = 640, 96
    rng = np.random.default_rng(2)
    codes, scales, _, x, t = make(m, n, 0.5, 4)
    scales[ti.mx4_scale_places(m, n)] = rng.integers(17, 237, (m, n // 32))
    y = torch.empty(n, device="cuda")
    T.check(T.teal_sparse_gemv_mx4(dev(codes), dev(scales), dev(x), t, y, m, n, workspace(T, m, n)))
    check(y, x, t, ti.mx4_values(codes, scales))


def test_offsets_past_32_bits(T):
    m, n = 300000, 32768                                     # 4.9 GB of codes
    q = torch.zeros(m, n // 2, dtype=torch.uint8, device="cuda")
    s = torch.full((T.teal_mx4_scale_bytes(m, n),), 120, dtype=torch.uint8, device="cuda")
    tail = 40
    codes = np.random.default_rng(0).integers(0, 256, (tail, n // 2), dtype=np.uint8)
    q[m - tail:] = dev(codes)
    x = np.zeros(m, np.float16)
    x[m - tail:] = ti.gaussian_x(tail, 1)
    y = torch.empty(n, device="cuda")
    T.check(T.teal_sparse_gemv_mx4(q, s, dev(x), 0.25, y, m, n, workspace(T, m, n)))
    values = ti.mx4_values(codes, np.full(ti.mx4_scale_bytes(tail, n), 120, np.uint8))
    check(y, x[m - tail:], 0.25, values)


def test_two_streams_and_a_captured_graph(T):
    m, n = 2048, 2048
    codes, scales, values, x, t = make(m, n, 0.5, 21)
    q, s, xd = dev(codes), dev(scales), dev(x)
    spaces = [workspace(T, m, n) for _ in range(2)]
    ys = [torch.empty(n, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, ws, y in zip(streams, spaces, ys):
            T.check(T.teal_sparse_gemv_mx4(q, s, xd, t, y, m, n, ws, stream=st))
    torch.cuda.synchronize()
    check(ys[0], x, t, values)
    assert torch.equal(ys[0], ys[1])
    graph = torch.cuda.CUDAGraph()
    captured = torch.empty(n, device="cuda")
    with torch.cuda.graph(graph):
        T.check(T.teal_sparse_gemv_mx4(q, s, xd, t, captured, m, n, spaces[0]))
    for k in range(4):
        captured.zero_()
        xd.copy_(dev(np.roll(x, k)))
        graph.replay()
        torch.cuda.synchronize()
        T.check(T.teal_sparse_gemv_mx4(q, s, xd, t, ys[0], m, n, spaces[0]))
        assert torch.equal(captured, ys[0])
        check(captured, np.roll(x, k), t, values)


@pytest.mark.parametrize("m,n", [(8192, 16640), (8256, 16480), (64, 2099200)])
def test_layout_of_a_matrix_larger_than_the_caches(T, m, n):
    """270 MB, read and written past the caches: the same as its parts laid out one by one."""
    g = torch.Generator(device="cuda").manual_seed(7)
    w = (0.02 * torch.randn(n, m, generator=g, device="cuda")).bfloat16()
    q, s = torch.empty(m, n // 2, dtype=torch.uint8, device="cuda"), torch.empty(T.teal_mx4_scale_bytes(m, n), dtype=torch.uint8, device="cuda")
    T.check(T.teal_pack_mx4(w, q, s, m, n))
    back = torch.empty_like(w)
    T.check(T.teal_unpack_mx4(q, s, back, m, n))
    scales = s.view(m // 8, -1, 8, 16)
    for j in range(0, n, 512 if n < 20000 else 1 << 16):
        part = w[j:j + 512]
        cols = part.shape[0]
        pq = torch.empty(m, cols // 2, dtype=torch.uint8, device="cuda")
        ps = torch.empty(T.teal_mx4_scale_bytes(m, cols), dtype=torch.uint8, device="cuda")
        T.check(T.teal_pack_mx4(part, pq, ps, m, cols))
        assert torch.equal(q[:, j // 2:(j + cols) // 2], pq) and torch.equal(scales[:, j // 512:(j + cols + 511) // 512], ps.view(m // 8, -1, 8, 16))
        pw = torch.empty(cols, m + 2, dtype=torch.bfloat16, device="cuda").flatten()[1:1 + cols * m]      # off the lines
        T.check(T.teal_unpack_mx4(pq, ps, pw, m, cols))
        assert torch.equal(back[j:j + cols], pw.view(cols, m))
