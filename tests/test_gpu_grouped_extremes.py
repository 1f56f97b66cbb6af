"""Weights and rows at the ends of their types through the grouped experts' products, on the GPU.

Nothing here has a tolerance: a row has one entry that is not zero, a power of two, so an output is one product, and that is
a number that fp32 has."""
import numpy as np
import pytest

import teal_inputs as ti
from test_gpu_mx4 import T, dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROWS = 256


def down(T, fmt, weights, experts, h, n):   # noqa: F811
    """h W^T for every row; row b goes to expert b % experts, which all have the same weights."""
    rows, f = h.shape
    order = torch.arange(rows, device="cuda").reshape(-1, experts).t().reshape(-1).int().contiguous()
    start = (torch.arange(experts + 1, device="cuda") * (rows // experts)).int()
    idx = (torch.arange(rows, device="cuda") % experts).int()[:, None].contiguous()
    weights = [w.expand(experts, *w.shape).contiguous() for w in weights]
    y, one = torch.empty(rows, n, device="cuda"), torch.ones(rows, 1, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_grouped_experts(rows, n), dtype=torch.uint8, device="cuda")
    call = T.teal_grouped_experts_bf16_down if fmt == "bf16" else T.teal_grouped_experts_mx4_down
    T.check(call(*weights, experts, order, start, rows, 1, idx, one, h[order.long()].contiguous(), y, f, n, ws))
    return y


def one_entry(rows, f, channel, exponent):
    """Row b has 2^exponent[b] at channel[b], zeros beside it."""
    h = torch.zeros(rows, f, dtype=torch.float64, device="cuda")
    h[torch.arange(rows, device="cuda"), channel] = torch.exp2(exponent)
    return h.bfloat16()


# few and many rows of an expert: tiles of 32 x 128, 64 x 128, 256 x 128 and (24000 columns) 256 x 256
@pytest.mark.parametrize("experts,n", [(64, 32), (16, 96), (1, 64), (1, 24000)])
def test_every_scale_and_code(T, experts, n):   # noqa: F811
    """Scale bytes 0 to 252, weights from 2^-128 to 6 * 2^125: every weight counts as what it is, subnormal ones too."""
    f = 256
    pick = np.arange(n, dtype=np.uint8) % 16
    codes = np.tile(pick[0::2] | pick[1::2] << 4, (f, 1))
    scales = np.zeros(ti.mx4_scale_bytes(f, n), np.uint8)
    bytes_ = np.minimum(np.arange(f), 252)
    scales[ti.mx4_scale_places(f, n)] = bytes_[:, None].astype(np.uint8)
    values = torch.from_numpy(ti.mx4_values(codes, scales)).cuda()
    channel = torch.arange(ROWS, device="cuda")
    # products of about 1
    h = one_entry(ROWS, f, channel, (127 - torch.from_numpy(bytes_).cuda()).double())
    y = down(T, "mx4", (dev(codes), dev(scales)), experts, h, n)
    want = h.double()[torch.arange(ROWS, device="cuda"), channel][:, None] * values
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("experts,n", [(64, 64), (16, 64), (1, 64), (1, 24000)])
@pytest.mark.parametrize("byte", [253, 254])
def test_weights_beyond_bf16_are_infinities(T, experts, n, byte):   # noqa: F811
    """As in teal_unpack_mx4, and in their own columns only."""
    f = 64
    pick = np.arange(n, dtype=np.uint8) % 16
    codes = np.zeros((f, n // 2), np.uint8)
    codes[5] = pick[0::2] | pick[1::2] << 4
    scales = np.zeros(ti.mx4_scale_bytes(f, n), np.uint8)
    places = ti.mx4_scale_places(f, n)
    scales[places[5]] = 127
    scales[places[5, 0]] = byte
    values = torch.from_numpy(ti.mx4_values(codes, scales)[5]).cuda()
    largest = 255 * 2.0 ** 120                              # of bf16
    values = torch.where(values.abs() > largest, torch.copysign(torch.full_like(values, float("inf")), values), values)
    assert int(torch.isinf(values).sum()) > 0
    y = down(T, "mx4", (dev(codes), dev(scales)), experts, one_entry(ROWS, f, torch.full((ROWS,), 5, device="cuda"),
                                                                    torch.zeros(ROWS, dtype=torch.float64, device="cuda")), n)
    assert torch.equal(y.double(), values.expand(ROWS, n))


@pytest.mark.parametrize("experts", [64, 16, 2, 1])
def test_every_bf16_number(T, experts):   # noqa: F811
    """All that are finite, subnormal ones too, as weights and as a row's entries, times one."""
    finite = np.arange(1 << 16, dtype=np.uint32)
    finite = finite[(finite & 0x7F80) != 0x7F80].astype(np.uint16)
    n = finite.size
    w = torch.zeros(8, n, dtype=torch.bfloat16, device="cuda")
    w[3] = dev(finite).view(torch.bfloat16)
    zero = torch.zeros(ROWS, dtype=torch.float64, device="cuda")
    y = down(T, "bf16", (w,), experts, one_entry(ROWS, 8, torch.full((ROWS,), 3, device="cuda"), zero), n)
    assert torch.equal(y, w[3].float().expand(ROWS, n))
    one = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    h = dev(finite).view(torch.bfloat16)
    for part in (h[:ROWS * 64], h[n // 2 - 32 * ROWS:n // 2 + 32 * ROWS], h[n - ROWS * 64:]):
        # each row has 64 numbers, and each column takes one of them
        part = part.reshape(ROWS, 64).contiguous()
        assert torch.equal(down(T, "bf16", (one,), experts, part, 64), part.float())


@pytest.mark.parametrize("up", [1.0, -1.3671875, 2.0 ** -20, 3.0 * 2.0 ** 60])
@pytest.mark.parametrize("experts", [64, 1])
def test_silu_of_every_bf16_number(T, experts, up):   # noqa: F811
    """H lies between the roundings of what is 2^-16 smaller and larger, by 2^-148 where that is subnormal; nothing below g = -87
    is larger than it may be; NaN and infinities come out as the formula in 32 bits has them."""
    every = dev(np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)).view(torch.bfloat16)
    f = every.numel()
    gate, other = (torch.zeros(experts, 8, f, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gate[:, 3], other[:, 3] = every, up
    rows = 128
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    x[:, 3] = 1
    order = torch.arange(rows, dtype=torch.int32, device="cuda")
    start = (torch.arange(experts + 1, device="cuda") * (rows // experts)).int()
    h = torch.empty(rows, f, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_grouped_experts_bf16_gate_up(gate, other, experts, order, start, rows, 1, x, h, 8, f))
    assert bool((h.view(torch.int16) == h[0].view(torch.int16)).all())
    h, g = h[0], every.double()
    want = g / (1 + torch.exp(-g)) * up
    room = want.abs() * 2.0 ** -16 + 2.0 ** -148
    low, high = ((want + s * room).float().bfloat16() for s in (-1, 1))
    ok = (h >= low) & (h <= high) | torch.isnan(want) & torch.isnan(h) | torch.isinf(want) & (h.double() == want)
    ok |= (g < -87) & (h.double().abs() <= 1.5e-36 * abs(up))
    assert bool(ok.all()), every[~ok][:8].tolist()
