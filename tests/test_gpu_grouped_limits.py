"""The grouped experts' products at the ends of what they accept, on the GPU: the most pairs, the widest matrices, the longest sums,
microscaled weights beyond 32-bit offsets.

Whole numbers throughout: sums are exact, and H is off by 2^-16 of itself before its rounding to bf16 and half a step of 2^-8 by
it (a gate below -87 may give 0)."""
import pytest

from test_gpu_grouped_experts import arranged
from test_gpu_mx4 import T  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def whole(gen, *shape, most=2):
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").bfloat16()


def pack(T, w):   # noqa: F811
    """Codes and scales of [experts][m][n] whole numbers of at most 4, which microscaled weights have."""
    experts, m, n = w.shape
    codes = torch.empty(experts, m, n // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(experts, T.teal_mx4_scale_bytes(m, n), dtype=torch.uint8, device="cuda")
    for e in range(experts):
        T.check(T.teal_pack_mx4(w[e].t().contiguous(), codes[e], scales[e], m, n))
    return codes, scales


def gate_up(T, fmt):   # noqa: F811
    return T.teal_grouped_experts_bf16_gate_up if fmt == "bf16" else T.teal_grouped_experts_mx4_gate_up


def down(T, fmt):   # noqa: F811
    return T.teal_grouped_experts_bf16_down if fmt == "bf16" else T.teal_grouped_experts_mx4_down


def check_h(h, g, u):
    want = g * torch.sigmoid(g) * u
    off = want.abs() * (2.0 ** -8 + 2.0 ** -15) + torch.where(g < -87, 1.5e-36 * u.abs(), 0.0) + 2.0 ** -133
    assert bool(((h.double() - want).abs() <= off).all())


def test_the_most_pairs(T):   # noqa: F811
    """2^24 of them over 1024 experts, some without one."""
    gen = torch.Generator(device="cuda").manual_seed(61)
    tokens, top_k, experts, m, f, n = 1 << 19, 32, 1024, 8, 8, 8
    idx = torch.randint(-8, experts, (tokens, top_k), generator=gen, device="cuda", dtype=torch.int32)
    pairs = tokens * top_k
    order, start = torch.empty(pairs, dtype=torch.int32, device="cuda"), torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    need = max(T.teal_workspace_bytes_arrange_experts(experts, pairs), T.teal_workspace_bytes_grouped_experts(pairs, n))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    T.check(T.teal_arrange_experts(idx, tokens, top_k, experts, order, start, ws))
    want_order, want_start = arranged(idx.cpu().numpy(), experts)
    assert torch.equal(order.cpu(), torch.from_numpy(want_order)) and torch.equal(start.cpu(), torch.from_numpy(want_start))
    gate, up, W = whole(gen, experts, m, f), whole(gen, experts, m, f), whole(gen, experts, f, n)
    x, h = whole(gen, tokens, m), torch.full((pairs, f), 7.0, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_grouped_experts_bf16_gate_up(gate, up, experts, order, start, tokens, top_k, x, h, m, f))
    used = int(start[experts])
    assert used < pairs and bool((h[used:] == 7.0).all())
    for a in range(0, used, 1 << 20):
        pair = order[a:min(used, a + (1 << 20))].long()
        e, row = idx.flatten()[pair].long(), x[pair // top_k].double()[:, None]
        check_h(h[a:a + (1 << 20)][:pair.numel()], *((row @ w[e].double())[:, 0] for w in (gate, up)))
    h = whole(gen, pairs, f)
    weight = torch.exp2(torch.randint(-2, 3, (tokens, top_k), generator=gen, device="cuda").float())
    y = torch.empty(tokens, n, device="cuda")
    T.check(T.teal_grouped_experts_bf16_down(W, experts, order, start, tokens, top_k, idx, weight, h, y, f, n, ws))
    place = torch.empty(pairs, dtype=torch.long, device="cuda")
    place[order.long()] = torch.arange(pairs, device="cuda")
    for b in range(0, tokens, 1 << 15):
        part = slice(b, b + (1 << 15))
        e = idx[part].long()
        row = h[place.view(tokens, top_k)[part]].double()[..., None, :]
        one = (row @ W[e.clamp(min=0)].double())[..., 0, :] * weight[part].double()[..., None] * (e >= 0)[..., None]
        assert torch.equal(y[part].double(), one.sum(1))


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens", [5, 300])
def test_the_widest_matrices(T, fmt, tokens):   # noqa: F811
    """Experts 2^20 wide, and a model width of 2^20, which W_down of 300 pairs takes in parts."""
    gen = torch.Generator(device="cuda").manual_seed(62)
    wide, m, experts = 1 << 20, 8, 2
    idx = (torch.arange(tokens, device="cuda") % experts).int()[:, None].contiguous()
    want_order, want_start = arranged(idx.cpu().numpy(), experts)
    group = (experts, torch.from_numpy(want_order).cuda(), torch.from_numpy(want_start).cuda(), tokens, 1)
    a, b = whole(gen, experts, m, wide), whole(gen, experts, m, wide)
    wa, wb = ((a,), (b,)) if fmt == "bf16" else (pack(T, a), pack(T, b))
    x, h = whole(gen, tokens, m), torch.empty(tokens, wide, dtype=torch.bfloat16, device="cuda")
    T.check(gate_up(T, fmt)(*wa, *wb, *group, x, h, m, wide))
    y, one = torch.empty(tokens, wide, device="cuda"), torch.ones(tokens, 1, device="cuda")
    size = T.teal_workspace_bytes_grouped_experts(tokens, wide)
    assert (size < tokens * wide * 4) == (tokens == 300)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    # m = 8 channels of H, which a place has in the experts' order
    few = whole(gen, tokens, m)
    T.check(down(T, fmt)(*wa, *group, idx, one, few, y, m, wide, ws))
    for e in range(experts):
        pairs = group[1][int(group[2][e]):int(group[2][e + 1])].long()
        places = torch.arange(int(group[2][e]), int(group[2][e + 1]), device="cuda")
        for c in range(0, wide, 1 << 18):
            part = slice(c, c + (1 << 18))
            check_h(h[places, part], x[pairs].double() @ a[e, :, part].double(), x[pairs].double() @ b[e, :, part].double())
            assert torch.equal(y[pairs, part].double(), few[places].double() @ a[e, :, part].double())


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens", [5, 300])
def test_the_longest_sums(T, fmt, tokens):   # noqa: F811
    """2^20 channels; whole numbers whose sums are below 2^24."""
    gen = torch.Generator(device="cuda").manual_seed(63)
    m, n, experts = 1 << 20, 32, 2
    idx = (torch.arange(tokens, device="cuda") % experts).int()[:, None].contiguous()
    want_order, want_start = arranged(idx.cpu().numpy(), experts)
    group = (experts, torch.from_numpy(want_order).cuda(), torch.from_numpy(want_start).cuda(), tokens, 1)
    w, h = whole(gen, experts, m, n), whole(gen, tokens, m, most=1)
    packed = (w,) if fmt == "bf16" else pack(T, w)
    y, one = torch.empty(tokens, n, device="cuda"), torch.ones(tokens, 1, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_grouped_experts(tokens, n), dtype=torch.uint8, device="cuda")
    T.check(down(T, fmt)(*packed, *group, idx, one, h, y, m, n, ws))
    out = torch.empty(tokens, n, dtype=torch.bfloat16, device="cuda")
    T.check(gate_up(T, fmt)(*packed, *packed, *group, h, out, m, n))
    for e in range(experts):
        a, b = int(group[2][e]), int(group[2][e + 1])
        pairs, places = group[1][a:b].long(), torch.arange(a, b, device="cuda")
        assert torch.equal(y[pairs].double(), h[places].double() @ w[e].double())
        g = h[pairs].double() @ w[e].double()
        check_h(out[places], g, g)


def test_microscaled_weights_beyond_32_bits(T):   # noqa: F811
    """600 experts of 4096 x 4096: 5 GB of codes; those before the last two have NaN scales."""
    gen = torch.Generator(device="cuda").manual_seed(64)
    experts, m, tokens = 600, 4096, 40
    codes = torch.empty(experts, m, m // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((experts, T.teal_mx4_scale_bytes(m, m)), 255, dtype=torch.uint8, device="cuda")
    assert codes[:-2].numel() > 2 ** 32
    w = whole(gen, 2, m, m)
    codes[-2:], scales[-2:] = pack(T, w)
    idx = torch.tensor([[experts - 1, experts - 2]] * tokens, dtype=torch.int32, device="cuda")
    want_order, want_start = arranged(idx.cpu().numpy(), experts)
    group = (experts, torch.from_numpy(want_order).cuda(), torch.from_numpy(want_start).cuda(), tokens, 2)
    x, h = whole(gen, tokens, m, most=1), torch.empty(2 * tokens, m, dtype=torch.bfloat16, device="cuda")
    T.check(T.teal_grouped_experts_mx4_gate_up(codes, scales, codes, scales, *group, x, h, m, m))
    for e in range(2):
        g = x.double() @ w[e].double()
        check_h(h[e * tokens:(e + 1) * tokens], g, g)
    h, y = whole(gen, 2 * tokens, m, most=1), torch.empty(tokens, m, device="cuda")
    ws = torch.zeros(T.teal_workspace_bytes_grouped_experts(2 * tokens, m), dtype=torch.uint8, device="cuda")
    T.check(T.teal_grouped_experts_mx4_down(codes, scales, *group, idx, torch.ones(tokens, 2, device="cuda"), h, y, m, m, ws))
    want = sum(h[e * tokens:(e + 1) * tokens].double() @ w[e].double() for e in range(2))
    assert torch.equal(y.double(), want)
