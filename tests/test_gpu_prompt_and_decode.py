"""A mixture of experts for a few tokens through the calls of many tokens and through those of a decode step, on the GPU: the
same numbers to what the two round differently.

Tolerance, for each output: x is exact in bf16 and fp16.  The sums g and u of m exact products are off by at most
m * 2^-23 * sum |x w| on either side.  They go through SiLU(g) * u, whose derivatives are at most 1.1 |u| and |g| in size.  That
value is off by 2^-16 and rounded by 2^-8 of itself (bf16, many tokens), or off by 2^-20 and rounded by 2^-11 of itself or 2^-25
(fp16, a decode step).  What h is off by goes through |W_down|, whose own sums of f products are off by
f * 2^-23 * sum |h w|, and the join of top_k rows adds top_k + 1 roundings of 2^-24."""
import pytest

from test_gpu_grouped_experts import Case
from test_gpu_mx4 import T  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def decode(T, c):   # noqa: F811
    """The calls of a decode step, dense, with c's weights, rows and choice."""
    g, u = (torch.empty(c.tokens, c.top_k, c.f, device="cuda") for _ in range(2))
    zero, y = torch.zeros(c.experts, device="cuda"), torch.empty(c.tokens, c.n, device="cuda")
    size = max(T.teal_workspace_bytes_experts(c.m, 2 * c.f, c.pairs), T.teal_workspace_bytes_experts(c.f, c.n, c.pairs))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    up, down = ((T.teal_sparse_experts_bf16, T.teal_sparse_experts_bf16_swiglu) if c.fmt == "bf16" else
                (T.teal_sparse_experts_mx4, T.teal_sparse_experts_mx4_swiglu))
    T.check(up(*([a, b] for a, b in zip(c.gate, c.up)), [zero, zero], [g, u], [c.f, c.f], c.experts, c.idx, c.tokens, c.top_k,
               c.x.half(), c.m, ws))
    T.check(down(*c.down, zero, y, c.experts, c.idx, c.weight, c.tokens, c.top_k, g, u, c.f, c.n, ws))
    return y


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("tokens,top_k,experts,m,f,n", [(1, 2, 8, 256, 96, 256), (8, 2, 8, 256, 96, 256), (5, 6, 16, 520, 160, 544),
                                                        (8, 4, 4, 1024, 768, 1024)])
def test_many_tokens_and_a_decode_step(T, fmt, tokens, top_k, experts, m, f, n):   # noqa: F811
    c = Case(T, fmt, tokens, top_k, experts, m, f, n, seed=3)
    c.x[c.x.abs() < 2.0 ** -14] = 0
    assert torch.equal(c.x.half().float(), c.x.float())
    y, want = c.run_down(c.run_gate_up()), decode(T, c)
    off = torch.zeros(c.pairs, n, dtype=torch.float64, device="cuda")
    part = torch.zeros_like(off)
    for e, _, pairs in c.places():
        x, weight = c.x[pairs // top_k].double(), c.weight.flatten()[pairs].double()[:, None]
        g, u = x @ c.gate64[e], x @ c.up64[e]
        off_g, off_u = (m * 2.0 ** -23 * (x.abs() @ w[e].abs()) for w in (c.gate64, c.up64))
        h = g * torch.sigmoid(g) * u
        from_sums = 1.1 * off_g * (u.abs() + off_u) + off_u * (g.abs() + off_g)
        size = h.abs() + from_sums
        off_h = 2 * from_sums + size * (2.0 ** -8 + 2.0 ** -16 + 2.0 ** -11 + 2.0 ** -19) + 2.0 ** -25 + 2.0 ** -133
        W = c.down64[e].abs()
        off[pairs] = weight * (off_h @ W + 2 * (f * 2.0 ** -23 + (top_k + 1) * 2.0 ** -24) * ((size + off_h) @ W))
        part[pairs] = weight * (h @ c.down64[e])
    off, part = off.unflatten(0, (tokens, top_k)).sum(1), part.unflatten(0, (tokens, top_k))
    # Close enough that an expert that is missing, or twice there, would be seen, at least if it is the token's largest:
    # a bound is that of all its experts together.
    assert bool((part.abs() > off[:, None]).any(-1).gather(1, c.weight.argmax(1, keepdim=True)).all())
    assert bool(((y.double() - want.double()).abs() <= off).all())
