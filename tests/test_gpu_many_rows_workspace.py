"""One workspace for the calls of many rows and then for those with counters behind its first region (stacks of groups, a whole
MLP), on the GPU: every call that asks for no more than the first region leaves it ready for them, bit for bit."""
import pytest

from test_gpu_many_rows import make_rows, product, random_ints
from test_gpu_mx4 import T  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class ManyRows:
    """An int8 product in slices, pairs sorted by expert (more than one chunk of them) and W_down of grouped experts."""

    def __init__(self, T, gen):   # noqa: F811
        self.T = T
        self.w8, self.scale = random_ints(gen, 4096, 1024), (torch.rand(1024, generator=gen, device="cuda") * 0.01).half()
        self.q, self.row_scale = make_rows(T, gen, 40, 4096)
        self.idx = torch.randint(0, 16, (5000, 2), generator=gen, device="cuda", dtype=torch.int32)
        self.down = torch.randn(16, 64, 264, generator=gen, device="cuda").bfloat16()
        self.h = torch.randn(10000, 64, generator=gen, device="cuda").bfloat16()
        self.weight = torch.rand(5000, 2, generator=gen, device="cuda")
        self.need = max(T.teal_workspace_bytes_gemm_w8(64, 4096, 1024), T.teal_workspace_bytes_arrange_experts(16, 10000),
                        T.teal_workspace_bytes_grouped_experts(10000, 264))

    def run(self, ws):
        T, order = self.T, torch.empty(10000, dtype=torch.int32, device="cuda")
        start, y = torch.empty(17, dtype=torch.int32, device="cuda"), torch.empty(5000, 264, device="cuda")
        many = torch.empty(40, 1024, device="cuda")
        T.check(T.teal_gemm_w8_ex([self.w8], [self.scale], [many], [1024], self.q, self.row_scale, 40, 4096, ws, tile_rows=64,
                                  tile_cols=128, splits=16))
        T.check(T.teal_arrange_experts(self.idx, 5000, 2, 16, order, start, ws))
        T.check(T.teal_grouped_experts_bf16_down(self.down, 16, order, start, 5000, 2, self.idx, self.weight, self.h, y, 64, 264, ws))
        assert torch.equal(many, product(self.q, self.row_scale, self.w8, self.scale))
        return y


@pytest.mark.parametrize("kind", ["stack", "mlp"])
def test_stacks_and_mlps_after_calls_of_many_rows(T, kind):   # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(91)
    rows = ManyRows(T, gen)

    def weights(*shape):
        return (0.05 * torch.randn(*shape, generator=gen, device="cuda")).bfloat16()

    x = torch.randn(512, generator=gen, device="cuda").half()
    if kind == "stack":
        counts, n, m = [1, 2], [72000, 520, 264], [512, 512]
        W = [weights(512, k) for k in n]
        size, first = T.teal_workspace_bytes_stack(counts, n, m), T.teal_workspace_bytes(512, n[0])

        def call(ws):
            ys = [torch.full((k,), float("nan"), device="cuda") for k in n]
            T.check(T.teal_sparse_gemv_bf16_stack(counts, W, [0.5] * 3, ys, n, [x, x], m, ws))
            return torch.cat(ys)
    else:
        f, d = 36000, 520
        gate, up, down = weights(512, f), weights(512, f), weights(f, d)
        size, first = T.teal_workspace_bytes_mlp(512, f, d), T.teal_mlp_down_region_offset(512, f)
        status = T.teal_mlp_status_offset(512, f, d)

        def call(ws):
            ys = [torch.full((k,), float("nan"), device="cuda") for k in (f, f, d)]
            T.check(T.teal_sparse_mlp_bf16(gate, up, down, x, 0.5, 0.5, 0.1, *ys, 512, f, d, ws))
            assert int(ws[status:status + 4].view(torch.int32)) == 0
            return torch.cat(ys)

    assert rows.need <= first
    want, want_rows = call(torch.zeros(size, dtype=torch.uint8, device="cuda")), rows.run(
        torch.zeros(rows.need, dtype=torch.uint8, device="cuda"))
    assert bool(torch.isfinite(want).all())
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        assert torch.equal(rows.run(ws), want_rows)
        assert torch.equal(call(ws), want)
