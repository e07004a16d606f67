"""What the operators around a packed projection hold their sums and values in."""
import pytest

torch = pytest.importorskip("torch")

BITS, GATES, PAIRS = 0x50420002, 0x50420003, 0x50420004


@pytest.fixture(scope="module")
def pb():
    from paper_2003_00822_amd import build
    build.ensure(verbose=False)
    from paper_2003_00822_amd import pb as _pb
    _pb.lib()
    return _pb


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


# rows, cols, bits, used, batch, layout, scales that do not halve.  Large batches: 192 workgroups of 128 rows and 128 vectors or more.
GROUPS = [
    (3100, 520, 12, 11, 1000, GATES, False), (3100, 300, 6, 6, 950, GATES, True), (3096, 1100, 3, 3, 1001, GATES, True),
    (3100, 515, 11, 11, 1000, BITS, False), (3100, 300, 3, 3, 990, BITS, True), (24600, 40, 16, 16, 65, BITS, False),
    (3090, 1100, 12, 12, 1021, PAIRS, False), (3100, 520, 16, 16, 1000, PAIRS, False), (6200, 33, 5, 5, 520, PAIRS, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,bits,m,batch,layout,odd", GROUPS)
def test_several_groups_of_bitlayers_give_the_product_of_matmul(pb, rows, cols, bits, m, batch, layout, odd):
    """The sum over the groups is in fp64 and rounded once, as in pb_matmul: the same bits."""
    lin = pb.PackedLinear(rand(1, rows, cols) * 0.05, bits, max_batch=batch, layout=layout)
    if odd:
        lin.scales[:bits] = torch.tensor([-1.5, 0.7, 0.01, 3.0, -0.2, 1.0][:bits], device="cuda") * 0.1
    X, bias = rand(2, batch, cols), rand(3, rows)
    X[[3, batch // 2, batch - 1]] *= 300                       # (values beyond three byte digits)
    for b in (None, bias):
        want = torch.empty((batch, rows), device="cuda")
        pb.pb_matmul_bias_act(lin.packed, lin.scales, lin.desc, m, X, batch, b, pb.PB_ACT_NONE, want, lin.workspace)
        if layout == GATES:
            H, pre = lin.gated(X, pb.PB_GATE_SILU, m, bias=b, keep=True)
            assert torch.equal(pre, want)
            assert torch.equal(lin.gated(X, pb.PB_GATE_SILU, m, bias=b), H)
            size = pb.pb_workspace_bytes(lin.desc, batch)
            ws, out = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda"), torch.empty_like(H)
            pb.pb_gated_linear(lin.packed, lin.scales, lin.desc, m, X, batch, b, pb.PB_GATE_SILU, out, None, ws)
            assert torch.equal(out, H) and (ws[size:] == 0xA5).all()
        else:
            none = torch.full((batch,), -1, dtype=torch.int32, device="cuda")
            adapters = pb.Adapters(torch.zeros((1, 1, cols), device="cuda"), torch.zeros((1, rows, 1), device="cuda"))
            assert torch.equal(lin.adapted(X, adapters, none, m, bias=b), want)
