"""Workspaces of the operators around a packed projection: one that is made for the largest batch serves every smaller one."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pb():
    from paper_2003_00822_amd import build
    build.ensure(verbose=False)
    from paper_2003_00822_amd import pb as _pb
    _pb.lib()
    return _pb


LAYERS = [(2048, 8192, 8), (4096, 4096, 8), (300, 700, 4), (16, 32768, 1), (70000, 33, 2), (1024, 4096, 8), (60, 40, 16)]


@pytest.mark.parametrize("rows,cols,bits", LAYERS)
def test_sizes_do_not_fall_with_the_batch(pb, rows, cols, bits):
    L, ref = pb.lib(), ctypes.byref
    for layout in (pb.PB_LAYOUT_TILE16_V1, pb.PB_LAYOUT_TILE16_GATES_V1, pb.PB_LAYOUT_TILE16_PAIRS_V1, pb.PB_LAYOUT_ROWMAJOR_V1):
        if layout == pb.PB_LAYOUT_TILE16_GATES_V1 and rows % 4:
            continue
        d = pb.pb_desc_init_layout(rows, cols, bits, layout)
        sizes = [L.pb_workspace_bytes, L.pb_grad_workspace_bytes]
        for count, rank in ((1, 8), (3, 256), (40, 33), (4096, 16)):
            a = pb.pb_adapters(count, rank, pb.PB_TYPE_F32, 0, None, None, None)
            sizes.append(lambda d, n, a=a: L.pb_adapters_workspace_bytes(d, ref(a), n))
        for size in sizes:
            of = [size(ref(d), n) for n in range(1, pb.PB_MAX_BATCH + 1)]
            assert all(a <= b for a, b in zip(of, of[1:])), (layout, [n + 1 for n in range(len(of) - 1) if of[n] > of[n + 1]][:5])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,largest,batches", [(2048, 8192, 236, (128, 200, 16)), (4096, 4096, 513, (512, 64, 1)), (1024, 4096, 65, (64, 33, 32))])
def test_a_workspace_of_the_largest_batch_serves_the_smaller_ones(pb, rows, cols, largest, batches):
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g).cuda()   # noqa: E731
    lin = pb.PackedLinear(rand(rows, cols) * 0.05, 8)
    adapters = pb.Adapters(rand(2, 256, cols).half(), rand(2, rows, 256).half())
    d, a = lin.desc, adapters.desc()
    size = pb.pb_adapters_workspace_bytes(d, a, largest)
    grad_size = pb.pb_grad_workspace_bytes(d, largest)
    ws, grad_ws = (torch.full((s + 4096,), 0xA5, dtype=torch.uint8, device="cuda") for s in (size, grad_size))
    for n in batches:
        X, dY = rand(n, cols), rand(n, rows)
        for index in (None, torch.from_numpy(np.random.default_rng(n).integers(-1, 2, n).astype(np.int32)).cuda()):
            Y, dX, dA, dB = torch.empty_like(dY), torch.empty_like(X), rand(2, 256, cols), rand(2, rows, 256)
            pb.pb_matmul_adapters(lin.packed, lin.scales, d, 8, X, n, a, index, None, Y, ws)
            pb.pb_matmul_adapters_grad(lin.packed, lin.scales, d, 8, X, dY, n, a, index, dX, dA, dB, ws)
            assert torch.equal(Y, lin.adapted(X, adapters, index))
            for got, want in zip((dX, dA, dB), lin.adapted_grad(X, dY, adapters, index)):
                assert torch.equal(got, want)
        pb.pb_matmul_grad(lin.packed, lin.scales, d, 8, dY, n, dX, grad_ws)
        assert torch.equal(dX, lin.grad(dY))
        torch.cuda.synchronize()
        assert (ws[size:] == 0xA5).all() and (grad_ws[grad_size:] == 0xA5).all()
