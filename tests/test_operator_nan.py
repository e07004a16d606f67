"""Gated blocks: a pre-activation that is NaN makes its unit's results NaN, and no others."""
import pytest

torch = pytest.importorskip("torch")

BITS, GATES, PAIRS, ROWS = 0x50420002, 0x50420003, 0x50420004, 0x50420001


@pytest.fixture(scope="module")
def pb():
    from paper_2003_00822_amd import build
    build.ensure(verbose=False)
    from paper_2003_00822_amd import pb as _pb
    _pb.lib()
    return _pb


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [0, 1, 2, 3])
@pytest.mark.parametrize("units,batch,layout", [(300, 1, GATES), (300, 6, GATES), (300, 60, GATES), (1550, 1000, GATES), (129, 1, BITS), (130, 9, PAIRS), (33, 2, ROWS)])
def test_a_bias_that_is_nan_shows(pb, units, batch, layout, gate):
    lin = pb.PackedLinear(rand(1, 2 * units, 200) * 0.1, 8, layout=layout)
    X, bias = rand(2, batch, 200), rand(3, 2 * units)
    clean = lin.gated(X, gate, bias=bias)
    bias[[5, units + 9]] = float("nan")
    H, pre = lin.gated(X, gate, bias=bias, keep=True)
    hit = [5, 9]
    others = [r for r in range(units) if r not in hit]
    assert torch.isnan(H[:, hit]).all() and torch.isnan(pre[:, [5, units + 9]]).all()
    assert torch.equal(H[:, others], clean[:, others])
    assert torch.equal(lin.gated(X, gate, bias=bias).isnan(), H.isnan())


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [0, 1, 2, 3])
@pytest.mark.parametrize("units,batch,layout", [(300, 3, GATES), (300, 100, GATES), (129, 5, BITS), (150, 40, PAIRS), (2000, 300, GATES)])
def test_the_slope_of_nan_is_nan(pb, units, batch, layout, gate):
    lin = pb.PackedLinear(rand(1, 2 * units, 100) * 0.1, 8, layout=layout)
    pre, dH = rand(2, batch, 2 * units), rand(3, batch, units)
    dX, dpre = lin.gated_grad(pre, dH, gate)
    pre[0, 4] = float("nan")                 # a gate
    pre[2, units + 7] = float("nan")         # a value
    got_X, got = lin.gated_grad(pre, dH, gate)
    want = dpre.clone()
    want[0, [4, units + 4]] = float("nan")   # dH u act'(g) and dH act(g)
    want[2, 7] = float("nan")                # dH u act'(g)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(), want.nan_to_num())
    others = [n for n in range(batch) if n not in (0, 2)]
    assert torch.isnan(got_X[[0, 2]]).all() and torch.isfinite(got_X[others]).all()
    # (the digits of a group of sixteen vectors may change with one of them: the others are compared as they would be without these two)
    if batch <= 32:
        assert torch.equal(got_X[others], dX[others])
