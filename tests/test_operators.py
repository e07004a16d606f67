"""Gated blocks, low-rank adapters and gradients through a packed matrix: refusals on the host, results on the GPU against the definitions in 64
bits.  Weights and scales of the references come from `oracle/`."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import pb_oracle as po   # noqa: E402

U = 2.0 ** -24      # half a step of fp32, relative


@pytest.fixture(scope="module")
def pb():
    from paper_2003_00822_amd import build
    build.ensure(verbose=False)
    from paper_2003_00822_amd import pb as _pb
    _pb.lib()
    return _pb


# ---- on the host ----
def test_arguments_rejected_before_launch(pb):
    L, ref = pb.lib(), ctypes.byref
    fake, odd, null = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0)
    d, rows = pb.pb_desc_init(64, 96, 4), pb.pb_desc_init_layout(64, 96, 4, pb.PB_LAYOUT_ROWMAJOR_V1)
    uneven = pb.pb_desc_init(65, 96, 4)

    def gated(d=d, m=4, x=fake, n=1, bias=null, gate=1, h=fake, pre=null, ws=fake, scales=fake):
        return L.pb_gated_linear(fake, scales, ref(d), m, x, n, bias, gate, h, pre, ws, null)
    for bad in (dict(d=uneven), dict(m=0), dict(m=5), dict(x=null), dict(n=0), dict(gate=4), dict(gate=-1), dict(h=null), dict(ws=null),
                dict(scales=null)):
        assert gated(**bad) == pb.PB_EINVAL, bad
    for bad in (dict(x=odd), dict(bias=odd), dict(h=odd), dict(pre=odd), dict(ws=odd)):
        assert gated(**bad) == pb.PB_EALIGN, bad
    assert gated(n=pb.PB_MAX_BATCH + 1) == pb.PB_ESIZE

    def grad(d=d, m=4, dy=fake, n=1, dx=fake, ws=fake, scales=fake, packed=fake):
        return L.pb_matmul_grad(packed, scales, ref(d), m, dy, n, dx, ws, null)
    for bad in (dict(d=rows), dict(m=0), dict(m=5), dict(dy=null), dict(n=0), dict(dx=null), dict(ws=null), dict(scales=null), dict(packed=null)):
        assert grad(**bad) == pb.PB_EINVAL, bad
    for bad in (dict(dy=odd), dict(dx=odd), dict(ws=odd), dict(scales=odd), dict(packed=odd)):
        assert grad(**bad) == pb.PB_EALIGN, bad
    assert grad(n=pb.PB_MAX_BATCH + 1) == pb.PB_ESIZE
    assert L.pb_matmul_grad(fake, fake, None, 4, fake, 1, fake, fake, null) == pb.PB_EINVAL

    def gated_grad(d=d, pre=fake, dh=fake, gate=1, dpre=fake, dx=fake):
        return L.pb_gated_linear_grad(fake, fake, ref(d), 4, pre, dh, 1, gate, dpre, dx, fake, null)
    for bad in (dict(d=rows), dict(d=uneven), dict(pre=null), dict(dh=null), dict(gate=9), dict(dpre=null), dict(dx=null)):
        assert gated_grad(**bad) == pb.PB_EINVAL, bad
    for bad in (dict(pre=odd), dict(dh=odd), dict(dpre=odd), dict(dx=odd)):
        assert gated_grad(**bad) == pb.PB_EALIGN, bad

    def ad(count=2, rank=3, type=1, A=0x1000, B=0x1000, scale=0x1000):
        return pb.pb_adapters(count, rank, type, 0, A, B, scale)

    def adapted(a, n=1, index=fake, y=fake, x=fake, d=d, m=4):
        return L.pb_matmul_adapters(fake, fake, ref(d), m, x, n, ref(a), index, null, y, fake, null)

    def adapted_grad(a, n=1, index=fake, x=fake, dy=fake, dx=fake, da=fake, db=fake, d=d, m=4):
        return L.pb_matmul_adapters_grad(fake, fake, ref(d), m, x, dy, n, ref(a), index, dx, da, db, fake, null)
    for f in (adapted, adapted_grad):
        for bad in (dict(count=0), dict(rank=0), dict(type=3), dict(type=-1), dict(A=None), dict(B=None)):
            assert f(ad(**bad)) == pb.PB_EINVAL, (f, bad)
        for bad in (dict(A=0x1008), dict(B=0x1008), dict(scale=0x1004)):
            assert f(ad(**bad)) == pb.PB_EALIGN, (f, bad)
        for bad in (dict(count=pb.PB_MAX_ADAPTERS + 1), dict(rank=pb.PB_MAX_RANK + 1)):
            assert f(ad(**bad)) == pb.PB_ESIZE, (f, bad)
        for bad in (dict(n=0), dict(x=null), dict(m=0), dict(m=5)):
            assert f(ad(), **bad) == pb.PB_EINVAL, (f, bad)
        assert f(ad(), index=odd) == pb.PB_EALIGN and f(ad(), n=pb.PB_MAX_BATCH + 1) == pb.PB_ESIZE
    assert adapted(ad(), y=null) == pb.PB_EINVAL and adapted(ad(), y=odd) == pb.PB_EALIGN
    assert adapted_grad(ad(), dy=null) == pb.PB_EINVAL and adapted_grad(ad(), dx=null, da=null, db=null) == pb.PB_EINVAL
    assert adapted_grad(ad(), d=rows) == pb.PB_EINVAL and adapted_grad(ad(), da=odd) == pb.PB_EALIGN
    assert L.pb_matmul_adapters(fake, fake, ref(d), 4, fake, 1, None, fake, null, fake, fake, null) == pb.PB_EINVAL


def test_a_reserved_field_that_is_set_is_refused(pb):
    d, fake, null = pb.pb_desc_init(64, 96, 4), ctypes.c_void_p(0x1000), ctypes.c_void_p(0)
    a = pb.pb_adapters(2, 3, pb.PB_TYPE_F32, 1, 0x1000, 0x1000, None)
    L, ref = pb.lib(), ctypes.byref
    assert L.pb_matmul_adapters(fake, fake, ref(d), 4, fake, 1, ref(a), null, null, fake, fake, null) == pb.PB_EINVAL
    assert L.pb_matmul_adapters_grad(fake, fake, ref(d), 4, fake, fake, 1, ref(a), null, fake, fake, fake, fake, null) == pb.PB_EINVAL


def test_workspace_sizes(pb):
    d, rows = pb.pb_desc_init(4096, 1000, 8), pb.pb_desc_init_layout(64, 96, 4, pb.PB_LAYOUT_ROWMAJOR_V1)
    assert pb.pb_grad_workspace_bytes(rows, 1) == 0 and pb.pb_grad_workspace_bytes(d, 0) == 0
    assert pb.pb_grad_workspace_bytes(d, pb.PB_MAX_BATCH + 1) == 0
    assert pb.pb_grad_workspace_bytes(d, 16) >= 16 * 4096 * 4          # four digits of every gradient
    a = pb.pb_adapters(3, 20, pb.PB_TYPE_F32, 0, None, None, None)
    assert pb.pb_adapters_workspace_bytes(d, a, 16) > max(pb.pb_grad_workspace_bytes(d, 16), pb.pb_workspace_bytes(d, 16))
    assert pb.pb_adapters_workspace_bytes(rows, a, 2) > pb.pb_workspace_bytes(rows, 2)
    a.rank = pb.PB_MAX_RANK + 1
    assert pb.pb_adapters_workspace_bytes(d, a, 16) == 0


def test_holders_refuse_what_does_not_fit(pb):
    z = torch.zeros
    with pytest.raises(TypeError, match="must both be"):
        pb.Adapters(z(2, 3, 8), z(2, 5, 3, dtype=torch.bfloat16))
    with pytest.raises(TypeError, match="must both be"):
        pb.Adapters(z(2, 3, 8, dtype=torch.float64), z(2, 5, 3, dtype=torch.float64))
    with pytest.raises(ValueError, match="rank"):
        pb.Adapters(z(2, 3, 8), z(2, 5, 4))
    with pytest.raises(ValueError, match="scale"):
        pb.Adapters(z(2, 3, 8), z(2, 5, 3), z(3))
    with pytest.raises(TypeError, match="A must be a CUDA/HIP tensor"):
        pb.Adapters(z(2, 3, 8), z(2, 5, 3))


def gate_of(gate, v):
    """The activation and its slope in 64 bits."""
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(over="ignore"):
        if gate == 3:
            return np.maximum(v, 0), (v > 0).astype(np.float64)
        if gate == 2:
            t = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
            th = np.tanh(t)
            return 0.5 * v * (1 + th), 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
        s = 1 / (1 + np.exp(-v))
        return (s, s * (1 - s)) if gate == 0 else (v * s, s + v * s * (1 - s))


@pytest.mark.parametrize("gate", [0, 1, 2, 3])
def test_slopes_of_the_references_against_differences(gate):
    v = np.array([-9.0, -3.0, -0.7, -1e-3, 1e-3, 0.4, 2.0, 8.0])
    h = 1e-5
    difference = (gate_of(gate, v + h)[0] - gate_of(gate, v - h)[0]) / (2 * h)
    # h^2 / 6 times the third derivative (below 3), and the rounding of the values (below 10 * 2^-53 / h)
    assert np.abs(difference - gate_of(gate, v)[1]).max() < 3 * h * h + 10 * 2.0 ** -53 / h


# ---- on the GPU ----
class Layer:
    """A packed layer and its matrix in 64 bits."""

    def __init__(self, pb, rows, cols, bits, layout=None, seed=1, scales=None):
        g = np.random.default_rng(seed)
        W = (g.standard_normal((rows, cols)) * 0.05).astype(np.float32)
        prep = po.prepare(W, bits)
        self.lin = pb.PackedLinear(torch.from_numpy(W).cuda(), bits, max_batch=1, layout=layout)
        self.layers, self.scales = prep["layers"], prep["scales"]
        if scales is not None:
            self.scales = scales
            self.lin.scales[:bits] = torch.from_numpy(scales).cuda()
        self.rows, self.cols, self.bits = rows, cols, bits

    def matrix(self, m):
        return sum(float(self.scales[i]) * self.layers[i].reshape(self.rows, self.cols).astype(np.float64) for i in range(m))


def fixed(X):
    return np.clip(np.trunc(X.astype(np.float64) * 65536.0), -2.0 ** 31, 2.0 ** 31 - 1) / 65536.0


def close(got, want, tol, what):
    got = got.detach().cpu().numpy().astype(np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want)
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d of %d wrong, first at %s: got %s want %s tolerance %s" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(tol, bad.shape)[bad][:3])


def grad_tolerance(dY, W, parts):
    """dY rounded to 2^-30 of its vector's largest value at most (four digits), or to half a unit of three digits, the largest value being 2^22 to
    2^23 units, 0.998 * 2^22 where the scaling is one less; `parts` sums rounded to fp32 and added one after the other."""
    half_a_unit = 2.0 ** -30 if len(dY) <= 32 else 2.0 ** -23 / 0.998
    return half_a_unit * np.abs(dY).max(axis=1, keepdims=True) * np.abs(W).sum(axis=0) + 2 * parts * U * (np.abs(dY) @ np.abs(W))


LAYOUTS = {"bits": 0x50420002, "gates": 0x50420003, "pairs": 0x50420004, "rows": 0x50420001}

GRADS = [  # rows, cols, bits, used, batch, layout
    (1, 1, 1, 1, 1, "bits"), (1, 1, 8, 8, 3, "pairs"), (17, 33, 2, 1, 1, "bits"), (64, 512, 8, 8, 16, "bits"), (63, 511, 4, 4, 15, "pairs"),
    (65, 513, 5, 3, 17, "bits"), (300, 700, 8, 8, 5, "bits"), (300, 700, 8, 7, 33, "pairs"), (1000, 1030, 6, 6, 32, "bits"),
    (2050, 260, 8, 5, 1, "bits"), (2050, 260, 3, 2, 64, "pairs"), (200, 2000, 8, 8, 65, "bits"), (513, 1537, 8, 8, 130, "pairs"),
    (260, 515, 11, 11, 20, "bits"), (260, 515, 16, 16, 70, "bits"), (260, 515, 16, 15, 9, "pairs"), (260, 515, 13, 9, 40, "pairs"),
    (20, 300, 4, 4, 7, "gates"), (1004, 333, 8, 8, 70, "gates"), (36, 100, 8, 6, 33, "gates"), (4096, 64, 8, 8, 2, "bits"),
    (129, 129, 2, 2, 257, "bits"), (96, 8200, 4, 3, 3, "bits"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,bits,m,batch,layout", GRADS)
def test_gradient_through_the_packed_matrix(pb, rows, cols, bits, m, batch, layout):
    layer = Layer(pb, rows, cols, bits, LAYOUTS[layout])
    g = np.random.default_rng(2)
    # vectors of very different sizes, values of different sizes in a vector
    dY = (g.standard_normal((batch, rows)) * 10.0 ** g.uniform(-30, 8, (batch, 1)) * 10.0 ** g.uniform(-4, 0, (batch, rows))).astype(np.float32)
    if batch > 2:
        dY[1] = 0
    dX = layer.lin.grad(torch.from_numpy(dY).cuda(), m)
    W = layer.matrix(m)
    d64 = dY.astype(np.float64)
    # at most 16 parts of the sum over up to 64 steps of rows, and three groups of bitlayers
    close(dX, d64 @ W, grad_tolerance(d64, W, 16 * 3) + 1e-44, "dX")


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,batches", [(520, 32768, (2, 7)), (40000, 40, (3, 7, 12, 20))])
def test_gradient_of_few_vectors_and_many_rows_or_columns(pb, rows, cols, batches):
    """Parts of the sum of more than eight steps of 64 rows; digits that do not fit a workgroup."""
    layer = Layer(pb, rows, cols, 1)
    W = layer.matrix(1)
    for batch in batches:
        dY = (np.random.default_rng(13).standard_normal((batch, rows)) * 10.0 ** np.arange(batch)[:, None]).astype(np.float32)
        dX = layer.lin.grad(torch.from_numpy(dY).cuda())
        d64 = dY.astype(np.float64)
        # at most 64 parts
        close(dX, d64 @ W, grad_tolerance(d64, W, 64), "dX")


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 20, 70])
@pytest.mark.parametrize("bits,m", [(3, 3), (6, 6)])
@pytest.mark.parametrize("layout", ["bits", "pairs"])
def test_gradient_with_scales_that_do_not_halve(pb, batch, bits, m, layout):
    scales = np.array([-1.5, 0.7, 0.01, 3.0, -0.2, 1.0, 0.3, 0.11][:bits], dtype=np.float32)
    layer = Layer(pb, 330, 600, bits, LAYOUTS[layout], scales=scales)
    dY = np.random.default_rng(3).standard_normal((batch, 330))
    dX = layer.lin.grad(torch.from_numpy(dY.astype(np.float32)).cuda(), m)
    d64, W = dY.astype(np.float32).astype(np.float64), layer.matrix(m)
    # every bitlayer by itself: the terms are those of the bitlayers
    terms = sum(abs(float(scales[i])) * layer.layers[i].reshape(330, 600) for i in range(m))
    close(dX, d64 @ W, grad_tolerance(d64, terms, 16 * m), "dX")


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [4, 40, 100])
def test_gradient_of_vectors_that_are_not_finite_or_tiny(pb, batch):
    layer = Layer(pb, 200, 300, 8)
    dY = np.random.default_rng(4).standard_normal((batch, 200)).astype(np.float32)
    dY[1, 7], dY[2, 199] = np.nan, -np.inf
    dY[3] *= 1e-42                                    # subnormal
    dY[0] *= np.float32(2.0 ** 120)
    got = layer.lin.grad(torch.from_numpy(dY).cuda()).cpu()
    assert torch.isnan(got[1:3]).all() and torch.isfinite(got[3:]).all() and torch.isfinite(got[0]).all()
    keep = [i for i in range(batch) if i not in (1, 2)]
    d64, W = dY[keep].astype(np.float64), layer.matrix(8)
    # (subnormal results: steps of 2^-149)
    close(got[keep], d64 @ W, grad_tolerance(d64, W, 16) + 16 * 2.0 ** -149, "dX")


GATED = [  # units, cols, bits, used, batch, layout
    (2, 40, 4, 4, 1, "gates"), (10, 77, 8, 5, 3, "gates"), (300, 515, 8, 8, 1, "gates"), (300, 515, 8, 8, 40, "gates"),
    (129, 515, 8, 8, 1, "bits"), (129, 1025, 5, 4, 17, "bits"), (64, 300, 8, 8, 5, "pairs"), (64, 300, 4, 3, 1, "pairs"),
    (33, 100, 3, 3, 2, "rows"), (1000, 64, 2, 2, 130, "gates"), (500, 2000, 8, 8, 9, "gates"), (150, 700, 12, 11, 6, "gates"),
    (150, 700, 12, 12, 1, "gates"), (700, 300, 8, 8, 700, "gates"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("units,cols,bits,m,batch,layout", GATED)
def test_gated_block(pb, units, cols, bits, m, batch, layout):
    layer = Layer(pb, 2 * units, cols, bits, LAYOUTS[layout])
    g = np.random.default_rng(5)
    X = g.standard_normal((batch, cols)).astype(np.float32)
    bias = g.standard_normal(2 * units).astype(np.float32)
    W = layer.matrix(m)
    for gate in range(4):
        for b in (None, bias):
            H, pre = layer.lin.gated(torch.from_numpy(X).cuda(), gate, m, bias=None if b is None else torch.from_numpy(b).cuda(), keep=True)
            want = fixed(X) @ W.T + (0 if b is None else b.astype(np.float64))
            # one rounding of the product, one of the sum with the bias, and the fp64 rounding of its terms
            size = np.abs(fixed(X) @ W.T) + np.abs(want)
            close(pre, want, U * size + 1e-12 * (np.abs(fixed(X)) @ np.abs(W.T)), "pre")
            # the gate on the pre-activations that the call used: a few roundings, and that of the argument of exp (|t| U, t of GELU is up to
            # four roundings off), which counts with the slope of the logistic function
            p = pre.cpu().numpy().astype(np.float64)
            v, u = p[:, :units], p[:, units:]
            a, da = gate_of(gate, v)
            close(H, a * u, 16 * U * np.abs(a * u) + 8 * U * np.abs(v * (1 + v * v)) * np.abs(da) * np.abs(u) + 8 * U * np.abs(v * a * u) +
                  4 * 2.0 ** -53 * np.abs(v * u) + 1e-40, "H")       # (the last: 1 + tanh of the reference)
            alone = layer.lin.gated(torch.from_numpy(X).cuda(), gate, m, bias=None if b is None else torch.from_numpy(b).cuda())
            assert torch.equal(alone, H)


LARGE = [  # rows, cols, bits, used, batch, layout, scales that do not halve: at least 192 workgroups of 128 rows and 128 vectors
    (3100, 515, 8, 8, 1000, "gates", False), (3096, 1100, 5, 4, 1001, "gates", False), (6200, 64, 2, 1, 500, "gates", False),
    (3100, 520, 12, 11, 1000, "gates", False), (3100, 300, 6, 6, 950, "gates", True), (3100, 515, 8, 8, 1000, "bits", False),
    (3090, 1100, 8, 7, 1021, "pairs", False), (6200, 33, 4, 4, 520, "pairs", False), (3100, 520, 16, 16, 1000, "pairs", False),
    (3100, 300, 3, 3, 990, "bits", True), (24600, 40, 8, 8, 65, "bits", False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,bits,m,batch,layout,odd_scales", LARGE)
def test_large_batches(pb, rows, cols, bits, m, batch, layout, odd_scales):
    """Values of three digits, and in some groups of sixteen vectors of four; a gated block, or a layer with adapters."""
    scales = np.array([-1.5, 0.7, 0.01, 3.0, -0.2, 1.0][:bits], dtype=np.float32) * 0.1 if odd_scales else None
    layer = Layer(pb, rows, cols, bits, LAYOUTS[layout], scales=scales)
    g = np.random.default_rng(12)
    X = g.standard_normal((batch, cols)).astype(np.float32)
    X[[3, batch // 2, batch - 1]] *= 300
    X[5, cols - 1], X[40, 0] = 1e9, -1e9                    # beyond the range of the fixed point
    bias = g.standard_normal(rows).astype(np.float32)
    W, Xd, bd = layer.matrix(m), torch.from_numpy(X).cuda(), torch.from_numpy(bias).cuda()
    product = fixed(X) @ W.T
    terms = sum(abs(float(layer.scales[i])) * layer.layers[i].reshape(rows, cols) for i in range(m)) if odd_scales else np.abs(W)
    # one rounding per group of bitlayers (at most three, or each bitlayer by itself) and its sum, one of the sum with the bias
    groups = m if odd_scales else 1 + (m > 8) + (m > 14)
    tol = U * (np.abs(product + bias) + 2 * groups * (np.abs(fixed(X)) @ terms.T if groups > 1 else np.abs(product))) + 1e-12 * (np.abs(fixed(X)) @ terms.T)
    if layout == "gates":
        units = rows // 2
        H, pre = layer.lin.gated(Xd, 1, m, bias=bd, keep=True)
        close(pre, product + bias, tol, "pre")
        p = pre.cpu().numpy().astype(np.float64)
        a, da = gate_of(1, p[:, :units])
        # (exp overflows at 2^128: a logistic function below 2^-128 is 0, as a factor of v u)
        tol = 16 * U * np.abs(a * p[:, units:]) + 8 * U * np.abs(p[:, :units] * da * p[:, units:]) + 2.0 ** -127 * np.abs(p[:, :units] * p[:, units:])
        close(H, a * p[:, units:], tol + 1e-40, "H")
        assert torch.equal(layer.lin.gated(Xd, 1, m, bias=bd), H)
    else:
        zero = pb.Adapters(torch.zeros((1, 1, cols), device="cuda"), torch.zeros((1, rows, 1), device="cuda"))
        Y = layer.lin.adapted(Xd, zero, torch.full((batch,), -1, dtype=torch.int32, device="cuda"), m, bias=bd)
        close(Y, product + bias, tol, "Y")


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [0, 1, 2, 3])
def test_gates_far_out(pb, gate):
    """Pre-activations up to the largest fp32 value: finite, and the limits of the gate."""
    layer = Layer(pb, 4, 32, 2)
    pre = torch.tensor([[-3e38, 3e38, 1.0, 1.0], [-1e20, 1e20, 1.0, -1.0], [-120.0, 120.0, 2.0, 2.0], [0.0, -0.0, 1.0, 1.0]], device="cuda")
    dX, dpre = layer.lin.gated_grad(pre, torch.ones((4, 2), device="cuda"), gate)
    assert torch.isfinite(dpre).all()
    a, da = gate_of(gate, pre.cpu().numpy()[:, :2].clip(-500, 500))
    a = np.where(np.abs(pre.cpu().numpy()[:, :2]) > 500, np.where(pre.cpu().numpy()[:, :2] > 0, pre.cpu().numpy()[:, :2] if gate else 1.0, 0.0), a)
    u = pre.cpu().numpy()[:, 2:]
    close(dpre, np.concatenate([u * da, a], axis=1), 1e-5 * np.concatenate([np.abs(u * da), np.abs(a)], axis=1) + 1e-30, "dpre")


@pytest.mark.gpu
@pytest.mark.parametrize("units,cols,bits,m,batch,layout", [c for c in GATED if c[5] != "rows"])
def test_gated_block_backward(pb, units, cols, bits, m, batch, layout):
    layer = Layer(pb, 2 * units, cols, bits, LAYOUTS[layout])
    g = np.random.default_rng(6)
    pre = (g.standard_normal((batch, 2 * units)) * 2).astype(np.float32)
    dH = (g.standard_normal((batch, units)) * 1e-3).astype(np.float32)
    W = layer.matrix(m)
    for gate in range(4):
        dX, dpre = layer.lin.gated_grad(torch.from_numpy(pre).cuda(), torch.from_numpy(dH).cuda(), gate, m)
        p, d = pre.astype(np.float64), dH.astype(np.float64)
        v, u = p[:, :units], p[:, units:]
        a, da = gate_of(gate, v)
        want = np.concatenate([d * u * da, d * a], axis=1)
        # the slope is a sum of parts up to s and |v| s (1 - s) (1 + 3 v^2 ...) in size, each a few roundings off, and those of exp's argument
        parts = 1 + np.abs(v) * (1 + v * v)
        close(dpre, want, 32 * U * np.concatenate([np.abs(d * u) * parts, np.abs(d) * parts], axis=1), "dpre")
        d64 = dpre.cpu().numpy().astype(np.float64)
        close(dX, d64 @ W, grad_tolerance(d64, W, 16 * 3), "dX")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["bits", "gates"])
def test_gated_block_against_differences(pb, layout):
    """<dX, e> against (L(x + h e) - L(x - h e)) / 2 h with L = sum dH H, the activations on a grid of 2^-24."""
    units, cols, batch, h = 40, 120, 6, 2.0 ** -6
    g = np.random.default_rng(7)
    W = torch.from_numpy((g.standard_normal((2 * units, cols)) * 0.1).astype(np.float32)).cuda()
    lin = pb.PackedLinear(W, 8, frac_bits=24, layout=LAYOUTS[layout])
    X, e = (torch.from_numpy(np.round(g.standard_normal((batch, cols)) * 2.0 ** 12).astype(np.float32) / 2.0 ** 12).cuda() for _ in range(2))
    dH = torch.from_numpy(g.standard_normal((batch, units)).astype(np.float32)).cuda()
    for gate in range(3):
        H, pre = lin.gated(X, gate, keep=True)
        dX, _ = lin.gated_grad(pre, dH, gate)
        plus, minus = (lin.gated(X + s * h * e, gate).double() for s in (1, -1))
        difference = ((plus - minus) * dH.double()).sum(dim=1) / (2 * h)
        along = (dX.double() * e.double()).sum(dim=1)
        # third derivatives of act(g) u along e (their size: |W e|^3 of about one) times h^2 / 6, summed over the units like |dH|
        tolerance = h * h * dH.double().abs().sum(dim=1) * 4
        assert ((difference - along).abs() <= tolerance).all(), (gate, difference, along, tolerance)
        assert (along.abs() > 4 * tolerance).any()


TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ADAPTED = [  # rows, cols, bits, used, batch, layout, count, rank, type, index
    (1, 1, 1, 1, 1, "bits", 1, 1, "f32", "mixed"), (64, 64, 8, 8, 1, "bits", 4, 8, "bf16", "mixed"), (100, 130, 4, 4, 5, "bits", 3, 7, "f16", "mixed"),
    (101, 131, 4, 3, 40, "pairs", 5, 16, "bf16", "mixed"), (300, 515, 8, 8, 64, "bits", 64, 17, "f32", "mixed"), (300, 516, 8, 8, 65, "bits", 2, 32, "f16", "mixed"),
    (257, 700, 8, 8, 129, "bits", 1, 64, "bf16", "none"), (257, 700, 8, 8, 33, "bits", 3, 65, "f32", "none"), (64, 300, 8, 8, 16, "bits", 2, 256, "bf16", "same"),
    (64, 300, 8, 8, 17, "bits", 2, 200, "f16", "mixed"), (1030, 64, 8, 8, 3, "bits", 300, 5, "f32", "mixed"), (64, 1030, 8, 8, 2, "bits", 4096, 3, "bf16", "mixed"),
    (40, 60, 2, 2, 4096, "bits", 7, 4, "f32", "mixed"), (40, 60, 2, 2, 1000, "bits", 1000, 4, "bf16", "mixed"), (60, 40, 8, 8, 50, "gates", 3, 12, "f16", "mixed"),
    (200, 90, 8, 8, 48, "bits", 5, 16, "bf16", "outside"), (33, 70, 3, 3, 4, "rows", 2, 4, "f32", "mixed"), (200, 2100, 8, 8, 100, "bits", 3, 20, "bf16", "mixed"),
    # sums in eight and in sixteen parts; several turns over the ranks; one adapter with all vectors beside many with none
    (200, 5000, 2, 2, 70, "bits", 2, 33, "bf16", "mixed"), (5000, 64, 2, 2, 20, "bits", 3, 50, "f32", "mixed"), (130, 300, 4, 4, 30, "bits", 2, 90, "f16", "mixed"),
    (70, 700, 8, 8, 200, "bits", 100, 24, "f16", "same"), (64, 300, 8, 8, 50, "bits", 40, 70, "bf16", "same"), (515, 320, 4, 4, 200, "bits", 1, 36, "bf16", "none"),
    # one vector
    (333, 700, 8, 8, 1, "bits", 5, 16, "f16", "same"), (60, 5000, 4, 4, 1, "bits", 3, 13, "f32", "none"), (600, 2100, 8, 3, 1, "gates", 2, 15, "bf16", "same"),
    (333, 700, 8, 8, 1, "bits", 5, 17, "bf16", "same"), (40, 9000, 2, 2, 1, "bits", 2, 4, "bf16", "outside"), (70, 300, 8, 8, 1, "pairs", 2, 16, "f16", "same"),
]


class AdapterCase:
    def __init__(self, pb, rows, cols, bits, m, batch, layout, count, rank, type, index):
        self.layer = Layer(pb, rows, cols, bits, LAYOUTS[layout])
        g = np.random.default_rng(8)
        rand = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32))   # noqa: E731
        dtype = TYPES[type]
        self.A, self.B, self.scale = (rand(count, rank, cols) * 0.3).to(dtype), (rand(count, rows, rank) * 0.3).to(dtype), rand(count).abs() + 0.5
        self.X, self.dY = rand(batch, cols), rand(batch, rows) * 1e-3
        if index == "none":
            self.index = None
            self.of = np.zeros(batch, dtype=np.int64)
        else:
            i = {"mixed": lambda: g.integers(-1, count, batch), "same": lambda: np.full(batch, count - 1),
                 "outside": lambda: g.choice([-1, -2 ** 31, count, 2 ** 31 - 1], batch)}[index]().astype(np.int32)
            self.index = torch.from_numpy(i)
            self.of = np.where((i >= 0) & (i < count), i, -1)
        self.adapters = pb.Adapters(self.A.cuda(), self.B.cuda(), self.scale.cuda())
        self.m, self.W = m, self.layer.matrix(m)

    def of_adapter(self, k):
        """A, B, scale, vectors, x, dy in 64 bits"""
        n = np.flatnonzero(self.of == k)
        return (self.A[k].double().numpy(), self.B[k].double().numpy(), float(self.scale[k]), n, self.X[n].double().numpy(), self.dY[n].double().numpy())

    def gpu(self, t):
        return None if t is None else t.cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("case", ADAPTED, ids=str)
def test_adapters_beside_the_packed_matrix(pb, case):
    c = AdapterCase(pb, *case)
    x64 = c.X.double().numpy()
    bias = torch.from_numpy(np.random.default_rng(9).standard_normal(case[0]).astype(np.float32))
    want = fixed(x64) @ c.W.T + bias.double().numpy()
    # a sum of K fp32 products is K U of its terms off at most, in any order; the product, the bias and the last sum one rounding each
    tol = 1e-12 * (np.abs(fixed(x64)) @ np.abs(c.W.T)) + 3 * U * (np.abs(fixed(x64) @ c.W.T) + np.abs(bias.double().numpy()))
    cols, rank = case[1], case[7]
    for k in set(c.of) - {-1}:
        A, B, s, n, x, _ = c.of_adapter(k)
        u, size = x @ A.T, np.abs(x) @ np.abs(A.T)
        want[n] += s * (u @ B.T)
        tol[n] += s * ((cols + rank + 8) * U * (size @ np.abs(B.T))) + 3 * U * np.abs(want[n])
    Y = c.layer.lin.adapted(c.X.cuda(), c.adapters, c.gpu(c.index), c.m, bias=bias.cuda())
    close(Y, want, tol + 1e-40, "Y")
    assert torch.equal(Y, c.layer.lin.adapted(c.X.cuda(), c.adapters, c.gpu(c.index), c.m, bias=bias.cuda()))
    without = c.layer.lin.adapted(c.X.cuda(), c.adapters, torch.full((case[4],), -1, dtype=torch.int32, device="cuda"), c.m)
    work = pb.alloc_workspace(c.layer.lin.desc, case[4])
    plain = torch.empty_like(without)
    pb.pb_matmul(c.layer.lin.packed, c.layer.lin.scales, c.layer.lin.desc, c.m, c.X.cuda(), case[4], plain, work)
    assert torch.equal(without, plain)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c in ADAPTED if c[5] != "rows"], ids=str)
def test_adapters_backward(pb, case):
    c = AdapterCase(pb, *case)
    rows, cols, batch, rank = case[0], case[1], case[4], case[7]
    d64 = c.dY.double().numpy()
    dX, tX = d64 @ c.W, grad_tolerance(d64, c.W, 16 * 3)
    dA, dB = np.zeros(c.A.shape), np.zeros(c.B.shape)
    tA, tB = np.zeros(c.A.shape), np.zeros(c.B.shape)
    for k in set(c.of) - {-1}:
        A, B, s, n, x, dy = c.of_adapter(k)
        t, t_size = s * (dy @ B), s * (np.abs(dy) @ np.abs(B))
        u, u_size = x @ A.T, np.abs(x) @ np.abs(A.T)
        dX[n] += t @ A
        dA[k], dB[k] = t.T @ x, s * (dy.T @ u)
        # sums of fp32 products, as in the forward pass
        tX[n] += (rows + rank + 8) * U * (t_size @ np.abs(A)) + 2 * U * np.abs(dX[n])
        tA[k] = (rows + len(n) + 8) * U * (t_size.T @ np.abs(x))
        tB[k] = (cols + len(n) + 8) * U * s * (np.abs(dy).T @ u_size)
    got = c.layer.lin.adapted_grad(c.X.cuda(), c.dY.cuda(), c.adapters, c.gpu(c.index), c.m)
    for g, want, tol, what in zip(got, (dX, dA, dB), (tX, tA, tB), ("dX", "dA", "dB")):
        close(g, want, tol + 1e-40, what)
    again = c.layer.lin.adapted_grad(c.X.cuda(), c.dY.cuda(), c.adapters, c.gpu(c.index), c.m, inputs=False)
    assert again[0] is None and torch.equal(again[1], got[1]) and torch.equal(again[2], got[2])


@pytest.mark.gpu
def test_a_vector_that_is_not_finite_stays_by_itself(pb):
    c = AdapterCase(pb, 100, 200, 8, 8, 40, "bits", 3, 5, "f32", "mixed")
    index = c.index.clone()
    index[7], index[8] = 1, -1
    X, dY = c.X.clone(), c.dY.clone()
    clean = c.layer.lin.adapted(X.cuda(), c.adapters, index.cuda())
    grads = c.layer.lin.adapted_grad(X.cuda(), dY.cuda(), c.adapters, index.cuda())
    X[7, 3], X[8, 5], dY[7, 2], dY[8, 1] = math.inf, math.nan, math.nan, math.inf
    got = c.layer.lin.adapted(X.cuda(), c.adapters, index.cuda())
    others = [n for n in range(40) if n not in (7, 8)]
    assert torch.equal(got[others], clean[others]) and not torch.isfinite(got[7]).any()
    dirty = c.layer.lin.adapted_grad(X.cuda(), dY.cuda(), c.adapters, index.cuda())
    assert torch.equal(dirty[0][others], grads[0][others]) and torch.isnan(dirty[0][[7, 8]]).all()
    for a, b in ((dirty[1], grads[1]), (dirty[2], grads[2])):      # the other adapters, vector 8 has none
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and not torch.isfinite(a[1]).all()


class Block:
    """A block as it is trained: a gated layer, and a projection back with adapters, all matrices packed."""

    def __init__(self, pb, cols=200, units=300, batch=24):
        g = np.random.default_rng(11)
        rand = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda()   # noqa: E731
        self.up = pb.PackedLinear(rand(2 * units, cols) * 0.05, 8, layout=pb.PB_LAYOUT_TILE16_GATES_V1)
        self.down = pb.PackedLinear(rand(cols, units) * 0.05, 8)
        self.adapters = pb.Adapters((rand(3, 8, units) * 0.1).bfloat16(), (rand(3, cols, 8) * 0.1).bfloat16(), torch.tensor([2.0, 1.0, 0.5]).cuda())
        self.index = torch.from_numpy(g.integers(-1, 3, batch).astype(np.int32)).cuda()
        self.X, self.dY = rand(batch, cols), rand(batch, cols) * 1e-2

    def step(self):
        H, pre = self.up.gated(self.X, 1, keep=True)
        Y = self.down.adapted(H, self.adapters, self.index)
        dH, dA, dB = self.down.adapted_grad(H, self.dY, self.adapters, self.index)
        dX, dpre = self.up.gated_grad(pre, dH, 1)
        return Y, dA, dB, dX, dpre


@pytest.mark.gpu
def test_a_block_forward_and_backward(pb):
    b = Block(pb)
    Y, dA, dB, dX, dpre = (t.double().cpu().numpy() for t in b.step())
    up = b.up.unpack().double().cpu().numpy() * float(b.up.scales[7])
    down = b.down.unpack().double().cpu().numpy() * float(b.down.scales[7])
    A, B, s = (t.double().cpu().numpy() for t in (b.adapters.A, b.adapters.B, b.adapters.scale))
    index, x, dy = b.index.cpu().numpy(), b.X.double().cpu().numpy(), b.dY.double().cpu().numpy()
    pre = fixed(x) @ up.T
    a, da = gate_of(1, pre[:, :300])
    H = a * pre[:, 300:]
    want, dH, wA, wB = fixed(H) @ down.T, dy @ down, np.zeros_like(A), np.zeros_like(B)
    for n, k in enumerate(index):
        if k >= 0:
            want[n] += s[k] * (B[k] @ (A[k] @ H[n]))
            t = s[k] * (B[k].T @ dy[n])
            dH[n] += A[k].T @ t
            wA[k] += np.outer(t, H[n])
            wB[k] += s[k] * np.outer(dy[n], A[k] @ H[n])
    wpre = np.concatenate([dH * pre[:, 300:] * da, dH * a], axis=1)
    # H may cross a border of its fixed point (2^-16) where it is rounded, 300 of them with weights of about 0.05: 0.05 * 2^-16 * 300 at most
    np.testing.assert_allclose(Y, want, atol=0.2 * 2.0 ** -16 * 300, rtol=0)
    # the others: chains of sums of up to 600 fp32 products, 600 U of terms of about 25 times the result's size
    for got, ref in ((dA, wA), (dB, wB), (dpre, wpre), (dX, wpre @ up)):
        assert np.abs(got - ref).max() <= 25 * 600 * U * np.abs(ref).max()


@pytest.mark.gpu
def test_a_captured_step_replays(pb):
    """A training step in a graph, replayed between eager work, with its inputs changed: the eager results every time."""
    b = Block(pb, batch=70)
    other = Block(pb, cols=120, units=90, batch=5)
    b.step()
    want_other = other.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step()
    torch.cuda.current_stream().wait_stream(side)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = b.step()
    with torch.cuda.graph(second):
        captured_other = other.step()
    for i in range(4):
        b.X.mul_(1.0 + 0.25 * i)
        b.index.copy_(torch.roll(b.index, i))
        eager = b.step()
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):                  # (graphs at the same time: their workspaces are their own)
            second.replay()
        torch.cuda.synchronize()
        for g, e in zip(captured, eager):
            assert torch.equal(g, e)
        for g, e in zip(captured_other, want_other):
            assert torch.equal(g, e)


@pytest.mark.gpu
def test_streams_and_shapes(pb):
    b = Block(pb)
    want = b.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = b.step()
    side.synchronize()
    for g, e in zip(on_side, want):
        assert torch.equal(g, e)
    X = b.X.reshape(4, 6, 200)
    assert torch.equal(b.up.gated(X), b.up.gated(b.X)) and torch.equal(b.up.gated(b.X[3]), b.up.gated(b.X[3:4]))
    with pytest.raises(ValueError, match="X must have vectors of 200"):
        b.up.gated(b.X[:, :100])
    with pytest.raises(ValueError, match="X must be contiguous"):
        b.up.gated(b.X.t().contiguous().t())
    with pytest.raises(ValueError, match="index must have the shape"):
        b.down.adapted(want[0].new_zeros(24, 300), b.adapters, b.index[:5])
    with pytest.raises(TypeError, match="index must have dtype"):
        b.down.adapted(want[0].new_zeros(24, 300), b.adapters, b.index.long())
    with pytest.raises(ValueError, match="adapters of a layer"):
        b.up.adapted(b.X, b.adapters, b.index)
    with pytest.raises(pb.PbError):
        b.up.gated(b.X, 7)
    with pytest.raises(pb.PbError):
        b.up.grad(want[4], 9)
    with pytest.raises(pb.PbError):
        b.up.grad(want[4], 0)
    with pytest.raises(ValueError, match="dH must have the shape"):
        b.up.gated_grad(want[4], want[4].new_zeros(3, 300))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_outputs_and_nothing_else_are_written(pb):
    """Rows behind the last vector of every output, and the inputs, stay as they are."""
    c = AdapterCase(pb, 90, 150, 8, 8, 21, "bits", 3, 6, "bf16", "mixed")
    lin, d, n = c.layer.lin, c.layer.lin.desc, 21
    X, dY, index = c.X.cuda(), c.dY.cuda(), c.index.cuda()
    desc = c.adapters.desc()
    guard = lambda *s: torch.full(s, 7.0, device="cuda")   # noqa: E731
    work = lambda size: torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")   # noqa: E731

    def check(ws, size, *outs):
        torch.cuda.synchronize()
        assert (ws[size:] == 0xA5).all()
        for out, rows in outs:
            assert (out[rows:] == 7.0).all() and not (out[:rows] == 7.0).all()
    Y, dX, dA, dB = guard(n + 2, 90), guard(n + 2, 150), guard(4, 6, 150), guard(4, 90, 6)
    size = pb.pb_adapters_workspace_bytes(d, desc, n)
    ws = work(size)
    pb.pb_matmul_adapters(lin.packed, lin.scales, d, 8, X, n, desc, index, None, Y, ws)
    check(ws, size, (Y, n))
    pb.pb_matmul_adapters_grad(lin.packed, lin.scales, d, 8, X, dY, n, desc, index, dX, dA, dB, ws)
    check(ws, size, (dX, n), (dA, 3), (dB, 3))
    size = pb.pb_grad_workspace_bytes(d, n)
    ws, dX = work(size), guard(n + 2, 150)
    pb.pb_matmul_grad(lin.packed, lin.scales, d, 8, dY, n, dX, ws)
    check(ws, size, (dX, n))
    H, pre, dpre, dX = guard(n + 2, 45), guard(n + 2, 90), guard(n + 2, 90), guard(n + 2, 150)
    size = pb.pb_workspace_bytes(d, n)
    ws = work(size)
    pb.pb_gated_linear(lin.packed, lin.scales, d, 8, X, n, None, 1, H, pre, ws)
    check(ws, size, (H, n), (pre, n))
    size = pb.pb_grad_workspace_bytes(d, n)
    ws = work(size)
    pb.pb_gated_linear_grad(lin.packed, lin.scales, d, 8, pre, H, n, 1, dpre, dX, ws)
    check(ws, size, (dpre, n), (dX, n))
    assert torch.equal(X.cpu(), c.X) and torch.equal(dY.cpu(), c.dY) and torch.equal(index.cpu(), c.index)


@pytest.mark.gpu
def test_native_and_python_operators_agree(pb):
    """The native forms of PackedLinear's operators against the Python functions behind them, unusual arguments to both, and stand-ins for the tensors."""
    if not isinstance(pb.pb_matmul, type(len)):
        pytest.skip("no native binding")
    b = Block(pb)
    bias, none = torch.randn(600, device="cuda"), torch.full((24,), -1, dtype=torch.int32, device="cuda")
    H, pre = b.up.gated(b.X, keep=True)
    calls = [
        ("gated", b.up, (b.X, 1, None, None, False)), ("gated", b.up, (b.X, 2, 5, bias, True)), ("gated", b.up, (b.X[5], 0, 8, None, True)),
        ("gated_grad", b.up, (pre, H, 1, None)), ("gated_grad", b.up, (pre.reshape(4, 6, 600), H, 3, 4)),
        ("grad", b.down, (b.dY, None)), ("grad", b.down, (b.dY[2], 3)),
        ("adapted", b.down, (H, b.adapters, b.index, None, None)), ("adapted", b.down, (H, b.adapters, None, 6, bias[:200].clone())),
        ("adapted", b.down, (H, pb.Adapters(b.adapters.A.float(), b.adapters.B.float()), none, None, None)),
        ("adapted_grad", b.down, (H, b.dY, b.adapters, b.index, None, True)), ("adapted_grad", b.down, (H, b.dY, b.adapters, None, 7, False)),
    ]
    for name, layer, args in calls:
        native, python = pb._methods[name](layer, *args), pb._PYTHON[name](layer, *args)
        native, python = ([t] if isinstance(t, torch.Tensor) else list(t) for t in (native, python))
        assert len(native) == len(python)
        for x, y in zip(native, python):
            assert (x is None and y is None) or torch.equal(x, y), name
    for name, layer, args, error in (
            ("gated", b.up, (b.X.double(), 1, None, None, False), TypeError), ("gated", b.up, (b.X.cpu(), 1, None, None, False), ValueError),
            ("gated", b.up, (b.X, 1, None, bias[:5], False), ValueError), ("gated", b.up, (b.X, 1, 9, None, False), pb.PbError),
            ("grad", b.down, (b.dY[:0], None), pb.PbError), ("adapted", b.down, (H, b.adapters, b.index.cpu(), None, None), ValueError),
            ("adapted_grad", b.down, (H, b.dY[:3], b.adapters, b.index, None, True), ValueError)):
        for f in (pb._methods[name], pb._PYTHON[name]):
            with pytest.raises(error):
                f(layer, *args)
    # the tensors that an optimizer puts in the place of others are the ones that count
    want = b.down.adapted(H, b.adapters, b.index)
    A = b.adapters.A
    b.adapters.A = torch.zeros_like(A)
    plain = b.down.adapted(H, b.adapters, none)
    assert torch.equal(b.down.adapted(H, b.adapters, b.index), plain) and not torch.equal(plain, want)
    b.adapters.A = A
    assert torch.equal(b.down.adapted(H, b.adapters, b.index), want)
    b.adapters.A = A[:, :, :10].contiguous()
    with pytest.raises(ValueError, match="another type or shape"):
        b.down.adapted(H, b.adapters, b.index)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 70])
def test_nothing_else_is_written_for_one_vector_and_for_many(pb, n):
    c = AdapterCase(pb, 90, 150, 8, 8, n, "bits", 3, 6, "f16", "same")
    lin, d, desc = c.layer.lin, c.layer.lin.desc, c.adapters.desc()
    X, dY, index = c.X.cuda(), c.dY.cuda(), c.index.cuda()
    Y, dX, dA, dB = (torch.full(s, 7.0, device="cuda") for s in ((n + 2, 90), (n + 2, 150), (4, 6, 150), (4, 90, 6)))
    size, grad_size = pb.pb_adapters_workspace_bytes(d, desc, n), pb.pb_grad_workspace_bytes(d, n)
    ws, grad_ws = (torch.full((s + 256,), 0xA5, dtype=torch.uint8, device="cuda") for s in (size, grad_size))
    pb.pb_matmul_adapters(lin.packed, lin.scales, d, 8, X, n, desc, index, None, Y, ws)
    pb.pb_matmul_adapters_grad(lin.packed, lin.scales, d, 8, X, dY, n, desc, index, dX, dA, dB, ws)
    torch.cuda.synchronize()
    assert (ws[size:] == 0xA5).all()
    for out, rows in ((Y, n), (dX, n), (dA, 3), (dB, 3)):
        assert (out[rows:] == 7.0).all() and not (out[:rows] == 7.0).all()
    dX.fill_(7.0)
    pb.pb_matmul_grad(lin.packed, lin.scales, d, 8, dY, n, dX, grad_ws)
    torch.cuda.synchronize()
    assert (grad_ws[grad_size:] == 0xA5).all() and (dX[n:] == 7.0).all() and not (dX[:n] == 7.0).all()


@pytest.mark.gpu
def test_adapters_beyond_32_bits(pb):
    """2.5e9 values of A, the last adapter used."""
    count, rank, rows, cols = 300, 256, 40, 32768
    layer = Layer(pb, rows, cols, 1)
    g = torch.Generator().manual_seed(3)
    a, b = (torch.randn(s, generator=g) * 0.1 for s in ((rank, cols), (rows, rank)))
    A, B = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((count, rank, cols), (count, rows, rank)))
    A[-1], B[-1] = a.cuda(), b.cuda()
    X, dY = torch.randn((3, cols), generator=g), torch.randn((3, rows), generator=g)
    index = torch.tensor([count - 1, -1, count - 1], dtype=torch.int32, device="cuda")
    adapters = pb.Adapters(A, B)
    Y = layer.lin.adapted(X.cuda(), adapters, index)
    dX, dA, dB = layer.lin.adapted_grad(X.cuda(), dY.cuda(), adapters, index)
    x, dy, a, b, W = X.double().numpy(), dY.double().numpy(), A[-1].double().cpu().numpy(), B[-1].double().cpu().numpy(), layer.matrix(1)
    on = np.array([[1.0], [0.0], [1.0]])
    u, t = x @ a.T * on, dy @ b * on
    # sums of K fp32 products: K U of their terms off at most, twice in a row
    off_u, off_t = (cols + 8) * U * (np.abs(x) @ np.abs(a).T), (rows + 8) * U * (np.abs(dy) @ np.abs(b))
    want = fixed(X.numpy()) @ W.T + u @ b.T
    close(Y, want, 4 * U * (np.abs(fixed(X.numpy())) @ np.abs(W).T + np.abs(want)) + off_u @ np.abs(b).T + (rank + 8) * U * (np.abs(u) @ np.abs(b).T), "Y")
    close(dX, dy @ W + t @ a, grad_tolerance(dy, W, 16) + off_t @ np.abs(a) + (rank + 8) * U * (np.abs(t) @ np.abs(a) + np.abs(dy @ W)), "dX")
    close(dA[-1], t.T @ x, off_t.T @ np.abs(x) + 8 * U * (np.abs(t).T @ np.abs(x)), "dA")
    close(dB[-1], dy.T @ u, np.abs(dy).T @ off_u + 8 * U * (np.abs(dy).T @ np.abs(u)), "dB")
    assert not dA[:-1].any() and not dB[:-1].any()


@pytest.mark.gpu
def test_batches_beyond_32_bits(pb):
    """4096 vectors of 530000 rows: 2.2e9 values of dY, Y and the pre-activations."""
    rows, cols, n, some = 530000, 32, 4096, [0, 1, 4095]
    torch.manual_seed(5)
    for layout in ("bits", "gates"):
        layer = Layer(pb, rows, cols, 1, LAYOUTS[layout])
        W = layer.matrix(1)
        dY, X = torch.randn((n, rows), device="cuda"), torch.randn((n, cols), device="cuda")
        x = fixed(X[some].cpu().numpy())
        d64 = dY[some].double().cpu().numpy()
        # (three digits: half a unit is 2^-23 of the largest value)
        tolerance = 2.0 ** -23 / 0.998 * np.abs(d64).max(axis=1, keepdims=True) * np.abs(W).sum(axis=0) + 2 * 64 * U * (np.abs(d64) @ np.abs(W))
        close(layer.lin.grad(dY)[some], d64 @ W, tolerance, "dX")
        y = x @ W.T
        if layout == "bits":
            adapters = pb.Adapters(torch.zeros((2, 3, cols), device="cuda"), torch.randn((2, rows, 3), device="cuda"))
            Y = layer.lin.adapted(X, adapters, torch.ones(n, dtype=torch.int32, device="cuda"))
            close(Y[some], y, 4 * U * np.abs(y) + 1e-30, "Y")
            dX, dA, dB = layer.lin.adapted_grad(X, dY, adapters, None)
            close(dX[some], d64 @ W, tolerance, "dX")
            assert dA[0].any() and not dA[1].any() and not dB.any()
            del Y, dX, dA, dB, adapters
        H, pre = layer.lin.gated(X, pb.PB_GATE_RELU, keep=True)
        close(pre[some], y, 4 * U * np.abs(y) + 1e-30, "pre")
        want = np.maximum(y[:, :rows // 2], 0) * y[:, rows // 2:]
        close(H[some], want, 16 * U * np.abs(want) + 1e-30, "H")
        del dY
        dX, dpre = layer.lin.gated_grad(pre, torch.ones_like(H), pb.PB_GATE_RELU)
        p = pre[some].double().cpu().numpy()
        want = np.concatenate([p[:, rows // 2:] * (p[:, :rows // 2] > 0), np.maximum(p[:, :rows // 2], 0)], axis=1)
        close(dpre[some], want, 4 * U * np.abs(want), "dpre")
        tolerance = 2.0 ** -23 / 0.998 * np.abs(want).max(axis=1, keepdims=True) * np.abs(W).sum(axis=0) + 2 * 64 * U * (np.abs(want) @ np.abs(W))
        close(dX[some], want @ W, tolerance, "dX")
        del H, pre, dX, dpre
        torch.cuda.empty_cache()


class Everything:
    """Every operator on the same layers, n vectors."""

    def __init__(self, pb, n):
        self.ffn, self.lin = Layer(pb, 360, 520, 8, LAYOUTS["gates"]).lin, Layer(pb, 333, 520, 8).lin
        torch.manual_seed(n)
        self.X, self.dY, self.dH = (torch.randn((n, k), device="cuda") for k in (520, 333, 180))
        self.adapters = pb.Adapters(*(torch.randn(s, device="cuda").half() for s in ((3, 11, 520), (3, 333, 11))))
        self.index = torch.randint(-1, 3, (n,), device="cuda", dtype=torch.int32)

    def __call__(self):
        H, pre = self.ffn.gated(self.X, keep=True)
        return [H, pre, *self.ffn.gated_grad(pre, self.dH), self.lin.grad(self.dY), self.lin.adapted(self.X, self.adapters, self.index),
                *self.lin.adapted_grad(self.X, self.dY, self.adapters, self.index)]


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5, 40, 300])
def test_captured_operators_follow_their_inputs(pb, n):
    every = Everything(pb, n)
    every()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = every()
    for i in range(4):
        for t in (every.X, every.dY, every.dH):
            t.mul_(-0.75).add_(0.01 * i)
        every.index.copy_(torch.roll(every.index, 1) if n > 1 else every.index * 0 + i - 1)
        eager = every()
        graph.replay()
        torch.cuda.synchronize()
        for g, e in zip(captured, eager):
            assert torch.equal(g, e)


@pytest.mark.gpu
def test_threads_share_layers(pb):
    """Four threads on streams of their own with the same layers and adapters."""
    import threading
    sets = [Everything(pb, n) for n in (1, 7, 40, 300)]
    for s in sets[1:]:
        s.ffn, s.lin, s.adapters = sets[0].ffn, sets[0].lin, sets[0].adapters
    want = [s() for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(s, w):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    got = s()
                    stream.synchronize()
                    if not all(torch.equal(g, e) for g, e in zip(got, w)):
                        wrong.append(len(s.X))
        except Exception as error:
            wrong.append(error)
    threads = [threading.Thread(target=work, args=a) for a in zip(sets, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong


@pytest.mark.gpu
@pytest.mark.parametrize("n", [20, 90])
def test_adapters_backward_one_gradient_at_a_time(pb, n):
    c = AdapterCase(pb, 190, 350, 8, 8, n, "bits", 3, 20, "bf16", "mixed")
    lin, d, desc = c.layer.lin, c.layer.lin.desc, c.adapters.desc()
    X, dY, index = c.X.cuda(), c.dY.cuda(), c.index.cuda()
    ws = torch.empty(pb.pb_adapters_workspace_bytes(d, desc, n), dtype=torch.uint8, device="cuda")
    want = lin.adapted_grad(X, dY, c.adapters, index)
    shapes = ((n, 350), (3, 20, 350), (3, 190, 20))
    for asked in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True), (True, True, False)):
        outs = [torch.full(s, 7.0, device="cuda") if a else None for s, a in zip(shapes, asked)]
        pb.pb_matmul_adapters_grad(lin.packed, lin.scales, d, 8, X, dY, n, desc, index, *outs, ws)
        torch.cuda.synchronize()
        for which, (got, w) in enumerate(zip(outs, want)):
            if got is None:
                continue
            # (the waves may share the vectors of an adapter in another way: sums of up to n products in another order, their values bounded by
            # sums of the terms' sizes, which are at most n times the largest ones')
            if which == 0:
                assert torch.equal(got, w)
            else:
                k = 1 if which == 1 else 2
                u = (X.double() if k == 1 else dY.double()).abs().max() * n * 2.0 ** -24 * (n + 16)
                factor = (c.dY.abs().double().sum(1).max() * c.B.abs().max().double() * c.scale.max().double()) if k == 1 else \
                    (c.X.abs().double().sum(1).max() * c.A.abs().max().double() * c.scale.max().double())
                assert (got.double() - w.double()).abs().max() <= u * factor
