"""Every compiled form of the operators' kernels: the host's choice of kernels depends on sizes, types and layouts in many ways, so the cases below and
those of test_operators.py are run on the launch recorder, which says what they reach, and on the GPU, where they are compared with the definitions."""
import json
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import test_operators as ops                                    # noqa: E402
from tests.test_launches import probe                                      # noqa: E402,F401  (a fixture)
from tests.test_operators import AdapterCase, Layer, LAYOUTS, close, pb    # noqa: E402,F401

U = 2.0 ** -24

# rows, cols, bits, used, batch, layout
GRADS = [
    # digits in memory, one, four and eight waves along the vectors; four and eight slots; several groups of bitlayers
    (4700, 4703, 3, 3, 17, "bits"), (4716, 4614, 4, 3, 17, "pairs"), (2872, 8315, 8, 8, 17, "bits"), (8493, 2574, 8, 8, 19, "pairs"),
    (410, 8301, 4, 4, 56, "bits"), (409, 8531, 2, 2, 52, "pairs"), (392, 8456, 8, 8, 58, "bits"), (387, 8935, 6, 6, 61, "pairs"), (400, 8400, 12, 11, 50, "bits"),
    (396, 8300, 8, 7, 49, "gates"),
    (402, 86, 4, 3, 1076, "bits"), (389, 67, 4, 3, 1450, "pairs"), (388, 92, 5, 5, 1050, "bits"), (402, 63, 8, 7, 1477, "pairs"), (401, 90, 16, 16, 1101, "bits"),
    (404, 90, 8, 8, 1100, "gates"),
    # scalings in a launch of their own
    (4276, 33, 2, 2, 346, "bits"), (4100, 70, 8, 8, 500, "pairs"), (4096, 500, 8, 8, 130, "bits"), (2100, 2300, 8, 8, 300, "bits"), (2304, 515, 8, 8, 1000, "gates"),
    (4096, 4096, 8, 8, 48, "bits"), (4096, 4096, 6, 6, 77, "pairs"),
]

# units, cols, bits, used, batch, activation bits; gate layout
GATED = [
    (10, 1758, 5, 4, 16, 8), (1268, 34, 1, 1, 424, 8), (10, 32, 4, 4, 3, 8), (1146, 36, 4, 4, 18, 8), (10, 1768, 5, 5, 17, 8), (2394, 33, 8, 7, 239, 8),
    (10, 37, 9, 9, 2, 8), (4008, 34, 7, 6, 21, 8), (10, 4404, 4, 3, 7, 16), (1028, 37, 4, 3, 285, 16), (10, 33, 4, 3, 2, 16), (3158, 33, 2, 1, 10, 16),
    (8, 4336, 5, 5, 7, 16), (998, 34, 9, 9, 279, 16), (10, 34, 8, 7, 2, 16), (3220, 75, 6, 6, 10, 16), (10, 8905, 2, 2, 5, 32), (3192, 35, 1, 1, 89, 32),
    (8, 35, 3, 3, 4, 32), (60, 33, 5, 4, 1081, 32), (10, 8965, 9, 8, 4, 32), (2240, 33, 6, 5, 100, 32), (12, 33, 6, 6, 2, 32), (372, 37, 6, 5, 178, 32),
    # k_gated_tile
    (470, 554, 4, 3, 1409, 8), (666, 107, 9, 9, 765, 8), (1398, 615, 5, 4, 225, 16), (428, 47, 9, 9, 524, 16), (814, 519, 4, 3, 270, 32), (216, 563, 9, 9, 331, 32),
    (1366, 1024, 8, 8, 24, 32), (1366, 1024, 8, 5, 33, 32), (5462, 2048, 8, 5, 24, 32), (5462, 2048, 4, 4, 17, 32),
    # tiles whose pre-activations go through memory, k_batch
    (5462, 2048, 8, 8, 48, 32), (5462, 1024, 8, 8, 64, 32), (2730, 700, 8, 8, 60, 16), (3658, 37, 4, 4, 314, 32), (2768, 36, 6, 6, 432, 32),
    # one vector: the ways of k_mfma
    (10, 36, 2, 1, 1, 8), (10, 34, 3, 2, 1, 16), (8, 34, 4, 4, 1, 32), (12, 8361, 1, 1, 1, 32), (12, 8787, 3, 2, 1, 32), (8, 8691, 7, 7, 1, 8),
    (12, 17001, 1, 1, 1, 32), (12, 17001, 2, 2, 1, 32), (14, 16500, 5, 5, 1, 16), (10, 30001, 1, 1, 1, 32), (10, 30001, 2, 2, 1, 32), (6, 32768, 8, 8, 1, 32),
    (40, 16384, 1, 1, 1, 32), (40, 16384, 4, 4, 1, 32),
]

TYPES = ("f32", "bf16", "f16")
RANKS = (9, 25, 40, 57)          # one to four rank tiles at once
# rows, cols, bits, used, batch, layout, count, rank, type, index
ADAPTED = [
    case for type in TYPES for rank in RANKS for case in (
        (300, 50, 4, 4, 3, "bits", 2, rank, type, "mixed"),               # u and t beside the join of the gradient's parts
        (2500, 36, 4, 4, 620, "bits", 3, rank, type, "mixed"),            # ... beside the scalings
        (48, 8900, 2, 2, 5, "pairs", 2, rank, type, "mixed"),             # u beside the activations' digits
        (36, 40, 5, 4, 40, "bits", 1, rank, type, "same"),                # waves that share an adapter's vectors
        (50, 44, 8, 8, 7, "pairs", 2, rank, type, "mixed"),               # ... that do not
    )
] + [
    # one vector behind k_mfma
    (24, 36, 2, 1, 1, "gates", 1, 1, "f32", "same"), (27, 34, 3, 2, 1, "bits", 3, 2, "f16", "same"), (16, 60, 4, 4, 1, "gates", 1, 7, "bf16", "same"),
    (20, 8221, 2, 1, 1, "gates", 2, 4, "f16", "same"), (28, 8739, 2, 2, 1, "bits", 10, 5, "f32", "same"), (18, 8988, 5, 5, 1, "bits", 1, 9, "bf16", "none"),
    (24, 17001, 1, 1, 1, "bits", 2, 16, "bf16", "same"), (25, 17001, 2, 2, 1, "bits", 2, 3, "f32", "same"), (26, 30001, 1, 1, 1, "bits", 2, 16, "f16", "same"),
    (20, 30001, 2, 2, 1, "gates", 2, 13, "bf16", "same"), (17, 32768, 8, 8, 1, "bits", 2, 8, "f32", "same"), (80, 16384, 1, 1, 1, "bits", 2, 8, "f32", "same"),
    (80, 16384, 4, 4, 1, "bits", 2, 8, "bf16", "same"),
]


def test_the_gpu_tests_reach_every_compiled_form(probe):          # noqa: F811
    of = {"f32": 0, "bf16": 1, "f16": 2}
    grads = [(*c[:5], LAYOUTS[c[5]]) for c in ops.GRADS + GRADS] + [(520, 32768, 1, 1, 7, LAYOUTS["bits"]), (40000, 40, 1, 1, 20, LAYOUTS["bits"])]
    gated = [(*c[:5], 32, LAYOUTS[c[5]]) for c in ops.GATED] + [(c[0] // 2, *c[1:5], 32, LAYOUTS[c[5]]) for c in ops.LARGE if c[5] == "gates"] + \
        [(*c, LAYOUTS["gates"]) for c in GATED]
    adapted = [(*c[:5], LAYOUTS[c[5]], c[6], c[7], of[c[8]], c[9] != "none") for c in ops.ADAPTED + ADAPTED] + \
        [(*c[:5], LAYOUTS[c[5]], 1, 1, 0, True) for c in ops.LARGE if c[5] != "gates"]
    reached, compiled = probe("""
        class Adapters(ctypes.Structure):
            _fields_ = [(n, ctypes.c_int32) for n in ("count", "rank", "type", "reserved")] + [(n, ctypes.c_void_p) for n in ("A", "B", "scale")]
        grads, gated, adapted = json.loads(sys.argv[3])
        reached, ref = set(), ctypes.byref
        def run(status):
            assert status == 0
            reached.update(k for k, _ in launches())
        for R, C, bits, m, N, layout in grads:
            run(L.pb_matmul_grad(F, F, ref(desc(R, C, bits, layout)), m, F, N, F, WORK, None))
        for units, C, bits, m, N, act, layout in gated:
            d = desc(2 * units, C, bits, layout, act)
            run(L.pb_gated_linear(F, F, ref(d), m, F, N, None, 1, F, F, WORK, None))
            run(L.pb_gated_linear(F, F, ref(d), m, F, N, None, 1, F, None, WORK, None))
            if layout != ROWS:
                run(L.pb_gated_linear_grad(F, F, ref(d), m, F, F, N, 1, F, F, WORK, None))
        for R, C, bits, m, N, layout, count, rank, type, indexed in adapted:
            d, a, index = desc(R, C, bits, layout), Adapters(count, rank, type, 0, 0x1000, 0x1000, None), F if indexed else None
            run(L.pb_matmul_adapters(F, F, ref(d), m, F, N, ref(a), index, None, F, WORK, None))
            if layout != ROWS:
                for asked in ((F, F, F), (None, F, F), (F, None, None)):
                    run(L.pb_matmul_adapters_grad(F, F, ref(d), m, F, F, N, ref(a), index, *asked, WORK, None))
        compiled = [mock.mock_kernel(i).decode() for i in range(mock.mock_kernels())]
        print(json.dumps([sorted(reached), [k for k in compiled if any(x in k for x in ("k_grad", "k_gated", "k_adapter", "k_batch", "k_mfma"))]]))
    """, json.dumps([grads, gated, adapted]))
    mine = [k for k in compiled if "k_mfma" not in k or re.search(r"k_mfmaILi\dELi\d+ELi\dELi[12]E", k)]      # (the plain product has tests of its own)
    assert len(mine) > 170
    assert not sorted(set(mine) - set(reached))


def spread(g, batch, rows):
    """Gradients: groups of sixteen vectors of normal values, and groups with a vector that has one large value beside small ones."""
    dY = torch.randn((batch, rows), generator=g)
    single = torch.randn((batch, rows), generator=g) * 1e-6
    single[torch.arange(batch), torch.randint(0, rows, (batch,), generator=g)] = 1.0
    n = torch.arange(batch)
    dY = torch.where(((n // 16 % 3 == 1) & (n % 16 == 7))[:, None], single, dY)
    return (dY * 10.0 ** torch.randint(-6, 7, (batch, 1), generator=g)).cuda()


def digits_of(dY, batch):
    """Half a unit of the integers of every vector: four digits, or three in a group of sixteen (of more than 32 vectors) without a large value."""
    largest = dY.abs().amax(dim=1)
    rows = dY.shape[1]
    wide = largest ** 2 * rows > (rows / 16 if rows < 2304 else 144 * max(1.0, rows / 4096)) * (dY ** 2).sum(dim=1)
    wide = torch.repeat_interleave(torch.stack([g.any() for g in wide.split(16)]), 16)[:len(dY)]
    return (torch.where(wide | (batch <= 32), 2.0 ** -30, 2.0 ** -23 / 0.995) * largest)[:, None]


def matrix(layer, m):
    """The matrix, and the sizes of its terms: eight bitlayers, then six at a time are summed exactly and rounded by themselves (a small negative code is a
    difference of two such terms)."""
    weights = [float(layer.scales[i]) * layer.layers[i].reshape(layer.rows, layer.cols).astype(np.float64) for i in range(m)]
    groups = [sum(weights[:8])] + [sum(weights[i:i + 6]) for i in range(8, m, 6)]
    return torch.from_numpy(layer.matrix(m)).cuda(), torch.from_numpy(sum(np.abs(g) for g in groups)).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,bits,m,batch,layout", GRADS)
def test_gradients(pb, rows, cols, bits, m, batch, layout):           # noqa: F811
    layer = Layer(pb, rows, cols, bits, LAYOUTS[layout])
    dY, (W, terms) = spread(torch.Generator().manual_seed(21), batch, rows), matrix(layer, m)
    d64 = dY.double()
    # parts of the sum of two steps of 64 rows or more, and up to three groups of bitlayers: each rounded, and added one after the other
    parts = ((rows + 127) // 128) * (1 + (m > 8) + (m > 14))
    tol = digits_of(d64, batch) * terms.sum(dim=0) + 2 * parts * U * (d64.abs() @ terms)
    got = layer.lin.grad(dY, m)
    assert ((got.double() - d64 @ W).abs() <= tol).all()
    assert torch.equal(layer.lin.grad(dY, m), got)


def gate_of(gate, v):
    """The activation and its slope in 64 bits, on the device."""
    if gate == 3:
        return v.clamp(min=0), (v > 0).double()
    if gate == 2:
        k = (8 / np.pi) ** 0.5
        s = torch.sigmoid(k * (v + 0.044715 * v ** 3))
        return v * s, s + v * s * (1 - s) * k * (1 + 3 * 0.044715 * v * v)
    s = torch.sigmoid(v)
    return (s, s * (1 - s)) if gate == 0 else (v * s, s + v * s * (1 - s))


@pytest.mark.gpu
@pytest.mark.parametrize("units,cols,bits,m,batch,act_bits", GATED)
def test_gated_blocks(pb, units, cols, bits, m, batch, act_bits):     # noqa: F811
    g = torch.Generator().manual_seed(22)
    rand = lambda *s: torch.randn(s, generator=g).cuda()              # noqa: E731
    # (the range of eight bits is +-4, that of sixteen +-8)
    lin = pb.PackedLinear(rand(2 * units, cols) * (0.5 / cols ** 0.5), bits, max_batch=batch, layout=pb.PB_LAYOUT_TILE16_GATES_V1, act_bits=act_bits,
                          frac_bits={8: 5, 16: 12, 32: 16}[act_bits])
    X, bias = rand(batch, cols), rand(2 * units)
    if batch > 20:
        X[17] *= 300                                                  # (four digits in some groups of sixteen vectors)
    for gate, b in ((1, bias), (2, None), (0, None), (3, bias)):
        product = torch.empty((batch, 2 * units), device="cuda")
        pb.pb_matmul_bias_act(lin.packed, lin.scales, lin.desc, m, X, batch, b, pb.PB_ACT_NONE, product, lin.workspace)
        H, pre = lin.gated(X, gate, m, bias=b, keep=True)
        assert torch.equal(pre, product)
        v, u = product.double()[:, :units], product.double()[:, units:]
        a, da = gate_of(gate, v)
        # a few roundings, and those of exp's argument (|t| U, four of t with GELU), which count with the slope of the logistic function; exp overflows
        # at 2^128
        tol = 16 * U * (a * u).abs() + 8 * U * (v * (1 + v * v) * da * u).abs() + 8 * U * (v * a * u).abs() + 2.0 ** -127 * (v * u).abs() + 1e-40
        assert ((H.double() - a * u).abs() <= tol).all()
        assert torch.equal(lin.gated(X, gate, m, bias=b), H)


@pytest.mark.gpu
@pytest.mark.parametrize("units,cols,bits,m,batch,act_bits", [c for c in GATED if c[5] == 32])
def test_gated_blocks_backward(pb, units, cols, bits, m, batch, act_bits):       # noqa: F811
    layer = Layer(pb, 2 * units, cols, bits, LAYOUTS["gates"])
    g = torch.Generator().manual_seed(23)
    pre, dH, (W, terms) = torch.randn((batch, 2 * units), generator=g).cuda() * 2, spread(g, batch, units), matrix(layer, m)
    parts = ((2 * units + 127) // 128) * (1 + (m > 8) + (m > 14))
    for gate in (1, 2):
        dX, dpre = layer.lin.gated_grad(pre, dH, gate, m)
        v, u, d = pre.double()[:, :units], pre.double()[:, units:], dH.double()
        a, da = gate_of(gate, v)
        # the slope: a sum of parts up to s and |v| s (1 - s) (1 + 3 v^2 ...) in size, each a few roundings off, and those of exp's argument
        size = 1 + v.abs() * (1 + v * v)
        close(dpre, torch.cat([d * u * da, d * a], dim=1).cpu().numpy(), (32 * U * torch.cat([(d * u).abs() * size, d.abs() * size], dim=1)).cpu().numpy(), "dpre")
        d64 = dpre.double()
        tol = digits_of(d64, batch) * terms.sum(dim=0) + 2 * parts * U * (d64.abs() @ terms)
        assert ((dX.double() - d64 @ W).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case", ADAPTED, ids=str)
def test_adapters(pb, case):            # noqa: F811
    ops.test_adapters_beside_the_packed_matrix(pb, case)


@pytest.mark.gpu
@pytest.mark.parametrize("case", ADAPTED, ids=str)
def test_adapters_backward(pb, case):   # noqa: F811
    ops.test_adapters_backward(pb, case)
    # dX alone
    c = AdapterCase(pb, *case)
    lin, d, a, n = c.layer.lin, c.layer.lin.desc, c.adapters.desc(), case[4]
    X, dY, index = c.X.cuda(), c.dY.cuda(), c.gpu(c.index)
    dX = torch.empty_like(X)
    pb.pb_matmul_adapters_grad(lin.packed, lin.scales, d, c.m, X, dY, n, a, index, dX, None, None, torch.empty(pb.pb_adapters_workspace_bytes(d, a, n),
                                                                                                           dtype=torch.uint8, device="cuda"))
    assert torch.equal(dX, lin.adapted_grad(X, dY, c.adapters, index, c.m)[0])
