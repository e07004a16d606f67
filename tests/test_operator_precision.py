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


def spread(seed, batch, rows):
    """Gradients: in groups of sixteen vectors, in turn, normal values, products of three normal values, one large value beside small ones in one vector of
    the group, and all of these."""
    g = torch.Generator().manual_seed(seed)
    dY = torch.randn((batch, rows), generator=g)
    heavy = dY * torch.randn((batch, rows), generator=g) * torch.randn((batch, rows), generator=g)
    single = torch.randn((batch, rows), generator=g) * 1e-6
    single[torch.arange(batch), torch.randint(0, rows, (batch,), generator=g)] = 1.0
    n = torch.arange(batch)
    kind = (n // 16) % 4
    dY = torch.where(((kind == 1) | (kind == 3) & (n % 3 == 0))[:, None], heavy, dY)
    dY = torch.where((((kind == 2) & (n % 16 == 5)) | (kind == 3) & (n % 3 == 1))[:, None], single, dY)
    return (dY * 10.0 ** torch.randint(-6, 7, (batch, 1), generator=g)).cuda()


def digits_are_enough(dX, dY, of_column, weight):
    """dX[n, c] = weight dY[n, of_column[c]] to within half a unit of dY's integers and the rounding of the result."""
    d64 = dY.double()
    batch, rows = dY.shape
    largest = d64.abs().amax(dim=1)
    ratio = largest ** 2 * rows / (d64 ** 2).sum(dim=1)
    limit = rows / 16 if rows < 2304 else 144 * max(1.0, rows / 4096)
    assert ((ratio / limit - 1).abs() > 1e-9).all()            # (else the side that a vector is on hangs on the rounding of the sums)
    wide = torch.repeat_interleave(torch.stack([(group > limit).any() for group in ratio.split(16)]), 16)[:batch]
    assert wide.any() and not wide.all()
    half = torch.where(wide, torch.tensor(2.0 ** -30, dtype=torch.float64, device="cuda"),
                       torch.tensor(2.0 ** -23 / 0.995, dtype=torch.float64, device="cuda")) * largest
    want = d64[:, of_column] * weight
    assert ((dX.double() - want).abs() <= half[:, None] * weight + 2.0 ** -24 * want.abs()).all()


# rows = columns (one weight in each), bits, batch, layout: digits and scalings in a launch of their own, in one, in the kernel of the product
DIGITS = [(600, 8, 2000, BITS), (600, 3, 1999, PAIRS), (1100, 8, 1100, BITS), (2300, 8, 300, BITS), (2300, 4, 330, PAIRS), (2560, 4, 520, BITS), (4500, 8, 90, BITS),
          (4096, 8, 60, BITS), (4096, 3, 50, PAIRS), (300, 8, 100, BITS)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,bits,batch,layout", DIGITS)
def test_gradients_have_the_digits_that_their_values_need(pb, rows, bits, batch, layout):
    """One weight per row and column: every value of dY comes out by itself."""
    perm = torch.randperm(rows, generator=torch.Generator().manual_seed(4)).cuda()
    W = torch.zeros((rows, rows), device="cuda")
    W[perm, torch.arange(rows, device="cuda")] = 1.0
    lin = pb.PackedLinear(W, bits, layout=layout)
    weight = float(lin.scales[bits - 1]) * int(lin.unpack().max())
    dY = spread(5, batch, rows)
    digits_are_enough(lin.grad(dY), dY, perm, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("units,bits,batch,layout", [(300, 8, 2000, GATES), (551, 8, 1000, BITS), (1200, 4, 300, GATES), (2048, 8, 60, PAIRS)])
def test_gradients_of_gated_blocks_have_the_digits_that_their_values_need(pb, units, bits, batch, layout):
    rows = 2 * units
    perm = torch.randperm(rows, generator=torch.Generator().manual_seed(4)).cuda()
    W = torch.zeros((rows, rows), device="cuda")
    W[perm, torch.arange(rows, device="cuda")] = 1.0
    lin = pb.PackedLinear(W, bits, layout=layout)
    weight = float(lin.scales[bits - 1]) * int(lin.unpack().max())
    # in every other group of sixteen vectors the values are all of the same size (ReLU passes them on)
    pre, dH = rand(6, batch, rows), spread(7, batch, units)
    even = torch.arange(batch, device="cuda") // 16 % 2 == 0
    pre[even] = 1.0
    dH[even] = 1.0 + 0.1 * rand(8, int(even.sum()), units).clamp(-3, 3)
    dX, dpre = lin.gated_grad(pre, dH, pb.PB_GATE_RELU)
    digits_are_enough(dX, dpre, perm, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 5, 40])
@pytest.mark.parametrize("rank", [5, 16, 21])
def test_a_scale_that_is_infinite_gives_infinities_and_stays_by_itself(pb, batch, rank):
    """scale B (A x) with an infinite scale: of the sign of B A x, whatever the rank is padded to."""
    lin = pb.PackedLinear(rand(1, 70, 90) * 0.1, 8, max_batch=batch)
    A, B, X = rand(2, 2, rank, 90).abs(), rand(3, 2, 70, 1).expand(2, 70, rank).contiguous(), rand(4, batch, 90).abs()
    index = torch.arange(batch, device="cuda", dtype=torch.int32) % 2
    Y = lin.adapted(X, pb.Adapters(A, B, torch.tensor([float("inf"), 1.0], device="cuda")), index)
    sign = B[0, :, 0].sign()                                    # (all ranks of a row have its sign, u is positive)
    assert torch.equal(Y[::2], (sign * float("inf")).expand(Y[::2].shape))
    clean = lin.adapted(X, pb.Adapters(A, B, torch.ones(2, device="cuda")), index)
    assert torch.equal(Y[1::2], clean[1::2])


@pytest.mark.gpu
@pytest.mark.parametrize("act_bits", [8, 16])
@pytest.mark.parametrize("batch", [1, 7, 100])
@pytest.mark.parametrize("layout", [BITS, PAIRS, GATES])
def test_adapters_beside_narrow_activations(pb, batch, act_bits, layout):
    lin = pb.PackedLinear(rand(1, 200, 700) * 0.05, 8, max_batch=batch, layout=layout, act_bits=act_bits, frac_bits=5 if act_bits == 8 else 12)
    X, A, B = rand(2, batch, 700), rand(3, 3, 11, 700) * 0.1, rand(4, 3, 200, 11) * 0.1
    index = torch.arange(batch, device="cuda", dtype=torch.int32) % 4          # (3: none)
    Y = lin.adapted(X, pb.Adapters(A, B), index)
    plain = torch.empty_like(Y)
    pb.pb_matmul(lin.packed, lin.scales, lin.desc, 8, X, batch, plain, lin.workspace)
    want, terms = plain.double(), plain.double().abs()
    for n in range(batch):
        if n % 4 < 3:
            want[n] += B[n % 4].double() @ (A[n % 4].double() @ X[n].double())
            # a sum of K fp32 products is K U of its terms off at most; one rounding of the sum
            terms[n] += (700 + 11 + 8) * (B[n % 4].abs().double() @ (A[n % 4].abs().double() @ X[n].abs().double())) + 2 * want[n].abs()
    assert ((Y.double() - want).abs() <= 2.0 ** -24 * terms).all()
    assert torch.equal(Y[3::4], plain[3::4])
