"""Block-scaled FP8 on the GPU: the quantizer bit for bit, the products exactly where sums are exact and within the instruction's error elsewhere."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import block128_reference as ref  # noqa: E402

ELEMS = ["e4m3", "e5m2"]


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2603_08713_amd as mx_

    mx_.load_library()
    return mx_


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---- quantizer ----------------------------------------------------------------------------------------------------
def same_quantized(mx, x, elem, block_rows, groups=1):
    rows, K = x.shape
    codes, scales = mx.mx_quantize_block128(x, elem, block_rows, groups)
    each = rows // groups
    for e in range(groups):
        want_codes, want_scales = ref.quantize(x[e * each:(e + 1) * each], block_rows, elem)
        n = want_scales.shape[0]
        assert torch.equal(codes[e * each:(e + 1) * each].cpu(), want_codes)
        got = scales[e * n:(e + 1) * n].cpu()
        assert torch.equal(got.view(torch.int32)[~got.isnan()], want_scales.view(torch.int32)[~want_scales.isnan()]) and torch.equal(got.isnan(), want_scales.isnan())


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows, K, ld", [(1, 16, 16), (1, 128, 128), (3, 112, 120), (5, 144, 144), (129, 272, 280), (64, 2880, 2880), (257, 400, 400), (17, 4096, 4104)])
def test_quantizer(mx, elem, block_rows, rows, K, ld):
    g = generator(rows + K)
    x = torch.randn((rows, ld), generator=g, device="cuda") * torch.exp(6 * torch.randn((rows, 1), generator=g, device="cuda"))
    x[:, ::37] *= 30.0
    same_quantized(mx, x.to(torch.bfloat16)[:, :K], elem, block_rows)


@pytest.mark.parametrize("elem", ELEMS)
def test_every_bf16_value_under_tops_of_every_mantissa(mx, elem):
    """All magnitudes below a top of each of the 128 mantissas: quotients midway between codes among them."""
    tops = torch.arange(0x4180, 0x4200, dtype=torch.int32)
    x = torch.zeros((128 * 18, 128), dtype=torch.int32)
    for i, top in enumerate(tops.tolist()):
        below = torch.arange(top - 127 * 18 + 1, top + 1)[-127 * 18:]  # 18 binades would be many codes alike: the neighbours of the top, and
        spread = (top - torch.arange(127 * 18) * 3).clamp_min(0)       # magnitudes 18 binades below it
        x[i * 18:(i + 1) * 18, 0] = top
        x[i * 18:(i + 1) * 18, 1:] = torch.where(torch.arange(127 * 18) % 2 == 0, below, spread).view(18, 127)
    x = torch.where((torch.arange(128) % 3 == 1)[None, :], x | 0x8000, x).to(torch.int16)
    same_quantized(mx, x.view(torch.bfloat16).cuda(), elem, 1)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_zeros_extremes_and_what_is_not_finite(mx, elem, block_rows):
    x = torch.randn((260, 640), generator=generator(5), device="cuda").to(torch.bfloat16)
    x[0] = 0.0
    x[1] = -0.0
    x[2, 5], x[3, 200], x[4, 130] = float("nan"), float("inf"), float("-inf")
    x[5:9] = (x[5:9].double() * 2.0 ** -130).to(torch.bfloat16)
    x[130:] = (x[130:].double() * 2.0 ** -118).to(torch.bfloat16)
    x[256:] = 0.0
    x[257, 300] = 3.3e38
    x[258, 7] = torch.tensor(1, dtype=torch.int16).view(torch.bfloat16)  # the smallest number
    same_quantized(mx, x, elem, block_rows)


@pytest.mark.parametrize("rows, K", [(1, 16), (130, 272), (2880, 144)])
def test_stacked_weights_have_blocks_of_their_own(mx, rows, K):
    x = torch.randn((3 * rows, K), generator=generator(8), device="cuda")
    x[rows:2 * rows] *= 50.0
    same_quantized(mx, x.to(torch.bfloat16), "e4m3", 128, 3)


def test_quantizer_writes_its_outputs_only(mx):
    x = torch.randn((7, 176), generator=generator(3), device="cuda").to(torch.bfloat16)
    for block_rows, n in ((1, 7), (128, 1)):
        codes = torch.full((9 * 176,), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((2 * n + 4,), -7.0, device="cuda")
        mx.mx_quantize_block128(x, "e4m3", block_rows, codes=codes[176:8 * 176].view(7, 176), scales=scales[1:1 + 2 * n].view(n, 2))
        want = ref.quantize(x, block_rows, "e4m3")
        assert torch.equal(codes[176:8 * 176].view(7, 176).cpu(), want[0]) and torch.equal(scales[1:1 + 2 * n].view(n, 2).cpu(), want[1])
        assert bool((codes[:176] == 0xA5).all()) and bool((codes[8 * 176:] == 0xA5).all()) and float(scales[0]) == -7.0 and bool((scales[1 + 2 * n:] == -7.0).all())
    empty = mx.mx_quantize_block128(torch.zeros((0, 128), dtype=torch.bfloat16, device="cuda"))
    assert empty[0].shape == (0, 128) and empty[1].shape == (0, 1)


# ---- products -------------------------------------------------------------------------------------------------------
def small_operand(gen, rows, K, scale_rows, elem):
    """Codes of 0, +-1, +-2 and scales that are powers of two: every sum is exact."""
    pick = torch.tensor([0.0, 1.0, -1.0, 2.0, -2.0], device="cuda")[torch.randint(0, 5, (rows, K), generator=gen, device="cuda")]
    scales = torch.exp2(torch.randint(-2, 3, (scale_rows, ref.blocks(K)), generator=gen, device="cuda").float())
    return pick.to(ref.F8[elem]).view(torch.uint8), scales


def real_operand(gen, mx, rows, K, block_rows, elem, groups=1):
    x = torch.randn((rows, K), generator=gen, device="cuda") * (1.0 if block_rows == 1 else 0.02)
    x[:, ::53] *= 10.0
    return mx.mx_quantize_block128(x.to(torch.bfloat16), elem, block_rows, groups)


SHAPES = [(1, 1, 16), (1, 16, 128), (3, 17, 112), (16, 128, 144), (5, 129, 1040), (33, 300, 2880), (64, 512, 4096), (65, 130, 272), (130, 257, 640), (300, 515, 1168),
          (257, 129, 128), (512, 640, 384), (1000, 1031, 2896)]


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("a, b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
def test_product_of_small_numbers_is_exact(mx, M, N, K, a, b):
    g = generator(M + N + K)
    ac, as_ = small_operand(g, M, K, M, a)
    bc, bs = small_operand(g, N, K, ref.blocks(N), b)
    want, _ = ref.product(ref.values(ac, as_, 1, a), ref.values(bc, bs, 128, b))
    wide = torch.full((M + 2, N + 5), 777.0, device="cuda")
    got = mx.mx_gemm_block128(a, ac, as_, b, bc, bs, "f32", out=wide[1:-1, 2:N + 2])
    assert torch.equal(got.double(), want)
    wide[1:-1, 2:N + 2] = 777.0
    assert bool((wide == 777.0).all())
    assert torch.equal(mx.mx_gemm_block128(a, ac, as_, b, bc, bs, "bf16").double(), want.float().to(torch.bfloat16).double())


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product_of_quantized_tensors(mx, M, N, K, out):
    g = generator(M * N + K)
    a, b = real_operand(g, mx, M, K, 1, "e4m3"), real_operand(g, mx, N, K, 128, "e4m3")
    want, size = ref.product(ref.values(*a, 1, "e4m3"), ref.values(*b, 128, "e4m3"))
    got = mx.mx_gemm_block128("e4m3", *a, "e4m3", *b, out).double()
    assert bool(((got - want).abs() <= ref.product_bound(want, size, K, out == "bf16")).all())


@pytest.mark.parametrize("M", [1, 20, 200, 600])
def test_nan_reaches_its_rows_and_columns_only(mx, M):
    """A NaN scale of a row, and one of a block of 128 columns; K ends inside a block, behind which the next row's codes lie."""
    N, K = 400, 656
    g = generator(M)
    ac, as_ = small_operand(g, M, K, M, "e4m3")
    bc, bs = small_operand(g, N, K, ref.blocks(N), "e4m3")
    as_[M // 2, 3] = float("nan")
    bs[1, 5] = float("nan")
    bc[311, 640] = 0x7F  # a NaN code
    got = mx.mx_gemm_block128("e4m3", ac, as_, "e4m3", bc, bs, "f32")
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[M // 2] = True
    bad[:, 128:256] = True
    bad[:, 311] = True
    assert torch.equal(got.isnan(), bad)


def offsets_of(counts):
    return torch.tensor([0] + list(counts), device="cuda").cumsum(0)


GROUPS = [([1], 16, 128), ([0, 3, 0, 1, 17, 0], 40, 272), ([130, 0, 64, 1, 300], 257, 400), ([5] * 70, 33, 144), ([700, 2, 0, 0, 515], 640, 1040), ([0, 0, 0], 48, 128),
          ([16] * 9, 300, 2880)]


@pytest.mark.parametrize("counts, N, K", GROUPS)
@pytest.mark.parametrize("index", [False, True])
def test_grouped_product_of_small_numbers_is_exact(mx, counts, N, K, index):
    g = generator(N + K + sum(counts))
    G, rows = len(counts), sum(counts)
    M = rows + 3  # rows behind the last group
    A = 11 + rows // 3 if index else M
    ac, as_ = small_operand(g, A, K, A, "e4m3")
    bc, bs = small_operand(g, G * N, K, G * ref.blocks(N), "e5m2")
    a_rows = torch.randint(0, A, (M,), generator=g, device="cuda").int() if index else None
    if index and rows > 4:
        a_rows[1], a_rows[3] = -1, A  # outside: rows of zeros
    out = torch.full((M, N), 777.0, device="cuda")
    mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e5m2", bc, bs, offsets_of(counts), N, "f32", a_rows=a_rows, out=out)
    a = torch.cat((ref.values(ac, as_, 1, "e4m3"), torch.zeros((1, K), dtype=torch.float64, device="cuda")))
    pick = torch.arange(M, device="cuda") if a_rows is None else torch.where((a_rows >= 0) & (a_rows < A), a_rows, A).long()
    at = 0
    for e, n in enumerate(counts):
        b = ref.values(bc[e * N:(e + 1) * N], bs[e * ref.blocks(N):(e + 1) * ref.blocks(N)], 128, "e5m2")
        assert torch.equal(out[at:at + n].double(), ref.product(a[pick[at:at + n]], b)[0]), e
        at += n
    assert bool((out[at:] == 777.0).all())


def test_grouped_rows_may_repeat_and_offsets_may_be_wrong(mx):
    """Offsets that lie outside, or decrease: rows in between are written or not, none outside C."""
    g = generator(4)
    N, K, M = 48, 256, 40
    ac, as_ = small_operand(g, M, K, M, "e4m3")
    bc, bs = small_operand(g, 3 * N, K, 3, "e4m3")
    for offsets in ([0, 50, 1 << 40, 1 << 41], [-5, 10, 3, 20], [1 << 62, -(1 << 62), 40, 40]):
        guarded = torch.full((M + 8, N), 777.0, device="cuda")
        mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e4m3", bc, bs, torch.tensor(offsets, device="cuda"), N, "f32", out=guarded[4:-4])
        assert bool((guarded[:4] == 777.0).all()) and bool((guarded[-4:] == 777.0).all())


def test_rows_and_scales_of_other_alignments(mx):
    """Scales that begin on any float, C on any element, a leading dimension that is odd."""
    g = generator(6)
    M, N, K = 70, 131, 400
    ac, as_ = small_operand(g, M, K, M, "e4m3")
    bc, bs = small_operand(g, N, K, ref.blocks(N), "e4m3")
    want, _ = ref.product(ref.values(ac, as_, 1, "e4m3"), ref.values(bc, bs, 128, "e4m3"))
    moved = lambda t: torch.cat((torch.zeros(1, device="cuda"), t.flatten()))[1:].view(t.shape)  # noqa: E731
    for dtype, name in ((torch.float32, "f32"), (torch.bfloat16, "bf16")):
        for shift, ld in ((0, N), (1, N), (3, N + 4), (1, N + 5)):
            buffer = torch.full((shift + M * ld + 3,), 777.0, dtype=dtype, device="cuda")
            out = buffer[shift:shift + M * ld].view(M, ld)[:, :N]
            mx.mx_gemm_block128("e4m3", ac, moved(as_), "e4m3", bc, moved(bs), name, out=out)
            assert torch.equal(out.double(), want.to(dtype).double())
            out.fill_(777.0)
            assert bool((buffer == 777.0).all())


def test_product_of_very_many_rows(mx):
    """More tiles of 64 rows than one launch takes: a kernel of larger ones.  A row is one 1 among 16, so that it picks a weight."""
    M, N = (1 << 28) + 70, 3
    one = int(torch.tensor(1.0).to(torch.float8_e4m3fn).view(torch.uint8))
    a = torch.zeros((M, 16), dtype=torch.uint8, device="cuda")
    a.view(-1)[:M // 16 * 256].view(-1, 16, 16).diagonal(dim1=1, dim2=2).fill_(one)
    a[M // 16 * 16:, 5] = one
    bc, bs = small_operand(generator(1), N, 16, 1, "e4m3")
    b = ref.values(bc, bs, 128, "e4m3").float()
    got = mx.mx_gemm_block128("e4m3", a, torch.ones((M, 1), device="cuda"), "e4m3", bc, bs, "bf16")
    assert bool((got[:M // 16 * 16].view(-1, 16, N) == b.T.to(torch.bfloat16)).all())
    assert bool((got[M // 16 * 16:] == b[:, 5].to(torch.bfloat16)).all())


def test_empty_products(mx):
    z = lambda r, c: torch.zeros((r, c), dtype=torch.uint8, device="cuda")  # noqa: E731
    s = lambda r, c: torch.zeros((r, c), device="cuda")  # noqa: E731
    assert mx.mx_gemm_block128("e4m3", z(0, 128), s(0, 1), "e4m3", z(5, 128), s(1, 1)).shape == (0, 5)
    assert mx.mx_gemm_block128("e4m3", z(4, 128), s(4, 1), "e4m3", z(0, 128), s(0, 1)).shape == (4, 0)
    out = torch.full((4, 5), 7.0, device="cuda")
    mx.mx_gemm_block128_grouped("e4m3", z(4, 128), s(4, 1), "e4m3", z(0, 128), s(0, 1), torch.zeros(1, dtype=torch.int64, device="cuda"), 5, "f32", out=out)
    assert bool((out == 7.0).all())


# ---- every kernel on problems that the rule gives to others ---------------------------------------------------------------------
@pytest.mark.parametrize("kernel", [1, 2, 3, 4, 5, 6, 7, 8, 9])
@pytest.mark.parametrize("M, N, K", [(1, 5, 16), (70, 300, 128), (129, 131, 2896), (300, 515, 144), (513, 257, 640), (257, 1100, 384)])
def test_every_kernel_is_exact_on_small_numbers(mx, kernel, M, N, K):
    g = generator(M + N + K)
    ac, as_ = small_operand(g, M, K, M, "e5m2")
    bc, bs = small_operand(g, N, K, ref.blocks(N), "e4m3")
    want, _ = ref.product(ref.values(ac, as_, 1, "e5m2"), ref.values(bc, bs, 128, "e4m3"))
    for dtype, name in ((torch.float32, "f32"), (torch.bfloat16, "bf16")):
        wide = torch.full((M + 2, N + 3), 777.0, dtype=dtype, device="cuda")
        with mx.forced(block128=kernel):
            mx.mx_gemm_block128("e5m2", ac, as_, "e4m3", bc, bs, name, out=wide[1:-1, 1:N + 1])
        assert torch.equal(wide[1:-1, 1:N + 1].double(), want.to(dtype).double())
        wide[1:-1, 1:N + 1] = 777.0
        assert bool((wide == 777.0).all())


@pytest.mark.parametrize("kernel", [1, 2, 3, 4, 5, 6, 7, 8, 9])
@pytest.mark.parametrize("index", [False, True])
def test_every_kernel_by_groups(mx, kernel, index):
    counts, N, K = [130, 0, 64, 1, 300, 0, 31] + [3] * 66, 257, 400
    g = generator(kernel)
    G, rows = len(counts), sum(counts)
    A = 90 if index else rows
    ac, as_ = small_operand(g, A, K, A, "e4m3")
    bc, bs = small_operand(g, G * N, K, G * ref.blocks(N), "e4m3")
    a_rows = torch.randint(0, A, (rows,), generator=g, device="cuda").int() if index else None
    out = torch.full((rows, N), 777.0, device="cuda")
    with mx.forced(block128=kernel):
        mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e4m3", bc, bs, offsets_of(counts), N, "f32", a_rows=a_rows, out=out)
    a = ref.values(ac, as_, 1, "e4m3")
    a = a if a_rows is None else a[a_rows.long()]
    at = 0
    for e, n in enumerate(counts):
        b = ref.values(bc[e * N:(e + 1) * N], bs[e * ref.blocks(N):(e + 1) * ref.blocks(N)], 128, "e4m3")
        assert torch.equal(out[at:at + n].double(), ref.product(a[at:at + n], b)[0]), e
        at += n


@pytest.mark.parametrize("kernel", [1, 2, 3, 4, 5, 6, 7, 8, 9])
def test_every_kernel_on_quantized_tensors(mx, kernel):
    M, N, K = 300, 400, 2896
    g = generator(3)
    a, b = real_operand(g, mx, M, K, 1, "e4m3"), real_operand(g, mx, N, K, 128, "e4m3")
    want, size = ref.product(ref.values(*a, 1, "e4m3"), ref.values(*b, 128, "e4m3"))
    with mx.forced(block128=kernel):
        got = mx.mx_gemm_block128("e4m3", *a, "e4m3", *b, "f32").double()
    assert bool(((got - want).abs() <= ref.product_bound(want, size, K, False)).all())


@pytest.mark.parametrize("M, N, K", [(4353, 4232, 144), (4353, 4232, 400), (2049, 8712, 272), (300, 520, 1040), (4353, 4232, 128)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_a_workgroup_takes_tile_after_tile(mx, M, N, K, out):
    """More than 256 tiles of 256 x 256, the last of a row and of a column cut off, K of two blocks and more (and of one)."""
    g = generator(M + K)
    ac, as_ = small_operand(g, M, K, M, "e4m3")
    bc, bs = small_operand(g, N, K, ref.blocks(N), "e4m3")
    want, _ = ref.product(ref.values(ac, as_, 1, "e4m3"), ref.values(bc, bs, 128, "e4m3"))
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    wide = torch.full((M + 2, N + 16), 777.0, dtype=dtype, device="cuda")
    with mx.forced(block128=8):
        mx.mx_gemm_block128("e4m3", ac, as_, "e4m3", bc, bs, out, out=wide[1:-1, 8:N + 8])
    assert torch.equal(wide[1:-1, 8:N + 8].double(), want.to(dtype).double())
    wide[1:-1, 8:N + 8] = 777.0
    assert bool((wide == 777.0).all())


@pytest.mark.parametrize("index", [False, True])
@pytest.mark.parametrize("K", [272, 528])
def test_tile_after_tile_by_groups(mx, index, K):
    counts, N = [3000, 0, 17, 700, 256, 0, 1] + [40] * 70 + [2100], 1096
    g = generator(K)
    G, rows = len(counts), sum(counts)
    A = 900 if index else rows
    ac, as_ = small_operand(g, A, K, A, "e4m3")
    bc, bs = small_operand(g, G * N, K, G * ref.blocks(N), "e4m3")
    a_rows = torch.randint(0, A, (rows,), generator=g, device="cuda").int() if index else None
    if index:
        a_rows[5], a_rows[3500] = -1, A
    out = torch.full((rows + 1, N), 777.0, device="cuda")
    with mx.forced(block128=8):
        mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e4m3", bc, bs, offsets_of(counts), N, "f32", a_rows=a_rows, out=out[:-1])
    a = torch.cat((ref.values(ac, as_, 1, "e4m3"), torch.zeros((1, K), dtype=torch.float64, device="cuda")))
    a = a[:-1] if a_rows is None else a[torch.where((a_rows >= 0) & (a_rows < A), a_rows, A).long()]
    at = 0
    for e, n in enumerate(counts):
        b = ref.values(bc[e * N:(e + 1) * N], bs[e * ref.blocks(N):(e + 1) * ref.blocks(N)], 128, "e4m3")
        assert torch.equal(out[at:at + n].double(), ref.product(a[at:at + n], b)[0]), e
        at += n
    assert bool((out[-1] == 777.0).all())


@pytest.mark.parametrize("kernel", [0, 2, 4, 5, 8, 9])
def test_more_groups_than_a_table_holds(mx, kernel):
    """1100 groups, most of one row or none, a few of more than a tile."""
    N, K = 40, 144
    counts = [(3 * i) % 4 % 3 for i in range(1100)]
    counts[7], counts[1030], counts[1099] = 300, 270, 530
    g = generator(9)
    rows = sum(counts)
    ac, as_ = small_operand(g, rows, K, rows, "e4m3")
    bc, bs = small_operand(g, len(counts) * N, K, len(counts), "e4m3")
    out = torch.full((rows + 2, N), 777.0, device="cuda")
    with mx.forced(**({"block128": kernel} if kernel else {})):
        mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e4m3", bc, bs, offsets_of(counts), N, "f32", out=out[:-2])
    a, b = ref.values(ac, as_, 1, "e4m3"), torch.cat([ref.values(bc[i * N:(i + 1) * N], bs[i:i + 1], 128, "e4m3") for i in range(len(counts))])
    of_row = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), torch.tensor(counts, device="cuda"))
    want = (a[:, None, :] * b.view(len(counts), N, K)[of_row]).sum(2)
    assert torch.equal(out[:-2].double(), want)
    assert bool((out[-2:] == 777.0).all())


# ---- scales near the smallest normal number, fp32 results, E5M2 tensors, many tiles a workgroup -----------------------------------
@pytest.mark.parametrize("kernel", [1, 2, 3, 4, 5, 6, 7, 8, 9])
@pytest.mark.parametrize("a, b", [("e4m3", "e4m3"), ("e5m2", "e5m2")])
def test_products_of_scales_below_the_normal_numbers(mx, kernel, a, b):
    """Scales down to the quantizer's floor, 2^-126: their product rounds to a multiple of 2^-149, which the blocks' sums multiply."""
    M, N, K = 70, 300, 656
    g = generator(kernel)
    codes = lambda rows, elem: (torch.randn((rows, K), generator=g, device="cuda") * ref.TOP[elem] / 8).clamp(-ref.TOP[elem], ref.TOP[elem]).to(ref.F8[elem])  # noqa: E731
    ac, bc = codes(M, a).view(torch.uint8), codes(N, b).view(torch.uint8)
    fraction = lambda *shape: 1 + torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    as_ = fraction(M, ref.blocks(K)) * torch.exp2(torch.randint(-126, -100, (M, 1), generator=g, device="cuda").float())
    bs = fraction(ref.blocks(N), ref.blocks(K)) * torch.exp2(torch.randint(-30, 0, (ref.blocks(N), 1), generator=g, device="cuda").float())
    as_[0], as_[1], as_[2] = 2.0 ** -126, 2.0 ** -126, 1.3 * 2.0 ** -73
    bs[1] = 1.7 * 2.0 ** -73
    with mx.forced(block128=kernel):
        got = mx.mx_gemm_block128(a, ac, as_, b, bc, bs, "f32").double()
    want, size = ref.product(ref.values(ac, as_, 1, a), ref.values(bc, bs, 128, b))
    # a product of scales is off by half of 2^-149 at most, and so is each of the blocks' multiply-adds
    ones = lambda rows: torch.ones((rows, ref.blocks(K)), device="cuda")  # noqa: E731
    _, codes_size = ref.product(ref.values(ac, ones(M), 1, a), ref.values(bc, ones(ref.blocks(N)), 128, b))
    assert bool(((got - want).abs() <= ref.product_bound(want, size, K, False) + 2.0 ** -149 * (codes_size + ref.blocks(K))).all())


@pytest.mark.parametrize("M, N, K", [(1, 512, 4096), (64, 512, 4096), (300, 515, 1168), (1000, 1031, 2896), (2100, 2060, 1024)])
@pytest.mark.parametrize("a, b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("larger", [1.0, 100.0])
def test_fp32_products_of_quantized_tensors_are_near(mx, M, N, K, a, b, larger):
    """N(0, 1), and one channel in a hundred larger.  Products are cut off 13 bits below the largest of 16 at the most, which alone would allow 2^-12 of the output's RMS for
    N(0, 1) (the largest of 16 is below four times their RMS); most have fewer bits than that, and 1e-4 is what is promised."""
    g = generator(M + N + K)
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, ::100] *= larger
    x = mx.mx_quantize_block128(x.to(torch.bfloat16), a)
    w = mx.mx_quantize_block128((0.02 * torch.randn((N, K), generator=g, device="cuda")).to(torch.bfloat16), b, 128)
    want, size = ref.product(ref.values(*x, 1, a), ref.values(*w, 128, b))
    got = mx.mx_gemm_block128(a, *x, b, *w, "f32").double()
    assert bool(((got - want).abs() <= ref.product_bound(want, size, K, False)).all())
    assert float((got - want).square().mean().sqrt()) <= 1e-4 * float(want.square().mean().sqrt())
    assert torch.equal(mx.mx_gemm_block128(a, *x, b, *w, "f32").double(), got)  # (the same sums every time)


@pytest.mark.parametrize("M, N, K", [(8449, 8456, 144), (8449, 8456, 400)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_a_workgroup_takes_many_tiles(mx, M, N, K, out):
    """34 x 34 tiles of 256 x 256 among 256 workgroups: four and five each, the last of a row and of a column cut off."""
    g = generator(M + K)
    ac, as_ = small_operand(g, M, K, M, "e4m3")
    bc, bs = small_operand(g, N, K, ref.blocks(N), "e5m2")
    want, _ = ref.product(ref.values(ac, as_, 1, "e4m3"), ref.values(bc, bs, 128, "e5m2"))
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    wide = torch.full((M + 2, N + 16), 777.0, dtype=dtype, device="cuda")
    with mx.forced(block128=8):
        mx.mx_gemm_block128("e4m3", ac, as_, "e5m2", bc, bs, out, out=wide[1:-1, 8:N + 8])
    assert torch.equal(wide[1:-1, 8:N + 8].double(), want.to(dtype).double())
    wide[1:-1, 8:N + 8] = 777.0
    assert bool((wide == 777.0).all())


@pytest.mark.parametrize("index", [False, True])
@pytest.mark.parametrize("K, out", [(144, "bf16"), (400, "f32")])
def test_many_tiles_by_groups(mx, index, K, out):
    """97 tile-rows by 12 columns among 256 workgroups; rows behind the last group stay."""
    counts, N = [3000, 0, 17, 700, 256, 0, 1] + [40] * 70 + [2100], 2904
    g = generator(K)
    G, rows = len(counts), sum(counts)
    A = 900 if index else rows + 1
    ac, as_ = small_operand(g, A, K, A, "e4m3")
    bc, bs = small_operand(g, G * N, K, G * ref.blocks(N), "e4m3")
    a_rows = torch.randint(0, A, (rows + 1,), generator=g, device="cuda").int() if index else None
    if index:
        a_rows[5], a_rows[3500], a_rows[7000] = -1, A, 1 << 30
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    c = torch.full((rows + 1, N), 777.0, dtype=dtype, device="cuda")
    with mx.forced(block128=8):
        mx.mx_gemm_block128_grouped("e4m3", ac, as_, "e4m3", bc, bs, offsets_of(counts), N, out, a_rows=a_rows, out=c)
    a = torch.cat((ref.values(ac, as_, 1, "e4m3"), torch.zeros((1, K), dtype=torch.float64, device="cuda")))
    a = a[:-1] if a_rows is None else a[torch.where((a_rows >= 0) & (a_rows < A), a_rows, A).long()]
    at = 0
    for e, n in enumerate(counts):
        b = ref.values(bc[e * N:(e + 1) * N], bs[e * ref.blocks(N):(e + 1) * ref.blocks(N)], 128, "e4m3")
        assert torch.equal(c[at:at + n].double(), ref.product(a[at:at + n], b)[0].to(dtype).double()), e
        at += n
    assert bool((c[-1] == 777.0).all())
