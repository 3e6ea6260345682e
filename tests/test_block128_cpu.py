"""Block-scaled FP8 and routing without a GPU: calls that are refused before a device is touched, and empty ones."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ENULL, EALIGN, EUNSUPPORTED = 0, -1, -2, -3, -4
A, FAR = 0x10000, 1 << 40  # fake device addresses, aligned to everything and far apart


@pytest.fixture(scope="module")
def lib():
    from paper_2603_08713_amd import binding
    from paper_2603_08713_amd import build as mxbuild

    if not os.path.exists(mxbuild.LIB):
        mxbuild.build()
    return binding.load_library()


def changed(base, **changes):
    assert set(changes) <= set(base)
    return list(dict(base, **changes).values())


QUANT = dict(elem=1, x=A, groups=2, rows=5, K=272, ldx=280, block_rows=128, codes=A, scales=A, stream=None)
GEMM = dict(ae=1, a=A, sa=A, be=2, b=A, sb=A, M=3, N=5, K=272, dtype=1, C=A, ldc=5, stream=None)
GROUPED = dict(ae=1, a=A, sa=A, count=4, index=A, be=2, b=A, sb=A, groups=2, offsets=A, M=3, N=5, K=272, dtype=1, C=A, ldc=5, stream=None)
PLAN = dict(dtype=0, logits=A, ld=40, T=300, n=A + FAR, E=40, k=4, score=1, bias=A + 2 * FAR, renorm=1, scale=1.0, experts=A + 3 * FAR, weights=A + 4 * FAR, offsets=A + 5 * FAR,
            rows=A + 6 * FAR, tokens=A + 7 * FAR, work=A + 8 * FAR, bytes=1 << 20, stream=None)
COMBINE = dict(ytype=1, y=A, R=10, ldy=40, rows=A + FAR, weights=A + 2 * FAR, T=3, k=2, N=40, otype=0, add=A + 3 * FAR, lda=40, out=A + 4 * FAR, ldo=40, stream=None)

BAD_PRODUCT = [(dict(ae=5), EINVAL), (dict(be=-1), EINVAL), (dict(ae=0), EUNSUPPORTED), (dict(be=3), EUNSUPPORTED), (dict(K=264), EUNSUPPORTED), (dict(K=0), EUNSUPPORTED),
               (dict(K=-16), EINVAL), (dict(K=(1 << 22) + 16), EINVAL), (dict(N=-1), EINVAL), (dict(M=-1), EINVAL), (dict(N=1 << 31, ldc=1 << 31), EINVAL),
               (dict(M=1 << 31), EINVAL), (dict(dtype=2), EINVAL), (dict(ldc=4), EINVAL), (dict(a=None), ENULL), (dict(sa=None), ENULL), (dict(b=None), ENULL), (dict(sb=None), ENULL),
               (dict(C=None), ENULL), (dict(a=A + 8), EALIGN), (dict(b=A + 4), EALIGN), (dict(sa=A + 2), EALIGN), (dict(sb=A + 1), EALIGN), (dict(C=A + 1), EALIGN)]


@pytest.mark.parametrize("name, base, bad", [
    ("mx_quantize_block128", QUANT, [(dict(elem=5), EINVAL), (dict(elem=0), EUNSUPPORTED), (dict(elem=4), EUNSUPPORTED), (dict(groups=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(K=-16), EINVAL),
                                     (dict(K=264), EUNSUPPORTED), (dict(K=(1 << 22) + 16, ldx=1 << 23), EUNSUPPORTED), (dict(ldx=264), EINVAL), (dict(ldx=276), EALIGN),
                                     (dict(block_rows=64), EINVAL), (dict(x=None), ENULL), (dict(codes=None), ENULL), (dict(scales=None), ENULL), (dict(x=A + 8), EALIGN),
                                     (dict(codes=A + 8), EALIGN), (dict(scales=A + 2), EALIGN), (dict(rows=1 << 31), EINVAL), (dict(groups=1 << 20, rows=1 << 20), EINVAL),
                                     (dict(groups=1 << 40, rows=1 << 40), EINVAL), (dict(block_rows=1, rows=1 << 28, groups=1, K=4096, ldx=4096), EINVAL)]),
    ("mx_gemm_block128", GEMM, BAD_PRODUCT),
    ("mx_gemm_block128_grouped", GROUPED, BAD_PRODUCT + [(dict(groups=-1), EINVAL), (dict(count=-1), EINVAL), (dict(index=None, count=2), EINVAL), (dict(offsets=None), ENULL),
                                                         (dict(offsets=A + 4), EALIGN), (dict(index=A + 2), EALIGN), (dict(count=1 << 31), EINVAL),
                                                         (dict(count=1 << 24), EUNSUPPORTED)]),
    ("mx_moe_plan", PLAN, [(dict(dtype=2), EINVAL), (dict(score=2), EINVAL), (dict(score=0), EUNSUPPORTED), (dict(T=-1), EINVAL), (dict(E=0), EINVAL), (dict(k=0), EINVAL), (dict(k=41), EINVAL),
                           (dict(k=33), EUNSUPPORTED), (dict(E=1025, ld=1025), EUNSUPPORTED), (dict(T=(1 << 20) + 1), EUNSUPPORTED), (dict(ld=39), EINVAL), (dict(bytes=100), EINVAL),
                           (dict(work=None), ENULL), (dict(logits=None), ENULL), (dict(experts=None), ENULL), (dict(weights=None), ENULL), (dict(offsets=None), ENULL),
                           (dict(rows=None), ENULL), (dict(tokens=None), ENULL), (dict(logits=A + 2), EALIGN), (dict(bias=A + 2 * FAR + 2), EALIGN), (dict(n=A + FAR + 4), EALIGN),
                           (dict(offsets=A + 4), EALIGN), (dict(work=A + 8 * FAR + 2), EALIGN), (dict(experts=A), EINVAL), (dict(weights=A + 300 * 160 - 4), EINVAL),
                           (dict(offsets=A + FAR), EINVAL), (dict(rows=A + 2 * FAR + 156), EINVAL), (dict(tokens=A + 6 * FAR), EINVAL), (dict(work=A + 3 * FAR + 4796), EINVAL)]),
    ("mx_moe_combine", COMBINE, [(dict(ytype=2), EINVAL), (dict(otype=-1), EINVAL), (dict(T=-1), EINVAL), (dict(k=-1), EINVAL), (dict(N=-1), EINVAL), (dict(R=-1), EINVAL), (dict(ldy=39), EINVAL),
                                 (dict(ldo=39), EINVAL), (dict(lda=39), EINVAL), (dict(k=1025), EINVAL), (dict(T=1 << 31), EINVAL), (dict(R=1 << 31, ldy=1 << 31), EINVAL), (dict(T=1 << 25), EINVAL), (dict(y=None), ENULL),
                                 (dict(rows=None), ENULL), (dict(weights=None), ENULL), (dict(out=None), ENULL), (dict(y=A + 1), EALIGN), (dict(out=A + 4 * FAR + 2), EALIGN),
                                 (dict(add=A + 3 * FAR + 2), EALIGN), (dict(rows=A + FAR + 2), EALIGN), (dict(out=A), EINVAL), (dict(out=A + FAR + 20), EINVAL),
                                 (dict(out=A + 2 * FAR), EINVAL), (dict(out=A + 3 * FAR + 4), EINVAL), (dict(out=A + 3 * FAR, ldo=44), EINVAL)]),
])
def test_refusals(lib, name, base, bad):
    call = getattr(lib, name)
    assert len(base) == len(call.argtypes)
    for changes, status in bad:
        assert call(*changed(base, **changes)) == status, (name, changes)


def test_what_is_not_refused(lib):
    """The same calls unchanged pass the arguments' checks: without a device they end at the device."""
    torch = pytest.importorskip("torch")
    if torch.cuda.device_count():
        pytest.skip("the addresses are made up")
    for name, base, changes in (("mx_quantize_block128", QUANT, {}), ("mx_quantize_block128", QUANT, dict(block_rows=1)), ("mx_gemm_block128", GEMM, {}),
                                ("mx_gemm_block128_grouped", GROUPED, {}), ("mx_gemm_block128_grouped", GROUPED, dict(index=None)), ("mx_moe_plan", PLAN, {}),
                                ("mx_moe_plan", PLAN, dict(n=None, bias=None, score=0, T=64, work=None, bytes=0)), ("mx_moe_combine", COMBINE, {}),
                                ("mx_moe_combine", COMBINE, dict(out=A + 3 * FAR)), ("mx_moe_combine", COMBINE, dict(add=None, lda=0, k=0, y=None, rows=None, weights=None))):
        assert getattr(lib, name)(*changed(base, **changes)) == EUNSUPPORTED, (name, changes)


def test_empty_calls_do_nothing(lib):
    assert lib.mx_quantize_block128(*changed(QUANT, rows=0, x=None, codes=None, scales=None)) == OK
    assert lib.mx_quantize_block128(*changed(QUANT, groups=0)) == OK and lib.mx_quantize_block128(*changed(QUANT, K=0)) == OK
    assert lib.mx_gemm_block128(*changed(GEMM, M=0, a=None)) == OK and lib.mx_gemm_block128(*changed(GEMM, N=0, b=None)) == OK
    assert lib.mx_gemm_block128_grouped(*changed(GROUPED, M=0)) == OK and lib.mx_gemm_block128_grouped(*changed(GROUPED, groups=0, offsets=None)) == OK
    assert lib.mx_moe_combine(*changed(COMBINE, T=0)) == OK and lib.mx_moe_combine(*changed(COMBINE, N=0)) == OK


def test_workspace_sizes(lib):
    size = lib.mx_moe_plan_workspace
    assert size(0, 8, 2) == 0 and size(64, 32, 4) == 0
    for T in (129, 500, 8192, 100000, 1 << 20):  # whole chunks' counts of 32 bits
        for E in (1, 8, 128, 1000, 1024):
            n = size(T, E, 1)
            assert n > 0 and n % (4 * E) == 0 and n <= 1024 * E * 4, (T, E)
    assert size(-1, 8, 2) == EINVAL and size(5, 0, 1) == EINVAL and size(5, 8, 9) == EINVAL and size(5, 1025, 1) == EUNSUPPORTED and size(5, 64, 33) == EUNSUPPORTED
    assert size((1 << 20) + 1, 8, 2) == EUNSUPPORTED


def test_division_of_block_numbers():
    """The quantizer's rows by multiplication, as its launch prepares it: exact for every block number below 2^31."""
    import random

    r = random.Random(0)
    for per_row in list(range(1, 300)) + [2 ** i + d for i in range(8, 16) for d in (-1, 0, 1)]:
        shift = 0
        while (1 << shift) < per_row:
            shift += 1
        magic = (((1 << shift) - per_row) * (1 << 32) + per_row - 1) // per_row
        assert 0 <= magic < 1 << 32
        for b in [0, 1, per_row - 1, per_row, (1 << 31) - 1, (1 << 31) - (1 << 31) % per_row - 1] + [r.randrange(1 << 31) for _ in range(40)]:
            assert ((b * magic >> 32) + b) >> shift == b // per_row, (per_row, b)


def test_binding_refuses_what_is_not_on_the_gpu():
    torch = pytest.importorskip("torch")
    import paper_2603_08713_amd as mx

    codes, scales = torch.zeros((2, 128), dtype=torch.uint8), torch.zeros((2, 1))
    i32 = torch.zeros((2, 1), dtype=torch.int32)
    for call in (lambda: mx.mx_quantize_block128(torch.zeros((2, 128), dtype=torch.bfloat16)), lambda: mx.mx_gemm_block128("e4m3", codes, scales, "e4m3", codes, scales[:1]),
                 lambda: mx.mx_gemm_block128_grouped("e4m3", codes, scales, "e4m3", codes, scales[:1], torch.zeros(2, dtype=torch.int64), 2),
                 lambda: mx.mx_moe_plan(torch.zeros((2, 8)), 1), lambda: mx.mx_moe_combine(scales, i32, scales), lambda: mx.mx_moe_plan(None, 1)):
        with pytest.raises(TypeError):
            call()
