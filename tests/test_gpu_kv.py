"""The paged MXFP4 cache on the GPU: plan, norm and rotation, write and read, against plain 64-bit implementations.  Codes, scales,
words and whole numbers are compared for equality, bf16 results too (they are one rounding of a value known to 53 bits)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2603_08713_amd as mx_

    mx_.load_library()
    return mx_


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(seed, T, H, D, scale=1.0):
    x = torch.randn((T, H, D), generator=_gen(seed), device="cuda") * scale
    x[..., D // 3] *= 20
    return x.to(torch.bfloat16)


def _filled_cache(mx, seed, pages, H, D, page, mbs):
    """A cache whose bytes all hold something."""
    g = _gen(seed)

    def fill(a):
        return None if a is None else torch.randint(0, 256, a.shape, generator=g, device="cuda", dtype=torch.uint8)

    return tuple(tuple(fill(a) for a in cache) for cache in mx.mx_kv_cache(pages, H, D, page, mbs))


def _copy(caches):
    return tuple(tuple(None if a is None else a.clone() for a in cache) for cache in caches)


def _same(got, want):
    return all((a is None and b is None) or torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def _cos_sin(positions, R):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    return torch.cat((angle.cos(), angle.sin()), -1).float().cuda()


# ---- plan ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("ctx, new, page, width, free, start, T", [
    ([5], [1], 16, 4, 3, 0, 1),
    ([16, 0, 31, 7], [1, 1, 1, 1], 16, 4, 9, 2, 4),                        # one begins a page, one fills its page
    ([0, 3, 0, 64, 100], [0, 70, 0, 33, 0], 32, 8, 20, 0, 110),            # requests without tokens; padding behind the last
    ([10, 10, 10], [40, 40, 40], 16, 8, 5, 1, 120),                        # pages run out
    ([10, 90], [100, 3], 16, 6, 30, 0, 103),                               # the table's row is at its end
    ([-4, 6], [-1, 2], 16, 4, 4, 0, 5),                                    # negative lengths count as none
    ([0] * 7, [1] * 7, 64, 2, 6, 100, 7),                                  # nothing free
    ([7, 7], [5, 5], 16, 4, 4, 0, 6),                                      # fewer places than tokens
    ([], [], 16, 0, 0, 3, 2),
    ([5], [0], 16, 1, 0, 0, 0),
])
def test_plan(mx, ctx, new, page, width, free, start, T):
    rng = np.random.default_rng(len(ctx) + T)
    S = len(ctx)
    table = rng.integers(0, 1000, (S, width)).astype(np.int32)
    free = rng.permutation(1000)[:free].astype(np.int32)
    want = ref.plan(np.array(ctx, np.int64), np.array(new, np.int64), page, table, free, start, T)
    t = torch.from_numpy(table).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = mx.mx_kv_plan(i32(ctx), i32(new), page, t, torch.from_numpy(free).cuda(), i32([start]), T)
    for name, g, w in zip(("row_offsets", "kv_lens", "slots", "positions"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert got[4].item() == want[4] and np.array_equal(t.cpu().numpy(), want[5])


@pytest.mark.parametrize("S, most, new, page", [(1, 3000, 5000, 64), (1025, 300, 1, 16), (4096, 90, 3, 32), (300, 2000, 900, 128), (63, 5, 9000, 256)])
def test_plan_of_many(mx, S, most, new, page):
    rng = np.random.default_rng(S)
    ctx, n = rng.integers(0, most, S), rng.integers(0, new + 1, S)
    width = (most + new) // page + 2
    table = rng.integers(0, 1 << 20, (S, width)).astype(np.int32)
    free = rng.permutation(int(n.sum()) // page + 2 * S + 5).astype(np.int32)
    T = int(n.sum()) + 3
    want = ref.plan(ctx, n, page, table, free, 4, T)
    t = torch.from_numpy(table).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = mx.mx_kv_plan(i32(ctx), i32(n), page, t, torch.from_numpy(free).cuda(), i32([4]), T)
    for name, g, w in zip(("row_offsets", "kv_lens", "slots", "positions"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert got[4].item() == want[4] and np.array_equal(t.cpu().numpy(), want[5])


@pytest.mark.parametrize("ctx, new, page, width, free, start, T", [
    ([7, 7], [5, 40], 16, 4, 6, 0, 6),                  # pages that begin beyond the places, one of a request that has some
    ([0, 0, 40], [20, 50, 33], 16, 5, 20, 1, 10),       # and those of requests that have none
    ([16, 3], [16, 1], 16, 3, 4, 0, 16),                # the last place ends a page
    ([16, 3], [17, 13], 16, 3, 4, 0, 16),               # the first token beyond begins one
    ([0, 30], [3, 5], 16, 4, 9, 0, 0),                  # no places at all
    ([0, 0], [100, 100], 16, 4, 9, 0, 40),              # the free list and the table's rows are at their ends
])
def test_plan_takes_the_pages_of_tokens_without_a_place(mx, ctx, new, page, width, free, start, T):
    """Fewer places than tokens: the pages of the others are counted in free_next, so they stand in the table too, and no entry is left from
    before - attention would read another request's page there."""
    test_plan(mx, ctx, new, page, width, free, start, T)


@pytest.mark.parametrize("S, most, new, page, part", [(1, 100, 70000, 16, 3), (1100, 300, 90, 16, 2), (4096, 90, 40, 32, 50), (70, 0, 5000, 64, 9)])
def test_plan_of_many_with_few_places(mx, S, most, new, page, part):
    rng = np.random.default_rng(S)
    ctx, n = rng.integers(0, most + 1, S), rng.integers(0, new + 1, S)
    width = (most + new) // page + 2
    table = rng.integers(0, 1 << 20, (S, width)).astype(np.int32)
    free = rng.permutation(int(n.sum()) // page + 2 * S + 5).astype(np.int32)
    T = int(n.sum()) // part
    want = ref.plan(ctx, n, page, table, free, 4, T)
    t = torch.from_numpy(table).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = mx.mx_kv_plan(i32(ctx), i32(n), page, t, torch.from_numpy(free).cuda(), i32([4]), T)
    for name, g, w in zip(("row_offsets", "kv_lens", "slots", "positions"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert got[4].item() == want[4] and np.array_equal(t.cpu().numpy(), want[5])


def test_plan_of_lengths_that_32_bits_cannot_add(mx):
    """Sums of new tokens and of pages beyond 2^31: the places that there are, every entry of the table, totals that stay at 2^31 - 1."""
    most = (1 << 31) - 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((5, 4), 77, dtype=torch.int32, device="cuda")
    offsets, lens, slots, positions, after = mx.mx_kv_plan(i32([20, 0, most, 0, 3]), i32([most, most, most, 5, -most]), 16, table, i32([9, 8, 7]), i32([1]), 12)
    assert offsets.tolist() == [0, most, 2 * most, 3 * most, 3 * most + 5, 3 * most + 5] and lens.tolist() == [most, most, most, 5, 3]
    # request 0 holds pages 0 and 1 of its row and takes entries 1 and 2 of the list (8 and 7); the others find it empty
    assert table.tolist() == [[77, 77, 8, 7], [-1, -1, -1, -1], [77, 77, 77, 77], [-1, 77, 77, 77], [77, 77, 77, 77]]
    assert positions.tolist() == list(range(20, 32)) and slots.tolist() == [77 * 16 + p for p in range(4, 16)]
    assert after.item() == 1 + -(-(20 + most) // 16) - 2 + -(-most // 16) + -(-2 * most // 16) - -(-most // 16) + 1


# ---- norm and rotation ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("norm, turn", [("both", "all"), ("none", "all"), ("both", "none"), ("k", "part"), ("none", "none")])
def test_norm_rope(mx, D, style, norm, turn):
    T, Hq, Hkv = 7, 5, 2
    qkv = _rows(D, T, Hq + 2 * Hkv, D)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]  # strided, as a projection leaves them
    g = _gen(1)
    qw = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) if norm == "both" else None
    kw = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) if norm != "none" else None
    R = 0 if turn == "none" else D if turn == "all" else D // 2
    table = _cos_sin(300, R) if R else None
    positions = torch.tensor([0, 299, 5, 300, -1, 17, 1 << 30], dtype=torch.int32, device="cuda") if R else None
    marked = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    got = mx.mx_qk_norm_rope(q, k, positions, table, qw, kw, 1e-5, style, q_out=marked[0].contiguous(), k_out=marked[1].contiguous())
    for x, w, y in ((q, qw, got[0]), (k, kw, got[1])):
        want = ref.to_bf16(ref.norm_rope(x, positions, table, w, 1e-5, style))
        y = y.cpu()
        if R:
            assert bool((y[4] == 7.0).all())  # a padding token
            assert bool(torch.isnan(y[3, :, :R].float()).all()) and bool(torch.isnan(y[6, :, :R].float()).all())
            want[4] = 7.0
        # the same bits, NaN wherever the definition has one
        assert torch.equal(torch.isnan(want.float()), torch.isnan(y.float()))
        assert torch.equal(torch.nan_to_num(want.float()), torch.nan_to_num(y.float()))
    mx.mx_qk_norm_rope(q, k, positions, table, qw, kw, 1e-5, style, q_out=q, k_out=k)  # in place, the same bits
    for x, y, keep in ((q, got[0], True), (k, got[1], True)):
        rows = [0, 1, 2, 3, 5, 6]
        assert np.array_equal(ref.bits(x[rows]), ref.bits(y[rows]))


def test_norm_rope_many_rows_and_one_side_only(mx):
    for T, Hq, Hkv in ((1025, 64, 8), (1, 1, 0), (33, 0, 3)):
        q, k = _rows(T, T, Hq, 128), _rows(T + 1, T, Hkv, 128)
        w = torch.linspace(0.5, 1.5, 128, device="cuda").to(torch.bfloat16)
        table = _cos_sin(2048, 128)
        positions = torch.arange(T, device="cuda").int()
        got = mx.mx_qk_norm_rope(q, k, positions, table, w, w)
        for x, y in ((q, got[0]), (k, got[1])):
            assert np.array_equal(ref.bits(ref.to_bf16(ref.norm_rope(x, positions, table, w, 1e-6, "half"))), ref.bits(y))


def test_norm_rope_extremes(mx):
    """Rows of zeros, infinities and NaN: what the formula gives, and nothing in other rows."""
    D = 128
    q = _rows(3, 6, 2, D)
    q[1] = 0
    q[2, :, 5] = float("inf")
    q[3, 0, 9] = float("nan")
    q[4] *= 1e30
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    table, positions = _cos_sin(10, D), torch.arange(6, device="cuda").int()
    got = mx.mx_qk_norm_rope(q, q[:, :0], positions, table, w, None)[0].cpu()
    want = ref.to_bf16(ref.norm_rope(q, positions, table, w, 1e-6, "half"))
    assert torch.equal(torch.isnan(want.float()), torch.isnan(got.float()))
    assert torch.equal(torch.nan_to_num(want.float()), torch.nan_to_num(got.float()))
    assert bool((got[1] == 0).all()) and not bool(torch.isnan(got[3, 1].float()).any())


# ---- write and read ---------------------------------------------------------------------------------------------
def _check_rows(oracle, caches, slots, k, v, rule, mbs):
    for cache, is_key, x in ((caches[0], True, k), (caches[1], False, v)):
        want = ref.quantized_rows(oracle, x, rule, mbs)
        for name, g, w in zip(("codes", "scales", "words"), ref.cached_rows(cache, is_key, slots), want):
            assert (g is None and w is None) or np.array_equal(g, w), (name, is_key)


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("mbs", [True, False])
@pytest.mark.parametrize("rule, page, T", [("oas", 16, 9), ("ocp", 64, 1), ("floor", 128, 130)])
def test_write_and_read(mx, oracle, D, mbs, rule, page, T):
    H = 3
    pages = T // page + 3
    caches = _filled_cache(mx, D, pages, H, D, page, mbs)
    before = _copy(caches)
    kv = _rows(D + T, T, 2 * H, D)
    k, v = kv[:, :H], kv[:, H:]
    if T > 4:
        k[2, 1, 40] = float("inf")
        v[3, 0, 3] = float("nan")
        k[1], v[4] = 0, -0.0
        k[3] *= 1e-30
        v[1] *= 2e36
    rng = np.random.default_rng(T)
    slots = rng.permutation(pages * page)[:T]
    if T > 8:
        slots[5], slots[7], slots[8] = -1, pages * page, 1 << 40  # outside: not written, not read
    ok = (slots >= 0) & (slots < pages * page)
    s = torch.from_numpy(slots).cuda()
    mx.mx_kv_write(k, v, s, *caches, rule)
    _check_rows(oracle, caches, slots[ok], k[ok], v[ok], rule, mbs)
    # and nothing else has changed
    for cache, old, is_key in ((caches[0], before[0], True), (caches[1], before[1], False)):
        others = np.setdiff1d(np.arange(pages * page), slots[ok])
        for a, b in zip(ref.cached_rows(cache, is_key, others), ref.cached_rows(old, is_key, others)):
            assert a is None or np.array_equal(a, b)
    for name, dtype in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        out = torch.full((2, T, H, D), 3.0, dtype=dtype, device="cuda")
        mx.mx_kv_read(s, *caches, name, k_out=out[0], v_out=out[1])
        for got, cache, is_key in ((out[0], caches[0], True), (out[1], caches[1], False)):
            want = torch.from_numpy(ref.values(*ref.cached_rows(cache, is_key, slots[ok]))).float().to(dtype)
            assert torch.equal(torch.nan_to_num(got[ok].cpu().float(), nan=-5.0), torch.nan_to_num(want.float(), nan=-5.0)), (name, is_key)
            assert bool((got[~ok] == 3.0).all())


def test_strided_rows_out_and_one_array_only(mx):
    """Outputs whose rows lie apart, and the C call that reads keys or values by themselves."""
    T, Hq, H, D, page = 9, 3, 2, 128, 4096
    caches = mx.mx_kv_cache(2, H, D, page)
    q, k, v = _rows(1, T, Hq, D), _rows(2, T, H, D), _rows(3, T, H, D)
    slots = torch.tensor([0, 4095, 4096, 8191, 17, 18, 19, 20, 5000], device="cuda")
    mx.mx_kv_write(k, v, slots, *caches)
    want = mx.mx_kv_read(slots, *caches)
    out = torch.full((T, 2 * H + 1, D), 3.0, dtype=torch.bfloat16, device="cuda")
    mx.mx_kv_read(slots, *caches, k_out=out[:, :H], v_out=out[:, H:2 * H])
    assert torch.equal(out[:, :H], want[0]) and torch.equal(out[:, H:2 * H], want[1]) and bool((out[:, 2 * H] == 3.0).all())
    for is_key in (True, False):
        one = torch.full((T, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
        at = [one.data_ptr() if is_key else None, H * D, None if is_key else one.data_ptr(), H * D]
        arrays = [a.data_ptr() for cache in caches for a in cache]
        assert mx.load_library().mx_kv_read(slots.data_ptr(), *arrays, 2, page, T, H, D, mx.MX_OUT_BF16, *at, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(one, want[0 if is_key else 1])
    table, positions = _cos_sin(16, D), torch.arange(T, device="cuda").int()
    turned = mx.mx_qk_norm_rope(q, k, positions, table)
    out = torch.full((T, Hq + H + 1, D), 3.0, dtype=torch.bfloat16, device="cuda")
    mx.mx_qk_norm_rope(q, k, positions, table, q_out=out[:, :Hq], k_out=out[:, Hq:Hq + H])
    assert torch.equal(out[:, :Hq], turned[0]) and torch.equal(out[:, Hq:Hq + H], turned[1]) and bool((out[:, Hq + H] == 3.0).all())


def test_write_equals_the_quantizer(mx):
    """The same bits as mx_quantize_mbs on the rows of a head."""
    T, H, D, page = 50, 4, 128, 32
    caches = mx.mx_kv_cache(3, H, D, page)
    k, v = _rows(1, T, H, D), _rows(2, T, H, D)
    slots = torch.arange(T, device="cuda") + 7
    mx.mx_kv_write(k, v, slots, *caches)
    for x, cache, is_key in ((k, caches[0], True), (v, caches[1], False)):
        want = mx.mx_quantize_mbs(x.reshape(T * H, D), "oas")
        for a, b in zip(ref.cached_rows(cache, is_key, slots.cpu().numpy()), want):
            assert np.array_equal(a.reshape(T * H, -1), b.cpu().numpy())
        back = mx.mx_dequantize(*want, "bf16")
        assert torch.equal(mx.mx_kv_read(slots, *caches)[0 if is_key else 1].reshape(T * H, D), back)


@pytest.mark.parametrize("D, style, norm, R, mbs, T, Hq, Hkv", [
    (128, "half", True, 128, True, 37, 8, 2), (64, "pairs", True, 64, False, 5, 3, 3), (96, "half", False, 48, True, 11, 4, 1), (256, "half", True, 128, True, 3, 2, 2),
    (192, "pairs", True, 96, True, 9, 2, 1), (128, "half", True, 0, True, 4, 2, 2), (128, "half", True, 128, True, 2100, 12, 4)])
def test_fused_write_is_the_two_calls(mx, D, style, norm, R, mbs, T, Hq, Hkv):
    page = 16
    pages = T // page + 2
    one, two = (_filled_cache(mx, 5, pages, Hkv, D, page, mbs) for _ in range(2))
    qkv = _rows(D + T, T, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    w = torch.linspace(0.5, 1.7, D, device="cuda").to(torch.bfloat16) if norm else None
    table = _cos_sin(T + 5, R) if R else None
    positions = torch.arange(T, device="cuda").int() + 1
    slots = torch.randperm(pages * page, generator=_gen(T), device="cuda")[:T]
    positions[T // 2] = T + 9  # beyond the table: NaN, stored as NaN blocks
    slots[1] = -1
    q_two, k_two = mx.mx_qk_norm_rope(q, k, positions, table, w, w, 1e-6, style)
    mx.mx_kv_write(k_two, v, slots, *two)
    q_one = mx.mx_qk_norm_rope_kv_write(q, k, v, positions, slots, table, *one, w, w, 1e-6, style)
    assert np.array_equal(ref.bits(q_one), ref.bits(q_two)) and _same(one, two)
    # a padding token is left out
    if R:
        positions[0] = -1
        again = _copy(one)
        q_out = torch.full_like(q_one, 9.0)
        mx.mx_qk_norm_rope_kv_write(q, k * 3, v * 3, positions, torch.where(torch.arange(T, device="cuda") == 0, slots, -1), table, *again, w, w, 1e-6, style,
                                    q_out=q_out)
        assert _same(again, one) and bool((q_out[0] == 9.0).all()) and not bool((q_out[1] == 9.0).all())


@pytest.mark.parametrize("T, Hq, Hkv, D", [(1500, 5, 3, 128), (3001, 5, 3, 128), (9000, 5, 7, 64), (700, 3, 5, 256), (12001, 5, 9, 128)])
def test_heads_that_a_wavefront_takes_in_part(mx, oracle, T, Hq, Hkv, D):
    """Sizes at which wavefronts take two, four and eight heads, none of them a divisor of the heads: norm and rotation, the write with and without them,
    the read."""
    page = 64
    pages = T // page + 2
    one, two = (_filled_cache(mx, 5, pages, Hkv, D, page, True) for _ in range(2))
    qkv = _rows(D + T, T, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    w = torch.linspace(0.5, 1.7, D, device="cuda").to(torch.bfloat16)
    table, positions = _cos_sin(T, D), torch.arange(T, device="cuda").int()
    slots = torch.randperm(pages * page, generator=_gen(T), device="cuda")[:T]
    q_two, k_two = mx.mx_qk_norm_rope(q, k, positions, table, w, w)
    some = torch.cat((torch.arange(70), torch.arange(T - 70, T)))
    for x, y in ((q, q_two), (k, k_two)):
        assert np.array_equal(ref.bits(ref.to_bf16(ref.norm_rope(x[some], positions[some], table, w, 1e-6, "half"))), ref.bits(y[some]))
    mx.mx_kv_write(k_two, v, slots, *two)
    q_one = mx.mx_qk_norm_rope_kv_write(q, k, v, positions, slots, table, *one, w, w)
    assert np.array_equal(ref.bits(q_one), ref.bits(q_two)) and _same(one, two)
    _check_rows(oracle, two, slots.cpu().numpy(), k_two, v, "oas", True)
    for got, cache, is_key in zip(mx.mx_kv_read(slots, *two), two, (True, False)):
        want = torch.from_numpy(ref.values(*ref.cached_rows(cache, is_key, slots.cpu().numpy()))).float().to(torch.bfloat16)
        assert torch.equal(got.cpu(), want)


def test_rows_on_another_stream_and_in_a_graph(mx):
    """Captured once and replayed over changed inputs, with eager work between the replays."""
    T, Hq, Hkv, D, page = 19, 4, 2, 128, 16
    caches = mx.mx_kv_cache(4, Hkv, D, page)
    qkv = _rows(1, T, Hq + 2 * Hkv, D)
    table, positions, slots = _cos_sin(64, D), torch.arange(T, device="cuda").int(), torch.arange(T, device="cuda")
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    q_out, outs = torch.empty_like(qkv[:, :Hq]).contiguous(), torch.empty((2, T, Hkv, D), dtype=torch.bfloat16, device="cuda")

    def work():
        mx.mx_qk_norm_rope_kv_write(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], positions, slots, table, *caches, w, w, q_out=q_out)
        mx.mx_kv_read(slots, *caches, k_out=outs[0], v_out=outs[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in (2, 3, 4):
        qkv.copy_(_rows(seed, T, Hq + 2 * Hkv, D))
        graph.replay()
        got = q_out.clone(), outs.clone()
        q_out.zero_()
        outs.zero_()
        work()
        torch.cuda.synchronize()
        assert torch.equal(got[0], q_out) and torch.equal(got[1], outs)


def test_refused_on_the_gpu(mx):
    k_cache, v_cache = mx.mx_kv_cache(2, 2, 128, 16)
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(3, device="cuda")
    for bad in (lambda: mx.mx_kv_write(x.float(), x, slots, k_cache, v_cache), lambda: mx.mx_kv_write(x, x, slots.int(), k_cache, v_cache),
                lambda: mx.mx_kv_write(x, x, slots[:2], k_cache, v_cache), lambda: mx.mx_kv_write(x, x, slots.cpu(), k_cache, v_cache),
                lambda: mx.mx_kv_write(x, x, slots, k_cache[:2] + (None,), v_cache), lambda: mx.mx_kv_write(x[..., :64], x[..., :64], slots, k_cache, v_cache),
                lambda: mx.mx_kv_write(x, x.transpose(1, 2).contiguous().transpose(1, 2), slots, k_cache, v_cache),
                lambda: mx.mx_kv_write(x, x, slots, (k_cache[0][:, :, :, :8],) + k_cache[1:], v_cache),
                lambda: mx.mx_kv_read(slots, k_cache, v_cache, "bf16", k_out=torch.empty((3, 2, 128), device="cuda")),
                lambda: mx.mx_qk_norm_rope(x, x[:2], slots.int(), torch.zeros((4, 128), device="cuda")),
                lambda: mx.mx_qk_norm_rope(x, x, slots.int(), torch.zeros((4, 24), device="cuda"))):
        with pytest.raises((TypeError, ValueError, mx.MxError)):
            bad()


# ---- the two ways through the binding ---------------------------------------------------------------------------
def _calls(mx):
    """name -> (call with all outputs given, what it writes)"""
    T, Hq, Hkv, D, page = 21, 4, 2, 128, 16
    qkv = _rows(3, T, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    one, two = mx.mx_kv_cache(3, Hkv, D, page), mx.mx_kv_cache(3, Hkv, D, page, use_mbs=False)
    table, positions, slots = _cos_sin(64, D), torch.arange(T, device="cuda").int(), torch.arange(T, device="cuda")
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    qo, ko, qf, kr, vr, out, lse = new(T, Hq, D), new(T, Hkv, D), new(T, Hq, D), new(T, Hkv, D), new(T, Hkv, D), new(T, Hq, D), new(T, Hq, dtype=torch.float32)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    blocks, plan = i32(0, 1, 2).reshape(1, 3), (new(2, dtype=torch.int64), i32(0), new(30, dtype=torch.int64), new(30, dtype=torch.int32), i32(0))
    arrays = lambda *caches: tuple(a for c in caches for a in c if a is not None)  # noqa: E731
    return {
        "kv_plan": (lambda: mx.mx_kv_plan(i32(20), i32(9), page, blocks, i32(5, 6), i32(0), 30, *plan), plan + (blocks,)),
        "qk_norm_rope": (lambda: mx.mx_qk_norm_rope(q, k, positions, table, w, None, q_out=qo, k_out=ko), (qo, ko)),
        "kv_write": (lambda: mx.mx_kv_write(k, v, slots, *two), arrays(*two)),
        "qk_norm_rope_kv_write": (lambda: mx.mx_qk_norm_rope_kv_write(q, k, v, positions, slots, table, *one, w, w, q_out=qf), arrays(*one) + (qf,)),
        "kv_read": (lambda: mx.mx_kv_read(slots, *one, k_out=kr, v_out=vr), (kr, vr)),
        "attention_kv": (lambda: mx.mx_attention_kv(qf, torch.tensor([0, T], device="cuda"), i32(T), i32(0, 1, 2).reshape(1, 3), *one, out=out, lse=lse), (out, lse)),
    }


def test_native_and_ctypes_marshalling_agree(mx, monkeypatch):
    native = mx.binding._native
    assert native is not None, "the build step makes _marshal.so"
    served = []

    class Recorder:
        def __getattr__(self, name):
            def call(*a):
                status = getattr(native, name)(*a)
                served.append((name, status))
                return status
            return call

    got = []
    for used in (Recorder(), None):
        monkeypatch.setattr(mx.binding, "_native", used)
        results = {}
        for name, (call, outputs) in _calls(mx).items():
            call()
            results[name] = [o.clone() for o in outputs]
        got.append(results)
    assert served == [(name, 0) for name in got[0]]
    for name in got[0]:
        assert all(torch.equal(a, b) for a, b in zip(got[0][name], got[1][name])), name
        assert any(bool((a != 0).any()) for a in got[0][name]), name


def test_native_marshalling_declines_what_the_binding_refuses(mx):
    native = mx.binding._native
    kc, vc = mx.mx_kv_cache(2, 2, 128, 16)
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    slots, lens, off = torch.arange(3, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    table = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    attend = lambda **k: native.attention_kv(*dict(dict(q=x, off=off, lens=lens, table=table, a=kc[0], b=kc[1], c=kc[2], d=vc[0], e=vc[1], f=vc[2], scale=1.0,  # noqa: E731
                                                        causal=True, window=0, out=x.clone(), lse=None, work=None), **k).values())
    assert attend() == 0 and attend(window=-1) == -1 and attend(work=torch.empty(0, dtype=torch.uint8, device="cuda")) == -1
    assert attend(q=x.float()) is None and attend(off=off[:1]) is None and attend(out=x[:2]) is None and attend(c=None) is None and attend(scale=1) is None
    assert attend(table=table.long()) is None and attend(lse=torch.zeros(3, 2)) is None and attend(a=kc[0].cpu()) is None
    assert native.kv_write(x, x, slots, *kc, *vc, "oas") == 0 and native.kv_write(x, x, slots, *kc, *vc, "best") is None
    assert native.kv_write(x, x[:, :1], slots, *kc, *vc, "oas") is None and native.kv_write(x, x, slots, *vc, *kc, "oas") is None
    assert native.kv_read(slots, *kc, *vc, "bf16", x.clone(), x.clone().float()) is None
    assert native.qk_norm_rope(x, x, None, torch.zeros((4, 128), device="cuda"), None, None, 1e-6, "half", x.clone(), x.clone()) is None


def test_attention_under_dispatch_modes(mx):
    """A mode of the caller's sees the workspace being allocated: one that hands on what it sees changes nothing, one that gives a tensor without memory
    is an exception."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    from torch.utils._python_dispatch import TorchDispatchMode

    class Passes(TorchDispatchMode):
        seen = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            Passes.seen += 1
            return func(*args, **(kwargs or {}))

    caches = mx.mx_kv_cache(2, 2, 128, 16)
    x = _rows(1, 3, 2, 128)
    mx.mx_kv_write(x, x, torch.arange(3, device="cuda"), *caches)
    off, lens = torch.tensor([0, 3], device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")
    table = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    want, out = mx.mx_attention_kv(x, off, lens, table, *caches), torch.zeros_like(x)
    with Passes():
        mx.mx_attention_kv(x, off, lens, table, *caches, out=out)
    assert Passes.seen and torch.equal(out, want)
    out.zero_()
    with pytest.raises((RuntimeError, TypeError, ValueError)):
        with FakeTensorMode(allow_non_fake_inputs=True):
            mx.mx_attention_kv(x, off, lens, table, *caches, out=out)
    assert not bool(out.any())
