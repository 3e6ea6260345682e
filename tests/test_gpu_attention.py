"""Attention over the paged MXFP4 cache against a plain 64-bit implementation (tests/kv_reference.py derives the tolerances)."""
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["few rows", "many rows"])
def mx(request):
    """Every test with either kernel: which of them a call takes goes by its sizes."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2603_08713_amd as mx_

    mx_.load_library()
    with mx_.forced(attention=1 if request.param == "few rows" else 2):
        yield mx_


class Batch:
    """Requests of n[s] queries on keys[s] keys over a cache whose unused bytes hold anything."""

    def __init__(self, mx, seed, n, keys, Hq, Hkv, D, page, mbs, spread=1.0, width=0, wide=0):
        self.mx = mx
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        need = [-(-max(0, L) // page) for L in keys]
        pages = sum(need) + 2
        order = rng.permutation(pages).astype(np.int32)
        table = rng.integers(-5, 2 * pages, (len(n), max([1, width] + need) + 1)).astype(np.int32)  # unused entries hold anything
        at = 0
        for s, c in enumerate(need):
            table[s, :c] = order[at:at + c]
            at += c
        self.table = torch.from_numpy(table).cuda()
        self.caches = tuple(tuple(None if a is None else torch.randint(0, 256, a.shape, generator=g, device="cuda", dtype=torch.uint8) for a in c)
                            for c in mx.mx_kv_cache(pages, Hkv, D, page, mbs))
        slots = np.concatenate([table[s, np.arange(L) // page].astype(np.int64) * page + np.arange(L) % page for s, L in enumerate(keys)] + [np.zeros(0, np.int64)])
        self.slots = slots
        rows = torch.randn((len(slots), 2 * Hkv, D), generator=g, device="cuda")
        rows[:, :Hkv, D // 5] *= 8
        rows = rows.to(torch.bfloat16)
        if len(slots):
            mx.mx_kv_write(rows[:, :Hkv], rows[:, Hkv:], torch.from_numpy(slots).cuda(), *self.caches)
        self.offsets = torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int64, device="cuda")
        self.lens = torch.tensor(list(keys), dtype=torch.int32, device="cuda")
        T = int(sum(n)) + wide  # rows behind the last request
        self.q = (torch.randn((T, Hq + 1, D), generator=g, device="cuda") * spread).to(torch.bfloat16)[:, :Hq]  # strided
        self.page = page

    def run(self, **how):
        T, Hq, D = self.q.shape
        out = torch.full((T, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((T, Hq), 6.0, device="cuda")
        self.mx.mx_attention_kv(self.q, self.offsets, self.lens, self.table, *self.caches, out=out, lse=lse, **how)
        return out, lse

    def check(self, scale=None, causal=True, window=0):
        out, lse = self.run(scale=scale, causal=causal, window=window)
        scale = self.q.shape[2] ** -0.5 if scale is None else scale
        want, want_lse, tol, tol_lse, written = ref.attention(self.q, self.offsets, self.lens, self.table, *self.caches, scale, causal, window)
        assert bool((out[~written] == 5.0).all()) and bool((lse[~written] == 6.0).all()), "rows behind the last request"
        got, got_lse = out.cpu().double().numpy()[written], lse.cpu().double().numpy()[written]
        want, want_lse, tol, tol_lse = want[written], want_lse[written], tol[written], tol_lse[written]
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse)), "NaN"
        assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse)), "rows without keys"
        assert (got[np.isneginf(want_lse)] == 0).all()
        fine = ~np.isnan(want)
        off = np.abs(got - want)[fine] - tol[fine]
        assert not off.size or off.max() <= 0, "off by %g more than %g" % (off.max(), tol[fine][off.argmax()])
        fine = np.isfinite(want_lse)
        off = np.abs(got_lse[fine] - want_lse[fine]) - tol_lse[fine]
        assert not off.size or off.max() <= 0, "lse off by %g more than %g" % (off.max(), tol_lse[fine][off.argmax()])
        return out, lse


# one token each: lengths around the sizes of pages, subtiles, tiles and pieces
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("mbs", [True, False])
@pytest.mark.parametrize("Hq, Hkv, page", [(8, 2, 16), (3, 3, 64), (20, 1, 32), (24, 8, 128)])
def test_single_tokens(mx, D, mbs, Hq, Hkv, page):
    keys = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 255, 256, 257, 300]
    Batch(mx, D + Hq, [1] * len(keys), keys, Hq, Hkv, D, page, mbs).check()


@pytest.mark.parametrize("D, page, mbs", [(128, 64, True), (64, 16, False), (96, 32, True), (256, 128, True)])
@pytest.mark.parametrize("L", [1000, 4097, 9000])
def test_long_contexts_are_cut(mx, D, page, mbs, L):
    Batch(mx, L, [1, 1], [L, 3], 8, 2, D, page, mbs).check()
    Batch(mx, L + 1, [3, 2], [L, L // 3], 4, 1, D, page, mbs).check()


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("mbs", [True, False])
@pytest.mark.parametrize("window", [0, 1, 40, 64])
def test_several_tokens_and_prompts(mx, D, mbs, window):
    # whole prompts, chunks behind a context, a request without rows, one without keys, more queries than keys
    Batch(mx, D + window, [70, 5, 0, 33, 9, 130], [70, 200, 50, 33, 4, 131], 6, 2, D, 16, mbs, wide=3).check(window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_all_keys(mx, D):
    Batch(mx, D, [40, 1, 7], [33, 190, 0], 4, 2, D, 32, True).check(causal=False)


@pytest.mark.parametrize("n, keys", [([1], [0]), ([1, 1, 1], [0, 0, 0]), ([4], [1]), ([100], [20]), ([0, 0], [5, 6]), ([1, 0, 1], [64, 64, 0])])
def test_rows_without_keys(mx, n, keys):
    b = Batch(mx, 1, n, keys, 8, 2, 128, 16, True, wide=2)
    b.check()
    b.check(window=3)
    b.check(causal=False)


def test_more_requests_than_lanes(mx):
    """Batches that a wavefront looks through 64 requests at a time, some of them without rows or keys, the lengths in no order."""
    rng = np.random.default_rng(40)
    for S, most, rows in ((64, 90, 2), (65, 40, 3), (200, 130, 2), (389, 20, 4)):
        n = [int(x) for x in rng.integers(0, rows + 1, S)]
        keys = [int(x) if rng.random() > 0.1 else 0 for x in rng.integers(1, most, S)]
        n[S // 2], keys[S // 2] = 70, 200
        Batch(mx, S, n, keys, 4, 2, 64, 16, True, wide=1).check()


@pytest.mark.parametrize("Hq, Hkv, D, page", [(128, 1, 64, 16), (96, 2, 128, 32), (7, 7, 256, 16), (5, 1, 192, 4096), (4, 2, 96, 4096)])
def test_many_heads_and_large_pages(mx, Hq, Hkv, D, page):
    """One key head for all queries, as many as queries, key heads by an odd number of queries; pages of 4096."""
    Batch(mx, Hq, [1, 9, 3], [150, 40, 70], Hq, Hkv, D, page, True).check()
    Batch(mx, Hq + 1, [30], [200], Hq, Hkv, D, page, False).check(window=50)


@pytest.mark.parametrize("window", [299, 300, 301, (1 << 30) - 1, 1 << 31, 1 << 40, (1 << 62)])
def test_windows_as_long_as_the_keys(mx, window):
    b = Batch(mx, 41, [1, 20, 5], [300, 300, 3], 4, 2, 128, 16, True)
    out, lse = b.check(window=window)
    if window >= 300:
        want, want_lse = b.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("n, keys", [([1, 1], [2000, 20]), ([50, 3], [70, 900])])
def test_strided_outputs(mx, D, n, keys):
    """Rows of the output apart from each other, with and without lse: the same bits, and nothing beside them."""
    b = Batch(mx, 42, n, keys, 4, 2, D, 16, True)
    want, _ = b.run()
    T, Hq, _ = want.shape
    for wide in (1, 3):
        out = torch.full((T + 1, Hq + wide, D), 9.0, dtype=torch.bfloat16, device="cuda")
        mx.mx_attention_kv(b.q, b.offsets, b.lens, b.table, *b.caches, out=out[:T, :Hq])
        assert torch.equal(out[:T, :Hq], want) and bool((out[:, Hq:] == 9.0).all()) and bool((out[T] == 9.0).all())


def test_large_scores_and_scales(mx):
    """Scores far apart: one key takes all of a row, and the running maximum moves often."""
    for spread, scale in ((30.0, None), (1.0, 5.0), (1e-3, None), (2.0, -0.3), (1.0, 0.0)):
        Batch(mx, 3, [1, 20], [500, 300], 8, 2, 128, 64, True, spread=spread).check(scale=scale)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("mbs", [True, False])
def test_values_as_large_as_they_may_be(mx, D, mbs):
    """|v| kv_lens of 2^118.2 of the 2^119 that are allowed, under the largest weights: 64 keys at score 0 and the others 7.9 powers of two above them,
    which is just too little for the running maximum to follow (300 2^7.9 2^110 = 2^126.1 in the sums)."""
    b = Batch(mx, 24, [1, 40, 2], [300, 300, 299], 4, 2, D, 16, mbs)
    H = 2
    rows = torch.zeros((len(b.slots), 2 * H, D), dtype=torch.bfloat16, device="cuda")
    j = torch.cat([torch.arange(L, device="cuda") for L in (300, 300, 299)])
    rows[:, :H, 0] = torch.where(j < 64, 0.0, 4.0)[:, None].to(torch.bfloat16)
    sign = torch.where(torch.arange(D, device="cuda") % 3 == 0, -1.0, 1.0)
    rows[:, H:] = (2.0 ** 110 * sign).to(torch.bfloat16)
    b.mx.mx_kv_write(rows[:, :H], rows[:, H:], torch.from_numpy(b.slots).cuda(), *b.caches)
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    out, _ = b.check(scale=7.9 * np.log(2.0) / 4.0)
    assert bool((out[:43].float() == 2.0 ** 110 * sign).all())


def test_missing_pages(mx):
    """Pages outside the cache hold no keys, and lengths beyond the table end with it."""
    b = Batch(mx, 4, [1, 30, 2, 1], [200, 150, 90, 40], 4, 2, 128, 16, True)
    pages = b.caches[0][1].shape[0]
    b.table[0, 3], b.table[0, 7] = -1, pages
    b.table[1, 0], b.table[1, 9] = 1 << 30, -(1 << 31)
    b.table[3, :] = -7
    b.check()
    b.check(window=33)
    b.lens[2] = 100000
    b.table[2, :] = b.table[2, 0]
    b.check()
    b.lens[:] = torch.tensor([-5, 2147483647, 0, -2147483648], dtype=torch.int32)
    b.run()  # (nothing to compare: positions of the second request are far beyond its keys)
    torch.cuda.synchronize()


def test_offsets_that_make_no_sense_stay_inside(mx):
    """Row offsets that run backwards, overlap or leave the tensor: no access outside, whatever the results."""
    b = Batch(mx, 5, [3, 4, 5, 6], [300, 20, 500, 70], 4, 2, 128, 16, True)
    for offsets in ([0, 18, 0, 18, 0], [5, 3, 2, 1, 0], [-9, -1, 1000, 1 << 40, -(1 << 62)], [0, 18, 18, 18, 18], [17, 1 << 62, 0, 4, 5]):
        b.offsets.copy_(torch.tensor(offsets, dtype=torch.int64))
        b.run()
        torch.cuda.synchronize()


def _slot(b, s, j):
    return int(b.table[s, j // b.page]), j % b.page


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("mbs", [True, False])
def test_nan_goes_where_it_is_seen(mx, D, mbs):
    """NaN blocks of keys and of values: in the rows that see them and in no other, whatever tile they share."""
    n, keys = [40, 1, 3], [40, 100, 70]
    b = Batch(mx, 6, n, keys, 4, 2, D, 16, mbs)
    clean, _ = b.run()
    p, at = _slot(b, 0, 30)
    b.caches[1][1][p, 1, D // 32 - 1, at] = 255   # value of key 30, head 1, last block
    p, at = _slot(b, 1, 77)
    b.caches[0][1][p, 0, 0, at] = 255             # key 77, head 0
    p, at = _slot(b, 2, 69)
    b.caches[1][1][p, 0, 0, at] = 255             # value that only the last query sees
    out, _ = b.check()
    nan = torch.isnan(out.float())
    assert not bool(nan[:30].any()) and bool(nan[30:40, 2:, D - 32:].all()) and not bool(nan[30:40, :2].any()) and not bool(nan[30:40, 2:, :D - 32].any())
    assert bool(nan[40, :2].all()) and not bool(nan[40, 2:].any())
    assert not bool(nan[41:43].any()) and bool(nan[43, :2, :32].all()) and not bool(nan[43, 2:].any())
    assert torch.equal(out[:30], clean[:30]) and torch.equal(out[41:43], clean[41:43])
    b.check(causal=False)
    b.check(window=7)


def test_nan_and_infinity_in_queries(mx):
    b = Batch(mx, 7, [1, 30], [100, 64], 4, 2, 128, 16, True)
    b.q[0, 1, 5] = float("nan")
    b.q[9, 2, 7] = float("inf")
    out, lse = b.run()
    nan = torch.isnan(out.float()).all(-1)
    assert bool(nan[0, 1]) and bool(nan[9, 2]) and int(nan.sum()) == 2 and int(torch.isnan(lse).sum()) == 2
    assert int(torch.isnan(out.float()).sum()) == 2 * 128


def _all_minus(b, dtype=torch.bfloat16):
    """Rewrites every key of the cache's requests as -1 in each element."""
    H, D = b.caches[0][1].shape[1], b.q.shape[2]
    rows = torch.full((len(b.slots), H, D), -1.0, dtype=dtype, device="cuda")
    v = torch.randn((len(b.slots), H, D), device="cuda").to(dtype)
    b.mx.mx_kv_write(rows, v, torch.from_numpy(b.slots).cuda(), *b.caches)


@pytest.mark.parametrize("D, mbs", [(64, True), (96, False), (128, True), (192, True), (256, False)])
@pytest.mark.parametrize("n, keys", [([1], [1]), ([1, 3, 2], [5000, 70, 0]), ([70, 5, 40], [70, 900, 12])])
def test_rows_whose_scores_are_all_minus_infinity(mx, D, mbs, n, keys):
    """exp(-inf - -inf): such a row is NaN, as its formula says, and not what a row without keys gets - whole rows and rows whose keys are cut,
    the same queries before their request's first key (zeros, -inf), and rows beside them."""
    b = Batch(mx, D, n, keys, 4, 2, D, 16, mbs)
    _all_minus(b)
    b.q.zero_()
    b.q[:, 1, 3] = float("inf")
    b.q[::2, 2, D - 1] = float("inf")
    out, lse = b.check()
    sees = ~torch.isneginf(lse[:, 0])
    assert bool(torch.isnan(out[sees, 1].float()).all()) and bool(torch.isnan(lse[sees, 1]).all()) and not bool(torch.isnan(out[:, 0].float()).any())
    b.check(window=3)
    b.check(causal=False)
    b.check(scale=-0.5)  # (+inf - +inf: NaN as well)


def test_minus_infinity_and_missing_pages(mx):
    """Whether such a row sees a key goes by the pages that exist: some, one in the middle, none."""
    n, keys = [1, 2, 30, 1], [3000, 200, 40, 500]
    b = Batch(mx, 21, n, keys, 4, 2, 128, 16, True)
    _all_minus(b)
    b.q.zero_()
    b.q[:, :, 0] = float("inf")
    pages = b.caches[0][1].shape[0]
    b.table[0, :] = -1
    b.table[1, :12] = pages  # (only the page of the last 8 keys is there)
    b.table[2, 1] = -7
    b.table[3, :9], b.table[3, 10:] = -1, 1 << 30  # (one page, between two tiles' borders)
    out, lse = b.check()
    assert bool((out[0] == 0).all()) and bool(torch.isneginf(lse[0]).all()) and bool(torch.isnan(out[1:].float()).all())
    b.check(window=5)
    b.check(causal=False)


def test_a_page_used_twice_and_a_shared_prefix(mx):
    """Requests that share pages, and a page that stands in a table twice."""
    b = Batch(mx, 8, [1, 2, 5], [150, 150, 150], 4, 2, 128, 16, True)
    b.table[1, :6] = b.table[0, :6]
    b.table[2, 3] = b.table[2, 1]
    b.check()


def test_results_do_not_depend_on_the_batch(mx):
    """A request alone and among others: within the tolerance of either, and twice the same call the same bits."""
    b = Batch(mx, 9, [1] * 9, [5000, 1, 77, 3000, 0, 64, 900, 2, 333], 8, 2, 128, 64, True)
    one, lse = b.check()
    again, lse_again = b.run()
    assert torch.equal(one, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("mbs", [True, False])
def test_nan_as_the_cache_write_stores_it(mx, D, mbs):
    """NaN and infinity in rows that mx_kv_write quantizes (scale byte 255 over codes that are all 0), of keys and of values, in tiles that every
    row sees whole and in tiles that a mask or a request's end cuts."""
    n, keys = [1, 40, 3], [300, 300, 333]
    b = Batch(mx, 22, n, keys, 4, 2, D, 16, mbs)
    at = np.cumsum([0] + keys)
    H = 2
    x = torch.randn((7, 2 * H, D), device="cuda").to(torch.bfloat16)
    x[0, 0, 5] = float("nan")           # request 0: key 20, head 0, the first block: a whole tile
    x[1, H + 1, D - 1] = float("-inf")  # request 0: value of key 130, head 1, the last block: a whole tile
    x[2, H, 33] = float("inf")          # request 0: value of key 299, head 0, the second block: the request's last tile
    x[3, H, 0] = float("nan")           # request 1: value of key 70, head 0: a whole tile for all of its rows
    x[4, H + 1, 40] = float("inf")      # request 1: value of key 290, which the last ten rows see
    x[5, 1, D - 2] = float("inf")       # request 1: key 295, head 1, which the last five rows see
    x[6, 1, 1] = float("nan")           # request 2: key 64, head 1
    where = [20, 130, 299, at[1] + 70, at[1] + 290, at[1] + 295, at[2] + 64]
    places = b.slots[where]
    b.mx.mx_kv_write(x[:, :H], x[:, H:], torch.from_numpy(places).cuda(), *b.caches)
    for cache, is_key, row, head, block in ((b.caches[0], True, 0, 0, 0), (b.caches[1], False, 2, 0, 1)):
        codes, scales, _ = ref.cached_rows(cache, is_key, places)
        assert scales[row, head, block] == 255 and not codes[row, head, 16 * block:16 * block + 16].any()
    out, lse = b.check()
    nan = torch.isnan(out.float())
    assert bool(nan[0, :2].all()) and bool(nan[0, 2:, D - 32:].all()) and not bool(nan[0, 2:, :D - 32].any())
    assert bool(nan[1:41, :2, :32].all()) and not bool(nan[1:41, :2, 32:].any()) and not bool(nan[1:31, 2:].any()) and bool(nan[36:41, 2:].all())
    assert not bool(nan[41:, :2].any()) and bool(nan[41:, 2:].all()) and bool(torch.isnan(lse[41:, 2:]).all())
    b.check(causal=False)
    b.check(window=100)


@pytest.mark.parametrize("n, keys", [([1] * 9, [5000, 1, 77, 3000, 0, 64, 900, 2, 333]), ([3, 130, 1, 20], [4000, 130, 77, 500])])
def test_each_request_alone(mx, n, keys):
    """A request of a batch by itself: its own rows, lengths and row of the table, within the tolerance as it is among others."""
    b = Batch(mx, 9, n, keys, 8, 2, 128, 64, True)
    b.check()
    q, offsets, lens, table = b.q, b.offsets.tolist(), b.lens, b.table
    for s in range(len(n)):
        b.q, b.offsets, b.lens, b.table = q[offsets[s]:offsets[s + 1]], torch.tensor([0, n[s]], device="cuda"), lens[s:s + 1], table[s:s + 1]
        b.check()


@pytest.mark.parametrize("n, keys", [([1, 1], [3000, 20]), ([50, 3], [70, 900])])
def test_workspaces_streams_and_graphs(mx, n, keys):
    """A caller's workspace with anything in it; another stream; captured and replayed over changed lengths and queries."""
    b = Batch(mx, 10, n, keys, 8, 2, 128, 16, True)
    T, Hq, D = b.q.shape
    want = b.check()
    size = mx.mx_attention_kv_workspace(len(n), T, Hq, 2, D)
    work = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    got = b.run(workspace=work[:size])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((work[size:] == 0xFF).all())
    if size:
        with pytest.raises(mx.binding.MxError):
            b.run(workspace=work[:size - 16])
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])

    def call():
        mx.mx_attention_kv(b.q, b.offsets, b.lens, b.table, *b.caches, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for cut in (0, 1, 17):
        b.lens.copy_(torch.tensor([max(0, L - cut) for L in keys], dtype=torch.int32))
        b.q.mul_(0.9)
        graph.replay()
        got = out.clone(), lse.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)


def test_a_serving_loop(mx, oracle):
    """Prompts, then single tokens: plan, norm and rotation with the cache write, attention, step after step from the GPU's own arrays, against the
    same steps in 64 bits on the rows that were stored."""
    S, Hq, Hkv, D, page, width = 3, 6, 2, 128, 16, 6
    k_cache, v_cache = mx.mx_kv_cache(12, Hkv, D, page)
    table = torch.full((S, width), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(12, device="cuda").int()
    lens, start = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    angle = torch.arange(128, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    cos_sin = torch.cat((angle.cos(), angle.sin()), -1).float().cuda()
    w = torch.linspace(0.6, 1.4, D, device="cuda").to(torch.bfloat16)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ctx = np.zeros(S, np.int64)
    for step, new in enumerate(([20, 7, 33], [1, 1, 1], [1, 0, 1], [2, 9, 1], [1, 1, 1])):
        T = sum(new) + 2  # a padded batch
        qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        n = torch.tensor(new, dtype=torch.int32, device="cuda")
        offsets, lens, slots, positions, start = mx.mx_kv_plan(lens, n, page, table, free, start, T)
        rotated = mx.mx_qk_norm_rope_kv_write(q, k, v, positions, slots, cos_sin, k_cache, v_cache, w, w)
        out = torch.full((T, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
        mx.mx_attention_kv(rotated, offsets, lens, table, k_cache, v_cache, out=out)
        ctx += np.array(new)
        assert np.array_equal(lens.cpu().numpy(), ctx) and start.item() == sum(-(-int(c) // page) for c in ctx)
        live = sum(new)
        assert bool((slots[live:] == -1).all()) and bool((out[live:] == 5.0).all())
        want_q = ref.to_bf16(ref.norm_rope(q[:live], positions[:live], cos_sin, w, 1e-6, "half"))
        want_k = ref.to_bf16(ref.norm_rope(k[:live], positions[:live], cos_sin, w, 1e-6, "half"))
        assert np.array_equal(ref.bits(rotated[:live]), ref.bits(want_q))
        places = slots[:live].cpu().numpy()
        for cache, is_key, x in ((k_cache, True, want_k), (v_cache, False, v[:live])):
            for a, b in zip(ref.cached_rows(cache, is_key, places), ref.quantized_rows(oracle, x, "oas", True)):
                assert np.array_equal(a, b)
        want, _, tol, _, written = ref.attention(rotated, offsets, lens, table, k_cache, v_cache, D ** -0.5, True, 0)
        assert written[:live].all() and not written[live:].any()
        assert (np.abs(out.cpu().double().numpy() - want) <= tol)[written].all()


def test_a_captured_serving_step(mx):
    """The serving step that the README shows, captured once and replayed step after step with the program's own eager work between the replays, against
    the same lines run eagerly on a cache of their own."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    once, step = next(b for b in text.split("```")[1::2] if "mx_kv_plan" in b).removeprefix("python").split("# a step:")
    once, step = compile(once, "README", "exec"), compile("#" + step, "README", "exec")
    S, Hq, Hkv, D, page, width, T = 3, 6, 2, 128, 16, 6, 45
    angle = torch.arange(128, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    w = torch.linspace(0.6, 1.4, D, device="cuda").to(torch.bfloat16)
    qkv = torch.zeros((T, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
    given = dict(torch=torch, mx=mx, num_pages=15, kv_heads=Hkv, head_dim=D, page_size=page, S=S, T=T, q_weight=w, k_weight=w,
                 cos_sin=torch.cat((angle.cos(), angle.sin()), -1).float().cuda(), free_pages=torch.randperm(15, device="cuda").int(),
                 new=torch.zeros(S, dtype=torch.int32, device="cuda"))

    def server():
        names = dict(given, block_table=torch.full((S, width), -1, dtype=torch.int32, device="cuda"))
        exec(once, names)
        return names

    def run(names):
        names.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:])
        exec(step, names)

    captured, eager = server(), server()
    run(captured)  # (no tokens yet: what a first call sets up)
    lens, start = captured["lens"], captured["start"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(captured)
    g = torch.Generator(device="cuda")
    g.manual_seed(31)
    ctx = np.zeros(S, np.int64)
    for tokens in ([20, 7, 13], [1, 1, 1], [1, 0, 1], [2, 9, 1], [1, 1, 1], [0, 0, 0], [30, 1, 1]):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        given["new"].copy_(torch.tensor(tokens, dtype=torch.int32))
        graph.replay()
        run(eager)
        torch.cuda.synchronize()
        ctx += np.array(tokens)
        live = sum(tokens)
        for name in ("lens", "start", "slots", "positions", "block_table"):
            assert torch.equal(captured[name], eager[name]), (name, tokens)
        assert np.array_equal(lens.cpu().numpy(), ctx) and start.item() == sum(-(-int(c) // page) for c in ctx)
        assert torch.equal(captured["out"][:live], eager["out"][:live])
        assert all(torch.equal(x, y) for name in ("k_cache", "v_cache") for x, y in zip(captured[name], eager[name]))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("ones, prompts", [([300, 1, 4000, 17], [(200, 200), (64, 700)]), ([5000], [(530, 530)])])
def test_prompts_and_single_tokens_by_two_calls(mx, D, ones, prompts):
    """A step of both kinds: one call for all, and a call for the requests of each kind into one output; the rows of the other kind stay as they are."""
    n, keys = [1] * len(ones) + [p[0] for p in prompts], ones + [p[1] for p in prompts]
    b = Batch(mx, 23 + D, n, keys, 8, 2, D, 32, True, wide=2)
    b.check()
    q, offsets, lens, table, k = b.q, b.offsets, b.lens, b.table, len(ones)
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    mx.mx_attention_kv(q[:k], offsets[:k + 1], lens[:k], table[:k], *b.caches, out=out[:k])
    assert bool((out[k:] == 5.0).all())
    first = out[:k].clone()
    mx.mx_attention_kv(q, offsets[k:], lens[k:], table[k:], *b.caches, out=out)
    assert torch.equal(out[:k], first) and bool((out[-2:] == 5.0).all())
    want, _, tol, _, written = ref.attention(q, offsets, lens, table, *b.caches, D ** -0.5, True, 0)
    assert (np.abs(out.cpu().double().numpy() - want) <= tol)[written].all()


@pytest.mark.parametrize("n, keys, many", [([128], [128], True), ([128], [700], True), ([512, 30, 600], [512, 900, 1000], True), ([100], [100], False),
                                           ([1] * 40, list(range(1, 400, 10)), False), ([3, 200], [4000, 300], False)])
def test_the_kernel_that_a_call_takes(n, keys, many):
    """Without a choice by the caller: the same bits as from the kernel that the sizes ask for, within the tolerance."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2603_08713_amd as mx

    b = Batch(mx, 11, n, keys, 32, 8, 128, 32, True, wide=1)
    out, lse = b.check()
    with mx.forced(attention=2 if many else 1):
        again, lse_again = b.run()
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


def test_a_cache_beyond_4_gib(mx):
    """Codes of more than 2^32 bytes an array: the same rows in the first and in the last pages give the same bits."""
    Hq, Hkv, D, page = 16, 4, 128, 64
    pages = (5 << 30) // (Hkv * page * D // 2)
    caches = mx.mx_kv_cache(pages, Hkv, D, page)
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    keys, n = 333, 70
    used = -(-keys // page)
    rows = torch.randn((keys, 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn((n, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    offsets, lens = torch.tensor([0, n], device="cuda"), torch.tensor([keys], dtype=torch.int32, device="cuda")
    j = torch.arange(keys, device="cuda")
    results = []
    for first in (0, pages - used):
        table = torch.arange(first, first + used, dtype=torch.int32, device="cuda")[None, :].contiguous()
        slots = first * page + j
        mx.mx_kv_write(rows[:, :Hkv], rows[:, Hkv:], slots, *caches)
        results.append((mx.mx_attention_kv(q, offsets, lens, table, *caches),) + tuple(mx.mx_kv_read(slots, *caches)))
    for low, high in zip(*results):
        assert torch.equal(low, high)


def test_refused_before_a_launch(mx):
    """A workspace of one byte that says it has many, queries that the key heads do not divide, a cache without heads."""
    b = Batch(mx, 13, [1, 2], [70, 20], 4, 2, 128, 16, True)
    size = mx.mx_attention_kv_workspace(2, 3, 4, 2, 128)
    one = torch.zeros(1, dtype=torch.uint8, device="cuda")
    for workspace in (one.expand(size + 1), torch.zeros((size + 1, 2), dtype=torch.uint8, device="cuda")[:, 0], one.cpu()):
        with pytest.raises(TypeError):
            b.run(workspace=workspace)
    b.q = b.q[:, :3]
    with pytest.raises(ValueError):
        b.run()
    with pytest.raises(ValueError):
        mx.mx_attention_kv(b.q, b.offsets, b.lens, b.table, *mx.mx_kv_cache(2, 0, 128, 16))


def test_a_million_tokens_at_once(mx):
    """2^26 rows: the last of them against the same rows in a call of their own size; the kernel for few rows refuses them."""
    T, Hq, Hkv, D, page, window, last = 1 << 20, 64, 8, 64, 16, 16, 300
    g = torch.Generator(device="cuda")
    g.manual_seed(14)
    caches = mx.mx_kv_cache(T // page, Hkv, D, page)
    table = torch.randperm(T // page, generator=g, device="cuda").int()[None, :].contiguous()
    used = -(-(last + window) // page)  # pages that the last rows see
    slots = (table[0, -used:].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()
    rows = torch.randn((used * page, 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    mx.mx_kv_write(rows[:, :Hkv], rows[:, Hkv:], slots, *caches)
    q = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets = torch.tensor([0, T], device="cuda")
    if mx.binding._forced("attention") == 1:
        with pytest.raises(mx.binding.MxError):
            mx.mx_attention_kv(q, offsets, i32(T), table, *caches, window=window)
        return
    out = mx.mx_attention_kv(q, offsets, i32(T), table, *caches, window=window)[T - last:]
    want, _, tol, _, _ = ref.attention(q[T - last:], torch.tensor([0, last], device="cuda"), i32(used * page), table[:, -used:], *caches, D ** -0.5, True, window)
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()


def test_as_many_rows_as_one_launch_holds(mx):
    """2^26 - 4 rows on pages that stand in the table again and again: rows of the beginning, the middle and the end."""
    if mx.binding._forced("attention") == 2:
        pytest.skip("the limit of the kernel for few rows")
    T, Hq, D, page, window, pages = (1 << 24) - 1, 4, 64, 16, 16, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(15)
    caches = mx.mx_kv_cache(pages, Hq, D, page)
    rows = torch.randn((pages * page, 2 * Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    mx.mx_kv_write(rows[:, :Hq], rows[:, Hq:], torch.arange(pages * page, device="cuda"), *caches)
    table = torch.randint(0, pages, (1, -(-T // page)), generator=g, device="cuda").int()
    q = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    out = mx.mx_attention_kv(q, torch.tensor([0, T], device="cuda"), lens, table, *caches, window=window)
    for end in (100, T // 2 // page * page, T):
        first = max(0, (end - 200) // page * page)
        n = end - max(first + window, 0) if first else end
        want, _, tol, _, _ = ref.attention(q[end - n:end], torch.tensor([0, n], device="cuda"), lens.fill_(end - first), table[:, first // page:-(-end // page)], *caches,
                                           D ** -0.5, True, window)
        assert (np.abs(out[end - n:end].cpu().double().numpy() - want) <= tol).all()
