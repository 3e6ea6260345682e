"""Routing among experts on the GPU: the plan's whole numbers exactly and its weights within fp32, the combination within its roundings, and a layer as it is used."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import block128_reference as ref  # noqa: E402


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


def same_plan(logits, k, scoring, bias, renormalize, got, scale=1.0, num_tokens=None):
    want = ref.plan(logits, k, scoring, bias, renormalize, scale, num_tokens)
    for name, a, b in zip(("experts", None, "row_offsets", "rows", "tokens"), got, want):
        if name:
            assert np.array_equal(a.cpu().numpy(), b), name
    w, exact = got[1].cpu().double().numpy(), want[1]
    assert np.array_equal(np.isnan(w), np.isnan(exact))
    # softmax: differences of logits are rounded (2^-24 of them, in numerator and sum), two exponentials of an ulp each, at most 22 additions, a division and a
    # product; sigmoid: in fp64, rounded once, `scale` being fp32 already
    finite = logits[torch.isfinite(logits)].double()
    spread = float(finite.max() - finite.min()) if finite.numel() else 0.0
    tolerance = (2 * spread + 32) * 2.0 ** -24 if scoring == "softmax" else 2.0 ** -23
    ok = ~np.isnan(exact)
    # (an exponential below the smallest normal number is off by up to 2^-149)
    assert np.all(np.abs(w - exact)[ok] <= tolerance * np.abs(exact)[ok] + 2.0 ** -148)


CASES = [(1, 1, 1), (1, 8, 2), (5, 4, 4), (64, 32, 4), (128, 60, 6), (129, 64, 8), (130, 65, 3), (300, 128, 8), (1000, 160, 6), (513, 256, 8), (40, 500, 32), (200, 512, 5), (64, 1000, 7),
         (150, 1024, 32), (9000, 16, 2)]


@pytest.mark.parametrize("T, E, k", CASES)
@pytest.mark.parametrize("scoring, with_bias", [("softmax", False), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("dtype, renormalize", [(torch.bfloat16, True), (torch.float32, False)])
def test_plan(mx, T, E, k, scoring, with_bias, dtype, renormalize):
    g = generator(T + E + k)
    logits = (2 * torch.randn((T, E), generator=g, device="cuda")).to(dtype)
    bias = 0.3 * torch.randn(E, generator=g, device="cuda") if with_bias else None
    same_plan(logits, k, scoring, bias, renormalize, mx.mx_moe_plan(logits, k, scoring, bias, renormalize, 2.5), float(np.float32(2.5)))


@pytest.mark.parametrize("T", [3, 100, 400])
@pytest.mark.parametrize("scoring, with_bias", [("softmax", False), ("sigmoid", False), ("sigmoid", True)])
def test_plan_ties_masks_and_what_is_not_finite(mx, T, scoring, with_bias):
    g = generator(T)
    E, k = 70, 5
    inf, nan = float("inf"), float("nan")
    logits = torch.randint(-2, 3, (T, E), generator=g, device="cuda").float()  # many equal ones
    logits[torch.rand((T, E), generator=g, device="cuda") < 0.2] = -0.0
    logits[0] = -inf  # no expert at all
    logits[1, 3:] = -inf  # fewer than k
    logits[2, 7] = nan
    if T > 3:
        logits[3, 9] = inf
        logits[4, 1], logits[4, 60] = inf, inf
        logits[5] = 1.0
        logits[6, :68] = -inf
        logits[7, 5], logits[7, 6] = nan, nan
        logits[8] = -300.0 - torch.arange(E, device="cuda")  # far below 0, all of them
    bias = torch.where(torch.arange(E, device="cuda") % 9 == 0, -inf, torch.randint(0, 2, (E,), generator=g, device="cuda").float()) if with_bias else None
    for renormalize in (False, True):
        same_plan(logits, k, scoring, bias, renormalize, mx.mx_moe_plan(logits, k, scoring, bias, renormalize))


@pytest.mark.parametrize("T", [7, 90, 777])
def test_plan_of_a_padded_batch(mx, T):
    logits = torch.randn((T, 20), generator=generator(1), device="cuda")
    for n in (0, 1, T // 2, T, T + 5, -3):
        logits[max(n, 0):] = float("nan")  # not read
        outputs = dict(experts=torch.full((T, 3), 9, dtype=torch.int32, device="cuda"), tokens=torch.full((T * 3,), 9, dtype=torch.int32, device="cuda"))
        got = mx.mx_moe_plan(logits, 3, num_tokens=torch.tensor([n], device="cuda"), **outputs)
        assert got[0] is outputs["experts"] and got[4] is outputs["tokens"]
        same_plan(logits, 3, "softmax", None, True, got, num_tokens=n)
        logits = torch.randn((T, 20), generator=generator(1), device="cuda")


def test_plan_of_strided_logits_and_none(mx):
    wide = torch.randn((300, 41), generator=generator(2), device="cuda").to(torch.bfloat16)
    same_plan(wide[:, 3:36], 4, "softmax", None, True, mx.mx_moe_plan(wide[:, 3:36], 4))
    for T in (0,):
        got = mx.mx_moe_plan(wide[:T, :9], 2)
        assert got[0].shape == (0, 2) and bool((got[2] == 0).all())


def test_plan_of_many_tokens(mx):
    """Chunks of 1024 tokens, more than 256 of them."""
    T, E, k = 300_001, 24, 2
    logits = torch.randn((T, E), generator=generator(3), device="cuda")
    experts, weights, offsets, rows, tokens = mx.mx_moe_plan(logits, k)
    chosen = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(experts.long(), chosen)
    order = torch.sort(chosen.flatten(), stable=True).indices
    assert torch.equal(tokens.long(), order // k)
    assert torch.equal(rows.flatten().long()[order], torch.arange(T * k, device="cuda"))
    assert torch.equal(offsets[1:], torch.bincount(chosen.flatten(), minlength=E).cumsum(0))


def test_plan_of_many_tokens_among_the_most_experts(mx):
    """2^19 and some tokens, 1024 experts: the largest tables in LDS."""
    T, E = (1 << 19) + 77, 1024
    chosen = torch.randint(0, E, (T, 1), generator=generator(4), device="cuda")
    chosen[5000:9000] = 1023
    logits = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda").scatter_(1, chosen, 8.0)
    experts, weights, offsets, rows, tokens = mx.mx_moe_plan(logits, 1, "sigmoid", torch.zeros(E, device="cuda"))
    assert torch.equal(experts.long(), chosen) and bool((weights == 1.0).all())
    order = torch.sort(chosen.flatten(), stable=True).indices
    assert torch.equal(tokens.long(), order)
    assert torch.equal(rows.flatten().long()[order], torch.arange(T, device="cuda"))
    assert torch.equal(offsets[1:], torch.bincount(chosen.flatten(), minlength=E).cumsum(0))


@pytest.mark.parametrize("T", [100, 1000])
def test_plan_writes_its_outputs_only(mx, T):
    E, k = 33, 4
    logits = torch.randn((T, E), generator=generator(9), device="cuda")
    need = mx.mx_moe_plan_workspace(T, E, k)
    sizes = dict(experts=(torch.int32, (T, k)), weights=(torch.float32, (T, k)), row_offsets=(torch.int64, (E + 1,)), rows=(torch.int32, (T, k)),
                 tokens=(torch.int32, (T * k,)), workspace=(torch.uint8, (need,)))
    guarded, inside = {}, {}
    for name, (dtype, shape) in sizes.items():
        n = int(np.prod(shape))
        guarded[name] = torch.full((n + 16,), 77, dtype=dtype, device="cuda")
        inside[name] = guarded[name][8:8 + n].view(shape)
    got = mx.mx_moe_plan(logits, k, **inside)
    same_plan(logits, k, "softmax", None, True, got)
    for name, t in guarded.items():
        assert bool((t[:8] == 77).all()) and bool((t[-8:] == 77).all()), name


# ---- combination ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T, k, N", [(1, 1, 8), (3, 2, 13), (64, 4, 2880), (9, 8, 2049), (130, 5, 4104), (2, 0, 40), (5, 33, 256)])
@pytest.mark.parametrize("y_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out, with_add", [("bf16", False), ("bf16", True), ("f32", True)])
def test_combine(mx, T, k, N, y_type, out, with_add):
    g = generator(T + k + N)
    R = T * k + 2
    out_type = torch.bfloat16 if out == "bf16" else torch.float32
    y = torch.randn((R, N), generator=g, device="cuda").to(y_type)
    rows = torch.randint(0, R, (T, k), generator=g, device="cuda").int()
    weights = torch.randn((T, k), generator=g, device="cuda")
    if k > 1:
        rows[0, 1], rows[-1, 0], rows[T // 2, k - 1] = -1, R, 1 << 30  # no such rows: left out, whatever their weights
        weights[0, 1], weights[-1, 0] = float("nan"), float("inf")
    y[0 if k else slice(0, 0)] = y[0 if k else slice(0, 0)]
    add = torch.randn((T, N), generator=g, device="cuda").to(out_type) if with_add else None
    got = mx.mx_moe_combine(y, rows, weights, add, out).double()
    there = (rows >= 0) & (rows < R)
    w = torch.where(there, weights, 0.0).double()
    parts = w[..., None] * y[torch.where(there, rows, 0).long()].double()
    want = parts.sum(1) + (add.double() if with_add else 0.0)
    size = parts.abs().sum(1) + (add.double().abs() if with_add else 0.0)
    # each multiply-add rounds once, by 2^-24 of a partial sum (at most `size`, and what went before)
    off = size * (k + 1) * 2.0 ** -24 * 1.001
    off = off + (want.abs() + off) * (2.0 ** -8 if out == "bf16" else 2.0 ** -24)
    assert bool(((got - want).abs() <= off).all())
    if add is not None:
        here = mx.mx_moe_combine(y, rows, weights, add, out, out=add)
        assert here is add and torch.equal(here.double(), got)


def test_combine_of_other_alignments(mx):
    g = generator(7)
    T, k, N = 6, 3, 64
    for shift, pad in ((0, 0), (1, 0), (0, 1), (8, 8), (4, 3)):
        def matrix(rows, dtype):
            ld = N + pad
            return torch.randn(shift + rows * ld + 8, generator=g, device="cuda").to(dtype)[shift:shift + rows * ld].view(rows, ld)[:, :N]

        y, add = matrix(T * k, torch.bfloat16), matrix(T, torch.bfloat16)
        buffer = torch.full((shift + T * (N + pad) + 8,), 77.0, dtype=torch.bfloat16, device="cuda")
        out = buffer[shift:shift + T * (N + pad)].view(T, N + pad)[:, :N]
        rows = torch.randperm(T * k, generator=g, device="cuda").view(T, k).int()
        weights = torch.rand((T, k), generator=g, device="cuda")
        mx.mx_moe_combine(y, rows, weights, add, "bf16", out=out)
        whole = mx.mx_moe_combine(y.contiguous(), rows, weights, add.contiguous(), "bf16")
        assert torch.equal(out, whole)
        out.fill_(77.0)
        assert bool((buffer == 77.0).all())


# ---- a layer ------------------------------------------------------------------------------------------------------------
class Layer:
    """Router, two projections an expert, and what every token keeps; all buffers of a captured step made once."""

    def __init__(self, mx, E, dim, hidden, k, seed):
        g = generator(seed)
        weight = lambda n, m: (torch.randn((n, m), generator=g, device="cuda") * m ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.mx, self.E, self.dim, self.hidden, self.k = mx, E, dim, hidden, k
        self.router = weight(E, dim)
        self.up = mx.mx_quantize_block128(weight(E * 2 * hidden, dim), "e4m3", 128, E)
        self.down = mx.mx_quantize_block128(weight(E * dim, hidden), "e4m3", 128, E)

    def __call__(self, x, num_tokens=None):
        mx = self.mx
        logits = x @ self.router.T
        experts, weights, offsets, rows, tokens = mx.mx_moe_plan(logits, self.k, num_tokens=num_tokens)
        a = mx.mx_quantize_block128(x)
        both = mx.mx_gemm_block128_grouped("e4m3", *a, "e4m3", *self.up, offsets, 2 * self.hidden, "bf16", a_rows=tokens,
                                           out=torch.zeros((tokens.numel(), 2 * self.hidden), dtype=torch.bfloat16, device="cuda"))
        act = torch.nn.functional.silu(both[:, :self.hidden]) * both[:, self.hidden:]
        h = mx.mx_quantize_block128(act)
        y = mx.mx_gemm_block128_grouped("e4m3", *h, "e4m3", *self.down, offsets, self.dim, "bf16")
        return dict(logits=logits, experts=experts, weights=weights, offsets=offsets, rows=rows, tokens=tokens, a=a, both=both, act=act, h=h, y=y,
                    out=mx.mx_moe_combine(y, rows, weights, x, "bf16"))


@pytest.mark.parametrize("T, n", [(1, 1), (48, 40), (700, 700)])
def test_a_layer_step_by_step(mx, T, n):
    E, dim, hidden, k = 12, 272, 400, 3
    layer = Layer(mx, E, dim, hidden, k, 11)
    x = torch.randn((T, dim), generator=generator(12), device="cuda").to(torch.bfloat16)
    s = layer(x, torch.tensor([n], device="cuda"))
    same_plan(s["logits"], k, "softmax", None, True, (s["experts"], s["weights"], s["offsets"], s["rows"], s["tokens"]), num_tokens=n)
    offsets = s["offsets"].tolist()
    assert offsets[-1] == n * k
    for name, q, rows, weight, N, out in (("up", s["a"], s["tokens"].long(), layer.up, 2 * hidden, s["both"]),
                                          ("down", s["h"], torch.arange(T * k, device="cuda"), layer.down, dim, s["y"])):
        a = ref.values(*q, 1, "e4m3")
        for e in range(E):
            at = slice(offsets[e], offsets[e + 1])
            b = ref.values(weight[0][e * N:(e + 1) * N], weight[1][e * ref.blocks(N):(e + 1) * ref.blocks(N)], 128, "e4m3")
            want, size = ref.product(a[rows[at]], b)
            assert bool(((out[at].double() - want).abs() <= ref.product_bound(want, size, a.shape[1], True)).all()), (name, e)
    codes, scales = ref.quantize(s["act"], 1, "e4m3")
    assert torch.equal(s["h"][0].cpu(), codes) and torch.equal(s["h"][1].cpu(), scales)
    want, size = x.double(), x.double().abs()
    for j in range(k):
        there = s["rows"][:, j:j + 1] >= 0
        part = torch.where(there, s["weights"][:, j:j + 1].double() * s["y"][s["rows"][:, j].clamp_min(0).long()].double(), 0.0)
        want, size = want + part, size + part.abs()
    off = size * (k + 1) * 2.0 ** -23
    assert bool(((s["out"].double() - want).abs() <= off + (want.abs() + off) * 2.0 ** -8).all())
    assert torch.equal(s["out"][n:], x[n:])  # padding goes through


def test_the_plan_serves_the_mxfp4_experts_too(mx):
    T, E, k, dim, N = 200, 8, 2, 256, 96
    g = generator(21)
    x = torch.randn((T, dim), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((E * N, dim), generator=g, device="cuda") * 0.06).to(torch.bfloat16)
    _, weights, offsets, rows, tokens = mx.mx_moe_plan(torch.randn((T, E), generator=g, device="cuda"), k)
    qa, qw = mx.mx_quantize_mbs(x[tokens.long()], "oas"), mx.mx_quantize_mbs(w, "oas")
    y = mx.mx_gemm_mbs_grouped(*qa, *qw, offsets, N, "f32")
    out = mx.mx_moe_combine(y, rows, weights, out_dtype="f32")
    a, b = mx.mx_dequantize(*qa, "f32").double(), mx.mx_dequantize(*qw, "f32").double().view(E, N, dim)
    of_row = torch.bucketize(torch.arange(T * k, device="cuda"), offsets[1:], right=True)
    exact = torch.stack([b[e] @ a[r] for r, e in enumerate(of_row.tolist())])
    want = (weights.double()[..., None] * exact[rows.long()]).sum(1)
    assert float((out.double() - want).abs().max()) <= 1e-3 * float(exact.square().mean().sqrt())  # the grouped product's own bound


@pytest.mark.parametrize("T", [64, 300])
def test_a_captured_step(mx, T):
    """The step replayed with other tokens, with eager work between: every replay gives what the eager step gives."""
    layer = Layer(mx, 16, 256, 384, 4, 31)
    x, n = torch.zeros((T, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    inputs = [(torch.randn((T, 256), generator=generator(40 + i), device="cuda").to(torch.bfloat16), m) for i, m in enumerate((T, T // 2, 1, 0, T - 3))]
    x.copy_(inputs[0][0])
    n.fill_(T)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            layer(x, n)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = layer(x, n)
    for round_ in range(2):
        for tokens, m in inputs:
            x.copy_(tokens)
            n.fill_(m)
            graph.replay()
            torch.cuda.synchronize()
            eager = layer(x, n)
            torch.cuda.synchronize()
            for name in ("experts", "weights", "offsets", "rows", "tokens", "both", "out"):
                assert torch.equal(made[name], eager[name]), (round_, m, name)


def test_two_streams_at_once(mx):
    """Calls with buffers of their own on two streams, over and over: the same results as one after the other."""
    layers = [Layer(mx, 16, 256, 384, 4, s) for s in (51, 52)]
    xs = [torch.randn((500, 256), generator=generator(60 + i), device="cuda").to(torch.bfloat16) for i in range(2)]
    want = [layer(x)["out"] for layer, x in zip(layers, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(layers[i](xs[i])["out"])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


# ---- scores that fp64 holds no longer ---------------------------------------------------------------------------------------
def renormalized_sigmoid(logits, experts, scale=1.0):
    """score / sum of the chosen scores, by the scores' logarithms: log(1 / (1 + exp(-x))) = -log(1 + exp(-x)), which far below 0 is x itself."""
    x = logits.cpu().double().numpy()
    e = experts.cpu().numpy()
    log = -np.logaddexp(0.0, -np.take_along_axis(x, np.maximum(e, 0).astype(np.int64), 1))
    log = np.where(e >= 0, log, -np.inf)
    w = np.exp(log - log.max(1, keepdims=True))
    return np.where(e >= 0, w / w.sum(1, keepdims=True) * scale, 0.0)


@pytest.mark.parametrize("T, E, k", [(16, 20, 5), (16, 70, 5), (100, 500, 20), (200, 33, 18), (700, 128, 8), (300, 1000, 32)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_plan_shares_scores_of_logits_far_below_zero(mx, T, E, k, with_bias, dtype):
    """Finite logits whose scores are 0 in 64 bits (or have lost bits there): divided by their sum they are exp(logit - largest), still."""
    g = generator(T + E + k)
    low = torch.finfo(dtype).min
    logits = torch.empty((T, E), device="cuda").uniform_(-820.0, -380.0, generator=g)
    few = torch.rand((T, E), generator=g, device="cuda") * 3
    logits[0] = -1e4
    logits[1] = low
    logits[2] = -1e9
    logits[2, 3:5] = -1e9 + 4096
    logits[3] = low
    logits[3, 11] = -2000.0  # the only one that counts
    logits[4] = -1e4 + 0 * few[4]
    logits[4, :3] = float("-inf")
    logits[5] = -745.0 - few[5]
    logits[6] = -708.0 - few[6]
    logits[7] = -500.0 - 60 * few[7]
    logits[8] = -485.0 - few[8]
    logits[9] = low
    logits[9, 2] = 3.0
    logits[10] = -1e17
    logits[11, 1:] = float("-inf")  # one expert, of no score
    logits[11, 0] = -5000.0
    logits[12] = -90.0 - 30 * few[12]
    logits = logits.to(dtype)
    bias = torch.randn(E, generator=g, device="cuda") if with_bias else None
    scale = 2.5
    experts, weights, offsets, rows, tokens = mx.mx_moe_plan(logits, k, "sigmoid", bias, True, scale)
    want = renormalized_sigmoid(logits, experts, scale)
    w = weights.cpu().double().numpy()
    assert not np.isnan(want).any()
    # fp64 up to here, whose exponentials of differences up to 2^10 are off by 2^-42; rounded to 32 bits once (half of 2^-149 below the normal numbers)
    assert np.all(np.abs(w - want) <= 2.0 ** -23 * want + 2.0 ** -149)
    # the choices, places and counts go by the logits as before
    same = ref.plan(logits, k, "sigmoid", bias, False)
    for a, b in ((experts, same[0]), (offsets, same[2]), (rows, same[3]), (tokens, same[4])):
        assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("T, E", [(3, 20), (3, 70), (100, 70), (700, 70), (200, 300)])
def test_plan_never_takes_an_expert_of_bias_minus_infinity(mx, T, E):
    """Not even where its logit is NaN or +inf: the plan is that of logits which are -inf there."""
    k = 6
    logits = torch.randn((T, E), generator=generator(T + E), device="cuda")
    bias = torch.randn(E, generator=generator(E), device="cuda")
    out = torch.arange(E, device="cuda") % 4 == 1
    bias[out] = float("-inf")
    logits[0, out] = float("nan")
    logits[1, 5], logits[2, 1] = float("nan"), float("inf")
    masked = logits.masked_fill(out, float("-inf"))
    for renormalize in (True, False):
        got = mx.mx_moe_plan(logits, k, "sigmoid", bias, renormalize)
        assert not bool(torch.isnan(got[1]).any())
        for a, b in zip(got, mx.mx_moe_plan(masked, k, "sigmoid", bias, renormalize)):
            assert torch.equal(a, b)
        same_plan(masked, k, "sigmoid", bias, renormalize, got)


@pytest.mark.parametrize("T, E", [(8, 24), (8, 100), (500, 100), (500, 300)])
def test_plan_scores_that_have_run_into_one_tie(mx, T, E):
    """Scores of 1 in 64 bits, and scores that the bias drowns, are equal whatever their logits: the lowest index is taken."""
    g = generator(E)
    far = torch.tensor([45.0, 40.0, 60.0, 3e4, float("inf")], device="cuda")
    logits = far[torch.randint(0, 5, (T, E), generator=g, device="cuda")]
    logits[T // 2:] = -far[torch.randint(0, 4, (T - T // 2, E), generator=g, device="cuda")]
    bias = torch.where(torch.arange(E, device="cuda") % 3 == 0, 0.25, 0.5)
    got = mx.mx_moe_plan(logits, 5, "sigmoid", bias, False)
    assert torch.equal(got[0], torch.tensor([1, 2, 4, 5, 7], dtype=torch.int32, device="cuda").expand(T, 5))
    same_plan(logits, 5, "sigmoid", bias, False, got)
