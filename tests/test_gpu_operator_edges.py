"""The embedding, the linear cross entropy and the gradient norm at values that a mask, a loss scale or an overflow
brings along.  Bounds as in test_gpu_operators.py, by element: a score that is far from all others counts for nothing, so its
own error does not either."""
import math

import pytest
import torch

from test_gpu_operators import E, TINY, TYPES, gen, half_step, picks, tokens_for, within

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min


@pytest.fixture(scope="module")
def hd(lib):
    h = lib.Handle(0)
    yield h
    h.close()


def masked_reference(x, w, tokens):
    """Loss, lse, gx, gw of the sum of losses in 64 bits and their bounds, for weights of any size and infinite ones."""
    D, V = x.shape[1], w.shape[0]
    u, tiny, terms = half_step(x.dtype), TINY[x.dtype], 6 if x.dtype == torch.float32 else 1
    kept = 0.0 if x.dtype == torch.float32 else u
    has, at = picks(tokens, V)
    X, W = x.double(), w.double()
    z = X @ W.t()
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    # a score's own error, where its probability is not zero (then z is finite and no further than 800 from lse)
    dz = torch.where(p > 0, (D + 8) * E * (X.abs() @ W.abs().t()), 0.0)
    span = torch.where(p > 0, (z - lse[:, None]).abs(), 0.0).amax(1).clamp(max=100.0)
    dlse = 2 * (p * dz).sum(1) + (3 * span + 4 + V ** 0.5 + 300) * E + 2 * E * lse.abs()
    rows = torch.arange(len(at), device="cuda")
    loss = lse - z[rows, at]
    dloss = torch.where(torch.isfinite(loss), dz[rows, at] + dlse + E * loss.abs(), 0.0)
    dp = p * ((dz + dlse[:, None]) + (3 * span[:, None] + 6 + lse.abs()[:, None]) * E)
    p[rows, at] -= 1.0
    G = p * has[:, None]
    dG = (dp + (kept + 3 * E) * G.abs()) * has[:, None]
    low = 2.0 ** -38 if x.dtype == torch.float16 else 0.0
    dG = dG + torch.where(G == 0, 0.0, low)
    gx, gw = G @ W, G.t() @ X
    dgx = dG @ W.abs() + (terms * V + 80) * E * (G.abs() @ W.abs())
    dgw = dG.t() @ X.abs() + (terms * len(at) + 80) * E * (G.abs().t() @ X.abs())
    return {"loss": (loss * has, dloss), "lse": (lse * has, dlse), "gx": (gx, dgx + u * (gx.abs() + dgx) + tiny), "gw": (gw, dgw + u * (gw.abs() + dgw) + tiny)}


def masked(g, N, D, V, value, gated, dtype=torch.float32):
    """Feature 0 is a gate, 1 or (every third row, where `gated`) 0; `value` in its weights masks every fifth class."""
    x, w = torch.randn(N, D, generator=g, device="cuda"), torch.randn(V, D, generator=g, device="cuda")
    x[:, 0] = 1.0
    if gated:
        x[::3, 0] = 0.0
    w[1::5, 0] = value
    tokens = tokens_for(g, (N,), V // 5) * 5                 # (classes that are not masked; -500 stands for none as well)
    return x.to(dtype), w.to(dtype), tokens


@pytest.mark.parametrize("N,D,V", [(9, 40, 130), (300, 40, 130), (300, 37, 130), (1500, 200, 1000)])
@pytest.mark.parametrize("value,gated", [(-math.inf, False), (LOWEST, True), (LOWEST, False), (-1e30, True), (-1e9, True), (-1e5, True)])
def test_fp32_classes_masked_by_a_weight(hd, N, D, V, value, gated):
    x, w, tokens = masked(gen(N + D), N, D, V, value, gated)
    ref = masked_reference(x, w, tokens)
    loss, lse = hd.xent_fprop(x, w, tokens)
    within(loss, *ref["loss"], "loss")
    within(lse, *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    within(gw, *ref["gw"], "gw")
    first = 0 if value >= -1e30 else 1                       # (0 times an infinite weight is not a number)
    within(gx[:, first:], ref["gx"][0][:, first:], ref["gx"][1][:, first:], "gx")


@pytest.mark.parametrize("dtype", TYPES[1:], ids=["bf16", "f16"])
@pytest.mark.parametrize("N", [6, 300])
@pytest.mark.parametrize("value", [-math.inf, "lowest"])
def test_16_bit_classes_masked_by_a_weight(hd, N, value, dtype):
    value = torch.finfo(dtype).min if value == "lowest" else value
    x, w, tokens = masked(gen(N), N, 40, 130, value, False, dtype)
    # (six rows: what the rounding of G leaves is taken along; this bound holds for both)
    ref = masked_reference(x, w, tokens)
    loss, lse = hd.xent_fprop(x, w, tokens)
    within(loss, *ref["loss"], "loss")
    within(lse, *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    within(gw, *ref["gw"], "gw")
    within(gx[:, 1:], ref["gx"][0][:, 1:], ref["gx"][1][:, 1:], "gx")


@pytest.mark.parametrize("N", [9, 300])
@pytest.mark.parametrize("size", [1e8, 1e15, 1e30])
def test_fp32_feature_that_meets_zero_weights(hd, N, size):
    """One feature far above the others, whose weights are zero: the others are what they are without it."""
    g = gen(60)
    x, w = torch.randn(N, 48, generator=g, device="cuda"), torch.randn(200, 48, generator=g, device="cuda")
    x[:, 5], w[:, 5] = size, 0.0
    tokens = tokens_for(g, (N,), 200)
    ref = masked_reference(x, w, tokens)
    loss, lse = hd.xent_fprop(x, w, tokens)
    within(loss, *ref["loss"], "loss")
    within(lse, *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    within(gx, *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")


@pytest.mark.parametrize("N", [5, 300])
@pytest.mark.parametrize("D", [1, 3, 4])
def test_fp32_scores_of_few_features(hd, N, D):
    """Scores are fp32 products: with one feature a loss is off by the rounding of a product, not of its factors."""
    g = gen(61)
    x, w = torch.randn(N, D, generator=g, device="cuda") * 8, torch.randn(2, D, generator=g, device="cuda") * 8
    w[1] = 0.0                                               # lse and loss follow one score each
    tokens = torch.ones(N, dtype=torch.int64, device="cuda")
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    _, lse = hd.xent_fprop(x, w, tokens)
    # D products and sums of half a step each; the smaller exponential, (3 t + 4) e of exp(-t), and the logarithm, 8 e; the
    # sum of the larger score and the logarithm, and the result
    bound = D * E * (x.double().abs() @ w.double().abs().t()).amax(1) + 8 * E + 2 * E * want.abs()
    within(lse, want, bound, "lse")


def within_or_beyond(got, ref, bound, what):
    """Where the bound reaches past fp32's largest value, 2^128, the result may be infinite: a probability of 1 - 1.3e-6
    times the lowest value is -3.402819e38, and 4.3e32 beside fp32's own lowest, -3.402823e38."""
    infinite = (got.abs() == math.inf) & (ref.sign() == got.sign()) & (ref.abs() + bound >= -LOWEST)
    within(torch.where(infinite, ref.float(), got), ref, bound, what)


@pytest.mark.parametrize("N,D,V", [(9, 40, 130), (300, 37, 130), (1500, 200, 1000)])
@pytest.mark.parametrize("value,gated", [(LOWEST, True), (LOWEST, False), (float.fromhex('0x1.ffp127'), False)])
def test_fp32_gradient_through_weights_near_the_largest_value(hd, N, D, V, value, gated):
    """A masked class's gradient of zero times its weight is zero.  (The last value is the first whose nearest bf16 is infinite,
    0x1.ffp127, with a sign that masks where the feature is -1.)"""
    x, w, tokens = masked(gen(N + D), N, D, V, value, gated)
    if value > 0:
        x[:, 0] = -1.0
    ref = masked_reference(x, w, tokens)
    _, lse = hd.xent_fprop(x, w, tokens)
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    within_or_beyond(gx, *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [6, 300])
def test_an_infinite_score_makes_the_normaliser_infinite(hd, N, dtype):
    """log(sum exp z) with one z = +inf is +inf: the loss of any other class is too, that of this class is inf - inf.  A row of
    nothing but -inf has lse = -inf."""
    g = gen(70)
    x, w = torch.randn(N, 24, generator=g, device="cuda"), torch.randn(150, 24, generator=g, device="cuda")
    x[:, 0] = 0.5
    x[1, 0], x[2, 0] = 1.0, -1.0
    x, w = x.to(dtype), w.to(dtype)
    tokens = torch.arange(N, device="cuda") % 150
    w[77, 0] = math.inf
    y = x.clone()
    y[3:, 0] = 0.0                                           # (0 times infinite: not a number)
    loss, lse = hd.xent_fprop(x, w, tokens)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    assert torch.equal(lse == math.inf, want == math.inf) and bool((lse[:2] == math.inf).all()) and bool(torch.isfinite(lse[2]))
    assert bool((loss[:2] == math.inf).all()) and bool(torch.isfinite(loss[2]))
    assert all(math.isnan(float(loss[n])) for n in range(77, N, 150))
    _, lse = hd.xent_fprop(y, w, tokens)
    assert bool(lse[3:].isnan().all()) and bool((lse[:2] == math.inf).all())
    w[:, 0] = -math.inf
    loss, lse = hd.xent_fprop(x, w, tokens)
    assert bool((lse[:2] == -math.inf).all()) and bool(loss[:2].isnan().all()) and bool((lse[2] == math.inf).all())


def test_an_error_that_an_earlier_call_left_is_not_this_call_s(hd):
    """A refused hipSetDevice leaves its error for the next hipGetLastError of the thread; launches that go well say so."""
    import ctypes
    g = gen(71)
    x, w, t = torch.randn(300, 24, generator=g, device="cuda"), torch.randn(50, 24, generator=g, device="cuda"), tokens_for(g, (300,), 50)
    y, gt, gw, loss, norm = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w), torch.empty(300, device="cuda"), torch.empty((), device="cuda")
    lse = hd.xent_fprop(x, w, t)[1]
    with open("/proc/self/maps") as f:
        runtime = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    for call in (lambda: hd.embedding_fprop(w, t, y=y), lambda: hd.embedding_accgrad(x, t, 50, gtable=gt), lambda: hd.xent_fprop(x, w, t, loss=loss, lse=lse),
                 lambda: hd.xent_backward(x, w, t, lse, want_gx=False, gw=gw), lambda: hd.grad_norm([x, w], norm=norm), lambda: hd.grad_clip([x, w], 1.0, norm=norm)):
        call()                                               # (what this allocates is there)
        assert runtime.hipSetDevice(4096) != 0
        call()
    runtime.hipGetLastError()
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [4, 8192])
@pytest.mark.parametrize("value,max_norm", [(5e37, 1e-37), (1.6e38, 3e-38), (5e37, 1e-44), (1e38, 2.0 ** -126)])
def test_clipping_by_factors_down_to_the_smallest(hd, value, max_norm, n):
    """Four equal elements, of norm twice theirs: each becomes max_norm / 2, off by the rounding of a product, or half the smallest step."""
    t = torch.zeros(n, device="cuda")
    t[:4] = value
    limit = float(torch.tensor(max_norm))
    hd.grad_clip([t], max_norm)
    assert float((t[:4].double() - limit / 2).abs().max()) <= 2 * E * limit / 2 + 2.0 ** -150 and float(t[4:].abs().sum()) == 0


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_the_norm_of_an_empty_list_is_float32_under_any_default_type(hd, default):
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        norms = hd.grad_norm([]), hd.grad_clip([], 1.0)
    finally:
        torch.set_default_dtype(before)
    for n in norms:
        assert n.dtype == torch.float32 and float(n) == 0


@pytest.mark.parametrize("N", [7, 90])
@pytest.mark.parametrize("k", [-131, -123, -110, -101, 88, 101, 110, 118, 127])
def test_xent_half_gradients_of_every_loss_scale(hd, N, k):
    """dL/dloss of 2^k and a scale that takes it back: the gradients are those of k = 0."""
    g = gen(72)
    x = torch.randn(N, 48, generator=g, device="cuda").half()
    w = torch.randn(200, 48, generator=g, device="cuda").mul_(0.3).half()
    tokens = tokens_for(g, (N,), 200, none=0.1)
    _, lse = hd.xent_fprop(x, w, tokens)
    for mean in (False, True):
        base = hd.xent_backward(x, w, tokens, lse, gloss=torch.full((N,), 1.0, device="cuda"), scale=0.0625, mean=mean)
        got = hd.xent_backward(x, w, tokens, lse, gloss=torch.full((N,), 2.0 ** k, device="cuda"), scale=0.0625 * 2.0 ** -k, mean=mean)
        assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [math.inf, math.nan])
@pytest.mark.parametrize("shape,planes", [((3, 70), False), ((3, 70), True), ((6,), False)])
def test_rows_without_a_token_are_zero_under_any_scale(hd, shape, planes, scale, dtype):
    """A loss scale that has overflowed: what takes no part stays zero, all else is infinite or not a number."""
    g = gen(73)
    V, D = 40, 24
    tokens = tokens_for(g, shape, V, none=0.3)
    tokens.view(-1)[:2] = torch.tensor([-1, 5], device="cuda")
    has, _ = picks(tokens, V)
    table = torch.randn(V, D, generator=g, device="cuda").to(dtype)
    y = hd.embedding_fprop(table, tokens, scale=scale, planes=planes)
    rows = y.flatten(2).transpose(1, 2).reshape(-1, D) if planes else y.reshape(-1, D)
    assert bool((rows[~has] == 0).all()) and not bool(torch.isfinite(rows[has]).any())
    x = torch.randn(y.shape, generator=g, device="cuda").to(dtype)
    gt = hd.embedding_accgrad(x, tokens, V, scale=scale, planes=planes)
    named = torch.zeros(V, dtype=torch.bool, device="cuda")
    named[tokens[(tokens >= 0)]] = True
    assert bool((gt[~named] == 0).all()) and not bool(torch.isfinite(gt[named]).any())
    _, lse = hd.xent_fprop(x, table, tokens, planes=planes)
    gx, _ = hd.xent_backward(x, table, tokens, lse, scale=scale, planes=planes)
    rows = gx.flatten(2).transpose(1, 2).reshape(-1, D) if planes else gx.reshape(-1, D)
    assert bool((rows[~has] == 0).all()) and not bool(torch.isfinite(rows[has]).any())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,D,V", [(5, 4470, 300), (5, 5001, 300), (260, 8200, 130), (3, 1 << 20, 5), (130, 1 << 20, 5)])
def test_xent_of_long_rows(hd, N, D, V, dtype):
    g = gen(74)
    x = torch.randn(N, D, generator=g, device="cuda").to(dtype)
    w = (torch.randn(V, D, generator=g, device="cuda") * (2 / math.sqrt(D))).to(dtype)
    tokens = tokens_for(g, (N,), V, none=0.1)
    tokens[0] = 3
    ref = masked_reference(x, w, tokens)
    loss, lse = hd.xent_fprop(x, w, tokens)
    within(loss, *ref["loss"], "loss")
    within(lse, *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    within(gx, *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")


def test_xent_of_rows_too_long_is_refused(hd, lib):
    x, w, t = torch.zeros(1, (1 << 20) + 1, device="cuda"), torch.zeros(2, (1 << 20) + 1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    with pytest.raises(lib.FFTConvError, match="unsupported"):
        hd.xent_fprop(x, w, t)
    with pytest.raises(lib.FFTConvError, match="unsupported"):
        hd.xent_backward(x, w, t, torch.zeros(1, device="cuda"))


@pytest.mark.parametrize("N", [3000, 40000])
def test_embedding_of_a_table_whose_tokens_take_four_digits(hd, N):
    """2^25 rows and tokens at both ends: whole numbers, exact in any order."""
    V = (1 << 25) + 3
    tokens = torch.randint(0, V, (N,), generator=gen(75), device="cuda")
    tokens[::7], tokens[1::7], tokens[2::7] = V - 1, 0, 1 << 24
    gy = torch.arange(N, device="cuda").float()[:, None] % 64
    got = hd.embedding_accgrad(gy, tokens, V)
    want = torch.zeros(V, 1, device="cuda").index_add_(0, tokens, gy)
    assert torch.equal(got, want)


def test_norm_and_clip_beyond_32_bit_offsets(hd):
    n = (1 << 31) + 12345
    t = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    t[0], t[1 << 30], t[-1] = 3.0, 4.0, 12.0
    assert float(hd.grad_norm([t])) == 13.0
    assert float(hd.grad_clip([t], 6.5)) == 13.0
    assert [float(t[i]) for i in (0, 1 << 30, n - 1)] == [1.5, 2.0, 6.0]
    assert float(hd.grad_norm([t])) == 6.5


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [2, 200])
@pytest.mark.parametrize("size", [3.0, 100.0, 333.0, 4000.0, 50000.0])
def test_gradients_of_far_scores_are_whole(hd, N, size, dtype):
    """Two classes' scores at 32 size and its opposite, all others' at zero: the probability of the first is one and of all others
    zero (e^-96 and less), so rows whose target it is have no gradient at all and the others' is a difference of two
    weights.  The scores, and so their difference from lse, are exact."""
    size = float(torch.tensor(size).to(dtype))
    w = torch.zeros(130, 8, device="cuda", dtype=dtype)
    w[7, 0], w[9, 0] = 32.0, -32.0
    x = torch.zeros(N, 8, device="cuda", dtype=dtype)
    x[:, 0] = size
    tokens = torch.full((N,), 7, dtype=torch.int64, device="cuda")
    tokens[1::2] = 9
    _, lse = hd.xent_fprop(x, w, tokens)
    assert bool((lse == 32 * size).all())
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    assert float(gx[0::2].abs().max()) == 0 and bool((gx[1::2, 0] == 64.0).all()) and float(gx[:, 1:].abs().max()) == 0
    odd = float(torch.tensor(size * (N // 2)).to(dtype))
    assert float(gw[7, 0]) == odd and float(gw[9, 0]) == -odd
    gw[[7, 9]] = 0
    assert float(gw.abs().max()) == 0
