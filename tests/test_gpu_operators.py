"""The embedding, the linear cross entropy and the gradient norm on the GPU against their formulas in 64 bits.

Bounds are derived, element by element, from where the kernels round.  u is half a step of the
operands' type (2^-8, 2^-11, 2^-24), e = 2^-24 half a step of fp32.
  - A sum of n products in fp32, in any order, is off by at most n e times the sum of their sizes.
  - exp of a difference t in fp32: t is off by e |t| and its product with log2(e) again, the hardware's power of
    two by a step: at most (3 |t| + 4) e of the result.
  - What is rounded to the operands' type is off by u of itself, or half its smallest step if that is more.
  - fp32 scores are formed from two fp16 terms of each value: 2^-22 of x, of w, and of their product for what is left
    out, 12 e of |x w| in all, and three products a term in the sum."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.fixture(scope="module")
def hd(lib):
    h = lib.Handle(0)
    yield h
    h.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_of(x, planes):
    return x.flatten(2).transpose(1, 2).reshape(-1, x.shape[1]) if planes else x.reshape(-1, x.shape[-1])


def tokens_for(g, shape, V, none=0.2, dtype=torch.int64):
    t = torch.randint(0, V, shape, generator=g, device="cuda")
    t[torch.rand(shape, generator=g, device="cuda") < none] = -100
    return t.to(dtype)


def picks(tokens, V):
    t = tokens.reshape(-1).long()
    has = (t >= 0) & (t < V)
    return has, torch.where(has, t, torch.zeros_like(t))


def within(got, ref, bound, what):
    got = got.double()
    assert got.shape == ref.shape, what
    assert bool(torch.isfinite(got).all()), what
    over = (got - ref).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()), float((got - ref).abs().max()))


# ---------------------------------------------------------------------------------- embedding
SHAPES = [((1,), 1, 1, False), ((1,), 1024, 32000, False), ((7,), 37, 5, False), ((3, 100), 64, 1000, False), ((5000,), 129, 3, False),
          ((2, 11, 11), 40, 300, True), ((3, 64), 64, 70000, True), ((5, 730), 33, 2000, True), ((20000,), 8, 1 << 21, False),
          ((999,), 4100, 50, False), ((1, 1), 3, 2, True), ((70000,), 24, 17, False)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape,D,V,planes", SHAPES)
def test_embedding(hd, shape, D, V, planes, dtype):
    g = gen(hash((shape, D, V)) % 1000)
    u, tiny = half_step(dtype), TINY[dtype]
    tokens = tokens_for(g, shape, V, dtype=torch.int32 if D % 2 else torch.int64)
    has, at = picks(tokens, V)
    table = torch.randn(V, D, generator=g, device="cuda").to(dtype)
    y = hd.embedding_fprop(table, tokens, scale=3.3, planes=planes)
    ref = table[at].double() * 3.3 * has[:, None]
    within(rows_of(y, planes), ref, (u + 3 * E) * ref.abs() + tiny, "fprop")

    gy = torch.randn(y.shape, generator=g, device="cuda").to(dtype)
    rows = rows_of(gy, planes).double() * has[:, None]
    ref = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, at, rows) * 0.7
    size = torch.zeros_like(ref).index_add_(0, at, rows.abs()) * 0.7
    count = torch.zeros(V, device="cuda", dtype=torch.float64).index_add_(0, at, has.double())[:, None]
    bound = (count + 3) * E * size + u * (ref.abs() + (count + 3) * E * size) + tiny
    got = hd.embedding_accgrad(gy, tokens, V, scale=0.7, planes=planes)
    within(got, ref, bound, "accGrad")
    assert bool((got[count[:, 0] == 0] == 0).all())
    again = hd.embedding_accgrad(gy, tokens, V, scale=0.7, planes=planes)
    assert torch.equal(got, again)                           # the order of a sum is the rows' own

    got = table.clone()
    hd.embedding_accgrad(gy, tokens, V, scale=0.7, planes=planes, gtable=got, accumulate=True)
    ref = ref + table.double()
    within(got, ref, bound + E * ref.abs() + u * (ref.abs() + bound), "accGrad, accumulated")
    assert torch.equal(got[count[:, 0] == 0], table[count[:, 0] == 0])


def test_embedding_without_rows(hd):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones(5, 4, device="cuda")
    assert hd.embedding_fprop(table, none).shape == (0, 4)
    assert bool((hd.embedding_accgrad(torch.empty(0, 4, device="cuda"), none, 5, gtable=table.clone()) == 0).all())
    assert bool((hd.embedding_accgrad(torch.empty(0, 4, device="cuda"), none, 5, gtable=table.clone(), accumulate=True) == 1).all())


def test_embedding_of_no_tokens_and_of_one_token(hd):
    """All rows without a token, whose gradients may be anything; all rows of one token."""
    tokens = torch.full((300,), -1, dtype=torch.int64, device="cuda")
    table = torch.randn(9, 20, generator=gen(1), device="cuda")
    assert bool((hd.embedding_fprop(table, tokens) == 0).all())
    assert bool((hd.embedding_accgrad(torch.full((300, 20), math.nan, device="cuda"), tokens, 9) == 0).all())
    tokens = torch.full((30000,), 4, dtype=torch.int64, device="cuda")
    gy = torch.ones(30000, 20, device="cuda")
    got = hd.embedding_accgrad(gy, tokens, 9)                # whole numbers: exact in any order
    assert bool((got[4] == 30000).all()) and float(got.abs().sum()) == 30000 * 20


def test_embedding_beyond_32_bit_offsets(hd):
    """A table of more than 2^31 elements: rows at its end are found, and their gradients land there."""
    V, D = (1 << 21) + 5, 1024
    table = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    last = torch.arange(V - 3, V, device="cuda")
    table[V - 3:] = torch.randn(3, D, generator=gen(2), device="cuda").to(torch.bfloat16)
    assert torch.equal(hd.embedding_fprop(table, last), table[V - 3:])
    got = hd.embedding_accgrad(table[V - 3:].clone(), last, V, gtable=torch.full_like(table, 2.0))
    assert torch.equal(got[V - 3:], table[V - 3:]) and float(got[:V - 3].abs().max()) == 0


# ---------------------------------------------------------------------------------- cross entropy
def xent_reference(x, w, tokens, gloss, scale, mean, planes, kept=None):
    """Loss, lse, gx, gw and how far each may be off, in 64 bits."""
    dtype, V, D = x.dtype, w.shape[0], w.shape[1]
    u, tiny = half_step(dtype), TINY[dtype]
    if kept is None:
        kept = 0.0 if dtype == torch.float32 else u          # fp32: G keeps three terms, all of it
    terms = 6 if dtype == torch.float32 else 1
    has, at = picks(tokens, V)
    X = torch.where(has[:, None], rows_of(x, planes).double(), torch.zeros((), device="cuda", dtype=torch.float64))
    W = w.double()
    z = X @ W.t()
    lse = torch.logsumexp(z, 1)
    cut = 12 if dtype == torch.float32 else 0
    dz = ((terms * D + 8 + cut) * E * (X.abs() @ W.abs().t())).amax(1)     # a score's error, the largest of its row
    span = (z.amax(1) - z.amin(1)).clamp(max=100.0)          # (smaller terms do not count)
    dlse = dz + (3 * span + 4 + V ** 0.5 + 300) * E + 2 * E * lse.abs()
    loss = lse - z.gather(1, at[:, None])[:, 0]
    dloss = dz + dlse + E * loss.abs()
    coef = has * scale / (max(1, int(has.sum())) if mean else 1)
    if gloss is not None:
        coef = coef * gloss.reshape(-1).double()
    p = torch.softmax(z, 1)
    dp = p * ((dz + dlse)[:, None] + (3 * (z - lse[:, None]).abs() + 6) * E)
    p[torch.arange(len(at), device="cuda"), at] -= 1.0
    G = p * coef[:, None]
    low = 2.0 ** -38 * coef.abs().max() if dtype == torch.float16 else 0.0
    dG = dp * coef.abs()[:, None] + (kept + 3 * E) * G.abs() + low * has[:, None]
    gx, gw = G @ W, G.t() @ X
    dgx = dG @ W.abs() + (terms * V + 80) * E * (G.abs() @ W.abs())
    dgw = dG.t() @ X.abs() + (terms * len(at) + 80) * E * (G.abs().t() @ X.abs())
    return {"loss": (loss * has, dloss), "lse": (lse * has, dlse),
            "gx": (gx, dgx + u * (gx.abs() + dgx) + tiny), "gw": (gw, dgw + u * (gw.abs() + dgw) + tiny)}


XENT = [((1,), 1, 1, False), ((1,), 64, 256, False), ((3,), 100, 5, False), ((64,), 64, 64, False), ((65,), 8, 65, False),
        ((257,), 72, 300, False), ((30, 10), 130, 1001, False), ((4, 11, 11), 33, 70, True), ((1000,), 256, 4097, False),
        ((2, 500), 384, 1000, True), ((700,), 513, 9000, False), ((2049,), 16, 3, False), ((17,), 1000, 20011, False), ((5, 1), 40, 129, True)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape,D,V,planes", XENT)
def test_xent(hd, shape, D, V, planes, dtype):
    g = gen(hash((shape, D, V)) % 1000 + 1)
    tokens = tokens_for(g, shape, V, none=0.0 if len(shape) == 1 and shape[0] < 4 else 0.2, dtype=torch.int32 if V % 2 else torch.int64)
    xs = (shape[0], D) + shape[1:] if planes else shape + (D,)
    x = torch.randn(xs, generator=g, device="cuda").to(dtype)
    w = (torch.randn(V, D, generator=g, device="cuda") * 2 / math.sqrt(D)).to(dtype)
    gloss = torch.randn(shape, generator=g, device="cuda") if D % 2 == 0 else None
    ref = xent_reference(x, w, tokens, gloss, 3.0, True, planes)
    loss, lse = hd.xent_fprop(x, w, tokens, planes=planes)
    within(loss.reshape(-1), *ref["loss"], "loss")
    within(lse.reshape(-1), *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=3.0, mean=True, planes=planes)
    within(rows_of(gx, planes), *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")
    # the same bits again, and each gradient alone
    loss2, _ = hd.xent_fprop(x, w, tokens, planes=planes)
    gx2, none = hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=3.0, mean=True, planes=planes, want_gw=False)
    none2, gw2 = hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=3.0, mean=True, planes=planes, want_gx=False)
    assert none is None and none2 is None
    assert torch.equal(loss, loss2) and torch.equal(gx, gx2) and torch.equal(gw, gw2)
    # added to what is there
    acc = w.clone()
    hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=3.0, mean=True, planes=planes, want_gx=False, gw=acc, accumulate=True)
    want, bound = ref["gw"]
    want = want + w.double()
    within(acc, want, bound + 2 * E * want.abs() + half_step(dtype) * (want.abs() + bound), "gw, accumulated")


@pytest.mark.parametrize("dtype", TYPES[1:], ids=["bf16", "f16"])
@pytest.mark.parametrize("N,T,D,V,mean", [(1, 0, 64, 20, True), (1, 0, 333, 1001, False), (2, 0, 1000, 20011, True), (4, 2, 40, 300, True), (8, 0, 8, 3, False), (8, 8, 256, 65536, True)])
def test_xent_gradients_of_few_rows_have_one_rounding(hd, N, T, D, V, mean, dtype):
    # What the rounding of a row's G leaves, at most half a step of it, is taken along, rounded itself: G is held
    # to u^2.  (With one rounding of G, u, a gradient made of one coefficient is up to 2 u off.)
    g = gen(N * 1000 + D)
    tokens = torch.randint(0, V, (N // T, T) if T else (N,), generator=g, device="cuda")
    if N > 2:
        tokens.view(-1)[1] = -1
    x = torch.randn((N // T, D, T) if T else (N, D), generator=g, device="cuda").to(dtype)
    w = (torch.randn(V, D, generator=g, device="cuda") / math.sqrt(D)).to(dtype)
    gloss = torch.randn(tokens.shape, generator=g, device="cuda")
    ref = xent_reference(x, w, tokens, gloss, 1.0, mean, bool(T), kept=half_step(dtype) ** 2)
    _, lse = hd.xent_fprop(x, w, tokens, planes=bool(T))
    gx, gw = hd.xent_backward(x, w, tokens, lse, gloss=gloss, mean=mean, planes=bool(T))
    within(rows_of(gx, bool(T)), *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")
    only_x, _ = hd.xent_backward(x, w, tokens, lse, gloss=gloss, mean=mean, planes=bool(T), want_gw=False)
    _, only_w = hd.xent_backward(x, w, tokens, lse, gloss=gloss, mean=mean, planes=bool(T), want_gx=False)
    assert torch.equal(gx, only_x) and torch.equal(gw, only_w)


@pytest.mark.parametrize("N", [1, 8])
def test_xent_gradients_of_few_rows_whose_loss_gradient_is_not_finite(hd, N):
    # gw's row of a class: G x, where G is the product of an infinite dL/dloss and a probability: infinite with x's sign
    x = torch.ones(N, 16, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(4, 16, device="cuda", dtype=torch.bfloat16)
    tokens = torch.zeros(N, device="cuda", dtype=torch.int64)
    _, lse = hd.xent_fprop(x, w, tokens)
    _, gw = hd.xent_backward(x, w, tokens, lse, gloss=torch.full((N,), math.inf, device="cuda"), want_gx=False)
    assert torch.equal(gw[1:], torch.full((3, 16), math.inf, device="cuda", dtype=torch.bfloat16)) and bool((gw[0] == -math.inf).all())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [5, 300])
def test_xent_rows_without_a_target_are_not_read(hd, N, dtype):
    g = gen(3)
    x = torch.randn(N, 40, generator=g, device="cuda").to(dtype)
    w = torch.randn(70, 40, generator=g, device="cuda").to(dtype)
    tokens = tokens_for(g, (N,), 70, none=0.5)
    tokens[1] = -1; tokens[2] = 70
    none = (tokens < 0) | (tokens >= 70)
    assert 0 < int(none.sum()) < N
    dirty = x.clone()
    dirty[none] = math.nan
    dirty[1] = math.inf
    clean = x.clone()
    clean[none] = 0
    got = [hd.xent_fprop(v, w, tokens) for v in (clean, dirty)]
    lse = got[0][1]
    grads = [hd.xent_backward(v, w, tokens, lse.masked_fill(none, f), gloss=torch.ones(N, device="cuda").masked_fill(none, f), mean=True)
             for v, f in ((clean, 0.0), (dirty, math.nan))]
    for a, b in zip(got + grads, got[::-1] + grads[::-1]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert bool(torch.isfinite(a[0]).all()) and bool(torch.isfinite(a[1]).all())
    assert bool((got[0][0][none] == 0).all()) and bool((lse[none] == 0).all()) and bool((grads[0][0][none] == 0).all())


@pytest.mark.parametrize("N", [0, 3, 400])
def test_xent_without_any_target(hd, N):
    x = torch.full((N, 24), math.nan, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(100, 24, generator=gen(4), device="cuda").to(torch.bfloat16)
    tokens = torch.full((N,), -1, dtype=torch.int64, device="cuda")
    loss, lse = hd.xent_fprop(x, w, tokens)
    assert loss.shape == (N,) and bool((loss == 0).all()) and bool((lse == 0).all())
    for mean in (False, True):
        gx, gw = hd.xent_backward(x, w, tokens, lse, mean=mean)
        assert bool((gx == 0).all()) and bool((gw == 0).all())
        acc = w.clone()
        hd.xent_backward(x, w, tokens, lse, mean=mean, gw=acc, accumulate=True)
        assert torch.equal(acc, w)


@pytest.mark.parametrize("N", [2, 200])
def test_xent_of_far_scores(hd, N):
    """Scores thousands apart: the normaliser is the largest score, nothing overflows; the target's own
    probability is 1 or 0 and the gradients are whole weights."""
    w = torch.zeros(130, 8, device="cuda")
    w[7, 0] = 1.0
    w[9, 0] = -1.0
    x = torch.zeros(N, 8, device="cuda")
    x[:, 0] = 4000.0
    tokens = torch.full((N,), 7, dtype=torch.int64, device="cuda")
    tokens[1::2] = 9
    loss, lse = hd.xent_fprop(x, w, tokens)
    assert bool((lse == 4000.0).all()) and bool((loss[0::2] == 0).all()) and bool((loss[1::2] == 8000.0).all())
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    assert bool((gx[0::2] == 0).all()) and bool((gx[1::2, 0] == 2.0).all()) and float(gx[:, 1:].abs().max()) == 0
    odd = N // 2
    assert float(gw[7, 0]) == 4000.0 * odd and float(gw[9, 0]) == -4000.0 * odd


def test_xent_nan_features_reach_the_loss(hd):
    for N in (2, 300):
        x = torch.randn(N, 16, generator=gen(5), device="cuda")
        x[1, 3] = math.nan
        w = torch.randn(50, 16, generator=gen(6), device="cuda")
        tokens = torch.zeros(N, dtype=torch.int64, device="cuda")
        loss, lse = hd.xent_fprop(x, w, tokens)
        assert math.isnan(float(loss[1])) and math.isnan(float(lse[1]))
        assert bool(torch.isfinite(loss[0])) and bool(torch.isfinite(loss[2:]).all())


@pytest.mark.parametrize("offset", [1, 2, 4])
def test_xent_weights_at_any_alignment(hd, offset):
    """Contiguous tensors that start anywhere in their storage."""
    g = gen(7)
    for dtype in (torch.bfloat16, torch.float32):
        w = torch.randn(300 * 64 + 8, generator=g, device="cuda").to(dtype)[offset:offset + 300 * 64].view(300, 64)
        for N in (9, 200):
            x = torch.randn(N * 64 + 8, generator=g, device="cuda").to(dtype)[offset:offset + N * 64].view(N, 64)
            tokens = tokens_for(g, (N,), 300)
            a, b = hd.xent_fprop(x, w, tokens), hd.xent_fprop(x.clone(), w.clone(), tokens)
            ref = xent_reference(x, w, tokens, None, 1.0, False, False)
            within(a[0], *ref["loss"], "loss")
            within(b[0], *ref["loss"], "loss")
            gx, gw = hd.xent_backward(x, w, tokens, a[1])
            within(gx, *ref["gx"], "gx")
            within(gw, *ref["gw"], "gw")


def test_xent_half_gradients_of_any_loss_scale(hd):
    """dL/dloss from 2^-20 to 2^20: G is held at a scale of its own, so gradients lose nothing to it."""
    g = gen(8)
    x = torch.randn(90, 48, generator=g, device="cuda").half()
    w = torch.randn(200, 48, generator=g, device="cuda").mul_(0.3).half()
    tokens = tokens_for(g, (90,), 200)
    _, lse = hd.xent_fprop(x, w, tokens)
    base = hd.xent_backward(x, w, tokens, lse, scale=16.0)
    for k in (-20, 20):
        gloss = torch.full((90,), 2.0 ** k, device="cuda")
        got = hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=16.0 * 2.0 ** -k)
        assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])


def test_xent_gradients_against_differences(hd):
    """Along a direction d of x and w, h = 2^-6: (L(+h) - L(-h)) / 2h.  Off by the losses' rounding over h and by
    h^2 / 6 of a third derivative.  A score moves by s' = x dw + dx w and curves by s'' = 2 dx dw, so with a and b their
    largest sizes that derivative is at most 8 a^3 + 6 a b a row (central moments over a range of 2 a and 2 b)."""
    g = gen(9)
    N, D, V, h = 12, 6, 9, 2.0 ** -6
    x, w = torch.randn(N, D, generator=g, device="cuda"), torch.randn(V, D, generator=g, device="cuda")
    dx, dw = torch.randn(N, D, generator=g, device="cuda") * 0.2, torch.randn(V, D, generator=g, device="cuda") * 0.2
    tokens = tokens_for(g, (N,), V)
    loss, lse = hd.xent_fprop(x, w, tokens)
    gx, gw = hd.xent_backward(x, w, tokens, lse)
    slope = float((gx.double() * dx.double()).sum() + (gw.double() * dw.double()).sum())
    up, down = (hd.xent_fprop(x + s * h * dx, w + s * h * dw, tokens)[0].double().sum() for s in (1, -1))
    a = (dx.double() @ w.double().t() + x.double() @ dw.double().t()).abs().amax(1) + 2 * h * (dx.double() @ dw.double().t()).abs().amax(1)
    b = 2 * (dx.double() @ dw.double().t()).abs().amax(1)
    third = float((8 * a ** 3 + 12 * a * b).sum())
    ref = xent_reference(x, w, tokens, None, 1.0, False, False)
    # 2 e of every x, w is lost in forming x + h d; with the losses' own error
    move = 2 * E * float(((x.abs() + 1) @ (w.abs() + 1).t()).amax(1).sum()) * 2
    noise = 2 * (float(ref["loss"][1].sum()) + move) / (2 * h)
    exactly = float(ref["gx"][1].mul(dx.abs()).sum() + ref["gw"][1].mul(dw.abs()).sum())
    assert abs(float(up - down) / (2 * h) - slope) <= h * h / 6 * third + noise + exactly
    assert h * h / 6 * third + noise + exactly < 0.2 * abs(slope) + 0.2


@pytest.mark.parametrize("ex,ew", [(0, 0), (-100, 100), (60, -60), (-120, 118), (-126, 120)])
def test_xent_fp32_rows_of_any_scale(hd, ex, ew):
    """Features around 2^ex, weights around 2^ew, each row spread over 2^12: the scores' two fp16 terms are scaled row by
    row.  A value is off by 2^-22 of itself or 2^-40 of its row's largest, products by three such errors."""
    g = gen(50)
    N, D, V = 500, 200, 1500
    x = torch.randn(N, D, generator=g, device="cuda") * torch.exp2(torch.randint(-12, 1, (N, D), generator=g, device="cuda").float())
    w = torch.randn(V, D, generator=g, device="cuda") / math.sqrt(D)
    x, w = torch.ldexp(x, torch.tensor(ex, device="cuda")), torch.ldexp(w, torch.tensor(ew, device="cuda"))
    tokens = tokens_for(g, (N,), V)
    ref = xent_reference(x, w, tokens, None, 1.0, False, False)
    has, _ = picks(tokens, V)
    X, W = x.double().abs() * has[:, None], w.double().abs()
    more = 3 * 2.0 ** -40 * (X.amax(1) * W.sum(1).max() + X.sum(1) * W.max()) + 2.0 ** -126
    loss, lse = hd.xent_fprop(x, w, tokens)
    within(loss, ref["loss"][0], ref["loss"][1] + 3 * more, "loss")
    within(lse, ref["lse"][0], ref["lse"][1] + 2 * more, "lse")


def test_xent_fp32_of_a_tiny_class(hd):
    """A class that no row comes near: its gradient is small in every row, and as exact as the others'."""
    g = gen(51)
    N, D, V = 300, 48, 200
    x = torch.randn(N, D, generator=g, device="cuda").abs()
    w = torch.randn(V, D, generator=g, device="cuda") * 0.1
    w[7] = -0.6                                             # p of about e^-20
    tokens = torch.full((N,), 3, dtype=torch.int64, device="cuda")
    _, lse = hd.xent_fprop(x, w, tokens)
    _, gw = hd.xent_backward(x, w, tokens, lse, want_gx=False)
    ref = xent_reference(x, w, tokens, None, 1.0, False, False)["gw"]
    within(gw, *ref, "gw")
    assert 0 < float(ref[0][7].max()) < 1e-3 and bool((ref[1][7] < 1e-3 * ref[0][7]).all())


def test_capture_without_an_eager_call_before(lib):
    h = lib.Handle(0)
    try:
        g = gen(52)
        x, w = torch.randn(700, 128, generator=g, device="cuda").bfloat16(), torch.randn(5000, 128, generator=g, device="cuda").bfloat16()
        t = tokens_for(g, (700,), 5000)
        ws = [torch.empty(h.xent_workspace_bytes(k, x.dtype, 700, 128, 5000), dtype=torch.uint8, device="cuda") for k in (lib.FPROP, lib.BPROP)]
        loss, lse = torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
        gx, gw = torch.empty_like(x), torch.empty_like(w)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.xent_fprop(x, w, t, loss=loss, lse=lse, ws=ws[0])
            h.xent_backward(x, w, t, lse, gx=gx, gw=gw, ws=ws[1])
        for _ in range(3):
            for v in (loss, gx, gw):
                v.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            want = h.xent_fprop(x, w, t)
            wg = h.xent_backward(x, w, t, want[1])
            assert torch.equal(loss, want[0]) and torch.equal(gx, wg[0]) and torch.equal(gw, wg[1])
    finally:
        h.close()


def test_a_captured_pass_keeps_its_buffer(lib):
    """A convolution pass captured on the handle's own buffer: operators that need more than that buffer holds run
    between the replays and leave it where it is."""
    h = lib.Handle(0)
    try:
        g = gen(53)
        x, w = torch.randn(8, 8, 13, 13, generator=g, device="cuda"), torch.randn(8, 8, 3, 3, generator=g, device="cuda")
        want = h.fft_conv_fprop(x, w).clone()
        y = torch.empty_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.fft_conv_fprop(x, w, y=y)
        for n in (300, 3000):
            f, c = torch.randn(n, 64, generator=g, device="cuda"), torch.randn(9000, 64, generator=g, device="cuda")
            t = tokens_for(g, (n,), 9000)
            _, lse = h.xent_fprop(f, c, t)
            h.xent_backward(f, c, t, lse)
            h.embedding_accgrad(f, t, 9000)
            y.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
    finally:
        h.close()


@pytest.mark.parametrize("seed", range(30))
def test_random_sizes(hd, seed):
    import random
    rng = random.Random(seed)

    def size(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    dtype, N, D, V = TYPES[seed % 3], size(1, 3000), size(1, 700), size(1, 9000)
    planes = rng.random() < 0.3
    T = size(1, 200)
    shape = (max(1, N // T), T) if planes else (N,)
    g = gen(seed)
    tokens = tokens_for(g, shape, V, none=rng.choice([0, 0.1, 0.5, 0.95]), dtype=rng.choice([torch.int32, torch.int64]))
    x = torch.randn((shape[0], D) + shape[1:] if planes else shape + (D,), generator=g, device="cuda").to(dtype)
    w = (torch.randn(V, D, generator=g, device="cuda") * rng.choice([0.1, 2, 8]) / math.sqrt(D)).to(dtype)
    gloss = torch.randn(shape, generator=g, device="cuda") if rng.random() < 0.5 else None
    mean, scale = rng.random() < 0.5, 64.0 if dtype == torch.float16 else 1.0
    ref = xent_reference(x, w, tokens, gloss, scale, mean, planes)
    loss, lse = hd.xent_fprop(x, w, tokens, planes=planes)
    within(loss.reshape(-1), *ref["loss"], "loss")
    within(lse.reshape(-1), *ref["lse"], "lse")
    gx, gw = hd.xent_backward(x, w, tokens, lse, gloss=gloss, scale=scale, mean=mean, planes=planes)
    within(rows_of(gx, planes), *ref["gx"], "gx")
    within(gw, *ref["gw"], "gw")


def test_xent_beyond_32_bit_offsets(hd):
    """More than 2^31 scores a piece: the gradients of rows at both ends."""
    N, D, V = (1 << 20) + 3, 16, 2050
    g = gen(10)
    x = torch.randn(N, D, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(V, D, generator=g, device="cuda").to(torch.bfloat16)
    tokens = torch.randint(0, V, (N,), generator=g, device="cuda")
    loss, lse = hd.xent_fprop(x, w, tokens)
    gx, _ = hd.xent_backward(x, w, tokens, lse)
    for at in (slice(0, 64), slice(N - 64, N)):
        ref = xent_reference(x[at], w, tokens[at], None, 1.0, False, False)
        within(loss[at], *ref["loss"], "loss")
        within(gx[at], *ref["gx"], "gx")


# ---------------------------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [0, 3], [5, 0, 8191, 8192, 8193], [7] * 300, [1 << 20, 3, 100001], [1 + 37 * k for k in range(129)]],
                         ids=["one", "empty", "pieces", "many", "large", "two_launches"])
def test_norm_and_clip(hd, sizes, dtype):
    g = gen(len(sizes))
    u, tiny = half_step(dtype), TINY[dtype]
    grads = [torch.randn(n, generator=g, device="cuda").to(dtype) for n in sizes]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    norm = hd.grad_norm(grads)
    assert abs(float(norm) - want) <= 2 * E * want
    for ratio in (0.3, 1.5):
        c = min(1.0, float(torch.tensor(want * ratio)) / want)
        out = [torch.full_like(t, math.nan) for t in grads]
        assert torch.equal(hd.grad_clip(grads, want * ratio, out=out), norm)
        inplace = [t.clone() for t in grads]
        hd.grad_clip(inplace, want * ratio)
        for t, o, i in zip(grads, out, inplace):
            ref = t.double() * c
            if t.numel():
                within(o, ref, (u + 4 * E) * ref.abs() + tiny, "clip")
            assert torch.equal(o, i)


def test_norm_of_mixed_types_and_any_alignment(hd):
    g = gen(20)
    base = torch.randn(40000, generator=g, device="cuda")
    grads = [base[1:20000], base.bfloat16()[3:30001], base.half()[5:6]]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    assert abs(float(hd.grad_norm(grads)) - want) <= 2 * E * want
    out = [torch.empty_like(t) for t in grads]
    hd.grad_clip(grads, want / 8, out=out)                   # close to a power of two
    for t, o in zip(grads, out):
        ref = t.double() * (float(torch.tensor(want / 8)) / want)
        within(o, ref, (half_step(t.dtype) + 4 * E) * ref.abs() + TINY[t.dtype], "clip")


def test_norm_where_squares_leave_fp32(hd):
    big = torch.full((4,), 1e30, device="cuda")
    small = torch.full((4,), 1e-30, device="cuda")
    assert abs(float(hd.grad_norm([big])) / 2e30 - 1) <= 4 * E
    assert abs(float(hd.grad_norm([small])) / 2e-30 - 1) <= 4 * E
    hd.grad_clip([big], 1.0)
    assert float((big - 0.5).abs().max()) <= 4 * E


@pytest.mark.parametrize("value,max_norm", [(1e38, 1e-3), (1e30, 1e-15), (3e37, 1.0), (1e-10, 1e-37)])
def test_clipping_by_any_factor(hd, value, max_norm):
    # four equal elements of norm twice theirs: each becomes max_norm / 2, off by the roundings of two factors and products
    t = torch.full((4,), value, device="cuda")
    hd.grad_clip([t], max_norm)
    assert float((t.double() - max_norm / 2).abs().max()) <= 5 * E * max_norm / 2 + 2.0 ** -150


@pytest.mark.parametrize("value", [math.nan, math.inf, 0.0])
def test_norms_that_say_nothing_leave_the_values(hd, value):
    t = torch.ones(5000, device="cuda") if value else torch.zeros(5000, device="cuda")
    t[4321] = value
    before, out = t.clone(), torch.empty_like(t)
    n1, n2 = hd.grad_clip([t], 0.5, out=[out]), hd.grad_clip([t], 0.5)
    for n in (n1, n2):
        assert math.isnan(float(n)) if math.isnan(value) else float(n) == value
    assert torch.equal(t.nan_to_num(9.0), before.nan_to_num(9.0)) and torch.equal(out.nan_to_num(9.0), before.nan_to_num(9.0))


@pytest.mark.parametrize("dtype", TYPES[:2], ids=["f32", "bf16"])
def test_a_norm_beyond_fp32_is_infinite_and_leaves_the_values(hd, dtype):
    t = torch.full((5000,), 3e38, device="cuda").to(dtype)
    before, out = t.clone(), torch.empty_like(t)
    assert math.isinf(float(hd.grad_norm([t]))) and math.isinf(float(hd.grad_clip([t], 1.0, out=[out]))) and math.isinf(float(hd.grad_clip([t], 1.0)))
    assert torch.equal(t, before) and torch.equal(out, before)


def test_an_empty_list_has_norm_zero(hd):
    assert float(hd.grad_norm([])) == 0 and float(hd.grad_clip([], 1.0)) == 0
    assert float(hd.grad_norm([torch.empty(0, device="cuda")])) == 0


# ---------------------------------------------------------------------------------- refusals that reach the library
def test_refusals(hd, lib):
    x, w = torch.zeros(6, 8, device="cuda"), torch.zeros(5, 8, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    short = torch.empty(16, dtype=torch.uint8, device="cuda")
    odd = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[4:]
    lse = torch.zeros(6, device="cuda")
    for call in (lambda ws: hd.embedding_accgrad(x, t, 5, ws=ws), lambda ws: hd.xent_fprop(x, w, t, ws=ws),
                 lambda ws: hd.xent_backward(x, w, t, lse, ws=ws), lambda ws: hd.grad_norm([x], ws=ws), lambda ws: hd.grad_clip([x], 1.0, ws=ws)):
        with pytest.raises(lib.FFTConvError, match="workspace"):
            call(short)
        with pytest.raises(lib.FFTConvError, match="invalid argument"):
            call(odd)
    flat = torch.ones(64, device="cuda")
    for limit in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(lib.FFTConvError, match="invalid argument"):
            hd.grad_clip([flat], limit)
    for grads, out in (([flat, flat], None), ([flat[:40], flat[30:]], None), ([flat[:30], flat[30:]], [flat[30:60], flat[:34]]),
                       ([flat], [flat[1:]])):
        with pytest.raises(lib.FFTConvError):
            hd.grad_clip(grads, 1.0, out=out)
    torch.cuda.synchronize()
    assert bool((flat == 1).all())
    hd.grad_clip([flat[:30], flat[30:]], 1.0)                # neighbours are no overlap
    other = torch.empty(64, device="cuda")
    hd.grad_clip([flat, flat], 1.0, out=[other, torch.empty_like(other)])     # read twice, written apart


# ---------------------------------------------------------------------------------- streams and graphs
def test_another_stream_and_a_handle_of_its_own(lib):
    """Two handles on two streams at once, each with its own workspace."""
    g = gen(30)
    x = torch.randn(700, 96, generator=g, device="cuda").bfloat16()
    w = torch.randn(3000, 96, generator=g, device="cuda").bfloat16()
    t = tokens_for(g, (700,), 3000)
    hs = [lib.Handle(0), lib.Handle(0)]
    try:
        want = hs[0].xent_fprop(x, w, t)
        wg = hs[0].xent_backward(x, w, t, want[1])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = []
        for _ in range(5):
            for h, s in zip(hs, streams):
                with torch.cuda.stream(s):
                    a = h.xent_fprop(x, w, t)
                    got.append(a + h.xent_backward(x, w, t, a[1]) + (h.embedding_accgrad(x, t, 3000), h.grad_norm([x, w])))
        torch.cuda.synchronize()
        for r in got:
            for a, b in zip(r[:4], want + wg):
                assert torch.equal(a, b)
            assert torch.equal(r[4], got[0][4]) and torch.equal(r[5], got[0][5])
    finally:
        for h in hs:
            h.close()


def test_capture_and_replay(hd, lib):
    g = gen(31)
    N, D, V = 400, 72, 1500
    dt = torch.bfloat16
    x, w = torch.randn(N, D, generator=g, device="cuda").to(dt), torch.randn(V, D, generator=g, device="cuda").to(dt)
    t = tokens_for(g, (N,), V)
    loss, lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    y, gx, gw, gt, norm = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w), torch.empty((), device="cuda")
    out = [torch.empty_like(gx), torch.empty_like(gt)]

    def scratch(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

    ws = [scratch(hd.xent_workspace_bytes(lib.FPROP, dt, N, D, V)), scratch(hd.xent_workspace_bytes(lib.BPROP, dt, N, D, V)),
          scratch(hd.embedding_workspace_bytes(dt, N, D, V)), scratch(hd.grad_workspace_bytes([gx, gt]))]

    def step():
        hd.embedding_fprop(w, t, y=y)
        hd.xent_fprop(x, w, t, loss=loss, lse=lse, ws=ws[0])
        hd.xent_backward(x, w, t, lse, mean=True, gx=gx, gw=gw, ws=ws[1])
        hd.embedding_accgrad(gx, t, V, gtable=gt, ws=ws[2])
        hd.grad_clip([gx, gt], 0.01, out=out, norm=norm, ws=ws[3])

    def result():
        torch.cuda.synchronize()
        return [v.clone() for v in (y, loss, lse, gx, gw, gt, norm, *out)]

    def eager():
        step()
        return result()

    eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        if rep:                                              # other inputs, and other work on the handle between replays
            x.copy_(torch.randn(N, D, generator=g, device="cuda"))
            t.copy_(tokens_for(g, (N,), V, none=0.1 + 0.2 * rep))
            hd.xent_fprop(torch.randn(3000, 64, generator=g, device="cuda"), torch.randn(9000, 64, generator=g, device="cuda"),
                          tokens_for(g, (3000,), 9000))
        want = eager()
        for v in (y, loss, lse, gx, gw, gt, norm, *out):
            v.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        for k, (a, b) in enumerate(zip(result(), want)):
            assert torch.equal(a, b), (rep, k)

    # under capture the handle's own workspace, which may move later, is refused
    refused = []
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(other):
        hd.embedding_fprop(w, t, y=y)
        for call in (lambda: hd.xent_fprop(x, w, t, loss=loss, lse=lse), lambda: hd.xent_backward(x, w, t, lse, gx=gx, gw=gw),
                     lambda: hd.embedding_accgrad(gx, t, V, gtable=gt), lambda: hd.grad_norm([gx], norm=norm),
                     lambda: hd.grad_clip([gx], 1.0, norm=norm)):
            try:
                call()
            except lib.FFTConvError as e:
                refused.append("workspace" in str(e))
    assert refused == [True] * 5


# ---------------------------------------------------------------------------------- all of them together
def test_a_training_step_from_tokens_to_clipped_gradients(hd):
    """Maps of tokens -> planes -> a convolution layer -> a class for every position -> loss, and all the way back, with the
    table and the classifier one tensor.  Against the same step in 64 bits on the CPU; a convolution pass
    is within 1e-4 of its largest value as everywhere in these tests, and what follows is linear in it."""
    g = gen(40)
    S, V, D, h, k = 3, 50, 8, 13, 3
    o = h - k + 1
    table = torch.randn(V, D, generator=g, device="cuda") * 0.5
    conv = torch.randn(D, D, k, k, generator=g, device="cuda") * 0.2
    tokens = tokens_for(g, (S, h, h), V, none=0.05)
    targets = tokens_for(g, (S, o, o), V, none=0.3)
    x = hd.embedding_fprop(table, tokens, scale=math.sqrt(D), planes=True)
    saved = torch.empty(hd.saved_bytes(S, D, D, h, h, k, k) // 4, device="cuda")
    y = hd.fft_conv_fprop_save(x, conv, saved)
    loss, lse = hd.xent_fprop(y, table, targets, planes=True)
    gy, gtable = hd.xent_backward(y, table, targets, lse, mean=True, planes=True)
    gx, gconv = hd.fft_conv_backward(gy, saved, D, h, h, k, k)
    hd.embedding_accgrad(gx, tokens, V, scale=math.sqrt(D), planes=True, gtable=gtable, accumulate=True)
    norm = hd.grad_norm([gtable, gconv])
    before = [gtable.clone(), gconv.clone()]
    hd.grad_clip([gtable, gconv], 0.05)

    T, C = table.double().cpu().requires_grad_(), conv.double().cpu().requires_grad_()
    tok, tgt = tokens.cpu(), targets.cpu()
    emb = torch.where((tok >= 0)[..., None], T[tok.clamp(min=0)], torch.zeros((), dtype=torch.float64)) * math.sqrt(D)
    feat = torch.nn.functional.conv2d(emb.permute(0, 3, 1, 2), C)
    z = feat.permute(0, 2, 3, 1) @ T.t()
    L = (torch.logsumexp(z, -1) - z.gather(-1, tgt.clamp(min=0)[..., None])[..., 0])[tgt >= 0]
    L.mean().backward()
    assert abs(float(loss.double().sum() / (targets >= 0).sum()) - float(L.detach().mean())) <= 1e-4
    want = [T.grad, C.grad]
    for got, ref in zip(before, want):
        assert float((got.cpu().double() - ref).abs().max()) <= 5e-4 * float(ref.abs().max())
    n = math.sqrt(sum(float(r.square().sum()) for r in want))
    assert abs(float(norm) - n) <= 1e-3 * n and n > 0.05
    for got, old in zip((gtable, gconv), before):
        ref = old.double() * (0.05 / float(norm))
        assert float((got.double() - ref).abs().max()) <= 1e-6 * float(ref.abs().max())
