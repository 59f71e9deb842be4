"""Accuracy and ranges of the token-model operators where a bound on every
element says too little: the error of whole outputs against that of their one
rounding, relative errors far from zero, infinities and NaN in every kernel of
the products, launches past one grid."""
import pytest

from tests.gpu_common import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def s():
    import paper_1912_11554_amd as nuts
    h = nuts.Sampler(0)
    yield h
    h.close()


def _torch():
    import torch
    return torch


def _gen(seed):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *q, std=1.0, t=torch.float32: (torch.randn(*q, device="cuda", generator=g) * std).to(t)


def _cdf(z):
    """The normal distribution function (torch's own cancels below -6)."""
    return 0.5 * _torch().special.erfc(-z * 0.5 ** 0.5)


def _act(z, kind):
    """act(z) and its slope, in z's 64 bits."""
    torch = _torch()
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "gelu":
        cdf = _cdf(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    p, q = torch.special.expit(z), torch.special.expit(-z)
    return (p, p * q) if kind == "sigmoid" else (z * p, p + z * p * q)


# --------------------------------------------------------------------------
# bf16 gradients.  With d = dy act'(z) in two parts, at most 2^-17 |d| is left
# out, and fp32 sums of up to n products add n 2^-24: next to the rounding of
# the output (1.7e-3 of its norm) both vanish, so an output's error is that
# rounding's, to a hundredth.  Rounded to bf16, d's error is as large again and
# independent: 1.4 times in all.

def _errors(got, ref):
    """Norm of got's error, in units of that of ref rounded once."""
    once = (ref.bfloat16().double() - ref).norm()
    return float((got.double() - ref).norm() / once)


BF16_SHAPES = [(200, 264, 136), (130, 520, 264), (520, 1032, 512), (1100, 1040, 200), (2050, 1032, 520)]


@pytest.mark.parametrize("shape", BF16_SHAPES)
@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
def test_bf16_linear_gradients_round_once(s, shape, act):
    torch = _torch()
    M, N, K = shape
    say("one rounding, linear", shape, act)
    rand, bf = _gen(M + N + K), torch.bfloat16
    x, w, dy = rand(M, K, t=bf), rand(N, K, std=K ** -0.5, t=bf), rand(M, N, t=bf)
    _, pre = s.linear(x, w, act=act, save=True)
    d = dy.double() * _act(pre.double(), act)[1]
    refs = d @ w.double(), d.T @ x.double()
    for got, ref in zip(s.linear_grad(dy, x, w, act=act, pre=pre), refs):
        assert _errors(got, ref) <= 1.01
    for got, ref in zip(s.linear_grad(dy, x, w, act=act, pre=pre, rounded=True), refs):
        assert 1.2 <= _errors(got, ref) <= 1.6


@pytest.mark.parametrize("shape", BF16_SHAPES)
def test_bf16_gated_gradients_round_once(s, shape):
    torch = _torch()
    M, F, K = shape
    say("one rounding, gated", shape)
    rand, bf = _gen(M + F + K + 1), torch.bfloat16
    x, dy = rand(M, K, t=bf), rand(M, F, t=bf)
    wg, wu = rand(F, K, std=K ** -0.5, t=bf), rand(F, K, std=K ** -0.5, t=bf)
    _, pre = s.gated(x, wg, wu, save=True)
    a, slope = _act(pre[0].double(), "silu")
    dg, du = dy.double() * pre[1].double() * slope, dy.double() * a
    refs = dg @ wg.double() + du @ wu.double(), dg.T @ x.double(), du.T @ x.double()
    for got, ref in zip(s.gated_grad(dy, x, wg, wu, pre), refs):
        assert _errors(got, ref) <= 1.01
    for got, ref in zip(s.gated_grad(dy, x, wg, wu, pre, rounded=True), refs):
        assert 1.2 <= _errors(got, ref) <= 1.6


def test_rounding_is_the_identity_where_nothing_is_rounded(s):
    # fp32, and bf16 without an activation
    torch = _torch()
    say("rounded, no effect")
    rand = _gen(9)
    for t, act in ((torch.float32, "silu"), (torch.bfloat16, "none")):
        x, w, dy = rand(70, 40, t=t), rand(50, 40, t=t), rand(70, 50, t=t)
        _, pre = s.linear(x, w, act=act, save=True)
        a, b = (s.linear_grad(dy, x, w, act=act, pre=pre, rounded=r) for r in (False, True))
        assert all(torch.equal(p, q) for p, q in zip(a, b))


# --------------------------------------------------------------------------
# Infinities and NaN.  Where an output's sum holds none, it is bit for bit what
# it is without them elsewhere; where it does, it is what the sum in 64 bits
# gives: NaN, or the same infinity.

def _same_limits(got, ref, clean, touched, what):
    torch = _torch()
    ref = ref.to(got.dtype)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN"
    inf = torch.isinf(ref)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    assert torch.equal(got[~touched], clean[~touched]), f"{what}: elsewhere"
    assert inf.any() and torch.isfinite(got).any(), what  # (the case has both)


def _touched(shape, rows, cols):
    t = _torch().zeros(shape, dtype=_torch().bool, device="cuda")
    t[rows] = True
    t[:, cols] = True
    return t


# M, N, K: 64 x 64 tiles on and off the 16-byte grid, with slices, 128 x 128, 256 x 256
PRODUCT_SHAPES = [(70, 40, 96), (300, 75, 137), (130, 128, 4096), (130, 100, 4099), (2560, 2600, 72), (3600, 3640, 72)]


@pytest.mark.parametrize("shape", PRODUCT_SHAPES)
@pytest.mark.parametrize("rounded", [False, True])
def test_infinite_factors_of_bf16_gradients(s, shape, rounded):
    # dz's second part times an infinity is an infinity of either sign, or 0 * inf
    torch = _torch()
    M, N, K = shape
    say("infinite factors", shape, rounded)
    rand, bf = _gen(M + N), torch.bfloat16
    x, w, dy = rand(M, K, t=bf), rand(N, K, t=bf), rand(M, N, t=bf)
    z = rand(M, N)
    clean = s.linear_grad(dy, x, w, act="silu", pre=z, rounded=rounded)
    x[5, 3], x[6, 7], w[9, 11], w[10, 13] = float("inf"), float("-inf"), float("-inf"), float("inf")
    dx, dw, db = s.linear_grad(dy, x, w, act="silu", pre=z, rounded=rounded)
    d = dy.double() * _act(z.double(), "silu")[1]
    _same_limits(dx, d @ w.double(), clean[0], _touched((M, K), [], [11, 13]), "dx")
    _same_limits(dw, d.T @ x.double(), clean[1], _touched((N, K), [], [3, 7]), "dw")
    assert torch.equal(db, clean[2])
    # the gated block: two products each with parts of their own
    x, w2, pre = rand(M, K, t=bf), rand(N, K, t=bf), rand(2, M, N)
    w = rand(N, K, t=bf)
    clean = s.gated_grad(dy, x, w, w2, pre, rounded=rounded)
    x[5, 3], w[9, 11], w2[10, 13] = float("inf"), float("-inf"), float("inf")
    got = s.gated_grad(dy, x, w, w2, pre, rounded=rounded)
    a, slope = _act(pre[0].double(), "silu")
    dg, du = dy.double() * pre[1].double() * slope, dy.double() * a
    _same_limits(got[0], dg @ w.double() + du @ w2.double(), clean[0], _touched((M, K), [], [11, 13]), "dx")
    _same_limits(got[1], dg.T @ x.double(), clean[1], _touched((N, K), [], [3]), "dwg")
    _same_limits(got[2], du.T @ x.double(), clean[2], _touched((N, K), [], [3]), "dwu")


def _plant(t):
    """Infinities, and a NaN whose set bits all lie in the lower half in fp32,
    in a matrix; (rows, columns) that they touch."""
    torch = _torch()
    t[3, 5], t[8, 2] = float("inf"), float("-inf")
    if t.dtype == torch.float32:
        t.view(torch.int32)[11, 7] = 0x7f800001
    else:
        t[11, 7] = float("nan")
    return [3, 8, 11], [5, 2, 7]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 40, 96), (40, 40, 96)] + PRODUCT_SHAPES)
def test_infinities_and_nan_in_every_product(s, shape, dtype):
    torch = _torch()
    M, N, K = shape
    say("infinities", shape, dtype)
    rand, t = _gen(M + N + 7), getattr(torch, dtype)
    x, w, w2, dy = rand(M, K, t=t), rand(N, K, t=t), rand(N, K, t=t), rand(M, N, t=t)
    none = []
    # forward: w's touch whole columns, x's whole rows
    y0, g0 = s.linear(x, w), s.gated(x, w, w2, act="none")
    wrows, wcols = _plant(w)
    xrows = none
    if M > 11:
        xrows, _ = _plant(x)
    y = x.double() @ w.double().T
    _same_limits(s.linear(x, w), y, y0, _touched((M, N), xrows, wrows), "y")
    # (an infinite product may meet a finite one of either sign, so NaN comes of it as 0 inf does)
    _same_limits(s.gated(x, w, w2, act="none"), y * (x.double() @ w2.double().T), g0, _touched((M, N), xrows, wrows), "gated")
    # gradients: w's columns are dx's, x's columns dw's, dy's rows dx's and its columns dw's
    clean = s.linear_grad(dy, rand(M, K, t=t), rand(N, K, t=t))
    x, w = rand(M, K, t=t), rand(N, K, t=t)
    clean = s.linear_grad(dy, x, w)
    _plant(w)
    dx, dw, db = s.linear_grad(dy, x, w)
    _same_limits(dx, dy.double() @ w.double(), clean[0], _touched((M, K), none, wcols), "dx")
    assert torch.equal(dw, clean[1])
    if M > 11:
        w = rand(N, K, t=t)
        clean = s.linear_grad(dy, x, w)
        dyrows, dycols = _plant(dy)
        dx, dw, db = s.linear_grad(dy, x, w)
        _same_limits(dx, dy.double() @ w.double(), clean[0], _touched((M, K), dyrows, none), "dx")
        _same_limits(dw, dy.double().T @ x.double(), clean[1], _touched((N, K), dycols, none), "dw")
        _same_limits(db, dy.double().sum(0), clean[2], _touched((1, N), none, dycols)[0], "dbias")


@pytest.mark.parametrize("shape", [(2, 40, 96)] + PRODUCT_SHAPES)
def test_values_at_the_top_of_the_fp32_range(s, shape):
    # the largest value times 1/2 and 2, and sums that the corrections reach the top of
    torch = _torch()
    M, N, K = shape
    say("top of the range", shape)
    rand = _gen(M + N + 8)
    x, w = rand(M, K), rand(N, K)
    big = torch.finfo(torch.float32).max
    x[:, 0] = 0
    x[1, 0] = big
    w[0::2, 0], w[1::2, 0] = 0.5, 2.0
    clean = s.linear(x, w)[:1]
    y = s.linear(x, w)
    assert (y[1, 0::2].double() / (big / 2) - 1).abs().max() <= 4 * U
    assert (y[1, 1::2] == float("inf")).all()
    assert torch.equal(y[:1], clean) and torch.isfinite(y[2:]).all()


@pytest.mark.parametrize("M", [3, 130])
@pytest.mark.parametrize("e", [-105, -120, -130, -149])
def test_small_fp32_factors(s, M, e):
    # tiles take a factor to multiples of 2^-133, few rows to fp32's own
    torch = _torch()
    say("small factors", M, e)
    K = 64
    rand = _gen(M - e)
    x = ((rand(M, K).abs() + 1).double() * 2.0 ** e).float()
    w = rand(40, K) * 2.0 ** 100
    ref, size = x.double() @ w.double().T, x.double() @ w.double().abs().T
    off = 2.0 ** -133 * w.double().abs().sum(1) if M > 64 else 0
    assert ((s.linear(x, w).double() - ref).abs() <= (K + 8) * U * size + off).all()


# --------------------------------------------------------------------------
# More blocks of work than one launch has workgroups.

@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradients_over_very_many_rows(s, dtype):
    # 2^26 rows and a few; whole numbers, so every sum is exact in any order
    torch = _torch()
    M, t = (1 << 26) + 35, getattr(torch, dtype)
    say("very many rows", dtype)
    g = torch.Generator(device="cuda").manual_seed(4)
    sign = lambda *q, t=t: (torch.randint(0, 2, q, device="cuda", generator=g, dtype=torch.int8) * 2 - 1).to(t)  # noqa: E731
    x, dy, z = sign(M, 1), sign(M, 1), sign(M, 1, t=torch.float32)
    w = torch.tensor([[3.0]], device="cuda", dtype=t)
    dz = torch.where(z > 0, dy, torch.zeros_like(dy))
    total = dz.sum(dtype=torch.float64)
    for bias in (True, False):
        dx, dw, db = s.linear_grad(dy, x, w, act="relu", pre=z, bias=bias)
        assert torch.equal(dx, 3 * dz)
        assert float(dw) == float((dz * x).sum(dtype=torch.float64).to(t))
        if bias:
            assert float(db) == float(total.to(t))
    pre = sign(2, M, 1, t=torch.float32)
    dx, dwg, dwu = s.gated_grad(dy, x, w, -w, pre, act="relu")
    on = (pre[0] > 0).to(t)
    dg, du = dy * on * pre[1].to(t), dy * on
    assert torch.equal(dx, 3 * dg - 3 * du)
    assert float(dwg) == float((dg * x).sum(dtype=torch.float64).to(t))
    assert float(dwu) == float((du * x).sum(dtype=torch.float64).to(t))


def test_bias_gradient_of_no_rows_by_very_many_columns(s):
    torch = _torch()
    N = (1 << 28) + 70
    say("no rows", N)
    e = torch.empty
    bf = torch.bfloat16
    db = s.linear_grad(e(0, N, dtype=bf, device="cuda"), e(0, 0, dtype=bf, device="cuda"),
                       e(N, 0, dtype=bf, device="cuda"), dx=False, dw=False)[2]
    assert db.shape == (N,) and not db.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_single_row_of_a_larger_tensor(s, dtype):
    # the last position of a sequence: a stride of 2^23 elements that nothing goes along
    torch = _torch()
    say("one row", dtype)
    t = getattr(torch, dtype)
    rand = _gen(12)
    T, D, N = 1 << 16, 128, 72
    x = torch.zeros(1, T, D, dtype=t, device="cuda")
    x[:, -1] = rand(1, D, t=t)
    row, w, u = x[:, -1], rand(N, D, t=t), rand(N, D, t=t)
    assert row.shape == (1, D) and row.stride(0) == 1 << 23
    one = row.clone()
    assert torch.equal(s.linear(row, w), s.linear(one, w))
    assert torch.equal(s.gated(row, w, u), s.gated(one, w, u))
    assert torch.equal(s.linear(row, rand(D, D, t=t) * 0, residual=row), one)
    _, pre = s.linear(one, w, act="silu", save=True)
    dy = rand(1, N, t=t)
    for a, b in zip(s.linear_grad(dy, row, w, act="silu", pre=pre), s.linear_grad(dy, one, w, act="silu", pre=pre)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M,V", [((1 << 21) + 9, 7), (4_000_003, 2), ((1 << 26) + 17, 1), ((1 << 20) + 3, 1040)])
def test_likelihood_of_very_many_rows(s, M, V):
    torch = _torch()
    say("likelihood", M, V)
    g = torch.Generator(device="cuda").manual_seed(6)
    dtype = torch.bfloat16 if V > 1000 else torch.float32
    z = torch.randn(M, V, device="cuda", generator=g).to(dtype)
    t = torch.randint(-1, V, (M,), device="cuda", generator=g)
    nll, total, dz = s.categorical(z, t, grad=True, scale=0.25)
    there = t >= 0
    for at in list(range(0, M, M // 5 + 1)) + [M - 30]:  # some rows of each part, and the last ones
        r = slice(at, at + 1000)
        zd, seen = z[r].double(), there[r]
        lse = torch.logsumexp(zd, 1)
        ref = torch.where(seen, lse - zd.gather(1, t[r].clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
        # (8 roundings of values of size |z|, |lse| < 16; sums of up to 1040 exponentials as a tree)
        assert ((nll[r].double() - ref).abs() <= 200 * U).all()
        p = torch.exp(zd - lse[:, None])
        p.scatter_add_(1, t[r].clamp(min=0)[:, None], -torch.ones_like(p[:, :1]))
        p *= 0.25 * seen[:, None]
        assert ((dz[r].double() - p).abs() <= 100 * U + (p.abs() * 2.0 ** -8 if V > 1000 else 0)).all()
    want = float(nll.sum(dtype=torch.float64))
    assert abs(float(total) - want) <= 1e-9 * abs(want) + 1e-9


def test_scale_in_every_call(s):
    import paper_1912_11554_amd as nuts
    torch = _torch()
    say("scales")
    ids, z = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 4, device="cuda")
    for scale in (1e39, 1e-40):
        for call in (lambda: s.embedding(ids, z, scale=scale), lambda: s.embedding_grad(ids, z, 2, scale=scale),
                     lambda: s.categorical(z, ids, grad=True, scale=scale)):
            with pytest.raises(nuts.NutsError) as e:
                call()
            assert e.value.code == nuts.NUTS_EINVAL and "scale" in str(e.value)
    big = torch.finfo(torch.float32).max
    assert torch.equal(s.embedding(ids, z, scale=big), z[:3])
    one = torch.full((1, 4), 2.0 ** 100, device="cuda")
    assert torch.equal(s.embedding(ids[:1], one, scale=2.0 ** -126), one * 2.0 ** -126)


# --------------------------------------------------------------------------
# Activations far from zero, relative to their own size.  In units of u = 2^-24
# an exponential is off by 4 (the unit's last place, the correction's rounding and
# product), a reciprocal by 2, every sum and product by 1.

def _points():
    torch = _torch()
    return torch.cat([torch.linspace(-80, 80, 40001), torch.linspace(-4, 4, 4001)]).cuda()


def _activated(s, z, act):
    """act(z) and its slope by the kernels: z as a layer of one input, and the
    gradient of its weights."""
    torch = _torch()
    one = torch.ones(1, 1, device="cuda")
    y, pre = s.linear(one, z[:, None], act=act, save=True)
    assert torch.equal(pre[0], z)
    dw = s.linear_grad(torch.ones_like(y), one, z[:, None], act=act, pre=pre, dx=False, bias=False)[1]
    return y[0].double(), dw[:, 0].double()


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_relative_error_of_the_logistic_function(s, act):
    torch = _torch()
    say("logistic", act)
    z = _points()
    zd = z.double()
    y, slope = _activated(s, z, act)
    ref, dref = _act(zd, act)
    assert ((y - ref).abs() <= 9 * U * ref.abs()).all()
    if act == "silu":  # (for z < 0; its two parts cancel near -1.28)
        p, q = torch.special.expit(zd), torch.special.expit(-zd)
        low = z < 0
        assert ((slope - dref).abs() <= 20 * U * (p + zd.abs() * p * q))[low].all()
    # the same function in the tiles' epilogue
    x = torch.ones(70, 1, device="cuda")
    assert torch.equal(s.linear(x, z[:, None], act=act), y.float().expand(70, -1))


def test_relative_error_of_the_gelu_slope(s):
    # the normal density takes 16 u; the distribution function's argument is rounded,
    # which z^2 u of its value goes with
    say("gelu slope")
    z = _points()
    z = z[z.abs() < 9]
    zd = z.double()
    torch = _torch()
    cdf, pdf = _cdf(zd), torch.exp(-zd * zd / 2) / (2 * torch.pi) ** 0.5
    slope = _activated(s, z, "gelu")[1]
    tol = (16 + 2 * zd * zd) * U * cdf + 16 * U * zd.abs() * pdf
    assert ((slope - (cdf + zd * pdf)).abs() <= tol).all()


def _slopes(s, z, act):
    """act's slope by the kernels, as the bias gradient of one row: no product
    (which would take values to multiples of 2^-133) is in the way."""
    torch = _torch()
    one = torch.ones(1, 1, device="cuda")
    _, pre = s.linear(one, z[:, None], act=act, save=True)
    return s.linear_grad(torch.ones_like(pre), one, z[:, None], act=act, pre=pre, dx=False, dw=False)[2].double()


def test_relative_error_of_the_logistic_slope(s):
    # p (1 - p): an exponential, and a reciprocal's square; silu's slope by it on both sides
    torch = _torch()
    say("logistic slope")
    z = _points()
    p, q = torch.special.expit(z.double()), torch.special.expit(-z.double())
    assert ((_slopes(s, z, "sigmoid") - p * q).abs() <= 16 * U * p * q).all()
    zd = z.double()
    assert ((_slopes(s, z, "silu") - (p + zd * p * q)).abs() <= 20 * U * (p + zd.abs() * p * q)).all()
    # NaN and infinities
    z = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda")
    for act, want in (("sigmoid", [0.0, 0.0]), ("silu", [1.0, 0.0])):
        slope = _slopes(s, z, act)
        assert torch.isnan(slope[0]) and slope[1:].tolist() == want
