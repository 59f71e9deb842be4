"""The token-model operators at the sizes that take the larger tiles of the
products (tests/token_shapes.py; tests/test_token_plan.py asks the plan), several
rows a thread, stores past the caches and more blocks than a launch, against
formulas in 64 bits on the device.

A product's error is looked at by the norm of each row and column, where a piece
in the wrong place shows at once (one product of n left out is n^-1/2 of the
norm).  With u = 2^-24 and rss the root of the sum of the products' squares:
  - the output's one rounding, as 1.03 times what rounding the exact result does;
  - an fp32 sum of n products in blocks of 32 or 16 is off by (n / 16)^1/2 u rss
    with n < 4200, fp32 factors by 4 u rss more: 64 u rss holds with a margin of 3;
  - an activation or its slope by 32 u, a product of factors by a few u;
  - a bf16 gradient's dz in two parts by at most 2^-17 of each."""
import pytest

from tests.gpu_common import say
from tests.token_shapes import TILES

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


def _act(z, kind):
    torch = _torch()
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "gelu":
        cdf = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    p, q = torch.special.expit(z), torch.special.expit(-z)
    return (p, p * q) if kind == "sigmoid" else (z * p, p + z * p * q)


def _rss(a, b):
    return ((a * a) @ (b * b)).sqrt()


def _near(got, ref, off, what):
    """Rows and columns of got against ref: one rounding, and `off` by element."""
    torch = _torch()
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    err, once = got.double() - ref, ref.to(got.dtype).double() - ref
    for dim in (0, 1):
        e, o, t = (v.norm(dim=dim) for v in (err, once, off))
        worst = int((e - 1.03 * o - t).argmax())
        assert (e <= 1.03 * o + t).all(), f"{what}, {('column', 'row')[dim]} {worst}: {e[worst]} over 1.03 {o[worst]} + {t[worst]}"


def _strided(t, more):
    """The same matrix as columns of a larger one."""
    big = _torch().full((t.shape[0], t.shape[1] + more), float("nan"), dtype=t.dtype, device="cuda")
    v = big[:, more // 2:more // 2 + t.shape[1]]
    v.copy_(t)
    return v


LINEAR = [c[1:5] for c in TILES if c[0] == "linear"]
GATED = [c[1:5] for c in TILES if c[0] == "gated"]


@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("strided", [False, True])
def test_linear_in_large_tiles(s, case, strided):
    torch = _torch()
    dtype, M, N, K = case
    t = getattr(torch, dtype)
    act = ("silu", "gelu", "sigmoid")[(M + N + K + strided) % 3]
    say("large tiles, linear", case, strided, act)
    rand = _gen(M + N + K)
    x, w, b, r, dy = rand(M, K, t=t), rand(N, K, std=K ** -0.5, t=t), rand(N, t=t), rand(M, N, t=t), rand(M, N, t=t)
    if strided:  # (rows stay on 16 bytes where they were)
        x, w, r, dy = (_strided(v, 16) for v in (x, w, r, dy))
    y, pre = s.linear(x, w, bias=b, act=act, residual=r, save=True)
    xd, wd, dyd = x.double(), w.double(), dy.double()
    z = xd @ wd.T + b.double()
    zoff = 64 * U * _rss(xd, wd.T) + 2 * U * z.abs()
    _near(pre, z, zoff, "pre")
    a, _ = _act(z, act)
    ref = a + r.double()
    _near(y, ref, 1.13 * zoff + 32 * U * (a.abs() + 1) + U * ref.abs(), "y")
    _, slope = _act(pre.double(), act)
    d = dyd * slope
    part = 64 * U + (2.0 ** -17 if dtype == "bfloat16" else 0)
    dx, dw, db = s.linear_grad(dy, x, w, act=act, pre=pre)
    _near(dx, d @ wd, part * _rss(d, wd) + 32 * U * _rss(dyd, wd), "dx")
    _near(dw, d.T @ xd, part * _rss(d.T, xd) + 32 * U * _rss(dyd.T, xd), "dw")
    _near(db[None], d.sum(0)[None], 96 * U * dyd.norm(dim=0)[None], "dbias")
    # without an activation dy itself is a factor
    dx, dw, db = s.linear_grad(dy, x, w)
    _near(dx, dyd @ wd, 64 * U * _rss(dyd, wd), "dx, none")
    _near(dw, dyd.T @ xd, 64 * U * _rss(dyd.T, xd), "dw, none")
    _near(db[None], dyd.sum(0)[None], 96 * U * dyd.norm(dim=0)[None], "dbias, none")


@pytest.mark.parametrize("case", GATED, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("strided", [False, True])
def test_gated_in_large_tiles(s, case, strided):
    torch = _torch()
    dtype, M, F, K = case
    t = getattr(torch, dtype)
    act = ("silu", "gelu")[(M + F + K + strided) % 2]
    say("large tiles, gated", case, strided, act)
    rand = _gen(M + F + K)
    x, dy = rand(M, K, t=t), rand(M, F, t=t)
    wg, wu = rand(F, K, std=K ** -0.5, t=t), rand(F, K, std=K ** -0.5, t=t)
    if strided:
        x, wg, wu, dy = (_strided(v, 16) for v in (x, wg, wu, dy))
    y, pre = s.gated(x, wg, wu, act=act, save=True)
    xd, gd, ud, dyd = x.double(), wg.double(), wu.double(), dy.double()
    g, u = xd @ gd.T, xd @ ud.T
    goff, uoff = 64 * U * _rss(xd, gd.T), 64 * U * _rss(xd, ud.T)
    _near(pre[0], g, goff, "g")
    _near(pre[1], u, uoff, "u")
    a, _ = _act(g, act)
    _near(y, a * u, (1.13 * goff + 32 * U * (a.abs() + 1)) * u.abs() + a.abs() * uoff + 2 * U * (a * u).abs(), "y")
    g, u = pre[0].double(), pre[1].double()
    a, slope = _act(g, act)
    dg, du, most = dyd * u * slope, dyd * a, dyd * u
    part = 64 * U + (2.0 ** -17 if dtype == "bfloat16" else 0)
    dx, dwg, dwu = s.gated_grad(dy, x, wg, wu, pre, act=act)
    _near(dx, dg @ gd + du @ ud, part * (_rss(dg, gd) + _rss(du, ud)) + 32 * U * (_rss(most, gd) + _rss(dyd * (a.abs() + 1), ud)), "dx")
    _near(dwg, dg.T @ xd, part * _rss(dg.T, xd) + 32 * U * _rss(most.T, xd), "dwg")
    _near(dwu, du.T @ xd, part * _rss(du.T, xd) + 32 * U * _rss((dyd * (a.abs() + 1)).T, xd), "dwu")


@pytest.mark.parametrize("case", [c for c in TILES if c[5][1][0] > 64], ids=lambda c: "-".join(map(str, c[:5])))
def test_limits_in_large_tiles(s, case):
    # an infinity in x touches one column of dw, one in w one column of dx, whatever dz's parts; all else keeps its bits
    torch = _torch()
    kind, dtype, M, N, K, _ = case
    t, inf = getattr(torch, dtype), float("inf")
    say("limits in large tiles", case[:5])
    rand = _gen(M + N)
    x, w, w2, dy = rand(M, K, t=t), rand(N, K, t=t), rand(N, K, t=t), rand(M, N, t=t)
    pre = rand(2, M, N)

    def call():
        if kind == "gated":
            return s.gated_grad(dy, x, w, w2, pre)[:2]
        return s.linear_grad(dy, x, w, act="silu", pre=pre[0], bias=False)[:2]

    clean = call()
    x[M - 2, 3], w[N - 3, 11] = -inf, inf
    d = dy.double() * _act(pre[0].double(), "silu")[1] * (pre[1].double() if kind == "gated" else 1)
    for got, was, col, sign in zip(call(), clean, (11, 3), (d[:, N - 3], -d[M - 2])):
        want = torch.where(sign > 0, inf, -inf).to(t)
        assert (sign != 0).all() and torch.equal(got[:, col], want)
        rest = [c for c in range(K) if c != col]
        assert torch.equal(got[:, rest], was[:, rest])


# --------------------------------------------------------------------------
# The embedding: several rows a thread, stores past the caches, blocks past a launch.

def _ids(N, V, seed):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = (V * torch.rand(N, device="cuda", generator=g, dtype=torch.float64) ** 3).long()
    ids[torch.rand(N, device="cuda", generator=g) < 0.1] = -1
    ids[N // 2], ids[N - 1] = V, V - 1
    return ids


# (a 16-byte run a thread, whole runs and overlapping ones; one element a thread; 128 MB and more)
EMBEDDINGS = [(4201, 300, 1024), (5003, 2000, 1001), (70001, 50, 3), (16501, 500, 4096), (33001, 70, 1028),
              (3001, 16500, 4096), (40000, 33000, 1032)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("case", EMBEDDINGS)
def test_large_embeddings(s, case, dtype):
    torch = _torch()
    N, V, D = case
    t = getattr(torch, dtype)
    say("large embedding", case, dtype)
    rand, ids, scale = _gen(N + V), _ids(N, V, D), 1.75
    table, dout = rand(V, D, t=t), rand(N, D, t=t)
    there = (ids >= 0) & (ids < V)
    at = torch.where(there, ids, 0)
    # (one product, rounded to fp32 and to the type)
    want = torch.where(there[:, None], (table.float() * scale).to(t)[at], torch.zeros((), dtype=t, device="cuda"))
    assert torch.equal(s.embedding(ids, table, scale=scale), want)
    assert torch.equal(s.embedding(ids, _strided(table, 5), scale=scale), want)
    got = s.embedding_grad(ids, dout, V, scale=scale)
    rows = dout[there].double() * scale
    ref = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, at[there], rows)
    size = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, at[there], rows.abs())
    n = torch.bincount(at[there], minlength=V)[:, None].double()
    once = ref.abs() * (2.0 ** -8 if dtype == "bfloat16" else U)
    assert ((got.double() - ref).abs() <= (n + 2) * U * size + 1.01 * once).all()
    assert not got[(n == 0)[:, 0]].any()
    assert torch.equal(got, s.embedding_grad(ids, dout, V, scale=scale))
    # rows off the 16-byte grid are stored through the caches: the same values
    out = torch.full((V, D + 1), 3.0, dtype=t, device="cuda")
    s.embedding_grad(ids, dout, V, scale=scale, out=out[:, 1:])
    assert torch.equal(out[:, 1:], got) and (out[:, 0] == 3).all()


def test_embedding_of_very_many_tokens(s):
    torch = _torch()
    N, V = (1 << 29) + 77, 1000
    say("very many tokens", N)
    table = _gen(1)(V, 1, t=torch.bfloat16)
    ids = torch.arange(N, device="cuda")
    ids %= V + 1  # (V: no token)
    out = s.embedding(ids, table, scale=2.0)
    want = torch.cat([2 * table[:, 0], torch.zeros(1, dtype=torch.bfloat16, device="cuda")])
    whole = N // (V + 1) * (V + 1)
    assert (out[:whole, 0].view(-1, V + 1) == want).all() and torch.equal(out[whole:, 0], want[:N - whole])


def test_embedding_gradient_of_very_many_classes(s):
    torch = _torch()
    N, V = 5000, (1 << 29) + 77
    say("very many classes", V)
    ids = torch.randperm(N, device="cuda") * (V // N)
    ids[7] = V - 1
    dout = _gen(2)(N, 1, t=torch.bfloat16)
    got = s.embedding_grad(ids, dout, V)
    assert torch.equal(got[ids], dout)
    assert int((got != 0).sum()) == int((dout != 0).sum())
