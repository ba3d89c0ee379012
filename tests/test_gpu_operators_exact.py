"""The operators on inputs whose sums are exact or short, so that the bounds are a few
roundings whatever the row's length: a lost or doubled term, and a digit given
away, show.  u = 2^-24 is fp32's half step.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1802_08435_amd import ops  # noqa: E402

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = math.inf
MIX = pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def within(got, ref, tol, what):
    err = (got.double() - ref.double()).abs()
    assert bool((err <= tol).all()), f"{what}: worst {float((err / tol).max()):.3g} times the tolerance"


# ---- log probabilities ------------------------------------------------------------


@MIX
@pytest.mark.parametrize("offset", [0.0, 48.0, 1000.0])
@pytest.mark.parametrize("n,v", [(5, 16), (70, 256), (3, 1000), (2, 2048), (2, 4096), (520, 5000), (1, 70000)])
def test_log_probabilities_do_not_depend_on_a_common_offset(n, v, offset, dt):
    """One class 12 ahead of the next and 200 of the others: log P is -6.1e-6 and -12 to the last digits,
    whatever all logits have in common.  s = 1 + e^-12 is off by two roundings, its logarithm by as much,
    the differences to the largest logit not at all."""
    z = torch.full((n, v), offset - 200.0, device="cuda")
    i = torch.arange(n, device="cuda")
    a, b = (7 * i + 3) % v, (11 * i + v // 2 + 5) % v
    b = torch.where(a == b, (b + 1) % v, b)
    z[i, a], z[i, b] = offset, offset - 12.0
    z = z.to(dt)
    zd = z.double()
    assert bool((zd[i, a] - zd[i, b] == 12.0).all())
    d = zd - zd.amax(-1, keepdim=True)
    ref = d - torch.log(torch.exp(d).sum(-1, keepdim=True))
    for tok in (a, b):
        for top in {2, 3, min(20, v)}:
            r = ops.token_logprobs(z, tok, top=top)
            want = ref[i, tok]
            within(r["logp"], want, 4 * U + 4 * U * want.abs(), "logp")
            assert torch.equal(r["top_idx"][:, :2], torch.stack([a, b], 1).int())
            want = ref.gather(-1, r["top_idx"].long())
            within(r["top_logp"], want, 4 * U + 4 * U * want.abs(), "top_logp")


def test_log_probabilities_of_rows_at_a_mask_s_value():
    """Every class at fp32's lowest or largest value: lse is that value, logp 0, the entropy log V; with a +inf, NaN."""
    for v in (16, 256, 5000, 70000):
        z = torch.stack([torch.full((v,), x, device="cuda") for x in (torch.finfo(F32).min, torch.finfo(F32).max, 1e29)])
        z[2, 1:] = INF
        r = ops.token_logprobs(z, torch.zeros(3, dtype=torch.int64, device="cuda"), top=3)
        assert torch.equal(r["lse"][:2], z[:2, 0]) and torch.equal(r["logp"][:2], torch.zeros(2, device="cuda"))
        assert torch.equal(r["top_logp"][:2], torch.zeros(2, 3, device="cuda"))
        within(r["entropy"][:2], torch.full((2,), math.log(v), device="cuda"), 4 * U * math.log(v), "entropy")
        assert all(bool(torch.isnan(r[k][2]).all()) for k in ("logp", "entropy", "lse", "top_logp"))


# ---- layer norm ------------------------------------------------------------


HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
WIDTHS = [33, 64, 257, 1000, 2048, 4099, 9000, 20001]


def depth(d):
    """Roundings on an element's way into a row's sum: up to 32 columns a thread, wide rows d / 1,024, and the threads'."""
    return max(32, d // 1024 + 8) + 16


@MIX
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_far_from_zero_keep_the_digits_of_their_spread(d, dt):
    """Steps of the type at 10,000 (fp32) or 1,024: x - m' is exact, so the result is off by the differences' sums
    alone, whose size is the spread's and the first mean's error e = depth u |x|."""
    off, step = {F32: (1e4, 0.125), F16: (1024.0, 1.0), BF16: (1024.0, 8.0)}[dt]
    g = torch.Generator(device="cuda").manual_seed(d)
    x = (off + step * torch.randint(0, 9, (7, d), generator=g, device="cuda")).to(dt)
    xd = x.double()
    m = xd.mean(-1, keepdim=True)
    var = ((xd - m) ** 2).mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt(var + 1e-5)
    h = (xd - m) * r
    k, e = depth(d), depth(d) * U * off
    size = var.sqrt() + e
    rel = (k + 8) * U * 2 * (var + e * e) / (var + 1e-5) + 4 * U
    y, mean, rstd = ops.layer_norm(x, stats=True)
    within(y, h, (k + 4) * U * size * r + 2 * U * (h.abs() + e * r) + h.abs() * rel + HALF[dt] * h.abs() * 1.001 + 2.0 ** -25,
           "y")
    within(mean, m[:, 0], U * off + (k + 4) * U * size[:, 0], "mean")
    within(rstd, r[:, 0], r[:, 0] * rel[:, 0], "rstd")


@pytest.mark.parametrize("d", WIDTHS)
def test_constant_rows_are_beta_wherever_they_lie(d):
    """Variance 0: what is left of x - m is (depth u) of the first mean's error depth u |x|, times 1 / sqrt(eps)."""
    for c in (0.1, 1e3 / 3, 1e6 / 3):
        beta = torch.arange(float(d), device="cuda")
        y, mean, rstd = ops.layer_norm(torch.full((3, d), c, device="cuda"), None, beta, eps=1e-5, stats=True)
        x = float(torch.tensor(c, dtype=F32))
        e = (depth(d) + 4) * U
        within(y, beta, e * e * x * 1e-5 ** -0.5 + 2 * U * beta.abs(), "y")
        within(mean, torch.full_like(mean, x), 2 * U * x, "mean")


def whole(*shape, seed, dt=F32, most=3):
    """Whole numbers -most .. most: sums of them are exact below 2^24."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda", dtype=torch.int8).to(dt)


@pytest.mark.parametrize("n", [0, 3])
def test_weight_gradients_of_the_widest_rows(n):
    """dgamma and dbeta of more than 2^27 columns, whose parts take more sums than a grid has room for."""
    d = (1 << 27) + 5
    x, dy = whole(n, d, seed=1, dt=BF16, most=1), whole(n, d, seed=2, dt=BF16)
    mean, rstd = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, mean, rstd, out=dy.clone() if n else None)
    assert torch.equal(dbeta, dy.sum(0, dtype=F32)) and torch.equal(dgamma, (dy * x).sum(0, dtype=F32))


NORM_SIZES = [(1, 1), (3, 2), (5, 7), (200, 16), (9, 63), (1600, 64), (17, 65), (33, 257), (12, 768), (7, 1000), (5, 1001),
              (6, 1024), (3, 2048), (4, 4096), (3, 4099), (2, 8192), (3, 8200), (3, 12001), (2, 40000), (5000, 24), (20001, 8),
              (3000, 768)]


@MIX
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_layer_norm_of_rows_with_exact_sums(n, d, dt):
    """Whole numbers that come in pairs x, -x: the mean is 0 and the sum of squares exact, so the statistics
    are off by the last operations' roundings alone."""
    g = torch.Generator(device="cuda").manual_seed(d)
    half = torch.randint(1, 4, (n, d // 2), generator=g, device="cuda")
    x = torch.cat([half, -half, torch.zeros(n, d % 2, device="cuda")], 1)
    x = x.gather(1, torch.rand(n, d, generator=g, device="cuda").argsort(1)).to(dt)
    y, mean, rstd = ops.layer_norm(x, stats=True)
    r = 1.0 / torch.sqrt((x.double() ** 2).mean(-1) + 1e-5)
    assert torch.equal(mean, torch.zeros(n, device="cuda"))
    within(rstd, r, 6 * U * r, "rstd")
    ref = x.double() * r[:, None]
    within(y, ref, 9 * U * ref.abs() + HALF[dt] * ref.abs() * 1.001 + 2.0 ** -25, "y")


@MIX
@pytest.mark.parametrize("d", [5, 16, 65, 257, 1001, 4099, 8200, 12001, 40000])
def test_layer_norm_of_rows_with_one_element(d, dt):
    """The only element that is not 0 at either end of the row and of what the threads, the waves and the rounds
    of a block take: mean 3 / d, which one element left out makes 0."""
    vw = 4 if dt == F32 else 8
    at = {vw * k + i for k in (1, 15, 16, 64, 256, 512, 1024, 2048, 4096) for i in (-1, 0)}
    at |= {0, 1, d // 2, d - 1, d - 2, d - vw}
    at = torch.tensor(sorted(p for p in at if 0 <= p < d), device="cuda")
    x = torch.zeros(len(at), d, device="cuda", dtype=dt)
    x[torch.arange(len(at), device="cuda"), at] = 3.0
    y, mean, rstd = ops.layer_norm(x, stats=True)
    m = 3.0 / d
    r = 1.0 / math.sqrt(9.0 / d - m * m + 1e-5)
    k = (depth(d) + 16) * U
    within(mean, torch.full_like(mean, m).double(), k * m + 2.0 ** -23 * m, "mean")
    within(rstd, torch.full_like(rstd, r).double(), k * r + 2.0 ** -23 * r, "rstd")
    ref = (x.double() - m) * r
    within(y, ref, 4 * k * (ref.abs() + m * r) + HALF[dt] * ref.abs() * 1.001 + 2.0 ** -25, "y")


@MIX
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_layer_norm_gradient_with_exact_sums(n, d, dt):
    """x of -1, 0 and 1 with mean 0 and rstd 1 given, whole dy and gamma: dgamma, dbeta and both sums of dx are exact."""
    x, dy = whole(n, d, seed=d, dt=dt, most=1), whole(n, d, seed=n + d, dt=dt)
    gamma = whole(d, seed=3, dt=dt, most=2)
    mean, rstd = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    h, g = x.double(), dy.double() * gamma.double()
    m0, m1 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    ref = g - h * m1 - m0
    for weights in (True, False):
        dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, mean, rstd, gamma, weights=weights)
        within(dx, ref, U * (4 * (m0.abs() + m1.abs()) + 2 * ref.abs()) + HALF[dt] * ref.abs() * 1.001 + 2.0 ** -25, "dx")
        if weights:
            assert torch.equal(dgamma, (dy.double() * h).sum(0).float()), "dgamma"
            assert torch.equal(dbeta, dy.double().sum(0).float()), "dbeta"


# ---- the table's gradient ------------------------------------------------------------


def ids_for(kind, n, v, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if kind == "one":
        return torch.full((n,), v // 2, device="cuda", dtype=torch.int64)
    ids = (((v + 1.0) ** u - 1.0) if kind == "skew" else u * v).long().clamp(0, v - 1)
    return ids.sort()[0] if kind == "sorted" else ids


@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (31, 5, 3), (257, 300, 65), (1600, 97, 64), (900, 33, 1000), (70, 9, 4099),
                                   (2047, 256, 9), (2048, 256, 100), (2049, 256, 17), (4096, 3, 40), (8193, 4, 257),
                                   (33000, 1, 40),
                                   (200000, 20, 16), (500000, 8, 33), (1023, 700, 48), (1025, 700, 48), (4096, 100000, 16),
                                   (4097, 70000, 24), (16384, 300, 7), (16385, 300, 7), (70001, 65537, 32), (70001, 3000, 1024),
                                   (300000, 50000, 8), (2200000, 1000, 8), (700001, 400, 4)])
@pytest.mark.parametrize("kind", ["even", "skew", "one", "sorted"])
def test_embed_gradient_with_exact_sums(n, v, d, kind):
    """Whole numbers and a scale of a power of two: a row lost or taken twice changes the sum, and nothing else does."""
    dout, ids = whole(n, d, seed=n + d, dt=BF16), ids_for(kind, n, v)
    ids[::11] = -1
    ids[5::13] = v
    on = (ids >= 0) & (ids < v)
    ref = torch.zeros(v, d, dtype=torch.int32, device="cuda").index_add_(0, ids[on], dout[on].int())
    for out in (F32, BF16):
        want = (ref.double() * 0.25).float().to(out)
        assert torch.equal(ops.embed_grad(dout, ids, v, scale=0.25, dtype=out), want), out


# ---- log probabilities: sums ------------------------------------------------------------


LOGP_SIZES = [(1, 1), (3, 2), (2, 15), (70, 16), (9, 17), (5, 63), (7, 65), (4, 255), (101, 256), (5, 257), (3, 511), (2, 513),
              (3, 1000), (3, 1025), (2, 2047), (2, 2049), (3, 4096), (2, 4099), (3, 8193), (1, 16385), (2, 40001), (1, 65537),
              (1, 131072), (520, 5001), (513, 40001)]


@MIX
@pytest.mark.parametrize("n,v", LOGP_SIZES)
def test_log_probabilities_of_equal_classes(n, v, dt):
    """s = V, exact in fp32 in any order: the logarithm's rounding and a subtraction's are all there is."""
    z = torch.full((n, v), 1.5, device="cuda", dtype=dt)
    r = ops.token_logprobs(z, torch.arange(n, device="cuda") * 7 % v, top=min(5, v))
    lv = math.log(v)
    within(r["logp"], torch.full((n,), -lv, device="cuda").double(), 4 * U * lv, "logp")
    within(r["entropy"], torch.full((n,), lv, device="cuda").double(), 4 * U * lv, "entropy")
    within(r["lse"], torch.full((n,), 1.5 + lv, device="cuda").double(), 4 * U * (1.5 + lv), "lse")
    assert torch.equal(r["top_idx"], torch.arange(min(5, v), device="cuda", dtype=torch.int32).expand(n, -1))


@MIX
@pytest.mark.parametrize("n,v", [(3, 257), (2, 513), (3, 1000), (2, 2049), (2, 4099), (1, 5000), (3, 8193), (1, 16385),
                                 (2, 40001), (1, 65537), (1, 131072), (513, 40001), (2, 65543)])
def test_log_probabilities_of_classes_at_the_borders(n, v, dt):
    """All classes masked but the first and last of each segment that a row of any length could be cut into, of the
    vectors there, of a block's rounds, and the row's last vector: s is their number."""
    at = set(range(max(0, v - 9), v)) | {0, 1, v // 2}
    for seg in {-(-(-(-v // k)) // 8) * 8 for k in (2, 3, 4, 5, 8, 9, 16, 17)} | {1024, 2048, 4096, 8192}:
        for j in range(seg, v, seg):
            at |= {j - 1, j}
    at = torch.tensor(sorted(at), device="cuda")
    if len(at) > 400:
        at = torch.cat([at[:200], at[-200:]])
    z = torch.full((n, v), -INF, device="cuda", dtype=dt)
    z[:, at] = -2.5
    k = len(at)
    top = min(32, k)
    r = ops.token_logprobs(z, at[torch.arange(n, device="cuda") % k], top=top)
    lk = math.log(k)
    within(r["logp"], torch.full((n,), -lk, device="cuda").double(), 4 * U * lk, "logp")
    within(r["entropy"], torch.full((n,), lk, device="cuda").double(), 4 * U * lk, "entropy")
    within(r["lse"], torch.full((n,), lk - 2.5, device="cuda").double(), 4 * U * (lk + 2.5), "lse")
    assert torch.equal(r["top_idx"], at[:top].int().expand(n, -1))
    # the gradient reaches each of them, and no masked class: p = 1 / k off by lse's rounding, exp's argument's and its own
    g = torch.ones(n, device="cuda")
    dz = ops.token_logprobs_grad(z, None, r["lse"], g_lse=g)
    p = torch.zeros(v, device="cuda", dtype=torch.float64)
    p[at] = 1.0 / k
    half = {F32: 0.0, BF16: 2.0 ** -8, F16: 2.0 ** -11}[dt]
    within(dz, p.expand(n, v), p * (U * (4 * (lk + 2.5) + 4 * lk + 8) + half * 1.001), "dlogits")


@MIX
@pytest.mark.parametrize("n,v", LOGP_SIZES)
def test_log_probabilities_by_the_sums_real_depth(n, v, dt):
    """Random rows with the bound of how the sums are made: a thread adds up to max(64, V / 256) terms, rescaled V / 4,096
    times at most, the threads and segments are joined in 16 steps; a term's exponent is off by
    (2 |d| + 4) u, and by as much again over its rescalings."""
    g = torch.Generator(device="cuda").manual_seed(n + v)
    z = (3.0 * torch.randn(n, v, generator=g, device="cuda")).to(dt)
    zd = z.double()
    m = zd.amax(-1)
    d = zd - m[:, None]
    e = torch.exp(d)
    s = e.sum(-1)
    p = e / s[:, None]
    e1, e2 = (p * d.abs()).sum(-1), (p * d * d).sum(-1)
    steps = max(64, v // 256) + 16 + 4 * (v // 4096 + 16) + 8
    rel = U * (steps + 4 * e1)
    ls = torch.log(s)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    r = ops.token_logprobs(z, t)
    lp = zd.gather(1, t[:, None])[:, 0] - m - ls
    within(r["logp"], lp, rel + U * (4 * ls.abs() + 2 * lp.abs() + 2 * (lp + ls).abs()) + 1e-30, "logp")
    within(r["lse"], m + ls, rel + U * (4 * ls.abs() + 2 * (m + ls).abs()) + 1e-30, "lse")
    h = ls + e1
    within(r["entropy"], h, rel * (1 + e1) + U * (e1 * steps + 4 * e2 + 4 * ls.abs() + 4 * e1 + 2 * h) + 1e-30, "entropy")


# ---- results that a caller leaves out ------------------------------------------------------------


def _addr(t):
    return None if t is None else t.data_ptr()


@pytest.mark.parametrize("n,v,top", [(50, 256, 3), (3, 5000, 0), (2, 70000, 8)])
def test_token_logprobs_without_some_of_its_results(n, v, top):
    from paper_1802_08435_amd import wavernn as W
    g = torch.Generator(device="cuda").manual_seed(v)
    z, t = torch.randn(n, v, generator=g, device="cuda"), torch.randint(-1, v, (n,), generator=g, device="cuda")
    want = ops.token_logprobs(z, t, top=top)
    L, st = W.lib(), torch.cuda.current_stream().cuda_stream
    size = max(L.wavernn_token_logprobs_workspace(n, v, top), 16)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for names in (("logp",), ("entropy",), ("lse",), ("logp", "lse"), ()):
        out = {k: torch.full((n,), 7.0, device="cuda") for k in names}
        tl, ti = torch.empty(n, top, device="cuda"), torch.empty(n, top, dtype=torch.int32, device="cuda")
        W._check(L.wavernn_token_logprobs(W.F32, z.data_ptr(), n, v, v, t.data_ptr(), 8, top, _addr(out.get("logp")),
                                          _addr(out.get("entropy")), _addr(out.get("lse")), _addr(tl) if top else None,
                                          _addr(ti) if top else None, ws.data_ptr(), size, st))
        assert all(torch.equal(out[k], want[k]) for k in names)
        if top:
            assert torch.equal(tl, want["top_logp"]) and torch.equal(ti, want["top_idx"])


@MIX
@pytest.mark.parametrize("n,d", [(2, 40), (700, 40), (50, 257), (700, 1001), (40, 9001), (3, 20000)])
def test_layer_norm_gradient_without_some_of_its_results(n, d, dt):
    from paper_1802_08435_amd import wavernn as W
    x, dy = whole(n, d, seed=d, dt=dt, most=1), whole(n, d, seed=n, dt=dt)
    _, mean, rstd = ops.layer_norm(x, stats=True)
    names = ("dx", "dgamma", "dbeta")
    want = dict(zip(names, ops.layer_norm_grad(dy, x, mean, rstd)))
    L, st = W.lib(), torch.cuda.current_stream().cuda_stream
    size = max(L.wavernn_layer_norm_grad_workspace(n, d), 16)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    code = {F32: W.F32, BF16: W.BF16, F16: W.F16}[dt]
    for use in (("dgamma", "dbeta"), ("dgamma",), ("dbeta",), ("dx", "dgamma"), ("dx", "dbeta"), ("dx",), ()):
        out = {k: torch.full_like(want[k], 7.0) for k in use}
        W._check(L.wavernn_layer_norm_grad(code, dy.data_ptr(), d, x.data_ptr(), d, n, d, W.F32, None, mean.data_ptr(),
                                           rstd.data_ptr(), _addr(out.get("dx")), d, _addr(out.get("dgamma")),
                                           _addr(out.get("dbeta")), ws.data_ptr(), size, st))
        assert all(torch.equal(out[k], want[k]) for k in use), use


@pytest.mark.parametrize("d", [64, 1000, 9000])
def test_rows_whose_variance_overflows_are_beta(d):
    """Spreads past fp32's range (finite sums): 1 / sqrt(inf) leaves beta, whatever is left of the mean."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x, beta = 1e33 * torch.randn(3, d, generator=g, device="cuda"), torch.arange(float(d), device="cuda")
    y, mean, rstd = ops.layer_norm(x, None, beta, stats=True)
    assert torch.equal(y, beta.expand(3, d)) and torch.equal(rstd, torch.zeros(3, device="cuda"))
