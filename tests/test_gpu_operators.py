"""The operators on callers' tensors against their formulas in 64 bits.

Tolerances, from the number formats alone.  u = 2^-24 is fp32's half step.  A
kernel's fp32 sum of n terms is off by at most (n + 1) u times the sum of the terms'
sizes whatever its order, exp(x) in fp32 by (2 |x| + 4) u of its value (the
argument's rounding and the function's last bit), and a result's own rounding
by eps / 2 of its type (bf16 2^-8, fp16 2^-11), below the type's normal range by half its
smallest step.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1802_08435_amd import ops  # noqa: E402

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -125, BF16: 2.0 ** -125, F16: 2.0 ** -25}
INF, NAN = math.inf, math.nan
MIX = pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(*shape, seed=0, dt=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen(seed), device="cuda") * scale).to(dt)


def close(got, ref, tol, what=""):
    """Equal where ref is not finite, within tol elsewhere."""
    got, ref = got.double(), ref.double()
    ref = torch.where(ref.abs() >= 2.0 ** 128, torch.sign(ref) * INF, ref)   # past fp32: rounds to infinity
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    assert torch.equal(got[torch.isinf(ref)], ref[torch.isinf(ref)]), f"{what}: infinities differ"
    err = (got - ref).abs()
    bad = fin & ~(err <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol)[bad].max()):.3g} times "
                           f"the tolerance at {bad.nonzero()[0].tolist()}")


# ---- log probabilities ------------------------------------------------------------


def ref_logp(z, tokens, top):
    """(logp, entropy, lse, top_logp, top_idx, tol) in 64 bits; z [n, v] as the kernel gets it."""
    n, v = z.shape
    z = z.double()
    dead = (z == -INF).all(-1)
    nan = torch.isnan(z).any(-1) | (z == INF).any(-1)
    m = torch.where(dead | nan, 0.0, z.amax(-1))
    d = z - m[:, None]
    e = torch.exp(d)
    s = e.sum(-1)
    lse = torch.where(nan, NAN, m + torch.log(s))
    ent = torch.log(s) - (e * torch.where(e > 0, d, 0.0)).sum(-1) / s
    ent = torch.where(dead, 0.0, ent)
    ent = torch.where(nan, NAN, ent)
    sub = torch.where(dead, 0.0, lse)
    t = torch.zeros(n, dtype=torch.int64, device="cuda") if tokens is None else tokens.long()
    pad = t < 0
    logp = z.gather(-1, t.clamp(0, v - 1)[:, None])[:, 0] - sub
    logp = torch.where(t >= v, NAN, logp)
    logp = torch.where(nan, NAN, logp)
    order = torch.where(torch.isnan(z), INF, z)
    # NaN above +inf: two stable sorts, by value and then by being NaN
    idx = torch.sort(order, dim=-1, descending=True, stable=True)[1]
    k2 = torch.sort(torch.isnan(z).gather(-1, idx).to(torch.uint8), dim=-1, descending=True, stable=True)[1]
    idx = idx.gather(-1, k2)[:, :top]
    top_logp = z.gather(-1, idx) - sub[:, None]
    top_logp = torch.where(nan[:, None], NAN, top_logp)
    # sum of at most v terms, the exponent's error weighed by p (|d| p sums to less than log v + 1), logs and
    # the subtractions of values as large as the largest logit
    zmax = torch.where(torch.isfinite(z) & (z.abs() < 1e30), z.abs(), 0.0).amax(-1)
    tol = U * (v + 16 + 2 * (math.log(v) + 1) + 8 * (zmax + math.log(v)))
    zero = lambda x: torch.where(pad if x.dim() == 1 else pad[:, None], torch.zeros((), dtype=x.dtype, device="cuda"), x)
    return (zero(logp), zero(ent), zero(lse), zero(top_logp), torch.where(pad[:, None], -1, idx).int(), tol)


def check_logp(z, tokens, top, **kw):
    r = ops.token_logprobs(z, tokens, top=top, **kw)
    zz = z.reshape(-1, z.shape[-1])
    tt = None if tokens is None else tokens.reshape(-1)
    n = zz.shape[0]
    logp, ent, lse, tl, ti, tol = ref_logp(zz, tt, top)
    v = zz.shape[1]
    # a logit far below the maximum is a large number of its own: its difference is rounded too
    far = lambda x: tol + 4 * U * torch.where(torch.isfinite(x), x.abs(), 0.0)
    if tokens is not None:
        close(r["logp"].reshape(n), logp, far(logp), "logp")
    close(r["entropy"].reshape(n), ent, tol * (2 + math.log(v)), "entropy")
    close(r["lse"].reshape(n), lse, far(lse), "lse")
    if top:
        assert torch.equal(r["top_idx"].reshape(n, top), ti), "alternatives differ"
        close(r["top_logp"].reshape(n, top), tl, tol[:, None] + 4 * U * torch.where(torch.isfinite(tl), tl.abs(), 0.0), "top_logp")
    return r


def tokens_for(n, v, seed=1, dtype=torch.int64):
    return torch.randint(0, v, (n,), generator=gen(seed), device="cuda").to(dtype)


SIZES = [(1, 1), (3, 2), (5, 3), (2, 15), (700, 16), (9, 17), (4, 33), (5, 63), (6, 64), (7, 65), (3, 100), (4, 255),
         (1001, 256), (5, 257), (3, 511), (2, 513), (3, 1000), (2, 1024), (3, 1025), (2, 2047), (3, 4096), (2, 4099),
         (3, 8193), (1, 16385), (2, 20000), (1, 65536), (3, 65537), (1, 131072), (600, 5000)]


@MIX
@pytest.mark.parametrize("n,v", SIZES)
def test_logprobs_sizes(n, v, dt):
    z = randn(n, v, seed=n + v, dt=dt, scale=3.0)
    for top in sorted({0, 1, min(5, v), min(32, v)}):
        check_logp(z, tokens_for(n, v), top)


@MIX
@pytest.mark.parametrize("n,v", [(9, 16), (9, 256), (5, 1000), (4, 5000), (2, 70000)])
def test_logprobs_special_rows(n, v, dt):
    """Padding (its logits NaN), every class masked, masks by -inf and by the type's lowest value, fewer
    classes left than alternatives asked for, all equal, NaN, +inf, zeros of both signs."""
    z = randn(14, v, seed=v, dt=dt, scale=3.0)
    lowest = torch.finfo(dt).min
    t = tokens_for(14, v)
    z[0] = NAN
    t[0] = -1
    z[1] = -INF
    z[2, : v - 2] = -INF
    t[2] = v - 1
    z[3] = -INF
    z[3, v // 2] = 1.5
    t[3] = 0
    z[4] = 0.25
    z[5, v // 3] = NAN
    z[6, v // 3] = INF
    z[7] = 0.0
    z[7, ::2] = -0.0
    z[8, : v // 2] = lowest
    z[9] = lowest
    z[10] = torch.finfo(dt).max
    z[11] = lowest
    z[11, v - 1] = torch.finfo(dt).max
    z[12, v // 2:] = -INF
    t[12] = v
    z[13, 0] = NAN
    z[13, 1] = INF
    t[13] = v + 5
    for top in (1, 4, min(v, 32)):
        check_logp(z, t, top)


@pytest.mark.parametrize("v", [256, 4096, 40000, 131072])
@pytest.mark.parametrize("order", ["rising", "falling", "clustered", "same16", "few", "apart", "three"])
def test_logprobs_alternatives_in_any_place(v, order):
    """The alternatives may lie anywhere: side by side, at one distance, among many equal ones."""
    j = torch.arange(v, device="cuda", dtype=F32)
    z = {"rising": j / v, "falling": -j / v, "clustered": torch.where((j > v // 2) & (j < v // 2 + 70), 2.0 + j / v, 0.0),
         "same16": (j % 16 == 3) * (1.0 + j / v), "few": torch.floor(j / (v / 5.0)),
         # a thousand large ones 1,024 or 2,048 classes apart and next to those; all but three masked
         "apart": torch.where(j % 2048 < 64, 1.0 + j / v, 0.0),
         "three": torch.where((j == 3) | (j == v // 2) | (j == v - 1), j / v, -INF)}[order]
    z = torch.stack([z, z.flip(0), z[torch.randperm(v, generator=gen(2), device="cuda")]])
    for dt in (F32, BF16):
        for top in (1, 7, 32):
            check_logp(z.to(dt), tokens_for(3, v), top)


@pytest.mark.parametrize("order", ["apart", "few", "three", "equal"])
def test_logprobs_alternatives_of_many_long_rows(order):
    """Enough rows that none is taken in segments, and more classes tie or lie close than are ranked at once."""
    n, v = 520, 40000
    j = torch.arange(v, device="cuda", dtype=F32)
    z = {"apart": torch.where(j % 2048 < 64, 1.0 + j / v, 0.0), "few": torch.floor(j / (v / 5.0)),
         "three": torch.where((j == 3) | (j == v // 2) | (j == v - 1), j / v, -INF), "equal": torch.zeros_like(j)}[order]
    z = torch.stack([torch.roll(z, 64 * i) for i in range(n)])
    for dt, top in ((F32, 9), (BF16, 9), (F16, 32)):
        check_logp(z.to(dt), tokens_for(n, v), top)


@MIX
def test_logprobs_views_and_token_types(dt):
    base = randn(6, 10, 300, seed=4, dt=dt, scale=2.0)
    for z in (base, base[:, :, 7:263], base[:, ::2, 1:258], base[2], base[1, 1], base[:, 3, 5:21]):
        check_logp(z, tokens_for(z.numel() // z.shape[-1], z.shape[-1], dtype=torch.int32).reshape(z.shape[:-1]), 3)
    one = randn(1, 77, seed=5, dt=dt)
    check_logp(one.expand(5, 77), tokens_for(5, 77), 4)
    check_logp(base[:, :, :256], None, 4)
    r = ops.token_logprobs(randn(0, 40, dt=dt), tokens_for(0, 40), top=2)
    assert r["logp"].shape == (0,) and r["top_idx"].shape == (0, 2)


def test_logprobs_far_rows():
    """Row offsets past 2^31 elements."""
    step = 2 ** 30 + 5
    store = torch.zeros(2 * step + 400, dtype=BF16, device="cuda")
    z = store.as_strided((3, 300), (step, 1))
    z.copy_(randn(3, 300, seed=8, dt=BF16))
    t = tokens_for(3, 300)
    r = check_logp(z, t, 5)
    dz = ops.token_logprobs_grad(z, t, r["lse"], g_logp=torch.ones(3, device="cuda"), out=z)
    assert dz.data_ptr() == z.data_ptr() and float(dz[2].float().abs().sum()) > 0.1
    assert float(store[300:step].float().abs().max()) == 0.0


def grad_formula(z, t, g_logp, g_ent, g_lse, idx, g_top):
    """(dz, tol) in 64 bits."""
    n, v = z.shape
    zd = z.double()
    logp, ent, lse, _, _, tol = ref_logp(z, t, 0)
    lp = zd - lse[:, None]
    p = torch.exp(lp)
    col = lambda g: torch.zeros(n, 1, dtype=torch.float64, device="cuda") if g is None else g.double()[:, None]
    gl, ge, gs = col(g_logp), col(g_ent), col(g_lse)
    gk = torch.zeros(n, 0, dtype=torch.float64, device="cuda") if g_top is None else g_top.double()
    lpz = torch.where(p > 0, lp, 0.0)
    dz = p * (gs - gl - gk.sum(-1, keepdim=True) - ge * (lpz + ent[:, None]))
    size = p * (gs.abs() + gl.abs() + gk.abs().sum(-1, keepdim=True) + ge.abs() * (lpz.abs() + ent[:, None].abs()))
    hot = torch.zeros_like(dz)
    if g_logp is not None:
        hot.scatter_add_(-1, t.clamp(0, v - 1).long()[:, None], gl)
    if g_top is not None:
        hot.scatter_add_(-1, idx.long(), gk)
    dz, size = dz + hot, size + hot.abs()
    off = (t < 0) | (lse == -INF)
    dz = torch.where(off[:, None], 0.0, dz)
    # p: its exponent's error, lse's, the function's; the products and sums of up to 40 terms
    rel = tol[:, None] + U * (4 * lpz.abs() + 64)
    rel_h = ge.abs() * p * (tol[:, None] * (3 + math.log(v)) + U * 4 * lpz.abs())
    tol_z = size * rel + rel_h + HALF[z.dtype] * dz.abs() * 1.001 + TINY[z.dtype]
    return dz, tol_z


@MIX
@pytest.mark.parametrize("n,v", [(3, 1), (9, 16), (65, 17), (33, 255), (500, 256), (7, 1000), (5, 4099), (3, 40001), (2, 70000)])
def test_logprobs_gradient(n, v, dt):
    z = randn(n, v, seed=n * v, dt=dt, scale=2.0)
    if v > 16:
        z[:, 5:9] = -INF
    t = tokens_for(n, v)
    t = torch.where((t >= 5) & (t < 9), 0, t)
    t[n - 1] = -1
    z[n - 1] = NAN
    k = min(6, max(1, v - 4))
    r = ops.token_logprobs(z, t, top=k)
    g = [randn(n, seed=20 + i) for i in range(3)] + [randn(n, k, seed=30)]
    g[0][n - 1] = NAN
    for use in ((1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 1, 1, 1)):
        gl, ge, gs, gk = (x if u else None for x, u in zip(g, use))
        dz = ops.token_logprobs_grad(z, t, r["lse"], r["entropy"], gl, ge, gs, r["top_idx"] if use[3] else None, gk)
        zero = lambda x: None if x is None else torch.nan_to_num(x)
        # the padded row's stand-in, whose gradient is zero anyway
        zr = torch.where((t < 0)[:, None], torch.zeros((), dtype=dt, device="cuda"), z)
        ref, tol = grad_formula(zr, t, zero(gl), ge, gs, r["top_idx"].clamp(min=0), gk)
        close(dz, ref, tol, f"dlogits {use}")
        keep = z.clone()
        assert torch.equal(ops.token_logprobs_grad(keep, t, r["lse"], r["entropy"], gl, ge, gs,
                                                   r["top_idx"] if use[3] else None, gk, out=keep).nan_to_num(7.0),
                           dz.nan_to_num(7.0)), "in place"


def test_logprobs_gradient_ignores_alternatives_that_are_no_class():
    z, t = randn(5, 50, seed=2), tokens_for(5, 50)
    r = ops.token_logprobs(z, t, top=2)
    g = randn(5, 4, seed=3)
    idx = torch.cat([r["top_idx"], torch.tensor([[-1, 50]] * 5, dtype=torch.int32, device="cuda")], 1)
    a = ops.token_logprobs_grad(z, t, r["lse"], top_idx=idx, g_top=g)
    assert torch.equal(a, ops.token_logprobs_grad(z, t, r["lse"], top_idx=r["top_idx"], g_top=g[:, :2].contiguous()))


def test_logprobs_gradient_special_rows():
    z = randn(5, 300, seed=3)
    z[1] = -INF                      # nothing left
    z[2, 10] = NAN
    z[3] = torch.finfo(F32).min
    z[3, :4] = 1.0
    t = tokens_for(5, 300)
    t[3], t[4] = 2, 300              # (300: past the classes)
    r = ops.token_logprobs(z, t)
    dz = ops.token_logprobs_grad(z, t, r["lse"], r["entropy"], g_logp=torch.ones(5, device="cuda"),
                                 g_entropy=torch.full((5,), 1e6, device="cuda"))
    assert torch.equal(dz[1], torch.zeros(300, device="cuda"))
    assert torch.isnan(dz[2]).all() and torch.isnan(dz[4]).all()
    assert torch.isfinite(dz[0]).all()
    assert torch.equal(dz[3, 4:], torch.zeros(296, device="cuda"))
    want = torch.tensor([-0.25, -0.25, 0.75, -0.25], device="cuda")
    # the entropy's part is p (log p + H) = 0 here but for the rounding of both, times 1e6
    assert (dz[3, :4] - want).abs().max() <= 0.25 * 1e6 * 16 * U + 4 * U


def test_logprobs_gradient_against_differences():
    """Along a random direction: L(z + h u) - L(z - h u) over 2 h in 64 bits, h = 2^-12: the difference's
    own error is h^2 / 6 times the third derivative (below 10 |u|^3 times the gradients' sizes here)."""
    n, v, k, h = 6, 40, 4, 2.0 ** -12
    z, t = randn(n, v, seed=1, scale=1.5), tokens_for(n, v)
    r = ops.token_logprobs(z, t, top=k)
    g = [randn(n, seed=40 + i) for i in range(3)]
    gk = randn(n, k, seed=44)
    dz = ops.token_logprobs_grad(z, t, r["lse"], r["entropy"], g[0], g[1], g[2], r["top_idx"], gk).double()

    def loss(x):
        lse = torch.logsumexp(x, -1)
        lp = x - lse[:, None]
        ent = -(lp.exp() * lp).sum(-1)
        return (g[0].double() * lp.gather(-1, t[:, None])[:, 0] + g[1].double() * ent + g[2].double() * lse).sum() + \
            (gk.double() * lp.gather(-1, r["top_idx"].long())).sum()

    for seed in range(4):
        u = randn(n, v, seed=50 + seed).double()
        num = (loss(z.double() + h * u) - loss(z.double() - h * u)) / (2 * h)
        size = sum(float(x.abs().sum()) for x in g) + float(gk.abs().sum())
        assert abs(float(num - (dz * u).sum())) <= size * (10 * float(u.abs().max()) ** 3 * h * h / 6 + 1e-5)


# ---- table lookup ------------------------------------------------------------


@MIX
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (3, 5, 2), (100, 7, 16), (333, 97, 64), (65, 40, 63), (9, 50, 257), (7, 11, 1000),
                                   (5, 300, 4096), (2, 9, 4099), (1000, 20, 8), (1, 3, 20000)])
def test_embed(n, v, d, dt):
    table = randn(v, d, seed=d, dt=dt)
    for idt in (torch.int64, torch.int32):
        ids = tokens_for(n, v, dtype=idt)
        if n > 2:
            ids[1] = -1
            ids[n - 1] = v
        for scale in (1.0, 0.3, math.sqrt(d)):
            for out in (dt, F32):
                got = ops.embed(table, ids, scale=scale, dtype=out)
                # one fp32 product (by the fp32 scale), rounded once
                want = (table.float()[ids.clamp(0, v - 1).long()] * torch.tensor(scale, dtype=F32, device="cuda")).to(out)
                want[ids < 0] = 0.0
                want[ids >= v] = NAN
                assert torch.equal(got.nan_to_num(123.0), want.nan_to_num(123.0))
                assert torch.equal(torch.isnan(got), torch.isnan(want))


def test_embed_views():
    wide = randn(30, 200, seed=1)
    ids = tokens_for(24, 30).reshape(4, 6)
    frames = torch.full((4, 6, 100), 7.0, device="cuda")
    for lo, d in ((0, 33), (33, 40), (73, 27)):      # fields side by side, from slices of a wider table
        ops.embed(wide[:, lo + 1:lo + 1 + d], ids, scale=2.0, out=frames[:, :, lo:lo + d])
    assert torch.equal(frames, 2.0 * wide[:, 1:101][ids])
    assert ops.embed(wide, ids[:0]).shape == (0, 6, 200)
    one = torch.tensor(4, device="cuda")             # a single id without dimensions
    assert torch.equal(ops.embed(wide, one), wide[4])


def ids_for(kind, n, v, seed=3):
    g = gen(seed)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if kind == "skew":
        ids = ((v + 1.0) ** u - 1.0).long().clamp(0, v - 1)
        ids = torch.randperm(v, generator=g, device="cuda")[ids]
    elif kind == "one":
        ids = torch.full((n,), v // 2, device="cuda", dtype=torch.int64)
    elif kind == "sorted":
        ids = (u * v).long().clamp(0, v - 1).sort()[0]
    elif kind == "none":
        ids = torch.full((n,), -1, device="cuda", dtype=torch.int64)
    else:
        ids = (u * v).long().clamp(0, v - 1)
    return ids


def check_embed_grad(dout, ids, v, scale, out):
    got = ops.embed_grad(dout, ids, v, scale=scale, dtype=out)
    d = dout.shape[-1]
    flat, x = ids.reshape(-1).long(), dout.reshape(-1, d).double()
    on = (flat >= 0) & (flat < v)
    s = torch.tensor(scale, dtype=F32).double().item()
    ref = torch.zeros(v, d, dtype=torch.float64, device="cuda").index_put_((flat[on],), x[on], accumulate=True)
    size = torch.zeros(v, d, dtype=torch.float64, device="cuda").index_put_((flat[on],), x[on].abs(), accumulate=True)
    count = torch.bincount(flat[on], minlength=v).double()[:, None]
    close(got, s * ref, abs(s) * size * U * (count + 2) * 1.001 + HALF[out] * (s * ref).abs() * 1.001 + TINY[out], "dtable")
    assert torch.equal(got[count[:, 0] == 0], torch.zeros_like(got[count[:, 0] == 0]))
    assert torch.equal(got, ops.embed_grad(dout, ids, v, scale=scale, dtype=out)), "not the same twice"


@MIX
@pytest.mark.parametrize("kind", ["even", "skew", "one", "sorted", "none"])
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (1, 400, 64), (31, 5, 3), (257, 300, 65), (1600, 97, 64), (4097, 70000, 24),
                                   (900, 33, 1000), (70, 9, 4099)])
def test_embed_gradient(n, v, d, kind, dt):
    dout = randn(n, d, seed=n + d, dt=dt)
    ids = ids_for(kind, n, v)
    if n > 30 and kind != "none":
        ids[3::7] = -1
        dout[3::7] = NAN                              # padding, whatever it holds
        ids[5] = v
    check_embed_grad(torch.where((ids < 0)[:, None], torch.zeros((), dtype=dt, device="cuda"), dout), ids, v, 0.7, dt)
    got = ops.embed_grad(dout, ids.int(), v, scale=0.7)
    clean = torch.where(((ids < 0) | (ids >= v))[:, None], torch.zeros((), dtype=dt, device="cuda"), dout)
    assert torch.equal(got, ops.embed_grad(clean, ids, v, scale=0.7))


@pytest.mark.parametrize("n,v,d,kind", [(20000, 3, 64, "even"), (70001, 65537, 32, "skew"), (70001, 255, 16, "sorted"),
                                        (140000, 1 << 20, 8, "skew"), (300000, 50000, 8, "skew"), (33000, 1, 40, "one"),
                                        (3000, 700, 48, "skew"), (4096, 100000, 16, "even"), (16000, 5000, 24, "skew"),
                                        (16384, 300, 7, "sorted"), (200000, 20, 16, "skew"), (500000, 8, 33, "even"),
                                        (2049, 256, 100, "skew"), (2048, 256, 1000, "one")])
def test_embed_gradient_many_tokens(n, v, d, kind):
    dout = randn(n, d, seed=1, dt=BF16)
    ids = ids_for(kind, n, v)
    ids[::11] = -1
    check_embed_grad(dout, ids, v, 1.0, F32)


@pytest.mark.parametrize("n,v,d,kind", [(70001, 3000, 1024, "skew"), (2200000, 1000, 8, "skew"), (700001, 400, 4, "sorted"),
                                        (5000, (1 << 27) + 5, 1, "even")])
def test_embed_gradient_largest(n, v, d, kind):
    """Long chunks, sort tiles of several pieces, numbers of 28 bits."""
    check_embed_grad(randn(n, d, seed=2, dt=BF16), ids_for(kind, n, v), v, 1.0, F32)


def test_embed_far_rows():
    """Table and result rows past 2^31 elements."""
    step = 2 ** 30 + 7
    store = torch.zeros(2 * step + 64, dtype=BF16, device="cuda")
    table = store.as_strided((3, 40), (step, 1))
    table.copy_(randn(3, 40, seed=6, dt=BF16))
    ids = torch.tensor([2, 1, 0], device="cuda")
    out = torch.zeros_like(store).as_strided((3, 40), (step, 1))
    assert torch.equal(ops.embed(table, ids, scale=2.0, out=out), 2.0 * table[ids])


def test_embed_gradient_views_and_no_tokens():
    wide = randn(6, 50, 100, seed=2)
    ids = tokens_for(300, 20).reshape(6, 50)
    check_embed_grad(wide[:, :, 3:68], ids, 20, 1.5, F32)
    one = randn(1, 24, seed=3)
    check_embed_grad(one.expand(300, 24), ids.reshape(300), 20, 1.0, F32)
    assert torch.equal(ops.embed_grad(wide[:0, 0], ids[:0, 0], 9), torch.zeros(9, 100, device="cuda"))


def test_embed_gradient_far_rows():
    """Rows of dout past 2^31 elements."""
    step = 2 ** 30 + 3
    store = torch.zeros(2 * step + 64, dtype=BF16, device="cuda")
    dout = store.as_strided((3, 40), (step, 1))
    dout.copy_(randn(3, 40, seed=5, dt=BF16))
    check_embed_grad(dout, torch.tensor([2, 0, 2], device="cuda"), 4, 1.0, F32)


# ---- layer norm ------------------------------------------------------------


def norm_ref(x, gamma, beta, eps):
    x = x.double()
    m = x.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt(((x - m) ** 2).mean(-1, keepdim=True) + eps)
    h = (x - m) * r
    g = 1.0 if gamma is None else gamma.double()
    b = 0.0 if beta is None else beta.double()
    return h * g + b, m, r, h


def norm_tol(x, r, h, d):
    """(of h, relative of r): the mean is off by (d + 2) u mean |x|, a difference by its own rounding too;
    the variance's sum by (d + 4) u, through r = v^(-1/2) by half that and a few roundings."""
    x = x.double()
    dm = (d + 2) * U * x.abs().mean(-1, keepdim=True)
    dh = (dm + U * (x.abs() + x.abs().mean(-1, keepdim=True))) * r
    # the differences' error in the variance: 2 mean |c| dm + dm^2, c the centred row
    dr = (d + 16) * U + (dm * r) + (dm * r) ** 2
    return dh + h.abs() * dr, dr


NORM_SIZES = [(1, 1), (3, 2), (5, 7), (200, 16), (9, 63), (1600, 64), (17, 65), (33, 257), (12, 768), (7, 1000), (5, 1001),
              (6, 1024), (3, 2048), (4, 4096), (3, 4099), (2, 8192), (3, 12001), (2, 40000)]


@MIX
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_layer_norm(n, d, dt):
    x = (randn(n, d, seed=d, scale=2.0) + randn(n, 1, seed=d + 1, scale=4.0)).to(dt)
    eps = 1e-5
    for wt in {F32, dt}:
        gamma, beta = (1.0 + randn(d, seed=2, scale=0.3)).to(wt), randn(d, seed=3).to(wt)
        for g, b in ((gamma, beta), (gamma, None), (None, beta), (None, None)):
            y, mean, rstd = ops.layer_norm(x, g, b, eps=eps, stats=True)
            ref, m, r, h = norm_ref(x, g, b, eps)
            th, tr = norm_tol(x, r, h, d)
            ga = 1.0 if g is None else g.double().abs()
            close(y, ref, ga * (th + 4 * U * h.abs()) + 2 * U * ref.abs() + HALF[dt] * ref.abs() * 1.001 + TINY[dt], "y")
            close(mean, m[:, 0], (d + 2) * U * x.double().abs().mean(-1) + U * m[:, 0].abs(), "mean")
            close(rstd, r[:, 0], (tr * r)[:, 0], "rstd")
    keep = x.clone()
    assert torch.equal(ops.layer_norm(keep, gamma, beta, out=keep), ops.layer_norm(x, gamma, beta)), "in place"


@MIX
@pytest.mark.parametrize("n,d", NORM_SIZES + [(1, 300), (5000, 24), (20001, 8), (3000, 768)])
def test_layer_norm_gradient(n, d, dt):
    x = (randn(n, d, seed=d, scale=2.0) + randn(n, 1, seed=d + 1)).to(dt)
    dy = randn(n, d, seed=d + 2, dt=dt)
    for wt in {F32, dt}:
        gamma = (1.0 + randn(d, seed=2, scale=0.3)).to(wt)
        for g in (gamma, None):
            _, mean, rstd = ops.layer_norm(x, g, None, stats=True)
            dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, mean, rstd, g)
            # the formula on the statistics given
            xd, m, r = x.double(), mean.double()[:, None], rstd.double()[:, None]
            h, w = (xd - m) * r, dy.double() * (1.0 if g is None else g.double())
            ref = r * (w - w.mean(-1, keepdim=True) - h * (w * h).mean(-1, keepdim=True))
            dh = 2 * U * (xd.abs() + m.abs()) * r + 2 * U * h.abs()
            size = r * (w.abs() + w.abs().mean(-1, keepdim=True) + h.abs() * (w * h).abs().mean(-1, keepdim=True))
            more = r * (dh * (w * h).abs().mean(-1, keepdim=True) + h.abs() * (w.abs() * dh).mean(-1, keepdim=True))
            close(dx, ref, size * (d + 16) * U + 2 * more + HALF[dt] * ref.abs() * 1.001 + TINY[dt], "dx")
            dyd = dy.double()
            close(dgamma, (dyd * h).sum(0), ((n + 4) * U * (dyd * h).abs() + dyd.abs() * dh).sum(0), "dgamma")
            close(dbeta, dyd.sum(0), ((n + 2) * U * dyd.abs()).sum(0), "dbeta")
            again = ops.layer_norm_grad(dy, x, mean, rstd, g)
            assert all(torch.equal(a, b) for a, b in zip((dx, dgamma, dbeta), again)), "not the same twice"
    only, none1, none2 = ops.layer_norm_grad(dy, x, mean, rstd, None, weights=False)
    assert torch.equal(only, dx) and none1 is None and none2 is None
    for name in ("dy", "x"):
        a = dict(dy=dy.clone(), x=x.clone())
        got = ops.layer_norm_grad(a["dy"], a["x"], mean, rstd, None, out=a[name])
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dgamma, dbeta))), f"in place of {name}"


def test_layer_norm_views_and_edges():
    base = randn(5, 8, 200, seed=1, dt=BF16, scale=3.0)
    for x in (base[:, :, 3:167], base[:, ::2, 1:65], base[0, 0], base[:, 0, :77]):
        out = torch.full(x.shape[:-1] + (x.shape[-1] + 9,), 5.0, dtype=BF16, device="cuda")
        y, mean, rstd = ops.layer_norm(x, stats=True, out=out[..., 2:2 + x.shape[-1]])
        assert torch.equal(y, ops.layer_norm(x.contiguous()))
        assert bool((out[..., :2] == 5.0).all()) and bool((out[..., 2 + x.shape[-1]:] == 5.0).all())
        dy = randn(*x.shape, seed=9, dt=BF16)
        a, b = ops.layer_norm_grad(dy, x, mean, rstd), ops.layer_norm_grad(dy, x.contiguous(), mean, rstd)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    row = randn(1, 50, seed=2)
    y = ops.layer_norm(row.expand(6, 50))
    assert torch.equal(y, y[:1].expand(6, 50))
    # no rows: gradients of the weights are zero
    dx, dg, db = ops.layer_norm_grad(base[:0, 0], base[:0, 0], torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    assert dx.shape == (0, 200) and torch.equal(dg, torch.zeros(200, device="cuda")) and torch.equal(db, dg)
    # a constant row has variance 0: y = beta
    y = ops.layer_norm(torch.full((2, 33), 3.0, device="cuda"), None, torch.arange(33.0, device="cuda"))
    assert torch.equal(y[1], torch.arange(33.0, device="cuda"))
    # a row with a NaN is NaN and touches no other
    x = randn(3, 64, seed=4)
    x[1, 5] = NAN
    y = ops.layer_norm(x)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


def test_layer_norm_far_rows():
    """Row offsets past 2^31 elements."""
    step = 2 ** 30 + 9
    store = torch.zeros(2 * step + 128, dtype=BF16, device="cuda")
    x = store.as_strided((3, 100), (step, 1))
    x.copy_(randn(3, 100, seed=7, dt=BF16))
    y, mean, rstd = ops.layer_norm(x, stats=True)
    near = x.contiguous()
    assert torch.equal(y, ops.layer_norm(near))
    far = ops.layer_norm_grad(x, x, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(far, ops.layer_norm_grad(near, near, mean, rstd)))


def test_layer_norm_large_mean():
    """A mean a thousand times the spread: the variance is taken about the mean."""
    x = randn(20, 500, seed=6) + 1000.0
    y = ops.layer_norm(x)
    ref, m, r, h = norm_ref(x, None, None, 1e-5)
    th, _ = norm_tol(x, r, h, 500)
    close(y, ref, th + 6 * U * h.abs(), "y")


def test_layer_norm_gradient_against_differences():
    n, d, h = 5, 30, 2.0 ** -10
    x, dy = randn(n, d, seed=1), randn(n, d, seed=2)
    gamma, beta = 1.0 + randn(d, seed=3, scale=0.3), randn(d, seed=4)
    _, mean, rstd = ops.layer_norm(x, gamma, beta, stats=True)
    dx, dg, db = ops.layer_norm_grad(dy, x, mean, rstd, gamma)
    loss = lambda a, g, b: (norm_ref(a, g, b, 1e-5)[0] * dy.double()).sum()
    for seed in range(3):
        u, ug, ub = randn(n, d, seed=60 + seed).double(), randn(d, seed=70 + seed).double(), randn(d, seed=80 + seed).double()
        num = (loss(x.double() + h * u, gamma.double() + h * ug, beta.double() + h * ub) -
               loss(x.double() - h * u, gamma.double() - h * ug, beta.double() - h * ub)) / (2 * h)
        ana = (dx.double() * u).sum() + (dg.double() * ug).sum() + (db.double() * ub).sum()
        # h^2 / 6 times a third derivative below 100 |u|^3 a row, and the fp32 gradients' own error
        assert abs(float(num - ana)) <= float(dy.abs().sum()) * (100 * 4.0 ** 3 * h * h / 6 + 1e-5)


# ---- streams, graphs, refusals ------------------------------------------------------------


def _everything(s, stream=None):
    """Every operator once on the inputs s."""
    r = ops.token_logprobs(s["z"], s["t"], top=3, stream=stream)
    big = ops.token_logprobs(s["big"], s["t"][:2], top=3, stream=stream)
    dz = ops.token_logprobs_grad(s["z"], s["t"], r["lse"], r["entropy"], g_logp=s["g"], g_entropy=s["g"], stream=stream)
    x = ops.embed(s["table"], s["ids"], scale=1.5, stream=stream)
    y, mean, rstd = ops.layer_norm(x, s["gamma"], s["beta"], stats=True, stream=stream)
    dx, dg, db = ops.layer_norm_grad(y, x, mean, rstd, s["gamma"], stream=stream)
    de = ops.embed_grad(dx, s["ids"], s["table"].shape[0], scale=1.5, stream=stream)
    ds = [ops.embed_grad(s["rows"][:n], s["many"][:n], 5000, stream=stream) for n in (3000, 12000, 40000)]
    return [r["logp"], r["entropy"], r["top_logp"], r["top_idx"], big["logp"], big["top_idx"], dz, x, y, dx, dg, db, de] + ds


def _inputs(seed):
    return dict(z=randn(700, 256, seed=seed), t=tokens_for(700, 256, seed=seed), big=randn(2, 90000, seed=seed, dt=BF16),
                g=randn(700, seed=seed + 1), table=randn(97, 64, seed=seed + 2), ids=tokens_for(2000, 97, seed=seed + 3),
                gamma=1.0 + randn(64, seed=seed + 4, scale=0.1), beta=randn(64, seed=seed + 5),
                rows=randn(40000, 24, seed=seed + 6, dt=BF16), many=ids_for("skew", 40000, 5000, seed=seed + 7))


def test_operators_on_another_stream():
    s = _inputs(1)
    want = _everything(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _everything(s, stream=side)
    noise = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]   # would take freed workspaces
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(noise) == 8


def test_operators_on_two_streams_at_once():
    sets = [_inputs(1), _inputs(2)]
    want = [_everything(s) for s in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[_everything(s, stream=st) for s, st in zip(sets, streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for turn in got:
        for a, b in zip(turn, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_operators_captured_and_replayed():
    """Two graphs of every operator, replayed by turns with new inputs and eager calls in between."""
    sets = [_inputs(1), _inputs(2)]
    for s in sets:
        _everything(s)
    torch.cuda.synchronize()
    graphs = []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _everything(s)
        graphs.append((g, s, out))
    for turn in range(3):
        for g, s, out in graphs:
            new = _inputs(10 * turn + 3)
            for k in s:
                s[k].copy_(new[k])
            want = _everything(s)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(out, want)):
                assert torch.equal(a, b), (turn, i)


def test_binding_refusals():
    z, t = randn(4, 16), tokens_for(4, 16)
    lse = randn(4)
    for call in (lambda: ops.token_logprobs(z.double(), t), lambda: ops.token_logprobs(z.t(), t),
                 lambda: ops.token_logprobs(z, t[:3]), lambda: ops.token_logprobs(z, t.float()),
                 lambda: ops.token_logprobs(z, t.cpu()), lambda: ops.token_logprobs(z[:, ::2], t),
                 lambda: ops.token_logprobs(z, tokens_for(8, 16)[::2]),
                 lambda: ops.token_logprobs_grad(z, t, lse.double()), lambda: ops.token_logprobs_grad(z, t, lse[:3]),
                 lambda: ops.token_logprobs_grad(z, t, lse, g_top=randn(4, 2)),
                 lambda: ops.token_logprobs_grad(z, t, lse, out=z.bfloat16()),
                 lambda: ops.embed(z[0], t), lambda: ops.embed(z, t, dtype=torch.float16),
                 lambda: ops.embed(z, t, out=randn(4, 15)), lambda: ops.embed(z, t.short()),
                 lambda: ops.embed_grad(z, t[:3], 5), lambda: ops.embed_grad(z.half(), t, 5, dtype=BF16),
                 lambda: ops.layer_norm(z, randn(15)), lambda: ops.layer_norm(z, randn(16, dt=BF16)),
                 lambda: ops.layer_norm(z.half(), randn(16, dt=F16), randn(16)),
                 lambda: ops.layer_norm_grad(z[:3], z, lse, lse), lambda: ops.layer_norm_grad(z, z, lse[:2], lse)):
        with pytest.raises(ValueError):
            call()
    from paper_1802_08435_amd import wavernn
    for call in (lambda: ops.token_logprobs(z, t, top=17), lambda: ops.token_logprobs(z, t, top=-1),
                 lambda: ops.embed_grad(z, t, 0), lambda: ops.layer_norm(z, eps=0.0),
                 lambda: ops.token_logprobs_grad(z, t, lse, g_entropy=lse)):
        with pytest.raises(wavernn.WaveRNNError):
            call()
