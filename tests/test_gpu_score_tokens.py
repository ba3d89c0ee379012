"""The operators in the models' own paths: scoring by log probabilities, entropies and
alternatives on every kind of model, and conditioning frames from labels."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1802_08435_amd import ops, synth, wavernn  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _model(kind):
    if kind == "small":
        return wavernn.Model(synth.make_weights(64, seed=1), dtype="f32", max_streams=2), 2, 60
    if kind == "dense":
        return wavernn.Model(synth.make_weights(256, seed=2, cond_dim=16), max_streams=3), 3, 333
    if kind == "sparse":
        return wavernn.Model(synth.make_weights(256, seed=3, cond_dim=16, block=(4, 4), density=0.1), r_format="bsr4x4"), 1, 120
    if kind == "fused":
        return wavernn.Model(synth.make_fused_weights(128, seed=4, cond_dim=16), max_streams=2), 2, 150
    w = synth.make_weights(128, seed=5, cond_dim=16, B=4, ctx_dim=32)
    return wavernn.Model(w), 1, 160


@pytest.mark.parametrize("kind", ["small", "dense", "sparse", "fused", "subscale"])
def test_score_tokens_equals_the_operator_on_the_logits(kind):
    m, S, T = _model(kind)
    cond = None if m.cond_dim == 0 else cuda(synth.features(S, T, cond_dim=16))
    tgt = cuda(synth.target_signal(S, T, seed=6, kind="uniform"))
    ref = m.score(tgt, cond=cond)
    u = tgt.to(torch.int32)
    parts = []
    for z, byte in ((ref["zc"], u // 256), (ref["zf"], u % 256)):
        if m.fused:
            parts += [ops.token_logprobs(z[..., 16 * k:16 * k + 16], b.contiguous(), top=4)
                      for k, b in ((0, byte // 16), (1, byte % 16))]
        else:
            parts.append(ops.token_logprobs(z, byte.contiguous(), top=4))
    r = m.score_tokens(tgt, cond=cond, top=4)
    m.device_status()
    for k in ("logp", "entropy", "top_logp", "top_idx"):
        want = torch.stack([p[k] for p in parts], 2)
        assert torch.equal(r[k], want), (kind, k)
    # the NLL is minus the sum, each off by a few fp32 roundings of values up to 2 ln 256 + |z|
    assert float((r["logp"].sum(-1) + ref["nll"]).abs().max()) <= 64 * 2.0 ** -24 * 32
    bare = m.score_tokens(tgt, cond=cond)
    assert bare["top_idx"] is None and torch.equal(bare["logp"], r["logp"])
    assert m.score_tokens(tgt[:, :0], cond=cond, top=2)["top_idx"].shape == (S, 0, 4 if m.fused else 2, 2)
    with pytest.raises(wavernn.WaveRNNError, match="top"):
        m.score_tokens(tgt, cond=cond, top=33)
    m.close()


def test_score_tokens_over_several_chunks():
    """More samples than the output layers take at a time (65,536)."""
    w = synth.make_weights(128, seed=7)
    m = wavernn.Model(w, max_streams=3)
    tgt = cuda(synth.target_signal(3, 30001, seed=8, kind="uniform"))
    r, ref = m.score_tokens(tgt, top=2), m.score(tgt)
    m.device_status()
    for q, z, byte in ((0, ref["zc"], tgt.to(torch.int32) // 256), (1, ref["zf"], tgt.to(torch.int32) % 256)):
        p = ops.token_logprobs(z, byte.contiguous(), top=2)
        for k in ("logp", "entropy", "top_logp", "top_idx"):
            assert torch.equal(r[k][:, :, q], p[k]), (q, k)
    m.close()


def _front(w, n_labels, d, seed=9):
    rng = np.random.default_rng(seed)
    w["E"] = rng.standard_normal((n_labels, d)).astype(np.float32)
    w["E_scale"] = float(np.sqrt(d))
    w["ln_g"] = (1.0 + 0.2 * rng.standard_normal(16)).astype(np.float32)
    w["ln_b"] = (0.2 * rng.standard_normal(16)).astype(np.float32)
    return w


@pytest.mark.parametrize("d", [16, 4])
def test_labels_condition_a_model(d):
    """Labels through the table and the norm, as frames or inside sample and score: the same bits."""
    S, T, fields = 2, 500, 16 // d
    w = _front(synth.make_weights(128, seed=10, cond_dim=16), 30, d)
    m = wavernn.Model(w, max_streams=2)
    n = -(-T // m.frame_len)
    labels = torch.randint(0, 30, (S, n, fields), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    labels[0, 1, 0] = -1
    frames = m.frames(labels)
    x = torch.where((labels >= 0)[..., None], cuda(w["E"])[labels.clamp(min=0)].double() * w["E_scale"], 0.0).reshape(S, n, 16)
    h = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-5)
    want = h * cuda(w["ln_g"]).double() + cuda(w["ln_b"]).double()
    # 16 terms a sum, values up to about 20: 64 roundings of that
    assert float((frames.double() - want).abs().max()) <= 64 * 2.0 ** -24 * 20
    assert torch.equal(m.sample(T, labels=labels, seed=3, n_streams=S), m.sample(T, cond=frames, seed=3, n_streams=S))
    tgt = cuda(synth.target_signal(S, T, seed=11))
    a, b = m.score_tokens(tgt, labels=labels, top=3), m.score_tokens(tgt, cond=frames, top=3)
    assert all(torch.equal(a[k], b[k]) for k in a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = m.frames(labels, stream=side)
    side.synchronize()
    assert torch.equal(on_side, frames)
    m.device_status()
    # features given, only normalised
    feat = cuda(synth.features(S, T, cond_dim=16))
    assert torch.equal(m.frames(feat), ops.layer_norm(feat, m.ln_g, m.ln_b))
    with pytest.raises(ValueError, match="one of the two"):
        m.sample(T, cond=frames, labels=labels, n_streams=S)
    with pytest.raises(ValueError, match="noalloc"):
        m.sample(T, labels=labels, n_streams=S, noalloc=True, out=torch.empty(S, T, dtype=torch.uint16, device="cuda"))
    with pytest.raises(ValueError, match="labels must be"):
        m.frames(labels[:, :, :1].expand(S, n, fields + 1).contiguous())
    m.close()


def test_front_end_gradient_against_differences():
    """frames_grad against central differences of the 64-bit front end."""
    w = _front(synth.make_weights(128, seed=12, cond_dim=16), 10, 8)
    m = wavernn.Model(w)
    g = torch.Generator(device="cuda").manual_seed(2)
    labels = torch.randint(-1, 10, (3, 40, 2), device="cuda", generator=g)
    df = torch.randn(3, 40, 16, device="cuda", generator=g)
    grads = m.frames_grad(labels, df)

    def loss(E, lg, lb):
        x = torch.where((labels >= 0)[..., None], E[labels.clamp(min=0)] * w["E_scale"], 0.0).reshape(3, 40, 16)
        c = x - x.mean(-1, keepdim=True)
        return ((c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * lg + lb) * df.double()).sum()

    p = [cuda(w[k]).double() for k in ("E", "ln_g", "ln_b")]
    step = 2.0 ** -14
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(20 + seed)
        u = [torch.randn(a.shape, device="cuda", generator=g).double() for a in p]
        num = (loss(*[a + step * b for a, b in zip(p, u)]) - loss(*[a - step * b for a, b in zip(p, u)])) / (2 * step)
        ana = sum(float((grads[k].double() * b).sum()) for k, b in zip(("E", "ln_g", "ln_b"), u))
        # the third derivative along u is below 1000 a frame (rows of spread over 1, |u| below 4), and fp32
        assert abs(float(num) - ana) <= float(df.abs().sum()) * (1000 * step * step / 6 + 1e-5)
    x = torch.randn(2, 7, 16, device="cuda", generator=g)
    by = m.frames_grad(x, df[:2, :7].contiguous())
    with pytest.raises(ValueError, match="float32"):
        m.frames(x.bfloat16())
    with pytest.raises(ValueError, match="contiguous"):
        m.frames(x.expand(2, 7, 16).transpose(0, 1))
    for bad in (df[:, :39], df[:, :, :8].contiguous(), df[:2].contiguous()):
        with pytest.raises(ValueError):
            m.frames_grad(labels, bad)
    assert by["E"] is None and by["x"].shape == x.shape
    m.close()


def test_a_front_end_that_does_not_fit_is_refused():
    w = synth.make_weights(64, seed=1)
    w["ln_g"] = np.ones(16, np.float32)
    with pytest.raises(ValueError, match="conditioning"):
        wavernn.Model(w, dtype="f32")
    w = synth.make_weights(128, seed=1, cond_dim=16)
    w["E"] = np.ones((4, 5), np.float32)
    with pytest.raises(ValueError, match="divisor"):
        wavernn.Model(w)
    m = wavernn.Model(synth.make_weights(128, seed=1, cond_dim=16))
    with pytest.raises(ValueError, match="label table"):
        m.frames(torch.zeros(1, 4, dtype=torch.int64, device="cuda"))
    m.close()


def test_score_tokens_on_another_stream_owns_its_results_there():
    """Results dropped on the host while the side stream may still write them: their memory is
    the side stream's, and what the current stream allocates next lies elsewhere."""
    w = synth.make_weights(128, seed=7)
    m = wavernn.Model(w, max_streams=2)
    tgt = cuda(synth.target_signal(2, 20000, seed=8, kind="uniform"))
    want = m.score_tokens(tgt, top=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.empty_cache()
    got = m.score_tokens(tgt, top=8, stream=side)
    sizes = [(t.shape, t.dtype) for t in got.values()]
    spans = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in got.values()]
    keep = m.score_tokens(tgt, top=8, stream=side)
    del got
    fresh = [torch.full(s, 7, dtype=d, device="cuda") for s, d in sizes]
    for t in fresh:
        for lo, hi in spans:
            assert t.data_ptr() + t.numel() * t.element_size() <= lo or hi <= t.data_ptr(), "memory of the side stream reused"
    side.synchronize()
    assert all(torch.equal(keep[k], want[k]) for k in want)
    m.device_status()
    m.close()


@pytest.mark.parametrize("kind", ["sparse", "dense"])
def test_scoring_rising_lengths_keeps_a_bounded_memory(kind):
    """Utterances of 1, 2, ... 24 thousand samples: what the model holds at the end is at most four times the longest
    call's share (all calls' shares would be 12.5 times that)."""
    if kind == "sparse":
        m = wavernn.Model(synth.make_weights(256, seed=3, block=(4, 4), density=0.1), r_format="bsr4x4")
        share = 2048
    else:
        m = wavernn.Model(synth.make_weights(256, seed=2))
        share = 4 * 256 + 4 * 128 + 2048
    tgt = cuda(synth.target_signal(1, 24000, seed=6, kind="uniform"))
    m.score_tokens(tgt[:, :100].contiguous())
    torch.cuda.synchronize()

    def held():   # outside torch's own pool
        free, total = torch.cuda.mem_get_info()
        return total - free - torch.cuda.memory_reserved()

    before = held()
    for n in range(1000, 24001, 1000):
        m.score_tokens(tgt[:, :n].contiguous())
    m.device_status()
    last = m.score_tokens(tgt)
    # (2 MiB: the granularity of each of a few allocations)
    assert held() - before <= 4 * share * 24000 + 16 * (2 << 20)
    assert torch.equal(m.score_tokens(tgt[:, :1000].contiguous())["logp"], last["logp"][:, :1000])
    m.close()
