"""The models' front end and score_tokens refuse tensors that the library would read out of
range or on the wrong device, before anything is launched.  No GPU is used: the
model has no handle, and its tensors stay on the CPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_1802_08435_amd import wavernn as W  # noqa: E402


def model(d=None, norm=False, fused=False, B=1):
    m = W.Model.__new__(W.Model)
    m.H, m.B, m.cond_dim, m.fused, m._h, m.device = 64, B, 16, fused, None, torch.device("cuda", 0)
    m.E = None if d is None else torch.zeros(5, d)
    m.E_scale, m.ln_eps = 1.0, 1e-5
    m.ln_g, m.ln_b = (torch.ones(16), torch.zeros(16)) if norm else (None, None)
    return m


@pytest.mark.parametrize("norm", [False, True])
def test_features_on_the_cpu(norm):
    """Without a layer norm they are the frames as they are, and only their address goes on."""
    m, x = model(norm=norm), torch.zeros(2, 7, 16)
    for call in (lambda: m.frames(x), lambda: m.sample(100, labels=x, n_streams=2), lambda: m.frames_grad(x, x)):
        with pytest.raises(ValueError, match="on the model's GPU"):
            call()


@pytest.mark.parametrize("call", ["sample", "sample_steps", "score", "score_tokens"])
def test_labels_of_other_utterances_than_the_call_s(call, monkeypatch):
    """Fewer would be read past their end."""
    m = model(d=8)
    monkeypatch.setattr(W.Model, "_check_scored", lambda *a: None)   # (a CPU target stands in)
    target = torch.zeros(3, 100, dtype=torch.uint16)
    run = {"sample": lambda x: m.sample(100, labels=x, n_streams=3), "sample_steps": lambda x: m.sample_steps(target, 0, 1, labels=x),
           "score": lambda x: m.score(target, labels=x), "score_tokens": lambda x: m.score_tokens(target, labels=x)}[call]
    for x in (torch.zeros(1, 7, 2, dtype=torch.int64), torch.zeros(4, 7, 2, dtype=torch.int64), torch.tensor(1)):
        with pytest.raises(ValueError, match="3 utterances"):
            run(x)


def test_labels_that_do_not_fit_the_table(monkeypatch):
    m = model(d=8)
    monkeypatch.setattr(W.Model, "_check_frames", lambda *a: None)
    df = torch.zeros(2, 7, 16)
    for x in (torch.zeros(2, 7, 3, dtype=torch.int64), torch.zeros(2, 7, dtype=torch.int64)):
        with pytest.raises(ValueError, match="labels must be"):
            m.frames(x)
        with pytest.raises(ValueError, match="labels must be"):
            m.frames_grad(x, df)
    with pytest.raises(ValueError, match="label table"):
        model().frames_grad(torch.zeros(2, 7, 2, dtype=torch.int64), df)


class OnGpu:
    """A tensor as the checks see one on a GPU: nothing here follows its address."""

    def __init__(self, t, index=0):
        self.t, self.device, self.is_cuda = t, torch.device("cuda", index), True

    def __getattr__(self, k):
        return getattr(self.t, k)


@pytest.mark.parametrize("B,fused", [(1, False), (4, False), (2, True)])
def test_score_tokens_checks_what_it_is_given(B, fused):
    m = model(B=B, fused=fused)
    S, rows = 2, 2 if fused else 2 * B
    target, cond = torch.zeros(S, 100, dtype=torch.uint16), torch.zeros(S, 3, 16)
    init = dict(h=torch.zeros(rows, 64), c=torch.zeros(S * B, dtype=torch.uint8), f=torch.zeros(S * B, dtype=torch.uint8))
    ok = {k: OnGpu(t) for k, t in init.items()}
    m._check_scored(OnGpu(target), OnGpu(cond), ok, None)
    m._check_scored(OnGpu(target[:, :0]), OnGpu(cond), None, None)
    m._check_scored(OnGpu(target), None, None, None)
    for bad in (target, OnGpu(target, 1), OnGpu(target.to(torch.int32)), OnGpu(target.view(-1)), OnGpu(target[:, ::2])):
        with pytest.raises(ValueError, match="target must be"):
            m._check_scored(bad, OnGpu(cond), None, None)
    with pytest.raises(ValueError, match="target must be"):
        m.score_tokens(target)

    class Away:
        device = torch.device("cuda", 1)

    with pytest.raises(ValueError, match="the stream is on"):
        m._check_scored(OnGpu(target), None, None, Away())
    for bad in (cond, OnGpu(cond.half()), OnGpu(cond[:, :, :8].contiguous()), OnGpu(cond.transpose(0, 1)), OnGpu(cond[0]),
                OnGpu(cond, 1)):
        with pytest.raises(ValueError, match="cond must be"):
            m._check_scored(OnGpu(target), bad, None, None)
    with pytest.raises(ValueError, match="cond holds"):
        m._check_scored(OnGpu(target), OnGpu(cond[:1]), None, None)
    for k, bad in (("h", init["h"]), ("h", OnGpu(init["h"][1:])), ("h", OnGpu(init["h"].double())), ("c", OnGpu(init["c"][1:])),
                   ("c", OnGpu(init["c"].int())), ("f", OnGpu(init["f"], 1)), ("f", OnGpu(init["f"][:1].expand(2 * B)))):
        with pytest.raises(ValueError, match="init's " + k):
            m._check_scored(OnGpu(target), OnGpu(cond), {**ok, k: bad}, None)
    m.cond_dim = 0                      # (a model without conditioning reads none)
    m._check_scored(OnGpu(target), cond, None, None)


def test_the_operators_import_with_a_torch_without_gpu_support(monkeypatch):
    import importlib.util
    from paper_1802_08435_amd import ops
    for k in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, k, raising=False)
    spec = importlib.util.spec_from_file_location("paper_1802_08435_amd.ops_copy", ops.__file__)
    copy = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(copy)
    with pytest.raises(ValueError, match="GPU"):
        copy.token_logprobs(torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64))
