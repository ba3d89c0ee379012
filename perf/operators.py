"""Operators at the two ends of a model over tokens, to be timed and compared.

What a model answers with: log probabilities of given tokens with the entropy and
the top alternatives of every distribution, and their gradient.  What conditions
it: rows of a table looked up by label with a scale, with the gradient of the
table, and layer norm of the rows, forward and backward.

Each case is one pass through one operator.  With ``own`` false a pass computes
the formulas with elementary torch operations in 32 bits, rounded once at the
end; with ``own`` true it calls the library.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one second of speech scored: both bytes of 24,000 samples, 256 classes, the best five of each
        dict(name="logp_bytes", op="logp", dt="f32", n=48000, v=256, top=5, pad=0.0, masked=0.0),
        # one token served from a large vocabulary, part of it masked: latency counts
        dict(name="logp_token", op="logp", dt="bf16", n=1, v=65536, top=8, pad=0.0, masked=0.1),
        # a training step's loss over a ragged, padded batch of bytes, with an entropy bonus
        dict(name="logp_train_bytes", op="logp_train", dt="f32", n=7681, v=256, pad=0.2, masked=0.0),
        # the loss of a large batch over a large vocabulary
        dict(name="logp_train_vocab", op="logp_train", dt="bf16", n=4096, v=65536, pad=0.05, masked=0.0),
        # conditioning frames of one utterance of 8 seconds from its labels
        dict(name="embed_frames", op="embed", dt="f32", out="f32", n=1600, v=97, d=64, pad=0.02, ids="runs"),
        # a batch of long token sequences into a wide model
        dict(name="embed_vocab", op="embed", dt="bf16", out="bf16", n=16384, v=65536, d=4096, pad=0.02, ids="skew"),
        # the label table's gradient: 64 utterances of one second, labels that last many frames
        dict(name="embed_grad_frames", op="embed_grad", dt="f32", out="f32", n=12800, v=97, d=64, pad=0.02, ids="runs"),
        # the table's gradient for a large vocabulary, a few tokens very frequent, many absent
        dict(name="embed_grad_vocab", op="embed_grad", dt="bf16", out="f32", n=16384, v=50021, d=1024, pad=0.02,
             ids="skew"),
        # conditioning frames of one utterance normalised
        dict(name="norm_frames", op="norm", dt="f32", wt="f32", n=1600, d=64),
        # the rows of a large batch
        dict(name="norm_rows", op="norm", dt="bf16", wt="bf16", n=16384, d=4096),
        # odd width, ragged number of rows, backward
        dict(name="norm_grad_odd", op="norm_grad", dt="f16", wt="f32", n=1999, d=1001),
        # the rows of a large batch, backward
        dict(name="norm_grad_rows", op="norm_grad", dt="bf16", wt="f32", n=16384, d=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "logp", "logp_train", "logp_train", "embed", "embed_grad", "norm", "norm_grad"])
    dt = rng.choice(["f32", "bf16", "f16"])
    pad = rng.choice([0.0, 0.02, 0.3])
    if op in ("logp", "logp_train"):
        if rng.random() < 0.5:                       # bytes and nibbles
            v = rng.choice([16, 32, 256, rng.randint(2, 300)])
            n = _log(rng, 1, 100000)
        else:                                        # vocabularies
            v = _log(rng, 300, 131072)
            n = _log(rng, 1, max(2, min(8192, (1 << 27) // v)))
        case = dict(op=op, dt=dt, n=n, v=v, pad=pad, masked=rng.choice([0.0, 0.0, 0.1, 0.4]))
        if op == "logp":
            case["top"] = rng.choice([0, 1, rng.randint(1, min(20, v // 2))])
        return case
    if op in ("embed", "embed_grad"):
        d = rng.choice([_log(rng, 8, 4096), 8 * _log(rng, 2, 512)])
        return dict(op=op, dt=dt, out=rng.choice([dt, "f32"]), n=_log(rng, 1, min(65536, (1 << 26) // d)),
                    v=_log(rng, 20, min(100000, (1 << 26) // d)), d=d, pad=pad, ids=rng.choice(["runs", "skew", "even"]))
    d = rng.choice([_log(rng, 16, 12000), 8 * _log(rng, 2, 1024)])
    return dict(op=op, dt=dt, wt=rng.choice([dt, "f32"]), n=_log(rng, 1, min(100000, (1 << 26) // d)), d=d)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, dt="f32"):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(DT[dt])


def _uniform(n, g):
    return torch.rand(n, generator=g, device="cuda", dtype=torch.float64)


def _ids(case, g):
    """Token numbers: uneven as in text ("skew"), labels that last for some frames ("runs"), or even."""
    n, v = case["n"], case["v"]
    kind = case.get("ids", "even")
    if kind == "skew":                               # the density of number k falls as 1 / (k + 1)
        order = torch.randperm(v, generator=g, device="cuda")
        ids = order[((v + 1.0) ** _uniform(n, g) - 1.0).long().clamp_(0, v - 1)]
    elif kind == "runs":
        start = _uniform(n, g) < 1.0 / 15.0
        labels = (_uniform(n, g) * v).long().clamp_(0, v - 1)
        ids = labels[torch.cumsum(start, 0)[:n].clamp_(max=n - 1)]
    else:
        ids = (_uniform(n, g) * v).long().clamp_(0, v - 1)
    if case["pad"] > 0.0:
        ids = torch.where(_uniform(n, g) < case["pad"], torch.full_like(ids, -1), ids)
    return ids


def _scale(case):
    return math.sqrt(case["d"])


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    if case["op"] in ("logp", "logp_train"):
        n, v = case["n"], case["v"]
        # logits of a trained model: spread of a few units, one class often well ahead
        z = _normal((n, v), g).mul_(2.5)
        z[torch.arange(n, device="cuda"), (_uniform(n, g) * v).long().clamp_(0, v - 1)] += 8.0
        st["tokens"] = _ids(case, g)
        if case["masked"] > 0.0:                     # classes that are not allowed, never the token itself
            off = _uniform(v, g) < case["masked"]
            off[torch.randperm(v, generator=g, device="cuda")[: v // 2 + 1]] = False
            keep = z[torch.arange(n, device="cuda"), st["tokens"].clamp(min=0)]
            z[:, off] = -math.inf
            z[torch.arange(n, device="cuda"), st["tokens"].clamp(min=0)] = keep
        st["logits"] = z.to(DT[case["dt"]])
        if case["op"] == "logp_train":
            st["g_logp"] = _normal((n,), g).mul_(0.1).sub_(1.0).div_(n)
            st["g_entropy"] = torch.full((n,), -0.01 / n, device="cuda")
        return st
    if case["op"] == "embed":
        st["ids"] = _ids(case, g)
        st["table"] = _normal((case["v"], case["d"]), g).mul_(0.02).to(DT[case["dt"]])
        return st
    if case["op"] == "embed_grad":
        st["ids"] = _ids(case, g)
        st["dout"] = _normal((case["n"], case["d"]), g, case["dt"])
        return st
    n, d = case["n"], case["d"]
    x = _normal((n, d), g).mul_(1.0 + 3.0 * _uniform(n, g).float()[:, None]).add_(_normal((n, 1), g))
    st["x"] = x.to(DT[case["dt"]])
    st["gamma"] = _normal((d,), g).mul_(0.2).add_(1.0).to(DT[case["wt"]])
    if case["op"] == "norm":
        st["beta"] = _normal((d,), g).mul_(0.2).to(DT[case["wt"]])
        return st
    st["dy"] = _normal((n, d), g, case["dt"])
    st["mean"] = torch.empty(n, device="cuda")
    st["rstd"] = torch.empty(n, device="cuda")
    step = max(1, (1 << 26) // d)
    for i in range(0, n, step):                      # as the forward pass left them
        x = st["x"][i:i + step].double()
        st["mean"][i:i + step] = x.mean(-1)
        st["rstd"][i:i + step] = 1.0 / torch.sqrt(x.var(-1, unbiased=False) + 1e-5)
    return st


# ---- plain forms ------------------------------------------------------------


def _plain_stats(z):
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1)
    ent = torch.log(s) - (e * torch.where(e > 0, d, 0.0)).sum(-1) / s
    return m[:, 0] + torch.log(s), ent


def _plain_logp(st):
    case, tokens = st["case"], st["tokens"]
    z = st["logits"].float()
    on = tokens >= 0
    lse, ent = _plain_stats(z)
    logp = z.gather(-1, tokens.clamp(min=0)[:, None])[:, 0] - lse
    out = dict(logp=torch.where(on, logp, 0.0), entropy=torch.where(on, ent, 0.0))
    if case["op"] == "logp_train":
        gl, ge = st["g_logp"], st["g_entropy"]
        lp = z - lse[:, None]
        p = torch.exp(lp)
        lp = torch.where(p > 0, lp, 0.0)
        dz = -p * (gl[:, None] + ge[:, None] * (lp + ent[:, None]))
        dz.scatter_add_(-1, tokens.clamp(min=0)[:, None], gl[:, None])
        out["dlogits"] = torch.where(on[:, None], dz, 0.0).to(DT[case["dt"]])
    elif case["top"]:
        idx, val = [], []
        num = torch.arange(case["v"], device="cuda")
        left = z.clone()
        for _ in range(case["top"]):
            best = left.amax(-1, keepdim=True)
            j = torch.where(left == best, num, case["v"]).amin(-1, keepdim=True)
            left.scatter_(-1, j, -math.inf)
            idx.append(j)
            val.append(best - lse[:, None])
        out["top_idx"] = torch.where(on[:, None], torch.cat(idx, 1), -1).int()
        out["top_logp"] = torch.where(on[:, None], torch.cat(val, 1), 0.0)
    return out


def _plain(st):
    case = st["case"]
    if case["op"] in ("logp", "logp_train"):
        return _plain_logp(st)
    if case["op"] == "embed":
        rows = st["table"][st["ids"].clamp(min=0)].float() * _scale(case)
        return torch.where((st["ids"] >= 0)[:, None], rows, 0.0).to(DT[case["out"]])
    if case["op"] == "embed_grad":
        on = (st["ids"] >= 0)[:, None]
        dt = torch.zeros(case["v"], case["d"], device="cuda")
        dt.index_add_(0, st["ids"].clamp(min=0), torch.where(on, st["dout"].float(), 0.0))
        return (dt * _scale(case)).to(DT[case["out"]])
    x, gamma = st["x"].float(), st["gamma"].float()
    if case["op"] == "norm":
        c = x - x.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5)
        return (c * r * gamma + st["beta"].float()).to(DT[case["dt"]])
    dy, r = st["dy"].float(), st["rstd"][:, None]
    h = (x - st["mean"][:, None]) * r
    g = dy * gamma
    dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    return dict(dx=dx.to(DT[case["dt"]]), dgamma=(dy * h).sum(0), dbeta=dy.sum(0))


def _own(st):
    from paper_1802_08435_amd import ops
    case = st["case"]
    if case["op"] == "logp":
        r = ops.token_logprobs(st["logits"], st["tokens"], top=case["top"])
        out = dict(logp=r["logp"], entropy=r["entropy"])
        if case["top"]:
            out["top_idx"], out["top_logp"] = r["top_idx"], r["top_logp"]
        return out
    if case["op"] == "logp_train":
        r = ops.token_logprobs(st["logits"], st["tokens"])
        dz = ops.token_logprobs_grad(st["logits"], st["tokens"], r["lse"], r["entropy"], g_logp=st["g_logp"],
                                     g_entropy=st["g_entropy"])
        return dict(logp=r["logp"], entropy=r["entropy"], dlogits=dz)
    if case["op"] == "embed":
        return ops.embed(st["table"], st["ids"], scale=_scale(case), dtype=DT[case["out"]])
    if case["op"] == "embed_grad":
        return ops.embed_grad(st["dout"], st["ids"], case["v"], scale=_scale(case), dtype=DT[case["out"]])
    if case["op"] == "norm":
        return ops.layer_norm(st["x"], st["gamma"], st["beta"], eps=1e-5)
    dx, dgamma, dbeta = ops.layer_norm_grad(st["dy"], st["x"], st["mean"], st["rstd"], st["gamma"])
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    b = {"f32": 4, "bf16": 2, "f16": 2}
    n, on = case["n"], 1.0 - case.get("pad", 0.0)
    if case["op"] in ("logp", "logp_train"):
        cells = n * case["v"]
        read = on * cells * b[case["dt"]] + 8 * n     # a padded row need not be read
        if case["op"] == "logp":
            return dict(bytes=int(read + n * (8 + 8 * case["top"])), flops=int(on * cells * 6))
        # two reads: the gradient needs the sum over the row; every row of it is written
        return dict(bytes=int(2 * read + cells * b[case["dt"]] + 24 * n), flops=int(on * cells * 14))
    if case["op"] == "embed":
        # a row looked up more than once is read once; at most every row of the table
        rows = min(on * n, case["v"])
        if case["ids"] == "skew":
            rows = min(rows, 0.6 * on * n)
        return dict(bytes=int(8 * n + rows * case["d"] * b[case["dt"]] + n * case["d"] * b[case["out"]]),
                    flops=int(on * n * case["d"]))
    if case["op"] == "embed_grad":
        return dict(bytes=int(8 * n + on * n * case["d"] * b[case["dt"]] + case["v"] * case["d"] * b[case["out"]]),
                    flops=int(on * n * case["d"] + case["v"] * case["d"]))
    cells = n * case["d"]
    if case["op"] == "norm":
        return dict(bytes=2 * cells * b[case["dt"]] + 2 * case["d"] * b[case["wt"]], flops=8 * cells)
    return dict(bytes=3 * cells * b[case["dt"]] + 8 * n + case["d"] * (b[case["wt"]] + 8), flops=14 * cells)


# ---- 64 bits ----------------------------------------------------------------


def _exact_logp(case, st):
    n, v = case["n"], case["v"]
    step = max(1, (1 << 25) // v)
    parts = []
    for i in range(0, n, step):
        z, t = st["logits"][i:i + step].double(), st["tokens"][i:i + step]
        lse = torch.logsumexp(z, -1, keepdim=True)
        lp = z - lse
        p = lp.exp()
        ent = -torch.special.xlogy(p, p).sum(-1)
        off = t < 0
        at = t.clamp(min=0)[:, None]
        r = dict(logp=lp.gather(-1, at)[:, 0].masked_fill(off, 0.0), entropy=ent.masked_fill(off, 0.0))
        if case["op"] == "logp_train":
            gl, ge = (st[k][i:i + step].double()[:, None] for k in ("g_logp", "g_entropy"))
            hot = torch.zeros_like(z).scatter_(-1, at, 1.0)
            r["dlogits"] = (gl * (hot - p) - ge * (torch.special.xlogy(p, p) + p * ent[:, None])).masked_fill(
                off[:, None], 0.0)
        elif case["top"]:
            val, idx = torch.sort(lp, dim=-1, descending=True, stable=True)
            r["top_idx"] = idx[:, :case["top"]].masked_fill(off[:, None], -1).int()
            r["top_logp"] = val[:, :case["top"]].masked_fill(off[:, None], 0.0)
        parts.append(r)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("logp", "logp_train"):
        return _exact_logp(case, st)
    if case["op"] == "embed":
        ids, out = st["ids"], torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
        on = ids >= 0
        out[on] = st["table"].double()[ids[on]] * _scale(case)
        return out
    if case["op"] == "embed_grad":
        on = st["ids"] >= 0
        out = torch.zeros(case["v"], case["d"], dtype=torch.float64, device="cuda")
        out.index_put_((st["ids"][on],), st["dout"][on].double() * _scale(case), accumulate=True)
        return out
    x, gamma = st["x"].double(), st["gamma"].double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    if case["op"] == "norm":
        return (x - mean) / torch.sqrt(var + 1e-5) * gamma + st["beta"].double()
    std = torch.sqrt(var + 1e-5)
    h = (x - mean) / std
    dy = st["dy"].double()
    g = dy * gamma
    d = case["d"]
    dx = (d * g - g.sum(-1, keepdim=True) - h * (g * h).sum(-1, keepdim=True)) / (d * std)
    return dict(dx=dx, dgamma=torch.einsum("nd,nd->d", dy, h), dbeta=dy.sum(0))
