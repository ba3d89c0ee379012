"""The operators on callers' tensors refuse bad arguments on the host, before any
launch: the C entry points by status and message, the binding by ValueError.
No GPU is used: pointers are never followed."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_1802_08435_amd import ops  # noqa: E402
from paper_1802_08435_amd import wavernn as W  # noqa: E402

P = ctypes.c_void_p(0x1000)      # never followed
ODD = ctypes.c_void_p(0x1001)
BIG = 1 << 40


def _logp(**kw):
    a = dict(dtype=W.F32, logits=P, n=4, v=16, stride=16, tokens=P, tb=8, top=0, logp=P, ent=P, lse=P, tl=P, ti=P, ws=P,
             wb=BIG)
    a.update(kw)
    return W.lib().wavernn_token_logprobs(*a.values(), None)


def _logp_grad(**kw):
    a = dict(dtype=W.F32, logits=P, n=4, v=16, stride=16, tokens=P, tb=8, lse=P, ent=P, gl=P, ge=P, gs=P, top=0, ti=P,
             gt=P, dz=P, dstride=16)
    a.update(kw)
    return W.lib().wavernn_token_logprobs_grad(*a.values(), None)


def _embed(**kw):
    a = dict(tdt=W.F32, table=P, v=16, d=8, tstride=8, ids=P, ib=8, n=4, scale=1.0, odt=W.F32, out=P, ostride=8)
    a.update(kw)
    return W.lib().wavernn_embed(*a.values(), None)


def _embed_grad(**kw):
    a = dict(dt=W.F32, dout=P, n=4, d=8, stride=8, ids=P, ib=8, v=16, scale=1.0, odt=W.F32, out=P, ws=P, wb=BIG)
    a.update(kw)
    return W.lib().wavernn_embed_grad(*a.values(), None)


def _norm(**kw):
    a = dict(dt=W.F32, x=P, n=4, d=8, xs=8, wdt=W.F32, g=P, b=P, eps=1e-5, y=ctypes.c_void_p(0x9000), ys=8, mean=P, rstd=P)
    a.update(kw)
    return W.lib().wavernn_layer_norm(*a.values(), None)


def _norm_grad(**kw):
    a = dict(dt=W.F32, dy=P, dys=8, x=ctypes.c_void_p(0x5000), xs=8, n=4, d=8, wdt=W.F32, g=P, mean=P, rstd=P,
             dx=ctypes.c_void_p(0x9000), dxs=8, dg=P, db=P, ws=P, wb=BIG)
    a.update(kw)
    return W.lib().wavernn_layer_norm_grad(*a.values(), None)


@pytest.mark.parametrize("call,bad,msg", [
    (_logp, dict(dtype=3), "dtype"), (_logp, dict(dtype=-1), "dtype"), (_logp, dict(n=-1), "n_rows"),
    (_logp, dict(n=1 << 31), "n_rows"), (_logp, dict(v=0), "n_classes"), (_logp, dict(logits=None), "logits is null"),
    (_logp, dict(logits=ODD), "aligned"), (_logp, dict(stride=-1), "stride"), (_logp, dict(stride=1 << 31), "stride"),
    (_logp, dict(tb=2), "token_bytes"), (_logp, dict(tokens=ODD), "aligned"), (_logp, dict(tokens=None), "without tokens"),
    (_logp, dict(top=-1), "top"), (_logp, dict(top=17), "top"), (_logp, dict(top=33, v=64), "top"),
    (_logp, dict(top=2, tl=None), "top_logp"), (_logp, dict(top=2, ti=None), "top_idx"),
    (_logp_grad, dict(dtype=9), "dtype"), (_logp_grad, dict(lse=None), "lse is null"),
    (_logp_grad, dict(tokens=None), "without tokens"), (_logp_grad, dict(ent=None), "without entropy"),
    (_logp_grad, dict(dz=None), "dlogits is null"), (_logp_grad, dict(dstride=15), "below the row"),
    (_logp_grad, dict(top=17), "top"), (_logp_grad, dict(top=2, gt=None), "g_top"),
    (_logp_grad, dict(top=2, ti=None), "top_idx"), (_logp_grad, dict(stride=17), "same row stride"),
    (_embed, dict(tdt=5), "dtype"), (_embed, dict(odt=W.BF16), "result's dtype"), (_embed, dict(v=0), "n_table"),
    (_embed, dict(v=1 << 31), "n_table"), (_embed, dict(d=0), "dim"), (_embed, dict(ib=1), "id_bytes"),
    (_embed, dict(ids=None), "ids is null"), (_embed, dict(n=-1), "n_ids"), (_embed, dict(table=None), "table is null"),
    (_embed, dict(out=None), "out is null"), (_embed, dict(ostride=7), "below the row"),
    (_embed_grad, dict(odt=W.F16), "result's dtype"), (_embed_grad, dict(v=0), "n_table"),
    (_embed_grad, dict(dout=None), "dout is null"), (_embed_grad, dict(out=None), "dtable is null"),
    (_embed_grad, dict(ids=ODD), "aligned"), (_embed_grad, dict(n=1 << 31), "n_ids"),
    (_norm, dict(eps=0.0), "eps"), (_norm, dict(eps=-1.0), "eps"), (_norm, dict(eps=float("nan")), "eps"),
    (_norm, dict(d=0), "dim"), (_norm, dict(wdt=W.BF16), "gamma's"), (_norm, dict(x=None), "x is null"),
    (_norm, dict(y=None), "y is null"), (_norm, dict(ys=7), "below the row"), (_norm, dict(y=P, ys=9), "same row stride"),
    (_norm, dict(g=ctypes.c_void_p(0x1002)), "aligned"),
    (_norm_grad, dict(mean=None), "mean or rstd"), (_norm_grad, dict(dy=None), "dy is null"),
    (_norm_grad, dict(dxs=7), "below the row"), (_norm_grad, dict(dx=P, dxs=16), "same row stride"),
    (_norm_grad, dict(wdt=W.F16), "gamma's"), (_norm_grad, dict(n=1 << 31), "n_rows"),
])
def test_entry_points_refuse(call, bad, msg):
    assert call(**bad) == W.E_INVALID
    assert msg in W.lib().wavernn_last_error().decode()


def test_workspace_sizes_and_refusal_of_a_short_workspace():
    L = W.lib()
    for fn, ok, bads in ((L.wavernn_token_logprobs_workspace, (4, 16, 2), [(-1, 16, 2), (4, 0, 0), (4, 16, 17), (4, 64, 33)]),
                         (L.wavernn_embed_grad_workspace, (4, 8, 16), [(-1, 8, 16), (4, 0, 16), (4, 8, 0), (1 << 31, 8, 16)]),
                         (L.wavernn_layer_norm_grad_workspace, (4, 8), [(-1, 8), (4, 0)])):
        assert fn(*ok) >= 0
        for b in bads:
            assert fn(*b) == -1, (fn, b)
    for need, call in ((L.wavernn_token_logprobs_workspace(1, 200000, 8),
                        lambda ws, wb: _logp(n=1, v=200000, stride=200000, top=8, ws=ws, wb=wb)),
                       (L.wavernn_embed_grad_workspace(50000, 8, 16), lambda ws, wb: _embed_grad(n=50000, ws=ws, wb=wb)),
                       (L.wavernn_layer_norm_grad_workspace(50000, 8), lambda ws, wb: _norm_grad(n=50000, ws=ws, wb=wb))):
        if need > 0:
            for ws, wb in ((None, need), (P, need - 1), (ctypes.c_void_p(0x1008), need)):
                assert call(ws, wb) == W.E_INVALID
                assert "workspace" in L.wavernn_last_error().decode()


def test_no_rows_launch_nothing():
    assert _logp(n=0, logits=None, tokens=None, logp=None) == W.OK
    assert _logp_grad(n=0, logits=None, dz=None) == W.OK
    assert _embed(n=0, ids=None, out=None) == W.OK
    assert _norm(n=0, x=None, y=None) == W.OK


def test_binding_refuses_cpu_tensors():
    z = torch.zeros(2, 4)
    i = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: ops.token_logprobs(z, i), lambda: ops.token_logprobs_grad(z, i, z[:, 0]),
                 lambda: ops.embed(z, i), lambda: ops.embed_grad(z, i, 4), lambda: ops.layer_norm(z),
                 lambda: ops.layer_norm_grad(z, z, z[:, 0], z[:, 0])):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_row_views():
    """Rows one distance apart are taken as they lie; any other view is refused."""
    t = torch.zeros(4, 6, 10)
    assert ops._rows("t", t) == (24, 10, 10)
    assert ops._rows("t", t[:, :, 2:7]) == (24, 5, 10)
    assert ops._rows("t", t[:, ::2, 2:7]) == (12, 5, 20)
    assert ops._rows("t", t[1]) == (6, 10, 10)
    assert ops._rows("t", t[0, 0]) == (1, 10, 10)
    assert ops._rows("t", t[:, :1]) == (4, 10, 60)
    assert ops._rows("t", t[:1, :1, :3]) == (1, 3, 3)
    assert ops._rows("t", torch.zeros(1, 5).expand(7, 5)) == (7, 5, 0)
    assert ops._rows("t", torch.zeros(1, 1, 5).expand(7, 3, 5)) == (21, 5, 0)
    assert ops._rows("t", torch.zeros(0, 3, 5)) == (0, 5, 5)
    assert ops._rows("t", torch.zeros(1, 5).as_strided((1, 5), (1 << 33, 1))) == (1, 5, 5)   # (no second row)
    assert ops._rows("t", torch.zeros(4, 1)[:, :1]) == (4, 1, 1)
    for bad in (t[..., ::2], t.transpose(1, 2), t[:, :4, :], torch.zeros(())):
        with pytest.raises(ValueError):
            ops._rows("t", bad)


def test_a_model_still_refuses_fp16_weights():
    c = W.Config(64, 0, 120, 1, 0, W.F16, W.R_DENSE, 1, -1, 0, 0)
    h = ctypes.c_void_p()
    assert W.lib().wavernn_create(ctypes.byref(c), ctypes.byref(W.Weights()), ctypes.byref(h)) == W.E_INVALID


def test_score_tokens_refuses():
    L = W.lib()
    assert L.wavernn_score_tokens(None, 1, 10, None, 0, None, None, 0, None, None, None, None, None) == W.E_INVALID
    assert "null model" in L.wavernn_last_error().decode()
