"""The 64-bit definitions of the operators around the products: gradients against differences of the forward functions, the
share of what dropout drops, refusals of the library's entry points (argument checks come before any GPU work)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_15102_amd as hlq
from oracle import around_oracle as ao
from paper_2406_15102_amd.autograd import grid_buckets, sequence_buckets

NAN = float("nan")


def _differences(f, x, step=1e-6):
    """Gradient of the number f(x) by central differences"""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        hi = f()
        x[i] = keep - step
        lo = f()
        x[i] = keep
        g[i] = (hi - lo) / (2 * step)
    return g


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_group_norm_gradients_against_differences(kind, p):
    rng = np.random.default_rng(kind)
    x, w, b, dy = rng.normal(size=(2, 5, 6)), rng.normal(size=6), rng.normal(size=6), rng.normal(size=(2, 5, 6))
    f = lambda: float((ao.group_norm_act(x, w, b, 3, 1e-3, kind, p, 11)[0] * dy).sum())   # noqa: E731
    got = ao.group_norm_act_backward(dy, x, w, b, 3, 1e-3, kind, p, 11)
    for g, v in zip(got, (x, w, b)):
        # central differences of step 1e-6: truncation 1e-12 times third derivatives, rounding 1e-16 / 1e-6; a kink of relu within the
        # step would show, and the draw has none
        np.testing.assert_allclose(g, _differences(f, v), rtol=1e-6, atol=2e-8)


@pytest.mark.parametrize("grid_w,Q,K,causal", [(0, 5, 5, True), (0, 2, 7, False), (2, 6, 6, False), (0, 6, 3, True)])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_map_gradients_against_differences(grid_w, Q, K, causal, p):
    rng = np.random.default_rng(Q * K)
    s, dP = rng.normal(size=(2, 2, Q, K)), rng.normal(size=(2, 2, Q, K))
    buckets = rng.integers(-1, 4, size=ao.rel_count(Q, K, grid_w))
    table = rng.normal(size=(4, 2))
    mask = (rng.random((2, 1, K)) < 0.8).astype(np.uint8)
    mask[1] = 0
    args = (buckets, mask, grid_w, causal, 0.7, p, 5)
    f = lambda: float((ao.rel_softmax(s, table, *args) * dP).sum())   # noqa: E731
    dS, dT = ao.rel_softmax_backward(dP, s, table, *args)
    np.testing.assert_allclose(dS, _differences(f, s), rtol=1e-6, atol=1e-9)
    np.testing.assert_allclose(dT, _differences(f, table), rtol=1e-6, atol=1e-9)
    assert not dS[1].any()                     # the batch that sees nothing


def test_what_dropout_drops():
    n = 1 << 18
    for p in (0.0, 0.1, 0.5, 1.0):
        f = ao.drop_factor(np.arange(n), p, 3)
        t = int(65536 * p + 0.5) / 65536
        # a binomial count: five standard deviations
        assert abs((f == 0).mean() - t) <= 5 * np.sqrt(t * (1 - t) / n)
        if 0 < p < 1:
            assert set(np.unique(f)) == {0.0, 1 / (1 - t)}
    a, b = (ao.drop_factor(np.arange(n), 0.5, s) == 0 for s in (3, 4))
    assert abs((a & b).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / n)         # two seeds are independent
    assert abs((a[1:] & a[:-1]).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / n)   # and neighbours


def test_bucket_helpers():
    of, n = grid_buckets(3, 4, signed=True)
    assert n == 35 and of.tolist() == list(range(35))
    of, n = grid_buckets(3, 4, signed=False)
    assert n == 12 and of.reshape(5, 7)[2, 3] == 0 and of.reshape(5, 7)[0, 0] == 11 and of.reshape(5, 7)[4, 1] == 10
    of, n = sequence_buckets(6, 6, 8)
    assert of.shape == (11,) and of[5] == 0 and of[4] == 1 and of[6] == 0 and int(of.max()) < 8      # keys ahead: bucket 0, never seen
    of, n = sequence_buckets(1, 300, 32)
    assert of[299] == 0 and of[298] == 1 and of[0] == 31
    of, n = sequence_buckets(40, 40, 16, causal=False)
    assert of[39] == 0 and of[38] == 1 and of[40] == 9 and int(of.max()) < 16
    for Q, K in ((1, 1), (3, 1), (1, 5)):
        assert sequence_buckets(Q, K, 2, causal=False)[0].shape == (Q + K - 1,)


# ---- refusals, without a GPU ----

FAKE = C.c_void_p(0x10000)      # never read: every call below is refused


def test_dropout_refuses():
    f = hlq.lib().hlq_dropout
    assert f(FAKE, None, 8, 0.1, 0, 2, FAKE, None) == 5
    for p in (-0.1, 1.5, NAN, float("inf")):
        assert f(FAKE, None, 8, p, 0, 0, FAKE, None) == 2
    assert f(FAKE, None, -1, 0.1, 0, 0, FAKE, None) == 2
    assert f(FAKE, None, (1 << 33) + 1, 0.1, 0, 0, FAKE, None) == 2      # more than the counter's words
    assert f(None, None, 8, 0.1, 0, 0, FAKE, None) == 1 and f(FAKE, None, 8, 0.1, 0, 0, None, None) == 1
    assert f(C.c_void_p(0x10001), None, 8, 0.1, 0, 0, FAKE, None) == 2 and f(C.c_void_p(0x10002), None, 8, 0.1, 0, 1, FAKE, None) == 2
    assert f(None, None, 0, 0.1, 0, 0, None, None) == 0                   # nothing to do


def test_group_norm_refuses():
    l = hlq.lib()

    def fwd(X=FAKE, w=FAKE, b=FAKE, Nb=2, P=4, Cc=8, G=2, eps=1e-5, act=0, p=0.0, dt=0, pdt=1, Y=FAKE, ws=FAKE, wsb=1 << 30):
        return l.hlq_group_norm_act(X, w, b, Nb, P, Cc, G, eps, act, p, 0, dt, pdt, Y, None, None, ws, wsb, None)

    assert fwd(X=None) == 1 and fwd(Y=None) == 1
    assert fwd(P=0) == 2 and fwd(G=3) == 2 and fwd(G=0) == 2 and fwd(Nb=-1) == 2 and fwd(Cc=0) == 2
    assert fwd(eps=0.0) == 2 and fwd(eps=NAN) == 2 and fwd(act=4) == 2 and fwd(act=-1) == 2 and fwd(p=1.1) == 2
    assert fwd(dt=2) == 5 and fwd(pdt=3) == 5
    assert fwd(Cc=2049, G=1) == 2 and fwd(Cc=2056, G=1) == 2 and fwd(Cc=1025, G=1) == 2          # groups wider than a workgroup takes
    assert fwd(Nb=1 << 20, Cc=1 << 12, G=32) == 2
    assert fwd(X=C.c_void_p(0x10001)) == 2 and fwd(w=C.c_void_p(0x10002)) == 2
    assert fwd(Nb=0) == 0
    big = dict(Nb=2, P=1 << 16, Cc=64, G=8)
    assert l.hlq_group_norm_workspace_bytes(2, 1 << 16, 64, 8, 0, 0) > 0
    assert fwd(wsb=8, **big) == 6 and fwd(ws=C.c_void_p(0x10008), **big) == 6
    assert l.hlq_group_norm_workspace_bytes(2, 4, 8, 3, 0, 0) == 0 and l.hlq_group_norm_workspace_bytes(2, 4, 8, 2, 9, 1) == 0

    def bwd(dY=FAKE, X=FAKE, mean=FAKE, rstd=FAKE, Nb=2, dX=FAKE, dw=FAKE, db=FAKE, ws=FAKE, wsb=1 << 30):
        return l.hlq_group_norm_act_backward(dY, X, FAKE, FAKE, mean, rstd, Nb, 4, 8, 2, 0, 0.0, 0, 0, 1, dX, dw, db, ws, wsb, None)

    assert bwd(dY=None) == 1 and bwd(X=None) == 1 and bwd(mean=None) == 1 and bwd(rstd=None) == 1
    assert bwd(dX=None, dw=None, db=None) == 1 and bwd(wsb=4) == 6
    assert bwd(Nb=0, dw=None, db=None) == 0


def test_map_refuses():
    l = hlq.lib()
    ok = dict(B=2, H=3, Q=4, K=4, grid_w=0, n_buckets=5, causal=0, mask_batches=0, mask_rows=0)

    def fwd(S=FAKE, table=FAKE, of=FAKE, mask=None, p=0.0, dt=0, tdt=1, out=FAKE, geom=True, **kw):
        g = hlq.hlq_rel_geom(**dict(ok, **kw))
        return l.hlq_rel_softmax(S, table, of, mask, C.byref(g) if geom else None, 1.0, p, 0, dt, tdt, out, None)

    assert fwd(geom=False) == 1 and fwd(S=None) == 1 and fwd(table=None) == 1 and fwd(of=None) == 1 and fwd(out=None) == 1
    assert fwd(dt=2) == 5 and fwd(tdt=7) == 5
    for bad in (dict(B=-1), dict(H=0), dict(H=65536), dict(Q=-1), dict(K=-4), dict(K=16385), dict(n_buckets=0), dict(grid_w=3), dict(causal=2),
                dict(grid_w=-1), dict(Q=6, grid_w=2), dict(Q=4097, K=4097, grid_w=17 * 241), dict(Q=4104, K=4104, grid_w=8), dict(mask_rows=1),
                dict(mask_batches=-1, mask_rows=1), dict(mask_batches=2, mask_rows=3), dict(B=1 << 30, H=60000, Q=1 << 30)):
        assert fwd(mask=FAKE, **bad) == 2, bad
    assert fwd(mask_batches=2, mask_rows=1) == 1                  # a mask is announced and none given
    assert fwd(p=NAN) == 2 and fwd(p=0.5, B=1 << 20, H=1 << 12) == 2      # more than the counter's words
    assert fwd(S=C.c_void_p(0x10001)) == 2 and fwd(of=C.c_void_p(0x10002)) == 2
    for none in (dict(B=0), dict(Q=0), dict(K=0)):
        assert fwd(S=None, table=None, of=None, out=None, **none) == 0
    g = hlq.hlq_rel_geom(**ok)
    need = l.hlq_rel_softmax_workspace_bytes(C.byref(g), 0)
    assert need > 0 and l.hlq_rel_softmax_workspace_bytes(C.byref(hlq.hlq_rel_geom(**dict(ok, H=0))), 0) == 0

    def bwd(dP=FAKE, dS=FAKE, dT=FAKE, ws=FAKE, wsb=1 << 30, **kw):
        g = hlq.hlq_rel_geom(**dict(ok, **kw))
        return l.hlq_rel_softmax_backward(dP, FAKE, FAKE, FAKE, None, C.byref(g), 1.0, 0.0, 0, 0, 1, dS, dT, ws, wsb, None)

    assert bwd(dP=None) == 1 and bwd(dS=None) == 1 and bwd(wsb=need - 1) == 6 and bwd(ws=C.c_void_p(0x10010)) == 6
    assert bwd(K=0, dP=None, dS=None, dT=None) == 0


def test_binding_refuses_wrong_tensors():
    x = torch.zeros((2, 4, 8))
    with pytest.raises(ValueError):
        hlq.hlq_dropout(x, torch.zeros((2, 4, 7)), 0.1, 0, x)
    with pytest.raises(ValueError):
        hlq.hlq_dropout(x, None, 0.1, 0, x.bfloat16())
    with pytest.raises(ValueError):
        hlq.hlq_group_norm_act(x, torch.ones(7), None, 2, 1e-5, 0, x.clone())
    with pytest.raises(ValueError):
        hlq.hlq_group_norm_act(x, torch.ones(8), torch.zeros(8).bfloat16(), 2, 1e-5, 0, x.clone())
    with pytest.raises(ValueError):
        hlq.hlq_group_norm_act(x, None, None, 2, 1e-5, 0, x.clone(), mean=torch.zeros(2))
    s = torch.zeros((1, 2, 3, 4))
    g = hlq.hlq_rel_geom(B=1, H=2, Q=3, K=4, n_buckets=5)
    with pytest.raises(ValueError):
        hlq.hlq_rel_softmax(s, torch.zeros((5, 2)), torch.zeros(5, dtype=torch.int32), None, g, 1.0, s.clone())
    with pytest.raises(ValueError):
        hlq.hlq_rel_softmax(s, torch.zeros((4, 2)), torch.zeros(6, dtype=torch.int32), None, g, 1.0, s.clone())
    with pytest.raises(ValueError):
        hlq.hlq_rel_softmax(s, torch.zeros((5, 2)), torch.zeros(6, dtype=torch.int32), torch.ones((1, 1, 4), dtype=torch.uint8), g, 1.0, s.clone())
    with pytest.raises(ValueError):      # nothing on the GPU
        hlq.hlq_dropout(x, None, 0.1, 0, x)
