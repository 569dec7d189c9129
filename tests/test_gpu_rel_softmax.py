"""hlq_rel_softmax and its gradients against the 64-bit definition: rows of one key to 16384, sequences and grids, masks that leave
rows empty, masked places that hold anything, dropout, both types of scores and tables."""
import numpy as np
import pytest
import torch

import paper_2406_15102_amd as hlq
from oracle import around_oracle as ao
from paper_2406_15102_amd.autograd import HlqRelSoftmax, HlqRelSoftmaxFunction, sequence_buckets

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def _rel_index(Q, K, grid_w):
    k, q = np.arange(K), np.arange(Q)
    if not grid_w:
        return k[None] - q[:, None] + Q - 1
    h = K // grid_w
    return (k[None] // grid_w - q[:, None] // grid_w + h - 1) * (2 * grid_w - 1) + k[None] % grid_w - q[:, None] % grid_w + grid_w - 1


def _call(s, dP, table, buckets, mask, grid_w, causal, scale, p, seed):
    B, H, Q, K = s.shape
    geom = hlq.hlq_rel_geom(B=B, H=H, Q=Q, K=K, grid_w=grid_w, n_buckets=table.shape[0], causal=int(causal),
                            mask_batches=0 if mask is None else mask.shape[0], mask_rows=0 if mask is None else mask.shape[1])
    S, D, T, F = s.to(DEV), dP.to(DEV), table.to(DEV), buckets.to(DEV)
    M = None if mask is None else mask.to(DEV)
    P, dS, dT = torch.full_like(S, 9), torch.full_like(S, 9), torch.full_like(T, 9)
    hlq.hlq_rel_softmax(S, T, F, M, geom, scale, P, p, seed)
    n = hlq.hlq_rel_softmax_workspace_bytes(geom, s.dtype)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    hlq.hlq_rel_softmax_backward(D, S, T, F, M, geom, scale, dS, dT, ws, p, seed)
    return P, dS, dT


def _check(s, dP, table, buckets, mask, grid_w, causal, scale, p, seed, out):
    """z is rounded three times (product, bias, difference from the maximum), each half a unit of |z| or of the range of z that
    counts (softmax forgets what is 40 below the maximum); the exponential is within two units, on bf16 scores one of an argument
    rounded once more; sums of up to 16384 positive terms, 64 in a row: 64 units.  So a probability is relatively right to
    e = (4 max |z| + 70) units, the sum of p dp to e of sum p |dp|, and the table's gradient is a sum of n such terms."""
    args = (table.double().numpy(), buckets.numpy(), None if mask is None else mask.numpy(), grid_w, causal, scale, p, seed)
    s64, d64 = s.double().numpy(), dP.double().numpy()
    rel = _rel_index(s.shape[2], s.shape[3], grid_w)
    pr = ao.rel_softmax(s64, *args, rel=rel)
    clean = ao.rel_softmax(s64, *args[:-2], 0.0, 0, rel=rel)
    dS, dT = ao.rel_softmax_backward(d64, s64, *args, rel=rel)
    P, gS, gT = (t.double().cpu().numpy() for t in out)
    finite = np.where(np.isfinite(s64), s64, 0)
    e = (4 * min(abs(scale) * np.abs(finite).max() + np.abs(args[0]).max(), 200.0) + 70) * U
    half = 2.0 ** -8 if s.dtype == BF16 else U
    tiny = 2.0 ** -126                                   # results below the smallest normal number may be flushed
    bad = np.abs(P - pr) - (half + e) * np.abs(pr) - tiny
    assert np.all(bad <= 0), float(bad.max())
    keep = 65536 / (65536 - int(65536 * p + 0.5))
    dp = np.where(np.isfinite(d64), np.abs(d64), 0).max() * keep
    bad = np.abs(gS - dS) - (half * np.abs(dS) + abs(scale) * clean * 4 * e * dp) - tiny
    assert np.all(bad <= 0), float(bad.max())
    th = 2.0 ** -8 if table.dtype == BF16 else U
    # every element of a column: the errors of its terms, and a sum of n terms in fp32 with at most 256 in a row
    total = (clean * 2 * dp).sum((0, 2, 3))[None, :]
    assert np.all(np.abs(gT - dT) <= th * np.abs(dT) + (4 * e + 256 * U) * total + tiny), float(np.abs(gT - dT).max())


def _inputs(B, H, Q, K, grid_w, dtype, tdt, n_buckets=6, seed=0):
    g = torch.Generator().manual_seed(seed + 1000 * K + Q)
    s = (3 * torch.randn((B, H, Q, K), generator=g)).to(dtype)
    dP = torch.randn((B, H, Q, K), generator=g).to(dtype)
    table = torch.randn((n_buckets, H), generator=g).to(tdt)
    of = torch.randint(0, n_buckets, (ao.rel_count(Q, K, grid_w),), generator=g, dtype=torch.int32)
    return s, dP, table, of


LENGTHS = [(1, 1), (1, 7), (3, 8), (5, 9), (49, 49), (7, 64), (65, 65), (2, 127), (128, 128), (31, 197), (1, 256), (40, 257), (3, 511), (2, 513),
           (1, 1000), (6, 1025), (1, 2048), (5, 2049), (1, 4096), (3, 4100), (2, 8192), (1, 8193), (2, 16384), (300, 20), (37, 1)]


@pytest.mark.parametrize("Q,K", LENGTHS)
@pytest.mark.parametrize("dtype,tdt", [(BF16, F32), (F32, BF16)])
def test_lengths_of_sequences(Q, K, dtype, tdt):
    B, H = (3, 2) if Q * K < 5000 else (2, 1)
    s, dP, table, of = _inputs(B, H, Q, K, 0, dtype, tdt)
    for causal, p in ((False, 0.0), (True, 0.2)):
        args = (table, of, None, 0, causal, 0.5, p, 3)
        _check(s, dP, *args, _call(s, dP, *args))


@pytest.mark.parametrize("h,w", [(1, 1), (1, 9), (9, 1), (7, 7), (5, 8), (8, 8), (12, 11), (14, 14), (16, 16), (20, 24), (33, 32), (46, 45)])
@pytest.mark.parametrize("dtype,tdt", [(BF16, BF16), (F32, F32)])
def test_grids(h, w, dtype, tdt):
    n = h * w
    B, H = (5, 2) if n <= 256 else (1, 1)
    s, dP, table, of = _inputs(B, H, n, n, w, dtype, tdt, n_buckets=ao.rel_count(n, n, w))
    of = torch.arange(table.shape[0], dtype=torch.int32)           # signed distances: a bucket each
    for p in (0.0, 0.1):
        args = (table, of, None, w, False, 0.25, p, 8)
        _check(s, dP, *args, _call(s, dP, *args))


def test_the_longest_grid():
    s, dP, table, of = _inputs(1, 1, 4096, 4096, 64, BF16, F32, n_buckets=100)
    args = (table, of, None, 64, False, 0.25, 0.0, 8)
    _check(s, dP, *args, _call(s, dP, *args))


@pytest.mark.parametrize("Q,K,grid_w", [(16, 16, 4), (5, 61, 0), (9, 300, 0), (2, 1500, 0), (3, 2500, 0), (4, 9000, 0)])
@pytest.mark.parametrize("rows", ["one", "all"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masks_that_leave_rows_empty(Q, K, grid_w, rows, dtype):
    """Whatever stands in masked places -- not a number, infinite, the type's lowest value -- nothing of it is seen."""
    B = 7
    s, dP, table, of = _inputs(B, 2, Q, K, grid_w, dtype, F32)
    g = torch.Generator().manual_seed(5)
    mask = (torch.rand((3, 1 if rows == "one" else Q, K), generator=g) < 0.6).to(torch.uint8)
    mask[1] = 0                                   # nothing at all
    mask[2, :, K // 2:] = 0
    if rows == "all":
        mask[0, Q // 2] = 0                       # one query sees nothing
    hidden = torch.from_numpy(~ao.rel_seen(B, Q, K, mask.numpy(), False))[:, None].expand(s.shape)
    for junk in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
        s2, d2 = s.masked_fill(hidden, junk), dP.masked_fill(hidden, junk)
        for causal in (False, True):
            args = (table, of, mask, grid_w, causal, 0.5, 0.1, 3)
            out = _call(s2, d2, *args)
            assert not bool(out[0].cpu()[hidden].any()) and not bool(out[1].cpu()[hidden].any())
            _check(s, dP, *args, out)


@pytest.mark.parametrize("B", [1, 3, 5])
@pytest.mark.parametrize("Q,K", [(1, 5), (3, 40), (3, 130), (5, 300), (3, 700), (2, 3000)])
def test_table_values_that_nothing_sees(B, Q, K):
    """A value of the table that only masked places reach changes nothing, whatever it is, and its gradient is zero."""
    s, dP, table, of = _inputs(B, 2, Q, K, 0, F32, F32)
    of[Q] = 3
    of[np.arange(len(of)) != Q] %= 3
    mask = torch.from_numpy(_rel_index(Q, K, 0) != Q).to(torch.uint8)[None] * 255
    want = _call(s, dP, table, of, mask, 0, False, 0.5, 0.1, 3)
    _check(s, dP, table, of, mask, 0, False, 0.5, 0.1, 3, want)
    for junk in (float("nan"), float("inf"), -float("inf"), torch.finfo(F32).min):
        other = table.clone()
        other[3] = junk
        got = _call(s, dP, other, of, mask, 0, False, 0.5, 0.1, 3)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert not bool(got[2][3].any())


def test_scores_of_minus_infinity_and_the_lowest_value():
    for dtype in (BF16, F32):
        s, dP, table, of = _inputs(2, 2, 6, 70, 0, dtype, F32)
        s[0, 0, 0] = -float("inf")                              # a row without anything
        s[0, 0, 1, 5:] = -float("inf")
        s[0, 1, 2] = torch.finfo(dtype).min                      # all alike: as if there were no scores
        s[1, 1, 3, 9:] = torch.finfo(dtype).min
        args = (table, of, None, 0, False, 1.0, 0.0, 3)
        out = _call(s, dP, *args)
        assert not bool(out[0][0, 0, 0].any()) and not bool(out[1][0, 0, 0].any())
        pr = ao.rel_softmax(s.double().numpy(), table.double().numpy(), of.numpy(), None, 0, False, 1.0, 0.0, 3)
        got = out[0].double().cpu().numpy()
        ok = np.ones(got.shape, bool)
        ok[0, 1, 2] = False                                     # there the bias is below the scores' last place: a plain average
        assert np.all(np.abs(got - pr)[ok] <= (2.0 ** -8 if dtype == BF16 else 200 * U) * pr[ok] + 1e-30)
        assert np.allclose(got[0, 1, 2], 1 / 70, rtol=2.0 ** -8 if dtype == BF16 else 64 * U)
        s[1, 0, 0, 3] = float("nan")
        s[1, 0, 1, 3] = float("inf")
        out = _call(s, dP, *args)
        assert bool(torch.isnan(out[0][1, 0, :2]).all()) and bool(torch.isfinite(out[0][1, 0, 2:]).all())


def test_buckets_that_are_none_and_shared_ones():
    s, dP, table, of = _inputs(3, 4, 20, 33, 0, F32, F32, n_buckets=300)
    of = torch.randint(-40, 340, of.shape, dtype=torch.int32, generator=torch.Generator().manual_seed(3))
    args = (table, of, None, 0, False, 0.5, 0.0, 3)
    out = _call(s, dP, *args)
    _check(s, dP, *args, out)
    unused = torch.tensor([c not in set(of.tolist()) for c in range(300)])
    assert not bool(out[2].cpu()[unused].any())
    args = (table, torch.zeros_like(of) + 7, None, 0, True, 0.5, 0.0, 3)
    _check(s, dP, *args, _call(s, dP, *args))


def test_many_batches_and_heads_repeat_bit_for_bit():
    for shape, grid_w in (((70, 5, 36, 36), 6), ((1, 40, 130, 130), 0), ((600, 1, 1, 90), 0)):
        s, dP, table, of = _inputs(*shape, grid_w, BF16, F32)
        args = (table, of, None, grid_w, False, 0.5, 0.1, 3)
        a, b = _call(s, dP, *args), _call(s, dP, *args)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        _check(s, dP, *args, a)


def test_any_address():
    s, dP, table, of = _inputs(2, 3, 9, 21, 0, BF16, F32)
    args = (table, of, None, 0, False, 0.5, 0.1, 3)
    ref = _call(s, dP, *args)
    n = s.numel()
    geom = hlq.hlq_rel_geom(B=2, H=3, Q=9, K=21, n_buckets=6)
    for off in (1, 2, 5):
        S, D = (torch.zeros(n + 9, dtype=BF16, device=DEV)[off:off + n].view(s.shape).copy_(t) for t in (s, dP))
        whole = [torch.full((n + 9,), 4, dtype=BF16, device=DEV) for _ in range(2)]
        P, dS = (t[off + 1:off + 1 + n].view(s.shape) for t in whole)
        hlq.hlq_rel_softmax(S, table.to(DEV), of.to(DEV), None, geom, 0.5, P, 0.1, 3)
        hlq.hlq_rel_softmax_backward(D, S, table.to(DEV), of.to(DEV), None, geom, 0.5, dS, None, None, 0.1, 3)
        assert torch.equal(P, ref[0]) and torch.equal(dS, ref[1])
        for t in whole:
            assert bool((t[:off + 1] == 4).all()) and bool((t[off + 1 + n:] == 4).all())


def test_places_beyond_32_bits():
    B, H, N = 34, 16, 2048                              # 2.3e9 scores
    of, n = sequence_buckets(N, N, 32)
    table = torch.randn((n, H), device=DEV)
    s = torch.empty((B, H, N, N), dtype=BF16, device=DEV)
    for b in range(B):
        s[b].normal_()
    geom = hlq.hlq_rel_geom(B=B, H=H, Q=N, K=N, n_buckets=n)
    out = torch.empty_like(s)
    hlq.hlq_rel_softmax(s, table, of.to(DEV), None, geom, 1.0, out)
    rel = torch.from_numpy(_rel_index(N, N, 0)).to(DEV)
    for b, h in ((B - 1, H - 1), (31, 15), (32, 0)):
        want = torch.softmax(s[b, h].double() + table[:, h].double()[of.to(DEV).long()[rel]], -1)
        assert float(((out[b, h].double() - want).abs() / want).max()) <= 2.0 ** -8 + 200 * U
    dS = torch.empty_like(s)
    hlq.hlq_rel_softmax_backward(out, s, table, of.to(DEV), None, geom, 1.0, dS)
    b, h = B - 1, H - 1
    pr = torch.softmax(s[b, h].double() + table[:, h].double()[of.to(DEV).long()[rel]], -1)
    dp = out[b, h].double()
    want = pr * (dp - (pr * dp).sum(-1, keepdim=True))
    assert float(((dS[b, h].double() - want).abs() - 2.0 ** -8 * want.abs() - pr * 400 * U * float(dp.max())).max()) <= 0


def test_nothing_to_do():
    of = torch.zeros(9, dtype=torch.int32, device=DEV)
    table = torch.ones((4, 2), device=DEV)
    for shape in ((0, 2, 5, 5), (3, 2, 0, 10), (3, 2, 10, 0)):
        s = torch.empty(shape, device=DEV)
        geom = hlq.hlq_rel_geom(B=shape[0], H=2, Q=shape[2], K=shape[3], n_buckets=4)
        dT = torch.ones_like(table)
        hlq.hlq_rel_softmax(s, table, of, None, geom, 1.0, s.clone())
        hlq.hlq_rel_softmax_backward(s, s, table, of, None, geom, 1.0, s.clone(), dT)
        assert not bool(dT.any())


def test_wrapper_and_module():
    m = HlqRelSoftmax(3, grid=(4, 5), signed=False, scale=0.3, p=0.2, device=DEV)
    s = torch.randn((4, 3, 20, 20), device=DEV).requires_grad_()
    y = m(s)
    gy = torch.randn_like(y)
    y.backward(gy)
    out = _call(s.detach().cpu(), gy.cpu(), m.table.detach().cpu(), m.buckets.cpu(), None, 5, False, 0.3, 0.2, m.seed + 1)
    assert torch.equal(y, out[0]) and torch.equal(s.grad, out[1]) and torch.equal(m.table.grad, out[2])
    m = HlqRelSoftmax(2, n_buckets=8, causal=True, device=DEV)
    m.eval()
    long, token = torch.randn((2, 2, 30, 30), device=DEV), None
    token = long[:, :, -1:].contiguous()
    assert torch.allclose(m(token), m(long)[:, :, -1:], rtol=1e-6, atol=1e-7)      # the last query by itself: one new token
    mask = torch.ones((2, 1, 30), dtype=torch.bool, device=DEV)
    mask[1] = False
    assert not bool(m(long, mask)[1].any())
    t = s.detach().transpose(2, 3).requires_grad_()                                 # not dense: copied
    z = HlqRelSoftmaxFunction.apply(t, torch.zeros((9, 3), device=DEV), torch.zeros(39, dtype=torch.int32, device=DEV))
    assert torch.allclose(z, torch.softmax(t.detach(), -1), rtol=1e-5, atol=1e-7)
