"""The operators around the products under HIP graph capture and on another stream than their inputs': they allocate nothing,
synchronise nothing and record no memset when a workspace is at hand, and every replay gives the eager result."""
import pytest
import torch

import paper_2406_15102_amd as hlq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _group_norm(P):
    g = torch.Generator(device=DEV).manual_seed(P)
    x, dy = (torch.randn((3, P, 48), generator=g, device=DEV).bfloat16() for _ in range(2))
    w, b = torch.randn(48, generator=g, device=DEV), torch.randn(48, generator=g, device=DEV)
    mean, rstd = torch.zeros((3, 6), device=DEV), torch.zeros((3, 6), device=DEV)
    out = [torch.zeros_like(x), mean, rstd, torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b)]
    n = max(256, *(hlq.hlq_group_norm_workspace_bytes(3, P, 48, 6, x.dtype, k) for k in (False, True)))
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)

    def call():
        hlq.hlq_group_norm_act(x, w, b, 6, 1e-5, 2, out[0], mean, rstd, ws, 0.1, 3)
        hlq.hlq_group_norm_act_backward(dy, x, w, b, mean, rstd, 6, 2, out[3], out[4], out[5], ws, 0.1, 3)
    return call, out, ws


def _map(K):
    g = torch.Generator(device=DEV).manual_seed(K)
    s, dP = (torch.randn((2, 3, K, K), generator=g, device=DEV) for _ in range(2))
    table = torch.randn((5, 3), generator=g, device=DEV)
    of = torch.randint(0, 5, (2 * K - 1,), generator=g, device=DEV, dtype=torch.int32)
    geom = hlq.hlq_rel_geom(B=2, H=3, Q=K, K=K, n_buckets=5, causal=1)
    ws = torch.zeros(hlq.hlq_rel_softmax_workspace_bytes(geom, s.dtype), dtype=torch.uint8, device=DEV)
    out = [torch.zeros_like(s), torch.zeros_like(s), torch.zeros_like(table)]

    def call():
        hlq.hlq_rel_softmax(s, table, of, None, geom, 0.5, out[0], 0.1, 3)
        hlq.hlq_rel_softmax_backward(dP, s, table, of, None, geom, 0.5, out[1], out[2], ws, 0.1, 3)
    return call, out, ws


def _dropout(n):
    x = torch.randn(n, device=DEV)
    out = [torch.zeros_like(x)]
    return (lambda: hlq.hlq_dropout(x, x, 0.2, 4, out[0])), out, torch.zeros(256, dtype=torch.uint8, device=DEV)


CASES = [(_group_norm, 100), (_group_norm, 5000), (_map, 33), (_map, 2100), (_dropout, 10007)]


@pytest.mark.parametrize("make,size", CASES)
def test_replays_from_a_captured_graph(make, size):
    call, out, ws = make(size)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            call()
    torch.cuda.current_stream().wait_stream(s)
    for rep in range(4):
        for t in out:
            t.zero_()
        ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), "replay %d differs from the eager result" % rep


@pytest.mark.parametrize("make,size", CASES)
def test_on_another_stream(make, size):
    call, out, ws = make(size)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    for t in out:
        t.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("P", [100, 5000])
def test_registered_and_own_workspace(P):
    """Without a workspace of its own a call takes the registered one, or refuses where that is too small."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((2, P, 64), generator=g, device=DEV)
    mean, rstd, dw = torch.empty((2, 8), device=DEV), torch.empty((2, 8), device=DEV), torch.empty(64, device=DEV)
    y, dx, dx2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    hlq.hlq_group_norm_act(x, None, None, 8, 1e-5, 2, y, mean, rstd)
    hlq.hlq_group_norm_act_backward(x, x, None, None, mean, rstd, 8, 2, dx, dw, None)
    try:
        hlq.hlq_set_workspace(torch.empty(256, dtype=torch.uint8, device=DEV))
        with pytest.raises(hlq.HlqError) as ei:
            hlq.hlq_group_norm_act_backward(x, x, None, None, mean, rstd, 8, 2, dx2, dw, None)
        assert ei.value.status == 6
        keep = torch.empty(hlq.hlq_group_norm_workspace_bytes(2, P, 64, 8, x.dtype, True), dtype=torch.uint8, device=DEV)
        hlq.hlq_set_workspace(keep)
        hlq.hlq_group_norm_act_backward(x, x, None, None, mean, rstd, 8, 2, dx2, dw, None)
        torch.cuda.synchronize()
    finally:
        hlq.hlq_set_workspace(None)
    assert torch.equal(dx, dx2)
