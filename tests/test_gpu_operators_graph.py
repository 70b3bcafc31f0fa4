"""The operators for language models captured in a CUDA graph: replays with other inputs in the same arrays give the bits of
the plain calls."""
import pytest
import torch

from helpers import selection_buffers
from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu


def worker(T, D, k, E, dtype):
    new = lambda *s: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    a = dict(x=new(T, D), dy=new(T, D), ys=new(T * k, D), gamma=f32(D), beta=f32(D), w=f32(T, k))
    ids = i32(T, k)
    out = dict(y=new(T, D), mean=f32(T), rstd=f32(T), dx=new(T, D), dgamma=f32(D), dbeta=f32(D), offsets=i32(E + 1), slot=i32(T, k), source=i32(T * k),
               xs=new(T * k, D), out=new(T, D), dys=new(T * k, D), dw=f32(T, k))
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")

    def call():
        sgdb.sgdb_layer_norm(a["x"], a["gamma"], a["beta"], 1e-5, out["y"], out["mean"], out["rstd"])
        sgdb.sgdb_route(ids, E, out["offsets"], out["slot"], out["source"])
        sgdb.sgdb_dispatch(out["y"], out["slot"], out["offsets"], out["xs"])
        sgdb.sgdb_combine(a["ys"], out["slot"], a["w"], out["out"])
        sgdb.sgdb_combine_backward(a["dy"], a["ys"], out["slot"], a["w"], out["offsets"], out["dys"], out["dw"])
        sgdb.sgdb_layer_norm_backward(a["dy"], a["x"], a["gamma"], out["mean"], out["rstd"], out["dx"], out["dgamma"], out["dbeta"], ws)

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for v in a.values():
            v.copy_(torch.randn(v.shape, device="cuda", generator=gen))
        ids.copy_(torch.randint(-1, E + 1, (T, k), device="cuda", generator=gen))

    return call, fill, list(out.values())


def server(B, R, C, dt_out):
    N, b, P = 4, 2, B * R * C
    W = N + b
    grad, theta, m = torch.empty(W, P, device="cuda"), torch.empty(P, device="cuda"), torch.empty(P, device="cuda")
    u, o = torch.empty(B, R, C, device="cuda"), torch.empty(B, R, C, dtype=dt_out, device="cuda")
    arrival, tags = torch.empty(W, device="cuda"), torch.zeros(W, dtype=torch.int32, device="cuda")
    mask, order, info = selection_buffers(W, N, "cuda")
    ws = torch.empty(sgdb.sgdb_step_orthogonal_workspace_bytes(B, R, C), dtype=torch.uint8, device="cuda")

    def call():
        sgdb.sgdb_orthogonalize(u, o, sgdb.NewtonSchulz(), ws)
        sgdb.sgdb_step_orthogonal(grad, B, R, C, arrival, tags, 0, N, b, theta, m, sgdb.OrthogonalOpt(), mask, order, info, ws)

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for v in (grad, theta, m, u, arrival):
            v.copy_(torch.randn(v.shape, device="cuda", generator=gen))

    return call, fill, [o, theta, m, mask, order, info]


CASES = {"ragged rows": lambda: worker(70, 333, 3, 5, torch.bfloat16), "whole chunks": lambda: worker(600, 2048, 2, 16, torch.float32),
         "single blocks": lambda: server(2, 130, 200, torch.bfloat16), "pairs of blocks": lambda: server(1, 2304, 1100, torch.float32)}


@pytest.mark.parametrize("case", CASES)
def test_replays(cuda_device, case):
    call, fill, outputs = CASES[case]()
    want = {}
    for seed in (1, 2, 3):
        fill(seed)
        call()
        want[seed] = [v.clone() for v in outputs]
    graph = torch.cuda.CUDAGraph()
    fill(1)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for seed in (2, 3, 2, 1):
        fill(seed)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want[seed]))
