"""Tensors of another GPU than the current one: the binding's operators refuse them, the layers make their GPU the current one.
One GPU is enough: the tests put another number in the current device's place."""
import contextlib

import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb
from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu


def calls():
    T, D, E, k, N, b = 6, 16, 4, 2, 2, 1
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    byte = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    ws = byte(sgdb.sgdb_step_orthogonal_workspace_bytes(1, 8, 8))
    return {
        "layer_norm": lambda: sgdb.sgdb_layer_norm(f(T, D), None, None, 1e-5, f(T, D)),
        "layer_norm_backward": lambda: sgdb.sgdb_layer_norm_backward(f(T, D), f(T, D), None, f(T), f(T), f(T, D)),
        "route": lambda: sgdb.sgdb_route(i(T, k), E, i(E + 1), i(T, k), i(T * k)),
        "dispatch": lambda: sgdb.sgdb_dispatch(f(T, D), i(T, k), i(E + 1), f(T * k, D)),
        "combine": lambda: sgdb.sgdb_combine(f(T * k, D), i(T, k), None, f(T, D)),
        "combine_backward": lambda: sgdb.sgdb_combine_backward(f(T, D), f(T * k, D), i(T, k), None, i(E + 1), f(T * k, D)),
        "orthogonalize": lambda: sgdb.sgdb_orthogonalize(f(8, 8), f(8, 8), sgdb.NewtonSchulz(), ws),
        "step_orthogonal": lambda: sgdb.sgdb_step_orthogonal(f(N + b, 64), 1, 8, 8, f(N + b), i(N + b), 0, N, b, f(64), f(64), sgdb.OrthogonalOpt(),
                                                             byte(N + b), i(N), i(2), ws),
    }


@pytest.mark.parametrize("name", ["layer_norm", "layer_norm_backward", "route", "dispatch", "combine", "combine_backward", "orthogonalize",
                                  "step_orthogonal"])
def test_the_binding_refuses_tensors_of_another_device(cuda_device, monkeypatch, name):
    call = calls()[name]
    call()
    monkeypatch.setattr(sgdb, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        call()


def test_the_layers_run_on_their_tensors_device(cuda_device, monkeypatch):
    T, D, E, k = 6, 16, 4, 2
    x, gamma = torch.randn(T, D, device="cuda", requires_grad=True), torch.randn(D, device="cuda")
    ys, w, ids = torch.randn(T * k, D, device="cuda", requires_grad=True), torch.rand(T, k, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda")

    def all_of_them():
        r = layers.route(ids, E)
        return [layers.layer_norm(x, gamma), layers.dispatch(x, r), layers.combine(ys, w, r)]

    want = all_of_them()
    entered = []

    @contextlib.contextmanager
    def device(d):
        entered.append(d)
        yield

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", device)
    got = all_of_them()
    assert entered == [x.device] * 4
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del entered[:]
    for y, leaf in zip(got, (x, x, ys)):
        layers_backward = torch.autograd.grad(y, leaf, torch.ones_like(y))
        assert layers_backward[0].shape == leaf.shape
    assert entered == [x.device] * 3
