"""The layers have no second derivatives: asking for them is an error, not a wrong number."""
import pytest
import torch

from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu


def calls():
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen).requires_grad_()  # noqa: E731
    ids = torch.randint(-1, 5, (20, 2), device="cuda", generator=gen).int()
    r = layers.route(ids, 5)
    x, gamma, beta = new(20, 24), new(24), new(24)
    ys, w = new(40, 24), new(20, 2)
    return {"layer_norm": (lambda: layers.layer_norm(x, gamma, beta), [x, gamma, beta]),
            "dispatch": (lambda: layers.dispatch(x, r), [x]), "combine": (lambda: layers.combine(ys, w, r), [ys, w])}


@pytest.mark.parametrize("name", ["layer_norm", "dispatch", "combine"])
def test_second_derivatives_are_refused(cuda_device, name):
    call, leaves = calls()[name]
    loss = lambda: (call() ** 3).sum() + sum((v ** 2).sum() for v in leaves)  # noqa: E731: a part whose second derivatives torch has
    first = torch.autograd.grad(loss(), leaves)
    with_graph = torch.autograd.grad(loss(), leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, with_graph))
    with pytest.raises(RuntimeError, match="once_differentiable"):
        sum((g ** 2).sum() for g in with_graph).backward()
