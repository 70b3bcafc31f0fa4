"""The layers take inputs as torch hands them over, whatever their strides: results and gradients are those of contiguous copies."""
import pytest
import torch

from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu

# a [rows, cols] view of other memory with the given values
FORMS = {
    "transposed": lambda v: v.t().contiguous().t(),
    "every other column": lambda v: torch.stack([v, v], -1).flatten(1)[:, ::2],
    "columns of a wider matrix": lambda v: torch.cat([v[:, :3], v, v], 1)[:, 3:3 + v.size(1)],
    "every other row": lambda v: torch.stack([v, v], 1).flatten(0, 1)[::2],
}


def run(f, tensors):
    """Output and gradients of f at views whose values are those of `tensors`."""
    leaves = [t.detach().requires_grad_(t.is_floating_point()) for t in tensors]
    out = f(*leaves)
    weight = torch.linspace(-1, 1, out.numel(), device="cuda").view(out.shape)
    return [out.detach()] + list(torch.autograd.grad((out.float() * weight).sum(), [v for v in leaves if v.requires_grad]))


def same(f, contiguous, views):
    for a, b in zip(run(f, contiguous), run(f, views)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", FORMS)
def test_any_strides(cuda_device, form, dtype):
    T, D, E, k = 24, 40, 5, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    view = FORMS[form]
    x, ys, w = new(T, D).to(dtype), new(T * k, D).to(dtype), new(T, k)
    ids = torch.randint(-1, E + 1, (T, k), device="cuda", generator=gen).int()
    r = layers.route(ids, E)
    for a, b in zip(vars(r).values(), vars(layers.route(view(ids), E)).values()):
        assert torch.equal(a, b)
    params = new(D, 2)
    same(layers.layer_norm, [x, params[:, 0].contiguous(), params[:, 1].contiguous()], [view(x), params[:, 0], params[:, 1]])
    same(lambda v: layers.layer_norm(v.view(2, T // 2, D)) if v.is_contiguous() else layers.layer_norm(v.unflatten(0, (2, T // 2))), [x], [view(x)])
    same(lambda v: layers.dispatch(v, r), [x], [view(x)])
    same(lambda y, v: layers.combine(y, v, r), [ys, w], [view(ys), view(w)])


def test_broadcast_inputs(cuda_device):
    """One row for all tokens, one weight for all choices: the gradient of the source is the sum that torch takes."""
    T, D, E, k = 12, 33, 4, 2
    gen = torch.Generator(device="cuda").manual_seed(2)
    row, ys = torch.randn(D, device="cuda", generator=gen), torch.randn(T * k, D, device="cuda", generator=gen)
    r = layers.route(torch.randint(0, E, (T, k), device="cuda", generator=gen).int(), E)
    for f, source, shape in ((layers.layer_norm, row, (T, D)), (lambda v: layers.dispatch(v, r), row, (T, D)),
                             (lambda v: layers.combine(ys, v, r), torch.randn(T, 1, device="cuda", generator=gen), (T, k))):
        a, b = source.clone().requires_grad_(), source.clone().requires_grad_()
        x, y = f(a.expand(shape)), f(b.expand(shape).contiguous())
        assert torch.equal(x, y)
        dout = torch.randn(x.shape, device="cuda", generator=gen)
        assert torch.equal(torch.autograd.grad(x, a, dout)[0], torch.autograd.grad(y, b, dout)[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_and_their_gradients_lie_alike_in_the_backward_call(cuda_device, dtype, monkeypatch):
    """layer norm's backward kernels read a row of x and of dy together where both begin as far from a 16-byte boundary."""
    T, D = 30, 41
    seen = []
    inner = layers.sgdb.sgdb_layer_norm_backward

    def watch(dy, x, *rest):
        seen.append((dy, x))
        return inner(dy, x, *rest)

    monkeypatch.setattr(layers.sgdb, "sgdb_layer_norm_backward", watch)
    whole = torch.randn(T + 3, D + 5, device="cuda").to(dtype)
    for x in (whole[:T, :D], whole[:T, 3:3 + D], whole[3:, :D].contiguous()[:T], whole.flatten()[1:1 + T * D].view(T, D)):
        x = x.detach().requires_grad_()
        other = torch.randn(3, D, device="cuda").to(dtype)
        y = torch.cat([other, layers.layer_norm(x)])  # the gradient is a piece of another tensor, 3 rows of odd width in
        want = torch.randn(T + 3, D, device="cuda").to(dtype)
        (got,) = torch.autograd.grad(y, x, want)
        dy, rows = seen.pop()
        assert (dy.data_ptr() - rows.data_ptr()) % 16 == 0 and (dy.stride(0) - rows.stride(0)) * dy.element_size() % 16 == 0
        z = x.detach().clone().requires_grad_()
        assert torch.equal(got, torch.autograd.grad(layers.layer_norm(z), z, want[3:].clone())[0])
