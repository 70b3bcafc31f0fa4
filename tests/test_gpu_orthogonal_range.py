"""Newton-Schulz rules near the end of fp16's range, which the host lets through, against the iteration in 64 bits."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rule", [(1, 240.0, 0.0, 0.0), (1, -240.0, 0.0, 0.0), (2, 15.0, 0.0, 0.0), (1, 1.0, 230.0, 0.0), (1, 0.0, 0.0, 230.0)])
@pytest.mark.parametrize("R,C", [(64, 96), (1, 40), (300, 130)])
def test_large_values(cuda_device, R, C, rule):
    """A matrix of rank one: its one singular value is 1 and one row holds nearly all of it, so that elements come close to the
    bounds.  X, A and B are rounded to 11 bits, two or three times in a row: 2^-9 of the result (Frobenius norm) is allowed."""
    u = torch.zeros(R, C, device="cuda")
    u[R // 2, C // 3] = 1.0
    u[:, C // 3] += 1e-3 * torch.randn(R, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ns = sgdb.NewtonSchulz(*rule)
    x = u.double() / (torch.linalg.matrix_norm(u.double()) + ns.eps)
    for _ in range(ns.steps):
        a = x @ x.mT
        x = ns.a * x + (ns.b * a + ns.c * a @ a) @ x
    out = torch.empty_like(u)
    ws = torch.empty(sgdb.sgdb_orthogonalize_workspace_bytes(1, R, C), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_orthogonalize(u, out, ns, ws)
    assert float((out.double() - x).norm() / x.norm()) <= 2.0 ** -9
