"""sgdb_step_orthogonal's arrays have to be as long as the workers and the matrices ask: shorter ones are refused, none is read
beyond its end."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
B, R, C, N, b = 2, 8, 16, 3, 1
W, P = N + b, B * R * C


def good():
    dev = "cuda"
    return dict(grad=torch.ones(W, P, device=dev), batch=B, rows=R, cols=C, arrival=torch.arange(1.0, W + 1, device=dev),
                tags=torch.zeros(W, dtype=torch.int32, device=dev), t=0, N=N, b=b, theta=torch.zeros(P, device=dev),
                momentum=torch.zeros(P, device=dev), opt=sgdb.OrthogonalOpt(), mask=torch.zeros(W, dtype=torch.uint8, device=dev),
                order=torch.zeros(N, dtype=torch.int32, device=dev), info=torch.zeros(2, dtype=torch.int32, device=dev),
                workspace=torch.empty(sgdb.sgdb_step_orthogonal_workspace_bytes(B, R, C), dtype=torch.uint8, device=dev), ld=P)


@pytest.mark.parametrize("name", ["arrival", "tags", "mask", "order", "info", "theta", "momentum", "grad"])
def test_short_arrays_are_refused(cuda_device, name):
    args = good()
    args[name] = args[name].reshape(-1)[:-1].clone()
    with pytest.raises(ValueError, match=name):
        sgdb.sgdb_step_orthogonal(**args)


def test_longer_ones_and_pieces_of_rows_are_taken(cuda_device):
    args = good()
    sgdb.sgdb_step_orthogonal(**args)
    want = args["theta"]
    args = good()
    wide = torch.zeros(W, P + 24, device="cuda")
    wide[:, 8:8 + P] = args["grad"]
    args.update(grad=wide.view(-1)[8:], ld=P + 24)
    for name in ("arrival", "tags", "mask", "order", "info"):
        args[name] = torch.cat([args[name], args[name]])
    sgdb.sgdb_step_orthogonal(**args)
    assert torch.equal(args["theta"], want)
