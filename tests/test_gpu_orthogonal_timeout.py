"""The waits of the orthogonalised update's products run out: the kernel ends normally, says SGDB_ERR_TIMEOUT in info and leaves
nothing behind.  Nothing is broken on purpose: with little patience a wait whose data is not there yet gives up, at other
places in other blocks and warps, every copy goes to a valid address and is waited for.  Afterwards, with the default
patience, the same call gives the bits that it gave before."""
import pytest
import torch

from helpers import selection_buffers
from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
NS = sgdb.NewtonSchulz()
# no patience at all (one probe decides); from less than a product's time to that of many products
LIMITS_NS = [0, 0, 1, 1_000, 3_000, 10_000, 30_000, 100_000, 300_000]


@pytest.fixture
def patience(cuda_device):
    yield sgdb.sgdb_set_wait_limit_ns
    sgdb.sgdb_set_wait_limit_ns(-1)


# tiles of 128 x 64 (one block each), and of 256 x 128 and 256 x 256 (pairs of blocks); flat, tall, several matrices
@pytest.mark.parametrize("dt_out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,C", [(1, 64, 64), (1, 256, 256), (3, 130, 200), (1, 2048, 2048), (1, 2304, 1100), (16, 512, 1408)])
def test_products_give_up_and_the_next_call_is_right(patience, B, R, C, dt_out):
    gen = torch.Generator(device="cuda").manual_seed(R + C)
    u = torch.randn(B, R, C, device="cuda", generator=gen)
    ws = torch.empty(sgdb.sgdb_orthogonalize_workspace_bytes(B, R, C), dtype=torch.uint8, device="cuda")
    info = torch.zeros(2, dtype=torch.int32, device="cuda")
    want = torch.empty(B, R, C, dtype=dt_out, device="cuda")
    sgdb.sgdb_orthogonalize(u, want, NS, ws, info)
    assert info.cpu().tolist() == [0, 0]
    for limit in LIMITS_NS:
        patience(limit)
        info.zero_()
        out = torch.empty_like(want)
        sgdb.sgdb_orthogonalize(u, out, NS, ws, info)
        status = info.cpu().tolist()
        assert status[0] == 0 and status[1] in (sgdb.SGDB_OK, sgdb.SGDB_ERR_TIMEOUT)
        if limit == 0:
            assert status[1] == sgdb.SGDB_ERR_TIMEOUT  # the first operands are not there at the first probe
        if status[1] == sgdb.SGDB_OK:
            assert torch.equal(out, want)
        else:  # a call that finds the time-out does nothing
            out.fill_(3.0)
            sgdb.sgdb_orthogonalize(u, out, NS, ws, info)
            assert bool((out == 3.0).all()) and info.cpu().tolist() == status
        patience(-1)
        info.zero_()
        out.fill_(5.0)
        sgdb.sgdb_orthogonalize(u, out, NS, ws, info)
        assert info.cpu().tolist() == [0, 0] and torch.equal(out, want)


def test_step_reports_it(patience):
    B, R, C, N, b = 2, 300, 500, 3, 1
    P, dev = B * R * C, "cuda"
    gen = torch.Generator(device=dev).manual_seed(2)
    grad = torch.randn(N + b, P, device=dev, generator=gen)
    arrival = torch.arange(1, N + b + 1, dtype=torch.float32, device=dev)
    tags = torch.zeros(N + b, dtype=torch.int32, device=dev)
    ws = torch.empty(sgdb.sgdb_step_orthogonal_workspace_bytes(B, R, C), dtype=torch.uint8, device=dev)

    def run():
        theta, m = torch.ones(P, device=dev), torch.zeros(P, device=dev)
        mask, order, info = selection_buffers(N + b, N, dev)
        sgdb.sgdb_step_orthogonal(grad, B, R, C, arrival, tags, 0, N, b, theta, m, sgdb.OrthogonalOpt(), mask, order, info, ws)
        return theta, m, info.cpu().tolist()

    want = run()
    assert want[2] == [N + b, sgdb.SGDB_OK]
    for limit in LIMITS_NS:
        patience(limit)
        assert run()[2][1] in ((sgdb.SGDB_ERR_TIMEOUT,) if limit == 0 else (sgdb.SGDB_OK, sgdb.SGDB_ERR_TIMEOUT))
        patience(-1)
        got = run()
        assert got[2] == want[2] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
