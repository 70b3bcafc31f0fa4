"""The operators of a layer of experts in 8 bits refuse what they can see on the host, before any CUDA call (no GPU needed)."""
import pytest
import torch

import f8_helpers as f8
from paper_1604_00981_b200 import binding as sgdb

lib = sgdb._lib
OK, INVALID, UNSUPPORTED = sgdb.SGDB_OK, sgdb.SGDB_ERR_INVALID_ARG, sgdb.SGDB_ERR_UNSUPPORTED
A = 1 << 12  # a non-null, aligned stand-in that is never dereferenced
BIG = (1 << 20) + 1


def refused(fn, good, **changes):
    for name, values in changes.items():
        for v in values:
            args = dict(good, **{name: v})
            assert getattr(lib, fn)(*args.values()) == INVALID, (fn, name, v)


def test_quantize():
    good = dict(x=A, dt=0, rows=4, width=200, ldx=200, q=A, fmt=0, ldq=208, scale=A, lds=2, stream=None)
    refused("sgdb_quantize", good, x=(None, A + 2), dt=(2, -1), rows=(-1, (1 << 30) + 1), width=(0, -1, BIG), ldx=(199,), q=(None,), fmt=(2, -1),
            ldq=(199,), scale=(None,), lds=(1, -1))
    assert lib.sgdb_quantize(*dict(good, rows=0, x=None, q=None, scale=None).values()) == OK


def test_quantize_matrices():
    good = dict(w=A, dt=1, batch=2, rows=130, cols=200, ldw=200, sw=26000, fmt=1, q=A, ldq=208, sq=130 * 208, qt=A, ldqt=144, sqt=200 * 144, scale=A,
                stream=None)
    refused("sgdb_quantize_matrices", good, w=(None, A + 1), dt=(2,), batch=(-1, 65536), rows=(0, BIG), cols=(0, BIG), ldw=(199,), sw=(25999,),
            fmt=(5,), ldq=(199,), sq=(10,), ldqt=(129,), sqt=(10,), scale=(None,))
    assert lib.sgdb_quantize_matrices(*dict(good, q=None, qt=None).values()) == INVALID
    assert lib.sgdb_quantize_matrices(*dict(good, batch=0).values()) == OK


def test_gate():
    good = dict(h=A, dt=0, rows=4, width=200, ldh=400, fmt=0, a=A, lda=200, a_scale=A, ldas=2, h8=A, ldh8=200, h_scale=A, ldhs=2, stream=None)
    refused("sgdb_gate", good, h=(None, A + 2), dt=(7,), rows=(-1,), width=(0, BIG), ldh=(399,), fmt=(2,), a=(None,), lda=(199,), a_scale=(None,),
            ldas=(1,), h8=(None,), ldh8=(199,), h_scale=(None,), ldhs=(1,))
    assert lib.sgdb_gate(*dict(good, rows=0, h=None).values()) == OK
    back = dict(da=A, ldda=200, dt=1, rows=4, width=200, fmt=0, h8=A, ldh8=200, h_scale=A, ldhs=2, dh=A, lddh=400, stream=None)
    refused("sgdb_gate_backward", back, da=(None, A + 1), ldda=(199,), dt=(3,), rows=(-2,), width=(0,), fmt=(-1,), h8=(None,), ldh8=(1,),
            h_scale=(None,), ldhs=(0,), dh=(None, A + 1), lddh=(399,))
    assert lib.sgdb_gate_backward(*dict(back, rows=0, da=None).values()) == OK


def test_experts_product():
    good = dict(x=A, fx=0, rows=10, depth=200, ldx=208, xs=A, ldxs=2, w=A, fw=1, E=3, width=70, ldw=208, sw=208 * 70, ws=A, sws=2, ws_n=2, ws_k=1,
                offsets=A, y=A, dt=0, ldy=70, info=A, stream=None)
    refused("sgdb_experts_product", good, x=(None, A + 8), fx=(2,), rows=(-1,), depth=(0, BIG), ldx=(192, 201), xs=(None,), ldxs=(1,), w=(None, A + 1),
            fw=(-1,), E=(0, 1025), width=(0, BIG), ldw=(192, 209), sw=(208 * 70 + 8, 208), ws=(None,), sws=(-1,), ws_n=(-1,), ws_k=(-1,),
            offsets=(None, A + 2), y=(None, A + 2), dt=(2,), ldy=(69,), info=(A + 1,))
    assert lib.sgdb_experts_product(*dict(good, rows=0, x=None, y=None).values()) == OK


def test_experts_gradient():
    need = sgdb.sgdb_experts_gradient_workspace_bytes(8192, 70, 200, 2)
    assert need >= 2 * 200 * 70 * 4  # few tiles and many rows: ranges of rows
    good = dict(dy=A, dt=0, rows=8192, width=70, lddy=70, x=A, fmt=0, depth=200, ldx=200, xs=A, ldxs=2, offsets=A, E=2, dw=A, dt_dw=0, lddw=200, sdw=14000,
                ws=A, ws_bytes=need, info=None, stream=None)
    refused("sgdb_experts_gradient", good, dy=(None, A + 2), dt=(2,), rows=(-1,), width=(0,), lddy=(69,), x=(None,), fmt=(3,), depth=(0,), ldx=(199,),
            xs=(None,), ldxs=(1,), offsets=(None, A + 1), E=(0, 1025), dw=(None, A + 1), dt_dw=(-1,), lddw=(199,), sdw=(13999,), ws=(None, A + 2),
            ws_bytes=(need - 1, 0), info=(A + 2,))
    for bad in ((-1, 8, 8, 1), (4, 0, 8, 1), (4, 8, BIG, 1), (4, 8, 8, 0), (4, 8, 8, 1025)):
        assert sgdb.sgdb_experts_gradient_workspace_bytes(*bad) == 0


def test_balance_loss():
    need = sgdb.sgdb_balance_loss_workspace_bytes(10, 6)
    assert need > 0
    good = dict(logits=A, dt=1, tokens=10, E=6, ld=6, expert=A, k=2, mask=None, loss=A, counts=A, slope=A, ws=A, ws_bytes=need, stream=None)
    refused("sgdb_balance_loss", good, logits=(None, A + 1), dt=(2,), tokens=(-1, (1 << 29) + 1), E=(0, 1025), ld=(5,), expert=(None, A + 2), k=(0, 33),
            loss=(None, A + 1), counts=(None,), slope=(None, A + 2), ws=(None, A + 2), ws_bytes=(need - 1,))
    back = dict(grad=A, logits=A, dt=0, tokens=10, E=6, ld=6, mask=None, slope=A, dlogits=A, ldd=6, stream=None)
    refused("sgdb_balance_loss_backward", back, grad=(None, A + 2), logits=(None, A + 2), dt=(-1,), tokens=(-1,), E=(0,), ld=(5,), slope=(None,),
            dlogits=(None, A + 1), ldd=(5,))
    assert lib.sgdb_balance_loss_backward(*dict(back, tokens=0, logits=None).values()) == OK
    for bad in ((-1, 4), (4, 0), (4, 1025)):
        assert sgdb.sgdb_balance_loss_workspace_bytes(*bad) == 0


def test_binding_refuses_shapes_and_types():
    """Tensors of the host are refused whatever else they are; the messages name the argument."""
    q, s = torch.empty(4, 16, dtype=torch.float8_e4m3fn), torch.empty(4, 1, dtype=torch.float8_e8m0fnu)
    for call in (lambda: sgdb.sgdb_quantize(torch.zeros(4, 16), q, s), lambda: sgdb.sgdb_quantize(torch.zeros(4, 16), torch.zeros(4, 16), s),
                 lambda: sgdb.sgdb_quantize_matrices(torch.zeros(4, 16), None, None, s), lambda: sgdb.sgdb_quantize_matrices(torch.zeros(1, 4, 16), None, None, s),
                 lambda: sgdb.sgdb_experts_product(q, s, q, s, None, torch.zeros(4, 3)), lambda: sgdb.empty_f8(3, 4, dtype=torch.float32)):
        with pytest.raises(ValueError):
            call()
    assert sgdb.empty_f8(3, 5, 17, dtype=torch.float8_e5m2).stride() == (160, 32, 1) and sgdb.empty_scale(7, 300).stride() == (16, 1)


@pytest.mark.parametrize("fmt", f8.FORMATS)
def test_the_tests_own_rounding(fmt):
    """The helper against a search through all numbers of the format."""
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(fmt).double()
    every = torch.sort(torch.unique(every[torch.isfinite(every)])).values
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(6, 128, dtype=torch.float64, generator=gen).float() * torch.exp2(torch.tensor([0.0, -130.0, 30.0, -5.0, 100.0, 0.0]))[:, None]
    x[5] = 0.0
    x[0, 3] = float("inf")
    x[0, 4] = float("nan")
    q, e = f8.quantized(x, fmt)
    for r in range(6):
        top = float(torch.where(torch.isfinite(x[r]), x[r].abs(), 0.0).max())
        er = int(e[r, 0])
        assert er == (0 if top == 0 else er) and top <= float(every[-1]) * 2.0 ** er and (er <= f8.LOWEST or top == 0 or top > float(every[-1]) * 2.0 ** (er - 1))
        v = x[r].double() / 2.0 ** er
        near = (v[:, None] - every[None, :]).abs().min(1).values
        got = q[r].double()
        assert bool((((got - v).abs() == near) | ~torch.isfinite(x[r])).all()) and bool(got[~torch.isfinite(x[r])].isnan().all())
