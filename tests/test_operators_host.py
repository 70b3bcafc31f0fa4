"""The operators for language models refuse what they can see on the host, before any CUDA call (no GPU needed)."""
import ctypes
import itertools

import pytest

from paper_1604_00981_b200 import binding as sgdb

lib = sgdb._lib
OK, INVALID = sgdb.SGDB_OK, sgdb.SGDB_ERR_INVALID_ARG
A = 1 << 12  # a non-null, aligned stand-in that is never dereferenced


def refused(fn, good, **changes):
    """Every change of a good argument list is refused with INVALID; the good one is not called (it would launch)."""
    for name, values in changes.items():
        for v in values:
            args = dict(good, **{name: v})
            assert getattr(lib, fn)(*args.values()) == INVALID, (fn, name, v)


LN = dict(x=A, dt=0, tokens=4, width=8, ldx=8, gamma=A, beta=A, dt_w=0, eps=1e-5, y=A, ldy=8, mean=A, rstd=A, stream=None)
NAN, INF = float("nan"), float("inf")


def test_layer_norm():
    refused("sgdb_layer_norm", LN, x=(None, A + 2), dt=(2, -1), tokens=(-1,), width=(0, -3, (1 << 20) + 1), ldx=(7, -8), gamma=(A + 1,),
            beta=(A + 2,), dt_w=(5,), eps=(-1.0, NAN, INF), y=(None, A + 1), ldy=(7,), mean=(A + 2,), rstd=(A + 1,))
    assert lib.sgdb_layer_norm(*dict(LN, tokens=0, x=None, y=None).values()) == OK


def test_layer_norm_backward():
    need = sgdb.sgdb_layer_norm_backward_workspace_bytes(4, 8)
    assert need >= 2 * 8 * 4
    good = dict(dy=A, lddy=8, x=A, ldx=8, dt=1, tokens=4, width=8, gamma=A, dt_w=1, mean=A, rstd=A, dx=A, lddx=8, dgamma=A, dbeta=A, dt_g=0,
                ws=A, ws_bytes=need, stream=None)
    refused("sgdb_layer_norm_backward", good, dy=(None, A + 1), lddy=(7,), x=(None,), ldx=(0,), dt=(2,), tokens=(-1,), width=(0,), gamma=(A + 1,),
            dt_w=(9,), mean=(None, A + 2), rstd=(None,), dx=(None, A + 1), lddx=(1,), dgamma=(A + 2,), dbeta=(A + 1,), dt_g=(-1,),
            ws=(None, A + 2), ws_bytes=(need - 1, 0))
    for bad in ((-1, 8), (4, 0), (4, (1 << 20) + 1)):
        assert sgdb.sgdb_layer_norm_backward_workspace_bytes(*bad) == 0


def test_experts():
    refused("sgdb_route", dict(expert=A, tokens=4, k=2, E=8, offsets=A, slot=A, source=A, stream=None), expert=(None, A + 2),
            tokens=(-1, (1 << 29) + 1), k=(0, 33), E=(0, 1025), offsets=(None, A + 1), slot=(None, A + 1), source=(None, A + 3))
    refused("sgdb_dispatch", dict(x=A, dt=0, tokens=4, width=8, ldx=8, slot=A, k=2, offsets=A, E=8, xs=A, ldxs=8, stream=None), x=(None, A + 2),
            dt=(3,), tokens=(-1,), width=(0,), ldx=(7,), slot=(None, A + 2), k=(0, 33), offsets=(None,), E=(0, 2000), xs=(None, A + 1), ldxs=(7,))
    refused("sgdb_combine", dict(ys=A, dt=0, tokens=4, width=8, ldys=8, slot=A, k=2, weights=A, out=A, ldout=8, stream=None), ys=(None, A + 2),
            dt=(3,), tokens=(-1,), width=(0,), ldys=(7,), slot=(None, A + 2), k=(0, 33), weights=(A + 2,), out=(None, A + 1), ldout=(7,))
    good = dict(dout=A, lddout=8, ys=A, ldys=8, dt=1, tokens=4, width=8, slot=A, k=2, weights=A, offsets=A, E=8, dys=A, lddys=8, dweights=A,
                stream=None)
    refused("sgdb_combine_backward", good, dout=(None, A + 1), lddout=(7,), ys=(None,), ldys=(7,), dt=(2,), tokens=(-1,), width=(0,), slot=(None,),
            k=(0, 33), weights=(A + 1,), offsets=(None, A + 2), E=(0,), dys=(None,), lddys=(7,), dweights=(A + 1,))


def ns(**kw):
    return ctypes.byref(sgdb.NewtonSchulz(**kw)._c())


def bad_rules():
    return [ns(steps=0), ns(steps=65), ns(a=NAN), ns(b=INF), ns(c=-INF), ns(eps=-1.0), ns(eps=NAN), ns(eps=INF), None]


def test_orthogonalize():
    need = sgdb.sgdb_orthogonalize_workspace_bytes(2, 5, 7)
    good = dict(u=A, dt=0, batch=2, rows=5, cols=7, ldu=7, stride_u=35, ns=ns(), out=A, dt_out=1, ldout=7, stride_out=35, ws=A, ws_bytes=need,
                info=None, stream=None)
    refused("sgdb_orthogonalize", good, u=(None, A + 2), dt=(2,), batch=(-1, 65536), rows=(0, 32769), cols=(0, 32769), ldu=(6,), stride_u=(34, -35),
            ns=bad_rules(), out=(None, A + 1), dt_out=(2,), ldout=(6,), stride_out=(34,), ws=(None,), ws_bytes=(need - 1,), info=(A + 2,))
    assert lib.sgdb_orthogonalize(*dict(good, batch=0, u=None, out=None, ws=None, ws_bytes=0).values()) == OK
    for bad in ((-1, 5, 5), (1, 0, 5), (1, 5, 32769), (65535, 32768, 32768)):
        assert sgdb.sgdb_orthogonalize_workspace_bytes(*bad) == 0
        assert sgdb.sgdb_step_orthogonal_workspace_bytes(*bad) == 0


def test_step_orthogonal():
    need = sgdb.sgdb_step_orthogonal_workspace_bytes(1, 5, 8)
    opt = lambda **kw: ctypes.byref(sgdb.OrthogonalOpt(**kw)._c())  # noqa: E731
    good = dict(grad=A, dt=0, batch=1, rows=5, cols=8, ld=40, arrival=A, tags=A, t=0, N=3, b=1, theta=A, momentum=A, opt=opt(), mask=A, order=A,
                info=A, ws=A, ws_bytes=need, stream=None)
    refused("sgdb_step_orthogonal", good, grad=(None, A + 4), dt=(2,), batch=(-1,), rows=(0,), cols=(0,), ld=(39,), arrival=(None,), tags=(None,),
            N=(0, 1025), b=(-1, 1022), theta=(None, A + 2), momentum=(None, A + 1), mask=(None,), order=(None,), info=(None,), ws=(None,),
            ws_bytes=(need - 1,),
            opt=[None] + [opt(**{k: v}) for k, v in itertools.product(("lr", "momentum", "weight_decay", "scale"), (NAN, INF))] +
                [opt(newton_schulz=sgdb.NewtonSchulz(steps=0))])


def test_tensors_of_the_wrong_kind_are_refused_by_the_binding():
    import torch

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        sgdb.sgdb_layer_norm(x, None, None, 1e-5, x, stream=None)
    with pytest.raises(ValueError):
        sgdb.sgdb_orthogonalize(x, x, sgdb.NewtonSchulz(), x)
    with pytest.raises(ValueError):
        sgdb._vec(x, 32, "gamma", torch.float32)  # not on a GPU
    with pytest.raises(ValueError):
        sgdb._code(torch.float16, "x")
