"""Newton-Schulz rules whose products leave fp16's range for some matrix are refused on the host; those within it are not (no
GPU needed: an accepted rule gets as far as the question for the device).  The bounds are worked out here by brute force
over the singular values."""
import ctypes

import numpy as np
import pytest

from paper_1604_00981_b200 import binding as sgdb

lib = sgdb._lib
A = 1 << 12  # a non-null, aligned stand-in that is never dereferenced
MOST = 65504 / 256


def largest(steps, a, b, c):
    """The largest of X (but the last), A and B over all singular values that begin in [0, 1]."""
    s = np.linspace(0.0, 1.0, 200_001)
    top = 0.0
    with np.errstate(all="ignore"):
        for _ in range(steps):
            t = s * s
            top = max(top, s.max(), t.max(), np.abs(a + b * t + c * t * t).max())
            s = np.abs(s * (a + b * t + c * t * t))
            if not np.isfinite(s).all():
                return np.inf
            s = np.linspace(0.0, s.max(), 200_001)  # whatever lies between may come from another matrix's step
    return top


def status(steps, a, b, c):
    ns = ctypes.byref(sgdb.NewtonSchulz(steps, a, b, c)._c())
    step = ctypes.byref(sgdb.OrthogonalOpt(newton_schulz=sgdb.NewtonSchulz(steps, a, b, c))._c())
    need = sgdb.sgdb_step_orthogonal_workspace_bytes(1, 8, 8)
    first = lib.sgdb_orthogonalize(A, 0, 1, 8, 8, 8, 64, ns, A, 0, 8, 64, A, need, None, None)
    second = lib.sgdb_step_orthogonal(A, 0, 1, 8, 8, 64, A, A, 0, 3, 1, A, A, step, A, A, A, A, need, None)
    assert first == second
    return first


OUT = [(1, 300.0, 0.0, 0.0), (1, 1.0, -400.0, 0.0), (1, 1.0, 0.0, 300.0), (2, 20.0, 0.0, 0.0), (3, 8.2872, -23.5959, 17.3004), (3, 3.4445, 4.775, 2.0315),
       (64, 1.3, 0.0, 0.0), (2, 3e38, -3e38, 3e38), (1, 0.0, 0.0, 260.0), (1, 1.0, 2000.0, -2000.0), (64, 2.5, 0.0, 0.01)]


@pytest.mark.parametrize("rule", OUT)
def test_rules_out_of_range_are_refused(rule):
    assert largest(*rule) > MOST
    assert status(*rule) == sgdb.SGDB_ERR_UNSUPPORTED


WITHIN = [(5, 3.4445, -4.775, 2.0315), (64, 3.4445, -4.775, 2.0315), (2, 1.875, -1.25, 0.375), (64, 1.875, -1.25, 0.375), (64, 1.5, -0.5, 0.0),
          (64, 2.0, -1.0, 0.0), (1, 240.0, 0.0, 0.0), (2, 15.0, 0.0, 0.0), (64, 1.0, 0.0, 0.0), (64, 0.0, 0.0, 0.0), (1, 8.2872, -23.5959, 17.3004), (64, -1.5, 0.5, 0.0)]


@pytest.mark.parametrize("rule", WITHIN)
def test_rules_within_it_are_not(rule):
    import torch

    assert largest(*rule) <= MOST / 1.02 ** 2
    if torch.cuda.is_available():
        pytest.skip("would launch with the stand-in addresses")
    assert status(*rule) == sgdb.SGDB_ERR_CUDA  # no device here: the arguments were in order
