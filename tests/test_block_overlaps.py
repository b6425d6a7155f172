"""Buffers of the norm's backward pass and of the few-token layer that share memory (CPU only:
refused on the host before anything is enqueued).  Each operand lies in a place of its own and
one is moved into another's at a time."""
import ctypes

import pytest
import torch

import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding

EC_OK, EC_ERR_ARG = 0, 1
GAP = 1 << 32


def places(sizes):
    """An address for each name, far from every other."""
    return {n: GAP * (i + 1) for i, n in enumerate(sizes)}


def shares(call, sizes, a, b):
    """Moves a onto b's first and last 16 bytes, and b's last onto a's first: all refused."""
    at = places(sizes)
    for where in (at[b], at[b] + (sizes[b] - 1) // 16 * 16, at[b] - (sizes[a] - 1) // 16 * 16):
        assert call(**{a: where}) == EC_ERR_ARG, (a, b, hex(where))
        assert "overlap" in ec.lib().ec_last_error().decode()


# ---- the norm's backward pass --------------------------------------------------

ROWS, D = 10, 64
NORM = {"H": ROWS * D * 2, "w": D * 2, "dY": ROWS * D * 2, "dH": ROWS * D * 2, "dX": ROWS * D * 2,
        "dw": D * 4, "ws": None}


def norm_backward(sizes=NORM, **over):
    a = {**places(NORM), **over}
    p = {n: ctypes.c_void_p(v) for n, v in a.items()}
    n = ec.lib().ec_rms_norm_workspace_size(1, ROWS, D)
    return ec.lib().ec_rms_norm_backward(1, ROWS, D, 1e-6, p["H"], p["w"], p["dY"], p["dH"],
                                         p["dX"], p["dw"], p["ws"], n, None)


@pytest.mark.parametrize("other", ["H", "w", "dY", "dH", "dX", "dw"])
def test_norm_backward_workspace(other):
    sizes = dict(NORM, ws=ec.lib().ec_rms_norm_workspace_size(1, ROWS, D))
    shares(norm_backward, sizes, "ws", other)
