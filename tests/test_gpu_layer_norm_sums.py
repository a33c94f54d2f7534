"""Weight gradients over many rows: sums whose fp32 chains grew with the number of rows.

Every term of a column is the same, dy = g_c and h = x_c (mean 0, rstd 1), so a long fp32 chain rounds the same way over and over:
chains of the lengths that these shapes had were off by 300 to 2000 u (u = 2^-24).  Bounds: a chain of at most 256 fp32
additions, 16 more inside a block, then 64 bits and a rounding of each partial sum and of the result; rows that no team holds
are added up in 64 bits throughout."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import U32, assert_within  # noqa: E402

pytestmark = GPU_MARKS


def _constant_columns(N, R, C):
    """(dy, x, mean, rstd) with equal rows, which take the memory of one, and the terms of dweight and dbias in 64 bits."""
    c = torch.arange(C, dtype=torch.float32, device=DEV) / C
    g, h = 0.1 + 0.9 * c, 1.5 - 0.4 * c
    dy, x = (v.expand(N, R, C) for v in (g, h))
    return dy, x, torch.zeros(N, R, device=DEV), torch.ones(N, R, device=DEV), g.double() * h.double(), g.double()


@pytest.mark.parametrize("N,R,C,chain", [(64, 100_000, 5, 0), (16, 8192, 20_000, 0), (16, 70_000, 1, 0), (600, 130_000, 16, 256),
                                         (260, 16_000, 1000, 256), (130, 3000, 16_384, 256), (300, 4000, 4000, 256)])
def test_chains_do_not_grow_with_the_rows(N, R, C, chain):
    import paper_2402_11857_amd as pkg

    say(f"case weight gradients of {N} x {R} equal rows of {C}")
    dy, x, mean, rstd, term_w, term_b = _constant_columns(N, R, C)
    dw, db = torch.full((N, C), 9.0, device=DEV), torch.full((N, C), 9.0, device=DEV)
    assert pkg.liec_layer_norm_backward(dy, x, mean, rstd, dweight=dw, dbias=db, need_dx=False) is None
    # h and its product round once each in fp32, a partial sum and the result once each
    u = (chain + (16 if chain else 0) + 4.1) * U32
    assert_within(dw, (R * term_w).expand(N, C), (R * term_w * u).expand(N, C), "dweight")
    assert_within(db, (R * term_b).expand(N, C), (R * term_b * u).expand(N, C), "dbias")


def test_sums_over_many_workers():
    import paper_2402_11857_amd as pkg

    N, R, C = 65_535, 2, 16
    say(f"case weight gradients of {N} workers with one sum")
    dy, x, mean, rstd, term_w, term_b = _constant_columns(N, R, C)
    weight = torch.ones(C, device=DEV).expand(N, C)
    dw, db = torch.full((C,), 9.0, device=DEV), torch.full((C,), 9.0, device=DEV)
    pkg.liec_layer_norm_backward(dy, x, mean, rstd, weight, dweight=dw, dbias=db, need_dx=False)
    # a block has two rows: no chain at all, and the workers' sums are added up in 64 bits
    u = (2 + 16 + 4.1) * U32
    assert_within(dw, N * R * term_w, N * R * term_w * u, "dweight")
    assert_within(db, N * R * term_b, N * R * term_b * u, "dbias")
