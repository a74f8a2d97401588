"""Calls whose grid would have 2^32 threads or more in one dimension are refused before anything is launched: the runtime launches a part of such a grid and reports no error.
(No kernel runs: every address here is made up.)"""
import os

import pytest

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build

UNSUPPORTED = -9


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    return tri.lib()


def address(i):
    return (i + 1) << 44  # far apart, aligned


@pytest.mark.parametrize("method", [tri.FWD_SUBST, tri.BLOCK_RECURSIVE, tri.NEUMANN, tri.MIXED, tri.BLOCK_DIRECT, tri.NEWTON_SCHULZ])
@pytest.mark.parametrize("op", [tri.F32, tri.F16, tri.BF16])
def test_matrices(L, method, op):
    for n in (1 << 26, (1 << 26) + 1, 1 << 30):
        assert L.tri_inv_ex(address(0), address(1), n, 16, op, method, op, None, 0) == UNSUPPORTED


@pytest.mark.parametrize("gate", [tri.GATE_SCALAR, tri.GATE_PER_CHANNEL, tri.GATE_NONE])
@pytest.mark.parametrize("method", [tri.FWD_SUBST, tri.BLOCK_RECURSIVE, tri.NEUMANN, tri.MIXED, tri.BLOCK_DIRECT, tri.NEWTON_SCHULZ])
@pytest.mark.parametrize("key", [tri.F32, tri.BF16])
def test_chunks(L, gate, method, key):
    for B, T, H in ((1 << 20, 16, 64), (1, 16 << 26, 1), (3, 16 << 20, 32)):
        assert L.gdn_chunk_tri_inv_ex(address(0), address(1), address(2), address(3), B, T, H, 32, 16, key, gate, method, key, None, 0) == UNSUPPORTED
