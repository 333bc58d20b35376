"""Coefficients of a tree object: the library reads 2 t_kv rows of n, so arrays that are smaller do not reach it."""
import types

import numpy as np
import pytest


@pytest.mark.parametrize("shape", [(7, 16), (8, 15), (8, 17), (128,), (2, 4, 16), (0, 16)])
def test_smaller_coefficients_are_refused(shape):
    from paper_2602_11470_amd import binding as B
    with pytest.raises(AssertionError):
        B.Tree(types.SimpleNamespace(n=16, h=None), types.SimpleNamespace(h=None, residues=4), 1, -24.0, 0.0, np.zeros(shape, dtype=np.int64))


@pytest.mark.parametrize("coeffs", [None, np.zeros((8, 16), dtype=np.int64), np.zeros((9, 16), dtype=np.int64)])
def test_others_arrive_there(coeffs):
    """Without a context every creation is refused."""
    from paper_2602_11470_amd import binding as B
    with pytest.raises(B.CachemirError) as e:
        B.Tree(types.SimpleNamespace(n=16, h=None), types.SimpleNamespace(h=None, residues=4), 1, -24.0, 0.0, coeffs)
    assert e.value.status == -1


@pytest.mark.gpu
def test_residues_of_a_cache():
    from paper_2602_11470_amd import binding as B
    ctx = B.config1()
    try:
        for heads, dim in ((8, 32), (3, 16), (16, 128), (8, 256)):
            kv = ctx.kv_create(heads, dim, 3)
            assert kv.residues == ctx.tree(kv).passes == ctx.rotary(heads, dim, 3, 4).residues if kv.residues <= 64 else True
    finally:
        ctx.close()
