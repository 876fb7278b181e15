"""Host checks of edges of the operators of token networks (no GPU)."""
import ctypes

import pytest

import paper_1911_04610_amd as xp

P = 1 << 20  # an aligned address that nothing reads


@pytest.mark.parametrize("rows,dim,shared", [(1 << 24, 4096, 1), (1 << 24, 2048, 4), (1 << 26, 64, 32), (1 << 20, 9000, 1), (1 << 30, 8, 32)])
def test_norm_weight_gradient_has_a_part_for_every_256_rows_of_a_thread(rows, dim, shared):
    """shared: rows that a workgroup holds at a time.  Each part is dim fp32 values."""
    a = xp.RmsnormBwdArgs(rows=rows, dim=dim, dtype=xp.BF16, eps=1e-6, dy=P, lddy=dim, h=2 * P, ldh=dim, weight=3 * P, grad_weight=4 * P)
    need = ctypes.c_size_t()
    assert xp.lib().xpipe_rmsnorm_bwd_query(ctypes.byref(a), ctypes.byref(need)) == xp.OK
    assert need.value >= rows // (256 * shared) * dim * 4
