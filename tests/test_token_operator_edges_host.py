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


def test_norm_epsilon_whose_root_leaves_fp32():
    """A zero row's n is 1 / sqrt(eps): infinite in fp32 it would make 0 n a NaN."""
    L, need = xp.lib(), ctypes.c_size_t()
    for eps, status in ((2.0 ** -252, xp.OK), (2.0 ** -253, xp.EINVAL), (1e-300, xp.EINVAL), (5e-324, xp.EINVAL)):
        a = xp.RmsnormFwdArgs(rows=4, dim=64, dtype=xp.F32, eps=eps, x=P, ldx=64, weight=2 * P, y=3 * P, ldy=64)
        if status != xp.OK:
            assert L.xpipe_rmsnorm_fwd(ctypes.byref(a), None) == status
        b = xp.RmsnormBwdArgs(rows=4, dim=64, dtype=xp.F32, eps=eps, dy=P, lddy=64, h=2 * P, ldh=64, weight=3 * P, dx=4 * P, lddx=64)
        assert L.xpipe_rmsnorm_bwd_query(ctypes.byref(b), ctypes.byref(need)) == status


def _attention(nq, nk, q_doc, k_doc):
    """The queries of a forward and a backward call over 2 sequences."""
    none, some = xp.Heads(None, 0, 0, 0), lambda p, n: xp.Heads(p * P, n * 128, 128, 64)
    q, k = (some(1, nq) if nq else none), (some(2, nk) if nk else none)
    f, b, need, got = xp.AttentionFwdArgs(), xp.AttentionBwdArgs(), ctypes.c_size_t(), []
    for a in (f, b):
        i = a.in_
        i.batch, i.nq, i.nk, i.heads, i.kv_heads, i.head_dim, i.dtype, i.scale = 2, nq, nk, 2, 2, 64, xp.BF16, 0.125
        i.q, i.k, i.v, i.q_doc, i.k_doc = q, k, some(3, nk) if nk else none, q_doc, k_doc
        a.o = some(4, nq) if nq else none
    b.dout, b.dq, b.dk, b.dv = (some(p, n) if n else none for p, n in ((5, nq), (6, nq), (7, nk), (8, nk)))
    b.stats = 9 * P if nq else None
    L = xp.lib()
    return L.xpipe_attention_fwd_query(ctypes.byref(f), ctypes.byref(need)), L.xpipe_attention_bwd_query(ctypes.byref(b), ctypes.byref(need))


def test_documents_of_nothing_may_be_null():
    """An empty tensor has no address: where one side is empty, documents of the other alone are no mistake."""
    ok = (xp.OK, xp.OK)
    assert _attention(5, 0, 10 * P, None) == ok and _attention(0, 5, None, 10 * P) == ok and _attention(0, 0, None, None) == ok
    assert _attention(5, 0, 10 * P, 11 * P) == ok and _attention(5, 6, 10 * P, 11 * P) == ok
    assert _attention(5, 6, 10 * P, None) == _attention(5, 6, None, 10 * P) == (xp.EINVAL, xp.EINVAL)
