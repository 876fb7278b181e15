"""Host checks of the operators around a stage (no GPU): every refusal comes
before anything is enqueued, the workspace queries, and the binding's own
checks.  Pointers that are only checked are made-up numbers."""
import ctypes

import pytest

import paper_1911_04610_amd as xp

P = 1 << 20  # an aligned address that nothing reads


def _fwd(**kw):
    a = xp.LinearFwdArgs(rows=4, cin=64, cout=32, dtype=xp.BF16, act=xp.ACT_NONE, x=P, ldx=64, W=2 * P, ldw=64, y=3 * P, ldy=32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _bwd(**kw):
    a = xp.LinearBwdArgs(rows=4, cin=64, cout=32, dtype=xp.BF16, act=xp.ACT_NONE, dz=P, lddz=32, x=2 * P, ldx=64, W=3 * P,
                         ldw=64, dx=4 * P, lddx=64, grad_W=5 * P, grad_b=6 * P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _query(a):
    need = ctypes.c_size_t(0)
    f = xp.lib().xpipe_linear_fwd_query if isinstance(a, xp.LinearFwdArgs) else xp.lib().xpipe_linear_bwd_query
    return f(ctypes.byref(a), ctypes.byref(need)), need.value


def _refused(a, status=xp.EINVAL):
    assert _query(a)[0] == status
    f = xp.lib().xpipe_linear_fwd if isinstance(a, xp.LinearFwdArgs) else xp.lib().xpipe_linear_bwd
    assert f(ctypes.byref(a), None, 0, None) == status
    assert xp.lib().xpipe_last_error()


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(cin=0), dict(cout=0), dict(cin=-3), dict(dtype=2), dict(dtype=-1), dict(act=4), dict(act=-1),
    dict(x=None), dict(W=None), dict(y=None), dict(x=P + 1), dict(W=P + 1), dict(y=P + 1), dict(ldx=63), dict(ldw=0), dict(ldy=31),
    dict(ldx=-64), dict(residual=4 * P, ldr=31), dict(preact=4 * P, ldz=31), dict(bias=4 * P + 2), dict(y=P), dict(y=2 * P),
    dict(preact=3 * P, ldz=32), dict(preact=P, ldz=64), dict(preact=6 * P, ldz=32, bias=6 * P), dict(residual=3 * P, ldr=40), dict(residual=5 * P, ldr=32, preact=5 * P, ldz=32),
    dict(y=7 * P, bias=7 * P), dict(dtype=xp.F32, x=P + 2),
])
def test_linear_forward_refusals(kw):
    _refused(_fwd(**kw))


@pytest.mark.parametrize("kw", [dict(ldx=(1 << 20) + 1), dict(ldy=1 << 21), dict(rows=1 << 30)])
def test_linear_forward_unsupported(kw):
    _refused(_fwd(**kw), xp.EUNSUPPORTED)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(cin=0), dict(dtype=7), dict(act=9), dict(dz=None), dict(x=None), dict(W=None), dict(dz=P + 1), dict(lddz=31),
    dict(ldx=60), dict(ldw=60), dict(lddx=60), dict(act=xp.ACT_GELU), dict(preact=7 * P, ldz=64), dict(act=xp.ACT_GELU, preact=7 * P, ldz=60),
    dict(residual=7 * P, ldr=60), dict(dx=P), dict(dx=2 * P), dict(dx=3 * P), dict(residual=4 * P, ldr=72), dict(grad_W=None),
    dict(grad_W=5 * P + 2), dict(grad_b=6 * P + 2), dict(grad_b=5 * P), dict(grad_W=P), dict(grad_W=2 * P), dict(grad_b=4 * P),
    dict(act=xp.ACT_RELU, preact=4 * P, ldz=72),
])
def test_linear_backward_refusals(kw):
    _refused(_bwd(**kw))


def test_linear_null_arguments_and_workspaces():
    L = xp.lib()
    need = ctypes.c_size_t(0)
    for q, f in ((L.xpipe_linear_fwd_query, L.xpipe_linear_fwd), (L.xpipe_linear_bwd_query, L.xpipe_linear_bwd)):
        assert q(None, ctypes.byref(need)) == xp.EINVAL and f(None, None, 0, None) == xp.EINVAL
    assert L.xpipe_linear_fwd_query(ctypes.byref(_fwd()), None) == xp.EINVAL
    # a backward always packs operands that chunks of 16 bytes do not fit: rows of 99 elements
    a = _bwd(rows=100, cin=99, ldx=99, ldw=99, lddx=99)
    st, size = _query(a)
    assert st == xp.OK and size >= 100 * 104 * 2 + 32 * 104 * 2
    for ws, n in ((None, size), (P, size - 1), (P + 128, size)):
        assert L.xpipe_linear_bwd(ctypes.byref(a), ws, n, None) == xp.EINVAL
    # and so does a forward of many results
    a = _fwd(rows=4096, cin=99, cout=4096, ldx=99, ldw=99, ldy=4096)
    st, size = _query(a)
    assert st == xp.OK and size >= 2 * 4096 * 104 * 2
    assert L.xpipe_linear_fwd(ctypes.byref(a), P, size - 1, None) == xp.EINVAL


def test_linear_query_follows_alignment_and_splits():
    assert _query(_fwd()) == (xp.OK, 0) and _query(_bwd()) == (xp.OK, 0)
    assert _query(_fwd(rows=4096, cin=4096, cout=4096, ldx=4096, ldw=4096, ldy=4096)) == (xp.OK, 0)
    # up to 32 rows nothing is packed; operands of many results that chunks of 16 bytes do not fit are
    odd = dict(cin=65, ldx=65, ldw=65)
    many = dict(rows=4096, cout=4096, ldy=4096)
    assert _query(_fwd(rows=32, **odd)) == (xp.OK, 0) and _query(_fwd(**many, **odd))[1] > 0
    assert _query(_fwd(x=P + 2, **many))[1] > 0 and _query(_fwd(ldx=68, **many))[1] > 0
    assert _query(_fwd(**many)) == (xp.OK, 0) and _query(_fwd(y=3 * P + 2, **many)) == (xp.OK, 0)  # results need no alignment
    # a long reduction for few results is split, and its parts' sums need memory
    long = _bwd(rows=16384, lddz=32, ldx=64)
    st, size = _query(long)
    assert st == xp.OK and size >= 2 * 32 * 64 * 4
    # one product's workspace does not depend on what the other one lacks
    assert _query(_bwd(rows=16384, lddz=32, ldx=64, dx=None, W=None)) == (xp.OK, size)
    assert _query(_bwd(dx=None, grad_W=None, grad_b=None, x=None, W=None)) == (xp.OK, 0)


def test_no_rows_and_no_tokens_do_nothing():
    L = xp.lib()
    assert L.xpipe_linear_fwd(ctypes.byref(_fwd(rows=0, x=None, W=None, y=None)), None, 0, None) == xp.OK
    assert L.xpipe_linear_bwd(ctypes.byref(_bwd(rows=0)), None, 0, None) == xp.OK
    assert L.xpipe_linear_bwd(ctypes.byref(_bwd(dx=None, grad_W=None, grad_b=None)), None, 0, None) == xp.OK
    assert L.xpipe_act_bwd(None, None, None, 0, xp.ACT_RELU, xp.F32, None) == xp.OK
    assert L.xpipe_embedding_fwd(None, None, 0, 5, 8, 1.0, xp.F32, None, None) == xp.OK
    assert L.xpipe_embedding_bwd(None, None, 0, 5, 8, 1.0, xp.F32, None, None, 0, None) == xp.OK


@pytest.mark.parametrize("args", [
    (None, P, P, 4, 0, 0), (P, None, P, 4, 0, 0), (P, P, None, 4, 0, 0), (P, P, P, -1, 0, 0), (P, P, P, 4, 4, 0), (P, P, P, 4, -1, 0),
    (P, P, P, 4, 0, 2), (P + 1, P, P, 4, 0, 1), (P, P + 2, P, 4, 0, 0),
])
def test_act_bwd_refusals(args):
    assert xp.lib().xpipe_act_bwd(*args, None) == xp.EINVAL


def test_embedding_refusals():
    L = xp.lib()
    ok = dict(table=P, tokens=2 * P, n=4, vocab=10, dim=8, scale=1.0, dtype=xp.BF16, y=3 * P)

    def fwd(**kw):
        a = dict(ok, **kw)
        return L.xpipe_embedding_fwd(a["table"], a["tokens"], a["n"], a["vocab"], a["dim"], a["scale"], a["dtype"], a["y"], None)

    def bwd(ws=4 * P, size=1 << 30, **kw):
        a = dict(ok, **kw)
        return L.xpipe_embedding_bwd(a["table"], a["tokens"], a["n"], a["vocab"], a["dim"], a["scale"], a["dtype"], a["y"], ws, size, None)

    bad = [dict(table=None), dict(tokens=None), dict(y=None), dict(n=-1), dict(vocab=0), dict(dim=0), dict(vocab=-2), dict(dtype=3),
           dict(scale=float("nan")), dict(scale=float("inf")), dict(table=P + 1), dict(tokens=P + 2), dict(y=P), dict(y=2 * P)]
    for kw in bad:
        assert fwd(**kw) == xp.EINVAL and bwd(**kw) == xp.EINVAL, kw
    assert fwd(y=3 * P + 1) == xp.EINVAL and bwd(y=3 * P + 2) == xp.EINVAL
    for kw in (dict(n=1 << 30), dict(vocab=1 << 30), dict(dim=(1 << 20) + 1)):
        assert fwd(**kw) == xp.EUNSUPPORTED and bwd(**kw) == xp.EUNSUPPORTED, kw
    need = ctypes.c_size_t(0)
    assert L.xpipe_embedding_bwd_query(5000, 10, 8, ctypes.byref(need)) == xp.OK and need.value > 5000 * 8
    for ws, size in ((None, need.value), (P, need.value - 1), (P + 64, need.value)):
        assert bwd(ws=ws, size=size, n=5000) == xp.EINVAL
    assert L.xpipe_embedding_bwd_query(-1, 10, 8, ctypes.byref(need)) == xp.EINVAL
    assert L.xpipe_embedding_bwd_query(4, 0, 8, ctypes.byref(need)) == xp.EINVAL
    assert L.xpipe_embedding_bwd_query(4, 10, 8, None) == xp.EINVAL
    assert L.xpipe_embedding_bwd_query(1024, 10, 8, ctypes.byref(need)) == xp.OK and need.value == 0


def test_grad_norm_refusals():
    L = xp.lib()
    T = lambda *ts: (xp.TensorDesc * max(len(ts), 1))(*ts)
    big = T((P, 1 << 22))
    need = ctypes.c_size_t(0)
    assert L.xpipe_grad_norm_query(big, 1, ctypes.byref(need)) == xp.OK and need.value == (1 << 22) // 16384 * 8
    n = need.value
    call = lambda t, k, dtype=0, mx=1.0, sq=None, out=2 * P, ws=3 * P, size=n: L.xpipe_grad_norm(t, k, dtype, mx, sq, out, ws, size, None)
    assert call(big, -1) == xp.EINVAL and call(None, 1) == xp.EINVAL and call(T((None, 5)), 1) == xp.EINVAL
    assert call(T((P, -1)), 1) == xp.EINVAL and call(big, 1, dtype=2) == xp.EINVAL and call(big, 1, out=None) == xp.EINVAL
    for mx in (0.0, -1.0, float("nan")):
        assert call(big, 1, mx=mx) == xp.EINVAL
    assert call(T((P + 2, 1 << 22)), 1) == xp.EINVAL and call(T((P + 1, 1 << 22)), 1, dtype=1) == xp.EINVAL
    assert call(big, 1, out=2 * P + 2) == xp.EINVAL and call(big, 1, sq=2 * P + 4) == xp.EINVAL
    assert call(big, 1, ws=None) == xp.EINVAL and call(big, 1, size=n - 1) == xp.EINVAL and call(big, 1, ws=3 * P + 4) == xp.EINVAL
    assert call(T((P, 1 << 40)), 1) == xp.EUNSUPPORTED
    assert L.xpipe_grad_norm_query(T((P, 32768)), 1, ctypes.byref(need)) == xp.OK and need.value == 0
    assert L.xpipe_grad_norm_query(big, 1, None) == xp.EINVAL
    assert L.xpipe_clip_coef(None, 1, 1.0, P, None) == xp.EINVAL and L.xpipe_clip_coef(P, 1, 1.0, None, None) == xp.EINVAL
    assert L.xpipe_clip_coef(P, -1, 1.0, 2 * P, None) == xp.EINVAL and L.xpipe_clip_coef(P, 1, 0.0, 2 * P, None) == xp.EINVAL
    assert L.xpipe_clip_coef(P + 4, 1, 1.0, 2 * P, None) == xp.EINVAL


def test_clipped_update_refusals():
    L, hp, rp = xp.lib(), xp.Hyper().c(0), xp.Rule().c()
    adam = lambda clip, W=P: L.xpipe_adam_flat_clipped(W, 2 * P, 3 * P, 4 * P, 8, ctypes.byref(hp), 1, None, 0, None, 0, clip, None)
    rule = lambda clip, W=P: L.xpipe_rule_flat_clipped(W, 2 * P, None, 3 * P, 4 * P, 5 * P, 8, ctypes.byref(rp), ctypes.byref(hp), 1,
                                                       None, 0, None, 0, clip, None)
    for f in (adam, rule):
        assert f(None) == xp.EINVAL and f(6 * P + 2) == xp.EINVAL and f(6 * P, W=None) == xp.EINVAL and f(6 * P, W=P + 4) == xp.EINVAL
    assert L.xpipe_stage_set_clip(None, 1.0, P, None, 0) == xp.EINVAL


def test_binding_refuses_cpu_tensors_and_mixed_arguments():
    import torch
    t = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    with pytest.raises(ValueError):
        xp.xpipe_linear_fwd(t(2, 8), t(4, 8), None, t(2, 4))
    with pytest.raises(ValueError):
        xp.xpipe_linear_bwd(t(2, 4), t(2, 8), t(4, 8), t(2, 8))
    with pytest.raises(ValueError):
        xp.xpipe_act_bwd(t(4), t(4), t(4), xp.ACT_RELU)
    with pytest.raises(ValueError):
        xp.xpipe_embedding_fwd(t(4, 8), t(3, dtype=torch.int32), t(3, 8))
    with pytest.raises(ValueError):
        xp.xpipe_embedding_bwd(t(3, 8), t(3, dtype=torch.int32), t(4, 8))
    with pytest.raises(ValueError):
        xp.xpipe_grad_norm([t(5)], 1.0, t(2))
    lst, swapped = xp.TensorList([t(3), t(70000)]), t(90000)
    assert lst.workspace_bytes == 6 * 8
    lst.tensors[1].data = swapped
    lst.refresh()  # read where it is now, with the workspace that its size needs
    assert (lst.descs[1].p, lst.descs[1].n, lst.workspace_bytes) == (swapped.data_ptr(), 90000, 7 * 8)
    with pytest.raises(ValueError):
        xp.TensorList([])
    with pytest.raises(ValueError):
        xp.TensorList([t(3), t(3, dtype=torch.bfloat16)])
    with pytest.raises(ValueError):
        xp.TensorList([t(3, 4).t()])


def test_binding_refuses_tables_that_32_bits_cannot_count():
    import torch
    meta = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="meta")
    tokens = meta(3, dtype=torch.int32)
    assert xp._check_embedding(meta(3, 8), "y", tokens, meta(70000, 8), -1) == (70000, 8, 3)
    with pytest.raises(ValueError):  # (cut to 32 bits: a table of five rows)
        xp._check_embedding(meta(3, 1), "y", tokens, meta((1 << 32) + 5, 1), -1)
    with pytest.raises(ValueError):
        xp._check_embedding(meta(3, 1 << 31), "y", tokens, meta(2, 1 << 31), -1)


def test_embedding_query_refuses_what_the_call_refuses():
    L, need = xp.lib(), ctypes.c_size_t(77)
    q = lambda *a: L.xpipe_embedding_bwd_query(*a, ctypes.byref(need))
    for sizes in ((1 << 30, 10, 8), (1 << 60, 10, 8), ((1 << 63) - 1, 1, 1), (4, 1 << 30, 8), (4, 10, (1 << 20) + 1)):
        assert q(*sizes) == xp.EUNSUPPORTED and need.value == 77, sizes
        assert L.xpipe_embedding_bwd(P, 2 * P, *sizes, 1.0, xp.BF16, 3 * P, 4 * P, 1 << 62, None) == xp.EUNSUPPORTED
    # the largest that both take: keys and positions twice, and two rows of partial sums for every 64 positions
    n, dim = (1 << 30) - 1, 1 << 20
    assert q(n, (1 << 30) - 1, dim) == xp.OK and need.value >= 16 * n + 8 * (n // 64) * dim
