"""Host checks of the operators of token networks (no GPU): every refusal comes before
anything is enqueued, the workspace queries, and the binding's own checks.  Pointers
that are only checked are made-up numbers."""
import ctypes

import pytest

import paper_1911_04610_amd as xp

P = 1 << 20  # an aligned address that nothing reads


def _rms_fwd(**kw):
    a = xp.RmsnormFwdArgs(rows=4, dim=64, dtype=xp.BF16, eps=1e-6, x=P, ldx=64, weight=2 * P, y=3 * P, ldy=64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rms_bwd(**kw):
    a = xp.RmsnormBwdArgs(rows=4, dim=64, dtype=xp.BF16, eps=1e-6, dy=P, lddy=64, h=2 * P, ldh=64, weight=3 * P, dx=4 * P, lddx=64,
                          grad_weight=5 * P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rms_refused(a, status=xp.EINVAL):
    L = xp.lib()
    if isinstance(a, xp.RmsnormFwdArgs):
        assert L.xpipe_rmsnorm_fwd(ctypes.byref(a), None) == status
    else:
        need = ctypes.c_size_t()
        assert L.xpipe_rmsnorm_bwd_query(ctypes.byref(a), ctypes.byref(need)) == status
        assert L.xpipe_rmsnorm_bwd(ctypes.byref(a), None, 0, None) == status
    assert L.xpipe_last_error()


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(dim=0), dict(dtype=2), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None),
    dict(weight=None), dict(y=None), dict(x=P + 1), dict(weight=2 * P + 2), dict(y=3 * P + 1), dict(ldx=63), dict(ldy=0),
    dict(residual=4 * P, ldr=63), dict(sum=4 * P, lds=60), dict(sum=3 * P, lds=64), dict(y=2 * P), dict(sum=2 * P, lds=64), dict(y=P, ldy=72),
    dict(sum=P, lds=72), dict(residual=4 * P, ldr=64, sum=4 * P, lds=80), dict(dtype=xp.F32, x=P + 2),
])
def test_norm_forward_refusals(kw):
    _rms_refused(_rms_fwd(**kw))


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(dim=0), dict(dtype=-1), dict(eps=0.0), dict(dy=None), dict(h=None), dict(weight=None), dict(dy=P + 1), dict(lddy=10),
    dict(ldh=63), dict(lddx=63), dict(dx=4 * P + 1), dict(grad_weight=5 * P + 1), dict(residual=6 * P, ldr=1), dict(dx=3 * P), dict(dx=P, lddx=72),
    dict(dx=2 * P, lddx=72), dict(residual=4 * P, ldr=72), dict(grad_weight=P), dict(grad_weight=2 * P), dict(grad_weight=3 * P), dict(grad_weight=4 * P),
])
def test_norm_backward_refusals(kw):
    _rms_refused(_rms_bwd(**kw))


def test_norm_unsupported_null_and_workspaces():
    L = xp.lib()
    for make in (_rms_fwd, _rms_bwd):
        _rms_refused(make(dim=32769), xp.EUNSUPPORTED)
        _rms_refused(make(rows=1 << 40), xp.EUNSUPPORTED)
    _rms_refused(_rms_fwd(ldx=(1 << 20) + 1), xp.EUNSUPPORTED)
    need = ctypes.c_size_t()
    assert L.xpipe_rmsnorm_fwd(None, None) == xp.EINVAL
    assert L.xpipe_rmsnorm_bwd(None, None, 0, None) == xp.EINVAL
    assert L.xpipe_rmsnorm_bwd_query(None, ctypes.byref(need)) == xp.EINVAL
    assert L.xpipe_rmsnorm_bwd_query(ctypes.byref(_rms_bwd()), None) == xp.EINVAL
    a = _rms_bwd(rows=10000)
    assert L.xpipe_rmsnorm_bwd_query(ctypes.byref(a), ctypes.byref(need)) == xp.OK and need.value > 0
    for ws, n in ((None, need.value), (P, need.value - 1), (P + 128, need.value)):
        assert L.xpipe_rmsnorm_bwd(ctypes.byref(a), ws, n, None) == xp.EINVAL
    for kw in (dict(grad_weight=None), dict(rows=1)):  # nothing to join
        a = _rms_bwd(**dict(dict(rows=10000), **kw))
        assert L.xpipe_rmsnorm_bwd_query(ctypes.byref(a), ctypes.byref(need)) == xp.OK and need.value == 0
    # nothing to do
    assert L.xpipe_rmsnorm_fwd(ctypes.byref(_rms_fwd(rows=0, x=None, y=None)), None) == xp.OK
    assert L.xpipe_rmsnorm_bwd(ctypes.byref(_rms_bwd(rows=0)), None, 0, None) == xp.OK
    assert L.xpipe_rmsnorm_bwd(ctypes.byref(_rms_bwd(dx=None, grad_weight=None)), None, 0, None) == xp.OK


@pytest.mark.parametrize("buckets,heads,far,both,status", [
    (0, 4, 128, 0, xp.EINVAL), (1, 4, 128, 0, xp.EINVAL), (33, 4, 128, 1, xp.EINVAL), (2, 4, 128, 1, xp.EINVAL), (32, 0, 128, 1, xp.EINVAL), (32, -1, 128, 1, xp.EINVAL),
    (32, 4, 8, 1, xp.EINVAL), (32, 4, 16, 0, xp.EINVAL), (32, 4, 0, 1, xp.EINVAL), (-32, 4, 128, 1, xp.EINVAL),
    (1026, 4, 4096, 1, xp.EUNSUPPORTED), (32, 4097, 128, 1, xp.EUNSUPPORTED), (32, 4, (1 << 20) + 1, 1, xp.EUNSUPPORTED),
])
def test_relative_bias_refusals(buckets, heads, far, both, status):
    L = xp.lib()
    assert L.xpipe_relbias_fwd(P, buckets, heads, far, both, 2 * P, None) == status
    assert L.xpipe_relbias_bwd(P, buckets, heads, far, both, 2 * P, None) == status


def test_relative_bias_buffers():
    L = xp.lib()
    for f in (L.xpipe_relbias_fwd, L.xpipe_relbias_bwd):
        for a, b in ((None, P), (P, None), (P + 2, 2 * P), (P, 2 * P + 1), (P, P)):
            assert f(a, 32, 4, 128, 1, b, None) == xp.EINVAL


def _inputs(a, **kw):
    i = a.in_
    i.batch, i.nq, i.nk, i.heads, i.kv_heads, i.head_dim, i.dtype, i.scale = 2, 100, 120, 4, 2, 64, xp.BF16, 0.125
    i.q, i.k, i.v = xp.Heads(P, 25600, 256, 64), xp.Heads(2 * P, 15360, 128, 64), xp.Heads(3 * P, 15360, 128, 64)
    for k, v in kw.items():
        setattr(i if hasattr(i, k) else a, k, v)
    return a


def _attn_fwd(**kw):
    return _inputs(xp.AttentionFwdArgs(o=xp.Heads(4 * P, 25600, 256, 64), stats=5 * P), **kw)


def _attn_bwd(**kw):
    return _inputs(xp.AttentionBwdArgs(dout=xp.Heads(4 * P, 25600, 256, 64), o=xp.Heads(5 * P, 25600, 256, 64), stats=6 * P,
                                       dq=xp.Heads(7 * P, 25600, 256, 64), dk=xp.Heads(8 * P, 15360, 128, 64), dv=xp.Heads(9 * P, 15360, 128, 64)), **kw)


def _attn(a):
    L, need = xp.lib(), ctypes.c_size_t()
    f, q = (L.xpipe_attention_fwd, L.xpipe_attention_fwd_query) if isinstance(a, xp.AttentionFwdArgs) else (L.xpipe_attention_bwd, L.xpipe_attention_bwd_query)
    return f, q(ctypes.byref(a), ctypes.byref(need)), need.value


def _attn_refused(a, status=xp.EINVAL):
    f, got, _ = _attn(a)
    assert got == status and f(ctypes.byref(a), P, 1 << 40, None) == status
    assert xp.lib().xpipe_last_error()


COMMON = [
    dict(batch=-1), dict(nq=-1), dict(nk=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(dtype=5), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e300), dict(scale=1e-300), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=float("nan")), dict(cap=1e-300), dict(scale=2e38), dict(cap=2e38), dict(scale=1e10, cap=1e-30),
    dict(prefix=10 * P), dict(q_doc=10 * P), dict(k_doc=10 * P), dict(bias=10 * P), dict(bias=10 * P, bias_range=-1), dict(q_len=10 * P + 2),
    dict(bias=10 * P + 1, bias_range=3), dict(q=xp.Heads(None, 1, 1, 1)), dict(k=xp.Heads(None, 1, 1, 1)), dict(v=xp.Heads(3 * P + 1, 15360, 128, 64)),
    dict(q=xp.Heads(P, -1, 256, 64)), dict(q=xp.Heads(P, 25600, -1, 64)), dict(k=xp.Heads(2 * P, 15360, 128, -64)),
]


@pytest.mark.parametrize("kw", COMMON)
def test_attention_refusals(kw):
    _attn_refused(_attn_fwd(**kw))
    _attn_refused(_attn_bwd(**kw))


@pytest.mark.parametrize("kw", [
    dict(o=xp.Heads(None, 1, 1, 1)), dict(o=xp.Heads(4 * P + 1, 25600, 256, 64)), dict(o=xp.Heads(P, 25600, 256, 64)), dict(o=xp.Heads(2 * P, 25600, 256, 64)),
    dict(stats=5 * P + 2), dict(stats=4 * P), dict(stats=P), dict(o=xp.Heads(4 * P, 0, 256, 64)), dict(o=xp.Heads(4 * P, 25600, 255, 64)),
    dict(o=xp.Heads(4 * P, 25600, 64, 64)), dict(o=xp.Heads(4 * P, 25600, 256, 63)), dict(q_len=4 * P),
])
def test_attention_forward_refusals(kw):
    _attn_refused(_attn_fwd(**kw))


@pytest.mark.parametrize("kw", [
    dict(dout=xp.Heads(None, 1, 1, 1)), dict(o=xp.Heads(None, 1, 1, 1)), dict(stats=None), dict(stats=6 * P + 1), dict(dq=xp.Heads(None, 1, 1, 1)),
    dict(dk=xp.Heads(None, 1, 1, 1)), dict(dv=xp.Heads(None, 1, 1, 1)), dict(dq=xp.Heads(P, 25600, 256, 64)), dict(dk=xp.Heads(9 * P, 15360, 128, 64)),
    dict(dq=xp.Heads(4 * P, 25600, 256, 64)), dict(dq=xp.Heads(5 * P, 25600, 256, 64)), dict(dv=xp.Heads(9 * P, 0, 128, 64)),
    dict(dk=xp.Heads(8 * P, 15360, 64, 64)), dict(grad_bias=11 * P), dict(bias=10 * P, bias_range=4, grad_bias=10 * P), dict(bias=10 * P, bias_range=4, grad_bias=7 * P),
    dict(bias=10 * P, bias_range=4, grad_bias=11 * P + 2), dict(stats=8 * P),
])
def test_attention_backward_refusals(kw):
    _attn_refused(_attn_bwd(**kw))


@pytest.mark.parametrize("kw", [
    dict(head_dim=129), dict(nq=1 << 24), dict(nk=1 << 24), dict(batch=1 << 20, nq=1 << 20), dict(batch=1 << 13, heads=1 << 10, kv_heads=1 << 10, nq=1, nk=1), dict(batch=65536, nq=1, nk=1), dict(bias=10 * P, bias_range=(1 << 20) + 1),
    dict(q=xp.Heads(P, 25600, (1 << 22) + 1, 64)), dict(k=xp.Heads(2 * P, 1 << 41, 128, 64)),
])
def test_attention_unsupported(kw):
    _attn_refused(_attn_fwd(**kw), xp.EUNSUPPORTED)
    _attn_refused(_attn_bwd(**kw), xp.EUNSUPPORTED)


def test_attention_workspaces():
    L = xp.lib()
    for make in (_attn_fwd, _attn_bwd):
        f, _, _ = _attn(make())
        need = ctypes.c_size_t()
        q = L.xpipe_attention_fwd_query if make is _attn_fwd else L.xpipe_attention_bwd_query
        assert f(None, None, 0, None) == xp.EINVAL and q(None, ctypes.byref(need)) == xp.EINVAL and q(ctypes.byref(make()), None) == xp.EINVAL
        a = make(q_doc=10 * P, k_doc=11 * P)
        f, st, size = _attn(a)
        assert st == xp.OK and size >= 2 * 2 * 16
        for ws, n in ((None, size), (P, size - 1), (P + 128, size)):
            assert f(ctypes.byref(a), ws, n, None) == xp.EINVAL
    assert _attn(_attn_fwd())[2] == 0
    # one new token over a long cache: parts of the keys; the backward's sums of each query row
    assert _attn(_attn_fwd(nq=1, nk=1 << 20))[2] > 2 * 4 * 64 * 4
    assert _attn(_attn_bwd())[2] >= 2 * 4 * 100 * 4


@pytest.mark.parametrize("kw", [dict(batch=0), dict(nq=0), dict(nk=0), dict(batch=0, nq=0, nk=0), dict(nq=0, nk=0), dict(nq=0, q_doc=10 * P, k_doc=11 * P),
                                dict(nk=0, bias=10 * P, bias_range=3)])
def test_attention_queries_of_nothing(kw):
    assert _attn(_attn_fwd(**kw))[1] == xp.OK and _attn(_attn_bwd(**kw))[1] == xp.OK


def test_attention_of_nothing_enqueues_nothing():
    none = xp.Heads(None, 0, 0, 0)
    a = _attn_fwd(nq=0, q=none, o=none, stats=None)
    assert _attn(a)[0](ctypes.byref(a), None, 0, None) == xp.OK
    a = _attn_bwd(batch=0, q=none, k=none, v=none, dout=none, o=none, dq=none, dk=none, dv=none, stats=None)
    assert _attn(a)[0](ctypes.byref(a), None, 0, None) == xp.OK


def test_bindings_refuse_cpu_tensors():
    torch = pytest.importorskip("torch")
    x, w, q = torch.zeros(4, 8), torch.ones(8), torch.zeros(1, 4, 2, 8)
    for call in (lambda: xp.xpipe_rmsnorm_fwd(x, w, x.clone()), lambda: xp.xpipe_rmsnorm_bwd(x, x, w, x.clone()),
                 lambda: xp.xpipe_relbias_fwd(torch.zeros(8, 2), torch.zeros(2, 17)), lambda: xp.xpipe_relbias_bwd(torch.zeros(2, 17), torch.zeros(8, 2)),
                 lambda: xp.xpipe_attention_fwd(q, q, q, q.clone()),
                 lambda: xp.xpipe_attention_bwd(q, q, q, q, q, torch.zeros(1, 2, 4, 2), q.clone(), q.clone(), q.clone())):
        with pytest.raises(ValueError):
            call()


def test_bindings_check_shapes_before_the_library():
    """The helpers that turn tensors into arguments, on CPU tensors as if they were device -1's."""
    torch = pytest.importorskip("torch")
    xp.lib()
    z = torch.zeros
    assert xp._heads("q", z(2, 5, 3, 8), torch.float32, -1, (2, 5, 3, 8))[1:] == (120, 24, 8)
    for bad in (z(2, 5, 3, 8).transpose(2, 3), z(2, 5, 3, 8, dtype=torch.float64), z(2, 5, 4, 8)):
        with pytest.raises(ValueError):
            xp._heads("q", bad, torch.float32, -1, (2, 5, 3, 8))
    for bad in (z(3, dtype=torch.int64), z(4, dtype=torch.int32), z(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            xp._ints("q_len", bad, -1, (3,))
    for bad in (z(3, 4), z(3, 5, dtype=torch.float64), z(5, 3).t()):
        with pytest.raises(ValueError):
            xp._floats("bias", bad, -1, (3, 5))
    q, k = z(2, 5, 4, 8), z(2, 7, 2, 8)
    given = lambda q=q, k=k, v=k, bias=None, **kw: xp._attention_inputs(q, k, v, -1, None, True, 0.0, bias, *[kw.get(n) for n in ("q_len", "k_len", "prefix", "q_doc", "k_doc")])
    assert given()[:10] == (2, 5, 7, 4, 2, 8, xp.F32, True, 0, 8 ** -0.5)
    for kw in (dict(q=z(2, 5, 8)), dict(k=z(2, 7, 8)), dict(v=z(2, 6, 2, 8)), dict(k=z(2, 7, 2, 9), v=z(2, 7, 2, 9)), dict(bias=z(4, 6)), dict(bias=z(3, 7)), dict(bias=z(7)),
               dict(q_doc=z(2, 7, dtype=torch.int32)), dict(prefix=z(5, dtype=torch.int32))):
        with pytest.raises(ValueError):
            given(**kw)
    for table, values in ((z(8, 2), z(2, 16)), (z(8, 2), z(3, 17)), (z(8, 2).double(), z(2, 17)), (z(2, 8).t(), z(2, 17)), (z(8), z(2, 17))):
        with pytest.raises(ValueError):
            xp._relbias(table, "bias", values, -1)
