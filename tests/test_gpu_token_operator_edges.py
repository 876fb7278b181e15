"""Edges of the operators of token networks on the GPU: values, sizes and places at which
a formula in 64 bits, or the same call in another layout, has to be met as anywhere else.
The bounds are those of test_gpu_token_operators.py, or written out at the test."""
import math

import pytest

import paper_1911_04610_amd as xp
import test_gpu_token_operators as usual
from test_gpu_token_operators import E24, Case, _close, _d, _dt, _gen, _half_step, _norm64, _torch

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- RMS norm
def _check_norm_backward(dy, h, w, eps, dtype):
    """dx and grad_weight within the bounds of test_norm_backward, and 3 * 2^-150 n more of dx: dy w, h c and their difference are
    fp32 values, which below 2^-126 are multiples of 2^-149, each rounded by half of that."""
    torch = _torch()
    u, (rows, dim) = _half_step(dtype), h.shape
    dx, gw = torch.full_like(dy, 7.0), torch.zeros(dim, device="cuda")
    xp.xpipe_rmsnorm_bwd(dy, h, w, dx, gw, eps=eps)
    h64, g64 = _d(h), _d(dy) * _d(w)
    n, _ = _norm64(h64, _d(w), eps)
    c, mag = n * n * (g64 * h64).mean(1, keepdim=True), n * n * (g64 * h64).abs().mean(1, keepdim=True)
    want = n * (g64 - h64 * c)
    tol = 6 * E24 * n * (g64.abs() + h64.abs() * (c.abs() + mag)) + 2 * E24 * want.abs() + 3 * 2.0 ** -150 * n
    _close(dx, want, u * (want.abs() + tol) + tol, "dx")
    terms = _d(dy) * h64 * n
    _close(gw, terms.sum(0), (rows / 256 + 20) * E24 * terms.abs().sum(0), "grad_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [40, 300, 1000, 2047, 4099, 9000, 20000])
def test_norm_products_that_leave_fp32(dim, dtype):
    """Rows whose h and dy are in fp32's range and whose products are not, among rows of ordinary size."""
    torch = _torch()
    g = _gen(dim)
    h, dy = torch.randn(9, dim, generator=g), torch.randn(9, dim, generator=g)
    h[1], dy[1] = h[1] * 1e15, dy[1] * 1e24
    h[4], dy[4] = h[4] * 1e-9, h[4] * 1e-36 + dy[4] * 1e-37
    h[5], dy[5] = h[5] * 1e14, h[5].abs() * 1e25 * torch.sign(h[5])
    dy[7] = 0
    w = 1 + 0.1 * torch.randn(dim, generator=g)
    _check_norm_backward(dy.to(_dt(dtype)).cuda(), h.to(_dt(dtype)).cuda(), w.cuda(), 1e-30, dtype)


def test_norm_of_more_rows_than_a_launch_has_workgroups():
    """2^22 + 3 rows of 1024 threads each, in place: more threads than a launch may have."""
    torch = _torch()
    rows, dim = (1 << 22) + 3, 8200
    if torch.cuda.mem_get_info()[0] < rows * dim * 2 + (8 << 30):
        pytest.skip("needs 77 GB of free memory")
    x = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 777, (1 << 21) - 1, 1 << 21, (1 << 21) + 5, rows - 4, rows - 1]).cuda()
    some, w = torch.randn(8, dim, generator=_gen(8)).bfloat16().cuda(), (1 + 0.1 * torch.randn(dim, generator=_gen(9))).cuda()
    x[at] = some
    want = torch.empty_like(some)
    xp.xpipe_rmsnorm_fwd(some, w, want)
    xp.xpipe_rmsnorm_fwd(x, w, x)
    assert torch.equal(x[at], want)
    del x
    torch.cuda.empty_cache()


def test_norm_weight_gradient_of_many_rows():
    """2^21 rows whose first 2048 are 2^24 times as large as the others: each fp32 sum that begins with one of them loses every
    term that follows, so the gradient is off by about its number of terms over 2^24, 256 + 20 at most."""
    torch = _torch()
    rows, dim, large = 1 << 21, 600, 2048
    h = torch.ones(rows, dim, dtype=torch.bfloat16, device="cuda")
    dy = torch.ones_like(h)
    dy[:large] = 2.0 ** 24
    gw = torch.zeros(dim, device="cuda")
    xp.xpipe_rmsnorm_bwd(dy, h, torch.ones(dim, device="cuda"), None, gw, eps=1e-12)
    want = torch.full((dim,), large * 2.0 ** 24 + rows - large, dtype=torch.float64)
    _close(gw, want, (256 + 20) * E24 * want, "grad_weight")


@pytest.mark.parametrize("rows,dim", [((1 << 19) + 1, 520), ((1 << 17) + 700, 2100), ((1 << 16) + 1, 8200)])
def test_norm_gradients_of_more_rows_than_a_launch_takes(rows, dim):
    """The rows of a second launch: their dx are those of a call of their own, and grad_weight has all rows' terms."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    make = lambda scale: (torch.randn(rows, dim, generator=g, device="cuda") * scale).bfloat16()
    dy, h, r, w = make(0.1), make(2.0), make(0.1), 1 + 0.1 * torch.randn(dim, generator=g, device="cuda")
    dx, gw = torch.empty_like(dy), torch.ones(dim, device="cuda")
    xp.xpipe_rmsnorm_bwd(dy, h, w, dx, gw, eps=1e-5, residual=r)
    for part in (slice(0, 300), slice(rows - 1000, rows)):
        alone = torch.empty_like(dx[part])
        xp.xpipe_rmsnorm_bwd(dy[part], h[part], w, alone, None, eps=1e-5, residual=r[part])
        assert torch.equal(dx[part], alone)
    want, size = torch.ones(dim, dtype=torch.float64, device="cuda"), torch.ones(dim, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 1 << 15):
        h64 = h[i:i + (1 << 15)].double()
        terms = dy[i:i + (1 << 15)].double() * h64 / (h64.square().mean(1, keepdim=True) + 1e-5).sqrt()
        want += terms.sum(0)
        size += terms.abs().sum(0)
    _close(gw, _d(want), (256 + 20) * E24 * _d(size), "grad_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_zero_rows_under_the_least_epsilon(dtype):
    """n = 2^126: y is 0 and dx 2^126 dy, exactly."""
    torch = _torch()
    for dim in (40, 700, 9000):
        x, w = torch.zeros(3, dim, dtype=_dt(dtype), device="cuda"), torch.ones(dim, device="cuda")
        dy, y, dx, gw = torch.full_like(x, 1.5), torch.full_like(x, 7.0), torch.full_like(x, 7.0), torch.zeros(dim, device="cuda")
        xp.xpipe_rmsnorm_fwd(x, w, y, eps=2.0 ** -252)
        xp.xpipe_rmsnorm_bwd(dy, x, w, dx, gw, eps=2.0 ** -252)
        assert bool(y.eq(0).all()) and bool(dx.float().eq(1.5 * 2.0 ** 126).all()) and bool(gw.eq(0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", [(8200, 512), (65600, 40), (16390, 100), (8195, 200)])
def test_norm_of_more_rows_than_workgroups(rows, dim, dtype):
    """Forward: a workgroup's second round of rows."""
    usual.test_norm_forward(rows, dim, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", [(300, 9000), (270, 20000), (600, 6000), (20000, 40), (2100, 1500)])
def test_norm_gradients_of_more_rows_than_workgroups(rows, dim, dtype):
    usual.test_norm_backward(rows, dim, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [40, 300, 2047, 4099, 9000, 20000])
def test_norm_extremes_in_every_type_and_width(dim, dtype):
    """Rows whose squares leave fp32 on either side and zero rows, among ordinary ones; values that are not finite stay in their row."""
    torch = _torch()
    u, g = _half_step(dtype), _gen(dim)
    x, w = torch.randn(11, dim, generator=g), (1 + 0.1 * torch.randn(dim, generator=g)).cuda()
    for row, by in ((1, 1e25), (2, 1e-30), (3, 0.0), (6, 1e18), (7, 1e-12)):
        x[row] *= by
    x[4, dim // 3], x[9, dim - 1] = math.nan, math.inf
    x, keep = x.to(_dt(dtype)).cuda(), torch.tensor([0, 1, 2, 3, 5, 6, 7, 8, 10])
    y = torch.full_like(x, 7.0)
    xp.xpipe_rmsnorm_fwd(x, w, y, eps=1e-30)
    _, want = _norm64(_d(x)[keep], _d(w), 1e-30)
    _close(_d(y)[keep], want, 8 * E24 * want.abs() * (1 + u) + u * want.abs(), "y")
    assert bool(y[3].eq(0).all()) and bool(y[4].isnan().all()) and bool(y[9, dim - 1].isnan())
    dy = torch.randn(11, dim, generator=g).to(_dt(dtype)).cuda()
    _check_norm_backward(dy[keep.cuda()], x[keep.cuda()], w, 1e-10, dtype)
    dx = torch.full_like(x, 7.0)
    xp.xpipe_rmsnorm_bwd(dy, x, w, dx, None, eps=1e-10)
    assert bool(_d(dx)[keep].isfinite().all()) and bool(dx[4].isnan().all()) and bool(dx[9].isnan().any())


# ---------------------------------------------------------------- relative position bias
@pytest.mark.parametrize("buckets,heads,far,both", [(64, 5, 4097, False), (32, 3, 4097, True), (64, 64, 32768, False), (64, 2, 32768, True), (5, 1, 9999, False),
                                                    (128, 2, 1 << 17, True)])
def test_relative_bias_over_long_distances(buckets, heads, far, both):
    """grad_table: 300 additions in fp64 one after another and in halves, and as many as distances in the sum that it is held to."""
    torch = _torch()
    n = buckets // 2 if both else buckets
    half, m, one = n // 2, n - n // 2, []
    for a in range(far + 1):  # (whole numbers; a bucket's first distance is never before the last bucket's)
        k = one[-1] if one else 0
        while k + 1 < n and (a > k if k + 1 <= half else a ** m * half ** (k + 1 - half) >= far ** (k + 1 - half) * half ** m):
            k += 1
        one.append(k)
    at = torch.tensor([one[-d] if d <= 0 else one[d] + n if both else 0 for d in range(-far, far + 1)])
    g = _gen(far + buckets)
    table, dbias, grad = torch.randn(buckets, heads, generator=g), torch.randn(heads, 2 * far + 1, generator=g), torch.randn(buckets, heads, generator=g)
    bias, got = torch.full((heads, 2 * far + 1), 7.0, device="cuda"), grad.cuda()
    xp.xpipe_relbias_fwd(table.cuda(), bias, bidirectional=both)
    assert torch.equal(bias.cpu(), table[at].t())
    xp.xpipe_relbias_bwd(dbias.cuda(), got, bidirectional=both)
    want = grad.double().index_add(0, at, dbias.t().double())
    size = grad.double().abs().index_add(0, at, dbias.t().double().abs())
    _close(got, want, E24 * want.abs() + (2 * far + 300) * 2.0 ** -53 * size, "grad_table")


# ---------------------------------------------------------------- attention: capped scores
def _scores(q, cap, **more):
    """The scores of rows q [n] of one column with one key of 1, as the statistics hold them: their log2(e) multiples."""
    torch = _torch()
    n = q.numel()
    q4, one = q.view(1, n, 1, 1), torch.ones(1, 1, 1, 1, dtype=q.dtype, device="cuda")
    stats = torch.full((1, 1, n, 2), 7.0, device="cuda")
    xp.xpipe_attention_fwd(q4, one, one, torch.empty_like(q4), scale=1.0, cap=cap, stats=stats, **more)
    assert bool(stats[..., 1].eq(1).all())
    return stats[0, 0, :, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [40, 400])
@pytest.mark.parametrize("cap", [0.5, 30.0, 1e4, 1e8, 1e30])
def test_capped_scores_to_their_own_size(cap, rows, dtype):
    """Every score within 26 * 2^-24 of itself, whatever the cap; in bf16 storage up to a cap of 64, 12 * 2^-24 of the cap.
    Below half the cap, 1 each for scale log2(e), the product, the polynomial's last step and its multiple, 1 for the
    rest of it.  Beyond, for q = 1 / (1 + exp(2 x)): 4 * 2^-24 of x, which moves q by 0.9 * 2^-24 at most, 0.5 for the exponential's step,
    1 for the sum, 2 for the reciprocal; 1 - 2 q doubles that, and 1 for its rounding, 2 for cap log2(e): 12 of the cap, whose
    0.46th part the score is at least."""
    torch = _torch()
    g = _gen(int(math.log2(cap)) + rows)
    q = cap * torch.exp2(torch.rand(rows, generator=g) * 17 - 12) * torch.sign(torch.randn(rows, generator=g))
    if cap > 100:
        q[::2] = torch.randn(rows // 2, generator=g) * 5  # scores of ordinary size under a cap that never binds
    q = q.to(_dt(dtype)).cuda()
    want = cap * torch.tanh(_d(q) / cap) / math.log(2)
    tol = 12 * E24 * cap / math.log(2) if dtype == "bf16" and cap <= 64 else 26 * E24 * want.abs()
    _close(_scores(q, cap), want, tol, "scores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_capped_scores_do_not_depend_on_their_neighbours(dtype):
    torch = _torch()
    for rows in (40, 400):
        q = (torch.randn(rows, generator=_gen(rows)) * 2).to(_dt(dtype)).cuda()
        other = q.clone()
        other[1::3] = 300.0
        a, b = _scores(q, 50.0), _scores(other, 50.0)
        keep = torch.arange(rows) % 3 != 1
        assert torch.equal(a.cpu()[keep], b.cpu()[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reach", [0, 20])
@pytest.mark.parametrize("shape", [(2, 100, 130, 2, 1, 64), (1, 3, 400, 4, 2, 128), (1, 90, 70, 2, 2, 128)])
def test_a_cap_that_never_binds(shape, reach, dtype):
    """Under a cap of 1e6 scores below 50 are themselves to 1e-9: results and gradients within the bounds of no cap."""
    Case(*shape, dtype, mask="causal", reach=reach).check(cap=1e6)


# ---------------------------------------------------------------- attention: documents
def test_attention_of_documents_of_nothing():
    """Queries with documents over no keys, and keys with documents and no queries: zeros, in every result."""
    torch = _torch()
    full = lambda *s: torch.full(s, 7.0, device="cuda")
    docs = lambda n: torch.zeros(2, n, dtype=torch.int32, device="cuda")
    for nq, nk in ((5, 0), (200, 0), (0, 5)):
        q, kv, o, st, bias = full(2, nq, 2, 8), full(2, nk, 1, 8), full(2, nq, 2, 8), full(2, 2, nq, 2), torch.ones(2, 9, device="cuda")
        how = dict(q_doc=docs(nq), k_doc=docs(nk), bias=bias, causal=True)
        xp.xpipe_attention_fwd(q, kv, kv, o, stats=st, **how)
        assert bool(o.eq(0).all()) and bool(st[..., 0].eq(-math.inf).all()) and bool(st[..., 1].eq(0).all())
        dq, dk, dv, gb = full(2, nq, 2, 8), full(2, nk, 1, 8), full(2, nk, 1, 8), torch.ones(2, 9, device="cuda")
        xp.xpipe_attention_bwd(full(2, nq, 2, 8), q, kv, kv, o, st, dq, dk, dv, gb, **how)
        assert bool(dq.eq(0).all()) and bool(dk.eq(0).all()) and bool(dv.eq(0).all()) and bool(gb.eq(1).all())


# ---------------------------------------------------------------- attention: results that meet in memory
@pytest.mark.parametrize("docs", [False, True])
def test_far_distances_of_heads_that_share_keys(docs):
    """Bias gradients that are almost all beyond the range: sums that a wave clears first and writes at each head's end."""
    torch = _torch()
    c = Case(2, 300, 300, 8, 2, 64, "f32", mask="causal", reach=1, docs=docs)
    c.check()
    o, stats = c.forward()
    first = c.backward(o, stats)[3]
    assert all(torch.equal(first, c.backward(o, stats)[3]) for _ in range(5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("docs", [False, True])
def test_few_queries_over_steps_of_one_wave(docs, dtype):
    """19 steps of the keys through a wave's own LDS, in as many waves as sequences and heads: within the bounds, and the same bits each time."""
    torch = _torch()
    c = Case(4, 1, 600, 512, 512, 8, dtype, mask="causal", ragged=True, docs=docs)
    c.check(train=False)
    first = c.forward()[0]
    assert all(torch.equal(first, c.forward()[0]) for _ in range(5))


# ---------------------------------------------------------------- attention: bits of P
def _as_f32(c):
    """The same call's values in fp32 storage: its bounds leave no room for rounded operands."""
    torch = _torch()
    d = Case.__new__(Case)
    d.__dict__.update(c.__dict__, dtype="f32", **{n: getattr(c, n).float() for n in ("q", "k", "v", "do")})
    return d


@pytest.mark.parametrize("cap,reach", [(0.0, 0), (20.0, 30)])
@pytest.mark.parametrize("shape", [(2, 1, 3000, 8, 2, 128), (1, 4, 900, 8, 1, 64), (40, 1, 200, 64, 64, 96), (3, 1, 40, 4, 4, 33)])
def test_few_queries_keep_16_bits_of_p(shape, cap, reach):
    """bf16 storage: within the bounds of fp32 products, o's own rounding, and 2^-16 of P (two bf16 values, the second
    of what the first leaves)."""
    c = Case(*shape, "bf16", mask="causal", cap=cap, reach=reach, ragged=True)
    o, tol = _as_f32(c).exact()["o"]
    size = _as_f32(c)
    size.v = size.v.abs()
    tol = tol + 2.0 ** -16 * size.exact()["o"][0]
    _close(c.forward()[0].permute(0, 2, 1, 3), o, tol + 2.0 ** -8 * (o.abs() + tol), "o")


# ---------------------------------------------------------------- attention: far apart in memory
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
def test_attention_long_offsets_in_training(odd, dtype):
    """Rows of every input and output more than 2^31 elements apart give the bits of neighbours (odd: rows that are copied first)."""
    torch = _torch()
    n, H, D, stride = 1040, 2, 64, (1 << 21) + odd
    buf = torch.empty(n * stride, dtype=_dt(dtype), device="cuda")
    far = lambda slot: buf.as_strided((1, n, H, D), (0, stride, D, 1), slot * 1024)
    g = _gen(3 + odd)
    near = [torch.randn(1, n, H, D, generator=g).to(_dt(dtype)).cuda() for _ in range(4)]
    bias = torch.randn(H, 41, generator=g).cuda()
    how = dict(causal=True, bias=bias)

    def both(q, k, v, do, o, dq, dk, dv):
        stats, gb = torch.empty(1, H, n, 2, device="cuda"), torch.zeros_like(bias)
        xp.xpipe_attention_fwd(q, k, v, o, stats=stats, **how)
        xp.xpipe_attention_bwd(do, q, k, v, o, stats, dq, dk, dv, gb, **how)
        return [o, dq, dk, dv, stats, gb]
    want = both(*near, *[torch.empty_like(near[0]) for _ in range(4)])
    places = [far(i) for i in range(8)]
    for to, t in zip(places, near):
        to.copy_(t)
    got = both(*places)
    for a, b, name in zip(want, got, ("o", "dq", "dk", "dv", "stats", "grad_bias")):
        assert torch.equal(a, b), name
