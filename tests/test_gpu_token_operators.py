"""GPU parity of the operators of token networks (RMS norm with the skip
connection, relative position bias by buckets, attention with its masks, cap and
bias, and their gradients) with their formulas in 64 bits, element by element.

Bounds.  u = 2^-8 (bf16) or 2^-24 (fp32) is half a step of the stored type.  A
sum of K fp32 products is off by at most (K + 2) 2^-23 times the sum of their
magnitudes (2^-23 and not 2^-24 per addition: the matrix unit may truncate).

Norm: sums over a row are fp64, n is rounded to fp32 once, the rest are at most
four fp32 operations: 6 * 2^-24 of the terms' magnitudes.

Attention, for a query i: a score s is off by at most
  E = (D + 2) 2^-23 scale sum |q||k|  +  4 * 2^-24 (|s| + max |s|)  +  cap 2^-22 (with a cap)
(the products, roundings of scale, cap, bias and the exponent's argument, the tanh), so P by
a factor within 1 +- eps, eps = expm1(2 max E) + (n + 8) 2^-23, and bf16 operands of the second
products round P and dX by uP = 2^-8 more (fp32: 0).  The rest is the formulas'
own propagation, written out in Case.exact.  A P, dS or dX below 2^-126, the least normal
fp32 value, may be flushed to zero (scores far below a row's largest): 2^-125 = TINY for each
of them, whatever its relative error."""
import math

import pytest

import paper_1911_04610_amd as xp

pytestmark = pytest.mark.gpu
E24, E23, TINY = 2.0 ** -24, 2.0 ** -23, 2.0 ** -125


def _torch():
    import torch
    return torch


def _dt(name):
    torch = _torch()
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _half_step(name):
    return {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[name]


def _gen(seed):
    g = _torch().Generator()
    g.manual_seed(seed)
    return g


def _d(t):
    return t.detach().cpu().double()


def _close(got, want, tol, what):
    got = _d(got)
    off = (got - want).abs()
    assert bool((off <= tol).all()), f"{what}: {float((off - tol).max()):.3e} over its bound, at {int((off - tol).argmax())}"


def _wide(g, shape, dtype, pitch=0, scale=1.0, offset=0):
    """A tensor of that shape on the GPU, its last dimension pitch elements longer in memory, starting offset into it."""
    torch = _torch()
    buf = torch.randn(*shape[:-1], shape[-1] + pitch, generator=g) * scale
    return buf.to(_dt(dtype)).cuda()[..., offset:offset + shape[-1]]


# ---------------------------------------------------------------- RMS norm
NORM = [(1, 1), (1, 4096), (3, 7), (5, 8), (64, 64), (17, 65), (9, 512), (33, 513), (7, 1000), (130, 1024), (4, 2047), (2049, 40),
        (3, 4096), (600, 4099), (2, 8192), (3, 8200), (2, 16384), (2, 32768), (2500, 520)]


def _norm64(h, w, eps):
    n = 1 / (h.square().mean(1, keepdim=True) + eps).sqrt()
    return n, h * n * w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", NORM)
def test_norm_forward(rows, dim, dtype):
    torch = _torch()
    g, u = _gen(rows * 7 + dim), _half_step(dtype)
    for k in range(3):
        pitch = (0, 3, 8)[k]
        x, r = _wide(g, (rows, dim), dtype, pitch), _wide(g, (rows, dim), dtype, pitch, 3.0, offset=min(pitch, 1)) if k != 1 else None
        w = (1 + 0.1 * torch.randn(dim, generator=g)).cuda()
        y, h = torch.full_like(x, 7.0), torch.full_like(x, 7.0) if k != 2 else None
        xp.xpipe_rmsnorm_fwd(x, w, y, eps=1e-5, residual=r, sum=h)
        h64 = _d(x) + (_d(r) if r is not None else 0)
        dh = E24 * h64.abs()  # the fp32 sum of two
        if h is not None:
            _close(h, h64, u * (h64.abs() + dh) + dh, "sum")
        n, y64 = _norm64(h64, _d(w), 1e-5)
        tol = 8 * E24 * y64.abs()  # h's rounding twice (itself, and in n), n, two products
        _close(y, y64, u * (y64.abs() + tol) + tol, "y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", NORM)
def test_norm_backward(rows, dim, dtype):
    torch = _torch()
    g, u = _gen(rows * 5 + dim), _half_step(dtype)
    for k in range(3):
        pitch = (0, 5, 8)[k]
        dy, h = _wide(g, (rows, dim), dtype, pitch, 0.1), _wide(g, (rows, dim), dtype, pitch, 2.0, offset=min(pitch, 2))
        r = _wide(g, (rows, dim), dtype, pitch, 0.1) if k != 1 else None
        w, gw = (1 + 0.1 * torch.randn(dim, generator=g)).cuda(), torch.randn(dim, generator=g).cuda()
        before = _d(gw)
        dx = torch.full_like(dy, 7.0) if k != 2 else None
        xp.xpipe_rmsnorm_bwd(dy, h, w, dx, gw, eps=1e-5, residual=r)
        h64, g64 = _d(h), _d(dy) * _d(w)
        n, _ = _norm64(h64, _d(w), 1e-5)
        c = n * n * (g64 * h64).mean(1, keepdim=True)
        mag_c = n * n * (g64 * h64).abs().mean(1, keepdim=True)  # dy w is rounded before it is summed
        if dx is not None:
            want = n * (g64 - h64 * c) + (_d(r) if r is not None else 0)
            tol = 6 * E24 * n * (g64.abs() + h64.abs() * (c.abs() + mag_c)) + 2 * E24 * want.abs()
            _close(dx, want, u * (want.abs() + tol) + tol, "dx")
        terms = _d(dy) * h64 * n
        _close(gw, before + terms.sum(0), (rows / 256 + 16) * E24 * terms.abs().sum(0) + 4 * E24 * terms.abs().sum(0) + 2 * E24 * before.abs(), "grad_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_in_place(dtype):
    """y, sum and dx in their inputs' buffers give the bits of separate ones."""
    torch = _torch()
    for rows, dim in ((5, 48), (20, 1000), (3, 6000), (2, 20000)):
        g = _gen(dim)
        x, r, w = _wide(g, (rows, dim), dtype), _wide(g, (rows, dim), dtype), torch.randn(dim, generator=g).cuda()
        y, h = torch.empty_like(x), torch.empty_like(x)
        xp.xpipe_rmsnorm_fwd(x, w, y, residual=r, sum=h)
        for ys, hs in (("x", "r"), ("r", "x"), ("x", None), (None, "x"), (None, "r")):
            b = {"x": x.clone(), "r": r.clone(), None: torch.empty_like(x)}
            other = torch.empty_like(x)
            y2, h2 = b[ys], b[hs] if hs is not None or ys is not None else other
            if y2 is h2:
                h2 = other
            xp.xpipe_rmsnorm_fwd(b["x"], w, y2, residual=b["r"], sum=h2)
            assert torch.equal(y2, y) and torch.equal(h2, h), (ys, hs)
        dx, gw = torch.empty_like(x), torch.zeros(dim, device="cuda")
        xp.xpipe_rmsnorm_bwd(x, h, w, dx, gw, residual=r)
        for k in range(3):
            t, gw2 = [x.clone(), h.clone(), r.clone()], torch.zeros(dim, device="cuda")
            xp.xpipe_rmsnorm_bwd(t[0], t[1], w, t[k], gw2, residual=t[2])
            assert torch.equal(t[k], dx) and torch.equal(gw2, gw), k


def test_norm_extremes():
    """Rows whose squares leave fp32, zero rows, and values that are not finite, which stay in their row."""
    torch = _torch()
    w = torch.ones(300, device="cuda")
    x = torch.randn(6, 300, generator=_gen(1)).cuda()
    x[1] *= 1e25
    x[2] *= 1e-30
    x[3] = 0
    x[4, 7] = math.nan
    x[5, 9] = math.inf
    y, dx, gw = torch.empty_like(x), torch.empty_like(x), torch.zeros(300, device="cuda")
    xp.xpipe_rmsnorm_fwd(x, w, y, eps=1e-6)
    _, want = _norm64(_d(x)[:4], _d(w), 1e-6)
    _close(y[:4], want, 8 * E24 * want.abs() + 1e-45, "y")
    assert bool(y[3].eq(0).all()) and bool(y[4].isnan().all()) and bool(y[5, 9].isnan())
    dy = torch.randn(6, 300, generator=_gen(2)).cuda()
    xp.xpipe_rmsnorm_bwd(dy, x, w, dx, gw, eps=1e-6)
    assert bool(dx[:4].isfinite().all()) and bool(dx[4].isnan().all()) and bool(gw.isnan().all())
    _close(dx[3], 1e3 * _d(dy[3]), 4 * E24 * 1e3 * _d(dy[3]).abs(), "dx of a zero row")


def test_norm_of_nothing_and_padding_columns():
    torch = _torch()
    w, e = torch.ones(5, device="cuda"), torch.empty(0, 5, device="cuda")
    gw = torch.ones(5, device="cuda")
    xp.xpipe_rmsnorm_fwd(e, w, e.clone())
    xp.xpipe_rmsnorm_bwd(e, e, w, e.clone(), gw)
    assert bool(gw.eq(1).all())
    buf = torch.full((9, 40), 3.0, device="cuda")
    y = buf[:, 4:37]
    x = torch.randn(9, 33, generator=_gen(3)).cuda()
    xp.xpipe_rmsnorm_fwd(x, torch.ones(33, device="cuda"), y)
    assert bool(buf[:, :4].eq(3).all()) and bool(buf[:, 37:].eq(3).all()) and not bool(y.eq(3).any())


# ---------------------------------------------------------------- relative position bias
def _bucket(away, n, far):
    """In whole numbers: the last bucket whose first distance is not beyond `away`."""
    half = n // 2
    if away < half:
        return away
    k = 0
    while half + k + 1 < n and away ** (n - half) * half ** (k + 1) >= far ** (k + 1) * half ** (n - half):
        k += 1
    return half + k


RELBIAS = [(32, 12, 128, True), (32, 1, 128, False), (4, 3, 5, True), (2, 2, 2, False), (8, 70, 64, True), (64, 5, 4096, False), (5, 4, 333, False),
           (16, 33, 1000, True), (6, 2, 27, True)]


@pytest.mark.parametrize("buckets,heads,far,both", RELBIAS)
def test_relative_bias(buckets, heads, far, both):
    torch = _torch()
    n = buckets // 2 if both else buckets
    one = [_bucket(a, n, far) for a in range(far + 1)]
    at = torch.tensor([one[-d] if d <= 0 else one[d] + n if both else 0 for d in range(-far, far + 1)])
    g = _gen(far)
    table, dbias, grad = torch.randn(buckets, heads, generator=g), torch.randn(heads, 2 * far + 1, generator=g), torch.randn(buckets, heads, generator=g)
    bias, got = torch.full((heads, 2 * far + 1), 7.0, device="cuda"), grad.cuda()
    xp.xpipe_relbias_fwd(table.cuda(), bias, bidirectional=both)
    assert torch.equal(bias.cpu(), table[at].t())
    xp.xpipe_relbias_bwd(dbias.cuda(), got, bidirectional=both)
    want = grad.double().index_add(0, at, dbias.t().double())
    _close(got, want, E24 * want.abs() + 2.0 ** -40, "grad_table")


# ---------------------------------------------------------------- attention
class Case:
    """Inputs of one call on the GPU, and which pairs its masks leave (in 64 bits on the CPU)."""

    def __init__(self, batch, nq, nk, heads, kv_heads, dim, dtype, mask="none", cap=0.0, reach=0, ragged=False, docs=False, pitch=0, seed=0,
                 scale=None, spread=1.0, layout="bthd", prefix=None, lens=None):
        torch = _torch()
        g = _gen(seed + nq * 3 + nk * 5 + dim)
        self.dtype, self.cap, self.mask, self.reach = dtype, cap, mask, reach
        self.sizes = (batch, nq, nk, heads, kv_heads, dim)

        def make(n, h):
            if layout == "bhtd":
                return _wide(g, (batch, h, n, dim), dtype, pitch, spread).transpose(1, 2)
            if layout == "packed":  # q, k and v of one projection side by side
                return _wide(g, (batch, n, 3 * h, dim), dtype, pitch, spread)[:, :, h:2 * h]
            return _wide(g, (batch, n, h, dim), dtype, pitch, spread)
        self.q, self.k, self.v, self.do = make(nq, heads), make(nk, kv_heads), make(nk, kv_heads), make(nq, heads)
        self.bias = torch.randn(heads, 2 * reach + 1, generator=g).cuda() if reach else None
        r = lambda lo, hi: torch.randint(lo, hi + 1, (batch,), generator=g, dtype=torch.int32)
        self.k_len, self.q_len = (r(0, nk), r(0, nq)) if ragged else (None, None)
        if lens is not None:
            self.q_len, self.k_len = (torch.tensor(v, dtype=torch.int32) for v in lens)
        self.prefix = (r(0, nk) if prefix is None else torch.tensor(prefix, dtype=torch.int32)) if mask == "prefix" else None
        self.q_doc = self.k_doc = None
        if docs:
            top = max(1, nk // 40)
            self.k_doc = torch.randint(-1, top + 1, (batch, nk), generator=g).sort(1).values.to(torch.int32)
            self.q_doc = torch.randint(-1, top + 1, (batch, nq), generator=g).sort(1).values.to(torch.int32)
            if docs == "any":  # in no order, and of any size
                self.k_doc, self.q_doc = (t[:, torch.randperm(t.shape[1], generator=g)] * 1000003 for t in (self.k_doc, self.q_doc))
            if nq == nk:
                self.q_doc = self.k_doc.clone()
        self.scale = dim ** -0.5 if scale is None else scale
        ql = self.q_len if self.q_len is not None else torch.full((batch,), nq)
        kl = self.k_len if self.k_len is not None else torch.full((batch,), nk)
        self.off = (kl - ql).long()
        i, j = torch.arange(nq)[None, :, None], torch.arange(nk)[None, None, :]
        see = (i < ql[:, None, None]) & (j < kl[:, None, None])
        self.distance = j - (i + self.off[:, None, None])
        if mask != "none":
            past = self.distance <= 0
            if mask == "prefix":
                past = past | (j < self.prefix[:, None, None])
            see = see & past
        if docs:
            see = see & (self.q_doc[:, :, None] == self.k_doc[:, None, :]) & (self.k_doc[:, None, :] >= 0)
        self.see = see[:, None]

    def how(self):
        c = lambda t: None if t is None else t.cuda()
        return dict(scale=self.scale, causal=self.mask != "none", cap=self.cap, bias=self.bias, q_len=c(self.q_len), k_len=c(self.k_len),
                    prefix=c(self.prefix), q_doc=c(self.q_doc), k_doc=c(self.k_doc))

    def forward(self, **more):
        torch = _torch()
        B, nq, nk, H, K, D = self.sizes
        o = torch.full((B, nq, H, D), 7.0, dtype=_dt(self.dtype), device="cuda")
        stats = torch.full((B, H, nq, 2), 7.0, device="cuda")
        xp.xpipe_attention_fwd(self.q, self.k, self.v, o, stats=stats, **dict(self.how(), **more))
        return o, stats

    def backward(self, o, stats, bias=True, **more):
        torch = _torch()
        B, nq, nk, H, K, D = self.sizes
        new = lambda n, h: torch.full((B, n, h, D), 7.0, dtype=_dt(self.dtype), device="cuda")
        dq, dk, dv = new(nq, H), new(nk, K), new(nk, K)
        gb = torch.zeros(H, 2 * self.reach + 1, device="cuda") if self.reach and bias else None
        xp.xpipe_attention_bwd(self.do, self.q, self.k, self.v, o, stats, dq, dk, dv, gb, **dict(self.how(), **more))
        return dq, dk, dv, gb

    def exact(self):
        """Everything in 64 bits, and the bounds."""
        torch = _torch()
        B, nq, nk, H, K, D = self.sizes
        u, uP = _half_step(self.dtype), 2.0 ** -8 if self.dtype == "bf16" else 0.0
        heads = lambda t: _d(t).permute(0, 2, 1, 3)
        q, do = heads(self.q), heads(self.do)
        k, v = heads(self.k).repeat_interleave(H // K, 1), heads(self.v).repeat_interleave(H // K, 1)
        kt, vt = k.transpose(2, 3).contiguous(), v.transpose(2, 3).contiguous()
        x = self.scale * (q @ kt)
        ex = (D + 2) * E23 * self.scale * (q.abs() @ kt.abs()) + 2 * E24 * x.abs()
        slope, eslope, s, E = torch.ones_like(x), torch.zeros_like(x), x, ex
        if self.cap:
            t = torch.tanh(x / self.cap)
            s, slope = self.cap * t, 1 - t * t
            E = ex + self.cap * 4 * E24
            eslope = 0.77 * ex / self.cap + 16 * E24
        at = (self.distance.clamp(-self.reach, self.reach) + self.reach)[:, None] if self.reach else None
        if self.reach:
            b64 = _d(self.bias)
            s = s + torch.stack([b64[:, at[n, 0]] for n in range(B)])
        s = s.masked_fill(~self.see, -math.inf)
        top = s.amax(3, keepdim=True) if nk else torch.full((B, H, nq, 1), -math.inf, dtype=torch.float64)
        base = torch.where(top == -math.inf, 0.0, top)
        size = torch.where(s == -math.inf, 0.0, s).abs()
        E = torch.where(s == -math.inf, 0.0, E + 4 * E24 * (size + (size.amax(3, keepdim=True) if nk else 0)))
        p = torch.exp(s - base)
        total = p.sum(3, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        eps = torch.expm1(2 * (E.amax(3, keepdim=True) if nk else torch.zeros(B, H, nq, 1))) + (nk + 8) * E23
        out = {}
        o, mag = p @ v, p @ v.abs()
        eo = (eps + uP * (1 + eps) + (nk + 2) * E23) * mag + TINY * v.abs().sum(2, keepdim=True)
        eo = eo + u * (o.abs() + eo)
        out["o"] = (o, eo)
        out["m"], out["l"] = (top, base, eps), total
        dp = do @ vt
        edp = (D + 2) * E23 * (do.abs() @ vt.abs())
        delta = (do * o).sum(3, keepdim=True)
        edelta = (p * (eps * dp.abs() + (1 + eps) * edp) + TINY * dp.abs()).sum(3, keepdim=True) + (nk + 2) * E23 * (p * dp.abs()).sum(3, keepdim=True)
        estored = (do.abs() * eo).sum(3, keepdim=True) + (D + 2) * E23 * (do * o).abs().sum(3, keepdim=True)
        eps = 2 * eps  # (the backward's P: statistics that were rounded, scores made again)
        ds = p * (dp - delta)
        err = lambda ed: (eps + 2 * E23) * ds.abs() + (1 + eps) * p * (edp + ed) + (E23 * p + TINY) * (dp.abs() + delta.abs()) + TINY
        edq, eds = err(estored), err(edelta)
        def side(ed):  # of dX / scale
            e = ed * slope + (ds.abs() + ed) * eslope + 2 * E24 * ds.abs() * slope + TINY
            return e + uP * ((ds * slope).abs() + e)
        dx = ds * slope
        shared = lambda t: t.reshape(B, K, H // K, nk, D).sum(2)
        def back(name, value, tol, perm=True):
            tol = tol + 2 * E24 * value.abs()
            tol = tol + u * (value.abs() + tol)
            out[name] = (value, tol)
        sc = self.scale
        back("dq", sc * (dx @ k), sc * (side(edq) @ k.abs() + (nk + 2) * E23 * (dx.abs() + side(edq)) @ k.abs()))
        dxt, et = dx.transpose(2, 3).contiguous(), side(eds).transpose(2, 3).contiguous()
        n = (nq * (H // K) + 2) * E23
        back("dk", sc * shared(dxt @ q), sc * shared((et + n * (dxt.abs() + et)) @ q.abs()))
        pt, ept = p.transpose(2, 3).contiguous(), ((eps + uP * (1 + eps)) * p + TINY).transpose(2, 3).contiguous()
        back("dv", shared(pt @ do), shared((ept + n * (pt + ept)) @ do.abs()))
        if self.reach:
            val, tol = torch.zeros(H, 2 * self.reach + 1, dtype=torch.float64), torch.zeros(H, 2 * self.reach + 1, dtype=torch.float64)
            count = 64 + 32 + nk / 32 * nq / 32  # additions that one term goes through in fp32, at most
            for b in range(B):
                ix = at[b, 0].reshape(-1)
                val.index_add_(1, ix, ds[b].reshape(H, -1))
                tol.index_add_(1, ix, (eds + count * E24 * ds.abs())[b].reshape(H, -1))
            out["gb"] = (val, tol + 2 * E24 * val.abs())
        return out

    def check(self, train=True, **more):
        torch = _torch()
        want = self.exact()
        o, stats = self.forward(**more)
        value, tol = want["o"]
        _close(o.permute(0, 2, 1, 3), value, tol, "o")
        seen = want["l"][..., 0] > 0
        m, l = _d(stats[..., 0]) * math.log(2), _d(stats[..., 1])
        assert torch.equal(l > 0, seen) and bool((m[~seen] == -math.inf).all()) and bool((o.permute(0, 2, 1, 3).cpu()[~seen] == 0).all())
        top, base, eps = want["m"]
        lse = (top[..., 0] + want["l"][..., 0].log())[seen]  # (m is one score's value or a rounding away from it)
        _close((m + l.log())[seen], lse, eps[..., 0].expand_as(seen)[seen] + 8 * E24 * (1 + lse.abs()), "stats")
        if not train:
            return
        dq, dk, dv, gb = self.backward(o, stats, **more)
        for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
            _close(got.permute(0, 2, 1, 3), *want[name], name)
        if gb is not None:
            _close(gb, *want["gb"], "grad_bias")


SHAPES = [  # batch, nq, nk, heads, kv_heads, dim
    (1, 1, 1, 1, 1, 1), (2, 1, 5, 2, 1, 64), (1, 3, 33, 4, 4, 8), (2, 31, 64, 2, 2, 33), (1, 65, 65, 6, 2, 128), (3, 77, 77, 4, 1, 40),
    (1, 128, 130, 2, 2, 64), (2, 200, 333, 3, 3, 72), (1, 300, 301, 4, 2, 128), (1, 513, 200, 1, 1, 96), (2, 130, 40, 2, 2, 16),
    (1, 150, 150, 2, 1, 97), (1, 70, 190, 2, 2, 65),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["none", "causal", "prefix"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, mask, dtype):
    Case(*shape, dtype, mask=mask).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask,ragged,docs", [("none", True, False), ("causal", True, False), ("prefix", True, False), ("none", False, True),
                                              ("causal", False, True), ("causal", True, True), ("none", True, "any"), ("prefix", True, True)])
@pytest.mark.parametrize("shape", [(3, 77, 77, 2, 1, 40), (2, 200, 333, 2, 2, 64), (2, 300, 300, 4, 2, 128), (4, 5, 150, 4, 2, 128)])
def test_attention_masks(shape, mask, ragged, docs, dtype):
    Case(*shape, dtype, mask=mask, ragged=ragged, docs=docs).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap,reach,mask,docs", [(2.0, 0, "none", False), (30.0, 0, "causal", False), (0.0, 1, "none", False), (0.0, 32, "none", False),
                                                 (0.0, 500, "causal", False), (5.0, 40, "prefix", False), (0.0, 100, "causal", True), (1.0, 17, "none", "any")])
@pytest.mark.parametrize("shape", [(3, 77, 77, 2, 1, 40), (2, 200, 333, 2, 2, 64), (2, 300, 301, 4, 2, 128), (2, 333, 100, 2, 1, 64)])
def test_attention_cap_and_bias(shape, cap, reach, mask, docs, dtype):
    Case(*shape, dtype, mask=mask, cap=cap, reach=reach, docs=docs, ragged=docs is False and reach == 32, spread=2.0).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 3000, 4, 2, 128), (3, 1, 1000, 8, 1, 64), (2, 4, 2000, 2, 2, 40), (1, 20, 1500, 8, 2, 128), (2, 1, 257, 1, 1, 128),
                                   (70, 1, 300, 2, 1, 64), (1, 16, 700, 8, 2, 96), (300, 2, 90, 2, 1, 16), (5, 1, 33, 3, 1, 128)])
def test_attention_few_queries(shape, dtype):
    """Few rows over many keys: rows of heads that share keys together, the keys in parts."""
    Case(*shape, dtype, mask="causal").check(train=False)
    Case(*shape, dtype, mask="causal", ragged=True, cap=10.0, reach=64, seed=1).check(train=False)
    Case(*shape, dtype, mask="none", docs=True, seed=2).check(train=False)
    Case(*shape, dtype, mask="causal", seed=3).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask,docs,cap,reach", [("causal", False, 0.0, 0), ("prefix", False, 20.0, 40), ("none", True, 0.0, 0)])
@pytest.mark.parametrize("shape", [(1, 90, 2100, 2, 1, 33), (1, 140, 2300, 1, 1, 96), (2, 30, 2081, 2, 2, 128), (1, 2080, 300, 2, 1, 64)])
def test_attention_many_keys(shape, mask, docs, cap, reach, dtype):
    Case(*shape, dtype, mask=mask, docs=docs, cap=cap, reach=reach, ragged=not docs).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,pitch", [("bhtd", 0), ("bhtd", 3), ("packed", 0), ("packed", 1), ("bthd", 1), ("bthd", 7), ("bthd", 8)])
def test_attention_layouts(layout, pitch, dtype):
    Case(2, 90, 130, 4, 2, 64, dtype, mask="causal", layout=layout, pitch=pitch).check()
    Case(1, 70, 70, 2, 2, 50, dtype, mask="none", layout=layout, pitch=pitch, reach=16).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_lengths(dtype):
    """Sequences of no, one and all keys and queries, and lengths beyond the tensors."""
    lens = ([0, 70, 70, 1, 70, 64, 99, -3], [70, 0, 1, 70, 70, 65, 99, 70])
    for mask in ("none", "causal", "prefix"):
        c = Case(8, 70, 70, 2, 1, 64, dtype, mask=mask, lens=([min(max(n, 0), 70) for n in lens[0]], [min(max(n, 0), 70) for n in lens[1]]),
                 prefix=[0, 3, 70, 1, 33, 64, 5, 9] if mask == "prefix" else None)
        torch = _torch()
        given = {"q_len": torch.tensor(lens[0], dtype=torch.int32).cuda(), "k_len": torch.tensor(lens[1], dtype=torch.int32).cuda()}
        c.check(**given)


def test_attention_of_nothing():
    torch = _torch()
    e = lambda *s: torch.full(s, 7.0, device="cuda")
    o, st = e(2, 5, 2, 8), e(2, 2, 5, 2)
    xp.xpipe_attention_fwd(e(2, 5, 2, 8), e(2, 0, 1, 8), e(2, 0, 1, 8), o, stats=st)
    assert bool(o.eq(0).all()) and bool(st[..., 0].eq(-math.inf).all()) and bool(st[..., 1].eq(0).all())
    dq = e(2, 5, 2, 8)
    xp.xpipe_attention_bwd(e(2, 5, 2, 8), e(2, 5, 2, 8), e(2, 0, 1, 8), e(2, 0, 1, 8), o, st, dq, e(2, 0, 1, 8), e(2, 0, 1, 8))
    assert bool(dq.eq(0).all())
    dk, dv = e(2, 5, 1, 8), e(2, 5, 1, 8)
    none = e(2, 0, 2, 8)
    xp.xpipe_attention_fwd(none, e(2, 5, 1, 8), e(2, 5, 1, 8), none.clone(), stats=e(2, 2, 0, 2))
    gb = torch.ones(2, 9, device="cuda")
    xp.xpipe_attention_bwd(none, none, e(2, 5, 1, 8), e(2, 5, 1, 8), none, e(2, 2, 0, 2), none.clone(), dk, dv, gb, bias=torch.ones(2, 9, device="cuda"))
    assert bool(dk.eq(0).all()) and bool(dv.eq(0).all()) and bool(gb.eq(1).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("few", [False, True])
def test_attention_padding_is_not_used(dtype, few):
    """NaN and infinities behind the lengths and in padding documents reach nothing."""
    torch = _torch()
    shape = (3, 4, 500, 4, 2, 64) if few else (3, 150, 150, 4, 2, 64)
    for docs in (False, True):
        c = Case(*shape, dtype, mask="causal", ragged=not docs, docs=docs, reach=20)
        clean = c.forward()
        grads = c.backward(*clean)
        for t, n, doc in ((c.q, c.q_len, c.q_doc), (c.do, c.q_len, c.q_doc), (c.k, c.k_len, c.k_doc), (c.v, c.k_len, c.k_doc)):
            for b in range(shape[0]):
                if docs:
                    t[b, (doc[b] < 0).cuda()] = math.nan
                else:
                    t[b, int(n[b]):] = math.inf if b else math.nan
        dirty = c.forward()
        assert all(torch.equal(x, y) for x, y in zip(clean, dirty))
        again = c.backward(*dirty)
        assert all(torch.equal(x, y) for x, y in zip(grads, again))


def test_attention_bias_that_masks():
    """-inf in the bias masks; the lowest value in every place of a row leaves the softmax of equal scores."""
    torch = _torch()
    for dtype in ("bf16", "f32"):
        c = Case(1, 100, 100, 2, 2, 64, dtype, reach=99)
        c.bias[:, 99 + 5:] = -math.inf  # only keys up to four ahead, and of head 1 none at all
        c.bias[1] = -math.inf
        c.check()
        low = Case(1, 70, 70, 1, 1, 64, dtype, reach=80)
        low.bias[:] = torch.finfo(torch.float32).min
        o, st = low.forward()
        mean = _d(low.v).mean(1, keepdim=True).expand_as(_d(o))
        _close(o, mean, (2 * _half_step(dtype) + 80 * E23) * _d(low.v).abs().mean(1, keepdim=True), "o")
        dv = low.backward(o, st)[2]
        want = _d(low.do).mean(1, keepdim=True).expand_as(_d(dv))
        _close(dv, want, (2 * _half_step(dtype) + 80 * E23) * _d(low.do).abs().mean(1, keepdim=True), "dv")


def test_attention_large_scores():
    """Scores in the thousands: one key takes all."""
    for dtype in ("bf16", "f32"):
        Case(1, 64, 200, 2, 1, 64, dtype, spread=30.0).check()
        Case(1, 64, 200, 2, 1, 64, dtype, spread=30.0, cap=50.0, mask="causal").check()
        Case(1, 64, 200, 2, 1, 64, dtype, spread=3.0, cap=0.5, reach=20).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_rows_stay_apart(dtype):
    """A sequence's and a head's results do not depend on the others, and repeated calls give the same bits."""
    torch = _torch()
    c = Case(3, 200, 200, 4, 2, 64, dtype, mask="causal", reach=30, ragged=True)
    o, st = c.forward()
    g = c.backward(o, st)
    o2, st2 = c.forward()
    g2 = c.backward(o2, st2)
    assert torch.equal(o, o2) and torch.equal(st, st2) and all(torch.equal(x, y) for x, y in zip(g, g2))
    one = lambda t: None if t is None else t[1:2]
    how = {k: (one(v.contiguous()) if k in ("q_len", "k_len") else v) for k, v in c.how().items()}
    alone = torch.empty_like(o[1:2])
    xp.xpipe_attention_fwd(c.q[1:2], c.k[1:2], c.v[1:2], alone, **how)
    assert torch.equal(alone, o[1:2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_gradient_against_differences(dtype):
    """The directional derivative of sum(do o) along each input, by differences of the forward in 64 bits, against the gradients."""
    torch = _torch()
    c = Case(1, 40, 50, 2, 1, 32, dtype, mask="causal", cap=3.0, reach=12)
    o, st = c.forward()
    dq, dk, dv, gb = c.backward(o, st)
    base = [_d(t) for t in (c.q, c.k, c.v, c.bias)]

    def loss(q, k, v, bias):
        heads = lambda t: t.permute(0, 2, 1, 3)
        x = c.scale * (heads(q) @ heads(k).repeat_interleave(2, 1).transpose(2, 3).contiguous())
        s = c.cap * torch.tanh(x / c.cap) + bias[:, c.distance[0].clamp(-12, 12) + 12][None]
        p = torch.softmax(s.masked_fill(~c.see, -math.inf), 3)
        return float((heads(_d(c.do)) * (p @ heads(v).repeat_interleave(2, 1))).sum())
    want = c.exact()
    for n, (grad, name) in enumerate(((dq, "dq"), (dk, "dk"), (dv, "dv"), (gb, "gb"))):
        along = torch.sign(_d(grad)) * (1 + torch.rand(grad.shape, generator=_gen(n)).double())
        h = 1e-4
        moved = [[t + (s * h * along if m == n else 0) for m, t in enumerate(base)] for s in (1, -1, 2, -2)]
        f = [loss(*t) for t in moved]
        slope = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * h)  # off by h^4 of the fifth derivative: below 1e-9 here
        tol = want[name][1] if name == "gb" else want[name][1].permute(0, 2, 1, 3)
        assert abs(float((_d(grad) * along).sum()) - slope) <= float((tol * along.abs()).sum()) + 1e-6 * abs(slope), name


def test_attention_long_offsets():
    """A cache whose keys lie more than 2^31 elements apart."""
    torch = _torch()
    nk, D, stride = 1040, 64, 1 << 21
    buf = torch.zeros(nk * stride, dtype=torch.bfloat16, device="cuda")
    kv = buf.as_strided((1, nk, 2, D), (0, stride, D, 1))
    k, v = kv[:, :, :1], kv[:, :, 1:]
    g = _gen(5)
    kv.copy_(torch.randn(1, nk, 2, D, generator=g).bfloat16())
    small = kv.contiguous()
    q = torch.randn(1, 3, 2, D, generator=g).bfloat16().cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    xp.xpipe_attention_fwd(q, k, v, a, causal=True)
    xp.xpipe_attention_fwd(q, small[:, :, :1], small[:, :, 1:], b, causal=True)
    assert torch.equal(a, b)


def test_attention_other_stream_and_graph():
    """On a stream of its own, and captured and replayed beside eager calls, each replay with the eager bits."""
    torch = _torch()
    c = Case(2, 150, 150, 4, 2, 64, "bf16", mask="causal", reach=20, docs=True)
    o, st = c.forward()
    want = c.backward(o, st)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o2, st2 = torch.empty_like(o), torch.empty_like(st)
    how = c.how()
    s.wait_stream(torch.cuda.current_stream())
    xp.xpipe_attention_fwd(c.q, c.k, c.v, o2, stats=st2, stream=s, **how)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(o, o2)
    x, w = torch.randn(150, 256, generator=_gen(1)).bfloat16().cuda(), torch.ones(256, device="cuda")
    y, dx, gw = torch.empty_like(x), torch.empty_like(x), torch.zeros(256, device="cuda")
    table, grad = torch.randn(16, 4, generator=_gen(2)).cuda(), torch.zeros(16, 4, device="cuda")
    bias, gb = torch.empty(4, 41, device="cuda"), torch.zeros(4, 41, device="cuda")
    how["bias"] = bias
    dq, dk, dv = torch.empty_like(c.q), torch.empty_like(c.k), torch.empty_like(c.v)
    zeros = [gw, grad, gb]

    def step():
        for z in zeros:
            z.zero_()
        xp.xpipe_relbias_fwd(table, bias)
        xp.xpipe_rmsnorm_fwd(x, w, y)
        xp.xpipe_attention_fwd(c.q, c.k, c.v, o2, stats=st2, **how)
        xp.xpipe_attention_bwd(c.do, c.q, c.k, c.v, o2, st2, dq, dk, dv, gb, **how)
        xp.xpipe_relbias_bwd(gb, grad)
        xp.xpipe_rmsnorm_bwd(y, x, w, dx, gw)
    outs = [y, dx, gw, grad, bias, gb, o2, st2, dq, dk, dv]
    step()
    eager = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        for t in outs:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs)), n
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs)), n
    del want


def test_a_block_of_a_token_network():
    """Embedding, norm, linear (q, k, v side by side), attention with a learned bias, linear with the skip connection,
    norm, linear; forward and backward in fp32 storage against autograd in 64 bits."""
    torch = _torch()
    B, n, H, D, V, R = 2, 60, 4, 16, 50, 24
    C, g = H * D, _gen(9)
    p = {"table": torch.randn(V, C, generator=g) * 0.5, "w1": 1 + 0.1 * torch.randn(C, generator=g), "qkv": torch.randn(3 * C, C, generator=g) * C ** -0.5,
         "rel": torch.randn(16, H, generator=g), "out": torch.randn(C, C, generator=g) * C ** -0.5, "w2": 1 + 0.1 * torch.randn(C, generator=g),
         "top": torch.randn(V, C, generator=g) * C ** -0.5}
    tokens, dz = torch.randint(0, V, (B * n,), generator=g, dtype=torch.int32), torch.randn(B * n, V, generator=g)
    P = {k: t.cuda() for k, t in p.items()}
    G = {k: torch.zeros_like(t) for k, t in P.items()}
    new = lambda *s: torch.empty(*s, device="cuda")
    tok, M = tokens.cuda(), B * n
    x, a, qkv, bias, o, h, h2, y2, z = new(M, C), new(M, C), new(M, 3 * C), new(H, 2 * R + 1), new(B, n, H, D), new(M, C), new(M, C), new(M, C), new(M, V)
    stats = new(B, H, n, 2)
    xp.xpipe_embedding_fwd(P["table"], tok, x)
    xp.xpipe_rmsnorm_fwd(x, P["w1"], a)
    xp.xpipe_linear_fwd(a, P["qkv"], None, qkv)
    q, k, v = qkv.view(B, n, 3, H, D).unbind(2)
    xp.xpipe_relbias_fwd(P["rel"], bias)
    xp.xpipe_attention_fwd(q, k, v, o, causal=True, bias=bias, cap=4.0, stats=stats)
    xp.xpipe_linear_fwd(o.view(M, C), P["out"], None, h)
    xp.xpipe_rmsnorm_fwd(h, P["w2"], y2, residual=x, sum=h2)
    xp.xpipe_linear_fwd(y2, P["top"], None, z)
    dy2, dh2, do, dqkv, da, dx, gb = new(M, C), new(M, C), new(B, n, H, D), new(M, 3 * C), new(M, C), new(M, C), torch.zeros(H, 2 * R + 1, device="cuda")
    xp.xpipe_linear_bwd(dz.cuda(), y2, P["top"], dy2, G["top"])
    xp.xpipe_rmsnorm_bwd(dy2, h2, P["w2"], dh2, G["w2"])
    xp.xpipe_linear_bwd(dh2, o.view(M, C), P["out"], do.view(M, C), G["out"])
    dq, dk, dv = dqkv.view(B, n, 3, H, D).unbind(2)
    xp.xpipe_attention_bwd(do, q, k, v, o, stats, dq, dk, dv, gb, causal=True, bias=bias, cap=4.0)
    xp.xpipe_relbias_bwd(gb, G["rel"])
    xp.xpipe_linear_bwd(dqkv, a, P["qkv"], da, G["qkv"])
    xp.xpipe_rmsnorm_bwd(da, x, P["w1"], dx, G["w1"], residual=dh2)
    xp.xpipe_embedding_bwd(dx, tok, G["table"])

    W = {k: t.double().requires_grad_() for k, t in p.items()}
    norm = lambda t, w: t / (t.square().mean(1, keepdim=True) + 1e-6).sqrt() * w
    X = W["table"][tokens.long()]
    Q, K, U = (norm(X, W["w1"]) @ W["qkv"].t()).view(B, n, 3, H, D).permute(2, 0, 3, 1, 4)
    d = torch.arange(n)[None, :] - torch.arange(n)[:, None]
    one = torch.tensor([_bucket(i, 8, R) for i in range(R + 1)])
    e = d.clamp(-R, R)
    at = one[e.abs()] + 8 * (e > 0)
    s = 4 * torch.tanh(Q @ K.transpose(2, 3) * D ** -0.5 / 4) + W["rel"][at].permute(2, 0, 1)
    O = torch.softmax(s.masked_fill(d > 0, -math.inf), 3) @ U
    Hh = X + O.permute(0, 2, 1, 3).reshape(M, C) @ W["out"].t()
    Z = norm(Hh, W["w2"]) @ W["top"].t()
    Z.backward(dz.double())
    # 2000 roundings of 2^-24 on the longest way through the block, by the 2-norm of each result
    for name, got, want in [("z", z, Z.detach())] + [(k, G[k], W[k].grad) for k in p]:
        off = float((_d(got) - want).norm() / want.norm())
        assert off <= 2000 * E24, f"{name}: {off:.3e}"
