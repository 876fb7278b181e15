"""The operators of token networks that are timed on this framework: the RMS norm
with the skip connection's addition and its gradients, the relative position bias
by buckets and its gradient, and attention with a capped score, a bias by distance
and causal, prefix and document masks, forward and with its gradients, through the
public entry points (own) and as plain torch.

Sizes are generic sizes of token models, from one token to 16384 rows and 32768 keys;
the widths are those of the other timed operators."""
import math
import random

import torch

own = False

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token through a block's norm, the skip connection added, as a generation step calls it
        dict(name="norm_1_token", op="norm", rows=1, dim=4096, dtype="bf16", residual=True, keep=True, pitch=0),
        # a large micro-batch through the same norm
        dict(name="norm_16384", op="norm", rows=16384, dim=4096, dtype="bf16", residual=True, keep=True, pitch=0),
        # the gradients of a micro-batch's norm, the skip connection's gradient added
        dict(name="norm_bwd_8192", op="norm_bwd", rows=8192, dim=2048, dtype="bf16", skip=True, pitch=0),
        # fp32 storage, odd sizes, rows of a wider buffer
        dict(name="norm_bwd_f32_ragged", op="norm_bwd", rows=1001, dim=999, dtype="f32", skip=False, pitch=3),
        # one layer's bias table and its gradient, both directions
        dict(name="relbias_128", op="relbias", buckets=32, heads=12, max_distance=128, both=True),
        # a bias over long distances, keys before the query only
        dict(name="relbias_32768", op="relbias", buckets=64, heads=64, max_distance=32768, both=False),
        # a generation step: one token of each of 8 sequences over their caches, of different lengths
        dict(name="attn_1_token", op="attn", batch=8, nq=1, nk=32768, heads=32, kv_heads=8, dim=128, dtype="bf16",
             mask="causal", cap=0.0, bias=0, ragged=True, pitch=0),
        # a short batch of padded sequences with a bias, no causal mask: an encoder's call
        dict(name="attn_77_bias", op="attn", batch=4, nq=77, nk=77, heads=8, kv_heads=8, dim=64, dtype="bf16",
             mask="none", cap=0.0, bias=32, ragged=True, pitch=0),
        # one long sequence with capped scores
        dict(name="attn_8192_cap", op="attn", batch=1, nq=8192, nk=8192, heads=16, kv_heads=16, dim=128, dtype="bf16",
             mask="causal", cap=50.0, bias=0, ragged=False, pitch=0),
        # a training step over documents packed into one row, with the learned bias
        dict(name="attn_train_docs_bias", op="attn_train", batch=2, nq=4096, nk=4096, heads=12, kv_heads=12, dim=64,
             dtype="bf16", mask="docs", cap=0.0, bias=128, ragged=False, pitch=0),
        # a training step with shared heads, each sequence's prefix visible to all of it
        dict(name="attn_train_prefix", op="attn_train", batch=2, nq=4096, nk=4096, heads=16, kv_heads=4, dim=128,
             dtype="bf16", mask="prefix", cap=0.0, bias=0, ragged=False, pitch=0),
        # fp32 storage, odd sizes, heads of a wider buffer, everything at once
        dict(name="attn_train_f32_ragged", op="attn_train", batch=3, nq=301, nk=333, heads=6, kv_heads=3, dim=40,
             dtype="f32", mask="causal", cap=30.0, bias=50, ragged=True, pitch=3),
    ]


def draw(rng):
    def size(lo, hi, unit=16):
        v = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return max(unit, v // unit * unit) if unit <= v and rng.random() < 0.6 else v

    op = rng.choice(("norm", "norm_bwd", "relbias", "attn", "attn", "attn_token", "attn_train", "attn_train", "attn_train"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("norm", "norm_bwd"):
        rows, dim = size(1, 65536), size(16, 16384)
        while rows * dim > 16384 * 2048 * (2 if dtype == "bf16" else 1):
            rows = -(-rows // 2)
        case = dict(op=op, rows=rows, dim=dim, dtype=dtype, pitch=rng.choice((0, 0, 5, 64)))
        if op == "norm":
            case.update(residual=rng.random() < 0.7, keep=rng.random() < 0.7)
        else:
            case.update(skip=rng.random() < 0.5)
        return case
    if op == "relbias":
        return dict(op=op, buckets=rng.choice((8, 16, 32, 64)), heads=size(1, 64, 1), max_distance=size(64, 32768, 1),
                    both=rng.random() < 0.5)
    kv_heads = rng.choice((1, 2, 4, 8))
    case = dict(heads=kv_heads * rng.choice((1, 1, 2, 4)), kv_heads=kv_heads,
                dim=rng.choice((64, 128, 64, 128, 16, 32, 80, 96, 72, 33)), dtype=dtype,
                cap=rng.choice((0.0, 0.0, 20.0, 50.0)), pitch=rng.choice((0, 0, 0, 1, 16)))
    if op == "attn_token":
        case.update(op="attn", batch=size(1, 16, 1), nq=rng.choice((1, 1, 2, 5)), nk=size(16, 32768), mask="causal",
                    bias=rng.choice((0, 0, 128)), ragged=rng.random() < 0.7)
        return case
    most = (2 ** 28 if op == "attn" else 2 ** 27) // (1 if dtype == "bf16" else 8)
    least = 32 if op == "attn_train" else 1  # (one key alone has no gradient: its softmax is constant)
    batch, nq = size(1, 16, 1), size(least, 8192)
    while batch * case["heads"] * nq * nq > most:
        batch, nq = (-(-batch // 2), nq) if batch > 1 and rng.random() < 0.5 else (batch, max(least, nq * 3 // 4))
    mask = rng.choice(("none", "causal", "causal", "prefix", "docs"))
    nk = nq if mask == "docs" or rng.random() < 0.7 else size(max(least, nq // 4), nq)
    case.update(op=op, batch=batch, nq=nq, nk=nk, mask=mask, bias=rng.choice((0, 0, 0, 64, 128, nk)),
                ragged=mask != "docs" and rng.random() < 0.5)
    return case


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """Of each sequence: its queries, its keys, its prefix, and its documents' lengths (what is left of them is padding)."""
    r = random.Random("%d %d %d" % (case["batch"], case["nq"], case["nk"]))
    nq, nk, out = case["nq"], case["nk"], []
    for _ in range(case["batch"]):
        kl = r.randint((nk + 1) // 2, nk) if case["ragged"] else nk
        ql = min(nq, max(1, r.randint((nq + 1) // 2, nq))) if case["ragged"] and nq > 8 else nq
        docs, left = [], nk - nk // 32
        while left > 0:
            docs.append(min(left, max(1, round(math.exp(r.uniform(math.log(32), math.log(max(33, nk / 2))))))))
            left -= docs[-1]
        out.append((ql, kl, r.randint(nk // 8, nk // 2), docs))
    return out


def _visible(case):
    """(query, key) pairs that the masks leave."""
    total = 0
    for ql, kl, prefix, docs in _lengths(case):
        if case["mask"] == "docs":
            total += sum(n * (n + 1) // 2 for n in docs)
            continue
        for i in range(ql):
            pos = i + kl - ql
            end = {"none": kl, "causal": pos + 1, "prefix": max(pos + 1, prefix)}[case["mask"]]
            total += max(0, min(end, kl))
    return total * case["heads"]


def _inputs(case, seed):
    """The case's inputs: tensors on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES.get(case.get("dtype"))
    normal = lambda *shape, scale=1.0: torch.randn(*shape, generator=g, device="cuda") * scale

    def wide(*shape, scale=1.0):  # a tensor of that shape, of a buffer with longer rows where the case says so
        return normal(*shape[:-1], shape[-1] + case["pitch"], scale=scale).to(dt)[..., :shape[-1]]

    op = case["op"]
    if op in ("norm", "norm_bwd"):
        n, c = case["rows"], case["dim"]
        d = dict(w=1 + normal(c, scale=0.1))
        if op == "norm":
            d.update(x=wide(n, c), r=wide(n, c, scale=3.0) if case["residual"] else None)
        else:
            d.update(dy=wide(n, c, scale=1e-2), h=wide(n, c, scale=3.0), r=wide(n, c, scale=1e-2) if case["skip"] else None,
                     gw=normal(c, scale=1e-2))
        return d
    if op == "relbias":
        b, h = case["buckets"], case["heads"]
        return dict(table=normal(b, h), grad=normal(b, h, scale=1e-2), dbias=normal(h, 2 * case["max_distance"] + 1, scale=1e-2))
    B, nq, nk, H, K, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    d = dict(q=wide(B, nq, H, D), k=wide(B, nk, K, D), v=wide(B, nk, K, D))
    if case["bias"]:
        d["bias"] = normal(H, 2 * case["bias"] + 1)
    if op == "attn_train":
        d["do"] = wide(B, nq, H, D, scale=1e-2)
        if case["bias"]:
            d["gbias"] = normal(H, 2 * case["bias"] + 1, scale=1e-2)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    lengths = _lengths(case)
    if case["ragged"]:
        d.update(q_len=ints([n[0] for n in lengths]), k_len=ints([n[1] for n in lengths]))
    if case["mask"] == "prefix":
        d["prefix"] = ints([n[2] for n in lengths])
    if case["mask"] == "docs":
        doc = [[j for j, n in enumerate(docs) for _ in range(n)] for _, _, _, docs in lengths]
        d["doc"] = ints([v + [-1] * (nk - len(v)) for v in doc])
    return d


def prepare(case, seed):
    d, op = _inputs(case, seed), case["op"]
    empty = lambda *shape, dtype=None: torch.empty(*shape, dtype=dtype or TYPES[case["dtype"]], device="cuda")
    out = {}
    if op == "norm":
        out = dict(y=empty(case["rows"], case["dim"]), h=empty(case["rows"], case["dim"]) if case["keep"] else None)
    elif op == "norm_bwd":
        out = dict(dx=empty(case["rows"], case["dim"]))
    elif op == "relbias":
        out = dict(bias=empty(case["heads"], 2 * case["max_distance"] + 1, dtype=torch.float32))
    else:
        for name in ("q_len", "k_len", "prefix", "doc", "bias", "gbias"):
            d.setdefault(name, None)
        B, nq, nk, H, K, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
        out = dict(o=empty(B, nq, H, D), stats=empty(B, H, nq, 2, dtype=torch.float32))
        if op == "attn_train":
            out.update(dq=empty(B, nq, H, D), dk=empty(B, nk, K, D), dv=empty(B, nk, K, D))
    return dict(case=dict(case), **d, **out)


# ---------------------------------------------------------------- one pass
def _plain_norm(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    y = h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * s["w"]
    return {"y": y.to(s["x"].dtype), "h": h.to(s["x"].dtype) if s["case"]["keep"] else None}


def _plain_norm_bwd(s):
    h, dy = s["h"].float(), s["dy"].float()
    n = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    g = dy * s["w"]
    dx = n * (g - h * (n * n * (g * h).mean(1, keepdim=True)))
    if s["r"] is not None:
        dx = dx + s["r"].float()
    s["gw"] += (dy * h * n).sum(0)
    return {"dx": dx.to(s["h"].dtype), "gw": s["gw"]}


def _plain_relbias(s):
    c, R = s["case"], s["case"]["max_distance"]
    n = c["buckets"] // 2 if c["both"] else c["buckets"]
    d = torch.arange(-R, R + 1, device="cuda")
    away = d.abs() if c["both"] else (-d).clamp(min=0)
    half = n // 2
    far = torch.log(away.double().clamp(min=half) / half) / math.log(R / half) * (n - half)
    bucket = torch.where(away < half, away, (half + torch.floor(far + 1e-9).long()).clamp(max=n - 1))
    if c["both"]:
        bucket = bucket + n * (d > 0).long()
    s["bias"].copy_(s["table"][bucket].t())
    in_bucket = (bucket == torch.arange(c["buckets"], device="cuda")[:, None]).double()
    s["grad"].copy_(s["grad"] + in_bucket @ s["dbias"].double().t().contiguous())
    return {"bias": s["bias"], "grad": s["grad"]}


def _geometry(s):
    """(which pairs the masks leave [B, 1, nq, nk], key position - query position of the first pair of each sequence [B])"""
    c = s["case"]
    i, j = torch.arange(c["nq"], device="cuda"), torch.arange(c["nk"], device="cuda")
    ql = s["q_len"] if s["q_len"] is not None else torch.full((c["batch"],), c["nq"], device="cuda")
    kl = s["k_len"] if s["k_len"] is not None else torch.full((c["batch"],), c["nk"], device="cuda")
    ahead = (kl - ql).long()
    see = (i[None, :, None] < ql[:, None, None]) & (j[None, None, :] < kl[:, None, None])
    if c["mask"] != "none":
        past = j[None, None, :] <= i[None, :, None] + ahead[:, None, None]
        if c["mask"] == "prefix":
            past = past | (j[None, None, :] < s["prefix"][:, None, None])
        see = see & past
    if c["mask"] == "docs":
        see = see & (s["doc"][:, :, None] == s["doc"][:, None, :]) & (s["doc"][:, None, :] >= 0)
    return see[:, None], -ahead


def _plain_attn(s):
    c = s["case"]
    B, nq, nk, H, K, D = (c[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    G, dt = H // K, s["q"].dtype
    see, first = _geometry(s)
    heads = lambda t: t.float().permute(0, 2, 1, 3)
    q, k, v = heads(s["q"]), heads(s["k"]).repeat_interleave(G, 1), heads(s["v"]).repeat_interleave(G, 1)
    x = q @ k.transpose(2, 3) * D ** -0.5
    t = None
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = c["cap"] * t
    if c["bias"]:
        at = torch.arange(nk, device="cuda")[None, None, :] - torch.arange(nq, device="cuda")[None, :, None] + first[:, None, None]
        x = x + s["bias"][:, at.clamp(-c["bias"], c["bias"]) + c["bias"]].transpose(0, 1)
    x = x.masked_fill(~see, -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = p @ v
    out = {"o": o.permute(0, 2, 1, 3).to(dt)}
    if c["op"] == "attn":
        return out
    do = heads(s["do"])
    dp = do @ v.transpose(2, 3)
    ds = p * (dp - (do * o).sum(3, keepdim=True))
    shared = lambda t: t.reshape(B, K, G, nk, D).sum(2).permute(0, 2, 1, 3).to(dt)
    out["dv"] = shared(p.transpose(2, 3) @ do)
    if c["bias"]:  # rows shifted so that a diagonal is a column, then the columns' sums
        wide = torch.nn.functional.pad(ds.flip(2), (0, nq)).reshape(B, H, -1)[:, :, :nq * (nk + nq - 1)]
        sums = wide.reshape(B, H, nq, nk + nq - 1).sum(2, dtype=torch.float64)
        at = torch.arange(1 - nq, nk, device="cuda")[None, :] + first[:, None]
        at = (at.clamp(-c["bias"], c["bias"]) + c["bias"]).reshape(-1, 1)
        in_place = (at == torch.arange(2 * c["bias"] + 1, device="cuda")).double()
        s["gbias"].copy_(s["gbias"] + sums.transpose(0, 1).reshape(H, -1) @ in_place)
        out["gbias"] = s["gbias"]
    if c["cap"]:
        ds = ds * (1 - t * t)
    ds = ds * D ** -0.5
    out["dq"] = (ds @ k).permute(0, 2, 1, 3).to(dt)
    out["dk"] = shared(ds.transpose(2, 3) @ q)
    return out


_PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "relbias": _plain_relbias, "attn": _plain_attn,
          "attn_train": _plain_attn}


def _own(s):
    import paper_1911_04610_amd as xp
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        xp.xpipe_rmsnorm_fwd(s["x"], s["w"], s["y"], eps=EPS, residual=s["r"], sum=s["h"])
        return {"y": s["y"], "h": s["h"]}
    if op == "norm_bwd":
        xp.xpipe_rmsnorm_bwd(s["dy"], s["h"], s["w"], s["dx"], s["gw"], eps=EPS, residual=s["r"])
        return {"dx": s["dx"], "gw": s["gw"]}
    if op == "relbias":
        xp.xpipe_relbias_fwd(s["table"], s["bias"], bidirectional=c["both"])
        xp.xpipe_relbias_bwd(s["dbias"], s["grad"], bidirectional=c["both"])
        return {"bias": s["bias"], "grad": s["grad"]}
    how = dict(causal=c["mask"] != "none", cap=c["cap"], bias=s["bias"], q_len=s["q_len"], k_len=s["k_len"],
               prefix=s["prefix"], q_doc=s["doc"], k_doc=s["doc"])
    if op == "attn":
        xp.xpipe_attention_fwd(s["q"], s["k"], s["v"], s["o"], **how)
        return {"o": s["o"]}
    xp.xpipe_attention_fwd(s["q"], s["k"], s["v"], s["o"], stats=s["stats"], **how)
    xp.xpipe_attention_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["stats"], s["dq"], s["dk"], s["dv"], s["gbias"], **how)
    out = {"o": s["o"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    return dict(out, gbias=s["gbias"]) if c["bias"] else out


def run(s):
    return _own(s) if own else _PLAIN[s["case"]["op"]](s)


# ---------------------------------------------------------------- work
def work(case):
    op, e = case["op"], 2 if case.get("dtype") == "bf16" else 4
    if op == "norm":
        n, c = case["rows"], case["dim"]
        return {"bytes": e * n * c * (2 + case["residual"] + case["keep"]) + 4 * c, "flops": 5 * n * c}
    if op == "norm_bwd":
        n, c = case["rows"], case["dim"]
        return {"bytes": e * n * c * (3 + case["skip"]) + 12 * c, "flops": 12 * n * c}
    if op == "relbias":
        n, h, b = 2 * case["max_distance"] + 1, case["heads"], case["buckets"]
        return {"bytes": 8 * n * h + 12 * b * h, "flops": n * h}
    B, nq, H, K, D = (case[k] for k in ("batch", "nq", "heads", "kv_heads", "dim"))
    pairs, keys = _visible(case), sum(n[1] for n in _lengths(case))
    moved = e * D * (2 * B * nq * H + 2 * keys * K)
    if op == "attn":
        return {"bytes": moved, "flops": 4 * D * pairs}
    return {"bytes": moved + e * D * (2 * B * nq * H + 2 * B * case["nk"] * K), "flops": 14 * D * pairs}


# ---------------------------------------------------------------- 64 bits
def _exact_norm(case, d):
    h = d["x"].double() if d["r"] is None else torch.add(d["x"].double(), d["r"].double())
    rms = torch.sqrt(torch.linalg.vector_norm(h, dim=1).square() / case["dim"] + EPS)
    return {"y": d["w"].double() * h / rms[:, None], "h": h if case["keep"] else None}


def _exact_norm_bwd(case, d):
    h, dy, w, C = d["h"].double(), d["dy"].double(), d["w"].double(), case["dim"]
    var = torch.linalg.vector_norm(h, dim=1).square() / C + EPS
    unit = h / var.sqrt()[:, None]
    g = dy * w
    along = torch.mv(g * unit, torch.full((C,), 1 / C, dtype=torch.float64, device="cuda"))
    dx = torch.addcmul(g, unit, along[:, None], value=-1) / var.sqrt()[:, None]
    if d["r"] is not None:
        dx.add_(d["r"].double())
    return {"dx": dx, "gw": d["gw"].double() + torch.mul(dy, unit).sum(dim=0)}


def _bucket(away, n, far):
    """The bucket of a distance, in whole numbers: the last whose first distance is not beyond it."""
    half = n // 2
    if away < half:
        return away
    lo, hi = half, n - 1  # bucket half + k starts where (away / half)^(n - half) >= (far / half)^k
    while lo < hi:
        mid = (lo + hi + 1) // 2
        k = mid - half
        if away ** (n - half) * half ** k >= far ** k * half ** (n - half):
            lo = mid
        else:
            hi = mid - 1
    return lo


def _exact_relbias(case, d):
    R, both = case["max_distance"], case["both"]
    n = case["buckets"] // 2 if both else case["buckets"]
    one = [_bucket(a, n, R) for a in range(R + 1)]
    at = torch.tensor([one[-x] if x < 0 else one[x] + n if both and x else one[0] for x in range(-R, R + 1)], device="cuda")
    grad = d["grad"].double()
    for b in range(case["buckets"]):
        grad[b] += d["dbias"].double()[:, at == b].sum(1)
    return {"bias": d["table"].double().index_select(0, at).t().contiguous(), "grad": grad}


def _exact_attn(case, d):
    B, nq, nk, H, K, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    train, R, cap, f64 = case["op"] == "attn_train", case["bias"], case["cap"], torch.float64
    zeros = lambda *shape: torch.zeros(*shape, dtype=f64, device="cuda")
    out = {"o": zeros(B, nq, H, D)}
    if train:
        out.update(dq=zeros(B, nq, H, D), dk=zeros(B, nk, K, D), dv=zeros(B, nk, K, D))
        if R:
            out["gbias"] = d["gbias"].double()
    for b, (ql, kl, prefix, docs) in enumerate(_lengths(case)):
        i = torch.arange(ql, device="cuda")[:, None] + (kl - ql)
        j = torch.arange(kl, device="cuda")[None, :]
        hidden = torch.zeros(ql, kl, dtype=torch.bool, device="cuda")
        if case["mask"] == "causal" or case["mask"] == "docs":
            hidden |= j > i
        if case["mask"] == "prefix":
            hidden |= (j > i) & (j >= prefix)
        if case["mask"] == "docs":
            ends = torch.tensor(docs, device="cuda").cumsum(0)
            of_q, of_k = torch.searchsorted(ends, i, right=True), torch.searchsorted(ends, j, right=True)
            hidden |= (of_q != of_k) | (of_k == len(docs))
        place = (j - i).clamp(-R, R) + R
        to_bias = zeros(H, ql, kl) if train and R else None
        for h in range(H):
            g = h // (H // K)
            q, k, v = d["q"][b, :ql, h].double(), d["k"][b, :kl, g].double(), d["v"][b, :kl, g].double()
            raw = torch.mm(q, k.t().contiguous()) / math.sqrt(D)
            score = cap * torch.tanh(raw / cap) if cap else raw
            if R:
                score = score + d["bias"][h].double()[place]
            score = torch.where(hidden, torch.full_like(score, -math.inf), score)
            w = torch.nan_to_num(torch.softmax(score, 1))  # (a row without a key: NaN, then 0)
            out["o"][b, :ql, h] = torch.mm(w, v)
            if not train:
                continue
            do = d["do"][b, :ql, h].double()
            out["dv"][b, :kl, g] += torch.mm(w.t().contiguous(), do)
            to_w = torch.mm(do, v.t().contiguous())
            to_s = w * (to_w - (w * to_w).sum(1, keepdim=True))
            if R:
                to_bias[h] = to_s
            if cap:
                to_s = to_s * torch.cosh(raw / cap).pow(-2)
            out["dq"][b, :ql, h] = torch.mm(to_s, k) / math.sqrt(D)
            out["dk"][b, :kl, g] += torch.mm(to_s.t().contiguous(), q) / math.sqrt(D)
        if train and R:
            for off in range(1 - ql, kl):
                at = min(max(off - (kl - ql), -R), R) + R
                out["gbias"][:, at] += torch.diagonal(to_bias, off, 1, 2).sum(1)
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    return {"norm": _exact_norm, "norm_bwd": _exact_norm_bwd, "relbias": _exact_relbias, "attn": _exact_attn,
            "attn_train": _exact_attn}[case["op"]](case, d)
