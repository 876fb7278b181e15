"""The operators around a stage that are timed on this framework: the linear
layer with bias, activation and residual in its epilogue and its gradients,
the embedding lookup and its gradient, and the updates clipped by the global
gradient norm, through the public entry points (own) and as plain torch.

Sizes: the small MLP (256 wide, micro-batch 32) and ResNet-101 (its parameter
tensors; its head of 2048 -> 200 over micro-batch 100) come from the stages that
the repository trains, the 1e8 parameters from its update sweep; the others are
generic sizes of token models, of one token up to 65536."""
import math
import random

import torch

own = False

LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
MOMENTUM, WEIGHT_DECAY, ALPHA, RULE_LR = 0.9, 5e-4, 0.99, 1e-2
STEP = 7  # completed updates before the timed one
S_FWD, S_BWD = 2, 1  # version differences of the predictions that the Adam update emits
CLIP_EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "silu")


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token through a projection with an activation, as a generation step calls it: the weights are read once
        dict(name="linear_1_token", op="linear", rows=1, cin=4096, cout=4096, dtype="bf16", act="silu", residual=False,
             keep=False, pitch=0),
        # a micro-batch of tokens through the first matrix of an MLP block, with the pre-activation kept for the backward
        dict(name="linear_512_gelu", op="linear", rows=512, cin=1024, cout=4096, dtype="bf16", act="gelu",
             residual=False, keep=True, pitch=0),
        # a large micro-batch through a wide block's second matrix, the skip connection added
        dict(name="linear_8192_skip", op="linear", rows=8192, cin=16384, cout=4096, dtype="bf16", act="none",
             residual=True, keep=False, pitch=0),
        # fp32 storage, odd sizes, rows of a wider buffer
        dict(name="linear_f32_ragged", op="linear", rows=777, cin=1030, cout=515, dtype="f32", act="relu",
             residual=True, keep=False, pitch=3),
        # the gradients of ResNet-101's classifier over one micro-batch
        dict(name="linear_bwd_head", op="linear_bwd", rows=100, cin=2048, cout=200, dtype="bf16", act="none",
             skip=False, pitch=0),
        # the gradients of an MLP block's second matrix: the data gradient goes through the activation before it
        dict(name="linear_bwd_8192", op="linear_bwd", rows=8192, cin=8192, cout=2048, dtype="bf16", act="gelu",
             skip=False, pitch=0),
        # odd sizes in both directions, with a skip connection's gradient
        dict(name="linear_bwd_ragged", op="linear_bwd", rows=1001, cin=999, cout=1333, dtype="bf16", act="silu",
             skip=True, pitch=0),
        # the first stage's input: 8 sequences of 512 tokens
        dict(name="embed_4096", op="embed", tokens=4096, vocab=32000, dim=1024, dtype="bf16", padded=False),
        # the table's gradient of a few short sequences, padded to one length
        dict(name="embed_bwd_256", op="embed_bwd", tokens=256, vocab=1000, dim=256, dtype="f32", padded=True),
        # the table's gradient of a large micro-batch: a token in 16 is the most frequent one
        dict(name="embed_bwd_65536", op="embed_bwd", tokens=65536, vocab=50000, dim=2048, dtype="bf16", padded=False),
        # momentum SGD on ResNet-101, clipped by the norm over all its parameter tensors
        dict(name="clip_sgd_resnet101", op="clip", rule="sgd", tensors=0, n=0, max_norm=1.0),
        # Adam with both predictions on one flat buffer of 1e8 parameters, clipped
        dict(name="clip_adam_1e8", op="clip", rule="adam", tensors=1, n=100_000_000, max_norm=1.0),
    ]


def draw(rng):
    def size(lo, hi, unit=64):
        v = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return max(unit, v // unit * unit) if unit <= v and rng.random() < 0.6 else v

    op = rng.choice(("linear", "linear", "linear_bwd", "linear_bwd", "embed", "embed_bwd", "clip"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("linear", "linear_bwd"):
        most = (1.0e12 if dtype == "bf16" else 1.5e11) / (2 if op == "linear" else 4)
        rows, cin, cout = size(1, 16384), size(16, 16384), size(16, 16384)
        while rows * cin * cout > most:
            rows, cin, cout = -(-rows // 2), -(-cin // 2), -(-cout // 2)
        case = dict(op=op, rows=rows, cin=cin, cout=cout, dtype=dtype, act=rng.choice(ACTS),
                    pitch=rng.choice((0, 0, 5, 64)))
        if op == "linear":
            case.update(residual=rng.random() < 0.5, keep=rng.random() < 0.5)
        else:
            case.update(skip=rng.random() < 0.5)
        return case
    if op in ("embed", "embed_bwd"):
        tokens, dim, vocab = size(1, 65536), size(16, 4096, 16), size(100, 130000, 1)
        while tokens * dim > 65536 * 2048:
            tokens = -(-tokens // 2)
        while vocab * dim > 50000 * 4096:
            vocab = -(-vocab // 2)
        return dict(op=op, tokens=tokens, vocab=vocab, dim=dim, dtype=dtype, padded=rng.random() < 0.5)
    return dict(op=op, rule=rng.choice(("adam", "sgd", "rmsprop")), tensors=size(1, 400, 1), n=size(1000, 10 ** 8, 1),
                max_norm=rng.choice((0.1, 1.0, 1e4)))


# ---------------------------------------------------------------- inputs
def _resnet101_tensors():
    """Element counts of ResNet-101's parameter tensors (200 classes), in buffer order."""
    bn = lambda c: [c, c]
    out, cin = [64 * 49 * 3] + bn(64), 64
    for g, blocks in enumerate((3, 4, 23, 3)):
        mid = 64 << g
        for j in range(blocks):
            out += [cin * mid] + bn(mid) + [9 * mid * mid] + bn(mid)
            out += [cin * 4 * mid] + bn(4 * mid) if j == 0 else []
            out += [4 * mid * mid] + bn(4 * mid)
            cin = 4 * mid
    return out + [200 * cin, 200]


def _tensors(case):
    """(offset, count) of the tensors in the flat buffer, and its length."""
    if case["tensors"] == 0:  # each at a multiple of 64 elements, as a stage lays them out
        counts = _resnet101_tensors()
        ends = [0]
        for c in counts:
            ends.append(ends[-1] + -(-c // 64) * 64)
        return list(zip(ends[:-1], counts)), ends[-1]
    k = min(case["tensors"], case["n"])
    cuts = sorted(random.Random(case["n"]).sample(range(1, case["n"]), k - 1)) if k > 1 else []
    ends = [0] + cuts + [case["n"]]
    return [(a, b - a) for a, b in zip(ends[:-1], ends[1:])], case["n"]


def _inputs(case, seed):
    """The case's inputs: tensors on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES.get(case.get("dtype"))
    normal = lambda *shape, scale=1.0: torch.randn(*shape, generator=g, device="cuda") * scale

    def rows_of(n, c, scale=1.0):  # [n, c], of a wider buffer where the case says so
        return normal(n, c + case["pitch"], scale=scale).to(dt)[:, :c]

    op = case["op"]
    if op in ("linear", "linear_bwd"):
        M, K, N = case["rows"], case["cin"], case["cout"]
        d = dict(x=rows_of(M, K), W=normal(N, K, scale=K ** -0.5).to(dt))
        if op == "linear":
            d.update(b=normal(N, scale=0.1), r=rows_of(M, N) if case["residual"] else None)
        else:
            d.update(dz=rows_of(M, N, scale=1e-2), gW=normal(N, K, scale=1e-2), gb=normal(N, scale=1e-2),
                     z=rows_of(M, K) if case["act"] != "none" else None, dres=rows_of(M, K, scale=1e-2) if case["skip"] else None)
        return d
    if op in ("embed", "embed_bwd"):
        n, V, D = case["tokens"], case["vocab"], case["dim"]
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        tok = torch.exp(u * math.log(V + 1)).long().clamp(1, V) - 1  # a token's frequency falls as 1 / rank
        if case["padded"]:  # one position in eight is padding
            tok = torch.where(torch.rand(n, generator=g, device="cuda") < 0.125, torch.full_like(tok, -1), tok)
        d = dict(tokens=tok.to(torch.int32))
        if op == "embed":
            d["table"] = normal(V, D, scale=0.02).to(dt)
        else:
            d.update(dy=normal(n, D, scale=1e-2).to(dt), grad=normal(V, D, scale=1e-3))
        return d
    n = _tensors(case)[1]
    d = dict(W=normal(n, scale=0.02), m=normal(n, scale=1e-3), v=torch.rand(n, generator=g, device="cuda") * 1e-4,
             G=normal(n, scale=1e-3))
    if case["rule"] != "adam":
        d["buf"] = normal(n, scale=1e-3)
    if case["rule"] == "rmsprop":
        d["sq"] = torch.rand(n, generator=g, device="cuda") * 1e-4
    return d


def prepare(case, seed):
    d, op = _inputs(case, seed), case["op"]
    empty = lambda *shape: torch.empty(*shape, dtype=TYPES[case["dtype"]], device="cuda")
    out = {}
    if op == "linear":
        out = dict(y=empty(case["rows"], case["cout"]), z=empty(case["rows"], case["cout"]) if case["keep"] else None)
    elif op == "linear_bwd":
        out = dict(dx=empty(case["rows"], case["cin"]))
    elif op == "embed":
        out = dict(y=empty(case["tokens"], case["dim"]))
    elif op == "clip":
        views, n = _tensors(case)
        out = dict(norm=torch.zeros(2, device="cuda"), grads=[d["G"][o:o + c] for o, c in views])
        if case["rule"] == "adam":
            out.update(pf=torch.empty(n, device="cuda"), pb=torch.empty(n, device="cuda"))
    return dict(case=dict(case), scale=float(case.get("dim", 1)) ** 0.5, **d, **out)


# ---------------------------------------------------------------- one pass
def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_linear(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    z = s["x"].float() @ s["W"].float().t() + s["b"]
    y = _act(z, c["act"])
    if c["residual"]:
        y = y + s["r"].float()
    return {"y": y.to(dt), "z": z.to(dt) if c["keep"] else None}


def _plain_linear_bwd(s):
    c, dt = s["case"], TYPES[s["case"]["dtype"]]
    dz, x = s["dz"].float(), s["x"].float()
    dx = dz @ s["W"].float()
    if c["act"] != "none":
        dx = dx * _act_grad(s["z"].float(), c["act"])
    if c["skip"]:
        dx = dx + s["dres"].float()
    s["gW"] += dz.t() @ x
    s["gb"] += dz.sum(0)
    return {"dx": dx.to(dt), "gW": s["gW"], "gb": s["gb"]}


def _plain_embed(s):
    t = s["tokens"].long()
    rows = s["table"][t.clamp(min=0)].float() * s["scale"]
    return {"y": (rows * (t >= 0)[:, None]).to(s["table"].dtype)}


def _plain_embed_bwd(s):
    t = s["tokens"].long()
    rows = s["dy"].float() * (s["scale"] * (t >= 0).float())[:, None]
    s["grad"].index_add_(0, t.clamp(min=0), rows)
    return {"grad": s["grad"]}


def _plain_clip(s):
    c, t = s["case"], STEP + 1
    norm = torch.cat(s["grads"]).square().sum().sqrt()
    coef = (c["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    g = s["G"] * coef
    if c["rule"] != "adam":
        g = g + WEIGHT_DECAY * s["W"]
    s["m"].mul_(BETA1).add_(g * (1 - BETA1))
    s["v"].mul_(BETA2).add_(g * g * (1 - BETA2))
    out = {"norm": torch.stack((norm, coef)), "W": s["W"], "m": s["m"], "v": s["v"]}
    if c["rule"] == "adam":
        mh, vh = s["m"] / (1 - BETA1 ** t), s["v"] / (1 - BETA2 ** t)
        s["W"] -= LR * mh / (vh.sqrt() + EPS)
        step = LR * mh / (vh + EPS).sqrt()
        return dict(out, pf=s["W"] - S_FWD * step, pb=s["W"] - S_BWD * step)
    if c["rule"] == "rmsprop":
        s["sq"].mul_(ALPHA).add_(g * g * (1 - ALPHA))
        g = g / (s["sq"].sqrt() + EPS)
        out["sq"] = s["sq"]
    s["buf"].mul_(MOMENTUM).add_(g)
    s["W"] -= RULE_LR * s["buf"]
    return dict(out, buf=s["buf"])


_PLAIN = {"linear": _plain_linear, "linear_bwd": _plain_linear_bwd, "embed": _plain_embed,
          "embed_bwd": _plain_embed_bwd, "clip": _plain_clip}


def _own(s):
    import paper_1911_04610_amd as xp
    c, op = s["case"], s["case"]["op"]
    act = {"none": xp.ACT_NONE, "relu": xp.ACT_RELU, "gelu": xp.ACT_GELU, "silu": xp.ACT_SILU}
    if op == "linear":
        xp.xpipe_linear_fwd(s["x"], s["W"], s["b"], s["y"], act=act[c["act"]], residual=s["r"], preact=s["z"])
        return {"y": s["y"], "z": s["z"]}
    if op == "linear_bwd":
        xp.xpipe_linear_bwd(s["dz"], s["x"], s["W"], s["dx"], s["gW"], s["gb"], act=act[c["act"]], preact=s["z"],
                            residual=s["dres"])
        return {"dx": s["dx"], "gW": s["gW"], "gb": s["gb"]}
    if op == "embed":
        xp.xpipe_embedding_fwd(s["table"], s["tokens"], s["y"], scale=s["scale"])
        return {"y": s["y"]}
    if op == "embed_bwd":
        xp.xpipe_embedding_bwd(s["dy"], s["tokens"], s["grad"], scale=s["scale"])
        return {"grad": s["grad"]}
    if "list" not in s:  # a training program keeps the list of its gradients
        s["list"] = xp.TensorList(s["grads"])
    hp = xp.Hyper(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS)
    xp.xpipe_grad_norm(s["list"], c["max_norm"], s["norm"])
    out = {"norm": s["norm"], "W": s["W"], "m": s["m"], "v": s["v"]}
    if c["rule"] == "adam":
        xp.xpipe_adam_flat(s["W"], s["m"], s["v"], s["G"], hp, STEP, zero_grad=False, pred_fwd=s["pf"], s_fwd=S_FWD,
                           pred_bwd=s["pb"], s_bwd=S_BWD, clip=s["norm"])
        return dict(out, pf=s["pf"], pb=s["pb"])
    rms = c["rule"] == "rmsprop"
    rule = xp.Rule(xp.RULE_RMSPROP if rms else xp.RULE_MOMENTUM_SGD, lr=RULE_LR, momentum=MOMENTUM,
                   weight_decay=WEIGHT_DECAY, alpha=ALPHA, eps=EPS)
    xp.xpipe_rule_flat(s["W"], s["buf"], s["sq"] if rms else None, s["m"], s["v"], s["G"], rule, hp, STEP,
                       zero_grad=False, clip=s["norm"])
    if rms:
        out["sq"] = s["sq"]
    return dict(out, buf=s["buf"])


def run(s):
    return _own(s) if own else _PLAIN[s["case"]["op"]](s)


# ---------------------------------------------------------------- work
def work(case):
    op, e = case["op"], 2 if case.get("dtype") == "bf16" else 4
    if op == "linear":
        M, K, N = case["rows"], case["cin"], case["cout"]
        return {"bytes": e * (M * K + N * K + M * N * (1 + case["residual"] + case["keep"])) + 4 * N, "flops": 2 * M * N * K}
    if op == "linear_bwd":
        M, K, N = case["rows"], case["cin"], case["cout"]
        more = (case["act"] != "none") + case["skip"]
        return {"bytes": e * (M * N + N * K + M * K * (2 + more)) + 8 * (N * K + N), "flops": 4 * M * N * K + M * N}
    if op in ("embed", "embed_bwd"):
        n, V, D = case["tokens"], case["vocab"], case["dim"]
        live = n * (0.875 if case["padded"] else 1.0)
        p = [math.log(1 + 1 / (i + 1)) / math.log(V + 1) for i in range(V)]
        distinct = sum(-math.expm1(live * math.log1p(-q)) if q < 1 else 1.0 for q in p)  # expected distinct tokens
        if op == "embed":
            return {"bytes": e * D * (n + distinct) + 4 * n, "flops": live * D}
        return {"bytes": e * D * live + 8 * D * distinct + 4 * n, "flops": 2 * live * D}
    n = _tensors(case)[1]
    per = {"adam": 36, "sgd": 36, "rmsprop": 44}[case["rule"]]
    return {"bytes": per * n, "flops": 20 * n}


# ---------------------------------------------------------------- 64 bits
def _exact_linear(case, d):
    z = torch.addmm(d["b"].double(), d["x"].double(), d["W"].double().t().contiguous())
    y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)),
         "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
    return {"y": y if d["r"] is None else y + d["r"].double(), "z": z if case["keep"] else None}


def _exact_linear_bwd(case, d):
    dz, x = d["dz"].double(), d["x"].double()
    dx = torch.mm(dz, d["W"].double())
    if case["act"] != "none":
        z = d["z"].double()
        if case["act"] == "relu":
            dx = torch.where(z > 0, dx, torch.zeros_like(dx))
        elif case["act"] == "gelu":
            dx.mul_(torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        else:
            sig = torch.sigmoid(z)
            dx.mul_(sig + z * sig * (1 - sig))
    if d["dres"] is not None:
        dx.add_(d["dres"].double())
    gW = torch.addmm(d["gW"].double(), dz.t().contiguous(), x)
    return {"dx": dx, "gW": gW, "gb": d["gb"].double() + dz.sum(dim=0)}


def _exact_embed(case, d):
    y = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
    at = (d["tokens"] >= 0).nonzero().flatten()
    y[at] = d["table"].index_select(0, d["tokens"][at].long()).double() * math.sqrt(case["dim"])
    return {"y": y}


def _exact_embed_bwd(case, d):
    at = (d["tokens"] >= 0).nonzero().flatten()
    grad = d["grad"].double()
    grad.index_add_(0, d["tokens"][at].long(), d["dy"][at].double(), alpha=math.sqrt(case["dim"]))
    return {"grad": grad}


def _exact_clip(case, d):
    total = sum(d["G"][o:o + c].double().dot(d["G"][o:o + c].double()).item() for o, c in _tensors(case)[0])
    norm = math.sqrt(total)
    coef = min(1.0, case["max_norm"] / (norm + CLIP_EPS))
    W, g, t = d["W"].double(), d["G"].double() * coef, STEP + 1
    if case["rule"] != "adam":
        g = g + WEIGHT_DECAY * W
    m = torch.lerp(g, d["m"].double(), BETA1)
    v = torch.lerp(g.square(), d["v"].double(), BETA2)
    out = {"norm": torch.tensor([norm, coef], dtype=torch.float64), "m": m, "v": v}
    if case["rule"] == "adam":
        mh, vh = m / -math.expm1(t * math.log(BETA1)), v / -math.expm1(t * math.log(BETA2))
        W = torch.addcdiv(W, mh, vh.sqrt() + EPS, value=-LR)
        root = (vh + EPS).sqrt()
        return dict(out, W=W, pf=torch.addcdiv(W, mh, root, value=-S_FWD * LR),
                    pb=torch.addcdiv(W, mh, root, value=-S_BWD * LR))
    if case["rule"] == "rmsprop":
        out["sq"] = torch.lerp(g.square(), d["sq"].double(), ALPHA)
        g = g / (out["sq"].sqrt() + EPS)
    buf = torch.add(g, d["buf"].double(), alpha=MOMENTUM)
    return dict(out, W=torch.add(W, buf, alpha=-RULE_LR), buf=buf)


def exact(case, seed):
    d = _inputs(case, seed)
    return {"linear": _exact_linear, "linear_bwd": _exact_linear_bwd, "embed": _exact_embed,
            "embed_bwd": _exact_embed_bwd, "clip": _exact_clip}[case["op"]](case, d)
