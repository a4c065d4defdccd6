"""The operators of a transformer block in a language-model worker's local step, as measured workloads.

Five operators, each in its plain form (elementary torch operations in 32 bits) and, where ``own``
is true, as the calls a user makes of this package:

  norm, norm_grad            layer norm after a residual addition; its gradient with the weight's and bias's
  rotary                     rotary positions on the heads of packed rows, and the inverse (its gradient)
  attention, attention_grad  attention within packed sequences; its gradient, which recomputes the probabilities

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes what a program
holds before the call, ``run`` is one pass, ``work`` what a pass cannot do without, ``exact`` the
same outputs in 64 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-5
MOST_VALUES = 1 << 28        # largest count of a drawn case's stream or head values
MOST_SCORES = 3_000_000_000  # largest count of scores, sequences padded to the longest
MOST_PAIRS = 2_000_000_000   # largest count of attended pairs times heads


def listed():
    return [
        # A handful of tokens: latency alone.
        {"name": "norm-few", "op": "norm", "tokens": 7, "width": 512, "x": "bfloat16", "branch": "", "out": "bfloat16", "weight": "bfloat16", "bias": True},
        # A training batch: the branch of the block before is added to an fp32 stream, the products read bf16.
        {"name": "norm-batch", "op": "norm", "tokens": 16384, "width": 4096, "x": "float32", "branch": "bfloat16", "out": "bfloat16", "weight": "float32", "bias": True},
        # A short batch of odd width.
        {"name": "norm-grad-short", "op": "norm_grad", "tokens": 333, "width": 257, "x": "float32", "out": "float32", "weight": "float32", "bias": True, "stream": False},
        # The training batch's gradient, added to the stream's.
        {"name": "norm-grad-batch", "op": "norm_grad", "tokens": 16384, "width": 4096, "x": "float32", "out": "bfloat16", "weight": "float32", "bias": True, "stream": True},
        # A handful of tokens of a small model, pairs side by side.
        {"name": "rotary-few", "op": "rotary", "tokens": 9, "heads": 8, "rest": 0, "dim": 64, "turned": 64, "interleaved": True, "dtype": "float32", "positions": "int64", "far": 300, "factor": 1.0, "inverse": False, "in_place": False},
        # Query and key heads of a batch's fused rows, in place, at far positions with frequencies for a longer context.
        {"name": "rotary-batch", "op": "rotary", "tokens": 16384, "heads": 40, "rest": 8, "dim": 128, "turned": 128, "interleaved": False, "dtype": "bfloat16", "positions": "int32", "far": 120000, "factor": 8.0, "inverse": False, "in_place": True},
        # A few short sequences of a small model: latency.
        {"name": "attention-short", "op": "attention", "tokens": 333, "sequences": 5, "tail": 0, "heads": 4, "kv_heads": 2, "dim": 64, "causal": True, "window": 0},
        # A packed training batch of documents, heads that share keys, some padding at the end.
        {"name": "attention-batch", "op": "attention", "tokens": 8192, "sequences": 6, "tail": 100, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "window": 0},
        # One long sequence, every token sees the last 4,096.
        {"name": "attention-window", "op": "attention", "tokens": 12289, "sequences": 1, "tail": 0, "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "window": 4096},
        # Gradients of the same short sequences.
        {"name": "attention-grad-short", "op": "attention_grad", "tokens": 333, "sequences": 5, "tail": 0, "heads": 4, "kv_heads": 2, "dim": 64, "causal": True, "window": 0},
        # ... of the packed batch.
        {"name": "attention-grad-batch", "op": "attention_grad", "tokens": 8192, "sequences": 6, "tail": 100, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "window": 0},
        # An encoder's: both directions, every head with keys of its own, an odd head width.
        {"name": "attention-grad-both-ways", "op": "attention_grad", "tokens": 5003, "sequences": 3, "tail": 0, "heads": 12, "kv_heads": 12, "dim": 72, "causal": False, "window": 0},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "rotary", "attention", "attention_grad", "attention_grad"])
    two = ["float32", "bfloat16"]
    if op in ("norm", "norm_grad"):
        width = rng.choice([64, 200, 256, 512, 768, 1000, 1024, 2048, 4096, 5120, 8192, rng.randrange(1, 700), rng.randrange(1, 1500) * 2, rng.randrange(100, 1500) * 8])
        case = {"op": op, "tokens": min(_log(rng, 1, 131072), MOST_VALUES // (4 * width)), "width": width, "x": rng.choice(two), "out": rng.choice(two), "weight": rng.choice(two), "bias": rng.random() < 0.6}
        case.update({"branch": rng.choice(["", *two])} if op == "norm" else {"stream": rng.random() < 0.5})
        return case
    if op == "rotary":
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256, 2 * rng.randrange(1, 100)])
        heads, rest = rng.randrange(1, 49), rng.choice([0, 0, rng.randrange(1, 9)])
        return {"op": op, "tokens": min(_log(rng, 1, 65536), MOST_VALUES // (2 * dim * (heads + rest))), "heads": heads, "rest": rest, "dim": dim, "turned": dim if rng.random() < 0.6 else 2 * rng.randrange(1, dim // 2 + 1),
                "interleaved": rng.random() < 0.5, "dtype": rng.choice(two), "positions": rng.choice(["int32", "int64"]), "far": _log(rng, 2, 1000000), "factor": rng.choice([1.0, 4.0, 16.0]),
                "inverse": rng.random() < 0.5, "in_place": rng.random() < 0.5}
    while True:
        kv_heads = rng.choice([1, 2, 4, 8, rng.randrange(1, 13)])
        case = {"op": op, "tokens": _log(rng, 1 if op == "attention" else 8, 16384), "kv_heads": kv_heads, "heads": kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8]), "dim": rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 8 * rng.randrange(1, 17)]),
                "causal": rng.random() < 0.75, "window": 0}
        case["tail"] = rng.choice([0, 0, rng.randrange(0, 200)]) if case["tokens"] > 1000 else 0
        case["sequences"] = _log(rng, 1, max(1, min(64, case["tokens"] // 4)))
        if case["causal"] and rng.random() < 0.3:
            case["window"] = _log(rng, 16, 4096)
        longest = max(_lengths(case))
        if case["heads"] * case["sequences"] * longest ** 2 <= MOST_SCORES and _pairs(case) * case["heads"] * case["dim"] <= MOST_PAIRS * 128 and case["tokens"] * case["heads"] * case["dim"] <= MOST_VALUES:
            return case


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _type(name):
    return getattr(torch, name)


def _lengths(case):
    """Lengths of a packed batch: documents differ by factors, now and then one is empty or a single token."""
    n, total = case["sequences"], case["tokens"] - case["tail"]
    rng = random.Random(case["tokens"] * 100 + n)
    share = [math.exp(rng.gauss(0.0, 0.7)) for _ in range(n)]
    lens = [int(total * s / sum(share)) for s in share]
    if n > 4:
        lens[1], lens[3] = min(lens[1], 1), 0
    lens[max(range(n), key=lambda k: lens[k])] += total - sum(lens)
    return lens


def _pairs(case):
    """Pairs of a query and a key that it sees."""
    total = 0
    for n in _lengths(case):
        if not case["causal"]:
            total += n * n
        else:
            w = min(case["window"] or n, n)
            total += w * (w + 1) // 2 + (n - w) * w
    return total


def _prepare_norm(case, seed):
    g = _generator(seed)
    t, h = case["tokens"], case["width"]
    # a stream as trained models have it: rows of different size, a few columns far above the others
    x = torch.randn(t, h, generator=g, device="cuda") * torch.exp(torch.randn(t, 1, generator=g, device="cuda") * 0.5)
    loud = torch.randint(0, h, (max(1, h // 500),), generator=g, device="cuda")
    x[:, loud] = x[:, loud] * 8.0 + 5.0
    s = {"case": case, "x": x.to(_type(case["x"])), "weight": (1.0 + 0.1 * torch.randn(h, generator=g, device="cuda")).to(_type(case["weight"]))}
    s["bias"] = _randn((h,), g, _type(case["weight"]), 0.1) if case["bias"] else None
    if case["op"] == "norm":
        s["branch"] = _randn((t, h), g, _type(case["branch"]), 0.5) if case["branch"] else None
        return s
    s["grad_out"] = _randn((t, h), g, _type(case["out"]), 1e-3)
    s["grad_sum"] = _randn((t, h), g, s["x"].dtype, 1e-3) if case["stream"] else None
    wide = s["x"].float()
    s["mean"] = wide.mean(1)
    s["rstd"] = torch.rsqrt((wide - s["mean"][:, None]).square().mean(1) + EPS)
    s["grad_weight"], s["grad_bias"] = torch.empty_like(s["weight"]), torch.empty_like(s["weight"]) if case["bias"] else None
    if own:
        from paper_2507_20424_b200 import binding
        s["ws"] = binding.alloc_layer_norm_workspace(t, h)
    return s


def _prepare_rotary(case, seed):
    g = _generator(seed)
    rows = _randn((case["tokens"], case["heads"] + case["rest"], case["dim"]), g, _type(case["dtype"]))
    half = case["turned"] // 2
    # a longer context by a larger base: the slowest frequency is divided by the factor, the fastest stays
    base = 10000.0 * case["factor"] ** (half / max(1, half - 1))
    freq = torch.tensor([base ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    start = int(torch.randint(0, case["far"], (1,), generator=g, device="cuda"))
    positions = ((torch.arange(case["tokens"], device="cuda") + start) % case["far"]).to(_type(case["positions"]))
    return {"case": case, "x": rows[:, :case["heads"]], "positions": positions, "freq": freq}


def _prepare_attention(case, seed):
    g = _generator(seed)
    t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    rows = _randn((t, h + 2 * kv, d), g, torch.bfloat16)                 # one product's rows: queries, keys, values
    lens = _lengths(case)
    s = {"case": case, "q": rows[:, :h], "k": rows[:, h:h + kv], "v": rows[:, h + kv:], "longest": max(lens),
         "starts": torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda"), "scale": 1 / math.sqrt(d)}
    if case["op"] == "attention_grad":
        got = _plain_attention(s)
        s["out"], s["lse"] = got["out"], got["lse"]
        s["grad_out"] = _randn((t, h, d), g, torch.bfloat16, 1e-2)
        grads = torch.empty_like(rows)
        s["grad_q"], s["grad_k"], s["grad_v"] = grads[:, :h], grads[:, h:h + kv], grads[:, h + kv:]
    if own:
        from paper_2507_20424_b200 import binding
        s["plan"] = binding.AttentionPlan(s["starts"], t)
        if case["op"] == "attention_grad":
            s["ws"] = binding.alloc_attention_workspace(t, h)
    return s


def prepare(case, seed):
    return {"norm": _prepare_norm, "norm_grad": _prepare_norm, "rotary": _prepare_rotary, "attention": _prepare_attention, "attention_grad": _prepare_attention}[case["op"]](case, seed)


# ---------------------------------------------------------------- plain forms

def _plain_norm(s):
    c, h = s["case"], s["x"]
    if s["branch"] is not None:
        h = (h.float() + s["branch"].float()).to(h.dtype)
    wide = h.float()
    mean = wide.sum(1) / c["width"]
    off = wide - mean[:, None]
    rstd = 1.0 / torch.sqrt((off * off).sum(1) / c["width"] + EPS)
    y = off * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = {"out": y.to(_type(c["out"])), "mean": mean, "rstd": rstd}
    return dict(out, sum=h) if s["branch"] is not None else out


def _plain_norm_grad(s):
    h, dy, r = s["case"]["width"], s["grad_out"].float(), s["rstd"][:, None]
    hat = (s["x"].float() - s["mean"][:, None]) * r
    u = dy * s["weight"].float()
    dx = r * (u - u.sum(1, keepdim=True) / h - hat * ((u * hat).sum(1, keepdim=True) / h))
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].float()
    out = {"x": dx.to(s["x"].dtype), "weight": s["grad_weight"].copy_((dy * hat).sum(0))}
    return dict(out, bias=s["grad_bias"].copy_(dy.sum(0))) if s["grad_bias"] is not None else out


def _plain_rotary(s):
    c, n = s["case"], s["case"]["turned"]
    angle = s["positions"].double()[:, None] * s["freq"]                 # in 64 bits: far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["inverse"]:
        sin = -sin
    x = s["x"].float()
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if c["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if c["interleaved"] else torch.cat(turned, -1)
    out = torch.cat((turned, x[..., n:]), -1)
    return s["x"].copy_(out) if c["in_place"] else out.to(s["x"].dtype)


def _padded(s):
    """Rows of each sequence, padded to the longest: indices [sequences, longest] into the tokens, and which of them are there."""
    starts = s["starts"].long()
    at = starts[:-1, None] + torch.arange(s["longest"], device="cuda")
    there = at < starts[1:, None]
    return at.clamp(max=s["case"]["tokens"] - 1), there


def _scores(s, at, there):
    """Scaled products of queries and keys [sequences, kv heads, heads that share one, longest, longest], -inf where a key is not seen."""
    c = s["case"]
    share = c["heads"] // c["kv_heads"]
    q = s["q"].float()[at].unflatten(2, (c["kv_heads"], share)).permute(0, 2, 3, 1, 4)
    k = s["k"].float()[at].permute(0, 2, 1, 3)[:, :, None]
    seen = there[:, None, :]
    i = torch.arange(s["longest"], device="cuda")
    if c["causal"]:
        seen = seen & (i[None, :] <= i[:, None])
    if c["window"]:
        seen = seen & (i[None, :] > i[:, None] - c["window"])
    return torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen[:, None, None], -math.inf), q, k


def _unpadded(x, at, there, tokens, fill=0.0):
    """[sequences, longest, ...] back to the tokens' rows; rows of no sequence hold `fill`."""
    out = torch.full((tokens, *x.shape[2:]), fill, device="cuda")
    out[at[there]] = x[there]
    return out


def _plain_attention(s):
    c = s["case"]
    at, there = _padded(s)
    z, _, _ = _scores(s, at, there)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v"].float()[at].permute(0, 2, 1, 3)[:, :, None]
    o = torch.matmul(p, v) / total
    lse = (top + torch.log(total))[..., 0]
    o = _unpadded(o.permute(0, 3, 1, 2, 4).flatten(2, 3), at, there, c["tokens"])
    lse = _unpadded(lse.permute(0, 3, 1, 2).flatten(2, 3), at, there, c["tokens"], -math.inf)
    return {"out": o.to(torch.bfloat16), "lse": lse.t().contiguous()}


def _plain_attention_grad(s):
    c = s["case"]
    share = c["heads"] // c["kv_heads"]
    at, there = _padded(s)
    split = lambda x: x[at].unflatten(2, (c["kv_heads"], share)).permute(0, 2, 3, 1, 4)  # noqa: E731
    z, q, k = _scores(s, at, there)
    lse = split(s["lse"].t()[..., None])
    p = z.sub_(lse).exp_()
    p.masked_fill_(~there[:, None, None, :, None], 0.0)                  # queries that are padding
    do = split(s["grad_out"].float())
    v = s["v"].float()[at].permute(0, 2, 1, 3)[:, :, None]
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    delta = (do * split(s["out"].float())).sum(-1, keepdim=True)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(s["scale"])
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q).sum(2)
    back = lambda x: _unpadded(x, at, there, c["tokens"])  # noqa: E731
    return {"q": s["grad_q"].copy_(back(dq.permute(0, 3, 1, 2, 4).flatten(2, 3))), "k": s["grad_k"].copy_(back(dk.transpose(1, 2))), "v": s["grad_v"].copy_(back(dv.transpose(1, 2)))}


def _own_run(s):
    from paper_2507_20424_b200 import binding
    c = s["case"]
    if c["op"] == "norm":
        got = binding.dppf_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, branch=s["branch"], out_dtype=_type(c["out"]))
        out = {"out": got.out, "mean": got.mean, "rstd": got.rstd}
        return dict(out, sum=got.sum) if s["branch"] is not None else out
    if c["op"] == "norm_grad":
        dx = binding.dppf_layer_norm_grad(s["grad_out"], s["x"], s["mean"], s["rstd"], s["weight"], s["grad_weight"], s["grad_bias"], grad_sum=s["grad_sum"], ws=s["ws"])
        out = {"x": dx, "weight": s["grad_weight"]}
        return dict(out, bias=s["grad_bias"]) if s["grad_bias"] is not None else out
    if c["op"] == "rotary":
        return binding.dppf_rotary(s["x"], s["positions"], s["freq"], interleaved=c["interleaved"], inverse=c["inverse"], out=s["x"] if c["in_place"] else None)
    if c["op"] == "attention":
        got = binding.dppf_attention(s["q"], s["k"], s["v"], s["plan"], causal=c["causal"], window=c["window"], scale=s["scale"])
        return {"out": got.out, "lse": got.lse}
    binding.dppf_attention_grad(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["plan"], causal=c["causal"], window=c["window"], scale=s["scale"],
                                grad_q=s["grad_q"], grad_k=s["grad_k"], grad_v=s["grad_v"], ws=s["ws"])
    return {"q": s["grad_q"], "k": s["grad_k"], "v": s["grad_v"]}


def run(state):
    if own:
        return _own_run(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "rotary": _plain_rotary, "attention": _plain_attention, "attention_grad": _plain_attention_grad}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = lambda name: {"float32": 4, "bfloat16": 2, "": 0}[name]  # noqa: E731
    t = case["tokens"]
    if case["op"] == "norm":
        h = case["width"]
        each = size(case["x"]) + size(case["out"]) + (size(case["branch"]) + size(case["x"]) if case["branch"] else 0)
        return {"bytes": t * h * each + 8 * t + h * size(case["weight"]) * (2 if case["bias"] else 1), "flops": 9 * t * h}
    if case["op"] == "norm_grad":
        h = case["width"]
        each = 2 * size(case["x"]) + size(case["out"]) + (size(case["x"]) if case["stream"] else 0)
        return {"bytes": t * h * each + 8 * t + h * size(case["weight"]) * (3 if case["bias"] else 2), "flops": 14 * t * h}
    if case["op"] == "rotary":
        moved = case["turned"] if case["in_place"] else case["dim"]
        return {"bytes": 2 * t * case["heads"] * moved * size(case["dtype"]) + t * (8 if case["positions"] == "int64" else 4), "flops": 3 * t * case["heads"] * case["turned"]}
    row = (2 * case["heads"] + 2 * case["kv_heads"]) * case["dim"] * 2    # q, k, v and out, or their gradients
    pairs = _pairs(case) * case["heads"] * case["dim"]
    if case["op"] == "attention":
        return {"bytes": t * (row + 4 * case["heads"]), "flops": 4 * pairs}
    return {"bytes": t * (2 * row + 4 * case["heads"]), "flops": 10 * pairs}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_norm(case, s):
    h = s["x"] if s["branch"] is None else (s["x"].double() + s["branch"].double()).to(s["x"].dtype)
    var, mean = torch.var_mean(h.double(), 1, correction=0)
    rstd = (var + EPS) ** -0.5
    y = torch.addcmul(torch.zeros((), dtype=torch.float64, device="cuda") if s["bias"] is None else s["bias"].double(), (h.double() - mean[:, None]) * rstd[:, None], s["weight"].double())
    out = {"out": y, "mean": mean, "rstd": rstd}
    return dict(out, sum=h.double()) if s["branch"] is not None else out


def _exact_norm_grad(case, s):
    x, dy, w, mean, r = (s[k].double() for k in ("x", "grad_out", "weight", "mean", "rstd"))
    hat = (x - mean[:, None]) * r[:, None]
    u = dy * w
    a, b = u.mean(1), torch.einsum("th,th->t", u, hat) / case["width"]
    dx = (u - a[:, None] - hat * b[:, None]) * r[:, None]
    if s["grad_sum"] is not None:
        dx += s["grad_sum"].double()
    out = {"x": dx, "weight": torch.einsum("th,th->h", dy, hat)}
    return dict(out, bias=dy.sum(0)) if s["grad_bias"] is not None else out


def _exact_rotary(case, s):
    n, out = case["turned"], s["x"].double().clone()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (-1.0 if case["inverse"] else 1.0) * s["positions"].double()[:, None] * s["freq"])[:, None]
    pairs = out[..., :n].unflatten(-1, (n // 2, 2)) if case["interleaved"] else out[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
    out[..., :n] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
    return out


def _exact_attention(case, s):
    """Sequence by sequence and head by head, some query rows at a time."""
    grad = case["op"] == "attention_grad"
    t, h, share, d = case["tokens"], case["heads"], case["heads"] // case["kv_heads"], case["dim"]
    zeros = lambda n: torch.zeros(t, n, d, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse = zeros(h), torch.full((h, t), -math.inf, dtype=torch.float64, device="cuda")
    got = {"q": zeros(h), "k": zeros(case["kv_heads"]), "v": zeros(case["kv_heads"])}
    starts = s["starts"].tolist()
    for a, e in zip(starts, starts[1:]):
        for r0 in range(a, e, 2048):
            r1 = min(e, r0 + 2048)
            c0 = max(a, r0 - case["window"] + 1) if case["window"] else a
            c1 = r1 if case["causal"] else e
            gap = torch.arange(r0, r1, device="cuda")[:, None] - torch.arange(c0, c1, device="cuda")
            hidden = (gap < 0) if case["causal"] else torch.zeros_like(gap, dtype=torch.bool)
            if case["window"]:
                hidden |= gap >= case["window"]
            for j in range(case["kv_heads"]):
                k, v = s["k"][c0:c1, j].double(), s["v"][c0:c1, j].double()
                for i in range(j * share, (j + 1) * share):
                    q = s["q"][r0:r1, i].double()
                    z = (q @ k.t() * s["scale"]).masked_fill(hidden, -math.inf)
                    if not grad:
                        lse[i, r0:r1] = torch.logsumexp(z, 1)
                        out[r0:r1, i] = torch.softmax(z, 1) @ v
                        continue
                    p, do = torch.exp(z - s["lse"][i, r0:r1, None].double()), s["grad_out"][r0:r1, i].double()
                    got["v"][c0:c1, j] += p.t() @ do
                    ds = p * (do @ v.t() - (do * s["out"][r0:r1, i].double()).sum(1, keepdim=True)) * s["scale"]
                    got["q"][r0:r1, i] += ds @ k
                    got["k"][c0:c1, j] += ds.t() @ q
    return got if grad else {"out": out, "lse": lse}


def exact(case, seed):
    """The same outputs from the definitions, in fp64, on the inputs that prepare() makes."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "rotary": _exact_rotary, "attention": _exact_attention, "attention_grad": _exact_attention}[case["op"]](case, s)
