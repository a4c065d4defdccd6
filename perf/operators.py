"""The operators of a language-model worker's local step, as measured workloads.

Three operators, each in its plain form (elementary torch operations in 32 bits) and, where ``own``
is true, as the calls a user makes of this package:

  embedding   rows of a table times a scale, and the table's gradient (sums over equal ids)
  policy      clipped policy loss with a KL term from logits: loss, log-probabilities, gradient
  adamw       one AdamW step over the many tensors of a model, states in 32 bits or in 8

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes what a program
holds before the call, ``run`` is one pass, ``work`` what a pass cannot do without, ``exact`` the
same outputs in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 256          # elements that share a scale in the 8-bit states
TOP = 448.0          # largest finite e4m3 value
TINY = 2.0 ** -126   # scales below the smallest normal fp32 number are taken as zero
BETA1, BETA2 = float(np.float32(0.9)), float(np.float32(0.999))
LR, EPS, DECAY = float(np.float32(5e-4)), float(np.float32(1e-8)), float(np.float32(0.01))
MOST_VALUES = 1 << 28   # largest count of logits, table entries or looked-up values of a drawn case


def listed():
    return [
        # A handful of new tokens of a decoding batch: latency alone.
        {"name": "lookup-decode", "op": "lookup", "tokens": 7, "vocab": 32000, "width": 512, "table": "bfloat16", "out": "bfloat16", "ids": "int64", "scale": 22.627417, "pad": 0.0},
        # The first layer of a training batch, fp32 master table, activations in bf16, some padding.
        {"name": "lookup-batch", "op": "lookup", "tokens": 16384, "vocab": 50000, "width": 1024, "table": "float32", "out": "bfloat16", "ids": "int64", "scale": 32.0, "pad": 0.1},
        # Its gradient over a short batch, written whole.
        {"name": "grad-short", "op": "lookup_grad", "tokens": 333, "vocab": 1009, "width": 257, "table": "float32", "out": "float32", "ids": "int32", "scale": 1.0, "pad": 0.0, "add": False},
        # The ordinary gradient: a fresh fp32 gradient of the table, bf16 activations.
        {"name": "grad-batch", "op": "lookup_grad", "tokens": 16384, "vocab": 50000, "width": 1024, "table": "float32", "out": "bfloat16", "ids": "int64", "scale": 32.0, "pad": 0.1, "add": False},
        # A long batch added to a gradient that is there already (tied to the last layer, or accumulated).
        {"name": "grad-long-add", "op": "lookup_grad", "tokens": 100003, "vocab": 131072, "width": 2048, "table": "float32", "out": "bfloat16", "ids": "int64", "scale": 1.0, "pad": 0.05, "add": True},
        # Few tokens: the vocabulary has to be split to fill the GPU.
        {"name": "policy-few", "op": "policy", "tokens": 9, "vocab": 32000, "stride": 32000, "dtype": "bfloat16", "masked": 0.0, "kl": True, "backward": True},
        # A micro batch with its prompt masked, odd vocabulary in rows of odd length.
        {"name": "policy-odd", "op": "policy", "tokens": 1500, "vocab": 50333, "stride": 50333, "dtype": "bfloat16", "masked": 0.4, "kl": True, "backward": True},
        # The ordinary large micro batch.
        {"name": "policy-batch", "op": "policy", "tokens": 4096, "vocab": 131072, "stride": 131072, "dtype": "bfloat16", "masked": 0.25, "kl": True, "backward": True},
        # Log-probabilities and loss alone (no gradient) of fp32 logits with a padded row.
        {"name": "policy-forward32", "op": "policy", "tokens": 2048, "vocab": 65537, "stride": 65600, "dtype": "float32", "masked": 0.3, "kl": False, "backward": False},
        # A small head or adapter: some twenty tensors, latency alone.
        {"name": "adamw-small", "op": "adamw", "bits": 32, "param": "float32", "grad": "float32", "total": 60011, "tensors": 20, "packed": True, "step": 3},
        # A worker of ViT-B/16 size (86,567,656 parameters) in its packed fp32 row.
        {"name": "adamw-row32", "op": "adamw", "bits": 32, "param": "float32", "grad": "float32", "total": 86567656, "tensors": 152, "packed": True, "step": 100},
        # A larger model in bf16 with 8-bit states.
        {"name": "adamw-bf16-8", "op": "adamw", "bits": 8, "param": "bfloat16", "grad": "bfloat16", "total": 300000037, "tensors": 290, "packed": False, "step": 1000},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _vocab(rng):
    v = _log(rng, 250, 260000)
    return v if rng.random() < 0.5 else max(256, v // 256 * 256)


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "policy", "adamw"])
    if op in ("lookup", "lookup_grad"):
        width = rng.choice([64, 128, 200, 256, 512, 768, 1000, 1024, 1536, 2048, 4096, 5120, 8192, rng.randrange(1, 700), rng.randrange(1, 700) * 2])
        vocab = min(_vocab(rng), MOST_VALUES // width)
        case = {"op": op, "tokens": min(_log(rng, 1, 131072), MOST_VALUES // (2 * width)), "vocab": vocab, "width": width,
                "table": rng.choice(["float32", "bfloat16"]), "out": rng.choice(["float32", "bfloat16"]), "ids": rng.choice(["int32", "int64"]),
                "scale": rng.choice([1.0, round(math.sqrt(width), 3)]), "pad": rng.choice([0.0, round(rng.uniform(0, 0.5), 2)])}
        if op == "lookup_grad":
            case["add"] = rng.random() < 0.5
        return case
    if op == "policy":
        vocab = _vocab(rng)
        tokens = _log(rng, 1, min(16384, MOST_VALUES // vocab))
        return {"op": op, "tokens": tokens, "vocab": vocab, "stride": vocab + rng.choice([0, 0, 8, rng.randrange(0, 100)]), "dtype": rng.choice(["bfloat16", "bfloat16", "float32"]),
                "masked": rng.choice([0.0, round(rng.uniform(0, 0.8), 2)]), "kl": rng.random() < 0.7, "backward": rng.random() < 0.75}
    total = _log(rng, 1000, 250_000_000)
    bits = rng.choice([8, 32])
    return {"op": op, "bits": bits, "param": rng.choice(["float32", "bfloat16"]), "grad": rng.choice(["float32", "bfloat16"]), "total": total,
            "tensors": max(1, min(total // 50, _log(rng, 1, 700))), "packed": rng.random() < 0.5, "step": _log(rng, 1, 100000)}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _token_ids(case, g):
    """Ids as text has them: a few very frequent, most rare (the logarithm of the rank is uniform); -1 where there is padding."""
    u = torch.rand(case["tokens"], generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp(0, case["vocab"] - 1)
    ids[torch.rand(case["tokens"], generator=g, device="cuda") < case["pad"]] = -1
    return ids.to(getattr(torch, case["ids"]))


def _distinct(case):
    """Expected number of distinct ids among the tokens."""
    v = np.arange(case["vocab"], dtype=np.float64)
    p = np.log1p(1.0 / (v + 1)) / math.log(case["vocab"] + 1) * (1 - case["pad"])
    return float(np.sum(-np.expm1(case["tokens"] * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def _sizes(case):
    """Element counts of the tensors of a model: many small ones (norms, biases), some large matrices; their sum is the case's total."""
    rng = random.Random(case["total"] * 1000 + case["tensors"])
    n, total = case["tensors"], case["total"]
    share = [math.exp(rng.gauss(0.0, 0.6)) * (1.0 if k % 3 else 0.001) for k in range(n)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    at = max(range(n), key=lambda k: sizes[k])
    sizes[at] += total - sum(sizes)
    return sizes


def _randn(n, g, std, dtype=torch.float32):
    """Normal values, a stretch at a time, rounded to the type."""
    out = torch.empty(n, dtype=dtype, device="cuda")
    for a in range(0, n, 1 << 26):
        out[a:a + (1 << 26)] = torch.randn(min(1 << 26, n - a), generator=g, device="cuda") * std
    return out


def _prepare_adamw(case, seed):
    g = _generator(seed)
    sizes = _sizes(case)
    align = 1 if case["packed"] else BLOCK                       # tensors back to back in a row, or each at a boundary of its own
    starts, slots, at, slot = [], [], 0, 0
    for n in sizes:
        starts.append(at)
        slots.append(slot)
        at += -(-n // align) * align
        slot += -(-n // BLOCK) * BLOCK
    sizes_t = torch.tensor(sizes, device="cuda")
    inside = torch.arange(sum(sizes), device="cuda") - (sizes_t.cumsum(0) - sizes_t).repeat_interleave(sizes_t)   # index within its tensor
    place = inside + torch.tensor(starts, device="cuda").repeat_interleave(sizes_t)                               # in the rows of parameters and gradients
    param = torch.zeros(at, dtype=getattr(torch, case["param"]), device="cuda")
    grad = torch.zeros(at, dtype=getattr(torch, case["grad"]), device="cuda")
    param[place] = _randn(len(place), g, 0.02, param.dtype)
    # gradients differ in size from tensor to tensor by orders of magnitude
    size = torch.exp(torch.randn(len(sizes), generator=g, device="cuda") * 1.5) * 1e-3
    grad[place] = (_randn(len(place), g, 1.0) * size.repeat_interleave(sizes_t)).to(grad.dtype)
    decays = [0.0 if n < 1000 else 1.0 for n in sizes]           # none for norms and biases
    state = {"case": case, "param": param, "grad": grad, "clip": torch.tensor([0.75], device="cuda"), "seed": case["step"]}
    if case["packed"]:
        state["decay"] = torch.zeros(at, device="cuda")
        state["decay"][place] = torch.tensor(decays, device="cuda").repeat_interleave(sizes_t)
    else:
        state["decay"] = torch.tensor(decays, device="cuda").repeat_interleave((sizes_t + align - 1) // align)[:, None]
    each = size.repeat_interleave(sizes_t)
    if case["bits"] == 32:
        m, v = torch.zeros(at, device="cuda"), torch.zeros(at, device="cuda")
        m[place] = _randn(len(place), g, 0.3) * each
        v[place] = (_randn(len(place), g, 0.5) * each).square() + 0.25 * each.square()
        state.update(m=m, v=v)
    else:
        sits = inside + torch.tensor(slots, device="cuda").repeat_interleave(sizes_t)                             # in the rows of the states
        blocks = torch.tensor([-(-n // BLOCK) for n in sizes], device="cuda")
        scale = size.repeat_interleave(blocks) / TOP
        mc, sc = torch.zeros(slot, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(slot, dtype=torch.float8_e4m3fn, device="cuda")
        mc.view(torch.int8)[sits] = (_randn(len(sits), g, 0.3 * TOP).clamp(-TOP, TOP)).to(torch.float8_e4m3fn).view(torch.int8)
        sc.view(torch.int8)[sits] = (_randn(len(sits), g, 0.3 * TOP).abs().clamp(0.01 * TOP, TOP)).to(torch.float8_e4m3fn).view(torch.int8)
        state.update(m=mc, s=sc, m_scale=scale * 0.7, s_scale=scale.clone())
        inner = torch.zeros(slot, dtype=torch.int32, device="cuda")
        inner[sits] = inside.to(torch.int32)
        state["inside"] = inner
        if case["packed"]:
            state["sits"], state["decay_slots"] = sits, torch.tensor(decays, device="cuda").repeat_interleave(blocks)[:, None]
        else:
            state["decay_slots"] = torch.tensor(decays, device="cuda").repeat_interleave(blocks)[:, None]
    if own:
        from paper_2507_20424_b200 import binding
        cut = lambda row, first: [row[a:a + n] for a, n in zip(first, sizes)]  # noqa: E731
        if case["bits"] == 32:
            more = {"exp_avgs": cut(state["m"], starts), "exp_avg_sqs": cut(state["v"], starts)}
        else:
            cut_b = lambda row: [row[a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in zip(slots, sizes)]  # noqa: E731
            more = {"exp_avgs": cut(state["m"], slots), "exp_avg_sqs": cut(state["s"], slots),
                    "exp_avg_scales": cut_b(state["m_scale"]), "exp_avg_sq_scales": cut_b(state["s_scale"])}
        state["tensors"] = binding.AdamWTensors(cut(param, starts), cut(grad, starts), state_bits=case["bits"], decay=decays, **more)
    return state


def _logits(case, g):
    """Logits of a trained model: wide noise and, on most rows, a few tokens far above it."""
    t, v = case["tokens"], case["vocab"]
    whole = torch.zeros(t, case["stride"], dtype=getattr(torch, case["dtype"]), device="cuda")
    target = torch.randint(0, v, (t,), generator=g, device="cuda")
    step = max(1, (1 << 26) // case["stride"])
    for a in range(0, t, step):
        z = torch.randn(min(step, t - a), v, generator=g, device="cuda") * 2.0
        up = 4.0 + 8.0 * torch.rand(len(z), 1, generator=g, device="cuda")
        z.scatter_add_(1, target[a:a + step, None], up)
        whole[a:a + step, :v] = z
    return whole[:, :v], target


def _prepare_policy(case, seed):
    g = _generator(seed)
    logits, target = _logits(case, g)
    t = case["tokens"]
    # the policy that sampled: some updates ago. Ratios are kept 1e-3 away from the clip's edges, so that no row hangs on a rounding.
    lp = torch.empty(t, device="cuda")
    step = max(1, (1 << 26) // case["vocab"])
    for a in range(0, t, step):
        z = logits[a:a + step].float() / 0.9
        lp[a:a + step] = z.gather(1, target[a:a + step, None])[:, 0] - torch.logsumexp(z, 1)
    drift = torch.randn(t, generator=g, device="cuda") * 0.15
    for edge in (math.log(0.8), math.log(1.28)):
        drift = torch.where((drift - edge).abs() < 1e-3, drift + 4e-3, drift)
    weights = (torch.rand(t, generator=g, device="cuda") >= case["masked"]).float()
    target = torch.where(weights > 0, target, torch.full_like(target, -100))
    state = {"case": case, "logits": logits, "target": target, "old": lp - drift, "ref": lp + torch.randn(t, generator=g, device="cuda") * 0.3 if case["kl"] else None,
             "advantage": torch.randn(t, generator=g, device="cuda") + 0.3, "weight": weights / weights.sum().clamp(min=1)}
    if case["backward"]:
        state["grad"] = torch.empty(t, case["stride"], dtype=logits.dtype, device="cuda")[:, :case["vocab"]]
    if own:
        from paper_2507_20424_b200 import binding
        state["ws"] = binding.alloc_policy_workspace(t)
    return state


def prepare(case, seed):
    if case["op"] == "adamw":
        return _prepare_adamw(case, seed)
    if case["op"] == "policy":
        return _prepare_policy(case, seed)
    g = _generator(seed)
    state = {"case": case, "ids": _token_ids(case, g)}
    t, v, h = case["tokens"], case["vocab"], case["width"]
    if case["op"] == "lookup":
        state["table"] = _randn(v * h, g, 0.02, getattr(torch, case["table"])).view(v, h)
        return state
    state["grad_out"] = _randn(t * h, g, 1e-3, getattr(torch, case["out"])).view(t, h)
    if case["add"]:
        state["grad_table"] = _randn(v * h, g, 1e-3, getattr(torch, case["table"])).view(v, h)
    else:
        state["grad_table"] = torch.empty(v, h, dtype=getattr(torch, case["table"]), device="cuda")
    if own:
        from paper_2507_20424_b200 import binding
        state["ws"] = binding.alloc_embedding_workspace(t, h)
    return state


# ---------------------------------------------------------------- plain forms

def _plain_lookup(s):
    c, ids = s["case"], s["ids"].long()
    rows = s["table"][ids.clamp(min=0)].float() * c["scale"]
    return torch.where((ids >= 0)[:, None], rows, 0.0).to(getattr(torch, c["out"]))


def _plain_lookup_grad(s):
    c, ids, table = s["case"], s["ids"].long(), s["grad_table"]
    rows = torch.where((ids >= 0)[:, None], s["grad_out"].float() * c["scale"], 0.0)
    if c["add"] and table.dtype == torch.float32:
        return table.index_add_(0, ids.clamp(min=0), rows)
    total = torch.zeros(table.shape, device="cuda").index_add_(0, ids.clamp(min=0), rows)
    return table.copy_(table.float() + total if c["add"] else total)


def _plain_policy(s):
    c, y = s["case"], s["target"].clamp(min=0)[:, None]
    live = s["weight"] > 0
    z = s["logits"].float() * (1 / 0.9)
    top = z.amax(1, keepdim=True)
    picked = z.gather(1, y)[:, 0] - top[:, 0]
    e = torch.exp_(z.sub_(top))
    total = e.sum(1)
    lp = picked - torch.log(total)
    ratio, a = torch.exp(lp - s["old"]), s["advantage"]
    clipped = ((a > 0) & (ratio > 1.28)) | ((a < 0) & (ratio < 0.8))
    loss = torch.where(a == 0, 0.0, -torch.minimum(ratio * a, ratio.clamp(0.8, 1.28) * a))
    slope = torch.where(clipped, 0.0, -ratio * a)
    kl = torch.zeros_like(lp)
    if c["kl"]:
        gap = s["ref"] - lp
        kl = torch.exp(gap) - gap - 1
        loss, slope = loss + 0.04 * kl, slope + 0.04 * (1 - torch.exp(gap))
    each = lambda x: torch.where(live, s["weight"] * x, 0.0)  # noqa: E731
    out = {"loss": each(loss).sum(), "kl": each(kl).sum(), "clipped": each(clipped.float()).sum(), "logp": torch.where(live, lp, 0.0)}
    if c["backward"]:
        slope = each(slope) / 0.9
        e.mul_((-slope / total)[:, None]).scatter_add_(1, y, slope[:, None])
        out["grad"] = s["grad"].copy_(torch.where(live[:, None], e, 0.0))
    return out


def _adamw_numbers(case):
    t = case["step"]
    return LR / (1 - BETA1 ** t), 1 / math.sqrt(1 - BETA2 ** t)


def _plain_adamw32(s):
    size, root = _adamw_numbers(s["case"])
    g = s["grad"].float() * s["clip"]
    m = s["m"].mul_(BETA1).add_(g * (1 - BETA1))
    v = s["v"].mul_(BETA2).add_(g * g * (1 - BETA2))
    p = s["param"].float().view(s["decay"].shape[0], -1) * (1 - LR * DECAY * s["decay"].view(s["decay"].shape[0], -1))
    s["param"].copy_(p.view(-1) - size * m / (torch.sqrt(v) * root + EPS))
    return {"param": s["param"], "m": m, "v": v}


def _hash_bits(inside, seed):
    """20 bits for each element: half a 32-bit hash (the finalizer of MurmurHash3) of the pair's number and the seed, shifted."""
    h = ((inside.long() >> 1) + seed * 0x9E3779B9) & 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    h = h ^ (h >> 16)
    return (((h >> ((inside & 1) * 16)) & 0xFFFF) << 4).int()


def _scales(x):
    scale = x.abs().amax(1, keepdim=True) * (1 / TOP)
    scale = torch.where(scale < TINY, 0.0, scale)
    return scale, torch.where(scale == 0, 0.0, 1 / scale)


def _plain_adamw8(s):
    size, root = _adamw_numbers(s["case"])
    packed = s["case"]["packed"]
    lay = lambda row: torch.zeros(len(s["inside"]), device="cuda").index_copy_(0, s["sits"], row.float()) if packed else row.float()  # noqa: E731
    g = (lay(s["grad"]) * s["clip"]).view(-1, BLOCK)
    m = s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]
    v = (s["s"].float().view(-1, BLOCK) * s["s_scale"][:, None]).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    root_v = torch.sqrt(v)
    p = lay(s["param"]).view(-1, BLOCK) * (1 - LR * DECAY * s["decay_slots"]) - size * m / (root_v * root + EPS)
    s["param"].copy_(p.view(-1)[s["sits"]] if packed else p.view(-1))
    scale, over = _scales(m)
    s["m"].copy_((m * over).view(-1).to(torch.float8_e4m3fn))
    s["m_scale"].copy_(scale[:, 0])
    scale, over = _scales(root_v)
    # rounded at random: an e4m3 number's bits are an fp32 number's from bit 20 on, once 2^-120 has matched the exponents
    bits = (root_v * over * 2.0 ** -120).view(torch.int32).view(-1)
    code = ((bits + _hash_bits(s["inside"], s["seed"])) >> 20).clamp(max=0x7E)
    code = torch.where((root_v.view(-1) > 0) & (over > 0).expand(-1, BLOCK).reshape(-1), code.clamp(min=1), code)
    s["s"].view(torch.uint8).copy_(code.to(torch.uint8))
    s["s_scale"].copy_(scale[:, 0])
    return {"param": s["param"], "m": s["m"], "m_scale": s["m_scale"], "s": s["s"], "s_scale": s["s_scale"]}


def _own_run(s):
    from paper_2507_20424_b200 import binding
    c = s["case"]
    if c["op"] == "lookup":
        return binding.dppf_embedding(s["table"], s["ids"], scale=c["scale"], out_dtype=getattr(torch, c["out"]))
    if c["op"] == "lookup_grad":
        binding.dppf_embedding_grad(s["grad_out"], s["ids"], s["grad_table"], scale=c["scale"], accumulate=c["add"], ws=s["ws"])
        return s["grad_table"]
    if c["op"] == "policy":
        out = binding.dppf_policy_loss(s["logits"], s["target"], s["old"], s["advantage"], s["weight"], ref_logp=s["ref"], clip_low=0.2, clip_high=0.28,
                                       kl_coef=0.04 if c["kl"] else 0.0, temperature=0.9, grad_logits=s.get("grad"), ws=s["ws"])
        got = {"loss": out.loss, "kl": out.kl, "clipped": out.clipped, "logp": out.logp}
        return dict(got, grad=s["grad"]) if c["backward"] else got
    binding.dppf_adamw_tensors(s["tensors"], LR, BETA1, BETA2, EPS, DECAY, c["step"], grad_scale=s["clip"], seed=s["seed"])
    return {k: s[k] for k in (("param", "m", "v") if c["bits"] == 32 else ("param", "m", "m_scale", "s", "s_scale"))}


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "adamw":
        return _plain_adamw32(state) if state["case"]["bits"] == 32 else _plain_adamw8(state)
    return {"lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "policy": _plain_policy}[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = lambda name: 4 if name == "float32" else 2  # noqa: E731
    if case["op"] == "adamw":
        n = case["total"]
        states = 16 * n if case["bits"] == 32 else 4 * n + 16 * n / BLOCK
        return {"bytes": n * (2 * size(case["param"]) + size(case["grad"])) + states, "flops": 14 * n}
    t = case["tokens"]
    if case["op"] == "policy":
        live = max(1.0, t * (1 - case["masked"]))
        b = live * case["vocab"] * size(case["dtype"]) + (t * case["vocab"] * size(case["dtype"]) if case["backward"] else 0)
        return {"bytes": b + 36 * t, "flops": live * case["vocab"] * (6 if case["backward"] else 4)}
    h, ids = case["width"], t * (8 if case["ids"] == "int64" else 4)
    unique, live = _distinct(case), t * (1 - case["pad"])
    if case["op"] == "lookup":
        return {"bytes": ids + unique * h * size(case["table"]) + t * h * size(case["out"]), "flops": live * h}
    rows = 2 * unique if case["add"] else case["vocab"]
    return {"bytes": ids + live * h * size(case["out"]) + rows * h * size(case["table"]), "flops": live * h}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_lookup(case, s):
    ids = s["ids"].long()
    out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
    out[ids >= 0] = s["table"][ids[ids >= 0]].double() * case["scale"]
    return out


def _exact_lookup_grad(case, s):
    ids = s["ids"].long()
    out = s["grad_table"].double() if case["add"] else torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    return out.index_add_(0, ids[ids >= 0], s["grad_out"][ids >= 0].double() * case["scale"])


def _exact_policy(case, s):
    t, v = case["tokens"], case["vocab"]
    out = {k: torch.zeros((), dtype=torch.float64, device="cuda") for k in ("loss", "kl", "clipped")}
    out["logp"] = torch.zeros(t, dtype=torch.float64, device="cuda")
    if case["backward"]:
        out["grad"] = torch.zeros(t, v, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // v)
    rows = torch.nonzero(s["weight"] > 0)[:, 0]
    for at in range(0, len(rows), step):
        r = rows[at:at + step]
        w, adv, y = s["weight"][r].double(), s["advantage"][r].double(), s["target"][r]
        logp = torch.log_softmax(s["logits"][r].double() / 0.9, 1)
        lp = logp.gather(1, y[:, None])[:, 0]
        q = torch.exp(lp - s["old"][r].double())
        inside = torch.where(adv > 0, q <= 1.28, torch.where(adv < 0, q >= 0.8, True))
        each = torch.where(inside, -q * adv, -q.clamp(0.8, 1.28) * adv)
        slope = torch.where(inside, -q * adv, 0.0)
        if case["kl"]:
            gap = s["ref"][r].double() - lp
            out["kl"] += (w * (torch.expm1(gap) - gap)).sum()
            each, slope = each + 0.04 * (torch.expm1(gap) - gap), slope - 0.04 * torch.expm1(gap)
        out["loss"] += (w * each).sum()
        out["clipped"] += w[~inside].sum()
        out["logp"][r] = lp
        if case["backward"]:
            probs = torch.exp(logp)
            d = torch.zeros_like(probs).scatter_(1, y[:, None], 1.0) - probs
            out["grad"][r] = d * (w * slope / 0.9)[:, None]
    return out


def _exact_adamw(case, s):
    t, b1, b2 = case["step"], BETA1, BETA2
    row = lambda x: x.double()  # noqa: E731
    if case["bits"] == 8 and case["packed"]:
        row = lambda x: torch.zeros(len(s["inside"]), dtype=torch.float64, device="cuda").index_copy_(0, s["sits"], x.double())  # noqa: E731
    g = row(s["grad"]) * s["clip"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = (s["m"].double().view(-1, BLOCK) * s["m_scale"].double()[:, None]).view(-1)
        v = (s["s"].double().view(-1, BLOCK) * s["s_scale"].double()[:, None]).square().view(-1)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    decay = s["decay"] if case["bits"] == 32 else s["decay_slots"]
    p = row(s["param"])
    p = (p.view(decay.shape[0], -1) * (1 - LR * DECAY * decay.double().view(decay.shape[0], -1))).view(-1)
    p = p - LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + EPS)
    if case["bits"] == 32:
        return {"param": p, "m": m, "v": v}
    out = {"param": p[s["sits"]] if case["packed"] else p}
    for name, x in (("m", m.view(-1, BLOCK)), ("s", torch.sqrt(v).view(-1, BLOCK))):
        scale = x.abs().amax(1) / TOP
        y = torch.where(scale[:, None] > 0, x / scale[:, None], 0.0)
        ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)     # spacing of e4m3 at y
        if name == "m":
            y = torch.round(y / ulp) * ulp
        else:
            n = s["inside"].cpu().numpy().astype(np.uint32)                             # the hash again, in wrapping 32-bit arithmetic
            k = (n >> np.uint32(1)) + np.uint32(s["seed"] * 0x9E3779B9 & 0xFFFFFFFF)
            k = (k ^ (k >> np.uint32(16))) * np.uint32(0x85EBCA6B)
            k = (k ^ (k >> np.uint32(13))) * np.uint32(0xC2B2AE35)
            k ^= k >> np.uint32(16)
            k = np.where(n & np.uint32(1), k >> np.uint32(16), k & np.uint32(0xFFFF))
            u = torch.from_numpy(k.astype(np.int32)).to("cuda").view(-1, BLOCK).double() / 65536
            q = torch.floor(y / ulp + u) * ulp
            y = torch.where(y > 0, q.clamp(2.0 ** -9, TOP), 0.0)
        out[name], out[name + "_scale"] = y.view(-1), scale
    return out


def exact(case, seed):
    """The same outputs from the definitions, in fp64, on the inputs that prepare() makes."""
    s = prepare(case, seed)
    return {"lookup": _exact_lookup, "lookup_grad": _exact_lookup_grad, "policy": _exact_policy, "adamw": _exact_adamw}[case["op"]](case, s)
