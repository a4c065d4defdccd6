"""Plain implementations in 64 bits of the operators of a language-model worker's local step."""
import numpy as np
import torch


def policy(logits, targets, old, adv, weight, ref=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, temperature=1.0):
    """(sums [3], logp [T], slope [T] = weight * dL/dlp, grad [T, V]) in fp64 on the CPU."""
    x = logits.detach().cpu().double()
    T, V = x.shape
    y, w = targets.cpu().long(), weight.cpu().double()
    live = (w != 0) & (y >= 0) & (y < V)
    old, adv = old.cpu().double(), adv.cpu().double()
    logp, grad, slope, sums = torch.zeros(T).double(), torch.zeros(T, V).double(), torch.zeros(T).double(), torch.zeros(3).double()
    for t in torch.nonzero(live)[:, 0].tolist():
        z = (x[t] - x[t].max()) / temperature              # differences first: at the type's lowest value log V would be rounded away
        lse = torch.logsumexp(z, 0)
        lp = z[y[t]] - lse
        q = torch.exp(lp - old[t])
        a = adv[t]
        clipped = bool((a > 0 and q > 1 + clip_high) or (a < 0 and q < 1 - clip_low))
        loss = torch.zeros(()).double() if a == 0 else -torch.minimum(q * a, q.clamp(1 - clip_low, 1 + clip_high) * a)
        s = 0.0 if clipped or a == 0 else -q * a
        if ref is not None:
            gap = ref[t].cpu().double() - lp
            k = torch.expm1(gap) - gap
            sums[1] += w[t] * k
            loss = loss + kl_coef * k
            s = s - kl_coef * torch.expm1(gap)
        sums[0] += w[t] * loss
        sums[2] += w[t] * clipped
        logp[t], slope[t] = lp, w[t] * s
        p = torch.exp(z - lse)
        grad[t] = -p * slope[t] / temperature
        grad[t, y[t]] += slope[t] / temperature
    return sums, logp, slope, grad


def embedding_grad(grad_out, ids, shape, scale, start=None):
    """(gradient, sum of magnitudes, count per row) in fp64."""
    ids = ids.cpu().long().reshape(-1)
    g = grad_out.detach().cpu().double().reshape(len(ids), shape[1]) * scale
    ok = (ids >= 0) & (ids < shape[0])
    out, mags = torch.zeros(shape).double(), torch.zeros(shape).double()
    out.index_add_(0, ids[ok], g[ok])
    mags.index_add_(0, ids[ok], g[ok].abs())
    if start is not None:
        out += start.cpu().double()
        mags += start.cpu().double().abs()
    return out, mags, torch.bincount(ids[ok], minlength=shape[0])


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step):
    """One AdamW step in fp64 (scalars as the fp32 numbers that the library receives)."""
    lr, beta1, beta2, eps, weight_decay = (float(np.float32(s)) for s in (lr, beta1, beta2, eps, weight_decay))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v


# ---- states in 8 bits: e4m3 codes with one scale per 256 elements

E4M3 = np.array([(-1.0 if c & 0x80 else 1.0) * ((c & 7) * 2.0 ** -9 if not c & 0x78 else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7)) for c in range(256)])


def blocks_of(x):
    """x padded with zeros to whole blocks, as [blocks, 256]."""
    n = -(-len(x) // 256) * 256
    return np.concatenate([x, np.zeros(n - len(x), x.dtype)]).reshape(-1, 256)


def decode(codes, scales, n):
    return (E4M3[blocks_of(codes)] * scales.astype(np.float64)[:, None]).reshape(-1)[:n]


def spacing(y):
    """Distance between neighbouring e4m3 magnitudes at y (in units of the scale)."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)


def random_bits(n, seed):
    """The 20 bits added below the kept ones when element i's root is rounded."""
    i = np.arange(n, dtype=np.uint64)
    h = ((i >> np.uint64(1)) + np.uint64((seed * 0x9E3779B9) & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x85EBCA6B)) & np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(13))) * np.uint64(0xC2B2AE35)) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(16)
    return np.where(i & np.uint64(1), h >> np.uint64(16), h & np.uint64(0xFFFF)).astype(np.uint32) << np.uint32(4)


def adamw8_states(g, mc, rc, ms, rs, beta1, beta2, seed):
    """New codes and scales in separately rounded fp32 operations: what the kernel has to give bit for bit."""
    f = np.float32
    b1, b2 = f(beta1), f(beta2)
    o1, o2 = f(1 - float(b1)), f(1 - float(b2))
    n = len(g)
    g = blocks_of(g.astype(f))
    m = blocks_of(E4M3[mc].astype(f)) * ms[:, None] * b1 + g * o1
    root = blocks_of(E4M3[rc].astype(f)) * rs[:, None]
    r = np.sqrt(root * root * b2 + g * g * o2)
    out = []
    for x in (m, r):
        scale = np.abs(x).max(1) * f(1 / 448)
        scale = np.where(scale < f(2.0 ** -126), f(0), scale)
        with np.errstate(divide="ignore"):
            over = np.where(scale == 0, f(0), f(1) / scale)
        out.append((x * over[:, None], scale))
    y, m_scale = out[0]
    m_codes = torch.from_numpy(y.reshape(-1)[:n].copy()).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    y, r_scale = out[1]
    y = y.reshape(-1)[:n].copy()
    codes = np.minimum(((y * f(2.0 ** -120)).view(np.uint32) + random_bits(n, seed)) >> np.uint32(20), np.uint32(0x7E))
    codes = np.where(y > 0, np.maximum(codes, 1), codes).astype(np.uint8)
    return m_codes, m_scale, codes, r_scale
