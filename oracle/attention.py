"""Plain 64-bit definitions of the attention half: projection with adapters, rotary positions, the paged cache, attention
of drafted tokens.  Loops over tokens and heads, CPU tensors in, float64 out.  Test infrastructure only."""
import math

import torch

PAGE = 64
TOP = {"int8": 127.0, "fp8": 448.0}


def project(X, aid, W, A, B, scale):
    X, W, A, B = X.double(), W.double(), A.double(), B.double()
    Y = X @ W
    for t, a in enumerate(aid.tolist()):
        if 0 <= a < len(A):
            Y[t] += float(scale[a]) * ((X[t] @ A[a]) @ B[a])
    return Y


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0):
    """(radians per position of every pair, magnitude)"""
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    magnitude = 1.0
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "ramp":
        def pair_of(turns):
            return rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
        mix = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3))) for i in range(rot // 2)]
        f = [x * (1 - w) + x / factor * w for x, w in zip(f, mix)]
        magnitude = 0.1 * math.log(factor) + 1.0
    elif scaling == "bands":
        keep = [min(1.0, max(0.0, (original * x / (2 * math.pi) - 1.0) / 3.0)) for x in f]
        f = [x * k + x / factor * (1 - k) for x, k in zip(f, keep)]
    return f, magnitude


def rotary(X, pos, freqs, magnitude, rot, layout, transpose=False):
    Y = X.double().clone()
    for t, p in enumerate(pos.tolist()):
        for i, f in enumerate(freqs):
            a, b = (i, i + rot // 2) if layout == "halves" else (2 * i, 2 * i + 1)
            c, s = math.cos(p * f), math.sin(p * f) * (-1.0 if transpose else 1.0)
            x, y = Y[t, :, a].clone(), Y[t, :, b].clone()
            Y[t, :, a] = magnitude * (x * c - y * s)
            Y[t, :, b] = magnitude * (x * s + y * c)
    return Y


def kept(x, format):
    """What a head [..., D] reads back as, before rounding to the storage type.  The codes are made in fp32 as documented."""
    if format == "plain":
        return x.double()
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(x).all(-1, keepdim=True)
    live = fine & (amax >= 2.0 ** -100)
    top = torch.full_like(amax, TOP[format])
    inv = torch.where(live, top / torch.where(live, amax, top), torch.zeros_like(amax))
    y = torch.where(live, x, torch.zeros_like(x)) * inv
    code = torch.round(y) if format == "int8" else y.to(torch.float8_e4m3fn).float()
    scale = torch.where(live, amax * torch.tensor(1.0 / TOP[format], dtype=torch.float32), torch.zeros_like(amax))
    out = code.double() * scale.double()
    return torch.where(fine, out, torch.full_like(out, math.nan))


def attend(Q, starts, ctx, tree, keys, values, scale, limit=None):
    """keys, values: per request [positions, kv_heads, D] float64.  Returns (out, lse, seen) with seen[t] = number of keys."""
    T, H, D = Q.shape
    out = torch.zeros(T, H, D, dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    for b in range(len(ctx)):
        t0, t1, c = int(starts[b]), int(starts[b + 1]), int(ctx[b])
        for i in range(t1 - t0):
            if tree is None:
                seen = list(range(c + i + 1))
            else:
                word = [int(w) & (1 << 64) - 1 for w in tree[t0 + i].tolist()]
                seen = list(range(c)) + [c + j for j in range(t1 - t0) if word[j // 64] >> (j % 64) & 1]
            if limit is not None:
                seen = [j for j in seen if j < limit]
            if not seen:
                continue
            K, V = keys[b][seen], values[b][seen]
            G = H // K.shape[1]
            for h in range(H):
                s = (K[:, h // G] @ Q[t0 + i, h].double()) * scale
                lse[t0 + i, h] = torch.logsumexp(s, 0)
                out[t0 + i, h] = torch.softmax(s, 0) @ V[:, h // G]
    return out, lse
