"""The operators around the mixture-of-experts layer, as cases that can be timed and compared.

A served layer has an attention half in front of its experts, for the same batch that mixes tokens of
several fine-tuned variants.  Four operators make it up:

  project   X W for all tokens and, beside it, each token's own low-rank adapter (X A_a) B_a
  rotary    heads rotated by their token's position
  cache     keys and values appended to pages of 64 tokens, in 8 bits or as they are, and read back
  attend    drafted tokens (a tree, a causal chunk, or one token) of many requests over their cache pages

over these ranges:

  tokens    project 1 .. 8192, rotary 1 .. 8192, cache 1 .. 4096 appended and up to 16384 read
  requests  attend 1 .. 64 with 1 .. 128 drafted tokens each and contexts of 0 .. 120000 tokens
  shapes    width 256 .. 6144, adapters 1 .. 64 of rank 4 .. 64, heads of 64 and 128, 1 .. 8 query heads to a key head
  types     bf16 and fp32; caches as they are, int8, fp8 (e4m3)

A case is a dict of plain values.  Lengths (contexts, drafted tokens) follow from the case, so that its
work does; values, positions, adapters and pages follow from the seed.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_PAGE = 64
_LEVELS = {"int8": 127.0, "fp8": 448.0}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # One decode step of three requests on a small model: the shortest call there is.
        _project("project_decode_t3", 3, 768, 2304, 2, 8, "bf16"),
        # Decode of a large model, one token each of 64 requests that use 48 different adapters.
        _project("project_decode_t64", 64, 4096, 6144, 48, 16, "bf16"),
        # The small model in full precision, an odd batch, rank 12, some tokens on the base model.
        _project("project_f32_t777", 777, 768, 2304, 5, 12, "f32", bare=0.3),
        # Prefill of a large model by two variants.
        _project("project_prefill_t8192", 8192, 4096, 6144, 2, 32, "bf16"),
        # A handful of fp32 heads, a quarter of each rotated in neighbours, the gradient's direction.
        _rotary("rotary_f32_t5", 5, 16, 0, 64, 16, "neighbours", "linear", "f32", 4000, True),
        # Queries and keys of a prefill, in place in the rows that the projection wrote (with the values
        # behind them), frequencies scaled for a long context.
        _rotary("rotary_prefill_t8192", 8192, 40, 8, 128, 128, "halves", "ramp", "bf16", 120000, False),
        # The keys and values of one decode step of 16 requests.
        _cache("cache_step_int8_t16", 16, 16, 8, 128, "bf16", "int8", True),
        # A prefill chunk, and the whole context handed on in plain form.
        _cache("cache_chunk_fp8_t4096", 4096, 16384, 8, 128, "bf16", "fp8", False),
        # Decode of four requests with short contexts.
        _attend("attend_decode_b4", 4, 1, 20, 700, 32, 8, 128, "bf16", "plain", False),
        # A small model in full precision, wide trees, no shared heads.
        _attend("attend_f32_tree_b6", 6, 40, 0, 1500, 12, 12, 64, "f32", "plain", True),
        # Speculative decoding of a full batch of requests.
        _attend("attend_tree_int8_b32", 32, 12, 0, 6000, 32, 8, 128, "bf16", "int8", True),
        # Speculative decoding over long contexts.
        _attend("attend_long_fp8_b8", 8, 16, 8000, 120000, 32, 8, 128, "bf16", "fp8", True),
    ]


def _project(name, T, d_in, d_out, adapters, rank, dtype, bare=0.0):
    return {"name": name, "op": "project", "T": T, "d_in": d_in, "d_out": d_out, "adapters": adapters, "rank": rank,
            "dtype": dtype, "bare": bare}


def _rotary(name, T, heads, behind, head_dim, rot, layout, scaling, dtype, span, transpose):
    return {"name": name, "op": "rotary", "T": T, "heads": heads, "behind": behind, "head_dim": head_dim, "rot": rot,
            "layout": layout, "scaling": scaling, "dtype": dtype, "span": span, "transpose": transpose}


def _cache(name, T, reads, kv_heads, head_dim, dtype, format, rotate):
    return {"name": name, "op": "cache", "T": T, "reads": reads, "kv_heads": kv_heads, "head_dim": head_dim,
            "dtype": dtype, "format": format, "rotate": rotate}


def _attend(name, requests, drafts, ctx_min, ctx_max, heads, kv_heads, head_dim, dtype, format, tree):
    return {"name": name, "op": "attend", "requests": requests, "drafts": drafts, "ctx_min": ctx_min, "ctx_max": ctx_max,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "format": format, "tree": tree}


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = _drawn(rng)
    del case["name"]
    return case


def _drawn(rng):
    op = rng.choice(["project", "rotary", "cache", "attend"])
    if op == "project":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        while True:
            T = _log(rng, 1, 8192 if dtype == "bf16" else 2048)
            d_in, d_out = 256 * _log(rng, 1, 16), 256 * _log(rng, 1, 24)
            if d_in != 3072 and d_out != 3072:
                break
        return _project("", T, d_in, d_out, _log(rng, 1, 64), rng.choice([4, 7, 8, 12, 16, 20, 32, 48, 64]), dtype,
                        rng.choice([0.0, 0.0, 0.3]))
    if op == "rotary":
        head_dim = rng.choice([64, 128])
        return _rotary("", _log(rng, 1, 8192), _log(rng, 1, 40), rng.choice([0, 3, 8]), head_dim,
                       rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4]), rng.choice(["halves", "neighbours"]),
                       rng.choice(["none", "linear", "base", "ramp", "bands"]), rng.choice(["bf16", "bf16", "f32"]),
                       _log(rng, 100, 1000000), rng.random() < 0.25)
    if op == "cache":
        dtype, format = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice(["plain", "int8", "fp8"])
        # (fp32 keys are rotated into plain pages only: a last bit of a rotated value may be another code of eight bits)
        return _cache("", _log(rng, 1, 4096), _log(rng, 1, 16384), rng.randint(1, 8), rng.choice([64, 128]), dtype, format,
                      rng.random() < 0.5 and (dtype == "bf16" or format == "plain"))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 7), (8, 4), (8, 1), (12, 1), (4, 2)])
    requests, tree = _log(rng, 1, 64), rng.random() < 0.6
    drafts = _log(rng, 1, 64 if tree else 128)
    most = min(120000, 960000 * 8 // (requests * kv_heads))
    if dtype == "f32":
        most = min(most, 200000 // requests)
    most = min(most, 16 * 8 * 4 * 120000 * 8 // (requests * drafts * kv_heads * group))  # scores of the plain form
    ctx_max = _log(rng, 16, max(17, most))
    return _attend("", requests, drafts, rng.choice([0, ctx_max // 2, ctx_max]), ctx_max, kv_heads * group, kv_heads,
                   rng.choice([64, 128]), dtype, rng.choice(["plain", "int8", "fp8"]) if dtype == "bf16" else "plain",
                   tree)


def _esz(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lengths(case):
    """Contexts and drafted tokens of the requests: they follow from the case alone."""
    rng = random.Random("%(requests)d %(drafts)d %(ctx_min)d %(ctx_max)d %(heads)d" % case)
    n = case["requests"]
    ctx = [rng.randint(case["ctx_min"], case["ctx_max"]) for _ in range(n)]
    drafts = [rng.randint((case["drafts"] + 1) // 2, case["drafts"]) for _ in range(n)]
    ctx[-1], drafts[-1] = case["ctx_max"], case["drafts"]  # the longest one that the program allows for
    return ctx, drafts


def work(case):
    e = _esz(case)
    if case["op"] == "project":
        T, K, N, R, n = (case[k] for k in ("T", "d_in", "d_out", "rank", "adapters"))
        used = min(n, T)
        return {"bytes": e * (T * K + K * N + T * N + used * R * (K + N)) + 4 * T + 4 * n,
                "flops": 2.0 * T * K * N + 2.0 * T * R * (K + N) * (1 - case["bare"])}
    if case["op"] == "rotary":
        n = case["T"] * case["heads"] * case["head_dim"]
        return {"bytes": 2 * n * e + 4 * case["T"], "flops": 3.0 * n * case["rot"] / case["head_dim"]}
    if case["op"] == "cache":
        rows = case["kv_heads"] * case["head_dim"] * 2
        kept = rows * (e if case["format"] == "plain" else 1) + (0 if case["format"] == "plain" else 8 * case["kv_heads"])
        return {"bytes": case["T"] * (rows * e + kept + 4) + case["reads"] * (rows * e + kept + 4),
                "flops": 2.0 * rows * (case["T"] + case["reads"])}
    ctx, drafts = _lengths(case)
    keys = sum(c + d for c, d in zip(ctx, drafts))
    pairs = sum(c * d + d * (d + 1) // 2 for c, d in zip(ctx, drafts))
    rows = case["kv_heads"] * case["head_dim"] * 2
    kept = rows * (e if case["format"] == "plain" else 1) + (0 if case["format"] == "plain" else 8 * case["kv_heads"])
    T = sum(drafts)
    return {"bytes": keys * kept + 2 * e * T * case["heads"] * case["head_dim"] + 4 * T * case["heads"],
            "flops": 4.0 * pairs * case["heads"] * case["head_dim"]}


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


_THETA, _ORIGINAL, _FACTOR = 10000.0, 4096, 8.0


def _frequencies(rot, scaling):
    """Radians per position of every pair of a head, and the factor on the rotated values."""
    f = [_THETA ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / _FACTOR for x in f], 1.0
    if scaling == "base":
        theta = _THETA * _FACTOR ** (rot / (rot - 2.0))
        return [theta ** (-2.0 * i / rot) for i in range(rot // 2)], 1.0
    if scaling == "ramp":  # as they are down to the pair that turns 32 times in the original context, divided from that of one turn on
        at = [rot * math.log(_ORIGINAL / (b * 2 * math.pi)) / (2 * math.log(_THETA)) for b in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = [1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3))) for i in range(rot // 2)]
        return [x * k + x / _FACTOR * (1 - k) for x, k in zip(f, keep)], 0.1 * math.log(_FACTOR) + 1.0
    if scaling == "bands":  # wavelengths up to a quarter of the original context stay, from the whole of it on they are stretched
        out = []
        for x in f:
            turns = _ORIGINAL * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            out.append(x * keep + x / _FACTOR * (1 - keep))
        return out, 1.0
    return f, 1.0


def _turns(freqs):
    """Turns per position in units of 2^-64: whole turns of an angle are what overflows."""
    t = [int(round(f / (2 * math.pi) * 2.0 ** 64)) for f in freqs]
    return torch.tensor([x - (1 << 64) if x >= 1 << 63 else x for x in t], dtype=torch.int64, device="cuda")


def _tree_words(rng, drafts):
    """A random tree over each request's drafted tokens: a token sees itself and the tokens it descends from."""
    words, most = [], max(drafts)
    for n in drafts:
        seen = []
        for i in range(n):
            parent = rng.randint(max(-1, i - 4), i - 1)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        words += seen
    wide = (most + 63) // 64
    out = [[(w >> 64 * k) & (1 << 64) - 1 for k in range(wide)] for w in words]
    return torch.tensor([[x - (1 << 64) if x >= 1 << 63 else x for x in r] for r in out], dtype=torch.int64, device="cuda")


def _quantised(x, format):
    """Codes and scales of rows of a head: the largest magnitude is the format's largest code."""
    if format == "plain":
        return x, None
    x = x.float()
    amax = x.abs().amax(-1)
    inv = torch.where(amax > 0, torch.full_like(amax, _LEVELS[format]) / amax, torch.zeros_like(amax))
    y = x * inv[..., None]
    code = torch.round(y).to(torch.int8) if format == "int8" else y.to(torch.float8_e4m3fn)
    return code, amax * (1.0 / _LEVELS[format])


def prepare(case, seed):
    g, dt = _gen(seed), _DT[case["dtype"]]
    s = {"case": case}
    if own:
        from paper_2505_06481_amd import attention
    if case["op"] == "project":
        T, K, N, R, n = (case[k] for k in ("T", "d_in", "d_out", "rank", "adapters"))
        s["X"] = _randn(g, T, K, dtype=dt)
        W = _randn(g, K, N, scale=0.02, dtype=dt)
        A = _randn(g, n, K, R, scale=K ** -0.5, dtype=dt)
        B = _randn(g, n, R, N, scale=0.1, dtype=dt)
        s["scale"] = torch.rand(n, generator=g, device="cuda") + 0.5
        aid = torch.randint(0, n, (T,), generator=g, device="cuda", dtype=torch.int32)
        bare = torch.rand(T, generator=g, device="cuda") < case["bare"]
        s["aid"] = torch.where(bare, torch.full_like(aid, -1), aid)
        if own:
            s["shape"] = attention.make_project_shape(T, K, N, n, R, case["dtype"])
            s["Wp"] = attention.pack_projection(s["shape"], W)
            s["Ap"], s["Bp"] = attention.pack_adapters(s["shape"], A, B)
            s["ws"] = attention.project_workspace(s["shape"])
        else:
            s["W"], s["A"], s["B"] = W, A, B
        return s
    if case["op"] == "rotary":
        T, H, D = case["T"], case["heads"], case["head_dim"]
        rows = _randn(g, T, H + case["behind"], D, dtype=dt)
        s["X"] = rows[:, :H]
        start = torch.randint(0, max(1, case["span"] - T), (1,), generator=g, device="cuda")
        s["pos"] = (start + torch.arange(T, device="cuda")).to(torch.int32)
        if own:
            steps, magnitude = attention.rotary_steps(case["rot"], _THETA, case["scaling"], _FACTOR, _ORIGINAL)
            s["steps"] = steps
            s["shape"] = attention.make_rotary_shape(T, H, D, case["rot"], case["layout"], case["dtype"], magnitude,
                                                     transpose=case["transpose"])
        else:
            freqs, s["magnitude"] = _frequencies(case["rot"], case["scaling"])
            s["steps"] = _turns(freqs)
        return s
    if case["op"] == "cache":
        T, R, H, D = case["T"], case["reads"], case["kv_heads"], case["head_dim"]
        pages = (max(T, R) + _PAGE - 1) // _PAGE + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int64)
        context = torch.arange(max(T, R), device="cuda")  # one long context on pages in any order; the last T tokens are new
        places = (order[context // _PAGE] * _PAGE + context % _PAGE).to(torch.int32)
        old = max(T, R) - T
        rows = _randn(g, T, 2 * H + 1, D, dtype=dt)
        s["K"], s["V"] = rows[:, :H], rows[:, H:2 * H]  # as a projection leaves them
        s["new"], s["reads"] = places[old:].contiguous(), places[len(places) - R:].contiguous()
        s["pos"] = torch.arange(old, old + T, device="cuda", dtype=torch.int32)
        K0, V0 = _randn(g, old, H, D, dtype=dt), _randn(g, old, H, D, dtype=dt)
        if own:
            s["shape"] = attention.make_cache_shape(pages, H, D, case["dtype"], case["format"])
            s["cache"] = attention.alloc_cache(s["shape"])
            attention.cache_append(s["shape"], K0, V0, places[:old].contiguous(), s["cache"])
            s["rotary"] = None
            if case["rotate"]:
                steps, magnitude = attention.rotary_steps(D, _THETA, "none", 1.0, _ORIGINAL)
                s["rotary"] = (attention.make_rotary_shape(T, H, D, D, "halves", case["dtype"], magnitude), steps, s["pos"])
        else:
            s["kept"] = []
            for x in (K0, V0):
                code, scale = _quantised(x, case["format"])
                all_codes = torch.zeros(pages * _PAGE, H, D, dtype=code.dtype, device="cuda")
                _as_bytes(all_codes)[places[:old].long()] = _as_bytes(code)
                all_scales = torch.zeros(pages * _PAGE, H, device="cuda")
                if scale is not None:
                    all_scales[places[:old].long()] = scale
                s["kept"] += [all_codes, all_scales]
            freqs, s["magnitude"] = _frequencies(D, "none")
            s["steps"] = _turns(freqs)
        return s
    ctx, drafts = _lengths(case)
    B, H, Hkv, D = case["requests"], case["heads"], case["kv_heads"], case["head_dim"]
    T, most = sum(drafts), max(drafts)
    lengths = [c + d for c, d in zip(ctx, drafts)]
    wide = max((n + _PAGE - 1) // _PAGE for n in lengths)
    own_pages = [(n + _PAGE - 1) // _PAGE for n in lengths]
    order = torch.randperm(sum(own_pages), generator=g, device="cuda").to(torch.int32)
    table, at = torch.zeros(B, wide, dtype=torch.int32, device="cuda"), 0
    for b, n in enumerate(own_pages):
        table[b, :n] = order[at:at + n]
        at += n
    s["pages"], s["Q"] = table, _randn(g, T, H, D, dtype=dt)
    s["ctx"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    starts = [0]
    for n in drafts:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["tree"] = _tree_words(random.Random(seed), drafts) if case["tree"] else None
    s["scale"] = D ** -0.5
    rows = sum(own_pages) * _PAGE
    loud = 1.0 + 5.0 * (torch.rand(Hkv, D, generator=g, device="cuda") < 0.03)  # keys have a few large channels
    K = torch.empty(rows, Hkv, D, dtype=dt, device="cuda")
    V = torch.empty(rows, Hkv, D, dtype=dt, device="cuda")
    for r in range(0, rows, 1 << 16):
        n = min(1 << 16, rows - r)
        K[r:r + n] = _randn(g, n, Hkv, D) * loud
        V[r:r + n] = _randn(g, n, Hkv, D)
    if own:
        cs = attention.make_cache_shape(sum(own_pages), Hkv, D, case["dtype"], case["format"])
        s["cache"] = attention.alloc_cache(cs)
        attention.cache_append(cs, K, V, torch.arange(rows, dtype=torch.int32, device="cuda"), s["cache"])
        s["shape"] = attention.make_attend_shape(cs, T, B, H, wide, most, s["scale"], max_keys=max(lengths), sum_keys=sum(lengths))
        s["ws"] = attention.attend_workspace(s["shape"])
    else:
        (s["Kc"], s["Ks"]), (s["Vc"], s["Vs"]) = _quantised_in_parts(K, case["format"]), _quantised_in_parts(V, case["format"])
        qi = torch.full((B, most), -1, dtype=torch.int64)
        for b, n in enumerate(drafts):
            qi[b, :n] = torch.arange(starts[b], starts[b] + n)
        s["qi"], s["longest"] = qi.cuda(), max(lengths)
    return s


def _as_bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _quantised_in_parts(x, format):
    if format == "plain":
        return x, None
    parts = [_quantised(p, format) for p in x.split(1 << 16)]
    return torch.cat([_as_bytes(c) for c, _ in parts]).view(parts[0][0].dtype), torch.cat([c for _, c in parts])


# ---------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2505_06481_amd import attention
        if op == "project":
            return attention.project(s["shape"], s["X"], s["aid"], s["Wp"], s["Ap"], s["Bp"], s["scale"], s["ws"])
        if op == "rotary":
            return attention.rotary(s["shape"], s["X"], s["pos"], s["steps"])
        if op == "cache":
            attention.cache_append(s["shape"], s["K"], s["V"], s["new"], s["cache"], rotary=s["rotary"])
            return attention.cache_read(s["shape"], s["cache"], s["reads"])
        return attention.attend(s["shape"], s["Q"], s["starts"], s["ctx"], s["tree"], s["pages"], s["cache"], s["ws"])
    return {"project": _plain_project, "rotary": _plain_rotary, "cache": _plain_cache, "attend": _plain_attend}[op](s)


def _plain_project(s):
    X = s["X"].float()
    K, (n, _, R) = X.shape[1], s["A"].shape
    U = X @ s["A"].float().permute(1, 0, 2).reshape(K, n * R)                # every adapter's
    mine = s["aid"][:, None] == torch.arange(n, device=X.device, dtype=torch.int32)
    U = U.view(-1, n, R) * torch.where(mine, s["scale"], torch.zeros_like(s["scale"]))[:, :, None]
    return (X @ s["W"].float() + U.view(-1, n * R) @ s["B"].float().view(n * R, -1)).to(s["X"].dtype)


def _rotated(x, pos, steps, magnitude, layout, transpose):
    """fp32 [T, H, rot] rotated; angles are exact to 2^-31 of a turn at any position."""
    turns = (pos.long()[:, None] * steps) >> 32
    angle = turns.float() * (math.pi * 2.0 ** -31)
    c, n = (torch.cos(angle) * magnitude)[:, None], (torch.sin(angle) * (-magnitude if transpose else magnitude))[:, None]
    if layout == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * n, a * n + b * c], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2)


def _plain_rotary(s):
    c, x = s["case"], s["X"].float()
    y = _rotated(x[..., :c["rot"]], s["pos"], s["steps"], s["magnitude"], c["layout"], c["transpose"])
    return torch.cat([y, x[..., c["rot"]:]], -1).to(s["X"].dtype)


def _plain_cache(s):
    K, V, new, reads, dt = s["K"], s["V"], s["new"].long(), s["reads"].long(), s["K"].dtype
    if s["case"]["rotate"]:
        K = _rotated(K.float(), s["pos"], s["steps"], s["magnitude"], "halves", False).to(dt)
    out = []
    for x, codes, scales in ((K, *s["kept"][:2]), (V, *s["kept"][2:])):
        code, scale = _quantised(x, s["case"]["format"])
        _as_bytes(codes)[new] = _as_bytes(code)
        got = _as_bytes(codes)[reads].view(codes.dtype)
        if scale is not None:
            scales[new] = scale
            got = (got.float() * scales[reads][..., None]).to(dt)
        out.append(got)
    return out


def _plain_attend(s):
    H, Hkv, D = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["head_dim"]
    B, n, G = *s["qi"].shape, H // Hkv
    j = torch.arange(s["longest"], device="cuda")
    rows = s["pages"].long()[:, j // _PAGE] * _PAGE + j % _PAGE

    def gathered(codes, scales):
        x = _as_bytes(codes)[rows].view(codes.dtype).float()
        return x if scales is None else x * scales[rows][..., None]

    q = s["Q"].float()[s["qi"].clamp(min=0)].view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    S = torch.matmul(q, gathered(s["Kc"], s["Ks"]).permute(0, 2, 3, 1).contiguous()) * s["scale"]
    ctx, i = s["ctx"].long()[:, None, None], torch.arange(n, device="cuda")[None, :, None]
    d = j[None, None, :] - ctx  # which drafted token a key is
    if s["tree"] is None:
        seen = d <= i
    else:
        words = s["tree"][s["qi"].clamp(min=0)]
        at = d.clamp(min=0, max=64 * words.shape[-1] - 1).expand(-1, n, -1)
        seen = (d < 0) | ((torch.gather(words, 2, at // 64) >> (at % 64) & 1) == 1)
    count = (s["starts"][1:] - s["starts"][:-1]).long()[:, None, None]
    seen = seen & (d < count)
    S = S.view(B, Hkv, n, G, -1).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = S.amax(-1, keepdim=True)
    P = S.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    total = P.sum(-1, keepdim=True)
    O = torch.matmul(P.view(B, Hkv, n * G, -1), gathered(s["Vc"], s["Vs"]).permute(0, 2, 1, 3).contiguous())
    O = O.view(B, Hkv, n, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    there = s["qi"] >= 0
    out = O.permute(0, 2, 1, 3, 4).reshape(B, n, H, D)[there]
    lse = (m + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, n, H)[there]
    return out.to(s["Q"].dtype), lse


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"project": _exact_project, "rotary": _exact_rotary, "cache": _exact_cache, "attend": _exact_attend}[case["op"]](s)


def _exact_project(s):
    X, aid = s["X"].double(), s["aid"]
    Y = X @ s["W"].double()
    for a in range(s["A"].shape[0]):
        rows = (aid == a).nonzero()[:, 0]
        if len(rows):
            Y[rows] += float(s["scale"][a]) * (X[rows] @ s["A"][a].double()) @ s["B"][a].double()
    return Y


def _exact_angles(case, pos, rot, scaling):
    freqs, magnitude = _frequencies(rot, scaling)
    return pos.double()[:, None, None] * torch.tensor(freqs, dtype=torch.float64, device=pos.device), magnitude


def _exact_turn(x, angle, magnitude, layout):
    z = torch.complex(*((x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]) if layout == "halves" else (x[..., 0::2], x[..., 1::2])))
    z = z * torch.polar(torch.full_like(angle, magnitude), angle)
    return torch.cat([z.real, z.imag], -1) if layout == "halves" else torch.view_as_real(z).flatten(-2)


def _exact_rotary(s):
    c = s["case"]
    x = s["X"].double().clone()
    angle, magnitude = _exact_angles(c, s["pos"], c["rot"], c["scaling"])
    x[..., :c["rot"]] = _exact_turn(x[..., :c["rot"]].contiguous(), -angle if c["transpose"] else angle, magnitude, c["layout"])
    return x


def _exact_cache(s):
    c, out = s["case"], []
    for x, codes, scales in ((s["K"], *s["kept"][:2]), (s["V"], *s["kept"][2:])):
        y = x.double()
        if c["rotate"] and x is s["K"]:
            angle, magnitude = _exact_angles(c, s["pos"], c["head_dim"], "none")
            y = _exact_turn(y.contiguous(), angle, magnitude, "halves").to(x.dtype).double()
        if c["format"] != "plain":
            step = y.abs().amax(-1, keepdim=True) / _LEVELS[c["format"]]
            unit = y / step.clamp(min=1e-300)
            y = (unit.round() if c["format"] == "int8" else unit.float().to(torch.float8_e4m3fn).double()) * step
        kept = codes.to(torch.float32).double() * (scales.double()[..., None] if c["format"] != "plain" else 1.0)
        kept[s["new"].long()] = y
        out.append(kept[s["reads"].long()])
    return out


def _exact_attend(s):
    H, Hkv, D = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["head_dim"]
    ctx, starts, G = s["ctx"].tolist(), s["starts"].tolist(), H // Hkv
    out, lse = torch.zeros(starts[-1], H, D, dtype=torch.float64, device="cuda"), torch.zeros(starts[-1], H, dtype=torch.float64, device="cuda")
    for b, c in enumerate(ctx):
        t0, t1 = starts[b], starts[b + 1]
        n = t1 - t0
        rows = (s["pages"][b].long()[:, None] * _PAGE + torch.arange(_PAGE, device="cuda")).flatten()[:c + n]
        K, V = (_as_bytes(s[k])[rows].view(s[k].dtype).float().double() for k in ("Kc", "Vc"))
        if s["Ks"] is not None:
            K, V = K * s["Ks"][rows].double()[..., None], V * s["Vs"][rows].double()[..., None]
        if s["tree"] is None:
            drafted = torch.tril(torch.ones(n, n, dtype=torch.bool, device="cuda"))
        else:
            bits = torch.arange(64, device="cuda")
            drafted = ((s["tree"][t0:t1, :, None] >> bits & 1) == 1).flatten(1)[:, :n]
        seen = torch.cat([torch.ones(n, c, dtype=torch.bool, device="cuda"), drafted], 1)
        for h in range(H):
            S = (s["Q"][t0:t1, h].double() @ K[:, h // G].T.contiguous()) * s["scale"]
            S = S.masked_fill(~seen, -math.inf)
            lse[t0:t1, h] = torch.logsumexp(S, -1)
            out[t0:t1, h] = torch.nan_to_num(torch.softmax(S, -1)) @ V[:, h // G]
    return out, lse
