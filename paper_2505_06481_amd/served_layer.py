"""One whole layer of a served family of variants, as an example of the library's two halves together.

A step takes the new tokens of many requests, of several variants: projection to queries, keys and values with each
variant's adapter, rotation, append to the paged cache, attention over it, output projection with adapters, and the
mixture-of-experts layer, whose pool the variants share.  The two normalisations and residual sums are plain torch.

    python -m paper_2505_06481_amd.served_layer          # a few speculative decoding steps on random weights
"""
from __future__ import annotations

import torch

from . import attention as at
from . import mmoe


def normalised(x):
    x32 = x.float()
    return (x32 * torch.rsqrt(x32.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class ServedLayer:
    """``W_qkv`` [d, (heads + 2 kv_heads) head_dim], ``W_out`` [heads head_dim, d] and their adapters ``(A, B, scale)`` with one
    adapter for each variant; ``experts``: dict(Wr, br, M, W1, W3, W2, top_k, act) in the plain layout.  ``format``: of the cache."""

    def __init__(self, W_qkv, qkv_adapters, W_out, out_adapters, experts, heads, kv_heads, head_dim, n_pages, format="int8",
                 base=1e6, scaling="none", factor=1.0, original=0):
        self.d, self.heads, self.kv_heads, self.head_dim = W_qkv.shape[0], heads, kv_heads, head_dim
        self.dtype = "bf16" if W_qkv.dtype == torch.bfloat16 else "f32"
        self.experts = dict(experts)
        self.V, self.rank = qkv_adapters[0].shape[0], qkv_adapters[0].shape[2]
        qkv, out = self._project_shape(1, *W_qkv.shape), self._project_shape(1, *W_out.shape)
        self.qkv = (at.pack_projection(qkv, W_qkv), *at.pack_adapters(qkv, *qkv_adapters[:2]), qkv_adapters[2])
        self.out = (at.pack_projection(out, W_out), *at.pack_adapters(out, *out_adapters[:2]), out_adapters[2])
        self.cache_shape = at.make_cache_shape(n_pages, kv_heads, head_dim, self.dtype, format)
        self.cache = at.alloc_cache(self.cache_shape)
        self.steps, self.magnitude = at.rotary_steps(head_dim, base, scaling, factor, original)
        e = self.experts
        self.S, _, self.d_ff = e["W1"].shape
        self.E = e["Wr"].shape[1]
        self.packed = mmoe.pack_weights(self._expert_shape(1), e.pop("W1"), e.pop("W3"), e.pop("W2"))

    def _project_shape(self, T, d_in, d_out):
        return at.make_project_shape(T, d_in, d_out, self.V, self.rank, self.dtype)

    def _expert_shape(self, T):
        return mmoe.make_shape(T, self.d, self.d_ff, self.V, self.E, self.S, self.experts["top_k"], self.dtype, self.experts["act"])

    def attention_half(self, X, vid, pos, places, starts, ctx, pages, max_drafts, tree=None):
        """What the attention half adds to X [T, d].  ``pos``: rotary position of each token, ``places`` its place in the cache;
        the rest as in attention.attend."""
        T, H, Hkv, D = X.shape[0], self.heads, self.kv_heads, self.head_dim
        qkv = self._project_shape(T, self.d, (H + 2 * Hkv) * D)
        rows = at.project(qkv, normalised(X), vid, *self.qkv, at.project_workspace(qkv)).view(T, H + 2 * Hkv, D)
        q, k, v = rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
        turn = at.make_rotary_shape(T, H, D, D, "halves", self.dtype, self.magnitude)
        at.rotary(turn, q, pos, self.steps, Y=q)
        at.cache_append(self.cache_shape, k, v, places, self.cache, rotary=(turn, self.steps, pos))
        shape = at.make_attend_shape(self.cache_shape, T, ctx.numel(), H, pages.shape[1], max_drafts, D ** -0.5,
                                     mask_words=tree.shape[1] if tree is not None else None)
        mixed, _ = at.attend(shape, q, starts, ctx, tree, pages, self.cache, at.attend_workspace(shape))
        out = self._project_shape(T, H * D, self.d)
        return at.project(out, mixed.view(T, H * D), vid, *self.out, at.project_workspace(out))

    def expert_half(self, X, vid):
        """What the experts add to X."""
        shape, e = self._expert_shape(X.shape[0]), self.experts
        return mmoe.layer_forward(shape, normalised(X), vid, e["Wr"], e["br"], e["M"], *self.packed, mmoe.alloc_workspace(shape))

    def step(self, X, vid, *where, **kw):
        X = X + self.attention_half(X, vid, *where, **kw)
        return X + self.expert_half(X, vid)


def example_layer(d=512, heads=8, kv_heads=2, head_dim=64, d_ff=768, V=3, E=4, rank=8, n_pages=64, format="int8", dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, scale):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def adapters(k, n):
        return randn(V, k, rank, scale=k ** -0.5), randn(V, rank, n, scale=0.3 * rank ** -0.5), torch.full((V,), 0.5, device="cuda")

    n = (heads + 2 * kv_heads) * head_dim
    M = torch.arange(E, device="cuda", dtype=torch.int32).repeat(V, 1)          # shared but for one expert of each later variant
    M[1:, 0] = E + torch.arange(V - 1, device="cuda", dtype=torch.int32)
    S = E + V - 1
    experts = dict(Wr=randn(V, E, d, scale=d ** -0.5), br=None, M=M, W1=randn(S, d, d_ff, scale=d ** -0.5), W3=randn(S, d, d_ff, scale=d ** -0.5),
                   W2=randn(S, d_ff, d, scale=d_ff ** -0.5), top_k=2, act="swiglu")
    return ServedLayer(randn(d, n, scale=d ** -0.5), adapters(d, n), randn(heads * head_dim, d, scale=(heads * head_dim) ** -0.5),
                       adapters(heads * head_dim, d), experts, heads, kv_heads, head_dim, n_pages, format)


def example_batch(requests, prompts, drafts, pages_each, V, step=0):
    """Two calls' arguments for `requests` requests: their prompts as causal chunks, then `drafts` drafted tokens each, a
    binary tree."""
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = torch.randperm(requests * pages_each, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(requests, pages_each).cuda()
    out = []
    for ctx, counts in (([0] * requests, prompts), (prompts, [drafts] * requests)):
        tree = None
        at_ = [torch.arange(c, c + n) for c, n in zip(ctx, counts)]                     # position in the cache
        pos = at_
        if counts is not prompts:
            seen, depth = [1], [0]
            for i in range(1, drafts):
                seen.append(seen[(i - 1) // 2] | 1 << i)
                depth.append(depth[(i - 1) // 2] + 1)
            tree = torch.tensor(seen * requests, dtype=torch.int64, device="cuda")[:, None]
            pos = [c + torch.tensor(depth) for c in ctx]
        places = torch.cat([pages[b].cpu()[a // 64] * 64 + a % 64 for b, a in enumerate(at_)])
        vid = torch.cat([torch.full((n,), b % V) for b, n in enumerate(counts)])
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        out.append((vid.to(**i32), torch.cat(pos).to(**i32), places.to(**i32), torch.tensor(starts, **i32), torch.tensor(ctx, **i32), pages,
                    max(counts), tree))
    return out


def main():
    layer = example_layer()
    chunk, draft = example_batch(4, [100, 7, 64, 1], 7, 2, layer.V)
    for name, (vid, *where) in (("prompts", chunk), ("drafted tokens", draft)):
        X = torch.randn(vid.numel(), layer.d, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
        Y = layer.step(X, vid, *where)
        torch.cuda.synchronize()
        print(f"{name}: {vid.numel()} tokens of {layer.V} variants, output rms {float(Y.float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
