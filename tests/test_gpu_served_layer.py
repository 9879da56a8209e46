"""The two halves together: a prompt chunk and a tree of drafted tokens through a whole layer, against the plain definitions.

The attention half is compared in the norm: seven roundings to bf16 on the way (normalised input, queries and keys twice, values,
mixed values, output), 2^-9 rms each at most relative to what they round, and 8-bit keys and values whose codes are off by one where a
rounded key differs: 7 * 2^-9 = 1.4 %, taken as 2 %.  The experts are compared with the oracle on the very input they got."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("format", ["plain", "int8", "fp8"])
def test_served_layer(oracle, format):
    import gpu_common as gc
    from oracle import attention as ref
    from paper_2505_06481_amd import served_layer as sl

    keep = {}  # the plain weights, on their way into their packed forms
    real_pack = sl.at.pack_projection, sl.at.pack_adapters, sl.mmoe.pack_weights

    def spy(key, f):
        def g(shape, *w):
            keep.setdefault(key, []).append([None if x is None else x.cpu() for x in w])
            return f(shape, *w)
        return g
    try:
        sl.at.pack_projection, sl.at.pack_adapters, sl.mmoe.pack_weights = (spy(k, f) for k, f in zip(("W", "AB", "pool"), real_pack))
        layer = sl.example_layer(format=format, seed=3)
    finally:
        sl.at.pack_projection, sl.at.pack_adapters, sl.mmoe.pack_weights = real_pack
    (Wq,), (Wo,) = keep["W"]
    (Aq, Bq), (Ao, Bo) = keep["AB"]
    W1, W3, W2 = keep["pool"][0]
    H, Hkv, D = layer.heads, layer.kv_heads, layer.head_dim
    freqs, m = ref.frequencies(D, 1e6)
    requests, prompts, drafts = 4, [100, 7, 64, 1], 7
    calls = sl.example_batch(requests, prompts, drafts, 2, layer.V)
    keys, values = [torch.zeros(0, Hkv, D, dtype=torch.float64) for _ in range(requests)], [torch.zeros(0, Hkv, D, dtype=torch.float64) for _ in range(requests)]
    bf = lambda x: x.to(torch.bfloat16)  # noqa: E731
    for n, (vid, pos, places, starts, ctx, pages, most, tree) in enumerate(calls):
        X = torch.randn(vid.numel(), layer.d, generator=torch.Generator().manual_seed(10 + n)).bfloat16()
        got = layer.attention_half(X.cuda(), vid, pos, places, starts, ctx, pages, most, tree)
        scale = torch.full((layer.V,), 0.5)
        rows = bf(ref.project(sl.normalised(X), vid.cpu(), Wq, Aq, Bq, scale)).view(-1, H + 2 * Hkv, D)
        q, k = (bf(ref.rotary(x, pos.cpu(), freqs, m, D, "halves")) for x in (rows[:, :H], rows[:, H:H + Hkv]))
        for b in range(requests):
            mine = slice(int(starts[b]), int(starts[b + 1]))
            keys[b] = torch.cat([keys[b], ref.kept(k[mine], format)])
            values[b] = torch.cat([values[b], ref.kept(rows[mine, H + Hkv:], format)])
        mixed, _ = ref.attend(q, starts.tolist(), ctx.tolist(), None if tree is None else tree.cpu(), keys, values, D ** -0.5)
        want = ref.project(bf(mixed.reshape(-1, H * D)), vid.cpu(), Wo, Ao, Bo, scale)
        err = (got.cpu().double() - want).norm() / want.norm()
        assert err < 0.02, f"{format}, call {n}: {err:.4f}"

        Z = (X.cuda() + got)
        Y = layer.expert_half(Z, vid)
        bits = lambda t: t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)  # noqa: E731
        inp = dict(X=bits(sl.normalised(Z)), vid=vid.cpu().numpy(), Wr=bits(layer.experts["Wr"]), br=None, M=layer.experts["M"].cpu().numpy(),
                   W1=bits(W1), W3=bits(W3), W2=bits(W2), S=layer.S)
        out = oracle.layer_forward(inp, 2, "bf16", "swiglu")
        gc.assert_close(gc.to_np64(Y), out["Y"], "bf16", f"experts, call {n}")
        assert torch.equal(layer.step(X.cuda(), vid, pos, places, starts, ctx, pages, most, tree), Z + Y)


def test_example_runs(capsys):
    from paper_2505_06481_amd import served_layer
    served_layer.main()
    assert "drafted tokens" in capsys.readouterr().out
