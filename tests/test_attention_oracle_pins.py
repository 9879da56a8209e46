"""The plain 64-bit definitions of the attention half against library calls and hand-computed values (no GPU)."""
import math

import torch

from oracle import attention as ref


def test_project_is_a_matrix_product_with_the_adapters_folded_in():
    g = torch.Generator().manual_seed(1)
    X, W, A, B = (torch.randn(*s, generator=g) for s in ((6, 8), (8, 5), (2, 8, 3), (2, 3, 5)))
    scale, aid = torch.tensor([0.5, 2.0]), torch.tensor([0, 1, -1, 1, 7, 0])
    Y = ref.project(X, aid, W, A, B, scale)
    for t, a in enumerate(aid.tolist()):
        M = W.double() + (float(scale[a]) * A[a].double() @ B[a].double() if 0 <= a < 2 else 0)
        assert torch.allclose(Y[t], X[t].double() @ M, atol=1e-12)


def test_rotary_turns_pairs():
    X = torch.tensor([[[1.0, 0.0, 0.0, 2.0]]])
    f = [math.pi / 2, math.pi]
    y = ref.rotary(X, torch.tensor([1]), f, 1.0, 4, "halves")[0, 0]     # pairs (1, 0) and (0, 2)
    assert torch.allclose(y, torch.tensor([0.0, 0.0, 1.0, -2.0], dtype=torch.float64), atol=1e-12)
    y = ref.rotary(X, torch.tensor([1]), f, 3.0, 4, "neighbours")[0, 0]  # pairs (1, 0) and (0, 2), times 3
    assert torch.allclose(y, torch.tensor([0.0, 3.0, 0.0, -6.0], dtype=torch.float64), atol=1e-12)
    back = ref.rotary(y.view(1, 1, 4), torch.tensor([1]), f, 1 / 3.0, 4, "neighbours", transpose=True)
    assert torch.allclose(back, X.double(), atol=1e-12)


def test_scalings_at_their_ends():
    plain, one = ref.frequencies(128)
    assert one == 1.0 and plain[0] == 1.0 and math.isclose(plain[32], 0.01)
    assert all(math.isclose(a, b / 4) for a, b in zip(ref.frequencies(128, 1e4, "linear", 4.0)[0], plain))
    base = ref.frequencies(128, 1e4, "base", 4.0)[0]
    assert base[0] == 1.0 and math.isclose(base[-1], plain[-1] / 4)  # the slowest pair is stretched by the whole factor
    for scaling in ("ramp", "bands"):
        f, m = ref.frequencies(128, 1e4, scaling, 4.0, 4096)
        assert f[0] == plain[0] and math.isclose(f[-1], plain[-1] / 4) and all(b / 4 - 1e-15 <= a <= b for a, b in zip(f, plain))
        assert math.isclose(m, 0.1 * math.log(4.0) + 1.0 if scaling == "ramp" else 1.0)


def test_the_library_gives_the_same_turns():
    from paper_2505_06481_amd import attention
    for rot in (16, 64, 128, 512):
        for scaling in ("none", "linear", "base", "ramp", "bands"):
            steps, m = attention.rotary_steps(rot, 10000.0, scaling, 8.0, 4096, device="cpu")
            f, want = ref.frequencies(rot, 10000.0, scaling, 8.0, 4096)
            assert abs(m - want) < 1e-6
            for s, x in zip(steps.tolist(), f):
                assert abs((s & (1 << 64) - 1) / 2.0 ** 64 - x / (2 * math.pi)) < 1e-16


def test_kept_heads():
    x = torch.tensor([[127.0, -63.4, 0.5, 1.5, 2.5, 0.0]])
    assert ref.kept(x, "int8").tolist() == [[127.0, -63.0, 0.0, 2.0, 2.0, 0.0]]  # a scale of one; ties to even
    y = ref.kept(torch.tensor([[448.0, 17.0, 19.0, -0.001]]), "fp8")
    assert y.tolist()[0][:3] == [448.0, 16.0, 20.0] and abs(y[0, 3]) <= 2.0 ** -9
    z = torch.stack([torch.zeros(4), torch.tensor([1.0, math.nan, 0.0, 0.0]), torch.tensor([math.inf, 1.0, 0.0, 0.0])])
    for format in ("int8", "fp8"):
        k = ref.kept(z, format)
        assert not k[0].any() and bool(torch.isnan(k[1:]).all())


def test_attend_is_masked_softmax_attention():
    g = torch.Generator().manual_seed(2)
    ctx, drafts, H, Hkv, D = [3, 0], [2, 3], 4, 2, 8
    keys = [torch.randn(c + n, Hkv, D, generator=g).double() for c, n in zip(ctx, drafts)]
    values = [torch.randn(c + n, Hkv, D, generator=g).double() for c, n in zip(ctx, drafts)]
    Q, starts = torch.randn(5, H, D, generator=g), [0, 2, 5]
    out, lse = ref.attend(Q, starts, ctx, None, keys, values, 0.3)
    tree = torch.tensor([[0b01], [0b11], [0b001], [0b011], [0b111]])
    assert torch.equal(ref.attend(Q, starts, ctx, tree, keys, values, 0.3)[0], out)  # a causal tree is the causal chunk
    for b in range(2):
        q = Q[starts[b]:starts[b + 1]].double().transpose(0, 1)
        k, v = (x[b].transpose(0, 1).repeat_interleave(2, 0) for x in (keys, values))
        mask = torch.ones(drafts[b], ctx[b] + drafts[b], dtype=torch.bool).tril(ctx[b])
        want = torch.nn.functional.scaled_dot_product_attention(q, k, v, attn_mask=mask, scale=0.3)
        assert torch.allclose(out[starts[b]:starts[b + 1]].transpose(0, 1), want, atol=1e-12)
    empty, l = ref.attend(Q, starts, ctx, torch.zeros(5, 1, dtype=torch.int64), keys, values, 0.3)
    assert not empty[2:].any() and bool((l[2:] == -math.inf).all()) and bool(empty[:2].any())
