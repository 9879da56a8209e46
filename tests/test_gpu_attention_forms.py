"""Forms of the attention half's operators at sizes and types beside those of test_gpu_attention.py, against the definitions in oracle/attention.py
(tolerances there but where a test derives its own)."""
import math

import pytest
import torch

from test_gpu_attention import KINDS, Paged, at, check_attend, close, gen_of, rand, ref, run_rotary  # noqa: F401 (at, ref: fixtures)
from test_gpu_project_values import SIZES, project

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("R", [2, 33])
def test_project_keeps_16_bits_of_the_adapters_product(at, ref, T, K, N, R):
    """Y = U_0 - U_1 of two nearly equal columns of U, which one bf16 part of each would leave no bits of.

    |err| <= 2^-16 (|U_0| + |U_1|) for U in two parts, twice the K 2^-24 sum |x a| of sums in fp32, and 2^-8 |Y| for the rounding of Y."""
    g = gen_of(50, T, R)
    X = rand(g, T, K, dtype="bf16")
    W, B = torch.zeros(K, N, dtype=torch.bfloat16), torch.zeros(2, R, N, dtype=torch.bfloat16)
    A = torch.zeros(2, K, R, dtype=torch.bfloat16)
    A[:, :, 0] = rand(g, 2, K, dtype="bf16")
    A[:, :, R - 1] = A[:, :, 0]
    A[:, ::16, R - 1] *= 1.0 + 2.0 ** -3
    B[:, 0], B[:, R - 1] = 1.0, -1.0
    aid, scale = torch.arange(T, dtype=torch.int32) % 2, torch.tensor([1.0, 0.7])
    some = torch.arange(min(T, 200))
    Y = project(at, X, aid, W, A, B, scale, "bf16")[some.cuda()]
    want = ref.project(X[some], aid[some], W, A, B, scale)
    a, f = A[aid[some].long()].double(), scale[aid[some].long()].double()[:, None]
    U = (X[some].double()[:, None] @ a)[:, 0] * f
    sums = (X[some].double().abs()[:, None] @ a.abs())[:, 0] * f
    size = (U[:, [0, R - 1]].abs() * 2.0 ** -16 + sums[:, [0, R - 1]] * K * 2.0 ** -24).sum(1, keepdim=True)
    close(Y, want, 2.0 ** -8 * want.abs() + size, f"{T} {R}")
    rounded = U.bfloat16().double()
    assert ((rounded[:, 0] - rounded[:, R - 1] - want[:, 0]).abs() > size[:, 0]).any()  # one part would not pass


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("start", [1 << 24, (1 << 31) - 9, -(1 << 31)])
def test_rotary_at_the_ends_of_the_positions(at, ref, start, layout):
    """Angles within 2^-26 turn and |pos| 2^-55 of the definition's."""
    for scaling in ("none", "ramp"):
        run_rotary(at, ref, 9, 2, 128, 128, layout, "f32", scaling=scaling, start=start)


@pytest.mark.parametrize("format", ["plain", "int8", "fp8"])
@pytest.mark.parametrize("layout,D,rot", [("halves", 128, 128), ("halves", 64, 32), ("neighbours", 128, 128), ("neighbours", 256, 48)])
def test_cache_rotates_keys_in_fp32(at, layout, D, rot, format):
    """The same bytes as rotating first and appending then."""
    g = gen_of(51, D, rot)
    T, H = 37, 3
    K, V = rand(g, T, H, D).cuda(), rand(g, T, H, D).cuda()
    pos = torch.randint(0, 200000, (T,), generator=g).to(torch.int32).cuda()
    steps, m = at.rotary_steps(rot, 10000.0, "ramp", 8.0, 4096)
    turn = at.make_rotary_shape(T, H, D, rot, layout, "f32", m)
    shape = at.make_cache_shape(2, H, D, "f32", format)
    places = (torch.randperm(128, generator=g)[:T]).to(torch.int32).cuda()
    a, b = at.alloc_cache(shape), at.alloc_cache(shape)
    for c in (a, b):
        for t in c:
            if t is not None:
                t.zero_()
    at.cache_append(shape, K, V, places, a, rotary=(turn, steps, pos))
    at.cache_append(shape, at.rotary(turn, K, pos, steps), V, places, b)
    for x, y in zip(a, b):
        assert x is y or torch.equal(x, y)


@pytest.mark.parametrize("dtype,format", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("ctx,drafts", [([0], [700]), ([1300], [257]), ([0, 500, 40, 3], [300, 1, 140, 1])])
def test_attend_prompts(at, ref, ctx, drafts, D, dtype, format):
    """Prompts of several hundred tokens: alone, on a context, beside single tokens of other requests."""
    g = gen_of(52, D, drafts[0])
    p = Paged(at, ref, g, ctx, drafts, 4, 2, D, dtype, format)
    check_attend(at, ref, p, 4, D, dtype, format, None)
    check_attend(at, ref, p, 4, D, dtype, format, None, max_keys=max(c + n for c, n in zip(ctx, drafts)), sum_keys=sum(ctx) + sum(drafts))
