"""Projections with adapters: what U = scale X A carries into the second product.

All products by the 64-bit definition (oracle/attention.py).  Token counts and shapes reach each of the ways in which U B is added: beside parts joined
afterwards, by tiles of both sizes, and apart for weights that are not finite."""
import math

import pytest
import torch

from test_gpu_attention import DT, at, close, gen_of, rand, ref  # noqa: F401 (at, ref: fixtures)

pytestmark = pytest.mark.gpu

SIZES = [(24, 256, 512), (300, 256, 512), (5000, 256, 512), (4200, 256, 4352)]


def project(at, X, aid, W, A, B, scale, dtype):
    (T, K), N, (n, _, R) = X.shape, W.shape[1], A.shape
    shape = at.make_project_shape(T, K, N, n, R, dtype)
    ws = at.project_workspace(shape)
    ws.fill_(0xFF)
    return at.project(shape, X.cuda(), aid.cuda(), at.pack_projection(shape, W.cuda()), *at.pack_adapters(shape, A.cuda(), B.cuda()), scale.cuda(), ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [1, 12, 16, 40])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_inputs_that_are_infinite(at, ref, T, K, N, R, dtype):
    """An infinity in X, positive weights: infinities in the token's whole row, as in the formula, whatever the rank is padded to."""
    g = gen_of(40, T, R)
    X, W = rand(g, T, K, dtype=dtype), rand(g, K, N, dtype=dtype).abs() + 0.5
    A, B = rand(g, 2, K, R, dtype=dtype).abs() + 0.5, rand(g, 2, R, N, dtype=dtype).abs() + 0.5
    X[3, 7], X[T - 2, 200], X[5, 0] = math.inf, -math.inf, math.nan
    aid = torch.arange(T, dtype=torch.int32) % 3 - 1
    aid[3], aid[T - 2], aid[5], aid[4] = 0, 1, 1, 0
    some = torch.tensor([3, T - 2, 5, 4])
    Y = project(at, X, aid, W, A, B, torch.ones(2), dtype).cpu()[some]
    want = ref.project(X[some], aid[some], W, A, B, torch.ones(2))
    assert torch.isinf(want[:2]).all() and torch.isnan(want[2]).all() and torch.isfinite(want[3]).all()
    close(Y[:3], want[:3], 0.0)
    assert torch.isfinite(Y[3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_weights_that_are_infinite(at, ref, T, K, N, dtype):
    """An infinity in an adapter's B gives the infinity of its sign, and NaN only where the formula does: where U is zero, or two of them meet."""
    g = gen_of(41, T)
    X, W = rand(g, T, K, dtype=dtype), rand(g, K, N, dtype=dtype, scale=1 / 16)
    A, B = rand(g, 3, K, 8, dtype=dtype, scale=1 / 16), rand(g, 3, 8, N, dtype=dtype)
    B[1, 3, ::2], B[1, 5, 1::8], B[1, 6, 4::32] = math.inf, -math.inf, math.inf
    aid = torch.arange(T, dtype=torch.int32) % 4
    aid[3:9] = 1
    X[4] = 0                                      # U is zero
    X[5] = 0
    X[5, 9], A[1, 9] = 1.0, 0.25                  # U is a power of two: its second part is zero
    some = torch.arange(24)
    Y = project(at, X, aid, W, A, B, torch.ones(3), dtype).cpu()[some]
    want = ref.project(X[some], aid[some], W, A, B, torch.ones(3))
    assert torch.isinf(want[5, ::2]).all() and torch.isnan(want[4, ::2]).all()
    hit = aid[some] == 1
    assert torch.equal(torch.isnan(Y), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(Y), inf) and torch.equal(Y[inf].double(), want[inf])
    assert inf[hit].any() and not inf[~hit].any()


@pytest.mark.parametrize("T,K,N", SIZES)
def test_adapters_near_the_end_of_the_range(at, ref, T, K, N):
    """U between bf16's largest number and fp32's, which rounds to infinity in bf16, and one that is tiny: both times B are ordinary numbers."""
    g = gen_of(42, T)
    X, W = torch.zeros(T, K, dtype=torch.bfloat16), torch.zeros(K, N, dtype=torch.bfloat16)
    X[:, 0] = 2.0 ** 64
    A, B = torch.zeros(2, K, 4, dtype=torch.bfloat16), rand(g, 2, 4, N, dtype="bf16")
    A[0, 0], A[1, 0] = 1.9921875 * 2.0 ** 63, 1.9921875 * 2.0 ** -124
    B[0] *= 2.0 ** -110
    B[1] *= 2.0 ** 60
    aid, scale = torch.arange(T, dtype=torch.int32) % 2, torch.tensor([1.003, 1.003])
    some = torch.tensor([0, 1, T - 2, T - 1])
    Y = project(at, X, aid, W, A, B, scale, "bf16")[some.cuda()]
    want, size = (ref.project(X[some], aid[some], W, A, b, scale) for b in (B, B.abs()))
    close(Y, want, 2.0 ** -8 * want.abs() + 2.0 ** -15 * size)  # 2^-16 of U, and fp32 sums of four
