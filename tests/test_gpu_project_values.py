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
