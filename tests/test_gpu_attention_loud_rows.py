"""Values far larger than the others (finite, legal) in rows that a token does not see, or sees with a vanishing probability: over 8-bit pages
they share a scale range with the rest.  Tolerances as in test_gpu_attention_scales: from a token's own probabilities and values."""
import pytest
import torch

from test_gpu_attention import Paged, at, gen_of, rand, ref  # noqa: F401 (at, ref: fixtures)
from test_gpu_attention_scales import DRAFTS, FORMATS, SHARED, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hints", [{}, SHARED], ids=["whole", "shared"])
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", DRAFTS[1:])
def test_loud_rows_that_are_hidden(at, ref, n, D, format, hints):
    """Each drafted token sees itself and the context; some of them hold values of 2^k.  In a chunk only the last one does."""
    g = gen_of(31, n, D)
    for ctx, k in ((0, 30), (9, 20), (60, 34), (130, 100)):
        V = rand(g, ctx + n, 2, D, dtype="bf16")
        loud = V.clone()
        loud[ctx + 1::3] *= 2.0 ** k
        tree = torch.tensor([[1 << i] for i in range(n)], dtype=torch.int64)
        p = Paged(at, ref, g, [ctx], [n], 8, 2, D, "bf16", format, V=[loud])
        check(at, ref, p, D, tree, H=8, **hints)
        last = V.clone()
        last[-1] *= 2.0 ** k
        p = Paged(at, ref, g, [ctx], [n], 8, 2, D, "bf16", format, V=[last])
        check(at, ref, p, D, None, H=8, **hints)


@pytest.mark.parametrize("hints", [{}, SHARED], ids=["whole", "shared"])
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("n", DRAFTS)
def test_loud_rows_of_small_probability(at, ref, n, format, hints):
    """Loud rows with scores far below the others: first, last, and between them; and quiet rows whose probability is all there is."""
    g = gen_of(32, n)
    D = 64
    for rows, down, k in ((range(64), 200, 30), (range(0, 1), 40, 40), (range(300, 301), 40, 40), (range(100, 260), 90, 60), (range(0, 300, 7), 25, 24),
                          (range(0, 300, 7), 160, 100), (range(20, 330), 60, -60)):
        rows = list(rows)
        K, V = rand(g, 330 + n, 1, D, dtype="bf16"), rand(g, 330 + n, 1, D, dtype="bf16")
        K[..., 0] = 4.0
        K[rows, :, 0] = 4.0 - down / 8.0  # scores of 8 times the difference below
        V[rows] *= 2.0 ** k
        p = Paged(at, ref, g, [330], [n], 4, 1, D, "bf16", format, K=[K], V=[V])
        p.Q[..., 0] = 8.0
        check(at, ref, p, D, None, scale=1.0, **hints)


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("n", DRAFTS)
def test_scales_at_the_ends_of_their_range(at, ref, n, format):
    """Values of 2^-95 and of 2^100, alone, one after the other, and beside scores that rise all the time."""
    g = gen_of(33, n)
    D = 64
    for exponents in ((-95, -95), (100, 100), (-90, 90), (90, -90), (-30, 30)):
        K, V = rand(g, 500 + n, 1, D, dtype="bf16"), rand(g, 500 + n, 1, D, dtype="bf16").clamp(-4, 4)
        V *= 2.0 ** torch.linspace(*exponents, 500 + n).round()[:, None, None].to(V.dtype)
        for rise in (0.0, 60.0, -60.0):
            K[..., 0] = (torch.linspace(0.0, rise, 500 + n) / 8.0)[:, None].to(K.dtype)
            p = Paged(at, ref, g, [500], [n], 4, 1, D, "bf16", format, K=[K], V=[V])
            p.Q[..., 0] = 8.0
            check(at, ref, p, D, None, scale=1.0)


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("n", DRAFTS)
def test_scores_beyond_what_references_tell_apart(at, ref, n, format):
    """Scores of 10^8, whose neighbours in fp32 are tens apart, with loud and quiet values: one key is all there is."""
    g = gen_of(34, n)
    for k in (0, 20, -60, 90):
        K, V = rand(g, 200 + n, 1, 64, dtype="bf16"), rand(g, 200 + n, 1, 64, dtype="bf16")
        V[::2] *= 2.0 ** k
        p = Paged(at, ref, g, [200], [n], 4, 1, 64, "bf16", format, K=[K], V=[V])
        check(at, ref, p, 64, None, scale=1e7)


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("n", [1, 12, 16])
def test_loud_rows_in_every_step(at, ref, n, format):
    """A loud row of small probability on every page of a long context: the reference is looked at again and again, and stays what it is."""
    g = gen_of(35, n)
    ctx, D = 6000, 64
    K, V = rand(g, ctx + n, 1, D, dtype="bf16"), rand(g, ctx + n, 1, D, dtype="bf16")
    K[..., 0] = 4.0
    K[7:ctx:50, :, 0] = 4.0 - 60 / 8.0
    V[7:ctx:50] *= 2.0 ** 40
    p = Paged(at, ref, g, [ctx], [n], 4, 1, D, "bf16", format, K=[K], V=[V])
    p.Q *= 0.25
    p.Q[..., 0] = 8.0
    check(at, ref, p, D, None, scale=1.0)
    check(at, ref, p, D, None, scale=1.0, max_keys=ctx + n, sum_keys=ctx + n)
