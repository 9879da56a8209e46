"""Attention over 8-bit pages whose value scales are zero or far apart, against the plain 64-bit definitions in oracle/attention.py.

Tolerances.  Codes are exact, a probability times its scale is rounded to fp16 (2^-11 of it), scores are sums of at most 256 terms in fp32
(2^-11 of a probability for scores of a few hundred), and the output is rounded to bf16 (u = 2^-8).  Products far below the row's largest are
subnormal in fp16, to the nearest 2^-24: off by 2^-25 where the largest is 2^5 or more, and times a code, at most 2^-30 of the largest
product times value for each of n keys.  |err| <= 2^-9 sum p |v| + u |out| + 2^-30 n sum p amax, with the row's own probabilities and values.
"""
import pytest
import torch

from test_gpu_attention import Paged, at, close, gen_of, rand, ref, trees  # noqa: F401 (at, ref: fixtures)

pytestmark = pytest.mark.gpu

FORMATS = ["int8", "fp8"]
# drafted tokens of four query heads each: 4 to 160 columns, every number of tiles and sets of columns
DRAFTS = [1, 6, 12, 16, 40]
SHARED = dict(max_keys=200_000, sum_keys=200_000)  # planned for far more keys than there are: shares, and their join


def check(at, ref, p, D, tree, scale=None, H=4, **hints):
    scale = D ** -0.5 if scale is None else scale
    shape = at.make_attend_shape(p.shape, p.T, len(p.ctx), H, p.wide, max(p.drafts), scale, mask_words=None if tree is None else tree.shape[1], **hints)
    ws = at.attend_workspace(shape)
    ws.fill_(0xFF)
    out, lse = at.attend(shape, p.Q.cuda(), p.starts.cuda(), torch.tensor(p.ctx, dtype=torch.int32).cuda(),
                         None if tree is None else tree.cuda(), p.pages.cuda(), p.cache, ws)
    torch.cuda.synchronize()
    want, want_lse = ref.attend(p.Q, p.starts, p.ctx, tree, p.keys, p.values, scale)
    size, _ = ref.attend(p.Q, p.starts, p.ctx, tree, p.keys, [v.abs() for v in p.values], scale)
    floor, _ = ref.attend(p.Q, p.starts, p.ctx, tree, p.keys, [v.abs().amax(-1, keepdim=True).expand(v.shape) for v in p.values], scale)
    what = f"ctx={p.ctx} drafts={p.drafts} D={D} {hints}"
    close(lse, want_lse, 1e-5 * (1 + want_lse.abs().nan_to_num(0, 0, 0)), what + " lse")
    close(out, want, 2.0 ** -9 * size + 2.0 ** -8 * want.abs() + 2.0 ** -30 * max(len(k) for k in p.keys) * floor, what)
    return out


@pytest.mark.parametrize("hints", [{}, SHARED], ids=["whole", "shared"])
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", DRAFTS)
def test_values_that_are_zero(at, ref, n, D, format, hints):
    """Rows of zeros, whose scale is zero: all of them, the only ones of a page, the first pages, a wavefront's first."""
    g = gen_of(30, n, D)
    tree = trees(g, [n])
    for ctx, zeros in ((0, range(n)), (64, range(64, 64 + n)), (200, range(200 + n)), (200, range(64)), (330, range(320)), (330, range(256, 330 + n))):
        V = rand(g, ctx + n, 1, D, dtype="bf16")
        V[list(zeros)] = 0
        p = Paged(at, ref, g, [ctx], [n], 4, 1, D, "bf16", format, V=[V])
        for mask in (None, tree):
            out = check(at, ref, p, D, mask, **hints)
            assert V.any() or not out.any()
