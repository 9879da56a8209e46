"""Workspaces of the attention over the cache, sized once for the largest call (host only)."""
import ctypes
import random

import pytest

from paper_2505_06481_amd import build as mbuild


@pytest.fixture(scope="module")
def at():
    if mbuild.is_stale():
        mbuild.build()
    from paper_2505_06481_amd import attention
    return attention


def need(at, shape):
    """mmoe::attend_need: what a call of this shape takes of its workspace (mmoe_attend refuses less)."""
    f = getattr(at.lib(), "_ZN4mmoe11attend_needERK17mmoe_attend_shape")
    f.restype, f.argtypes = ctypes.c_size_t, [ctypes.c_void_p]
    return f(ctypes.addressof(shape))


def test_workspace_serves_smaller_batches(at):
    """Single tokens over up to 94 pages: 8 requests take more than 128 do."""
    cs = at.make_cache_shape(20000, 8, 128, "bf16", "int8")
    sizes = {n: at.attend_workspace_bytes(at.make_attend_shape(cs, n, n, 32, 94, 1, 1.0)) for n in (1, 2, 4, 8, 16, 64, 128, 512)}
    assert list(sizes.values()) == sorted(sizes.values())
    for n in sizes:
        assert need(at, at.make_attend_shape(cs, n, n, 32, 94, 1, 1.0)) <= sizes[n]


@pytest.mark.parametrize("dtype,format", [("bf16", "plain"), ("bf16", "int8"), ("bf16", "fp8"), ("f32", "plain")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_workspace_is_never_less_for_smaller_calls(at, D, dtype, format):
    rng = random.Random(D)
    for _ in range(150):
        kv, G = rng.choice([1, 2, 8, 32]), rng.choice([1, 4, 7, 16])
        cs = at.make_cache_shape(1000, kv, D, dtype, format)
        n, drafts, pages = (int(2 ** rng.uniform(0, top)) for top in (11, 9, 11))
        hint = rng.choice([0, 0, rng.randint(1, n * pages * 64)])
        whole = at.make_attend_shape(cs, n * drafts, n, kv * G, pages, drafts, 1.0, sum_keys=hint)
        most = at.attend_workspace_bytes(whole)
        assert most >= need(at, whole) > 0
        for _ in range(12):
            n2, d2, p2 = (max(1, int(x * rng.random() ** 3)) for x in (n, drafts, pages))
            keys = rng.choice([0, rng.randint(1, p2 * 64)])
            total = rng.randint(1, n2 * p2 * 64)
            if hint:
                total = min(total, hint)
            elif rng.random() < 0.3:
                total = 0
            T = rng.randint(1, n2 * d2)
            part = at.make_attend_shape(cs, T, n2, kv * G, p2, d2, 1.0, max_keys=keys, sum_keys=total)
            assert need(at, part) <= most and (hint or at.attend_workspace_bytes(part) <= most)


def test_grids_that_no_launch_has(at):
    """A launch has fewer than 2^32 threads: calls beyond are refused by the host, and no plan has a join beyond."""
    cs = at.make_cache_shape(1 << 20, 8, 128, "bf16", "int8")
    for n, prompt in ((2048, 4096), (512, 65536), (1 << 16, 64)):
        assert need(at, at.make_attend_shape(cs, n + prompt, n, 32, 2000, prompt, 1.0)) > 0
        assert at.attend_workspace_bytes(at.make_attend_shape(cs, n + prompt, n, 32, 2000, prompt, 1.0)) > 0
    one = at.make_cache_shape(1 << 20, 1, 128, "bf16", "int8")
    assert at.attend_workspace_bytes(at.make_attend_shape(one, 1 << 20, 1, 64, 2000, 1 << 20, 1.0)) > 0
    assert at.attend_workspace_bytes(at.make_attend_shape(one, 1 << 24, 1, 64, 2000, 1 << 24, 1.0)) == 0
