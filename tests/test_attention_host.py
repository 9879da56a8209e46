"""What the attention half's entry points refuse, and sizes that the host computes (no GPU: checks fail before any launch)."""
import ctypes

import pytest

from paper_2505_06481_amd import build as mbuild

P = ctypes.c_void_p(4096)  # never dereferenced
NONE = None
OK, NULL, DIM, DTYPE, WORKSPACE, ALIGN, MULTIPLE, LIMIT, HEAD, STRIDE, FORMAT = 0, -1, -2, -4, -6, -7, -8, -9, -12, -13, -14


@pytest.fixture(scope="module")
def at():
    if mbuild.is_stale():
        mbuild.build()
    from paper_2505_06481_amd import attention
    return attention


def project(at, shape, X=P, aid=P, Wp=P, Ap=P, Bp=P, scale=P, Y=P, ws=P, ws_bytes=1 << 40):
    return at._entry("mmoe_project")(ctypes.addressof(shape), X, aid, Wp, Ap, Bp, scale, Y, ws, ws_bytes, NONE)


def test_project_refuses(at):
    ok = (8, 256, 512, 3, 16, "bf16")
    make = at.make_project_shape
    for k in ("X", "aid", "Wp", "Ap", "Bp", "scale", "Y"):
        assert project(at, make(*ok), **{k: NONE}) == NULL, k
    assert project(at, make(*ok), ws=NONE) == WORKSPACE and project(at, make(*ok), ws_bytes=255) == WORKSPACE
    assert project(at, make(*ok), X=ctypes.c_void_p(4104)) == ALIGN and project(at, make(*ok), ws=ctypes.c_void_p(4096 + 16)) == ALIGN
    for bad, rc in (((0, 256, 512, 3, 16, 1), DIM), ((8, 0, 512, 3, 16, 1), DIM), ((8, 256, 512, -1, 16, 1), DIM), ((8, 256, 512, 3, 0, 1), DIM),
                    ((8, 256, 512, 3, 16, 2), DTYPE), ((8, 128, 512, 3, 16, 1), MULTIPLE), ((8, 256, 520, 3, 16, 1), MULTIPLE),
                    ((8, 256, 512, 3, 129, 1), LIMIT), ((8, 256, 512, 1025, 16, 1), LIMIT), ((8, 131072, 512, 3, 16, 1), LIMIT),
                    ((1 << 25, 256, 512, 3, 16, 1), LIMIT)):
        s = make(*bad)
        assert project(at, s) == rc, bad
        assert at.project_workspace_bytes(s) == 0
        assert at._entry("mmoe_pack_projection")(ctypes.addressof(s), P, P, NONE) == rc
    for ld in (dict(ldx=248), dict(ldx=260), dict(ldy=504), dict(ldy=516), dict(ldx=-256)):
        assert project(at, make(*ok, **ld)) == STRIDE, ld
    assert at._entry("mmoe_pack_adapters")(ctypes.addressof(make(8, 256, 512, 0, 0, 1)), P, P, P, P, NONE) == DIM


def test_project_workspace_grows_with_the_tokens(at):
    for dtype in ("bf16", "f32"):
        for n, R, K, N in ((0, 0, 4096, 4096), (2, 16, 4096, 6144), (64, 64, 768, 2304), (5, 100, 256, 256)):
            sizes = [at.project_workspace_bytes(at.make_project_shape(T, K, N, n, R, dtype)) for T in range(1, 700)] + \
                    [at.project_workspace_bytes(at.make_project_shape(T, K, N, n, R, dtype)) for T in (1024, 4096, 16384)]
            assert sizes == sorted(sizes)


def test_rotary_refuses(at):
    def call(shape, X=P, pos=P, steps=P, Y=P):
        return at._entry("mmoe_rotary")(ctypes.addressof(shape), X, pos, steps, Y, NONE)
    ok = dict(T=4, heads=3, head_dim=64, rot=32, layout=0, dtype=1)
    make = lambda **kw: at.make_rotary_shape(**(ok | kw))  # noqa: E731
    for k in ("X", "pos", "steps", "Y"):
        assert call(make(), **{k: NONE}) == NULL
        assert call(make(), **{k: ctypes.c_void_p(4098)}) == ALIGN
    for kw, rc in ((dict(T=0), DIM), (dict(heads=0), DIM), (dict(dtype=3), DTYPE), (dict(layout=2), FORMAT), (dict(transpose=2), FORMAT),
                   (dict(head_dim=60), HEAD), (dict(head_dim=528), HEAD), (dict(rot=0), HEAD), (dict(rot=24), HEAD), (dict(rot=80), HEAD)):
        assert call(make(**kw)) == rc, kw
    for strides in ((60, 0, 0, 0), (0, 32, 0, 0), (68, 64, 0, 0), (0, 0, 100, 64), (64, 64, 0, 0), (192, 65, 0, 0)):
        s = make()
        s.x_token, s.x_head, s.y_token, s.y_head = strides
        assert call(s) == STRIDE, strides
    steps, m = (ctypes.c_uint64 * 64)(), ctypes.c_float()
    f = at._entry("mmoe_rotary_steps")
    good = (64, 1e4, 0, 1.0, 0)
    assert f(*good, ctypes.addressof(steps), ctypes.addressof(m)) == OK and m.value == 1.0
    assert f(*good, NONE, ctypes.addressof(m)) == NULL
    for args, rc in (((60, 1e4, 0, 1.0, 0), HEAD), ((1024, 1e4, 0, 1.0, 0), HEAD), ((64, 1e4, 5, 1.0, 0), FORMAT), ((64, 1.0, 0, 1.0, 0), LIMIT),
                     ((64, float("nan"), 0, 1.0, 0), LIMIT), ((64, 1e4, 1, 0.5, 0), LIMIT), ((64, 1e4, 3, 2.0, 0), DIM)):
        assert f(*args, ctypes.addressof(steps), ctypes.addressof(m)) == rc, args


def test_cache_refuses(at):
    def append(shape, T=4, strides=(0, 0, 0, 0), K=P, V=P, places=P, turn=NONE, pos=P, steps=P, pointers=(P, P, P, P)):
        rows, c = at._CacheRows(T, *strides), at._CachePointers(*pointers)
        t = ctypes.addressof(turn) if turn is not None else NONE
        return at._entry("mmoe_cache_append")(ctypes.addressof(shape), ctypes.addressof(rows), K, V, places, t, pos, steps,
                                              ctypes.addressof(c), NONE)

    def read(shape, R=4, places=P, K=P, V=P, pointers=(P, P, P, P)):
        c = at._CachePointers(*pointers)
        return at._entry("mmoe_cache_read")(ctypes.addressof(shape), ctypes.addressof(c), R, places, K, V, NONE)
    ok = (4, 2, 64, "bf16", "int8")
    s = at.make_cache_shape(*ok)
    for bad, rc in (((0, 2, 64, 1, 1), DIM), ((4, 0, 64, 1, 1), DIM), ((4, 2, 96, 1, 1), HEAD), ((4, 2, 64, 5, 1), DTYPE), ((4, 2, 64, 1, 3), FORMAT),
                    ((1 << 26, 2, 64, 1, 1), LIMIT), ((4, 1025, 64, 1, 1), LIMIT)):
        b = at.make_cache_shape(*bad)
        assert append(b) == rc and read(b) == rc and at.cache_bytes(b) == (0, 0), bad
        with pytest.raises(ValueError):
            at.alloc_cache(b)
    for k in ("K", "V", "places"):
        assert append(s, **{k: NONE}) == NULL and append(s, **{k: ctypes.c_void_p(4098)}) == ALIGN
        assert read(s, **{k: NONE}) == NULL
    for i in range(4):
        pointers = [P] * 4
        pointers[i] = NONE
        assert append(s, pointers=pointers) == NULL and read(s, pointers=pointers) == NULL
        pointers[i] = ctypes.c_void_p(4100)
        assert append(s, pointers=pointers) == ALIGN
    assert append(s, T=0) == DIM and read(s, R=0) == DIM and append(s, T=1 << 25) == LIMIT
    for strides in ((100, 0, 0, 0), (0, 0, 0, 60), (130, 64, 0, 0), (64, 64, 0, 0)):
        assert append(s, strides=strides) == STRIDE, strides
    turn = at.make_rotary_shape(4, 2, 64, 64, "halves", "bf16")
    assert append(s, turn=turn, pos=NONE) == NULL and append(s, turn=turn, steps=NONE) == NULL
    assert append(s, turn=at.make_rotary_shape(4, 2, 128, 64, "halves", "bf16")) == HEAD
    assert append(s, turn=at.make_rotary_shape(4, 2, 64, 64, "halves", "f32")) == DTYPE
    assert append(s, turn=at.make_rotary_shape(4, 2, 64, 40, "halves", "bf16")) == HEAD


def test_cache_sizes(at):
    assert at.cache_bytes(at.make_cache_shape(3, 2, 128, "bf16", "plain")) == (3 * 2 * 64 * 128 * 2, 0)
    assert at.cache_bytes(at.make_cache_shape(3, 2, 128, "f32", "plain")) == (3 * 2 * 64 * 128 * 4, 0)
    assert at.cache_bytes(at.make_cache_shape(3, 2, 128, "f32", "int8")) == (3 * 2 * 64 * 128, 3 * 2 * 64 * 4)
    assert at.cache_bytes(at.make_cache_shape(1 << 22, 8, 128, "bf16", "fp8"))[0] == (1 << 22) * 8 * 64 * 128  # past 32 bits


def test_attend_refuses(at):
    def call(shape, Q=P, starts=P, ctx=P, tree=P, pages=P, out=P, lse=P, ws=P, ws_bytes=1 << 50, pointers=(P, P, P, P)):
        c = at._CachePointers(*pointers)
        return at._entry("mmoe_attend")(ctypes.addressof(shape), Q, starts, ctx, tree, pages, ctypes.addressof(c), out, lse, ws, ws_bytes, NONE)
    cache = at.make_cache_shape(8, 2, 64, "bf16", "int8")

    def make(cache=cache, **kw):
        words = kw.pop("mask_words", None)
        a = dict(T=6, n_requests=2, heads=4, max_pages=4, max_drafts=3, scale=0.125) | kw
        return at.make_attend_shape(cache, mask_words=words, **a)
    for k in ("Q", "starts", "ctx", "pages", "out"):
        assert call(make(), **{k: NONE}) == NULL, k
    for k in ("Q", "starts", "ctx", "tree", "pages", "out", "lse"):
        assert call(make(), **{k: ctypes.c_void_p(4098)}) == ALIGN, k
    assert call(make(), ws=NONE) == WORKSPACE and call(make(), ws_bytes=8) == WORKSPACE
    assert call(make(), pointers=(P, P, NONE, P)) == NULL
    for kw, rc in ((dict(T=0), DIM), (dict(n_requests=0), DIM), (dict(heads=0), DIM), (dict(max_pages=0), DIM), (dict(max_drafts=0), DIM),
                   (dict(heads=5), HEAD), (dict(heads=2 * 65), HEAD), (dict(max_pages=1 << 25), LIMIT), (dict(scale=float("nan")), LIMIT),
                   (dict(scale=float("inf")), LIMIT), (dict(mask_words=-1), DIM), (dict(max_keys=-1), DIM), (dict(sum_keys=-1), DIM)):
        s = make(**kw)
        assert call(s) == rc and at.attend_workspace_bytes(s) == 0, kw
    assert call(make(mask_words=0)) == DIM  # a tree without words
    assert call(make(cache=at.make_cache_shape(8, 2, 64, "f32", "int8"))) == FORMAT
    assert call(make(cache=at.make_cache_shape(8, 2, 72, "bf16", "plain"))) == HEAD
    assert call(make(n_requests=1 << 20, T=1 << 24, max_drafts=1 << 14)) == LIMIT  # a grid that does not fit
    s = make()
    s.q_token, s.q_head = 4 * 64, 60
    assert call(s) == STRIDE
    s = make()
    s.o_token, s.o_head = 4 * 64 - 8, 64
    assert call(s) == STRIDE


def test_binding_refuses(at):
    import torch
    cpu = torch.zeros(4, 256, dtype=torch.bfloat16)
    s = at.make_project_shape(4, 256, 256, 0, 0, "bf16")
    with pytest.raises(ValueError):
        at.project(s, cpu, None, cpu, None, None, None, cpu)
    with pytest.raises(ValueError):
        at.rotary(at.make_rotary_shape(4, 4, 64, 64, "halves", "bf16"), cpu.view(4, 4, 64), cpu, cpu, Y=cpu.view(4, 4, 64))
    with pytest.raises(KeyError):
        at.make_cache_shape(4, 1, 64, "bf16", "int4")
    with pytest.raises(KeyError):
        at.make_rotary_shape(4, 1, 64, 64, "thirds", "bf16")
