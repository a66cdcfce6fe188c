"""The norm of many gradients and the clipped ones against the oracle: tile sizes, types, lists longer than a launch, values whose
squares leave fp32's range, infinities, captured graphs, the block's and the model's gradients, refusals."""
import ctypes as C

import numpy as np
import pytest

import workload
from oracle import rollout as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS32 = 2.0 ** -24
HALF = {"f32": EPS32, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_13236_amd import tiled
    c = tiled.Context(n_streams=2)
    yield c
    c.close()


def quant(a, dtype):
    a = np.asarray(a, np.float32)
    return workload.round_through_bf16(a.reshape(-1)).reshape(a.shape) if dtype == "bf16" else a


def gradients(seed, shapes, dtypes, std=1.0):
    r = np.random.default_rng(seed)
    return [quant(std * r.standard_normal(s), d) for s, d in zip(shapes, dtypes)]


def check(got, norm, G, dtypes, max_norm, eps):
    want, n = R.clip_grad_norm(G, max_norm, eps)
    # the norm in 64 bits, rounded to fp32 once; the factor in 64 bits, each product rounded once to fp32 and once to the type
    assert abs(norm - n) <= EPS32 * n, (norm, n)
    for g, w, d in zip(got, want, dtypes):
        bound = (HALF[d] + (EPS32 if d == "bf16" else 0.0)) * np.abs(w) * (1 + 1e-6) + 2.0 ** -150
        assert (np.abs(g - w) <= bound).all()


SETS = {
    "one": ([(1,)], ["f32"]),
    "odd": ([(7, 5), (13,), (3, 4, 5), (2, 3, 2, 3), (1, 1)], ["f32", "bf16", "f32", "bf16", "f32"]),
    "pieces": ([(300, 400), (16384,), (16385,), (40000, 3)], ["f32", "bf16", "f32", "bf16"]),
    "many": ([(5 + k, 1 + k % 7) for k in range(150)], ["f32", "bf16"] * 75),
}


@pytest.mark.parametrize("name", sorted(SETS))
@pytest.mark.parametrize("tile", [1000000, 64, 7])
@pytest.mark.parametrize("max_norm", [1.0, 1e9])
@pytest.mark.parametrize("in_place", [False, True])
def test_sets(ctx, name, tile, max_norm, in_place):
    from paper_2504_13236_amd import tiled
    shapes, dtypes = SETS[name]
    if name == "pieces" and tile == 7:
        tile = 100
    G = gradients(1, shapes, dtypes)
    T = [tiled.TiledTensor.from_numpy(ctx, g, (tile,) * g.ndim, d) for g, d in zip(G, dtypes)]
    O = T if in_place else [tiled.TiledTensor.zeros(ctx, g.shape, (tile,) * g.ndim, d) for g, d in zip(G, dtypes)]
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, T, norm, O=O, max_norm=max_norm, eps=1e-6)
    got = [o.download() for o in O]
    check(got, float(norm), G, dtypes, max_norm, 1e-6)
    if not in_place:
        assert all(np.array_equal(t.download(), g) for t, g in zip(T, G))
        ctx.wait()
        norm.zero_()
        torch.cuda.synchronize()
        tiled.clip_grad_norm(ctx, T, norm)                     # the norm alone
        ctx.wait()
        assert abs(float(norm) - R.clip_grad_norm(G, 1.0, 0.0)[1]) <= EPS32 * float(norm)
    if max_norm > 1e8:
        assert all(np.array_equal(g, w) for g, w in zip(got, G))      # not clipped: the same bits
    for t in set(T + O):
        t.close()


@pytest.mark.parametrize("std", [1e-30, 1e-23, 1e20, 1e37])
def test_squares_beyond_fp32(ctx, std):
    from paper_2504_13236_amd import tiled
    G = gradients(2, [(1000,), (33, 3)], ["f32", "f32"], std)
    T = [tiled.TiledTensor.from_numpy(ctx, g, (128,) * g.ndim) for g in G]
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, T, norm, O=T, max_norm=1e-3 * std, eps=0.0)
    got = [t.download() for t in T]
    check(got, float(norm), G, ["f32", "f32"], 1e-3 * std, 0.0)
    for t in T:
        t.close()


@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_norm_that_is_no_number_leaves_the_gradients(ctx, what, in_place):
    from paper_2504_13236_amd import tiled
    g = gradients(3, [(50, 7)], ["f32"])[0]
    g[17, 3] = what
    t = tiled.TiledTensor.from_numpy(ctx, g, (20, 7))
    o = t if in_place else tiled.TiledTensor.zeros(ctx, g.shape, (20, 7))
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, [t], norm, O=[o], max_norm=1e-3)
    got = o.download()
    assert np.array_equal(got, g, equal_nan=True)
    assert np.isnan(float(norm)) if np.isnan(what) else float(norm) == np.inf
    for x in {t, o}:
        x.close()


def test_zero_gradients_and_absent_tiles(ctx):
    from paper_2504_13236_amd import tiled
    absent = lambda i: i[0] == 1
    g = gradients(4, [(30, 8)], ["f32"])[0]
    g[10:20] = 0.0
    t, z = tiled.TiledTensor.from_numpy(ctx, g, (10, 8), absent=absent), tiled.TiledTensor.zeros(ctx, (100,), (30,))
    o = tiled.TiledTensor.zeros(ctx, (30, 8), (10, 8), absent=absent)
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, [t, z], norm, O=[o, z], max_norm=0.5)
    check([o.download(), z.download()], float(norm), [g, np.zeros(100)], ["f32", "f32"], 0.5, 1e-6)
    tiled.clip_grad_norm(ctx, [z], norm, O=[z], max_norm=0.5, eps=0.0)          # a norm of zero
    assert not z.download().any() and float(norm) == 0.0
    tiled.clip_grad_norm(ctx, [t], norm, O=[t], max_norm=float("inf"))
    assert np.array_equal(t.download(), g)
    for x in (t, z, o):
        x.close()


def test_large_tiles_and_fixed_order(ctx):
    """64 M elements in one tile and in many: the same bits run after run."""
    from paper_2504_13236_amd import tiled
    n = (1 << 26) + 3
    t = tiled.TiledTensor.zeros(ctx, (n,), (n,))
    v = t.tile_view(0)
    v.copy_(torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"))
    want = float(v.double().square().sum().sqrt())
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    seen = set()
    for _ in range(4):
        tiled.clip_grad_norm(ctx, [t], norm)
        ctx.wait()
        seen.add(float(norm))
    assert len(seen) == 1 and abs(seen.pop() - want) <= EPS32 * want * 1.001
    before = v.clone()
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, [t], norm, O=[t], max_norm=3.0)
    ctx.wait()
    f = 3.0 / (want + 1e-6)
    assert float((v.double() - before.double() * f).abs().max()) <= EPS32 * float(before.abs().max()) * f * (1 + 1e-6)
    t.close()


def to_bf16(v):
    """64-bit values in bf16's normal range, rounded to its 8 bits once, ties to even."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(m * 256.0) / 256.0, e)


@pytest.mark.parametrize("n", [1, 100003])
@pytest.mark.parametrize("factor", [0.5 * (1 + 3 * 2.0 ** -8) * (1 - 2.0 ** -40), 0.5 * (1 + 2.0 ** -8) * (1 + 2.0 ** -40), 0.3, 1.0 / 3.0])
def test_bf16_results_are_rounded_once(ctx, n, factor):
    """Products next to the middle between two bf16 numbers, nearer to it than fp32 can tell: rounded to fp32 on the way they would fall on it."""
    from paper_2504_13236_amd import tiled
    r = np.random.default_rng(11)
    g = np.zeros(n) if n > 1 else np.ones(1)
    if n > 1:
        # one 1.0 makes up the norm, next to which the squares of the others vanish in 64 bits
        g = to_bf16(2.0 ** -60 * (1.0 + r.random(n)) * r.choice([-1.0, 1.0], n))
        g[n // 2], g[n // 3] = 1.0, -2.0 ** -60
    t, o = tiled.TiledTensor.from_numpy(ctx, g, (1000,), "bf16"), tiled.TiledTensor.zeros(ctx, (n,), (1000,), "bf16")
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, [t], norm, O=[o], max_norm=factor, eps=0.0)
    got = o.download().astype(np.float64)
    assert float(norm) == 1.0
    assert np.array_equal(got, to_bf16(g * factor))
    t.close()
    o.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_norm_beyond_fp32(ctx, dtype):
    """Finite in 64 bits: the gradients are clipped by it, and the caller is told infinity."""
    from paper_2504_13236_amd import tiled
    G = [quant(np.full((40,), 3e38), dtype), quant(np.array([1e30, -2e38]), dtype)]
    T = [tiled.TiledTensor.from_numpy(ctx, g, (16,), dtype) for g in G]
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, T, norm, O=T, max_norm=1e3)
    want, n = R.clip_grad_norm(G, 1e3, 1e-6)
    assert 3.4028236e38 < n < np.inf and float(norm) == np.inf
    for t, w in zip(T, want):
        assert (np.abs(t.download() - w) <= HALF[dtype] * np.abs(w) * (1 + 1e-6)).all()
        t.close()


def test_a_small_tile_beside_one_of_more_than_2_31_elements(ctx):
    """Tiles of 65536 x 32770 bf16 elements and what is left, 65536 x 1: the memory behind the small one is not looked at."""
    from paper_2504_13236_amd import capi, tiled
    big, small = 65536 * 32770, 65536
    buf = torch.full((big + small + 4096,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    buf[big + small:] = float("inf")
    h = C.c_void_p()
    capi.nnt_tensor_create(ctx.h, capi.NNT_BF16, 2, capi.i64_array((65536, 32771)), capi.i64_array((65536, 32770)),
                           capi.ptr_array([buf.data_ptr(), buf.data_ptr() + 2 * big]), C.byref(h))
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    cfg = capi.nnt_clip_cfg(2.0 ** -3, 0.0)
    capi.nnt_clip_grad_norm(ctx.h, C.byref(cfg), 1, capi.ptr_array([h.value]), capi.ptr_array([h.value]), norm.data_ptr())
    ctx.wait()
    # 65536 * 32771 squares of 2^-10: their sum is a whole multiple of 2^-20, exact in 64 bits
    want = (65536 * 32771) ** 0.5 * 2.0 ** -10
    assert abs(float(norm) - want) <= EPS32 * want
    clipped = 2.0 ** -10 * 2.0 ** -3 / want
    for part in (buf[:1 << 20], buf[big - (1 << 20):big + small]):
        assert float((part.double() - clipped).abs().max()) <= (HALF["bf16"] + EPS32) * clipped
    assert torch.isinf(buf[big + small:]).all()
    capi.nnt_tensor_destroy(h)


def test_captured_and_replayed(ctx):
    from paper_2504_13236_amd import capi, tiled
    G = gradients(5, [(64, 64), (64,), (100, 33)], ["f32"] * 3)
    T = [tiled.TiledTensor.from_numpy(ctx, g, (48,) * g.ndim) for g in G]
    norm = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    tiled.clip_grad_norm(ctx, T, norm)
    ctx.wait()
    g = C.c_void_p()
    capi.nnt_capture_begin(ctx.h)
    tiled.clip_grad_norm(ctx, T, norm, O=T, max_norm=2.0)
    capi.nnt_capture_end(ctx.h, C.byref(g))
    for k in range(4):
        G = gradients(60 + k, [x.shape for x in G], ["f32"] * 3, std=10.0 ** (k - 2))
        for t, x in zip(T, G):
            t.upload(x)
        capi.nnt_graph_launch(g)
        check([t.download() for t in T], float(norm), G, ["f32"] * 3, 2.0, 1e-6)
        tiled.clip_grad_norm(ctx, T, norm)
        ctx.wait()
    capi.nnt_graph_destroy(g)
    for t in T:
        t.close()


@pytest.mark.parametrize("granularity", [0, 1])
def test_gradients_of_blocks_and_models(granularity):
    """nnt_gpt2_block_clip, _stack_clip, _model_clip: all of the gradients and nothing else."""
    from paper_2504_13236_amd import capi, tiled
    tiles = dict(e=16, m=32, s=8, b=2, j=2, i=16)
    with tiled.Context(n_streams=3, granularity=granularity) as ctx:
        blocks = [tiled.Gpt2Block(ctx, 32, 2, 64, 16, 2, tiles, adam=False) for _ in range(2)]
        model = tiled.Gpt2Model(ctx, blocks, 50, 20)
        norm = torch.zeros(1, device="cuda")
        r = np.random.default_rng(7)

        def fill():
            G = []
            for slots in [b.slots[capi.NNT_BLK_GRAD:capi.NNT_BLK_GRAD + 12] for b in blocks] + [model.slots[capi.NNT_MDL_GRAD:capi.NNT_MDL_GRAD + 4]]:
                G.append([(t, r.standard_normal(t.shape).astype(np.float32)) for t in slots])
                for t, a in G[-1]:
                    t.upload(a)
            return G

        for who, which in ((blocks[1], [1]), (model.stack, [0, 1]), (model, [0, 1, 2])):
            G = fill()
            who.clip(norm, max_norm=3.0, eps=1e-6)
            ctx.wait()
            mine = [x for k in which for x in G[k]]
            check([t.download() for t, _ in mine], float(norm), [a for _, a in mine], ["f32"] * len(mine), 3.0, 1e-6)
            for k in set(range(3)) - set(which):
                assert all(np.array_equal(t.download(), a) for t, a in G[k])
        model.close()
        for b in blocks:
            b.close()


def test_refusals(ctx):
    from paper_2504_13236_amd import capi, tiled
    T = tiled.TiledTensor
    a, b, c = (T.zeros(ctx, (30, 20), (10, 20)) for _ in range(3))
    wrong = [T.zeros(ctx, (30, 21), (10, 21)), T.zeros(ctx, (30, 20), (15, 20)), T.zeros(ctx, (30, 20), (10, 20), "bf16"),
             T.zeros(ctx, (30, 20), (10, 20), absent=lambda i: i[0] == 2)]
    norm = torch.full((1,), -3.0, device="cuda")
    torch.cuda.synchronize()

    def call(G, O, max_norm=1.0, eps=1e-6, n=None, norm=norm.data_ptr()):
        cfg = capi.nnt_clip_cfg(max_norm, eps)
        arr = lambda L: capi.ptr_array([t.h.value if t is not None else None for t in L]) if L is not None else None
        return capi.nnt_clip_grad_norm.raw(ctx.h, C.byref(cfg), len(G) if n is None else n, arr(G), arr(O), norm)
    bad = capi.NNT_EINVAL
    nan = float("nan")
    assert call([a], None, n=0) == bad and call([a], None, n=-1) == bad and call([a], None, norm=None) == bad
    for kw in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=nan), dict(eps=-1e-9), dict(eps=nan), dict(eps=float("inf"))):
        assert call([a], [a], **kw) == bad, kw
    assert call([a, None], None) == bad and call([a], [None]) == bad
    assert call([a, a], None) == bad and call([a, b], [c, c]) == bad and call([a, b], [b, a]) == bad and call([a, b], [b, c]) == bad
    for w in wrong:
        assert call([a], [w]) == bad
    assert capi.nnt_clip_grad_norm.raw(ctx.h, None, 1, capi.ptr_array([a.h.value]), None, norm.data_ptr()) == bad
    assert capi.nnt_clip_grad_norm.raw(ctx.h, C.byref(capi.nnt_clip_cfg(1.0, 0.0)), 1, None, None, norm.data_ptr()) == bad
    with tiled.Context(n_streams=1) as other:
        x = T.zeros(other, (30, 20), (10, 20))
        assert call([x], None) == bad and call([a], [x]) == bad
        x.close()
    ctx.wait()
    assert float(norm) == -3.0
    assert call([a, b], [a, c]) == capi.NNT_OK
    ctx.wait()
    assert float(norm) == 0.0
    for t in [a, b, c] + wrong:
        t.close()
