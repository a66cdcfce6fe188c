"""GPU parity of the orthogonalisation by Newton-Schulz products and of the optimiser step made of it against the fp64 oracle, over shapes,
tilings, types and groups of matrices, and what they refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_util import quant
from oracle import definition as D

pytestmark = pytest.mark.gpu

A, B, CC = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


def bound(want, steps=5, a=A):
    """Distance in the Frobenius norm that rounding may cost.  A perturbation of X grows by at most `a` per step (the iteration's slope at
    0, its largest), so one of the set-up by a^steps and one of step t by a^(steps - t): factors kept to 2^-22, sums to sqrt(k) 2^-24, for
    A, A^2 and B X, come to 8 times 2^-22 a^steps of |X_0| = 1 in all while the iterates are small, and to 64 times 2^-22 of the result once they
    are not."""
    return 2.0 ** -22 * (8 * a ** steps + 64 * np.linalg.norm(want))


def gradient(r, rows, cols, rank=None):
    """A falling spectrum over a floor of noise, as a few tokens make it."""
    k = rank or max(1, min(rows, cols) // 3)
    G = (r.standard_normal((rows, k)) / np.sqrt(1 + np.arange(k))) @ r.standard_normal((k, cols)) + 0.1 * r.standard_normal((rows, cols))
    return np.float32(1e-3 * G)


def ns(capi, steps=5, a=A, b=B, c=CC, eps=1e-7):
    return capi.nnt_newton_schulz_cfg(a, b, c, eps, steps)


def handles(mods, ts):
    return mods[0].ptr_array([t.h.value if t is not None else None for t in ts])


SHAPES = [((1, 1), (1, 1)), ((1, 40), (1, 40)), ((40, 1), (7, 1)), ((3, 5), (2, 2)), ((64, 64), (64, 64)), ((64, 256), (32, 32)), ((65, 63), (65, 63)), ((129, 400), (100, 128)),
          ((400, 129), (128, 100)), ((192, 192), (37, 64)), ((777, 1111), (300, 300)), ((1111, 777), (300, 300)), ((30, 2500), (30, 1000)), ((64, 5000), (64, 900)), ((4100, 33), (1000, 33)), ((20, 17000), (20, 17000)), ((64, 1024), (64, 1024)), ((64, 1089), (30, 500)), ((1536, 2100), (512, 512)), ((2100, 1536), (2100, 1536))]


@pytest.mark.parametrize("types", ["f32 f32", "bf16 bf16", "f32 bf16", "bf16 f32"])
@pytest.mark.parametrize("shape,base", SHAPES)
def test_orthogonalize(mods, shape, base, types):
    capi, tiled = mods
    tin, tout = types.split()
    G = quant(gradient(np.random.default_rng(sum(shape)), *shape), tin)
    want = D.orthogonalize(G)
    with tiled.Context(n_streams=2) as ctx:
        tG = tiled.TiledTensor.from_numpy(ctx, np.float32(G), base, tin)
        before = tG.buf.clone()
        tO = tiled.TiledTensor(ctx, tout, shape, base)
        tO.buf.fill_(0x5a)
        torch.cuda.synchronize()
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [tG]), handles(mods, [tO]))
        got = tO.download().astype(np.float64)
        half = 2.0 ** -8 if tout == "bf16" else 2.0 ** -24
        assert np.linalg.norm(got - want) <= bound(want) + half * np.linalg.norm(want)
        assert torch.equal(tG.buf, before)
        # the gaps between tiles stay as they were
        touched = torch.zeros_like(tO.buf, dtype=torch.bool)
        for k, idx in enumerate(tO.tile_index):
            n = int(np.prod(tO.tile_shape(idx))) * tO.esize
            touched[tO.offsets[k]:tO.offsets[k] + n] = True
        assert (tO.buf[~touched] == 0x5a).all()
        # in place: the same bit for bit
        if tin == tout:
            capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [tG]), handles(mods, [tG]))
            np.testing.assert_array_equal(tG.download(), np.float32(got))


@pytest.mark.parametrize("steps,a,b,c", [(1, A, B, CC), (2, A, B, CC), (3, 2.0, -1.5, 0.5), (12, 1.5, -0.5, 0.0), (8, A, B, CC)])
def test_iterations(mods, steps, a, b, c):
    capi, tiled = mods
    G = np.random.default_rng(1).standard_normal((150, 200)).astype(np.float32)
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    with tiled.Context(n_streams=1) as ctx:
        tG, tO = tiled.TiledTensor.from_numpy(ctx, G, (64, 100)), tiled.TiledTensor(ctx, "f32", G.shape, (64, 100))
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, steps, a, b, c)), 1, handles(mods, [tG]), handles(mods, [tO]))
        assert np.linalg.norm(tO.download() - want) <= bound(want, steps, a)


@pytest.mark.parametrize("shape", [(50, 70), (768, 2304), (700, 3000)])
@pytest.mark.parametrize("steps,a,b,c", [(1, A, B, CC), (2, A, B, CC), (3, A, B, CC), (4, 2.0, -1.5, 0.5), (7, 1.5, -0.5, 0.0)])
def test_iterations_of_narrow_and_of_long_matrices(mods, shape, steps, a, b, c):
    """One launch per step, and two steps at once with one left over or none."""
    capi, tiled = mods
    G = np.random.default_rng(2).standard_normal(shape).astype(np.float32)
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    with tiled.Context(n_streams=1) as ctx:
        tG, tO = tiled.TiledTensor.from_numpy(ctx, G, (64, 1000)), tiled.TiledTensor(ctx, "f32", G.shape, (64, 1000))
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, steps, a, b, c)), 1, handles(mods, [tG]), handles(mods, [tO]))
        assert np.linalg.norm(tO.download() - want) <= bound(want, steps, a)


@pytest.mark.parametrize("shape", [(64, 256), (256, 64), (64, 64), (60, 900), (200, 300), (300, 2000)])
def test_every_entry_of_one_step(mods, shape):
    """No entry is off by more than its own factors: 2^-20 (four times 2^-22) of a X and of the norms that B X is made of."""
    capi, tiled = mods
    for seed in range(3):
        G = gradient(np.random.default_rng(seed), *shape)
        want = D.orthogonalize(G, steps=1)
        X = G.astype(np.float64) / np.linalg.norm(G.astype(np.float64))
        X = X if shape[0] <= shape[1] else X.T
        S = X @ X.T
        limit = 2.0 ** -20 * (A * np.abs(X) + (abs(B) + CC) * np.linalg.norm(S, axis=1)[:, None] * np.linalg.norm(X, axis=0)[None, :])
        limit = limit if shape[0] <= shape[1] else limit.T
        with tiled.Context(n_streams=1) as ctx:
            tG, tO = tiled.TiledTensor.from_numpy(ctx, G, (100, 256)), tiled.TiledTensor(ctx, "f32", shape, (100, 256))
            capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, 1)), 1, handles(mods, [tG]), handles(mods, [tO]))
            d = np.abs(tO.download() - want)
            assert (d <= limit + 2.0 ** -24 * np.abs(want)).all(), (seed, (d / limit).max())


def test_pairs_of_steps_stay_in_range(mods):
    """Coefficients that the iteration itself can take, but not the polynomial of two steps: those go one by one."""
    capi, tiled = mods
    a, b, c = 3.9, -5.2, 2.1
    G = gradient(np.random.default_rng(8), 512, 2560)
    want = D.orthogonalize(G, a, b, c, 1e-7, 2)
    with tiled.Context(n_streams=1) as ctx:
        tG, tO = tiled.TiledTensor.from_numpy(ctx, G, (512, 2560)), tiled.TiledTensor(ctx, "f32", G.shape, (512, 2560))
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, 2, a, b, c)), 1, handles(mods, [tG]), handles(mods, [tO]))
        assert np.linalg.norm(tO.download() - want) <= bound(want, 2, a)


@pytest.mark.parametrize("shape", [(4096, 4096), (2500, 8300), (6000, 3000)])
def test_large_matrices(mods, shape):
    """The largest macro-tiles, ends inside them, tall and wide; against plain products in 64 bits on the device."""
    capi, tiled = mods
    g = torch.Generator(device="cuda").manual_seed(5)
    G = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)
    X = G.double() / torch.linalg.vector_norm(G.double())
    flip = shape[0] > shape[1]
    X = X.t().contiguous() if flip else X
    for _ in range(5):
        S = torch.mm(X, X.t())
        X = A * X + torch.mm(B * S + CC * torch.mm(S, S), X)
    want = X.t() if flip else X
    with tiled.Context(n_streams=2) as ctx:
        base = (3000, 3000)
        tG, tO = tiled.TiledTensor(ctx, "f32", shape, base), tiled.TiledTensor(ctx, "f32", shape, base)
        for k, idx in enumerate(tG.tile_index):
            tG.tile_view(k).copy_(G[tG.slices(idx)].t().reshape(-1))
        torch.cuda.synchronize()
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [tG]), handles(mods, [tO]))
        ctx.wait()
        err = 0.0
        for k, idx in enumerate(tO.tile_index):
            w = want[tO.slices(idx)]
            err += (tO.tile_view(k).view(w.shape[1], w.shape[0]).t().double() - w).square().sum().item()
        norm = torch.linalg.vector_norm(want).item()
        assert err ** 0.5 <= 2.0 ** -22 * (8 * A ** 5 + 64 * norm)


def test_offsets_beyond_32_bits(mods):
    """2.2e9 elements in one tile, the longest side there is; against the iteration of its Gram matrix in 64 bits.  A column more is refused."""
    capi, tiled = mods
    rows, cols = 520, 65535 * 64
    with tiled.Context(n_streams=1) as ctx:
        t = tiled.TiledTensor(ctx, "f32", (rows, cols), (rows, cols))
        G = t.buf.view(torch.float32).view(cols, rows)
        G.normal_(generator=torch.Generator(device="cuda").manual_seed(6))
        S = torch.zeros(rows, rows, device="cuda", dtype=torch.float64)
        for c in range(0, cols, 1 << 18):
            x = G[c:c + (1 << 18)].double()
            S += torch.mm(x.t().contiguous(), x)
        length = S.diagonal().sum().sqrt()
        S /= length ** 2
        Q = torch.eye(rows, device="cuda", dtype=torch.float64) / length
        for _ in range(5):
            F = A * torch.eye(rows, device="cuda", dtype=torch.float64) + B * S + CC * torch.mm(S, S)
            Q, S = torch.mm(F, Q), torch.mm(torch.mm(F, S), F)
        at = torch.cat([torch.arange(k, k + 70, device="cuda") for k in (0, 2 ** 31 // rows - 30, 2 ** 32 // rows // 2 + 200, cols - 70)])
        want = torch.mm(G[at].double(), Q.t().contiguous())
        torch.cuda.synchronize()
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [t]), handles(mods, [t]))
        ctx.wait()
        # The bound of the whole matrix is for its norm, here of `at`'s part of it.  Sums this long count by themselves: at least 8 parts of
        # A's contraction, 16 columns to an addition, each step's A off by 2^-24 of the root of their number, which b + 2 c = 9 passes on, five times.
        norm = torch.linalg.vector_norm(want).item()
        limit = bound(np.zeros(1)) * (len(at) / cols) ** 0.5 + bound(norm, a=0.0) + 2.0 ** -24 * norm * (1 + 45 * (cols / 128) ** 0.5)
        assert torch.linalg.vector_norm(G[at].double() - want).item() <= limit
        longer = tiled.TiledTensor(ctx, "bf16", (1, cols + 1), (1, cols + 1), fill=0)
        assert capi.nnt_orthogonalize.raw(ctx.h, C.byref(ns(capi)), 1, handles(mods, [longer]), handles(mods, [longer])) == capi.NNT_EINVAL


def test_contractions_of_very_different_lengths_in_one_group(mods):
    """The long contraction is cut into more parts than the short one has steps."""
    capi, tiled = mods
    r = np.random.default_rng(9)
    Gs = [gradient(r, 100, 6000), gradient(r, 70, 66), gradient(r, 130, 90)]
    with tiled.Context(n_streams=1) as ctx:
        G = [tiled.TiledTensor.from_numpy(ctx, x, (64, 1000)) for x in Gs]
        O = [tiled.TiledTensor(ctx, "f32", x.shape, (64, 1000)) for x in Gs]
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 3, handles(mods, G), handles(mods, O))
        for x, o in zip(Gs, O):
            want = D.orthogonalize(x)
            assert np.linalg.norm(o.download() - want) <= bound(want)


def test_scales_zeros_and_values_that_are_no_numbers(mods):
    """Gradients of any size (squares that overflow or vanish in fp32), single entries, zeros; NaN and infinity."""
    capi, tiled = mods
    r = np.random.default_rng(2)
    G = gradient(r, 100, 130)
    want = D.orthogonalize(G, eps=1e-30)
    one = np.zeros((100, 130), np.float32)
    one[57, 3] = 1e-8
    with tiled.Context(n_streams=2) as ctx:
        def run(G, eps):
            tG, tO = tiled.TiledTensor.from_numpy(ctx, np.float32(G), (64, 64)), tiled.TiledTensor(ctx, "f32", G.shape, (64, 64))
            capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, eps=eps)), 1, handles(mods, [tG]), handles(mods, [tO]))
            return tO.download()
        for scale in (1e30, 1e-25, 1e3):
            assert np.linalg.norm(run(np.float32(G * np.float32(scale)), 1e-30) - want) <= bound(want) + 2.0 ** -24 * A ** 5
        assert not run(np.zeros((100, 130)), 1e-7).any()
        assert np.linalg.norm(run(one, 1e-7) - D.orthogonalize(one, eps=1e-7)) <= bound(one)
        for v in (np.nan, np.inf):
            bad = G.copy()
            bad[3, 5] = v
            assert np.isnan(run(bad, 1e-7)).all()


@pytest.mark.parametrize("shape", [(20, 30), (100, 130)])
def test_lengths_near_the_ends_of_32_bits(mods, shape):
    """Matrices whose length, or 2^12 over it, fp32 does not hold, and an eps that it does not hold either."""
    capi, tiled = mods
    G = gradient(np.random.default_rng(3), *shape)
    with tiled.Context(n_streams=2) as ctx:
        for largest in (2.0 ** -123, 2.0 ** 127):
            x = np.float32(G / np.abs(G).max() * largest)
            want = D.orthogonalize(x, eps=1e-300)
            tG, tO = tiled.TiledTensor.from_numpy(ctx, x, (64, 64)), tiled.TiledTensor(ctx, "f32", G.shape, (64, 64))
            capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, eps=1e-300)), 1, handles(mods, [tG]), handles(mods, [tO]))
            assert np.linalg.norm(tO.download() - want) <= bound(want)
        zero = tiled.TiledTensor.from_numpy(ctx, np.zeros(shape, np.float32), (64, 64))
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi, eps=1e-300)), 1, handles(mods, [zero]), handles(mods, [tO]))
        assert not tO.download().any()


@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("scale", ["none", "aspect", "rms"])
@pytest.mark.parametrize("low", [False, True])
def test_muon_step_on_a_group(mods, nesterov, scale, low):
    """Matrices of different shapes and tilings in one call, two steps in a row."""
    capi, tiled = mods
    r = np.random.default_rng(3)
    shapes = [((192, 64), (32, 32)), ((64, 64), (64, 64)), ((256, 64), (100, 64)), ((64, 256), (64, 100)), ((5, 3), (2, 2)), ((300, 333), (128, 300)), ((1, 77), (1, 50))]
    code = dict(none=capi.NNT_MUON_SCALE_NONE, aspect=capi.NNT_MUON_SCALE_ASPECT, rms=capi.NNT_MUON_SCALE_RMS)[scale]
    cfg = capi.nnt_muon_cfg(0.05, 0.9, 0.1, nesterov, code, ns(capi))
    with tiled.Context(n_streams=2) as ctx:
        P, M, G = [[tiled.TiledTensor.from_numpy(ctx, np.float32(a(*s)), b) for s, b in shapes]
                   for a in (lambda *s: 0.02 * r.standard_normal(s), lambda *s: gradient(r, *s), lambda *s: gradient(r, *s))]
        LP = [tiled.TiledTensor(ctx, "bf16", s, b) if k % 2 == 0 else None for k, (s, b) in enumerate(shapes)] if low else None
        for _ in range(2):
            before = [(p.download(), m.download(), g.download()) for p, m, g in zip(P, M, G)]
            capi.nnt_muon_step(ctx.h, C.byref(cfg), len(shapes), handles(mods, G), handles(mods, P), handles(mods, M), handles(mods, LP) if low else None)
            for k, (p0, m0, g0) in enumerate(before):
                q, n = D.muon_step(p0, g0, m0, 0.05, 0.9, 0.1, bool(nesterov), scale)
                s = 0.05 * {"none": 1.0, "aspect": max(1.0, p0.shape[0] / p0.shape[1]) ** 0.5, "rms": 0.2 * max(p0.shape) ** 0.5}[scale]
                O = (0.995 * p0 - q) / s
                got = P[k].download().astype(np.float64)
                # M: a product and a sum, half a step each (a fused one: of the result); then the factors of U are off by as much
                assert np.abs(M[k].download() - n).max() <= 2.0 ** -23 * (np.abs(n).max() + np.abs(g0).max())
                # P: two roundings (the decayed parameter and the result), the constants' own
                add = 2.0 ** -22 * (np.linalg.norm(p0) + np.linalg.norm(q)) + s * 2.0 ** -22 * np.linalg.norm(O)
                assert np.linalg.norm(got - q) <= s * 1.5 * bound(O) + add, (k, np.linalg.norm(got - q))
                if low and LP[k] is not None:
                    np.testing.assert_array_equal(LP[k].download(), np.float32(quant(got, "bf16")))
                np.testing.assert_array_equal(G[k].download(), g0)


@pytest.mark.parametrize("shape,count", [((64, 64), 40), ((512, 512), 20), ((700, 300), 17)])
def test_many_matrices(mods, shape, count):
    """More matrices than one set of launches takes: each as by itself, up to the order of sums in larger macro-tiles."""
    capi, tiled = mods
    r = np.random.default_rng(4)
    with tiled.Context(n_streams=3) as ctx:
        Gs = [gradient(r, *shape) for _ in range(count)]
        G = [tiled.TiledTensor.from_numpy(ctx, g, (256, 256)) for g in Gs]
        O = [tiled.TiledTensor(ctx, "f32", shape, (256, 256)) for _ in Gs]
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), count, handles(mods, G), handles(mods, O))
        got = [o.download() for o in O]
        for k in {0, 1, 15, 16, count // 2, count - 1}:
            want = D.orthogonalize(Gs[k])
            assert np.linalg.norm(got[k] - want) <= bound(want)
        # again: the same bit for bit
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), count, handles(mods, G), handles(mods, O))
        for o, first in zip(O, got):
            np.testing.assert_array_equal(o.download(), first)


@pytest.mark.parametrize("shape", [(64, 256), (60, 500), (200, 300)])
def test_results_in_the_place_of_earlier_inputs(mods, shape):
    """O[k] = G[k - 1], eleven in a row: every input is read before its place is taken."""
    capi, tiled = mods
    n = 12
    G = [gradient(np.random.default_rng(k), *shape) for k in range(n)]
    with tiled.Context(n_streams=4) as ctx:
        t = [tiled.TiledTensor.from_numpy(ctx, g, (33, 256)) for g in G]
        t.append(tiled.TiledTensor(ctx, "f32", shape, (33, 256)))
        # G: 0 .. n-1; O: n, 0, 1, ...
        capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), n, handles(mods, t[:n]), handles(mods, [t[n]] + t[:n - 1]))
        for k in range(n):
            want = D.orthogonalize(G[k])
            assert np.linalg.norm((t[n] if k == 0 else t[k - 1]).download() - want) <= bound(want) + 2.0 ** -24 * np.linalg.norm(want)


def test_matrices_after_tasks_that_make_them(mods):
    """The step waits for the product that writes the gradient, and what reads the parameter waits for the step, on any streams."""
    capi, tiled = mods
    r = np.random.default_rng(5)
    e, n = 200, 96
    X, Y, P0 = r.standard_normal((e, n)).astype(np.float32), r.standard_normal((e, n)).astype(np.float32), 0.02 * r.standard_normal((e, e)).astype(np.float32)
    with tiled.Context(n_streams=4) as ctx:
        def T(a, dt="f32"):
            return tiled.TiledTensor.from_numpy(ctx, np.float32(a), (128, 128), dt)
        tX, tY, tP, tM, tG, tZ = T(X), T(Y), T(P0), T(np.zeros((e, e))), T(np.zeros((e, e))), T(np.zeros((e, n)))
        cfg = capi.nnt_muon_cfg(0.1, 0.9, 0.0, 1, capi.NNT_MUON_SCALE_NONE, ns(capi))
        p, m = P0.astype(np.float64), np.zeros((e, e))
        for _ in range(3):
            capi.nnt_gemm(ctx.h, 1.0, 0, tY.h, 1, tX.h, 0.0, tG.h, 1, 0, None)
            capi.nnt_muon_step(ctx.h, C.byref(cfg), 1, handles(mods, [tG]), handles(mods, [tP]), handles(mods, [tM]), None)
            capi.nnt_gemm(ctx.h, 1.0, 0, tP.h, 0, tX.h, 0.0, tZ.h, 1, 0, None)
            p, m = D.muon_step(p, Y.astype(np.float64) @ X.T, m, 0.1, 0.9)
        Z = p @ X
        assert np.abs(tZ.download() - Z).max() <= 1e-4 * np.abs(Z).max()


def test_captured_and_replayed(mods):
    capi, tiled = mods
    r = np.random.default_rng(6)
    with tiled.Context(n_streams=2) as ctx:
        def T(a):
            return tiled.TiledTensor.from_numpy(ctx, np.float32(a), (100, 128))
        P0 = 0.02 * r.standard_normal((200, 300))
        G, P, M = T(gradient(r, 200, 300)), T(P0), T(np.zeros((200, 300)))
        cfg = capi.nnt_muon_cfg(0.1, 0.9, 0.0, 1, 0, ns(capi))

        def go():
            capi.nnt_muon_step(ctx.h, C.byref(cfg), 1, handles(mods, [G]), handles(mods, [P]), handles(mods, [M]), None)
        g = C.c_void_p()
        capi.nnt_capture_begin(ctx.h)
        with pytest.raises(capi.NntError):                    # the workspace is not there yet
            go()
        capi.nnt_capture_end(ctx.h, C.byref(g))
        capi.nnt_graph_destroy(g)
        go()
        ctx.wait()
        capi.nnt_capture_begin(ctx.h)
        go()
        capi.nnt_capture_end(ctx.h, C.byref(g))
        for i in range(4):
            start = (P.download(), M.download())
            capi.nnt_graph_launch(g)
            replayed = (P.download(), M.download())
            P.upload(start[0])
            M.upload(start[1])
            if i == 1:                                        # an eager call that needs a larger workspace: the graph keeps its own
                big = T(gradient(r, 900, 1200))
                capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [big]), handles(mods, [big]))
            go()
            np.testing.assert_array_equal(P.download(), replayed[0])
            np.testing.assert_array_equal(M.download(), replayed[1])
        # narrow and other matrices in one call inside a capture: nothing is recorded if the workspace is too small
        narrow, wide = T(gradient(r, 40, 300)), T(gradient(r, 1500, 2000))
        capi.nnt_capture_begin(ctx.h)
        before = ctx.stats()["launches"]
        assert capi.nnt_orthogonalize.raw(ctx.h, C.byref(ns(capi)), 2, handles(mods, [narrow, wide]), handles(mods, [narrow, wide])) == capi.NNT_ESTATE
        assert ctx.stats()["launches"] == before
        empty = C.c_void_p()
        capi.nnt_capture_end(ctx.h, C.byref(empty))
        capi.nnt_graph_destroy(empty)
        held = ctx.stats()["device_workspace_bytes"]
        capi.nnt_graph_destroy(g)
        assert ctx.stats()["device_workspace_bytes"] < held


def test_calls_side_by_side(mods):
    """Calls that share the workspace by halves, between them one that takes all of it: on four streams the same bits as on one."""
    capi, tiled = mods
    shapes = [(300, 500), (200, 300), (65, 70), (40, 900), (64, 64), (4096, 4100), (300, 500), (900, 200), (30, 4000), (128, 900)]
    G = [torch.randn(*s, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") for k, s in enumerate(shapes)]
    results = []
    for streams in (1, 2, 4):
        with tiled.Context(n_streams=streams) as ctx:
            t, o = [[tiled.TiledTensor(ctx, "f32", s, s, fill=0) for s in shapes] for _ in range(2)]
            for x, g in zip(t, G):
                x.tile_view(0).copy_(g.t().reshape(-1))
            torch.cuda.synchronize()
            for _ in range(3):
                for x, y in zip(t, o):
                    capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), 1, handles(mods, [x]), handles(mods, [y]))
            ctx.wait()
            results.append([y.tile_view(0).clone() for y in o])
            torch.cuda.synchronize()
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    for g, a in zip(G[:5], results[0]):
        want = D.orthogonalize(g.cpu().numpy())
        assert np.linalg.norm(a.view(g.shape[1], g.shape[0]).t().cpu().numpy() - want) <= bound(want) + 2.0 ** -24 * np.linalg.norm(want)


def test_two_graphs_with_one_workspace(mods):
    """Matrices of every kind in two graphs that share the workspace, replayed in turn with an eager call between."""
    capi, tiled = mods
    r = np.random.default_rng(9)
    with tiled.Context(n_streams=4) as ctx:
        def group():
            G = [gradient(r, *s) for s in ((64, 64), (250, 60), (40, 300), (200, 300), (300, 1500))]
            t = [tiled.TiledTensor.from_numpy(ctx, g, (100, 128)) for g in G]
            o = [tiled.TiledTensor(ctx, "f32", g.shape, (100, 128)) for g in G]
            return G, t, o

        def go(t, o):
            capi.nnt_orthogonalize(ctx.h, C.byref(ns(capi)), len(t), handles(mods, t), handles(mods, o))
        groups, graphs, want = [group() for _ in range(3)], [], []
        for G, t, o in groups:
            go(t, o)
            want.append([x.download() for x in o])
            assert all(np.linalg.norm(w - D.orthogonalize(g)) <= bound(w) for w, g in zip(want[-1], G))
        for _, t, o in groups[:2]:
            g = C.c_void_p()
            capi.nnt_capture_begin(ctx.h)
            go(t, o)
            capi.nnt_capture_end(ctx.h, C.byref(g))
            graphs.append(g)
        for _ in range(4):
            for _, _, o in groups:
                for x in o:
                    x.buf.fill_(0x5a)
            torch.cuda.synchronize()
            capi.nnt_graph_launch(graphs[0])
            go(*groups[2][1:])
            capi.nnt_graph_launch(graphs[1])
            for (_, _, o), ws in zip(groups, want):
                for x, w in zip(o, ws):
                    np.testing.assert_array_equal(x.download(), w)
        for g in graphs:
            capi.nnt_graph_destroy(g)


def test_refusals(mods):
    capi, tiled = mods
    with tiled.Context(n_streams=1) as ctx, tiled.Context(n_streams=1) as other:
        def T(shape=(20, 30), b=(8, 30), dtype="f32", c=ctx, absent=None):
            return tiled.TiledTensor(c, dtype, shape, b, absent, fill=0)
        G, P, M, O = T(), T(), T(), T()
        low = T(dtype="bf16")

        def orth(cfg=None, g=G, o=O, n=1):
            return capi.nnt_orthogonalize.raw(ctx.h, C.byref(cfg or ns(capi)), n, handles(mods, [g]), handles(mods, [o]))

        def muon(cfg=None, g=G, p=P, m=M, lp=None, it=None, n=1):
            c = capi.nnt_muon_cfg(*(cfg or (0.1, 0.9, 0.0, 0, 0)), it or ns(capi))
            return capi.nnt_muon_step.raw(ctx.h, C.byref(c), n, handles(mods, [g]), handles(mods, [p]), handles(mods, [m]), handles(mods, [lp]) if lp else None)
        E = capi.NNT_EINVAL
        wrong = [T((20, 31), (8, 31)), T((20, 30), (10, 30)), T((20, 30, 1), (8, 30, 1)), T((20,), (8,)), T(c=other), T(absent=lambda idx: idx[0] == 1), None]
        for t in wrong:
            assert orth(o=t) == E and muon(g=t) == E and muon(p=t) == E and muon(m=t) == E
        for t in wrong[:-1] + [T()]:
            assert muon(lp=t) == E
        assert muon(p=low) == E and muon(m=low) == E and muon(g=low) == E
        assert orth(n=0) == E and muon(n=0) == E
        assert muon(p=G) == E and muon(m=G) == E and muon(m=P) == E
        nan, inf = float("nan"), float("inf")
        for it in (ns(capi, 0), ns(capi, 65), ns(capi, eps=0.0), ns(capi, eps=-1.0), ns(capi, eps=nan), ns(capi, a=nan), ns(capi, b=inf), ns(capi, a=20.0), ns(capi, 40, a=4.0, b=0.0, c=0.0), ns(capi, c=90.0)):
            assert orth(it) == E and muon(it=it) == E
        for cfg in ((-0.1, 0.9, 0.0, 0, 0), (nan, 0.9, 0.0, 0, 0), (0.1, 1.0, 0.0, 0, 0), (0.1, -0.1, 0.0, 0, 0), (0.1, 0.9, inf, 0, 0), (0.1, 0.9, 0.0, 0, 3), (0.1, 0.9, 0.0, 0, -1)):
            assert muon(cfg) == E
        two = capi.nnt_orthogonalize.raw
        assert two(ctx.h, C.byref(ns(capi)), 2, handles(mods, [G, P]), handles(mods, [O, O])) == E
        assert two(ctx.h, C.byref(ns(capi)), 2, handles(mods, [G, O]), handles(mods, [O, M])) == E
        c = capi.nnt_muon_cfg(0.1, 0.9, 0.0, 0, 0, ns(capi))
        assert capi.nnt_muon_step.raw(ctx.h, C.byref(c), 2, handles(mods, [G, G]), handles(mods, [P, P]), handles(mods, [M, O]), None) == E
        assert capi.nnt_muon_step.raw(ctx.h, None, 1, handles(mods, [G]), handles(mods, [P]), handles(mods, [M]), None) == E
        assert b"nnt_muon_step" in capi.nnt_last_error(ctx.h)
        assert orth() == capi.NNT_OK and muon(lp=low) == capi.NNT_OK                                        # the context is still good
        ctx.wait()
