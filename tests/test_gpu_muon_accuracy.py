"""How far the orthogonalisation is from 64 bits beside the same iteration with fp32 products, also on matrices whose rows, columns or values
differ by many orders of magnitude."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import definition as D

pytestmark = pytest.mark.gpu

A, B, CC = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


def handles(mods, ts):
    return mods[0].ptr_array([t.h.value for t in ts])


def fp32_products(G, steps, eps, a=A, b=B, c=CC):
    """The iteration with everything in fp32, by the installed library's products."""
    flip = G.shape[0] > G.shape[1]
    X = G.T if flip else G
    X = torch.from_numpy(np.ascontiguousarray(X.astype(np.float64) / (np.linalg.norm(X.astype(np.float64)) + eps), dtype=np.float32)).cuda()
    for _ in range(steps):
        S = torch.mm(X, X.t())
        X = a * X + torch.mm(b * S + c * torch.mm(S, S), X)
    X = X.cpu().numpy().astype(np.float64)
    return X.T if flip else X


def orthogonalize(mods, G, steps, eps, base, a=A, b=B, c=CC):
    capi, tiled = mods
    with tiled.Context(n_streams=1) as ctx:
        tG, tO = tiled.TiledTensor.from_numpy(ctx, G, base), tiled.TiledTensor(ctx, "f32", G.shape, base)
        cfg = capi.nnt_newton_schulz_cfg(a, b, c, eps, steps)
        capi.nnt_orthogonalize(ctx.h, C.byref(cfg), 1, handles(mods, [tG]), handles(mods, [tO]))
        return tO.download().astype(np.float64)


def falling(r, m, n):
    k = max(1, min(m, n) // 3)
    return np.float32(1e-3 * ((r.standard_normal((m, k)) / np.sqrt(1 + np.arange(k))) @ r.standard_normal((k, n)) + 0.1 * r.standard_normal((m, n))))


# The usual coefficients for five steps.  Once a singular value s has arrived, they make it go to and fro between 0.7 and 1.2, and a deviation of it grows by the
# slope a + 3 b s^2 + 5 c s^4, 3.8 at 1.2, from step to step, whatever the arithmetic: two results of 20 steps are as far apart as chance has it (fp32 products between
# 3e-6 and 5e-5).  Long iterations are therefore those of coefficients that arrive at 1 with slope 0 (2 - 4.5 + 2.5) and double small values.
USUAL, LONG = (5, A, B, CC), (45, 2.0, -1.5, 0.5)

# two steps at once, cut contractions, single steps, one launch, a launch per step; either orientation
SHAPES = [(512, 2560), (2560, 512), (256, 1536), (300, 333), (333, 300), (60, 200), (200, 60), (48, 2000), (2000, 48)]

# The error as a whole.  A value of two fp16 halves is off by 0.85 times 2^-24 of its size (root of the mean square), one of fp32 by 0.42; the term
# lo lo that a product leaves out is 0.72 times 2^-24 of it.  A product of two rounded factors: the root of 2 * 0.85^2 + 0.72^2 = 1.40 against that of
# 2 * 0.42^2 = 0.59, 2.4 times as much, if the sums, which are in fp32 either way, cost nothing.
WHOLE = 2.5


@pytest.mark.parametrize("kind", ["gauss", "falling", "columns"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("iteration", [USUAL, LONG])
def test_as_near_to_64_bits_as_fp32_products(mods, shape, iteration, kind):
    steps, a, b, c = iteration
    r = np.random.default_rng(sum(shape))
    G = falling(r, *shape) if kind == "falling" else r.standard_normal(shape).astype(np.float32)
    if kind == "columns":                                     # along the long side, six orders of magnitude
        s = 10.0 ** r.uniform(-6, 0, max(shape))
        G = np.float32(G * (s[None, :] if shape[0] < shape[1] else s[:, None]))
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    plain = np.linalg.norm(fp32_products(G, steps, 1e-7, a, b, c) - want)
    got = np.linalg.norm(orthogonalize(mods, G, steps, 1e-7, (256, 1024), a, b, c) - want)
    assert got <= WHOLE * plain, "%.2e of the result, fp32 products %.2e" % (got / np.linalg.norm(want), plain / np.linalg.norm(want))


# One row's error: a factor is off by up to 2^-22 of its size (two halves of 11 bits) or 2^-24 (fp32), four times as much.
ROW = 4.0


def rows_off(got, want, columns=False):
    """Largest error of a row of X (or of a column) in its length."""
    d, w = (got - want, want) if (got.shape[0] <= got.shape[1]) != columns else ((got - want).T, want.T)
    return (np.linalg.norm(d, axis=1) / np.linalg.norm(w, axis=1)).max()


@pytest.mark.parametrize("scale", [1e-4, 1e-6, 1e-8, 1e-10])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("iteration", [USUAL, LONG])
def test_rows_much_smaller_than_the_others(mods, shape, iteration, scale):
    """Half of X's rows scaled down: each comes up to the others' size with the relative precision it started with."""
    steps, a, b, c = iteration
    G = np.random.default_rng(sum(shape)).standard_normal(shape).astype(np.float32)
    if shape[0] <= shape[1]:
        G[shape[0] // 2:] *= np.float32(scale)
    else:
        G[:, shape[1] // 2:] *= np.float32(scale)
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    plain, got = (rows_off(f, want) for f in (fp32_products(G, steps, 1e-7, a, b, c), orthogonalize(mods, G, steps, 1e-7, (256, 1024), a, b, c)))
    assert got <= ROW * plain, "%.2e of a row, fp32 products %.2e" % (got, plain)


@pytest.mark.parametrize("shape", SHAPES)
def test_rows_of_every_size(mods, shape):
    """Thirty orders of magnitude from the first row to the last, a row of zeros among them."""
    r = np.random.default_rng(sum(shape))
    m = min(shape)
    s = 10.0 ** r.permutation(np.linspace(-30, 0, m))
    s[m // 3] = 0.0
    G = r.standard_normal((m, max(shape))) * s[:, None]
    G = np.float32(G if shape[0] <= shape[1] else G.T)
    want = D.orthogonalize(G)
    plain, got = fp32_products(G, 5, 1e-7), orthogonalize(mods, G, 5, 1e-7, (100, 300))
    zero, want, plain, got = [(x if shape[0] <= shape[1] else x.T) for x in (got, want, plain, got)]
    assert not zero[m // 3].any()
    keep = np.arange(m) != m // 3
    assert rows_off(got[keep], want[keep]) <= ROW * rows_off(plain[keep], want[keep])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("length", [1e-9, 1e-14, 1e-30])
def test_matrices_far_below_eps(mods, shape, length):
    G = falling(np.random.default_rng(sum(shape)), *shape)
    G = np.float32(G * (length / np.linalg.norm(G.astype(np.float64))))
    want = D.orthogonalize(G)
    plain, got = (np.linalg.norm(f - want) for f in (fp32_products(G, 5, 1e-7), orthogonalize(mods, G, 5, 1e-7, (256, 1024))))
    assert got <= WHOLE * plain, "%.2e of the result, fp32 products %.2e" % (got / np.linalg.norm(want), plain / np.linalg.norm(want))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("steps,a,b,c", [(1, 2.0, -20.0, 20.0), (60, 1.5, -0.5, 0.0), (20, 0.3, 0.0, 0.0), (6, 0.25, 0.2, 0.1), (3, -2.0, 1.0, 0.0)])
def test_other_coefficients(mods, shape, steps, a, b, c):
    """The largest polynomials that are taken, iterations that go on for long, ones that shrink what they are given, a negative sign; half of the rows small."""
    G = np.random.default_rng(sum(shape)).standard_normal(shape).astype(np.float32)
    if shape[0] <= shape[1]:
        G[::2] *= np.float32(1e-5)
    else:
        G[:, ::2] *= np.float32(1e-5)
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    plain, got = (rows_off(f, want) for f in (fp32_products(G, steps, 1e-7, a, b, c), orthogonalize(mods, G, steps, 1e-7, (256, 1024), a, b, c)))
    assert got <= ROW * max(plain, 2.0 ** -24 * steps), "%.2e of a row, fp32 products %.2e" % (got, plain)


@pytest.mark.parametrize("shape,steps,launches", [((64, 256), 5, 1), ((40, 900), 5, 2 + 5), ((512, 512), 1, 2 + 3), ((777, 1111), 5, 2 + 3 * 5),
                                                  # two steps at once: 7 products in place of 6, and X X^T once, whose parts are added up by a launch of their own
                                                  ((512, 2560), 1, 2 + 4), ((512, 2560), 2, 2 + 8), ((512, 2560), 4, 2 + 16), ((512, 2560), 5, 2 + 16 + 4), ((2560, 512), 5, 2 + 16 + 4)])
def test_launches_are_counted(mods, shape, steps, launches):
    capi, tiled = mods
    with tiled.Context(n_streams=1) as ctx:
        tG, tO = (tiled.TiledTensor(ctx, "f32", shape, (256, 1024), fill=0) for _ in range(2))
        cfg = capi.nnt_newton_schulz_cfg(A, B, CC, 1e-7, steps)
        before = ctx.stats()["launches"]
        capi.nnt_orthogonalize(ctx.h, C.byref(cfg), 1, handles(mods, [tG]), handles(mods, [tO]))
        assert ctx.stats()["launches"] - before == launches
        ctx.wait()


@pytest.mark.parametrize("shape", [(4096, 4096), (4096, 16384), (9000, 2500)])
def test_small_rows_of_large_matrices(mods, shape):
    """The largest macro-tiles, alone and with two steps at once; the references on the device."""
    capi, tiled = mods
    rows, cols = shape
    G = torch.randn(cols, rows, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")      # axes reversed: columns of the matrix first
    X = G.t() if rows <= cols else G
    X[1::2] *= 1e-6                                           # every other row of X (a view of G)

    def iterate(dtype):
        Y = X.to(dtype)
        Y = (Y.double() / (torch.linalg.vector_norm(Y.double()) + 1e-7)).to(dtype)
        for _ in range(5):
            S = torch.mm(Y, Y.t())
            Y = A * Y + torch.mm(B * S + CC * torch.mm(S, S), Y)
        return Y.double()
    want = iterate(torch.float64)
    length = torch.linalg.vector_norm(want, dim=1)
    plain = (torch.linalg.vector_norm(iterate(torch.float32) - want, dim=1) / length).max().item()
    with tiled.Context(n_streams=1) as ctx:
        t = tiled.TiledTensor(ctx, "f32", shape, (3000, 5000))
        for k, idx in enumerate(t.tile_index):
            t.tile_view(k).copy_(G[tuple(reversed(t.slices(idx)))].reshape(-1))
        torch.cuda.synchronize()
        cfg = capi.nnt_newton_schulz_cfg(A, B, CC, 1e-7, 5)
        capi.nnt_orthogonalize(ctx.h, C.byref(cfg), 1, handles(mods, [t]), handles(mods, [t]))
        ctx.wait()
        for k, idx in enumerate(t.tile_index):
            part = G[tuple(reversed(t.slices(idx)))]
            part.copy_(t.tile_view(k).view(part.shape))
    got = (torch.linalg.vector_norm((G.t() if rows <= cols else G).double() - want, dim=1) / length).max().item()
    assert got <= ROW * plain, "%.2e of a row, fp32 products %.2e" % (got, plain)


@pytest.mark.parametrize("kind", ["columns", "both", "one entry a row"])
@pytest.mark.parametrize("scale", [1e-4, 1e-8])
@pytest.mark.parametrize("shape", [(64, 64), (50, 200), (64, 1000), (300, 300), (700, 700), (512, 2560), (2560, 512)])
@pytest.mark.parametrize("iteration", [USUAL, LONG])
def test_columns_much_smaller_than_the_others(mods, shape, iteration, scale, kind):
    """Half of X's columns scaled down, or its rows too, or a matrix of one entry to a row, of any size: a column, too, keeps the precision it started with.  (fp32 products of single
    entries are exact at 1, so the last rounding of the halves counts there: 2^-24 of the result.)"""
    steps, a, b, c = iteration
    r = np.random.default_rng(sum(shape))
    m, n = min(shape), max(shape)
    if kind == "one entry a row":
        G = np.zeros((m, n))
        G[np.arange(m), r.permutation(n)[:m]] = scale ** r.uniform(0, 1, m)
    else:
        G = r.standard_normal((m, n))
        G[:, n // 2:] *= scale
        if kind == "both":
            G[m // 2:] *= scale
    G = np.float32(G if shape[0] <= shape[1] else G.T)
    want = D.orthogonalize(G, a, b, c, 1e-7, steps)
    plain, got = fp32_products(G, steps, 1e-7, a, b, c), orthogonalize(mods, G, steps, 1e-7, (256, 1024), a, b, c)
    off, own = np.linalg.norm(plain - want), np.linalg.norm(got - want)
    assert own <= ROW * max(off, 2.0 ** -24 * np.linalg.norm(want)), "%.2e of the result, fp32 products %.2e" % (own / np.linalg.norm(want), off / np.linalg.norm(want))
    if steps == 5 and kind != "one entry a row":
        plain, got = rows_off(plain, want, True), rows_off(got, want, True)
        assert got <= ROW * plain, "%.2e of a column, fp32 products %.2e" % (got, plain)


# Coefficients that shrink: 0.6^64 is 2^-47, and a row or column of 2^-112 of the others ends below fp32's last bit, 2^-149, where 0.6 times it is rounded up to itself.  A step is a
# product with `a` alone, so that a result is off by 2^-24 of itself a step for each of the roundings (of `a`, of the product, X_0 three times), and by the last bit.
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("scale,eps", [(2.0**-112, 1e-7), (1.0, 1e36)])
def test_what_shrinks_into_the_last_bit_stays_a_number(mods, shape, columns, scale, eps):
    r = np.random.default_rng(1 + sum(shape))
    G = r.standard_normal(shape).astype(np.float32)
    (G.T if columns else G)[3] *= np.float32(scale)
    X = G.astype(np.float64) / (np.linalg.norm(G.astype(np.float64)) + eps)
    got = orthogonalize(mods, G, 64, eps, (256, 1024), 0.6, 0.0, 0.0)
    assert np.all(np.isfinite(got))
    want = 0.6**64 * X
    off = np.abs(got - want) - (2 * 64 + 4) * 2.0**-24 * np.abs(want)
    assert off.max() <= 4 * 2.0**-149
