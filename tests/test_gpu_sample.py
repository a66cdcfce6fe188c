"""Drawn tokens against the oracle: filters and their combinations, equal logits, vocabularies in tiles of any size and longer than a
workgroup's registers, infinities and NaN, lists of columns, captured graphs, refusals."""
import ctypes as C

import numpy as np
import pytest

import workload
from oracle import rollout as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_13236_amd import tiled
    c = tiled.Context(n_streams=2)
    yield c
    c.close()


def quant(a, dtype):
    a = np.asarray(a, np.float32)
    return workload.round_through_bf16(a.reshape(-1)).reshape(a.shape) if dtype == "bf16" else a


def logits(seed, N_v, n, dtype, std=2.0, peaks=True):
    r = np.random.default_rng(seed)
    x = std * r.standard_normal((N_v, n))
    if peaks:
        for c in range(n):
            x[r.integers(0, N_v, min(N_v, 12)), c] += 12.0 * r.random() * r.random(min(N_v, 12))
    return quant(x, dtype), r.random(n).astype(np.float32)


def draw(ctx, X, u, dtype, tile_v=1024, shape=None, columns=None, logp=True, tiles=(4, 3), **filters):
    """Tokens and log-probabilities of the columns of X [N_v, n] (as [N_v, N_s, N_b] where `shape` = (N_s, N_b))."""
    from paper_2504_13236_amd import tiled
    N_s, N_b = shape or (1, X.shape[1])
    t = tiled.TiledTensor.from_numpy(ctx, X.reshape(X.shape[0], N_s, N_b, order="F"), (tile_v,) + tiles, dtype)
    du = torch.from_numpy(np.asarray(u, np.float32)).cuda()
    tokens = torch.full((len(u),), -77, dtype=torch.int32, device="cuda")
    lp = torch.full((len(u),), -77.0, device="cuda") if logp else None
    dc = torch.from_numpy(np.asarray(columns, np.int32)).cuda() if columns is not None else None
    torch.cuda.synchronize()
    tiled.sample_tokens(ctx, t, du, tokens, lp, dc, **filters)
    ctx.wait()
    back = t.download()
    assert np.array_equal(np.nan_to_num(back.reshape(X.shape, order="F"), nan=0.5), np.nan_to_num(X, nan=0.5))       # only read
    t.close()
    return tokens.cpu().numpy(), lp.cpu().numpy() if logp else None


def check(X, u, got, columns=None, **filters):
    tokens, logp = got
    for i in range(len(u)):
        x = X[:, i if columns is None else columns[i]].astype(np.float64)
        t, lp = R.sample_token(x, u[i], **filters)
        assert tokens[i] == t, (i, tokens[i], t)
        if logp is not None:
            # the sum of N_v exponentials in fp32 (2^-22 of each, their differences of at most 100 rounded once) meets in 64 bits; the result is rounded once
            assert abs(logp[i] - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -21, (i, logp[i], lp)


FILTERS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(temperature=1.7), dict(top_k=1), dict(top_k=5), dict(top_k=50), dict(top_p=0.9),
           dict(top_p=0.5, temperature=0.8), dict(top_p=1e-9), dict(min_p=0.05), dict(min_p=1.0), dict(top_k=20, top_p=0.8), dict(top_k=40, min_p=0.1, temperature=1.3),
           dict(top_k=30, top_p=0.95, min_p=0.02, temperature=0.6), dict(top_k=10 ** 6), dict(top_p=0.999999), dict(temperature=1e-4, top_p=0.9),
           dict(temperature=1e9, top_p=0.3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("filters", FILTERS, ids=lambda f: "_".join("%s%g" % kv for kv in f.items()) or "none")
def test_filters(ctx, dtype, filters):
    X, u = logits(3, 3001, 24, dtype)
    check(X, u, draw(ctx, X, u, dtype, **filters), **filters)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N_v,tile_v", [(1, 1), (2, 2), (3, 1), (7, 5), (63, 64), (64, 8), (257, 100), (1025, 1024), (4096, 4096), (5000, 333), (8192, 1000),
                                        (20011, 8192), (50304, 8192)])
def test_vocabularies(ctx, dtype, N_v, tile_v):
    X, u = logits(N_v, N_v, 3, dtype)
    for filters in (dict(), dict(top_k=7, temperature=0.9), dict(top_p=0.9)):
        check(X, u, draw(ctx, X, u, dtype, tile_v=tile_v, **filters), **filters)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_vocabularies(ctx, dtype):
    for N_v, tile_v in ((100003, 16384), (262144, 262144)):
        X, u = logits(N_v, N_v, 2, dtype, std=1.0, peaks=False)
        for filters in (dict(), dict(top_k=1000), dict(top_k=60000, top_p=0.7), dict(top_p=0.95), dict(min_p=0.02)):
            check(X, u, draw(ctx, X, u, dtype, tile_v=tile_v, **filters), **filters)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N_v", [100, 3000, 9000])
def test_equal_logits(ctx, dtype, N_v):
    """All logits alike, or of three values: prefixes end among equals, the lowest numbers stay."""
    n = 9
    u = ((np.arange(n) + 0.37) / n).astype(np.float32)
    flat = np.full((N_v, n), 1.25, np.float32)
    for filters in (dict(), dict(top_k=17), dict(top_p=0.5), dict(top_k=N_v - 1, top_p=0.999), dict(temperature=0.0)):
        check(flat, u, draw(ctx, flat, u, dtype, **filters), **filters)
    three = np.random.default_rng(N_v).choice(np.array([-1.0, 0.0, 2.0], np.float32), (N_v, n))
    for filters in (dict(top_k=N_v // 2), dict(top_k=5), dict(top_p=0.6), dict(top_p=0.97), dict(top_k=N_v // 2, top_p=0.9), dict(temperature=0.0)):
        check(three, u, draw(ctx, three, u, dtype, **filters), **filters)
    zeros = np.where(np.arange(N_v)[:, None] % 2, 0.0, -0.0).astype(np.float32) * np.ones((1, n), np.float32)
    check(zeros, u, draw(ctx, zeros, u, dtype, top_k=N_v // 3), top_k=N_v // 3)          # -0 and 0 are equal


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_close_logits_far_from_the_others(ctx, dtype):
    """Thousands of different values within a small part of the column's range: the part that holds the border is divided again."""
    r = np.random.default_rng(4)
    x = 40.0 + 1e-3 * r.random((9000, 4))
    x[0], x[17] = 41.0, -1e4
    x, u = quant(x, dtype), r.random(4).astype(np.float32)
    for filters in (dict(top_k=4000), dict(top_p=0.4), dict(top_k=7000, top_p=0.61)):
        check(x, u, draw(ctx, x, u, dtype, **filters), **filters)
    x[3], x[4] = 3e38, -3e38                                     # a range beyond fp32
    x = quant(x, dtype)
    for filters in (dict(top_k=4000), dict(top_p=0.4), dict()):
        check(x, u, draw(ctx, x, u, dtype, **filters), **filters)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("filters", [dict(), dict(temperature=0.0), dict(top_k=3), dict(top_p=0.7), dict(top_k=40, top_p=0.9, min_p=0.3)])
def test_infinities_and_nan(ctx, dtype, filters):
    X, u = logits(9, 2000, 8, dtype)
    X[:, 0] = -np.inf
    X[:, 1] = np.nan
    X[:1990, 2] = -np.inf
    X[5, 3], X[1500, 3], X[1999, 3] = np.inf, np.inf, np.inf
    X[::3, 4] = np.nan
    X[1:, 5] = -np.inf
    X[:, 6] = -3.4e38 if dtype == "f32" else quant(np.array([-3.3e38]), "bf16")[0]
    X[77, 6] = -1e38 if dtype == "f32" else quant(np.array([-1e38]), "bf16")[0]
    tokens, logp = draw(ctx, X, u, dtype, **filters)
    assert list(tokens[:2]) == [-1, -1] and not logp[:2].any()
    check(X, u, (tokens, logp), **filters)


def test_random_numbers_outside_their_range(ctx):
    X = np.log(np.array([[1.0], [2.0], [1.0]])).astype(np.float32) * np.ones((1, 6), np.float32)
    u = np.array([-1.0, np.nan, 1.0, 5.0, np.inf, 0.25], np.float32)
    tokens, _ = draw(ctx, X, u, "f32")
    assert list(tokens) == [0, 0, 2, 2, 2, 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_by_list(ctx, dtype):
    X, u = logits(12, 700, 15, dtype)
    columns = [14, 3, 3, 0, 7, 11, 3]
    u = np.random.default_rng(1).random(len(columns)).astype(np.float32)
    check(X, u, draw(ctx, X, u, dtype, shape=(5, 3), columns=columns, tiles=(2, 2), top_k=30), columns, top_k=30)
    tokens, logp = draw(ctx, X, np.full(4, 0.5), dtype, shape=(5, 3), columns=[-1, 15, 2 ** 31 - 1, -2 ** 31], top_p=0.5)
    assert list(tokens) == [-1] * 4 and not logp.any()
    check(X, u[:4], draw(ctx, X, u[:4], dtype, shape=(5, 3), tiles=(5, 3), logp=False))          # the first four, no log-probabilities


def test_as_token_logprob_gives_them(ctx):
    from paper_2504_13236_amd import capi, tiled
    X, u = logits(21, 5000, 6, "bf16")
    t = tiled.TiledTensor.from_numpy(ctx, X.reshape(5000, 1, 6), (2048, 1, 6), "bf16")
    lp2 = tiled.TiledTensor.zeros(ctx, (1, 6), (1, 6))
    tokens, logp = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")
    tiled.sample_tokens(ctx, t, torch.from_numpy(u).cuda(), tokens, logp, temperature=0.7, top_p=0.8)
    ctx.wait()
    capi.nnt_token_logprob(ctx.h, t.h, tokens.data_ptr(), lp2.h)
    np.testing.assert_allclose(logp.cpu().numpy(), lp2.download()[0], atol=2.0 ** -20, rtol=2.0 ** -23)
    t.close()
    lp2.close()


def test_frequencies(ctx):
    """20000 draws from one distribution: each token within five standard deviations of its share."""
    x = np.log(np.array([0.3, 0.05, 0.25, 0.2, 0.15, 0.05]))
    n = 20000
    X = np.repeat(x[:, None], n, 1).astype(np.float32)
    u = np.random.default_rng(8).random(n).astype(np.float32)
    tokens, _ = draw(ctx, X, u, "f32", tiles=(1, 999), top_k=4)
    p = np.array([0.3, 0, 0.25, 0.2, 0.15, 0]) / 0.9
    share = np.bincount(tokens, minlength=6) / n
    assert (np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / n) + 1e-12).all(), share


def test_captured_and_replayed(ctx):
    from paper_2504_13236_amd import capi, tiled
    X, u = logits(31, 6000, 8, "f32")
    t = tiled.TiledTensor.from_numpy(ctx, X.reshape(6000, 1, 8), (1500, 1, 8))
    du, tokens, logp = torch.from_numpy(u).cuda(), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    g = C.c_void_p()
    capi.nnt_capture_begin(ctx.h)
    tiled.sample_tokens(ctx, t, du, tokens, logp, top_k=100, top_p=0.9)
    capi.nnt_capture_end(ctx.h, C.byref(g))
    for k in range(4):
        X, u = logits(40 + k, 6000, 8, "f32")
        t.upload(X.reshape(6000, 1, 8))
        du.copy_(torch.from_numpy(u))
        torch.cuda.synchronize()
        capi.nnt_graph_launch(g)
        ctx.wait()
        check(X, u, (tokens.cpu().numpy(), logp.cpu().numpy()), top_k=100, top_p=0.9)
        again = draw(ctx, X, u, "f32", tile_v=6000, top_k=100, top_p=0.9)
        assert np.array_equal(again[0], tokens.cpu().numpy())
    capi.nnt_graph_destroy(g)
    t.close()


def test_refusals(ctx):
    from paper_2504_13236_amd import capi, tiled
    T = tiled.TiledTensor
    X, flat = T.zeros(ctx, (100, 2, 3), (64, 2, 3)), T.zeros(ctx, (100, 6), (64, 6))
    holes = T.zeros(ctx, (100, 2, 3), (64, 2, 3), absent=lambda i: i[0] == 1)
    u, tokens = torch.zeros(8, device="cuda"), torch.full((8,), -5, dtype=torch.int32, device="cuda")

    def call(X=X, n=6, u=u.data_ptr(), tokens=tokens.data_ptr(), columns=None, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0):
        cfg = capi.nnt_sample_cfg(temperature, top_p, min_p, top_k)
        return capi.nnt_sample_tokens.raw(ctx.h, C.byref(cfg), X.h if X else None, columns, n, u, tokens, None)
    nan, inf = float("nan"), float("inf")
    bad = [dict(temperature=-1.0), dict(temperature=nan), dict(temperature=inf), dict(top_p=0.0), dict(top_p=1.1), dict(top_p=nan), dict(min_p=-0.1),
           dict(min_p=1.5), dict(min_p=nan), dict(top_k=-1), dict(n=0), dict(n=-3), dict(n=7), dict(n=1 << 22, columns=tokens.data_ptr()), dict(X=None), dict(u=None),
           dict(tokens=None), dict(X=flat), dict(X=holes)]
    for kw in bad:
        assert call(**kw) == capi.NNT_EINVAL, kw
    assert capi.nnt_sample_tokens.raw(ctx.h, None, X.h, None, 6, u.data_ptr(), tokens.data_ptr(), None) == capi.NNT_EINVAL
    ctx.wait()
    assert (tokens == -5).all()
    assert call() == capi.NNT_OK
    ctx.wait()
    assert (tokens[:6] == 0).all() and (tokens[6:] == -5).all()
    for t in (X, flat, holes):
        t.close()


def odd_columns(r, N_v):
    """bf16 columns of what has no code of its own, one kind each: zeros of both signs, tiny ones, masked ones, large ones."""
    def base(std=2.0):
        return std * r.standard_normal(N_v)
    cols = {}
    x = base()
    x[::2] = 0.0
    x[1::4] = -0.0
    cols["zeros"] = x
    x = -np.abs(base()) - 0.1
    x[::3] = 0.0
    cols["zeros on top"] = x
    cols["all zero"] = np.where(np.arange(N_v) % 3 == 1, -0.0, 0.0)
    x = base()
    x[r.integers(0, N_v, 300)] = 1e-5 * r.standard_normal(300)
    cols["some tiny"] = x
    cols["all tiny"] = 1e-4 * base()
    x = -np.abs(base(0.5)) - 0.01
    x[100:160] = 1e-6 * r.standard_normal(60)
    cols["tiny on top"] = x
    x = base()
    x[500:] = -1e4
    cols["masked by -1e4"] = x
    x = base()
    x[: N_v - 40] = -np.inf
    cols["masked by -inf"] = x
    cols["all negative"] = -np.abs(base()) - 3.0
    cols["all below the codes"] = -300.0 - np.abs(base(20.0))
    x = base(60.0)
    x[7] = 300.0
    cols["above the codes"] = x
    x = base()
    x[11], x[12] = 1e30, np.nan
    cols["far above"] = x
    cols["wide"] = base(50.0)
    cols["narrow"] = 5.0 + 0.01 * base()
    return cols


@pytest.mark.parametrize("filters", [dict(), dict(temperature=0.0), dict(top_k=30), dict(top_k=6000), dict(top_p=0.9), dict(top_p=0.3, temperature=3.0), dict(min_p=0.5),
                                     dict(top_k=5000, top_p=0.97, min_p=1e-4), dict(temperature=200.0), dict(temperature=200.0, top_p=0.8), dict(temperature=0.01, top_k=100)],
                         ids=lambda f: "_".join("%s%g" % kv for kv in f.items()) or "none")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_has_no_code(ctx, dtype, filters):
    r = np.random.default_rng(77)
    cols = odd_columns(r, 12345)
    X = quant(np.stack(list(cols.values()), 1), dtype)
    u = r.random(X.shape[1]).astype(np.float32)
    check(X, u, draw(ctx, X, u, dtype, tile_v=5000, **filters), **filters)


@pytest.mark.parametrize("filters", [dict(), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.5)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_in_long_columns(ctx, dtype, filters):
    X, u = logits(10, 12345, 6, dtype)
    X[[5, 4999, 5000, 12344], 0] = np.inf
    X[12344, 1] = np.inf
    X[::2, 2], X[7001, 2] = np.nan, np.inf
    X[:, 3] = -np.inf
    X[9999, 3] = -2.0
    X[:, 4] = np.nan
    check(X, u, draw(ctx, X, u, dtype, tile_v=5000, **filters), **filters)
    check(X[:, :5], u[:5], draw(ctx, X[:, :5], u[:5], dtype, tile_v=5000, logp=False, **filters), **filters)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_borders_of_the_lists(ctx, dtype):
    """top-k at the ends of what is listed, and thousands of equal logits on top of it."""
    r = np.random.default_rng(5)
    X = quant(2.0 * r.standard_normal((20000, 6)), dtype)
    X[:, 1] = np.where(r.random(20000) < 0.3, 4.0, X[:, 1])
    X[:, 2] = np.where(r.random(20000) < 0.101, 50.0, X[:, 2])
    X[:, 3] = np.round(X[:, 3])
    u = r.random(6).astype(np.float32)
    for k in (1, 2, 511, 512, 513, 1024, 2048, 2049, 19999, 20000, 20001):
        for more in (dict(), dict(top_p=0.6)):
            f = dict(top_k=k, **more)
            check(X, u, draw(ctx, X, u, dtype, tile_v=20000, **f), **f)


def test_many_columns_of_many_kinds(ctx):
    """More columns than the chip takes at once, of both types, against each other's neighbours: nothing of a column reaches another."""
    r = np.random.default_rng(6)
    for dtype in ("bf16", "f32"):
        X = quant((1.0 + 3.0 * r.random(1200)) * r.standard_normal((9000, 1200)), dtype)
        X[:, ::7] = np.round(X[:, ::7])
        u = r.random(1200).astype(np.float32)
        f = dict(top_p=0.85, temperature=0.9)
        tokens, logp = draw(ctx, X, u, dtype, tile_v=4096, tiles=(1, 500), **f)
        pick = r.integers(0, 1200, 60)
        check(X[:, pick], u[pick], (tokens[pick], logp[pick]), **f)
        assert (tokens >= 0).all() and (tokens < 9000).all()
