"""GPU parity of the log-probabilities of given tokens, the policy loss and the preference loss (with their gradients) against the
fp64 oracle, over types, lengths, tilings, masks and the forms that the header allows, and what they refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_util import quant
from oracle import definition as D

pytestmark = pytest.mark.gpu

# Bounds.  An exponential: rounding of the difference and of its product with 1/ln 2, 2^-24 |t| each for |t| up to 30, and 2^-23 of the
# instruction: 4e-6 of its value.  The sum: the same, and 2^-24 for each of some 60 additions in a row.  logp = difference - log(sum)
# in 64 bits: 8e-6, then half a step of its value.  The gradient g (onehot - p): p to 1.2e-5 of its value, g to another 1.2e-5.
REL = 2.5e-5
LOGP = 8e-6
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


def dev_i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32).reshape(-1, order="F"))).cuda()


class Call:
    """The arguments of one call on the device, and what it leaves."""

    def __init__(self, mods, ctx, X, lab, base, dtype, in_place=False, gradient=True, **positions):
        capi, tiled = self.mods = mods
        self.ctx, self.dtype, self.shape = ctx, dtype, X.shape
        self.X = tiled.TiledTensor.from_numpy(ctx, np.asarray(X, np.float32), base, dtype)
        self.before = self.X.buf.clone()
        self.dX = self.X if in_place else tiled.TiledTensor(ctx, dtype, X.shape, base) if gradient else None
        if self.dX is not None and not in_place:
            self.dX.buf.fill_(0x5a)
        self.logp = tiled.TiledTensor(ctx, "f32", X.shape[1:], base[1:])
        self.logp.buf.fill_(0x5a)
        self.lab = dev_i32(lab)
        self.pos = {}
        for k, a in positions.items():
            if a is not None:
                a = np.asarray(a, np.float32)
                self.pos[k] = tiled.TiledTensor.from_numpy(ctx, a, base[1:] if a.ndim == 2 else base[2:], "f32")
        n = X.shape[1] * X.shape[2]
        self.losses = torch.full((n + 8,), 7.0, device="cuda")       # 8 more than the call may write
        self.rewards = torch.full((X.shape[2] + 8,), 7.0, device="cuda")
        self.loss = torch.full((2,), 7.0, device="cuda")
        torch.cuda.synchronize()

    def p(self, k):
        return self.pos[k].h if k in self.pos else None

    def logprob(self):
        self.mods[0].nnt_token_logprob(self.ctx.h, self.X.h, self.lab.data_ptr(), self.logp.h)

    def policy(self, lo=0.2, hi=0.2, kl=0.0, reduction=0):
        cfg = self.mods[0].nnt_policy_cfg(lo, hi, kl, reduction)
        self.mods[0].nnt_policy_loss(self.ctx.h, C.byref(cfg), self.X.h, self.lab.data_ptr(), self.p("old"), self.p("ref"), self.p("adv"),
                                     self.dX.h if self.dX is not None else None, self.logp.h, self.losses.data_ptr(), self.loss.data_ptr())

    def preference(self, beta=0.1, soft=0.0, reduction=0):
        cfg = self.mods[0].nnt_preference_cfg(beta, soft, reduction)
        self.mods[0].nnt_preference_loss(self.ctx.h, C.byref(cfg), self.X.h, self.lab.data_ptr(), self.p("ref"),
                                         self.dX.h if self.dX is not None else None, self.logp.h, self.rewards.data_ptr(),
                                         self.losses.data_ptr(), self.loss.data_ptr())

    def close_to(self, got, want, rel, add, what):
        got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
        bad = ~(np.abs(got - want) <= rel * np.abs(want) + add)
        assert not bad.any(), "%s: %d off, first at %s: %r for %r" % (what, bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0])

    def check_logp(self, want):
        self.close_to(self.logp.download(), want, HALF["f32"], LOGP, "logp")
        if self.dX is not self.X:
            assert torch.equal(self.X.buf, self.before), "the logits were touched"

    def check_gradient(self, want, has):
        got = self.dX.download()
        g = np.abs(want).max(axis=0)                          # of the order of |dloss/dlogp| (1 - p): the label's entry
        scale = np.abs(want).sum(axis=0)                      # g (1 - p) at the label, the same again over the others
        assert np.all(g <= scale)
        self.close_to(got, want, HALF[self.dtype] + REL, REL * scale[None], "gradient")
        assert not got[:, ~has].any(), "gradient of a position without a label"

    def check_sum(self, n, want):
        losses = self.losses[:n].double()
        assert (self.losses[n:] == 7.0).all() and self.loss[1] == 7.0
        assert abs(self.loss[0].item() - losses.sum().item()) <= 2.0 ** -23 * losses.abs().sum().item()
        return losses.cpu().numpy()


def labels_for(r, N_v, N_s, N_b, masked=0.3):
    lab = r.integers(0, N_v, (N_s, N_b))
    if masked and N_s * N_b > 1:
        out = r.random((N_s, N_b)) < masked
        lab[out] = r.choice([-1, -100, N_v, 2 ** 31 - 1, -2 ** 31], out.sum())
    return lab


def has_label(lab, N_v):
    return (lab >= 0) & (lab < N_v)


def logits_for(r, lab, N_v, dtype):
    X = 2.0 * r.standard_normal((N_v,) + lab.shape)
    has = has_label(lab, N_v)
    s, b = np.nonzero(has)
    X[lab[s, b], s, b] += r.uniform(0, 12, len(s))
    return quant(X, dtype)


# shapes (N_v, N_s, N_b) and tiles: one token; vocabularies smaller than a vector; every instance of registers; columns too long for
# them; tiles that end inside a vector; more tiles than fit the table in LDS
SHAPES = [((1, 1, 1), (1, 1, 1)), ((3, 2, 2), (2, 1, 2)), ((257, 5, 3), (100, 2, 2)), ((1000, 4, 2), (1000, 4, 2)), ((777, 3, 4), (10, 2, 1)),
          ((4099, 3, 2), (4099, 3, 1)), ((16390, 2, 2), (5001, 2, 2)), ((33001, 3, 1), (8192, 2, 1)), ((50304, 1, 1), (8192, 1, 1)),
          ((50305, 2, 2), (50305, 2, 2)), ((57350, 2, 1), (8192, 2, 1)), ((66001, 1, 2), (66001, 1, 2)), ((70001, 2, 2), (16384, 1, 2)), ((140003, 1, 2), (32768, 1, 1))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,base", SHAPES)
def test_token_logprob(mods, shape, base, dtype):
    r = np.random.default_rng(sum(shape) + 31 * sum(base))
    lab = labels_for(r, *shape)
    X = logits_for(r, lab, shape[0], dtype)
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, base, dtype)
        c.logprob()
        c.check_logp(D.token_logprob(X, lab))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,base", SHAPES)
def test_policy_loss_shapes(mods, shape, base, dtype):
    r = np.random.default_rng(sum(shape) + 31 * sum(base))
    lab = labels_for(r, *shape)
    X = logits_for(r, lab, shape[0], dtype)
    has = has_label(lab, shape[0])
    lp = D.token_logprob(X, lab)
    old, ref = (lp + 0.3 * r.standard_normal(lab.shape)).astype(np.float32), (lp + 0.3 * r.standard_normal(lab.shape)).astype(np.float32)
    adv = r.standard_normal(lab.shape).astype(np.float32)
    for a in (old, ref, adv):
        a[~has] = np.nan                                      # whatever stands behind a prompt or in front of an answer
    X[:, ~has] = np.nan
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, base, dtype, old=old, ref=ref, adv=adv)
        c.policy(0.2, 0.3, 0.1, 1)
        X[:, ~has] = 0.0
        L, losses, logp, dX = D.policy_loss(X, lab, old, ref, adv, 0.2, 0.3, 0.1, "tokens")
        c.close_to(c.logp.download(), logp, HALF["f32"], LOGP, "logp")
        c.check_gradient(dX, has)
        got = c.check_sum(lab.size, losses)
        # r to 1.2e-5, e^k - k - 1 moves by less than 1.2e-5 (e^|k| + 1)
        w = D.position_weights(has, "tokens").reshape(-1, order="F")
        c.close_to(got, losses.reshape(-1, order="F"), 1e-6, w * 2e-4, "losses")
        assert not got[~has.reshape(-1, order="F")].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reduction", [0, 1, 2])
@pytest.mark.parametrize("form", ["in place", "loss only", "no old", "no ref", "per sequence"])
def test_policy_loss_forms(mods, form, reduction, dtype):
    r = np.random.default_rng(5)
    N_v, N_s, N_b, base = 1201, 23, 5, (500, 8, 2)
    lab = labels_for(r, N_v, N_s, N_b)
    lab[:, 1] = -1                                            # a sequence without any
    X = logits_for(r, lab, N_v, dtype)
    has = has_label(lab, N_v)
    lp = D.token_logprob(X, lab)
    old = None if form == "no old" else np.float32(lp + 0.3 * r.standard_normal(lab.shape))
    ref = None if form == "no ref" else np.float32(lp + 0.3 * r.standard_normal(lab.shape))
    adv = np.float32(r.standard_normal(N_b if form == "per sequence" else lab.shape))
    kl = 0.0 if form == "no ref" else 0.2
    with mods[1].Context(n_streams=3) as ctx:
        c = Call(mods, ctx, X, lab, base, dtype, in_place=form == "in place", gradient=form != "loss only", old=old, ref=ref, adv=adv)
        c.policy(0.1, 0.25, kl, reduction)
        L, losses, logp, dX = D.policy_loss(X, lab, old, ref, adv, 0.1, 0.25, kl, ("sum", "tokens", "sequences")[reduction])
        c.check_logp(logp)
        if form != "loss only":
            c.check_gradient(dX, has)
        got = c.check_sum(lab.size, losses)
        w = D.position_weights(has, ("sum", "tokens", "sequences")[reduction]).reshape(-1, order="F")
        c.close_to(got, losses.reshape(-1, order="F"), 1e-6, w * 2e-4, "losses")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,base", [((3, 1, 2), (2, 1, 1)), ((257, 5, 4), (100, 2, 3)), ((777, 3, 2), (10, 2, 2)), ((4099, 33, 6), (1500, 16, 6)), ((50305, 2, 2), (8192, 2, 2)),
                                        ((140003, 1, 2), (32768, 1, 1)), ((999, 700, 2), (999, 300, 2))])
@pytest.mark.parametrize("reduction", [0, 2])
def test_preference_loss(mods, shape, base, dtype, reduction):
    r = np.random.default_rng(sum(shape) + 31 * sum(base))
    lab = labels_for(r, *shape)
    if shape[2] > 2:
        lab[:, 1] = -1                                        # an answer without any token
    X = logits_for(r, lab, shape[0], dtype)
    has = has_label(lab, shape[0])
    ref = np.float32(D.token_logprob(X, lab) + 0.3 * r.standard_normal(lab.shape))
    ref[~has] = np.nan
    X[:, ~has] = np.nan
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, base, dtype, ref=ref)
        c.preference(0.3, 0.05, reduction)
        X[:, ~has] = 0.0
        L, losses, rewards, logp, dX = D.preference_loss(X, lab, ref, 0.3, 0.05, reduction == 2)
        c.close_to(c.logp.download(), logp, HALF["f32"], LOGP, "logp")
        n = has.sum(axis=0)
        got = c.rewards.cpu().numpy()
        assert (got[shape[2]:] == 7.0).all()
        c.close_to(got[:shape[2]], rewards, HALF["f32"], 0.3 * LOGP * n, "rewards")
        # the slope moves by a quarter of the margin's error at most
        dz = 0.3 * LOGP * (n[:shape[2] // 2] + n[shape[2] // 2:])
        c.close_to(c.check_sum(shape[2] // 2, losses), losses, 2.0 ** -23, dz, "losses")
        slope = np.abs(dX).sum(axis=0)
        assert np.all(np.isfinite(slope))
        scale = 0.3 * np.concatenate([dz, dz])[None, None, :] * np.ones(dX.shape)
        got = c.dX.download()
        c.close_to(got, dX, HALF[dtype] + REL, REL * slope[None] + scale, "gradient")
        assert not got[:, ~has].any()


@pytest.mark.parametrize("form", ["in place", "loss only", "no ref"])
def test_preference_loss_forms(mods, form):
    r = np.random.default_rng(6)
    N_v, N_s, N_b, base = 1201, 23, 4, (500, 8, 2)
    lab = labels_for(r, N_v, N_s, N_b)
    X = logits_for(r, lab, N_v, "f32")
    ref = None if form == "no ref" else np.float32(D.token_logprob(X, lab) + 0.3 * r.standard_normal(lab.shape))
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, base, "f32", in_place=form == "in place", gradient=form != "loss only", ref=ref)
        c.preference(0.1, 0.0)
        L, losses, rewards, logp, dX = D.preference_loss(X, lab, ref, 0.1, 0.0)
        c.check_logp(logp)
        assert abs(c.loss[0].item() - L) <= 1e-4 * abs(L)
        if form != "loss only":
            got = c.dX.download()
            c.close_to(got, dX, 2e-4, 2e-4 * np.abs(dX).sum(axis=0)[None], "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N_v,base_v", [(1000, 300), (50304, 8192), (140003, 32768)])
def test_banned_tokens(mods, N_v, base_v, dtype):
    """Logits of -inf and of the type's lowest value: probability and gradient 0; whole stretches of them, so that some threads see nothing else."""
    r = np.random.default_rng(7)
    lab = r.integers(0, N_v // 8, (3, 2))
    X = quant(r.standard_normal((N_v, 3, 2)), dtype)
    lowest = -3.3895313892515355e38 if dtype == "bf16" else np.finfo(np.float32).min
    X[N_v // 8:, 0, :] = -np.inf
    X[N_v // 8:, 1, :] = lowest
    X[:N_v // 8, 2, 1] = -np.inf
    lab[2, 1] = N_v - 1
    old = np.float32(D.token_logprob(X, lab) + 0.1)
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, (base_v, 2, 2), dtype, old=old, adv=np.ones(2))
        c.policy()
        L, losses, logp, dX = D.policy_loss(X, lab, old, None, np.ones(2))
        c.check_logp(logp)
        c.check_gradient(dX, has_label(lab, N_v))
        assert not c.dX.download()[N_v // 8:, :2].any()
        c.logprob()
        c.check_logp(logp)
        # a label that is banned itself: logp is -inf
        lab[0, 0] = N_v - 1
        c.lab = dev_i32(lab)
        c.logprob()
        assert c.logp.download()[0, 0] == -np.inf


def test_nan_in_a_column_stays_in_it(mods):
    r = np.random.default_rng(8)
    lab = r.integers(0, 900, (4, 2))
    X = r.standard_normal((900, 4, 2)).astype(np.float32)
    X[17, 1, 0] = np.nan
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, (256, 4, 2), "f32", adv=np.ones(2))
        c.policy()
        dX, logp = c.dX.download(), c.logp.download()
        assert np.isnan(logp[1, 0]) and np.isnan(dX[:, 1, 0]).all() and np.isnan(c.loss[0].item())
        ok = np.ones((4, 2), bool)
        ok[1, 0] = False
        assert np.isfinite(logp[ok]).all() and np.isfinite(dX[:, ok]).all()


def device_want(x, lab, g):
    """logp and gradient of columns x [n, N_v] in 64 bits on the device; g: dloss/dlogp of each."""
    x, lab = x.double(), torch.as_tensor(lab, device="cuda").long()[:, None]
    logp = torch.log_softmax(x, 1)
    d = -logp.exp() * g[:, None]
    d.scatter_add_(1, lab, g[:, None].clone())
    return logp.gather(1, lab)[:, 0], d


def test_offsets_beyond_32_bits(mods):
    """One tile of 3.3e9 logits: the first and the last sequence have labels, everything between is padding."""
    capi, tiled = mods
    N_v, N_s, N_b = 50304, 1024, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    with tiled.Context(n_streams=1) as ctx:
        X = tiled.TiledTensor(ctx, "bf16", (N_v, N_s, N_b), (N_v, N_s, N_b))
        dX = tiled.TiledTensor(ctx, "bf16", (N_v, N_s, N_b), (N_v, N_s, N_b))
        x, d = X.buf.view(torch.bfloat16).view(N_b, N_s, N_v), dX.buf.view(torch.bfloat16).view(N_b, N_s, N_v)
        x.fill_(float("nan"))
        d.fill_(float("nan"))
        lab = torch.full((N_b, N_s), -1, dtype=torch.int32, device="cuda")
        for b in (0, N_b - 1):
            x[b] = torch.randn(N_s, N_v, generator=g, device="cuda")
            lab[b] = torch.randint(0, N_v, (N_s,), generator=g, device="cuda", dtype=torch.int32)
        logp, adv = (tiled.TiledTensor(ctx, "f32", (N_s, N_b), (N_s, N_b), fill=0) for _ in range(2))
        adv.buf.view(torch.float32).fill_(1.0)
        losses, loss = torch.zeros(N_s * N_b, device="cuda"), torch.zeros(1, device="cuda")
        torch.cuda.synchronize()
        capi.nnt_policy_loss(ctx.h, C.byref(capi.nnt_policy_cfg(0.2, 0.2, 0.0, 0)), X.h, lab.data_ptr(), None, None, adv.h, dX.h, logp.h,
                             losses.data_ptr(), loss.data_ptr())
        ctx.wait()
        got = logp.buf.view(torch.float32).view(N_b, N_s).double()
        for b in (0, N_b - 1):
            want, dwant = device_want(x[b], lab[b], torch.full((N_s,), -1.0, device="cuda", dtype=torch.float64))
            assert ((got[b] - want).abs() <= HALF["f32"] * want.abs() + LOGP).all()
            assert ((d[b].double() - dwant).abs() <= (HALF["bf16"] + REL) * dwant.abs() + REL * 2).all()
        assert not d[1:N_b - 1].any() and not got[1:N_b - 1].any()


def test_longest_columns(mods):
    """Nearly as many vectors as a column may have, in 4194 tiles, and one more than it may have."""
    capi, tiled = mods
    N_v, n = 4193999, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(n, N_v, generator=g, device="cuda")
    lab = np.array([0, N_v - 1, 2097152, 4193000], np.int32)
    with tiled.Context(n_streams=1) as ctx:
        def T(shape, base):
            return tiled.TiledTensor(ctx, "f32", shape, base, fill=0)
        X, dX = T((N_v, 1, n), (1000, 1, n)), T((N_v, 1, n), (1000, 1, n))
        at = [X.slices(idx)[0] for idx in X.tile_index]
        for k, sl in enumerate(at):
            X.tile_view(k).copy_(x[:, sl].reshape(-1))
        logp, dlab = T((1, n), (1, n)), dev_i32(lab)
        rewards, losses, loss = (torch.zeros(n, device="cuda") for _ in range(3))
        want, _ = device_want(x, lab, torch.zeros(n, device="cuda", dtype=torch.float64))
        torch.cuda.synchronize()

        def check(slope):
            ctx.wait()
            assert ((logp.buf.view(torch.float32)[:n].double() - want).abs() <= HALF["f32"] * want.abs() + LOGP).all()
            _, dwant = device_want(x, lab, slope)
            for k, sl in enumerate(at):
                got, w = dX.tile_view(k).view(n, -1).double(), dwant[:, sl]
                assert ((got - w).abs() <= (HALF["f32"] + REL) * w.abs() + REL * 2 * slope.abs()[:, None] * (w.abs() > 0.1 * slope.abs()[:, None])).all()
        adv = T((n,), (n,))
        adv.buf.view(torch.float32)[:n].fill_(1.0)
        torch.cuda.synchronize()
        capi.nnt_policy_loss(ctx.h, C.byref(capi.nnt_policy_cfg(0.2, 0.2, 0.0, 0)), X.h, dlab.data_ptr(), None, None, adv.h, dX.h, logp.h,
                             losses.data_ptr(), loss.data_ptr())
        check(torch.full((n,), -1.0, device="cuda", dtype=torch.float64))
        capi.nnt_preference_loss(ctx.h, C.byref(capi.nnt_preference_cfg(1.0, 0.0, 0)), X.h, dlab.data_ptr(), None, dX.h, logp.h, rewards.data_ptr(),
                                 losses.data_ptr(), loss.data_ptr())
        slope = torch.sigmoid(want[:2] - want[2:]) - 1.0
        check(torch.cat([slope, -slope]))
        long = T((4195001, 1, 1), (1000, 1, 1))                    # 250 vectors to a tile: 2^20 are 4194.3 tiles
        assert capi.nnt_token_logprob.raw(ctx.h, long.h, dlab.data_ptr(), T((1, 1), (1, 1)).h) == capi.NNT_EINVAL


@pytest.mark.parametrize("reduction", [1, 2])
@pytest.mark.parametrize("N_s,N_b", [(40, 1030), (33, 1023), (32, 70), (1, 2050), (3000, 2), (5, 1)])
def test_weights_of_many_and_of_few_sequences(mods, N_s, N_b, reduction):
    """Logits that are all alike: every position's loss is its weight times -A."""
    capi, tiled = mods
    r = np.random.default_rng(N_s + N_b)
    lab = labels_for(r, 3, N_s, N_b, 0.4)
    if N_b > 1:
        lab[:, N_b // 2] = -1                                     # a sequence without any label
    w = D.position_weights(has_label(lab, 3), ("sum", "tokens", "sequences")[reduction])
    with tiled.Context(n_streams=1) as ctx:
        c = Call(mods, ctx, np.zeros((3, N_s, N_b), np.float32), lab, (3, N_s, N_b), "f32", gradient=False, adv=np.ones(N_b))
        c.policy(reduction=reduction)
        ctx.wait()
        got = c.losses[:N_s * N_b].cpu().numpy().reshape(N_s, N_b, order="F")
        # 1 / n, 1 / count and their product: a rounding each, and half of one for the count's own quotient
        c.close_to(got, -w, 4 * 2.0 ** -24, 0.0, "weights")


def test_ratio_beyond_32_bits(mods):
    """exp(90) is more than fp32 holds: without an advantage the position still has no loss and no gradient."""
    capi, tiled = mods
    X = np.zeros((40, 4, 1), np.float32)
    X[3] = 5.0
    lab = np.full((4, 1), 3)
    logp = D.token_logprob(X, lab)
    old = np.float32(logp - np.array([[90.0], [0.1], [500.0], [0.0]]))
    adv = np.float32([[0.0], [1.5], [0.0], [0.0]])
    with tiled.Context(n_streams=1) as ctx:
        c = Call(mods, ctx, X, lab, (16, 4, 1), "f32", old=old, adv=adv)
        c.policy()
        ctx.wait()
        loss, losses, _, want = D.policy_loss(X, lab, old, None, adv)
        c.close_to(c.check_sum(4, loss), losses.reshape(-1, order="F"), 3e-5, 0.0, "losses")
        c.check_gradient(want, np.ones((4, 1), bool))
        assert not c.dX.download()[:, [0, 2, 3]].any()


def test_answer_that_cannot_be_given(mods):
    """A rejected answer with a token of probability 0: the margin is infinite, the loss and the gradients are 0; the other way round the loss is infinite."""
    capi, tiled = mods
    X = np.random.default_rng(4).standard_normal((40, 2, 4)).astype(np.float32)
    lab = np.random.default_rng(5).integers(0, 40, (2, 4))
    X[lab[1, 2], 1, 2] = -np.inf
    X[lab[0, 1], 0, 1] = -np.inf
    with tiled.Context(n_streams=1) as ctx:
        c = Call(mods, ctx, X, lab, (16, 2, 4), "f32")
        c.preference()
        ctx.wait()
        got = c.losses[:2].cpu().numpy()
        assert got[0] == 0.0 and got[1] == np.inf and c.loss[0].item() == np.inf
        assert not c.dX.download()[:, :, [0, 2]].any()
        assert c.rewards[2].item() == -np.inf


def test_losses_from_four_streams_and_repeated(mods):
    """Independent calls on one context at once, each with its own tensors, twice over: the same results bit for bit; and a
    loss that reads the log-probabilities which an earlier call wrote."""
    r = np.random.default_rng(9)
    N_v, N_s, N_b, base = 5000, 40, 4, (2000, 16, 4)
    with mods[1].Context(n_streams=4) as ctx:
        calls = []
        for i in range(6):
            lab = labels_for(r, N_v, N_s, N_b)
            X = logits_for(r, lab, N_v, "bf16")
            calls.append((Call(mods, ctx, X, lab, base, "bf16", adv=r.standard_normal(N_b)), Call(mods, ctx, X, lab, base, "bf16"), X, lab))
        for c, other, *_ in calls:
            other.logp.buf.zero_()
            c.pos["old"] = c.pos["ref"] = other.logp
        torch.cuda.synchronize()
        first = None
        for _ in range(3):
            for c, other, X, lab in calls:
                other.logprob()
                c.preference(0.2, 0.1, 2)
                c.pos["old"] = c.pos["ref"] = other.logp
                c.policy(0.2, 0.2, 0.1, 2)
            ctx.wait()
            now = [torch.cat([c.dX.buf, c.logp.buf, c.losses.view(torch.uint8), c.rewards.view(torch.uint8)]) for c, *_ in calls]
            torch.cuda.synchronize()                          # the copies are made on torch's stream, the next calls run on the context's
            assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
            first = now
        for c, other, X, lab in calls:
            adv = c.pos["adv"].download()
            _, losses, logp, dX = D.policy_loss(X, lab, D.token_logprob(X, lab), D.token_logprob(X, lab), adv, 0.2, 0.2, 0.1, "sequences")
            c.check_logp(logp)
            c.check_gradient(dX, has_label(lab, N_v))


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_losses_captured_and_replayed(mods, kind):
    capi, tiled = mods
    r = np.random.default_rng(10)
    N_v, N_s, N_b, base = 3001, 19, 4, (1024, 8, 4)
    with tiled.Context(n_streams=2) as ctx:
        lab = labels_for(r, N_v, N_s, N_b)
        X = logits_for(r, lab, N_v, "f32")
        ref = np.float32(D.token_logprob(X, lab))
        c = Call(mods, ctx, X, lab, base, "f32", ref=ref, old=ref, adv=r.standard_normal(N_b))
        go = (lambda: c.policy(0.2, 0.2, 0.1, 1)) if kind == "policy" else (lambda: c.preference(0.2, 0.1))
        g = C.c_void_p()
        capi.nnt_capture_begin(ctx.h)
        with pytest.raises(capi.NntError):                    # the scratch is not there yet
            go()
        capi.nnt_capture_end(ctx.h, C.byref(g))
        capi.nnt_graph_destroy(g)
        go()
        ctx.wait()
        capi.nnt_capture_begin(ctx.h)
        go()
        capi.nnt_capture_end(ctx.h, C.byref(g))
        for i in range(4):
            Xi = logits_for(np.random.default_rng(20 + i), lab, N_v, "f32")
            c.X.upload(Xi)
            c.loss.zero_()
            torch.cuda.synchronize()
            capi.nnt_graph_launch(g)
            ctx.wait()
            got = [t.clone() for t in (c.dX.buf, c.logp.buf, c.losses, c.loss, c.rewards)]
            torch.cuda.synchronize()
            # eager work of the same kind between the replays, with more scratch than the graph was recorded with
            if i == 1:
                big = Call(mods, ctx, np.zeros((64, 40000, 2)), np.zeros((40000, 2), int), (64, 40000, 2), "f32")
                big.preference()
            go()
            ctx.wait()
            assert all(torch.equal(a, b) for a, b in zip(got, (c.dX.buf, c.logp.buf, c.losses, c.loss, c.rewards)))
        capi.nnt_graph_destroy(g)


def test_refusals(mods):
    capi, tiled = mods
    r = np.random.default_rng(11)
    N_v, N_s, N_b, base = 50, 6, 4, (20, 4, 2)
    with tiled.Context(n_streams=2) as ctx, tiled.Context(n_streams=1) as other:
        def T(shape, b, dtype="f32", c=ctx):
            return tiled.TiledTensor(c, dtype, shape, b, fill=0)
        X, dX, logp, pos = T((N_v, N_s, N_b), base), T((N_v, N_s, N_b), base), T((N_s, N_b), base[1:]), T((N_s, N_b), base[1:])
        lab = dev_i32(np.zeros((N_s, N_b)))
        f = torch.zeros(64, device="cuda")
        P, L = f.data_ptr(), lab.data_ptr()
        good_p, good_q = capi.nnt_policy_cfg(0.2, 0.2, 0.1, 1), capi.nnt_preference_cfg(0.1, 0.0, 0)

        def bad(fn, *args, code=capi.NNT_EINVAL):
            assert fn.raw(ctx.h, *args) == code, args
        odd = [T((N_s, N_b), (6, 2)), T((N_s, N_b), base[1:], "bf16"), T((N_s + 1, N_b), base[1:]), T((N_s, N_b), base[1:], c=other)]
        bad(capi.nnt_token_logprob, None, L, logp.h)
        bad(capi.nnt_token_logprob, X.h, None, logp.h)
        bad(capi.nnt_token_logprob, X.h, L, None)
        bad(capi.nnt_token_logprob, pos.h, L, logp.h)
        for t in odd:
            bad(capi.nnt_token_logprob, X.h, L, t.h)
            bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, t.h, pos.h, pos.h, dX.h, logp.h, P, P)
            bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, t.h, pos.h, dX.h, logp.h, P, P)
            bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, t.h, dX.h, logp.h, P, P)
            bad(capi.nnt_preference_loss, C.byref(good_q), X.h, L, t.h, dX.h, logp.h, P, P, P)
        gone = tiled.TiledTensor(ctx, "f32", (N_v, N_s, N_b), base, absent=lambda idx: idx[0] == 1)
        assert capi.nnt_token_logprob.raw(ctx.h, gone.h, L, logp.h) == capi.NNT_EINVAL
        for d in (gone, T((N_v, N_s, N_b), (50, 4, 2)), T((N_v, N_s, N_b), base, "bf16"), T((N_v, N_s, N_b), base, c=other)):
            bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, pos.h, d.h, logp.h, P, P)
            bad(capi.nnt_preference_loss, C.byref(good_q), X.h, L, pos.h, d.h, logp.h, P, P, P)
        for cfg in ((-0.1, 0.2, 0.1, 0), (1.5, 0.2, 0.1, 0), (0.2, -1.0, 0.1, 0), (0.2, 0.2, -0.1, 0), (0.2, 0.2, 0.1, 3), (0.2, 0.2, 0.1, -1),
                    (float("nan"), 0.2, 0.1, 0), (0.2, float("inf"), 0.1, 0), (0.2, 0.2, float("nan"), 0)):
            bad(capi.nnt_policy_loss, C.byref(capi.nnt_policy_cfg(*cfg)), X.h, L, pos.h, pos.h, pos.h, dX.h, logp.h, P, P)
        bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, None, pos.h, dX.h, logp.h, P, P)          # a KL term without a reference
        bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, None, dX.h, logp.h, P, P)
        bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, pos.h, dX.h, pos.h, P, P)          # logp is one of the inputs
        bad(capi.nnt_policy_loss, None, X.h, L, pos.h, pos.h, pos.h, dX.h, logp.h, P, P)
        bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, pos.h, dX.h, logp.h, None, P)
        bad(capi.nnt_policy_loss, C.byref(good_p), X.h, L, pos.h, pos.h, T((N_b,), (3,)).h, dX.h, logp.h, P, P)
        for cfg in ((0.0, 0.0, 0), (-1.0, 0.0, 0), (0.1, -0.1, 0), (0.1, 0.6, 0), (0.1, 0.0, 1), (0.1, 0.0, 7), (float("nan"), 0.0, 0)):
            bad(capi.nnt_preference_loss, C.byref(capi.nnt_preference_cfg(*cfg)), X.h, L, pos.h, dX.h, logp.h, P, P, P)
        bad(capi.nnt_preference_loss, C.byref(good_q), X.h, L, pos.h, dX.h, logp.h, None, P, P)
        X3, l3 = T((N_v, N_s, 3), base), T((N_s, 3), base[1:])
        bad(capi.nnt_preference_loss, C.byref(good_q), X3.h, L, None, None, l3.h, P, P, P)                  # no pairs
        assert b"even batch" in capi.nnt_last_error(ctx.h)
        capi.nnt_policy_loss(ctx.h, C.byref(good_p), X.h, L, pos.h, pos.h, pos.h, dX.h, logp.h, P, P)      # the context is still good
        ctx.wait()
        # at tile granularity the calls are one task each, as elsewhere
        ctx.set_granularity(capi.NNT_GRAN_TILE)
        before = ctx.stats()["tasks"]
        capi.nnt_token_logprob(ctx.h, X.h, L, logp.h)
        assert ctx.stats()["tasks"] == before + 1
        assert abs(logp.download() + np.log(N_v)).max() < 1e-5
