"""The losses on given tokens entry by entry: every gradient entry within its own rounding, over the instances that many columns, large gradients and odd
addresses take, and labels that are themselves banned."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_util import quant
from oracle import definition as D
from test_gpu_token_losses import HALF, LOGP, REL, Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N_v,base_v", [(100, 30), (1000, 300), (50304, 8192), (140003, 32768)])
def test_labels_that_are_banned(mods, N_v, base_v, dtype):
    """A label whose logit is -inf: logp is -inf, and against itself (no old policy) the ratio is 1, whatever the advantage."""
    r = np.random.default_rng(11)
    lab = r.integers(0, N_v, (3, 2))
    X = quant(r.standard_normal((N_v, 3, 2)), dtype)
    for s, b in ((0, 0), (1, 0), (2, 1)):
        X[lab[s, b], s, b] = -np.inf
    adv = np.array([[1.5, -2.0], [0.0, 1.0], [0.5, -0.75]])
    with np.errstate(invalid="ignore"):
        L, losses, logp, dX = D.policy_loss(X, lab, None, None, adv)
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, (base_v, 2, 2), dtype, adv=adv)
        c.policy()
        banned = np.isneginf(logp)
        assert banned.sum() == 3
        got = c.logp.download()
        assert np.isneginf(got[banned]).all()
        c.close_to(got[~banned], logp[~banned], HALF["f32"], LOGP, "logp")
        c.close_to(c.check_sum(lab.size, losses), losses.reshape(-1, order="F"), 1e-6, 0.0, "losses")
        c.close_to(c.dX.download(), dX, HALF[dtype] + REL, REL * np.abs(adv)[None] * (np.arange(N_v)[:, None, None] == lab[None]), "gradient")


class Columns:
    """Logits made on the device, N_s x N_b columns of N_v, and what the losses of them are in 64 bits."""

    def __init__(self, mods, ctx, dtype, shape, base, seed):
        capi, tiled = self.mods = mods
        self.ctx, self.dtype, self.shape = ctx, dtype, shape
        N_v, N_s, N_b = shape
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.x = (2.0 * torch.randn(N_b, N_s, N_v, generator=g, device="cuda")).to(t)
        self.lab = torch.randint(0, N_v, (N_b, N_s), generator=g, device="cuda", dtype=torch.int32)
        at = self.lab.long().unsqueeze(-1)
        self.x.scatter_(2, at, (self.x.gather(2, at).float() + 12.0 * torch.rand(N_b, N_s, 1, generator=g, device="cuda")).to(t))
        out = torch.rand(N_b, N_s, generator=g, device="cuda") < 0.2
        self.lab[out] = -1
        self.has = ~out
        self.X, self.dX = (tiled.TiledTensor(ctx, dtype, shape, base) for _ in range(2))
        self.dX.buf.fill_(0x5a)
        for k, idx in enumerate(self.X.tile_index):
            self.X.tile_view(k).copy_(self.of_tile(self.x, idx).reshape(-1))
        self.logp, self.ref, self.adv = (tiled.TiledTensor(ctx, "f32", shape[1:], base[1:], fill=0) for _ in range(3))
        self.losses, self.rewards, self.loss = torch.zeros(N_s * N_b, device="cuda"), torch.zeros(N_b, device="cuda"), torch.zeros(1, device="cuda")
        x = self.x.double()
        self.want = torch.log_softmax(x, 2)
        self.label_logp = torch.where(self.has, self.want.gather(2, self.lab.long().clamp_min(0).unsqueeze(-1))[..., 0], torch.zeros((), dtype=torch.float64, device="cuda"))

    def of_tile(self, a, idx):
        """The part of an array (axes reversed) that a tile holds."""
        return a[tuple(reversed(self.X.slices(idx)))]

    def dense(self, t):
        """A tensor of one value per position as [N_b, N_s]."""
        out = torch.empty(self.shape[2], self.shape[1], device="cuda", dtype=torch.float64)
        for k, idx in enumerate(t.tile_index):
            part = out[tuple(reversed(t.slices(idx)))]
            part.copy_(t.tile_view(k).view(part.shape).double())
        return out

    def fill(self, t, a):
        for k, idx in enumerate(t.tile_index):
            t.tile_view(k).copy_(a[tuple(reversed(t.slices(idx)))].float().reshape(-1))

    def check_logp(self):
        d = (self.dense(self.logp) - self.label_logp).abs()
        assert (d <= HALF["f32"] * self.label_logp.abs() + LOGP).all(), d.max()

    def check_gradient(self, g, slack):
        """dX = g ([j = label] - softmax): each entry to its own rounding, the label's, where 1 - p cancels, to REL of g; `slack`: relative error of g besides."""
        g = torch.where(self.has, g, torch.zeros_like(g))
        p = self.want.exp_()
        want = p.mul_(-g.unsqueeze(-1))
        at = self.lab.long().clamp_min(0).unsqueeze(-1)
        limit = want.abs().mul_(REL + slack)
        limit.scatter_add_(2, at, ((REL + slack) * g.abs()).unsqueeze(-1))
        want.scatter_add_(2, at, g.unsqueeze(-1))
        limit.add_(want.abs(), alpha=HALF[self.dtype])        # the result's own rounding
        for k, idx in enumerate(self.dX.tile_index):
            w, l = self.of_tile(want, idx), self.of_tile(limit, idx)
            got = self.dX.tile_view(k).view(w.shape).double()
            bad = ~((got - w).abs() <= l)
            assert not bad.any(), "tile %d: %d of %d, first %s: %r for %r" % (k, bad.sum(), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), w[bad][0].item())


# (N_v, N_s, N_b), tiles: one wavefront to a column with few and with many registers; four to a long column of many; the widest columns in registers; a column read twice;
# gradients of more than 128 MiB on addresses of any element, in fp32 and bf16
MANY = [("f32", (513, 300, 2), (200, 128, 1)), ("f32", (1024, 128, 4), (1024, 128, 4)), ("f32", (4093, 171, 3), (1000, 64, 2)), ("bf16", (1000, 256, 2), (333, 100, 2)),
        ("bf16", (1021, 520, 1), (1021, 520, 1)), ("bf16", (4090, 150, 4), (1500, 64, 4)), ("f32", (20011, 520, 2), (8192, 128, 2)), ("bf16", (20011, 520, 2), (8192, 128, 2)),
        ("f32", (16000, 64, 4), (5000, 64, 4)), ("f32", (33001, 280, 4), (8191, 100, 4)), ("bf16", (33001, 560, 4), (8191, 100, 4)), ("f32", (140003, 65, 4), (32767, 64, 4)),
        ("bf16", (140003, 130, 4), (32767, 64, 4)), ("f32", (65536, 130, 4), (8192, 130, 4)), ("bf16", (50304, 360, 4), (8192, 360, 4))]


@pytest.mark.parametrize("dtype,shape,base", MANY)
def test_policy_loss_entry_by_entry(mods, dtype, shape, base):
    capi, tiled = mods
    with tiled.Context(n_streams=2) as ctx:
        c = Columns(mods, ctx, dtype, shape, base, sum(shape))
        g = torch.Generator(device="cuda").manual_seed(1)
        adv = torch.randn(shape[2], shape[1], generator=g, device="cuda")
        c.fill(c.adv, adv)
        torch.cuda.synchronize()
        # against itself: dloss/dlogp = -A, without an error of its own
        capi.nnt_policy_loss(ctx.h, C.byref(capi.nnt_policy_cfg(0.2, 0.2, 0.0, 0)), c.X.h, c.lab.data_ptr(), None, None, c.adv.h, c.dX.h, c.logp.h, c.losses.data_ptr(), c.loss.data_ptr())
        ctx.wait()
        c.check_logp()
        assert torch.equal(c.losses.view(shape[2], shape[1]), torch.where(c.has, -adv, torch.zeros_like(adv)))
        c.check_gradient(-adv.double(), 0.0)
        # the log-probabilities alone, by kernels of their own
        c.logp.buf.fill_(0x5a)
        torch.cuda.synchronize()
        capi.nnt_token_logprob(ctx.h, c.X.h, c.lab.data_ptr(), c.logp.h)
        ctx.wait()
        c.check_logp()


@pytest.mark.parametrize("dtype,shape,base", [m for m in MANY if m[1][2] % 2 == 0])
def test_preference_loss_entry_by_entry(mods, dtype, shape, base):
    capi, tiled = mods
    beta, soft, n = 0.1, 0.05, shape[2] // 2
    with tiled.Context(n_streams=2) as ctx:
        c = Columns(mods, ctx, dtype, shape, base, sum(shape))
        ref = c.label_logp + 0.1 * torch.randn(shape[2], shape[1], generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
        c.fill(c.ref, ref)
        torch.cuda.synchronize()
        capi.nnt_preference_loss(ctx.h, C.byref(capi.nnt_preference_cfg(beta, soft, 2)), c.X.h, c.lab.data_ptr(), c.ref.h, c.dX.h, c.logp.h, c.rewards.data_ptr(),
                                 c.losses.data_ptr(), c.loss.data_ptr())
        ctx.wait()
        c.check_logp()
        R = c.rewards.double()
        count = c.has.sum(1)
        want = beta * torch.where(c.has, c.label_logp - c.dense(c.ref), torch.zeros_like(c.label_logp)).sum(1)
        assert ((R - want).abs() <= HALF["f32"] * want.abs() + beta * LOGP * count).all()
        # the gradient that belongs to these rewards, which are rounded to 32 bits on their way out: the slope moves by a quarter of that at most
        z = R[:n] - R[n:]
        slope = (torch.sigmoid(z) - (1.0 - soft)) * beta / n
        slack = (HALF["f32"] * (R[:n].abs() + R[n:].abs()) / 4 * beta / n / slope.abs()).max().item()
        c.check_gradient(torch.cat([slope, -slope]).unsqueeze(-1) * c.has, slack)


@pytest.mark.parametrize("term", ["ratio", "kl"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ratios_beyond_32_bits(mods, dtype, term):
    """exp(89.5) is no number of fp32, but a two-thousandth of it is: loss and gradient are weighted before they are rounded."""
    r = np.random.default_rng(12)
    N_v, N_s, N_b = 50, 1000, 2
    lab = r.integers(0, N_v, (N_s, N_b))
    X = quant(r.standard_normal((N_v, N_s, N_b)), dtype)
    logp = D.token_logprob(X, lab)
    old, ref = logp.copy(), logp.copy()
    if term == "ratio":
        old[::50] -= 89.5                                     # a negative advantage is not clipped from above
    else:
        ref[::50] += 89.5
    old, ref = np.float32(old), np.float32(ref)
    adv = -np.ones((N_s, N_b))
    L, losses, logp, dX = D.policy_loss(X, lab, old, ref, adv, 0.2, 0.2, 0.5, "tokens")
    assert np.abs(losses).max() > 1e35
    with mods[1].Context(n_streams=2) as ctx:
        c = Call(mods, ctx, X, lab, (N_v, 128, 2), dtype, old=old, ref=ref, adv=adv)
        c.policy(0.2, 0.2, 0.5, 1)
        # e^d moves by the 8e-6 of itself that a log-probability may be off; around d = 0 the loss does by as much of the weight
        w = 1.0 / lab.size
        got = c.losses[:lab.size].double().cpu().numpy()
        assert np.isfinite(got).all()
        c.close_to(got, losses.reshape(-1, order="F"), LOGP + 2.0 ** -22, 2 * LOGP * w, "losses")
        g = np.abs(dX).sum(axis=0)
        c.close_to(c.dX.download(), dX, HALF[dtype] + REL + LOGP, (REL + LOGP) * g[None] + 2 * LOGP * w, "gradient")
