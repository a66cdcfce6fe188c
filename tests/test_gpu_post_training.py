"""Post-training of a small language model on the device: log-probabilities of the reference policy, the policy loss or the preference
loss, the backward pass and the Muon step, as one flow, against the fp64 oracle's composition of the same definitions."""
import ctypes as C

import numpy as np
import pytest
import torch

import workload
from gpu_util import TOL, relerr
from oracle import definition as D

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


class Problem:
    """Two blocks, their parameters and a batch whose prompts and paddings have no label."""

    def __init__(self, dtype, N_v=200, tile_v=64):
        self.cfg = cfg = workload.CONFIGS[1].replace(dtype=dtype)
        self.N_v, self.tile_v = N_v, tile_v
        r = np.random.default_rng(41)
        self.inputs = [workload.generate(cfg.replace(index=1 + 5 * i)) for i in range(2)]
        # a head that is sure of something: differences of log-probabilities around 1
        self.wte = (0.3 * r.standard_normal((cfg.N_e, N_v))).astype(np.float32)
        self.wpe = (0.1 * r.standard_normal((cfg.N_e, cfg.N_s))).astype(np.float32)
        self.gf = (1.0 + 0.05 * r.standard_normal(cfg.N_e)).astype(np.float32)
        self.bf = (0.05 * r.standard_normal(cfg.N_e)).astype(np.float32)
        self.tok = r.integers(0, N_v, (cfg.N_s, cfg.N_b))
        self.lab = r.integers(0, N_v, (cfg.N_s, cfg.N_b))
        self.lab[:cfg.N_s // 4] = -1
        self.lab[-5:, 1] = N_v
        self.has = (self.lab >= 0) & (self.lab < N_v)
        self.adv = r.standard_normal(cfg.N_b).astype(np.float32)
        self.shift = 0.15 * r.standard_normal(self.lab.shape).astype(np.float32)       # how far the old policy is from this one
        self.pos = np.repeat(np.arange(cfg.N_s)[:, None], cfg.N_b, axis=1)

    # ---- oracle
    def logits(self, params=None, wte=None):
        cfg = self.cfg
        ps = params or [{k: np.asarray(i[k], np.float64) for k in workload.PARAM_NAMES} for i in self.inputs]
        W = np.asarray(self.wte if wte is None else wte, np.float64)
        X = D.embedding_fwd(W, self.tok) + D.embedding_fwd(self.wpe.astype(np.float64), self.pos)
        caches = []
        for p in ps:
            X, c = D.block_forward(p, X, cfg.N_h, cfg.eps, cfg.gelu)
            caches.append(c)
        Xf, mean, rstd = D.layernorm_fwd(X, self.gf, self.bf, cfg.eps)
        return np.tensordot(W, Xf, (0, 0)), (ps, W, X, caches, Xf, mean, rstd)

    def gradients(self, saved, dlogits):
        ps, W, X, caches, Xf, mean, rstd = saved
        dX, dgf, dbf = D.layernorm_bwd(X, self.gf, mean, rstd, np.tensordot(W, dlogits, (1, 0)))
        out = [None, None]
        for i in (1, 0):
            dX, out[i] = D.block_backward(ps[i], caches[i], dX, self.cfg.N_h, self.cfg.gelu)
        dwte = np.tensordot(Xf, dlogits, ((1, 2), (1, 2))) + D.embedding_bwd(dX, self.tok, self.N_v)
        return out, dict(wte=dwte, wpe=D.embedding_bwd(dX, self.pos, self.cfg.N_s), gamma=dgf, beta=dbf)

    # ---- device
    def model(self, tiled, ctx, adam=True):
        cfg, tiles = self.cfg, workload.base_tiles(self.cfg)
        blks = [tiled.Gpt2Block(ctx, cfg.N_e, cfg.N_h, cfg.N_m, cfg.N_s, cfg.N_b, tiles, dtype=cfg.dtype, adam=adam) for _ in range(2)]
        for b, inp in zip(blks, self.inputs):
            b.set_params({k: inp[k] for k in workload.PARAM_NAMES})
        m = tiled.Gpt2Model(ctx, blks, self.N_v, self.tile_v)
        m.set_params(self.wte, self.wpe, self.gf, self.bf)
        m.set_batch(self.tok, self.lab)
        return m

    def check_gradients(self, m, blocks, own, more):
        """`more`: by how much of itself dloss/dlogp moves with the errors of the log-probabilities; the gradients are linear in it."""
        tol = TOL[self.cfg.dtype] + more
        for i, b in enumerate(m.blocks):
            for k in workload.PARAM_NAMES:
                assert relerr(b.grad(k).download(), blocks[i][k]) <= tol, (i, k)
        for k, ref in own.items():
            assert relerr(getattr(m, k)["g"].download(), ref) <= tol, k


def close(m):
    m.close()
    for b in m.blocks:
        b.close()


MATRICES = ("W_qkv", "W_o", "W_1", "W_2")


def check_muon(m, before, lr, hyper):
    """The new parameters are the oracle's step from the device's own gradients (how exact those are is checked by themselves)."""
    for b, (params, momenta) in zip(m.blocks, before):
        for k in MATRICES:
            g = b.grad(k).download().astype(np.float64)
            p, n = D.muon_step(params[k], g, momenta[k], **hyper)
            assert relerr(b.moment(k, "m").download(), n) <= 1e-6, k
            got = b.param(k).download().astype(np.float64)
            # fp16 halves and fp32 sums: 2^-22 of every factor, times at most 3.4445^5 where singular values are small
            s = lr * 0.2 * np.sqrt(max(p.shape))
            assert np.linalg.norm(got - p) <= s * 1.5 * 2.0 ** -22 * (8 * 3.4445 ** 5 + 64 * np.sqrt(min(p.shape))) + 1e-6 * np.linalg.norm(p), k
            if b.dtype == 1:
                low = b.slots[m.capi.NNT_BLK_LOWP + MATRICES.index(k)].download()
                np.testing.assert_array_equal(low, torch.from_numpy(np.float32(got)).bfloat16().float().numpy())
        for k in ("b_qkv", "gamma2"):
            g = b.grad(k).download().astype(np.float64)
            p, mm, vv = D.adam_step(params[k], g, np.zeros_like(g), np.zeros_like(g), 1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
            assert relerr(b.moment(k, "m").download(), mm) <= 1e-5 and relerr(b.moment(k, "v").download(), vv) <= 1e-5
            assert np.abs(b.param(k).download() - p).max() <= 1e-6 + 1e-5 * np.abs(p).max(), k


def snapshot(m):
    return [({k: b.param(k).download().astype(np.float64) for k in workload.PARAM_NAMES}, {k: b.moment(k, "m").download().astype(np.float64) for k in MATRICES})
            for b in m.blocks]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_policy_step(mods, dtype):
    capi, tiled = mods
    q = Problem(dtype)
    logits, saved = q.logits()
    lp = D.token_logprob(logits, q.lab)
    old = np.float32(lp + q.shift)
    ref = np.float32(lp - 2 * q.shift)
    L, losses, _, dlogits = D.policy_loss(logits, q.lab, old, ref, q.adv, 0.2, 0.25, 0.1, "tokens")
    blocks, own = q.gradients(saved, dlogits)
    with tiled.Context(n_streams=4) as ctx:
        m = q.model(tiled, ctx)
        m.capi = capi
        now, logp = m.per_position(), m.per_position()
        m.logprob(now)
        # bf16: logits as exact as the framework's activations are held to be, 2e-2 of the largest one; a log-probability is off by a logit and the
        # logarithm of a sum of such
        assert np.abs(now.download() - lp).max() <= (2e-5 if dtype == "f32" else 2 * TOL["bf16"] * np.abs(logits).max())
        with pytest.raises(capi.NntError):                    # the logits hold no gradient
            m.backward()
        adv = tiled.TiledTensor.from_numpy(ctx, q.adv, m.logits.base[2:])
        told, tref = m.per_position(old), m.per_position(ref)
        if dtype == "bf16":
            # the ratio sees the rounding of the logits: take the device's own log-probabilities as the point to be near to
            here = now.download()
            old, ref = np.float32(np.where(q.has, here + q.shift, 0)), np.float32(np.where(q.has, here - 2 * q.shift, 0))
            told.upload(old)
            tref.upload(ref)
        m.forward_policy(adv, logp, old=told, ref=tref, clip_low=0.2, clip_high=0.25, kl_coef=0.1, reduction="tokens")
        np.testing.assert_array_equal(logp.download(), now.download())
        if dtype == "f32":
            got = m.col_loss.cpu().numpy().reshape(q.cfg.N_b, q.cfg.N_s).T
            assert np.abs(got - losses).max() <= 1e-4 * np.abs(losses).max() and abs(m.loss.item() - L) <= 1e-4 * max(abs(L), np.abs(losses).max())
        m.backward()
        ctx.wait()
        if dtype == "f32":
            # dloss/dlogp = -r A + kl (1 - e^k): r and e^k move by the 2e-5 of themselves that logp may be off (asserted above), and with |A| <= 2.5 and
            # kl e^k <= 0.2 the second part is at most as large again where the first is clipped
            q.check_gradients(m, blocks, own, 4e-5)
        before = snapshot(m)
        m.muon(1, lr=0.02, momentum=0.9)
        check_muon(m, before, 0.02, dict(lr=0.02, momentum=0.9, nesterov=True, scale="rms"))
        # the policy after it is another one
        after = m.per_position()
        m.logprob(after)
        assert np.abs(after.download() - now.download()).max() > 1e-3
        close(m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_preference_step(mods, dtype):
    capi, tiled = mods
    q = Problem(dtype)
    assert q.cfg.N_b % 2 == 0
    logits, saved = q.logits()
    ref = np.float32(D.token_logprob(logits, q.lab) + q.shift)
    L, losses, rewards, lp, dlogits = D.preference_loss(logits, q.lab, ref, 0.2, 0.1, True)
    blocks, own = q.gradients(saved, dlogits)
    with tiled.Context(n_streams=4) as ctx:
        m = q.model(tiled, ctx)
        m.capi = capi
        logp = m.per_position()
        m.forward_preference(logp, ref=m.per_position(ref), beta=0.2, label_smoothing=0.1)
        m.backward()
        ctx.wait()
        if dtype == "f32":
            assert np.abs(logp.download() - lp).max() <= 2e-5
            assert np.abs(m.rewards.cpu().numpy() - rewards).max() <= 0.2 * 2e-5 * q.has.sum(axis=0).max()
            assert abs(m.loss.item() - L) <= 1e-4 * L
            # the slope sig(z) - 0.9 moves by at most z's error, of up to 2 n log-probabilities times beta, and is at least 0.1 of it in size here
            q.check_gradients(m, blocks, own, 10 * 0.2 * 2e-5 * 2 * q.has.sum(axis=0).max())
        else:
            # (as in the step above, for every position)
            assert np.abs(m.rewards.cpu().numpy() - rewards).max() <= 0.2 * 2 * TOL["bf16"] * np.abs(logits).max() * q.has.sum(axis=0).max()
        before = snapshot(m)
        m.stack.muon(1, lr=0.02, momentum=0.9)
        check_muon(m, before, 0.02, dict(lr=0.02, momentum=0.9, nesterov=True, scale="rms"))
        close(m)


def test_gradients_against_differences(mods):
    """The directional derivative of both losses along a random direction of one matrix, by central differences of the device's own fp32 losses:
    rounding of a loss of about 1 is 1e-6 of it, the step moves it by a few hundredths, the cubic term stays below 1 %."""
    capi, tiled = mods
    q = Problem("f32")
    r = np.random.default_rng(3)
    logits, _ = q.logits()
    lp = D.token_logprob(logits, q.lab)
    old, ref = np.float32(lp), np.float32(lp + q.shift)
    with tiled.Context(n_streams=2) as ctx:
        m = q.model(tiled, ctx, adam=False)
        logp, told, tref = m.per_position(), m.per_position(old), m.per_position(ref)
        adv = tiled.TiledTensor.from_numpy(ctx, q.adv, m.logits.base[2:])
        # (a clip range that this step does not reach: the loss is smooth)
        losses = {"policy": lambda: m.forward_policy(adv, logp, old=told, ref=tref, clip_low=0.9, clip_high=9.0, kl_coef=0.2, reduction="sum"),
                  "preference": lambda: m.forward_preference(logp, ref=tref, beta=0.5, reduction="sum")}
        for name, go in losses.items():
            go()
            m.backward()
            ctx.wait()
            for b, k in ((m.blocks[0], "W_1"), (m.blocks[1], "W_qkv")):
                p, g = b.param(k).download(), b.grad(k).download().astype(np.float64)
                d = r.standard_normal(p.shape)
                d *= 0.5 / np.linalg.norm(d)
                d += 0.5 * g / np.linalg.norm(g)
                f = []
                h = 2e-2 / max(1.0, np.linalg.norm(g))
                for sign in (1, -1):
                    b.param(k).upload(np.float32(p + sign * h * d))
                    go()
                    ctx.wait()
                    f.append(m.col_loss.double().sum().item() if name == "policy" else m.loss.double().item())
                b.param(k).upload(p)
                want = float((g * d).sum())
                assert abs((f[0] - f[1]) / (2 * h) - want) <= 2e-2 * abs(want), (name, k)
        close(m)


def test_step_captured_and_replayed(mods):
    capi, tiled = mods
    q = Problem("f32")
    with tiled.Context(n_streams=2) as ctx:
        m = q.model(tiled, ctx)
        logp, old = m.per_position(), m.per_position()
        adv = tiled.TiledTensor.from_numpy(ctx, q.adv, m.logits.base[2:])

        def go():
            m.forward_policy(adv, logp, old=old, ref=old, kl_coef=0.1)
            m.backward()
            m.muon(1, lr=0.01)
        m.logprob(old)
        go()
        ctx.wait()
        g = C.c_void_p()
        capi.nnt_capture_begin(ctx.h)
        go()
        capi.nnt_capture_end(ctx.h, C.byref(g))
        tensors = [b.param(k) for b in m.blocks for k in MATRICES] + [b.moment(k, "m") for b in m.blocks for k in MATRICES] + [m.wte["p"], m.wte["m"], m.wte["v"]]
        every = [t for b in m.blocks for t in b.slots[:48] if t is not None] + [t for t in m.slots[:16] if t is not None]
        for i in range(3):
            ctx.wait()
            kept = [t.buf.clone() for t in every]
            torch.cuda.synchronize()
            capi.nnt_graph_launch(g)
            replayed = [t.download() for t in tensors]
            for t, k in zip(every, kept):
                t.buf.copy_(k)
            torch.cuda.synchronize()
            go()
            for t, a in zip(tensors, replayed):
                # (positions that share a token are summed in any order)
                assert relerr(t.download(), a) <= 1e-5
            assert relerr(logp.download(), old.download()) > 1e-4        # the policy moves
        capi.nnt_graph_destroy(g)
        close(m)


def test_refusals(mods):
    capi, tiled = mods
    q = Problem("f32")
    with tiled.Context(n_streams=1) as ctx:
        m = q.model(tiled, ctx, adam=False)
        logp, wrong = m.per_position(), tiled.TiledTensor(ctx, "f32", (q.cfg.N_s + 1, q.cfg.N_b), m.logits.base[1:], fill=0)
        cfg, acfg, pcfg, dcfg = tiled.muon_cfg(), capi.nnt_adam_cfg(1e-3, 0.9, 0.999, 1e-8, 0.0), capi.nnt_policy_cfg(0.2, 0.2, 0.0, 0), capi.nnt_preference_cfg(0.1, 0.0, 0)
        b = m.blocks[0]
        assert capi.nnt_gpt2_block_muon.raw(b.h, C.byref(cfg), 1, C.byref(acfg)) == capi.NNT_ESTATE          # no moments
        assert capi.nnt_gpt2_stack_muon.raw(m.stack.h, C.byref(cfg), 1, C.byref(acfg)) == capi.NNT_ESTATE
        for bad in ((None, 1, C.byref(acfg)), (C.byref(cfg), 0, C.byref(acfg)), (C.byref(cfg), 1, None)):
            assert capi.nnt_gpt2_block_muon.raw(b.h, *bad) == capi.NNT_EINVAL
            assert capi.nnt_gpt2_stack_muon.raw(m.stack.h, *bad) == capi.NNT_EINVAL
            assert capi.nnt_gpt2_model_muon.raw(m.h, *bad) == capi.NNT_EINVAL
        T, P, L = m.tokens.data_ptr(), m.pos.data_ptr(), m.labels.data_ptr()
        f = m.col_loss.data_ptr()
        assert capi.nnt_gpt2_model_logprob.raw(m.h, T, P, L, wrong.h) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_logprob.raw(m.h, T, P, None, logp.h) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_forward_policy.raw(m.h, T, P, L, C.byref(pcfg), wrong.h, None, logp.h, logp.h, f, f) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_forward_policy.raw(m.h, T, P, L, None, None, None, logp.h, logp.h, f, f) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_forward_preference.raw(m.h, T, P, L, C.byref(dcfg), wrong.h, logp.h, f, f, f) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_forward_preference.raw(m.h, None, P, L, C.byref(dcfg), None, logp.h, f, f, f) == capi.NNT_EINVAL
        assert capi.nnt_gpt2_model_backward.raw(m.h) == capi.NNT_ESTATE                                       # nothing has been differentiated
        for fn in (capi.nnt_gpt2_block_muon, capi.nnt_gpt2_stack_muon, capi.nnt_gpt2_model_muon):
            assert fn.raw(None, C.byref(cfg), 1, C.byref(acfg)) == capi.NNT_EINVAL
        ctx.wait()
        close(m)
