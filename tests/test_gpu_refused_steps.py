"""What a refused optimiser step or forward pass of the language model leaves as it was."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest

from test_gpu_post_training import MATRICES, Problem, check_muon, close, snapshot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    from paper_2504_13236_amd import capi, tiled
    return capi, tiled


def with_gradients(q, tiled, ctx):
    m = q.model(tiled, ctx)
    logp = m.per_position()
    m.forward_preference(logp)
    m.backward()
    ctx.wait()
    return m


@pytest.mark.parametrize("whose", ["block", "stack", "model"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_muon_refused_inside_a_capture_records_nothing(mods, whose, dtype):
    """The vectors' table of pointers does not exist yet and cannot be made there: neither may the matrices be updated."""
    capi, tiled = mods
    q = Problem(dtype)
    with tiled.Context(n_streams=2) as ctx:
        m = with_gradients(q, tiled, ctx)
        cfg, acfg = tiled.muon_cfg(lr=0.02, momentum=0.9), capi.nnt_adam_cfg(1e-3, 0.9, 0.999, 1e-8, 0.0)
        call, h = {"block": (capi.nnt_gpt2_block_muon, m.blocks[1].h), "stack": (capi.nnt_gpt2_stack_muon, m.stack.h), "model": (capi.nnt_gpt2_model_muon, m.h)}[whose]
        if whose != "block":
            m.blocks[0].muon(1, lr=0.0)                       # the first block is prepared, the second is not
        # the matrices' workspace is there
        tiled.muon_step(ctx, *[[f(b, k) for b in m.blocks for k in MATRICES] for f in (lambda b, k: b.grad(k), lambda b, k: b.param(k), lambda b, k: b.moment(k, "m"))], lr=0.0)
        ctx.wait()
        before = snapshot(m)
        g = C.c_void_p()
        capi.nnt_capture_begin(ctx.h)
        launches = ctx.stats()["launches"]
        assert call.raw(h, C.byref(cfg), 1, C.byref(acfg)) == capi.NNT_ESTATE
        assert ctx.stats()["launches"] == launches
        capi.nnt_capture_end(ctx.h, C.byref(g))
        capi.nnt_graph_launch(g)
        ctx.wait()
        capi.nnt_graph_destroy(g)
        for (p0, m0), (p1, m1) in zip(before, snapshot(m)):
            for k in MATRICES:
                np.testing.assert_array_equal(p0[k], p1[k])
                np.testing.assert_array_equal(m0[k], m1[k])
        # the same call outside of a capture is one whole step
        if whose == "block":
            assert call.raw(h, C.byref(cfg), 1, C.byref(acfg)) == capi.NNT_OK
            check_muon(SimpleNamespace(blocks=m.blocks[1:], capi=capi), before[1:], 0.02, dict(lr=0.02, momentum=0.9, nesterov=True, scale="rms"))
        ctx.wait()
        close(m)


@pytest.mark.parametrize("which", ["logprob", "policy", "preference"])
def test_refused_ends_of_the_forward_pass_leave_the_last_one(mods, which):
    """A call that is refused launches nothing, and the pass before it can still go backward."""
    capi, tiled = mods
    q = Problem("f32")
    with tiled.Context(n_streams=2) as ctx:
        m = q.model(tiled, ctx)
        logp, wrong = m.per_position(), tiled.TiledTensor(ctx, "f32", (q.cfg.N_s + 1, q.cfg.N_b), m.logits.base[1:], fill=0)
        adv = tiled.TiledTensor.from_numpy(ctx, q.adv, m.logits.base[2:])
        T, P, L, f = m.tokens.data_ptr(), m.pos.data_ptr(), m.labels.data_ptr(), m.col_loss.data_ptr()
        pcfg, dcfg = capi.nnt_policy_cfg(0.2, 0.2, 0.1, 0), capi.nnt_preference_cfg(-1.0, 0.0, 0)

        def backward():
            m.backward()
            ctx.wait()
            return [b.grad(k).download() for b in m.blocks for k in MATRICES] + [m.gamma["g"].download()]
        m.forward_policy(adv, logp)
        first = backward()
        m.forward_policy(adv, logp)
        ctx.wait()
        launches = ctx.stats()["launches"]
        if which == "logprob":
            assert capi.nnt_gpt2_model_logprob.raw(m.h, T, P, L, wrong.h) == capi.NNT_EINVAL
        elif which == "policy":                               # a KL term without a reference
            assert capi.nnt_gpt2_model_forward_policy.raw(m.h, T, P, L, C.byref(pcfg), None, None, adv.h, logp.h, f, f) == capi.NNT_EINVAL
        else:                                                 # a negative strength
            assert capi.nnt_gpt2_model_forward_preference.raw(m.h, T, P, L, C.byref(dcfg), None, logp.h, f, f, f) == capi.NNT_EINVAL
        assert ctx.stats()["launches"] == launches
        for a, b in zip(first, backward()):
            np.testing.assert_array_equal(a, b)
        close(m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_muon_in_tile_granularity(mods, dtype):
    """One task per tile for the vectors: the same step."""
    capi, tiled = mods
    q = Problem(dtype)
    results = []
    for granularity in (capi.NNT_GRAN_OP, capi.NNT_GRAN_TILE):
        with tiled.Context(n_streams=3) as ctx:
            m = with_gradients(q, tiled, ctx)
            capi.nnt_ctx_set_granularity(ctx.h, granularity)
            m.muon(1, lr=0.02, momentum=0.9)
            ctx.wait()
            results.append([b.param(k).download() for b in m.blocks for k in MATRICES + ("b_qkv", "gamma2")] + [m.wte["p"].download(), m.gamma["p"].download()])
            close(m)
    # (the embeddings' gradients are sums over positions in any order: Adam's first step is lr times their sign, and moves by it where they are 0)
    for a, b in zip(results[0][:-2] + results[0][-1:], results[1][:-2] + results[1][-1:]):
        assert np.abs(a - b).max() <= 1e-6 * np.abs(a).max() + 1e-7
    assert np.abs(results[0][-2] - results[1][-2]).max() <= 2.1e-3
