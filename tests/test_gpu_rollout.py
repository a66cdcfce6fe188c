"""Cache, attention over it, drawn tokens and clipped gradients as they are used: a model generates over a cache what its forward pass over
whole sequences says, in parts and token by token, with draws that feed the next step; and one iteration of a policy's training."""
import ctypes as C

import numpy as np
import pytest

from gpu_util import TOL
from oracle import rollout as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

N_V = 61


def make(ctx, dtype, N_s, N_b, share=None, N_e=64, N_h=4, n_blocks=2, h_tiles=2, seed=3):
    """A small model; with `share` one of another sequence length on the same parameters."""
    from paper_2504_13236_amd import tiled
    h = N_e // N_h
    tiles = dict(e=h_tiles * h, m=96, s=8, b=2, j=h_tiles, i=h)
    blocks = [tiled.Gpt2Block(ctx, N_e, N_h, 2 * N_e, N_s, N_b, tiles, dtype=dtype, share=None if share is None else share.blocks[k]) for k in range(n_blocks)]
    model = tiled.Gpt2Model(ctx, blocks, N_V, 24, share=share)
    if share is None:
        r = np.random.default_rng(seed)
        for b in blocks:
            p = {n: 0.25 * r.standard_normal(b.param(n).shape) for n in tiled.PARAM_SLOTS}
            p["gamma1"], p["gamma2"] = 1 + 0.1 * p["gamma1"], 1 + 0.1 * p["gamma2"]
            b.set_params(p)
        model.set_params(0.6 * r.standard_normal((N_e, N_V)), 0.3 * r.standard_normal((N_e, N_s)), 1 + 0.1 * r.standard_normal(N_e), 0.1 * r.standard_normal(N_e))
    return model


def cache_for(ctx, model, page, n_positions, dtype):
    from paper_2504_13236_amd import tiled
    b = model.blocks[0].cfg
    per = -(-n_positions // page)
    c = tiled.PagedCache(ctx, len(model.blocks), b.N_e // b.N_h, b.N_h, b.N_h, page, per * model.N_b + 3, model.N_b, per + 1, dtype=dtype)
    c.reserve([n_positions] * model.N_b)
    return c


def ints(a):
    t = torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()
    torch.cuda.synchronize()
    return t


def close(*models):
    for m in models:
        m.close()
        for b in m.blocks:
            b.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("part", [1, 5, 16])
def test_generation_over_a_cache_is_the_whole_forward_pass(dtype, part):
    """Given tokens in parts of `part` through the cache: the logits of the forward pass over whole sequences (each is within the framework's bound
    of the exact ones, so they are within twice that of each other)."""
    from paper_2504_13236_amd import tiled
    with tiled.Context(n_streams=3) as ctx:
        N_s, N_b = 16, 3
        whole = make(ctx, dtype, N_s, N_b)
        step = make(ctx, dtype, part, N_b, share=whole)
        tokens = np.random.default_rng(5).integers(0, N_V, (N_s, N_b))
        whole.set_batch(tokens, np.zeros_like(tokens))
        logp = whole.per_position()
        whole.logprob(logp)
        want = whole.logits.download()
        cache = cache_for(ctx, whole, 5, N_s, dtype)
        drawn = torch.zeros(part * N_b, dtype=torch.int32, device="cuda")
        u = torch.full((part * N_b,), 0.5, device="cuda")
        for s0 in range(0, N_s, part):
            n = min(part, N_s - s0)
            batch = np.zeros((part, N_b), int)
            batch[:n] = tokens[s0:s0 + n]
            pos = np.repeat(np.minimum(np.arange(s0, s0 + part), N_s - 1)[:, None], N_b, 1)
            t, p, start, count = ints(batch.T.reshape(-1)), ints(pos.T.reshape(-1)), ints([s0] * N_b), ints([n] * N_b)
            step.sample(cache, start, u, drawn, count=count, positions=p, tokens=t, top_k=9)
            got = step.logits.download()[:, :n]
            ref = want[:, s0:s0 + n]
            assert np.abs(got - ref).max() <= 2 * TOL[dtype] * np.abs(want).max()
            d = drawn.cpu().numpy().reshape(N_b, part)
            for b in range(N_b):
                for i in range(n):
                    assert d[b, i] == R.sample_token(got[:, i, b], 0.5, top_k=9)[0]
        close(step, whole)


def test_draws_feed_the_next_step_without_a_wait():
    """A chain of steps on four streams, each lookup of tokens waiting for the draw before it; eager, and captured and replayed per step; sequences of
    different lengths.  The log-probabilities of what was drawn are those that the forward pass over the whole answers gives."""
    from paper_2504_13236_amd import capi, tiled
    with tiled.Context(n_streams=4) as ctx:
        N_s, N_b, first = 24, 4, [6, 1, 3, 4]
        whole = make(ctx, "f32", N_s, N_b)
        prompt, step = make(ctx, "f32", 6, N_b, share=whole), make(ctx, "f32", 1, N_b, share=whole)
        r = np.random.default_rng(6)
        tokens = r.integers(0, N_V, (N_s, N_b))
        n_new = 14
        uniforms = torch.from_numpy(r.random((n_new, N_b)).astype(np.float32)).cuda()
        starts = torch.tensor([[f + k - 1 for f in first] for k in range(n_new)], dtype=torch.int32, device="cuda")
        t_prompt, zero, count = ints(tokens[:6].T.reshape(-1)), ints([0] * N_b), ints(first)
        columns = ints([f - 1 + 6 * b for b, f in enumerate(first)])
        results = []
        for captured in (False, True):
            cache = cache_for(ctx, whole, 4, N_s, "f32")
            drawn = torch.zeros((n_new, N_b), dtype=torch.int32, device="cuda")
            logp = torch.zeros((n_new, N_b), device="cuda")
            torch.cuda.synchronize()

            def go(k):
                if k == 0:
                    prompt.sample(cache, zero, uniforms[0], drawn[0], count=count, columns=columns, logp=logp[0], tokens=t_prompt, top_p=0.9, temperature=0.9)
                else:
                    step.sample(cache, starts[k], uniforms[k], drawn[k], logp=logp[k], positions=starts[k], tokens=drawn[k - 1], top_p=0.9, temperature=0.9)
            if captured:
                for k in range(2):
                    go(k)                         # plans and scratch exist from here on
                ctx.wait()
                g = C.c_void_p()
                capi.nnt_capture_begin(ctx.h)
                for k in range(n_new):
                    go(k)
                capi.nnt_capture_end(ctx.h, C.byref(g))
                for _ in range(3):
                    drawn.zero_()
                    torch.cuda.synchronize()
                    capi.nnt_graph_launch(g)
                    ctx.wait()
                capi.nnt_graph_destroy(g)
            else:
                for k in range(n_new):
                    go(k)
            ctx.wait()
            results.append((drawn.cpu().numpy(), logp.cpu().numpy()))
        assert np.array_equal(results[0][0], results[1][0]) and np.array_equal(results[0][1], results[1][1])
        d, lp = results[0]
        answer, labels = tokens.copy(), np.full((N_s, N_b), -1)
        for b, f in enumerate(first):
            answer[f:f + n_new, b] = d[:, b]
            labels[f - 1:f - 1 + n_new, b] = d[:, b]
        whole.set_batch(answer, labels)
        got = whole.per_position()
        whole.logprob(got)
        full = got.download()
        scale = np.abs(whole.logits.download()).max()
        for b, f in enumerate(first):
            assert np.abs(full[f - 1:f - 1 + n_new, b] - lp[:, b]).max() <= 4 * TOL["f32"] * scale
        close(step, prompt, whole)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_iteration_of_a_policys_training(dtype):
    """Answers drawn over a cache, their log-probabilities, the policy loss and its gradients, clipped, and a step of the optimiser: the clipped gradients are
    the unclipped ones times one factor, and the step is that of those gradients."""
    from paper_2504_13236_amd import capi, tiled
    with tiled.Context(n_streams=2) as ctx:
        N_s, N_b, n_prompt = 12, 4, 3
        whole = make(ctx, dtype, N_s, N_b)
        prompt, step = make(ctx, dtype, n_prompt, N_b, share=whole), make(ctx, dtype, 1, N_b, share=whole)
        r = np.random.default_rng(8)
        tokens = r.integers(0, N_V, (N_s, N_b))
        cache = cache_for(ctx, whole, 4, N_s, dtype)
        u = torch.from_numpy(r.random((N_s, N_b)).astype(np.float32)).cuda()
        drawn = torch.zeros((N_s, N_b), dtype=torch.int32, device="cuda")
        t, zero = ints(tokens[:n_prompt].T.reshape(-1)), ints([0] * N_b)
        columns = ints([n_prompt - 1 + n_prompt * b for b in range(N_b)])
        starts = [ints([s] * N_b) for s in range(N_s)]
        prompt.sample(cache, zero, u[n_prompt], drawn[n_prompt], columns=columns, tokens=t, temperature=1.2)
        for s in range(n_prompt, N_s - 1):
            step.sample(cache, starts[s], u[s + 1], drawn[s + 1], tokens=drawn[s], positions=starts[s], temperature=1.2)
        ctx.wait()
        tokens[n_prompt:] = drawn.cpu().numpy()[n_prompt:]
        assert (tokens >= 0).all() and (tokens < N_V).all()
        labels = np.full((N_s, N_b), -1)
        labels[n_prompt - 1:N_s - 1] = tokens[n_prompt:]
        whole.set_batch(tokens, labels)
        old, logp = whole.per_position(), whole.per_position()
        whole.logprob(old)
        adv = whole.per_position(np.broadcast_to(r.standard_normal(N_b), (N_s, N_b)))
        whole.forward_policy(adv, logp, old=old, reduction="tokens")
        whole.backward()
        grads = [b.slots[capi.NNT_BLK_GRAD + p] for b in whole.blocks for p in range(12)] + [whole.slots[capi.NNT_MDL_GRAD + p] for p in range(4)]
        before = [g.download() for g in grads]
        norm = torch.zeros(1, device="cuda")
        torch.cuda.synchronize()
        want, n = R.clip_grad_norm(before, 0.05, 1e-6)
        assert n > 0.06
        whole.clip(norm, max_norm=0.05)
        for g, w in zip(grads, want):
            assert (np.abs(g.download() - w) <= 2.0 ** -24 * np.abs(w) * (1 + 1e-6) + 2.0 ** -150).all()
        assert abs(float(norm) - n) <= 2.0 ** -24 * n
        p0 = whole.blocks[0].param("W_o").download()
        whole.adam(1, lr=1e-2, eps=1e-3)
        g = want[1]
        assert whole.blocks[0].slots[capi.NNT_BLK_GRAD + 1] is grads[1]
        # the first step of Adam: lr g / (|g| + eps)
        assert np.abs(whole.blocks[0].param("W_o").download() - (p0 - 1e-2 * g / (np.abs(g) + 1e-3))).max() <= 1e-5 * np.abs(p0).max()
        # the model that generates sees the new parameters
        step.sample(cache, starts[4], u[5], drawn[5], tokens=drawn[4], positions=starts[4])
        ctx.wait()
        close(step, prompt, whole)


def test_refusals():
    from paper_2504_13236_amd import capi, tiled
    with tiled.Context(n_streams=2) as ctx:
        whole = make(ctx, "f32", 8, 2)
        step = make(ctx, "f32", 1, 2, share=whole)
        cache = cache_for(ctx, whole, 4, 8, "f32")
        z, u, nxt = ints([0, 0]), torch.zeros(2, device="cuda"), torch.full((2,), -9, dtype=torch.int32, device="cuda")
        with pytest.raises(ValueError):
            step.sample(cache, z, u, nxt[:1])
        with pytest.raises(ValueError):
            cache.reserve([80, 80])
        bad = capi.NNT_EINVAL
        K, V = capi.ptr_array([t.h.value for t in cache.K]), capi.ptr_array([t.h.value for t in cache.V])

        def call(m=step, ccfg=None, scfg=None, K=K, V=V, tokens=nxt, n=2, columns=None):
            c, s = ccfg or cache.cfg(z), scfg or capi.nnt_sample_cfg(1.0, 1.0, 0.0, 0)
            return capi.nnt_gpt2_model_sample.raw(m.h, tokens.data_ptr() if tokens is not None else None, z.data_ptr(), C.byref(c), K, V, C.byref(s), columns, n,
                                                  u.data_ptr(), nxt.data_ptr(), None)
        few = cache.cfg(z)
        few.N_kv = 2
        wrong = cache.cfg(z)
        wrong.max_pages = 0
        swapped = capi.ptr_array([cache.K[0].h.value, None])
        for kw in (dict(tokens=None), dict(K=None), dict(V=None), dict(ccfg=few), dict(ccfg=wrong), dict(K=swapped), dict(K=V), dict(n=3), dict(n=0),
                   dict(scfg=capi.nnt_sample_cfg(-1.0, 1.0, 0.0, 0))):
            assert call(**kw) == bad, kw
        ctx.wait()
        assert (nxt == -9).all()
        # nothing to go backward from after a step of generation
        assert call() == capi.NNT_OK
        assert capi.nnt_gpt2_model_backward.raw(step.h) == capi.NNT_ESTATE
        assert capi.nnt_gpt2_block_backward.raw(step.blocks[0].h, step.stack.dacts[1].h, step.stack.dacts[0].h) == capi.NNT_ESTATE
        ctx.wait()
        assert (nxt >= 0).all()
        close(step, whole)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_position_embeddings_have_gradients_like_them(dtype):
    from paper_2504_13236_amd import capi, tiled
    with tiled.Context(n_streams=1) as ctx:
        whole = make(ctx, dtype, 8, 2)
        step = make(ctx, dtype, 1, 2, share=whole)
        short = tiled.TiledTensor.zeros(ctx, (whole.N_e, 1), (step.slots[capi.NNT_MDL_WPE].base[0], 1))
        others = [capi.NNT_MDL_WPE + k for k in (capi.NNT_MDL_GRAD, capi.NNT_MDL_ADAM_M, capi.NNT_MDL_ADAM_V)]
        if dtype == "bf16":
            others.append(capi.NNT_MDL_LOWP + capi.NNT_MDL_WPE)
        for slot in others:
            slots = list(step.slots)
            slots[slot] = short if slot < capi.NNT_MDL_LOWP else tiled.TiledTensor.zeros(ctx, (whole.N_e, 1), (short.base[0], 1), "bf16")
            h = C.c_void_p()
            assert capi.nnt_gpt2_model_create.raw(ctx.h, C.byref(step.blocks[0].cfg), N_V, 24, step.stack.h,
                                                  capi.ptr_array([t.h.value if t is not None else None for t in slots]), C.byref(h)) == capi.NNT_EINVAL, slot
            if slots[slot] is not short:
                slots[slot].close()
        short.close()
        close(step, whole)

def test_pages_are_handed_out_and_taken_back():
    from paper_2504_13236_amd import tiled
    with tiled.Context(n_streams=1) as ctx:
        c = tiled.PagedCache(ctx, 1, 8, 1, 1, 4, 6, 3, 4)
        c.reserve([5, 0, 9])
        assert [len(p) for p in c.of] == [2, 0, 3] and len({x for p in c.of for x in p}) == 5
        c.reserve([5, 4, 1])
        assert [len(p) for p in c.of] == [2, 1, 3] and not c.free
        with pytest.raises(ValueError):
            c.reserve([9, 0, 0])
        c.release(2)
        c.reserve([12, 0, 0])
        table = c.pages.cpu().numpy()
        assert (table[2] == -1).all() and (table[0, :3] >= 0).all() and table[0, 3] == -1
