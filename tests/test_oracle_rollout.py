"""Pins of the oracle's cache, attention over it, drawn tokens and clipped gradients that do not go through the oracle: dense attention of
CPU torch in float64, closed forms, frequencies; and the entry points' answers without a context."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import rollout as R


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_is_a_complex_product(pairs):
    r = np.random.default_rng(1)
    x, angle = r.standard_normal(10), r.standard_normal((4, 3))
    y = R.rotated(x, 2, np.concatenate([np.cos(angle), np.sin(angle)]), pairs)
    z = (x[0:8:2] + 1j * x[1:8:2]) if pairs else (x[:4] + 1j * x[4:8])
    z = z * np.exp(1j * angle[:, 2])
    np.testing.assert_allclose(y[:8], np.stack([z.real, z.imag], 1).reshape(-1) if pairs else np.concatenate([z.real, z.imag]), rtol=1e-14)
    np.testing.assert_array_equal(y[8:], x[8:])


@pytest.mark.parametrize("window", [0, 3])
def test_attention_over_pages_is_dense_causal_attention(window):
    r = np.random.default_rng(2)
    h, N_h, N_kv, N_s, N_b, P, n_pages = 8, 4, 2, 5, 2, 4, 9
    QKV = r.standard_normal(((N_h + 2 * N_kv) * h, N_s, N_b))
    K, V = r.standard_normal((2, h, n_pages * P, N_kv))
    pages = np.array([[3, 0], [7, 1], [2, -1], [8, 5]])
    start, count = np.array([6, 2]), np.array([5, 3])
    K, V = R.cache_append(QKV, K, V, P, N_h, pages, start, count)
    B, _ = R.cache_attention(QKV, K, V, np.full((N_h * h, N_s, N_b), 7.0), P, N_h, 0.3, pages, start, count, window=window)
    for b in range(N_b):
        at = [pages[p // P, b] * P + p % P for p in range(start[b] + count[b])]
        for j in range(N_h):
            q, k, v = (torch.from_numpy(np.ascontiguousarray(a.T)) for a in (QKV[j * h:(j + 1) * h, :count[b], b], K[:, at, j // 2], V[:, at, j // 2]))
            np.testing.assert_array_equal(k[start[b]:].numpy(), QKV[(N_h + j // 2) * h:(N_h + j // 2 + 1) * h, :count[b], b].T)
            key, query = torch.arange(len(at)), torch.arange(start[b], len(at))[:, None]
            mask = (key <= query) & ((key > query - window) if window else True)
            o = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None], attn_mask=mask[None], scale=0.3)[0]
            np.testing.assert_allclose(B[j * h:(j + 1) * h, :count[b], b].T, o.numpy(), rtol=1e-12, atol=1e-13)
    assert (B[:, 3:, 1] == 7.0).all()


def test_pages_that_are_not_there_are_neither_written_nor_seen():
    r = np.random.default_rng(3)
    QKV, K, V = r.standard_normal((3 * 8, 4, 1)), np.zeros((8, 4, 1)), np.zeros((8, 4, 1))
    pages = np.array([[-1], [1], [2]])               # page 2 is beyond the pool of two pages of two positions
    k, v = R.cache_append(QKV, K, V, 2, 1, pages, np.array([1]))
    assert not k[:, :2].any() and k[:, 2:].any(0).all()
    B, _ = R.cache_attention(QKV, k, v, np.ones((8, 4, 1)), 2, 1, 1.0, pages, np.array([1]))
    assert not B[:, 0].any() and B[:, 1].any()
    np.testing.assert_allclose(B[:, 1, 0], QKV[16:, 1, 0])      # one key only
    k, _ = R.cache_append(QKV, K, V, 2, 1, pages, np.array([-2]))
    assert not k[:, 0:2].any() and not k[:, 2:].any()


def test_drawn_tokens_follow_the_filtered_distribution():
    x = np.log(np.array([0.1, 0.4, 0.05, 0.4, 0.05]))
    n = 2000
    us = (np.arange(n) + 0.5) / n
    shares = lambda **f: np.bincount([R.sample_token(x, u, **f)[0] for u in us], minlength=5) / n
    np.testing.assert_allclose(shares(), [0.1, 0.4, 0.05, 0.4, 0.05], atol=1e-3)
    np.testing.assert_allclose(shares(top_k=1), [0, 1, 0, 0, 0])                    # equal logits: the lower number
    np.testing.assert_allclose(shares(top_k=3), np.array([1, 4, 0, 4, 0]) / 9, atol=1e-3)
    np.testing.assert_allclose(shares(top_p=0.85), np.array([1, 4, 0, 4, 0]) / 9, atol=1e-3)
    np.testing.assert_allclose(shares(top_k=3, top_p=0.4), [0, 1, 0, 0, 0])         # 0.4 of 0.9: the first alone
    np.testing.assert_allclose(shares(min_p=0.2), np.array([1, 4, 0, 4, 0]) / 9, atol=1e-3)
    np.testing.assert_allclose(shares(temperature=0.5), np.array([0.01, 0.16, 0.0025, 0.16, 0.0025]) / 0.335, atol=1e-3)
    assert R.sample_token(x, 0.9, temperature=0.0)[0] == 1
    assert abs(R.sample_token(x, 0.0, top_k=2)[1] - np.log(0.4)) < 1e-14


def test_draws_from_odd_columns():
    assert R.sample_token(np.array([np.nan, -np.inf]), 0.5) == (-1, 0.0)
    t, lp = R.sample_token(np.array([0.0, np.inf, 5.0, np.inf, np.nan]), 0.6, top_p=0.9)
    assert t == 3 and abs(lp + np.log(2)) < 1e-15
    x = np.zeros(4)
    assert [R.sample_token(x, u)[0] for u in (-1.0, np.nan, 0.25, 0.999, 1.0, 7.0)] == [0, 0, 1, 3, 3, 3]
    assert [R.sample_token(x, u, top_p=0.5)[0] for u in (0.0, 0.499, 0.5, 0.99)] == [0, 0, 1, 1]


def test_clipping():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    o, n = R.clip_grad_norm(g, 1.0, 0.0)
    assert n == 5.0 and np.allclose(o[0], [0.6, 0.0]) and np.allclose(o[1], 0.8)
    t = [torch.tensor(a, requires_grad=True) for a in g]
    for p, a in zip(t, g):
        p.grad = torch.tensor(a)
    torch.nn.utils.clip_grad_norm_(t, 2.0)
    o, _ = R.clip_grad_norm(g, 2.0, 1e-6)
    for p, a in zip(t, o):
        np.testing.assert_allclose(p.grad.numpy(), a, rtol=1e-12)
    o, n = R.clip_grad_norm([np.array([np.inf, 1.0])], 1.0, 0.0)
    assert n == np.inf and o[0][1] == 1.0


def test_calls_without_a_context_or_an_object():
    from paper_2504_13236_amd import capi
    cache, sample, clip = capi.nnt_cache_cfg(), capi.nnt_sample_cfg(1.0, 1.0, 0.0, 0), capi.nnt_clip_cfg(1.0, 0.0)
    bad = capi.NNT_EINVAL
    assert capi.nnt_cache_append.raw(None, C.byref(cache), None, None, None) == bad
    assert capi.nnt_cache_attention.raw(None, C.byref(cache), 1.0, None, None, None, None) == bad
    assert capi.nnt_sample_tokens.raw(None, C.byref(sample), None, None, 1, None, None, None) == bad
    assert capi.nnt_clip_grad_norm.raw(None, C.byref(clip), 1, None, None, None) == bad
    assert capi.nnt_gpt2_block_clip.raw(None, C.byref(clip), None) == bad
    assert capi.nnt_gpt2_stack_clip.raw(None, C.byref(clip), None) == bad
    assert capi.nnt_gpt2_model_clip.raw(None, C.byref(clip), None) == bad
    assert capi.nnt_gpt2_block_forward_cached.raw(None, C.byref(cache), None, None, None, None) == bad
    assert capi.nnt_gpt2_stack_forward_cached.raw(None, C.byref(cache), None, None) == bad
    assert capi.nnt_gpt2_model_sample.raw(None, None, None, C.byref(cache), None, None, C.byref(sample), None, 1, None, None, None) == bad


def test_lists_of_different_lengths_never_reach_the_library():
    from paper_2504_13236_amd import tiled
    with pytest.raises(ValueError):
        tiled.clip_grad_norm(None, [1, 2], None, O=[1])
    with pytest.raises(ValueError):
        tiled.sample_tokens(None, None, torch.zeros(3), torch.zeros(2, dtype=torch.int32))
