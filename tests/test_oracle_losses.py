"""Pins of the oracle's losses on given tokens and of its matrix-wise optimiser that do not go through the oracle: CPU torch in float64 with
autograd, closed forms, singular values and finite differences."""
import math

import numpy as np
import pytest
import torch

from oracle import definition as D


def problem(seed, N_v=11, N_s=5, N_b=4):
    r = np.random.default_rng(seed)
    X = 2.0 * r.standard_normal((N_v, N_s, N_b))
    lab = r.integers(0, N_v, (N_s, N_b))
    lab[0, 0], lab[3, 1], lab[:, 2] = -1, N_v, -7
    base = D.token_logprob(X, lab)
    return X, lab, base + 0.3 * r.standard_normal(lab.shape), base + 0.3 * r.standard_normal(lab.shape), r.standard_normal(lab.shape)


def torch_logp(X, lab):
    tx = torch.from_numpy(X).requires_grad_(True)
    has = torch.from_numpy((lab >= 0) & (lab < X.shape[0]))
    at = torch.from_numpy(np.where(has.numpy(), lab, 0).astype(np.int64)).unsqueeze(0)
    return tx, has, torch.where(has, torch.log_softmax(tx, 0).gather(0, at)[0], torch.zeros((), dtype=torch.float64))


def test_token_logprob():
    X, lab, *_ = problem(1)
    _, _, lp = torch_logp(X, lab)
    np.testing.assert_allclose(D.token_logprob(X, lab), lp.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(D.token_logprob(np.zeros((7, 2, 1)), np.zeros((2, 1), int)), -math.log(7), rtol=1e-14)
    np.testing.assert_allclose(D.token_logprob(X + 50.0, lab), D.token_logprob(X, lab), atol=1e-12)


@pytest.mark.parametrize("reduction", ["sum", "tokens", "sequences"])
@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_loss_against_autograd(reduction, kl):
    X, lab, old, ref, adv = problem(2)
    tx, has, lp = torch_logp(X, lab)
    r = torch.where(has, (lp - torch.from_numpy(old)).exp(), torch.ones((), dtype=torch.float64))
    A = torch.from_numpy(adv)
    l = -torch.min(r * A, torch.clamp(r, 0.9, 1.15) * A)
    k = torch.where(has, torch.from_numpy(ref) - lp, torch.zeros((), dtype=torch.float64))
    l = torch.where(has, l + kl * (k.exp() - k - 1), torch.zeros((), dtype=torch.float64))
    if reduction == "tokens":
        l = l / 13                                    # 20 positions, 1 + 1 + 5 of them without a label
    elif reduction == "sequences":
        l = l / torch.tensor([4.0, 4.0, 1.0, 5.0], dtype=torch.float64) / 3
    l.sum().backward()
    L, losses, logp, dX = D.policy_loss(X, lab, old, ref, adv, 0.1, 0.15, kl, reduction)
    np.testing.assert_allclose(losses, l.detach().numpy(), rtol=1e-11, atol=1e-13)
    np.testing.assert_allclose(L, l.sum().item(), rtol=1e-11)
    # (inside the clip range torch shares the gradient among the two equal terms, which adds up to the same)
    np.testing.assert_allclose(dX, tx.grad.numpy(), rtol=1e-9, atol=1e-13)
    assert not dX[:, 0, 0].any() and not dX[:, :, 2].any() and losses[3, 1] == 0


def test_policy_loss_clips_one_side_only_and_broadcasts():
    X, lab, old, _, _ = problem(3)
    lp = D.token_logprob(X, lab)
    # a ratio of 2 with a positive advantage earns no more than 1 + clip, a ratio of 1/2 all of its loss; the other way round for a negative one
    for ratio, A, want, moves in ((2.0, 1.0, -1.2, False), (0.5, 1.0, -0.5, True), (2.0, -1.0, 2.0, True), (0.5, -1.0, 0.8, False)):
        _, losses, _, dX = D.policy_loss(X, lab, lp - math.log(ratio), None, np.full(4, A), 0.2, 0.2)
        has = (lab >= 0) & (lab < X.shape[0])
        np.testing.assert_allclose(losses[has], want, rtol=1e-12)
        assert bool(np.abs(dX).max() > 1e-3) == moves
    _, a, _, da = D.policy_loss(X, lab, None, None, np.arange(4.0))
    _, b, _, db = D.policy_loss(X, lab, lp, None, np.tile(np.arange(4.0), (5, 1)))
    np.testing.assert_allclose(a, b, atol=1e-14)
    np.testing.assert_allclose(da, db, atol=1e-14)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("soft", [0.0, 0.1])
def test_preference_loss_against_autograd_and_differences(mean, soft):
    X, lab, _, ref, _ = problem(4)
    tx, has, lp = torch_logp(X, lab)
    R = 0.5 * torch.where(has, lp - torch.from_numpy(ref), torch.zeros((), dtype=torch.float64)).sum(0)
    z = R[:2] - R[2:]
    l = -((1 - soft) * torch.nn.functional.logsigmoid(z) + soft * torch.nn.functional.logsigmoid(-z))
    if mean:
        l = l / 2
    l.sum().backward()
    L, losses, rewards, _, dX = D.preference_loss(X, lab, ref, 0.5, soft, mean)
    np.testing.assert_allclose(losses, l.detach().numpy(), rtol=1e-12)
    np.testing.assert_allclose(rewards, R.detach().numpy(), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(dX, tx.grad.numpy(), rtol=1e-9, atol=1e-14)
    for at in ((3, 1, 0), (5, 2, 3), (0, 0, 2)):
        P, M = X.copy(), X.copy()
        P[at] += 1e-6
        M[at] -= 1e-6
        fd = (D.preference_loss(P, lab, ref, 0.5, soft, mean)[0] - D.preference_loss(M, lab, ref, 0.5, soft, mean)[0]) / 2e-6
        assert abs(fd - dX[at]) < 1e-8


# ------------------------------------------------------------------ Newton-Schulz iteration
@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (7, 7), (5, 12), (12, 5)])
def test_orthogonalize_acts_on_singular_values_only(shape):
    """O = U f(S) V^T with the scalar iteration f, whatever the shape; O(G^T) = O(G)^T; scaling of G does not matter."""
    r = np.random.default_rng(5)
    G = r.standard_normal(shape)
    U, S, Vt = np.linalg.svd(G, full_matrices=False)
    s = S / (np.linalg.norm(S) + 1e-7)
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    O = D.orthogonalize(G)
    np.testing.assert_allclose(O, (U * s) @ Vt, atol=1e-10)
    np.testing.assert_allclose(D.orthogonalize(G.T), O.T, atol=1e-10)
    np.testing.assert_allclose(D.orthogonalize(100.0 * G), O, atol=1e-6)
    assert not D.orthogonalize(np.zeros(shape)).any()


def test_orthogonalize_cubic_iteration_reaches_the_polar_factor():
    G = np.random.default_rng(6).standard_normal((6, 9))
    U, _, Vt = np.linalg.svd(G, full_matrices=False)
    np.testing.assert_allclose(D.orthogonalize(G, 1.5, -0.5, 0.0, 1e-12, 40), U @ Vt, atol=1e-10)


def test_muon_step_by_hand():
    r = np.random.default_rng(7)
    p, g, m = (r.standard_normal((8, 3)) for _ in range(3))
    q, n = D.muon_step(p, g, m, 0.1, 0.9, 0.01, True, "aspect")
    np.testing.assert_allclose(n, 0.9 * m + g)
    np.testing.assert_allclose(q, 0.999 * p - 0.1 * math.sqrt(8 / 3) * D.orthogonalize(g + 0.9 * n), atol=1e-14)
    q, _ = D.muon_step(p, g, m, 0.1, 0.9, 0.0, False, "rms")
    np.testing.assert_allclose(q, p - 0.1 * 0.2 * math.sqrt(8) * D.orthogonalize(n), atol=1e-14)
    q, _ = D.muon_step(p.T, g.T, m.T, 0.1, 0.0, 0.0, False, "aspect")
    np.testing.assert_allclose(q, (p - 0.1 * D.orthogonalize(g)).T, atol=1e-14)
