"""The losses on given tokens entry by entry: every gradient entry within its own rounding, over the instances that many columns, large gradients and odd
addresses take, and labels that are themselves banned."""
import numpy as np
import pytest
import torch

from gpu_util import quant
from oracle import definition as D
from test_gpu_token_losses import HALF, LOGP, REL, Call, has_label, labels_for, logits_for

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
