"""The operators of post-training and of matrix-wise optimisation, as cases that can be timed and compared: what a
program calls around the language model's logits (log-probabilities of given tokens, the clipped policy loss with its KL
term, the preference loss of answer pairs, each with the gradient of the logits) and for the update of its weight matrices
(orthogonalisation by Newton-Schulz products, the Muon step made of it).

With `own` false `run` computes them in plain form, elementary torch operations in 32 bits; with `own` true it calls the
framework's entry points.  Arrays have their axes reversed against the framework's tensors (first axis of a tiled tensor
last): logits [N_v, N_s, N_b] are (N_b, N_s, N_v), a matrix of `rows` x `cols` is (cols, rows).  Outputs that the framework
keeps in tiles are returned tile by tile, first axis fastest.
"""
from __future__ import annotations

import itertools
import math

import torch

own = False

#: the policy loss's clip range and weight of the KL term, the preference loss's strength, as commonly set
POLICY = dict(clip_low=0.2, clip_high=0.2, kl_coef=0.04)
PREFERENCE = dict(beta=0.1, label_smoothing=0.05)
#: the quintic iteration's coefficients, five steps
NEWTON_SCHULZ = dict(a=3.4445, b=-4.7750, c=2.0315, eps=1e-7, steps=5)
MUON = dict(lr=0.02, momentum=0.95, weight_decay=0.01)


# ------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the score of one sampled token, as a sampler asks for it: the smallest call, one column of GPT-2's padded vocabulary
        _logits("logprob_token_f32", "logprob", "f32", 50304, 1, 1, 8192, 1),
        # the old or reference policy's log-probabilities of a whole batch of answers
        _logits("logprob_batch_bf16", "logprob", "bf16", 50304, 1024, 8, 8192, 512),
        # a policy step of a small model with an odd vocabulary on short odd answers, ragged tiles everywhere
        _logits("policy_odd_f32", "policy", "f32", 6513, 37, 3, 1500, 16, reduction="sum"),
        # a policy step on a batch of answers, logits and gradients in bf16: bound by memory
        _logits("policy_batch_bf16", "policy", "bf16", 50304, 1024, 8, 8192, 512, reduction="tokens"),
        # the same with a long vocabulary in fp32: columns of 400 KB, more than a workgroup's registers hold
        _logits("policy_long_vocabulary_f32", "policy", "f32", 100003, 256, 2, 16384, 256, reduction="sequences"),
        # three pairs of odd length in fp32
        _logits("preference_ragged_f32", "preference", "f32", 32003, 333, 6, 8192, 128),
        # two pairs of full-length answers in bf16
        _logits("preference_batch_bf16", "preference", "bf16", 50304, 1024, 4, 8192, 512),
        # the update of one adapter matrix of odd sizes
        dict(name="orthogonalize_odd_f32", kind="orthogonalize", dtype="f32", matrices="777x1111", tile=300),
        # a bf16 gradient of a GPT-2-medium block's first MLP matrix, the result in bf16
        dict(name="orthogonalize_tall_bf16", kind="orthogonalize", dtype="bf16", matrices="4096x1024", tile=512),
        # the four matrices of the smallest block: next to no work, latency counts
        dict(name="muon_block_tiny_f32", kind="muon", dtype="f32", matrices="192x64 64x64 256x64 64x256", tile=64),
        # the output projections of GPT-2 small's twelve blocks in one call
        dict(name="muon_projections_f32", kind="muon", dtype="f32", matrices=" ".join(["768x768"] * 12), tile=768),
        # the output projection of a 50B-class block with its bf16 copy: the largest products
        dict(name="muon_wide_bf16", kind="muon", dtype="bf16", matrices="8192x8192", tile=4096),
    ]


def _logits(name, kind, dtype, N_v, N_s, N_b, tile_v, tile_s, **more):
    return dict(name=name, kind=kind, dtype=dtype, N_v=N_v, N_s=N_s, N_b=N_b, tile_v=tile_v, tile_s=tile_s, **more)


def _shapes(c):
    """(rows, columns) of a case's matrices."""
    return [tuple(int(n) for n in m.split("x")) for m in c["matrices"].split()]


#: the dearest listed cases: no drawn one costs more
MOST_LOGITS_BYTES = 2 * 2 * 50304 * 1024 * 8
MOST_MATRIX_FLOPS = 5 * 4 * 1.0 * 8192 ** 3
MOST_OUTPUTS = 60


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= MOST_LOGITS_BYTES and w["flops"] <= MOST_MATRIX_FLOPS and _outputs(c) <= MOST_OUTPUTS:
            return c


def _outputs(c):
    """How many arrays a pass hands back, tile by tile."""
    if c["kind"] in ("orthogonalize", "muon"):
        per = 1 if c["kind"] == "orthogonalize" else 3 if c["dtype"] == "bf16" else 2
        return per * sum(len(_cuts(m, (c["tile"], c["tile"]))) for m in _shapes(c))
    of_logp = len(_cuts((c["N_s"], c["N_b"]), _act_base(c)[1:]))
    return of_logp if c["kind"] == "logprob" else of_logp * (1 + -(-c["N_v"] // c["tile_v"])) + 3


def _log(rng, lo, hi):
    """An integer between lo and hi, spread evenly over its logarithm: round sizes and odd ones alike."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice((1, 1, 8, 64))
    return max(lo, min(hi, (n + step // 2) // step * step))


def _draw(rng):
    kind, dtype = rng.choice(("logprob", "policy", "policy", "preference", "preference", "orthogonalize", "muon", "muon")), rng.choice(("f32", "bf16"))
    if kind in ("orthogonalize", "muon"):
        count = rng.choice((1, 1, 2, 4, 12))
        shapes = [(_log(rng, 32, 8192), _log(rng, 32, 8192))] * count
        if rng.random() < 0.3:                                     # the matrices of a block
            e = _log(rng, 32, 2048)
            shapes = [(3 * e, e), (e, e), (4 * e, e), (e, 4 * e)]
        return dict(kind=kind, dtype=dtype, matrices=" ".join("%dx%d" % m for m in shapes), tile=rng.choice((128, 256, 300, 400, 512, 1024, 2048, 4096)))
    c = dict(kind=kind, dtype=dtype, N_v=_log(rng, 256, 131072), N_s=_log(rng, 1, 2048), N_b=rng.randint(1, 8),
             tile_v=rng.choice((1024, 1500, 4096, 8192, 16384, 131072)), tile_s=rng.choice((64, 128, 300, 512, 2048)))
    if kind == "preference":
        c["N_b"] = 2 * rng.randint(1, 4)
    if kind == "policy":
        c["reduction"] = rng.choice(("sum", "tokens", "sequences"))
    return c


# ------------------------------------------------------------------------------------------------- inputs
class _Inputs:
    """The inputs of a case, drawn one after the other from the seed: the same for prepare() and exact()."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) + 250413236)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape, std=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float32)

    def ints(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _inputs(c, seed):
    i = _Inputs(seed, c["dtype"])
    d = {}
    if c["kind"] in ("orthogonalize", "muon"):
        # gradients as a few tokens make them: a falling spectrum of rank 64 over a floor of noise
        G, P, M = [], [], []
        for rows, cols in _shapes(c):
            r = min(64, rows, cols)
            fall = torch.arange(1, r + 1, device="cuda", dtype=torch.float32).rsqrt()

            def gradient():
                return ((i.normal(cols, r) * fall) @ i.normal(r, rows)).add_(i.normal(cols, rows, std=0.3)).mul_(1e-3)
            G.append(gradient().to(i.dtype) if c["kind"] == "orthogonalize" else gradient())
            if c["kind"] == "muon":
                P.append(i.normal(cols, rows, std=0.02))
                M.append(gradient().mul_(5.0))
        d.update(G=G, P=P, M=M)
        return d
    V, S, B = c["N_v"], c["N_s"], c["N_b"]
    X = torch.empty(B, S, V, device="cuda", dtype=i.dtype)
    labels = i.ints(V, B, S)
    for b in range(B):
        x = i.normal(S, V, std=2.0)
        # the model finds many of its own tokens likely
        x.scatter_add_(1, labels[b].long().unsqueeze(1), i.uniform(S, 1) * 12.0)
        X[b] = x
    at = torch.arange(S, device="cuda")
    if S >= 8:
        # the prompt in front and the padding behind carry no loss
        lead, tail = i.ints(S // 2, B, 1), i.ints(S // 4 + 1, B, 1)
        labels = torch.where((at >= lead) & (at < S - tail), labels, torch.full_like(labels, -1))
        if B >= 3 and c["kind"] == "policy":
            labels[B - 1] = -1                     # an answer that was cut away altogether
    d.update(X=X, labels=labels)
    if c["kind"] == "logprob":
        return d
    logp = torch.stack([_logprob(x.float() if x.dtype != torch.float32 else x.clone(), lab)[0] for x, lab in zip(X, labels)]).float()
    d["ref"] = logp + i.normal(B, S, std=0.3)
    if c["kind"] == "policy":
        d["old"] = logp + i.normal(B, S, std=0.15)
        d["adv"] = i.normal(B).unsqueeze(1).expand(B, S).contiguous()
    return d


# ------------------------------------------------------------------------------------------------- the program's state
class _State:
    def __init__(self, case):
        self.case, self.tensors, self.ctx, self.out = case, [], None, None

    def tensor(self, dtype, shape, base, a=None):
        """A tiled tensor (axes in the framework's order), filled with `a` (axes reversed)."""
        from paper_2504_13236_amd import tiled
        t = tiled.TiledTensor(self.ctx, dtype, shape, base)
        self.tensors.append(t)
        if a is None:
            t.buf.zero_()
        else:
            for k, cut in enumerate(_cuts(shape, base)):
                t.tile_view(k).copy_(a[cut].reshape(-1))
        return t

    def __del__(self):
        try:
            for t in self.tensors:
                t.close()
        except Exception:       # the interpreter is ending
            pass


_ctx = None


def _context():
    global _ctx
    if _ctx is None:
        from paper_2504_13236_amd import tiled
        _ctx = tiled.Context(n_streams=2)
    return _ctx


def _cuts(shape, base):
    """Slices of the reversed array, one per tile, first axis of the framework's tensor fastest."""
    grid = [-(-n // min(b, n)) for n, b in zip(shape, base)]
    return [tuple(slice(k * min(b, n), min(n, (k + 1) * min(b, n))) for k, b, n in zip(idx, reversed(base), reversed(shape)))
            for idx in itertools.product(*[range(g) for g in reversed(grid)])]


def _tiles(name, a, base):
    """The tiles of a dense array as the framework's tensor holds them (views)."""
    shape = tuple(reversed(a.shape))
    return {"%s_%d" % (name, k): a[cut] for k, cut in enumerate(_cuts(shape, base))}


def _own_tiles(name, t):
    return {"%s_%d" % (name, k): t.tile_view(k).view(*reversed(t.tile_shape(idx))) for k, idx in enumerate(t.tile_index)}


def _act_base(c):
    return (c["tile_v"], c["tile_s"], c["N_b"])


def prepare(case, seed):
    c, d = case, _inputs(case, seed)
    s = _State(case)
    if not own:
        s.d = d
        if c["kind"] == "muon":
            d["LP"] = [p.bfloat16() for p in d["P"]] if c["dtype"] == "bf16" else []
        torch.cuda.synchronize()
        return s
    from paper_2504_13236_amd import capi
    s.ctx = _context()
    s.out = {}
    kind, dt = c["kind"], c["dtype"]
    if kind in ("orthogonalize", "muon"):
        t = c["tile"]
        mats = dict(G=[], P=[], M=[], LP=[], O=[])
        for n, (rows, cols) in enumerate(_shapes(c)):
            def mat(name, dtype, a=None):
                x = s.tensor(dtype, (rows, cols), (t, t), a)
                mats[name].append(x)
                if name != "G":
                    s.out.update(_own_tiles("%s%d" % (name, n), x))
            if kind == "orthogonalize":
                mat("G", dt, d["G"][n])
                mat("O", dt)
            else:
                mat("G", "f32", d["G"][n])
                mat("P", "f32", d["P"][n])
                mat("M", "f32", d["M"][n])
                if dt == "bf16":
                    mat("LP", "bf16", d["P"][n])
        s.mats = {k: capi.ptr_array([x.h.value for x in v]) if v else None for k, v in mats.items()}
        ns = capi.nnt_newton_schulz_cfg(NEWTON_SCHULZ["a"], NEWTON_SCHULZ["b"], NEWTON_SCHULZ["c"], NEWTON_SCHULZ["eps"], NEWTON_SCHULZ["steps"])
        s.cfg = ns if kind == "orthogonalize" else capi.nnt_muon_cfg(MUON["lr"], MUON["momentum"], MUON["weight_decay"], 1, capi.NNT_MUON_SCALE_RMS, ns)
    else:
        V, S, B = c["N_v"], c["N_s"], c["N_b"]
        base = _act_base(c)
        s.X, s.labels = s.tensor(dt, (V, S, B), base, d["X"]), d["labels"]
        s.logp = s.tensor("f32", (S, B), base[1:])
        s.out.update(_own_tiles("logp", s.logp))
        if kind != "logprob":
            s.dX = s.tensor(dt, (V, S, B), base)
            s.ref = s.tensor("f32", (S, B), base[1:], d["ref"])
            s.losses = torch.zeros(B // 2 if kind == "preference" else B * S, device="cuda")
            s.loss = torch.zeros(1, device="cuda")
            s.out.update(_own_tiles("dX", s.dX), losses=s.losses, loss=s.loss)
        if kind == "policy":
            s.old, s.adv = s.tensor("f32", (S, B), base[1:], d["old"]), s.tensor("f32", (S, B), base[1:], d["adv"])
            reduction = dict(sum=capi.NNT_REDUCE_SUM, tokens=capi.NNT_REDUCE_TOKENS, sequences=capi.NNT_REDUCE_SEQUENCES)[c["reduction"]]
            s.cfg = capi.nnt_policy_cfg(POLICY["clip_low"], POLICY["clip_high"], POLICY["kl_coef"], reduction)
        if kind == "preference":
            s.rewards = torch.zeros(B, device="cuda")
            s.out["rewards"] = s.rewards
            s.cfg = capi.nnt_preference_cfg(PREFERENCE["beta"], PREFERENCE["label_smoothing"], capi.NNT_REDUCE_SEQUENCES)
    torch.cuda.synchronize()
    s.ctx.wait()
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import ctypes

    from paper_2504_13236_amd import capi
    c, h, kind = s.case, s.ctx.h, s.case["kind"]
    if kind == "logprob":
        capi.nnt_token_logprob(h, s.X.h, s.labels.data_ptr(), s.logp.h)
    elif kind == "policy":
        capi.nnt_policy_loss(h, ctypes.byref(s.cfg), s.X.h, s.labels.data_ptr(), s.old.h, s.ref.h, s.adv.h, s.dX.h, s.logp.h,
                             s.losses.data_ptr(), s.loss.data_ptr())
    elif kind == "preference":
        capi.nnt_preference_loss(h, ctypes.byref(s.cfg), s.X.h, s.labels.data_ptr(), s.ref.h, s.dX.h, s.logp.h,
                                 s.rewards.data_ptr(), s.losses.data_ptr(), s.loss.data_ptr())
    elif kind == "orthogonalize":
        capi.nnt_orthogonalize(h, ctypes.byref(s.cfg), len(_shapes(c)), s.mats["G"], s.mats["O"])
    else:
        capi.nnt_muon_step(h, ctypes.byref(s.cfg), len(_shapes(c)), s.mats["G"], s.mats["P"], s.mats["M"], s.mats["LP"])
    return s.out


def _logprob(x, labels):
    """Log-probabilities of the labels (0 where there is none), and what the gradient needs: e^(x - max) in place of x, its sum.
    The logarithm and the differences are taken in 64 bits: a reward is a sum of many of them in which the large parts cancel."""
    at, has = labels.long().clamp_min(0).unsqueeze(-1), labels >= 0
    top = x.amax(-1, keepdim=True)
    x_label = x.gather(-1, at)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    logp = (x_label.double() - top.double() - total.double().log())[..., 0]
    return torch.where(has, logp, torch.zeros_like(logp)), e, total


def _logits_gradient(e, total, labels, g, dtype):
    """g (onehot - softmax), with g = dL/dlogp of each position (0 where there is no label)."""
    g = g.float()
    e.mul_(-g.unsqueeze(-1) / total)
    e.scatter_add_(-1, labels.long().clamp_min(0).unsqueeze(-1), g.unsqueeze(-1))
    return e.to(dtype)


def _weights(labels, reduction):
    has = (labels >= 0).double()
    if reduction == "tokens":
        return has / has.sum().clamp_min(1.0)
    if reduction == "sequences":
        n = has.sum(-1, keepdim=True)
        return has / n.clamp_min(1.0) / (n > 0).double().sum().clamp_min(1.0)
    return has


def _orthogonalize(U):
    """Newton-Schulz iteration on a (cols, rows) array, transposed or not the same up to a transposition."""
    n = NEWTON_SCHULZ
    flip = U.shape[0] > U.shape[1]
    X = U.t() if flip else U
    X = X / ((X * X).sum().sqrt() + n["eps"])
    for _ in range(n["steps"]):
        A = X @ X.t()
        X = n["a"] * X + (n["b"] * A + n["c"] * (A @ A)) @ X
    return X.t() if flip else X


def _run_plain(s):
    c, d, kind = s.case, s.d, s.case["kind"]
    if kind == "orthogonalize":
        out = {}
        for n, G in enumerate(d["G"]):
            out.update(_tiles("O%d" % n, _orthogonalize(G.float()).to(G.dtype), (c["tile"], c["tile"])))
        return out
    if kind == "muon":
        out, base = {}, (c["tile"], c["tile"])
        for n, (G, P, M) in enumerate(zip(d["G"], d["P"], d["M"])):
            M.mul_(MUON["momentum"]).add_(G)
            O = _orthogonalize(G + MUON["momentum"] * M)
            P.mul_(1.0 - MUON["lr"] * MUON["weight_decay"]).sub_(O, alpha=MUON["lr"] * 0.2 * math.sqrt(max(G.shape)))
            out.update(_tiles("P%d" % n, P, base), **_tiles("M%d" % n, M, base))
            if d["LP"]:
                d["LP"][n].copy_(P)
                out.update(_tiles("LP%d" % n, d["LP"][n], base))
        return out
    X, labels, base = d["X"], d["labels"], _act_base(c)
    logp, e, total = _logprob(X.float() if X.dtype != torch.float32 else X.clone(), labels)
    out = _tiles("logp", logp.float(), base[1:])
    if kind == "logprob":
        return out
    has = labels >= 0
    zero = torch.zeros_like(logp)
    if kind == "policy":
        w = _weights(labels, c["reduction"])
        r = torch.where(has, (logp - d["old"]).exp(), zero)
        adv = torch.where(has, d["adv"], zero)
        free, held = r * adv, r.clamp(1.0 - POLICY["clip_low"], 1.0 + POLICY["clip_high"]) * adv
        k = torch.where(has, d["ref"] - logp, zero)
        losses = w * (-torch.minimum(free, held) + POLICY["kl_coef"] * (k.exp() - k - 1.0))
        g = w * (torch.where(free <= held, -free, zero) + POLICY["kl_coef"] * (1.0 - k.exp()))
        out.update(losses=losses.float().reshape(-1), loss=losses.sum().float().reshape(1))
    else:
        p, beta, soft = c["N_b"] // 2, PREFERENCE["beta"], PREFERENCE["label_smoothing"]
        rewards = beta * torch.where(has, logp - d["ref"], zero).sum(-1)
        z = rewards[:p] - rewards[p:]
        losses = (1.0 - soft) * torch.nn.functional.softplus(-z) + soft * torch.nn.functional.softplus(z)
        slope = (torch.sigmoid(z) - (1.0 - soft)) * beta / p
        g = torch.cat([slope, -slope]).unsqueeze(-1) * has
        losses = losses / p
        out.update(rewards=rewards.float(), losses=losses.float(), loss=losses.sum().float().reshape(1))
    out.update(_tiles("dX", _logits_gradient(e, total, labels, g, X.dtype), base))
    return out


# ------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    w = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] in ("orthogonalize", "muon"):
        flops = byts = 0.0
        for rows, cols in _shapes(c):
            m, n = min(rows, cols), max(rows, cols)
            # X X^T and A^2 are symmetric: half of each; then B X
            flops += NEWTON_SCHULZ["steps"] * (1.0 * m * m * n + 1.0 * m ** 3 + 2.0 * m * m * n)
            # gradient in, result out; or gradient, weights and momentum in, weights, momentum (and the bf16 copy) out
            byts += rows * cols * (2 * w if c["kind"] == "orthogonalize" else 20 + (2 if w == 2 else 0))
        return dict(flops=flops, bytes=byts)
    n, T = c["N_v"] * c["N_s"] * c["N_b"], c["N_s"] * c["N_b"]
    if c["kind"] == "logprob":
        return dict(flops=4.0 * n, bytes=n * w + 8 * T)
    return dict(flops=8.0 * n, bytes=2 * n * w + (24 if c["kind"] == "policy" else 16) * T)


# ------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    """From the definitions, one sequence or matrix at a time."""
    c, d = case, _inputs(case, seed)
    out = {}
    if c["kind"] in ("orthogonalize", "muon"):
        base = (c["tile"], c["tile"])
        n = NEWTON_SCHULZ
        for k, (rows, cols) in enumerate(_shapes(c)):
            G = d["G"][k].double()
            if c["kind"] == "muon":
                M = MUON["momentum"] * d["M"][k].double() + G
                U = G + MUON["momentum"] * M
            else:
                U = G
            W = U.t() if rows <= cols else U                        # rows x cols with the short side first, or its transpose
            W = W / (torch.linalg.vector_norm(W) + n["eps"])
            eye = torch.eye(W.shape[0], dtype=torch.float64, device=W.device)
            for _ in range(n["steps"]):
                A = torch.mm(W, W.t())
                W = torch.mm(n["a"] * eye + n["b"] * A + n["c"] * torch.mm(A, A), W)
            O = W.t() if rows <= cols else W
            if c["kind"] == "orthogonalize":
                out.update(_tiles("O%d" % k, O, base))
            else:
                P = (1.0 - MUON["lr"] * MUON["weight_decay"]) * d["P"][k].double() - MUON["lr"] * 0.2 * math.sqrt(max(rows, cols)) * O
                out.update(_tiles("P%d" % k, P, base), **_tiles("M%d" % k, M, base))
                if c["dtype"] == "bf16":
                    out.update(_tiles("LP%d" % k, P, base))
        return out
    B, S, V = d["X"].shape
    labels, dev = d["labels"].long(), d["X"].device
    has = labels >= 0
    logp = torch.zeros(B, S, dtype=torch.float64, device=dev)
    for b in range(B):
        lp = torch.log_softmax(d["X"][b].double(), -1)
        rows = has[b].nonzero()[:, 0]
        logp[b, rows] = lp[rows, labels[b, rows]]
    base = _act_base(c)
    out.update(_tiles("logp", logp, base[1:]))
    if c["kind"] == "logprob":
        return out
    # losses as functions of the log-probabilities, differentiated by torch
    lp = logp.clone().requires_grad_(True)
    if c["kind"] == "policy":
        counts = has.sum(-1)
        if c["reduction"] == "tokens":
            w = has.double() / max(int(counts.sum()), 1)
        elif c["reduction"] == "sequences":
            w = has.double() / counts.clamp_min(1).unsqueeze(1) / max(int((counts > 0).sum()), 1)
        else:
            w = has.double()
        old, ref, adv = (torch.where(has, d[k].double(), torch.zeros_like(logp)) for k in ("old", "ref", "adv"))
        ratio = torch.exp(lp - old)
        inside = torch.where(adv >= 0, ratio <= 1.0 + POLICY["clip_high"], ratio >= 1.0 - POLICY["clip_low"])
        border = torch.where(adv >= 0, torch.full_like(adv, 1.0 + POLICY["clip_high"]), torch.full_like(adv, 1.0 - POLICY["clip_low"]))
        gain = adv * torch.where(inside, ratio, border)
        losses = w * (-gain + POLICY["kl_coef"] * (torch.exp(ref - lp) - (ref - lp) - 1.0))
    else:
        p, beta, soft = B // 2, PREFERENCE["beta"], PREFERENCE["label_smoothing"]
        rewards = beta * (torch.where(has, lp - d["ref"].double(), torch.zeros_like(logp))).sum(-1)
        z = rewards[:p] - rewards[p:]
        losses = -((1.0 - soft) * torch.nn.functional.logsigmoid(z) + soft * torch.nn.functional.logsigmoid(-z)) / p
        out["rewards"] = rewards.detach()
    losses.sum().backward()
    g = torch.where(has, lp.grad, torch.zeros_like(logp))
    out.update(losses=losses.detach().reshape(-1), loss=losses.detach().sum().reshape(1))
    dX = torch.empty(B, S, V, dtype=torch.float64, device=dev)
    for b in range(B):
        dX[b] = torch.softmax(d["X"][b].double(), -1) * -g[b].unsqueeze(-1)
        rows = has[b].nonzero()[:, 0]
        dX[b, rows, labels[b, rows]] += g[b, rows]
    out.update(_tiles("dX", dX, base))
    return out
