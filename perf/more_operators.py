"""The operators around a policy's training step, as cases that can be timed and compared: keys and values written to a paged cache
with their position rotation, the attention of new tokens over that cache, tokens drawn from the logits with the usual filters
(the rollout), and the norm of all gradients with the clipped ones (the update).

With `own` false `run` computes them in plain form, elementary torch operations in 32 bits; with `own` true it calls the
framework's entry points.  Arrays have their axes reversed against the framework's tensors (first axis of a tiled tensor
last): projections [R, N_s, N_b] are (N_b, N_s, R), a cache [h, pages * page, N_kv] tiled (h, page, N_kv) is (pages, N_kv, page, h).
Outputs that the framework keeps in tiles are returned tile by tile, first axis fastest.
"""
from __future__ import annotations

import itertools
import math

import torch

own = False

CLIP = dict(max_norm=1.0, eps=1e-6)
ROTATION_BASE = 10000.0


# ------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one new token of each of 16 sequences of GPT-2 small's heads: the smallest write, latency counts
        _cache("append_token_bf16", "append", "bf16", N_h=12, N_kv=12, h=64, N_s=1, N_b=16, context=1024, page=16),
        # eight prompts of different lengths, keys rotated, in fp32: bound by memory
        _cache("append_prompts_f32", "append", "f32", N_h=12, N_kv=12, h=64, N_s=1024, N_b=8, context=0, page=64, rotation="halves"),
        # one token of one short sequence: the smallest attention, latency counts
        _cache("attend_token_f32", "attend", "f32", N_h=12, N_kv=12, h=64, N_s=1, N_b=1, context=100, page=16),
        # a batch of answers in the middle of generation: one token each, ragged contexts of up to 4096
        _cache("attend_batch_bf16", "attend", "bf16", N_h=12, N_kv=12, h=64, N_s=1, N_b=64, context=4096, page=64),
        # one sequence of 131072 tokens, four query heads to a cached one, rotated queries: few rows, a long axis
        _cache("attend_long_bf16", "attend", "bf16", N_h=32, N_kv=8, h=128, N_s=1, N_b=1, context=131071, page=256, rotation="halves"),
        # a prompt that comes in parts: 200 new tokens of each of four sequences on what is cached of them, GPT-2 XL's 25 heads
        _cache("attend_part_bf16", "attend", "bf16", N_h=25, N_kv=25, h=64, N_s=200, N_b=4, context=3000, page=32),
        # a few drafted tokens of seven sequences at once, heads of an odd size in threes, only the last 500 tokens seen
        _cache("attend_window_f32", "attend", "f32", N_h=6, N_kv=2, h=96, N_s=3, N_b=7, context=1777, page=24, rotation="pairs", window=500),
        # the next token of one sequence over GPT-2's padded vocabulary, the smallest draw
        _sample("sample_token_f32", "f32", 50304, 1, top_k=50),
        # the next tokens of a batch of rollouts, the likeliest tokens up to 95 % of the mass
        _sample("sample_batch_bf16", "bf16", 50304, 1024, temperature=0.8, top_p=0.95),
        # an odd vocabulary longer than a workgroup's registers, flat distribution, unlikely tokens cut off
        _sample("sample_long_vocabulary_f32", "f32", 100003, 64, temperature=1.3, min_p=0.02),
        # the twelve gradients of the smallest block
        dict(name="clip_block_tiny_f32", kind="clip", dtype="f32", blocks=1, N_e=64, N_v=0, N_pos=0, tile=64),
        # all gradients of GPT-2 small (148 tensors, 124.5 M parameters), collected over micro-batches
        dict(name="clip_model_f32", kind="clip", dtype="f32", blocks=12, N_e=768, N_v=50304, N_pos=1024, tile=768),
    ]


def _cache(name, kind, dtype, rotation="none", window=0, **more):
    return dict(name=name, kind=kind, dtype=dtype, rotation=rotation, window=window, **more)


def _sample(name, dtype, N_v, N_b, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, tile_v=8192):
    return dict(name=name, kind="sample", dtype=dtype, N_v=N_v, N_b=N_b, tile_v=tile_v, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


#: the dearest listed cases: no drawn one costs more
MOST_CACHE_BYTES = 2 * 2 * 131072 * 8 * 128
MOST_PAIRS = 4 * 25 * 200 * 3200 * 64
MOST_APPENDED = 8 * 1024 * 12 * 64 * 4
MOST_LOGITS_BYTES = 2 * 50304 * 1024
MOST_GRADIENTS = 124.5e6


def _log(rng, lo, hi, steps=(1, 1, 8, 64)):
    """An integer between lo and hi, spread evenly over its logarithm: round sizes and odd ones alike."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice(steps)
    return max(lo, min(hi, (n + step // 2) // step * step))


def draw(rng):
    while True:
        c = _draw(rng)
        if c["kind"] == "clip":
            ok = sum(math.prod(s) for s in _shapes(c)) <= MOST_GRADIENTS
        elif c["kind"] == "sample":
            ok = c["N_v"] * c["N_b"] * (2 if c["dtype"] == "bf16" else 4) <= MOST_LOGITS_BYTES
        else:
            w = 2 if c["dtype"] == "bf16" else 4
            cached = (c["context"] + c["N_s"]) * c["N_b"] * c["N_kv"] * c["h"] * 2 * w
            ok = cached <= MOST_CACHE_BYTES and c["N_s"] * c["N_b"] * c["N_kv"] * c["h"] * w <= MOST_APPENDED
            ok = ok and (c["kind"] == "append" or c["N_s"] * c["N_b"] * c["N_h"] * (c["context"] + c["N_s"]) * c["h"] <= MOST_PAIRS)
        if ok:
            return c


def _draw(rng):
    kind, dtype = rng.choice(("append", "attend", "attend", "attend", "sample", "sample", "clip")), rng.choice(("f32", "bf16"))
    if kind == "clip":
        return dict(kind=kind, dtype=dtype, blocks=rng.choice((1, 1, 2, 6, 12, 24)), N_e=_log(rng, 32, 2048), N_v=rng.choice((0, _log(rng, 256, 50304))),
                    N_pos=_log(rng, 64, 2048), tile=rng.choice((64, 300, 512, 768, 1024, 2048)))
    if kind == "sample":
        return dict(kind=kind, dtype=dtype, N_v=_log(rng, 256, 131072), N_b=_log(rng, 1, 1024), tile_v=rng.choice((1024, 1500, 8192, 16384, 131072)),
                    temperature=rng.choice((0.0, 0.6, 0.8, 1.0, 1.0, 1.3)), top_k=rng.choice((0, 0, 1, 20, 50, 1000)), top_p=rng.choice((1.0, 1.0, 0.5, 0.9, 0.95)),
                    min_p=rng.choice((0.0, 0.0, 0.02, 0.1)))
    N_kv, group, h = rng.choice((1, 2, 4, 8, 12, 25)), rng.choice((1, 1, 1, 2, 4, 8)), rng.choice((32, 64, 64, 80, 96, 128, 128))
    return dict(kind=kind, dtype=dtype, N_h=N_kv * group, N_kv=N_kv, h=h, N_s=rng.choice((1, 1, 1, _log(rng, 2, 16, (1,)), _log(rng, 17, 512))),
                N_b=_log(rng, 1, 128, (1, 1, 8)), context=_log(rng, 1, 131071), page=rng.choice((8, 16, 24, 32, 64, 128, 256)),
                rotation=rng.choice(("none", "halves", "pairs")), window=rng.choice((0, 0, 0, _log(rng, 16, 4096))))


def _shapes(c):
    """The parameters of a model (of its blocks alone where it has no vocabulary), axes as the framework has them."""
    e = c["N_e"]
    block = [(3 * e, e), (e, e), (4 * e, e), (e, 4 * e), (3 * e,), (e,), (4 * e,), (e,), (e,), (e,), (e,), (e,)]
    return block * c["blocks"] + ([(e, c["N_v"]), (e, c["N_pos"]), (e,), (e,)] if c["N_v"] else [])


def _tensor_dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------------------------------------- inputs
class _Inputs:
    """The inputs of a case, drawn one after the other from the seed: the same for prepare() and exact()."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) + 250413236)
        self.dtype = dtype

    def normal(self, *shape, std=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float32)

    def ints(self, lo, hi, *shape):
        """lo <= i < hi"""
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _inputs(c, seed):
    i = _Inputs(seed, _tensor_dtype(c))
    if c["kind"] == "clip":
        G = _flat(c)
        for g in _views(c, G):
            g.copy_(i.normal(g.numel(), std=3e-4 * (1.0 + 2.0 * float(len(g) % 3))))
        return dict(G=G)
    if c["kind"] == "sample":
        V, B = c["N_v"], c["N_b"]
        X = torch.empty(B, V, device="cuda", dtype=i.dtype)
        for b0 in range(0, B, 128):
            n = min(128, B - b0)
            x = i.normal(n, V, std=2.0)
            # a few tokens stand out, by more or less: columns that are almost decided and columns that are not
            at = i.ints(0, V, n, 24).long()
            x.scatter_add_(1, at, i.uniform(n, 24) * i.uniform(n, 1) * 14.0)
            X[b0:b0 + n] = x
        return dict(X=X, u=i.uniform(B))
    N_s, N_b, h, P, N_kv, context = c["N_s"], c["N_b"], c["h"], c["page"], c["N_kv"], c["context"]
    d = dict(Z=i.normal(N_b, N_s, (c["N_h"] + 2 * N_kv) * h).to(i.dtype))
    # contexts of different lengths, the first one whole; new tokens of different number where there are several, one sequence without any
    d["start"] = i.ints(context // 4, context + 1, N_b)
    d["start"][0] = context
    d["count"] = i.ints(1, N_s + 1, N_b)
    d["count"][0] = N_s
    if N_b >= 4 and N_s > 1:
        d["count"][N_b - 1] = 0
    most = -(-(context + N_s) // P)
    per = (d["start"] + d["count"] + (P - 1)) // P
    n_pages = most * N_b + 3
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(int(seed) + 1)).to("cuda", torch.int32)
    first = torch.cumsum(per, 0) - per
    at = torch.arange(most, device="cuda")
    d["pages"] = torch.where(at < per[:, None], free[(first[:, None] + at).clamp_max(n_pages - 1).long()], torch.full((), -1, device="cuda", dtype=torch.int32))
    if c["kind"] == "attend":
        d["K"], d["V"] = (torch.empty(n_pages, N_kv, P, h, device="cuda", dtype=i.dtype) for _ in range(2))
        for pool in (d["K"], d["V"]):
            for k in range(0, n_pages, 256):
                pool[k:k + 256] = i.normal(*pool[k:k + 256].shape)
    else:
        d["K"], d["V"] = (torch.zeros(n_pages, N_kv, P, h, device="cuda", dtype=i.dtype) for _ in range(2))
    if c["rotation"] != "none":
        # cosines, then sines, of position / base^(2 k / h): from angles in 64 bits
        p = torch.arange(context + N_s, device="cuda", dtype=torch.float64)
        angle = p[:, None] * ROTATION_BASE ** (-2.0 / h * torch.arange(h // 2, device="cuda", dtype=torch.float64))
        d["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    return d


def _flat(c):
    """One buffer for all gradients, each tile of each tensor on a boundary of 256 bytes, zeros between them."""
    return torch.zeros(_places(c)[1], device="cuda", dtype=_tensor_dtype(c))


def _places(c):
    """[per tensor: (first element, behind the last one, [offset of each tile])], elements in all"""
    step = 128 if c["dtype"] == "bf16" else 64
    at, out = 0, []
    for shape in _shapes(c):
        offsets, base = [], [min(n, c["tile"]) for n in shape]
        first = at
        for cut in _cuts(shape, base):
            offsets.append(at)
            n = math.prod(s.stop - s.start for s in cut)
            end = at + n
            at += -(-n // step) * step
        out.append((first, end, offsets))
    return out, at


def _views(c, flat):
    """What of the buffer belongs to each tensor (with the gaps between its tiles)."""
    return [flat[first:end] for first, end, _ in _places(c)[0]]


# ------------------------------------------------------------------------------------------------- the program's state
class _State:
    def __init__(self, case):
        self.case, self.tensors, self.handles = case, [], []

    def tensor(self, dtype, shape, base, a=None):
        """A tiled tensor (axes in the framework's order), filled with `a` (axes reversed) or zeros."""
        from paper_2504_13236_amd import tiled
        t = tiled.TiledTensor(self.ctx, dtype, shape, base)
        self.tensors.append(t)
        if a is None:
            t.buf.zero_()
        else:
            for k, cut in enumerate(_cuts(shape, base)):
                t.tile_view(k).copy_(a[cut].reshape(-1))
        return t

    def handle(self, dtype, shape, base, pointers):
        """A tensor on memory that the program has already."""
        import ctypes

        from paper_2504_13236_amd import capi
        h = ctypes.c_void_p()
        capi.nnt_tensor_create(self.ctx.h, capi.NNT_F32 if dtype == "f32" else capi.NNT_BF16, len(shape), capi.i64_array(shape),
                               capi.i64_array(base), capi.ptr_array(pointers), ctypes.byref(h))
        self.handles.append(h)
        return h

    def __del__(self):
        try:
            from paper_2504_13236_amd import capi
            for h in self.handles:
                capi.nnt_tensor_destroy(h)
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


def _rows_base(c):
    """Tiles of the attention's result: up to eight heads, 512 positions."""
    return (min(c["N_h"], 8) * c["h"], 512, c["N_b"])


def prepare(case, seed):
    c, d = case, _inputs(case, seed)
    s = _State(case)
    s.d = d
    if not own:
        if c["kind"] == "clip":
            s.G, s.O = _views(c, d["G"]), _flat(c)
        elif c["kind"] != "sample":
            # (a program knows the lengths of its sequences)
            s.starts, s.counts = d["start"].tolist(), d["count"].tolist()
            s.b, s.i = (torch.arange(c["N_s"], device="cuda") < d["count"][:, None]).nonzero(as_tuple=True)
        torch.cuda.synchronize()
        return s
    from paper_2504_13236_amd import capi
    s.ctx = _context()
    kind, dt = c["kind"], c["dtype"]
    if kind == "clip":
        s.O, s.norm = _flat(c), torch.zeros(1, device="cuda")
        both = []
        for flat in (d["G"], s.O):
            hs = []
            for shape, (_, _, offsets) in zip(_shapes(c), _places(c)[0]):
                base = [min(n, c["tile"]) for n in shape]
                hs.append(s.handle(dt, shape, base, [flat.data_ptr() + o * flat.element_size() for o in offsets]).value)
            both.append(capi.ptr_array(hs))
        s.G, s.out_tensors = both
        s.cfg = capi.nnt_clip_cfg(CLIP["max_norm"], CLIP["eps"])
    elif kind == "sample":
        s.X = s.tensor(dt, (c["N_v"], 1, c["N_b"]), (c["tile_v"], 1, c["N_b"]), d["X"].view(c["N_b"], 1, c["N_v"]))
        s.tokens, s.logp = torch.zeros(c["N_b"], device="cuda", dtype=torch.int32), torch.zeros(c["N_b"], device="cuda")
        s.cfg = capi.nnt_sample_cfg(c["temperature"], c["top_p"], c["min_p"], c["top_k"])
    else:
        h, P, N_kv, R = c["h"], c["page"], c["N_kv"], (c["N_h"] + 2 * c["N_kv"]) * c["h"]
        s.Z = s.tensor(dt, (R, c["N_s"], c["N_b"]), (8 * h, 512, c["N_b"]), d["Z"])
        n = d["K"].shape[0]
        step = N_kv * P * h * d["K"].element_size()
        s.K, s.V = (s.handle(dt, (h, n * P, N_kv), (h, P, N_kv), [d[k].data_ptr() + p * step for p in range(n)]) for k in ("K", "V"))
        s.cfg = capi.nnt_cache_cfg()
        s.cfg.N_h, s.cfg.N_kv, s.cfg.max_pages, s.cfg.window = c["N_h"], N_kv, d["pages"].shape[1], c["window"]
        s.cfg.pages, s.cfg.start, s.cfg.count = d["pages"].data_ptr(), d["start"].data_ptr(), d["count"].data_ptr()
        if c["rotation"] != "none":
            s.table = s.tensor("f32", (h, c["context"] + c["N_s"]), (h, c["context"] + c["N_s"]), d["table"])
            s.cfg.rotation = s.table.h.value
            s.cfg.rotate = capi.NNT_ROTATE_HALVES if c["rotation"] == "halves" else capi.NNT_ROTATE_PAIRS
        if kind == "attend":
            s.B = s.tensor(dt, (c["N_h"] * h, c["N_s"], c["N_b"]), _rows_base(c))
            s.out = _own_tiles("B", s.B)
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
    if kind == "append":
        capi.nnt_cache_append(h, ctypes.byref(s.cfg), s.Z.h, s.K, s.V)
        return dict(K=s.d["K"], V=s.d["V"])
    if kind == "attend":
        capi.nnt_cache_attention(h, ctypes.byref(s.cfg), c["h"] ** -0.5, s.Z.h, s.K, s.V, s.B.h)
        return s.out
    if kind == "sample":
        capi.nnt_sample_tokens(h, ctypes.byref(s.cfg), s.X.h, None, c["N_b"], s.d["u"].data_ptr(), s.tokens.data_ptr(), s.logp.data_ptr())
        return dict(tokens=s.tokens, logp=s.logp)
    capi.nnt_clip_grad_norm(h, ctypes.byref(s.cfg), len(s.G), s.G, s.out_tensors, s.norm.data_ptr())
    return dict(O=s.O, norm=s.norm)


def _rotated(c, x, table):
    """x (tokens, heads, h) in 32 bits, table (tokens, h): cosines, then sines."""
    if c["rotation"] == "none":
        return x
    cos, sin = table[:, None, :c["h"] // 2], table[:, None, c["h"] // 2:]
    if c["rotation"] == "halves":
        a, b = x[..., :c["h"] // 2], x[..., c["h"] // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _run_plain(s):
    c, d, kind = s.case, s.d, s.case["kind"]
    if kind == "clip":
        norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s.G]).sum().sqrt()
        factor = (CLIP["max_norm"] / (norm + CLIP["eps"])).clamp_max(1.0)
        for g, o in zip(s.G, _views(c, s.O)):
            o.copy_(g.float() * factor.float())
        return dict(O=s.O, norm=norm.float().reshape(1))
    if kind == "sample":
        return _sample_plain(c, d["X"], d["u"])
    h, P, N_h, N_kv = c["h"], c["page"], c["N_h"], c["N_kv"]
    Z = d["Z"].view(c["N_b"], c["N_s"], N_h + 2 * N_kv, h)
    table = d.get("table")
    if kind == "append":
        b, i = s.b, s.i
        p = d["start"].long()[b] + i
        page, slot = d["pages"][b, p // P].long(), p % P
        x = Z[b, i].float()
        k = _rotated(c, x[:, N_h:N_h + N_kv], table[p] if table is not None else None)
        d["K"][page, :, slot] = k.to(d["K"].dtype)
        d["V"][page, :, slot] = x[:, N_h + N_kv:].to(d["V"].dtype)
        return dict(K=d["K"], V=d["V"])
    out = torch.zeros(c["N_b"], c["N_s"], N_h * h, device="cuda", dtype=Z.dtype)
    for b in range(c["N_b"]):
        start, n = s.starts[b], s.counts[b]
        if n == 0:
            continue
        total = start + n
        pages = d["pages"][b, :-(-total // P)].long()
        K, V = (d[k][pages].transpose(0, 1).reshape(N_kv, -1, h)[:, :total].float() for k in ("K", "V"))
        q = _rotated(c, Z[b, :n, :N_h].float(), table[start:total] if table is not None else None)
        q = q.view(n, N_kv, N_h // N_kv, h).permute(1, 2, 0, 3).reshape(N_kv, -1, h) * h ** -0.5
        scores = torch.matmul(q, K.transpose(1, 2)).view(N_kv, N_h // N_kv, n, total)
        key, query = torch.arange(total, device="cuda"), torch.arange(start, total, device="cuda")[:, None]
        seen = key <= query
        if c["window"]:
            seen &= key > query - c["window"]
        scores.masked_fill_(~seen, -math.inf)
        e = (scores - scores.amax(-1, keepdim=True)).exp()
        o = torch.matmul(e.view(N_kv, -1, total), V).view(N_kv, N_h // N_kv, n, h) / e.sum(-1, keepdim=True)
        out[b, :n] = o.permute(2, 0, 1, 3).reshape(n, N_h * h).to(out.dtype)
    return _tiles("B", out, _rows_base(c))


def _sample_plain(c, X, u):
    """Weights, sums and borders in 64 bits: a drawn token changes with the last bit of a running sum."""
    tokens, logps = [], []
    for x, r in zip(X.split(64), u.split(64)):
        x = x.double()
        x = torch.where(x.isnan(), torch.full((), -math.inf, dtype=torch.float64, device=x.device), x)
        top = x.amax(-1, keepdim=True)
        if c["temperature"] == 0.0:
            token = x.argmax(-1)
        else:
            e = torch.exp((x - top) / c["temperature"])
            # likeliest first, among equals the lowest index
            order = torch.sort(x, dim=-1, descending=True, stable=True)[1]
            falling = e.gather(-1, order)
            keep = torch.ones_like(falling, dtype=torch.bool)
            if c["top_k"]:
                keep[:, c["top_k"]:] = False
            sums = (falling * keep).cumsum(-1)
            if c["top_p"] < 1.0:
                keep &= torch.nn.functional.pad(sums[:, :-1], (1, 0)) < c["top_p"] * sums[:, -1:]
            keep &= falling >= c["min_p"]
            kept = torch.zeros_like(e).scatter_(-1, order, falling * keep)
            sums = kept.cumsum(-1)
            token = (sums > r.double()[:, None] * sums[:, -1:]).to(torch.int8).argmax(-1)
        tokens.append(token.int())
        logps.append((x.gather(-1, token[:, None]) - top - torch.exp(x - top).sum(-1, keepdim=True).log())[:, 0].float())
    return dict(tokens=torch.cat(tokens), logp=torch.cat(logps))


# ------------------------------------------------------------------------------------------------- what a pass needs
def _lengths(c):
    """Contexts and new tokens as _inputs draws them, on the average: the first sequence whole, the others 5/8 of the context and half the tokens."""
    rest = c["N_b"] - 1
    n = c["N_s"] if c["N_s"] == 1 else (c["N_s"] + 1) / 2
    return [(c["context"], c["N_s"])] + [(0.625 * c["context"], n)] * rest


def work(case):
    c = case
    w = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "clip":
        n = sum(math.prod(s) for s in _shapes(c))
        # the factor is known once all has been read: in again, out
        return dict(flops=3.0 * n, bytes=3.0 * n * w)
    if c["kind"] == "sample":
        n = c["N_v"] * c["N_b"]
        return dict(flops=4.0 * n, bytes=n * w + 12 * c["N_b"])
    h, N_h, N_kv = c["h"], c["N_h"], c["N_kv"]
    byts = flops = 0.0
    for start, n in _lengths(c):
        if c["kind"] == "append":
            byts += n * 4 * N_kv * h * w + (n * h * 4 if c["rotation"] != "none" else 0)
            flops += n * 3 * N_kv * h
        else:
            seen = min(start + n, c["window"] + n) if c["window"] else start + n
            byts += seen * 2 * N_kv * h * w + n * 2 * N_h * h * w
            flops += 4.0 * n * (min(start + n / 2, c["window"]) if c["window"] else start + n / 2) * N_h * h
    return dict(flops=flops, bytes=byts)


# ------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    """From the definitions, one sequence, one cached head or one column at a time."""
    c, d = case, _inputs(case, seed)
    if c["kind"] == "clip":
        norm = torch.linalg.vector_norm(d["G"].double())
        return dict(O=d["G"].double() * min(1.0, CLIP["max_norm"] / (float(norm) + CLIP["eps"])), norm=norm.reshape(1))
    if c["kind"] == "sample":
        return _sample_exact(c, d["X"], d["u"])
    N_b, N_s, h, P, N_h, N_kv = c["N_b"], c["N_s"], c["h"], c["page"], c["N_h"], c["N_kv"]
    Z = d["Z"].view(N_b, N_s, N_h + 2 * N_kv, h)

    def turn(x, first):
        """Rows of consecutive positions as complex numbers times e^(i angle), the table's values."""
        if c["rotation"] == "none":
            return x
        t = d["table"][first:first + len(x)].double()
        z = torch.complex(t[:, :h // 2], t[:, h // 2:])
        if c["rotation"] == "halves":
            y = torch.complex(x[:, :h // 2], x[:, h // 2:]) * z
            return torch.cat([y.real, y.imag], 1)
        y = torch.view_as_complex(x.reshape(len(x), h // 2, 2).contiguous()) * z
        return torch.view_as_real(y).reshape(len(x), h)

    if c["kind"] == "append":
        K, V = d["K"].double(), d["V"].double()
        for b in range(N_b):
            start, n = int(d["start"][b]), int(d["count"][b])
            for j in range(N_kv):
                k, v = turn(Z[b, :n, N_h + j].double(), start), Z[b, :n, N_h + N_kv + j].double()
                done = 0
                while done < n:
                    page, slot = int(d["pages"][b, (start + done) // P]), (start + done) % P
                    m = min(P - slot, n - done)
                    K[page, j, slot:slot + m] = k[done:done + m]
                    V[page, j, slot:slot + m] = v[done:done + m]
                    done += m
        return dict(K=K, V=V)
    out = torch.zeros(N_b, N_s, N_h * h, dtype=torch.float64, device="cuda")
    for b in range(N_b):
        start, n = int(d["start"][b]), int(d["count"][b])
        if n == 0:
            continue
        total = start + n
        pages = d["pages"][b, :-(-total // P)].long()
        first = max(0, start + 1 - c["window"]) if c["window"] else 0
        bias = torch.zeros(n, total - first, dtype=torch.float64, device="cuda")
        for i in range(n):
            bias[i, start + i + 1 - first:] = -math.inf
            if c["window"]:
                bias[i, :max(0, start + i + 1 - c["window"] - first)] = -math.inf
        for j in range(N_kv):
            K, V = (d[k][pages, j].reshape(-1, h)[first:total].double() for k in ("K", "V"))
            for g in range(N_h // N_kv):
                head = j * (N_h // N_kv) + g
                q = turn(Z[b, :n, head].double(), start)
                out[b, :n, head * h:(head + 1) * h] = torch.softmax(torch.mm(q, K.t()) / math.sqrt(h) + bias, -1) @ V
    return _tiles("B", out, _rows_base(c))


def _sample_exact(c, X, u):
    tokens, logps = [], []
    for x, r in zip(X, u):
        x = x.double()
        logp = torch.log_softmax(x, -1)
        if c["temperature"] == 0.0:
            token = int((x == x.max()).nonzero()[0, 0])
        else:
            p = torch.exp((x - x.max()) / c["temperature"])
            index = torch.sort(x, descending=True, stable=True)[1]
            n = min(c["top_k"] or len(x), len(x))
            mass = p[index[:n]].cumsum(0)
            if c["top_p"] < 1.0:
                # as many as it takes to reach the share
                n = min(n, int((mass < c["top_p"] * mass[-1]).sum()) + 1)
            n = min(n, int((p >= c["min_p"]).sum()))
            chosen = index[:n].sort()[0]
            mass = p[chosen].cumsum(0)
            token = int(chosen[min(int((mass <= float(r) * mass[-1]).sum()), n - 1)])
        tokens.append(token)
        logps.append(logp[token])
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda"), logp=torch.stack(logps))
