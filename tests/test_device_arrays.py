"""Device arrays that the helpers of tiled.py hand to the calls on a cache, of drawn tokens and of clipped gradients by their address: their type, number
and place are looked at first.  (Everything here is refused before the library is asked.)"""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

CTX = SimpleNamespace(device=0, h=None)


@pytest.fixture(scope="module")
def tiled():
    from paper_2504_13236_amd import tiled
    return tiled


def a_cache(tiled, N_b=3, n_layers=2):
    c = object.__new__(tiled.PagedCache)
    layer = SimpleNamespace(h=SimpleNamespace(value=None), shape=(8, 32, 1))
    c.ctx, c.N_b, c.N_h, c.N_kv, c.max_pages, c.window, c.rotation, c.rotate = CTX, N_b, 1, 1, 4, 0, None, 0
    c.pages, c.K, c.V = torch.full((N_b, 4), -1, dtype=torch.int32), [layer] * n_layers, [layer] * n_layers
    return c


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


WRONG_INTS = [i32(3).long(), i32(3).float(), i32(2), i32(6)[::2], i32(0)]


@pytest.mark.parametrize("wrong", WRONG_INTS, ids=lambda t: "%s%s" % (t.dtype, tuple(t.shape)))
def test_lengths_of_a_cache(tiled, wrong):
    c = a_cache(tiled)
    with pytest.raises(ValueError, match="start: 3 contiguous entries"):
        c.cfg(wrong)
    with pytest.raises(ValueError, match="start: on cpu"):
        c.cfg(i32(3), wrong)
    c.ctx = SimpleNamespace(device=0)
    z = SimpleNamespace(shape=(24, 1, 3), h=None)
    for call in (lambda: c.append(z, wrong), lambda: c.attention(z, z, wrong)):
        with pytest.raises(ValueError, match="start"):
            call()


def test_a_count_is_looked_at_too(tiled, monkeypatch):
    looked = []
    monkeypatch.setattr(tiled, "_device_entries", lambda ctx, name, t, dtype, n: looked.append((name, dtype, n)) or 16)
    a_cache(tiled).cfg(i32(3), i32(3))
    assert looked == [("start", torch.int32, 3), ("count", torch.int32, 3)]


def test_a_cache_of_other_sequences_or_blocks(tiled):
    c, start = a_cache(tiled), i32(3)
    with pytest.raises(ValueError, match="another number"):
        c.append(SimpleNamespace(shape=(24, 1, 4), h=None), start)
    with pytest.raises(ValueError, match="another number"):
        c.attention(SimpleNamespace(shape=(24, 1, 2), h=None), None, start)
    block = object.__new__(tiled.Gpt2Block)
    block.ctx, block.h, block.act_shape = CTX, None, (8, 1, 4)
    with pytest.raises(ValueError, match="another number"):
        block.forward_cached(c, None, None, start)
    block.act_shape = (8, 1, 3)
    stack = object.__new__(tiled.Gpt2Stack)
    stack.ctx, stack.h = CTX, None
    for n in (1, 3):
        stack.blocks = [block] * n
        with pytest.raises(ValueError, match="another number"):
            stack.forward_cached(c, start)


@pytest.mark.parametrize("name,wrong", [("uniforms", torch.zeros(4, dtype=torch.float64)), ("uniforms", torch.zeros(4, dtype=torch.float16)), ("uniforms", torch.zeros(3)),
                                        ("uniforms", torch.zeros(8)[::2]), ("tokens", i32(4).long()), ("tokens", i32(8)[::2]), ("tokens", i32(5)), ("logp", torch.zeros(4).double()),
                                        ("logp", torch.zeros(5)), ("columns", i32(4).long()), ("columns", i32(3))])
def test_arrays_of_a_draw(tiled, name, wrong, monkeypatch):
    monkeypatch.setattr(torch, "device", lambda *a: torch.zeros(0).device)         # (the place is not what is wrong)
    a = dict(uniforms=torch.zeros(4), tokens=i32(4), logp=torch.zeros(4), columns=i32(4))
    a[name] = wrong
    with pytest.raises(ValueError, match="%s: 4 contiguous|one length" % name):
        tiled.sample_tokens(CTX, SimpleNamespace(h=None), **a)
    model = object.__new__(tiled.Gpt2Model)
    model.ctx, model.h, model.blocks, model.N_s, model.N_b = CTX, None, [None] * 2, 1, 3
    model.tokens = model.pos = i32(3)
    a["next"] = a.pop("tokens")
    with pytest.raises(ValueError, match="%s: 4 contiguous|one length" % name):
        model.sample(a_cache(tiled), i32(3), **a)
    a[name if name != "tokens" else "next"] = dict(uniforms=torch.zeros(4), tokens=i32(4), logp=torch.zeros(4), columns=i32(4))[name]
    for kw in (dict(tokens=i32(3).long()), dict(tokens=i32(2)), dict(positions=i32(6)[::2]), dict(positions=torch.zeros(3))):
        with pytest.raises(ValueError, match="%s: 3 contiguous" % list(kw)[0]):
            model.sample(a_cache(tiled), i32(3), **a, **kw)


@pytest.mark.parametrize("wrong", [torch.zeros(1, dtype=torch.float64), torch.zeros(0), torch.zeros(1)], ids=lambda t: "%s%s%s" % (t.dtype, tuple(t.shape), t.device))
def test_where_a_norm_goes(tiled, wrong):
    with pytest.raises(ValueError, match="norm"):
        tiled.clip_grad_norm(CTX, [], wrong)
    for kind in (tiled.Gpt2Block, tiled.Gpt2Stack, tiled.Gpt2Model):
        x = object.__new__(kind)
        x.ctx, x.h = CTX, None
        with pytest.raises(ValueError, match="norm"):
            x.clip(wrong)


def test_the_table_of_pages_is_there_when_reserve_returns(tiled, monkeypatch):
    """The copy is waited for on the cache's device, whichever is the current one."""
    waited = []
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: waited.append(device))
    c = a_cache(tiled)
    c.page, c.free, c.of = 4, [2, 1, 0], [[], [], []]
    c.reserve([5, 0, 1])
    assert c.pages.tolist() == [[0, 1, -1, -1], [-1] * 4, [2, -1, -1, -1]]
    c.release(0)
    assert c.pages.tolist()[0] == [-1] * 4
    assert waited == [c.pages.device] * 2
