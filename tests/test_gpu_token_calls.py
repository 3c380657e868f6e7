"""How the Python calls of rotary positions and the token cache take their arguments."""
import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

pytestmark = pytest.mark.gpu


def _setup():
    cache = fdb.TokenCache.empty(1, 2, 16, 64, torch.float32)
    rope = fdb.Rope(fdb.fd_rope_frequencies(64)[0])
    x = torch.randn(1, 3, 2, 64, device="cuda")
    return cache, rope, x, torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)


def test_inputs_that_require_grad():
    """Refused while gradients are recorded, where they would be lost in silence; taken under no_grad, in a Function's
    forward, and detached."""
    cache, rope, x, pos = _setup()
    leaf = x.clone().requires_grad_()
    slots = cache.choose(pos)
    calls = [lambda t: rope(t[0], pos[0]), lambda t: cache.attend(t, pos), lambda t: cache.append(t, x, pos, slots),
             lambda t: cache.append(x, t, pos, slots), lambda t: cache.insert(t, t, pos)]
    before = [t.clone() for t in (cache.k, cache.v, cache.pos, cache.weight)]
    for call in calls:
        for t in (leaf, leaf * 2.0):
            with pytest.raises(ValueError, match="grad"):
                call(t)
    assert all(torch.equal(a, b) for a, b in zip(before, (cache.k, cache.v, cache.pos, cache.weight)))
    with pytest.raises(ValueError, match="grad"):
        fdb.TokenCache(cache.k.clone().requires_grad_(), cache.v, cache.pos, cache.weight).attend(x, pos)
    for call in calls:
        call(leaf.detach())
        with torch.no_grad():
            call(leaf)

    class Turn(torch.autograd.Function):
        """The rotation in training: its gradient is the inverse rotation's."""
        @staticmethod
        def forward(ctx, t):
            return rope(t, pos[0])

        @staticmethod
        def backward(ctx, g):
            return rope.inverted()(g, pos[0])

    w = torch.randn_like(x[0])
    (Turn.apply(leaf[0]) * w).sum().backward()
    assert torch.equal(leaf.grad[0], rope.inverted()(w, pos[0]))


def test_coordinates_of_one_axis():
    """append takes them as [batch, n] or [batch, n, 1], as a rotation does; other shapes are refused."""
    cache, rope, x, pos = _setup()
    slots, coords = cache.choose(pos), pos * 7 + 2
    cache.append(x, x, pos, slots, rope, coords[..., None].contiguous())
    want = cache.k.clone()
    cache.k.zero_()
    cache.append(x, x, pos, slots, rope, coords)
    assert torch.equal(cache.k, want) and bool(want.any())
    for bad in (coords[0], coords[:, :2].contiguous(), coords[..., None].expand(1, 3, 2).contiguous(), coords.long()):
        with pytest.raises(ValueError):
            cache.append(x, x, pos, slots, rope, bad)
    three = fdb.Rope(rope.freq, torch.zeros(32, dtype=torch.int32, device="cuda"), 3)
    with pytest.raises(ValueError):
        cache.append(x, x, pos, slots, three, coords)
