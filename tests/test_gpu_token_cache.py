"""Rotary positions and the token cache (choice of slots, append) on the GPU against
plain implementations in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(shape, generator=_gen(seed), dtype=torch.float64)


def _same(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and bool(torch.equal(a, b))


# ------------------------------------------------------------------ rotary positions

def rope_ref(x, coords, freq, axis, layout, mag, inverse):
    """x [tokens, heads, dim] fp64, coords [tokens, axes]: (rotated, bound on the error of an
    fp32 computation of it)."""
    half = len(freq)
    ax = np.zeros(half, int) if axis is None else np.asarray(axis)
    ang = coords.double().numpy()[:, ax] * np.asarray(freq)
    cos, sin = (torch.from_numpy(mag * f(ang))[:, None] for f in (np.cos, np.sin))
    if inverse:
        sin = -sin
    i0 = torch.arange(half) * 2 if layout == "interleaved" else torch.arange(half)
    i1 = i0 + 1 if layout == "interleaved" else i0 + half
    y, err = x.clone(), torch.zeros_like(x)
    y[..., i0] = x[..., i0] * cos - x[..., i1] * sin
    y[..., i1] = x[..., i0] * sin + x[..., i1] * cos
    # sine and cosine in fp32: half a step of the reduced angle (at most pi 2^-24), two steps of the function,
    # one of the magnitude, two of the products and the sum: below 8 steps of 2^-24, each of |x0| + |x1|
    e = abs(mag) * 8 * 2.0 ** -24 * (x[..., i0].abs() + x[..., i1].abs())
    err[..., i0] = e
    err[..., i1] = e
    return y, err


def _check_rope(got, x, coords, freq, axis, layout, mag, inverse):
    ref, err = rope_ref(x.double(), coords, freq, axis, layout, mag, inverse)
    # the one rounding to the type: half a step (below the normal range, half the least step)
    fi = torch.finfo(got.dtype)
    tol = err + fi.eps / 2 * (ref.abs() + err) + fi.tiny * fi.eps / 2
    assert bool(((got.double() - ref).abs() <= tol).all())
    half = len(freq)
    assert _same(got[..., 2 * half:], x[..., 2 * half:])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("tokens,heads,dim,rot", [
    (1, 1, 2, 2), (1, 8, 64, 64), (3, 5, 64, 32), (257, 3, 128, 96), (19, 24, 64, 20), (7, 2, 33, 30), (5, 1, 512, 512),
    (1300, 1, 32, 32), (4, 300, 64, 16), (2, 3, 64, 0)])
def test_rope(dtype, layout, tokens, heads, dim, rot):
    x = _randn(1, tokens, heads, dim).to(dtype)
    coords = torch.randint(-50, 5000, (tokens, 1), generator=_gen(2), dtype=torch.int32)
    freq = fdb.fd_rope_frequencies(rot)[0] if rot else np.empty(0)
    rope = fdb.Rope(freq, layout=layout)
    got = rope(x.cuda(), coords.cuda()).cpu()
    _check_rope(got, x, coords, freq, None, layout, 1.0, False)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands"])
def test_rope_far_positions_and_axes(layout, scaling):
    """Three coordinates, positions up to 2^31 - 1, scaled frequencies, a magnitude."""
    sections, parts, mag = [16, 24, 24], [], 1.0
    for s in sections:
        f, mag = fdb.fd_rope_frequencies(s, 10000.0, scaling, 4.0, 4096.0)
        parts.append(f)
    freq, axis = np.concatenate(parts), np.repeat([0, 1, 2], [8, 12, 12])
    coords = torch.randint(0, 2 ** 31 - 1, (65, 3), generator=_gen(3), dtype=torch.int32)
    coords[0] = 2 ** 31 - 1
    x = _randn(4, 65, 3, 64).float()
    rope = fdb.Rope(freq, axis, 3, layout, mag)
    got = rope(x.cuda(), coords.cuda()).cpu()
    ref, err = rope_ref(x.double(), coords, freq, axis, layout, float(np.float32(mag)), False)
    # + the angle's own error in 64 bits: two roundings of up to 2^31 / (2 pi) turns, here and in the reference
    err = err + 4 * 2 * math.pi * 2.0 ** -53 * 2 ** 31 / (2 * math.pi) * mag * 2 * x.double().abs().amax()
    assert bool(((got.double() - ref).abs() <= err + 2.0 ** -24 * ref.abs()).all())


def test_rope_inverse_is_the_gradient():
    """The inverse turns back, and equals the gradient of the rotation (its transpose) on differences."""
    freq = fdb.fd_rope_frequencies(32)[0]
    rope = fdb.Rope(freq, magnitude=1.25)
    x, w = _randn(5, 9, 2, 64).float(), _randn(6, 9, 2, 64).float()
    coords = torch.arange(9, dtype=torch.int32) * 37
    inv = rope.inverted()
    _check_rope(inv(w.cuda(), coords.cuda()).cpu(), w, coords[:, None], freq, None, "interleaved", 1.25, True)
    y = rope(x.cuda(), coords.cuda()).cpu().double()
    g = inv(w.cuda(), coords.cuda()).cpu().double()
    # <rope(x), w> = <x, inverse(w)> for every x, so the inverse is the gradient
    lhs, rhs = (y * w.double()).sum(), (x.double() * g).sum()
    slack = 16 * 2.0 ** -24 * 1.25 * 2 * (x.double().abs().amax() * w.double().abs().sum())
    assert abs(lhs - rhs) <= slack
    # a step along one element moves the output by the gradient's column
    for at in [(0, 0, 0), (3, 1, 7), (8, 0, 31), (8, 1, 40)]:
        x2 = x.clone()
        x2[at] += 1.0
        dy = ((rope(x2.cuda(), coords.cuda()).cpu().double() - y) * w.double()).sum()
        assert abs(dy - g[at]) <= 64 * 2.0 ** -24 * 1.25 * 2 * 8 * 8


def test_rope_strides_alignment_and_in_place():
    freq = fdb.fd_rope_frequencies(48)[0]
    coords = torch.randint(0, 999, (11,), generator=_gen(7), dtype=torch.int32).cuda()
    for dtype in (F16, F32):
        for layout in ("interleaved", "half"):
            rope = fdb.Rope(freq, layout=layout)
            big = _randn(8, 11, 9, 80).to(dtype).cuda()
            plain = rope(big[:, 2:7, :64].contiguous(), coords)
            # a slice of a fused projection, rows that start off 16 bytes, heads before tokens
            assert _same(rope(big[:, 2:7, :64], coords), plain)
            off = torch.empty(11 * 5 * 64 + 1, dtype=dtype, device="cuda")[1:].view(11, 5, 64)
            off.copy_(big[:, 2:7, :64])
            assert _same(rope(off, coords), plain)
            out = torch.empty(5, 11, 64, dtype=dtype, device="cuda").transpose(0, 1)
            assert rope(big[:, 2:7, :64], coords, out=out) is out and _same(out, plain)
            # in place: only the rotated heads change
            before = big.clone()
            view = big[:, 2:7, :64]
            rope(view, coords, out=view)
            assert _same(view, plain)
            assert _same(big[:, :2], before[:, :2]) and _same(big[:, 7:], before[:, 7:])
            assert _same(big[..., 64:], before[..., 64:])


def test_rope_no_tokens_and_capture():
    rope = fdb.Rope(fdb.fd_rope_frequencies(64)[0])
    assert rope(torch.empty(0, 3, 64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 3, 64)
    x, pos = torch.randn(5, 3, 64, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rope(x, pos, out=out, stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope(x, pos, out=out)
    for i in range(3):
        x.copy_(torch.randn(5, 3, 64, device="cuda"))
        pos.add_(1000 * i)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert _same(got, rope(x, pos))


# ------------------------------------------------------------------ choice of slots

def slots_ref(at, weight, pos, keep_first, keep_recent):
    """The rule on Python integers and floats."""
    B, G, C = at.shape
    n = pos.shape[1]
    out = np.full((B, G, n), -1, np.int32)
    for b in range(B):
        valid = [i for i in range(n) if pos[b, i] >= 0]
        if not valid:
            continue
        newest = max(int(pos[b, i]) for i in valid)
        for g in range(G):
            def key(s):
                p, w = int(at[b, g, s]), float(weight[b, g, s])
                w = -math.inf if math.isnan(w) else w
                c = 0 if p < 0 else 3 if p < keep_first else 2 if p > newest - keep_recent else 1
                return (c, w if c else 0.0, s)
            taken = sorted(sorted(range(C), key=key)[:len(valid)])
            for i, s in zip(valid, taken):
                out[b, g, i] = s
    return out


def _slots(at, weight, pos, first, recent):
    B, G, _ = at.shape
    out = torch.full((B, G, pos.shape[1]), -7, dtype=torch.int32, device="cuda")
    fdb.fd_token_slots_device(torch.from_numpy(at).cuda(), torch.from_numpy(weight).cuda(),
                              torch.from_numpy(pos).cuda(), out, first, recent)
    return out.cpu().numpy()


@pytest.mark.parametrize("C,n", [(1, 1), (2, 2), (5, 3), (64, 1), (64, 64), (97, 31), (1000, 999), (4096, 100),
                                 (4097, 130), (16384, 16384), (16385, 5), (20001, 777), (70000, 1), (70000, 66)])
@pytest.mark.parametrize("kind", ["full", "ties", "some_empty", "special"])
def test_slots(C, n, kind):
    r = np.random.default_rng(C * 31 + n)
    B, G = 2, 2
    at = np.stack([r.permutation(2 * C)[:C] for _ in range(B * G)]).reshape(B, G, C).astype(np.int32)
    weight = r.gamma(0.3, 1.0, (B, G, C)).astype(np.float32)
    if kind == "ties":
        weight = r.integers(0, 3, (B, G, C)).astype(np.float32)
    if kind == "some_empty":
        at[r.random((B, G, C)) < 0.3 * n / C] = -1
    if kind == "special":
        weight[r.random((B, G, C)) < 0.2] = np.float32("nan")
        weight[r.random((B, G, C)) < 0.2] = -np.inf
        weight[r.random((B, G, C)) < 0.2] = np.inf
        weight[r.random((B, G, C)) < 0.2] = -0.0
        weight[r.random((B, G, C)) < 0.1] = -1e-42
        at[0, 0, :] = -5
    pos = np.broadcast_to(2 * C + np.arange(n), (B, n)).astype(np.int32).copy()
    if kind in ("some_empty", "special") and n > 2:
        pos[0, r.random(n) < 0.4] = -1  # padding in between
        pos[1, n // 2:] = -1            # and behind
    for first, recent in [(0, 0), (4, max(1, C // 3)), (3 * C, 0), (0, 4 * C)]:
        got = _slots(at, weight, pos, first, recent)
        assert np.array_equal(got, slots_ref(at, weight, pos, first, recent)), (first, recent)


def test_slots_all_padding_and_largest_positions():
    at = np.array([[[0, 2 ** 31 - 1, 5, -2 ** 31]]], np.int32)
    w = np.array([[[3, 1, 2, 0]]], np.float32)
    assert (_slots(at, w, np.full((1, 3), -1, np.int32), 0, 0) == -1).all()
    for recent in (0, 1, 2 ** 31 - 1):
        pos = np.array([[2 ** 31 - 1, -3, 7]], np.int32)
        assert np.array_equal(_slots(at, w, pos, 1, recent), slots_ref(at, w, pos, 1, recent))


def test_slots_most_tokens():
    """65536 new tokens with padding, over more slots than registers hold."""
    r = np.random.default_rng(0)
    C, n = 70001, 65536
    at = r.permutation(C).astype(np.int32).reshape(1, 1, C)
    w = r.standard_normal((1, 1, C)).astype(np.float32)
    pos = (C + np.arange(n)).astype(np.int32).reshape(1, n)
    pos[0, r.random(n) < 0.1] = -1
    assert np.array_equal(_slots(at, w, pos, 9, 1000), slots_ref(at, w, pos, 9, 1000))


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("D,rot,layout,axes", [(64, 64, "interleaved", 3), (128, 64, "half", 1), (32, 20, "half", 1),
                                               (64, 6, "interleaved", 1), (128, 0, "half", 1)])
@pytest.mark.parametrize("B,G,C,n", [(1, 1, 1, 1), (2, 3, 40, 7), (1, 2, 700, 600)])
def test_append(dtype, D, rot, layout, axes, B, G, C, n):
    r = np.random.default_rng(n)
    # rows of a larger buffer: strides that are not the shape's
    kbuf = _randn(1, B, G + 1, C, D + 32).to(dtype).cuda()
    vbuf = _randn(2, B, G, C + 1, D).to(dtype).cuda()
    at = torch.full((B, G, C), -1, dtype=torch.int32).cuda()
    w = torch.rand(B, G, C, generator=_gen(3)).cuda()
    cache = fdb.TokenCache(kbuf[:, :G, :, :D], vbuf[:, :, :C], at, w)
    qkv = _randn(4, B, n, 4 * G, D).to(dtype).cuda()
    k, v = qkv[:, :, G:2 * G], qkv[:, :, 3 * G:]
    pos = torch.from_numpy(r.integers(0, 9999, (B, n)).astype(np.int32))
    slots = torch.from_numpy(np.stack([r.permutation(C)[:n] for _ in range(B * G)]).reshape(B, G, n).astype(np.int32))
    if n > 2:
        pos[:, 1] = -1         # padding keeps its slot as it was
        slots[:, :, 2] = C     # outside: left out
        slots[0, 0, 0] = -1
    freq = fdb.fd_rope_frequencies(rot)[0] if rot else np.empty(0)
    axis = np.arange(rot // 2) % axes if axes > 1 else None
    rope = fdb.Rope(freq, axis, axes, layout, 1.1) if rot else None
    coords = torch.from_numpy(r.integers(0, 500, (B, n, axes)).astype(np.int32)) if axes > 1 else None
    want_k, want_v, want_at, want_w = (t.clone() for t in (kbuf, vbuf, at, w))
    cache.append(k, v, pos.cuda(), slots.cuda(), rope, None if coords is None else coords.cuda())
    turned = k.cpu()
    if rope:
        c = (pos[..., None] if coords is None else coords).reshape(B * n, axes)
        flat = rope(k.reshape(B * n, G, D), c.cuda()).cpu()
        _check_rope(flat, k.reshape(B * n, G, D).cpu(), c, freq, axis, layout, float(np.float32(1.1)), False)
        turned = flat.view(B, n, G, D)
    for b in range(B):
        for g in range(G):
            for i in range(n):
                s = int(slots[b, g, i])
                if pos[b, i] >= 0 and 0 <= s < C:
                    want_k[b, g, s, :D] = turned[b, i, g]
                    want_v[b, g, s] = v[b, i, g]
                    want_at[b, g, s] = pos[b, i]
                    want_w[b, g, s] = 0
    for got, want in ((kbuf, want_k), (vbuf, want_v), (at, want_at), (w, want_w)):
        assert _same(got, want)
