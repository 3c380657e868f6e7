"""Refusals of the token cache and of rotary positions that need no GPU: rows that would be written twice,
scales beyond fp32, inputs whose gradient would be lost."""
import ctypes
import itertools
import math
import random

import numpy as np
import pytest

from paper_2607_14898_amd import flashdecoder as fdb
from tests.test_token_cache_host import A, INVALID, _append_call, _attend_call, _lib, _rope_call, cache_struct


def _overlap(strides, extents, width):
    """Two rows of `width` elements that share one, by brute force."""
    seen = np.sort([sum(i * s for i, s in zip(at, strides)) for at in itertools.product(*map(range, extents))])
    return len(seen) > 1 and int(np.diff(seen).min()) < width


def _says(lib, status, word):
    assert status == INVALID
    return word in lib.fd_last_error().decode()


def test_rows_of_out_that_overlap():
    lib = _lib()
    r = random.Random(0)
    kinds = set()
    for _ in range(400):
        T, H, D = r.randint(1, 7), r.randint(1, 7), r.choice([4, 8, 16])
        ts, hs = (D + r.choice([0, 1, 3, D, r.randint(0, 6 * D)]) for _ in range(2))
        if r.random() < 0.4:  # views of one tensor
            ts, hs = r.choice([(H * D, D), (D, T * D), (2 * H * D + 5, 2 * D)])
        want = _overlap((ts, hs), (T, H), D)
        kinds.add((want, ts >= H * hs or hs >= T * ts))
        # (x NULL: a layout that is not refused is told that, before any device work)
        st = _rope_call(lib, _small_rope(), x=None, dim=D, tokens=T, heads=H, xt=D, xh=D, ot=ts, oh=hs)
        assert _says(lib, st, "overlap") == want, (T, H, D, ts, hs)
    assert len(kinds) >= 3
    assert _says(lib, _rope_call(lib, tokens=4, heads=2, dim=64, xt=64, xh=64, ot=64, oh=64), "overlap")
    # far and many: found, or seen to nest, at once
    assert _says(lib, _rope_call(lib, x=None, tokens=2 ** 31 - 1, heads=65536, ot=65536 * 64, oh=64), "NULL")
    assert _says(lib, _rope_call(lib, x=None, tokens=2 ** 31 - 1, heads=65536, ot=64 * 65535, oh=64), "overlap")


def _small_rope():
    s = fdb.fd_rope(ctypes.sizeof(fdb.fd_rope), 4, 0, 1, A, None, 1.0, 0)
    return s


def test_rows_of_attention_and_cache_that_overlap():
    lib = _lib()
    r = random.Random(1)
    found = {True: 0, False: 0}
    for _ in range(400):
        B, G, C = r.randint(1, 4), r.randint(1, 4), r.randint(1, 9)
        s = [64 * r.randint(1, 14) + r.choice([0, 0, 8]) for _ in range(3)]
        if r.random() < 0.4:
            s = r.choice([[G * C * 64, C * 64, 64], [64, B * C * 64, B * 64], [C * 64, B * C * 64, 64]])
        want = _overlap(s, (B, G, C), 64)
        found[want] += 1
        plain = (G * C * 64, C * 64, 64)
        for at in ("k_stride", "v_stride"):
            c = cache_struct(batch=B, groups=G, capacity=C, k_stride=plain, v_stride=plain)
            setattr(c, at, (ctypes.c_int64 * 3)(*s))
            assert _says(lib, _append_call(lib, c, slots=None, ks=(512, 128, 64)), "overlap") == want, (B, G, C, s)
            # (read alone they may)
            assert not _says(lib, _attend_call(lib, c, heads=G, n=1, pos=A + 1), "overlap")
        c = cache_struct(batch=B, groups=G, k_stride=(G * 1024, 1024, 64), v_stride=(G * 1024, 1024, 64))
        st = _attend_call(lib, c, qs=(4096, 64, 1024), os_=(s[0], s[2], s[1]), heads=G, n=C, ws=None)
        assert _says(lib, st, "overlap") == want, (B, G, C, s)
    assert min(found.values()) > 50


def test_scales_beyond_fp32():
    """The kernels work in powers of two: a scale whose scale / ln 2 is no fp32 number is refused."""
    lib = _lib()
    most = float(np.finfo(np.float32).max) * math.log(2)
    for scale in (most * 1.0001, 3e38, float(np.finfo(np.float32).max)):
        assert _says(lib, _attend_call(lib, scale=scale), "scale"), scale
    for scale in (most * 0.9999, 1e30, 1e-38):
        assert _says(lib, _attend_call(lib, scale=scale, ws=None), "workspace"), scale


def test_numbers_beyond_int32():
    """A count of 2^32 is not taken for 0, nor 2^32 + 64 for 64."""
    import torch
    _lib()
    z = torch.zeros(1, 1, 4, dtype=torch.int32)
    for kw in (dict(keep_recent=2 ** 32), dict(keep_first=2 ** 32 + 4), dict(keep_recent=2 ** 31)):
        with pytest.raises(ValueError, match=next(iter(kw))):
            fdb.fd_token_slots_device(z, torch.zeros(1, 1, 4), z[0], z, **kw)
    for rot_dim in (2 ** 32 + 64, -2 ** 32 + 64):
        with pytest.raises(ValueError, match="rot_dim"):
            fdb.fd_rope_frequencies(rot_dim)
    with pytest.raises(fdb.FlashDecoderError):
        fdb.fd_rope_frequencies(2 ** 31 - 2)
    with pytest.raises(ValueError, match="n_axes"):
        fdb.Rope(torch.ones(32, dtype=torch.float64), n_axes=2 ** 32 + 1)
