"""Host side of rotary positions and the token cache: frequencies, and every refusal that needs no GPU."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

INVALID, UNSUPPORTED = fdb.FD_ERR_INVALID_ARGUMENT, fdb.FD_ERR_UNSUPPORTED


def _lib():
    if not os.path.exists(fdb.LIB_PATH):
        pytest.skip("libflashdecoder.so not built")
    return fdb.load_library()


@pytest.mark.parametrize("rot", [2, 4, 22, 64, 512])
def test_frequencies(rot):
    _lib()
    i = np.arange(rot // 2)
    plain = 10000.0 ** (-2.0 * i / rot)
    f, m = fdb.fd_rope_frequencies(rot)
    np.testing.assert_allclose(f, plain, rtol=1e-14)
    assert m == 1.0
    f, m = fdb.fd_rope_frequencies(rot, scaling="linear", factor=8.0)
    np.testing.assert_allclose(f, plain / 8, rtol=1e-14)
    f, m = fdb.fd_rope_frequencies(rot, scaling="base", factor=8.0)
    assert f[0] == 1.0 and m == 1.0
    if rot > 2:  # the slowest pair is slowed down by the factor
        np.testing.assert_allclose(f[-1], plain[-1] / 8, rtol=1e-12)
    f, m = fdb.fd_rope_frequencies(rot, scaling="bands", factor=8.0, trained_length=2048.0)
    turns = 2048 * plain / (2 * math.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    np.testing.assert_allclose(f, keep * plain + (1 - keep) * plain / 8, rtol=1e-14)
    assert m == np.float32(1 + 0.1 * math.log(8))


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=514), dict(rot_dim=-2), dict(theta=1.0),
                                dict(theta=math.inf), dict(theta=math.nan), dict(scaling="linear", factor=0.5),
                                dict(scaling="base", factor=math.inf), dict(scaling="linear", factor=math.nan),
                                dict(scaling="bands", factor=2.0), dict(scaling="bands", factor=2.0, trained_length=-1.0),
                                dict(scaling="bands", factor=2.0, trained_length=9.0, fast_turns=1.0, slow_turns=1.0),
                                dict(scaling="bands", factor=2.0, trained_length=9.0, slow_turns=-1.0)])
def test_frequency_refusals(kw):
    _lib()
    with pytest.raises(fdb.FlashDecoderError) as e:
        fdb.fd_rope_frequencies(**{"rot_dim": 64, **kw})
    assert e.value.status == INVALID
    with pytest.raises(ValueError):
        fdb.fd_rope_frequencies(64, scaling="other")


# plausible device addresses: every call below is refused, or has nothing to do, before they are used
A = 1 << 20


def _rope(**kw):
    s = fdb.fd_rope(ctypes.sizeof(fdb.fd_rope), 64, 0, 1, A, None, 1.0, 0)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _rope_call(lib, rope=None, x=A, dtype=2, tokens=4, heads=2, dim=64, xt=128, xh=64, coords=A, out=A, ot=128, oh=64):
    r = _rope() if rope is None else rope
    return lib.fd_rope_device(ctypes.byref(r), x, dtype, tokens, heads, dim, xt, xh, coords, out, ot, oh, None)


def test_struct_sizes():
    assert ctypes.sizeof(fdb.fd_rope) == 40
    assert ctypes.sizeof(fdb.fd_token_cache) == 104


def test_rope_refusals():
    lib = _lib()
    assert lib.fd_rope_device(None, A, 2, 4, 2, 64, 128, 64, A, A, 128, 64, None) == INVALID
    for kw in (dict(struct_size=8), dict(rot_dim=-2), dict(rot_dim=63), dict(rot_dim=66), dict(layout=2),
               dict(n_axes=0), dict(n_axes=5), dict(freq=None), dict(freq=A + 4), dict(axis=A + 2),
               dict(magnitude=math.nan), dict(magnitude=math.inf)):
        assert _rope_call(lib, _rope(**kw)) == INVALID, kw
    for kw in (dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(tokens=2 ** 31), dict(heads=0), dict(heads=65537),
               dict(dim=0), dict(dim=513), dict(xt=-1), dict(ot=63), dict(oh=63), dict(xh=1 << 48), dict(x=None),
               dict(out=None), dict(coords=None), dict(x=A + 1), dict(coords=A + 2), dict(xt=256)):
        assert _rope_call(lib, **kw) == INVALID, kw
    assert lib.fd_last_error()
    assert _rope_call(lib, tokens=0, x=None, out=None, coords=None) == fdb.FD_OK


def _slots_call(lib, at=A, w=A, B=2, G=2, C=16, pos=A, n=4, first=0, recent=0, out=A, ws=None, size=0):
    return lib.fd_token_slots_device(at, w, B, G, C, pos, n, first, recent, out, ws, size, None)


def test_slots_refusals():
    lib = _lib()
    for kw in (dict(B=0), dict(G=0), dict(C=0), dict(n=-1), dict(n=17), dict(C=1 << 20, n=65537), dict(first=-1),
               dict(recent=-1), dict(at=None), dict(w=None), dict(pos=None), dict(out=None), dict(at=A + 1),
               dict(out=A + 2)):
        assert _slots_call(lib, **kw) == INVALID, kw
    for kw in (dict(C=(1 << 24) + 1), dict(B=256, G=256)):
        assert _slots_call(lib, **kw) == UNSUPPORTED, kw
    assert _slots_call(lib, n=0, at=None) == fdb.FD_OK
    size = ctypes.c_size_t()
    for args, need in (((2, 2, 16384, 99), 0), ((2, 2, 16385, 1), 0), ((2, 2, 40000, 100), 4 * 3 * 100 * 4),
                       ((1, 1, 40000, 30000), 0)):
        assert lib.fd_token_slots_workspace(*args, ctypes.byref(size)) == fdb.FD_OK and size.value == need, args
    assert lib.fd_token_slots_workspace(2, 2, 40000, 100, None) == INVALID
    assert lib.fd_token_slots_workspace(2, 2, 100, 101, ctypes.byref(size)) == INVALID
    assert lib.fd_token_slots_workspace(2, 2, (1 << 24) + 1, 1, ctypes.byref(size)) == UNSUPPORTED
    for kw in (dict(ws=None), dict(ws=A, size=4799), dict(ws=A + 2, size=4800)):
        assert _slots_call(lib, C=40000, n=100, **kw) == INVALID, kw


def cache_struct(**kw):
    I3 = ctypes.c_int64 * 3
    s = fdb.fd_token_cache(ctypes.sizeof(fdb.fd_token_cache), 1, 2, 2, 16, 64, A, A, I3(2048, 1024, 64),
                           I3(2048, 1024, 64), A, A)
    for k, v in kw.items():
        setattr(s, k, I3(*v) if isinstance(v, tuple) else v)
    return s


BAD_CACHES = [(dict(struct_size=1), INVALID), (dict(dtype=3), INVALID), (dict(batch=0), INVALID),
              (dict(groups=-1), INVALID), (dict(capacity=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
              (dict(head_dim=256), UNSUPPORTED), (dict(capacity=(1 << 24) + 1), UNSUPPORTED),
              (dict(batch=256, groups=256), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=None), INVALID),
              (dict(pos=None), INVALID), (dict(weight=None), INVALID), (dict(k=A + 8), INVALID),
              (dict(v=A + 2), INVALID), (dict(pos=A + 1), INVALID), (dict(k_stride=(2048, 1024, 63)), INVALID),
              (dict(k_stride=(2048, 1024, 68)), INVALID), (dict(v_stride=(0, 1024, 64)), INVALID),
              (dict(v_stride=(2048, -1024, 64)), INVALID), (dict(v_stride=(1 << 48, 1024, 64)), INVALID),
              (dict(v_stride=(1 << 40, 1 << 30, 1 << 23)), UNSUPPORTED)]


def _append_call(lib, cache=None, rope=None, k=A, ks=(512, 128, 64), v=A, vs=(512, 128, 64), n=4, pos=A, coords=None,
                 slots=A):
    I3 = ctypes.c_int64 * 3
    c = cache_struct() if cache is None else cache
    return lib.fd_token_append_device(ctypes.byref(c), None if rope is None else ctypes.byref(rope), k,
                                      I3(*ks) if ks else None, v, I3(*vs) if vs else None, n, pos, coords, slots, None)


def test_append_refusals():
    lib = _lib()
    I3 = ctypes.c_int64 * 3
    assert lib.fd_token_append_device(None, None, A, I3(), A, I3(), 1, A, None, A, None) == INVALID
    for kw, status in BAD_CACHES:
        assert _append_call(lib, cache_struct(**kw)) == status, kw
    for kw in (dict(n=-1), dict(n=2 ** 31 - 1), dict(k=None), dict(v=None), dict(ks=None), dict(vs=None),
               dict(pos=None), dict(slots=None), dict(k=A + 8), dict(v=A + 4), dict(pos=A + 1), dict(coords=A + 2),
               dict(ks=(512, 128, 60)), dict(vs=(512, 130, 64)), dict(rope=_rope(rot_dim=66)),
               dict(rope=_rope(n_axes=3))):
        assert _append_call(lib, **kw) == INVALID, kw
    assert _append_call(lib, n=0, k=None, slots=None) == fdb.FD_OK


def _attend_call(lib, cache=None, q=A, qs=(1024, 256, 64), heads=4, n=3, pos=A, scale=0.125, causal=1, out=A,
                 os_=(1024, 256, 64), lse=A, decay=1.0, w=A, ws=A, size=1 << 40):
    I3 = ctypes.c_int64 * 3
    c = cache_struct() if cache is None else cache
    return lib.fd_token_attend_device(ctypes.byref(c), q, I3(*qs) if qs else None, heads, n, pos, scale, causal, out,
                                      I3(*os_) if os_ else None, lse, decay, w, ws, size, None)


def test_attend_refusals():
    lib = _lib()
    size = ctypes.c_size_t()
    for kw, status in BAD_CACHES:
        assert _attend_call(lib, cache_struct(**kw)) == status, kw
        assert lib.fd_token_attend_workspace(ctypes.byref(cache_struct(**kw)), 4, 3, 1, ctypes.byref(size)) == status
    c = cache_struct()
    assert lib.fd_token_attend_workspace(ctypes.byref(c), 4, 3, 1, None) == INVALID
    assert lib.fd_token_attend_workspace(ctypes.byref(c), 3, 3, 1, ctypes.byref(size)) == INVALID
    assert lib.fd_token_attend_workspace(ctypes.byref(c), 4, 0, 1, ctypes.byref(size)) == fdb.FD_OK and size.value == 0
    assert lib.fd_token_attend_workspace(ctypes.byref(c), 4, 3, 1, ctypes.byref(size)) == fdb.FD_OK and size.value > 0
    need = size.value
    for kw in (dict(heads=0), dict(heads=3), dict(heads=-2), dict(n=-1), dict(q=None), dict(out=None), dict(pos=None),
               dict(qs=None), dict(os_=None), dict(q=A + 8), dict(out=A + 2), dict(pos=A + 1), dict(lse=A + 2),
               dict(w=A + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
               dict(decay=math.inf), dict(decay=math.nan), dict(qs=(1024, 256, 60)), dict(qs=(1024, 0, 64)),
               dict(os_=(1024, 250, 64)), dict(ws=None), dict(ws=A + 8), dict(size=need - 1), dict(size=0)):
        assert _attend_call(lib, **kw) == INVALID, kw
    for kw in (dict(heads=4, n=1 << 24), dict(heads=514, n=1)):
        assert _attend_call(lib, **kw) == UNSUPPORTED, kw
    huge = cache_struct(batch=300, groups=200, capacity=1 << 20, k_stride=(1 << 40, 1 << 30, 64),
                        v_stride=(1 << 40, 1 << 30, 64))
    assert _attend_call(lib, huge, heads=200) == UNSUPPORTED
    assert _attend_call(lib, n=0, q=None, ws=None, w=None) in (fdb.FD_OK, fdb.FD_ERR_DEVICE)  # nothing to launch


def test_binding_refusals():
    """Wrong tensors are refused before anything reaches the library."""
    _lib()
    f64 = torch.ones(32, dtype=torch.float64)
    with pytest.raises(ValueError):
        fdb.Rope(f64)  # not on a GPU
    with pytest.raises(ValueError):
        fdb.Rope(f64, layout="other")
    k = torch.zeros(1, 1, 4, 64)
    with pytest.raises(ValueError):
        fdb.TokenCache(k, k, torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(1, 1, 4))
    with pytest.raises(ValueError):
        fdb.TokenCache(k.double(), k.double(), torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(1, 1, 4))
    z = torch.zeros(1, 1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        fdb.fd_token_slots_device(z, torch.zeros(1, 1, 4), z[0], z)
