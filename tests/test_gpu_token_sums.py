"""Attention over very long token caches, and of very many rows: sums in fp32 that do not lose to their length.

Every slot holds the same value, and its score is 0 in one slot of 32 and -d in the others, so that the results
are known in closed form at any length. Equal terms added one by one are the worst case of a running sum: over
2^19 of them it is off by up to 5e-3.
"""
import math

import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = 2.0 ** -24
D = 32


def _cache(G, C, dtype, d, values):
    """Groups one slot apart in one buffer: 16-byte strides of any size are allowed where nothing is written."""
    k = torch.zeros(C + G, D, device="cuda", dtype=dtype)
    k[:, 0] = -d
    k[::32, 0] = 0
    v = values.cuda().to(dtype).expand(C + G, D).contiguous()
    k, v = (torch.as_strided(t, (1, G, C, D), (C * D, D, D, 1)) for t in (k, v))
    return fdb.TokenCache(k, v, torch.zeros(1, G, C, dtype=torch.int32, device="cuda"),
                          torch.zeros(1, G, C, device="cuda"))


def _queries(n, heads, dtype):
    q = torch.zeros(1, n, heads, D, device="cuda", dtype=dtype)
    q[..., 0] = 1
    return q, torch.zeros(1, n, dtype=torch.int32, device="cuda")


def _check(out, lse, values, C, d, dtype, adds, steps):
    """adds: roundings that a probability's share of the row sum passes; steps: those of a product in P V."""
    total = C / 32 * (1 + 31 * math.exp(-d))
    # exp2 within two steps, its argument rounded twice (score times log2 e, and the shift)
    ex = 2 * U * 2 + 4 * U * (d + 8)
    tol = ex + adds * U
    assert float((lse.double() - math.log(total)).abs().max()) <= tol + 4 * U * math.log(total)
    want = values.to(dtype).double()
    half = torch.finfo(dtype).eps / 2
    # all probabilities are 1 or e^-d: their rounding to 16 bits (chunks) may be as large for every slot
    err = want.abs() * (2 * tol + steps * U + (half if dtype != F32 else 0) + half)
    assert bool(((out.double().cpu() - want).abs().amax((0, 1, 2)) <= err).all())
    return total, tol


VALUES = torch.tensor([1.0 + i / 37.0 for i in range(D)])


@pytest.mark.parametrize("dtype,C", [(BF16, 2 ** 20), (F16, 2 ** 19 + 77 * 32), (F32, 2 ** 18)])
def test_chunks_over_long_caches(dtype, C):
    n, heads, d = 16384, 4, 0.6875  # 512 tiles of rows: no parts
    cache = _cache(1, C, dtype, d, VALUES)
    q, pos = _queries(n, heads, dtype)
    out, lse = cache.attend(q, pos, scale=1.0, causal=False, track=False)
    # 32 keys of a tile in a lane, 256 tiles to a fold (4096 slots: 128 of 32), the folds, two halves; fp32 MFMAs take
    # keys one by one, 16-bit ones 16 at a time
    fold = 4096 if dtype == F32 else 16384
    adds = 32 + 256 + -(-C // fold) + 2
    _check(out, lse, VALUES, C, d, dtype, adds, fold + -(-C // fold) + 8)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_single_tokens_over_long_caches(dtype):
    G, C, d = 768, 2 ** 18, 0.6875  # more groups than workgroups fit: parts only for their length
    cache = _cache(G, C, dtype, d, VALUES)
    q, pos = _queries(1, G, dtype)
    w = torch.empty_like(cache.weight)
    out, lse = cache.attend(q, pos, scale=1.0, weight_out=w)
    # 4096 slots of a wave: 16 keys of a tile in a lane, 128 tiles, 4 waves and two halves, 16 parts
    total, tol = _check(out, lse, VALUES, C, d, dtype, 16 + 128 + 8 + 16, 4096 + 8 + 16)
    for g in (0, 5, 767):
        k = cache.k[0, g, :, 0].double()
        want = torch.exp(k) / total
        assert float(((w[0, g].double() - want) / want).abs().max()) <= 2 * tol + 4 * U * (d + math.log2(total)) + 4 * U


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_of_many_rows(dtype):
    n, heads, d = 2 ** 18, 4, 0.6875
    C = 196608 if dtype == BF16 else 98304  # as many workgroups as fit: parts of the rows only for their length
    cache = _cache(1, C, dtype, d, VALUES)
    q, pos = _queries(n, heads, dtype)
    out, lse = cache.attend(q, pos, scale=1.0, causal=False)
    fold = 4096 if dtype == F32 else 16384
    total, tol = _check(out[:, :1024], lse[..., :1024], VALUES, C, d, dtype, 32 + 256 + -(-C // fold) + 2, fold + 64)
    want = n * heads * torch.exp(cache.k[0, 0, :, 0].double()) / total
    # 1024 rows of a lane in a part, 32 lanes (5 steps), 32 parts
    err = 2 * tol + 4 * U * (d + math.log2(total)) + (1024 + 5 + 32 + 4) * U
    assert float(((cache.weight[0, 0].double() - want) / want).abs().max()) <= err
