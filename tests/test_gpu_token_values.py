"""Attention over a token cache whose values are not finite, or as large as the type allows: what a row
gets may not depend on how the slots are parted among waves and workgroups."""
import math

import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _steep(n, C, dtype, low=-200.0, N=3, D=64):
    """One group whose slots from 32 on score `low` against every query, the first 32 zero: slot s lies at
    position s; the first half of the tokens sees all but the last slot, the second half all."""
    gen = torch.Generator().manual_seed(C + n)
    k = torch.zeros(1, 1, C, D)
    k[..., 32:, 0] = low
    v = torch.randn(1, 1, C, D, generator=gen)
    q = torch.zeros(1, n, N, D)
    q[..., 0] = 1.0
    at = torch.arange(C, dtype=torch.int32).view(1, 1, C)
    pos = torch.where(torch.arange(n) < n // 2, C - 2, C - 1).to(torch.int32).view(1, n)
    return [t.cuda() for t in (k.to(dtype), v.to(dtype), at, torch.zeros(1, 1, C), q.to(dtype), pos)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("C", [65, 230, 9000])
@pytest.mark.parametrize("track", [False, True])
def test_values_that_are_not_finite_far_below_the_maximum(dtype, n, C, track):
    """Probabilities are positive, so an infinity or a NaN among a row's values reaches it, however small the
    probability and whichever wave or part holds it."""
    k, v, at, weight, q, pos = _steep(n, C, dtype)
    want = v[0, 0, :32].double().mean(0).cpu()  # e^-200 of the others is below half a step of any type
    v[0, 0, 33, 1] = INF
    v[0, 0, C // 2, 2] = -INF
    v[0, 0, C // 2, 3] = NAN
    v[0, 0, 33, 4], v[0, 0, C // 2, 4] = INF, -INF
    v[0, 0, C - 1, 5] = NAN  # seen by the later tokens alone
    v[0, 0, C - 1, 6] = INF
    cache = fdb.TokenCache(k, v, at, weight)
    out, lse = cache.attend(q, pos, scale=1.0, causal=True, track=track)
    out = out[0].cpu().double()
    assert bool((out[..., 1] == INF).all()) and bool((out[..., 2] == -INF).all())
    assert bool(out[..., 3].isnan().all()) and bool(out[..., 4].isnan().all())
    assert bool(out[n // 2:, :, 5].isnan().all()) and bool((out[n // 2:, :, 6] == INF).all())
    # equal probabilities 1 / 32 of 32 values: exact but for 32 sums in fp32, the division and the output's rounding
    half = torch.finfo(dtype).eps / 2
    tol = 34 * 2.0 ** -24 * v[0, 0, :32].double().abs().mean(0).cpu() + half * want.abs() + torch.finfo(dtype).tiny
    fine = [0, *range(7, 64)]
    assert bool(((out - want).abs() <= tol)[..., fine].all())
    early = ((out - want).abs() <= tol)[: n // 2]
    assert bool(early[..., 5:7].all())
    tol_lse = 34 * 2.0 ** -24 + 4 * 2.0 ** -24 * math.log(32)
    assert float((lse.double() - math.log(32)).abs().max()) <= tol_lse


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("C", [64, 700, 9000])
def test_values_near_the_largest(dtype, n, C):
    """Values up to a quarter of the type's largest: their weighted mean is finite, and so is the result, whatever
    the sums before the division would come to."""
    D, N = 64, 3
    gen = torch.Generator().manual_seed(C + n)
    k = torch.zeros(1, 1, C, D)
    k[..., 0] = torch.randint(-40, 41, (C,), generator=gen) / 8.0  # exact in every type, as are the products below
    v = (0.25 + 0.75 * torch.rand(1, 1, C, D, generator=gen)) * (torch.finfo(dtype).max / 4)
    v[..., 32:] *= -1
    k, v = k.to(dtype), v.to(dtype)
    q = torch.zeros(1, n, N, D)
    q[..., 0] = torch.tensor([0.0, 1.0, -0.5])
    at, pos = torch.zeros(1, 1, C, dtype=torch.int32), torch.zeros(1, n, dtype=torch.int32)
    x = torch.tensor([0.0, 1.0, -0.5]).double()[:, None] * k[0, 0, :, 0].double()
    p, vd = torch.softmax(x, -1), v[0, 0].double()
    want = p @ vd
    # as for ordinary values: scaled scores and log-sum, C + 32 sums and products in fp32, probabilities and the
    # output rounded to the type
    u, half = 2.0 ** -24, torch.finfo(dtype).eps / 2
    rel = 2 * (4 * u * (5 + 8)) + (C + 32) * u
    tol = (p @ vd.abs()) * (rel + (half if dtype != F32 else u)) + half * want.abs()
    for track in (False, True):
        cache = fdb.TokenCache(k.cuda(), v.cuda(), at.cuda(), torch.zeros(1, 1, C).cuda())
        out, lse = cache.attend(q.to(dtype).cuda(), pos.cuda(), scale=1.0, track=track)
        assert bool(((out[0].cpu().double() - want).abs() <= tol).all())
        assert float((lse[0].cpu().double() - torch.logsumexp(x, -1)[:, None]).abs().max()) <= rel + 4 * u * 20
        if track:
            total = n * p.sum(0)
            assert bool(((cache.weight[0, 0].cpu().double() - total).abs() <= total * (2 * rel + (3 * n + 8) * u)).all())
