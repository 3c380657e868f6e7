"""Every variant that the token attention's and the choice of slots' plans can pick, at sizes that pick it: what the
workspace's size says of the plan is checked beside the results, which are compared in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2607_14898_amd import flashdecoder as fdb
from tests.test_gpu_token_cache import _slots
from tests.test_token_plan_host import parts_floats, up64, workspace

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
NAMES = {F16: "f16", BF16: "bf16", F32: "f32"}
U = 2.0 ** -24
INF = math.inf


def make(B, G, N, D, n, C, dtype, seed=0, fill=0.95, rise=0.0):
    """Slots at random positions, some empty and holding NaN; tokens across the range of positions, one of seven
    padding; rise: how far the scores climb along the slots."""
    gen = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    k, v, q = rnd(B, G, C, D).to(dtype), rnd(B, G, C, D).to(dtype), rnd(B, n, N, D).to(dtype)
    at = torch.randint(0, 2 * C, (B, G, C), generator=gen, device="cuda", dtype=torch.int32)
    at[torch.rand(B, G, C, generator=gen, device="cuda") > fill] = -1
    pos = torch.randint(0, 2 * C, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    if rise:
        k[..., 0] = (torch.arange(C, device="cuda") / C * rise).to(dtype)
        q[..., 0] = D ** 0.5
    if n > 1:
        pos[:, ::7] = -1
    empty = at < 0
    k[empty], v[empty] = math.nan, INF
    weight = torch.rand(B, G, C, generator=gen, device="cuda")
    weight[empty] = math.nan
    return k, v, at, weight, q, pos


def ref(k, v, at, weight, q, pos, scale, causal, decay):
    """(out, lse, weight) in 64 bits and bounds on the error of the library's arithmetic, a group at a time."""
    B, G, C, D = k.shape
    n, N = q.shape[1], q.shape[2]
    h = N // G
    half = torch.finfo(q.dtype).eps / 2
    sharp = half if q.dtype != F32 else U  # (chunks: probabilities rounded to the cache's type)
    if n * h <= 64 and q.dtype != F32:
        sharp = half * half  # single tokens: as a sum of two such values
    out, lse = torch.zeros(B, n, N, D, dtype=torch.float64, device="cuda"), torch.zeros(B, N, n, dtype=torch.float64, device="cuda")
    t_out, t_lse = torch.zeros_like(out), torch.zeros_like(lse)
    w, t_w = torch.zeros(weight.shape, dtype=torch.float64, device="cuda"), torch.zeros(weight.shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        for g in range(G):
            some = at[b, g] >= 0
            kk, vv = (torch.where(some[:, None], t[b, g].double(), 0.0) for t in (k, v))
            qq = q[b, :, g * h:(g + 1) * h].double().reshape(n * h, D)
            see = (some[None] & (pos[b] >= 0)[:, None])
            if causal:
                see = see & (at[b, g][None] <= pos[b][:, None])
            see = see.repeat_interleave(h, 0)
            x = (qq @ kk.T.contiguous() * scale).masked_fill(~see, -INF)
            big = (qq.abs() @ kk.abs().T.contiguous() * scale).masked_fill(~see, 0.0).amax(-1)
            top = x.amax(-1)
            none = top == -INF
            l = torch.logsumexp(x, -1)
            p = torch.exp(x - torch.where(none, 0.0, l)[:, None])
            o, spread = p @ vv, p @ vv.abs()
            # scores: D products summed in fp32, three roundings of the scaled score, one of the log-sum it is taken
            # from; exp2 and log2 within two steps; sums over the slots in fp32
            seen = see.sum(-1)
            ex = (D + 3) * U * big + 4 * U * (x.masked_fill(~see, 0.0).abs().amax(-1) + 8)
            rel = torch.where(none, 0.0, 2 * ex + (seen + 32) * U)
            t_o = spread * (rel + sharp)[:, None] + (seen * 2.0 ** -31)[:, None] * vv.abs().max() + half * o.abs() \
                + torch.finfo(q.dtype).tiny
            t_l = torch.where(none, 0.0, ex + (seen + 24) * U + 4 * U * torch.where(none, 0.0, l).abs())
            heads = slice(g * h, (g + 1) * h)
            out[b, :, heads], t_out[b, :, heads] = o.view(n, h, D), t_o.view(n, h, D)
            lse[b, heads], t_lse[b, heads] = l.view(n, h).T, t_l.view(n, h).T
            old = torch.where(some, decay * weight[b, g].double().nan_to_num(0.0), 0.0)
            w[b, g] = torch.where(some, old + p.sum(0), 0.0)
            t_w[b, g] = (p * (rel + 8 * U)[:, None]).sum(0) + (2 + n * h) * U * w[b, g].abs()
    return (out, lse, w), (t_out, t_lse, t_w)


def near(got, want, tol, name):
    got = got.double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    bad = ~((got - want).abs() <= tol) & ~inf
    assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


def check(k, v, at, weight, q, pos, causal=True, decay=0.75):
    scale = q.shape[-1] ** -0.5
    cache = fdb.TokenCache(k, v, at, weight)
    w = torch.full_like(weight, math.nan)
    out, lse = cache.attend(q, pos, causal=causal, decay=decay, weight_out=w)
    want, tol = ref(k, v, at, weight, q, pos, float(np.float32(scale)), causal, float(np.float32(decay)))
    near(out, want[0], tol[0], "out")
    near(lse, want[1], tol[1], "lse")
    near(w, want[2], tol[2], "weight")
    out2, lse2 = cache.attend(q, pos, causal=causal, track=False)
    near(out2, want[0], tol[0], "out without weights")
    near(lse2, want[1], tol[1], "lse without weights")
    again = torch.empty_like(w)
    out3, lse3 = cache.attend(q, pos, causal=causal, decay=decay, weight_out=again)
    assert torch.equal(out3, out) and torch.equal(lse3, lse) and torch.equal(again, w)
    return out, want[0], tol[0]


TYPES = [(F16, 64), (F16, 128), (BF16, 32), (BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)]


@pytest.mark.parametrize("dtype,D", TYPES)
def test_weights_written_by_one_wave(dtype, D):
    """One part of slots and of rows, a wave's keys to itself: weights go straight to the cache."""
    B, G, N, n, C = 64, 8, 32, 20, 500
    assert workspace(B, G, C, D, N, n, NAMES[dtype], 0) == 0
    assert workspace(B, G, C, D, N, n, NAMES[dtype]) == up64(B * G * n * N // G)
    check(*make(B, G, N, D, n, C, dtype, seed=D))


@pytest.mark.parametrize("dtype,D", TYPES)
def test_weights_from_parts_of_the_rows(dtype, D):
    B, G, N, n, C = 1, 2, 8, 330, 700
    R, name = n * N // G, NAMES[dtype]
    extra = workspace(B, G, C, D, N, n, name) - workspace(B, G, C, D, N, n, name, 0) - up64(G * R)
    assert extra > 0 and extra == up64(G * (R // 256) * C)
    check(*make(B, G, N, D, n, C, dtype, seed=D), causal=D != 64)


@pytest.mark.parametrize("dtype,D", TYPES)
def test_few_rows_of_many_slots(dtype, D):
    """Weights four slots a thread (2^19 slots and more in all)."""
    B, G, N, n, C = 16, 8, 24, 1, 4099
    check(*make(B, G, N, D, n, C, dtype, seed=D, fill=0.7))


@pytest.mark.parametrize("dtype,D", TYPES)
def test_few_rows_in_many_parts(dtype, D):
    """More than 64 parts of the slots; 33 to 64 rows, in two tiles."""
    for N, n in ((4, 1), (7, 7)):
        B, G, C = 1, 1, 20000
        got = workspace(B, G, C, D, N, n, NAMES[dtype], 0)
        assert got > parts_floats(1, 64, N * n, D)
        check(*make(B, G, N, D, n, C, dtype, seed=D + n, rise=9.0))


@pytest.mark.parametrize("dtype,D,C", [(F16, 64, 9000), (BF16, 128, 9000), (BF16, 32, 17000), (F32, 64, 9000),
                                       (F32, 128, 4500)])
def test_chunks_of_several_scans(dtype, D, C):
    """One part of several ranges of 4096 slots, with folds of the sums in between from 16384 (fp32: 4096) slots on;
    the scores climb, so that the shift is another one at every fold."""
    B, G, N, n = 128, 4, 4, 70
    assert (workspace(B, G, C, D, N, n, NAMES[dtype], 0) > 0) == (C > (4096 if dtype == F32 else 16384))
    k, v, at, weight, q, pos = make(B, G, N, D, n, C, dtype, seed=C, rise=40.0)
    few = [t[:1].contiguous() for t in (k, v, at, weight, q, pos)]
    # (the reference for one request in 128: the rest has the same plan and is compared among itself)
    k[1:], v[1:], at[1:], weight[1:], q[1:], pos[1:] = (t.expand_as(full[1:]) for t, full in
                                                        zip(few, (k, v, at, weight, q, pos)))
    cache = fdb.TokenCache(k, v, at, weight)
    w = torch.empty_like(weight)
    out, lse = cache.attend(q, pos, weight_out=w, decay=0.75)
    want, tol = ref(*few, float(np.float32(D ** -0.5)), True, 0.75)
    near(out[:1], want[0], tol[0], "out")
    near(lse[:1], want[1], tol[1], "lse")
    near(w[:1], want[2], tol[2], "weight")
    assert torch.equal(out[1:], out[:1].expand_as(out[1:])) and torch.equal(w[1:], w[:1].expand_as(w[1:]))
    # values that are not finite, first and last range: what a row sees reaches it, the rest does not
    some = (at[0, 0] >= 0).nonzero()[:, 0].tolist()
    slot = {3: some[5], 7: some[-5], 11: some[len(some) // 2]}
    v[:, 0, slot[3], 3], v[:, 0, slot[7], 7], v[:, 0, slot[11], 11] = INF, -INF, math.nan
    out2, _ = cache.attend(q, pos, track=False)
    assert torch.equal(out2[1:].nan_to_num(3.0), out2[:1].expand_as(out2[1:]).nan_to_num(3.0))
    got = out2[0].double()
    for d, s in slot.items():
        sees = pos[0] >= at[0, 0, s]
        assert bool(sees.any()) and not bool(sees.all())
        mine = got[sees, 0, d]
        assert bool((mine == INF).all() if d == 3 else (mine == -INF).all() if d == 7 else mine.isnan().all())
    hit = torch.zeros_like(got, dtype=torch.bool)
    for d, s in slot.items():
        hit[pos[0] >= at[0, 0, s], 0, d] = True
    assert bool((((got - want[0][0]).abs() <= tol[0][0]) | hit).all())


# (sizes at which the bound of the sums, C half steps of fp32, leaves one rounding to the type visible)
@pytest.mark.parametrize("dtype,n,C", [(F16, 1, 64), (F16, 4, 64), (F16, 8, 40), (BF16, 1, 64), (BF16, 4, 64),
                                       (BF16, 8, 290), (BF16, 1, 700)])
def test_few_rows_keep_more_than_one_rounding_of_their_probabilities(dtype, n, C):
    """Values of both signs, so that the output is far below what is added up and its own rounding hides nothing.
    Queries of one dimension make the scores exact."""
    D, N = 128, 8
    gen = torch.Generator().manual_seed(C + n)
    k = torch.zeros(1, 1, C, D)
    k[..., 0] = torch.randint(-64, 65, (C,), generator=gen) / 64.0
    q = torch.zeros(1, n, N, D)
    q[..., 0] = torch.randint(1, 17, (n, N), generator=gen) / 8.0
    v = (torch.rand(1, 1, C, D, generator=gen) + 0.5) * (torch.randint(0, 2, (1, 1, C, D), generator=gen) * 2 - 1)
    v = v.to(dtype)
    x = (q[0, :, :, 0, None] * k[0, 0, :, 0]).double()
    vd, p = v[0, 0].double(), torch.softmax(x, -1)
    want, spread = p @ vd, p @ vd.abs()
    half = torch.finfo(dtype).eps / 2
    rel = 2 * 4 * U * (2 + 8) + (C + 32) * U
    tol = spread * (rel + half * half) + C * 2.0 ** -31 * 1.5 + half * want.abs()
    # the bound tells probabilities rounded once from these: their error passes it somewhere (in the oracle)
    e = torch.exp(x - x.amax(-1, keepdim=True))
    once = e.to(dtype).double() @ vd / e.sum(-1, keepdim=True)
    assert bool(((once - want).abs() > tol).any())
    at, pos = torch.zeros(1, 1, C, dtype=torch.int32), torch.zeros(1, n, dtype=torch.int32)
    for track in (False, True):
        cache = fdb.TokenCache(k.to(dtype).cuda(), v.cuda(), at.cuda(), torch.zeros(1, 1, C).cuda())
        out, _ = cache.attend(q.to(dtype).cuda(), pos.cuda(), scale=1.0, track=track)
        assert bool(((out[0].cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("C,n", [(65536, 5000), (131072, 8192), (40000, 9000)])
@pytest.mark.parametrize("ties", [False, True])
def test_choice_among_more_candidates_than_registers_hold(C, n, ties):
    """A second launch over more than 16384 of the chunks' choices, and a choice that chunks would not shorten."""
    chunks = -(-C // 16384)
    assert chunks * n > 16384
    r = np.random.default_rng(C + n)
    B, G = 2, 2
    at = np.stack([r.permutation(2 * C)[:C] for _ in range(B * G)]).reshape(B, G, C).astype(np.int32)
    at[0, 1, r.random(C) < 0.05] = -1
    weight = r.integers(0, 3, (B, G, C)).astype(np.float32) if ties else r.gamma(0.3, 1.0, (B, G, C)).astype(np.float32)
    weight[1, 0, r.random(C) < 0.01] = np.nan
    pos = np.broadcast_to(2 * C + np.arange(n), (B, n)).astype(np.int32).copy()
    pos[1, r.random(n) < 0.3] = -1
    first, recent = 9, C // 2
    got = _slots(at, weight, pos, first, recent)
    for b in range(B):
        valid = np.nonzero(pos[b] >= 0)[0]
        newest = int(pos[b].max())
        for g in range(G):
            p, w = at[b, g].astype(np.int64), weight[b, g].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            kind = np.where(p < 0, 0, np.where(p < first, 3, np.where(p > newest - recent, 2, 1)))
            order = np.lexsort((np.arange(C), np.where(kind > 0, w, 0.0), kind))
            want = np.full(n, -1)
            want[valid] = np.sort(order[: len(valid)])
            assert np.array_equal(got[b, g], want), (b, g)


@pytest.mark.parametrize("B,G,C", [(1, 1, 131072), (2, 3, 150001), (1, 2, 1 << 20), (8, 4, 131100), (33, 2, 131100), (2, 2, 3000),
                                   (2, 2, 4097)])
def test_one_token_among_many_slots(B, G, C):
    """In one launch and in chunks, with ties, empty slots and padding."""
    r = np.random.default_rng(C)
    at = r.integers(0, 2 * C, (B, G, C)).astype(np.int32)
    weight = r.integers(1, 50, (B, G, C)).astype(np.float32)
    weight[0, 0, C - 1] = 0.0
    if G > 1:
        at[:, 1, C - 2] = -1
        weight[0, 1, C // 2] = np.nan
    pos = np.full((B, 1), 2 * C, np.int32)
    pos[B // 2 if B > 1 else 1:] = -1
    for first, recent in ((3, C // 2), (0, 0), (2 * C, 0)):
        got = _slots(at, weight, pos, first, recent)
        for b in range(B):
            for g in range(G):
                if pos[b, 0] < 0:
                    assert got[b, g, 0] == -1
                    continue
                p, w = at[b, g].astype(np.int64), weight[b, g].astype(np.float64)
                kind = np.where(p < 0, 0, np.where(p < first, 3, np.where(p > 2 * C - recent, 2, 1)))
                w = np.where(kind > 0, np.where(np.isnan(w), -np.inf, w), 0.0)
                assert got[b, g, 0] == np.lexsort((np.arange(C), w, kind))[0], (b, g, first)
