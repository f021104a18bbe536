"""Chunked attention over the 4-bit cache, the attention weight its tokens receive and eviction, on a B200 against plain 64-bit forms.

Tolerances count roundings: half a step of a type relative to the value is U[type] = finfo.eps / 2; sums of n terms in fp32
are off by at most n U[f32] times the sum of the terms' sizes; ex2.approx and the reciprocal by 2 U[f32]."""
import math

import pytest
import torch

import serving_reference as R
from test_serving_gpu import DEV, SHAPES, U, U32, S, filled_cache, gen, randn, table_of, within  # noqa: F401

pytestmark = pytest.mark.gpu
U16 = torch.finfo(torch.float16).eps / 2
BF = torch.bfloat16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def held(cache, table, i, m):
    """Keys and values of the first m tokens of sequence i, in 64 bits [m, heads, D]."""
    pages = table[i, :-(-m // cache.page_size)].long()
    return [R.values(c[pages].transpose(1, 2).flatten(0, 1)[:m], p[pages].transpose(1, 2).flatten(0, 1)[:m])[0]
            for c, p in ((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params))]


# ------------------------------------------------------------------------------------------------ reading into outputs made there
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("tokens", [1, 7, 701])
def test_read_makes_outputs_of_zeros_where_there_is_no_slot(S, dtype, d, group, tokens):
    g = gen(tokens)
    cache = filled_cache(S, 6, 16, 3, d, group, g)
    slots = torch.randint(-40, 96, (tokens,), generator=g, device=g.device).to(DEV)
    for beyond in (False, True):
        if beyond:
            slots[tokens // 2] = 96
        spoiled = [torch.full((tokens, 3, d), math.nan, dtype=dtype, device=DEV) for _ in range(2)]       # what the allocator hands out next
        del spoiled
        k, v = cache.read(slots, dtype)
        ko, vo = (torch.zeros(tokens, 3, d, dtype=dtype, device=DEV) for _ in range(2))
        cache.read(slots, k_out=ko, v_out=vo)
        assert torch.equal(k, ko) and torch.equal(v, vo) and (k[(slots < 0) | (slots >= 96)] == 0).all()
        if beyond:
            with pytest.raises(S.GcError, match="slot"):
                cache.query_status()
        else:
            cache.query_status()
        ko.fill_(3.0)
        cache.read(slots.clamp(max=95), k_out=ko)                # rows of a given output stay as they were
        assert (ko[slots < 0] == 3).all()


# ------------------------------------------------------------------------------------------------ chunks
def chunk_reference(cache, q, new, table, lens, scale):
    """q [tokens, heads, D] -> (o, tolerance) for the rows that sequences own."""
    g = q.shape[1] // cache.kv_heads
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(o)
    a = 0
    for i, (n, m) in enumerate(zip(new, lens)):
        if n and m:
            k, v = held(cache, table, i, m)
            lim = (torch.arange(n, device=DEV) + m - n + 1).clamp(min=0)
            for h in range(q.shape[1]):
                qq, kk, vv = q[a:a + n, h].double(), k[:, h // g], v[:, h // g]
                ref, size = R.head_all(qq, kk, vv, lim, scale)
                # Scores: keys rounded to fp16, half a step each, and a sum of D products in fp32.  A weight is off by that and by its
                # exponent's own rounding (a product, a sum and the reference, of numbers up to the largest score); all weights together
                # move the mean by at most twice the mean size.  Probabilities and values: half a step of fp16 each (2^-25 and
                # 2^-36 below its smallest normal number); sums over keys in fp32; the joining of pieces: 16 more steps.
                top = scale * (qq.abs() @ kk.abs().T).amax(-1, keepdim=True)
                expo = (U16 + (kk.shape[1] + 8) * U32) * top + 4 * U32
                tol[a:a + n, h] = (2 * expo.expm1() + 2 * U16 + (m + 16) * U32) * size + 2.0 ** -25 + m * 2.0 ** -36 * vv.abs().max() + U[BF] * ref.abs()
                o[a:a + n, h] = ref
        a += n
    return o, tol


def chunk_case(S, new, lens, hq, hk, d, group, page, seed=0, qscale=1.0, scale=None, tail=3, max_length=None, pages=None):
    g = gen(seed)
    count = pages or sum(-(-x // page) for x in lens) + 2
    cache = filled_cache(S, count, page, hk, d, group, g)
    table = table_of(lens, page, count, g)
    q = randn(sum(new) + tail, hq + 1, d, g=g, dtype=BF, scale=qscale)[:, :hq]
    out = torch.full((sum(new) + tail, hq + 2, d), 0.375, dtype=BF, device=DEV)[:, 1:hq + 1]
    cu = i32([0] + new).cumsum(0).to(torch.int32)
    got = cache.attend_chunk(q, cu, table, i32(lens), out=out, scale=scale, max_length=max_length)
    cache.query_status()
    assert got is out
    ref, tol = chunk_reference(cache, q, new, table, lens, d ** -0.5 if scale is None else scale)
    within(out[:sum(new)], ref[:sum(new)], tol[:sum(new)])
    assert (out[sum(new):] == 0.375).all()                       # rows behind the last sequence
    return cache, q, cu, table, out


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("hq,hk", [(4, 4), (8, 2), (14, 2), (16, 1)])
def test_chunk_shapes(S, d, group, page, hq, hk):
    chunk_case(S, [5, 0, 1, 130, 40, 1], [300, 17, 129, 130, 700, 1], hq, hk, d, group, page, seed=hq + d)


@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 1), (3, 1)])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 42, 43, 85, 86, 127, 128, 129, 256, 257, 600])
def test_chunk_lengths(S, n, hq, hk):
    # around the edges of tiles, items and blocks of keys, with nothing, one token and several blocks before the chunk
    for before in (0, 1, 127, 128, 500):
        chunk_case(S, [n], [n + before], hq, hk, 64, 64, 32, seed=n + before)


@pytest.mark.parametrize("d,group,new,lens,hq,hk", [(128, 64, [48], [20011], 8, 1), (128, 32, [3], [9001], 4, 2), (64, 32, [40, 1], [30000, 12], 8, 2),
                                                    (96, 32, [300, 2], [5000, 4999], 2, 1), (128, 128, [1, 700, 1, 1], [3000, 2500, 1, 900], 8, 4)])
def test_chunk_in_many_pieces(S, d, group, new, lens, hq, hk):
    chunk_case(S, new, lens, hq, hk, d, group, 64, seed=new[0])


def test_chunk_bound_above_the_lengths(S):
    chunk_case(S, [7, 200], [100, 333], 8, 2, 128, 64, 16, seed=3, max_length=336)


@pytest.mark.parametrize("d,group", [(64, 64), (128, 32)])
def test_chunk_more_sequences_than_the_list_in_shared_memory(S, d, group):
    new = [(i * 7) % 4 for i in range(700)]
    lens = [n + (i * 13) % 50 for i, n in enumerate(new)]
    chunk_case(S, new, lens, 4, 2, d, group, 16, seed=1)
    chunk_case(S, [3] * 158, [40] * 158, 4, 2, d, group, 16, seed=2)         # (the list's last places)
    chunk_case(S, [3] * 161, [40] * 161, 4, 2, d, group, 16, seed=3)


@pytest.mark.parametrize("count", [156, 157, 158])
def test_chunk_lists_of_either_kind_about_full(S, count):
    # (3 count + 3) rows of two heads: at most 159, 160 and 161 items a head, of which 160 fit the list in shared memory
    chunk_case(S, [3] * count, [40 + i % 5 for i in range(count)], 4, 2, 64, 64, 16, seed=count)


def test_chunk_list_in_shared_memory_full_of_items(S):
    chunk_case(S, [1] * 160, [1 + 3 * i for i in range(160)], 1, 1, 64, 64, 16, seed=4, tail=0)      # 160 rows: 160 items
    chunk_case(S, [256] * 80, [300] * 80, 1, 1, 64, 64, 16, seed=5, tail=0)                          # 80 items, room for 160


@pytest.mark.parametrize("hq,hk", [(17, 1), (100, 1), (256, 1), (512, 2)])
def test_chunk_of_many_heads_that_share(S, hq, hk):
    # up to an item for every token
    chunk_case(S, [1, 3, 0, 9], [200, 3, 5, 140], hq, hk, 64, 32, 16, seed=hq)
    chunk_case(S, [2], [3000], hq, hk, 128, 64, 64, seed=hq + 1)


def test_chunk_rows_that_see_nothing(S):
    # more new tokens than the sequence has: the first rows see none; no token at all: all of them
    _, q, _, _, out = chunk_case(S, [10, 6, 300], [4, 0, 130], 4, 2, 64, 32, 16, seed=4)
    assert (out[:6] == 0).all() and (out[10:16] == 0).all() and (out[16:186] == 0).all() and (out[186:316] != 0).any()


def test_chunk_of_nothing(S):
    cache = filled_cache(S, 4, 16, 2, 64, 32, gen(0))
    table = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    q = randn(2, 4, 64, g=gen(1), dtype=BF)
    assert (cache.attend_chunk(q, i32([0]), table, i32([])) == 0).all()      # no sequence owns a row
    assert cache.attend_chunk(q[:0], i32([0, 0]), i32([[0]]), i32([5])).shape == (0, 4, 64)
    out = torch.full((2, 4, 64), 2.0, dtype=BF, device=DEV)
    cache.attend_chunk(q, i32([0, 0, 0]), i32([[0], [1]]), i32([5, 0]), out=out)
    assert (out == 2).all()


@pytest.mark.parametrize("new", [[40], [200], [1]])
def test_chunk_ignores_what_its_rows_do_not_see(S, new):
    # NaN behind the sequence, in a page's rest and in the chunk's own later tokens; rows that see them are NaN in those columns alone
    d, group, m = 128, 32, 333
    cache, q, cu, table, want = chunk_case(S, new, [m], 8, 2, d, group, 16, seed=8, tail=0)
    n, ln = new[0], i32([m])
    for x in (cache.k_params, cache.v_params):
        x[table[0, m // 16], :, m % 16:] = math.nan
    assert torch.equal(cache.attend_chunk(q, cu, table, ln), want)
    t = m - n + n // 2                                           # a token in the middle of the chunk
    keep = cache.v_params.clone()
    cache.v_params[table[0, t // 16], 1, t % 16, 2] = math.nan   # head 1, elements 64 .. 95
    got = cache.attend_chunk(q, cu, table, ln)
    seen = torch.zeros_like(got, dtype=torch.bool)
    seen[n // 2:, 4:, 64:96] = True
    assert torch.isnan(got[seen]).all() and torch.equal(got[~seen], want[~seen])
    cache.v_params.copy_(keep)
    cache.v_params[table[0, t // 16], 1, t % 16, 2, 1] = math.inf
    assert torch.equal(torch.isnan(cache.attend_chunk(q, cu, table, ln)), seen)
    cache.v_params.copy_(keep)
    cache.k_params[table[0, t // 16], 0, t % 16, 0, 0] = -math.inf           # a key: whole rows of its heads
    got = cache.attend_chunk(q, cu, table, ln)
    seen[:] = False
    seen[n // 2:, :4] = True
    assert torch.isnan(got[seen]).all() and torch.equal(got[~seen], want[~seen])
    cache.query_status()


@pytest.mark.parametrize("d,group", SHAPES)
def test_chunk_values_held_as_nan_all_over(S, d, group):
    # single groups of single tokens anywhere: exactly the rows and columns that see them are NaN
    g = gen(17)
    new, lens, hk, page = [150, 9], [1500, 700], 2, 64
    cache, q, cu, table, want = chunk_case(S, new, lens, 4, hk, d, group, page, seed=18, tail=0)
    seen = torch.zeros_like(want, dtype=torch.bool)
    for _ in range(30):
        i = int(torch.randint(0, 2, (1,), generator=g, device=DEV))
        t = int(torch.randint(lens[i] - new[i] - 3, lens[i], (1,), generator=g, device=DEV))
        h, gr = int(torch.randint(0, hk, (1,), generator=g, device=DEV)), int(torch.randint(0, d // group, (1,), generator=g, device=DEV))
        cache.v_params[table[i, t // page], h, t % page, gr, 0] = math.nan
        first = sum(new[:i]) + max(0, t - (lens[i] - new[i]))
        seen[first:sum(new[:i + 1]), 2 * h:2 * h + 2, gr * group:(gr + 1) * group] = True
    got = cache.attend_chunk(q, cu, table, i32(lens))
    assert torch.equal(torch.isnan(got), seen) and torch.equal(got[~seen], want[~seen])


@pytest.mark.parametrize("power_q,power_k", [(0, 0), (40, -30), (-60, 10), (100, -90), (12, -13)])
def test_chunk_sizes_of_queries_and_keys(S, power_q, power_k):
    # powers of two of the queries only move exponents; keys below 2^-14 lose bits, which the tolerance has (2^-25 each)
    g = gen(5)
    d, m, n = 64, 400, 37
    cache = filled_cache(S, 30, 16, 2, d, 64, g)
    cache.k_params.mul_(2.0 ** power_k)
    table = table_of([m], 16, 30, g)
    q = (randn(n, 4, d, g=g) * 2.0 ** power_q).to(BF)
    scale = d ** -0.5 * 2.0 ** (-power_q - power_k)
    out = cache.attend_chunk(q, i32([0, n]), table, i32([m]), scale=scale)
    cache.query_status()
    ref, tol = chunk_reference(cache, q, [n], table, [m], scale)
    lost = 2.0 ** -25 * scale * q.double().abs().sum(-1, keepdim=True) if power_k < -10 else 0
    within(out, ref, tol + (2 * torch.expm1(torch.as_tensor(lost, device=DEV)) * 6 if power_k < -10 else 0))


def lost(cache, params, table, i, m):
    """What a key or value of sequence i may be off by besides half a step, [heads]: 17 2^-25, or, where a head's largest parameters (the size of
    lo and of 16 scale together) are below 2^-8 and so in other units, 17 2^-38 of them, but 17 2^-125 at least."""
    p = params[table[i, :-(-m // cache.page_size)].long()].transpose(1, 2).flatten(0, 1)[:m].double().abs()
    u = (p[..., 0] + 16 * p[..., 1]).amax((0, 2))
    return 17 * torch.where(u < 2.0 ** -8, 2.0 ** -38 * u + 2.0 ** -125, torch.full_like(u, 2.0 ** -25))


def lifted_reference(cache, q, new, table, lens, scale):
    """chunk_reference for keys and values of any size."""
    g = q.shape[1] // cache.kv_heads
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(o)
    a = 0
    for i, (n, m) in enumerate(zip(new, lens)):
        if n and m:
            k, v = held(cache, table, i, m)
            k_off, v_off = lost(cache, cache.k_params, table, i, m), lost(cache, cache.v_params, table, i, m)
            lim = (torch.arange(n, device=DEV) + m - n + 1).clamp(min=0)
            last = (lim - 1).clamp(min=0)
            for h in range(q.shape[1]):
                qq, kk, vv = q[a:a + n, h].double(), k[:, h // g], v[:, h // g]
                ref, size = R.head_all(qq, kk, vv, lim, scale)
                top = scale * (qq.abs() @ kk.abs().T)
                top = torch.cummax(top, -1).values.gather(1, last[:, None])          # of what the row sees
                vmax = vv.abs().max()
                expo = (U16 + (kk.shape[1] + 8) * U32) * top + scale * k_off[h // g] * qq.abs().sum(-1, keepdim=True) + 4 * U32
                # (Means of the same values differ by twice the largest at most, whatever their weights: where scores are so large that their
                # errors decide, the first term would be infinite.)
                moved = torch.minimum(2 * expo.clamp(max=30).expm1() * size, 2 * vmax)
                tol[a:a + n, h] = moved + (2 * U16 + (m + 16) * U32) * size + v_off[h // g] + m * 2.0 ** -36 * vmax + U[BF] * ref.abs()
                o[a:a + n, h] = ref
        a += n
    return o, tol


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("power_q,power_k,power_v", [(0, 0, -8), (40, -30, 0), (100, -90, -90), (0, -16, -16), (0, -20, -24), (12, -13, -13), (0, 0, -60), (-60, 10, -30)])
def test_chunk_keys_and_values_of_any_size(S, d, group, power_q, power_k, power_v):
    g = gen(5 + d)
    new, lens, page = [37, 300, 1], [400, 1300, 5000], 16
    count = sum(-(-m // page) for m in lens)
    cache = filled_cache(S, count, page, 2, d, group, g)
    cache.k_params.mul_(2.0 ** power_k)
    cache.v_params.mul_(2.0 ** power_v)
    table = table_of(lens, page, count, g)
    q = (randn(sum(new), 4, d, g=g) * 2.0 ** power_q).to(BF)
    scale = d ** -0.5 * 2.0 ** (-power_q - power_k)
    out = cache.attend_chunk(q, i32([0] + new).cumsum(0).to(torch.int32), table, i32(lens), scale=scale)
    cache.query_status()
    ref, tol = lifted_reference(cache, q, new, table, lens, scale)
    within(out, ref, tol)
    assert (ref.abs().amax() > 16 * tol.amax()).all()            # an output of zeros, or of equal weights, would not pass
    one = cache.attend(q[-1:, None].contiguous(), table[2:], i32(lens[2:]), scale=scale)[:, 0]
    if power_v >= -30:                                           # (attend loses smaller values)
        assert ((out[-1:].double() - one.double()).abs() <= 3 * tol[-1:] + 2 * U[BF] * 2.0 ** power_v).all()


@pytest.mark.parametrize("d,group", [(64, 64), (96, 32), (128, 32), (128, 128)])
@pytest.mark.parametrize("new,lens", [([9, 40], [1500, 700]), ([300], [2100]), ([5], [40000])])
@pytest.mark.parametrize("ramp", ["up", "down", "steps", "zeros first"])
def test_chunk_sizes_that_change_along_a_sequence(S, d, group, new, lens, ramp):
    # keys and values that grow and shrink by dozens of binades, by token
    g = gen(7)
    page, hk = 32, 2
    count = sum(-(-m // page) for m in lens)
    cache = filled_cache(S, count, page, hk, d, group, g)
    table = table_of(lens, page, count, g)
    for i, m in enumerate(lens):
        t = torch.arange(m, device=DEV)
        x = t / m
        by = {"up": -60 * (1 - x), "down": -60 * x, "steps": -20.0 * ((t // 300) % 3), "zeros first": torch.where(t < min(300, m // 2), -math.inf, -30.0)}[ramp].floor()
        by = torch.exp2(by.clamp(max=0))[:, None, None, None]
        at = table[i, t // page].long()
        for p in (cache.k_params, cache.v_params):
            p[at, :, t % page] = (p[at, :, t % page].float() * by).to(BF)
    q = randn(sum(new), 4, d, g=g, dtype=BF)
    for scale in (d ** -0.5, d ** -0.5 * 2.0 ** 20):             # scores that count, or only the small keys' (the large ones' decide their rows)
        out = cache.attend_chunk(q, i32([0] + new).cumsum(0).to(torch.int32), table, i32(lens), scale=scale)
        cache.query_status()
        ref, tol = lifted_reference(cache, q, new, table, lens, scale)
        within(out, ref, tol)


def test_chunk_sizes_do_not_go_by_what_is_not_finite_or_behind_the_sequence(S):
    # small keys and values next to groups of NaN and infinity, and to anything in the rest of the last page
    g = gen(8)
    d, m, n = 128, 333, 40
    cache = filled_cache(S, 30, 16, 2, d, 32, g)
    for x in (cache.k_params, cache.v_params):
        x.mul_(2.0 ** -40)
    table = table_of([m], 16, 30, g)
    q = (randn(n, 4, d, g=g) * 2.0 ** 20).to(BF)
    scale = d ** -0.5 * 2.0 ** 20
    cu, ln = i32([0, n]), i32([m])
    want = cache.attend_chunk(q, cu, table, ln, scale=scale)
    ref, tol = lifted_reference(cache, q, [n], table, [m], scale)
    within(want, ref, tol)
    for x in (cache.k_params, cache.v_params):
        x[table[0, m // 16], :, m % 16:] = 3.0
    assert torch.equal(cache.attend_chunk(q, cu, table, ln, scale=scale), want)
    cache.v_params[table[0, 3], 1, 5, 2] = math.nan              # head 1, elements 64 .. 95
    cache.v_params[table[0, 9], 1, 6, 2, 1] = math.inf
    cache.k_params[table[0, (m - 1) // 16], 0, (m - 1) % 16, 0, 0] = -math.inf       # the newest token's key of head 0: the last row
    got = cache.attend_chunk(q, cu, table, ln, scale=scale)
    seen = torch.zeros_like(got, dtype=torch.bool)
    seen[:, 2:, 64:96] = True
    seen[-1, :2] = True
    assert torch.isnan(got[seen]).all() and torch.equal(got[~seen], want[~seen])
    cache.query_status()


@pytest.mark.parametrize("power", [40, 0, -60])
def test_chunk_infinite_queries_leave_their_neighbours_scale(S, power):
    # rows are scaled by a power of two, exactly: without the infinity the other rows are the same to the last bit
    g = gen(6)
    cache = filled_cache(S, 30, 16, 2, 64, 64, g)
    table = table_of([400], 16, 30, g)
    q = (randn(37, 4, 64, g=g) * 2.0 ** power).to(BF)
    x = q.clone()
    x[4, 1, 3], x[4, 2, 63], x[36, 0, 0] = math.inf, -math.inf, math.inf
    want, got = (cache.attend_chunk(y, i32([0, 37]), table, i32([400]), scale=0.125 * 2.0 ** -power) for y in (q, x))
    same = torch.ones(37, 4, dtype=torch.bool, device=DEV)
    same[4, 1] = same[4, 2] = same[36, 0] = False
    assert torch.equal(got[same], want[same]) and torch.isnan(got[~same]).all()


def test_chunk_scores_that_rise_and_fall(S):
    for seed, qscale in ((1, 8.0), (2, 0.01), (3, 30.0)):
        chunk_case(S, [90, 300], [1500, 640], 4, 2, 128, 64, 32, seed=seed, qscale=qscale)


def test_chunk_rows_of_zeros_and_of_what_is_not_finite(S):
    cache, q, cu, table, want = chunk_case(S, [70], [500], 4, 2, 64, 32, 16, seed=9, tail=0)
    x = q.clone()
    x[3, 1], x[5, 0, 7], x[60, 3, 1] = 0, math.nan, math.inf
    got = cache.attend_chunk(x, cu, table, i32([500]))
    assert torch.isnan(got[5, 0]).all() and torch.isnan(got[60, 3]).all() and torch.isfinite(got[3, 1]).all()
    same = torch.ones(70, 4, dtype=torch.bool, device=DEV)
    same[3, 1] = same[5, 0] = same[60, 3] = False
    ref, tol = chunk_reference(cache, q, [70], table, [500], 64 ** -0.5)
    within(got[same], ref[same], tol[same])


def test_chunk_reports_what_only_the_device_sees(S):
    from paper_2301_01333_b200 import binding as B
    cache, q, cu, table, _ = chunk_case(S, [5, 9], [40, 60], 4, 2, 64, 32, 16, seed=6, tail=0)
    ln = i32([40, 60])

    def reported(match, *args, **kw):
        cache.attend_chunk(*args, **kw)
        with pytest.raises(B.GcError, match=match):
            cache.query_status()
        cache.query_status()
    bad = table.clone()
    bad[1, 2] = cache.pages
    reported("page", q, cu, bad, ln)
    bad[1, 2] = -1
    reported("page", q, cu, bad, ln)
    reported("longer than max_length", q, cu, table, i32([40, 61]), max_length=60)
    reported("longer than max_length", q, cu, table, i32([-1, 60]))
    reported("offsets", q, i32([0, 9, 5]), table, ln)
    reported("offsets", q, i32([0, 5, 15]), table, ln)
    reported("offsets", q, i32([-1, 5, 14]), table, ln)
    for x in (cache.k_params, cache.v_params):
        keep = x.clone()
        x[table[0, 1], 1, 3, 1, 0] = 70000.0
        reported("65504", q, cu, table, ln)
        x.copy_(keep)
        x[table[0, 1], 1, 3, 1, 1] = 5000.0                      # 15 times that
        reported("65504", q, cu, table, ln)
        x.copy_(keep)
        x[table[0, 1], 1, 3, 1] = torch.tensor([65280.0, 0.0])   # fits
        cache.attend_chunk(q, cu, table, ln)
        cache.query_status()
        x.copy_(keep)
    reported("score", (q.float() * 2.0 ** 26).to(BF), cu, table, ln, scale=64.0)
    cache.attend_chunk(q, cu, table, ln)
    cache.query_status()


def test_chunk_of_single_tokens_agrees_with_attend(S):
    # the same numbers but for rounding: K, V and the probabilities to fp16 here, probabilities to bf16 there
    d, lens = 128, [300, 1, 77, 1200]
    cache, q, cu, table, out = chunk_case(S, [1] * 4, lens, 8, 2, d, 64, 32, seed=11, tail=0)
    other = cache.attend(q[:, None].contiguous(), table, i32(lens))[:, 0]
    _, tol = chunk_reference(cache, q, [1] * 4, table, lens, d ** -0.5)
    assert ((out - other).abs().double() <= 2 * tol + 2 * U[BF] * (1 + other.abs().double())).all()


# ------------------------------------------------------------------------------------------------ weights
def lse_and_weights(cache, q, table, lens, scale, lse=None):
    """(lse [b, n, hq], weights of every token [b][t, hk], their tolerances) in 64 bits."""
    b, n, hq, d = q.shape
    g = hq // cache.kv_heads
    all_lse = torch.full((b, n, hq), -math.inf, dtype=torch.float64, device=DEV)
    off = torch.zeros_like(all_lse)
    got = []
    for i, m in enumerate(lens):
        if m == 0:
            got.append((torch.zeros(0, cache.kv_heads, dtype=torch.float64, device=DEV),) * 2)
            continue
        k, _ = held(cache, table, i, m)
        qq = q[i].double().unflatten(1, (-1, g))                               # [n, hk, g, d]
        s = scale * torch.einsum("nhgd,thd->nhgt", qq, k)
        hidden = torch.arange(m, device=DEV) >= (torch.arange(n, device=DEV) + m - n + 1)[:, None]
        s = s.masked_fill(hidden[:, None, None], -math.inf)
        all_lse[i] = torch.logsumexp(s, -1).flatten(1)
        # A score is a sum of d products of q and 16 + code, minus 16 sum q, sizes up to 47 scale sum |q| in all; then
        # exponents: products and sums of numbers up to the score's and the logarithm's size.
        ks = cache.k_params[table[i, :-(-m // cache.page_size)].long()].double().abs().nan_to_num(0.).amax()
        size = scale * 47 * ks * qq.abs().sum(-1) * (d + 4) + 4 * (s.masked_fill(hidden[:, None, None], 0).abs().amax(-1) + 8)
        off[i] = (size * U32).flatten(1)
        use = all_lse[i] if lse is None else lse[i].double()
        p = torch.exp(s - use.unflatten(1, (-1, g))[..., None]).masked_fill(hidden[:, None, None], 0).nan_to_num(posinf=0.)
        p = torch.where((use == -math.inf).unflatten(1, (-1, g))[..., None], torch.zeros_like(p), p)
        err = (p * (torch.expm1(size * U32) + (4 + 4 * use.abs().clamp(max=1e3).unflatten(1, (-1, g))) * U32)[..., None]).sum((0, 2))
        got.append((p.sum((0, 2)).T, (err + (n * g) * U32 * p.sum((0, 2))).T))
    return all_lse, off, got


def weigh_case(S, lens, n, hq, hk, d, group, page, seed=0, decay=1.0, out=False, max_length=None, scale=None):
    g = gen(seed)
    pages = sum(-(-x // page) for x in lens) + 3
    cache = filled_cache(S, pages, page, hk, d, group, g)
    table = table_of(lens, page, pages, g)
    q = randn(len(lens), n, hq + 1, d, g=g, dtype=BF)[:, :, :hq]
    ln = i32(lens)
    lse = torch.full((len(lens), n, hq), 7.0, device=DEV)
    o = cache.attend(q, table, ln, lse=lse, max_length=max_length, scale=scale)
    assert torch.equal(o, cache.attend(q, table, ln, max_length=max_length, scale=scale))      # as it was without
    sc = d ** -0.5 if scale is None else scale
    ref, off, _ = lse_and_weights(cache, q, table, lens, sc)
    assert torch.equal(lse == -math.inf, ref == -math.inf)
    fin = ref > -math.inf
    m = max(lens + [1])
    # (the sum of m exponentials, the logarithm, the reference added)
    within(lse[fin], ref[fin], (off + (m / 16 + 64) * U32 + 8 * U32 * (ref.abs().nan_to_num(posinf=0.) + 8))[fin])
    w = torch.rand(pages, hk, page, generator=g, device=DEV)
    old = w.clone()
    where = torch.full_like(w, -3.0) if out else None
    got = cache.weigh(w, q, lse, table, ln, decay=decay, out=where, max_length=max_length, scale=scale)
    cache.query_status()
    assert got is (where if out else w)
    _, _, rows = lse_and_weights(cache, q, table, lens, sc, lse)
    expect, tol = (torch.full_like(old, -3.0) if out else old).double(), torch.zeros_like(old, dtype=torch.float64)
    for i, m in enumerate(lens):
        t = torch.arange(m, device=DEV)
        at = table[i, t // page].long()
        expect[at, :, t % page] = decay * old[at, :, t % page].double() + rows[i][0]
        tol[at, :, t % page] = rows[i][1] + 3 * U32 * expect[at, :, t % page].abs()
    within(got, expect, tol)
    if out:
        assert torch.equal(w, old)
    return cache, q, lse, table, ln


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n,hq,hk", [(1, 4, 4), (1, 8, 2), (2, 14, 2), (5, 4, 2), (1, 16, 1)])
def test_weigh_shapes(S, d, group, page, n, hq, hk):
    weigh_case(S, [300, 0, 1, 33, 700, 5], n, hq, hk, d, group, page, seed=d + hq)


@pytest.mark.parametrize("n,hq,hk", [(16, 16, 4), (16, 8, 1), (9, 32, 2), (16, 40, 1)])
def test_weigh_many_columns(S, n, hq, hk):
    weigh_case(S, [500, 16, 129], n, hq, hk, 64, 32, 16, seed=n + hq, decay=0.5)      # up to 640 of them: several passes


@pytest.mark.parametrize("lens", [[1, 2, 3, 5, 7, 11, 31], [100, 333, 511], [1000, 1023], [4099], [12345, 3]])
@pytest.mark.parametrize("n,hq,hk", [(1, 4, 4), (3, 16, 2)])
def test_logarithms_and_weights_of_equal_scores(S, lens, n, hq, hk):
    # Queries of zero: t tokens seen weigh 1 / t each, and the sum of their exponentials is t exactly.  Its logarithm is off by a step or so of the
    # function and half a step of the constant and of the product, 6 U32 of itself; a weight by that, its exponent's product and the exponential.
    g = gen(sum(lens))
    page = 16
    count = sum(-(-m // page) for m in lens)
    cache = filled_cache(S, count, page, hk, 64, 32, g)
    table, ln = table_of(lens, page, count, g), i32(lens)
    q = torch.zeros(len(lens), n, hq, 64, dtype=BF, device=DEV)
    lse = torch.empty(len(lens), n, hq, device=DEV)
    cache.attend(q, table, ln, lse=lse)
    seen = torch.tensor(lens, device=DEV)[:, None] - (n - 1) + torch.arange(n, device=DEV)
    ref = torch.where(seen > 0, seen.clamp(min=1).double().log(), -math.inf)[..., None].expand(-1, -1, hq)
    some = ref > -math.inf
    assert torch.equal(lse == -math.inf, ~some)
    assert ((lse.double() - ref)[some].abs() <= 6 * U32 * ref[some]).all()
    w = cache.weigh(cache.new_weights(), q, lse, table, ln)
    cache.query_status()
    for i, m in enumerate(lens):
        t = torch.arange(m, device=DEV)
        got = w[table[i, t // page].long(), :, t % page].double()
        want = sum((t < s).double() / max(int(s), 1) * (hq // hk) for s in seen[i])[:, None]
        assert ((got - want).abs() <= (10 * math.log(m + 1) + 4 + n * hq) * U32 * want).all()


@pytest.mark.parametrize("d,group", SHAPES)
def test_weight_of_a_single_token_is_one(S, d, group):
    # What attend and weigh make of a score is the same number.  The exponent of its weight in attend stands near 64, half a step there is 2^-18
    # binades; the logarithm, the score and their difference are off by half steps of numbers up to their size (the score's power of two, 1.45 times it).
    g = gen(d)
    cache = filled_cache(S, 9, 16, 2, d, group, g)
    table, ln = torch.arange(9, device=DEV, dtype=torch.int32)[:, None], torch.ones(9, dtype=torch.int32, device=DEV)
    q = randn(9, 1, 8, d, g=g, dtype=BF)
    lse = torch.empty(9, 1, 8, device=DEV)
    cache.attend(q, table, ln, lse=lse)
    for h in range(4):                                           # one query head of a key/value head at a time
        alone = torch.full_like(lse, -math.inf)
        alone[..., [h, h + 4]] = lse[..., [h, h + 4]]
        w = cache.weigh(cache.new_weights(), q, alone, table, ln)
        off = (w[:, :, 0].double() - 1).abs()
        assert (off <= math.log(2) * 2.0 ** -18 + 8 * U32 * (1 + 1.45 * alone[:, 0, [h, h + 4]].double().abs())).all()
        assert (w[:, :, 1:] == 0).all()


@pytest.mark.parametrize("n,hq,hk", [(1, 41, 1), (1, 256, 1), (3, 200, 1), (16, 512, 2)])
def test_weigh_of_many_heads_that_share(S, n, hq, hk):
    weigh_case(S, [90, 1, 300], n, hq, hk, 128, 64, 16, seed=n + hq)      # up to 4096 columns


def test_tables_without_pages(S):
    # every sequence is empty, and the tables have no width
    cache = filled_cache(S, 4, 16, 2, 64, 32, gen(2))
    table, ln = torch.zeros(3, 0, dtype=torch.int32, device=DEV), i32([0, 0, 0])
    q = randn(5, 4, 64, g=gen(3), dtype=BF)
    assert (cache.attend_chunk(q, i32([0, 2, 2, 5]), table, ln) == 0).all()
    lse, w = torch.zeros(3, 1, 4, device=DEV), torch.rand(4, 2, 16, device=DEV)
    keep = w.clone()
    assert (cache.attend(q[:3, None].contiguous(), table, ln, lse=lse) == 0).all() and (lse == -math.inf).all()
    assert torch.equal(cache.weigh(w, q[:3, None].contiguous(), lse, table, ln), keep)
    lengths, kept = cache.evict(w, table, ln, 8, 2)
    assert (lengths == 0).all() and (kept == -1).all() and torch.equal(w, keep)
    cache.query_status()


@pytest.mark.parametrize("decay,out", [(1.0, True), (0.5, False), (0.0, True), (0.0, False)])
def test_weigh_decay_and_output(S, decay, out):
    weigh_case(S, [100, 64, 65], 2, 8, 2, 128, 64, 32, seed=3, decay=decay, out=out)


@pytest.mark.parametrize("lens,max_length", [([8000], None), ([3000, 31, 32, 33, 4097], 4112), ([1] * 60, 16), (list(range(0, 90)), 96)])
def test_weigh_lengths(S, lens, max_length):
    weigh_case(S, lens, 1, 8, 2, 128, 64, 16, seed=len(lens), max_length=max_length)


def test_weigh_queries_before_the_sequence_and_without_logarithm(S):
    # more queries than tokens: the first ones see nothing; an lse of minus infinity adds nothing even where there is something
    cache, q, lse, table, ln = weigh_case(S, [2, 40, 0], 4, 4, 2, 64, 32, 16, seed=4)
    assert (lse[0, :2] == -math.inf).all() and (lse[2] == -math.inf).all() and torch.isfinite(lse[0, 2:]).all()
    w = cache.new_weights()
    assert w.shape == (cache.pages, 2, 16) and (w == 0).all()
    cache.weigh(w, q, torch.full_like(lse, -math.inf), table, ln)
    assert (w == 0).all()


def test_weigh_ignores_what_it_is_not_asked_about(S):
    cache, q, lse, table, ln = weigh_case(S, [37, 50], 1, 4, 2, 64, 32, 16, seed=5)
    want = cache.weigh(cache.new_weights(), q, lse, table, ln, decay=0.0)
    w = torch.full_like(want, math.nan)
    cache.k_params[table[0, 2], :, 5:] = math.nan                # behind the sequence
    cache.v_params.fill_(math.nan)
    out = torch.zeros_like(want)
    cache.weigh(w, q, lse, table, ln, decay=0.0, out=out)        # what the weights were is not looked at
    assert torch.equal(out, want)
    cache.k_params[table[1, 0], 1, 3] = math.nan                 # a key of head 1: its own weight alone
    lse2 = lse.clone()
    out2 = cache.weigh(w, q, lse2, table, ln, decay=0.0, out=torch.zeros_like(want))
    assert torch.isnan(out2[table[1, 0], 1, 3]) and torch.isnan(out2).sum() == 1


def test_weigh_reports_pages_and_lengths(S):
    from paper_2301_01333_b200 import binding as B
    cache, q, lse, table, ln = weigh_case(S, [37, 50], 1, 4, 2, 64, 32, 16, seed=6)
    for bad_table, bad_ln, kw in ((table.clone().index_fill_(1, i32([1]).long(), 999), ln, {}), (table, i32([37, 51]), dict(max_length=50)), (table, i32([-2, 5]), {})):
        cache.weigh(cache.new_weights(), q, lse, bad_table, bad_ln, **kw)
        with pytest.raises(B.GcError, match="page|length"):
            cache.query_status()
        cache.query_status()


# ------------------------------------------------------------------------------------------------ eviction
def kept_reference(scores, n, keep, recent):
    """Positions, before, of the tokens at 0 .. min(n, keep) - 1 after; scores: a list of n numbers."""
    if n <= keep:
        return list(range(n))
    stays = set(range(n - recent, n))
    rest = sorted(range(n - recent), key=lambda t: (0 if math.isnan(scores[t]) else 1, -scores[t] if not math.isnan(scores[t]) else 0, t))
    stays |= set(rest[:keep - recent])
    behind = iter(sorted(t for t in stays if t >= keep))
    return [t if t in stays else next(behind) for t in range(keep)]


def evict_case(S, lens, keep, recent, hk, d, group, page, scores_of, seed=0, copies=False, max_length=None):
    g = gen(seed)
    pages = sum(-(-x // page) for x in lens) + 2
    extra = len(lens) * -(-max(keep, 1) // page) if copies else 0
    cache = filled_cache(S, pages + extra, page, hk, d, group, g)
    table = table_of(lens, page, pages, g)
    out_table = None
    if copies:
        out_table = (pages + torch.randperm(extra, generator=g, device=DEV)).to(torch.int32).view(len(lens), -1)
    scores = scores_of((pages + extra, hk, page), g)
    arrays = [cache.k_codes, cache.k_params, cache.v_codes, cache.v_params, scores]
    before = [x.clone() for x in arrays]
    lengths, kept = cache.evict(scores, table, i32(lens), keep, recent, max_length=max_length, out_table=out_table)
    cache.query_status()
    assert lengths.tolist() == [min(n, keep) for n in lens] and kept.shape == (len(lens), hk, keep)
    want = [x.clone() for x in before]
    to = table if out_table is None else out_table
    for i, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        at = table[i, t // page].long()
        mine = before[4][at, :, t % page].tolist()               # [n][hk]
        m = min(n, keep)
        for h in range(hk):
            ref = kept_reference([x[h] for x in mine], n, keep, recent)
            assert kept[i, h].tolist() == ref + [-1] * (keep - m)
            src, dst = torch.tensor(ref, device=DEV, dtype=torch.long), torch.arange(m, device=DEV)
            for x, y in zip(want, before):
                x[to[i, dst // page].long(), h, dst % page] = y[table[i, src // page].long(), h, src % page]
            rest = torch.arange(m, n if out_table is None else -(-m // page) * page, device=DEV)
            want[4][to[i, rest // page].long(), h, rest % page] = 0
    live = torch.zeros(pages + extra, page, dtype=torch.bool, device=DEV)
    for i, n in enumerate(lens):
        t = torch.arange(min(n, keep), device=DEV)
        live[to[i, t // page].long(), t % page] = True
    bits = {torch.float32: torch.int32, BF: torch.int16, torch.uint8: torch.uint8}
    for k, (x, y, z) in enumerate(zip(arrays, want, before)):
        x, y, z = (v.view(bits[v.dtype]) for v in (x, y, z))
        if k < 4:                                                # what the kept positions hold; all else of a copy is as it was
            assert torch.equal(x.transpose(1, 2)[live], y.transpose(1, 2)[live])
            if copies:
                assert torch.equal(x.transpose(1, 2)[~live], z.transpose(1, 2)[~live])
        else:
            assert torch.equal(x, y)


def rand(shape, g):
    return torch.rand(shape, generator=g, device=DEV)


def few_values(shape, g):
    return torch.randint(0, 4, shape, generator=g, device=DEV).float() / 4 - 0.25


def awkward(shape, g):
    some = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, -1.5, 1e-42, -1e-42, 3e38, 2.0], device=DEV)
    return some[torch.randint(0, 10, shape, generator=g, device=DEV)]


@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("scores_of", [rand, few_values, awkward])
@pytest.mark.parametrize("d,group", SHAPES)
def test_evict_shapes(S, d, group, scores_of, copies):
    evict_case(S, [300, 0, 64, 65, 1, 500], 64, 9, 2, d, group, 16, scores_of, seed=d, copies=copies)


@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("keep,recent", [(0, 0), (1, 0), (1, 1), (50, 50), (16, 0), (17, 1), (199, 3), (200, 0), (400, 17)])
def test_evict_budgets(S, keep, recent, copies):
    evict_case(S, [200, 20, 201, 16], keep, recent, 3, 64, 32, 16, few_values, seed=keep, copies=copies)


@pytest.mark.parametrize("lens,keep,recent,hk", [([5000], 1000, 64, 1), ([9000, 4000], 2222, 0, 2), ([1027] * 40, 500, 100, 4), ([20000], 19000, 500, 1), ([3000], 2999, 1, 2)])
@pytest.mark.parametrize("scores_of", [rand, few_values])
def test_evict_on_one_and_on_several_ctas(S, lens, keep, recent, hk, scores_of):
    evict_case(S, lens, keep, recent, hk, 64, 64, 64, scores_of, seed=keep)


def test_evict_copies_of_sequences_that_share_pages(S):
    # a common beginning, kept by each sequence by its own budget; the sources stay as they are
    g = gen(9)
    page, hk, keep, recent = 16, 2, 50, 6
    cache = filled_cache(S, 40, page, hk, 64, 32, g)
    order = torch.randperm(40, generator=g, device=DEV).to(torch.int32)
    table = torch.stack([order[:8], torch.cat([order[:5], order[8:11]]), torch.cat([order[:5], order[11:14]])])
    lens, to = [128, 100, 40], order[16:28].view(3, 4)
    scores = rand((40, hk, page), g)
    before = [x.clone() for x in (cache.k_codes, cache.v_params, scores)]
    lengths, kept = cache.evict(scores, table, i32(lens), keep, recent, out_table=to)
    cache.query_status()
    assert lengths.tolist() == [50, 50, 40]
    for i, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        mine = before[2][table[i, t // page].long(), :, t % page].tolist()
        for h in range(hk):
            ref = kept_reference([x[h] for x in mine], n, keep, recent)
            assert kept[i, h, :len(ref)].tolist() == ref
            src, dst = torch.tensor(ref, device=DEV), torch.arange(len(ref), device=DEV)
            for x, y in zip((cache.k_codes, cache.v_params, scores), before):
                assert torch.equal(x[to[i, dst // page].long(), h, dst % page], y[table[i, src // page].long(), h, src % page])
    for x, y in zip((cache.k_codes, cache.v_params, scores), before):
        assert torch.equal(x[order[:16].long()], y[order[:16].long()])


def test_evict_of_more_sequences_than_ctas_fit(S):
    # more (sequence, head) pairs than two an SM, each longer than a small CTA's usual share; and some of them short
    evict_case(S, [4300 if i % 3 else i for i in range(80)], 700, 33, 4, 64, 64, 32, few_values)


def test_evict_scores_that_are_all_alike(S):
    evict_case(S, [3000, 100], 700, 20, 2, 64, 64, 32, lambda shape, g: torch.ones(shape, device=DEV), seed=1)     # the oldest stay


def test_evict_more_positions_than_shared_memory_holds(S):
    # eight CTAs of 40960 keys each hold 327680
    g = gen(2)
    n, keep, recent, page = 400_003, 1000, 10, 256
    pages = -(-n // page)
    cache = S.KV4Cache.allocate(pages, page, 1, 64, 64)
    scores = (torch.randint(0, 50_000, (pages, 1, page), generator=g, device=DEV)).float()
    table = torch.arange(pages, device=DEV, dtype=torch.int32)[None]
    flat = scores.flatten()[:n].clone()
    lengths, kept = cache.evict(scores, table, i32([n]), keep, recent)
    cache.query_status()
    order = torch.sort(flat[:n - recent], descending=True, stable=True).indices[:keep - recent]
    stays = torch.cat([order, torch.arange(n - recent, n, device=DEV)])
    assert lengths.item() == keep and torch.equal(kept.flatten().long().sort().values, stays.sort().values)
    assert torch.equal(scores.flatten()[:keep], flat[kept.flatten().long()]) and (scores.flatten()[keep:n] == 0).all()


def test_evict_reports_pages_and_lengths(S):
    from paper_2301_01333_b200 import binding as B
    cache = filled_cache(S, 12, 16, 2, 64, 32, gen(3))
    table = torch.arange(12, device=DEV, dtype=torch.int32).view(2, 6)
    for bad, ln, kw in ((table.clone().fill_(12), i32([60, 60]), {}), (table, i32([60, 97]), {}), (table, i32([60, -1]), {}), (table, i32([60, 60]), dict(max_length=59)),
                        (table, i32([60, 60]), dict(out_table=i32([[99, 99], [-1, 5]])))):
        cache.evict(cache.new_weights(), bad, ln, 20, 2, **kw)
        with pytest.raises(B.GcError, match="page|length"):
            cache.query_status()
        cache.query_status()


# ------------------------------------------------------------------------------------------------ together
def _server(S, seed=0, d=64, group=32, hq=8, hk=2, page=16):
    """Two sequences whose prompts arrive in chunks, then steps that weigh, then an eviction, then steps again."""
    g = gen(seed)
    lens, width = [70, 45], 12
    cache = S.KV4Cache.allocate(2 * width, page, hk, d, group)
    table = torch.randperm(2 * width, generator=g, device=DEV).to(torch.int32).view(2, width)
    qkv = randn(2, 160, hq + 2 * hk, d, g=g, dtype=BF)
    weights, done, outs = cache.new_weights(), [0, 0], []

    def append(new):
        rows, slots = [], []
        for b, n in enumerate(new):
            t = torch.arange(done[b], done[b] + n, device=DEV)
            rows.append(qkv[b, seen[b]:seen[b] + n])
            slots.append(table[b, t // page].long() * page + t % page)
            done[b] += n
            seen[b] += n
        x = torch.cat(rows)
        cache.append(x[:, hq:hq + hk], x[:, hq + hk:], torch.cat(slots))
        return x[:, :hq]
    seen = [0, 0]
    for new in ([32, 32], [30, 0], [8, 13]):
        q = append(new)
        outs.append(("chunk", q, list(new), list(done), cache.attend_chunk(q, i32([0] + new).cumsum(0).to(torch.int32), table, i32(done))))
    for step in range(20):
        q = append([1, 1]).unsqueeze(1).contiguous()
        lse = torch.empty(2, 1, hq, device=DEV)
        o = cache.attend(q, table, i32(done), lse=lse)
        cache.weigh(weights, q, lse, table, i32(done), decay=0.9)
        outs.append(("step", q, None, list(done), o))
        if step == 9:
            ln, kept = cache.evict(weights, table, i32(done), 40, 8)
            done[:] = ln.tolist()
            outs.append(("evict", kept, None, list(done), weights.clone()))
    cache.query_status()
    return cache, table, weights, outs, done


def test_chunks_steps_weights_and_eviction_together(S):
    cache, table, weights, outs, done = _server(S)
    # after the eviction: 40 tokens and ten more steps; the last step against what the cache holds now
    assert done == [50, 50] and outs[13][3] == [40, 40]
    kept = outs[13][1]
    assert (kept[:, :, :40] >= 0).all() and all(len(set(kept[b, h].tolist())) == 40 for b in range(2) for h in range(2))
    for b, n in enumerate((80, 55)):                             # the newest eight stayed
        assert all(set(range(n - 8, n)) <= set(kept[b, h].tolist()) for h in range(2))
    kind, q, _, lens, o = outs[-1]
    from test_serving_gpu import attend_reference
    ref, tol = attend_reference(cache, q, table, lens, 64 ** -0.5, 32)
    within(o, ref, tol)
    assert torch.isfinite(weights).all() and (weights >= 0).all()
    # all weight that was given out is still there or was given up with its token: what a step adds sums to one per query head
    before = weights.clone()
    lse = torch.empty(2, 1, 8, device=DEV)
    cache.attend(q, table, i32(lens), lse=lse)
    cache.weigh(weights, q, lse, table, i32(lens))
    added = (weights - before).double().sum((0, 2))
    assert ((added - 2 * 4).abs() <= 8 * 200 * U32 * (1 + before.max().item())).all()


def test_a_prompt_in_chunks_is_the_prompt(S):
    # chunk by chunk, and all at once through the prompt kernel over what the cache holds, rounded to bf16 there
    g = gen(21)
    d, hq, hk, page, n = 128, 8, 2, 32, 700
    cache = S.KV4Cache.allocate(24, page, hk, d, 64)
    table = torch.randperm(24, generator=g, device=DEV).to(torch.int32)[None]
    qkv = randn(n, hq + 2 * hk, d, g=g, dtype=BF)
    t = torch.arange(n, device=DEV)
    slots = table[0, t // page].long() * page + t % page
    out, at = [], 0
    for c in (1, 255, 256, 100, 88):
        cache.append(qkv[at:at + c, hq:hq + hk], qkv[at:at + c, hq + hk:], slots[at:at + c])
        at += c
        out.append(cache.attend_chunk(qkv[at - c:at, :hq], i32([0, c]), table, i32([at])))
    out = torch.cat(out)
    once = cache.attend_chunk(qkv[:, :hq], i32([0, n]), table, i32([n]))
    ref, tol = chunk_reference(cache, qkv[:, :hq], [n], table, [n], d ** -0.5)
    within(out, ref, tol)
    within(once, ref, tol)
    k, v = cache.read(slots)
    prompt = S.attention_prompt(qkv[:, :hq], k, v, i32([0, n]))
    # bf16 keys and probabilities: eight times fp16's half steps in the scores and the weights
    assert ((prompt.double() - out.double()).abs() <= 10 * tol).all()


def test_results_do_not_depend_on_the_run(S):
    a, b = _server(S, 5), _server(S, 5)
    assert all(torch.equal(x[4], y[4]) for x, y in zip(a[3], b[3])) and torch.equal(a[2], b[2])
    for x, y in zip((a[0].k_codes, a[0].v_params), (b[0].k_codes, b[0].v_params)):
        assert torch.equal(x, y)


def _call(S, seed):
    """A chunk call, weights and an eviction into other pages as one function, whose inputs can be replaced in place."""
    g = gen(seed)
    lens, new, page, hk = [900, 333], [70, 1], 32, 2
    cache = filled_cache(S, 80, page, hk, 128, 64, g)
    table, ln, cu = table_of(lens, page, 60, g), i32(lens), i32([0, 70, 71])
    to = torch.arange(60, 76, device=DEV, dtype=torch.int32).view(2, 8)
    q = randn(71, 8, 128, g=g, dtype=BF)
    q1 = randn(2, 1, 8, 128, g=g, dtype=BF)
    base = torch.rand(80, hk, page, generator=g, device=DEV)

    def run():
        o = cache.attend_chunk(q, cu, table, ln)
        lse = torch.empty(2, 1, 8, device=DEV)
        s = cache.attend(q1, table, ln, lse=lse)
        w = cache.weigh(base, q1, lse, table, ln, decay=0.5, out=torch.zeros_like(base))
        m, kept = cache.evict(w, table, ln, 250, 16, out_table=to)
        o2 = cache.attend(q1, to, m)
        return [o, s, lse, w, m, kept, o2]
    return run, q, cache


def test_two_captured_graphs_share_nothing(S):
    calls = [_call(S, s) for s in (31, 32)]
    want = [[x.clone() for x in run()] for run, _, _ in calls]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for run, _, _ in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run())
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        for o in outs:
            o[0].fill_(math.nan)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):                        # both at once
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
    for (_, q, cache), o, g, w in zip(calls, outs, graphs, want):    # a replay sees new inputs
        q.neg_()
        g.replay()
        torch.cuda.synchronize()
        assert not torch.equal(o[0], w[0]) and torch.equal(o[3], w[3])
        cache.query_status()


def test_calls_on_a_stream_of_their_own_and_closely_one_after_another(S):
    run, q, cache = _call(S, 41)
    want = [x.clone() for x in run()]
    real = q.clone()
    q.zero_()
    run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        q.copy_(real)                                            # a launch on another stream would overtake this, and see zeros
        got = [run() for _ in range(20)]
    s.synchronize()
    assert all(torch.equal(x, y) for g in got for x, y in zip(g, want))


@pytest.mark.parametrize("new,lens,hq,hk,d,group,page", [([48], [60000], 8, 1, 128, 64, 64), ([1] * 12 + [150, 96], [500 * i for i in range(1, 13)] + [3000, 2000], 16, 4, 128, 64, 64),
                                                         ([300, 40], [9000, 9000], 4, 2, 64, 32, 16), ([64], [20000], 8, 1, 96, 32, 256)])
def test_chunk_calls_in_close_succession(S, new, lens, hq, hk, d, group, page):
    # many blocks of keys to a CTA, and nothing between the calls: every one gives what the first gave
    cache, q, cu, table, out = chunk_case(S, new, lens, hq, hk, d, group, page, seed=7, tail=0)
    outs = [torch.zeros_like(out) for _ in range(60)]
    for o in outs:
        cache.attend_chunk(q, cu, table, i32(lens), out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) for o in outs)
    ln = i32(lens)
    for _ in range(5):                                           # without even the lengths' copy in between
        for o in outs:
            cache.attend_chunk(q, cu, table, ln, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) for o in outs)
    cache.query_status()


def test_cache_of_more_than_two_to_the_32_bytes(S):
    # 40000 pages of 256 tokens and 8 heads of 128: 5.2 GB of codes, 10.2 million tokens; the sequence lies in the last pages
    pages, page, hk, d = 40000, 256, 8, 128
    small = filled_cache(S, 6, page, hk, d, 64, gen(51))
    cache = S.KV4Cache.allocate(pages, page, hk, d, 64)
    at = torch.tensor([39999, 39000, 35001, 1, 39998, 38000], device=DEV)
    for x, y in zip((cache.k_codes, cache.k_params, cache.v_codes, cache.v_params), (small.k_codes, small.k_params, small.v_codes, small.v_params)):
        x[at] = y
    q, q1 = randn(50, 16, d, g=gen(52), dtype=BF), randn(1, 2, 16, d, g=gen(53), dtype=BF)
    got = []
    for c, table, to in ((small, torch.arange(4), [4, 5]), (cache, at[:4], [39998, 38000])):
        table, ln, lse = table.to(torch.int32).to(DEV)[None], i32([1000]), torch.empty(1, 2, 16, device=DEV)
        o = c.attend_chunk(q, i32([0, 50]), table, ln)
        s = c.attend(q1, table, ln, lse=lse)
        w = c.weigh(c.new_weights(), q1, lse, table, ln)
        m, kept = c.evict(w, table, ln, 400, 16, out_table=i32([to]))
        got.append([o, s, lse, w[table[0].long()], kept, c.attend(q1, i32([to]), m)])
        c.query_status()
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_refusals_leave_everything_as_it_was(S):
    from paper_2301_01333_b200 import binding as B
    cache = filled_cache(S, 8, 16, 2, 64, 32, gen(61))
    table, ln, cu = torch.arange(8, device=DEV, dtype=torch.int32).view(2, 4), i32([40, 30]), i32([0, 3, 5])
    q, q1, lse, w = randn(5, 4, 64, g=gen(62), dtype=BF), randn(2, 1, 4, 64, g=gen(63), dtype=BF), torch.zeros(2, 1, 4, device=DEV), cache.new_weights()
    before = [x.clone() for x in (cache.k_codes, cache.v_params, w)]
    out = torch.ones_like(q)
    bad = [(ValueError, lambda: cache.attend_chunk(q.float(), cu, table, ln)), (ValueError, lambda: cache.attend_chunk(q[:, :3].transpose(1, 2), cu, table, ln)),
           (ValueError, lambda: cache.attend_chunk(q, cu.long(), table, ln)), (ValueError, lambda: cache.attend_chunk(q, cu, table[:1], ln)),
           (ValueError, lambda: cache.attend_chunk(q, cu, table, ln[:1])), (ValueError, lambda: cache.attend_chunk(q, cu, table.long(), ln)),
           (ValueError, lambda: cache.attend_chunk(q, cu, table, ln, out=out[:1].expand(5, 4, 64))), (ValueError, lambda: cache.attend_chunk(q.cpu(), cu, table, ln)),
           (B.GcError, lambda: cache.attend_chunk(q[:, :3], cu, table, ln)), (B.GcError, lambda: cache.attend_chunk(q, cu, table, ln, max_length=65)),
           (B.GcError, lambda: cache.attend_chunk(q, cu, table, ln, scale=0.0)), (TypeError, lambda: cache.attend_chunk(q, cu, table, ln, scale="x")),
           (TypeError, lambda: cache.attend_chunk(None, cu, table, ln)), (TypeError, lambda: cache.attend_chunk(q, [0, 3, 5], table, ln)),
           (ValueError, lambda: cache.attend(q1, table, ln, lse=lse[:, 0])), (ValueError, lambda: cache.attend(q1, table, ln, lse=lse.double())),
           (ValueError, lambda: cache.weigh(w[:7], q1, lse, table, ln)), (ValueError, lambda: cache.weigh(w.half(), q1, lse, table, ln)),
           (ValueError, lambda: cache.weigh(w, q1, lse[:1], table, ln)), (ValueError, lambda: cache.weigh(w, q1[0], lse, table, ln)),
           (ValueError, lambda: cache.weigh(w, q1, lse, table, ln, out=w.transpose(1, 2))), (B.GcError, lambda: cache.weigh(w, q1, lse, table, ln, decay=-1.0)),
           (TypeError, lambda: cache.weigh(w, q1, None, table, ln)), (B.GcError, lambda: cache.evict(w, table, ln, 8, 9)), (B.GcError, lambda: cache.evict(w, table, ln, -1)),
           (ValueError, lambda: cache.evict(w[:, :1], table, ln, 8)), (ValueError, lambda: cache.evict(w, table[:, ::2], ln, 8)), (TypeError, lambda: cache.evict(w, table, ln, 8.5)),
           (B.GcError, lambda: cache.evict(w, table, ln, 20, out_table=i32([[1], [2]]))), (ValueError, lambda: cache.evict(w, table, ln, 8, out_table=i32([[1]]))),
           (ValueError, lambda: cache.evict(w.clone().requires_grad_(), table, ln, 8)), (ValueError, lambda: cache.attend_chunk(q.clone().requires_grad_(), cu, table, ln))]
    for error, call in bad:
        with pytest.raises(error):
            call()
    cache.query_status()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((cache.k_codes, cache.v_params, w), before)) and (out == 1).all()


def test_outputs_that_were_given_count_as_written(S):
    cache = filled_cache(S, 8, 16, 2, 64, 32, gen(71))
    table, ln, cu = torch.arange(8, device=DEV, dtype=torch.int32).view(2, 4), i32([40, 30]), i32([0, 3, 5])
    q, q1, lse, w = randn(5, 4, 64, g=gen(72), dtype=BF), randn(2, 1, 4, 64, g=gen(73), dtype=BF), torch.zeros(2, 1, 4, device=DEV), cache.new_weights()
    out = torch.zeros_like(q)

    def version(call, *tensors):
        was = [t._version for t in tensors]
        call()
        assert all(t._version > v for t, v in zip(tensors, was))
    version(lambda: cache.attend_chunk(q, cu, table, ln, out=out), out)
    version(lambda: cache.attend(q1, table, ln, lse=lse), lse)
    version(lambda: cache.weigh(w, q1, lse, table, ln), w)
    version(lambda: cache.evict(w, table, ln, 8, 2), w, cache.k_codes, cache.v_params)


def test_evicting_again_after_growing_by_the_recent_ones_keeps_the_newest(S):
    # the documented use: a sequence is cut once it has grown by `recent`, again and again; ages by a list that follows `kept`
    g = gen(81)
    page, hk, keep, recent = 16, 2, 48, 16
    cache = filled_cache(S, 4, page, hk, 64, 32, g)
    table = torch.randperm(4, generator=g, device=DEV).to(torch.int32)[None]
    scores = torch.zeros(4, hk, page, device=DEV)
    ages, born = [list(range(48)) for _ in range(hk)], 48
    for _ in range(6):
        t = torch.arange(48, 64, device=DEV)
        for h in range(hk):
            ages[h] += list(range(born, born + recent))
        born += recent
        at = table[0, t // page].long()
        scores[at, :, t % page] = 0
        t = torch.arange(64, device=DEV)
        scores[table[0, t // page].long(), :, t % page] += torch.rand(64, hk, generator=g, device=DEV)
        lengths, kept = cache.evict(scores, table, i32([64]), keep, recent)
        assert lengths.item() == keep
        for h in range(hk):
            ages[h] = [ages[h][x] for x in kept[0, h].tolist()]
            assert set(range(born - recent, born)) <= set(ages[h])
    cache.query_status()


@pytest.mark.parametrize("new,lens,hq,hk,d,group,page", [([48], [60000], 8, 1, 128, 64, 64), ([1] * 12 + [150, 96], [500 * i for i in range(1, 13)] + [3000, 2000], 16, 4, 128, 32, 64),
                                                         ([300, 40], [9000, 9000], 4, 2, 64, 32, 16), ([64], [20000], 8, 1, 96, 32, 256)])
def test_chunk_calls_over_small_values_in_close_succession(S, new, lens, hq, hk, d, group, page):
    # parts whose units have to be looked for, among parts of ordinary size: every call gives what the first gave
    cache, q, cu, table, _ = chunk_case(S, new, lens, hq, hk, d, group, page, seed=7, tail=0)
    for i, m in enumerate(lens):
        t = torch.arange(m, device=DEV)
        at, small = table[i, t // page].long(), (t // 700 % 3 != i % 3)[:, None, None, None]
        for p, power in ((cache.k_params, -15), (cache.v_params, -22)):
            p[at, :, t % page] = torch.where(small, p[at, :, t % page] * 2.0 ** power, p[at, :, t % page])
    ln = i32(lens)
    want = cache.attend_chunk(q, cu, table, ln)
    ref, tol = lifted_reference(cache, q, new, table, lens, d ** -0.5)
    within(want, ref, tol)
    outs = [torch.zeros_like(want) for _ in range(60)]
    torch.cuda.synchronize()
    for _ in range(5):
        for o in outs:
            cache.attend_chunk(q, cu, table, ln, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    cache.query_status()
