"""The operators of the served attention block on a B200 against plain 64-bit forms.

Tolerances count roundings: half a step of a type relative to the value is U[type] = finfo.eps / 2; sums of n terms in fp32
are off by at most n U[f32] times the sum of the terms' sizes; ex2.approx and the reciprocal by 2 U[f32]."""
import math

import pytest
import torch

import serving_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float32)}
U32 = U[torch.float32]


@pytest.fixture(scope="module")
def S():
    from paper_2301_01333_b200 import build as gc_build
    gc_build.build()
    from paper_2301_01333_b200 import serving
    return serving


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(*shape, g, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(*shape, generator=g, device=DEV)).to(dtype)


def within(got, ref, tol):
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all()
    off = (got.double() - ref).abs() - tol
    assert off.max().item() <= 0, f"off by {off.max().item()} more than allowed"


# ------------------------------------------------------------------------------------------------ norm and rotation
def rope_case(S, t, hq, hk, d, rot, dtype, interleaved, norm=True, weights=True, factor=1.0, far=4096, strided=True, seed=0, pad=0):
    g = gen(seed)
    if strided:
        x = randn(t, hq + 2 * hk + 1, d + pad, g=g, dtype=dtype, scale=2.0)[..., :d]
        q, k = x[:, :hq], x[:, hq + 1:hq + 1 + hk]
    else:
        q, k = randn(t, hq, d, g=g, dtype=dtype), randn(t, hk, d, g=g, dtype=dtype)
    pos = torch.randint(-3, far, (t,), generator=g, device=DEV)
    inv = S.rotary_inv_freq(rot, device=DEV)
    qw, kw = (randn(d, g=g, dtype=dtype), randn(d, g=g, dtype=dtype)) if weights else (None, None)
    qo, ko = S.qk_norm_rope(q, k, pos, inv, qw, kw, norm=norm, eps=1e-5, interleaved=interleaved, attention_factor=factor)
    for x, w, got in ((q, qw, qo), (k, kw, ko)):
        ref, size = R.rope(x, w, pos, inv, norm, 1e-5, interleaved, factor)
        # the norm: a sum of d squares under a root (d / 2), root, quotient, two products; the rotation: angle rounded to fp32
        # below pi (4 U), sincosf (4 U), factor, two products, a sum
        tol = (d / 2 + 4 + 12) * U32 * size * abs(factor) + (U[dtype] * ref.abs() if dtype != torch.float32 else 0)
        within(got, ref, tol + 1e-30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 64), (96, 48), (80, 80), (256, 256), (192, 50), (32, 2), (18, 10), (2, 2), (128, 0)])
def test_rope_layouts(S, dtype, interleaved, d, rot):
    rope_case(S, 5, 6, 2, d, rot, dtype, interleaved)


@pytest.mark.parametrize("t,hq,hk", [(1, 1, 1), (1, 32, 8), (3, 0, 2), (7, 5, 0), (1300, 3, 1), (1501, 8, 2)])
def test_rope_sizes(S, t, hq, hk):
    rope_case(S, t, hq, hk, 128, 128, torch.bfloat16, False, seed=t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_far_positions_factor_and_options(S, dtype):
    rope_case(S, 9, 4, 4, 128, 128, dtype, False, factor=1.3, far=1 << 30)
    rope_case(S, 9, 4, 4, 64, 32, dtype, True, norm=False, factor=-0.5)
    rope_case(S, 9, 4, 4, 64, 64, dtype, False, weights=False, strided=False)
    rope_case(S, 9, 4, 4, 64, 64, dtype, False, pad=1)          # rows that are not 16-byte aligned


def test_rope_in_place_and_no_tokens(S):
    g = gen(1)
    qkv = randn(33, 10, 64, g=g, dtype=torch.bfloat16)
    q, k, rest = qkv[:, :6], qkv[:, 6:8], qkv[:, 8:].clone()
    pos, inv = torch.arange(33, device=DEV), S.rotary_inv_freq(64, device=DEV)
    qo, ko = S.qk_norm_rope(q, k, pos, inv)
    S.qk_norm_rope(q, k, pos, inv, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, 8:], rest)
    a, b = S.qk_norm_rope(q[:0], k[:0], pos[:0], inv)
    assert a.shape == (0, 6, 64) and b.shape == (0, 2, 64)


def test_rope_zero_rows_and_non_finite_rows_stay_apart(S):
    g = gen(2)
    x = randn(4, 3, 128, g=g, dtype=torch.float32)
    x[1] = 0
    x[2, 1, 7] = math.inf
    pos, inv = torch.arange(4, device=DEV), S.rotary_inv_freq(128, device=DEV)
    q, _ = S.qk_norm_rope(x, x[:, :1], pos, inv)
    assert (q[1] == 0).all() and torch.isnan(q[2, 1]).any()
    assert torch.isfinite(q[0]).all() and torch.isfinite(q[3]).all() and torch.isfinite(q[2, 0]).all()


# ------------------------------------------------------------------------------------------------ the cache
def spread(t, page, pages, g):
    order = torch.randperm(pages, generator=g, device=DEV)
    at = torch.arange(t, device=DEV)
    return order[at // page] * page + at % page


SHAPES = [(64, 32), (64, 64), (96, 32), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("t,h,page", [(1, 1, 16), (37, 3, 32), (130, 2, 256)])
def test_cache_write_and_read_are_exact(S, dtype, d, group, t, h, page):
    g = gen(t + d)
    pages = -(-t // page) + 2
    cache = S.KV4Cache.allocate(pages, page, h, d, group)
    slots = spread(t, page, pages, g)
    if t > 5:
        slots[4] = -1
    kv = randn(t, 2 * h + 1, d, g=g) * torch.exp2(3 * randn(d, g=g))
    kv[0, 0] = 1.5                                               # one value throughout: scale 0
    if t > 20:
        kv[7] = (torch.arange(d, device=DEV) % 16) * 0.5 + 0.25 * (torch.arange(d, device=DEV) % 2)    # ties between codes
        kv[8] = 0
        kv[9] = 1e-39                                            # subnormal
        kv[10] = torch.where(torch.arange(d, device=DEV) % 2 == 0, 1e-42, 3e-41)
    kv = kv.to(dtype)
    k, v = kv[:, :h], kv[:, h:2 * h]
    before = [x.clone() for x in (cache.k_codes, cache.k_params, cache.v_codes, cache.v_params)]
    cache.append(k, v, slots)
    cache.query_status()
    ok = slots >= 0
    p, o = slots[ok] // page, slots[ok] % page
    for x, codes, params, c0, p0 in ((k, cache.k_codes, cache.k_params, before[0], before[1]),
                                     (v, cache.v_codes, cache.v_params, before[2], before[3])):
        code, lo, scale = R.quantise(x[ok], group)
        got = codes[p, :, o]
        assert torch.equal(torch.stack([got & 15, got >> 4], -1).flatten(-2).double(), code)
        assert torch.equal(params[p, :, o].double(), torch.stack([lo, scale], -1))
        c0[p, :, o], p0[p, :, o] = got, params[p, :, o]          # and nothing else was written
        assert torch.equal(codes, c0) and torch.equal(params, p0)
    for out in (torch.float32, torch.bfloat16):
        ko, vo = torch.full((t, h, d), 7.0, dtype=out, device=DEV), torch.full((t, h + 1, d), 7.0, dtype=out, device=DEV)[:, :h]
        cache.read(slots, k_out=ko, v_out=vo)
        for got, codes, params in ((ko, cache.k_codes, cache.k_params), (vo, cache.v_codes, cache.v_params)):
            want = R.values(codes[p, :, o], params[p, :, o])[0].float().to(out)      # the product is exact, the sum rounded once
            assert torch.equal(got[ok], want) and (got[~ok] == 7.0).all()


def test_cache_rows_that_are_not_aligned(S):
    g = gen(5)
    cache = S.KV4Cache.allocate(3, 16, 2, 64, 32)
    x = randn(20, 4, 65, g=g, dtype=torch.bfloat16)[..., 1:]
    slots = spread(20, 16, 3, g)
    cache.append(x[:, :2], x[:, 2:], slots)
    a = cache.read(slots, torch.float32)
    y = torch.empty(20, 4, 67, device=DEV)[..., 3:]
    cache.read(slots, k_out=y[:, :2], v_out=y[:, 2:])
    assert torch.equal(a[0], y[:, :2]) and torch.equal(a[1], y[:, 2:])
    code, lo, scale = R.quantise(x[:, :2], 32)
    held = (lo[..., None] + code.unflatten(-1, (2, 32)) * scale[..., None]).flatten(-2)
    assert torch.equal(a[0].double(), held.float().double())


def test_cache_non_finite_groups_are_held_as_nan(S):
    cache = S.KV4Cache.allocate(1, 16, 1, 128, 32)
    x = torch.ones(4, 1, 128, device=DEV)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 70], x[2, 0, 71] = math.nan, -math.inf, 3e38, -3e38
    x[3, 0, 96:] = torch.arange(32, device=DEV)
    slots = torch.arange(4, device=DEV)
    cache.append(x, torch.zeros_like(x), slots)
    k, v = cache.read(slots, torch.float32)
    bad = torch.zeros(4, 4, dtype=torch.bool, device=DEV)
    bad[0, 0] = bad[1, 1] = bad[2, 2] = True
    nan = torch.isnan(k[:, 0]).unflatten(-1, (4, 32))
    assert torch.equal(nan.all(-1), bad) and torch.equal(nan.any(-1), bad) and (v == 0).all()


def test_cache_slots_out_of_bounds_are_reported(S):
    cache = S.KV4Cache.allocate(2, 16, 1, 64, 64)
    x = torch.ones(3, 1, 64, device=DEV)
    for call in (lambda s: cache.append(x, x, s), lambda s: cache.read(s)):
        call(torch.tensor([0, 32, 1], device=DEV))
        with pytest.raises(S.GcError, match="slot"):
            cache.query_status()
        cache.query_status()                                     # cleared
    assert (cache.read(torch.tensor([0, 1], device=DEV), torch.float32)[0] == 1).all()


# ------------------------------------------------------------------------------------------------ attention over the cache
def filled_cache(S, pages, page, h, d, group, g):
    cache = S.KV4Cache.allocate(pages, page, h, d, group)
    for codes, params in ((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, device=DEV, dtype=torch.uint8))
        params[..., 0] = -2.2 - 0.4 * randn(*params.shape[:-1], g=g)
        params[..., 1] = 0.2 + 0.2 * torch.rand(params.shape[:-1], generator=g, device=DEV)
    return cache


def table_of(lens, page, pages, g, width=None):
    need = [-(-n // page) for n in lens]
    width = width or max(need + [1])
    table = torch.full((len(lens), width), -7, dtype=torch.int32, device=DEV)
    order, at = torch.randperm(pages, generator=g, device=DEV).to(torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def attend_reference(cache, q, table, lens, scale, group, edge=False):
    b, n, hq, d = q.shape
    g = hq // cache.kv_heads
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(o)
    for i, m in enumerate(lens):
        if m == 0:
            continue
        pages = table[i, :-(-m // cache.page_size)].long()
        k, _ = R.values(cache.k_codes[pages].transpose(1, 2).flatten(0, 1)[:m], cache.k_params[pages].transpose(1, 2).flatten(0, 1)[:m])
        v, lo = R.values(cache.v_codes[pages].transpose(1, 2).flatten(0, 1)[:m], cache.v_params[pages].transpose(1, 2).flatten(0, 1)[:m])
        ks = cache.k_params[pages].double().abs().nan_to_num(0.).amax()
        lim = torch.arange(n, device=DEV) + (m - n + 1)
        for h in range(hq):
            qq = q[i, :, h].double()
            f = R.head if edge else R.head_all
            o[i, :, h], size = f(qq, k[:, h // g], v[:, h // g], lim, scale)
            _, coded = f(qq, k[:, h // g], (v - lo)[:, h // g], lim, scale)
            # p' = bf16(p scale): half a step of every code's part.  An exponent is a sum of d products of q and 16 + code,
            # minus 16 sum q (sizes up to 47 scale sum |q| in all, d + 4 fp32 steps): p is off by that relative to itself, and
            # so is the sum of p; then the offsets' sum and the sum over keys, in fp32 (16 / 15 and n terms, |v| + 32 scale each)
            expo = scale * ks * 47 * qq.abs().sum(-1, keepdim=True) * (d + 4) * U32 + 4 * U32
            tol[i, :, h] = U[torch.bfloat16] * coded + (2 * expo + (m / 64 + 64) * 40 * U32) * (size + 1) + U[torch.bfloat16] * o[i, :, h].abs()
    return o, tol


def attend_case(S, lens, n, hq, hk, d, group, page, seed=0, max_length=None, scale=None, qscale=1.0):
    g = gen(seed)
    pages = sum(-(-x // page) for x in lens) + 2
    cache = filled_cache(S, pages, page, hk, d, group, g)
    table = table_of(lens, page, pages, g)
    q = randn(len(lens), n, hq + 1, d, g=g, dtype=torch.bfloat16, scale=qscale)[:, :, :hq]
    out = cache.attend(q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), max_length=max_length, scale=scale)
    cache.query_status()
    ref, tol = attend_reference(cache, q, table, lens, d ** -0.5 if scale is None else scale, group)
    within(out, ref, tol)
    return cache, q, table, out


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("hq,hk", [(4, 4), (8, 2), (14, 2), (16, 1)])
def test_attend_shapes(S, d, group, page, hq, hk):
    attend_case(S, [1, 77, 0, 300, 16, 31, 33], 1, hq, hk, d, group, page, seed=d + group)


@pytest.mark.parametrize("n", [1, 2, 5, 16])
@pytest.mark.parametrize("hq,hk", [(2, 2), (12, 2), (48, 2)])
def test_attend_several_queries(S, n, hq, hk):
    attend_case(S, [n, n - 1, 1, 200, 513], n, hq, hk, 128, 64, 32, seed=n)


@pytest.mark.parametrize("lens", [[1], [256], [257], [4000], [5001, 3, 2600]])
@pytest.mark.parametrize("max_length", [None, 8192])
def test_attend_split_lengths(S, lens, max_length):
    g = gen(9)
    page = 64
    pages = sum(-(-x // page) for x in lens) + 2
    cache = filled_cache(S, pages, page, 2, 128, 64, g)
    table = table_of(lens, page, pages, g, width=128)
    q = randn(len(lens), 1, 8, 128, g=g, dtype=torch.bfloat16)
    out = cache.attend(q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), max_length=max_length)
    ref, tol = attend_reference(cache, q, table, lens, 128 ** -0.5, 64)
    within(out, ref, tol)
    again = cache.attend(q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), max_length=max_length)
    assert torch.equal(out, again)                               # joined in a fixed order
    cache.query_status()


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("lens,hq,hk", [([6000], 6, 2), ([9000, 40], 4, 2), ([700 + 97 * i for i in range(15)], 8, 8)])
def test_attend_in_many_and_in_few_pieces(S, d, group, n, lens, hq, hk):
    attend_case(S, lens, n, hq, hk, d, group, 64, seed=n + d)


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("n,hq,hk", [(1, 16, 16), (3, 32, 16), (5, 32, 8)])
def test_attend_many_short_sequences(S, d, group, n, hq, hk):
    lens = [7 * i * i % 131 for i in range(30)]
    attend_case(S, lens, n, hq, hk, d, group, 16, seed=n + d)
    attend_case(S, [x % 33 for x in lens[:7]], n, hq, hk, d, group, 32, seed=n + d + 1, max_length=32)


def test_attend_many_longer_sequences(S):
    attend_case(S, [13 * i * i % 701 + 1 for i in range(89)] + [1000], 1, 32, 16, 128, 64, 64, seed=5)


@pytest.mark.parametrize("n", [1, 3])
def test_attend_many_short_sequences_ignore_what_lies_behind(S, n):
    g = gen(19)
    b, page, h, d, group = 70, 32, 8, 128, 64
    lens = [1 + 11 * i % 95 for i in range(b)]
    cache = filled_cache(S, 3 * b, page, h, d, group, g)
    table = torch.randperm(3 * b, generator=g, device=DEV).to(torch.int32).reshape(b, 3)
    q = randn(b, n, 2 * h, d, g=g, dtype=torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = cache.attend(q, table, ln)
    ref, tol = attend_reference(cache, q, table, lens, d ** -0.5, group)
    within(want, ref, tol)
    for i, m in enumerate(lens):
        for t in range(m, 3 * page):
            for params in (cache.k_params, cache.v_params):
                params[table[i, t // page], :, t % page] = torch.tensor([math.nan, math.inf], device=DEV, dtype=torch.bfloat16)
    for i, m in enumerate(lens):                                 # pages behind the last are not looked at either
        table[i, -(-m // page):] = 1 << 30
    assert torch.equal(cache.attend(q, table, ln), want)
    cache.query_status()
    ln[5], ln[6] = 97, -1
    cache.attend(q, table, ln)
    with pytest.raises(S.GcError):
        cache.query_status()


def test_attend_scores_that_rise_and_fall(S):
    # scores of hundreds of binades in both directions: the reference has to be raised many times, and old parts vanish
    attend_case(S, [700, 129], 1, 8, 2, 128, 32, 16, seed=3, qscale=40.0)
    attend_case(S, [700, 129], 2, 8, 2, 64, 64, 16, seed=4, scale=3.0)


@pytest.mark.parametrize("d,group", SHAPES)
def test_attend_ignores_what_lies_behind_a_sequence(S, d, group):
    g = gen(11)
    lens, page, n = [37, 5, 18], 32, 3
    cache = filled_cache(S, 5, page, 2, d, group, g)
    table = table_of(lens, page, 5, g)
    for b, m in enumerate(lens):                                 # infinities and NaN in every slot behind the last token
        last = table[b, (m - 1) // page]
        for params in (cache.k_params, cache.v_params):
            params[last, :, m % page or page:] = torch.tensor([math.nan, math.inf], device=DEV, dtype=torch.bfloat16)
    for params in (cache.k_params, cache.v_params):              # and in the newest token of one sequence: its last query's business
        params[table[0, 36 // page], :, 36 % page] = math.nan
    q = randn(3, n, 4, d, g=g, dtype=torch.bfloat16)
    out = cache.attend(q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
    ref, tol = attend_reference(cache, q, table, lens, d ** -0.5, group, edge=True)
    assert torch.isnan(out[0, 2]).all()
    out[0, 2], ref[0, 2], tol[0, 2] = 0, 0, 0
    within(out, ref, tol)


@pytest.mark.parametrize("power", [30, -36])
def test_attend_values_of_unlike_size(S, power):
    # values times a power of two: every step scales with it exactly, and nothing overflows or vanishes
    cache, q, table, out = attend_case(S, [900, 33, 257], 2, 8, 2, 128, 32, 16, seed=5)
    cache.v_params.mul_(2.0 ** power)
    cache.k_params.mul_(2.0 ** power)
    big = cache.attend((q.float() * 2.0 ** -power).bfloat16(), table, torch.tensor([900, 33, 257], dtype=torch.int32, device=DEV))
    assert torch.equal(big, out * 2.0 ** power)


def test_attend_reports_bad_pages_and_lengths(S):
    g = gen(12)
    cache = filled_cache(S, 4, 16, 1, 64, 64, g)
    q = randn(2, 1, 2, 64, g=g, dtype=torch.bfloat16)
    table = torch.tensor([[0, 4], [1, 2]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([20, 20], dtype=torch.int32, device=DEV)
    out = cache.attend(q, table, lens)
    with pytest.raises(S.GcError, match="page"):
        cache.query_status()
    ref, tol = attend_reference(cache, q[1:], table[1:], [20], 0.125, 64)
    within(out[1:], ref, tol)                                    # the other sequence is untouched by it
    for bad in ([33, 1], [-1, 1]):
        cache.attend(q, torch.zeros_like(table), torch.tensor(bad, dtype=torch.int32, device=DEV))
        with pytest.raises(S.GcError, match="length"):
            cache.query_status()
    cache.attend(q, torch.zeros_like(table), torch.tensor([32, 0], dtype=torch.int32, device=DEV), max_length=32)
    cache.query_status()


# ------------------------------------------------------------------------------------------------ prompts
def prompt_case(S, nq, nk, hq, hk, d, causal, seed=0, tail=0, scale=None, qscale=1.0, poison=False):
    g = gen(seed)
    cu_q = torch.tensor([0] + nq, device=DEV).cumsum(0).to(torch.int32)
    cu_k = torch.tensor([0] + nk, device=DEV).cumsum(0).to(torch.int32)
    tq, tk = sum(nq) + tail, sum(nk) + tail
    q = randn(tq, hq + 1, d, g=g, dtype=torch.bfloat16, scale=qscale)[:, :hq]
    kv = randn(tk, 2 * hk, d, g=g, dtype=torch.bfloat16)
    k, v = kv[:, :hk], kv[:, hk:]
    if poison:                                                   # rows no sequence owns hold anything
        k[sum(nk):], v[sum(nk):], q[sum(nq):] = math.nan, math.inf, math.nan
    out = torch.full((tq, hq, d), 0.25, dtype=torch.bfloat16, device=DEV)
    status = S.new_status(DEV)
    S.attention_prompt(q, k, v, cu_q, cu_k, causal=causal, out=out, scale=scale, status=status)
    S.query_status(status)
    c = d ** -0.5 if scale is None else scale
    for b in range(len(nq)):
        a0, a1, c0, c1 = int(cu_q[b]), int(cu_q[b + 1]), int(cu_k[b]), int(cu_k[b + 1])
        lim = torch.arange(a1 - a0, device=DEV) + (nk[b] - nq[b] + 1) if causal else torch.full((a1 - a0,), nk[b], device=DEV)
        for h in range(hq):
            if a1 == a0:
                continue
            qq = q[a0:a1, h].double()
            kk, vv = k[c0:c1, h // (hq // hk)].double(), v[c0:c1, h // (hq // hk)].double()
            ref, size = R.head_all(qq, kk, vv, lim, c)
            big = (qq.abs() @ kk.abs().T).amax(-1, keepdim=True) if c1 > c0 else torch.zeros(a1 - a0, 1, device=DEV)
            # p rounded to bf16 (half a step of every term); exponents: d fp32 steps of their size, and the reference; sums over
            # nk keys in fp32; the output's rounding
            tol = U[torch.bfloat16] * size + 2 * (c * big * (d + 4) * U32 + 4 * U32) * size + (nk[b] / 16 + 16) * U32 * size + U[torch.bfloat16] * ref.abs()
            within(out[a0:a1, h], ref, tol)
    assert (out[sum(nq):] == 0.25).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 255, 256, 257, 400])
def test_prompt_lengths(S, causal, d, n):
    prompt_case(S, [n], [n], 2, 1, d, causal, seed=n)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_prompt_packed(S, causal, d):
    n = [3, 0, 200, 1, 513, 64, 0, 130]
    prompt_case(S, n, n, 6, 2, d, causal, seed=d, tail=70, poison=True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("n", [1, 127, 128, 129, 255, 256, 257, 400])
def test_prompt_lengths_of_many_heads(S, causal, d, n):
    prompt_case(S, [n, 130, 0, n + 3], [n + 1, 130, 5, n], 40, 8, d, causal, seed=n, tail=3, poison=True)


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_continued_and_rows_that_see_nothing(S, causal):
    prompt_case(S, [5, 300, 1, 7, 260, 40], [700, 301, 129, 0, 3, 40], 4, 4, 128, causal, seed=1)
    prompt_case(S, [5, 300, 1, 7, 260, 40], [128, 301, 256, 0, 140, 39], 3, 1, 64, causal, seed=2)


def test_prompt_without_any_key_and_without_any_row(S):
    prompt_case(S, [3, 300], [0, 0], 2, 1, 64, True, seed=1)
    x = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    cu = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert S.attention_prompt(x, x, x, cu).shape == (0, 2, 64)
    y = torch.full((4, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    assert (S.attention_prompt(y, y, y, cu[:1], out=y.clone()) == 3.0).all()          # no sequence: nothing is written


def test_prompt_more_work_than_ctas(S):
    prompt_case(S, [900, 17, 1500, 333], [900, 17, 1500, 333], 16, 4, 128, True, seed=3)
    prompt_case(S, [900, 17, 1500, 333], [1000, 900, 1600, 333], 32, 32, 64, True, seed=4)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [[1024], [1025], [1407], [1536, 1100], [2049, 0, 1300, 1027]])
def test_prompt_long_sequences_of_wide_heads(S, causal, n):
    # 1024 tokens a sequence and more on average: pairs of CTAs, 512 rows each
    prompt_case(S, n, n, 4, 2, 128, causal, seed=len(n) + n[0], tail=40, poison=True)


def test_prompt_long_sequences_continued(S):
    prompt_case(S, [1300, 1, 1800], [1300 + 333, 129, 1700], 3, 3, 128, True, seed=13, tail=5, poison=True)
    prompt_case(S, [1300, 900, 1800], [0, 40, 2000], 2, 1, 128, False, seed=14)
    prompt_case(S, [4100], [4100], 20, 4, 128, True, seed=15)
    prompt_case(S, [1200], [1200], 2, 2, 128, True, seed=16, qscale=30.0)


def test_prompt_many_sequences(S):
    # more pieces than the sorted work list holds
    g = torch.Generator().manual_seed(0)
    n = torch.randint(0, 5, (1400,), generator=g).tolist()
    n[700] = 300
    prompt_case(S, n, n, 1, 1, 64, True, seed=5)


def test_prompt_scores_that_rise(S):
    prompt_case(S, [700], [700], 2, 2, 128, True, seed=6, qscale=30.0)
    prompt_case(S, [700], [700], 2, 2, 64, False, seed=7, scale=4.0)


def test_prompt_neighbours_that_are_not_finite(S):
    # keys, values and queries of one sequence hold NaN and infinities: its neighbours, whose tiles reach into it, stay clean;
    # so do the rows before a NaN key of their own sequence
    g = gen(8)
    cu = torch.tensor([0, 130, 258, 328], dtype=torch.int32, device=DEV)
    q, k, v = (randn(328, 2, 64, g=g, dtype=torch.bfloat16) for _ in range(3))
    clean = S.attention_prompt(q, k, v, cu)
    q[130:258], k[130:200], v[130:258] = math.nan, math.inf, math.inf
    k[129], k[327] = math.nan, math.nan
    got = S.attention_prompt(q, k, v, cu)
    keep = torch.ones(328, dtype=torch.bool, device=DEV)
    keep[129:258], keep[327] = False, False
    assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[[129, 327]]).all()


def test_prompt_offsets_out_of_bounds_are_reported(S):
    q = torch.zeros(300, 2, 64, dtype=torch.bfloat16, device=DEV)
    for cu in ([0, 200, 100, 300], [0, 301, 301, 301], [-1, 10, 20, 300]):
        status = S.new_status(DEV)
        S.attention_prompt(q, q, q, torch.tensor(cu, dtype=torch.int32, device=DEV), status=status)
        with pytest.raises(S.GcError, match="offsets"):
            S.query_status(status)


# ------------------------------------------------------------------------------------------------ together, streams, graphs
class Block:
    """An attention block as a server would run it: projections are given; norm and rotation, cache, attention."""

    def __init__(self, S, hq, hk, d, page, pages, group, seed):
        g = gen(seed)
        self.S, self.hq, self.hk, self.d, self.page = S, hq, hk, d, page
        self.cache = S.KV4Cache.allocate(pages, page, hk, d, group)
        self.inv = S.rotary_inv_freq(d, scaling="bands", factor=4.0, original_length=256, device=DEV)
        self.qw, self.kw = 1 + 0.1 * randn(d, g=g, dtype=torch.bfloat16), 1 + 0.1 * randn(d, g=g, dtype=torch.bfloat16)

    def turn(self, qkv, pos):
        q, k = self.S.qk_norm_rope(qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hk], pos, self.inv, self.qw, self.kw)
        return q, k, qkv[:, self.hq + self.hk:]


@pytest.mark.parametrize("d,group,hq,hk", [(128, 32, 8, 2), (64, 64, 12, 12), (96, 32, 6, 1)])
def test_block_prompt_then_steps(S, d, group, hq, hk):
    """Two prompts, then three steps of one token and one of two: each query's output against 64-bit attention over what
    the cache holds (the prompt's own attention over the values read back from it), from the same rotated queries."""
    g = gen(40 + d)
    page, lens = 16, [70, 33]
    blk = Block(S, hq, hk, d, page, 16, group, 41)
    table = torch.tensor([[3, 1, 4, 15, 9, 2], [6, 5, 8, 7, 0, 10]], dtype=torch.int32, device=DEV)

    def slots(b, first, n):
        t = torch.arange(first, first + n, device=DEV)
        return table[b, t // page].long() * page + t % page
    # prompts
    qkv = randn(sum(lens), hq + 2 * hk, d, g=g, dtype=torch.bfloat16)
    pos = torch.cat([torch.arange(n, device=DEV) for n in lens])
    where = torch.cat([slots(b, 0, n) for b, n in enumerate(lens)])
    q, k, v = blk.turn(qkv, pos)
    blk.cache.append(k, v, where)
    k_held, v_held = blk.cache.read(where)
    cu = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device=DEV)
    status = S.new_status(DEV)
    out = S.attention_prompt(q, k_held, v_held, cu, status=status)
    S.query_status(status)
    start = 0
    for b, n in enumerate(lens):
        for h in range(hq):
            kk, vv = k_held[start:start + n, h // (hq // hk)].double(), v_held[start:start + n, h // (hq // hk)].double()
            ref, size = R.head_all(q[start:start + n, h].double(), kk, vv, torch.arange(1, n + 1, device=DEV), d ** -0.5)
            expo = d ** -0.5 * (q[start:start + n, h].double().abs() @ kk.abs().T).amax(-1, keepdim=True) * (d + 4) * U32 + 4 * U32
            within(out[start:start + n, h], ref, (2 * U[torch.bfloat16] + 2 * expo + 100 * U32) * size)
        start += n
    # steps
    for n in (1, 1, 1, 2):
        qkv = randn(2 * n, hq + 2 * hk, d, g=g, dtype=torch.bfloat16)
        pos = torch.cat([torch.arange(m, m + n, device=DEV) for m in lens])
        q, k, v = blk.turn(qkv, pos)
        blk.cache.append(k, v, torch.cat([slots(b, m, n) for b, m in enumerate(lens)]))
        lens = [m + n for m in lens]
        q = q.unflatten(0, (2, n))
        out = blk.cache.attend(q, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
        ref, tol = attend_reference(blk.cache, q, table, lens, d ** -0.5, group)
        within(out, ref, tol)
    blk.cache.query_status()


def _step_inputs(S, seed, t=64, hq=8, hk=2, d=128, page=32):
    g = gen(seed)
    blk = Block(S, hq, hk, d, page, 400, 64, seed)
    lens = torch.randint(2000, 2600, (3,), generator=g, device=DEV).to(torch.int32)
    table = torch.randperm(400, generator=g, device=DEV).to(torch.int32)[:300].reshape(3, 100)
    qkv = randn(3, hq + 2 * hk, d, g=g, dtype=torch.bfloat16)
    for codes, params in ((blk.cache.k_codes, blk.cache.k_params), (blk.cache.v_codes, blk.cache.v_params)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, device=DEV, dtype=torch.uint8))
        params[..., 0] = -1 + 0.1 * randn(*params.shape[:-1], g=g)
        params[..., 1] = 0.1
    prompt = randn(700, hq + 2 * hk, d, g=g, dtype=torch.bfloat16)
    cu = torch.tensor([0, 300, 301, 700], dtype=torch.int32, device=DEV)

    def step():
        q, k, v = blk.turn(qkv, (lens - 1).long())
        last = (lens - 1).long()
        blk.cache.append(k, v, table.gather(1, (last // page)[:, None])[:, 0].long() * page + last % page)
        kr, vr = blk.cache.read(last)
        o = blk.cache.attend(q[:, None], table, lens, max_length=3200)
        p = S.attention_prompt(prompt[:, :hq], prompt[:, hq:hq + hk], prompt[:, hq + hk:], cu)
        return [q, k, kr, vr, o, p]
    return step, qkv, blk


def test_two_captured_graphs_share_nothing(S):
    steps = [_step_inputs(S, s) for s in (51, 52)]
    want = [[x.clone() for x in step()] for step, _, _ in steps]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for step, _, _ in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        for o in outs:
            for x in o:
                x.fill_(math.nan)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):                        # both at once, on streams of their own
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
    for (_, qkv, blk), o, g, w in zip(steps, outs, graphs, want):   # a replay sees new inputs
        qkv.copy_(-qkv)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o[0], -w[0]) and not torch.equal(o[4], w[4])
        blk.cache.query_status()


def test_calls_on_a_stream_of_their_own(S):
    step, qkv, _ = _step_inputs(S, 61)
    want = [x.clone() for x in step()]
    real = qkv.clone()
    qkv.zero_()
    step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        qkv.copy_(real)                                          # a launch on another stream would overtake this, and see zeros
        got = step()
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_that_follow_one_another_closely(S):
    # each call reads what the one before it wrote (or overwrites what it read), with nothing of another kind in between; rows
    # begin in the middle of a memory sector.  Against the same calls with the device at rest between them.
    g = gen(81)
    b, hq, hk, d, page, rounds = 300, 8, 2, 64, 16, 24
    room = randn(b * (hq + 2 * hk) * d + 8, g=g, dtype=torch.bfloat16)
    begin = room.clone()
    rows = room[8:].view(b, hq + 2 * hk, d)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    pages = -(-rounds // page)
    table = torch.randperm(b * pages, generator=g, device=DEV).to(torch.int32).reshape(b, pages)
    inv = S.rotary_inv_freq(d, device=DEV)
    pos = [torch.randint(0, 5000, (b,), generator=g, device=DEV) for _ in range(rounds)]
    slots = [table[:, i // page].long() * page + i % page for i in range(rounds)]
    lens = [torch.full((b,), i + 1, dtype=torch.int32, device=DEV) for i in range(rounds)]
    cu = torch.arange(b + 1, dtype=torch.int32, device=DEV)
    cache = S.KV4Cache.allocate(b * pages, page, hk, d, 32)
    mid = torch.empty(b, 1, hq, d, dtype=torch.bfloat16, device=DEV)

    def run(between):
        room.copy_(begin)
        for x in (cache.k_codes, cache.k_params, cache.v_codes, cache.v_params):
            x.zero_()
        kept = []
        for i in range(rounds):
            S.qk_norm_rope(q, k, pos[i], inv, q_out=q, k_out=k)
            between()
            cache.append(k, v, slots[i])
            between()
            cache.attend(q[:, None], table, lens[i], out=mid)
            between()
            S.attention_prompt(mid[:, 0], k, v, cu, out=q)
            between()
            cache.read(slots[i], k_out=k, v_out=v)
            between()
            if i % 6 == 5:
                kept.append((room.clone(), mid.clone()))
        return kept + [(cache.k_codes.clone(), cache.v_params.clone())]
    want = run(torch.cuda.synchronize)
    run(lambda: None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(lambda: None)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    cache.query_status()


def test_results_do_not_depend_on_the_run(S):
    step, _, _ = _step_inputs(S, 71)
    first = [x.clone() for x in step()]
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(step(), first))


def test_cache_of_more_than_two_to_the_32_bytes(S):
    # codes beyond 4 GB: the last pages of a cache of 270000 pages of 256 tokens, one head of 128
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("not enough memory")
    pages, page = 270000, 256
    assert pages * page * 64 > 1 << 32
    cache = S.KV4Cache.allocate(pages, page, 1, 128, 128)
    g = gen(81)
    n = 300
    k, v = randn(n, 1, 128, g=g, dtype=torch.bfloat16), randn(n, 1, 128, g=g, dtype=torch.bfloat16)
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device=DEV)
    t = torch.arange(n, device=DEV)
    slots = table[0, t // page].long() * page + t % page
    cache.append(k, v, slots)
    code, lo, scale = R.quantise(k, 128)
    kr, _ = cache.read(slots, torch.float32)
    assert torch.equal(kr.double(), (lo + code * scale).float().double())
    q = randn(1, 1, 4, 128, g=g, dtype=torch.bfloat16)
    out = cache.attend(q, table, torch.tensor([n], dtype=torch.int32, device=DEV))
    ref, tol = attend_reference(cache, q, table, [n], 128 ** -0.5, 128)
    within(out, ref, tol)
    cache.query_status()


def test_refusals_leave_everything_as_it_was(S):
    cache = S.KV4Cache.allocate(4, 16, 2, 64, 32)
    x = torch.ones(3, 2, 64, device=DEV, dtype=torch.bfloat16)
    slots = torch.arange(3, device=DEV)
    q = torch.ones(1, 1, 4, 64, device=DEV, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    out = torch.full((3, 2, 64), 5.0, device=DEV, dtype=torch.bfloat16)
    inv = S.rotary_inv_freq(64, device=DEV)
    V, T, G = ValueError, TypeError, S.GcError
    cases = [
        (V, lambda: cache.append(x[:2], x, slots)), (V, lambda: cache.append(x, x.float(), slots)), (T, lambda: cache.append(x.half(), x.half(), slots)),
        (V, lambda: cache.append(x, x, slots.int())), (V, lambda: cache.append(x.cpu(), x, slots)), (V, lambda: cache.append(x, x, slots[None])),
        (V, lambda: cache.append(x.transpose(1, 2).contiguous().transpose(1, 2), x, slots)),
        (V, lambda: cache.read(slots, k_out=out[:1].expand(3, 2, 64), v_out=out)), (T, lambda: cache.read(slots, torch.float16)),
        (V, lambda: cache.attend(q.float(), table, lens)), (V, lambda: cache.attend(q[..., :32], table, lens)), (V, lambda: cache.attend(q, table.long(), lens)),
        (V, lambda: cache.attend(q, table, lens.long())), (V, lambda: cache.attend(q, table.expand(2, 4), lens)), (G, lambda: cache.attend(q, table, lens, max_length=65)),
        (G, lambda: cache.attend(q, table, lens, max_length=-1)), (G, lambda: cache.attend(q, table, lens, scale=0.0)), (G, lambda: cache.attend(q, table, lens, scale=math.nan)),
        (G, lambda: cache.attend(q[:, :, :3], table, lens)), (G, lambda: cache.attend(q.expand(1, 17, 4, 64), table, lens)),
        (V, lambda: cache.attend(q, table, lens, out=q[:, :, :1].expand(1, 1, 4, 64))),
        (G, lambda: cache.attend(torch.ones(1, 1, 4, 65, device=DEV, dtype=torch.bfloat16)[..., 1:], table, lens)),
        (V, lambda: S.attention_prompt(x.float(), x, x, cu)), (V, lambda: S.attention_prompt(x, x[:, :, :32], x, cu)), (G, lambda: S.attention_prompt(x, x, x, cu, scale=-1.0)),
        (V, lambda: S.attention_prompt(x, x, x, cu.long())), (V, lambda: S.attention_prompt(x, x, x, cu, cu[:1])), (V, lambda: S.attention_prompt(x, x, x, cu, out=out[:1])),
        (V, lambda: S.attention_prompt(x, x, x, cu, out=out[:1].expand(3, 2, 64))), (G, lambda: S.attention_prompt(x[..., :32], x[..., :32], x[..., :32], cu)),
        (G, lambda: S.attention_prompt(x, torch.ones(3, 3, 64, device=DEV, dtype=torch.bfloat16), torch.ones(3, 3, 64, device=DEV, dtype=torch.bfloat16), cu)),
        (G, lambda: S.attention_prompt(x, x[:, :1].expand(3, 2, 64), x, cu)),
        (V, lambda: S.qk_norm_rope(x, x, slots.int(), inv)), (V, lambda: S.qk_norm_rope(x, x.float(), slots, inv)), (T, lambda: S.qk_norm_rope(x.half(), x.half(), slots, inv)),
        (G, lambda: S.qk_norm_rope(x, x, slots, torch.ones(33, device=DEV))), (G, lambda: S.qk_norm_rope(x, x, slots, inv, eps=-1.0)),
        (V, lambda: S.qk_norm_rope(x, x, slots, inv, x[0, 0].float())), (V, lambda: S.qk_norm_rope(x, x, slots, inv, q_out=out[:1].expand(3, 2, 64))),
        (G, lambda: S.qk_norm_rope(x[..., :63], x[..., :63], slots, inv[:8])), (T, lambda: S.qk_norm_rope(x, None, slots, inv)),
    ]
    for i, (kind, call) in enumerate(cases):
        with pytest.raises(kind):
            call()
            print("case", i, "was not refused")
    assert (cache.k_codes == 0).all() and (cache.v_params == 0).all() and (out == 5.0).all()
    cache.query_status()
