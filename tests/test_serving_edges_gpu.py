"""The operators of the served attention block on a B200, at the edges of what their documentation allows: numbers that are not
finite, batches that are laid out in unusual ways, calls right behind what wrote their inputs."""
import math

import pytest
import torch

import serving_reference as R
from test_serving_gpu import (DEV, S, attend_reference, filled_cache, gen, prompt_case, randn, rope_case, table_of,  # noqa: F401 (S: the fixture)
                              within)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ numbers that are not finite
@pytest.mark.parametrize("d,group", [(64, 64), (96, 32), (128, 32), (128, 128)])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("lens,bound", [([33, 5, 18], 96), ([20, 31, 32], 32), ([2000, 150, 6000], 6016)])
def test_attend_of_queries_that_are_not_finite(S, d, group, n, lens, bound):
    # a query that holds a NaN has no finite score: its output is NaN, in one piece or many, and no other query's is touched
    g = gen(d + n)
    page, hk, hq = 32, 2, 6
    pages = sum(-(-x // page) for x in lens) + 2
    cache = filled_cache(S, pages, page, hk, d, group, g)
    table = table_of(lens, page, pages, g, width=bound // page)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = randn(len(lens), n, hq, d, g=g, dtype=torch.bfloat16)
    want = cache.attend(q, table, ln, max_length=bound)
    q[0, n - 1, 1, 5] = math.nan
    q[2, 0, 4] = math.nan
    got = cache.attend(q, table, ln, max_length=bound)
    bad = torch.zeros(got.shape[:3], dtype=torch.bool, device=DEV)
    bad[0, n - 1, 1] = bad[2, 0, 4] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])
    cache.query_status()


@pytest.mark.parametrize("d,group", [(64, 64), (96, 32), (128, 64)])
@pytest.mark.parametrize("lens,bound", [([40, 33], 96), ([32, 9], 32), ([3000, 600], 3008)])
def test_attend_over_keys_that_are_all_held_as_nan(S, d, group, lens, bound):
    # every key of one head is held as NaN, so no score is a number: the queries of that head are NaN, those of the other are not
    g = gen(d)
    page, hk, hq = 32, 2, 4
    pages = sum(-(-x // page) for x in lens) + 2
    cache = filled_cache(S, pages, page, hk, d, group, g)
    table = table_of(lens, page, pages, g, width=bound // page)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = randn(len(lens), 1, hq, d, g=g, dtype=torch.bfloat16)
    want = cache.attend(q, table, ln, max_length=bound)
    cache.k_params[:, 0] = math.nan
    got = cache.attend(q, table, ln, max_length=bound)
    assert torch.isnan(got[:, :, :2]).all() and torch.equal(got[:, :, 2:], want[:, :, 2:])
    cache.query_status()


def test_attend_over_a_stretch_of_keys_held_as_nan(S):
    # one stretch of 700 tokens, more than any warp's tiles in a row: whoever sees it is NaN
    g = gen(3)
    page, m = 64, 5000
    cache = filled_cache(S, 80, page, 1, 128, 128, g)
    table = table_of([m, m], page, 160, g)[:1].clamp(max=79)
    table[0] = torch.randperm(80, generator=g, device=DEV)[:table.shape[1]].to(torch.int32)
    ln = torch.tensor([m], dtype=torch.int32, device=DEV)
    q = randn(1, 1, 4, 128, g=g, dtype=torch.bfloat16)
    for t in range(1200, 1900):
        cache.k_params[table[0, t // page], :, t % page] = math.nan
    assert torch.isnan(cache.attend(q, table, ln)).all()
    ln[0] = 1200
    ref, tol = attend_reference(cache, q, table, [1200], 128 ** -0.5, 128)
    within(cache.attend(q, table, ln), ref, tol)


# ------------------------------------------------------------------------------------------------ next to the framework's other kernels
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_between_attention_subgraphs(S, d):
    # both kinds hold tensor memory, and blocks of both fit on an SM side by side: calls right behind one another, in a captured
    # graph too, give what they give alone
    from paper_2301_01333_b200 import binding as B
    from paper_2301_01333_b200 import workloads as W
    w = W.mha_bf16(batch=16, heads=12, seq=128, head_dim=64)
    part = B.CompiledPartition(w.graph, 0)
    ins, outs = B.device_inputs(w), B.device_outputs(w.graph)
    g = gen(d)
    n = [100, 30, 700, 1, 260]
    cu = torch.tensor([0] + n, device=DEV).cumsum(0).to(torch.int32)
    x = randn(sum(n), 12, d, g=g, dtype=torch.bfloat16)
    o = torch.zeros(sum(n), 8, d, dtype=torch.bfloat16, device=DEV)
    status = S.new_status(DEV)

    def prompt():
        S.attention_prompt(x[:, :8], x[:, 8:10], x[:, 10:], cu, out=o, status=status)
    part.execute(ins, outs)
    prompt()
    torch.cuda.synchronize()
    want = o.clone(), outs[0].clone()

    def run():
        for _ in range(20):
            part.execute(ins, outs)
            prompt()
            prompt()
            part.execute(ins, outs)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        o.fill_(math.nan)
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(outs[0], want[1])
    S.query_status(status)
    part.query_status()
    del graph
    part.close()


# ------------------------------------------------------------------------------------------------ right behind what wrote the inputs
@pytest.mark.parametrize("lens,hq,hk,n", [([2046], 8, 2, 1), ([1278, 3070, 126, 5], 8, 8, 2), ([1023 + 128 * i for i in range(20)], 4, 1, 1)])
def test_attend_right_behind_the_kernel_that_moves_the_lengths(S, lens, hq, hk, n):
    # a captured step that adds one to the lengths in place, directly before attention in pieces, over the border of a block of 128
    g = gen(len(lens))
    page, bound = 64, 4096
    pages = sum(-(-(x + 8) // page) for x in lens)
    cache = filled_cache(S, pages, page, hk, 128, 64, g)
    table = table_of([x + 8 for x in lens], page, pages, g, width=bound // page)
    q = randn(len(lens), n, hq, 128, g=g, dtype=torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    start = ln.clone()
    want = []
    for i in range(6):
        fresh = start + (i + 1)
        torch.cuda.synchronize()
        want.append(cache.attend(q, table, fresh, max_length=bound))
    ref, tol = attend_reference(cache, q, table, [x + 6 for x in lens], 128 ** -0.5, 64)
    within(want[-1], ref, tol)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ln.add_(1)
        cache.attend(q, table, ln, max_length=bound, out=out)
    for rep in range(4):
        ln.copy_(start)
        for w in want:                                           # one replay behind the other, nothing in between but the copy
            graph.replay()
            assert torch.equal(out.clone(), w)
    one = torch.cuda.CUDAGraph()
    outs = [torch.empty_like(q) for _ in want]
    with torch.cuda.graph(one):                                  # and all steps in one graph
        for o in outs:
            ln.add_(1)
            cache.attend(q, table, ln, max_length=bound, out=o)
    for rep in range(4):
        ln.copy_(start)
        one.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    cache.query_status()


# ------------------------------------------------------------------------------------------------ prompts in unusual batches
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hk", [(64, 6, 2), (128, 16, 4), (96, 5, 5)])
def test_prompt_batches_beyond_the_work_list(S, causal, d, hq, hk):
    # more pieces than the sorted list holds, several heads, sequences of several pieces among empty ones: bit for bit what the same
    # sequences give a hundred at a time, and a few of them against 64 bits
    r = torch.Generator().manual_seed(d)
    n = torch.randint(0, 40, (2500,), generator=r)
    n[torch.randint(0, 2500, (300,), generator=r)] = 0
    n[[3, 900, 901, 2499]] = torch.tensor([700, 257, 513, 1100])
    lens = n.tolist()
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    g = gen(d)
    x = randn(int(cu[-1]) + 9, hq + 2 * hk, d, g=g, dtype=torch.bfloat16)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    status = S.new_status(DEV)
    out = torch.full((x.shape[0], hq, d), 0.25, dtype=torch.bfloat16, device=DEV)
    S.attention_prompt(q, k, v, cu.to(DEV), causal=causal, out=out, status=status)
    S.query_status(status)
    assert (out[int(cu[-1]):] == 0.25).all()
    for b0 in range(0, 2500, 100):
        t0, t1 = int(cu[b0]), int(cu[b0 + 100])
        part = S.attention_prompt(q[t0:t1], k[t0:t1], v[t0:t1], (cu[b0:b0 + 101] - t0).to(DEV), causal=causal)
        assert torch.equal(out[t0:t1], part)
    U = torch.finfo(torch.bfloat16).eps / 2
    for b in (0, 3, 900, 1501, 2499):
        t0, m = int(cu[b]), lens[b]
        if m == 0:
            continue
        lim = torch.arange(1, m + 1, device=DEV) if causal else torch.full((m,), m, device=DEV)
        for h in range(hq):
            ref, size = R.head_all(q[t0:t0 + m, h].double(), k[t0:t0 + m, h // (hq // hk)].double(), v[t0:t0 + m, h // (hq // hk)].double(), lim, d ** -0.5)
            # probabilities rounded to bf16 and the output's own rounding; what fp32 adds is below a hundredth of that
            within(out[t0:t0 + m, h], ref, 1.01 * U * size + U * ref.abs() + 1e-6)


def test_prompt_work_grows_with_the_batch_and_not_with_its_square(S):
    def took(batch):
        x = torch.zeros(batch, 1, 64, dtype=torch.bfloat16, device=DEV)
        cu, out = torch.arange(batch + 1, dtype=torch.int32, device=DEV), torch.empty_like(x)
        best = math.inf
        for _ in range(5):
            begin, end = torch.cuda.Event(True), torch.cuda.Event(True)
            torch.cuda.synchronize()
            begin.record()
            S.attention_prompt(x, x, x, cu, out=out)
            end.record()
            end.synchronize()
            best = min(best, begin.elapsed_time(end))
        return best
    assert took(16000) < 60 * took(1000)                         # sixteen times the work; searched from the start each time, it is hundreds


# ------------------------------------------------------------------------------------------------ gradients
def test_tensors_that_require_a_gradient_are_refused(S):
    x = torch.ones(3, 2, 64, device=DEV, dtype=torch.bfloat16)
    g = x.clone().requires_grad_()
    w = torch.nn.Parameter(x[0, 0].clone())
    pos, inv = torch.arange(3, device=DEV), S.rotary_inv_freq(64, device=DEV)
    cu = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    cache = S.KV4Cache.allocate(2, 16, 2, 64, 32)
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    cache.append(x, x, pos)
    calls = [lambda: S.qk_norm_rope(g, x, pos, inv), lambda: S.qk_norm_rope(x, g, pos, inv), lambda: S.qk_norm_rope(x, x, pos, inv, w),
             lambda: S.qk_norm_rope(x, x, pos, inv, None, w), lambda: S.qk_norm_rope(x, x, pos, inv, q_out=g.clone()),
             lambda: S.qk_norm_rope(x, x, pos, inv, k_out=g.clone()), lambda: cache.append(g, x, pos), lambda: cache.append(x, g, pos),
             lambda: cache.read(pos, k_out=g.clone()), lambda: cache.read(pos, v_out=g.clone()), lambda: cache.attend(g[None, :1], table, lens),
             lambda: cache.attend(x[None, :1], table, lens, out=g[None, :1].clone()), lambda: S.attention_prompt(g, x, x, cu),
             lambda: S.attention_prompt(x, g, x, cu), lambda: S.attention_prompt(x, x, g, cu), lambda: S.attention_prompt(x, x, x, cu, out=g.clone())]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="gradient"):
            call()
            print("call", i, "was not refused")
    with torch.no_grad():
        for call in calls:
            call()
    with torch.inference_mode():
        S.qk_norm_rope(x, x, pos, inv, w)
    cache.query_status()


def test_outputs_that_were_given_count_as_written(S):
    # what autograd keeps for a backward pass and a call then overwrites is missed there, as after any write in place
    x = torch.ones(3, 2, 64, device=DEV, dtype=torch.bfloat16)
    pos, inv = torch.arange(3, device=DEV), S.rotary_inv_freq(64, device=DEV)
    cu = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    cache = S.KV4Cache.allocate(2, 16, 2, 64, 32)
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    a, b = torch.empty_like(x), torch.empty_like(x)
    one = torch.empty(1, 1, 2, 64, device=DEV, dtype=torch.bfloat16)
    for call, outs in ((lambda: S.qk_norm_rope(x, x, pos, inv, q_out=a, k_out=b), (a, b)),
                       (lambda: cache.append(x, x, pos), (cache.k_codes, cache.k_params, cache.v_codes, cache.v_params)),
                       (lambda: cache.read(pos, k_out=a, v_out=b), (a, b)), (lambda: cache.attend(x[None, :1], table, lens, out=one), (one,)),
                       (lambda: S.attention_prompt(x, x, x, cu, out=a), (a,))):
        before = [t._version for t in outs]
        inputs = x._version
        call()
        assert [t._version for t in outs] == [v + 1 for v in before] and x._version == inputs
    w = torch.ones_like(a).requires_grad_()
    y = (w * a).sum()
    S.attention_prompt(x, x, x, cu, out=a)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    with torch.inference_mode():                                 # tensors without a count
        c = torch.empty_like(x)
        S.attention_prompt(x, x, x, cu, out=c)
    cache.query_status()


# ------------------------------------------------------------------------------------------------ the cache's memory
def test_a_cache_is_made_for_its_tensors(S):
    # the kernels get pointers that were taken once: other tensors, or other memory under the same ones, must not go unnoticed
    cache = S.KV4Cache.allocate(2, 16, 2, 64, 32)
    x, slots = torch.ones(3, 2, 64, device=DEV), torch.arange(3, device=DEV)
    cache.append(x, x, slots)
    for name in ("k_codes", "k_params", "v_codes", "v_params", "status", "page_size"):
        with pytest.raises(AttributeError, match="fixed"):
            setattr(cache, name, getattr(cache, name))
    cache.note = "other names are free"
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    kept = cache.v_params.data
    cache.v_params.data = kept.clone()
    for call in (lambda: cache.append(x, x, slots), lambda: cache.read(slots), lambda: cache.attend(torch.ones(1, 1, 4, 64, device=DEV).bfloat16(), table, lens)):
        with pytest.raises(ValueError, match="moved"):
            call()
    cache.v_params.data = kept
    assert (cache.read(slots, torch.float32)[1] == 1).all()
    cache.query_status()


# ------------------------------------------------------------------------------------------------ status words
def test_prompt_without_a_status_word_of_its_own_is_heard_of(S, monkeypatch):
    q = torch.zeros(300, 2, 64, dtype=torch.bfloat16, device=DEV)
    bad = torch.tensor([0, 200, 100, 300], dtype=torch.int32, device=DEV)
    good = torch.tensor([0, 100, 200, 300], dtype=torch.int32, device=DEV)
    S.query_status()                                             # nothing has gone wrong yet
    S.attention_prompt(q, q, q, bad)
    with pytest.raises(S.GcError, match="offsets"):
        S.query_status()
    S.query_status()                                             # cleared
    own = S.new_status(DEV)
    S.attention_prompt(q, q, q, bad, status=own)
    S.attention_prompt(q, q, q, good)
    S.query_status()
    with pytest.raises(S.GcError, match="offsets"):
        S.query_status(own)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.attention_prompt(q, q, q, bad)
        with pytest.raises(S.GcError, match="offsets"):
            S.query_status()
    offsets, out = good.clone(), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.attention_prompt(q, q, q, offsets, out=out)
    graph.replay()
    S.query_status()
    offsets.copy_(bad)
    graph.replay()
    with pytest.raises(S.GcError, match="offsets"):
        S.query_status()
    monkeypatch.setattr(S, "_words", {})                         # as if no call had been made yet
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(other):
        with pytest.raises(ValueError, match="capture"):
            S.attention_prompt(q, q, q, good, out=out)
        S.attention_prompt(q, q, q, good, out=out, status=own)
    other.replay()
    S.query_status(own)


# ------------------------------------------------------------------------------------------------ sizes of values
def sized_cache(S, m, n, size_k=1.0, size_v=1.0, seed=0):
    g = gen(seed)
    cache = filled_cache(S, 2 + m // 64, 64, 2, 128, 32, g)
    cache.k_params.mul_(size_k)
    cache.v_params.mul_(size_v)
    table = table_of([m], 64, 2 + m // 64, g)
    q = randn(1, n, 4, 128, g=g, dtype=torch.bfloat16, scale=1.0 / size_k)
    return cache, table, q, torch.tensor([m], dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("m", [20, 400, 3000])
@pytest.mark.parametrize("n", [1, 5])
def test_attend_reports_values_it_cannot_sum(S, m, n):
    cache, table, q, ln = sized_cache(S, m, n)
    want = cache.attend(q, table, ln)
    cache.query_status()
    held = cache.v_params.clone()
    at = m // 2
    for big in ((2.0 ** 34, 0.5), (-(2.0 ** 34), 0.5), (-1.0, 2.0 ** 33), (3e38, 0.0)):
        cache.v_params[table[0, at // 64], 1, at % 64, 2] = torch.tensor(big, device=DEV).bfloat16()
        cache.attend(q, table, ln)
        with pytest.raises(S.GcError, match="exceeds"):
            cache.query_status()
        cache.v_params.copy_(held)
    for t in range(m, table.shape[1] * 64):                      # behind the sequence, and in keys, any size is fine
        cache.v_params[table[0, t // 64], :, t % 64] = 2.0 ** 60
    cache.k_params[table[0, at // 64], 0, at % 64] = 2.0 ** -60
    cache.attend(q, table, ln)
    cache.query_status()
    cache.v_params[table[0, at // 64], 1, at % 64, 2] = math.nan  # a group that could not be held is no matter of size
    out = cache.attend(q, table, ln)
    cache.query_status()
    assert torch.isnan(out[0, -1, 2:, 64:96]).all() and torch.isfinite(out[:, :, 2:, :64]).all() and want.shape == out.shape


@pytest.mark.parametrize("power_k,power_v", [(0, 29), (60, 0), (-60, 0), (0, -39)])
def test_attend_sizes_of_keys_and_values(S, power_k, power_v):
    m = 700
    cache, table, q, ln = sized_cache(S, m, 3, 2.0 ** power_k, 2.0 ** power_v)
    out = cache.attend(q, table, ln)
    cache.query_status()
    cache.v_params.mul_(2.0 ** -power_v)                         # exactly the values of ordinary size
    cache.k_params.mul_(2.0 ** -power_k)
    q = (q.double() * 2.0 ** power_k).bfloat16()
    ref, tol = attend_reference(cache, q, table, [m], 128 ** -0.5, 32)
    # a weight times a scale below 2^-57 may be missing: at most 15 of them for each token
    within(out.double() * 2.0 ** -power_v, ref, tol + 15 * m * 2.0 ** (-57 - power_v))


def test_slots_that_are_no_vector_are_refused(S):
    cache = S.KV4Cache.allocate(2, 16, 2, 64, 32)
    for bad, kind in ((None, TypeError), ([0, 1], TypeError), (torch.zeros((), dtype=torch.int64, device=DEV), ValueError),
                      (torch.zeros(2, 2, dtype=torch.int64, device=DEV), ValueError), (torch.zeros(2, dtype=torch.int32, device=DEV), ValueError)):
        with pytest.raises(kind, match="slots"):
            cache.read(bad)
    cache.query_status()


# ------------------------------------------------------------------------------------------------ launch shapes
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t", [593, 700, 1183, 1187])
@pytest.mark.parametrize("d,rot,pad", [(128, 128, 0), (128, 64, 0), (96, 96, 0), (80, 48, 0), (64, 64, 1), (50, 22, 0)])
def test_rope_several_tokens_to_a_block(S, dtype, interleaved, t, d, rot, pad):
    # two and four tokens to a block, the last block not full: lanes without elements, partly rotated heads, rows that are not aligned
    rope_case(S, t, 3, 2, d, rot, dtype, interleaved, seed=t + d, pad=pad)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", [16, 17])
@pytest.mark.parametrize("n", [[1024], [1025], [130, 1, 700, 60]])
def test_prompt_items_of_128_and_of_256_rows(S, causal, heads, n):
    # (tokens / 128 + sequences) x heads is 144 and 153 for 1024 tokens, either side of 148 SMs, where items become twice as long
    prompt_case(S, n, n, heads, 1 if heads == 16 else 17, 64, causal, seed=heads + len(n), tail=3, poison=True)


# ------------------------------------------------------------------------------------------------ sizes of scores
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_too_large_for_their_weights_are_reported(S, sign):
    # every key is the same, so every output is 1, or, with scores (2^17 sqrt(128) sizes) above 2^26, the call says that it cannot tell
    d, m = 128, 300
    k, v = torch.full((m, 1, d), 2.0 ** 17, device=DEV).bfloat16(), torch.ones(m, 1, d, device=DEV).bfloat16()
    cu = torch.tensor([0, m], dtype=torch.int32, device=DEV)
    cache = S.KV4Cache.allocate(20, 16, 1, d, 128)
    cache.append(k, v, torch.arange(m, device=DEV))
    table, ln = torch.arange(20, dtype=torch.int32, device=DEV)[None], torch.tensor([m], dtype=torch.int32, device=DEV)
    status = S.new_status(DEV)
    for size, bad in ((1.0, False), (1.37, False), (1.37 * 2.0 ** 4, False), (1.37 * 2.0 ** 14, True), (1.71 * 2.0 ** 20, True)):
        q = torch.full((m, 2, d), sign * size, device=DEV).bfloat16()
        for call, query in ((lambda: S.attention_prompt(q, k, v, cu, status=status), lambda: S.query_status(status)),
                            (lambda: cache.attend(q[None, :1], table, ln), cache.query_status),
                            (lambda: cache.attend(q[None, :5], table.expand(1, 20), ln, max_length=m), cache.query_status)):
            out = call()
            if bad:
                with pytest.raises(S.GcError, match="score"):
                    query()
            else:
                query()
                # the weights are rounded to bf16, and so is the output: half a step each
                within(out, torch.ones_like(out, dtype=torch.float64), torch.full_like(out, 1 / 128, dtype=torch.float64))
    q = torch.full((m, 2, d), sign * math.inf, device=DEV).bfloat16()      # infinite scores: NaN, and nothing to report
    S.attention_prompt(q, k, v, cu, status=status)
    S.query_status(status)
    cache.attend(q[None, :1], table, ln)
    cache.query_status()
