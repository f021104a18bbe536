"""The operators of a served attention block, as they are measured: their sizes, inputs, plain forms and 64-bit values.

  qk_norm_rope      RMS norm of every query and key head and the rotation by position, one pass
  kv4_write         keys and values written into a paged 4-bit cache, and read back as the values the cache now holds
  kv4_read          rows of the cache read back (a prefix that another sequence shares, a cache that is moved)
  attention_kv4     a few new queries per sequence against the 4-bit cache
  attention_prompt  whole prompts, causal, grouped heads, sequences packed one behind the other

``run`` computes the plain form with elementary torch operations in 32 bits (angles in 64) and one rounding at the
end, or, with ``own`` set, makes the calls a user makes of ``paper_2301_01333_b200.serving``.

The 4-bit cache.  ``codes`` u8 [pages, heads, page, D / 2], element 2 j of a row in the low half of byte j, and
``params`` bf16 [pages, heads, page, D / group, 2] = (lo, scale) per group of `group` consecutive elements.  With d the
group's elements: lo = the largest bf16 <= min(d), scale = the smallest bf16 >= (max(d) - lo) / 15, code = the integer
nearest to (d - lo) / scale (ties to even; 0 where scale is 0), all of exact quotients; the value held is lo + code * scale.
Token t lives at slot = page * page_size + offset; a negative slot marks a padding row, which is skipped.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one step of sixteen running sequences: latency of a small launch
        dict(name="rope_step", op="qk_norm_rope", tokens=16, hq=32, hk=8, d=128, rot=128, interleaved=False, norm=True,
             dtype="bf16", far=131072),
        # a chunk of prompt tokens of a long-context model, half of each head rotated, interleaved pairs
        dict(name="rope_prompt", op="qk_norm_rope", tokens=8191, hq=32, hk=8, d=128, rot=64, interleaved=True, norm=True,
             dtype="bf16", far=1048576),
        # 32-bit activations, 16 heads of 64 (the encoder heads this framework runs), whole head rotated
        dict(name="rope_float", op="qk_norm_rope", tokens=1537, hq=16, hk=16, d=64, rot=64, interleaved=False, norm=True,
             dtype="f32", far=4096),
        # the new tokens of 48 sequences, finest scales, smallest pages, some rows padding
        dict(name="write_step", op="kv4_write", tokens=48, pad=5, hk=8, d=128, group=32, page=16, dtype="bf16"),
        # the keys and values of 24000 prompt tokens
        dict(name="write_prompt", op="kv4_write", tokens=24000, pad=0, hk=8, d=128, group=64, page=64, dtype="bf16"),
        # 32-bit activations, heads of 64 with one scale each
        dict(name="write_float", op="kv4_write", tokens=4099, pad=3, hk=16, d=64, group=64, page=32, dtype="f32"),
        # a shared prefix of 65000 tokens read back for another use
        dict(name="read_prefix", op="kv4_read", tokens=65000, pad=0, hk=8, d=128, group=128, page=64, dtype="bf16"),
        # a few short conversations: latency counts
        dict(name="attend_small", op="attention_kv4", batch=5, queries=1, longest=300, hq=32, hk=8, d=128, group=32, page=16,
             mix=1),
        # a full batch of ragged lengths, one of them empty
        dict(name="attend_batch", op="attention_kv4", batch=64, queries=1, longest=8192, hq=32, hk=8, d=128, group=64,
             page=64, mix=2),
        # one very long context, four queries at a time (a draft being checked), 64 query heads
        dict(name="attend_long", op="attention_kv4", batch=1, queries=4, longest=131071, hq=64, hk=8, d=128, group=128,
             page=128, mix=3),
        # short prompts of an encoder-sized model: 12 heads of 64, no sharing
        dict(name="prompt_short", op="attention_prompt", batch=7, longest=128, before=0, hq=12, hk=12, d=64, causal=True,
             tail=0, mix=4),
        # one long prompt, grouped heads
        dict(name="prompt_long", op="attention_prompt", batch=1, longest=16384, before=0, hq=16, hk=4, d=128, causal=True,
             tail=0, mix=5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qk_norm_rope", "kv4_write", "kv4_read", "attention_kv4", "attention_kv4", "attention_prompt",
                     "attention_prompt"])
    if op == "qk_norm_rope":
        hk = rng.choice([1, 2, 4, 5, 8, 16])
        hq = hk * rng.choice([1, 2, 3, 4, 8])
        d = rng.choice([32, 64, 80, 96, 128, 192, 256])
        rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 8191 * 40 * 128 * 2 // ((hq + hk) * d * (4 if dtype == "f32" else 2))
        return dict(op=op, tokens=_log(rng, 1, min(8191, most)), hq=hq, hk=hk, d=d, rot=rot - rot % 2,
                    interleaved=rng.random() < 0.5, norm=rng.random() < 0.8, dtype=dtype, far=_log(rng, 64, 1 << 20))
    hk = rng.choice([1, 2, 4, 8, 16])
    d = rng.choice([64, 64, 96, 128, 128])
    group = rng.choice([g for g in (32, 64, 128) if d % g == 0])
    page = rng.choice([16, 32, 64, 128])
    if op in ("kv4_write", "kv4_read"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = (24000 if op == "kv4_write" else 65000) * 8 * 128 * 2 // (hk * d * (4 if dtype == "f32" else 2))
        tokens = _log(rng, 1, min(24000, most))
        return dict(op=op, tokens=tokens, pad=rng.choice([0, 0, tokens // 7]), hk=hk, d=d, group=group, page=page, dtype=dtype)
    g = rng.choice([1, 2, 3, 4, 6, 8, 16])
    if op == "attention_kv4":
        batch = _log(rng, 1, 96)
        most = 64 * 8192 * 8 * 128 // (batch * hk * d)
        return dict(op=op, batch=batch, queries=rng.choice([1, 1, 1, 2, 3, 5, 8]), longest=_log(rng, 1, max(2, min(131071, most // max(1, g // 4)))),
                    hq=hk * g, hk=hk, d=d, group=group, page=page, mix=rng.randrange(1 << 20))
    batch = _log(rng, 1, 24)
    hk = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 3, 4, 6, 8])
    most = int(math.sqrt(16384.0 * 16384.0 * 16 / (batch * hk * g)))
    return dict(op=op, batch=batch, longest=_log(rng, 1, min(16384, most)), before=rng.choice([0, 0, 0, 1]), hq=hk * g, hk=hk,
                d=d, causal=rng.random() < 0.8, tail=rng.choice([0, 0, 9]), mix=rng.randrange(1 << 20))


# ------------------------------------------------------------------------------------------------- sizes and inputs
def _lengths(case):
    """Lengths of the sequences: the first has the longest, the others anything below, one of a larger batch is empty."""
    r = np.random.RandomState(case["mix"])
    n = r.randint(1, case["longest"] + 1, case["batch"])
    n[0] = case["longest"]
    if case["batch"] > 4:
        n[3] = 0
    return n.astype(np.int64)


def _prompt_lengths(case):
    """(queries, keys) of every sequence; with `before`, some keys precede the first query (a continued prompt)."""
    nq = _lengths(case)
    r = np.random.RandomState(case["mix"] + 1)
    if not case["before"]:
        return nq, nq.copy()
    nq = np.maximum(nq // 2, np.minimum(nq, 1))
    return nq, nq + r.randint(0, case["longest"] // 2 + 1, case["batch"]) * (nq > 0)


def _spread_slots(tokens, page, pages, gen):
    """Tokens in order, page after page, the pages in any order."""
    order = torch.randperm(pages, generator=gen, device=DEV)
    t = torch.arange(tokens, device=DEV)
    return order[t // page] * page + t % page


def _random_cache(pages, hk, page, d, group, gen):
    """What writing normally distributed rows leaves in a cache, without the writing."""
    shape = (pages, hk, page)
    codes = torch.randint(0, 256, shape + (d // 2,), generator=gen, device=DEV, dtype=torch.uint8)
    params = torch.empty(shape + (d // group, 2), device=DEV, dtype=torch.bfloat16)
    params[..., 0] = -2.2 - 0.4 * torch.randn(shape + (d // group,), generator=gen, device=DEV)
    params[..., 1] = 0.2 + 0.2 * torch.rand(shape + (d // group,), generator=gen, device=DEV)
    return codes, params


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case)
    op = case["op"]
    if op == "qk_norm_rope":
        t, hq, hk, d = case["tokens"], case["hq"], case["hk"], case["d"]
        # queries and keys as a projection leaves them: side by side, with the values behind them
        qkv = (2.0 * torch.randn(t, hq + 2 * hk, d, generator=gen, device=DEV)).to(_TYPE[case["dtype"]])
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        s["pos"] = torch.randint(0, case["far"], (t,), generator=gen, device=DEV)
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])).float()
        s["factor"] = 1.0 if case["far"] <= 4096 else 1.15
        s["qw"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(_TYPE[case["dtype"]])
        s["kw"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(_TYPE[case["dtype"]])
    elif op in ("kv4_write", "kv4_read"):
        t, hk, d, group, page = case["tokens"], case["hk"], case["d"], case["group"], case["page"]
        pages = -(-t // page) + 3
        s["slots"] = _spread_slots(t, page, pages, gen)
        if case["pad"]:
            s["slots"][-case["pad"]:] = -1
        s["k_codes"], s["k_params"] = _random_cache(pages, hk, page, d, group, gen)
        s["v_codes"], s["v_params"] = _random_cache(pages, hk, page, d, group, gen)
        if op == "kv4_write":
            kv = torch.randn(t, 2 * hk, d, generator=gen, device=DEV)
            kv *= torch.exp2(torch.randn(d, generator=gen, device=DEV))          # channels of unlike size, as keys have
            kv = kv.to(_TYPE[case["dtype"]])
            s["k"], s["v"] = kv[:, :hk], kv[:, hk:]
        s["k_out"] = torch.zeros(t, hk, d, device=DEV, dtype=_TYPE[case["dtype"]])
        s["v_out"] = torch.zeros(t, hk, d, device=DEV, dtype=_TYPE[case["dtype"]])
    elif op == "attention_kv4":
        n, page, d, group = _lengths(case), case["page"], case["d"], case["group"]
        need = -(-n // page)
        width, pages = int(need.max()), int(need.sum()) + 2
        order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
        at = np.concatenate([[0], np.cumsum(need)])[:-1, None] + np.arange(width)[None, :]
        used = torch.from_numpy(np.arange(width)[None, :] < need[:, None]).to(DEV)
        at = torch.from_numpy(np.minimum(at, pages - 1)).to(DEV)
        s["table"] = torch.where(used, order[at], torch.full_like(order[at], -1))
        s["lengths"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
        s["longest"] = case["longest"]
        s["k_codes"], s["k_params"] = _random_cache(pages, case["hk"], page, d, group, gen)
        s["v_codes"], s["v_params"] = _random_cache(pages, case["hk"], page, d, group, gen)
        s["q"] = torch.randn(case["batch"], case["queries"], case["hq"], d, generator=gen, device=DEV).to(torch.bfloat16)
    else:
        nq, nk = _prompt_lengths(case)
        hq, hk, d = case["hq"], case["hk"], case["d"]
        tq, tk = int(nq.sum()) + case["tail"], int(nk.sum()) + case["tail"]
        if case["before"]:
            s["q"] = torch.randn(tq, hq, d, generator=gen, device=DEV).to(torch.bfloat16)
            kv = torch.randn(tk, 2 * hk, d, generator=gen, device=DEV).to(torch.bfloat16)
            s["k"], s["v"] = kv[:, :hk], kv[:, hk:]
        else:
            qkv = torch.randn(tq, hq + 2 * hk, d, generator=gen, device=DEV).to(torch.bfloat16)
            s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["cu_q"] = torch.from_numpy(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)).to(DEV)
        s["cu_k"] = torch.from_numpy(np.concatenate([[0], np.cumsum(nk)]).astype(np.int32)).to(DEV)
        s["most_q"], s["most_k"] = max(1, int(nq.max())), max(1, int(nk.max()))
        s["out"] = torch.full((tq, hq, d), 0.25, device=DEV, dtype=torch.bfloat16)    # rows behind the last sequence keep this
    return s


# ------------------------------------------------------------------------------------------------- the plain forms
def _rotate(x, w, cos, sin, case):
    x = x.float()
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
    r = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rope(s):
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()
    cos, sin = (angle.cos() * s["factor"]).float()[:, None], (angle.sin() * s["factor"]).float()[:, None]
    return {"q": _rotate(s["q"], s["qw"], cos, sin, s["case"]).to(s["q"].dtype),
            "k": _rotate(s["k"], s["kw"], cos, sin, s["case"]).to(s["k"].dtype)}


def _bf16_below(x):
    """The largest bf16 <= x: the bit pattern cut off, one step further down where that went up (negative numbers)."""
    bits = x.contiguous().view(torch.int32)
    cut = bits & -65536
    return torch.where((cut != bits) & (bits < 0), cut + 65536, cut).view(torch.float32)


def _plain_write(x, slots, codes, params):
    """In 64 bits where a value lies next to a border.  The divisors are tensors: a division by a number multiplies by
    its rounded reciprocal, which moves exact quotients off their borders."""
    page, group = codes.shape[2], codes.shape[3] * 2 // params.shape[3]
    x = x.float().unflatten(-1, (-1, group))
    lo = _bf16_below(x.amin(-1))
    step = (x.amax(-1).double() - lo) / torch.full_like(lo, 15, dtype=torch.float64)
    scale = -_bf16_below(-step.float())
    scale = torch.where(scale < step, (scale.view(torch.int32) + 65536).view(torch.float32), scale)
    ratio = (x.double() - lo[..., None]) / scale[..., None]
    code = torch.where(scale[..., None] > 0, ratio, torch.zeros_like(ratio)).round().clamp(0, 15).to(torch.uint8).flatten(-2)
    byte = code[..., 0::2] | (code[..., 1::2] << 4)
    keep = (slots >= 0).nonzero()[:, 0]
    at = slots[keep]
    codes[at // page, :, at % page] = byte[keep]
    params[at // page, :, at % page] = torch.stack([lo, scale], -1)[keep].to(torch.bfloat16)


def _values(codes, params, pages, offsets):
    """The rows of a cache at [pages, :, offsets], as 32-bit numbers [..., heads, D]."""
    c, p = codes[pages, :, offsets], params[pages, :, offsets].float()
    v = torch.stack([c & 15, c >> 4], -1).flatten(-2).float().unflatten(-1, (p.shape[-2], -1))
    return (p[..., 0, None] + v * p[..., 1, None]).flatten(-2)


def _plain_read(s):
    page, slots = s["case"]["page"], s["slots"]
    keep = (slots >= 0).nonzero()[:, 0]
    at = slots[keep]
    s["k_out"][keep] = _values(s["k_codes"], s["k_params"], at // page, at % page).to(s["k_out"].dtype)
    s["v_out"][keep] = _values(s["v_codes"], s["v_params"], at // page, at % page).to(s["v_out"].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _softmax_product(scores, seen, v):
    """softmax of the scores where `seen` says so, times v; zero in a row that sees nothing.  Overwrites the scores."""
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = scores.sum(-1, keepdim=True)
    return torch.matmul(scores, v) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_attend(s):
    case, q = s["case"], s["q"].float()
    b, n, hq, d = q.shape
    hk, page = case["hk"], case["page"]
    t = torch.arange(s["longest"], device=DEV)
    pages = s["table"][:, t // page].long().clamp(min=0)
    offsets = (t % page).expand_as(pages)
    seen = t < s["lengths"][:, None, None] - (n - 1) + torch.arange(n, device=DEV)[:, None]          # [b, n, t]
    k = _values(s["k_codes"], s["k_params"], pages, offsets).transpose(1, 2)                        # [b, hk, t, d]
    scores = torch.matmul(q.unflatten(2, (hk, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3) * d ** -0.5, k.transpose(2, 3))
    k = None
    v = _values(s["v_codes"], s["v_params"], pages, offsets).transpose(1, 2)
    seen = seen[:, None, :, None].expand(b, 1, n, hq // hk, -1).flatten(2, 3)
    o = _softmax_product(scores, seen, v)
    return {"o": o.unflatten(2, (n, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3).to(torch.bfloat16)}


def _plain_prompt(s):
    case = s["case"]
    hk, d = case["hk"], case["d"]
    nq, nk = s["cu_q"].diff().long(), s["cu_k"].diff().long()
    i, j = torch.arange(s["most_q"], device=DEV), torch.arange(s["most_k"], device=DEV)
    rows = s["cu_q"][:-1, None].long() + i
    cols = s["cu_k"][:-1, None].long() + j
    seen = (j < nk[:, None, None]).expand(-1, s["most_q"], -1)
    if case["causal"]:
        seen = seen & (j <= i[:, None] + (nk - nq)[:, None, None])
    q = s["q"][rows.clamp(max=s["q"].shape[0] - 1)].float().unflatten(2, (hk, -1)).permute(0, 2, 3, 1, 4)  # [b, hk, g, i, d]
    k = s["k"][cols.clamp(max=s["k"].shape[0] - 1)].float().permute(0, 2, 1, 3)[:, :, None]
    v = s["v"][cols.clamp(max=s["v"].shape[0] - 1)].float().permute(0, 2, 1, 3)[:, :, None]
    scores = torch.matmul(q.mul_(d ** -0.5), k.transpose(-1, -2).expand(-1, -1, q.shape[2], -1, -1))
    o = _softmax_product(scores, seen[:, None, None], v.expand(-1, -1, q.shape[2], -1, -1))
    at = (i < nq[:, None]).nonzero()
    s["out"][rows[at[:, 0], at[:, 1]]] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[at[:, 0], at[:, 1]].to(torch.bfloat16)
    return {"o": s["out"]}


# ------------------------------------------------------------------------------------------------- the user's calls
def _own(s):
    from paper_2301_01333_b200 import serving
    case = s["case"]
    op = case["op"]
    if op == "qk_norm_rope":
        q, k = serving.qk_norm_rope(s["q"], s["k"], s["pos"], s["inv_freq"], s["qw"], s["kw"], norm=case["norm"], eps=1e-6,
                                    interleaved=case["interleaved"], attention_factor=s["factor"])
        return {"q": q, "k": k}
    if op == "attention_prompt":
        return {"o": serving.attention_prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=case["causal"], out=s["out"])}
    if "cache" not in s:           # the handle a program makes once over its cache's memory
        s["cache"] = serving.KV4Cache(s["k_codes"], s["k_params"], s["v_codes"], s["v_params"])
    cache = s["cache"]
    if op == "attention_kv4":
        return {"o": cache.attend(s["q"], s["table"], s["lengths"], max_length=s["longest"])}
    if op == "kv4_write":
        cache.append(s["k"], s["v"], s["slots"])
    k, v = cache.read(s["slots"], k_out=s["k_out"], v_out=s["v_out"])
    return {"k": k, "v": v}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "qk_norm_rope":
        return _plain_rope(state)
    if op == "attention_kv4":
        return _plain_attend(state)
    if op == "attention_prompt":
        return _plain_prompt(state)
    if op == "kv4_write":
        _plain_write(state["k"], state["slots"], state["k_codes"], state["k_params"])
        _plain_write(state["v"], state["slots"], state["v_codes"], state["v_params"])
    return _plain_read(state)


def work(case):
    op, d = case["op"], case["d"]
    if op == "qk_norm_rope":
        n, size = case["tokens"] * (case["hq"] + case["hk"]) * d, 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * n * size + 8 * case["tokens"] + 2 * case["rot"] + 2 * d * size, "flops": 8 * n}
    if op in ("kv4_write", "kv4_read"):
        rows = (case["tokens"] - case["pad"]) * case["hk"] * 2
        plain, held = rows * d * (4 if case["dtype"] == "f32" else 2), rows * (d // 2 + d // case["group"] * 4)
        # a written row is read once and held once; reading it back reads what is held and writes the values
        return {"bytes": (2 * plain + 2 * held if op == "kv4_write" else plain + held) + 8 * case["tokens"], "flops": 6 * rows * d}
    if op == "attention_kv4":
        n = _lengths(case)
        held = float(n.sum()) * case["hk"] * 2 * (d // 2 + d // case["group"] * 4)
        q = case["batch"] * case["queries"] * case["hq"] * d * 2
        pages = float((-(-n // case["page"])).sum())
        return {"bytes": held + 2 * q + 4 * pages + 4 * case["batch"], "flops": 4.0 * float(n.sum()) * case["queries"] * case["hq"] * d}
    nq, nk = _prompt_lengths(case)
    nq, nk = nq.astype(np.float64), nk.astype(np.float64)
    pairs = nq * nk - nq * (nq - 1) / 2 if case["causal"] else nq * nk
    size = 2 * d * (2 * nq.sum() * case["hq"] + 2 * nk.sum() * case["hk"]) + 8 * (case["batch"] + 1)
    return {"bytes": float(size), "flops": 4.0 * float(pairs.sum()) * case["hq"] * d}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_head(q, k, v, limit):
    """One head of one sequence: q [i, d], k / v [j, d] in 64 bits; row i sees the first limit[i] keys."""
    p = q @ k.T / math.sqrt(q.shape[-1])
    p.masked_fill_(torch.arange(k.shape[0], device=DEV) >= limit[:, None], -math.inf)
    return torch.nan_to_num(torch.softmax(p, -1)) @ v


def _exact_group(x):
    """(lo, scale, codes) of groups [..., group] in 64 bits: numbers of eight significant bits below and above."""
    def eight(y, towards):
        _, e = torch.frexp(y)
        step = torch.ldexp(torch.ones_like(y), e - 8)
        return torch.where(y == 0, y, towards(y / step) * step)
    lo = eight(x.min(-1).values, torch.floor)
    fifteen = torch.full_like(lo, 15)              # a tensor: an exact quotient has to stay one
    scale = eight((x.max(-1).values - lo) / fifteen, torch.ceil)
    unit = torch.where(scale == 0, torch.ones_like(scale), scale)
    return lo, scale, torch.clamp(torch.round((x - lo[..., None]) / unit[..., None]), 0, 15) * (scale > 0)[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    op, d = case["op"], case["d"]
    if op == "qk_norm_rope":
        angle = s["pos"].double()[:, None, None] * s["inv_freq"].double()
        turn = torch.polar(torch.full_like(angle, s["factor"]), angle)
        out = {}
        for name, weight in (("q", s["qw"]), ("k", s["kw"])):
            x = s[name].double()
            if case["norm"]:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6) * weight.double()
            pairs = x[..., :case["rot"]].unflatten(-1, (-1, 2) if case["interleaved"] else (2, -1))
            axis = -1 if case["interleaved"] else -2
            z = torch.complex(pairs.select(axis, 0), pairs.select(axis, 1)) * turn
            x[..., :case["rot"]] = torch.stack([z.real, z.imag], axis).flatten(-2)
            out[name] = x
        return out
    if op in ("kv4_write", "kv4_read"):
        out = {}
        ok = s["slots"] >= 0
        for name in ("k", "v"):
            if op == "kv4_write":
                lo, scale, code = _exact_group(s[name].double().reshape(case["tokens"], case["hk"], -1, case["group"]))
                x = (lo[..., None] + scale[..., None] * code).reshape(case["tokens"], case["hk"], d)
            else:
                rows = s["slots"].clamp(min=0)
                c = s[name + "_codes"].transpose(1, 2).reshape(-1, case["hk"], d // 2)[rows].double()
                high = torch.floor(c / 16)
                c = torch.stack([c - 16 * high, high], -1).reshape(case["tokens"], case["hk"], -1, case["group"])
                p = s[name + "_params"].transpose(1, 2).reshape(-1, case["hk"], d // case["group"], 2)[rows].double()
                x = (p[..., :1] + c * p[..., 1:]).reshape(case["tokens"], case["hk"], d)
            out[name] = torch.where(ok[:, None, None], x, torch.zeros_like(x))
        return out
    g = case["hq"] // case["hk"]
    if op == "attention_kv4":
        n, page = _lengths(case), case["page"]
        o = torch.zeros(s["q"].shape, device=DEV, dtype=torch.float64)
        for b in range(case["batch"]):
            m = int(n[b])
            if not m:
                continue
            pages = s["table"][b, :-(-m // page)].long()
            held = []
            for name in ("k", "v"):
                c = s[name + "_codes"][pages].transpose(1, 2).reshape(-1, case["hk"], d // 2)[:m].double()
                p = s[name + "_params"][pages].transpose(1, 2).reshape(-1, case["hk"], d // case["group"], 2)[:m].double()
                high = torch.floor(c / 16)
                c = torch.stack([c - 16 * high, high], -1).reshape(m, case["hk"], -1, case["group"])
                held.append((p[..., :1] + c * p[..., 1:]).reshape(m, case["hk"], d))
            limit = m - case["queries"] + 1 + torch.arange(case["queries"], device=DEV)
            for h in range(case["hq"]):
                o[b, :, h] = _exact_head(s["q"][b, :, h].double(), held[0][:, h // g], held[1][:, h // g], limit)
        return {"o": o}
    nq, nk = _prompt_lengths(case)
    o = s["out"].double()
    a = c = 0
    for i, j in zip(nq.tolist(), nk.tolist()):
        limit = torch.arange(i, device=DEV) + (j - i + 1) if case["causal"] else torch.full((i,), j, device=DEV)
        for h in range(case["hq"] if i else 0):
            k, v = s["k"][c:c + j, h // g].double(), s["v"][c:c + j, h // g].double()
            o[a:a + i, h] = _exact_head(s["q"][a:a + i, h].double(), k, v, limit)
        a, c = a + i, c + j
    return {"o": o}
