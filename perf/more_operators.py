"""The operators that let a paged 4-bit cache take prompts in chunks and keep it within a budget, as they are measured: their
sizes, inputs, plain forms and 64-bit values.

  attend_chunk  any number of new tokens per sequence, packed one behind the other, against the cache
  weigh         the attention weight every cached token received, added to what it has received so far
  evict         the tokens of the largest scores and the newest ones kept, moved together into pages of their own

``run`` computes the plain form with elementary torch operations in 32 bits and one rounding at the end, or, with ``own``
set, makes the calls a user makes of ``paper_2301_01333_b200.serving``.

The cache.  ``codes`` u8 [pages, heads, page, D / 2], element 2 j of a row in the low half of byte j, and ``params`` bf16
[pages, heads, page, D / group, 2] = (lo, scale) per group of `group` consecutive elements; the value held is lo + code *
scale.  Token t of a sequence lives at offset t % page of page block_table[sequence, t // page].  Weights and scores are fp32
[pages, heads, page], paged like the cache.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"


def listed():
    return [
        # a few short conversations, each with a handful of new tokens: latency counts
        dict(name="chunk_step", op="attend_chunk", batch=4, new=24, single=0.0, longest=700, hq=32, hk=8, d=128, group=32,
             page=16, tail=0, mix=1),
        # one step of a server: some prompts arrive in chunks, the other sequences have one new token each
        dict(name="chunk_mixed", op="attend_chunk", batch=32, new=192, single=0.75, longest=4096, hq=32, hk=8, d=128, group=64,
             page=64, tail=9, mix=2),
        # a chunk of a long prompt
        dict(name="chunk_long", op="attend_chunk", batch=1, new=1024, single=0.0, longest=33001, hq=16, hk=4, d=128, group=128,
             page=128, tail=0, mix=3),
        # a question of 48 tokens about a long text, eight query heads on one
        dict(name="chunk_question", op="attend_chunk", batch=1, new=48, single=0.0, longest=60000, hq=8, hk=1, d=128, group=64,
             page=64, tail=0, mix=4),
        # whole prompts of an encoder-sized model, through the cache: 12 heads of 64, no sharing
        dict(name="chunk_prompts", op="attend_chunk", batch=6, new=1500, single=0.0, longest=1500, hq=12, hk=12, d=64, group=64,
             page=32, tail=0, mix=5),
        # one step of a few short conversations
        dict(name="weigh_step", op="weigh", batch=5, queries=1, longest=300, hq=32, hk=8, d=128, group=32, page=16, decay=1.0,
             mix=6),
        # a full batch of ragged lengths, one of them empty; old weight fades
        dict(name="weigh_batch", op="weigh", batch=64, queries=1, longest=8192, hq=32, hk=8, d=128, group=64, page=64,
             decay=0.984375, mix=7),
        # the last sixteen queries of a long prompt, which say what of it to keep
        dict(name="weigh_window", op="weigh", batch=1, queries=16, longest=65000, hq=16, hk=4, d=128, group=128, page=128,
             decay=0.0, mix=8),
        # short conversations cut back to 256 tokens
        dict(name="evict_step", op="evict", batch=5, longest=300, keep=256, recent=32, hk=8, d=128, group=32, page=16, mix=9),
        # a batch that exceeds its budget
        dict(name="evict_batch", op="evict", batch=48, longest=4099, keep=2048, recent=128, hk=8, d=64, group=64, page=32, mix=10),
        # a long prompt, of which a part is kept
        dict(name="evict_prompt", op="evict", batch=1, longest=131071, keep=8192, recent=64, hk=8, d=128, group=64, page=64,
             mix=11),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["attend_chunk", "attend_chunk", "weigh", "evict"])
    hk = rng.choice([1, 2, 3, 4, 8, 16])
    d = rng.choice([64, 64, 96, 128, 128])
    group = rng.choice([g for g in (32, 64, 128) if d % g == 0])
    page = rng.choice([16, 32, 64, 128, 256])
    mix = rng.randrange(1 << 20)
    if op == "evict":
        batch = _log(rng, 1, 64)
        longest = _log(rng, 2, min(131071, 131071 * 8 // (batch * hk)))
        keep = _log(rng, 1, max(1, min(8192, longest, 8192 * 8 * 128 // (batch * hk * d))))
        return dict(op=op, batch=batch, longest=longest, keep=keep, recent=rng.choice([0, keep // 16, keep // 2, keep]), hk=hk,
                    d=d, group=group, page=page, mix=mix)
    g = rng.choice([1, 2, 3, 4, 6, 8])
    if op == "weigh":
        batch = _log(rng, 1, 96)
        queries = rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
        most = min(64 * 8192 * 8 * 128 // (batch * hk * d), 64 * 8192 * 32 // (batch * queries * hk * g))
        return dict(op=op, batch=batch, queries=queries, longest=_log(rng, 1, min(131071, most)), hq=hk * g, hk=hk, d=d,
                    group=group, page=page, decay=rng.choice([1.0, 1.0, 0.875, 0.0]), mix=mix)
    batch = _log(rng, 1, 40)
    new = _log(rng, 1, 2048)
    # as many scores as the long chunk has, as many cached elements as the batch
    most = min(1024 * 33001 * 16 // (batch * new * hk * g), 32 * 4096 * 8 * 128 // (batch * hk * d))
    longest = _log(rng, 1, min(60000, most))
    return dict(op=op, batch=batch, new=new, single=rng.choice([0.0, 0.0, 0.75]), longest=longest, hq=hk * g, hk=hk, d=d,
                group=group, page=page, tail=rng.choice([0, 0, 9]), mix=mix)


# ------------------------------------------------------------------------------------------------- sizes and inputs
def _lengths(case):
    """Lengths of the sequences: the first has the longest, the others anything below, one of a larger batch is empty."""
    r = np.random.RandomState(case["mix"])
    n = r.randint(1, case["longest"] + 1, case["batch"])
    n[0] = case["longest"]
    if case["batch"] > 4:
        n[3] = 0
    return n.astype(np.int64)


def _new(case):
    """New tokens of the sequences: the first has the most, a share of the others one each, one of a larger batch none."""
    r = np.random.RandomState(case["mix"] + 1)
    n = r.randint(1, case["new"] + 1, case["batch"])
    n[r.random_sample(case["batch"]) < case["single"]] = 1
    n[0] = case["new"]
    if case["batch"] > 4:
        n[2] = 0
    return np.minimum(n, _lengths(case))


def _pages(n, page, gen, spare=2):
    """(block table, pages in all) of sequences of n tokens: their pages in any order, -1 behind the last."""
    need = -(-n // page)
    width, pages = max(1, int(need.max())), int(need.sum()) + spare
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    at = np.concatenate([[0], np.cumsum(need)])[:-1, None] + np.arange(width)[None, :]
    used = torch.from_numpy(np.arange(width)[None, :] < need[:, None]).to(DEV)
    at = torch.from_numpy(np.minimum(at, pages - 1)).to(DEV)
    return torch.where(used, order[at], torch.full_like(order[at], -1)), pages


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
    op, n, hk, d, group, page = case["op"], _lengths(case), case["hk"], case["d"], case["group"], case["page"]
    s["longest"] = case["longest"]
    s["lengths"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
    s["table"], pages = _pages(n, page, gen)
    first = pages
    if op == "evict":
        # the pages the kept tokens go to lie behind those they come from
        m = np.minimum(n, case["keep"])
        s["out_table"], more = _pages(m, page, gen)
        s["out_table"] = torch.where(s["out_table"] >= 0, s["out_table"] + pages, s["out_table"])
        pages += more
        t = torch.arange(case["keep"], device=DEV)
        at = s["out_table"][:, t.clamp(max=int(max(1, m.max())) - 1) // page].long() * page + t % page
        s["slots"] = torch.where(t < torch.from_numpy(m).to(DEV)[:, None], at, torch.full_like(at, -1)).flatten()
    s["k_codes"], s["k_params"] = _random_cache(pages, hk, page, d, group, gen)
    if op != "weigh":
        s["v_codes"], s["v_params"] = _random_cache(pages, hk, page, d, group, gen)
    if op == "attend_chunk":
        new = _new(case)
        tokens = int(new.sum()) + case["tail"]
        # queries as a projection leaves them: the new keys and values, which the cache has by now, behind them
        s["q"] = torch.randn(tokens, case["hq"] + 2 * hk, d, generator=gen, device=DEV).to(torch.bfloat16)[:, :case["hq"]]
        s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        s["most"] = max(1, int(new.max()))
        s["out"] = torch.full((tokens, case["hq"], d), 0.25, device=DEV, dtype=torch.bfloat16)  # rows behind the last sequence keep this
    elif op == "weigh":
        s["q"] = torch.randn(case["batch"], case["queries"], case["hq"], d, generator=gen, device=DEV).to(torch.bfloat16)
        # what the queries have received so far, and the place of what they will have
        s["weights"] = torch.rand(pages, hk, page, generator=gen, device=DEV)
        s["out"] = torch.zeros(pages, hk, page, device=DEV)
        scores, seen = _scores(s)
        scores.masked_fill_(~seen, -math.inf)
        s["lse"] = torch.logsumexp(scores, -1).unflatten(2, (case["queries"], -1)).transpose(1, 2).flatten(2, 3).contiguous()
        del scores, seen
        # the attention before this call has left the cache's values behind as well, which are not looked at here
        s["v_codes"], s["v_params"] = s["k_codes"], s["k_params"]
    else:
        # weights as attention gives them: few large ones, many small ones, equal ones among these
        w = torch.rand(first, hk, page, generator=gen, device=DEV).clamp_(min=1e-4).pow_(-1.5).mul_(1 / 64)
        s["scores"] = torch.cat([torch.where(w < 0.02, torch.full_like(w, 1 / 64), w), torch.zeros(pages - first, hk, page, device=DEV)])
        s["keep"], s["recent"] = case["keep"], case["recent"]
    return s


# ------------------------------------------------------------------------------------------------- the plain forms
def _values(codes, params, pages, offsets):
    """The rows of a cache at [pages, :, offsets], as 32-bit numbers [..., heads, D]."""
    c, p = codes[pages, :, offsets], params[pages, :, offsets].float()
    v = torch.stack([c & 15, c >> 4], -1).flatten(-2).float().unflatten(-1, (p.shape[-2], -1))
    return (p[..., 0, None] + v * p[..., 1, None]).flatten(-2)


def _places(s, table):
    """(pages, offsets) [batch, longest] of every sequence's tokens."""
    page = s["case"]["page"]
    t = torch.arange(s["longest"], device=DEV)
    pages = table[:, (t // page).clamp(max=table.shape[1] - 1)].long().clamp(min=0)
    return pages, (t % page).expand_as(pages)


def _scores(s):
    """Scores [batch, kv heads, queries * sharing heads, longest] and which of them count, for queries [batch, queries, heads, D]."""
    case, q = s["case"], s["q"].float()
    n, hk = q.shape[1], case["hk"]
    t = torch.arange(s["longest"], device=DEV)
    seen = t < s["lengths"][:, None, None] - (n - 1) + torch.arange(n, device=DEV)[:, None]           # [b, n, t]
    k = _values(s["k_codes"], s["k_params"], *_places(s, s["table"])).transpose(1, 2)                 # [b, hk, t, d]
    scores = torch.matmul(q.unflatten(2, (hk, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3) * case["d"] ** -0.5, k.transpose(2, 3))
    return scores, seen[:, None, :, None].expand(-1, 1, -1, case["hq"] // hk, -1).flatten(2, 3)


def _plain_chunk(s):
    case = s["case"]
    hk = case["hk"]
    new = s["cu"].diff().long()
    i, t = torch.arange(s["most"], device=DEV), torch.arange(s["longest"], device=DEV)
    rows = s["cu"][:-1, None].long() + i
    seen = t < (s["lengths"] - new)[:, None, None] + 1 + i[:, None]                                   # [b, i, t]
    q = s["q"][rows.clamp(max=s["q"].shape[0] - 1)].float().unflatten(2, (hk, -1)).permute(0, 2, 3, 1, 4)   # [b, hk, g, i, d]
    g = q.shape[2]
    k = _values(s["k_codes"], s["k_params"], *_places(s, s["table"])).transpose(1, 2)
    scores = torch.matmul(q.flatten(2, 3) * case["d"] ** -0.5, k.transpose(2, 3))
    k = None
    scores.unflatten(2, (g, -1)).masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = scores.sum(-1, keepdim=True)
    v = _values(s["v_codes"], s["v_params"], *_places(s, s["table"])).transpose(1, 2)
    o = (torch.matmul(scores, v) / torch.where(total == 0, torch.ones_like(total), total)).unflatten(2, (g, -1))
    at = (i < new[:, None]).nonzero()
    s["out"][rows[at[:, 0], at[:, 1]]] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[at[:, 0], at[:, 1]].to(torch.bfloat16)
    return {"o": s["out"]}


def _plain_weigh(s):
    case = s["case"]
    scores, seen = _scores(s)
    lse = s["lse"].unflatten(2, (case["hk"], -1)).permute(0, 2, 1, 3).flatten(2, 3)
    scores.sub_(lse[..., None]).exp_().masked_fill_(~seen, 0.0)
    received = scores.sum(2).transpose(1, 2)                                                          # [b, t, hk]
    pages, offsets = _places(s, s["table"])
    at = (torch.arange(s["longest"], device=DEV) < s["lengths"][:, None]).nonzero()
    pages, offsets, received = pages[at[:, 0], at[:, 1]], offsets[at[:, 0], at[:, 1]], received[at[:, 0], at[:, 1]]
    s["out"][pages, :, offsets] = case["decay"] * s["weights"][pages, :, offsets] + received
    return {"weights": s["out"]}


def _plain_evict(s):
    case, keep = s["case"], s["keep"]
    n = s["lengths"].long()[:, None, None]
    t = torch.arange(s["longest"], device=DEV)
    pages, offsets = _places(s, s["table"])
    score = s["scores"][pages, :, offsets].transpose(1, 2)                                            # [b, hk, t]
    score = torch.where(t >= n - s["recent"], torch.full_like(score, math.inf), score)
    score = torch.where(t >= n, torch.full_like(score, -math.inf), score)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :keep]
    stays = torch.zeros_like(score, dtype=torch.bool).scatter_(-1, order, True) & (t < n)
    # position i < keep has token i if that stays; the other positions get, in order, the tokens behind that stay
    hole, mover = ~stays & (t < torch.minimum(n, torch.full_like(n, keep))), stays & (t >= keep)
    filled, moved = hole.nonzero(), mover.nonzero()                                                   # as many, in the same order
    source = torch.where(stays, t, torch.full_like(t, -1))
    source[filled[:, 0], filled[:, 1], filled[:, 2]] = moved[:, 2]
    kept = torch.full((score.shape[0], score.shape[1], keep), -1, device=DEV, dtype=torch.int64)
    kept[..., :source.shape[2]] = source[..., :keep]
    b, h, i = (kept >= 0).nonzero().unbind(1)
    t = kept[b, h, i]
    page = case["page"]
    from_page, to_page = s["table"][b, t // page].long(), s["out_table"][b, i // page].long()
    for held in ("k_codes", "k_params", "v_codes", "v_params", "scores"):
        s[held][to_page, h, i % page] = s[held][from_page, h, t % page]
    at = s["slots"].clamp(min=0)
    ok = (s["slots"] >= 0)[:, None, None]
    k, v = (torch.where(ok, _values(s[x + "_codes"], s[x + "_params"], at // page, at % page), torch.zeros((), device=DEV)).to(torch.bfloat16) for x in "kv")
    return {"lengths": s["lengths"].clamp(max=keep), "kept": kept.to(torch.int32), "scores": s["scores"], "k": k, "v": v}


# ------------------------------------------------------------------------------------------------- the user's calls
def _own(s):
    from paper_2301_01333_b200 import serving
    case = s["case"]
    if "cache" not in s:           # the handle a program makes once over its cache's memory
        s["cache"] = serving.KV4Cache(s["k_codes"], s["k_params"], s["v_codes"], s["v_params"])
    cache = s["cache"]
    if case["op"] == "attend_chunk":
        return {"o": cache.attend_chunk(s["q"], s["cu"], s["table"], s["lengths"], max_length=s["longest"], out=s["out"])}
    if case["op"] == "weigh":
        return {"weights": cache.weigh(s["weights"], s["q"], s["lse"], s["table"], s["lengths"], decay=case["decay"],
                                       max_length=s["longest"], out=s["out"])}
    lengths, kept = cache.evict(s["scores"], s["table"], s["lengths"], s["keep"], s["recent"], max_length=s["longest"],
                                out_table=s["out_table"])
    k, v = cache.read(s["slots"])
    return {"lengths": lengths, "kept": kept, "scores": s["scores"], "k": k, "v": v}


def run(state):
    if own:
        return _own(state)
    return {"attend_chunk": _plain_chunk, "weigh": _plain_weigh, "evict": _plain_evict}[state["case"]["op"]](state)


def work(case):
    n, hk, d = _lengths(case), case["hk"], case["d"]
    row = d // 2 + d // case["group"] * 4                              # a token's keys, or its values, of one head
    pages = 4.0 * float((-(-n // case["page"])).sum()) + 4.0 * case["batch"]
    if case["op"] == "attend_chunk":
        new = _new(case).astype(np.float64)
        used = float(n[new > 0].sum())
        pairs = float((new * n - new * (new - 1) / 2).sum())
        return {"bytes": used * hk * 2 * row + 4 * d * float(new.sum()) * case["hq"] + pages, "flops": 4.0 * pairs * case["hq"] * d}
    if case["op"] == "weigh":
        q = case["batch"] * case["queries"] * case["hq"]
        weight = float(n.sum()) * hk * (8 if case["decay"] else 4)
        return {"bytes": float(n.sum()) * hk * row + weight + q * (2 * d + 4) + pages, "flops": 2.0 * float(n.sum()) * case["queries"] * case["hq"] * d}
    # every score read, kept rows read and written with theirs, and read back as values
    kept = float(np.minimum(n, case["keep"]).sum()) * hk
    return {"bytes": 4.0 * float(n.sum()) * hk + kept * (2 * (2 * row) + 4 + 4) + kept * (2 * row + 4 * d) + 2 * pages, "flops": 2.0 * kept * d}


# ------------------------------------------------------------------------------------------------- 64 bits
def _held(s, name, b, m):
    """What the cache holds of the first m tokens of sequence b, in 64 bits [m, heads, D]."""
    case = s["case"]
    pages = s["table"][b, :-(-m // case["page"])].long()
    c = s[name + "_codes"][pages].transpose(1, 2).reshape(-1, case["hk"], case["d"] // 2)[:m].double()
    p = s[name + "_params"][pages].transpose(1, 2).reshape(-1, case["hk"], case["d"] // case["group"], 2)[:m].double()
    high = torch.floor(c / 16)
    c = torch.stack([c - 16 * high, high], -1).reshape(m, case["hk"], -1, case["group"])
    return (p[..., :1] + c * p[..., 1:]).reshape(m, case["hk"], case["d"])


def exact(case, seed):
    s = prepare(case, seed)
    n, hk, d, page = _lengths(case).tolist(), case["hk"], case["d"], case["page"]
    if case["op"] == "attend_chunk":
        g = case["hq"] // hk
        o = s["out"].double()
        a = 0
        for b, new in enumerate(_new(case).tolist()):
            if not new:
                continue
            k, v = _held(s, "k", b, n[b]), _held(s, "v", b, n[b])
            hidden = torch.arange(n[b], device=DEV) >= (torch.arange(new, device=DEV) + (n[b] - new + 1))[:, None]
            for h in range(case["hq"]):
                p = s["q"][a:a + new, h].double() @ k[:, h // g].T / math.sqrt(d)
                o[a:a + new, h] = torch.softmax(p.masked_fill_(hidden, -math.inf), -1) @ v[:, h // g]
            a += new
        return {"o": o}
    if case["op"] == "weigh":
        g = case["hq"] // hk
        w = s["out"].double()
        for b, m in enumerate(n):
            if not m:
                continue
            k = _held(s, "k", b, m)
            p = torch.einsum("jhgd,thd->htjg", s["q"][b].double().unflatten(1, (hk, g)), k) / math.sqrt(d)
            p = torch.exp(p - s["lse"][b].double().unflatten(1, (hk, g)).transpose(0, 1)[:, None])
            hidden = torch.arange(m, device=DEV)[:, None] >= m - case["queries"] + 1 + torch.arange(case["queries"], device=DEV)
            p = p.masked_fill_(hidden[None, :, :, None], 0.0).sum((2, 3))                            # [hk, t]
            t = torch.arange(m, device=DEV)
            at = s["table"][b, t // page].long()
            w[at, :, t % page] = case["decay"] * s["weights"][at, :, t % page].double() + p.T
        return {"weights": w}
    keep, recent = case["keep"], case["recent"]
    kept = np.full((case["batch"], hk, keep), -1, np.int64)
    scores = s["scores"].double()
    values = [torch.zeros(case["batch"], keep, hk, d, device=DEV, dtype=torch.float64) for _ in "kv"]
    for b, m in enumerate(n):
        if not m:
            continue
        have = min(m, keep)
        t = np.arange(m)
        old = s["scores"][s["table"][b, torch.from_numpy(t // page).to(DEV)].long(), :, torch.from_numpy(t % page).to(DEV)].cpu().numpy()
        for h in range(hk):
            stays = set(range(max(0, m - recent), m))
            rest = np.lexsort((t[:max(0, m - recent)], -old[:max(0, m - recent), h]))[:max(0, have - len(stays))]
            stays |= set(rest.tolist())
            behind = iter(sorted(x for x in stays if x >= have))
            kept[b, h, :have] = [i if i in stays else next(behind) for i in range(have)]
        i = torch.arange(have, device=DEV)
        to = s["out_table"][b, i // page].long()
        source = torch.from_numpy(kept[b, :, :have]).to(DEV)                                          # [hk, have]
        scores[to, :, i % page] = torch.from_numpy(old).to(DEV).double().T.gather(1, source).T
        for x, name in zip(values, "kv"):
            x[b, :have] = _held(s, name, b, m).gather(0, source.T[..., None].expand(-1, -1, d))
    return {"lengths": s["lengths"].clamp(max=keep), "kept": torch.from_numpy(kept).to(DEV).to(torch.int32), "scores": scores,
            "k": values[0].flatten(0, 1), "v": values[1].flatten(0, 1)}
