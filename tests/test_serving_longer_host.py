"""Refusals of chunked attention over the 4-bit cache, of the weights its tokens receive and of eviction that need no GPU: made
before a device is touched."""
import ctypes as C
import math

import pytest
import torch

from paper_2301_01333_b200 import binding as B
from test_serving_host import ALIGN, ARG, P, SHAPE, UNSUPPORTED, S, attend, cache, heads, refused  # noqa: F401


def chunk(**kw):
    d = dict(batch=1, q_heads=4, q_tokens=5, table_width=4, max_length=64, table_stride=4, scale=1.0, reserved_=0, q=heads(P, 256), out=heads(P, 256),
             cu_q=P, block_table=P, lengths=P)
    d.update(kw)
    return B.gc_attention_kv4_chunk_t(**d)


def weigh(**kw):
    d = dict(batch=1, queries=1, q_heads=4, table_width=4, table_stride=4, max_length=64, scale=1.0, q=P, q_batch_stride=256, q_query_stride=256,
             q_head_stride=64, lse=P, block_table=P, lengths=P, weights=P, out=P, decay=1.0, reserved_=0)
    d.update(kw)
    return B.gc_kv4_weigh_t(**d)


def evict(**kw):
    d = dict(batch=1, keep=8, recent=4, max_length=64, table_width=4, out_table_width=0, table_stride=4, out_table_stride=0, block_table=P, out_table=0,
             lengths=P, out_lengths=P, kept=P, scores=P)
    d.update(kw)
    return B.gc_kv4_evict_t(**d)


def test_chunk_refusals(S):
    for status, kw in [(SHAPE, dict(batch=-1)), (SHAPE, dict(q_tokens=-1)), (SHAPE, dict(q_heads=3)), (SHAPE, dict(q_heads=0)),
                       (UNSUPPORTED, dict(q_heads=2 * 257)), (ARG, dict(scale=0.0)), (ARG, dict(scale=math.nan)), (SHAPE, dict(max_length=-1)),
                       (SHAPE, dict(max_length=65)), (SHAPE, dict(table_width=-1, max_length=0)), (SHAPE, dict(table_stride=-4)), (ARG, dict(cu_q=0)),
                       (ARG, dict(lengths=0)), (ARG, dict(block_table=0)), (ALIGN, dict(cu_q=P + 2)), (ALIGN, dict(lengths=P + 1)),
                       (ALIGN, dict(block_table=P + 2)), (ARG, dict(q=heads(0))), (ALIGN, dict(q=heads(P + 8))), (ALIGN, dict(out=heads(P, 132))),
                       (SHAPE, dict(out=heads(P, -256))), (UNSUPPORTED, dict(q_tokens=1 << 31)), (UNSUPPORTED, dict(batch=1 << 21)),
                       (UNSUPPORTED, dict(q_tokens=1 << 28, max_length=1 << 27, table_width=1 << 23))]:
        refused(status, lambda: B.gc_attention_kv4_chunk(0, cache(), chunk(**kw), P, 1 << 40))
    refused(UNSUPPORTED, lambda: B.gc_attention_kv4_chunk(0, cache(head_dim=80), chunk(), P, 1 << 40))
    refused(SHAPE, lambda: B.gc_attention_kv4_chunk_workspace_bytes(cache(), chunk(q_heads=3)))
    B.gc_attention_kv4_chunk(0, cache(), chunk(batch=0), None, 0)
    B.gc_attention_kv4_chunk(0, cache(), chunk(q_tokens=0, q=heads(0)), None, 0)
    assert B.gc_attention_kv4_chunk_workspace_bytes(cache(), chunk(q_tokens=0)) == 0


def test_weigh_refusals(S):
    for status, kw in [(SHAPE, dict(batch=-1)), (SHAPE, dict(q_heads=3)), (UNSUPPORTED, dict(queries=0)), (UNSUPPORTED, dict(queries=17)),
                       (UNSUPPORTED, dict(q_heads=2 * 257)), (ARG, dict(scale=-1.0)), (ARG, dict(decay=-0.5)), (ARG, dict(decay=math.nan)),
                       (ARG, dict(decay=math.inf)), (SHAPE, dict(max_length=65)), (SHAPE, dict(max_length=-1)), (ARG, dict(q=0)), (ARG, dict(lse=0)),
                       (ARG, dict(lengths=0)), (ARG, dict(weights=0)), (ARG, dict(out=0)), (ARG, dict(block_table=0)), (ALIGN, dict(q=P + 8)),
                       (ALIGN, dict(q_head_stride=65)), (SHAPE, dict(q_batch_stride=-256)), (ALIGN, dict(lse=P + 2)), (ALIGN, dict(weights=P + 1)),
                       (UNSUPPORTED, dict(batch=1 << 23))]:
        refused(status, lambda: B.gc_kv4_weigh(0, cache(), weigh(**kw)))
    B.gc_kv4_weigh(0, cache(), weigh(batch=0, q=0))
    B.gc_kv4_weigh(0, cache(), weigh(max_length=0, q=0))


def test_evict_refusals(S):
    for status, kw in [(SHAPE, dict(batch=-1)), (ARG, dict(keep=-1)), (ARG, dict(recent=-1)), (ARG, dict(recent=9)), (SHAPE, dict(max_length=-1)),
                       (SHAPE, dict(max_length=65)), (ARG, dict(lengths=0)), (ARG, dict(out_lengths=0)), (ARG, dict(kept=0)), (ARG, dict(scores=0)),
                       (ARG, dict(block_table=0)), (ALIGN, dict(scores=P + 8)), (ALIGN, dict(kept=P + 2)), (SHAPE, dict(out_table=P, out_table_width=0)),
                       (ALIGN, dict(out_table=P + 2, out_table_width=1)), (SHAPE, dict(out_table=P, out_table_width=1, out_table_stride=-1)),
                       (UNSUPPORTED, dict(batch=1 << 20, keep=1 << 20)), (UNSUPPORTED, dict(batch=1 << 30))]:
        refused(status, lambda: B.gc_kv4_evict(0, cache(), evict(**kw), P, 1 << 40))
    refused(ARG, lambda: B.gc_kv4_evict(0, cache(), evict(), None, 0))            # holes and what fills them: 2 x 2 heads x 8 numbers
    assert B.gc_kv4_evict_workspace_bytes(cache(), evict()) == 2 * 2 * 8 * 4
    assert B.gc_kv4_evict_workspace_bytes(cache(), evict(keep=64)) == 0 and B.gc_kv4_evict_workspace_bytes(cache(), evict(keep=60)) == 2 * 2 * 4 * 4
    B.gc_kv4_evict(0, cache(), evict(batch=0), None, 0)


def test_evict_refuses_budgets_that_leave_no_room_to_count(S):
    # new positions are counted in 32 bits, a cluster's threads (8 x 1024) at a time: the last step may not pass 2^31
    top = (1 << 31) - 1
    for keep in (top - 65535, top - 8191, top):
        refused(UNSUPPORTED, lambda: B.gc_kv4_evict_workspace_bytes(cache(kv_heads=1), evict(keep=keep)))
        refused(UNSUPPORTED, lambda: B.gc_kv4_evict(0, cache(kv_heads=1), evict(keep=keep), P, 1 << 40))
        refused(UNSUPPORTED, lambda: B.gc_kv4_evict_workspace_bytes(cache(kv_heads=1), evict(keep=0, recent=0, max_length=keep, table_width=1 << 30)))
    assert B.gc_kv4_evict_workspace_bytes(cache(kv_heads=1), evict(keep=top - 65536)) == 0


def test_lse_refusals(S):
    refused(ARG, lambda: B.gc_attention_kv4_lse(0, cache(), attend(), 0, None, 0))
    refused(ALIGN, lambda: B.gc_attention_kv4_lse(0, cache(), attend(), P + 2, None, 0))
    refused(UNSUPPORTED, lambda: B.gc_attention_kv4_lse(0, cache(), attend(queries=17), P, None, 0))
    B.gc_attention_kv4_lse(0, cache(), attend(batch=0), 0, None, 0)


def test_descriptors_have_the_layout_of_the_header(S):
    assert C.sizeof(B.gc_attention_kv4_chunk_t) == 40 + 2 * 24 + 3 * 8
    assert C.sizeof(B.gc_kv4_weigh_t) == 32 + 4 * 8 + 5 * 8 + 8 and C.sizeof(B.gc_kv4_evict_t) == 24 + 2 * 8 + 6 * 8


def test_a_cache_on_the_cpu_is_refused_before_its_methods(S):
    with pytest.raises(ValueError, match="CUDA"):
        S.KV4Cache.allocate(1, 16, 1, 64, 64, device="cpu")
    with pytest.raises(TypeError, match="torch.Tensor"):
        S.KV4Cache.attend_chunk(None, [1], None, None, None)
    assert torch.is_tensor(torch.zeros(1))
