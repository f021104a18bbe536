"""Host-side checks of the served attention block's operators that need no GPU: refusals of the C entry points (made before a
device is touched), the torch side's refusal of CPU tensors, the cache's argument checks, rotary frequencies."""
import ctypes as C
import math

import pytest
import torch

from paper_2301_01333_b200 import binding as B
from paper_2301_01333_b200 import build as gc_build


@pytest.fixture(scope="module")
def S():
    gc_build.build()
    from paper_2301_01333_b200 import serving
    return serving


P = 1 << 20                                     # an aligned address nothing is ever read from: every call below is refused


def heads(p=P, t=128, h=64):
    return B.gc_heads_t(p, t, h)


def cache(**kw):
    d = dict(cuda_device=0, page_size=16, num_pages=4, kv_heads=2, head_dim=64, group=32, reserved_=0, k_codes=P, k_params=P, v_codes=P,
             v_params=P, status=0)
    d.update(kw)
    return B.gc_kv4_cache_t(**d)


def rope(**kw):
    d = dict(cuda_device=0, dtype=1, tokens=3, q_heads=2, k_heads=2, head_dim=64, rot_dim=64, interleaved=0, norm=1, eps=1e-6, attention_factor=1.0,
             q=heads(), k=heads(), q_out=heads(), k_out=heads(), q_weight=P, k_weight=P, positions=P, inv_freq=P)
    d.update(kw)
    return B.gc_qk_norm_rope_t(**d)


def attend(**kw):
    d = dict(batch=1, queries=1, q_heads=4, table_width=4, table_stride=4, max_length=64, scale=1.0, q=P, q_batch_stride=256, q_query_stride=256,
             q_head_stride=64, out=P, o_batch_stride=256, o_query_stride=256, o_head_stride=64, block_table=P, lengths=P)
    d.update(kw)
    return B.gc_attention_kv4_t(**d)


def prompt(**kw):
    d = dict(cuda_device=0, batch=1, q_tokens=3, k_tokens=3, q_heads=2, kv_heads=2, head_dim=64, causal=1, scale=1.0, reserved_=0, q=heads(), k=heads(),
             v=heads(), out=heads(), cu_q=P, cu_k=P, status=0)
    d.update(kw)
    return B.gc_attention_prompt_t(**d)


ARG, UNSUPPORTED, SHAPE, ALIGN = B.GC_ERR_INVALID_ARG, B.GC_ERR_UNSUPPORTED, B.GC_ERR_SHAPE, B.GC_ERR_ALIGNMENT


def refused(status, call):
    with pytest.raises(B.GcError) as e:
        call()
    assert e.value.status == status and ":" in str(e.value)


def test_qk_norm_rope_refusals(S):
    for status, kw in [(UNSUPPORTED, dict(dtype=2)), (SHAPE, dict(tokens=-1)), (UNSUPPORTED, dict(head_dim=258)), (UNSUPPORTED, dict(head_dim=63)),
                       (SHAPE, dict(rot_dim=66)), (SHAPE, dict(rot_dim=31)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=math.nan)),
                       (ARG, dict(attention_factor=math.inf)), (UNSUPPORTED, dict(q_heads=5000)), (ARG, dict(q=heads(0))), (ARG, dict(k_out=heads(0))),
                       (ALIGN, dict(q=heads(P + 1))), (SHAPE, dict(q=heads(P, -128))), (ARG, dict(positions=0)), (ALIGN, dict(positions=P + 4)),
                       (ALIGN, dict(q_weight=P + 1)), (UNSUPPORTED, dict(tokens=1 << 40))]:
        refused(status, lambda: B.gc_qk_norm_rope(0, rope(**kw)))
    B.gc_qk_norm_rope(0, rope(tokens=0, q=heads(0)))            # nothing to do: nothing to refuse
    B.gc_qk_norm_rope(0, rope(q_heads=0, k_heads=0))


@pytest.mark.parametrize("call", ["append", "read"])
def test_cache_refusals(S, call):
    f = B.gc_kv4_append if call == "append" else B.gc_kv4_read
    for status, kw in [(UNSUPPORTED, dict(head_dim=80)), (UNSUPPORTED, dict(group=48)), (UNSUPPORTED, dict(head_dim=96, group=64)),
                       (UNSUPPORTED, dict(page_size=24)), (UNSUPPORTED, dict(page_size=8)), (UNSUPPORTED, dict(page_size=512)), (SHAPE, dict(num_pages=0)),
                       (SHAPE, dict(kv_heads=0)), (ARG, dict(v_params=0)), (ALIGN, dict(k_codes=P + 8)), (ALIGN, dict(status=P + 2))]:
        refused(status, lambda: f(0, cache(**kw), 1, 3, heads(), heads(), P))
    refused(UNSUPPORTED, lambda: f(0, cache(), 4, 3, heads(), heads(), P))
    refused(SHAPE, lambda: f(0, cache(), 1, -1, heads(), heads(), P))
    refused(ARG, lambda: f(0, cache(), 1, 3, heads(0), heads(), P))
    refused(ALIGN, lambda: f(0, cache(), 0, 3, heads(), heads(P + 2), P))
    refused(ALIGN, lambda: f(0, cache(), 1, 3, heads(), heads(), P + 4))
    refused(ARG, lambda: f(0, cache(), 1, 3, heads(), heads(), 0))
    refused(UNSUPPORTED, lambda: f(0, cache(), 1, 1 << 40, heads(), heads(), P))
    f(0, cache(), 1, 0, heads(0), heads(0), 0)


def test_attention_kv4_refusals(S):
    for status, kw in [(SHAPE, dict(q_heads=3)), (SHAPE, dict(q_heads=0)), (UNSUPPORTED, dict(queries=0)), (UNSUPPORTED, dict(queries=17)),
                       (UNSUPPORTED, dict(q_heads=2 * 257)), (ARG, dict(scale=0.0)), (ARG, dict(scale=math.inf)), (SHAPE, dict(max_length=65)),
                       (SHAPE, dict(max_length=-1)), (SHAPE, dict(table_width=-1, max_length=0)), (SHAPE, dict(batch=-1)), (ARG, dict(q=0)),
                       (ARG, dict(lengths=0)), (ARG, dict(block_table=0)), (ALIGN, dict(q=P + 8)), (ALIGN, dict(out=P + 2)),
                       (ALIGN, dict(q_head_stride=65)), (SHAPE, dict(o_query_stride=-64)), (ALIGN, dict(lengths=P + 1)),
                       (UNSUPPORTED, dict(batch=1 << 23))]:
        refused(status, lambda: B.gc_attention_kv4(0, cache(), attend(**kw), None, 0))
    refused(UNSUPPORTED, lambda: B.gc_attention_kv4(0, cache(head_dim=256), attend(), None, 0))
    B.gc_attention_kv4(0, cache(), attend(batch=0), None, 0)


def test_attention_kv4_refuses_more_rows_than_a_launch_takes(S):
    many = dict(batch=1 << 20, queries=16, q_heads=512)          # 2^20 x 16 x 512 = 2^33 rows of the output
    refused(UNSUPPORTED, lambda: B.gc_attention_kv4(0, cache(), attend(**many), None, 0))


def test_attention_prompt_refusals(S):
    for status, kw in [(UNSUPPORTED, dict(head_dim=80)), (SHAPE, dict(batch=-1)), (SHAPE, dict(q_heads=3)), (SHAPE, dict(kv_heads=0)),
                       (ARG, dict(scale=math.nan)), (ARG, dict(scale=-1.0)), (UNSUPPORTED, dict(q_tokens=1 << 29)), (ARG, dict(q=heads(0))),
                       (ALIGN, dict(k=heads(P + 8))), (ALIGN, dict(v=heads(P, 132))), (ALIGN, dict(out=heads(P, 128, 60))), (ARG, dict(cu_q=0)),
                       (ALIGN, dict(cu_k=P + 2)), (ALIGN, dict(status=P + 1)), (SHAPE, dict(out=heads(P, -128)))]:
        refused(status, lambda: B.gc_attention_prompt(0, prompt(**kw)))
    B.gc_attention_prompt(0, prompt(batch=0))
    B.gc_attention_prompt(0, prompt(q_tokens=0, q=heads(0)))


def test_status_word_refusals(S):
    refused(ARG, lambda: B.gc_serving_status(0, 0))
    refused(ALIGN, lambda: B.gc_serving_status(0, P + 2))


def test_descriptors_have_the_layout_of_the_header(S):
    assert C.sizeof(B.gc_heads_t) == 24 and C.sizeof(B.gc_qk_norm_rope_t) == 48 + 4 * 24 + 32
    assert C.sizeof(B.gc_kv4_cache_t) == 32 + 5 * 8 and C.sizeof(B.gc_attention_kv4_t) == 32 + 10 * 8 and C.sizeof(B.gc_attention_prompt_t) == 48 + 4 * 24 + 24


def test_tensors_on_the_cpu_are_refused(S):
    x, pos, inv = torch.zeros(2, 2, 64), torch.zeros(2, dtype=torch.int64), torch.ones(32)
    cu = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: S.qk_norm_rope(x, x, pos, inv), lambda: S.KV4Cache.allocate(1, 16, 1, 64, 64, device="cpu"),
                 lambda: S.attention_prompt(x.bfloat16(), x.bfloat16(), x.bfloat16(), cu)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        S.qk_norm_rope(x, x, None, inv)


def test_cache_shapes_are_checked(S):
    codes, params = torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1, 16, 2, 2, dtype=torch.bfloat16)
    for bad in ((codes[0], params, codes, params), (codes, params, codes[:1], params), (codes, params.float(), codes, params),
                (codes, params[:, :, :, :, :1], codes, params), (codes.transpose(1, 2), params, codes, params),
                (codes, torch.zeros(2, 1, 16, 3, 2, dtype=torch.bfloat16), codes, torch.zeros(2, 1, 16, 3, 2, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            S.KV4Cache(*bad)
    with pytest.raises(ValueError):
        S.KV4Cache.allocate(1, 16, 1, 64, 48, device="cpu")


def test_rotary_inv_freq(S):
    f = S.rotary_inv_freq(128)
    assert f.dtype == torch.float32 and f.shape == (64,) and f[0] == 1
    want = torch.tensor([10000.0 ** (-2 * i / 128) for i in range(64)], dtype=torch.float64)
    assert torch.equal(f, want.float())
    assert torch.equal(S.rotary_inv_freq(128, scaling="linear", factor=8.0), (want / 8).float())
    base = S.rotary_inv_freq(128, scaling="base", factor=8.0).double()
    assert base[0] == 1 and abs(base[-1] / want[-1] - 1 / 8) < 1e-6 and (base[1:] < want[1:]).all()
    bands = S.rotary_inv_freq(128, scaling="bands", factor=8.0, original_length=4096, low=1.0, high=4.0).double()
    turns = 4096 * want / (2 * math.pi)
    assert torch.equal(bands[turns >= 4], want[turns >= 4].float().double())
    assert torch.equal(bands[turns <= 1], (want[turns <= 1] / 8).float().double())
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and ((bands < want) & (bands > want / 8))[mid].all()
    assert S.rotary_inv_freq(0).shape == (0,) and torch.equal(S.rotary_inv_freq(2), torch.ones(1))
    for bad in (lambda: S.rotary_inv_freq(3), lambda: S.rotary_inv_freq(64, scaling="x"), lambda: S.rotary_inv_freq(64, scaling="linear", factor=0.5),
                lambda: S.rotary_inv_freq(64, scaling="bands", factor=2.0, low=4.0, high=1.0)):
        with pytest.raises(ValueError):
            bad()
