"""The operators of a served attention block on torch tensors: argument checks and marshalling for the ``gc_qk_norm_rope``,
``gc_kv4_*`` and ``gc_attention_*`` entry points of ``include/gc.h``, which state what each computes.

All of them are asynchronous on the current stream of their tensors' device, take strided tensors (the last dimension
contiguous), can be captured into a CUDA graph, and raise ``GcError`` (or ``TypeError`` / ``ValueError`` for tensors of the
wrong type, shape or device) before anything is launched.  What only the device can see - a slot, page, length or offset out
of bounds - leaves the outputs of that call undefined and is recorded in a status word: ``KV4Cache.query_status()``, or
``query_status(word)`` for the word given to ``attention_prompt``.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import binding as B
from .binding import GcError  # noqa: F401

_DTYPE = {torch.float32: 0, torch.bfloat16: 1}


def _stream(device: torch.device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _index(device: torch.device) -> int:
    if device.type != "cuda":
        raise ValueError(f"tensors must be on a CUDA device, not {device}")
    return device.index


def _vector(name: str, t: torch.Tensor, n: int, dtype: torch.dtype, device: torch.device) -> int:
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or t.device != device or not (n < 2 or t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {n} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(name: str, t: torch.Tensor, shape, dtype: torch.dtype, device: torch.device) -> B.gc_heads_t:
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    s = t.stride()
    if s[2] != 1 and shape[2] > 1 and t.numel():
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return B.gc_heads_t(t.data_ptr(), s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0)


def _no_alias(name: str, t: torch.Tensor) -> None:
    """An output whose rows share memory (an expanded tensor) would be written by several threads at once."""
    for n, s in zip(t.shape, t.stride()):
        if n > 1 and s == 0:
            raise ValueError(f"{name}: an output cannot be an expanded tensor")


def rotary_inv_freq(rot_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                    original_length: int = 8192, low: float = 1.0, high: float = 4.0, device=None) -> torch.Tensor:
    """The frequencies base ** (-2 i / rot_dim), i < rot_dim / 2, fp32, for ``qk_norm_rope``; for contexts `factor` times the
    length the model learned, scaled by

      "linear"  every frequency divided by factor (positions squeezed into the learned range);
      "base"    a larger base, base * factor ** (rot_dim / (rot_dim - 2)): the slowest frequency divided by factor, the fastest kept;
      "bands"   frequencies that turn at least `high` times in original_length kept, those that turn at most `low` times divided
                by factor, linear in the number of turns between."""
    if rot_dim < 0 or rot_dim % 2:
        raise ValueError("rot_dim must be even")
    if scaling not in (None, "linear", "base", "bands"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling and not factor >= 1.0:
        raise ValueError("factor must be at least 1")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / max(rot_dim, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        if not high > low:
            raise ValueError("high must exceed low")
        turns = original_length * f / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f.to(torch.float32).to(device) if device is not None else f.to(torch.float32)


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, inv_freq: torch.Tensor,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, *, norm: bool = True,
                 eps: float = 1e-6, interleaved: bool = False, attention_factor: float = 1.0,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """RMS norm over each head of q [tokens, q_heads, head_dim] and k [tokens, k_heads, head_dim] (fp32 or bf16; weights
    [head_dim] of the same type, None = ones; norm=False: none) and rotation of the first 2 len(inv_freq) elements by
    positions (int64 [tokens]) times inv_freq (fp32).  Pairs (i, i + rot / 2), or (2 i, 2 i + 1) if interleaved.  Returns
    (q_out, k_out); q_out=q, k_out=k works in place."""
    device, dtype = q.device, q.dtype
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q and k must be [tokens, heads, head_dim]")
    if dtype not in _DTYPE:
        raise TypeError(f"q must be float32 or bfloat16, not {dtype}")
    dev = _index(device)
    t, hq, d = q.shape
    hk = k.shape[1]
    if q_out is None:
        q_out = torch.empty((t, hq, d), dtype=dtype, device=device)
    else:
        _no_alias("q_out", q_out)
    if k_out is None:
        k_out = torch.empty((t, hk, d), dtype=dtype, device=device)
    else:
        _no_alias("k_out", k_out)
    half = inv_freq.shape[0] if inv_freq.dim() == 1 else -1
    desc = B.gc_qk_norm_rope_t(
        dev, _DTYPE[dtype], t, hq, hk, d, 2 * half, interleaved, norm, eps, attention_factor,
        _heads("q", q, q.shape, dtype, device), _heads("k", k, (t, hk, d), dtype, device),
        _heads("q_out", q_out, q.shape, dtype, device), _heads("k_out", k_out, (t, hk, d), dtype, device),
        None if q_weight is None else _vector("q_weight", q_weight, d, dtype, device),
        None if k_weight is None else _vector("k_weight", k_weight, d, dtype, device),
        _vector("positions", positions, t, torch.int64, device), _vector("inv_freq", inv_freq, half, torch.float32, device))
    B.gc_qk_norm_rope(_stream(device), desc)
    return q_out, k_out


def new_status(device="cuda") -> torch.Tensor:
    """A status word for ``attention_prompt``."""
    return torch.zeros(1, dtype=torch.int32, device=device)


def query_status(word: torch.Tensor) -> None:
    """Synchronise the current stream; raise GcError for what the device recorded in `word`, and clear it."""
    with torch.cuda.device(word.device):
        B.gc_serving_status(_stream(word.device), word.data_ptr())


class KV4Cache:
    """A paged cache of keys and values in 4 bits over four dense tensors:

      codes   uint8    [pages, kv_heads, page_size, head_dim / 2]
      params  bfloat16 [pages, kv_heads, page_size, head_dim / group, 2]

    page_size a power of two from 16 to 256, head_dim 64, 96 or 128, group 32, 64 or 128.  The object keeps the tensors alive
    and a status word, nothing else: it may be used on any stream, as far as the caller orders the accesses."""

    def __init__(self, k_codes: torch.Tensor, k_params: torch.Tensor, v_codes: torch.Tensor, v_params: torch.Tensor):
        if k_codes.dim() != 4 or k_params.dim() != 5:
            raise ValueError("codes must be [pages, heads, page_size, head_dim / 2], params [pages, heads, page_size, groups, 2]")
        pages, heads, page, half = k_codes.shape
        groups = k_params.shape[3]
        for name, t, shape, dtype in (("k_codes", k_codes, k_codes.shape, torch.uint8), ("v_codes", v_codes, k_codes.shape, torch.uint8),
                                      ("k_params", k_params, (pages, heads, page, groups, 2), torch.bfloat16),
                                      ("v_params", v_params, (pages, heads, page, groups, 2), torch.bfloat16)):
            if t.shape != shape or t.dtype != dtype or t.device != k_codes.device or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on {k_codes.device}")
        if groups == 0 or (2 * half) % groups:
            raise ValueError("the groups must divide the head dimension")
        self.device = k_codes.device
        dev = _index(self.device)
        self.pages, self.kv_heads, self.page_size, self.head_dim, self.group = pages, heads, page, 2 * half, 2 * half // groups
        self.k_codes, self.k_params, self.v_codes, self.v_params = k_codes, k_params, v_codes, v_params
        self.status = new_status(self.device)
        self._desc = B.gc_kv4_cache_t(dev, page, pages, heads, 2 * half, self.group, 0, k_codes.data_ptr(), k_params.data_ptr(),
                                      v_codes.data_ptr(), v_params.data_ptr(), self.status.data_ptr())

    @classmethod
    def allocate(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, group: int = 64, device="cuda") -> "KV4Cache":
        """A cache of `pages` empty pages (zeros: every value held is 0)."""
        if group <= 0 or head_dim % group:
            raise ValueError("group must divide head_dim")
        shape = (pages, kv_heads, page_size)

        def codes():
            return torch.zeros(shape + (head_dim // 2,), dtype=torch.uint8, device=device)

        def params():
            return torch.zeros(shape + (head_dim // group, 2), dtype=torch.bfloat16, device=device)
        return cls(codes(), params(), codes(), params())

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """Write rows k, v [tokens, kv_heads, head_dim] (fp32 or bf16) at slots (int64 [tokens], page * page_size + offset;
        negative: the row is skipped).  No slot may be named twice in a call."""
        n, dtype = slots.shape[0], k.dtype
        if dtype not in _DTYPE:
            raise TypeError(f"k must be float32 or bfloat16, not {dtype}")
        shape = (n, self.kv_heads, self.head_dim)
        B.gc_kv4_append(_stream(self.device), self._desc, _DTYPE[dtype], n, _heads("k", k, shape, dtype, self.device),
                        _heads("v", v, shape, dtype, self.device), _vector("slots", slots, n, torch.int64, self.device))

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, k_out: Optional[torch.Tensor] = None,
             v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The values held at slots, [tokens, kv_heads, head_dim], of type dtype or that of the outputs given; rows of negative
        slots are left as they were (zeros in outputs made here)."""
        n = slots.shape[0]
        shape = (n, self.kv_heads, self.head_dim)
        if k_out is not None:
            dtype = k_out.dtype
        elif v_out is not None:
            dtype = v_out.dtype
        if dtype not in _DTYPE:
            raise TypeError(f"values are read as float32 or bfloat16, not {dtype}")
        if k_out is None:
            k_out = torch.zeros(shape, dtype=dtype, device=self.device)
        else:
            _no_alias("k_out", k_out)
        if v_out is None:
            v_out = torch.zeros(shape, dtype=dtype, device=self.device)
        else:
            _no_alias("v_out", v_out)
        B.gc_kv4_read(_stream(self.device), self._desc, _DTYPE[dtype], n, _heads("k_out", k_out, shape, dtype, self.device),
                      _heads("v_out", v_out, shape, dtype, self.device), _vector("slots", slots, n, torch.int64, self.device))
        return k_out, v_out

    def attend(self, q: torch.Tensor, block_table: torch.Tensor, lengths: torch.Tensor, *, scale: Optional[float] = None,
               max_length: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q bf16 [batch, queries, q_heads, head_dim] over the sequences block_table (int32 [batch, width], pages in
        order) names, lengths (int32 [batch]) counting the tokens appended so far, the queries' own among them: query j sees
        the first lengths - (queries - 1) + j of them.  scale: head_dim ** -0.5 if not given; max_length: a bound of lengths the
        caller knows (the work is laid out for it; a longer sequence is an error), width * page_size if not given."""
        device = self.device
        if q.dim() != 4 or q.dtype != torch.bfloat16 or q.device != device or q.shape[3] != self.head_dim:
            raise ValueError(f"q must be bfloat16 [batch, queries, q_heads, {self.head_dim}] on {device}")
        b, n, hq, d = q.shape
        qs = q.stride()
        if qs[3] != 1:
            raise ValueError("q: the last dimension must be contiguous")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or block_table.shape[0] != b or block_table.device != device:
            raise ValueError(f"block_table must be int32 [{b}, width] on {device}")
        width = block_table.shape[1]
        ts = block_table.stride()
        if ts[1] != 1 and width > 1:
            raise ValueError("block_table: rows must be contiguous")
        if out is None:
            out = torch.empty((b, n, hq, d), dtype=torch.bfloat16, device=device)
        else:
            if out.shape != q.shape or out.dtype != torch.bfloat16 or out.device != device or out.stride(3) != 1:
                raise ValueError("out must be like q, its last dimension contiguous")
            _no_alias("out", out)
        os = out.stride()
        desc = B.gc_attention_kv4_t(
            b, n, hq, width, ts[0], width * self.page_size if max_length is None else max_length,
            d ** -0.5 if scale is None else scale, q.data_ptr(),
            qs[0] if b > 1 else 0, qs[1] if n > 1 else 0, qs[2] if hq > 1 else 0, out.data_ptr(),
            os[0] if b > 1 else 0, os[1] if n > 1 else 0, os[2] if hq > 1 else 0,
            block_table.data_ptr(), _vector("lengths", lengths, b, torch.int32, device))
        need = B.gc_attention_kv4_workspace_bytes(self._desc, desc)
        # from torch's allocator, so that calls on several streams or in several captured graphs never share it
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        B.gc_attention_kv4(_stream(device), self._desc, desc, ws.data_ptr() if need else None, need)
        return out

    def query_status(self) -> None:
        """Synchronise the current stream; raise GcError if a call found a slot, page or length out of bounds since the last one."""
        query_status(self.status)


def attention_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: Optional[torch.Tensor] = None, *,
                     causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of packed sequences, bf16: q [q_tokens, q_heads, head_dim], k and v [k_tokens, kv_heads, head_dim]; sequence b owns
    query rows cu_q[b] .. cu_q[b + 1] and key rows cu_k[b] .. cu_k[b + 1] (int32 [batch + 1]; cu_k = cu_q if not given).  causal:
    query row i of nq sees the first i + 1 + nk - nq keys.  A row that sees none is zero; rows no sequence owns are left as they
    were in a given `out`, and are zero in one made here."""
    device = q.device
    dev = _index(device)
    if q.dim() != 3 or k.dim() != 3 or q.dtype != torch.bfloat16:
        raise ValueError("q, k and v must be bfloat16 [tokens, heads, head_dim]")
    t, hq, d = q.shape
    tk, hk = k.shape[0], k.shape[1]
    if cu_k is None:
        cu_k = cu_q
    nb = cu_q.shape[0]
    if nb < 1:
        raise ValueError("cu_q must have batch + 1 elements")
    if out is None:
        out = torch.zeros((t, hq, d), dtype=torch.bfloat16, device=device)
    else:
        _no_alias("out", out)
    if status is not None and (status.dtype != torch.int32 or status.device != device):
        raise ValueError(f"status must be an int32 tensor on {device}")
    desc = B.gc_attention_prompt_t(
        dev, nb - 1, t, tk, hq, hk, d, causal, d ** -0.5 if scale is None else scale, 0,
        _heads("q", q, (t, hq, d), torch.bfloat16, device), _heads("k", k, (tk, hk, d), torch.bfloat16, device),
        _heads("v", v, (tk, hk, d), torch.bfloat16, device), _heads("out", out, (t, hq, d), torch.bfloat16, device),
        _vector("cu_q", cu_q, nb, torch.int32, device), _vector("cu_k", cu_k, nb, torch.int32, device),
        None if status is None else status.data_ptr())
    B.gc_attention_prompt(_stream(device), desc)
    return out
