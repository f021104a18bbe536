"""The operators of a served attention block on torch tensors: argument checks and marshalling for the ``gc_qk_norm_rope``,
``gc_kv4_*`` and ``gc_attention_*`` entry points of ``include/gc.h``, which state what each computes.

They serve: no gradient is recorded, and a tensor that requires one is refused unless gradients are off (``torch.no_grad()``).
All of them are asynchronous on the current stream of their tensors' device, take strided tensors (the last dimension
contiguous), can be captured into a CUDA graph (after a first call outside the capture, which loads their kernels), and raise
``GcError`` (or ``TypeError`` / ``ValueError`` for tensors of the wrong type, shape or device) before anything is launched.  What only the device can see - a slot, page, length or offset out
of bounds - leaves the outputs of that call undefined and is recorded in a status word: ``KV4Cache.query_status()`` for a cache's
calls, ``query_status()`` for those of ``attention_prompt``, or ``query_status(word)`` where it was given a word of its own.
"""
from __future__ import annotations

import ctypes
import math
from typing import Dict, Optional, Tuple

import torch

from . import binding as B
from .binding import GcError  # noqa: F401

B.load_library()
try:
    from . import _serving
except ImportError as e:
    raise ImportError(f"the torch side of the library is missing: build it with `python -m paper_2301_01333_b200.build` ({e})") from e
_serving.set_error_class(GcError)


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
    return _serving.qk_norm_rope(q, k, positions, inv_freq, q_weight, k_weight, norm, eps, interleaved, attention_factor, q_out, k_out)


def new_status(device="cuda") -> torch.Tensor:
    """A status word for ``attention_prompt``."""
    return torch.zeros(1, dtype=torch.int32, device=device)


_words: Dict[int, torch.Tensor] = {}            # by device: the word of attention_prompt calls that are given none


def _word_of(device: torch.device) -> torch.Tensor:
    word = _words.get(device.index)
    if word is None:
        with torch.cuda.device(device):
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a device's first attention_prompt is made outside of a capture, or is given a status word")
            word = new_status(device)
            torch.cuda.current_stream().synchronize()            # the word is zero before a call on any stream
        word = _words.setdefault(device.index, word)
    return word


def query_status(word: Optional[torch.Tensor] = None) -> None:
    """Synchronise the current stream; raise GcError for what the device recorded in `word`, and clear it.  Without a word: what
    ``attention_prompt`` calls on the current device recorded that were given none."""
    if word is None:
        word = _word_of(torch.device("cuda", torch.cuda.current_device()))
    if not isinstance(word, torch.Tensor):
        raise TypeError("a status word is a torch.Tensor, as new_status makes it")
    if word.dtype != torch.int32 or word.numel() != 1 or not word.is_cuda:
        raise ValueError(f"a status word is one int32 on a CUDA device, as new_status makes it, not {word.dtype} {tuple(word.shape)} on {word.device}")
    with torch.cuda.device(word.device):
        B.gc_serving_status(torch.cuda.current_stream(word.device).cuda_stream, word.data_ptr())


class KV4Cache:
    """A paged cache of keys and values in 4 bits over four dense tensors:

      codes   uint8    [pages, kv_heads, page_size, head_dim / 2]
      params  bfloat16 [pages, kv_heads, page_size, head_dim / group, 2]

    page_size a power of two from 16 to 256, head_dim 64, 96 or 128, group 32, 64 or 128.  The object keeps the tensors alive
    and a status word, nothing else: it may be used on any stream, as far as the caller orders the accesses.  It is made for these
    tensors: they cannot be replaced by others, and a call is refused once the memory of one has been."""

    def __init__(self, k_codes: torch.Tensor, k_params: torch.Tensor, v_codes: torch.Tensor, v_params: torch.Tensor):
        for name, t in (("k_codes", k_codes), ("k_params", k_params), ("v_codes", v_codes), ("v_params", v_params)):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
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
        if self.device.type != "cuda":
            raise ValueError(f"a cache lives on a CUDA device, not {self.device}")
        self.pages, self.kv_heads, self.page_size, self.head_dim, self.group = pages, heads, page, 2 * half, 2 * half // groups
        self.k_codes, self.k_params, self.v_codes, self.v_params = self._tensors = k_codes, k_params, v_codes, v_params
        self.status = new_status(self.device)
        self._desc = B.gc_kv4_cache_t(self.device.index, page, pages, heads, 2 * half, self.group, 0, k_codes.data_ptr(), k_params.data_ptr(),
                                      v_codes.data_ptr(), v_params.data_ptr(), self.status.data_ptr())
        self._at = ctypes.addressof(self._desc)

    def __setattr__(self, name, value):
        if "_at" in self.__dict__ and name in self.__dict__:
            raise AttributeError(f"{name} of a KV4Cache is fixed: make another one over other tensors")
        super().__setattr__(name, value)

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
        _serving.kv4_append(self._at, k, v, slots, self._tensors)

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, k_out: Optional[torch.Tensor] = None,
             v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The values held at slots, [tokens, kv_heads, head_dim], of type dtype or that of the outputs given; rows of negative
        slots are left as they were (zeros in outputs made here)."""
        if not isinstance(slots, torch.Tensor):
            raise TypeError("slots must be a torch.Tensor")
        if slots.dim() != 1:
            raise ValueError(f"slots must be a vector, not {tuple(slots.shape)}")
        if k_out is None or v_out is None:
            like = k_out if k_out is not None else v_out
            shape = (slots.shape[0], self.kv_heads, self.head_dim)
            made = torch.zeros(shape, dtype=dtype if like is None else like.dtype, device=self.device)
            k_out, v_out = (made, torch.zeros_like(made)) if like is None else (made if k_out is None else k_out, made if v_out is None else v_out)
        _serving.kv4_read(self._at, slots, k_out, v_out, self._tensors)
        return k_out, v_out

    def attend(self, q: torch.Tensor, block_table: torch.Tensor, lengths: torch.Tensor, *, scale: Optional[float] = None,
               max_length: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q bf16 [batch, queries, q_heads, head_dim] over the sequences block_table (int32 [batch, width], pages in
        order) names, lengths (int32 [batch]) counting the tokens appended so far, the queries' own among them: query j sees
        the first lengths - (queries - 1) + j of them.  scale: head_dim ** -0.5 if not given; max_length: a bound of lengths the
        caller knows (the work is laid out for it; a longer sequence is an error), width * page_size if not given.  A value above 2^32
        or a score above 2^26 in size, more than the sums and weights can hold, is reported by ``query_status()``; values below
        2^-40 lose accuracy."""
        return _serving.kv4_attend(self._at, q, block_table, lengths, scale, max_length, out, self._tensors)

    def query_status(self) -> None:
        """Synchronise the current stream; raise GcError if a call found a slot, page or length out of bounds since the last one."""
        query_status(self.status)


def attention_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: Optional[torch.Tensor] = None, *,
                     causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of packed sequences, bf16: q [q_tokens, q_heads, head_dim], k and v [k_tokens, kv_heads, head_dim]; sequence b owns
    query rows cu_q[b] .. cu_q[b + 1] and key rows cu_k[b] .. cu_k[b + 1] (int32 [batch + 1]; cu_k = cu_q if not given).  causal:
    query row i of nq sees the first i + 1 + nk - nq keys.  A row that sees none is zero; rows no sequence owns are left as they
    were in a given `out`, and are zero in one made here.  status: a word (``new_status``) for what only the device can see; the
    device's own, which ``query_status()`` reads, if not given.  A finite score above 2^26 in size is reported there as well."""
    if not isinstance(q, torch.Tensor):
        raise TypeError("q must be a torch.Tensor")
    if out is None:
        out = torch.zeros(q.shape, dtype=torch.bfloat16, device=q.device)
    if status is None and q.is_cuda:
        status = _word_of(q.device)
    return _serving.attention_prompt(q, k, v, cu_q, cu_k, causal, scale, out, status)
