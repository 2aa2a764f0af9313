"""Attention over a growing sequence of frames: a layer that is trained on whole sequences, takes a prompt at once and then one token after the
other, with the bsga kernels: norms of queries and keys with the position rotation, attention with a sliding window of frames and
first tokens that stay visible, attention of single tokens over a paged cache.

Integration shape only, as GlobalAttentionBlock: random weights.
"""
from __future__ import annotations

from contextlib import contextmanager
from typing import List, Optional, Sequence

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

from . import binding as B
from .block import _calls_are_watched


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_weight, k_weight, q_bias, k_bias, positions, norm, eps, base):
        ctx.save_for_backward(q, k, q_weight, k_weight, q_bias, k_bias, positions)
        ctx.args, ctx.with_v = dict(norm=norm, eps=eps, base=base), v is not None
        return B.bsga_qk_norm_rope(q, k, positions, q_weight, k_weight, q_bias, k_bias, v=v, norm=norm, eps=eps, base=base)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        q, k, q_weight, k_weight, q_bias, k_bias, positions = ctx.saved_tensors
        got = B.bsga_qk_norm_rope_bwd(dq.contiguous(), dk.contiguous(), q, k, positions, q_weight, k_weight, q_bias, k_bias,
                                      dv=dv.contiguous() if ctx.with_v else None, **ctx.args)
        of = [None if g is None else g.to(q.dtype) for g in got]
        return (*of, None, None, None, None)


class _WindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, sinks, frame, q_start, softmax_scale):
        ctx.args = dict(window=window, sinks=sinks, frame=frame, q_start=q_start, softmax_scale=softmax_scale)
        out, lse = B.bsga_window_attn(q, k, v, return_lse=True, **ctx.args)
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        return (*B.bsga_window_attn_bwd(dout.contiguous(), q, k, v, out, lse, **ctx.args), None, None, None, None, None)


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, q_bias: Optional[torch.Tensor] = None,
                 k_bias: Optional[torch.Tensor] = None, norm: Optional[str] = "rms", eps: float = 1e-6, base: float = 10000.0):
    """bsga_qk_norm_rope with gradients: q [N, H, 64], k and v [N, Hkv, 64] -> (q [H, N, 64], k [Hkv, N, 64], v or None)."""
    return _QkNormRope.apply(q, k, v, q_weight, k_weight, q_bias, k_bias, positions, norm, eps, base)


def window_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, window: Optional[int] = None, sinks: int = 0, frame: int = 1,
                     q_start: Optional[int] = None, softmax_scale: Optional[float] = None) -> torch.Tensor:
    """bsga_window_attn with gradients: q [H, N, 64], k and v [Hkv, M, 64] -> [H, N, 64]."""
    return _WindowAttention.apply(q, k, v, window, sinks, frame, q_start, softmax_scale)


class PagedCache:
    """Keys and values of several sequences in pages [pages, kv_heads, page, 64], and which page holds which tokens.  The bookkeeping is
    the host's; grow() and trim() bring the device's table and lengths up to date on the current stream.  Places of the table without a page, of
    freed ones too, hold -1, which bsga_paged_attn takes for page 0: check_seen() tells whether a window reaches them.
    width: pages of the longest sequence, by default all.  The attention is dealt out by it, so a table much wider than its sequences is slow: 16
    sequences of 12,000 tokens on 4 key heads, page 64, take 38 us with a width of 188 and 225 with 3,008."""

    def __init__(self, sequences: int, pages: int, kv_heads: int, page: int = 64, width: Optional[int] = None, dtype=torch.bfloat16,
                 device="cuda"):
        self.page, self.width = page, pages if width is None else width
        self.k = torch.zeros((pages, kv_heads, page, 64), dtype=dtype, device=device)
        self.v = torch.zeros_like(self.k)
        self.page_table = torch.full((sequences, self.width), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self._free = list(range(pages - 1, -1, -1))
        self._pages: List[List[int]] = [[] for _ in range(sequences)]
        self._length = [0] * sequences
        self._freed = [(0, 0)] * sequences  # (all of a sequence's freed pages lie in [first, end))

    def _send(self, values, like: torch.Tensor) -> torch.Tensor:
        return torch.tensor(values, dtype=torch.int32).to(like.device)

    def grow(self, counts: Sequence[int]) -> torch.Tensor:
        """Room for counts[b] more tokens of each sequence; returns their slots (int32, those of sequence 0 first), for
        bsga_qk_norm_rope.  Raises without changing anything if the pages do not suffice."""
        if len(counts) != len(self._length) or min(counts) < 0:
            raise ValueError("counts must have one number >= 0 for each sequence")
        need = [-(-(n + c) // self.page) - len(p) for n, c, p in zip(self._length, counts, self._pages)]
        if sum(need) > len(self._free):
            raise RuntimeError(f"the cache has {len(self._free)} free pages, {sum(need)} needed")
        if any(len(p) + m > self.width for p, m in zip(self._pages, need)):
            raise RuntimeError(f"a sequence is longer than the table's {self.width} pages")
        slots: List[int] = []
        for b, c in enumerate(counts):
            if need[b] > 0:
                first = len(self._pages[b])
                self._pages[b] += [self._free.pop() for _ in range(need[b])]
                self.page_table[b, first:first + need[b]] = self._send(self._pages[b][first:], self.page_table)
            slots += [self._pages[b][i // self.page] * self.page + i % self.page for i in range(self._length[b], self._length[b] + c)]
            self._length[b] += c
        both = self._send(self._length + slots, self.lengths)  # (one way to the device for the two)
        lengths, slots = both.split((len(counts), len(slots)))
        self.lengths.copy_(lengths)
        return slots

    @contextmanager
    def growing(self, counts: Sequence[int]):
        """grow(), taken back if the body, which neither grows nor trims the cache itself, fails."""
        slots = self.grow(counts)
        try:
            yield slots
        except BaseException:
            emptied = []
            for b in range(len(counts) - 1, -1, -1):  # (pages go back in the order that hands them out again as before)
                self._length[b] -= counts[b]
                keep = -(-self._length[b] // self.page)
                if keep < len(self._pages[b]):
                    emptied.append((b, keep, len(self._pages[b])))
                    self._free += reversed(self._pages[b][keep:])
                    del self._pages[b][keep:]
            for b, first, end in emptied:
                self.page_table[b, first:end] = -1
            self.lengths.copy_(torch.tensor(self._length, dtype=torch.int32))
            raise

    def trim(self, window: Optional[int], sinks: int = 0, frame: int = 1) -> int:
        """Frees the pages that no later query sees (window = None: none); returns how many."""
        if (window is not None and window < 1) or sinks < 0 or frame < 1:
            raise ValueError(f"window must be at least one frame, or None, sinks >= 0 and frame >= 1, got {window}, {sinks} and {frame}")
        if window is None:
            return 0
        freed = 0
        for b, n in enumerate(self._length):
            if n == 0:
                continue
            lo = max(0, ((n - 1) // frame + 1 - window) * frame)
            gone = [i for i in range(-(-min(sinks, lo) // self.page), lo // self.page) if self._pages[b][i] >= 0]
            if not gone:
                continue
            for i in gone:
                self._free.append(self._pages[b][i])
                self._pages[b][i] = -1
            first, end = gone[0], gone[-1] + 1  # (what lies between them is freed)
            self.page_table[b, first:end] = -1
            before = self._freed[b]
            self._freed[b] = (first, end) if before[0] == before[1] else (min(first, before[0]), max(end, before[1]))
            freed += len(gone)
        return freed

    def check_seen(self, window: Optional[int], sinks: int = 0, frame: int = 1) -> None:
        """Raises if the next token of a sequence would see tokens whose pages trim() has freed."""
        for b, (first, end) in enumerate(self._freed):
            if first == end:
                continue
            lo = 0 if window is None else max(0, (self._length[b] // frame + 1 - window) * frame)
            kept, near = -(-min(sinks, lo) // self.page), lo // self.page  # pages [0, kept) and from `near` on are seen
            if any(self._pages[b][i] < 0 for part in (range(first, min(kept, end)), range(max(first, near), end)) for i in part):
                raise ValueError(f"sequence {b} of the cache: tokens that a window of {window} with {sinks} first tokens sees have been freed")


def _takes(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor) -> bool:
    """Whether a linear layer goes by bsga_linear: what that takes and gains by (GlobalAttentionBlock has the widths and what was measured), and
    where torch's operation would be no more than its result."""
    if type(x) is not torch.Tensor or torch.is_autocast_enabled() or _calls_are_watched():
        return False
    at = x.get_device()
    for t in (x, weight, bias):  # (a step of a few tokens is bound by the host: no more than is needed)
        if (t.dtype is not torch.bfloat16 or t.get_device() != at or at < 0 or not t.is_contiguous() or t.data_ptr() % 16
                or type(t) is not torch.nn.Parameter and type(t) is not torch.Tensor):
            return False
    shape, (rows, D) = x.shape, weight.shape
    N = shape[0]
    if len(shape) != 2 or N < 1 or shape[1] != D or (D > 1280 and (D > 2048 or N > 4096)):
        return False
    return max((N + 256) * D, (rows + 256) * D, N * rows) * 2 < 1 << 31


class StreamAttention(torch.nn.Module):
    """One attention layer of such a model: x [N, heads * 64] -> [N, heads * 64], `kv_heads` key heads, norms of queries and keys for each
    head (with `eps` beside the mean square or the variance), rotation by positions ([N] or [N, axes] int32; by default a token's place in the
    sequence), window of `window` frames of `frame` tokens and the first `sinks` tokens (see bsga_window_attn).

    forward(x) takes a whole sequence, with gradients; prefill(x, cache, b) the same for sequence b of an empty cache, and fills it;
    step(x, cache) one more token for every sequence of the cache.  With frame > 1 that is another function than forward() and prefill(), whose tokens
    see their whole frame: a token that comes alone sees its own frame up to itself, since the others are not there yet.  There is no way yet to
    take a whole new frame on a cache."""

    def __init__(self, heads: int = 16, kv_heads: Optional[int] = None, window: Optional[int] = None, sinks: int = 0, frame: int = 1,
                 norm: str = "rms", base: float = 10000.0, dtype=torch.bfloat16, device="cuda", seed: int = 0, eps: float = 1e-6):
        super().__init__()
        self.heads, self.kv_heads = heads, heads if kv_heads is None else kv_heads
        self.seen = dict(window=window, sinks=sinks, frame=frame)
        self.norm, self.base, self.eps = norm, base, eps
        d, rows = heads * 64, (heads + 2 * self.kv_heads) * 64
        g = torch.Generator(device="cpu").manual_seed(seed)

        def w(*shape, scale):
            return torch.nn.Parameter((torch.randn(*shape, generator=g) * scale).to(dtype).to(device))

        self.w_qkv, self.b_qkv = w(rows, d, scale=d ** -0.5), w(rows, scale=0.02)
        self.w_out, self.b_out = w(d, d, scale=d ** -0.5), w(d, scale=0.02)
        one = torch.ones(64, dtype=dtype, device=device)
        self.q_weight, self.k_weight = torch.nn.Parameter(one.clone()), torch.nn.Parameter(one.clone())
        bias = norm == "layer"
        self.q_bias = torch.nn.Parameter(torch.zeros_like(one)) if bias else None
        self.k_bias = torch.nn.Parameter(torch.zeros_like(one)) if bias else None

    def _split(self, qkv: torch.Tensor):
        H, K = self.heads, self.kv_heads
        qkv = qkv.view(qkv.shape[0], H + 2 * K, 64)
        return qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]

    def _places(self, n: int, device) -> torch.Tensor:
        return torch.arange(n, dtype=torch.int32, device=device)

    def forward(self, x: torch.Tensor, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        q, k, v = self._split(F.linear(x, self.w_qkv, self.b_qkv))
        positions = self._places(x.shape[0], x.device) if positions is None else positions
        q, k, v = qk_norm_rope(q, k, v, positions, self.q_weight, self.k_weight, self.q_bias, self.k_bias, norm=self.norm, eps=self.eps, base=self.base)
        o = window_attention(q, k, v, **self.seen)
        return F.linear(o.transpose(0, 1).reshape(x.shape[0], self.heads * 64), self.w_out, self.b_out)

    def _linear(self, x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor) -> torch.Tensor:
        return B.bsga_linear(x, weight, bias) if _takes(x, weight, bias) else F.linear(x, weight, bias)

    @torch.no_grad()
    def prefill(self, x: torch.Tensor, cache: PagedCache, b: int, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        if cache._length[b] != 0:
            raise ValueError(f"sequence {b} of the cache is not empty")
        N = x.shape[0]
        counts = [0] * len(cache._length)
        counts[b] = N
        with cache.growing(counts) as slots:
            q, k, v = self._split(self._linear(x, self.w_qkv, self.b_qkv))
            positions = self._places(N, x.device) if positions is None else positions
            q, k, v = B.bsga_qk_norm_rope(q, k, positions, self.q_weight, self.k_weight, self.q_bias, self.k_bias, v=v, norm=self.norm, eps=self.eps,
                                          base=self.base)
            # (what the attention reads in one piece goes into the pages as well; it is normed and turned already)
            B.bsga_qk_norm_rope(k.transpose(0, 1), k.transpose(0, 1), v=v.transpose(0, 1), norm=None, k_cache=cache.k, v_cache=cache.v, slots=slots)
            o = B.bsga_window_attn(q, k, v, **self.seen)
            return self._linear(B.bsga_merge_heads(o) if N > 0 else o.view(0, self.heads * 64), self.w_out, self.b_out)

    @torch.no_grad()
    def step(self, x: torch.Tensor, cache: PagedCache, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [sequences, heads * 64], one token for each sequence."""
        cache.check_seen(**self.seen)
        positions = cache.lengths.clone() if positions is None else positions
        with cache.growing([1] * x.shape[0]) as slots:
            q, k, v = self._split(self._linear(x, self.w_qkv, self.b_qkv))
            q, _, _ = B.bsga_qk_norm_rope(q, k, positions, self.q_weight, self.k_weight, self.q_bias, self.k_bias, v=v, norm=self.norm, eps=self.eps,
                                          base=self.base, k_cache=cache.k, v_cache=cache.v, slots=slots)
            o = B.bsga_paged_attn(q.transpose(0, 1), cache.k, cache.v, cache.page_table, cache.lengths, **self.seen)
            return self._linear(o.view(x.shape[0], -1), self.w_out, self.b_out)
