"""A paged key/value cache that serves sequences from their prompt to their last token.

The prompt is attended by the prefill calls (rbs_select + rbs_sparse_prefill, or rbs_prefill_varlen for packed prompts), whose
queries and keys `write` norms and rotates on their way; every generated token by `attend`.  One block table serves all layers.
Arithmetic is entirely in the library's kernels; this module holds the tensors and hands them over.  `extend`, `write`, `attend` and `read`
wait for nothing on the host and update their tensors in place, so that a captured graph of a decode step can be replayed.
"""
from __future__ import annotations

import math

import torch

from .binding import (PagedStep, RbsError, _qk_norm_rope_write_int4, rbs_paged_decode, rbs_paged_decode_int4, rbs_paged_extend, rbs_paged_read_int4,
                      rbs_qk_norm_rope_paged)


def rope_frequencies(rot_dim: int, base: float, *, scaling: str | None = None, factor: float = 1.0, trained_len: int = 0, fast: float = 32.0,
                     slow: float = 1.0, device="cuda"):
    """(inv_freq [rot_dim / 2] fp32, magnitude) of rotary positions: pair i turns by position * base ** (-2 i / rot_dim).
    scaling, for contexts of `factor` times the trained length:
      None      none
      "linear"  every frequency divided by the factor
      "ntk"     the base raised by factor ** (rot_dim / (rot_dim - 2)): the slowest pair is slowed by the factor, the fastest not
      "yarn"    (Peng et al. 2023, "YaRN") pairs with more than `fast` turns over trained_len tokens as they are, with fewer than
                `slow` turns divided by the factor, a linear ramp over the pairs between; magnitude 0.1 ln(factor) + 1"""
    if rot_dim <= 0 or rot_dim % 8 != 0 or rot_dim > 128 or not base > 1.0 or not factor >= 1.0:
        raise RbsError("rope_frequencies: rot_dim must be a multiple of 8 up to 128, base above 1, factor at least 1")
    i = torch.arange(0, rot_dim, 2, dtype=torch.float64)
    magnitude = 1.0
    if scaling == "ntk":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    freq = base ** (-i / rot_dim)
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "yarn":
        if trained_len <= 0 or not fast > slow > 0.0:
            raise RbsError("rope_frequencies: yarn needs trained_len and fast > slow > 0")
        pair_of = lambda turns: rot_dim * math.log(trained_len / (2.0 * math.pi * turns)) / (2.0 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair_of(fast)), 0), min(math.ceil(pair_of(slow)), rot_dim - 1)
        ramp = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        freq = freq * (1.0 - ramp) + freq / factor * ramp
        magnitude = 0.1 * math.log(factor) + 1.0
    elif scaling not in (None, "ntk"):
        raise RbsError(f"rope_frequencies: unknown scaling {scaling!r}")
    return freq.to(torch.float32).to(device), magnitude


class PagedCache:
    """bits 16: k, v [layers, pages, page_size, kv_heads, d] bf16.  bits 4: k, v each a pair of uint8 tensors, codes [layers, pages, page_size,
    kv_heads, d / 2] and scales [layers, pages, page_size, kv_heads, d / 16] (pages of head rows, which attention reads fastest; see
    rbs_paged_write_int4).  block_table [seqs, max_pages], lens [seqs], used [1]: int32."""

    def __init__(self, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, n_seqs: int, max_pages: int, device, d: int = 128, bits: int = 16):
        if bits not in (4, 16):
            raise RbsError("PagedCache: bits must be 4 or 16")
        self.device = torch.device(device)
        self.page_size, self.n_pages, self.bits = page_size, n_pages, bits
        if bits == 16:
            self.k = torch.empty(n_layers, n_pages, page_size, n_kv_heads, d, dtype=torch.bfloat16, device=self.device)
            self.v = torch.empty_like(self.k)
        else:
            self.k, self.v = (tuple(torch.empty(n_layers, n_pages, n_kv_heads, page_size, width, dtype=torch.uint8, device=self.device).transpose(2, 3)
                                    for width in (d // 2, d // 16)) for _ in range(2))
        self.block_table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=self.device)
        self._state = torch.zeros(n_seqs + 1, dtype=torch.int32, device=self.device)
        self.lens, self.used = self._state[:n_seqs], self._state[n_seqs:]
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device=self.device)      # -1: no page

    def _layer(self, layer: int):
        """Keys and values of a layer, as the calls take them."""
        if self.bits == 16:
            return self.k[layer], self.v[layer]
        return (self.k[0][layer], self.k[1][layer]), (self.v[0][layer], self.v[1][layer])

    def extend(self, new_lens: torch.Tensor, n_tokens: int) -> PagedStep:
        """Room for new_lens[s] more tokens of each sequence, packed into n_tokens rows; their positions and slots.  Tokens count in lens
        whether or not there was a page for them: see short()."""
        n = self.lens.shape[0]
        state = torch.empty_like(self._state)
        out = PagedStep(state[:n], *(torch.empty(m, dtype=torch.int32, device=self.device) for m in (n + 1, n_tokens, n_tokens)), state[n:])
        rbs_paged_extend(self.lens, new_lens, self.block_table, self.free_pages, self.page_size, self.n_pages, n_tokens, free_used=self.used, out=out)
        self._state.copy_(state)
        return out

    def write(self, layer: int, Q, K, V, step: PagedStep, inv_freq, **turn):
        """Norms and rotates Q, K of the tokens of `step` and keeps K and V.  Returns Q'; out_k, if given, receives K' too.  Keywords as
        rbs_qk_norm_rope_paged."""
        call = rbs_qk_norm_rope_paged if self.bits == 16 else _qk_norm_rope_write_int4
        return call(Q, K, V, step.positions, step.slots, inv_freq, *self._layer(layer), **turn)

    def attend(self, layer: int, Q, **more):
        """Attention of one token per sequence, Q [seqs, heads, d], over all that its sequence holds.  Keywords as rbs_paged_decode."""
        call = rbs_paged_decode if self.bits == 16 else rbs_paged_decode_int4
        return call(Q, *self._layer(layer), self.block_table, self.lens, **more)

    def read(self, layer: int, n_rows: int, starts: torch.Tensor | None = None, **out):
        """What the sequences hold (from token starts[s] on) as packed bf16 rows for the prefill calls: K, V [n_rows, kv_heads, d] and the prefix
        sums cu [seqs + 1] of the sequences' rows.  Of a cache in 4 bits only: rows of one in 16 are in k and v as they are.  Keywords as
        rbs_paged_read_int4."""
        if self.bits != 4:
            raise RbsError("PagedCache.read: a cache in 16 bits holds its rows as they are")
        cu = torch.zeros(self.lens.shape[0] + 1, dtype=torch.int32, device=self.device)
        torch.cumsum(self.lens if starts is None else (self.lens - starts).clamp_(min=0), 0, dtype=torch.int32, out=cu[1:])
        return (*rbs_paged_read_int4(*self._layer(layer), self.block_table, cu, n_rows, starts=starts, **out), cu)

    def short(self) -> list[int]:
        """Sequences with tokens that got no page because the pool had run out.  Those tokens were not kept and `attend` leaves them out,
        however many pages become free later: such a sequence has to be released and begun again.  Waits for the device."""
        held = (self.lens.long() + self.page_size - 1) // self.page_size
        missing = (self.block_table < 0) & (torch.arange(self.block_table.shape[1], device=self.device) < held[:, None])
        return missing.any(1).nonzero()[:, 0].tolist()

    def release(self, seqs) -> list[int]:
        """Ends sequences (a list of their rows): their pages become free.  Between steps, on the host's time: waits for the device.
        Returns what short() says of the sequences that go on."""
        ended = sorted(set(int(s) for s in seqs))
        if not ended:
            return self.short()
        if ended[0] < 0 or ended[-1] >= self.lens.shape[0]:
            raise RbsError(f"PagedCache.release: sequences are 0 .. {self.lens.shape[0] - 1}")
        rows = torch.tensor(ended, dtype=torch.long, device=self.device)
        held = (self.lens[rows].long() + self.page_size - 1) // self.page_size
        index = torch.arange(self.block_table.shape[1], device=self.device)
        pages = self.block_table[rows][index < held[:, None]]
        left = self.free_pages[min(int(self.used), self.n_pages):]
        free = torch.cat((left[left >= 0], pages[pages >= 0]))
        self.free_pages.fill_(-1)
        self.free_pages[:free.numel()] = free
        self.block_table[rows] = -1
        self.lens[rows] = 0
        self.used.zero_()
        return self.short()
