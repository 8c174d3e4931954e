"""A paged, quantised cache of attention keys and values: the buffers of one layer and the calls on them.

A token's head is a group of the codec (zero point and step in binary32, codes of 8 or 4 bits, rounded to nearest); token slot s is
offset s % page_size of page s // page_size.  Which pages belong to which sequence is the program's business: it hands over slots for
writing and reading, and a table of pages per sequence for the attention.
"""
from __future__ import annotations

import torch

from . import binding as B

__all__ = ["PagedCache"]


class PagedCache:
    """Keys and values of one layer: `pages` pages of `page_size` tokens (a power of two from 16 to 1024) of `heads` heads of `dim` = 64,
    128 or 256 elements."""

    def __init__(self, pages: int, page_size: int, heads: int, dim: int, key_bits: int = 8, value_bits: int = 8, device="cuda"):
        if key_bits not in (4, 8) or value_bits not in (4, 8):
            raise ValueError("key_bits and value_bits must be 4 or 8")
        self.pages, self.page_size, self.heads, self.dim = pages, page_size, heads, dim
        shape = (pages, heads, page_size)
        self.key_codes = torch.zeros((*shape, dim * key_bits // 8), dtype=torch.uint8, device=device)
        self.key_header = torch.zeros((*shape, 2), device=device)
        self.value_codes = torch.zeros((*shape, dim * value_bits // 8), dtype=torch.uint8, device=device)
        self.value_header = torch.zeros((*shape, 2), device=device)

    @property
    def buffers(self):
        """As the binding's calls take them."""
        return self.key_codes, self.key_header, self.value_codes, self.value_header

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self.buffers)

    def slots(self, table, sequence, position):
        """Slots (int64) of the tokens at `position` of the sequences `sequence` (int64 tensors of one shape) under a table of pages."""
        return table[sequence, position // self.page_size].long() * self.page_size + position % self.page_size

    def write(self, k, v, slots) -> None:
        """Quantises k and v [tokens, heads, dim] into the slots."""
        B.cache_write(k, v, slots, *self.buffers)

    def read(self, slots, dtype, k=None, v=None):
        """(keys, values) [tokens, heads, dim] of the slots."""
        return B.cache_read(slots, *self.buffers, self.dim, dtype, k, v)

    def attend(self, q, table, lengths, query_start, max_query: int, max_length: int, **options):
        """Attention of new tokens over the cached ones, their own among them (binding.cache_attention; options: scale, softcap, window, out)."""
        return B.cache_attention(q, *self.buffers, table, lengths, query_start, max_query, max_length, **options)
