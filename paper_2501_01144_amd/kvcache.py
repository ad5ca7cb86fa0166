"""Value cache with a high-precision residual chunk (paper, Appendix C).

Values are multiplied over the token axis (P V), so they are quantized along it:
the cache holds the quantized transpose V^T [head_dim, capacity] in blocks of 32
tokens.  A block can only be quantized when all its 32 tokens are known, and
requantizing it for every new token would repeat work and compound errors, so
the most recent, incomplete chunk (fewer than 32 tokens) stays in bf16 and is
quantized once, when it is full.  Keys are multiplied over the head dimension
and need no such care: each new key row is quantized on its own (dfp4.quantize).

Host-side bookkeeping only; the arithmetic is in the library's kernels
(dfp4_quantize_t_at).  Unwritten blocks of the cache are zero (code 0, exponent
byte 0), so a product over the whole capacity with zero-padded probabilities
equals the product over the tokens present.

PagedCache and PagedBatch are the same idea for many sequences, keys and values and all KV heads of a layer: the device memory of a
paged cache and the arrays that describe a batch, for dfp4.paged_write, dfp4.paged_read and dfp4.paged_attention.
"""
import ctypes

import torch

from . import dfp4

BLOCK = 32


class ValueCache:
    def __init__(self, head_dim, capacity_tokens, device):
        assert capacity_tokens % BLOCK == 0 and head_dim % 8 == 0
        self.head_dim, self.capacity = head_dim, capacity_tokens
        self.q = dfp4.QTensor(
            torch.zeros((head_dim, capacity_tokens // 2), dtype=torch.uint8, device=device),
            torch.zeros((head_dim, capacity_tokens // BLOCK), dtype=torch.uint8, device=device),
            torch.zeros((head_dim, capacity_tokens // BLOCK), dtype=torch.uint8, device=device),
            head_dim, capacity_tokens)
        self.residual = torch.zeros((BLOCK, head_dim), dtype=torch.bfloat16, device=device)
        self.n_quantized = 0           # tokens held in 4-bit form (a multiple of 32)
        self.n_residual = 0            # tokens held in bf16 (< 32)

    @property
    def n_tokens(self):
        return self.n_quantized + self.n_residual

    def append(self, v):
        """v: bf16 [t, head_dim], the values of t new tokens."""
        assert v.dtype == torch.bfloat16 and v.dim() == 2 and v.shape[1] == self.head_dim
        assert self.n_tokens + v.shape[0] <= self.capacity, "value cache full"
        pos = 0
        while pos < v.shape[0]:
            if self.n_residual == 0 and v.shape[0] - pos >= BLOCK:
                # whole chunks go straight to 4 bits
                rows = (v.shape[0] - pos) // BLOCK * BLOCK
                dfp4.quantize_t_at(v[pos:pos + rows].contiguous(), self.q, self.n_quantized)
                self.n_quantized += rows
                pos += rows
                continue
            take = min(BLOCK - self.n_residual, v.shape[0] - pos)
            self.residual[self.n_residual:self.n_residual + take] = v[pos:pos + take]
            self.n_residual += take
            pos += take
            if self.n_residual == BLOCK:
                dfp4.quantize_t_at(self.residual, self.q, self.n_quantized)
                self.n_quantized += BLOCK
                self.n_residual = 0

    def residual_values(self):
        """bf16 [n_residual, head_dim]: the tokens not yet quantized."""
        return self.residual[:self.n_residual]


class PagedCache:
    """Pages of `page_tokens` tokens (a multiple of 32) in 4 bits, and slots for the values of incomplete chunks of 32 tokens, which
    are bf16 until the chunk is whole: one slot for a sequence as long as it lives.  A slot also keeps the chunk before, so that a length may
    be taken back (drafted tokens that are not accepted) by up to SLOT_CHUNKS * 32 - 32 tokens from the largest that it has had: give the
    next batch the smaller length, the tokens after it are written again."""

    SLOT_CHUNKS = 2

    def __init__(self, n_pages, page_tokens, kv_heads, head_dim, n_slots, device):
        cell = dfp4.paged_cell_bytes(head_dim)
        assert cell > 0, "head_dim: 64, 96, 128, 192 or 256"
        assert page_tokens > 0 and page_tokens % BLOCK == 0 and kv_heads > 0 and n_pages >= 0 and n_slots >= 0
        self.n_pages, self.page_tokens, self.kv_heads, self.head_dim, self.n_slots = n_pages, page_tokens, kv_heads, head_dim, n_slots
        self.pages = torch.zeros((n_pages, kv_heads, page_tokens // BLOCK, cell), dtype=torch.uint8, device=device)
        self.residual = torch.zeros((n_slots, kv_heads, self.SLOT_CHUNKS, head_dim, BLOCK), dtype=torch.bfloat16, device=device)
        self.c = dfp4._CCache(self.pages.data_ptr() if n_pages else 0, self.residual.data_ptr() if n_slots else 0, n_pages, page_tokens,
                              n_slots, kv_heads, head_dim, self.SLOT_CHUNKS)
        self.at = ctypes.addressof(self.c)       # for the native module


class PagedBatch:
    """What a call has to know of its sequences (include/dfp4.h, dfp4_batch): int32 tensors on the device.

    cu_tokens [batch + 1]: sequence b brings rows cu_tokens[b] .. cu_tokens[b + 1] - 1; lengths [batch]: its tokens with these;
    table [batch, width]: its pages; slots [batch]: its slot.  max_new, max_length: bounds that the host knows, 0: none (they decide
    how work is split, not what is computed).  tokens: rows in all, where a call cannot take them from its arguments (paged_read);
    where it is not given it is read from cu_tokens whenever it is asked for, which waits for the device."""

    def __init__(self, cu_tokens, lengths, table, slots, max_new=0, max_length=0, tokens=None):
        n = lengths.numel()
        assert cu_tokens.numel() == n + 1 and slots.numel() == n and table.dim() == 2 and table.shape[0] == n
        for t in (cu_tokens, lengths, table, slots):
            assert t.dtype == torch.int32 and t.is_cuda and t.is_contiguous()
        self.cu_tokens, self.lengths, self.table, self.slots = cu_tokens, lengths, table, slots     # (their contents may change, they not)
        self.max_new, self.max_length, self._tokens = max_new, max_length, tokens
        self._c = dfp4._CBatch(cu_tokens.data_ptr(), lengths.data_ptr(), table.data_ptr(), slots.data_ptr(), n, table.shape[1], 0, max_new, max_length)
        self.at = ctypes.addressof(self._c)      # for the native module, which fills in the rows

    @property
    def tokens(self):
        # (the contents of cu_tokens may change: nothing is kept)
        return int(self.cu_tokens[-1]) if self._tokens is None else self._tokens

    def c(self, tokens):
        b = dfp4._CBatch.from_buffer_copy(self._c)
        b.tokens = tokens
        return b
