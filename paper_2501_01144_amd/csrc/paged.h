// The paged 4-bit cache: where a cell keeps what, and what a kernel knows of a batch.
//
// A cell holds 32 tokens of one KV head.  Its parts lie as the attention kernel's lanes read them (lane = 16 g + c).
//   K codes  [token][unit of 16 elements, 8 bytes].  Of 128 elements lane (g, c) takes half g % 2 of blocks g / 2 and 2 + g / 2 (a product adds
//            over them in any order).  Where 128 are whole, both halves of a lane lie together (k_unit), so that it loads 16 bytes
//   V codes  [d][dword of 8 tokens]: a lane takes the 32 tokens of a d
//   K exps   [token % 4][block][token / 4]: a lane takes the 8 tokens 4 t + i of a block, t = 0 .. 7
//   K ids    [token % 4][pair][token / 4]: dialects of blocks p and p + 2 of a 128 in one byte
//   V exps   [d % 16][d / 16]       V ids  [d % 16 / 2][d / 16]: dialects of d (even) and d + 1
// A code dword holds element j in the low nibble of byte j and element 4 + j in its high nibble, so that two table look-ups give
// the bytes in order.
#pragma once
#include "common.h"
#include "formatbook.h"
#include "page_of.h"

namespace dfp4 {

template <int D>
struct Cell {
    static constexpr int NB = D / 32;                    // blocks of a key
    static constexpr int KT = (NB + 3) / 4;              // 128 elements of a key
    static constexpr int NJ = D / 16;                    // 16-row tiles of V^T
    static constexpr int VE = (NJ + 3) / 4 * 4;          // bytes of a row of V exps
    static constexpr int NP = 2 * KT;                    // dialect bytes of a key
    // all of a cell's keys, then all of its values: each is loaded to LDS as it lies
    static constexpr uint32_t kKExps = 16 * D, kKIds = kKExps + 32 * NB, kKeys = kKIds + 32 * NP, kVCodes = kKeys, kVExps = kVCodes + 16 * D,
                              kVIds = kVExps + 16 * VE, kValues = kVIds + 8 * VE - kVCodes, kBytes = (kKeys + kValues + 63) / 64 * 64;
    // blocks of the kt-th 128
    static constexpr int blocks(int kt) { return NB - 4 * kt < 4 ? NB - 4 * kt : 4; }
    // place (in units of 8 bytes) of elements 16 u .. 16 u + 15 of a key
    static __host__ __device__ constexpr int k_unit(int u) {
        return blocks(u / 8) == 4 ? u / 8 * 8 + u % 4 * 2 + u % 8 / 4 : u;
    }
};

// the same for a head dimension known at run time; 0 if it is not supported
inline uint32_t cell_bytes(int64_t D) {
    return D == 64 ? Cell<64>::kBytes : D == 96 ? Cell<96>::kBytes : D == 128 ? Cell<128>::kBytes : D == 192 ? Cell<192>::kBytes
         : D == 256 ? Cell<256>::kBytes : 0;
}
template <class F>
inline void with_head_dim(int64_t D, F&& f) {
    if (D == 64) f(std::integral_constant<int, 64>{});
    else if (D == 96) f(std::integral_constant<int, 96>{});
    else if (D == 128) f(std::integral_constant<int, 128>{});
    else if (D == 192) f(std::integral_constant<int, 192>{});
    else f(std::integral_constant<int, 256>{});
}

struct PagedArgs {
    uint8_t* pages;
    uint16_t* residual;
    const int32_t *cu, *lengths, *table, *slots;
    int n_pages, n_slots, slot_chunks, page_chunks, kv_heads, batch, width, tokens;
    PageDivision pages_of;           // by page_chunks
};

inline PagedArgs paged_args(const dfp4_cache& c, const dfp4_batch& b) {
    return PagedArgs{c.pages, c.residual, b.cu_tokens, b.lengths, b.table, b.slots, (int)c.n_pages, (int)c.n_slots, c.slot_chunks == 2 ? 2 : 1,
                     (int)(c.page_tokens / 32), (int)c.kv_heads, (int)b.batch, (int)b.table_width, (int)b.tokens,
                     page_division((uint32_t)(c.page_tokens / 32))};
}

// New tokens of the sequence with most, or, where the caller does not know, of one with as many as the others: 48 sequences with one token
// each, 32 heads of 128 on 8, 8192 keys: attention 100 us, taken for one sequence's 48 tokens 250 (256 rows a workgroup).
inline int64_t likely_new(const dfp4_batch& b) {
    if (b.max_new == 0) return (b.tokens + b.batch - 1) / b.batch;
    return b.max_new < b.tokens ? b.max_new : b.tokens;
}

// New tokens [first, first + n) of the dense arrays are positions [length - n, length) of the sequence.
struct Sequence {
    int first, n, length, slot;      // slot -1: none
};

__device__ __forceinline__ Sequence sequence(const PagedArgs& p, int b) {
    const int t0 = min(max(p.cu[b], 0), p.tokens), t1 = min(max(p.cu[b + 1], t0), p.tokens);
    const int64_t most = (int64_t)p.width * p.page_chunks * 32;
    const int slot = p.slots[b];
    return Sequence{t0, t1 - t0, (int)min((int64_t)max(p.lengths[b], 0), most), slot >= 0 && slot < p.n_slots ? slot : -1};
}

// Where the cell of a chunk of 32 tokens lies in the pool, given its page's number in the table; -1 where that is none of the pool's.
// (The pool has fewer than 2^31 cells.)
__device__ __forceinline__ uint32_t cell_number(const PagedArgs& p, int head, int chunk, int in_table, int page) {
    return ((uint32_t)page * (uint32_t)p.kv_heads + (uint32_t)head) * (uint32_t)p.page_chunks + (uint32_t)(chunk - in_table * p.page_chunks);
}
template <int D>
__device__ __forceinline__ int64_t cell_offset(const PagedArgs& p, int head, int chunk, int in_table, int page) {
    const bool there = (uint32_t)page < (uint32_t)p.n_pages;
    const int64_t at = (int64_t)((uint64_t)cell_number(p, head, chunk, in_table, there ? page : 0) * Cell<D>::kBytes);
    return there ? at : (int64_t)-1;
}
__device__ __forceinline__ int place_in_table(const PagedArgs& p, int chunk) { return page_of(p.pages_of, chunk); }

// the cell of a chunk that the length says is there
template <int D>
__device__ __forceinline__ uint8_t* cell(const PagedArgs& p, int b, int head, int chunk) {
    const int in_table = place_in_table(p, chunk);
    const int64_t at = cell_offset<D>(p, head, chunk, in_table, p.table[(int64_t)b * p.width + in_table]);
    return at < 0 ? nullptr : p.pages + at;
}

// The cells of four consecutive chunks, of those below `limit` (which the length says are there).  The numbers of their pages are
// loaded a step ahead, so that the addresses need not wait for the table: by lanes 0 .. 3, or as scalars.
__device__ __forceinline__ int four_pages(const PagedArgs& p, int b, int chunk0, int limit) {
    const int chunk = min(chunk0 + (int)(threadIdx.x & 3u), limit - 1);
    return p.table[(int64_t)b * p.width + place_in_table(p, max(chunk, 0))];
}
struct Four {
    int64_t c0, c1, c2, c3;
    __device__ __forceinline__ uint32_t there() const {             // bit k: chunk k
        return (c0 >= 0 ? 1u : 0u) | (c1 >= 0 ? 2u : 0u) | (c2 >= 0 ? 4u : 0u) | (c3 >= 0 ? 8u : 0u);
    }
};
// The same with the pages' numbers in scalar registers, for addresses that are wave-uniform.
struct FourPages { int n0, n1, n2, n3; };
__device__ __forceinline__ FourPages four_pages_uniform(const PagedArgs& p, int b, int chunk0, int limit) {
    // (constant memory for the time of the kernel: scalar loads, which wait for nothing that goes to vector registers or LDS)
    typedef const __attribute__((address_space(4))) int32_t* Table;
    const Table row = (Table)(uintptr_t)(p.table + (int64_t)b * p.width);
    auto one = [&](int k) { return row[place_in_table(p, max(min(chunk0 + k, limit - 1), 0))]; };
    return FourPages{one(0), one(1), one(2), one(3)};
}
template <int D>
__device__ __forceinline__ Four four_cells(const PagedArgs& p, int head, int chunk0, int limit, const FourPages& pages) {
    auto one = [&](int k, int page) {
        const int chunk = chunk0 + k;
        const int64_t to = cell_offset<D>(p, head, chunk, place_in_table(p, chunk), page);
        return chunk < limit ? to : (int64_t)-1;
    };
    return Four{one(0, pages.n0), one(1, pages.n1), one(2, pages.n2), one(3, pages.n3)};
}

// a chunk's bf16 [head_dim, 32] in a slot: chunks take its places in turn
template <int D>
__device__ __forceinline__ uint16_t* residual(const PagedArgs& p, int slot, int head, int chunk) {
    return p.residual + (((int64_t)slot * p.kv_heads + head) * p.slot_chunks + (chunk & (p.slot_chunks - 1))) * (D * 32);
}

int launch_paged_write(const void* k, int64_t ks, int64_t khs, const void* v, int64_t vs, int64_t vhs, const dfp4_cache& cache,
                       const dfp4_batch& batch, hipStream_t stream);
int launch_paged_read(const dfp4_cache& cache, const dfp4_batch& batch, void* k, void* v, int dtype, hipStream_t stream);

struct AttentionArgs {
    PagedArgs paged;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    const float* slopes;
    float* partial;                  // [tokens, heads, splits, head_dim], then [tokens, heads, splits, 2]
    int64_t q_stride, q_head_stride, out_stride, out_head_stride;
    float scale, softcap;
    int heads, window, splits, split_steps;
    int rows;                        // query rows of a workgroup
};
size_t paged_attention_workspace_bytes(const dfp4_cache& cache, const dfp4_batch& batch, int64_t heads, int64_t window);
int paged_attention_rows(const dfp4_cache& cache, const dfp4_batch& batch, int64_t heads, int64_t window);
int launch_paged_attention(AttentionArgs a, const dfp4_cache& cache, const dfp4_batch& batch, hipStream_t stream);

struct NormRopeArgs {
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    const float *q_weight, *k_weight, *inv_freq;
    const int32_t* positions;
    int64_t q_stride, q_head_stride, k_stride, k_head_stride;
    int heads, kv_heads, tokens, head_dim, rotary, interleaved;
    float eps;
};
int launch_norm_rope(const NormRopeArgs& a, hipStream_t stream);

}  // namespace dfp4
