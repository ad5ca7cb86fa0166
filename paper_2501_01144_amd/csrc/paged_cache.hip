// The paged 4-bit cache written and read back (paper, Appendix C: keys quantized along the head dimension as they come, values
// along the tokens, 32 at a time; values of the incomplete chunk stay bf16).  The per-block arithmetic is that of the other
// quantizers (quant_pass.h), the layout of a cell is in paged.h.
// Bound by memory where there is much of it: 4 x 4096 tokens, 8 heads of 128: write 23 us (86 MB, 3.7 TB/s), read 17 us (5.0 TB/s), in
// f32 28 (5.5).  One token of 64 sequences: write 6 us, read 5, most of it the dependent loads (batch, table, rows) and the launch.
#include <type_traits>

#include "paged.h"
#include "quant_pass.h"

namespace dfp4 {

namespace {

constexpr int kThreads = 256;

struct WriteArgs {
    PagedArgs paged;
    const uint16_t *k, *v;
    int64_t k_stride, k_head_stride, v_stride, v_head_stride;
};

// eight nibbles (element j in bits 4 j) to the cell's order (element j in the low nibble of byte j, 4 + j in the high one), and back
__device__ __forceinline__ uint32_t spread(uint32_t x) {           // four nibbles to the low nibbles of four bytes
    x = (x | (x << 8)) & 0x00ff00ffu;
    return (x | (x << 4)) & 0x0f0f0f0fu;
}
__device__ __forceinline__ uint32_t to_cell(uint32_t c) { return spread(c & 0xffffu) | (spread(c >> 16) << 4); }

// place of a token's key scales and dialects among those of its chunk (`per_key` blocks or pairs of a key)
__device__ __forceinline__ uint32_t key_meta(uint32_t token, uint32_t per_key, uint32_t i) { return ((token & 3u) * per_key + i) * 8u + (token >> 2); }

// lane `lane`'s neighbour four lanes on (all lanes active)
__device__ __forceinline__ uint32_t next_quad(uint32_t v) { return (uint32_t)__shfl_xor((int)v, 4); }
__device__ __forceinline__ uint32_t quad_after(uint32_t v, uint32_t lanes) { return (uint32_t)__shfl_down((int)v, lanes); }

// One workgroup: one KV head's share of one chunk of 32 positions of one sequence.  The values of the last chunks also go to the slot (two:
// so many that the length may be taken back by 32 tokens; one: the incomplete chunk's), by their own workgroup, except where the
// first touched chunk's older values still lie in the same place: that chunk's workgroup does it then, after it has read them.
// A key's block is a quad of lanes; lanes of a token are a power of two, so that blocks p and p + 2, whose dialects share a byte,
// are in one wave.  A chunk of values is turned through LDS.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_write_kernel(WriteArgs a) {
    using C = Cell<D>;
    constexpr uint32_t kLanes = D <= 64 ? 8 : D <= 128 ? 16 : 32;   // of a token
    constexpr uint32_t kPitch = D + 2;
    __shared__ __attribute__((aligned(16))) uint8_t lds_i[kDialects * 32];
    __shared__ __attribute__((aligned(16))) uint8_t lds_v[kPairs * 32];
    __shared__ __attribute__((aligned(4))) uint16_t s_v[32 * kPitch];
    const uint32_t tid = threadIdx.x, sub = tid & 3u;
    const int b = (int)(blockIdx.x / (uint32_t)a.paged.kv_heads), head = (int)(blockIdx.x % (uint32_t)a.paged.kv_heads);
    const Sequence s = sequence(a.paged, b);
    const int start = s.length - s.n, from = max(start, 0);          // positions from .. length - 1 are written
    const int first = from / 32, last = (s.length - 1) / 32;         // touched chunks
    if (from >= s.length || first + (int)blockIdx.y > last) return;
    if (tid < 32) reinterpret_cast<uint4*>(lds_i)[tid] = reinterpret_cast<const uint4*>(g_quant_tables.near_i)[tid];
    else if (tid < 48) reinterpret_cast<uint4*>(lds_v)[tid - 32] = reinterpret_cast<const uint4*>(g_quant_tables.vote1)[tid - 32];
    const uint16_t* kh = a.k + head * a.k_head_stride;
    const uint16_t* vh = a.v + head * a.v_head_stride;
    auto row = [&](int position) { return (int64_t)(s.first + position - start); };          // of the dense arrays
    const int places = a.paged.slot_chunks, first_kept = s.slot < 0 ? last + 1 : places > 1 ? max(s.length - 32, 0) / 32 : s.length / 32;
    auto first_stores = [&](int chunk) { return chunk >= first_kept && chunk > first && (from & 31) != 0 && (chunk - first) % places == 0; };

    for (int chunk = first + (int)blockIdx.y; chunk <= last; chunk += (int)gridDim.y) {
        uint8_t* const at = cell<D>(a.paged, b, head, chunk);
        const int lo = max(from, chunk * 32), hi = min(s.length, chunk * 32 + 32);
        const bool whole = hi == chunk * 32 + 32, in_slot = chunk >= first_kept && !first_stores(chunk);
        __syncthreads();                                             // tables; s_v of the chunk before
        if (whole) {
            const int old = lo - chunk * 32;                         // values that the slot holds (the first chunk's)
            for (uint32_t i = tid; i < (uint32_t)(hi - lo) * (D / 8); i += kThreads) {
                const uint32_t t = i / (D / 8), d = i % (D / 8) * 8u;
                const uint4 x = *reinterpret_cast<const uint4*>(vh + row(lo + (int)t) * a.v_stride + d);
                uint32_t* dst = reinterpret_cast<uint32_t*>(&s_v[(old + t) * kPitch + d]);
                dst[0] = x.x; dst[1] = x.y; dst[2] = x.z; dst[3] = x.w;
            }
            if (old > 0) {
                const uint16_t* r = s.slot >= 0 ? residual<D>(a.paged, s.slot, head, chunk) : nullptr;
                for (uint32_t i = tid; i < D * 4u; i += kThreads) {  // eight tokens of a d
                    const uint32_t d = i >> 2, t = (i & 3u) * 8u;
                    if ((int)t >= old) continue;
                    const uint4 x = r ? *reinterpret_cast<const uint4*>(r + d * 32u + t) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if ((int)t + j < old) s_v[(t + j) * kPitch + d] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                }
            }
        }
        // keys (the loop runs the same number of times in every lane: neighbours exchange)
        for (uint32_t base = 0; base < (uint32_t)(hi - lo) * kLanes; base += kThreads) {
            const uint32_t t = (base + tid) / kLanes, dd = (base + tid) % kLanes, block = dd >> 2;
            const bool on = t < (uint32_t)(hi - lo) && dd < D / 8;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (on) x = *reinterpret_cast<const uint4*>(kh + row(lo + (int)t) * a.k_stride + dd * 8u);
            uint32_t code, ebyte, dial;
            dfp4_pass_small(x, lds_v, lds_i, code, ebyte, dial);
            const uint32_t above = quad_after(dial, 8);              // block + 2's
            if (on && at) {
                const uint32_t token = (uint32_t)(lo - chunk * 32) + t;
                const uint32_t unit = (uint32_t)C::k_unit((int)(dd >> 1));
                *reinterpret_cast<uint32_t*>(at + token * (D / 2) + unit * 8u + (dd & 1u) * 4u) = to_cell(code);
                if (sub == 0) {
                    at[C::kKExps + key_meta(token, C::NB, block)] = (uint8_t)ebyte;
                    const uint32_t in = block & 3u;
                    if (in < 2)
                        at[C::kKIds + key_meta(token, C::NP, (block >> 2) * 2u + in)] =
                            (uint8_t)(dial | (block + 2u < (uint32_t)C::NB ? above << 4 : 0u));
                }
            }
        }
        __syncthreads();
        if (whole) {
            for (uint32_t i = tid; i < D * 4u; i += kThreads) {      // D * 4 is a multiple of the 256 threads
                const uint32_t d = i >> 2;
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = (uint32_t)s_v[(sub * 8u + 2 * j) * kPitch + d] | ((uint32_t)s_v[(sub * 8u + 2 * j + 1) * kPitch + d] << 16);
                if (in_slot) *reinterpret_cast<uint4*>(residual<D>(a.paged, s.slot, head, chunk) + i * 8u) = make_uint4(w[0], w[1], w[2], w[3]);
                uint32_t code, ebyte, dial;
                dfp4_pass_small(make_uint4(w[0], w[1], w[2], w[3]), lds_v, lds_i, code, ebyte, dial);
                const uint32_t beside = next_quad(dial);             // d ^ 1's
                if (at) {
                    *reinterpret_cast<uint32_t*>(at + C::kVCodes + d * 16u + sub * 4u) = to_cell(code);
                    if (sub == 0) {
                        at[C::kVExps + (d & 15u) * C::VE + (d >> 4)] = (uint8_t)ebyte;
                        if (!(d & 1u)) at[C::kVIds + ((d & 15u) >> 1) * C::VE + (d >> 4)] = (uint8_t)(dial | (beside << 4));
                    }
                }
            }
        }
        // (16 bytes of a whole chunk's values went to the slot from the registers above)
        for (int c = max(chunk, first_kept); c <= last; ++c) {
            if (!(c == chunk ? in_slot && !whole : chunk == first && first_stores(c))) continue;
            uint16_t* r = residual<D>(a.paged, s.slot, head, c);
            const int t0 = max(from, c * 32), n = min(s.length, c * 32 + 32) - t0;
            for (uint32_t i = tid; i < (uint32_t)n * D; i += kThreads) {
                const uint32_t t = i / D, d = i % D;
                r[d * 32u + ((uint32_t)(t0 & 31) + t)] = vh[row(t0 + (int)t) * a.v_stride + d];
            }
        }
    }
}

struct ReadArgs {
    PagedArgs paged;
    void *k, *v;
};

__device__ __forceinline__ void store8(float* y, const float (&v)[8]) {
    reinterpret_cast<float4*>(y)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(y)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t* y, const float (&v)[8]) {      // exact: the values have few bits
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (as_u(v[2 * j]) >> 16) | (as_u(v[2 * j + 1]) & 0xffff0000u);
    *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
}

// the eight values of a code dword in the cell's order
__device__ __forceinline__ void expand8(uint32_t c, const uint2 row, uint32_t ebyte, float (&v)[8]) {
    const uint32_t lo = __builtin_amdgcn_perm(row.y, row.x, c & 0x07070707u), hi = __builtin_amdgcn_perm(row.y, row.x, (c >> 4) & 0x07070707u);
    const int e = (int)ebyte - 128;                                  // 0.5 u 2^(byte - 127)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = as_f(as_u(ldexpf((float)((lo >> (8 * j)) & 0xffu), e)) | ((c << (28 - 8 * j)) & 0x80000000u));
        v[4 + j] = as_f(as_u(ldexpf((float)((hi >> (8 * j)) & 0xffu), e)) | ((c << (24 - 8 * j)) & 0x80000000u));
    }
}

// One workgroup as in paged_write_kernel; values are turned through LDS (as bf16: exact).
template <int D, class T>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(ReadArgs a) {
    using C = Cell<D>;
    constexpr uint32_t kPitch = D + 8;                               // rows of 16-byte pieces
    __shared__ __attribute__((aligned(16))) uint8_t s_book[kDialects * 8];
    __shared__ __attribute__((aligned(16))) uint16_t s_v[32 * kPitch];
    const uint32_t tid = threadIdx.x;
    const int b = (int)(blockIdx.x / (uint32_t)a.paged.kv_heads), head = (int)(blockIdx.x % (uint32_t)a.paged.kv_heads);
    const Sequence s = sequence(a.paged, b);
    if (s.n == 0) return;
    // chunks of positions -32 .. -1 too: tokens before position 0 are read as zeros
    const int start = s.length - s.n, first = start >= 0 ? start / 32 : -((31 - start) / 32), last = s.length > 0 ? (s.length - 1) / 32 : -1;
    if (tid < kDialects * 8) s_book[tid] = kBook[tid / 8][tid % 8];
    const uint2* const book = reinterpret_cast<const uint2*>(s_book);
    for (int chunk = first + (int)blockIdx.y; chunk <= last; chunk += (int)gridDim.y) {
        const uint8_t* const at = chunk >= 0 ? cell<D>(a.paged, b, head, chunk) : nullptr;
        const int lo = max(start, chunk * 32), hi = min(s.length, chunk * 32 + 32);
        const uint32_t n = (uint32_t)(hi - lo), t0 = (uint32_t)(lo - chunk * 32);
        const bool whole = hi == chunk * 32 + 32;
        __syncthreads();
        for (uint32_t i = tid; i < D * 4u; i += kThreads) {
            const uint32_t d = i >> 2, sub = i & 3u;
            uint16_t x[8];
            if (whole) {
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (at) {
                    const uint32_t dial = (at[C::kVIds + ((d & 15u) >> 1) * C::VE + (d >> 4)] >> (4u * (d & 1u))) & 15u;
                    expand8(*reinterpret_cast<const uint32_t*>(at + C::kVCodes + d * 16u + sub * 4u), book[dial],
                            at[C::kVExps + (d & 15u) * C::VE + (d >> 4)], v);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (uint16_t)(as_u(v[j]) >> 16);
            } else {
                const bool there = at && s.slot >= 0;
                const uint4 w = there ? *reinterpret_cast<const uint4*>(residual<D>(a.paged, s.slot, head, chunk) + d * 32u + sub * 8u) : make_uint4(0, 0, 0, 0);
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (uint16_t)(u[j / 2] >> (16 * (j & 1)));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s_v[(sub * 8u + j) * kPitch + d] = x[j];
        }
        __syncthreads();
        for (uint32_t i = tid; i < n * (D / 8); i += kThreads) {
            const uint32_t t = i / (D / 8), dd = i % (D / 8), token = t0 + t;
            const int64_t to = ((int64_t)(s.first + lo - start + (int)t) * a.paged.kv_heads + head) * D + dd * 8u;
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (at) {
                const uint32_t block = dd >> 2, in = block & 3u;
                const uint32_t ids = at[C::kKIds + key_meta(token, C::NP, (block >> 2) * 2u + (in & 1u))];
                expand8(*reinterpret_cast<const uint32_t*>(at + token * (D / 2) + (uint32_t)C::k_unit((int)(dd >> 1)) * 8u + (dd & 1u) * 4u),
                        book[(ids >> (in & 2u ? 4u : 0u)) & 15u], at[C::kKExps + key_meta(token, C::NB, block)], v);
            }
            store8(static_cast<T*>(a.k) + to, v);
            const uint4 w = *reinterpret_cast<const uint4*>(&s_v[token * kPitch + dd * 8u]);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = as_f((u[j / 2] >> (16 * (j & 1))) << 16);
            store8(static_cast<T*>(a.v) + to, v);
        }
    }
}

// Workgroups along the chunks of 32 positions that the new tokens of a sequence touch.  Where the caller does not know how many that is at
// most, one sequence may have most of them: then for as many as it could have, but for no more than 16384 in all, of which those without a
// chunk cost 0.3 ns each (one token of 1000 sequences: 22 us, with workgroups for 1000 tokens of each 104).
uint32_t chunk_groups(const dfp4_cache& c, const dfp4_batch& b) {
    int64_t chunks = (likely_new(b) + 62) / 32;
    if (b.max_new == 0) {
        const int64_t could = (b.tokens + 62) / 32, cheap = 16384 / (b.batch * c.kv_heads), more = could < cheap ? could : cheap;
        if (more > chunks) chunks = more;
    }
    return (uint32_t)(chunks < 65535 ? chunks : 65535);
}

}  // namespace

int launch_paged_write(const void* k, int64_t ks, int64_t khs, const void* v, int64_t vs, int64_t vhs, const dfp4_cache& cache,
                       const dfp4_batch& batch, hipStream_t stream) {
    const WriteArgs a{paged_args(cache, batch), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), ks, khs, vs, vhs};
    const dim3 grid((uint32_t)(batch.batch * cache.kv_heads), chunk_groups(cache, batch));
    with_head_dim(cache.head_dim, [&](auto d) {
        hipLaunchKernelGGL((paged_write_kernel<decltype(d)::value>), grid, dim3(kThreads), 0, stream, a);
    });
    return check_launch();
}

int launch_paged_read(const dfp4_cache& cache, const dfp4_batch& batch, void* k, void* v, int dtype, hipStream_t stream) {
    const ReadArgs a{paged_args(cache, batch), k, v};
    const dim3 grid((uint32_t)(batch.batch * cache.kv_heads), chunk_groups(cache, batch));
    with_head_dim(cache.head_dim, [&](auto d) {
        constexpr int kD = decltype(d)::value;
        if (dtype == DFP4_BF16) hipLaunchKernelGGL((paged_read_kernel<kD, uint16_t>), grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((paged_read_kernel<kD, float>), grid, dim3(kThreads), 0, stream, a);
    });
    return check_launch();
}

}  // namespace dfp4
