// Products of a sparse layer's experts on the block-scaled matrix instruction (include/dfp4.h; operand layout: fp6_pack.h, gemm_native.hip).
//
// Rows (pairs of a token and an expert) come in the plan's order.  Three ways, by how many an expert has (rules at kFewRows, token_by_token):
//   many   rows are quantized to FP6 in operand order, an expert's from a group of kGroupRows on, so that every tile has one expert
//          (experts_quantize_kernel, experts_gather_kernel), and the large block-scaled kernel takes tiles of 256 or 128 of them with the
//          weights' FP6 form (gemm_native.hip, kExperts, kGated).  Bound by the tiles' operands on their way to the compute units and by what
//          stands before and after a tile's loop (the matrix instructions are busy 32 % of the time up), down by what leaves and is added too
//          (4096 tokens of 8 of 64 experts x 2048: 268 MB; the product 103 us, matrix instructions busy 16 %, the sums 50 us, 5.7 TB/s).
//   few    experts_few_kernel streams the weights' 4-bit form past rows that lie in LDS.  Bound by that stream.
//   a few tokens, down   experts_token_kernel, one launch.
// The weights' two forms cost memory (0.79 + 0.56 bytes an element) and spare either way a pass over them.
// Gate and up rows take turns in both: a lane then holds both numbers that an element of h is made of (few: weights are the instruction's
// first operand, rows its second).  Down, rows leave weighted by nothing, in fp32, and experts_join_kernel adds a token's in their order: no sum
// depends on when a workgroup runs, and y is rounded once, whatever way its rows took.  (Rows in bf16 are half of what is moved there, but
// where a token's experts cancel, their roundings are more than all of y: of 8 normal rows, weights of one sign, 1 % of y is off by 33 half steps.)
#include <math.h>
#include <type_traits>
#include "experts.h"
#include "fp6_pack.h"
#include "quant_pass.h"

namespace dfp4 {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

inline int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }
inline int64_t steps_of(int64_t K) { return (K / kBlock + 1) / 2; }

// rows of an expert's matrix in the packed form (gate and up take turns), and those padded to 256
inline int64_t expert_rows(const dfp4_experts& w) { return w.gated ? 2 * w.rows : w.rows; }
inline int64_t padded_rows(const dfp4_experts& w) { return up256(expert_rows(w)); }

struct Packed {
    uint8_t* bits;
    uint8_t* scales;
};
inline Packed packed_at(void* p, int64_t rows, int64_t K) {
    uint8_t* at = static_cast<uint8_t*>(p);
    return Packed{at, at + native_scale_offset(rows, K, true)};
}
__device__ __forceinline__ size_t scale_at(size_t tile, size_t step, size_t S) { return ((tile >> 2) * S + step) * 256 + (tile & 3); }

// ---- weights

// The 4-bit form for products of few rows: a quad of blocks (128 elements) of a tile of 32 packed rows is 64 lanes x 16 bytes of codes for each
// of two steps, then 64 dwords: exponent bytes of the steps, dialects of the four blocks.  Lane (h, r) has half h of both of a step's blocks
// of row r, and the exponents of block h (the order of the instruction's FP8 operands).
constexpr int kQuadBytes = 2304;
inline int64_t quads_of(int64_t K) { return (K / kBlock + 3) / 4; }
inline int64_t row_tiles(const dfp4_experts& w) { return (expert_rows(w) + 31) / 32; }

struct PackArgs {
    const uint8_t *codes[2], *dial[2], *expo[2];
    Packed to;
    uint8_t* quads;
    int rows, KB, S, gated, tiles, Q;            // tiles of 32 packed rows of an expert in `quads`, quads of blocks
};

// One wave per (tile, step); lane (kh, c) takes row c of the tile, block 2 step + kh.  What is not there is zeros.  The 4-bit form of the same:
// half kh of both blocks of a step.
__global__ __launch_bounds__(256) void experts_pack_kernel(PackArgs p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kh = lane >> 5, c = lane & 31;
    const int s = blockIdx.x * 4 + wave;
    if (s >= p.S) return;
    const int64_t expert = blockIdx.z, tile = expert * gridDim.y + blockIdx.y;
    const int at = (int)blockIdx.y * 32 + c, kb = 2 * s + kh;
    const int row = p.gated ? at >> 1 : at, which = p.gated ? at & 1 : 0;
    uint4 codes = make_uint4(0, 0, 0, 0);
    uint32_t eb = 0, dl = 7;
    if (row < p.rows && kb < p.KB) {
        const int64_t blk = (expert * p.rows + row) * p.KB + kb;
        __builtin_memcpy(&codes, (which ? p.codes[1] : p.codes[0]) + blk * 16, 16);
        eb = (which ? p.expo[1] : p.expo[0])[blk];
        dl = (which ? p.dial[1] : p.dial[0])[blk] & 15u;
    }
    const Fp6Lane v = pack6_lane(codes, g_fp6_book.w[dl][0], g_fp6_book.w[dl][1]);
    *reinterpret_cast<uint4*>(p.to.bits + fp6_lo(tile, s, p.S) + lane * 16) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    *reinterpret_cast<uint2*>(p.to.bits + fp6_hi(tile, s, p.S) + fp6_hi_lane(lane) * 8) = make_uint2(v.w[4], v.w[5]);
    p.to.scales[scale_at(tile, s, p.S) + lane * 4] = (uint8_t)eb;
    if ((int)blockIdx.y >= p.tiles) return;
    // the other half-wave's block: its half `kh` for half 0 of its own, its dialect
    uint8_t* quad = p.quads + ((expert * p.tiles + blockIdx.y) * p.Q + (s >> 1)) * kQuadBytes;
    const uint32_t keep0 = kh ? codes.z : codes.x, keep1 = kh ? codes.w : codes.y, give0 = kh ? codes.x : codes.z, give1 = kh ? codes.y : codes.w;
    const uint32_t got0 = __shfl_xor(give0, 32), got1 = __shfl_xor(give1, 32), other = __shfl_xor(dl, 32);
    *reinterpret_cast<uint4*>(quad + (s & 1) * 1024 + lane * 16) = kh ? make_uint4(got0, got1, keep0, keep1) : make_uint4(keep0, keep1, got0, got1);
    const uint32_t first = kh ? other : dl, second = kh ? dl : other;
    uint8_t* meta = quad + 2048 + lane * 4;
    meta[s & 1] = (uint8_t)eb;
    meta[2 + (s & 1)] = (uint8_t)(first | second << 4);
    if (s == p.S - 1 && (p.S & 1)) {                             // no second step
        *reinterpret_cast<uint4*>(quad + 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
        meta[1] = 0;
        meta[3] = 0x77;
    }
}

// ---- rows

struct QuantizeArgs {
    const uint16_t* x;
    int64_t ld;
    const int32_t *rows, *order, *row_at;        // number of rows (device)
    Packed to;
    uint32_t k, KB, S;                           // k: rows are tokens', pair / k; 0: rows are the plan's own
    int64_t bound;                               // rows, at most
};

// Rows quantized in the plan's order (the arithmetic of the quantizer, quant_pass.h; as quantize_native_kernel, but for the rows' places).
// A wave takes 8 rows x 8 blocks; what is behind the last row is left as it is: it is multiplied, and its results are not kept.
// 32768 rows x 1024 27 to 29 us: 3.3 TB/s, vector instructions busy 54 % of the time, so by neither alone.  Tried: scale bytes through LDS, so that they leave as whole lines (31.8);
// the larger tables of half as many lookups (25.6).
constexpr int kQThreads = 256, kQWaves = kQThreads / 64, kPasses = 4;
__global__ __launch_bounds__(kQThreads) void experts_quantize_kernel(QuantizeArgs p) {
    __shared__ __attribute__((aligned(16))) uint8_t lds_q[kDialects * 32];
    __shared__ __attribute__((aligned(16))) uint8_t lds_s[kPairs * 32];
    __shared__ uint32_t s_fp6[kDialects * 2];
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t quad_id = lane >> 2, sub = lane & 3u, rq = quad_id >> 1, kh = quad_id & 1u;
    if (threadIdx.x < 32) reinterpret_cast<uint4*>(lds_q)[threadIdx.x] = reinterpret_cast<const uint4*>(g_quant_tables.near_i)[threadIdx.x];
    else if (threadIdx.x < 48) reinterpret_cast<uint4*>(lds_s)[threadIdx.x - 32] = reinterpret_cast<const uint4*>(g_quant_tables.vote1)[threadIdx.x - 32];
    else if (threadIdx.x >= 64 && threadIdx.x < 64 + kDialects * 2) s_fp6[threadIdx.x - 64] = (&g_fp6_book.w[0][0])[threadIdx.x - 64];
    __syncthreads();
    const int64_t present = *p.rows, rows = present < p.bound ? present : p.bound;
    const uint32_t sgroups = (p.S + 3u) / 4u;
    const int64_t units = (rows + 7) / 8 * sgroups;
    for (int64_t u = (int64_t)blockIdx.x * kQWaves + wave; u < units; u += (int64_t)gridDim.x * kQWaves) {
        const int64_t rg = u / sgroups;
        const uint32_t sg = (uint32_t)(u - rg * sgroups);
        const int64_t row = rg * 8 + rq;
        const bool row_ok = row < rows;
        const int64_t r = row_ok ? row : rows - 1;
        const uint16_t* xr = p.x + (p.k ? (int64_t)((uint32_t)p.order[r] / p.k) : r) * p.ld;
        const uint32_t to = (uint32_t)p.row_at[r], tile = to >> 5, slot = kh * 32u + (to & 31u);
        uint4 w[kPasses];
        bool on[kPasses];
#pragma unroll
        for (int q = 0; q < kPasses; ++q) {
            const uint32_t kb = (sg * 4u + q) * 2u + kh;
            on[q] = row_ok && kb < p.KB;
            w[q] = on[q] ? *reinterpret_cast<const uint4*>(xr + (size_t)kb * kBlock + sub * 8u) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < kPasses; ++q) {
            uint32_t code, eb, dl;
            dfp4_pass_small(w[q], lds_s, lds_q, code, eb, dl);
            const uint32_t step = sg * 4u + q;
            uint32_t lo24, hi24;                                       // 48 bits: low 32, those from bit 16, the upper 16
            pack6_quarter(code, s_fp6[dl * 2], s_fp6[dl * 2 + 1], lo24, hi24);
            const uint32_t lo32 = lo24 | (hi24 << 24), mid32 = (lo24 >> 16) | (hi24 << 8), hi16 = hi24 >> 8;
            const uint32_t next_lo = quad<0x39>(lo32);                 // of the lane after this one
            const uint32_t next_mid = quad<0x39>(mid32);
            const uint32_t lo_of_2 = quad<0xAA>(lo32);                 // lane 2's low dword
            const bool store = row_ok && step < p.S;                   // (a missing second block of the last step: zeros)
            if (store && sub == 0) {
                const uint4 v = on[q] ? make_uint4(lo32, hi16 | (next_lo << 16), next_mid, lo_of_2) : make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(p.to.bits + fp6_lo(tile, step, p.S) + slot * 16u) = v;
                p.to.scales[scale_at(tile, step, p.S) + slot * 4u] = on[q] ? (uint8_t)eb : (uint8_t)0;
            }
            if (store && sub == 2)
                *reinterpret_cast<uint2*>(p.to.bits + fp6_hi(tile, step, p.S) + fp6_hi_lane(slot) * 8u) =
                    on[q] ? make_uint2(hi16 | (next_lo << 16), next_mid) : make_uint2(0, 0);
        }
    }
}

struct GatherArgs {
    const uint8_t *codes, *dial, *expo;          // quantized tokens
    const int32_t *used, *order;
    const PlanGroup* halves;
    Packed to;
    int64_t most;                                // halves, at most
    uint32_t k;
    int KB, S;
};

// Quantized tokens rewritten in operand order for each of their experts, in whole lines.  A wave takes 128 rows and two steps; lane (kh, c) row c of
// each of four tiles, block 2 step + kh.  With the quantizer before it (8.5 us) 4096 tokens of 2048, 8 experts each, take 33 us; quantizing every row
// 45.7, bound by the quantizer's arithmetic; a token once, written to its places, 57 (16 bytes here and there).
__global__ __launch_bounds__(256) void experts_gather_kernel(GatherArgs p) {
    __shared__ uint2 s_fp6[kDialects];
    if (threadIdx.x < kDialects) s_fp6[threadIdx.x] = make_uint2(g_fp6_book.w[threadIdx.x][0], g_fp6_book.w[threadIdx.x][1]);
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kh = lane >> 5, c = lane & 31;
    const int steps8 = (p.S + 7) / 8;
    const int64_t units = min((int64_t)*p.used, p.most) * steps8;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t half = u / steps8;
        const int s0 = (int)(u - half * steps8) * 8 + wave * 2;
        const PlanGroup g = p.halves[half];
        if (s0 >= p.S) continue;
        uint4 codes[4][2];
        uint32_t e[4], d[4];                     // of four blocks: both steps', both lanes'
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t row = (int64_t)((uint32_t)p.order[g.row0 + min(t * 32 + c, g.rows - 1)] / p.k) * p.KB;
            __builtin_memcpy(&e[t], p.expo + row + 2 * s0, 4);               // (behind the last block: another row's, not used; the workspace has room)
            __builtin_memcpy(&d[t], p.dial + row + 2 * s0, 4);
#pragma unroll
            for (int q = 0; q < 2; ++q) codes[t][q] = *reinterpret_cast<const uint4*>(p.codes + (row + min(2 * (s0 + q) + kh, p.KB - 1)) * 16);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int s = s0 + q, at = 8 * (2 * q + kh);
            if (s >= p.S) break;
            const bool on = 2 * s + kh < p.KB;
            uint32_t scale = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t * 32 >= g.rows) break;
                const size_t tile = (size_t)(g.at >> 5) + t;
                const uint2 tab = s_fp6[(d[t] >> at) & 15u];
                const Fp6Lane v = pack6_lane(on ? codes[t][q] : make_uint4(0, 0, 0, 0), tab.x, tab.y);
                *reinterpret_cast<uint4*>(p.to.bits + fp6_lo(tile, s, p.S) + lane * 16) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
                *reinterpret_cast<uint2*>(p.to.bits + fp6_hi(tile, s, p.S) + fp6_hi_lane(lane) * 8) = make_uint2(v.w[4], v.w[5]);
                scale |= (on ? (e[t] >> at) & 255u : 0) << (8 * t);
            }
            *reinterpret_cast<uint32_t*>(p.to.scales + ((size_t)(g.at >> 7) * p.S + s) * 256 + lane * 4) = scale;
        }
    }
}

struct CodesArgs {
    const uint16_t* x;
    int64_t ld;
    const int32_t* rows;                         // how many there are (device), or null: all
    uint32_t* codes;
    uint8_t *dial, *expo;
    int64_t bound;
    int KB;
};

// Rows in their 4-bit form, as dfp4_quantize leaves it, as many as there are (what is behind them may be anything, infinities too)
__global__ __launch_bounds__(256) void experts_codes_kernel(CodesArgs p) {
    __shared__ __attribute__((aligned(16))) uint8_t lds_q[kDialects * 32];
    __shared__ __attribute__((aligned(16))) uint8_t lds_s[kPairs * 32];
    if (threadIdx.x < 32) reinterpret_cast<uint4*>(lds_q)[threadIdx.x] = reinterpret_cast<const uint4*>(g_quant_tables.near_i)[threadIdx.x];
    else if (threadIdx.x < 48) reinterpret_cast<uint4*>(lds_s)[threadIdx.x - 32] = reinterpret_cast<const uint4*>(g_quant_tables.vote1)[threadIdx.x - 32];
    __syncthreads();
    const int64_t rows = p.rows ? min((int64_t)*p.rows, p.bound) : p.bound, quarters = rows * p.KB * 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quarters; i += (int64_t)gridDim.x * 256) {
        const int64_t blk = i >> 2, row = blk / p.KB;
        const uint4 w = *reinterpret_cast<const uint4*>(p.x + row * p.ld + (blk - row * p.KB) * kBlock + (i & 3) * 8);
        uint32_t code, eb, dl;
        dfp4_pass_small(w, lds_s, lds_q, code, eb, dl);
        p.codes[i] = code;
        if ((i & 3) == 0) {
            p.expo[blk] = (uint8_t)eb;
            p.dial[blk] = (uint8_t)dl;
        }
    }
}

// ---- products of few rows an expert

// FP8 E4M3 bit patterns of a dialect's 8 magnitudes (0.5 u, all exact)
constexpr uint8_t e4m3_of_half_units(int u) {
    int e = -1;                                                        // floor(log2(0.5 u))
    for (int v = u; v > 1; v >>= 1) ++e;
    return u == 0 ? 0 : (uint8_t)(((e + 7) << 3) | (((u << 3) >> (e + 1)) & 7));
}
struct F8Book { uint32_t w[kDialects][2]; };
constexpr F8Book make_f8_book() {
    F8Book b{};
    for (int d = 0; d < kDialects; ++d)
        for (int j = 0; j < 8; ++j) b.w[d][j / 4] |= (uint32_t)e4m3_of_half_units(kBook[d][j]) << (8 * (j % 4));
    return b;
}
static __device__ const F8Book g_f8_book = make_f8_book();

struct FewArgs {
    const uint16_t* x;                           // rows in bf16, quantized on their way to LDS; or null:
    int64_t ld;
    const uint8_t *x_codes, *x_dial, *x_expo;    // quantized rows [.., K]
    const uint8_t* quads;                        // the weights' 4-bit form
    const int32_t *used, *order;
    const PlanGroup* plan;
    void* out;                                   // up: bf16 [row][rows / 2], down: f32 [row][rows]
    int64_t blocks;                              // at most
    uint32_t k;                                  // rows of x are tokens', pair / k; 0: the plan's own
    bool single;                                 // one token
    int KB, Q, rows, tiles;                      // blocks, quads of blocks; packed rows of an expert, tiles of 32 of them
};

__device__ __forceinline__ uint16_t bf16_of(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
// 8 codes -> FP8: elements 0, 2, 4, 6 and 1, 3, 5, 7 (rows and weights the same way, so that the order within a half of a block is free)
__device__ __forceinline__ void expand8(uint32_t c, uint2 tab, uint32_t& even, uint32_t& odd) {
    even = __builtin_amdgcn_perm(tab.y, tab.x, c & 0x07070707u) | ((c << 4) & 0x80808080u);
    odd = __builtin_amdgcn_perm(tab.y, tab.x, (c >> 4) & 0x07070707u) | (c & 0x80808080u);
}

// A quad of weights of a lane.  Loads go through a buffer's descriptor, made anew for each, that has no records for a quad behind the wave's last: such a
// load moves nothing.  (A load behind a branch would be waited for together with all others.)
struct Quad {
    uint4 c[2];
    uint32_t meta;
};
__device__ __forceinline__ void load_quad(Quad& q, const uint8_t* at, bool there, int lane) {
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(at), 0, there ? kQuadBytes : 0, 0x00027000);
#pragma unroll
    for (int step = 0; step < 2; ++step)
        q.c[step] = __builtin_bit_cast(uint4, (v4u)__builtin_amdgcn_raw_buffer_load_b128(from, lane * 16 + step * 1024, 0, 0));
    q.meta = __builtin_amdgcn_raw_buffer_load_b32(from, lane * 4 + 2048, 0, 0);
}

// A workgroup keeps the rows of a block (MT 1: up to 32, 2: up to 64) in LDS as FP8 and streams its expert's weights past them: 16 waves, SPLIT of which share K of a tile of 32
// packed rows of weights.  Weights go from memory to registers kAhead quads ahead, over the ends of tiles, and are expanded there.
// Bound by the weights' stream (0.5625 bytes an element): 64 tokens of 2 of 8 experts, 4096 x 14336 up, 104 to 109 us = 5.0 TB/s, a large copy's rate; with
// blocks of more than 32 rows among them, whose K takes two turns in LDS, 121 to 125.  Registers: with two tiles of rows 8 to 24 bytes of a thread's are in
// scratch memory (down, SPLIT 16: 60).  Tried: FP6 weights (a third more bytes); the last quad loaded again where there is none (whole K in a wave 7 % slower over 300 drawn
// products); offsets of quads in vector registers (two tiles of rows 5 to 20 % slower).  One token of 8 of 128 experts, 2048 x 1024 up, is bound
// by loads in turn (plan, row, weights): 7.8 us, 8.3 with the sums over waves in four steps.
template <bool GATED, int MT, int SPLIT>
__global__ __launch_bounds__(1024, 4) void experts_few_kernel(FewArgs p) {
    constexpr int kQuads = 32, kTiles = 16 / SPLIT, kAhead = 4;       // quads of 32 rows in LDS; tiles at a time
    __shared__ __attribute__((aligned(16))) uint8_t s_x[kQuads][2][2][64][16];           // [quad][step][block][lane], of the second tile of rows from quad 16 on
    __shared__ __attribute__((aligned(16))) uint16_t s_xs[kQuads][64];                   // exponents of a quad's two steps
    __shared__ float s_red[SPLIT > 1 ? 16 : 1][4][64];
    __shared__ uint2 s_tab[kDialects];
    __shared__ __attribute__((aligned(16))) uint8_t s_index[kDialects * 32], s_vote[kPairs * 32];
    __shared__ int32_t s_row[kListRows[2]];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = wave % SPLIT, sub = wave / SPLIT, h = lane >> 5, c = lane & 31;
    if (tid < kDialects) s_tab[tid] = make_uint2(g_f8_book.w[tid][0], g_f8_book.w[tid][1]);
    else if (p.x && tid >= 64 && tid < 96) reinterpret_cast<uint4*>(s_index)[tid - 64] = reinterpret_cast<const uint4*>(g_quant_tables.near_i)[tid - 64];
    else if (p.x && tid >= 128 && tid < 144) reinterpret_cast<uint4*>(s_vote)[tid - 128] = reinterpret_cast<const uint4*>(g_quant_tables.vote1)[tid - 128];
    const int batches = (p.tiles + kTiles - 1) / kTiles;
    // (one token: as many blocks as there can be, some without rows, and its row is known: a load less, twice, before the first that counts)
    const int64_t used = p.single ? p.blocks : min((int64_t)*p.used, p.blocks), items = used * batches;
    const int64_t lo = items * blockIdx.x / gridDim.x, hi = items * (blockIdx.x + 1) / gridDim.x;
    if (lo >= hi) return;

    // where this wave is: item (block of rows and batch of tiles), chunk of K (of all 32 quads, or of 16 for two tiles of rows)
    struct At {
        int64_t item, block;
        int batch, chunk, tiles;
        PlanGroup g;
    };
    auto begin = [&](int64_t item) {
        At a;
        a.item = item;
        a.block = item / batches;
        a.batch = (int)(item - a.block * batches);
        a.chunk = 0;
        a.g = p.plan[a.block];
        a.tiles = MT == 1 || a.g.rows <= 32 ? 1 : 2;
        return a;
    };
    auto last_chunk_of = [&](const At& a) { return (a.chunk + 1) * (kQuads / a.tiles) >= p.Q; };
    auto after = [&](const At& a) {
        At n = a;
        if (!last_chunk_of(a)) ++n.chunk;
        else if (a.item + 1 < hi) n = begin(a.item + 1);
        return n;
    };
    // its quads there: the first one's address and their number
    struct Segment {
        const uint8_t* at;
        int first, n;
    };
    auto segment = [&](const At& a) {
        const int chunk = kQuads / a.tiles, in = min(chunk, p.Q - a.chunk * chunk), per = (in + SPLIT - 1) / SPLIT, first = part * per;
        const int tile = a.batch * kTiles + sub, n = tile < p.tiles ? max(0, min(in, first + per) - first) : 0;
        return Segment{p.quads + (((int64_t)a.g.expert * p.tiles + tile) * p.Q + a.chunk * chunk + first) * kQuadBytes, first, n};
    };
    Quad ring[kAhead];
    auto load = [&](Quad& q, const Segment& s, int i) { load_quad(q, s.at + (int64_t)i * kQuadBytes, i < s.n, lane); };
    v16f acc[MT];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[i][x] = 0.0f;
    };
    auto multiply = [&](const Quad& q, int at, int tiles) {          // quad `at` of the chunk, tiles of rows there are
        int xs[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) xs[i] = s_xs[(at + 16 * i) % kQuads][lane];           // (the second: of no use where there is one)
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const uint32_t d = q.meta >> (16 + 8 * step);
            const uint2 t0 = s_tab[d & 15u], t1 = s_tab[(d >> 4) & 15u];
            uint32_t w[8];
            expand8(q.c[step].x, t0, w[0], w[1]);
            expand8(q.c[step].y, t0, w[2], w[3]);
            expand8(q.c[step].z, t1, w[4], w[5]);
            expand8(q.c[step].w, t1, w[6], w[7]);
            const v8i wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], (int)w[6], (int)w[7]};
            v8i xv[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i >= tiles) break;
                const int4 a = *reinterpret_cast<const int4*>(s_x[at + 16 * i][step][0][lane]), b = *reinterpret_cast<const int4*>(s_x[at + 16 * i][step][1][lane]);
                xv[i] = v8i{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i >= tiles) break;
                if (step == 0) acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv, xv[i], acc[i], 0, 0, 0, (int)q.meta, 0, xs[i]);
                else acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv, xv[i], acc[i], 0, 0, 1, (int)q.meta, 1, xs[i]);
            }
            // the operands are in use until here (a result must not overlap them, see gemm_f8.hip)
#pragma unroll
            for (int i = 0; i < MT; ++i) asm volatile("" : "+v"(acc[i]) : "v"(wv), "v"(xv[i]));
        }
    };
    auto row_of = [&](int r) { return p.single && GATED ? (int64_t)0 : (int64_t)s_row[r]; };
    // rows of the chunk into LDS; blocks behind the last of a quad as zeros
    auto stage = [&](const At& a, bool other_rows) {
        const int rows = min(32 * MT, a.g.rows), q0 = a.chunk * (kQuads / a.tiles), blocks = min(kQuads / a.tiles, p.Q - q0) * 4;
        __syncthreads();                                             // what was there is done with
        if (other_rows && !(p.single && GATED)) {
            if (tid < rows) {
                const int64_t row = (int64_t)a.g.row0 + tid;
                s_row[tid] = p.k ? (int32_t)((uint32_t)p.order[row] / p.k) : (int32_t)row;
            }
            __syncthreads();
        }
        // (four lanes a block: the quantizer's arithmetic)
        if (p.x)
            for (int i = tid; i < rows * blocks * 4; i += 1024) {
                const int r = i / (blocks * 4), b = (i >> 2) - r * blocks, kb = q0 * 4 + b, quarter = i & 3;
                const bool on = kb < p.KB;
                const uint4 v = on ? *reinterpret_cast<const uint4*>(p.x + row_of(r) * p.ld + kb * kBlock + quarter * 8) : make_uint4(0, 0, 0, 0);
                uint32_t code, e, d;
                dfp4_pass_small(v, s_vote, s_index, code, e, d);
                uint2 to;
                expand8(code, s_tab[d], to.x, to.y);
                const int q = (r >> 5) * 16 + (b >> 2), l = (quarter >> 1) * 32 + (r & 31);
                *reinterpret_cast<uint2*>(&s_x[q][(b >> 1) & 1][b & 1][l][(quarter & 1) * 8]) = to;
                if (quarter == 0) reinterpret_cast<uint8_t*>(&s_xs[q][(b & 1) * 32 + (r & 31)])[(b >> 1) & 1] = on ? (uint8_t)e : 0;
            }
        else for (int i0 = tid; i0 < rows * blocks; i0 += 2048) {
            // two at a time, so that their loads are
            uint4 codes[2];
            uint32_t e[2], d[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = min(i0 + 1024 * u, rows * blocks - 1), r = i / blocks, b = i - r * blocks;
                const int64_t blk = row_of(r) * p.KB + min(q0 * 4 + b, p.KB - 1);
                codes[u] = *reinterpret_cast<const uint4*>(p.x_codes + blk * 16);
                e[u] = p.x_expo[blk];
                d[u] = p.x_dial[blk];
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = i0 + 1024 * u, r = i / blocks, b = i - r * blocks;
                if (i >= rows * blocks) break;
                const bool on = q0 * 4 + b < p.KB;
                const uint2 tab = on ? s_tab[d[u] & 15u] : make_uint2(0, 0);
                uint4 lo4, hi4;
                expand8(codes[u].x, tab, lo4.x, lo4.y);
                expand8(codes[u].y, tab, lo4.z, lo4.w);
                expand8(codes[u].z, tab, hi4.x, hi4.y);
                expand8(codes[u].w, tab, hi4.z, hi4.w);
                const int q = (r >> 5) * 16 + (b >> 2), l = r & 31;
                *reinterpret_cast<uint4*>(s_x[q][(b >> 1) & 1][b & 1][l]) = lo4;
                *reinterpret_cast<uint4*>(s_x[q][(b >> 1) & 1][b & 1][32 + l]) = hi4;
                reinterpret_cast<uint8_t*>(&s_xs[q][(b & 1) * 32 + l])[(b >> 1) & 1] = on ? (uint8_t)e[u] : 0;
            }
        }
        __syncthreads();
    };
    // registers x and x + 1 (x even) of lane (h, c): packed rows 8 (x / 4) + 4 h + x % 4 and the next, row c
    auto emit = [&](const At& a, int i, int tile, int x, float v0, float v1) {
        const int r = i * 32 + c, n = tile * 32 + 8 * (x >> 2) + 4 * h + (x & 3);
        if (tile >= p.tiles || r >= a.g.rows || n >= p.rows) return;
        const int64_t row = (int64_t)a.g.row0 + r;
        if constexpr (GATED) static_cast<uint16_t*>(p.out)[row * (p.rows >> 1) + (n >> 1)] = bf16_of(v0 < kFarGate ? silu_far(v0, v1) : silu_times(v0, v1));
        else *reinterpret_cast<float2*>(static_cast<float*>(p.out) + row * p.rows + n) = make_float2(v0, v1);
    };

    At now = begin(lo);
    Segment seg = segment(now);
#pragma unroll
    for (int d = 0; d < kAhead; ++d) load(ring[d], seg, d);
    int64_t staged_block = -1;
    int staged_chunk = 0;
    clear();
    for (;;) {
        const bool last_chunk = last_chunk_of(now), last = last_chunk && now.item + 1 >= hi;
        if (staged_block != now.block || staged_chunk != now.chunk) {
            stage(now, staged_block != now.block);
            staged_block = now.block, staged_chunk = now.chunk;
        }
        const At then = after(now);
        Segment next = segment(then);
        if (last) next.n = 0;
        if (seg.n == 0) {
#pragma unroll
            for (int d = 0; d < kAhead; ++d) load(ring[d], next, d);
        }
        for (int q = 0; q < seg.n; q += kAhead) {
            const bool more = q + kAhead < seg.n;
#pragma unroll
            for (int d = 0; d < kAhead; ++d) {
                if (q + d < seg.n) multiply(ring[d], seg.first + q + d, now.tiles);
                load(ring[d], more ? seg : next, more ? q + kAhead + d : d);
            }
        }
        if (last_chunk) {
            if constexpr (SPLIT == 1) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int x = 0; x < 16; x += 2)
                        if (i < now.tiles) emit(now, i, now.batch * kTiles + sub, x, acc[i][x], acc[i][x + 1]);
            } else if (now.tiles == 1 && p.Q <= kQuads / 2) {
                // the parts of K are added in their order, all registers at once through the half of LDS that the rows leave
                float(*red)[16][64] = reinterpret_cast<float(*)[16][64]>(s_x[kQuads / 2]);
                __syncthreads();
#pragma unroll
                for (int x = 0; x < 16; ++x) red[wave][x][lane] = acc[0][x];
                __syncthreads();
#pragma unroll 1
                for (int job = wave; job < 8 * kTiles; job += 16) {
                    const int tile = job >> 3, x = (job & 7) * 2;
                    float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
                    for (int w = 0; w < SPLIT; ++w) {
                        v0 += red[tile * SPLIT + w][x][lane];
                        v1 += red[tile * SPLIT + w][x + 1][lane];
                    }
                    emit(now, 0, now.batch * kTiles + tile, x, v0, v1);
                }
            } else {
                // four registers at a time
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (i >= now.tiles) break;
#pragma unroll
                    for (int x4 = 0; x4 < 16; x4 += 4) {
                        __syncthreads();
#pragma unroll
                        for (int x = 0; x < 4; ++x) s_red[wave][x][lane] = acc[i][x4 + x];
                        __syncthreads();
                        for (int job = wave; job < 2 * kTiles; job += 16) {
                            const int tile = job >> 1, x = (job & 1) * 2;
                            float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
                            for (int w = 0; w < SPLIT; ++w) {
                                v0 += s_red[tile * SPLIT + w][x][lane];
                                v1 += s_red[tile * SPLIT + w][x + 1][lane];
                            }
                            emit(now, i, now.batch * kTiles + tile, x4 + x, v0, v1);
                        }
                    }
                }
            }
            clear();
        }
        if (last) return;
        now = then;
        seg = next;
    }
}

// ---- a few tokens, down: their results whole

struct TokenArgs {
    const uint16_t* h;
    int64_t ld;
    const uint8_t* quads;
    const int32_t *place, *expert;
    const float* weights;
    void* y;
    int64_t pairs;
    int experts, k, KB, Q, rows, tiles;
};
constexpr int kTokenElements = 48 << 10;         // of a token's rows, in LDS

// A workgroup a token and 32 results: its 16 waves share the quads of all the token's experts (a wave's are neighbours, of one or a few
// experts), add them with the router's weights and join in the order of the waves.  Rows are quantized by every workgroup anew, on their way
// to LDS, while the first weights come.  Bound by latency: one token of 8 of 128 experts, 2048 x 1024, 8.5 us, of which 5.7 are what an empty call takes.
template <bool BF16>
__global__ __launch_bounds__(1024, 4) void experts_token_kernel(TokenArgs p) {
    constexpr int kAhead = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t s_rows[];  // [j][step][block][half][16], then exponents [j][quad][half][2]
    __shared__ float s_red[16][32];
    __shared__ uint2 s_tab[kDialects];
    __shared__ __attribute__((aligned(16))) uint8_t s_index[kDialects * 32], s_vote[kPairs * 32];
    __shared__ int32_t s_row[kMaxChoice], s_expert[kMaxChoice];
    __shared__ float s_weight[kMaxChoice];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int tile = blockIdx.x;
    const int64_t token = blockIdx.y;
    if (tid < kDialects) s_tab[tid] = make_uint2(g_f8_book.w[tid][0], g_f8_book.w[tid][1]);
    else if (tid >= 64 && tid < 96) reinterpret_cast<uint4*>(s_index)[tid - 64] = reinterpret_cast<const uint4*>(g_quant_tables.near_i)[tid - 64];
    else if (tid >= 128 && tid < 144) reinterpret_cast<uint4*>(s_vote)[tid - 128] = reinterpret_cast<const uint4*>(g_quant_tables.vote1)[tid - 128];
    else if (tid >= 192 && tid < 192 + p.k) {
        const int j = tid - 192;
        const int32_t row = p.place[token * p.k + j], expert = p.expert[token * p.k + j];
        const float weight = p.weights[token * p.k + j];
        const bool there = row >= 0 && row < p.pairs && (uint32_t)expert < (uint32_t)p.experts;
        s_row[j] = there ? row : -1;
        s_expert[j] = there ? expert : 0;
        s_weight[j] = there ? weight : 0.0f;
    }
    __syncthreads();
    const int units = p.k * p.Q, lo = units * wave / 16, hi = units * (wave + 1) / 16;
    Quad ring[kAhead];
    auto load = [&](Quad& q, int u) {
        const int j = min(u, units - 1) / p.Q, expert = __builtin_amdgcn_readfirstlane(s_expert[j]);
        load_quad(q, p.quads + (((int64_t)expert * p.tiles + tile) * p.Q + (u - j * p.Q)) * kQuadBytes, u < hi, lane);
    };
#pragma unroll
    for (int d = 0; d < kAhead; ++d) load(ring[d], lo + d);
    const int blocks = p.Q * 4;
    uint8_t* s_scale = s_rows + (size_t)p.k * p.Q * 128;
    for (int i = tid; i < p.k * blocks * 4; i += 1024) {
        const int j = i / (blocks * 4), b = (i >> 2) - j * blocks, quarter = i & 3;
        const bool on = b < p.KB && s_row[j] >= 0;
        const uint4 v = on ? *reinterpret_cast<const uint4*>(p.h + (int64_t)s_row[j] * p.ld + b * kBlock + quarter * 8) : make_uint4(0, 0, 0, 0);
        uint32_t code, e, d;
        dfp4_pass_small(v, s_vote, s_index, code, e, d);
        uint2 to;
        expand8(code, s_tab[d], to.x, to.y);
        *reinterpret_cast<uint2*>(s_rows + (size_t)(j * blocks + b) * 32 + (quarter >> 1) * 16 + (quarter & 1) * 8) = to;
        if (quarter == 0) s_scale[(j * p.Q + (b >> 2)) * 4 + (b & 1) * 2 + ((b >> 1) & 1)] = on ? (uint8_t)e : 0;
    }
    __syncthreads();
    v16f acc, sum;
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[x] = sum[x] = 0.0f;
    int before = lo / p.Q;
    for (int u0 = lo; u0 < hi; u0 += kAhead) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
            const int u = u0 + d;
            if (u < hi) {
                const int j = u / p.Q;
                if (j != before) {
                    const float w = s_weight[before];
#pragma unroll
                    for (int x = 0; x < 16; ++x) sum[x] += w * acc[x], acc[x] = 0.0f;
                    before = j;
                }
                const int xs = *reinterpret_cast<const uint16_t*>(s_scale + u * 4 + h * 2);
#pragma unroll
                for (int step = 0; step < 2; ++step) {
                    const uint32_t dl = ring[d].meta >> (16 + 8 * step);
                    const uint2 t0 = s_tab[dl & 15u], t1 = s_tab[(dl >> 4) & 15u];
                    uint32_t w[8];
                    expand8(ring[d].c[step].x, t0, w[0], w[1]);
                    expand8(ring[d].c[step].y, t0, w[2], w[3]);
                    expand8(ring[d].c[step].z, t1, w[4], w[5]);
                    expand8(ring[d].c[step].w, t1, w[6], w[7]);
                    const v8i wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], (int)w[6], (int)w[7]};
                    const uint8_t* from = s_rows + (size_t)u * 128 + step * 64 + h * 16;
                    const int4 a = *reinterpret_cast<const int4*>(from), b = *reinterpret_cast<const int4*>(from + 32);
                    const v8i xv = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                    if (step == 0) acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv, xv, acc, 0, 0, 0, (int)ring[d].meta, 0, xs);
                    else acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv, xv, acc, 0, 0, 1, (int)ring[d].meta, 1, xs);
                    asm volatile("" : "+v"(acc) : "v"(wv), "v"(xv));       // (as above)
                }
            }
            load(ring[d], u + kAhead);
        }
    }
    if (hi > lo) {
        const float w = s_weight[before];
#pragma unroll
        for (int x = 0; x < 16; ++x) sum[x] += w * acc[x];
    }
    // every column is the token's
    if ((lane & 31) == 0) {
#pragma unroll
        for (int x = 0; x < 16; ++x) s_red[wave][8 * (x >> 2) + 4 * h + (x & 3)] = sum[x];
    }
    __syncthreads();
    if (tid < 32) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) v += s_red[w][tid];
        const int n = tile * 32 + tid;
        if (n < p.rows) {
            if constexpr (BF16) static_cast<uint16_t*>(p.y)[token * p.rows + n] = bf16_of(v);
            else static_cast<float*>(p.y)[token * p.rows + n] = v;
        }
    }
}

struct JoinArgs {
    const float* part;
    const float* weights;
    const int32_t* place;
    void* y;
    int64_t tokens, pairs;
    int k, dim;
};

// y[token] = sum over j of weights[token, j] * part[place]; a token has 2^lanes threads of eight elements.  Four rows at a time, none
// behind a branch: one that is absent reads row 0 and is left out.
template <bool BF16>
__global__ __launch_bounds__(256) void experts_join_kernel(JoinArgs p, int lanes) {
    for (int64_t token = (int64_t)blockIdx.x * (256 >> lanes) + (threadIdx.x >> lanes); token < p.tokens; token += (int64_t)gridDim.x * (256 >> lanes)) {
        const int32_t* place = p.place + token * p.k;
        const float* weights = p.weights + token * p.k;
        for (int d = (int)(threadIdx.x & ((1u << lanes) - 1)) * 8; d < p.dim; d += 8 << lanes) {
            float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int j0 = 0; j0 < p.k; j0 += 4) {
                float4 u[4][2];
                bool there[4];
                float w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int j = min(j0 + q, p.k - 1);
                    const int32_t row = place[j];
                    there[q] = j0 + q < p.k && row >= 0 && row < p.pairs;
                    w[q] = weights[j];
                    const float4* from = reinterpret_cast<const float4*>(p.part + (int64_t)(there[q] ? row : 0) * p.dim + d);
                    u[q][0] = from[0], u[q][1] = from[1];
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (!there[q]) continue;
                    const float v[8] = {u[q][0].x, u[q][0].y, u[q][0].z, u[q][0].w, u[q][1].x, u[q][1].y, u[q][1].z, u[q][1].w};
#pragma unroll
                    for (int x = 0; x < 8; ++x) y[x] += w[q] * v[x];
                }
            }
            if constexpr (BF16) {
                typedef __bf16 v8b __attribute__((ext_vector_type(8)));
                v8b o;
#pragma unroll
                for (int x = 0; x < 8; ++x) o[x] = (__bf16)y[x];
                *reinterpret_cast<v8b*>(static_cast<uint16_t*>(p.y) + token * p.dim + d) = o;
            } else {
                float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.y) + token * p.dim + d);
                to[0] = make_float4(y[0], y[1], y[2], y[3]);
                to[1] = make_float4(y[4], y[5], y[6], y[7]);
            }
        }
    }
}

// The experts that tokens go to, were all alike
inline int64_t active_experts(const dfp4_plan& plan) {
    const int64_t pairs = plan.tokens * plan.k;
    if (pairs >= 8 * plan.experts) return plan.experts;
    const double none = pow(1.0 - 1.0 / (double)plan.experts, (double)pairs);
    const int64_t n = (int64_t)((double)plan.experts * (1.0 - none) + 0.5);
    return n > 0 ? n : 1;
}
// Rows an expert up to which weights are streamed past them; both sides, us, few / many, up: 16 rows 117 / 148, 32 rows 132 / 152, 71 / 73, 105 / 94, 47 / 35,
// 40 rows 71 / 48, 48 rows 130 / 156, 50 rows 112 / 98, 64 rows 70 / 74; down: 16 rows 63 / 110, 32 rows 84 / 114, 42 / 52, 84 / 55, 37 / 29, 42 rows 32 / 23, 48 rows 163 / 117,
// 64 rows 66 / 55.  Of 54 products up and 58 down of 4 to 100 rows the better one is missed by 5 % in the mean (lines at 24 and 40: 5 and 6 %)
constexpr int64_t kFewRows = 34;
// Whether the large kernel takes 128 rows at a time instead of 256: where an expert has no more than 160 (half / whole: 42 rows 28 / 33 us, 128 rows 88 / 91 and
// 126 / 143, 250 rows 76 / 63, 117 / 107; down 64 rows 57 / 55, 128 rows 73 / 76, 512 rows 207 / 181), or tiles of 256 would leave half of the compute units idle (325 rows,
// 4 columns of tiles, 27.6 / 33.7).  Of 81 drawn products the better one is missed by 0.7 % in the mean, of 44 others, down, by 0.8 %.
inline bool half_tiles(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t active = active_experts(plan), rows = plan.tokens * plan.k / active;
    return rows <= 160 || active * ((rows + 255) / 256) * (padded_rows(w) / 256) * 2 <= device_cu_count();
}
// Whether tokens are taken one by one (down): where there are few, and weights that several of them read, again for each, cost less than the two
// launches that are spared (4 us): 4 tokens of 8 of 128 experts 11.9 us instead of 17.5, 8 tokens 21.7 and 22.5, 16 tokens 40 and 30
inline bool token_by_token(const dfp4_plan& plan, const dfp4_experts& w) {
    if (w.gated || plan.k * quads_of(w.K) * 128 > kTokenElements || plan.tokens * row_tiles(w) > 2 * device_cu_count()) return false;
    const int64_t again = plan.tokens * plan.k - active_experts(plan);
    return again * w.rows * w.K <= 28 << 20;
}

// How many waves share K in products of few rows, by rounds of items over the compute units: a wave takes 1.08 us for a quad (the chip's memory among its waves), an item 2 us
// more, a sum over waves 1.5 to 2.9 for 32 rows, K in turns 2.5 a turn.  Of 234 drawn products the best of the five is missed by 2.2 % in the mean
// (always two: 12 %).  From 10 rows an expert on, some have more than 32.
inline int waves_of_K(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t active = active_experts(plan), tiles = row_tiles(w), cus = device_cu_count();
    const int Q = (int)quads_of(w.K), two = plan.tokens * plan.k > 10 * active ? 2 : 1, turns = (Q * two + 31) / 32;
    int split = 1;
    float least = 0.0f;
    for (int s = 1; s <= 16; s *= 2) {
        const int64_t per = 16 / s, n = active * ((tiles + per - 1) / per), rounds = (n + cus - 1) / cus;
        const int chunk = Q < 32 / two ? Q : 32 / two, quads = turns * ((chunk + s - 1) / s);
        const float sum = s == 1 ? 0.0f : s == 16 ? 2.85f : s == 8 ? 2.0f : 1.47f;
        const float us = (float)rounds * (1.08f * (float)quads + 2.0f + (float)two * (sum + (turns > 1 ? 2.46f * (float)turns : 0.0f)));
        if (s == 1 || us < least) least = us, split = s;
    }
    return split;
}

// workspace: rows in operand order, or in their 4-bit form (few), and down their products
struct Workspace {
    bool many;
    int64_t rows, codes, dial, expo, part, total;
};
inline Workspace workspace_of(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t pairs = plan.tokens * plan.k;
    Workspace x{};
    x.many = pairs > kFewRows * active_experts(plan);
    if (x.many) {
        x.rows = plan_list(pairs, plan.experts, 0) * kGroupRows;
        x.part = up256((int64_t)native_packed_bytes(x.rows, w.K, true));
        // Quantized once a token where that spares more than the launch that it adds: 333 tokens of 5 experts, 1440 elements each, 28.0 us instead of 23.6
        // (all of up), 4096 of 8, 2048 each, 158 instead of 167
        if (w.gated && plan.k > 1 && pairs * w.K >= 1 << 25) {
            x.codes = x.part;
            x.dial = x.codes + up256(plan.tokens * (w.K / 2));
            x.expo = x.dial + up256(plan.tokens * (w.K / kBlock) + 4);
            x.part = x.expo + up256(plan.tokens * (w.K / kBlock) + 4);
        }
    } else {
        x.rows = w.gated ? plan.tokens : pairs;
        x.dial = up256(x.rows * (w.K / 2));
        x.expo = x.dial + up256(x.rows * (w.K / kBlock));
        x.part = x.expo + up256(x.rows * (w.K / kBlock));
    }
    x.total = x.part + (w.gated ? 0 : up256(pairs * w.rows * 4));
    return x;
}

}  // namespace

// where the 4-bit form lies in the packed weights
static int64_t quads_offset(const dfp4_experts& w) { return up256((int64_t)native_packed_bytes(w.experts * padded_rows(w), w.K, true)); }

size_t expert_weights_bytes(int64_t experts, int64_t rows, int64_t K, bool gated) {
    const dfp4_experts w{nullptr, experts, rows, K, gated ? 1 : 0};
    return (size_t)(quads_offset(w) + up256(experts * row_tiles(w) * quads_of(K) * kQuadBytes));
}

int launch_expert_weights(dfp4_tensor gate, dfp4_tensor up, const dfp4_experts& w, hipStream_t stream) {
    PackArgs p{};
    p.codes[0] = gate.codes, p.dial[0] = gate.dialect, p.expo[0] = gate.exponent;
    p.codes[1] = up.codes, p.dial[1] = up.dialect, p.expo[1] = up.exponent;
    p.to = packed_at(w.packed, w.experts * padded_rows(w), w.K);
    p.rows = (int)w.rows, p.KB = (int)(w.K / kBlock), p.S = (int)steps_of(w.K), p.gated = w.gated ? 1 : 0;
    p.quads = static_cast<uint8_t*>(w.packed) + quads_offset(w), p.tiles = (int)row_tiles(w), p.Q = (int)quads_of(w.K);
    const dim3 grid((unsigned)((p.S + 3) / 4), (unsigned)(padded_rows(w) / 32), (unsigned)w.experts);
    hipLaunchKernelGGL(experts_pack_kernel, grid, dim3(256), 0, stream, p);
    return check_launch();
}

ExpertsWay experts_way(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t pairs = plan.tokens * plan.k;
    if (token_by_token(plan, w)) return ExpertsWay{1, 16, kWithin};
    const Workspace ws = workspace_of(plan, w);
    if (ws.many) return ExpertsWay{half_tiles(plan, w) ? 128 : 256, 1, ws.codes ? kOnceAToken : kBefore};
    // Quantized by the workgroups that take them where that is little work: a launch less (2.5 us), but 1.1 us a workgroup and 8192 elements
    // (16 rows of 4096: 112 us instead of 107)
    return ExpertsWay{pairs > 32 ? 64 : 32, waves_of_K(plan, w), pairs * w.K <= active_experts(plan) * 12288 ? kWithin : kBefore};
}

// Whether one launch holds the tiles of a product of many rows (fewer than 2^32 threads)
bool experts_fit(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t pairs = plan.tokens * plan.k;
    return !workspace_of(plan, w).many || plan_list(pairs, plan.experts, half_tiles(plan, w) ? 1 : 0) * (padded_rows(w) / 256) < (1 << 24) - 8;
}

size_t experts_workspace_bytes(const dfp4_plan& plan, const dfp4_experts& w) { return (size_t)workspace_of(plan, w).total; }

template <bool GATED, int MT>
static void launch_few(const FewArgs& p, int split, dim3 grid, hipStream_t stream) {
    if (split == 1) hipLaunchKernelGGL((experts_few_kernel<GATED, MT, 1>), grid, dim3(1024), 0, stream, p);
    else if (split == 2) hipLaunchKernelGGL((experts_few_kernel<GATED, MT, 2>), grid, dim3(1024), 0, stream, p);
    else if (split == 4) hipLaunchKernelGGL((experts_few_kernel<GATED, MT, 4>), grid, dim3(1024), 0, stream, p);
    else if (split == 8) hipLaunchKernelGGL((experts_few_kernel<GATED, MT, 8>), grid, dim3(1024), 0, stream, p);
    else hipLaunchKernelGGL((experts_few_kernel<GATED, MT, 16>), grid, dim3(1024), 0, stream, p);
}

int launch_experts(const ExpertsArgs& a, hipStream_t stream) {
    const int64_t pairs = a.plan.tokens * a.plan.k, S = steps_of(a.w.K);
    const Workspace ws = workspace_of(a.plan, a.w);
    const ExpertsWay way = experts_way(a.plan, a.w);
    const PlanView plan = plan_view(a.plan);
    const int cus = device_cu_count();
    if (way.rows == 1) {
        TokenArgs p{};
        p.h = a.x, p.ld = a.ld;
        p.quads = static_cast<const uint8_t*>(a.w.packed) + quads_offset(a.w);
        p.place = plan.place, p.expert = plan.expert, p.weights = a.weights;
        p.y = a.out, p.pairs = pairs, p.experts = (int)a.plan.experts;
        p.k = (int)a.plan.k, p.KB = (int)(a.w.K / kBlock), p.Q = (int)quads_of(a.w.K), p.rows = (int)a.w.rows, p.tiles = (int)row_tiles(a.w);
        const dim3 grid((unsigned)p.tiles, (unsigned)a.plan.tokens);
        const size_t lds = (size_t)p.k * p.Q * 132;
        if (a.out_dtype == DFP4_BF16) hipLaunchKernelGGL((experts_token_kernel<true>), grid, dim3(1024), lds, stream, p);
        else hipLaunchKernelGGL((experts_token_kernel<false>), grid, dim3(1024), lds, stream, p);
        return check_launch();
    }
    void* out = a.w.gated ? a.out : a.workspace + ws.part;
    if (way.rows >= 128) {
        QuantizeArgs q{};
        q.x = a.x, q.ld = a.ld;
        q.rows = plan.offsets + a.plan.experts, q.order = plan.order, q.row_at = plan.row_at;
        q.to = packed_at(a.workspace, ws.rows, a.w.K);
        q.k = a.w.gated ? (uint32_t)a.plan.k : 0, q.KB = (uint32_t)(a.w.K / kBlock), q.S = (uint32_t)S;
        q.bound = pairs;
        if (way.quantized == kOnceAToken) {
            const dfp4_tensor x{a.workspace + ws.codes, a.workspace + ws.dial, a.workspace + ws.expo, a.plan.tokens, a.w.K};
            const int rc = launch_quantize(false, a.x, a.plan.tokens, a.w.K, a.ld, x, stream);
            if (rc != DFP4_OK) return rc;
            const GatherArgs g{x.codes, x.dialect, x.exponent, plan.used + 1, plan.order, plan.list[1], q.to, plan_list(pairs, a.plan.experts, 1),
                               (uint32_t)a.plan.k, (int)q.KB, (int)S};
            const int64_t wgs = g.most * ((S + 7) / 8);
            hipLaunchKernelGGL(experts_gather_kernel, dim3((unsigned)(wgs < 16 * cus ? wgs : 16 * cus)), dim3(256), 0, stream, g);
        } else {
            const int64_t units = (pairs + 7) / 8 * ((S + 3) / 4), want = (units + kQWaves - 1) / kQWaves;
            hipLaunchKernelGGL(experts_quantize_kernel, dim3((unsigned)(want < 8 * cus ? want : 8 * cus)), dim3(kQThreads), 0, stream, q);
        }
        ExpertTiles t{};
        t.a = q.to.bits, t.a_scales = native_scale_offset(ws.rows, a.w.K, true);
        t.w = a.w.packed, t.w_scales = native_scale_offset(a.w.experts * padded_rows(a.w), a.w.K, true);
        t.half = way.rows == 128;
        t.used = plan.used + (t.half ? 1 : 0), t.list = plan.list[t.half ? 1 : 0], t.most = plan_list(pairs, a.plan.experts, t.half ? 1 : 0);
        t.K = (int)a.w.K, t.rows = (int)expert_rows(a.w), t.tiles = (int)(padded_rows(a.w) / 256);
        t.gated = a.w.gated != 0;
        t.out = out;
        const int rc = launch_expert_tiles(t, stream);
        if (rc != DFP4_OK) return rc;
    } else {
        const dfp4_tensor x{a.workspace, a.workspace + ws.dial, a.workspace + ws.expo, ws.rows, a.w.K};
        FewArgs p{};
        if (way.quantized == kWithin) {
            p.x = a.x, p.ld = a.ld;
        } else {
            const CodesArgs c{a.x, a.ld, a.w.gated ? nullptr : plan.offsets + a.plan.experts, reinterpret_cast<uint32_t*>(x.codes), x.dialect, x.exponent, ws.rows,
                              (int)(a.w.K / kBlock)};
            const int64_t wgs = (ws.rows * (a.w.K / 8) + 255) / 256;
            hipLaunchKernelGGL(experts_codes_kernel, dim3((unsigned)(wgs < 16 * cus ? wgs : 16 * cus)), dim3(256), 0, stream, c);
        }
        p.x_codes = x.codes, p.x_dial = x.dialect, p.x_expo = x.exponent;
        p.quads = static_cast<const uint8_t*>(a.w.packed) + quads_offset(a.w);
        p.used = plan.used + 2, p.order = plan.order, p.plan = plan.list[2];
        p.out = out, p.blocks = plan_list(pairs, a.plan.experts, 2);
        p.k = a.w.gated ? (uint32_t)a.plan.k : 0, p.single = a.plan.tokens == 1;
        p.KB = (int)(a.w.K / kBlock), p.Q = (int)quads_of(a.w.K), p.rows = (int)expert_rows(a.w), p.tiles = (int)row_tiles(a.w);
        const int64_t items = p.blocks * ((p.tiles + 16 / way.waves - 1) / (16 / way.waves));
        const dim3 grid((unsigned)(items < cus ? items : cus));
        if (a.w.gated && way.rows == 32) launch_few<true, 1>(p, way.waves, grid, stream);
        else if (a.w.gated) launch_few<true, 2>(p, way.waves, grid, stream);
        else if (way.rows == 32) launch_few<false, 1>(p, way.waves, grid, stream);
        else launch_few<false, 2>(p, way.waves, grid, stream);
    }
    if (!a.w.gated) {
        const JoinArgs j{static_cast<const float*>(out), a.weights, plan.place, a.out, a.plan.tokens, pairs, (int)a.plan.k, (int)a.w.rows};
        int lanes = 0;
        while (lanes < 8 && (8 << lanes) < a.w.rows) ++lanes;
        const int64_t wgs = (a.plan.tokens + (256 >> lanes) - 1) / (256 >> lanes);
        const dim3 jg((unsigned)(wgs < (1 << 20) ? wgs : 1 << 20));
        if (a.out_dtype == DFP4_BF16) hipLaunchKernelGGL((experts_join_kernel<true>), jg, dim3(256), 0, stream, j, lanes);
        else hipLaunchKernelGGL((experts_join_kernel<false>), jg, dim3(256), 0, stream, j, lanes);
    }
    return check_launch();
}

}  // namespace dfp4
