// Products of a sparse layer's experts on the block-scaled matrix instruction (include/dfp4.h; operand layout: fp6_pack.h, gemm_native.hip).
//
// Rows (pairs of a token and an expert) come in the plan's order, an expert's from a group of kGroupRows on, so that every tile of rows
// has one expert.  experts_quantize_kernel quantizes rows straight into operand order, experts_kernel multiplies a tile of 32 rows with 32
// rows of its expert's weights; down, experts_join_kernel adds a token's rows in a fixed order.
// Gate and up rows take turns in the packed weights, and weights are the instruction's first operand, rows its second: a lane then holds
// both numbers that an element of h is made of.
#include <type_traits>
#include "experts.h"
#include "fp6_pack.h"
#include "quant_pass.h"

namespace dfp4 {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kFmtFp6 = 2;                       // E2M3

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

struct PackArgs {
    const uint8_t *codes[2], *dial[2], *expo[2];
    Packed to;
    int rows, KB, S, gated;
};

// One wave per (tile, step); lane (kh, c) takes row c of the tile, block 2 step + kh.  What is not there is zeros.
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

// ---- products

struct ProductArgs {
    Packed a, w;
    const int32_t* used;
    const PlanGroup* plan;
    void* out;                                   // up: bf16 [row][rows / 2], down: f32 [row][rows]
    int64_t groups;                              // at most
    int S, rows, tiles, row_tiles;               // of an expert: packed rows, tiles of 32 with padding, tiles that have rows
};

__device__ __forceinline__ uint16_t bf16_of(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float silu_times(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

// 32 rows x 32 packed rows of weights a workgroup; its 16 waves share K and add their sums in a fixed order through LDS.
template <bool GATED>
__global__ __launch_bounds__(1024, 4) void experts_kernel(ProductArgs p) {
    __shared__ float s_red[8][16][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int S = p.S, per = (S + 15) / 16, s_lo = min(S, wave * per), s_hi = min(S, s_lo + per);
    const int64_t used = min((int64_t)*p.used, p.groups), total = used * 8 * p.row_tiles;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
        const int64_t eighth = id / p.row_tiles;
        const PlanGroup group = p.plan[eighth >> 3];
        const int t = (int)(id - eighth * p.row_tiles), skip = (int)(eighth & 7) * 32, rows = min(32, group.rows - skip);
        if (rows <= 0) continue;
        const int64_t row0 = (int64_t)group.row0 + skip;
        const size_t a_tile = (size_t)eighth, w_tile = (size_t)group.expert * p.tiles + t;
        v16f acc;
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[x] = 0.0f;
        for (int s = s_lo; s < s_hi; ++s) {
            const uint4 alo = *reinterpret_cast<const uint4*>(p.a.bits + fp6_lo(a_tile, s, S) + lane * 16);
            const uint2 ahi = *reinterpret_cast<const uint2*>(p.a.bits + fp6_hi(a_tile, s, S) + fp6_hi_lane(lane) * 8);
            const uint4 wlo = *reinterpret_cast<const uint4*>(p.w.bits + fp6_lo(w_tile, s, S) + lane * 16);
            const uint2 whi = *reinterpret_cast<const uint2*>(p.w.bits + fp6_hi(w_tile, s, S) + fp6_hi_lane(lane) * 8);
            const int as = p.a.scales[scale_at(a_tile, s, S) + lane * 4], ws = p.w.scales[scale_at(w_tile, s, S) + lane * 4];
            const v8i a = {(int)alo.x, (int)alo.y, (int)alo.z, (int)alo.w, (int)ahi.x, (int)ahi.y, 0, 0};
            const v8i w = {(int)wlo.x, (int)wlo.y, (int)wlo.z, (int)wlo.w, (int)whi.x, (int)whi.y, 0, 0};
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, acc, kFmtFp6, kFmtFp6, 0, ws, 0, as);
        }
        __syncthreads();                                       // the sums of the round before are read
        if (wave >= 8) {
#pragma unroll
            for (int x = 0; x < 16; ++x) s_red[wave - 8][x][lane] = acc[x];
        }
        __syncthreads();
        if (wave < 8) {
#pragma unroll
            for (int x = 0; x < 16; ++x) s_red[wave][x][lane] += acc[x];
        }
        __syncthreads();
        // register x of lane (h, c): packed row 8 (x / 4) + 4 h + x % 4, row c
        const int c = lane & 31, h = lane >> 5;
        auto sum = [&](int x) {
            float v = 0.0f;
#pragma unroll
            for (int w8 = 0; w8 < 8; ++w8) v += s_red[w8][x][lane];
            return v;
        };
        if constexpr (GATED) {
            const int x = 2 * wave, n = t * 32 + 8 * (x >> 2) + 4 * h + (x & 3);
            if (wave < 8 && c < rows && n < p.rows)
                static_cast<uint16_t*>(p.out)[(row0 + c) * (p.rows >> 1) + (n >> 1)] = bf16_of(silu_times(sum(x), sum(x + 1)));
        } else {
            const int x = wave, n = t * 32 + 8 * (x >> 2) + 4 * h + (x & 3);
            if (c < rows && n < p.rows) static_cast<float*>(p.out)[(row0 + c) * p.rows + n] = sum(x);
        }
    }
}

struct JoinArgs {
    const void* part;
    const float* weights;
    const int32_t* place;
    void* y;
    int64_t tokens, pairs;
    int k, dim;
};

// y[token] = sum over j of weights[token, j] * part[place], four elements a thread; PART16: part in bf16
template <bool BF16, bool PART16>
__global__ __launch_bounds__(256) void experts_join_kernel(JoinArgs p) {
    const int64_t quads = p.dim / 4, total = p.tokens * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t token = i / quads, d = (i - token * quads) * 4;
        float4 y = make_float4(0, 0, 0, 0);
        for (int j = 0; j < p.k; ++j) {
            const int32_t row = p.place[token * p.k + j];
            if (row < 0 || row >= p.pairs) continue;
            const float w = p.weights[token * p.k + j];
            float4 v;
            if constexpr (PART16) {
                const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.part) + (int64_t)row * p.dim + d);
                v = make_float4(as_f(u.x << 16), as_f(u.x & 0xffff0000u), as_f(u.y << 16), as_f(u.y & 0xffff0000u));
            } else {
                v = *reinterpret_cast<const float4*>(static_cast<const float*>(p.part) + (int64_t)row * p.dim + d);
            }
            y.x += w * v.x, y.y += w * v.y, y.z += w * v.z, y.w += w * v.w;
        }
        if constexpr (BF16)
            *reinterpret_cast<ushort4*>(static_cast<uint16_t*>(p.y) + token * p.dim + d) = make_ushort4(bf16_of(y.x), bf16_of(y.y), bf16_of(y.z), bf16_of(y.w));
        else
            *reinterpret_cast<float4*>(static_cast<float*>(p.y) + token * p.dim + d) = y;
    }
}

// workspace: rows in operand order, and down their products
struct Workspace {
    int64_t rows, part, total;
};
inline Workspace workspace_of(const dfp4_plan& plan, const dfp4_experts& w) {
    const int64_t pairs = plan.tokens * plan.k;
    Workspace x{};
    x.rows = plan_groups(pairs, plan.experts) * kGroupRows;
    x.part = up256((int64_t)native_packed_bytes(x.rows, w.K, true));
    x.total = x.part + (w.gated ? 0 : up256(pairs * w.rows * 4));
    return x;
}

}  // namespace

size_t expert_weights_bytes(int64_t experts, int64_t rows, int64_t K, bool gated) {
    const dfp4_experts w{nullptr, experts, rows, K, gated ? 1 : 0};
    return native_packed_bytes(experts * padded_rows(w), K, true);
}

int launch_expert_weights(dfp4_tensor gate, dfp4_tensor up, const dfp4_experts& w, hipStream_t stream) {
    PackArgs p{};
    p.codes[0] = gate.codes, p.dial[0] = gate.dialect, p.expo[0] = gate.exponent;
    p.codes[1] = up.codes, p.dial[1] = up.dialect, p.expo[1] = up.exponent;
    p.to = packed_at(w.packed, w.experts * padded_rows(w), w.K);
    p.rows = (int)w.rows, p.KB = (int)(w.K / kBlock), p.S = (int)steps_of(w.K), p.gated = w.gated ? 1 : 0;
    const dim3 grid((unsigned)((p.S + 3) / 4), (unsigned)(padded_rows(w) / 32), (unsigned)w.experts);
    hipLaunchKernelGGL(experts_pack_kernel, grid, dim3(256), 0, stream, p);
    return check_launch();
}

size_t experts_workspace_bytes(const dfp4_plan& plan, const dfp4_experts& w) { return (size_t)workspace_of(plan, w).total; }

int launch_experts(const ExpertsArgs& a, hipStream_t stream) {
    const int64_t pairs = a.plan.tokens * a.plan.k, S = steps_of(a.w.K);
    const Workspace ws = workspace_of(a.plan, a.w);
    const PlanView plan = plan_view(a.plan);
    const int cus = device_cu_count();
    QuantizeArgs q{};
    q.x = a.x, q.ld = a.ld;
    q.rows = plan.offsets + a.plan.experts, q.order = plan.order, q.row_at = plan.row_at;
    q.to = packed_at(a.workspace, ws.rows, a.w.K);
    q.k = a.w.gated ? (uint32_t)a.plan.k : 0, q.KB = (uint32_t)(a.w.K / kBlock), q.S = (uint32_t)S;
    q.bound = pairs;
    const int64_t units = (pairs + 7) / 8 * ((S + 3) / 4), want = (units + kQWaves - 1) / kQWaves;
    hipLaunchKernelGGL(experts_quantize_kernel, dim3((unsigned)(want < 8 * cus ? want : 8 * cus)), dim3(kQThreads), 0, stream, q);
    ProductArgs p{};
    p.a = q.to;
    p.w = packed_at(a.w.packed, a.w.experts * padded_rows(a.w), a.w.K);
    p.used = plan.used, p.plan = plan.groups;
    p.out = a.w.gated ? a.out : a.workspace + ws.part;
    p.groups = plan_groups(pairs, a.plan.experts);
    p.S = (int)S, p.rows = (int)expert_rows(a.w), p.tiles = (int)(padded_rows(a.w) / 32), p.row_tiles = (p.rows + 31) / 32;
    const bool many = pairs >= 64 * a.w.experts, part16 = many && a.out_dtype == DFP4_BF16;
    if (many) {
        ExpertTiles t{};
        t.a = q.to.bits, t.a_scales = native_scale_offset(ws.rows, a.w.K, true);
        t.w = a.w.packed, t.w_scales = native_scale_offset(a.w.experts * padded_rows(a.w), a.w.K, true);
        t.used = plan.used, t.groups = plan.groups, t.max_groups = p.groups;
        t.K = (int)a.w.K, t.rows = p.rows, t.tiles = p.tiles / 8;
        t.gated = a.w.gated != 0, t.half = false;
        t.out = p.out, t.out_dtype = a.out_dtype;
        const int rc = launch_expert_tiles(t, stream);
        if (rc != DFP4_OK) return rc;
    } else {
        const int64_t all = p.groups * 8 * p.row_tiles;
        const dim3 grid((unsigned)(all < (1 << 20) ? all : 1 << 20));
        if (a.w.gated) hipLaunchKernelGGL((experts_kernel<true>), grid, dim3(1024), 0, stream, p);
        else hipLaunchKernelGGL((experts_kernel<false>), grid, dim3(1024), 0, stream, p);
    }
    if (!a.w.gated) {
        const JoinArgs j{p.out, a.weights, plan.place, a.out, a.plan.tokens, pairs, (int)a.plan.k, (int)a.w.rows};
        const int64_t wgs = (a.plan.tokens * (a.w.rows / 4) + 255) / 256;
        const dim3 jg((unsigned)(wgs < (1 << 20) ? wgs : 1 << 20));
        if (part16) hipLaunchKernelGGL((experts_join_kernel<true, true>), jg, dim3(256), 0, stream, j);
        else if (a.out_dtype == DFP4_BF16) hipLaunchKernelGGL((experts_join_kernel<true, false>), jg, dim3(256), 0, stream, j);
        else hipLaunchKernelGGL((experts_join_kernel<false, false>), jg, dim3(256), 0, stream, j);
    }
    return check_launch();
}

}  // namespace dfp4
