// Operators of a sparse layer (include/dfp4.h): the plan's layout, arguments of the launchers.
#pragma once
#include "common.h"

namespace dfp4 {

constexpr int kMaxExperts = 1024;
constexpr int kMaxChoice = 32;                        // experts of a token
constexpr int64_t kMaxPairs = (int64_t)1 << 27;
// Rows of the products come in groups: an expert's rows begin with a group, so that a group has one expert.  256 rows are the largest
// tile of the products.
constexpr int kGroupRows = 256;

// Rows of an expert, from the plan's row `row0` on; `at`: its first row among the padded ones
struct PlanGroup {
    int32_t expert, row0, rows, at;
};
// Three lists of them: groups, halves of 128 rows and, for products of few rows, blocks of 64; only what has rows
constexpr int kListRows[3] = {kGroupRows, 128, 64};
__host__ __device__ inline int64_t plan_list(int64_t pairs, int64_t experts, int list) { return pairs / kListRows[list] + (pairs < experts ? pairs : experts); }
// The plan is made by up to 64 workgroups of shares of the pairs, each a multiple of 1024: one up to 2048 pairs
inline int64_t plan_share(int64_t pairs) { return pairs <= 2048 ? 2048 : ((pairs + 63) / 64 + 1023) / 1024 * 1024; }
inline int64_t plan_shares(int64_t pairs) { return pairs <= 0 ? 1 : (pairs + plan_share(pairs) - 1) / plan_share(pairs); }
// Arrays of a plan, one after the other (the first three are public)
struct PlanView {
    int32_t* offsets;        // [experts + 1]
    int32_t* order;          // [pairs] pair of a row, -1 behind the last
    int32_t* place;          // [pairs] row of a pair, -1: none
    int32_t* row_at;         // [pairs] group * kGroupRows + row in it, of a row
    int32_t* expert;         // [pairs] of a pair, -1: none
    int32_t* used;           // [3] of each list
    PlanGroup* list[3];      // 16-byte aligned
    int32_t* counts;         // [shares][experts], where there are several
};
struct PlanSizes {
    int64_t list_at[3], counts_at, total;      // int32
};
inline PlanSizes plan_sizes(int64_t pairs, int64_t experts) {
    PlanSizes s;
    s.counts_at = (experts + 1 + 4 * pairs + 3 + 3) / 4 * 4;
    for (int q = 0; q < 3; ++q) {
        s.list_at[q] = s.counts_at;
        s.counts_at += 4 * plan_list(pairs, experts, q);
    }
    s.total = s.counts_at + (plan_shares(pairs) > 1 ? plan_shares(pairs) * experts : 0);
    return s;
}
inline PlanView plan_view(const dfp4_plan& p) {
    const int64_t pairs = p.tokens * p.k;
    const PlanSizes s = plan_sizes(pairs, p.experts);
    PlanView v;
    v.offsets = p.data;
    v.order = v.offsets + p.experts + 1;
    v.place = v.order + pairs;
    v.row_at = v.place + pairs;
    v.expert = v.row_at + pairs;
    v.used = v.expert + pairs;
    for (int q = 0; q < 3; ++q) v.list[q] = reinterpret_cast<PlanGroup*>(p.data + s.list_at[q]);
    v.counts = p.data + s.counts_at;
    return v;
}

struct RouteArgs {
    const void* logits;
    const float* bias;
    int32_t* ids;
    float* weights;
    int64_t ld;
    float scale;
    int tokens, experts, k, groups, kept, best;
    bool bf16, sigmoid, renormalize;
};

struct AddNormArgs {
    const uint16_t* y;
    const void* residual;
    void* residual_out;
    const uint16_t* gate;
    const float *post, *weight;
    uint16_t* normed;
    int64_t y_ld, residual_ld, gate_ld;
    float scale, eps;
    int64_t tokens;
    int dim;
    bool wide;               // the residual in f32
};

// silu(g) * u by the hardware's exponential and reciprocal (1 ulp each; the rounding of the exponent is 2^-23 |g| of the result for negative g,
// far below a rounding to bf16): six instructions, where a division in full would take ten more, in an epilogue that nothing runs beside.
// Behind kFarGate exp(-g) nears the end of fp32, while its product with u need not: there silu(g) is g exp(g), of which exp(g / 2) goes once to g and
// once to u (silu_far).  An element's own gate decides; one form for all (t = exp(-|g| / 2), ten instructions) takes 4096 tokens of 8 of 64
// experts 151.6 instead of 147.3 us.
constexpr float kFarGate = -80.0f;
__device__ __forceinline__ float silu_times(float g, float u) {
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g)) * u;
}
__device__ __forceinline__ float silu_far(float g, float u) {
    const float t = __builtin_amdgcn_exp2f(0.72134752f * g);
    return (g * t) * (u * t);
}

// The way that a product takes (dfp4_experts_way)
enum { kWithin = 0, kBefore = 1, kOnceAToken = 2 };
struct ExpertsWay {
    int rows, waves, quantized;
};

// An experts' product: rows of `x` (up: a token's, down: a pair's) with the experts' matrices
struct ExpertsArgs {
    const uint16_t* x;
    int64_t ld;
    dfp4_plan plan;
    dfp4_experts w;
    void* out;               // up: bf16 [pairs, rows of w]; down: [tokens, rows of w]
    int out_dtype;
    const float* weights;    // down: [tokens, k]
    uint8_t* workspace;
};

// the products of many rows (gemm_native.hip): tiles of 256 or 128 rows of a group and 256 of the weights
struct ExpertTiles {
    const void *a, *w;       // packed rows and weights, and the offsets of their scales
    size_t a_scales, w_scales;
    const int32_t* used;     // of the list that matches `half`
    const PlanGroup* list;
    int64_t most;
    int K, rows, tiles;      // packed rows of an expert, tiles of 256 of them
    bool gated, half;        // half: tiles of 128 rows
    void* out;               // gated: bf16 [row][rows / 2], else f32 [row][rows]
};
int launch_expert_tiles(const ExpertTiles& t, hipStream_t stream);

int launch_route(const RouteArgs& a, hipStream_t stream);
int launch_expert_plan(const int32_t* ids, const dfp4_plan& plan, hipStream_t stream);
int launch_add_norm(const AddNormArgs& a, hipStream_t stream);
size_t expert_weights_bytes(int64_t experts, int64_t rows, int64_t K, bool gated);
int launch_expert_weights(dfp4_tensor gate, dfp4_tensor up, const dfp4_experts& w, hipStream_t stream);
ExpertsWay experts_way(const dfp4_plan& plan, const dfp4_experts& w);
bool experts_fit(const dfp4_plan& plan, const dfp4_experts& w);
size_t experts_workspace_bytes(const dfp4_plan& plan, const dfp4_experts& w);
int launch_experts(const ExpertsArgs& a, hipStream_t stream);

}  // namespace dfp4
