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

// Groups that `pairs` rows of `experts` experts can take, at most
__host__ __device__ inline int64_t plan_groups(int64_t pairs, int64_t experts) { return pairs / kGroupRows + (pairs < experts ? pairs : experts); }

struct PlanGroup {
    int32_t expert, row0, rows, none;      // rows 0: behind the last group
};
// Arrays of a plan, one after the other (the first three are public)
struct PlanView {
    int32_t* offsets;        // [experts + 1]
    int32_t* order;          // [pairs] pair of a row, -1 behind the last
    int32_t* place;          // [pairs] row of a pair, -1: none
    int32_t* row_at;         // [pairs] group * kGroupRows + row in it, of a row
    int32_t* used;           // [1] groups
    PlanGroup* groups;       // 16-byte aligned
};
__host__ __device__ inline int64_t plan_groups_at(int64_t pairs, int64_t experts) { return (experts + 1 + 3 * pairs + 1 + 3) / 4 * 4; }
inline PlanView plan_view(const dfp4_plan& p) {
    const int64_t pairs = p.tokens * p.k;
    PlanView v;
    v.offsets = p.data;
    v.order = v.offsets + p.experts + 1;
    v.place = v.order + pairs;
    v.row_at = v.place + pairs;
    v.used = v.row_at + pairs;
    v.groups = reinterpret_cast<PlanGroup*>(p.data + plan_groups_at(pairs, p.experts));
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
    const int32_t* used;
    const PlanGroup* groups;
    int64_t max_groups;
    int K, rows, tiles;      // packed rows of an expert, tiles of 256 of them
    bool gated, half;        // half: tiles of 128 rows
    void* out;               // gated: bf16 [row][rows / 2], else [row][rows] of out_dtype
    int out_dtype;
};
int launch_expert_tiles(const ExpertTiles& t, hipStream_t stream);

int launch_route(const RouteArgs& a, hipStream_t stream);
int launch_expert_plan(const int32_t* ids, const dfp4_plan& plan, hipStream_t stream);
int launch_add_norm(const AddNormArgs& a, hipStream_t stream);
size_t expert_weights_bytes(int64_t experts, int64_t rows, int64_t K, bool gated);
int launch_expert_weights(dfp4_tensor gate, dfp4_tensor up, const dfp4_experts& w, hipStream_t stream);
size_t experts_workspace_bytes(const dfp4_plan& plan, const dfp4_experts& w);
int launch_experts(const ExpertsArgs& a, hipStream_t stream);

}  // namespace dfp4
