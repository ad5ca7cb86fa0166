// Operators of a sparse layer (include/dfp4.h): the plan's layout, arguments of the launchers.
#pragma once
#include "common.h"

namespace dfp4 {

constexpr int kMaxExperts = 1024;
constexpr int kMaxChoice = 32;                        // experts of a token
constexpr int64_t kMaxPairs = (int64_t)1 << 27;
// Rows of the products come in groups: an expert's rows begin with a group, so that a group has one expert.  128 rows share the scale
// dwords of a packed operand.
constexpr int kGroupRows = 128;

// Groups that `pairs` rows of `experts` experts can take, at most
__host__ __device__ inline int64_t plan_groups(int64_t pairs, int64_t experts) { return pairs / kGroupRows + (pairs < experts ? pairs : experts); }

// int32 arrays of a plan, one after the other (the first three are public)
struct PlanView {
    int32_t* offsets;        // [experts + 1]
    int32_t* order;          // [pairs] pair of a row, -1 behind the last
    int32_t* place;          // [pairs] row of a pair, -1: none
    int32_t* first_group;    // [experts + 1]
    int32_t* group_expert;   // [groups] -1 behind the last
    int32_t* row_at;         // [pairs] group * kGroupRows + row in it, of a row
};
inline PlanView plan_view(const dfp4_plan& p) {
    const int64_t pairs = p.tokens * p.k;
    PlanView v;
    v.offsets = p.data;
    v.order = v.offsets + p.experts + 1;
    v.place = v.order + pairs;
    v.first_group = v.place + pairs;
    v.group_expert = v.first_group + p.experts + 1;
    v.row_at = v.group_expert + plan_groups(pairs, p.experts);
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

int launch_route(const RouteArgs& a, hipStream_t stream);
int launch_expert_plan(const int32_t* ids, const dfp4_plan& plan, hipStream_t stream);
int launch_add_norm(const AddNormArgs& a, hipStream_t stream);
size_t expert_weights_bytes(int64_t experts, int64_t rows, int64_t K, bool gated);
int launch_expert_weights(dfp4_tensor gate, dfp4_tensor up, const dfp4_experts& w, hipStream_t stream);
size_t experts_workspace_bytes(const dfp4_plan& plan, const dfp4_experts& w);
int launch_experts(const ExpertsArgs& a, hipStream_t stream);

}  // namespace dfp4
