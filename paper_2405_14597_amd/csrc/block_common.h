// Interface of the kernels between a block's projections: per-head norm and rotation (qk_norm_rope.hip), attention over
// packed sequences (attention.hip), low-rank adapters beside a projection (lora.hip).
#pragma once
#include "is_common.h"

namespace intscale {

// Rows of heads: head h of row m at base + m * ld + h * head_dim.
struct RopeArgs {
    const __half *q, *k, *v;         // v may be nullptr
    const __half *gamma_q, *gamma_k; // [head_dim], or nullptr: no norm
    const float* inv_freq;           // [rot_dim / 2]
    const int32_t* positions;        // [M]
    const int64_t* kv_rows;          // [M] row of k_out / v_out, or nullptr: row m
    __half *q_out, *k_out, *v_out;
    long long ldq, ldk, ldv, ldqo, ldko, ldvo;  // elements
    long long cache_rows;            // rows of k_out / v_out
    int M, heads_q, heads_k, head_dim, rot_dim;
    float eps;
    bool interleaved;
};
hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream);

struct AttnArgs {
    const __half *q, *k, *v;
    __half* out;
    long long ldq, ldk, ldv, ldo;    // elements
    const int32_t* q_offsets;        // [seqs + 1]
    const int64_t* kv_starts;        // [seqs], or nullptr: q_offsets
    const int32_t* kv_lens;          // [seqs], or nullptr: the lengths of q
    long long kv_rows;               // rows of k and v
    int M, seqs, max_q, max_kv;
    int heads_kv, group;             // query heads = heads_kv * group
    float scale;
    bool causal;
    // set by the launcher
    int few_rows = 0;                // sequences of no more packed rows (rows * group) take the kernel for few rows
    int slots = 0, least_tiles = 0;  // its workgroups for each key head, and the fewest tiles of one
    float* few_o = nullptr;          // [slot][2][key head][few_rows][head_dim], unnormalised
    float2* few_ml = nullptr;        // [slot][2][key head][few_rows]: maximum (in powers of two) and sum
    int tile_chunk = 0;              // keys of a row tile's workgroup
    float* part_o = nullptr;         // [chunk index][M * query heads][head_dim]
    float2* part_ml = nullptr;       // [chunk index][M * query heads]
};
struct AttnPlan {
    bool tiles = false;              // sequences of more than few_rows packed rows are expected
    int tile_chunk = 0, tile_chunks = 1;  // keys of a row tile's workgroup, chunks of the longest sequence
    int few_rows = 0;                // 0: the kernel for few rows is not launched
    int slots = 0, least_tiles = 0;
    bool few_cut = false;            // a sequence may lie in several workgroups' runs
};
AttnPlan attention_plan(int M, int seqs, int max_q, int max_kv, int heads_kv, int group, int head_dim, bool own_lens);
size_t attention_workspace_bytes(const AttnPlan& p, int M, int heads_kv, int group, int head_dim);
hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, int head_dim, void* workspace, hipStream_t stream);

struct LoraArgs {
    const __half *x, *a, *b, *base;  // x [M,K], a [adapters,R,K], b [adapters,N,R]; base [M,N], may be out, may be nullptr
    const int32_t* row_adapter;      // [M]
    const float* scales;             // [adapters], or nullptr
    const int32_t* ranks;            // [adapters], or nullptr
    __half* out;                     // [M,N]
    long long ldx, ldb, ldo;         // elements; ldb: base's
    int M, N, K, R, adapters;
    float* inner = nullptr;          // workspace: [slab][M][R] sums of x a^T over a slab of K
    int slabs = 1;
};
size_t lora_workspace_bytes(int M, int N, int K, int R);
hipError_t launch_lora_add(const LoraArgs& a, void* workspace, hipStream_t stream);

}  // namespace intscale
