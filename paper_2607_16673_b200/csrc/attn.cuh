// Declarations of the attention-layer kernels: parameter blocks, launchers and the checks they share.
#pragma once

#include "speca_common.cuh"

namespace speca {

constexpr int kAttnMaxTree = 1024;      // nodes of a sequence with a parent array: they are kept in shared memory
constexpr int kAttnMaxChain = 8192;     // nodes of a sequence without one

struct AttnParams {
    int32_t L, B, H, HK, T;
    float scale;
    int32_t max_nodes, page_shift, n_pages, max_pages, max_depth;
    int32_t withhold_first_load;    // failure-detection test: CTA 0 never requests its first keys
    int32_t misplaced;              // failure-detection test: CTAs take their shared memory for misaligned
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16 *k_cache, *v_cache, *o;
    const int32_t *node_offsets, *parent, *page_table, *kv_len, *path_idx, *path_len;
    int32_t *status;
    void *workspace;
};

struct NormParams {
    int64_t q_layer, q_token, k_layer, k_token;      // strides in elements
    const float *q_weight, *k_weight, *inv_freq;
    __nv_bfloat16 *q_out, *k_out;
    float eps, rope_scale;
    int32_t rot, interleaved;
};

size_t attend_workspace_bytes(const speca_attn_dims *d);
void attend_set_withhold(int on);
void attend_set_misplaced(int on);
int launch_attend(const AttnParams &p, int d_head, cudaStream_t st);
int launch_norm_rope(const AttnParams &p, const NormParams &n, int d_head, cudaStream_t st);
int launch_commit_kv(const AttnParams &p, int d_head, int32_t *kv_len_out, cudaStream_t st);
int launch_copy_pages(const AttnParams &p, int d_head, const int32_t *src, const int32_t *dst, int32_t n, cudaStream_t st);

// Packed nodes of sequence b: 0, or the status bit of what is wrong with them.
__device__ __forceinline__ int sequence_nodes(const AttnParams &p, int b, int &base, int &n)
{
    base = p.node_offsets[b];
    const int end = p.node_offsets[b + 1];
    n = end - base;
    // (compared before the difference is trusted: offsets of opposite sign overflow it)
    if (base < 0 || end < base || end > p.T || (b == p.B - 1 && end != p.T) || (b == 0 && base != 0)) return SPECA_STATUS_BAD_OFFSETS;
    return n > p.max_nodes ? SPECA_STATUS_TOO_MANY : 0;
}

}  // namespace speca
