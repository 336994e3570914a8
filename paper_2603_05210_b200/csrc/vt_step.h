// A draft layer's decode step: host side of rotary positions, tree attention and verification (vt_rope.cu, vt_attn.cu,
// vt_verify.cu).
#pragma once

#include "vt_launch.h"

namespace vt {

constexpr unsigned int kStatusPage = 2u;       // status word, beside kStatusTimeout: a page id outside the cache was met

constexpr int kVerifyMaxTokens = 1024;
constexpr int kVerifyMaxV = 4 << 20, kVerifyMaxVDrawn = 384 << 10;

vt_status launch_rope_table(uint64_t* table, int rot_dim, double base, int scaling, double factor, double low, double high, double original_len,
                            cudaStream_t st);

// After validation.  cache null: k goes to k_out and there is no v.
struct RopeCall {
    vt_heads q, k, v, q_out, k_out;
    const int32_t *positions, *cu_tokens;
    const uint64_t* table;
    int N, Hq, Hkv, D, rot_dim;
    float amplitude;
    int options;
    const vt_cache* cache;
};
vt_status launch_rope(const RopeCall& c, cudaStream_t st);

vt_status launch_tree_mask(const int32_t* parents, const int32_t* cu_tokens, const int32_t* lens, int N, int B, int32_t* mask, int mask_words,
                           int32_t* positions, cudaStream_t st);

struct AttnCall {
    vt_heads q, out;
    const int32_t *cu_tokens, *mask;
    const vt_cache* cache;
    float* lse;
    int mask_words, N, Hq, max_tokens;
    float scale;
};
size_t attn_workspace_bytes(int Hq, int heads, int D, int max_tokens);
vt_status launch_attn(const AttnCall& c, void* workspace, cudaStream_t st);

struct VerifyCall {
    const float *probs, *u_accept, *u_sample, *draft_probs;
    const int32_t *tokens, *parents, *cu_tokens, *draft_ids, *d2t;
    int64_t ld_probs, ld_draft;
    int N, B, V, Vd, max_tokens;
    int32_t *n_accepted, *path, *out_tokens;
};
vt_status launch_verify(const VerifyCall& c, cudaStream_t st);

#ifdef __CUDACC__
// The request that token n belongs to: the last b with cu[b] <= n.  -1 for a token outside all of them.  Whatever cu holds, the
// answer is -1 or lies in [0, B).
__device__ __forceinline__ int request_of(const int32_t* cu, int B, int n) {
    int lo = 0, hi = B;                          // cu[lo] <= n < cu[hi], if at all
    if (n < cu[0] || n >= cu[B]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= n) lo = mid;
        else hi = mid;
    }
    return lo;
}
// Its first token, as the attention and the verification take it: whatever cu holds, no earlier one than 0.
__device__ __forceinline__ int first_of(const int32_t* cu, int b) { return max(cu[b], 0); }
#endif

}  // namespace vt
