// Gradient of token scoring (vt_score.cu).  With p = e^(z - lse) and upstream gradients gl of the log probability and ge of
// the entropy,
//
//   G[m, v] = scale * ( gl_m (1[v = t_m] - p) - ge_m p (log p + H_m) )      dh = G W      dW = G^T h
//
// The logits are multiplied out again (the forward pass wrote none) and turned into G on the way out of tensor memory;
// G goes to memory once, in bf16, because it is an operand of both remaining products - the one rounding in between.
// Rows that are not scored have G = 0 and, so that nothing in their hidden state can reach dW (0 * NaN is NaN), the
// product for dW reads a copy of h in which they are zero.
#include "vt_score.h"

#include "vt_gemm.cuh"

namespace vt {

struct EpiScoreGrad {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        const int32_t* tokens;
        const float *lse, *entropy, *grad_logprobs, *grad_entropy;
        uint16_t* G;
        int64_t ldg;
        float scale;
        int V;
    };
    struct State {
        float lse, H, gl, ge;
        int tok;
    };
    static __device__ __forceinline__ void row(State& st, const Params& ep, const GemmProblem&, int m) {
        st.tok = (unsigned)ep.tokens[m] < (unsigned)ep.V ? ep.tokens[m] : -1;
        st.lse = ep.lse[m];
        st.gl = ep.scale * ep.grad_logprobs[m];
        st.ge = ep.grad_entropy ? ep.scale * ep.grad_entropy[m] : 0.0f;
        st.H = ep.grad_entropy ? ep.entropy[m] : 0.0f;
    }
    static __device__ __forceinline__ void ahead(State&, const Params&, const GemmProblem&, int, int, int) {}
    static __device__ __forceinline__ void cols8(State& st, const Params& ep, const GemmProblem&, int, int n, int, const float (&x)[8],
                                                 const float (&)[8], float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float logp = fmaf(ep.scale, x[i], -st.lse);
            const float p = ex2_approx(logp * kLog2e);
            float g = -p * fmaf(st.ge, logp + st.H, st.gl);
            if (n + i == st.tok) g += st.gl;
            out[0][i] = st.tok < 0 ? 0.0f : g;
        }
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem&, int, int, int m, int n) { return ep.G + (size_t)m * ep.ldg + n; }
    static __device__ __forceinline__ int64_t ld(const Params& ep, const GemmProblem&, int) { return ep.ldg; }
};

// The hidden states with the rows that are not scored set to zero.  Bound by its bytes: 4 d per row.
__global__ void __launch_bounds__(256) score_rows_kernel(const uint16_t* h, int64_t ldh, const int32_t* tokens, int M, int d, int V, uint16_t* out) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int per_row = d >> 3;
    const long long n = (long long)M * per_row;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const int m = (int)(i / per_row), c = (int)(i - (long long)m * per_row);
        uint4 v = make_uint4(0, 0, 0, 0);
        if ((unsigned)tokens[m] < (unsigned)V) v = *reinterpret_cast<const uint4*>(h + m * ldh + 8 * c);
        *reinterpret_cast<uint4*>(out + (size_t)m * d + 8 * c) = v;
    }
}

// G's rows: whole 16-byte runs of columns, so that a tensor map can read them
static int64_t grad_ld(int V) { return (int64_t)round_up((size_t)V, 64); }

size_t score_backward_workspace_bytes(int M, int d, int V) {
    return kHeaderBytes + round_up((size_t)M * grad_ld(V) * 2, 256) + round_up((size_t)M * d * 2, 256);
}

vt_status launch_score_backward(const ScoreCall& c, const float* lse, const float* entropy, const float* grad_logprobs,
                                const float* grad_entropy, void* grad_h, void* grad_W, void* workspace, cudaStream_t st) {
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    WsHeader* hdr = reinterpret_cast<WsHeader*>(base);
    const int64_t ld = grad_ld(c.V);
    uint16_t* G = reinterpret_cast<uint16_t*>(base + kHeaderBytes);
    uint16_t* h0 = reinterpret_cast<uint16_t*>(base + kHeaderBytes + round_up((size_t)c.M * ld * 2, 256));
    const GemmOperand W{c.W, c.V, c.d, c.d}, g{G, c.M, c.V, ld};
    vt_status r;
    if (grad_W) {   // h without the rows that are not scored
        const long long n = (long long)c.M * (c.d >> 3);
        const int grid = (int)std::min<long long>((n + 255) / 256, 8 * kGemmSms);
        cudaError_t e = launch_pdl(score_rows_kernel, grid, 256, 0, st, reinterpret_cast<const uint16_t*>(c.h), c.ldh, c.tokens,
                                   c.M, c.d, c.V, h0);
        count_launch();
        if (e == cudaSuccess) e = cudaGetLastError();
        if (e != cudaSuccess) return cuda_fail(e);
    }
    {   // G: [M, V], summed over d
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        // columns in runs of eight: the last run may reach into the rows' padding, which nobody reads
        p.prob[0].M = c.M;
        p.prob[0].N = (int)round_up((size_t)c.V, 8);
        p.prob[0].b0 = 1;
        p.prob[0].nk0 = ceil_div(c.d, kBoxK);
        p.hdr = hdr;
        if (!gemm_plan(&p, false, false, false, EpiScoreGrad::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], GemmOperand{c.h, c.M, c.d, c.ldh}, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], W, gemm_box_b(p, false, pair))) != VT_OK) return r;
        const EpiScoreGrad::Params ep{c.tokens, lse, entropy, grad_logprobs, grad_entropy, G, ld, c.scale, c.V};
        if ((r = gemm_launch<false, false, EpiScoreGrad>(maps, p, pair, ep, st)) != VT_OK) return r;
    }
    if (grad_h) {   // dh = G W: [M, d], summed over the vocabulary; W has d running fastest
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        p.prob[0].M = c.M;
        p.prob[0].N = c.d;
        p.prob[0].b0 = 1;
        p.prob[0].nk0 = ceil_div(c.V, kBoxK);
        p.b_early = 1;
        p.hdr = hdr;
        if (!gemm_plan(&p, false, true, false, EpiStore::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], g, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], W, gemm_box_b(p, true, pair))) != VT_OK) return r;
        if ((r = gemm_store(maps, p, pair, false, true, &grad_h, st)) != VT_OK) return r;
    }
    if (!grad_W) return VT_OK;
    // dW = G^T h: [V, d], summed over the M rows
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    p.n_prob = 1;
    p.prob[0].M = c.V;
    p.prob[0].N = c.d;
    p.prob[0].b0 = 1;
    p.prob[0].nk0 = ceil_div(c.M, kBoxK);
    p.hdr = hdr;
    if (!gemm_plan(&p, true, true, false, EpiStore::kScratch, &pair)) return VT_ERR_SHAPE;
    if ((r = gemm_map(&maps.map[0], g, gemm_box_a(p, true))) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], GemmOperand{h0, c.M, c.d, c.d}, gemm_box_b(p, true, pair))) != VT_OK) return r;
    return gemm_store(maps, p, pair, true, true, &grad_W, st);
}

}  // namespace vt
