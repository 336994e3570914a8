// Gradient of token scoring (vt_score.cu).  With p = e^(z - lse) and upstream gradients gl of the log probability and ge of
// the entropy,
//
//   G[m, v] = scale * ( gl_m (1[v = t_m] - p) - ge_m p (log p + H_m) )      dh = G W      dW = G^T h
//
// The logits are multiplied out again (the forward pass wrote none) and turned into G on the way out of tensor memory;
// G goes to memory once, in bf16, because it is an operand of both remaining products - the one rounding in between.
// Nearly all of a row of G that is not next to nothing is one entry, the given token's, so that entry's rounding moves a whole
// row of dh, and of dW, by up to 2^-8 of itself; with few rows the result's error was 1.4 to 1.6 times that of one rounding.
// What the rounding took from that entry is therefore kept in fp32 and given back before the products are rounded: times its
// row of W to dh, times its row of h to its token's row of dW (error now 1.00 to 1.07 times that of one rounding).  For dW that
// is a kernel of its own over the rows of the given tokens, whose sums the product leaves in fp32: added in the product's
// epilogue, the rows of h held every tile up.  255 rows, 13264 x 2048, forward and backward: 81.6 us without any of it, 88.2
// this way, 101 in the epilogue; 4096 rows, 32000 x 4096: 0 to 3 % on 2700.
// Rows that are not scored have G = 0 and, so that nothing in their hidden state can reach dW (0 * NaN is NaN), the
// product for dW reads a copy of h in which they are zero.
#include <climits>

#include "vt_score.h"

#include "vt_gemm.cuh"

namespace vt {

constexpr int kNone = INT_MAX;

struct EpiScoreGrad {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = false;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        const int32_t* tokens;
        const float *lse, *entropy, *grad_logprobs, *grad_entropy;
        uint16_t* G;
        float* rest;            // [M] what rounding the given token's entry left over
        int32_t* first;         // per token: the first row it was given to, or kNone; null when nobody asks
        int32_t* count;         // per token: the rows it was given to
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
    static __device__ __forceinline__ void cols8(State& st, const Params& ep, const GemmProblem& q, int m, int n, int, const float (&x)[8],
                                                 const float (&)[8], float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float logp = fmaf(ep.scale, x[i], -st.lse);
            const float p = ex2_approx(logp * kLog2e);
            const float g = -p * fmaf(st.ge, logp + st.H, st.gl);
            out[0][i] = st.tok < 0 ? 0.0f : g;
        }
        // one test for the eight: a branch in every column kept them from being worked on side by side (+2 us of 21)
        if ((unsigned)(st.tok - n) < 8u && m < q.M) {
            float rest = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n + i == st.tok) {
                    out[0][i] += st.gl;
                    rest = out[0][i] - __bfloat162float(__float2bfloat16_rn(out[0][i]));
                }
            ep.rest[m] = rest;
            if (ep.first) {
                atomicMin(ep.first + st.tok, m);
                atomicAdd(ep.count + st.tok, 1);
            }
        }
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem&, int, int, int m, int n) { return ep.G + (size_t)m * ep.ldg + n; }
    static __device__ __forceinline__ int64_t ld(const Params& ep, const GemmProblem&, int) { return ep.ldg; }
};

// Adds r times eight bf16 values.
__device__ __forceinline__ void add_scaled(float (&out)[8], float r, const uint4& v) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[2 * i] = fmaf(r, __uint_as_float(u[i] << 16), out[2 * i]);
        out[2 * i + 1] = fmaf(r, __uint_as_float(u[i] & 0xFFFF0000u), out[2 * i + 1]);
    }
}

// Stores dh: row m, adding rest[m] W[t_m], which is requested two runs of columns ahead.
struct EpiGradH {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = false;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        uint16_t* out;
        const uint16_t* W;
        const int32_t* tokens;
        const float* rest;
        int V;
    };
    struct State {
        float r;                    // 0: nothing to add
        const uint16_t* src;
        uint4 v[2][2];
    };
    static __device__ __forceinline__ void row(State& st, const Params& ep, const GemmProblem& q, int m) {
        const int tok = ep.tokens[m];
        const bool scored = (unsigned)tok < (unsigned)ep.V;
        st.src = scored ? ep.W + (size_t)tok * q.N : nullptr;
        st.r = scored ? ep.rest[m] : 0.0f;
    }
    static __device__ __forceinline__ void ahead(State& st, const Params&, const GemmProblem& q, int, int n, int slot) {
        if (st.src == nullptr) return;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (n + 8 * i < q.N) st.v[slot][i] = *reinterpret_cast<const uint4*>(st.src + n + 8 * i);
    }
    static __device__ __forceinline__ void cols8(State& st, const Params&, const GemmProblem& q, int m, int n, int e, const float (&x)[8],
                                                 const float (&)[8], float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[0][i] = x[i];
        if (m < q.M && n < q.N && st.r != 0.0f) add_scaled(out[0], st.r, st.v[e >> 4][(e >> 3) & 1]);
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem& q, int, int, int m, int n) { return ep.out + (size_t)m * q.N + n; }
    static __device__ __forceinline__ int64_t ld(const Params&, const GemmProblem& q, int) { return q.N; }
};

// Stores dW; the sums of a token's row also go, in fp32, to row first[token] of `sums`.
struct EpiGradW {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = true;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        uint16_t* out;
        const int32_t* first;
        float* sums;
    };
    struct State {
        int first;
    };
    static __device__ __forceinline__ void row(State& st, const Params& ep, const GemmProblem&, int m) { st.first = ep.first[m]; }
    static __device__ __forceinline__ bool wants(const State& st) { return st.first != kNone; }
    static __device__ __forceinline__ float* sums(const State& st, const Params& ep, const GemmProblem& q) { return ep.sums + (size_t)st.first * q.N; }
    static __device__ __forceinline__ void ahead(State&, const Params&, const GemmProblem&, int, int, int) {}
    static __device__ __forceinline__ void cols8(State&, const Params&, const GemmProblem&, int, int, int, const float (&x)[8], const float (&)[8],
                                                 float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[0][i] = x[i];
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem& q, int, int, int m, int n) { return ep.out + (size_t)m * q.N + n; }
    static __device__ __forceinline__ int64_t ld(const Params&, const GemmProblem& q, int) { return q.N; }
};

// Copies rows of h, zeros in place of those that are not scored, and clears `first` and `count`.
constexpr int kRowThreads = 256;
__global__ void __launch_bounds__(kRowThreads) score_rows_kernel(const uint16_t* h, int64_t ldh, const int32_t* tokens, int d, int V, uint16_t* out,
                                                                 int32_t* first, int32_t* count) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int m = blockIdx.x;
    const bool scored = (unsigned)tokens[m] < (unsigned)V;
    for (int c = threadIdx.x * 8; c < d; c += kRowThreads * 8)
        *reinterpret_cast<uint4*>(out + (size_t)m * d + c) = scored ? *reinterpret_cast<const uint4*>(h + m * ldh + c) : make_uint4(0, 0, 0, 0);
    // in 64 bits: M blocks of 256 threads pass 2^31 from 8388608 rows on
    for (long long v = (long long)m * kRowThreads + threadIdx.x; v < V; v += (long long)gridDim.x * kRowThreads) {
        first[v] = kNone;
        count[v] = 0;
    }
}

// dW's rows of the given tokens once more, for each token v
//   dW[v] = sums[first row of v] + sum of rest[i] h[i] over the rows i whose token is v
// A block per row.  A token of few rows (most have one) is the work of its first row's block, which adds them in their order, a
// thread to eight columns.  The rows of a token with more than wide_from of them share it: each of their blocks takes runs of 64
// columns by its rank among them, 32 rows side by side, joined in a fixed order.  (One block adding all rows one after the other took
// 0.34 us a row and 2048 columns, after everything else: a whole gradient of 4096 rows, 32000 x 4096, took 2.5 ms with tokens all over
// the vocabulary, 3.0 ms with a quarter of the rows on one token and 5.3 ms with all of them; now 2.5 to 2.6 ms, whatever the tokens.)
// Bound by latencies, or by the 8 d bytes a row.  What is added comes from before the product that this waits for, so the
// first columns' share is ready by then.
constexpr int kGivenRows = 2048;            // rows that are searched for a token at a time
constexpr int kWideCols = 64;
__global__ void __launch_bounds__(kRowThreads) score_given_kernel(const uint16_t* h, int64_t ldh, const int32_t* tokens, const float* rest,
                                                                  const int32_t* first, const int32_t* count, const float* sums, int M, int d,
                                                                  int V, int wide_from, uint16_t* dW) {
    constexpr int kWarps = kRowThreads / 32, kRuns = kGivenRows / kRowThreads;
    __shared__ int list[kGivenRows], found[kWarps];
    __shared__ float part[kWarps][kWideCols];
    const int m = blockIdx.x, t = threadIdx.x, warp = t >> 5, lane = t & 31, tok = tokens[m];
    const bool scored = (unsigned)tok < (unsigned)V;
    const int from = scored ? __ldcg(first + tok) : kNone, n = scored ? __ldcg(count + tok) : 0;
    const bool wide = n > wide_from;
    if (!scored || (!wide && from != m)) {
        grid_dependency_wait();
        return;
    }
    // lists the token's rows among [i0, min(i0 + kGivenRows, end)), in order; returns their number
    auto list_rows = [&](int i0, int end) {
        unsigned hit[kRuns];
        int mine = 0;
#pragma unroll
        for (int j = 0; j < kRuns; ++j) {
            const unsigned i = (unsigned)i0 + (unsigned)((warp * kRuns + j) * 32 + lane);
            hit[j] = __ballot_sync(0xFFFFFFFFu, i < (unsigned)end && tokens[i] == tok);
            mine += __popc(hit[j]);
        }
        __syncthreads();                    // whoever still read the last list is done
        if (lane == 0) found[warp] = mine;
        __syncthreads();
        int at = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            at += w < warp ? found[w] : 0;
            all += found[w];
        }
#pragma unroll
        for (int j = 0; j < kRuns; ++j) {
            if (hit[j] >> lane & 1u) list[at + __popc(hit[j] & ((1u << lane) - 1u))] = i0 + (warp * kRuns + j) * 32 + lane;
            at += __popc(hit[j]);
        }
        __syncthreads();
        return all;
    };
    // adds rows list[j0], list[j0 + step], ... below k at columns c .. c + 7 to sum, four of them in flight
    auto add_rows = [&](float (&sum)[8], int j0, int step, int k, int c) {
        for (int j = j0; j < k; j += 4 * step) {
            uint4 v[4];
            float r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const bool is = j + u * step < k;
                const int i = list[is ? j + u * step : j];
                v[u] = *reinterpret_cast<const uint4*>(h + i * ldh + c);
                r[u] = __ldcg(rest + i);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u * step < k) add_scaled(sum, r[u], v[u]);
        }
    };
    auto finish = [&](const float (&sum)[8], int c) {
        const float4* src = reinterpret_cast<const float4*>(sums + (size_t)from * d + c);
        const float4 a = src[0], b = src[1];
        const float all[8] = {sum[0] + a.x, sum[1] + a.y, sum[2] + a.z, sum[3] + a.w, sum[4] + b.x, sum[5] + b.y, sum[6] + b.z, sum[7] + b.w};
        store_bf16x8(dW + (size_t)tok * d + c, all);
    };
    if (!wide) {
        int k = 0;                          // rows listed; all of them fit one list nearly always, and it then serves every run of columns
        for (int c0 = 0; c0 < d; c0 += kRowThreads * 8) {
            const int c = c0 + t * 8;
            float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (n == 1) {
                if (c < d) add_scaled(sum, __ldcg(rest + m), *reinterpret_cast<const uint4*>(h + m * ldh + c));
            } else {
                int left = n;
                for (int i0 = m; left > 0 && i0 < M; i0 += kGivenRows) {
                    if (k < n) k = list_rows(i0, M);
                    if (c < d) add_rows(sum, 0, 1, k, c);
                    left -= k;
                }
            }
            if (c0 == 0) grid_dependency_wait();
            if (c < d) finish(sum, c);
        }
    } else {
        const int runs = (d + kWideCols - 1) / kWideCols;
        int rank = 0;
        for (int i0 = from; i0 < m && rank < runs; i0 += kGivenRows) rank += list_rows(i0, m);
        if (rank >= runs) {
            grid_dependency_wait();
            return;
        }
        for (int run = rank; run < runs; run += n) {
            const int c = run * kWideCols + (lane & 7) * 8;
            float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            int left = n;
            for (int i0 = from; left > 0 && i0 < M; i0 += kGivenRows) {
                const int k = list_rows(i0, M);
                if (c < d) add_rows(sum, warp * 4 + (lane >> 3), kWarps * 4, k, c);
                left -= k;
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 8);
                sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 16);
                if (lane < 8) part[warp][lane * 8 + i] = sum[i];
            }
            __syncthreads();
            if (run == rank) grid_dependency_wait();
            if (t < 8 && c < d) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum[i] = part[0][t * 8 + i];
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) sum[i] += part[w][t * 8 + i];
                }
                finish(sum, c);
            }
            __syncthreads();
        }
    }
    grid_launch_dependents();
}

// G's rows: whole 16-byte runs of columns, so that a tensor map can read them
static int64_t grad_ld(int V) { return (int64_t)round_up((size_t)V, 64); }

// A token with more rows than this is shared among their blocks.  Sharing one searches the rows once per block that takes part: no
// more than 128 tokens are, so that of many rows those searches stay below what the products take.
static int given_wide_from(int M) { return std::max(32, M / 128); }

struct GradSpace {              // offsets in the workspace
    size_t G, h0, rest, first, count, sums, total;
};
static GradSpace grad_space(int M, int d, int V) {
    GradSpace w;
    w.G = kHeaderBytes;
    w.h0 = w.G + round_up((size_t)M * grad_ld(V) * 2, 256);
    w.rest = w.h0 + round_up((size_t)M * d * 2, 256);
    w.first = w.rest + round_up((size_t)M * 4, 256);
    w.count = w.first + round_up((size_t)V * 4, 256);
    w.sums = w.count + round_up((size_t)V * 4, 256);
    w.total = w.sums + round_up((size_t)M * d * 4, 256);
    return w;
}
size_t score_backward_workspace_bytes(int M, int d, int V) { return grad_space(M, d, V).total; }

vt_status launch_score_backward(const ScoreCall& c, const float* lse, const float* entropy, const float* grad_logprobs,
                                const float* grad_entropy, void* grad_h, void* grad_W, void* workspace, cudaStream_t st) {
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    WsHeader* hdr = reinterpret_cast<WsHeader*>(base);
    const int64_t ld = grad_ld(c.V);
    const GradSpace space = grad_space(c.M, c.d, c.V);
    uint16_t* G = reinterpret_cast<uint16_t*>(base + space.G);
    uint16_t* h0 = reinterpret_cast<uint16_t*>(base + space.h0);
    float* rest = reinterpret_cast<float*>(base + space.rest);
    int32_t* first = reinterpret_cast<int32_t*>(base + space.first);
    int32_t* count = reinterpret_cast<int32_t*>(base + space.count);
    float* sums = reinterpret_cast<float*>(base + space.sums);
    const GemmOperand W{c.W, c.V, c.d, c.d}, g{G, c.M, c.V, ld};
    vt_status r;
    if (grad_W) {
        cudaError_t e = launch_pdl(score_rows_kernel, c.M, kRowThreads, 0, st, reinterpret_cast<const uint16_t*>(c.h), c.ldh, c.tokens,
                                   c.d, c.V, h0, first, count);
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
        const EpiScoreGrad::Params ep{c.tokens, lse, entropy, grad_logprobs, grad_entropy, G, rest, grad_W ? first : nullptr, count, ld, c.scale, c.V};
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
        if (!gemm_plan(&p, false, true, false, EpiGradH::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], g, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], W, gemm_box_b(p, true, pair))) != VT_OK) return r;
        const EpiGradH::Params ep{reinterpret_cast<uint16_t*>(grad_h), reinterpret_cast<const uint16_t*>(c.W), c.tokens, rest, c.V};
        if ((r = gemm_launch<false, true, EpiGradH>(maps, p, pair, ep, st)) != VT_OK) return r;
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
    if (!gemm_plan(&p, true, true, false, EpiGradW::kScratch, &pair)) return VT_ERR_SHAPE;
    if ((r = gemm_map(&maps.map[0], g, gemm_box_a(p, true))) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], GemmOperand{h0, c.M, c.d, c.d}, gemm_box_b(p, true, pair))) != VT_OK) return r;
    const EpiGradW::Params ep{reinterpret_cast<uint16_t*>(grad_W), first, sums};
    if ((r = gemm_launch<true, true, EpiGradW>(maps, p, pair, ep, st)) != VT_OK) return r;
    cudaError_t e = launch_pdl(score_given_kernel, c.M, kRowThreads, 0, st, reinterpret_cast<const uint16_t*>(c.h), c.ldh, c.tokens,
                               rest, first, count, sums, c.M, c.d, c.V, given_wide_from(c.M), reinterpret_cast<uint16_t*>(grad_W));
    count_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

}  // namespace vt
