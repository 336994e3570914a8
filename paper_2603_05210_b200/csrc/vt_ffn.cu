// Gated feed-forward block of a draft layer, y = (act(x Wg^T) * (x Wu^T)) Wd^T, and its backward pass.
//
// Forward, two launches:
//   1. gate and up in one product: a tile's accumulator holds the same features of both, side by side, so the activation
//      and the product of the two are formed on the way out of tensor memory; only a = act(g) * u goes to memory, rounded
//      to bf16 because it is an operand of the next product (a training step also keeps g and u, in fp32);
//   2. y = a Wd^T.
// Backward, three launches:
//   1. da = dy Wd, and from it with the kept g and u, in fp32, the three operands of the rest:
//      dg = da u act'(g), du = da act(g), a = act(g) u, each rounded once to bf16 as it is stored;
//   2. dx = dg Wg + du Wu, one sum over both;
//   3. dWg = dg^T x, dWu = du^T x, dWd = dy^T a, three products in one grid.
// g and u are kept in fp32 rather than bf16: a rounded g would enter act' and be rounded again in dg, and the gradients'
// error would grow from 1.4 to 1.7 times that of one rounding.
#include "vt_ffn.h"

#include "vt_gemm.cuh"

namespace vt {

struct ActValue {
    float value, slope;
};
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// act(g) and act'(g).  SiLU: g s, s (1 + g (1 - s)) with s = 1 / (1 + e^-g).  GELU (tanh form): with b = sqrt(2/pi) (g +
// 0.044715 g^3), (1 + tanh b) / 2 = 1 / (1 + e^-2b) = s, so act = g s and act' = s (1 + g (1 - s) 2 b').  1 - s cancels only where
// s is 1 to the last bit and the term it is in is nothing beside the 1.  The activation is a template parameter: a tile of da
// spent more time on this than on its product when it was asked for element by element.
template <int ACT>
__device__ __forceinline__ ActValue act_eval(float g) {
    constexpr float kLog2 = 1.4426950408889634f, k2 = 1.5957691216057308f;      // log2 e, 2 sqrt(2 / pi)
    float s, gg = g;
    if constexpr (ACT == VT_ACT_GELU) {
        const float q = g * g;
        s = rcp_approx(1.0f + ex2_approx(-kLog2 * k2 * g * fmaf(0.044715f, q, 1.0f)));
        gg = g * (k2 * fmaf(0.134145f, q, 1.0f));
        if (q > 1e4f) gg = 0.0f;                           // far out s is 0 or 1 and the term nothing, before it overflows
    } else {
        s = rcp_approx(1.0f + ex2_approx(-kLog2 * g));
    }
    ActValue r;
    r.value = g * s;
    r.slope = s * fmaf(gg, 1.0f - s, 1.0f);
    return r;
}

// The kept projections, [M, 2 f] floats: g of all features, then u, in blocks of 32 rows (the last block: of the rows left) x 4
// features, rows of a block one after the other.  The 32 rows of a warp's accumulators are then one contiguous run, read
// and written at full width whatever tiles either pass uses.
__device__ __forceinline__ float* saved_at(float* saved, int M, int f2, int m, int col) {
    const int m0 = m & ~31, rows = min(32, M - m0);
    return saved + (size_t)m0 * f2 + (size_t)(col >> 2) * (rows * 4) + (m - m0) * 4;
}

template <int ACT>
struct EpiGateUp {
    static constexpr bool kDual = true;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = false;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        uint16_t* a;        // [M, f] bf16
        float* saved;       // see saved_at, or null
    };
    struct State {};
    static __device__ __forceinline__ void row(State&, const Params&, const GemmProblem&, int) {}
    static __device__ __forceinline__ void ahead(State&, const Params&, const GemmProblem&, int, int, int) {}
    static __device__ __forceinline__ void cols8(State&, const Params& ep, const GemmProblem& q, int m, int n, int, const float (&g)[8],
                                                 const float (&u)[8], float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[0][i] = act_eval<ACT>(g[i]).value * u[i];
        if (ep.saved && m < q.M && n < q.N) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<float4*>(saved_at(ep.saved, q.M, 2 * q.N, m, n + i)) = make_float4(g[i], g[i + 1], g[i + 2], g[i + 3]);
                *reinterpret_cast<float4*>(saved_at(ep.saved, q.M, 2 * q.N, m, q.N + n + i)) = make_float4(u[i], u[i + 1], u[i + 2], u[i + 3]);
            }
        }
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem& q, int, int, int m, int n) { return ep.a + (size_t)m * q.N + n; }
    static __device__ __forceinline__ int64_t ld(const Params&, const GemmProblem& q, int) { return q.N; }
};

template <int ACT>
struct EpiActGrad {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = false;
    static constexpr int kOuts = 3;         // dg, du, a
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        float* saved;           // see saved_at; only read
        uint16_t* dgu;          // [M, 2f] bf16: dg, then du
        uint16_t* a;            // [M, f] bf16
    };
    struct State {
        float4 g[2][4], u[2][4];      // the next two runs of 16 columns
    };
    static __device__ __forceinline__ void row(State&, const Params&, const GemmProblem&, int) {}
    static __device__ __forceinline__ void ahead(State& st, const Params& ep, const GemmProblem& q, int m, int n, int slot) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + 4 * i < q.N) {
                st.g[slot][i] = *reinterpret_cast<const float4*>(saved_at(ep.saved, q.M, 2 * q.N, m, n + 4 * i));
                st.u[slot][i] = *reinterpret_cast<const float4*>(saved_at(ep.saved, q.M, 2 * q.N, m, q.N + n + 4 * i));
            }
    }
    static __device__ __forceinline__ void cols8(State& st, const Params& ep, const GemmProblem&, int, int, int e, const float (&da)[8],
                                                 const float (&)[8], float (&out)[3][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 g4 = st.g[e >> 4][(e & 15) + i >> 2], u4 = st.u[e >> 4][(e & 15) + i >> 2];
            const float g = (i & 3) == 0 ? g4.x : (i & 3) == 1 ? g4.y : (i & 3) == 2 ? g4.z : g4.w;
            const float u = (i & 3) == 0 ? u4.x : (i & 3) == 1 ? u4.y : (i & 3) == 2 ? u4.z : u4.w;
            const ActValue v = act_eval<ACT>(g);
            out[0][i] = da[i] * u * v.slope;
            out[1][i] = da[i] * v.value;
            out[2][i] = v.value * u;
        }
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem& q, int, int o, int m, int n) {
        return o == 2 ? ep.a + (size_t)m * q.N + n : ep.dgu + (size_t)m * 2 * q.N + (o == 1 ? q.N : 0) + n;
    }
    static __device__ __forceinline__ int64_t ld(const Params&, const GemmProblem& q, int o) { return o == 2 ? q.N : 2 * q.N; }
};

static inline int k_blocks(int k) { return (k + kBoxK - 1) / kBoxK; }

static GemmProblem problem(int M, int N, int a0, int b0, int nk0, int a1 = 0, int b1 = 0, int nk1 = 0) {
    GemmProblem q{};
    q.M = M;
    q.N = N;
    q.a0 = a0;
    q.b0 = b0;
    q.nk0 = nk0;
    q.a1 = a1;
    q.b1 = b1;
    q.nk1 = nk1;
    return q;
}

size_t ffn_workspace_bytes(int M, int d, int f) {
    (void)d;
    return kHeaderBytes + round_up((size_t)M * f * 2, 256);
}

size_t ffn_backward_workspace_bytes(int M, int d, int f) {
    (void)d;
    return kHeaderBytes + round_up((size_t)M * f * 4, 256) + round_up((size_t)M * f * 2, 256);
}

vt_status launch_ffn(const FfnCall& c, void* y, float* saved, void* workspace, cudaStream_t st) {
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    uint16_t* a = reinterpret_cast<uint16_t*>(base + kHeaderBytes);
    const GemmOperand x{c.x, c.M, c.d, c.ldx}, wg{c.W_gate, c.f, c.d, c.d}, wu{c.W_up, c.f, c.d, c.d}, wd{c.W_down, c.d, c.f, c.f};
    vt_status r;
    {
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        p.prob[0] = problem(c.M, c.f, 0, 1, k_blocks(c.d), 0, 2, 0);
        p.hdr = reinterpret_cast<WsHeader*>(base);
        if (!gemm_plan(&p, false, false, true, EpiGateUp<VT_ACT_SILU>::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], x, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wg, gemm_box_b(p, false, pair))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[2], wu, gemm_box_b(p, false, pair))) != VT_OK) return r;
        r = c.act == VT_ACT_GELU ? gemm_launch<false, false, EpiGateUp<VT_ACT_GELU>>(maps, p, pair, {a, saved}, st)
                                 : gemm_launch<false, false, EpiGateUp<VT_ACT_SILU>>(maps, p, pair, {a, saved}, st);
        if (r != VT_OK) return r;
    }
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    p.n_prob = 1;
    p.prob[0] = problem(c.M, c.d, 0, 1, k_blocks(c.f));
    p.b_early = 1;
    p.hdr = reinterpret_cast<WsHeader*>(base);
    if (!gemm_plan(&p, false, false, false, EpiStore::kScratch, &pair)) return VT_ERR_SHAPE;
    if ((r = gemm_map(&maps.map[0], GemmOperand{a, c.M, c.f, c.f}, gemm_box_a(p, false))) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], wd, gemm_box_b(p, false, pair))) != VT_OK) return r;
    return gemm_store(maps, p, pair, false, false, &y, st);
}

vt_status launch_ffn_backward(const FfnCall& c, const float* saved, const void* grad_y, int64_t ld_grad_y, void* grad_x,
                              void* grad_W_gate, void* grad_W_up, void* grad_W_down, void* workspace, cudaStream_t st) {
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    WsHeader* hdr = reinterpret_cast<WsHeader*>(base);
    uint16_t* dgu = reinterpret_cast<uint16_t*>(base + kHeaderBytes);
    uint16_t* a = reinterpret_cast<uint16_t*>(base + kHeaderBytes + round_up((size_t)c.M * c.f * 4, 256));
    const GemmOperand x{c.x, c.M, c.d, c.ldx}, dy{grad_y, c.M, c.d, ld_grad_y};
    const GemmOperand wg{c.W_gate, c.f, c.d, c.d}, wu{c.W_up, c.f, c.d, c.d}, wd{c.W_down, c.d, c.f, c.f};
    const GemmOperand dg{dgu, c.M, c.f, 2 * (int64_t)c.f}, du{dgu + c.f, c.M, c.f, 2 * (int64_t)c.f}, av{a, c.M, c.f, c.f};
    vt_status r;
    {   // da = dy Wd: [M, f], summed over d; Wd [d, f] has f running fastest
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        p.prob[0] = problem(c.M, c.f, 0, 1, k_blocks(c.d));
        p.hdr = hdr;
        if (!gemm_plan(&p, false, true, false, EpiActGrad<VT_ACT_SILU>::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], dy, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wd, gemm_box_b(p, true, pair))) != VT_OK) return r;
        float* kept = const_cast<float*>(saved);
        r = c.act == VT_ACT_GELU ? gemm_launch<false, true, EpiActGrad<VT_ACT_GELU>>(maps, p, pair, {kept, dgu, a}, st)
                                 : gemm_launch<false, true, EpiActGrad<VT_ACT_SILU>>(maps, p, pair, {kept, dgu, a}, st);
        if (r != VT_OK) return r;
    }
    if (grad_x) {   // dx = dg Wg + du Wu: [M, d], summed over f twice
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        p.prob[0] = problem(c.M, c.d, 0, 1, k_blocks(c.f), 2, 3, k_blocks(c.f));
        p.b_early = 1;
        p.hdr = hdr;
        if (!gemm_plan(&p, false, true, false, EpiStore::kScratch, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], dg, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wg, gemm_box_b(p, true, pair))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[2], du, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[3], wu, gemm_box_b(p, true, pair))) != VT_OK) return r;
        if ((r = gemm_store(maps, p, pair, false, true, &grad_x, st)) != VT_OK) return r;
    }
    // dWg = dg^T x, dWu = du^T x: [f, d]; dWd = dy^T a: [d, f]; all summed over the M rows
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    const int nk = k_blocks(c.M);
    p.hdr = hdr;
    void* outs[kGemmMaxProblems];
    auto add = [&](void* out, const GemmProblem& q) {
        if (!out) return;
        outs[p.n_prob] = out;
        p.prob[p.n_prob++] = q;
    };
    add(grad_W_gate, problem(c.f, c.d, 0, 3, nk));
    add(grad_W_up, problem(c.f, c.d, 1, 3, nk));
    add(grad_W_down, problem(c.d, c.f, 2, 4, nk));
    if (p.n_prob == 0) return VT_OK;
    if (!gemm_plan(&p, true, true, false, EpiStore::kScratch, &pair)) return VT_ERR_SHAPE;
    const int box_a = gemm_box_a(p, true), box_b = gemm_box_b(p, true, pair);
    if ((r = gemm_map(&maps.map[0], dg, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], du, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[2], dy, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[3], x, box_b)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[4], av, box_b)) != VT_OK) return r;
    return gemm_store(maps, p, pair, true, true, outs, st);
}

}  // namespace vt
