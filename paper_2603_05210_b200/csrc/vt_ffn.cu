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
// act(g) and act'(g).  SiLU: g s, s (1 + g (1 - s)) with s = 1 / (1 + e^-g).  GELU (tanh form): with b = sqrt(2/pi) (g +
// 0.044715 g^3), (1 + tanh b) / 2 = 1 / (1 + e^-2b) = s, so act = g s and act' = s + g s (1 - s) * 2 b'.
__device__ __forceinline__ ActValue act_eval(int act, float g) {
    float b2 = g, slope2 = 1.0f;
    if (act == VT_ACT_GELU) {
        constexpr float k2 = 1.5957691216057308f;          // 2 sqrt(2 / pi)
        b2 = k2 * g * fmaf(0.044715f * g, g, 1.0f);
        slope2 = k2 * fmaf(0.134145f * g, g, 1.0f);
    }
    const float e = __expf(-b2);
    const float s = __fdividef(1.0f, 1.0f + e);            // e = inf: 0
    const float rest = b2 < -40.0f ? 1.0f : e * s;         // 1 - s without cancellation
    ActValue r;
    r.value = g * s;
    r.slope = fmaf(g * s * rest, slope2, s);
    return r;
}

struct EpiGateUp {
    static constexpr bool kDual = true;
    static constexpr bool kStateful = false;
    struct Params {
        uint16_t* a;        // [M, f] bf16
        float* saved;       // [M, 2f] (g, then u), or null
        int act;
    };
    struct State {};
    static __device__ __forceinline__ void row(State&, const Params&, const GemmProblem&, int) {}
    static __device__ __forceinline__ void cols8(State&, const Params& ep, const GemmProblem& q, int m, int n, const float* g, const float* u) {
        float a[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = act_eval(ep.act, g[i]).value * u[i];
        store_bf16x8(ep.a + (size_t)m * q.N + n, a);
        if (ep.saved) {
            float* gs = ep.saved + (size_t)m * 2 * q.N + n;
            float* us = gs + q.N;
            *reinterpret_cast<float4*>(gs) = make_float4(g[0], g[1], g[2], g[3]);
            *reinterpret_cast<float4*>(gs + 4) = make_float4(g[4], g[5], g[6], g[7]);
            *reinterpret_cast<float4*>(us) = make_float4(u[0], u[1], u[2], u[3]);
            *reinterpret_cast<float4*>(us + 4) = make_float4(u[4], u[5], u[6], u[7]);
        }
    }
};

struct EpiActGrad {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    struct Params {
        const float* saved;     // [M, 2f]
        uint16_t* dgu;          // [M, 2f] bf16: dg, then du
        uint16_t* a;            // [M, f] bf16
        int act;
    };
    struct State {};
    static __device__ __forceinline__ void row(State&, const Params&, const GemmProblem&, int) {}
    static __device__ __forceinline__ void cols8(State&, const Params& ep, const GemmProblem& q, int m, int n, const float* da) {
        const size_t at = (size_t)m * 2 * q.N + n;
        float g[8], u[8], dg[8], du[8], a[8];
        *reinterpret_cast<float4*>(g) = *reinterpret_cast<const float4*>(ep.saved + at);
        *reinterpret_cast<float4*>(g + 4) = *reinterpret_cast<const float4*>(ep.saved + at + 4);
        *reinterpret_cast<float4*>(u) = *reinterpret_cast<const float4*>(ep.saved + at + q.N);
        *reinterpret_cast<float4*>(u + 4) = *reinterpret_cast<const float4*>(ep.saved + at + q.N + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const ActValue v = act_eval(ep.act, g[i]);
            dg[i] = da[i] * u[i] * v.slope;
            du[i] = da[i] * v.value;
            a[i] = v.value * u[i];
        }
        store_bf16x8(ep.dgu + at, dg);
        store_bf16x8(ep.dgu + at + q.N, du);
        store_bf16x8(ep.a + (size_t)m * q.N + n, a);
    }
};

static inline int k_blocks(int k) { return (k + kBoxK - 1) / kBoxK; }

static GemmProblem problem(int M, int N, int a0, int b0, int nk0, void* out, int a1 = 0, int b1 = 0, int nk1 = 0) {
    GemmProblem q{};
    q.M = M;
    q.N = N;
    q.a0 = a0;
    q.b0 = b0;
    q.nk0 = nk0;
    q.a1 = a1;
    q.b1 = b1;
    q.nk1 = nk1;
    q.out = out;
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
        p.prob[0] = problem(c.M, c.f, 0, 1, k_blocks(c.d), nullptr, 0, 2, 0);
        p.hdr = reinterpret_cast<WsHeader*>(base);
        if (!gemm_plan(&p, false, false, true, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], x, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wg, gemm_box_b(p, false, pair))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[2], wu, gemm_box_b(p, false, pair))) != VT_OK) return r;
        const EpiGateUp::Params ep{a, saved, c.act};
        if ((r = gemm_launch<false, false, EpiGateUp>(maps, p, pair, ep, st)) != VT_OK) return r;
    }
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    p.n_prob = 1;
    p.prob[0] = problem(c.M, c.d, 0, 1, k_blocks(c.f), y);
    p.hdr = reinterpret_cast<WsHeader*>(base);
    if (!gemm_plan(&p, false, false, false, &pair)) return VT_ERR_SHAPE;
    if ((r = gemm_map(&maps.map[0], GemmOperand{a, c.M, c.f, c.f}, gemm_box_a(p, false))) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], wd, gemm_box_b(p, false, pair))) != VT_OK) return r;
    return gemm_store(maps, p, pair, false, false, st);
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
        p.prob[0] = problem(c.M, c.f, 0, 1, k_blocks(c.d), nullptr);
        p.hdr = hdr;
        if (!gemm_plan(&p, false, true, false, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], dy, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wd, gemm_box_b(p, true, pair))) != VT_OK) return r;
        const EpiActGrad::Params ep{saved, dgu, a, c.act};
        if ((r = gemm_launch<false, true, EpiActGrad>(maps, p, pair, ep, st)) != VT_OK) return r;
    }
    if (grad_x) {   // dx = dg Wg + du Wu: [M, d], summed over f twice
        GemmMaps maps{};
        GemmParams p{};
        bool pair = false;
        p.n_prob = 1;
        p.prob[0] = problem(c.M, c.d, 0, 1, k_blocks(c.f), grad_x, 2, 3, k_blocks(c.f));
        p.hdr = hdr;
        if (!gemm_plan(&p, false, true, false, &pair)) return VT_ERR_SHAPE;
        if ((r = gemm_map(&maps.map[0], dg, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[1], wg, gemm_box_b(p, true, pair))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[2], du, gemm_box_a(p, false))) != VT_OK) return r;
        if ((r = gemm_map(&maps.map[3], wu, gemm_box_b(p, true, pair))) != VT_OK) return r;
        if ((r = gemm_store(maps, p, pair, false, true, st)) != VT_OK) return r;
    }
    // dWg = dg^T x, dWu = du^T x: [f, d]; dWd = dy^T a: [d, f]; all summed over the M rows
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    const int nk = k_blocks(c.M);
    p.hdr = hdr;
    if (grad_W_gate) p.prob[p.n_prob++] = problem(c.f, c.d, 0, 3, nk, grad_W_gate);
    if (grad_W_up) p.prob[p.n_prob++] = problem(c.f, c.d, 1, 3, nk, grad_W_up);
    if (grad_W_down) p.prob[p.n_prob++] = problem(c.d, c.f, 2, 4, nk, grad_W_down);
    if (p.n_prob == 0) return VT_OK;
    if (!gemm_plan(&p, true, true, false, &pair)) return VT_ERR_SHAPE;
    const int box_a = gemm_box_a(p, true), box_b = gemm_box_b(p, true, pair);
    if ((r = gemm_map(&maps.map[0], dg, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], du, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[2], dy, box_a)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[3], x, box_b)) != VT_OK) return r;
    if ((r = gemm_map(&maps.map[4], av, box_b)) != VT_OK) return r;
    return gemm_store(maps, p, pair, true, true, st);
}

}  // namespace vt
