// Log probabilities of given tokens under a head, with entropy, log-sum-exp and the k best alternatives.
//
//   x[m, v] = sum_j h[m, j] W[v, j]     z = scale * x     lse = log sum_v e^z     logprob = z[t] - lse
//   H = -sum_v p log p = log s - E[z - max],  s = sum_v e^(z - max),  E[y] = sum_v e^(z - max) y / s
//
// One pass over the head: no logit is written.  gemm_kernel gives every epilogue thread a row of the tile and a range
// of its columns; the thread folds them into a running (max, s, e = sum of (x - max) e^(z - max)) - kept about the
// maximum, because lse and E[z] are both large where H is small - and into a register list of its k best logits, and
// picks the given token's logit when it comes by.  At the end of a run of tiles it writes one record; a second, small
// kernel (one block per row) joins a row's records.  Records are joined in the order of their columns and the list's
// keys are distinct, so the result does not depend on which block ran when.
#include "vt_score.h"

#include "vt_gemm.cuh"

namespace vt {

constexpr float kMasked = -1e38f;          // stands for a column past the vocabulary: e^ gives 0, and nothing finite is below it

struct ScoreRecords {
    float4* stats;                         // [M][L]: max, s, e, unused
    unsigned long long* keys;              // [M][L][k] descending, 0 = none
    float* given;                          // [M] the given token's logit
    int L;                                 // records per row
};

template <int KR>
struct EpiScore {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = true;
    struct Params {
        const int32_t* tokens;
        ScoreRecords rec;
        float c;                           // scale * log2(e)
        int M, V, k;
    };
    static constexpr int KL = KR > 0 ? KR : 1;
    struct State {
        float mx, s, e;
        int tok;
        float v[KL];
        int ix[KL];
    };
    static __device__ __forceinline__ void begin(State& st, const Params& ep, int m) {
        st.mx = kMasked;
        st.s = st.e = 0.0f;
        st.tok = ep.tokens != nullptr && m < ep.M ? ep.tokens[m] : -1;
        if constexpr (KR > 0) {
#pragma unroll
            for (int j = 0; j < KL; ++j) { st.v[j] = kMasked; st.ix[j] = -1; }
        }
    }
    static __device__ __forceinline__ void cols16(State& st, const Params& ep, int m, int col, int live, float (&x)[16]) {
        if (live < 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = i < live ? x[i] : kMasked;
        }
        float cm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        cm = fmaxf(cm, fmaxf(fmaxf(fmaxf(x[8], x[9]), fmaxf(x[10], x[11])), fmaxf(fmaxf(x[12], x[13]), fmaxf(x[14], x[15]))));
        const float nm = fmaxf(st.mx, cm);
        const float back = st.mx - nm, f = ex2_approx(back * ep.c);
        float s0 = 0.0f, s1 = 0.0f, e0 = 0.0f, e1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float y0 = x[i] - nm, y1 = x[i + 1] - nm;
            const float p0 = ex2_approx(y0 * ep.c), p1 = ex2_approx(y1 * ep.c);
            s0 += p0;
            s1 += p1;
            e0 = fmaf(p0, y0, e0);
            e1 = fmaf(p1, y1, e1);
        }
        st.e = fmaf(f, fmaf(back, st.s, st.e), e0 + e1);
        st.s = fmaf(f, st.s, s0 + s1);
        st.mx = nm;
        const int at = st.tok - col;
        if ((unsigned)at < (unsigned)min(live, 16)) {
            float g = x[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) g = at == i ? x[i] : g;
            ep.rec.given[m] = g;
        }
        if constexpr (KR > 0) {
            if (__any_sync(0xFFFFFFFFu, cm > st.v[KL - 1])) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (__any_sync(0xFFFFFFFFu, x[i] > st.v[KL - 1])) rows_insert<KL>(st.v, st.ix, x[i], col + i);
            }
        }
    }
    static __device__ __forceinline__ void end(State& st, const Params& ep, int m, int list) {
        if (m >= ep.M) return;
        const size_t at = (size_t)m * ep.rec.L + list;
        ep.rec.stats[at] = make_float4(st.mx, st.s, st.e, 0.0f);
        if constexpr (KR > 0) {
#pragma unroll
            for (int j = 0; j < KL; ++j)
                if (j < ep.k) ep.rec.keys[at * ep.k + j] = st.ix[j] >= 0 ? make_key(st.v[j], st.ix[j]) : 0ull;
        }
    }
};

// ------------------------------------------------------------------------------------------ the join of a row's records
constexpr int kJoinThreads = 128;
constexpr int kJoinCand = 1024;
constexpr int kJoinHeld = 8;               // lists a thread keeps the best key of in registers

struct ScoreJoin {
    ScoreRecords rec;
    ScoreOut out;
    const int32_t* tokens;
    int V;
    float scale;
};

// One block per row, bound by the latency of its few loads: all records of a thread's lists are requested together.
__global__ void __launch_bounds__(kJoinThreads) score_join_kernel(const ScoreJoin p) {
    __shared__ float3 parts[kJoinThreads / 32];
    __shared__ unsigned long long heads[kJoinThreads], cand[kJoinCand];
    __shared__ unsigned long long bound_s;
    __shared__ int n_cand;
    const int m = blockIdx.x, t = threadIdx.x, L = p.rec.L, k = p.out.k;
    if (t == 0) { n_cand = 0; bound_s = 1ull; }
    grid_dependency_wait();
    const ScoreOut& o = p.out;
    if (!row_scored(p.tokens, p.V, m)) {
        if (t == 0) {
            if (o.logprobs) o.logprobs[m] = 0.0f;
            if (o.entropy) o.entropy[m] = 0.0f;
            if (o.lse) o.lse[m] = 0.0f;
        }
        for (int j = t; j < k; j += kJoinThreads) {
            o.top_ids[(size_t)m * k + j] = -1;
            o.top_logprobs[(size_t)m * k + j] = 0.0f;
        }
        return;
    }
    const float4* stats = p.rec.stats + (size_t)m * L;
    const unsigned long long* keys = p.rec.keys + (size_t)m * L * k;
    const float c = p.scale * kLog2e;
    const float given = o.logprobs ? p.rec.given[m] : 0.0f;
    float mx = kMasked, s = 0.0f, e = 0.0f;
    unsigned long long held[kJoinHeld], head = 0ull;
    auto fold = [&](float rmx, float rs, float re) {
        const float nm = fmaxf(mx, rmx), b0 = mx - nm, b1 = rmx - nm;
        const float f0 = ex2_approx(b0 * c), f1 = ex2_approx(b1 * c);
        e = fmaf(f0, fmaf(b0, s, e), f1 * fmaf(b1, rs, re));
        s = fmaf(f0, s, f1 * rs);
        mx = nm;
    };
    {
        float4 r[kJoinHeld];
#pragma unroll
        for (int i = 0; i < kJoinHeld; ++i) {
            const int l = t + i * kJoinThreads;
            r[i] = l < L ? stats[l] : make_float4(kMasked, 0.0f, 0.0f, 0.0f);
            held[i] = l < L && k > 0 ? keys[(size_t)l * k] : 0ull;
        }
#pragma unroll
        for (int i = 0; i < kJoinHeld; ++i) {
            fold(r[i].x, r[i].y, r[i].z);
            head = held[i] > head ? held[i] : head;
        }
    }
    for (int l = t + kJoinHeld * kJoinThreads; l < L; l += kJoinThreads) {
        const float4 r = stats[l];
        fold(r.x, r.y, r.z);
        if (k > 0) {
            const unsigned long long key = keys[(size_t)l * k];
            head = key > head ? key : head;
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float rmx = __shfl_xor_sync(0xFFFFFFFFu, mx, d), rs = __shfl_xor_sync(0xFFFFFFFFu, s, d), re = __shfl_xor_sync(0xFFFFFFFFu, e, d);
        // both lanes of a pair must come to the same bits: the lower lane's part first
        const bool low = (t & d) == 0;
        const float amx = low ? mx : rmx, as = low ? s : rs, ae = low ? e : re;
        const float bmx = low ? rmx : mx, bs = low ? rs : s, be = low ? re : e;
        mx = amx;
        s = as;
        e = ae;
        fold(bmx, bs, be);
    }
    if ((t & 31) == 0) parts[t >> 5] = make_float3(mx, s, e);
    heads[t] = head;
    __syncthreads();
    mx = parts[0].x;
    s = parts[0].y;
    e = parts[0].z;
#pragma unroll
    for (int w = 1; w < kJoinThreads / 32; ++w) fold(parts[w].x, parts[w].y, parts[w].z);
    const float log_s = logf(s);
    if (t == 0) {
        if (o.lse) o.lse[m] = fmaf(p.scale, mx, log_s);
        if (o.entropy) o.entropy[m] = log_s - p.scale * (e / s);
        if (o.logprobs) o.logprobs[m] = p.scale * (given - mx) - log_s;
    }
    if (k == 0) return;

    // The k best of L descending lists.  The k-th largest of the threads' best heads bounds the winners from below: k keys
    // at least that large exist.  The keys not below it are gathered, and a key's place is the number of keys above it.
    if (head != 0ull) {
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < kJoinThreads; ++i) above += heads[i] > head ? 1 : 0;
        if (above == k - 1) bound_s = head;
    }
    __syncthreads();
    const unsigned long long bound = bound_s;          // 1 (every key) when fewer than k threads have one
    auto gather = [&](int l, unsigned long long key) {
        for (int j = 0; key >= bound;) {
            const int at = atomicAdd(&n_cand, 1);      // the order of the candidates does not matter: their ranks decide
            if (at < kJoinCand) cand[at] = key;
            if (++j == k) break;
            key = keys[(size_t)l * k + j];
        }
    };
#pragma unroll
    for (int i = 0; i < kJoinHeld; ++i) gather(t + i * kJoinThreads, held[i]);
    for (int l = t + kJoinHeld * kJoinThreads; l < L; l += kJoinThreads) gather(l, keys[(size_t)l * k]);
    __syncthreads();
    const int n = n_cand;
    auto emit = [&](int j, unsigned long long key) {
        const size_t at = (size_t)m * k + j;
        o.top_ids[at] = key != 0ull ? key_index(key) : -1;
        o.top_logprobs[at] = key != 0ull ? p.scale * (key_logit(key) - mx) - log_s : -INFINITY;
    };
    if (n <= kJoinCand) {
        for (int i = t; i < n; i += kJoinThreads) {
            const unsigned long long key = cand[i];
            int above = 0;
#pragma unroll 4
            for (int q = 0; q < n; ++q) above += cand[q] > key ? 1 : 0;
            if (above < k) emit(above, key);
        }
        for (int j = n + t; j < k; j += kJoinThreads) emit(j, 0ull);
        return;
    }
    // Too many for the buffer (the winners sit in few lists): the largest key below the last winner, k times.
    unsigned long long last = ~0ull;
    for (int j = 0; j < k; ++j) {
        unsigned long long best = 0ull;
        for (int l = t; l < L; l += kJoinThreads)
            for (int i = 0; i < k; ++i) {
                const unsigned long long key = keys[(size_t)l * k + i];
                if (key < last) { best = key > best ? key : best; break; }
            }
        best = warp_max_key(best);
        __syncthreads();
        if ((t & 31) == 0) heads[t >> 5] = best;
        __syncthreads();
        for (int i = 0; i < kJoinThreads / 32; ++i) best = heads[i] > best ? heads[i] : best;
        if (t == 0) emit(j, best);
        last = best;
    }
}

// ------------------------------------------------------------------------------------------ host
static bool score_plan(int M, int d, int V, GemmParams* p, bool* pair) {
    p->n_prob = 1;
    p->prob[0] = GemmProblem{};
    p->prob[0].M = M;
    p->prob[0].N = V;
    p->prob[0].b0 = 1;
    p->prob[0].nk0 = ceil_div(d, kBoxK);
    return gemm_plan_rows(p, pair);
}
static int score_records(const GemmParams& p) { return p.prob[0].chunks_n * 2 * p.rep; }

size_t score_workspace_bytes(int M, int d, int V, int k) {
    GemmParams p{};
    bool pair = false;
    if (!score_plan(M, d, V, &p, &pair)) return 0;
    const size_t rows = (size_t)M * score_records(p);
    return kHeaderBytes + round_up(rows * sizeof(float4), 256) + round_up(rows * k * 8, 256) + round_up((size_t)M * 4, 256);
}

template <int KR>
static vt_status run_score(const GemmMaps& maps, const GemmParams& p, bool pair, const ScoreCall& c, const ScoreRecords& rec, int k,
                           cudaStream_t st) {
    const typename EpiScore<KR>::Params ep{c.tokens, rec, c.scale * kLog2e, c.M, c.V, k};
    return gemm_launch<false, false, EpiScore<KR>>(maps, p, pair, ep, st);
}

vt_status launch_score(const ScoreCall& c, const ScoreOut& o, void* workspace, cudaStream_t st) {
    GemmMaps maps{};
    GemmParams p{};
    bool pair = false;
    if (!score_plan(c.M, c.d, c.V, &p, &pair)) return VT_ERR_SHAPE;
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    p.hdr = reinterpret_cast<WsHeader*>(base);
    ScoreRecords rec;
    rec.L = score_records(p);
    const size_t rows = (size_t)c.M * rec.L;
    rec.stats = reinterpret_cast<float4*>(base + kHeaderBytes);
    rec.keys = reinterpret_cast<unsigned long long*>(base + kHeaderBytes + round_up(rows * sizeof(float4), 256));
    rec.given = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(rec.keys) + round_up(rows * o.k * 8, 256));
    vt_status r = gemm_map(&maps.map[0], GemmOperand{c.h, c.M, c.d, c.ldh}, gemm_box_a(p, false));
    if (r != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], GemmOperand{c.W, c.V, c.d, c.d}, gemm_box_b(p, false, pair))) != VT_OK) return r;
    if (o.k == 0) r = run_score<0>(maps, p, pair, c, rec, o.k, st);
    else if (o.k <= 4) r = run_score<4>(maps, p, pair, c, rec, o.k, st);
    else if (o.k <= 8) r = run_score<8>(maps, p, pair, c, rec, o.k, st);
    else if (o.k <= 20) r = run_score<20>(maps, p, pair, c, rec, o.k, st);
    else r = run_score<VT_MAX_K>(maps, p, pair, c, rec, o.k, st);
    if (r != VT_OK) return r;
    const ScoreJoin join{rec, o, c.tokens, c.V, c.scale};
    cudaError_t e = launch_pdl(score_join_kernel, c.M, kJoinThreads, 0, st, join);
    count_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

}  // namespace vt
