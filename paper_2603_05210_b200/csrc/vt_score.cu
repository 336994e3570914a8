// Log probabilities of given tokens under a head, with entropy, log-sum-exp and the k best alternatives.
//
//   x[m, v] = sum_j h[m, j] W[v, j]     z = scale * x     lse = log sum_v e^z     logprob = z[t] - lse
//   H = -sum_v p log p = log s - E[z - max],  s = sum_v e^(z - max),  E[y] = sum_v e^(z - max) y / s
//
// One pass over the head.  gemm_kernel gives every epilogue thread a row of the tile and a range of its columns; the thread
// folds them into a running (max, s, e = sum of t 2^t, t = (x - max) scale log2 e) - kept about the maximum, because lse and E[z]
// are both large where H is small, and in units of t, because sums of x - max overflow where the scale is next to nothing - and picks the given token's logit when it comes by.  At the end of a run of tiles it
// writes one record; a second, small kernel (one block per row) joins a row's records.  The k best come in one of two ways:
//   listed  no logit is written; every thread keeps a register list of its k best, and the join merges the lists;
//   kept    the logits go to the workspace, and the join reads back the handful of ranges whose maximum is not below the
//           k-th largest maximum of all.
// Lists cost the epilogue more the longer they are (and their first tile most, so that long runs of tiles pay), kept logits
// their bytes and a longer join.  Measured, us, listed / kept (and without alternatives):
//     M = 33, V = 32000, d = 4096       k = 8: 55.9 / 53.8   k = 20: 70.9 / 57.3       (48.1)
//     M = 61, V = 32000, d = 4096       k = 8: 55.2 / 54.6   k = 20: 71.8 / 58.4
//     M = 128, V = 32000, d = 4096      k = 4: 63.8 / 70.1   k = 20: 84.5 / 72.8       (55.6)
//     M = 300, V = 8000, d = 2048       k = 8: 39.1 / 43.3   k = 20: 62.0 / 46.2       (27.6)
//     M = 256, V = 32000, d = 2048      k = 8: 50.8 / 61.1   k = 20: 72.5 / 65.5
//     M = 128, V = 100000, d = 4096     k = 8: 142 / 153     k = 20: 153 / 165         (134)
//     M = 4096, V = 32000, d = 4096     k = 8: 754 / 951     k = 20: 894 / 981         (687)
// hence keep_logits() below.
// Records are joined in the order of their columns and ranked by distinct keys, so the result does not depend on which
// block ran when.
#include <cfloat>

#include "vt_score.h"

#include "vt_gemm.cuh"

namespace vt {

constexpr float kLowest = -FLT_MAX;       // the running maximum of no columns: no finite logit is below it

struct ScoreRecords {
    float4* stats;                         // [M][L]: max, s, e, unused
    unsigned long long* keys;              // listed: [M][L][k] descending, 0 = none
    float* logits;                         // kept: [M][ld]
    float* given;                          // [M] the given token's logit
    int64_t ld;
    int L;                                 // records per row
    int parts, NT, tiles_per_item;         // record -> columns: parts per item, columns per tile, tiles per item
};

constexpr float kLn2 = 0.6931471805599453f;
// scale * log2(e), finite: (max - max) times it has to be 0
__host__ __device__ inline float exponent_scale(float scale) { return fminf(scale * kLog2e, FLT_MAX); }

constexpr int kListQueue = 24;             // candidates a thread queues between insertions
constexpr int kListMax = 20;                // entries of the longest list
constexpr int kKeepLogits = -1;            // EpiScore<kKeepLogits>: the kept form

// KR: entries of a thread's list (0: no alternatives wanted), or kKeepLogits.
template <int KR>
struct EpiScore {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = true;
    static constexpr int kOuts = 0;
    static constexpr uint32_t kScratch = KR > 0 ? kListQueue * kGemmEpiWarps * 32 * 5 : 0;
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
        bool first;
        float bound;                       // k logits of the row are known to be at least this large
        float v[KL];
        int ix[KL];
    };
    static __device__ __forceinline__ void begin(State& st, const Params& ep, int m) {
        st.mx = kLowest;
        st.s = st.e = 0.0f;
        st.tok = ep.tokens != nullptr && m < ep.M ? ep.tokens[m] : -1;
        st.first = true;
        st.bound = -INFINITY;
#pragma unroll
        for (int j = 0; j < KL; ++j) { st.v[j] = -INFINITY; st.ix[j] = -1; }
    }
    static constexpr int kThreads = kGemmEpiWarps * 32;
    // the largest float below x (-inf: itself)
    static __device__ __forceinline__ float below(float x) {
        if (x == -INFINITY) return x;
        const int b = __float_as_int(x + 0.0f);
        return b == 0 ? -__int_as_float(1) : __int_as_float(b > 0 ? b - 1 : b + 1);
    }
    // columns past the vocabulary: below every logit
    static __device__ __forceinline__ void mask(float (&x)[16], int live) {
        if (live < 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = i < live ? x[i] : -INFINITY;
        }
    }
    // Adds 2^t and t 2^t of a run's columns.  PART: of the first `live` of them; that the others' terms are 0
    // cannot be left to the exponential, which a scale near 0 takes to 1 for any finite logit.
    template <bool PART>
    static __device__ __forceinline__ void add_terms(const float (&x)[16], int live, float nm, float c, float (&s)[2], float (&e)[2]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float t = !PART || i < live ? (x[i] - nm) * c : 0.0f;
            const float p = !PART || i < live ? ex2_approx(t) : 0.0f;
            s[i & 1] += p;
            e[i & 1] = fmaf(p, t, e[i & 1]);
        }
    }
    static __device__ __forceinline__ void tile(State& st, const Params& ep, int m, const AccColumns& cols, unsigned char* scratch) {
        float g[KL];
        if constexpr (KR > 0) {
#pragma unroll
            for (int j = 0; j < KL; ++j) g[j] = -INFINITY;
        }
        for (int ch = cols.ch0; ch < cols.ch1; ++ch) {
            float x[16];
            const int live = cols.load(ch, x), col = cols.col0 + ch * 16;
            if (live <= 0) break;
            mask(x, live);
            float gm[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) gm[i] = fmaxf(fmaxf(x[4 * i], x[4 * i + 1]), fmaxf(x[4 * i + 2], x[4 * i + 3]));
            const float nm = fmaxf(st.mx, fmaxf(fmaxf(gm[0], gm[1]), fmaxf(gm[2], gm[3])));
            const float back = st.s > 0.0f ? (st.mx - nm) * ep.c : 0.0f, f = ex2_approx(back);     // nothing summed yet: nothing to rescale
            float s2[2] = {0.0f, 0.0f}, e2[2] = {0.0f, 0.0f};
            if (live >= 16) add_terms<false>(x, 16, nm, ep.c, s2, e2);
            else add_terms<true>(x, live, nm, ep.c, s2, e2);
            st.e = fmaf(f, fmaf(back, st.s, st.e), e2[0] + e2[1]);
            st.s = fmaf(f, st.s, s2[0] + s2[1]);
            st.mx = nm;
            const int at = st.tok - col;
            if ((unsigned)at < (unsigned)min(live, 16)) {
                float t = x[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) t = at == i ? x[i] : t;
                ep.rec.given[m] = t;
            }
            if constexpr (KR == kKeepLogits) {
                if (m < ep.M) {            // rows are whole runs of 16 columns long
                    float4* to = reinterpret_cast<float4*>(ep.rec.logits + (size_t)m * ep.rec.ld + col);
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                }
            }
            if constexpr (KR > 0) {
                if (st.first) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) vals_insert<KL>(g, gm[i]);
                }
            }
        }
        if constexpr (KR > 0) {
            // The logits that may be among the row's best - above the list's last entry, and in the thread's first tile not
            // below the KR-th largest of the maxima of groups of four, which KR logits reach - are queued (lanes meet
            // theirs at different columns) and inserted together, one per lane and turn.
            if (st.first) st.bound = below(g[KL - 1]);
            st.first = false;
            const uint32_t qx0 = smem_u32(scratch) + threadIdx.x * 4u;
            const uint32_t qc0 = smem_u32(scratch) + kListQueue * kThreads * 4u + threadIdx.x;
            uint32_t qx = qx0, qc = qc0;
            auto insert_queued = [&]() {
                const int cnt = (int)(qx - qx0) / (kThreads * 4);
                const int most = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)cnt);
                for (int i = 0; i < most; ++i) {
                    const float x = i < cnt ? reinterpret_cast<const float*>(scratch)[i * kThreads + threadIdx.x] : -INFINITY;   // beats nothing
                    rows_insert<KL>(st.v, st.ix, x, cols.col0 + (int)scratch[kListQueue * kThreads * 4 + i * kThreads + threadIdx.x]);
                }
                qx = qx0;
                qc = qc0;
            };
            for (int ch = cols.ch0; ch < cols.ch1; ++ch) {
                float x[16];
                const int live = cols.load(ch, x);
                if (live <= 0) break;
                mask(x, live);
                const float tau = fmaxf(st.v[KL - 1], st.bound);
#pragma unroll
                for (int i = 0; i < 16; ++i)       // without a branch: a few of a warp's 32 rows queue something at nearly every column
                    asm volatile(
                        "{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %2, %3;\n\t@p st.shared.f32 [%0], %2;\n\t@p st.shared.u8 [%1], %4;\n\t"
                        "@p add.u32 %0, %0, %5;\n\t@p add.u32 %1, %1, %6;\n\t}"
                        : "+r"(qx), "+r"(qc) : "f"(x[i]), "f"(tau), "r"(ch * 16 + i), "n"(kThreads * 4), "n"(kThreads) : "memory");
                if (__any_sync(0xFFFFFFFFu, qx - qx0 > (uint32_t)(kListQueue - 16) * kThreads * 4)) insert_queued();
            }
            insert_queued();
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
constexpr int kJoinHeld = 8;               // records a thread keeps in registers
constexpr int kJoinRanges = 512;

struct ScoreJoin {
    ScoreRecords rec;
    ScoreOut out;
    const int32_t* tokens;
    int V;
    float scale;
};

// Sum (SUM) or maximum over the block, the same bits in every thread.
template <int T, bool SUM>
__device__ __forceinline__ float block_reduce(float v, float* buf) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float r = __shfl_xor_sync(0xFFFFFFFFu, v, d);
        v = SUM ? v + r : fmaxf(v, r);
    }
    if constexpr (T > 32) {
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
        __syncthreads();
        v = buf[0];
#pragma unroll
        for (int w = 1; w < T / 32; ++w) v = SUM ? v + buf[w] : fmaxf(v, buf[w]);
    }
    return v;
}

// One block per row.  Nothing but latency bounds it: a thread's records are all requested before the first is used, and
// the steps between barriers are short.  256 threads for few rows, one warp where the rows fill the SMs by themselves
// (4096 rows, k = 4: 29 us of 128-thread blocks before, see the launch rule).
template <int T, bool KEPT>
__global__ void __launch_bounds__(T) score_join_kernel(const ScoreJoin p) {
    constexpr int kCand = T >= 128 ? 1024 : 256;
    __shared__ float buf[3][T / 32];
    __shared__ __align__(16) uint32_t heads[T];
    __shared__ unsigned long long cand[kCand], wins[T / 32];
    __shared__ int n_cand, n_ranges, ranges[KEPT ? kJoinRanges : 1];
    const int m = blockIdx.x, t = threadIdx.x, L = p.rec.L, k = p.out.k;
    const ScoreOut& o = p.out;
    if (t == 0) n_cand = n_ranges = 0;
    grid_dependency_wait();
    const float4* stats = p.rec.stats + (size_t)m * L;
    const unsigned long long* keys = p.rec.keys + (size_t)m * L * k;
    const float c = exponent_scale(p.scale);
    const bool scored = row_scored(p.tokens, p.V, m);
    const float given = p.tokens != nullptr ? p.rec.given[m] : 0.0f;      // stale where the row is not scored, and then not used
    // a thread's records in registers, with the best key of each; kept: the range by its maximum
    float4 r[kJoinHeld];
    unsigned long long held[kJoinHeld];
#pragma unroll
    for (int i = 0; i < kJoinHeld; ++i) {
        const int l = t + i * T;
        r[i] = l < L ? stats[l] : make_float4(kLowest, 0.0f, 0.0f, 0.0f);
        if constexpr (!KEPT) held[i] = l < L && k > 0 ? keys[(size_t)l * k] : 0ull;
    }
    if (!scored) {
        if (t == 0) {
            if (o.logprobs) o.logprobs[m] = 0.0f;
            if (o.entropy) o.entropy[m] = 0.0f;
            if (o.lse) o.lse[m] = 0.0f;
        }
        for (int j = t; j < k; j += T) {
            o.top_ids[(size_t)m * k + j] = -1;
            o.top_logprobs[(size_t)m * k + j] = 0.0f;
        }
        return;
    }
    auto range_key = [](const float4& q) { return q.y > 0.0f ? make_key(q.x, 0) : 0ull; };
    float mx = kLowest;
    uint32_t head = 0u;
#pragma unroll
    for (int i = 0; i < kJoinHeld; ++i) {
        if constexpr (KEPT) held[i] = range_key(r[i]);
        mx = fmaxf(mx, r[i].x);
        head = max(head, (uint32_t)(held[i] >> 32));
    }
    for (int l = t + kJoinHeld * T; l < L; l += T) {
        const float4 q = stats[l];
        mx = fmaxf(mx, q.x);
        if (k > 0) head = max(head, (uint32_t)((KEPT ? range_key(q) : keys[(size_t)l * k]) >> 32));
    }
    heads[t] = head;
    mx = block_reduce<T, false>(mx, buf[0]);
    float s = 0.0f, e = 0.0f;
    auto fold = [&](const float4& q) {
        const float back = q.y > 0.0f ? (q.x - mx) * c : 0.0f, f = ex2_approx(back);       // a record of no columns adds 0
        s = fmaf(f, q.y, s);
        e = fmaf(f, fmaf(back, q.y, q.z), e);
    };
#pragma unroll
    for (int i = 0; i < kJoinHeld; ++i) fold(r[i]);
    for (int l = t + kJoinHeld * T; l < L; l += T) fold(stats[l]);
    s = block_reduce<T, true>(s, buf[1]);
    e = block_reduce<T, true>(e, buf[2]);
    const float log_s = logf(s);
    if (t == 0) {
        if (o.lse) o.lse[m] = fmaf(p.scale, mx, log_s);
        if (o.entropy) o.entropy[m] = log_s - kLn2 * (e / s);
        if (o.logprobs) o.logprobs[m] = p.scale * (given - mx) - log_s;
    }
    if (k == 0) return;

    // The k-th largest of the maxima of 64 (32) groups of ranges bounds the winners from below: k logits at least that large
    // exist.  The logits not below it are gathered, and a key's place is the number of keys above it.  Every warp finds the
    // bound for itself, in k rounds of a warp-wide maximum (equal maxima leave together: the bound is then lower, and holds).
    __syncthreads();
    uint32_t g0 = 0u, g1 = 0u, b = 0u;
    if constexpr (T == 32) {
        g0 = head;
    } else {
#pragma unroll
        for (int i = 0; i < T / 64; ++i) {
            const uint2 h = *reinterpret_cast<const uint2*>(heads + 64 * i + 2 * (t & 31));
            g0 = max(g0, h.x);
            g1 = max(g1, h.y);
        }
    }
    for (int j = 0; j < k; ++j) {
        b = __reduce_max_sync(0xFFFFFFFFu, max(g0, g1));
        g0 = g0 == b ? 0u : g0;
        g1 = g1 == b ? 0u : g1;
    }
    const unsigned long long bound = b != 0u ? (unsigned long long)b << 32 : 1ull;   // 1 (every key) when fewer than k groups have one
    auto candidate = [&](unsigned long long key) {
        const int at = atomicAdd(&n_cand, 1);          // the order of the candidates does not matter: their ranks decide
        if (at < kCand) cand[at] = key;
    };
    const float* row = p.rec.logits + (size_t)m * p.rec.ld;
    if constexpr (KEPT) {
        // the ranges that reach the bound ...
        auto gather = [&](int l, unsigned long long key) {
            if (key < bound) return;
            const int at = atomicAdd(&n_ranges, 1);
            if (at < kJoinRanges) ranges[at] = l;
        };
#pragma unroll
        for (int i = 0; i < kJoinHeld; ++i) gather(t + i * T, held[i]);
        for (int l = t + kJoinHeld * T; l < L; l += T) gather(l, range_key(stats[l]));
        __syncthreads();
        // ... and their logits: a warp per range, a lane per four columns, four tiles in flight
        const float bound_x = b != 0u ? key_logit(bound) : -INFINITY;
        const bool all = n_ranges > kJoinRanges;       // more than the buffer names: every range
        const int nr = all ? L : n_ranges, nch = p.rec.NT >> 4, tiles = p.rec.tiles_per_item;
        for (int i = t >> 5; i < nr; i += T / 32) {
            const int l = all ? i : ranges[i];
            const int item = l / p.rec.parts, part = l - item * p.rec.parts;
            const int c0 = part * nch / p.rec.parts * 16 + (t & 31) * 4, c1 = (part + 1) * nch / p.rec.parts * 16;
            const int first = item * tiles * p.rec.NT;
            for (int cc = c0; cc < c1; cc += 128)
                for (int tile = 0; tile < tiles; tile += 4) {
                    float4 x[4];
                    int col[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        col[u] = first + (tile + u) * p.rec.NT + cc;
                        if (tile + u >= tiles) col[u] = p.V;
                        if (col[u] < p.V) x[u] = *reinterpret_cast<const float4*>(row + col[u]);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (col[u] + q < p.V && v[q] >= bound_x) candidate(make_key(v[q], col[u] + q));
                    }
                }
        }
    } else {
        auto gather = [&](int l, unsigned long long key) {
            for (int j = 0; key >= bound;) {
                candidate(key);
                if (++j == k) break;
                key = keys[(size_t)l * k + j];
            }
        };
#pragma unroll
        for (int i = 0; i < kJoinHeld; ++i) gather(t + i * T, held[i]);
        for (int l = t + kJoinHeld * T; l < L; l += T) gather(l, keys[(size_t)l * k]);
    }
    __syncthreads();
    const int n = n_cand;
    auto emit = [&](int j, unsigned long long key) {
        const size_t at = (size_t)m * k + j;
        o.top_ids[at] = key != 0ull ? key_index(key) : -1;
        o.top_logprobs[at] = key != 0ull ? p.scale * (key_logit(key) - mx) - log_s : -INFINITY;
    };
    if (n <= kCand) {
        for (int i = t; i < n; i += T) {
            const unsigned long long key = cand[i];
            int above = 0;
#pragma unroll 4
            for (int q = 0; q < n; ++q) above += cand[q] > key ? 1 : 0;
            if (above < k) emit(above, key);
        }
        for (int j = n + t; j < k; j += T) emit(j, 0ull);
        return;
    }
    // Too many for the buffer (ties, or winners in few lists): the largest key below the last winner, k times.
    unsigned long long last = ~0ull;
    for (int j = 0; j < k; ++j) {
        unsigned long long best = 0ull;
        if constexpr (KEPT) {
            for (int col = t; col < p.V; col += T) {
                const unsigned long long key = make_key(row[col], col);
                if (key < last && key > best) best = key;
            }
        } else {
            for (int l = t; l < L; l += T)
                for (int i = 0; i < k; ++i) {
                    const unsigned long long key = keys[(size_t)l * k + i];
                    if (key < last) { best = key > best ? key : best; break; }
                }
        }
        best = warp_max_key(best);
        __syncthreads();
        if ((t & 31) == 0) wins[t >> 5] = best;
        __syncthreads();
        for (int i = 0; i < T / 32; ++i) best = wins[i] > best ? wins[i] : best;
        if (t == 0) emit(j, best);
        last = best;
    }
}

// ------------------------------------------------------------------------------------------ host
static int list_entries(int k) { return k == 0 ? 0 : k <= 4 ? 4 : k <= 8 ? 8 : kListMax; }
// Whether the logits are kept (see the top of this file): always where a list would be too long, for long lists up to where
// the bytes cost as much, and for short ones only where so few rows leave the epilogue uncovered.
static bool keep_logits(int M, int k, size_t bytes) {
    if (k == 0) return false;
    if (k > kListMax) return true;
    return bytes <= (k > 8 ? (size_t)40 << 20 : M <= 128 ? (size_t)8 << 20 : 0);
}

struct ScorePlan {
    GemmParams p;
    bool pair;
    int KR;
    int64_t ld;
    int L;
    size_t stats, keys, logits, given, total;      // offsets in the workspace
};

static bool score_plan(int M, int d, int V, int k, ScorePlan* s) {
    s->p = GemmParams{};
    s->p.n_prob = 1;
    s->p.prob[0].M = M;
    s->p.prob[0].N = V;
    s->p.prob[0].b0 = 1;
    s->p.prob[0].nk0 = ceil_div(d, kBoxK);
    s->ld = (int64_t)round_up((size_t)V, 16);
    const size_t kept = (size_t)M * s->ld * 4;
    s->KR = keep_logits(M, k, kept) ? kKeepLogits : list_entries(k);
    if (!gemm_plan_rows(&s->p, s->KR > 0 ? EpiScore<4>::kScratch : 0u, s->KR > 0, &s->pair)) return false;
    s->L = s->p.prob[0].chunks_n * 2 * s->p.rep;
    const size_t rows = (size_t)M * s->L;
    s->stats = kHeaderBytes;
    s->keys = s->stats + round_up(rows * sizeof(float4), 256);
    s->logits = s->keys + (s->KR > 0 ? round_up(rows * k * 8, 256) : 0);
    s->given = s->logits + (s->KR == kKeepLogits ? round_up(kept, 256) : 0);
    s->total = s->given + round_up((size_t)M * 4, 256);
    return true;
}

size_t score_workspace_bytes(int M, int d, int V, int k) {
    ScorePlan s;
    return score_plan(M, d, V, k, &s) ? s.total : 0;
}

template <int KR>
static vt_status run_score(const GemmMaps& maps, const ScorePlan& s, const ScoreCall& c, const ScoreRecords& rec, const ScoreOut& o,
                           cudaStream_t st) {
    const typename EpiScore<KR>::Params ep{c.tokens, rec, exponent_scale(c.scale), c.M, c.V, o.k};
    vt_status r = gemm_launch<false, false, EpiScore<KR>>(maps, s.p, s.pair, ep, st);
    if (r != VT_OK) return r;
    const ScoreJoin join{rec, o, c.tokens, c.V, c.scale};
    constexpr bool kept = KR == kKeepLogits;
    // Few rows: 256 threads each.  Many: one warp for short lists (it bounds 32 winners at most), four for kept ranges, which
    // are read one per warp at a time.
    const bool many = c.M > 2 * kGemmSms;
    cudaError_t e;
    if (many && kept) e = launch_pdl(score_join_kernel<128, kept>, c.M, 128, 0, st, join);
    else if (many && o.k <= 32) e = launch_pdl(score_join_kernel<32, kept>, c.M, 32, 0, st, join);
    else e = launch_pdl(score_join_kernel<256, kept>, c.M, 256, 0, st, join);
    count_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

vt_status launch_score(const ScoreCall& c, const ScoreOut& o, void* workspace, size_t workspace_bytes, cudaStream_t st) {
    ScorePlan s;
    if (!score_plan(c.M, c.d, c.V, o.k, &s)) return VT_ERR_SHAPE;
    if (workspace_bytes < s.total) return VT_ERR_WORKSPACE;
    unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
    s.p.hdr = reinterpret_cast<WsHeader*>(base);
    ScoreRecords rec;
    rec.stats = reinterpret_cast<float4*>(base + s.stats);
    rec.keys = reinterpret_cast<unsigned long long*>(base + s.keys);
    rec.logits = reinterpret_cast<float*>(base + s.logits);
    rec.given = reinterpret_cast<float*>(base + s.given);
    rec.ld = s.ld;
    rec.L = s.L;
    rec.parts = 2 * s.p.rep;
    rec.NT = s.p.NT;
    rec.tiles_per_item = s.p.tiles_per_item;
    GemmMaps maps{};
    vt_status r = gemm_map(&maps.map[0], GemmOperand{c.h, c.M, c.d, c.ldh}, gemm_box_a(s.p, false));
    if (r != VT_OK) return r;
    if ((r = gemm_map(&maps.map[1], GemmOperand{c.W, c.V, c.d, c.d}, gemm_box_b(s.p, false, s.pair))) != VT_OK) return r;
    switch (s.KR) {
        case kKeepLogits: return run_score<kKeepLogits>(maps, s, c, rec, o, st);
        case 0: return run_score<0>(maps, s, c, rec, o, st);
        case 4: return run_score<4>(maps, s, c, rec, o, st);
        case 8: return run_score<8>(maps, s, c, rec, o, st);
        default: return run_score<kListMax>(maps, s, c, rec, o, st);
    }
}

}  // namespace vt
