// Verification of drafted tokens against the target's probabilities (see vt_verify_tokens).
//
// A cluster of eight CTAs takes a request.  Which child of a node is looked at next depends on the last answer, but what an answer needs,
// p[parent][token] and q[parent][token], does not: all of them are fetched at once, and the way down the tree is then a walk through shared
// memory that every CTA makes for itself.  Only the rows' sums need the cluster: each CTA owns an eighth of the vocabulary, adds up its part
// in 64 bits in a fixed order and gives the sum to the others through distributed shared memory.  The token that follows is found from the
// sums: the CTA, then the warp whose range the target falls into, then 128 ids of it, four of those, the id.
//
// After j rejections at a node what is left is max(p - S q, 0) with one number S, because max(max(a - b, 0) - c, 0) = max(a - b - c, 0) for
// c >= 0: no row is written anywhere.  q lives on the trimmed vocabulary, so the node's q is laid out over the CTAs' ids in shared memory
// first: each CTA sends an eighth of q to where d2t says.
// Drafts chosen without chance need no sums on the way (Z falls by p of each child), and a bitmap of rejected children in q's place.
//
// Bound: latency.  Seven memory round trips follow one another (offsets, nodes, gathers, q, the row, a part of it again, four ids), with two
// to four synchronisations of a cluster between them; the bytes of one row of p (and q) per request take a tenth of that for 16 requests.
// Measured with a vocabulary of 128256, in a graph: one chain of six drawn from 32000 ids 13.0 us, 16 trees of 60 best ones 10.7 us, 64 chains of
// eight 37 us drawn and 22 us best (bytes: 8 and 5): 512 CTAs at two per SM are 1.7 waves, each with the whole chain of round trips.
// The code is fetched as it goes, once per call and SM, so less of it is faster: the sum in one loop in place of a vector and a scalar one, and
// the target sought by warp sums of 128 ids in place of lanes with runs of their own, took the 16 trees from 12.6 us to 10.7.  (Sums of 128 ids
// kept by every warp for the search: 15 us.  1024 threads a CTA: 22 us.  q found through an index of the ids instead of laid out: a drawn chain
// 15.0 us.  One id per lane and load, which needs no boundaries: 11.3 and 14.2 us.)
#include "vt_step.h"
#include "vt_tc.cuh"

namespace vt {

constexpr int kVerifyCtas = 8;               // per request
constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyBatch = 4;              // entries of q that a thread has on their way
constexpr int kVerifyRuns = 4;               // runs of 128 ids that a warp looks through at once
constexpr int kVerifyRun = kVerifyWarps * 128;       // a CTA's share of the vocabulary is a multiple of it: whole runs of 128 per warp

struct VerifyParams {
    VerifyCall c;
    int share;                               // ids per CTA
};

// Adds up one value per thread (across lanes, then warps), then one per CTA of the cluster in the order of their ranks.
// Every thread gets the total; warp_sums and cta_sums keep the parts.  cta_sums is written by the other CTAs: the caller alternates two.
__device__ __forceinline__ double cluster_total(double x, double* warp_sums, double* cta_sums, uint32_t rank) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    __syncthreads();                         // the last total's readers of warp_sums are done
    if (lane == 0) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        double s = lane < kVerifyWarps ? warp_sums[lane] : 0.0;
#pragma unroll
        for (int o = kVerifyWarps / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane < kVerifyCtas)
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(cluster_map_shared(smem_u32(cta_sums + rank), (uint32_t)lane)), "d"(s) : "memory");
    }
    cluster_sync_all();
    double total = 0.0;
    for (int r = 0; r < kVerifyCtas; ++r) total += cta_sums[r];
    return total;
}

template <bool DRAWN>
__global__ void __launch_bounds__(kVerifyThreads, 2)
verify_kernel(const __grid_constant__ VerifyParams prm) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double warp_sums[kVerifyWarps], cta_sums[2][kVerifyCtas];
    const VerifyCall& c = prm.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_cta_rank();
    const int b = blockIdx.x / kVerifyCtas;
    // A row of p is dealt out from the 16-byte boundary at or before its first id: with `skew` numbers before that, id i stands at i + skew, and
    // this CTA has the places first .. first + share - 1.
    const int first = (int)rank * prm.share;
    // this CTA's q (DRAWN), or a bit per id that is out; then the nodes
    float* left_q = reinterpret_cast<float*>(smem);
    uint32_t* out_bits = reinterpret_cast<uint32_t*>(smem);
    const uint32_t lead = DRAWN ? (uint32_t)prm.share * 4u : (uint32_t)prm.share / 8u;
    float* node_p = reinterpret_cast<float*>(smem + lead);
    float* node_q = node_p + c.max_tokens;
    float* node_u = node_q + c.max_tokens;
    int* node_token = reinterpret_cast<int*>(node_u + c.max_tokens);
    int* node_parent = node_token + c.max_tokens;
    int* path = node_parent + c.max_tokens;

    const int words = DRAWN ? prm.share : prm.share / 32;
    auto clear = [&]() {
        for (int i = 4 * tid; i < words; i += 4 * kVerifyThreads) *reinterpret_cast<uint4*>(out_bits + i) = make_uint4(0u, 0u, 0u, 0u);
    };
    clear();
    cluster_sync_all();                      // every CTA of the cluster runs, and has cleared its own, before another writes into its shared memory
    grid_dependency_wait();
    if (tid == 0) grid_launch_dependents();

    const int begin = min(max(c.cu_tokens[b], 0), c.N), end = min(max(c.cu_tokens[b + 1], begin), c.N);
    const int T = min(end - begin, c.max_tokens);
    for (int t = tid; t < T; t += kVerifyThreads) {
        const int up = c.parents[begin + t], token = c.tokens[begin + t];
        float p = 0.0f, q = 1.0f;
        bool in = t > 0 && up >= 0 && up < t && (unsigned)token < (unsigned)c.V;
        int di = 0;
        if (DRAWN) {
            di = c.draft_ids[begin + t];
            in = in && (unsigned)di < (unsigned)c.Vd;
        }
        if (in) {
            p = c.probs[(int64_t)(begin + up) * c.ld_probs + token];
            if (DRAWN) q = fmaxf(c.draft_probs[(int64_t)(begin + up) * c.ld_draft + di], 0.0f);
            node_u[t] = c.u_accept[begin + t];
        }
        node_p[t] = p > 0.0f ? p : 0.0f;
        node_q[t] = q;
        node_token[t] = token;
        node_parent[t] = in ? up : -1;
    }
    const double u_follow = fmax((double)c.u_sample[b], 0.0);
    __syncthreads();
    if (!DRAWN) {                            // a child with the token of an earlier one: nothing is left of it by then
        for (int t = tid; t < T; t += kVerifyThreads) {
            bool again = false;
            const int up = node_parent[t], token = node_token[t];
            for (int s = max(up, 0) + 1; s < t && up >= 0; ++s) again |= node_parent[s] == up && node_token[s] == token;
            if (again) node_p[t] = 0.0f;     // read by nobody else before the barrier
        }
        __syncthreads();
    }

    int buffer = 0;
    auto skew_of = [&](int x) { return (int)(reinterpret_cast<uintptr_t>(c.probs + (int64_t)(begin + x) * c.ld_probs) >> 2 & 3u); };
    // lays out q of a node; without q the children of the last one, once
    bool cleared = true;
    auto lay_out = [&](int x) {
        if (DRAWN && !cleared) {
            __syncthreads();                 // the last node's has been read
            clear();
            cluster_sync_all();
        }
        cleared = false;
        const int skew = skew_of(x);
        if (DRAWN) {
            const float* q = c.draft_probs + (int64_t)(begin + x) * c.ld_draft;
            if (c.d2t) {
                const int i0 = (int)((long long)c.Vd * rank / kVerifyCtas), i1 = (int)((long long)c.Vd * (rank + 1) / kVerifyCtas);
#pragma unroll 1
                for (int i = i0 + tid; i < i1; i += kVerifyBatch * kVerifyThreads) {
                    int at[kVerifyBatch];
                    float v[kVerifyBatch];
#pragma unroll
                    for (int k = 0; k < kVerifyBatch; ++k) {
                        const int e = min(i + k * kVerifyThreads, i1 - 1);
                        at[k] = c.d2t[e];
                        v[k] = q[e];
                    }
#pragma unroll
                    for (int k = 0; k < kVerifyBatch; ++k) {
                        if (i + k * kVerifyThreads >= i1 || (unsigned)at[k] >= (unsigned)c.V) continue;
                        const unsigned place = (unsigned)(at[k] + skew), owner = place / (unsigned)prm.share;
                        asm volatile("st.shared::cluster.f32 [%0], %1;"
                                     ::"r"(cluster_map_shared(smem_u32(left_q + (place - owner * (unsigned)prm.share)), owner)), "f"(fmaxf(v[k], 0.0f)) : "memory");
                    }
                }
                cluster_sync_all();
            } else {
                for (int i = max(skew - first, 0) + tid; i < min(prm.share, c.Vd + skew - first); i += kVerifyThreads) left_q[i] = fmaxf(q[first + i - skew], 0.0f);
                __syncthreads();
            }
        } else {
            for (int t = tid; t < T; t += kVerifyThreads) {
                const unsigned at = (unsigned)node_token[t] + (unsigned)skew - (unsigned)first;
                if (node_parent[t] == x && at < (unsigned)prm.share) atomicOr(&out_bits[at >> 5], 1u << (at & 31));
            }
            __syncthreads();
        }
    };
    const int per_warp = prm.share / kVerifyWarps;
    // what is left of this CTA's ids i .. i + 3 after node x, i a multiple of four; nothing of those outside start .. end - 1
    auto left4 = [&](const float* row, int i, int start, int end, double S, bool whole, double (&l)[4]) {
        float p[4];
        if (i >= start && i + 3 < end) {
            const float4 v = *reinterpret_cast<const float4*>(row + i);
            p[0] = v.x, p[1] = v.y, p[2] = v.z, p[3] = v.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = i + k >= start && i + k < end ? row[i + k] : 0.0f;
        }
        const int in = min(i, prm.share - 4);                // where p is 0 past it all
        if (DRAWN) {
            const float4 v = *reinterpret_cast<const float4*>(left_q + in);
            const float q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const double d = (double)fmaxf(p[k], 0.0f), less = fmax(d - S * (double)q[k], 0.0);
                l[k] = whole ? d : less;
            }
        } else {
            const uint32_t out = whole ? 0u : out_bits[in >> 5] >> (in & 31);
#pragma unroll
            for (int k = 0; k < 4; ++k) l[k] = out >> k & 1u ? 0.0 : (double)fmaxf(p[k], 0.0f);
        }
    };
    // this thread's part of the sum of what is left after node x; a warp's ids are consecutive
    auto part = [&](int x, double S, bool whole) -> double {
        const int skew = skew_of(x), start = max(skew - first, 0), i0 = warp * per_warp, i1 = min(i0 + per_warp, c.V + skew - first);
        const float* row = c.probs + (int64_t)(begin + x) * c.ld_probs + (first - skew);
        double sum = 0.0;
        if (DRAWN) {
            auto left = [&](float p, int i) {
                if (whole) return p > 0.0f ? (double)p : 0.0;
                return fmax((double)fmaxf(p, 0.0f) - S * (double)left_q[i], 0.0);
            };
            const int ahead = start > i0 ? 4 : 0;
#pragma unroll 8
            for (int i = i0 + ahead + 4 * lane; i + 3 < i1; i += 128) {
                const float4 p = *reinterpret_cast<const float4*>(row + i);
                sum += (left(p.x, i) + left(p.y, i + 1)) + (left(p.z, i + 2) + left(p.w, i + 3));
            }
            const int rest = max(i0 + ahead, i1 & ~3) + lane;
            if (rest < i1) sum += left(row[rest], rest);
            if (lane < ahead && lane >= start && lane < i1) sum += left(row[lane], lane);
            return sum;
        }
#pragma unroll 8
        for (int i = i0 + 4 * lane; i < i1; i += 128) {
            double l[4];
            left4(row, i, start, i1, S, whole, l);
            sum += (l[0] + l[1]) + (l[2] + l[3]);
        }
        return sum;
    };

    // ---- down the tree; every thread of every CTA takes the same way
    int x = 0, n = 0, laid = -1;
    double S = 0.0, Z = 1.0;
    bool summed = false;                     // Z is the sum of what is left, and its parts are in place
    for (int child = 1; T > 0;) {
        int next = T;                        // the next child of x
        for (int s = child; s < T; s += 32) {
            const unsigned found = __ballot_sync(0xFFFFFFFFu, s + lane < T && node_parent[min(s + lane, T - 1)] == x);
            if (found) {
                next = s + __ffs((int)found) - 1;
                break;
            }
        }
        if (next >= T) break;
        const double p = node_p[next], q = node_q[next];
        const double r = DRAWN ? fmax(p - S * q, 0.0) : p;
        if (r > 0.0 && (double)node_u[next] * q * Z < r) {
            if (tid == 0) path[n] = next;
            ++n;
            x = next;
            S = 0.0;
            Z = 1.0;
            summed = false;
        } else if (DRAWN) {
            S += Z;
            if (laid != x) lay_out(x);
            laid = x;
            Z = cluster_total(part(x, S, false), warp_sums, cta_sums[buffer ^= 1], rank);
            summed = true;
        } else {
            Z -= p;
        }
        child = next + 1;
    }

    // ---- the token that follows
    if (T > 0) {
        bool whole = DRAWN && !summed;
        if (!DRAWN) lay_out(x);
        double total = Z;
        for (bool known = summed;; known = false) {          // once more, of the whole row, where nothing is left; the same in every CTA
            if (!known) total = cluster_total(part(x, S, whole), warp_sums, cta_sums[buffer ^= 1], rank);
            if (total > 0.0 || whole) break;
            whole = true;
        }
        const double* sums = cta_sums[buffer];
        const double target = u_follow * total;
        // the first CTA, then the first warp, whose range goes past the target; the last with anything in it when rounding leaves none
        int own = -1, last = -1;
        double before = 0.0;
        for (int r = 0; r < kVerifyCtas && own < 0; ++r) {
            if (sums[r] > 0.0) last = r;
            if (before + sums[r] > target) own = r;
            else before += sums[r];
        }
        const bool past = own < 0;
        if (past) own = last;
        if (own == (int)rank) {
            int w = -1, last_w = -1;
            for (int i = 0; i < kVerifyWarps && w < 0; ++i) {
                if (warp_sums[i] > 0.0) last_w = i;
                if (!past && before + warp_sums[i] > target) w = i;
                else before += warp_sums[i];
            }
            const bool past_w = w < 0;
            if (past_w) w = last_w;
            if (w == warp) {
                const int skew = skew_of(x), start = max(skew - first, 0), i0 = warp * per_warp, i1 = min(i0 + per_warp, c.V + skew - first);
                const float* row = c.probs + (int64_t)(begin + x) * c.ld_probs + (first - skew);
                // the 128 ids whose sum goes past the target (or the last with anything in them), four such runs at a time ...
                int at = -1, last_at = -1;
                double before_last = before;
                for (int g = i0; g < i1 && at < 0; g += 128 * kVerifyRuns) {
                    double run[kVerifyRuns];
#pragma unroll
                    for (int k = 0; k < kVerifyRuns; ++k) {
                        double l[4];
                        left4(row, g + 128 * k + 4 * lane, start, i1, S, whole, l);
                        run[k] = (l[0] + l[1]) + (l[2] + l[3]);
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                        for (int k = 0; k < kVerifyRuns; ++k) run[k] += __shfl_xor_sync(0xFFFFFFFFu, run[k], o);
#pragma unroll
                    for (int k = 0; k < kVerifyRuns; ++k) {
                        if (at >= 0 || !(run[k] > 0.0)) continue;
                        last_at = g + 128 * k;
                        before_last = before;
                        if (!past_w && before + run[k] > target) at = last_at;
                        else before += run[k];
                    }
                }
                const bool past_r = at < 0;
                // ... and in it the id: the lane of four, then the one
                int found = -1;
                if (last_at >= 0) {
                    double l[4];
                    const int i = last_at + 4 * lane;
                    left4(row, i, start, i1, S, whole, l);
                    double upto = (l[0] + l[1]) + (l[2] + l[3]);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double w = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                        if (lane >= o) upto += w;
                    }
                    double c4 = before_last + __shfl_up_sync(0xFFFFFFFFu, upto, 1);
                    if (lane == 0) c4 = before_last;
                    int latest = -1;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        c4 += l[k];
                        if (l[k] > 0.0) {
                            latest = i + k;
                            if (found < 0 && !past_r && c4 > target) found = i + k;
                        }
                    }
                    const unsigned over = __ballot_sync(0xFFFFFFFFu, found >= 0), some = __ballot_sync(0xFFFFFFFFu, latest >= 0);
                    found = over ? __shfl_sync(0xFFFFFFFFu, found, __ffs((int)over) - 1) : some ? __shfl_sync(0xFFFFFFFFu, latest, 31 - __clz((int)some)) : -1;
                }
                if (lane == 0) c.out_tokens[(int64_t)b * c.max_tokens + n] = found < 0 ? -1 : first + found - skew;
            }
        }
        if (own < 0 && rank == 0 && tid == 0) c.out_tokens[(int64_t)b * c.max_tokens + n] = -1;
    }
    __syncthreads();                         // path
    if (rank == 0) {
        if (tid == 0) c.n_accepted[b] = n;
        for (int j = tid; j < c.max_tokens; j += kVerifyThreads) {
            const int64_t at = (int64_t)b * c.max_tokens + j;
            c.path[at] = j < n ? path[j] : -1;
            if (j < n) c.out_tokens[at] = node_token[path[j]];
            else if (j > n || T <= 0) c.out_tokens[at] = -1;
        }
    }
    cluster_sync_all();                      // nobody leaves while others' sums may still arrive
}

vt_status launch_verify(const VerifyCall& c, cudaStream_t st) {
    VerifyParams p{c, 0};
    const bool drawn = c.draft_probs != nullptr;
    const bool skewed = (c.ld_probs & 3) != 0 || (reinterpret_cast<uintptr_t>(c.probs) & 15u) != 0;
    p.share = (int)(((long long)c.V + (skewed ? 3 : 0) + kVerifyCtas * kVerifyRun - 1) / (kVerifyCtas * kVerifyRun)) * kVerifyRun;
    const size_t smem = (drawn ? (size_t)p.share * 4 : (size_t)p.share / 8) + (size_t)c.max_tokens * 24;
    static std::atomic<unsigned long long> configured[2];
    void (*kernel)(VerifyParams) = drawn ? verify_kernel<true> : verify_kernel<false>;
    if (vt_status r = ensure_max_dyn_smem(reinterpret_cast<const void*>(kernel), kMaxDynSmem - 1024, &configured[drawn]); r != VT_OK) return r;
    cudaError_t e = launch_pdl_cluster(kernel, kVerifyCtas, c.B * kVerifyCtas, kVerifyThreads, smem, st, p);
    count_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

}  // namespace vt
