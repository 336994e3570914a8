// Verification of drafted tokens against the target's probabilities (see vt_verify_tokens).
//
// A cluster of eight CTAs takes a request.  Which child of a node is looked at next depends on the last answer, but what an answer needs,
// p[parent][token] and q[parent][token], does not: all of them are fetched at once, and the way down the tree is then a walk through shared
// memory that every CTA makes for itself.  Only the rows' sums need the cluster: each CTA owns an eighth of the vocabulary, adds up its part
// in 64 bits in a fixed order and gives the sum to the others through distributed shared memory.  The token that follows is found from the
// sums: the CTA, then the warp whose range the target falls into, then the lane's thirty-second of that, then the id.
//
// After j rejections at a node what is left is max(p - S q, 0) with one number S, because max(max(a - b, 0) - c, 0) = max(a - b - c, 0) for
// c >= 0: no row is written anywhere.  q lives on the trimmed vocabulary, so the node's q is laid out over the CTAs' ids in shared memory
// first: each CTA sends an eighth of q to where d2t says.
// Drafts chosen without chance need no sums on the way (Z falls by p of each child), and a bitmap of rejected children in q's place.
//
// Bound: latency.  Seven memory round trips follow one another (offsets, nodes, gathers, q, the row, a lane's part of it, the id); the bytes of
// one row of p (and q) per request take a tenth of that for 16 requests.  (Going through the warp's range 32 ids at a time, each behind a load,
// took 17 of 23 us.)
#include "vt_step.h"
#include "vt_tc.cuh"

namespace vt {

constexpr int kVerifyCtas = 8;               // per request
constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
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
    const int first_id = (int)rank * prm.share, ids = max(0, min(prm.share, c.V - first_id));
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
    // lays out q of a node, or its children
    bool cleared = true;
    auto lay_out = [&](int x) {
        if (!cleared) {
            __syncthreads();                 // the last node's has been read
            clear();
            if (DRAWN) cluster_sync_all();
            else __syncthreads();
        }
        cleared = false;
        if (DRAWN) {
            const float* q = c.draft_probs + (int64_t)(begin + x) * c.ld_draft;
            if (c.d2t) {
                const int i0 = (int)((long long)c.Vd * rank / kVerifyCtas), i1 = (int)((long long)c.Vd * (rank + 1) / kVerifyCtas);
#pragma unroll 8
                for (int i = i0 + tid; i < i1; i += kVerifyThreads) {
                    const int at = c.d2t[i];
                    const float v = fmaxf(q[i], 0.0f);
                    if ((unsigned)at < (unsigned)c.V) {
                        const unsigned owner = (unsigned)at / (unsigned)prm.share;
                        asm volatile("st.shared::cluster.f32 [%0], %1;"
                                     ::"r"(cluster_map_shared(smem_u32(left_q + ((unsigned)at - owner * (unsigned)prm.share)), owner)), "f"(v) : "memory");
                    }
                }
                cluster_sync_all();
            } else {
                for (int i = tid; i < min(ids, c.Vd - first_id); i += kVerifyThreads) left_q[i] = fmaxf(q[first_id + i], 0.0f);
                __syncthreads();
            }
        } else {
            for (int t = tid; t < T; t += kVerifyThreads) {
                const unsigned at = (unsigned)(node_token[t] - first_id);
                if (node_parent[t] == x && at < (unsigned)ids) atomicOr(&out_bits[at >> 5], 1u << (at & 31));
            }
            __syncthreads();
        }
    };
    // what is left of id first_id + i, whose probability is p
    auto left = [&](float p, int i, double S, bool whole) -> double {
        if (whole) return p > 0.0f ? (double)p : 0.0;
        if (DRAWN) return fmax((double)fmaxf(p, 0.0f) - S * (double)left_q[i], 0.0);
        return p > 0.0f && !(out_bits[i >> 5] >> (i & 31) & 1u) ? (double)p : 0.0;
    };
    // this thread's part of the sum of what is left after node x; a warp's ids are consecutive
    const int per_warp = prm.share / kVerifyWarps;
    const bool vector = (c.ld_probs & 3) == 0 && (reinterpret_cast<uintptr_t>(c.probs) & 15u) == 0;
    auto part = [&](int x, double S, bool whole) -> double {
        const float* row = c.probs + (int64_t)(begin + x) * c.ld_probs + first_id;
        const int i0 = warp * per_warp, i1 = min(i0 + per_warp, ids);
        double sum = 0.0;
        if (vector) {
#pragma unroll 8
            for (int i = i0 + 4 * lane; i + 3 < i1; i += 128) {
                const float4 p = *reinterpret_cast<const float4*>(row + i);
                sum += (left(p.x, i, S, whole) + left(p.y, i + 1, S, whole)) + (left(p.z, i + 2, S, whole) + left(p.w, i + 3, S, whole));
            }
            const int rest = i0 + (max(i1 - i0, 0) & ~3) + lane;
            if (rest < i1) sum += left(row[rest], rest, S, whole);
        } else {
#pragma unroll 8
            for (int i = i0 + lane; i < i1; i += 32) sum += left(row[i], i, S, whole);
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
        double total = Z;
        if (!summed) {
            if (!whole) lay_out(x);
            total = cluster_total(part(x, S, whole), warp_sums, cta_sums[buffer ^= 1], rank);
        }
        if (!(total > 0.0) && !whole) {      // the same in every CTA
            whole = true;
            total = cluster_total(part(x, S, whole), warp_sums, cta_sums[buffer ^= 1], rank);
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
                const float* row = c.probs + (int64_t)(begin + x) * c.ld_probs + first_id;
                const int i0 = warp * per_warp, i1 = min(i0 + per_warp, ids);
                // a lane per run of `len` consecutive ids: the run whose sum goes past the target (or the last with anything in it) ...
                const int len = per_warp / 32, r0 = i0 + lane * len, r1 = min(r0 + len, i1);
                double run = 0.0;
                if (vector) {
#pragma unroll 8
                    for (int i = r0; i + 3 < r1; i += 4) {
                        const float4 p = *reinterpret_cast<const float4*>(row + i);
                        run += (left(p.x, i, S, whole) + left(p.y, i + 1, S, whole)) + (left(p.z, i + 2, S, whole) + left(p.w, i + 3, S, whole));
                    }
                    for (int i = r0 + (max(r1 - r0, 0) & ~3); i < r1; ++i) run += left(row[i], i, S, whole);
                } else {
#pragma unroll 8
                    for (int i = r0; i < r1; ++i) run += left(row[i], i, S, whole);
                }
                auto up_to = [&](double v) {                 // sum over the lanes up to this one
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double w = __shfl_up_sync(0xFFFFFFFFu, v, o);
                        if (lane >= o) v += w;
                    }
                    return v;
                };
                const double cum = before + up_to(run);
                const unsigned some = __ballot_sync(0xFFFFFFFFu, run > 0.0);
                const unsigned over = __ballot_sync(0xFFFFFFFFu, !past_w && run > 0.0 && cum > target);
                const int at = over ? __ffs((int)over) - 1 : some ? 31 - __clz((int)some) : 0;
                const bool past_r = over == 0;
                before = __shfl_sync(0xFFFFFFFFu, cum - run, at);
                // ... and in it the id
                int found = -1, latest = -1;
                for (int i = i0 + at * len, e = min(i + len, i1); i < e && found < 0; i += 32) {
                    const double l = i + lane < e ? left(row[i + lane], i + lane, S, whole) : 0.0;
                    const double c32 = before + up_to(l);
                    const unsigned any = __ballot_sync(0xFFFFFFFFu, l > 0.0), past = __ballot_sync(0xFFFFFFFFu, !past_r && l > 0.0 && c32 > target);
                    if (past) found = i + __ffs((int)past) - 1;
                    if (any) latest = i + 31 - __clz((int)any);
                    before = __shfl_sync(0xFFFFFFFFu, c32, 31);
                }
                if (found < 0) found = latest;
                if (lane == 0) c.out_tokens[(int64_t)b * c.max_tokens + n] = found < 0 ? -1 : first_id + found;
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
    p.share = (int)(((long long)c.V + kVerifyCtas * kVerifyRun - 1) / (kVerifyCtas * kVerifyRun)) * kVerifyRun;
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
