// The matrix products behind token scoring and the gated feed-forward block: one tcgen05 kernel whose epilogue is a
// template parameter, for results of any size.
//
//   D[m, n] = sum_k A[m, k] * B[n, k]         bf16 operands, exact products, fp32 sums in tensor memory
//
// Either operand may be stored with k running fastest ([m][k], "K-major") or with m (n) running fastest ([k][m],
// "MN-major"): the tensor core takes both from a 128-byte swizzled TMA box, so no gradient needs a transposed copy.
// A launch takes one to three products (GemmProblem): a product may sum over two pairs of operands one after the other
// (dg Wg + du Wu), or its columns may come in two halves from two matrices (gate and up rows of one feature side by side
// in one accumulator).
//
// Work is cut into tiles of 128 or 256 rows x NT columns:
//   PAIR    clusters of two CTAs share each MMA (cta_group::2): 256 rows x NT <= 256 columns, either CTA fetches its
//           128 rows of A and half the columns of B.  For more than 128 rows: a CTA then moves 32 KB per 64-deep k-block
//           of 2 * 128 * 256 * 64 FLOP, half of what two separate 128 x 128 tiles would.
//   single  128 rows x NT <= 256 columns.  Few rows of A are fetched as a box of their own height; the MMA's other rows
//           compute on whatever shared memory holds and land in lanes nobody reads.  For an epilogue with work to do per
//           column (scoring) the tile can hold at most 64 (32) rows of A two (four) times, one copy per group of TMEM
//           lanes: every epilogue warp then finds rows, each copy taking its own share of the columns.
// bf16 results leave through shared memory, 128 bytes of a row at a time.  A thread's own 16-byte stores, 32 rows apart, held the
// tiles of short sums (dW of 300 rows) to 1.3 TB/s, TMA stores of 64-byte rows to 1.9.
//   splits  (single only) a cluster of up to eight CTAs divides the k range of one tile.  Each CTA owns a share of the
//           columns: the others write their partial sums of it into its shared memory, and it adds them up in the order
//           of the CTAs and finishes them: no atomics, the same bits every time.
// The CTAs are persistent (except with splits).  Warps 0-7: epilogue, warps 8 and 9: TMA producers, warp 10: MMA issuer;
// two accumulators in tensor memory, so the epilogue of a tile runs under the MMAs of the next.
// All waits are bounded; one that runs out sets the workspace's status word and the CTA unwinds.
#pragma once

#include "vt_common.cuh"
#include "vt_launch.h"
#include "vt_tc.cuh"

namespace vt {

constexpr int kGemmEpiWarps = 8;
constexpr int kGemmProducers = 2;           // they take the ring's stages in turn: issuing a stage's copies takes one warp 700 cycles
constexpr int kGemmThreads = (kGemmEpiWarps + kGemmProducers + 1) * 32;
constexpr int kGemmMaxStages = 16;
constexpr int kGemmMaxProblems = 3;
constexpr int kGemmMaxMaps = 6;
constexpr int kGemmGroupRows = 8;           // row tiles that share their column tiles before the next group (L2 reuse)
constexpr int kGemmSms = 148;               // the plans are made for this many SMs; a device with fewer runs them in more waves

struct GemmProblem {
    int M, N;                    // rows and columns of D (with `dual`: columns of either half)
    int a0, b0, nk0;             // tensor maps and 64-deep k-blocks of the first pair of operands
    int a1, b1, nk1;             // ... of the second (nk1 = 0: there is none)
    int tiles_m, chunks_n;       // row tiles; items along the columns
    int tiles_n;                 // column tiles
    int first_item;
};

struct GemmMaps {
    CUtensorMap map[kGemmMaxMaps];
};

struct GemmParams {
    GemmProblem prob[kGemmMaxProblems];
    int n_prob, n_items;
    int b_early;                 // 1: B's first stages are fetched ahead of the dependency wait.  For a call's second product and
                                 // later ones whose B the kernel just before does not write: every kernel here waits for its own
                                 // predecessor before it lets its successor start, so whatever was written ahead of the call or
                                 // by its earlier kernels is there.
    int tiles_per_item;          // consecutive column tiles of one row tile that a CTA takes in a row
    int NT;                      // accumulator columns of a tile
    int dual;                    // 1: columns [0, NT/2) from map b0, [NT/2, NT) from map b1, the same rows of both
    int rep;                     // copies of A's rows in a tile: 1, 2 or 4 (single only)
    int splits;                  // CTAs that share one tile's k range (single only)
    uint32_t x_rows, x_part;     // with splits: rows of the exchanged sums, and bytes an owner gets from each CTA (over the ring)
    int n_stages;
    int kbs;                     // k-blocks per ring stage
    uint32_t a_rows;             // rows of A's box (K-major); `rep` of them, 128 / rep rows apart
    uint32_t a_bytes, b_bytes;   // bytes of one k-block of A (B) in shared memory
    uint32_t tx_bytes;           // bytes a CTA's copies of one k-block deliver
    uint32_t blk_bytes, stage_bytes;     // one k-block of both; kbs of them
    uint32_t idesc;
    uint32_t tmem_cols, acc_cols;    // allocation; columns between the two accumulators
    uint32_t scratch_off;        // the epilogue's own shared memory (Epi::kScratch bytes), from the 1024-aligned base
    uint32_t bar_off;            // barriers
    uint32_t total_smem;
    unsigned long long wait_ns;      // limit of every wait
    WsHeader* hdr;
};

// A tile's place.
struct GemmItem {
    int prob, mt, nt0, n_tiles;
};

#ifdef __CUDACC__

__device__ __forceinline__ void acc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

// Descriptor of an MN-major bf16 tile as TMA boxes of 64 (m or n) x 64 (k) leave it: 64 elements of m are one 128-byte
// swizzled row, 8 k rows are 1024 bytes apart, the next 64 elements of m one box (8192 bytes) further on.
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t addr) {
    uint64_t desc = 0;
    desc |= (uint64_t)((addr & 0x3FFFFu) >> 4);
    desc |= (uint64_t)(8192 >> 4) << 16;                 // leading byte offset: between groups of 64 elements of m
    desc |= (uint64_t)(1024 >> 4) << 32;                 // stride byte offset: between groups of 8 k
    desc |= (uint64_t)1 << 46;
    desc |= (uint64_t)2 << 61;
    return desc;
}

// One arrival on an mbarrier of another CTA of the cluster that orders nothing in memory.
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t bar_cluster) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}

// One lane of a converged warp (the same one every time).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// The bounded wait by a whole warp, with an answer the compiler knows to be the same in every lane.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, limit_ns)) != 0;
}

__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// What the roles need of a launch's problems at every tile, in shared memory: loads from the parameters at a computed offset
// took each role over a thousand cycles a tile.
struct GemmTable {
    GemmProblem prob[kGemmMaxProblems];
};
__device__ __forceinline__ GemmItem gemm_item(const GemmTable& tab, int n_prob, int tiles_per_item, int item) {
    GemmItem it;
    it.prob = 0;
    while (it.prob + 1 < n_prob && item >= tab.prob[it.prob + 1].first_item) ++it.prob;
    const GemmProblem& q = tab.prob[it.prob];
    const unsigned local = (unsigned)(item - q.first_item);
    const unsigned per_group = (unsigned)(kGemmGroupRows * q.chunks_n);
    const unsigned g = local / per_group, r = local - g * per_group;
    const unsigned gm = (unsigned)min(kGemmGroupRows, q.tiles_m - (int)g * kGemmGroupRows);
    const unsigned ch = gm == kGemmGroupRows ? r / kGemmGroupRows : r / gm;
    it.mt = (int)(g * kGemmGroupRows + (r - ch * gm));
    it.nt0 = (int)ch * tiles_per_item;
    it.n_tiles = min(tiles_per_item, q.tiles_n - it.nt0);
    return it;
}

// A thread's share of a finished tile: runs [ch0, ch1) of 16 accumulator columns of its row.
struct AccColumns {
    uint32_t taddr;              // tensor-memory address of the row group's column 0
    int ch0, ch1;
    int col0, N;                 // the tile's first column of D; columns of D
    // all lanes must call it; returns how many of the 16 columns lie inside D (<= 0: none)
    __device__ __forceinline__ int load(int ch, float (&x)[16]) const {
        uint32_t u[16];
        __syncwarp();                // the lanes part where rows differ (given tokens, rows past the last)
        acc_ld16(taddr + (uint32_t)(ch * 16), u);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(u[e]);
        return N - (col0 + ch * 16);
    }
};

// Staging of bf16 results: per warp and output 32 rows of two units of 32 columns (one unit where there are several outputs),
// the 16-byte chunks of a row permuted so that neither a column of chunks nor a row of them meets a bank twice.
constexpr int gemm_stage_units(int outs) { return outs > 1 ? 1 : 2; }
constexpr uint32_t gemm_stage_bytes(int outs) { return kGemmEpiWarps * (uint32_t)(gemm_stage_units(outs) * outs) * 32u * 64u; }
template <int UNITS>
__device__ __forceinline__ uint32_t stage_offset(int row, int chunk) {
    return UNITS == 2 ? (uint32_t)row * 128u + (uint32_t)((chunk ^ (row & 7)) << 4) : (uint32_t)row * 64u + (uint32_t)((chunk ^ (row >> 1 & 3)) << 4);
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// Eight fp32 values as bf16 (nearest-even) to a 16-byte aligned address.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void store_bf16x8(uint16_t* at, const float* x) {
    *reinterpret_cast<uint4*>(at) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

__device__ __forceinline__ void st_shared_bf16x8(uint32_t at, const float (&x)[8]) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(pack_bf16(x[0], x[1])), "r"(pack_bf16(x[2], x[3])),
                 "r"(pack_bf16(x[4], x[5])), "r"(pack_bf16(x[6], x[7])) : "memory");
}

// Epilogue that rounds the sums once to bf16 and stores them row-major.
struct EpiStore {
    static constexpr bool kDual = false;
    static constexpr bool kStateful = false;
    static constexpr bool kSums = false;
    static constexpr int kOuts = 1;
    static constexpr uint32_t kScratch = gemm_stage_bytes(kOuts);
    struct Params {
        uint16_t* out[kGemmMaxProblems];      // [M, N] of each product
    };
    struct State {};
    static __device__ __forceinline__ void row(State&, const Params&, const GemmProblem&, int) {}
    static __device__ __forceinline__ void ahead(State&, const Params&, const GemmProblem&, int, int, int) {}
    static __device__ __forceinline__ void cols8(State&, const Params&, const GemmProblem&, int, int, int, const float (&x)[8], const float (&)[8], float (&out)[1][8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[0][i] = x[i];
    }
    static __device__ __forceinline__ uint16_t* at(const Params& ep, const GemmProblem& q, int prob, int, int m, int n) {
        return ep.out[prob] + (size_t)m * q.N + n;
    }
    static __device__ __forceinline__ int64_t ld(const Params&, const GemmProblem& q, int) { return q.N; }
};

// An epilogue provides kDual (its columns come in two halves) and either
//   kStateful   it works through all tiles of an item with a state of its own (never with splits): begin(), then tile() per
//               tile with its share of the columns, in runs of 16 that it reads through an AccColumns, then end()
// or kOuts bf16 matrices, each value from its own column(s):
//   row()       once per tile and row, before the accumulator is waited for
//   ahead()     two runs of 16 columns in advance: requests what cols8 will need for the run at column n, into slot 0 or 1
//   cols8()     eight columns (of either half), at e in the two slots' 32: out[o][i] are the values to round and store
//   at(), ld()  where output o's row m, column n lies; elements between its rows
// With kSums, rows that wants() names also have their sums stored in fp32, from sums() on.  (Not cols8's work: a branch in
// every eight columns kept them from being worked on side by side, 24 -> 31 us for 13264 x 2048 over 255.)
template <bool PAIR, bool A_MN, bool B_MN, class Epi>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmMaps maps, const __grid_constant__ GemmParams p,
            const __grid_constant__ typename Epi::Params ep) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char* smem = smem_raw + (base - raw);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kProducer = kGemmEpiWarps, kIssuer = kGemmEpiWarps + kGemmProducers;
    const int S = p.n_stages;
    const uint32_t rank = (PAIR || p.splits > 1) ? cluster_cta_rank() : 0u;
    const bool leader = !PAIR || rank == 0u;
    const int cluster = PAIR ? (int)blockIdx.x >> 1 : p.splits > 1 ? (int)blockIdx.x / p.splits : (int)blockIdx.x;
    const int n_clusters = PAIR ? (int)gridDim.x >> 1 : p.splits > 1 ? (int)gridDim.x / p.splits : (int)gridDim.x;

    const uint32_t bar_full = base + p.bar_off, bar_empty = bar_full + 8u * S;
    const uint32_t bar_accf = bar_empty + 8u * S, bar_acce = bar_accf + 16u, bar_drain = bar_acce + 16u;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + p.bar_off + 8u * (2 * S + 5));
    GemmTable& tab = *reinterpret_cast<GemmTable*>(smem + p.bar_off + 8u * (2 * S + 6));
    const int n_prob = p.n_prob, tiles_per_item = p.tiles_per_item;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    if (warp == kProducer && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.map[p.prob[0].a0]) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.map[p.prob[0].b0]) : "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(bar_full + 8u * s, 1);
            mbar_init(bar_empty + 8u * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_accf + 8u * b, 1);
            mbar_init(bar_acce + 8u * b, PAIR ? 2 * kGemmEpiWarps : kGemmEpiWarps);
        }
        mbar_init(bar_drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (tid >= 32 && tid < 32 + kGemmMaxProblems) tab.prob[tid - 32] = p.prob[tid - 32];
    if (warp == kIssuer) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(p.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(p.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_proxy_async();
    tc_fence_before();
    if constexpr (PAIR) cluster_sync_all();      // the other CTA's barriers are initialised before anything arrives on them
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // Nothing above touches global memory (the tensor maps are kernel parameters): under programmatic dependent launch it
    // overlaps the previous kernel's tail.
    const bool producer = warp >= kProducer && warp < kIssuer;
    if (!(p.b_early && producer)) grid_dependency_wait();
    if (tid == 0) grid_launch_dependents();

    auto fail = [&]() {
        *abort_flag = 1;
        atomicOr(&p.hdr->status, kStatusTimeout);
    };
    // the k-blocks of a product that this CTA multiplies
    auto k_range = [&](const GemmProblem& q, int& k0, int& k1) {
        const int nk = q.nk0 + q.nk1;
        k0 = p.splits > 1 ? (int)((long long)nk * (int)rank / p.splits) : 0;
        k1 = p.splits > 1 ? (int)((long long)nk * ((int)rank + 1) / p.splits) : nk;
    };
    // Where every CTA reads the same rows of A, each starts its k range somewhere else and wraps around: in step, they would
    // all ask for the same few lines of L2 at once.
    auto k_start = [&](const GemmProblem& q, int k0, int k1) {
        return !PAIR && q.tiles_m == 1 ? k0 + (int)((long long)(k1 - k0) * cluster / n_clusters) : k0;
    };

    int issued = 0;                    // a producer warp's ring stages so far, of either warp
    if (producer) {
        // ------------------------------------------------------------------ TMA producers
        // The whole warp runs the loop and one elected lane issues: with uniform control flow the copies' operands are formed
        // in uniform registers.  Everything the loop needs is read from the parameters ahead of it.
        {
            int s = 0;
            uint32_t wrap = 0, dst = base, bar_f = bar_full, bar_e = bar_empty;
            bool ok = true;
            const int kbs = p.kbs;
            const uint32_t stage_bytes = p.stage_bytes, blk_bytes = p.blk_bytes, a_bytes = p.a_bytes, b_bytes = p.b_bytes;
            const uint32_t tx = p.tx_bytes * (PAIR ? 2u : 1u);
            const int n_items = p.n_items, NT = p.NT, half = NT >> 1, rep = p.rep;
            const bool dual = p.dual != 0, two_b = !PAIR && !B_MN && dual;
            const uint32_t a_box = 16384u / (uint32_t)rep;
            // rows of B that one row tile alone reads are the first to leave L2 again: what is read twice stays
            const bool b_once = !PAIR && !B_MN && p.prob[0].tiles_m == 1;
            const uint64_t once = l2_policy_evict_first();
            const uint32_t bar_shift = PAIR ? cluster_map_shared(base, 0u) - base : 0u;    // both CTAs' bytes count on the leader's barrier
            int early = p.b_early ? 0 : -1;       // stages whose B is on its way before the dependency wait; -1: none to be
            for (int item = cluster; item < n_items && ok; item += n_clusters) {
                const GemmItem it = gemm_item(tab, n_prob, tiles_per_item, item);
                const GemmProblem& q = tab.prob[it.prob];
                const int row0 = it.mt * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0);
                const CUtensorMap *ma0 = &maps.map[q.a0], *ma1 = &maps.map[q.a1], *mb0 = &maps.map[q.b0], *mb1 = &maps.map[q.b1];
                if (PAIR && dual && rank) mb0 = mb1;            // the halves of a pair's tile come from one matrix each
                const int nk0 = q.nk0;
                int k0, k1;
                k_range(q, k0, k1);
                const int kb_first = k_start(q, k0, k1);
                for (int t = 0; t < it.n_tiles && ok; ++t) {
                    const int nt = it.nt0 + t;
                    const int col0 = dual ? nt * half : nt * NT + (PAIR ? (int)rank * half : 0);   // first row of B this CTA fetches
                    // one stage: nb k-blocks from kj on (wrapping at k1), to ring address `to`
                    auto issue = [&](int kj, int nb, uint32_t to, uint32_t bar_local, bool with_a, bool with_b) {
                        if (leader && with_b) mbar_arrive_expect_tx(bar_local, tx * (uint32_t)nb);
                        const uint32_t bar = bar_local + bar_shift;
                        auto load = [&](uint32_t at, const CUtensorMap* m, int cx, int cy) {
                            if constexpr (PAIR) tma_load_2d_pair(at, m, cx, cy, bar);
                            else tma_load_2d(at, m, cx, cy, bar);
                        };
                        for (int j = 0; j < nb; ++j, to += blk_bytes) {
                            const bool second = kj >= nk0;
                            const int x = (second ? kj - nk0 : kj) * kBoxK;
                            const CUtensorMap *ma = second ? ma1 : ma0, *mb = second ? mb1 : mb0;
                            const uint32_t dstb = to + a_bytes;
                            if (with_b) {
                                if constexpr (B_MN) {
                                    for (uint32_t o = 0; o < b_bytes; o += 8192u) load(dstb + o, mb, col0 + (int)(o >> 7), x);
                                } else if (b_once) {
                                    tma_load_2d_hint(dstb, mb, x, col0, bar, once);
                                    if (two_b) tma_load_2d_hint(dstb + (uint32_t)half * 128u, mb1, x, col0, bar, once);
                                } else {
                                    load(dstb, mb, x, col0);
                                    if (two_b) load(dstb + (uint32_t)half * 128u, mb1, x, col0);
                                }
                            }
                            if (with_a) {
                                if constexpr (A_MN) {
                                    load(to, ma, row0, x);
                                    load(to + 8192u, ma, row0 + 64, x);
                                } else {
                                    for (int r = 0; r < rep; ++r) load(to + (uint32_t)r * a_box, ma, x, row0);
                                }
                            }
                            if (++kj == k1) kj = k0;
                        }
                    };
                    if (early == 0) {                           // the ring's first filling, as far as this tile goes
                        int kj = kb_first;
                        early = min(S, (k1 - k0 + kbs - 1) / kbs);
                        for (int i = 0; i < early; ++i) {
                            const int nb = min(kbs, k1 - k0 - i * kbs);
                            if ((i & (kGemmProducers - 1)) == warp - kProducer && elect_one())
                                issue(kj, nb, base + (uint32_t)i * stage_bytes, bar_full + 8u * i, false, true);
                            __syncwarp();
                            kj += nb;
                            if (kj >= k1) kj -= k1 - k0;
                        }
                        grid_dependency_wait();
                    }
                    int kb = kb_first;
                    for (int i = k0; i < k1; i += kbs) {
                        const int nb = min(kbs, k1 - i);
                        const bool mine = (issued & (kGemmProducers - 1)) == warp - kProducer;
                        if (mine && wrap > 0 && !mbar_wait_warp(bar_e, (wrap - 1) & 1u, p.wait_ns)) { fail(); ok = false; break; }
                        if (mine && elect_one()) issue(kb, nb, dst, bar_f, true, issued >= early);
                        __syncwarp();
                        ++issued;
                        kb += nb;
                        if (kb >= k1) kb -= k1 - k0;
                        dst += stage_bytes;
                        bar_f += 8u;
                        bar_e += 8u;
                        if (++s == S) {
                            s = 0;
                            ++wrap;
                            dst = base;
                            bar_f = bar_full;
                            bar_e = bar_empty;
                            if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) { ok = false; break; }
                        }
                    }
                }
            }
        }
    } else if (warp == kIssuer) {
        // ------------------------------------------------------------------ MMA issuer (of a pair: the leader's)
        if (leader) {
            int s = 0, n = 0;                  // ring stage; tiles so far
            uint32_t phase = 0;
            bool ok = true;
            const uint64_t a_desc0 = A_MN ? smem_desc_sw128_mn(base) : smem_desc_sw128(base);
            const uint64_t b_desc0 = B_MN ? smem_desc_sw128_mn(base + p.a_bytes) : smem_desc_sw128(base + p.a_bytes);
            constexpr uint32_t a_step = A_MN ? 128u : 2u, b_step = B_MN ? 128u : 2u;   // 16 of k: two 8-row groups, or 32 bytes of a row
            const int kbs = p.kbs;
            const uint32_t stage_units = p.stage_bytes >> 4, blk_units = p.blk_bytes >> 4, idesc = p.idesc, acc_cols = p.acc_cols;
            const int n_items = p.n_items;
            uint64_t a = a_desc0, b = b_desc0;
            uint32_t bar_f = bar_full, bar_e = bar_empty;
            for (int item = cluster; item < n_items && ok; item += n_clusters) {
                const GemmItem it = gemm_item(tab, n_prob, tiles_per_item, item);
                int k0, k1;
                k_range(tab.prob[it.prob], k0, k1);
                for (int t = 0; t < it.n_tiles && ok; ++t, ++n) {
                    const int buf = n & 1;
                    if (n >= 2 && !mbar_wait_warp(bar_acce + 8u * buf, (uint32_t)((n >> 1) - 1) & 1u, p.wait_ns)) { fail(); ok = false; break; }
                    if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d_tmem = tmem_base + (uint32_t)buf * acc_cols;
                    uint32_t accumulate = 0u;
                    for (int kb = k0; kb < k1; kb += kbs) {
                        if (!mbar_wait_warp(bar_f, phase, p.wait_ns)) { fail(); ok = false; break; }
                        tc_fence_after();
                        const int nb = min(kbs, k1 - kb);
                        if (elect_one()) {
                            uint64_t aj = a, bj = b;
                            for (int j = 0; j < nb; ++j, aj += blk_units, bj += blk_units) {
#pragma unroll
                                for (uint32_t i = 0; i < 4; ++i) {
                                    const uint32_t acc = i == 0 && j == 0 ? accumulate : 1u;
                                    if constexpr (PAIR) tc_mma_bf16_pair(d_tmem, aj + i * a_step, bj + i * b_step, idesc, acc);
                                    else tc_mma_bf16(d_tmem, aj + i * a_step, bj + i * b_step, idesc, acc);
                                }
                            }
                            if constexpr (PAIR) tc_commit_pair_both(bar_e);
                            else tc_commit(bar_e);
                        }
                        __syncwarp();
                        accumulate = 1u;
                        a += stage_units;
                        b += stage_units;
                        bar_f += 8u;
                        bar_e += 8u;
                        if (++s == S) {
                            s = 0;
                            phase ^= 1u;
                            a = a_desc0;
                            b = b_desc0;
                            bar_f = bar_full;
                            bar_e = bar_empty;
                        }
                    }
                    if (ok && elect_one()) {
                        if constexpr (PAIR) tc_commit_pair_both(bar_accf + 8u * buf);
                        else tc_commit(bar_accf + 8u * buf);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        const int quad = warp & 3;                                 // the TMEM lanes this warp can read
        const int tile_rows = 128 / p.rep;                         // distinct rows of this CTA's tile
        const int r = (quad * 32 + lane) & (tile_rows - 1);        // the thread's row
        const int part = (warp >> 2) * p.rep + (quad * 32) / tile_rows, parts = 2 * p.rep;
        const int cols = Epi::kDual ? p.NT >> 1 : p.NT;            // columns of D in a tile
        const int nch = (cols + 15) >> 4, ng = (cols + 31) >> 5;
        const int ch0 = part * nch / parts, ch1 = (part + 1) * nch / parts;   // runs of 16 columns this thread takes,
        const int g0 = part * ng / parts, g1 = (part + 1) * ng / parts;       // or of 32 where they are stored in bulk
        constexpr int kStageUnits = gemm_stage_units(Epi::kOuts);
        constexpr uint32_t kStageBytes = kStageUnits * 32 * 64;
        const uint32_t stage_at = base + p.scratch_off + (uint32_t)warp * (Epi::kScratch / kGemmEpiWarps);
        int n = 0;
        for (int item = cluster; item < p.n_items; item += n_clusters) {
            const GemmItem it = gemm_item(tab, n_prob, tiles_per_item, item);
            const GemmProblem& q = tab.prob[it.prob];
            const int m = it.mt * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0) + r;
            typename Epi::State st;
            if constexpr (Epi::kStateful) Epi::begin(st, ep, m);
            for (int t = 0; t < it.n_tiles; ++t, ++n) {
                const int buf = n & 1;
                const int col0 = (it.nt0 + t) * cols;
                if constexpr (!Epi::kStateful) {
                    if (p.splits == 1 && m < q.M) {
                        Epi::row(st, ep, q, m);
                        Epi::ahead(st, ep, q, m, col0 + g0 * 32, 0);
                        Epi::ahead(st, ep, q, m, col0 + g0 * 32 + 16, 1);
                    }
                }
                bool got = false;
                if (!__any_sync(0xFFFFFFFFu, *abort_flag != 0)) {  // warp-uniform: tcgen05.ld needs the whole warp
                    got = __all_sync(0xFFFFFFFFu, mbar_wait(bar_accf + 8u * buf, (uint32_t)(n >> 1) & 1u, p.wait_ns));
                    if (!got) fail();
                }
                if (!got) continue;
                tc_fence_after();
                if (p.splits > 1) break;                           // the tile is finished below, with the rest of the cluster
                const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)buf * p.acc_cols;
                // The accumulator has been read: the MMAs of the tile after next may start.  Relaxed, as nothing in memory is
                // handed over: a release would wait for this warp's stores of results, 1600 cycles a tile.
                bool released = false;
                auto release = [&]() {
                    released = true;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (PAIR) mbar_arrive_cluster_relaxed(cluster_map_shared(bar_acce + 8u * buf, 0u));
                        else mbar_arrive(bar_acce + 8u * buf);
                    }
                };
                if constexpr (Epi::kStateful) {
                    Epi::tile(st, ep, m, AccColumns{taddr, ch0, ch1, col0, q.N}, smem + p.scratch_off);
                } else if (m - lane < q.M) {                       // some row of this warp exists
                    // 32 columns at a time to the warp's staging rows (kStageUnits times 32 columns), and from there to memory whenever
                    // they are full, several lanes to a row
                    const int rows_here = min(32, q.M - (m - lane));
                    for (int g = g0; g < g1; ++g) {
                        const int unit = (g - g0) % kStageUnits;
                        uint32_t u[32], w[Epi::kDual ? 32 : 1];
                        __syncwarp();                              // tcgen05.ld is the whole warp's; rows part in what they ask for and store
                        acc_ld16(taddr + (uint32_t)(g * 32), reinterpret_cast<uint32_t(&)[16]>(u[0]));
                        if (g * 32 + 16 < cols) acc_ld16(taddr + (uint32_t)(g * 32 + 16), reinterpret_cast<uint32_t(&)[16]>(u[16]));
                        if constexpr (Epi::kDual) {
                            acc_ld16(taddr + (uint32_t)(cols + g * 32), reinterpret_cast<uint32_t(&)[16]>(w[0]));
                            if (g * 32 + 16 < cols) acc_ld16(taddr + (uint32_t)(cols + g * 32 + 16), reinterpret_cast<uint32_t(&)[16]>(w[16]));
                        }
                        tc_wait_ld();
                        if (g + 1 == g1) release();
                        if constexpr (Epi::kSums) {
                            if (m < q.M && Epi::wants(st)) {
                                float* to = Epi::sums(st, ep, q) + col0 + g * 32;
#pragma unroll
                                for (int e = 0; e < 32; e += 4)
                                    if (g * 32 + e < cols && col0 + g * 32 + e < q.N)
                                        *reinterpret_cast<uint4*>(to + e) = make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            const int c = g * 32 + e;
                            if (c >= cols) break;                  // the other half, or the next tile's
                            float x[8], y[8], out[Epi::kOuts][8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                x[i] = __uint_as_float(u[e + i]);
                                y[i] = Epi::kDual ? __uint_as_float(w[Epi::kDual ? e + i : 0]) : 0.0f;
                            }
                            Epi::cols8(st, ep, q, m, col0 + c, e, x, y, out);
#pragma unroll
                            for (int o = 0; o < Epi::kOuts; ++o)
                                st_shared_bf16x8(stage_at + (uint32_t)o * kStageBytes + stage_offset<kStageUnits>(lane, unit * 4 + e / 8), out[o]);
                            if ((e & 8) && m < q.M) Epi::ahead(st, ep, q, m, col0 + c + 24, e >> 4);      // the next group's run of this slot
                        }
                        if (unit + 1 < kStageUnits && g + 1 < g1) continue;
                        __syncwarp();
                        const int shift = unit + 2;                // 4 or 8 chunks of 16 bytes are staged per row
                        const int j = lane & ((1 << shift) - 1), r0 = lane >> shift, c = (g - unit) * 32 + j * 8;
                        if (c < cols && col0 + c < q.N) {
#pragma unroll
                            for (int o = 0; o < Epi::kOuts; ++o) {
                                uint16_t* to = Epi::at(ep, q, it.prob, o, m - lane, col0 + c);
                                const int64_t ld = Epi::ld(ep, q, o);
                                uint4 v[4];
                                for (int half = 0; half <= unit; ++half) {       // all rows: four turns, or twice that
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        v[i] = ld_shared_v4(stage_at + (uint32_t)o * kStageBytes +
                                                            stage_offset<kStageUnits>(r0 + ((half * 4 + i) << (5 - shift)), j));
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const int r = r0 + ((half * 4 + i) << (5 - shift));
                                        if (r < rows_here) *reinterpret_cast<uint4*>(to + r * ld) = v[i];
                                    }
                                }
                            }
                        }
                        __syncwarp();
                    }
                }
                if (!released) release();
            }
            if constexpr (Epi::kStateful) Epi::end(st, ep, m, it.nt0 / p.tiles_per_item * parts + part);
        }
    }

    if constexpr (!PAIR && !Epi::kStateful) {
        if (p.splits > 1) {
            const GemmItem it = gemm_item(tab, n_prob, tiles_per_item, cluster);
            const GemmProblem& q = tab.prob[it.prob];
            const int cols = Epi::kDual ? p.NT >> 1 : p.NT, groups = cols >> 3;
            const int rows = min(128, q.M - it.mt * 128);
            cluster_sync_all();                                    // every ring is idle: the sums go where it was
            const int r = (warp & 3) * 32 + lane;
            if (warp < kGemmEpiWarps && (warp & 3) * 32 < rows && __all_sync(0xFFFFFFFFu, *abort_flag == 0)) {
                // partial sums to the owners of their columns, eight columns at a time
                const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
                const int nch = (cols + 15) >> 4, half = warp >> 2;
                for (int ch = half * nch / 2; ch < (half + 1) * nch / 2; ++ch) {
                    uint32_t u[16], w[16];
                    __syncwarp();                                  // lanes past the rows have not stored what the others have
                    acc_ld16(taddr + (uint32_t)(ch * 16), u);
                    if constexpr (Epi::kDual) acc_ld16(taddr + (uint32_t)(cols + ch * 16), w);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        const int g = ch * 2 + (e >> 3);
                        if (g >= groups || r >= rows) break;
                        int owner = (int)((unsigned)(g * p.splits) / (unsigned)groups);
                        if (g >= (owner + 1) * groups / p.splits) ++owner;     // shares are [owner * groups / splits, ...); splits <= groups
                        const int local = g - owner * groups / p.splits;
                        // four columns of all rows in a run: a warp's 16-byte stores lie side by side
                        const uint32_t run = p.x_rows * 16u;
                        const uint32_t to = cluster_map_shared(base + rank * p.x_part, (uint32_t)owner) +
                                            (uint32_t)local * (Epi::kDual ? 4u : 2u) * run + (uint32_t)r * 16u;
                        st_cluster_v4(to, u[e], u[e + 1], u[e + 2], u[e + 3]);
                        st_cluster_v4(to + run, u[e + 4], u[e + 5], u[e + 6], u[e + 7]);
                        if constexpr (Epi::kDual) {
                            st_cluster_v4(to + 2u * run, w[e], w[e + 1], w[e + 2], w[e + 3]);
                            st_cluster_v4(to + 3u * run, w[e + 4], w[e + 5], w[e + 6], w[e + 7]);
                        }
                    }
                }
            }
            cluster_sync_all();                                    // every partial sum is where it belongs
            if (warp < kGemmEpiWarps && !*abort_flag) {
                const int g0 = (int)rank * groups / p.splits, g1 = ((int)rank + 1) * groups / p.splits;   // this CTA's runs of 8 columns
                for (int e = tid; e < rows * (g1 - g0); e += kGemmEpiWarps * 32) {
                    const int g = e / rows, er = e - g * rows;
                    const int col = it.nt0 * cols + (g0 + g) * 8, m = it.mt * 128 + er;
                    if (col >= q.N) continue;
                    typename Epi::State st;
                    Epi::row(st, ep, q, m);
                    Epi::ahead(st, ep, q, m, col, 0);
                    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, y[8] = {0, 0, 0, 0, 0, 0, 0, 0}, out[Epi::kOuts][8];
                    const unsigned char* from = smem + ((size_t)g * (Epi::kDual ? 4 : 2) * p.x_rows + er) * 16;
                    for (int s = 0; s < p.splits; ++s, from += p.x_part) {
                        const float4* f = reinterpret_cast<const float4*>(from);
                        const float4 v0 = f[0], v1 = f[p.x_rows];
                        x[0] += v0.x; x[1] += v0.y; x[2] += v0.z; x[3] += v0.w;
                        x[4] += v1.x; x[5] += v1.y; x[6] += v1.z; x[7] += v1.w;
                        if constexpr (Epi::kDual) {
                            const float4 w0 = f[2 * p.x_rows], w1 = f[3 * p.x_rows];
                            y[0] += w0.x; y[1] += w0.y; y[2] += w0.z; y[3] += w0.w;
                            y[4] += w1.x; y[5] += w1.y; y[6] += w1.z; y[7] += w1.w;
                        }
                    }
                    if constexpr (Epi::kSums) {
                        if (Epi::wants(st)) {
                            float4* to = reinterpret_cast<float4*>(Epi::sums(st, ep, q) + col);
                            to[0] = make_float4(x[0], x[1], x[2], x[3]);
                            to[1] = make_float4(x[4], x[5], x[6], x[7]);
                        }
                    }
                    Epi::cols8(st, ep, q, m, col, 0, x, y, out);
#pragma unroll
                    for (int o = 0; o < Epi::kOuts; ++o) store_bf16x8(Epi::at(ep, q, it.prob, o, m, col), out[o]);
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();                             // every role is done, and knows whether one of them gave up
    if (__builtin_expect(*abort_flag != 0, 0)) { // MMAs and copies in flight must end before their memory is given back
        if (warp == kIssuer && leader && elect_one()) {
            if constexpr (PAIR) tc_commit_pair(bar_drain);
            else tc_commit(bar_drain);
            (void)mbar_wait(bar_drain, 0u, p.wait_ns);
        }
        if (producer && lane == 0) {
            const unsigned long long now = global_timer_ns();
            if (leader) {                        // of a pair: for both, which leave together
                for (int i = max(0, issued - S); i < issued; ++i)
                    if ((i & (kGemmProducers - 1)) == warp - kProducer)
                        (void)mbar_wait_until(bar_full + 8u * (i % S), (uint32_t)(i / S) & 1u, now + p.wait_ns);
            } else {                             // copies past the leader's last stage are counted nowhere: longer than any takes
                while (global_timer_ns() - now < 1000000ull) { }
            }
        }
        __syncwarp();
        tc_fence_before();
        __syncthreads();
    }
    if constexpr (PAIR) cluster_sync_all();      // neither CTA leaves while the other's MMAs or arrivals may still reach it
    tc_fence_after();
    if (warp == kIssuer) {
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
    }
}

// See vt_test_withhold_copies: 0, or the limit of the calling thread's products' waits in microseconds.
int gemm_withheld_us();
// Notes a launch for vt_test_products.
void gemm_note(bool pair, int NT, int splits, int items, int at_once);

// Launches the kernel for a finished plan (`pair` as the plan chose).
template <bool A_MN, bool B_MN, class Epi>
inline vt_status gemm_launch(const GemmMaps& maps, const GemmParams& plan, bool pair, const typename Epi::Params& ep, cudaStream_t st) {
    GemmParams withheld;
    const GemmParams& p = gemm_withheld_us() > 0 ? withheld : plan;
    static std::atomic<unsigned long long> configured_pair{0}, configured_single{0};
    auto* kernel = pair ? gemm_kernel<true, A_MN, B_MN, Epi> : gemm_kernel<false, A_MN, B_MN, Epi>;
    if (vt_status rc = ensure_max_dyn_smem(reinterpret_cast<const void*>(kernel), kMaxDynSmem, pair ? &configured_pair : &configured_single);
        rc != VT_OK)
        return rc;
    int sms = 0;
    if (vt_status rc = device_sm_count(&sms); rc != VT_OK) return rc;
    if (const int us = gemm_withheld_us(); us > 0) {     // a test of the unwinding: each stage waits for 16 bytes more than come
        withheld = plan;
        withheld.tx_bytes += 16;
        withheld.wait_ns = (unsigned long long)us * 1000ull;
    }
    const int cluster = pair ? 2 : p.splits;
    const int grid = pair ? 2 * std::max(1, std::min(sms / 2, p.n_items)) : p.splits > 1 ? p.n_items * p.splits : std::min(sms, p.n_items);
    cudaError_t e = cluster > 1 ? launch_pdl_cluster(kernel, cluster, grid, kGemmThreads, p.total_smem, st, maps, p, ep)
                                : launch_pdl(kernel, grid, kGemmThreads, p.total_smem, st, maps, p, ep);
    count_launch();
    gemm_note(pair, p.NT, p.splits, p.n_items, grid / cluster);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

#endif  // __CUDACC__

// ------------------------------------------------------------------------------------------ host
inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
inline size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }

// Chooses tile shape, CTA pairs and k-splits for the products in p->prob (M, N, nk0, nk1 set) and fills in the rest of p
// except the maps' indices, outputs and hdr.  False when the work is too large to number its tiles.
// scratch_bytes: the epilogue's kScratch.
bool gemm_plan(GemmParams* p, bool a_mn, bool b_mn, bool dual, uint32_t scratch_bytes, bool* pair);
// The same for token scoring: one product, both operands K-major, whole k range in every CTA.  long_runs: the first tile of a run
// costs the epilogue far more than the others.
bool gemm_plan_rows(GemmParams* p, uint32_t scratch_bytes, bool long_runs, bool* pair);
// Rows of the box each operand's tensor map has (64 columns wide; MN-major operands: 64).
inline int gemm_box_a(const GemmParams& p, bool a_mn) { return a_mn ? 64 : (int)p.a_rows; }
int gemm_box_b(const GemmParams& p, bool b_mn, bool pair);

// One or more products whose sums are rounded once to bf16 and stored in out[i] (row-major, N columns a row), operands of the
// given majors.
vt_status gemm_store(const GemmMaps& maps, const GemmParams& p, bool pair, bool a_mn, bool b_mn, void* const* out, cudaStream_t st);

// A bf16 matrix operand in global memory: rows x cols, rows ld elements apart.
struct GemmOperand {
    const void* ptr;
    int rows, cols;
    int64_t ld;
};
// make_tensor_map_bf16 for rows that lie ld elements apart (ld a multiple of 8; defined beside it).
vt_status make_tensor_map_bf16_ld(CUtensorMap* map, const void* ptr, int rows, int d, int64_t ld, int box_rows);
inline vt_status gemm_map(CUtensorMap* map, const GemmOperand& o, int box_rows) {
    return make_tensor_map_bf16_ld(map, o.ptr, o.rows, o.cols, o.ld, box_rows);
}

}  // namespace vt
