// Attention of drafted tokens over a paged cache (see vt_tree_attention).
//
// out = sum_i e^{x_i - lse} v_i over the attended positions, x = scale q.k: one pass over keys and values, with the running maximum and sum
// of each row, as two tcgen05 products per tile of 128 positions - S = Q K^T, then O += P V with P = 2^{(S - m) scale log2 e} in bf16, the
// operand type of the product.  Scores, maxima, sums and O are fp32.  lse comes from the sum l of the weights before they are rounded.  With few rows O
// is divided by the sum of the rounded ones: a weight far above the others then loses nothing (error of whole outputs over 4096 ragged positions 2.09e-3 ->
// 1.88e-3, 1.65e-3 of it the rounding of out; 24 x 8 over 2500 +0.6 us).  With many, where a stream's exponentials are what it waits for, O is divided by l:
// the second sum took 110 -> 113.6 us for two long documents under 60 tokens, and 58 -> 62.5 for 16 x 60 over 8000 with heads of 64.
//
// Rows.  All query heads of a key head and all drafted tokens of a request read the same keys, so they are the rows of one product: row
// t G + g for token t and head g of G.  A block of rows is up to two tiles of 128 TMEM lanes (a TMA box of G heads x 128 / G tokens fills a tile
// in that order).
//
// Two streams.  S, P and O of two streams live in tensor memory: O0, O1, S0, S1, 128 columns each; P takes the place of its S.  While
// four warps work out one stream's exponentials, the tensor cores multiply for the other.  With two row tiles a stream is a row tile
// and both read each key tile; with one, the streams take the key tiles in turn, and are joined when the rows are finished.
//
// Few rows (REP, 32 at most).  A tile of 128 lanes is a quarter full at best, and one warp of four would have all the exponentials.  So q stands in
// all four groups of 32 lanes, each warp takes 32 of a tile's 128 positions (its weights of the others are 0), and the eight parts of O, by stream
// and warp, are added up at the item's end.  The products cost the same, the exponentials a quarter (64 x 1 over 4096: 113 -> 100 us).
//
// Work.  The lengths are known on the device alone, so the cut is made there: all key tiles of all (request, key head, row block) in a row,
// a run of equal weight to each CTA.  A run begins and ends inside an item, and a long item lies in many runs: a CTA writes what it has
// of such an item (unnormalised O, m, l in fp32) to the workspace, and a second kernel joins the pieces.  No atomics: the same bits every time.
// Where the host can see that no item is longer than kAttnWhole tiles, items are not cut and there is one launch.
//
// O is rescaled only when a row's maximum grows by more than 2^8 over the one in use (P then stays below 2^8, its sum in fp32): the
// rescale, done by the stream's own warps, is rare after the first tiles.
//
// Roles: warps 0-3 and 4-7 softmax of stream 0 and 1 (and the end of an item), warp 8 the planner and TMA producer of q and K, warp 11 that of V,
// warp 9 MMA issuer (of stream 0 alone with few rows, stream 1 then has warp 12), warp 10 the cleaner: in tiles where something is masked it turns
// infinities and NaN of V into the largest finite number, so that a weight of 0 keeps them out.
// All waits are bounded; one that runs out sets the status word and every role leaves.
//
// Turns of the ring.  K and V tiles take places in one order (AttnPiece::k_at), place P stage P mod ST, turn P / ST, and the cleaner passes
// every place in that order.  A wait names a turn by its parity and also passes when the turn before is not over, so whoever waits has to
// know that it is; ST is 5 at least, and "passed" is said of the cleaner:
//   a producer   that loaded P - ST itself has seen P - 2 ST empty.  Otherwise it waits for v_clean(P - ST) before kv_empty(P - ST): that place is
//                passed only when it was loaded, after the other producer saw P - 2 ST empty.  And P - 2 ST has been passed by then, as its own last place,
//                3 before P at most, came behind the emptying of the place ST before that.
//   one issuer   takes all value places, 3 apart at most, and all key places behind the values before them: P - ST has been passed.
//   two issuers  A stream's K(j) follows its V(j - 2), one place before it; later values of a stream are 3 or 4 behind its last.  K(0) and K(1), places 0
//                and 1 of an item, follow its last values, 2 places before the item at most, or, where the last item (of one tile) had none for it,
//                the O of the item before.  V(0) lies at 1 or 2, V(1) at 3 or 4: with 7 stages or more the same holds.  With fewer (heads of 128) an
//                item's first weights are waited for before its values: they come behind the last item's O, so all of that one's places have been
//                passed.  (With heads of 64 too: 24 x 8 over 2500 57.4 -> 58.3 us.)
// (With the values first, or without a look at v_clean in the producers, copies of a slow stream's tiles were overtaken: no error, wrong values.)
//
// Bound and measured (in a graph, a copy at 6.46 TB/s and 1673 TFLOP/s in bf16 as the floors; requests x tokens over positions, 32 heads over 8
// of 128 where nothing else stands):
//   2 x 8 over 100000             134 us   floor 127: bytes of the cache, 6.1 TB/s
//   64 x 1 over 4096, ragged       98 us   floor 86: bytes, 5.7 TB/s
//   24 x 8 over 2500, 32 heads of 64 each, ragged   58 us   floor 40: bytes, 768 items of 20 tiles at most, each with a beginning and an end
//   16 x 60 over 8000, ragged      72 to 78 us   floor 54: a stream's exponentials and its products follow one another: 4140 cycles for a pair of steps
//                                          whose products, and whose exponentials, would each take 2048
//   1 x 60 over 4000             21.6 us   floor 3: latency; 88 runs of two or three tiles and the join
//   1 x 1 over 700                11.4 us  floor 0.5: latency of launch, plan, copy, two products, epilogue, join
//   1 x 4099 over 0, a chain       171 us  floor 82: products, of 65 blocks with half a tile each that the chain cuts off; what else is not taken apart
//   1 x 4099 over 120000           8.4 ms  floor 4.9: products and exponentials in turn, as with 16 x 60
#include "vt_step.h"
#include "vt_tc.cuh"

#include <cfloat>

namespace vt {

int gemm_withheld_us();                      // see vt_test_withhold_copies

constexpr int kAttnKeys = 128;               // positions per tile
constexpr int kAttnProducer = 8, kAttnIssuer = 9, kAttnCleaner = 10, kAttnProducerV = 11, kAttnIssuer1 = 12;      // (the last with few rows alone)
constexpr int attn_threads(bool few) { return (few ? 13 : 12) * 32; }
constexpr int kAttnPieces = 4;               // pieces the planner may be ahead
constexpr int kAttnCtas = 148;               // runs at most
constexpr int kAttnWhole = 4;                // tiles of an item that is not worth cutting (16 x 60 over 440: 20 us, cut 24.5; 1 x 60 over 900: cut 18, 25 with 8 tiles)
constexpr int kAttnMaxStages = 12;
constexpr int kAttnItemCost = 4;             // what an item's beginning and end cost, in its tiles (24 x 8 over 2500: 57 us; with 2 tiles 71, 3 60, 6 58)
constexpr float kAttnSlack = 8.0f;           // how far (in powers of two) a maximum may grow before O is rescaled
constexpr uint32_t kAttnTmemO = 0, kAttnTmemS = 256;

struct AttnSplit {                           // an item that several CTAs have pieces of
    int rows;                                // 0: none
    int token0, head0, n_pieces, first_cta;
    int first_slot;                          // of the first piece: 0 where its CTA's run begins with the item
    int pad[2];
};
static_assert(sizeof(AttnSplit) == 32, "one sector");

struct AttnParams {
    const int32_t *cu, *lens, *page_table, *mask;
    int64_t table_stride;
    uint16_t* out;
    int64_t out_ts, out_hs;
    float* lse;
    WsHeader* hdr;
    AttnSplit* splits;                       // [n_splits]
    float2* part_ml;                         // [gridDim.x][2][rows]: (m, l) of a piece's rows
    float* part_o;                           // [gridDim.x][2][D / 4][rows][4]
    int rows_max;                            // rows of a block at most
    int N, B, Hq, Hkv, G, max_tokens, mask_words, n_pages, page_size, max_pages;
    int tpt;                                 // tokens per row tile
    int box_tokens;                          // tokens in a box of q
    int whole;                               // 1: items are not cut
    int blocks;                              // row blocks of a request at most
    int entries, n_splits;                   // entries of the join: one for every item there may be, where rows are many and those no more than CTAs (else 0); all in all
    int min_run;                             // the least weight of a CTA's run, 2 at least
    int n_stages;
    uint32_t stages_inv;                     // 2^32 / n_stages, rounded up
    uint32_t q_block, q_slot;                // bytes of 64 columns of a row tile; of a row tile
    uint32_t q_tx, page_tx;                  // bytes of a q tile; of one box of keys
    uint32_t shared_off, bar_off, withheld;              // withheld: see vt_test_withhold_copies
    float scale, scale_log2, scale_inv;      // scale_inv: 1 / scale_log2, 0 where that is no number
    unsigned long long wait_ns;
};

#ifdef __CUDACC__

__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tc_ld64(uint32_t taddr, uint32_t (&r)[64]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// Descriptor of V as an operand whose columns (of the head) run fastest: 64 columns are one 128-byte swizzled row, 8 positions are 1024
// bytes apart, the next 64 columns a block of 128 positions further on.
__device__ __forceinline__ uint64_t attn_v_desc(uint32_t addr) {
    uint64_t desc = 0;
    desc |= (uint64_t)((addr & 0x3FFFFu) >> 4);
    desc |= (uint64_t)((kAttnKeys * 128) >> 4) << 16;
    desc |= (uint64_t)(1024 >> 4) << 32;
    desc |= (uint64_t)1 << 46;
    desc |= (uint64_t)2 << 61;
    return desc;
}
__device__ __forceinline__ bool attn_elect() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// fence_proxy_async for shared memory alone: it does not wait for stores of results.
__device__ __forceinline__ void fence_proxy_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// adds two packed bf16 to two sums
__device__ __forceinline__ void attn_add_bf16x2(float& lo, float& hi, uint32_t v) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}" : "+f"(lo), "+f"(hi) : "r"(v));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t attn_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// mbar_wait in few instructions.  The kernel's roles each run their code a handful of times in a short call, so its size is latency: the
// first version, 167 KB with everything unrolled, spent more cycles on fetching instructions than on a short item.
__device__ __forceinline__ bool attn_wait(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
    unsigned long long t0 = 0;
    uint32_t spins = 0;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 0xFFu) == 0) {
            const unsigned long long now = global_timer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > limit_ns) return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool attn_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return __all_sync(0xFFFFFFFFu, ok != 0);
}
// n / d for n < 2^31 d.
__device__ __noinline__ long long attn_div(long long n, long long d) {
    return (n | d) <= 0xFFFFFFFFll ? (long long)((uint32_t)n / (uint32_t)d) : n / d;
}

// ------------------------------------------------------------------------------------------ the cut
struct AttnRequest {
    int first, T, L;                         // first token, tokens, earlier positions
};
// Whatever the arrays hold, the tokens lie inside [0, N) and the positions inside the table.
__device__ __forceinline__ AttnRequest attn_request(const AttnParams& p, int b) {
    AttnRequest q;
    const long long cap = (long long)p.max_pages * p.page_size;
    q.first = min(max(p.cu[b], 0), p.N);
    q.T = min(min(max(p.cu[b + 1], q.first), p.N) - q.first, p.max_tokens);
    q.L = (int)min(min((long long)max(p.lens[b], 0), cap), 0x7FFF0000ll - q.T);
    return q;
}
// The positions that tokens [.., t_end) of a request may attend, and the tiles they take.
__device__ __forceinline__ int attn_keys(const AttnParams& p, const AttnRequest& q, int t_end) {
    const long long cap = (long long)p.max_pages * p.page_size;
    return (int)min((long long)q.L + (p.mask ? q.T : min(q.T, t_end)), cap);
}
__device__ __forceinline__ int attn_tiles(int keys) { return max(1, (keys + kAttnKeys - 1) / kAttnKeys); }
__device__ __forceinline__ int attn_blocks(const AttnParams& p, const AttnRequest& q) { return (q.T + 2 * p.tpt - 1) / (2 * p.tpt); }
// What a tile of a block of so many tokens weighs: with two row tiles twice as much is worked out for it (4 ragged trees of 40 over 30000: 87 us
// when all weigh the same, 70 so).
__device__ __forceinline__ int attn_tile_weight(const AttnParams& p, int tokens) { return tokens > p.tpt ? 2 : 1; }
// What a key head of a request weighs: its items' tiles, and kAttnItemCost more for each item.
__device__ __forceinline__ long long attn_head_weight(const AttnParams& p, const AttnRequest& q) {
    const int blocks = attn_blocks(p, q);
    long long n = 0;
    if (p.mask) {                            // all blocks but the last are full, and as long
        const int last = attn_tile_weight(p, q.T - (blocks - 1) * 2 * p.tpt);
        return blocks > 0 ? (2ll * (blocks - 1) + last) * (kAttnItemCost + attn_tiles(attn_keys(p, q, q.T))) : 0;
    }
#pragma unroll 1
    for (int i = 0; i < blocks; ++i)
        n += (long long)attn_tile_weight(p, q.T - i * 2 * p.tpt) * (kAttnItemCost + attn_tiles(attn_keys(p, q, (i + 1) * 2 * p.tpt)));
    return n;
}
// W units in C runs, the first `more` of them a unit longer than the others.
struct AttnCut {
    long long base, more;
    __device__ __forceinline__ AttnCut(long long W, int C) {
        base = attn_div(W, C);
        more = W - base * C;
    }
    __device__ __forceinline__ long long start(int c) const { return base * c + min((long long)c, more); }
    __device__ __forceinline__ int of(long long g) const {       // the run that unit g lies in
        const long long at = more * (base + 1);
        const long long n = g < at ? g : g - at, d = g < at ? base + 1 : base;
        return (int)((g < at ? 0 : more) + attn_div(n, d));
    }
};

// Block i of a key head of a request, and its places from `at` on.
struct AttnItem {
    int tok0, ntok, keys, tiles, heavy;      // heavy: log2 of a tile's weight
    long long begin, first, end;             // its place, its first tile's, the next item's
    __device__ __forceinline__ AttnItem(const AttnParams& p, const AttnRequest& q, int i, long long at) {
        tok0 = i * 2 * p.tpt;
        ntok = min(2 * p.tpt, q.T - tok0);
        keys = attn_keys(p, q, tok0 + ntok);
        tiles = attn_tiles(keys);
        heavy = attn_tile_weight(p, ntok) - 1;
        begin = at;
        first = at + (kAttnItemCost << heavy);
        end = first + ((long long)tiles << heavy);
    }
    // what the join has to know where several runs have tiles of the item
    __device__ __forceinline__ AttnSplit split(const AttnParams& p, const AttnRequest& q, int h, const AttnCut& cut) const {
        AttnSplit r{};
        const int c0 = cut.of(first);
        r.n_pieces = cut.of(end - 1 - heavy) - c0 + 1;       // (to the last tile's place)
        r.rows = r.n_pieces > 1 ? ntok * p.G : 0;
        r.token0 = q.first + tok0;
        r.head0 = h * p.G;
        r.first_cta = c0;
        r.first_slot = cut.start(c0) >= begin ? 0 : 1;
        return r;
    }
};

// What a CTA does of one item; the planner's message to the other roles.
struct __align__(16) AttnPiece {
    int n;                                   // key tiles; 0: nothing more
    int b, h, t0;                            // request, key head, first tile
    int keys, open;                          // positions of the item; tiles from `open` on hold some that some row may not attend
    int L, T, first;                         // of the request: earlier positions, tokens, first token
    int tok0, ntok;                          // the block's tokens
    int dual;                                // two row tiles
    int cut;                                 // others have pieces of the item, too
    int slot;                                // in the workspace: 0 for the item the CTA's run begins in, 1 for the one it ends in
    int pad[2];

    // half-steps: products of one stream with one tile
    __device__ __forceinline__ int steps() const { return n << dual; }
    // places of K(t0 + j) and V(t0 + j) in the order of loads: K0, K1, V0, K2, V1, ..., the last V
    __device__ __forceinline__ uint32_t k_at(int j) const { return j == 0 ? 0u : 2u * j - 1u; }
    __device__ __forceinline__ uint32_t v_at(int j) const { return j + 1 < n ? 2u * j + 2u : 2u * j + 1u; }
    // the j that place e holds V(t0 + j) of; -1 where it holds K((e + 1) / 2)
    __device__ __forceinline__ int value_at(uint32_t e) const { return e + 1u == 2u * n ? n - 1 : e & 1u ? -1 : (int)(e >> 1) - 1; }
};

// Bits of the 32 positions from lens + u0 on that a token attends (u0 may be negative: earlier positions).
__device__ __forceinline__ uint32_t attn_bits(const int32_t* row, int words, int t, int T, int u0) {
    if (u0 <= -32) return 0xFFFFFFFFu;
    const int up = u0 < 0 ? -u0 : 0;         // that many earlier positions come first
    const int u = u0 + up;                   // >= 0
    uint32_t bits;
    if (row) {
        const int w = u >> 5, s = u & 31;
        const uint32_t lo = w < words ? (uint32_t)row[w] : 0u, hi = w + 1 < words ? (uint32_t)row[w + 1] : 0u;
        bits = __funnelshift_r(lo, hi, s);
        const int n = T - u;
        bits &= n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
    } else {
        const int n = t + 1 - u;
        bits = n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
    }
    return up ? bits << up | ((1u << up) - 1u) : bits;
}

// Steps of 16 positions that hold any of the piece's j-th tile.
__device__ __forceinline__ int attn_k_steps(const AttnPiece& w, int j) {
    return min(kAttnKeys / 16, (w.keys - (w.t0 + j) * kAttnKeys + 15) >> 4);
}

struct AttnMaps {
    CUtensorMap q, k, v;
};
struct AttnShared {
    AttnPiece piece[kAttnPieces];
    float2 ms[2][128];                       // (m, l) of the streams' rows, where one item has both
    uint32_t tmem;
    int abort;
};

template <int D, bool REP>
__global__ void __launch_bounds__(attn_threads(REP), 1)
attn_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnParams p) {
    constexpr uint32_t kTile = kAttnKeys * D * 2;            // bytes of a K or V tile: D / 64 blocks of 128 positions x 128 bytes
    constexpr uint32_t kBlock = kAttnKeys * 128;
    // D fp32, A and B bf16; S: as many columns as positions (N / 8 from bit 17 on), both K-major; O: D columns, V with its columns fastest
    constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);

    // q's two slots, the ring, then what AttnShared and the barriers take.  No static part, so that the whole begins at a multiple of 1024.
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    AttnShared& sh = *reinterpret_cast<AttnShared*>(smem + p.shared_off);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ST = (uint32_t)p.n_stages;
    const uint32_t q_smem = base, ring = base + 2u * p.q_slot;
    const uint32_t kv_full = base + p.bar_off, kv_empty = kv_full + 8u * ST, v_clean = kv_empty + 8u * ST;
    const uint32_t q_full = v_clean + 8u * ST, q_empty = q_full + 16u, s_full = q_empty + 16u, p_full = s_full + 16u;
    const uint32_t o_full = p_full + 16u, meet = o_full + 8u, drain = meet + 8u;
    const uint32_t piece_full = drain + 16u, piece_empty = piece_full + 8u * kAttnPieces;
    volatile int* abort_flag = &sh.abort;

    if (tid == 0) {
        for (uint32_t s = 0; s < ST; ++s) {
            mbar_init(kv_full + 8u * s, 1);
            mbar_init(kv_empty + 8u * s, 3);                 // the products of either stream, and the cleaner
            mbar_init(v_clean + 8u * s, 1);
        }
        for (uint32_t s = 0; s < 2; ++s) {
            mbar_init(q_full + 8u * s, 1);
            mbar_init(q_empty + 8u * s, REP ? 3 : 1);        // the products that read it, and the end of the item, which works in it
            mbar_init(s_full + 8u * s, 1);
            mbar_init(p_full + 8u * s, 4);
        }
        for (uint32_t s = 0; s < kAttnPieces; ++s) {
            mbar_init(piece_full + 8u * s, 1);
            mbar_init(piece_empty + 8u * s, attn_threads(REP) / 32 - 1);
        }
        mbar_init(o_full, REP ? 2 : 1);
        mbar_init(meet, 8);
        mbar_init(drain, 1);
        mbar_init(drain + 8u, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kAttnProducer && lane < 3)
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &maps.q : lane == 1 ? &maps.k : &maps.v) : "memory");
    if (warp == kAttnIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    grid_dependency_wait();
    if (tid == 0) grid_launch_dependents();

    // A warp whose wait runs out reports it and leaves its loop; so do the others when their own waits run out.
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        if (__all_sync(0xFFFFFFFFu, attn_wait(bar, parity, p.wait_ns))) return true;
        *abort_flag = 1;
        atomicOr(&p.hdr->status, kStatusTimeout);
        return false;
    };
    // ring places by number: stage and parity of the turn
    auto turn_of = [&](uint32_t place) { return __umulhi(place, p.stages_inv); };
    uint32_t taken = 0;
    auto take = [&](AttnPiece& w) -> bool {
        const uint32_t s = taken % kAttnPieces;
        if (!wait(piece_full + 8u * s, taken / kAttnPieces & 1u)) return false;
        ++taken;
        w = sh.piece[s];
        __syncwarp();
        if (lane == 0) mbar_arrive(piece_empty + 8u * s);
        return w.n > 0;
    };

    // Copies of a piece's key tiles, or of its value tiles, from ring place `loads` on: a lane per box, column block lane / np, page lane % np of
    // the tile.  A box costs the warp 100 cycles, so either kind has a warp of its own.
    bool bad = false;
    uint32_t own = 0, last_place = 0;                        // bit d of own: place last_place - d is this warp's
    auto copy_tiles = [&](const AttnPiece& w, uint32_t loads, bool values) -> bool {
        const int pr = min(p.page_size, kAttnKeys), np = kAttnKeys / pr;
        const int col = lane / np, pg = lane - col * np;
        const bool mine = col < D / 64;
        const int tpp = p.page_size / kAttnKeys;             // tiles per page, 0 or 1 where a tile has whole pages
        const uint32_t box_at = ring + (uint32_t)col * kBlock + (uint32_t)(pg * pr) * 128u;
        const CUtensorMap* map = values ? &maps.v : &maps.k;
        const int32_t* row = p.page_table + w.b * p.table_stride;
        const int end = (w.keys - pg * pr + kAttnKeys - 1) / kAttnKeys - w.t0;      // the lane's boxes end with this j
        auto page_of = [&](int j) -> int {
            if (j >= w.n || !mine || j >= end) return -1;
            return row[tpp > 1 ? (unsigned)(w.t0 + j) / (unsigned)tpp : (unsigned)((w.t0 + j) * np + pg)];
        };
        const int last_tile = attn_tiles(w.keys) - 1 - w.t0;
        int page = page_of(0);
#pragma unroll 1
        for (int j = 0; j < w.n; ++j) {
            const int page_next = page_of(j + 1);            // one ahead of its use
            const uint32_t place = loads + (values ? w.v_at(j) : w.k_at(j)), turn = turn_of(place), stage = place - turn * ST;
            own <<= place - last_place;
            last_place = place;
            // the other producer's tile in the stage: has it come?  Then, is the stage empty?  (In the first turn there is nothing to wait for.)
            if ((!(own >> ST & 1u) && !wait(v_clean + 8u * stage, (turn & 1u) ^ 1u)) || !wait(kv_empty + 8u * stage, (turn & 1u) ^ 1u)) return false;
            own |= 1u;
            const bool there = mine && j < end;
            uint32_t boxes = (uint32_t)np * (D / 64);
            if (j == last_tile) boxes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, there));
            const uint32_t bar = kv_full + 8u * stage;
            if (lane == 0) mbar_arrive_expect_tx(bar, boxes * p.page_tx + p.withheld);
            __syncwarp();
            if (there) {
                bad |= (unsigned)page >= (unsigned)p.n_pages;
                const int off = tpp > 1 ? (int)((unsigned)(w.t0 + j) % (unsigned)tpp) * kAttnKeys : 0;
                tma_load_4d(box_at + stage * kTile, map, col * 64, off, w.h, page, bar);
            }
            __syncwarp();
            page = page_next;
        }
        return true;
    };

    uint32_t loads = 0;                                      // ring places used by the pieces before
    uint32_t q_n = 0;                                        // q slots used by them
    if (warp == kAttnProducer) {
        // ---------------------------------------------------------------- producer: this CTA's run, piece by piece, and the copies for it
        const int cta = (int)blockIdx.x, per = (p.B + 31) / 32;          // requests per lane
        const int b0 = min(lane * per, p.B), b1 = min(b0 + per, p.B);
        long long sum = 0;
#pragma unroll 1
        for (int b = b0; b < b1; ++b) sum += attn_head_weight(p, attn_request(p, b)) * p.Hkv;
        long long at = sum;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xFFFFFFFFu, at, o);
            if (lane >= o) at += v;
        }
        const long long W = __shfl_sync(0xFFFFFFFFu, at, 31);
        at -= sum;
        const int C = (int)max(1ll, min((long long)gridDim.x, attn_div(W, p.min_run)));
        const AttnCut cut(W, C);
        const long long g0 = cta < C ? cut.start(cta) : 0, g1 = cta < C ? cut.start(cta + 1) : 0;
        uint32_t made = 0;
        AttnSplit split{};
        auto publish = [&](const AttnPiece& w) -> bool {
            const uint32_t s = made % kAttnPieces, turn = made / kAttnPieces;
            if (turn > 0 && !wait(piece_empty + 8u * s, (turn - 1u) & 1u)) return false;
            if (lane == 0) {
                sh.piece[s] = w;
                mbar_arrive(piece_full + 8u * s);
            }
            __syncwarp();
            ++made;
            return true;
        };
        bool ok = true;
        if (g1 > g0) {
            const unsigned here = __ballot_sync(0xFFFFFFFFu, at <= g0 && g0 < at + sum);
            const int from = __ffs((int)here) - 1;
            long long s = __shfl_sync(0xFFFFFFFFu, at, from);            // where the request, then the item, begins
            bool first = true;
#pragma unroll 1
            for (int b = __shfl_sync(0xFFFFFFFFu, b0, from); b < p.B && s < g1 && ok; ++b) {
                const AttnRequest q = attn_request(p, b);
                if (q.T <= 0) continue;
                const long long weight = attn_head_weight(p, q);
                int h = 0;
                if (s + weight * p.Hkv <= g0) {
                    s += weight * p.Hkv;
                    continue;
                }
                if (s < g0) {
                    const long long skip = g0 - s;
                    h = (int)attn_div(skip, weight);
                    s += h * weight;
                }
                const int blocks = attn_blocks(p, q);
#pragma unroll 1
                for (; h < p.Hkv && s < g1 && ok; ++h) {
#pragma unroll 1
                    for (int i = 0; i < blocks && s < g1 && ok; ++i) {
                        AttnPiece w;
                        const AttnItem it(p, q, i, s);
                        s = it.end;
                        if (s <= g0) continue;
                        // a tile goes to the run that its place lies in; not cut: the item to the run it begins in
                        const long long lo = p.whole ? (it.begin >= g0 ? 0 : it.tiles) : (max(g0 - it.first, 0ll) + it.heavy) >> it.heavy;
                        const long long hi = p.whole ? it.tiles : min((g1 - it.first + it.heavy) >> it.heavy, (long long)it.tiles);
                        if (hi <= lo) continue;
                        w.tok0 = it.tok0;
                        w.ntok = it.ntok;
                        w.keys = it.keys;
                        w.n = (int)(hi - lo);
                        w.t0 = (int)lo;
                        w.b = b;
                        w.h = h;
                        w.open = min(w.keys, q.L + (p.mask ? 0 : w.tok0 + 1)) / kAttnKeys;
                        w.L = q.L;
                        w.T = q.T;
                        w.first = q.first;
                        w.dual = w.ntok > p.tpt;
                        w.cut = w.n < it.tiles;
                        w.slot = it.begin <= g0 ? 0 : 1;
                        w.pad[0] = w.pad[1] = 0;
                        ok = publish(w);
                        if (!ok) break;
#pragma unroll 1
                        for (int s = 0; s < 1 + w.dual && ok; ++s, ++q_n) {          // rows of q
                            const uint32_t slot = q_n & 1u, turn = q_n >> 1;
                            if (turn > 0 && !wait(q_empty + 8u * slot, (turn - 1u) & 1u)) { ok = false; break; }
                            if (attn_elect()) {
                                const uint32_t bar = q_full + 8u * slot, to = q_smem + slot * p.q_slot;
                                mbar_arrive_expect_tx(bar, p.q_tx + p.withheld);
#pragma unroll
                                for (int c = 0; c < D / 64; ++c)
#pragma unroll
                                    for (int k = 0; k < (REP ? 4 : 1); ++k)
                                        tma_load_3d(to + c * p.q_block + k * 4096, &maps.q, c * 64, w.h * p.G, w.first + w.tok0 + s * p.tpt, bar);
                            }
                            __syncwarp();
                        }
                        ok = ok && copy_tiles(w, loads, false);
                        loads += 2u * w.n;
                        // many items: the first CTA whose run begins behind the item's first tile names it for the join
                        if (p.entries == 0 && first && w.t0 > 0 && cut.of(it.first) == cta - 1) split = it.split(p, q, h, cut);
                        first = false;
                    }
                }
            }
        }
        if (ok) {
            AttnPiece end;
            end.n = 0;
            (void)publish(end);
        }
        if (!REP && cta < p.entries) {                       // few items: each has its entry
            const int b = cta / (p.Hkv * p.blocks), h = cta / p.blocks - b * p.Hkv, i = cta % p.blocks, from = b / per;
            long long s = __shfl_sync(0xFFFFFFFFu, at, from);
#pragma unroll 1
            for (int o = from * per; o < b; ++o) s += attn_head_weight(p, attn_request(p, o)) * p.Hkv;
            const AttnRequest q = attn_request(p, b);
            s += h * attn_head_weight(p, q);
            if (q.T > 0 && i < attn_blocks(p, q)) {
#pragma unroll 1
                for (int j = 0; j < i; ++j) s = AttnItem(p, q, j, s).end;
                split = AttnItem(p, q, i, s).split(p, q, h, cut);
            }
        }
        if (lane == 0 && cta < p.n_splits) p.splits[cta] = split;
        if (bad) atomicOr(&p.hdr->status, kStatusPage);
    } else if (warp == kAttnProducerV) {
        // ---------------------------------------------------------------- producer of values
        bool ok = true;
        for (AttnPiece w; ok && take(w); loads += 2u * w.n) ok = copy_tiles(w, loads, true);
        if (bad) atomicOr(&p.hdr->status, kStatusPage);
    } else if (warp == kAttnIssuer || (REP && warp == kAttnIssuer1)) {
        // ---------------------------------------------------------------- MMA issuers
        // A product takes 64 cycles, a wait 120.  Few rows: an issuer per stream, as one for both would be what all wait for.  Otherwise one for
        // both: P V and the next S of one stream, then of the other, so that the streams' scores are ready at different times (with an issuer
        // each, both fall into step, and exponentials and products take turns instead of overlapping: two long documents under 60 drafted
        // tokens 120 -> 133 us).  Where the next keys are there, they are not asked for between the two products: 4520 -> 4140 cycles for
        // both streams' half-steps, 2430 of them a stream's exponentials.  (The first half of P V as soon as half the weights are there: 115 ->
        // 120 us.)  Such a call draws 1000 W: it runs at 1.97 GHz for some milliseconds and at 1.6 GHz when repeated for seconds.
        bool ok = true;
        uint32_t p_phase = 0;
        uint32_t o_phase = 1, item = 0;
        const int own = REP ? (warp == kAttnIssuer ? 0 : 1) : 0;             // the first half-step it issues
        for (AttnPiece w; ok && take(w);) {
            const int H = w.steps();
            if (REP && !wait(q_full + 8u * (q_n & 1u), (q_n >> 1) & 1u)) break;
#pragma unroll 1
            for (int i = own - 2; i < H; i += REP ? 2 : 1) { // P V of half-step i, then S of the stream's next
                const int s = i & 1;
                const bool more = i + 2 < H;
                const uint32_t k_place = loads + w.k_at((i + 2) >> w.dual), k_turn = turn_of(k_place), k_st = k_place - k_turn * ST;
                const uint32_t qn = q_n + (w.dual ? (uint32_t)s : 0u), q_at = qn & 1u;
                auto score = [&]() {
                    const uint32_t idesc = kIdescS | ((uint32_t)attn_k_steps(w, (i + 2) >> w.dual) << 18);
                    const uint64_t a = smem_desc_sw128(q_smem + q_at * p.q_slot), bd = smem_desc_sw128(ring + k_st * kTile);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        tc_mma_bf16(tmem + kAttnTmemS + 128u * s, a + (uint64_t)((k >> 2) * (p.q_block >> 4) + (k & 3) * 2),
                                    bd + (uint64_t)((k >> 2) * (kBlock >> 4) + (k & 3) * 2), idesc, k > 0 ? 1u : 0u);
                    tc_commit(s_full + 8u * s);
                    tc_commit(kv_empty + 8u * k_st);
                    if (!REP && (i + 2) >> w.dual == w.n - 1) tc_commit(q_empty + 8u * q_at);
                };
                bool keys = false;                           // the next ones are there already: both products go out in one
                if (i >= 0) {
                    const uint32_t place = loads + w.v_at(i >> w.dual), turn = turn_of(place), st = place - turn * ST;
                    const int steps = attn_k_steps(w, i >> w.dual);
                    uint32_t bar0 = v_clean + 8u * st, par0 = turn & 1u, bar1 = p_full + 8u * s, par1 = p_phase >> s & 1u;
                    if (REP && D == 128 && i < 2) {      // an item's first weights before its values
                        const uint32_t bar = bar0, par = par0;
                        bar0 = bar1, par0 = par1, bar1 = bar, par1 = par;
                    }
                    if (!wait(bar0, par0)) { ok = false; break; }
                    if (!REP) keys = more && i + 2 > w.dual && attn_test(kv_full + 8u * k_st, k_turn & 1u);
                    if (!wait(bar1, par1)) { ok = false; break; }
                    p_phase ^= 1u << s;
                    tc_fence_after();
                    if (attn_elect()) {
                        const uint64_t bd = attn_v_desc(ring + st * kTile);
#pragma unroll
                        for (int k = 0; k < kAttnKeys / 16; ++k)
                            if (k < steps) tc_mma_bf16_ts(tmem + kAttnTmemO + 128u * s, tmem + kAttnTmemS + 128u * s + 8u * k, bd + (uint64_t)(128 * k), kIdescO,
                                                          i >= 2 || k > 0 ? 1u : 0u);
                        tc_commit(kv_empty + 8u * st);
                        if (!REP && i == H - 1) tc_commit(o_full);
                        if (keys) score();
                    }
                    __syncwarp();
                }
                if (more && !keys) {
                    if (!REP && i + 2 <= w.dual && !wait(q_full + 8u * q_at, (qn >> 1) & 1u)) { ok = false; break; }
                    if (!wait(kv_full + 8u * k_st, k_turn & 1u)) { ok = false; break; }
                    tc_fence_after();
                    if (attn_elect()) score();
                    __syncwarp();
                }
            }
            if (!ok) break;
            if constexpr (REP) {                             // also of a stream that has no part in the item: none is a phase ahead
                if (item++ > 0 && !wait(o_full, o_phase)) break;
                o_phase ^= 1u;
                if (attn_elect()) {
                    tc_commit(q_empty + 8u * (q_n & 1u));
                    tc_commit(o_full);
                }
                __syncwarp();
            }
            loads += 2u * w.n;
            q_n += 1u + w.dual;
        }
    } else if (warp == kAttnCleaner) {
        // ---------------------------------------------------------------- cleaner
        bool ok = true;
        for (AttnPiece w; ok && take(w);) {
#pragma unroll 1
            for (uint32_t e = 0; e < 2u * w.n; ++e) {        // every place, in order: a barrier is never a phase ahead of it
                const uint32_t place = loads + e, turn = turn_of(place), st = place - turn * ST;
                if (!wait(kv_full + 8u * st, turn & 1u)) { ok = false; break; }
                const int j = w.value_at(e);
                if (j >= 0 && w.t0 + j >= w.open) {
                    // positions all rows attend stay as they are, and no product reads past the last 16 that hold any
                    const int tile0 = (w.t0 + j) * kAttnKeys;
                    const int r0 = max(0, min(kAttnKeys, w.L - tile0)), r1 = attn_k_steps(w, j) * 16;
#pragma unroll 1
                    for (int c = 0; c < D / 64; ++c) {
#pragma unroll 4
                        for (int i = r0 * 8 + lane; i < r1 * 8; i += 32) {
                            uint4* u = reinterpret_cast<uint4*>(smem + (ring - base) + st * kTile + c * kBlock + i * 16);
                            uint4 x = *u;
                            // an exponent of ones carries into the bit above it
                            const uint32_t full = ((x.x & 0x7F807F80u) + 0x00800080u) | ((x.y & 0x7F807F80u) + 0x00800080u) |
                                                  ((x.z & 0x7F807F80u) + 0x00800080u) | ((x.w & 0x7F807F80u) + 0x00800080u);
                            if (__builtin_expect((full & 0x80008000u) != 0u, 0)) {
                                uint32_t* y = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
                                for (int g = 0; g < 4; ++g) {
                                    if ((y[g] & 0x7F800000u) == 0x7F800000u) y[g] = (y[g] & 0x8000FFFFu) | 0x7F7F0000u;
                                    if ((y[g] & 0x00007F80u) == 0x00007F80u) y[g] = (y[g] & 0xFFFF8000u) | 0x00007F7Fu;
                                }
                                *u = x;
                            }
                        }
                    }
                    fence_proxy_async_shared();
                    __syncwarp();
                }
                if (lane == 0) {
                    mbar_arrive(v_clean + 8u * st);
                    // for the stream that does not read it, too
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(kv_empty + 8u * st), "r"(w.dual ? 1u : 2u) : "memory");
                }
            }
            loads += 2u * w.n;
        }
    } else {
        // ---------------------------------------------------------------- softmax, and the end of an item
        const int s = warp >> 2, quad = warp & 3;
        const int r = quad * 32 + lane;                      // the thread's lane of its stream's tiles
        const uint32_t lane_at = (uint32_t)(quad * 32) << 16;
        const uint32_t t_s = tmem + kAttnTmemS + 128u * s + lane_at, t_o = tmem + kAttnTmemO + 128u * s + lane_at;
        bool ok = true;
        uint32_t s_phase = 0, o_phase = 0, meet_phase = 0, item = 0;
        auto meet_others = [&]() -> bool {                   // the eight warps here
            __syncwarp();
            if (lane == 0) mbar_arrive(meet);
            meet_phase ^= 1u;
            return wait(meet, meet_phase ^ 1u);
        };
        for (AttnPiece w; ok && take(w);) {
            const int H = w.steps();
            const int tile_tokens = w.dual ? (s ? w.ntok - p.tpt : p.tpt) : w.ntok;
            const int rows = tile_tokens * p.G;              // of this stream's tile
            const int my_row = REP ? lane : r;               // of the tile
            const bool real = my_row < rows, busy = REP || quad * 32 < rows;
            const int t = w.tok0 + (w.dual ? s * p.tpt : 0) + (real ? my_row / p.G : 0);      // its token within the request
            float m = -INFINITY, l = 0.0f, lr = 0.0f;        // lr (few rows): of the rounded weights
#pragma unroll 1
            for (int i = s; i < H; i += 2) {
                if (!wait(s_full + 8u * s, s_phase)) { ok = false; break; }
                s_phase ^= 1u;
                if (busy) {
                    tc_fence_after();
                    const int j = w.t0 + (i >> w.dual);
                    // where a tile's row has grown past the maximum in use (mx - m is infinite while nothing has been attended yet)
                    auto raise = [&](float mx) {
                        const bool grow = real && mx > m && !((mx - m) * p.scale_log2 <= kAttnSlack);
                        if (__any_sync(0xFFFFFFFFu, grow)) {
                            const float f = grow ? ex2_approx((m - mx) * p.scale_log2) : 1.0f;
                            if (grow) {
                                m = mx;
                                l *= f;
                                lr *= f;
                            }
                            if (i >= 2) {
#pragma unroll 1
                                for (int c = 0; c < D / 32; ++c) {
                                    uint32_t o[32];
                                    tc_ld32(t_o + 32u * c, o);
                                    tc_wait_ld();
#pragma unroll
                                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                    tc_st32(t_o + 32u * c, o);
                                }
                            }
                        }
                    };
                    auto seen = [&](int c) -> uint32_t {     // which of the tile's positions 32 c .. the row attends
                        const int32_t* row = p.mask ? p.mask + (int64_t)(w.first + t) * p.mask_words : nullptr;
                        const int at = j * kAttnKeys + 32 * c, n = w.keys - at;
                        const uint32_t bits = attn_bits(row, p.mask_words, t, w.T, at - w.L);
                        return bits & (n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u);
                    };
                    if constexpr (REP) {
                        // the warp's own 32 positions of the tile; its weights of the others are 0
                        uint32_t x[32], pk[16];
                        tc_ld32(t_s + 32u * quad, x);
                        tc_wait_ld();
                        if (j >= w.open) {
                            const uint32_t bits = seen(quad);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(bits >> e & 1u)) x[e] = 0xFF800000u;
                        }
                        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                        for (int e = 0; e < 32; e += 2) top[(e >> 1) & 1] = max3(top[(e >> 1) & 1], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                        __syncwarp();
                        raise(fmaxf(top[0], top[1]));
                        const float ref = m == -INFINITY ? 0.0f : -m * p.scale_log2;
                        const uint64_t k2 = pack2(p.scale_log2, p.scale_log2), r2 = pack2(ref, ref);
                        uint64_t sum0 = 0ull, sum1 = 0ull;
                        float lr0 = 0.0f, lr1 = 0.0f;
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float a, b;
                            unpack2(fma2(pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), k2, r2), a, b);
                            a = ex2_approx(a);
                            b = ex2_approx(b);
                            if (e & 2) sum1 = add2(sum1, pack2(a, b));
                            else sum0 = add2(sum0, pack2(a, b));
                            pk[e / 2] = attn_bf16x2(a, b);
                            attn_add_bf16x2(lr0, lr1, pk[e / 2]);
                        }
                        tc_st16(t_s + 16u * quad, pk);           // over scores of its own lanes, which it has read
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = 0u;
#pragma unroll
                        for (int k = 1; k < 4; ++k) tc_st16(t_s + 16u * ((quad + k) & 3), pk);
                        float a, b;
                        unpack2(add2(sum0, sum1), a, b);
                        l += a + b;
                        lr += lr0 + lr1;
                    } else {
                        if (j >= w.open) {                       // what the row does not attend: -infinity, back in its place
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
                                const uint32_t bits = seen(c);
                                uint32_t x[32];
                                __syncwarp();
                                tc_ld32(t_s + 32u * c, x);
                                tc_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!(bits >> e & 1u)) x[e] = 0xFF800000u;
                                tc_st32(t_s + 32u * c, x);
                            }
                            tc_wait_st();
                        }
                        // The scores are read twice, half of them at a time, for their maximum and for the weights.  (One pass with the old maximum,
                        // made again where it grew too much, has fewer instructions to issue but four times as many to fetch, as all weights wait in
                        // registers: slower by 5 to 10 %.  All scores kept in registers from the first reading: 111 -> 123 us for two long documents
                        // under 60 tokens, half of them 117; 32 at a time, the next on their way: the same.)
                        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            uint32_t x[64];
                            tc_ld64(t_s + 64u * c, x);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 64; e += 2) top[(e >> 1) & 3] = max3(top[(e >> 1) & 3], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                        }
                        raise(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
                        const float ref = m == -INFINITY ? 0.0f : -m * p.scale_log2;
                        const uint64_t k2 = pack2(p.scale_log2, p.scale_log2), r2 = pack2(ref, ref);
                        uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            uint32_t x[64], pk[32];
                            tc_ld64(t_s + 64u * c, x);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 64; e += 2) {
                                float a, b;
                                unpack2(fma2(pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), k2, r2), a, b);
                                a = ex2_approx(a);
                                b = ex2_approx(b);
                                if (e & 2) sum1 = add2(sum1, pack2(a, b));
                                else sum0 = add2(sum0, pack2(a, b));
                                pk[e / 2] = attn_bf16x2(a, b);
                            }
                            tc_st32(t_s + 32u * c, pk);          // over scores that have been read
                        }
                        float a, b;
                        unpack2(add2(sum0, sum1), a, b);
                        l += a + b;
                    }
                    tc_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8u * s);
            }
            // ---- the item's end: a piece of it to the workspace, or its rows
            if (!ok || !wait(o_full, o_phase)) { ok = false; break; }
            o_phase ^= 1u;
            tc_fence_after();
            const bool both = !w.dual && H > 1;              // the streams hold different positions of the same rows
            const size_t piece = (size_t)(blockIdx.x * 2 + w.slot);
            if constexpr (REP) {
                // Eight parts of each row, by stream and warp, meet in the item's slot of q: all columns of up to 8 rows at a time, half of those
                // of 16, a quarter of those of 32.  A thread adds up four columns of a row.
                float4* xs = reinterpret_cast<float4*>(smem + (item++ & 1u) * p.q_slot);
                // O has the rounded weights, so their sum lr is what it is divided by.  Instead of (m, l, lr) with l = 2^y lr, the rest of the way goes
                // with (m + y / (scale log2 e), lr), which has both: lse comes from l, O / lr has weights that add up to 1.  |l / lr - 1| <= 2^-8.
                if (lr > 0.0f && p.scale_inv > 0.0f) {
                    const float d = __fdividef(l - lr, lr);
                    m = fmaf(d * kLog2e * (1.0f - d * (0.5f - d * (1.0f / 3.0f))), p.scale_inv, m);
                    l = lr;
                }
                const int log_rows = rows <= 8 ? 3 : rows <= 16 ? 4 : 5, rounds = 1 << (log_rows - 3), quads = (D / 4) >> (log_rows - 3);
                sh.ms[s][r] = make_float2(m, l);
#pragma unroll 1
                for (int round = 0; round < rounds; ++round) {
                    if (s == 0 || both) {
                        const uint32_t at = t_o + (uint32_t)(round * quads * 4);
#pragma unroll 1
                        for (int c = 0; c < quads; c += 4) { // 16 columns at a time
                            uint32_t o[16];
                            tc_ld16(at + 4u * c, o);
                            tc_wait_ld();
                            if (real) {
                                float4* to = xs + ((((s * 4 + quad) * quads + c) << log_rows) + lane);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    to[e << log_rows] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                                                                    __uint_as_float(o[4 * e + 3]));
                            }
                            __syncwarp();
                        }
                    }
                    if (!meet_others()) { ok = false; break; }
                    const int row = tid & ((1 << log_rows) - 1), parts = both ? 8 : 4;
                    if (row < rows) {
                        float2 ml[8];
                        float top = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            ml[k] = sh.ms[k >> 2][(k & 3) * 32 + row];
                            top = fmaxf(top, ml[k].x);
                        }
                        const float ref = top == -INFINITY ? 0.0f : top;
                        float total = 0.0f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            ml[k].x = ex2_approx((ml[k].x - ref) * p.scale_log2);
                            total = fmaf(ml[k].y, ml[k].x, total);
                        }
                        const float inv = w.cut ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
                        const int my_t = row / p.G, head = w.h * p.G + (row - my_t * p.G);
                        const int64_t token = w.first + w.tok0 + my_t;
                        for (int cq = tid >> log_rows; cq < quads; cq += 256 >> log_rows) {
                            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                if (k >= parts) break;
                                const float4 u = xs[((k * quads + cq) << log_rows) + row];
                                v = make_float4(fmaf(u.x, ml[k].x, v.x), fmaf(u.y, ml[k].x, v.y), fmaf(u.z, ml[k].x, v.z), fmaf(u.w, ml[k].x, v.w));
                            }
                            const int cq_all = round * quads + cq;
                            if (w.cut) reinterpret_cast<float4*>(p.part_o)[(piece * (D / 4) + cq_all) * p.rows_max + row] = v;
                            else
                                *reinterpret_cast<uint2*>(p.out + token * p.out_ts + (int64_t)head * p.out_hs + 4 * cq_all) =
                                    make_uint2(attn_bf16x2(v.x * inv, v.y * inv), attn_bf16x2(v.z * inv, v.w * inv));
                            if (cq_all == 0) {
                                if (w.cut) p.part_ml[piece * p.rows_max + row] = make_float2(top, total);
                                else if (p.lse) p.lse[token * p.Hq + head] = total == 0.0f ? -INFINITY : top * p.scale + logf(total);
                            }
                        }
                    }
                    if (round + 1 < rounds && !meet_others()) { ok = false; break; }
                }
                if (!ok) break;
                fence_proxy_async_shared();                         // the slot's next contents come by TMA
                tc_fence_before();
                if (!meet_others()) { ok = false; break; }
                if (tid == 0) mbar_arrive(q_empty + 8u * ((item - 1u) & 1u));
                continue;
            }
            float f0 = 1.0f, f1 = 0.0f;                      // weights of stream 0's (of this stream's) and stream 1's O
            if (both) {
                sh.ms[s][r] = make_float2(m, l);
                if (!meet_others()) { ok = false; break; }
                const float2 a = sh.ms[0][r], b = sh.ms[1][r];
                m = fmaxf(a.x, b.x);
                f0 = a.x == m ? 1.0f : ex2_approx((a.x - m) * p.scale_log2);
                f1 = b.x == m ? 1.0f : ex2_approx((b.x - m) * p.scale_log2);
                l = a.y * f0 + b.y * f1;
            }
            if (busy && (w.dual || both || s == 0)) {
                const int row = (w.dual ? s * p.tpt * p.G : 0) + r, head = w.h * p.G + (real ? r % p.G : 0);
                const uint32_t o_at = w.dual ? t_o : tmem + kAttnTmemO + lane_at;
                const int c0 = both ? s * (D / 64) : 0, c1 = both ? c0 + D / 64 : D / 32;        // runs of 32 columns
                const float inv = w.cut ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
                uint16_t* to = p.out + (int64_t)(w.first + t) * p.out_ts + (int64_t)head * p.out_hs;
#pragma unroll 1
                for (int c = c0; c < c1; ++c) {
                    __syncwarp();
                    uint32_t o[32];
                    tc_ld32(o_at + 32u * c, o);
                    if (both) {
                        uint32_t o1[32];
                        tc_ld32(o_at + 128u + 32u * c, o1);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f0 + __uint_as_float(o1[e]) * f1);
                    } else {
                        tc_wait_ld();
                    }
                    if (!real) continue;
                    if (w.cut) {
                        float4* po = reinterpret_cast<float4*>(p.part_o) + (piece * (D / 4) + 8 * c) * p.rows_max + row;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            po[(size_t)e * p.rows_max] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                                                     __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t v[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                v[u] = attn_bf16x2(__uint_as_float(o[e + 2 * u]) * inv, __uint_as_float(o[e + 2 * u + 1]) * inv);
                            *reinterpret_cast<uint4*>(to + 32 * c + e) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
                if (real && (w.dual || s == 0)) {
                    if (w.cut) p.part_ml[piece * p.rows_max + row] = make_float2(m, l);
                    else if (p.lse) p.lse[(int64_t)(w.first + t) * p.Hq + head] = l == 0.0f ? -INFINITY : m * p.scale + logf(l);
                }
                tc_fence_before();
            }
            if (!meet_others()) ok = false;                  // both streams' O and (m, l) have been read; neither is an item ahead
        }
    }

    tc_fence_before();
    __syncthreads();
    if (__builtin_expect(*abort_flag != 0, 0)) {             // copies and MMAs in flight must end before their memory is given back
        if ((warp == kAttnIssuer || warp == kAttnIssuer1) && attn_elect()) {
            const uint32_t bar = drain + (warp == kAttnIssuer ? 0u : 8u);
            tc_commit(bar);
            (void)mbar_wait(bar, 0u, p.wait_ns);
        }
        if ((warp == kAttnProducer || warp == kAttnProducerV) && lane == 0) {        // longer than any copy takes
            const unsigned long long now = global_timer_ns();
            while (global_timer_ns() - now < 1000000ull) { }
        }
        __syncwarp();
        tc_fence_before();
        __syncthreads();
    }
    tc_fence_after();
    if (warp == kAttnIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// ------------------------------------------------------------------------------------------ joining an item's pieces
// lse and out of rows that several CTAs have pieces of: weights 2^{(m_c - m) scale log2 e}, pieces in the order of the CTAs.  Block (c, y) takes
// entry c, every gridDim.y-th group of the item's rows; an entry is an item, where rows are many and there may be no more items than CTAs, or the item that CTA c
// is the first to go on with; a thread has four columns of a row and asks for all it needs of BATCH pieces
// at once, so that an item of as many pieces costs one memory round trip behind its entry.  Each thread works its row's weights out for
// itself: a step through shared memory, and finding the groups by a sum over all entries, took 25 us where this takes 8.
// Eight pieces at a time with few rows, where pieces are many and their latencies are what it costs (one token of eight heads on a key head over 60000: the
// whole call 25.6 us, 29.7 with four); else four (16 x 60 over 8000: eight take 2 us more).
template <int D, int BATCH>
__global__ void __launch_bounds__(256)
attn_join_kernel(const __grid_constant__ AttnParams p) {
    constexpr int kRows = 1024 / D, kQuads = D / 4;          // rows and runs of four columns that 256 threads cover
    grid_dependency_wait();
    if (threadIdx.x == 0) grid_launch_dependents();
    const AttnSplit d = p.splits[blockIdx.x];
    const int cq = (int)threadIdx.x / kRows;
    for (int row = (int)blockIdx.y * kRows + (int)threadIdx.x % kRows; row < d.rows; row += (int)gridDim.y * kRows) {
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int i0 = 0; i0 < d.n_pieces; i0 += BATCH) {
            float2 ml[BATCH];
            float4 v[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = i0 + k;
                ml[k] = make_float2(-INFINITY, 0.0f);
                v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (i < d.n_pieces) {
                    const size_t piece = (size_t)(d.first_cta + i) * 2 + (i == 0 ? d.first_slot : 0);
                    ml[k] = p.part_ml[piece * p.rows_max + row];
                    v[k] = reinterpret_cast<const float4*>(p.part_o)[(piece * kQuads + cq) * p.rows_max + row];
                }
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) top = fmaxf(top, ml[k].x);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float f = ex2_approx((m - ref) * p.scale_log2);
            m = top;
            l *= f;
            o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float w = ex2_approx((ml[k].x - ref) * p.scale_log2);
                l = fmaf(ml[k].y, w, l);
                o = make_float4(fmaf(v[k].x, w, o.x), fmaf(v[k].y, w, o.y), fmaf(v[k].z, w, o.z), fmaf(v[k].w, w, o.w));
            }
        }
        const float n = l == 0.0f ? 0.0f : 1.0f / l;
        const int t = row / p.G, token = d.token0 + t, head = d.head0 + (row - t * p.G);
        *reinterpret_cast<uint2*>(p.out + (int64_t)token * p.out_ts + (int64_t)head * p.out_hs + 4 * cq) =
            make_uint2(attn_bf16x2(o.x * n, o.y * n), attn_bf16x2(o.z * n, o.w * n));
        if (cq == 0 && p.lse) p.lse[(int64_t)token * p.Hq + head] = l == 0.0f ? -INFINITY : m * p.scale + logf(l);
    }
}

#endif  // __CUDACC__

// ------------------------------------------------------------------------------------------ host
static int attn_rows(int Hq, int heads, int max_tokens) {    // of a block, at most
    const int G = Hq / heads, tpt = 128 / G;
    return std::min(2 * tpt, max_tokens) * G;
}
struct AttnLayout {
    size_t splits, ml, o, total;
};
static AttnLayout attn_layout(int Hq, int heads, int D, int max_tokens) {
    const size_t rows = (size_t)attn_rows(Hq, heads, max_tokens), pieces = 2 * kAttnCtas;
    AttnLayout a;
    a.splits = kHeaderBytes;
    a.ml = (a.splits + kAttnCtas * sizeof(AttnSplit) + 255) / 256 * 256;
    a.o = (a.ml + pieces * rows * sizeof(float2) + 255) / 256 * 256;
    a.total = (a.o + pieces * rows * D * sizeof(float) + 255) / 256 * 256;
    return a;
}
size_t attn_workspace_bytes(int Hq, int heads, int D, int max_tokens) { return attn_layout(Hq, heads, D, max_tokens).total; }

// (defined beside make_tensor_map_bf16)
vt_status make_tensor_map_bf16_nd(CUtensorMap* map, const void* ptr, int rank, const uint64_t* dims, const uint64_t* strides, const uint32_t* box,
                                  bool alone);

static vt_status cache_map(CUtensorMap* map, const void* ptr, const vt_cache& a, int64_t token, int64_t head, int64_t page) {
    const uint64_t dims[4] = {(uint64_t)a.head_dim, (uint64_t)a.page_size, (uint64_t)a.heads, (uint64_t)a.n_pages};
    const uint64_t strides[3] = {(uint64_t)token * 2, (uint64_t)head * 2, (uint64_t)page * 2};
    const uint32_t box[4] = {(uint32_t)kBoxK, (uint32_t)std::min(a.page_size, kAttnKeys), 1, 1};
    // 64 columns whose neighbours in memory belong to another head, and to another time (24 x 8 over 10000, D = 64: 475 -> 410 us)
    return make_tensor_map_bf16_nd(map, ptr, 4, dims, strides, box, a.head_dim == kBoxK && token != a.head_dim);
}

template <int D, bool REP>
static vt_status run_attn(const AttnMaps& maps, const AttnParams& p, int C, uint32_t smem, cudaStream_t st) {
    static std::atomic<unsigned long long> configured{0};
    if (vt_status r = ensure_max_dyn_smem(reinterpret_cast<const void*>(attn_kernel<D, REP>), kMaxDynSmem, &configured); r != VT_OK) return r;
    cudaError_t e = launch_pdl(attn_kernel<D, REP>, C, attn_threads(REP), smem, st, maps, p);
    count_launch();
    if (e == cudaSuccess && !p.whole) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)p.n_splits, (unsigned)((p.rows_max + 1024 / D - 1) / (1024 / D)));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, attn_join_kernel<D, REP ? 8 : 4>, p);
        count_launch();
    }
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

vt_status launch_attn(const AttnCall& c, void* workspace, cudaStream_t st) {
    const vt_cache& a = *c.cache;
    const int D = a.head_dim;
    int sms = 0;
    if (vt_status r = device_sm_count(&sms); r != VT_OK) return r;
    const int C = std::min(sms, kAttnCtas);
    AttnParams p{};
    p.cu = c.cu_tokens;
    p.lens = a.lens;
    p.page_table = a.page_table;
    p.table_stride = a.table_stride;
    p.mask = c.mask;
    p.mask_words = c.mask_words;
    p.out = reinterpret_cast<uint16_t*>(c.out.ptr);
    p.out_ts = c.out.token_stride;
    p.out_hs = c.out.head_stride;
    p.lse = c.lse;
    const AttnLayout lay = attn_layout(c.Hq, a.heads, D, c.max_tokens);
    unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
    p.hdr = reinterpret_cast<WsHeader*>(ws);
    p.splits = reinterpret_cast<AttnSplit*>(ws + lay.splits);
    p.part_ml = reinterpret_cast<float2*>(ws + lay.ml);
    p.part_o = reinterpret_cast<float*>(ws + lay.o);
    p.rows_max = attn_rows(c.Hq, a.heads, c.max_tokens);
    p.N = c.N;
    p.B = a.B;
    p.Hq = c.Hq;
    p.Hkv = a.heads;
    p.G = c.Hq / a.heads;
    p.max_tokens = c.max_tokens;
    p.n_pages = a.n_pages;
    p.page_size = a.page_size;
    p.max_pages = a.max_pages;
    p.tpt = 128 / p.G;
    p.box_tokens = std::min(p.tpt, c.max_tokens);
    p.whole = (long long)a.max_pages * a.page_size <= (long long)kAttnWhole * kAttnKeys;
    const bool few = p.rows_max <= 32;
    p.blocks = (std::min(c.max_tokens, c.N) + 2 * p.tpt - 1) / (2 * p.tpt);
    const long long items = (long long)a.B * a.heads * p.blocks;
    // Most CTAs name no item where there are few: 30 blocks each for 240 rows, only to leave (1 x 60 over 4000: 24 us so, 21.6 with an entry per item).
    // With few rows there are four at most, and the entries' code costs as much.
    p.entries = !p.whole && !few && items <= C ? (int)items : 0;
    p.n_splits = p.whole ? 0 : p.entries > 0 ? p.entries : C;
    p.min_run = p.rows_max > 128 ? 6 : 2;                      // (1 x 60 over 4000: 24.7 us with 8, 23.6 with 6)
    p.scale = c.scale;
    p.scale_log2 = c.scale * kLog2e;
    p.scale_inv = c.scale >= FLT_MIN ? 1.0f / p.scale_log2 : 0.0f;
    p.wait_ns = kWaitLimitNs;
    if (const int us = gemm_withheld_us(); us > 0) {         // a test of the unwinding: copies fall 16 bytes short
        p.withheld = 16;
        p.wait_ns = (unsigned long long)us * 1000ull;
    }
    const uint32_t rows = (uint32_t)(p.box_tokens * p.G);
    p.q_block = few ? 16384u : (rows + 7) / 8 * 1024;
    p.q_slot = p.q_block * (D / 64);
    p.q_tx = rows * 128u * (D / 64) * (few ? 4u : 1u);
    p.page_tx = (uint32_t)std::min(p.page_size, kAttnKeys) * 128u;
    // five stages of 32 KB beside two full row tiles: 160 KB in flight
    const uint32_t tile = kAttnKeys * D * 2, tail = sizeof(AttnShared) + 8 * (3 * kAttnMaxStages + 12 + 2 * kAttnPieces);
    p.n_stages = (int)std::min((uint32_t)kAttnMaxStages, ((uint32_t)kMaxDynSmem - tail - 2 * p.q_slot) / tile);
    constexpr int kRoom = kMaxDynSmem - (int)sizeof(AttnShared) - 8 * (3 * kAttnMaxStages + 12 + 2 * kAttnPieces);
    static_assert((kRoom - 2 * 32768) / (kAttnKeys * 128 * 2) >= 5 && (kRoom - 2 * 16384) / (kAttnKeys * 64 * 2) >= 7, "see the turns of the ring");
    p.stages_inv = (uint32_t)((0x100000000ull + p.n_stages - 1) / p.n_stages);
    p.shared_off = 2 * p.q_slot + p.n_stages * tile;
    p.bar_off = p.shared_off + sizeof(AttnShared);
    const uint32_t smem = p.shared_off + tail;
    AttnMaps maps;
    {
        const uint64_t dims[3] = {(uint64_t)D, (uint64_t)c.Hq, (uint64_t)c.N};
        const uint64_t strides[2] = {(uint64_t)c.q.head_stride * 2, (uint64_t)c.q.token_stride * 2};
        const uint32_t box[3] = {(uint32_t)kBoxK, (uint32_t)p.G, (uint32_t)p.box_tokens};
        if (vt_status r = make_tensor_map_bf16_nd(&maps.q, c.q.ptr, 3, dims, strides, box, false); r != VT_OK) return r;
    }
    if (vt_status r = cache_map(&maps.k, a.k, a, a.k_token_stride, a.k_head_stride, a.k_page_stride); r != VT_OK) return r;
    if (vt_status r = cache_map(&maps.v, a.v, a, a.v_token_stride, a.v_head_stride, a.v_page_stride); r != VT_OK) return r;
    if (few) return D == 64 ? run_attn<64, true>(maps, p, C, smem, st) : run_attn<128, true>(maps, p, C, smem, st);
    return D == 64 ? run_attn<64, false>(maps, p, C, smem, st) : run_attn<128, false>(maps, p, C, smem, st);
}

}  // namespace vt
