// Plans of the matrix products in vt_gemm.cuh, and the products that are stored as they are.
#include "vt_gemm.cuh"

namespace vt {

// Shared memory of a plan whose tile shape is chosen; false if it does not fit.
static bool gemm_layout(GemmParams* p, bool a_mn, bool b_mn, bool pair) {
    p->a_bytes = 128u * 128u;
    p->b_bytes = (uint32_t)(pair ? p->NT / 2 : p->NT) * 128u;
    p->blk_bytes = p->a_bytes + (uint32_t)round_up(p->b_bytes, 1024);
    // A hand-over of a stage costs the issuing threads some 300 cycles, more than the MMAs of a k-block on a narrow tile: as
    // many k-blocks per stage as leave three stages, at most four.
    p->kbs = std::max(1, std::min(4, (int)(72 * 1024 / p->blk_bytes)));
    p->stage_bytes = p->blk_bytes * (uint32_t)p->kbs;
    const size_t bar_bytes = (size_t)(2 * kGemmMaxStages + 5) * 8 + 16;
    const size_t partial = p->splits > 1 ? (size_t)(128 / p->rep) * (p->NT + 4) * 4 : 0;
    p->n_stages = std::min<int>(kGemmMaxStages, (int)((kMaxDynSmem - 1024 - round_up(bar_bytes, 128)) / p->stage_bytes));
    if (p->n_stages < 2) return false;
    p->bar_off = (uint32_t)round_up(std::max((size_t)p->n_stages * p->stage_bytes, partial), 128);
    p->total_smem = (uint32_t)(p->bar_off + bar_bytes + 1024);
    // D fp32, A and B bf16, M = 128 (a pair: 256), N; bits 15 and 16: A, B MN-major
    p->idesc = (1u << 4) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
               ((uint32_t)(p->NT >> 3) << 17) | ((uint32_t)((pair ? 256 : 128) >> 4) << 24);
    p->acc_cols = 32;
    while (p->acc_cols < (uint32_t)p->NT) p->acc_cols *= 2;
    p->tmem_cols = 2 * p->acc_cols;
    return p->total_smem <= (uint32_t)kMaxDynSmem;
}

static bool gemm_number_items(GemmParams* p, bool pair) {
    const int TM = pair ? 256 : 128, cols = p->dual ? p->NT / 2 : p->NT;
    long long items = 0;
    for (int i = 0; i < p->n_prob; ++i) {
        GemmProblem& q = p->prob[i];
        q.tiles_m = ceil_div(q.M, TM);
        q.tiles_n = ceil_div(q.N, cols);
        q.chunks_n = ceil_div(q.tiles_n, p->tiles_per_item);
        q.first_item = (int)items;
        items += (long long)q.tiles_m * q.chunks_n;
        if (items > (1 << 28)) return false;
    }
    p->n_items = (int)items;
    return true;
}

// Time of a plan in SM cycles, to compare plans with: per 64-deep k-block the tensor core takes 2 cycles per accumulator
// column (128 rows; a pair the same), at least 130, and the operands come in at about 55 bytes a cycle; weights from HBM
// at 24 bytes a cycle and SM when all of them stream.  Each tile adds its read-out, each launch its fill.
bool gemm_plan(GemmParams* p, bool a_mn, bool b_mn, bool dual, bool* pair_out) {
    int maxM = 0, max_nk = 0;
    for (int i = 0; i < p->n_prob; ++i) {
        maxM = std::max(maxM, p->prob[i].M);
        max_nk = std::max(max_nk, p->prob[i].nk0 + p->prob[i].nk1);
    }
    p->dual = dual;
    p->tiles_per_item = 1;
    double best = -1;
    int best_nt = 0, best_splits = 1;
    bool best_pair = false;
    const int one_rep = a_mn ? 1 : maxM <= 32 ? 4 : maxM <= 64 ? 2 : 1;
    for (int pair = 0; pair < 2; ++pair) {
        if (pair && maxM <= 128) continue;
        const int step = b_mn ? (pair ? 128 : 64) : pair ? 32 : 16;
        for (int nt = 256; nt >= step; nt -= step) {
            const int cols = dual ? nt / 2 : nt;
            long long tiles = 0;
            for (int i = 0; i < p->n_prob; ++i)
                tiles += (long long)ceil_div(p->prob[i].M, pair ? 256 : 128) * ceil_div(p->prob[i].N, cols);
            for (int s = 1; s <= (pair ? 1 : std::min(8, max_nk)); ++s) {
                const double in_bytes = (128.0 + (pair ? nt / 2 : nt)) * 128.0;
                double per_kb = std::max(std::max(2.0 * nt, 130.0), in_bytes / 55.0);
                const long long slots = pair ? kGemmSms / 2 : kGemmSms;
                const double waves = (double)((tiles * s + slots - 1) / slots);
                const double share = std::min(1.0, (double)(tiles * s) / (double)slots);
                per_kb = std::max(per_kb, nt * 128.0 * (pair ? 0.5 : 1.0) / 24.0 * (maxM <= 256 ? share : 0.0));
                const double tail = 1500.0 + 12.0 * cols + (s > 1 ? 2500.0 + 4.0 * nt : 0.0);
                const double cost = waves * (ceil_div(max_nk, s) * per_kb + 300.0) + tail;
                if (best < 0 || cost < best) {
                    best = cost;
                    best_nt = nt;
                    best_splits = s;
                    best_pair = pair != 0;
                }
            }
        }
    }
    p->NT = best_nt;
    p->splits = best_splits;
    p->rep = best_pair ? 1 : one_rep;
    *pair_out = best_pair;
    return gemm_number_items(p, best_pair) && gemm_layout(p, a_mn, b_mn, best_pair);
}

// Scoring: every row needs all columns, so nothing but the tile width and the number of tiles a CTA takes in a row is
// free.  Chosen for the fewest rounds of equal work over the SMs (a round costs its columns plus about 24 columns' worth
// of hand-over); among equals the longer runs, which leave fewer records to merge.
bool gemm_plan_rows(GemmParams* p, bool* pair_out) {
    const GemmProblem& q = p->prob[0];
    const bool pair = q.M > 128;
    const int slots = pair ? kGemmSms / 2 : kGemmSms, step = pair ? 32 : 16;
    const long long tiles_m = ceil_div(q.M, pair ? 256 : 128);
    double best = -1;
    int best_nt = 0, best_c = 1;
    for (int nt = 256; nt >= step; nt -= step) {
        const long long tiles_n = ceil_div(q.N, nt);
        for (int c = 1; c <= 16; ++c) {
            const long long items = tiles_m * ceil_div(tiles_n, c);
            const double rounds = (double)((items + slots - 1) / slots);
            const double cost = rounds * c * (nt + 24.0) + 40.0 / c;
            if (best < 0 || cost < best) {
                best = cost;
                best_nt = nt;
                best_c = c;
            }
        }
    }
    p->dual = 0;
    p->NT = best_nt;
    p->tiles_per_item = best_c;
    p->splits = 1;
    p->rep = pair ? 1 : q.M <= 32 ? 4 : q.M <= 64 ? 2 : 1;
    *pair_out = pair;
    return gemm_number_items(p, pair) && gemm_layout(p, false, false, pair);
}

int gemm_box_a(const GemmParams& p, bool a_mn) { return a_mn ? 64 : 128 / p.rep; }
int gemm_box_b(const GemmParams& p, bool b_mn, bool pair) { return b_mn ? 64 : (pair || p.dual) ? p.NT / 2 : p.NT; }

vt_status gemm_store(const GemmMaps& maps, const GemmParams& p, bool pair, bool a_mn, bool b_mn, cudaStream_t st) {
    const EpiStore::Params none{};
    if (!a_mn && !b_mn) return gemm_launch<false, false, EpiStore>(maps, p, pair, none, st);
    if (!a_mn) return gemm_launch<false, true, EpiStore>(maps, p, pair, none, st);
    return gemm_launch<true, true, EpiStore>(maps, p, pair, none, st);
}

}  // namespace vt
