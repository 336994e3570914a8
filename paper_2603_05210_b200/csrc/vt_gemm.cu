// Plans of the matrix products in vt_gemm.cuh, and the products that are stored as they are.
#include <cmath>
#include <cstring>

#include "vt_gemm.cuh"

namespace vt {

// Shared memory of a plan whose tile shape is chosen; false if it does not fit.
static bool gemm_layout(GemmParams* p, bool a_mn, bool b_mn, bool pair, uint32_t scratch_bytes) {
    int max_m = 0;
    for (int i = 0; i < p->n_prob; ++i) max_m = std::max(max_m, p->prob[i].M);
    const int tile_rows = 128 / p->rep;
    if (p->splits > 1) scratch_bytes = 0;        // its results are not staged
    const int box_m = (int)round_up((size_t)std::min(max_m, 128), 8);
    p->a_rows = (uint32_t)(a_mn ? 128 : std::min(tile_rows, box_m));
    p->a_bytes = p->rep > 1 ? 16384u : p->a_rows * 128u;
    p->b_bytes = (uint32_t)(pair ? p->NT / 2 : p->NT) * 128u;
    p->tx_bytes = p->a_rows * 128u * (uint32_t)p->rep + p->b_bytes;
    p->blk_bytes = p->a_bytes + (uint32_t)round_up(p->b_bytes, 1024);
    const size_t bar_bytes = (size_t)(2 * kGemmMaxStages + 6) * 8 + sizeof(GemmTable);      // barriers, two words, the problems
    const int groups = (p->dual ? p->NT / 2 : p->NT) / 8;
    p->x_rows = (uint32_t)box_m;
    p->x_part = p->x_rows * (uint32_t)(ceil_div(groups, p->splits) * (p->dual ? 16 : 8) * 4);
    const size_t partial = p->splits > 1 ? (size_t)p->x_part * p->splits : 0;
    const size_t over = 16384 - p->a_bytes;      // an MMA reads 128 rows of A wherever they end
    const size_t room = kMaxDynSmem - 2048 - round_up(bar_bytes, 128) - scratch_bytes - over;
    // A hand-over of a stage costs the issuing threads some 300 cycles, more than the MMAs of a k-block on a narrow tile: as
    // many k-blocks per stage as leave three stages, at most four.
    p->kbs = std::max(1, std::min(4, (int)(room / (3 * p->blk_bytes))));
    p->stage_bytes = p->blk_bytes * (uint32_t)p->kbs;
    p->n_stages = std::min<int>(kGemmMaxStages, (int)(room / p->stage_bytes));
    if (p->n_stages < 2) return false;
    p->scratch_off = (uint32_t)round_up(std::max((size_t)p->n_stages * p->stage_bytes + over, partial), 1024);
    p->bar_off = p->scratch_off + scratch_bytes;
    p->total_smem = (uint32_t)(p->bar_off + bar_bytes + 1024);
    // D fp32, A and B bf16, M = 128 (a pair: 256), N; bits 15 and 16: A, B MN-major
    p->idesc = (1u << 4) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
               ((uint32_t)(p->NT >> 3) << 17) | ((uint32_t)((pair ? 256 : 128) >> 4) << 24);
    p->acc_cols = 32;
    while (p->acc_cols < (uint32_t)p->NT) p->acc_cols *= 2;
    p->tmem_cols = 2 * p->acc_cols;
    p->wait_ns = kWaitLimitNs;
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

// Plans by shape, the last few of each thread: a plan weighs a hundred and more alternatives, which takes longer than the
// launch it is for.
struct PlanCache {
    struct Key {
        int n[3][4], n_prob, kind;
        bool operator==(const Key& o) const { return memcmp(this, &o, sizeof(Key)) == 0; }
    };
    struct Entry {
        Key key;
        GemmParams plan;
        bool pair, used;
    };
    static constexpr int kEntries = 32;
    Entry e[kEntries];
    int next;

    static Key key_of(const GemmParams& p, int kind) {
        Key k;
        memset(&k, 0, sizeof(k));
        k.n_prob = p.n_prob;
        k.kind = kind;
        for (int i = 0; i < p.n_prob; ++i) {
            k.n[i][0] = p.prob[i].M;
            k.n[i][1] = p.prob[i].N;
            k.n[i][2] = p.prob[i].nk0;
            k.n[i][3] = p.prob[i].nk1;
        }
        return k;
    }
    // what a plan does not decide stays the caller's
    static void take(const GemmParams& plan, GemmParams* p) {
        GemmParams r = plan;
        r.hdr = p->hdr;
        r.b_early = p->b_early;
        for (int i = 0; i < p->n_prob; ++i) {
            r.prob[i].a0 = p->prob[i].a0;
            r.prob[i].b0 = p->prob[i].b0;
            r.prob[i].a1 = p->prob[i].a1;
            r.prob[i].b1 = p->prob[i].b1;
        }
        *p = r;
    }
    bool find(const Key& k, GemmParams* p, bool* pair) const {
        for (const Entry& x : e)
            if (x.used && x.key == k) {
                take(x.plan, p);
                *pair = x.pair;
                return true;
            }
        return false;
    }
    void keep(const Key& k, const GemmParams& p, bool pair) {
        e[next] = Entry{k, p, pair, true};
        next = (next + 1) % kEntries;
    }
};
static thread_local PlanCache g_plans{};

// Clusters of `size` single-CTA tiles that the device holds at once (the SMs of a cluster lie in one GPC, so large
// clusters leave SMs over).  Without a device: what a B200 measured.
static int cluster_slots(int size) {
    static std::atomic<int> cached[9];
    static const int kUsual[9] = {0, 148, 74, 44, 35, 28, 22, 16, 14};
    int n = cached[size].load(std::memory_order_relaxed);
    if (n == 0) {
        n = kUsual[size];
        if (size > 1) {
            static std::atomic<unsigned long long> configured{0};
            auto* kernel = gemm_kernel<false, false, false, EpiStore>;
            int sms = 0, found = 0;
            if (device_sm_count(&sms) == VT_OK &&
                ensure_max_dyn_smem(reinterpret_cast<const void*>(kernel), kMaxDynSmem, &configured) == VT_OK) {
                cudaLaunchConfig_t cfg{};
                cfg.gridDim = dim3((unsigned)(sms / size * size));
                cfg.blockDim = dim3((unsigned)kGemmThreads);
                cfg.dynamicSmemBytes = kMaxDynSmem;
                cudaLaunchAttribute attr[1];
                attr[0].id = cudaLaunchAttributeClusterDimension;
                attr[0].val.clusterDim.x = (unsigned)size;
                attr[0].val.clusterDim.y = 1;
                attr[0].val.clusterDim.z = 1;
                cfg.attrs = attr;
                cfg.numAttrs = 1;
                if (cudaOccupancyMaxActiveClusters(&found, kernel, &cfg) == cudaSuccess && found > 0) n = found;
            }
            (void)cudaGetLastError();
        }
        cached[size].store(n, std::memory_order_relaxed);
    }
    return n;
}

// Time of a plan in SM cycles, to compare plans with.  Per 64-deep k-block the tensor core takes 2 cycles per accumulator
// column (128 rows; a pair the same); the issuing threads take some 250 for the MMAs and copies of a narrow tile and share
// 400 per stage; an SM takes in 40 bytes a cycle from HBM and 58 from L2 (measured with 22 and with 148 CTAs at work), and
// weights stream at 24 bytes a cycle and SM when all of them take part.  Each round of tiles adds its fill, the last its
// read-out, and splits the exchange of their partial sums.
bool gemm_plan(GemmParams* p, bool a_mn, bool b_mn, bool dual, uint32_t scratch_bytes, bool* pair_out) {
    const PlanCache::Key key = PlanCache::key_of(*p, (a_mn ? 1 : 0) | (b_mn ? 2 : 0) | (dual ? 4 : 0) | (int)scratch_bytes << 5);
    if (g_plans.find(key, p, pair_out)) return true;
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
    for (int pair = 0; pair < 2; ++pair) {
        if (pair && maxM <= 128) continue;
        const int step = b_mn ? (pair ? 128 : 64) : pair ? 32 : 16;
        for (int nt = 256; nt >= step; nt -= step) {
            const int cols = dual ? nt / 2 : nt;
            long long tiles = 0;
            for (int i = 0; i < p->n_prob; ++i)
                tiles += (long long)ceil_div(p->prob[i].M, pair ? 256 : 128) * ceil_div(p->prob[i].N, cols);
            const double a_rows = std::min(128, maxM);
            const double blk = (a_rows + (pair ? nt / 2 : nt)) * 128.0;
            const double per_stage = std::max(1.0, std::min(4.0, floor(64.0 * 1024 / blk)));
            const double issue = std::max(2.0 * nt, 250.0 + 400.0 / per_stage);
            for (int s = 1; s <= (pair ? 1 : std::min(std::min(8, max_nk), cols / 8)); ++s) {      // every CTA a k-block and a run of columns
                const long long slots = pair ? kGemmSms / 2 : cluster_slots(s);
                const double rounds = (double)((tiles + slots - 1) / slots);
                const double busy = std::min(1.0, (double)tiles / (double)slots);
                double per_kb = std::max(issue, blk / (maxM <= 256 ? 40.0 : 58.0));
                per_kb = std::max(per_kb, nt * 128.0 * (pair ? 0.5 : 1.0) / 24.0 * (maxM <= 256 ? busy : 0.0));
                const double tail = 1500.0 + 12.0 * cols;
                // the exchange: two barriers and a last round trip, and its bytes at the 12 a cycle that an SM sends to others
                const double exchange = s > 1 ? 3500.0 + a_rows * nt * 4.0 * (s - 1) / s / 12.0 : 0.0;
                const double cost = rounds * (ceil_div(max_nk, s) * per_kb + 1200.0 + exchange) + tail;
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
    p->rep = 1;
    *pair_out = best_pair;
    if (!gemm_number_items(p, best_pair) || !gemm_layout(p, a_mn, b_mn, best_pair, scratch_bytes)) return false;
    g_plans.keep(key, *p, best_pair);
    return true;
}

// Scoring: every row needs all columns, so nothing but the tile width and the number of tiles a CTA takes in a row is
// free.  Chosen for the fewest rounds of equal work over the SMs (a round costs its columns plus about 24 columns' worth
// of hand-over).  Where the first tile of a run is dear, a run pays for it once: 40 columns' worth, so that up to sixteen
// tiles in a row are taken as long as they do not leave SMs idle for more than that; elsewhere runs are short, which keeps
// the ranges that records stand for short.
bool gemm_plan_rows(GemmParams* p, uint32_t scratch_bytes, bool long_runs, bool* pair_out) {
    const PlanCache::Key key = PlanCache::key_of(*p, 8 | (long_runs ? 16 : 0) | (int)scratch_bytes << 5);
    if (g_plans.find(key, p, pair_out)) return true;
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
            const double cost = rounds * (c * (nt + 24.0) + (long_runs ? 40.0 : 0.5));
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
    while (p->rep > 1 && 2 * p->rep > p->NT / 16) p->rep /= 2;      // a copy without columns of its own is no use
    *pair_out = pair;
    if (!gemm_number_items(p, pair) || !gemm_layout(p, false, false, pair, scratch_bytes)) return false;
    g_plans.keep(key, *p, pair);
    return true;
}

int gemm_box_b(const GemmParams& p, bool b_mn, bool pair) { return b_mn ? 64 : (pair || p.dual) ? p.NT / 2 : p.NT; }

vt_status gemm_store(const GemmMaps& maps, const GemmParams& p, bool pair, bool a_mn, bool b_mn, void* const* out, cudaStream_t st) {
    EpiStore::Params ep{};
    for (int i = 0; i < p.n_prob; ++i) ep.out[i] = reinterpret_cast<uint16_t*>(out[i]);
    if (!a_mn && !b_mn) return gemm_launch<false, false, EpiStore>(maps, p, pair, ep, st);
    if (!a_mn) return gemm_launch<false, true, EpiStore>(maps, p, pair, ep, st);
    return gemm_launch<true, true, EpiStore>(maps, p, pair, ep, st);
}

static thread_local int g_withheld_us = 0;
int gemm_withheld_us() { return g_withheld_us; }

static thread_local struct {
    int n, row[16][5];
} g_noted{};
void gemm_note(bool pair, int NT, int splits, int items, int at_once) {
    if (g_noted.n == 16) return;
    int* r = g_noted.row[g_noted.n++];
    r[0] = pair;
    r[1] = NT;
    r[2] = splits;
    r[3] = items;
    r[4] = at_once;
}

}  // namespace vt

extern "C" vt_status vt_test_withhold_copies(int limit_us) {
    if (limit_us < 0 || limit_us > 100000) return VT_ERR_SHAPE;
    vt::g_withheld_us = limit_us;
    return VT_OK;
}

extern "C" int vt_test_products(int* out, int max) {
    const int n = std::min(vt::g_noted.n, std::max(max, 0));
    if (out) memcpy(out, vt::g_noted.row, (size_t)n * sizeof(vt::g_noted.row[0]));
    vt::g_noted.n = 0;
    return out ? n : 0;
}
