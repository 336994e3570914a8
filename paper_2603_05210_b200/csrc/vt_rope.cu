// Rotary positions: the table of frequencies, the turn itself (forward and back), and the write into a paged cache.
//
// y = a R(position * w_i) x on pairs of a head's elements.  What the angle needs is position * w_i without its whole turns.  With w_i in
// turns per position, as a fraction of 2^64, the product modulo 2^64 is just that, exactly: one 64-bit multiplication, no reduction of
// a large argument, and the table's rounding (2^-53 of w_i) is all that far positions multiply.  The top 32 bits, as a float in
// half turns, go to sincospif.
//
// Bound: bytes, each element read and written once.  A pair's sine and cosine are the same in all heads, so a block takes a token, computes
// each of its angles once into shared memory and goes over the heads, 16 elements (two 16-byte chunks) per thread and turn: 8 pairs whichever
// way they lie.  Each thread computing its own angles instead would cost as many cycles as the copy (64 heads' worth of the same sines).
// A thread has one such unit on its way, the first while the angles are worked out, and sixteen small blocks fill an SM: with blocks of 256 and four
// tokens, and two units on their way after the angles, 8192 tokens took 65 us (forward and back, graph) in
// place of 60 (87 % of a copy's rate), and 4099 into a cache 21.8 in place of 19.7 (79 %; the request and the page are three loads in a row).
#include "vt_step.h"

namespace vt {

constexpr int kRopeThreads = 128;
constexpr int kRopeBlocks = 16;              // per SM

__global__ void rope_table_kernel(uint64_t* table, int rot_dim, double base, int scaling, double factor, double low, double high, double original_len) {
    grid_dependency_wait();
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= rot_dim / 2) return;
    const double pi = 3.14159265358979323846;
    const double share = 2.0 * i / rot_dim;
    double w = pow(base, -share);
    if (scaling == VT_ROPE_LINEAR) {
        w /= factor;
    } else if (scaling == VT_ROPE_BASE) {
        if (rot_dim > 2) w = pow(base * pow(factor, (double)rot_dim / (rot_dim - 2)), -share);
    } else if (scaling == VT_ROPE_WAVELENGTH) {
        const double turns = original_len * w / (2.0 * pi);
        const double s = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
        w = w * s + w / factor * (1.0 - s);
    } else if (scaling == VT_ROPE_RAMP) {
        const double per = rot_dim / (2.0 * log(base));
        const double i0 = fmax(floor(per * log(original_len / (2.0 * pi * high))), 0.0);
        const double i1 = fmin(ceil(per * log(original_len / (2.0 * pi * low))), rot_dim - 1.0);
        const double s = fmin(fmax((i - i0) / fmax(i1 - i0, 1e-3), 0.0), 1.0);
        w = w * (1.0 - s) + w / factor * s;
    }
    const double turns = w / (2.0 * pi);
    table[i] = (uint64_t)llrint((turns - floor(turns)) * 18446744073709551616.0 * 0.5) << 1;      // [0, 2^63] doubled: 2^64 is 0
}

struct RopeParams {
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out, *v_out;          // with a cache: its keys and values
    int64_t q_ld, q_hs, k_ld, k_hs, v_ld, v_hs, qo_ld, qo_hs, ko_ld, ko_hs, vo_ld, vo_hs;       // ko, vo: of a token's place in its page
    int64_t k_page, v_page, table_stride;
    const int32_t *positions, *cu, *lens, *page_table;
    const uint64_t* table;
    int N, Hq, Hkv, D, rot, B, n_pages, page_size, max_pages;
    float amplitude;
};

__device__ __forceinline__ void rope_unpack(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 rope_pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool INTERLEAVED, bool INVERSE, bool CACHE>
__global__ void __launch_bounds__(kRopeThreads, kRopeBlocks)
rope_kernel(const __grid_constant__ RopeParams p) {
    extern __shared__ float4 turned[];                   // [rot / 4]: two pairs' (cos, sin)
    __shared__ int64_t place_k, place_v;                 // where the token's keys and values go, -1: nowhere
    __shared__ int real;
    grid_dependency_wait();
    const int tid = threadIdx.x, pairs = p.rot >> 1;
    const int64_t n = blockIdx.x;
    const int per_head = p.D >> 4, rotated = p.rot >> 4;
    const int all = (p.Hq + (CACHE ? 2 : 1) * p.Hkv) * per_head, step = kRopeThreads * gridDim.y;

    struct Unit {                                        // 16 elements of a head; pairs 8 i .. 8 i + 7 lie in a row, or in 8 of either half
        uint4 u0, u1;
        int head, i;
    };
    auto load = [&](Unit& u, int e) {
        u.head = e / per_head;
        u.i = e - u.head * per_head;
        const int head = u.head;
        const uint16_t* from;
        bool rotates = u.i < rotated;
        if (head < p.Hq) {
            from = p.q + n * p.q_ld + head * p.q_hs;
        } else if (head < p.Hq + p.Hkv) {
            from = p.k + n * p.k_ld + (head - p.Hq) * p.k_hs;
        } else {
            from = p.v + n * p.v_ld + (head - p.Hq - p.Hkv) * p.v_hs;
            rotates = false;
        }
        const bool halves = !INTERLEAVED && rotates;
        const int c0 = halves ? 8 * u.i : 16 * u.i;
        u.u0 = *reinterpret_cast<const uint4*>(from + c0);
        u.u1 = *reinterpret_cast<const uint4*>(from + (halves ? c0 + pairs : c0 + 8));
    };
    // the first one is on its way while the angles are worked out
    Unit unit;
    int e = blockIdx.y * kRopeThreads + tid;
    if (e < all) load(unit, e);

    float2* cs = reinterpret_cast<float2*>(turned);
    const int64_t position = p.positions[n];
    for (int i = tid; i < pairs; i += kRopeThreads) {
        const uint64_t turn = p.table[i] * (uint64_t)position;
        const float half = (float)(int32_t)(uint32_t)(turn >> 32) * 4.656612873077393e-10f;     // 2^-31: in half turns, [-1, 1]
        float s, c;
        sincospif(half, &s, &c);
        cs[i] = make_float2(c * p.amplitude, (INVERSE ? -s : s) * p.amplitude);
    }
    if (CACHE && tid == 0) {
        const int b = request_of(p.cu, p.B, (int)n);
        int64_t pk = -1, pv = -1;
        if (b >= 0) {
            const int64_t at = (int64_t)p.lens[b] + n - first_of(p.cu, b);
            const int64_t pg = at / p.page_size;
            if (at >= 0 && pg < p.max_pages) {
                const int page = p.page_table[b * p.table_stride + pg];
                if ((unsigned)page < (unsigned)p.n_pages) {
                    pk = page * p.k_page + (at - pg * p.page_size) * p.ko_ld;
                    pv = page * p.v_page + (at - pg * p.page_size) * p.vo_ld;
                }
            }
        }
        place_k = pk;
        place_v = pv;
        real = b >= 0;
    }
    __syncthreads();
    grid_launch_dependents();

    if (CACHE && !real) return;
    auto finish = [&](Unit& u) {
        const int i = u.i;
        int head = u.head;
        bool rotates = i < rotated;
        uint16_t* to;
        if (head < p.Hq) {
            to = p.q_out + n * p.qo_ld + head * p.qo_hs;
        } else if ((head -= p.Hq) < p.Hkv) {
            if (CACHE && place_k < 0) return;
            to = p.k_out + (CACHE ? place_k : n * p.ko_ld) + head * p.ko_hs;
        } else {
            if (place_v < 0) return;
            to = p.v_out + place_v + (head - p.Hkv) * p.vo_hs;
            rotates = false;
        }
        const bool halves = !INTERLEAVED && rotates;
        const int c0 = halves ? 8 * i : 16 * i, c1 = halves ? c0 + pairs : c0 + 8;
        if (rotates) {
            float x0[8], x1[8], y0[8], y1[8];
            rope_unpack(u.u0, x0);
            rope_unpack(u.u1, x1);
            const float4* f = reinterpret_cast<const float4*>(cs + 8 * i);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const float4 g = f[m];                   // pairs 2 m and 2 m + 1
                if (INTERLEAVED) {
                    float(&x)[8] = m < 2 ? x0 : x1;
                    float(&y)[8] = m < 2 ? y0 : y1;
                    const int o = 4 * (m & 1);
                    y[o] = x[o] * g.x - x[o + 1] * g.y;
                    y[o + 1] = x[o + 1] * g.x + x[o] * g.y;
                    y[o + 2] = x[o + 2] * g.z - x[o + 3] * g.w;
                    y[o + 3] = x[o + 3] * g.z + x[o + 2] * g.w;
                } else {
                    y0[2 * m] = x0[2 * m] * g.x - x1[2 * m] * g.y;
                    y1[2 * m] = x1[2 * m] * g.x + x0[2 * m] * g.y;
                    y0[2 * m + 1] = x0[2 * m + 1] * g.z - x1[2 * m + 1] * g.w;
                    y1[2 * m + 1] = x1[2 * m + 1] * g.z + x0[2 * m + 1] * g.w;
                }
            }
            u.u0 = rope_pack(y0);
            u.u1 = rope_pack(y1);
        }
        *reinterpret_cast<uint4*>(to + c0) = u.u0;
        *reinterpret_cast<uint4*>(to + c1) = u.u1;
    };
    while (e < all) {
        finish(unit);
        e += step;
        if (e < all) load(unit, e);
    }
}

// One thread per token: up its parents, which are earlier tokens, so the way ends.
__global__ void tree_mask_kernel(const int32_t* parents, const int32_t* cu, const int32_t* lens, int N, int B, int32_t* mask, int words,
                                 int32_t* positions) {
    grid_dependency_wait();
    const int n = blockIdx.x * blockDim.x + threadIdx.x;
    if (n >= N) return;
    const int b = request_of(cu, B, n);
    if (b < 0) return;
    const int first = first_of(cu, b);
    int32_t* row = mask ? mask + (int64_t)n * words : nullptr;
    if (row)
        for (int w = 0; w < words; ++w) row[w] = 0;
    int depth = -1;
    uint32_t bits = 0u;                                   // of word `at`; the way goes down through the words
    int at = -1;
    for (int t = n - first;;) {
        ++depth;
        if (t >> 5 != at) {
            if (row && at >= 0 && at < words) row[at] = (int32_t)bits;
            at = t >> 5;
            bits = 0u;
        }
        bits |= 1u << (t & 31);
        const int up = parents[first + t];
        if (up < 0 || up >= t) break;
        t = up;
    }
    if (row && at < words) row[at] = (int32_t)bits;
    if (positions) positions[n] = depth + (lens ? lens[b] : 0);
}

// ------------------------------------------------------------------------------------------ host
static vt_status launched(cudaError_t e) {
    count_launch();
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? VT_OK : cuda_fail(e);
}

vt_status launch_rope_table(uint64_t* table, int rot_dim, double base, int scaling, double factor, double low, double high, double original_len,
                            cudaStream_t st) {
    return launched(launch_pdl(rope_table_kernel, (rot_dim / 2 + 63) / 64, 64, 0, st, table, rot_dim, base, scaling, factor, low, high, original_len));
}

vt_status launch_rope(const RopeCall& c, cudaStream_t st) {
    RopeParams p{};
    auto in = [](const vt_heads& h) { return reinterpret_cast<const uint16_t*>(h.ptr); };
    p.q = in(c.q);
    p.q_ld = c.q.token_stride;
    p.q_hs = c.q.head_stride;
    p.k = in(c.k);
    p.k_ld = c.k.token_stride;
    p.k_hs = c.k.head_stride;
    p.q_out = reinterpret_cast<uint16_t*>(c.q_out.ptr);
    p.qo_ld = c.q_out.token_stride;
    p.qo_hs = c.q_out.head_stride;
    if (c.cache) {
        const vt_cache& a = *c.cache;
        p.v = in(c.v);
        p.v_ld = c.v.token_stride;
        p.v_hs = c.v.head_stride;
        p.k_out = reinterpret_cast<uint16_t*>(a.k);
        p.ko_ld = a.k_token_stride;
        p.ko_hs = a.k_head_stride;
        p.k_page = a.k_page_stride;
        p.v_out = reinterpret_cast<uint16_t*>(a.v);
        p.vo_ld = a.v_token_stride;
        p.vo_hs = a.v_head_stride;
        p.v_page = a.v_page_stride;
        p.page_table = a.page_table;
        p.lens = a.lens;
        p.table_stride = a.table_stride;
        p.n_pages = a.n_pages;
        p.page_size = a.page_size;
        p.max_pages = a.max_pages;
        p.B = a.B;
    } else {
        p.k_out = reinterpret_cast<uint16_t*>(c.k_out.ptr);
        p.ko_ld = c.k_out.token_stride;
        p.ko_hs = c.k_out.head_stride;
    }
    p.positions = c.positions;
    p.cu = c.cu_tokens;
    p.table = c.table;
    p.N = c.N;
    p.Hq = c.Hq;
    p.Hkv = c.Hkv;
    p.D = c.D;
    p.rot = c.rot_dim;
    p.amplitude = c.amplitude;
    int sms = 0;
    if (vt_status r = device_sm_count(&sms); r != VT_OK) return r;
    // Few tokens: each on several blocks, as long as all of them run at once.
    const int units = (c.Hq + (c.cache ? 2 : 1) * c.Hkv) * (c.D / 16);
    dim3 grid((unsigned)c.N);
    grid.y = (unsigned)std::min((units + kRopeThreads - 1) / kRopeThreads, std::max(1, kRopeBlocks * sms / c.N));
    const size_t smem = (size_t)c.rot_dim * sizeof(float);
    void (*kernel)(RopeParams) = nullptr;
    const bool il = (c.options & VT_ROPE_INTERLEAVED) != 0, inv = (c.options & VT_ROPE_INVERSE) != 0;
    if (c.cache) kernel = il ? rope_kernel<true, false, true> : rope_kernel<false, false, true>;
    else if (inv) kernel = il ? rope_kernel<true, true, false> : rope_kernel<false, true, false>;
    else kernel = il ? rope_kernel<true, false, false> : rope_kernel<false, false, false>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kRopeThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return launched(cudaLaunchKernelEx(&cfg, kernel, p));
}

vt_status launch_tree_mask(const int32_t* parents, const int32_t* cu_tokens, const int32_t* lens, int N, int B, int32_t* mask, int mask_words,
                           int32_t* positions, cudaStream_t st) {
    return launched(launch_pdl(tree_mask_kernel, (N + 127) / 128, 128, 0, st, parents, cu_tokens, lens, N, B, mask, mask_words, positions));
}

}  // namespace vt
