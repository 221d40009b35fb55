// Rows of keys and values into the pages of a cache and back, quantised to e4m3 with a scale per row on the way.
#include "common.h"
#include "convert.h"

namespace moe {
namespace {

// Eight elements of a type as they lie in memory, and as floats.
template <int TYPE>
struct Eight;
template <>
struct Eight<MOE_BF16> {
    u32x4 u;
    __device__ void get(float (&v)[8]) const {
#pragma unroll
        for (int c = 0; c < 4; ++c) { v[2 * c] = bf16_lo(u[c]); v[2 * c + 1] = bf16_hi(u[c]); }
    }
    __device__ void set(const float (&v)[8]) {
#pragma unroll
        for (int c = 0; c < 4; ++c) u[c] = to_bf16x2(v[2 * c], v[2 * c + 1]);
    }
};
template <>
struct Eight<MOE_F32> {
    f32x4 lo, hi;
    __device__ void get(float (&v)[8]) const {
#pragma unroll
        for (int c = 0; c < 4; ++c) { v[c] = lo[c]; v[4 + c] = hi[c]; }
    }
    __device__ void set(const float (&v)[8]) {
#pragma unroll
        for (int c = 0; c < 4; ++c) { lo[c] = v[c]; hi[c] = v[4 + c]; }
    }
};
template <>
struct Eight<MOE_E4M3> {
    u32x2 u;
    __device__ void get(float (&v)[8]) const {
        float a[4], b[4];
        from_e4m3x4(u[0], a);
        from_e4m3x4(u[1], b);
#pragma unroll
        for (int c = 0; c < 4; ++c) { v[c] = a[c]; v[4 + c] = b[c]; }
    }
    __device__ void set(const float (&v)[8]) {
        u[0] = to_e4m3x4(v[0], v[1], v[2], v[3]);
        u[1] = to_e4m3x4(v[4], v[5], v[6], v[7]);
    }
};

// One side of the copy: keys or values.
struct Side {
    void* rows;         // [n, heads, dim], tokens `stride` elements apart
    long stride;
    void* pages;        // [pages, heads, page, dim]
    float* scales;      // [pages, heads, page], e4m3 only
};

template <bool STREAM, int TYPE>
__device__ inline Eight<TYPE> load_eight(const Eight<TYPE>* p) {
    Eight<TYPE> e;
    if constexpr (TYPE == MOE_F32) {
        e.lo = load_from<STREAM>(&p->lo);
        e.hi = load_from<STREAM>(&p->hi);
    } else {
        e.u = load_from<STREAM>(&p->u);
    }
    return e;
}
template <bool STREAM, int TYPE>
__device__ inline void store_eight(Eight<TYPE>* p, const Eight<TYPE>& e) {
    if constexpr (TYPE == MOE_F32) {
        store_to<STREAM>(&p->lo, e.lo);
        store_to<STREAM>(&p->hi, e.hi);
    } else {
        store_to<STREAM>(&p->u, e.u);
    }
}

// A row (token, head) is held by LANES lanes with eight elements each.  Bound by memory.  Where rows are quantised, the wait for a row's
// maximum is made worth two rows: the same lanes take its key and its value, both requested before either is used (16384 tokens of 8 x 128:
// 17.8 us, 19.8 with a block for each).  Else half of the blocks take the keys, half the values (32768 tokens of 64 x 64 read: 193 us, 204
// with both in the same lanes).  Rows go by runs of four tokens, in a run by head: a token's rows lie together in the plain array, the rows
// of tokens that follow one another in the pages (32768 tokens of 64 x 64 read: 184 us, 190 token by token; 16384 written: 90, 92.5; runs of
// 2 to 16 are within 4 % of this, of 32 up to 10 % slower).  STREAM 1: non-temporal stores, 2: loads too.
constexpr int kRun = 4;
template <int TYPE, int CACHE, int LANES, bool WRITE, int STREAM>
__global__ __launch_bounds__(256) void kv_kernel(Side k, Side v, const int32_t* __restrict__ slots, int n, int heads, int eights,
                                                 int page_bits, int n_slots) {
    constexpr int kSides = WRITE && CACHE == MOE_E4M3 ? 2 : 1;
    const int lane = threadIdx.x % LANES;
    const long total = (static_cast<long>(n) + kRun - 1) / kRun * kRun * heads, step = static_cast<long>(gridDim.x) * (256 / LANES);
    for (long row = static_cast<long>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES; row < total; row += step) {
        const long pair = row / kRun, run = pair / heads, token = run * kRun + row % kRun;
        const int head = static_cast<int>(pair - run * heads);
        if (token >= n) continue;
        const int slot = slots[token];
        const bool there = slot >= 0 && slot < n_slots;          // others are nowhere: not written, read as zeros
        if (WRITE && !there) continue;
        const long page = slot >> page_bits, in_page = slot & ((1 << page_bits) - 1);
        const long at = ((page * heads + head) << page_bits) + in_page;
        const Side* sides[2] = {kSides == 2 || blockIdx.y == 0 ? &k : &v, &v};
        Eight<TYPE>* plain[kSides];
        Eight<CACHE>* cached[kSides];
#pragma unroll
        for (int i = 0; i < kSides; ++i) {
            plain[i] = reinterpret_cast<Eight<TYPE>*>(sides[i]->rows) + (token * sides[i]->stride) / 8 + head * eights + lane;
            cached[i] = reinterpret_cast<Eight<CACHE>*>(sides[i]->pages) + at * eights + lane;
        }
        float f[kSides][8] = {}, scale[kSides];
        if constexpr (WRITE) {
            Eight<TYPE> e[kSides];
#pragma unroll
            for (int i = 0; i < kSides; ++i)
                if (lane < eights) e[i] = load_eight<STREAM == 2>(plain[i]);
#pragma unroll
            for (int i = 0; i < kSides; ++i) {
                if (lane < eights) e[i].get(f[i]);
                if constexpr (CACHE == MOE_E4M3) {
                    float top = 0.f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) top = fmaxf(top, fabsf(f[i][c]));
                    scale[i] = e4m3_scale(lanes_max<LANES>(top));
                    if (lane == 0) sides[i]->scales[at] = scale[i];
                    const OverScale over(scale[i]);
#pragma unroll
                    for (int c = 0; c < 8; ++c) f[i][c] = over(f[i][c]);
                }
                if (lane >= eights) continue;
                Eight<CACHE> out;
                out.set(f[i]);
                store_eight<STREAM != 0>(cached[i], out);
            }
        } else if (lane < eights) {
            Eight<CACHE> e[kSides];
            if (there) {
#pragma unroll
                for (int i = 0; i < kSides; ++i) {
                    e[i] = load_eight<STREAM == 2>(cached[i]);
                    scale[i] = CACHE == MOE_E4M3 ? sides[i]->scales[at] : 1.f;
                }
#pragma unroll
                for (int i = 0; i < kSides; ++i) {
                    e[i].get(f[i]);
                    if constexpr (CACHE == MOE_E4M3)
#pragma unroll
                        for (int c = 0; c < 8; ++c) f[i][c] *= scale[i];
                }
            }
#pragma unroll
            for (int i = 0; i < kSides; ++i) {
                Eight<TYPE> out;
                out.set(f[i]);
                store_eight<STREAM != 0>(plain[i], out);
            }
        }
    }
}

template <int TYPE, int CACHE, bool WRITE, int STREAM>
void launch(const moe_kv_cfg& c, int n, const Side& k, const Side& v, const int32_t* slots, hipStream_t s) {
    const int eights = c.head_dim / 8, bits = __builtin_ctz(c.page_size);
    const long rows = (static_cast<long>(n) + kRun - 1) / kRun * kRun * c.heads;
    auto run = [&](auto kernel, int lanes) {
        const long blocks = (rows + 256 / lanes - 1) / (256 / lanes), most = 1 << 20;     // one row per group of lanes, up to many millions of rows
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks < most ? blocks : most), WRITE && CACHE == MOE_E4M3 ? 1 : 2), dim3(256), 0, s, k, v, slots, n, c.heads, eights,
                           bits, c.pages << bits);
    };
    if (eights <= 8) run(kv_kernel<TYPE, CACHE, 8, WRITE, STREAM>, 8);
    else if (eights <= 16) run(kv_kernel<TYPE, CACHE, 16, WRITE, STREAM>, 16);
    else run(kv_kernel<TYPE, CACHE, 32, WRITE, STREAM>, 32);
}

// What is more than the caches hold does better without them.  us through the caches / non-temporal stores / loads too (in brackets with a
// kernel behind them that adds k and v), heads of 128, bf16:
//   writes to bf16, 16 heads:   4096 tokens (67 MB) 11.2 / 11.3 / 13.1, 8192 (134 MB) 26.3 / 20.3 / 23.4, 16384 (268 MB) 47.7 / 45.7 / 44.4
//   reads from bf16, 16 heads:  4096 12.0 (20.4) / 11.7 (22.0) / 13.5 (24.0), 8192 26.3 (43.0) / 20.7 (44.5) / 24.3 (42.8),
//                               32768 (537 MB) 93.5 (159.9) / 89.7 (157.2) / 87.6 (157.5); fp32 as large: 95.2 / 95.0 / 101.6
//   reads from e4m3, 8 heads:   4096 (25 MB) 7.2 (12.3) / 5.7 (12.2) / 7.5 (14.3), 16384 (102 MB) 26.5 (41.9) / 17.7 (43.4) / 24.2 (42.5),
//                               100000 (621 MB) 149.8 (257.9) / 138.0 (240.3) / 136.6 (239.9)
template <int TYPE, int CACHE, bool WRITE>
int launch_for_size(const moe_kv_cfg& c, int n, const Side& k, const Side& v, const int32_t* slots, hipStream_t s) {
    const size_t each = 2 * static_cast<size_t>(n) * c.heads * c.head_dim;
    const size_t moved = each * ((TYPE == MOE_F32 ? 4 : 2) + (CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1));
    constexpr bool kLoadsToo = WRITE || TYPE == MOE_BF16, kAlways = !WRITE && CACHE == MOE_E4M3;
    if (kLoadsToo && moved > size_t(WRITE ? 200 : 320) << 20) launch<TYPE, CACHE, WRITE, kLoadsToo ? 2 : 1>(c, n, k, v, slots, s);
    else if (kAlways || moved > size_t(80) << 20) launch<TYPE, CACHE, WRITE, 1>(c, n, k, v, slots, s);
    else launch<TYPE, CACHE, WRITE, kAlways ? 1 : 0>(c, n, k, v, slots, s);
    MOE_LAUNCH_CHECK("kv_kernel");
    return MOE_OK;
}

template <bool WRITE>
int for_types(const moe_kv_cfg& c, int n, const Side& k, const Side& v, const int32_t* slots, hipStream_t s) {
    if (c.dtype == MOE_BF16)
        return c.cache_dtype == MOE_BF16 ? launch_for_size<MOE_BF16, MOE_BF16, WRITE>(c, n, k, v, slots, s)
                                         : launch_for_size<MOE_BF16, MOE_E4M3, WRITE>(c, n, k, v, slots, s);
    if (c.cache_dtype == MOE_F32) return launch_for_size<MOE_F32, MOE_F32, WRITE>(c, n, k, v, slots, s);
    return c.cache_dtype == MOE_BF16 ? launch_for_size<MOE_F32, MOE_BF16, WRITE>(c, n, k, v, slots, s)
                                     : launch_for_size<MOE_F32, MOE_E4M3, WRITE>(c, n, k, v, slots, s);
}

}  // namespace

int launch_kv_write(const moe_kv_cfg& c, int n, const void* k, long k_stride, const void* v, long v_stride, const int32_t* slots,
                    void* k_pages, void* v_pages, float* k_scales, float* v_scales, hipStream_t s) {
    return for_types<true>(c, n, Side{const_cast<void*>(k), k_stride, k_pages, k_scales}, Side{const_cast<void*>(v), v_stride, v_pages, v_scales},
                           slots, s);
}

int launch_kv_read(const moe_kv_cfg& c, int n, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                   const int32_t* slots, void* k, long k_stride, void* v, long v_stride, hipStream_t s) {
    return for_types<false>(c, n, Side{k, k_stride, const_cast<void*>(k_pages), const_cast<float*>(k_scales)},
                            Side{v, v_stride, const_cast<void*>(v_pages), const_cast<float*>(v_scales)}, slots, s);
}

}  // namespace moe
