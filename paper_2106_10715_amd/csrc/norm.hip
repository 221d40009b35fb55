// Residual addition, root-mean-square norm and the output in e4m3 with scales, in one pass: the row stays in registers between
// the sum of its squares and its scaling.
#include "common.h"
#include "convert.h"

namespace moe {
namespace {

// ROW threads hold one row, V pieces of 16 bytes each; a block of at least 256 threads.  STREAM 1: non-temporal stores, 2: loads too.
template <bool BF16, int ROW, int V, int STREAM>
__global__ __launch_bounds__(ROW < 256 ? 256 : ROW) void add_norm_kernel(const u32x4* x, const u32x4* residual,
                                                                        const u32x4* __restrict__ weight, u32x4* sum, u32x4* y,
                                                                        uint32_t* __restrict__ q, float* __restrict__ q_scale, int T,
                                                                        int pieces, int group, float eps, float inv_d) {
    constexpr int E = BF16 ? 8 : 4;                        // elements of a piece
    constexpr int kRows = ROW < 256 ? 256 / ROW : 1;
    constexpr int kWaves = ROW / 64;
    __shared__ float part[2][kWaves > 1 ? kWaves : 1];
    const int lane = ROW < 256 ? threadIdx.x % ROW : threadIdx.x;
    const long row = static_cast<long>(blockIdx.x) * kRows + (ROW < 256 ? threadIdx.x / ROW : 0);
    if (ROW < 256 && row >= T) return;                     // (no barrier in these)
    const long at = row * pieces;
    auto widen = [](u32x4 u, float* v) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (BF16) {
                v[2 * c] = bf16_lo(u[c]);
                v[2 * c + 1] = bf16_hi(u[c]);
            } else {
                v[c] = __uint_as_float(u[c]);
            }
        }
    };
    auto narrow = [](const float* v) {
        u32x4 u;
#pragma unroll
        for (int c = 0; c < 4; ++c) u[c] = BF16 ? to_bf16x2(v[2 * c], v[2 * c + 1]) : __float_as_uint(v[c]);
        return u;
    };
    // all threads of a row get the sum or maximum of their values
    auto over_row = [&](float v, bool maximum, int which) {
        v = maximum ? lanes_max<64>(v) : lanes_sum<64>(v);
        if (kWaves == 1) return v;
        if (threadIdx.x % 64 == 0) part[which][threadIdx.x / 64] = v;
        __syncthreads();
        v = part[which][0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) v = maximum ? fmaxf(v, part[which][i]) : v + part[which][i];
        return v;
    };

    u32x4 xr[V], rr[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int p = lane + i * ROW;
        if (p < pieces) xr[i] = load_from<STREAM == 2>(x + at + p);
        if (p < pieces && residual != nullptr) rr[i] = load_from<STREAM == 2>(residual + at + p);
    }
    float v[V][E], squares = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int p = lane + i * ROW;
        if (p >= pieces) {
#pragma unroll
            for (int c = 0; c < E; ++c) v[i][c] = 0.f;
            continue;
        }
        widen(xr[i], v[i]);
        if (residual != nullptr) {
            float r[E];
            widen(rr[i], r);
#pragma unroll
            for (int c = 0; c < E; ++c) v[i][c] += r[c];
        }
        if (sum != nullptr) store_to<STREAM != 0>(sum + at + p, narrow(v[i]));
#pragma unroll
        for (int c = 0; c < E; ++c) squares = fmaf(v[i][c], v[i][c], squares);
    }
    const float rms = rsqrtf(over_row(squares, false, 0) * inv_d + eps);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int p = lane + i * ROW;
        if (p >= pieces) continue;
        float w[E];
        widen(weight[p], w);
#pragma unroll
        for (int c = 0; c < E; ++c) {
            v[i][c] = v[i][c] * rms * w[c];
            top = fmaxf(top, fabsf(v[i][c]));
        }
        if (y != nullptr) store_to<STREAM != 0>(y + at + p, narrow(v[i]));
    }
    if (q == nullptr) return;
    const int groups = group == 0 ? 1 : pieces * E / group;
    float scale = 0.f;
    if (group == 0) {
        scale = e4m3_scale(over_row(top, true, 1));
        if (lane == 0) q_scale[row] = scale;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int p = lane + i * ROW;
        if (group != 0) {                                  // a group is a run of group / E lanes, all inside the row or all outside
            float g = 0.f;
#pragma unroll
            for (int c = 0; c < E; ++c) g = fmaxf(g, fabsf(v[i][c]));
            for (int o = 1; o < group / E; o *= 2) g = fmaxf(g, __shfl_xor(g, o));
            scale = e4m3_scale(g);
            if (p < pieces && p % (group / E) == 0) q_scale[row * groups + p / (group / E)] = scale;
        }
        if (p >= pieces) continue;
        const OverScale over(scale);
#pragma unroll
        for (int c = 0; c < E; ++c) v[i][c] = over(v[i][c]);
        if constexpr (BF16)
            store_to<STREAM != 0>(reinterpret_cast<u32x2*>(q) + at + p, u32x2{to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3]), to_e4m3x4(v[i][4], v[i][5], v[i][6], v[i][7])});
        else
            store_to<STREAM != 0>(q + at + p, to_e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3]));
    }
}

template <bool BF16, int STREAM>
void launch(const moe_norm_cfg& c, const void* x, const void* residual, const void* weight, void* sum, void* y, void* q, float* q_scale,
            hipStream_t s) {
    const int pieces = c.d / (BF16 ? 8 : 4);
    auto run = [&](auto kernel, int row) {
        const int rows = row < 256 ? 256 / row : 1;
        hipLaunchKernelGGL(kernel, dim3((c.T + rows - 1) / rows), dim3(row < 256 ? 256 : row), 0, s, static_cast<const u32x4*>(x),
                           static_cast<const u32x4*>(residual), static_cast<const u32x4*>(weight), static_cast<u32x4*>(sum),
                           static_cast<u32x4*>(y), static_cast<uint32_t*>(q), q_scale, c.T, pieces, c.q_group, c.eps, 1.f / c.d);
    };
    // one piece per thread where a block can hold the row so (65536 x 4096: 345 us with 512 threads, 370 with 256 of two pieces; threads without a
    // piece cost nothing: as many bytes in rows of 4096, 5120, 8192, 12288 take 167, 167, 173, 170)
    if (pieces <= 64) run(add_norm_kernel<BF16, 64, 1, STREAM>, 64);
    else if (pieces <= 128) run(add_norm_kernel<BF16, 64, 2, STREAM>, 64);
    else if (pieces <= 256) run(add_norm_kernel<BF16, 256, 1, STREAM>, 256);
    else if (pieces <= 512) run(add_norm_kernel<BF16, 512, 1, STREAM>, 512);
    else if (pieces <= 1024) run(add_norm_kernel<BF16, 512, 2, STREAM>, 512);
    else if (pieces <= 2048) run(add_norm_kernel<BF16, 1024, 2, STREAM>, 1024);
    else if (pieces <= 4096) run(add_norm_kernel<BF16, 1024, 4, STREAM>, 1024);
    else if constexpr (!BF16) run(add_norm_kernel<BF16, 1024, 8, STREAM>, 1024);
}

// What is more than the caches hold does better without them, even if the next kernel reads y: us alone (and with a kernel behind it that
// reads y) through the caches / non-temporal stores / loads too, d 4096 in bf16:  2048 rows (67 MB) 10.8 (16.9) / 10.6 (18.3) / 12.8 (21.0),
// 4096 rows (134 MB) 26.1 (40.2) / 20.4 (38.0) / 23.6 (36.3), 16384 rows (537 MB) 94.2 (140.9) / 88.9 (140.7) / 86.5 (132.6).
template <bool BF16>
void launch_for_size(const moe_norm_cfg& c, const void* x, const void* residual, const void* weight, void* sum, void* y, void* q, float* q_scale,
                     hipStream_t s) {
    const size_t es = BF16 ? 2 : 4, each = static_cast<size_t>(c.T) * c.d;
    const size_t moved = each * (es * (1 + (residual != nullptr) + (sum != nullptr) + (y != nullptr)) + (q != nullptr));
    if (moved <= size_t(100) << 20) launch<BF16, 0>(c, x, residual, weight, sum, y, q, q_scale, s);
    else if (moved <= size_t(320) << 20) launch<BF16, 1>(c, x, residual, weight, sum, y, q, q_scale, s);
    else launch<BF16, 2>(c, x, residual, weight, sum, y, q, q_scale, s);
}

}  // namespace

int launch_add_norm(const moe_norm_cfg& c, const void* x, const void* residual, const void* weight, void* sum, void* y, void* q,
                    float* q_scale, hipStream_t s) {
    if (c.dtype == MOE_BF16) launch_for_size<true>(c, x, residual, weight, sum, y, q, q_scale, s);
    else launch_for_size<false>(c, x, residual, weight, sum, y, q, q_scale, s);
    MOE_LAUNCH_CHECK("add_norm_kernel");
    return MOE_OK;
}

}  // namespace moe
