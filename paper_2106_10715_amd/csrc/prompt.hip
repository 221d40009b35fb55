// Attention of many new tokens per sequence over a paged cache of keys and values.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "convert.h"
#include "scores.h"

namespace moe {
namespace {

struct Prompt {
    const void* q;
    long q_stride;
    const char *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *table, *lens, *starts, *first, *end;
    void* out;
    float* lse;
    int tokens, B, heads, group, dim, pages, page_bits, table_pages, window;
    float scale;                            // times log2 e
    ScoreArgs scores;
};

template <int CACHE>
__device__ inline float cached(const char* row, int i) {
    if constexpr (CACHE == MOE_F32) return reinterpret_cast<const float*>(row)[i];
    else if constexpr (CACHE == MOE_BF16) return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[i]) << 16);
    else return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(static_cast<unsigned char>(row[i])), 0);
}

// A wave for each (token, query head): a lane for each of 64 keys, then for each four columns of the values.
template <bool F32, int CACHE>
__global__ __launch_bounds__(64) void prompt_kernel(Prompt a) {
    constexpr int kWidth = CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1;
    const int lane = threadIdx.x, token = blockIdx.x, head = blockIdx.y, kv = head / a.group;
    int lo = 0, hi = a.B;                   // the sequence: the last that begins at or before the token
    auto start = [&](int b) { return min(max(a.starts[b], 0), a.tokens); };
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (start(mid) <= token) lo = mid;
        else hi = mid;
    }
    if (token < start(lo) || token >= start(lo + 1)) return;
    const int b = lo, len = min(max(a.lens[b], 0), a.table_pages << a.page_bits), place = len - start(b + 1) + token;
    int from = a.first != nullptr ? max(a.first[token], 0) : 0, to = min(a.end != nullptr ? a.end[token] : place + 1, len);
    if (a.window > 0) from = max(from, place - a.window + 1);
    __shared__ float q[256], weights[64];
    __shared__ long rows[64];
    for (int i = lane; i < a.dim; i += 64) {
        const long at = token * a.q_stride + head * a.dim + i;
        q[i] = F32 ? static_cast<const float*>(a.q)[at] : static_cast<float>(static_cast<const __bf16*>(a.q)[at]);
    }
    __syncthreads();
    HeadScores<true> hs;
    hs.load(a.scores, head);
    float m = -INFINITY, l = 0.f, o[4] = {};
    for (int t0 = from; t0 < to; t0 += 64) {
        const int t = t0 + lane, page = t < to ? min(max(a.table[static_cast<long>(b) * a.table_pages + (t >> a.page_bits)], 0), a.pages - 1) : 0;
        const long row = ((static_cast<long>(page) * a.heads + kv) << a.page_bits) + (t & ((1 << a.page_bits) - 1));
        float x[1] = {0.f};
        if (t < to) {
            for (int i = 0; i < a.dim; ++i) x[0] = fmaf(cached<CACHE>(a.k_pages + row * a.dim * kWidth, i), q[i], x[0]);
            if constexpr (CACHE == MOE_E4M3) x[0] *= a.k_scales[row];
        }
        x[0] *= a.scale;
        if (a.scores.cap > 0.f) cap_scores(a.scores, x);
        if (a.scores.slopes != nullptr) x[0] = fmaf(-hs.slope, fabsf(static_cast<float>(place - t)), x[0]);
        if (a.scores.bias != nullptr) x[0] += hs.bias(a.scores, place - t, true);
        if (t >= to) x[0] = -INFINITY;
        const float now = fmaxf(m, lanes_max<64>(x[0])), ref = now == -INFINITY ? 0.f : now, keep = __builtin_amdgcn_exp2f(m - ref);
        const float p = __builtin_amdgcn_exp2f(x[0] - ref);
        m = now;
        l = l * keep + lanes_sum<64>(p);
        __syncthreads();
        weights[lane] = CACHE == MOE_E4M3 && t < to ? p * a.v_scales[row] : p;
        rows[lane] = row;
        __syncthreads();
        for (int c = 0; c < 4; ++c) o[c] *= keep;
        for (int j = 0; j < min(64, to - t0); ++j)
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < a.dim) o[c] = fmaf(weights[j], cached<CACHE>(a.v_pages + rows[j] * a.dim * kWidth, lane + 64 * c), o[c]);
    }
    const long at = static_cast<long>(token) * a.heads * a.group + head;
    for (int c = 0; c < 4; ++c) {
        const float v = l == 0.f ? 0.f : o[c] / l;
        if (lane + 64 * c >= a.dim) continue;
        if constexpr (F32) static_cast<float*>(a.out)[at * a.dim + lane + 64 * c] = v;
        else static_cast<__bf16*>(a.out)[at * a.dim + lane + 64 * c] = static_cast<__bf16>(v);
    }
    if (lane == 0 && a.lse != nullptr) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <bool F32, int CACHE>
int launch(const Prompt& a, hipStream_t s) {
    hipLaunchKernelGGL((prompt_kernel<F32, CACHE>), dim3(a.tokens, a.heads * a.group), dim3(64), 0, s, a);
    MOE_LAUNCH_CHECK("prompt_kernel");
    return MOE_OK;
}

}  // namespace

size_t attn_prompt_workspace_bytes(const moe_kv_cfg& kv, const moe_prompt_cfg& c) { return 256; }

int launch_attn_prompt(const moe_kv_cfg& kv, const moe_prompt_cfg& c, const Scores& scores, const void* q, long q_stride, const void* k_pages,
                       const void* v_pages, const float* k_scales, const float* v_scales, const int32_t* table, const int32_t* lens,
                       const int32_t* starts, const int32_t* first, const int32_t* end, void* out, float* lse, void* ws, hipStream_t s) {
    Prompt a;
    a.q = q;
    a.q_stride = q_stride;
    a.k_pages = static_cast<const char*>(k_pages);
    a.v_pages = static_cast<const char*>(v_pages);
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.table = table;
    a.lens = lens;
    a.starts = starts;
    a.first = first;
    a.end = end;
    a.out = out;
    a.lse = lse;
    a.tokens = c.tokens;
    a.B = c.B;
    a.heads = kv.heads;
    a.group = c.q_heads / kv.heads;
    a.dim = kv.head_dim;
    a.pages = kv.pages;
    a.page_bits = __builtin_ctz(kv.page_size);
    a.table_pages = c.table_pages;
    a.window = c.window;
    a.scale = (c.scale > 0.f ? c.scale : 1.f / sqrtf(static_cast<float>(kv.head_dim))) * kLog2E;
    a.scores = ScoreArgs(scores);
    if (kv.dtype == MOE_BF16) return kv.cache_dtype == MOE_BF16 ? launch<false, MOE_BF16>(a, s) : launch<false, MOE_E4M3>(a, s);
    if (kv.cache_dtype == MOE_F32) return launch<true, MOE_F32>(a, s);
    return kv.cache_dtype == MOE_BF16 ? launch<true, MOE_BF16>(a, s) : launch<true, MOE_E4M3>(a, s);
}

}  // namespace moe
