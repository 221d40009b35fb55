// Scores that are capped by a tanh or get a bias by distance, in the units of the attention kernels: logits times log2 e.
#pragma once
#include <hip/hip_runtime.h>

#include "common.h"

namespace moe {

constexpr float kLog2E = 1.4426950408889634f;

struct ScoreArgs {
    float cap = 0.f, over_cap = 0.f;        // times log2 e, and its inverse; 0: not capped
    bool fine = false;                      // whether a capped score is to be good to a few units in its own last place, not the cap's
    int back = 0, ahead = 0;
    const float *slopes = nullptr, *bias = nullptr;
    ScoreArgs() = default;
    // dtype: of the activations.  With 16 bits and caps up to 64 a score may be off by 5 units of 2^-24 of the cap, 1.9e-5: the output's rounding alone is 2^-8.
    ScoreArgs(const Scores& s, int dtype)
        : cap(s.cap * kLog2E), over_cap(s.cap > 0.f ? 1.f / (s.cap * kLog2E) : 0.f), fine(dtype == MOE_F32 || s.cap > 64.f), back(s.back), ahead(s.ahead), slopes(s.slopes), bias(s.bias) {}
};

// tanh.  Below 0.75 an odd polynomial, fitted to tanh(z) / z in z^2 for the least relative error (3.4e-9; with its roundings 1e-7): 1 - 2 / (e^2z + 1)
// alone, which is taken above it, is off by units of 1 and not of z.  Of 2^24 scores within ten caps of zero, caps from 1 to 1000, a capped score was off by at most
// 6.2 units of 2^-24 of its value with both, by 4.7 of the cap with the quotient alone.  Where that is enough it is taken for all
// (attention of 8192 tokens in documents, 16 heads of 256: 255 us with both, 205 with it alone, 167 without a cap).
__device__ inline float small_tanh(float z) {
    const float u = z * z;
    float p = 0.00172035361f;
    p = fmaf(p, u, -0.00762702851f);
    p = fmaf(p, u, 0.0214308724f);
    p = fmaf(p, u, -0.0538856313f);
    p = fmaf(p, u, 0.133325785f);
    p = fmaf(p, u, -0.333333075f);
    p = fmaf(p, u, 1.f);
    return p * z;
}
__device__ inline float large_tanh(float z) {
    const float e = __builtin_amdgcn_exp2f(z * (2.f * kLog2E));
    return 1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f);
}
constexpr float kSmall = 0.75f;

// N scores x; cap * tanh(x / cap) out.  All lanes of the wave.
template <int N>
__device__ inline void cap_scores(const ScoreArgs& a, float (&x)[N]) {
    if (!a.fine) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = a.cap * large_tanh(x[i] * a.over_cap);
        return;
    }
    bool large = false;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        z[i] = x[i] * a.over_cap;
        large |= !(fabsf(z[i]) < kSmall);
        x[i] = a.cap * small_tanh(z[i]);
    }
    if (__any(large))
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(fabsf(z[i]) < kSmall)) x[i] = a.cap * large_tanh(z[i]);
}

// Where the bias of a head for distance 0 lies, and the bias for distance d from there, times log2 e.
__device__ inline int bias_row(const ScoreArgs& a, int head) { return head * (a.back + a.ahead + 1) + a.ahead; }
__device__ inline float bias_at(const ScoreArgs& a, int row, int d) { return a.bias[row + min(max(d, -a.ahead), a.back)] * kLog2E; }

// What scores have of their query's head.
struct HeadScores {
    float slope, last, first;               // times log2 e: what a step of distance costs; the bias of far keys, before the query and after it
    __device__ void load(const ScoreArgs& a, int head) {
        const int row = bias_row(a, head);
        slope = a.slopes != nullptr ? a.slopes[head] * kLog2E : 0.f;
        last = a.bias != nullptr ? bias_at(a, row, a.back) : 0.f;
        first = a.bias != nullptr ? bias_at(a, row, -a.ahead) : 0.f;
    }
};

}  // namespace moe
