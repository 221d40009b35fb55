// Attention of one new token per sequence over a paged cache of keys and values.
//
// For sequence b and query head n over key head h:  l_t = scale q_n . k_t,  out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(l_t log2 e - m),
// with a running m, one pass over the cached tokens.  Bound by reading the cache once.
//
// Both products are matrix instructions of 16 x 16 with the query heads of a key head as the 16 columns (idle columns of small groups
// cost nothing where the cache's rows are what has to be waited for):
//   S^T[token, head] = K Q^T   a lane's operands are 16-byte pieces of a row of K as they lie in memory,
//   O^T[dim, head] += V^T P^T  a lane's sums S are, of its head, the four tokens of its quarter of the wave: with two runs of 16 tokens it
//                              holds eight of 32 tokens, just what this product wants of P^T in that lane, if V^T is given with its
//                              tokens in the same order.  It is: a lane loads its pieces of those eight rows of V and swaps the
//                              16-bit halves of pairs of rows.
// So neither K, V nor P passes through the LDS.
//
// The work is the list of all (sequence, key head, run of 128 tokens); every block takes an equal stretch of it, found from the lengths on
// the device, whatever they are.  A sequence's head that lies in several blocks' stretches is left by each as an unscaled sum with its
// maximum and its weight, and joined by a second kernel in the order of the tokens.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "convert.h"

namespace moe {
namespace {

constexpr int kUnit = 128;          // tokens a block takes in one step: 32 per wave
constexpr float kSlack = 8.f;       // the running maximum is raised only where a logit passes it by more than this (as a power of two)

struct Attn {
    const void* q;
    long q_stride;
    const char *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *table, *lens;
    void* out;
    float* lse;
    float *part_o, *part_ml;        // [workers][2][heads of an item][dim], [workers][2][heads of an item][2]
    int B, heads, group, chunks, dim, pages, page_bits, table_pages, window;
    float scale;                    // times log2 e
};

// The tokens [first, end) sequence b attends to, and `base`, `first` rounded down to a run of 16 (which lies in one page).
struct Span {
    int first, end, base, units;
};
__device__ inline Span span_of(const Attn& a, int b) {
    Span s;
    s.end = min(max(a.lens[b], 0), a.table_pages << a.page_bits);
    s.first = a.window > 0 ? max(0, s.end - a.window) : 0;
    s.base = s.first & ~15;
    s.units = (s.end - s.base + kUnit - 1) / kUnit;
    return s;
}

// Stretch `i` of `n` things cut into `w` stretches as even as can be, and the stretch thing r lies in.
__device__ inline long cut_at(long n, int w, int i) {
    const long q = n / w, rest = n - q * w;
    return i * q + min(static_cast<long>(i), rest);
}
__device__ inline int cut_of(long n, int w, long r) {
    const long q = n / w, rest = n - q * w;
    return static_cast<int>(r < rest * (q + 1) ? r / (q + 1) : rest + (r - rest * (q + 1)) / q);
}

// How a cache type and the arithmetic that goes with the activations' type lie in the lanes.
template <bool F32, int CACHE, int DIM>
struct Layout {
    static constexpr int kWidth = CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1;
    static constexpr int kPiece = 16 / kWidth;                 // elements of a 16-byte piece of K
    static constexpr int kPieces = DIM / (4 * kPiece);         // pieces of a row per lane: lane quarter g holds piece 4 i + g
    static constexpr int kHalves = DIM > 128 ? 2 : 1;          // V: a row is read in runs of up to 128 elements
    static constexpr int kOwn = DIM > 128 ? 8 : DIM / 16;      // of which each of 16 lanes holds this many
};

template <int BYTES>
struct Raw;
template <> struct Raw<4> { uint32_t w[1]; };
template <> struct Raw<8> { uint32_t w[2]; };
template <> struct Raw<16> { uint32_t w[4]; };
template <> struct Raw<32> { uint32_t w[8]; };
template <int BYTES>
__device__ inline Raw<BYTES> load_raw(const char* p) {
    Raw<BYTES> r;
    if constexpr (BYTES == 4) r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (BYTES == 8) { const u32x2 u = *reinterpret_cast<const u32x2*>(p); r.w[0] = u[0]; r.w[1] = u[1]; }
    if constexpr (BYTES >= 16)
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u32x4 u = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
            for (int c = 0; c < 4; ++c) r.w[4 * i + c] = u[c];
        }
    return r;
}

// N elements of a cache type as N / 2 pairs of bf16 (e4m3 values are bf16 values), and as floats.
template <int CACHE, int N>
__device__ inline void to_pairs(const uint32_t* w, uint32_t* out) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if constexpr (CACHE == MOE_BF16) out[i] = w[i];
        else if (i % 2 == 0) out[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i / 2], 1.f, false));
        else out[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i / 2], 1.f, true));
    }
}
template <int CACHE, int N>
__device__ inline void to_floats(const uint32_t* w, float* out) {
    if constexpr (CACHE == MOE_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = __uint_as_float(w[i]);
    } else if constexpr (CACHE == MOE_BF16) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { out[2 * i] = bf16_lo(w[i]); out[2 * i + 1] = bf16_hi(w[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            float f[4];
            from_e4m3x4(w[i], f);
#pragma unroll
            for (int c = 0; c < 4; ++c) out[4 * i + c] = f[c];
        }
    }
}

// Over the four lanes that hold the same head.
__device__ inline float quarters_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float quarters_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// One wave's attention of 16 * NT query heads over some of an item's tokens.
template <bool F32, int CACHE, int DIM, int NT>
struct Wave {
    using L = Layout<F32, CACHE, DIM>;
    static constexpr int kSteps = L::kPiece / 8;                                    // bf16: matrix instructions of one piece of K
    float q32[F32 ? NT : 1][F32 ? L::kPieces : 1][F32 ? L::kPiece : 1];             // Q^T, fp32 or bf16
    bf16x8 q16[F32 ? 1 : NT][F32 ? 1 : L::kPieces][F32 ? 1 : kSteps];
    f32x4 o[NT][L::kHalves][L::kOwn];                                               // O^T: dim 128 half + own (4 g + r) + j, head l % 16
    float m[NT], l[NT];                                                             // maximum (the same in all quarters), weight of the own tokens

    // the query heads [head0, head0 + n_heads) of sequence b
    __device__ void start(const Attn& a, int b, int head0, int n_heads, int lane) {
        const int n = lane % 16, g = lane / 16;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -INFINITY;
            l[t] = 0.f;
#pragma unroll
            for (int h = 0; h < L::kHalves; ++h)
#pragma unroll
                for (int j = 0; j < L::kOwn; ++j) o[t][h][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            const bool there = 16 * t + n < n_heads;
            const long row = b * a.q_stride + static_cast<long>(head0 + 16 * t + n) * a.dim;
#pragma unroll
            for (int i = 0; i < L::kPieces; ++i) {
                const int d0 = (4 * i + g) * L::kPiece;
                const bool in = there && d0 < a.dim;
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < L::kPiece; c += 4) {
                        f32x4 u = {0.f, 0.f, 0.f, 0.f};
                        if (in) u = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + row + d0 + c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) q32[t][i][c + e] = u[e];
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        u32x4 u = {0, 0, 0, 0};
                        if (in) u = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + row + d0 + 8 * s);
                        q16[t][i][s] = __builtin_bit_cast(bf16x8, u);
                    }
                }
            }
        }
    }

    // Tokens [t0, t0 + 32) of sequence b and key head h, t0 a multiple of 16; those outside of the span weigh nothing.
    __device__ void step(const Attn& a, const Span& span, int b, int h, int t0, int lane) {
        const int n = lane % 16, g = lane / 16;
        constexpr int kRowBytes = L::kOwn * L::kWidth;
        Raw<16> k[2][L::kPieces];
        Raw<kRowBytes> v[2][4][L::kHalves];
        f32x4 ks[2], vs[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = min(t0 + 16 * r, (span.end - 1) & ~15);                // (past the end: any rows that exist)
            const int page = min(max(a.table[static_cast<long>(b) * a.table_pages + (t >> a.page_bits)], 0), a.pages - 1);
            const long at = ((static_cast<long>(page) * a.heads + h) << a.page_bits) + (t & ((1 << a.page_bits) - 1));
            const char* kr = a.k_pages + at * a.dim * L::kWidth;
            const char* vr = a.v_pages + at * a.dim * L::kWidth;
#pragma unroll
            for (int i = 0; i < L::kPieces; ++i) {
                k[r][i] = Raw<16>{};
                if ((4 * i + g) * L::kPiece < a.dim) k[r][i] = load_raw<16>(kr + (n * a.dim + (4 * i + g) * L::kPiece) * L::kWidth);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int hf = 0; hf < L::kHalves; ++hf) {
                    v[r][c][hf] = Raw<kRowBytes>{};
                    if (128 * hf + L::kOwn * n < a.dim)
                        v[r][c][hf] = load_raw<kRowBytes>(vr + ((4 * g + c) * a.dim + 128 * hf + L::kOwn * n) * L::kWidth);
                }
            if constexpr (CACHE == MOE_E4M3) {
                ks[r] = *reinterpret_cast<const f32x4*>(a.k_scales + at + 4 * g);
                vs[r] = *reinterpret_cast<const f32x4*>(a.v_scales + at + 4 * g);
            }
        }

        f32x4 s[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                s[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) {
                    if constexpr (F32) {
                        float f[L::kPiece];
                        to_floats<CACHE, L::kPiece>(k[r][i].w, f);
#pragma unroll
                        for (int c = 0; c < L::kPiece; ++c)
                            s[t][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[c], q32[t][i][c], s[t][r], 0, 0, 0);
                    } else {
                        u32x4 pairs[kSteps];
                        to_pairs<CACHE, L::kPiece>(k[r][i].w, reinterpret_cast<uint32_t*>(pairs));
#pragma unroll
                        for (int st = 0; st < kSteps; ++st)
                            s[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pairs[st]), q16[t][i][st], s[t][r], 0, 0, 0);
                    }
                }
            }

        const bool edge = t0 < span.first || t0 + 32 > span.end;
        if (edge) {                                            // rows that do not count may hold anything
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int t = t0 + 16 * r + 4 * g + c;
                    if (t >= span.first && t < span.end) continue;
#pragma unroll
                    for (int hf = 0; hf < L::kHalves; ++hf) v[r][c][hf] = Raw<kRowBytes>{};
                    if constexpr (CACHE == MOE_E4M3) vs[r][c] = 0.f;
                }
        }

        float p[NT][2][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float x = s[t][r][c] * a.scale;
                    if constexpr (CACHE == MOE_E4M3) x *= ks[r][c];
                    const int tok = t0 + 16 * r + 4 * g + c;
                    if (edge && (tok < span.first || tok >= span.end)) x = -INFINITY;
                    p[t][r][c] = x;
                    top = fmaxf(top, x);
                }
            if (__any(top > m[t] + kSlack)) {                  // (always where m is still -inf and some token counts)
                const float now = fmaxf(m[t], quarters_max(top));
                const float keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[t] - now);
                m[t] = now;
                l[t] *= keep;
#pragma unroll
                for (int hf = 0; hf < L::kHalves; ++hf)
#pragma unroll
                    for (int j = 0; j < L::kOwn; ++j) o[t][hf][j] *= keep;
            }
            const float ref = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float e = __builtin_amdgcn_exp2f(p[t][r][c] - ref);
                    l[t] += e;
                    if constexpr (CACHE == MOE_E4M3) p[t][r][c] = e * vs[r][c];
                    else p[t][r][c] = e;
                }
        }

        if constexpr (F32) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int hf = 0; hf < L::kHalves; ++hf) {
                        float f[L::kOwn];
                        to_floats<CACHE, L::kOwn>(v[r][c][hf].w, f);
#pragma unroll
                        for (int j = 0; j < L::kOwn; ++j)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
                                o[t][hf][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j], p[t][r][c], o[t][hf][j], 0, 0, 0);
                    }
        } else {
            bf16x8 pp[NT];                                     // weights of at most 2^8, rounded to 8 bits for the matrix instruction
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                u32x4 u;
#pragma unroll
                for (int c = 0; c < 4; ++c) u[c] = to_bf16x2(p[t][c / 2][2 * (c % 2)], p[t][c / 2][2 * (c % 2) + 1]);
                pp[t] = __builtin_bit_cast(bf16x8, u);
            }
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf) {
                uint32_t pairs[8][L::kOwn / 2];
#pragma unroll
                for (int c = 0; c < 8; ++c) to_pairs<CACHE, L::kOwn>(v[c / 4][c % 4][hf].w, pairs[c]);
#pragma unroll
                for (int j = 0; j < L::kOwn; ++j) {
                    u32x4 u;                                   // dim j of the eight tokens
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        u[c] = __builtin_amdgcn_perm(pairs[2 * c + 1][j / 2], pairs[2 * c][j / 2], j % 2 == 0 ? 0x05040100u : 0x07060302u);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        o[t][hf][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), pp[t], o[t][hf][j], 0, 0, 0);
                }
            }
        }
    }
};

// Heads of a work item and the LDS the waves' sums are joined in.
template <int DIM, int NT>
struct Join {
    static constexpr int kCols = DIM > 128 ? 128 : DIM;
    float o[4][16][kCols + 4];
    float m[4][16 * NT], l[4][16 * NT];
};

template <bool F32>
__device__ inline void store_out(const Attn& a, long at, float v) {
    if constexpr (F32) static_cast<float*>(a.out)[at] = v;
    else static_cast<__bf16*>(a.out)[at] = static_cast<__bf16>(v);
}

template <bool F32, int CACHE, int DIM, int NT>
__global__ __launch_bounds__(256, 2) void attn_kernel(Attn a) {
    using L = Layout<F32, CACHE, DIM>;
    using J = Join<DIM, NT>;
    constexpr int kHeads = 16 * NT;
    extern __shared__ char lds[];
    J& join = *reinterpret_cast<J*>(lds);
    int* before = reinterpret_cast<int*>(lds + sizeof(J));            // [B + 1] units of the sequences before
    __shared__ int wave_total[4];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);

    {                                                                 // the running sum of the sequences' units
        const int per = (a.B + 255) / 256;
        int own = 0;
        for (int i = 0; i < per; ++i)
            if (tid * per + i < a.B) own += span_of(a, tid * per + i).units;
        int incl = own;
        for (int o = 1; o < 64; o *= 2) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 63) wave_total[wave] = incl;
        __syncthreads();
        int at = incl - own;
        for (int w = 0; w < wave; ++w) at += wave_total[w];
        for (int i = 0; i < per; ++i)
            if (tid * per + i < a.B) {
                before[tid * per + i] = at;
                at += span_of(a, tid * per + i).units;
            }
        if (tid == 255) before[a.B] = at;                             // (all of the later threads' sums are empty)
        __syncthreads();
    }
    const int per_unit = a.heads * a.chunks;                          // items of a sequence
    const int q_heads = a.heads * a.group;

    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {               // sequences without tokens
        if (before[b + 1] != before[b]) continue;
        for (int i = tid; i < q_heads * a.dim; i += 256) store_out<F32>(a, static_cast<long>(b) * q_heads * a.dim + i, 0.f);
        for (int i = tid; i < q_heads && a.lse != nullptr; i += 256) a.lse[static_cast<long>(b) * q_heads + i] = -INFINITY;
    }

    const long total = static_cast<long>(before[a.B]) * per_unit;
    long at = cut_at(total, gridDim.x, blockIdx.x);
    const long stop = cut_at(total, gridDim.x, blockIdx.x + 1);
    if (at >= stop) return;
    int b = 0;                                                        // the last sequence that starts at or before `at`
    for (int step = 4096; step > 0; step /= 2)
        if (b + step < a.B && static_cast<long>(before[b + step]) * per_unit <= at) b += step;
    bool first_item = true;
    while (at < stop) {
        while (static_cast<long>(before[b + 1]) * per_unit <= at) ++b;
        const Span span = span_of(a, b);
        const long in_b = at - static_cast<long>(before[b]) * per_unit;
        const int item = static_cast<int>(in_b / span.units), u0 = static_cast<int>(in_b - static_cast<long>(item) * span.units);
        const int u1 = static_cast<int>(min(static_cast<long>(span.units), u0 + (stop - at)));
        const int h = item / a.chunks, chunk = item - h * a.chunks;
        const int head0 = h * a.group + chunk * kHeads, n_heads = min(kHeads, a.group - chunk * kHeads);

        Wave<F32, CACHE, DIM, NT> w;
        w.start(a, b, head0, n_heads, lane);
        for (int u = u0; u < u1; ++u) {
            const int t0 = span.base + u * kUnit + 32 * wave;
            if (t0 < span.end) w.step(a, span, b, h, t0, lane);
        }

        // the four waves' sums of each head, by the largest of their maxima
        const int n = lane % 16, g = lane / 16;
        float factor[NT], top[NT], weight[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float l = quarters_sum(w.l[t]);
            if (g == 0) {
                join.m[wave][16 * t + n] = w.m[t];
                join.l[wave][16 * t + n] = l;
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            top[t] = fmaxf(fmaxf(join.m[0][16 * t + n], join.m[1][16 * t + n]), fmaxf(join.m[2][16 * t + n], join.m[3][16 * t + n]));
            const float ref = top[t] == -INFINITY ? 0.f : top[t];
            weight[t] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) weight[t] = fmaf(join.l[i][16 * t + n], __builtin_amdgcn_exp2f(join.m[i][16 * t + n] - ref), weight[t]);
            factor[t] = __builtin_amdgcn_exp2f(w.m[t] - ref);
        }
        const bool whole = u0 == 0 && u1 == span.units;
        const long slot = (2L * blockIdx.x + (first_item ? 0 : 1)) * kHeads;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (whole) {
                factor[t] /= weight[t];
                if (wave == 0 && g == 0 && 16 * t + n < n_heads && a.lse != nullptr)
                    a.lse[static_cast<long>(b) * q_heads + head0 + 16 * t + n] = (top[t] + __builtin_amdgcn_logf(weight[t])) * 0.6931471805599453f;
            } else if (wave == 0 && g == 0) {
                a.part_ml[(slot + 16 * t + n) * 2] = top[t];
                a.part_ml[(slot + 16 * t + n) * 2 + 1] = weight[t];
            }
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf) {
                if (t + hf > 0) __syncthreads();
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < L::kOwn; ++j) join.o[wave][n][L::kOwn * (4 * g + r) + j] = w.o[t][hf][j][r] * factor[t];
                __syncthreads();
                const int rows = min(16, n_heads - 16 * t), cols = min(J::kCols, a.dim - 128 * hf);
                for (int i = tid; i < rows * J::kCols; i += 256) {
                    const int row = i / J::kCols, col = i % J::kCols;
                    if (col >= cols) continue;
                    const float v = (join.o[0][row][col] + join.o[1][row][col]) + (join.o[2][row][col] + join.o[3][row][col]);
                    if (whole) store_out<F32>(a, (static_cast<long>(b) * q_heads + head0 + 16 * t + row) * a.dim + 128 * hf + col, v);
                    else a.part_o[(slot + 16 * t + row) * a.dim + 128 * hf + col] = v;
                }
            }
        }
        __syncthreads();
        at += u1 - u0;
        first_item = false;
    }
}

// Joins the parts of the items that lie in several blocks' stretches: one block for each sequence and query head.
template <bool F32>
__global__ __launch_bounds__(256) void attn_join_kernel(Attn a, int workers, int item_heads) {
    __shared__ int sums[4];
    __shared__ float parts[256];
    const int tid = threadIdx.x;
    const int q_heads = a.heads * a.group;
    const int b = blockIdx.x / q_heads, head = blockIdx.x - b * q_heads;
    const int h = head / a.group, chunk = (head - h * a.group) / item_heads, row = head - h * a.group - chunk * item_heads;
    int mine = 0, all = 0;
    for (int i = tid; i < a.B; i += 256) {
        const int u = span_of(a, i).units;
        all += u;
        if (i < b) mine += u;
    }
    auto over_block = [&](int v) {
        for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
        __syncthreads();
        if (tid % 64 == 0) sums[tid / 64] = v;
        __syncthreads();
        return sums[0] + sums[1] + sums[2] + sums[3];
    };
    const long per_unit = static_cast<long>(a.heads) * a.chunks;
    const long start = over_block(mine) * per_unit, total = over_block(all) * per_unit;
    const int units = span_of(a, b).units;
    if (units == 0) return;
    const long r0 = start + static_cast<long>(h * a.chunks + chunk) * units;
    const int w0 = cut_of(total, workers, r0), w1 = cut_of(total, workers, r0 + units - 1);
    if (w0 == w1) return;                                             // one block had it all
    const int first_slot = cut_at(total, workers, w0) == r0 ? 0 : 1;
    auto slot_of = [&](int w) { return (2L * w + (w == w0 ? first_slot : 0)) * item_heads + row; };

    float top = -INFINITY;
    for (int w = w0 + tid; w <= w1; w += 256) top = fmaxf(top, a.part_ml[slot_of(w) * 2]);
    top = lanes_max<64>(top);
    if (tid % 64 == 0) parts[tid / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
    const float ref = top == -INFINITY ? 0.f : top;
    float weight = 0.f;
    __syncthreads();
    for (int w = w0 + tid; w <= w1; w += 256) weight = fmaf(a.part_ml[slot_of(w) * 2 + 1], __builtin_amdgcn_exp2f(a.part_ml[slot_of(w) * 2] - ref), weight);
    weight = lanes_sum<64>(weight);
    if (tid % 64 == 0) parts[tid / 64] = weight;
    __syncthreads();
    weight = (parts[0] + parts[1]) + (parts[2] + parts[3]);
    if (tid == 0 && a.lse != nullptr) a.lse[static_cast<long>(b) * q_heads + head] = (top + __builtin_amdgcn_logf(weight)) * 0.6931471805599453f;

    // columns of 64, four rows of threads over the parts
    for (int c0 = 0; c0 < a.dim; c0 += 64) {
        const int col = c0 + tid % 64;
        float v = 0.f;
        if (col < a.dim)
            for (int w = w0 + tid / 64; w <= w1; w += 4)
                v = fmaf(a.part_o[slot_of(w) * a.dim + col], __builtin_amdgcn_exp2f(a.part_ml[slot_of(w) * 2] - ref), v);
        __syncthreads();
        parts[tid] = v;
        __syncthreads();
        if (tid < 64 && col < a.dim)
            store_out<F32>(a, (static_cast<long>(b) * q_heads + head) * a.dim + col,
                           ((parts[tid] + parts[tid + 64]) + (parts[tid + 128] + parts[tid + 192])) / weight);
    }
}

constexpr int kMaxWorkers = 1024;

int item_heads_of(const moe_kv_cfg& kv, const moe_attn_cfg& c) { return c.q_heads / kv.heads <= 16 ? 16 : 32; }

template <bool F32, int CACHE, int DIM, int NT>
int launch(const moe_kv_cfg& kv, const Attn& a, hipStream_t s) {
    int dev = 0;
    const DeviceInfo* info = nullptr;
    if (int rc = device_info(&dev, &info)) return rc;
    const long longest = a.window > 0 ? std::min(static_cast<long>(a.table_pages) << a.page_bits, a.window + 15L) : static_cast<long>(a.table_pages) << a.page_bits;
    const long units = (longest + kUnit - 1) / kUnit;
    const long all = units * a.B * a.heads * a.chunks;
    const int workers = static_cast<int>(std::min(std::min(all, static_cast<long>(kMaxWorkers)), 4L * info->compute_units));
    const size_t lds = sizeof(Join<DIM, NT>) + sizeof(int) * (a.B + 1);
    hipLaunchKernelGGL((attn_kernel<F32, CACHE, DIM, NT>), dim3(workers), dim3(256), lds, s, a);
    MOE_LAUNCH_CHECK("attn_kernel");
    if (units > 1) {
        hipLaunchKernelGGL((attn_join_kernel<F32>), dim3(a.B * a.heads * a.group), dim3(256), 0, s, a, workers, 16 * NT);
        MOE_LAUNCH_CHECK("attn_join_kernel");
    }
    return MOE_OK;
}

template <bool F32, int CACHE>
int for_sizes(const moe_kv_cfg& kv, const Attn& a, hipStream_t s) {
    const bool two = a.group > 16;
    if (a.dim <= 64) return two ? launch<F32, CACHE, 64, 2>(kv, a, s) : launch<F32, CACHE, 64, 1>(kv, a, s);
    if (a.dim <= 128) return two ? launch<F32, CACHE, 128, 2>(kv, a, s) : launch<F32, CACHE, 128, 1>(kv, a, s);
    return two ? launch<F32, CACHE, 256, 2>(kv, a, s) : launch<F32, CACHE, 256, 1>(kv, a, s);
}

}  // namespace

size_t attn_workspace_bytes(const moe_kv_cfg& kv, const moe_attn_cfg& c) {
    const size_t rows = 2 * static_cast<size_t>(kMaxWorkers) * item_heads_of(kv, c);
    return align256(rows * kv.head_dim * 4) + align256(rows * 8);
}

int launch_attn_decode(const moe_kv_cfg& kv, const moe_attn_cfg& c, const void* q, long q_stride, const void* k_pages, const void* v_pages,
                       const float* k_scales, const float* v_scales, const int32_t* table, const int32_t* lens, void* out, float* lse,
                       void* ws, hipStream_t s) {
    Attn a;
    a.q = q;
    a.q_stride = q_stride;
    a.k_pages = static_cast<const char*>(k_pages);
    a.v_pages = static_cast<const char*>(v_pages);
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.table = table;
    a.lens = lens;
    a.out = out;
    a.lse = lse;
    a.B = c.B;
    a.heads = kv.heads;
    a.group = c.q_heads / kv.heads;
    const int item_heads = item_heads_of(kv, c);
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(2 * static_cast<size_t>(kMaxWorkers) * item_heads * kv.head_dim * 4));
    a.chunks = (a.group + item_heads - 1) / item_heads;
    a.dim = kv.head_dim;
    a.pages = kv.pages;
    a.page_bits = __builtin_ctz(kv.page_size);
    a.table_pages = c.table_pages;
    a.window = c.window;
    a.scale = (c.scale > 0.f ? c.scale : 1.f / sqrtf(static_cast<float>(kv.head_dim))) * 1.4426950408889634f;
    if (kv.dtype == MOE_BF16) return kv.cache_dtype == MOE_BF16 ? for_sizes<false, MOE_BF16>(kv, a, s) : for_sizes<false, MOE_E4M3>(kv, a, s);
    if (kv.cache_dtype == MOE_F32) return for_sizes<true, MOE_F32>(kv, a, s);
    return kv.cache_dtype == MOE_BF16 ? for_sizes<true, MOE_BF16>(kv, a, s) : for_sizes<true, MOE_E4M3>(kv, a, s);
}

}  // namespace moe
