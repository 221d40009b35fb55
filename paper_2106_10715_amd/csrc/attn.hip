// Attention of one new token per sequence over a paged cache of keys and values.
//
// For sequence b and query head n over key head h:  l_t = scale q_n . k_t,  out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(l_t log2 e - m),
// with a running m, one pass over the cached tokens.  Bound by reading the cache once.
//
// Both products are matrix instructions of 16 x 16 with the query heads of a key head as the 16 columns (idle columns of small groups
// cost nothing where the cache's rows are what has to be waited for):
//   S^T[token, head] = K Q^T   rows of K come in whole runs of 16 tokens as they lie in memory and are turned to the operand's order
//                              (lane = token) through LDS that belongs to the wave alone,
//   O^T[dim, head] += V^T P^T  a lane's sums S are, of its head, the four tokens of its quarter of the wave: with two runs of 16 tokens it
//                              holds eight of 32 tokens, just what this product wants of P^T in that lane, if V^T is given with its
//                              tokens in the same order.  It is: a lane loads its pieces of those eight rows of V and swaps the
//                              16-bit halves of pairs of rows.
// So neither V nor P passes through the LDS, and no wave waits for another while it reads.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "convert.h"

namespace moe {
namespace {

constexpr int kUnit = 128;          // tokens: the grain in which the work is shared out
constexpr int kListed = 2048;       // up to so many sequences' lengths are kept in LDS (64 KB with what else is there)
constexpr float kSlack = 8.f;       // the running maximum is raised only where a logit passes it by more than this (as a power of two)

// An item of the work, a (sequence, key head), cut where a worker's stretch begins: written by that worker, for the join.
struct Cut {
    int rows;                       // its first query head's row of out and lse; -1: nothing is cut here, or not for the first time
    int first, last;                // slot of its first part, worker of its last (in between: the slots 2 w)
    int pad;
};

struct Attn {
    const void* q;
    long q_stride;
    const char *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *table, *lens;
    void* out;
    float* lse;
    float *part_o, *part_ml;        // [workers][2][group][dim], [workers][2][group][2]: unscaled sums; their maximum and weight
    Cut* cuts;                      // [workers]
    int B, heads, group, chunks, dim, pages, page_bits, table_pages, window;
    float scale;                    // times log2 e
};

// The tokens [first, end) sequence b attends to, and `base`, `first` rounded down to a run of 16 (which lies in one page).
struct Span {
    int first, end, base, units;
};
__device__ inline Span span_of(const Attn& a, int len) {
    Span s;
    s.end = min(max(len, 0), a.table_pages << a.page_bits);
    s.first = a.window > 0 ? max(0, s.end - a.window) : 0;
    s.base = s.first & ~15;
    s.units = (s.end - s.base + kUnit - 1) / kUnit;
    return s;
}

// `n` things cut into `w` stretches as even as can be: where stretch i begins, and the stretch thing r lies in.
struct Cuts {
    long q, rest;
    // n / d for n below 2^50 (a quotient of doubles is off by one at most)
    __device__ static long over(long n, long d) {
        long r = static_cast<long>(static_cast<double>(n) / static_cast<double>(d));
        if (r * d > n) --r;
        return r;
    }
    __device__ Cuts(long n, int w) : q(over(n, w)), rest(n - q * w) {}
    __device__ long at(int i) const { return i * q + min(static_cast<long>(i), rest); }
    __device__ int of(long r) const { return static_cast<int>(r < rest * (q + 1) ? over(r, q + 1) : rest + over(r - rest * (q + 1), q)); }
};

// Waves a SIMD holds of the kernels for heads of up to `dim` and one or two column tiles: what their registers come to (512 / waves), and
// how many blocks of four waves a compute unit is given.
constexpr int waves_of(bool f32, int dim, bool two) {
    if (dim <= 64) return two || f32 ? 3 : 4;
    if (dim <= 128) return two || f32 ? 2 : 3;
    return 1;
}

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// How a cache type and the arithmetic that goes with the activations' type lie in the lanes.
template <bool F32, int CACHE, int DIM>
struct Layout {
    static constexpr int kWidth = CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1;
    static constexpr int kPiece = 16 / kWidth;                 // elements of a 16-byte piece of K
    static constexpr int kPieces = DIM / (4 * kPiece);         // pieces of a row per lane: lane quarter g holds piece 4 i + g
    static constexpr int kHalves = DIM > 128 ? 2 : 1;          // V: a row is read in runs of up to 128 elements
    static constexpr int kOwn = DIM > 128 ? 8 : DIM / 16;      // of which each of 16 lanes holds this many
    static constexpr int kRun = 16 * DIM * kWidth;             // bytes of 16 rows of K
    static constexpr bool kStaged = kRun <= 8192;              // whether they pass through the LDS
};

template <int BYTES>
struct Raw;
template <> struct Raw<4> { uint32_t w[1]; };
template <> struct Raw<8> { uint32_t w[2]; };
template <> struct Raw<16> { uint32_t w[4]; };
template <> struct Raw<32> { uint32_t w[8]; };
// `bytes` bytes of the cache from an address that is the same for the whole wave.  Loads from it take a lane's 32-bit offset and a wave's
// without any arithmetic on pairs of registers, and give zeros past the end.  Non-temporal: the cache is read once.
__device__ inline __amdgpu_buffer_rsrc_t stretch_of(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}
template <int BYTES>
__device__ inline Raw<BYTES> load_raw(__amdgpu_buffer_rsrc_t from, uint32_t at, uint32_t wave_at) {
    constexpr int kNonTemporal = 2;
    Raw<BYTES> r;
    if constexpr (BYTES == 4) r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, wave_at, kNonTemporal);
    if constexpr (BYTES == 8) { const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(from, at, wave_at, kNonTemporal); r.w[0] = u[0]; r.w[1] = u[1]; }
    if constexpr (BYTES >= 16)
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(from, at + 16 * i, wave_at, kNonTemporal);
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

    uint32_t k_at[L::kPieces], k_in[L::kPieces], k_out[L::kPieces], v_at[L::kHalves];    // of this lane: bytes from a run's first row, bytes in the LDS
    int row_bytes;

    // What does not change from item to item.  Where rows are shorter than DIM, pieces past their end are taken from their last piece:
    // Q has zeros there, and columns past the end are not stored.
    __device__ void lay_out(const Attn& a, int lane) {
        const int n = lane % 16, g = lane / 16, per = a.dim / L::kPiece;
        row_bytes = a.dim * L::kWidth;
#pragma unroll
        for (int i = 0; i < L::kPieces; ++i) {
            if constexpr (!L::kStaged) {
                k_at[i] = n * row_bytes + 16 * min(4 * i + g, per - 1);
                continue;
            }
            const int at = min(64 * i + lane, 16 * per - 1), token = at / per, piece = at - token * per;
            k_at[i] = 16 * at;
            k_in[i] = 16 * (token * 4 * L::kPieces + ((piece ^ token) & (4 * L::kPieces - 1)));          // 16 tokens' pieces: in 16 different places of a row
            k_out[i] = 16 * (n * 4 * L::kPieces + ((min(4 * i + g, per - 1) ^ n) & (4 * L::kPieces - 1)));
        }
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf) v_at[hf] = 4 * g * row_bytes + min(128 * hf + L::kOwn * n, a.dim - L::kOwn) * L::kWidth;
    }

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

    // The pages of the runs of up to 32 steps from token t0 on, `stride` tokens apart: lane 2 s + r holds that of run r of step s.
    __device__ static int pages_of(const Attn& a, const Span& span, int b, int t0, int stride, int lane) {
        const int t = min(t0 + (lane / 2) * stride + 16 * (lane % 2), (span.end - 1) & ~15);        // (past the end: a run that exists)
        return min(max(a.table[static_cast<long>(b) * a.table_pages + (t >> a.page_bits)], 0), a.pages - 1);
    }

    // Tokens [t0, t0 + 32) of key head h, t0 a multiple of 16, step `at_step` of `ids`; those outside of the span weigh nothing.
    // `mine`: a run of K in LDS that no other wave touches.
    __device__ void step(char* mine, const Attn& a, const Span& span, int ids, int at_step, int h, int t0, int lane) {
        const int g = lane / 16;
        constexpr int kRowBytes = L::kOwn * L::kWidth;
        Raw<16> k[2][L::kPieces];
        Raw<kRowBytes> v[2][4][L::kHalves];
        f32x4 ks[2], vs[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = min(t0 + 16 * r, (span.end - 1) & ~15), page = __builtin_amdgcn_readlane(ids, 2 * at_step + r);
            const long at = ((static_cast<long>(page) * a.heads + h) << a.page_bits) + (t & ((1 << a.page_bits) - 1));
            const auto kr = stretch_of(a.k_pages + at * row_bytes, 16 * row_bytes), vr = stretch_of(a.v_pages + at * row_bytes, 16 * row_bytes);
#pragma unroll
            for (int i = 0; i < L::kPieces; ++i) k[r][i] = load_raw<16>(kr, k_at[i], 0);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int hf = 0; hf < L::kHalves; ++hf) v[r][c][hf] = load_raw<kRowBytes>(vr, v_at[hf], c * row_bytes);
            if constexpr (CACHE == MOE_E4M3) {
                ks[r] = __builtin_bit_cast(f32x4, load_raw<16>(stretch_of(a.k_scales + at, 64), 16 * g, 0));
                vs[r] = __builtin_bit_cast(f32x4, load_raw<16>(stretch_of(a.v_scales + at, 64), 16 * g, 0));
            }
        }
        if constexpr (L::kStaged) {
            // (A wave's LDS operations are done in their order: it needs no barrier between what it writes and reads.)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) *reinterpret_cast<u32x4*>(mine + k_in[i]) = __builtin_bit_cast(u32x4, k[r][i]);
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) k[r][i] = __builtin_bit_cast(Raw<16>, *reinterpret_cast<const u32x4*>(mine + k_out[i]));
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

// The LDS of a block: the waves' runs of K, then, where waves share an item, their sums.
template <bool F32, int CACHE, int DIM, int NT, int TEAM>
struct Lds {
    static constexpr int kCols = DIM > 128 ? 128 : DIM;
    struct Sums {
        float o[4][16][kCols + 4];
        float m[4][16 * NT], l[4][16 * NT];
    };
    using L = Layout<F32, CACHE, DIM>;
    static constexpr size_t kRun = L::kStaged ? L::kRun : 0;                             // of one wave
    static constexpr size_t kBytes = TEAM == 1 || 4 * kRun > sizeof(Sums) ? 4 * kRun : sizeof(Sums);
};

template <bool F32>
__device__ inline void store_out(const Attn& a, long at, float v) {
    if constexpr (F32) static_cast<float*>(a.out)[at] = v;
    else static_cast<__bf16*>(a.out)[at] = static_cast<__bf16>(v);
}
__device__ inline float natural_log_of_sum(float m, float weight) { return (m + __builtin_amdgcn_logf(weight)) * 0.6931471805599453f; }

// One sequence and key head, units [u0, u1): all query heads over them, 16 * NT at a time, by the TEAM waves of a worker.  Results go to out
// and lse where the units are all there are, else to part `slot`.
template <bool F32, int CACHE, int DIM, int NT, int TEAM>
__device__ void attend(const Attn& a, Wave<F32, CACHE, DIM, NT>& w, char* lds, const Span& span, int b, int h, int u0, int u1, int chunk0, int chunk1,
                       long slot, int wave, int lane) {
    using L = Layout<F32, CACHE, DIM>;
    using S = Lds<F32, CACHE, DIM, NT, TEAM>;
    constexpr int kHeads = 16 * NT, kStride = 32 * TEAM;
    char* mine = lds + wave * S::kRun;
    const int n = lane % 16, g = lane / 16, q_heads = a.heads * a.group;
    const bool whole = u0 == 0 && u1 == span.units;
    for (int chunk = chunk0; chunk < chunk1; ++chunk) {
        const int in_group = chunk * kHeads, head0 = h * a.group + in_group, n_heads = min(kHeads, a.group - in_group);
        int t0 = span.base + u0 * kUnit + (TEAM > 1 ? 32 * wave : 0);
        const int t_end = min(span.end, span.base + u1 * kUnit);
        int ids = t0 < t_end ? w.pages_of(a, span, b, t0, kStride, lane) : 0;
        w.start(a, b, head0, n_heads, lane);
        while (t0 < t_end) {
            const int steps = min(32, (t_end - t0 + kStride - 1) / kStride);
            for (int s = 0; s < steps; ++s) w.step(mine, a, span, ids, s, h, t0 + s * kStride, lane);
            t0 += steps * kStride;
            if (t0 < t_end) ids = w.pages_of(a, span, b, t0, kStride, lane);
        }

        float l[NT], top[NT], weight[NT], factor[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            l[t] = quarters_sum(w.l[t]);
            top[t] = w.m[t];
            weight[t] = l[t];
            factor[t] = 1.f;
        }
        if constexpr (TEAM > 1) {                              // the waves' sums of each head, by the largest of their maxima
            auto& sums = *reinterpret_cast<typename S::Sums*>(lds);
            __syncthreads();                                   // all waves are done with their runs of K
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (g == 0) {
                    sums.m[wave][16 * t + n] = w.m[t];
                    sums.l[wave][16 * t + n] = l[t];
                }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int c = 16 * t + n;
                top[t] = fmaxf(fmaxf(sums.m[0][c], sums.m[1][c]), fmaxf(sums.m[2][c], sums.m[3][c]));
                const float ref = top[t] == -INFINITY ? 0.f : top[t];
                weight[t] = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) weight[t] = fmaf(sums.l[i][c], __builtin_amdgcn_exp2f(sums.m[i][c] - ref), weight[t]);
                factor[t] = __builtin_amdgcn_exp2f(w.m[t] - ref);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int head = 16 * t + n;                       // of the chunk
            if (whole) factor[t] /= weight[t];
            if ((TEAM == 1 || wave == 0) && g == 0 && head < n_heads) {
                if (!whole) {
                    a.part_ml[(slot * a.group + in_group + head) * 2] = top[t];
                    a.part_ml[(slot * a.group + in_group + head) * 2 + 1] = weight[t];
                } else if (a.lse != nullptr) {
                    a.lse[static_cast<long>(b) * q_heads + head0 + head] = natural_log_of_sum(top[t], weight[t]);
                }
            }
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf) {
                const long to_out = (static_cast<long>(b) * q_heads + head0) * a.dim + 128 * hf;
                const long to_part = (slot * a.group + in_group) * a.dim + 128 * hf;
                if constexpr (TEAM == 1) {
                    if (head < n_heads)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int col = L::kOwn * (4 * g + r);
                            if (128 * hf + col >= a.dim) continue;
#pragma unroll
                            for (int j = 0; j < L::kOwn; j += 4) {
                                const float v[4] = {w.o[t][hf][j][r] * factor[t], w.o[t][hf][j + 1][r] * factor[t], w.o[t][hf][j + 2][r] * factor[t],
                                                    w.o[t][hf][j + 3][r] * factor[t]};
                                const long at = static_cast<long>(head) * a.dim + col + j;
                                if (!whole) *reinterpret_cast<f32x4*>(a.part_o + to_part + at) = f32x4{v[0], v[1], v[2], v[3]};
                                else if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to_out + at) = f32x4{v[0], v[1], v[2], v[3]};
                                else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + to_out + at) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
                            }
                        }
                } else {
                    auto& sums = *reinterpret_cast<typename S::Sums*>(lds);
                    if (t + hf > 0) __syncthreads();
                    if (head < n_heads)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int j = 0; j < L::kOwn; ++j) sums.o[wave][n][L::kOwn * (4 * g + r) + j] = w.o[t][hf][j][r] * factor[t];
                    __syncthreads();
                    const int rows = min(16, n_heads - 16 * t), cols = min(S::kCols, a.dim - 128 * hf);
                    for (int i = 64 * wave + lane; i < rows * S::kCols; i += 256) {
                        const int row = i / S::kCols, col = i % S::kCols;
                        if (col >= cols) continue;
                        const float v = (sums.o[0][row][col] + sums.o[1][row][col]) + (sums.o[2][row][col] + sums.o[3][row][col]);
                        const long at = static_cast<long>(16 * t + row) * a.dim + col;
                        if (whole) store_out<F32>(a, to_out + at, v);
                        else a.part_o[to_part + at] = v;
                    }
                }
            }
        }
        if constexpr (TEAM > 1) __syncthreads();               // the LDS is K's again
    }
}

// A sequence without tokens: this thread's share of its outputs.
template <bool F32>
__device__ inline void store_nothing(const Attn& a, int b, int head0, int n_heads, int tid) {
    const long row = static_cast<long>(b) * a.heads * a.group + head0;
    for (int i = tid; i < n_heads * a.dim; i += 256) store_out<F32>(a, row * a.dim + i, 0.f);
    for (int i = tid; i < n_heads && a.lse != nullptr; i += 256) a.lse[row + i] = -INFINITY;
}

// Short sequences: a block for each sequence, key head and 16 * NT of its query heads; nothing is split.
template <bool F32, int CACHE, int DIM, int NT>
__global__ __launch_bounds__(256, waves_of(F32, DIM, NT == 2)) void attn_short_kernel(Attn a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    const int item = blockIdx.x / a.chunks, chunk = blockIdx.x - item * a.chunks, b = item / a.heads, h = item - b * a.heads;
    Wave<F32, CACHE, DIM, NT> w;
    w.lay_out(a, lane);
    const Span span = span_of(a, a.lens[b]);
    if (span.units == 0) {
        store_nothing<F32>(a, b, h * a.group + chunk * 16 * NT, min(16 * NT, a.group - chunk * 16 * NT), threadIdx.x);
        return;
    }
    attend<F32, CACHE, DIM, NT, 4>(a, w, lds, span, b, h, 0, span.units, chunk, chunk + 1, 0, wave, lane);
}

// The work is the list of all (sequence, key head, unit of tokens); every worker, a block's four waves (TEAM 4) or a wave (TEAM 1), takes an
// equal stretch of it, found from the lengths on the device, whatever they are.  An item that lies in several stretches is left by each as a
// part, and joined by attn_join_kernel in the order of the tokens.
template <bool F32, int CACHE, int DIM, int NT, int TEAM>
__global__ __launch_bounds__(256, waves_of(F32, DIM, NT == 2)) void attn_kernel(Attn a, int top_step) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* before = reinterpret_cast<int*>(lds + Lds<F32, CACHE, DIM, NT, TEAM>::kBytes);       // [B + 1] units of the sequences before
    int* list = before + a.B + 1;                                     // their lengths, where there is room
    const bool listed = a.B <= kListed;
    __shared__ int wave_total[4];
    const int tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
    Wave<F32, CACHE, DIM, NT> w;
    {
        const int per = (a.B + 255) / 256, b0 = tid * per, b1 = min(b0 + per, a.B);
        int own = 0;
        for (int i = b0; i < b1; ++i) {
            const int len = a.lens[i];
            if (listed) list[i] = len;
            own += span_of(a, len).units;
        }
        w.lay_out(a, lane);
        int incl = own;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 63) wave_total[wave] = incl;
        __syncthreads();
        int at = incl - own;
        for (int i = 0; i < wave; ++i) at += wave_total[i];
        for (int i = b0; i < b1; ++i) {
            before[i] = at;
            at += span_of(a, listed ? list[i] : a.lens[i]).units;
        }
        if (tid == 255) before[a.B] = at;                             // (the later threads' sums are empty)
        __syncthreads();
    }
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
        if (before[b + 1] == before[b]) store_nothing<F32>(a, b, 0, a.heads * a.group, tid);

    const int worker = TEAM == 1 ? 4 * blockIdx.x + wave : blockIdx.x, workers = gridDim.x * (4 / TEAM);
    const Cuts cuts(static_cast<long>(uniform(before[a.B])) * a.heads, workers);
    long at = cuts.at(worker);
    const long stop = cuts.at(worker + 1);
    int b = 0;                                                        // the last sequence that starts at or before `at`
#pragma unroll 1
    for (int step = top_step; step > 0; step /= 2)
        if (b + step < a.B && static_cast<long>(uniform(before[b + step])) * a.heads <= at) b += step;
    Cut cut{-1, 0, 0, 0};
    bool first_item = true;
    while (at < stop) {
        while (static_cast<long>(uniform(before[b + 1])) * a.heads <= at) ++b;
        const Span span = span_of(a, uniform(listed ? list[b] : a.lens[b]));
        const int in_b = static_cast<int>(at - static_cast<long>(uniform(before[b])) * a.heads);        // (below heads * units <= 2^27)
        const int h = in_b / span.units, u0 = in_b - h * span.units;
        const int u1 = static_cast<int>(min(static_cast<long>(span.units), u0 + (stop - at)));
        if (u0 > 0 && cuts.at(worker - 1) <= at - u0)                 // begun in the stretch before (only a worker's first item can have)
            cut = Cut{(b * a.heads + h) * a.group, 2 * (worker - 1) + (cuts.at(worker - 1) == at - u0 ? 0 : 1), cuts.of(at - u0 + span.units - 1), 0};
        attend<F32, CACHE, DIM, NT, TEAM>(a, w, lds, span, b, h, u0, u1, 0, a.chunks, 2L * worker + (first_item ? 0 : 1), wave, lane);
        at += u1 - u0;
        first_item = false;
    }
    if (lane == 0 && (TEAM == 1 || wave == 0)) a.cuts[worker] = cut;
}

// Joins an item's parts, row by row (query head): blocks (w, y) those of the item that is cut for the first time where worker w's stretch
// begins.  With TEAM 4 a block's waves share a row, with TEAM 1 (few parts) each wave has one of its own.
template <bool F32, int TEAM>
__global__ __launch_bounds__(256) void attn_join_kernel(Attn a) {
    __shared__ f32x4 sums[TEAM == 4 ? 256 : 1];
    constexpr int kLanes = 64 * TEAM, kAhead = 8;
    const int w = blockIdx.x, tid = threadIdx.x, lane = TEAM == 4 ? tid : tid % 64;
    const int row = TEAM == 4 ? blockIdx.y : 4 * blockIdx.y + tid / 64;
    const Cut cut = a.cuts[w];
    if (cut.rows < 0 || row >= a.group) return;
    const int parts = cut.last - w + 2;
    auto slot_of = [&](int i) { return static_cast<long>(i == 0 ? cut.first : 2 * (w - 1 + i)) * a.group + row; };
    float top = -INFINITY, weight = 0.f;
    for (int i = tid % 64; i < parts; i += 64) top = fmaxf(top, a.part_ml[slot_of(i) * 2]);
    top = lanes_max<64>(top);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int i = tid % 64; i < parts; i += 64)
        weight = fmaf(a.part_ml[slot_of(i) * 2 + 1], __builtin_amdgcn_exp2f(a.part_ml[slot_of(i) * 2] - ref), weight);
    weight = lanes_sum<64>(weight);
    const int quads = a.dim / 4, at_once = kLanes / quads;            // threads of a part, parts at once
    const int mine = lane / quads, col = lane - mine * quads;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = mine; i0 < parts && mine < at_once; i0 += kAhead * at_once) {
        f32x4 p[kAhead];
        float m[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {                            // past the last: the last again, with no weight
            const long slot = slot_of(min(i0 + j * at_once, parts - 1));
            p[j] = *reinterpret_cast<const f32x4*>(a.part_o + slot * a.dim + 4 * col);
            m[j] = a.part_ml[slot * 2];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + j * at_once >= parts) break;
            const float f = __builtin_amdgcn_exp2f(m[j] - ref);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = fmaf(p[j][c], f, v[c]);
        }
    }
    const long head = static_cast<long>(cut.rows) + row;
    if (lane == 0 && a.lse != nullptr) a.lse[head] = natural_log_of_sum(top, weight);
    if constexpr (TEAM == 4) {
        sums[lane] = v;
        __syncthreads();
        if (mine == 0)
            for (int i = 1; i < at_once; ++i) v += sums[lane + i * quads];
    } else {
        const f32x4 own = v;
        for (int i = 1; i < at_once; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] += __shfl(own[c], (lane + i * quads) % 64);
    }
    if (mine == 0)
#pragma unroll
        for (int c = 0; c < 4; ++c) store_out<F32>(a, head * a.dim + 4 * col + c, v[c] / weight);
}

// How a call is cut.  Sequences of at most kShortUnits units are not split: a block for each.  Else the list of units is cut into a stretch per
// worker: waves by themselves where there are many items for groups of one column tile (no wave waits for another between items), else blocks.
constexpr int kShortUnits = 4, kManyItems = 1024, kMaxUnits = 256;
struct Plan {
    bool is_short;
    int team, blocks, workers;
};
Plan plan_of(const moe_kv_cfg& kv, const moe_attn_cfg& c, int compute_units) {
    const long room = static_cast<long>(c.table_pages) * kv.page_size;
    const long longest = c.window > 0 ? std::min(room, c.window + 15L) : room, units = (longest + kUnit - 1) / kUnit;
    const long items = static_cast<long>(c.B) * kv.heads;
    Plan p;
    p.is_short = units <= kShortUnits;
    p.team = c.q_heads / kv.heads <= 16 && items >= kManyItems ? 1 : 4;
    const int resident = waves_of(kv.dtype == MOE_F32, kv.head_dim, kv.dtype == MOE_BF16 && c.q_heads / kv.heads > 16);
    const int per_cu = p.team == 4 ? std::min(2, resident) : resident;
    p.blocks = static_cast<int>(std::min(units * items, static_cast<long>(per_cu) * std::min(compute_units, kMaxUnits)));
    p.workers = p.blocks * (4 / p.team);
    return p;
}

// The workspace: the parts' sums, their maxima and weights, the cuts.
struct Parts {
    size_t ml, cuts, bytes;
    Parts(const moe_kv_cfg& kv, const moe_attn_cfg& c) {
        const Plan p = plan_of(kv, c, kMaxUnits);
        const size_t rows = p.is_short ? 0 : 2 * static_cast<size_t>(p.workers) * (c.q_heads / kv.heads);
        ml = align256(rows * kv.head_dim * 4);
        cuts = ml + align256(rows * 8);
        bytes = std::max(cuts + align256(p.is_short ? 0 : p.workers * sizeof(Cut)), size_t(256));
    }
};

template <bool F32, int CACHE, int DIM, int NT>
int launch(const moe_kv_cfg& kv, const moe_attn_cfg& c, Attn& a, hipStream_t s) {
    int dev = 0;
    const DeviceInfo* info = nullptr;
    if (int rc = device_info(&dev, &info)) return rc;
    const Plan p = plan_of(kv, c, info->compute_units);
    a.chunks = (a.group + 16 * NT - 1) / (16 * NT);
    if (p.is_short) {
        hipLaunchKernelGGL((attn_short_kernel<F32, CACHE, DIM, NT>), dim3(a.B * a.heads * a.chunks), dim3(256), (Lds<F32, CACHE, DIM, NT, 4>::kBytes), s, a);
        MOE_LAUNCH_CHECK("attn_short_kernel");
        return MOE_OK;
    }
    int top_step = 1;
    while (2 * top_step < a.B) top_step *= 2;
    const size_t list = sizeof(int) * ((a.B <= kListed ? 2 : 1) * a.B + 1);
    if constexpr (NT == 1)
        if (p.team == 1)
            hipLaunchKernelGGL((attn_kernel<F32, CACHE, DIM, NT, 1>), dim3(p.blocks), dim3(256), (Lds<F32, CACHE, DIM, NT, 1>::kBytes) + list, s, a, top_step);
    if (p.team == 4)
        hipLaunchKernelGGL((attn_kernel<F32, CACHE, DIM, NT, 4>), dim3(p.blocks), dim3(256), (Lds<F32, CACHE, DIM, NT, 4>::kBytes) + list, s, a, top_step);
    MOE_LAUNCH_CHECK("attn_kernel");
    if (p.team == 1) hipLaunchKernelGGL((attn_join_kernel<F32, 1>), dim3(p.workers, (a.group + 3) / 4), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_join_kernel<F32, 4>), dim3(p.workers, a.group), dim3(256), 0, s, a);
    MOE_LAUNCH_CHECK("attn_join_kernel");
    return MOE_OK;
}

// fp32 products have no room for a second column tile in registers: larger groups read the cache again, 16 heads at a time.
template <bool F32, int CACHE>
int for_sizes(const moe_kv_cfg& kv, const moe_attn_cfg& c, Attn& a, hipStream_t s) {
    if constexpr (!F32)
        if (a.group > 16) {
            if (a.dim <= 64) return launch<F32, CACHE, 64, 2>(kv, c, a, s);
            return a.dim <= 128 ? launch<F32, CACHE, 128, 2>(kv, c, a, s) : launch<F32, CACHE, 256, 2>(kv, c, a, s);
        }
    if (a.dim <= 64) return launch<F32, CACHE, 64, 1>(kv, c, a, s);
    return a.dim <= 128 ? launch<F32, CACHE, 128, 1>(kv, c, a, s) : launch<F32, CACHE, 256, 1>(kv, c, a, s);
}

}  // namespace

size_t attn_workspace_bytes(const moe_kv_cfg& kv, const moe_attn_cfg& c) { return Parts(kv, c).bytes; }

int launch_attn_decode(const moe_kv_cfg& kv, const moe_attn_cfg& c, const void* q, long q_stride, const void* k_pages, const void* v_pages,
                       const float* k_scales, const float* v_scales, const int32_t* table, const int32_t* lens, void* out, float* lse,
                       void* ws, hipStream_t s) {
    const Parts parts(kv, c);
    char* base = static_cast<char*>(ws);
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
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(base + parts.ml);
    a.cuts = reinterpret_cast<Cut*>(base + parts.cuts);
    a.B = c.B;
    a.heads = kv.heads;
    a.group = c.q_heads / kv.heads;
    a.chunks = 0;                                                     // set where the column tiles are chosen
    a.dim = kv.head_dim;
    a.pages = kv.pages;
    a.page_bits = __builtin_ctz(kv.page_size);
    a.table_pages = c.table_pages;
    a.window = c.window;
    a.scale = (c.scale > 0.f ? c.scale : 1.f / sqrtf(static_cast<float>(kv.head_dim))) * 1.4426950408889634f;
    if (kv.dtype == MOE_BF16) return kv.cache_dtype == MOE_BF16 ? for_sizes<false, MOE_BF16>(kv, c, a, s) : for_sizes<false, MOE_E4M3>(kv, c, a, s);
    if (kv.cache_dtype == MOE_F32) return for_sizes<true, MOE_F32>(kv, c, a, s);
    return kv.cache_dtype == MOE_BF16 ? for_sizes<true, MOE_BF16>(kv, c, a, s) : for_sizes<true, MOE_E4M3>(kv, c, a, s);
}

}  // namespace moe
