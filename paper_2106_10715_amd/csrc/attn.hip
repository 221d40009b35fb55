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

constexpr int kUnit = 128;          // tokens a block takes in one step, 32 for each of its four waves: the grain in which the work is shared out
constexpr int kToll = 2;            // what the beginning and the end of an item cost, in units: short items take a block's time too
constexpr int kAsk = 32;            // steps whose pages a wave looks up at once
constexpr int kMaxB = 4096;         // sequences
constexpr float kSlack = 8.f;       // the running maximum is raised only where a logit passes it by more than this (as a power of two)

// An item of the work, a (sequence, key head, 16 * NT of its query heads), cut where a worker's stretch begins: written by that worker, for
// the join.
struct Cut {
    int rows;                       // its key head's first row of out and lse; -1: nothing is cut here, or not for the first time
    int first, last;                // slot of its first part, worker of its last (in between: the slots 2 w)
    int in_group;                   // its first query head in the key head's group
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
    int B, heads, group, chunks, items, item_rows, dim, pages, page_bits, table_pages, window;
    int over_row;                   // 2^16 over the pieces of a row, rounded up: a quotient of numbers below 2^10 is a product and a shift
    float scale;                    // times log2 e
};

// The tokens [first, end) sequence b attends to, and `base`, `first` rounded down to a run of 16 (which lies in one page).
struct Span {
    int first, end, base, units;
    __device__ int places() const { return units == 0 ? 0 : units + kToll; }        // in the list of all work
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
    __device__ Cuts(long n, int w, double one_over_w) : q(static_cast<long>(static_cast<double>(n) * one_over_w)) {
        q += q * w > n ? -1 : (q + 1) * w <= n ? 1 : 0;
        rest = n - q * w;
    }
    __device__ long at(int i) const { return i * q + min(static_cast<long>(i), rest); }
    __device__ int of(long r) const { return static_cast<int>(r < rest * (q + 1) ? over(r, q + 1) : rest + over(r - rest * (q + 1), q)); }
};

// Waves a SIMD has room for: with two, a wave has 256 registers.
constexpr int waves_of(bool f32, int cache, int dim, int nt) { return nt == 1 && (dim <= 64 || (dim <= 128 && !f32 && cache == MOE_E4M3)) ? 2 : 1; }

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// How rows of a cache type lie in the lanes.
template <int CACHE, int DIM>
struct Layout {
    static constexpr int kWidth = CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1;
    static constexpr int kPiece = 16 / kWidth;                 // elements of a 16-byte piece of K
    static constexpr int kPieces = DIM / (4 * kPiece);         // pieces of a row per lane: lane quarter g holds piece 4 i + g
    static constexpr int kHalves = DIM > 128 ? 2 : 1;          // V: a row is read in runs of up to 128 elements
    static constexpr int kOwn = DIM > 128 ? 8 : DIM / 16;      // of which each of 16 lanes holds this many
    static constexpr int kRun = 16 * DIM * kWidth;             // bytes of 16 rows of K
    static constexpr bool kStaged = kRun <= 8192;              // whether they pass through the LDS
    static constexpr bool kAhead = DIM <= 128;                 // whether a second tile has room in registers (40 x 2048 tokens, e4m3, 256 wide: 45.8 us with, 41.4 without)
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

// N bf16 or e4m3 values as N / 2 pairs of bf16 (e4m3 values are bf16 values).
template <int CACHE, int N>
__device__ inline void to_pairs(const uint32_t* w, uint32_t* out) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if constexpr (CACHE == MOE_BF16) out[i] = w[i];
        else if (i % 2 == 0) out[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i / 2], 1.f, false));
        else out[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i / 2], 1.f, true));
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

constexpr float kMost = 0x1.fep127f;        // the largest bf16 value

// Two values as bf16, and what that leaves of them.  CUT: their upper halves (rounded, the largest finite values would be infinite).
template <bool CUT = false>
__device__ inline uint32_t take_bf16x2(float& lo, float& hi) {
    const uint32_t u = CUT ? __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u) : to_bf16x2(lo, hi);
    lo -= bf16_lo(u);
    hi -= bf16_hi(u);
    return u;
}

// One wave's attention of 16 * NT query heads over some of an item's tokens.
//
// An fp32 cache takes the fp32 matrix instruction.  The other caches' values are bf16 values: the bf16 instruction multiplies them exactly, with
// fp32 queries in three parts of 8 bits (all of their bits; a third of the fp32 instruction's time), and the weights p, of at most 2^8, in as
// many parts as the output is worth: three for fp32, two for bf16 (with one, its rounding would be as large an error as the output's own; the
// second costs nothing, 256 sequences in e4m3 take 349.8 us with one and 349.1 with two).
template <bool F32, int CACHE, int DIM, int NT>
struct Wave {
    using L = Layout<CACHE, DIM>;
    static constexpr bool kWide = CACHE == MOE_F32;                                 // fp32 products
    static constexpr int kSteps = L::kPiece / 8;                                    // bf16: matrix instructions of one piece of K
    static constexpr int kPartsQ = F32 ? 3 : 1, kPartsP = F32 ? 3 : 2;
    float q32[F32 ? NT : 1][F32 ? L::kPieces : 1][F32 ? L::kPiece : 1];             // Q^T as it came, fp32
    bf16x8 q16[kWide ? 1 : kPartsQ][kWide ? 1 : NT][kWide ? 1 : L::kPieces][kWide ? 1 : kSteps];
    f32x4 o[NT][L::kHalves][L::kOwn];                                               // O^T: dim 128 half + own (4 g + r) + j, head l % 16
    float m[NT], l[NT];                                                             // maximum (the same in all quarters), weight of the own tokens

    uint32_t k_at[L::kPieces], k_in[L::kPieces], k_out[L::kPieces], v_at[L::kHalves];    // of this lane: bytes from a run's first row, bytes in the LDS
    int row_bytes;

    // What does not change from item to item.  Where rows are shorter than DIM, K has zeros past their end as Q has (a zero of Q would make NaN of an
    // infinity): past the end of a load, or as clear_past_end leaves them.  Columns of V past the end are taken from the last ones and not stored.
    __device__ void lay_out(const Attn& a, int lane) {
        const int n = lane % 16, g = lane / 16, per = a.dim / L::kPiece;
        row_bytes = a.dim * L::kWidth;
#pragma unroll
        for (int i = 0; i < L::kPieces; ++i) {
            if constexpr (!L::kStaged) {
                k_at[i] = 4 * i + g < per ? n * row_bytes + 16 * (4 * i + g) : 0x7fffff00;
                continue;
            }
            const int at = min(64 * i + lane, 16 * per - 1), token = (at * a.over_row) >> 16, piece = at - token * per;
            k_at[i] = 16 * at;
            k_in[i] = 16 * (token * 4 * L::kPieces + ((piece ^ token) & (4 * L::kPieces - 1)));          // 16 tokens' pieces: in 16 different places of a row
            k_out[i] = 16 * (n * 4 * L::kPieces + (((4 * i + g) ^ n) & (4 * L::kPieces - 1)));
        }
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf) v_at[hf] = 4 * g * row_bytes + min(128 * hf + L::kOwn * n, a.dim - L::kOwn) * L::kWidth;
    }

    // Zeros past the rows' ends in the wave's run of K in LDS.  Nothing is written over them, and each is read by its own lane alone.
    __device__ void clear_past_end(const Attn& a, char* mine, int lane) const {
        if constexpr (L::kStaged)
            if (a.dim % (4 * L::kPiece) != 0)
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i)
                    if (4 * i + lane / 16 >= a.dim / L::kPiece) *reinterpret_cast<u32x4*>(mine + k_out[i]) = u32x4{0, 0, 0, 0};
    }

    __device__ void reset() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -INFINITY;
            l[t] = 0.f;
#pragma unroll
            for (int h = 0; h < L::kHalves; ++h)
#pragma unroll
                for (int j = 0; j < L::kOwn; ++j) o[t][h][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }

    // Requests the query heads [head0, head0 + n_heads) of sequence b; zeros in the columns and past the row's end.
    __device__ void load_q(const Attn& a, int b, int head0, int n_heads, int lane) {
        constexpr int kBytes = F32 ? 4 : 2;
        const int n = lane % 16, g = lane / 16;
        const auto rows = stretch_of(static_cast<const char*>(a.q) + (b * a.q_stride + static_cast<long>(head0) * a.dim) * kBytes, n_heads * a.dim * kBytes);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < L::kPieces; ++i) {
                const int d0 = (4 * i + g) * L::kPiece;
                const uint32_t at = d0 < a.dim ? ((16 * t + n) * a.dim + d0) * kBytes : 0x7fffff00;
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < L::kPiece; c += 4) {
                        const f32x4 u = __builtin_bit_cast(f32x4, load_raw<16>(rows, at + 4 * c, 0));
#pragma unroll
                        for (int e = 0; e < 4; ++e) q32[t][i][c + e] = u[e];
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) q16[0][t][i][s] = __builtin_bit_cast(bf16x8, load_raw<16>(rows, at + 16 * s, 0));
                }
            }
    }

    // Once the queries are wanted.
    __device__ void split_q() {
        if constexpr (F32 && !kWide)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s)
#pragma unroll
                        for (int part = 0; part < kPartsQ; ++part) {
                            u32x4 u;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                float &lo = q32[t][i][8 * s + 2 * c], &hi = q32[t][i][8 * s + 2 * c + 1];
                                u[c] = part == 0 ? take_bf16x2<true>(lo, hi) : take_bf16x2(lo, hi);
                            }
                            q16[part][t][i][s] = __builtin_bit_cast(bf16x8, u);
                        }
    }

    // The pages of the runs of up to kAsk steps from token t0 on: lane 2 s + r holds that of run r of step s, `tokens` from step to step.
    __device__ static int pages_of(const Attn& a, const Span& span, int b, int t0, int lane, int tokens) {
        const int t = min(t0 + (lane / 2) * tokens + 16 * (lane % 2), (span.end - 1) & ~15);        // (past the end: a run that exists)
        return a.table[static_cast<long>(b) * a.table_pages + (t >> a.page_bits)];
    }

    // 32 tokens' rows of one key head as they come from the cache.
    static constexpr int kRowBytes = L::kOwn * L::kWidth;
    struct Tile {
        Raw<16> k[2][L::kPieces];
        Raw<kRowBytes> v[2][4][L::kHalves];
        f32x4 ks[2], vs[2];
    };

    // Requests tokens [t0, t0 + 32) of key head h, t0 a multiple of 16, step `s` of `ids`; reads nothing if not `wanted`.
    __device__ void load(Tile& x, const Attn& a, const Span& span, int ids, int s, int h, int t0, bool wanted, int lane) const {
        const int g = lane / 16, bytes = wanted ? 16 * row_bytes : 0;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = min(t0 + 16 * r, (span.end - 1) & ~15), page = min(max(__builtin_amdgcn_readlane(ids, (2 * s + r) & 63), 0), a.pages - 1);
            const long at = ((static_cast<long>(page) * a.heads + h) << a.page_bits) + (t & ((1 << a.page_bits) - 1));
            const auto kr = stretch_of(a.k_pages + at * row_bytes, bytes), vr = stretch_of(a.v_pages + at * row_bytes, bytes);
#pragma unroll
            for (int i = 0; i < L::kPieces; ++i) x.k[r][i] = load_raw<16>(kr, k_at[i], 0);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int hf = 0; hf < L::kHalves; ++hf) x.v[r][c][hf] = load_raw<kRowBytes>(vr, v_at[hf], c * row_bytes);
            if constexpr (CACHE == MOE_E4M3) {
                x.ks[r] = __builtin_bit_cast(f32x4, load_raw<16>(stretch_of(a.k_scales + at, wanted ? 64 : 0), 16 * g, 0));
                x.vs[r] = __builtin_bit_cast(f32x4, load_raw<16>(stretch_of(a.v_scales + at, wanted ? 64 : 0), 16 * g, 0));
            }
        }
    }

    // Attends to the tile of tokens [t0, t0 + 32); those outside of the span weigh nothing.
    // `mine`: a run of K in LDS that no other wave touches.
    __device__ void step(Tile& x, char* mine, const Attn& a, const Span& span, int t0, int lane) {
        const int g = lane / 16;
        auto &k = x.k;
        auto &v = x.v;
        auto &ks = x.ks, &vs = x.vs;
        if constexpr (L::kStaged) {
            // A wave's LDS operations are done in their order: between what its lanes write and read only the compiler has to keep it.
            auto in_order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); };
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                in_order();
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) *reinterpret_cast<u32x4*>(mine + k_in[i]) = __builtin_bit_cast(u32x4, k[r][i]);
                in_order();
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) k[r][i] = __builtin_bit_cast(Raw<16>, *reinterpret_cast<const u32x4*>(mine + k_out[i]));
            }
        }

        // The lesser parts of fp32 queries have a sum of their own: a part that is zero, or of the other sign, makes NaN of an infinite key, as what is
        // left of an infinite query does, and then the leading part's sum, which is not finite either, is the logit.
        f32x4 s[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                s[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
                f32x4 rest = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::kPieces; ++i) {
                    if (4 * i * L::kPiece >= a.dim) break;
                    if constexpr (kWide) {
#pragma unroll
                        for (int c = 0; c < L::kPiece; ++c)
                            s[t][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[r][i].w[c]), q32[t][i][c], s[t][r], 0, 0, 0);
                    } else {
                        u32x4 pairs[kSteps];
                        to_pairs<CACHE, L::kPiece>(k[r][i].w, reinterpret_cast<uint32_t*>(pairs));
#pragma unroll
                        for (int st = 0; st < kSteps; ++st) {
                            const auto at = __builtin_bit_cast(bf16x8, pairs[st]);
#pragma unroll
                            for (int part = kPartsQ - 1; part > 0; --part) rest = __builtin_amdgcn_mfma_f32_16x16x32_bf16(at, q16[part][t][i][st], rest, 0, 0, 0);
                            s[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(at, q16[0][t][i][st], s[t][r], 0, 0, 0);
                        }
                    }
                }
                if constexpr (F32 && !kWide)
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[t][r][c] += __builtin_amdgcn_fmed3f(rest[c], -kMost, kMost);       // (the lower bound for NaN)
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

        if constexpr (kWide) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int hf = 0; hf < L::kHalves; ++hf)
#pragma unroll
                        for (int j = 0; j < L::kOwn; ++j)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
                                o[t][hf][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r][c][hf].w[j]), p[t][r][c], o[t][hf][j], 0, 0, 0);
        } else {
            bf16x8 weights[NT][kPartsP];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int part = 0; part < kPartsP; ++part) {
                    u32x4 u;
#pragma unroll
                    for (int c = 0; c < 4; ++c) u[c] = take_bf16x2(p[t][c / 2][2 * (c % 2)], p[t][c / 2][2 * (c % 2) + 1]);
                    weights[t][part] = __builtin_bit_cast(bf16x8, u);
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
#pragma unroll
                        for (int part = kPartsP - 1; part >= 0; --part)
                            o[t][hf][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), weights[t][part], o[t][hf][j], 0, 0, 0);
                }
            }
        }
    }
};

template <bool F32>
__device__ inline void store_out(const Attn& a, long at, float v) {
    if constexpr (F32) static_cast<float*>(a.out)[at] = v;
    else static_cast<__bf16*>(a.out)[at] = static_cast<__bf16>(v);
}
__device__ inline float natural_log_of_sum(float m, float weight) { return (m + __builtin_amdgcn_logf(weight)) * 0.6931471805599453f; }

// One sequence and key head, units [u0, u1), and 16 * NT of its query heads.  slot -1: the units are all there are, else the part's place.
struct Item {
    int b, h, chunk, u0, u1;
    long slot;
    Span span;
};

// The waves' sums of up to 16 heads over up to 128 columns.
template <int DIM, int NT>
struct Sums {
    static constexpr int kCols = DIM > 128 ? 128 : DIM;
    float o[4][16][kCols + 4];
    float m[4][16 * NT], l[4][16 * NT];
};

// A barrier for what lies in LDS: loads from memory stay on their way across it.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Joins the four waves' sums of an item and stores its results, or its part's.  The block's last barrier before the next call comes after
// every use of `sums`.
template <bool F32, int CACHE, int DIM, int NT>
__device__ void finish(const Attn& a, const Wave<F32, CACHE, DIM, NT>& w, Sums<DIM, NT>& sums, const Item& it, int wave, int lane) {
    using L = Layout<CACHE, DIM>;
    constexpr int kCols = Sums<DIM, NT>::kCols;
    const int n = lane % 16, g = lane / 16, tid = 64 * wave + lane;
    const int in_group = 16 * NT * it.chunk, n_heads = min(16 * NT, a.group - in_group);
    const long head0 = (static_cast<long>(it.b) * a.heads + it.h) * a.group + in_group, part0 = it.slot * a.group + in_group;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float l = quarters_sum(w.l[t]);
        if (g == 0) {
            sums.m[wave][16 * t + n] = w.m[t];
            sums.l[wave][16 * t + n] = l;
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf) {
            if (16 * t + n < n_heads)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < L::kOwn; j += 4)
                        *reinterpret_cast<f32x4*>(&sums.o[wave][n][L::kOwn * (4 * g + r) + j]) =
                            f32x4{w.o[t][hf][j][r], w.o[t][hf][j + 1][r], w.o[t][hf][j + 2][r], w.o[t][hf][j + 3][r]};
            lds_barrier();
            const int rows = min(16, n_heads - 16 * t), quads = min(kCols, a.dim - 128 * hf) / 4;
            for (int i = tid; i < rows * (kCols / 4); i += 256) {
                const int row = i / (kCols / 4), col = i % (kCols / 4), c = 16 * t + row;
                if (col >= quads) continue;
                const float top = fmaxf(fmaxf(sums.m[0][c], sums.m[1][c]), fmaxf(sums.m[2][c], sums.m[3][c])), ref = top == -INFINITY ? 0.f : top;
                float weight = 0.f;
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const float f = __builtin_amdgcn_exp2f(sums.m[i4][c] - ref);
                    const f32x4 o = *reinterpret_cast<const f32x4*>(&sums.o[i4][row][4 * col]);
                    weight = fmaf(sums.l[i4][c], f, weight);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], f, v[e]);
                }
                if (it.slot >= 0) {
                    *reinterpret_cast<f32x4*>(a.part_o + (part0 + c) * a.dim + 128 * hf + 4 * col) = v;
                    if (hf == 0 && col == 0) {
                        a.part_ml[(part0 + c) * 2] = top;
                        a.part_ml[(part0 + c) * 2 + 1] = weight;
                    }
                    continue;
                }
                const long at = (head0 + c) * a.dim + 128 * hf + 4 * col;
                const float inv = weight == 0.f ? 0.f : 1.f / weight;         // logits of -infinity alone: as if there were no tokens
                if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = v * inv;
                else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = u32x2{to_bf16x2(v[0] * inv, v[1] * inv), to_bf16x2(v[2] * inv, v[3] * inv)};
                if (hf == 0 && col == 0 && a.lse != nullptr) a.lse[head0 + c] = natural_log_of_sum(top, weight);
            }
            lds_barrier();
        }
}

// The items a block works on, one after the other.
struct Feed {
    const Attn& a;
    const int *before, *list;       // places of the sequences before; lengths
    int worker, b;
    long at, stop;
    bool first;

    __device__ long before_of(int i) const { return static_cast<long>(uniform(before[i])) * a.items; }
    __device__ Span span(int i) const { return span_of(a, uniform(list[i])); }
    // The last sequence that begins at or before a place: 64 of them, then those up to the next of the 64, looked at by a lane each.
    __device__ int sequence_at(long place) const {
        const int lane = threadIdx.x % 64;
        auto last_of = [&](int i) { return __popcll(__ballot(i < a.B && static_cast<long>(before[min(i, a.B)]) * a.items <= place)) - 1; };
        const int from = a.B > 64 ? 64 * last_of(64 * lane) : 0;
        return from + last_of(from + lane);
    }
    // A cut that would leave an item's beginning to one block and its tokens to the next is moved to before it.  i: the sequence it lies in.
    __device__ long moved(long place, int& i) const {
        i = sequence_at(place);
        if (place >= before_of(a.B)) return place;
        const int in_b = static_cast<int>(place - before_of(i)), in_item = in_b % span(i).places();
        return in_item <= kToll ? place - in_item : place;
    }
    __device__ Feed(const Attn& args, const int* before_, const int* list_, const Cuts& cuts, int worker_)
        : a(args), before(before_), list(list_), worker(worker_), first(true) {
        int end;
        at = moved(cuts.at(worker), b);
        stop = moved(cuts.at(worker + 1), end);
    }
    // The piece at `at`, which must be below `stop`.
    __device__ Item piece() {
        while (before_of(b + 1) <= at) ++b;
        Item it;
        it.b = b;
        it.span = span(b);
        const int in_b = static_cast<int>(at - before_of(b)), places = it.span.places();       // (below items * places < 2^28)
        const int item = in_b / places, in_item = in_b - item * places;
        it.h = item / a.chunks;
        it.chunk = item - it.h * a.chunks;
        it.u0 = max(0, in_item - kToll);
        it.u1 = static_cast<int>(min(static_cast<long>(places), in_item + (stop - at))) - kToll;
        it.slot = it.u0 == 0 && it.u1 == it.span.units ? -1 : 2L * worker + (first ? 0 : 1);
        return it;
    }
    __device__ bool next(Item& it) {
        at += it.u1 - it.u0 + (it.u0 == 0 ? kToll : 0);
        first = false;
        if (at >= stop) return false;
        it = piece();
        return true;
    }
};

// Works through items, `more` saying which comes next.  A wave has two tiles on the way while it attends to a third (kAhead), the next
// item's first ones among them, so that what an item's end costs is its barriers and not the memory's answer.  TEAM waves share an item's tokens, `wave` this one's number;
// `end(item)` stores what they have found.
template <int TEAM, bool F32, int CACHE, int DIM, int NT, typename More, typename End>
__device__ void work(const Attn& a, Wave<F32, CACHE, DIM, NT>& w, char* mine, Item it, More more, End end, int wave, int lane) {
    using L = Layout<CACHE, DIM>;
    constexpr int kStep = 32 * TEAM;
    constexpr bool kAskEarly = !(F32 && DIM > 128);              // (with the next queries beside its sums, a wave of these would spill up to 63 registers)
    typename Wave<F32, CACHE, DIM, NT>::Tile x, y;
    auto begin = [&](const Item& i) { return i.span.base + i.u0 * kUnit + 32 * wave; };
    auto limit = [&](const Item& i) { return min(i.span.end, i.span.base + i.u1 * kUnit); };
    auto steps_from = [&](const Item& i, int t) { return max(0, min(kAsk, (limit(i) - t + kStep - 1) / kStep)); };
    auto ask_q = [&](const Item& i) { w.load_q(a, i.b, i.h * a.group + 16 * NT * i.chunk, min(16 * NT, a.group - 16 * NT * i.chunk), lane); };
    int t = begin(it), steps = steps_from(it, t), ids = w.pages_of(a, it.span, it.b, t, lane, kStep);
    ask_q(it);
    w.reset();
    if constexpr (L::kAhead) w.load(x, a, it.span, ids, 0, it.h, t, steps > 0, lane);
    w.clear_past_end(a, mine, lane);
    w.split_q();
    while (true) {
        Item then = it;
        const bool last = t + kAsk * kStep >= limit(it), any = !last || more(then);
        const int then_t = last ? begin(then) : t + kAsk * kStep, then_steps = any ? steps_from(then, then_t) : 0;
        const int then_ids = w.pages_of(a, then.span, then.b, any ? then_t : t, lane, kStep);
        if constexpr (L::kAhead) {
            if (steps == 0) w.load(x, a, then.span, then_ids, 0, then.h, then_t, then_steps > 0, lane);
            for (int s = 0; s < steps; s += 2) {
                w.load(y, a, it.span, ids, s + 1, it.h, t + (s + 1) * kStep, s + 1 < steps, lane);
                w.step(x, mine, a, it.span, t + s * kStep, lane);
                const bool here = s + 2 < steps, over = s + 2 >= steps;
                w.load(x, a, over ? then.span : it.span, over ? then_ids : ids, over ? 0 : s + 2, over ? then.h : it.h, over ? then_t : t + (s + 2) * kStep,
                       here || (over && then_steps > 0), lane);
                if (s + 1 < steps) w.step(y, mine, a, it.span, t + (s + 1) * kStep, lane);
            }
        } else {
            for (int s = 0; s < steps; ++s) {
                w.load(x, a, it.span, ids, s, it.h, t + s * kStep, true, lane);
                w.step(x, mine, a, it.span, t + s * kStep, lane);
            }
        }
        if (last) {
            if constexpr (kAskEarly)
                if (any) ask_q(then);
            end(it);
            w.reset();
            if (!any) return;
            if constexpr (!kAskEarly) ask_q(then);
            w.split_q();
        }
        it = then;
        t = then_t;
        steps = then_steps;
        ids = then_ids;
    }
}

// Outputs of query heads of a sequence without tokens.
template <bool F32>
__device__ inline void store_nothing(const Attn& a, long row, int n_heads, int tid, int threads) {
    for (int i = tid; i < n_heads * a.dim; i += threads) store_out<F32>(a, row * a.dim + i, 0.f);
    for (int i = tid; i < n_heads && a.lse != nullptr; i += threads) a.lse[row + i] = -INFINITY;
}

// A block for each sequence, key head and 16 * NT of its query heads; nothing is split.
template <bool F32, int CACHE, int DIM, int NT>
__global__ __launch_bounds__(256, waves_of(F32, CACHE, DIM, NT)) void attn_short_kernel(Attn a) {
    __shared__ __attribute__((aligned(16))) char runs[4][Layout<CACHE, DIM>::kStaged ? Layout<CACHE, DIM>::kRun : 16];
    __shared__ Sums<DIM, NT> sums;
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    const int pair = blockIdx.x / a.chunks;
    Item it{pair / a.heads, pair % a.heads, static_cast<int>(blockIdx.x % a.chunks), 0, 0, -1, {}};
    Wave<F32, CACHE, DIM, NT> w;
    w.lay_out(a, lane);
    it.span = span_of(a, a.lens[it.b]);
    it.u1 = it.span.units;
    if (it.u1 == 0) {
        store_nothing<F32>(a, static_cast<long>(pair) * a.group + 16 * NT * it.chunk, min(16 * NT, a.group - 16 * NT * it.chunk), threadIdx.x, 256);
        return;
    }
    work<4>(a, w, runs[wave], it, [](Item&) { return false; }, [&](const Item& i) { finish(a, w, sums, i, wave, lane); }, wave, lane);
}

// The results of a wave that has had an item to itself.
template <bool F32, int CACHE, int DIM, int NT>
__device__ void finish_alone(const Attn& a, const Wave<F32, CACHE, DIM, NT>& w, const Item& it, int lane) {
    constexpr int kOwn = Layout<CACHE, DIM>::kOwn;
    const int n = lane % 16, g = lane / 16, in_group = 16 * NT * it.chunk, n_heads = min(16 * NT, a.group - in_group);
    const long head0 = (static_cast<long>(it.b) * a.heads + it.h) * a.group + in_group;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float l = quarters_sum(w.l[t]), inv = l == 0.f ? 0.f : 1.f / l;
        const int c = 16 * t + n;
        if (c >= n_heads) continue;
        if (g == 0 && a.lse != nullptr) a.lse[head0 + c] = natural_log_of_sum(w.m[t], l);
#pragma unroll
        for (int hf = 0; hf < Layout<CACHE, DIM>::kHalves; ++hf)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 128 * hf + kOwn * (4 * g + r);
                if (d >= a.dim) continue;                             // (a.dim is a multiple of kOwn)
                const long at = (head0 + c) * a.dim + d;
#pragma unroll
                for (int j = 0; j < kOwn; j += 4) {
                    const f32x4 v = f32x4{w.o[t][hf][j][r], w.o[t][hf][j + 1][r], w.o[t][hf][j + 2][r], w.o[t][hf][j + 3][r]} * inv;
                    if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at + j) = v;
                    else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at + j) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
                }
            }
    }
}

// Many short sequences: a wave for each item, and no wait for others.
template <bool F32, int CACHE, int DIM, int NT>
__global__ __launch_bounds__(256, waves_of(F32, CACHE, DIM, NT)) void attn_wave_kernel(Attn a) {
    __shared__ __attribute__((aligned(16))) char runs[4][Layout<CACHE, DIM>::kStaged ? Layout<CACHE, DIM>::kRun : 16];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), index = 4 * blockIdx.x + wave;
    if (index >= a.B * a.items) return;                               // (no barrier in this kernel)
    const int pair = index / a.chunks;
    Item it{pair / a.heads, pair % a.heads, index % a.chunks, 0, 0, -1, {}};
    Wave<F32, CACHE, DIM, NT> w;
    w.lay_out(a, lane);
    it.span = span_of(a, uniform(a.lens[it.b]));
    it.u1 = it.span.units;
    if (it.u1 == 0) {
        store_nothing<F32>(a, static_cast<long>(pair) * a.group + 16 * NT * it.chunk, min(16 * NT, a.group - 16 * NT * it.chunk), lane, 64);
        return;
    }
    work<1>(a, w, runs[wave], it, [](Item&) { return false; }, [&](const Item& i) { finish_alone(a, w, i, lane); }, 0, lane);
}

// The work is the list of all (sequence, key head, 16 * NT of its query heads, unit of tokens); every block takes an equal stretch of it, found from the lengths on the
// device, whatever they are.  An item that lies in several stretches is left by each as a part, and joined by attn_join_kernel in the order of
// the tokens.
template <bool F32, int CACHE, int DIM, int NT>
__global__ __launch_bounds__(256, waves_of(F32, CACHE, DIM, NT)) void attn_kernel(Attn a, double one_over_workers) {
    __shared__ __attribute__((aligned(16))) char runs[4][Layout<CACHE, DIM>::kStaged ? Layout<CACHE, DIM>::kRun : 16];
    __shared__ Sums<DIM, NT> sums;
    __shared__ int before[kMaxB + 1], list[kMaxB], wave_total[4];       // places of the sequences before; lengths
    const int tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
    Wave<F32, CACHE, DIM, NT> w;
    {
        const int per = (a.B + 255) / 256, b0 = tid * per, b1 = min(b0 + per, a.B);
        int own = 0;
        for (int i = b0; i < b1; ++i) {
            const int len = a.lens[i];
            list[i] = len;
            own += span_of(a, len).places();
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
            at += span_of(a, list[i]).places();
        }
        if (tid == 255) before[a.B] = at;                             // (the later threads' sums are empty)
        __syncthreads();
    }
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
        if (before[b + 1] == before[b]) store_nothing<F32>(a, static_cast<long>(b) * a.heads * a.group, a.heads * a.group, tid, 256);

    const int worker = blockIdx.x;
    const Cuts cuts(static_cast<long>(uniform(before[a.B])) * a.items, gridDim.x, one_over_workers);
    Feed feed(a, before, list, cuts, worker);
    Cut cut{-1, 0, 0, 0};
    if (feed.at < feed.stop) {
        const Item it = feed.piece();
        const long start = feed.at - it.u0 - kToll, left = cuts.at(worker - 1);
        if (it.u0 > 0 && left <= start + kToll)                       // begun in the stretch before
            cut = Cut{(it.b * a.heads + it.h) * a.group, 2 * (worker - 1) + (left >= start ? 0 : 1), cuts.of(start + it.span.units + kToll - 1), 16 * NT * it.chunk};
        if (tid == 0) a.cuts[worker] = cut;
        work<4>(a, w, runs[wave], it, [&](Item& i) { return feed.next(i); }, [&](const Item& i) { finish(a, w, sums, i, wave, lane); }, wave, lane);
    } else if (tid == 0) {
        a.cuts[worker] = cut;
    }
}

// Joins an item's parts, row by row (query head): blocks (w, y) those of the item that is cut for the first time where worker w's stretch
// begins.  With few parts each wave has a row of its own (TEAM 1), else a block's waves share one (TEAM 4).
template <bool F32, int TEAM>
__global__ __launch_bounds__(256) void attn_join_kernel(Attn a) {
    __shared__ f32x4 sums[TEAM == 4 ? 256 : 1];
    constexpr int kLanes = 64 * TEAM, kAhead = 8;
    const int w = blockIdx.x, tid = threadIdx.x, lane = TEAM == 4 ? tid : tid % 64;
    const Cut cut = a.cuts[w];
    const int in_item = TEAM == 4 ? blockIdx.y : 4 * blockIdx.y + tid / 64, row = cut.in_group + in_item;
    if (cut.rows < 0 || in_item >= a.item_rows || row >= a.group) return;
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
        for (int c = 0; c < 4; ++c) store_out<F32>(a, head * a.dim + 4 * col + c, weight == 0.f ? 0.f : v[c] / weight);
}

// How a call is cut: a wave or a block for each item, or, where sequences can be longer than `whole_units`, a stretch of the list of units for each block.
constexpr int kMaxUnits = 256;
struct Plan {
    bool alone, is_short;           // a wave for each item; a block for each item
    int workers;
};
// Matrix columns, in sixteens, that take a key head's query heads.  fp32 products and heads of over 128 have no room for a second sixteen in
// registers (256 wide in bf16: 185 spilled): larger groups read the cache again for each.
int columns_of(const moe_kv_cfg& kv, int group) { return kv.dtype == MOE_BF16 && kv.head_dim <= 128 && group > 16 ? 2 : 1; }
int chunks_of(const moe_kv_cfg& kv, const moe_attn_cfg& c) {
    const int group = c.q_heads / kv.heads, rows = 16 * columns_of(kv, group);
    return (group + rows - 1) / rows;
}
// Units up to which an item is left whole.  A split costs a join and the search for the cuts, 5 to 6 us, and two units per item; a whole item the
// time of one block alone, per unit 0.8 us (64 wide in bf16) to 1.1 (128 wide) where two tiles are in flight, else 2 to 2.5.  More items than
// compute units hide each other's waits.  us split / whole, ragged lengths, bf16:
//   64 heads of 64, bf16 cache:      1 x 1000 12.4 / 10.1, 4 x 2048 19.8 / 17.3, 40 x 2048 117.4 / 113.5, but 1 x 2048 14.6 / 16.1
//   64 over 8 of 128, e4m3 cache:    16 x 1500 17.7 / 17.5, 64 x 2048 36.0 / 32.8, 200 x 1000 60.0 / 48.8, but 16 x 2048 19.1 / 21.7
//   32 over 8 of 128, bf16 cache:    4 x 700 11.8 / 11.0, 16 x 1000 16.2 / 14.4, 200 x 1000 77.2 / 73.0, but 4 x 1000 12.3 / 13.3, 16 x 1500 18.3 / 19.2
//   16 over 2 of 256, bf16 cache:    16 x 500 15.7 / 14.5, but 4 x 700 13.9 / 19.7, 16 x 700 14.0 / 18.2;  64 x 700 22.0 / 20.7, 200 x 1000 47.2 / 47.3
//   40 heads of 160, bf16 cache:     2 x 1000 16.4 / 23.0, 40 x 1000 105.3 / 106.6 (all full: 175.5 / 192.1)
//   64 heads of 160, e4m3 cache:     4 x 700 21.0 / 18.0, 40 x 1000 143.9 / 129.3, 40 x 1500 185.6 / 168.4, but 64 over 8 of 192: 8 x 1000 17.0 / 20.8
//   32 over 8 of 128, fp32 over bf16: 16 x 700 15.4 / 12.2, 40 x 1000 24.0 / 18.4, 200 x 1000 78.8 / 74.7 (all full: 141.5 / 142.8);
//                                    40 heads of 160: 4 x 1000 23.8 / 26.8, 8 x 1000 34.2 / 27.9 (all full: 48.1 / 54.7), 40 x 1000 117 / 112 (181 / 197)
//   12 over 4 of 80, fp32 cache:     16 x 500 17.0 / 15.9, 64 x 700 28.0 / 23.1, 64 x 1000 31.9 / 28.9, but 4 x 700 14.5 / 21.9, 16 x 700 17.2 / 20.7, 200 x 1000
//                                    65.8 / 71.0;  40 heads of 80: 40 x 700 93.6 / 93.7 (all full: 142.6 / 159.4)
//   16 over 4 of 256, fp32 cache:    2 x 128 17.7 / 13.1, 16 x 256 41.1 / 31.7, 64 x 500 77.3 / 72.0, but 2 x 500 19.4 / 43.1, 16 x 384 42.0 / 48.4,
//                                    200 x 700 242 / 249 (all full: 357 / 419)
int row_bytes_of(const moe_kv_cfg& kv) { return kv.head_dim * (kv.cache_dtype == MOE_F32 ? 4 : kv.cache_dtype == MOE_BF16 ? 2 : 1); }
int whole_units(const moe_kv_cfg& kv, long items) {
    if (kv.cache_dtype == MOE_F32) return kv.head_dim > 128 && items < 256 ? 2 : 4;
    if (kv.head_dim > 128) return kv.cache_dtype == MOE_E4M3 && items >= 128 ? 8 : 4;
    if (kv.dtype == MOE_F32) return items >= 64 ? 8 : 4;
    const int row_bytes = row_bytes_of(kv);
    if (row_bytes > 128) return items >= 64 ? 8 : 6;
    return items >= 256 ? 16 : items >= 128 ? 12 : items >= 64 ? 8 : 6;
}
// Items from which each gets a wave and not a block, by the most tokens an item can have.  A block's other waves have nothing to do in short
// items but are waited for, and hold its place.  us with a block / a wave for each, ragged lengths:
//   64 heads of 64, bf16, 2560 items:    32 tokens 13.8 / 8.1, 128 17.2 / 13.3, 256 21.3 / 20.6, 500 32.6 / 36.4; 10240 items: 500 115.4 / 111.7
//   64 heads of 128, bf16, 10240 items:  32 146.4 / 50.4, 128 166.3 / 79.8, 256 198.8 / 125.0, 500 275.4 / 215.5
//   32 over 8 of 128, bf16, 320 items:   32 9.6 / 6.3, 128 9.7 / 9.4, 256 10.7 / 13.7
//   12 over 4 of 80, fp32, 640 items:    32 20.3 / 9.8, 128 22.3 / 18.6, 256 28.3 / 29.8
long least_alone(long tokens) { return tokens <= 32 ? 320 : tokens <= kUnit ? 640 : tokens <= 2 * kUnit ? 1024 : tokens <= 4 * kUnit ? 4096 : 1L << 40; }
Plan plan_of(const moe_kv_cfg& kv, const moe_attn_cfg& c, int compute_units) {
    const long room = static_cast<long>(c.table_pages) * kv.page_size;
    const long longest = c.window > 0 ? std::min(room, c.window + 15L) : room, units = (longest + kUnit - 1) / kUnit;
    const long items = static_cast<long>(c.B) * kv.heads * chunks_of(kv, c);
    Plan p;
    p.alone = items >= least_alone(longest);
    p.is_short = p.alone || units <= whole_units(kv, items);
    // Blocks per compute unit: one leaves fewer parts, two fill the gaps between items where rows are short and items many.  us with one / two, full
    // batches (ragged ones):
    //   64 over 8 of 64, e4m3:       64 x 2080 41.3 / 33.8 (31.2 / 26.2), 256 x 4000 262 / 233 (148 / 116), but 32 x 4000 37.3 / 39.8 (28.1 / 27.2)
    //   32 over 8 of 32, bf16:       64 x 4000 58.6 / 54.2 (40.5 / 36.2);   1 x 20000 14.8 / 15.8
    //   32 over 8 of 64, bf16:       64 x 4000 124.9 / 87.4 (50.0 / 51.4), 256 x 4000 325 / 327 (173 / 175)
    //   64 heads of 64, bf16:        40 x 4000 414 / 400 (202 / 205);   fp32 cache: 40 x 1024 212 / 213 (119 / 125)
    const int per_unit = kv.head_dim <= 64 && row_bytes_of(kv) <= 128 && items >= 2 * kMaxUnits ? 2 : 1;
    p.workers = static_cast<int>(std::min(units * items, static_cast<long>(per_unit) * std::min(compute_units, kMaxUnits)));
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
    a.chunks = chunks_of(kv, c);
    a.items = a.heads * a.chunks;
    const int per = a.dim / Layout<CACHE, DIM>::kPiece;
    a.over_row = (65536 + per - 1) / per;
    a.item_rows = std::min(16 * NT, a.group);
    if (p.alone) {
        hipLaunchKernelGGL((attn_wave_kernel<F32, CACHE, DIM, NT>), dim3((a.B * a.items + 3) / 4), dim3(256), 0, s, a);
        MOE_LAUNCH_CHECK("attn_wave_kernel");
        return MOE_OK;
    }
    if (p.is_short) {
        hipLaunchKernelGGL((attn_short_kernel<F32, CACHE, DIM, NT>), dim3(a.B * a.heads * a.chunks), dim3(256), 0, s, a);
        MOE_LAUNCH_CHECK("attn_short_kernel");
        return MOE_OK;
    }
    hipLaunchKernelGGL((attn_kernel<F32, CACHE, DIM, NT>), dim3(p.workers), dim3(256), 0, s, a, 1.0 / p.workers);
    MOE_LAUNCH_CHECK("attn_kernel");
    if (a.B * a.items >= p.workers) hipLaunchKernelGGL((attn_join_kernel<F32, 1>), dim3(p.workers, (a.item_rows + 3) / 4), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_join_kernel<F32, 4>), dim3(p.workers, a.item_rows), dim3(256), 0, s, a);
    MOE_LAUNCH_CHECK("attn_join_kernel");
    return MOE_OK;
}

template <bool F32, int CACHE>
int for_sizes(const moe_kv_cfg& kv, const moe_attn_cfg& c, Attn& a, hipStream_t s) {
    if constexpr (!F32)
        if (columns_of(kv, a.group) == 2) return a.dim <= 64 ? launch<F32, CACHE, 64, 2>(kv, c, a, s) : launch<F32, CACHE, 128, 2>(kv, c, a, s);
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
    a.chunks = a.items = a.item_rows = a.over_row = 0;                        // set where the column tiles are chosen
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
