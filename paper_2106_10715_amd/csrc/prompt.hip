// Attention of many new tokens per sequence over a paged cache of keys and values.
//
// For query row n (a token and a query head) over the keys t of its stretch:  out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(l_t log2 e - m), with a running m,
// one pass over the keys.  The rows of a sequence are its new tokens' query heads of one key head, token by token: a block takes 32 of them for each of its
// waves, so that all heads of a group read a key once, and goes through the keys in tiles that it keeps in LDS, the next one on its way in registers.
//
// Both products are matrix instructions of 32 x 32 with the query rows as columns:
//   S^T[key, row] = K Q^T,     O^T[dim, row] += V^T P^T.
// A lane's sums S are, of its row, the keys 8 a + 4 (lane / 32) + b, a and b from 0 to 3: what the second product wants of P^T in that lane, if V^T is given with
// its keys in the same order.  So P never leaves its lane.  In 16 bits V^T comes from LDS by reads that turn blocks of 4 keys x 16 columns; in fp32 an operand
// is one number and the order is that of the reads.
//
// Bound by the matrix pipes where sequences are long and scores plain (16384 tokens, 32 heads over 8 of 128: 1.95 ms, 1.13 PFLOP/s; the pipes are busy for 64 % of a
// clock that the card lowers to 1.6 GHz meanwhile).  Elsewhere no pipe is full: at 64 columns a weight has as many cycles of exponential, bias and rounding as of products
// (8 x 2048 tokens, 64 heads of 64, a table of biases: 240 us, vector instructions issue in 55 % of the cycles, products in 22 %; of its cycles a wave issues in 45 %, waits
// for its turn in 21 % and for data or a barrier in 34 %; 8192 tokens in documents, 16 heads of 256, capped: 212 us, 57 % and 27 %; 42, 27 and 31 %).  Few rows over a long
// cache are bound by making their tiles (16 x 33 tokens after 8000 in e4m3: 148 us, 1.8 TB/s).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "convert.h"
#include "scores.h"

namespace moe {

// What the objects that this file is compiled to share (PROMPT_PART: 0 and 1 16-bit activations without and with scores of their own, 2 and 3 fp32).
namespace prompt {

struct Prompt {
    const void* q;
    long q_stride;
    const char *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *table, *lens, *starts, *first, *end;
    void* out;
    float* lse;
    int tokens, B, heads, group, dim, pages, page_bits, table_pages, window;
    int parts;                              // stretches that an item's keys are cut into, each a block's
    float *part_o, *part_ml;                // [parts][tokens * query heads][dim], [parts][tokens * query heads][2]: unscaled sums; their maximum and weight (-1: no sums)
    float scale;                            // times log2 e
    ScoreArgs scores;
};

// How a call is cut.
struct Plan {
    int dim, waves, rows;                   // the kernel's columns, a block's waves and rows
    long tiles;                             // of rows, at most (a sequence's last may not be full)
    int parts;
};

int launch_bf16(const Prompt& a, const Plan& p, int cache, hipStream_t s);
int launch_bf16_scored(const Prompt& a, const Plan& p, int cache, hipStream_t s);
int launch_f32(const Prompt& a, const Plan& p, int cache, hipStream_t s);
int launch_f32_scored(const Prompt& a, const Plan& p, int cache, hipStream_t s);

}  // namespace prompt

namespace {

using prompt::Plan;
using prompt::Prompt;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kSlack = 8.f;               // the running maximum is raised only where a logit passes it by more than this (as a power of two)

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int wave_min(int v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v = min(v, __shfl_xor(v, o));
    return uniform(v);
}
__device__ inline int wave_max(int v) { return -wave_min(-v); }
// A barrier for what lies in LDS: loads from memory stay on their way across it.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// Over the two lanes that hold the same row.
__device__ inline float halves_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float halves_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// How a block of WAVES waves holds its tiles.
template <bool F32, int CACHE, int DIM, int WAVES>
struct Shape {
    // Rows of over 128 columns have two waves, which both make their weights and have half of the columns of O each: with all of them a 16-bit wave has no room
    // in 256 registers, and with 512 the compiler moves O from accumulation registers and back in every tile (8192 tokens in documents, 16 heads, capped: 328 us, so, otherwise as it was then, 280);
    // in fp32 it would keep some in scratch memory.
    static constexpr int kShare = DIM > 128 ? 2 : 1;
    static constexpr int kThreads = 64 * WAVES, kRows = 32 * WAVES / kShare;
    static constexpr int kKeys = DIM > 128 ? 32 : 64;                               // keys of a tile
    static constexpr int kBlocks = kKeys / 32, kColumns = DIM / 32 / kShare;        // S in 32 keys, O of a wave in 32 columns
    static constexpr int kPerWord = F32 ? 1 : 2;                                    // weights in a register
    static constexpr bool kTurns = WAVES == 8;                                      // two waves of the block share a SIMD: one multiplies while the other weighs
    static constexpr int kDeep = kTurns ? 3 : 2;                                    // tiles in LDS
    static constexpr int kBias = F32 || DIM > 64 ? 2240 : 4096;                     // biases in LDS, a block's share of it left
    static constexpr int kWidth = F32 ? 4 : 2, kCached = CACHE == MOE_F32 ? 4 : CACHE == MOE_BF16 ? 2 : 1;
    static constexpr int kRowBytes = DIM * kWidth, kPieces = kRowBytes / 16;        // a row in LDS
    static constexpr int kFrom = DIM * kCached / 16;                                // 16-byte pieces of a row as it comes
    static constexpr int kTo = kWidth / kCached;                                    // of which each makes so many in LDS
    static constexpr int kLoads = kKeys * kFrom / kThreads;
    static constexpr int kTile = kKeys * kRowBytes;                                 // bytes
    static_assert(64 / kFrom <= 16 && kLoads * kThreads == kKeys * kFrom, "a load of a wave lies in one run of 16 tokens, and all waves load as much");
    static constexpr int kStep = kThreads / kFrom;                                  // rows from a lane's load to its next
    static_assert(kThreads % kFrom == 0 && kStep % 4 == 0, "a lane's loads have the same piece of their rows");
};

// The item a block works on: a sequence, some of its rows, and the keys they see.
struct Item {
    int b, rows;                            // the sequence; where the block's rows end
    int row0, token0, place0;               // the block's first row; the sequence's first token in q, and its place
    int len, part;
};

// Tile `index` from the end of the list of all sequences' tiles of `rows` rows; false: there is none.  64 sequences at a time, the last first.
__device__ inline bool find(const Prompt& a, int index, int rows, Item& it) {
    const int lane = threadIdx.x % 64;
    int before = 0;
    for (int b0 = a.B - 1; b0 >= 0; b0 -= 64) {
        const int b = b0 - lane;
        int s = 0, n = 0, len = 0;
        if (b >= 0) {
            s = min(max(a.starts[b], 0), a.tokens);
            n = max(min(max(a.starts[b + 1], 0), a.tokens) - s, 0);
            len = a.lens[b];
        }
        const int tiles = (n * a.group + rows - 1) / rows;                          // (tokens * group < 2^31)
        int upto = tiles;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned long long found = __ballot(before + upto > index);
        if (found != 0) {
            const int at = __builtin_ctzll(found);
            it.b = b0 - at;
            const int tile = before + __shfl(upto, at) - 1 - index;                 // of the sequence
            const int new_tokens = __shfl(n, at), all = new_tokens * a.group, of = (all + rows - 1) / rows;
            const int each = ((all + of - 1) / of + 31) & ~31;                      // as many in each of the sequence's tiles, in whole waves
            it.row0 = uniform(min(tile * each, all));
            it.rows = uniform(min(tile * each + each, all));
            it.token0 = uniform(__shfl(s, at));
            it.b = uniform(it.b);
            it.len = uniform(min(max(__shfl(len, at), 0), a.table_pages << a.page_bits));
            it.place0 = it.len - uniform(new_tokens);
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

// The keys [lo, hi) that a token sees; lo = hi where there are none.
__device__ inline void stretch_of(const Prompt& a, const Item& it, int token, int& lo, int& hi) {
    const int place = it.place0 + token;
    lo = a.first != nullptr ? max(a.first[it.token0 + token], 0) : 0;
    hi = min(a.end != nullptr ? a.end[it.token0 + token] : place + 1, it.len);
    if (a.window > 0) lo = max(lo, place - a.window + 1);
    hi = max(hi, lo);
}

// SCORED: scores may be capped or get a bias by distance.  PARTS: an item's keys may be cut, and the sums are left for the join.
template <bool F32, int CACHE, int DIM, int WAVES, bool SCORED, bool PARTS>
struct Block {
    using H = Shape<F32, CACHE, DIM, WAVES>;
    static constexpr bool kScaled = CACHE == MOE_E4M3 && !F32;                      // keys and values have scales, which their products do not
    static constexpr bool kRowScales = CACHE == MOE_E4M3 && F32;                    // their rows are multiplied with them
    struct Lds {
        __attribute__((aligned(256))) char k[H::kDeep][H::kTile], v[H::kDeep][H::kTile];
        float ks[H::kDeep][H::kKeys], vs[H::kDeep][H::kKeys];                                    // kScaled: scales of the keys, times a.scale, and of the values, a tile ahead of them
        // Values that are not finite lie in v as zeros.  odd: 1 + the first key of a tile that has any; up, down: the bits of a piece's elements that
        // were infinity or NaN, and -infinity or NaN.
        int odd[H::kDeep];
        __attribute__((aligned(16))) unsigned char up[H::kDeep][H::kKeys][H::kPieces], down[H::kDeep][H::kKeys][H::kPieces];
        float bias[SCORED ? H::kBias : 1];                                          // the group's biases times log2 e, if there is room for them, their ends repeated
    };
    // A wave's rows are of up to 32 neighbouring tokens: a tile that has a distance within the biases has none that is further outside of them than this.
    static constexpr int kPad = 100;
    const Prompt& a;
    Lds& lds;
    const Item& it;
    int head, lane, wave;                                                           // key head
    int wave_rows, wave_column;                                                     // a wave's first row in the block, and its first 32 columns of O
    int width;                                                                      // a head's biases in LDS
    bool tabled;                                                                    // whether they are there
    int first, end, all_from, all_to;                                               // keys that some of the block's rows see; that all of them see

    // ---- a tile from the cache to LDS ----
    u32x4 k_raw[H::kLoads], v_raw[H::kLoads];
    float k_scale[F32 ? H::kLoads : 1], v_scale[F32 ? H::kLoads : 1];               // e4m3: of the rows, or (16-bit products) of key `lane`
    int from;                                                                       // of this lane: bytes from its wave's first row
    int at_row, at_piece;                                                           // of this lane: row and piece (as it comes) of its first load
    uint32_t stale;                                                                 // the buffers, by bits, for which the wave has noted values that are not finite

    // Pieces of a row lie in LDS at places that differ from row to row, so that rows of a column are in different banks: a column of K is read 16 bytes by row,
    // of V in 64 bytes of four rows.  A piece's number and the row's change of it are combined by exclusive or, so that from one piece's place the others' follow.
    __device__ static int k_place(int row, int piece) { return row * H::kRowBytes + 16 * (piece ^ (H::kPieces >= 16 ? row & 15 : (row >> 1) & 7)); }
    __device__ static int v_place(int row, int piece) {
        if constexpr (F32) return row * H::kRowBytes + 16 * piece;
        else return row * H::kRowBytes + 16 * (piece ^ (H::kPieces >= 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1)));
    }
    // What lies in LDS from the beginning.
    __device__ void set_up() {
        if (threadIdx.x < H::kDeep) lds.odd[threadIdx.x] = 0;
        stale = 0;
        static_assert(sizeof(lds.up) % 16 == 0, "cleared 16 bytes at a time");
        for (int i = threadIdx.x; i < static_cast<int>(sizeof(lds.up) / 16); i += H::kThreads) {
            reinterpret_cast<u32x4*>(lds.up)[i] = u32x4{0, 0, 0, 0};
            reinterpret_cast<u32x4*>(lds.down)[i] = u32x4{0, 0, 0, 0};
        }
        if constexpr (SCORED)
            if (tabled)
                for (int i = threadIdx.x; i < a.group * width; i += H::kThreads) {
                    const int h = i / width, d = i - h * width - kPad;
                    lds.bias[i] = a.scores.bias[static_cast<long>(head * a.group + h) * (width - 2 * kPad) + min(max(d, 0), width - 2 * kPad - 1)] * kLog2E;
                }
    }
    __device__ void lay_out() {
        if constexpr (SCORED) {
            width = a.scores.back + a.scores.ahead + 1 + 2 * kPad;
            tabled = a.scores.bias != nullptr && static_cast<long>(a.group) * width <= H::kBias;
        }
        const int row_bytes = a.dim * H::kCached, i = 64 * wave + lane;
        at_row = i / H::kFrom;
        at_piece = i % H::kFrom;                                                    // (the same in all loads)
        from = 16 * at_piece < row_bytes ? (lane / H::kFrom) * row_bytes + 16 * at_piece : 0x7fffff00;
    }
    // Where the rows of the wave's loads begin, looked up for kAsked tiles at once: lane kSlots s + j has load j of the s-th of them.
    static constexpr int kSlots = H::kLoads <= 1 ? 1 : H::kLoads <= 2 ? 2 : H::kLoads <= 4 ? 4 : 8, kAsked = 64 / kSlots;
    int ids, own_id;                                                                // the pages of the next kAsked tiles; kScaled, the first wave: of key `lane` of the next tile
    uint32_t held[2], held4[kRowScales ? 2 : 1];                                    // where the rows of the present ones lie, in bytes; and their scales
    struct Rows {
        uint32_t lo[H::kLoads], hi[H::kLoads], lo4[kRowScales ? H::kLoads : 1], hi4[kRowScales ? H::kLoads : 1];
    };
    __device__ static uint64_t both(uint32_t lo, uint32_t hi) { return static_cast<uint64_t>(hi) << 32 | lo; }
    __device__ long row_of(int id, int t) const {
        return ((static_cast<long>(min(max(id, 0), a.pages - 1)) * a.heads + head) << a.page_bits) + (t & ((1 << a.page_bits) - 1));
    }
    __device__ int page_of(int t) const { return a.table[static_cast<long>(it.b) * a.table_pages + (min(t, end - 1) >> a.page_bits)]; }
    __device__ int asked(int t0) const { return t0 + lane / kSlots * H::kKeys + (lane % kSlots * H::kThreads + 64 * wave) / H::kFrom; }
    __device__ void locate(int t0, uint32_t index, Rows& r) {                       // index: of the tile, from the first
        if (index % kAsked == 0) {
            const long row = row_of(ids, asked(t0)), bytes = row * (a.dim * H::kCached);
            held[0] = static_cast<uint32_t>(bytes);
            held[1] = static_cast<uint32_t>(bytes >> 32);
            if constexpr (kRowScales) {
                held4[0] = static_cast<uint32_t>(4 * row);
                held4[1] = static_cast<uint32_t>(4 * row >> 32);
            }
            ids = page_of(asked(t0 + kAsked * H::kKeys));
        }
#pragma unroll
        for (int j = 0; j < H::kLoads; ++j) {
            const int from_lane = (index % kAsked) * kSlots + j;
            r.lo[j] = __builtin_amdgcn_readlane(held[0], from_lane);
            r.hi[j] = __builtin_amdgcn_readlane(held[1], from_lane);
            if constexpr (kRowScales) {
                r.lo4[j] = __builtin_amdgcn_readlane(held4[0], from_lane);
                r.hi4[j] = __builtin_amdgcn_readlane(held4[1], from_lane);
            }
        }
    }
    // Requests keys [t0, t0 + kKeys) of one side; zeros outside of [first, end), which a WHOLE tile does not reach.
    template <bool WHOLE>
    __device__ void load(const char* pages, const float* scales, const Rows& r, int t0, u32x4 (&raw)[H::kLoads], float (&scale)[F32 ? H::kLoads : 1]) const {
        const int row_bytes = a.dim * H::kCached;
#pragma unroll
        for (int j = 0; j < H::kLoads; ++j) {
            const int t = t0 + (j * H::kThreads + 64 * wave) / H::kFrom + lane / H::kFrom;
            const bool there = WHOLE || (t >= first && t < end);
            const auto rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pages) + both(r.lo[j], r.hi[j]), 0, 16 * row_bytes, 0x00027000);
            raw[j] = __builtin_amdgcn_raw_buffer_load_b128(rows, there ? from : 0x7fffff00, 0, 0);
            if constexpr (kRowScales) {
                const auto from4 = reinterpret_cast<const char*>(scales) + both(r.lo4[j], r.hi4[j]);
                scale[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from4), 0, 64, 0x00027000),
                                                                                there ? 4 * (lane / H::kFrom) : 0x7fffff00, 0, 0));
            }
        }
    }
    template <bool WHOLE>
    __device__ void load_k(const Rows& r, int t0) {
        load<WHOLE>(a.k_pages, a.k_scales, r, t0, k_raw, k_scale);
        if constexpr (kScaled)                                                      // the scales of keys and values, both a tile ahead: weights are made with them
            if (wave == 0) {
                const int t = t0 + lane;
                const long row = row_of(own_id, t);
                const bool there = WHOLE || (t >= first && t < end);
                k_scale[0] = there ? a.k_scales[row] : 0.f;
                v_scale[0] = there ? a.v_scales[row] : 0.f;
                own_id = page_of(t + H::kKeys);
            }
    }
    // One piece as it came in the form of the products.
    __device__ static void widen(const u32x4& raw, float scale, u32x4 (&out)[H::kTo]) {
        if constexpr (H::kTo == 1) {
            out[0] = raw;
        } else if constexpr (!F32) {                                                // e4m3 values are bf16 values
#pragma unroll
            for (int c = 0; c < 8; ++c)
                out[c / 4][c % 4] = __builtin_bit_cast(uint32_t, c % 2 == 0 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[c / 2], 1.f, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[c / 2], 1.f, true));
        } else if constexpr (CACHE == MOE_BF16) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                out[c / 2][2 * (c % 2)] = raw[c] << 16;
                out[c / 2][2 * (c % 2) + 1] = raw[c] & 0xffff0000u;
            }
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float v[4];
                from_e4m3x4(raw[c], v);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[c][e] = __float_as_uint(v[e] * scale);
            }
        }
    }
    // Put what came into buffer `to`.
    __device__ void store_k(int to) {
        char* const k = lds.k[to];
#pragma unroll
        for (int j = 0; j < H::kLoads; ++j) {
            u32x4 out[H::kTo];
            widen(k_raw[j], F32 ? k_scale[F32 ? j : 0] : 1.f, out);
#pragma unroll
            for (int c = 0; c < H::kTo; ++c) *reinterpret_cast<u32x4*>(k + (k_place(at_row, at_piece * H::kTo + c) ^ 16 * (j * H::kStep & 15)) + j * H::kStep * H::kRowBytes) = out[c];
        }
        if constexpr (kScaled)
            if (wave == 0 && lane < H::kKeys) {
                lds.ks[to][lane] = k_scale[0] * a.scale;
                lds.vs[to][lane] = v_scale[0];
            }
    }
    // `edge`: some row does not see some of these keys, so that values that are not finite are looked for.
    __device__ void store_v(int to, int t0, bool edge) {
        if (edge) {
            uint32_t most = 0;                                                      // (bf16: of two, side by side)
#pragma unroll
            for (int j = 0; j < H::kLoads; ++j) {
                u32x4 out[H::kTo];
                widen(v_raw[j], F32 ? v_scale[F32 ? j : 0] : 1.f, out);
#pragma unroll
                for (int c = 0; c < 4 * H::kTo; ++c) {
                    const uint32_t u = out[c / 4][c % 4];
                    if constexpr (F32) {
                        most = max(most, u & 0x7fffffffu);
                    } else {
                        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
                        most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, u & 0x7fff7fffu)));
                    }
                }
            }
            const bool odd = most >= 0x7f800000u || (!F32 && (most & 0xffffu) >= 0x7f80u);
            if (__any(odd) || (stale >> to & 1) != 0) {
                put_v<true>(to, t0);
                stale = (stale & ~(1u << to)) | (__any(odd) ? 1u << to : 0u);
                return;
            }
        }
        put_v<false>(to, t0);
    }
    template <bool ODD>
    __device__ void put_v(int to, int t0) {
        char* const v = lds.v[to];
#pragma unroll
        for (int j = 0; j < H::kLoads; ++j) {
            u32x4 out[H::kTo];
            widen(v_raw[j], F32 ? v_scale[F32 ? j : 0] : 1.f, out);
            if constexpr (ODD)
#pragma unroll
                for (int c = 0; c < H::kTo; ++c) clear(to, t0, at_row + j * H::kStep, at_piece * H::kTo + c, out[c]);
#pragma unroll
            for (int c = 0; c < H::kTo; ++c) *reinterpret_cast<u32x4*>(v + v_place(at_row, at_piece * H::kTo + c) + j * H::kStep * H::kRowBytes) = out[c];
        }
    }
    // Takes what is not finite out of a piece of V, and notes it.
    __device__ void clear(int to, int t0, int row, int piece, u32x4& u) {
        uint32_t up = 0, down = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int part = 0; part < (F32 ? 1 : 2); ++part) {
                const uint32_t bits = F32 ? u[c] : part == 0 ? u[c] << 16 : u[c] & 0xffff0000u;
                const float f = __uint_as_float(bits);
                const bool more = !(f < INFINITY), less = !(f > -INFINITY);
                const int bit = F32 ? c : 2 * c + part;
                up |= more ? 1u << bit : 0u;
                down |= less ? 1u << bit : 0u;
                if (more || less) u[c] &= F32 ? 0u : part == 0 ? 0xffff0000u : 0xffffu;
            }
        lds.up[to][row][piece] = static_cast<unsigned char>(up);
        lds.down[to][row][piece] = static_cast<unsigned char>(down);
        if ((up | down) != 0) lds.odd[to] = t0 + 1;
    }

    // ---- a wave's 32 rows ----
    static constexpr int kSteps = F32 ? DIM / 8 : DIM / 16;                         // pieces of Q that a lane holds, 16 bytes each
    u32x4 q[kSteps];
    f32x16 o[H::kColumns];
    float m, l;
    int lo, hi, place, own;                                                         // of this lane's row; own: its query head in the group
    int wave_first, wave_end, whole_from, whole_to;                                 // keys that some of the wave's rows see; that all of them see
    HeadScores hs;

    // A lane's part of S^T of a tile, as logits.
    __device__ void products(int buf, f32x16 (&s)[H::kBlocks]) const {
        const int at = buf * H::kTile + k_place(lane % 32, lane / 32);
#pragma unroll
        for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            if (F32 && 8 * st >= a.dim) break;
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb) {
                const u32x4 u = *reinterpret_cast<const u32x4*>(lds.k[0] + (at ^ (32 * st)) + 32 * kb * H::kRowBytes);
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(u[c]), __uint_as_float(q[st][c]), s[kb], 0, 0, 0);
                } else {
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u), __builtin_bit_cast(bf16x8, q[st]), s[kb], 0, 0, 0);
                }
            }
        }
    }
    // The key of sum i of a lane in block kb, from the tile's first.
    __device__ static constexpr int key_of(int kb, int i) { return 32 * kb + 8 * (i / 4) + i % 4; }

    // What a lane reads of V for 16 keys (bf16) and 32 columns; at: v_at.
    __device__ int v_at(int buf) const { return buf * H::kTile + v_place(4 * (lane / 32) + (lane % 16) / 4, 0) + 32 * ((lane / 16) % 2) + 8 * (lane % 4); }
    __device__ bf16x8 turned(int at, int ks, int column) const {
        const char* const from = lds.v[0] + (at ^ (64 * column)) + 16 * ks * H::kRowBytes;
        typedef __attribute__((address_space(3))) i16x4* Place;
        const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(from)), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(from + 8 * H::kRowBytes));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // In 16 bits a weight is one bf16 value, rounded after it has entered the sum of weights: off by 2^-8 of itself at most, as an output by its own rounding.  Outputs
    // are off by 0.0018 to 0.0024 of their norm, with fp32 weights by 0.0017; a second part would be half again as many products (heads of over 128: a third).
    struct Weights {
        uint32_t u[H::kBlocks][16 / H::kPerWord];
        __device__ void set(int kb, int i, float x, float y) { u[kb][i / H::kPerWord] = F32 ? __float_as_uint(x) : to_bf16x2(x, y); }
        __device__ void clear() {
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16 / H::kPerWord; ++i) u[kb][i] = 0;
        }
        // They are made before what follows (the compiler would move the exponentials past the barrier, to the products).
        __device__ void hold() {
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16 / H::kPerWord; ++i) asm volatile("" : "+v"(u[kb][i]));
        }
        // bf16: the operand of 16 keys
        __device__ bf16x8 keys(int ks) const { return __builtin_bit_cast(bf16x8, u32x4{u[ks / 2][4 * (ks % 2)], u[ks / 2][4 * (ks % 2) + 1], u[ks / 2][4 * (ks % 2) + 2], u[ks / 2][4 * (ks % 2) + 3]}); }
    };
    // The weights of the keys of the tile at t0 from their products, as operands of the next product.  The sums of earlier tiles are brought to the maximum.
    // PLAIN: the wave's rows see all of them.
    template <bool PLAIN>
    __device__ void weigh(f32x16 (&s)[H::kBlocks], Weights& w, int buf, int t0) {
        const int h = lane / 32;
        const bool edge = !PLAIN && (t0 < whole_from || t0 + H::kKeys > whole_to);
        float mult = kScaled ? 1.f : a.scale, shift = 0.f;
        if constexpr (kScaled)
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 each = *reinterpret_cast<const f32x4*>(&lds.ks[buf][key_of(kb, i) + 4 * h]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[kb][i + c] *= each[c];
                }
        if constexpr (SCORED) score(s, t0, mult, shift);
        if (edge)
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = t0 + key_of(kb, i) + 4 * h;
                    if (static_cast<uint32_t>(t - lo) >= static_cast<uint32_t>(hi - lo)) s[kb][i] = -INFINITY;
                }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
        top = halves_max(fmaf(top, mult, shift));
        if (__any(top > m + kSlack)) {                                              // (always where m is still -inf and some key counts)
            const float now = fmaxf(m, top), keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= keep;
#pragma unroll
            for (int c = 0; c < H::kColumns; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[c][i] *= keep;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float sum[4];
#pragma unroll
        for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float p[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    p[c] = __builtin_amdgcn_exp2f(fmaf(s[kb][i + c], mult, shift - ref));
                    sum[c] = kb == 0 && i == 0 ? p[c] : sum[c] + p[c];
                }
                if constexpr (kScaled) {                                            // (a scale that is not finite may be that of a key the row does not see)
                    const f32x4 each = *reinterpret_cast<const f32x4*>(&lds.vs[buf][key_of(kb, i) + 4 * h]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) p[c] = edge && p[c] == 0.f ? 0.f : p[c] * each[c];
                }
#pragma unroll
                for (int c = 0; c < 4; c += H::kPerWord) w.set(kb, i + c, p[c], p[c + H::kPerWord - 1]);
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        asm volatile("" : "+v"(l));
        w.hold();
    }
    // The order of the products of a tile: reads from LDS some of them ahead.
    template <bool NEXT, bool THIS>
    __device__ static void schedule() {
        constexpr int kRead = 0x100, kProduct = 0x008, kAhead = 6;
        constexpr int kFirst = NEXT ? kSteps * H::kBlocks : 0, kSecond = THIS ? 2 * H::kBlocks * H::kColumns : 0;
        if constexpr (!F32) {
            __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
            for (int i = 0; i < kFirst - kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
            }
#pragma unroll
            for (int i = kFirst > kAhead ? kFirst - kAhead : 0; i < kFirst + kSecond; ++i) {
                __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
            }
        }
    }

    // O^T += V^T P^T.
    __device__ void values(int buf, const Weights& w) {
        if constexpr (F32) {
            const float* const v = reinterpret_cast<const float*>(lds.v[buf]) + 4 * (lane / 32) * DIM + 32 * wave_column + lane % 32;
#pragma unroll
            for (int c = 0; c < H::kColumns; ++c) {
                if (32 * (wave_column + c) >= a.dim) break;
#pragma unroll
                for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[key_of(kb, i) * DIM + 32 * c], __uint_as_float(w.u[kb][i / H::kPerWord]), o[c], 0, 0, 0);
            }
        } else {
            const int at = v_at(buf);
#pragma unroll
            for (int ks = 0; ks < 2 * H::kBlocks; ++ks)
#pragma unroll
                for (int c = 0; c < H::kColumns; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(turned(at, ks, wave_column + c), w.keys(ks), o[c], 0, 0, 0);
        }
    }
    // The column of sum i of a lane in block c.
    __device__ int column_of(int c, int i) const {
        return 32 * (wave_column + c) + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
    }
    // Values that are not finite under rows of which some may not see them: a weight of zero times such a value would be no number, so the product has zeros in
    // their places, and the rows that see them get them here.
    __device__ void add_odd(int buf, int t0) {
        constexpr int kEach = 16 / H::kWidth;
#pragma unroll 1
        for (int key = 0; key < H::kKeys; ++key) {
            const bool counts = static_cast<uint32_t>(t0 + key - lo) < static_cast<uint32_t>(hi - lo);
            int from = column_of(0, 0);
            asm("" : "+v"(from));                                                   // (so that no places of this rare case are kept in registers)
#pragma unroll
            for (int c = 0; c < H::kColumns; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int column = from + 32 * c + 2 * i;
                    const uint32_t up = lds.up[buf][key][column / kEach] >> column % kEach, down = lds.down[buf][key][column / kEach] >> column % kEach;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (counts && up >> e & 1) o[c][i + e] += INFINITY;
                        if (counts && down >> e & 1) o[c][i + e] -= INFINITY;
                    }
                }
        }
    }

    // Logits are then s * mult + shift.
    __device__ void score(f32x16 (&s)[H::kBlocks], int t0, float& mult, float& shift) const {
        const int d0 = place - t0 - 4 * (lane / 32);                                // the distance of the lane's first key
        if (a.scores.cap > 0.f) {
#pragma unroll
            for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 8) {
                    float x[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) x[c] = s[kb][i + c] * mult;
                    cap_scores(a.scores, x);
#pragma unroll
                    for (int c = 0; c < 8; ++c) s[kb][i + c] = x[c];
                }
            mult = 1.f;
        }
        if (a.scores.slopes != nullptr) {
            const float slope = hs.slope / mult;
            if (__all(d0 >= H::kKeys - 1)) {                                        // all of the keys before the rows: |d| = d0 - key
                shift = -hs.slope * static_cast<float>(d0);
#pragma unroll
                for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(slope, static_cast<float>(key_of(kb, i)), s[kb][i]);
            } else {
#pragma unroll
                for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(-slope, fabsf(static_cast<float>(d0 - key_of(kb, i))), s[kb][i]);
            }
        }
        if (a.scores.bias != nullptr) {
            const bool behind = __all(d0 - (H::kKeys - 1) >= a.scores.back), ahead = __all(d0 <= -a.scores.ahead);
            if (behind || ahead) {
                shift += behind ? hs.last : hs.first;
            } else if (tabled) {
                const float* const from = &lds.bias[own * width + d0 + a.scores.ahead + kPad - (H::kKeys - 1)];
#pragma unroll
                for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(s[kb][i], mult, from[H::kKeys - 1 - key_of(kb, i)]);
                mult = 1.f;
            } else {
                const int row = bias_row(a.scores, head * a.group + own);
#pragma unroll
                for (int kb = 0; kb < H::kBlocks; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(s[kb][i], mult, bias_at(a.scores, row, d0 - key_of(kb, i)));
                mult = 1.f;
            }
        }
    }

    // The block's rows, the keys they see, and the wave's queries.
    __device__ void begin() {
        const int tokens = (it.rows + a.group - 1) / a.group;
        const int from_token = it.row0 / a.group, to_token = tokens - 1;
        int low = 0x7fffffff, high = 0, last_low = 0, first_high = 0x7fffffff;
        for (int i = from_token + lane; i <= to_token; i += 64) {
            int x, y;
            stretch_of(a, it, i, x, y);
            last_low = max(last_low, x);
            first_high = min(first_high, x < y ? y : -1);
            if (x < y) {
                low = min(low, x);
                high = max(high, y);
            }
        }
        first = wave_min(low);
        end = wave_max(high);
        if (PARTS && first < end) {                                           // a part of the keys' tiles
            const int base = first & ~(H::kKeys - 1), tiles = (end - base + H::kKeys - 1) / H::kKeys;
            const int from = static_cast<int>(static_cast<long>(tiles) * it.part / a.parts), to = static_cast<int>(static_cast<long>(tiles) * (it.part + 1) / a.parts);
            first = max(first, base + from * H::kKeys);
            end = min(end, base + to * H::kKeys);
        }
        all_from = wave_max(last_low);
        all_to = wave_min(first_high);
        const int row = it.row0 + wave_rows + lane % 32;
        const bool real = row < it.rows;
        const int token = real ? row / a.group : tokens - 1, in_group = real ? row - token * a.group : 0;
        place = it.place0 + token;
        own = in_group;
        stretch_of(a, it, token, lo, hi);
        if (!real) {                                                                // rows past the last: as if they saw all, and not stored
            lo = 0;
            hi = 0x7fffffff;
        }
        const bool some = real && lo < hi;
        wave_first = wave_min(some ? lo : 0x7fffffff);
        wave_end = wave_max(some ? hi : 0);
        whole_from = wave_max(real ? lo : 0);
        whole_to = wave_min(some || !real ? hi : -1);
        const long at = (it.token0 + token) * a.q_stride + (static_cast<long>(head) * a.group + in_group) * a.dim;
        constexpr int kElements = 16 / H::kWidth;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            const int d = (2 * st + lane / 32) * kElements;
            q[st] = u32x4{0, 0, 0, 0};
            if (real && d < a.dim) q[st] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) + (at + d) * H::kWidth);
        }
        if constexpr (SCORED) hs.load(a.scores, head * a.group + in_group);
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < H::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    }

    __device__ void finish() {
        l = halves_sum(l);
        const int row = it.row0 + wave_rows + lane % 32, h = lane / 32;
        if (row >= it.rows) return;
        const int token = row / a.group;
        const long at = static_cast<long>(it.token0 + token) * a.heads * a.group + head * a.group + (row - token * a.group);
        constexpr bool part = PARTS;
        const float inv = part ? 1.f : l == 0.f ? 0.f : 1.f / l;
        float* const part_o = a.part_o + (static_cast<long>(it.part) * a.tokens * a.heads * a.group + at) * a.dim;
        if (h == 0 && wave_column == 0) {
            if (part) *reinterpret_cast<f32x2*>(a.part_ml + (static_cast<long>(it.part) * a.tokens * a.heads * a.group + at) * 2) = f32x2{m, first < end ? l : -1.f};
            else if (a.lse != nullptr) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        }
        if (part && first >= end) return;                                           // (a part without keys: its weight says so)
#pragma unroll
        for (int c = 0; c < H::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * (wave_column + c) + 8 * (i / 4) + 4 * h;
                if (d >= a.dim) continue;
                const f32x4 v = f32x4{o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]} * inv;
                if (part) *reinterpret_cast<f32x4*>(part_o + d) = v;
                else if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at * a.dim + d) = v;
                else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at * a.dim + d) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
            }
    }

    // A wave weighs tile t (the exponentials), then multiplies: the keys of tile t + 1, the values of tile t.  With two waves of the block on a SIMD (kTurns) the
    // second half of them, `late`, has its barrier between the two and the first half before them, so that one of the two has the matrix pipes while the other weighs:
    //     the first half           | weigh 0    multiply 0 | weigh 1    multiply 1 | ..
    //     the second half  weigh 0 | multiply 0 weigh 1    | multiply 1 weigh 2    | ..
    // Between the barriers of t and t + 1, K of t + 1 and V of t are read; the first half, weighing t, puts its share of K of t + 2 and V of t + 1 into LDS, the second
    // half, weighing t + 1, its share of K of t + 3 and V of t + 2: three buffers, and what is read after a barrier was put before it.
    // Where all waves are late, K of t + 2 and V of t + 1 are put there: two buffers, K a tile less ahead.
    __device__ void run() {
        lay_out();
        begin();
        if (first < end) {
            const bool late = !H::kTurns || wave >= 4;
            const int base = first & ~(H::kKeys - 1);
            auto edge = [&](int t0) { return t0 < all_from || t0 + H::kKeys > all_to; };
            auto mine = [&](int t0) { return t0 < end && t0 < wave_end && t0 + H::kKeys > wave_first; };
            auto after = [](int buf) { return buf == H::kDeep - 1 ? 0 : buf + 1; };
            ids = page_of(asked(base));
            own_id = kScaled ? page_of(base + lane) : 0;
            Rows rows;                                                              // of the K that is on its way
            locate(base, 0, rows);
            load_k<false>(rows, base);
            set_up();
            if constexpr (H::kTurns) load<false>(a.v_pages, a.v_scales, rows, base, v_raw, v_scale);
            lds_barrier();
            store_k(0);
            int next = base, to = 0;
            uint32_t index = 0;                                                     // the tile whose K is on its way, its number and buffer; the V on its way is that before it
            auto ask = [&](auto plain, bool v) {
                constexpr bool kPlain = decltype(plain)::value;
                if (kPlain || (v && next < end)) load<kPlain>(a.v_pages, a.v_scales, rows, next, v_raw, v_scale);
                next += H::kKeys;
                ++index;
                to = after(to);
                if (kPlain || next < end) {
                    locate(next, index, rows);
                    load_k<kPlain>(rows, next);
                }
            };
            auto put = [&](auto plain) {
                constexpr bool kPlain = decltype(plain)::value;
                const int before = next - H::kKeys;
                if (kPlain || before < end) store_v(to == 0 ? H::kDeep - 1 : to - 1, before, !kPlain && edge(before));
                if (kPlain || next < end) store_k(to);
            };
            constexpr std::false_type kAny;
            ask(kAny, !H::kTurns);
            if constexpr (H::kTurns) {
                put(kAny);
                ask(kAny, true);
            }
            lds_barrier();
            f32x16 s[H::kBlocks];
            if (mine(base)) {
                products(0, s);
                schedule<true, false>();
            }
            // Tiles at t0 from plain_from to plain_to: the wave's rows see all of it and the block's all of the tiles that are put or asked for meanwhile.
            constexpr int kLead = H::kDeep - 1;
            const int plain_from = max(max(all_from, whole_from), max(first, wave_first));
            const int plain_to = min(min(end - (kLead + 2) * H::kKeys, all_to - kLead * H::kKeys), min(whole_to - H::kKeys, wave_end - 2 * H::kKeys));
            int buf = 0, t0 = base;
            auto step = [&](auto plain) {
                constexpr bool kPlain = decltype(plain)::value;
                if (!late) lds_barrier();
                put(plain);
                ask(plain, true);
                const bool now = kPlain || mine(t0);
                Weights w;
                if (now) weigh<kPlain>(s, w, buf, t0);
                else w.clear();
                if (late) lds_barrier();
                __builtin_amdgcn_sched_barrier(0);
                const int then = after(buf);
                if (now || mine(t0 + H::kKeys)) {                                   // (both products where one would do: the other's weights are zero, or its sums not used)
                    __builtin_amdgcn_s_setprio(1);
                    products(then, s);
                    values(buf, w);
                    schedule<true, true>();
                    __builtin_amdgcn_s_setprio(0);
                }
                if (!kPlain && edge(t0) && uniform(lds.odd[buf]) == t0 + 1) add_odd(buf, t0);
                __builtin_amdgcn_sched_barrier(0);
                buf = then;
                t0 += H::kKeys;
            };
            while (t0 < end) {
                step(kAny);
#pragma unroll 1
                while (t0 >= plain_from && t0 <= plain_to) step(std::true_type());
            }
        }
        finish();
    }
};

// Waves that a SIMD has room for: with two, a wave has 256 registers.
constexpr int waves_of(bool f32) { return f32 ? 1 : 2; }

template <bool F32, int CACHE, int DIM, int WAVES, bool SCORED, bool PARTS>
__global__ __launch_bounds__(64 * WAVES, waves_of(F32)) void prompt_kernel(Prompt a) {
    using B = Block<F32, CACHE, DIM, WAVES, SCORED, PARTS>;
    __shared__ typename B::Lds lds;
    Item it;
    // the key heads first: blocks that read the same keys are a multiple of the heads apart, with eight of them on one XCD
    const int index = blockIdx.x / a.heads;
    it.part = PARTS ? index % a.parts : 0;
    if (!find(a, PARTS ? index / a.parts : index, B::H::kRows, it) || it.row0 >= it.rows) return;
    B block{a, lds, it};
    block.head = blockIdx.x % a.heads;
    block.lane = threadIdx.x % 64;
    block.wave = uniform(threadIdx.x / 64);
    block.wave_rows = 32 * (block.wave % (WAVES / B::H::kShare));
    block.wave_column = block.wave / (WAVES / B::H::kShare) * B::H::kColumns;
    block.run();
}

// Joins an item's parts: the row of a token and query head by DIM / 4 neighbouring threads, in the order of the keys.  All that have keys count, those whose
// maximum is -infinity too: logits of -infinity add zeros, logits that are all NaN leave the maximum as it was and make the row NaN, as in a call that is not cut.
template <bool F32, int DIM>
__global__ __launch_bounds__(256) void prompt_join_kernel(Prompt a) {
    const long rows = static_cast<long>(a.tokens) * a.heads * a.group, row = static_cast<long>(blockIdx.x) * (1024 / DIM) + threadIdx.x / (DIM / 4);
    const int d = 4 * (threadIdx.x % (DIM / 4));
    if (row >= rows || d >= a.dim) return;
    const int token = static_cast<int>(row / (a.heads * a.group));
    if (token < a.starts[0] || token >= a.starts[a.B]) return;
    float top = -INFINITY, weight = 0.f;
    for (int i = 0; i < a.parts; ++i) top = fmaxf(top, a.part_ml[(i * rows + row) * 2]);
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.parts; ++i) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + (i * rows + row) * 2);
        if (ml[1] < 0.f) continue;                                                  // no sums were written there
        const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
        const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + (i * rows + row) * a.dim + d);
        weight = fmaf(ml[1], f, weight);
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = fmaf(o[c], f, v[c]);
    }
    const float inv = weight == 0.f ? 0.f : 1.f / weight;
    if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + row * a.dim + d) = v * inv;
    else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + row * a.dim + d) = u32x2{to_bf16x2(v[0] * inv, v[1] * inv), to_bf16x2(v[2] * inv, v[3] * inv)};
    if (d == 0 && a.lse != nullptr) a.lse[row] = (top + __builtin_amdgcn_logf(weight)) * 0.6931471805599453f;
}

template <bool F32, int CACHE, int DIM, int WAVES, bool SCORED>
int launch(const Prompt& a, const Plan& p, hipStream_t s) {
    static_assert(Shape<F32, CACHE, DIM, WAVES>::kRows == (F32 && DIM > 128 ? 64 : WAVES == 8 && DIM <= 128 ? 256 : 128), "as plan_of says");
    const dim3 blocks(static_cast<unsigned>(p.tiles * a.heads * a.parts));
    if (a.parts == 1) {
        hipLaunchKernelGGL((prompt_kernel<F32, CACHE, DIM, WAVES, SCORED, false>), blocks, dim3(64 * WAVES), 0, s, a);
        MOE_LAUNCH_CHECK("prompt_kernel");
    } else if constexpr (WAVES == 4 || DIM > 128) {
        hipLaunchKernelGGL((prompt_kernel<F32, CACHE, DIM, WAVES, SCORED, true>), blocks, dim3(64 * WAVES), 0, s, a);
        MOE_LAUNCH_CHECK("prompt_kernel");
        const long rows = static_cast<long>(a.tokens) * a.heads * a.group, each = 1024 / DIM;
        hipLaunchKernelGGL((prompt_join_kernel<F32, DIM>), dim3(static_cast<unsigned>((rows + each - 1) / each)), dim3(256), 0, s, a);
        MOE_LAUNCH_CHECK("prompt_join_kernel");
    }
    return MOE_OK;
}

template <bool F32, int CACHE, int DIM, bool SCORED>
int for_waves(const Prompt& a, const Plan& p, hipStream_t s) {
    if constexpr (!F32 && DIM > 128) return launch<F32, CACHE, DIM, 8, SCORED>(a, p, s);
    else if constexpr (F32) return launch<F32, CACHE, DIM, 4, SCORED>(a, p, s);
    else if constexpr (DIM == 128 && !SCORED) return p.waves == 8 ? launch<F32, CACHE, DIM, 8, SCORED>(a, p, s) : launch<F32, CACHE, DIM, 4, SCORED>(a, p, s);
    else return launch<F32, CACHE, DIM, 4, SCORED>(a, p, s);
}

template <bool F32, int CACHE, bool SCORED>
int for_sizes(const Prompt& a, const Plan& p, hipStream_t s) {
    if (p.dim == 64) return for_waves<F32, CACHE, 64, SCORED>(a, p, s);
    return p.dim == 128 ? for_waves<F32, CACHE, 128, SCORED>(a, p, s) : for_waves<F32, CACHE, 256, SCORED>(a, p, s);
}

}  // namespace

namespace prompt {

#if PROMPT_PART == 0
int launch_bf16(const Prompt& a, const Plan& p, int cache, hipStream_t s) {
    return cache == MOE_BF16 ? for_sizes<false, MOE_BF16, false>(a, p, s) : for_sizes<false, MOE_E4M3, false>(a, p, s);
}
#elif PROMPT_PART == 1
int launch_bf16_scored(const Prompt& a, const Plan& p, int cache, hipStream_t s) {
    return cache == MOE_BF16 ? for_sizes<false, MOE_BF16, true>(a, p, s) : for_sizes<false, MOE_E4M3, true>(a, p, s);
}
#elif PROMPT_PART == 2
int launch_f32(const Prompt& a, const Plan& p, int cache, hipStream_t s) {
    if (cache == MOE_F32) return for_sizes<true, MOE_F32, false>(a, p, s);
    return cache == MOE_BF16 ? for_sizes<true, MOE_BF16, false>(a, p, s) : for_sizes<true, MOE_E4M3, false>(a, p, s);
}
#else
int launch_f32_scored(const Prompt& a, const Plan& p, int cache, hipStream_t s) {
    if (cache == MOE_F32) return for_sizes<true, MOE_F32, true>(a, p, s);
    return cache == MOE_BF16 ? for_sizes<true, MOE_BF16, true>(a, p, s) : for_sizes<true, MOE_E4M3, true>(a, p, s);
}
#endif

}  // namespace prompt

#if PROMPT_PART == 0
namespace {

constexpr int kUnits = 256;         // compute units, also of the plan that sizes the workspace
// Blocks of four waves, two to a compute unit, or of eight that take turns, one to a unit: these read keys half as often, but all rows of a block wait for each other,
// so that short stretches are better off with four, and where weights cost more than products nothing is gained by turns.  us with four / eight, in 16 bits if no type
// is named (ragged lengths where there are several; + n: after n cached tokens, of which the host knows what the table has room for):
//   32 heads over 8 of 128:  1 x 2048 60.8 / 60.0, 40 x 500 84 / 93, 16 x 1500 158.5 / 158.2, but 8 x 2048 139 / 136, 1 x 4096 152 / 141, 1 x 8192 549 / 506, 4 x 2048 + 8000 1157 / 1060;
//                            e4m3 1 x 16384 2335 / 2173, 8 x 4096 504 / 492;  with a cap 1 x 8192 778 / 800;  4 x 4096 in a window of 256 173 / 186, of 512 225 / 225, of 1024 325 / 314
//   64 heads over 8 of 128:  32 x 1024 349 / 355, 40 x 640 227 / 245, but 1 x 2048 86 / 81, 8 x 512 + 8000 1063 / 974;  e4m3 64 x 500 297 / 333, but 4 x 1024 + 4000 668 / 620
//   32 heads of 128:         1 x 2048 56.8 / 58.3, e4m3 8 x 1500 117 / 126, but 1 x 4096 153 / 144, e4m3 2 x 4096 177 / 161
//   64 heads of 64:          8 x 2048 176 / 208 (with a table of biases 246 / 278), 1 x 4096 177 / 188
bool in_turns(const moe_kv_cfg& kv, const Plan& p, long each, int group, long keys, bool scored) {
    return kv.dtype == MOE_BF16 && p.dim == 128 && !scored && p.parts == 1 && each >= 2048 && keys >= 1536 && each >= (keys >= 4096 ? 512L : 1536L) * group;
}
Plan plan_of(const moe_kv_cfg& kv, const moe_prompt_cfg& c, bool scored) {
    Plan p;
    const bool f32 = kv.dtype == MOE_F32;
    const int group = c.q_heads / kv.heads, sequences = std::max(1, std::min(c.B, c.tokens));
    const long rows = static_cast<long>(c.tokens) * group, each = (rows + sequences - 1) / sequences;      // of a key head; of a sequence, in the mean
    p.dim = kv.head_dim <= 64 ? 64 : kv.head_dim <= 128 ? 128 : 256;
    p.rows = f32 && p.dim > 128 ? 64 : 128;
    p.tiles = rows / p.rows + sequences;
    // Few items: their keys are cut, down to 256 of them.
    const long items = p.tiles * kv.heads, slots = (f32 || p.dim > 128 ? 1 : 2) * kUnits;
    const long room = static_cast<long>(c.table_pages) * kv.page_size, keys = c.window > 0 ? std::min(room, c.window + each / group + 64) : room;
    p.parts = static_cast<int>(std::max(1L, std::min({slots / std::max(items, 1L), keys / 256, 16L})));
    p.waves = !f32 && p.dim > 128 ? 8 : 4;
    if (in_turns(kv, p, each, group, keys, scored)) {
        p.waves = 8;
        p.rows = 256;
        p.tiles = rows / p.rows + sequences;
    }
    return p;
}
// The workspace: the parts' sums, their maxima and weights.
struct Parts {
    size_t ml, bytes;
    Parts(const moe_kv_cfg& kv, const moe_prompt_cfg& c) {
        const int parts = plan_of(kv, c, false).parts;                              // (the same for all scores)
        const size_t rows = parts == 1 ? 0 : static_cast<size_t>(parts) * c.tokens * c.q_heads;
        ml = align256(rows * kv.head_dim * 4);
        bytes = std::max(ml + align256(rows * 8), size_t(256));
    }
};

}  // namespace

size_t attn_prompt_workspace_bytes(const moe_kv_cfg& kv, const moe_prompt_cfg& c) { return Parts(kv, c).bytes; }

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
    a.window = std::min(c.window, 1 << 26);                                        // (of no effect from 2^24 + 2^22 on)
    a.scale = (c.scale > 0.f ? c.scale : 1.f / sqrtf(static_cast<float>(kv.head_dim))) * kLog2E;
    a.scores = ScoreArgs(scores, kv.dtype);
    const Plan p = plan_of(kv, c, scores.any());
    const Parts parts(kv, c);
    a.parts = p.parts;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + parts.ml);
    if (kv.dtype == MOE_BF16) return scores.any() ? prompt::launch_bf16_scored(a, p, kv.cache_dtype, s) : prompt::launch_bf16(a, p, kv.cache_dtype, s);
    return scores.any() ? prompt::launch_f32_scored(a, p, kv.cache_dtype, s) : prompt::launch_f32(a, p, kv.cache_dtype, s);
}
#endif

}  // namespace moe
