// Rotary positions: pairs of a head's columns turned by angles that grow with the token's place.
//
// Bound by reading and writing the rows once (16384 tokens of 32 + 8 heads of 128 in bf16: 58 us, 5.8 TB/s both ways together).  All heads of a token turn by the same angles, so a block takes some tokens, computes each
// (token, pair)'s sine and cosine once, into LDS, and turns all of their heads with them.  Angles are fp64 products, of which only the part
// of a turn is kept: a place of a million times a frequency has, in fp32, no digit left that says where on the circle it is.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "convert.h"

namespace moe {
namespace {

constexpr int kThreads = 256;

struct Rope {
    RopeSide q, k;
    const int32_t* positions;
    const double* freqs;
    int n, dim, rot, tokens, heads, pieces, row_pieces;      // tokens of a block, heads of both sides; pieces of a row that are turned, and all of them
    uint32_t over_heads;                                     // 2^32 / heads, rounded up (more than one head): a quotient of numbers below 2^20 is a product's upper half
    float amplitude;
};

// V elements of a row, in registers and memory.
template <bool BF16, int V>
struct Piece {
    static constexpr int kBytes = V * (BF16 ? 2 : 4);
    typedef uint32_t Words __attribute__((ext_vector_type(kBytes > 4 ? kBytes / 4 : 2)));
    uint32_t u[kBytes >= 4 ? kBytes / 4 : 1];
    template <bool STREAM>
    __device__ void load(const void* p) {
        if constexpr (kBytes > 4) {
            const Words r = load_from<STREAM>(static_cast<const Words*>(p));
#pragma unroll
            for (int c = 0; c < kBytes / 4; ++c) u[c] = r[c];
        } else if constexpr (kBytes == 4) {
            u[0] = *static_cast<const uint32_t*>(p);
        } else {
            u[0] = *static_cast<const uint16_t*>(p);
        }
    }
    template <bool STREAM>
    __device__ void store(void* p) const {
        if constexpr (kBytes > 4) {
            Words r;
#pragma unroll
            for (int c = 0; c < kBytes / 4; ++c) r[c] = u[c];
            store_to<STREAM>(static_cast<Words*>(p), r);
        } else if constexpr (kBytes == 4) {
            *static_cast<uint32_t*>(p) = u[0];
        } else {
            *static_cast<uint16_t*>(p) = static_cast<uint16_t>(u[0]);
        }
    }
    __device__ float get(int i) const {
        if constexpr (!BF16) return __uint_as_float(u[i]);
        else return i % 2 == 0 ? bf16_lo(u[i / 2]) : bf16_hi(u[i / 2]);
    }
    __device__ void set(const float (&v)[V]) {
#pragma unroll
        for (int c = 0; c < (BF16 ? (V + 1) / 2 : V); ++c) {
            if constexpr (!BF16) u[c] = __float_as_uint(v[c]);
            else if constexpr (V == 1) u[c] = to_bf16x2(v[0], 0.f);
            else u[c] = to_bf16x2(v[2 * c], v[2 * c + 1]);
        }
    }
};

// HALF: an item is V pairs, a piece of either half; else V / 2 pairs in one piece.  Items past the turned columns copy one piece.  A thread has the same
// piece of every row it works on, and requests kBatch of them at once, the first before the sines are computed.  STREAM 1: non-temporal stores, 2: loads too.
constexpr int kBatch = 4;
template <bool BF16, bool HALF, int V, int STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(Rope a) {
    __shared__ float sines[kThreads], cosines[kThreads];
    constexpr int kBytes = BF16 ? 2 : 4;
    const int tid = threadIdx.x, pairs = a.rot / 2, first = blockIdx.x * a.tokens, tokens = min(a.tokens, a.n - first);
    const int rows = tokens * a.heads, per = kThreads / a.row_pieces, piece = tid % a.row_pieces, begin = tid < per * a.row_pieces ? tid / a.row_pieces : rows;
    const bool turns = piece < a.pieces;
    const int at = turns ? piece * V * kBytes : (a.rot + (piece - a.pieces) * V) * kBytes, half = pairs * kBytes;
    Piece<BF16, V> x[kBatch], y[HALF ? kBatch : 1];
    int token[kBatch];
    char* out[kBatch];
    auto ask = [&](int row0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int row = row0 + i * per;
            out[i] = nullptr;
            if (row >= rows) continue;
            token[i] = a.heads == 1 ? row : static_cast<int>(__umulhi(static_cast<uint32_t>(row), a.over_heads));
            const int in_token = row - token[i] * a.heads;
            const RopeSide& side = in_token < a.q.heads ? a.q : a.k;
            const int head = in_token < a.q.heads ? in_token : in_token - a.q.heads;
            const char* in = static_cast<const char*>(side.in) + ((first + token[i]) * side.in_stride + head * a.dim) * kBytes + at;
            char* to = static_cast<char*>(side.out) + ((first + token[i]) * side.out_stride + head * a.dim) * kBytes + at;
            if (!turns && in == to) continue;
            out[i] = to;
            x[i].template load<STREAM == 2>(in);
            if constexpr (HALF)
                if (turns) y[i].template load<STREAM == 2>(in + half);
        }
    };
    ask(begin);
    if (tid < tokens * pairs) {
        const int of = tid / pairs, pair = tid - of * pairs;
        const double turn = static_cast<double>(a.positions[first + of]) * a.freqs[pair] * 0.15915494309189533577;
        float s, c;
        sincospif(2.f * static_cast<float>(turn - rint(turn)), &s, &c);
        sines[tid] = s * a.amplitude;
        cosines[tid] = c * a.amplitude;
    }
    __syncthreads();
    for (int row0 = begin; row0 < rows; row0 += kBatch * per) {
        if (row0 != begin) ask(row0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (out[i] == nullptr) continue;
            if (!turns) {
                x[i].template store<STREAM != 0>(out[i]);
                continue;
            }
            const float *s = sines + token[i] * pairs + piece * (HALF ? V : V / 2), *k = cosines + (s - sines);
            if constexpr (HALF) {
                float u[V], v[V];
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    const float l = x[i].get(c), r = y[i].get(c);
                    u[c] = l * k[c] - r * s[c];
                    v[c] = l * s[c] + r * k[c];
                }
                x[i].set(u);
                y[i].set(v);
                x[i].template store<STREAM != 0>(out[i]);
                y[i].template store<STREAM != 0>(out[i] + half);
            } else {
                float u[V];
#pragma unroll
                for (int c = 0; c < V / 2; ++c) {
                    const float l = x[i].get(2 * c), r = x[i].get(2 * c + 1);
                    u[2 * c] = l * k[c] - r * s[c];
                    u[2 * c + 1] = l * s[c] + r * k[c];
                }
                x[i].set(u);
                x[i].template store<STREAM != 0>(out[i]);
            }
        }
    }
}

template <bool BF16, bool HALF, int V>
void launch(Rope a, hipStream_t s) {
    const bool tail = (a.q.heads > 0 && a.q.in != a.q.out) || (a.k.heads > 0 && a.k.in != a.k.out);
    a.pieces = HALF ? a.rot / 2 / V : a.rot / V;
    a.row_pieces = a.pieces + (tail ? (a.dim - a.rot) / V : 0);
    // Tokens per block: so that each thread has a sine and cosine to compute, where there are blocks enough (16384 x 40 heads of 128: four).
    // What is more than the caches hold does better without them, as the norm's arrays and the cache's.
    a.tokens = std::max(1, std::min(kThreads / (a.rot / 2), a.n / 2048));
    const dim3 blocks(static_cast<unsigned>((static_cast<long>(a.n) + a.tokens - 1) / a.tokens));
    const size_t moved = 2 * static_cast<size_t>(a.n) * a.heads * a.dim * (BF16 ? 2 : 4);
    if (moved <= size_t(100) << 20) hipLaunchKernelGGL((rope_kernel<BF16, HALF, V, 0>), blocks, dim3(kThreads), 0, s, a);
    else if (moved <= size_t(300) << 20) hipLaunchKernelGGL((rope_kernel<BF16, HALF, V, 1>), blocks, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((rope_kernel<BF16, HALF, V, 2>), blocks, dim3(kThreads), 0, s, a);
}

template <bool BF16>
void for_sizes(const Rope& a, bool half, hipStream_t s) {
    const int run = half ? a.rot / 2 : a.rot;                // elements that lie together; as dim is a multiple of 16, what follows them does too
    if constexpr (BF16)
        if (run % 8 == 0) return half ? launch<BF16, true, 8>(a, s) : launch<BF16, false, 8>(a, s);
    if (run % 4 == 0) return half ? launch<BF16, true, 4>(a, s) : launch<BF16, false, 4>(a, s);
    if (run % 2 == 0) return half ? launch<BF16, true, 2>(a, s) : launch<BF16, false, 2>(a, s);
    launch<BF16, true, 1>(a, s);                             // (of neighbours there is an even number)
}

}  // namespace

int launch_rope(const moe_rope_cfg& c, int n, const int32_t* positions, const double* freqs, const RopeSide& q, const RopeSide& k, hipStream_t s) {
    Rope a;
    a.q = q;
    a.k = k;
    a.positions = positions;
    a.freqs = freqs;
    a.n = n;
    a.dim = c.head_dim;
    a.rot = c.rot_dim;
    a.heads = q.heads + k.heads;
    a.tokens = a.pieces = a.row_pieces = 0;                  // set where the pieces' width is chosen
    a.over_heads = static_cast<uint32_t>(((uint64_t(1) << 32) + a.heads - 1) / a.heads);
    a.amplitude = c.amplitude == 0.f ? 1.f : c.amplitude;
    if (c.dtype == MOE_BF16) for_sizes<true>(a, c.pairs == MOE_PAIRS_HALF, s);
    else for_sizes<false>(a, c.pairs == MOE_PAIRS_HALF, s);
    MOE_LAUNCH_CHECK("rope_kernel");
    return MOE_OK;
}

}  // namespace moe
