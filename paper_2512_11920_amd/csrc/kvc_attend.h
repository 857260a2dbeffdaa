// Attention over a paged cache: what a wave does with 32 tokens.
//
// The scores are made transposed, S^T = K Q^T, and the output too, O^T = V^T P^T, with matrix instructions of 16 x 16 x 32.  A wave holds 16
// query rows: row n belongs to the lanes n, n + 16, n + 32, n + 48, and everything about it (maximum, sum, output) stays in them.
// The sums over channels and over tokens take their terms in any order, so the order is chosen for the lanes:
//   * of 32 tokens, token 8g + 4u + r is row 4g + r of score tile u.  A lane of group g = lane / 16 then gets the scores
//     of tokens 8g..8g+7, and those are the terms it holds of P^T in the second product: the scores become weights in place.
//   * in the second product a lane holds V of the same 8 tokens for the channels w*n..w*n+w-1 of a piece of 16w channels.  It loads them
//     as they lie (16w * 2 bytes of a row, shared by 16 lanes) and pairs tokens with one byte permutation a register; channel w*n + j
//     goes to row n of output tile j.  A lane ends up with 4w consecutive channels of its row.
// So keys and values go from memory to registers and from there to the matrix unit, without LDS and without a word to another lane.
//
// Tokens that do not exist (behind the end, in a block that is not there) are read from a row of zeros: their scores are
// replaced by -infinity, and their values add weight zero times zero, whatever the cache holds in their place.
#pragma once
#include "kvc_cache.h"

namespace kvc {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // tokens

// Weights are 2^(x - m + kLift), x the score in powers of two and m a maximum that may lag by kLag: FP16 holds them with 11 bits from 2^(kLift + kLag)
// = 2^14 (its largest is below 2^16) down to 2^-14, that is 2^-24 of the largest weight; smaller ones keep fewer bits, down to 2^-34.
constexpr float kLift = 10.f, kLag = 4.f;

// 512 bytes of zeros: a row of the widest head
static __device__ __align__(16) const uint16_t kZeroRow[256] = {};

// Pieces of a row's channels: 128s, then a 64, then a 32.
constexpr int piece_count(int d) { return d / 128 + d / 64 % 2 + d / 32 % 2; }
constexpr int piece_before(int d, int p) { return p <= d / 128 ? 128 * p : p == d / 128 + 1 ? d / 128 * 128 + (d / 64 % 2 ? 64 : 32) : d; }
template <int D, int P>
struct Piece {
    static constexpr int before = piece_before(D, P), w = (piece_before(D, P + 1) - before) / 16;  // channels before it; channels of a lane
    static constexpr int regs = before / 32;                                                     // 32-bit registers of a token before it
};

// Where tokens are: a sequence's or a prefix's row of a block table, and the pages of one KV head.
struct Source {
    const int32_t* table;
    const uint16_t* k;  // page of the head in block 0
    const uint16_t* v;
    uint32_t len;       // tokens, at most the row's blocks hold
};

// Blocks of the 32 tokens from t on, as the table names them; -1: none, or the token is behind the end.  Where 8 tokens from a multiple of 8 on share a
// block (EIGHT: N is a multiple of 8) a lane holds the two that it needs, of its keys and of its values; else that of token `lane` mod 32, and asks the others.
template <bool EIGHT>
struct Blocks {
    int32_t of[EIGHT ? 2 : 1];

    __device__ int32_t key(int u) const { return EIGHT ? of[0] : __shfl(of[0], 8 * ((threadIdx.x & 15) >> 2) + 4 * u + (threadIdx.x & 3)); }
    __device__ int32_t value(int j) const { return EIGHT ? of[EIGHT ? 1 : 0] : __shfl(of[0], 8 * ((threadIdx.x & 63) >> 4) + j); }
    // token of t.. whose block of[i] is
    __device__ static uint32_t token(int i) {
        const uint32_t lane = threadIdx.x & 63;
        return !EIGHT ? lane & 31 : i == 0 ? 8 * ((lane & 15) >> 2) : 8 * (lane >> 4);
    }
    __device__ void end_at(uint32_t t, uint32_t len) {  // no blocks from token len on
#pragma unroll
        for (int i = 0; i < (EIGHT ? 2 : 1); ++i) of[i] = t + token(i) < len ? of[i] : -1;
    }
};
__device__ inline int32_t block_of(const AttendArgs& a, const Source& s, uint32_t t) { return t < s.len ? s.table[fast_div(t, a.by_N)] : -1; }
template <bool EIGHT>
__device__ inline Blocks<EIGHT> find_blocks(const AttendArgs& a, const Source& s, uint32_t t) {
    Blocks<EIGHT> b;
#pragma unroll
    for (int i = 0; i < (EIGHT ? 2 : 1); ++i) b.of[i] = block_of(a, s, t + b.token(i));
    return b;
}
__device__ inline bool in_cache(const AttendArgs& a, int32_t block) {
    if (block < a.n_cache_blocks) return block >= 0;
    atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
    return false;
}
// row of token t in its block, in elements
__device__ inline int64_t place(const AttendArgs& a, int32_t block, uint32_t t) {
    return block * a.g.block_stride + (int64_t)((t - fast_div(t, a.by_N) * (uint32_t)a.g.N) * (uint32_t)a.g.row_stride);
}

// K and V of 32 tokens as a lane holds them.
template <int D>
struct Tokens {
    uint4v k[2][D / 32];    // [score tile][step of 32 channels]: 8 channels
    uint32_t v[8][D / 32];  // [token]: the lane's channels of every piece
};

template <int D, bool EIGHT>
__device__ inline void load_keys(Tokens<D>& x, const AttendArgs& a, const Source& s, const Blocks<EIGHT>& b, uint32_t t) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const uint32_t first = t + 8 * (n >> 2) + (n & 3);
    int64_t at = 0;
    bool have = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (u == 0 || !EIGHT) {
            const int32_t block = b.key(u);
            have = in_cache(a, block);
            at = place(a, block, first + 4 * u);
        }
        const uint16_t* row = have && first + 4 * u < s.len ? s.k + at + (EIGHT ? 4 * u * a.g.row_stride : 0) : kZeroRow;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) x.k[u][c] = *reinterpret_cast<const uint4v*>(row + 32 * c + 8 * g);
    }
}

template <int D, int P>
__device__ inline void load_pieces(Tokens<D>& x, int j, const uint16_t* row, int n) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
        const uint16_t* p = row + Q::before + Q::w * n;
        if constexpr (Q::w == 8) {
            const uint4v r = *reinterpret_cast<const uint4v*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) x.v[j][Q::regs + e] = r[e];
        } else if constexpr (Q::w == 4) {
            const uint2v r = *reinterpret_cast<const uint2v*>(p);
            x.v[j][Q::regs] = r[0];
            x.v[j][Q::regs + 1] = r[1];
        } else {
            x.v[j][Q::regs] = *reinterpret_cast<const uint32_t*>(p);
        }
        load_pieces<D, P + 1>(x, j, row, n);
    }
}

// -> bit j: token t + 8g + j exists
template <int D, bool EIGHT>
__device__ inline uint32_t load_values(Tokens<D>& x, const AttendArgs& a, const Source& s, const Blocks<EIGHT>& b, uint32_t t) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, first = t + 8 * (lane >> 4);
    uint32_t there = 0;
    int64_t at = 0;
    bool have = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j == 0 || !EIGHT) {
            const int32_t block = b.value(j);
            have = in_cache(a, block);
            at = place(a, block, first + j);
        }
        const bool here = have && first + j < s.len;
        there |= here ? 1u << j : 0u;
        load_pieces<D, 0>(x, j, here ? s.v + at + (EIGHT ? j * a.g.row_stride : 0) : kZeroRow, n);
    }
    return there;
}

// The two halves of a wave, and the two rows of 16 lanes of each half, change places: what a lane and its partners hold, joined.
__device__ inline float both16(float v, bool sum) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return sum ? __uint_as_float(r[0]) + __uint_as_float(r[1]) : fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float both32(float v, bool sum) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return sum ? __uint_as_float(r[0]) + __uint_as_float(r[1]) : fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The largest of a row's four lanes, and their sum.
__device__ inline float row_max(float v) { return both32(both16(v, false), false); }
__device__ inline float row_sum(float v) { return both32(both16(v, true), true); }

// 2^x by the hardware's instruction alone: what would be a subnormal number is zero.
__device__ inline float power2(float x) { return __builtin_amdgcn_exp2f(x); }

// Running softmax of 16 rows: output tiles, the reference that weights are relative to, and the lane's part of their sum.
template <int D>
struct Rows {
    uint4v q[D / 32];
    float4v o[D / 16];  // tile of piece P, channel j of w: o[Piece::before / 16 + j]
    float m, l;
};

template <int D>
__device__ inline void clear(Rows<D>& r) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) r.o[i] = float4v{0.f, 0.f, 0.f, 0.f};
    r.m = -INFINITY;
    r.l = 0.f;
}

template <int D>
__device__ inline void scores(float4v (&s)[2], const Rows<D>& r, const Tokens<D>& x) {
    s[0] = s[1] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u)
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, x.k[u][c]), __builtin_bit_cast(half8, r.q[c]), s[u], 0, 0, 0);
}

// Scores of tokens t + 8g.. become weights, of those below the row's limit that exist; the row's reference follows their maximum.  (Maxima pass
// NaN over, so a reference is never NaN; the weights' sum keeps it.)
template <int D>
__device__ inline half8 weights(Rows<D>& r, const float4v (&s)[2], float scale_log2, uint32_t there, uint32_t t, uint32_t limit) {
    const uint32_t first = t + 8 * ((threadIdx.x & 63) >> 4), n = limit > first ? limit - first : 0;
    const uint32_t seen = there & (n >= 8 ? 0xFFu : ~(~0u << n));
    float v[8], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = seen >> j & 1 ? s[j / 4][j % 4] * scale_log2 : -INFINITY;
        top = fmaxf(top, v[j]);
    }
    top = row_max(top);
    if (__any(top > r.m + kLag)) {  // (a row's first token too: its reference is -infinity)
        const float m = fmaxf(r.m, top), f = r.m == -INFINITY ? 0.f : power2(r.m - m);
        r.m = m;
        r.l *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) r.o[i] *= f;
    }
    const float low = (r.m == -INFINITY ? 0.f : r.m) - kLift;
    half8 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float w = power2(v[j] - low);
        r.l += w;
        p[j] = (_Float16)w;
    }
    return p;
}

// Eight tokens' values of the lane's channel of output tile j of piece P.
template <int D, int P>
__device__ inline uint4v value_column(const Tokens<D>& x, int j) {
    uint4v v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = __builtin_amdgcn_perm(x.v[2 * e + 1][Piece<D, P>::regs + j / 2], x.v[2 * e][Piece<D, P>::regs + j / 2], j & 1 ? 0x07060302u : 0x05040100u);
    return v;
}

template <int D, int R, int P = 0>
__device__ inline void add_values(Rows<D> (&r)[R], const Tokens<D>& x, const half8 (&p)[R]) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int j = 0; j < Q::w; ++j) {
            const half8 v = __builtin_bit_cast(half8, value_column<D, P>(x, j));
#pragma unroll
            for (int i = 0; i < R; ++i) r[i].o[Q::before / 16 + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[i], r[i].o[Q::before / 16 + j], 0, 0, 0);
        }
        add_values<D, R, P + 1>(r, x, p);
    }
}

// Where a tile holds tokens that some rows see and others do not, a value that is infinite or NaN must reach the former alone, and weight zero times it is
// NaN.  In such a tile these values are counted (a product of ones), the rows that see any get the infinity, or both, and the values become zero.
// 1.0 in each half that is an infinity of this sign, or NaN
__device__ inline uint32_t ones_where(uint32_t v, uint32_t infinity) {
    const uint32_t lo = v & 0xFFFFu, hi = v >> 16;
    return (lo == infinity || (lo & 0x7FFFu) > 0x7C00u ? 0x3C00u : 0u) | (hi == infinity || (hi & 0x7FFFu) > 0x7C00u ? 0x3C000000u : 0u);
}
template <int D, int R, int P = 0>
__device__ inline void add_infinite(Rows<D> (&r)[R], const Tokens<D>& x, const half8 (&seen)[R]) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int j = 0; j < Q::w; ++j) {
            const uint4v v = value_column<D, P>(x, j);
#pragma unroll
            for (uint32_t sign = 0; sign < 2; ++sign) {
                uint4v one;
#pragma unroll
                for (int e = 0; e < 4; ++e) one[e] = ones_where(v[e], sign ? 0xFC00u : 0x7C00u);
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const float4v n = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, one), seen[i], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[i].o[Q::before / 16 + j][e] += n[e] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
                }
                __builtin_amdgcn_sched_barrier(0);  // (one at a time: there are few registers)
            }
        }
        add_infinite<D, R, P + 1>(r, x, seen);
    }
}

// The tile from t on of a sequence of `len` tokens, of whose last n_q - 1 some rows see less than others.
template <int D, int R>
__device__ inline void add_tile(Rows<D> (&r)[R], Tokens<D>& x, const half8 (&p)[R], uint32_t t, uint32_t len, uint32_t n_q, const uint32_t (&limit)[R]) {
    if (n_q > 1 && t + kTile + n_q - 1 > len) {
        uint32_t carry = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < D / 32; ++e) carry |= (x.v[j][e] & 0x7C007C00u) + 0x04000400u;  // an exponent of ones carries into the sign
        if (__any(carry & 0x80008000u)) {
            const uint32_t first = t + 8 * ((threadIdx.x & 63) >> 4);
            half8 seen[R];
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) seen[i][j] = first + j < limit[i] ? (_Float16)1.f : (_Float16)0.f;
            add_infinite<D, R>(r, x, seen);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    const uint32_t all = ((x.v[j][e] & 0x7C007C00u) + 0x04000400u) >> 15 & 0x00010001u;
                    x.v[j][e] &= ~(all * 0xFFFFu);
                }
        }
    }
    add_values<D, R>(r, x, p);
}

template <int D, int P>
__device__ inline void store_pieces(const Rows<D>& r, uint16_t* out, float f, int g) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
        uint32_t v[2 * Q::w];
#pragma unroll
        for (int e = 0; e < 2 * Q::w; ++e) {  // channels 2e and 2e+1 of the lane's 4w: w*i + j
            const int c = 2 * e;
            half2 h;
            h[0] = (_Float16)(r.o[Q::before / 16 + c % Q::w][c / Q::w] * f);
            h[1] = (_Float16)(r.o[Q::before / 16 + (c + 1) % Q::w][(c + 1) / Q::w] * f);
            v[e] = __builtin_bit_cast(uint32_t, h);
        }
        uint16_t* p = out + Q::before + 4 * Q::w * g;
#pragma unroll
        for (int e = 0; e < Q::w / 2; ++e) *reinterpret_cast<uint4*>(p + 8 * e) = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        store_pieces<D, P + 1>(r, out, f, g);
    }
}

// The same channels as they are summed, in 32 bits.
template <int D, int P = 0>
__device__ inline void store_sums(const Rows<D>& r, float* out, int g) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
        float* p = out + Q::before + 4 * Q::w * g;
#pragma unroll
        for (int e = 0; e < Q::w; ++e) {
            float4v v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = r.o[Q::before / 16 + (4 * e + i) % Q::w][(4 * e + i) / Q::w];
            *reinterpret_cast<float4v*>(p + 4 * e) = v;
        }
        store_sums<D, P + 1>(r, out, g);
    }
}

// log-sum-exp of a row whose weights are relative to 2^m and sum to l
__device__ inline float lse_of(float m, float l) { return l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : l == l ? -INFINITY : l; }

}  // namespace kvc
