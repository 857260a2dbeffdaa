// A wave's 32 tokens of a cache in 4 bits.  What a lane holds of them becomes what attention over FP16 works with (kvc_attend.h) by conversions alone: a code and its exponent are
// an FP16 number exactly, so nothing is lost on the way.
//
// As sums over channels take their terms in any order, lane group g = lane / 16 has the channels 4w*g..4w*g+4w-1 of a piece of 16w: 2w bytes in a row, all of one
// exponent.  (FP16 keys are taken 8 channels at a time: 4 * w/8 times 16 bytes.)  Values are as there: channels w*n..w*n+w-1 of 8 tokens, w/2 bytes of each row.
#pragma once
#include "kvc_divide.h"
#include "kvc_fp4.h"

namespace kvc {

// Memory that loads name as such: where the compiler cannot tell memory from LDS a load waits for both, and for all before it.
typedef const __attribute__((address_space(1))) uint8_t* bytes_at;
template <class T>
__device__ inline T load_from(bytes_at p) { return *reinterpret_cast<const __attribute__((address_space(1))) T*>(p); }

// Rows of codes, and exponents, of tokens that do not exist: zeros.  8 rows of the widest head.
static __device__ __align__(16) const uint8_t kZeroCodes[1024] = {};

// Where tokens are: as Source, with the pages of one KV head in 4 bits
struct SourceFp4 {
    const int32_t* table;
    uint32_t len;
    const uint8_t* k;
    const uint8_t* v;
};

// Entries of the block table for the 32 tokens from t on, as Blocks has them (kvc_attend.h), looked up whether the tokens are there or not: loads that are always made can be waited for
// one by one.  (There is a token.)
template <bool EIGHT>
__device__ inline Blocks<EIGHT> look_up(const AttendArgs& a, const int32_t* table, uint32_t len, uint32_t t) {
    Blocks<EIGHT> b;
#pragma unroll
    for (int i = 0; i < (EIGHT ? 2 : 1); ++i) b.of[i] = load_from<int32_t>((bytes_at)(table + fast_div(min(t + b.token(i), len - 1), a.by_N)));
    return b;
}

template <int D>
struct KeysFp4 {
    uint32_t c[2][D / 32];         // [score tile]: codes
    uint32_t e[piece_count(D)][2];  // exponents of 8 tokens, or of the two
};
template <int D, bool EIGHT>
struct ValuesFp4 {
    uint32_t c[8][piece_count(D)];              // [token]: codes of a piece
    uint32_t e[piece_count(D)][EIGHT ? 2 : 8];  // exponents of 8 tokens, or one each
};

template <int BYTES>
__device__ inline void load_codes(uint32_t* to, bytes_at p) {
    if constexpr (BYTES == 16) {
        const uint4v r = load_from<uint4v>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = r[i];
    } else if constexpr (BYTES == 8) {
        const uint2v r = load_from<uint2v>(p);
        to[0] = r[0];
        to[1] = r[1];
    } else if constexpr (BYTES == 4) {
        *to = load_from<uint32_t>(p);
    } else if constexpr (BYTES == 2) {
        *to = load_from<uint16_t>(p);
    } else {
        *to = load_from<uint8_t>(p);
    }
}

template <int D, int P = 0>
__device__ inline void load_key_codes(KeysFp4<D>& x, int u, bytes_at row, uint32_t g) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
        load_codes<2 * Q::w>(&x.c[u][Q::regs], row + Q::before / 2 + 2 * Q::w * g);
        load_key_codes<D, P + 1>(x, u, row, g);
    }
}
// group of 32 channels that a lane's keys are of, and its values
template <int D, int P>
__device__ inline uint32_t key_group(uint32_t g) { return Piece<D, P>::before / 32 + Piece<D, P>::w * g / 8; }
template <int D, int P>
__device__ inline uint32_t value_group(uint32_t n) { return Piece<D, P>::before / 32 + Piece<D, P>::w * n / 32; }

// exps: the exponents of a token's first group, `step` bytes before those of the next group
template <int D, bool EIGHT, int P = 0>
__device__ inline void load_key_exps(KeysFp4<D>& x, int u, bytes_at exps, uint32_t step, uint32_t g) {
    if constexpr (P < piece_count(D)) {
        bytes_at p = exps + key_group<D, P>(g) * step;
        if constexpr (EIGHT) load_codes<8>(x.e[P], p);
        else load_codes<1>(&x.e[P][u], p);
        load_key_exps<D, EIGHT, P + 1>(x, u, exps, step, g);
    }
}

// Row of token t in its block.
__device__ inline uint32_t row_of(const AttendArgs& a, uint32_t t) { return t - fast_div(t, a.by_N) * (uint32_t)a.g.N; }

// Whether a block is there: an entry of a token that exists, and within the cache.  `bad` notes entries beyond it.
__device__ inline bool is_there(const AttendArgs& a, int32_t block, bool exists, bool& bad) {
    const bool beyond = block >= a.n_cache_blocks;
    bad = bad || (exists && beyond);
    return exists && block >= 0 && !beyond;
}

// live: whether there is such a tile at all.
template <int D, bool EIGHT>
__device__ inline void load_keys(KeysFp4<D>& x, const AttendArgs& a, const Fp4Pages& f, const SourceFp4& s, const Blocks<EIGHT>& b, uint32_t t, bool live, bool& bad) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, octet = t + 8 * (n >> 2);
    const bytes_at zero = (bytes_at)kZeroCodes, pages = (bytes_at)s.k;
    if constexpr (EIGHT) {
        const int32_t block = b.key(0);
        const bool have = is_there(a, block, live && octet < s.len, bad);
        const uint32_t row = row_of(a, octet);
        bytes_at page = pages + block * f.block;
        bytes_at codes = have ? page + (row + (n & 3)) * (D / 2) : zero;  // (rows behind the last token are the page's all the same, and not seen)
        load_key_codes<D>(x, 0, codes, g);
        load_key_codes<D>(x, 1, codes + 4 * (D / 2), g);
        load_key_exps<D, true>(x, 0, have ? page + f.exps + row : zero, have ? (uint32_t)a.g.N : 0, g);
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = octet + 4 * u + (n & 3);
            const int32_t block = b.key(u);
            const bool have = is_there(a, block, live && at < s.len, bad);
            const uint32_t row = row_of(a, at);
            bytes_at page = pages + block * f.block;
            load_key_codes<D>(x, u, have ? page + row * (D / 2) : zero, g);
            load_key_exps<D, false>(x, u, have ? page + f.exps + row : zero, have ? (uint32_t)a.g.N : 0, g);
        }
    }
}

template <int D, bool EIGHT, int P = 0>
__device__ inline void load_value_codes(ValuesFp4<D, EIGHT>& x, int j, bytes_at row, uint32_t n) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
        load_codes<Q::w / 2>(&x.c[j][P], row + Q::before / 2 + Q::w / 2 * n);
        load_value_codes<D, EIGHT, P + 1>(x, j, row, n);
    }
}
template <int D, bool EIGHT, int P = 0>
__device__ inline void load_value_exps(ValuesFp4<D, EIGHT>& x, int j, bytes_at exps, uint32_t step, uint32_t n) {
    if constexpr (P < piece_count(D)) {
        bytes_at p = exps + value_group<D, P>(n) * step;
        if constexpr (EIGHT) load_codes<8>(x.e[P], p);
        else load_codes<1>(&x.e[P][j], p);
        load_value_exps<D, EIGHT, P + 1>(x, j, exps, step, n);
    }
}

// -> bit j: token t + 8g + j exists
template <int D, bool EIGHT>
__device__ inline uint32_t load_values(ValuesFp4<D, EIGHT>& x, const AttendArgs& a, const Fp4Pages& f, const SourceFp4& s, const Blocks<EIGHT>& b, uint32_t t, bool live, bool& bad) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, first = t + 8 * (lane >> 4);
    const bytes_at zero = (bytes_at)kZeroCodes, pages = (bytes_at)s.v;
    if constexpr (EIGHT) {
        const int32_t block = b.value(0);
        const bool have = is_there(a, block, live && first < s.len, bad);
        const uint32_t row = row_of(a, first);
        bytes_at page = pages + block * f.block;
        bytes_at codes = have ? page + row * (D / 2) : zero;
#pragma unroll
        for (int j = 0; j < 8; ++j) load_value_codes<D, true>(x, j, codes + j * (D / 2), n);
        load_value_exps<D, true>(x, 0, have ? page + f.exps + row : zero, have ? (uint32_t)a.g.N : 0, n);
        const uint32_t exist = s.len - min(first, s.len);
        return !have ? 0 : exist >= 8 ? 0xFF : ~(~0u << exist);
    } else {
        uint32_t there = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int32_t block = b.value(j);
            const bool have = is_there(a, block, live && first + j < s.len, bad);
            const uint32_t row = row_of(a, first + j);
            bytes_at page = pages + block * f.block;
            there |= have ? 1u << j : 0u;
            load_value_codes<D, false>(x, j, have ? page + row * (D / 2) : zero, n);
            load_value_exps<D, false>(x, j, have ? page + f.exps + row : zero, have ? (uint32_t)a.g.N : 0, n);
        }
        return there;
    }
}

// 2^e from its byte; 255 makes NaN of any code, as the conversion has it
__device__ inline float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight channels of FP16, from a register of codes.
__device__ inline uint4v eight_channels(uint32_t codes, float scale) {
    uint4v r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
    return r;
}

template <int D, bool EIGHT, int P = 0>
__device__ inline void expand_keys(Tokens<D>& to, const KeysFp4<D>& x) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float scale = power_of(EIGHT ? x.e[P][u] >> 8 * (threadIdx.x & 3) & 255 : x.e[P][u]);
#pragma unroll
            for (int c = 0; c < Q::w / 2; ++c) to.k[u][Q::regs + c] = eight_channels(x.c[u][Q::regs + c], scale);
        }
        expand_keys<D, EIGHT, P + 1>(to, x);
    }
}
// Values of the tokens of `there`, bit j of token t + 8g + j; the others become zero.
template <int D, bool EIGHT, int P = 0>
__device__ inline void expand_values(Tokens<D>& to, const ValuesFp4<D, EIGHT>& x, uint32_t there) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float scale = power_of(!(there >> j & 1) ? 0 : EIGHT ? x.e[P][EIGHT ? j / 4 : 0] >> 8 * (j % 4) & 255 : x.e[P][EIGHT ? 0 : j]);
            to.v[j][Q::regs] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.c[j][P], scale, 0));
            if constexpr (Q::w > 2) to.v[j][Q::regs + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.c[j][P], scale, 1));
            if constexpr (Q::w > 4) {
                to.v[j][Q::regs + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.c[j][P], scale, 2));
                to.v[j][Q::regs + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x.c[j][P], scale, 3));
            }
        }
        expand_values<D, EIGHT, P + 1>(to, x, there);
    }
}

// A row's query, its channels in the order of the keys'.
template <int D, int P = 0>
__device__ inline void load_query(uint4v (&q)[D / 32], const uint16_t* row, uint32_t g) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int c = 0; c < Q::w / 2; ++c) q[Q::regs + c] = *reinterpret_cast<const uint4v*>(row + Q::before + 4 * Q::w * g + 8 * c);
        load_query<D, P + 1>(q, row, g);
    }
}

}  // namespace kvc
