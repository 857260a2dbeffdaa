// A wave's 32 tokens of a cache in 4 bits.  What a lane holds of them becomes what attention over FP16 works with (kvc_attend.h) by conversions alone: a code and an exponent that
// append wrote are an FP16 number exactly, so nothing is lost on the way.
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

// Where 32 tokens are: blocks as the table names them, and rows in the blocks.  Where 8 tokens from a multiple of 8 on share a block (EIGHT: N is a multiple of 8) a lane holds those of the first
// of its 8 keys and of its 8 values; else of token `lane` mod 32, and asks the others.
template <bool EIGHT>
struct Spots {
    int32_t block[EIGHT ? 2 : 1];
    uint32_t row[EIGHT ? 2 : 1];
};
// Looks up tile after tile.  From one to the next of a sequence a token's place moves on by 32 tokens: so many blocks and so many rows, and another block where that leaves the block.  What the
// table says is asked for whether the tokens are there or not: loads that are always made can be waited for one by one.
template <bool EIGHT>
struct Finder {
    static constexpr int kSpots = EIGHT ? 2 : 1;
    uint32_t entry[kSpots], row[kSpots];

    // token of a tile that spot i is of
    __device__ static uint32_t token(int i) {
        const uint32_t lane = threadIdx.x & 63;
        return !EIGHT ? lane & 31 : i == 0 ? 8 * ((lane & 15) >> 2) : 8 * (lane >> 4);
    }
    // first: tile t is not the one behind the last that was looked up.  len: tokens of the sequence, not 0
    __device__ Spots<EIGHT> find(const AttendArgs& a, const int32_t* table, uint32_t len, uint32_t t, bool first) {
        const uint32_t N = (uint32_t)a.g.N, last = fast_div(len - 1, a.by_N);
        Spots<EIGHT> s;
        if (first) {
#pragma unroll
            for (int i = 0; i < kSpots; ++i) {
                entry[i] = fast_div(t * kTile + token(i), a.by_N);
                row[i] = t * kTile + token(i) - entry[i] * N;
            }
        } else {
            const uint32_t blocks = fast_div(kTile, a.by_N), rows = kTile - blocks * N;
#pragma unroll
            for (int i = 0; i < kSpots; ++i) {
                row[i] += rows;
                const bool leaves = row[i] >= N;
                row[i] -= leaves ? N : 0;
                entry[i] += blocks + (leaves ? 1 : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kSpots; ++i) {
            s.block[i] = load_from<int32_t>((bytes_at)(table + min(entry[i], last)));
            s.row[i] = row[i];
        }
        return s;
    }
};
// A block and a row: of the lane's keys (score tile u) or values (token j).
struct Spot {
    int32_t block;
    uint32_t row;
};
template <bool EIGHT>
__device__ inline Spot key_spot(const Spots<EIGHT>& s, int u) {
    if constexpr (EIGHT) return {s.block[0], s.row[0] + 4 * u + (threadIdx.x & 3)};
    const int lane = 8 * ((threadIdx.x & 15) >> 2) + 4 * u + (threadIdx.x & 3);
    return {__shfl(s.block[0], lane), (uint32_t)__shfl((int)s.row[0], lane)};
}
template <bool EIGHT>
__device__ inline Spot value_spot(const Spots<EIGHT>& s, int j) {
    if constexpr (EIGHT) return {s.block[EIGHT ? 1 : 0], s.row[EIGHT ? 1 : 0] + j};
    const int lane = 8 * ((threadIdx.x & 63) >> 4) + j;
    return {__shfl(s.block[0], lane), (uint32_t)__shfl((int)s.row[0], lane)};
}
// Whether a token that exists has a block; `bad` notes entries beyond the cache.
__device__ inline bool is_there(const AttendArgs& a, int32_t block, bool exists, bool& bad) {
    const bool in = (uint32_t)block < (uint32_t)min(a.n_cache_blocks, (int64_t)INT32_MAX + 1);  // (not what is below zero)
    bad = bad || (exists && !in && block >= 0);
    return exists && in;
}
// The page of a block (its bytes are counted in 32 bits), from the head's page of block 0 on.
__device__ inline bytes_at page_of(const uint8_t* pages, const Fp4Pages& f, int32_t block) { return (bytes_at)pages + (uint64_t)(uint32_t)block * (uint32_t)f.block; }

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

template <int D, bool EIGHT, int P = 0>
__device__ inline void load_key_exps(KeysFp4<D>& x, int u, bytes_at exps, bool have, uint32_t N, uint32_t g) {
    if constexpr (P < piece_count(D)) {
        const bytes_at p = have ? exps + key_group<D, P>(g) * N : (bytes_at)kZeroCodes;
        if constexpr (EIGHT) load_codes<8>(x.e[P], p);
        else load_codes<1>(&x.e[P][u], p);
        load_key_exps<D, EIGHT, P + 1>(x, u, exps, have, N, g);
    }
}

// live: whether there is such a tile at all.
template <int D, bool EIGHT>
__device__ inline void load_keys(KeysFp4<D>& x, const AttendArgs& a, const Fp4Pages& f, const SourceFp4& s, const Spots<EIGHT>& spots, uint32_t t, bool live, bool& bad) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, octet = t + 8 * (n >> 2), N = (uint32_t)a.g.N;
    if constexpr (EIGHT) {
        const Spot at = key_spot<EIGHT>(spots, 0);
        const bool have = is_there(a, at.block, live && octet < s.len, bad);
        const bytes_at page = page_of(s.k, f, at.block), codes = have ? page + at.row * (D / 2) : (bytes_at)kZeroCodes;  // (rows behind the last token are the page's all the same, and not seen)
        load_key_codes<D>(x, 0, codes, g);
        load_key_codes<D>(x, 1, codes + 4 * (D / 2), g);
        load_key_exps<D, true>(x, 0, page + f.exps + spots.row[0], have, N, g);
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Spot at = key_spot<EIGHT>(spots, u);
            const bool have = is_there(a, at.block, live && octet + 4 * u + (n & 3) < s.len, bad);
            const bytes_at page = page_of(s.k, f, at.block);
            load_key_codes<D>(x, u, have ? page + at.row * (D / 2) : (bytes_at)kZeroCodes, g);
            load_key_exps<D, false>(x, u, page + f.exps + at.row, have, N, g);
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
__device__ inline void load_value_exps(ValuesFp4<D, EIGHT>& x, int j, bytes_at exps, bool have, uint32_t N, uint32_t n) {
    if constexpr (P < piece_count(D)) {
        const bytes_at p = have ? exps + value_group<D, P>(n) * N : (bytes_at)kZeroCodes;
        if constexpr (EIGHT) load_codes<8>(x.e[P], p);
        else load_codes<1>(&x.e[P][j], p);
        load_value_exps<D, EIGHT, P + 1>(x, j, exps, have, N, n);
    }
}

// -> bit j: token t + 8g + j exists
template <int D, bool EIGHT>
__device__ inline uint32_t load_values(ValuesFp4<D, EIGHT>& x, const AttendArgs& a, const Fp4Pages& f, const SourceFp4& s, const Spots<EIGHT>& spots, uint32_t t, bool live, bool& bad) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, first = t + 8 * (lane >> 4), N = (uint32_t)a.g.N;
    if constexpr (EIGHT) {
        const Spot at = value_spot<EIGHT>(spots, 0);
        const bool have = is_there(a, at.block, live && first < s.len, bad);
        const bytes_at page = page_of(s.v, f, at.block), codes = have ? page + at.row * (D / 2) : (bytes_at)kZeroCodes;
#pragma unroll
        for (int j = 0; j < 8; ++j) load_value_codes<D, true>(x, j, codes + j * (D / 2), n);
        load_value_exps<D, true>(x, 0, page + f.exps + at.row, have, N, n);
        const uint32_t exist = s.len - min(first, s.len);
        return !have ? 0 : exist >= 8 ? 0xFF : ~(~0u << exist);
    } else {
        uint32_t there = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const Spot at = value_spot<EIGHT>(spots, j);
            const bool have = is_there(a, at.block, live && first + j < s.len, bad);
            const bytes_at page = page_of(s.v, f, at.block);
            there |= have ? 1u << j : 0u;
            load_value_codes<D, false>(x, j, have ? page + at.row * (D / 2) : (bytes_at)kZeroCodes, n);
            load_value_exps<D, false>(x, j, page + f.exps + at.row, have, N, n);
        }
        return there;
    }
}

// 2^e, from byte `at` of a register: the conversion looks at nothing but bits 23 to 30 (a test compares all codes under all exponents that append writes, beside any others; 255 makes NaN of any code), so the byte is turned there and
// its neighbours may be anywhere.
__device__ inline float power_of(uint32_t bytes, uint32_t at) { return __uint_as_float(__builtin_amdgcn_alignbit(bytes, bytes, (8 * at + 9) & 31)); }

// Channels 2c and 2c + 1 of a register of codes.
__device__ inline half2 two_channels(uint32_t codes, float scale, int c) {  // (c a constant)
    return __builtin_bit_cast(half2, c == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0)
                                     : c == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1)
                                     : c == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2)
                                              : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
}
// Eight channels of FP16, from a register of codes.
__device__ inline uint4v eight_channels(uint32_t codes, float scale) {
    uint4v r;
#pragma unroll
    for (int c = 0; c < 4; ++c) r[c] = __builtin_bit_cast(uint32_t, two_channels(codes, scale, c));
    return r;
}

template <int D, bool EIGHT, int P = 0>
__device__ inline void expand_keys(Tokens<D>& to, const KeysFp4<D>& x) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float scale = power_of(x.e[P][u], EIGHT ? threadIdx.x & 3 : 0);
#pragma unroll
            for (int c = 0; c < Q::w / 2; ++c) to.k[u][Q::regs + c] = eight_channels(x.c[u][Q::regs + c], scale);
        }
        expand_keys<D, EIGHT, P + 1>(to, x);
    }
}
// 2^e of token j of a lane's 8, of the exponents of one piece
template <bool EIGHT>
__device__ inline float exponent(const uint32_t (&e)[EIGHT ? 2 : 8], int j) { return power_of(e[EIGHT ? j / 4 : j], EIGHT ? j % 4 : 0); }
// Exponents of the tokens of `there` (bit j: token j of 8), in the place of the others zero, which makes zeros of their codes.
template <int D, bool EIGHT>
__device__ inline void keep_values(ValuesFp4<D, EIGHT>& x, uint32_t there) {
    if constexpr (EIGHT) {
        uint32_t mask[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) mask[i] = ((there >> 4 * i & 15) * 0x00204081u & 0x01010101u) * 255;  // (a bit to a byte)
#pragma unroll
        for (int p = 0; p < piece_count(D); ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) x.e[p][i] &= mask[i];
    } else {
#pragma unroll
        for (int p = 0; p < piece_count(D); ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) x.e[p][j] = there >> j & 1 ? x.e[p][j] : 0;
    }
}
template <int D, bool EIGHT, int P = 0>
__device__ inline void expand_values(Tokens<D>& to, const ValuesFp4<D, EIGHT>& x) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float scale = exponent<EIGHT>(x.e[P], j);
#pragma unroll
            for (int c = 0; c < Q::w / 2; ++c) to.v[j][Q::regs + c] = __builtin_bit_cast(uint32_t, two_channels(x.c[j][P], scale, c));
        }
        expand_values<D, EIGHT, P + 1>(to, x);
    }
}

// A row's query, its channels in the order of the keys': where the 8 of its k-th register of four are.
template <int D>
__device__ constexpr uint32_t query_channel(int k, uint32_t g) {
    uint32_t at = 0;
    for (int p = 0; p < piece_count(D); ++p) {
        const int before = piece_before(D, p), w = (piece_before(D, p + 1) - before) / 16;
        if (k >= before / 32) at = before + 4 * w * g + 8 * (k - before / 32);
    }
    return at;
}
template <int D>
__device__ inline void load_query(uint4v (&q)[D / 32], const uint16_t* row, uint32_t g) {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) q[k] = *reinterpret_cast<const uint4v*>(row + query_channel<D>(k, g));
}

}  // namespace kvc
