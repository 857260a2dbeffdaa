// Rows into a cache held in 4 bits, and its blocks back to FP16.
//
// A magnitude is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e, e of 32 channels of a token.  gfx950 converts pairs both ways in one instruction, to the nearest (halfway to the even
// code), beyond 6 to 6; a test compares them with the definition for every finite FP16 value.  2^e times a code that comes out is an FP16 number, as e is 13 at most and FP16 values are
// multiples of 2^-24, of which the smallest make codes of 1, 2, 3, 4 and 6 alone.
#include "kvc_fp4.h"

namespace kvc {

typedef _Float16 half2f __attribute__((ext_vector_type(2)));

// (a value of its own: of a vector's element the compiler takes the first one's bits)
__device__ inline half2f pair(uint32_t v) { return __builtin_bit_cast(half2f, v); }

// Exponent byte of a group whose largest magnitude has the FP16 bits m: the smallest e with m <= 7 * 2^e, so that nothing is off by more than 2^e; 13 at most, so that 4 * 2^e is an FP16 number.
__device__ inline uint32_t exponent_byte(uint32_t m) {
    const uint32_t bits = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)m));
    const uint32_t e = ((bits + 0x1FFFFF) >> 23) - 2;  // (7 * 2^e is 1.75 * 2^(e+2): a larger mantissa goes on to the next power)
    return m == 0 ? 0 : min(e, 140u);
}

// What 8 channels of a row become: codes, and the exponent of the 32 channels that four lanes have.
struct Packed {
    uint32_t codes, exp;
};
__device__ inline Packed packed(const uint4v& r) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, max(r[j] & 0x7FFFu, r[j] >> 16 & 0x7FFFu));
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    const bool finite = m < 0x7C00;
    Packed p;
    p.exp = finite ? exponent_byte(m) : 255;
    const float scale = __uint_as_float(finite && m ? p.exp << 23 : 127u << 23);
    p.codes = 0;
    p.codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(p.codes, pair(r[0]), scale, 0);
    p.codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(p.codes, pair(r[1]), scale, 1);
    p.codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(p.codes, pair(r[2]), scale, 2);
    p.codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(p.codes, pair(r[3]), scale, 3);
    p.codes = finite ? p.codes : 0;
    return p;
}

// ---- append: a workgroup per T new tokens of a sequence, a lane per 16 bytes of their K and V rows, four lanes to a group of 32 channels.  The rows are asked for first of all, as where they go takes two
// reads that follow from each other (the length, the table).  Bound by memory: of a token, 4 d bytes are read and 17 d / 16 written for each KV head.  512 tokens of each of 16 sequences, 8 KV heads of 128
// channels: 11.8 us, 3.6 TB/s (the exponents are single bytes, 16 tokens' side by side; a workgroup per page's 16 positions would write them together, but takes 17.1 us to the 13.6 that this took then, as
// it has fewer rows on their way); one token of 4 x 64 2.2 us.
template <uint32_t T>
__global__ __launch_bounds__(256) void k_append_fp4(AppendFp4Args x) {
    const AppendArgs& a = x.a;
    __shared__ int64_t block_at[T];  // bytes from the beginning of a cache to the token's block; -1: no place
    __shared__ uint32_t row_at[T];
    const uint32_t s = fast_div(blockIdx.x, x.by_turns), i0 = (blockIdx.x - s * x.turns) * T, tid = threadIdx.x, n = min(T, (uint32_t)a.n_new - i0);
    const uint32_t each = (uint32_t)(a.n_kv * a.g.lpr), N = (uint32_t)a.g.N;  // (a multiple of 4, so a group's lanes are there together)
    for (uint32_t c0 = 0; c0 < 2 * each; c0 += blockDim.x) {
        const uint32_t c = c0 + tid;
        const bool v = c >= each;
        const uint32_t e = v ? c - each : c, h = fast_div(e, a.by_lpr), k = e - h * (uint32_t)a.g.lpr;
        const int64_t* strides = v ? a.v_strides : a.k_strides;
        const uint16_t* from = (v ? a.v_new : a.k_new) + s * strides[0] + h * strides[2] + 8 * k;
        uint4v r[T];
#pragma unroll
        for (uint32_t i = 0; i < T; ++i) {
            r[i] = uint4v{0, 0, 0, 0};
            if (c < 2 * each && i < n) r[i] = *reinterpret_cast<const uint4v*>(from + (i0 + i) * strides[1]);
        }
        if (c0 == 0) {
            if (tid < n) {
                const int64_t t = (int64_t)a.lens[s] - a.n_new + i0 + tid;
                int64_t at = -1;
                if (t >= 0) {
                    const uint32_t entry = fast_div((uint32_t)t, a.by_N);
                    row_at[tid] = (uint32_t)t - entry * N;
                    const bool beyond = entry >= (uint32_t)a.max_blocks;
                    const int32_t block = beyond ? -1 : a.table[(int64_t)s * a.max_blocks + entry];
                    if (beyond || block >= a.n_cache_blocks) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
                    else if (block >= 0) at = block * x.f.block;
                }
                block_at[tid] = at;
            }
            __syncthreads();
        }
        if (c >= 2 * each) break;
        uint8_t* pages = (v ? x.v_cache : x.k_cache) + (int64_t)h * x.f.page;
#pragma unroll
        for (uint32_t i = 0; i < T; ++i) {
            if (i >= n || block_at[i] < 0) continue;  // (for all lanes alike)
            const Packed p = packed(r[i]);
            uint8_t* page = pages + block_at[i];
            *reinterpret_cast<uint32_t*>(page + row_at[i] * (uint32_t)(a.g.d / 2) + 4 * k) = p.codes;
            if ((k & 3) == 0) page[x.f.exps + k / 4 * N + row_at[i]] = (uint8_t)p.exp;
        }
    }
}

constexpr int64_t kUnpackKept = 32 << 20;  // bytes of a call whose stores the caches keep

// ---- unpack: a workgroup per 16 KB of FP16, a lane per 8 channels, four of them on their way before the first store.  Bound by memory: 64 MB of FP16 from 17.8 MB 11.1 us, the stores at 5.7 TB/s.
// PAST: stores go past the caches, where there are many: a prompt chunk's 64 MB behind an append 22.4 us with it, 25.9 without, 59 MB in two calls 17.9 and 17.8, 256 KB 11.3 and 9.7.
template <bool PAST>
__global__ __launch_bounds__(256) void k_unpack_fp4(UnpackFp4Args a) {
    const uint32_t i = fast_div(blockIdx.x, a.by_pieces), piece = blockIdx.x - i * (uint32_t)a.pieces;
    const int32_t src = a.src ? a.src[i] : (int32_t)i, dst = a.dst ? a.dst[i] : (int32_t)i;
    if (src < 0 || dst < 0) return;
    if (src >= a.n_cache_blocks || dst >= a.n_out_blocks) {
        if (threadIdx.x == 0) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
        return;
    }
    const uint8_t* x = a.cache + src * a.f.block;
    uint16_t* y = a.out + dst * a.g.block_stride;
    uint32_t codes[kCopyChunks / 256], exps[kCopyChunks / 256];
    int64_t at[kCopyChunks / 256];
#pragma unroll
    for (int k = 0; k < kCopyChunks / 256; ++k) {
        const uint32_t c = piece * kCopyChunks + k * 256 + threadIdx.x;
        at[k] = -1;
        codes[k] = exps[k] = 0;
        if (c < (uint32_t)a.chunks) {
            const uint32_t line = fast_div(c, a.by_lpr), in_row = c - line * (uint32_t)a.g.lpr, page = fast_div(line, a.by_N), row = line - page * (uint32_t)a.g.N;
            const uint8_t* p = x + (int64_t)page * a.f.page;
            codes[k] = reinterpret_cast<const uint32_t*>(p + row * (uint32_t)(a.g.d / 2))[in_row];
            exps[k] = p[a.f.exps + in_row / 4 * (uint32_t)a.g.N + row];
            at[k] = page * a.g.page_stride + row * a.g.row_stride + 8 * in_row;
        }
    }
#pragma unroll
    for (int k = 0; k < kCopyChunks / 256; ++k) {
        const float scale = __uint_as_float(exps[k] << 23);
        uint4v r;
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes[k], scale, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes[k], scale, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes[k], scale, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes[k], scale, 3));
        if (at[k] < 0) continue;
        if (PAST) __builtin_nontemporal_store(r, reinterpret_cast<uint4v*>(y + at[k]));
        else *reinterpret_cast<uint4v*>(y + at[k]) = r;
    }
}

hipError_t launch_append_fp4(const AppendFp4Args& a, hipStream_t s) {
    const unsigned threads = (unsigned)std::min<int64_t>(256, (2ll * a.a.n_kv * a.a.g.lpr + 63) / 64 * 64);
    return launch_kernel(a.wide ? k_append_fp4<kTurn> : k_append_fp4<1>, dim3((unsigned)a.a.n_seq * a.turns), dim3(threads), s, a);
}
hipError_t launch_unpack_fp4(const UnpackFp4Args& a, hipStream_t s) {
    const bool past = (int64_t)a.n * a.chunks * 16 > kUnpackKept;
    return launch_kernel(past ? k_unpack_fp4<true> : k_unpack_fp4<false>, dim3((unsigned)a.pieces * (unsigned)a.n), dim3(256), s, a);
}

}  // namespace kvc
