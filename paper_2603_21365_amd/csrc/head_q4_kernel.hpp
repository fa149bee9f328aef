// The LM head in four bits: a weight is s (c - 8), c of four bits, s a 16-bit scale that `group` columns of a row share.
//
// The codes' layout is the matrix cores'.  A tile is 16 rows of the head and 128 columns, 1024 bytes, 16 for each lane of a wave; lane l has row l % 16, and in its
// dword j the eight columns 32 j + 8 (l / 16) ..+7: what it supplies to the 16 x 16 x 32 matrix step on the tile's columns 32 j ..+31.  Within a dword column 2i has bits
// 4i ..+3 and column 2i + 1 bits 16 + 4i ..+3, and one mask takes the same nibble of both.
// A group's sum is
//     sum x (c - 8) = 16 sum x ((c - 8) / 16),
// the operands (c - 8) / 16 and the products exact, the sums in fp32, and the scale is applied to it in fp32.  No weight is rounded, and a column whose weight is zero adds
// nothing, neither to a sum nor to its roundings.  (Operands 1 + c / 16, a shift and an and-or for two, with sums that start from -1.5 sum x, save six instructions of
// fourteen for eight codes in bf16, but round every sum at the size of 24 |x| whatever the weights are: twelve columns of no weight, 5000 times as large as the others, made
// errors of 2e-4 to 4e-4 of the logits in the mean square, where these are 5e-8 to 9e-8 with and without such columns.)
#pragma once
#include <type_traits>

#include "device_utils.hpp"

namespace tide {

constexpr int kQ4Rows = 16, kQ4Cols = 128, kQ4TileBytes = 1024;
constexpr int kQ4Threads = 256;

__device__ __forceinline__ float q4_scale(uint32_t bits, bool half) {
    return half ? (float)__builtin_bit_cast(_Float16, (uint16_t)bits) : bf16_bits_to_f32(bits);
}

// The same where `half` is all ones or zero, without a branch.
__device__ __forceinline__ float q4_scale_select(uint32_t bits, uint32_t half) {
    const uint32_t a = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)bits)), b = bits << 16;
    return __uint_as_float((a & half) | (b & ~half));
}

// Two values rounded to 16 bits.
template <int DT> __device__ __forceinline__ uint32_t q4_pair(float a, float b) {
    if constexpr (DT == kBF16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

// The columns col + 32 j ..+7, j = 0 .. 3, of row t, as they lie in memory; zeros beyond the row and the rows.
struct Q4Rows {
    const char* x;
    int64_t row_bytes;
    int T, d;
    bool chunks;               // bases and strides in 16-byte chunks
};
template <int DT> struct Q4Raw {
    u32x4 c[4][Storage<DT>::kBytes / 2];
};
template <int DT> __device__ __forceinline__ void q4_raw(const Q4Rows& p, int t, int col, Q4Raw<DT>& raw) {
    constexpr int kB = Storage<DT>::kBytes;
    const char* row = p.x + (int64_t)t * p.row_bytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = col + 32 * j;
#pragma unroll
        for (int h = 0; h < kB / 2; ++h) raw.c[j][h] = u32x4{0, 0, 0, 0};
        if (t >= p.T || at >= p.d) continue;
        if (p.chunks && at + 8 <= p.d) {
#pragma unroll
            for (int h = 0; h < kB / 2; ++h) raw.c[j][h] = *reinterpret_cast<const u32x4*>(row + (int64_t)at * kB + 16 * h);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (at + e >= p.d) continue;
                if constexpr (DT == kF32) raw.c[j][e / 4][e % 4] = *reinterpret_cast<const uint32_t*>(row + (int64_t)(at + e) * 4);
                else raw.c[j][0][e / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(row + (int64_t)(at + e) * 2) << (16 * (e % 2));
            }
        }
    }
}
// Eight of them in 32 bits, the sum of their magnitudes, and the bits of the largest magnitude (infinities and NaN above all else).
template <int DT> __device__ __forceinline__ void q4_values(const u32x4 (&c)[Storage<DT>::kBytes / 2], float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (DT == kF32) {
            x[e] = __uint_as_float(c[0][e]);
            x[4 + e] = __uint_as_float(c[1][e]);
        } else if constexpr (DT == kBF16) {
            x[2 * e] = __uint_as_float(c[0][e] << 16);
            x[2 * e + 1] = __uint_as_float(c[0][e] & 0xffff0000u);
        } else {
            const f16x2 h = __builtin_bit_cast(f16x2, (uint32_t)c[0][e]);
            x[2 * e] = (float)h[0];
            x[2 * e + 1] = (float)h[1];
        }
    }
}
template <int DT> __device__ __forceinline__ float q4_size8(const u32x4 (&c)[Storage<DT>::kBytes / 2]) {
    float x[8];
    q4_values<DT>(c, x);
    return ((fabsf(x[0]) + fabsf(x[1])) + (fabsf(x[2]) + fabsf(x[3]))) + ((fabsf(x[4]) + fabsf(x[5])) + (fabsf(x[6]) + fabsf(x[7])));
}
template <int DT> __device__ __forceinline__ uint32_t q4_most8(const u32x4 (&c)[Storage<DT>::kBytes / 2]) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    if constexpr (DT == kF32) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) m = max(m, max(c[0][e] & 0x7fffffffu, c[1][e] & 0x7fffffffu));
        return m;
    } else {
        u16x2 m = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, c[0][e] & 0x7fff7fffu));
        const uint32_t bits = max((uint32_t)m[0], (uint32_t)m[1]);
        return DT == kBF16 ? bits << 16 : __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)bits));
    }
}

struct Q4WeightParams {
    Q4Rows x;                  // quantise: the weights, V rows
    char* W_out;               // read back
    int64_t row_bytes;
    char* codes;
    uint16_t* scales;
    int V, d, blocks, groups;  // tiles of 128 columns; groups of a row
    bool half, chunks;         // scales in fp16; rows in 16-byte chunks
    int64_t tiles;
};

// The largest magnitude (its bits: infinities and NaN above all else) of the lane's values in each of the tile's groups.
template <int kRuns> __device__ __forceinline__ void q4_group_max(uint32_t (&most)[4]) {
#pragma unroll
    for (int j = 0; j < 4; j += kRuns) {
        uint32_t m = most[j];
#pragma unroll
        for (int i = 1; i < kRuns; ++i) m = max(m, most[j + i]);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, kWave));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, kWave));
#pragma unroll
        for (int i = 0; i < kRuns; ++i) most[j + i] = m;
    }
}

// The scale of a group whose largest magnitude is `most`: most / 7, rounded once.  The quotient is first rounded to odd (its last bit set where it is not exact, by the
// sign of the exact remainder), so that the rounding to the scale's type sees on which side of a midpoint it lies.
__device__ __forceinline__ uint32_t q4_scale_bits(uint32_t most, bool half) {
    const float a = __uint_as_float(most), q = a / 7.0f, rest = fmaf(-7.0f, q, a);
    uint32_t bits = __float_as_uint(q);
    if (rest != 0.0f) bits = (rest < 0.0f ? bits - 1 : bits) | 1;
    const float odd = __uint_as_float(bits);
    uint32_t s = half ? __builtin_bit_cast(uint16_t, (_Float16)odd) : __builtin_bit_cast(uint16_t, (__bf16)odd);
    const bool lost = most >= 0x7f800000u || s == (half ? 0x7c00u : 0x7f80u);
    return lost ? (half ? 0x7e00u : 0x7fc0u) : s;
}
// Eight weights' codes in a word: w / s to the nearest integer, ties to even, within +-7.  The product with the reciprocal, improved by its exact remainder, is the quotient rounded
// once.  Weights of 16 bits: their quotients by a scale are halves of integers or further than 2^-20 from one, so rounding it again is exact.  fp32: the remainder after
// the nearest integer, exact as well, says whether it was; a quotient so near to a tie is rare enough for a branch.  `s` and `inv`: zero where the codes are to be 8.
template <int DT> __device__ __forceinline__ uint32_t q4_codes(const float (&w)[8], float s, float inv) {
    float q[8];
    bool ties = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float t = w[e] * inv;
        if constexpr (DT != kF32) t = fmaf(fmaf(-t, s, w[e]), inv, t);
        q[e] = __builtin_amdgcn_fmed3f(rintf(t), -7.0f, 7.0f);
        if constexpr (DT == kF32) ties |= fabsf(fmaf(-q[e], s, w[e])) >= 0.5f * s;
    }
    if constexpr (DT == kF32) {
        if (ties) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float rest = fmaf(-q[e], s, w[e]), off = fabsf(rest) - 0.5f * s;
                const bool odd = (int)q[e] & 1;
                if (off > 0.0f || (off == 0.0f && odd)) q[e] = __builtin_amdgcn_fmed3f(q[e] + copysignf(1.0f, rest), -7.0f, 7.0f);
            }
        }
    }
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) word |= (uint32_t)(q[e] + 8.0f) << (4 * (e >> 1) + 16 * (e & 1));
    return word;
}

// A wave per tile: read once, quantised in registers (bf16, 128000 x 4096, groups of 128 / 32: 245 / 232 us, 5.4 / 5.8 TB/s).
template <int DT, int kRuns> __global__ __launch_bounds__(kQ4Threads) void tide_head_quantize_kernel(Q4WeightParams p) {
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.tiles) return;
    const int lane = threadIdx.x % kWave, g = lane >> 4, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks), v = tile * kQ4Rows + (lane & 15);
    Q4Raw<DT> raw;
    q4_raw<DT>(p.x, v, kb * kQ4Cols + 8 * g, raw);
    uint32_t most[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) most[j] = q4_most8<DT>(raw.c[j]);
    q4_group_max<kRuns>(most);
    // a scale for each group: of the 16 lanes of four that have a group's largest magnitudes, those of number g make that of group g (mod the number of groups)
    constexpr int kPer = 4 / kRuns;
    uint32_t mine = most[0];
#pragma unroll
    for (int gr = 1; gr < kPer; ++gr) mine = g % kPer == gr ? most[gr * kRuns] : mine;
    const uint32_t sb = q4_scale_bits(mine, p.half);
    if (g < kPer && kb * kPer + g < p.groups) p.scales[((int64_t)tile * p.groups + kb * kPer + g) * kQ4Rows + (lane & 15)] = (uint16_t)sb;
    float s = q4_scale(sb, p.half);
    const bool some = s > 0.0f;                        // neither zero nor NaN
    // tiny ones: scale and weights a power of two larger, so that the reciprocal is finite and the remainders exact
    const float up = !some ? 0.0f : s < 0x1p-100f ? 0x1p64f : 1.0f;
    s = some ? s * up : 0.0f;
    const float inv = some ? 1.0f / s : 0.0f;
    u32x4 out;
#pragma unroll
    for (int gr = 0; gr < kPer; ++gr) {
        const int from = gr * 16 + (lane & 15);
        const float s_gr = kPer == 1 ? s : __shfl(s, from, kWave), inv_gr = kPer == 1 ? inv : __shfl(inv, from, kWave), up_gr = kPer == 1 ? up : __shfl(up, from, kWave);
#pragma unroll
        for (int j = gr * kRuns; j < (gr + 1) * kRuns; ++j) {
            float x[8];
            q4_values<DT>(raw.c[j], x);
            if (up_gr != 1.0f) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = up_gr != 0.0f ? x[e] * up_gr : 0.0f;
            }
            out[j] = q4_codes<DT>(x, s_gr, inv_gr);
        }
    }
    *reinterpret_cast<u32x4*>(p.codes + at * kQ4TileBytes + lane * 16) = out;
}

// A wave per tile: the values that codes and scales stand for, each rounded once.  A lane makes 16 bytes at a time, and the lanes whole rows of the tile, one after the other (bf16,
// 128000 x 4096: 198 us, 6.6 TB/s; in the codes' order, stores of 64 bytes of a row, 317; with stores that stay in L2 239).
template <int DT, int kRuns> __global__ __launch_bounds__(kQ4Threads) void tide_head_dequantize_kernel(Q4WeightParams p) {
    constexpr int kB = Storage<DT>::kBytes, N = 16 / kB, kLanes = kQ4Cols / N, kStores = kQ4Rows * kLanes / kWave;
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.tiles) return;
    const int lane = threadIdx.x % kWave, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks);
    const int octet = lane % kLanes * N / 8, half = DT == kF32 ? lane & 1 : 0, j = octet >> 2, g = octet & 3, col = kb * kQ4Cols + lane % kLanes * N, row0 = lane / kLanes;
    const int group = min((kb * 4 + j) / kRuns, p.groups - 1);
    uint32_t codes[kStores], scales[kStores];
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
        const int row = row0 + i * (kQ4Rows / kStores);
        codes[i] = *reinterpret_cast<const uint32_t*>(p.codes + at * kQ4TileBytes + (g * 16 + row) * 16 + j * 4);
        scales[i] = p.scales[((int64_t)tile * p.groups + group) * kQ4Rows + row];
    }
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
        const int v = tile * kQ4Rows + row0 + i * (kQ4Rows / kStores);
        const float s = q4_scale(scales[i], p.half);
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int k = e + half * 4;
            x[e] = s * (float)((int)(codes[i] >> (4 * (k >> 1) + 16 * (k & 1)) & 15u) - 8);
        }
        if (v >= p.V || col >= p.d) continue;
        char* out = p.W_out + (int64_t)v * p.row_bytes + (int64_t)col * kB;
        if (p.chunks && col + N <= p.d) {
            u32x4 c;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (DT == kF32) c[e] = __float_as_uint(x[e]);
                else c[e] = q4_pair<DT>(x[2 * e], x[2 * e + 1]);
            }
            __builtin_nontemporal_store(c, reinterpret_cast<u32x4*>(out));
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (col + e >= p.d) continue;
                if constexpr (DT == kF32) *reinterpret_cast<float*>(out + e * 4) = x[e];
                else *reinterpret_cast<uint16_t*>(out + e * 2) = (uint16_t)q4_pair<DT>(x[e], 0.0f);
            }
        }
    }
}

template <int E> __device__ __forceinline__ f32x4 q4_mma(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (E == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// Eight codes as numbers (c - 8) / 16, in pairs.
//   fp16  a nibble in the lowest mantissa bits of 64, whose steps are 1/16, or in the next four of 4, and a packed subtraction of 64.5 or 4.5: a shift, four and-or and four
//         subtractions.  (The constants from registers, as the and-or takes no literals.)
//   bf16  there is no packed arithmetic of that type: with its top bit turned a code is a signed number of four bits, which one instruction makes a float of a 16th of (of a byte's
//         lower nibble); the upper halves of two are a pair.  Fourteen instructions.
template <int B> __device__ __forceinline__ float q4_sixteenths(uint32_t w) { return __builtin_amdgcn_cvt_off_f32_i4(B == 0 ? w : B == 3 ? w >> 24 : w >> 8 * B & 0xffu); }
template <int E> struct Q4Centred {
    __device__ __forceinline__ u32x4 expand(uint32_t w) const {
        const uint32_t u = w ^ 0x88888888u;
        uint32_t v = u >> 4;
        asm("" : "+v"(v));                             // (so that its bytes stay bytes, which the conversion can select, and do not become fields of u, which it cannot)
        auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
        return u32x4{pair(q4_sixteenths<0>(u), q4_sixteenths<2>(u)), pair(q4_sixteenths<0>(v), q4_sixteenths<2>(v)), pair(q4_sixteenths<1>(u), q4_sixteenths<3>(u)),
                     pair(q4_sixteenths<1>(v), q4_sixteenths<3>(v))};
    }
};
template <> struct Q4Centred<kF16> {
    uint32_t low = 0x000f000fu, next = 0x00f000f0u, sixty_four = 0x54005400u, four = 0x44004400u;
    __device__ __forceinline__ Q4Centred() { asm("" : "+s"(low), "+s"(next), "+v"(sixty_four), "+v"(four)); }
    __device__ __forceinline__ u32x4 expand(uint32_t w) const {
        const uint32_t v = w >> 8;
        const f16x2 a = {(_Float16)64.5f, (_Float16)64.5f}, b = {(_Float16)4.5f, (_Float16)4.5f};
        auto less = [](uint32_t bits, f16x2 by) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, bits) - by); };
        return u32x4{less((w & low) | sixty_four, a), less((w & next) | four, b), less((v & low) | sixty_four, a), less((v & next) | four, b)};
    }
};
// fp32 rows are three bf16 planes that add up to them exactly: the first eight significant bits, the next eight, the last eight, cut off and not rounded, so that none is
// larger than the value.
template <int DT> constexpr int kQ4Planes = DT == kF32 ? 3 : 1;
template <int DT> constexpr int kQ4Elem = DT == kF32 ? (int)kBF16 : DT;
// A group has a sum of its first plane's products and another of the rest's: the first's terms have few bits, so that it is all but exact, and the other is 2^-8 of it, and so are
// its roundings.
template <int DT> constexpr int kQ4Sums = DT == kF32 ? 2 : 1;

// ---- Rows under a head in four bits: what the two kernels share.

// The operands of a block of 128 columns from what four groups of lanes, `apart` lanes each, have of its rows: fragment j, plane to x + (j planes + plane) * step.  Where a row's
// magnitudes in a group of columns add up to 2^126 or more (infinities, NaN) its values there are NaN, so that no logit of the row is a number; below that no sum of a group's
// products leaves the range.
template <int DT, int kRuns> __device__ __forceinline__ void q4_put(const Q4Raw<DT>& raw, int apart, char* x, int step) {
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += kRuns) {
        float size = 0.0f;
#pragma unroll
        for (int j = j0; j < j0 + kRuns; ++j) size += q4_size8<DT>(raw.c[j]);
        size += __shfl_xor(size, apart, kWave);
        size += __shfl_xor(size, 2 * apart, kWave);
        const uint32_t nan = size < 0x1p126f ? 0u : 0x7fff7fffu;
#pragma unroll
        for (int j = j0; j < j0 + kRuns; ++j) {
            if constexpr (DT == kF32) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(raw.c[j][e / 4][e % 4]);
#pragma unroll
                for (int plane = 0; plane < 3; ++plane) {
                    u32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t a = __float_as_uint(y[2 * e]) & 0xffff0000u, b = __float_as_uint(y[2 * e + 1]) & 0xffff0000u;
                        v[e] = a >> 16 | b | nan;
                        y[2 * e] -= __uint_as_float(a);
                        y[2 * e + 1] -= __uint_as_float(b);
                    }
                    *reinterpret_cast<u32x4*>(x + (j * 3 + plane) * step) = v;
                }
            } else {
                *reinterpret_cast<u32x4*>(x + j * step) = raw.c[j][0] | u32x4{nan, nan, nan, nan};
            }
        }
    }
}

struct Q4Head {
    const char* codes;
    const uint16_t* scales;
    int V, tiles, blocks, groups;
    bool half;                 // scales in fp16
};
// The scales of NT tiles in a wave's kilobyte of LDS: 32 / NT groups of each, 32 bytes a group; lane l brings eight rows of one.
template <int NT> __device__ __forceinline__ u32x4 q4_scales(const Q4Head& h, int tile0, int group0, int lane) {
    constexpr int kLanes = kWave / NT;
    const int tile = min(tile0 + lane / kLanes, h.tiles - 1), l = lane % kLanes, group = min(group0 + l / 2, h.groups - 1);      // (a group of padding: its sums are zero)
    return *reinterpret_cast<const u32x4*>(h.scales + ((int64_t)tile * h.groups + group) * kQ4Rows + (l & 1) * 8);
}
__device__ __forceinline__ float q4_scale_at(const char* mine, int NT, int n, int group, int lane, uint32_t half) {
    return q4_scale_select(*reinterpret_cast<const uint16_t*>(mine + n * (1024 / NT) + group * 32 + (lane & 15) * 2), half);
}

// Where a launch would leave CUs idle, or where not all columns of a few rows fit in LDS, workgroups have a part of the columns, by blockIdx.y, and another launch adds up their sums.
struct Q4JoinParams {
    const float* part;         // [parts][T][V]
    float* out;
    int64_t out_stride;
    int T, V, parts, pieces;   // of a row
};
constexpr int kQ4JoinRun = 4;
__global__ __launch_bounds__(kQ4Threads) void tide_head_q4_join_kernel(Q4JoinParams p) {
    const int t = blockIdx.x / p.pieces, v0 = (blockIdx.x - t * p.pieces) * kQ4JoinRun * kQ4Threads + threadIdx.x;
    const int64_t all = (int64_t)p.T * p.V;
    float sum[kQ4JoinRun] = {};
    for (int part = 0; part < p.parts; ++part)
#pragma unroll
        for (int e = 0; e < kQ4JoinRun; ++e) {
            const int v = v0 + e * kQ4Threads;
            if (v < p.V) sum[e] += p.part[part * all + (int64_t)t * p.V + v];
        }
#pragma unroll
    for (int e = 0; e < kQ4JoinRun; ++e) {
        const int v = v0 + e * kQ4Threads;
        if (v < p.V) p.out[(int64_t)t * p.out_stride + v] = sum[e];
    }
}

// ---- Few rows, up to 16: all of them in LDS.
//
// A workgroup lays the rows out once -- as fragments, 16 bytes (eight columns) of each row side by side -- and its waves then stream tiles of codes, each wave NT tiles at a
// time, kDepth blocks of 128 columns ahead.  The scales come a kilobyte at a time through LDS (a load of each step's scales, 32 bytes of use, cost 4 of 50 us at one row, 128000 x 4096).
// Where there are few tokens, `split` waves share the columns of a wave's tiles and add up their sums, in order, through LDS.
// Bound by reading the codes and making operands of them, which take 34 of these us in vector instructions (bf16, 128000 x 4096, groups of 128: 51 us at one row, 5.3 TB/s with
// the scales, 54 at 8, 56 at 16; a pure read of as much 41).
struct Q4FewParams {
    Q4Rows x;
    Q4Head head;
    float* out;
    int64_t out_stride, part_stride;
    int part_blocks;           // of 128 columns, of a part
    int sets;                  // of tokens, each a workgroup's at a time
    int rows_log;              // rows in LDS: a power of two
    int split;
};
constexpr int kQ4FewThreads = 1024;

struct Q4FewLds {
    int scales, sums, bytes;
};
template <int DT, int NT> __host__ __device__ inline Q4FewLds q4_few_lds(int rows_log, int blocks, int waves, int split) {
    Q4FewLds l{};
    l.scales = blocks * 4 * kQ4Planes<DT> * (64 << rows_log);
    l.sums = l.scales + waves * 1024;
    l.bytes = l.sums + (split > 1 ? waves * NT * 1024 : 0);
    return l;
}

// (One tile a wave: up to 72 registers, so that seven workgroups of four waves share a CU; fp32 rows' three terms would not fit, and five do.  With 76 one row took 3 % longer.)
template <int DT, int kRuns, int NT, int kDepth> __global__ __launch_bounds__(kQ4FewThreads, NT == 1 && DT != kF32 ? 7 : 4) void tide_head_q4_few_kernel(Q4FewParams p) {
    constexpr int E = kQ4Elem<DT>, P = kQ4Planes<DT>, kSums = kQ4Sums<DT>, kPer = 4 / kRuns;
    constexpr int kScaleBlocks = 32 / NT / kPer;       // blocks of 128 columns whose scales a kilobyte holds
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int log = p.rows_log, rows = 1 << log, all = p.head.blocks, kb0 = blockIdx.y * p.part_blocks, blocks = min(p.part_blocks, all - kb0);
    float* const out = p.out + blockIdx.y * p.part_stride;
    const Q4FewLds at = q4_few_lds<DT, NT>(log, blocks, waves, p.split);

    // the wave's tiles: NT of each set, blocks `begin` ..+`own`.  The first of them are on their way while the rows are laid out
    const int unit = wave / p.split, part = wave - unit * p.split, units = waves / p.split;
    const int begin = part * blocks / p.split, own = (part + 1) * blocks / p.split - begin, first = kb0 + begin;
    const int passes = (p.sets - blockIdx.x + gridDim.x - 1) / gridDim.x;
    auto tile_of = [&](int pass) { return ((int)(blockIdx.x + pass * gridDim.x) * units + unit) * NT; };
    u32x4 c[kDepth][NT];
    int f_pass = 0, f_at = 0;                          // what is fetched next
    const char* f_codes[NT];
    auto point = [&](int pass) {
        const int tile0 = tile_of(pass);
#pragma unroll
        for (int n = 0; n < NT; ++n) f_codes[n] = p.head.codes + ((int64_t)min(tile0 + n, p.head.tiles - 1) * all + first) * kQ4TileBytes;
    };
    point(0);
    auto fetch = [&](int slot) {
#pragma unroll
        for (int n = 0; n < NT; ++n) c[slot][n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(f_codes[n] + (uint32_t)(f_at * kQ4TileBytes) + lane * 16));
        if (++f_at == own) {
            f_at = 0;
            point(++f_pass);
        }
    };
    u32x4 s_next;
    auto fetch_scales = [&](int pass, int i) { s_next = q4_scales<NT>(p.head, tile_of(min(pass, passes - 1)), (first + i) * kPer, lane); };
    const int steps = passes * own;
    fetch_scales(0, 0);
#pragma unroll
    for (int slot = 0; slot < kDepth; ++slot)
        if (slot < steps) fetch(slot);

    for (int item = threadIdx.x; item < blocks * 4 << log; item += blockDim.x) {
        const int row = item & (rows - 1), g = item >> log & 3, kb = item >> (log + 2);
        Q4Raw<DT> raw;
        q4_raw<DT>(p.x, row, (kb0 + kb) * kQ4Cols + 8 * g, raw);
        q4_put<DT, kRuns>(raw, rows, lds + ((kb * 16 * P + g) << (log + 4)) + row * 16, 64 << log);
    }
    __syncthreads();

    const Q4Centred<E> centred;
    const uint32_t half = p.head.half ? 0xffffffffu : 0u;
    const char* const my_x = lds + ((lane >> 4) << (log + 4)) + (lane & (rows - 1)) * 16;
    char* const my_scales = lds + at.scales + wave * 1024;
    f32x4 total[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) total[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int pass = 0, i = 0, s_at = 0;
    auto step = [&](const u32x4 (&now)[NT]) {
        if (s_at == 0) {
            *reinterpret_cast<u32x4*>(my_scales + lane * 16) = s_next;
            if (i + kScaleBlocks < own) fetch_scales(pass, i + kScaleBlocks);
            else fetch_scales(pass + 1, 0);
        }
        const char* x = my_x + ((begin + i) * 4 * P << (log + 6));
#pragma unroll
        for (int gr = 0; gr < kPer; ++gr) {
            f32x4 sum[kSums][NT] = {};
#pragma unroll
            for (int j = gr * kRuns; j < (gr + 1) * kRuns; ++j) {
                u32x4 w[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) w[n] = centred.expand(now[n][j]);
#pragma unroll
                for (int plane = 0; plane < P; ++plane) {
                    const u32x4 a = *reinterpret_cast<const u32x4*>(x + ((j * P + plane) << (log + 6)));
#pragma unroll
                    for (int n = 0; n < NT; ++n) sum[plane > 0][n] = q4_mma<E>(a, w[n], sum[plane > 0][n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float s = q4_scale_at(my_scales, NT, n, s_at * kPer + gr, lane, half);
                if constexpr (kSums > 1) sum[0][n] += sum[1][n];
#pragma unroll
                for (int e = 0; e < 4; ++e) total[n][e] = fmaf(s, sum[0][n][e], total[n][e]);
            }
        }
        if (++s_at == kScaleBlocks) s_at = 0;
        if (++i < own) return;
        if (p.split > 1) {
            f32x4* const sums = reinterpret_cast<f32x4*>(lds + at.sums);
            __syncthreads();                       // (the last pass's sums have been read)
#pragma unroll
            for (int n = 0; n < NT; ++n) sums[(wave * NT + n) * kWave + lane] = total[n];
            __syncthreads();
            if (part == 0)
                for (int m = 1; m < p.split; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const f32x4 more = sums[((wave + m) * NT + n) * kWave + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[n][e] += more[e];
                    }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int v = (tile_of(pass) + n) * kQ4Rows + (lane & 15);
            const bool writes = part == 0 && v < p.head.V;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = 4 * (lane >> 4) + e;
                if (writes && t < p.x.T) out[(int64_t)t * p.out_stride + v] = 16.0f * total[n][e];
                total[n][e] = 0.0f;
            }
        }
        ++pass;
        i = 0;
        s_at = 0;
    };
    // whole rounds of the ring while there is something left to fetch, then what is in it
    int left = steps;
    for (; left >= 2 * kDepth; left -= kDepth)
#pragma unroll
        for (int slot = 0; slot < kDepth; ++slot) {
            u32x4 now[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) now[n] = c[slot][n];
            fetch(slot);
            step(now);
        }
    for (; left > 0; left -= kDepth)
#pragma unroll
        for (int slot = 0; slot < kDepth; ++slot) {
            if (slot >= left) break;
            u32x4 now[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) now[n] = c[slot][n];
            if (slot + kDepth < left) fetch(slot);
            step(now);
        }
}

// ---- Many rows.
//
// The rows are first laid out in memory: for 16 MT rows and 128 columns one region, the fragments.
template <int DT, int MT> constexpr int kQ4Region = 4 * kQ4Planes<DT> * MT * 1024;
struct Q4LayParams {
    Q4Rows x;
    char* out;
    int blocks;
    int64_t waves;             // row tiles of all row blocks, times blocks
};
template <int DT, int kRuns, int MT> __global__ __launch_bounds__(kQ4Threads) void tide_head_q4_lay_kernel(Q4LayParams p) {
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.waves) return;
    const int lane = threadIdx.x % kWave, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks), rb = tile / MT, rt = tile - rb * MT;
    Q4Raw<DT> raw;
    q4_raw<DT>(p.x, tile * 16 + (lane & 15), kb * kQ4Cols + 8 * (lane >> 4), raw);
    q4_put<DT, kRuns>(raw, 16, p.out + ((int64_t)rb * p.blocks + kb) * kQ4Region<DT, MT> + rt * 1024 + lane * 16, MT * 1024);
}

// A workgroup has 16 MT rows and its waves NT tiles of 16 tokens each.  Everything comes to LDS by transfers that no register waits for: the rows' regions in two
// stages, for all waves, behind a barrier for each block of 128 columns; each wave's codes in two or three stages and its scales, a kilobyte at a time, in two.  The
// transfers are inline assembly, which the compiler does not count, and the waits for them are written out; there are no other loads from memory in the loop.
// Some dozen rows are bound by making operands of the codes (two thirds of the vector instructions at 48 rows, which are 38 us) beside the matrix steps (20), many by the matrix
// steps under the power limit (bf16, 128000 x 4096, groups of 128: 48 rows 76 us, 512 rows 467, 1.15 PFLOP/s.  Codes and scales through registers took a fifth longer at
// 48 rows, a tenth at 512).
struct Q4ManyParams {
    const char* regions;
    Q4Head head;
    float* out;
    int64_t out_stride, part_stride;
    int part_blocks;           // of 128 columns, of a part
    int T, row_blocks;
    int sets;                  // of tokens: a workgroup has a set and a row block at a time
    bool by_xcd;               // the row blocks of a set run on one XCD (workgroups whose numbers are equal modulo 8), for its codes to be in that L2
};
// Four tiles a wave, eight waves; or two tiles and sixteen waves
template <int NT> constexpr int kQ4ManyThreads = 2048 / NT;
template <int NT> __host__ __device__ constexpr int q4_many_lds(int region, int stages, int waves) { return 2 * region + waves * (stages * NT + 2) * 1024; }
template <int DT, int MT, int NT> constexpr int kQ4CodeStages = q4_many_lds<NT>(kQ4Region<DT, MT>, 3, kQ4ManyThreads<NT> / kWave) <= 158 * 1024 ? 3 : 2;

// 64 lanes x 16 bytes from memory to a kilobyte of LDS (m0 as in the head products).  The wait states: five between a vector instruction that wrote the base and this one.
__device__ __forceinline__ void q4_transfer(uint32_t lds, const char* base, uint32_t lane_bytes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_bytes), "s"(base) : "memory");
}

template <int DT, int kRuns, int MT, int NT> __global__ __launch_bounds__(kQ4ManyThreads<NT>) void tide_head_q4_many_kernel(Q4ManyParams p) {
    constexpr int E = kQ4Elem<DT>, P = kQ4Planes<DT>, kSums = kQ4Sums<DT>, kPer = 4 / kRuns, kRegion = kQ4Region<DT, MT>, kStages = kQ4CodeStages<DT, MT, NT>, kSteps = kRuns * P, kAhead = 2;
    constexpr int kScaleBlocks = 32 / NT / kPer;       // blocks of 128 columns whose scales a kilobyte holds
    static_assert(kScaleBlocks >= 2, "a kilobyte is requested two blocks before it is read");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int all = p.head.blocks, kb0 = blockIdx.y * p.part_blocks, blocks = min(p.part_blocks, all - kb0);
    const int xcd = p.by_xcd ? blockIdx.x & 7 : 0, xcds = p.by_xcd ? 8 : 1, first_item = blockIdx.x / xcds, stride = gridDim.x / xcds;
    const int items = (p.sets - xcd + xcds - 1) / xcds * p.row_blocks, passes = (items - first_item + stride - 1) / stride;
    if (first_item >= items) return;
    auto item_of = [&](int pass) { return first_item + min(pass, passes - 1) * stride; };
    auto tile_of = [&](int pass) { return ((item_of(pass) / p.row_blocks * xcds + xcd) * waves + wave) * NT; };

    char* const my_codes = lds + 2 * kRegion + wave * (kStages * NT + 2) * 1024;
    char* const my_scales = my_codes + kStages * NT * 1024;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds, lane16 = lane * 16;
    const uint32_t codes0 = lds0 + (uint32_t)(my_codes - lds), scales0 = codes0 + kStages * NT * 1024;
    // the regions of the rows: every wave a part of each
    const char* regions = p.regions + ((int64_t)(item_of(0) % p.row_blocks) * all + kb0) * kRegion;
    int x_pass = 0, x_kb = 0, x_stage = 0;
    auto request_region = [&] {
        const char* from = regions + (int64_t)x_kb * kRegion;
        for (int i = wave * 1024; i < kRegion; i += waves * 1024) q4_transfer(lds0 + x_stage * kRegion + i, from + i, lane16);
        if (++x_kb == blocks) x_kb = 0, regions = p.regions + ((int64_t)(item_of(++x_pass) % p.row_blocks) * all + kb0) * kRegion;
        x_stage ^= 1;
    };
    // the wave's codes; beyond its last block: the last tiles again, into a stage that nothing reads
    int f_pass = 0, f_kb = 0, f_stage = 0, f_tile = tile_of(0);
    auto request_codes = [&] {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            q4_transfer(codes0 + (f_stage * NT + n) * 1024, p.head.codes + ((int64_t)min(f_tile + n, p.head.tiles - 1) * all + kb0 + f_kb) * kQ4TileBytes, lane16);
        if (++f_kb == blocks) f_kb = 0, f_tile = tile_of(++f_pass);
        if (++f_stage == kStages) f_stage = 0;
    };
    // and its scales: lane l brings eight rows of a group, 64 / NT lanes those of a tile
    int s_stage = 0;
    auto request_scales = [&](int pass, int kb) {
        constexpr int kLanes = kWave / NT;
        const int tile0 = tile_of(pass), l = lane % kLanes, tile = min(tile0 + lane / kLanes, p.head.tiles - 1) - min(tile0, p.head.tiles - 1);
        const int group = min((kb0 + kb) * kPer + l / 2, p.head.groups - 1);       // (a group of padding: its sums are zero)
        q4_transfer(scales0 + s_stage * 1024, (const char*)(p.head.scales + (int64_t)min(tile0, p.head.tiles - 1) * p.head.groups * kQ4Rows),
                    ((uint32_t)(tile * p.head.groups + group) * kQ4Rows + (l & 1) * 8) * 2);
        s_stage ^= 1;
    };
    request_scales(0, 0);
    request_region();
#pragma unroll
    for (int i = 1; i < kStages; ++i) request_codes();

    const Q4Centred<E> centred;
    const uint32_t half = p.head.half ? 0xffffffffu : 0u;
    f32x4 total[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int rt = 0; rt < MT; ++rt) total[n][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int stage = 0, c_stage = 0, s_at = 0, s_read = 0;
    for (int pass = 0; pass < passes; ++pass) {
        for (int kb = 0; kb < blocks; ++kb) {
            // What this block reads has arrived: with three stages all but the last request for codes; the wave has read what the next requests overwrite, and behind the
            // barrier so have all
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(kStages == 3 ? NT : 0) : "memory");
            if (s_at == 0) {
                if (kb + kScaleBlocks < blocks) request_scales(pass, kb + kScaleBlocks);
                else request_scales(pass + 1, 0);
            }
            request_region();
            request_codes();
            const char* const x = lds + stage * kRegion + lane * 16;
            u32x4 c[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) c[n] = *reinterpret_cast<const u32x4*>(my_codes + (c_stage * NT + n) * 1024 + lane * 16);
#pragma unroll
            for (int gr = 0; gr < kPer; ++gr) {
                // fragments are read kAhead steps of NT matrix steps ahead of their use; the codes of a step are expanded beside the matrix steps of the
                // one before
                auto fragment = [&](int step) { return *reinterpret_cast<const u32x4*>(x + ((gr * kSteps + step % kSteps) * MT + step / kSteps) * 1024); };
                u32x4 a[kAhead], w[kRuns][NT];
#pragma unroll
                for (int step = 0; step < kAhead; ++step) a[step] = fragment(step);
                float s[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s[n] = q4_scale_at(my_scales + s_read * 1024, NT, n, s_at * kPer + gr, lane, half);
                    w[0][n] = centred.expand(c[n][gr * kRuns]);
                }
#pragma unroll
                for (int rt = 0; rt < MT; ++rt) {
                    f32x4 sum[kSums][NT] = {};
#pragma unroll
                    for (int step = 0; step < kSteps; ++step) {
                        const int at = rt * kSteps + step;
                        const u32x4 now = a[at % kAhead];
                        if (at + kAhead < MT * kSteps) a[at % kAhead] = fragment(at + kAhead);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int n = 0; n < NT; ++n) sum[step % P > 0][n] = q4_mma<E>(now, w[step / P][n], sum[step % P > 0][n]);
                        if (rt == 0 && step % P == 0 && step / P + 1 < kRuns) {
#pragma unroll
                            for (int n = 0; n < NT; ++n) w[step / P + 1][n] = centred.expand(c[n][gr * kRuns + step / P + 1]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (kSums > 1) sum[0][n] += sum[1][n];
                        total[n][rt] = __builtin_elementwise_fma(f32x4{s[n], s[n], s[n], s[n]}, sum[0][n], total[n][rt]);
                        asm volatile("" : "+v"(total[n][rt]));     // here: not behind the next branch, with all sums kept until then
                    }
                }
            }
            stage ^= 1;
            if (++c_stage == kStages) c_stage = 0;
            if (++s_at == kScaleBlocks || kb + 1 == blocks) s_at = 0, s_read ^= 1;
        }
        int quad = 4 * (lane >> 4);
        asm volatile("" : "+v"(quad));                 // (the rows' addresses are made here, not kept over the loop)
#pragma unroll
        for (int rt = 0; rt < MT; ++rt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = (item_of(pass) % p.row_blocks * MT + rt) * 16 + quad + e;
                float* const out = p.out + blockIdx.y * p.part_stride + (int64_t)t * p.out_stride + (lane & 15);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int v0 = (tile_of(pass) + n) * kQ4Rows;
                    if (t < p.T && v0 + (lane & 15) < p.head.V) out[v0] = 16.0f * total[n][rt][e];
                    total[n][rt][e] = 0.0f;
                }
            }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last transfers: the LDS is another workgroup's afterwards
}

}  // namespace tide
