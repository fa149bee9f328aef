// The LM head in four bits: a weight is s (c - 8), c of four bits, s a 16-bit scale that `group` columns of a row share.
//
// The codes' layout is the matrix cores'.  A tile is 16 rows of the head and 128 columns, 1024 bytes, 16 for each lane of a wave; lane l has row l % 16, and in its
// dword j the eight columns 32 j + 8 (l / 16) ..+7: what it supplies to the 16 x 16 x 32 matrix step on the tile's columns 32 j ..+31.  Within a dword column 2i has bits
// 4i ..+3 and column 2i + 1 bits 16 + 4i ..+3, so that one shift and one and-or make a pair of adjacent 16-bit values:
// the code in the top mantissa bits of a number in [1, 2), 1 + c / 16.  A group's sum is then
//     sum x (c - 8) = 16 (sum x (1 + c / 16) - 1.5 sum x),
// the products exact, the sums in fp32, and the scale is applied to it in fp32.  No weight is rounded.
#pragma once
#include "device_utils.hpp"

namespace tide {

constexpr int kQ4Rows = 16, kQ4Cols = 128, kQ4TileBytes = 1024;
constexpr int kQ4Threads = 256;

__device__ __forceinline__ float q4_scale(uint32_t bits, bool half) {
    return half ? (float)__builtin_bit_cast(_Float16, (uint16_t)bits) : bf16_bits_to_f32(bits);
}

// Elements col .. col+7 of a row, zeros from d on.
template <int DT> __device__ __forceinline__ void q4_load8(const char* row, int col, int d, bool chunks, float (&x)[8]) {
    constexpr int kB = Storage<DT>::kBytes;
    if (chunks && col + 8 <= d) {
#pragma unroll
        for (int h = 0; h < kB / 2; ++h) {
            const u32x4 c = *reinterpret_cast<const u32x4*>(row + (int64_t)col * kB + 16 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (DT == kF32) {
                    x[4 * h + e] = __uint_as_float(c[e]);
                } else if constexpr (DT == kBF16) {
                    x[2 * e] = __uint_as_float(c[e] << 16);
                    x[2 * e + 1] = __uint_as_float(c[e] & 0xffff0000u);
                } else {
                    const f16x2 p = __builtin_bit_cast(f16x2, (uint32_t)c[e]);
                    x[2 * e] = (float)p[0];
                    x[2 * e + 1] = (float)p[1];
                }
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = 0.0f;
        if (col + e < d) {
            const char* p = row + (int64_t)(col + e) * kB;
            if constexpr (DT == kF32) x[e] = *reinterpret_cast<const float*>(p);
            else if constexpr (DT == kBF16) x[e] = bf16_bits_to_f32(*reinterpret_cast<const uint16_t*>(p));
            else x[e] = (float)*reinterpret_cast<const _Float16*>(p);
        }
    }
}
// Two values rounded to 16 bits.
template <int DT> __device__ __forceinline__ uint32_t q4_pair(float a, float b) {
    if constexpr (DT == kBF16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

struct Q4WeightParams {
    const char* W;             // quantise: in; read back: unused
    char* W_out;
    int64_t row_bytes;
    char* codes;
    uint16_t* scales;
    int V, d, blocks, groups;  // tiles of 128 columns; groups of a row
    int per_block;             // waves' tiles in a row of tiles: blocks, for the index arithmetic
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
// The code of a weight: |w| / s to the nearest integer, ties to even, at most 7.  The quotient only proposes the integer below; on which side of the half
// the weight lies is the sign of one fused multiply-add, which no rounding changes.
__device__ __forceinline__ uint32_t q4_code(float w, float s, float inv) {
    const float a = fabsf(w), k = fminf(floorf(a * inv), 7.0f), r = fmaf(-(k + 0.5f), s, a);
    int q = (int)k;
    if (r > 0.0f || (r == 0.0f && (q & 1))) ++q;
    q = min(q, 7);
    return (uint32_t)(8 + (w < 0.0f ? -q : q));
}

// A wave per tile: read once, quantised in registers.
template <int DT, int kRuns> __global__ __launch_bounds__(kQ4Threads) void tide_head_quantize_kernel(Q4WeightParams p) {
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.tiles) return;
    const int lane = threadIdx.x % kWave, g = lane >> 4, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks), v = tile * kQ4Rows + (lane & 15);
    float x[4][8];
    uint32_t most[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = 0.0f;
        if (v < p.V) q4_load8<DT>(p.W + (int64_t)v * p.row_bytes, kb * kQ4Cols + 32 * j + 8 * g, p.d, p.chunks, x[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        most[j] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) most[j] = max(most[j], __float_as_uint(x[j][e]) & 0x7fffffffu);
    }
    q4_group_max<kRuns>(most);
    u32x4 out;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t sb = q4_scale_bits(most[j], p.half);
        const int group = (kb * 4 + j) / kRuns;
        if (j % kRuns == 0 && g == 0 && group < p.groups) p.scales[((int64_t)tile * p.groups + group) * kQ4Rows + lane] = (uint16_t)sb;
        float s = q4_scale(sb, p.half);
        const bool some = s > 0.0f;                    // neither zero nor NaN
        const float up = s < 0x1p-100f ? 0x1p64f : 1.0f;      // both a power of two larger, so that the reciprocal is finite
        s *= up;
        const float inv = some ? 1.0f / s : 0.0f;
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) word |= (some ? q4_code(x[j][e] * up, s, inv) : 8u) << (4 * (e >> 1) + 16 * (e & 1));
        out[j] = word;
    }
    *reinterpret_cast<u32x4*>(p.codes + at * kQ4TileBytes + lane * 16) = out;
}

// A wave per tile: the values that codes and scales stand for, each rounded once.
template <int DT, int kRuns> __global__ __launch_bounds__(kQ4Threads) void tide_head_dequantize_kernel(Q4WeightParams p) {
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.tiles) return;
    const int lane = threadIdx.x % kWave, g = lane >> 4, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks), v = tile * kQ4Rows + (lane & 15);
    if (v >= p.V) return;
    const u32x4 codes = *reinterpret_cast<const u32x4*>(p.codes + at * kQ4TileBytes + lane * 16);
    constexpr int kB = Storage<DT>::kBytes;
    char* row = p.W_out + (int64_t)v * p.row_bytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int col = kb * kQ4Cols + 32 * j + 8 * g, group = (kb * 4 + j) / kRuns;
        if (col >= p.d) continue;
        const float s = q4_scale(p.scales[((int64_t)tile * p.groups + group) * kQ4Rows + (lane & 15)], p.half);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s * (float)((int)(codes[j] >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8);
        if (p.chunks && col + 8 <= p.d) {
#pragma unroll
            for (int h = 0; h < kB / 2; ++h) {
                u32x4 c;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (DT == kF32) c[e] = __float_as_uint(x[4 * h + e]);
                    else c[e] = q4_pair<DT>(x[2 * e], x[2 * e + 1]);
                }
                *reinterpret_cast<u32x4*>(row + (int64_t)col * kB + 16 * h) = c;
            }
        } else {
            for (int e = 0; e < 8 && col + e < p.d; ++e) {
                if constexpr (DT == kF32) *reinterpret_cast<float*>(row + (int64_t)(col + e) * 4) = x[e];
                else *reinterpret_cast<uint16_t*>(row + (int64_t)(col + e) * 2) = (uint16_t)q4_pair<DT>(x[e], 0.0f);
            }
        }
    }
}

// Rows as the matrix cores take them: per 16 rows and 32 columns a fragment of 1024 bytes (lane l: row l % 16, columns 8 (l / 16) ..+7), zeros beyond T and d.
// fp32 rows become three bf16 planes that add up to them exactly: the first eight significant bits, the next eight, the last eight, cut off and not rounded, so that
// none is larger than the value.
struct Q4RowParams {
    const char* x;
    int64_t row_bytes;
    char* out;
    int T, d, steps;           // steps of 32 columns, of whole tiles of codes
    bool chunks;
    int64_t fragments;
};
template <int DT> constexpr int kQ4Planes = DT == kF32 ? 3 : 1;
template <int DT> constexpr int kQ4Elem = DT == kF32 ? (int)kBF16 : DT;

template <int DT> __global__ __launch_bounds__(kQ4Threads) void tide_head_q4_rows_kernel(Q4RowParams p) {
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.fragments) return;
    const int lane = threadIdx.x % kWave, tile = (int)(at / p.steps), step = (int)(at - (int64_t)tile * p.steps), t = tile * 16 + (lane & 15);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    if (t < p.T) q4_load8<DT>(p.x + (int64_t)t * p.row_bytes, step * 32 + 8 * (lane >> 4), p.d, p.chunks, x);
    char* out = p.out + at * (kQ4Planes<DT> * kQ4TileBytes) + lane * 16;
#pragma unroll
    for (int plane = 0; plane < kQ4Planes<DT>; ++plane) {
        u32x4 c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DT == kF32) {
                const uint32_t a = __float_as_uint(x[2 * e]) & 0xffff0000u, b = __float_as_uint(x[2 * e + 1]) & 0xffff0000u;
                c[e] = a >> 16 | b;
                x[2 * e] -= __uint_as_float(a);
                x[2 * e + 1] -= __uint_as_float(b);
            } else {
                c[e] = q4_pair<DT>(x[2 * e], x[2 * e + 1]);
            }
        }
        *reinterpret_cast<u32x4*>(out + plane * kQ4TileBytes) = c;
    }
}

template <int E> __device__ __forceinline__ f32x4 q4_mma(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (E == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// Eight codes as numbers 1 + c / 16.
template <int E> __device__ __forceinline__ u32x4 q4_expand(uint32_t w) {
    if constexpr (E == kBF16) {
        constexpr uint32_t kMask = 0x00780078u, kOne = 0x3f803f80u;
        return u32x4{(w << 3 & kMask) | kOne, (w >> 1 & kMask) | kOne, (w >> 5 & kMask) | kOne, (w >> 9 & kMask) | kOne};
    } else {
        constexpr uint32_t kMask = 0x03c003c0u, kOne = 0x3c003c00u;
        return u32x4{(w << 6 & kMask) | kOne, (w << 2 & kMask) | kOne, (w >> 2 & kMask) | kOne, (w >> 6 & kMask) | kOne};
    }
}
template <int E> constexpr uint32_t kQ4Offset = E == kBF16 ? 0xbfc0bfc0u : 0xbe00be00u;      // -1.5, twice

struct Q4LogitParams {
    const char* rows;          // fragments
    const char* codes;
    const uint16_t* scales;
    float* out;
    int64_t out_stride;
    int T, V, blocks, groups, row_tiles;
    bool half;
    int64_t waves;
};

// A wave per 16 rows and 16 tokens.
template <int DT, int kRuns> __global__ __launch_bounds__(kQ4Threads) void tide_head_q4_kernel(Q4LogitParams p) {
    constexpr int E = kQ4Elem<DT>, P = kQ4Planes<DT>;
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.waves) return;
    const int lane = threadIdx.x % kWave, tile = (int)(at / p.row_tiles), rt = (int)(at - (int64_t)tile * p.row_tiles);
    const char* codes = p.codes + (int64_t)tile * p.blocks * kQ4TileBytes + lane * 16;
    const char* rows = p.rows + (int64_t)rt * p.blocks * 4 * P * kQ4TileBytes + lane * 16;
    const uint16_t* scales = p.scales + (int64_t)tile * p.groups * kQ4Rows + (lane & 15);
    const u32x4 offset = {kQ4Offset<E>, kQ4Offset<E>, kQ4Offset<E>, kQ4Offset<E>};
    f32x4 total = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int kb = 0; kb < p.blocks; ++kb) {
        const u32x4 c = *reinterpret_cast<const u32x4*>(codes + (int64_t)kb * kQ4TileBytes);
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += kRuns) {
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = j0; j < j0 + kRuns; ++j) {
                const u32x4 w = q4_expand<E>(c[j]);
#pragma unroll
                for (int plane = 0; plane < P; ++plane) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(rows + ((int64_t)(kb * 4 + j) * P + plane) * kQ4TileBytes);
                    sum = q4_mma<E>(x, offset, sum);
                    sum = q4_mma<E>(x, w, sum);
                }
            }
            const int group = min((kb * 4 + j0) / kRuns, p.groups - 1);      // (a group of padding adds zero)
            const float s = q4_scale(scales[group * kQ4Rows], p.half);
#pragma unroll
            for (int i = 0; i < 4; ++i) total[i] = fmaf(s, sum[i], total[i]);
        }
    }
    const int v = tile * kQ4Rows + (lane & 15);
    if (v >= p.V) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = rt * 16 + 4 * (lane >> 4) + i;
        if (t < p.T) p.out[(int64_t)t * p.out_stride + v] = 16.0f * total[i];
    }
}

}  // namespace tide
