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

// The same where `half` is all ones or zero, without a branch.
__device__ __forceinline__ float q4_scale_select(uint32_t bits, uint32_t half) {
    const uint32_t a = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)bits)), b = bits << 16;
    return __uint_as_float((a & half) | (b & ~half));
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

template <int E> __device__ __forceinline__ f32x4 q4_mma(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (E == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// Eight codes as numbers 1 + c / 16: a shift and an and-or for two (the constants from registers, as that instruction takes no literals).
template <int E> struct Q4Ones {
    uint32_t mask = E == kBF16 ? 0x00780078u : 0x03c003c0u, one = E == kBF16 ? 0x3f803f80u : 0x3c003c00u;
    __device__ __forceinline__ Q4Ones() { asm("" : "+s"(mask), "+v"(one)); }
    __device__ __forceinline__ u32x4 expand(uint32_t w) const {
        if constexpr (E == kBF16) return u32x4{(w << 3 & mask) | one, (w >> 1 & mask) | one, (w >> 5 & mask) | one, (w >> 9 & mask) | one};
        else return u32x4{(w << 6 & mask) | one, (w << 2 & mask) | one, (w >> 2 & mask) | one, (w >> 6 & mask) | one};
    }
};
// fp32 rows are three bf16 planes that add up to them exactly: the first eight significant bits, the next eight, the last eight, cut off and not rounded, so that none is
// larger than the value.
template <int DT> constexpr int kQ4Planes = DT == kF32 ? 3 : 1;
template <int DT> constexpr int kQ4Elem = DT == kF32 ? (int)kBF16 : DT;

// ---- Rows under a head in four bits: what the two kernels share.

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
template <int DT> __device__ __forceinline__ float q4_sum8(const u32x4 (&c)[Storage<DT>::kBytes / 2]) {
    float x[8];
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
    return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}
// The operands of a block of 128 columns from what four groups of lanes, `apart` lanes each, have of its rows: fragment j, plane to x + (j planes + plane) * step, and the
// sum of each group of columns times -1.5 to offs[group * offs_step].
template <int DT, int kRuns> __device__ __forceinline__ void q4_put(const Q4Raw<DT>& raw, int g, int apart, char* x, int step, float* offs, int offs_step) {
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += kRuns) {
        float sum = 0.0f;
#pragma unroll
        for (int j = j0; j < j0 + kRuns; ++j) {
            sum += q4_sum8<DT>(raw.c[j]);
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
                        v[e] = a >> 16 | b;
                        y[2 * e] -= __uint_as_float(a);
                        y[2 * e + 1] -= __uint_as_float(b);
                    }
                    *reinterpret_cast<u32x4*>(x + (j * 3 + plane) * step) = v;
                }
            } else {
                *reinterpret_cast<u32x4*>(x + j * step) = raw.c[j][0];
            }
        }
        sum += __shfl_xor(sum, apart, kWave);
        sum += __shfl_xor(sum, 2 * apart, kWave);
        if (g == 0) offs[j0 / kRuns * offs_step] = -1.5f * sum;
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

// ---- Few rows, up to 16: all of them in LDS.
//
// A workgroup lays the rows out once -- as fragments, 16 bytes (eight columns) of each row side by side, with the groups' sums times -1.5, which the matrix steps of a
// group start from: no instruction is spent on the offset -- and its waves then stream tiles of codes, each wave NT tiles at a time, kDepth blocks of 128
// columns ahead.  The scales come a kilobyte at a time through LDS (a load of each step's scales, 32 bytes of use, cost 4 of 50 us at one row, 128000 x 4096).
// Where there are few tokens, `split` waves share the columns of a wave's tiles and add up their sums, in order, through LDS.
struct Q4FewParams {
    Q4Rows x;
    Q4Head head;
    float* out;
    int64_t out_stride;
    int sets;                  // of tokens, each a workgroup's at a time
    int rows_log;              // rows in LDS: a power of two
    int split;
};
constexpr int kQ4FewThreads = 1024;

struct Q4FewLds {
    int offs, scales, sums, bytes;
};
template <int DT, int kRuns, int NT> __host__ __device__ inline Q4FewLds q4_few_lds(int rows_log, int blocks, int waves, int split) {
    Q4FewLds l{};
    l.offs = blocks * 4 * kQ4Planes<DT> * (64 << rows_log);
    l.scales = l.offs + blocks * (4 / kRuns) * (4 << (rows_log < 2 ? 2 : rows_log));
    l.sums = l.scales + waves * 1024;
    l.bytes = l.sums + (split > 1 ? waves * NT * 1024 : 0);
    return l;
}

template <int DT, int kRuns, int NT> __global__ __launch_bounds__(kQ4FewThreads) void tide_head_q4_few_kernel(Q4FewParams p) {
    constexpr int E = kQ4Elem<DT>, P = kQ4Planes<DT>, kPer = 4 / kRuns, kDepth = NT == 1 ? 4 : 2;
    constexpr int kScaleBlocks = 32 / NT / kPer;       // blocks of 128 columns whose scales a kilobyte holds
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int log = p.rows_log, rows = 1 << log, offs_log = log < 2 ? 2 : log, blocks = p.head.blocks;
    const Q4FewLds at = q4_few_lds<DT, kRuns, NT>(log, blocks, waves, p.split);

    // the wave's tiles: NT of each set, blocks `begin` ..+`own`.  The first of them are on their way while the rows are laid out
    const int unit = wave / p.split, part = wave - unit * p.split, units = waves / p.split;
    const int begin = part * blocks / p.split, own = (part + 1) * blocks / p.split - begin;
    const int passes = (p.sets - blockIdx.x + gridDim.x - 1) / gridDim.x;
    auto tile_of = [&](int pass) { return ((int)(blockIdx.x + pass * gridDim.x) * units + unit) * NT; };
    u32x4 c[kDepth][NT];
    int f_pass = 0, f_at = 0;                          // what is fetched next; beyond the last tile: the last again, for nothing
    const char* f_codes[NT];
    auto point = [&](int pass) {
        const int tile0 = tile_of(min(pass, passes - 1));
#pragma unroll
        for (int n = 0; n < NT; ++n) f_codes[n] = p.head.codes + ((int64_t)min(tile0 + n, p.head.tiles - 1) * blocks + begin) * kQ4TileBytes;
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
    auto fetch_scales = [&](int pass, int i) { s_next = q4_scales<NT>(p.head, tile_of(min(pass, passes - 1)), (begin + i) * kPer, lane); };
#pragma unroll
    for (int slot = 0; slot < kDepth; ++slot) fetch(slot);
    fetch_scales(0, 0);

    for (int item = threadIdx.x; item < blocks * 4 << log; item += blockDim.x) {
        const int row = item & (rows - 1), g = item >> log & 3, kb = item >> (log + 2);
        Q4Raw<DT> raw;
        q4_raw<DT>(p.x, row, kb * kQ4Cols + 8 * g, raw);
        q4_put<DT, kRuns>(raw, g, rows, lds + ((kb * 16 * P + g) << (log + 4)) + row * 16, 64 << log, reinterpret_cast<float*>(lds + at.offs) + (kb * kPer << offs_log) + row, 1 << offs_log);
    }
    __syncthreads();

    const Q4Ones<E> ones;
    const uint32_t half = p.head.half ? 0xffffffffu : 0u;
    const char* const my_x = lds + ((lane >> 4) << (log + 4)) + (lane & (rows - 1)) * 16;
    const float* const my_offs = reinterpret_cast<const float*>(lds + at.offs) + (4 * (lane >> 4) & ((1 << offs_log) - 1));
    char* const my_scales = lds + at.scales + wave * 1024;
    f32x4 total[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) total[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int pass = 0, i = 0, s_at = 0;
    for (int left = passes * own; left > 0; left -= kDepth) {
#pragma unroll
        for (int slot = 0; slot < kDepth; ++slot) {    // (beyond the last block: what was fetched again, into sums that nothing takes)
            if (s_at == 0) {
                *reinterpret_cast<u32x4*>(my_scales + lane * 16) = s_next;
                if (i + kScaleBlocks < own) fetch_scales(pass, i + kScaleBlocks);
                else fetch_scales(pass + 1, 0);
            }
            u32x4 now[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) now[n] = c[slot][n];
            fetch(slot);
            const char* x = my_x + ((begin + i) * 4 * P << (log + 6));
            const float* offs = my_offs + ((begin + i) * kPer << offs_log);
#pragma unroll
            for (int gr = 0; gr < kPer; ++gr) {
                f32x4 sum[NT];
                const f32x4 start = *reinterpret_cast<const f32x4*>(offs + (gr << offs_log));
#pragma unroll
                for (int n = 0; n < NT; ++n) sum[n] = start;
#pragma unroll
                for (int j = gr * kRuns; j < (gr + 1) * kRuns; ++j) {
                    u32x4 w[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) w[n] = ones.expand(now[n][j]);
#pragma unroll
                    for (int plane = 0; plane < P; ++plane) {
                        const u32x4 a = *reinterpret_cast<const u32x4*>(x + ((j * P + plane) << (log + 6)));
#pragma unroll
                        for (int n = 0; n < NT; ++n) sum[n] = q4_mma<E>(a, w[n], sum[n]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float s = q4_scale_at(my_scales, NT, n, s_at * kPer + gr, lane, half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) total[n][e] = fmaf(s, sum[n][e], total[n][e]);
                }
            }
            if (++s_at == kScaleBlocks) s_at = 0;
            if (++i < own) continue;
            if (p.split > 1 && pass < passes) {
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
                const bool writes = pass < passes && part == 0 && v < p.head.V;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int t = 4 * (lane >> 4) + e;
                    if (writes && t < p.x.T) p.out[(int64_t)t * p.out_stride + v] = 16.0f * total[n][e];
                    total[n][e] = 0.0f;
                }
            }
            ++pass;
            i = 0;
            s_at = 0;
        }
    }
}

// ---- Many rows.
//
// The rows are first laid out in memory: for 16 MT rows and 128 columns one region, the fragments and behind them the groups' sums times -1.5, whole kilobytes.
template <int DT, int kRuns, int MT> struct Q4Region {
    static constexpr int kX = 4 * kQ4Planes<DT> * MT * 1024, kOffs = (4 / kRuns * MT * 64 + 1023) / 1024 * 1024, kBytes = kX + kOffs;
};
struct Q4LayParams {
    Q4Rows x;
    char* out;
    int blocks;
    int64_t waves;             // row tiles of all row blocks, times blocks
};
template <int DT, int kRuns, int MT> __global__ __launch_bounds__(kQ4Threads) void tide_head_q4_lay_kernel(Q4LayParams p) {
    using R = Q4Region<DT, kRuns, MT>;
    const int64_t at = (int64_t)blockIdx.x * (kQ4Threads / kWave) + threadIdx.x / kWave;
    if (at >= p.waves) return;
    const int lane = threadIdx.x % kWave, tile = (int)(at / p.blocks), kb = (int)(at - (int64_t)tile * p.blocks), rb = tile / MT, rt = tile - rb * MT;
    Q4Raw<DT> raw;
    q4_raw<DT>(p.x, tile * 16 + (lane & 15), kb * kQ4Cols + 8 * (lane >> 4), raw);
    char* region = p.out + ((int64_t)rb * p.blocks + kb) * R::kBytes;
    q4_put<DT, kRuns>(raw, lane >> 4, 16, region + rt * 1024 + lane * 16, MT * 1024, reinterpret_cast<float*>(region + R::kX) + rt * 16 + (lane & 15), MT * 16);
}

// A workgroup has 16 MT rows and its waves NT tiles of 16 tokens each.  The regions of the rows go through a ring of three stages in LDS by transfers that no register waits
// for; the codes through registers, a block or two ahead; a barrier for each block of 128 columns.  The transfers are inline assembly, which the compiler does not
// count, so the waits for them are written out: at a block's start all but the transfers and loads of the two blocks after the one that requested its
// region may be under way.
struct Q4ManyParams {
    const char* regions;
    Q4Head head;
    float* out;
    int64_t out_stride;
    int T, row_blocks;
    int sets, set_grid;        // sets of tokens, each a workgroup's at a time; workgroups that share them (a multiple of 8)
};
constexpr int kQ4ManyThreads = 512;
constexpr int kQ4Stages = 3;
template <int DT, int kRuns, int MT> constexpr int kQ4ManyLds = kQ4Stages * Q4Region<DT, kRuns, MT>::kBytes + kQ4ManyThreads / kWave * 1024;

// 64 lanes x 16 bytes from memory to a kilobyte of LDS (m0 as in the head products).  The wait states: five between a vector instruction that wrote the base and this one.
__device__ __forceinline__ void q4_transfer(uint32_t lds, const char* base, uint32_t lane16) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane16), "s"(base) : "memory");
}

template <int DT, int kRuns, int MT, int NT> __global__ __launch_bounds__(kQ4ManyThreads) void tide_head_q4_many_kernel(Q4ManyParams p) {
    using R = Q4Region<DT, kRuns, MT>;
    constexpr int E = kQ4Elem<DT>, P = kQ4Planes<DT>, kPer = 4 / kRuns, kDepth = MT * NT >= 32 ? 1 : 2;
    constexpr int kScaleBlocks = 32 / NT / kPer;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    // workgroups of the same tokens run on one XCD (numbers that are equal modulo 8), for their codes to be in its L2
    const int eighth = blockIdx.x & 7, rest = blockIdx.x >> 3, row_block = rest % p.row_blocks, set0 = rest / p.row_blocks * 8 + eighth, blocks = p.head.blocks;
    if (set0 >= p.sets) return;
    const int passes = (p.sets - set0 + p.set_grid - 1) / p.set_grid;
    auto tile_of = [&](int pass) { return ((set0 + pass * p.set_grid) * waves + wave) * NT; };

    const char* const regions = p.regions + (int64_t)row_block * blocks * R::kBytes;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds, lane16 = lane * 16;
    int x_kb = 0, x_stage = 0;
    auto request = [&] {
        const char* from = regions + (int64_t)x_kb * R::kBytes;
        for (int i = wave * 1024; i < R::kBytes; i += waves * 1024) q4_transfer(lds0 + x_stage * R::kBytes + i, from + i, lane16);
        if (++x_kb == blocks) x_kb = 0;
        if (++x_stage == kQ4Stages) x_stage = 0;
    };
    u32x4 c[kDepth][NT];
    int f_pass = 0, f_at = 0;
    const char* f_codes[NT];
    auto point = [&](int pass) {
        const int tile0 = tile_of(min(pass, passes - 1));
#pragma unroll
        for (int n = 0; n < NT; ++n) f_codes[n] = p.head.codes + (int64_t)min(tile0 + n, p.head.tiles - 1) * blocks * kQ4TileBytes;
    };
    point(0);
    auto fetch = [&](int slot) {
#pragma unroll
        for (int n = 0; n < NT; ++n) c[slot][n] = *reinterpret_cast<const u32x4*>(f_codes[n] + (uint32_t)(f_at * kQ4TileBytes) + lane * 16);
        if (++f_at == blocks) {
            f_at = 0;
            point(++f_pass);
        }
    };
    u32x4 s_next;
    auto fetch_scales = [&](int pass, int i) { s_next = q4_scales<NT>(p.head, tile_of(min(pass, passes - 1)), i * kPer, lane); };
    fetch_scales(0, 0);
    request();
    request();
#pragma unroll
    for (int slot = 0; slot < kDepth; ++slot) fetch(slot);

    const Q4Ones<E> ones;
    const uint32_t half = p.head.half ? 0xffffffffu : 0u;
    char* const my_scales = lds + kQ4Stages * R::kBytes + wave * 1024;
    f32x4 total[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int rt = 0; rt < MT; ++rt) total[n][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int pass = 0, i = 0, s_at = 0, stage = 0;
    // requested after a block's region: the rest of the region's block (a fetch), the next block (transfers, a fetch)
    constexpr int kUnderWay = R::kBytes / 1024 / (kQ4ManyThreads / kWave) + (kDepth == 1 ? 1 : 2) * NT;
    for (int left = passes * blocks; left > 0; left -= kDepth) {
#pragma unroll
        for (int slot = 0; slot < kDepth; ++slot) {    // (beyond the last block: into sums that nothing takes)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(kUnderWay) : "memory");
            request();
            if (s_at == 0) {
                *reinterpret_cast<u32x4*>(my_scales + lane * 16) = s_next;
                if (i + kScaleBlocks < blocks) fetch_scales(pass, i + kScaleBlocks);
                else fetch_scales(pass + 1, 0);
            }
            u32x4 now[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) now[n] = c[slot][n];
            fetch(slot);
            const char* x = lds + stage * R::kBytes + lane * 16;
            const float* offs = reinterpret_cast<const float*>(lds + stage * R::kBytes + R::kX) + 4 * (lane >> 4);
#pragma unroll
            for (int gr = 0; gr < kPer; ++gr) {
                u32x4 w[kRuns][NT];
                float s[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int j = 0; j < kRuns; ++j) w[j][n] = ones.expand(now[n][gr * kRuns + j]);
                    s[n] = q4_scale_at(my_scales, NT, n, s_at * kPer + gr, lane, half);
                }
#pragma unroll
                for (int rt = 0; rt < MT; ++rt) {
                    f32x4 sum[NT];
                    const f32x4 start = *reinterpret_cast<const f32x4*>(offs + (gr * MT + rt) * 16);
#pragma unroll
                    for (int n = 0; n < NT; ++n) sum[n] = start;
#pragma unroll
                    for (int j = 0; j < kRuns; ++j)
#pragma unroll
                        for (int plane = 0; plane < P; ++plane) {
                            const u32x4 a = *reinterpret_cast<const u32x4*>(x + (((gr * kRuns + j) * P + plane) * MT + rt) * 1024);
#pragma unroll
                            for (int n = 0; n < NT; ++n) sum[n] = q4_mma<E>(a, w[j][n], sum[n]);
                        }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[n][rt][e] = fmaf(s[n], sum[n][e], total[n][rt][e]);
                }
            }
            if (++stage == kQ4Stages) stage = 0;
            if (++s_at == kScaleBlocks) s_at = 0;
            if (++i < blocks) continue;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int v = (tile_of(pass) + n) * kQ4Rows + (lane & 15);
                const bool writes = pass < passes && v < p.head.V;
#pragma unroll
                for (int rt = 0; rt < MT; ++rt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = (row_block * MT + rt) * 16 + 4 * (lane >> 4) + e;
                        if (writes && t < p.T) p.out[(int64_t)t * p.out_stride + v] = 16.0f * total[n][rt][e];
                        total[n][rt][e] = 0.0f;
                    }
            }
            ++pass;
            i = 0;
            s_at = 0;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last transfers: the LDS is another workgroup's afterwards
}

}  // namespace tide
