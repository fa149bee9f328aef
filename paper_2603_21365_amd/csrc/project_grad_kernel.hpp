// Gradient of the exit projection (project_kernel.hpp): y = n * gain with n = h * r, r = 1 / sqrt(mean(h^2) + eps), so with u = dy * gain
//     dh = r * (u - n * mean(u * n))          mean(u * n) = r * sum(u * h) / d
//     dgain = sum over tokens of dy * n
// One pass: a workgroup takes rows in turn, every thread its chunks of the row (h and dy in registers between the two sums and the
// write) and the same columns of dgain, which it adds up over its rows in registers; the workgroups' sums are joined by a second launch, in
// order, so the result does not depend on timing.  Rows without a source (no exit and no last-layer state) have a gradient of zero.
#pragma once
#include "project_kernel.hpp"

namespace tide {

struct ProjectGradParams {
    const char* hidden;
    int64_t ckpt_stride_bytes, row_stride_bytes;
    const char* final_hidden;        // or null
    int64_t final_row_stride_bytes;
    const int32_t* exit_layer;       // [T]
    const float* gain;               // [d] or null
    const char* grad_out;
    int64_t grad_out_row_bytes;
    char* grad;
    int64_t grad_row_bytes;
    float* part;                     // [gridDim.x][d] sums of dgain, or null
    int C, T, d;
    float eps;
    int32_t layer_id[32];
};

template <int DT> __device__ __forceinline__ void project_widen(u32x4 c, float (&v)[Storage<DT>::kElems]) {
    if constexpr (DT == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(c[e]);
    } else if constexpr (DT == kF16) {
        const f16x8 h = __builtin_bit_cast(f16x8, c);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(c[e] << 16);
            v[2 * e + 1] = __uint_as_float(c[e] & 0xffff0000u);
        }
    }
}
template <int DT> __device__ __forceinline__ u32x4 project_round(const float (&v)[Storage<DT>::kElems]) {
    if constexpr (DT == kF32) {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else if constexpr (DT == kF16) {
        f16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = static_cast<_Float16>(v[e]);
        return __builtin_bit_cast(u32x4, o);
    } else {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = static_cast<__bf16>(v[e]);
        return __builtin_bit_cast(u32x4, o);
    }
}

template <int DT, int kChunks>
__global__ __launch_bounds__(kProjectThreads) void tide_project_grad_kernel(const ProjectGradParams p) {
    constexpr int E = Storage<DT>::kElems;
    __shared__ float part[2][2][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nchunk = p.d * Storage<DT>::kBytes / 16;
    const float inv_d = 1.0f / (float)p.d;
    float sum[kChunks][E];
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[j][e] = 0.0f;
    int turn = 0;
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        const int32_t layer = p.exit_layer[t];
        int c_hit = -1;
        for (int c = 0; c < p.C; ++c) c_hit = (p.layer_id[c] == layer) ? c : c_hit;
        const char* src = c_hit >= 0 ? p.hidden + (int64_t)c_hit * p.ckpt_stride_bytes + (int64_t)t * p.row_stride_bytes
                          : p.final_hidden ? p.final_hidden + (int64_t)t * p.final_row_stride_bytes : nullptr;
        char* dst = p.grad + (int64_t)t * p.grad_row_bytes;
        if (!src) {                                    // (the same for the whole workgroup)
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
                if (tid + j * kProjectThreads < nchunk) reinterpret_cast<u32x4*>(dst)[tid + j * kProjectThreads] = u32x4{0, 0, 0, 0};
            continue;
        }
        const char* dy = p.grad_out + (int64_t)t * p.grad_out_row_bytes;
        u32x4 h[kChunks], g[kChunks];
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int q = tid + j * kProjectThreads, at = min(q, nchunk - 1);
            h[j] = reinterpret_cast<const u32x4*>(src)[at];
            g[j] = reinterpret_cast<const u32x4*>(dy)[at];
            if (q >= nchunk) h[j] = g[j] = u32x4{0, 0, 0, 0};
        }
        float ss = 0.0f, uh = 0.0f;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            float hv[E], gv[E];
            project_widen<DT>(h[j], hv);
            project_widen<DT>(g[j], gv);
            const int at = min(tid + j * kProjectThreads, nchunk - 1) * E;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                ss = fmaf(hv[e], hv[e], ss);
                uh = fmaf(gv[e] * hv[e], p.gain ? p.gain[at + e] : 1.0f, uh);
            }
        }
        ss = wave_sum(ss);
        uh = wave_sum(uh);
        if (lane == 0) {
            part[turn][0][wave] = ss;
            part[turn][1][wave] = uh;
        }
        __syncthreads();                               // one barrier a row: the next row with a source puts its sums into the other half
        ss = (part[turn][0][0] + part[turn][0][1]) + (part[turn][0][2] + part[turn][0][3]);
        uh = (part[turn][1][0] + part[turn][1][1]) + (part[turn][1][2] + part[turn][1][3]);
        const float r = inv_rms_f32(ss, inv_d, p.eps), back = r * r * uh * inv_d;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            float hv[E], gv[E], o[E];
            project_widen<DT>(h[j], hv);
            project_widen<DT>(g[j], gv);
            const int q = tid + j * kProjectThreads, at = min(q, nchunk - 1) * E;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = p.gain ? gv[e] * p.gain[at + e] : gv[e];
                o[e] = r * fmaf(-back, hv[e], u);
                sum[j][e] = fmaf(gv[e], hv[e] * r, sum[j][e]);
            }
            if (q < nchunk) reinterpret_cast<u32x4*>(dst)[q] = project_round<DT>(o);
        }
        turn ^= 1;
    }
    if (!p.part) return;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int q = tid + j * kProjectThreads;
        if (q < nchunk) {
#pragma unroll
            for (int e = 0; e < E; e += 4)
                reinterpret_cast<f32x4*>(p.part + (int64_t)blockIdx.x * p.d + q * E)[e / 4] = f32x4{sum[j][e], sum[j][e + 1], sum[j][e + 2], sum[j][e + 3]};
        }
    }
}

// dgain: the workgroups' sums, 32 columns per workgroup, eight threads a column, joined in a fixed order.
__global__ __launch_bounds__(256) void tide_project_gain_kernel(const float* part, int parts, int d, float* out) {
    __shared__ float sum[8][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
    float s = 0.0f;
    if (col < d)
        for (int i = slice; i < parts; i += 8) s += part[(int64_t)i * d + col];
    sum[slice][threadIdx.x & 31] = s;
    __syncthreads();
    if (slice == 0 && col < d) {
        const int c = threadIdx.x;
        out[col] = ((sum[0][c] + sum[1][c]) + (sum[2][c] + sum[3][c])) + ((sum[4][c] + sum[5][c]) + (sum[6][c] + sum[7][c]));
    }
}

}  // namespace tide
