// Gradient of the exit projection (project_kernel.hpp): y = n * gain with n = h * r, r = 1 / sqrt(mean(h^2) + eps), so with u = dy * gain
//     dh = r * (u - n * mean(u * n))          mean(u * n) = r * sum(u * h) / d
//     dgain = sum over tokens of dy * n
// One pass: a workgroup takes rows in turn, every thread its chunks of the row (h and dy in registers between the two sums and the
// write) and the same columns of dgain, which it adds up over its rows in registers; the workgroups' sums are joined by a second launch, in
// order, so the result does not depend on timing. Bound by memory: T = 8192, d = 4096 in bf16 takes 43 us for 201 MB (4.7 TB/s, a copy of
// 1 GiB 5.0) and 4.6 for the second launch; the first form, without the next row's request ahead, took 152.   Rows without a source (no exit and no last-layer state) have a gradient of
// zero, and so have rows whose dy is zero throughout (tokens without a target), whatever they hold: 0 * NaN is kept out of dgain.
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

// kWavePerRow: four rows at a time, one per wave (rows of up to 4 KiB); otherwise one.  kHeld: the gain in registers, and the next row requested before
// this one's sums are taken (rows of up to four chunks a thread: more would spill).
template <int DT, int kChunks, bool kWavePerRow>
__global__ __launch_bounds__(kProjectThreads) void tide_project_grad_kernel(const ProjectGradParams p) {
    constexpr int E = Storage<DT>::kElems;
    constexpr bool kHeld = kChunks * E <= 32;
    constexpr int kStep = kWavePerRow ? kWave : kProjectThreads;
    static_assert(!kWavePerRow || kHeld, "");
    __shared__ float part[2][2][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = kWavePerRow ? lane : threadIdx.x;
    const int nchunk = p.d * Storage<DT>::kBytes / 16;
    const float inv_d = 1.0f / (float)p.d;
    float sum[kChunks][E], held[kHeld ? kChunks : 1][E];
    auto load_gain = [&](int j, float (&v)[E]) {
        const int at = min(tid + j * kStep, nchunk - 1) * E;
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const f32x4 x = p.gain ? *reinterpret_cast<const f32x4*>(p.gain + at + e) : f32x4{1.0f, 1.0f, 1.0f, 1.0f};
            v[e] = x[0], v[e + 1] = x[1], v[e + 2] = x[2], v[e + 3] = x[3];
        }
    };
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[j][e] = 0.0f;
        if constexpr (kHeld) load_gain(j, held[j]);
    }
    auto layer_of = [&](int t) { return t < p.T ? p.exit_layer[t] : 0; };
    auto source = [&](int t, int32_t layer) -> const char* {
        if (t >= p.T) return nullptr;
        int c_hit = -1;
        for (int c = 0; c < p.C; ++c) c_hit = (p.layer_id[c] == layer) ? c : c_hit;   // layers are distinct: at most one hit
        return c_hit >= 0 ? p.hidden + (int64_t)c_hit * p.ckpt_stride_bytes + (int64_t)t * p.row_stride_bytes
               : p.final_hidden ? p.final_hidden + (int64_t)t * p.final_row_stride_bytes : nullptr;
    };
    u32x4 h[kChunks], g[kChunks];
    auto load_row = [&](const char* src, int t) {
        const char* dy = p.grad_out + (int64_t)t * p.grad_out_row_bytes;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int q = tid + j * kStep, at = min(q, nchunk - 1);
            h[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src) + at);
            g[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(dy) + at);
            if (q >= nchunk) h[j] = g[j] = u32x4{0, 0, 0, 0};
        }
    };
    int t = kWavePerRow ? blockIdx.x * 4 + wave : blockIdx.x, turn = 0;
    const int stride = kWavePerRow ? gridDim.x * 4 : gridDim.x;
    const char* src = source(t, layer_of(t));
    int32_t next_layer = layer_of(t + stride);
    if (src) load_row(src, t);
    for (; t < p.T; t += stride) {
        const char* next = source(t + stride, next_layer);
        next_layer = layer_of(t + 2 * stride);
        char* dst = p.grad + (int64_t)t * p.grad_row_bytes;
        if (!src) {                                    // (the same for the whole workgroup)
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
                if (tid + j * kStep < nchunk) reinterpret_cast<u32x4*>(dst)[tid + j * kStep] = u32x4{0, 0, 0, 0};
            src = next;
            if (src) load_row(src, t + stride);
            continue;
        }
        float hv[kChunks][E], gv[kChunks][E];
        float ss = 0.0f, uh = 0.0f;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            project_widen<DT>(h[j], hv[j]);
            project_widen<DT>(g[j], gv[j]);
            if constexpr (!kHeld) load_gain(j, held[0]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                ss = fmaf(hv[j][e], hv[j][e], ss);
                uh = fmaf(gv[j][e] * hv[j][e], held[kHeld ? j : 0][e], uh);
            }
        }
        if constexpr (kHeld) {
            if (next) load_row(next, t + stride);
        }
        ss = wave_sum(ss);
        uh = wave_sum(uh);
        if constexpr (!kWavePerRow) {
            if (lane == 0) {
                part[turn][0][wave] = ss;
                part[turn][1][wave] = uh;
            }
            __syncthreads();                           // one barrier a row: the next row with a source puts its sums into the other half
            ss = (part[turn][0][0] + part[turn][0][1]) + (part[turn][0][2] + part[turn][0][3]);
            uh = (part[turn][1][0] + part[turn][1][1]) + (part[turn][1][2] + part[turn][1][3]);
        }
        float r = inv_rms_f32(ss, inv_d, p.eps), back = r * r * uh * inv_d;
        if (uh != uh) {                                // (the same for the row) a NaN in the row or dy, or an infinity against a zero: no dy, no gradient
            bool any = false;
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) any |= gv[j][e] != 0.0f;
            if constexpr (kWavePerRow) any = __any(any);
            else any = __syncthreads_or(any);
            if (!any) {
                r = back = 0.0f;
#pragma unroll
                for (int j = 0; j < kChunks; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) hv[j][e] = 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            float o[E];
            if constexpr (!kHeld) load_gain(j, held[0]);
            const int q = tid + j * kStep;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                o[e] = r * fmaf(-back, hv[j][e], gv[j][e] * held[kHeld ? j : 0][e]);
                sum[j][e] = fmaf(gv[j][e], hv[j][e] * r, sum[j][e]);
            }
            if (q < nchunk) __builtin_nontemporal_store(project_round<DT>(o), reinterpret_cast<u32x4*>(dst) + q);
        }
        if constexpr (!kHeld) {
            if (next) load_row(next, t + stride);
        }
        src = next;
        turn ^= 1;
    }
    if (!p.part) return;
    if constexpr (kWavePerRow) {                       // the waves' sums, joined in order
        __shared__ f32x4 all[4][kChunks * E / 4][kWave];
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
#pragma unroll
            for (int e = 0; e < E; e += 4) all[wave][(j * E + e) / 4][lane] = f32x4{sum[j][e], sum[j][e + 1], sum[j][e + 2], sum[j][e + 3]};
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const int i = (j * E + e) / 4;
                const f32x4 v = (all[0][i][lane] + all[1][i][lane]) + (all[2][i][lane] + all[3][i][lane]);
                sum[j][e] = v[0], sum[j][e + 1] = v[1], sum[j][e + 2] = v[2], sum[j][e + 3] = v[3];
            }
    }
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int q = tid + j * kStep;
        if (q < nchunk) {
#pragma unroll
            for (int e = 0; e < E; e += 4)
                reinterpret_cast<f32x4*>(p.part + (int64_t)blockIdx.x * p.d + q * E)[e / 4] = f32x4{sum[j][e], sum[j][e + 1], sum[j][e + 2], sum[j][e + 3]};
        }
    }
}

// dgain: the workgroups' sums, 32 columns per workgroup of 1024 threads: eight threads take four columns each of every 128th sum, then the 128 are joined in
// a fixed order.
constexpr int kProjectGainThreads = 1024;
__global__ __launch_bounds__(kProjectGainThreads) void tide_project_gain_kernel(const float* part, int parts, int d, float* out) {
    __shared__ float sum[128][33];
    const int c4 = (threadIdx.x & 7) * 4, slice = threadIdx.x >> 3, col = blockIdx.x * 32 + c4;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < d)                                       // (d is a multiple of four)
        for (int i = slice; i < parts; i += 128) s += *reinterpret_cast<const f32x4*>(part + (int64_t)i * d + col);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[slice][c4 + e] = s[e];
    __syncthreads();
    const int c = threadIdx.x & 31, k = threadIdx.x >> 5;          // 32 threads a column, four sums each
    float v = (sum[k][c] + sum[k + 32][c]) + (sum[k + 64][c] + sum[k + 96][c]);
    __syncthreads();
    sum[k][c] = v;
    __syncthreads();
    if (k == 0 && blockIdx.x * 32 + c < d) {
        v = 0.0f;
        for (int i = 0; i < 32; ++i) v += sum[i][c];
        out[blockIdx.x * 32 + c] = v;
    }
}

}  // namespace tide
