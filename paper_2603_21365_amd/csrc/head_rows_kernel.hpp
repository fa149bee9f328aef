// What stands around the products of the head operators (head_gemm_kernel.hpp): the rows that have a gradient, the teacher's
// probabilities, the scales of 16-bit planes, padded or split copies, and the sums that finish a call.
//
// Rows without a gradient -- no target, a teacher without entries, an upstream gradient of zero -- are left out of the three products of
// the gradient: the others are gathered, which makes their number the products' size (a tenth of a training batch is typically masked) and keeps
// whatever such rows hold (NaN, infinities) out of dW, where a zero weight would not (0 * NaN).
#pragma once
#include "head_gemm_kernel.hpp"

namespace tide {

constexpr int kHeadRowThreads = 256;
constexpr int kHeadCtlThreads = 1024;
constexpr int kHeadMaxBlocks = 2048;       // workgroups that search for the largest magnitude

// Largest finite magnitude of W, one per workgroup (as bits: the order of non-negative floats).  Infinities and NaN are passed
// over: they give what they give whatever the scale, and must not cost the other rows theirs.
__global__ __launch_bounds__(kHeadRowThreads) void tide_head_max_kernel(const char* rows, int64_t row_bytes, int64_t n_rows, int d, uint32_t* out) {
    __shared__ uint32_t part[4];
    uint32_t m = 0;
    const bool chunks = ((uintptr_t)rows | (uintptr_t)row_bytes) % 16 == 0 && d % 4 == 0;
    auto take = [&](uint32_t b) { b &= 0x7fffffffu; m = b < 0x7f800000u && b > m ? b : m; };
    if (chunks) {                                      // contiguous rows as one, else each workgroup rows of its own; eight chunks a thread at a time
        const bool flat = row_bytes == (int64_t)d * 4;
        const int64_t n = flat ? 1 : n_rows, per_row = flat ? n_rows * (d / 4) : d / 4;
        const int64_t first = flat ? (int64_t)blockIdx.x * kHeadRowThreads : 0, step = flat ? (int64_t)gridDim.x * kHeadRowThreads : kHeadRowThreads;
        for (int64_t r = flat ? 0 : blockIdx.x; r < n; r += gridDim.x) {
            const u32x4* row = reinterpret_cast<const u32x4*>(rows + r * row_bytes);
            for (int64_t i = first + threadIdx.x; i < per_row; i += 8 * step) {
                u32x4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = row[min(i + u * step, per_row - 1)];
#pragma unroll
                for (int u = 0; u < 8; ++u) take(v[u][0]), take(v[u][1]), take(v[u][2]), take(v[u][3]);
            }
        }
    } else {
        for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x)
            for (int i = threadIdx.x; i < d; i += kHeadRowThreads) take(reinterpret_cast<const uint32_t*>(rows + r * row_bytes)[i]);
    }
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s, kWave));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) out[blockIdx.x] = max(max(part[0], part[1]), max(part[2], part[3]));
}

// The power of two that brings a largest magnitude into [2^14, 2^15): the upper end of fp16, so that small elements keep their bits.  (0 for none, or none finite.)
__device__ __forceinline__ int head_exponent(uint32_t max_bits) { return max_bits == 0 || max_bits >= 0x7f800000u ? 0 : 141 - max(1, (int)(max_bits >> 23)); }

enum : int { kHeadGradAsIs = 0, kHeadGradCommon = 1, kHeadGradOwn = 2 };      // the power of two that a row of G is multiplied by: none, one for all, its own
struct HeadCtlParams {
    HeadCtl* ctl;
    const uint32_t* w_max;     // fp32: the workgroups' maxima
    int w_blocks;
    int grads;                 // 0: W's scale only
    int grad_scale;            // kHeadGrad..., as G is held in bf16, in fp16, or in planes
    int T, V;
    const int32_t* target;     // [T], or null and
    const uint8_t* taught;     // [T] whether the teacher has entries
    const float* grad;         // [T] upstream
    const float* lse;          // [T]
    float tau;
    int32_t* source;           // [T] out: the live rows' tokens, ascending
    int32_t* place;            // [T] out: a token's live row, or -1
    float4* row_const;         // [T] out, of live rows: lse * log2 e, grad * tau * 2^s, and as integers the target or the token, and s
};

// One workgroup: W's and the gradients' scales, and the list of live rows in token order (each thread a run of tokens).
__global__ __launch_bounds__(kHeadCtlThreads) void tide_head_ctl_kernel(const HeadCtlParams p) {
    __shared__ uint32_t max_of[2][16];
    __shared__ int count_of[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t m[2] = {0, 0};
    for (int i = tid; i < p.w_blocks; i += kHeadCtlThreads) m[0] = max(m[0], p.w_max[i]);
    const int per = p.grads ? (p.T + kHeadCtlThreads - 1) / kHeadCtlThreads : 0;
    const int t0 = min(p.T, tid * per), t1 = min(p.T, t0 + per);
    auto live = [&](int t) {
        const float g = p.grad[t];
        const bool there = p.target ? (uint32_t)p.target[t] < (uint32_t)p.V : p.taught[t] != 0;
        return there && g != 0.0f;
    };
    int n = 0;
    for (int t = t0; t < t1; ++t)
        if (live(t)) {
            ++n;
            const uint32_t b = __float_as_uint(fabsf(p.grad[t] * p.tau));
            m[1] = b < 0x7f800000u ? max(m[1], b) : m[1];      // (a gradient that is not finite takes no other row's bits)
        }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], s, kWave));
        if (lane == 0) max_of[j][wave] = m[j];
    }
    int upto = n;                                      // live rows of this wave's lanes up to this one
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const int o = __shfl_up(upto, s, kWave);
        if (lane >= s) upto += o;
    }
    if (lane == 63) count_of[wave] = upto;
    __syncthreads();
    int before = upto - n, all = 0;
    for (int w = 0; w < 16; ++w) {
        all += count_of[w];
        if (w < wave) before += count_of[w];
        for (int j = 0; j < 2; ++j) m[j] = max(m[j], max_of[j][w]);
    }
    const int common = p.grad_scale == kHeadGradCommon ? head_exponent(m[1]) : 0;
    for (int t = t0; t < t1; ++t) {
        const bool l = live(t);
        p.place[t] = l ? before : -1;
        if (l) {
            const float g = p.grad[t] * p.tau;
            const int s = p.grad_scale == kHeadGradOwn ? head_exponent(__float_as_uint(fabsf(g))) : common;
            p.source[before] = t;
            p.row_const[before] = float4{p.lse[t] * 1.4426950408889634f, ldexpf(g, s), __int_as_float(p.target ? p.target[t] : t), __int_as_float(s)};
            ++before;
        }
    }
    if (tid == 0) {
        HeadCtl c;
        c.live = all;
        c.w_exp = head_exponent(m[0]);
        c.dw_exp = common;
        *p.ctl = c;
    }
}

// Chunk c (eight elements) of a row, zeros beyond d.  chunks: whole chunks at 16-byte addresses.
template <int DT> __device__ __forceinline__ void head_load8(const char* row, int c, int d, bool chunks, u32x4 (&v)[DT == kF32 ? 2 : 1]) {
    constexpr int kW = DT == kF32 ? 2 : 1;             // 16-byte pieces of a chunk's source
    if (chunks) {
#pragma unroll
        for (int w = 0; w < kW; ++w) v[w] = reinterpret_cast<const u32x4*>(row)[c * kW + w];
    } else if constexpr (DT == kF32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e & 3] = 8 * c + e < d ? reinterpret_cast<const uint32_t*>(row)[8 * c + e] : 0u;
    } else {
        const uint16_t* e = reinterpret_cast<const uint16_t*>(row) + 8 * c;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = 8 * c + 2 * k < d ? e[2 * k] : 0, hi = 8 * c + 2 * k + 1 < d ? e[2 * k + 1] : 0;
            v[0][k] = lo | hi << 16;
        }
    }
}
// The chunk times 2^n as two fp16 planes.
__device__ __forceinline__ void head_split8(const u32x4 (&v)[2], int n, char* hi_row, char* lo_row, int c) {
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = ldexpf(__uint_as_float(v[e / 4][e & 3]), n);
        hi[e] = static_cast<_Float16>(x);
        lo[e] = static_cast<_Float16>((x - (float)hi[e]) * kHeadLow);      // the difference is exact
    }
    reinterpret_cast<u32x4*>(hi_row)[c] = __builtin_bit_cast(u32x4, hi);
    reinterpret_cast<u32x4*>(lo_row)[c] = __builtin_bit_cast(u32x4, lo);
}

// Rows into the form the products read: gathered (source != null), padded with zeros to whole 16-byte chunks, fp32 ones as two fp16 planes.
// stacked != 0: all of them a second time, behind the last.
// fp32: row_const == null: W, times 2^w_exp; otherwise the rows of x for dW, each times 2^(dw_exp - its row of G's): what is worked out here of `largest`, the
// greatest exponents that tide_head_rows_kernel's workgroups have found.
// A workgroup has rows_each rows, taken as one list of chunks, four a thread at a time.
template <int DT>
__global__ __launch_bounds__(kHeadRowThreads) void tide_head_copy_kernel(const char* rows, int64_t row_bytes, int64_t n_rows, int rows_each, int d, const int32_t* source,
                                                                         HeadCtl* ctl, const float4* row_const, const int32_t* largest, int blocks, int stacked, char* out,
                                                                         int64_t out_row_bytes, int64_t plane_bytes) {
    const int64_t live = source ? ctl->live : n_rows, r0 = (int64_t)blockIdx.x * rows_each;
    if (r0 >= live) return;
    int scale = 0;
    if constexpr (DT == kF32) {
        scale = ctl->w_exp;
        if (row_const) {
            __shared__ int part[4];
            int most = INT_MIN;
            for (int i = threadIdx.x; i < blocks; i += kHeadRowThreads) most = max(most, largest[i]);
#pragma unroll
            for (int s = 1; s < kWave; s <<= 1) most = max(most, __shfl_xor(most, s, kWave));
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
            __syncthreads();
            most = max(max(part[0], part[1]), max(part[2], part[3]));
            scale = most == INT_MIN ? 0 : 14 - most;
            if (blockIdx.x == 0 && threadIdx.x == 0) ctl->dw_exp = scale;
        }
    }
    const bool chunks = ((uintptr_t)rows | (uintptr_t)row_bytes) % 16 == 0 && d % 8 == 0;
    const int per_row = (int)(out_row_bytes / 16), total = (int)min((int64_t)rows_each, live - r0) * per_row;
    constexpr int kU = 4, kW = DT == kF32 ? 2 : 1;     // 16-byte pieces of a chunk's source
    for (int i0 = threadIdx.x; i0 < total; i0 += kU * kHeadRowThreads) {
        u32x4 v[kU][kW];
        int64_t r[kU];
        int c[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int i = min(i0 + u * kHeadRowThreads, total - 1), q = i / per_row;
            r[u] = r0 + q;
            c[u] = i - q * per_row;
            const char* row = rows + (source ? (int64_t)source[r[u]] : r[u]) * row_bytes;
            head_load8<DT>(row, c[u], d, chunks, v[u]);
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            if (i0 + u * kHeadRowThreads >= total) break;
            char* to = out + r[u] * out_row_bytes;
            if constexpr (DT != kF32) {
                reinterpret_cast<u32x4*>(to)[c[u]] = v[u][0];
                if (stacked) reinterpret_cast<u32x4*>(to + live * out_row_bytes)[c[u]] = v[u][0];
            } else {
                head_split8(v[u], row_const ? scale - __float_as_int(row_const[r[u]].w) : scale, to, to + plane_bytes, c[u]);
            }
        }
    }
}

// fp32 rows of x for the logits, as planes: gathered (source != null), padded, each times the power of two that suits its own largest finite magnitude, so that
// a row's size is no other row's matter.  largest (with row_const): per workgroup, the greatest exponent of a row's largest magnitude less its row of G's power.
// A row per workgroup; kWavePerRow: a wave (d up to 2048: four chunks a lane at most).  The second read of a row is a cache's.
template <bool kWavePerRow>
__global__ __launch_bounds__(kHeadRowThreads) void tide_head_rows_kernel(const char* rows, int64_t row_bytes, int n_rows, int d, const int32_t* source, const HeadCtl* ctl,
                                                                         const float4* row_const, char* out, int64_t out_row_bytes, int64_t plane_bytes, int32_t* exps, int32_t* largest) {
    constexpr int kStep = kWavePerRow ? kWave : kHeadRowThreads, kRows = kWavePerRow ? 4 : 1;
    __shared__ uint32_t part[2][4];
    __shared__ int most_of[4];
    const int wave = threadIdx.x >> 6, tid = kWavePerRow ? threadIdx.x & 63 : threadIdx.x;
    const int live = source ? ctl->live : n_rows, per_row = (int)(out_row_bytes / 16);
    const bool chunks = ((uintptr_t)rows | (uintptr_t)row_bytes) % 16 == 0 && d % 8 == 0;
    int most = INT_MIN, turn = 0;
    for (int r = blockIdx.x * kRows + (kWavePerRow ? wave : 0); r < live; r += gridDim.x * kRows) {
        const char* row = rows + (int64_t)(source ? source[r] : r) * row_bytes;
        uint32_t m = 0;
        for (int c = tid; c < per_row; c += kStep) {
            u32x4 v[2];
            head_load8<kF32>(row, c, d, chunks, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = v[e / 4][e & 3] & 0x7fffffffu;
                m = b < 0x7f800000u && b > m ? b : m;
            }
        }
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s, kWave));
        if constexpr (!kWavePerRow) {
            if ((threadIdx.x & 63) == 0) part[turn][wave] = m;
            __syncthreads();                           // one barrier a row: the next row's maxima go into the other half
            m = max(max(part[turn][0], part[turn][1]), max(part[turn][2], part[turn][3]));
            turn ^= 1;
        }
        const int n = head_exponent(m);
        if (m != 0 && row_const) most = max(most, 14 - n - __float_as_int(row_const[r].w));
        if (tid == 0) exps[r] = n;
        char* to = out + r * out_row_bytes;
        for (int c = tid; c < per_row; c += kStep) {
            u32x4 v[2];
            head_load8<kF32>(row, c, d, chunks, v);
            head_split8(v, n, to, to + plane_bytes, c);
        }
    }
    if (!largest) return;
    if ((threadIdx.x & 63) == 0) most_of[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) largest[blockIdx.x] = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
}

// The teacher of one row: a wave, lanes over its K entries.  An entry counts if its token is one of the vocabulary's and its value is not -inf.  Differences from
// the largest value are taken before they are divided by tau: a row of the type's lowest value, which masks are made of, would overflow at tau < 1 otherwise.
struct HeadTeacher {
    float m, log_sum;          // largest value and log of the sum of exp((value - m) / tau)
    bool any;
};
__device__ __forceinline__ float head_wave_max(float v) {
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) v = fmaxf(v, __shfl_xor(v, s, kWave));
    return v;
}
__device__ __forceinline__ HeadTeacher head_teacher(const float* values, const int32_t* ids, int K, int V, float inv_tau, int lane) {
    float m = -INFINITY;
    bool any = false;
    for (int k = lane; k < K; k += kWave)
        if ((uint32_t)ids[k] < (uint32_t)V && values[k] != -INFINITY) {
            any = true;
            m = fmaxf(m, values[k]);
        }
    m = head_wave_max(m);
    float s = 0.0f;
    for (int k = lane; k < K; k += kWave)
        if ((uint32_t)ids[k] < (uint32_t)V && values[k] != -INFINITY) s += expf((values[k] - m) * inv_tau);
    return HeadTeacher{m, logf(wave_sum(s)), __any(any) != 0};
}

// [T][K] probabilities of the teacher (zero where it has no entry), and which rows have any.
__global__ __launch_bounds__(kHeadRowThreads) void tide_head_teacher_kernel(const float* values, const int32_t* ids, int T, int K, int V, float inv_tau,
                                                                            float* wanted, uint8_t* taught) {
    const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (t >= T) return;
    values += (int64_t)t * K, ids += (int64_t)t * K, wanted += (int64_t)t * K;
    const HeadTeacher h = head_teacher(values, ids, K, V, inv_tau, lane);
    for (int k = lane; k < K; k += kWave) {
        const bool there = (uint32_t)ids[k] < (uint32_t)V && values[k] != -INFINITY;
        wanted[k] = there ? expf((values[k] - h.m) * inv_tau - h.log_sum) : 0.0f;
    }
    if (lane == 0) taught[t] = h.any;
}

struct HeadFinishParams {
    const float2* part;        // [parts][T]
    int parts, T, K, V;
    float tau;
    const int32_t* ids;        // [T][K]
    const float* values;       // [T][K] teacher's values, or null: one hard target
    float* z;                  // [T][K] logits of the row's own tokens; with a teacher an output, zeros where there is no token
    float *loss, *lse;         // [T] out
};

// 16 rows per workgroup: 64 threads join a row's partial maxima and sums, then a wave takes its loss.
__global__ __launch_bounds__(1024) void tide_head_finish_kernel(const HeadFinishParams p) {
    __shared__ float2 part[64][17];
    const int tid = threadIdx.x, r = tid & 15, slice = tid >> 4, t = blockIdx.x * 16 + r;
    float m = -INFINITY, s = 0.0f;
    const float c1 = 1.4426950408889634f / p.tau;
    auto join = [c1](float& m, float& s, float m1, float s1) {
        const float top = fmaxf(m, m1), at = top == -INFINITY ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f((m - at) * c1) + s1 * __builtin_amdgcn_exp2f((m1 - at) * c1);
        m = top;
    };
    if (t < p.T)
        for (int i = slice; i < p.parts; i += 8 * 64) {        // eight loads at a time
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = i + u * 64 < p.parts ? p.part[(int64_t)(i + u * 64) * p.T + t] : float2{-INFINITY, 0.0f};
#pragma unroll
            for (int u = 0; u < 8; ++u) join(m, s, v[u].x, v[u].y);
        }
    part[slice][r] = float2{m, s};
    __syncthreads();
    const int wave = tid >> 6, lane = tid & 63, row = blockIdx.x * 16 + wave;      // wave w finishes row w
    const float2 v = part[lane][wave];
    m = v.x, s = v.y;
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) {
        const float m1 = __shfl_xor(m, x, kWave), s1 = __shfl_xor(s, x, kWave);
        join(m, s, m1, s1);
    }
    if (row >= p.T) return;
    const float log_s = logf(s), lse = m / p.tau + log_s;
    const int32_t* ids = p.ids + (int64_t)row * p.K;
    float* z = p.z + (int64_t)row * p.K;
    if (!p.values) {
        if (lane == 0) {
            p.lse[row] = lse;
            p.loss[row] = (uint32_t)ids[0] < (uint32_t)p.V ? (m - z[0]) / p.tau + log_s : 0.0f;
        }
        return;
    }
    const float inv_tau = 1.0f / p.tau;
    const float* values = p.values + (int64_t)row * p.K;
    const HeadTeacher h = head_teacher(values, ids, p.K, p.V, inv_tau, lane);
    float sum = 0.0f;
    for (int k = lane; k < p.K; k += kWave) {
        if ((uint32_t)ids[k] >= (uint32_t)p.V) {
            z[k] = 0.0f;
        } else if (values[k] != -INFINITY) {
            const float log_q = (values[k] - h.m) * inv_tau - h.log_sum, q = expf(log_q);
            sum += q == 0.0f ? 0.0f : q * (log_q + (m - z[k]) * inv_tau + log_s);      // (a NaN among the values is the row's loss, as it is its gradient)
        }
    }
    sum = wave_sum(sum);
    if (lane == 0) {
        p.lse[row] = lse;
        p.loss[row] = h.any ? p.tau * p.tau * sum : 0.0f;
    }
}

// dx, and dW where its k is in slices (place == null: every row is there): the slices' sums in order, scaled back, rounded once to the storage type; zeros in
// the rows that have no gradient.
template <int DT>
__global__ __launch_bounds__(kHeadRowThreads) void tide_head_dx_kernel(const float* acc, int slices, int64_t slice, int acc_ld, int stacked, const int32_t* place,
                                                                       const float4* row_const, const HeadCtl* ctl, int T, int d, char* out, int64_t out_row_bytes) {
    const bool chunks = ((uintptr_t)out | (uintptr_t)out_row_bytes) % 16 == 0 && d % 8 == 0;
    for (int t = blockIdx.x; t < T; t += gridDim.x) {
        const int i = place ? place[t] : t;
        const int back = !place ? -ctl->dw_exp : i >= 0 ? -(ctl->w_exp + __float_as_int(row_const[i].w)) : 0;
        char* to = out + (int64_t)t * out_row_bytes;
        for (int c = threadIdx.x; c < acc_ld / 8; c += kHeadRowThreads) {
            f32x4 a = {0, 0, 0, 0}, b = a;
            if (i >= 0) {
                const float* from = acc + (int64_t)i * acc_ld + 8 * c;
                auto add = [&](const float* from) {        // eight slices' loads at a time, added in order
                    for (int s0 = 0; s0 < slices; s0 += 8) {
                        f32x4 v[8][2];
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            const f32x4* at = reinterpret_cast<const f32x4*>(from + min(s0 + u, slices - 1) * slice);
                            v[u][0] = at[0], v[u][1] = at[1];
                        }
#pragma unroll
                        for (int u = 0; u < 8; ++u)
                            if (s0 + u < slices) a += v[u][0], b += v[u][1];
                    }
                };
                add(from);
                if (stacked) add(from + (int64_t)ctl->live * acc_ld);        // the part of G's second plane
            }
            a = head_shifted(a, back);
            b = head_shifted(b, back);
            if (chunks) {
                if constexpr (DT == kF32) {
                    reinterpret_cast<f32x4*>(to)[2 * c] = a;
                    reinterpret_cast<f32x4*>(to)[2 * c + 1] = b;
                } else {
                    reinterpret_cast<u32x4*>(to)[c] = u32x4{head_round2<DT>(a[0], a[1]), head_round2<DT>(a[2], a[3]), head_round2<DT>(b[0], b[1]), head_round2<DT>(b[2], b[3])};
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * c + e < d) head_put<DT>(to, 8 * c + e, e < 4 ? a[e & 3] : b[e & 3]);
            }
        }
    }
}

}  // namespace tide
