// The rules of decoding on rows of logits: penalties for tokens of the past, biases, a grammar's mask; and the token with the largest of the logits so ruled.
//
// A workgroup has a slice of a row's tokens.  It counts the row's past in a table of its slice in LDS (one word per token), lays the biases beside it, then
// passes over the slice's logits once.  Integer counts do not depend on the order of their atomics, and the entries of one token's bias are added by one thread, in their
// order: the results do not depend on timing.
#pragma once
#include "device_utils.hpp"

namespace tide {

constexpr int kRuleThreads = 256;

struct RuleParams {
    const char* z;
    char* out;
    int64_t row_bytes, out_row_bytes;
    int T, V, H, B;
    int slice, slices;         // tokens of a slice (a multiple of 32), slices of a row
    const int32_t *past, *past_len, *prompt_len;
    const float *repetition, *presence, *frequency;
    const int32_t* bias_ids;
    const float* bias_values;
    const uint32_t* allowed;
    int words;                 // of a row's mask
    int32_t* token;
    float* log_prob;
    uint4* part;               // [T][slices], where a row has several
};

// The largest of some logits, its token, and the sum of exp(others - largest).  Nothing yet: token -1.  A NaN among them: NaN, which stays.
struct Best {
    float most;
    int32_t token;
    float rest;
};
__device__ __forceinline__ Best best_none() { return Best{-INFINITY, -1, 0.0f}; }
__device__ __forceinline__ Best best_of(const Best& a, const Best& b) {
    if (b.token < 0) return Best{a.most, a.token, a.rest + b.rest};      // (b.rest: zero, or NaN)
    if (a.token < 0) return Best{b.most, b.token, a.rest + b.rest};
    const bool first = a.most > b.most || (a.most == b.most && a.token < b.token);
    const Best &hi = first ? a : b, &lo = first ? b : a;
    // (equal infinities: the difference is no number and the sum becomes none, as the log-probability of one of two infinities is)
    return Best{hi.most, hi.token, hi.rest + (1.0f + lo.rest) * __expf(lo.most - hi.most)};
}
__device__ __forceinline__ Best best_exchange(const Best& a, int x) {
    return Best{__shfl_xor(a.most, x, kWave), __shfl_xor(a.token, x, kWave), __shfl_xor(a.rest, x, kWave)};
}
__device__ __forceinline__ Best best_of_wave(Best a) {
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) a = best_of(a, best_exchange(a, x));
    return a;
}
__device__ __forceinline__ void best_write(const Best& a, int32_t* token, float* log_prob) {
    const bool none = a.token < 0, wrong = a.rest != a.rest;
    *token = none || wrong ? -1 : a.token;
    *log_prob = wrong ? __uint_as_float(0x7fc00000u) : none ? -INFINITY : -log1pf(a.rest);
}

template <int DT> __device__ __forceinline__ void rule_load(const char* p, float (&x)[16 / Storage<DT>::kBytes]) {
    uint32_t c[4];
    __builtin_memcpy(c, p, 16);                        // rows of odd sizes: aligned to their elements only
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (DT == kF32) {
            x[e] = __uint_as_float(c[e]);
        } else if constexpr (DT == kBF16) {
            x[2 * e] = __uint_as_float(c[e] << 16);
            x[2 * e + 1] = __uint_as_float(c[e] & 0xffff0000u);
        } else {
            const f16x2 h = __builtin_bit_cast(f16x2, c[e]);
            x[2 * e] = (float)h[0];
            x[2 * e + 1] = (float)h[1];
        }
    }
}
template <int DT> __device__ __forceinline__ float rule_load1(const char* p) {
    if constexpr (DT == kF32) return *reinterpret_cast<const float*>(p);
    else if constexpr (DT == kBF16) return bf16_bits_to_f32(*reinterpret_cast<const uint16_t*>(p));
    else return (float)*reinterpret_cast<const _Float16*>(p);
}
template <int DT> __device__ __forceinline__ void rule_store1(char* p, float x) {
    if constexpr (DT == kF32) *reinterpret_cast<float*>(p) = x;
    else if constexpr (DT == kBF16) *reinterpret_cast<__bf16*>(p) = (__bf16)x;
    else *reinterpret_cast<_Float16*>(p) = (_Float16)x;
}
template <int DT> __device__ __forceinline__ void rule_store(char* p, const float (&x)[16 / Storage<DT>::kBytes]) {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (DT == kF32) c[e] = __float_as_uint(x[e]);
        else if constexpr (DT == kBF16) c[e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * e], (__bf16)x[2 * e + 1]});
        else c[e] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * e], (_Float16)x[2 * e + 1]});
    }
    __builtin_memcpy(p, c, 16);
}

// One logit's rules; every operation rounded by itself, in the order of the formula.
struct RuleRow {
    float repetition, presence, frequency;
};
__device__ __forceinline__ float rule_past(float a, uint32_t count, const RuleRow& r) {
#pragma clang fp contract(off)
    if (count) a = a > 0.0f ? a / r.repetition : a * r.repetition;
    if (count > 1) {
        const float often = r.frequency * (float)(count >> 1);
        a = a - (often + r.presence);
    }
    return a;
}

// The tables of a slice, in LDS.
struct RuleTables {
    uint32_t* counts;          // of a token: twice the times that it was generated, and bit 0 where the prompt has it
    float* bias;               // the sum of a token's entries, where it has any
    uint32_t *biased, *twice;  // a bit for each token with an entry, with several
};
// The layout; returns its bytes.
__host__ __device__ inline int rule_tables(char* base, int slice, bool past, bool bias, RuleTables* t) {
    int at = 0;
    t->counts = (uint32_t*)base;
    if (past) at += slice * 4;
    t->bias = (float*)(base + at);
    if (bias) at += slice * 4;
    t->biased = (uint32_t*)(base + at);
    if (bias) at += slice / 8;
    t->twice = (uint32_t*)(base + at);
    if (bias) at += slice / 8;
    return at;
}
__device__ __forceinline__ void rule_fill(const RuleParams& p, int t, int v0, int width, const RuleTables& tab) {
    const int tid = threadIdx.x;
    if (p.H)
        for (int i = tid; i < p.slice; i += kRuleThreads) tab.counts[i] = 0;
    if (p.B)
        for (int i = tid; i < p.slice / 32; i += kRuleThreads) tab.biased[i] = tab.twice[i] = 0;
    __syncthreads();
    if (p.H) {
        const int32_t* past = p.past + (int64_t)t * p.H;
        const int n = p.past_len ? min(p.past_len[t], p.H) : p.H, prompt = p.prompt_len ? p.prompt_len[t] : 0;
        for (int i = tid; i < n; i += kRuleThreads) {
            const uint32_t at = (uint32_t)past[i] - (uint32_t)v0;      // (a negative token is beyond any slice)
            if (at >= (uint32_t)width) continue;
            if (i >= prompt) atomicAdd(&tab.counts[at], 2u);
            else atomicOr(&tab.counts[at], 1u);
        }
    }
    if (p.B) {
        const int32_t* ids = p.bias_ids + (int64_t)t * p.B;
        const float* values = p.bias_values + (int64_t)t * p.B;
        for (int k = tid; k < p.B; k += kRuleThreads) {
            const uint32_t at = (uint32_t)ids[k] - (uint32_t)v0, bit = 1u << (at & 31);
            if (at < (uint32_t)width && (atomicOr(&tab.biased[at / 32], bit) & bit)) atomicOr(&tab.twice[at / 32], bit);
        }
        __syncthreads();
        for (int k = tid; k < p.B; k += kRuleThreads) {
            const int32_t id = ids[k];
            const uint32_t at = (uint32_t)id - (uint32_t)v0;
            if (at >= (uint32_t)width) continue;
            float sum = values[k];
            if (tab.twice[at / 32] >> (at & 31) & 1) { // the first entry of a token adds up the others, in their order
                bool first = true;
                for (int m = 0; m < k && first; ++m) first = ids[m] != id;
                if (!first) continue;
                for (int m = k + 1; m < p.B; ++m)
                    if (ids[m] == id) sum += values[m];
            }
            tab.bias[at] = sum;
        }
    }
    __syncthreads();
}

template <int DT, bool kPick> __global__ __launch_bounds__(kRuleThreads) void tide_logit_rules_kernel(RuleParams p) {
    constexpr int kB = Storage<DT>::kBytes, N = 16 / kB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Best of_wave[kRuleThreads / kWave];
    const int t = blockIdx.x / p.slices, part = blockIdx.x - t * p.slices, v0 = part * p.slice, width = min(p.slice, p.V - v0);
    RuleTables tab;
    rule_tables(lds, p.slice, p.H != 0, p.B != 0, &tab);
    if (p.H || p.B) rule_fill(p, t, v0, width, tab);
    const RuleRow row = {p.repetition ? p.repetition[t] : 1.0f, p.presence ? p.presence[t] : 0.0f, p.frequency ? p.frequency[t] : 0.0f};
    const char* z = p.z + (int64_t)t * p.row_bytes;
    char* out = kPick ? nullptr : p.out + (int64_t)t * p.out_row_bytes;
    const uint32_t* allowed = p.allowed ? p.allowed + (int64_t)t * p.words : nullptr;
    Best best = best_none();
    for (int i = threadIdx.x * N; i < width; i += kRuleThreads * N) {
        const int v = v0 + i, n = min(N, width - i);
        float a[N];
        if (n == N) {
            rule_load<DT>(z + (int64_t)v * kB, a);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) a[e] = e < n ? rule_load1<DT>(z + (int64_t)(v + e) * kB) : -INFINITY;
        }
        if (p.H) {
#pragma unroll
            for (int e = 0; e < N; ++e) a[e] = rule_past(a[e], tab.counts[i + e], row);
        }
        if (p.B) {
            const uint32_t bits = tab.biased[i / 32] >> (i & 31);
            if (bits & ((1u << N) - 1)) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (bits >> e & 1) a[e] += tab.bias[i + e];
            }
        }
        if (allowed) {
            const uint32_t bits = allowed[v / 32] >> (v & 31);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (!(bits >> e & 1)) a[e] = -INFINITY;
        }
        if constexpr (!kPick) {
            if (n == N) {
                rule_store<DT>(out + (int64_t)v * kB, a);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (e < n) rule_store1<DT>(out + (int64_t)(v + e) * kB, a[e]);
            }
        } else {
            float most = a[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most = fmaxf(most, a[e]);
            int own = -1;
            if (most > best.most) {
#pragma unroll
                for (int e = N - 1; e >= 0; --e) own = a[e] == most ? e : own;
                if (best.token >= 0) best.rest = (1.0f + best.rest) * __expf(best.most - most);
                best.most = most;
                best.token = v + own;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (best.token >= 0 ? e != own : a[e] != a[e]) best.rest += __expf(a[e] - best.most);
            }
        }
    }
    if constexpr (kPick) {
        best = best_of_wave(best);
        if (threadIdx.x % kWave == 0) of_wave[threadIdx.x / kWave] = best;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < kRuleThreads / kWave; ++w) best = best_of(best, of_wave[w]);
            if (p.slices == 1) best_write(best, p.token + t, p.log_prob + t);
            else p.part[(int64_t)t * p.slices + part] = make_uint4(__float_as_uint(best.most), (uint32_t)best.token, __float_as_uint(best.rest), 0u);
        }
    }
}

// The slices of a row joined: a wave per row.
__global__ __launch_bounds__(kRuleThreads) void tide_logit_join_kernel(const uint4* part, int T, int slices, int32_t* token, float* log_prob) {
    const int t = blockIdx.x * (kRuleThreads / kWave) + threadIdx.x / kWave;
    if (t >= T) return;
    Best best = best_none();
    for (int i = threadIdx.x % kWave; i < slices; i += kWave) {
        const uint4 q = part[(int64_t)t * slices + i];
        best = best_of(best, Best{__uint_as_float(q.x), (int32_t)q.y, __uint_as_float(q.z)});
    }
    best = best_of_wave(best);
    if (threadIdx.x % kWave == 0) best_write(best, token + t, log_prob + t);
}

}  // namespace tide
