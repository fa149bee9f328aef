// The rules of decoding on rows of logits: penalties for tokens of the past, biases, a grammar's mask; and the token with the largest of the logits so ruled.
//
// A workgroup has a slice of a row's tokens, up to 32768.  It counts the row's past in a table of its slice in LDS, 16 bits a token (32 for pasts that could
// overflow them), then passes over the slice's logits once, the first of which are requested before the counting.  A bias is the business of the thread that
// has its first entry: it fetched the logit before anything was written, adds up the token's entries in their order and deals with the token in place of the
// pass.  Integer counts do not depend on the order of their atomics and every sum has a fixed order: the results do not depend on timing.
//
// Small calls are bound by the launch and the latency of a few dependent loads (one row of 128000 tokens in fp32, past of 700, 8 biases, mask: 4.9 us, with the largest
// 5.9 and 1.8 for the join), large ones by vector instructions: 256 such rows with pasts of 4096 and 16 biases take 41 us, 3.3 TB/s, of which the past's rules, which
// some lane of a wave nearly always needs, are half of the instructions and the exponentials a fifth.
#pragma once
#include "device_utils.hpp"

namespace tide {

constexpr int kRuleThreads = 1024, kRuleJoinThreads = 256, kRuleWaves = 8;      // waves a SIMD: two workgroups a CU

struct RuleParams {
    const char* z;
    char* out;
    int64_t row_bytes, out_row_bytes;
    int T, V, H, B;
    int slice, slices;         // tokens of a slice (a multiple of 128), slices of a row
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

// exp(d), d <= 0 or NaN, to 2^-22: 2^t of t = d log2 e rounded, which alone is off by up to 2^-24 |d| (1.2e-6 at d = -20), and what the rounding left, d - t ln 2, of ln 2 in two
// parts.  (Below -150 all is zero, and -inf would leave no number.)  Four instructions a logit more than 2^t alone: a call of 256 rows of 128000 in fp32 42 -> 44 us, in bf16 35 -> 38.
__device__ __forceinline__ float rule_exp(float d) {
    d = __builtin_elementwise_maximum(d, -150.0f);
    const float t = d * 0x1.715476p+0f, rest = fmaf(-t, -0x1.05c61p-29f, fmaf(-t, 0x1.62e430p-1f, d)), e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, rest, e);
}

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
    return Best{hi.most, hi.token, hi.rest + (1.0f + lo.rest) * rule_exp(lo.most - hi.most)};
}
// The same over a wave: the largest, the lowest of its tokens, then every lane's sum relative to it, added up in a fixed order.
template <int kCtrl> __device__ __forceinline__ uint32_t dpp_u32(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xF, 0xF, false); }
template <typename F> __device__ __forceinline__ uint32_t wave_fold(uint32_t v, F&& f) {
    v = f(v, dpp_u32<kDppXor1>(v));
    v = f(v, dpp_u32<kDppXor2>(v));
    v = f(v, dpp_u32<kDppHalfMirror>(v));
    v = f(v, dpp_u32<kDppRor8>(v));
    v = f(v, (uint32_t)__shfl_xor((int)v, 16, kWave));
    return f(v, (uint32_t)__shfl_xor((int)v, 32, kWave));
}
__device__ __forceinline__ Best best_of_wave(const Best& a) {
    const float most = __uint_as_float(wave_fold(__float_as_uint(a.most), [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }));
    // (no token: the largest unsigned number)
    const int32_t token = (int32_t)wave_fold(a.most == most ? (uint32_t)a.token : ~0u, [](uint32_t x, uint32_t y) { return min(x, y); });
    float rest = a.rest;
    if (a.token >= 0) rest = a.token == token ? rest : (1.0f + rest) * rule_exp(a.most - most);
    return Best{most, token, wave_sum(rest)};
}
__device__ __forceinline__ void best_write(const Best& a, int32_t* token, float* log_prob) {
    const bool none = a.token < 0, wrong = a.rest != a.rest;
    *token = none || wrong ? -1 : a.token;
    *log_prob = wrong ? __uint_as_float(0x7fc00000u) : none ? -INFINITY : -log1pf(a.rest);
}

// 16 bytes of logits, as they lie in memory (rows of odd sizes: aligned to their elements only), and single ones.
template <int DT> __device__ __forceinline__ float rule_value(const u32x4& raw, int e) {
    if constexpr (DT == kF32) return __uint_as_float(raw[e]);
    else if constexpr (DT == kBF16) return __uint_as_float(e % 2 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(e % 2 ? raw[e / 2] >> 16 : raw[e / 2]));
}
template <int DT> __device__ __forceinline__ uint32_t rule_bits(float a) {
    if constexpr (DT == kF32) return __float_as_uint(a);
    else if constexpr (DT == kBF16) return __builtin_bit_cast(uint16_t, (__bf16)a);
    else return __builtin_bit_cast(uint16_t, (_Float16)a);
}
template <int DT> constexpr uint32_t kRuleLow = DT == kF32 ? 0xff800000u : DT == kBF16 ? 0xff80u : 0xfc00u;      // -inf
template <int DT> __device__ __forceinline__ void rule_insert(u32x4& raw, int e, uint32_t bits) {
    if constexpr (DT == kF32) raw[e] = bits;
    else raw[e / 2] = e % 2 ? (raw[e / 2] & 0xffffu) | bits << 16 : (raw[e / 2] & 0xffff0000u) | bits;
}
template <int DT> __device__ __forceinline__ uint32_t rule_load1(const char* p) {
    if constexpr (DT == kF32) return *reinterpret_cast<const uint32_t*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
}
template <int DT> __device__ __forceinline__ void rule_store1(char* p, uint32_t bits) {
    if constexpr (DT == kF32) *reinterpret_cast<uint32_t*>(p) = bits;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)bits;
}

// The past's rules for one logit; every operation rounded by itself, in the order of the formula.  Division by the row's penalty: times its reciprocal in 64 bits, which
// is off by 2^-52 of the quotient, and a quotient of two 24-bit numbers is never that near to a midpoint of two 24-bit ones (2^-49): rounded to 32 bits it is the quotient
// rounded once.  (Quotients below 2^-126, which have fewer bits, may be off by one of their steps where they lie at a midpoint.)
struct RuleRow {
    float repetition, presence, frequency;
    double inverse;
};
__device__ __forceinline__ float rule_past(float a, uint32_t count, const RuleRow& r) {
#pragma clang fp contract(off)
    const float less = (float)((double)a * r.inverse), more = a * r.repetition;
    a = a > 0.0f ? less : more;
    if (count > 1) {
        const float often = r.frequency * (float)(count >> 1);
        a = a - (often + r.presence);
    }
    return a;
}

// A slice's tables in LDS.  A token's count: twice the times that it was generated, and bit 0 where the prompt has it.
struct RuleTables {
    int counts, ids, values, biased, twice, bytes;     // biased, twice: a bit for each token that has an entry, several
};
__host__ __device__ inline RuleTables rule_tables(int slice, int count_bytes, int B) {
    RuleTables t{};
    const int entries = (B + 3) / 4 * 4;
    t.ids = t.counts + slice * count_bytes;
    t.values = t.ids + entries * 4;
    t.biased = t.values + entries * 4;
    t.twice = t.biased + (B ? slice / 8 : 0);
    t.bytes = t.twice + (B ? slice / 8 : 0);
    return t;
}

// kWide: counts of 32 bits.
template <int DT, bool kPick, bool kWide> __global__ __launch_bounds__(kRuleThreads, kRuleWaves) void tide_logit_rules_kernel(RuleParams p) {
    constexpr int kB = Storage<DT>::kBytes, N = 16 / kB, kStep = kRuleThreads * N;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Best of_wave[kRuleThreads / kWave];
    __shared__ int entries[kRuleThreads / kWave];
    const int tid = threadIdx.x, t = blockIdx.x / p.slices, part = blockIdx.x - t * p.slices, v0 = part * p.slice, width = min(p.slice, p.V - v0), whole = width & -N;
    const char* const z = p.z + (int64_t)t * p.row_bytes + (int64_t)v0 * kB;
    char* const out = kPick ? nullptr : p.out + (int64_t)t * p.out_row_bytes + (int64_t)v0 * kB;
    const uint32_t* const allowed = p.allowed ? p.allowed + (int64_t)t * p.words + v0 / 32 : nullptr;

    // 16 bytes a thread ahead: with the other waves' that is enough, and the registers of more are another workgroup's
    u32x4 raw;
    uint32_t may = 0xffffffffu;
    auto request = [&](int i) {
        if (i >= whole) return;
        if (allowed) may = allowed[i / 32] >> (i & 31);
        __builtin_memcpy(&raw, z + (int64_t)i * kB, 16);
    };
    request(tid * N);

    const RuleTables at = rule_tables(p.slice, p.H ? (kWide ? 4 : 2) : 0, p.B);
    uint32_t* const counts = reinterpret_cast<uint32_t*>(lds + at.counts);
    uint32_t *const biased = reinterpret_cast<uint32_t*>(lds + at.biased), *const twice = reinterpret_cast<uint32_t*>(lds + at.twice);
    RuleRow row = {1.0f, 0.0f, 0.0f, 1.0};
    // this thread's single tokens of the slice, or -1: its bias's, where that is the first entry of its token, and one of those behind the last whole 16 bytes
    int bias_at = -1, tail_at = tid < width - whole ? whole + tid : -1;
    float bias = 0.0f;
    uint32_t bias_bits = 0, tail_bits = tail_at >= 0 ? rule_load1<DT>(z + (int64_t)tail_at * kB) : 0;
    if (p.H || p.B) {
        const int32_t* const past = p.past + (int64_t)t * p.H;
        // 16 tokens a thread at a time; the first are requested before the tables are cleared
        constexpr int kTokens = 4 * kRuleThreads;
        const int whole_past = p.H & ~3;
        int32_t some[4][4], last = -1;
        auto bring = [&](int i0) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * kTokens + tid * 4;
                if (i < whole_past) __builtin_memcpy(some[u], past + i, 16);
            }
        };
        bring(0);
        if (tid < p.H - whole_past) last = past[whole_past + tid];
        const int n = p.H && p.past_len ? min(p.past_len[t], p.H) : p.H, prompt = p.prompt_len ? p.prompt_len[t] : 0;
        if (p.repetition) row.repetition = p.repetition[t];
        if (p.presence) row.presence = p.presence[t];
        if (p.frequency) row.frequency = p.frequency[t];
        if (tid < p.B) {
            const int32_t bias_id = p.bias_ids[(int64_t)t * p.B + tid];
            bias = p.bias_values[(int64_t)t * p.B + tid];
            if ((uint32_t)bias_id - (uint32_t)v0 < (uint32_t)width) bias_at = bias_id - v0;
            if (bias_at >= 0) bias_bits = rule_load1<DT>(z + (int64_t)bias_at * kB);
        }
        for (int i = tid * 16; i < at.bytes; i += kRuleThreads * 16)
            if (i < at.ids || i >= at.biased) *reinterpret_cast<u32x4*>(lds + i) = u32x4{0, 0, 0, 0};
        if (tid < (p.B + 3) / 4 * 4) {
            reinterpret_cast<int32_t*>(lds + at.ids)[tid] = -1;        // (no entry)
        }
        __syncthreads();
        auto count = [&](int32_t token, int i) {
            const uint32_t v = (uint32_t)token - (uint32_t)v0;         // (a negative token is beyond any slice)
            if (i >= n || v >= (uint32_t)width) return;
            uint32_t* const word = kWide ? counts + v : counts + v / 2;
            const int shift = kWide ? 0 : 16 * (v & 1);
            if (i >= prompt) atomicAdd(word, 2u << shift);
            else atomicOr(word, 1u << shift);
        };
        for (int i0 = 0; i0 < n; i0 += 4 * kTokens) {
            if (i0) bring(i0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * kTokens + tid * 4;
                if (i >= min(n, whole_past)) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) count(some[u][e], i + e);
            }
        }
        if (tid < p.H - whole_past) count(last, whole_past + tid);
        if (p.B) {
            const uint32_t bit = 1u << (bias_at & 31);
            if (bias_at >= 0 && (atomicOr(&biased[bias_at / 32], bit) & bit)) atomicOr(&twice[bias_at / 32], bit);
            __syncthreads();
            // The entries of tokens that have several, by wave and in their order: their threads look through them for their token's.  The first entry of a token adds up the
            // others, the others' threads have nothing left to do.  (64 rows of 50261 tokens in bf16, 300 biases, half of
            // them on a seventh of the tokens: 11.9 us; token after token, a wave at a time, 14.4.)
            const int lane = tid % kWave, wave = tid / kWave;
            const uint64_t several = __ballot(bias_at >= 0 && (twice[bias_at / 32] & bit));
            const int mine = wave * kWave + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(several >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)several, 0));
            const bool one_of = several >> lane & 1;
            if (one_of) {
                reinterpret_cast<int32_t*>(lds + at.ids)[mine] = bias_at;
                reinterpret_cast<float*>(lds + at.values)[mine] = bias;
            }
            if (lane == 0) entries[wave] = __popcll(several);
            __syncthreads();
            if (several) {
                bool first = true;
                for (int w = 0; w * kWave < p.B; ++w) {
                    const int n = __builtin_amdgcn_readfirstlane(entries[w]);
                    for (int m = w * kWave; m < w * kWave + n; m += 4) {
                        const u32x4 id = *reinterpret_cast<const u32x4*>(lds + at.ids + m * 4);
                        const f32x4 value = *reinterpret_cast<const f32x4*>(lds + at.values + m * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool same = (int)id[e] == bias_at && one_of;
                            first = first && !(same && m + e < mine);
                            bias = same && m + e > mine ? bias + value[e] : bias;
                        }
                    }
                }
                if (!first) bias_at = -1;
            }
            if (tail_at >= 0 && (biased[tail_at / 32] >> (tail_at & 31) & 1)) tail_at = -1;
        }
        __syncthreads();
        row.inverse = 1.0 / (double)row.repetition;
    }

    Best best = best_none();
    for (int i = tid * N; i < whole; i += kStep) {
        u32x4 now = raw;
        const uint32_t bits = may;
        request(i + kStep);
        float a[N];
        if constexpr (kPick) {
#pragma unroll
            for (int e = 0; e < N; ++e) a[e] = rule_value<DT>(now, e);
        }
        if (p.H) {
            uint32_t c[kWide ? N : N / 2];
#pragma unroll
            for (int w = 0; w < (kWide ? N : N / 2); ++w) c[w] = counts[(kWide ? i : i / 2) + w];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t count = kWide ? c[e] : c[e / 2] >> (16 * (e % 2)) & 0xffffu;
                if (count) {
                    if constexpr (kPick) a[e] = rule_past(a[e], count, row);
                    else rule_insert<DT>(now, e, rule_bits<DT>(rule_past(rule_value<DT>(now, e), count, row)));
                }
            }
        }
        if constexpr (!kPick) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (!(bits >> e & 1)) rule_insert<DT>(now, e, kRuleLow<DT>);
            __builtin_memcpy(out + (int64_t)i * kB, &now, 16);
        } else {
            uint32_t out_of_it = ~bits;                // masked, or a bias's thread's
            if (p.B) out_of_it |= biased[i / 32] >> (i & 31);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (out_of_it >> e & 1) a[e] = -INFINITY;
            float most = a[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most = fmaxf(most, a[e]);
            int own = -1;
            if (most > best.most) {
#pragma unroll
                for (int e = N - 1; e >= 0; --e) own = a[e] == most ? e : own;
                if (best.token >= 0) best.rest = (1.0f + best.rest) * rule_exp(best.most - most);
                best.most = most;
                best.token = v0 + i + own;
            }
            const float base = fmaxf(best.most, -3.4028235e38f);   // (nothing but -inf yet: zeros, and a NaN is one)
#pragma unroll
            for (int e = 0; e < N; ++e) best.rest += rule_exp((e == own ? -INFINITY : a[e]) - base);
        }
    }
    // the single tokens
    if constexpr (!kPick) {
        if (p.B) __syncthreads();                      // (the pass wrote the biases' tokens without them)
    }
    auto single = [&](int v, uint32_t bits, float more) {
        uint32_t count = 0;
        if (p.H) count = kWide ? counts[v] : counts[v / 2] >> (16 * (v & 1)) & 0xffffu;
        const bool in = !allowed || (allowed[v / 32] >> (v & 31) & 1), touched = count || bias_at == v;
        float a = rule_value<DT>(u32x4{bits, 0, 0, 0}, 0);
        if (count) a = rule_past(a, count, row);
        if (bias_at == v) a += more;
        if constexpr (!kPick) {
            rule_store1<DT>(out + (int64_t)v * kB, !in ? kRuleLow<DT> : touched ? rule_bits<DT>(a) : bits);
        } else if (in) {
            if (a != a) best.rest = a;
            else if (a > -INFINITY) best = best_of(best, Best{a, v0 + v, 0.0f});
        }
    };
    if (bias_at >= 0) single(bias_at, bias_bits, bias);
    if (tail_at >= 0) single(tail_at, tail_bits, 0.0f);
    if constexpr (kPick) {
        best = best_of_wave(best);
        if (tid % kWave == 0) of_wave[tid / kWave] = best;
        __syncthreads();
        if (tid < kWave) {
            best = best_of_wave(tid < kRuleThreads / kWave ? of_wave[tid] : best_none());
            if (tid == 0) {
                if (p.slices == 1) best_write(best, p.token + t, p.log_prob + t);
                else p.part[(int64_t)t * p.slices + part] = make_uint4(__float_as_uint(best.most), (uint32_t)best.token, __float_as_uint(best.rest), 0u);
            }
        }
    }
}

// The slices of a row joined: a wave per row.
__global__ __launch_bounds__(kRuleJoinThreads) void tide_logit_join_kernel(const uint4* part, int T, int slices, int32_t* token, float* log_prob) {
    const int t = blockIdx.x * (kRuleJoinThreads / kWave) + threadIdx.x / kWave;
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
