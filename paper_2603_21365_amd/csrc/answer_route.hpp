// Host side of the answer operators (include/tide_route.h): the LM head in four bits and the rules of decoding.  Argument checks, the division of the work and the launches.
// Included by tide_route.hip behind head_route.hpp, whose limits of T and V it shares.
#pragma once

namespace {

constexpr int kMostLds = 158 * 1024;                   // dynamic LDS of a workgroup: some is left for what a kernel has beside it
constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1;      // a launch has fewer than 2^32 threads, a workgroup 256 (of the rules: 1024)

struct Q4Shape {
    int64_t V, d, group;
    int scale_dtype;
    int64_t tiles() const { return (V + kQ4Rows - 1) / kQ4Rows; }
    int64_t blocks() const { return (d + kQ4Cols - 1) / kQ4Cols; }
    int64_t groups() const { return (d + group - 1) / group; }
};

int check_q4(const Q4Shape& s, int dtype, const void* codes, const void* scales) {
    if (dtype != TIDE_F32 && dtype != TIDE_F16 && dtype != TIDE_BF16) return fail(TIDE_ERR_INVALID_ARG, "dtype %d is not a tide_dtype_t", dtype);
    if (s.scale_dtype != TIDE_F16 && s.scale_dtype != TIDE_BF16) return fail(TIDE_ERR_INVALID_ARG, "scale_dtype %d: TIDE_F16 or TIDE_BF16", s.scale_dtype);
    if (s.d <= 0) return fail(TIDE_ERR_INVALID_ARG, "d = %lld must be positive", (long long)s.d);
    if (s.d > kMaxHidden) return fail(TIDE_ERR_UNSUPPORTED, "d = %lld: hidden sizes from 1 to 16384", (long long)s.d);
    if (s.V <= 0) return fail(TIDE_ERR_INVALID_ARG, "V = %lld must be positive", (long long)s.V);
    if (s.V > kHeadMostVocab) return fail(TIDE_ERR_UNSUPPORTED, "V = %lld exceeds %lld", (long long)s.V, (long long)kHeadMostVocab);
    if (s.group != 32 && s.group != 64 && s.group != 128) return fail(TIDE_ERR_UNSUPPORTED, "group = %lld: 32, 64 or 128 columns", (long long)s.group);
    if (!codes || !scales) return fail(TIDE_ERR_INVALID_ARG, "codes and scales must not be NULL");
    if (((uintptr_t)codes | (uintptr_t)scales) & 15) return fail(TIDE_ERR_ALIGNMENT, "codes and scales must be 16-byte aligned");
    return TIDE_OK;
}
// Rows of an operand: a base and a stride that are multiples of an element.
int check_q4_rows(const void* rows, int64_t stride, int64_t d, int dtype, const char* name) {
    const size_t eb = elem_bytes(dtype);
    if (!rows) return fail(TIDE_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (stride < d) return fail(TIDE_ERR_INVALID_ARG, "%s: the row stride must be at least d", name);
    if ((uintptr_t)rows % eb) return fail(TIDE_ERR_ALIGNMENT, "%s must be aligned to its elements", name);
    return TIDE_OK;
}
bool q4_chunks(const void* rows, int64_t stride, int dtype) { return (((uintptr_t)rows | ((size_t)stride * elem_bytes(dtype))) & 15) == 0; }

template <typename F> int by_runs(int64_t group, F&& f) {
    using std::integral_constant;
    if (group == 32) return f(integral_constant<int, 1>{});
    if (group == 64) return f(integral_constant<int, 2>{});
    return f(integral_constant<int, 4>{});
}

int q4_weights(const void* W, void* W_out, int dtype, const Q4Shape& s, int64_t w_row_stride, const void* codes, const void* scales, hipStream_t st) {
    int rc = check_q4(s, dtype, codes, scales);
    if (rc || (rc = check_q4_rows(W ? W : W_out, w_row_stride, s.d, dtype, "W"))) return rc;
    const int64_t tiles = s.tiles() * s.blocks(), blocks = (tiles + 3) / 4;
    if (blocks > kMostBlocks) return fail(TIDE_ERR_UNSUPPORTED, "V = %lld rows of d = %lld are too many for one call", (long long)s.V, (long long)s.d);
    Q4WeightParams p{};
    p.W_out = (char*)W_out;
    p.row_bytes = w_row_stride * (int64_t)elem_bytes(dtype);
    p.codes = (char*)codes;
    p.scales = (uint16_t*)scales;
    p.V = (int)s.V;
    p.d = (int)s.d;
    p.blocks = (int)s.blocks();
    p.groups = (int)s.groups();
    p.half = s.scale_dtype == TIDE_F16;
    p.chunks = q4_chunks(W ? W : W_out, w_row_stride, dtype);
    p.tiles = tiles;
    p.x = Q4Rows{(const char*)W, p.row_bytes, p.V, p.d, p.chunks};
    by_dtype(dtype, [&](auto dt) {
        return by_runs(s.group, [&](auto runs) {
            constexpr int DT = decltype(dt)::value, kRuns = decltype(runs)::value;
            if (W) hipLaunchKernelGGL((tide_head_quantize_kernel<DT, kRuns>), dim3((unsigned)blocks), dim3(kQ4Threads), 0, st, p);
            else hipLaunchKernelGGL((tide_head_dequantize_kernel<DT, kRuns>), dim3((unsigned)blocks), dim3(kQ4Threads), 0, st, p);
            return 0;
        });
    });
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

// A kernel's dynamic LDS beyond the default, once per device.
template <auto kKernel> int raise_lds() {
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    int rc = current_device(&dev);
    if (rc) return rc;
    if (!raised[dev].load(std::memory_order_relaxed)) {
        TIDE_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds));
        raised[dev].store(true, std::memory_order_relaxed);
    }
    return TIDE_OK;
}

// How the rows under a head in four bits are divided.
struct Q4Plan {
    int planes;                // bf16 terms of a row's value
    int64_t T, tiles, blocks;  // blocks: of a part
    int per;                   // groups of a block of 128 columns
    unsigned cus;
    int parts;                 // of the columns; several: a second launch adds them up
    // few rows
    int rows_log, nt, waves, split, lds;
    // many rows: tiles of 16 rows of a row block, row blocks, LDS; waves as above
    int mt;
    int64_t row_blocks;
    bool few;

    int few_lds(int log, int nt_, int waves_, int split_) const {
        return (int)(blocks * 4 * planes * (64 << log)) + waves_ * 1024 + (split_ > 1 ? waves_ * nt_ * 1024 : 0);
    }
    int64_t sets() const { return (tiles + waves * nt - 1) / (waves * nt); }
};
constexpr int kQ4MostParts = 16;
constexpr int64_t kQ4PartBytes = (int64_t)32 << 20;    // of all parts' logits
bool q4_parts_fit(int64_t T, int64_t V, int parts) { return parts == 1 || 4 * T * V * parts <= kQ4PartBytes; }
// The parts of the columns with which few rows fit in LDS (`most` bytes), with `waves` waves' scales; 0: too many.
int q4_few_parts(int dtype, int64_t T, int64_t d, int waves, int most) {
    Q4Plan p{};
    p.planes = dtype == TIDE_F32 ? kQ4Planes<kF32> : 1;
    int log = 0;
    while ((1 << log) < T && log < 4) ++log;
    const int64_t all = (d + kQ4Cols - 1) / kQ4Cols;
    for (int parts = 1; T <= 16 && parts <= std::min<int64_t>(kQ4MostParts, all); ++parts) {
        p.blocks = (all + parts - 1) / parts;
        if (p.few_lds(log, 2, waves, 1) <= most) return parts;
    }
    return 0;
}
bool q4_by_xcd(int64_t sets) { return sets >= 64; }
constexpr int kQ4SmallLds = 32 * 1024;                 // of a workgroup of which several share a CU
constexpr int kQ4ManyTiles[] = {8, 6, 4, 3, 2};        // of 16 rows, of a row block; fp32 rows: 2
Q4Plan q4_plan(int dtype, int64_t T, const Q4Shape& s, unsigned cus) {
    Q4Plan p{};
    p.planes = dtype == TIDE_F32 ? kQ4Planes<kF32> : 1;
    p.T = T, p.tiles = s.tiles(), p.blocks = s.blocks(), p.per = (int)(128 / s.group), p.cus = cus, p.parts = 1;
    while ((1 << p.rows_log) < T && p.rows_log < 4) ++p.rows_log;
    const int64_t all = p.blocks;
    const int fit = q4_few_parts(dtype, T, s.d, 16, kMostLds);
    p.few = fit > 0 && q4_parts_fit(T, s.V, fit);
    if (p.few) {
        // Rows that do not fit whole: in so many parts that several workgroups share a CU, as long as the parts' logits are a small part of the traffic (a sixteenth of the codes).
        if (fit > 1) {
            const int small_parts = q4_few_parts(dtype, T, s.d, 4, kQ4SmallLds);
            p.parts = (int)std::max<int64_t>(fit, std::min<int64_t>(small_parts ? small_parts : kQ4MostParts, s.d / (256 * T)));
            if (!q4_parts_fit(T, s.V, p.parts)) p.parts = fit;
            p.blocks = (all + p.parts - 1) / p.parts, p.parts = (int)((all + p.blocks - 1) / p.blocks);
        }
        // Rows that leave room for several workgroups a CU: small ones, which start and end apart from each other; else one of as many waves as share its CU's tokens
        // evenly, two tiles a wave where there are enough (bf16, d = 4096, V = 128000, us, 4 waves of one tile / 16 of two: T = 1 51 / 51, 8 61 / 52, 16 93 / 55; V = 32000, T = 1 17 / 42).
        const bool small = p.few_lds(p.rows_log, 1, 4, 1) <= kQ4SmallLds;
        const int64_t share = std::max<int64_t>(1, cus / p.parts);
        p.nt = !small && p.tiles >= 24 * share ? 2 : 1;
        p.waves = small ? 4 : (int)std::min<int64_t>(16, std::max<int64_t>(4, (p.tiles + p.nt * share - 1) / (p.nt * share)));
        p.split = 1;
        // few tokens: waves share tiles while there are no more than eight a CU (us, a tile's columns on 1 / 2 / 4 waves; bf16, T = 1, d = 4096: V = 8000 15.7 / 10.1 / 8.3, 16000 16.2 / 12.0 / 11.4,
        // 32003 19.9 / 17.8 / 18.0, 64000 31.5 / 31.2 / 30.6; T = 8, V = 16000 19.0 / 15.3 / 15.9, 64000 38.4 / 40.0 / 44.1; fp32, T = 4, d = 1600, V = 32003 13.2 / 13.0 / 13.6.  At four of 237
        // shapes, of one or two rows, the rule is more than a tenth behind the best of the three: 8192 columns, V = 32003, T = 1 38 / 32 / 31)
        while (p.split < 4 && p.tiles * p.split * p.parts * 2 <= 8 * (int64_t)cus && p.split * 4 <= all - (p.parts - 1) * p.blocks) p.split *= 2;
        if (p.split > 1) p.waves = 4;
        p.lds = p.few_lds(p.rows_log, p.nt, p.waves, p.split);
        return p;
    }
    // Many rows: what a CU's workgroups take, in us, fitted to measured launches of 140 shapes in all their divisions (the choice is 2.1 % off the fastest of them on average and 22 % at most).  What a block
    // of 128 columns takes a workgroup from end to end, in which the CU's other workgroups work, grows with a wave's tiles of rows; what it takes of the CU for 512 tokens, with
    // the workgroup's share of them; so do a workgroup's results at its end.  Parts of the columns cost a launch and their logits' traffic, and fill CUs where there are few tokens.
    // (bf16, us, one part of the largest workgroups / these: d = 8192, V = 1822, T = 43 275 / 33; d = 5120, V = 32401, T = 112 144 / 59; d = 2560, V = 45641, T = 147 86 / 69.)
    double least = 0;
    for (int mt : kQ4ManyTiles) {
        if (p.planes > 1 && mt != 2) continue;
        const int nt = mt == 8 ? 4 : 2, most = 32 / nt, region = 4 * p.planes * mt * 1024;
        const int stages = 2 * region + most * (3 * nt + 2) * 1024 <= kMostLds ? 3 : 2;
        const double rows = mt * p.planes, alone = 0.15 + (0.06 + 0.01 * p.per) * rows * (nt == 4 ? 1.4 : 1.0), all_tokens = 0.4 + (0.03 + 0.012 * p.per) * rows;
        for (int waves : {most, most / 4}) {
            const int64_t row_blocks = (T + 16 * mt - 1) / (16 * mt), sets = (p.tiles + waves * nt - 1) / (waves * nt);
            const int64_t items = (q4_by_xcd(sets) ? (sets + 7) / 8 * 8 : sets) * row_blocks;
            const int64_t together = std::min(most / waves, kMostLds / (2 * region + waves * (stages * nt + 2) * 1024));
            const double share = (double)waves / most;
            for (int parts = 1; parts <= kQ4MostParts && 2 * parts <= std::max<int64_t>(2, all) && q4_parts_fit(T, s.V, parts); parts *= 2) {
                const int64_t blocks = (all + parts - 1) / parts, each = (items * parts + cus - 1) / cus, rounds = (each + together - 1) / together;
                const double work = blocks * (rounds * (alone + 0.02 * p.per * share) + each * all_tokens * share) + 0.5 * each * mt * share + (parts > 1 ? 4.5 + T * s.V * parts * 1e-6 : 0);
                if (least == 0 || work < least) least = work, p.mt = mt, p.nt = nt, p.waves = waves, p.row_blocks = row_blocks, p.parts = parts, p.blocks = blocks;
            }
        }
    }
    p.parts = (int)((all + p.blocks - 1) / p.blocks);
    return p;
}

// The rows' regions.  Row blocks of 16 mt rows for any mt: no matter how many tokens, and more than any call of fewer rows takes.
int64_t q4_lay_bytes(int dtype, int64_t T, int64_t d) {
    const int64_t planes = dtype == TIDE_F32 ? kQ4Planes<kF32> : 1, blocks = (d + kQ4Cols - 1) / kQ4Cols;
    int64_t tiles = 0;
    for (int mt : kQ4ManyTiles)
        if (planes == 1 || mt == 2) tiles = std::max(tiles, (T + 16 * mt - 1) / (16 * mt) * mt);
    return (tiles * blocks * 4 * planes * 1024 + 255) & ~int64_t(255);
}

constexpr int64_t kMostRuleRows = kMostBlocks / 4;     // a workgroup of 1024 threads each, at least
constexpr int64_t kMostPast = (int64_t)1 << 30;
constexpr int64_t kMostBias = kRuleThreads;            // a thread each
constexpr int kRuleOneSlice = 24576;
constexpr int kRuleMostSlice = 32768;                 // 64 KiB of counts: two workgroups a CU with up to 992 biases a row (8 bytes each, two bits a token), one with more

// Slices of a row: as few as leave every CU two workgroups, of whole rounds of the workgroup's threads.  One where it spares the pick its second launch and is not the longer for it (us,
// 44 rows in fp32: 16000 tokens, pasts of 500 14.3 -> 12.1; 24000, pasts of 8000, 300 biases 15.1 -> 14.5; 32000 of these 15.1 -> 16.1).
struct RuleShape {
    int dtype;
    int64_t T, V, H;
    bool pick;
    unsigned cus = 256;
    bool wide() const { return H >= 32768; }           // counts beyond 16 bits
    int slice() const {
        const int64_t round = 16 / (int64_t)elem_bytes(dtype) * kRuleThreads, most = wide() ? kRuleMostSlice / 2 : kRuleMostSlice;
        if (pick && V <= std::min<int64_t>(kRuleOneSlice, most)) return (int)((V + 127) / 128 * 128);
        const int64_t slices = std::max<int64_t>((V + most - 1) / most, std::min<int64_t>((2 * (int64_t)cus + T - 1) / T, (V + round - 1) / round));
        return (int)(((V + slices - 1) / slices + 127) / 128 * 128);
    }
    int64_t slices() const { return (V + slice() - 1) / slice(); }
};

struct RuleCall {
    const void* z;
    int dtype;
    int64_t T, V, row_stride;
    const int32_t* past;
    int64_t H;
    const int32_t *past_len, *prompt_len;
    const float *repetition, *presence, *frequency;
    const int32_t* bias_ids;
    const float* bias_values;
    int64_t B;
    const uint32_t* allowed;
    void* out;                 // rules
    int64_t out_stride;
    int32_t* token;            // pick
    float* log_prob;
    void* workspace;
    size_t workspace_bytes;
    hipStream_t st;
};

int check_rules(const RuleCall& c, bool pick) {
    if (c.dtype != TIDE_F32 && c.dtype != TIDE_F16 && c.dtype != TIDE_BF16) return fail(TIDE_ERR_INVALID_ARG, "dtype %d is not a tide_dtype_t", c.dtype);
    if (c.T < 0) return fail(TIDE_ERR_INVALID_ARG, "T = %lld is negative", (long long)c.T);
    if (c.T > kMostRuleRows) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld exceeds %lld", (long long)c.T, (long long)kMostRuleRows);
    if (c.V <= 0) return fail(TIDE_ERR_INVALID_ARG, "V = %lld must be positive", (long long)c.V);
    if (c.V > kHeadMostVocab) return fail(TIDE_ERR_UNSUPPORTED, "V = %lld exceeds %lld", (long long)c.V, (long long)kHeadMostVocab);
    if (c.H < 0 || c.B < 0) return fail(TIDE_ERR_INVALID_ARG, "H = %lld and B = %lld must not be negative", (long long)c.H, (long long)c.B);
    if (c.H > kMostPast) return fail(TIDE_ERR_UNSUPPORTED, "H = %lld exceeds %lld", (long long)c.H, (long long)kMostPast);
    if (c.B > kMostBias) return fail(TIDE_ERR_UNSUPPORTED, "B = %lld: up to %lld biases of a row", (long long)c.B, (long long)kMostBias);
    if (c.row_stride < c.V) return fail(TIDE_ERR_INVALID_ARG, "row_stride must be at least V");
    if (!pick && c.out_stride < c.V) return fail(TIDE_ERR_INVALID_ARG, "out_row_stride must be at least V");
    if (c.T > 0) {
        if (!c.z) return fail(TIDE_ERR_INVALID_ARG, "logits must not be NULL");
        if (c.H && !c.past) return fail(TIDE_ERR_INVALID_ARG, "past must not be NULL where H is not 0");
        if (c.B && (!c.bias_ids || !c.bias_values)) return fail(TIDE_ERR_INVALID_ARG, "bias_ids and bias_values must not be NULL where B is not 0");
        if (pick ? !c.token || !c.log_prob : !c.out) return fail(TIDE_ERR_INVALID_ARG, pick ? "token and log_prob must not be NULL" : "out must not be NULL");
    }
    const size_t eb = elem_bytes(c.dtype);
    if (((uintptr_t)c.z | (uintptr_t)c.out) % eb) return fail(TIDE_ERR_ALIGNMENT, "logits and out must be aligned to their elements");
    if (((uintptr_t)c.past | (uintptr_t)c.past_len | (uintptr_t)c.prompt_len | (uintptr_t)c.repetition | (uintptr_t)c.presence | (uintptr_t)c.frequency | (uintptr_t)c.bias_ids |
         (uintptr_t)c.bias_values | (uintptr_t)c.allowed | (uintptr_t)c.token | (uintptr_t)c.log_prob) & 3)
        return fail(TIDE_ERR_ALIGNMENT, "4-byte arrays must be aligned to their elements");
    if (!pick && c.T > 0 && (c.out != c.z || (c.T > 1 && c.out_stride != c.row_stride))) {
        // rows that overlap others than themselves would be read after they are written
        const int64_t width = c.V * (int64_t)eb, in = c.row_stride * (int64_t)eb, to = c.out_stride * (int64_t)eb;
        const int64_t a = (int64_t)(uintptr_t)c.z, b = (int64_t)(uintptr_t)c.out;
        bool apart = a + (c.T - 1) * in + width <= b || b + (c.T - 1) * to + width <= a;
        if (!apart && in == to && c.T > 1) {           // columns of the same rows
            const int64_t off = ((b - a) % in + in) % in;
            apart = off >= width && in - off >= width;
        }
        if (!apart) return fail(TIDE_ERR_INVALID_ARG, "out must be the logits themselves or not overlap them");
    }
    return TIDE_OK;
}

int run_rules(const RuleCall& c, bool pick) {
    int rc = check_rules(c, pick);
    if (rc || c.T == 0) return rc;
    RuleShape s{c.dtype, c.T, c.V, c.H, pick};
    if ((rc = resident_cus(&s.cus))) return rc;
    const int64_t slices = s.slices(), blocks = c.T * slices;
    if (blocks > kMostRuleRows) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld rows of V = %lld logits are too many for one call", (long long)c.T, (long long)c.V);
    if (pick && slices > 1) {
        const size_t need = (size_t)blocks * sizeof(uint4);
        if (!c.workspace || c.workspace_bytes < need) return fail(TIDE_ERR_WORKSPACE, "this call needs %zu bytes of workspace, %zu given", need, c.workspace ? c.workspace_bytes : 0);
        if ((uintptr_t)c.workspace & 15) return fail(TIDE_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
    }
    RuleParams p{};
    const int64_t eb = (int64_t)elem_bytes(c.dtype);
    p.z = (const char*)c.z;
    p.out = (char*)c.out;
    p.row_bytes = c.row_stride * eb;
    p.out_row_bytes = c.out_stride * eb;
    p.T = (int)c.T;
    p.V = (int)c.V;
    p.H = (int)c.H;
    p.B = (int)c.B;
    p.slice = s.slice();
    p.slices = (int)slices;
    p.past = c.past, p.past_len = c.past_len, p.prompt_len = c.prompt_len;
    p.repetition = c.repetition, p.presence = c.presence, p.frequency = c.frequency;
    p.bias_ids = c.bias_ids, p.bias_values = c.bias_values;
    p.allowed = c.allowed;
    p.words = (int)((c.V + 31) / 32);
    p.token = c.token, p.log_prob = c.log_prob;
    p.part = (uint4*)c.workspace;
    const int lds = rule_tables(p.slice, p.H ? (s.wide() ? 4 : 2) : 0, p.B).bytes;
    rc = by_dtype(c.dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto picks, auto wide) -> int {
            constexpr bool kPick = decltype(picks)::value, kWide = decltype(wide)::value;
            const int rc2 = raise_lds<&tide_logit_rules_kernel<DT, kPick, kWide>>();
            if (rc2) return rc2;
            hipLaunchKernelGGL((tide_logit_rules_kernel<DT, kPick, kWide>), dim3((unsigned)blocks), dim3(kRuleThreads), lds, c.st, p);
            return TIDE_OK;
        };
        if (s.wide()) return pick ? go(std::true_type{}, std::true_type{}) : go(std::false_type{}, std::true_type{});
        return pick ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{});
    });
    if (rc) return rc;
    if (pick && slices > 1) hipLaunchKernelGGL(tide_logit_join_kernel, dim3((unsigned)((c.T + 3) / 4)), dim3(kRuleJoinThreads), 0, c.st, p.part, p.T, p.slices, c.token, c.log_prob);
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

}  // namespace

extern "C" {

int tide_head_quantize_q4(const void* W, int dtype, int64_t V, int64_t d, int64_t w_row_stride, int64_t group, void* codes, void* scales, int scale_dtype, void* stream) {
    g_err[0] = 0;
    if (!W) return fail(TIDE_ERR_INVALID_ARG, "W must not be NULL");
    return q4_weights(W, nullptr, dtype, Q4Shape{V, d, group, scale_dtype}, w_row_stride, codes, scales, (hipStream_t)stream);
}

int tide_head_dequantize_q4(const void* codes, const void* scales, int scale_dtype, int64_t V, int64_t d, int64_t group, void* W, int dtype, int64_t w_row_stride, void* stream) {
    g_err[0] = 0;
    return q4_weights(nullptr, W, dtype, Q4Shape{V, d, group, scale_dtype}, w_row_stride, codes, scales, (hipStream_t)stream);
}

size_t tide_head_logits_q4_bytes(int dtype, int64_t T, int64_t d, int64_t V) {
    g_err[0] = 0;
    if ((dtype != TIDE_F32 && dtype != TIDE_F16 && dtype != TIDE_BF16) || T < 0 || T > kHeadMostRows || d <= 0 || d > kMaxHidden || V <= 0 || V > kHeadMostVocab) {
        fail(TIDE_ERR_UNSUPPORTED, "unsupported dtype %d, T = %lld, d = %lld or V = %lld", dtype, (long long)T, (long long)d, (long long)V);
        return 0;
    }
    if (q4_few_parts(dtype, T, d, 16, kMostLds) == 1) return 0;
    return (size_t)(q4_lay_bytes(dtype, T, d) + std::min(kQ4PartBytes, 4 * T * V * kQ4MostParts));
}

int tide_head_logits_q4(const void* x, int dtype, int64_t T, int64_t d, int64_t V, int64_t x_row_stride, const void* codes, const void* scales, int scale_dtype, int64_t group,
                        float* logits, int64_t logits_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    const Q4Shape s{V, d, group, scale_dtype};
    int rc = check_q4(s, dtype, codes, scales);
    if (rc) return rc;
    if (T < 0) return fail(TIDE_ERR_INVALID_ARG, "T = %lld is negative", (long long)T);
    if (T > kHeadMostRows) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld exceeds %lld", (long long)T, (long long)kHeadMostRows);
    if (T == 0) return TIDE_OK;
    if ((rc = check_q4_rows(x, x_row_stride, d, dtype, "x"))) return rc;
    if (!logits) return fail(TIDE_ERR_INVALID_ARG, "logits must not be NULL");
    if (logits_row_stride < V) return fail(TIDE_ERR_INVALID_ARG, "logits_row_stride must be at least V");
    if ((uintptr_t)logits & 3) return fail(TIDE_ERR_ALIGNMENT, "logits must be aligned to a float");
    if ((T + 15) / 16 * s.tiles() > 4 * kMostBlocks) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld rows of V = %lld logits are too many for one call", (long long)T, (long long)V);
    const size_t need = tide_head_logits_q4_bytes(dtype, T, d, V);
    if (need && (!workspace || workspace_bytes < need))
        return fail(TIDE_ERR_WORKSPACE, "this call needs %zu bytes of workspace, %zu given", need, workspace ? workspace_bytes : 0);
    if (need && ((uintptr_t)workspace & 255)) return fail(TIDE_ERR_ALIGNMENT, "the workspace must be 256-byte aligned");
    unsigned cus = 0;
    if ((rc = resident_cus(&cus))) return rc;
    const Q4Plan plan = q4_plan(dtype, T, s, cus);
    hipStream_t st = (hipStream_t)stream;
    const Q4Rows rows{(const char*)x, x_row_stride * (int64_t)elem_bytes(dtype), (int)T, (int)d, q4_chunks(x, x_row_stride, dtype)};
    float* const sums = plan.parts > 1 ? (float*)((char*)workspace + q4_lay_bytes(dtype, T, d)) : logits;
    const int64_t sums_stride = plan.parts > 1 ? V : logits_row_stride, part_stride = plan.parts > 1 ? T * V : 0;
    const Q4Head head{(const char*)codes, (const uint16_t*)scales, (int)V, (int)s.tiles(), (int)s.blocks(), (int)s.groups(), scale_dtype == TIDE_F16};
    using std::integral_constant;
    rc = by_dtype(dtype, [&](auto dt) -> int {
        return by_runs(group, [&](auto runs) -> int {
            constexpr int DT = decltype(dt)::value, kRuns = decltype(runs)::value;
            auto few = [&](auto tiles) -> int {
                constexpr int NT = decltype(tiles)::value, kDepth = NT == 1 ? 4 : 2;
                int rc2 = raise_lds<&tide_head_q4_few_kernel<DT, kRuns, NT, kDepth>>();
                if (rc2) return rc2;
                const int per_set = plan.waves / plan.split * NT, sets = (int)((plan.tiles + per_set - 1) / per_set);
                // (as many as LDS and registers have room for)
                const int together = std::max(1, std::min(kMostLds / plan.lds, plan.waves > 4 ? 1 : dtype == TIDE_F32 ? 5 : 7));
                const Q4FewParams p{rows, head, sums, sums_stride, part_stride, (int)plan.blocks, sets, plan.rows_log, plan.split};
                const int64_t grid = std::min<int64_t>(sets, std::max<int64_t>(1, (int64_t)cus * together / plan.parts));
                hipLaunchKernelGGL((tide_head_q4_few_kernel<DT, kRuns, NT, kDepth>), dim3((unsigned)grid, (unsigned)plan.parts), dim3(plan.waves * kWave), plan.lds, st, p);
                return TIDE_OK;
            };
            auto many = [&](auto row_tiles) -> int {
                constexpr int MT = decltype(row_tiles)::value, NT = MT == 8 ? 4 : 2;
                int rc2 = raise_lds<&tide_head_q4_many_kernel<DT, kRuns, MT, NT>>();
                if (rc2) return rc2;
                const Q4LayParams lay{rows, (char*)workspace, head.blocks, plan.row_blocks * MT * head.blocks};
                hipLaunchKernelGGL((tide_head_q4_lay_kernel<DT, kRuns, MT>), dim3((unsigned)((lay.waves + 3) / 4)), dim3(kQ4Threads), 0, st, lay);
                const int64_t sets = plan.sets();
                const bool by_xcd = q4_by_xcd(sets);
                const Q4ManyParams p{(const char*)workspace, head, sums, sums_stride, part_stride, (int)plan.blocks, (int)T, (int)plan.row_blocks, (int)sets, by_xcd};
                const int lds = q4_many_lds<NT>(kQ4Region<DT, MT>, kQ4CodeStages<DT, MT, NT>, plan.waves);
                const int64_t together = std::min<int64_t>(kMostLds / lds, kQ4ManyThreads<NT> / kWave / plan.waves);
                const int64_t items = by_xcd ? (sets + 7) / 8 * 8 * plan.row_blocks : (sets * plan.row_blocks + 7) / 8 * 8;      // (an XCD that has a set more than others has room for it)
                const int64_t grid = std::min(items, std::max<int64_t>(8, cus * together / plan.parts / 8 * 8));
                hipLaunchKernelGGL((tide_head_q4_many_kernel<DT, kRuns, MT, NT>), dim3((unsigned)grid, (unsigned)plan.parts), dim3(plan.waves * kWave), lds, st, p);
                return TIDE_OK;
            };
            if (plan.few) return plan.nt == 2 ? few(integral_constant<int, 2>{}) : few(integral_constant<int, 1>{});
            if constexpr (DT != kF32) {
                if (plan.mt == 8) return many(integral_constant<int, 8>{});
                if (plan.mt == 6) return many(integral_constant<int, 6>{});
                if (plan.mt == 4) return many(integral_constant<int, 4>{});
                if (plan.mt == 3) return many(integral_constant<int, 3>{});
            }
            return many(integral_constant<int, 2>{});
        });
    });
    if (rc) return rc;
    if (plan.parts > 1) {
        const Q4JoinParams p{sums, logits, logits_row_stride, (int)T, (int)V, plan.parts, (int)((V + kQ4JoinRun * kQ4Threads - 1) / (kQ4JoinRun * kQ4Threads))};
        hipLaunchKernelGGL(tide_head_q4_join_kernel, dim3((unsigned)(T * p.pieces)), dim3(kQ4Threads), 0, st, p);
    }
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

int tide_logit_rules(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const int32_t* past, int64_t H, const int32_t* past_len, const int32_t* prompt_len,
                     const float* repetition, const float* presence, const float* frequency, const int32_t* bias_ids, const float* bias_values, int64_t B, const uint32_t* allowed,
                     void* out, int64_t out_row_stride, void* stream) {
    g_err[0] = 0;
    RuleCall c{};
    c.z = logits, c.dtype = dtype, c.T = T, c.V = V, c.row_stride = row_stride;
    c.past = past, c.H = H, c.past_len = past_len, c.prompt_len = prompt_len;
    c.repetition = repetition, c.presence = presence, c.frequency = frequency;
    c.bias_ids = bias_ids, c.bias_values = bias_values, c.B = B, c.allowed = allowed;
    c.out = out, c.out_stride = out_row_stride, c.st = (hipStream_t)stream;
    return run_rules(c, false);
}

size_t tide_logit_pick_bytes(int64_t T, int64_t V) {
    g_err[0] = 0;
    if (T < 0 || T > kMostRuleRows || V < 1 || V > kHeadMostVocab) {
        fail(TIDE_ERR_UNSUPPORTED, "unsupported T = %lld or V = %lld", (long long)T, (long long)V);
        return 0;
    }
    if (V <= kRuleMostSlice / 2) return 0;             // one slice, however long the past
    return (size_t)std::max<int64_t>(T, 1) * ((V + 1023) / 1024) * sizeof(uint4);
}

int tide_logit_pick(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const int32_t* past, int64_t H, const int32_t* past_len, const int32_t* prompt_len,
                    const float* repetition, const float* presence, const float* frequency, const int32_t* bias_ids, const float* bias_values, int64_t B, const uint32_t* allowed,
                    int32_t* token, float* log_prob, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    RuleCall c{};
    c.z = logits, c.dtype = dtype, c.T = T, c.V = V, c.row_stride = row_stride;
    c.past = past, c.H = H, c.past_len = past_len, c.prompt_len = prompt_len;
    c.repetition = repetition, c.presence = presence, c.frequency = frequency;
    c.bias_ids = bias_ids, c.bias_values = bias_values, c.B = B, c.allowed = allowed;
    c.token = token, c.log_prob = log_prob;
    c.workspace = workspace, c.workspace_bytes = workspace_bytes, c.st = (hipStream_t)stream;
    return run_rules(c, true);
}

}  // extern "C"
