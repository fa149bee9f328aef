// Host side of the answer operators (include/tide_route.h): the LM head in four bits and the rules of decoding.  Argument checks, the division of the work and the launches.
// Included by tide_route.hip behind head_route.hpp, whose limits of T and V it shares.
#pragma once

namespace {

constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1;      // a launch has fewer than 2^32 threads, a workgroup 256

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
    p.W = (const char*)W;
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

size_t q4_rows_bytes(int dtype, int64_t T, const Q4Shape& s) {
    return (size_t)((T + 15) / 16) * s.blocks() * 4 * kQ4TileBytes * (dtype == TIDE_F32 ? kQ4Planes<kF32> : 1);
}

constexpr int64_t kMostPast = (int64_t)1 << 30;
constexpr int64_t kMostBias = 1024;                    // entries of one token are joined by a search through them
constexpr int kRuleMostSlice = 8192;

// Slices of a row: as few as leave every CU four workgroups.
struct RuleShape {
    int64_t T, V;
    unsigned cus = 256;
    int slice() const {
        const int64_t want = (T * V + 4 * (int64_t)cus - 1) / (4 * (int64_t)cus);
        return (int)std::min<int64_t>(kRuleMostSlice, std::max<int64_t>(1024, (want + 1023) / 1024 * 1024));
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
    if (c.T > kHeadMostRows) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld exceeds %lld", (long long)c.T, (long long)kHeadMostRows);
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
    RuleShape s{c.T, c.V};
    if ((rc = resident_cus(&s.cus))) return rc;
    const int64_t slices = s.slices(), blocks = c.T * slices;
    if (blocks > kMostBlocks) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld rows of V = %lld logits are too many for one call", (long long)c.T, (long long)c.V);
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
    RuleTables none;
    const int lds = rule_tables(nullptr, p.slice, p.H != 0, p.B != 0, &none);
    rc = by_dtype(c.dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto kernel) -> int {
            if (lds > 48 * 1024) TIDE_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
            hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRuleThreads), lds, c.st, p);
            return TIDE_OK;
        };
        return pick ? go(&tide_logit_rules_kernel<DT, true>) : go(&tide_logit_rules_kernel<DT, false>);
    });
    if (rc) return rc;
    if (pick && slices > 1) hipLaunchKernelGGL(tide_logit_join_kernel, dim3((unsigned)((c.T + 3) / 4)), dim3(kRuleThreads), 0, c.st, p.part, p.T, p.slices, c.token, c.log_prob);
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

size_t tide_head_logits_q4_bytes(int dtype, int64_t T, int64_t d) {
    g_err[0] = 0;
    if ((dtype != TIDE_F32 && dtype != TIDE_F16 && dtype != TIDE_BF16) || T < 0 || T > kHeadMostRows || d < 1 || d > kMaxHidden) {
        fail(TIDE_ERR_UNSUPPORTED, "unsupported dtype %d, T = %lld or d = %lld", dtype, (long long)T, (long long)d);
        return 0;
    }
    return std::max<size_t>(256, q4_rows_bytes(dtype, T, Q4Shape{1, d, 128, TIDE_BF16}));
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
    const int64_t row_tiles = (T + 15) / 16, waves = row_tiles * s.tiles(), blocks = (waves + 3) / 4;
    if (blocks > kMostBlocks) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld rows of V = %lld logits are too many for one call", (long long)T, (long long)V);
    const size_t need = q4_rows_bytes(dtype, T, s);
    if (!workspace || workspace_bytes < need) return fail(TIDE_ERR_WORKSPACE, "this call needs %zu bytes of workspace, %zu given", need, workspace ? workspace_bytes : 0);
    if ((uintptr_t)workspace & 255) return fail(TIDE_ERR_ALIGNMENT, "the workspace must be 256-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    Q4RowParams r{};
    r.x = (const char*)x;
    r.row_bytes = x_row_stride * (int64_t)elem_bytes(dtype);
    r.out = (char*)workspace;
    r.T = (int)T;
    r.d = (int)d;
    r.steps = (int)s.blocks() * 4;
    r.chunks = q4_chunks(x, x_row_stride, dtype);
    r.fragments = row_tiles * r.steps;
    Q4LogitParams p{};
    p.rows = (const char*)workspace;
    p.codes = (const char*)codes;
    p.scales = (const uint16_t*)scales;
    p.out = logits;
    p.out_stride = logits_row_stride;
    p.T = (int)T;
    p.V = (int)V;
    p.blocks = (int)s.blocks();
    p.groups = (int)s.groups();
    p.row_tiles = (int)row_tiles;
    p.half = scale_dtype == TIDE_F16;
    p.waves = waves;
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        hipLaunchKernelGGL((tide_head_q4_rows_kernel<DT>), dim3((unsigned)((r.fragments + 3) / 4)), dim3(kQ4Threads), 0, st, r);
        return by_runs(group, [&](auto runs) {
            hipLaunchKernelGGL((tide_head_q4_kernel<DT, decltype(runs)::value>), dim3((unsigned)blocks), dim3(kQ4Threads), 0, st, p);
            return 0;
        });
    });
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
    if (T < 0 || T > kHeadMostRows || V < 1 || V > kHeadMostVocab) {
        fail(TIDE_ERR_UNSUPPORTED, "unsupported T = %lld or V = %lld", (long long)T, (long long)V);
        return 0;
    }
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
