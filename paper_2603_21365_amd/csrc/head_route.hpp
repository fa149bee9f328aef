// Host side of the head operators (include/tide_route.h): argument checks, the division of the work, the workspace's layout and the launches.
// Included by tide_route.hip, whose error reporting and device queries it uses.
#pragma once

namespace {

// The tile that the rows of a call take.  Few rows: the products with x W^T are bound by reading W, so their tiles are 128 columns wide and leave half of a
// CU's LDS, so that two workgroups are there and one's first and last stages overlap with the other's (bf16, T = 33, d = 8192,
// V = 20000: 110 us as 79 tiles of 256 columns, 83 as 157 of 128).  dx reads W across and stays 256 wide.
using HeadTile32 = HeadTile<1, 8, 2, 1, 4, 4>;
using HeadTile64 = HeadTile<2, 4, 2, 2, 3, 3>;
using HeadTile16F = HeadTile<1, 8, 1, 1, 4, 4, 4>;      // fp32 rows as they are
using HeadTile32F = HeadTile<1, 8, 2, 1, 4, 4, 4>;
using HeadTile48F = HeadTile<1, 8, 3, 1, 3, 3, 4>;
using HeadTile64F = HeadTile<2, 4, 2, 2, 3, 3, 4>;
using HeadTile128 = HeadTile<2, 4, 4, 4, 4, 3>;
using HeadTile192 = HeadTile<4, 2, 3, 8, 3, 2>;
using HeadTile256 = HeadTile<4, 2, 4, 8, 3, 2>;
using HeadRows32 = HeadTile<1, 8, 2, 2, 4, 4>;
using HeadRows64 = HeadTile<2, 4, 2, 4, 4, 4>;
// fp32 rows as they are up to here, planes beyond (V = 100000, d = 4096, us: T = 65 806 / 1429, 96 809 / 1436, 128 1024 / 1445; 192 would be three tiles of 64).
constexpr int kHeadDirectRows = 128;
constexpr int kHeadCols = 256;
constexpr int64_t kHeadMostRows = (int64_t)1 << 22, kHeadMostVocab = (int64_t)1 << 23;
constexpr int64_t kHeadMostTiles = ((int64_t)1 << 23) - 8;      // a launch has fewer than 2^32 threads, a tile 512
constexpr int kHeadMostTop = 1024;
constexpr size_t kHeadPieceBytes = (size_t)256 << 20;      // G of a piece of the vocabulary: as much as stays in the last-level cache (256 MiB to 4 GiB: no difference)

template <typename F> int by_head_tile(int rows, F&& f) {
    switch (rows) {
    case 32: return f(HeadTile32{});
    case 64: return f(HeadTile64{});
    case 128: return f(HeadTile128{});
    case 192: return f(HeadTile192{});
    default: return f(HeadTile256{});
    }
}
template <typename F> int by_head_rows(int rows, F&& f) {
    switch (rows) {
    case 32: return f(HeadRows32{});
    case 64: return f(HeadRows64{});
    case 128: return f(HeadTile128{});
    case 192: return f(HeadTile192{});
    default: return f(HeadTile256{});
    }
}

struct HeadShape {
    int dtype;
    int64_t T, d, V, K;
    bool wide = false;             // G in two planes whatever T
    unsigned cus = 256;
    int64_t dp() const { return (d + 7) / 8 * 8; }                      // elements of a padded row of 16-bit values
    int planes() const { return dtype == TIDE_F32 ? 2 : 1; }
    bool copied(bool grads) const { return direct(grads) ? false : dtype == TIDE_F32 || d % 8 != 0; }     // the products read copies of x and W
    int64_t plane_bytes(int64_t rows) const { return rows * dp() * 2; }
    static int rows_for(int64_t T) {
        if (T <= 32) return 32;
        if (T <= 64) return 64;
        // A tile of 128 / 192 rows takes 60 / 80 % of the time of one of 256 (d = 4096, V = 65536, us a tile row: 66-108); the least of those decides
        int best = 256;
        int64_t least = (T + 255) / 256 * 100;
        if ((T + 191) / 192 * 80 < least) best = 192, least = (T + 191) / 192 * 80;
        if ((T + 127) / 128 * 60 < least) best = 128;
        return best;
    }
    // The products with x W^T: the same, but tiles of 64 rows and 128 columns where the large ones fill less than half of the CUs and these fit one round of two a
    // CU (with the slices of dW, a step in bf16 at T = 2142, d = 768, V = 1147 141 -> 102 us; fp16, T = 8000, d = 1024, V = 1000 302 -> 181).
    int rows_per_tile() const {
        const int rows = rows_for(T);
        if (rows <= 64) return rows;
        return 2 * ((T + rows - 1) / rows) * col_tiles() < (int64_t)cus && (T + 63) / 64 * ((V + HeadTile64::kP - 1) / HeadTile64::kP) <= 2 * (int64_t)cus ? 64 : rows;
    }
    int64_t row_tiles() const { return (T + rows_per_tile() - 1) / rows_per_tile(); }
    // G in the type of the rows, as a program has it that keeps its logits in that type.  What its rounding leaves goes into a second plane where the caller asks for it,
    // and up to 64 rows: there a row of dx can hang on one element of G, and the products are bound by reading W and writing dW (the gradient call with one / two
    // planes, bf16, d = 4096, V = 128000, ms: T = 1 0.66 / 0.66, 33 0.69 / 0.75, 64 0.70 / 0.79, 128 0.78 / 0.96, 322 1.29 / 1.82, 8192 20.6 / 35.4).
    int g_planes() const { return dtype == TIDE_F32 || T <= 64 || wide ? 2 : 1; }
    // 16-bit operands: the second plane follows as further rows -- of dx, so that W is read once, and of k in dW (of x, too)
    int64_t stacked() const { return dtype != TIDE_F32 && g_planes() == 2 ? T : 0; }
    int rows_of_dx() const { return rows_for(T + stacked()); }
    int64_t col_tiles() const { return (V + kHeadCols - 1) / kHeadCols; }
    // Rows and columns of a tile of the statistics.  Few rows: as many tiles as the narrowest multiple of the CUs that holds them, so that each CU reads as much of W
    // (bf16, d = 4096, V = 128000: 1000 tiles of 128 columns 186 us / 1024 of 125 180).
    int stats_rows() const { return direct(false) ? std::min(rows_for(T), 64) : rows_per_tile(); }
    int pitch() const {
        const int rows = stats_rows();
        if (rows > 64) return kHeadCols;
        if (T > 64) return HeadTile64::kP;
        const int64_t tiles = ((V + HeadTile32::kP - 1) / HeadTile32::kP + cus - 1) / cus * cus;
        return (int)((V + tiles - 1) / tiles);
    }
    int64_t parts() const { return (V + pitch() - 1) / pitch() * (stats_rows() <= 64 ? 1 : stats_rows() == 128 ? HeadTile128::kParts : HeadTile256::kParts); }
    static_assert(HeadTile192::kParts == HeadTile256::kParts, "");
    static_assert(HeadTile32::kP == HeadTile64::kP && HeadTile32::kP == HeadTile32F::kP && HeadTile32::kP == HeadTile16F::kP && HeadTile32::kP == HeadTile48F::kP && HeadTile32::kP == HeadTile64F::kP && HeadTile32::kParts == 1 && HeadTile64::kParts == 1, "");
    // fp32 rows without planes: the forward call on few rows, which is bound by reading W once
    bool direct(bool grads) const { return dtype == TIDE_F32 && !grads && T <= kHeadDirectRows && d % 4 == 0; }
    // columns of a piece of the vocabulary in the gradient: equal pieces whose G is at most kHeadPieceBytes
    int64_t piece() const {
        const int64_t tiles = std::max<int64_t>(1, (int64_t)(kHeadPieceBytes / ((size_t)std::max<int64_t>(T, 1) * g_planes() * 2 * kHeadCols)));
        const int64_t pieces = (col_tiles() + tiles - 1) / tiles;
        return (col_tiles() + pieces - 1) / pieces * kHeadCols;
    }
    // workgroups that share a tile's piece of the vocabulary in dx = G W: what fills the chip once
    int dx_slices() const {
        const int64_t tiles = (T + stacked() + rows_of_dx() - 1) / rows_of_dx() * ((d + kHeadCols - 1) / kHeadCols);
        return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(cus / std::max<int64_t>(tiles, 1), 64), piece() / kHeadCols));
    }
    // the same for dW = G^T x, over the rows: at least four stages each (few tiles: a vocabulary of a few thousand tokens)
    int dw_slices() const {
        const int64_t tiles = piece() / kHeadCols * ((d + kHeadCols - 1) / kHeadCols);
        return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(cus / tiles, 32), (T + 255) / 256));
    }
    // What a workspace has room for: bounds of the sizes above that grow with T, so that a workspace for the most rows of a program serves every smaller call
    // (tiles, pieces and slices change with T, and what they take goes up and down).
    int64_t part_room() const {                        // parts() * T
        const int64_t few = ((V + HeadTile32::kP - 1) / HeadTile32::kP + cus - 1) / cus * cus, many = (V + HeadTile64::kP - 1) / HeadTile64::kP + 1;
        return T <= 64 ? few * T : std::max(few * 64, many * T);
    }
    int64_t g_room() const {                           // bytes of T * g_planes() * piece() elements
        const int64_t rows = std::max<int64_t>(T * g_planes(), T > 64 ? 128 : 0);
        return std::min(rows * col_tiles() * kHeadCols * 2, std::max((int64_t)kHeadPieceBytes, T * g_planes() * kHeadCols * 2));
    }
    int64_t dx_room() const {                          // rows of dx_slices() * (T + stacked())
        const int64_t rows = std::max<int64_t>(T + stacked(), T > 64 ? 128 : 0), tiles = (d + kHeadCols - 1) / kHeadCols;
        return std::max(rows, std::min(std::min<int64_t>(64, col_tiles()) * rows, cus * kHeadCols / tiles));      // (as many slices as fill the chip once)
    }
    int64_t dw_room() const {                          // rows of dw_slices() * piece(), where any number of rows up to T takes slices
        const int64_t tiles = (d + kHeadCols - 1) / kHeadCols, most = std::max<int64_t>(1, (int64_t)kHeadPieceBytes / (std::max<int64_t>(T, 1) * g_planes() * 2 * kHeadCols));
        const int64_t least = (std::min(col_tiles(), most) + 1) / 2;      // tiles of a piece: equal pieces are more than half of the largest
        if (T <= 256 || 2 * least * tiles > (int64_t)cus) return 0;
        return std::min(std::min<int64_t>(32, (T + 255) / 256) * col_tiles() * kHeadCols, cus * kHeadCols / tiles);
    }
};

// The workspace of a call: counted with a null base, laid out with the caller's.
struct HeadSpace {
    char* base;
    size_t at = 0;
    template <typename T> T* take(size_t n) {
        T* p = base ? reinterpret_cast<T*>(base + at) : nullptr;
        at += (n * sizeof(T) + 255) & ~size_t(255);
        return p;
    }
};
struct HeadWork {
    HeadCtl* ctl;
    uint32_t* w_max;
    int32_t *x_exp, *largest;  // fp32 planes: the rows' powers of two, and what the workgroups found for dW's
    char *x, *w;               // copies: the rows (of the gradient: the live ones), the weights
    char* x_dw;                // the rows as dW's sum takes them
    float2* part;
    float* z;
    int32_t *source, *place;
    float4* row_const;
    float* wanted;
    uint8_t* taught;
    char* g;
    float *acc, *dw;
};
size_t head_layout(const HeadShape& s, bool grads, void* base, HeadWork* out) {
    HeadSpace sp{(char*)base};
    HeadWork w{};
    w.ctl = sp.take<HeadCtl>(1);
    if (s.dtype == TIDE_F32 && !s.direct(grads)) {
        w.w_max = sp.take<uint32_t>(kHeadMaxBlocks);
        w.x_exp = sp.take<int32_t>((size_t)s.T);
        if (grads) w.largest = sp.take<int32_t>(kHeadMaxBlocks);
    }
    if (s.copied(grads)) w.w = sp.take<char>((size_t)s.plane_bytes(s.V) * s.planes());
    if (s.copied(grads) || grads) w.x = sp.take<char>((size_t)s.plane_bytes(std::max(s.T + (grads ? s.stacked() : 0), grads && s.T > 64 ? (int64_t)128 : 0)) * s.planes());
    w.x_dw = s.dtype == TIDE_F32 && grads ? sp.take<char>((size_t)s.plane_bytes(s.T) * 2) : w.x;
    if (!grads) {
        w.part = sp.take<float2>((size_t)s.part_room());
        if (!s.K) w.z = sp.take<float>((size_t)s.T);
    } else {
        w.source = sp.take<int32_t>((size_t)s.T);
        w.place = sp.take<int32_t>((size_t)s.T);
        w.row_const = sp.take<float4>((size_t)s.T);
        if (s.K) {
            w.wanted = sp.take<float>((size_t)s.T * s.K);
            w.taught = sp.take<uint8_t>((size_t)s.T);
        }
        w.g = sp.take<char>((size_t)s.g_room());
        w.acc = sp.take<float>((size_t)s.dx_room() * s.dp());
        w.dw = sp.take<float>((size_t)s.dw_room() * s.dp());
    }
    if (out) *out = w;
    return sp.at;
}

template <int DT, int OutDT, int kMode, class Tile> int launch_head(int64_t q_rows, int64_t p_rows, hipStream_t st, HeadGemmParams& p) {
    static std::atomic<bool> raised[kMaxDevices];
    int dev = 0;
    int rc = current_device(&dev);
    if (rc) return rc;
    if (!raised[dev].load(std::memory_order_relaxed)) {
        TIDE_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&tide_head_gemm_kernel<DT, OutDT, kMode, Tile>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     Tile::kLdsBytes));
        raised[dev].store(true, std::memory_order_relaxed);
    }
    if (!p.pitch) p.pitch = Tile::kP;
    const int64_t tq = (q_rows + Tile::kQ - 1) / Tile::kQ;
    p.tiles_p = (int)((p_rows + p.pitch - 1) / p.pitch);
    if (tq * p.tiles_p == 0) return TIDE_OK;
    unsigned cus = 0;
    if ((rc = resident_cus(&cus))) return rc;
    int64_t grid = (tq * p.tiles_p * p.k_slices + 7) / 8 * 8;
    if (kLoops<kMode, Tile>) grid = std::min<int64_t>(grid, cus);
    hipLaunchKernelGGL((tide_head_gemm_kernel<DT, OutDT, kMode, Tile>), dim3((unsigned)grid), dim3(Tile::kThreads), Tile::kLdsBytes, st, p);
    return TIDE_OK;
}
// The products of fp32 operands run on fp16 planes.
template <int DT> constexpr int kHeadElem = DT == kF32 ? (int)kF16 : DT;

struct HeadCall {
    HeadShape s;
    const void *x, *W;
    int64_t x_stride, w_stride;
    const int32_t* ids;        // targets, or the teacher's tokens
    const float* values;       // teacher's values, or null
    float tau;
    float *loss, *lse, *z;     // forward
    const float *lse_in, *grad;
    void *dx, *dW;
    int64_t dx_stride, dw_stride;
    void* workspace;
    size_t workspace_bytes;
    hipStream_t st;
};

int check_head(const HeadCall& c, bool grads) {
    const HeadShape& s = c.s;
    if (s.dtype != TIDE_F32 && s.dtype != TIDE_F16 && s.dtype != TIDE_BF16) return fail(TIDE_ERR_INVALID_ARG, "dtype %d is not a tide_dtype_t", s.dtype);
    if (s.T < 0) return fail(TIDE_ERR_INVALID_ARG, "T = %lld is negative", (long long)s.T);
    if (s.T > kHeadMostRows) return fail(TIDE_ERR_UNSUPPORTED, "T = %lld exceeds %lld", (long long)s.T, (long long)kHeadMostRows);
    if (s.d <= 0) return fail(TIDE_ERR_INVALID_ARG, "d = %lld must be positive", (long long)s.d);
    if (s.d > kMaxHidden) return fail(TIDE_ERR_UNSUPPORTED, "d = %lld: hidden sizes from 1 to 16384", (long long)s.d);
    if (s.V <= 0) return fail(TIDE_ERR_INVALID_ARG, "V = %lld must be positive", (long long)s.V);
    if (s.V > kHeadMostVocab) return fail(TIDE_ERR_UNSUPPORTED, "V = %lld exceeds %lld", (long long)s.V, (long long)kHeadMostVocab);
    if (s.row_tiles() * ((s.V + HeadTile32::kP - 1) / HeadTile32::kP) > kHeadMostTiles)
        return fail(TIDE_ERR_UNSUPPORTED, "T = %lld rows of V = %lld logits are too many for one call", (long long)s.T, (long long)s.V);
    if (s.K < 0 || s.K > kHeadMostTop) return fail(TIDE_ERR_UNSUPPORTED, "K = %lld: 1 to %d entries of a teacher", (long long)s.K, kHeadMostTop);
    if (!(c.tau > 0.0f) || !(c.tau <= 1e30f) || c.tau < 1e-30f) return fail(TIDE_ERR_INVALID_ARG, "tau = %g must be positive and finite", (double)c.tau);
    if (c.x_stride < s.d || c.w_stride < s.d) return fail(TIDE_ERR_INVALID_ARG, "row strides of x and W must be at least d");
    const int64_t most = (int64_t)1 << 22;             // elements: 256 rows of a tile at 32-bit offsets
    if (c.x_stride > most || c.w_stride > most) return fail(TIDE_ERR_UNSUPPORTED, "row strides of x and W must be at most %lld", (long long)most);
    const size_t eb = elem_bytes(s.dtype);
    auto check_rows = [&](const void* p, int64_t stride, const char* name) {
        const size_t unit = chunked_rows(s.dtype, s.d) ? 16 : eb;
        if (((uintptr_t)p % unit) || ((size_t)stride * eb % unit)) return fail(TIDE_ERR_ALIGNMENT, "%s: base and row stride must be multiples of %zu bytes", name, unit);
        return (int)TIDE_OK;
    };
    if (!c.W || (s.T > 0 && (!c.x || !c.ids))) return fail(TIDE_ERR_INVALID_ARG, "x, W and the targets / top_ids must not be NULL");
    if (s.K && s.T > 0 && !c.values) return fail(TIDE_ERR_INVALID_ARG, "top_values must not be NULL");
    int rc;
    if ((rc = check_rows(c.x, c.x_stride, "x")) || (rc = check_rows(c.W, c.w_stride, "W"))) return rc;
    if (!grads) {
        if (s.T > 0 && (!c.loss || !c.lse || (s.K && !c.z))) return fail(TIDE_ERR_INVALID_ARG, "loss, lse and z must not be NULL");
    } else {
        if (s.T > 0 && (!c.lse_in || !c.grad)) return fail(TIDE_ERR_INVALID_ARG, "lse and grad_loss must not be NULL");
        if ((c.dx && c.dx_stride < s.d) || (c.dW && c.dw_stride < s.d)) return fail(TIDE_ERR_INVALID_ARG, "row strides of dx and dW must be at least d");
        if ((rc = check_rows(c.dx, c.dx ? c.dx_stride : 0, "dx")) || (rc = check_rows(c.dW, c.dW ? c.dw_stride : 0, "dW"))) return rc;
    }
    if (((uintptr_t)c.ids | (uintptr_t)c.values | (uintptr_t)c.loss | (uintptr_t)c.lse | (uintptr_t)c.z | (uintptr_t)c.lse_in | (uintptr_t)c.grad) & 3)
        return fail(TIDE_ERR_ALIGNMENT, "4-byte arrays must be aligned to their elements");
    return TIDE_OK;
}

int head_space(const HeadCall& c, bool grads, HeadWork* w) {
    const size_t need = head_layout(c.s, grads, nullptr, nullptr);
    if (!c.workspace || c.workspace_bytes < need) return fail(TIDE_ERR_WORKSPACE, "this call needs %zu bytes of workspace, %zu given", need, c.workspace ? c.workspace_bytes : 0);
    if ((uintptr_t)c.workspace & 255) return fail(TIDE_ERR_ALIGNMENT, "the workspace must be 256-byte aligned");
    head_layout(c.s, grads, c.workspace, w);
    return TIDE_OK;
}

// Rows per workgroup of the copies: 2048 chunks of eight elements, eight a thread.
int64_t head_copy_rows(int64_t chunks) { return std::max<int64_t>(1, 8 * kHeadRowThreads / chunks); }
void head_max(const void* rows, int64_t stride, int64_t n, int64_t d, uint32_t* out, int* blocks, hipStream_t st) {
    *blocks = (int)std::min<int64_t>(n, kHeadMaxBlocks);
    if (*blocks) hipLaunchKernelGGL(tide_head_max_kernel, dim3(*blocks), dim3(kHeadRowThreads), 0, st, (const char*)rows, stride * 4, n, (int)d, out);
}
template <int DT> void head_copy(const HeadShape& s, const void* rows, int64_t stride, int64_t n, const int32_t* source, const HeadWork& w, const float4* row_const, int blocks, char* out, hipStream_t st,
                                 bool stacked = false) {
    if (n == 0) return;
    const int64_t rows_each = head_copy_rows(s.dp() / 8);
    hipLaunchKernelGGL((tide_head_copy_kernel<DT>), dim3((unsigned)((n + rows_each - 1) / rows_each)), dim3(kHeadRowThreads), 0, st, (const char*)rows, stride * Storage<DT>::kBytes, n, (int)rows_each,
                       (int)s.d, source, w.ctl, row_const, w.largest, blocks, (int)stacked, out, s.dp() * 2, s.plane_bytes(n));
}
// fp32 rows of x as planes for the logits; returns the workgroups, each of which leaves a greatest exponent where there are gradients (row_const).
int head_rows(const HeadShape& s, const void* x, int64_t stride, const int32_t* source, const HeadWork& w, const float4* row_const, hipStream_t st) {
    if (s.T == 0) return 0;
    const bool wave_rows = s.dp() <= 2048;
    const unsigned blocks = (unsigned)std::min<int64_t>(wave_rows ? (s.T + 3) / 4 : s.T, kHeadMaxBlocks);
    auto kernel = wave_rows ? &tide_head_rows_kernel<true> : &tide_head_rows_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kHeadRowThreads), 0, st, (const char*)x, stride * 4, (int)s.T, (int)s.d, source, w.ctl, row_const, w.x, s.dp() * 2, s.plane_bytes(s.T), w.x_exp,
                       row_const ? w.largest : nullptr);
    return (int)blocks;
}
// x or W as an operand: the caller's rows, or the copy's planes of n rows.
HeadOperand head_operand(const HeadShape& s, const void* rows, int64_t stride, const char* copy, int64_t n) {
    if (copy) return HeadOperand{{copy, copy + (s.planes() - 1) * s.plane_bytes(n)}, s.dp() * 2};
    return HeadOperand{{(const char*)rows, (const char*)rows}, stride * (int64_t)elem_bytes(s.dtype)};
}

int head_forward(HeadCall& c) {
    int rc = check_head(c, false);
    if (rc || c.s.T == 0) return rc;
    if ((rc = resident_cus(&c.s.cus))) return rc;
    const HeadShape& s = c.s;
    HeadWork w;
    if ((rc = head_space(c, false, &w))) return rc;
    rc = by_dtype(s.dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        const bool direct = s.direct(false);
        if (DT == kF32 && !direct) {
            HeadCtlParams cp{};
            cp.ctl = w.ctl;
            cp.w_max = w.w_max;
            head_max(c.W, c.w_stride, s.V, s.d, w.w_max, &cp.w_blocks, c.st);
            hipLaunchKernelGGL(tide_head_ctl_kernel, dim3(1), dim3(kHeadCtlThreads), 0, c.st, cp);
        }
        if (s.copied(false)) {
            if (DT == kF32) head_rows(s, c.x, c.x_stride, nullptr, w, nullptr, c.st);
            else head_copy<DT>(s, c.x, c.x_stride, s.T, nullptr, w, nullptr, 0, w.x, c.st);
            head_copy<DT>(s, c.W, c.w_stride, s.V, nullptr, w, nullptr, 0, w.w, c.st);
        }
        HeadGemmParams p{};
        p.q = head_operand(s, c.x, c.x_stride, w.x, s.T);
        p.p = head_operand(s, c.W, c.w_stride, w.w, s.V);
        p.q_rows = (int)s.T;
        p.p_rows = (int)s.V;
        p.k = s.copied(false) ? (int)s.dp() : (int)s.d;
        p.segments = DT == kF32 && !direct ? 3 : 1;
        p.k_slices = 1;
        p.ctl = DT == kF32 && !direct ? w.ctl : nullptr;
        p.q_exp = w.x_exp;
        p.c1 = 1.4426950408889634f / c.tau;
        p.ids = c.ids;
        p.K = s.K ? (int)s.K : 1;
        p.part = w.part;
        p.pitch = s.pitch();
        p.z_out = s.K ? c.z : w.z;
        int rc2 = TIDE_OK;
        if (direct) {
            if constexpr (DT == kF32)
                rc2 = s.T <= 16 ? launch_head<kF32, kF32, kHeadStats, HeadTile16F>(s.T, s.V, c.st, p) : s.T <= 32 ? launch_head<kF32, kF32, kHeadStats, HeadTile32F>(s.T, s.V, c.st, p) : s.T <= 48 || (s.T > 64 && s.T <= 96) ? launch_head<kF32, kF32, kHeadStats, HeadTile48F>(s.T, s.V, c.st, p)
                     : launch_head<kF32, kF32, kHeadStats, HeadTile64F>(s.T, s.V, c.st, p);
        } else {
            rc2 = by_head_tile(s.rows_per_tile(), [&](auto tile) { return launch_head<kHeadElem<DT>, DT, kHeadStats, decltype(tile)>(s.T, s.V, c.st, p); });
        }
        if (rc2) return rc2;
        HeadFinishParams f{};
        f.part = w.part;
        f.parts = (int)s.parts();
        f.T = (int)s.T;
        f.K = p.K;
        f.V = (int)s.V;
        f.tau = c.tau;
        f.ids = c.ids;
        f.values = c.values;
        f.z = p.z_out;
        f.loss = c.loss;
        f.lse = c.lse;
        hipLaunchKernelGGL(tide_head_finish_kernel, dim3((unsigned)((s.T + 15) / 16)), dim3(1024), 0, c.st, f);
        return TIDE_OK;
    });
    if (rc) return rc;
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

int head_backward(HeadCall& c) {
    int rc = check_head(c, true);
    if (rc || (!c.dx && !c.dW)) return rc;
    if ((rc = resident_cus(&c.s.cus))) return rc;
    const HeadShape& s = c.s;
    HeadWork w;
    if ((rc = head_space(c, true, &w))) return rc;
    rc = by_dtype(s.dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value, E = kHeadElem<DT>;
        HeadCtlParams cp{};
        cp.ctl = w.ctl;
        cp.w_max = w.w_max;
        if constexpr (DT == kF32) head_max(c.W, c.w_stride, s.V, s.d, w.w_max, &cp.w_blocks, c.st);
        if (s.K && s.T)
            hipLaunchKernelGGL(tide_head_teacher_kernel, dim3((unsigned)((s.T + 3) / 4)), dim3(kHeadRowThreads), 0, c.st, c.values, c.ids, (int)s.T, (int)s.K, (int)s.V,
                               1.0f / c.tau, w.wanted, w.taught);
        cp.grads = 1;
        cp.grad_scale = DT == kF32 ? (int)kHeadGradOwn : DT == kF16 ? (int)kHeadGradCommon : (int)kHeadGradAsIs;
        cp.T = (int)s.T;
        cp.V = (int)s.V;
        cp.target = s.K ? nullptr : c.ids;
        cp.taught = w.taught;
        cp.grad = c.grad;
        cp.lse = c.lse_in;
        cp.tau = c.tau;
        cp.source = w.source;
        cp.place = w.place;
        cp.row_const = w.row_const;
        hipLaunchKernelGGL(tide_head_ctl_kernel, dim3(1), dim3(kHeadCtlThreads), 0, c.st, cp);
        if constexpr (DT == kF32) {
            const int blocks = head_rows(s, c.x, c.x_stride, w.source, w, w.row_const, c.st);
            if (c.dW) head_copy<DT>(s, c.x, c.x_stride, s.T, w.source, w, w.row_const, blocks, w.x_dw, c.st);
        } else {
            head_copy<DT>(s, c.x, c.x_stride, s.T, w.source, w, nullptr, 0, w.x, c.st, s.stacked() != 0);
        }
        if (s.copied(true)) head_copy<DT>(s, c.W, c.w_stride, s.V, nullptr, w, nullptr, 0, w.w, c.st);
        const HeadOperand x = head_operand(s, nullptr, 0, w.x, s.T), x_dw = head_operand(s, nullptr, 0, w.x_dw, s.T), W = head_operand(s, c.W, c.w_stride, w.w, s.V);
        const int64_t piece = s.piece(), g_plane = s.T * piece * 2;
        const HeadOperand g{{w.g, w.g + (s.stacked() ? 0 : s.g_planes() - 1) * g_plane}, piece * 2};
        const int slices = s.dx_slices(), dw_slices = s.dw_slices();
        for (int64_t v0 = 0; v0 < s.V; v0 += piece) {
            const int64_t width = std::min(piece, s.V - v0);
            const HeadOperand Wv{{W.plane[0] + v0 * W.row_bytes, W.plane[1] + v0 * W.row_bytes}, W.row_bytes};
            HeadGemmParams p{};
            p.ctl = w.ctl;
            p.segments = DT == kF32 ? 3 : 1;
            p.k_slices = 1;
            int rc2 = TIDE_OK;
            if (s.T) {
                HeadGemmParams a = p;
                a.q = x;
                a.p = Wv;
                a.q_rows = (int)s.T;
                a.p_rows = (int)width;
                a.k = (int)s.dp();
                a.c1 = 1.4426950408889634f / c.tau;
                a.ids = c.ids;
                a.K = s.K ? (int)s.K : 1;
                a.v0 = (int)v0;
                a.q_exp = w.x_exp;
                a.row_const = w.row_const;
                a.wanted = w.wanted;
                a.g_out = w.g;
                a.g_row_bytes = g.row_bytes;
                a.g_plane_bytes = g.plane[1] - g.plane[0];
                a.stacked = s.stacked() != 0;
                rc2 = by_head_tile(s.rows_per_tile(), [&](auto tile) { return launch_head<E, DT, kHeadGrad, decltype(tile)>(s.T, width, c.st, a); });
                if (rc2) return rc2;
            }
            if (s.T && c.dx) {
                HeadGemmParams a = p;
                a.q = g;
                a.p = Wv;
                a.stacked = s.stacked() != 0;
                a.q_rows = (int)s.T;
                a.p_rows = (int)s.dp();
                a.k = (int)width;
                a.k_slices = slices;
                a.acc_out = w.acc;
                a.acc_slice = (s.T + s.stacked()) * s.dp();
                a.acc_ld = (int)s.dp();
                a.accumulate = v0 != 0;
                rc2 = by_head_rows(s.rows_of_dx(), [&](auto tile) { return launch_head<E, DT, kHeadRows, decltype(tile)>(s.T + s.stacked(), s.dp(), c.st, a); });
                if (rc2) return rc2;
            }
            if (c.dW) {
                HeadGemmParams a = p;
                a.q = g;
                a.p = x_dw;
                a.q_rows = (int)width;
                a.p_rows = (int)s.d;
                a.k = (int)s.T;
                a.stacked = s.stacked() != 0;
                a.out = (char*)c.dW + v0 * c.dw_stride * Storage<DT>::kBytes;
                a.out_row_elems = c.dw_stride;
                a.out_aligned = chunked_rows(s.dtype, s.d);
                if (dw_slices > 1) {
                    a.k_slices = dw_slices;
                    a.acc_out = w.dw;
                    a.acc_slice = piece * s.dp();
                    a.acc_ld = (int)s.dp();
                }
                if ((rc2 = launch_head<E, DT, kHeadWeights, HeadTile256>(width, s.d, c.st, a))) return rc2;
                if (dw_slices > 1)
                    hipLaunchKernelGGL((tide_head_dx_kernel<DT>), dim3((unsigned)std::min<int64_t>(width, 4096)), dim3(kHeadRowThreads), 0, c.st, w.dw, dw_slices, piece * s.dp(),
                                       (int)s.dp(), 0, (const int32_t*)nullptr, (const float4*)nullptr, w.ctl, (int)width, (int)s.d, a.out, c.dw_stride * Storage<DT>::kBytes);
            }
        }
        if (s.T && c.dx)
            hipLaunchKernelGGL((tide_head_dx_kernel<DT>), dim3((unsigned)std::min<int64_t>(s.T, 4096)), dim3(kHeadRowThreads), 0, c.st, w.acc, slices, (s.T + s.stacked()) * s.dp(), (int)s.dp(), (int)(s.stacked() != 0), w.place,
                               w.row_const, w.ctl, (int)s.T, (int)s.d, (char*)c.dx, c.dx_stride * Storage<DT>::kBytes);
        return TIDE_OK;
    });
    if (rc) return rc;
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

constexpr int kProjectGradMaxBlocks = 1024;
// Rows of up to 4 KiB: four at a time, a wave each.
bool project_grad_wave_rows(int64_t row_bytes) { return row_bytes <= 4096; }
// As many workgroups as have rows in equal rounds: at most two per CU, four where each then has four rounds or more, which is where the requests in flight
// outweigh the sums that each leaves (two / four, us, bf16: T = 1000, d = 4096 11.2 / 15.2, 4000 27.4 / 27.2, 8192 47.8 / 43.1; d = 768, T = 16384 23.5 / 18.5;
// d = 2048, T = 3000 12.0 / 13.1).
int project_grad_blocks(int64_t T, int64_t row_bytes, unsigned cus) {
    const int64_t turns = project_grad_wave_rows(row_bytes) ? (T + 3) / 4 : T;
    const int64_t most = std::min<int64_t>((turns >= 16 * (int64_t)cus ? 4 : 2) * cus, kProjectGradMaxBlocks);
    const int64_t rounds = std::max<int64_t>(1, (turns + most - 1) / most);
    return (int)((turns + rounds - 1) / rounds);
}

HeadShape head_gradient_shape(int dtype, int64_t T, int64_t d, int64_t V, int64_t K) { return HeadShape{dtype & ~TIDE_HEAD_WIDE, T, d, V, K, (dtype & TIDE_HEAD_WIDE) != 0}; }

}  // namespace

extern "C" {

size_t tide_head_workspace_bytes(int dtype, int64_t T, int64_t d, int64_t V, int64_t K, int gradient) {
    g_err[0] = 0;
    HeadCall c{};
    c.s = gradient ? head_gradient_shape(dtype, T, d, V, K) : HeadShape{dtype, T, d, V, K};
    c.tau = 1.0f;
    c.x_stride = c.w_stride = (d + 7) / 8 * 8;
    alignas(256) static char some[256];                // checks of pointers that are not asked about
    c.x = c.W = some;
    c.ids = (const int32_t*)some;
    c.values = c.lse_in = c.grad = (const float*)some;
    c.loss = c.lse = c.z = (float*)some;
    if (check_head(c, gradient != 0)) return 0;
    int dev = 0;                    // without a device: the answer for a 256-CU one
    if (hipGetDevice(&dev) == hipSuccess) {
        if (resident_cus(&c.s.cus) != TIDE_OK) c.s.cus = 256;
    } else {
        (void)hipGetLastError();
    }
    return head_layout(c.s, gradient != 0, nullptr, nullptr);
}

int tide_head_loss(const void* x, int dtype, int64_t T, int64_t d, int64_t V, int64_t x_row_stride, const void* W, int64_t w_row_stride, const int32_t* target, float* loss,
                   float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    HeadCall c{};
    c.s = HeadShape{dtype, T, d, V, 0};
    c.x = x, c.W = W, c.x_stride = x_row_stride, c.w_stride = w_row_stride;
    c.ids = target, c.tau = 1.0f, c.loss = loss, c.lse = lse;
    c.workspace = workspace, c.workspace_bytes = workspace_bytes, c.st = (hipStream_t)stream;
    return head_forward(c);
}

int tide_head_loss_grad(const void* x, int dtype, int64_t T, int64_t d, int64_t V, int64_t x_row_stride, const void* W, int64_t w_row_stride, const int32_t* target,
                        const float* lse, const float* grad_loss, void* dx, int64_t dx_row_stride, void* dW, int64_t dw_row_stride, void* workspace, size_t workspace_bytes,
                        void* stream) {
    g_err[0] = 0;
    HeadCall c{};
    c.s = head_gradient_shape(dtype, T, d, V, 0);
    c.x = x, c.W = W, c.x_stride = x_row_stride, c.w_stride = w_row_stride;
    c.ids = target, c.tau = 1.0f, c.lse_in = lse, c.grad = grad_loss;
    c.dx = dx, c.dx_stride = dx_row_stride, c.dW = dW, c.dw_stride = dw_row_stride;
    c.workspace = workspace, c.workspace_bytes = workspace_bytes, c.st = (hipStream_t)stream;
    return head_backward(c);
}

int tide_head_distill(const void* x, int dtype, int64_t T, int64_t d, int64_t V, int64_t x_row_stride, const void* W, int64_t w_row_stride, const float* top_values,
                      const int32_t* top_ids, int64_t K, float tau, float* loss, float* lse, float* z, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    if (K < 1) return fail(TIDE_ERR_INVALID_ARG, "K = %lld must be at least 1", (long long)K);
    HeadCall c{};
    c.s = HeadShape{dtype, T, d, V, K};
    c.x = x, c.W = W, c.x_stride = x_row_stride, c.w_stride = w_row_stride;
    c.ids = top_ids, c.values = top_values, c.tau = tau, c.loss = loss, c.lse = lse, c.z = z;
    c.workspace = workspace, c.workspace_bytes = workspace_bytes, c.st = (hipStream_t)stream;
    return head_forward(c);
}

int tide_head_distill_grad(const void* x, int dtype, int64_t T, int64_t d, int64_t V, int64_t x_row_stride, const void* W, int64_t w_row_stride, const float* top_values,
                           const int32_t* top_ids, int64_t K, float tau, const float* lse, const float* grad_loss, void* dx, int64_t dx_row_stride, void* dW,
                           int64_t dw_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    if (K < 1) return fail(TIDE_ERR_INVALID_ARG, "K = %lld must be at least 1", (long long)K);
    HeadCall c{};
    c.s = head_gradient_shape(dtype, T, d, V, K);
    c.x = x, c.W = W, c.x_stride = x_row_stride, c.w_stride = w_row_stride;
    c.ids = top_ids, c.values = top_values, c.tau = tau, c.lse_in = lse, c.grad = grad_loss;
    c.dx = dx, c.dx_stride = dx_row_stride, c.dW = dW, c.dw_stride = dw_row_stride;
    c.workspace = workspace, c.workspace_bytes = workspace_bytes, c.st = (hipStream_t)stream;
    return head_backward(c);
}

size_t tide_exit_project_grad_bytes(int64_t T, int64_t d) {
    if (T < 0 || d < 1 || d > kMaxHidden) return 0;
    return ((size_t)std::min<int64_t>(std::max<int64_t>(T, 1), kProjectGradMaxBlocks) * d * sizeof(float) + 255) & ~size_t(255);
}

int tide_exit_project_grad(const void* hidden, int dtype, int64_t C, int64_t T, int64_t d, int64_t ckpt_stride, int64_t row_stride, const void* final_hidden,
                           int64_t final_row_stride, const int32_t* exit_layer, const int32_t* layer_ids, const float* norm_gain, float eps, const void* grad_out,
                           int64_t grad_out_row_stride, void* grad_rows, int64_t grad_row_stride, float* grad_gain, void* workspace, size_t workspace_bytes, void* stream) {
    g_err[0] = 0;
    int rc = check_common(hidden, dtype, C, T, d, kBottleneck, ckpt_stride, row_stride, hidden, reinterpret_cast<const float*>(hidden), eps, true);
    if (rc) return rc;
    if (!layer_ids || (T > 0 && (!exit_layer || !grad_out || !grad_rows)))
        return fail(TIDE_ERR_INVALID_ARG, "exit_layer, layer_ids (host), grad_out and grad_rows must not be NULL");
    if (grad_out_row_stride < d || grad_row_stride < d || (final_hidden && final_row_stride < d))
        return fail(TIDE_ERR_INVALID_ARG, "row strides of grad_out, grad_rows and final_hidden must be at least d");
    const size_t eb = elem_bytes(dtype);
    if (((uintptr_t)grad_out | (uintptr_t)grad_rows | (uintptr_t)final_hidden | (uintptr_t)norm_gain | ((size_t)grad_out_row_stride * eb) | ((size_t)grad_row_stride * eb) |
         (final_hidden ? (size_t)final_row_stride * eb : 0)) & 15)
        return fail(TIDE_ERR_ALIGNMENT, "grad_out, grad_rows, final_hidden and norm_gain bases and the row strides must be multiples of 16 bytes");
    if ((uintptr_t)grad_gain & 3) return fail(TIDE_ERR_ALIGNMENT, "grad_gain must be aligned to a float");
    ProjectGradParams p;
    std::memset(&p, 0, sizeof(p));
    for (int64_t c = 0; c < C; ++c) {
        if (c > 0 && layer_ids[c] <= layer_ids[c - 1]) return fail(TIDE_ERR_INVALID_ARG, "layer_ids must be strictly ascending");
        p.layer_id[c] = layer_ids[c];
    }
    if (T == 0 && !grad_gain) return TIDE_OK;
    unsigned cus = 0;
    if ((rc = resident_cus(&cus))) return rc;
    const int blocks = project_grad_blocks(T, d * (int64_t)eb, cus);
    const bool joined = grad_gain && blocks != 1;      // one workgroup's sums are the gradient
    if (joined && blocks) {
        const size_t need = (size_t)blocks * d * sizeof(float);
        if (!workspace || workspace_bytes < need) return fail(TIDE_ERR_WORKSPACE, "this call needs %zu bytes of workspace, %zu given", need, workspace ? workspace_bytes : 0);
        if ((uintptr_t)workspace & 15) return fail(TIDE_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
    }
    if (!joined && ((uintptr_t)grad_gain & 15)) return fail(TIDE_ERR_ALIGNMENT, "grad_gain must be 16-byte aligned");
    p.hidden = (const char*)hidden;
    p.ckpt_stride_bytes = ckpt_stride * (int64_t)eb;
    p.row_stride_bytes = row_stride * (int64_t)eb;
    p.final_hidden = (const char*)final_hidden;
    p.final_row_stride_bytes = final_row_stride * (int64_t)eb;
    p.exit_layer = exit_layer;
    p.gain = norm_gain;
    p.grad_out = (const char*)grad_out;
    p.grad_out_row_bytes = grad_out_row_stride * (int64_t)eb;
    p.grad = (char*)grad_rows;
    p.grad_row_bytes = grad_row_stride * (int64_t)eb;
    p.part = joined ? (float*)workspace : grad_gain;
    p.C = (int)C;
    p.T = (int)T;
    p.d = (int)d;
    p.eps = eps;
    hipStream_t st = (hipStream_t)stream;
    const bool wave_rows = project_grad_wave_rows(d * (int64_t)eb);
    const int64_t step = wave_rows ? kWave : kProjectThreads, per_thread = (d * (int64_t)eb / 16 + step - 1) / step;
    if (blocks)
        by_dtype(dtype, [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            auto go = [&](auto chunks, auto wave) {
                hipLaunchKernelGGL((tide_project_grad_kernel<DT, decltype(chunks)::value, decltype(wave)::value>), dim3(blocks), dim3(kProjectThreads), 0, st, p);
                return 0;
            };
            using std::integral_constant;
            if (wave_rows) {
                if (per_thread <= 2) return go(integral_constant<int, 2>{}, std::true_type{});
                return go(integral_constant<int, 4>{}, std::true_type{});
            }
            if (per_thread <= 2) return go(integral_constant<int, 2>{}, std::false_type{});
            if (per_thread <= 4) return go(integral_constant<int, 4>{}, std::false_type{});
            if constexpr (DT == kF32) {                // rows above 32 KiB
                if (per_thread > 8) return go(integral_constant<int, 16>{}, std::false_type{});
            }
            return go(integral_constant<int, 8>{}, std::false_type{});
        });
    if (joined) hipLaunchKernelGGL(tide_project_gain_kernel, dim3((unsigned)((d + 31) / 32)), dim3(kProjectGainThreads), 0, st, (const float*)workspace, blocks, (int)d, grad_gain);
    TIDE_HIP(hipGetLastError());
    return TIDE_OK;
}

}  // extern "C"
