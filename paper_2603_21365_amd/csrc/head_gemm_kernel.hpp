// The matrix products of the head operators: z = x W^T of rows x [T, d] under an LM head W [V, d], what a softmax over the V
// columns needs of z, and the two products of its gradient.  The logits are never kept: they are made a tile at a time, in
// registers, and leave as
//   kHeadStats   per row, of a tile's or a wave's columns, the maximum and the sum of exponentials relative to it, and the logits of the row's own few tokens;
//   kHeadGrad    G = (softmax - wanted) * scale of a piece of the vocabulary, in 16 bits (or two planes of 16), for the two products that follow;
//   kHeadRows    dx += G W over that piece (fp32, a buffer per k slice);
//   kHeadWeights dW = G^T x of that piece, complete, or in k slices where its tiles are few.
// The gradient makes the logits a second time, so a training step is four products where one that keeps T x V logits has three.
//
// One tile of kQ x kP output elements per workgroup of eight waves, k in stages of 64 elements (fp32 rows: 32).  "q" is the operand whose rows are
// the output's rows, "p" the one whose rows are its columns: a matrix-core step takes the p fragment first, so a lane holds ONE
// output row and, in its registers, runs of four consecutive columns (softmax: sums over columns stay in the lane).
//
// Both operands go through LDS by direct transfers (16 bytes a lane, no registers), a ring of stages for each; what lies outside the operand is
// fetched as zeros by the buffer descriptor's bound, so ragged rows, columns and k cost no instruction in the loop.  An operand
// whose k runs along memory rows (x, W in the logits; G in dx) is read as fragments of 16 bytes; one whose k runs ACROSS memory rows
// (W in dx; G and x in dW) lies in LDS as it lies in memory and is read by the transposing LDS loads, so no transposed copy of
// W, x or G is ever made.
//
// The waves work as two groups of four, one wave of each per SIMD, that take turns: while one group's matrix steps run (a phase of 32 k elements, 512 cycles),
// the other reads its fragments for the next phase and issues transfers; every phase ends in a barrier.  Left to itself (both groups in step, reads and
// steps mixed by the compiler) the same kernel is 6 % slower (T = 4096, d = 4096, V = 128000: 3.50 / 3.27 ms).  A stage's slot is free when the group that
// is behind has read its second half, so the transfers issued in stage k fill the slots of stage k - 1.
//
// The transfers are inline assembly: of the builtin the compiler makes every LDS read wait for all outstanding transfers, as it cannot
// tell the ring's slots apart.  They have no output registers; they are ordered by explicit counts and the phases' barriers.  A stage is 128 bytes of
// a memory row: with 64 every cache line came twice from L2, and the CU's load path was the bound (4.0 ms).
//
// fp32 operands are taken apart into two fp16 planes, x * 2^s = hi + 2^-12 lo + O(2^-23 x), and a product is three passes over k: hi lo + lo hi, whose sums are
// multiplied by 2^-12, then hi hi (what is dropped is 2^-22 of a term at most).  With the largest magnitude in [2^14, 2^15) lo reaches the same, and the two hold
// every value of more than 2^-30 of the largest to 22 bits and the others to 2^-51 of it (lo as it is: 2^-17 and 2^-39, and an improbable token, p = 1e-10,
// had two decimal digits in its row of dW).  s is one for W; a row of x has its own in the logits, and a row of G its own, so that no row's size reaches
// another row's loss or dx.  dW adds up rows of G and x: there a row of x takes 2^c less the power that its row of G has, with one c for the call, so that the
// largest |g x| sets the scale.  The fp32 matrix instructions have 1/16 of the 16-bit rate;
// the forward call on few rows takes them all the same, on the rows as they are, as there reading W is the bound.
#pragma once
#include <type_traits>

#include "device_utils.hpp"
#include "prefill_dma_kernel.hpp"

namespace tide {

enum : int { kHeadStats = 0, kHeadGrad = 1, kHeadRows = 2, kHeadWeights = 3 };

// What one call finds out on the device before its products (head_rows_kernel.hpp).
struct HeadCtl {
    int live;                      // rows that have a gradient
    int w_exp;                     // the power of two that W was multiplied by (fp32)
    int dw_exp;                    // the same of dW's sums
};

constexpr int kHeadRowBytes = 128;                   // of a row along k in a stage: a whole cache line

struct HeadOperand {
    const char* plane[2];
    int64_t row_bytes;
};

struct HeadGemmParams {
    HeadOperand q, p;
    int q_rows, p_rows, k;     // of these the one that counts live rows is replaced by ctl->live
    int segments;              // passes over k: 1, or 3 for operands of two planes
    int tiles_p, k_slices;
    int pitch;                 // columns of a tile: kP, or fewer (statistics) where that gives every CU as many
    const HeadCtl* ctl;        // null where nothing is scaled and every row counts (16-bit statistics)
    const int32_t* q_exp;      // logits of planes: [q_rows] the power of two that a row of x was multiplied by
    // statistics and G
    float c1;                  // log2(e) / tau
    const int32_t* ids;        // [T][K] the tokens' own entries of the vocabulary; others than 0 .. V - 1: none
    int K, v0;                 // p row 0 is token v0
    float2* part;              // statistics: [tiles_p * kParts][q_rows] largest logit and sum of exp((logit - it) / tau)
    float* z_out;              // statistics: [q_rows][K]
    const float4* row_const;   // G: of each row lse * log2 e, grad * tau * 2^s, and as integers the target (wanted == null) or the token, and s
    const float* wanted;       // G: [T][K] or null (one)
    char* g_out;               // G: rounded to 16 bits, and (g_plane_bytes != 0) what that leaves in a second plane
    int64_t g_row_bytes, g_plane_bytes;
    // dx
    float* acc_out;            // [k_slices][acc_rows][acc_ld]
    int64_t acc_slice;         // elements
    int acc_ld, accumulate;
    int stacked;               // G's second plane follows its live rows as as many further ones (16-bit operands): rows of dx, of k in dW
    // dW
    char* out;
    int64_t out_row_elems;
    int out_aligned;           // rows of whole 16-byte chunks
};

// kSQ, kSP: stages of each operand that its part of LDS holds.  EB: bytes of an element (4: fp32 rows as they are).
template <int WQ, int WP, int BQ, int BP, int SQ, int SP, int EB = 2> struct HeadTile {
    static constexpr int kWQ = WQ, kWP = WP, kBQ = BQ, kBP = BP, kSQ = SQ, kSP = SP, kEB = EB;
    static constexpr int kWaves = WQ * WP, kThreads = kWaves * kWave, kK = kHeadRowBytes / EB;
    static constexpr bool kTurns = BQ * BP >= 16;                // two groups of waves that take turns (few rows: bound by memory, one barrier a stage)
    static constexpr int kQ = WQ * BQ * 16, kP = WP * BP * 16;
    static constexpr int kQBytes = kQ * kHeadRowBytes, kPBytes = kP * kHeadRowBytes, kRingBytes = SQ * kQBytes + SP * kPBytes;
    static constexpr int kCols = BP * 16, kLd = kCols + 4;       // a wave's columns; its rows in LDS after the loop, padded against bank conflicts
    static constexpr int kStageBytes = kWaves * 16 * kLd * 4;    // 16 rows of every wave
    static constexpr bool kJoined = WP > 2;                      // the statistics of a tile's columns leave as one
    static constexpr int kParts = kJoined ? 1 : WP, kJoinBytes = kJoined ? WP * kQ * 8 : 0;
    static constexpr int kLdsBytes = kRingBytes > kStageBytes + kJoinBytes ? kRingBytes : kStageBytes + kJoinBytes;
    static_assert(kWaves == 8 && SP >= 2 && SQ >= SP, "two groups of four waves");
    static_assert(kLdsBytes <= 160 * 1024, "LDS of a CU");
};
constexpr float kHeadLow = 4096.0f;                  // what the second plane of an fp32 value holds its part multiplied by
constexpr uint32_t kHeadNowhere = 0x80000000u;       // an offset at the descriptor's bound: fetched as zeros

// 64 lanes x 16 bytes from memory (offsets voff from the descriptor's base) to 1 KiB of LDS at byte `lds`.  m0 is written and not named: the compiler keeps
// nothing there between instructions (it is reserved; clang refuses it in a list of clobbers) and sets it before each use of its own, of which these kernels have none.
__device__ __forceinline__ void head_dma(uint32_t lds, uint32_t voff, u32x4 rsrc) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(rsrc) : "memory");
}
template <int n> __device__ __forceinline__ void head_wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(n) : "memory"); }

// One operand's transfers: kRows tile rows of a stage, instruction n = wave + kWaves i of kInstr, a ring of kSlots stages at byte `lds`.
template <int kRows, bool kAcross, int kWaves, int kEB = 2> struct HeadFeed {
    static constexpr int kK = kHeadRowBytes / kEB, kBytes = kRows * kHeadRowBytes, kInstr = kBytes / 1024, kN = (kInstr + kWaves - 1) / kWaves;
    uint32_t voff[kN];
    int along;                 // first k element of this lane's chunks within a stage (along), or the first one's k row (across)
    const char* base;
    int64_t step;
    int issued, kk, fill;      // stages issued, the next one's number within its segment, its slot's byte

    // Position of chunk c of a memory row in LDS, chosen so that the lanes that read at a time cover all banks.  Along: 128-byte rows, 16 of them at one
    // chunk.  Across: rows of 512 bytes, 32 bytes of each of eight.
    static __device__ __forceinline__ int place_along(int row, int c) { return c ^ ((row >> 1) & 7); }
    static __device__ __forceinline__ int place_across(int kr, int c) {
        static_assert(!kAcross || (kRows == 256 && kEB == 2), "");
        return c ^ ((kr & 3) << 1 | (kr >> 3 & 1) << 3);
    }

    // plane: the one that the first segment takes
    __device__ __forceinline__ void init(const HeadOperand& o, int plane, int row0, int rows, int first, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int n = wave + kWaves * i;
            if constexpr (!kAcross) {
                const int r = 8 * n + (lane >> 3), c = place_along(r, lane & 7);
                voff[i] = row0 + r < rows ? (uint32_t)r * (uint32_t)o.row_bytes + c * 16 : kHeadNowhere;
                if (i == 0) along = c * (16 / kEB);        // (the same for all: their rows differ by multiples of 16)
            } else {
                const int byte = n * 1024 + lane * 16, kr = byte / (kRows * 2), c = place_across(kr, byte % (kRows * 2) >> 4);
                voff[i] = row0 + c * 8 < rows ? (uint32_t)kr * (uint32_t)o.row_bytes + c * 16 : kHeadNowhere;
                if (i == 0) along = kr;
            }
        }
        step = kAcross ? kK * o.row_bytes : kHeadRowBytes;
        issued = kk = fill = 0;
        seek(o, plane, row0, first);
    }
    __device__ __forceinline__ void seek(const HeadOperand& o, int plane, int row0, int stage) {
        base = o.plane[plane] + (kAcross ? (int64_t)row0 * 2 : (int64_t)row0 * o.row_bytes) + stage * step;
    }
    // The next stage's transfers: `n` stages in segments of `nk`, k_elems elements of k from stage `first` on; `second`: the segment that takes the second
    // plane.  Beyond the last stage zeros are fetched all the same, so that the counts of outstanding transfers hold.
    template <int kSlots>
    __device__ __forceinline__ void issue(uint32_t lds, const HeadOperand& o, int second, int row0, int n, int nk, int first, int k_elems, int wave) {
        const int left = issued < n ? k_elems - (first + kk) * kK : 0;
        u32x4 rsrc;
        rsrc[0] = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
        rsrc[1] = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32) & 0xffffu);
        rsrc[2] = __builtin_amdgcn_readfirstlane(left > 0 ? kHeadNowhere : 0u);
        rsrc[3] = 0x00020000u;
        // A scalar register that a vector instruction has written (v_readfirstlane) is good for a memory instruction's descriptor five wait states later; the compiler
        // sees to that for its own instructions, not for those in inline assembly.
        asm volatile("s_nop 4" : "+s"(rsrc));
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (kInstr % kWaves != 0 && wave + kWaves * i >= kInstr) break;
            const int at = kAcross ? along + kWaves * i * (1024 / (kRows * 2)) : along;
            head_dma(lds + fill + (wave + kWaves * i) * 1024, at < left ? voff[i] : kHeadNowhere, rsrc);
        }
        base += step;
        fill = fill + kBytes == kSlots * kBytes ? 0 : fill + kBytes;
        ++issued;
        if (++kk == nk && issued < n) {                   // the next segment
            kk = 0;
            seek(o, issued == second * nk ? 1 : 0, row0, first);
        }
    }
};

typedef __attribute__((address_space(3))) char head_lds;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 head_lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 head_lds_u32x4;

template <int DT> __device__ __forceinline__ uint32_t head_round2(float a, float b) {
    if constexpr (DT == kF16) {
        const f16x2 h = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        const bf16x2 h = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
        return __builtin_bit_cast(uint32_t, h);
    }
}

__device__ __forceinline__ f32x4 head_shifted(f32x4 v, int n) { return f32x4{ldexpf(v[0], n), ldexpf(v[1], n), ldexpf(v[2], n), ldexpf(v[3], n)}; }
template <int DT> __device__ __forceinline__ float head_rounded(float v) {
    if constexpr (DT == kF16) return (float)static_cast<_Float16>(v);
    else return (float)static_cast<__bf16>(v);
}
template <int DT> __device__ __forceinline__ void head_put(char* row, int i, float v) {
    if constexpr (DT == kF32) reinterpret_cast<float*>(row)[i] = v;
    else if constexpr (DT == kF16) reinterpret_cast<_Float16*>(row)[i] = static_cast<_Float16>(v);
    else reinterpret_cast<__bf16*>(row)[i] = static_cast<__bf16>(v);
}

// The fragment of block b (16 tile rows) and k group g (32 elements) of an operand at `at`: lane l gets row l % 16, the 8 k values of quarter l / 16.
template <int kRows, bool kAcross> __device__ __forceinline__ u32x4 head_fragment(head_lds* at, int b, int g, int lane) {
    typedef HeadFeed<kRows, kAcross, 8> Feed;
    if constexpr (!kAcross) {
        const int row = lane & 15, c = Feed::place_along(row, 4 * g + (lane >> 4));        // (16 b changes nothing: places repeat every 16 rows)
        return *(head_lds_u32x4*)(at + (16 * b + row) * 128 + c * 16);
    } else {
        // two loads of four k rows: a group of 16 lanes supplies 4 rows x 16 columns and each lane receives one column
        const int i = lane & 15, c = 2 * b + ((i & 3) >> 1);
        s16x4 v[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int kr = 32 * g + 8 * (lane >> 4) + 4 * s + (i >> 2);
            v[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((head_lds_s16x4*)(at + kr * (kRows * 2) + Feed::place_across(kr, c) * 16 + (i & 1) * 8));
        }
        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
        const u32x2 a = __builtin_bit_cast(u32x2, v[0]), d = __builtin_bit_cast(u32x2, v[1]);
        return u32x4{a[0], a[1], d[0], d[1]};
    }
}

// The same of fp32 rows: lane l gets the 8 k values of quarter l / 16 of 32.
struct HeadFloats {
    f32x4 v[2];
};
template <int kRows> __device__ __forceinline__ HeadFloats head_fragment_f32(head_lds* at, int b, int lane) {
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    typedef HeadFeed<kRows, false, 8, 4> Feed;
    const int row = lane & 15, c = 2 * (lane >> 4);
    head_lds* from = at + (16 * b + row) * 128;
    return HeadFloats{{*(lds_f32x4*)(from + Feed::place_along(row, c) * 16), *(lds_f32x4*)(from + Feed::place_along(row, c + 1) * 16)}};
}

// acc[16x16] += A[16 x 32] * B[32 x 16].  With operands that are not zeros the chip runs into its power limit before its rate: back to back from registers this
// shape does 2.09 PFLOP/s where 32 x 32 x 16 does 1.84 (2.42 / 2.45 on zeros), as it moves half the accumulators per product.
template <int DT> __device__ __forceinline__ f32x4 head_mma(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (DT == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// fp32: eight steps of four k values, one from each quarter of the lanes, for up to 128 rows.  (A few rows are bound by reading W; three bf16 terms a value, split as the
// fragments are read, cost as many cycles in the vector ALU as these in the matrix cores, and
// the fragments of x in every wave: 32003 x 768 32.2 / 26.6 us at T = 17, 100000 x 4096 418 / 328 at T = 20; adding up
// in blocks costs 3 us of that at T = 17 and none at T = 1.)
template <int DT> __device__ __forceinline__ f32x4 head_mma(const HeadFloats& a, const HeadFloats& b, f32x4 acc) {
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i >> 2][i & 3], b.v[i >> 2][i & 3], acc, 0, 0, 0);
    return acc;
}

// Item `at` of the eighth of the work that XCD `xcd` (workgroup id mod 8) has: the work is a list of k_slices x tiles_q x tiles_p tiles that goes through groups
// of 8 row tiles column by column, so that the 32 tiles an XCD works on at a time share 8 row tiles and 4 column tiles in its L2.
__device__ __forceinline__ bool head_item(int xcd, int at, int tiles_q, int tiles_p, int k_slices, int& tq, int& tp, int& slice) {
    const int tiles = tiles_q * tiles_p, total = tiles * k_slices, per_xcd = (total + 7) >> 3;
    int t = xcd * per_xcd + at;
    if (at >= per_xcd || t >= total) return false;
    slice = t / tiles;
    t -= slice * tiles;
    const int group = t / (8 * tiles_p), q0 = group * 8, nq = min(8, tiles_q - q0), in = t - q0 * tiles_p;
    tp = in / nq;
    tq = q0 + (in - tp * nq);
    return true;
}

// Two blocks of 16 x 16 in 16 bits, as the matrix steps leave them (lane quarter h: columns 4 h .. 4 h + 3 of a row of each), exchanged so that a lane has eight
// consecutive columns: 8 h .. 8 h + 7 of the 32.
__device__ __forceinline__ u32x4 head_gather8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_permlane32_swap_b32 %2, %3\n\ts_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\tv_permlane16_swap_b32 %2, %3"
        : "+v"(a0), "+v"(b0), "+v"(a1), "+v"(b1));
    return u32x4{a0, a1, b0, b1};
}

// DT: the operands' element type, kF16 or kBF16 (kF32: fp32 rows as they are, statistics of few rows only).  OutDT: the caller's type (kF32 over kF16: planes).
// dx and dW: a workgroup per CU, which goes through its share of the tiles and requests the first stages of the next one before it deals with the results of
// the last (dW of 290 live rows, d = 4096, V = 128000: 627 / 596 us).  The others: a workgroup per tile; their results need LDS and loads, and gathering them in
// registers with the next stages under way is 3 to 6 % slower.
template <int kMode, class Tile> constexpr bool kLoops = Tile::kTurns && (kMode == kHeadRows || kMode == kHeadWeights);
template <int DT, int OutDT, int kMode, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void tide_head_gemm_kernel(const HeadGemmParams p) {
    constexpr bool kQAcross = kMode == kHeadWeights, kPAcross = kMode == kHeadRows || kMode == kHeadWeights;
    constexpr bool kPlanes = DT != OutDT;
    constexpr int kBQ = Tile::kBQ, kBP = Tile::kBP, kCols = Tile::kCols;
    typedef HeadFeed<Tile::kQ, kQAcross, Tile::kWaves, Tile::kEB> FeedQ;
    typedef HeadFeed<Tile::kP, kPAcross, Tile::kWaves, Tile::kEB> FeedP;
    static_assert((DT == kF32) == (Tile::kEB == 4) && (DT != kF32 || kMode == kHeadStats), "");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wq = wave % Tile::kWQ, wp = wave / Tile::kWQ;
    const int live = kMode == kHeadStats ? 0 : __builtin_amdgcn_readfirstlane(p.ctl->live);
    const int q_rows = kMode == kHeadGrad ? live : kMode == kHeadRows ? live << p.stacked : p.q_rows;
    const int k_elems = kMode == kHeadWeights ? live << p.stacked : p.k;
    const int tiles_q = (q_rows + Tile::kQ - 1) / Tile::kQ;
    const uint32_t lds_q = (uint32_t)(size_t)(head_lds*)smem, lds_p = lds_q + Tile::kSQ * Tile::kQBytes;

    // ---- one tile's k loop: n stages, the slice's part of every segment: of planes (hi, lo), (lo, hi), (hi, hi)
    int tq, tp, slice, q0, p0, p_end, first, nk, n;
    FeedQ fq;
    FeedP fp;
    auto set_item = [&] {
        q0 = tq * Tile::kQ, p0 = tp * p.pitch, p_end = min(p.p_rows, p0 + p.pitch);
        const int per = (k_elems + Tile::kK - 1) / Tile::kK;
        first = (int)((int64_t)per * slice / p.k_slices);
        nk = (int)((int64_t)per * (slice + 1) / p.k_slices) - first;
        n = nk * p.segments;
        fq.init(p.q, 0, q0, q_rows, first, wave, lane);
        fp.init(p.p, kPlanes, p0, p_end, first, wave, lane);
    };
    // Step s issues stage s + kSP of p, then stage s + kSQ of q.
    auto issue_p = [&] { fp.template issue<Tile::kSP>(lds_p, p.p, 0, p0, n, nk, first, k_elems, wave); };
    auto issue_q = [&] { fq.template issue<Tile::kSQ>(lds_q, p.q, 1, q0, n, nk, first, k_elems, wave); };
    auto issue_first = [&] {
#pragma unroll
        for (int s = -Tile::kSQ; s < -1; ++s) {
            if (s + Tile::kSP >= 0) issue_p();
            issue_q();
        }
    };
    // Waits until all but the last kSP - 2 steps of this wave's transfers, and the q transfers of the step before those where q is further ahead than p,
    // have landed: the next stage, in the loop.  (Memory operations of the last tile's results that are still outstanding are waited for too.)
    auto landed = [&] {
        constexpr int kSteps = Tile::kSP - 2, kAhead = Tile::kSQ > Tile::kSP ? 1 : 0;
        constexpr int kNP = FeedP::kN, kNQ = FeedQ::kInstr / Tile::kWaves, kRest = FeedQ::kInstr % Tile::kWaves;
        static_assert(FeedP::kInstr % Tile::kWaves == 0, "");
        if (kRest != 0 && wave < kRest) head_wait_vm<kSteps * kNP + (kSteps + kAhead) * (kNQ + 1)>();
        else head_wait_vm<kSteps * kNP + (kSteps + kAhead) * kNQ>();
    };
    f32x4 acc[kBP][kBQ];
    std::conditional_t<DT == kF32, HeadFloats, u32x4> aq[kBQ], ap[kBP];
    auto read = [&](auto g_c, int slot_q, int slot_p) {
        constexpr int g = decltype(g_c)::value;
        head_lds* at = (head_lds*)smem;
#pragma unroll
        for (int j = 0; j < kBQ; ++j) {
            if constexpr (DT == kF32) aq[j] = head_fragment_f32<Tile::kQ>(at + slot_q, wq * kBQ + j, lane);
            else aq[j] = head_fragment<Tile::kQ, kQAcross>(at + slot_q, wq * kBQ + j, g, lane);
        }
#pragma unroll
        for (int i = 0; i < kBP; ++i) {
            if constexpr (DT == kF32) ap[i] = head_fragment_f32<Tile::kP>(at + Tile::kSQ * Tile::kQBytes + slot_p, wp * kBP + i, lane);
            else ap[i] = head_fragment<Tile::kP, kPAcross>(at + Tile::kSQ * Tile::kQBytes + slot_p, wp * kBP + i, g, lane);
        }
    };
    auto multiply = [&] {
#pragma unroll
        for (int i = 0; i < kBP; ++i)
#pragma unroll
            for (int j = 0; j < kBQ; ++j) acc[i][j] = head_mma<DT>(ap[i], aq[j], acc[i][j]);
    };
    // Planes, before stage k: where the passes with a second plane end, their sums take their place.
    auto low_done = [&](int k) {
        if constexpr (kPlanes) {
            if (k == 2 * nk)
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int j = 0; j < kBQ; ++j) acc[i][j] *= 1.0f / kHeadLow;
        }
    };
    constexpr std::integral_constant<int, 0> g0;
    constexpr std::integral_constant<int, 1> g1;
    auto k_loop = [&] {
        int slot_q = 0, slot_p = 0;
#pragma unroll
        for (int i = 0; i < kBP; ++i)
#pragma unroll
            for (int j = 0; j < kBQ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (Tile::kTurns) {
            landed();
            ring_barrier();
            const int group = wave >> 2;
            if (group == 1) ring_barrier();
            for (int k = 0; k < n; ++k) {
                const int next_q = slot_q + Tile::kQBytes == Tile::kSQ * Tile::kQBytes ? 0 : slot_q + Tile::kQBytes;
                const int next_p = slot_p + Tile::kPBytes == Tile::kSP * Tile::kPBytes ? 0 : slot_p + Tile::kPBytes;
                auto edge = [] { __builtin_amdgcn_sched_barrier(0); ring_barrier(); __builtin_amdgcn_sched_barrier(0); };
                low_done(k);
                read(g0, slot_q, slot_p);
                issue_p();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                edge();
                multiply();
                edge();
                read(g1, slot_q, slot_p);
                issue_q();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (group == 1) landed();
                edge();
                multiply();
                __builtin_amdgcn_sched_barrier(0);
                if (group == 0) landed();
                edge();
                slot_q = next_q;
                slot_p = next_p;
            }
            if (group == 0) ring_barrier();
        } else {
            static_assert(Tile::kTurns || Tile::kSQ == Tile::kSP, "");
            f32x4 sum[kBP][kBQ];                           // fp32: sums of 128 products each are added up here, so that the roundings do not pile up over k
#pragma unroll
            for (int i = 0; i < kBP; ++i)
#pragma unroll
                for (int j = 0; j < kBQ; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            auto fold = [&] {
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int j = 0; j < kBQ; ++j) {
                        sum[i][j] += acc[i][j];
                        acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    }
            };
            for (int k = 0; k < n; ++k) {
                low_done(k);
                landed();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // this wave has read all of stage k - 1, whose slot is filled next
                ring_barrier();
                issue_p();
                issue_q();
                read(g0, slot_q, slot_p);
                multiply();
                if constexpr (Tile::kK == 64) {
                    read(g1, slot_q, slot_p);
                    multiply();
                } else if ((k & 3) == 3) {
                    fold();
                }
                slot_q = slot_q + Tile::kQBytes == Tile::kSQ * Tile::kQBytes ? 0 : slot_q + Tile::kQBytes;
                slot_p = slot_p + Tile::kPBytes == Tile::kSP * Tile::kPBytes ? 0 : slot_p + Tile::kPBytes;
            }
            if constexpr (DT == kF32) {
                fold();
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int j = 0; j < kBQ; ++j) acc[i][j] = sum[i][j];
            }
        }
        head_wait_vm<0>();                                 // (zeros beyond the last stage)
        __syncthreads();                                   // every wave has read the ring
    };

    // ---- what becomes of a tile of which this lane has row `row` of each 16 and columns 16 i + 4 h + (0 .. 3) of each 16
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((address_space(3))) f32x2 lds_f32x2;
    typedef __attribute__((address_space(3))) float lds_float;
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    lds_float* stage = (lds_float*)((head_lds*)smem + wave * 16 * Tile::kLd * 4);        // statistics and G: 16 of the wave's rows
    lds_f32x2* joined = (lds_f32x2*)((head_lds*)smem + Tile::kStageBytes);                // statistics: [kWP][kQ] maxima and sums
    const int row = lane & 15, h = lane >> 4;
    auto to_lds = [&](int j) {
#pragma unroll
        for (int i = 0; i < kBP; ++i) *(lds_f32x4*)(stage + row * Tile::kLd + 16 * i + 4 * h) = acc[i][j];
    };
    auto lds_fence = [] {                                  // the wave's own LDS accesses stay in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // Which of the row's own tokens ids[k0 .. k0 + 32) are among the first `there` columns from token `base` on: bit k - k0.  Each of the four lanes that
    // share a row looks at every fourth, eight loads at a time.
    auto own_tokens = [&](const int32_t* ids, int k0, int base, int there) {
        uint32_t mine = 0, id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = (uint32_t)ids[min(k0 + 4 * u + h, p.K - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int c = (int)(id[u] - (uint32_t)base);
            mine |= k0 + 4 * u + h < p.K && c >= 0 && c < there ? 1u << (4 * u + h) : 0u;
        }
        return mine;
    };
    // The logits of row t, of the products of its plane and W's.  (Not a factor: 2^s of a small row under a small W would overflow.)
    auto planes_back = [&](int j, int t) {
        const int back = -(p.ctl->w_exp + p.q_exp[min(t, q_rows - 1)]);
#pragma unroll
        for (int i = 0; i < kBP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = ldexpf(acc[i][j][e], back);
    };
    auto results = [&](int q0, int p0, int p_end, int slice) {
        const int col0 = p0 + wp * kCols;                  // the wave's first column
        const bool ragged = col0 + kCols > p_end;
#pragma unroll
        for (int j = 0; j < kBQ; ++j) {
            const int t = q0 + (wq * kBQ + j) * 16 + row;
            if constexpr (kMode == kHeadStats) {
                if constexpr (kPlanes) planes_back(j, t);
                if (ragged) {
#pragma unroll
                    for (int i = 0; i < kBP; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = col0 + 16 * i + 4 * h + e >= p_end ? -INFINITY : acc[i][j][e];
                }
                float m = -INFINITY;
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
                m = fmaxf(m, __shfl_xor(m, 16, kWave));
                m = fmaxf(m, __shfl_xor(m, 32, kWave));
                // The maximum stays a logit: the differences from it are exact where they count, so neither its size nor a factor's rounding gets into the sum.
                const float shift = m == -INFINITY ? 0.0f : m;
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f((acc[i][j][e] - shift) * p.c1);
                s = add_xor<32>(add_xor<16>(s));
                if constexpr (Tile::kJoined) {                // with the other waves' columns, below
                    if (h == 0) joined[wp * Tile::kQ + (wq * kBQ + j) * 16 + row] = f32x2{m, s};
                } else {
                    if (h == 0 && t < q_rows) p.part[(int64_t)((p0 / p.pitch) * Tile::kWP + wp) * q_rows + t] = float2{m, s};
                }
                const int32_t* ids = p.ids + (int64_t)min(t, q_rows - 1) * p.K;
                const int there = t < q_rows ? min(kCols, p_end - col0) : 0;
                bool staged = false;
                for (int k0 = 0; k0 < p.K; k0 += 32) {
                    uint32_t mine = 0;
                    if (p.K == 1) {
                        const int c = (int)((uint32_t)ids[0] - (uint32_t)col0);
                        mine = h == 0 && c >= 0 && c < there ? 1u : 0u;
                    } else {
                        mine = own_tokens(ids, k0, col0, there);
                    }
                    if (!__any(mine != 0)) continue;
                    if (!staged) to_lds(j);
                    staged = true;
                    lds_fence();
                    for (; mine != 0; mine &= mine - 1) {
                        const int k = k0 + __builtin_ctz(mine);
                        p.z_out[(int64_t)t * p.K + k] = stage[row * Tile::kLd + ids[k] - col0];
                    }
                    lds_fence();
                }
            } else if constexpr (kMode == kHeadGrad) {
                if constexpr (kPlanes) planes_back(j, t);
                const int t_in = min(t, q_rows - 1);
                const float4 rc = p.row_const[t_in];
                const int own = __float_as_int(rc.z);
#pragma unroll
                for (int i = 0; i < kBP; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = t < q_rows ? rc.y * __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], p.c1, -rc.x)) : 0.0f;
                if (ragged) {
#pragma unroll
                    for (int i = 0; i < kBP; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = col0 + 16 * i + 4 * h + e >= p_end ? 0.0f : acc[i][j][e];
                }
                to_lds(j);
                lds_fence();
                const int there = t < q_rows ? min(kCols, p_end - col0) : 0;
                auto subtract = [&](int c, float w) { stage[row * Tile::kLd + c] = fmaf(-w, rc.y, stage[row * Tile::kLd + c]); };
                if (!p.wanted) {
                    const int c = own - p.v0 - col0;
                    if (c >= 0 && c < there && (c >> 2 & 3) == h) subtract(c, 1.0f);
                } else {
                    const int64_t at = (int64_t)own * p.K;
                    for (int k0 = 0; k0 < p.K; k0 += 32) {
                        uint32_t mine = own_tokens(p.ids + at, k0, p.v0 + col0, there);
                        if (!__any(mine != 0)) continue;
                        mine |= __shfl_xor(mine, 16, kWave);           // all of the row's; each lane then deals with its own columns, in order
                        mine |= __shfl_xor(mine, 32, kWave);
                        for (; mine != 0; mine &= mine - 1) {
                            const int k = k0 + __builtin_ctz(mine), c = p.ids[at + k] - p.v0 - col0;
                            if ((c >> 2 & 3) == h) subtract(c, p.wanted[at + k]);
                        }
                    }
                }
                lds_fence();
                constexpr int kLanes = kCols / 8, kRowsAtOnce = 64 / kLanes;      // 16 bytes of G a lane
#pragma unroll
                for (int r0 = 0; r0 < 16; r0 += kRowsAtOnce) {
                    const int r = r0 + lane / kLanes, c = lane % kLanes * 8, tr = t - row + r;
                    if (r >= 16 || tr >= q_rows) continue;
                    const f32x4 a = *(lds_f32x4*)(stage + r * Tile::kLd + c), b = *(lds_f32x4*)(stage + r * Tile::kLd + c + 4);
                    char* dst = p.g_out + (int64_t)tr * p.g_row_bytes + (int64_t)(col0 + c) * 2;
                    *reinterpret_cast<u32x4*>(dst) = u32x4{head_round2<DT>(a[0], a[1]), head_round2<DT>(a[2], a[3]), head_round2<DT>(b[0], b[1]), head_round2<DT>(b[2], b[3])};
                    const int64_t plane = p.stacked ? q_rows * p.g_row_bytes : p.g_plane_bytes;
                    if (plane) {
                        f32x4 x, y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[e] = (a[e] - head_rounded<DT>(a[e])) * (kPlanes ? kHeadLow : 1.0f);
                            y[e] = (b[e] - head_rounded<DT>(b[e])) * (kPlanes ? kHeadLow : 1.0f);
                        }
                        *reinterpret_cast<u32x4*>(dst + plane) = u32x4{head_round2<DT>(x[0], x[1]), head_round2<DT>(x[2], x[3]), head_round2<DT>(y[0], y[1]), head_round2<DT>(y[2], y[3])};
                    }
                }
                lds_fence();
            } else if constexpr (kMode == kHeadRows) {
                if (t < q_rows) {
                    float* dst = p.acc_out + slice * p.acc_slice + (int64_t)t * p.acc_ld;
#pragma unroll
                    for (int i = 0; i < kBP; ++i) {
                        const int c = col0 + 16 * i + 4 * h;
                        if (c >= p.acc_ld) continue;
                        f32x4* at = reinterpret_cast<f32x4*>(dst + c);
                        *at = p.accumulate ? acc[i][j] + *at : acc[i][j];
                    }
                }
            } else {
                if (p.acc_out) {                           // a k slice's part, as for dx
                    if (t < q_rows) {
                        float* dst = p.acc_out + slice * p.acc_slice + (int64_t)t * p.acc_ld;
#pragma unroll
                        for (int i = 0; i < kBP; ++i)
                            if (col0 + 16 * i + 4 * h < p.acc_ld) *reinterpret_cast<f32x4*>(dst + col0 + 16 * i + 4 * h) = acc[i][j];
                    }
                    continue;
                }
                const int shift = -p.ctl->dw_exp;
                auto back = [shift](f32x4 v) { return OutDT == kBF16 ? v : head_shifted(v, shift); };      // (bf16: G has no scale)
                constexpr int kBytes = Storage<OutDT>::kBytes;
                char* dst = p.out + (int64_t)t * p.out_row_elems * kBytes;
                if (p.out_aligned) {
                    if constexpr (kBytes == 4) {
#pragma unroll
                        for (int i = 0; i < kBP; ++i) {
                            const int c = col0 + 16 * i + 4 * h;
                            if (t < q_rows && c < p.p_rows) *reinterpret_cast<f32x4*>(dst + c * 4) = back(acc[i][j]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kBP; i += 2) {
                            const f32x4 a = back(acc[i][j]), b = back(acc[i + 1][j]);
                            const u32x4 v = head_gather8(head_round2<OutDT>(a[0], a[1]), head_round2<OutDT>(a[2], a[3]), head_round2<OutDT>(b[0], b[1]), head_round2<OutDT>(b[2], b[3]));
                            const int c = col0 + 16 * i + 8 * h;
                            if (t < q_rows && c < p.p_rows) *reinterpret_cast<u32x4*>(dst + c * 2) = v;
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kBP; ++i) {
                        const f32x4 v = back(acc[i][j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = col0 + 16 * i + 4 * h + e;
                            if (t < q_rows && c < p.p_rows) head_put<OutDT>(dst, c, v[e]);
                        }
                    }
                }
            }
        }
        if constexpr (kMode == kHeadStats && Tile::kJoined) {
            __syncthreads();
            const int r = threadIdx.x;
            if (r < Tile::kQ && q0 + r < q_rows) {
                float m = -INFINITY, s = 0.0f;
#pragma unroll
                for (int w = 0; w < Tile::kWP; ++w) m = fmaxf(m, joined[w * Tile::kQ + r][0]);
#pragma unroll
                for (int w = 0; w < Tile::kWP; ++w) s += joined[w * Tile::kQ + r][1] * __builtin_amdgcn_exp2f((joined[w * Tile::kQ + r][0] - (m == -INFINITY ? 0.0f : m)) * p.c1);
                p.part[(int64_t)(p0 / p.pitch) * q_rows + q0 + r] = float2{m, s};
            }
        }
    };

    const int xcd = blockIdx.x & 7;
    int at = blockIdx.x >> 3;
    if (!head_item(xcd, at, tiles_q, p.tiles_p, p.k_slices, tq, tp, slice)) return;
    set_item();
    issue_first();
    if constexpr (kLoops<kMode, Tile>) {
        for (;;) {
            k_loop();
            const int done_q0 = q0, done_p0 = p0, done_end = p_end, done_slice = slice;
            at += gridDim.x >> 3;
            const bool more = head_item(xcd, at, tiles_q, p.tiles_p, p.k_slices, tq, tp, slice);
            if (more) {
                set_item();
                issue_first();
            }
            results(done_q0, done_p0, done_end, done_slice);
            if (!more) break;
        }
    } else {
        k_loop();
        results(q0, p0, p_end, slice);
    }
}

}  // namespace tide
