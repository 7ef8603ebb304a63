// Gradients of the expert layer: matrix products grouped by expert, by its rows
//   dx[r][h] = sum_n dy[r][n] w[e][n][h]          (tiles of rows x hidden elements, a walk over the output features)
// and by its weights
//   dw[e][n][h] = sum_r dy[r][n] x[r][h]          (tiles of output features x hidden elements, a walk over the expert's rows).
// In both an operand's elements lie the other way round than the matrix instructions take them: along the axis that stays, not along
// the one that is summed over.
#include "monta_internal.hpp"

#include <algorithm>

namespace monta {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct GradArgs {
    ExpertArgs a;           // lo, hi of the experts' rows, E, H, N, max_rows
    const void *dy, *x, *w;
    void *dx, *dw;
    bool stream_dw;         // dw goes past the cache
};

// Tile of dw of workgroup `block`, numbered like those of find_row_tile; e < 0: none.
template <int BR>
__device__ __forceinline__ RowTile find_weight_tile(const ExpertArgs &a, int nct, uint32_t block)
{
    const uint32_t L = (uint32_t)tile_number(block);
    RowTile t;
    const int tiles = (a.N + BR - 1) / BR;
    const uint32_t per = (uint32_t)tiles * (uint32_t)nct, e = L / per;         // per: at most 2^14 squared
    if (e >= (uint32_t)a.E) return t;
    t.e = (int)e;
    place_in_panels(t, L - e * per, tiles, nct);
    t.row0 = max(a.lo[e], 0);
    t.row_end = max(t.row0, min(a.hi_base[e] + a.hi_len[e], a.max_rows));
    return t;
}

template <bool DW, int BR, bool RAGGED_LAST>
__device__ __forceinline__ RowTile find_grad_tile(const ExpertArgs &a, int nct, uint32_t block, int lane, int *scratch)
{
    static_assert(!DW || !RAGGED_LAST, "all tiles of dw are whole walks");
    if constexpr (DW) return find_weight_tile<BR>(a, nct, block);
    else return find_row_tile<BR, RAGGED_LAST>(a, nct, block, lane, scratch);
}

// --------------------------------------------------------------------------------------------- bf16
//
// Steps of 64 elements of the summed axis.  An operand whose elements lie along that axis ("flat": dy in dx) is kept in LDS as rows of
// 128 bytes, piece c of row r at position c ^ ((r / 2) % 8), and read 16 bytes at a time.  One that lies across it ("deep") is kept as it
// comes, 64 rows of C elements, and read by the transposing LDS read: 16 lanes hand in 4 rows of 16 elements and get a column of 4 each;
// two of them are the 8 elements of an MFMA's fragment.  Its swizzle keeps the 8 rows of 32 bytes that half a wave reads (rows 8 g + j, g = 0, 1,
// j = 0..3; rows of 256 bytes or more begin on the same bank, of 128 every second) in different banks: the 32-byte segment s of row k sits at
// s ^ f(k).
template <int C>
__device__ __forceinline__ constexpr int deep_swizzle(int k)
{
    static_assert(C == 64 || C >= 128, "deep operand: width");
    if constexpr (C == 64) return ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
    else return (k & 3) | ((k >> 3) & 1) << 2;
}

// Where lane `lane` of the load of chunk c (1 KiB of LDS) of a deep operand of C elements finds its 16 bytes: the position is fixed by the
// instruction, so the swizzle is applied here.  `exist`: elements of a row from the tile's first on.
template <int C>
__device__ __forceinline__ uint32_t deep_at(int c, int lane, uint32_t pitch, int exist)
{
    constexpr int per = 2 * C / 16;
    const int k = (c * 64 + lane) / per, p = lane % per, from = ((p >> 1) ^ deep_swizzle<C>(k)) * 2 + (p & 1);
    return from * 8 < exist ? (uint32_t)k * pitch + (uint32_t)from * 16 : kOutOfRange;
}

// Half of the 8 elements along the summed axis of a fragment: rows k .. k+3 of a deep operand, or k+4 .. k+7 (4 rows further on).
// __restrict__: without alias information on the read the compiler waits for every outstanding load to LDS before it.
[[maybe_unused]] __device__ __forceinline__ s16x4 read_deep(lds_s16x4 *__restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }
[[maybe_unused]] __device__ __forceinline__ bf16x8 whole_fragment(s16x4 lo, s16x4 hi) { return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)); }

// A tile of 32 RB x 32 CB of the output, rows (of dx) or output features (of dw) x hidden elements, by 2 x 2 waves of 16 RB x 16 CB.
template <int RB, int CB>
struct GradShape {
    static constexpr int BR = 32 * RB, BC = 32 * CB;
    static constexpr int kRowStage = BR * 128, kColStage = BC * 128, kSink = 2 * (kRowStage + kColStage), kLdsBytes = kSink + 1024;
    static_assert((RB == 4 || RB == 8) && RB == CB && kLdsBytes <= 160 * 1024, "gradient tile: shape");
};

// A step's operands go straight to LDS while the step before it is multiplied: two stages, the loads of step s + 2 issued into the place of
// s under the second half of s, when every wave has read all of s.  (Through registers, a step ahead of LDS: 8192 rows x 8192 x 8192, two
// experts, dw 898 us; so 820 to 855, 1.29 to 1.34 PFLOP/s; without any loads 772.)  Fragments come in two sets: the second half of a step is read under the MFMAs of the
// first, the first half of the next step under those of the second.  One barrier per step, between the halves.  A step's time covers an L2
// hit but no miss, so each workgroup also touches, a step ahead of the loads, one word per line of its share of the tiles that it shares with
// the others on its XCD.
// A tile of dx of at most XR rows x CW hidden elements: so little arithmetic per step that the step is as long as its loads take to arrive.
// NST stages, the loads of NST - 1 steps in flight; 4 waves, each all rows x CW / 4 columns.  A step's fragments are read at its start.  Every wave issues
// the same number of loads per step, also past the end (out of range: no traffic), because the wait for a stage counts the younger loads.
template <int XR, int CW, int NST>
struct GradShort {
    static constexpr int kStage = (XR + CW) * 128, kLdsBytes = NST * kStage;
    static constexpr int kLoadsR = XR / 32, kLoadsC = CW / 32, kYounger = (NST - 2) * (kLoadsR + kLoadsC);      // 1 KiB loads per wave and step
    static constexpr int kWait = 0x0070 | (kYounger & 15) | ((kYounger >> 4) << 14);                         // vmcnt(kYounger), lgkmcnt(0)
    static constexpr int RB = XR / 16, CB = CW / 64;
    static_assert(XR % 32 == 0 && (CW == 64 || CW == 128) && NST >= 3 && kYounger < 64, "short gradient tile: shape");
};

template <int XR, int CW, int NST>
__device__ __forceinline__ void grad_short_tile(const GradArgs &b, int e, int row0, int row_end, int col0, unsigned char *lds)
{
    using G = GradShort<XR, CW, NST>;
    const ExpertArgs &a = b.a;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));      // share nothing with the caller's other path, which has no register left to keep it in
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const uint32_t pitch_c = (uint32_t)a.H * 2, pitch_r = (uint32_t)a.N * 2;
    const char *const from_c = static_cast<const char *>(b.w) + ((int64_t)e * a.N * a.H + col0) * 2;
    const auto rows = make_rsrc(static_cast<const char *>(b.dy) + (int64_t)row0 * pitch_r, (uint32_t)(row_end - row0) * pitch_r);
    const int nsteps = (a.N + 63) / 64;
    uint32_t at_c[G::kLoadsC], at_r[G::kLoadsR];
    int p_r[G::kLoadsR];
#pragma unroll
    for (int q = 0; q < G::kLoadsC; ++q) at_c[q] = deep_at<CW>(wave * G::kLoadsC + q, lane, pitch_c, a.H - col0);
#pragma unroll
    for (int q = 0; q < G::kLoadsR; ++q) {
        const int row = (wave * G::kLoadsR + q) * 8 + (lane >> 3);
        p_r[q] = (lane & 7) ^ ((row >> 1) & 7);
        at_r[q] = (uint32_t)row * pitch_r + p_r[q] * 16;
    }
    auto issue = [&](int step, int slot) {
        const int left = __builtin_amdgcn_readfirstlane(min(max(a.N - step * 64, 0), 64));
        const auto cols = make_rsrc(from_c + (int64_t)step * 64 * pitch_c, left > 0 ? (uint32_t)left * pitch_c - (uint32_t)col0 * 2u : 0u);
        unsigned char *const base = lds + slot * G::kStage;
#pragma unroll
        for (int q = 0; q < G::kLoadsC; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(cols, (lds_void *)(base + XR * 128 + (wave * G::kLoadsC + q) * 1024), 16, at_c[q], 0, 0, 0);
#pragma unroll
        for (int q = 0; q < G::kLoadsR; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void *)(base + (wave * G::kLoadsR + q) * 1024), 16,
                                                     p_r[q] * 8 < left ? at_r[q] + (uint32_t)step * 128u : kOutOfRange, 0, 0, 0);
    };
    f32x4 acc[G::RB][G::CB];
#pragma unroll
    for (int i = 0; i < G::RB; ++i)
#pragma unroll
        for (int j = 0; j < G::CB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    const int kl = 8 * g + (m >> 2), sw = deep_swizzle<CW>(kl);
    const unsigned char *const pc = lds + XR * 128 + kl * (2 * CW) + (m & 3) * 8, *const pr = lds + m * 128;
    const int nb = (row_end - row0 + 15) / 16;                     // 16-row blocks with rows of the segment
#pragma unroll
    for (int q = 0; q < NST - 1; ++q) issue(q, q);
    // with at most half of the row blocks in use only those are multiplied
    auto run = [&](auto blocks) {
        constexpr int BLOCKS = decltype(blocks)::value;
        int slot = 0;
        for (int step = 0; step < nsteps; ++step) {
            __builtin_amdgcn_s_waitcnt(G::kWait);                  // stage `step` has landed; this wave's reads of the one before are done
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            issue(step + NST - 1, slot == 0 ? NST - 1 : slot - 1); // where stage step - 1 was
            const int at = slot * G::kStage;
            bf16x8 fr[2][BLOCKS], fc[2][G::CB];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                for (int j = 0; j < G::CB; ++j) {
                    const unsigned char *const p = pc + at + ks * 64 * CW + ((wave * G::CB + j) ^ sw) * 32;
                    const s16x4 lo = read_deep((lds_s16x4 *)(p)), hi = read_deep((lds_s16x4 *)(p + 8 * CW));
                    fc[ks][j] = whole_fragment(lo, hi);
                }
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i) fr[ks][i] = *reinterpret_cast<const bf16x8 *>(pr + at + ((4 * ks + g) ^ ((m >> 1) & 7)) * 16 + i * 2048);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int j = 0; j < G::CB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[ks][j], fr[ks][i], acc[i][j], 0, 0, 0);
            slot = slot == NST - 1 ? 0 : slot + 1;
        }
    };
    if (2 * nb <= G::RB) run(std::integral_constant<int, G::RB / 2>{});
    else run(std::integral_constant<int, G::RB>{});
    __bf16 *const out = static_cast<__bf16 *>(b.dx);
#pragma unroll
    for (int i = 0; i < G::RB; ++i) {
        const int64_t r = row0 + i * 16 + m;
        if (r < row_end) {
#pragma unroll
            for (int j = 0; j < G::CB; ++j) {
                const int h = col0 + wave * (CW / 4) + j * 16 + 4 * g;
                if (h < a.H) {
                    bf16x4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = (__bf16)acc[i][j][v];
                    *reinterpret_cast<bf16x4 *>(out + r * a.H + h) = o;
                }
            }
        }
    }
}

// The rows of a ragged tile of dx are split evenly between the two row halves: the loop is compiled for RB / 2 to RB blocks of 16
// rows each, so that only rows in use are requested, read and multiplied.
template <bool DW, int RB, int CB, bool RAGGED_LAST>
__device__ __forceinline__ void grad_bf16_tile(const GradArgs &b, uint32_t block, unsigned char *lds)
{
#if defined(__HIP_DEVICE_COMPILE__)         // the matrix instruction is written out: nothing for the host pass to parse
    using G = GradShape<RB, CB>;
    constexpr int BR = G::BR, BC = G::BC;
    const ExpertArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int wr = wave >> 1, wc = wave & 1;
    const RowTile t = find_grad_tile<DW, BR, RAGGED_LAST>(a, (a.H + BC - 1) / BC, block, lane, reinterpret_cast<int *>(lds));
    const int e = __builtin_amdgcn_readfirstlane(t.e);
    if (e < 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(t.row0), row_end = __builtin_amdgcn_readfirstlane(t.row_end);
    const int64_t H = a.H, N = a.N;
    // Tiles of dx of at most 64 rows last as long as their weights take to arrive: four stages of them on their way.  Those of RAGGED_LAST come in
    // halves of 128 columns, twice the workgroups with twice the loads; in place both halves follow one another (dx of 4096 x 7168 x 2048 over 64
    // experts, top-8, most of which have few rows: 600 us, as 256 x 256 620).
    if constexpr (!DW && RB == 8) {
        if (row_end - row0 <= kShortTileRows) {
            constexpr int kCols = RAGGED_LAST ? 128 : BC;
            const int from = __builtin_amdgcn_readfirstlane(t.ct) * kCols;
            for (int c = from; c < min(from + kCols, a.H); c += 128) {
                grad_short_tile<kShortTileRows, 128, 5>(b, e, row0, row_end, c, lds);
                __builtin_amdgcn_s_waitcnt(0x0070);                // the loads past the end have come back
                __syncthreads();
            }
            return;
        }
    }
    // out0: first output feature of a tile of dw
    const int col0 = __builtin_amdgcn_readfirstlane(t.ct) * BC, out0 = DW ? __builtin_amdgcn_readfirstlane(t.rt) * BR : 0;
    const int depth = DW ? row_end - row0 : a.N;                   // of the summed axis
    const int nsteps = (depth + 63) / 64;

    // columns: x (dw) or w (dx), deep in both; rows: dy, deep (dw) or flat (dx).  Descriptors of deep operands begin at a step's first row.
    const uint32_t pitch_c = (uint32_t)a.H * 2, pitch_r = (uint32_t)a.N * 2;
    const char *from_c = static_cast<const char *>(DW ? b.x : b.w) + (DW ? (int64_t)row0 * H : (int64_t)e * N * H) * 2 + (int64_t)col0 * 2;
    const char *from_r = static_cast<const char *>(b.dy) + ((int64_t)row0 * N + out0) * 2;
    const auto flat = make_rsrc(from_r, DW ? 0u : (uint32_t)(row_end - row0) * pitch_r);
    auto records = [&](int step, uint32_t pitch, int cut) {       // rows of a deep operand in the step, none past the end
        const int left = min(max(depth - step * 64, 0), 64);       // a clamp in one vector instruction: back into a scalar register
        return (uint32_t)__builtin_amdgcn_readfirstlane(left > 0 ? left * (int)pitch - cut * 2 : 0);
    };
    auto cols_of = [&](int step) { return make_rsrc(from_c + (int64_t)step * 64 * pitch_c, records(step, pitch_c, col0)); };
    auto rows_of = [&](int step) { return DW ? make_rsrc(from_r + (int64_t)step * 64 * pitch_r, records(step, pitch_r, out0)) : flat; };
    // the early touches: thread `tid` has line tid of a step's 64 rows of BC / 64 lines (deep) or of its rows (flat)
    constexpr int kLinesC = BC / 64, kLinesR = BR / 64;
    const int side = __builtin_amdgcn_readfirstlane(t.side), share = __builtin_amdgcn_readfirstlane(t.share), ct = __builtin_amdgcn_readfirstlane(t.ct);
    const uint32_t touch_c = tid < 64 * kLinesC && tid * side / (64 * kLinesC) == share && col0 + tid % kLinesC * 64 < a.H
                                 ? (uint32_t)(tid / kLinesC) * pitch_c + (uint32_t)(tid % kLinesC) * 128u : kOutOfRange;
    const bool my_rows = (tid >> 6) == (ct & 3);
    const uint32_t touch_r = !my_rows ? kOutOfRange : DW ? (tid < 64 * kLinesR && out0 + tid % kLinesR * 64 < a.N ? (uint32_t)(tid / kLinesR) * pitch_r + (uint32_t)(tid % kLinesR) * 128u : kOutOfRange)
                                                     : (tid < BR ? (uint32_t)tid * pitch_r : kOutOfRange);
    auto touch = [&](int step) {
        lds_void *const sink = (lds_void *)(lds + G::kSink + wave * 256);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(cols_of(step), sink, 4, touch_c, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of(step), sink, 4, DW || step * 64 >= a.N ? (DW ? touch_r : kOutOfRange) : touch_r + (touch_r == kOutOfRange ? 0u : (uint32_t)step * 128u), 0, 0, 0);
    };
    uint32_t at_c[CB];
#pragma unroll
    for (int q = 0; q < CB; ++q) at_c[q] = deep_at<BC>(wave * CB + q, lane, pitch_c, a.H - col0);
    unsigned char *const lds_r = lds, *const lds_c = lds + 2 * G::kRowStage;
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    f32x4 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    // no instruction near it reads the accumulator: the next MFMA on the same one is half a step away, and the epilogue waits first
    bf16x8 fr[2][RB], fc[2][CB];
    auto mma = [&](int set, int i, int j) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(fc[set][j]), "v"(fr[set][i])); };

    // All steps, NB row blocks per half.
    auto run = [&](auto nbc) {
        constexpr int NB = decltype(nbc)::value;
        // this lane's place in a deep operand: row 8 g + m / 4, quarter m % 4 of a segment
        const int kl = 8 * g + (m >> 2), sw = deep_swizzle<BC>(kl);      // the same for both widths
        const unsigned char *const fc0 = lds_c + kl * (2 * BC) + (m & 3) * 8;
        const unsigned char *const fr0 = DW ? lds_r + kl * (2 * BR) + (m & 3) * 8 : lds_r + (wr * 16 * NB + m) * 128;
        // Fragment r of half `ks` of the step in `stage`: those of the columns, then those of the rows.  Part 0 and part 1 of a deep one; a flat
        // one is read whole as part 0.
        s16x4 lo;
        auto read = [&](int set, int stage, int ks, int r, int part) {
            if (r < CB || DW) {
                const int pitch = r < CB ? 2 * BC : 2 * BR, seg = r < CB ? wc * CB + r : wr * RB + r - CB;
                const unsigned char *const p = r < CB ? fc0 + stage * G::kColStage : fr0 + stage * G::kRowStage;
                const s16x4 v = read_deep((lds_s16x4 *)(p + ks * 32 * pitch + (seg ^ sw) * 32 + part * 4 * pitch));
                if (part == 0) lo = v;
                else if (r < CB) fc[set][r] = whole_fragment(lo, v);
                else fr[set][r - CB] = whole_fragment(lo, v);
            } else if (part == 0) {
                fr[set][r - CB] = *reinterpret_cast<const bf16x8 *>(fr0 + stage * G::kRowStage + ((4 * ks + g) ^ ((m >> 1) & 7)) * 16 + (r - CB) * 2048);
            }
        };
        uint32_t at_r[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int c = wave * NB + q, row = c * 8 + (lane >> 3), p = (lane & 7) ^ ((row >> 1) & 7);
            at_r[q] = DW ? deep_at<BR>(c, lane, pitch_r, a.N - out0) : (uint32_t)row * pitch_r + p * 16;
        }
        auto issue_c = [&](__amdgpu_buffer_rsrc_t r, int stage, int q) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds_c + stage * G::kColStage + (wave * CB + q) * 1024), 16, at_c[q], 0, 0, 0);
        };
        auto issue_r = [&](__amdgpu_buffer_rsrc_t r, int step, int stage, int q) {
            uint32_t at = at_r[q];
            if (!DW) {
                const int p = (lane & 7) ^ ((((wave * NB + q) * 8 + (lane >> 3)) >> 1) & 7);
                at = step * 64 + p * 8 < a.N ? at + (uint32_t)step * 128u : kOutOfRange;
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds_r + stage * G::kRowStage + (wave * NB + q) * 1024), 16, at, 0, 0, 0);
        };
        // Half a step: NB x CB MFMAs on fragment set `set`; evenly between them the reads of the other set's fragments and, if `refill`,
        // the loads of step `step`.  One wave has a SIMD to itself: an instruction issues in 4 clocks, an MFMA takes 16, so up to three others
        // behind each cost nothing (in bursts behind every fourth 1 % more time).
        constexpr int kMfmas = NB * CB, kReads = NB + CB;
        auto half_step = [&](int set, int stage, int ks, auto refill, int step) {
            constexpr int each = decltype(refill)::value ? 3 : 2, actions = each * kReads;
            const auto rc = cols_of(step), rr = rows_of(step);
#pragma unroll
            for (int n = 0; n < kMfmas; ++n) {
#pragma unroll
                for (int k = n * actions / kMfmas; k < (n + 1) * actions / kMfmas; ++k) {
                    const int r = k / each, what = k % each;
                    if (what < 2) read(set ^ 1, stage, ks, r, what);
                    else if (r < CB) issue_c(rc, step & 1, r);
                    else issue_r(rr, step, step & 1, r - CB);
                }
                mma(set, n / CB, n % CB);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const auto rc = cols_of(step), rr = rows_of(step);
#pragma unroll
            for (int q = 0; q < CB; ++q) issue_c(rc, step, q);
#pragma unroll
            for (int q = 0; q < NB; ++q) issue_r(rr, step, step, q);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70 | (kReads & 15) | (kReads >> 4 << 14));       // stage 0: younger are the loads of stage 1
        touch(2);
        barrier();
#pragma unroll
        for (int r = 0; r < 2 * kReads; ++r) read(0, 0, 0, r / 2, r % 2);
        for (int s = 0; s < nsteps; ++s) {
            half_step(0, s & 1, 1, std::false_type{}, 0);
            __builtin_amdgcn_s_waitcnt(0x0070 | 2);                // this wave has read all of stage s, its part of stage s + 1 has landed: younger are two touches
            barrier();
            half_step(1, (s & 1) ^ 1, 0, std::true_type{}, s + 2);
            touch(s + 3);
        }
    };
    int nb = RB;
    if constexpr (DW) {
        if (nsteps > 0) run(std::integral_constant<int, RB>{});
    } else {
        nb = max((row_end - row0 + 31) / 32, (RB + 1) / 2);
        if (RB == 8 && nb == 7) run(std::integral_constant<int, (RB == 8 ? 7 : RB)>{});
        else if (RB == 8 && nb == 6) run(std::integral_constant<int, (RB == 8 ? 6 : RB)>{});
        else if (RB == 8 && nb == 5) run(std::integral_constant<int, (RB == 8 ? 5 : RB)>{});
        else if (RB == 4 && nb == 3) run(std::integral_constant<int, (RB == 4 ? 3 : RB)>{});
        else if (RB > 1 && nb == RB / 2) run(std::integral_constant<int, (RB > 1 ? RB / 2 : RB)>{});
        else run(std::integral_constant<int, RB>{});
    }
    asm volatile("s_nop 15\n\ts_nop 15");                          // the last MFMAs' results
    __builtin_amdgcn_sched_barrier(0);

    // acc[i][j][v]: row 16 i + lane % 16 of the wave's rows, hidden element 16 j + 4 (lane / 16) + v of its columns.  Through LDS, block of
    // 16 rows by block, so that rows leave as whole pieces of 16 bytes, 32 CB bytes of each side by side.  (8 bytes a lane straight from the registers:
    // 268 MB of weights' gradients in 101 us.)  dw is read by nobody soon and is streamed past the cache, where it would drive out the weights: both
    // gradients of 128 rows x 4096 x 4096, 8 experts, 153 and 125 us, of 1024 rows 203 and 190.  Where it leaves in
    // parts of half lines only with rows enough (at its flag).  dx gains 1 %, but is read next.
    __builtin_amdgcn_s_waitcnt(0x0070);                            // nor written: the loads past the end have come back
    barrier();                                                     // the stages are not read any more
    constexpr int kOutPitch = 32 * CB + 16;                        // 16 bytes of padding: the 16 rows that a store of 8 bytes a lane hits begin on different banks
    unsigned char *const own = lds + wave * (16 * kOutPitch);
    static_assert(4 * 16 * kOutPitch <= G::kLdsBytes, "gradient tile: room for a block of rows per wave");
    char *const out = static_cast<char *>(DW ? b.dw : b.dx) + ((DW ? (int64_t)e * N * H : 0) + col0 + wc * 16 * CB) * 2;
    const int l2 = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // asked for again: kept through the loop it would be spilled
    auto leave = [&](auto past_cache) {                            // a question at each store would cost dw of few rows a third
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            if (i >= nb) break;
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                bf16x4 o;
#pragma unroll
                for (int v = 0; v < 4; ++v) o[v] = (__bf16)acc[i][j][v];
                *reinterpret_cast<bf16x4 *>(own + (l2 & 15) * kOutPitch + j * 32 + (l2 >> 4) * 8) = o;
            }
            constexpr int kLanes = 2 * CB, kRows = 64 / kLanes;        // lanes per row, rows per store
#pragma unroll
            for (int q = 0; q < 16 / kRows; ++q) {
                const int row = q * kRows + l2 / kLanes, p = l2 % kLanes;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(own + row * kOutPitch + p * 16);
                const int64_t r = (DW ? out0 : row0) + wr * 16 * nb + i * 16 + row;
                if (r < (DW ? a.N : row_end) && col0 + wc * 16 * CB + p * 8 < a.H) {
                    u32x4 *const to = reinterpret_cast<u32x4 *>(out + r * H * 2 + p * 16);
                    if constexpr (DW && decltype(past_cache)::value) __builtin_nontemporal_store(v, to);
                    else *to = v;
                }
            }
        }
    };
    if (DW && b.stream_dw) leave(std::true_type{});
    else leave(std::false_type{});
#else
    (void)b;
    (void)block;
    (void)lds;
#endif
}

// A tile of dw of 64 x 64 for outputs of few tiles: the four waves share the rows of the expert instead of the tile, steps of 32 rows in
// turn, each with NST stages of its own and no barrier, and their sums are added at the end, in the order of the waves.  Twice the operand
// bytes per product of a 128 x 128 tile, but four times the workgroups and half the walk.
template <int NST>
struct GradSlim {
    static constexpr int kStage = 2 * 64 * 64, kLdsBytes = 4 * NST * kStage, kPitch = 64 * 4 + 16;
    static constexpr int kLoads = 8, kYounger = (NST - 2) * kLoads;
    static constexpr int kWait = 0x0070 | (kYounger & 15) | ((kYounger >> 4) << 14);                         // vmcnt(kYounger), lgkmcnt(0)
    static_assert(NST >= 2 && kYounger < 64 && 4 * 64 * kPitch <= 160 * 1024, "slim gradient tile: shape");
    static constexpr int kLds = kLdsBytes > 4 * 64 * kPitch ? kLdsBytes : 4 * 64 * kPitch;
};

template <int NST>
__device__ __forceinline__ void grad_slim_tile(const GradArgs &b, const RowTile &t, unsigned char *lds)
{
    using G = GradSlim<NST>;
    const ExpertArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int e = __builtin_amdgcn_readfirstlane(t.e), row0 = __builtin_amdgcn_readfirstlane(t.row0), depth = __builtin_amdgcn_readfirstlane(t.row_end) - row0;
    const int64_t H = a.H, N = a.N;
    const int col0 = __builtin_amdgcn_readfirstlane(t.ct) * 64, out0 = __builtin_amdgcn_readfirstlane(t.rt) * 64;
    const uint32_t pitch_c = (uint32_t)a.H * 2, pitch_r = (uint32_t)a.N * 2;
    const char *const from_c = static_cast<const char *>(b.x) + ((int64_t)row0 * H + col0) * 2;
    const char *const from_r = static_cast<const char *>(b.dy) + ((int64_t)row0 * N + out0) * 2;
    uint32_t at_c[4], at_r[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) at_c[q] = deep_at<64>(q, lane, pitch_c, a.H - col0), at_r[q] = deep_at<64>(q, lane, pitch_r, a.N - out0);
    unsigned char *const own = lds + wave * (NST * G::kStage);
    auto issue = [&](int step, int slot) {
        const int first = (step * 4 + wave) * 32, left = __builtin_amdgcn_readfirstlane(min(max(depth - first, 0), 32));
        const auto cols = make_rsrc(from_c + (int64_t)first * pitch_c, left > 0 ? (uint32_t)left * pitch_c - (uint32_t)col0 * 2u : 0u);
        const auto rows = make_rsrc(from_r + (int64_t)first * pitch_r, left > 0 ? (uint32_t)left * pitch_r - (uint32_t)out0 * 2u : 0u);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(cols, (lds_void *)(own + slot * G::kStage + q * 1024), 16, at_c[q], 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void *)(own + slot * G::kStage + 4096 + q * 1024), 16, at_r[q], 0, 0, 0);
        }
    };
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    const int kl = 8 * g + (m >> 2), sw = deep_swizzle<64>(kl);
    const unsigned char *const from = own + kl * 128 + (m & 3) * 8;
    bf16x8 fc[2][4], fr[2][4];
    // reads the fragments of stage `slot` into set `set`
    auto read = [&](int set, int slot) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned char *const p = from + slot * G::kStage + (j ^ sw) * 32;
            const s16x4 cl = read_deep((lds_s16x4 *)(p)), ch = read_deep((lds_s16x4 *)(p + 512));
            const s16x4 rl = read_deep((lds_s16x4 *)(p + 4096)), rh = read_deep((lds_s16x4 *)(p + 4096 + 512));
            fc[set][j] = whole_fragment(cl, ch);
            fr[set][j] = whole_fragment(rl, rh);
        }
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[set][j], fr[set][i], acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int q = 0; q < NST; ++q) issue(q, q);
    __builtin_amdgcn_s_waitcnt(0x0f70 | ((NST - 1) * 8 & 15) | (((NST - 1) * 8) >> 4 << 14));        // stage 0
    asm volatile("" ::: "memory");
    read(0, 0);
    // past the end there are zeros, which a walk of an odd number of steps multiplies too
    const int nsteps = (depth + 127) / 128;
    int slot = 0;
    for (int step = 0; step < nsteps; step += 2) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            __builtin_amdgcn_s_waitcnt(G::kWait);                  // the next stage has landed; this one has been read
            asm volatile("" ::: "memory");
            issue(step + half + NST, slot);
            slot = slot == NST - 1 ? 0 : slot + 1;
            read(half ^ 1, slot);
            __builtin_amdgcn_sched_barrier(0);                     // left alone the reads come behind the products: 15 % more time
            multiply(half);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                            // the loads past the end have come back
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(lds);
    constexpr int kRow = G::kPitch / 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4 *>(sums + (wave * 64 + i * 16 + m) * kRow + j * 16 + 4 * g) = acc[i][j];
    __syncthreads();
    __bf16 *const out = static_cast<__bf16 *>(b.dw) + (int64_t)e * N * H;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int row = q * 32 + tid / 8, c = tid % 8 * 8;
        f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            lo += *reinterpret_cast<const f32x4 *>(sums + (w * 64 + row) * kRow + c);
            hi += *reinterpret_cast<const f32x4 *>(sums + (w * 64 + row) * kRow + c + 4);
        }
        bf16x8 o;
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] = (__bf16)lo[v], o[4 + v] = (__bf16)hi[v];
        if (out0 + row < a.N && col0 + c < a.H) *reinterpret_cast<bf16x8 *>(out + (int64_t)(out0 + row) * H + col0 + c) = o;
    }
}

// --------------------------------------------------------------------------------------------- fp32
//
// Tiles of BR x 64 by 2 x 2 waves, steps of 32 elements of the summed axis, NST stages straight to LDS, the loads of NST - 1 in flight.  A
// 32-bit element has nothing to be transposed with: a deep operand, 32 rows of BR or 64 elements, is read element by element, MFMA v of half a
// step taking rows 4 g + v of it (g the lane's group of 16), a flat one 16 bytes at a time, which are the same rows' elements.  Swizzles: flat as in
// bf16; deep, the 64-byte segment s of row k at s ^ (k / 4) % 4, so that the four groups' rows are in different banks.  What bounds it is the
// fp32 matrix rate, and with few steps the way to the first.  Two stages of 64 rows, 32 KiB or five workgroups a CU, do better than three,
// three a CU (both gradients, us: 1024 rows x 1024 x 1024, 8 experts 56 and 62, 600 x 2048 x 2048, 4 experts 109 and 116, 8192 x 1024 x 1024 310 and 312), but for 32 rows,
// whose walks are short of work (2 rows x 1024 x 1024 17 and 19): three, 36 KiB, which leave four workgroups a CU where dw goes out with them.
template <int BR, int NST>
struct GradShapeF32 {
    static constexpr int BC = 64, kStage = (BR + BC) * 128, kLdsBytes = NST * kStage;
    static constexpr int kLoadsR = BR / 32, kLoadsC = BC / 32, kYounger = (NST - 2) * (kLoadsR + kLoadsC);      // 1 KiB loads per wave and step
    static constexpr int kWait = 0x0070 | (kYounger & 15) | ((kYounger >> 4) << 14);                         // vmcnt(kYounger), lgkmcnt(0)
    static constexpr int RB = BR / 32;
    static_assert((BR == 32 || BR == 64) && NST >= 2 && kYounger < 64, "fp32 gradient tile: shape");
};

// as deep_at, for 32 rows of 64 fp32 elements
[[maybe_unused]] __device__ __forceinline__ uint32_t deep_at_f32(int c, int lane, uint32_t pitch, int exist)
{
    const int k = (c * 64 + lane) / 16, p = lane % 16, from = ((p >> 2) ^ ((k >> 2) & 3)) * 4 + (p & 3);
    return from * 4 < exist ? (uint32_t)k * pitch + (uint32_t)from * 16 : kOutOfRange;
}

template <bool DW, int BR, int NST>
__device__ __forceinline__ void grad_f32_tile(const GradArgs &b, const RowTile &t, unsigned char *lds)
{
    using G = GradShapeF32<BR, NST>;
    static_assert(!DW || BR == 64, "a deep operand has 64 elements");
    const ExpertArgs &a = b.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4, wr = wave >> 1, wc = wave & 1;
    const int e = __builtin_amdgcn_readfirstlane(t.e), row0 = __builtin_amdgcn_readfirstlane(t.row0), row_end = __builtin_amdgcn_readfirstlane(t.row_end);
    const int64_t H = a.H, N = a.N;
    const int col0 = __builtin_amdgcn_readfirstlane(t.ct) * G::BC, out0 = DW ? __builtin_amdgcn_readfirstlane(t.rt) * BR : 0;
    const int depth = DW ? row_end - row0 : a.N, nsteps = (depth + 31) / 32;
    const uint32_t pitch_c = (uint32_t)a.H * 4, pitch_r = (uint32_t)a.N * 4;
    const char *const from_c = static_cast<const char *>(DW ? b.x : b.w) + (DW ? (int64_t)row0 * H : (int64_t)e * N * H) * 4 + (int64_t)col0 * 4;
    const char *const from_r = static_cast<const char *>(b.dy) + ((int64_t)row0 * N + out0) * 4;
    const auto flat = make_rsrc(from_r, DW ? 0u : (uint32_t)(row_end - row0) * pitch_r);
    uint32_t at_c[G::kLoadsC], at_r[G::kLoadsR];
    int p_r[G::kLoadsR];
#pragma unroll
    for (int q = 0; q < G::kLoadsC; ++q) at_c[q] = deep_at_f32(wave * G::kLoadsC + q, lane, pitch_c, a.H - col0);
#pragma unroll
    for (int q = 0; q < G::kLoadsR; ++q) {
        const int c = wave * G::kLoadsR + q, row = c * 8 + (lane >> 3);
        p_r[q] = (lane & 7) ^ ((row >> 1) & 7);
        at_r[q] = DW ? deep_at_f32(c, lane, pitch_r, a.N - out0) : (uint32_t)row * pitch_r + p_r[q] * 16;
    }
    auto issue = [&](int step, int slot) {
        const int left = __builtin_amdgcn_readfirstlane(min(max(depth - step * 32, 0), 32));       // of the summed axis in this step, none past the end
        const auto cols = make_rsrc(from_c + (int64_t)step * 32 * pitch_c, left > 0 ? (uint32_t)left * pitch_c - (uint32_t)col0 * 4u : 0u);
        const auto deep = make_rsrc(from_r + (int64_t)step * 32 * pitch_r, DW && left > 0 ? (uint32_t)left * pitch_r - (uint32_t)out0 * 4u : 0u);
        unsigned char *const base = lds + slot * G::kStage;
#pragma unroll
        for (int q = 0; q < G::kLoadsC; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(cols, (lds_void *)(base + BR * 128 + (wave * G::kLoadsC + q) * 1024), 16, at_c[q], 0, 0, 0);
#pragma unroll
        for (int q = 0; q < G::kLoadsR; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(DW ? deep : flat, (lds_void *)(base + (wave * G::kLoadsR + q) * 1024), 16,
                                                     DW ? at_r[q] : p_r[q] * 4 < left ? at_r[q] + (uint32_t)step * 128u : kOutOfRange, 0, 0, 0);
    };
    f32x4 acc[G::RB][2];
#pragma unroll
    for (int i = 0; i < G::RB; ++i) acc[i][0] = acc[i][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < NST - 1; ++q) issue(q, q);
    // One wave's blocks of 16 rows and 16 columns that exist: at the edge of the output it multiplies only those, which leaves its SIMD to other
    // workgroups (10 experts of 516 x 516: the last of nine column tiles has four columns).
    const int rows_left = DW ? a.N - out0 - wr * (BR / 2) : row_end - row0 - wr * (BR / 2), cols_left = a.H - col0 - wc * 32;
    const int nr = min(max((rows_left + 15) / 16, 0), G::RB), nc = min(max((cols_left + 15) / 16, 0), 2);
    // A loop for each count: conditions in one loop, around the products or around their reads too, give the same bits and take longer (both gradients,
    // calls of one graph, us: 1155 x 516 x 516, 10 experts, top-3 40.6, 43.0 and 50.5; 256 x 516 x 516 20.8, 23.1 and 26.4; 64 x 68 x 1000, 16 experts
    // 16.5, 23.5 and 31.8; 1024 x 1024 x 1024, 8 experts, without edges, 102, 104 and 116).
    auto walk = [&](auto rows, auto columns) {
        constexpr int NR = decltype(rows)::value, NC = decltype(columns)::value;
        int slot = 0;
        for (int step = 0; step < nsteps; ++step) {
            __builtin_amdgcn_s_waitcnt(G::kWait);                  // stage `step` has landed; this wave's reads of the one before are done
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            issue(step + NST - 1, slot == 0 ? NST - 1 : slot - 1); // where stage step - 1 was
            const unsigned char *const base = lds + slot * G::kStage;
            slot = slot == NST - 1 ? 0 : slot + 1;
#pragma unroll
            for (int ks = 0; ks < (NR * NC > 0 ? 2 : 0); ++ks) {
                // row k = 16 ks + 4 g + v: (k / 4) % 4 = g
                f32x4 fr[NR > 0 ? NR : 1];
                float fc[NC > 0 ? NC : 1][4];
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    if constexpr (DW) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) fr[i][v] = *reinterpret_cast<const float *>(base + (16 * ks + 4 * g + v) * 256 + ((wr * 2 + i) ^ g) * 64 + m * 4);
                    } else {
                        const int row = wr * (BR / 2) + i * 16 + m;
                        fr[i] = *reinterpret_cast<const f32x4 *>(base + row * 128 + ((4 * ks + g) ^ ((m >> 1) & 7)) * 16);
                    }
                }
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) fc[j][v] = *reinterpret_cast<const float *>(base + BR * 128 + (16 * ks + 4 * g + v) * 256 + ((wc * 2 + j) ^ g) * 64 + m * 4);
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int i = 0; i < NR; ++i)
#pragma unroll
                        for (int j = 0; j < NC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fc[j][v], fr[i][v], acc[i][j], 0, 0, 0);
            }
        }
    };
    constexpr std::integral_constant<int, 0> none{};
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 2> two{};
    if (nr == 0 || nc == 0) walk(none, none);
    else if (G::RB == 2 && nr == 2 && nc == 2) walk(std::integral_constant<int, G::RB>{}, two);
    else if (G::RB == 2 && nr == 2) walk(std::integral_constant<int, G::RB>{}, one);
    else if (nc == 2) walk(one, two);
    else walk(one, one);
    float *const out = static_cast<float *>(DW ? b.dw : b.dx) + (DW ? (int64_t)e * N * H : 0);
#pragma unroll
    for (int i = 0; i < G::RB; ++i) {
        const int64_t r = (DW ? out0 : row0) + wr * (BR / 2) + i * 16 + m;
        if (r < (DW ? a.N : row_end)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = col0 + wc * 32 + j * 16 + 4 * g;
                if (h < a.H) *reinterpret_cast<f32x4 *>(out + r * H + h) = acc[i][j];
            }
        }
    }
}

// --------------------------------------------------------------------------------------------- host

// workgroups for tiles of BR x BC: of dx, as many as the rows can need (each expert may end in a ragged tile); of dw, exactly as many as there are
int64_t whole_blocks(int64_t n) { return (n + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds); }

template <bool DW>
int64_t grad_grid(const ExpertArgs &a, int64_t BR, int64_t BC, int64_t rows_bound)
{
    const int64_t row_tiles = DW ? a.E * ((a.N + BR - 1) / BR) : rows_bound / BR + std::min<int64_t>(a.E, rows_bound);
    return whole_blocks(row_tiles * ((a.H + BC - 1) / BC));
}

// The forms: a tile's code for workgroup `block`, its LDS, the workgroups of a launch, the workgroups per CU that its registers allow.
template <bool DW, int RB, int CB, bool RAGGED_LAST = false>
struct Wide {
    using G = GradShape<RB, CB>;
    static constexpr int kLds = G::kLdsBytes, kPerCu = RB * CB == 64 ? 1 : 2;
    static int64_t grid(const ExpertArgs &a, int64_t rows_bound)
    {
        // the short ragged tiles come in halves
        return grad_grid<DW>(a, G::BR, G::BC, rows_bound) + (RAGGED_LAST ? whole_blocks((int64_t)a.E * ((a.H + G::BC - 1) / G::BC)) : 0);
    }
    static __device__ __forceinline__ void run(const GradArgs &b, uint32_t block, unsigned char *lds) { grad_bf16_tile<DW, RB, CB, RAGGED_LAST>(b, block, lds); }
};

template <int XR, int CW, int NST>
struct Short {
    static constexpr int kLds = GradShort<XR, CW, NST>::kLdsBytes, kPerCu = 2;
    static int64_t grid(const ExpertArgs &a, int64_t rows_bound) { return grad_grid<false>(a, XR, CW, rows_bound); }
    static __device__ __forceinline__ void run(const GradArgs &b, uint32_t block, unsigned char *lds)
    {
        const RowTile t = find_grad_tile<false, XR, false>(b.a, (b.a.H + CW - 1) / CW, block, threadIdx.x & 63, nullptr);
        const int e = __builtin_amdgcn_readfirstlane(t.e);
        if (e >= 0)
            grad_short_tile<XR, CW, NST>(b, e, __builtin_amdgcn_readfirstlane(t.row0), __builtin_amdgcn_readfirstlane(t.row_end),
                                         __builtin_amdgcn_readfirstlane(t.ct) * CW, lds);
    }
};

template <int NST>
struct Slim {
    static constexpr int kLds = GradSlim<NST>::kLds, kPerCu = 2;
    static int64_t grid(const ExpertArgs &a, int64_t rows_bound) { return grad_grid<true>(a, 64, 64, rows_bound); }
    static __device__ __forceinline__ void run(const GradArgs &b, uint32_t block, unsigned char *lds)
    {
        const RowTile t = find_grad_tile<true, 64, false>(b.a, (b.a.H + 63) / 64, block, threadIdx.x & 63, nullptr);
        if (__builtin_amdgcn_readfirstlane(t.e) >= 0) grad_slim_tile<NST>(b, t, lds);
    }
};

template <bool DW, int BR, int NST>
struct F32 {
    static constexpr int kLds = GradShapeF32<BR, NST>::kLdsBytes, kPerCu = 2;
    static int64_t grid(const ExpertArgs &a, int64_t rows_bound) { return grad_grid<DW>(a, BR, 64, rows_bound); }
    static __device__ __forceinline__ void run(const GradArgs &b, uint32_t block, unsigned char *lds)
    {
        const RowTile t = find_grad_tile<DW, BR, false>(b.a, (b.a.H + 63) / 64, block, threadIdx.x & 63, nullptr);
        if (__builtin_amdgcn_readfirstlane(t.e) >= 0) grad_f32_tile<DW, BR, NST>(b, t, lds);
    }
};

template <typename Form>
__global__ __launch_bounds__(256, Form::kPerCu) void grad_kernel(GradArgs b)
{
    extern __shared__ __align__(16) unsigned char grad_lds[];
#if defined(__HIP_DEVICE_COMPILE__)
    Form::run(b, blockIdx.x, grad_lds);
#else
    (void)b;
    (void)grad_lds;
#endif
}

// Both gradients in one launch, the first `split` workgroups those of dx or, if dw_first, of dw: a walk along the longer axis begins first.
template <typename Dx, typename Dw>
__global__ __launch_bounds__(256, Dx::kPerCu < Dw::kPerCu ? Dx::kPerCu : Dw::kPerCu) void grad_both_kernel(GradArgs b, uint32_t split, bool dw_first)
{
    extern __shared__ __align__(16) unsigned char grad_lds[];
#if defined(__HIP_DEVICE_COMPILE__)
    const bool first = blockIdx.x < split;
    const uint32_t block = first ? blockIdx.x : blockIdx.x - split;
    if (first != dw_first) Dx::run(b, block, grad_lds);
    else Dw::run(b, block, grad_lds);
#else
    (void)b;
    (void)grad_lds;
    (void)split;
    (void)dw_first;
#endif
}

template <typename Form>
int launch_form(const GradArgs &b, int64_t rows_bound, hipStream_t st)
{
    const int64_t grid = Form::grid(b.a, rows_bound);
    if (!launchable(grid, 256)) return MONTA_ERR_UNSUPPORTED;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(grad_kernel<Form>), Form::kLds, lds_opt_in)) return rc;
    LaunchTimer timer(MONTA_K_EXPERT_BACKWARD, st);
    hipLaunchKernelGGL((grad_kernel<Form>), dim3((unsigned)grid), dim3(256), Form::kLds, st, b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <typename Dx, typename Dw>
int launch_both(const GradArgs &b, int64_t rows_bound, hipStream_t st)
{
    constexpr int lds = Dx::kLds > Dw::kLds ? Dx::kLds : Dw::kLds;
    const int64_t of_dx = Dx::grid(b.a, rows_bound), of_dw = Dw::grid(b.a, rows_bound), grid = of_dx + of_dw;
    const bool dw_first = rows_bound / std::min<int64_t>(b.a.E, rows_bound) > b.a.N;
    if (!launchable(grid, 256)) return MONTA_ERR_UNSUPPORTED;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(grad_both_kernel<Dx, Dw>), lds, lds_opt_in)) return rc;
    LaunchTimer timer(MONTA_K_EXPERT_BACKWARD, st);
    hipLaunchKernelGGL((grad_both_kernel<Dx, Dw>), dim3((unsigned)grid), dim3(256), lds, st, b, (uint32_t)(dw_first ? of_dw : of_dx), dw_first);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

// Which tile.  Measured on MI355X, three sets of buffers in turn, us; tokens x hidden x features, experts, top-2 (64 experts: top-8).
// dx in tiles of 32 x 64, 32 x 128, 64 x 128, 128 x 128, 256 x 256 and those with the ragged tiles last:
//   1 x 4096 x 4096, 8     21   29   30   31   61   34        256 x 1024 x 1024, 8      8.9  8.3  11   13   23   21
//   64 x 4096 x 4096, 8    58   48   48   51   90   52        2048 x 512 x 512, 4       7.5  6.8  8.6  10   20   20
//   256 x 4096 x 4096, 8   82   78   66   54   91   92        4096 x 1024 x 1024, 8     49   44   35   32   36   38
//   1024 x 4096 x 4096, 8  202  189  130  147  108  115       256 x 2048 x 1024, 64     64   60   59   65   68   77
//   2048 x 4096 x 4096, 8  360  308  222  208  195  155       2000 x 7168 x 2048, 64    1332 1177 833  739  627  667
// so 256 x 256 where most CUs get one, below that what gives every CU one or two.  Deep operands want wide tiles: a row of 64 elements is
// one line.  A walk of less than 512 features is over before a workgroup alone on its CU has begun the next: in 256 x 256 and in 128 x 128 with both
// gradients in one launch 2735 x 2264 x 168, 4, top-4, 50 and 36, 5107 x 2480 x 112, 8, top-2, 43 and 34, 4096 x 2048 x 256, 8 36 and 31, x 512 56 and 55.  dw in tiles of 128 x 128 and 256 x 256:
//   1 x 4096 x 4096, 8     47   56                            1024 x 1024 x 1024, 8     11   16
//   256 x 4096 x 4096, 8   78   80                            4096 x 1024 x 512, 32     19   18
//   2048 x 4096 x 4096, 8  176  164                           3000 x 1000 x 3000, 4     51   47
//   8192 x 2048 x 2048, 4  154  111                           512 x 2048 x 1024, 64     74   75 (both gradients 169 154)
//   148 x 8192 x 288, 21   32   44                            823 x 4096 x 120, 32      15   23
//   64 x 4096 x 4096, 8    67   70                            400 x 1032 x 4096, 16     54   53
// and where a few CUs have all of it, in tiles of 128 x 128 and in slim ones of 64 x 64 (both gradients in brackets):
//   8192 x 512 x 512, 2    64   31   (70   38)             1024 x 512 x 512, 4      6.6  5.0 (9.0  7.1)
//   8192 x 512 x 512, 4    37   19   (45   34)             4096 x 64 x 64, 2        35   15  (35   16)
//   8192 x 512 x 768, 4    24   18   (35   33)             64 x 512 x 512, 4        4.9  4.5 (6.0  6.1)
//   8192 x 1024 x 512, 4   39   38   (71   70)             1024 x 512 x 512, 8      5.7  6.2 (7.8  11)
// Few tiles: both gradients go out together, as alone neither fills the chip to its end (us, one after the other and together: 1 x 1024 x 1024, 8 experts 13.7
// and 9.1, 256 tokens 16.8 and 12.9, 4096 tokens 53.8 and 49.9; but 64 x 4096 x 4096, where dx then has as little room as dw, 122 and
// 154, and the large tiles of 8192 x 4096 x 4096 906 and 1000).  fp32 always: 4096 x 1024 x 1024, 8 experts 351 and 310.
// The longer walk first: 8192 x 512 x 512, 4 experts, dx first and dw first, 71 and 48, fp32 214 and 150; 1 x 1024 x 1024, fp32, 17 and 23.
int launch_grads(const GradArgs &b, bool bf16, int64_t rows_bound, hipStream_t st)
{
    const int64_t active = std::min<int64_t>(b.a.E, rows_bound), r = rows_bound / active;
    auto tiles = [&](int64_t R, int64_t C) { return active * ((b.a.H + C - 1) / C) * (2 * r + R) / (2 * R); };
    auto launch = [&](auto dx, auto dw, auto together) -> int {
        using Dx = decltype(dx);
        using Dw = decltype(dw);
        if constexpr (decltype(together)::value)
            if (b.dx && b.dw) return launch_both<Dx, Dw>(b, rows_bound, st);
        if (b.dx && b.dw && !launchable(Dw::grid(b.a, rows_bound), 256)) return MONTA_ERR_UNSUPPORTED;        // before dx goes out
        if (b.dx)
            if (int rc = launch_form<Dx>(b, rows_bound, st)) return rc;
        return b.dw ? launch_form<Dw>(b, rows_bound, st) : MONTA_OK;
    };
    constexpr std::true_type together{};
    constexpr std::false_type apart{};
    if (!bf16) {
        if (tiles(64, 64) <= 1024) return launch(F32<false, 32, 3>{}, F32<true, 64, 2>{}, together);
        return launch(F32<false, 64, 2>{}, F32<true, 64, 2>{}, together);
    }
    const bool big_dw = r > 48 && b.a.N > 128 && b.a.H > 128 && (int64_t)b.a.E * ((b.a.N + 255) / 256) * ((b.a.H + 255) / 256) >= 192;
    const int64_t dw_tiles = (int64_t)b.a.E * ((b.a.N + 127) / 128) * ((b.a.H + 127) / 128);
    auto with_dw = [&](auto dx) {
        if (dw_tiles <= 96) return launch(dx, Slim<2>{}, together);
        if (big_dw) return launch(dx, Wide<true, 8, 8>{}, apart);
        return dw_tiles <= 768 ? launch(dx, Wide<true, 4, 4>{}, together) : launch(dx, Wide<true, 4, 4>{}, apart);
    };
    if (tiles(32, 64) <= 256) return with_dw(Short<32, 64, 4>{});
    if (r <= 24 || tiles(32, 128) <= 400) return with_dw(Short<32, 128, 3>{});
    if (r > 56 && b.a.N >= 512 && tiles(256, 256) >= 160) {
        const bool ragged_last = r > 384 && b.a.E * ((b.a.H + 255) / 256) <= 256;
        auto large = [&](auto dx) {
            if (big_dw) return launch(dx, Wide<true, 8, 8>{}, apart);
            return dw_tiles <= 96 ? launch(dx, Slim<2>{}, apart) : launch(dx, Wide<true, 4, 4>{}, apart);
        };
        return ragged_last ? large(Wide<false, 8, 8, true>{}) : large(Wide<false, 8, 8>{});
    }
    if (r <= 56 || tiles(64, 128) <= 700) return with_dw(Short<64, 128, 3>{});
    return with_dw(Wide<false, 4, 4>{});
}

}  // namespace
}  // namespace monta

using namespace monta;

extern "C" int monta_expert_linear_backward(const monta_cfg *cfg, const void *dy, const void *x_final, const void *w_exp, int32_t out_features,
                                            void *dx_final, void *dw_exp, const void *ws, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, ws, &c)) return rc;
    if (!dy || !ws || (!dx_final && !dw_exp) || (dx_final && !w_exp) || (dw_exp && !x_final)) return MONTA_ERR_NULL;
    if (misaligned(dy, 16) || misaligned(x_final, 16) || misaligned(w_exp, 16) || misaligned(dx_final, 16) || misaligned(dw_exp, 16) || misaligned(ws, 16))
        return MONTA_ERR_ALIGN;
    const int bpe = c.bf16 ? 2 : 4;
    if (out_features < 1 || (int64_t)out_features * bpe % 16 != 0) return MONTA_ERR_INVALID;
    if (out_features > kBigMaxHidden || c.H > kBigMaxHidden || c.max_rows > kMostRows) return MONTA_ERR_UNSUPPORTED;
    const int64_t nx = c.max_rows * c.row_bytes, ny = c.max_rows * out_features * bpe, nw = (int64_t)c.s.E * out_features * c.row_bytes;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{dy, ny}, {x_final, nx}, {w_exp, nw}, {ws, c.ws_bytes}};
    for (const auto &r : read)
        if (r.p && ((dx_final && overlap(dx_final, nx, r.p, r.n)) || (dw_exp && overlap(dw_exp, nw, r.p, r.n)))) return MONTA_ERR_INVALID;
    if (dx_final && dw_exp && overlap(dx_final, nx, dw_exp, nw)) return MONTA_ERR_INVALID;
    GradArgs b{};
    b.a.E = (int16_t)c.s.E;
    b.a.H = c.H;
    b.a.N = out_features;
    b.a.max_rows = c.s.max_rows;
    expert_ranges(c.s, c.p, -1, &b.a);
    b.dy = dy;
    b.x = x_final;
    b.w = w_exp;
    b.dx = dx_final;
    b.dw = dw_exp;
    // Parts of half lines, of rows that are not whole 64 bytes or of a base between two, are streamed only where a tile's walk gives them time.  dw alone, through
    // the cache and streamed, us: 64 experts of 2048 x 1768, 1 row 141 and 179, 4 rows 158 and 176, 16 rows 167 and 173, 32 rows 171 and 167;
    // 400 x 1768, 1 row 29 and 32, 8 rows 34 and 33; 8 of 4096 x 4104, 1 row 84 and 95, 16 rows 99 and 90, 64 rows 104 and 96; 4424 x 1792, 16
    // bytes behind a line, 1 row 301 and 445, 64 rows 384 and 363; 64 bytes behind it 217 and 218, 326 and 294; on it 210 and 188, 318 and 277;
    // 64 experts of 2048 x 1824, rows of 57 half lines, 1 row 117 and 106, 8 rows 147 and 119.
    const bool whole = c.row_bytes % 64 == 0 && !misaligned(dw_exp, 64);
    b.stream_dw = whole || c.kept_bound >= 16 * std::min<int64_t>(c.s.E, c.kept_bound);
    return launch_grads(b, c.bf16, c.kept_bound, static_cast<hipStream_t>(stream));
}
