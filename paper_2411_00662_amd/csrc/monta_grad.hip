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
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct GradArgs {
    ExpertArgs a;           // lo, hi of the experts' rows, E, H, N, max_rows
    const void *dy, *x, *w;
    void *out;
};

// What a tile of the output belongs to.
struct GradTile {
    int e, row0, row_end;   // expert; rows of the tile (dx), or all rows of the expert (dw)
    int rt, ct;             // row tile and column tile inside the expert
};

// Tile of this workgroup; e < 0: none.  Logical tile numbers go out in blocks of 256, 32 consecutive ones to each XCD (hardware deals
// consecutive workgroups round robin to the 8 XCDs, each with its own L2); inside an expert the numbering is (panel of 8 row
// tiles, column tile, row tile), so that an XCD's workgroups share operand tiles.
template <bool DW, int BR>
__device__ __forceinline__ GradTile find_grad_tile(const ExpertArgs &a, int nct, int lane)
{
    constexpr int P = 8;
    const int64_t jx = blockIdx.x / kXcds;
    const int64_t L = (jx / 32) * (32 * kXcds) + (int64_t)(blockIdx.x % kXcds) * 32 + jx % 32;
    GradTile t{-1, 0, 0, 0, 0};
    int tiles;
    uint32_t in;
    int lo, hi;
    if constexpr (DW) {
        tiles = (a.N + BR - 1) / BR;
        const int64_t e = L / ((int64_t)tiles * nct);
        if (e >= a.E) return t;
        in = (uint32_t)(L - e * tiles * nct);
        t.e = (int)e;
        lo = a.lo[e];
        hi = a.hi_base[e] + a.hi_len[e];
    } else {
        const ExpertTileHit hit = find_expert_tile<BR>(a, nct, L, lane);
        if (hit.e >= a.E) return t;
        t.e = hit.e;
        in = hit.L;
        tiles = hit.tiles;
        lo = hit.lo;
        hi = hit.hi;
    }
    const int full = tiles / P;
    const bool whole = in < (uint32_t)(full * P) * (uint32_t)nct;
    const uint32_t rem = whole ? in % (uint32_t)(P * nct) : in - (uint32_t)(full * P) * (uint32_t)nct;
    const int side = whole ? P : tiles - full * P;
    t.e = __builtin_amdgcn_readfirstlane(t.e);
    t.ct = __builtin_amdgcn_readfirstlane((int)(rem / (uint32_t)side));
    t.rt = __builtin_amdgcn_readfirstlane((whole ? (int)(in / (uint32_t)(P * nct)) : full) * P + (int)(rem % (uint32_t)side));
    hi = min(hi, a.max_rows);
    lo = max(lo, 0);
    t.row0 = __builtin_amdgcn_readfirstlane(DW ? lo : lo + t.rt * BR);
    t.row_end = __builtin_amdgcn_readfirstlane(DW ? max(hi, lo) : min(hi, lo + (t.rt + 1) * BR));
    if (!DW && t.row0 >= t.row_end) t.e = -1;
    return t;
}

// --------------------------------------------------------------------------------------------- bf16
//
// Steps of 64 elements of the summed axis go straight to LDS.  An operand whose elements lie along that axis ("flat": dy in dx) is
// stored as rows of 128 bytes, piece c of row r at position c ^ ((r / 2) % 8), and read 16 bytes at a time.  One that lies across it ("deep") is
// stored as it comes, 64 rows of C elements, and read by the transposing LDS read: 16 lanes hand in 4 rows of 16 elements and get a
// column of 4 each; two of them are the 8 elements of an MFMA's fragment.  Its swizzle keeps the 8 rows of 32 bytes that half a wave
// reads (rows 8 g + j, g = 0, 1, j = 0..3) in different banks: the 32-byte segment s of row k sits at segment s ^ f(k).
template <int C>
__device__ __forceinline__ constexpr int deep_swizzle(int k)
{
    if constexpr (C >= 128) return (k & 3) | ((k >> 3) & 1) << 2;          // rows of 256 bytes or more begin on the same bank
    else if constexpr (C == 64) return ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
    else return (k >> 3) & 1;
}

// BR x BC: tile of the output, rows (of dx) or output features (of dw) x hidden elements; WR x WC waves; NST stages, the loads of NST - 1
// in flight.
template <int BR, int BC, int WR, int WC, int NST>
struct GradShape {
    static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
    static constexpr int kStageBytes = (BR + BC) * 128, kLdsBytes = NST * kStageBytes;
    static constexpr int kCR = BR / 8 / kWaves, kCC = BC / 8 / kWaves, kLoads = kCR + kCC;        // 1 KiB loads per wave and step
    static constexpr int kRB = BR / WR / 16, kCB = BC / WC / 16;
    static constexpr int kYounger = (NST - 2) * kLoads;
    static constexpr int kWait = 0x0070 | (kYounger & 15) | ((kYounger >> 4) << 14);              // vmcnt(kYounger), lgkmcnt(0)
    static_assert(BR % (8 * kWaves) == 0 && BC % (8 * kWaves) == 0 && BR >= 32 && BC >= 32 && kYounger < 64 && kLdsBytes <= 160 * 1024, "gradient tile: shape");
};

// A deep operand's loads: 64 rows of C elements from `base` on, `pitch` bytes apart, of which `cols` elements exist.
template <int C, int CHUNKS>
struct DeepLoads {
    static constexpr int kRowsPerChunk = 1024 / (2 * C);
    uint32_t at[CHUNKS];
    __device__ __forceinline__ DeepLoads(int first_chunk, int lane, uint32_t pitch, int cols)
    {
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int k = (first_chunk + q) * kRowsPerChunk + lane * 16 / (2 * C), p = lane % (C / 8);
            const int from = ((p >> 1) ^ deep_swizzle<C>(k)) * 2 + (p & 1);
            at[q] = from * 8 < cols ? (uint32_t)k * pitch + from * 16 : kOutOfRange;
        }
    }
};

// the 8 elements along the summed axis of one fragment: rows k .. k+3 and k+4 .. k+7 of a deep operand
__device__ __forceinline__ bf16x8 read_deep(const unsigned char *p, int next4)
{
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + next4));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <bool DW, int BR, int BC, int WR, int WC, int NST>
__device__ __forceinline__ void grad_bf16_tile(const GradArgs &b, unsigned char *grad_lds)
{
    using G = GradShape<BR, BC, WR, WC, NST>;
    const ExpertArgs &a = b.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int wr = wave / WC, wc = wave % WC;
    const GradTile t = find_grad_tile<DW, BR>(a, (a.H + BC - 1) / BC, lane);
    if (t.e < 0) return;
    const int64_t H = a.H, N = a.N;
    const int col0 = t.ct * BC, out0 = DW ? t.rt * BR : 0;         // out0: first output feature of a tile of dw
    const int depth = DW ? t.row_end - t.row0 : a.N;               // of the summed axis
    const int nsteps = (depth + 63) / 64;

    // columns: x (dw) or w (dx), deep in both; rows: dy, deep (dw) or flat (dx)
    const uint32_t pitch_c = (uint32_t)a.H * 2, pitch_r = (uint32_t)a.N * 2;
    const char *from_c = static_cast<const char *>(DW ? b.x : b.w) + (DW ? (int64_t)t.row0 * H : (int64_t)t.e * N * H) * 2 + (int64_t)col0 * 2;
    const char *from_r = static_cast<const char *>(b.dy) + ((int64_t)t.row0 * N + out0) * 2;
    const DeepLoads<BC, G::kCC> cols(wave * G::kCC, lane, pitch_c, a.H - col0);
    const DeepLoads<BR, G::kCR> rows_deep(wave * G::kCR, lane, pitch_r, a.N - out0);
    const int lr = lane >> 3;
    auto piece = [&](int c) { return (lane & 7) ^ ((4 * c + (lr >> 1)) & 7); };
    const auto flat = make_rsrc(from_r, DW ? 0u : (uint32_t)(t.row_end - t.row0) * pitch_r);
    auto issue = [&](int step, int slot) {
        unsigned char *const base = grad_lds + slot * G::kStageBytes;
        // rows of a deep operand in this step, none past the end; the descriptor begins at the step's first, `cut` bytes into its row
        const int left = min(max(depth - step * 64, 0), 64);
        auto records = [&](uint32_t pitch, uint32_t cut) { return left > 0 ? (uint32_t)left * pitch - cut : 0u; };
        const auto rc = make_rsrc(from_c + (int64_t)step * 64 * pitch_c, records(pitch_c, (uint32_t)col0 * 2));
#pragma unroll
        for (int q = 0; q < G::kCC; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rc, (lds_void *)(base + BR * 128 + (wave * G::kCC + q) * 1024), 16, cols.at[q], 0, 0, 0);
        if constexpr (DW) {
            const auto rr = make_rsrc(from_r + (int64_t)step * 64 * pitch_r, records(pitch_r, (uint32_t)out0 * 2));
#pragma unroll
            for (int q = 0; q < G::kCR; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rr, (lds_void *)(base + (wave * G::kCR + q) * 1024), 16, rows_deep.at[q], 0, 0, 0);
        } else {
#pragma unroll
            for (int q = 0; q < G::kCR; ++q) {
                const int c = wave * G::kCR + q;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(flat, (lds_void *)(base + c * 1024), 16,
                                                         piece(c) * 8 < left ? (uint32_t)(c * 8 + lr) * pitch_r + (uint32_t)step * 128u + piece(c) * 16 : kOutOfRange,
                                                         0, 0, 0);
            }
        }
    };

    f32x4 acc[G::kRB][G::kCB];
#pragma unroll
    for (int i = 0; i < G::kRB; ++i)
#pragma unroll
        for (int j = 0; j < G::kCB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

    // this lane's place in a deep operand: row 8 g + m / 4, quarter m % 4 of a segment
    const int kl = 8 * g + (m >> 2);
    const unsigned char *const pc = grad_lds + BR * 128 + kl * (2 * BC) + (m & 3) * 8;
    const unsigned char *const pr = DW ? grad_lds + kl * (2 * BR) + (m & 3) * 8 : grad_lds + (wr * (BR / WR) + m) * 128;
    const int sc = deep_swizzle<BC>(kl), sr = deep_swizzle<BR>(kl);

#pragma unroll
    for (int q = 0; q < NST - 1; ++q) issue(q, q);
    int slot = 0;
    for (int step = 0; step < nsteps; ++step) {
        __builtin_amdgcn_s_waitcnt(G::kWait);                      // stage `step` has landed; this wave's reads of the one before are done
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(step + NST - 1, slot == 0 ? NST - 1 : slot - 1);     // where stage step - 1 was
        const int buf = slot * G::kStageBytes;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 fr[G::kRB], fc[G::kCB];
#pragma unroll
            for (int i = 0; i < G::kRB; ++i) {
                if constexpr (DW) fr[i] = read_deep(pr + buf + ks * 64 * BR + ((wr * G::kRB + i) ^ sr) * 32, 8 * BR);
                else fr[i] = *reinterpret_cast<const bf16x8 *>(pr + buf + ((4 * ks + g) ^ ((m >> 1) & 7)) * 16 + i * 2048);
            }
#pragma unroll
            for (int j = 0; j < G::kCB; ++j) fc[j] = read_deep(pc + buf + ks * 64 * BC + ((wc * G::kCB + j) ^ sc) * 32, 8 * BC);
#pragma unroll
            for (int i = 0; i < G::kRB; ++i)
#pragma unroll
                for (int j = 0; j < G::kCB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[j], fr[i], acc[i][j], 0, 0, 0);
        }
        slot = slot == NST - 1 ? 0 : slot + 1;
    }

    // acc[i][j][v]: row 16 i + lane % 16 of the wave's rows, hidden element 16 j + 4 (lane / 16) + v of its columns
    __bf16 *const out = static_cast<__bf16 *>(b.out) + (DW ? (int64_t)t.e * N * H : 0);
#pragma unroll
    for (int i = 0; i < G::kRB; ++i) {
        const int64_t r = (DW ? out0 : t.row0) + wr * (BR / WR) + i * 16 + m;
        if (r < (DW ? a.N : t.row_end)) {
#pragma unroll
            for (int j = 0; j < G::kCB; ++j) {
                const int h = col0 + wc * (BC / WC) + j * 16 + 4 * g;
                if (h < a.H) {
                    bf16x4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[v] = (__bf16)acc[i][j][v];
                    *reinterpret_cast<bf16x4 *>(out + r * H + h) = o;
                }
            }
        }
    }
}

template <bool DW, int BR, int BC, int WR, int WC, int NST>
__global__ __launch_bounds__(64 * WR * WC) void grad_bf16_kernel(GradArgs b)
{
    extern __shared__ __align__(16) unsigned char grad_lds[];
    grad_bf16_tile<DW, BR, BC, WR, WC, NST>(b, grad_lds);
}

// --------------------------------------------------------------------------------------------- fp32
//
// 64 x 64 tiles by 2 x 2 waves, 32 elements of the summed axis at a time through registers into LDS, where both operands lie with that
// axis outside (rows of 64 elements): a 32-bit element has nothing to be transposed with.  What bounds it is the fp32 matrix rate.
constexpr int kF32Tile = 64, kF32Depth = 32, kF32Pitch = 68;

template <bool DW>
__global__ __launch_bounds__(256) void grad_f32_kernel(GradArgs b)
{
    __shared__ __align__(16) float rows[kF32Depth][kF32Pitch], cols[kF32Depth][kF32Pitch];
    const ExpertArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, g = lane >> 4, wr = wave >> 1, wc = wave & 1;
    const GradTile t = find_grad_tile<DW, kF32Tile>(a, (a.H + kF32Tile - 1) / kF32Tile, lane);
    if (t.e < 0) return;
    const int64_t H = a.H, N = a.N;
    const int col0 = t.ct * kF32Tile, out0 = DW ? t.rt * kF32Tile : 0;
    const int depth = DW ? t.row_end - t.row0 : a.N;
    const float *dy = static_cast<const float *>(b.dy) + (int64_t)t.row0 * N, *from_c = DW ? static_cast<const float *>(b.x) + (int64_t)t.row0 * H
                                                                                           : static_cast<const float *>(b.w) + (int64_t)t.e * N * H;
    constexpr f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 pr[2], pc[2];
    // piece q of this thread: deep operands, four elements of row k = piece / 16; flat ones, elements 4 (piece % 8) of row piece / 8
    auto fetch = [&](int k0) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int p = tid + 256 * q, k = k0 + p / 16, c = p % 16 * 4;
            pc[q] = k < depth && col0 + c < a.H ? *reinterpret_cast<const f32x4 *>(from_c + (int64_t)k * H + col0 + c) : zero;
            if constexpr (DW) {
                pr[q] = k < depth && out0 + c < a.N ? *reinterpret_cast<const f32x4 *>(dy + (int64_t)k * N + out0 + c) : zero;
            } else {
                const int r = p / 8, n = k0 + p % 8 * 4;
                pr[q] = t.row0 + r < t.row_end && n < depth ? *reinterpret_cast<const f32x4 *>(dy + (int64_t)r * N + n) : zero;
            }
        }
    };
    f32x4 acc[2][2] = {{zero, zero}, {zero, zero}};
    fetch(0);
    for (int k0 = 0; k0 < depth; k0 += kF32Depth) {
        __syncthreads();                                           // the previous step has been read
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int p = tid + 256 * q;
            *reinterpret_cast<f32x4 *>(&cols[p / 16][p % 16 * 4]) = pc[q];
            if constexpr (DW) {
                *reinterpret_cast<f32x4 *>(&rows[p / 16][p % 16 * 4]) = pr[q];
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v) rows[p % 8 * 4 + v][p / 8] = pr[q][v];
            }
        }
        __syncthreads();
        if (k0 + kF32Depth < depth) fetch(k0 + kF32Depth);
#pragma unroll
        for (int s = 0; s < kF32Depth / 4; ++s) {                  // group g's element: row 8 g + s, so that the groups are in two bank halves
            float fr[2], fc[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fr[i] = rows[8 * g + s][wr * 32 + i * 16 + m];
                fc[i] = cols[8 * g + s][wc * 32 + i * 16 + m];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fc[j], fr[i], acc[i][j], 0, 0, 0);
        }
    }
    float *const out = static_cast<float *>(b.out) + (DW ? (int64_t)t.e * N * H : 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t r = (DW ? out0 : t.row0) + wr * 32 + i * 16 + m;
        if (r < (DW ? a.N : t.row_end)) {
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
template <bool DW>
int64_t grad_grid(const ExpertArgs &a, int64_t BR, int64_t BC, int64_t rows_bound)
{
    const int64_t row_tiles = DW ? a.E * ((a.N + BR - 1) / BR) : rows_bound / BR + std::min<int64_t>(a.E, rows_bound);
    const int64_t n = row_tiles * ((a.H + BC - 1) / BC);
    return (n + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds);
}

template <bool DW, int BR, int BC, int WR, int WC, int NST>
int launch_grad_bf16(const GradArgs &b, int64_t rows_bound, hipStream_t st)
{
    using G = GradShape<BR, BC, WR, WC, NST>;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(grad_bf16_kernel<DW, BR, BC, WR, WC, NST>), G::kLdsBytes, lds_opt_in)) return rc;
    const int64_t grid = grad_grid<DW>(b.a, BR, BC, rows_bound);
    if (grid > 0x7fffffff) return MONTA_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((grad_bf16_kernel<DW, BR, BC, WR, WC, NST>), dim3((unsigned)grid), dim3(G::kThreads), G::kLdsBytes, st, b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <bool DW>
int launch_grad(const GradArgs &b, bool bf16, int64_t rows_bound, hipStream_t st)
{
    LaunchTimer timer(MONTA_K_EXPERT_BACKWARD, st);
    if (!bf16) {
        const int64_t grid = grad_grid<DW>(b.a, kF32Tile, kF32Tile, rows_bound);
        if (grid > 0x7fffffff) return MONTA_ERR_UNSUPPORTED;
        hipLaunchKernelGGL((grad_f32_kernel<DW>), dim3((unsigned)grid), dim3(256), 0, st, b);
        MONTA_HIP_TRY(hipGetLastError());
        return MONTA_OK;
    }
    const int64_t active = std::min<int64_t>(b.a.E, rows_bound), r = rows_bound / active;
    if (!DW && r <= 48) return launch_grad_bf16<DW, 32, 128, 1, 4, 3>(b, rows_bound, st);
    return launch_grad_bf16<DW, 128, 128, 2, 2, 2>(b, rows_bound, st);
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
    if (out_features > kBigMaxHidden || c.H > kBigMaxHidden) return MONTA_ERR_UNSUPPORTED;
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
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dx_final) {
        b.out = dx_final;
        if (int rc = launch_grad<false>(b, c.bf16, c.kept_bound, st)) return rc;
    }
    if (dw_exp) {
        b.out = dw_exp;
        if (int rc = launch_grad<true>(b, c.bf16, c.kept_bound, st)) return rc;
    }
    return MONTA_OK;
}
