// Expert layer on 8-bit rows and 8-bit weights with a scale for each block of 128 along the hidden axis.
#include "monta_internal.hpp"

#include <algorithm>

namespace monta {

int64_t fp8_row_bytes(int64_t hidden);

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxHidden8 = 65536;

struct Expert8Args {
    ExpertArgs a;
    const float *w_scales;  // [E][ceil(N / 128)][nb]
    int32_t row8;           // bytes of a row of x
    int32_t nb;             // blocks of 128 along the hidden axis: steps of the walk
};

// A tile of XR rows x WR output features by WX x WW waves, each (XR / WX) x (WR / WW); NST stages of 128 bytes of every row, which is
// one block of the hidden axis, go straight to LDS, the loads of NST - 1 of them in flight.
template <int XR, int WR, int WX, int WW, int NST>
struct Tile8 {
    static constexpr int kWaves = WX * WW, kThreads = 64 * kWaves;
    static constexpr int kScaleBytes = kWaves * 256;                            // a scale per lane: at least XR of them
    static constexpr int kStageBytes = (XR + WR) * 128 + kScaleBytes, kLdsBytes = NST * kStageBytes;
    static constexpr int kCX = XR / 8 / kWaves, kCW = WR / 8 / kWaves, kLoads = kCX + kCW + 1;      // per wave and step
    static constexpr int kRB = XR / WX / 16, kCB = WR / WW / 16;
    static constexpr int kYounger = (NST - 2) * kLoads;
    static constexpr int kWait = 0x0070 | (kYounger & 15) | ((kYounger >> 4) << 14);     // vmcnt(kYounger), lgkmcnt(0)
    static_assert(XR % (8 * kWaves) == 0 && WR % (8 * kWaves) == 0 && XR <= kThreads && 128 % (WR / WW) == 0 && kYounger < 64 && kLdsBytes <= 160 * 1024,
                  "8-bit expert tile: shape");
};

template <int XR, int WR, int WX, int WW, int NST, bool F32>
__device__ __forceinline__ void expert8_tile(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w, void *__restrict__ y,
                                             const Expert8Args &b, unsigned char *lds8)
{
    using G = Tile8<XR, WR, WX, WW, NST>;
    const ExpertArgs &a = b.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int wx = wave / WW, ww = wave % WW;
    const int nct = (a.N + WR - 1) / WR;
    // logical tile numbers in blocks of 256, 32 consecutive ones per XCD; inside an expert (panel of 8 row tiles, column tile, row tile)
    const int64_t jx = blockIdx.x / kXcds;
    const int64_t L = (jx / 32) * (32 * kXcds) + (int64_t)(blockIdx.x % kXcds) * 32 + jx % 32;
    const ExpertTileHit hit = find_expert_tile<XR>(a, nct, L, lane);
    const int e = __builtin_amdgcn_readfirstlane(hit.e);
    if (e >= a.E) return;                                          // surplus workgroup
    constexpr int P = 8;
    const int full = hit.tiles / P;
    const bool whole = hit.L < (uint32_t)(full * P) * (uint32_t)nct;
    const uint32_t rem = whole ? hit.L % (uint32_t)(P * nct) : hit.L - (uint32_t)(full * P) * (uint32_t)nct;
    const int side = whole ? P : hit.tiles - full * P;             // row tiles of the panel
    const int ct = __builtin_amdgcn_readfirstlane((int)(rem / (uint32_t)side));
    const int rt = (whole ? (int)(hit.L / (uint32_t)(P * nct)) : full) * P + (int)(rem % (uint32_t)side);
    const int row0 = __builtin_amdgcn_readfirstlane(hit.lo + rt * XR);
    const int row_end = __builtin_amdgcn_readfirstlane(min(min(hit.hi, a.max_rows), row0 + XR));
    if (row0 < 0 || row0 >= row_end) return;
    const int col0 = ct * WR;
    const auto rx = make_rsrc(x + (int64_t)row0 * b.row8, (uint32_t)(row_end - row0) * (uint32_t)b.row8);
    const auto rw = make_rsrc(w + ((int64_t)e * a.N + col0) * a.H, (uint32_t)min(a.N - col0, WR) * (uint32_t)a.H);

    // Rows are 128 bytes in LDS; piece c of row r sits at position c ^ ((r / 2) % 8).  A chunk of 8 rows is one load of a wave.
    const int lr = lane >> 3;
    auto piece = [&](int c) { return (lane & 7) ^ ((4 * c + (lr >> 1)) & 7); };
    const uint32_t rows8 = (uint32_t)b.row8, roww = (uint32_t)a.H;
    const uint32_t scale_at = (uint32_t)(wave * 64 + lane) * rows8 + roww;
    auto issue = [&](int step, int slot) {
        unsigned char *const base = lds8 + slot * G::kStageBytes;
        const int left = step < b.nb ? a.H / 16 - step * 8 : 0;     // pieces of the row in this step; none past the end
        const uint32_t so = step < b.nb ? (uint32_t)step * 128u : 0u;
#pragma unroll
        for (int q = 0; q < G::kCW; ++q) {
            const int c = wave * G::kCW + q;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void *)(base + (XR / 8 + c) * 1024), 16,
                                                     piece(c) < left ? (uint32_t)(c * 8 + lr) * roww + piece(c) * 16 : kOutOfRange, so, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < G::kCX; ++q) {
            const int c = wave * G::kCX + q;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(base + c * 1024), 16,
                                                     piece(c) < left ? (uint32_t)(c * 8 + lr) * rows8 + piece(c) * 16 : kOutOfRange, so, 0, 0);
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(base + (XR + WR) * 128 + wave * 256), 4, left > 0 ? scale_at + (uint32_t)step * 4u : kOutOfRange, 0, 0, 0);
    };

    f32x4 acc[G::kRB][G::kCB];
#pragma unroll
    for (int i = 0; i < G::kRB; ++i)
#pragma unroll
        for (int j = 0; j < G::kCB; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    // the scales of the wave's features, which lie in one block: 64 steps at a time, one per lane
    const float *const ws = b.w_scales + ((int64_t)e * ((a.N + 127) / 128) + min(col0 + ww * (WR / WW), a.N - 1) / 128) * b.nb;
    float sw64 = 0.f;

#pragma unroll
    for (int q = 0; q < NST - 1; ++q) issue(q, q);
    int slot = 0;
    const unsigned char *const px = lds8 + (wx * (XR / WX) + m) * 128, *const pw = lds8 + (XR + ww * (WR / WW) + m) * 128;
    const unsigned char *const ps = lds8 + (XR + WR) * 128 + (wx * (XR / WX) + m) * 4;
    const int k0 = (g ^ ((m >> 1) & 7)) * 16, k1 = ((4 + g) ^ ((m >> 1) & 7)) * 16;
    for (int step = 0; step < b.nb; ++step) {
        if (step % 64 == 0) sw64 = ws[min(step + lane, b.nb - 1)];
        __builtin_amdgcn_s_waitcnt(G::kWait);                      // stage `step` has landed; this wave's reads of the one before are done
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(step + NST - 1, slot == 0 ? NST - 1 : slot - 1);     // where stage step - 1 was
        const int buf = slot * G::kStageBytes;
        const float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sw64), step % 64));
        u32x4 fx[G::kRB][2];
        float sc[G::kRB];
#pragma unroll
        for (int i = 0; i < G::kRB; ++i) {
            fx[i][0] = *reinterpret_cast<const u32x4 *>(px + buf + k0 + i * 2048);
            fx[i][1] = *reinterpret_cast<const u32x4 *>(px + buf + k1 + i * 2048);
            sc[i] = *reinterpret_cast<const float *>(ps + buf + i * 64) * sw;
        }
#pragma unroll
        for (int j = 0; j < G::kCB; ++j) {
            u32x4 fw[2];
            fw[0] = *reinterpret_cast<const u32x4 *>(pw + buf + k0 + j * 2048);
            fw[1] = *reinterpret_cast<const u32x4 *>(pw + buf + k1 + j * 2048);
            if constexpr (!F32) {
                const i32x8 f = __builtin_bit_cast(i32x8, __builtin_shufflevector(fw[0], fw[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int i = 0; i < G::kRB; ++i) {
                    const i32x8 r = __builtin_bit_cast(i32x8, __builtin_shufflevector(fx[i][0], fx[i][1], 0, 1, 2, 3, 4, 5, 6, 7));
                    const f32x4 part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f, r, (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(part[v], sc[i], acc[i][j][v]);
                }
            } else {
                // every e4m3 number is a bf16 number, and a product of two is an fp32 number
                auto wide = [](u32x4 c, int h) {
                    bf16x8 o;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[2 * h + q], 1.f, false);
                        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[2 * h + q], 1.f, true);
                        o[4 * q] = lo[0], o[4 * q + 1] = lo[1], o[4 * q + 2] = hi[0], o[4 * q + 3] = hi[1];
                    }
                    return o;
                };
                bf16x8 f[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) f[q] = wide(fw[q / 2], q % 2);
#pragma unroll
                for (int i = 0; i < G::kRB; ++i) {
                    f32x4 part = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[q], wide(fx[i][q / 2], q % 2), part, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(part[v], sc[i], acc[i][j][v]);
                }
            }
        }
        slot = slot == NST - 1 ? 0 : slot + 1;
    }

    // acc[i][j][v]: row 16 i + lane % 16 of the wave's rows, output feature 16 j + 4 (lane / 16) + v of its columns
#pragma unroll
    for (int i = 0; i < G::kRB; ++i) {
        const int64_t r = row0 + wx * (XR / WX) + i * 16 + m;
        if (r < row_end) {
#pragma unroll
            for (int j = 0; j < G::kCB; ++j) {
                const int n = col0 + ww * (WR / WW) + j * 16 + 4 * g;
                if (n < a.N) {
                    if constexpr (F32) {
                        *reinterpret_cast<f32x4 *>(static_cast<float *>(y) + r * a.N + n) = acc[i][j];
                    } else {
                        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                        bf16x4 o;
#pragma unroll
                        for (int v = 0; v < 4; ++v) o[v] = (__bf16)acc[i][j][v];
                        *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(y) + r * a.N + n) = o;
                    }
                }
            }
        }
    }
}

template <int XR, int WR, int WX, int WW, int NST, bool F32>
__global__ __launch_bounds__(64 * WX * WW) void expert8_kernel(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w,
                                                              void *__restrict__ y, Expert8Args b)
{
    extern __shared__ __align__(16) unsigned char lds8[];
    expert8_tile<XR, WR, WX, WW, NST, F32>(x, w, y, b, lds8);
}

template <int XR, int WR, int WX, int WW, int NST, bool F32>
int launch_expert8(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, hipStream_t st)
{
    using G = Tile8<XR, WR, WX, WW, NST>;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(expert8_kernel<XR, WR, WX, WW, NST, F32>), G::kLdsBytes, lds_opt_in)) return rc;
    const int64_t row_tiles = rows_bound / XR + std::min<int64_t>(b.a.E, rows_bound), nct = (b.a.N + WR - 1) / WR;
    const int64_t grid = (row_tiles * nct + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds);
    if (grid > 0x7fffffff) return MONTA_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((expert8_kernel<XR, WR, WX, WW, NST, F32>), dim3((unsigned)grid), dim3(G::kThreads), G::kLdsBytes, st,
                       static_cast<const unsigned char *>(x), static_cast<const unsigned char *>(w), y, b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <bool F32>
int launch_expert8_tiled(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, int64_t kept_bound, hipStream_t st)
{
    const int64_t active = std::min<int64_t>(b.a.E, kept_bound), r = kept_bound / active;
    auto tiles = [&](int64_t R, int64_t C) { return active * ((b.a.N + C - 1) / C) * (2 * r + R) / (2 * R); };
    if (r <= 24 || tiles(64, 128) <= 256) return launch_expert8<32, 64, 1, 4, 4, F32>(x, w, y, b, rows_bound, st);
    if (r <= 96 || tiles(256, 256) <= 256) return launch_expert8<64, 128, 2, 2, 3, F32>(x, w, y, b, rows_bound, st);
    return launch_expert8<256, 128, 4, 2, 3, F32>(x, w, y, b, rows_bound, st);
}

}  // namespace
}  // namespace monta

using namespace monta;

extern "C" int monta_expert_linear_fp8(const monta_cfg *cfg, const void *x_rows, const void *w_codes, const float *w_scales, int32_t out_features,
                                       void *y, const void *ws, int slice, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, ws, &c)) return rc;
    if (!x_rows || !w_codes || !w_scales || !y || !ws) return MONTA_ERR_NULL;
    if (misaligned(x_rows, 16) || misaligned(w_codes, 16) || misaligned(w_scales, 4) || misaligned(y, 16) || misaligned(ws, 16)) return MONTA_ERR_ALIGN;
    const int bpe = c.bf16 ? 2 : 4;
    if (out_features < 1 || (int64_t)out_features * bpe % 16 != 0 || c.H % 16 != 0) return MONTA_ERR_INVALID;
    if (slice < -1 || slice >= c.s.S) return MONTA_ERR_INVALID;
    if (c.H > kMaxHidden8) return MONTA_ERR_UNSUPPORTED;
    Expert8Args b{};
    b.row8 = (int32_t)fp8_row_bytes(c.H);
    b.nb = (c.H + 127) / 128;
    b.w_scales = w_scales;
    const int64_t ny = c.max_rows * out_features * bpe;
    if (overlap(y, ny, x_rows, c.max_rows * b.row8) || overlap(y, ny, w_codes, (int64_t)c.s.E * out_features * c.H) ||
        overlap(y, ny, w_scales, (int64_t)c.s.E * ((out_features + 127) / 128) * b.nb * 4) || overlap(y, ny, ws, c.ws_bytes))
        return MONTA_ERR_INVALID;
    b.a.E = (int16_t)c.s.E;
    b.a.H = c.H;
    b.a.N = out_features;
    b.a.max_rows = c.s.max_rows;
    expert_ranges(c.s, c.p, slice, &b.a);
    const int64_t rows_bound = slice_kept_bound(c.s, c.kept_bound, slice);
    hipStream_t st = static_cast<hipStream_t>(stream);
    LaunchTimer timer(MONTA_K_EXPERT_SCALED, st);
    return c.bf16 ? launch_expert8_tiled<false>(x_rows, w_codes, y, b, rows_bound, c.kept_bound, st)
                  : launch_expert8_tiled<true>(x_rows, w_codes, y, b, rows_bound, c.kept_bound, st);
}
