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

// The product of 16 output features (a lane's 32 codes of one: pieces g and 4 + g of the block, g = lane / 16) and 16 rows over a block.
template <bool F32>
__device__ __forceinline__ f32x4 block_product(const u32x4 (&w)[2], const u32x4 (&x)[2])
{
    f32x4 part = {0.f, 0.f, 0.f, 0.f};
    if constexpr (!F32) {
        const i32x8 f = __builtin_bit_cast(i32x8, __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7));
        const i32x8 r = __builtin_bit_cast(i32x8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
        part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f, r, part, 0, 0, 0, 0, 0, 0);
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
#pragma unroll
        for (int q = 0; q < 4; ++q) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(w[q / 2], q % 2), wide(x[q / 2], q % 2), part, 0, 0, 0);
    }
    return part;
}

// A tile of XR rows x WR output features by WX x WW waves, each (XR / WX) x (WR / WW); NST stages of 128 bytes of every row, which is
// one block of the hidden axis, go straight to LDS, the loads of NST - 1 of them in flight.  64 x 4096 x 4096, 8 experts, top-2, in 32 x 64: 25 to
// 28 us, 136 MB of weights at 4.9 to 5.4 TB/s.
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
                                             const Expert8Args &b, int e, int row0, int row_end, int col0, unsigned char *lds8, int start = 0)
{
    using G = Tile8<XR, WR, WX, WW, NST>;
    const ExpertArgs &a = b.a;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));      // share nothing with the caller's other path, which has no register left to keep it in
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int wx = wave / WW, ww = wave % WW;
    const auto rx = make_rsrc(x + (int64_t)row0 * b.row8, (uint32_t)(row_end - row0) * (uint32_t)b.row8);
    const auto rw = make_rsrc(w + ((int64_t)e * a.N + col0) * a.H, (uint32_t)min(a.N - col0, WR) * (uint32_t)a.H);

    // Rows are 128 bytes in LDS; piece c of row r sits at position c ^ ((r / 2) % 8).  A chunk of 8 rows is one load of a wave.
    const int lr = lane >> 3;
    auto piece = [&](int c) { return (lane & 7) ^ ((4 * c + (lr >> 1)) & 7); };
    const uint32_t rows8 = (uint32_t)b.row8, roww = (uint32_t)a.H;
    const uint32_t scale_at = (uint32_t)(wave * 64 + lane) * rows8 + roww;
    // The walk begins at step `start` and goes round.  Past its end nothing is fetched.
    auto place = [&](int step) { return step + start >= b.nb ? step + start - b.nb : step + start; };
    auto issue = [&](int step, int slot) {
        unsigned char *const base = lds8 + slot * G::kStageBytes;
        const int at = step < b.nb ? place(step) : 0;
        const int left = step < b.nb ? a.H / 16 - at * 8 : 0;       // pieces of the row in this step
        const uint32_t so = (uint32_t)at * 128u;
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
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(base + (XR + WR) * 128 + wave * 256), 4, left > 0 ? scale_at + (uint32_t)at * 4u : kOutOfRange, 0, 0, 0);
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
        const int at = place(step);
        if (at % 64 == 0 || step == 0) {
            sw64 = ws[min(at / 64 * 64 + lane, b.nb - 1)];
            asm volatile("" : "+v"(sw64));                         // waited for here: left to its use, every step would wait for its loads
        }
        __builtin_amdgcn_s_waitcnt(G::kWait);                      // stage `step` has landed; this wave's reads of the one before are done
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(step + NST - 1, slot == 0 ? NST - 1 : slot - 1);     // where stage step - 1 was
        const int buf = slot * G::kStageBytes;
        const float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sw64), at % 64));
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
#pragma unroll
            for (int i = 0; i < G::kRB; ++i) {
                const f32x4 part = block_product<F32>(fw, fx[i]);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(part[v], sc[i], acc[i][j][v]);
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

// Few tiles: a walk along the hidden axis would be all latency.  The W waves of a workgroup share the blocks of a tile of 16 rows x 16 CB
// output features, wave after wave, D of them at a time straight to registers: 16 bytes a lane, the lanes of a row side by side.  The
// waves' sums meet in LDS and are added in the order of the waves.
template <int CB, int W, int D, bool F32>
__global__ __launch_bounds__(64 * W) void expert8_split_kernel(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w, void *__restrict__ y,
                                                               Expert8Args b)
{
    constexpr int WR = 16 * CB, kPitch = WR + 4;
    static_assert(128 % WR == 0 && W * 16 * kPitch * 4 <= 64 * 1024, "8-bit split tile: shape");
    __shared__ __align__(16) float sums[W * 16 * kPitch];
    const ExpertArgs &a = b.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const RowTile t = find_row_tile<16, false>(a, (a.N + WR - 1) / WR, blockIdx.x, lane, nullptr);
    const int e = __builtin_amdgcn_readfirstlane(t.e);
    if (e < 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(t.row0), row_end = __builtin_amdgcn_readfirstlane(t.row_end);
    const int col0 = __builtin_amdgcn_readfirstlane(t.ct) * WR;
    const auto rx = make_rsrc(x + (int64_t)row0 * b.row8, (uint32_t)(row_end - row0) * (uint32_t)b.row8);
    const auto rw = make_rsrc(w + ((int64_t)e * a.N + col0) * a.H, (uint32_t)min(a.N - col0, WR) * (uint32_t)a.H);
    const float *const ws = b.w_scales + ((int64_t)e * ((a.N + 127) / 128) + col0 / 128) * b.nb;
    f32x4 acc[CB];
#pragma unroll
    for (int j = 0; j < CB; ++j) acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int first = wave; first < b.nb; first += W * D) {
        u32x4 fx[D][2], fw[D][CB][2];
        float sx[D], sw[D];
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int step = first + d * W;                        // past the end everything is out of range: zeros
            sw[d] = ws[min(step, b.nb - 1)];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = step * 128 + h * 64 + g * 16;
#pragma unroll
                for (int j = 0; j < CB; ++j)
                    fw[d][j][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, at < a.H ? (j * 16 + m) * a.H + at : (int)kOutOfRange, 0, 0));
                fx[d][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, at < a.H ? m * b.row8 + at : (int)kOutOfRange, 0, 0));
            }
            sx[d] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rx, step < b.nb ? m * b.row8 + a.H + step * 4 : (int)kOutOfRange, 0, 0));
        }
        __builtin_amdgcn_sched_barrier(0);                         // all loads first
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const float scale = sx[d] * (first + d * W < b.nb ? sw[d] : 0.f);      // the last block's may be infinite: not past the end
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const f32x4 part = block_product<F32>(fw[d][j], fx[d]);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[j][v] = __builtin_fmaf(part[v], scale, acc[j][v]);
            }
        }
    }
    // acc[j][v]: row lane % 16, output feature 16 j + 4 (lane / 16) + v
#pragma unroll
    for (int j = 0; j < CB; ++j) *reinterpret_cast<f32x4 *>(sums + (wave * 16 + m) * kPitch + j * 16 + 4 * g) = acc[j];
    __syncthreads();
    static_assert(16 * WR / 4 <= 64 * W, "8-bit split tile: four features a lane");
    const int row = tid / (WR / 4), c = tid % (WR / 4) * 4;
    if (row0 + row < row_end && row < 16 && col0 + c < a.N) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < W; ++p) v += *reinterpret_cast<const f32x4 *>(sums + (p * 16 + row) * kPitch + c);
        const int64_t at = (int64_t)(row0 + row) * a.N + col0 + c;
        if constexpr (F32) {
            *reinterpret_cast<f32x4 *>(static_cast<float *>(y) + at) = v;
        } else {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            bf16x4 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = (__bf16)v[k];
            *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(y) + at) = o;
        }
    }
}

// At least two workgroups of 256 per CU: with more registers than 256 per lane the compiler would take the products through the
// accumulator registers, a move for each.
template <int XR, int WR, int WX, int WW, int NST, bool F32>
__global__ __launch_bounds__(64 * WX * WW, 2) void expert8_kernel(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w,
                                                                 void *__restrict__ y, Expert8Args b)
{
    extern __shared__ __align__(16) unsigned char lds8[];
    const RowTile t = find_row_tile<XR, false>(b.a, (b.a.N + WR - 1) / WR, blockIdx.x, threadIdx.x & 63, nullptr);
    const int e = __builtin_amdgcn_readfirstlane(t.e);
    if (e < 0) return;
#if defined(__HIP_DEVICE_COMPILE__)
    expert8_tile<XR, WR, WX, WW, NST, F32>(x, w, y, b, e, __builtin_amdgcn_readfirstlane(t.row0), __builtin_amdgcn_readfirstlane(t.row_end),
                                           __builtin_amdgcn_readfirstlane(t.ct) * WR, lds8,
                                           b.a.spread ? walk_start(e * ((b.a.N + WR - 1) / WR) + __builtin_amdgcn_readfirstlane(t.ct), b.nb) : 0);
#else
    (void)x;
    (void)w;
    (void)y;
    (void)lds8;
#endif
}

// Long segments: a 256 x 256 tile of y by 4 x 2 waves, two per SIMD, each 64 rows x 128 features, the features of one block of the weights.  The blocks'
// sums cannot stay in the accumulators of the matrix instructions: each is a product of its own, of 32 clocks, whose four results a lane
// scales and adds in four more instructions, 16 clocks, under the other wave's products.  A result is used four products later, so that
// nothing waits for it.
// 8192 x 4096 x 4096, 8 experts, top-2: 270 to 305 us by the box, 1.8 to 2.0 PFLOP/s; without its loads 235, so what bounds it is the matrix pipe
// and the scaling beside it at the clock the card holds (a library product of one scale reaches 2.5), and LDS beside them: stages written and fragments
// read are 256 KiB a step, as many clocks as its products.
// 8192 x 8192 x 8192, 2 experts, 500 to 545 us, 2.0 to 2.2.
// A tile of at most 128 rows computes for half as long and waits for its weights: 128 x 256 or 64 x 256, three stages.  4096 x 7168 x 2048 with
// 64 experts, top-8, a load of which 21 experts have most and 43 at most 100 rows, takes 360 us with both, 370 with the higher one alone, 396
// without; 512 rows for every expert 556 to 560 us with and without.
// Two stages of 64 KiB.  One barrier per step, before the last two of the eight columns of products: then every wave has read all of
// stage s, and stage s + 1 is there; the loads of s + 2 go to the place of s under those two, as do the reads of the next step's first
// fragments, each row fragment right behind its last use.
constexpr int kBig8 = 256, kBig8Stage = 2 * kBig8 * 128 + 2048, kBig8Sink = 2 * kBig8Stage;
constexpr int kBig8LdsBytes = Tile8<128, kBig8, 2, 4, 3>::kLdsBytes;

template <bool RAGGED_LAST, bool TAIL>
__device__ __forceinline__ void expert8_big_tile(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w, __bf16 *__restrict__ y,
                                                 const Expert8Args &b, const RowTile &t, unsigned char *lds8)
{
    const ExpertArgs &a = b.a;
    const int e = __builtin_amdgcn_readfirstlane(t.e);
    if (e < 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(t.row0), row_end = __builtin_amdgcn_readfirstlane(t.row_end);
    const int col0 = __builtin_amdgcn_readfirstlane(t.ct) * kBig8;
    if (row_end - row0 <= 128) {
        using Half = Tile8<128, kBig8, 2, 4, 3>;
        using Quarter = Tile8<kShortTileRows, kBig8, 2, 4, 3>;
        using Last = Tile8<kShortTileRows, 128, 2, 4, 5>;
        static_assert(std::max({Half::kLdsBytes, Quarter::kLdsBytes, Last::kLdsBytes}) <= kBig8LdsBytes, "8-bit lower tiles: stages must fit the kernel's LDS");
        if (row_end - row0 > kShortTileRows) {
            expert8_tile<128, kBig8, 2, 4, 3, false>(x, w, y, b, e, row0, row_end, col0, lds8);
        } else if constexpr (RAGGED_LAST) {                        // by halves of the column tile, twice the workgroups
            const int from = __builtin_amdgcn_readfirstlane(t.ct) * 128;
            if (from < a.N) expert8_tile<kShortTileRows, 128, 2, 4, 5, false>(x, w, y, b, e, row0, row_end, from, lds8);
        } else {
            expert8_tile<kShortTileRows, kBig8, 2, 4, 3, false>(x, w, y, b, e, row0, row_end, col0, lds8);
        }
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int wx = wave >> 1, ww = wave & 1;
    const auto rx = make_rsrc(x + (int64_t)row0 * b.row8, (uint32_t)(row_end - row0) * (uint32_t)b.row8);
    const auto rw = make_rsrc(w + ((int64_t)e * a.N + col0) * a.H, (uint32_t)min(a.N - col0, kBig8) * (uint32_t)a.H);
    // a wave's loads: four neighbouring chunks of 8 rows of x and of w each; chunks 16 rows apart have the same swizzle
    const int lr = lane >> 3;
    uint32_t at_x[2], at_w[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int row = (wave * 4 + q) * 8 + lr;
        const int piece = (lane & 7) ^ ((row >> 1) & 7);
        at_x[q] = (uint32_t)row * (uint32_t)b.row8 + piece * 16;
        at_w[q] = (uint32_t)row * (uint32_t)a.H + piece * 16;
    }
    const uint32_t at_s = wave < 4 ? (uint32_t)(wave * 64 + lane) * (uint32_t)b.row8 + (uint32_t)a.H : kOutOfRange;
    // Load l of step `step`: 4 of w, 4 of x, the rows' scales (64 rows a wave; waves 4 to 7 ask for none).  Past the end the last step is fetched again, into
    // a place that is not read any more.  TAIL: the pieces of the last step that lie past the end of a row are out of range.
    auto issue = [&](int step, int l) {
        unsigned char *const base = lds8 + (step & 1) * kBig8Stage;
        const int from = min(step, b.nb - 1);
        if (l < 8) {
            const int q = l & 3;
            uint32_t at = l < 4 ? at_w[q & 1] : at_x[q & 1];
            if (q >> 1) {
                uint32_t rows = 16u * (uint32_t)(l < 4 ? a.H : b.row8);
                asm volatile("" : "+s"(rows));                     // added at each use: offsets kept would be spilled
                at += rows;
            }
            if constexpr (TAIL) {
                int me = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
                asm volatile("" : "+v"(me));                       // found again each time, as well
                const int p = (me & 7) ^ (((wave * 32 + (q & 1) * 8 + (me >> 3)) >> 1) & 7);
                at |= p >= a.H / 16 - from * 8 ? kOutOfRange : 0u;
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(l < 4 ? rw : rx, (lds_void *)(base + (l < 4 ? kBig8 * 128 : 0) + (wave * 4 + q) * 1024), 16, at,
                                                     (uint32_t)from * 128u, 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(base + 2 * kBig8 * 128 + wave * 256), 4, at_s, (uint32_t)from * 4u, 0, 0);
        }
    };

    // The early touches: a step's loads have a step's time to arrive, which covers an L2 hit but no miss, so each workgroup touches, a step
    // ahead of them, one word per row of its share of the rows that it shares with the others on its XCD: waves 0 to 3 of x, with four column
    // tiles, waves 4 to 7 of w, with the row tiles of the panel.
    const int row_of_lane = (wave & 3) * 64 + lane;
    const bool mine = wave < 4 ? wave == (__builtin_amdgcn_readfirstlane(t.ct) & 3)
                               : row_of_lane * __builtin_amdgcn_readfirstlane(t.side) / kBig8 == __builtin_amdgcn_readfirstlane(t.share);
    const uint32_t at_touch = mine ? (uint32_t)row_of_lane * (uint32_t)(wave < 4 ? b.row8 : a.H) : kOutOfRange;
    const auto rt = wave < 4 ? rx : rw;
    auto touch = [&](int step) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rt, (lds_void *)(lds8 + kBig8Sink + wave * 256), 4, at_touch, (uint32_t)min(step, b.nb - 1) * 128u, 0, 0);
    };

    f32x4 acc[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    const float *const ws = b.w_scales + ((int64_t)e * ((a.N + 127) / 128) + min(col0 + ww * 128, a.N - 1) / 128) * b.nb;
    const int k0 = (g ^ ((m >> 1) & 7)) * 16, k1 = ((4 + g) ^ ((m >> 1) & 7)) * 16;
    const unsigned char *const pw = lds8 + kBig8 * 128 + (ww * 128 + m) * 128;

    // all steps, NB blocks of 16 rows per wave: the rows of a ragged tile are split evenly over the four rows of waves
    auto run = [&](auto nbc) {
        constexpr int NB = decltype(nbc)::value, kFirstLoads = 2 * NB * 9 / (4 * NB);
        const unsigned char *const px = lds8 + (wx * 16 * NB + m) * 128, *const ps = lds8 + 2 * kBig8 * 128 + (wx * 16 * NB + m) * 4;
        auto fragment = [&](const unsigned char *p, int stage, int block) {
            const u32x4 lo = *reinterpret_cast<const u32x4 *>(p + stage * kBig8Stage + block * 2048 + k0);
            const u32x4 hi = *reinterpret_cast<const u32x4 *>(p + stage * kBig8Stage + block * 2048 + k1);
            return __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        float sw64 = ws[min(lane, b.nb - 1)];                       // the scales of the wave's features: 64 steps at a time, one per lane
#pragma unroll
        for (int l = 0; l < 9; ++l) issue(0, l);
#pragma unroll
        for (int l = 0; l < kFirstLoads; ++l) issue(1, l);          // the rest in the first step
        __builtin_amdgcn_s_waitcnt(0x0f70 | kFirstLoads);
        asm volatile("" : "+v"(sw64));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        i32x8 fx[NB], fw[4];                                       // a column's weights are read two columns ahead
        float sc[NB], raw[NB];                                     // of the present step; of the next, as they are stored
        constexpr int D = 4;                                       // a step's 8 NB products are a multiple of it: the ring begins anew with each
        f32x4 product[D];                                          // the youngest
#pragma unroll
        for (int n = 0; n < D; ++n) product[n] = (f32x4){0.f, 0.f, 0.f, 0.f};
        float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sw64), 0));
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            fx[i] = fragment(px, 0, i);
            raw[i] = *reinterpret_cast<const float *>(ps + i * 64);
            sc[i] = 0.f;
        }
        fw[0] = fragment(pw, 0, 0);
        fw[1] = fragment(pw, 0, 1);
        // scales and adds product number n of a step (row block n % NB, column block n / NB)
        auto add = [&](const f32x4 &p, int n) {
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[n % NB][n / NB][v] = __builtin_fmaf(p[v], sc[n % NB], acc[n % NB][n / NB][v]);
            asm volatile("" : "+v"(acc[n % NB][n / NB]));          // here: moved to the end of the step the products would need 128 registers
        };
        for (int s = 0; s < b.nb; ++s) {
            const int stage = s & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j == 6) {
                    __builtin_amdgcn_s_waitcnt(0x0070 | 1);        // this wave's part of stage s + 1 has landed (younger: a touch), it has read all of stage s
                    asm volatile("" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    if ((s + 1) % 64 == 0) {
                        sw64 = ws[min(s + 1 + lane, b.nb - 1)];
                        asm volatile("" : "+v"(sw64));
                    }
                }
                fw[(j + 2) % 4] = j < 6 ? fragment(pw, stage, j + 2) : fragment(pw, stage ^ 1, j - 6);
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const int n = j * NB + i;
                    f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[j % 4], fx[i], (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                    asm volatile("" : "+v"(p));                    // issued here, not where its result is used
                    if (n < D) {
                        const int old = 8 * NB + n - D;
                        add(product[n % D], old);
                        if (old >= 7 * NB) sc[old % NB] = raw[old % NB] * sw;      // a row block's new scale, behind its last product of the step before
                    } else {
                        add(product[n % D], n - D);
                    }
                    product[n % D] = p;
                    if (j == 7) {
                        fx[i] = fragment(px, stage ^ 1, i);
                        raw[i] = *reinterpret_cast<const float *>(ps + (stage ^ 1) * kBig8Stage + i * 64);
                    }
                    // the loads of step s + 2 begin behind the barrier and end in the second column of step s + 1: as a burst they would hold up the wave
                    const int slot = (j + 2) % 8 * NB + i;
                    if (slot < 4 * NB) {
#pragma unroll
                        for (int l = slot * 9 / (4 * NB); l < (slot + 1) * 9 / (4 * NB); ++l) issue(j >= 6 ? s + 2 : s + 1, l);
                    } else if (slot == 4 * NB) {
                        touch(s + 2);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sw64), (s + 1) % 64));
        }
#pragma unroll
        for (int n = 8 * NB - D; n < 8 * NB; ++n) add(product[n % D], n);
    };
    const int nb = (row_end - row0 + 63) / 64;                     // more than 128 rows
    if (nb == 3) run(std::integral_constant<int, 3>{});
    else run(std::integral_constant<int, 4>{});

    // acc[i][j][v]: row 16 i + lane % 16 of the wave's rows, output feature 16 j + 4 (lane / 16) + v of its columns.  Through LDS, block of 16 rows
    // by block, so that rows leave as whole pieces of 16 bytes, 256 bytes of each side by side.
    __builtin_amdgcn_s_waitcnt(0x0070);                            // the loads past the end have come back
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();                                  // and nobody reads the stages any more
    asm volatile("" ::: "memory");
    constexpr int kOutPitch = 256 + 16;
    static_assert(kBig8Sink + 2048 <= kBig8LdsBytes && 8 * 16 * kOutPitch <= kBig8LdsBytes, "8-bit large tile: room for a block of rows per wave");
    unsigned char *const own = lds8 + wave * (16 * kOutPitch);
    __bf16 *const to = y + col0 + ww * 128;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= nb) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            bf16x4 o;
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = (__bf16)acc[i][j][v];
            *reinterpret_cast<bf16x4 *>(own + m * kOutPitch + j * 32 + g * 8) = o;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = q * 4 + (lane >> 4), p = lane & 15;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(own + row * kOutPitch + p * 16);
            const int64_t r = row0 + wx * 16 * nb + i * 16 + row;
            if (r < row_end && col0 + ww * 128 + p * 8 < a.N) *reinterpret_cast<u32x4 *>(to + r * a.N + p * 8) = v;
        }
    }
}

template <bool RAGGED_LAST, bool TAIL>
__global__ __launch_bounds__(512, 2) void expert8_big_kernel(const unsigned char *__restrict__ x, const unsigned char *__restrict__ w, __bf16 *__restrict__ y,
                                                             Expert8Args b)
{
    extern __shared__ __align__(16) unsigned char lds8[];
    const RowTile t = find_row_tile<kBig8, RAGGED_LAST>(b.a, (b.a.N + kBig8 - 1) / kBig8, blockIdx.x, threadIdx.x & 63, reinterpret_cast<int *>(lds8));
#if defined(__HIP_DEVICE_COMPILE__)
    expert8_big_tile<RAGGED_LAST, TAIL>(x, w, y, b, t, lds8);
#else
    (void)x;
    (void)w;
    (void)y;
    (void)t;
#endif
}

template <int XR, int WR, int WX, int WW, int NST, bool F32>
int launch_expert8(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, hipStream_t st)
{
    using G = Tile8<XR, WR, WX, WW, NST>;
    const int64_t row_tiles = rows_bound / XR + std::min<int64_t>(b.a.E, rows_bound), nct = (b.a.N + WR - 1) / WR;
    const int64_t grid = (row_tiles * nct + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds);
    if (!launchable(grid, G::kThreads)) return MONTA_ERR_UNSUPPORTED;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(expert8_kernel<XR, WR, WX, WW, NST, F32>), G::kLdsBytes, lds_opt_in)) return rc;
    hipLaunchKernelGGL((expert8_kernel<XR, WR, WX, WW, NST, F32>), dim3((unsigned)grid), dim3(G::kThreads), G::kLdsBytes, st,
                       static_cast<const unsigned char *>(x), static_cast<const unsigned char *>(w), y, b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <int CB, int W, int D, bool F32>
int launch_expert8_split(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, hipStream_t st)
{
    const int64_t row_tiles = rows_bound / 16 + std::min<int64_t>(b.a.E, rows_bound), nct = (b.a.N + 16 * CB - 1) / (16 * CB);
    const int64_t grid = (row_tiles * nct + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds);
    if (!launchable(grid, 64 * W)) return MONTA_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((expert8_split_kernel<CB, W, D, F32>), dim3((unsigned)grid), dim3(64 * W), 0, st, static_cast<const unsigned char *>(x),
                       static_cast<const unsigned char *>(w), y, b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <bool RAGGED_LAST, bool TAIL>
int launch_expert8_big_k(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, hipStream_t st)
{
    constexpr int lds = kBig8LdsBytes;
    const int64_t nct = (b.a.N + kBig8 - 1) / kBig8, row_tiles = rows_bound / kBig8 + std::min<int64_t>(b.a.E, rows_bound);
    const int64_t tiles = (row_tiles + (RAGGED_LAST ? b.a.E : 0)) * nct;              // short ragged tiles come in halves
    const int64_t grid = (tiles + 32 * kXcds - 1) / (32 * kXcds) * (32 * kXcds);
    if (!launchable(grid, 512)) return MONTA_ERR_UNSUPPORTED;
    static LdsOptIn lds_opt_in;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(expert8_big_kernel<RAGGED_LAST, TAIL>), lds, lds_opt_in)) return rc;
    hipLaunchKernelGGL((expert8_big_kernel<RAGGED_LAST, TAIL>), dim3((unsigned)grid), dim3(512), lds, st, static_cast<const unsigned char *>(x),
                       static_cast<const unsigned char *>(w), static_cast<__bf16 *>(y), b);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

template <bool RAGGED_LAST>
int launch_expert8_big(const void *x, const void *w, void *y, const Expert8Args &b, int64_t rows_bound, hipStream_t st)
{
    return b.a.H % 128 ? launch_expert8_big_k<RAGGED_LAST, true>(x, w, y, b, rows_bound, st) : launch_expert8_big_k<RAGGED_LAST, false>(x, w, y, b, rows_bound, st);
}

// Which tile.  Measured on MI355X, three sets of buffers in turn, us; tokens x hidden x features, experts, top-2 (64 experts: top-8), in tiles of
// 32 x 64, 32 x 128, 64 x 128, 128 x 128 and 256 x 256:
//   1 x 4096 x 4096, 8      13   16   20   26   30         256 x 1024 x 1024, 8     9.3  7.3  9.3  11   16
//   64 x 4096 x 4096, 8     31   35   36   38   41         2048 x 512 x 512, 4      7.6  6.1  9.5  10   14
//   256 x 4096 x 4096, 8    49   47   45   44   50         4096 x 1024 x 512, 32    24   22   20   18   22
//   512 x 4096 x 4096, 8    75   70   62   60   59         512 x 2048 x 1024, 64    51   45   41   35   35
//   1024 x 4096 x 4096, 8   127  112  86   88   68         256 x 2048 x 1024, 64    36   35   28   29   30
//   2048 x 4096 x 4096, 8   229  197  144  124  120        512 x 7168 x 2048, 64    296  255  223  196  186
//   16 x 7168 x 2048, 64    134  143  143  149  143        1024 x 7168 x 2048, 64   475  399  322  289  228
// 256 x 256 with the ragged tiles in place and last, those of at most 64 rows by halves: an even load leaves each expert whole tiles and a few
// rows, which then share the last round, but read the weights again:
//   2048 x 4096 x 4096, 8  120  92   (load skewed 70   71)     8192 x 4096 x 4096, 16  310  305
//   4096 x 7168 x 2048, 8  187  137                           4096 x 2048 x 2048, 16  71   52   (35   41)
//   8192 x 4096 x 4096, 8  313  303                           4096 x 4096 x 2048, 32           (118  134)
//   8192 x 8192 x 8192, 2  519  507                           4096 x 7168 x 2048, 64  566  613  (352  388)
// Few tiles: those of 32 x 64, and split ones of 16 x 16 by 8 waves and 16 x 32 by 4 (calls of one graph, one after the other):
//   1 x 4096 x 4096, 8     13.7 9.0  9.0                      1 x 1024 x 1024, 8      5.9  3.9  4.3
//   1 x 4096 x 1024, 8     12.9 5.9  7.9                      1 x 512 x 4096, 8       4.3  4.0  4.0
//   3 x 8192 x 552, top-1  21.9 8.2  12                       40 x 2048 x 512, 4      8.6  5.3  6.0
//   8 x 8192 x 2048, top-1 22.5 17.1 18.9                     100 x 4096 x 512, 4     13.6 12.5 9.8
//   8 x 4096 x 4096, 8     24   28   30                       196 x 2048 x 88, 8      8.4  7.5  6.1
//   1 x 7168 x 2048, 64    24.6 26.1 26.3                     64 x 2048 x 2048, 8     8.9  22   16
//   60 x 4096 x 2048, top-1, 4  13.9 16.7                     60 x 4096 x 1024, 2     13.6 -    9.4
//   4 x 512 x 512, 64      4.4  5.0                           256 x 2048 x 256, 8     8.6  -    9.2
// Walks that start at different steps (walk_start) on weights' rows of whole 4 KiB, in 32 x 64: 64 x 4096 x 4096, 8 31.0 and 26.4 us, 8 tokens 27.5 and
// 23.7; but 256 tokens 49.1 and 49.3, rows of 7168 133.8 and 139.3.
template <bool F32>
int launch_expert8_tiled(const void *x, const void *w, void *y, Expert8Args b, int64_t rows_bound, int64_t kept_bound, int slice, hipStream_t st)
{
    // of the whole problem, also for a slice: it then runs as the whole would, and its rows are the same bit for bit
    const int64_t active = std::min<int64_t>(b.a.E, kept_bound), r = kept_bound / active;
    auto tiles = [&](int64_t R, int64_t C) { return active * ((b.a.N + C - 1) / C) * (2 * r + R) / (2 * R); };
    auto split_tiles = [&](int64_t C) { return active * ((b.a.N + C - 1) / C) * std::max<int64_t>(2 * r + 16, 32) / 32; };
    if (r <= 24 && split_tiles(16) <= (r <= 8 && b.nb >= 8 ? 1024 : 512)) return launch_expert8_split<1, 8, 2, F32>(x, w, y, b, rows_bound, st);
    if (split_tiles(32) <= (b.nb >= 32 ? 512 : 256)) return launch_expert8_split<2, 4, 4, F32>(x, w, y, b, rows_bound, st);
    if (r <= 24 || tiles(32, 64) <= 160) {
        b.a.spread = b.a.H % 4096 == 0;
        return launch_expert8<32, 64, 1, 4, 4, F32>(x, w, y, b, rows_bound, st);
    }
    if constexpr (!F32) {
        if (tiles(32, 128) <= 300) return launch_expert8<32, 128, 1, 4, 3, F32>(x, w, y, b, rows_bound, st);
        if (r > 48 && tiles(256, 256) >= 120) {
            // ragged tiles last: whole segments only, the search needs their lengths
            const bool ragged_last = slice < 0 && r > 384 && (int64_t)b.a.E * ((b.a.N + kBig8 - 1) / kBig8) < 256;
            return ragged_last ? launch_expert8_big<true>(x, w, y, b, rows_bound, st) : launch_expert8_big<false>(x, w, y, b, rows_bound, st);
        }
    }
    if (r > 48 && tiles(128, 128) >= 200) return launch_expert8<128, 128, 2, 2, 2, F32>(x, w, y, b, rows_bound, st);
    return launch_expert8<64, 128, 1, 4, 3, F32>(x, w, y, b, rows_bound, st);
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
    if (c.H > kMaxHidden8 || out_features > kBigMaxHidden || c.max_rows > kMostRows) return MONTA_ERR_UNSUPPORTED;
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
    return c.bf16 ? launch_expert8_tiled<false>(x_rows, w_codes, y, b, rows_bound, c.kept_bound, slice, st)
                  : launch_expert8_tiled<true>(x_rows, w_codes, y, b, rows_bound, c.kept_bound, slice, st);
}
