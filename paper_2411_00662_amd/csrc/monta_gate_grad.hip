// Gradients of the gate projection, by the tokens' rows and by the weights:
//   dx[t][h] = sum_e dl[t][e] w[e][h] + dadd[t][h],     dw[e][h] = sum_t dl[t][e] x[t][h].
// Few experts against many hidden elements: bound by reading x and dadd and writing dx once, as long as the products keep up.
#include "monta_internal.hpp"

#include <algorithm>

namespace monta {
namespace {

struct GateGradArgs {
    const float *dl;
    const void *x, *w, *dadd;
    void *dx;
    float *dw;              // the sums of each share of the tokens, [shares][E][H]; with one share the result
    int64_t T;
    int32_t E, H;
    int32_t blocks, shares;             // column blocks; shares of the tokens
};

// What workgroup `block` does: column block `col`, and of the steps of tokens every `shares`-th from the one numbered `share` on.  All workgroups so move through
// the rows together, in one window of them for each buffer: with a run of neighbouring steps for each share 65536 x 7168 over 8 experts took 373 us in 18 runs and
// 344 in nine, so 363 and 331.  Consecutive workgroups, which go to the XCDs in turn, have consecutive column blocks of a share: 369 us for 64 experts, 383 with
// all blocks of a share on one XCD, although each XCD so reads dl for itself (both with two parts of dl for dx instead of three).
struct GatePart {
    int share, col;
};
__device__ __forceinline__ GatePart gate_part(const GateGradArgs &a, uint32_t block, int width)
{
    GatePart p;
    p.share = (int)(block / (uint32_t)a.blocks);
    p.col = (int)(block % (uint32_t)a.blocks) * width;
    return p;
}

// --------------------------------------------------------------------------------------------- fp32
//
// fp32 activations: fp32 products on the matrix cores (16 x 16 x 4).  A wave has 16 CT columns of a step's 16 tokens and the
// weights of its columns in registers; the gradient of the logits, which all waves of the workgroup need in both orders, goes through LDS.
//   dx: rows h, columns t, summed over e: a lane gets 4 neighbours of one token, four lanes 64 bytes.
//   dw: rows h, columns e, summed over t.  Row r of tile i is column CT r + i, so that a lane's elements of x are neighbours.
// Up to 32 experts bound by memory (8192 x 4096, 8 experts, dadd: 402 MB in 76 us with the sums of the shares, 5.3 TB/s), from 64 on by the products, which the 16 of
// a tile's columns or the 4 of its sum that are no experts cost too (64 experts 107 us, 80 TFLOP/s of products; a large library product reaches 151).

template <int EB>
constexpr int tiles_of() { return EB <= 4 ? 4 : 16 / EB; }

template <int N>
struct Piece {                  // N neighbouring elements of a row
    static_assert(N == 1 || N == 2 || N == 4, "piece: elements");
    typedef float V __attribute__((ext_vector_type(N == 1 ? 2 : N)));       // one alone is kept in the first of two
    V v;
    __device__ __forceinline__ void clear() { v = (V)0.f; }
    __device__ __forceinline__ void get(const float *p)
    {
        if constexpr (N == 1) v[0] = *p;
        else v = *reinterpret_cast<const V *>(p);
    }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};

constexpr int kStepTokens = 16;

template <int EB>
__global__ __launch_bounds__(256, 2) void gate_backward_f32_kernel(GateGradArgs a)
{
    constexpr int CT = tiles_of<EB>(), CW = 16 * CT, kPitch = 16 * EB + 4;
    __shared__ float dlt[2][kStepTokens][kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, g = lane >> 4;
    const GatePart part = gate_part(a, blockIdx.x, 4 * CW);
    const int64_t H = a.H;
    const int col = part.col + wave * CW;                          // first column of the wave
    const bool want_dx = a.dx != nullptr, want_dw = a.dw != nullptr;
    const float *const in = static_cast<const float *>(a.x), *const weights = static_cast<const float *>(a.w), *const dadd = static_cast<const float *>(a.dadd);
    float *const to_dx = static_cast<float *>(a.dx);

    f32x4 sum[EB][CT];
#pragma unroll
    for (int j = 0; j < EB; ++j)
#pragma unroll
        for (int i = 0; i < CT; ++i) sum[j][i] = (f32x4){0.f, 0.f, 0.f, 0.f};

    float dl[EB];
    Piece<CT> x[4];
    Piece<4> add[CT];
    auto fetch = [&](int64_t t0) {
        const int64_t t = t0 + (tid >> 4);
#pragma unroll
        for (int q = 0; q < EB; ++q) {
            const int e = (tid & 15) + 16 * q;
            dl[q] = t < a.T && e < a.E ? a.dl[t * a.E + e] : 0.f;
        }
        if (want_dw)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int64_t at = t0 + 4 * s + g;
                x[s].clear();
                if (at < a.T && col + m * CT < a.H) x[s].get(in + at * H + col + m * CT);
            }
        if (want_dx)
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const int h = col + 16 * i + 4 * g;
                add[i].clear();
                if (a.dadd && t0 + m < a.T && h < a.H) add[i].get(dadd + (t0 + m) * H + h);
            }
    };
    const int64_t first = (int64_t)part.share * kStepTokens, stride = (int64_t)a.shares * kStepTokens;
    fetch(first);
    float w[CT][4 * EB];
    if (want_dx)
#pragma unroll
        for (int kk = 0; kk < 4 * EB; ++kk)
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const int e = 4 * kk + g, h = col + 16 * i + m;
                w[i][kk] = e < a.E && h < a.H ? weights[e * H + h] : 0.f;
            }
    int buf = 0;
    for (int64_t t0 = first; t0 < a.T; t0 += stride, buf ^= 1) {
#pragma unroll
        for (int q = 0; q < EB; ++q) dlt[buf][tid >> 4][(tid & 15) + 16 * q] = dl[q];
        Piece<CT> x0[4];
        f32x4 out[CT];
#pragma unroll
        for (int s = 0; s < 4; ++s) x0[s] = x[s];
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) out[i][v] = add[i][v];
        __syncthreads();                                           // of two buffers the other one has been read by all before this
        if (t0 + stride < a.T) fetch(t0 + stride);
        if (want_dx) {
#pragma unroll
            for (int kk = 0; kk < 4 * EB; ++kk) {
                const float b = dlt[buf][m][4 * kk + g];
#pragma unroll
                for (int i = 0; i < CT; ++i) out[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i][kk], b, out[i], 0, 0, 0);
            }
            if (t0 + m < a.T)
#pragma unroll
                for (int i = 0; i < CT; ++i) {
                    const int h = col + 16 * i + 4 * g;
                    if (h >= a.H) continue;
                    *reinterpret_cast<f32x4 *>(to_dx + (t0 + m) * H + h) = out[i];
                }
        }
        if (want_dw)
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int j = 0; j < EB; ++j) {
                    const float b = dlt[buf][4 * s + g][16 * j + m];
#pragma unroll
                    for (int i = 0; i < CT; ++i) sum[j][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x0[s][i], b, sum[j][i], 0, 0, 0);
                }
    }
    if (want_dw)
#pragma unroll
        for (int j = 0; j < EB; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int e = 16 * j + m, h = col + (4 * g + v) * CT;
                if (e >= a.E || h >= a.H) continue;
                float *const to = a.dw + ((int64_t)part.share * a.E + e) * H + h;
#pragma unroll
                for (int i = 0; i < CT; ++i) to[i] = sum[j][i][v];
            }
}

// --------------------------------------------------------------------------------------------- bf16
//
// bf16 activations on the bf16 matrix instruction (16 x 16 x 32).  A gradient of a logit is split into three bf16 numbers
// of 8 bits each, whose products are exact: fp32 sums of dw, and of dx until it is rounded, since experts may cancel each other, or dadd their sum (with two of the
// three dx would be off by 2^-16 of its terms).  A step is 32 tokens; a wave has 64 columns of it.
//   dx: rows h, columns t, summed over e.  The wave keeps the weights of its columns in registers.  Row r of tile i is column 32 (i / 2) + 8 (r / 4)
//       + 4 (i % 2) + r % 4, so that a lane gets 8 neighbours of one token and four lanes 64 bytes.
//   dw: rows h, columns e, summed over t.  Both operands lie across the summed axis: they are kept in LDS as they come, rows of 32 bytes' segments, and
//       read by the transposing LDS read, as in the experts' gradients.  A wave's x is its own, straight from memory to LDS in a ring of stages; the
//       split gradients are the workgroup's, in two buffers, so that a step has one barrier.
// dx takes the place of the step's x in LDS, the same lanes' both, and leaves in whole lines of 128 bytes past the cache: in halves of lines, as the products leave
// it, storing alone took 282 us of 65536 x 7168 over 8 experts, so 184.
// Loads and stores go through descriptors that end at the last token, and lanes past the last column hand in an address past every descriptor: no
// branch, every step issues the same number of them, also past the end, and the wait for a stage of x counts the younger ones.
// 65536 x 7168, 64 experts: 1.9 GB in 400 to 415 us in a run of calls, 4.6 to 4.7 TB/s (the first three at the full clock 375, those after them up to 560, until the
// clock has settled), of which the matrix pipe is busy 42 %; 8 experts 330 (5.7); 8192 x 4096, 8 experts, dadd: 201 MB in 36 us and 3 for the sums of the shares.  (fp32
// products 1552 and 58.  With two parts of dl for dx 64 experts take 375, 32 327 for 338, 8 as long.)

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kSplitTokens = 32, kStages = 3;      // tokens of a step; stages of x
// x, dadd and dx go past the cache, whatever their size.  us, so and through it, alone and with the layer norm's gradient behind, which reads dx: 600 x 4096 9.9 / 22.3 and
// 9.9 / 21.8, 4096 x 4096 23.4 / 53.9 and 22.8 / 54.0 (but 53 and 48.5 where all buffers stay in the cache), 8192 x 4096 39.0 / 89 and 41.1 / 90, 12288 x 4096 55.0 / 125
// and 57.9 / 127.
[[maybe_unused]] constexpr int kNt = 2;

// Segment s of row k sits at s ^ row_swizzle<C>(k) in rows of C elements: the 8 rows (8 g + j, g = 0, 1, j = 0..3) of which half a wave reads a
// segment each are then in different banks.
template <int C>
__device__ __forceinline__ constexpr int row_swizzle(int k)
{
    if constexpr (C == 32) return (k >> 3) & 1;
    else if constexpr (C == 64) return ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
    else return (k & 3) | ((k >> 3) & 1) << 2;
}

// __restrict__ here and below: without alias information on an access to LDS the compiler waits for every outstanding load to LDS before it.
[[maybe_unused]] __device__ __forceinline__ bf16x8 read_across(lds_s16x4 *__restrict__ p, int four_rows)
{
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(reinterpret_cast<__attribute__((address_space(3))) char *>(p) + four_rows));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
[[maybe_unused]] __device__ __forceinline__ bf16x8 read_along(lds_bf16x8 *__restrict__ p) { return *p; }
[[maybe_unused]] __device__ __forceinline__ void put(lds_u32x4 *__restrict__ p, u32x4 v) { *p = v; }

// Eight neighbours of dl as three bf16 numbers each, one piece `pitch` bytes behind the other: the upper 8 of a number's 24 bits, the next 8 and the rest.  They are
// cut off, not rounded: no finite number becomes an infinity.
template <int pitch>
[[maybe_unused]] __device__ __forceinline__ void split_eight(const f32x4 (&dl)[2], unsigned char *to)
{
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(dl[i / 4][i % 4]);
#pragma unroll
    for (int piece = 0; piece < 3; ++piece) {
        u32x4 b;
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302u);      // the upper halves of two
        if (piece < 2)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) - __uint_as_float(v[i] & 0xffff0000u));
        put((lds_u32x4 *)(to + piece * pitch), b);
    }
}

// The weights of BC columns from `col` on, rows of experts, zeros past the last expert and column, to LDS by all waves.
template <int EP, int BC, int kThreads>
[[maybe_unused]] __device__ __forceinline__ void fetch_weights(const GateGradArgs &a, int col, unsigned char *lds, int wave, int lane)
{
    constexpr int kLoads = EP * BC * 2 / 16 / kThreads, kPerRow = BC / 8;
    const uint32_t pitch = (uint32_t)a.H * 2;
    const auto from = make_rsrc(static_cast<const __bf16 *>(a.w) + col, a.dx ? (uint32_t)a.E * pitch - (uint32_t)col * 2u : 0u);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int at = (wave * kLoads + q) * 64 + lane, row = at / kPerRow, p = at % kPerRow;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)(lds + (wave * kLoads + q) * 1024), 16,
                                                 col + p * 8 < a.H ? (uint32_t)row * pitch + (uint32_t)p * 16u : kOutOfRange, 0, 0, 0);
    }
}

// Tile i of those, experts 32 ks to 32 ks + 31, of the columns from `first` on: row r is column 32 (i / 2) + 8 (r / 4) + 4 (i % 2) + r % 4 of them.
template <int BC>
[[maybe_unused]] __device__ __forceinline__ bf16x8 weight_fragment(unsigned char *lds, int first, int ks, int i, int m, int g)
{
    return read_across((lds_s16x4 *)(lds + (32 * ks + 8 * g + (m >> 2)) * (2 * BC) + first * 2 + i / 2 * 64 + (m & 3) * 16 + i % 2 * 8), 4 * 2 * BC);
}

template <int EB, int NW>
struct GateShape {
    static_assert(EB <= 4, "gate gradient: experts");
    static constexpr int CT = 4, NST = kStages;
    static constexpr int kThreads = 64 * NW, CW = 16 * CT, BC = NW * CW;        // columns of a wave, of a workgroup of NW
    static constexpr int EP = EB == 1 ? 32 : 16 * EB;               // experts, in whole steps of the sum of dx
    static constexpr int KS = EP / 32;
    static constexpr int kRow = 2 * EP, kPiece = kSplitTokens * kRow, kDl = 3 * kPiece;
    static constexpr int kRowX = 2 * CW, kX = kSplitTokens * kRowX;
    static constexpr int kStage = NW * kX, kLdsX = NST * kStage, kLdsBytes = kLdsX + 2 * kDl;
    static constexpr int kWeights = EP * BC * 2, kAtWeights = kLdsBytes - kWeights;      // before the first step, behind its stage
    static constexpr int kItems = kSplitTokens * EP / 8, kItemsEach = (kItems + kThreads - 1) / kThreads;      // 8 neighbours of dl
    static constexpr int kLoadsX = kX / 1024, kPerRowX = CW / 8;
    static constexpr int kOut = CT / 2;                             // pieces of a token's columns in a lane
    // accesses that every step issues after a stage's: the stages behind it, dadd and stores.  (dl is waited for by its use, and a wave
    // without a part in it may skip its loads.)
    static constexpr int kSurely = (NST - 2) * kLoadsX + 2 * 2 * kOut;
    static constexpr int kLate = (NST - 2) * kLoadsX + 2 * kOut + 2 * kItemsEach;           // those that need not have come back: the stages, the stores, dl
    static constexpr int kYounger = kLate < kSurely ? kLate : kSurely;
    static constexpr int wait_for(int vmcnt) { return 0x0070 | (vmcnt & 15) | ((vmcnt >> 4) << 14); }      // and lgkmcnt(0)
    static_assert(NST >= 3 && kYounger < 64 && kAtWeights >= kStage, "gate gradient: stages");
};

template <int EB, int NW>
__global__ __launch_bounds__(64 * NW, 2) void gate_backward_bf16_kernel([[maybe_unused]] GateGradArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = GateShape<EB, NW>;
    constexpr int CT = G::CT, NST = kStages;
    extern __shared__ __align__(16) unsigned char gate_lds[];
    unsigned char *const lds_x = gate_lds, *const lds_dl = gate_lds + G::kLdsX;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const GatePart part = gate_part(a, blockIdx.x, G::BC);
    const int col = part.col + wave * G::CW, H = a.H, E = a.E;
    const uint32_t pitch = (uint32_t)H * 2;
    const bool whole4 = (E & 3) == 0;
    // what a descriptor may reach of `rows` rows, from the first one's column `col` on: nothing of no rows, and nothing past the last column
    auto bytes_of = [&](int rows) { return rows > 0 && col < H ? (uint32_t)rows * pitch - (uint32_t)col * 2u : 0u; };

    f32x4 sum[EB][CT];
#pragma unroll
    for (int j = 0; j < EB; ++j)
#pragma unroll
        for (int i = 0; i < CT; ++i) sum[j][i] = (f32x4){0.f, 0.f, 0.f, 0.f};

    // this lane's places in a step: of x and dx, of dadd
    uint32_t at_x[G::kLoadsX], at_o[2][G::kOut];
#pragma unroll
    for (int q = 0; q < G::kLoadsX; ++q) {                         // the place in LDS is fixed by the instruction, so the swizzle is applied here
        const int row = (q * 64 + lane) / G::kPerRowX, at = lane % G::kPerRowX, p = ((at >> 1) ^ row_swizzle<G::CW>(row)) * 2 + (at & 1);
        at_x[q] = col + p * 8 < H ? (uint32_t)row * pitch + (uint32_t)p * 16u : kOutOfRange;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int q = 0; q < G::kOut; ++q) {
            const int h = 32 * q + 8 * g;
            at_o[half][q] = col + h < H ? (uint32_t)(16 * half + m) * pitch + (uint32_t)h * 2u : kOutOfRange;
        }

    unsigned char *const my_x = lds_x + wave * G::kX;
    const int64_t first = (int64_t)part.share * kSplitTokens, stride = (int64_t)a.shares * kSplitTokens;
    auto rows_at = [&](int64_t t0) { return __builtin_amdgcn_readfirstlane((int)max((int64_t)0, min((int64_t)kSplitTokens, a.T - t0))); };
    auto issue = [&](int64_t t0, int stage) {
        const int rows = rows_at(t0);
        const auto from = make_rsrc(static_cast<const __bf16 *>(a.x) + (t0 * H + col), a.dw ? bytes_of(rows) : 0u);
#pragma unroll
        for (int q = 0; q < G::kLoadsX; ++q) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)(my_x + stage + q * 1024), 16, at_x[q], 0, 0, kNt);
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    u32x4 add[2][G::kOut];
    f32x4 dl[G::kItemsEach][2];
    auto fetch_dl = [&](int64_t t0) {
        const int rows = rows_at(t0);
        const auto from_dl = make_rsrc(a.dl + t0 * E, (uint32_t)rows * (uint32_t)E * 4u);
#pragma unroll
        for (int n = 0; n < G::kItemsEach; ++n) {
            const int item = tid + G::kThreads * n, row = item / (G::EP / 8), e0 = item % (G::EP / 8) * 8;
            const uint32_t at = ((uint32_t)row * (uint32_t)E + (uint32_t)e0) * 4u;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                if (whole4) {
                    dl[n][v] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_dl, row < kSplitTokens && e0 + 4 * v < E ? at + 16u * v : kOutOfRange, 0, 0));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dl[n][v][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                            from_dl, row < kSplitTokens && e0 + 4 * v + i < E ? at + 16u * v + 4u * i : kOutOfRange, 0, 0));
                }
            }
        }
    };
    auto fetch_add = [&](int64_t t0) {
        const int rows = rows_at(t0);
        const auto from_add = make_rsrc(static_cast<const __bf16 *>(a.dadd) + (t0 * H + col), a.dadd ? bytes_of(rows) : 0u);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int q = 0; q < G::kOut; ++q) add[half][q] = __builtin_amdgcn_raw_buffer_load_b128(from_add, at_o[half][q], 0, kNt);
    };

    // this lane's places in LDS: row 8 g + m / 4, quarter m % 4 of a segment, for what is read across; row m, half g % 2 of a segment along
    const int ka = 8 * g + (m >> 2), across_x = ka * G::kRowX + (m & 3) * 8, across_dl = ka * G::kRow + (m & 3) * 8, along_dl = m * G::kRow + (g & 1) * 16;
    const int sx = row_swizzle<G::CW>(ka) * 32, sd = row_swizzle<G::EP>(ka) * 32, sl = row_swizzle<G::EP>(m) * 32, so = row_swizzle<G::CW>(m) * 32;

    auto split = [&](unsigned char *to_dl) {
#pragma unroll
        for (int n = 0; n < G::kItemsEach; ++n) {
            const int item = tid + G::kThreads * n, row = item / (G::EP / 8), p = item % (G::EP / 8);
            if (G::kItems % G::kThreads == 0 || item < G::kItems)
                split_eight<G::kPiece>(dl[n], to_dl + row * G::kRow + ((p >> 1) ^ row_swizzle<G::EP>(row)) * 32 + (p & 1) * 16);
        }
    };
    issue(first, 0);
    fetch_weights<G::EP, G::BC, G::kThreads>(a, part.col, gate_lds + G::kAtWeights, wave, lane);
    fetch_dl(first);
    fetch_add(first);
    __builtin_amdgcn_s_waitcnt(0x0070);
    barrier();
    bf16x8 w[G::KS][CT];
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
        for (int i = 0; i < CT; ++i) w[ks][i] = weight_fragment<G::BC>(gate_lds + G::kAtWeights, wave * G::CW, ks, i, m, g);
    __builtin_amdgcn_s_waitcnt(0xc07f);                            // lgkmcnt(0): read by this wave, and behind the barrier by all
    barrier();
#pragma unroll
    for (int q = 1; q < NST - 1; ++q) issue(first + q * stride, q * G::kStage);
    int buf = 0, stage = 0;
    split(lds_dl);
    fetch_dl(first + stride);
    for (int64_t t0 = first; t0 < a.T; t0 += stride) {
        f32x4 out[2][CT];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < CT; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const uint32_t word = add[half][i / 2][i % 2 * 2 + v / 2];
                    out[half][i][v] = __uint_as_float(v % 2 ? word & 0xffff0000u : word << 16);
                }
        __builtin_amdgcn_s_waitcnt(G::wait_for(G::kYounger));                      // this step's x has landed, this wave's part of dl is written
        barrier();                                                 // of two buffers of dl the other one has been read by all before this
        fetch_add(t0 + stride);
        issue(t0 + (NST - 1) * stride, stage == 0 ? (NST - 1) * G::kStage : stage - G::kStage);       // where the step before was

        const unsigned char *const dls = lds_dl + buf;
        unsigned char *const xs = my_x + stage;
        bf16x8 fx[CT];
#pragma unroll
        for (int i = 0; i < CT; ++i) fx[i] = read_across((lds_s16x4 *)(xs + across_x + ((i * 32) ^ sx)), 4 * G::kRowX);
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
            for (int piece = 0; piece < 3; ++piece)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bf16x8 b = read_along((lds_bf16x8 *)(dls + piece * G::kPiece + half * 16 * G::kRow + along_dl + (((2 * ks + (g >> 1)) * 32) ^ sl)));
#pragma unroll
                    for (int i = 0; i < CT; ++i) out[half][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[ks][i], b, out[half][i], 0, 0, 0);
                }
        // dx takes the place of x, in the same layout, and leaves it in whole lines
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int q = 0; q < G::kOut; ++q) {
                bf16x8 o;
#pragma unroll
                for (int v = 0; v < 8; ++v) o[v] = (__bf16)out[half][2 * q + v / 4][v % 4];
                const int c = 4 * q + g;                           // its piece of the row
                put((lds_u32x4 *)(xs + (16 * half + m) * G::kRowX + ((c >> 1) * 32 ^ so) + (c & 1) * 16), __builtin_bit_cast(u32x4, o));
            }
        {
            const auto to = make_rsrc(static_cast<__bf16 *>(a.dx) + (t0 * H + col), a.dx ? bytes_of(rows_at(t0)) : 0u);
#pragma unroll
            for (int q = 0; q < G::kLoadsX; ++q)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, read_along((lds_bf16x8 *)(xs + q * 1024 + lane * 16))), to, at_x[q], 0, kNt);
        }
#pragma unroll
        for (int j = 0; j < EB; ++j)
#pragma unroll
            for (int piece = 0; piece < 3; ++piece) {
                const bf16x8 b = read_across((lds_s16x4 *)(dls + piece * G::kPiece + across_dl + ((j * 32) ^ sd)), 4 * G::kRow);
#pragma unroll
                for (int i = 0; i < CT; ++i) sum[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i], b, sum[j][i], 0, 0, 0);
            }
        buf ^= G::kDl;
        split(lds_dl + buf);                                       // for the next step, among this one's products
        fetch_dl(t0 + 2 * stride);
        stage = stage == (NST - 1) * G::kStage ? 0 : stage + G::kStage;
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                            // the loads past the end have come back: the LDS is another workgroup's after this
    if (a.dw)
#pragma unroll
        for (int j = 0; j < EB; ++j)
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const int e = 16 * j + m, h = col + 16 * i + 4 * g;
                if (e < E && h < H) *reinterpret_cast<f32x4 *>(a.dw + ((int64_t)part.share * E + e) * H + h) = sum[j][i];
            }
#endif
}

// More than 64 experts: what is read from LDS for each product grows with the experts that a wave has, so eight waves share both sums another way.
//   dw: a wave has 64 experts and 64 columns.
//   dx: a wave has 16 tokens of the step, all experts and a quarter of the workgroup's columns; the rows leave a step later, when all waves have written
//       their parts of them.
// 16384 x 4096 with dadd, 256 experts: 201 us, 128 experts 113: 1.03 and 0.91 PFLOP/s of bf16 products, the matrix pipe busy 49 and 43 % of the time; the steps of
// both waves of a SIMD are in step.  (With two parts of dl for dx 183 and 103, and in waves of 32 columns, all experts, 283.)
template <int EB>
struct GateWide {
    static_assert(EB == 8 || EB == 16, "wide gate gradient: experts");
    static constexpr int NST = kStages, kWaves = 8, kThreads = 64 * kWaves, kGroups = EB / 4, kColumnGroups = kWaves / kGroups, BC = 64 * kColumnGroups;
    static constexpr int DC = BC / 4, CD = DC / 16, kOut = CD / 2;  // columns of a wave's part of dx, tiles, pieces of 16 bytes in a lane
    static constexpr int EP = 16 * EB, KS = EP / 32;
    static constexpr int kRow = 2 * EP, kPiece = kSplitTokens * kRow, kDl = 3 * kPiece, kItemsEach = kSplitTokens * EP / 8 / kThreads;
    static constexpr int kRowX = 2 * BC, kX = kSplitTokens * kRowX, kLoadsX = kX / 1024 / kWaves, kPerRowX = BC / 8;
    // the next step's dl is split before dw's products or after them, and the one after it requested then: 16384 x 4096, 256 experts 201 us and 220, 128 experts 113.4 and 112.5
    static constexpr bool kSplitEarly = EB == 16;
    static constexpr int kLdsX = NST * kX, kLdsOut = 2 * kX, kLdsBytes = kLdsX + kLdsOut + 2 * kDl;
    static constexpr int kWeights = EP * BC * 2, kAtWeights = kLdsBytes - kWeights;      // before the first step, behind its stage
    // as in GateShape
    static constexpr int kSurely = (NST - 2) * kLoadsX + kLoadsX + kOut;
    static constexpr int kLate = (NST - 2) * kLoadsX + 2 * kItemsEach, kYounger = kLate < kSurely ? kLate : kSurely;
    static constexpr int wait_for(int vmcnt) { return 0x0070 | (vmcnt & 15) | ((vmcnt >> 4) << 14); }      // and lgkmcnt(0)
    static_assert(NST >= 3 && kLdsBytes <= 160 * 1024 && kAtWeights >= kX, "wide gate gradient: stages");
};

template <int EB>
__global__ __launch_bounds__(512, 2) void gate_backward_wide_kernel([[maybe_unused]] GateGradArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = GateWide<EB>;
    constexpr int NST = kStages;
    extern __shared__ __align__(16) unsigned char gate_lds[];
    unsigned char *const lds_x = gate_lds, *const lds_out = lds_x + G::kLdsX, *const lds_dl = lds_out + G::kLdsOut;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int group = wave / G::kColumnGroups, column = wave % G::kColumnGroups, half = wave / 4, quarter = wave % 4;
    const GatePart part = gate_part(a, blockIdx.x, G::BC);
    const int H = a.H, E = a.E;
    const uint32_t pitch = (uint32_t)H * 2;
    const bool whole4 = (E & 3) == 0;
    // what a descriptor may reach of `rows` rows, from the first one's column part.col on: nothing of no rows, and nothing past the last column
    auto bytes_of = [&](int rows) { return rows > 0 ? (uint32_t)rows * pitch - (uint32_t)part.col * 2u : 0u; };

    f32x4 sum[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[j][i] = (f32x4){0.f, 0.f, 0.f, 0.f};

    uint32_t at_x[G::kLoadsX], at_o[G::kOut];
#pragma unroll
    for (int q = 0; q < G::kLoadsX; ++q) {                         // the place in LDS is fixed by the instruction, so the swizzle is applied here
        const int row = ((wave * G::kLoadsX + q) * 64 + lane) / G::kPerRowX, at = lane % G::kPerRowX, p = ((at >> 1) ^ row_swizzle<G::BC>(row)) * 2 + (at & 1);
        at_x[q] = part.col + p * 8 < H ? (uint32_t)row * pitch + (uint32_t)p * 16u : kOutOfRange;
    }
#pragma unroll
    for (int q = 0; q < G::kOut; ++q) {
        const int h = quarter * G::DC + 32 * q + 8 * g;
        at_o[q] = part.col + h < H ? (uint32_t)(16 * half + m) * pitch + (uint32_t)h * 2u : kOutOfRange;
    }
    const int64_t first = (int64_t)part.share * kSplitTokens, stride = (int64_t)a.shares * kSplitTokens;
    auto rows_at = [&](int64_t t0) { return __builtin_amdgcn_readfirstlane((int)max((int64_t)0, min((int64_t)kSplitTokens, a.T - t0))); };
    auto issue = [&](int64_t t0, int stage) {
        const auto from = make_rsrc(static_cast<const __bf16 *>(a.x) + (t0 * H + part.col), a.dw ? bytes_of(rows_at(t0)) : 0u);
#pragma unroll
        for (int q = 0; q < G::kLoadsX; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)(lds_x + stage + (wave * G::kLoadsX + q) * 1024), 16, at_x[q], 0, 0, kNt);
    };
    u32x4 add[G::kOut];
    f32x4 dl[G::kItemsEach][2];
    auto fetch_dl = [&](int64_t t0) {
        const auto from = make_rsrc(a.dl + t0 * E, (uint32_t)rows_at(t0) * (uint32_t)E * 4u);
#pragma unroll
        for (int n = 0; n < G::kItemsEach; ++n) {
            const int item = tid + G::kThreads * n, row = item / (G::EP / 8), e0 = item % (G::EP / 8) * 8;
            const uint32_t at = ((uint32_t)row * (uint32_t)E + (uint32_t)e0) * 4u;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                if (whole4) {
                    dl[n][v] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, e0 + 4 * v < E ? at + 16u * v : kOutOfRange, 0, 0));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dl[n][v][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, e0 + 4 * v + i < E ? at + 16u * v + 4u * i : kOutOfRange, 0, 0));
                }
            }
        }
    };
    auto fetch_add = [&](int64_t t0) {
        const auto from = make_rsrc(static_cast<const __bf16 *>(a.dadd) + (t0 * H + part.col), a.dadd ? bytes_of(rows_at(t0)) : 0u);
#pragma unroll
        for (int q = 0; q < G::kOut; ++q) add[q] = __builtin_amdgcn_raw_buffer_load_b128(from, at_o[q], 0, kNt);
    };
    auto split = [&](unsigned char *to_dl) {
#pragma unroll
        for (int n = 0; n < G::kItemsEach; ++n) {
            const int item = tid + G::kThreads * n, row = item / (G::EP / 8), p = item % (G::EP / 8);
            split_eight<G::kPiece>(dl[n], to_dl + row * G::kRow + ((p >> 1) ^ row_swizzle<G::EP>(row)) * 32 + (p & 1) * 16);
        }
    };
    auto leave = [&](int64_t t0, const unsigned char *from, uint32_t bytes) {
        const auto to = make_rsrc(static_cast<__bf16 *>(a.dx) + (t0 * H + part.col), a.dx ? bytes : 0u);
#pragma unroll
        for (int q = 0; q < G::kLoadsX; ++q)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, read_along((lds_bf16x8 *)(from + (wave * G::kLoadsX + q) * 1024 + lane * 16))), to,
                                                   at_x[q], 0, kNt);
    };

    const int ka = 8 * g + (m >> 2), across_x = ka * G::kRowX + (m & 3) * 8, across_dl = ka * G::kRow + (m & 3) * 8, along_dl = (16 * half + m) * G::kRow + (g & 1) * 16;
    const int sx = row_swizzle<G::BC>(ka) * 32, sd = row_swizzle<G::EP>(ka) * 32, sl = row_swizzle<G::EP>(m) * 32, so = row_swizzle<G::BC>(m) * 32;

    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    issue(first, 0);
    fetch_weights<G::EP, G::BC, G::kThreads>(a, part.col, gate_lds + G::kAtWeights, wave, lane);
    fetch_dl(first);
    fetch_add(first);
    __builtin_amdgcn_s_waitcnt(0x0070);
    barrier();
    bf16x8 w[G::KS][G::CD];
#pragma unroll
    for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
        for (int i = 0; i < G::CD; ++i) w[ks][i] = weight_fragment<G::BC>(gate_lds + G::kAtWeights, quarter * G::DC, ks, i, m, g);
    __builtin_amdgcn_s_waitcnt(0xc07f);                            // lgkmcnt(0): read by this wave, and behind the barrier by all
    barrier();
#pragma unroll
    for (int q = 1; q < NST - 1; ++q) issue(first + q * stride, q * G::kX);
    int buf = 0, stage = 0, out_at = 0;
    split(lds_dl);
    fetch_dl(first + stride);
    int64_t t0 = first;
    for (; t0 < a.T; t0 += stride) {
        f32x4 out[G::CD];
#pragma unroll
        for (int i = 0; i < G::CD; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint32_t word = add[i / 2][i % 2 * 2 + v / 2];
                out[i][v] = __uint_as_float(v % 2 ? word & 0xffff0000u : word << 16);
            }
        __builtin_amdgcn_s_waitcnt(G::wait_for(G::kYounger));      // this step's x has landed, this wave's parts of dl and of the last rows of dx are written
        barrier();                                                 // of two buffers of dl and dx the other one has been read by all before this
        leave(t0 - stride, lds_out + (G::kX - out_at), t0 > first ? bytes_of(rows_at(t0 - stride)) : 0u);
        fetch_add(t0 + stride);
        issue(t0 + (NST - 1) * stride, stage == 0 ? (NST - 1) * G::kX : stage - G::kX);       // where the step before was

        auto next_dl = [&](unsigned char *to) {                    // for the next step, among this one's products
            split(to);
            fetch_dl(t0 + 2 * stride);
        };
        const unsigned char *const dls = lds_dl + buf, *const xs = lds_x + stage;
        bf16x8 fx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) fx[i] = read_across((lds_s16x4 *)(xs + across_x + (((column * 4 + i) * 32) ^ sx)), 4 * G::kRowX);
#pragma unroll
        for (int ks = 0; ks < G::KS; ++ks)
#pragma unroll
            for (int piece = 0; piece < 3; ++piece) {
                const bf16x8 b = read_along((lds_bf16x8 *)(dls + piece * G::kPiece + along_dl + (((2 * ks + (g >> 1)) * 32) ^ sl)));
#pragma unroll
                for (int i = 0; i < G::CD; ++i) out[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[ks][i], b, out[i], 0, 0, 0);
            }
#pragma unroll
        for (int q = 0; q < G::kOut; ++q) {
            bf16x8 o;
#pragma unroll
            for (int v = 0; v < 8; ++v) o[v] = (__bf16)out[2 * q + v / 4][v % 4];
            const int c = quarter * (G::DC / 8) + 4 * q + g;       // its piece of the row
            put((lds_u32x4 *)(lds_out + out_at + (16 * half + m) * G::kRowX + ((c >> 1) * 32 ^ so) + (c & 1) * 16), __builtin_bit_cast(u32x4, o));
        }
        if constexpr (G::kSplitEarly) next_dl(lds_dl + (buf ^ G::kDl));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int piece = 0; piece < 3; ++piece) {
                const bf16x8 b = read_across((lds_s16x4 *)(dls + piece * G::kPiece + across_dl + (((group * 4 + j) * 32) ^ sd)), 4 * G::kRow);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i], b, sum[j][i], 0, 0, 0);
            }
        buf ^= G::kDl;
        if constexpr (!G::kSplitEarly) next_dl(lds_dl + buf);
        stage = stage == (NST - 1) * G::kX ? 0 : stage + G::kX;
        out_at = G::kX - out_at;
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                            // the loads past the end have come back: the LDS is another workgroup's after this
    barrier();
    leave(t0 - stride, lds_out + (G::kX - out_at), bytes_of(rows_at(t0 - stride)));
    if (a.dw)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 16 * (group * 4 + j) + m, h = part.col + column * 64 + 16 * i + 4 * g;
                if (e < E && h < H) *reinterpret_cast<f32x4 *>(a.dw + ((int64_t)part.share * E + e) * H + h) = sum[j][i];
            }
#endif
}

// Adds the shares' sums: a workgroup takes 32 vectors of them, its eight groups of 32 lanes every eighth share each, four loads at a time.
__global__ __launch_bounds__(256) void gate_dweight_kernel(const f32x4 *partial, f32x4 *dw, int shares, int64_t n)
{
    __shared__ f32x4 part[8][32];
    const int c = threadIdx.x % 32, r = threadIdx.x / 32;
    const int64_t i = (int64_t)blockIdx.x * 32 + c;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (i < n)
        for (int q = r; q < shares; q += 4 * 8) {
            f32x4 p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) p[u] = q + u * 8 < shares ? partial[(int64_t)(q + u * 8) * n + i] : (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 4; ++u) v += p[u];
        }
    part[r][c] = v;
    __syncthreads();
    if (r == 0 && i < n) {
#pragma unroll
        for (int u = 1; u < 8; ++u) v += part[u][c];
        dw[i] = v;
    }
}

// --------------------------------------------------------------------------------------------- host

template <int EB>
int launch_wide(const GateGradArgs &a, hipStream_t st)
{
    using G = GateWide<EB>;
    const auto kernel = gate_backward_wide_kernel<EB>;
    static LdsOptIn opted;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(kernel), G::kLdsBytes, opted)) return rc;
    hipLaunchKernelGGL(kernel, dim3(a.blocks * a.shares), dim3(G::kThreads), G::kLdsBytes, st, a);
    return MONTA_OK;
}

template <int EB, int NW>
int launch_split(const GateGradArgs &a, hipStream_t st)
{
    using G = GateShape<EB, NW>;
    const auto kernel = gate_backward_bf16_kernel<EB, NW>;
    static LdsOptIn opted;
    if (int rc = opt_in_lds(reinterpret_cast<const void *>(kernel), G::kLdsBytes, opted)) return rc;
    hipLaunchKernelGGL(kernel, dim3(a.blocks * a.shares), dim3(G::kThreads), G::kLdsBytes, st, a);
    return MONTA_OK;
}

// f(blocks of 16 experts), a power of two
template <typename F>
int with_expert_blocks(int E, F f)
{
    using std::integral_constant;
    if (E <= 16) return f(integral_constant<int, 1>{});
    if (E <= 32) return f(integral_constant<int, 2>{});
    if (E <= 64) return f(integral_constant<int, 4>{});
    if (E <= 128) return f(integral_constant<int, 8>{});
    return f(integral_constant<int, 16>{});
}

// Eight waves share the split gradients of up to 64 experts, and twice as many columns are waited for together: from 2^27 elements on, where splitting takes time
// (33 to 64 experts; us, four waves twice a CU, four waves and eight: 65536 x 7168 406, 459 and 411, with dadd 577, 585 and 521; 32768 x 4096 with dadd 160, 170 and 158;
// but 8192 x 7168 85, 82 and 88; 512 x 2048 14, 14 and 18; 65536 x 7168 with 32 experts 366, 339 and 340).
bool eight_waves(const Call &c) { return (int64_t)c.s.T * c.H >= (1 << 27); }

struct GatePlan {
    int blocks, shares;
};

GatePlan plan_gate_grad(const Call &c)
{
    const int width = with_expert_blocks(c.s.E, [&](auto eb) {
        constexpr int EB = decltype(eb)::value;
        if (!c.bf16) return 64 * tiles_of<EB>();
        if constexpr (EB > 4) return (int)GateWide<EB>::BC;
        return EB == 4 && eight_waves(c) ? 512 : 256;
    });
    GatePlan p;
    p.blocks = (c.H + width - 1) / width;
    // one step a share where there are few: 1155 x 516 fp32 8.6 us, with four steps 10.7; but up to 64 tokens alone, without a second launch: 64 x 4096 bf16 6.1
    // us, in two shares 7.1
    // Workgroups: one a CU where memory is the bound, two where products are (fp32 from 33 experts on).  us, one and two a CU: 65536 x 7168 bf16, 32 experts 339 and
    // 366, 8 experts 330 and 352, 131072 x 4096 332 and 346, 16384 x 4096 over 256 201 and 214; 8192 x 4096 fp32, 8, 32, 64 and 128 experts 75.5, 79.8, 106, 195 and 76.9, 83.4, 107, 172.
    const int wgs = c.bf16 || c.s.E <= 32 ? 256 : 512;
    const int64_t T = c.s.T, step = c.bf16 ? kSplitTokens : kStepTokens;
    p.shares = (int)std::min<int64_t>(std::max(1, wgs / p.blocks), T <= 64 ? 1 : (T + step - 1) / step);
    return p;
}

constexpr int kGateMaxHidden = 1 << 20;

}  // namespace
}  // namespace monta

using namespace monta;

extern "C" {

int monta_gate_backward_scratch_bytes(const monta_cfg *cfg, size_t *bytes)
{
    if (!bytes) return MONTA_ERR_NULL;
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (c.H > kGateMaxHidden) return MONTA_ERR_UNSUPPORTED;
    const GatePlan p = plan_gate_grad(c);
    *bytes = p.shares > 1 ? (size_t)p.shares * c.s.E * c.H * 4 : 16;
    return MONTA_OK;
}

int monta_gate_backward(const monta_cfg *cfg, const float *dlogits, const void *x, const void *w_gate, const void *dadd, void *dx, float *dw_gate,
                        void *scratch, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!dlogits || (!dx && !dw_gate) || (dx && !w_gate) || (dw_gate && (!x || !scratch))) return MONTA_ERR_NULL;
    if (misaligned(dlogits, 4) || misaligned(x, 16) || misaligned(w_gate, 16) || misaligned(dadd, 16) || misaligned(dx, 16) || misaligned(dw_gate, 16) ||
        misaligned(scratch, 16))
        return MONTA_ERR_ALIGN;
    if (dadd && !dx) return MONTA_ERR_INVALID;
    if (c.H > kGateMaxHidden) return MONTA_ERR_UNSUPPORTED;
    const GatePlan p = plan_gate_grad(c);
    const int64_t T = c.s.T, E = c.s.E, n = T * c.row_bytes, nw = E * c.H * 4, np = p.shares > 1 ? p.shares * nw : 16;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{dlogits, T * E * 4}, {x, n}, {w_gate, E * c.row_bytes}, {dadd, n}}, written[] = {{dx, n}, {dw_gate, nw}, {dw_gate ? scratch : nullptr, np}};
    for (const auto &w : written) {
        if (!w.p) continue;
        for (const auto &r : read) {
            if (!r.p) continue;
            // a step's part of dadd is in registers before anything of the step's dx is stored, by the same lane (fp32), the same wave or behind a
            // barrier (bf16, more than 64 experts): dx may be dadd as a whole, unless that is another argument, too
            if (w.p == dx && &r == &read[3] ? !same_or_apart(dx, dadd, n) : overlap(w.p, w.n, r.p, r.n)) return MONTA_ERR_INVALID;
        }
        for (const auto &o : written)
            if (&o != &w && o.p && overlap(w.p, w.n, o.p, o.n)) return MONTA_ERR_INVALID;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const GateGradArgs a = {dlogits, x, w_gate, dadd, dx, dw_gate && p.shares > 1 ? static_cast<float *>(scratch) : dw_gate, T, c.s.E, c.H, p.blocks, p.shares};
    {
        LaunchTimer timer(MONTA_K_GATE_BACKWARD, st);
        const int rc = with_expert_blocks(c.s.E, [&](auto eb) {
            constexpr int EB = decltype(eb)::value;
            if (c.bf16) {
                if constexpr (EB == 4)
                    if (eight_waves(c)) return launch_split<EB, 8>(a, st);
                if constexpr (EB > 4) return launch_wide<EB>(a, st);
                else return launch_split<EB, 4>(a, st);
            }
            hipLaunchKernelGGL((gate_backward_f32_kernel<EB>), dim3(p.blocks * p.shares), dim3(256), 0, st, a);
            return (int)MONTA_OK;
        });
        if (rc) return rc;
        MONTA_HIP_TRY(hipGetLastError());
    }
    if (dw_gate && p.shares > 1) {
        LaunchTimer timer(MONTA_K_GATE_DWEIGHT, st);
        const int64_t n4 = E * c.H / 4;
        hipLaunchKernelGGL(gate_dweight_kernel, dim3((unsigned)((n4 + 31) / 32)), dim3(256), 0, st, static_cast<const f32x4 *>(scratch),
                           reinterpret_cast<f32x4 *>(dw_gate), p.shares, n4);
        MONTA_HIP_TRY(hipGetLastError());
    }
    return MONTA_OK;
}

}  // extern "C"
