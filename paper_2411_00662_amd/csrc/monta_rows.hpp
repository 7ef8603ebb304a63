// Rows that pass through registers once: what the kernels of the norms and of the combine's gradient share.
//
// A row of `vpr` 16-byte vectors belongs to L lanes, a vector each and NV of them L apart, so that a wave's loads cover whole
// lines: 16 or 64 lanes of a wave (several rows per workgroup, sums by lane moves), or a workgroup of 256, 512 or 1024.
#pragma once

#include "monta_internal.hpp"

#include <algorithm>

namespace monta {

int64_t fp8_row_bytes(int64_t hidden);      // defined in monta_norm.hip

namespace {

constexpr int kBlock = 128;                        // elements that share a scale
constexpr float kE4m3Max = 448.f;
constexpr float kAmaxFloor = 9.094947017729282e-13f;        // 2^-40
constexpr int kMaxVecs = 2048;                     // 16-byte vectors of the longest row: 1024 lanes of two

template <bool BF16>
struct Elem {
    static constexpr int kPerVec = BF16 ? 8 : 4;
    static constexpr int kBlockLanes = kBlock / kPerVec;             // neighbouring vectors that share a scale
};

template <bool BF16>
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[Elem<BF16>::kPerVec])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        } else {
            f[i] = __uint_as_float(v[i]);
        }
    }
}

template <bool STREAM>
__device__ __forceinline__ u32x4 load(const u32x4 *p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool STREAM>
__device__ __forceinline__ void store(u32x4 *p, u32x4 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// nearest-even; NaN stays NaN
template <bool BF16>
__device__ __forceinline__ u32x4 pack(const float (&f)[Elem<BF16>::kPerVec])
{
    if constexpr (BF16) {
        bf16x8 b;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (__bf16)f[i];
        return __builtin_bit_cast(u32x4, b);
    } else {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
        return v;
    }
}

// Sum over the L lanes (at most a wave) that share a row; every one of them gets it.
template <int L>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// The same over a whole row: across waves through `part`, the row's own, which the caller alternates from row to row, so that one
// barrier keeps a row's sums from the next row's.
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *part)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<(L < kWave ? L : kWave)>(v[i]);
    if constexpr (L > kWave) {
        constexpr int W = L / kWave;
        const int wave = threadIdx.x % L / kWave;
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) part[i * W + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) t += part[i * W + w];
            v[i] = t;
        }
    }
}

template <int L>
constexpr int threads_of() { return L <= kWave ? 256 : L; }
// of the norm's gradient: two rows of 256 lanes, for eight waves a CU with as few partial sums as four would leave
template <int L>
constexpr int backward_threads_of() { return L <= kWave ? 256 : L < 512 ? 512 : L; }

// A row's 8-bit form: the codes of vector i and, from the first lane of a block, the block's scale.  All lanes take part; `mine`: this one stores.
template <bool BF16, int L>
__device__ __forceinline__ void store_codes(const float (&v)[Elem<BF16>::kPerVec], int i, bool mine, unsigned char *to, int H)
{
    constexpr int EV = Elem<BF16>::kPerVec;
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < EV; ++e) amax = fmaxf(amax, __builtin_fabsf(v[e]));
#pragma unroll
    for (int d = 1; d < Elem<BF16>::kBlockLanes && d < L; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d, kWave));
    amax = fmaxf(amax, kAmaxFloor);
    const float up = kE4m3Max / amax;
    uint32_t c[EV / 4];
#pragma unroll
    for (int e = 0; e < EV / 4; ++e) {
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * e] * up, v[4 * e + 1] * up, 0, false);
        c[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * e + 2] * up, v[4 * e + 3] * up, word, true);
    }
    if (mine) {
        if constexpr (BF16) *reinterpret_cast<uint2 *>(to + i * 8) = make_uint2(c[0], c[1]);
        else *reinterpret_cast<uint32_t *>(to + i * 4) = c[0];
        if (i % Elem<BF16>::kBlockLanes == 0) reinterpret_cast<float *>(to + H)[i / Elem<BF16>::kBlockLanes] = amax / kE4m3Max;
    }
}

// The rest of the row's last line: fewer than 32 words.
template <int L>
__device__ __forceinline__ void clear_tail(unsigned char *row, int row8_bytes, int H, int l)
{
    uint32_t *to = reinterpret_cast<uint32_t *>(row);
    for (int i = H / 4 + (H + kBlock - 1) / kBlock + l; i < row8_bytes / 4; i += L) to[i] = 0u;
}

// --------------------------------------------------------------------------------------------- host

// f(lanes of a row, vectors of a lane): few lanes for short rows, so that no wave is mostly idle
template <typename F>
int with_long_row(int vpr, F f)             // more than 256 vectors
{
    using std::integral_constant;
    if (vpr <= 512) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (vpr <= 1024) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

template <typename F>
int with_row_shape(int vpr, F f)
{
    using std::integral_constant;
    if (vpr <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (vpr <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (vpr <= 256) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    return with_long_row(vpr, f);
}

// f(bf16, streamed, lanes of a row, vectors of a lane), all of them as types; `row` knows the last two
template <typename Row, typename F>
int with_types(bool bf16, bool streamed, Row row, F f)
{
    return row([&](auto lanes, auto vecs) {
        if (bf16) return streamed ? f(std::true_type{}, std::true_type{}, lanes, vecs) : f(std::true_type{}, std::false_type{}, lanes, vecs);
        return streamed ? f(std::false_type{}, std::true_type{}, lanes, vecs) : f(std::false_type{}, std::false_type{}, lanes, vecs);
    });
}

template <typename F>
int with_form(bool bf16, bool streamed, int vpr, F f)
{
    return with_types(bf16, streamed, [&](auto g) { return with_row_shape(vpr, g); }, f);
}

inline int rows_per_wg(int vpr) { return vpr <= 16 ? 16 : vpr <= 64 ? 4 : 1; }
inline int backward_rows_per_wg(int vpr) { return vpr <= 16 ? 16 : vpr <= 64 ? 4 : vpr <= 512 ? 2 : 1; }

constexpr int kNormGrid = 1 << 16;

// From three quarters of the memory-side cache (256 MiB) on what a call touches is streamed past it.  Rows of 4096 bf16, plain and streamed, us:
//                                      110 MB       140 MB       170 MB       200 MB       230 MB       260 MB       300 MB       400 MB
//   three sets in turn   norm          24.1  21.9   29.8  26.4   34.3  30.6   39.2  35.1   44.6  39.6   49.2  44.0   56.5  50.1   73.2  65.1
//                        its gradient  25.3  25.5   32.3  30.0   37.4  34.4   42.5  37.9   48.0  42.5   53.1  47.0   59.9  52.4   77.3  72.8
//                        the combine's 23.1  21.7   30.2  26.2   36.3  30.3   41.0  34.5   46.5  38.5   51.5  42.7   59.0  48.2   76.8  62.4
//   one set, all of it   norm          19.0  21.2   23.1  25.8   27.8  30.1   31.7  34.9   35.8  39.3   40.9  43.8   50.2  49.8   72.7  64.8
//   in the cache         its gradient  23.0  25.3   27.1  29.9   31.4  34.2   34.7  37.8   39.4  42.3   43.8  46.9   50.5  52.5   76.6  68.1
//                        the combine's 19.0  19.9   22.6  24.9   27.5  30.2   31.9  34.8   35.8  38.3   40.3  42.5   48.0  48.3   75.7  62.1
//   three sets, with the norm          28.7  30.9   34.7  36.3   41.7  42.4   47.3  47.0   55.2  51.4   61.9  57.8   68.8  67.7
//   gate beside it that  its gradient  31.8  34.2   38.2  40.9   44.5  45.0   49.2  48.5   54.8  54.2   60.4  62.3   69.8  73.5
//   reads out, dout, dy  the combine's 31.0  33.6   39.4  38.8   49.4  49.2   55.5  56.4   63.0  64.5   69.9  71.3   79.6  81.1
// The line is where the last of these break even: below it a call may find its inputs in the cache, and the next one its result.  (Of
// the gradient of the norm only the loads are streamed.)  It does not depend on whole lines: 330 MB in rows of 72, 520, 1032, 4104 and 7168 elements, on
// 128 bytes or 16 past them, are streamed in 0.85 to 1.03 of the plain time.
constexpr int64_t kStreamFrom = 192ll << 20;

// rows of partial sums: each is written and read again, and costs more than a row of the norm itself
inline int backward_grid(const Call &c)
{
    const int rows = backward_rows_per_wg(c.s.vpr);
    return (int)std::min<int64_t>(((int64_t)c.s.T + rows - 1) / rows, c.s.vpr <= 64 ? 512 : 256);
}

}  // namespace
}  // namespace monta
