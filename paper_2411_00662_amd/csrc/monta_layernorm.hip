// Layer norm ahead of the gate and the experts, with its gradient: rows that pass through registers once, bound by memory.
#include "monta_rows.hpp"
#include "monta_lanes.hpp"

namespace monta {
namespace {

// Sums around a mean that is not known yet.  A wave takes its own share's mean m_w, from a first sum, and its other sums around that;
// the waves' shares are then joined by
//   sum (s - m)^2 = sum_w [ M2_w + n_w d_w^2 ],   sum g (s - m) = sum_w [ G1_w + d_w G0_w ],   d_w = m_w - m,
// which has no difference of large numbers, and takes one barrier for both steps.  Means are quotients: from a product with 1 / n the compiler may make a
// fused difference for some elements of a row and not for others, and a row of equal numbers would not have a spread of zero.
//
// The first sum is off by some 2^-24 of the row's magnitude, which may be more than the row is spread: fp32 rows of equal numbers at 12345 came out as 0.5 instead of
// 0.  So where a mean is larger than the spread around it, the mean of the differences from it, `rest`, is a second part of it, and the other sums are taken
// again around both: off by 2^-24 of the spread, for two more passes over the registers of such rows (8192 x 4096 bf16 with a mean of 50 spreads 52.3 us instead of
// 51.3, the gradient 57.8 instead of 52).  Elsewhere the first sum's error is one of the spread's magnitude already: a second part has as much, and for bf16 rows,
// whose sums are mostly exact, more (codes that differ from those of 64 bits 371 for 240 of 268 million).
//
// Elements of a row that wave w of its L lanes holds, NV vectors of EV elements a lane.
template <int L, int NV, int EV>
__device__ __forceinline__ float wave_share(int vpr, int w)
{
    int n = 0;
#pragma unroll
    for (int q = 0; q < NV; ++q) n += min(max(vpr - q * L - w * kWave, 0), L < kWave ? L : kWave);
    return (float)(n * EV);
}

// --------------------------------------------------------------------------------------------- norm
//
//   s = x + residual, rounded to the activation type and stored; m = mean(s), r = 1 / sqrt(mean((s - m)^2) + eps); v = (s - m) r w + b
//   out = v rounded once; codes and scales of v as in monta_rmsnorm.
// 8192 x 4096 bf16 with a residual, both outputs: 303 MB in 51 us, 5.9 TB/s; the root-mean-square norm, with one sum and no barrier's wait less, takes 48.
template <bool BF16, int L, int NV, bool STREAM>
__global__ __launch_bounds__(threads_of<L>()) void layernorm_kernel(const u32x4 *x, const u32x4 *residual, const u32x4 *w, const u32x4 *bias, u32x4 *sum,
                                                                    u32x4 *out, unsigned char *rows8, int T, int vpr, int row8_bytes, float eps)
{
    constexpr int EV = Elem<BF16>::kPerVec, kRows = threads_of<L>() / L, LW = L < kWave ? L : kWave, W = L > kWave ? L / kWave : 1;
    constexpr u32x4 zero = {0u, 0u, 0u, 0u};
    __shared__ float part[2][3 * W];                                // alternated, so that one barrier keeps a row's sums from the next row's
    const int l = threadIdx.x % L, wave = l / kWave;
    const uint32_t group = threadIdx.x / L;
    const int H = vpr * EV;
    u32x4 wv[NV], bv[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        wv[q] = l + q * L < vpr ? w[l + q * L] : zero;
        bv[q] = bias && l + q * L < vpr ? bias[l + q * L] : zero;
    }
    const int peer = threadIdx.x % W;                              // the wave whose share this lane joins to the row
    const float share = fmaxf(wave_share<L, NV, EV>(vpr, wave), 1.f);
    const float of_peer = wave_share<L, NV, EV>(vpr, peer);

    int parity = 0;
    // every lane goes round as often as the others: the moves between lanes and the barrier take all of them.  Unsigned: base passes T by up to
    // a round, and T may be 2^31 - 1
    for (uint32_t base = blockIdx.x * kRows; base < (uint32_t)T; base += gridDim.x * kRows, parity ^= 1) {
        const bool live = base + group < (uint32_t)T;
        const int64_t row = live ? base + group : (uint32_t)T - 1;
        u32x4 s[NV], add[NV];
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int i = l + q * L;
            s[q] = i < vpr ? load<STREAM>(x + row * vpr + i) : zero;
            if (residual) add[q] = i < vpr ? load<STREAM>(residual + row * vpr + i) : zero;
        }
        float total = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            float a[EV];
            unpack<BF16>(s[q], a);
            if (residual) {
                float b[EV];
                unpack<BF16>(add[q], b);
#pragma unroll
                for (int e = 0; e < EV; ++e) a[e] += b[e];
                s[q] = pack<BF16>(a);
                unpack<BF16>(s[q], a);
            }
#pragma unroll
            for (int e = 0; e < EV; ++e) total += a[e];
        }
        total = group_sum<LW>(total);
        float mean = total / share, rest = 0.f, m2 = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            float a[EV];
            unpack<BF16>(s[q], a);
            if (l + q * L < vpr)
#pragma unroll
                for (int e = 0; e < EV; ++e) m2 = __builtin_fmaf(a[e] - mean, a[e] - mean, m2);
        }
        m2 = group_sum<LW>(m2);
        const bool far = share * mean * mean > m2;
        if (__any(far)) {                                          // a wave may have several rows: each has its own sums only
            float more = 0.f, again = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                float a[EV];
                unpack<BF16>(s[q], a);
                if (l + q * L < vpr)
#pragma unroll
                    for (int e = 0; e < EV; ++e) more += a[e] - mean;
            }
            more = group_sum<LW>(more) / share;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                float a[EV];
                unpack<BF16>(s[q], a);
                if (l + q * L < vpr)
#pragma unroll
                    for (int e = 0; e < EV; ++e) {
                        const float c = a[e] - mean - more;
                        again = __builtin_fmaf(c, c, again);
                    }
            }
            again = group_sum<LW>(again);
            if (far) {
                rest = more;
                m2 = again;
            }
        }
        if constexpr (W > 1) {
            float *const p = part[parity];
            if (threadIdx.x % kWave == 0) {
                p[wave] = total;
                p[W + wave] = rest;
                p[2 * W + wave] = m2;
            }
            __syncthreads();
            // lane v of each group of W joins wave v's share
            total = p[peer];
            mean = group_sum<W>(total) / (float)H;
            float c = total / fmaxf(of_peer, 1.f) - mean + p[W + peer];
            const float inside = p[2 * W + peer];
            m2 = group_sum<W>(__builtin_fmaf(of_peer * c, c, inside));
            rest = 0.f;
            if ((float)H * mean * mean > m2) {
                rest = group_sum<W>(of_peer * c) / (float)H;
                c -= rest;
                m2 = group_sum<W>(__builtin_fmaf(of_peer * c, c, inside));
            }
        }
        const float r = 1.f / __builtin_sqrtf(m2 / (float)H + eps);
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int i = l + q * L;
            float v[EV], g[EV], b[EV];
            unpack<BF16>(s[q], v);
            unpack<BF16>(wv[q], g);
            unpack<BF16>(bv[q], b);
#pragma unroll
            for (int e = 0; e < EV; ++e) v[e] = __builtin_fmaf((v[e] - mean - rest) * r, g[e], b[e]);
            const bool mine = live && i < vpr;
            if (mine && residual) store<STREAM>(sum + row * vpr + i, s[q]);
            if (mine && out) store<STREAM>(out + row * vpr + i, pack<BF16>(v));
            if (rows8) {
                if (i >= vpr)
#pragma unroll
                    for (int e = 0; e < EV; ++e) v[e] = 0.f;          // no part of the last block
                store_codes<BF16, L>(v, i, mine, rows8 + row * row8_bytes, H);
            }
        }
        if (rows8 && live) clear_tail<L>(rows8 + row * row8_bytes, row8_bytes, H, l);
    }
}

// With n = (s - m) r and g = dout w:  dx = r (g - mean(g) - n mean(g n)) + dsum,  dw = sum over the rows of dout n,  db = that of dout.
// A workgroup walks over rows and keeps the weight's and the bias's shares in registers; the next row is requested before the present one's
// sums are known.  Both gradients' partial sums, 2 H in a row per workgroup, are added by layernorm_dparams_kernel: a fixed order, no atomics.  Of few
// rows one workgroup writes the gradients itself.  8192 x 4096 bf16 with dsum: 268 MB in 52 us, 4 of them for the partial sums,
// 5.2 TB/s.
template <bool BF16, int L, int NV, bool STREAM>
__global__ __launch_bounds__(backward_threads_of<L>()) void layernorm_backward_kernel(const u32x4 *s_in, const u32x4 *w, const u32x4 *dout, const u32x4 *dsum,
                                                                                      u32x4 *dx, float *partial, float *dweight, float *dbias, int T, int vpr,
                                                                                      float eps)
{
    constexpr int EV = Elem<BF16>::kPerVec, kRows = backward_threads_of<L>() / L, LW = L < kWave ? L : kWave, W = L > kWave ? L / kWave : 1;
    constexpr u32x4 zero = {0u, 0u, 0u, 0u};
    __shared__ f32x4 part[2][kRows][W];
    __shared__ float rests[2][kRows][W];
    const int l = threadIdx.x % L, wave = l / kWave;
    const uint32_t group = threadIdx.x / L;
    const int H = vpr * EV;
    u32x4 wv[NV];
    float dw[NV][EV], db[NV][EV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        wv[q] = l + q * L < vpr ? w[l + q * L] : zero;
#pragma unroll
        for (int e = 0; e < EV; ++e) dw[q][e] = db[q][e] = 0.f;
    }
    const int peer = threadIdx.x % W;                              // the wave whose share this lane joins to the row
    const float share = fmaxf(wave_share<L, NV, EV>(vpr, wave), 1.f);
    const float of_peer = wave_share<L, NV, EV>(vpr, peer);
    constexpr bool kAhead = L < 1024;                               // 1024 lanes have no registers for a second row
    u32x4 s[NV], d[NV], t[NV];
    auto fetch = [&](uint32_t base) {
        const int64_t row = min(base + group, (uint32_t)T - 1);
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int i = l + q * L;
            s[q] = i < vpr ? load<STREAM>(s_in + row * vpr + i) : zero;
            d[q] = i < vpr ? load<STREAM>(dout + row * vpr + i) : zero;
            t[q] = dsum && i < vpr ? load<STREAM>(dsum + row * vpr + i) : zero;
        }
    };
    int parity = 0;
    if (kAhead) fetch(blockIdx.x * kRows);
    for (uint32_t base = blockIdx.x * kRows; base < (uint32_t)T; base += gridDim.x * kRows, parity ^= 1) {
        const bool live = base + group < (uint32_t)T;
        const int64_t row = live ? base + group : (uint32_t)T - 1;
        if (!kAhead) fetch(base);
        u32x4 s0[NV], d0[NV], t0[NV];
        float total = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            s0[q] = s[q];
            d0[q] = d[q];
            t0[q] = t[q];
            float a[EV];
            unpack<BF16>(s0[q], a);
#pragma unroll
            for (int e = 0; e < EV; ++e) total += a[e];
        }
        if (kAhead && base + gridDim.x * kRows < (uint32_t)T) fetch(base + gridDim.x * kRows);
        total = group_sum<LW>(total);
        float mean = total / share, rest = 0.f, m2 = 0.f, g0 = 0.f, g1 = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            float a[EV], b[EV], g[EV];
            unpack<BF16>(s0[q], a);
            unpack<BF16>(d0[q], b);
            unpack<BF16>(wv[q], g);
            if (l + q * L < vpr)
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    const float c = a[e] - mean, p = b[e] * g[e];
                    m2 = __builtin_fmaf(c, c, m2);
                    g0 += p;
                    g1 = __builtin_fmaf(c, p, g1);
                }
        }
        m2 = group_sum<LW>(m2);
        g0 = group_sum<LW>(g0);
        g1 = group_sum<LW>(g1);
        const bool far = share * mean * mean > m2;
        if (__any(far)) {
            float more = 0.f, again = 0.f, again1 = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q) asm volatile("" : "+v"(s0[q]), "+v"(d0[q]));      // unpacked anew: 1024 lanes have no registers for both forms
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                float a[EV];
                unpack<BF16>(s0[q], a);
                if (l + q * L < vpr)
#pragma unroll
                    for (int e = 0; e < EV; ++e) more += a[e] - mean;
            }
            more = group_sum<LW>(more) / share;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                float a[EV], b[EV], g[EV];
                unpack<BF16>(s0[q], a);
                unpack<BF16>(d0[q], b);
                unpack<BF16>(wv[q], g);
                if (l + q * L < vpr)
#pragma unroll
                    for (int e = 0; e < EV; ++e) {
                        const float c = a[e] - mean - more;
                        again = __builtin_fmaf(c, c, again);
                        again1 = __builtin_fmaf(c, b[e] * g[e], again1);
                    }
            }
            again = group_sum<LW>(again);
            again1 = group_sum<LW>(again1);
            if (far) {
                rest = more;
                m2 = again;
                g1 = again1;
            }
        }
        if constexpr (W > 1) {
            f32x4 *const p = part[parity][group];
            if (threadIdx.x % kWave == 0) {
                p[wave] = (f32x4){total, m2, g0, g1};
                rests[parity][group][wave] = rest;
            }
            __syncthreads();
            const f32x4 u = p[peer];
            mean = group_sum<W>(u[0]) / (float)H;
            float c = u[0] / fmaxf(of_peer, 1.f) - mean + rests[parity][group][peer];
            m2 = group_sum<W>(__builtin_fmaf(of_peer * c, c, u[1]));
            rest = 0.f;
            if ((float)H * mean * mean > m2) {
                rest = group_sum<W>(of_peer * c) / (float)H;
                c -= rest;
                m2 = group_sum<W>(__builtin_fmaf(of_peer * c, c, u[1]));
            }
            g0 = group_sum<W>(u[2]);
            g1 = group_sum<W>(__builtin_fmaf(c, u[2], u[3]));
        }
        const float r = 1.f / __builtin_sqrtf(m2 / (float)H + eps);
        // dx = r (g - c0 - (s - m) c1) + dsum; r * r is infinite where the spread is below 5e-20
        const float c0 = g0 / (float)H, c1 = r * (r * (g1 / (float)H));
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int i = l + q * L;
            float a[EV], b[EV], g[EV], o[EV];
            unpack<BF16>(s0[q], a);
            unpack<BF16>(d0[q], b);
            unpack<BF16>(wv[q], g);
            unpack<BF16>(t0[q], o);
#pragma unroll
            for (int e = 0; e < EV; ++e) {
                const float c = a[e] - mean - rest;
                o[e] = __builtin_fmaf(r, __builtin_fmaf(-c, c1, __builtin_fmaf(b[e], g[e], -c0)), o[e]);
                if (live) {
                    dw[q][e] = __builtin_fmaf(b[e], c * r, dw[q][e]);
                    db[q][e] += b[e];
                }
            }
            if (live && i < vpr) dx[row * vpr + i] = pack<BF16>(o);
        }
    }
    // a workgroup alone has the gradients themselves
    const bool alone = gridDim.x == 1;
    float *const to_w = alone ? dweight : partial + (int64_t)blockIdx.x * 2 * H, *const to_b = alone ? dbias : to_w + H;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
            if (l + q * L < vpr)
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    to_w[(l + q * L) * EV + e] = dw[q][e];
                    if (to_b) to_b[(l + q * L) * EV + e] = db[q][e];
                }
    } else {
        __shared__ float cols[kRows][L * NV * EV];                  // the rows' groups, then one row of sums
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < EV; ++e) cols[group][(l + q * L) * EV + e] = which ? db[q][e] : dw[q][e];
            __syncthreads();
            for (int h = threadIdx.x; h < H; h += backward_threads_of<L>()) {
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < kRows; ++g) v += cols[g][h];
                if (which == 0) to_w[h] = v;
                else if (to_b) to_b[h] = v;
            }
        }
    }
}

// Adds `n` rows of 2 H partial sums, of which the first H are the weight's gradient and the others the bias's: a workgroup takes 32 columns,
// its 32 half waves every 32nd row each, eight loads at a time.
__global__ __launch_bounds__(1024) void layernorm_dparams_kernel(const float *partial, float *dweight, float *dbias, int n, int H)
{
    __shared__ float part[32][33];
    const int c = threadIdx.x % 32, r = threadIdx.x / 32, h = blockIdx.x * 32 + c, cols = dbias ? 2 * H : H;
    float v = 0.f;
    if (h < cols)
        for (int i = r; i < n; i += 8 * 32) {
            float p[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] = i + q * 32 < n ? partial[(int64_t)(i + q * 32) * 2 * H + h] : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) v += p[q];
        }
    part[r][c] = v;
    __syncthreads();
    if (r == 0 && h < cols) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += part[i][c];
        (h < H ? dweight : dbias - H)[h] = t;
    }
}

// --------------------------------------------------------------------------------------------- host

// f(lanes of a row, vectors of a lane): lanes of one wave as far as their registers go, since a row of several waves meets at a barrier, and no more
// than the row has vectors for.  us, these forms and one vector for each of 64 or 256 lanes: norm of 16384 x 768 bf16 20.7 and 34.4, 16384 x 1024 26.3 and
// 34.6, 65536 x 256 25.9 and 32.9; its gradient 26.7 and 62.0, 29.3 and 64.0, 29.4 and 49.9.  Beyond 128 vectors the norm has no use for it (8192 x 2048 in
// one wave 27.5, in four 26.3), its gradient has (34.0 and 38.9; 16384 x 1536 43.7 and 67.9, with four vectors 46.2).
template <typename F>
int with_short_row(int vpr, F f)
{
    using std::integral_constant;
    if (vpr <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (vpr <= 32) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (vpr <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
}

template <typename F>
int with_norm_row(int vpr, F f)
{
    return vpr <= 128 ? with_short_row(vpr, f) : with_row_shape(vpr, f);
}

template <typename F>
int with_gradient_row(int vpr, F f)
{
    using std::integral_constant;
    if (vpr <= 128) return with_short_row(vpr, f);
    if (vpr <= 192) return f(integral_constant<int, 64>{}, integral_constant<int, 3>{});
    if (vpr <= 256) return f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    return with_long_row(vpr, f);
}

// Workgroups of the gradient, and so rows of partial sums, each of which is written and read again and costs more than a row of the norm itself.  us, 256 and
// 512 of them: 8192 x 2048 bf16 34.0 and 39.0, 16384 x 1024 29.3 and 30.2 (but 16384 x 768 26.7 and 24.0, 16384 x 1536 43.7 and 40.3), of one vector 65536 x 256 34.4
// and 29.4, 48222 x 120 15.5 and 13.7.  One workgroup has whole sums and needs no second launch, which gains as long as its rounds take less than that one: us, one
// workgroup and two launches, 4 rounds of lanes with one vector 5.4 to 5.8 and 7.8 to 8.2 (128 and 512 features, bf16), 6 rounds 6.0 to 7.3 and 6.1 to 8.0; of more
// vectors, 2 rounds 5.3 and 8.0 (1024 features), 8.2 and 9.1 (2048), 7.6 and 8.7 (4096), 12.6 and 13.1 (8192), 3 rounds 6.1 and 8.2, 10.6 and 9.0, 9.6 and 8.7,
// 14.7 and 13.1.  Of more vectors as few as have the same number of rounds: us, 256 and so many, 1100 x 2048 bf16 13.3 and 12.4, 600 x 4096 13.8 and 12.5, 300 x 8192
// 21.8 and 18.4 (1155 x 516 fp32 7.9 to 9.0 and 8.2 to 8.5, by where the library is loaded), but with one vector 9000 x 256 10.0 and 10.5.
struct GradientGrid {
    int workgroups, most;           // the most of any call of as many tokens or fewer: scratch for more tokens does for fewer
};

GradientGrid gradient_grid(const Call &c)
{
    GradientGrid g;
    with_gradient_row(c.s.vpr, [&](auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, rows = backward_threads_of<L>() / L;
        constexpr bool small = L <= kWave && decltype(vecs)::value == 1;
        const int64_t rounds = ((int64_t)c.s.T + rows - 1) / rows;
        g.most = (int)std::min<int64_t>(rounds, small ? 512 : 256);
        const int64_t each = small ? 1 : (rounds + g.most - 1) / g.most;
        g.workgroups = rounds <= (small ? 4 : 2) ? 1 : small ? g.most : (int)((rounds + each - 1) / each);
        return MONTA_OK;
    });
    return g;
}

}  // namespace
}  // namespace monta

using namespace monta;

extern "C" {

int monta_layernorm(const monta_cfg *cfg, const void *x, const void *residual, const void *weight, const void *bias, float eps, void *sum,
                    void *out, void *out_fp8, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!x || !weight || (!out && !out_fp8) || (residual && !sum)) return MONTA_ERR_NULL;
    if (misaligned(x, 16) || misaligned(residual, 16) || misaligned(weight, 16) || misaligned(bias, 16) || misaligned(sum, 16) || misaligned(out, 16) ||
        misaligned(out_fp8, 16))
        return MONTA_ERR_ALIGN;
    if (!(eps >= 0.f) || eps > 3.4e38f) return MONTA_ERR_INVALID;
    if (sum && !residual) return MONTA_ERR_INVALID;
    if (out_fp8 && c.H % 16 != 0) return MONTA_ERR_INVALID;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    const int64_t n = c.s.T * c.row_bytes, row8 = fp8_row_bytes(c.H), n8 = c.s.T * row8;
    // a row has been read as a whole before anything of it is stored, so whole buffers may be the same, except that out and sum are two
    for (const void *p : {x, residual})
        if (p && ((sum && !same_or_apart(sum, p, n)) || (out && !same_or_apart(out, p, n)) || (out_fp8 && overlap(out_fp8, n8, p, n)))) return MONTA_ERR_INVALID;
    for (const void *p : {weight, bias})
        if (p && ((sum && overlap(sum, n, p, c.row_bytes)) || (out && overlap(out, n, p, c.row_bytes)) || (out_fp8 && overlap(out_fp8, n8, p, c.row_bytes))))
            return MONTA_ERR_INVALID;
    if (sum && ((out && overlap(out, n, sum, n)) || (out_fp8 && overlap(out_fp8, n8, sum, n)))) return MONTA_ERR_INVALID;
    if (out && out_fp8 && overlap(out_fp8, n8, out, n)) return MONTA_ERR_INVALID;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LaunchTimer timer(MONTA_K_LAYERNORM, st);
    const int64_t touched = n * (residual ? 3 : 1) + (out ? n : 0) + (out_fp8 ? n8 : 0);
    const auto row = [&](auto f) { return with_norm_row(c.s.vpr, f); };
    with_types(c.bf16, touched >= kStreamFrom, row, [&](auto bf, auto streamed, auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value, kRows = threads_of<L>() / L;
        const int wgs = (int)std::min<int64_t>(((int64_t)c.s.T + kRows - 1) / kRows, kNormGrid);
        hipLaunchKernelGGL((layernorm_kernel<decltype(bf)::value, L, NV, decltype(streamed)::value>), dim3(wgs), dim3(threads_of<L>()), 0, st,
                           static_cast<const u32x4 *>(x), static_cast<const u32x4 *>(residual), static_cast<const u32x4 *>(weight),
                           static_cast<const u32x4 *>(bias), static_cast<u32x4 *>(sum), static_cast<u32x4 *>(out), static_cast<unsigned char *>(out_fp8),
                           c.s.T, c.s.vpr, (int)row8, eps);
        return MONTA_OK;
    });
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

int monta_layernorm_scratch_bytes(const monta_cfg *cfg, size_t *bytes)
{
    if (!bytes) return MONTA_ERR_NULL;
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    *bytes = (size_t)gradient_grid(c).most * c.H * 8;
    return MONTA_OK;
}

int monta_layernorm_backward(const monta_cfg *cfg, const void *sum, const void *weight, float eps, const void *dout, const void *dsum, void *dx,
                             float *dweight, float *dbias, void *scratch, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!sum || !weight || !dout || !dx || !dweight || !scratch) return MONTA_ERR_NULL;
    if (misaligned(sum, 16) || misaligned(weight, 16) || misaligned(dout, 16) || misaligned(dsum, 16) || misaligned(dx, 16) || misaligned(dweight, 4) ||
        misaligned(dbias, 4) || misaligned(scratch, 16))
        return MONTA_ERR_ALIGN;
    if (!(eps >= 0.f) || eps > 3.4e38f) return MONTA_ERR_INVALID;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    const int grid = gradient_grid(c).workgroups;
    const int64_t n = c.s.T * c.row_bytes, np = (int64_t)grid * c.H * 8, nw = (int64_t)c.H * 4;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{sum, n}, {dout, n}, {dsum, n}, {weight, c.row_bytes}}, written[] = {{dx, n}, {dweight, nw}, {dbias, nw}, {scratch, np}};
    for (const auto &w : written) {
        if (!w.p) continue;
        for (const auto &r : read) {
            if (!r.p) continue;
            // a row is stored by the lanes that have read it, after all of them have: dx may be any of the three as a whole
            if (w.p == dx && r.p != weight ? !same_or_apart(dx, r.p, n) : overlap(w.p, w.n, r.p, r.n)) return MONTA_ERR_INVALID;
        }
        for (const auto &o : written)
            if (&o != &w && o.p && overlap(w.p, w.n, o.p, o.n)) return MONTA_ERR_INVALID;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *partial = static_cast<float *>(scratch);
    {
        LaunchTimer timer(MONTA_K_LAYERNORM_BACKWARD, st);
        const auto row = [&](auto f) { return with_gradient_row(c.s.vpr, f); };
        with_types(c.bf16, n * (dsum ? 4 : 3) >= kStreamFrom, row, [&](auto bf, auto streamed, auto lanes, auto vecs) {
            constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value;
            hipLaunchKernelGGL((layernorm_backward_kernel<decltype(bf)::value, L, NV, decltype(streamed)::value>), dim3(grid), dim3(backward_threads_of<L>()), 0, st,
                               static_cast<const u32x4 *>(sum), static_cast<const u32x4 *>(weight), static_cast<const u32x4 *>(dout),
                               static_cast<const u32x4 *>(dsum), static_cast<u32x4 *>(dx), partial, dweight, dbias, c.s.T, c.s.vpr, eps);
            return MONTA_OK;
        });
        MONTA_HIP_TRY(hipGetLastError());
    }
    if (grid == 1) return MONTA_OK;
    LaunchTimer timer(MONTA_K_LAYERNORM_DPARAMS, st);
    hipLaunchKernelGGL(layernorm_dparams_kernel, dim3(((dbias ? 2 : 1) * c.H + 31) / 32), dim3(1024), 0, st, partial, dweight, dbias, grid, c.H);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

}  // extern "C"
