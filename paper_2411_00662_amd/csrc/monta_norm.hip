// Root-mean-square norm ahead of the gate and the experts, with its gradient, and the gradient of the combine: rows that pass
// through registers once.  All three are bound by memory.
#include "monta_rows.hpp"

namespace monta {
namespace {

// --------------------------------------------------------------------------------------------- norm
//
//   s = x + residual, rounded to the activation type and stored; r = 1 / sqrt(mean(s^2) + eps); v = s r w
//   out = v rounded once; codes = e4m3(v * (448 / amax)), scale = amax / 448 with amax the largest magnitude of v in the block,
//   at least 2^-40.
//
// The norm is that of the stored sum, which is what the gradient reads again.  v itself goes to 8 bits, not its rounding to 16:
// one rounding each.  e4m3 ends at 448: the largest value of a block times (448 / amax) is at most 448 (1 + 2^-23), which rounds to 448.
// A block of zeros, or of values below 2^-40, keeps a finite factor.
// 8192 x 4096 bf16 with a residual, both outputs: 303 MB in 48.8 us, 6.2 TB/s; a copy of that size reaches 6.2 to 6.5.
template <bool BF16, int L, int NV, bool STREAM>
__global__ __launch_bounds__(threads_of<L>()) void rmsnorm_kernel(const u32x4 *x, const u32x4 *residual, const u32x4 *w, u32x4 *sum,
                                                                  u32x4 *out, unsigned char *rows8, int T, int vpr, int row8_bytes, float eps)
{
    constexpr int EV = Elem<BF16>::kPerVec, kRows = threads_of<L>() / L;
    __shared__ float part[2][L > kWave ? L / kWave : 1];
    const int l = threadIdx.x % L;
    const uint32_t group = threadIdx.x / L;
    const int H = vpr * EV;
    u32x4 wv[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) wv[q] = l + q * L < vpr ? w[l + q * L] : (u32x4){0u, 0u, 0u, 0u};

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
            s[q] = i < vpr ? load<STREAM>(x + row * vpr + i) : (u32x4){0u, 0u, 0u, 0u};
            if (residual) add[q] = i < vpr ? load<STREAM>(residual + row * vpr + i) : (u32x4){0u, 0u, 0u, 0u};
        }
        float ss[1] = {0.f};
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
            for (int e = 0; e < EV; ++e) ss[0] = __builtin_fmaf(a[e], a[e], ss[0]);
        }
        row_sums<L>(ss, part[parity]);
        const float r = 1.f / __builtin_sqrtf(ss[0] / (float)H + eps);
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int i = l + q * L;
            float v[EV], g[EV];
            unpack<BF16>(s[q], v);
            unpack<BF16>(wv[q], g);
#pragma unroll
            for (int e = 0; e < EV; ++e) v[e] = v[e] * r * g[e];
            const bool mine = live && i < vpr;
            if (mine && residual) store<STREAM>(sum + row * vpr + i, s[q]);
            if (mine && out) store<STREAM>(out + row * vpr + i, pack<BF16>(v));
            if (rows8) {
                store_codes<BF16, L>(v, i, mine, rows8 + row * row8_bytes, H);
            }
        }
        if (rows8 && live) clear_tail<L>(rows8 + row * row8_bytes, row8_bytes, H, l);
    }
}

// With n = s r and g = dout w:  dx = r (g - n mean(g n)) + dsum,  dw = sum over the rows of dout n.
// A workgroup walks over rows and keeps the weight's and its gradient's share in registers; the next row is requested before the
// present one's sums are known.  The gradient's partial sums, one row of H per workgroup, are added by rmsnorm_dweight_kernel: a fixed
// order, no atomics.
// 8192 x 4096 bf16 with dsum: 268 MB in 48 us with the sum of the partials, 5.6 TB/s; one row of 256 lanes a workgroup instead of two
// takes 51, 1155 x 2048 bf16 11.1 for 9.9, 1155 x 516 fp32 9.2 for 8.2 (1155 x 2048 fp32 12.0 either way).
template <bool BF16, int L, int NV, bool STREAM>
__global__ __launch_bounds__(backward_threads_of<L>()) void rmsnorm_backward_kernel(const u32x4 *s_in, const u32x4 *w, const u32x4 *dout, const u32x4 *dsum,
                                                                           u32x4 *dx, float *partial, int T, int vpr, float eps)
{
    constexpr int EV = Elem<BF16>::kPerVec, kRows = backward_threads_of<L>() / L;
    constexpr u32x4 zero = {0u, 0u, 0u, 0u};
    __shared__ float part[2][kRows][2 * (L > kWave ? L / kWave : 1)];
    const int l = threadIdx.x % L;
    const uint32_t group = threadIdx.x / L;
    const int H = vpr * EV;
    u32x4 wv[NV];
    float dw[NV][EV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        wv[q] = l + q * L < vpr ? w[l + q * L] : zero;
#pragma unroll
        for (int e = 0; e < EV; ++e) dw[q][e] = 0.f;
    }
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
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            s0[q] = s[q];
            d0[q] = d[q];
            t0[q] = t[q];
            float a[EV], b[EV], g[EV];
            unpack<BF16>(s0[q], a);
            unpack<BF16>(d0[q], b);
            unpack<BF16>(wv[q], g);
#pragma unroll
            for (int e = 0; e < EV; ++e) {
                sums[0] = __builtin_fmaf(a[e], a[e], sums[0]);
                sums[1] = __builtin_fmaf(a[e], b[e] * g[e], sums[1]);
            }
        }
        if (kAhead && base + gridDim.x * kRows < (uint32_t)T) fetch(base + gridDim.x * kRows);
        row_sums<L>(sums, part[parity][group]);
        const float r = 1.f / __builtin_sqrtf(sums[0] / (float)H + eps);
        // dx = r (g - s c) + dsum.  r * r is infinite where the row's magnitude is below 5e-20; elsewhere the product from there keeps its rounding
        const float rr = r * r, mean = sums[1] / (float)H, c = rr <= 3.4028234663852886e38f ? rr * mean : r * (r * mean);
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
                o[e] = __builtin_fmaf(r, __builtin_fmaf(-a[e], c, b[e] * g[e]), o[e]);
                if (live) dw[q][e] = __builtin_fmaf(b[e], a[e] * r, dw[q][e]);
            }
            if (live && i < vpr) dx[row * vpr + i] = pack<BF16>(o);
        }
    }
    float *to = partial + (int64_t)blockIdx.x * H;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
            if (l + q * L < vpr)
#pragma unroll
                for (int e = 0; e < EV; ++e) to[(l + q * L) * EV + e] = dw[q][e];
    } else {
        __shared__ float cols[kRows][L * NV * EV];                  // the rows' groups, then one row of sums
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < EV; ++e) cols[group][(l + q * L) * EV + e] = dw[q][e];
        __syncthreads();
        for (int h = threadIdx.x; h < H; h += backward_threads_of<L>()) {
            float v = 0.f;
#pragma unroll
            for (int g = 0; g < kRows; ++g) v += cols[g][h];
            to[h] = v;
        }
    }
}

// Adds `n` rows of H partial sums: a workgroup takes 32 columns, its 32 half waves every 32nd row each, eight loads at a time (one at a
// time costs 1.5 us of the 9.7 that 1155 x 516 fp32 then takes, all of it latency).
__global__ __launch_bounds__(1024) void rmsnorm_dweight_kernel(const float *partial, float *dweight, int n, int H)
{
    __shared__ float part[32][33];
    const int c = threadIdx.x % 32, r = threadIdx.x / 32, h = blockIdx.x * 32 + c;
    float v = 0.f;
    if (h < H)
        for (int i = r; i < n; i += 8 * 32) {                      // eight loads at a time
            float p[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] = i + q * 32 < n ? partial[(int64_t)(i + q * 32) * H + h] : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) v += p[q];
        }
    part[r][c] = v;
    __syncthreads();
    if (r == 0 && h < H) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += part[i][c];
        dweight[h] = t;
    }
}

// --------------------------------------------------------------------------------------------- gradient of the combine
//
// out[t] = sum_j g[t][j] y[row(t, j)]:   dy[row(t, j)] = g[t][j] dout[t],   dg[t][j] = <dout[t], y[row(t, j)]>.
// A token's lanes keep its row of dout in registers and go over its kept choices, the next one's row of y on its way while the present
// one is multiplied.  A wave knows all choices from one load, lane j's is choice j (k <= 32); a dropped one has no row: its gate's gradient is 0.
// 8192 x 4096 bf16 over 8 experts, top-2: 336 MB in 52.9 us, 6.3 TB/s.
template <bool BF16, int L, int NV, bool STREAM>
__global__ __launch_bounds__(threads_of<L>()) void combine_backward_kernel(const u32x4 *dout, const u32x4 *y, const float *gates, u32x4 *dy,
                                                                           float *dgates, const int32_t *pos_final, int T, int k, int vpr, int max_rows)
{
    static_assert(L >= kWave, "a wave has one token");
    constexpr int EV = Elem<BF16>::kPerVec, kRows = threads_of<L>() / L, W = L / kWave;
    constexpr u32x4 zero = {0u, 0u, 0u, 0u};
    __shared__ float part[2][32][W];                                // alternated, so that one barrier keeps a token's sums from the next one's
    const int l = threadIdx.x % L, lane = threadIdx.x % kWave, wave = l / kWave;
    int parity = 0;
    // a whole wave goes round, and with L > 64 the whole workgroup
    for (uint32_t t = blockIdx.x * kRows + __builtin_amdgcn_readfirstlane(threadIdx.x / L); t < (uint32_t)T; t += gridDim.x * kRows, parity ^= 1) {
        const int64_t tk = (int64_t)t * k;
        const int pos = lane < k ? pos_final[tk + lane] : -1;
        const float gate = lane < k ? gates[tk + lane] : 0.f;
        u32x4 d[NV], cur[NV];
#pragma unroll
        for (int q = 0; q < NV; ++q) d[q] = l + q * L < vpr ? dout[(int64_t)t * vpr + l + q * L] : zero;
        const bool kept = pos >= 0 && pos < max_rows;
        unsigned long long left = __ballot(kept);
        auto row_of = [&](int j) { return (int64_t)__builtin_amdgcn_readlane(pos, j); };
        auto fetch = [&](int64_t row, u32x4(&to)[NV]) {
#pragma unroll
            for (int q = 0; q < NV; ++q) to[q] = l + q * L < vpr ? load<STREAM>(y + row * vpr + l + q * L) : zero;
        };
        float mine = 0.f;                                          // lane j: the wave's share of choice j's gradient
        if (left) fetch(row_of(__builtin_ctzll(left)), cur);
        while (left) {
            const int j = __builtin_ctzll(left);
            left &= left - 1;
            u32x4 next[NV];
            if (left) fetch(row_of(__builtin_ctzll(left)), next);
            const int64_t row = row_of(j);
            const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(gate), j));
            float dot = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int i = l + q * L;
                float a[EV], b[EV];
                unpack<BF16>(d[q], a);
                unpack<BF16>(cur[q], b);
#pragma unroll
                for (int e = 0; e < EV; ++e) {
                    dot = __builtin_fmaf(a[e], b[e], dot);
                    a[e] *= g;
                }
                if (i < vpr) store<STREAM>(dy + row * vpr + i, pack<BF16>(a));
            }
            dot = lanes_sum<kWave>(dot);
            if (lane == j) mine = dot;
#pragma unroll
            for (int q = 0; q < NV; ++q) cur[q] = next[q];
        }
        if constexpr (W == 1) {
            if (lane < k) dgates[tk + lane] = mine;
        } else {
            float(*const sums)[W] = part[parity];
            if (lane < k) sums[lane][wave] = mine;
            __syncthreads();
            if (l < k) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) v += sums[l][w];
                dgates[tk + l] = v;
            }
        }
    }
}

// --------------------------------------------------------------------------------------------- host

// HIP launches fewer than 2^32 threads; with up to 1024 a workgroup these are half of that.  Fewer tokens have a workgroup, or a wave, each.
constexpr int64_t kCombineGrid = 1 << 21;
}  // namespace

int64_t fp8_row_bytes(int64_t hidden) { return (hidden + 4 * ((hidden + kBlock - 1) / kBlock) + 127) / 128 * 128; }

}  // namespace monta

using namespace monta;

extern "C" {

int monta_fp8_rows(const monta_cfg *cfg, monta_cfg *rows, int64_t *row_bytes)
{
    if (!rows || !row_bytes) return MONTA_ERR_NULL;
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (c.H % 16 != 0) return MONTA_ERR_INVALID;
    const int64_t bytes = fp8_row_bytes(c.H);
    if (bytes / 2 > 0x7fffffff) return MONTA_ERR_UNSUPPORTED;
    monta_cfg r = *cfg;
    r.dtype = MONTA_BF16;
    r.hidden = (int32_t)(bytes / 2);
    Call moved;
    if (int rc = open_call(&r, nullptr, &moved)) return rc;
    *rows = r;
    *row_bytes = bytes;
    return MONTA_OK;
}

int monta_rmsnorm(const monta_cfg *cfg, const void *x, const void *residual, const void *weight, float eps, void *sum, void *out,
                  void *out_fp8, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!x || !weight || (!out && !out_fp8) || (residual && !sum)) return MONTA_ERR_NULL;
    if (misaligned(x, 16) || misaligned(residual, 16) || misaligned(weight, 16) || misaligned(sum, 16) || misaligned(out, 16) || misaligned(out_fp8, 16))
        return MONTA_ERR_ALIGN;
    if (!(eps >= 0.f) || eps > 3.4e38f) return MONTA_ERR_INVALID;
    if (sum && !residual) return MONTA_ERR_INVALID;
    if (out_fp8 && c.H % 16 != 0) return MONTA_ERR_INVALID;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    const int64_t n = c.s.T * c.row_bytes, row8 = fp8_row_bytes(c.H), n8 = c.s.T * row8;
    // a row has been read as a whole before anything of it is stored, so whole buffers may be the same, except that out and sum are two
    if (sum && (!same_or_apart(sum, x, n) || !same_or_apart(sum, residual, n) || overlap(sum, n, weight, c.row_bytes))) return MONTA_ERR_INVALID;
    if (out && (!same_or_apart(out, x, n) || (residual && !same_or_apart(out, residual, n)) || (sum && overlap(out, n, sum, n)) ||
                overlap(out, n, weight, c.row_bytes)))
        return MONTA_ERR_INVALID;
    if (out_fp8 && (overlap(out_fp8, n8, x, n) || (residual && overlap(out_fp8, n8, residual, n)) || overlap(out_fp8, n8, weight, c.row_bytes) ||
                    (sum && overlap(out_fp8, n8, sum, n)) || (out && overlap(out_fp8, n8, out, n))))
        return MONTA_ERR_INVALID;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LaunchTimer timer(MONTA_K_NORM, st);
    const int wgs = (int)std::min<int64_t>(((int64_t)c.s.T + rows_per_wg(c.s.vpr) - 1) / rows_per_wg(c.s.vpr), kNormGrid);
    const int64_t touched = n * (residual ? 3 : 1) + (out ? n : 0) + (out_fp8 ? n8 : 0);
    with_form(c.bf16, touched >= kStreamFrom, c.s.vpr, [&](auto bf, auto streamed, auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value;
        hipLaunchKernelGGL((rmsnorm_kernel<decltype(bf)::value, L, NV, decltype(streamed)::value>), dim3(wgs), dim3(threads_of<L>()), 0, st,
                           static_cast<const u32x4 *>(x), static_cast<const u32x4 *>(residual), static_cast<const u32x4 *>(weight),
                           static_cast<u32x4 *>(sum), static_cast<u32x4 *>(out), static_cast<unsigned char *>(out_fp8), c.s.T, c.s.vpr, (int)row8, eps);
        return MONTA_OK;
    });
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

int monta_rmsnorm_scratch_bytes(const monta_cfg *cfg, size_t *bytes)
{
    if (!bytes) return MONTA_ERR_NULL;
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    *bytes = (size_t)backward_grid(c) * c.H * 4;
    return MONTA_OK;
}

int monta_rmsnorm_backward(const monta_cfg *cfg, const void *sum, const void *weight, float eps, const void *dout, const void *dsum, void *dx,
                           float *dweight, void *scratch, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!sum || !weight || !dout || !dx || !dweight || !scratch) return MONTA_ERR_NULL;
    if (misaligned(sum, 16) || misaligned(weight, 16) || misaligned(dout, 16) || misaligned(dsum, 16) || misaligned(dx, 16) || misaligned(dweight, 4) ||
        misaligned(scratch, 16))
        return MONTA_ERR_ALIGN;
    if (!(eps >= 0.f) || eps > 3.4e38f) return MONTA_ERR_INVALID;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    const int grid = backward_grid(c);
    const int64_t n = c.s.T * c.row_bytes, np = (int64_t)grid * c.H * 4, nw = (int64_t)c.H * 4;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{sum, n}, {dout, n}, {dsum, n}, {weight, c.row_bytes}};
    for (const auto &r : read) {
        if (!r.p) continue;
        if (overlap(scratch, np, r.p, r.n) || overlap(dweight, nw, r.p, r.n)) return MONTA_ERR_INVALID;
        // a row is stored by the lanes that have read it, after all of them have: dx may be any of the three as a whole
        if (r.p == weight ? overlap(dx, n, r.p, r.n) : !same_or_apart(dx, r.p, n)) return MONTA_ERR_INVALID;
    }
    if (overlap(scratch, np, dx, n) || overlap(scratch, np, dweight, nw) || overlap(dx, n, dweight, nw)) return MONTA_ERR_INVALID;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *partial = static_cast<float *>(scratch);
    {
        LaunchTimer timer(MONTA_K_NORM_BACKWARD, st);
        with_form(c.bf16, n * (dsum ? 4 : 3) >= kStreamFrom, c.s.vpr, [&](auto bf, auto streamed, auto lanes, auto vecs) {
            constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value;
            hipLaunchKernelGGL((rmsnorm_backward_kernel<decltype(bf)::value, L, NV, decltype(streamed)::value>), dim3(grid), dim3(backward_threads_of<L>()), 0, st,
                               static_cast<const u32x4 *>(sum), static_cast<const u32x4 *>(weight), static_cast<const u32x4 *>(dout),
                               static_cast<const u32x4 *>(dsum), static_cast<u32x4 *>(dx), partial, c.s.T, c.s.vpr, eps);
            return MONTA_OK;
        });
        MONTA_HIP_TRY(hipGetLastError());
    }
    LaunchTimer timer(MONTA_K_NORM_DWEIGHT, st);
    hipLaunchKernelGGL(rmsnorm_dweight_kernel, dim3((c.H + 31) / 32), dim3(1024), 0, st, partial, dweight, grid, c.H);
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

int monta_combine_backward(const monta_cfg *cfg, const void *dout, const void *y, const float *gates, void *dy, float *dgates, const void *ws,
                           void *stream)
{
    Call c;
    if (int rc = open_call(cfg, ws, &c)) return rc;
    if (!dout || !y || !gates || !dy || !dgates || !ws) return MONTA_ERR_NULL;
    if (misaligned(dout, 16) || misaligned(y, 16) || misaligned(dy, 16) || misaligned(ws, 16) || misaligned(gates, 4) || misaligned(dgates, 4))
        return MONTA_ERR_ALIGN;
    if (c.s.vpr > kMaxVecs) return MONTA_ERR_UNSUPPORTED;
    const int64_t n = c.s.T * c.row_bytes, nr = c.max_rows * c.row_bytes, ng = (int64_t)c.s.T * c.s.k * 4;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{dout, n}, {y, nr}, {gates, ng}, {ws, c.ws_bytes}};
    for (const auto &r : read)
        if (overlap(dy, nr, r.p, r.n) || overlap(dgates, ng, r.p, r.n)) return MONTA_ERR_INVALID;
    if (overlap(dy, nr, dgates, ng)) return MONTA_ERR_INVALID;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LaunchTimer timer(MONTA_K_COMBINE_BACKWARD, st);
    with_form(c.bf16, n + 2 * c.kept_bound * c.row_bytes >= kStreamFrom, c.s.vpr, [&](auto bf, auto streamed, auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value < kWave ? kWave : decltype(lanes)::value, NV = decltype(vecs)::value, kRows = threads_of<L>() / L;
        const unsigned wgs = (unsigned)std::min<int64_t>(((int64_t)c.s.T + kRows - 1) / kRows, kCombineGrid);
        hipLaunchKernelGGL((combine_backward_kernel<decltype(bf)::value, L, NV, decltype(streamed)::value>), dim3(wgs), dim3(threads_of<L>()), 0, st,
                           static_cast<const u32x4 *>(dout), static_cast<const u32x4 *>(y), gates, static_cast<u32x4 *>(dy),
                           dgates, c.p.pos_final, c.s.T, c.s.k, c.s.vpr, c.s.max_rows);
        return MONTA_OK;
    });
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

}  // extern "C"
