// Gradients of the gate projection, by the tokens' rows and by the weights:
//   dx[t][h] = sum_e dl[t][e] w[e][h] + dadd[t][h],     dw[e][h] = sum_t dl[t][e] x[t][h].
// Few experts against many hidden elements: bound by reading x and dadd and writing dx once, as long as the products keep up.
#include "monta_internal.hpp"

#include <algorithm>

namespace monta {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct GateGradArgs {
    const float *dl;
    const void *x, *w, *dadd;
    void *dx;
    float *dw;              // sums of each run of tokens, [runs][E][H]; with one run the result
    int64_t T;
    int32_t E, H, per;      // tokens of a run, a multiple of the step
    int32_t blocks, each;   // column blocks; workgroups of an XCD
};

// What workgroup `block` does: the workgroups of an XCD go through the column blocks of a run one after the other, so that its dl is read from
// memory once and then found in the XCD's L2.
struct GatePart {
    int64_t t0, t1;
    int run, col;
};
__device__ __forceinline__ GatePart gate_part(const GateGradArgs &a, uint32_t block, int runs, int width)
{
    GatePart p;
    const uint32_t n = block % kXcds * (uint32_t)a.each + block / kXcds;
    p.run = (int)(n / (uint32_t)a.blocks);
    p.col = (int)(n % (uint32_t)a.blocks) * width;
    if (p.run >= runs) p.run = -1;
    p.t0 = (int64_t)p.run * a.per;
    p.t1 = min(p.t0 + a.per, a.T);
    return p;
}

// --------------------------------------------------------------------------------------------- exact products
//
// fp32 products on the matrix cores (16 x 16 x 4), for fp32 and for bf16 activations.  A wave has 16 CT columns of a step's 16 tokens and the
// weights of its columns in registers; the gradient of the logits, which all waves of the workgroup need in both orders, goes through LDS.
//   dx: rows h, columns t, summed over e.  Row r of tile i is column 4 CT (r / 4) + 4 i + r % 4, so that a lane gets 4 CT neighbours of one token.
//   dw: rows h, columns e, summed over t.  Row r of tile i is column CT r + i, so that a lane's elements of x are neighbours.

template <int EB>
constexpr int tiles_of() { return EB <= 4 ? 4 : 16 / EB; }

template <bool BF16, int N>
struct Piece {                  // N neighbouring elements of a row
    static_assert(N == 1 || N == 2 || N == 4, "piece: elements");
    typedef std::conditional_t<BF16, __bf16, float> E1;
    typedef E1 V __attribute__((ext_vector_type(N == 1 ? 2 : N)));      // one alone is kept in the first of two
    V v;
    __device__ __forceinline__ void clear()
    {
        v = (V)(E1)0.f;
    }
    __device__ __forceinline__ void get(const void *base, int64_t at)
    {
        const E1 *p = static_cast<const E1 *>(base) + at;
        if constexpr (N == 1) v[0] = *p;
        else v = *reinterpret_cast<const V *>(p);
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
};

constexpr int kStepTokens = 16;

template <bool BF16, int EB>
__global__ __launch_bounds__(256) void gate_backward_kernel(GateGradArgs a, int runs)
{
    constexpr int CT = tiles_of<EB>(), CW = 16 * CT, kPitch = 16 * EB + 4;
    __shared__ float dlt[2][kStepTokens][kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, g = lane >> 4;
    const GatePart part = gate_part(a, blockIdx.x, runs, 4 * CW);
    if (part.run < 0) return;
    const int64_t H = a.H;
    const int col = part.col + wave * CW;                          // first column of the wave
    const bool want_dx = a.dx != nullptr, want_dw = a.dw != nullptr;

    float w[CT][4 * EB];
    if (want_dx)
#pragma unroll
        for (int kk = 0; kk < 4 * EB; ++kk)
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const int e = 4 * kk + g, h = col + (m >> 2) * (4 * CT) + 4 * i + (m & 3);
                Piece<BF16, 1> p;
                p.clear();
                if (e < a.E && h < a.H) p.get(a.w, e * H + h);
                w[i][kk] = p[0];
            }
    f32x4 sum[EB][CT];
#pragma unroll
    for (int j = 0; j < EB; ++j)
#pragma unroll
        for (int i = 0; i < CT; ++i) sum[j][i] = (f32x4){0.f, 0.f, 0.f, 0.f};

    float dl[EB];
    Piece<BF16, CT> x[4];
    Piece<BF16, 4> add[CT];
    auto fetch = [&](int64_t t0) {
        const int64_t t = t0 + (tid >> 4);
#pragma unroll
        for (int q = 0; q < EB; ++q) {
            const int e = (tid & 15) + 16 * q;
            dl[q] = t < part.t1 && e < a.E ? a.dl[t * a.E + e] : 0.f;
        }
        if (want_dw)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int64_t at = t0 + 4 * s + g;
                x[s].clear();
                if (at < part.t1 && col + m * CT < a.H) x[s].get(a.x, at * H + col + m * CT);
            }
        if (want_dx)
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                const int h = col + 4 * CT * g + 4 * i;
                add[i].clear();
                if (a.dadd && t0 + m < part.t1 && h < a.H) add[i].get(a.dadd, (t0 + m) * H + h);
            }
    };
    fetch(part.t0);
    int buf = 0;
    for (int64_t t0 = part.t0; t0 < part.t1; t0 += kStepTokens, buf ^= 1) {
#pragma unroll
        for (int q = 0; q < EB; ++q) dlt[buf][tid >> 4][(tid & 15) + 16 * q] = dl[q];
        Piece<BF16, CT> x0[4];
        f32x4 out[CT];
#pragma unroll
        for (int s = 0; s < 4; ++s) x0[s] = x[s];
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) out[i][v] = add[i][v];
        __syncthreads();                                           // of two buffers the other one has been read by all before this
        if (t0 + kStepTokens < part.t1) fetch(t0 + kStepTokens);
        if (want_dx) {
#pragma unroll
            for (int kk = 0; kk < 4 * EB; ++kk) {
                const float b = dlt[buf][m][4 * kk + g];
#pragma unroll
                for (int i = 0; i < CT; ++i) out[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i][kk], b, out[i], 0, 0, 0);
            }
            if (t0 + m < part.t1)
#pragma unroll
                for (int i = 0; i < CT; ++i) {
                    const int h = col + 4 * CT * g + 4 * i;
                    if (h >= a.H) continue;
                    const int64_t at = (t0 + m) * H + h;
                    if constexpr (BF16) {
                        bf16x4 o;
#pragma unroll
                        for (int v = 0; v < 4; ++v) o[v] = (__bf16)out[i][v];
                        *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.dx) + at) = o;
                    } else {
                        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.dx) + at) = out[i];
                    }
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
                float *const to = a.dw + ((int64_t)part.run * a.E + e) * H + h;
#pragma unroll
                for (int i = 0; i < CT; ++i) to[i] = sum[j][i][v];
            }
}

// Adds the runs' sums, eight loads at a time.
__global__ __launch_bounds__(256) void gate_dweight_kernel(const f32x4 *partial, f32x4 *dw, int runs, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < runs; r += 8) {
            f32x4 p[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] = r + q < runs ? partial[(r + q) * n + i] : (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 8; ++q) v += p[q];
        }
        dw[i] = v;
    }
}

// --------------------------------------------------------------------------------------------- host

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

struct GatePlan {
    int width, blocks, per, runs;
};

GatePlan plan_gate_grad(const Call &c)
{
    GatePlan p;
    p.width = with_expert_blocks(c.s.E, [](auto eb) { return 4 * 16 * tiles_of<decltype(eb)::value>(); });
    p.blocks = (c.H + p.width - 1) / p.width;
    const int64_t T = c.s.T, most = std::max<int64_t>(1, 512 / p.blocks), wanted = std::min<int64_t>(most, (T + 63) / 64);
    const int64_t per = ((T + wanted - 1) / wanted + kStepTokens - 1) / kStepTokens * kStepTokens;
    p.per = (int)std::min<int64_t>(per, 0x7ffffff0);
    p.runs = (int)((T + p.per - 1) / p.per);
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
    *bytes = p.runs > 1 ? (size_t)p.runs * c.s.E * c.H * 4 : 16;
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
    const int64_t T = c.s.T, E = c.s.E, n = T * c.row_bytes, nw = E * c.H * 4, np = p.runs > 1 ? p.runs * nw : 16;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{dlogits, T * E * 4}, {x, n}, {w_gate, E * c.row_bytes}, {dadd, n}}, written[] = {{dx, n}, {dw_gate, nw}, {dw_gate ? scratch : nullptr, np}};
    for (const auto &w : written) {
        if (!w.p) continue;
        for (const auto &r : read) {
            if (!r.p) continue;
            // an element of dadd is read by the lane that stores dx there: dx may be dadd as a whole
            if (w.p == dx && r.p == dadd ? !same_or_apart(dx, dadd, n) : overlap(w.p, w.n, r.p, r.n)) return MONTA_ERR_INVALID;
        }
        for (const auto &o : written)
            if (&o != &w && o.p && overlap(w.p, w.n, o.p, o.n)) return MONTA_ERR_INVALID;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int each = (p.blocks * p.runs + kXcds - 1) / kXcds;
    const GateGradArgs a = {dlogits, x, w_gate, dadd, dx, dw_gate && p.runs > 1 ? static_cast<float *>(scratch) : dw_gate, T, c.s.E, c.H, p.per, p.blocks, each};
    {
        LaunchTimer timer(MONTA_K_GATE_BACKWARD, st);
        with_expert_blocks(c.s.E, [&](auto eb) {
            constexpr int EB = decltype(eb)::value;
            if (c.bf16) hipLaunchKernelGGL((gate_backward_kernel<true, EB>), dim3(each * kXcds), dim3(256), 0, st, a, p.runs);
            else hipLaunchKernelGGL((gate_backward_kernel<false, EB>), dim3(each * kXcds), dim3(256), 0, st, a, p.runs);
            return MONTA_OK;
        });
        MONTA_HIP_TRY(hipGetLastError());
    }
    if (dw_gate && p.runs > 1) {
        LaunchTimer timer(MONTA_K_GATE_DWEIGHT, st);
        const int64_t n4 = E * c.H / 4;
        hipLaunchKernelGGL(gate_dweight_kernel, dim3((unsigned)std::min<int64_t>((n4 + 255) / 256, 4096)), dim3(256), 0, st, static_cast<const f32x4 *>(scratch),
                           reinterpret_cast<f32x4 *>(dw_gate), p.runs, n4);
        MONTA_HIP_TRY(hipGetLastError());
    }
    return MONTA_OK;
}

}  // extern "C"
