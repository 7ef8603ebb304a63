// The router's losses, and the gradient from the gates and those losses to the logits.
//
// A token's E logits belong to L lanes of a wave with V vectors of four each, E <= 4 L V: vector v of lane l is that of experts 4 (v L + l) and on.  Sums over
// a token's experts are moves between its lanes, and what they, a logarithm and a quotient cost falls with the number of lanes: the gradient of 32768 tokens
// over 256 experts takes 21 us with 64 lanes, 19 with 16 (both stored through the cache).
#include "monta_internal.hpp"
#include "monta_lanes.hpp"

#include <algorithm>

namespace monta {
namespace {

constexpr float kNone = -__builtin_inff();

// Four numbers at p, of which the first `exist` are there; the others are `rest`.
__device__ __forceinline__ f32x4 load_some(const float *p, int exist, float rest)
{
    if (exist >= 4) return *reinterpret_cast<const f32x4_any *>(p);
    f32x4 v = {rest, rest, rest, rest};
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < exist) v[i] = p[i];
    return v;
}

template <bool STREAM>
__device__ __forceinline__ void store_some(float *p, int exist, f32x4 v)
{
    if (exist >= 4) {
        if constexpr (STREAM) __builtin_nontemporal_store((f32x4_any)v, reinterpret_cast<f32x4_any *>(p));
        else *reinterpret_cast<f32x4_any *>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < exist) p[i] = v[i];
}

// e^x for x <= 0 (NaN counts as -infinity): x log2(e) in two parts, of which the first has all but 2^-24 of it, 2^(h + l) = 2^h (1 + l ln 2).  One
// multiplication alone loses |x| / 2 steps of the result.  Below -128 the result is less than the smallest fp32 number.
__device__ __forceinline__ float exp_neg(float x)
{
    constexpr double kLog2e = 1.4426950408889634074;
    constexpr float kHigh = (float)kLog2e, kLow = (float)(kLog2e - (double)kHigh);
    x = plain_max(x, -128.f);
    const float h = x * kHigh, l = __builtin_fmaf(x, kLow, __builtin_fmaf(x, kHigh, -h)), p = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(p, l * 0.69314718056f, p);
}

template <int V>
struct Softmax {
    f32x4 p[V];    // of the lane's experts; 0 past the last one
    float lse;     // log of the sum of all exponentials
};

// of the L lanes' logits; kNone past the last expert.  A reciprocal of one step, a logarithm of base 2 of one step: the sum lies in 1 .. 256.
template <int L, int V>
__device__ __forceinline__ Softmax<V> softmax(const f32x4 (&v)[V])
{
    float top = kNone;
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) top = plain_max(top, __builtin_canonicalizef(v[i / 4][i % 4]));      // a NaN from memory may be a signalling one
    top = group_max<L>(top);
    Softmax<V> s;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) {
        const float e = exp_neg(v[i / 4][i % 4] - top);
        s.p[i / 4][i % 4] = e;
        sum += e;
    }
    sum = group_sum<L>(sum);
    const float inv = __builtin_amdgcn_rcpf(sum);
    // without a number, or with +infinity, the sum is 0: 0 times infinity makes that NaN as the probabilities are, and changes no other
    s.lse = __builtin_fmaf(0.f, inv, __builtin_fmaf(__builtin_amdgcn_logf(sum), 0.69314718056f, top));
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) s.p[i / 4][i % 4] *= inv;
    return s;
}

// a token's logits, or others of its row
template <int L, int V>
__device__ __forceinline__ void load_row(f32x4 (&v)[V], const float *row, int l, int E, bool there)
{
#pragma unroll
    for (int q = 0; q < V; ++q) {
        const int e = 4 * (q * L + l);
        v[q] = (f32x4){kNone, kNone, kNone, kNone};
        if (there && e < E) v[q] = load_some(row + e, E - e, kNone);
    }
}

// --------------------------------------------------------------------------------------------- losses
//
// Over the n tokens that are no padding:  c[e] = pairs that chose e, f[e] = E c[e] / (k n), P[e] = mean of p[t][e];
//   balance = sum_e f[e] P[e],   z = mean of lse[t]^2.
// A workgroup sums a run of tokens; its E + 1 sums and E + 1 counts are a column each of `partial`, one word a workgroup, which
// route_loss_join_kernel adds, a wave a column.  One workgroup alone finishes by itself.
// A workgroup of the join has eight experts (one for all of them takes 12 us for 256 experts and 4.4 for 64, which is what a CU takes to fetch the columns).
// The balance loss is the sum of their shares, which the last one to arrive adds, in the experts' order: who that is says a counter, which the
// kernel before has cleared.
// 65536 tokens over 64 experts, top-8, a mask: 19 MB in 11.0 us, of which 7 the first launch; over 256 69 MB in 20.

constexpr int kLossThreads = 1024, kLossWaves = kLossThreads / kWave, kLossGrid = 256, kMaxExperts = 256;
constexpr int kJoinExperts = 8, kMostJoins = kMaxExperts / kJoinExperts;        // experts of a workgroup that joins
static_assert(kMostJoins <= kWave, "a lane has a workgroup's share");

// Words of `partial`: 2 (E + 1) columns of G, then the counter, then the joins' shares.
__host__ __device__ constexpr int64_t loss_counter(int E, int G) { return 2 * (int64_t)(E + 1) * G; }
inline int64_t loss_scratch(int E, int G) { return (loss_counter(E, G) + 1 + kMostJoins) * 4; }

struct LossOut {
    float *losses;
    int32_t *counts;
    float *means;
};

// Mean probability, count and share of the balance loss of expert e, from its sums over the n tokens.
__device__ __forceinline__ float finish_expert(const LossOut &o, int e, float sum, int count, int n, int E, int k)
{
    const float mean = n > 0 ? sum / (float)n : 0.f;
    o.means[e] = mean;
    o.counts[e] = count;
    return n > 0 ? (float)count * ((float)E / (float)k) / (float)n * mean : 0.f;
}

__device__ __forceinline__ void finish_losses(const LossOut &o, float balance, float z, int n, int E)
{
    o.losses[0] = balance;
    o.losses[1] = n > 0 ? z / (float)n : 0.f;
    o.counts[E] = n;
}

template <int L, int V>
__global__ __launch_bounds__(kLossThreads) void route_loss_kernel(const float *logits, const int32_t *idx, const uint8_t *mask, float *partial, LossOut o,
                                                                  int T, int E, int k, int per)
{
    constexpr int kTokens = kLossThreads / L, kAtOnce = V == 1 ? 2 : 1;         // tokens of a round; rounds whose logits are requested together
    __shared__ float sums[kLossWaves][kMaxExperts + 1], all[kMaxExperts + 1], part[kMaxExperts / kWave];
    __shared__ int32_t cnt[kMaxExperts + 1];
    const int tid = threadIdx.x, l = tid % L, wave = tid / kWave;
    for (int i = tid; i <= E; i += kLossThreads) cnt[i] = 0;
    __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * per, t1 = min(t0 + per, (int64_t)T);
    f32x4 v[kAtOnce][V];
    bool live[kAtOnce];
    auto fetch = [&](int64_t base) {
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int64_t t = base + q * kTokens + tid / L;
            live[q] = t < t1 && (!mask || mask[t]);
            load_row<L, V>(v[q], logits + t * E, l, E, t < t1);
        }
    };
    fetch(t0);                                                     // on their way while the choices are counted
    {
        const int64_t p0 = t0 * k, pairs = (t1 - t0) * k;
        for (int64_t p = tid; p < pairs; p += kLossThreads) {
            const int e = idx[p0 + p];
            const bool counts = !mask || mask[t0 + (uint32_t)p / (uint32_t)k];
            if ((uint32_t)e < (uint32_t)E && counts) atomicAdd(&cnt[e], 1);
        }
    }
    f32x4 acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float z = 0.f;
    int n = 0;
    for (int64_t base = t0; base < t1; base += kTokens * kAtOnce) {
        if (base > t0) fetch(base);
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            if (base + q * kTokens >= t1) break;                    // all lanes together
            const Softmax<V> s = softmax<L, V>(v[q]);
            if (live[q]) {
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += s.p[i];
                if (l == 0) {
                    z = __builtin_fmaf(s.lse, s.lse, z);
                    ++n;
                }
            }
        }
    }
#pragma unroll
    for (int d = L; d < kWave; d <<= 1) {
#pragma unroll
        for (int i = 0; i < 4 * V; ++i) acc[i / 4][i % 4] += __shfl_xor(acc[i / 4][i % 4], d, kWave);
        z += __shfl_xor(z, d, kWave);
        n += __shfl_xor(n, d, kWave);
    }
    if (tid % kWave < L)
#pragma unroll
        for (int i = 0; i < 4 * V; ++i) {
            const int e = 4 * (i / 4 * L + l) + i % 4;
            if (e < E) sums[wave][e] = acc[i / 4][i % 4];
        }
    if (tid % kWave == 0) {
        sums[wave][E] = z;
        atomicAdd(&cnt[E], n);
    }
    __syncthreads();
    const bool alone = gridDim.x == 1;
    for (int i = tid; i <= E; i += kLossThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kLossWaves; ++w) v += sums[w][i];
        if (alone) {
            all[i] = v;
        } else {
            partial[(int64_t)i * gridDim.x + blockIdx.x] = v;
            reinterpret_cast<int32_t *>(partial)[(int64_t)(E + 1 + i) * gridDim.x + blockIdx.x] = cnt[i];
        }
    }
    if (!alone) {
        if (blockIdx.x == 0 && tid == 0) reinterpret_cast<int32_t *>(partial)[loss_counter(E, gridDim.x)] = 0;
        return;
    }
    __syncthreads();
    const float f = group_sum<kWave>(tid < E ? finish_expert(o, tid, all[tid], cnt[tid], cnt[E], E, k) : 0.f);
    if (tid < kMaxExperts && tid % kWave == 0) part[tid / kWave] = f;
    __syncthreads();
    if (tid == 0) finish_losses(o, (part[0] + part[1]) + (part[2] + part[3]), all[E], cnt[E], E);
}

__global__ __launch_bounds__(256) void route_loss_join_kernel(float *partial, LossOut o, int G, int E, int k)
{
    constexpr int kWaves = 4, kEach = kJoinExperts / kWaves;        // experts of a wave
    static_assert(kLossGrid == 4 * kWave, "a lane has four words of a column");
    __shared__ float part[kWaves];
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, e0 = blockIdx.x * kJoinExperts + wave * kEach;
    auto column = [&](int c) { return load_some(partial + (int64_t)c * G + 4 * lane, G - 4 * lane, 0.f); };
    auto total = [](f32x4 v) { return group_sum<kWave>((v[0] + v[1]) + (v[2] + v[3])); };
    auto count = [](f32x4 v) {
        int n = (__float_as_int(v[0]) + __float_as_int(v[1])) + (__float_as_int(v[2]) + __float_as_int(v[3]));
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) n += __shfl_xor(n, d, kWave);
        return n;
    };
    f32x4 sums[kEach], counts[kEach];
    const f32x4 tokens = column(2 * E + 1), squares = column(E);
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        const int e = min(e0 + q, E - 1);
        sums[q] = column(e);
        counts[q] = column(E + 1 + e);
    }
    const int n = count(tokens);
    const float z = total(squares);
    float f = 0.f;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        const float sum = total(sums[q]);
        const int c = count(counts[q]);
        if (e0 + q < E && lane == 0) f += finish_expert(o, e0 + q, sum, c, n, E, k);
    }
    if (lane == 0) part[wave] = f;
    __syncthreads();
    float *const shares = partial + loss_counter(E, G) + 1;
    if (tid == 0) {
        __hip_atomic_store(shares + blockIdx.x, (part[0] + part[1]) + (part[2] + part[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(reinterpret_cast<int32_t *>(shares - 1), 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last || wave != 0) return;
    const float balance = group_sum<kWave>(lane < (int)gridDim.x ? __hip_atomic_load(shares + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f);
    if (lane == 0) finish_losses(o, balance, z, n, E);
}

// --------------------------------------------------------------------------------------------- gradient by the logits
//
// Gates g_j of the chosen i_j, their gradients d_j, D = sum_j g_j d_j; p the softmax over all experts:
//   renormalised over the choices:  dl[i_j] += g_j (d_j - D);     otherwise:  dl[i_j] += g_j d_j,  dl[e] -= p[e] D.
// The losses' part, with their gradients b and c, f and n as above:
//   dl[e] += p[e] ( b / n (f[e] - sum_i p[i] f[i]) + 2 c / n lse ).
// A workgroup takes 256 / L tokens.  A thread has a pair: it goes over its token's pairs in LDS for D, and puts what its expert gets (once, by the
// first of its pairs if an expert is named twice) into the token's row in LDS, which the token's lanes then add to what p asks for.  The next tokens' logits and
// pairs are on their way meanwhile.  32768 tokens over 256 experts, top-8: 70 MB in 17 us, 65536 over 64 40 MB in 11: 4.8 TB/s with the
// launch taken off, beside vector instructions in half of a SIMD's cycles.  A form without barriers,
// each wave with rows of its own in LDS, takes as long.

constexpr int kGradThreads = 256, kRouteGrid = 1024;
// From 2^21 logits on their gradients go past the cache.  us, stored plainly and streamed, alone and with monta_gate_backward of so many features behind: 65536 x 64
// 12.4 / 83.6 and 11.4 / 83.2 (1024 features), 16384 x 128 7.7 / 48.4 and 6.9 / 48.3 (1024), 8192 x 256 7.8 / 108 and 7.2 / 108 (4096), 32768 x 256 18.6 / 80.1 and 16.7 /
// 80.1 (512), 65536 x 256 35.5 / 397 and 28.8 / 401 (2048); 16384 x 64, fewer, 5.7 / 78.6 and 5.7 / 78.8 (4096).
inline bool stream_logits(int64_t T, int64_t E) { return T * E >= 1 << 21; }

struct RouteGradArgs {
    const float *logits, *gates, *dgates, *dlosses;
    const int32_t *idx, *counts;
    const uint8_t *mask;
    float *dlogits;
    int32_t T, E, k, renorm;
    FastDiv by_k;
};

template <int L, int V>
constexpr int grad_lds(int k)       // bytes: rows, D, and of each pair product, gate and expert
{
    return kGradThreads / L * (4 * L * V + 1 + 3 * k) * 4;
}

template <int L, int V, bool SOFTMAX, bool STREAM>
__global__ __launch_bounds__(kGradThreads) void route_backward_kernel(RouteGradArgs a)
{
    constexpr int kTokens = kGradThreads / L, kRow = 4 * L * V;
    extern __shared__ __align__(16) float route_lds[];
    const int tid = threadIdx.x, l = tid % L, mine = tid / L, k = a.k;
    float *const row = route_lds, *const dots = row + kTokens * kRow, *const prod = dots + kTokens, *const gate = prod + kTokens * k;
    int32_t *const expert = reinterpret_cast<int32_t *>(gate + kTokens * k);
    const int64_t chunks = ((int64_t)a.T + kTokens - 1) / kTokens;
    // what the next tokens need: their logits, and this thread's pairs
    constexpr int kEach = kTokens * (kRow < 32 ? kRow : 32) / kGradThreads;      // k <= E <= 4 L V, k <= 32
    f32x4 v[V], f[V];
    float pair_gate[kEach], pair_grad[kEach];
    int32_t pair_expert[kEach];
    uint8_t pair_mask[kEach];
    bool live;
    auto fetch = [&](int64_t chunk) {
        const int64_t t = chunk * kTokens + mine;
        if (a.dgates) {
            const int64_t p0 = chunk * kTokens * k;
            const int pairs = (int)min((int64_t)kTokens, a.T - chunk * kTokens) * k;
#pragma unroll
            for (int q = 0; q < kEach; ++q) {
                const int p = tid + q * kGradThreads;
                if (p < pairs) {
                    pair_expert[q] = a.idx[p0 + p];
                    pair_gate[q] = a.gates[p0 + p];
                    pair_grad[q] = a.dgates[p0 + p];
                    pair_mask[q] = a.mask ? a.mask[chunk * kTokens + p / a.by_k] : 1;
                }
            }
        }
        live = t < a.T && (!a.mask || a.mask[t]);
        if constexpr (SOFTMAX) load_row<L, V>(v, a.logits + t * a.E, l, a.E, t < a.T);
    };
    fetch(blockIdx.x);
    float b = 0.f, c = 0.f;
    if (SOFTMAX) {
        float scale = 0.f;
        if (a.dlosses) {
            const float n = (float)max(a.counts[a.E], 1);
            b = a.dlosses[0] / n;
            c = 2.f * (a.dlosses[1] / n);
            scale = (float)a.E / ((float)k * n);
        }
#pragma unroll
        for (int i = 0; i < 4 * V; ++i) {
            const int e = 4 * (i / 4 * L + l) + i % 4;
            f[i / 4][i % 4] = a.dlosses && e < a.E ? (float)a.counts[e] * scale : 0.f;
        }
    }
    for (int64_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        const int64_t t0 = chunk * kTokens, t = t0 + mine;
        const int tokens = (int)min((int64_t)kTokens, a.T - t0);
        const bool there = mine < tokens, mine_live = live;
#pragma unroll
        for (int q = 0; q < V; ++q) *reinterpret_cast<f32x4 *>(row + mine * kRow + 4 * (q * L + l)) = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (l == 0) dots[mine] = 0.f;
        if (a.dgates) {
            const int pairs = tokens * k;
#pragma unroll
            for (int q = 0; q < kEach; ++q) {
                const int p = tid + q * kGradThreads;
                if (p >= pairs) break;
                const bool counts = (uint32_t)pair_expert[q] < (uint32_t)a.E && pair_mask[q];
                expert[p] = counts ? pair_expert[q] : -1;
                gate[p] = counts ? pair_gate[q] : 0.f;
                prod[p] = counts ? pair_gate[q] * pair_grad[q] : 0.f;
            }
            __syncthreads();
            for (int p = tid; p < pairs; p += kGradThreads) {
                const int tok = p / a.by_k, first = tok * k, e = expert[p];
                float dot = 0.f, sp = 0.f, sg = 0.f;
                bool owner = e >= 0;
                for (int i = 0; i < k; ++i) {
                    const float q = prod[first + i];
                    dot += q;
                    if (expert[first + i] == e) {
                        sp += q;
                        sg += gate[first + i];
                        owner = owner && first + i >= p;
                    }
                }
                if (owner) row[tok * kRow + e] = a.renorm ? __builtin_fmaf(-sg, dot, sp) : sp;
                if (p == first) dots[tok] = dot;
            }
        }
        __syncthreads();
        f32x4 d[V], now[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
            d[q] = *reinterpret_cast<const f32x4 *>(row + mine * kRow + 4 * (q * L + l));
            if constexpr (SOFTMAX) now[q] = v[q];
        }
        if (chunk + gridDim.x < chunks) fetch(chunk + gridDim.x);
        if constexpr (SOFTMAX) {
            const Softmax<V> s = softmax<L, V>(now);
            const float dot = a.renorm ? 0.f : dots[mine];
            float pf = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * V; ++i) pf = __builtin_fmaf(s.p[i / 4][i % 4], f[i / 4][i % 4], pf);
            pf = group_sum<L>(pf);
            const float every = __builtin_fmaf(c, s.lse, -dot);
#pragma unroll
            for (int i = 0; i < 4 * V; ++i)
                d[i / 4][i % 4] = __builtin_fmaf(s.p[i / 4][i % 4], __builtin_fmaf(b, f[i / 4][i % 4] - pf, every), d[i / 4][i % 4]);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int e = 4 * (q * L + l);
            if (!mine_live) d[q] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (there && e < a.E) store_some<STREAM>(a.dlogits + t * a.E + e, a.E - e, d[q]);
        }
        __syncthreads();                                           // the next tokens' pairs take the place of these
    }
}

// f(lanes of a token, vectors of a lane)
template <typename F>
int with_lanes(int E, F f)
{
    using std::integral_constant;
    if (E <= 4) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (E <= 8) return f(integral_constant<int, 2>{}, integral_constant<int, 1>{});
    if (E <= 16) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (E <= 32) return f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    if (E <= 64) return f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
    if (E <= 128) return f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
    return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
}

int lanes_of(int E)
{
    return with_lanes(E, [](auto lanes, auto) { return (int)decltype(lanes)::value; });
}

// workgroups of the losses: whole rounds of tokens each
constexpr int kAlone = 4;         // up to so many one workgroup takes them alone: 256 tokens over 64 experts 5.7 us, two launches 9.0; eight rounds 12.5 and 8.8
int loss_grid(const Shape &s, int *per)
{
    const int64_t round = kLossThreads / lanes_of(s.E), rounds = (s.T + round - 1) / round;
    const int64_t each = rounds <= kAlone ? rounds : (rounds + kLossGrid - 1) / kLossGrid;
    *per = (int)std::min<int64_t>(each * round, 0x7fffffff);
    return (int)((rounds + each - 1) / each);
}

}  // namespace
}  // namespace monta

using namespace monta;

extern "C" {

int monta_route_loss_scratch_bytes(const monta_cfg *cfg, size_t *bytes)
{
    if (!bytes) return MONTA_ERR_NULL;
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    int per;
    // workgroups take whole rounds, so that more tokens may have fewer of them; scratch for more tokens does for fewer all the same
    const int64_t round = kLossThreads / lanes_of(c.s.E);
    *bytes = (size_t)loss_scratch(c.s.E, std::max(loss_grid(c.s, &per), (int)std::min<int64_t>((c.s.T + round - 1) / round, kLossGrid)));
    return MONTA_OK;
}

int monta_route_loss(const monta_cfg *cfg, const float *logits, const int32_t *topk_idx, const uint8_t *token_mask, float *losses, int32_t *counts,
                     float *means, void *scratch, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!logits || !topk_idx || !losses || !counts || !means || !scratch) return MONTA_ERR_NULL;
    if (misaligned(logits, 4) || misaligned(topk_idx, 4) || misaligned(losses, 4) || misaligned(counts, 4) || misaligned(means, 4) || misaligned(scratch, 16))
        return MONTA_ERR_ALIGN;
    int per;
    const int grid = loss_grid(c.s, &per);
    const int64_t T = c.s.T, E = c.s.E;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{logits, T * E * 4}, {topk_idx, T * c.s.k * 4}, {token_mask, T}},
      written[] = {{losses, 8}, {counts, (E + 1) * 4}, {means, E * 4}, {scratch, loss_scratch(c.s.E, grid)}};
    for (const auto &w : written) {
        for (const auto &r : read)
            if (r.p && overlap(w.p, w.n, r.p, r.n)) return MONTA_ERR_INVALID;
        for (const auto &o : written)
            if (&o != &w && overlap(w.p, w.n, o.p, o.n)) return MONTA_ERR_INVALID;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    float *partial = static_cast<float *>(scratch);
    const LossOut o = {losses, counts, means};
    {
        LaunchTimer timer(MONTA_K_ROUTE_LOSS, st);
        with_lanes(c.s.E, [&](auto lanes, auto vecs) {
            hipLaunchKernelGGL((route_loss_kernel<decltype(lanes)::value, decltype(vecs)::value>), dim3(grid), dim3(kLossThreads), 0, st, logits, topk_idx,
                               token_mask, partial, o, c.s.T, c.s.E, c.s.k, per);
            return MONTA_OK;
        });
        MONTA_HIP_TRY(hipGetLastError());
    }
    if (grid > 1) {
        LaunchTimer timer(MONTA_K_ROUTE_LOSS, st);
        hipLaunchKernelGGL(route_loss_join_kernel, dim3((c.s.E + kJoinExperts - 1) / kJoinExperts), dim3(256), 0, st, partial, o, grid, c.s.E, c.s.k);
        MONTA_HIP_TRY(hipGetLastError());
    }
    return MONTA_OK;
}

int monta_route_backward(const monta_cfg *cfg, const float *logits, const int32_t *topk_idx, const float *gates, const float *dgates,
                         const uint8_t *token_mask, const float *dlosses, const int32_t *counts, float *dlogits, void *stream)
{
    Call c;
    if (int rc = open_call(cfg, nullptr, &c)) return rc;
    if (!logits || !dlogits || (!dgates && !dlosses) || (dgates && (!topk_idx || !gates)) || (dlosses && !counts)) return MONTA_ERR_NULL;
    if (misaligned(logits, 4) || misaligned(topk_idx, 4) || misaligned(gates, 4) || misaligned(dgates, 4) || misaligned(dlosses, 4) || misaligned(counts, 4) ||
        misaligned(dlogits, 4))
        return MONTA_ERR_ALIGN;
    const int64_t T = c.s.T, E = c.s.E, pairs = T * c.s.k * 4;
    const struct {
        const void *p;
        int64_t n;
    } read[] = {{logits, T * E * 4}, {topk_idx, pairs}, {gates, pairs}, {dgates, pairs}, {token_mask, T}, {dlosses, 8}, {counts, (E + 1) * 4}};
    for (const auto &r : read)
        if (r.p && overlap(dlogits, T * E * 4, r.p, r.n)) return MONTA_ERR_INVALID;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const RouteGradArgs a = {logits, gates, dgates, dlosses, topk_idx, counts, token_mask, dlogits, c.s.T, c.s.E, c.s.k, c.s.renorm, c.s.by_k};
    const bool softmax = dlosses || (dgates && !c.s.renorm);
    LaunchTimer timer(MONTA_K_ROUTE_BACKWARD, st);
    with_lanes(c.s.E, [&](auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, V = decltype(vecs)::value, kTokens = kGradThreads / L;
        const int grid = (int)std::min<int64_t>((T + kTokens - 1) / kTokens, kRouteGrid), lds = grad_lds<L, V>(c.s.k);
        auto launch = [&](auto with_softmax, auto streamed) {
            hipLaunchKernelGGL((route_backward_kernel<L, V, decltype(with_softmax)::value, decltype(streamed)::value>), dim3(grid), dim3(kGradThreads), lds, st, a);
            return MONTA_OK;
        };
        if (stream_logits(T, E)) return softmax ? launch(std::true_type{}, std::true_type{}) : launch(std::false_type{}, std::true_type{});
        return softmax ? launch(std::true_type{}, std::false_type{}) : launch(std::false_type{}, std::false_type{});
    });
    MONTA_HIP_TRY(hipGetLastError());
    return MONTA_OK;
}

}  // extern "C"
