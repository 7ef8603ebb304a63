// Device code and argument types that the kernels of all translation units share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace monta {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kWave = 64;

// meta[] slots (int32)
enum { META_R = 0, META_ALIVE = 1, META_C = 2, META_FINAL_ROWS = 4, META_SLOTS = 16 };

struct PlanPtrs {
    int32_t *meta, *counts, *kept, *offsets, *n, *stage_off, *unit_base, *send_rows, *unit_rows;
    int32_t *pos_final, *pos_stage, *row_map, *block_counts, *block_base, *local_rank, *kept_prefix;
};

// n / d for 0 <= n < 2^16 and d < 2^15, by a multiplication: an integer division takes about 40 instructions
struct FastDiv {
    uint32_t d, m;
};
inline FastDiv fast_div(int d) { return {(uint32_t)d, d > 1 ? (uint32_t)((1ull << 32) / (uint32_t)d + 1) : 0u}; }
__device__ __forceinline__ int operator/(int n, FastDiv f) { return f.m ? (int)__umulhi((uint32_t)n, f.m) : n; }

struct Shape {
    int32_t T, E, k, ep, tp, S, U, Tu;
    int32_t TB;        // tokens per route workgroup
    int32_t bpu;       // route workgroups per unit
    int32_t num_blocks;
    int32_t C;         // per-expert capacity
    int32_t renorm;
    int32_t vpr;       // 16-byte vectors per activation row
    int32_t lpr;       // lanes cooperating on one row in the movers (power of two <= kMoverThreads)
    int32_t max_rows;  // rows STAGE / FINAL hold; every row index read from a table is checked against it
    int32_t cache;     // CachePolicy bits: which streams of the movers use non-temporal accesses
    int32_t padded;    // 1: FINAL is [E][C][H] (expert e at row e*C), 0: compact
    int32_t lazy;      // 1: the single pass requests a token's row only when it knows that one of its choices is kept
    int32_t rl;        // lanes that share one token in the route kernel (1, 2, 4 or 8)
    FastDiv by_E, by_k, by_k1, by_Tu, by_ep;       // for the pairs of a route workgroup (by_k1: k - 1) and for small problems
    int32_t fast_plan; // 1: every workgroup reduces the histogram table; 0: block_scan_kernel scans it first
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kXcds = 8;

struct ExpertArgs {
    const int32_t *lo;      // [E] first row of the expert's range
    const int32_t *hi_base; // [E] one past its last row is hi_base[e] + hi_len[e] ...
    const int32_t *hi_len;  // [E] ... or hi_base[e] alone if this is nullptr
    int16_t E;              // one word for three fields: an argument of its own is one more trip to memory in a chain of them
    int8_t spread;          // 1: the short tiles' walks along the hidden axis start at different steps (walk_start)
    int8_t deal;            // the short tiles' numbers go to the XCDs in blocks of 1 << deal
    int32_t H, N, max_rows;
    int64_t stream_from;    // first row of all experts' weights (expert * N + column) that is requested as streaming (kStreamLoad)
                            // where one workgroup reads it
};

// The expert whose tiles include logical tile number L, found without walking the experts one by one (a walk costs
// one dependent table read per expert before the workgroup can start): 64 experts at a time, one per lane, a wave
// scan of their tile counts, a ballot for the first lane whose running total passes L.  Every lane of every wave
// takes part and gets the same answer.  e == E: no such tile (a surplus workgroup).
struct ExpertTileHit {
    int e, lo, hi, tiles;     // expert, its row range [lo, hi), its row tiles
    uint32_t L;               // tile number inside the expert: at most the number asked for, which is below 2^31, as grids are
};

// WHOLE: only the whole tiles of a segment count (its ragged last tile is numbered elsewhere); `all` returns the
// number of tiles counted over all experts when L lies past them.
template <int BM, bool WHOLE = false>
__device__ __forceinline__ ExpertTileHit find_expert_tile(const ExpertArgs &a, int nct, int64_t L, int lane,
                                                          int64_t *all = nullptr)
{
    ExpertTileHit h;
    h.e = a.E;
    h.lo = h.hi = h.tiles = 0;
    h.L = 0;
    int64_t before = 0;                                            // tiles of the experts of earlier rounds
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
        const int e = e0 + lane;
        int lo = 0, hi = 0, tiles = 0;
        if (e < a.E) {
            lo = a.lo[e];
            hi = a.hi_base[e] + (a.hi_len ? a.hi_len[e] : 0);
            tiles = hi > lo ? (int)(((int64_t)hi - lo + (WHOLE ? 0 : BM - 1)) / BM) : 0;
        }
        const int64_t cnt = (int64_t)tiles * nct;
        int64_t incl = cnt;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int64_t o = __shfl_up(incl, d, kWave);
            if (lane >= d) incl += o;
        }
        // 64 bits, and by a shuffle: from a lane read the compiler knows the tile's number for uniform and divides it in scalar code,
        // four long chains of which cost every large tile's workgroup about 2 us (128 experts of 1024 x 480, 512 rows each 97 and 94).
        // The quotients themselves are of 32 bits: those of 64 cost short tiles up to 2 % (fp32, 8 of 512 x 2496, 105 rows 28.9 and 28.3)
        const int64_t total = __shfl(incl, kWave - 1, kWave);
        if (L < before + total) {
            // an expert without tiles repeats its predecessor's running total, so the first lane past L has tiles
            const unsigned long long past = __ballot(L < before + incl);
            const int src = __ffsll((long long)past) - 1;
            h.e = e0 + src;
            h.lo = __shfl(lo, src, kWave);
            h.hi = __shfl(hi, src, kWave);
            h.tiles = __shfl(tiles, src, kWave);
            h.L = (uint32_t)(L - before - (__shfl(incl, src, kWave) - __shfl(cnt, src, kWave)));
            return h;
        }
        before += total;
    }
    if (all) *all = before;
    return h;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}
typedef __attribute__((address_space(3))) void lds_void;

constexpr uint32_t kOutOfRange = 0x80000000u;                      // a lane offset past every descriptor: no access

constexpr int kBigMaxHidden = 1 << 20;                             // a tile's 256 rows end far below it
constexpr int64_t kMostRows = 0x7fffffff - 4096;                   // row numbers some steps past the last one are still numbers of 32 bits

// Where tile number `tile` starts its walk along the hidden axis.  Rows that are a multiple of 4096 bytes apart begin on the same memory
// channels, so that workgroups which walk in step all wait for a few of them: 256 MiB of weights in rows of 8192 bytes, 64 rows a workgroup,
// read and nothing else, arrive in 52 us, at 14336 bytes a row in 39 (6.9 TB/s); with the starts spread over the row in 39 and 39.  The
// multiplier spreads consecutive tiles evenly over any number of steps.  Rows have to be whole steps.
__device__ __forceinline__ int walk_start(int tile, int nsteps)
{
    return (int)(((uint32_t)tile * 40503u & 0xffffu) * (uint32_t)nsteps >> 16);
}

// ------------------------------------------------------------------ tiles of a grouped product

constexpr int kShortTileRows = 64;       // ragged tiles up to this many rows run as short tiles, where a kernel has those

// What a tile of the output belongs to.
struct RowTile {
    int e = -1, row0 = 0, row_end = 0;   // expert (none: < 0); its rows
    int rt = 0, ct = 0;                  // row tile and column tile inside the expert
    int side = 1, share = 0;             // row tiles next to one another on one column tile; which of them
};

// Logical tile number of workgroup `block`: they go out in blocks of 256, 32 consecutive ones to each XCD (hardware deals consecutive
// workgroups round robin to the 8 XCDs, each with its own L2).
__device__ __forceinline__ int64_t tile_number(uint32_t block)
{
    const int64_t j = block / kXcds;
    return (j / 32) * (32 * kXcds) + (int64_t)(block % kXcds) * 32 + j % 32;
}

// Inside an expert the numbering is (panel of 8 row tiles, column tile, row tile), so that an XCD's workgroups share operand tiles.
__device__ __forceinline__ void place_in_panels(RowTile &t, uint32_t in, int tiles, int nct)
{
    constexpr int P = 8;
    const int full = tiles / P;
    const bool whole = in < (uint32_t)(full * P) * (uint32_t)nct;
    const uint32_t rem = whole ? in % (uint32_t)(P * nct) : in - (uint32_t)(full * P) * (uint32_t)nct;
    t.side = whole ? P : tiles - full * P;
    t.ct = (int)(rem / (uint32_t)t.side);
    t.share = (int)(rem % (uint32_t)t.side);
    t.rt = (whole ? (int)(in / (uint32_t)(P * nct)) : full) * P + t.share;
}

// Tile of BR rows of workgroup `block`.  RAGGED_LAST: the whole tiles of all experts come first and the segments' ragged last tiles after
// them, the one with the most rows first, so that the last round of workgroups consists of the tiles that cost least; those of at most
// kShortTileRows rows as halves of the column tile (ct counts halves).  For whole segments (hi_len), at least 256 threads and E <= 256; `scratch`: 257
// words of LDS that nothing else uses yet.
template <int BR, bool RAGGED_LAST>
__device__ __forceinline__ RowTile find_row_tile(const ExpertArgs &a, int nct, uint32_t block, int lane, int *scratch)
{
    const int64_t L = tile_number(block);
    RowTile t;
    int lo, hi;
    int64_t whole_tiles = 0;
    const ExpertTileHit hit = find_expert_tile<BR, RAGGED_LAST>(a, nct, L, lane, &whole_tiles);
    if (hit.e < a.E) {
        t.e = hit.e;
        lo = hit.lo;
        hi = hit.hi;
        place_in_panels(t, hit.L, hit.tiles, nct);
    } else if constexpr (RAGGED_LAST) {
        // position (L - whole tiles) / nct in the order (rows of the ragged tile, descending; expert, ascending), of the halves 2 nct
        const int64_t Lr = L - whole_tiles;
        const int tid = threadIdx.x;
        int mine = 0;
        if (tid < a.E) {
            const int first = a.lo[tid], last = a.hi_base[tid] + a.hi_len[tid];
            mine = last > first ? (last - first) % BR : 0;
            scratch[tid] = mine;
        }
        if (tid == 0) scratch[256] = -1;
        __syncthreads();
        int rank = 0, long_ones = 0;
        for (int o = 0; o < a.E; ++o) {
            const int other = scratch[o];
            long_ones += other > kShortTileRows ? 1 : 0;
            rank += other > mine || (other == mine && o < tid) ? 1 : 0;
        }
        const int64_t halves = Lr - (int64_t)long_ones * nct;      // number among the halves
        if (mine > 0 && rank == (halves < 0 ? Lr / nct : long_ones + halves / (2 * nct))) scratch[256] = tid;
        __syncthreads();
        t.e = scratch[256];
        __syncthreads();                                           // everyone has read it before the stages are laid down
        if (t.e < 0) return t;
        lo = a.lo[t.e];
        hi = a.hi_base[t.e] + a.hi_len[t.e];
        t.ct = (int)(halves < 0 ? Lr % nct : halves % (2 * nct));
        t.rt = (hi - lo) / BR;
    } else {
        return t;
    }
    hi = min(hi, a.max_rows);
    lo = max(lo, 0);
    t.row0 = lo + t.rt * BR;
    t.row_end = min(hi, t.row0 + BR);
    if (t.row0 >= t.row_end) t.e = -1;
    return t;
}

}  // namespace monta
