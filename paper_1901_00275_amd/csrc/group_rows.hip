// Rows sent to the cells (experts) they were given to, and back: a stable counting sort of the n w (row, choice) pairs by
// cell, the rows gathered in that order, and their weighted sums row by row, with the gradients of both.
//
// The sort goes by digits of at most DIGIT bits, the lowest first, and keeps the order of equal ones: every workgroup counts
// the digits of a tile, the counts of a digit are summed over the tiles, and the workgroup ranks its pairs: a wave's
// pairs in turn, 64 at a time, those of one digit told apart by ballots.  No atomics on memory, so the order is the pairs' own.
// What bounds it are launches of 5 to 11 us, each some waits for memory one behind the other: 640 000 pairs and 65 536 cells
// (two digits) 51 us in seven launches, 13 MB of pairs and places.  Up to SMALL_PAIRS pairs of one digit take one launch.
// The rest moves memory: 16 bytes at a time, several rows' loads under way.  640 000 rows of 384 bytes
// gathered 41 us (6.0 TB/s written), 16 384 rows of 8 x 4 KB combined 109 us (5.4 TB/s; with a branch around each load
// 136), the gradient of 5 003 x 6 x 2 KB 26 us (5.0).
#include "learn.h"

#include <type_traits>

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_t;

#define DIGIT 11
#define BINS (1 << DIGIT)
#define GNT 256          // threads of a workgroup of the sort
#define GWAVES (GNT / 64)
#define SMALL_NT 1024    // threads where one workgroup sorts everything
#define SMALL_PAIRS 16384

// lanes whose digit is this lane's
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool there)
{
    uint64_t m = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1;
        const uint64_t v = __ballot(one);
        m &= one ? v : ~v;
    }
    return m;
}

struct SortPass {
    const int32_t *cell;         // the first pass reads the cells, the later ones keys and pairs
    const uint2 *moved;          // {key, pair}
    uint2 *moved_out;
    uint32_t *to;                // where each went, in the order they came; the last pass: -1 if it is dropped
    int32_t *place, *source;     // the only pass
    int64_t *off;
    uint32_t *count;             // [tiles][bins]
    uint32_t *total;             // [bins]
    int64_t pairs;
    int cells, shift, bits, tile, tiles;
    bool last, only;
};

__device__ __forceinline__ uint32_t key_at(const SortPass &a, int64_t i)
{
    if (!a.cell) return a.moved[i].x;
    const uint32_t c = (uint32_t)a.cell[i];
    return c < (uint32_t)a.cells ? c : (uint32_t)a.cells; // (dropped pairs stand behind all cells)
}

__global__ __launch_bounds__(GNT) void k_group_count(SortPass a)
{
    __shared__ uint32_t h[BINS];
    const int bins = 1 << a.bits;
    for (int b = threadIdx.x; b < bins; b += GNT) h[b] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * a.tile;
    const int count = (int)(a.pairs - i0 < a.tile ? a.pairs - i0 : a.tile);
#pragma unroll 8
    for (int i = threadIdx.x; i < count; i += GNT) atomicAdd(&h[(key_at(a, i0 + i) >> a.shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += GNT) a.count[(int64_t)blockIdx.x * bins + b] = h[b];
}

// wave-wide inclusive sum
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    return v;
}

// exclusive sums of a digit's counts over the tiles: 16 digits a workgroup, the tiles in 64 slices
#define SLICES 64
__global__ __launch_bounds__(SLICES * 16) void k_group_tiles(uint32_t *count, uint32_t *total, int tiles, int bins)
{
    __shared__ uint32_t sum[16][SLICES + 1];
    const int b = threadIdx.x & 15, slice = threadIdx.x >> 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int digit = blockIdx.x * 16 + b, per = (tiles + SLICES - 1) / SLICES;
    const int t0 = slice * per, t1 = digit < bins ? min(t0 + per, tiles) : 0;
    uint32_t s = 0;
#pragma unroll 8
    for (int t = t0; t < t1; ++t) s += count[(int64_t)t * bins + digit];
    sum[b][slice] = s;
    __syncthreads();
    const uint32_t own = sum[wave][lane], upto = wave_scan(own, lane); // (a wave: a digit's slices)
    sum[wave][lane] = upto - own;
    if (lane == 63 && blockIdx.x * 16 + wave < bins) total[blockIdx.x * 16 + wave] = upto;
    __syncthreads();
    s = sum[b][slice];
#pragma unroll 8
    for (int t = t0; t < t1; ++t) {
        const uint32_t v = count[(int64_t)t * bins + digit];
        count[(int64_t)t * bins + digit] = s;
        s += v;
    }
}

// in place: exclusive sums of v[0 .. bins) by NT threads, v in LDS; the values behind are not touched
template <int NT>
__device__ __forceinline__ void block_scan(uint32_t *v, int bins, uint32_t *wsum)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (bins + NT - 1) / NT;
    uint32_t sum = 0;
    for (int i = tid * per; i < min(tid * per + per, bins); ++i) sum += v[i];
    const uint32_t s = wave_scan(sum, lane);
    if (lane == 63) wsum[wave] = s;
    __syncthreads();
    uint32_t base = s - sum;
    for (int w = 0; w < wave; ++w) base += wsum[w];
    for (int i = tid * per; i < min(tid * per + per, bins); ++i) {
        const uint32_t t = v[i];
        v[i] = base;
        base += t;
    }
    __syncthreads();
}

// The pairs of a wave (i0 .. i0 + count) to their places, HELD at a time: their keys, and where they have moved already the
// pairs themselves, are asked for together.  at[digit] is the next place of a digit, kept up by the wave alone.
#define HELD 8
__device__ __forceinline__ void hold(const SortPass &a, int64_t i0, int lane, uint32_t (&key)[HELD], uint32_t (&pair)[HELD])
{
#pragma unroll
    for (int u = 0; u < HELD; ++u) { // (no branch around a load, it would wait for it)
        const int64_t i = min(i0 + u * 64 + lane, a.pairs - 1);
        const uint2 v = a.cell ? make_uint2((uint32_t)a.cell[i], (uint32_t)i) : a.moved[i];
        key[u] = v.x;
        pair[u] = v.y;
    }
    if (a.cell)
#pragma unroll
        for (int u = 0; u < HELD; ++u) key[u] = min(key[u], (uint32_t)a.cells);
}
__device__ __forceinline__ void place_held(const SortPass &a, uint32_t *at, int64_t i0, int count, int lane, const uint32_t (&key)[HELD], const uint32_t (&pair)[HELD])
{
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
        if (u * 64 >= count) break;
        const bool there = u * 64 + lane < count;
        const uint32_t digit = there ? (key[u] >> a.shift) & ((1u << a.bits) - 1) : 0;
        const uint64_t same = same_digit(digit, a.bits, there);
        uint32_t p = 0;
        if (there) p = at[digit] + __popcll(same & below);
        wave_lds_order();
        if (there && !(same & below)) at[digit] += __popcll(same);
        wave_lds_order();
        if (!there) continue;
        if (!a.only) {
            a.moved_out[p] = make_uint2(key[u], pair[u]);
            a.to[i0 + u * 64 + lane] = a.last && key[u] >= (uint32_t)a.cells ? 0xFFFFFFFFu : p;
        } else {
            const bool in = key[u] < (uint32_t)a.cells;
            a.source[p] = in ? (int32_t)pair[u] : -1;
            a.place[pair[u]] = in ? (int32_t)p : -1;
        }
    }
}
__device__ __forceinline__ void place_pairs(const SortPass &a, uint32_t *at, int64_t i0, int count, int lane)
{
    uint32_t key[HELD], pair[HELD];
    for (int i = 0; i < count; i += HELD * 64) {
        hold(a, i0 + i, lane, key, pair);
        place_held(a, at, i0 + i, count - i, lane, key, pair);
    }
}

__global__ __launch_bounds__(GNT) void k_group_place(SortPass a)
{
    __shared__ uint32_t first[BINS], at[GWAVES][BINS], wsum[GWAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = 1 << a.bits;
    uint32_t key[HELD], pair[HELD]; // the wave's first pairs, asked for before all else
    hold(a, (int64_t)blockIdx.x * a.tile + wave * (a.tile / GWAVES), lane, key, pair);
    uint32_t before[BINS / GNT]; // of each digit, in the tiles before this one
#pragma unroll
    for (int i = 0; i < BINS / GNT; ++i) {
        const int b = i * GNT + tid;
        if (b < bins) before[i] = a.count[(int64_t)blockIdx.x * bins + b];
    }
    for (int b = tid; b < bins; b += GNT) {
        first[b] = a.total[b];
        for (int w = 0; w < GWAVES; ++w) at[w][b] = 0;
    }
    __syncthreads();
    block_scan<GNT>(first, bins, wsum);
    if (a.only && blockIdx.x == 0) // (cells + 1 <= bins)
        for (int b = tid; b <= a.cells; b += GNT) a.off[b] = first[b];
    const int64_t i0 = (int64_t)blockIdx.x * a.tile;
    const int per = a.tile / GWAVES, count = (int)max((int64_t)0, min((int64_t)per, a.pairs - i0 - wave * per));
    for (int i = HELD * 64 + lane; i < count; i += 64) atomicAdd(&at[wave][(key_at(a, i0 + wave * per + i) >> a.shift) & (bins - 1)], 1u);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
        if (u * 64 + lane < count) atomicAdd(&at[wave][(key[u] >> a.shift) & (bins - 1)], 1u);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BINS / GNT; ++i) {
        const int b = i * GNT + tid;
        if (b >= bins) continue;
        uint32_t next = first[b] + before[i];
        for (int w = 0; w < GWAVES; ++w) {
            const uint32_t c = at[w][b];
            at[w][b] = next;
            next += c;
        }
    }
    __syncthreads();
    place_held(a, at[wave], i0 + wave * per, count, lane, key, pair);
    if (count > HELD * 64) place_pairs(a, at[wave], i0 + wave * per + HELD * 64, count - HELD * 64, lane);
}

// Few pairs, few cells: one workgroup, one launch
__global__ __launch_bounds__(SMALL_NT) void k_group_small(SortPass a)
{
    extern __shared__ uint32_t lds[]; // [16][bins] a wave's next places, [bins] a digit's first
    constexpr int W = SMALL_NT / 64;
    __shared__ uint32_t wsum[W];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = 1 << a.bits;
    uint32_t *first = lds + W * bins;
    for (int b = tid; b < W * bins; b += SMALL_NT) lds[b] = 0;
    __syncthreads();
    const int per = ((int)a.pairs + W * 64 - 1) / (W * 64) * 64, i0 = wave * per, count = max(0, min(per, (int)a.pairs - i0));
    for (int i = lane; i < count; i += 64) atomicAdd(&lds[wave * bins + key_at(a, i0 + i)], 1u);
    __syncthreads();
    for (int b = tid; b < bins; b += SMALL_NT) {
        uint32_t sum = 0;
        for (int w = 0; w < W; ++w) sum += lds[w * bins + b];
        first[b] = sum;
    }
    __syncthreads();
    block_scan<SMALL_NT>(first, bins, wsum);
    for (int b = tid; b < bins; b += SMALL_NT) {
        uint32_t next = first[b];
        if (b <= a.cells) a.off[b] = next;
        for (int w = 0; w < W; ++w) {
            const uint32_t c = lds[w * bins + b];
            lds[w * bins + b] = next;
            next += c;
        }
    }
    __syncthreads();
    place_pairs(a, lds + wave * bins, i0, count, lane);
}

// Few pairs, many cells: one workgroup takes all passes in LDS, k_group_end the rest.  (6 pairs, 57 575 cells, with the gather: 29 us by a
// launch for each step, 18 now; 4 096 pairs, 65 536 cells 30 and 22.)
#define FEW_DIGIT 9
#define FEW_SORTED 4096
__global__ __launch_bounds__(SMALL_NT) void k_group_few(SortPass a)
{
    constexpr int W = SMALL_NT / 64, MOST = 1 << FEW_DIGIT;
    extern __shared__ uint32_t lds[]; // {key, pair} [2][FEW_SORTED], [W][bins] a wave's next places, [bins] a digit's first
    __shared__ uint32_t wsum[W];
    uint2 *from = (uint2 *)lds, *to = from + FEW_SORTED;
    uint32_t *at = (uint32_t *)(to + FEW_SORTED), *first = at + W * MOST;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pairs = (int)a.pairs;
    const int per = (pairs + W * 64 - 1) / (W * 64) * 64, i0 = wave * per, i1 = min(i0 + per, pairs);
    for (int i = tid; i < pairs; i += SMALL_NT) from[i] = make_uint2(key_at(a, i), (uint32_t)i);
    for (int shift = 0; shift < a.bits; shift += FEW_DIGIT) {
        const int bits = min(FEW_DIGIT, a.bits - shift), bins = 1 << bits;
        for (int b = tid; b < W * bins; b += SMALL_NT) at[b] = 0;
        __syncthreads();
        for (int i = i0 + lane; i < i1; i += 64) atomicAdd(&at[wave * bins + ((from[i].x >> shift) & (bins - 1))], 1u);
        __syncthreads();
        for (int b = tid; b < bins; b += SMALL_NT) {
            uint32_t sum = 0;
            for (int w = 0; w < W; ++w) sum += at[w * bins + b];
            first[b] = sum;
        }
        __syncthreads();
        block_scan<SMALL_NT>(first, bins, wsum);
        for (int b = tid; b < bins; b += SMALL_NT) {
            uint32_t next = first[b];
            for (int w = 0; w < W; ++w) {
                const uint32_t c = at[w * bins + b];
                at[w * bins + b] = next;
                next += c;
            }
        }
        __syncthreads();
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        for (int i = i0; i < i1; i += 64) {
            const bool there = i + lane < i1;
            const uint2 v = from[there ? i + lane : i];
            const uint32_t digit = (v.x >> shift) & (bins - 1);
            const uint64_t same = same_digit(digit, bits, there);
            uint32_t *next = at + wave * bins + digit;
            if (there) to[*next + __popcll(same & below)] = v;
            wave_lds_order();
            if (there && !(same & below)) *next += __popcll(same);
            wave_lds_order();
        }
        __syncthreads();
        uint2 *t = from;
        from = to;
        to = t;
    }
    for (int p = tid; p < pairs; p += SMALL_NT) {
        const uint2 v = from[p];
        a.moved_out[p] = v;
        a.to[v.y] = v.x < (uint32_t)a.cells ? (uint32_t)p : 0xFFFFFFFFu;
    }
}

// What several passes leave to be written, all of it in order: off[c], the first place whose cell is c or more; source; and
// place, by following a pair through the passes.  (Written by the last pass, the places lay 4 bytes here and 4 there: 640 000
// pairs, 65 536 cells, that pass 20 us and the offsets 6; now 11 and 9.)
#define SAMPLES 512 // keys among which a cell's first is looked for in LDS: ten fewer reads of memory one behind the other, 11 -> 9 us
struct GroupEnd {
    const uint2 *moved;
    const uint32_t *to[3];
    int64_t pairs;
    int passes, cells, off_blocks;
    int64_t *off;
    int32_t *place, *source;
};
__global__ __launch_bounds__(256) void k_group_end(GroupEnd a)
{
    if ((int)blockIdx.x < a.off_blocks) {
        __shared__ uint32_t sample[SAMPLES];
        const int64_t step = a.pairs / (SAMPLES - 1) + 1; // (the last lies past the end)
        for (int i = threadIdx.x; i < SAMPLES; i += 256) sample[i] = i * step < a.pairs ? a.moved[i * step].x : 0xFFFFFFFFu;
        __syncthreads();
        const int c = blockIdx.x * 256 + threadIdx.x;
        if (c > a.cells) return;
        int before = 0; // samples below c
        for (int b = SAMPLES / 2; b > 0; b >>= 1)
            if (sample[before + b - 1] < (uint32_t)c) before += b;
        int64_t lo = before > 0 ? (before - 1) * step + 1 : 0, hi = min(before * step, a.pairs);
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (a.moved[mid].x < (uint32_t)c)
                lo = mid + 1;
            else
                hi = mid;
        }
        a.off[c] = lo;
        return;
    }
    const int64_t i = (int64_t)(blockIdx.x - a.off_blocks) * 256 + threadIdx.x;
    if (i >= a.pairs) return;
    const uint2 own = a.moved[i];
    uint32_t p = a.to[0][i];
    for (int q = 1; q < a.passes; ++q) p = a.to[q][p];
    a.source[i] = own.x < (uint32_t)a.cells ? (int32_t)own.y : -1;
    a.place[i] = (int32_t)p;
}

__global__ __launch_bounds__(256) void k_group_none(int cells, int64_t *off)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c <= cells) off[c] = 0;
}

struct GroupPlan {
    int passes, bits[3], tile, tiles;
    size_t count_off, total_off, moved_off[2], to_off[3], bytes;
    bool small, few;
};

static GroupPlan group_plan(int64_t pairs, int cells)
{
    GroupPlan p = {};
    int bits = 1;
    while (((int64_t)1 << bits) < (int64_t)cells + 1) ++bits;
    p.passes = (bits + DIGIT - 1) / DIGIT;
    for (int i = 0, left = bits; i < p.passes; ++i) {
        p.bits[i] = (left + p.passes - i - 1) / (p.passes - i);
        left -= p.bits[i];
    }
    p.small = p.passes == 1 && pairs <= SMALL_PAIRS;
    p.few = p.passes > 1 && pairs <= FEW_SORTED;
    if (p.few) {
        p.passes = 1;
        p.bits[0] = bits;
    }
    // tiles: enough of them for every compute unit, large enough that the counts are fewer than the pairs
    p.tile = GWAVES * HELD * 64 / 2;
    while (p.tile < 8192 && pairs / p.tile > 512) p.tile *= 2;
    p.tiles = (int)((pairs + p.tile - 1) / p.tile);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = (off + bytes + 255) & ~(size_t)255;
        return at;
    };
    if (!p.small) {
        p.count_off = take((size_t)BINS * p.tiles * 4);
        p.total_off = take((size_t)BINS * 4);
        if (p.passes > 1 || p.few)
            for (int i = 0; i < 2; ++i) p.moved_off[i] = take((size_t)pairs * sizeof(uint2));
        if (p.passes > 1 || p.few)
            for (int i = 0; i < p.passes; ++i) p.to_off[i] = take((size_t)pairs * 4);
    }
    p.bytes = off + 256;
    return p;
}

size_t group_workspace(int64_t pairs, int cells) { return group_plan(pairs, cells).bytes; }

int launch_group_rows(const int32_t *cell, int64_t pairs, int cells, int64_t *off, int32_t *place, int32_t *source, void *ws,
                      hipStream_t st)
{
    const dim3 cgrid((unsigned)(cells / 256 + 1));
    if (pairs == 0) {
        hipLaunchKernelGGL(k_group_none, cgrid, dim3(256), 0, st, cells, off);
        return (int)hipGetLastError();
    }
    const GroupPlan p = group_plan(pairs, cells);
    char *base = (char *)ws;
    SortPass a = {};
    a.cell = cell;
    a.place = place;
    a.source = source;
    a.off = off;
    a.count = (uint32_t *)(base + p.count_off);
    a.total = (uint32_t *)(base + p.total_off);
    a.pairs = pairs;
    a.cells = cells;
    a.tile = p.tile;
    a.tiles = p.tiles;
    a.only = p.passes == 1;
    if (p.small) {
        a.bits = p.bits[0];
        const size_t bytes = (size_t)(SMALL_NT / 64 + 1) * (4u << a.bits);
        if (bytes > 49152) { // (48 KB of dynamic LDS need no asking)
            const hipError_t e = hipFuncSetAttribute((const void *)k_group_small, hipFuncAttributeMaxDynamicSharedMemorySize, (SMALL_NT / 64 + 1) * BINS * 4);
            if (e != hipSuccess) return (int)e;
        }
        hipLaunchKernelGGL(k_group_small, dim3(1), dim3(SMALL_NT), bytes, st, a);
        return (int)hipGetLastError();
    }
    GroupEnd end = {nullptr, {}, pairs, p.passes, cells, (int)cgrid.x, off, place, source};
    const dim3 ends((unsigned)(cgrid.x + (pairs + 255) / 256));
    if (p.few) {
        a.bits = p.bits[0];
        a.moved_out = (uint2 *)(base + p.moved_off[0]);
        a.to = (uint32_t *)(base + p.to_off[0]);
        end.moved = a.moved_out;
        end.to[0] = a.to;
        const size_t bytes = 2 * FEW_SORTED * sizeof(uint2) + (SMALL_NT / 64 + 1) * (4u << FEW_DIGIT);
        const hipError_t e = hipFuncSetAttribute((const void *)k_group_few, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return (int)e;
        hipLaunchKernelGGL(k_group_few, dim3(1), dim3(SMALL_NT), bytes, st, a);
        hipLaunchKernelGGL(k_group_end, ends, dim3(256), 0, st, end);
        return (int)hipGetLastError();
    }
    for (int i = 0; i < p.passes; ++i) {
        a.bits = p.bits[i];
        a.last = i == p.passes - 1;
        a.moved_out = (uint2 *)(base + p.moved_off[i & 1]);
        a.to = (uint32_t *)(base + p.to_off[i]);
        end.to[i] = a.to;
        hipLaunchKernelGGL(k_group_count, dim3((unsigned)p.tiles), dim3(GNT), 0, st, a);
        hipLaunchKernelGGL(k_group_tiles, dim3((unsigned)(((1 << a.bits) + 15) / 16)), dim3(SLICES * 16), 0, st, a.count, a.total,
                           p.tiles, 1 << a.bits);
        hipLaunchKernelGGL(k_group_place, dim3((unsigned)p.tiles), dim3(GNT), 0, st, a);
        a.cell = nullptr;
        a.moved = a.moved_out;
        a.shift += a.bits;
    }
    if (p.passes > 1) {
        end.moved = a.moved;
        hipLaunchKernelGGL(k_group_end, ends, dim3(256), 0, st, end);
    }
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
// A piece of a row: 16 bytes, less where a row has fewer.  The memory takes them at any value's address, so rows of all sizes and
// alignments go this way; the last piece of a row ends where the row does and overlaps the one before it, whose values it
// writes again.  WHOLE: all rows lie on 16 bytes; they are stored past the caches, which others would need to put their lines
// together.  (5 000 x 8 rows of 2 050 bytes combined: 61 us value by value, 17 so.)
template <typename T, int BYTES, bool WHOLE>
struct Piece {
    static constexpr int N = BYTES / (int)sizeof(T);
    using Word = std::conditional_t<BYTES == 16, u32x4, std::conditional_t<BYTES == 8, u32x2, std::conditional_t<BYTES == 4, uint32_t, uint16_t>>>;
    typedef Word At __attribute__((aligned(sizeof(T))));
    T v[N];
    // the first value of piece c
    static __device__ __forceinline__ uint32_t at(uint32_t c, int d) { return WHOLE ? c * N : min(c * N, (uint32_t)(d - N)); }
};
template <typename T, int BYTES, bool WHOLE>
__device__ __forceinline__ Piece<T, BYTES, WHOLE> load_piece(const T *p)
{
    using P = Piece<T, BYTES, WHOLE>;
    return __builtin_bit_cast(P, *(const typename P::At *)p);
}
template <typename T, int BYTES, bool WHOLE>
__device__ __forceinline__ void store_piece(T *p, const Piece<T, BYTES, WHOLE> &r)
{
    using P = Piece<T, BYTES, WHOLE>;
    if constexpr (WHOLE)
        __builtin_nontemporal_store(__builtin_bit_cast(typename P::Word, r), (typename P::At *)p);
    else
        *(typename P::At *)p = __builtin_bit_cast(typename P::Word, r);
}

#define ROW_NT 256
#define ROW_ITEMS 4 // pieces a thread has under way

struct RowsArgs {
    int64_t n;
    int w, d;
    uint32_t per;  // pieces of a row
    uint32_t rows; // rows of a workgroup
    int64_t block; // the launch's first workgroup
    const int32_t *index; // source or place
    const float *weight;
};

// y[p] = x[source[p] / w]: the pieces of a workgroup's rows, ROW_ITEMS a thread at a time
template <typename T, int BYTES, bool WHOLE>
__global__ __launch_bounds__(ROW_NT) void k_gather_rows(RowsArgs a, const T *__restrict__ x, T *__restrict__ y)
{
    using P = Piece<T, BYTES, WHOLE>;
    const int64_t places = a.n * a.w, p0 = (a.block + blockIdx.x) * a.rows;
    const uint32_t pieces = (uint32_t)min((int64_t)a.rows, places - p0) * a.per;
    for (uint32_t i0 = threadIdx.x; i0 < pieces; i0 += ROW_NT * ROW_ITEMS) {
        P v[ROW_ITEMS];
        int64_t to[ROW_ITEMS];
#pragma unroll
        for (int u = 0; u < ROW_ITEMS; ++u) {
            const uint32_t i = i0 + u * ROW_NT, r = i / a.per, c = i - r * a.per;
            to[u] = -1;
            if (i >= pieces) continue;
            const int32_t s = a.index[p0 + r];
            if ((int64_t)s >= places || s < 0) continue; // (a place behind the last pair)
            v[u] = load_piece<T, BYTES, WHOLE>(x + (int64_t)((uint32_t)s / (uint32_t)a.w) * a.d + P::at(c, a.d));
            to[u] = (p0 + r) * a.d + P::at(c, a.d);
        }
#pragma unroll
        for (int u = 0; u < ROW_ITEMS; ++u)
            if (to[u] >= 0) store_piece<T, BYTES, WHOLE>(y + to[u], v[u]);
    }
}

// out[i] = sum over the row's choices of weight y[place], in their order, in fp32
template <typename T, int BYTES, bool WHOLE, int U>
__global__ __launch_bounds__(ROW_NT) void k_combine_rows(RowsArgs a, const T *__restrict__ y, T *__restrict__ out)
{
    using P = Piece<T, BYTES, WHOLE>;
    const int64_t places = a.n * a.w, r0 = (a.block + blockIdx.x) * a.rows;
    const uint32_t pieces = (uint32_t)min((int64_t)a.rows, a.n - r0) * a.per;
    for (uint32_t i = threadIdx.x; i < pieces; i += ROW_NT) {
        const uint32_t r = i / a.per, at = P::at(i - r * a.per, a.d);
        const int32_t *pl = a.index + (r0 + r) * a.w;
        const float *wt = a.weight ? a.weight + (r0 + r) * a.w : (const float *)pl; // (read either way: a branch around a load would wait for it)
        float s[P::N] = {};
        for (int q0 = 0; q0 < a.w; q0 += U) { // (so many rows' loads under way)
            P v[U];
            float f[U];
            int32_t p[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                p[q] = pl[min(q0 + q, a.w - 1)];
                f[q] = wt[min(q0 + q, a.w - 1)];
            }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const bool in = q0 + q < a.w && (uint32_t)p[q] < (uint64_t)places;
                v[q] = load_piece<T, BYTES, WHOLE>(y + (in ? (int64_t)p[q] * a.d : 0) + at);
                if (!a.weight) f[q] = 1.f;
                if (!in) p[q] = -1;
            }
#pragma unroll
            for (int q = 0; q < U; ++q)
#pragma unroll
                for (int e = 0; e < P::N; ++e) s[e] = p[q] < 0 ? s[e] : fmaf(f[q], (float)v[q].v[e], s[e]);
        }
        P o;
#pragma unroll
        for (int e = 0; e < P::N; ++e) o.v[e] = (T)s[e];
        store_piece<T, BYTES, WHOLE>(out + (r0 + r) * a.d + at, o);
    }
}

// dy[place] = weight dout[i], dweight[i][c] = <dout[i], y[place]>: L lanes eight choices of a row
// (all choices of a row one after the other: 1 337 x 64 rows of 1 516 bytes 110 us, now 64)
template <typename T, int BYTES, bool WHOLE, int L>
__global__ __launch_bounds__(ROW_NT) void k_combine_back(RowsArgs a, const T *__restrict__ dout, const T *__restrict__ y,
                                                         T *__restrict__ dy, float *__restrict__ dweight)
{
    using P = Piece<T, BYTES, WHOLE>;
    const int lane = threadIdx.x & (L - 1);
    const uint32_t eights = (a.w + 7) / 8, id = (uint32_t)((a.block + blockIdx.x) * (ROW_NT / L) + threadIdx.x / L); // (n w < 2^31)
    const int64_t places = a.n * a.w, r = id / eights;
    if (r >= a.n) return;
    const int q0 = (int)(id % eights) * 8;
    const float *weight = a.weight ? a.weight : (const float *)a.index; // (read either way: a branch around a load would wait for it)
    int32_t at[8];
    int64_t p[8];
    float f[8], dot[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const int64_t i = r * a.w + min(q0 + q, a.w - 1);
        at[q] = a.index[i];
        f[q] = weight[i];
        dot[q] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        p[q] = q0 + q < a.w && (uint32_t)at[q] < (uint64_t)places ? at[q] : -1;
        if (!a.weight) f[q] = 1.f;
    }
    for (uint32_t c = lane; c < a.per; c += L) {
        const uint32_t c0 = P::at(c, a.d), again = c * P::N - c0; // (values that the piece before had)
        const P g = load_piece<T, BYTES, WHOLE>(dout + r * a.d + c0);
        P v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (dweight) v[q] = load_piece<T, BYTES, WHOLE>(y + max(p[q], (int64_t)0) * a.d + c0);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (p[q] < 0) continue;
            P o;
#pragma unroll
            for (int e = 0; e < P::N; ++e) {
                o.v[e] = (T)(f[q] * (float)g.v[e]);
                if (dweight && e >= (int)again) dot[q] = fmaf((float)g.v[e], (float)v[q].v[e], dot[q]);
            }
            if (dy) store_piece<T, BYTES, WHOLE>(dy + p[q] * a.d + c0, o);
        }
    }
    if (!dweight) return;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) dot[q] += __shfl_xor(dot[q], o, 64);
        if (lane == 0 && q0 + q < a.w) dweight[r * a.w + q0 + q] = p[q] < 0 ? 0.f : dot[q];
    }
}

// go(bytes of a piece, WHOLE)
template <typename T, typename F>
static void by_pieces(int d, const void *p, const void *q, const void *r, F &&go)
{
    const uint64_t bytes = (uint64_t)d * sizeof(T);
    if ((bytes | (uintptr_t)p | (uintptr_t)q | (uintptr_t)r) % 16 == 0)
        go(std::integral_constant<int, 16>{}, std::true_type{});
    else if (bytes >= 16)
        go(std::integral_constant<int, 16>{}, std::false_type{});
    else if (bytes >= 8)
        go(std::integral_constant<int, 8>{}, std::false_type{});
    else if (bytes >= 4)
        go(std::integral_constant<int, 4>{}, std::false_type{});
    else
        go(std::integral_constant<int, sizeof(T)>{}, std::false_type{});
}

// rows of a workgroup: about `pieces` pieces
static uint32_t rows_of(uint32_t per, uint32_t pieces) { return per >= pieces ? 1 : pieces / per; }

// a.block and so many workgroups of each launch: a grid has fewer than 2^32 threads
template <typename F>
static void in_launches(RowsArgs &a, int64_t groups, F &&launch)
{
    const int64_t most = 1 << 23;
    for (a.block = 0; a.block < groups; a.block += most) launch(dim3((unsigned)(groups - a.block < most ? groups - a.block : most)));
}

template <typename T>
static int gather(const RowsArgs &args, const T *x, T *y, hipStream_t st)
{
    RowsArgs a = args;
    auto go = [&](auto BYTES, auto WHOLE) {
        constexpr int V = decltype(BYTES)::value;
        constexpr bool W = decltype(WHOLE)::value;
        a.per = (a.d + Piece<T, V, W>::N - 1) / Piece<T, V, W>::N;
        a.rows = rows_of(a.per, ROW_NT * ROW_ITEMS);
        in_launches(a, (a.n * a.w + a.rows - 1) / a.rows, [&](dim3 groups) {
            hipLaunchKernelGGL((k_gather_rows<T, V, W>), groups, dim3(ROW_NT), 0, st, a, x, y);
        });
    };
    by_pieces<T>(a.d, x, y, nullptr, go);
    return (int)hipGetLastError();
}

template <typename T>
static int combine(const RowsArgs &args, const T *y, T *out, hipStream_t st)
{
    RowsArgs a = args;
    auto go = [&](auto BYTES, auto WHOLE) {
        constexpr int V = decltype(BYTES)::value;
        constexpr bool W = decltype(WHOLE)::value;
        a.per = (a.d + Piece<T, V, W>::N - 1) / Piece<T, V, W>::N;
        a.rows = rows_of(a.per, ROW_NT);
        const auto kern = a.w > 8 ? k_combine_rows<T, V, W, 16> : k_combine_rows<T, V, W, 8>;
        in_launches(a, (a.n + a.rows - 1) / a.rows, [&](dim3 groups) { hipLaunchKernelGGL(kern, groups, dim3(ROW_NT), 0, st, a, y, out); });
    };
    by_pieces<T>(a.d, y, out, nullptr, go);
    return (int)hipGetLastError();
}

template <typename T>
static int combine_back(const RowsArgs &args, const T *dout, const T *y, T *dy, float *dweight, hipStream_t st)
{
    RowsArgs a = args;
    auto go = [&](auto BYTES, auto WHOLE) {
        constexpr int V = decltype(BYTES)::value;
        constexpr bool W = decltype(WHOLE)::value;
        a.per = (a.d + Piece<T, V, W>::N - 1) / Piece<T, V, W>::N;
        auto lanes = [&](auto L) {
            constexpr int N = decltype(L)::value, R = ROW_NT / N;
            in_launches(a, (a.n * ((a.w + 7) / 8) + R - 1) / R, [&](dim3 groups) {
                hipLaunchKernelGGL((k_combine_back<T, V, W, N>), groups, dim3(ROW_NT), 0, st, a, dout, y, dy, dweight);
            });
        };
        if (a.per > 32)
            lanes(std::integral_constant<int, 64>{});
        else if (a.per > 16)
            lanes(std::integral_constant<int, 32>{});
        else
            lanes(std::integral_constant<int, 16>{});
    };
    by_pieces<T>(a.d, dout, y, dy, go);
    return (int)hipGetLastError();
}

int launch_gather_rows(int dtype, const void *x, int64_t n, int w, int d, const int32_t *source, void *y, hipStream_t st)
{
    const RowsArgs a = {n, w, d, 0, 0, 0, source, nullptr};
    if (dtype == VLQ_F32) return gather(a, (const float *)x, (float *)y, st);
    return gather(a, (const uint16_t *)x, (uint16_t *)y, st); // (values are moved, not looked at)
}

int launch_combine_rows(int dtype, const void *y, int64_t n, int w, int d, const int32_t *place, const float *weight, void *out,
                        hipStream_t st)
{
    const RowsArgs a = {n, w, d, 0, 0, 0, place, weight};
    switch (dtype) {
    case VLQ_F32: return combine(a, (const float *)y, (float *)out, st);
    case VLQ_F16: return combine(a, (const _Float16 *)y, (_Float16 *)out, st);
    default: return combine(a, (const bf16_t *)y, (bf16_t *)out, st);
    }
}

int launch_combine_rows_backward(int dtype, const void *dout, const void *y, int64_t n, int w, int d, const int32_t *place,
                                 const float *weight, void *dy, float *dweight, hipStream_t st)
{
    const RowsArgs a = {n, w, d, 0, 0, 0, place, weight};
    switch (dtype) {
    case VLQ_F32: return combine_back(a, (const float *)dout, (const float *)y, (float *)dy, dweight, st);
    case VLQ_F16: return combine_back(a, (const _Float16 *)dout, (const _Float16 *)y, (_Float16 *)dy, dweight, st);
    default: return combine_back(a, (const bf16_t *)dout, (const bf16_t *)y, (bf16_t *)dy, dweight, st);
    }
}
