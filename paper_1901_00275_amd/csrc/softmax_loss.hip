// Softmax cross entropy of n rows against the k centroids (or the k rows of an output layer), the n x k logits not kept,
// and its gradient:
//
//   l_ij = s <x_i, c_j> + b_j,  loss_i = log sum_j exp l_ij - l_iy,  G_ij = g_i (p_ij - [j = y_i]),  p_ij = exp(l_ij) / sum
//   dx_i = s sum_j G_ij c_j,  dc_j = s sum_i G_ij x_i,  db_j = sum_i G_ij.
//
// Four products of n x k x d: the logits forward, and backward the logits again (instead of n k probabilities kept between the
// calls) and the two gradients.
// Three forms, by rules on the sizes (loss_is_few, grads_are_few, narrow_dim):
//  - few (softmax_loss_few.hip): little is done with each centroid, everything is read as it lies;
//  - narrow (softmax_loss_narrow.hip): up to 128 dimensions (256 of 16-bit values), the probabilities never leave the registers;
//  - wide (here): tiles of 256 x 256 on the fp16 matrix cores, the probabilities written a piece at a time.  16-bit centroids are taken
//    as they lie up to LIE_ROWS rows (as_they_lie), the rows' image then holds the rows' own bits.
// This file has the images of both latter forms, the merging of statistics, the sums over parts, and all calls.
//
// Operands are otherwise rewritten as fp16 with a power-of-two scale (per row of x, per 16 rows of c, one per
// matrix where the rows are the summed index):
//  - fp16 values are taken as they are, bf16 values lose nothing down to 2^-31 of the largest of their scale (that is brought to
//    [2^14, 2^15), fp16's smallest step is 2^-24);
//  - an fp32 value is the sum of two fp16 values, hi + lo, with an error of 2^-23 of itself or 2^-39 of the largest of its scale (scales end
//    at 2^126: where the largest is below 2^-112 that is 2^-151, less than half of fp32's smallest step);
//    a product of two is hi hi + hi lo + lo hi, off by 2^-21 of |a||b| at most: three products where a split in three bf16 parts
//    takes six.
// All sums are fp32 (the accumulators of the matrix cores), maxima and sums of the softmax are fp32.
//
// Image of a matrix: blocks of 128 rows x units of 32 indices; an 8 KB page per (block, unit, part) holds 8 groups of 16 rows,
// of each the 64 chunks of 8 values in the order of the lanes that read them (chunk c of row r at 16 c + r % 16), so that a page
// is copied to LDS as it lies there and read without bank conflicts.
//
// Backward, a piece of the centroids at a time (at most PIECE values): P = 2^15 (p - [j = y]) is written as fp16 images of two parts
// in both orders, for the sums over j and over i.  The lanes of the product hold four consecutive j of one i, and four i (16 apart) of one
// j: the image summed over i has its indices in that order, so neither needs an exchange between lanes.
#include "loss_image.h"

#include <math.h>

#define LNT 512              // threads of the product kernels
#define LOSS_ROWS 8192       // rows that go through the products together
#define PIECE (1 << 26)      // values of P kept at a time
// Up to so many dimensions the narrow form, of two parts and of 16-bit values: what a workgroup keeps fits the registers.  us of a
// step against the wide form: 8 192 x 32 000 x 129 bf16 567 : 1 542, x 192 fp16 675 : 1 473, x 256 bf16 816 : 1 564; 1 000 x 20 000 x 160
// bf16 92 : 177, 300 x 32 000 x 256 bf16 109 : 165; forward 8 192 x 32 000 x 256 bf16 141 : 205, 2 735 x 2 322 x 190 19 : 22.
#define NARROW_DIM 128
#define NARROW_DIM_16 256
#define NARROW_GROUPS 1024   // its workgroups that run at a time: four a compute unit forward, half as many backward
#define NARROW_LEAST 4       // tiles of 32 rows that a workgroup of it takes at least (forward half as many)
// Where little is done with each centroid, rows and centroids are taken as they lie (softmax_loss_few.hip): rewriting them first,
// and tiles that leave most of the chip idle, cost more.  Measured in us, these against the others.
// Forward: 1 000 x 1 000 x 1 000 bf16 20 : 38, 8 000 x 120 x 500 fp32 27 : 54, 8 000 x 120 x 1 000 bf16 25 : 45, 535 x 975 x 1 248
// fp32 45 : 85, 128 x 65 536 x 64 fp16 17 : 31; the narrow form holds out longer: 1 000 x 5 000 x 96 fp32 39 : 19,
// 2 000 x 5 000 x 96 bf16 26 : 20, 70 x 65 536 x 96 fp32 29 : 41, 500 x 3 000 x 160 bf16 12 : 14, 1 000 x 2 000 x 192 16 : 15, 2 000 x 1 500 x 256
// 24 : 16, 80 x 40 000 x 160 21 : 26.
#define FEW_ROWS 64
#define FEW_WORK 1e9          // products
#define FEW_NARROW_ROWS 128   // against the narrow form
#define FEW_NARROW_WORK 1.2e8
#define FEW_NARROW_WORK_16 3e8 // beyond NARROW_DIM dimensions
// A step with the gradients (their products are fp32's, an eighth of the others' rate, but with few rows or centroids the others' tiles
// are mostly empty): 5 366 x 24 x 2 016 fp16 56 : 129, 3 x 30 x 224 fp16 22 : 29, 500 x 500 x 500 fp32 31 : 103, bf16 24 : 65,
// 8 000 x 32 x 2 000 fp32 134 : 282, 32 x 16 000 x 2 000 bf16 138 : 211, 8 000 x 64 x 4 000 bf16 274 : 362, 64 x 65 536 x 1 024 bf16
// 406 : 368, 1 000 x 1 000 x 300 bf16 52 : 70, 300 x 800 x 1 200 bf16 44 : 86, 1 000 x 2 000 x 300 bf16 87 : 77, 300 x 3 000 x 300 fp32 72 : 97,
// 1 000 x 2 000 x 200 fp32 104 : 88.  Narrow: 300 x 300 x 128 bf16 22 : 26, 5 000 x 200 x 64 38 : 34, 300 x 3 000 x 96 29 : 34, 1 000 x 1 000 x 128
// 37 : 33, 1 000 x 1 000 x 96 fp32 45 : 43, 100 x 16 384 x 128 fp32 78 : 60; 600 x 300 x 256 bf16 26 : 35, 1 000 x 500 x 160 30 : 31, 500 x 1 500 x 192
// 36 : 35, 300 x 4 000 x 160 43 : 36, 300 x 3 000 x 250 46 : 53, 500 x 2 500 x 200 50 : 41, 4 000 x 400 x 200 58 : 44.
#define FEW_GRAD_ROWS 64         // rows or centroids at most
#define FEW_GRAD_THIN_WORK 2.5e9 // with so few
#define FEW_GRAD_WORK 3e8      // with more
#define FEW_GRAD_NARROW_WORK 5e7
#define FEW_GRAD_NARROW_WORK_16 1.5e8
#define FEW_PAIRS (1 << 24)   // values of G, in fp32
// Up to so many inverse scales every workgroup that needs their largest finds it: a step of 256 x 16 384 x 96 fp32 57.0 -> 55.5 us, of
// 4 095 x 16 384 x 96 fp16 215 -> 212; 4 095 x 65 536 x 128 fp32 870 either way.
#define SMALL_SCALES 8192
#define MERGE_ROWS 2048      // up to so many rows four a workgroup are merged, not sixteen

// ---------------------------------------------------------------------------
// images
// ---------------------------------------------------------------------------
// A row counts if its label is a centroid; a centroid if its bias is not -inf.  What does not count is written as zeros.
__device__ __forceinline__ bool row_counts(const int32_t *label, int k, const float *bias, int64_t r)
{
    if (label) return (uint32_t)label[r] < (uint32_t)k;
    return !bias || bias[r] != -INFINITY;
}

// Image of the rows of X, 16 rows a workgroup; a scale per row (OWN) or for all 16.  inv: 1 / scale, as many.
// A wave takes every fourth unit, as the lanes lie in its pages; up to 4 HELD units the values wait in registers for their
// scale, beyond that they are read again.  Bound by memory.  (128 MB with 128 rows a workgroup and a scale for all of them:
// 99 us, for want of loads under way; 238 MB of rows of 64 units read twice 138 us, what a die's workgroups hold is more
// than its L2.)
// RAW: the image of the values' own bits (the scale is found all the same); pages NULL: only the scale.
template <typename T, bool OWN, int NP, int HELD, bool RAW>
__device__ __forceinline__ void pack_rows(int block, const T *__restrict__ X, int64_t rows, int d, int units,
                                          const int32_t *__restrict__ label, int k, const float *__restrict__ bias,
                                          u32x4 *__restrict__ pages, float *__restrict__ inv, bool vec)
{
    __shared__ float rmax[4][16];
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, wave = tid >> 6;
    const int64_t r0 = (int64_t)block * 16;
    const bool in = r0 + l < rows;
    const T *row = X + (in ? r0 + l : 0) * d; // (rows past the end: the first, not used)
    Eight<T> v[HELD];
    auto load = [&](int u0) {
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            const int u = u0 + 4 * q + wave;
            if (u < units) v[q] = load8(row, u * 32 + (lane >> 4) * 8, d, vec);
        }
    };
    load(0);
    const bool counts = in && row_counts(label, k, bias, r0 + l);
    int ex = 0;
    if constexpr (!__is_same(T, _Float16)) {
        float mx = 0.f;
        for (int u0 = 0; u0 < units; u0 += 4 * HELD) {
            if (u0 > 0) load(u0);
#pragma unroll
            for (int q = 0; q < HELD; ++q)
                if (u0 + 4 * q + wave < units)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float m = fabsf((float)v[q].v[e]);
                        if (m < INFINITY) mx = fmaxf(mx, m);
                    }
        }
        if (!counts) mx = 0.f;
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (lane < 16) rmax[wave][l] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(rmax[0][l], rmax[1][l]), fmaxf(rmax[2][l], rmax[3][l])); // of the lane's row
        if (!OWN)
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        ex = scale_exponent(mx);
    }
    if (tid < 16) {
        if (OWN)
            inv[r0 + tid] = pow2i(-ex);
        else if (tid == 0)
            inv[block] = pow2i(-ex);
    }
    if (!pages) return;
    const float s = pow2i(ex);
    u32x4 *to = pages + (int64_t)(block >> 3) * units * NP * PAGE + (block & 7) * 64 + lane;
    for (int u0 = 0; u0 < units; u0 += 4 * HELD) {
        if (units > 4 * HELD && (u0 > 0 || !__is_same(T, _Float16))) load(u0);
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            const int u = u0 + 4 * q + wave;
            if (u >= units) continue;
            if constexpr (RAW) {
                to[(int64_t)u * PAGE] = counts ? *(const u32x4 *)v[q].v : u32x4{0, 0, 0, 0};
            } else {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = counts ? (float)v[q].v[e] * s : 0.f;
                half8 h[NP];
                split8<NP>(f, h);
#pragma unroll
                for (int p = 0; p < NP; ++p) to[(int64_t)(u * NP + p) * PAGE] = __builtin_bit_cast(u32x4, h[p]);
            }
        }
    }
}

// Image of X's columns: its rows are the dimensions, its indices the rows of X, 64 rows x 128 dimensions a workgroup, turned in LDS.
// ORDER 1: index s of 64 is row (s >> 2) + 16 (s & 3), the order in which the lanes of k_loss_p hold them; 2: index s of 32 is row
// 16 (s / 4 % 2) + 4 (s / 8) + s % 4, as the lanes of k_loss_narrow hold them.
template <typename T, int ORDER, int NP>
__device__ __forceinline__ void pack_cols(int block, int dblock, const T *__restrict__ X, int64_t rows, int d, int units,
                                          const int32_t *__restrict__ label, int k, const float *__restrict__ bias,
                                          u32x4 *__restrict__ pages, float inv, bool vec)
{
    // (an odd number of words a row: neither the rows' writes nor the columns' reads meet in a bank more than they must)
    using Held = std::conditional_t<NP == 2, float, _Float16>;
    constexpr int LD = NP == 2 ? 129 : 130;
    __shared__ __align__(16) Held t[64 * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r0 = (int64_t)block * 64;
    const int d0 = dblock * 128;
    const float s = 1.f / inv; // (a power of two)
    Eight<T> v[4];
    bool counts[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = q * 16 + (tid >> 4);
        const bool in = r0 + r < rows;
        v[q] = load8(X + (in ? r0 + r : 0) * d, d0 + (tid & 15) * 8, d, vec);
        counts[q] = in && row_counts(label, k, bias, r0 + r);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        Held *to = t + (q * 16 + (tid >> 4)) * LD + (tid & 15) * 8;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = counts[q] ? (float)v[q].v[e] * s : 0.f;
        if constexpr (NP == 2) {
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = f[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const _Float16 two[2] = {(_Float16)f[e], (_Float16)f[e + 1]};
                *(uint32_t *)(to + e) = *(const uint32_t *)two;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int e = it & 1, grp = (it >> 1) + 2 * wave; // (a wave: two groups of 16 dimensions, both units)
        Held f[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int i = e * 32 + (lane >> 4) * 8 + q;
            const int r = ORDER == 1 ? (i >> 2) + 16 * (i & 3) : ORDER == 2 ? e * 32 + 16 * (q >> 2) + 4 * (lane >> 4) + (q & 3) : i;
            f[q] = t[r * LD + grp * 16 + (lane & 15)];
        }
        const int64_t u = (int64_t)block * 2 + e;
        u32x4 *to = pages + ((int64_t)dblock * units + u) * NP * PAGE + grp * 64 + lane;
        if constexpr (NP == 2) {
            half8 h[2];
            split8<2>(f, h);
            to[0] = __builtin_bit_cast(u32x4, h[0]);
            to[PAGE] = __builtin_bit_cast(u32x4, h[1]);
        } else {
            to[0] = *(const u32x4 *)f;
        }
    }
}

struct PackArgs {
    const void *x, *c;
    int64_t n;
    int d, k, units;
    const int32_t *label;
    const float *bias, *g, *stats;
    float scale;
    u32x4 *ximg, *cimg, *xcols, *ccols;
    float *rinv, *cinv, *gn, *bias2;
    f32x4 *row;
    int32_t *lab;
    LossHeader *hdr;
    bool vec, raw, halves;
    bool small;          // no launch for the header
    int64_t rinvs, cinvs; // inverse scales
    int xblocks, cblocks, dblocks, xunits, cunits; // workgroups for x, for c; units of the columns' images
};

// A row's numbers: factor s log2(e) / scale, and backward its maximum, the factors of P in either order (2^15 / z, and with
// g / max g); a row that does not count, or has no logit above -inf, gets the maximum +inf and no label.
__device__ __forceinline__ void row_numbers(const PackArgs &a, int64_t i, float inv, float top)
{
    const bool in = i < a.n && (uint32_t)a.label[i] < (uint32_t)a.k;
    f32x4 r = {in ? a.scale * LOG2E * (a.raw ? 1.f : inv) : 0.f, INFINITY, 0.f, 0.f};
    float f = 0.f;
    bool ok = in;
    if (a.stats && in) {
        const float m = a.stats[2 * i], z = a.stats[2 * i + 1];
        ok = m != -INFINITY;
        if (ok) {
            f = top > 0.f ? a.g[i] / top : a.g[i]; // (zero, or no finite one is there)
            r[1] = m;
            r[2] = P_ONE / z;
            r[3] = P_ONE / z * f;
        } else {
            r[0] = 0.f;
        }
    }
    a.row[i] = r;
    a.lab[i] = ok ? a.label[i] : -1;
    if (a.gn) a.gn[i] = ok ? f * P_ONE : 0.f;
}

// Both matrices' images in one launch; forward the rows' numbers.  RAW: x's image of its own bits, of c only what is asked for
// (cimg NULL, cinv: its scales).
template <typename T, int NP, int HELD, bool RAW>
__global__ __launch_bounds__(256) void k_pack_rows(PackArgs a)
{
    const int b = blockIdx.x - a.xblocks;
    if (b >= 0) {
        const int j = b * 16 + threadIdx.x; // the bias in units of log 2, -inf past the last centroid
        if (threadIdx.x < 16) a.bias2[j] = j < a.k ? (a.bias ? bias_log2(a.bias[j]) : 0.f) : -INFINITY;
        if (a.cinv) pack_rows<T, false, NP, HELD, RAW>(b, (const T *)a.c, a.k, a.d, a.units, nullptr, a.k, a.bias, a.cimg, a.cinv, a.vec);
        return;
    }
    pack_rows<T, true, NP, HELD, RAW>(blockIdx.x, (const T *)a.x, a.n, a.d, a.units, a.label, a.k, nullptr, a.ximg, a.rinv, a.vec);
    if (a.stats) return;
    __syncthreads();
    if (threadIdx.x < 16) row_numbers(a, (int64_t)blockIdx.x * 16 + threadIdx.x, a.rinv[(int64_t)blockIdx.x * 16 + threadIdx.x], 0.f);
}

// Backward: the largest inverse scale of x's rows (0), of c's (1), the largest |g| (2), in every thread
template <int NT>
__device__ __forceinline__ float header_value(const PackArgs &a, int which)
{
    __shared__ float s[NT / 64];
    float mx = 0.f;
    if (which == 2) {
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < a.n; i += NT) {
            const float v = fabsf(a.g[i]);
            if ((uint32_t)a.label[i] < (uint32_t)a.k && v < INFINITY) mx = fmaxf(mx, v);
        }
    } else {
        if (a.halves) return 1.f; // (fp16 values are not scaled)
        const float *v = which == 0 ? a.rinv : a.cinv;
        const int64_t count = !v ? 0 : which == 0 ? a.rinvs : a.cinvs;
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < count; i += NT) mx = fmaxf(mx, v[i]);
    }
    mx = __uint_as_float(wave_max_u32(__float_as_uint(mx)));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = mx;
    __syncthreads();
    mx = s[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) mx = fmaxf(mx, s[w]);
    __syncthreads();
    return mx;
}
__device__ __forceinline__ void header_write(const PackArgs &a, int which, float v)
{
    if (threadIdx.x == 0) (which == 0 ? a.hdr->xinv : which == 1 ? a.hdr->cinv : a.hdr->top) = v;
}

// The header by a launch of its own, a workgroup each.  (An atomic of every workgroup of k_pack_rows on one address took 43 us at
// 65 536 centroids.)
__global__ __launch_bounds__(1024) void k_loss_header(PackArgs a) { header_write(a, blockIdx.x, header_value<1024>(a, blockIdx.x)); }

// Backward: both matrices' columns, and the rows' numbers.  a.small: every workgroup finds what it needs of the header by itself,
// the last one writes it.
template <typename T, int XORDER, int CORDER, int NP>
__global__ __launch_bounds__(256) void k_pack_cols(PackArgs a)
{
    int b = blockIdx.x;
    if (b < a.xblocks) {
        const float inv = a.small ? header_value<256>(a, 0) : a.hdr->xinv;
        pack_cols<T, XORDER, NP>(b / a.dblocks, b % a.dblocks, (const T *)a.x, a.n, a.d, a.xunits, a.label, a.k, nullptr, a.xcols, inv, a.vec);
        return;
    }
    b -= a.xblocks;
    if (b < a.cblocks) {
        const float inv = a.small ? header_value<256>(a, 1) : a.hdr->cinv;
        pack_cols<T, CORDER, NP>(b / a.dblocks, b % a.dblocks, (const T *)a.c, a.k, a.d, a.cunits, nullptr, a.k, a.bias, a.ccols, inv, a.vec);
        return;
    }
    const int64_t i = (int64_t)(b - a.cblocks) * 256 + threadIdx.x; // (the workgroups cover the padded rows)
    const float top = a.small ? header_value<256>(a, 2) : a.hdr->top;
    row_numbers(a, i, a.rinv[i], top);
    if (a.small && blockIdx.x == gridDim.x - 1) {
        header_write(a, 2, top);
        header_write(a, 1, header_value<256>(a, 1));
        header_write(a, 0, header_value<256>(a, 0));
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
// One operand of a product: its image, pages from a block to the next, first page of the sum
struct Operand {
    const u32x4 *pages;
    int64_t block; // pages per block of 128 rows
    int64_t first;
};

// acc = A B^T over `units` units of 32 indices, of A in NPA parts and B in NPB: as many pages of every block each.
// A tile of two blocks of A by two of B; eight waves, 2 x 4, of 128 rows of A x 64 of B each.  A lane's acc[i][j][r] is row
// 16 i + 4 (lane / 16) + r, column 16 j + lane % 16 of its wave's part.
//
// A goes through LDS (a ring of four units, asked for three ahead, there one ahead), the fragments of B straight to registers:
// through LDS as well its 128 bytes a clock were the bound.  Between two barriers a wave has one unit; its memory
// operations are spread between the products of its fragments, and the first fragments of A are read a unit ahead, so that the products go on
// behind the barrier at once.  8 192 x 8 192 x 2 048, one part, on random operands: 1.46 PFLOP/s, x 8 192: 1.51 (both operands
// through LDS, copies asked for together: 1.10 and 1.42; products from registers alone: 1.75 and 1.92).
template <int NPA, int NPB>
struct Product {
    static constexpr int RING = 4, AHEAD = 3, PAGES = 2 * NPA; // pages of A of a unit
    static constexpr int BAHEAD = NPB == 1 ? 3 : 1, NB = BAHEAD + 1; // units that B's fragments are asked for ahead (a unit of two parts takes two or three times as long)
    static constexpr int ROUND = 4 * NPB + PAGES;             // memory operations of a wave and unit
    static constexpr int LDS = RING * PAGES * PAGE * 16;
    static_assert(RING > AHEAD, "a unit takes the place of the one before the present");

    static __device__ __forceinline__ void run(const Operand &A, const Operand &B, int64_t ablk, int64_t bblk, int units, u32x4 *lds,
                                               f32x4 (&acc)[8][4])
    {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const u32x4 *a0 = A.pages + (ablk * A.block + A.first) * PAGE;
        const u32x4 *b0 = B.pages + ((bblk + ((wave >> 1) & 1)) * B.block + B.first) * PAGE + (wave & 1) * 4 * 64 + lane;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // page q of unit t (behind the last: of the last, not used); the place in LDS is that of t all the same
        auto copy_page = [&](int t, int q) {
            u32x4 *dst = lds + ((t & (RING - 1)) * PAGES + q) * PAGE + wave * 64;
            const u32x4 *src = a0 + ((q / NPA) * A.block + (int64_t)min(t, units - 1) * NPA + q % NPA) * PAGE;
            const __amdgpu_buffer_rsrc_t page = __builtin_amdgcn_make_buffer_rsrc((void *)src, 0, PAGE * 16, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(page, (__attribute__((address_space(3))) void *)dst, 16, tid * 16, 0, 0, 0);
        };
        half8 a[8][NPA];
        u32x4 b[NB][NPB][4];
        auto read_a = [&](int t, int i) {
#pragma unroll
            for (int p = 0; p < NPA; ++p)
                a[i][p] = __builtin_bit_cast(half8, lds[((t & (RING - 1)) * PAGES + (wave >> 2) * NPA + p) * PAGE + i * 64 + lane]);
        };
        auto load_b = [&](int t, int slot, int q) { b[slot][q / 4][q % 4] = b0[((int64_t)min(t, units - 1) * NPB + q / 4) * PAGE + q % 4 * 64]; };
        // a wave's memory operations come in rounds, round t: B of unit t + BAHEAD, then A of unit t + AHEAD
#pragma unroll
        for (int t = -AHEAD; t < 0; ++t) {
            if (t + BAHEAD >= 0)
#pragma unroll
                for (int q = 0; q < 4 * NPB; ++q) load_b(t + BAHEAD, t + BAHEAD, q);
            asm volatile("" ::: "memory");
#pragma unroll
            for (int q = 0; q < PAGES; ++q) copy_page(t + AHEAD, q);
            asm volatile("" ::: "memory");
        }
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BAHEAD == 3 ? 2 * ROUND : PAGES + ROUND)) : "memory");
        read_a(0, 0);
        read_a(0, 1);
        auto unit = [&](int t, auto SLOT) {
            constexpr int slot = decltype(SLOT)::value;
            // A of unit t + 1 has arrived: it came with round t - 2; everyone is done with unit t - 1
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(ROUND) : "memory");
            read_a(t, 2);
            read_a(t, 3);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (NPB == 2)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][0], __builtin_bit_cast(half8, b[slot][NPB - 1][j]), acc[i][j], 0, 0, 0);
                if (NPA == 2)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][NPA - 1], __builtin_bit_cast(half8, b[slot][0][j]), acc[i][j], 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][0], __builtin_bit_cast(half8, b[slot][0][j]), acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 4)
#pragma unroll
                    for (int q = 0; q < NPB; ++q) load_b(t + BAHEAD, (slot + BAHEAD) % NB, i * NPB + q);
                else if (i - 4 < PAGES)
                    copy_page(t + AHEAD, i - 4);
                if (i < 4) read_a(t, i + 4);
                if (i == 4) read_a(t + 1, 0);
                if (i == 5) read_a(t + 1, 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        for (int t = 0; t < units; t += NB) {
#define LOSS_UNIT(s) \
    if (s < NB && (s == 0 || t + s < units)) unit(t + s, std::integral_constant<int, s % NB>{})
            LOSS_UNIT(0);
            LOSS_UNIT(1);
            LOSS_UNIT(2);
            LOSS_UNIT(3);
#undef LOSS_UNIT
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // (what was asked for behind the last unit)
    }
};

// The same where the rows of A are taken as they lie (16-bit values, rows on 16 bytes): the logits of an output layer, whose
// k x d values are not rewritten first.  A step is two units, 128 bytes of a row, so that whole lines are read; of 256 rows x
// eight chunks in LDS chunk c of row r lies at place c ^ (r % 8), so that the 16 rows of a fragment are read without bank
// conflicts.  B is an image of the values' own bits.
__device__ __forceinline__ f32x4 multiply16(_Float16, const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply16(bf16_t, const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// (B as it lies as well cost more than its image: 1 000 x 16 384 x 512 fp16 33 us instead of 22 and 5 for the image.)
template <typename T>
struct ProductRows {
    static constexpr int RING = 4, AHEAD = 3, STEP = TILE * 8; // chunks of a step
    static constexpr int ROUND = 12;                           // memory operations of a wave and step
    static constexpr int LDS = RING * STEP * 16;

    // c: the tile's first row, `rows` of them are there
    static __device__ __forceinline__ void run(const T *c, int rows, int d, const Operand &B, int64_t bblk, int units, u32x4 *lds,
                                               f32x4 (&acc)[8][4])
    {
        const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const u32x4 *b0 = B.pages + ((bblk + ((wave >> 1) & 1)) * B.block + B.first) * PAGE + (wave & 1) * 4 * 64 + lane;
        const int steps = units / 2; // (units are even)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // a wave copies 32 rows, eight at a time; rows past the end are the last one, not looked at
        const int chunk = (lane & 7) ^ (lane >> 3);
        int off[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) off[q] = min(wave * 32 + 8 * q + (lane >> 3), rows - 1) * d * 2 + chunk * 16;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)c, 0, 1 << 30, 0x00020000);
        auto copy = [&](int t, int q) {
            u32x4 *dst = lds + (t & (RING - 1)) * STEP + (wave * 32 + 8 * q) * 8;
            t = min(t, steps - 1);
            int o = off[q];
            if ((t + 1) * 64 > d && t * 64 + chunk * 8 >= d) o = 1 << 30; // (behind the row's end: zeros)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)dst, 16, o, t * 128, 0, 0);
        };
        u32x4 a[8], b[2][2][4];
        const int at[2] = {((wave >> 2) * 128 + l) * 8 + (g ^ (l & 7)), ((wave >> 2) * 128 + l) * 8 + ((4 + g) ^ (l & 7))};
        auto read_a = [&](int t, int h, int i) { a[i] = lds[(t & (RING - 1)) * STEP + at[h] + i * 128]; };
        auto load_b = [&](int t, int slot, int h, int j) { b[slot][h][j] = b0[(int64_t)(2 * min(t, steps - 1) + h) * PAGE + j * 64]; };
        // a wave's memory operations come in rounds, round t: B of step t + 1, A of step t + AHEAD
#pragma unroll
        for (int t = -AHEAD; t < 0; ++t) {
            if (t == -1)
#pragma unroll
                for (int q = 0; q < 8; ++q) load_b(0, 0, q / 4, q % 4);
            asm volatile("" ::: "memory");
#pragma unroll
            for (int q = 0; q < 4; ++q) copy(t + AHEAD, q);
            asm volatile("" ::: "memory");
        }
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(4 + ROUND) : "memory");
        read_a(0, 0, 0);
        read_a(0, 0, 1);
        auto half = [&](int t, auto SLOT, auto HALF) {
            constexpr int slot = decltype(SLOT)::value, h = decltype(HALF)::value;
            // A of step t + 1 has arrived: it came with round t - 2; everyone is done with step t - 1
            if (h == 0) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(ROUND) : "memory");
            read_a(t, h, 2);
            read_a(t, h, 3);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = multiply16(T(), a[i], b[slot][h][j], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                if (i < 4)
                    load_b(t + 1, slot ^ 1, h, i);
                else if (i < 6)
                    copy(t + AHEAD, 2 * h + i - 4);
                if (i < 4) read_a(t, h, i + 4);
                if (i == 4 || i == 5) read_a(t + h, h ^ 1, i - 4);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        for (int t = 0; t < steps; t += 2) {
            half(t, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
            half(t, std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
            if (t + 1 < steps) {
                half(t + 1, std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{});
                half(t + 1, std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // (what was asked for behind the last step)
    }
};

// The tile of a workgroup: workgroups go to the eight dies in turn, so each die is given a run of neighbouring tiles, within
// which eight tiles of B by a few of A share their pages in the die's L2.
__device__ __forceinline__ void tile_of(int b, int mt, int nt, int *m, int *n)
{
    const int total = mt * nt, per = total >> 3, rest = total & 7, die = b & 7, at = b >> 3;
    const int id = die * per + min(die, rest) + at;
    const int band = id / (8 * mt), width = min(8, nt - band * 8), in = id - band * 8 * mt;
    *m = in / width;
    *n = band * 8 + in - *m * width;
}

struct LogitArgs {
    Operand A, B; // centroids, rows
    const float *cinv, *bias2;
    const f32x4 *row;
    const int32_t *lab;
    const void *c; // the piece's first centroid as it lies, and how many there are from there on
    int rows, d;
    int units, mt, nt;
    int npad;
    int m_first; // first centroid of the piece
    // forward
    float2 *part; // [mt * 2][npad] {maximum, sum} of 128 centroids
    float *mine;  // [npad] the label's logit
    // backward
    const float *gn;
    u32x2 *pj, *pi; // P's images, summed over j and over i
    int jblock, iblock; // pages per block of either
    float *dbpart;  // [npad / 64][mt * 256] or NULL
};

// The products of a tile from images of either matrix in PARTS parts, or with the centroids as they lie.  There a centroid that
// does not count is not zero, so its logits have to be told.
template <int PARTS>
struct FromImages {
    static constexpr int LDS = Product<PARTS, PARTS>::LDS;
    static constexpr bool TOLD = false;
    static __device__ __forceinline__ void run(const LogitArgs &a, int mt, int nt, u32x4 *lds, f32x4 (&acc)[8][4])
    {
        Product<PARTS, PARTS>::run(a.A, a.B, mt * 2, nt * 2, a.units, lds, acc);
    }
    static __device__ __forceinline__ float inverse(const LogitArgs &a, int group) { return a.cinv[group]; }
};
template <typename T>
struct FromRows {
    static constexpr int LDS = ProductRows<T>::LDS;
    static constexpr bool TOLD = true;
    static __device__ __forceinline__ void run(const LogitArgs &a, int mt, int nt, u32x4 *lds, f32x4 (&acc)[8][4])
    {
        ProductRows<T>::run((const T *)a.c + (int64_t)mt * TILE * a.d, max(1, a.rows - mt * TILE), a.d, a.B, nt * 2, a.units, lds, acc);
    }
    static __device__ __forceinline__ float inverse(const LogitArgs &, int) { return 1.f; }
};

// Forward: per row the maximum and the sum over the 128 centroids of a wave's part.  A lane holds 32 centroids of each of
// four rows, so most of the reduction stays in its registers.  Bound by the matrix cores: 8 192 x 50 001 x 2 048 bf16 1 240 us (1.35
// PFLOP/s, the library's product of this size 1.33); 1 000 x 16 384 x 512 fp16 22 us (0.76: one round of 256 tiles, whose
// start, sixteen units and end cannot hide behind each other).
template <class FORM>
__global__ __launch_bounds__(LNT, 2) void k_loss_stats(LogitArgs a)
{
    extern __shared__ u32x4 lds[];
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int mt, nt;
    tile_of(blockIdx.x, a.mt, a.nt, &mt, &nt);
    f32x4 acc[8][4];
    FORM::run(a, mt, nt, lds, acc);
    const int m0 = mt * TILE + (wave >> 2) * 128, n0 = nt * TILE + (wave & 3) * 64;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float ci = FORM::inverse(a, (m0 >> 4) + i);
        const f32x4 b2 = *(const f32x4 *)(a.bias2 + m0 + 16 * i + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float f = a.row[n0 + 16 * j + l][0] * ci;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                acc[i][j][r] = FORM::TOLD && b2[r] == -INFINITY ? -INFINITY : fmaf(acc[i][j][r], f, b2[r]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * j + l;
        float m = -INFINITY, z = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[i][j][r]);
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float m1 = m == -INFINITY ? 0.f : m; // (all masked: every term is zero)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) z += __builtin_amdgcn_exp2f(acc[i][j][r] - m1);
        z += __shfl_xor(z, 16, 64);
        z += __shfl_xor(z, 32, 64);
        if (g == 0) a.part[(int64_t)(mt * 2 + (wave >> 2)) * a.npad + n] = make_float2(m, z);
        const int rel = a.lab[n] - m0;
        if (__any((uint32_t)rel < 128u)) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (rel == 16 * i + 4 * g + r) a.mine[n] = acc[i][j][r];
        }
    }
}

// A row's statistics and loss from its parts: R rows a workgroup of 256, 256 / R threads each.  Rows lie side by side; where
// there are few of them a row has more threads.
template <int R>
__global__ __launch_bounds__(256) void k_loss_merge(const float2 *part, int parts, int npad, const float *mine, const int32_t *lab, int k,
                                                    const float *bias, int64_t n, float *stats, float *loss)
{
    constexpr int T = 256 / R;
    const int r = threadIdx.x % R, t = threadIdx.x / R;
    const int64_t i = (int64_t)blockIdx.x * R + r;
    const int64_t in = min(i, n - 1);
    const int label = lab[in];
    const float own = mine[in];
    float2 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = make_float2(-INFINITY, 0.f);
    for (int p = t; p < parts; p += 4 * T) { // (no branch around a load, it would wait for it)
        float2 w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = part[(int64_t)min(p + u * T, parts - 1) * npad + in];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = join(v[u], p + u * T < parts ? w[u] : make_float2(-INFINITY, 0.f));
    }
    v[0] = join(join(v[0], v[1]), join(v[2], v[3]));
#pragma unroll
    for (int o = R; o < 64; o *= 2) v[0] = join(v[0], make_float2(__shfl_xor(v[0].x, o, 64), __shfl_xor(v[0].y, o, 64)));
    __shared__ float2 s[4][R];
    if ((threadIdx.x & 63) < R) s[threadIdx.x >> 6][r] = v[0];
    __syncthreads();
    if (t != 0 || i >= n) return;
    v[0] = join(join(s[0][r], s[1][r]), join(s[2][r], s[3][r]));
    const float m = v[0].x, z = v[0].y;
    stats[2 * i] = m;
    stats[2 * i + 1] = z;
    if (!loss) return;
    float l = LN2 * (m - own) + logf(z);
    if ((uint32_t)label >= (uint32_t)k)
        l = 0.f;
    else if (m == -INFINITY)
        l = INFINITY;
    else if (own == -MOST && m > -MOST && bias) // (a bias that these units have no number for: nothing shows beside it)
        l = LN2 * m - bias[label];
    loss[i] = l;
}

// Backward: P of a tile, as images in both orders, and the sums over a wave's 64 rows for the bias.  The logits are rounded as they
// were forward, so that p adds up to one where a large bias takes up some of the products' bits, or all.
// 8 192 x 50 001 x 2 048 bf16 in seven pieces 1 750 us (0.96 PFLOP/s): the product, and behind it 3.3 GB of images.
template <class FORM>
__global__ __launch_bounds__(LNT, 2) void k_loss_p(LogitArgs a)
{
    extern __shared__ u32x4 lds[];
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int mt, nt;
    tile_of(blockIdx.x, a.mt, a.nt, &mt, &nt);
    f32x4 acc[8][4];
    FORM::run(a, mt, nt, lds, acc);
    const int m0 = mt * TILE + (wave >> 2) * 128, n0 = nt * TILE + (wave & 3) * 64; // (within the piece)
    f32x4 row[4];
    int rel[4];
    float gn[4];
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * j + l;
        row[j] = a.row[n];
        rel[j] = a.lab[n] - a.m_first - m0 - 4 * g; // (16 i + r where the lane holds the label)
        if (a.lab[n] < 0) rel[j] = -1;
        gn[j] = a.gn[n];
        any |= (uint32_t)rel[j] < 128u && (rel[j] & 12) == 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float ci = FORM::inverse(a, (m0 >> 4) + i);
        const f32x4 b2 = *(const f32x4 *)(a.bias2 + m0 + 16 * i + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float f = row[j][0] * ci;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                acc[i][j][r] = FORM::TOLD && b2[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], f, b2[r]) - row[j][1]);
        }
    }
    const bool labels = __any(any);
    // image summed over j: the rows of its blocks are the rows i, the lane's four r are half a chunk
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * j + l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f32x4 v = acc[i][j] * row[j][2];
            if (labels)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (rel[j] == 16 * i + r) v[r] -= P_ONE;
            const int jj = m0 + 16 * i; // index of the sum, from the piece's first
            u32x2 *to = a.pj + (((int64_t)(n >> 7) * a.jblock + (jj >> 5) * P_PARTS) * PAGE + ((n >> 4) & 7) * 64 +
                                16 * (2 * (i & 1) + (g >> 1)) + l) * 2 + (g & 1);
            half4 h, lo;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                _Float16 hi, rest;
                halves<P_PARTS>(v[r], hi, rest);
                h[r] = hi;
                lo[r] = rest;
            }
            to[0] = __builtin_bit_cast(u32x2, h);
            to[PAGE * 2] = __builtin_bit_cast(u32x2, lo);
        }
    }
    // image summed over i, weighted by g: the rows of its blocks are the centroids (row 4 r + g of 16 is centroid 4 g + r),
    // the lane's four rows j are half a chunk
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            half4 h, lo;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v = acc[i][j][r] * row[j][3];
                if (labels && rel[j] == 16 * i + r) v -= gn[j];
                sum += v;
                _Float16 hi, rest;
                halves<P_PARTS>(v, hi, rest);
                h[j] = hi;
                lo[j] = rest;
            }
            u32x2 *to = a.pi + (((int64_t)(m0 >> 7) * a.iblock + ((n0 >> 5) + (l >> 3)) * P_PARTS) * PAGE + i * 64 +
                                16 * ((l >> 1) & 3) + 4 * r + g) * 2 + (l & 1);
            to[0] = __builtin_bit_cast(u32x2, h);
            to[PAGE * 2] = __builtin_bit_cast(u32x2, lo);
            if (a.dbpart) {
                sum = row16_sum(sum);
                if (l == 0) a.dbpart[(int64_t)(n0 >> 6) * (a.mt * TILE) + m0 + 16 * i + 4 * g + r] = sum;
            }
        }
}

// One gradient: out[row][dim] = scale weight sum over the index of A[dim] B[row]
struct GradOut {
    Operand A, B; // columns' image (rows: dimensions), P's image
    int units, mt, nt, splits, per; // units of the sum, tiles, and parts that the sum is cut into, `per` units each
    int rows, d;
    bool permuted; // rows of B in the order 4 r + g
    int mode;      // 0: typed; 1: fp32 slabs without the scale and `top`, stored; 2: added to what is there
    void *out;     // typed [rows x d], or slabs [splits][rows x d]
    int64_t slab;
    const float *inv, *top; // inverse scale of the columns' image, largest |g|
    const float *gn;        // dx: a row's g relative to that, in units of P_ONE
    float scale;
    bool vec;
};

// Both gradients of a piece in one launch, the one with the longer sums first: the tiles of one alone (256 in a piece of 8 192 x 8 192
// at 2 048 dimensions) leave compute units waiting for the last.  8 192 x 50 001 x 2 048 bf16 4 850 us (1.38 PFLOP/s, two products
// for the parts of P); of a piece's 790 us about 27 are the sums of dx, which are read, added to and written again.  Smaller pieces
// repeat that more often (2^25 values of P: a step of 8 780 us against 8 320), larger ones gain little for twice the memory (2^27: 8 230).
template <typename T, int NP>
__global__ __launch_bounds__(LNT, 2) void k_loss_grads(GradOut first, GradOut second, int nfirst)
{
    extern __shared__ u32x4 lds[];
    const bool one = (int)blockIdx.x < nfirst;
    const GradOut &a = one ? first : second;
    const int b = one ? blockIdx.x : blockIdx.x - nfirst;
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles = a.mt * a.nt, split = b / tiles;
    int mt, nt;
    tile_of(b - split * tiles, a.mt, a.nt, &mt, &nt);
    Operand A = a.A, B = a.B;
    A.first += (int64_t)split * a.per * NP;
    B.first += (int64_t)split * a.per * P_PARTS;
    f32x4 acc[8][4];
    Product<NP, P_PARTS>::run(A, B, (int64_t)mt * 2, (int64_t)nt * 2, min(a.per, a.units - split * a.per), lds, acc);
    const int m0 = mt * TILE + (wave >> 2) * 128 + 4 * g, n0 = nt * TILE + (wave & 3) * 64 + (a.permuted ? 4 * (l & 3) + (l >> 2) : l);
    const float unit = grad_unit(*a.inv), top = *a.top;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * j;
        if (n >= a.rows) continue;
        const float w = a.gn ? a.gn[n] * (1.f / P_ONE) : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = m0 + 16 * i;
            if (m >= a.d) continue;
            const int64_t at = (int64_t)n * a.d + m;
            if (a.mode == 0) {
                store4((T *)a.out + at, acc[i][j] * unit * w * a.scale * top, a.d - m, a.vec);
            } else {
                float *p = (float *)a.out + split * a.slab + at;
                f32x4 v = acc[i][j] * unit * w;
                if (a.mode == 2) {
                    if (a.vec)
                        v += *(const f32x4 *)p;
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (m + e < a.d) v[e] += p[e];
                }
                store4(p, v, a.d - m, a.vec);
            }
        }
    }
}

// From so many parts on the four waves of a workgroup share those of 256 values (a step of 3 855 x 11 x 657 fp32, 46 parts of dc, 8 us less)
#define SUM_SHARED 8
struct SlabSum {
    const float *slabs;
    int splits;
    int64_t first, blocks; // workgroups of this launch
    int64_t count;
    const float *top; // what P's images are relative to, or NULL
    void *out;
};
// dbias of a piece: sums over the rows' parts, 64 centroids a workgroup, four waves taking the parts in turn
struct BiasSum {
    const float *part;
    int slots, ld, count, blocks;
    const float *top;
    bool add;
    float *out;
};
__device__ __forceinline__ void bias_sum(int block, const BiasSum &a)
{
    __shared__ float sum[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = block * 64 + lane;
    float s = 0.f;
    if (j < a.count)
#pragma unroll 4
        for (int p = wave; p < a.slots; p += 4) s += a.part[(int64_t)p * a.ld + j];
    sum[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || j >= a.count) return;
    s = (sum[0][lane] + sum[1][lane]) + (sum[2][lane] + sum[3][lane]);
    if (a.top) s = s * (1.f / P_ONE) * *a.top;
    a.out[j] = a.add ? a.out[j] + s : s;
}

// out = scale * sum of the slabs, of both gradients, four values a thread
template <typename T>
__global__ __launch_bounds__(256) void k_loss_sums(SlabSum x, SlabSum c, BiasSum bias, float scale)
{
    if (blockIdx.x >= x.blocks + c.blocks) {
        bias_sum((int)(blockIdx.x - x.blocks - c.blocks), bias);
        return;
    }
    const bool first = blockIdx.x < x.blocks;
    const SlabSum &a = first ? x : c;
    const bool share = a.splits >= SUM_SHARED;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t at = a.first + (first ? blockIdx.x : blockIdx.x - x.blocks), i = (share ? at * 64 + lane : at * 256 + threadIdx.x) * 4;
    const float top = a.top ? *a.top : 1.f;
    const bool vec = a.count % 4 == 0 && (uintptr_t)a.out % (4 * sizeof(T)) == 0;
    const int count = (int)min((int64_t)4, a.count - i), by = share ? 4 : 1;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (i >= a.count) {
        if (!share) return;
    } else if (vec) {
#pragma unroll 8
        for (int p = share ? wave : 0; p < a.splits; p += by) s += *(const f32x4 *)(a.slabs + p * a.count + i);
    } else {
#pragma unroll 4
        for (int p = share ? wave : 0; p < a.splits; p += by)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += a.slabs[p * a.count + min(i + e, a.count - 1)];
    }
    if (share) {
        __shared__ f32x4 sum[3][64];
        if (wave > 0) sum[wave - 1][lane] = s;
        __syncthreads();
        if (wave > 0 || i >= a.count) return;
        s = (s + sum[0][lane]) + (sum[1][lane] + sum[2][lane]);
    }
    store4((T *)a.out + i, s * scale * top, count, vec);
}

// No rows: the gradients of centroids and bias are zero
template <typename T>
__global__ __launch_bounds__(256) void k_loss_none(T *dc, int64_t count, float *dbias, int k)
{
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += step) {
        if (dc) dc[i] = (T)0.f;
        if (dbias && i < k) dbias[i] = 0.f;
    }
}

// ---------------------------------------------------------------------------
// calls
// ---------------------------------------------------------------------------
static int64_t pad_to(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Where a call's data lies in its workspace
struct LossPlan {
    int np;                  // fp16 parts of a value
    int64_t n, npad, kpad;
    int d, units, dblocks;   // units of 32 indices of a row's image, blocks of 128 dimensions
    int64_t rows, rpad;      // rows that go through the products together
    int64_t piece;           // centroids whose P is kept at a time
    int xsplit, csplit;      // parts that the sums of dx (over a piece) and dc (over `rows`) are cut into
    bool xslab, cslab;
    bool few;                // softmax_loss_few.hip
    float *G;
    int kp;
    bool narrow;             // softmax_loss_narrow.hip
    int xper, cper;          // its tiles of a part
    LossHeader *hdr;
    u32x4 *ximg, *cimg, *xcols, *ccols, *pj, *pi;
    float *rinv, *cinv, *bias2, *mine, *gn, *dbpart, *xsum, *csum;
    f32x4 *row;
    int32_t *lab;
    float2 *part;
    size_t bytes;
};

// Parts of a sum over `units` units, so that `tiles` of them fill the chip: each at least eight units long, and the slabs
// together no larger than 256 MB.
static int sum_parts(int64_t tiles, int64_t units, int64_t out_bytes)
{
    int64_t s = 256 / (tiles < 1 ? 1 : tiles);
    if (s > units / 8) s = units / 8;
    if (s * out_bytes > (256ll << 20)) s = (256ll << 20) / out_bytes;
    if (s <= 1) return 1;
    const int64_t per = (units + s - 1) / s;
    return (int)((units + per - 1) / per); // (no part is empty)
}

// The narrow form: parts of `per` tiles of 32, fewer where their slabs would take more than 256 MB
static int narrow_parts(int64_t tiles, int64_t per, int64_t out_bytes, int *tiles_each)
{
    int64_t s = (tiles + per - 1) / per;
    if (s * out_bytes > (256ll << 20)) s = (256ll << 20) / out_bytes;
    if (s < 1) s = 1;
    const int64_t each = (tiles + s - 1) / s;
    *tiles_each = (int)each;
    return (int)((tiles + each - 1) / each);
}

// Tiles of a workgroup, so that all of them fill the chip's `slots` a whole number of times (a half to three, whatever the sums over parts
// and the starts of more workgroups leave as the shortest): xq and cq workgroups side by side, xt and ct tiles to go through,
// x_bytes and c_bytes of a part's sums (0: none), us of a tile.  (Always two rounds, whatever was left for a
// third: with P in one part a step of 2 710 x 9 867 x 192 fp16 131 us, 107 so; 300 x 32 000 x 256 bf16 125 and 100, 8 192 x 32 000 x 256
// 703 and 648.  `us` of a tile 30 or 60 % larger: the same times.)
static int64_t narrow_per(int64_t xq, int64_t xt, int64_t cq, int64_t ct, int64_t slots, int64_t least, double x_bytes, double c_bytes, double us)
{
    int64_t best = least;
    double best_us = 1e30;
    for (int halves : {1, 2, 4, 6}) { // (half a round: a workgroup has a compute unit for itself, and takes 0.8 of the time)
        const int64_t most = slots * halves / 2;
        int64_t per = (xq * xt + cq * ct) / most;
        if (per < least) per = least;
        int64_t xs, cs;
        for (;; per += 1 + per / 16) {
            xs = (xt + per - 1) / per;
            cs = cq ? (ct + per - 1) / per : 0;
            if (xq * xs + cq * cs <= most || (xs == 1 && cs <= 1)) break;
        }
        const int64_t longest = xs == 1 && cs <= 1 ? (xt > ct ? xt : ct) : per, groups = xq * xs + cq * cs;
        const double sums = (xs > 1 ? xs * x_bytes : 0.) + (cs > 1 ? cs * c_bytes : 0.);
        const double turns = 2 * groups <= slots ? 0.8 : (double)((groups + slots - 1) / slots);
        const double t = turns * (longest + 2) * us + sums / 3.3e6; // (written and read, mostly in the last-level cache)
        if (t < best_us) {
            best_us = t;
            best = per;
        }
    }
    return best;
}

static int narrow_dim(int dtype) { return dtype == VLQ_F32 ? NARROW_DIM : NARROW_DIM_16; }

static bool loss_is_few(int dtype, int64_t n, int d, int k)
{
    const double work = (double)n * d * k;
    if (n <= FEW_ROWS) return true;
    if (d > narrow_dim(dtype)) return work <= FEW_WORK;
    return n <= FEW_NARROW_ROWS || work <= (d <= NARROW_DIM ? FEW_NARROW_WORK : FEW_NARROW_WORK_16);
}
static bool grads_are_few(int dtype, int64_t n, int d, int k)
{
    const double work = (double)n * d * k;
    if (n * pad_to(k, 32) > FEW_PAIRS) return false;
    if (d > narrow_dim(dtype)) return work <= (n <= FEW_GRAD_ROWS || k <= FEW_GRAD_ROWS ? FEW_GRAD_THIN_WORK : FEW_GRAD_WORK);
    return work <= (d <= NARROW_DIM ? FEW_GRAD_NARROW_WORK : FEW_GRAD_NARROW_WORK_16);
}

static LossPlan loss_plan(int dtype, int64_t n, int d, int k, bool backward, void *ws)
{
    LossPlan p = {};
    if (n < 1) n = 1; // (a call without rows plans for one)
    p.np = dtype == VLQ_F32 ? 2 : 1;
    p.n = n;
    p.npad = pad_to(n, TILE);
    p.kpad = pad_to(k, TILE);
    p.d = d;
    p.units = (d + 31) / 32;
    p.narrow = d <= narrow_dim(dtype);
    const double tile = 0.27 * p.units * (p.np == 2 ? 2.7 : 1.) * narrow_rows(p.np, p.units) / 128; // us of one in the narrow form, two workgroups a compute unit
    if (p.np == 1 && !p.narrow) p.units += p.units & 1; // (ProductRows takes two at a time)
    p.dblocks = d <= 128 ? 1 : (int)(pad_to(d, 256) / 128);
    p.rows = n < LOSS_ROWS ? n : LOSS_ROWS;
    p.rpad = pad_to(p.rows, TILE);
    p.piece = PIECE / p.rpad / TILE * TILE;
    if (p.piece < TILE) p.piece = TILE;
    if (p.piece > p.kpad) p.piece = p.kpad;
    size_t off = 0;
    auto take = [&](auto *&ptr, size_t count) {
        off = (off + 255) & ~(size_t)255;
        ptr = ws ? (std::remove_reference_t<decltype(ptr)>)((char *)ws + off) : nullptr;
        off += count * sizeof(*ptr);
    };
    p.few = backward && grads_are_few(dtype, n, d, k);
    if (p.few) {
        p.kp = (int)pad_to(k, 32);
        take(p.G, (size_t)n * p.kp);
        p.xsplit = few_parts(n, k, d);
        p.csplit = few_parts(k, n, d);
        p.xslab = p.xsplit > 1;
        p.cslab = p.csplit > 1;
        take(p.dbpart, (size_t)p.csplit * p.kp);
        take(p.xsum, p.xslab ? (size_t)p.xsplit * n * d : 0);
        take(p.csum, p.cslab ? (size_t)p.csplit * k * d : 0);
        p.bytes = (off + 255) & ~(size_t)255;
        return p;
    }
    const size_t page = (size_t)PAGE * p.np;
    take(p.hdr, 1);
    take(p.ximg, p.npad / 128 * p.units * page);
    take(p.cimg, p.kpad / 128 * p.units * page);
    take(p.rinv, p.npad);
    take(p.cinv, p.kpad / 16);
    take(p.bias2, p.kpad);
    take(p.row, p.npad);
    take(p.lab, p.npad);
    if (!backward && p.narrow) {
        const int64_t xq = p.npad / narrow_rows(p.np, p.units), xt = p.kpad / 32;
        p.xsplit = narrow_parts(xt, narrow_per(xq, xt, 0, 0, NARROW_GROUPS, NARROW_LEAST / 2, p.npad * 8., 0., tile / 3), p.npad * 8, &p.xper);
        take(p.mine, p.npad);
        take(p.part, p.xsplit * p.npad);
    } else if (!backward) {
        take(p.mine, p.rpad);
        take(p.part, p.kpad / 128 * p.rpad);
    } else {
        const int mt = p.dblocks / 2;
        take(p.gn, p.npad);
        take(p.xcols, p.npad / 32 * p.dblocks * page);
        take(p.ccols, p.kpad / 32 * p.dblocks * page);
        if (p.narrow) {
            const int64_t rows = narrow_rows(p.np, p.units), xq = p.npad / rows, cq = p.kpad / rows, xt = p.kpad / 32, ct = p.npad / 32;
            const int64_t per = narrow_per(xq, xt, cq, ct, NARROW_GROUPS / 2, NARROW_LEAST, n * d * 4., (double)k * d * 4, tile);
            p.xsplit = narrow_parts(xt, per, n * d * 4, &p.xper);
            p.csplit = narrow_parts(ct, per, (int64_t)k * d * 4, &p.cper);
            p.xslab = p.xsplit > 1;
            p.cslab = p.csplit > 1;
            take(p.dbpart, p.csplit * p.kpad);
            take(p.xsum, p.xslab ? (size_t)p.xsplit * n * d : 0);
            take(p.csum, p.cslab ? (size_t)p.csplit * k * d : 0);
            p.bytes = (off + 255) & ~(size_t)255;
            return p;
        }
        take(p.pj, p.rpad * p.piece / 8 * P_PARTS);
        take(p.pi, p.rpad * p.piece / 8 * P_PARTS);
        take(p.dbpart, p.rpad / 64 * p.piece);
        p.xsplit = sum_parts(p.rpad / TILE * mt, p.piece / 32, n * d * 4);
        p.csplit = sum_parts(p.piece / TILE * mt, p.rpad / 32, (int64_t)k * d * 4);
        p.xslab = p.xsplit > 1 || p.kpad > p.piece;
        p.cslab = p.csplit > 1 || n > p.rows;
        take(p.xsum, p.xslab ? (size_t)p.xsplit * n * d : 0);
        take(p.csum, p.cslab ? (size_t)p.csplit * k * d : 0);
    }
    p.bytes = (off + 255) & ~(size_t)255;
    return p;
}

size_t loss_workspace(int dtype, int64_t n, int d, int k, bool backward)
{
    const size_t forward = loss_is_few(dtype, n, d, k) ? ((size_t)(k / 32 + 1) * 8 + 4) * (n < 1 ? 1 : n) : loss_plan(dtype, n, d, k, false, nullptr).bytes;
    if (!backward) return forward;
    const size_t both = loss_plan(dtype, n, d, k, true, nullptr).bytes;
    return both < forward ? forward : both;
}

template <typename K>
static hipError_t allow_lds(K kern, size_t bytes)
{
    return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

#define LOSS_TRY(e)                              \
    do {                                         \
        const hipError_t e_ = (e);               \
        if (e_ != hipSuccess) return (int)e_;    \
    } while (0)

// The wide form takes the centroids as they lie (ProductRows) where that saves more than it costs: the products are a tenth
// slower, most where a row is a multiple of 4 KB and all rows of a tile come through the same channel of the L2.  us of a step, these
// against images: 284 x 50 632 x 1 376 fp16 590 : 659, 1 000 x 30 000 x 1 024 fp16 452 : 484, 4 096 x 32 000 x 2 048 bf16 2 720 : 2 786,
// 8 192 x 50 001 x 2 048 bf16 8 314 : 8 316.
#define LIE_ROWS 4096
template <typename T>
static bool as_they_lie(const LossArgs &a, const LossPlan &p)
{
    return sizeof(T) == 2 && !p.narrow && a.n <= LIE_ROWS && a.d % 8 == 0 && (uintptr_t)a.c % 16 == 0;
}

// The images of rows and centroids, and the rest of what the products need: one launch, two or three backward
template <typename T, int NP>
static void loss_images(const LossArgs &a, const LossPlan &p, bool backward, hipStream_t st)
{
    PackArgs g = {a.x, a.c, a.n, a.d, a.k, p.units, a.label, a.bias, a.grad, backward ? a.stats : nullptr, a.scale, p.ximg, p.cimg,
                  p.xcols, p.ccols, p.rinv, p.cinv, p.gn, p.bias2, p.row, p.lab, p.hdr, a.d % 8 == 0, as_they_lie<T>(a, p), __is_same(T, _Float16)};
    g.rinvs = p.npad;
    g.cinvs = p.kpad / 16;
    g.small = g.rinvs + g.cinvs <= SMALL_SCALES;
    g.xblocks = (int)(p.npad / 16);
    g.cblocks = (int)(p.kpad / 16);
    const dim3 packs((unsigned)(g.xblocks + g.cblocks));
    auto pack = [&](auto RAW) {
        if (p.units <= 16)
            hipLaunchKernelGGL((k_pack_rows<T, NP, 4, decltype(RAW)::value>), packs, dim3(256), 0, st, g);
        else
            hipLaunchKernelGGL((k_pack_rows<T, NP, 16, decltype(RAW)::value>), packs, dim3(256), 0, st, g);
    };
    if constexpr (NP == 1) {
        if (g.raw) {
            g.cimg = nullptr;
            if (!backward || !a.dx || g.halves) g.cinv = nullptr; // (the centroids' columns want a scale)
            pack(std::true_type{});
        } else {
            pack(std::false_type{});
        }
    } else {
        pack(std::false_type{});
    }
    if (backward && !g.small) hipLaunchKernelGGL(k_loss_header, dim3(3), dim3(1024), 0, st, g);
    if (!backward) return;
    g.dblocks = p.dblocks;
    g.xunits = (int)(p.npad / 32);
    g.cunits = (int)(p.kpad / 32);
    g.xblocks = a.dc ? g.xunits / 2 * p.dblocks : 0;
    g.cblocks = a.dx ? g.cunits / 2 * p.dblocks : 0;
    const dim3 grid((unsigned)(g.xblocks + g.cblocks + p.npad / 256));
    if (p.narrow)
        hipLaunchKernelGGL((k_pack_cols<T, 2, 2, NP>), grid, dim3(256), 0, st, g);
    else
        hipLaunchKernelGGL((k_pack_cols<T, 1, 0, NP>), grid, dim3(256), 0, st, g);
}

template <int NP>
static LogitArgs logit_args(const LossArgs &a, const LossPlan &p, int64_t r0, int64_t rpad, int64_t c0, int64_t cpad)
{
    LogitArgs g = {};
    const int64_t block = (int64_t)p.units * NP;
    g.A = {p.cimg + c0 / 128 * block * PAGE, block, 0};
    g.B = {p.ximg + r0 / 128 * block * PAGE, block, 0};
    g.c = (const char *)a.c + c0 * a.d * (NP == 1 ? 2 : 4);
    g.rows = (int)(a.k - c0);
    g.d = a.d;
    g.cinv = p.cinv + c0 / 16;
    g.bias2 = p.bias2 + c0;
    g.row = p.row + r0;
    g.lab = p.lab + r0;
    g.units = p.units;
    g.mt = (int)(cpad / TILE);
    g.nt = (int)(rpad / TILE);
    g.npad = (int)rpad;
    g.m_first = (int)c0;
    return g;
}

static void launch_merge(const float2 *part, int parts, int npad, const float *mine, const int32_t *lab, int k, const float *bias, int64_t n,
                         float *stats, float *loss, hipStream_t st)
{
    if (n <= FEW_ROWS)
        hipLaunchKernelGGL(k_loss_merge<1>, dim3((unsigned)n), dim3(256), 0, st, part, parts, npad, mine, lab, k, bias, n, stats, loss);
    else if (n <= MERGE_ROWS)
        hipLaunchKernelGGL(k_loss_merge<4>, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, st, part, parts, npad, mine, lab, k, bias, n, stats, loss);
    else
        hipLaunchKernelGGL(k_loss_merge<16>, dim3((unsigned)((n + 15) / 16)), dim3(256), 0, st, part, parts, npad, mine, lab, k, bias, n, stats, loss);
}

static int loss_few(const LossArgs &a, hipStream_t st)
{
    const int groups = few_groups(a.dtype, a.n, a.d, a.k);
    float2 *part = (float2 *)a.ws;
    float *mine = (float *)(part + (int64_t)groups * a.n);
    FewArgs f = {a.x, a.c, a.bias, a.label, a.scale * LOG2E, (int)a.n, a.d, a.k};
    f.part = part;
    f.mine = mine;
    launch_loss_few(a.dtype, f, false, st);
    launch_merge(part, groups, (int)a.n, mine, a.label, a.k, a.bias, a.n, a.stats, a.loss, st);
    return (int)hipGetLastError();
}

template <typename T, int NP>
static int loss_forward(const LossArgs &a, hipStream_t st)
{
    if (loss_is_few(a.dtype, a.n, a.d, a.k)) return loss_few(a, st);
    const LossPlan p = loss_plan(a.dtype, a.n, a.d, a.k, false, a.ws);
    loss_images<T, NP>(a, p, false, st);
    if (p.narrow) {
        NarrowArgs g = {};
        const int rows = narrow_rows(NP, p.units);
        g.units = p.units;
        g.d = a.d;
        g.row = p.row;
        g.lab = p.lab;
        g.cinv = p.cinv;
        g.bias2 = p.bias2;
        g.part = p.part;
        g.mine = p.mine;
        g.npad = (int)p.npad;
        g.x = {p.ximg, p.cimg, nullptr, (int)(p.npad / rows), (int)(p.kpad / 32), p.xsplit, p.xper, (int)a.n};
        LOSS_TRY((hipError_t)launch_loss_narrow_stats(a.dtype, g, st));
        launch_merge(p.part, p.xsplit, g.npad, p.mine, p.lab, a.k, a.bias, a.n, a.stats, a.loss, st);
        return (int)hipGetLastError();
    }
    using Images = FromImages<NP>;
    using Rows = std::conditional_t<NP == 1, FromRows<T>, Images>;
    const bool lie = as_they_lie<T>(a, p);
    const auto kern = lie ? k_loss_stats<Rows> : k_loss_stats<Images>;
    const size_t bytes = lie ? Rows::LDS : Images::LDS;
    LOSS_TRY(allow_lds(kern, bytes));
    for (int64_t r0 = 0; r0 < a.n; r0 += p.rows) {
        const int64_t rows = a.n - r0 < p.rows ? a.n - r0 : p.rows, rpad = pad_to(rows, TILE);
        LogitArgs g = logit_args<NP>(a, p, r0, rpad, 0, p.kpad);
        g.part = p.part;
        g.mine = p.mine;
        hipLaunchKernelGGL(kern, dim3((unsigned)(g.mt * g.nt)), dim3(LNT), bytes, st, g);
        launch_merge(p.part, g.mt * 2, g.npad, p.mine, g.lab, a.k, a.bias, rows, a.stats + 2 * r0, a.loss ? a.loss + r0 : nullptr, st);
    }
    return (int)hipGetLastError();
}

template <typename T, int NP>
static int loss_backward(const LossArgs &a, hipStream_t st)
{
    if (a.n == 0) {
        const int64_t count = (int64_t)a.k * a.d;
        hipLaunchKernelGGL(k_loss_none<T>, dim3((unsigned)(count < 4096 * 256 ? (count + 255) / 256 : 4096)), dim3(256), 0, st, (T *)a.dc, count, a.dbias, a.k);
        return (int)hipGetLastError();
    }
    const LossPlan p = loss_plan(a.dtype, a.n, a.d, a.k, true, a.ws);
    if (!p.few) loss_images<T, NP>(a, p, true, st);
    const float *top = p.few ? nullptr : &p.hdr->top;
    auto bias_part = [&](int slots, int64_t ld, int64_t c0, int64_t count, bool add) {
        return BiasSum{p.dbpart, slots, (int)ld, (int)count, (int)((count + 63) / 64), top, add, a.dbias + c0};
    };
    auto finish = [&](BiasSum bias) {
        auto side = [&](float *slabs, int splits, int64_t count, void *out) { return SlabSum{slabs, splits, 0, 0, count, top, out}; };
        auto left = [](const SlabSum &s) { // workgroups of the next launch: a grid has fewer than 2^32 threads
            const int64_t each = s.splits >= SUM_SHARED ? 256 : 1024, most = 1 << 22, l = (s.count + each - 1) / each - s.first;
            return l < most ? l : most;
        };
        SlabSum x = {}, c = {};
        if (a.dx && p.xslab) x = side(p.xsum, p.xsplit, a.n * a.d, a.dx);
        if (a.dc && p.cslab) c = side(p.csum, p.csplit, (int64_t)a.k * a.d, a.dc);
        for (;;) {
            x.blocks = left(x);
            c.blocks = left(c);
            const int64_t blocks = x.blocks + c.blocks + bias.blocks;
            if (!blocks) break;
            hipLaunchKernelGGL(k_loss_sums<T>, dim3((unsigned)blocks), dim3(256), 0, st, x, c, bias, a.scale);
            x.first += x.blocks;
            c.first += c.blocks;
            bias.blocks = 0;
        }
    };
    if (p.few) {
        FewArgs f = {a.x, a.c, a.bias, a.label, a.scale * LOG2E, (int)a.n, a.d, a.k};
        f.stats = a.stats;
        f.grad = a.grad;
        f.G = p.G;
        f.kp = p.kp;
        launch_loss_few(a.dtype, f, true, st);
        const bool bias = a.dbias != nullptr;
        f.scale = a.scale;
        if (a.dx) f.dx = few_side(a.n, a.k, a.d, p.xsplit, p.xslab ? (void *)p.xsum : a.dx, p.xslab);
        if (a.dc || bias) f.dc = few_side(a.k, a.n, a.d, p.csplit, !a.dc ? nullptr : p.cslab ? (void *)p.csum : a.dc, p.cslab);
        f.db = !bias ? nullptr : p.cslab ? p.dbpart : a.dbias;
        launch_loss_few_grads(a.dtype, f, st);
        finish(bias && p.cslab ? bias_part(p.csplit, p.kp, 0, a.k, false) : BiasSum{});
        return (int)hipGetLastError();
    }
    if (p.narrow) {
        NarrowArgs g = {};
        const int rows = narrow_rows(NP, p.units);
        g.units = p.units;
        g.d = a.d;
        g.row = p.row;
        g.lab = p.lab;
        g.gn = p.gn;
        g.cinv = p.cinv;
        g.bias2 = p.bias2;
        g.hdr = p.hdr;
        g.dbpart = a.dbias ? p.dbpart : nullptr;
        g.kpad = (int)p.kpad;
        g.scale = a.scale;
        if (a.dx) {
            g.x = {p.ximg, p.cimg, p.ccols, (int)(p.npad / rows), (int)(p.kpad / 32), p.xsplit, p.xper, (int)a.n, p.xslab,
                   p.xslab ? (void *)p.xsum : a.dx, a.d % 4 == 0 && (p.xslab || (uintptr_t)a.dx % 16 == 0)};
            g.nx = g.x.qblocks * g.x.splits;
        }
        if (a.dc || a.dbias)
            g.c = {p.cimg, p.ximg, p.xcols, (int)(p.kpad / rows), (int)(p.npad / 32), p.csplit, p.cper, a.k, p.cslab,
                   !a.dc ? nullptr : p.cslab ? (void *)p.csum : a.dc,
                   a.d % 4 == 0 && (p.cslab || (uintptr_t)a.dc % 16 == 0)};
        LOSS_TRY((hipError_t)launch_loss_narrow(a.dtype, g, st));
        finish(a.dbias ? bias_part(p.csplit, p.kpad, 0, a.k, false) : BiasSum{});
        return (int)hipGetLastError();
    }
    const bool lie = as_they_lie<T>(a, p);
    using Rows = std::conditional_t<NP == 1, FromRows<T>, FromImages<NP>>;
    LOSS_TRY(lie ? allow_lds(k_loss_p<Rows>, Rows::LDS) : allow_lds(k_loss_p<FromImages<NP>>, FromImages<NP>::LDS));
    using Sums = Product<NP, P_PARTS>;
    LOSS_TRY(allow_lds(k_loss_grads<T, NP>, Sums::LDS));
    const int mt = p.dblocks / 2;
    const bool vec = a.d % 4 == 0, whole = a.n <= p.rows && p.kpad <= p.piece; // (one piece: dbias with the other sums)
    for (int64_t r0 = 0; r0 < a.n; r0 += p.rows) {
        const int64_t rows = a.n - r0 < p.rows ? a.n - r0 : p.rows, rpad = pad_to(rows, TILE);
        for (int64_t c0 = 0; c0 < p.kpad; c0 += p.piece) {
            const int64_t cpad = p.kpad - c0 < p.piece ? p.kpad - c0 : p.piece;
            LogitArgs g = logit_args<NP>(a, p, r0, rpad, c0, cpad);
            g.gn = p.gn + r0;
            g.pj = (u32x2 *)p.pj;
            g.pi = (u32x2 *)p.pi;
            g.jblock = (int)(cpad / 32 * P_PARTS);
            g.iblock = (int)(rpad / 32 * P_PARTS);
            g.dbpart = a.dbias ? p.dbpart : nullptr;
            if (lie)
                hipLaunchKernelGGL(k_loss_p<Rows>, dim3((unsigned)(g.mt * g.nt)), dim3(LNT), Rows::LDS, st, g);
            else
                hipLaunchKernelGGL(k_loss_p<FromImages<NP>>, dim3((unsigned)(g.mt * g.nt)), dim3(LNT), FromImages<NP>::LDS, st, g);
            if (a.dbias && !whole) {
                const BiasSum bias = bias_part((int)(rpad / 64), cpad, c0, a.k - c0 < cpad ? a.k - c0 : cpad, r0 > 0);
                hipLaunchKernelGGL(k_loss_sums<T>, dim3((unsigned)bias.blocks), dim3(256), 0, st, SlabSum{}, SlabSum{}, bias, a.scale);
            }
            GradOut x = {}, c = {};
            if (a.dx) {
                x.A = {p.ccols, p.kpad / 32 * NP, c0 / 32 * NP};
                x.B = {p.pj, g.jblock, 0};
                x.units = (int)(cpad / 32);
                x.mt = mt;
                x.nt = g.nt;
                x.splits = p.xsplit;
                x.per = (x.units + p.xsplit - 1) / p.xsplit;
                x.splits = (x.units + x.per - 1) / x.per; // (a shorter last piece may need fewer: its other slabs stay as they are)
                x.rows = (int)rows;
                x.mode = p.xslab ? (c0 > 0 ? 2 : 1) : 0;
                x.out = p.xslab ? (void *)(p.xsum + r0 * a.d) : (void *)((T *)a.dx + r0 * a.d);
                x.slab = a.n * a.d;
                x.inv = &p.hdr->cinv;
                x.gn = p.gn + r0;
                x.vec = vec && (p.xslab || (uintptr_t)a.dx % 16 == 0);
            }
            if (a.dc) {
                const int64_t cols = a.k - c0 < cpad ? a.k - c0 : cpad;
                c.A = {p.xcols, p.npad / 32 * NP, r0 / 32 * NP};
                c.B = {p.pi, g.iblock, 0};
                c.units = (int)(rpad / 32);
                c.mt = mt;
                c.nt = g.mt;
                c.splits = p.csplit;
                c.per = (c.units + p.csplit - 1) / p.csplit;
                c.splits = (c.units + c.per - 1) / c.per;
                c.permuted = true;
                c.rows = (int)cols;
                c.mode = p.cslab ? (r0 > 0 ? 2 : 1) : 0;
                c.out = p.cslab ? (void *)(p.csum + c0 * a.d) : (void *)((T *)a.dc + c0 * a.d);
                c.slab = (int64_t)a.k * a.d;
                c.inv = &p.hdr->xinv;
                c.vec = vec && (p.cslab || (uintptr_t)a.dc % 16 == 0);
            }
            x.d = c.d = a.d;
            x.scale = c.scale = a.scale;
            x.top = c.top = top;
            const int nx = x.mt * x.nt * x.splits, nc = c.mt * c.nt * c.splits;
            if (nx + nc == 0) continue;
            if (c.per > x.per)
                hipLaunchKernelGGL((k_loss_grads<T, NP>), dim3((unsigned)(nx + nc)), dim3(LNT), Sums::LDS, st, c, x, nc);
            else
                hipLaunchKernelGGL((k_loss_grads<T, NP>), dim3((unsigned)(nx + nc)), dim3(LNT), Sums::LDS, st, x, c, nx);
        }
    }
    finish(a.dbias && whole ? bias_part((int)(p.rpad / 64), p.kpad, 0, a.k, false) : BiasSum{});
    return (int)hipGetLastError();
}

int launch_softmax_loss(const LossArgs &a, hipStream_t st)
{
    switch (a.dtype) {
    case VLQ_F32: return loss_forward<float, 2>(a, st);
    case VLQ_F16: return loss_forward<_Float16, 1>(a, st);
    default: return loss_forward<bf16_t, 1>(a, st);
    }
}

int launch_softmax_loss_backward(const LossArgs &a, hipStream_t st)
{
    switch (a.dtype) {
    case VLQ_F32: return loss_backward<float, 2>(a, st);
    case VLQ_F16: return loss_backward<_Float16, 1>(a, st);
    default: return loss_backward<bf16_t, 1>(a, st);
    }
}
