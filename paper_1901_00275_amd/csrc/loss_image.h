// What the kernels of the softmax loss (softmax_loss.hip, softmax_loss_narrow.hip) share: values and their fp16 parts, the
// images of matrices, the gradients' outputs.
#pragma once
#include "learn.h"

#include <type_traits>

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_t;

#define PAGE 512      // 16-byte chunks of a page: 128 rows x 32 indices
#define TILE 256      // rows of all images are padded to this
#define P_ONE 32768.f // 2^15, what a probability of one is in P
// P has two fp16 parts, 22 bits, whatever the operands' type: with one part the sums of a gradient were off by 1.5e-4 of their terms, which
// showed in 2 to 8 % of bf16 outputs, and by far more than the outputs' own rounding where the terms all but cancel (centroids
// with a mean of 30 times their spread: 4.4e-3 of dx)
#define P_PARTS 2
#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f
#define MOST __FLT_MAX__

// A bias in units of log 2.  A finite one stays finite: fp32's lowest value is a usual mask, and only -infinity takes a centroid out.
__device__ __forceinline__ float bias_log2(float b)
{
    const float v = b * LOG2E;
    return fabsf(b) < INFINITY ? fminf(fmaxf(v, -MOST), MOST) : v;
}

// Exponent of the power of two that brings mx to [2^14, 2^15)
// (a row of zeros takes the largest: it has no part in the largest inverse scale of its matrix)
__device__ __forceinline__ int scale_exponent(float mx)
{
    const int ex = mx > 0.f ? 14 - ((int)(__float_as_uint(mx) >> 23) - 127) : 126;
    return min(max(ex, -126), 126);
}
__device__ __forceinline__ float pow2i(int ex) { return __uint_as_float((uint32_t)(127 + ex) << 23); }

// eight values of a row from index i on, zeros past its end
template <typename T>
struct Eight {
    // 16 bytes at a value's address (four words, written so that the type depends on T, as its alignment does)
    typedef uint32_t At __attribute__((ext_vector_type(4 * sizeof(T) / sizeof(T)), aligned(sizeof(T))));
    T v[8];
};
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T *row, int i, int d, bool vec)
{
    Eight<T> r;
    using At = typename Eight<T>::At;
    if (vec) { // (d is a multiple of 8)
        u32x4 *w = (u32x4 *)r.v;
#pragma unroll
        for (int p = 0; p < (int)sizeof(T) / 2; ++p) w[p] = i < d ? ((const At *)(row + i))[p] : At{0, 0, 0, 0};
    } else if (i + 8 <= d) {
        u32x4 *w = (u32x4 *)r.v;
#pragma unroll
        for (int p = 0; p < (int)sizeof(T) / 2; ++p) w[p] = ((const At *)(row + i))[p];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = i + e < d ? row[i + e] : (T)0.f;
    }
    return r;
}

// v as one or two fp16 parts.  The value is taken as it is in fp32: where it is a product, the compiler may otherwise round it to
// fp16 in one step for the one use of hi and in two for the other, and hi and lo no longer fit together.
template <int NP>
__device__ __forceinline__ void halves(float v, _Float16 &hi, _Float16 &lo)
{
    if (NP == 2) asm("" : "+v"(v));
    hi = (_Float16)v;
    if (NP == 2) lo = (_Float16)(v - (float)hi);
}
template <int NP>
__device__ __forceinline__ void split8(const float (&v)[8], half8 (&h)[NP])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        halves<NP>(v[e], hi, lo);
        h[0][e] = hi;
        if (NP == 2) h[NP - 1][e] = lo;
    }
}

// The statistics of two sets of logits together
__device__ __forceinline__ float2 join(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - base) + b.y * __builtin_amdgcn_exp2f(b.x - base));
}

// What a backward call knows of its matrices as a whole
struct LossHeader {
    float xinv, cinv; // inverse scales of the columns' images
    float top;        // largest |g|
};
// What a sum is multiplied with to be one of x's or c's own values times P: a power of two, the inverse scales of the columns' image and of
// P.  The rows' gradients come in relative to the largest, that one and the call's scale last, one by one: multiplied together first they
// left fp32's range where the results do not (largest |grad| of 2^-96 and less, 2^98 and more).
__device__ __forceinline__ float grad_unit(float inv) { return inv * (1.f / P_ONE); }

template <typename T>
__device__ __forceinline__ void store4(T *p, const f32x4 &v, int count, bool vec)
{
    if (vec && count >= 4) {
        if constexpr (sizeof(T) == 4) {
            *(f32x4 *)p = v;
        } else {
            T t[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
            *(u32x2 *)p = *(u32x2 *)t;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) p[e] = (T)v[e];
}

// ---- softmax_loss_few.hip ----
struct FewSide { // one gradient: rows, length of its sum, the parts that is cut into, steps of 16 of a part
    int rows, sum, parts, per;
    int rtiles, dtiles, blocks; // tiles of 32 rows, of 64 dimensions (256 where the waves do not share a sum), workgroups
    bool share;                 // the four waves of a workgroup share a tile's sum
    bool slab;                  // slabs [parts][rows x d], or typed and times the scale
    void *out;                  // (NULL: dbias alone)
};
struct FewArgs {
    const void *x, *c;
    const float *bias;
    const int32_t *label;
    float scale2; // in units of log 2
    int n, d, k;
    int groups; // of centroids
    // forward
    float2 *part; // [groups][n]
    float *mine;
    // backward
    const float *stats, *grad;
    float *G; // [n][kp]
    int kp;
    FewSide dx, dc;
    float *db; // [parts of dc][kp], or dbias itself
    float scale;
};
int few_groups(int dtype, int64_t n, int d, int k);
int few_parts(int64_t rows, int64_t sum, int d);
FewSide few_side(int64_t rows, int64_t sum, int d, int parts, void *out, bool slab);
void launch_loss_few(int dtype, const FewArgs &a, bool backward, hipStream_t st); // statistics, or G
void launch_loss_few_grads(int dtype, const FewArgs &a, hipStream_t st);

// ---- softmax_loss_narrow.hip ----
// rows that a workgroup keeps: 256 halve the traffic of LDS where their sums and fragments fit the registers (of 256 dimensions those of
// 128 rows take all 256 of a wave, and one is spilled)
constexpr int narrow_rows(int parts, int units) { return parts == 2 || units >= 4 ? 128 : 256; }
struct NarrowSide {
    const u32x4 *q, *r, *rt; // images of the gradient's rows, of the other matrix's rows and columns
    int qblocks, tiles, splits, per; // workgroups side by side; tiles of the other matrix, in so many parts of `per`
    int rows;
    int mode; // 0: typed; 1: slabs [splits][rows x d], without the scale and g's largest
    void *out;
    bool vec;
};
struct NarrowArgs {
    NarrowSide x, c;
    int units, d, nx; // workgroups of the first side
    const f32x4 *row; // per row of x: factor, maximum, factors of P
    const int32_t *lab;
    const float *gn, *cinv, *bias2;
    const LossHeader *hdr;
    float *dbpart; // [splits of c][kpad] or NULL
    int kpad;
    float scale;
    // forward (the first side alone)
    float2 *part; // [splits][npad] {maximum, sum}
    float *mine;  // [npad] the label's logit
    int npad;
};
int launch_loss_narrow_stats(int dtype, const NarrowArgs &a, hipStream_t st); // 0 or a hipError_t
int launch_loss_narrow(int dtype, const NarrowArgs &a, hipStream_t st); // 0 or a hipError_t
