// The softmax loss and its gradients where little is done with each centroid: few rows, or little work.  Rows and centroids are read
// as they lie, nothing is rewritten first.
//
// Logits: every wave multiplies 16 G centroids with up to 64 rows (NT tiles of 16); 16-bit values on their own matrix instructions,
// fp32 on the fp32 ones (a read of 4 bytes needs 16 NT multiplications, which these do in time up to NT = 4).  Up to 64 rows
// the centroids pass once and bound it (65 536 x 1 024 bf16, one row: 25 us, 5.4 TB/s), beyond that the rows' fragments from the caches
// do; where there are few workgroups the waits for them do, and S waves share the dimensions of a tile.
//
// Gradients: G_ij = g_i (p_ij - [j = y_i]) is written in fp32, then dx = s G C and dc = s G^T X on the fp32 matrix instructions, 16-bit
// values widened as they are read: their rate is an eighth of fp16's, but nothing is padded to 256 rows or written as an image.
// Bound by the waits for turns of loads: 5 366 x 24 x 2 016 fp16 G 13 us, gradients 28, of which the products take 7; 500 x 500 x 500
// fp32 10 and 16.  With more work the products show (64 x 65 536 x 1 024 bf16: 112 of a step's 406 us at fp32's rate of 154 TFLOP/s).
#include "loss_image.h"

#define FEW_WIDE 65536 // from so many centroids on a wave takes 32 of them: then there are waves enough
#define FEW_GROUPS 512 // with fewer workgroups of eight waves they have two tiles

template <typename T>
struct FewPiece { // what a lane reads of a row at a time: its share of STEP indices
    static constexpr int N = 16 / sizeof(T), STEP = 4 * N;
    typedef uint32_t At __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T)))); // 16 bytes at a value's address
    T v[N];
};
// How rows are read: WHOLE, a row is a number of pieces; ENDED, its last piece ends where the row does, and what the one before had is
// made zero; SHORT, a row is less than a piece.  The memory takes 16 bytes at any value's address.  (A step of 3 855 x 11 x 657
// fp32 52 us value by value, 35 so; 500 x 500 x 500 bf16 by two values 40, 26 so.)
enum { WHOLE, ENDED, SHORT };
// Every address is clamped into the row, what lies past its end is made zero afterwards: a branch around a load would wait for it.
// Where one tile of rows is all there is (THIN), memory bounds it, and what is not there is not asked for (65 536 x 1 024 bf16,
// one row 27 us; clamped 28, with the other 15 rows 29).
template <typename T, int FORM, bool THIN>
__device__ __forceinline__ FewPiece<T> few_piece(const T *row, int i, int d, bool there)
{
    using P = FewPiece<T>;
    using At = typename P::At;
    if constexpr (FORM == WHOLE && THIN) {
        u32x4 v = {0, 0, 0, 0};
        if (there && i < d) v = *(const At *)(row + i);
        return __builtin_bit_cast(P, v);
    } else if constexpr (FORM == WHOLE) {
        const u32x4 v = *(const At *)(row + min(i, d - P::N));
        return __builtin_bit_cast(P, i < d ? v : u32x4{0, 0, 0, 0});
    } else if constexpr (FORM == ENDED) {
        const int at = min(i, d - P::N);
        P r = __builtin_bit_cast(P, (u32x4) * (const At *)(row + at));
#pragma unroll
        for (int e = 0; e < P::N; ++e) r.v[e] = at + e >= i ? r.v[e] : (T)0.f;
        return r;
    } else {
        P r;
#pragma unroll
        for (int e = 0; e < P::N; ++e) {
            const T v = row[min(i + e, d - 1)];
            r.v[e] = i + e < d ? v : (T)0.f;
        }
        return r;
    }
}
__device__ __forceinline__ void few_multiply(const FewPiece<float> &a, const FewPiece<float> &b, f32x4 &acc)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], acc, 0, 0, 0);
}
__device__ __forceinline__ void few_multiply(const FewPiece<_Float16> &a, const FewPiece<_Float16> &b, f32x4 &acc)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(*(const half8 *)a.v, *(const half8 *)b.v, acc, 0, 0, 0);
}
__device__ __forceinline__ void few_multiply(const FewPiece<bf16_t> &a, const FewPiece<bf16_t> &b, f32x4 &acc)
{
    typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)a.v, *(const bf16x8 *)b.v, acc, 0, 0, 0);
}

// The logits' products of centroids m0 .. and rows n0 ..; of S waves the first has them
template <typename T, int FORM, int W, int S, int G, int NT>
__device__ __forceinline__ void few_logits(const FewArgs &a, int m0, int n0, int tile, int slice, f32x4 (&acc)[G][NT])
{
    constexpr int STEP = FewPiece<T>::STEP, N = FewPiece<T>::N, U = 16 / (G + NT) < 2 ? 2 : 16 / (G + NT);
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
    const T *crow[G], *xrow[NT]; // (past the last: the first, whose logits are not used)
#pragma unroll
    for (int i = 0; i < G; ++i) crow[i] = (const T *)a.c + (int64_t)(m0 + 16 * i + l < a.k ? m0 + 16 * i + l : 0) * a.d;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        xrow[j] = (const T *)a.x + (int64_t)(n0 + 16 * j + l < a.n ? n0 + 16 * j + l : 0) * a.d;
#pragma unroll
        for (int i = 0; i < G; ++i) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int k0 = slice * U * STEP; k0 < a.d; k0 += S * U * STEP) {
        FewPiece<T> cv[U][G], xv[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < G; ++i) cv[u][i] = few_piece<T, FORM, NT == 1>(crow[i], k0 + g * N + u * STEP, a.d, true);
#pragma unroll
            for (int j = 0; j < NT; ++j) xv[u][j] = few_piece<T, FORM, NT == 1>(xrow[j], k0 + g * N + u * STEP, a.d, NT > 1 || l < a.n);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) few_multiply(cv[u][i], xv[u][j], acc[i][j]);
    }
    if constexpr (S > 1) {
        __shared__ f32x4 sum[S - 1][W][G * NT][64];
        if (slice > 0)
#pragma unroll
            for (int e = 0; e < G * NT; ++e) sum[slice - 1][tile][e][lane] = acc[e / NT][e % NT];
        __syncthreads();
        if (slice == 0)
#pragma unroll
            for (int o = 0; o < S - 1; ++o)
#pragma unroll
                for (int e = 0; e < G * NT; ++e) acc[e / NT][e % NT] += sum[o][tile][e][lane];
    }
}

// The bias of a lane's centroids, asked for before the products
template <int G>
__device__ __forceinline__ void few_bias(const FewArgs &a, int m0, int g, float (&b)[G][4])
{
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) b[i][r] = 0.f;
    if (a.bias)
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) b[i][r] = a.bias[min(m0 + 16 * i + 4 * g + r, a.k - 1)];
}

// Forward: maxima and sums of a workgroup's centroids, and the labels' logits
template <typename T, int FORM, int W, int S, int G, int NT>
__global__ __launch_bounds__(W * S * 64) void k_loss_few(FewArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4, wave = (tid >> 6) % W, slice = (tid >> 6) / W;
    const int group = blockIdx.x % a.groups, m0 = (group * W + wave) * 16 * G, n0 = (int)(blockIdx.x / a.groups) * 16 * NT;
    f32x4 acc[G][NT];
    float bias[G][4];
    int label[NT];
    few_bias<G>(a, m0, g, bias);
#pragma unroll
    for (int j = 0; j < NT; ++j) label[j] = a.label[min(n0 + 16 * j + l, a.n - 1)];
    few_logits<T, FORM, W, S, G, NT>(a, m0, n0, wave, slice, acc);
    __shared__ float2 s[W][16 * NT];
    if (slice == 0)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = n0 + 16 * j + l, lab = n < a.n ? label[j] : -1;
        float m = -INFINITY, z = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = m0 + 16 * i + 4 * g + r;
                const float b = c >= a.k ? -INFINITY : bias_log2(bias[i][r]);
                const float v = b == -INFINITY ? -INFINITY : fmaf(acc[i][j][r], a.scale2, b);
                if (c == lab && c < a.k) a.mine[n] = v;
                m = fmaxf(m, v);
                acc[i][j][r] = v;
            }
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float m1 = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) z += __builtin_amdgcn_exp2f(acc[i][j][r] - m1);
        z += __shfl_xor(z, 16, 64);
        z += __shfl_xor(z, 32, 64);
        if (g == 0) s[wave][16 * j + l] = make_float2(m, z);
    }
    __syncthreads();
    if (tid >= 16 * NT || n0 + tid >= a.n) return;
    float2 v = s[0][tid];
#pragma unroll
    for (int w = 1; w < W; ++w) v = join(v, s[w][tid]);
    a.part[(int64_t)group * a.n + n0 + tid] = v;
}

// Backward: G of a tile.  A row that does not count has zeros; a centroid that was taken out has p = 0.
template <typename T, int FORM, int W, int S, int G, int NT>
__global__ __launch_bounds__(W * S * 64) void k_loss_few_g(FewArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4, wave = (tid >> 6) % W, slice = (tid >> 6) / W;
    const int group = blockIdx.x % a.groups, m0 = (group * W + wave) * 16 * G, n0 = (int)(blockIdx.x / a.groups) * 16 * NT;
    f32x4 acc[G][NT];
    float bias[G][4], grad[NT];
    float2 stats[NT];
    int label[NT];
    few_bias<G>(a, m0, g, bias);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t n = min(n0 + 16 * j + l, a.n - 1);
        label[j] = a.label[n];
        stats[j].x = a.stats[2 * n];
        stats[j].y = a.stats[2 * n + 1];
        grad[j] = a.grad[n];
    }
    few_logits<T, FORM, W, S, G, NT>(a, m0, n0, wave, slice, acc);
    if (slice > 0) return;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = n0 + 16 * j + l, lab = label[j];
        if (n >= a.n) continue;
        const float m = stats[j].x, z = stats[j].y, gn = grad[j];
        const bool ok = (uint32_t)lab < (uint32_t)a.k && m != -INFINITY;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int c0 = m0 + 16 * i + 4 * g;
            if (c0 >= a.kp) continue;
            f32x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = c0 + r;
                const float b = c >= a.k ? -INFINITY : bias_log2(bias[i][r]);
                const float p = b == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], a.scale2, b) - m) / z;
                v[r] = !ok || c >= a.k ? 0.f : gn * (c == lab ? p - 1.f : p);
            }
            *(f32x4 *)(a.G + (int64_t)n * a.kp + c0) = v;
        }
    }
}

// Four values at any value's address
template <typename T>
__device__ __forceinline__ void load4(T (&v)[4], const T *p)
{
    typedef std::conditional_t<sizeof(T) == 4, u32x4, u32x2> Word;
    typedef Word At __attribute__((aligned(sizeof(T))));
    *(Word *)v = *(const At *)p;
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_dims(T *p, const f32x4 &v, int count)
{
    typedef std::conditional_t<sizeof(T) == 4, u32x4, u32x2> Word;
    typedef Word At __attribute__((aligned(sizeof(T))));
    const T t[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    if constexpr (VEC) {
        *(At *)p = *(const Word *)t;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < count) p[e] = t[e];
    }
}

// A gradient's tile of 32 rows x 64 dimensions a wave: sum over q of G's 32 rows and 64 values of the other matrix's row q, in steps of
// 16 q.  The order of the 16 within a step is free as long as both operands have it, and which rows and dimensions a tile's
// lanes stand for is, too: a lane reads four neighbouring dimensions (and, for dx, four neighbouring q of G) at once.
template <typename T, bool VEC, bool CENT>
__device__ __forceinline__ void few_grad(const FewArgs &a, const FewSide &s, int b, f32x4 (*sum)[8][64])
{
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = s.rtiles * s.dtiles, part = b / tiles, tile = b - part * tiles, dt = tile / s.rtiles;
    const int r0 = (tile - dt * s.rtiles) * 32, dim0 = (s.share ? dt : dt * 4 + wave) * 64 + 4 * l;
    const int dim = VEC ? min(dim0, a.d - 4) : dim0; // (the last four end where the row does, some of them taken twice)
    const int steps = (s.sum + 15) / 16, p1 = min(steps, (part + 1) * s.per), by = s.share ? 4 : 1;
    const T *rows = (const T *)(CENT ? a.x : a.c);
    const float *bias = a.bias ? a.bias : a.G; // (read either way: a branch around a load would wait for it)
    f32x4 acc[2][4];
    float db[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int st = part * s.per + (s.share ? wave : 0); st < p1; st += 2 * by) {
        float A[2][2][4], B[2][4][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int q0 = (st + h * by) * 16 + 4 * g;
            const bool there = st + h * by < p1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = there && q0 + e < s.sum;
                const int q = in ? q0 + e : 0;
                bool keep;
                if (CENT)
                    keep = (uint32_t)a.label[q] < (uint32_t)a.k;
                else
                    keep = !a.bias | (bias[q] != -INFINITY);
                keep &= in;
                const T *row = rows + (int64_t)q * a.d; // (dimensions past the end are not stored)
                T v[4];
                if constexpr (VEC)
                    load4(v, row + dim);
                else
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = row[min(dim + u, a.d - 1)];
#pragma unroll
                for (int u = 0; u < 4; ++u) B[h][e][u] = keep ? (float)v[u] : 0.f;
                if constexpr (CENT) {
                    const float2 v = *(const float2 *)(a.G + (int64_t)q * a.kp + r0 + 2 * l);
                    A[h][0][e] = in ? v.x : 0.f;
                    A[h][1][e] = in ? v.y : 0.f;
                }
            }
            if constexpr (!CENT)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const f32x4 v = *(const f32x4 *)(a.G + (int64_t)min(r0 + 16 * t + l, s.rows - 1) * a.kp + (there ? q0 : 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) A[h][t][e] = there ? v[e] : 0.f;
                }
        }
        __builtin_amdgcn_sched_barrier(0); // (all loads of a turn are asked for before its first product)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (CENT)
#pragma unroll
                    for (int t = 0; t < 2; ++t) db[t] += A[h][t][e];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int u = 0; u < 4; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[h][t][e], B[h][e][u], acc[t][u], 0, 0, 0);
            }
    }
    if (CENT && a.db) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            db[t] += __shfl_xor(db[t], 16, 64);
            db[t] += __shfl_xor(db[t], 32, 64);
        }
    }
    if (s.share) {
        __shared__ float dbs[3][2][16];
        if (wave > 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (CENT && g == 0) dbs[wave - 1][t][l] = db[t];
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[wave - 1][t * 4 + u][lane] = acc[t][u];
            }
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (CENT) db[t] += dbs[w][t][l];
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[t][u] += sum[w][t * 4 + u][lane];
            }
    }
    if (CENT && a.db && dim0 == 4 * l && g == 0)
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (r0 + 2 * l + t < s.rows) a.db[(int64_t)part * a.kp + r0 + 2 * l + t] = db[t];
    if (!s.out || dim0 >= a.d) return;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = r0 + (CENT ? 2 * (4 * g + r) + t : 16 * t + 4 * g + r);
            if (row >= s.rows) continue;
            const f32x4 v = {acc[t][0][r], acc[t][1][r], acc[t][2][r], acc[t][3][r]};
            if (s.slab)
                store_dims<VEC>((float *)s.out + ((int64_t)part * s.rows + row) * a.d + dim, v, a.d - dim);
            else
                store_dims<VEC>((T *)s.out + (int64_t)row * a.d + dim, v * a.scale, a.d - dim);
        }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_loss_few_grads(FewArgs a)
{
    __shared__ f32x4 sum[3][8][64];
    if ((int)blockIdx.x < a.dc.blocks)
        few_grad<T, VEC, true>(a, a.dc, blockIdx.x, sum);
    else
        few_grad<T, VEC, false>(a, a.dx, blockIdx.x - a.dc.blocks, sum);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// Tiles of a workgroup, centroids of a wave, waves that share a tile's dimensions: two tiles a workgroup where eight would leave
// compute units without one, then with four waves each where every one of them has something to do; 32 centroids a wave where
// there are plenty.
struct FewShape {
    bool small, wide, shared;
    int groups;
};
static FewShape few_shape(int dtype, int64_t n, int d, int k)
{
    FewShape f;
    f.small = (k + 127) / 128 * ((n + 63) / 64) < FEW_GROUPS;
    f.wide = !f.small && k >= FEW_WIDE;
    f.shared = f.small && (int64_t)d * (dtype == VLQ_F32 ? 4 : 2) >= 768;
    const int each = f.small ? 32 : f.wide ? 256 : 128;
    f.groups = (k + each - 1) / each;
    return f;
}
int few_groups(int dtype, int64_t n, int d, int k) { return few_shape(dtype, n, d, k).groups; }

template <typename T>
static void few(int dtype, const FewArgs &args, bool backward, hipStream_t st)
{
    FewArgs a = args;
    const FewShape f = few_shape(dtype, a.n, a.d, a.k);
    a.groups = f.groups;
    auto go = [&](auto FORM, auto W, auto S, auto G, auto NT) {
        constexpr int R = 16 * decltype(NT)::value, WS = decltype(W)::value * decltype(S)::value;
        const dim3 grid((unsigned)(a.groups * ((a.n + R - 1) / R)));
        if (backward)
            hipLaunchKernelGGL((k_loss_few_g<T, decltype(FORM)::value, decltype(W)::value, decltype(S)::value, decltype(G)::value, decltype(NT)::value>),
                               grid, dim3(WS * 64), 0, st, a);
        else
            hipLaunchKernelGGL((k_loss_few<T, decltype(FORM)::value, decltype(W)::value, decltype(S)::value, decltype(G)::value, decltype(NT)::value>),
                               grid, dim3(WS * 64), 0, st, a);
    };
    auto rows = [&](auto FORM, auto W, auto S, auto G) {
        // tiles of 64 rows, of fewer where compute units would go without a workgroup (a step of 3 855 x 11 x 657 fp32 100 -> 60 us,
        // 64 x 1 000 x 1 024 fp32 26 -> 14; asking for 700 workgroups 535 x 975 x 1 248 fp32 44 -> 53)
        int tiles = 4;
        while (tiles > 1 && (a.n <= 8 * tiles || (int64_t)a.groups * ((a.n + 16 * tiles - 1) / (16 * tiles)) < 256)) tiles /= 2;
        if (tiles == 1)
            go(FORM, W, S, G, std::integral_constant<int, 1>{});
        else if (tiles == 2)
            go(FORM, W, S, G, std::integral_constant<int, 2>{});
        else
            go(FORM, W, S, G, std::integral_constant<int, 4>{});
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 8> eight;
    auto cells = [&](auto FORM) {
        if (f.shared)
            rows(FORM, two, four, one);
        else if (f.small)
            rows(FORM, two, one, one);
        else if (f.wide)
            rows(FORM, eight, one, two);
        else
            rows(FORM, eight, one, one);
    };
    if (a.d % FewPiece<T>::N == 0)
        cells(std::integral_constant<int, WHOLE>{});
    else if (a.d > FewPiece<T>::N)
        cells(std::integral_constant<int, ENDED>{});
    else
        cells(std::integral_constant<int, SHORT>{});
}
void launch_loss_few(int dtype, const FewArgs &a, bool backward, hipStream_t st)
{
    switch (dtype) {
    case VLQ_F32: return few<float>(dtype, a, backward, st);
    case VLQ_F16: return few<_Float16>(dtype, a, backward, st);
    default: return few<bf16_t>(dtype, a, backward, st);
    }
}

// A sum of fewer steps than this is a wave's alone
#define FEW_SHARED_STEPS 16
// Parts of a sum, so that the tiles fill the chip twice: of twelve steps at least, three a wave; of 32 where there are 64 tiles,
// as adding the parts up costs a launch.  (8 000 x 1 000 x 64 fp32 104 : 118 us with half as many, 500 x 500 x 500 bf16 52 : 58
// with parts of 8 steps, 1 000 x 128 x 64 fp32 40 : 66 without.)
int few_parts(int64_t rows, int64_t sum, int d)
{
    const int64_t steps = (sum + 15) / 16, tiles = (rows + 31) / 32 * ((d + 63) / 64);
    int64_t s = steps / (tiles >= 64 ? 32 : 12);
    if (s > 512 / tiles) s = 512 / tiles;
    if (s * rows * d * 4 > (256ll << 20)) s = (256ll << 20) / (rows * d * 4);
    if (s <= 1) return 1;
    const int64_t per = (steps + s - 1) / s;
    return (int)((steps + per - 1) / per); // (no part is empty)
}
FewSide few_side(int64_t rows, int64_t sum, int d, int parts, void *out, bool slab)
{
    FewSide s = {};
    const int steps = (int)((sum + 15) / 16);
    s.rows = (int)rows;
    s.sum = (int)sum;
    s.parts = parts;
    s.per = (steps + parts - 1) / parts;
    s.share = steps >= FEW_SHARED_STEPS;
    s.rtiles = (int)((rows + 31) / 32);
    s.dtiles = s.share ? (d + 63) / 64 : (d + 255) / 256;
    if (!out) s.dtiles = 1;
    s.blocks = s.rtiles * s.dtiles * parts;
    s.slab = slab;
    s.out = out;
    return s;
}

template <typename T>
static void few_grads(const FewArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(a.dx.blocks + a.dc.blocks));
    if (a.d >= 4)
        hipLaunchKernelGGL((k_loss_few_grads<T, true>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((k_loss_few_grads<T, false>), grid, dim3(256), 0, st, a);
}
void launch_loss_few_grads(int dtype, const FewArgs &a, hipStream_t st)
{
    switch (dtype) {
    case VLQ_F32: return few_grads<float>(a, st);
    case VLQ_F16: return few_grads<_Float16>(a, st);
    default: return few_grads<bf16_t>(a, st);
    }
}
