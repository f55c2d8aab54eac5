// The softmax loss and its gradients for up to 128 dimensions, 256 of 16-bit values: no piece of the n x k probabilities leaves the registers.
//
// A workgroup keeps 128 rows (256 of up to 96 16-bit values) of one matrix, of x for dx and of c for dc: their fragments and their gradient's
// sums stay in registers while tiles of 32 rows of the other matrix pass through LDS, its image and the image of its
// columns.  Per tile a wave multiplies 32 rows of the other matrix with its own (S = R Q^T), turns S into P with the row's
// maximum and sum, and multiplies the other matrix's columns with P (dQ^T += R^T P).  S has four consecutive r of one q in a lane; P as the
// second operand wants eight: those of both 16-row halves are taken together, which is an order of the 32 indices that the
// columns' image is written in.
//
// Each side computes the logits, 8 n k d operations together where the wide form takes 6 n k d; but that one writes P twice
// and reads it twice, 16 bytes a pair, which bounds it at so few dimensions.
//
// Bound by the matrix cores and the arithmetic between their products: 4 095 x 65 536 x 128 fp32 (three products each) 740 us,
// 1.11 PFLOP/s, the matrix cores busy 60 % of the time at the 1.87 GHz that the card then holds; forward 180 us, 1.15.  The
// products and the arithmetic of two tiles woven into each other by hand gained nothing over two workgroups a compute unit
// with the products' waves preferred.
// 16-bit values (one product for the logits, two with the parts of P): 8 192 x 32 000 x 256 bf16, gradients 740 us (1.09 PFLOP/s), forward
// 136 (0.98): there the fragments' reads from LDS take as long as the products that they feed.  A step of x 129 567.
// Few rows (256 x 16 384 x 96 fp32, 20 us): 256 workgroups of eight tiles each, whose steps follow one another.
#include "loss_image.h"

#define NARROW_NT 256
// What a workgroup does: the gradient of rows, that of centroids, or forward the maxima and sums of rows
enum { ROWS, CENTROIDS, STATS };

template <typename T, int DU, int DO>
__device__ __forceinline__ void narrow(const NarrowArgs &a, const NarrowSide &s, int b, u32x4 *lds)
{
    constexpr int NP = sizeof(T) == 4 ? 2 : 1, Q = narrow_rows(NP, DU), QB = Q / 64, DB = 2 * DU;
    constexpr bool CENT = DO == CENTROIDS;
    constexpr int CHUNKS = (DO == STATS ? 2 : 4) * DU * NP; // KB of a tile: rows, then columns
    constexpr int STAGE = (CHUNKS + 2) * 64;        // and two KB for the rows' numbers, in 16-byte pieces
    const int tid = threadIdx.x, lane = tid & 63, l = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int split = b / s.qblocks, q0 = (b - split * s.qblocks) * Q + wave * 16 * QB;
    const int t0 = split * s.per, t1 = min(s.tiles, t0 + s.per);

    auto copy16 = [&](const void *src, int bytes, u32x4 *dst) { // 16 bytes a lane, zeros behind `bytes`
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)src, 0, bytes, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)dst, 16, lane * 16, 0, 0, 0);
    };
    auto copy4 = [&](const void *src, int bytes, u32x4 *dst) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)src, 0, bytes, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)dst, 4, lane * 4, 0, 0, 0);
    };
    auto copy_tile = [&](int t) {
        u32x4 *dst = lds + (t & 1) * STAGE;
        const u32x4 *rows = s.r + (int64_t)(t >> 2) * a.units * NP * PAGE + (t & 3) * 128;
        const u32x4 *cols = s.rt + (int64_t)t * NP * PAGE;
#pragma unroll
        for (int e = 0; e < (CHUNKS + 3) / 4; ++e) {
            const int c = e * 4 + wave; // (rows: page c / 2, group c % 2; columns: part, then group of 16 dimensions)
            if (CHUNKS % 4 && c >= CHUNKS) break;
            const int cc = c - 2 * DU * NP, dim = cc % DB; // (group of 16 dimensions: eight a block of the columns' image)
            const u32x4 *src = c < 2 * DU * NP ? rows + (c >> 1) * PAGE + (c & 1) * 64
                                               : cols + ((int64_t)(dim >> 3) * s.tiles * NP + cc / DB) * PAGE + (dim & 7) * 64;
            copy16(src, 1024, dst + c * 64);
        }
        u32x4 *num = dst + CHUNKS * 64;
        if (CENT) { // {factor, maximum, -, factor of P} [32], labels [32], the label's share [32]: zeros fill a wave's copy up
            if (wave == 0) copy16(a.row + t * 32, 512, num);
            if (wave == 1) copy4(a.lab + t * 32, 128, num + 64);
            if (wave == 2) copy4(a.gn + t * 32, 128, num + 80);
        } else if (wave == 3) {
            copy4(a.bias2 + t * 32, 128, num);
        }
    };

    half8 qf[DU][NP][QB];
#pragma unroll
    for (int u = 0; u < DU; ++u)
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int j = 0; j < QB; ++j)
                qf[u][p][j] = __builtin_bit_cast(
                    half8, s.q[(((int64_t)(q0 >> 7) * a.units + u) * NP + p) * PAGE + (((q0 >> 4) & 7) + j) * 64 + lane]);
    float f[QB], m[QB], z[QB], db[QB]; // x: factor, maximum, factor of P; c: factor, bias
    int lab[QB];
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const int q = q0 + 16 * j + l;
        db[j] = 0.f;
        if (CENT) {
            f[j] = a.cinv[q >> 4];
            m[j] = a.bias2[q];
        } else {
            const f32x4 v = a.row[q];
            f[j] = v[0];
            m[j] = DO == STATS ? -INFINITY : v[1];
            z[j] = DO == STATS ? 0.f : v[2];
            lab[j] = a.lab[q];
        }
    }
    f32x4 acc[DB][QB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < QB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    copy_tile(t0);
    float cinv[2], next[2]; // inverse scales of this tile and the next one
#pragma unroll
    for (int i = 0; i < 2; ++i) next[i] = CENT ? 0.f : a.cinv[t0 * 2 + i];
    for (int t = t0; t < t1; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads(); // (this tile has arrived, and nobody reads the other buffer any more)
        if (t + 1 < t1) copy_tile(t + 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            cinv[i] = next[i];
            if (!CENT) next[i] = a.cinv[min(t + 1, t1 - 1) * 2 + i];
        }
        const u32x4 *st = lds + (t & 1) * STAGE;
        const float *num = (const float *)(st + CHUNKS * 64);
        f32x4 S[2][QB];
        __builtin_amdgcn_s_setprio(1); // (the products go first, another wave's arithmetic takes the slots between them)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < QB; ++j) S[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < DU; ++u) {
            half8 r[NP][2];
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) r[p][i] = __builtin_bit_cast(half8, st[((u * NP + p) * 2 + i) * 64 + lane]);
            if (NP == 2) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < QB; ++j) S[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[0][i], qf[u][NP - 1][j], S[i][j], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < QB; ++j) S[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[NP - 1][i], qf[u][0][j], S[i][j], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < QB; ++j) S[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[0][i], qf[u][0][j], S[i][j], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (DO == STATS) {
            // a lane keeps the maximum and the sum of the logits that it has met of each of its rows
            const int base = 32 * t + 4 * g;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 b2 = *(const f32x4 *)(num + 16 * i + 4 * g);
                const float ci = cinv[i];
#pragma unroll
                for (int j = 0; j < QB; ++j) {
                    const float fj = f[j] * ci;
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[i][j][r] = fmaf(S[i][j][r], fj, b2[r]);
                }
            }
            bool any = false;
#pragma unroll
            for (int j = 0; j < QB; ++j) {
                float top = m[j];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, S[i][j][r]);
                const float at = top == -INFINITY ? 0.f : top; // (all masked so far: every term is zero)
                z[j] *= __builtin_amdgcn_exp2f(m[j] - at);
                m[j] = top;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[j] += __builtin_amdgcn_exp2f(S[i][j][r] - at);
                any |= (uint32_t)(lab[j] - 32 * t) < 32u;
            }
            if (__any(any)) {
#pragma unroll
                for (int j = 0; j < QB; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (lab[j] == base + 16 * i + r) a.mine[q0 + 16 * j + l] = S[i][j][r];
            }
            continue;
        }
        // P, in units of 2^15, from the logits rounded as they were forward
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (CENT) {
                f32x4 row[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) row[r] = *(const f32x4 *)(num + (16 * i + 4 * g + r) * 4);
#pragma unroll
                for (int j = 0; j < QB; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        S[i][j][r] = __builtin_amdgcn_exp2f(fmaf(S[i][j][r], row[r][0] * f[j], m[j]) - row[r][1]) * row[r][3];
            } else {
                const f32x4 b2 = *(const f32x4 *)(num + 16 * i + 4 * g);
                const float ci = cinv[i];
#pragma unroll
                for (int j = 0; j < QB; ++j) {
                    const float fj = f[j] * ci;
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[i][j][r] = __builtin_amdgcn_exp2f(fmaf(S[i][j][r], fj, b2[r]) - m[j]) * z[j];
                }
            }
        }
        // the labels' own
        if (CENT) {
            const int *rl = (const int *)(num + 256);
            if (__any((uint32_t)(rl[lane & 31] - q0) < 16u * QB)) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = 16 * i + 4 * g + r, of = rl[at] - q0 - l;
                        const float gn = num[320 + at];
#pragma unroll
                        for (int j = 0; j < QB; ++j)
                            if (of == 16 * j) S[i][j][r] -= gn;
                    }
            }
        } else {
            bool any = false;
#pragma unroll
            for (int j = 0; j < QB; ++j) any |= (uint32_t)(lab[j] - 32 * t) < 32u;
            if (__any(any)) {
#pragma unroll
                for (int j = 0; j < QB; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (lab[j] - 32 * t == 16 * i + 4 * g + r) S[i][j][r] -= P_ONE;
            }
        }
        half8 P[P_PARTS][QB];
#pragma unroll
        for (int j = 0; j < QB; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = S[i][j][r];
                    _Float16 hi, lo;
                    halves<P_PARTS>(v, hi, lo);
                    P[0][j][4 * i + r] = hi;
                    P[1][j][4 * i + r] = lo;
                    if (CENT) db[j] += v;
                }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            half8 c[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) c[p] = __builtin_bit_cast(half8, st[(2 * DU * NP + p * DB + i) * 64 + lane]);
#pragma unroll
            for (int j = 0; j < QB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[0], P[1][j], acc[i][j], 0, 0, 0);
            if (NP == 2)
#pragma unroll
                for (int j = 0; j < QB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[NP - 1], P[0][j], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < QB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[0], P[0][j], acc[i][j], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
    }

    if constexpr (DO == STATS) {
#pragma unroll
        for (int j = 0; j < QB; ++j) {
            float2 v = make_float2(m[j], z[j]);
            v = join(v, make_float2(__shfl_xor(v.x, 16, 64), __shfl_xor(v.y, 16, 64)));
            v = join(v, make_float2(__shfl_xor(v.x, 32, 64), __shfl_xor(v.y, 32, 64)));
            if (g == 0) a.part[(int64_t)split * a.npad + q0 + 16 * j + l] = v;
        }
        return;
    }
    const float unit = grad_unit(CENT ? a.hdr->xinv : a.hdr->cinv), top = a.hdr->top;
    float *slab = (float *)s.out + (int64_t)split * s.rows * a.d;
#pragma unroll
    for (int j = 0; j < QB; ++j) {
        const int q = q0 + 16 * j + l;
        if (CENT && a.dbpart) {
            float v = db[j];
            v += __shfl_xor(v, 16, 64);
            v += __shfl_xor(v, 32, 64);
            if (g == 0) a.dbpart[(int64_t)split * a.kpad + q] = v;
        }
        if (q >= s.rows || !s.out) continue;
        const float w = CENT ? 1.f : a.gn[q] * (1.f / P_ONE);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            const int dim = 16 * i + 4 * g;
            if (dim >= a.d) continue;
            if (s.mode == 0)
                store4((T *)s.out + (int64_t)q * a.d + dim, acc[i][j] * unit * w * a.scale * top, a.d - dim, s.vec);
            else
                store4(slab + (int64_t)q * a.d + dim, acc[i][j] * unit * w, a.d - dim, s.vec);
        }
    }
}

template <typename T, int DU>
__global__ __launch_bounds__(NARROW_NT, 2) void k_loss_narrow(NarrowArgs a)
{
    extern __shared__ u32x4 lds[];
    if ((int)blockIdx.x < a.nx)
        narrow<T, DU, ROWS>(a, a.x, blockIdx.x, lds);
    else
        narrow<T, DU, CENTROIDS>(a, a.c, blockIdx.x - a.nx, lds);
}

template <typename T, int DU>
__global__ __launch_bounds__(NARROW_NT, 2) void k_loss_narrow_stats(NarrowArgs a)
{
    extern __shared__ u32x4 lds[];
    narrow<T, DU, STATS>(a, a.x, blockIdx.x, lds);
}

template <typename T, bool GRADS>
static int narrow_units(const NarrowArgs &a, hipStream_t st)
{
    auto go = [&](auto units) -> int {
        constexpr int DU = decltype(units)::value, KB = (GRADS ? 4 : 2) * DU * (sizeof(T) == 4 ? 2 : 1) + 2;
        const auto kern = GRADS ? k_loss_narrow<T, DU> : k_loss_narrow_stats<T, DU>;
        constexpr size_t bytes = 2 * KB * 1024;
        if (bytes > 49152) { // (48 KB of dynamic LDS need no asking)
            const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e != hipSuccess) return (int)e;
        }
        const int blocks = GRADS ? a.nx + a.c.qblocks * a.c.splits : a.x.qblocks * a.x.splits;
        hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(NARROW_NT), bytes, st, a);
        return 0;
    };
    if constexpr (sizeof(T) == 2)
        switch (a.units) {
        case 5: return go(std::integral_constant<int, 5>{});
        case 6: return go(std::integral_constant<int, 6>{});
        case 7: return go(std::integral_constant<int, 7>{});
        case 8: return go(std::integral_constant<int, 8>{});
        }
    switch (a.units) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    default: return go(std::integral_constant<int, 4>{});
    }
}

int launch_loss_narrow_stats(int dtype, const NarrowArgs &a, hipStream_t st)
{
    switch (dtype) {
    case VLQ_F32: return narrow_units<float, false>(a, st);
    case VLQ_F16: return narrow_units<_Float16, false>(a, st);
    default: return narrow_units<bf16_t, false>(a, st);
    }
}

int launch_loss_narrow(int dtype, const NarrowArgs &a, hipStream_t st)
{
    switch (dtype) {
    case VLQ_F32: return narrow_units<float, true>(a, st);
    case VLQ_F16: return narrow_units<_Float16, true>(a, st);
    default: return narrow_units<bf16_t, true>(a, st);
    }
}
