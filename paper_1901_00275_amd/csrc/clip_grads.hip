// The norm of all gradients together, and the gradients brought to at most a given norm:
//     norm = sqrt(sum g^2),  out = g min(1, max_norm / norm).
// Bound by memory: two launches, each reads the gradients once, the second writes.  Tensors are cut into chunks, a workgroup
// each; squares are summed in fp64 (they neither overflow nor vanish, and the order of the chunks' sums is fixed).  The second
// launch takes the chunks from the last to the first: what the first launch read last is still in the 256 MB cache.  What comes
// before the last CLIP_STAY bytes is read past the caches, in both launches: 800 MB of bf16 488 -> 464 us (8.5 MB past the
// caches cost 11.4 instead of 10.2): 5.3 TB/s, where a copy of this size has 4.7.
// The tensors' addresses travel in the kernels' arguments, so nothing on the host has to outlive the call.
#include "learn.h"

#include <type_traits>

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16_t;

#define CLIP_NT 256
#define CLIP_TENSORS 140   // tensors of a launch (their table is part of the arguments, which end at 4 KB)
#define CLIP_PARTS 8192    // up to so many sums are added up by every workgroup of the second launch
#define CLIP_CHUNKS 4096   // chunks that the gradients are cut into, about
#define CLIP_LEAST 8192    // values of a chunk at least
#define CLIP_STAY (160 << 20) // bytes at the end that are left in the cache between the launches

struct ClipTable {
    const void *in[CLIP_TENSORS];
    void *out[CLIP_TENSORS];
    int64_t count[CLIP_TENSORS]; // values, times four, plus the type
    int first[CLIP_TENSORS];     // a tensor's first chunk within the launch
    int tensors, chunks;
    int64_t chunk; // values of a chunk
    int stay;      // the chunks from here on stay in the cache
};
static_assert(sizeof(ClipTable) + 64 <= 4096, "the arguments of a launch");

// the tensor of chunk b
__device__ __forceinline__ int find_tensor(const ClipTable &a, int b)
{
    int lo = 0, hi = a.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.first[mid] <= b)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// sum over the workgroup in a fixed order, in every thread
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double s[CLIP_NT / 64];
    v = wave_sum_f64(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
#pragma unroll
    for (int w = 0; w < CLIP_NT / 64; ++w) v += s[w];
    __syncthreads();
    return v;
}

// 16 bytes at a value's address: the memory takes them at any (120 M bf16 values off 16 bytes 335 us value by value, 145 so, 122 on them)
template <typename T>
struct Sixteen {
    static constexpr int N = 16 / sizeof(T);
    typedef uint32_t At __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
};
template <bool STAY, typename T>
__device__ __forceinline__ u32x4 load16(const T *p)
{
    using At = typename Sixteen<T>::At;
    return STAY ? *(const At *)p : __builtin_nontemporal_load((const At *)p);
}

template <typename T, bool STAY>
__device__ __forceinline__ double squares(const T *p, int64_t count)
{
    constexpr int N = 16 / sizeof(T);
    double s = 0.;
    int64_t i = threadIdx.x;
    const int64_t whole = count / N;
    double s2[4] = {};
    for (; i + 3 * CLIP_NT < whole; i += 4 * CLIP_NT) {
        T v[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u) *(u32x4 *)v[u] = load16<STAY>(p + (i + u * CLIP_NT) * N);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) s2[u] = fma((double)(float)v[u][e], (double)(float)v[u][e], s2[u]);
    }
    for (; i < whole; i += CLIP_NT) {
        T v[N];
        *(u32x4 *)v = load16<STAY>(p + i * N);
#pragma unroll
        for (int e = 0; e < N; ++e) s = fma((double)(float)v[e], (double)(float)v[e], s);
    }
    s += (s2[0] + s2[1]) + (s2[2] + s2[3]);
    i = whole * N + threadIdx.x;
    for (; i < count; i += CLIP_NT) s = fma((double)(float)p[i], (double)(float)p[i], s);
    return s;
}

// f(type, STAY) of a chunk
template <typename F>
__device__ __forceinline__ void of_type(int dtype, bool stay, F &&f)
{
    auto typed = [&](auto s) {
        if (dtype == VLQ_F32)
            f(0.f, s);
        else if (dtype == VLQ_F16)
            f((_Float16)0.f, s);
        else
            f((bf16_t)0.f, s);
    };
    if (stay)
        typed(std::true_type{});
    else
        typed(std::false_type{});
}

__global__ __launch_bounds__(CLIP_NT) void k_grad_squares(ClipTable a, double *part)
{
    const int b = blockIdx.x, t = find_tensor(a, b);
    const void *in = a.in[t];
    const int dtype = (int)(a.count[t] & 3);
    const int64_t i0 = (int64_t)(b - a.first[t]) * a.chunk, count = min(a.chunk, (a.count[t] >> 2) - i0);
    double s = 0.;
    of_type(dtype, b >= a.stay, [&](auto type, auto stay) {
        using T = decltype(type);
        s = squares<T, decltype(stay)::value>((const T *)in + i0, count);
    });
    s = block_sum(s);
    if (threadIdx.x == 0) part[b] = s;
}

__device__ __forceinline__ double sum_parts(const double *part, int parts)
{
    double s = 0.;
    for (int i = threadIdx.x; i < parts; i += CLIP_NT) s += part[i];
    return block_sum(s);
}

// The norm as it is returned: one that is finite stays so (infinity says that the values were left as they are)
__device__ __forceinline__ float norm_out(double n) { return n < INFINITY ? fminf((float)n, __FLT_MAX__) : (float)n; }

// many parts become one, and the norm of no tensors
__global__ __launch_bounds__(CLIP_NT) void k_grad_norm(const double *part, int parts, double *sum, float *norm)
{
    const double s = sum_parts(part, parts);
    if (threadIdx.x != 0) return;
    if (sum) *sum = s;
    if (norm) *norm = norm_out(sqrt(s));
}

// (the factor is fp64: 1e-45 / 1e38 is no fp32 number, and the launch waits for memory either way)
template <typename T, bool STAY>
__device__ __forceinline__ void scale_values(const T *p, T *o, int64_t count, double f)
{
    constexpr int N = 16 / sizeof(T);
    int64_t i = threadIdx.x;
    const bool past = (uintptr_t)o % 16 == 0; // (parts of a cache's line are put together in the cache)
    using At = typename Sixteen<T>::At;
    const int64_t whole = count / N;
    for (; i < whole; i += 4 * CLIP_NT) {
        T v[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * CLIP_NT < whole) *(u32x4 *)v[u] = load16<STAY>(p + (i + u * CLIP_NT) * N);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * CLIP_NT < whole) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[u][e] = (T)(float)((float)v[u][e] * f);
                u32x4 *to = (u32x4 *)(o + (i + u * CLIP_NT) * N);
                if (past)
                    __builtin_nontemporal_store(*(u32x4 *)v[u], to);
                else
                    *(At *)to = *(u32x4 *)v[u];
            }
    }
    i = whole * N + threadIdx.x;
    for (; i < count; i += CLIP_NT) o[i] = (T)(float)((float)p[i] * f);
}

__global__ __launch_bounds__(CLIP_NT) void k_grad_scale(ClipTable a, const double *part, int parts, float max_norm, float *norm)
{
    const double n = sqrt(sum_parts(part, parts));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = norm_out(n);
    // (a norm that is not finite leaves the gradients as they are)
    const double f = n > (double)max_norm && n < INFINITY ? (double)max_norm / n : 1.;
    const int b = a.chunks - 1 - blockIdx.x, t = find_tensor(a, b);
    const void *in = a.in[t];
    void *out = a.out[t];
    if (f == 1. && in == out) return;
    const int dtype = (int)(a.count[t] & 3);
    const int64_t i0 = (int64_t)(b - a.first[t]) * a.chunk, count = min(a.chunk, (a.count[t] >> 2) - i0);
    of_type(dtype, b >= a.stay, [&](auto type, auto stay) {
        using T = decltype(type);
        scale_values<T, decltype(stay)::value>((const T *)in + i0, (T *)out + i0, count, f);
    });
}

static int64_t clip_chunk(int tensors, const int64_t *counts)
{
    int64_t total = 0;
    for (int i = 0; i < tensors; ++i) total += counts[i];
    const int64_t c = (total / CLIP_CHUNKS + 2047) / 2048 * 2048;
    return c < CLIP_LEAST ? CLIP_LEAST : c;
}

static int64_t clip_parts(int tensors, const int64_t *counts)
{
    const int64_t chunk = clip_chunk(tensors, counts);
    int64_t parts = 0;
    for (int i = 0; i < tensors; ++i) parts += (counts[i] + chunk - 1) / chunk;
    return parts;
}

size_t clip_workspace(int tensors, const int64_t *counts) { return (size_t)(clip_parts(tensors, counts) + 32) * 8; }

int launch_clip_grads(int tensors, const int *dtypes, const int64_t *counts, const void *const *in, float max_norm,
                      void *const *out, float *norm, void *ws, hipStream_t st)
{
    const int64_t chunk = clip_chunk(tensors, counts), parts = clip_parts(tensors, counts);
    double *sum = (double *)ws, *part = sum + 32;
    int64_t stay = parts;
    for (int64_t t = tensors - 1, left = CLIP_STAY; t >= 0 && left > 0; --t) {
        const int64_t chunks = (counts[t] + chunk - 1) / chunk, fit = left / (chunk * type_bytes(dtypes[t]));
        stay -= chunks < fit ? chunks : fit;
        left = chunks < fit ? left - chunks * chunk * type_bytes(dtypes[t]) : 0;
    }
    // one launch per table of tensors; back: from the last table to the first
    auto tables = [&](bool back, auto &&launch) {
        int64_t before = back ? parts : 0;
        for (int at = back ? tensors - 1 : 0; back ? at >= 0 : at < tensors;) {
            ClipTable a;
            a.tensors = a.chunks = 0;
            a.chunk = chunk;
            const int step = back ? -1 : 1;
            int picked[CLIP_TENSORS];
            for (; a.tensors < CLIP_TENSORS && (back ? at >= 0 : at < tensors); at += step) {
                if (counts[at] == 0) continue;
                picked[a.tensors++] = at;
            }
            if (a.tensors == 0) break;
            int first = 0;
            for (int i = 0; i < a.tensors; ++i) {
                const int t = picked[back ? a.tensors - 1 - i : i];
                a.in[i] = in[t];
                a.out[i] = out ? out[t] : nullptr;
                a.count[i] = counts[t] * 4 + dtypes[t];
                a.first[i] = first;
                first += (int)((counts[t] + chunk - 1) / chunk);
            }
            a.chunks = first;
            if (back) before -= first;
            a.stay = (int)(stay > before ? stay - before : 0);
            launch(a, before);
            if (!back) before += first;
        }
    };
    tables(false, [&](const ClipTable &a, int64_t before) {
        hipLaunchKernelGGL(k_grad_squares, dim3((unsigned)a.chunks), dim3(CLIP_NT), 0, st, a, part + before);
    });
    const double *from = part;
    int count = (int)parts;
    if (parts == 0 || parts > CLIP_PARTS || !out) {
        hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(CLIP_NT), 0, st, part, count, sum, norm);
        from = sum;
        count = 1;
        norm = nullptr;
    }
    if (out)
        tables(true, [&](const ClipTable &a, int64_t) {
            hipLaunchKernelGGL(k_grad_scale, dim3((unsigned)a.chunks), dim3(CLIP_NT), 0, st, a, from, count, max_norm, norm);
            norm = nullptr;
        });
    return (int)hipGetLastError();
}
