// Clipping by the global norm: n = sqrt(sum g^2) over all gradients, g = min(1, max_norm / (n + 1e-6)) g.
//
// Two passes over the gradients, which is what the definition needs: one for the sum, one for the product. The tensors are cut into
// chunks of CHUNK entries, and every workgroup takes a contiguous range of the chunks of all tensors, so that many small
// tensors and a few large ones fill the chip alike. Squares are added in 64 bits (no overflow at any fp32 value, nor in the factor, where the norm itself is beyond fp32;
// the adders keep up with the memory four times over), each workgroup's sum goes to a place of its own and the second pass adds these in a
// fixed order in every workgroup: the same bits every time, without atomics or a launch in between. The second pass walks its range
// backwards: what the first one read last is what the caches still hold.
//
// Bound by the memory: 5.2 GB of fp32 take 2840 us (sum 760, 6.9 TB/s; product 2050, 5.1); 22 MB, which stay in the caches, 18.6 us in two launches.
//
// Compiled with NaNs honoured: a gradient that is not finite has to show in the norm.
#include <algorithm>

#include "common.h"

namespace maxsim {

constexpr int CLIP_TENSORS = 110; // that fit the arguments of a launch (4 KB; 100 tensors of 1000 entries: 16.9 us, by way of the table in memory 19.3)

struct ClipTensors {
    const void *g[CLIP_TENSORS];
    void *out[CLIP_TENSORS];
    int64_t numel[CLIP_TENSORS];
    int64_t chunk[CLIP_TENSORS]; // first chunk of the tensor among those of all
    int32_t dtype[CLIP_TENSORS];
};
// The same in memory, for any number of tensors
struct ClipTable {
    const void **g;
    void **out;
    int64_t *numel, *chunk;
    int32_t *dtype;
};

namespace {

constexpr int WG = 256;
constexpr int CHUNK = 2048;
constexpr int MAX_WG = 1536; // six to a compute unit, all resident at a time (5.2 GB: 2850 us; eight 2900, four 3120; 22 MB take 18.6 with four to eight)
// Gradients of so many bytes do not stay in the caches (256 MB before the memory) until the second pass: they are moved past them.
// 24 layers of 2048 in fp32 (5.2 GB): 3030 us without the hint, 2900 with it; 6 layers of 384 (22 MB): 18.6 and 21.4.
constexpr int64_t STREAM_BYTES = int64_t(256) << 20;

template <class T> __device__ __forceinline__ double to_double(T x) { return (double)(float)x; }

// f(values of 16 bytes as floats, ...) over the entries [0, n) of a chunk; entries may lie at any address that is a multiple of their size
template <class T> struct Vec {
    static constexpr int V = 16 / sizeof(T);
    T x[V];
};
// 16 bytes at any address that is a multiple of the entries' size; ONCE: that the caches need not keep
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
template <bool ONCE, class T> __device__ __forceinline__ Vec<T> load_vec(const T *p)
{
    const u32x4 *at = reinterpret_cast<const u32x4 *>(p);
    return __builtin_bit_cast(Vec<T>, ONCE ? __builtin_nontemporal_load(at) : *at);
}
template <bool ONCE, class T> __device__ __forceinline__ void store_vec(T *p, const Vec<T> &r)
{
    u32x4 *at = reinterpret_cast<u32x4 *>(p);
    if constexpr (ONCE)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), at);
    else
        *at = __builtin_bit_cast(u32x4, r);
}

template <bool ONCE, class T> __device__ __forceinline__ double chunk_squares(const T *g, int n)
{
    constexpr int V = Vec<T>::V, STEPS = CHUNK / (WG * V);
    double sum = 0.0;
    if (n == CHUNK) {
        Vec<T> x[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            x[s] = load_vec<ONCE>(g + (s * WG + threadIdx.x) * V);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double v = to_double(x[s].x[i]);
                sum = __builtin_fma(v, v, sum);
            }
    } else {
        for (int e = threadIdx.x; e < n; e += WG) {
            const double v = to_double(g[e]);
            sum = __builtin_fma(v, v, sum);
        }
    }
    return sum;
}
template <bool ONCE, class T> __device__ __forceinline__ void chunk_scaled(const T *g, T *out, int n, float by, float more)
{
    constexpr int V = Vec<T>::V, STEPS = CHUNK / (WG * V);
    if (n == CHUNK) {
        Vec<T> x[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            x[s] = load_vec<ONCE>(g + (s * WG + threadIdx.x) * V);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                x[s].x[i] = (T)((float)x[s].x[i] * by * more);
            store_vec<ONCE>(out + (s * WG + threadIdx.x) * V, x[s]);
        }
    } else {
        for (int e = threadIdx.x; e < n; e += WG)
            out[e] = (T)((float)g[e] * by * more);
    }
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int m = 32; m; m >>= 1)
        x += __shfl_xor(x, m, 64);
    return x;
}
__device__ __forceinline__ double wg_sum(double x) // the same in every thread
{
    __shared__ double part[WG / 64];
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < WG / 64; ++w)
        s += part[w];
    return s;
}

// The tensor that a chunk lies in: the last one whose first chunk is not after it (a tensor without entries shares its first chunk with
// the next one and is never that). 64 probes a step, one per lane, since a step is a round trip to memory.
template <class Tensors> __device__ __forceinline__ int find_tensor(const Tensors &t, int n, int64_t chunk)
{
    int lo = 0, end = n; // tensors before lo start at or before the chunk, those from end on after it
    while (lo < end) {
        const int step = (end - lo + 63) >> 6, at = lo + ((threadIdx.x & 63) + 1) * step - 1;
        const uint64_t below = __builtin_amdgcn_ballot_w64(at < end && t.chunk[at < end ? at : 0] <= chunk);
        lo += __builtin_popcountll(below) * step;
        end = min(end, lo + step - 1);
    }
    return __builtin_amdgcn_readfirstlane(lo) - 1;
}

template <bool ONCE, class Tensors> __global__ void __launch_bounds__(WG) clip_sum_kernel(Tensors t, int n, int64_t chunks, double *part)
{
    const int64_t c0 = chunks * blockIdx.x / gridDim.x, c1 = chunks * (blockIdx.x + 1) / gridDim.x;
    int i = find_tensor(t, n, c0);
    double sum = 0.0;
    for (int64_t c = c0; c < c1; ++c) {
        while (i + 1 < n && t.chunk[i + 1] <= c)
            ++i;
        const int64_t e = (c - t.chunk[i]) * CHUNK, left = t.numel[i] - e;
        const int m = left < CHUNK ? (int)left : CHUNK;
        if (t.dtype[i] == MAXSIM_F32)
            sum += chunk_squares<ONCE>(static_cast<const float *>(t.g[i]) + e, m);
        else if (t.dtype[i] == MAXSIM_F16)
            sum += chunk_squares<ONCE>(static_cast<const _Float16 *>(t.g[i]) + e, m);
        else
            sum += chunk_squares<ONCE>(static_cast<const __bf16 *>(t.g[i]) + e, m);
    }
    sum = wg_sum(sum);
    if (threadIdx.x == 0)
        part[blockIdx.x] = sum;
}

template <bool ONCE, class Tensors> __global__ void __launch_bounds__(WG) clip_scale_kernel(Tensors t, int n, int64_t chunks, const double *part, int parts, float max_norm, float *norm)
{
    double sum = 0.0;
    for (int x = threadIdx.x; x < parts; x += WG)
        sum += part[x];
    const double total = sqrt(wg_sum(sum));
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *norm = (float)total;
    // The factor in 64 bits, since the norm of fp32 numbers need not be one; one that fp32 holds badly or not at all as a product of two
    const double by0 = (double)max_norm / (total + 1e-6);
    const bool small = by0 < 0x1p-100;
    const float by = small ? 0x1p-100f : (float)(by0 < 1.0 || by0 != by0 ? by0 : 1.0), more = small ? (float)(by0 * 0x1p100) : 1.0f;
    const int64_t c0 = chunks * blockIdx.x / gridDim.x, c1 = chunks * (blockIdx.x + 1) / gridDim.x;
    if (c0 >= c1)
        return;
    int i = find_tensor(t, n, c1 - 1);
    for (int64_t c = c1 - 1; c >= c0; --c) {
        while (t.chunk[i] > c)
            --i;
        if (by == 1.0f && t.out[i] == t.g[i]) // nothing changes
            continue;
        const int64_t e = (c - t.chunk[i]) * CHUNK, left = t.numel[i] - e;
        const int m = left < CHUNK ? (int)left : CHUNK;
        if (t.dtype[i] == MAXSIM_F32)
            chunk_scaled<ONCE>(static_cast<const float *>(t.g[i]) + e, static_cast<float *>(t.out[i]) + e, m, by, more);
        else if (t.dtype[i] == MAXSIM_F16)
            chunk_scaled<ONCE>(static_cast<const _Float16 *>(t.g[i]) + e, static_cast<_Float16 *>(t.out[i]) + e, m, by, more);
        else
            chunk_scaled<ONCE>(static_cast<const __bf16 *>(t.g[i]) + e, static_cast<__bf16 *>(t.out[i]) + e, m, by, more);
    }
}

// A part of the table from the launch's arguments into memory
__global__ void __launch_bounds__(128) clip_table_kernel(ClipTensors t, int n, ClipTable to, int first)
{
    const int i = threadIdx.x;
    if (i < n) {
        to.g[first + i] = t.g[i];
        to.out[first + i] = t.out[i];
        to.numel[first + i] = t.numel[i];
        to.chunk[first + i] = t.chunk[i];
        to.dtype[first + i] = t.dtype[i];
    }
}

} // namespace

int64_t clip_workspace(int n) { return MAX_WG * 8 + (n > CLIP_TENSORS ? (int64_t)n * 36 : 0); }

hipError_t clip_launch(const void *const *g, void *const *out, const int64_t *numel, const int32_t *dtype, int n, float max_norm, float *norm, void *workspace, hipStream_t stream)
{
    double *part = static_cast<double *>(workspace);
    char *at = reinterpret_cast<char *>(part + MAX_WG);
    ClipTable table = {reinterpret_cast<const void **>(at), reinterpret_cast<void **>(at + 8 * (int64_t)n), reinterpret_cast<int64_t *>(at + 16 * (int64_t)n),
                       reinterpret_cast<int64_t *>(at + 24 * (int64_t)n), reinterpret_cast<int32_t *>(at + 32 * (int64_t)n)};
    int64_t chunks = 0, bytes = 0;
    ClipTensors t = {};
    int held = 0;
    for (int i = 0; i < n; ++i) {
        if (held == CLIP_TENSORS) {
            clip_table_kernel<<<1, 128, 0, stream>>>(t, held, table, i - held);
            held = 0;
        }
        t.g[held] = g[i];
        t.out[held] = out[i];
        t.numel[held] = numel[i];
        t.chunk[held] = chunks;
        t.dtype[held] = dtype[i];
        ++held;
        chunks += (numel[i] + CHUNK - 1) / CHUNK;
        bytes += numel[i] * (dtype[i] == MAXSIM_F32 ? 4 : 2);
    }
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(chunks, MAX_WG));
    if (n > CLIP_TENSORS)
        clip_table_kernel<<<1, 128, 0, stream>>>(t, held, table, n - held);
    auto go = [&](auto once, auto tensors) {
        constexpr bool ONCE = decltype(once)::value;
        clip_sum_kernel<ONCE><<<grid, WG, 0, stream>>>(tensors, n, chunks, part);
        clip_scale_kernel<ONCE><<<grid, WG, 0, stream>>>(tensors, n, chunks, part, (int)grid, max_norm, norm);
    };
    auto choose = [&](auto tensors) { bytes >= STREAM_BYTES ? go(std::true_type{}, tensors) : go(std::false_type{}, tensors); };
    n <= CLIP_TENSORS ? choose(t) : choose(table);
    return hipGetLastError();
}

} // namespace maxsim
