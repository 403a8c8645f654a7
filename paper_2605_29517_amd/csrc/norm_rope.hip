// Norms of queries and keys with rotary positions in the same pass: for every head's row x of d entries, with the weights w of its kind,
//     r = 1 / sqrt(mean x^2 + eps),   h = x r w,   y = scale R(p f) h on the first `rot` entries and h on the rest,
// and the gradient: g = scale R(p f)^T dy (dy itself on the rest),
//     dx = r (g w - x r^2 mean(g w x)),   dw = sum over the rows of its kind of g x r.
//
// A group of lanes holds a row, each lane the same entries of every row it takes: pairs that turn together lie in one lane, which in the gradient
// also adds up its share of dw. dw leaves in one line for each workgroup and kind, joined by a second kernel in a fixed order: the same bits
// every time. The next row is on its way while one is worked on, all heads of a token share its angles, the weights are in LDS.
//
// Bound by the memory: 16384 tokens of 40 heads of 128, bf16 (336 MB), 59 us, 5.7 TB/s both ways; the gradient (503 MB) 111 us, of which dw's second kernel takes 6. 64 tokens of one
// step 5.2 us, the call.
#include <algorithm>

#include "rope.h"
#include "rows.h"

namespace maxsim {

struct NormTensor {
    char *p;
    int64_t token, head; // strides, bytes
};

struct NormParams {
    NormTensor X, Y, dX; // Y: the result, or the gradient that arrives
    const void *weight[2];
    float *dweight[2];
    int w_dtype;
    RopeAngles angles;
    int64_t tokens;
    int heads[2]; // queries first, then keys
    int d, rot;
    float eps, inv_d;
    int group;       // lanes of a row: a power of two
    int per_turn;    // tokens whose angles are in LDS at a time
    int64_t per_wg;  // tokens of a workgroup
    int64_t runs;    // of so many tokens
    Divisor by_heads[2]; // (in the forward direction the first one is for all heads)
    float *part;     // [runs][2][d]
};

namespace {

constexpr int WG = 256;
constexpr int MAX_WIDTH = 512;
constexpr int MAX_TABLE = 2048; // (token, pair) entries of a workgroup: 16 KB of LDS

// HALVES: a lane takes V pairs (i, i + rot / 2). NEIGHBOURS: V entries, pairs (2 i, 2 i + 1). The entries from rot on: V, or two V where there are pairs
// of pieces. ANY (V = 1): a pair or an entry at a time, wherever they lie.
enum NormPairs { HALVES, NEIGHBOURS, ANY, ANY_NEIGHBOURS };

__device__ __forceinline__ float weight_at(const void *w, int dtype, int i)
{
    if (!w)
        return 1.0f;
    if (dtype == MAXSIM_F32)
        return static_cast<const float *>(w)[i];
    if (dtype == MAXSIM_F16)
        return (float)static_cast<const _Float16 *>(w)[i];
    return (float)static_cast<const __bf16 *>(w)[i];
}

// The sum over groups of G lanes, a power of two; every lane gets it
__device__ __forceinline__ float group_sum(float x, int G)
{
    auto lane = [&](auto how) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(how)::value, 0xf, 0xf, true)); };
    if (G > 1)
        x += lane(std::integral_constant<int, 0xb1>{}); // the neighbour
    if (G > 2)
        x += lane(std::integral_constant<int, 0x4e>{}); // two away
    if (G > 4)
        x += lane(std::integral_constant<int, 0x141>{}); // mirrored in eight lanes: one of the other four
    if (G > 8)
        x += lane(std::integral_constant<int, 0x140>{}); // and in sixteen
    if (G > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (G > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// The sum over the groups of G lanes of a wavefront, lane by lane; every group gets it
__device__ __forceinline__ float rows_sum(float x, int G)
{
    auto turned = [&](auto how) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(how)::value, 0xf, 0xf, true)); };
    if (G <= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (G <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    // rotations within sixteen lanes
    if (G <= 8)
        x += turned(std::integral_constant<int, 0x128>{});
    if (G <= 4)
        x += turned(std::integral_constant<int, 0x124>{});
    if (G <= 2)
        x += turned(std::integral_constant<int, 0x122>{});
    if (G <= 1)
        x += turned(std::integral_constant<int, 0x121>{});
    return x;
}

// N: pieces of a lane. A piece is two times V entries (the second V of a plain one are not there), or V with NEIGHBOURS. The gradient with HALVES and V = 8 is held to 128 registers, with
// five of them in scratch (24 bytes a lane): 16384 tokens of 40 heads of 128 113 us, with 135 registers, three wavefronts to a SIMD and no scratch 117; 3850 tokens of 20 heads 29 and 33. All
// gradients keep 41 to 101 scalars in lanes of a vector register.
template <int DT, int V, NormPairs PAIRS, int N, bool BACK, bool ONCE> __global__ void __launch_bounds__(WG, N == 1 && BACK ? 4 : 1) norm_rope_kernel(NormParams p)
{
    typedef typename Elem<DT>::T T;
    constexpr bool TWO = PAIRS != NEIGHBOURS; // pieces have a second half
    constexpr int E = TWO ? 2 * V : V;        // entries of a piece
    __shared__ float2 table[MAX_TABLE];
    __shared__ float sums[BACK ? WG / 64 * 16 * 16 : 1]; // dw of a workgroup's wavefronts; that of wide groups goes where the angles were
    static_assert(sizeof table >= sizeof(float) * WG * 16, "room for groups of 64 lanes");
    __shared__ float weights[2][MAX_WIDTH]; // of queries and keys
    const int64_t wg = (int64_t)blockIdx.y * GRID_ROW + blockIdx.x;
    if (wg >= p.runs)
        return;
    const int64_t begin = wg * p.per_wg, end = begin + p.per_wg < p.tokens ? begin + p.per_wg : p.tokens;
    for (int i = threadIdx.x; i < p.d; i += WG) {
        weights[0][i] = weight_at(p.weight[0], p.w_dtype, i);
        weights[1][i] = weight_at(p.weight[1], p.w_dtype, i);
    }

    const int half = p.rot / 2, G = p.group, sub = threadIdx.x & (G - 1), row0 = threadIdx.x / G, rows = WG / G;
    // where a lane's pieces lie
    const int pairs = PAIRS == NEIGHBOURS ? p.rot / V : half / V; // pieces that turn
    const int pieces = PAIRS == NEIGHBOURS ? p.d / V : pairs + (p.d - p.rot) / V;
    int at[N], at2[N], pair[N]; // the entries, their partners, their first angle; -1: not there
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int c = sub + u * G;
        const bool turns = c < pairs;
        at[u] = c >= pieces ? -1 : PAIRS == NEIGHBOURS ? c * V : turns ? (PAIRS == ANY_NEIGHBOURS ? 2 * c : c * V) : p.rot + (c - pairs) * V;
        at2[u] = !turns || !TWO ? -1 : PAIRS == ANY_NEIGHBOURS ? 2 * c + 1 : c * V + half;
        pair[u] = turns ? (PAIRS == NEIGHBOURS ? c * V / 2 : c * V) : -1;
    }

    struct Row { // as it lies in memory
        Pack<T, V> a[N], c[N];
    };
    // All heads of the run's tokens; in the gradient those of one kind at a time, whose dw the lanes add up
    constexpr int KINDS = BACK ? 2 : 1;
#pragma unroll 1
    for (int kind = 0; kind < KINDS; ++kind) {
        const int heads = !BACK ? p.heads[0] + p.heads[1] : kind ? p.heads[1] : p.heads[0], head0 = kind ? p.heads[0] : 0;
        const Divisor by_heads = p.by_heads[kind];
        float dw[BACK ? N : 1][BACK ? E : 1] = {};

        for (int64_t token0 = begin; token0 < end; token0 += p.per_turn) {
            const int n = (int)(end - token0 < p.per_turn ? end - token0 : p.per_turn);
            auto place = [&](const NormTensor &y, int x) {
                const int t = (int)by_heads.div(x), head = head0 + x - t * heads;
                return reinterpret_cast<T *>(y.p + (token0 + t) * y.token + head * y.head);
            };
            auto load = [&](const NormTensor &y, int x) {
                const T *row = place(y, x);
                Row r = {};
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    if (at[u] >= 0)
                        r.a[u] = load_row<T, V, ONCE>(row + at[u]);
                    if constexpr (TWO)
                        if (at2[u] >= 0)
                            r.c[u] = load_row<T, V, ONCE>(row + at2[u]);
                }
                return r;
            };
            auto unpack = [&](const Row &r, float (&to)[N][E]) {
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        to[u][v] = (float)r.a[u].x[v];
                        if constexpr (TWO)
                            to[u][V + v] = (float)r.c[u].x[v];
                    }
            };
            auto store = [&](const NormTensor &y, int x, const float (&from)[N][E]) {
                T *row = place(y, x);
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    Pack<T, V> a, c;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        a.x[v] = (T)from[u][v];
                        if constexpr (TWO)
                            c.x[v] = (T)from[u][V + v];
                    }
                    if (at[u] >= 0)
                        store_row<ONCE>(row + at[u], a);
                    if constexpr (TWO)
                        if (at2[u] >= 0)
                            store_row<ONCE>(row + at2[u], c);
                }
            };
            // (inverse: the sign of the sines)
            auto turn = [&](float (&h)[N][E], int t, float sign) {
#pragma unroll
                for (int u = 0; u < N; ++u)
                    if (pair[u] >= 0) {
                        const float2 *cs = table + t * half + pair[u];
#pragma unroll
                        for (int v = 0; v < (TWO ? V : V / 2); ++v) {
                            const float2 r = cs[v];
                            float &a = TWO ? h[u][v] : h[u][2 * v], &c = TWO ? h[u][V + v] : h[u][2 * v + 1];
                            const float s = r.y * sign, a1 = a * r.x - c * s, c1 = a * s + c * r.x;
                            a = a1;
                            c = c1;
                        }
                    }
            };
            // entry v of piece u (of a piece that is not there, any: its entries are zeros)
            auto weight = [&](const float *w, int u, int v) { return TWO && v >= V ? w[(at2[u] >= 0 ? at2[u] : 0) + v - V] : w[(at[u] >= 0 ? at[u] : 0) + v]; };

            // a row's entries are on their way while the angles or the row before it are worked on
            Row next = {}, next_up = {};
            if (row0 < n * heads) {
                next = load(p.X, row0);
                if constexpr (BACK)
                    next_up = load(p.Y, row0);
            }
            if (kind == 0 || p.per_wg > p.per_turn || G > 16) { // (the keys of a short run find the queries' angles)
                __syncthreads();
                rope_table<WG>(p.angles, token0, n, table);
                __syncthreads();
            }
            for (int x = row0; x < n * heads; x += rows) {
                const int t = (int)by_heads.div(x);
                int of = BACK ? kind : x - t * heads >= p.heads[0];
                if constexpr (BACK)
                    asm volatile("" : "+s"(of)); // (16 registers of weights, kept over the loop, would cost a wavefront)
                const float *w = weights[of];
                float X[N][E], h[N][E];
                unpack(next, X);
                if constexpr (BACK)
                    unpack(next_up, h);
                if (x + rows < n * heads) {
                    next = load(p.X, x + rows);
                    if constexpr (BACK)
                        next_up = load(p.Y, x + rows);
                }
                float sum = 0.0f, dot = 0.0f;
                if constexpr (BACK)
                    turn(h, t, -1.0f);
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int v = 0; v < E; ++v) {
                        sum += X[u][v] * X[u][v];
                        if constexpr (BACK)
                            dot += h[u][v] * weight(w, u, v) * X[u][v];
                    }
                sum = group_sum(sum, G);
                if constexpr (BACK)
                    dot = group_sum(dot, G);
                const float r = rsqrtf(sum * p.inv_d + p.eps);
                if constexpr (BACK) {
                    const float mean = dot * p.inv_d * r * r;
                    asm volatile("" : "+s"(of));
                    w = weights[of];
#pragma unroll
                    for (int u = 0; u < N; ++u)
#pragma unroll
                        for (int v = 0; v < E; ++v) {
                            dw[u][v] += h[u][v] * (X[u][v] * r);
                            h[u][v] = r * (h[u][v] * weight(w, u, v) - X[u][v] * mean);
                        }
                    store(p.dX, x, h);
                } else {
#pragma unroll
                    for (int u = 0; u < N; ++u)
#pragma unroll
                        for (int v = 0; v < E; ++v)
                            h[u][v] = X[u][v] * r * weight(w, u, v);
                    turn(h, t, 1.0f);
                    store(p.Y, x, h);
                }
            }
        }

        if constexpr (BACK) {
            // the workgroup's share of dw: over the rows of a wavefront by lanes, over the wavefronts through LDS
            float *out = p.part + (2 * wg + kind) * p.d, *shared = G > 16 ? reinterpret_cast<float *>(table) : sums;
            const int wave = threadIdx.x >> 6;
            constexpr int M = N * E <= 16 ? N : 1; // pieces at a time
#pragma unroll
            for (int u0 = 0; u0 < N; u0 += M) {
                __syncthreads();
#pragma unroll
                for (int u = u0; u < u0 + M; ++u)
#pragma unroll
                    for (int v = 0; v < E; ++v) {
                        const float sum = rows_sum(dw[u][v], G);
                        if ((threadIdx.x & 63) < G)
                            shared[((wave * M + u - u0) * E + v) * G + sub] = sum;
                    }
                __syncthreads();
                for (int x = threadIdx.x; x < M * E * G; x += WG) {
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < WG / 64; ++k)
                        sum += shared[k * M * E * G + x];
                    // where entry v of lane l's piece u lies
                    const int l = x & (G - 1), uv = x / G, v = uv % E, c = l + (u0 + uv / E) * G;
                    const bool turns = c < pairs, second = TWO && v >= V;
                    int to;
                    if (PAIRS == NEIGHBOURS)
                        to = c * V + v;
                    else if (PAIRS == ANY_NEIGHBOURS)
                        to = turns ? 2 * c + second : p.rot + c - pairs;
                    else
                        to = turns ? c * V + v + (second ? half - V : 0) : p.rot + (c - pairs) * V + v;
                    if (c < pieces && (turns || !second))
                        out[to] = sum;
                }
            }
        }
    }
}

// dw of both kinds from the workgroups' lines: 16 columns of a workgroup, 64 threads to a column, each with every 64th line
constexpr int WEIGHT_WG = 1024;
__global__ void __launch_bounds__(WEIGHT_WG) norm_weight_kernel(NormParams p)
{
    __shared__ float shared[WEIGHT_WG / 64][16];
    const int kind = blockIdx.y;
    if (!p.dweight[kind])
        return;
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
    const float *line = p.part + kind * p.d + col;
    float sum = 0.0f;
    if (col < p.d) {
#pragma unroll 8
        for (int i = part; i < (int)p.runs; i += WEIGHT_WG / 16)
            sum += line[2 * (int64_t)i * p.d];
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 16)
        shared[threadIdx.x >> 6][threadIdx.x & 15] = sum;
    __syncthreads();
    if (part == 0 && col < p.d) {
        sum = shared[0][threadIdx.x];
#pragma unroll
        for (int k = 1; k < WEIGHT_WG / 64; ++k)
            sum += shared[k][threadIdx.x];
        p.dweight[kind][col] = sum;
    }
}

// Runs of tokens in the gradient, each of which leaves two lines of dw: two to each of the 1024 places for workgroups that the gradient with HALVES and V = 8 has (16384 tokens of 40 heads of
// 128: 113 us; 1280 runs 127, 4096 119). That with NEIGHBOURS, of 91 registers, has 1280, which such a number fills one and a half times.
constexpr int64_t MAX_RUNS = 2048;

// How many tokens a workgroup takes
template <bool BACK> void plan(NormParams &p)
{
    const int pass = WG / p.group, heads = p.heads[0] + p.heads[1]; // rows at a time
    if (BACK) {
        // the chip's slots filled once, or eight passes to a workgroup (3850 tokens of 20 heads of 128: four tokens each 24 us, six 27, two 38)
        p.per_wg = std::max<int64_t>(1, std::min<int64_t>(8 * pass / heads, (p.tokens + 1023) / 1024));
        p.per_wg = std::max(p.per_wg, (p.tokens + MAX_RUNS - 1) / MAX_RUNS);
    } else {
        // three passes to a workgroup, fewer where the chip would not be full
        const int64_t rows = p.tokens * heads;
        int64_t per = 3 * pass;
        while (per > pass && rows / per < 1024)
            per /= 2;
        p.per_wg = std::max<int64_t>(1, per / heads);
    }
    p.runs = (p.tokens + p.per_wg - 1) / p.per_wg;
    for (int kind = 0; kind < 2; ++kind)
        p.by_heads[kind] = Divisor((uint32_t)std::max(1, BACK ? p.heads[kind] : heads));
    p.per_turn = (int)std::max<int64_t>(1, std::min<int64_t>(MAX_TABLE / (p.rot / 2), 32));
}

template <int DT, int V, NormPairs PAIRS, bool BACK> hipError_t by_pieces(NormParams &p, hipStream_t stream)
{
    const int half = p.rot / 2;
    const int pieces = PAIRS == NEIGHBOURS ? p.d / V : half / V + (p.d - p.rot) / V;
    p.group = 1;
    while (p.group < pieces && p.group < 64)
        p.group *= 2;
    plan<BACK>(p);
    const dim3 grid = grid_rows(p.runs);
    auto go = [&](auto n, auto once) { norm_rope_kernel<DT, V, PAIRS, decltype(n)::value, BACK, decltype(once)::value><<<grid, WG, 0, stream>>>(p); };
    const bool once = V > 1 && p.tokens * (p.heads[0] + p.heads[1]) * p.d * (int64_t)sizeof(typename Elem<DT>::T) * (BACK ? 3 : 2) >= PAST_CACHES;
    if constexpr (V < 8) {
        if (pieces > 64) {
            go(std::integral_constant<int, 8 / V>{}, std::false_type{});
            return hipGetLastError();
        }
    }
    if (once)
        go(std::integral_constant<int, 1>{}, std::integral_constant<bool, (V > 1)>{});
    else
        go(std::integral_constant<int, 1>{}, std::false_type{});
    return hipGetLastError();
}

// The widest pieces that both parts of a row divide into (36000 tokens of 8 heads of 80, 40 entries turn, bf16: in fours 33 us, the gradient 58;
// an entry at a time 98 and 104)
template <int DT, int V, bool BACK> hipError_t by_pairs(NormParams &p, bool neighbours, hipStream_t stream)
{
    const int half = p.rot / 2;
    if (neighbours ? p.d % V == 0 && p.rot % V == 0 : half % V == 0 && (p.d - p.rot) % V == 0)
        return neighbours ? by_pieces<DT, V, NEIGHBOURS, BACK>(p, stream) : by_pieces<DT, V, HALVES, BACK>(p, stream);
    if constexpr (V > 2)
        return by_pairs<DT, V / 2, BACK>(p, neighbours, stream);
    else
        return neighbours ? by_pieces<DT, 1, ANY_NEIGHBOURS, BACK>(p, stream) : by_pieces<DT, 1, ANY, BACK>(p, stream);
}

template <bool BACK> hipError_t launch(NormParams &p, int dtype, bool neighbours, hipStream_t stream)
{
    if (dtype == MAXSIM_F32)
        return by_pairs<MAXSIM_F32, 4, BACK>(p, neighbours, stream);
    if (dtype == MAXSIM_F16)
        return by_pairs<MAXSIM_F16, 8, BACK>(p, neighbours, stream);
    return by_pairs<MAXSIM_BF16, 8, BACK>(p, neighbours, stream);
}

NormParams params(const void *X, int64_t tokens, int heads, int d, const int64_t *strides, int dtype, const void *q_weight, const void *k_weight, int w_dtype, int q_heads, float eps,
                  const RopeAngles &angles)
{
    const int64_t size = dtype == MAXSIM_F32 ? 4 : 2;
    NormParams p = {};
    p.X = {static_cast<char *>(const_cast<void *>(X)), strides[0] * size, strides[1] * size};
    p.weight[0] = q_weight;
    p.weight[1] = k_weight;
    p.w_dtype = w_dtype;
    p.angles = angles;
    p.tokens = tokens;
    p.heads[0] = q_heads;
    p.heads[1] = heads - q_heads;
    p.d = d;
    p.rot = 2 * angles.half;
    p.eps = eps;
    p.inv_d = 1.0f / (float)d;
    return p;
}

} // namespace

hipError_t norm_rope_launch(const void *X, int64_t tokens, int heads, int d, const int64_t *strides, int dtype, const void *q_weight, const void *k_weight, int w_dtype, int q_heads,
                            float eps, const RopeAngles &angles, bool neighbours, void *Y, hipStream_t stream)
{
    const int64_t size = dtype == MAXSIM_F32 ? 4 : 2;
    NormParams p = params(X, tokens, heads, d, strides, dtype, q_weight, k_weight, w_dtype, q_heads, eps, angles);
    p.Y = {static_cast<char *>(Y), strides[2] * size, strides[3] * size};
    return launch<false>(p, dtype, neighbours, stream);
}

int64_t norm_rope_backward_workspace(int64_t, int, int d) { return 4 * 2 * MAX_RUNS * d; }

hipError_t norm_rope_backward_launch(const void *X, const void *dY, int64_t tokens, int heads, int d, const int64_t *strides, int dtype, const void *q_weight, const void *k_weight,
                                     int w_dtype, int q_heads, float eps, const RopeAngles &angles, bool neighbours, void *dX, float *dq_weight, float *dk_weight, void *workspace,
                                     hipStream_t stream)
{
    const int64_t size = dtype == MAXSIM_F32 ? 4 : 2;
    NormParams p = params(X, tokens, heads, d, strides, dtype, q_weight, k_weight, w_dtype, q_heads, eps, angles);
    p.Y = {static_cast<char *>(const_cast<void *>(dY)), strides[2] * size, strides[3] * size};
    p.dX = {static_cast<char *>(dX), strides[4] * size, strides[5] * size};
    p.part = static_cast<float *>(workspace);
    p.dweight[0] = dq_weight;
    p.dweight[1] = dk_weight;
    hipError_t e = launch<true>(p, dtype, neighbours, stream);
    if (e != hipSuccess || (!p.dweight[0] && !p.dweight[1]))
        return e;
    norm_weight_kernel<<<dim3((unsigned)((d + 15) / 16), 2), WEIGHT_WG, 0, stream>>>(p);
    return hipGetLastError();
}

} // namespace maxsim
