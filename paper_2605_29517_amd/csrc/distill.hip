// Distillation from a teacher's top scores. Of a row of scores s, with entries e = 0 .. k - 1 that name columns j_e and hold the teacher's scores t_e:
//     p = softmax(t / tau) over the entries that count,   q = softmax(s / tau) over all columns,
//     loss = sum_e p_e (log p_e - log q_{j_e}),   ds_j = u / tau (q_j - sum over e with j_e = j of p_e).
// An entry counts where its column is in the row and neither its score nor the column's is minus infinity (a document without tokens).
//
// One group of threads to a row: a wavefront for short rows, a workgroup for longer ones, several workgroups where there are few long rows. Every
// thread forms a maximum and a sum of exponentials of its own, which are then brought together. For the gradient rows of up to 128 KB stay in registers; it
// is q everywhere first, then the listed columns again.
//
// A gradient that follows the losses forms the row's maximum and sum again instead of taking one fp32 log of the sum, which for scores 560 temperatures from zero (28 at 0.05) costs q
// 3 10^-5, where the row's own numbers cost 10^-7. It takes 164 us instead of 160 for 4096 rows of 50001, bf16, 99 instead of 93 for 500 of 100003, fp32, 21 instead of 15 for 64 of them.
//
// Bound by the memory: 4096 rows of 50001, bf16 (410 MB): the loss 70 us, 5.9 TB/s read, the gradient 166, 4.9 TB/s both ways, with or without the loss; 500 rows of 100003, fp32, too long for registers, 98 us;
// 64 rows of 1000 6.1 us, latency.
//
// Compiled with NaNs honoured: a score that is not a number has to show in its row's loss and gradient.
#include <algorithm>

#include "rows.h"

namespace maxsim {

namespace {

enum DistillMode { LOSS, GRAD }; // (the gradient with or without the loss)

struct DistillParams {
    const void *scores, *teacher;
    const int32_t *index; // null: entry e is column e
    void *g;
    float *loss;      // or null
    float *lse;       // LOSS: or null
    const float *up;  // GRAD: a row's upstream gradient, or null and
    float weight;     // this one for all
    int64_t ld, g_ld; // entries from row to row
    int n, b, k;
    int t_dtype;
    int slots;   // of the table that finds entries of one column: a power of two, twice k at least
    int shift;   // 32 less the power
    int pieces;  // of a row, each of a workgroup of its own
    float2 *stats; // [n][pieces] of every piece, its maximum and its sum of exponentials to that; null: they pass through the gradient
    float inv_tau, c; // c: log2(e) / tau
};

constexpr float LN2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float teacher_score(const DistillParams &p, int64_t i)
{
    if (p.t_dtype == MAXSIM_F32)
        return static_cast<const float *>(p.teacher)[i];
    if (p.t_dtype == MAXSIM_F16)
        return (float)static_cast<const _Float16 *>(p.teacher)[i];
    return (float)static_cast<const __bf16 *>(p.teacher)[i];
}

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// Values that every thread of a group of TH has, combined over the group in a fixed order. `spare`: TH / 64 floats for each of N values.
template <int TH, int N, class Op> __device__ __forceinline__ void combine(float (&x)[N], float *spare, Op op)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        x[i] = wave_butterfly(x[i], op);
    if constexpr (TH > 64) {
        constexpr int W = TH / 64;
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                spare[i * W + w] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = spare[i * W];
#pragma unroll
            for (int k = 1; k < W; ++k)
                x[i] = op(x[i], spare[i * W + k]);
        }
    }
}

template <int TH> __device__ __forceinline__ void group_sync()
{
    if constexpr (TH > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

constexpr float NOTHING = -__builtin_huge_valf();

// The pieces of V entries of a row, from its first address that is a multiple of 16 bytes on (rows of 50001 entries of 16 bits: the loss 87 us, in
// pieces from the row's start 87 where rows of 50048 take 74), of which a workgroup takes some. The entries before and behind them go to threads of the first and the last
// part one by one.
template <class T, int V> struct RowPieces {
    int begin, end, head;
    int64_t lone; // this thread's entry that is in no piece; -1: none

    __device__ __forceinline__ RowPieces(const T *row, int b, int part, int parts, int tid)
    {
        head = (int)((0 - reinterpret_cast<uintptr_t>(row)) & 15) / (int)sizeof(T);
        head = head < b ? head : b;
        const int all = (b - head) / V, each = (all + parts - 1) / parts;
        begin = part * each < all ? part * each : all;
        end = begin + each < all ? begin + each : all;
        const int before = part == 0 ? head : 0, behind = part == parts - 1 ? b - head - all * V : 0;
        lone = tid < before ? tid : tid < before + behind ? head + all * V + tid - before : -1;
    }
    // as it lies in memory; minus infinities where there is none
    template <bool ONCE> __device__ __forceinline__ u32x4 load(const T *row, int c) const
    {
        u32x4 y = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, _Float16>::value ? 0xfc00fc00u : 0xff80ff80u;
        if (c < end)
            y = __builtin_bit_cast(u32x4, load_row<T, V, ONCE>(row + head + (int64_t)c * V));
        return y;
    }
};

// Entry v of a piece. A piece stays as it was read, its entries are taken out where they are needed: as floats, and the exponentials with them,
// they would take two and four times the registers.
template <class T> __device__ __forceinline__ float entry(const u32x4 &y, int v)
{
    if constexpr (sizeof(T) == 4)
        return __uint_as_float(y[v]);
    else if constexpr (std::is_same<T, _Float16>::value)
        return (float)__builtin_bit_cast(f16x8, y)[v];
    else
        return __uint_as_float(v & 1 ? y[v / 2] & 0xffff0000u : y[v / 2] << 16);
}
// What was taken out before is forgotten.
__device__ __forceinline__ void as_read(u32x4 &y)
{
    asm volatile("" : "+v"(y));
    __builtin_amdgcn_sched_barrier(0); // (or it would be forgotten before it is used)
}

// A maximum and the sum of exponentials to it. Exponents are (s - top) c: whatever the scores' size, no thread's sum overflows, also not that of one that has seen nothing but a mask
// (s c - top c in one rounding, an operation less, does where 2^-24 of top c passes 128: masks of -10^9 at a temperature of 0.05, the lowest score of the type at most; 4096 rows of
// 12001, bf16: the loss 24.2 and 25.3 us, the gradient 45.2 and 46.3).
struct Softmax {
    float top = NOTHING, zero = 0.0f, sum = 0.0f; // zero: the top, or 0 where there is none

    __device__ __forceinline__ void raise(float to, float c) // to another maximum
    {
        const float z = to == NOTHING ? 0.0f : to;
        sum *= top == NOTHING ? 0.0f : exp2_of((zero - z) * c);
        top = to;
        zero = z;
    }
    // KEPT: the pieces are needed again
    template <class T, int V, bool KEPT, int N> __device__ __forceinline__ void add(u32x4 (&y)[N], float c)
    {
        float to = top;
#pragma unroll
        for (int u = 0; u < N; ++u) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                to = fmaxf(to, entry<T>(y[u], v));
            if constexpr (KEPT)
                as_read(y[u]);
        }
        raise(to, c);
#pragma unroll
        for (int u = 0; u < N; ++u) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                sum += exp2_of((entry<T>(y[u], v) - zero) * c);
            if constexpr (KEPT) {
                asm volatile("" : "+v"(sum)); // (here, and not where the sum is needed)
                as_read(y[u]);
            }
        }
    }
    __device__ __forceinline__ void add(float x, float c)
    {
        raise(fmaxf(top, x), c);
        sum += exp2_of((x - zero) * c);
    }
};

constexpr int BATCH = 4; // pieces on their way at a time (4096 rows of 50001, bf16, the gradient: 182 us, with eight 192)

template <int TH, bool ONCE, class T, int V> __device__ __forceinline__ void sweep(Softmax &s, const T *row, const RowPieces<T, V> &pieces, int tid, float c)
{
    const float lone = pieces.lone >= 0 ? (float)row[pieces.lone] : NOTHING;
    for (int p = pieces.begin + tid; p < pieces.end; p += TH * BATCH) {
        u32x4 y[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
            y[u] = pieces.template load<ONCE>(row, p + u * TH);
        s.add<T, V, false>(y, c);
    }
    s.add(lone, c);
}

// The maximum and sum of a part of a row. Without a workspace every part of the row finds them where its own gradient begins, which it writes over once it has
// read them: rows have more than 32 KB for each of P - 1 parts, so that the last and smallest of P parts, 1024 at most, has 16368 bytes at least; the sums take 8 P.
constexpr int STATS_WG = 512;
template <class T, int V> __device__ __forceinline__ T *sums_of_parts(const DistillParams &p, int64_t i, const RowPieces<T, V> &part) { return static_cast<T *>(p.g) + i * p.g_ld + part.head + (int64_t)part.begin * V; }
constexpr int SUM_BYTES = sizeof(float2);
template <int DT, int V> __global__ void __launch_bounds__(STATS_WG) distill_stats_kernel(DistillParams p)
{
    typedef typename Elem<DT>::T T;
    __shared__ float spare[2][STATS_WG / 64];
    const int64_t i = blockIdx.x / (unsigned)p.pieces;
    const int part = blockIdx.x % (unsigned)p.pieces;
    Softmax s;
    const T *row = static_cast<const T *>(p.scores) + i * p.ld;
    sweep<STATS_WG, false>(s, row, RowPieces<T, V>(row, p.b, part, p.pieces, threadIdx.x), threadIdx.x, p.c);
    float top[1] = {s.top};
    combine<STATS_WG>(top, spare[0], Max{});
    s.raise(top[0], p.c);
    float sum[1] = {s.sum};
    combine<STATS_WG>(sum, spare[1], Sum{});
    const float2 both = make_float2(top[0], sum[0]);
    if (p.stats) {
        if (threadIdx.x == 0)
            p.stats[blockIdx.x] = both;
    } else {
        constexpr int E = SUM_BYTES / sizeof(T);
        for (int o = threadIdx.x; o < p.pieces; o += STATS_WG)
            store_row(sums_of_parts(p, i, RowPieces<T, V>(row, p.b, o, p.pieces, threadIdx.x)) + part * E, __builtin_bit_cast(Pack<T, E>, both));
    }
}

// TH: threads of a group; KEEP: pieces of V entries that a thread keeps (0: the row is read again for the gradient).
template <int DT, int V, DistillMode MODE, int TH, int KEEP, bool ONCE> __global__ void __launch_bounds__(TH > 256 ? TH : 256) distill_kernel(DistillParams p)
{
    typedef typename Elem<DT>::T T;
    extern __shared__ char lds[];
    const int groups = blockDim.x / TH, group = TH > 64 ? 0 : __builtin_amdgcn_readfirstlane((int)(threadIdx.x / TH)), tid = threadIdx.x % TH;
    const int64_t wg = (int64_t)blockIdx.y * GRID_ROW + blockIdx.x, unit = wg * groups + group;
    const bool parts = MODE == GRAD && TH > 64 && p.pieces > 1; // (a loss takes the parts' sums alone)
    const int64_t i = parts ? (int64_t)((unsigned)wg / (unsigned)p.pieces) : unit; // (of few rows: fewer than 2^32)
    const int part = parts ? (int)((unsigned)wg % (unsigned)p.pieces) : 0;
    if (i >= p.n)
        return; // (the whole group)
    const int k = p.k, b = p.b;
    constexpr int W = TH / 64;
    float *spare = reinterpret_cast<float *>(lds); // TH > 64: 6 W floats, not used twice
    int32_t *idx = reinterpret_cast<int32_t *>(lds + (TH > 64 ? 24 * W : 0)) + 3 * k * group;
    float *prob = reinterpret_cast<float *>(idx + k), *own = prob + k;
    int32_t *key = idx + 3 * k, *first = key + p.slots, *many = first + p.slots; // TH > 64: the table

    const T *row = static_cast<const T *>(p.scores) + i * p.ld;
    T *dst = static_cast<T *>(p.g) + i * p.g_ld;
    const float weight = MODE == GRAD ? p.up ? p.up[i] : p.weight : 0.0f;
    const RowPieces<T, V> pieces(row, b, part, parts ? p.pieces : 1, tid);

    // a thread's first entry, then its part of the row, then the score that the entry names: all on their way at once
    int j0 = -1;
    float t0 = 0.0f, s0 = NOTHING;
    if (tid < k) {
        j0 = p.index ? p.index[i * k + tid] : tid;
        t0 = teacher_score(p, i * k + tid);
    }
    u32x4 x[KEEP > 0 ? KEEP : 1];
    if constexpr (KEEP > 0) {
#pragma unroll
        for (int j = 0; j < KEEP; ++j)
            x[j] = pieces.template load<ONCE>(row, tid + j * TH);
    }
    const float lone = KEEP > 0 && pieces.lone >= 0 ? (float)row[pieces.lone] : NOTHING;
    if (j0 >= 0 && j0 < b)
        s0 = (float)row[j0];

    // the row's maximum and sum, as far as this thread sees them
    Softmax soft;
    if constexpr (KEEP > 0) {
        soft.add<T, V, true>(x, p.c);
        soft.add(lone, p.c);
    } else if (TH > 64 && p.pieces > 1) {
        for (int o = tid; o < p.pieces; o += TH) {
            constexpr int E = SUM_BYTES / sizeof(T);
            const float2 of = p.stats ? p.stats[i * p.pieces + o] : __builtin_bit_cast(float2, load_row<T, E>(sums_of_parts(p, i, pieces) + o * E));
            Softmax other;
            other.top = of.x;
            other.zero = of.x == NOTHING ? 0.0f : of.x;
            other.sum = of.y;
            const float top = fmaxf(soft.top, other.top);
            soft.raise(top, p.c);
            other.raise(top, p.c);
            soft.sum += other.sum;
        }
    } else {
        sweep<TH, ONCE && MODE == LOSS>(soft, row, pieces, tid, p.c);
    }

    // where the row is written over, the scores that entries name are read before any thread writes
    const bool over = MODE == GRAD && p.g == p.scores;
    if (over)
        for (int e = tid; e < k; e += TH) {
            const int j = e < TH ? j0 : p.index ? p.index[i * k + e] : e;
            own[e] = e < TH ? s0 : j >= 0 && j < b ? (float)row[j] : NOTHING;
        }

    // u / tau q = 2^((s - zero) c) share by
    float zero = 0.0f, total = 0.0f, by = 0.0f, share = 0.0f;
    auto gradient = [&](float s) { return exp2_of((s - zero) * p.c) * share; };
    if constexpr (MODE == GRAD) {
        // q does not wait for the teacher
        float top[1] = {soft.top};
        combine<TH>(top, spare, Max{});
        soft.raise(top[0], p.c);
        float sum[1] = {soft.sum};
        combine<TH>(sum, spare + W, Sum{});
        zero = soft.zero;
        total = sum[0];
        by = weight * p.inv_tau;
        share = 1.0f / total;
        auto put = [&](int c, const u32x4 &y) {
            Pack<T, V> r;
#pragma unroll
            for (int v = 0; v < V; ++v)
                r.x[v] = (T)(exp2_of((entry<T>(y, v) - zero) * p.c) * (share * by));
            if (c < pieces.end)
                store_row<ONCE>(dst + pieces.head + (int64_t)c * V, r);
        };
        if constexpr (KEEP > 0) {
#pragma unroll
            for (int j = 0; j < KEEP; ++j)
                put(tid + j * TH, x[j]);
        } else {
            for (int c = pieces.begin + tid; c < pieces.end; c += TH * BATCH) {
                u32x4 y[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u)
                    y[u] = pieces.template load<ONCE>(row, c + u * TH);
#pragma unroll
                for (int u = 0; u < BATCH; ++u)
                    put(c + u * TH, y[u]);
            }
        }
        if (pieces.lone >= 0)
            dst[pieces.lone] = (T)(gradient(KEEP > 0 ? lone : (float)row[pieces.lone]) * by);
    }

    // the teacher's entries
    constexpr int ROW = MODE == LOSS, USED = 2 - 2 * ROW; // a loss brings the row's numbers together with the teacher's
    float tops[1 + ROW] = {NOTHING};
    if constexpr (ROW)
        tops[1] = soft.top;
    float counted = 0.0f;
    for (int e = tid; e < k; e += TH) {
        int j = j0;
        float s = s0, t = t0;
        if (e >= TH) {
            j = p.index ? p.index[i * k + e] : e;
            t = teacher_score(p, i * k + e);
            s = over ? own[e] : j >= 0 && j < b ? (float)row[j] : NOTHING;
        }
        const bool counts = j >= 0 && j < b && !(s == NOTHING) && !(t == NOTHING);
        idx[e] = counts ? j : -1;
        prob[e] = t;
        own[e] = s;
        if (counts) {
            tops[0] = fmaxf(tops[0], t);
            counted += 1.0f;
        }
    }
    combine<TH>(tops, spare + USED * W, Max{});
    const float t_top = tops[0];
    float sums[2 + ROW] = {0.0f, counted}; // of the teacher's, how many count
    if constexpr (ROW) {
        soft.raise(tops[1], p.c);
        zero = soft.zero;
        sums[2] = soft.sum;
    }
    for (int e = tid; e < k; e += TH)
        if (idx[e] >= 0) {
            prob[e] = exp2_of((prob[e] - t_top) * p.c);
            sums[0] += prob[e];
        }
    combine<TH>(sums, spare + (USED + 1 + ROW) * W, Sum{});
    const bool some = sums[1] > 0.0f;
    if constexpr (ROW)
        total = sums[2];

    if (MODE == LOSS || p.loss) { // (the same for all threads)
        float loss[1] = {0.0f};
        const float t_log = log2f(sums[0]), log2_sum = log2f(total);
        for (int e = tid; e < k; e += TH)
            if (idx[e] >= 0) {
                const float q = prob[e] / sums[0];
                const float log_p = ((e < TH ? t0 : teacher_score(p, i * k + e)) - t_top) * p.c - t_log, log_q = (own[e] - zero) * p.c - log2_sum; // (to the base 2)
                loss[0] += q != 0.0f ? q * (log_p - log_q) : 0.0f;
            }
        combine<TH>(loss, spare + 5 * W, Sum{});
        if (tid == 0 && part == 0) {
            p.loss[i] = loss[0] * LN2;
            if (MODE == LOSS && p.lse)
                p.lse[i] = fmaf(zero, p.inv_tau, log2_sum * LN2);
        }
    }
    if constexpr (MODE == GRAD) {
        if (!some) { // (q is taken back)
            for (int c = pieces.begin + tid; c < pieces.end; c += TH)
                store_row<ONCE>(dst + pieces.head + (int64_t)c * V, Pack<T, V>{});
            if (pieces.lone >= 0)
                dst[pieces.lone] = (T)0.0f;
        }
        // columns of another workgroup's part are its to write
        const int64_t lo = part == 0 ? 0 : pieces.head + (int64_t)pieces.begin * V, hi = part == (parts ? p.pieces - 1 : 0) ? b : pieces.head + (int64_t)pieces.end * V;
        // the listed columns: the first entry of a column writes it, with the sum of all of its entries
        if (!p.index) { // (one entry to a column)
            group_sync<TH>();
            for (int e = tid; e < k; e += TH)
                if (idx[e] >= lo && idx[e] < hi)
                    dst[e] = (T)((gradient(own[e]) - prob[e] / sums[0]) * by);
            return;
        }
        if constexpr (TH > 64) {
            for (int h = tid; h < p.slots; h += TH) {
                key[h] = -1;
                first[h] = k;
                many[h] = 0;
            }
        }
        group_sync<TH>();
        if constexpr (TH > 64) {
            auto slot_of = [&](int j) {
                // Columns in even steps must not lie side by side: multiplied by 2^32 times the golden ratio's fraction (multiplicative hashing), folded, and once more by that
                // of the root of two. 1024 columns in any step up to 200000 are found in 1.5 places on average and in 2.7 at the worst step, random ones in 1.5; one multiplication: 484.
                uint32_t h = (uint32_t)j * 0x9e3779b9u;
                h = (h ^ h >> 15) * 0x6a09e667u >> p.shift;
                for (;;) {
                    const int old = atomicCAS(&key[h], -1, j);
                    if (old == -1 || old == j)
                        return h;
                    h = (h + 1) & (uint32_t)(p.slots - 1);
                }
            };
            for (int e = tid; e < k; e += TH)
                if (idx[e] >= 0) {
                    const uint32_t h = slot_of(idx[e]);
                    atomicMin(&first[h], e);
                    atomicAdd(&many[h], 1);
                }
            __syncthreads();
            for (int e = tid; e < k; e += TH)
                if (idx[e] >= 0) {
                    const uint32_t h = slot_of(idx[e]);
                    if (first[h] == e && idx[e] >= lo && idx[e] < hi) {
                        float sum = prob[e];
                        if (many[h] > 1)
                            for (int o = e + 1; o < k; ++o)
                                sum += idx[o] == idx[e] ? prob[o] : 0.0f;
                        dst[idx[e]] = (T)((gradient(own[e]) - sum / sums[0]) * by);
                    }
                }
        } else {
            for (int e = tid; e < k; e += TH) {
                const int j = idx[e];
                bool leads = j >= 0;
                float sum = 0.0f;
                for (int o = 0; o < k; ++o) {
                    const bool same = idx[o] == j;
                    sum += same ? prob[o] : 0.0f;
                    leads = leads && !(same && o < e);
                }
                if (leads)
                    dst[j] = (T)((gradient(own[e]) - sum / sums[0]) * by);
            }
        }
    }
}

template <int DT, int V, DistillMode MODE, int TH, int KEEP> hipError_t go(const DistillParams &p, hipStream_t stream)
{
    const int groups = TH > 64 ? 1 : p.n > 1024 ? 4 : 1;
    const size_t lds = (TH > 64 ? 24 * (TH / 64) + 12 * (size_t)p.slots : 0) + 12 * (size_t)p.k * groups;
    const int64_t units = (int64_t)p.n * (TH > 64 ? MODE == LOSS ? 1 : p.pieces : 1);
    const dim3 grid = grid_rows((units + groups - 1) / groups);
    const int64_t bytes = (int64_t)p.n * p.b * (int64_t)sizeof(typename Elem<DT>::T) * (MODE == LOSS ? 1 : 2);
    if (TH > 64 && bytes >= PAST_CACHES)
        distill_kernel<DT, V, MODE, TH, KEEP, (TH > 64)><<<grid, TH * groups, lds, stream>>>(p);
    else
        distill_kernel<DT, V, MODE, TH, KEEP, false><<<grid, TH * groups, lds, stream>>>(p);
    return hipGetLastError();
}

constexpr int64_t KEPT_PIECES = 8192; // of 16 bytes: rows that stay in a workgroup's registers

template <int DT, DistillMode MODE> hipError_t by_size(DistillParams &p, hipStream_t stream)
{
    constexpr int V = DT == MAXSIM_F32 ? 4 : 8;
    const int64_t chunks = p.b / V;
    if (p.pieces > 1) {
        distill_stats_kernel<DT, V><<<(unsigned)((int64_t)p.n * p.pieces), STATS_WG, 0, stream>>>(p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        return go<DT, V, MODE, 256, 0>(p, stream);
    }
    const bool few = p.k <= 128 || !p.index; // (a wavefront compares its entries one by one)
    if constexpr (MODE == GRAD) {
        if (few && chunks <= 64)
            return go<DT, V, MODE, 64, 1>(p, stream);
        if (few && chunks <= 256)
            return go<DT, V, MODE, 64, 4>(p, stream);
        if (chunks <= 512)
            return go<DT, V, MODE, 256, 2>(p, stream);
        if (chunks <= 1024)
            return go<DT, V, MODE, 256, 4>(p, stream); // (4096 rows of 6001, bf16: 27.5 us, with eight pieces 36)
        if (chunks <= 2048)
            return go<DT, V, MODE, 256, 8>(p, stream);
        if (chunks <= KEPT_PIECES)
            return go<DT, V, MODE, 512, 16>(p, stream); // (4096 rows of 50001, bf16: 164 us; 1024 threads with eight pieces, one workgroup to a compute unit, 204)
        return go<DT, V, MODE, 1024, 0>(p, stream);
    } else {
        return few && chunks <= 256 ? go<DT, V, MODE, 64, 0>(p, stream) : chunks <= 8192 ? go<DT, V, MODE, 256, 0>(p, stream) : go<DT, V, MODE, 1024, 0>(p, stream);
    }
}

template <DistillMode MODE> hipError_t by_dtype(DistillParams &p, int dtype, hipStream_t stream)
{
    if (dtype == MAXSIM_F32)
        return by_size<MAXSIM_F32, MODE>(p, stream);
    if (dtype == MAXSIM_F16)
        return by_size<MAXSIM_F16, MODE>(p, stream);
    return by_size<MAXSIM_BF16, MODE>(p, stream);
}

// Parts of a row, where there are fewer rows than would fill the chip and they are long
constexpr int64_t SPLIT_BYTES = 32768;
int pieces_of(int64_t n, int64_t b, int dtype, int num_cu)
{
    const int64_t bytes = b * (dtype == MAXSIM_F32 ? 4 : 2);
    if (n >= num_cu || bytes <= SPLIT_BYTES)
        return 1;
    return (int)std::min<int64_t>(std::min<int64_t>(2 * num_cu / n, (bytes + SPLIT_BYTES - 1) / SPLIT_BYTES), 1024);
}

} // namespace

int64_t distill_workspace(int n, int64_t b, int dtype, int num_cu)
{
    const int pieces = pieces_of(n, b, dtype, num_cu);
    return pieces > 1 ? 8 * (int64_t)n * pieces : 0;
}

// g null: loss and lse; otherwise the gradient by up or, where that is null, by weight, and the loss, if it is wanted
hipError_t distill_launch(const void *scores, int n, int b, int64_t ld, int dtype, const void *teacher, int t_dtype, const int32_t *index, int k, float tau, float *loss, float *lse,
                          const float *up, float weight, void *g, int64_t g_ld, void *workspace, int num_cu, hipStream_t stream)
{
    int slots = 2, shift = 31;
    for (; slots < 2 * k; slots *= 2)
        --shift;
    // In place, a workgroup may not write a part of a row of which another one still reads entries. The gradient of rows that stay in registers takes one workgroup a row
    // (200 rows of 30000, fp32: 16.4 us, in four parts 21.5; 64 of 50001, bf16: 14.3 and 15.0).
    const bool whole = g && (g == scores || b / (dtype == MAXSIM_F32 ? 4 : 8) <= KEPT_PIECES);
    const int pieces = whole ? 1 : pieces_of(n, b, dtype, num_cu);
    DistillParams p = {scores, teacher, index, g, loss, lse, up, weight, ld, g_ld, n, b, k, t_dtype, slots, shift, pieces, pieces > 1 && !up ? static_cast<float2 *>(workspace) : nullptr,
                       1.0f / tau, (float)(1.44269504088896340736 / (double)tau)};
    return g ? by_dtype<GRAD>(p, dtype, stream) : by_dtype<LOSS>(p, dtype, stream);
}

} // namespace maxsim
