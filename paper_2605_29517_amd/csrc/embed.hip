// Embedding lookup, Y[t] = scale W[v(t)], and its gradient, dW[v] = scale sum over the tokens t with v(t) = v of dY[t].
//
// The lookup moves rows; a lane takes pieces of up to 32 bytes of any row. The gradient first sorts the token positions by id, in an order of the ids
// that deals them to ranges in turn. Few tokens of little data: embed_small_kernel gives every workgroup a range, whose tokens it looks for among all, counts, lays down in order and
// adds up. More of them: embed_scan_kernel does the same up to the sums, without a word from the other workgroups: where its first position belongs is the
// number of tokens of the ranges before, which it has seen, too. Many tokens, for 2^19 ids at a time: embed_split_kernel sorts chunks of them by range, each within itself,
// and embed_place_kernel collects a range's parts from the chunks; where a range begins is the sum over the chunks of where it begins in them. Then a row of dW
// is one sum over a run of the sorted positions. A run of more than `slice` positions is cut at multiples of it in the sorted order; the pieces' sums are joined in a
// fixed order. No atomics on results: the same bits every time.
//
// Bound by the memory: the lookup of 16384 rows of 2048, fp32 to bf16, 25.7 us (110 MB past the caches); the gradient of 45000 tokens of 768, bf16 to fp32 with a table of
// 50001, 82 us, of which the sums take 49 (190 MB) and sorting 17; of 262144 tokens of 1024, bf16, 214 us, the sums 150 (743 MB, 4.9 TB/s) and sorting 38. Few tokens by latency: 900 of 256 7.2 us.
#include <algorithm>

#include "rows.h"

namespace maxsim {

namespace {

constexpr int WG = 256;
constexpr int SORT_WG = 1024;
constexpr int SORT_WAVES = SORT_WG / 64;
constexpr int MAX_RANGE = 512; // ids of a sorting workgroup: 16 waves' counters take 32 KB of LDS
constexpr int RANGE_BITS = 9;
constexpr int KEPT = 256;      // positions that a wave keeps from its first look; of more it looks again

struct LookupParams {
    const void *W, *tokens;
    void *Y;
    int64_t n;
    uint32_t vocab;
    int d, per_wg, chunks;
    Divisor by_chunks;
    float scale;
};

// The id of a token, counted from the id `first` on, as 32 bits, 2^32 - 1 where it names none of the `vocab` rows from there (first + vocab < 2^31: what lies before them, negative ids
// and those beyond the table are `vocab` or more away)
template <bool WIDE> __device__ __forceinline__ uint32_t token_id(const void *tokens, int64_t t, uint32_t vocab, uint32_t first = 0)
{
    if constexpr (WIDE) {
        const uint64_t v = static_cast<const uint64_t *>(tokens)[t] - first;
        return v < vocab ? (uint32_t)v : 0xffffffffu;
    } else {
        const uint32_t v = static_cast<const uint32_t *>(tokens)[t] - first;
        return v < vocab ? v : 0xffffffffu;
    }
}

template <int TO, int V> __device__ __forceinline__ Pack<typename Elem<TO>::T, V> rounded(const float (&x)[V])
{
    Pack<typename Elem<TO>::T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i)
        r.x[i] = (typename Elem<TO>::T)x[i];
    return r;
}

// A row's last piece ends with the row and may overlap the one before it (the same values).
template <int FROM, int TO, int V, bool WIDE, bool ONCE> __global__ void __launch_bounds__(WG) embed_kernel(LookupParams p)
{
    typedef typename Elem<FROM>::T T;
    typedef typename Elem<TO>::T U;
    const int64_t token0 = ((int64_t)blockIdx.y * GRID_ROW + blockIdx.x) * p.per_wg;
    if (token0 >= p.n)
        return;
    const int n = (int)(p.n - token0 < p.per_wg ? p.n - token0 : p.per_wg);
    for (int x = threadIdx.x; x < n * p.chunks; x += WG) {
        const int t = (int)p.by_chunks.div(x), c = x - t * p.chunks;
        const int e = c * V < p.d - V ? c * V : p.d - V;
        const uint32_t v = token_id<WIDE>(p.tokens, token0 + t, p.vocab);
        float y[V] = {};
        if (v != 0xffffffffu) {
            const Pack<T, V> w = load_row<T, V>(static_cast<const T *>(p.W) + (int64_t)v * p.d + e);
#pragma unroll
            for (int i = 0; i < V; ++i)
                y[i] = (float)w.x[i] * p.scale;
        }
        store_row<ONCE>(static_cast<U *>(p.Y) + (token0 + t) * p.d + e, rounded<TO>(y));
    }
}

// Ids in another order, in which frequent ones, whose numbers a tokenizer mostly puts side by side, lie in different ranges: blocks of 2^block ids are dealt
// to the ranges in turn (262144 tokens of 1024, ids by frequency: 199 us, in their own order 387, since a range has half of all tokens; shuffled ids 199 and 189)
struct Order {
    int block, ranges, range; // range: places of a range; ranges 0: the ids' own order
    Divisor by_ranges, by_range;

    // the range of an id, and its place there
    __device__ __forceinline__ uint32_t range_of(uint32_t v, uint32_t &place) const
    {
        const uint32_t q = v >> block, line = by_ranges.div(q);
        place = line << block | (v & ((1u << block) - 1));
        return q - line * (uint32_t)ranges;
    }
    // the id at a place in the order (there are places behind the last id)
    __device__ __forceinline__ uint32_t id_at(uint32_t u) const
    {
        if (ranges == 0)
            return u;
        const uint32_t g = by_range.div(u), place = u - g * (uint32_t)range;
        return ((place >> block) * (uint32_t)ranges + g) << block | (place & ((1u << block) - 1));
    }
};

struct SortParams {
    const void *tokens;
    int64_t n;
    uint32_t vocab, rows; // rows: places in the order
    Order order;
    int range;          // places of a workgroup
    int32_t *row_start; // [rows + 1]
    int32_t *at;        // [n] positions by place and, within a place, in order
    int32_t *key;       // [n] their places
};

__device__ __forceinline__ uint64_t lanes_before() { return (uint64_t(1) << (threadIdx.x & 63)) - 1; }

// LDS of one wavefront, written by some of its lanes and then read by others
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The lanes of a wavefront that have the same number of BITS bits
template <int BITS> __device__ __forceinline__ uint64_t lanes_like(bool has, uint32_t x)
{
    const uint64_t all = __builtin_amdgcn_ballot_w64(has);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
    for (int i = 0; i < BITS; ++i) {
        const uint32_t mine = (uint32_t)((int32_t)(x << (31 - i)) >> 31); // all ones where the bit is set
        const uint64_t ones = __builtin_amdgcn_ballot_w64((int32_t)mine < 0);
        lo &= ~((uint32_t)ones ^ mine);
        hi &= ~((uint32_t)(ones >> 32) ^ mine);
    }
    return (uint64_t)hi << 32 | lo;
}

// Frequent ids fill most of a wavefront: those of the first lane's id, and all where few others are left, are dealt with an id at a time.
constexpr int MANY = 16, FEW = 2;

// Counts the lanes' numbers in `count`.
__device__ __forceinline__ void count_lanes(bool has, uint32_t x, int32_t *count)
{
    const uint64_t all = __builtin_amdgcn_ballot_w64(has);
    if (all == 0)
        return;
    const uint32_t x0 = __builtin_amdgcn_readlane(x, __builtin_ctzll(all));
    const uint64_t same = __builtin_amdgcn_ballot_w64(has && x == x0);
    const int n = __popcll(same);
    if (n < MANY || !(has && x == x0)) {
        if (has)
            atomicAdd(&count[x], 1);
    } else if ((same & lanes_before()) == 0) {
        atomicAdd(&count[x], n);
    }
}

// Where a lane's element goes that is counted by `next`: after those of its number in the lanes before it
template <int BITS> __device__ __forceinline__ int next_place(bool has, uint32_t x, int32_t *next)
{
    uint64_t left = __builtin_amdgcn_ballot_w64(has);
    int to = 0;
    while (left) { // (the same for all lanes)
        const uint32_t x0 = __builtin_amdgcn_readlane(x, __builtin_ctzll(left));
        const uint64_t same = __builtin_amdgcn_ballot_w64(has && x == x0);
        if (__popcll(same) < MANY && __popcll(left) > FEW)
            break;
        if (has && x == x0) {
            to = next[x0] + __popcll(same & lanes_before());
            wave_fence();
            if ((same & lanes_before()) == 0)
                next[x0] = to + __popcll(same);
        }
        wave_fence();
        left &= ~same;
    }
    if (left) {
        const bool mine = (left >> (threadIdx.x & 63)) & 1;
        const uint64_t same = lanes_like<BITS>(mine, x);
        if (mine)
            to = next[x] + __popcll(same & lanes_before());
        wave_fence();
        if (mine && (same >> (threadIdx.x & 63)) == 1) // the last of them
            next[x] = to + 1;
        wave_fence();
    }
    return to;
}

// Inclusive sums over the threads of a workgroup of W wavefronts; `part`: W numbers
template <int W> __device__ __forceinline__ int scan_wg(int x, int32_t *part)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int other = __shfl_up(x, s);
        x += lane >= s ? other : 0;
    }
    __syncthreads();
    if (lane == 63)
        part[w] = x;
    __syncthreads();
    for (int k = 0; k < w; ++k)
        x += part[k];
    return x;
}

// A workgroup's look at all ids for those of its range
struct Scan {
    int32_t count[SORT_WAVES][MAX_RANGE];
    uint32_t kept[SORT_WAVES][KEPT];
    int32_t part[SORT_WAVES], below[SORT_WAVES];
};

// f(to, position, place in the range) for all tokens of a workgroup's range of `rows` places, by place and, within one, in order, counted from
// what `starts` gave back: starts(tokens of the ranges before, of thread r: where place r begins, how many it has).
template <bool WIDE, class Starts, class F> __device__ __forceinline__ void scan_range(const SortParams &p, Scan &s, uint32_t range, uint32_t rows, Starts starts, F f)
{
    const uint32_t lo = range * (uint32_t)p.range;
    // whether an id is of the range, its place there, whether it is of a range before
    auto look = [&](uint32_t v, uint32_t &r, bool &before) {
        if (p.order.ranges == 0) {
            r = v - lo;
            before = v < lo;
            return r < rows;
        }
        const uint32_t g = v == 0xffffffffu ? v : p.order.range_of(v, r);
        before = g < range;
        return g == range;
    };
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int k = 0; k < SORT_WAVES; ++k)
        if ((int)threadIdx.x < p.range)
            s.count[k][threadIdx.x] = 0;
    __syncthreads();

    // every wavefront looks at a run of the tokens
    const int64_t run = ((p.n + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
    const int64_t t0 = w * run < p.n ? w * run : p.n, t1 = t0 + run < p.n ? t0 + run : p.n;
    constexpr int U = 8;
    int below = 0, found = 0;
    for (int64_t t = t0; t < t1; t += 64 * U) {
        uint32_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = t + 64 * u + lane;
            v[u] = token_id<WIDE>(p.tokens, at < t1 ? at : t1 - 1, p.vocab);
            v[u] = at < t1 ? v[u] : 0xffffffffu;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t r = 0;
            bool before;
            const bool hit = look(v[u], r, before);
            below += before;
            const uint64_t hits = __builtin_amdgcn_ballot_w64(hit);
            if (hits) {
                const int slot = found + __popcll(hits & lanes_before());
                if (hit) {
                    atomicAdd(&s.count[w][r], 1);
                    if (slot < KEPT)
                        s.kept[w][slot] = (uint32_t)(t + 64 * u + lane - t0) << RANGE_BITS | r;
                }
                found += __popcll(hits);
            }
        }
    }
#pragma unroll
    for (int x = 32; x > 0; x /= 2)
        below += __shfl_xor(below, x);
    if (lane == 0)
        s.below[w] = below;
    __syncthreads();

    // where every (id, wavefront) begins
    int base = 0;
#pragma unroll
    for (int k = 0; k < SORT_WAVES; ++k)
        base += s.below[k];
    int mine = 0;
    const int r = threadIdx.x;
    if (r < (int)rows)
        for (int k = 0; k < SORT_WAVES; ++k)
            mine += s.count[k][r];
    int start = scan_wg<SORT_WAVES>(mine, s.part) - mine;
    start += starts(base, start, mine);
    if (r < (int)rows)
        for (int k = 0; k < SORT_WAVES; ++k) {
            const int c = s.count[k][r];
            s.count[k][r] = start;
            start += c;
        }
    __syncthreads();

    // the positions, 64 at a time: those of one id find their order among themselves
    auto place = [&](bool has, uint32_t x, int64_t t) {
        const int to = next_place<RANGE_BITS>(has, x, s.count[w]);
        if (has)
            f(to, t, x);
    };
    if (found <= KEPT) {
        for (int i = 0; i < found; i += 64) {
            const bool has = i + lane < found;
            const uint32_t x = s.kept[w][has ? i + lane : 0];
            place(has, x & ((1u << RANGE_BITS) - 1), t0 + (x >> RANGE_BITS));
        }
    } else {
        for (int64_t t = t0; t < t1; t += 64) {
            const int64_t at = t + lane;
            uint32_t r = 0;
            bool before;
            const bool hit = look(at < t1 ? token_id<WIDE>(p.tokens, at, p.vocab) : 0xffffffffu, r, before);
            if (__builtin_amdgcn_ballot_w64(hit))
                place(hit, r, at);
        }
    }
}

constexpr uint32_t SCAN_ROW = 1 << 21; // workgroups of a row of the grid, which holds fewer than 2^32 threads
template <bool WIDE> __global__ void __launch_bounds__(SORT_WG) embed_scan_kernel(SortParams p)
{
    __shared__ Scan s;
    const uint32_t range = blockIdx.y * SCAN_ROW + blockIdx.x, lo = range * (uint32_t)p.range; // (below 2^32 in the grid's last row, too)
    if (lo >= p.rows)
        return;
    const uint32_t rows = p.rows - lo < (uint32_t)p.range ? p.rows - lo : (uint32_t)p.range;
    scan_range<WIDE>(
        p, s, range, rows,
        [&](int base, int start, int n) {
            if (threadIdx.x < rows) {
                p.row_start[lo + threadIdx.x] = base + start;
                if (lo + threadIdx.x + 1 == p.rows)
                    p.row_start[p.rows] = base + start + n;
            }
            return base;
        },
        [&](int to, int64_t t, uint32_t r) {
            p.at[to] = (int32_t)t;
            p.key[to] = (int32_t)(lo + r);
        });
}

constexpr int SPLIT_WG = 512;
constexpr int SPLIT_WAVES = SPLIT_WG / 64;
constexpr int MAX_RANGES = 1024, RANGES_BITS = 10;
constexpr int MAX_CHUNKS = 1024;

struct SplitParams {
    const void *tokens;
    int64_t n;
    uint32_t first, vocab; // the ids from the first one on
    int chunk, chunks;   // tokens of a chunk: a multiple of 4 SPLIT_WG
    Order order;
    uint32_t *list;      // [chunks][chunk] of every chunk, its tokens by range and in order: (position in the chunk, id in the range)
    int32_t *begin;      // [chunks][ranges + 1] where a range begins among them
    int32_t *row_start, *at, *key; // (by places in the order)
};

template <bool WIDE> __global__ void __launch_bounds__(SPLIT_WG) embed_split_kernel(SplitParams p)
{
    __shared__ int32_t count[SPLIT_WAVES][MAX_RANGES];
    __shared__ int32_t part[SPLIT_WAVES];
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t chunk0 = (int64_t)blockIdx.x * p.chunk;
    const int run = p.chunk / SPLIT_WAVES; // tokens of a wavefront
    constexpr int U = 4; // 64 U tokens of a wavefront at a time; those of the smallest chunks stay where they are for the second look
    for (int k = 0; k < SPLIT_WAVES; ++k)
        for (int i = threadIdx.x; i < p.order.ranges; i += SPLIT_WG)
            count[k][i] = 0;
    uint32_t v[U];
    auto look = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t t = chunk0 + w * run + i + 64 * u + lane;
            v[u] = token_id<WIDE>(p.tokens, t < p.n ? t : p.n - 1, p.vocab, p.first);
            v[u] = t < p.n ? v[u] : 0xffffffffu;
        }
    };
    look(0);
    __syncthreads();
    for (int i = 0; i < run; i += 64 * U) {
        if (i > 0)
            look(i);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v[u] != 0xffffffffu) {
                uint32_t place;
                atomicAdd(&count[w][p.order.range_of(v[u], place)], 1);
            }
    }
    __syncthreads();

    // where every (range, wavefront) begins: a thread takes two neighbouring ranges
    int32_t *begin = p.begin + (int64_t)blockIdx.x * (p.order.ranges + 1);
    const int r0 = 2 * threadIdx.x;
    int sum[2] = {0, 0};
#pragma unroll
    for (int y = 0; y < 2; ++y)
        if (r0 + y < p.order.ranges)
            for (int k = 0; k < SPLIT_WAVES; ++k)
                sum[y] += count[k][r0 + y];
    int to = scan_wg<SPLIT_WAVES>(sum[0] + sum[1], part) - sum[0] - sum[1];
#pragma unroll
    for (int y = 0; y < 2; ++y)
        if (r0 + y < p.order.ranges) {
            begin[r0 + y] = to;
            for (int k = 0; k < SPLIT_WAVES; ++k) {
                const int c = count[k][r0 + y];
                count[k][r0 + y] = to;
                to += c;
            }
            if (r0 + y + 1 == p.order.ranges)
                begin[p.order.ranges] = to;
        }
    __syncthreads();

    uint32_t *list = p.list + chunk0;
    for (int i = 0; i < run; i += 64 * U) {
        if (run > 64 * U)
            look(i);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool has = v[u] != 0xffffffffu;
            uint32_t place = 0;
            const uint32_t g = has ? p.order.range_of(v[u], place) : 0;
            const int to = next_place<RANGES_BITS>(has, g, count[w]);
            if (has)
                list[to] = (uint32_t)(w * run + i + 64 * u + lane) << RANGE_BITS | place;
        }
    }
}

__global__ void __launch_bounds__(SORT_WG) embed_place_kernel(SplitParams p)
{
    __shared__ int32_t count[SORT_WAVES][MAX_RANGE];
    __shared__ int32_t from[MAX_CHUNKS + 1], source[MAX_CHUNKS]; // where a chunk's part begins among the range's tokens, and in the chunk's list
    __shared__ int32_t part[SORT_WAVES];
    const int lane = threadIdx.x & 63, tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int g = blockIdx.x;
    const uint32_t lo = g * (uint32_t)p.order.range, rows = p.order.range;
    int a = 0, e = 0;
    if (tid < p.chunks) {
        a = p.begin[(int64_t)tid * (p.order.ranges + 1) + g];
        e = p.begin[(int64_t)tid * (p.order.ranges + 1) + g + 1];
    }
    for (int k = 0; k < SORT_WAVES; ++k)
        if (tid < p.order.range)
            count[k][tid] = 0;
    const int upto = scan_wg<SORT_WAVES>(e - a, part);
    from[tid + 1] = upto;
    source[tid] = a;
    if (tid == 0)
        from[0] = 0;
    const int before = scan_wg<SORT_WAVES>(a, part); // (its barriers publish the above, too)
    __syncthreads();
    if (tid == SORT_WG - 1)
        part[0] = before;
    __syncthreads();
    const int base = part[0], m = from[MAX_CHUNKS];
    __syncthreads();

    // tokens i + lane, i + 64 + lane, .. of the range: their positions, and their ids in the range
    constexpr int U = 4;
    struct Batch { // as it was read (what is taken out here would be waited for here)
        uint32_t x[U];
        int32_t base[U];
        __device__ __forceinline__ int32_t at(int u) const { return base[u] + (int32_t)(x[u] >> RANGE_BITS); }
        __device__ __forceinline__ uint32_t id(int u) const { return x[u] & ((1u << RANGE_BITS) - 1); }
    };
    auto look = [&](int i, int end) {
        Batch y;
        // the last chunk whose part does not begin after the token: first for the first and the last of them, by two lanes
        const int last = (i + 64 * U < end ? i + 64 * U : end) - 1;
        auto find = [&](auto &c, auto &upper, int step, auto token) {
            for (; step > 1; step = (step + 1) / 2)
#pragma unroll
                for (int u = 0; u < (int)(sizeof c / sizeof c[0]); ++u) {
                    const int mid = (c[u] + upper[u]) / 2;
                    const bool after = from[mid] > token(u);
                    upper[u] = after && mid > c[u] ? mid : upper[u];
                    c[u] = after ? c[u] : mid;
                }
        };
        int edge[1] = {0}, none[1] = {p.chunks};
        find(edge, none, p.chunks, [&](int) { return lane == 0 ? i : last; });
        const int c0 = __builtin_amdgcn_readlane(edge[0], 0), c1 = __builtin_amdgcn_readlane(edge[0], 1) + 1;
        int c[U], upper[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            c[u] = c0;
            upper[u] = c1;
        }
        find(c, upper, c1 - c0, [&](int u) { return i + 64 * u + lane < last ? i + 64 * u + lane : last; });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = i + 64 * u + lane;
            y.x[u] = p.list[(int64_t)c[u] * p.chunk + source[c[u]] + ((k < end ? k : end - 1) - from[c[u]])];
            y.base[u] = c[u] * p.chunk;
        }
        return y;
    };
    // the same of a chunk's part, from its token o on
    auto look_part = [&](int c, int o) {
        Batch y;
        const int size = from[c + 1] - from[c];
        const uint32_t *list = p.list + (int64_t)c * p.chunk + source[c];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = o + 64 * u + lane;
            y.x[u] = size > 0 ? list[k < size ? k : size - 1] : 0;
            y.base[u] = c * p.chunk;
        }
        return y;
    };
    // A wavefront takes a run of the range's tokens, wherever they lie, or, of a crowded range, the parts of some chunks, which need no search (16400 tokens of
    // a range: 32 us by the search, a crowded range is what the kernel waits for). f is called with batches in order; the next one is on its way meanwhile:
    // a wait for a load is also one for the stores before it.
    const bool crowded = m >= 64 * p.chunks;
    const int run = ((m + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
    const int i0 = w * run < m ? w * run : m, i1 = i0 + run < m ? i0 + run : m;
    const int parts = (p.chunks + SORT_WAVES - 1) / SORT_WAVES, c0 = w * parts < p.chunks ? w * parts : p.chunks, c1 = c0 + parts < p.chunks ? c0 + parts : p.chunks;
    Batch now = {}, next = {};
    auto batches = [&](auto f) {
        if (crowded) {
            struct Spot {
                int c, o;
            };
            auto left_at = [&](Spot s) { return __builtin_amdgcn_readfirstlane(from[s.c + 1] - from[s.c]) - s.o; };
            auto after = [&](Spot s) { return s.c < c1 && left_at(s) > 64 * U ? Spot{s.c, s.o + 64 * U} : Spot{s.c + 1, 0}; };
            Spot a = {c0, 0}, b = after(a), d = after(b);
            Batch third = {};
            if (a.c < c1)
                now = look_part(a.c, a.o);
            if (b.c < c1)
                next = look_part(b.c, b.o);
            while (a.c < c1) {
                if (d.c < c1)
                    third = look_part(d.c, d.o);
                f(left_at(a), now);
                a = b;
                b = d;
                d = after(d);
                now = next;
                next = third;
            }
        } else {
            for (int i = i0; i < i1; i += 64 * U) {
                if (i + 64 * U < i1)
                    next = look(i + 64 * U, i1);
                f(i1 - i, now);
                if (i + 64 * U < i1)
                    now = next;
            }
        }
    };
    if (!crowded && i0 < i1)
        now = look(i0, i1);
    batches([&](int left, const Batch &y) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            count_lanes(64 * u + lane < left, y.id(u), count[w]);
    });
    if (!crowded && run > 64 * U) // (otherwise they are still there)
        now = look(i0, i1);
    __syncthreads();
    int mine = 0;
    if (tid < (int)rows)
        for (int k = 0; k < SORT_WAVES; ++k)
            mine += count[k][tid];
    int start = base + scan_wg<SORT_WAVES>(mine, part) - mine;
    if (tid < (int)rows) {
        p.row_start[lo + tid] = start;
        if (g + 1 == p.order.ranges && tid + 1 == (int)rows)
            p.row_start[lo + rows] = start + mine;
        for (int k = 0; k < SORT_WAVES; ++k) {
            const int c = count[k][tid];
            count[k][tid] = start;
            start += c;
        }
    }
    __syncthreads();
    batches([&](int left, const Batch &y) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool has = 64 * u + lane < left;
            if (__builtin_amdgcn_ballot_w64(has) == 0)
                continue;
            const int to = next_place<RANGE_BITS>(has, y.id(u), count[w]);
            if (has) {
                p.at[to] = y.at(u);
                p.key[to] = (int32_t)(lo + y.id(u));
            }
        }
    });
}

struct SumParams {
    const void *dY;
    void *dW;
    const int32_t *row_start, *at, *key;
    float *part; // [slices][2][d]: of a slice, the sum that belongs to a run from before it, and the one that belongs to a run that begins in it
    uint32_t vocab, rows; // rows: places in the order of the ids
    Order order;
    int d, slice, slices;
    int chunks, per_wg; // pieces of a row; rows of a workgroup
    int slices_per_wg;
    Divisor by_chunks;
    int slice_wgs; // workgroups for the slices; the others are for the rows
    int accumulate;
    float scale;
};

constexpr int ITEMS = 4; // pieces of a thread at a time
// Loads on their way within a run: eight in the slices' long ones (262144 tokens of 1024: 192 us, with four 247), four in the rows' short ones, where eight cost
// wavefronts (51200 tokens of 768: 72 us, eight 80, two 75)
constexpr int SLICE_LOADS = 8, ROW_LOADS = 4;
constexpr int MAX_ROWS = 256; // of a workgroup
constexpr int STAGED = 512;   // positions that a workgroup has in LDS

// sum of dY[at[i]] over i = s .. e, V entries from column c, in order
template <int FROM, int U, bool ONCE, class At, int V> __device__ __forceinline__ void sum_run(const SumParams &p, const At *at, int s, int e, int c, float (&sum)[V])
{
    typedef typename Elem<FROM>::T T;
    const T *dY = static_cast<const T *>(p.dY) + c;
    int i = s;
    for (; i + U <= e; i += U) {
        Pack<T, V> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            x[u] = load_row<T, V, ONCE>(dY + (int64_t)at[i + u] * p.d);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < V; ++k)
                sum[k] += (float)x[u].x[k];
    }
    for (; i < e; ++i) {
        const Pack<T, V> x = load_row<T, V, ONCE>(dY + (int64_t)at[i] * p.d);
#pragma unroll
        for (int k = 0; k < V; ++k)
            sum[k] += (float)x.x[k];
    }
}

template <int TO, int V> __device__ __forceinline__ void put_row(const SumParams &p, uint32_t u, int c, float (&sum)[V])
{
    typedef typename Elem<TO>::T U;
    const uint32_t v = p.order.id_at(u);
    if (v >= p.vocab)
        return;
    U *dst = static_cast<U *>(p.dW) + (int64_t)v * p.d + c;
#pragma unroll
    for (int k = 0; k < V; ++k)
        sum[k] *= p.scale;
    if (p.accumulate) {
        const Pack<U, V> old = load_row<U, V>(dst);
#pragma unroll
        for (int k = 0; k < V; ++k)
            sum[k] += (float)old.x[k];
    }
    store_row(dst, rounded<TO>(sum));
}

// Few tokens of few entries: a workgroup finds the tokens of its range of ids and adds their rows at once. A row of more than RUN tokens is added in runs
// of RUN at least by all threads, the runs joined in order.
constexpr int SMALL_TOKENS = 4096, RUN = 16;

template <int FROM, int TO, int V, bool WIDE> __global__ void __launch_bounds__(SORT_WG) embed_small_kernel(SortParams sort, SumParams p)
{
    __shared__ union {
        Scan scan;
        float part[SORT_WG * V]; // (once the positions are in order)
    } lds;
    constexpr int MAX_LONG = SMALL_TOKENS / (RUN + 1);
    __shared__ uint16_t at[SMALL_TOKENS];
    __shared__ int32_t first[MAX_RANGE + 1], long_rows[MAX_LONG], longs;
    const int tid = threadIdx.x;
    const uint32_t rows = (uint32_t)sort.range, lo = blockIdx.x * rows;
    if (tid == 0)
        longs = 0;
    scan_range<WIDE>(
        sort, lds.scan, blockIdx.x, rows,
        [&](int, int start, int n) {
            if (tid < (int)rows) {
                first[tid] = start;
                if (tid + 1 == (int)rows)
                    first[rows] = start + n;
                if (n > RUN)
                    long_rows[atomicAdd(&longs, 1)] = tid; // (their order does not matter)
            }
            return 0;
        },
        [&](int to, int64_t t, uint32_t) { at[to] = (uint16_t)t; });
    __syncthreads();
    for (int x = tid; x < (int)rows * p.chunks; x += SORT_WG) {
        const int y = (int)p.by_chunks.div(x), k = x - y * p.chunks, c = k * V < p.d - V ? k * V : p.d - V;
        const int s = first[y], e = first[y + 1];
        if (e - s > RUN || (p.accumulate && s == e))
            continue;
        float sum[V] = {};
        sum_run<FROM, 8, false>(p, at, s, e, c, sum);
        put_row<TO>(p, lo + y, c, sum);
    }
    const int pieces = p.chunks < SORT_WG ? p.chunks : SORT_WG, splits = SORT_WG / pieces;
    const int y = tid / pieces, x = tid - y * pieces;
    for (int i = 0; i < longs; ++i) { // (the same for all threads)
        const int row = long_rows[i], s = first[row], e = first[row + 1];
        const int each = (e - s + splits - 1) / splits > RUN ? (e - s + splits - 1) / splits : RUN, runs = (e - s + each - 1) / each;
        for (int k0 = 0; k0 < p.chunks; k0 += pieces) {
            const int k = k0 + x, c = k * V < p.d - V ? k * V : p.d - V;
            const bool there = y < runs && k < p.chunks;
            float sum[V] = {};
            if (there)
                sum_run<FROM, 8, false>(p, at, s + y * each, s + (y + 1) * each < e ? s + (y + 1) * each : e, c, sum);
            __syncthreads();
#pragma unroll
            for (int m = 0; m < V; ++m)
                lds.part[m * SORT_WG + tid] = sum[m];
            __syncthreads();
            if (there && y == 0) {
                for (int o = 1; o < runs; ++o)
#pragma unroll
                    for (int m = 0; m < V; ++m)
                        sum[m] += lds.part[m * SORT_WG + o * pieces + x];
                put_row<TO>(p, lo + row, c, sum);
            }
        }
    }
}

template <int V> __device__ __forceinline__ void put_part(const SumParams &p, int64_t i, int c, const float (&sum)[V])
{
    Pack<float, V> out;
#pragma unroll
    for (int j = 0; j < V; ++j)
        out.x[j] = sum[j];
    store_row(p.part + i * p.d + c, out);
}

template <int FROM, int TO, int V, bool ONCE> __global__ void __launch_bounds__(WG) embed_sum_kernel(SumParams p)
{
    __shared__ int32_t first[MAX_ROWS + 1], staged[STAGED];
    const int64_t wg = (int64_t)blockIdx.y * GRID_ROW + blockIdx.x;
    if (wg < p.slice_wgs) {
        const int n = p.row_start[p.rows];
        for (int x = threadIdx.x; x < p.slices_per_wg * p.chunks; x += WG) {
            const int y = (int)p.by_chunks.div(x), k = x - y * p.chunks;
            const int c = k * V < p.d - V ? k * V : p.d - V;
            const int64_t i = wg * p.slices_per_wg + y;
            if (i >= p.slices || i * p.slice >= n)
                continue;
            const int i0 = (int)i * p.slice, i1 = i0 + p.slice < n ? i0 + p.slice : n;
            const int v0 = p.key[i0], v1 = p.key[i1 - 1];
            const int s0 = p.row_start[v0], e0 = p.row_start[v0 + 1], s1 = p.row_start[v1], e1 = p.row_start[v1 + 1];
            if (s0 < i0 && e0 - s0 > p.slice) {
                float sum[V] = {};
                sum_run<FROM, SLICE_LOADS, ONCE>(p, p.at, i0, e0 < i1 ? e0 : i1, c, sum);
                put_part(p, 2 * i, c, sum);
            }
            if (s1 >= i0 && e1 - s1 > p.slice) {
                float sum[V] = {};
                sum_run<FROM, SLICE_LOADS, ONCE>(p, p.at, s1, i1, c, sum);
                put_part(p, 2 * i + 1, c, sum);
            }
        }
        return;
    }
    const int64_t v0 = (wg - p.slice_wgs) * p.per_wg;
    if (v0 >= p.rows)
        return;
    const int rows = p.rows - v0 < p.per_wg ? (int)(p.rows - v0) : p.per_wg;
    for (int i = threadIdx.x; i <= rows; i += WG)
        first[i] = p.row_start[v0 + i];
    __syncthreads();
    const int base = first[0], m = first[rows] - base;
    const bool few = m <= STAGED;
    if (few) {
        for (int i = threadIdx.x; i < m; i += WG)
            staged[i] = p.at[base + i];
        __syncthreads();
    }
    // a thread's pieces some at a time: most rows have one token or none, and all of their first ones are on their way before any is waited for
    typedef typename Elem<FROM>::T T;
    auto sum_rows = [&](const int32_t *at) {
        for (int x0 = threadIdx.x; x0 < rows * p.chunks; x0 += WG * ITEMS) {
            Pack<T, V> one[ITEMS];
            int row[ITEMS], col[ITEMS], s[ITEMS], e[ITEMS];
    #pragma unroll
            for (int u = 0; u < ITEMS; ++u) {
                const int x = x0 + u * WG, y = x < rows * p.chunks ? (int)p.by_chunks.div(x) : -1, k = x - y * p.chunks;
                row[u] = y;
                col[u] = k * V < p.d - V ? k * V : p.d - V;
                s[u] = y >= 0 ? first[y] - base : 0;
                e[u] = y >= 0 ? first[y + 1] - base : 0;
                if (y >= 0 && (e[u] - s[u] > p.slice || (p.accumulate && s[u] == e[u]))) // (not this workgroup's, or not to be touched)
                    row[u] = -1;
                one[u] = Pack<T, V>{};
                if (row[u] >= 0 && s[u] < e[u])
                    one[u] = load_row<T, V, ONCE>(static_cast<const T *>(p.dY) + (int64_t)at[s[u]] * p.d + col[u]);
            }
    #pragma unroll
            for (int u = 0; u < ITEMS; ++u) {
                if (row[u] < 0)
                    continue;
                float sum[V];
    #pragma unroll
                for (int k = 0; k < V; ++k)
                    sum[k] = (float)one[u].x[k];
                if (s[u] + 1 < e[u])
                    sum_run<FROM, ROW_LOADS, ONCE>(p, at, s[u] + 1, e[u], col[u], sum);
                put_row<TO>(p, (uint32_t)(v0 + row[u]), col[u], sum);
            }
        }
    };
    if (few)
        sum_rows(staged);
    else
        sum_rows(p.at + base);
}

// The rows whose run is cut: a workgroup to each slice in which such a run begins. The slices' sums are dealt in order to `splits` threads of
// a piece of the row, whose sums are added in order.
constexpr int JOIN_WG = 1024;
template <int TO, int V> __global__ void __launch_bounds__(JOIN_WG) embed_join_kernel(SumParams p)
{
    __shared__ float shared[JOIN_WG * V];
    const int64_t i = blockIdx.x, i0 = i * p.slice, i1 = i0 + p.slice;
    if (i1 > p.row_start[p.rows])
        return;
    const int v = p.key[i1 - 1];
    const int64_t s = p.row_start[v], e = p.row_start[v + 1];
    if (s < i0 || e - s <= p.slice)
        return;
    const int64_t last = (e - 1) / p.slice;
    const int pieces = p.chunks < JOIN_WG ? p.chunks : JOIN_WG, splits = JOIN_WG / pieces;
    const int y = threadIdx.x / pieces, x = threadIdx.x - y * pieces;
    const int64_t each = (last - i + splits) / splits; // slices of a thread
    for (int k0 = 0; k0 < p.chunks; k0 += pieces) {
        const int k = k0 + x, c = k * V < p.d - V ? k * V : p.d - V;
        const bool there = y < splits && k < p.chunks;
        float sum[V] = {};
        if (there) {
            const int64_t j0 = i + y * each, j1 = j0 + each < last + 1 ? j0 + each : last + 1;
#pragma unroll 8
            for (int64_t j = j0; j < j1; ++j) {
                const Pack<float, V> a = load_row<float, V>(p.part + (2 * j + (j == i)) * p.d + c);
#pragma unroll
                for (int m = 0; m < V; ++m)
                    sum[m] += a.x[m];
            }
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < V; ++m)
            shared[m * JOIN_WG + threadIdx.x] = sum[m];
        __syncthreads();
        if (there && y == 0) {
            for (int o = 1; o < splits; ++o)
#pragma unroll
                for (int m = 0; m < V; ++m)
                    sum[m] += shared[m * JOIN_WG + o * pieces + x];
            put_row<TO>(p, (uint32_t)v, c, sum);
        }
    }
}

template <class F> hipError_t by_dtype(int dtype, F &&f)
{
    if (dtype == MAXSIM_F32)
        return f(std::integral_constant<int, MAXSIM_F32>{});
    if (dtype == MAXSIM_F16)
        return f(std::integral_constant<int, MAXSIM_F16>{});
    return f(std::integral_constant<int, MAXSIM_BF16>{});
}

// Rows of a workgroup: about a thousand pieces, fewer where the chip would not be full
int rows_per_wg(int64_t rows, int chunks)
{
    int64_t per = std::min(MAX_ROWS, std::max(1, 1024 / chunks));
    while (per > 1 && rows / per < 2048)
        per /= 2;
    return (int)per;
}

// Positions of a slice: short ones, so that no row keeps a workgroup long, of many tokens longer ones, which are joined sooner (51200 tokens of 768: 64 71 us,
// 32 72, 16 90; 262144 of 1024: 128 191 us, 64 204, 256 204; 12600 of 168, whose pieces take few threads: 16 30 us, 64 35)
int slice_of(int64_t n, int d) { return n * d < (1 << 23) ? 16 : n < (1 << 17) ? 64 : 128; }

// How the positions are sorted: in chunks, where there are more tokens than a look by every workgroup pays for. More than MAX_IDS ids are taken some at a time, each with launches of its
// own, unless the tokens are few: every workgroup's look takes a time in proportion to tokens times ids (rows of 4, bf16, 20000 tokens, 700000 ids: 46 us, in two parts 61; 10^7 ids 357 and 551;
// 50000 tokens 77 and 66, 632 and 602; 300000 tokens 363 and 174; 10^6 tokens 1409 and 467).
struct SortPlan {
    bool split;
    bool dealt; // ids to the ranges in turn
    int range, ranges, block, chunk, chunks; // block: of the order, a power of two
    int64_t rows; // places in the order
};
constexpr int64_t SCAN_TOKENS = 8192, SCAN_TOKENS_OF_MANY_IDS = 49152;
constexpr int64_t MAX_IDS = MAX_RANGE * MAX_RANGES;
int64_t ids_at_a_time(int64_t n, int64_t vocab) { return n > SCAN_TOKENS_OF_MANY_IDS ? std::min(vocab, MAX_IDS) : vocab; }
SortPlan sort_plan(int64_t n, int64_t vocab, int d)
{
    SortPlan s;
    s.range = (int)std::min<int64_t>(MAX_RANGE, (vocab + 255) / 256);
    s.ranges = (int)((vocab + s.range - 1) / s.range);
    s.chunk = 4 * SPLIT_WG;
    while ((n + s.chunk - 1) / s.chunk > MAX_CHUNKS) // (2^17 tokens at most: a position in a chunk and a place in a range share 32 bits)
        s.chunk *= 2;
    s.split = n > SCAN_TOKENS && s.ranges <= MAX_RANGES;
    s.chunks = s.split ? (int)((n + s.chunk - 1) / s.chunk) : 0;
    s.dealt = s.ranges <= MAX_RANGES;
    s.block = 0;
    s.rows = vocab;
    if (s.dealt) {
        // rows of dW that lie together have 32 entries or more, where a range has as many ids (300000 tokens of 16, frequent ids first: 191 us, with 128 entries 219)
        while (2 << s.block <= s.range && (int64_t)d << s.block < 32)
            ++s.block;
        const int64_t blocks = (vocab + (1 << s.block) - 1) >> s.block;
        s.range = (int)((blocks + s.ranges - 1) / s.ranges) << s.block; // (not more than MAX_RANGE, which is a multiple of a block)
        s.rows = (int64_t)s.range * s.ranges;
    }
    return s;
}
// All in one launch, where the ids of a range may all be tokens of one workgroup, which adds them up alone: 1440 tokens of 256, fp32, 7.6 us, in three launches 13.6; 4000 of 256, bf16,
// vocabulary 50001, 13 and 21, half of them one id 26 and 23. Beyond 2 MB that id would cost too much (4000 of 1024, bf16: 14 and 17, half of them one id 56 and 22).
// A workgroup takes all pieces of its range's rows at once: where their indices do not divide (wide rows of single entries), the other kernels take a row at a time.
bool is_small(const SortPlan &s, int64_t n, int64_t vocab, int d, int size, int w_size, int chunks)
{
    return n <= SMALL_TOKENS && n * d * size <= (2 << 20) && vocab * d * w_size < PAST_CACHES && (vocab + 255) / 256 <= MAX_RANGE &&
           Divisor::divides_below((int64_t)s.range * chunks, chunks);
}
// Entries of a piece of dW: added to what is there, the pieces of a row may not overlap
int entries_of_piece(int d, int full, bool accumulate) { return d >= full && !(accumulate && d % full != 0) ? full : 1; }
int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

} // namespace

hipError_t embed_launch(const void *W, int64_t vocab, int d, int dtype, const void *tokens, bool wide, int64_t n, float scale, void *Y, int y_dtype, hipStream_t stream)
{
    return by_dtype(dtype, [&](auto from) {
        return by_dtype(y_dtype, [&](auto to) {
            constexpr int FROM = decltype(from)::value, TO = decltype(to)::value, FULL = FROM == MAXSIM_F32 && TO == MAXSIM_F32 ? 4 : 8;
            auto go = [&](auto v, auto w) {
                constexpr int V = decltype(v)::value;
                const int chunks = (d + V - 1) / V, per = rows_per_wg(n, chunks);
                const LookupParams p = {W, tokens, Y, n, (uint32_t)vocab, d, per, chunks, Divisor((uint32_t)chunks), scale};
                if (n * d * (TO == MAXSIM_F32 ? 4 : 2) >= PAST_CACHES)
                    embed_kernel<FROM, TO, V, decltype(w)::value, true><<<grid_rows((n + per - 1) / per), WG, 0, stream>>>(p);
                else
                    embed_kernel<FROM, TO, V, decltype(w)::value, false><<<grid_rows((n + per - 1) / per), WG, 0, stream>>>(p);
                return hipGetLastError();
            };
            const std::integral_constant<int, FULL> full{};
            const std::integral_constant<int, 1> one{};
            if (wide)
                return d >= FULL ? go(full, std::true_type{}) : go(one, std::true_type{});
            return d >= FULL ? go(full, std::false_type{}) : go(one, std::false_type{});
        });
    });
}

int64_t embed_backward_workspace(int64_t n, int64_t vocab, int d)
{
    const SortPlan s = sort_plan(n, ids_at_a_time(n, vocab), d);
    const int64_t slices = (n + slice_of(n, d) - 1) / slice_of(n, d), sums = slices > 1 ? 8 * slices * d : 0;
    // (the chunks' lists are done with when the slices' sums begin)
    return up16(4 * (s.rows + 1)) + 2 * up16(4 * n) + std::max(sums, s.split ? 4 * (int64_t)s.chunks * (s.chunk + s.ranges + 1) : 0);
}

// dW's `vocab` rows from the id `first` on
static hipError_t some_rows(const void *dY, int dtype, const void *tokens, bool wide, int64_t n, int64_t first, int64_t vocab, int d, float scale, bool accumulate, void *dW, int w_dtype,
                            void *workspace, hipStream_t stream)
{
    char *ws = static_cast<char *>(workspace);
    const SortPlan s = sort_plan(n, vocab, d);
    const int64_t rows = s.rows;
    int32_t *row_start = reinterpret_cast<int32_t *>(ws), *at = reinterpret_cast<int32_t *>(ws + up16(4 * (rows + 1))), *key = at + up16(4 * n) / 4;
    float *part = reinterpret_cast<float *>(key + up16(4 * n) / 4);
    const Order order = s.dealt ? Order{s.block, s.ranges, s.range, Divisor((uint32_t)s.ranges), Divisor((uint32_t)s.range)} : Order{0, 0, 0, Divisor(1), Divisor(1)};
    const int piece = entries_of_piece(d, dtype == MAXSIM_F32 || w_dtype == MAXSIM_F32 ? 4 : 8, accumulate), chunks = (d + piece - 1) / piece;
    const bool small = is_small(s, n, vocab, d, dtype == MAXSIM_F32 ? 4 : 2, w_dtype == MAXSIM_F32 ? 4 : 2, chunks);
    const SortParams scan = {tokens, n, (uint32_t)vocab, (uint32_t)rows, order, s.range, row_start, at, key};
    if (small) {
        // (sorts by itself)
    } else if (s.split) {
        uint32_t *list = reinterpret_cast<uint32_t *>(part);
        int32_t *begin = reinterpret_cast<int32_t *>(list + (int64_t)s.chunks * s.chunk);
        const SplitParams p = {tokens, n, (uint32_t)first, (uint32_t)vocab, s.chunk, s.chunks, order, list, begin, row_start, at, key};
        if (wide)
            embed_split_kernel<true><<<(unsigned)s.chunks, SPLIT_WG, 0, stream>>>(p);
        else
            embed_split_kernel<false><<<(unsigned)s.chunks, SPLIT_WG, 0, stream>>>(p);
        embed_place_kernel<<<(unsigned)s.ranges, SORT_WG, 0, stream>>>(p);
    } else {
        const dim3 grid(std::min((unsigned)s.ranges, SCAN_ROW), ((unsigned)s.ranges + SCAN_ROW - 1) / SCAN_ROW);
        if (wide)
            embed_scan_kernel<true><<<grid, SORT_WG, 0, stream>>>(scan);
        else
            embed_scan_kernel<false><<<grid, SORT_WG, 0, stream>>>(scan);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    return by_dtype(dtype, [&](auto from) {
        return by_dtype(w_dtype, [&](auto to) {
            constexpr int FROM = decltype(from)::value, TO = decltype(to)::value, FULL = FROM == MAXSIM_F32 || TO == MAXSIM_F32 ? 4 : 8;
            auto go = [&](auto v) {
                constexpr int V = decltype(v)::value;
                const int slice = slice_of(n, d), per = rows_per_wg(rows, chunks);
                const int slices = n > slice ? (int)((n + slice - 1) / slice) : 0, slices_per = std::max(1, WG / chunks), slice_wgs = (slices + slices_per - 1) / slices_per;
                const SumParams p = {dY, dW, row_start, at, key, part, (uint32_t)vocab, (uint32_t)rows, order, d, slice, slices, chunks, per, slices_per, Divisor((uint32_t)chunks), slice_wgs, accumulate, scale};
                if (small) {
                    if (wide)
                        embed_small_kernel<FROM, TO, V, true><<<(unsigned)s.ranges, SORT_WG, 0, stream>>>(scan, p);
                    else
                        embed_small_kernel<FROM, TO, V, false><<<(unsigned)s.ranges, SORT_WG, 0, stream>>>(scan, p);
                    return hipGetLastError();
                }
                const dim3 grid = grid_rows(slice_wgs + (rows + per - 1) / per);
                if (n * d * (FROM == MAXSIM_F32 ? 4 : 2) + vocab * d * (TO == MAXSIM_F32 ? 4 : 2) >= PAST_CACHES)
                    embed_sum_kernel<FROM, TO, V, true><<<grid, WG, 0, stream>>>(p);
                else
                    embed_sum_kernel<FROM, TO, V, false><<<grid, WG, 0, stream>>>(p);
                if (slices > 0)
                    embed_join_kernel<TO, V><<<(unsigned)slices, JOIN_WG, 0, stream>>>(p);
                return hipGetLastError();
            };
            return piece == FULL ? go(std::integral_constant<int, FULL>{}) : go(std::integral_constant<int, 1>{});
        });
    });
}

hipError_t embed_backward_launch(const void *dY, int dtype, const void *tokens, bool wide, int64_t n, int64_t vocab, int d, float scale, bool accumulate, void *dW, int w_dtype,
                                 void *workspace, hipStream_t stream)
{
    const int64_t ids = ids_at_a_time(n, vocab), row = (int64_t)d * (w_dtype == MAXSIM_F32 ? 4 : 2);
    for (int64_t first = 0; first < vocab; first += ids) {
        const hipError_t e = some_rows(dY, dtype, tokens, wide, n, first, std::min(ids, vocab - first), d, scale, accumulate, static_cast<char *>(dW) + first * row, w_dtype, workspace, stream);
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

} // namespace maxsim
