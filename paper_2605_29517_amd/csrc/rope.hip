// Rotary positions: y = scale R(p f) x on the first `rot` entries of every head, the rest copied.
//
// Each entry is read once and written once; what else there is to do is one angle per (token, pair), shared by the token's heads. A
// workgroup takes some tokens, puts their cosines and sines into LDS, and then moves chunks of 16 bytes through registers. The angle is
// reduced in 64 bits (its fraction of a turn), so that positions of 10^6 keep the accuracy of small ones. Bound by the memory: 16 x 1024
// tokens of 40 heads of 128, bf16 (336 MB), 54.8 us, 6.1 TB/s; fp32 texts of 1.1 GB 189 us, 5.9; a few tokens (32 of 16 heads of 64, fp16) by
// the launch, 3.1 us.
#include <algorithm>

#include "common.h"

namespace maxsim {

struct RopeParams {
    const char *X;
    char *Y;
    int64_t x_token, x_head, y_token, y_head; // bytes
    const float *freqs;
    const int32_t *positions, *offsets;
    int64_t tokens, b;
    int heads, d, rot;
    float scale, sign; // sign: -1 for the inverse rotation
    int per_wg;        // tokens of a workgroup
    int neighbours;    // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2)
};

namespace {

constexpr int WG = 256;
constexpr int MAX_TABLE = 2048; // (token, pair) entries of a workgroup: 16 KB of LDS

template <int DT> struct Elem;
template <> struct Elem<MAXSIM_F32> {
    typedef float T;
};
template <> struct Elem<MAXSIM_F16> {
    typedef _Float16 T;
};
template <> struct Elem<MAXSIM_BF16> {
    typedef __bf16 T;
};

// V entries that lie together
template <class T, int V> struct Pack {
    T x[V];
};
template <class T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const char *p)
{
    Pack<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
// 16 bytes; ONCE: that the caches need not keep
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <class T, int V, bool ONCE> __device__ __forceinline__ Pack<T, V> load_pack_aligned(const char *p)
{
    const u32x4 *at = reinterpret_cast<const u32x4 *>(p);
    return __builtin_bit_cast(Pack<T, V>, ONCE ? __builtin_nontemporal_load(at) : *at);
}
template <bool ONCE, class T, int V> __device__ __forceinline__ void store_pack_aligned(char *p, const Pack<T, V> &r)
{
    u32x4 *at = reinterpret_cast<u32x4 *>(p);
    if constexpr (ONCE)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), at);
    else
        *at = __builtin_bit_cast(u32x4, r);
}

enum RopePairs { HALVES, HALVES_ANY, NEIGHBOURS, SINGLE };

// V: entries of a chunk. HALVES: a lane takes a chunk of the first half and its partner (rot / 2 is a multiple of V). HALVES_ANY: a
// lane takes one chunk and reads the partners of its entries from where they lie, so that a head's row is read twice, the second time
// from the cache. NEIGHBOURS: pairs lie inside a chunk. SINGLE (V = 1): a lane takes one pair or one plain entry, wherever they lie.
// 30000 tokens of 16 heads, bf16: d = 128 HALVES 40.6 us, HALVES_ANY 51.6; neighbours 43.2, SINGLE 82.4; 36 of 64 entries HALVES_ANY 32.6, SINGLE 70.2.
// In place, HALVES_ANY could read a partner that another lane has already turned: SINGLE, whose lanes hold both.
template <int DT, int V, RopePairs PAIRS, bool ONCE> __global__ void __launch_bounds__(WG) rope_kernel(RopeParams p)
{
    typedef typename Elem<DT>::T T;
    constexpr int SIZE = sizeof(T);
    __shared__ float2 table[MAX_TABLE];
    const int half = p.rot / 2;
    const int64_t token0 = ((int64_t)blockIdx.y * GRID_ROW + blockIdx.x) * p.per_wg;
    if (token0 >= p.tokens)
        return;
    const int n = (int)(p.tokens - token0 < p.per_wg ? p.tokens - token0 : p.per_wg);

    int64_t seq0 = 0, seq1 = 0; // the first sequences that start after the first and after the last token
    if (p.offsets) {
        lower_bound_offsets2(p.offsets, p.b, token0 + 1, token0 + n, seq0, seq1);
        seq0 = seq0 > p.b ? p.b : seq0;
        seq1 = seq1 > p.b ? p.b : seq1;
    }
    for (int x = threadIdx.x; x < n * half; x += WG) {
        const int t = x / half, pair = x - t * half;
        const int64_t token = token0 + t;
        int64_t at = token;
        if (p.positions) {
            at = p.positions[token];
        } else if (p.offsets) {
            int64_t lo = seq0, hi = seq1; // the first sequence that starts after this token
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (p.offsets[mid] > token)
                    hi = mid;
                else
                    lo = mid + 1;
            }
            at = token - (lo > 0 ? p.offsets[lo - 1] : 0);
        }
        double turns = (double)at * (double)p.freqs[pair] * 0.15915494309189533577; // 1 / (2 pi)
        turns -= __builtin_rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        table[x] = make_float2(c * p.scale, s * p.scale * p.sign);
    }
    __syncthreads();

    // chunks of a head: those of the first half and the plain ones, or all
    const int plain = (p.d - p.rot) / V;
    const int chunks = PAIRS == HALVES || PAIRS == SINGLE ? half / V + plain : p.d / V;
    const int per_token = p.heads * chunks;
    for (int x = threadIdx.x; x < n * per_token; x += WG) {
        const int t = x / per_token, y = x - t * per_token;
        const int head = y / chunks, c = y - head * chunks;
        const char *src = p.X + (token0 + t) * p.x_token + head * p.x_head;
        char *dst = p.Y + (token0 + t) * p.y_token + head * p.y_head;
        const float2 *cs = table + t * half;
        if constexpr (PAIRS == HALVES) {
            if (c < half / V) {
                const int e = c * V;
                Pack<T, V> u = load_pack_aligned<T, V, ONCE && PAIRS != HALVES_ANY>(src + e * SIZE), v = load_pack_aligned<T, V, ONCE && PAIRS != HALVES_ANY>(src + (e + half) * SIZE);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float2 r = cs[e + i];
                    const float a = (float)u.x[i], b = (float)v.x[i];
                    u.x[i] = (T)(a * r.x - b * r.y);
                    v.x[i] = (T)(a * r.y + b * r.x);
                }
                store_pack_aligned<ONCE>(dst + e * SIZE, u);
                store_pack_aligned<ONCE>(dst + (e + half) * SIZE, v);
            } else {
                const int e = p.rot + (c - half / V) * V;
                store_pack_aligned<ONCE>(dst + e * SIZE, load_pack_aligned<T, V, ONCE && PAIRS != HALVES_ANY>(src + e * SIZE));
            }
        } else if constexpr (PAIRS == SINGLE) {
            if (c < half) {
                const int e = p.neighbours ? 2 * c : c, f = p.neighbours ? e + 1 : e + half;
                const float2 r = cs[c];
                const float a = (float)*reinterpret_cast<const T *>(src + e * SIZE), b = (float)*reinterpret_cast<const T *>(src + f * SIZE);
                *reinterpret_cast<T *>(dst + e * SIZE) = (T)(a * r.x - b * r.y);
                *reinterpret_cast<T *>(dst + f * SIZE) = (T)(a * r.y + b * r.x);
            } else {
                const int e = p.rot + c - half;
                *reinterpret_cast<T *>(dst + e * SIZE) = *reinterpret_cast<const T *>(src + e * SIZE);
            }
        } else if constexpr (PAIRS == NEIGHBOURS) {
            const int e = c * V;
            Pack<T, V> u = load_pack_aligned<T, V, ONCE && PAIRS != HALVES_ANY>(src + e * SIZE);
#pragma unroll
            for (int i = 0; i < V; i += 2)
                if (e + i < p.rot) {
                    const float2 r = cs[(e + i) / 2];
                    const float a = (float)u.x[i], b = (float)u.x[i + 1];
                    u.x[i] = (T)(a * r.x - b * r.y);
                    u.x[i + 1] = (T)(a * r.y + b * r.x);
                }
            store_pack_aligned<ONCE>(dst + e * SIZE, u);
        } else { // (not in place: another lane may have written a partner)
            const int e = c * V;
            Pack<T, V> u = load_pack_aligned<T, V, ONCE && PAIRS != HALVES_ANY>(src + e * SIZE);
            Pack<T, V> v = u;
            if (e + V <= half)
                v = load_pack<T, V>(src + (e + half) * SIZE);
            else if (e >= half && e + V <= p.rot)
                v = load_pack<T, V>(src + (e - half) * SIZE);
            else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (e + i < p.rot)
                        v.x[i] = *reinterpret_cast<const T *>(src + (e + i < half ? e + i + half : e + i - half) * SIZE);
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (e + i < p.rot) {
                    const bool low = e + i < half;
                    const float2 r = cs[low ? e + i : e + i - half];
                    const float a = (float)u.x[i], b = (float)v.x[i];
                    u.x[i] = (T)(low ? a * r.x - b * r.y : b * r.y + a * r.x);
                }
            store_pack_aligned<ONCE>(dst + e * SIZE, u);
        }
    }
}

// From so many bytes read and written on, the next kernel finds little of them in the caches (256 MB before the memory): then they are
// moved past them. 16 x 1024 tokens of 40 heads of 128, bf16 (336 MB): 68.6 us without the hint, 54.1 with it; fp32 texts of 1.1 GB 197 and 189.
constexpr int64_t STREAM_BYTES = int64_t(128) << 20;

template <int DT, bool ONCE> void launch(RopeParams p, bool wide, hipStream_t stream)
{
    constexpr int V = DT == MAXSIM_F32 ? 4 : 8;
    const int half = p.rot / 2;
    const RopePairs pairs = !wide ? SINGLE : p.neighbours ? NEIGHBOURS : half % V == 0 && p.rot % V == 0 ? HALVES : p.X == p.Y ? SINGLE : HALVES_ANY;
    const int64_t per_token = (int64_t)p.heads * (pairs == SINGLE ? p.d : p.d / V);
    // about a thousand chunks to a workgroup, fewer where the chip would not be full
    int64_t per = std::max<int64_t>(1, 1024 / per_token);
    while (per > 1 && p.tokens / per < 2048)
        per /= 2;
    p.per_wg = (int)std::min<int64_t>(per, MAX_TABLE / std::max(1, half));
    const dim3 grid = grid_rows((p.tokens + p.per_wg - 1) / p.per_wg);
    if (pairs == SINGLE)
        rope_kernel<DT, 1, SINGLE, false><<<grid, WG, 0, stream>>>(p);
    else if (pairs == NEIGHBOURS)
        rope_kernel<DT, V, NEIGHBOURS, ONCE><<<grid, WG, 0, stream>>>(p);
    else if (pairs == HALVES)
        rope_kernel<DT, V, HALVES, ONCE><<<grid, WG, 0, stream>>>(p);
    else
        rope_kernel<DT, V, HALVES_ANY, ONCE><<<grid, WG, 0, stream>>>(p);
}

} // namespace

bool rope_width_ok(int rot) { return rot / 2 <= MAX_TABLE; }

// Strides in entries.
hipError_t rope_launch(const void *X, int64_t tokens, int heads, int d, int64_t x_token, int64_t x_head, int dtype, const float *freqs, int rot,
                       const int32_t *positions, const int32_t *offsets, int64_t b, float scale, bool neighbours, bool inverse, void *Y, int64_t y_token, int64_t y_head,
                       hipStream_t stream)
{
    const int size = dtype == MAXSIM_F32 ? 4 : 2;
    RopeParams p = {static_cast<const char *>(X), static_cast<char *>(Y), x_token * size, x_head * size, y_token * size, y_head * size, freqs, positions, offsets, tokens, b,
                    heads, d, rot, scale, inverse ? -1.0f : 1.0f, 0, neighbours};
    const bool wide = (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)p.x_token | (uintptr_t)p.x_head | (uintptr_t)p.y_token | (uintptr_t)p.y_head | (uintptr_t)(d * size)) & 15) == 0;
    auto go = [&](auto once) {
        constexpr bool ONCE = decltype(once)::value;
        if (dtype == MAXSIM_F32)
            launch<MAXSIM_F32, ONCE>(p, wide, stream);
        else if (dtype == MAXSIM_F16)
            launch<MAXSIM_F16, ONCE>(p, wide, stream);
        else
            launch<MAXSIM_BF16, ONCE>(p, wide, stream);
    };
    if (2 * tokens * heads * d * size >= STREAM_BYTES)
        go(std::true_type{});
    else
        go(std::false_type{});
    return hipGetLastError();
}

} // namespace maxsim
