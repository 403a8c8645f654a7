// Shared parts of the attention kernels: packed sequences, tiles in LDS, products.
//
// All products are 32x32x16 MFMAs with the tokens of the wavefront's own side as columns, so that a lane keeps ONE of its 32 columns:
//   scores      S^T [key][query] = K Q^T   (A: rows of K from LDS, B: the query rows, in registers)
//   values      O^T [d][query]  += V^T P^T (A: V read transposed from LDS, B: P^T, as it left the softmax)
// A lane (c = lane % 32, h = lane / 32) holds of S^T the rows 8 (r / 4) + 4 h + r % 4, r = 0 .. 15, of column c. Statistics over a
// column are then in-lane apart from one exchange between the halves, and registers 8 s .. 8 s + 7, rounded to 16 bits, are the
// B operand of step s of the next product as they are, if its A operand takes the rows in the same order: the transposing read
// gives a lane four consecutive rows, and rows 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 are two such reads.
#pragma once
#include <algorithm>

#include "common.h"

namespace maxsim {

struct AttnRows { // a packed tensor [tokens, heads, d], strides in bytes
    char *p;
    int64_t head;
    uint32_t token; // (below 2^25: a tile's rows are addressed in 32 bits)
};

// Division of n < 2^31 by a number that the launch knows
struct AttnDivisor {
    uint32_t by, mul, shift;
    static AttnDivisor of(uint32_t by)
    {
        uint32_t s = 0;
        while ((uint64_t(1) << s) < by)
            ++s;
        return {by, (uint32_t)((uint64_t(1) << (31 + s)) / by + 1), 31 + s}; // (exact: n times the excess of mul * by is below 2^(31 + s))
    }
    __device__ __forceinline__ int quotient(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
    __device__ __forceinline__ int operator()(int &n) const // leaves the remainder
    {
        const int q = quotient(n);
        n -= q * (int)by;
        return q;
    }
};

struct AttnParams {
    AttnRows Q, K, V, O, dO, dQ, dK, dV;
    const int32_t *q_off, *k_off; // [b + 1]
    float *lse;                   // [q_tokens, hq]
    float *part_o, *part_lse;     // [n_split, q_tokens, hq, d], [n_split, q_tokens, hq]: partial results of the split forward
    float *part_k, *part_v;       // [n_split, k_tokens, hkv, d]: partial sums of dK (without scale) and dV
    float *stat;                  // [hq, 2, q_tokens]: -lse / scale and -delta (the backward's own)
    int b, q_tokens, k_tokens;
    int hq, hkv, d;
    // query heads that share keys: row r of a sequence is token r / pack, head r % pack of the group (there are less than 2^30 rows)
    int pack;
    int n_slots; // see attn_find_slot
    int n_split; // pieces of the keys
    int n_wg;    // workgroups that the launch is for
    AttnDivisor by_pack, by_slots, by_split, by_hkv;
    int same; // queries and keys have the same rows: one pair of offsets to read
    int causal;
    float scale, scale_log2; // scale_log2 = scale * log2(e)
};

// Rows of one sequence
struct AttnSeq {
    int start, len;
};
__device__ __forceinline__ AttnSeq attn_seq(const int32_t *off, int i, int tokens)
{
    const int s = min(max(off[i], 0), tokens), e = min(max(off[i + 1], s), tokens);
    return {s, e - s};
}

// Whether a sequence has tile t of `rows` rows is not known to the host, which has no lengths. Sequence i gets the tile slots
// [first(i), first(i + 1)), first(i) = floor(offset_i * mul / rows) + i, mul the rows of a token: always as many as it needs and at most
// one too many, so that the launch is tokens * mul / rows + b tiles and a slot finds its sequence, the last i with first(i) <= slot, by a
// search over the offsets. Each step of a search is a round trip to memory before anything else can start: the first looks at the 64
// sequences around the place that equal lengths would give, and mostly ends it (always up to 63 sequences). All lanes active, slot uniform.
struct AttnPlace {
    int i, first; // the sequence, and its first slot
    AttnSeq s;
};
template <int ROWS> __device__ __forceinline__ AttnPlace attn_find_slot(const int32_t *off, int b, int tokens, int mul, int slot, int n_slots)
{
    const int guess = (int)((float)slot * (float)b * __builtin_amdgcn_rcpf((float)n_slots)) - 32;
    const int lo = __builtin_amdgcn_readfirstlane(max(min(guess, b - 63), 0));
    const int at = lo + (threadIdx.x & 63);
    const int v = min(max(off[min(at, b)], 0), tokens);
    const uint64_t below = __builtin_amdgcn_ballot_w64(at < b && (int)((uint32_t)v * (uint32_t)mul / ROWS) + at <= slot);
    const int n = __builtin_popcountll(below);
    AttnPlace x;
    if (n > 0 && n < 64) {
        x.i = lo + n - 1;
        x.s.start = __builtin_amdgcn_readlane(v, n - 1);
        x.s.len = max(__builtin_amdgcn_readlane(v, n) - x.s.start, 0);
    } else {
        OffsetSearch s; // the first i in [0, b) with first(i) > slot, b if there is none
        s.begin(b - 1);
        while (s.open()) {
            const uint32_t p = s.probe(threadIdx.x & 63);
            const bool in = p < s.end;
            const int first = (int)((uint32_t)min(max(off[in ? p : 0u], 0), tokens) * (uint32_t)mul / ROWS) + (int)p;
            s.narrow(__builtin_amdgcn_ballot_w64(in && first <= slot));
        }
        const int i = __builtin_amdgcn_readfirstlane(s.lo);
        x.i = max(i - 1, 0);
        x.s = attn_seq(off, x.i, tokens);
    }
    x.first = (int)((uint32_t)x.s.start * (uint32_t)mul / ROWS) + x.i;
    return x;
}

// A tile of rows in LDS: CH chunks of 16 bytes a row, chunk c of row r at position c ^ swizzle(r). LDS serves 256 bytes at a time, 64
// banks of 4: a read of one chunk of sixteen consecutive rows (the operand as it lies) and a transposing read of 64 bytes of four
// rows (both halves of it) then both meet every bank once.
template <int DP> struct AttnTile {
    static constexpr int CH = DP / 8, ROW = DP * 2;
    static __device__ __forceinline__ constexpr int swizzle(int r)
    {
        return (CH % 16 == 0 ? (r & 3) << 2 : CH == 8 ? ((r >> 1) & 1) << 2 : 0) | ((r >> 2) & 3);
    }
};

// 16 (or 4) bytes per lane from base + offset to LDS, lane l's to dst + 16 l (4 l). Assembly, because the compiler puts a wait for all
// loads into LDS before every LDS read that it cannot tell from their destination, which is the other buffer here; attn_arrive waits
// for them. No vector register is written; m0, which names the destination, has no other user in these kernels.
__device__ __forceinline__ uint32_t attn_lds(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }
template <bool ONCE> __device__ __forceinline__ void attn_load_lds16(const char *base, uint32_t offset, uint32_t dst)
{
    if constexpr (ONCE) // read once: the caches need not keep it
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(base), "s"(dst) : "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(dst) : "memory");
}
__device__ __forceinline__ void attn_load_lds4(const void *base, uint32_t offset, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(offset), "s"(base), "s"(dst) : "memory");
}

// Copies ROWS consecutive rows of one head to LDS, NW wavefronts together; a wavefront's instruction fills 1 KB. Rows past `last`
// are the last one's copies and chunks past the row's end are the last chunk's: what is masked later is finite, and of this sequence.
template <int DP, int ROWS, int NW, bool ONCE = false> struct AttnCopy {
    static constexpr int CH = DP / 8, N = ROWS * CH / 64, PER = (N + NW - 1) / NW;
    static constexpr bool EVEN = NW * 64 % (16 * CH) == 0; // a lane's rows are STEP apart, its chunk is the same in all of them
    static constexpr int STEP = NW * 64 / CH;
    int first; // this lane's place among the chunks of the first instruction
    uint32_t at0;
    __device__ __forceinline__ void init(int w, int lane, int d)
    {
        first = w * 64 + lane;
        at0 = at(first, d);
    }
    static __device__ __forceinline__ uint32_t at(int place, int d) // byte in its row of the chunk that belongs to a place
    {
        return min((place % CH) ^ AttnTile<DP>::swizzle(place / CH), d / 8 - 1) * 16;
    }
    // rows row0 .. of the head that starts at `head` (uniform); row0 <= last
    __device__ __forceinline__ void issue(const char *head, uint32_t token_stride, int row0, int last, uint32_t tile, int w, int d) const
    {
        const char *base = head + (uint64_t)(uint32_t)row0 * token_stride;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (N % NW != 0 && w + NW * i >= N)
                break;
            const int place = first + NW * 64 * i, r = EVEN ? first / CH + STEP * i : place / CH;
            attn_load_lds16<ONCE>(base, (uint32_t)min(r, last - row0) * token_stride + (EVEN ? at0 : at(place, d)), tile + (w + NW * i) * 1024);
        }
    }
};

// Waits until this wavefront's copies are in LDS and everybody has come here
__device__ __forceinline__ void attn_arrive()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int DT> __device__ __forceinline__ void attn_mma(const uint4 &a, const uint4 &b, f32x16 &c) { Traits<fmt(DT, 8)>::mma(a, b, c); }

template <int DT> __device__ __forceinline__ uint32_t attn_pack2(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 x = {a, b};
    if constexpr (DT == MAXSIM_F16) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
    } else {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
    }
}
template <int DT> __device__ __forceinline__ float attn_float(uint32_t bits16)
{
    if constexpr (DT == MAXSIM_F16)
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
    else
        return __uint_as_float(bits16 << 16);
}
// Registers 8 s .. 8 s + 7 of a result as the B operand of step s (rounded to nearest even, 16 bits)
template <int DT> __device__ __forceinline__ uint4 attn_operand(const f32x16 &x, int s)
{
    return make_uint4(attn_pack2<DT>(x[8 * s], x[8 * s + 1]), attn_pack2<DT>(x[8 * s + 2], x[8 * s + 3]), attn_pack2<DT>(x[8 * s + 4], x[8 * s + 5]),
                      attn_pack2<DT>(x[8 * s + 6], x[8 * s + 7]));
}

// Where a lane reads a tile's rows as they lie (A operand, chunk 2 u + h of row `32 block + c`)
template <int DP> struct AttnRowRead {
    int base, swz;
    __device__ __forceinline__ AttnRowRead(int lane) : base((lane & 31) * AttnTile<DP>::ROW), swz(AttnTile<DP>::swizzle(lane & 31) ^ (lane >> 5)) {}
    __device__ __forceinline__ uint4 get(const char *tile, int block, int u) const
    {
        return *reinterpret_cast<const uint4 *>(tile + block * 32 * AttnTile<DP>::ROW + base + (((2 * u) ^ swz) << 4));
    }
};

// Where a lane reads a tile transposed (A operand: row m = entry 32 block + m of d, k = tile rows 16 s + 4 h + {0 .. 3, 8 .. 11})
template <int DP> struct AttnColRead {
    int base, chunk;
    __device__ __forceinline__ AttnColRead(int lane)
    {
        const int i = lane & 15, h = lane >> 5, r = 4 * h + (i >> 2);
        base = r * AttnTile<DP>::ROW + 8 * (i & 1);
        chunk = (2 * ((lane >> 4) & 1) + ((i >> 1) & 1)) ^ AttnTile<DP>::swizzle(r);
    }
    __device__ __forceinline__ uint4 get(const char *tile, int block, int s) const
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        const char *at = tile + s * 16 * AttnTile<DP>::ROW + base;
        // (eight rows on, the swizzle differs in bit 1)
        const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + (((4 * block) ^ chunk) << 4))));
        const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * AttnTile<DP>::ROW + (((4 * block + 2) ^ chunk) << 4))));
        return make_uint4(x.x, x.y, y.x, y.y);
    }
};

// Over the two halves of a wavefront: the same in both
__device__ __forceinline__ float attn_halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float attn_halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A lane's part of a row of 16-bit values as the B operand (chunk 2 u + h in step u), zeros past the row's end
template <int U> __device__ __forceinline__ void attn_load_row(const char *row, int d, int h, uint4 (&x)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u)
        x[u] = *reinterpret_cast<const uint4 *>(row + min(2 * u + h, d / 8 - 1) * 16);
}
// ... and its arrival: before the loop, or the compiler waits in it
template <int U> __device__ __forceinline__ void attn_have_row(int d, int h, uint4 (&x)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = (2 * u + h) * 8 < d;
        x[u] = make_uint4(in ? x[u].x : 0, in ? x[u].y : 0, in ? x[u].z : 0, in ? x[u].w : 0);
        asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
    }
}

// Four consecutive entries of a row
template <int DT> __device__ __forceinline__ void attn_store4(char *row, int entry, float a, float b, float c, float d)
{
    *reinterpret_cast<uint2 *>(row + entry * 2) = make_uint2(attn_pack2<DT>(a, b), attn_pack2<DT>(c, d));
}

// A wavefront's result, 32 columns of `by` times x, as rows of 16-bit values: through 32 rows of LDS of its own, so that a store takes whole
// rows instead of 8 bytes of 32 of them. place(r): where row r < n goes.
template <int DT, int DP, class Place> __device__ __forceinline__ void attn_store_tile(char *lds, const f32x16 (&x)[DP / 32], float by, int lane, int d, int n, Place &&place)
{
    typedef AttnTile<DP> T;
    const int c = lane & 31, h = lane >> 5;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<uint2 *>(lds + c * T::ROW + (((4 * b + r / 4) ^ T::swizzle(c)) << 4) + 8 * h) =
                make_uint2(attn_pack2<DT>(x[b][r] * by, x[b][r + 1] * by), attn_pack2<DT>(x[b][r + 2] * by, x[b][r + 3] * by));
#pragma unroll
    for (int k = 0; k < T::CH / 2; ++k) {
        const int row = (k * 64 + lane) / T::CH, chunk = (k * 64 + lane) % T::CH;
        const uint4 v = *reinterpret_cast<const uint4 *>(lds + row * T::ROW + ((chunk ^ T::swizzle(row)) << 4));
        if (row < n && chunk * 8 < d)
            *reinterpret_cast<uint4 *>(place(row) + chunk * 16) = v;
    }
}

// f(integral_constant DP) for the smallest compiled width that holds d
template <class F> hipError_t attn_width(int d, F &&f)
{
    if (d <= 32)
        return f(std::integral_constant<int, 32>{});
    if (d <= 64)
        return f(std::integral_constant<int, 64>{});
    if (d <= 96)
        return f(std::integral_constant<int, 96>{});
    if (d <= 128)
        return f(std::integral_constant<int, 128>{});
    return f(std::integral_constant<int, 256>{});
}
constexpr int ATTN_WIDEST = 256;
// Keys (or query rows) of a tile in LDS, so that two tiles of two tensors take 64 KB at most
constexpr int attn_tile(int dp) { return dp > 128 ? 32 : 64; }

} // namespace maxsim
