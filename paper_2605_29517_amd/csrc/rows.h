// Rows of tensors in memory, entry by entry or in pieces of up to 32 bytes, for the kernels of the encoder's operators (not part of the public ABI).
#pragma once
#include "common.h"

namespace maxsim {

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
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// V entries at any address that is a multiple of their size, in as few pieces as 16 bytes allow (the memory pipes take any address; a piece
// that crosses a line takes two of its turns); ONCE: that the caches need not keep
template <class T, int V, bool ONCE = false> __device__ __forceinline__ Pack<T, V> load_row(const T *p)
{
    Pack<T, V> r;
    if constexpr (V == 1) {
        r.x[0] = *p;
    } else if constexpr (sizeof r == 4) {
        const u32_any *at = reinterpret_cast<const u32_any *>(p);
        r = __builtin_bit_cast(Pack<T, V>, ONCE ? __builtin_nontemporal_load(at) : *at);
    } else if constexpr (sizeof r == 8) {
        const u32x2_any *at = reinterpret_cast<const u32x2_any *>(p);
        r = __builtin_bit_cast(Pack<T, V>, ONCE ? __builtin_nontemporal_load(at) : *at);
    } else {
        static_assert(sizeof r % 16 == 0, "pieces of 16 bytes");
        struct Raw {
            u32x4 x[sizeof r / 16];
        } raw;
        const u32x4_any *at = reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
        for (unsigned i = 0; i < sizeof r / 16; ++i)
            raw.x[i] = ONCE ? __builtin_nontemporal_load(at + i) : at[i];
        r = __builtin_bit_cast(Pack<T, V>, raw);
    }
    return r;
}
template <bool ONCE = false, class T, int V> __device__ __forceinline__ void store_row(T *p, const Pack<T, V> &r)
{
    if constexpr (V == 1) {
        *p = r.x[0];
    } else if constexpr (sizeof r == 4) {
        u32_any *at = reinterpret_cast<u32_any *>(p);
        const u32_any v = __builtin_bit_cast(uint32_t, r);
        if constexpr (ONCE)
            __builtin_nontemporal_store(v, at);
        else
            *at = v;
    } else if constexpr (sizeof r == 8) {
        u32x2_any *at = reinterpret_cast<u32x2_any *>(p);
        const u32x2_any v = __builtin_bit_cast(u32x2_any, r);
        if constexpr (ONCE)
            __builtin_nontemporal_store(v, at);
        else
            *at = v;
    } else {
        static_assert(sizeof r % 16 == 0, "pieces of 16 bytes");
        struct Raw {
            u32x4 x[sizeof r / 16];
        };
        const Raw raw = __builtin_bit_cast(Raw, r);
        u32x4_any *at = reinterpret_cast<u32x4_any *>(p);
#pragma unroll
        for (unsigned i = 0; i < sizeof r / 16; ++i) {
            if constexpr (ONCE)
                __builtin_nontemporal_store((u32x4_any)raw.x[i], at + i);
            else
                at[i] = raw.x[i];
        }
    }
}

// From so many bytes read and written on, the next kernel finds little of them in the caches (256 MB before the memory): then they are
// moved past them.
constexpr int64_t STREAM_BYTES = int64_t(128) << 20;
// Where a program runs through several tensors in turn the hint pays later: norms of 168 MB 52 us without it and 55 with it, of 336 MB 77 and 75.
constexpr int64_t PAST_CACHES = int64_t(256) << 20;

// x / d by a multiplication, for x d < 2^32 (beyond, a quotient may be one too high: who launches the kernel sees to it)
struct Divisor {
    uint32_t d, m;

    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by), m(by == 1 ? 0 : (uint32_t)(((uint64_t(1) << 32) + by - 1) / by)) {}
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return m ? __umulhi(x, m) : x; }
    static bool divides_below(int64_t n, int64_t by) { return n * by <= int64_t(1) << 32; } // all x < n
};

} // namespace maxsim
