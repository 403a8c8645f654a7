// Attention over packed sequences, forward: O = softmax(scale Q K^T + mask) V and the logarithm of the softmax's sum.
//
// One pass over the keys with a running maximum and sum (in 32 bits): a workgroup owns ROWS rows (a row: one token of one query
// head; the heads that share keys lie side by side, so that a token's whole group reads K and V once), a wavefront 32 of them, and
// walks the keys in tiles of 64 (32 at d = 256) that are copied to LDS one tile ahead. P is rounded to the inputs' 16-bit type for the second
// product (relative error at most 2^-8 in bf16, 2^-11 in fp16 and the 2^-32 of the largest weight that stand at LIFT: no more than the rounding of the
// output, of any size up to 2^21 keys; the sum that divides it stays in 32 bits).
#include "attention.h"

#include <cmath>

namespace maxsim {
namespace {

constexpr float NO_MAXIMUM = -3.4028234664e38f; // of a row that has seen no key, the lowest finite number, so that no difference of infinities arises
constexpr float LAZY = 8.0f;                    // the maximum may lag by this many powers of two
// fp16 has no normal numbers below 2^-14 and none below 2^-24, while the sum in 32 bits counts every weight: P are taken 2^7 times as large, which with
// LAZY is at most 2^15. Then a weight is off by its rounding and by 2^-32 of the largest at most (2^-25 without): of one key and 10^5 others of 2^-26 of its
// weight 10^-5 of the result is lost instead of all that the others make, 10^-3.
template <int DT> constexpr float LIFT = DT == MAXSIM_F16 ? 7.0f : 0.0f;
// P = exp2(scale_log2 S - scale_log2 top) by one fma, with top among the scores S as they are. The fma's product is exact and the number that it
// subtracts is rounded, so that all of a row's P are off by one factor, which the sum that divides them shares: 2^-4 of an exponent at
// FAR, but more than P can hold from 2^28 on. Further out than FAR the difference is taken first: scores of +-10^38 (bf16) are told apart as fp32 tells them.
// (In the branch that moves the maximum, which such rows take at every step: as a branch of its own, the prompt's kernel copied its scores around it, and
// 16 sequences of 9 to 130 new tokens took 133 us instead of 120.)
constexpr float FAR = 1048576.0f;

// The softmax's sum, of which a row has up to millions of terms that may round alike (equal keys): a step's terms are added as a tree, and the steps with
// what the last addition lost. Added one by one, 2^17 equal keys put lse 226 times as far off as the rounding of the scores may; so it is half of
// that, for 1 to 2 % of the time (250 short texts 71.2 -> 72.2 us, a long prompt 546 -> 547, 16 x 1024 tokens of heads of 256 159 -> 162).
struct AttnSum {
    float sum, lost; // sum - lost is the value
    __device__ __forceinline__ void add(float x)
    {
        const float y = x - lost, t = sum + y;
        lost = (t - sum) - y;
        sum = t;
    }
    __device__ __forceinline__ void scale(float by)
    {
        sum *= by;
        lost *= by;
    }
};
template <int N> __device__ __forceinline__ float attn_tree(const float *x)
{
    if constexpr (N == 1)
        return x[0];
    else
        return attn_tree<N / 2>(x) + attn_tree<N - N / 2>(x + N / 2);
}
__device__ __forceinline__ float attn_tree(const f32x16 &x)
{
    float y[16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
        y[r] = x[r];
    return attn_tree<16>(y);
}

// Of a row that sees keys
template <int DT> __device__ __forceinline__ float attn_lse(const AttnParams &p, float top, float sum)
{
    return __builtin_fmaf(top, p.scale, (__builtin_amdgcn_logf(sum) - LIFT<DT>) * 0.69314718055994531f);
}

// A column's result: O = o / sum and lse, or the same of a piece. `seen`: that there is a key, which the mask says and not the sum, so that a sum which
// is not a number shows in lse (with NaNs not honoured by the compiler a comparison of it would say anything).
template <int DT, int NB> __device__ __forceinline__ void attn_write(const AttnParams &p, const f32x16 (&o)[NB], float lse, float sum, bool seen, int piece, int token, int head, int h)
{
    const float by = seen ? 1.0f / sum : 0.0f;
    lse = seen ? lse : neg_inf();
    const int at = token * p.hq + head;
    if (p.n_split > 1) {
        float *part = p.part_o + ((int64_t)piece * (p.q_tokens * p.hq) + at) * p.d;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                if (32 * b + 2 * r < p.d)
                    *reinterpret_cast<float4 *>(part + 32 * b + 2 * r + 4 * h) = make_float4(o[b][r] * by, o[b][r + 1] * by, o[b][r + 2] * by, o[b][r + 3] * by);
        if (h == 0)
            p.part_lse[(int64_t)piece * (p.q_tokens * p.hq) + at] = lse;
        return;
    }
    char *row = p.O.p + (uint64_t)(uint32_t)token * p.O.token + head * p.O.head;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            if (32 * b + 2 * r < p.d)
                attn_store4<DT>(row, 32 * b + 2 * r + 4 * h, o[b][r] * by, o[b][r + 1] * by, o[b][r + 2] * by, o[b][r + 3] * by);
    if (p.lse && h == 0)
        p.lse[at] = lse;
}

// Long sequences are bound by the matrix units under the power limit: one causal prompt of 8192 tokens, 32 heads of 128 over 8, 519 us, 545 on a
// warm card (1010-1060 TFLOP/s; compute units 93 % busy, their matrix units 59 % of that at 1.8 of 2.4 GHz), 16 x 1024 tokens of 8 heads of 256 over one 162 us (850).
// Short ones are bound by latency and by the exponentials: 250 texts of 64 to 300 tokens, 12 heads of 64, 72-80 us. Two workgroups of four wavefronts to a
// compute unit (four at d <= 64): eight wavefronts to a tile of K and V take 2 % off long sequences and put 7 % on such texts.
// B, the blocks of 32 keys between two looks at the maximum: 2 hides more behind the products where the registers allow it (d = 128: prompt 518 us,
// 523 with 1; 16 sequences of 9 to 130 new tokens 125 and 127; 500 texts of 150 tokens at d = 64 115 with 1, 122 with 2; d = 32 70 and 76).
template <int DT, int DP, int NW> __global__ void __launch_bounds__(NW * 64, DP > 64 ? 2 : 4) attn_fwd_kernel(AttnParams p)
{
    constexpr int ROWS = NW * 32, U = DP / 16, NB = DP / 32, TILE = attn_tile(DP);
    constexpr int B = DP == 96 || DP == 128 ? 2 : 1;
    constexpr int TILE_BYTES = TILE * DP * 2;
    __shared__ __attribute__((aligned(16))) char lds[4 * TILE_BYTES]; // two of K, two of V

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Every XCD takes a contiguous range of (kv head, tile, piece): tiles that read the same keys meet in one L2 (prompt of 8192 tokens
    // 538 us, tile by tile over all heads 955). The last tiles, which see the most keys under a causal mask, come first.
    const int wg = blockIdx.y * (int)GRID_ROW + blockIdx.x; // (those from n_wg on leave below, with the slots that no sequence has: by then the wait for the arguments has passed)
    int v = xcd_grouped(wg, p.n_wg), u = p.by_split(v);
    const int piece = v, hk = p.by_slots(u), slot = p.n_slots - 1 - u;

    const AttnPlace place = attn_find_slot<ROWS>(p.q_off, p.b, p.q_tokens, p.pack, slot, p.n_slots);
    const AttnSeq q = place.s, k = p.same ? q : attn_seq(p.k_off, place.i, p.k_tokens);
    const int first = (slot - place.first) * ROWS, rows = q.len * p.pack;
    if (wg >= p.n_wg || first < 0 || first >= rows)
        return;

    // this lane's row: the same in both halves
    const int row = first + w * 32 + (lane & 31);
    int head = min(row, rows - 1);
    const int token = p.by_pack(head);
    head += hk * p.pack;
    const int ahead = k.len - q.len; // query t sees the keys up to t + ahead
    const int limit = p.causal ? max(0, min(k.len, token + ahead + 1)) : k.len;
    // keys that the rows of the workgroup and of the wavefront see, and those that all rows of the wavefront see
    const int wg_keys = p.causal ? max(0, min(k.len, p.by_pack.quotient(min(first + ROWS, rows) - 1) + ahead + 1)) : k.len;
    const int wave_keys = first + w * 32 < rows ? __builtin_amdgcn_readlane(limit, 31) : 0, all_keys = __builtin_amdgcn_readfirstlane(limit);

    uint4 qf[U];
    const char *q_row = p.Q.p + (uint64_t)(uint32_t)(q.start + token) * p.Q.token + head * p.Q.head;
    attn_load_row(q_row, p.d, h, qf);

    const char *k_head = p.K.p + (uint64_t)(uint32_t)k.start * p.K.token + hk * p.K.head, *v_head = p.V.p + (uint64_t)(uint32_t)k.start * p.V.token + hk * p.V.head;
    AttnCopy<DP, TILE, NW> copy;
    copy.init(w, lane, p.d);
    const AttnRowRead<DP> k_read(lane);
    const AttnColRead<DP> v_read(lane);

    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[b][r] = 0.0f;
    float top = NO_MAXIMUM, less = 0.0f; // the maximum, and what is subtracted
    uint64_t far = 0; // rows of the wavefront that are
    AttnSum sums = {0.0f, 0.0f};

    const int tiles = (wg_keys + TILE - 1) / TILE;
    int over = tiles;
    const int per = p.by_split(over), t0 = per * piece + min(piece, over), t1 = t0 + per + (piece < over);
    auto issue = [&](int t) {
        const uint32_t to = attn_lds(lds) + (t & 1) * 2 * TILE_BYTES;
        copy.issue(k_head, p.K.token, t * TILE, k.len - 1, to, w, p.d);
        copy.issue(v_head, p.V.token, t * TILE, k.len - 1, to + TILE_BYTES, w, p.d);
    };
    // B blocks of 32 keys of a tile; key0: the first of them
    auto step = [&](const char *kt, const char *vt, int key0) {
        f32x16 s[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[b][r] = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
                attn_mma<DT>(k_read.get(kt, b, u), qf[u], s[b]);
        }
        if (key0 + 32 * B > all_keys) {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[b][r] = key0 + 32 * b + acc_row(r, h) < limit ? s[b][r] : neg_inf();
        }
        float m = s[0][0];
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                m = fmaxf(m, s[b][r]);
        m = attn_halves_max(m);
        // A maximum that grows by less than 2^LAZY is left where it is (the result is the same whatever number is subtracted)
        if (far | __builtin_amdgcn_ballot_w64((m - top) * p.scale_log2 > LAZY)) {
            const float to = fmaxf(m, top), by = __builtin_amdgcn_exp2f((top - to) * p.scale_log2);
            top = to;
            less = __builtin_fmaf(top, p.scale_log2, -LIFT<DT>);
            sums.scale(by);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[b][r] *= by;
            far = __builtin_amdgcn_ballot_w64(fabsf(less) > FAR);
            if (far) {
                less = -LIFT<DT>;
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[b][r] -= top;
            }
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], p.scale_log2, -less));
        float part[B];
#pragma unroll
        for (int b = 0; b < B; ++b)
            part[b] = attn_tree(s[b]);
        sums.add(attn_tree<B>(part));
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 pf = attn_operand<DT>(s[b], x);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    attn_mma<DT>(v_read.get(vt, nb, 2 * b + x), pf, o[nb]);
            }
    };
    if (t0 < t1)
        issue(t0);
    attn_have_row(p.d, h, qf);
    for (int t = t0; t < t1; ++t) {
        attn_arrive();
        if (t + 1 < t1)
            issue(t + 1);
        const char *kt = lds + (t & 1) * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
        const int key0 = t * TILE;
        if (key0 >= wave_keys)
            continue;
#pragma unroll
        for (int b = 0; b < TILE / 32; b += B)
            if (b == 0 || key0 + 32 * b < wave_keys)
                step(kt + b * 32 * DP * 2, vt + b * 32 * DP * 2, key0 + 32 * b);
    }

    const float sum = attn_halves_sum(sums.sum - sums.lost);
    if (p.n_split > 1) {
        if (row < rows)
            attn_write<DT>(p, o, attn_lse<DT>(p, top, sum), sum, limit > t0 * TILE, piece, q.start + token, head, h);
        return;
    }
    __syncthreads(); // (nobody reads the tiles any more)
    const bool seen = limit > 0; // (as in attn_write)
    attn_store_tile<DT, DP>(lds + w * 32 * DP * 2, o, seen ? 1.0f / sum : 0.0f, lane, p.d, rows - first - w * 32, [&](int r) {
        int g = first + w * 32 + r;
        const uint32_t t = q.start + p.by_pack(g);
        return p.O.p + (uint64_t)t * p.O.token + (hk * p.pack + g) * p.O.head;
    });
    if (p.lse && h == 0 && row < rows)
        p.lse[(q.start + token) * p.hq + head] = seen ? attn_lse<DT>(p, top, sum) : neg_inf();
}

// The same for few rows per sequence (single tokens against kept keys): what counts is that keys and values stream at the memory's
// rate. A wavefront owns all 32 rows of the workgroup and every NF-th tile of 32 keys of the piece, which it copies to a ring in
// LDS of its own, RING tiles of K and of V ahead: nothing waits for another wavefront, and two workgroups keep 100 KB on their way to a compute
// unit. The wavefronts' results are joined through LDS at the end. Bound by the memory: one token after each of 64 x 2048 .. 8192 keys, 8
// heads of 128 (1.4 GB), 244 us, 5.9 TB/s; one token after 100003 keys of two heads (102 MB) 20-21 us and 6 for the join.
// Workgroups go round the XCDs one by one: in contiguous ranges, as in the other kernel, unequal sequences load the XCDs unequally
// (16 sequences of 500 .. 16000 keys 117 us, 87 so; 32 x 4000 keys of 16 heads 181 and 164).
constexpr int NF = 2;
template <int DT, int DP> __global__ void __launch_bounds__(NF * 64, 1) attn_few_kernel(AttnParams p)
{
    constexpr int U = DP / 16, NB = DP / 32;
    constexpr int KEYS = 32, TILE_BYTES = KEYS * DP * 2, RING = 16384 / TILE_BYTES, LOADS = TILE_BYTES / 1024;
    __shared__ __attribute__((aligned(16))) char lds[NF * RING * 2 * TILE_BYTES];

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (the heads of a piece, whose rows lie side by side, run at the same time)
    const int wg = blockIdx.y * (int)GRID_ROW + blockIdx.x;
    int v = wg, u = p.by_hkv(v);
    const int hk = v, slot = p.by_split(u), piece = u;

    const AttnPlace place = attn_find_slot<32>(p.q_off, p.b, p.q_tokens, p.pack, slot, p.n_slots);
    const AttnSeq q = place.s, k = p.same ? q : attn_seq(p.k_off, place.i, p.k_tokens);
    const int first = (slot - place.first) * 32, rows = q.len * p.pack;
    if (wg >= p.n_wg || first < 0 || first >= rows)
        return;
    const int row = first + (lane & 31);
    int head = min(row, rows - 1);
    const int token = p.by_pack(head);
    head += hk * p.pack;
    const int ahead = k.len - q.len;
    const int limit = p.causal ? max(0, min(k.len, token + ahead + 1)) : k.len;
    const int wave_keys = __builtin_amdgcn_readlane(limit, 31), all_keys = __builtin_amdgcn_readfirstlane(limit);

    const char *k_head = p.K.p + (uint64_t)(uint32_t)k.start * p.K.token + hk * p.K.head, *v_head = p.V.p + (uint64_t)(uint32_t)k.start * p.V.token + hk * p.V.head;
    AttnCopy<DP, KEYS, 1, true> copy;
    copy.init(0, lane, p.d);
    const AttnRowRead<DP> k_read(lane);
    const AttnColRead<DP> v_read(lane);

    const int tiles = (wave_keys + KEYS - 1) / KEYS;
    int over = tiles;
    const int per = p.by_split(over), start = per * piece + min(piece, over), t0 = start + w, t1 = start + per + (piece < over);
    const int n = t0 < t1 ? (t1 - t0 + NF - 1) / NF : 0; // tiles of this wavefront: t0, t0 + NF, ...
    char *ring = lds + w * RING * 2 * TILE_BYTES;
    auto issue_k = [&](int j) { copy.issue(k_head, p.K.token, (t0 + NF * j) * KEYS, k.len - 1, attn_lds(ring) + (j % RING) * 2 * TILE_BYTES, 0, p.d); };
    auto issue_v = [&](int j) { copy.issue(v_head, p.V.token, (t0 + NF * j) * KEYS, k.len - 1, attn_lds(ring) + (j % RING) * 2 * TILE_BYTES + TILE_BYTES, 0, p.d); };
    for (int j = 0; j < RING && j < n; ++j) {
        issue_k(j);
        issue_v(j);
    }
    uint4 qf[U];
    attn_load_row(p.Q.p + (uint64_t)(uint32_t)(q.start + token) * p.Q.token + head * p.Q.head, p.d, h, qf);
    attn_have_row(p.d, h, qf);

    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[b][r] = 0.0f;
    float top = NO_MAXIMUM, less = 0.0f; // the maximum, and what is subtracted
    uint64_t far = 0; // rows of the wavefront that are
    AttnSum sums = {0.0f, 0.0f};
    for (int j = 0; j < n; ++j) {
        const char *kt = ring + (j % RING) * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
        const int key0 = (t0 + NF * j) * KEYS;
        // the newest copies may stay on their way: everything after this K, and after this V
        if (j + RING - 1 < n)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((2 * RING - 1) * LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            attn_mma<DT>(k_read.get(kt, 0, u), qf[u], s);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // K has been read
        if (j + RING < n)
            issue_k(j + RING);
        if (key0 + KEYS > all_keys) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[r] = key0 + acc_row(r, h) < limit ? s[r] : neg_inf();
        }
        float m = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r)
            m = fmaxf(m, s[r]);
        m = attn_halves_max(m);
        if (far | __builtin_amdgcn_ballot_w64((m - top) * p.scale_log2 > LAZY)) {
            const float to = fmaxf(m, top), by = __builtin_amdgcn_exp2f((top - to) * p.scale_log2);
            top = to;
            less = __builtin_fmaf(top, p.scale_log2, -LIFT<DT>);
            sums.scale(by);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[b][r] *= by;
            far = __builtin_amdgcn_ballot_w64(fabsf(less) > FAR);
            if (far) {
                less = -LIFT<DT>;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] -= top;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2, -less));
        sums.add(attn_tree(s));
        if (j + RING < n)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((2 * RING - 1) * LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint4 pf = attn_operand<DT>(s, x);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                attn_mma<DT>(v_read.get(vt, nb, x), pf, o[nb]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // V has been read
        if (j + RING < n)
            issue_v(j + RING);
    }
    float sum = attn_halves_sum(sums.sum - sums.lost);

    // the others' results, when nobody reads the rings any more
    constexpr int RESULT = (NB * 16 + 2) * 64;
    static_assert((NF - 1) * RESULT * 4 <= (int)sizeof(lds), "fits the rings");
    float *results = reinterpret_cast<float *>(lds);
    __syncthreads();
    if (w > 0) {
        float *mine = results + (w - 1) * RESULT + lane;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mine[(b * 16 + r) * 64] = o[b][r];
        mine[NB * 16 * 64] = top;
        mine[(NB * 16 + 1) * 64] = sum;
    }
    __syncthreads();
    if (w > 0)
        return;
#pragma unroll
    for (int x = 1; x < NF; ++x) {
        const float *theirs = results + (x - 1) * RESULT + lane;
        const float top2 = theirs[NB * 16 * 64], sum2 = theirs[(NB * 16 + 1) * 64];
        const float to = fmaxf(top, top2), by = __builtin_amdgcn_exp2f((top - to) * p.scale_log2), by2 = __builtin_amdgcn_exp2f((top2 - to) * p.scale_log2);
        top = to;
        sum = sum * by + sum2 * by2;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[b][r] = o[b][r] * by + theirs[(b * 16 + r) * 64] * by2;
    }
    if (row < rows)
        attn_write<DT>(p, o, attn_lse<DT>(p, top, sum), sum, limit > start * KEYS, piece, q.start + token, head, h);
}

// Joins the pieces of a row: weights exp(lse_piece - lse). Eight lanes read 128 bytes of a piece; PIECES such groups, 1 or the 8 of a wavefront,
// take pieces of the same row in turn (many pieces of few rows spread over the chip that way).
constexpr int MOST_PIECES = 256;
template <int DT, int PIECES> __global__ void __launch_bounds__(256) attn_join_kernel(AttnParams p)
{
    static_assert(PIECES == 1 || PIECES == 8, "a lane's group or its wavefront");
    const int64_t n = (int64_t)p.q_tokens * p.hq;
    const int blocks = (p.d + 31) / 32;
    const int group = threadIdx.x >> 3, g = group % PIECES;
    const int64_t unit = ((int64_t)blockIdx.y * GRID_ROW + blockIdx.x) * (32 / PIECES) + group / PIECES;
    const bool in = unit < n * blocks;
    const int64_t at = in ? unit / blocks : 0;
    const int e = min((int)(unit % blocks) * 32 + (int)(threadIdx.x & 7) * 4, p.d - 4); // (past the row's end: its last four again)
    const float *lse = p.part_lse + at;

    float top = NO_MAXIMUM, sum = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (PIECES == 1) {
        for (int s = 0; s < p.n_split; ++s)
            top = fmaxf(top, lse[s * n]);
    } else {
        for (int s = threadIdx.x & 63; s < p.n_split; s += 64)
            top = fmaxf(top, lse[s * n]);
#pragma unroll
        for (int m = 32; m; m >>= 1)
            top = fmaxf(top, __shfl_xor(top, m, 64));
    }
    constexpr int AT_ONCE = PIECES == 1 ? 4 : 8; // loads on their way; past the last piece it is read again, for nothing
    for (int s0 = g; s0 < p.n_split; s0 += PIECES * AT_ONCE) {
        float l[AT_ONCE];
        float4 y[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int s = min(s0 + i * PIECES, p.n_split - 1);
            l[i] = lse[s * n];
            y[i] = *reinterpret_cast<const float4 *>(p.part_o + (s * n + at) * p.d + e);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const float by = s0 + i * PIECES < p.n_split ? __builtin_amdgcn_exp2f((l[i] - top) * 1.44269504088896341f) : 0.0f;
            sum += by;
            o[0] = __builtin_fmaf(by, y[i].x, o[0]);
            o[1] = __builtin_fmaf(by, y[i].y, o[1]);
            o[2] = __builtin_fmaf(by, y[i].z, o[2]);
            o[3] = __builtin_fmaf(by, y[i].w, o[3]);
        }
    }
#pragma unroll
    for (int m = 8; m < 8 * PIECES; m <<= 1) {
        sum += __shfl_xor(sum, m, 64);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] += __shfl_xor(o[i], m, 64);
    }
    if (g != 0)
        return;
    if (!in)
        return;
    const bool seen = __float_as_uint(sum) != 0; // (by its bits: a piece that is not a number makes the sum one)
    const float by = seen ? 1.0f / sum : 0.0f;
    const int64_t token = at / p.hq;
    const int head = (int)(at % p.hq);
    attn_store4<DT>(p.O.p + token * p.O.token + head * p.O.head, e, o[0] * by, o[1] * by, o[2] * by, o[3] * by);
    if (p.lse && e == 0)
        p.lse[at] = seen ? top + __builtin_amdgcn_logf(sum) * 0.69314718055994531f : neg_inf();
}

struct AttnPlan {
    int pack, n_slots, n_split;
    bool few; // attn_few_kernel
};
constexpr int NW = 4;

// Few rows per sequence and more keys and values than FEW_BYTES: attn_few_kernel. Both kernels with their best pieces, caches cold: 64 x 8192
// keys of two heads of 128 (537 MB) 98 us -> 92, ragged caches of 16 x 500 .. 16000 keys of eight heads (455 MB) 93 -> 87, of 32 x 100 .. 8000
// keys of 16 heads (1.1 GB) 194 -> 182; below, its longer start counts: one sequence of 2000 keys (2 MB) 12.1 -> 13.7, 4000 of eight heads
// (16 MB) 13.3 -> 13.8, 16 x 4000 of four heads of 64 (66 MB) 20.0 -> 21.1.
constexpr double FEW_BYTES = 1e8;

AttnPlan attn_plan(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu)
{
    AttnPlan x;
    x.pack = hq / hkv;
    const double bytes = (double)k_tokens * hkv * d * 4;
    x.few = q_tokens * x.pack <= 32 * b && bytes >= FEW_BYTES;
    const int rows = x.few ? 32 : NW * 32;
    x.n_slots = (int)(q_tokens * x.pack / rows + b);
    // Pieces of the keys: the number whose estimate is least, in microseconds. A workgroup's start takes 3, a tile of 64 keys of d = 128 1.06
    // if it has the compute unit for itself and 1.5 beside another one; the memory gives 6.4 TB/s, and pieces of unequal sequences end at
    // different times; joining takes a launch and a round trip of fp32 results. Over 28 shapes of one to 500 new tokens, 1 to 200
    // sequences and 500 to 131072 keys, equal and ragged, the choice takes 3 % longer than the best number on average and 19 % at most: one
    // token after 2000 keys of two heads 37 us in one piece, 10.8 in 12; 100 tokens after 8192 keys 141 and 27 (23 in 16 pieces).
    const double full = 2.0 * num_cu, wgs = (double)((q_tokens * x.pack + b * rows - 1) / (b * rows)) * b * hkv, tiles = std::max(1.0, (double)k_tokens / b / 64);
    const double width = (d + 32) / 160.0, join = (double)q_tokens * hq * d * 8 / 6.0e6;
    double best = 0;
    x.n_split = 1;
    const int fill = (int)(full / wgs); // the most pieces that run at the same time
    for (int n = 1, next; n <= MOST_PIECES && n <= std::max(1.0, tiles / 2) && (double)x.n_slots * hkv * n < (1 << 24); n = n < fill && fill < next ? fill : next) {
        next = n < 8 ? n + 1 : n + n / 4;
        const double rounds = std::max(1.0, wgs * n / full) + 0.2, step = 1.06 + 0.88 * std::max(0.0, std::min(1.0, wgs * n / full) - 0.5);
        const double compute = rounds * std::ceil(tiles / n) * step * width, memory = bytes / 6.4e6 * (1 + 0.2 / n);
        const double time = std::sqrt(compute * compute + memory * memory) + 3.0 * rounds + (n > 1 ? 3.0 + n * join : 0.0);
        if (n == 1 || time < best) {
            best = time;
            x.n_split = n;
        }
    }
    return x;
}

} // namespace

int64_t attention_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu)
{
    const AttnPlan x = attn_plan(b, q_tokens, k_tokens, hq, hkv, d, num_cu);
    return x.n_split > 1 ? x.n_split * q_tokens * hq * (int64_t)(d + 1) * 4 : 0;
}

hipError_t attention_launch(AttnParams p, int dtype, void *workspace, int num_cu, hipStream_t stream)
{
    const AttnPlan x = attn_plan(p.b, p.q_tokens, p.k_tokens, p.hq, p.hkv, p.d, num_cu);
    p.pack = x.pack;
    p.n_slots = x.n_slots;
    p.n_split = x.n_split;
    p.part_o = static_cast<float *>(workspace);
    p.part_lse = p.part_o + (x.n_split > 1 ? (int64_t)x.n_split * p.q_tokens * p.hq * p.d : 0);
    p.by_pack = AttnDivisor::of(x.pack);
    p.by_slots = AttnDivisor::of(x.n_slots);
    p.by_split = AttnDivisor::of(x.n_split);
    p.by_hkv = AttnDivisor::of(p.hkv);
    p.n_wg = x.n_slots * p.hkv * x.n_split;
    const dim3 grid = grid_rows(p.n_wg);
    const hipError_t e = attn_width(p.d, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        if (x.few) {
            if (dtype == MAXSIM_F16)
                attn_few_kernel<MAXSIM_F16, DP><<<grid, NF * 64, 0, stream>>>(p);
            else
                attn_few_kernel<MAXSIM_BF16, DP><<<grid, NF * 64, 0, stream>>>(p);
        } else if (dtype == MAXSIM_F16) {
            attn_fwd_kernel<MAXSIM_F16, DP, NW><<<grid, NW * 64, 0, stream>>>(p);
        } else {
            attn_fwd_kernel<MAXSIM_BF16, DP, NW><<<grid, NW * 64, 0, stream>>>(p);
        }
        return hipGetLastError();
    });
    if (e != hipSuccess || x.n_split == 1)
        return e;
    const int64_t units = (int64_t)p.q_tokens * p.hq * ((p.d + 31) / 32);
    auto join = [&](auto pieces) {
        constexpr int PIECES = decltype(pieces)::value;
        const dim3 wgs = grid_rows((units * PIECES + 31) / 32);
        if (dtype == MAXSIM_F16)
            attn_join_kernel<MAXSIM_F16, PIECES><<<wgs, 256, 0, stream>>>(p);
        else
            attn_join_kernel<MAXSIM_BF16, PIECES><<<wgs, 256, 0, stream>>>(p);
    };
    // 16 pieces of 32 rows of 128 (128 units) 19.0 us with a group for a row's pieces, 13.6 with eight; of 4800 rows (19200) 46.8 and 46.5,
    // 6 pieces of those 39.1 and 42.3, 6 of 1600 rows (6400) 35.5 and 35.7
    if (x.n_split < (units > 8192 ? 16 : 6))
        join(std::integral_constant<int, 1>{});
    else
        join(std::integral_constant<int, 8>{});
    return hipGetLastError();
}

} // namespace maxsim
