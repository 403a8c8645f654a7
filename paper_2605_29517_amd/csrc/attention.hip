// Attention over packed sequences, forward: O = softmax(scale Q K^T + mask) V and the logarithm of the softmax's sum.
//
// One pass over the keys with a running maximum and sum (in 32 bits): a workgroup owns ROWS rows (a row: one token of one query
// head; the heads that share keys lie side by side, so that a token's whole group reads K and V once), a wavefront 32 of them, and
// walks the keys in tiles of 64 that are copied to LDS one tile ahead. P is rounded to the inputs' 16-bit type for the second
// product (relative error 2^-9 in bf16, 2^-12 in fp16, no more than the rounding of the output; the sum that divides it
// stays in 32 bits).
#include "attention.h"

namespace maxsim {
namespace {

constexpr int TILE = 64;                // keys per step
constexpr float NO_MAXIMUM = -1.0e30f;  // of a row that has seen no key: finite, so that no difference of infinities arises
constexpr float LAZY = 8.0f;            // the maximum may lag by this many powers of two: P <= 2^8, far from overflow in fp16

template <int DT, int DP, int NW> __global__ void __launch_bounds__(NW * 64, 2) attn_fwd_kernel(AttnParams p)
{
    constexpr int ROWS = NW * 32, U = DP / 16, NB = DP / 32;
    constexpr int TILE_BYTES = TILE * DP * 2;
    __shared__ __attribute__((aligned(16))) char lds[4 * TILE_BYTES]; // two of K, two of V

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Every XCD takes a contiguous range of (kv head, tile, piece): tiles that read the same keys meet in one L2. The last tiles, which see
    // the most keys under a causal mask, come first.
    int v = xcd_grouped(blockIdx.x, gridDim.x);
    const int piece = v % p.n_split;
    v /= p.n_split;
    const int slot = p.n_slots - 1 - v % p.n_slots, hk = v / p.n_slots;

    const int64_t i = attn_find_slot(p.q_off, p.b, p.q_tokens, p.pack, ROWS, slot);
    const AttnSeq q = attn_seq(p.q_off, i, p.q_tokens), k = attn_seq(p.k_off, i, p.k_tokens);
    const int64_t first = (int64_t)(slot - attn_first_slot(p.q_off, i, p.q_tokens, p.pack, ROWS)) * ROWS, rows = (int64_t)q.len * p.pack;
    if (first < 0 || first >= rows)
        return;

    // this lane's row: the same in both halves
    const int64_t row = first + w * 32 + (lane & 31);
    const int64_t row_ok = min(row, rows - 1);
    const int token = (int)(row_ok / p.pack);
    const int head = hk * p.pack + (int)(row_ok % p.pack);
    const int ahead = k.len - q.len; // query t sees the keys up to t + ahead
    const int limit = p.causal ? max(0, min(k.len, token + ahead + 1)) : k.len;
    // keys that the rows of the workgroup and of the wavefront see, and those that all rows of the wavefront see
    const int64_t wg_last = min(first + ROWS, rows) - 1;
    const int wg_keys = p.causal ? max(0, min(k.len, (int)(wg_last / p.pack) + ahead + 1)) : k.len;
    const int wave_keys = __builtin_amdgcn_readlane(limit, 31), all_keys = __builtin_amdgcn_readfirstlane(limit);

    uint4 qf[U];
    const char *q_row = p.Q.p + (q.start + token) * p.Q.token + head * p.Q.head;
    attn_load_row(q_row, p.d, h, qf);

    const char *k_head = p.K.p + k.start * p.K.token + hk * p.K.head, *v_head = p.V.p + k.start * p.V.token + hk * p.V.head;
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
    float top = NO_MAXIMUM, sum = 0.0f;

    const int tiles = (wg_keys + TILE - 1) / TILE;
    const int t0 = (int)((int64_t)tiles * piece / p.n_split), t1 = (int)((int64_t)tiles * (piece + 1) / p.n_split);
    auto issue = [&](int t) {
        const uint32_t to = attn_lds(lds) + (t & 1) * 2 * TILE_BYTES;
        copy.issue(k_head, p.K.token, t * TILE, k.len - 1, to, w);
        copy.issue(v_head, p.V.token, t * TILE, k.len - 1, to + TILE_BYTES, w);
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
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[b][r] = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
                attn_mma<DT>(k_read.get(kt, b, u), qf[u], s[b]);
        }
        if (key0 + TILE > all_keys) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[b][r] = key0 + 32 * b + acc_row(r, h) < limit ? s[b][r] : neg_inf();
        }
        float m = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                m = fmaxf(m, s[b][r]);
        m = attn_halves_max(m) * p.scale_log2;
        // A maximum that grows by less than 2^LAZY is left where it is (the result is the same whatever number is subtracted)
        if (__builtin_amdgcn_ballot_w64(m > top + LAZY)) {
            const float to = fmaxf(m, top), by = __builtin_amdgcn_exp2f(top - to);
            top = to;
            sum *= by;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[b][r] *= by;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], p.scale_log2, -top));
                sum += s[b][r];
            }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 pf = attn_operand<DT>(s[b], x);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    attn_mma<DT>(v_read.get(vt, nb, 2 * b + x), pf, o[nb]);
            }
    }

    sum = attn_halves_sum(sum);
    if (row >= rows)
        return;
    const bool seen = sum > 0.0f;
    const float by = seen ? 1.0f / sum : 0.0f;
    const float lse = seen ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : neg_inf();
    const int64_t at = (q.start + token) * p.hq + head;
    if (p.n_split > 1) {
        float *part = p.part_o + ((int64_t)piece * p.q_tokens * p.hq + at) * p.d;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                if (32 * b + 2 * r + 4 * h < p.d)
                    *reinterpret_cast<float4 *>(part + 32 * b + 2 * r + 4 * h) = make_float4(o[b][r] * by, o[b][r + 1] * by, o[b][r + 2] * by, o[b][r + 3] * by);
        if (h == 0)
            p.part_lse[(int64_t)piece * p.q_tokens * p.hq + at] = lse;
        return;
    }
    char *o_row = p.O.p + (q.start + token) * p.O.token + head * p.O.head;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            if (32 * b + 2 * r + 4 * h < p.d)
                attn_store4<DT>(o_row, 32 * b + 2 * r + 4 * h, o[b][r] * by, o[b][r + 1] * by, o[b][r + 2] * by, o[b][r + 3] * by);
    if (p.lse && h == 0)
        p.lse[at] = lse;
}

// Joins the pieces: weights exp(lse_piece - lse), a thread per four entries of a row
template <int DT> __global__ void __launch_bounds__(256) attn_join_kernel(AttnParams p)
{
    const int64_t n = p.q_tokens * p.hq;
    const int per = p.d / 4;
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, at = x / per;
    const int e = (int)(x % per) * 4;
    if (at >= n)
        return;
    float top = neg_inf();
    for (int s = 0; s < p.n_split; ++s)
        top = fmaxf(top, p.part_lse[s * n + at]);
    float sum = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (top > neg_inf())
        for (int s = 0; s < p.n_split; ++s) {
            const float by = __builtin_amdgcn_exp2f((p.part_lse[s * n + at] - top) * 1.44269504088896341f);
            const float4 y = *reinterpret_cast<const float4 *>(p.part_o + (s * n + at) * p.d + e);
            sum += by;
            o[0] += by * y.x;
            o[1] += by * y.y;
            o[2] += by * y.z;
            o[3] += by * y.w;
        }
    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
    const int64_t token = at / p.hq;
    const int head = (int)(at % p.hq);
    attn_store4<DT>(p.O.p + token * p.O.token + head * p.O.head, e, o[0] * by, o[1] * by, o[2] * by, o[3] * by);
    if (p.lse && e == 0)
        p.lse[at] = sum > 0.0f ? top + __builtin_amdgcn_logf(sum) * 0.69314718055994531f : neg_inf();
}

struct AttnPlan {
    int pack, n_slots, n_split;
};
constexpr int NW = 4;

AttnPlan attn_plan(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int num_cu)
{
    AttnPlan x;
    x.pack = hq / hkv;
    const int64_t slots = q_tokens * x.pack / (NW * 32) + b;
    x.n_slots = (int)slots;
    // pieces of the keys where the workgroups would leave compute units idle: as many as fill them twice, of at least four tiles of an average sequence
    const int64_t busy = slots * hkv, mean = k_tokens / b / TILE;
    int64_t split = busy >= num_cu ? 1 : (2 * num_cu + busy - 1) / busy;
    split = std::min<int64_t>(split, mean / 4);
    x.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(split, 64));
    return x;
}

} // namespace

int64_t attention_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu)
{
    const AttnPlan x = attn_plan(b, q_tokens, k_tokens, hq, hkv, num_cu);
    return x.n_split > 1 ? x.n_split * q_tokens * hq * (int64_t)(d + 1) * 4 : 0;
}

hipError_t attention_launch(AttnParams p, int dtype, void *workspace, int num_cu, hipStream_t stream)
{
    const AttnPlan x = attn_plan(p.b, p.q_tokens, p.k_tokens, p.hq, p.hkv, num_cu);
    p.pack = x.pack;
    p.n_slots = x.n_slots;
    p.n_split = x.n_split;
    p.part_o = static_cast<float *>(workspace);
    p.part_lse = p.part_o + (x.n_split > 1 ? x.n_split * p.q_tokens * p.hq * (int64_t)p.d : 0);
    const unsigned grid = (unsigned)(x.n_slots * p.hkv * x.n_split);
    const hipError_t e = attn_width(p.d, [&](auto dp) {
        if (dtype == MAXSIM_F16)
            attn_fwd_kernel<MAXSIM_F16, decltype(dp)::value, NW><<<grid, NW * 64, 0, stream>>>(p);
        else
            attn_fwd_kernel<MAXSIM_BF16, decltype(dp)::value, NW><<<grid, NW * 64, 0, stream>>>(p);
        return hipGetLastError();
    });
    if (e != hipSuccess || x.n_split == 1)
        return e;
    const unsigned join = (unsigned)((p.q_tokens * p.hq * (p.d / 4) + 255) / 256);
    if (dtype == MAXSIM_F16)
        attn_join_kernel<MAXSIM_F16><<<join, 256, 0, stream>>>(p);
    else
        attn_join_kernel<MAXSIM_BF16><<<join, 256, 0, stream>>>(p);
    return hipGetLastError();
}

} // namespace maxsim
