// Gradient of the attention over packed sequences.
//
// The probabilities are computed again from the scores and the kept logarithm of their sum: P = exp(scale S - lse). Two kernels, each
// of which owns what it writes, so that nothing is added in an order that changes from run to run:
//   dQ      a workgroup owns query rows and walks the keys, as the forward does: S, dP = dO V^T, dS = P (dP - delta), dQ += dS K.
//           It also leaves what the second kernel's sums start from, -lse / scale and -delta = -sum_d dO O.
//   dK, dV  a workgroup owns keys and walks the queries of all heads that share them: S, dP, dV += P^T dO, dK += dS^T Q.
// Scores and dP are thus computed twice, seven products instead of five (eight where dS is kept in two parts, nine in the exact pass); adding dQ
// up from the second kernel would need an fp32 array of dQ and atomics. P and dS are rounded to the inputs' type for the last products (as P is
// in the forward). dQ of long sequences is bound, as the forward, by the matrix units under the power limit: 4 x 4096 causal tokens of 32
// heads of 128 over 8 take 750 us (compute units 92 % busy, their matrix units 61 % of that; 5 registers of 256 are spilled at d = 128, 12 in fp16, outside the loops). dK and dV of
// these take 1160-1200, with compute units busy 78 % of the time: a sequence's key tiles go out before the next one's, and the last sequence's heaviest start late. 250 texts of
// 64 to 300 tokens, 12 heads of 64, take 112-123 and 120-133 us, bound by latency and by reading Q, K, V and dO once in each kernel (85 us each at a copy's rate).
#include "attention.h"

namespace maxsim {
namespace {

constexpr int NW = 4;
constexpr int Q_TILE = 32; // query rows per step of the dK, dV kernel
// What the rounding of O puts into delta = sum_d dO O shows in dQ and dK where rows look at few keys: their errors are up to 1.9 times
// what the rounding of the outputs alone makes, where 1.41 follows from the rounding of dS. Three things keep them at 1.1 to 1.45:
//   dK    takes delta plus the sum of dS over the row's keys, which is what delta was short of (it is zero for the right one);
//   dQ    of rows of up to EXACT_KEYS keys: delta is summed from P dP in a pass of its own, which needs no O;
//   dQ    of more keys: dS is rounded in two parts, so that delta's part is nearly all that is left; one product more, beside the same operand.
// Under a causal mask rows of more than SPLIT_KEYS_CAUSAL keys bring little of the gradient beside the first rows, and stay as they are; not so where
// keys are kept before the first row, which all see many then (256 rows of heads of 64 after 600 kept keys: 1.60 times without the
// second part, 1.23 with it; the gradient of eight times 256 rows after 1244 to 3744 keys, 16 heads of 128 over 4, takes 235 us for 214).
// What the last two of the three cost: 500 texts of 100 tokens, 16 heads of 128 over 4, 379 us of gradient without, 396 with; 64 x 1024 tokens of
// 12 heads of 64, no mask, 745 and 826.
constexpr int EXACT_KEYS = 128, SPLIT_KEYS_CAUSAL = 512;
constexpr float LOG2E = 1.44269504088896341f;

template <int DT, int DP> __global__ void __launch_bounds__(NW * 64, DP > 128 ? 1 : 2) attn_dq_kernel(AttnParams p)
{
    constexpr int ROWS = NW * 32, U = DP / 16, NB = DP / 32, TILE = attn_tile(DP);
    constexpr int TILE_BYTES = TILE * DP * 2;
    __shared__ __attribute__((aligned(16))) char lds[4 * TILE_BYTES]; // two of K, two of V

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wg = blockIdx.y * (int)GRID_ROW + blockIdx.x; // (those from n_wg on leave below, with the slots that no sequence has: by then the wait for the arguments has passed)
    int v = xcd_grouped(wg, p.n_wg); // (as in the forward)
    const int hk = p.by_slots(v), slot = p.n_slots - 1 - v;

    const AttnPlace place = attn_find_slot<ROWS>(p.q_off, p.b, p.q_tokens, p.pack, slot, p.n_slots);
    const AttnSeq q = place.s, k = p.same ? q : attn_seq(p.k_off, place.i, p.k_tokens);
    const int first = (slot - place.first) * ROWS, rows = q.len * p.pack;
    if (wg >= p.n_wg || first < 0 || first >= rows)
        return;

    const int row = first + w * 32 + (lane & 31);
    int head = min(row, rows - 1);
    const int token = p.by_pack(head);
    head += hk * p.pack;
    const int ahead = k.len - q.len;
    const int limit = p.causal ? max(0, min(k.len, token + ahead + 1)) : k.len;
    const int wg_keys = p.causal ? max(0, min(k.len, p.by_pack.quotient(min(first + ROWS, rows) - 1) + ahead + 1)) : k.len;
    const int wave_keys = first + w * 32 < rows ? __builtin_amdgcn_readlane(limit, 31) : 0, all_keys = __builtin_amdgcn_readfirstlane(limit);

    const char *k_head = p.K.p + (uint64_t)(uint32_t)k.start * p.K.token + hk * p.K.head, *v_head = p.V.p + (uint64_t)(uint32_t)k.start * p.V.token + hk * p.V.head;
    AttnCopy<DP, TILE, NW> copy;
    copy.init(w, lane, p.d);
    const AttnRowRead<DP> row_read(lane);
    const AttnColRead<DP> col_read(lane);
    const int tiles = (wg_keys + TILE - 1) / TILE;
    const bool exact = wg_keys <= EXACT_KEYS, twice = !exact && (!p.causal || wg_keys <= SPLIT_KEYS_CAUSAL || ahead > 0);
    auto issue = [&](int buffer, int t) {
        const uint32_t to = attn_lds(lds) + buffer * 2 * TILE_BYTES;
        copy.issue(k_head, p.K.token, t * TILE, k.len - 1, to, w, p.d);
        copy.issue(v_head, p.V.token, t * TILE, k.len - 1, to + TILE_BYTES, w, p.d);
    };
    if (tiles)
        issue(0, 0);

    uint4 qf[U], gf[U];
    const uint64_t at = (uint32_t)(q.start + token);
    attn_load_row(p.Q.p + at * p.Q.token + head * p.Q.head, p.d, h, qf);
    attn_load_row(p.dO.p + at * p.dO.token + head * p.dO.head, p.d, h, gf);
    float lse2 = p.lse[at * p.hq + head] * LOG2E;
    float delta = 0.0f;
    if (!exact) {
        uint4 of[U];
        attn_load_row(p.O.p + at * p.O.token + head * p.O.head, p.d, h, of);
        attn_have_row(p.d, h, gf);
        attn_have_row(p.d, h, of);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t a[4] = {gf[u].x, gf[u].y, gf[u].z, gf[u].w}, b[4] = {of[u].x, of[u].y, of[u].z, of[u].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                delta = __builtin_fmaf(attn_float<DT>(a[e] & 0xffff), attn_float<DT>(b[e] & 0xffff), delta);
                delta = __builtin_fmaf(attn_float<DT>(a[e] >> 16), attn_float<DT>(b[e] >> 16), delta);
            }
        }
        delta = attn_halves_sum(delta);
    }
    attn_have_row(p.d, h, qf);
    attn_have_row(p.d, h, gf);
    asm volatile("" : "+v"(lse2)); // (arrived)

    // P and dP + from of a block of 32 keys
    auto scores = [&](const char *kt, const char *vt, int b, int key, float from, f32x16 &s, f32x16 &g) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = 0.0f;
            g[r] = from;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            attn_mma<DT>(row_read.get(kt, b, u), qf[u], s);
#pragma unroll
        for (int u = 0; u < U; ++u)
            attn_mma<DT>(row_read.get(vt, b, u), gf[u], g);
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2, -lse2));
        if (key + 32 > all_keys) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[r] = key + acc_row(r, h) < limit ? s[r] : 0.0f;
        }
    };
    int buffer = 0;
    if (exact) {
        for (int t = 0; t < tiles; ++t) {
            attn_arrive();
            issue(buffer ^ 1, t + 1 < tiles ? t + 1 : 0);
            const char *kt = lds + buffer * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
            buffer ^= 1;
            for (int b = 0; b < TILE / 32 && t * TILE + 32 * b < wave_keys; ++b) {
                f32x16 s, g;
                scores(kt, vt, b, t * TILE + 32 * b, 0.0f, s, g);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    delta = __builtin_fmaf(s[r], g[r], delta);
            }
        }
        delta = attn_halves_sum(delta);
    }

    f32x16 dq[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            dq[b][r] = 0.0f;
    float rest = 0.0f; // sum of dS over the row's keys: what delta is short of
    auto walk = [&](auto twice_) {
        for (int t = 0; t < tiles; ++t) {
            attn_arrive();
            if (t + 1 < tiles)
                issue(buffer ^ 1, t + 1);
            const char *kt = lds + buffer * 2 * TILE_BYTES, *vt = kt + TILE_BYTES;
            buffer ^= 1;
#pragma unroll
            for (int b = 0; b < TILE / 32; ++b) {
                if (t * TILE + 32 * b >= wave_keys)
                    break;
                f32x16 s, g;
                scores(kt, vt, b, t * TILE + 32 * b, -delta, s, g); // (the sums of dP start at -delta)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] *= g[r];
                    rest += s[r];
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint4 ds = attn_operand<DT>(s, x);
                    uint4 more;
                    if constexpr (decltype(twice_)::value) {
                        const uint32_t u[4] = {ds.x, ds.y, ds.z, ds.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[8 * x + 2 * e] -= attn_float<DT>(u[e] & 0xffff);
                            s[8 * x + 2 * e + 1] -= attn_float<DT>(u[e] >> 16);
                        }
                        more = attn_operand<DT>(s, x);
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const uint4 a = col_read.get(kt, nb, 2 * b + x);
                        attn_mma<DT>(a, ds, dq[nb]);
                        if constexpr (decltype(twice_)::value)
                            attn_mma<DT>(a, more, dq[nb]);
                    }
                }
            }
        }
    };
    if (twice)
        walk(std::true_type{});
    else
        walk(std::false_type{});
    delta += attn_halves_sum(rest);
    if (row < rows)
        p.stat[(int64_t)(2 * head + h) * p.q_tokens + at] = h ? -delta : -lse2 / p.scale_log2;
    __syncthreads(); // (nobody reads the tiles any more)
    attn_store_tile<DT, DP>(lds + w * 32 * DP * 2, dq, p.scale, lane, p.d, rows - first - w * 32, [&](int r) {
        int g = first + w * 32 + r;
        const uint32_t t = q.start + p.by_pack(g);
        return p.dQ.p + (uint64_t)t * p.dQ.token + (hk * p.pack + g) * p.dQ.head;
    });
}

// NK: wavefronts of 32 keys, which share the tiles of queries; the gradient of 4 x 4096 causal tokens, 32 heads of 128 over 8, took 2626 us with one, 2091 with two, 1997
// with four and 2037 with eight.
// A wavefront owns 32 keys (columns) of one key head; at d = 256 the registers hold the gradients of half of d, and blockIdx.z says which.
constexpr int NK = 4;
constexpr int dkv_slices(int dp) { return dp > 128 ? 2 : 1; }
constexpr int dkv_buffer(int dp) { return 2 * Q_TILE * dp * 2 + 256; } // Q, dO, 32 of -lse / scale, 32 of -delta
template <int DT, int DP> __global__ void __launch_bounds__(NK * 64, DP > 128 ? 1 : DP > 64 ? 2 : 3) attn_dkv_kernel(AttnParams p)
{
    constexpr int KEYS = NK * 32, U = DP / 16, SLICES = dkv_slices(DP), SLICE = DP / SLICES, NB = SLICE / 32, C = 2 * NB;
    const int slice = SLICES > 1 ? blockIdx.z : 0;
    constexpr int TILE_BYTES = Q_TILE * DP * 2, BUF = dkv_buffer(DP);
    extern __shared__ __attribute__((aligned(16))) char lds[]; // two buffers

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wg = blockIdx.y * (int)GRID_ROW + blockIdx.x; // (those from n_wg on leave below, with the slots that no sequence has: by then the wait for the arguments has passed)
    int v = xcd_grouped(wg, p.n_wg), x = p.by_split(v); // (of each sequence the first tiles, which the most queries see under a causal mask, come first)
    const int piece = v, hk = p.by_slots(x), slot = x;

    const AttnPlace place = attn_find_slot<KEYS>(p.k_off, p.b, p.k_tokens, 1, slot, p.n_slots);
    const AttnSeq k = place.s, q = p.same ? k : attn_seq(p.q_off, place.i, p.q_tokens);
    const int first = (slot - place.first) * KEYS, ahead = k.len - q.len;
    if (wg >= p.n_wg || first < 0 || first >= k.len)
        return;
    const int wave_key = first + w * 32, key = wave_key + (lane & 31);
    const uint64_t at = (uint32_t)(k.start + min(key, k.len - 1));

    // steps: tiles of query rows that see any of the keys, for every head of the group
    const int q0 = p.causal ? max(0, first - ahead) / Q_TILE : 0, q1 = (q.len + Q_TILE - 1) / Q_TILE;
    const int per_head = max(0, q1 - q0);
    int over = per_head * p.pack;
    const int per = p.by_split(over), step0 = per * piece + min(piece, over), steps = per + (piece < over); // of this piece

    AttnCopy<DP, Q_TILE, NK> copy;
    copy.init(w, lane, p.d);
    AttnRowRead<DP> row_read(lane);
    AttnColRead<DP> col_read(lane);
    int next_g = per_head ? step0 / per_head : 0, next_t = q0 + step0 - next_g * per_head; // of the next copy
    auto issue = [&](int n) {
        const int head = hk * p.pack + next_g, row0 = next_t * Q_TILE;
        const uint32_t to = attn_lds(lds) + (n & 1) * BUF;
        copy.issue(p.Q.p + (uint64_t)(uint32_t)q.start * p.Q.token + head * p.Q.head, p.Q.token, row0, q.len - 1, to, w, p.d);
        copy.issue(p.dO.p + (uint64_t)(uint32_t)q.start * p.dO.token + head * p.dO.head, p.dO.token, row0, q.len - 1, to + TILE_BYTES, w, p.d);
        if (w == 0) {
            int l = lane;
            asm volatile("" : "+v"(l)); // (worked out here: kept, the offset is spilled)
            attn_load_lds4(p.stat + 2 * (int64_t)head * p.q_tokens + q.start + row0, (uint32_t)(min(l & 31, q.len - 1 - row0) + (l < 32 ? 0 : p.q_tokens)) * 4, to + 2 * TILE_BYTES);
        }
        if (++next_t == q1) {
            next_t = q0;
            ++next_g;
        }
    };
    const int next_tile = next_t;
    if (steps)
        issue(0);

    uint4 kf[U], vf[U];
    attn_load_row(p.K.p + at * p.K.token + hk * p.K.head, p.d, h, kf);
    attn_load_row(p.V.p + at * p.V.token + hk * p.V.head, p.d, h, vf);
    attn_have_row(p.d, h, kf);
    attn_have_row(p.d, h, vf);
    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            dk[b][r] = dv[b][r] = 0.0f;

    int tile = next_tile;
    for (int n = 0; n < steps; ++n) {
        attn_arrive();
        if (n + 1 < steps)
            issue(n + 1);
        const char *qt = lds + (n & 1) * BUF, *gt = qt + TILE_BYTES;
        const f32x4 *stat = reinterpret_cast<const f32x4 *>(gt + TILE_BYTES);
        const int row0 = tile * Q_TILE;
        if (++tile == q1)
            tile = q0;
        if (wave_key >= k.len || (p.causal && row0 + Q_TILE - 1 + ahead < wave_key))
            continue;
        // The products of S, dV, dP and dK as one stream of MFMAs whose A operands are read from LDS AHEAD of them: left to itself the
        // compiler waits for each operand before it asks for the next one, there being few registers to spare. (Three ahead spill at d = 128:
        // 16 x 1024 causal tokens of 16 heads over 4, dQ, dK and dV 341 us, two 314; at d = 256 three 886, two 894.)
        constexpr int TO_DV = U, TO_DP = U + C, TO_DK = 2 * U + C, STEPS = 2 * U + 2 * C, AHEAD = DP == 128 ? 2 : 3;
        uint4 a[AHEAD];
        auto read = [&](auto step) {
            constexpr int I = decltype(step)::value;
            if constexpr (I < STEPS) {
                if constexpr (I == 0 || I == TO_DV || I == TO_DP || I == TO_DK) // (addresses are worked out where they are used: kept from one product to another they spill)
                    asm volatile("" : "+v"(row_read.swz), "+v"(col_read.chunk));
                if constexpr (I < TO_DV)
                    a[I % AHEAD] = row_read.get(qt, 0, I);
                else if constexpr (I < TO_DP)
                    a[I % AHEAD] = col_read.get(gt + slice * SLICE * 2, (I - TO_DV) % NB, (I - TO_DV) / NB);
                else if constexpr (I < TO_DK)
                    a[I % AHEAD] = row_read.get(gt, 0, I - TO_DP);
                else
                    a[I % AHEAD] = col_read.get(qt + slice * SLICE * 2, (I - TO_DK) % NB, (I - TO_DK) / NB);
            }
        };
        // the sums start from what is subtracted from them: S - lse / scale, dP - delta
        f32x16 s, g;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 l = stat[r / 2 + h];
            s[r] = l[0], s[r + 1] = l[1], s[r + 2] = l[2], s[r + 3] = l[3];
        }
        static_for<AHEAD>(read);
        __builtin_amdgcn_sched_barrier(0);
        uint4 b; // of P, then of dS
        static_for<STEPS>([&](auto step) {
            constexpr int I = decltype(step)::value;
            if constexpr (I == TO_DV) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = __builtin_amdgcn_exp2f(s[r] * p.scale_log2);
                if (row0 + Q_TILE > q.len || (p.causal && row0 + ahead < wave_key + 31)) {
                    const int from = p.causal ? key - ahead : 0; // the first query that sees this lane's key
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int t = row0 + acc_row(r, h);
                        s[r] = t >= from && t < q.len ? s[r] : 0.0f;
                    }
                }
            } else if constexpr (I == TO_DP) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 d = stat[8 + r / 2 + h];
                    g[r] = d[0], g[r + 1] = d[1], g[r + 2] = d[2], g[r + 3] = d[3];
                }
            } else if constexpr (I == TO_DK) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] *= g[r];
            }
            if constexpr (I == TO_DV || I == TO_DV + NB || I == TO_DK || I == TO_DK + NB)
                b = attn_operand<DT>(s, I == TO_DV || I == TO_DK ? 0 : 1);
            if constexpr (I < TO_DV)
                attn_mma<DT>(a[I % AHEAD], kf[I], s);
            else if constexpr (I < TO_DP)
                attn_mma<DT>(a[I % AHEAD], b, dv[(I - TO_DV) % NB]);
            else if constexpr (I < TO_DK)
                attn_mma<DT>(a[I % AHEAD], vf[I - TO_DP], g);
            else
                attn_mma<DT>(a[I % AHEAD], b, dk[(I - TO_DK) % NB]);
            read(std::integral_constant<int, I + AHEAD>{});
            __builtin_amdgcn_sched_barrier(0);
        });
    }
    const int d0 = slice * SLICE, d = min(p.d - d0, SLICE);
    if (p.n_split > 1) {
        const int64_t part = ((int64_t)piece * p.k_tokens + k.start + key) * p.hkv + hk;
        if (key < k.len) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    if (32 * b + 2 * r < d) {
                        const int e = d0 + 32 * b + 2 * r + 4 * h;
                        *reinterpret_cast<float4 *>(p.part_k + part * p.d + e) = make_float4(dk[b][r], dk[b][r + 1], dk[b][r + 2], dk[b][r + 3]);
                        *reinterpret_cast<float4 *>(p.part_v + part * p.d + e) = make_float4(dv[b][r], dv[b][r + 1], dv[b][r + 2], dv[b][r + 3]);
                    }
        }
        return;
    }
    __syncthreads(); // (nobody reads the tiles any more)
    char *rows = lds + w * 32 * SLICE * 2;
    const uint32_t token = k.start + wave_key;
    attn_store_tile<DT, SLICE>(rows, dk, p.scale, lane, d, k.len - wave_key, [&](int r) { return p.dK.p + (uint64_t)(token + r) * p.dK.token + hk * p.dK.head + d0 * 2; });
    attn_store_tile<DT, SLICE>(rows, dv, 1.0f, lane, d, k.len - wave_key, [&](int r) { return p.dV.p + (uint64_t)(token + r) * p.dV.token + hk * p.dV.head + d0 * 2; });
}

// Adds the pieces up, in their order; a thread per four entries of a row
template <int DT> __global__ void __launch_bounds__(256) attn_dkv_join_kernel(AttnParams p)
{
    const int64_t x = ((int64_t)blockIdx.y * GRID_ROW + blockIdx.x) * 256 + threadIdx.x, n = (int64_t)p.k_tokens * p.hkv * p.d;
    if (x * 4 >= n)
        return;
    float4 k = make_float4(0.0f, 0.0f, 0.0f, 0.0f), v = k;
#pragma unroll 4
    for (int s = 0; s < p.n_split; ++s) {
        const float4 a = *reinterpret_cast<const float4 *>(p.part_k + s * n + x * 4), b = *reinterpret_cast<const float4 *>(p.part_v + s * n + x * 4);
        k = make_float4(k.x + a.x, k.y + a.y, k.z + a.z, k.w + a.w);
        v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
    }
    const int64_t row = x * 4 / p.d;
    const int e = (int)(x * 4 % p.d), hk = (int)(row % p.hkv);
    const int64_t token = row / p.hkv;
    attn_store4<DT>(p.dK.p + token * p.dK.token + hk * p.dK.head, e, k.x * p.scale, k.y * p.scale, k.z * p.scale, k.w * p.scale);
    attn_store4<DT>(p.dV.p + token * p.dV.token + hk * p.dV.head, e, v.x, v.y, v.z, v.w);
}

// Pieces of the queries of a key tile: few key heads and short batches leave most compute units idle otherwise (one sequence of 1000 keys with one head
// is eight workgroups: all gradients 304 us, 64 in the pieces chosen here). An estimate in microseconds: a step of a workgroup takes 2 at d = 128
// with the chip full, its start 5, joining a launch and a round trip of fp32 sums.
int dkv_pieces(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu)
{
    const double full = 2.0 * num_cu, work = (double)(k_tokens / (NK * 32) + b) * hkv, steps = std::max(1.0, (double)q_tokens / b / Q_TILE) * (hq / hkv);
    const double step = 2.0 * (d + 64) / 192, join = (double)k_tokens * hkv * d * 16 / 4.0e6;
    int best_n = 1;
    double best = 0;
    for (int n = 1; n <= 64 && n <= std::max(1.0, steps / 4) && work * n < (1 << 24); ++n) {
        const double time = (std::max(1.0, work * n / full) + 0.6) * (steps / n * step + 5.0) + (n > 1 ? 4.0 + n * join : 0.0);
        if (n == 1 || time < (best_n == 1 ? 0.85 : 1.0) * best) {
            best = time;
            best_n = n;
        }
    }
    return best_n;
}

} // namespace

// dK and dV of the widest heads take 64.5 KB of LDS
hipError_t attention_backward_init_device()
{
    const int bytes = 2 * dkv_buffer(ATTN_WIDEST);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(attn_dkv_kernel<MAXSIM_F16, ATTN_WIDEST>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void *>(attn_dkv_kernel<MAXSIM_BF16, ATTN_WIDEST>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

int64_t attention_backward_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu)
{
    const int n = dkv_pieces(b, q_tokens, k_tokens, hq, hkv, d, num_cu);
    return (q_tokens * hq * 8 + 15) / 16 * 16 + (n > 1 ? n * k_tokens * hkv * d * 8 : 0);
}

hipError_t attention_backward_launch(AttnParams p, int dtype, void *workspace, int num_cu, hipStream_t stream)
{
    p.pack = p.hq / p.hkv;
    p.by_pack = AttnDivisor::of(p.pack);
    p.n_split = dkv_pieces(p.b, p.q_tokens, p.k_tokens, p.hq, p.hkv, p.d, num_cu);
    p.by_split = AttnDivisor::of(p.n_split);
    p.stat = static_cast<float *>(workspace);
    p.part_k = p.stat + ((int64_t)p.q_tokens * p.hq * 2 + 3) / 4 * 4;
    p.part_v = p.part_k + (int64_t)p.n_split * p.k_tokens * p.hkv * p.d;
    const hipError_t e = attn_width(p.d, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        p.n_slots = p.q_tokens * p.pack / (NW * 32) + p.b;
        p.by_slots = AttnDivisor::of(p.n_slots);
        p.n_wg = p.n_slots * p.hkv;
        if (dtype == MAXSIM_F16)
            attn_dq_kernel<MAXSIM_F16, DP><<<grid_rows(p.n_wg), NW * 64, 0, stream>>>(p);
        else
            attn_dq_kernel<MAXSIM_BF16, DP><<<grid_rows(p.n_wg), NW * 64, 0, stream>>>(p);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) // (nothing reads row statistics that have not been written)
            return e;
        p.n_slots = p.k_tokens / (NK * 32) + p.b;
        p.by_slots = AttnDivisor::of(p.n_slots);
        p.n_wg = p.n_slots * p.hkv * p.n_split;
        dim3 grid = grid_rows(p.n_wg);
        grid.z = dkv_slices(DP);
        if (dtype == MAXSIM_F16)
            attn_dkv_kernel<MAXSIM_F16, DP><<<grid, NK * 64, 2 * dkv_buffer(DP), stream>>>(p);
        else
            attn_dkv_kernel<MAXSIM_BF16, DP><<<grid, NK * 64, 2 * dkv_buffer(DP), stream>>>(p);
        return hipGetLastError();
    });
    if (e != hipSuccess || p.n_split == 1)
        return e;
    const dim3 join = grid_rows(((int64_t)p.k_tokens * p.hkv * p.d / 4 + 255) / 256);
    if (dtype == MAXSIM_F16)
        attn_dkv_join_kernel<MAXSIM_F16><<<join, 256, 0, stream>>>(p);
    else
        attn_dkv_join_kernel<MAXSIM_BF16><<<join, 256, 0, stream>>>(p);
    return hipGetLastError();
}

} // namespace maxsim
