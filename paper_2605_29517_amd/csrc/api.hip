// C ABI of the library: argument checks, device query, kernel selection.  See include/maxsim.h.
#include <hip/hip_runtime.h>

#include <cstring>
#include <mutex>

#include "attention.h"
#include "rope.h"

namespace maxsim {
hipError_t forward_launch(FwdParams p, int dtype, int d, int num_cu, hipStream_t stream);
bool forward_width_supported(int dtype, int d);
hipError_t backward_launch(const void *Q, int n_q, int l_q, const void *D, const int32_t *offsets, int64_t b, int l_d,
                           int64_t total_tokens, int d, int dtype, const int32_t *argmax, const float *dscore, float *dQ,
                           float *dD, int num_cu, hipStream_t stream);
hipError_t csr_build_launch(const int32_t *argmax, int n_q, int64_t b, int l_q, int l_d, int32_t *row_ptr,
                            int32_t *col_idx, int num_cu, hipStream_t stream);
hipError_t backward_csr_launch(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d, int dtype,
                               const int32_t *argmax, const float *dscore, int32_t *row_ptr, int32_t *col_idx, float *dQ,
                               float *dD, int num_cu, hipStream_t stream);
bool csr_static_fits(int n_q, int64_t b, int l_q, int l_d);
hipError_t backward_csr_static_launch(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d, int dtype,
                                      const int32_t *argmax, const float *dscore, float *dQ, float *dD, int num_cu,
                                      hipStream_t stream);
hipError_t quantize_launch(const void *X, int64_t rows, int dtype, int8_t *X_i8, float *scale, hipStream_t stream);
bool i8_wide_width_ok(int d);
hipError_t forward_i8_wide_launch(const int8_t *Q, const float *qs, int n_q, int l_q, const int8_t *D, const float *ds,
                                  const int32_t *offsets, int64_t b, int l_d, int64_t total_tokens, int d, float *scores,
                                  int64_t ld, int num_cu, hipStream_t stream);
hipError_t quantize_wide_launch(const void *X, int64_t rows, int d, int dtype, int8_t *X_i8, float *scale, hipStream_t stream);
hipError_t forward_i8_launch(const int8_t *Q, const float *qs, int n_q, int l_q, const int8_t *D, const float *ds,
                             const int32_t *offsets, int64_t b, int l_d, int64_t total_tokens, float *scores,
                             int64_t ld, int num_cu, hipStream_t stream);
hipError_t ce_grad_launch(const float *scores, int n, int b, float tau, float *g, float *loss, hipStream_t stream);
bool rope_width_ok(int rot);
hipError_t rope_launch(const void *X, int64_t tokens, int heads, int d, int64_t x_token, int64_t x_head, int dtype, const float *freqs, int rot,
                       const int32_t *positions, const int32_t *offsets, int64_t b, float scale, bool neighbours, bool inverse, void *Y, int64_t y_token, int64_t y_head,
                       hipStream_t stream);
int64_t attention_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu);
hipError_t attention_launch(AttnParams p, int dtype, void *workspace, int num_cu, hipStream_t stream);
int64_t attention_backward_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, int num_cu);
hipError_t attention_backward_launch(AttnParams p, int dtype, void *workspace, int num_cu, hipStream_t stream);
int64_t clip_workspace(int n);
hipError_t clip_launch(const void *const *g, void *const *out, const int64_t *numel, const int32_t *dtype, int n, float max_norm, float *norm, void *workspace, hipStream_t stream);
hipError_t embed_launch(const void *W, int64_t vocab, int d, int dtype, const void *tokens, bool wide, int64_t n, float scale, void *Y, int y_dtype, hipStream_t stream);
int64_t embed_backward_workspace(int64_t n, int64_t vocab, int d);
hipError_t embed_backward_launch(const void *dY, int dtype, const void *tokens, bool wide, int64_t n, int64_t vocab, int d, float scale, bool accumulate, void *dW, int w_dtype,
                                 void *workspace, hipStream_t stream);
hipError_t norm_rope_launch(const void *X, int64_t tokens, int heads, int d, const int64_t *strides, int dtype, const void *q_weight, const void *k_weight, int w_dtype, int q_heads,
                            float eps, const RopeAngles &angles, bool neighbours, void *Y, hipStream_t stream);
int64_t norm_rope_backward_workspace(int64_t tokens, int heads, int d);
hipError_t norm_rope_backward_launch(const void *X, const void *dY, int64_t tokens, int heads, int d, const int64_t *strides, int dtype, const void *q_weight, const void *k_weight,
                                     int w_dtype, int q_heads, float eps, const RopeAngles &angles, bool neighbours, void *dX, float *dq_weight, float *dk_weight, void *workspace,
                                     hipStream_t stream);
int64_t distill_workspace(int n, int64_t b, int dtype, int num_cu);
hipError_t distill_launch(const void *scores, int n, int b, int64_t ld, int dtype, const void *teacher, int t_dtype, const int32_t *index, int k, float tau, float *loss, float *lse,
                          const float *up, float weight, void *g, int64_t g_ld, void *workspace, int num_cu, hipStream_t stream);
hipError_t forward_splitd_init_device();
hipError_t forward_wide_init_device();
hipError_t forward_i8_init_device();
hipError_t backward_init_device();
hipError_t attention_backward_init_device();
} // namespace maxsim

namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// (by its bits: the library is compiled as if there were no NaNs)
bool is_nan(float x)
{
    uint32_t u;
    memcpy(&u, &x, sizeof u);
    return (u & 0x7fffffffu) > 0x7f800000u;
}

bool dtype_ok(int dt) { return dt == MAXSIM_F32 || dt == MAXSIM_F16 || dt == MAXSIM_BF16; }

// Compute-unit count of the current device, queried once per device.
int num_cu()
{
    static int cached[64] = {0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return 256;
    if (cached[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            n = 256;
        cached[dev] = n;
    }
    return cached[dev];
}

// int8 scoring: the kernels built around 128-byte rows, or (other widths) the slab kernel / the plain inner loop over d
static hipError_t i8_launch_any(const int8_t *Q, const float *qs, int n_q, int l_q, const int8_t *D, const float *ds,
                                const int32_t *offsets, int64_t b, int l_d, int64_t total_tokens, int d, float *scores,
                                int64_t ld, int cus, hipStream_t stream)
{
    if (d == maxsim::D_MODEL)
        return maxsim::forward_i8_launch(Q, qs, n_q, l_q, D, ds, offsets, b, l_d, total_tokens, scores, ld, cus, stream);
    return maxsim::forward_i8_wide_launch(Q, qs, n_q, l_q, D, ds, offsets, b, l_d, total_tokens, d, scores, ld, cus, stream);
}
static bool i8_width_ok(int d) { return d == maxsim::D_MODEL || maxsim::i8_wide_width_ok(d); }

// embedding widths of the backward entry points: whole 16-byte chunks of 8 elements, up to 64 slabs of 128 columns
bool backward_width_ok(int d) { return d >= 8 && d <= 8192 && d % 8 == 0; }
// the dD kernels address Q rows through 32-bit byte offsets: Q must stay below 4 GiB
// and the dQ kernel addresses D rows through 32-bit offsets in units of 16 bytes: D must stay below 64 GiB
bool backward_q_ok(int n_q, int l_q, int d, int dtype, int64_t total_tokens)
{
    const int64_t row_bytes = (int64_t)d * (dtype == MAXSIM_F32 ? 4 : 2);
    return (int64_t)n_q * l_q * row_bytes < (int64_t(1) << 32) && total_tokens <= ((int64_t(1) << 36) - 1) / row_bytes;
}

// Per-device set-up, done once per device under a lock (two host threads may make their first call at once):
// the kernels that use more than 64 KB of LDS are allowed to (every instantiation), and the static scratch
// array's device address is looked up.  maxsim_init runs it for the current device; every entry point runs it
// after its argument checks, so that callers who never call maxsim_init lose nothing but the freedom to make
// their first call on a device under stream capture.
int ensure_init()
{
    static bool done[64] = {};
    static std::mutex guard;
    std::lock_guard<std::mutex> lock(guard);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return MAXSIM_ERR_LAUNCH;
    if (done[dev])
        return MAXSIM_OK;
    if (maxsim::forward_wide_init_device() != hipSuccess || maxsim::forward_splitd_init_device() != hipSuccess ||
        maxsim::forward_i8_init_device() != hipSuccess || maxsim::backward_init_device() != hipSuccess || maxsim::attention_backward_init_device() != hipSuccess)
        return MAXSIM_ERR_LAUNCH;
    done[dev] = true;
    return MAXSIM_OK;
}

int finish(hipError_t e) { return e == hipSuccess ? MAXSIM_OK : MAXSIM_ERR_LAUNCH; }

// One copy stream per device for the out-of-core path, created on first use at the default
// priority and kept until the process ends.
hipStream_t copy_stream()
{
    static hipStream_t cached[64] = {nullptr};
    static std::mutex guard; // two host threads may make their first streamed call at once
    std::lock_guard<std::mutex> lock(guard);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return nullptr;
    if (!cached[dev]) {
        hipStream_t st = nullptr;
        if (hipStreamCreateWithFlags(&st, hipStreamNonBlocking) != hipSuccess)
            return nullptr;
        cached[dev] = st;
    }
    return cached[dev];
}

// Whether the rows of an output [tokens, heads, d] lie apart: a token's heads before the next token, or a head's tokens before the next head (strides >= 0)
bool rows_apart(int64_t tokens, int64_t heads, int64_t d, int64_t token, int64_t head)
{
    if (token < d || head < d)
        return false;
    return tokens == 1 || heads == 1 || token >= __int128(heads - 1) * head + d || head >= __int128(tokens - 1) * token + d;
}

// The size of an element, and the alignment that a pointer to it needs
uintptr_t size_of(int dt) { return dt == MAXSIM_F32 ? 4 : 2; }

// Embedding: what both directions look at
int embed_common(const void *table, maxsim_dtype t_dtype, const void *rows, maxsim_dtype r_dtype, const void *tokens, int token_bytes, int64_t n, int64_t vocab, int d, float scale)
{
    if (!table || !rows || !tokens || n < 1 || vocab < 1 || d < 1 || !dtype_ok((int)t_dtype) || !dtype_ok((int)r_dtype) || (token_bytes != 4 && token_bytes != 8) || is_nan(scale))
        return MAXSIM_ERR_INVALID;
    if (!aligned(table, size_of(t_dtype)) || !aligned(rows, size_of(r_dtype)) || !aligned(tokens, token_bytes))
        return MAXSIM_ERR_INVALID;
    return n >= (int64_t(1) << 31) || vocab >= (int64_t(1) << 31) - 1 || d > 65536 ? MAXSIM_ERR_UNSUPPORTED : MAXSIM_OK;
}

// Norms with rotary positions: sizes, pointers and strides ([n] pairs in `plain` where none are given); the last tensor is written
int norm_rope_common(const void *const *t, int n, int64_t tokens, int heads, int d, const int64_t *&strides, int64_t *plain, maxsim_dtype dtype, const void *q_weight,
                     const void *k_weight, maxsim_dtype w_dtype, int q_heads, float eps, const float *freqs, int rot, const int32_t *positions, const int32_t *offsets, int64_t b,
                     float scale)
{
    if (tokens < 1 || heads < 1 || q_heads < 0 || q_heads > heads || d < 2 || !freqs || rot < 2 || rot > d || rot % 2 != 0 || !dtype_ok((int)dtype) || !dtype_ok((int)w_dtype) ||
        (offsets && b < 1) || is_nan(scale) || is_nan(eps) || eps < 0.0f)
        return MAXSIM_ERR_INVALID;
    if (!aligned(q_weight, size_of(w_dtype)) || !aligned(k_weight, size_of(w_dtype)) || !aligned(freqs, 4) || !aligned(positions, 4) || !aligned(offsets, 4))
        return MAXSIM_ERR_INVALID;
    for (int i = 0; i < 2 * n; ++i)
        plain[i] = i % 2 ? d : (int64_t)heads * d;
    strides = strides ? strides : plain;
    for (int i = 0; i < n; ++i) {
        if (!t[i] || !aligned(t[i], size_of(dtype)) || strides[2 * i] < 0 || strides[2 * i + 1] < 0)
            return MAXSIM_ERR_INVALID;
    }
    const int64_t *last = strides + 2 * n - 2;
    if (!rows_apart(tokens, heads, d, last[0], last[1]))
        return MAXSIM_ERR_INVALID;
    for (int i = 0; i < n - 1; ++i) // in place, but other rows: those that are still to be read would be written over
        if (t[i] == t[n - 1] && ((tokens > 1 && strides[2 * i] != last[0]) || (heads > 1 && strides[2 * i + 1] != last[1])))
            return MAXSIM_ERR_INVALID;
    return d > 512 || heads > 8192 || tokens >= (int64_t(1) << 31) || b >= (int64_t(1) << 31) ? MAXSIM_ERR_UNSUPPORTED : MAXSIM_OK;
}

// Distillation: what all three entry points look at
int distill_common(const void *scores, int n, int64_t b, int64_t stride, maxsim_dtype dtype, const void *teacher, maxsim_dtype t_dtype, const int32_t *index, int k, float tau)
{
    if (!scores || !teacher || n < 1 || b < 1 || k < 1 || stride < b || !dtype_ok((int)dtype) || !dtype_ok((int)t_dtype) || is_nan(tau) || !(tau > 1e-30f) || !(tau < 1e30f))
        return MAXSIM_ERR_INVALID;
    if (!aligned(scores, size_of(dtype)) || !aligned(teacher, size_of(t_dtype)) || !aligned(index, 4) || (!index && k != b))
        return MAXSIM_ERR_INVALID;
    return k > 1024 || b >= (int64_t(1) << 31) || stride >= (int64_t(1) << 40) ? MAXSIM_ERR_UNSUPPORTED : MAXSIM_OK;
}

// Attention: sizes, then pointers and strides of the packed tensors
int attention_sizes_ok(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d)
{
    if (b < 1 || q_tokens < 1 || k_tokens < 1 || hq < 1 || hkv < 1 || hq % hkv != 0 || d < 1)
        return MAXSIM_ERR_INVALID;
    if (d % 8 != 0 || d > maxsim::ATTN_WIDEST || hq > (1 << 16))
        return MAXSIM_ERR_UNSUPPORTED;
    // tiles and rows are counted in 31 bits: tokens * heads rows, (rows / 32 + sequences) tiles of every head
    const int64_t most = int64_t(1) << 30;
    if (q_tokens >= most || k_tokens >= most || b >= (int64_t(1) << 24) || (q_tokens + 32 * b) * hq >= most || (k_tokens / 128 + b) * hkv >= most)
        return MAXSIM_ERR_UNSUPPORTED;
    return MAXSIM_OK;
}

struct AttnTensor {
    maxsim::AttnRows *to;
    const void *p;
    int heads;
    int64_t rows; // of an output, 0 otherwise
};

int attention_common(maxsim::AttnParams &p, const AttnTensor *t, int n, const int64_t *strides, const int32_t *q_offsets, const int32_t *k_offsets, int64_t b, int64_t q_tokens,
                     int64_t k_tokens, int hq, int hkv, int d, int dtype, int causal, float scale, const void *workspace, int64_t workspace_bytes, int64_t needed)
{
    if (int rc = attention_sizes_ok(b, q_tokens, k_tokens, hq, hkv, d))
        return rc;
    if (!q_offsets || !k_offsets || !aligned(q_offsets, 4) || !aligned(k_offsets, 4) || !dtype_ok(dtype) || is_nan(scale) || !(scale > 1e-30f && scale < 1e30f)) // (-lse / scale is a finite number)
        return MAXSIM_ERR_INVALID;
    if (dtype == MAXSIM_F32)
        return MAXSIM_ERR_UNSUPPORTED;
    for (int i = 0; i < n; ++i) {
        const int64_t token = strides ? strides[2 * i] : (int64_t)t[i].heads * d, head = strides ? strides[2 * i + 1] : d;
        if (!t[i].p || !aligned(t[i].p, 16) || token < 0 || head < 0 || token % 8 != 0 || head % 8 != 0)
            return MAXSIM_ERR_INVALID;
        if (t[i].rows && !rows_apart(t[i].rows, t[i].heads, d, token, head))
            return MAXSIM_ERR_INVALID;
        if (token >= (1 << 24) || head >= (int64_t(1) << 40))
            return MAXSIM_ERR_UNSUPPORTED;
        *t[i].to = {static_cast<char *>(const_cast<void *>(t[i].p)), head * 2, (uint32_t)token * 2};
    }
    if (needed > 0 && (!workspace || !aligned(workspace, 16)))
        return MAXSIM_ERR_INVALID;
    if (workspace_bytes < needed)
        return MAXSIM_ERR_SCRATCH;
    p.q_off = q_offsets;
    p.k_off = k_offsets;
    p.b = (int)b;
    p.q_tokens = (int)q_tokens;
    p.k_tokens = (int)k_tokens;
    p.hq = hq;
    p.hkv = hkv;
    p.d = d;
    // (the same offsets over other numbers of rows are cut to each side's own, as any offsets are: no row is read that is not there)
    p.same = q_offsets == k_offsets && q_tokens == k_tokens;
    p.causal = causal != 0;
    p.scale = scale;
    p.scale_log2 = scale * 1.44269504088896341f;
    return MAXSIM_OK;
}

int forward_common(const void *Q, int n_q, int l_q, const void *D, const int32_t *offsets, int64_t b, int l_d,
                   int64_t total_tokens, int d, int dtype, float *scores, int32_t *argmax, void *stream)
{
    if (!Q || !D || !scores || n_q < 1 || l_q < 1 || b < 1 || !dtype_ok(dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D, 16) || !aligned(scores, 4) || !aligned(argmax, 4) || !aligned(offsets, 4))
        return MAXSIM_ERR_INVALID;
    if (!maxsim::forward_width_supported(dtype, d))
        return MAXSIM_ERR_UNSUPPORTED;
    // index ranges the kernels rely on: token counts and block ids fit in int32
    if (total_tokens >= (int64_t(1) << 31) || (int64_t)n_q * ((l_q + 31) / 32) >= (int64_t(1) << 24) ||
        b >= (int64_t(1) << 31))
        return MAXSIM_ERR_UNSUPPORTED;
    maxsim::FwdParams p = {};
    p.Q = static_cast<const char *>(Q);
    p.D = static_cast<const char *>(D);
    p.offsets = offsets;
    p.scores = scores;
    p.argmax = argmax;
    p.b = b;
    p.total_tokens = total_tokens;
    p.n_q = n_q;
    p.l_q = l_q;
    p.l_d = l_d;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::forward_launch(p, dtype, d, num_cu(), static_cast<hipStream_t>(stream)));
}

// Out-of-core driver shared by the streamed entry points: block k + 1 is copied on the copy stream while
// block k is scored on the caller's stream; two staging halves, events in both directions.
// copy(half, first, docs, copy_stream) enqueues the host-to-device copies of a block,
// launch(half, first, docs) enqueues its kernel on the caller's stream.
template <typename Copy, typename Launch>
int stream_blocks(hipStream_t compute, int64_t b, int64_t block_docs, Copy copy_block, Launch launch_block)
{
    hipStream_t copy = copy_stream();
    if (!copy)
        return MAXSIM_ERR_LAUNCH;
    // events: block k copied (per staging half), staging half free again (its kernel has run)
    hipEvent_t copied[2] = {nullptr, nullptr}, freed[2] = {nullptr, nullptr}, entry = nullptr;
    bool ok = hipEventCreateWithFlags(&entry, hipEventDisableTiming) == hipSuccess;
    for (int i = 0; i < 2 && ok; ++i)
        ok = hipEventCreateWithFlags(&copied[i], hipEventDisableTiming) == hipSuccess &&
             hipEventCreateWithFlags(&freed[i], hipEventDisableTiming) == hipSuccess;
    int rc = ok ? MAXSIM_OK : MAXSIM_ERR_LAUNCH;
    // the staging buffer may still be in use by work already enqueued on the caller's stream
    if (rc == MAXSIM_OK && (hipEventRecord(entry, compute) != hipSuccess || hipStreamWaitEvent(copy, entry, 0) != hipSuccess))
        rc = MAXSIM_ERR_LAUNCH;
    const int64_t n_blocks = (b + block_docs - 1) / block_docs;
    for (int64_t k = 0; k < n_blocks && rc == MAXSIM_OK; ++k) {
        const int half = (int)(k & 1);
        const int64_t first = k * block_docs;
        const int64_t docs = (b - first < block_docs) ? b - first : block_docs;
        hipError_t e = hipSuccess;
        if (k >= 2)
            e = hipStreamWaitEvent(copy, freed[half], 0); // the kernel that read this half two blocks ago
        if (e == hipSuccess)
            e = copy_block(half, first, docs, copy);
        if (e == hipSuccess)
            e = hipEventRecord(copied[half], copy);
        if (e == hipSuccess)
            e = hipStreamWaitEvent(compute, copied[half], 0);
        if (e == hipSuccess)
            e = launch_block(half, first, docs);
        if (e == hipSuccess)
            e = hipEventRecord(freed[half], compute);
        if (e != hipSuccess)
            rc = MAXSIM_ERR_LAUNCH;
    }
    // destroying an event that is still pending only releases it once it has completed
    if (entry)
        (void)hipEventDestroy(entry);
    for (int i = 0; i < 2; ++i) {
        if (copied[i])
            (void)hipEventDestroy(copied[i]);
        if (freed[i])
            (void)hipEventDestroy(freed[i]);
    }
    return rc;
}

} // namespace

extern "C" {

int maxsim_init(void) { return ensure_init(); }

const char *maxsim_strerror(int code)
{
    switch (code) {
    case MAXSIM_OK: return "ok";
    case MAXSIM_ERR_INVALID: return "invalid argument (null or misaligned pointer, non-positive size, bad dtype)";
    case MAXSIM_ERR_UNSUPPORTED: return "unsupported shape (an embedding width or a size outside what this entry point is built for)";
    case MAXSIM_ERR_LAUNCH: return "HIP reported an error at kernel launch";
    case MAXSIM_ERR_SCRATCH: return "sizes exceed the library's static scratch buffer (use the entry point that takes caller buffers) or the workspace given";
    default: return "unknown maxsim error code";
    }
}

int maxsim_forward(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d, maxsim_dtype dtype,
                   float *scores, int32_t *argmax, void *stream)
{
    if (l_d < 1)
        return MAXSIM_ERR_INVALID;
    if (b > 0 && (int64_t)l_d > ((int64_t(1) << 31) - 1) / b)
        return (Q && D && scores) ? MAXSIM_ERR_UNSUPPORTED : MAXSIM_ERR_INVALID;
    return forward_common(Q, n_q, l_q, D, nullptr, b, l_d, b * (int64_t)l_d, d, (int)dtype, scores, argmax, stream);
}

int maxsim_forward_streamed(const void *Q, int n_q, int l_q, const void *D_host, int64_t b, int l_d, int d,
                            maxsim_dtype dtype, int64_t block_docs, void *staging, float *scores, void *stream)
{
    if (!Q || !D_host || !staging || !scores || n_q < 1 || l_q < 1 || b < 1 || l_d < 1 || block_docs < 1 ||
        !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D_host, 16) || !aligned(staging, 16) || !aligned(scores, 4))
        return MAXSIM_ERR_INVALID;
    if (!maxsim::forward_width_supported((int)dtype, d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (block_docs > b)
        block_docs = b;
    if (block_docs > ((int64_t(1) << 31) - 1) / l_d || (int64_t)n_q * ((l_q + 31) / 32) >= (int64_t(1) << 24))
        return MAXSIM_ERR_UNSUPPORTED;
    const int64_t doc_bytes = (int64_t)l_d * d * ((int)dtype == MAXSIM_F32 ? 4 : 2);
    if (int rc = ensure_init())
        return rc;
    hipStream_t compute = static_cast<hipStream_t>(stream);
    const int cus = num_cu();
    return stream_blocks(
        compute, b, block_docs,
        [&](int half, int64_t first, int64_t docs, hipStream_t copy) {
            return hipMemcpyAsync(static_cast<char *>(staging) + half * block_docs * doc_bytes,
                                  static_cast<const char *>(D_host) + first * doc_bytes, (size_t)(docs * doc_bytes),
                                  hipMemcpyHostToDevice, copy);
        },
        [&](int half, int64_t first, int64_t docs) {
            maxsim::FwdParams p = {};
            p.Q = static_cast<const char *>(Q);
            p.D = static_cast<const char *>(staging) + half * block_docs * doc_bytes;
            p.scores = scores + first;
            p.b = docs;
            p.ld = b;
            p.total_tokens = docs * (int64_t)l_d;
            p.n_q = n_q;
            p.l_q = l_q;
            p.l_d = l_d;
            return maxsim::forward_launch(p, (int)dtype, d, cus, compute);
        });
}

int maxsim_forward_i8_streamed(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q, const int8_t *D_i8_host,
                               const float *d_scale_host, int64_t b, int l_d, int d, int64_t block_docs,
                               int8_t *staging_codes, float *staging_scales, float *scores, void *stream)
{
    if (!Q_i8 || !q_scale || !D_i8_host || !d_scale_host || !staging_codes || !staging_scales || !scores || n_q < 1 ||
        l_q < 1 || b < 1 || l_d < 1 || block_docs < 1)
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q_i8, 16) || !aligned(D_i8_host, 16) || !aligned(staging_codes, 16) || !aligned(q_scale, 4) ||
        !aligned(d_scale_host, 4) || !aligned(staging_scales, 4) || !aligned(scores, 4))
        return MAXSIM_ERR_INVALID;
    if (!i8_width_ok(d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (block_docs > b)
        block_docs = b;
    if (block_docs > ((int64_t(1) << 31) - 1) / l_d || (int64_t)n_q * ((l_q + 31) / 32) >= (int64_t(1) << 24) || l_q > 1024)
        return MAXSIM_ERR_UNSUPPORTED;
    const int64_t doc_bytes = (int64_t)l_d * d;
    if (int rc = ensure_init())
        return rc;
    hipStream_t compute = static_cast<hipStream_t>(stream);
    const int cus = num_cu();
    return stream_blocks(
        compute, b, block_docs,
        [&](int half, int64_t first, int64_t docs, hipStream_t copy) {
            hipError_t e = hipMemcpyAsync(staging_codes + half * block_docs * doc_bytes, D_i8_host + first * doc_bytes,
                                          (size_t)(docs * doc_bytes), hipMemcpyHostToDevice, copy);
            if (e != hipSuccess)
                return e;
            return hipMemcpyAsync(staging_scales + half * block_docs * l_d, d_scale_host + first * l_d,
                                  (size_t)(docs * l_d) * sizeof(float), hipMemcpyHostToDevice, copy);
        },
        [&](int half, int64_t first, int64_t docs) {
            return i8_launch_any(Q_i8, q_scale, n_q, l_q, staging_codes + half * block_docs * doc_bytes,
                                 staging_scales + half * block_docs * l_d, nullptr, docs, l_d, docs * (int64_t)l_d, d,
                                 scores + first, b, cus, compute);
        });
}

int maxsim_forward_ragged(const void *Q, int n_q, int l_q, const void *D_packed, const int32_t *doc_offsets, int64_t b,
                          int64_t total_tokens, int d, maxsim_dtype dtype, float *scores, int32_t *argmax, void *stream)
{
    if (!doc_offsets || total_tokens < 1)
        return MAXSIM_ERR_INVALID;
    return forward_common(Q, n_q, l_q, D_packed, doc_offsets, b, 0, total_tokens, d, (int)dtype, scores, argmax, stream);
}

int maxsim_backward(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d, maxsim_dtype dtype,
                    const int32_t *argmax, const float *dscore, float *dQ, float *dD, void *stream)
{
    if (!Q || !D || !argmax || !dscore || !dQ || !dD || n_q < 1 || l_q < 1 || b < 1 || l_d < 1 || !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D, 16) || !aligned(argmax, 4) || !aligned(dscore, 4) || !aligned(dQ, 16) ||
        !aligned(dD, 16))
        return MAXSIM_ERR_INVALID;
    if (b > ((int64_t(1) << 31) - 1) / l_d || (int64_t)n_q * l_q >= (int64_t(1) << 31) ||
        (int64_t)n_q * b >= (int64_t(1) << 40))
        return MAXSIM_ERR_UNSUPPORTED;
    if (!backward_width_ok(d) || !backward_q_ok(n_q, l_q, d, (int)dtype, b * (int64_t)l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::backward_launch(Q, n_q, l_q, D, nullptr, b, l_d, b * (int64_t)l_d, d, (int)dtype, argmax, dscore,
                                          dQ, dD, num_cu(), static_cast<hipStream_t>(stream)));
}

int maxsim_backward_ragged(const void *Q, int n_q, int l_q, const void *D_packed, const int32_t *doc_offsets, int64_t b,
                           int64_t total_tokens, int d, maxsim_dtype dtype, const int32_t *argmax, const float *dscore,
                           float *dQ, float *dD_packed, void *stream)
{
    if (!Q || !D_packed || !doc_offsets || !argmax || !dscore || !dQ || !dD_packed || n_q < 1 || l_q < 1 || b < 1 ||
        total_tokens < 1 || !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D_packed, 16) || !aligned(doc_offsets, 4) || !aligned(argmax, 4) ||
        !aligned(dscore, 4) || !aligned(dQ, 16) || !aligned(dD_packed, 16))
        return MAXSIM_ERR_INVALID;
    if (!backward_width_ok(d) || !backward_q_ok(n_q, l_q, d, (int)dtype, total_tokens))
        return MAXSIM_ERR_UNSUPPORTED;
    if (total_tokens >= (int64_t(1) << 31) || b >= (int64_t(1) << 31) || (int64_t)n_q * l_q >= (int64_t(1) << 31) ||
        (int64_t)n_q * b >= (int64_t(1) << 40))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::backward_launch(Q, n_q, l_q, D_packed, doc_offsets, b, 0, total_tokens, d, (int)dtype, argmax,
                                          dscore, dQ, dD_packed, num_cu(), static_cast<hipStream_t>(stream)));
}

static bool csr_shape_ok(int n_q, int64_t b, int l_q, int l_d)
{
    return l_d <= 4096 && b * (int64_t)l_d < (int64_t(1) << 31) - 1 && b < (int64_t(1) << 31) &&
           (int64_t)n_q * l_q < (int64_t(1) << 31) && (int64_t)n_q * l_q * b < (int64_t(1) << 31);
}

int maxsim_csr_build(const int32_t *argmax, int n_q, int64_t b, int l_q, int l_d, int32_t *row_ptr, int32_t *col_idx,
                     void *stream)
{
    if (!argmax || !row_ptr || !col_idx || n_q < 1 || l_q < 1 || b < 1 || l_d < 1)
        return MAXSIM_ERR_INVALID;
    if (!aligned(argmax, 4) || !aligned(row_ptr, 4) || !aligned(col_idx, 4))
        return MAXSIM_ERR_INVALID;
    if (!csr_shape_ok(n_q, b, l_q, l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::csr_build_launch(argmax, n_q, b, l_q, l_d, row_ptr, col_idx, num_cu(),
                                           static_cast<hipStream_t>(stream)));
}

int maxsim_backward_csr(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d, maxsim_dtype dtype,
                        const int32_t *argmax, const float *dscore, int32_t *row_ptr, int32_t *col_idx, float *dQ,
                        float *dD, void *stream)
{
    if (!Q || !D || !argmax || !dscore || !row_ptr || !col_idx || !dQ || !dD || n_q < 1 || l_q < 1 || b < 1 || l_d < 1 ||
        !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D, 16) || !aligned(argmax, 4) || !aligned(dscore, 4) || !aligned(row_ptr, 4) ||
        !aligned(col_idx, 4) || !aligned(dQ, 16) || !aligned(dD, 16))
        return MAXSIM_ERR_INVALID;
    if (!csr_shape_ok(n_q, b, l_q, l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (!backward_width_ok(d) || !backward_q_ok(n_q, l_q, d, (int)dtype, b * (int64_t)l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::backward_csr_launch(Q, n_q, l_q, D, b, l_d, d, (int)dtype, argmax, dscore, row_ptr, col_idx, dQ,
                                              dD, num_cu(), static_cast<hipStream_t>(stream)));
}

int maxsim_backward_csr_static(const void *Q, int n_q, int l_q, const void *D, int64_t b, int l_d, int d,
                               maxsim_dtype dtype, const int32_t *argmax, const float *dscore, float *dQ, float *dD,
                               void *stream)
{
    if (!Q || !D || !argmax || !dscore || !dQ || !dD || n_q < 1 || l_q < 1 || b < 1 || l_d < 1 || !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q, 16) || !aligned(D, 16) || !aligned(argmax, 4) || !aligned(dscore, 4) || !aligned(dQ, 16) ||
        !aligned(dD, 16))
        return MAXSIM_ERR_INVALID;
    if (!csr_shape_ok(n_q, b, l_q, l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (!backward_width_ok(d) || !backward_q_ok(n_q, l_q, d, (int)dtype, b * (int64_t)l_d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (!maxsim::csr_static_fits(n_q, b, l_q, l_d))
        return MAXSIM_ERR_SCRATCH;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::backward_csr_static_launch(Q, n_q, l_q, D, b, l_d, d, (int)dtype, argmax, dscore, dQ, dD, num_cu(),
                                                     static_cast<hipStream_t>(stream)));
}

int maxsim_quantize_rows_i8(const void *X, int64_t rows, int d, maxsim_dtype dtype, int8_t *X_i8, float *scale,
                            void *stream)
{
    if (!X || !X_i8 || !scale || rows < 1 || !dtype_ok((int)dtype))
        return MAXSIM_ERR_INVALID;
    if (!aligned(X, 16) || !aligned(X_i8, 16) || !aligned(scale, 4))
        return MAXSIM_ERR_INVALID;
    if (!i8_width_ok(d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (rows >= (int64_t(1) << 40))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    if (d != maxsim::D_MODEL)
        return finish(maxsim::quantize_wide_launch(X, rows, d, (int)dtype, X_i8, scale, static_cast<hipStream_t>(stream)));
    return finish(maxsim::quantize_launch(X, rows, (int)dtype, X_i8, scale, static_cast<hipStream_t>(stream)));
}

int maxsim_forward_i8(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q, const int8_t *D_i8,
                      const float *d_scale, int64_t b, int l_d, int d, float *scores, void *stream)
{
    if (!Q_i8 || !q_scale || !D_i8 || !d_scale || !scores || n_q < 1 || l_q < 1 || b < 1 || l_d < 1)
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q_i8, 16) || !aligned(D_i8, 16) || !aligned(q_scale, 4) || !aligned(d_scale, 4) || !aligned(scores, 4))
        return MAXSIM_ERR_INVALID;
    if (!i8_width_ok(d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (b >= (int64_t(1) << 31) || (int64_t)n_q * ((l_q + 31) / 32) >= (int64_t(1) << 24) ||
        l_q > 1024 || b * (int64_t)l_d >= (int64_t(1) << 31))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(i8_launch_any(Q_i8, q_scale, n_q, l_q, D_i8, d_scale, nullptr, b, l_d, b * (int64_t)l_d, d, scores, b,
                                num_cu(), static_cast<hipStream_t>(stream)));
}

int maxsim_forward_i8_ragged(const int8_t *Q_i8, const float *q_scale, int n_q, int l_q, const int8_t *D_i8_packed,
                             const float *d_scale_packed, const int32_t *doc_offsets, int64_t b, int64_t total_tokens,
                             int d, float *scores, void *stream)
{
    if (!Q_i8 || !q_scale || !D_i8_packed || !d_scale_packed || !doc_offsets || !scores || n_q < 1 || l_q < 1 || b < 1 ||
        total_tokens < 1)
        return MAXSIM_ERR_INVALID;
    if (!aligned(Q_i8, 16) || !aligned(D_i8_packed, 16) || !aligned(q_scale, 4) || !aligned(d_scale_packed, 4) ||
        !aligned(doc_offsets, 4) || !aligned(scores, 4))
        return MAXSIM_ERR_INVALID;
    if (!i8_width_ok(d))
        return MAXSIM_ERR_UNSUPPORTED;
    if (b >= (int64_t(1) << 31) || total_tokens >= (int64_t(1) << 31) ||
        (int64_t)n_q * ((l_q + 31) / 32) >= (int64_t(1) << 24) || l_q > 1024)
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(i8_launch_any(Q_i8, q_scale, n_q, l_q, D_i8_packed, d_scale_packed, doc_offsets, b, 0, total_tokens, d,
                                scores, b, num_cu(), static_cast<hipStream_t>(stream)));
}

int maxsim_ce_grad(const float *scores, int n, int b, float tau, float *g, float *loss, void *stream)
{
    if (!scores || !g || n < 1 || b < n || !(tau > 0.0f))
        return MAXSIM_ERR_INVALID;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::ce_grad_launch(scores, n, b, tau, g, loss, static_cast<hipStream_t>(stream)));
}

int maxsim_rope(const void *X, int64_t tokens, int heads, int d, int64_t x_token_stride, int64_t x_head_stride, maxsim_dtype dtype, const float *freqs, int rot,
                const int32_t *positions, const int32_t *offsets, int64_t b, float scale, int neighbours, int inverse, void *Y, int64_t y_token_stride, int64_t y_head_stride,
                void *stream)
{
    if (!X || !Y || !freqs || tokens < 1 || heads < 1 || d < 2 || rot < 2 || rot > d || rot % 2 != 0 || !dtype_ok((int)dtype) || (offsets && b < 1) || is_nan(scale))
        return MAXSIM_ERR_INVALID;
    if (x_token_stride < 0 || x_head_stride < 0 || !rows_apart(tokens, heads, d, y_token_stride, y_head_stride))
        return MAXSIM_ERR_INVALID;
    const uintptr_t size = dtype == MAXSIM_F32 ? 4 : 2;
    if (!aligned(X, size) || !aligned(Y, size) || !aligned(freqs, 4) || !aligned(positions, 4) || !aligned(offsets, 4))
        return MAXSIM_ERR_INVALID;
    if (!maxsim::rope_width_ok(rot) || tokens >= (int64_t(1) << 31) || b >= (int64_t(1) << 31) || (int64_t)heads * d >= (int64_t(1) << 24))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::rope_launch(X, tokens, heads, d, x_token_stride, x_head_stride, (int)dtype, freqs, rot, positions, offsets, b, scale, neighbours != 0, inverse != 0, Y,
                                      y_token_stride, y_head_stride, static_cast<hipStream_t>(stream)));
}

int64_t maxsim_attention_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d)
{
    return attention_sizes_ok(b, q_tokens, k_tokens, hq, hkv, d) != MAXSIM_OK ? 0 : maxsim::attention_workspace(b, q_tokens, k_tokens, hq, hkv, d, num_cu());
}

int maxsim_attention(const void *Q, const void *K, const void *V, const int64_t *strides, const int32_t *q_offsets, const int32_t *k_offsets, int64_t b, int64_t q_tokens,
                     int64_t k_tokens, int hq, int hkv, int d, maxsim_dtype dtype, int causal, float scale, void *O, float *lse, void *workspace, int64_t workspace_bytes,
                     void *stream)
{
    maxsim::AttnParams p = {};
    const AttnTensor t[4] = {{&p.Q, Q, hq}, {&p.K, K, hkv}, {&p.V, V, hkv}, {&p.O, O, hq, q_tokens}};
    if (int rc = attention_common(p, t, 4, strides, q_offsets, k_offsets, b, q_tokens, k_tokens, hq, hkv, d, dtype, causal, scale, workspace, workspace_bytes,
                                  maxsim_attention_workspace(b, q_tokens, k_tokens, hq, hkv, d)))
        return rc;
    if (!aligned(lse, 4))
        return MAXSIM_ERR_INVALID;
    p.lse = lse;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::attention_launch(p, (int)dtype, workspace, num_cu(), static_cast<hipStream_t>(stream)));
}

int64_t maxsim_attention_backward_workspace(int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d)
{
    return attention_sizes_ok(b, q_tokens, k_tokens, hq, hkv, d) != MAXSIM_OK ? 0 : maxsim::attention_backward_workspace(b, q_tokens, k_tokens, hq, hkv, d, num_cu());
}

int maxsim_attention_backward(const void *Q, const void *K, const void *V, const void *O, const float *lse, const void *dO, const int64_t *strides, const int32_t *q_offsets,
                              const int32_t *k_offsets, int64_t b, int64_t q_tokens, int64_t k_tokens, int hq, int hkv, int d, maxsim_dtype dtype, int causal, float scale,
                              void *dQ, void *dK, void *dV, void *workspace, int64_t workspace_bytes, void *stream)
{
    maxsim::AttnParams p = {};
    const AttnTensor t[8] = {{&p.Q, Q, hq}, {&p.K, K, hkv}, {&p.V, V, hkv}, {&p.O, O, hq}, {&p.dO, dO, hq}, {&p.dQ, dQ, hq, q_tokens}, {&p.dK, dK, hkv, k_tokens}, {&p.dV, dV, hkv, k_tokens}};
    if (int rc = attention_common(p, t, 8, strides, q_offsets, k_offsets, b, q_tokens, k_tokens, hq, hkv, d, dtype, causal, scale, workspace, workspace_bytes,
                                  maxsim_attention_backward_workspace(b, q_tokens, k_tokens, hq, hkv, d)))
        return rc;
    if (!lse || !aligned(lse, 4))
        return MAXSIM_ERR_INVALID;
    p.lse = const_cast<float *>(lse); // (read)
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::attention_backward_launch(p, (int)dtype, workspace, num_cu(), static_cast<hipStream_t>(stream)));
}

int64_t maxsim_clip_workspace(int n) { return n < 1 ? 0 : maxsim::clip_workspace(n); }

int maxsim_clip_grad_norm(const void *const *grads, void *const *out, const int64_t *numel, const int32_t *dtypes, int n, float max_norm, float *norm, void *workspace,
                          int64_t workspace_bytes, void *stream)
{
    if (!grads || !out || !numel || !dtypes || n < 1 || !norm || !aligned(norm, 4) || !workspace || !aligned(workspace, 16) || is_nan(max_norm) || max_norm < 0.0f)
        return MAXSIM_ERR_INVALID;
    if (workspace_bytes < maxsim::clip_workspace(n))
        return MAXSIM_ERR_SCRATCH;
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        const uintptr_t size = dtypes[i] == MAXSIM_F32 ? 4 : 2;
        if (!dtype_ok(dtypes[i]) || numel[i] < 0 || (numel[i] > 0 && (!grads[i] || !out[i])) || !aligned(grads[i], size) || !aligned(out[i], size))
            return MAXSIM_ERR_INVALID;
        if (numel[i] > (int64_t(1) << 50) || (total += numel[i]) > (int64_t(1) << 50))
            return MAXSIM_ERR_UNSUPPORTED;
    }
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::clip_launch(grads, out, numel, dtypes, n, max_norm, norm, workspace, static_cast<hipStream_t>(stream)));
}

int maxsim_embed(const void *W, int64_t vocab, int d, maxsim_dtype dtype, const void *tokens, int token_bytes, int64_t n, float scale, void *Y, maxsim_dtype y_dtype, void *stream)
{
    if (int rc = embed_common(W, dtype, Y, y_dtype, tokens, token_bytes, n, vocab, d, scale))
        return rc;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::embed_launch(W, vocab, d, (int)dtype, tokens, token_bytes == 8, n, scale, Y, (int)y_dtype, static_cast<hipStream_t>(stream)));
}

int64_t maxsim_embed_backward_workspace(int64_t n, int64_t vocab, int d)
{
    return n < 1 || vocab < 1 || d < 1 || n >= (int64_t(1) << 27) || vocab >= (int64_t(1) << 31) - 1 || d > 65536 ? 0 : maxsim::embed_backward_workspace(n, vocab, d);
}

int maxsim_embed_backward(const void *dY, maxsim_dtype dtype, const void *tokens, int token_bytes, int64_t n, int64_t vocab, int d, float scale, int accumulate, void *dW,
                          maxsim_dtype w_dtype, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (int rc = embed_common(dW, w_dtype, dY, dtype, tokens, token_bytes, n, vocab, d, scale))
        return rc;
    if (n >= (int64_t(1) << 27))
        return MAXSIM_ERR_UNSUPPORTED;
    if (!workspace || !aligned(workspace, 16))
        return MAXSIM_ERR_INVALID;
    if (workspace_bytes < maxsim::embed_backward_workspace(n, vocab, d))
        return MAXSIM_ERR_SCRATCH;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::embed_backward_launch(dY, (int)dtype, tokens, token_bytes == 8, n, vocab, d, scale, accumulate != 0, dW, (int)w_dtype, workspace,
                                                static_cast<hipStream_t>(stream)));
}

int maxsim_norm_rope(const void *X, int64_t tokens, int heads, int d, const int64_t *strides, maxsim_dtype dtype, const void *q_weight, const void *k_weight, maxsim_dtype w_dtype,
                     int q_heads, float eps, const float *freqs, int rot, const int32_t *positions, const int32_t *offsets, int64_t b, float scale, int neighbours, void *Y,
                     void *stream)
{
    int64_t plain[4];
    const void *t[2] = {X, Y};
    if (int rc = norm_rope_common(t, 2, tokens, heads, d, strides, plain, dtype, q_weight, k_weight, w_dtype, q_heads, eps, freqs, rot, positions, offsets, b, scale))
        return rc;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::norm_rope_launch(X, tokens, heads, d, strides, (int)dtype, q_weight, k_weight, (int)w_dtype, q_heads, eps,
                                           {freqs, positions, offsets, b, rot / 2, scale, 1.0f}, neighbours != 0, Y, static_cast<hipStream_t>(stream)));
}

int64_t maxsim_norm_rope_backward_workspace(int64_t tokens, int heads, int d)
{
    return tokens < 1 || heads < 1 || d < 2 || d > 512 || heads > 8192 || tokens >= (int64_t(1) << 31) ? 0 : maxsim::norm_rope_backward_workspace(tokens, heads, d);
}

int maxsim_norm_rope_backward(const void *X, const void *dY, int64_t tokens, int heads, int d, const int64_t *strides, maxsim_dtype dtype, const void *q_weight, const void *k_weight,
                              maxsim_dtype w_dtype, int q_heads, float eps, const float *freqs, int rot, const int32_t *positions, const int32_t *offsets, int64_t b, float scale,
                              int neighbours, void *dX, float *dq_weight, float *dk_weight, void *workspace, int64_t workspace_bytes, void *stream)
{
    int64_t plain[6];
    const void *t[3] = {X, dY, dX};
    if (int rc = norm_rope_common(t, 3, tokens, heads, d, strides, plain, dtype, q_weight, k_weight, w_dtype, q_heads, eps, freqs, rot, positions, offsets, b, scale))
        return rc;
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4) || !workspace || !aligned(workspace, 16))
        return MAXSIM_ERR_INVALID;
    if (workspace_bytes < maxsim::norm_rope_backward_workspace(tokens, heads, d))
        return MAXSIM_ERR_SCRATCH;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::norm_rope_backward_launch(X, dY, tokens, heads, d, strides, (int)dtype, q_weight, k_weight, (int)w_dtype, q_heads, eps,
                                                    {freqs, positions, offsets, b, rot / 2, scale, 1.0f}, neighbours != 0, dX, dq_weight, dk_weight, workspace,
                                                    static_cast<hipStream_t>(stream)));
}

int64_t maxsim_distill_workspace(int n, int64_t b, maxsim_dtype dtype)
{
    return n < 1 || b < 1 || b >= (int64_t(1) << 31) || !dtype_ok((int)dtype) ? 0 : maxsim::distill_workspace(n, b, (int)dtype, num_cu());
}

int maxsim_distill(const void *scores, int n, int64_t b, int64_t stride, maxsim_dtype dtype, const void *teacher, maxsim_dtype t_dtype, const int32_t *index, int k, float tau,
                   float *loss, float *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (int rc = distill_common(scores, n, b, stride, dtype, teacher, t_dtype, index, k, tau))
        return rc;
    const int64_t needed = maxsim_distill_workspace(n, b, dtype);
    if (!loss || !aligned(loss, 4) || !aligned(lse, 4) || (needed > 0 && (!workspace || !aligned(workspace, 16))))
        return MAXSIM_ERR_INVALID;
    if (workspace_bytes < needed)
        return MAXSIM_ERR_SCRATCH;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::distill_launch(scores, n, (int)b, stride, (int)dtype, teacher, (int)t_dtype, index, k, tau, loss, lse, nullptr, 0.0f, nullptr, 0, workspace, num_cu(),
                                         static_cast<hipStream_t>(stream)));
}

int maxsim_distill_backward(const void *scores, int n, int64_t b, int64_t stride, maxsim_dtype dtype, const void *teacher, maxsim_dtype t_dtype, const int32_t *index, int k, float tau,
                            const float *lse, const float *dloss, void *g, int64_t g_stride, void *stream)
{
    if (int rc = distill_common(scores, n, b, stride, dtype, teacher, t_dtype, index, k, tau))
        return rc;
    if (!lse || !dloss || !g || !aligned(lse, 4) || !aligned(dloss, 4) || !aligned(g, size_of(dtype)) || g_stride < b || (g == scores && n > 1 && g_stride != stride))
        return MAXSIM_ERR_INVALID;
    if (g_stride >= (int64_t(1) << 40))
        return MAXSIM_ERR_UNSUPPORTED;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::distill_launch(scores, n, (int)b, stride, (int)dtype, teacher, (int)t_dtype, index, k, tau, nullptr, nullptr, dloss, 0.0f, g, g_stride,
                                         nullptr, num_cu(), static_cast<hipStream_t>(stream)));
}

int maxsim_distill_grad(const void *scores, int n, int64_t b, int64_t stride, maxsim_dtype dtype, const void *teacher, maxsim_dtype t_dtype, const int32_t *index, int k, float tau,
                        float weight, void *g, int64_t g_stride, float *loss, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (int rc = distill_common(scores, n, b, stride, dtype, teacher, t_dtype, index, k, tau))
        return rc;
    const int64_t needed = maxsim_distill_workspace(n, b, dtype);
    if (!g || !aligned(g, size_of(dtype)) || g_stride < b || (g == scores && n > 1 && g_stride != stride) || !aligned(loss, 4) || is_nan(weight) || (needed > 0 && (!workspace || !aligned(workspace, 16))))
        return MAXSIM_ERR_INVALID;
    if (g_stride >= (int64_t(1) << 40))
        return MAXSIM_ERR_UNSUPPORTED;
    if (workspace_bytes < needed)
        return MAXSIM_ERR_SCRATCH;
    if (int rc = ensure_init())
        return rc;
    return finish(maxsim::distill_launch(scores, n, (int)b, stride, (int)dtype, teacher, (int)t_dtype, index, k, tau, loss, nullptr, nullptr, weight, g, g_stride, workspace, num_cu(),
                                         static_cast<hipStream_t>(stream)));
}

} // extern "C"
