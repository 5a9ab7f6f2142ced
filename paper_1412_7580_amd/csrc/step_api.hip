// C ABI of the operators around the convolution passes (include/fftconv.h): argument checks,
// workspace, and the launches of embedding.hip, xent_*.hip and grad_norm.hip.
#include "context.hpp"
#include "operands.hpp"

#include <algorithm>
#include <cmath>
#include <new>

using namespace fc;

namespace {

// Calls work on the handle's device, whichever is current, and leave the caller's current.
struct OnDevice {
    int before = -1;
    hipError_t error;
    explicit OnDevice(int device) {
        int now = -1;
        error = hipGetDevice(&now);
        if (error == hipSuccess && now != device) {
            error = hipSetDevice(device);
            if (error == hipSuccess) before = now;
        }
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

constexpr long kMost = 1L << 30;      // rows, features, classes: positions are held in 32 bits
constexpr int kMostFeatures = 1 << 20;    // of the cross entropy: a tile's byte offsets are

int check_sizes(int dtype, int token_bits, long N, int D, int V, int T) {
    if (dtype < 0 || dtype > 2 || (token_bits != 32 && token_bits != 64)) return FFTCONV_INVALID_ARG;
    if (N < 0 || D <= 0 || V <= 0 || T < 0 || (T > 0 && N % T)) return FFTCONV_INVALID_ARG;
    if (N > kMost || D > kMost || V > kMost) return FFTCONV_UNSUPPORTED;
    return FFTCONV_OK;
}

// The workspace of a call: the caller's, or the handle's buffer for these operators.  A captured call keeps the
// address it was given for as long as its graph lives, and that buffer moves when a later call needs more:
// under capture only the caller's will do.
int workspace(fftconv_ctx *c, size_t need, void **ws, size_t bytes) {
    if (*ws) {
        if (reinterpret_cast<size_t>(*ws) & 15) return FFTCONV_INVALID_ARG;
        return bytes < need ? FFTCONV_WORKSPACE_TOO_SMALL : FFTCONV_OK;
    }
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(c->stream, &cap) == hipSuccess && cap != hipStreamCaptureStatusNone) return FFTCONV_WORKSPACE_TOO_SMALL;
    if (c->step_ws_bytes < need) {
        hipError_t e;
        if (c->step_ws) {
            if ((e = hipStreamSynchronize(c->stream)) != hipSuccess) return hip_fail(c, e);
            (void)hipFree(c->step_ws);
            c->step_ws = nullptr; c->step_ws_bytes = 0;
        }
        if ((e = hipMalloc(&c->step_ws, need)) != hipSuccess) return hip_fail(c, e);
        c->step_ws_bytes = need;
    }
    *ws = c->step_ws;
    return FFTCONV_OK;
}

int done(fftconv_ctx *c, hipError_t e) { return e == hipSuccess ? FFTCONV_OK : hip_fail(c, e); }

int check_list(int count, const void *const *grads, const long *sizes, const int *dtypes) {
    if (count < 0 || (count > 0 && (!grads || !sizes || !dtypes))) return FFTCONV_INVALID_ARG;
    long total = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || (sizes[i] > 0 && !grads[i]) || dtypes[i] < 0 || dtypes[i] > 2) return FFTCONV_INVALID_ARG;
        if (sizes[i] > (1L << 40) || (total += sizes[i]) > (1L << 42)) return FFTCONV_UNSUPPORTED;
    }
    return FFTCONV_OK;
}

// No element may be written twice, nor be read as another tensor's after it was written.
int check_apart(int count, const void *const *grads, const long *sizes, const int *dtypes, void *const *out, const float *norm) {
    struct Range { size_t from, to; int tensor; bool written; };
    Range *r = new (std::nothrow) Range[2 * (size_t)count + 1];
    if (!r) return FFTCONV_HIP_ERROR;
    int n = 0;
    r[n++] = Range{(size_t)norm, (size_t)norm + sizeof(float), count, true};
    for (int i = 0; i < count; ++i) {
        if (!sizes[i]) continue;
        const size_t bytes = (size_t)sizes[i] * type_bytes(dtypes[i]), in = (size_t)grads[i], to = (size_t)out[i];
        r[n++] = Range{to, to + bytes, i, true};
        if (in != to) r[n++] = Range{in, in + bytes, i, false};
    }
    std::sort(r, r + n, [](const Range &a, const Range &b) { return a.from < b.from; });
    bool ok = true;
    size_t any = 0, written = 0;          // the ends of the furthest range, and of the furthest written one
    for (int i = 0; i < n && ok; ++i) {
        ok = r[i].from >= (r[i].written ? any : written);
        any = std::max(any, r[i].to);
        if (r[i].written) written = std::max(written, r[i].to);
    }
    delete[] r;
    return ok ? FFTCONV_OK : FFTCONV_INVALID_ARG;
}

int run_norm(fftconv_ctx *hd, int count, const void *const *grads, const long *sizes, const int *dtypes, void *const *out,
             float max_norm, float *norm, void *ws, size_t ws_bytes) {
    const OnDevice on(hd->device);
    if (on.error != hipSuccess) return hip_fail(hd, on.error);
    if (int rc = workspace(hd, grad_norm_bytes(count, sizes) + 256, &ws, ws_bytes); rc != FFTCONV_OK) return rc;
    return done(hd, launch_grad_norm(count, grads, sizes, dtypes, out, max_norm, norm, ws, hd->stream));
}

}  // namespace

extern "C" {

int fftconv_embedding_fprop(fftconv_handle hd, int dtype, const void *table, const void *tokens, int token_bits, void *y,
                            long N, int D, int V, int T, float scale) {
    if (!hd) return FFTCONV_INVALID_ARG;
    if (int rc = check_sizes(dtype, token_bits, N, D, V, T); rc != FFTCONV_OK) return rc;
    if (N == 0) return FFTCONV_OK;
    if (!table || !tokens || !y) return FFTCONV_INVALID_ARG;
    if (!embedding_fits(false, dtype, N, D, V, T)) return FFTCONV_UNSUPPORTED;
    const OnDevice on(hd->device);
    if (on.error != hipSuccess) return hip_fail(hd, on.error);
    return done(hd, launch_embedding_fprop(dtype, table, Tokens{tokens, token_bits == 64, V}, y, N, D, T, scale, hd->stream));
}

size_t fftconv_embedding_workspace_bytes(int dtype, long N, int D, int V, int T) {
    if (check_sizes(dtype, 64, N, D, V, T) != FFTCONV_OK || !embedding_fits(true, dtype, N, D, V, T)) return 0;
    return embedding_accgrad_bytes(dtype, N, D, V, T);
}

int fftconv_embedding_accgrad(fftconv_handle hd, int dtype, const void *gy, const void *tokens, int token_bits, void *gtable,
                              long N, int D, int V, int T, float scale, int accumulate, void *ws, size_t ws_bytes) {
    if (!hd || !gtable) return FFTCONV_INVALID_ARG;
    if (int rc = check_sizes(dtype, token_bits, N, D, V, T); rc != FFTCONV_OK) return rc;
    if (N > 0 && (!gy || !tokens)) return FFTCONV_INVALID_ARG;
    if (!embedding_fits(true, dtype, N, D, V, T)) return FFTCONV_UNSUPPORTED;
    const OnDevice on(hd->device);
    if (on.error != hipSuccess) return hip_fail(hd, on.error);
    if (N > 0)
        if (int rc = workspace(hd, embedding_accgrad_bytes(dtype, N, D, V, T), &ws, ws_bytes); rc != FFTCONV_OK) return rc;
    return done(hd, launch_embedding_accgrad(dtype, gy, Tokens{tokens, token_bits == 64, V}, gtable, N, D, T, scale,
                                             accumulate != 0, ws, hd->stream));
}

size_t fftconv_xent_workspace_bytes(int pass, int dtype, long N, int D, int V) {
    if (check_sizes(dtype, 64, N, D, V, 0) != FFTCONV_OK || D > kMostFeatures || (pass != FFTCONV_FPROP && pass != FFTCONV_BPROP)) return 0;
    if (!xent_fits(pass == FFTCONV_BPROP, dtype, N, D, V, 0)) return 0;
    return xent_bytes(pass == FFTCONV_BPROP, dtype, N, D, V, false);
}

int fftconv_xent_fprop(fftconv_handle hd, int dtype, const void *x, const void *wt, const void *targets, int token_bits,
                       float *loss, float *lse, long N, int D, int V, int T, void *ws, size_t ws_bytes) {
    if (!hd) return FFTCONV_INVALID_ARG;
    if (int rc = check_sizes(dtype, token_bits, N, D, V, T); rc != FFTCONV_OK) return rc;
    if (N == 0) return FFTCONV_OK;
    if (!x || !wt || !targets || !loss || !lse) return FFTCONV_INVALID_ARG;
    if (D > kMostFeatures || !xent_fits(false, dtype, N, D, V, T)) return FFTCONV_UNSUPPORTED;
    const OnDevice on(hd->device);
    if (on.error != hipSuccess) return hip_fail(hd, on.error);
    if (int rc = workspace(hd, xent_bytes(false, dtype, N, D, V, !ws && !(reinterpret_cast<size_t>(wt) & 15)), &ws, ws_bytes); rc != FFTCONV_OK) return rc;
    XentCall c{};
    c.dtype = dtype; c.x = x; c.wt = wt; c.tok = Tokens{targets, token_bits == 64, V};
    c.N = N; c.D = D; c.V = V; c.T = T; c.loss = loss; c.lse = lse;
    return done(hd, dtype == kF32 ? xent_fprop_f32(c, ws, hd->stream) : dtype == kBF16 ? xent_fprop_bf16(c, ws, hd->stream)
                                                                                       : xent_fprop_f16(c, ws, hd->stream));
}

int fftconv_xent_backward(fftconv_handle hd, int dtype, const void *x, const void *wt, const void *targets, int token_bits,
                          const float *lse, const float *gloss, void *gx, void *gw, long N, int D, int V, int T,
                          float scale, int mean, int accumulate, void *ws, size_t ws_bytes) {
    if (!hd) return FFTCONV_INVALID_ARG;
    if (int rc = check_sizes(dtype, token_bits, N, D, V, T); rc != FFTCONV_OK) return rc;
    if (N > 0 && (!x || !wt || !targets || !lse)) return FFTCONV_INVALID_ARG;
    if (D > kMostFeatures || !xent_fits(true, dtype, N, D, V, T)) return FFTCONV_UNSUPPORTED;
    const OnDevice on(hd->device);
    if (on.error != hipSuccess) return hip_fail(hd, on.error);
    if (N == 0)      // no rows: the weights' gradient is zero, as the table's of no tokens is
        return gw ? done(hd, launch_embedding_accgrad(dtype, nullptr, Tokens{nullptr, 0, V}, gw, 0, D, 0, 0.f, accumulate != 0,
                                                      nullptr, hd->stream)) : FFTCONV_OK;
    if (!gx && !gw) return FFTCONV_OK;
    if (int rc = workspace(hd, xent_bytes(true, dtype, N, D, V, !ws && !(reinterpret_cast<size_t>(wt) & 15)), &ws, ws_bytes); rc != FFTCONV_OK) return rc;
    XentCall c{};
    c.dtype = dtype; c.x = x; c.wt = wt; c.tok = Tokens{targets, token_bits == 64, V};
    c.N = N; c.D = D; c.V = V; c.T = T; c.lse = const_cast<float *>(lse); c.gloss = gloss;
    c.gx = gx; c.gw = gw; c.scale = scale; c.mean = mean != 0; c.accumulate = accumulate != 0;
    return done(hd, dtype == kF32 ? xent_backward_f32(c, ws, hd->stream) : dtype == kBF16 ? xent_backward_bf16(c, ws, hd->stream)
                                                                                          : xent_backward_f16(c, ws, hd->stream));
}

size_t fftconv_grad_workspace_bytes(int count, const long *sizes) {
    if (count < 0 || (count > 0 && !sizes)) return 0;
    for (int i = 0; i < count; ++i)
        if (sizes[i] < 0 || sizes[i] > (1L << 40)) return 0;
    return grad_norm_bytes(count, sizes) + 256;
}

int fftconv_grad_norm(fftconv_handle hd, int count, const void *const *grads, const long *sizes, const int *dtypes, float *norm,
                      void *ws, size_t ws_bytes) {
    if (!hd || !norm) return FFTCONV_INVALID_ARG;
    if (int rc = check_list(count, grads, sizes, dtypes); rc != FFTCONV_OK) return rc;
    return run_norm(hd, count, grads, sizes, dtypes, nullptr, 0.f, norm, ws, ws_bytes);
}

int fftconv_grad_clip(fftconv_handle hd, int count, const void *const *grads, const long *sizes, const int *dtypes,
                      void *const *out, float max_norm, float *norm, void *ws, size_t ws_bytes) {
    if (!hd || !norm || !(max_norm > 0.f) || std::isinf(max_norm) || (count > 0 && !out)) return FFTCONV_INVALID_ARG;
    if (int rc = check_list(count, grads, sizes, dtypes); rc != FFTCONV_OK) return rc;
    for (int i = 0; i < count; ++i)
        if (sizes[i] > 0 && !out[i]) return FFTCONV_INVALID_ARG;
    if (int rc = check_apart(count, grads, sizes, dtypes, out, norm); rc != FFTCONV_OK) return rc;
    return run_norm(hd, count, grads, sizes, dtypes, out, max_norm, norm, ws, ws_bytes);
}

}  // extern "C"
