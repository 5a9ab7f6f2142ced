/*
 * Plain-C caller of the operators around the passes: embedding, linear cross entropy, gradient norm, on
 * device buffers of the HIP runtime, against their formulas in double; and the refusals that need
 * a handle.  Prints one line per check and exits 0 only if all hold.
 */
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "fftconv.h"

#define HIP_OK(call) do { hipError_t e_ = (call); if (e_ != hipSuccess) { \
    fprintf(stderr, "%s: %s\n", #call, hipGetErrorString(e_)); exit(2); } } while (0)

enum { N = 37, D = 20, V = 53 };
static int failed = 0;

static void expect(const char *what, int ok) {
    printf("%-60s %s\n", what, ok ? " ok" : " WRONG");
    failed += !ok;
}
static void *upload(const void *h, size_t bytes) {
    void *d;
    HIP_OK(hipMalloc(&d, bytes));
    HIP_OK(hipMemcpy(d, h, bytes, hipMemcpyHostToDevice));
    return d;
}
static float *download(const void *d, size_t n) {
    float *h = (float *)malloc(n * sizeof(float));
    HIP_OK(hipDeviceSynchronize());
    HIP_OK(hipMemcpy(h, d, n * sizeof(float), hipMemcpyDeviceToHost));
    return h;
}
static int close_to(const float *got, const double *want, size_t n, double tol) {
    double top = 0, err = 0;
    for (size_t i = 0; i < n; ++i) {
        const double e = fabs(got[i] - want[i]);
        if (!(e <= err)) err = e;
        if (fabs(want[i]) > top) top = fabs(want[i]);
    }
    return err <= tol * top;
}
static uint64_t state = 88172645463325252ull;
static float uniform(void) {
    state ^= state << 13; state ^= state >> 7; state ^= state << 17;
    return (float)(state >> 40) * (2.0f / 16777216.0f) - 1.0f;
}

int main(void) {
    fftconv_handle hd;
    if (fftconv_create(&hd, 0) != FFTCONV_OK) return 2;
    float x[N * D], w[V * D], one[N];
    int64_t t[N];
    for (int i = 0; i < N * D; ++i) x[i] = uniform();
    for (int i = 0; i < V * D; ++i) w[i] = uniform();
    for (int n = 0; n < N; ++n) { t[n] = n % 9 == 4 ? -1 : (n * 31) % V; one[n] = 1; }
    void *dx = upload(x, sizeof x), *dw = upload(w, sizeof w), *dt = upload(t, sizeof t), *dy, *dloss, *dlse, *dgx, *dgw, *dnorm, *ws;
    HIP_OK(hipMalloc(&dy, sizeof x)); HIP_OK(hipMalloc(&dloss, sizeof one)); HIP_OK(hipMalloc(&dlse, sizeof one));
    HIP_OK(hipMalloc(&dgx, sizeof x)); HIP_OK(hipMalloc(&dgw, sizeof w)); HIP_OK(hipMalloc(&dnorm, 16));
    const size_t fwd = fftconv_xent_workspace_bytes(FFTCONV_FPROP, FFTCONV_F32, N, D, V), bwd = fftconv_xent_workspace_bytes(FFTCONV_BPROP, FFTCONV_F32, N, D, V);
    HIP_OK(hipMalloc(&ws, fwd + bwd));

    /* embedding */
    static double ey[N * D], eg[V * D], loss[N], lse[N], gx[N * D], gw[V * D];
    for (int n = 0; n < N; ++n)
        for (int d = 0; d < D; ++d) {
            ey[n * D + d] = t[n] < 0 ? 0 : 2.0 * w[t[n] * D + d];
            if (t[n] >= 0) eg[t[n] * D + d] += 0.5 * x[n * D + d];
        }
    int rc = fftconv_embedding_fprop(hd, FFTCONV_F32, dw, dt, 64, dy, N, D, V, 0, 2.0f);
    expect("embedding_fprop", rc == FFTCONV_OK && close_to(download(dy, N * D), ey, N * D, 1e-6));
    rc = fftconv_embedding_accgrad(hd, FFTCONV_F32, dx, dt, 64, dgw, N, D, V, 0, 0.5f, 0, NULL, 0);
    expect("embedding_accgrad", rc == FFTCONV_OK && close_to(download(dgw, V * D), eg, V * D, 1e-6));

    /* cross entropy, mean over the rows that have a target */
    int rows = 0;
    for (int n = 0; n < N; ++n) rows += t[n] >= 0;
    for (int n = 0; n < N; ++n) {
        if (t[n] < 0) continue;
        double z[V], top = -1e300, sum = 0;
        for (int v = 0; v < V; ++v) {
            z[v] = 0;
            for (int d = 0; d < D; ++d) z[v] += (double)x[n * D + d] * w[v * D + d];
            if (z[v] > top) top = z[v];
        }
        for (int v = 0; v < V; ++v) sum += exp(z[v] - top);
        lse[n] = top + log(sum);
        loss[n] = lse[n] - z[t[n]];
        for (int v = 0; v < V; ++v) {
            const double g = (exp(z[v] - lse[n]) - (v == t[n])) / rows;
            for (int d = 0; d < D; ++d) { gx[n * D + d] += g * w[v * D + d]; gw[v * D + d] += g * x[n * D + d]; }
        }
    }
    rc = fftconv_xent_fprop(hd, FFTCONV_F32, dx, dw, dt, 64, (float *)dloss, (float *)dlse, N, D, V, 0, ws, fwd);
    expect("xent_fprop", rc == FFTCONV_OK && close_to(download(dloss, N), loss, N, 1e-5) && close_to(download(dlse, N), lse, N, 1e-5));
    rc = fftconv_xent_backward(hd, FFTCONV_F32, dx, dw, dt, 64, (float *)dlse, NULL, dgx, dgw, N, D, V, 0, 1.0f, 1, 0, ws, bwd);
    expect("xent_backward", rc == FFTCONV_OK && close_to(download(dgx, N * D), gx, N * D, 1e-5) && close_to(download(dgw, V * D), gw, V * D, 1e-5));

    /* norm of both gradients, and clipping in place */
    double norm = 0;
    for (int i = 0; i < N * D; ++i) norm += gx[i] * gx[i];
    for (int i = 0; i < V * D; ++i) norm += gw[i] * gw[i];
    norm = sqrt(norm);
    const void *grads[2] = {dgx, dgw};
    void *out[2] = {dgx, dgw};
    const long sizes[2] = {N * D, V * D};
    const int types[2] = {FFTCONV_F32, FFTCONV_F32};
    rc = fftconv_grad_clip(hd, 2, grads, sizes, types, out, (float)(norm / 3), (float *)dnorm, NULL, 0);
    for (int i = 0; i < V * D; ++i) gw[i] /= 3;
    expect("grad_clip", rc == FFTCONV_OK && close_to(download(dnorm, 1), &norm, 1, 1e-5) && close_to(download(dgw, V * D), gw, V * D, 1e-5));
    const double third = norm / 3;
    rc = fftconv_grad_norm(hd, 2, grads, sizes, types, (float *)dnorm, ws, fftconv_grad_workspace_bytes(2, sizes));
    expect("grad_norm", rc == FFTCONV_OK && close_to(download(dnorm, 1), &third, 1, 1e-5));

    /* refusals */
#define FPROP(dtype, x_, w_, t_, bits, l_, s_, n_, d_, v_, T_, ws_, b_) \
    fftconv_xent_fprop(hd, dtype, x_, w_, t_, bits, (float *)l_, (float *)s_, n_, d_, v_, T_, ws_, b_)
    expect("no features", FPROP(0, NULL, dw, dt, 64, dloss, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("no weights", FPROP(0, dx, NULL, dt, 64, dloss, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("no targets", FPROP(0, dx, dw, NULL, 64, dloss, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("no loss", FPROP(0, dx, dw, dt, 64, NULL, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("unknown type", FPROP(3, dx, dw, dt, 64, dloss, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("16-bit targets", FPROP(0, dx, dw, dt, 16, dloss, dlse, N, D, V, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("rows that are no whole samples", FPROP(0, dx, dw, dt, 64, dloss, dlse, N, D, V, 5, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("too many features", FPROP(0, dx, dw, dt, 64, dloss, dlse, N, (1 << 20) + 1, V, 0, NULL, 0) == FFTCONV_UNSUPPORTED);
    expect("a short workspace", FPROP(0, dx, dw, dt, 64, dloss, dlse, N, D, V, 0, ws, fwd - 1) == FFTCONV_WORKSPACE_TOO_SMALL);
    expect("a misplaced workspace", FPROP(0, dx, dw, dt, 64, dloss, dlse, N, D, V, 0, (char *)ws + 8, 1 << 20) == FFTCONV_INVALID_ARG);
    expect("no rows", FPROP(0, NULL, NULL, NULL, 64, NULL, NULL, 0, D, V, 0, NULL, 0) == FFTCONV_OK);
    expect("no gradient asked for", fftconv_xent_backward(hd, 0, dx, dw, dt, 64, (float *)dlse, NULL, NULL, NULL, N, D, V, 0, 1.0f, 0, 0, NULL, 0) == FFTCONV_OK);
    expect("no lse", fftconv_xent_backward(hd, 0, dx, dw, dt, 64, NULL, NULL, dgx, NULL, N, D, V, 0, 1.0f, 0, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("no table", fftconv_embedding_fprop(hd, 0, NULL, dt, 64, dy, N, D, V, 0, 1.0f) == FFTCONV_INVALID_ARG);
    expect("no table's gradient", fftconv_embedding_accgrad(hd, 0, dx, dt, 64, NULL, N, D, V, 0, 1.0f, 0, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("a grid beyond one launch", fftconv_embedding_fprop(hd, 0, dw, dt, 64, dy, 1 << 30, 1 << 30, V, 1, 1.0f) == FFTCONV_UNSUPPORTED);
    expect("no norm", fftconv_grad_norm(hd, 2, grads, sizes, types, NULL, NULL, 0) == FFTCONV_INVALID_ARG);
    const void *holes[2] = {dgx, NULL};
    expect("a list with a hole", fftconv_grad_norm(hd, 2, holes, sizes, types, (float *)dnorm, NULL, 0) == FFTCONV_INVALID_ARG);
    void *same[2] = {dgw, dgw};
    expect("one output twice", fftconv_grad_clip(hd, 2, grads, sizes, types, same, 1.0f, (float *)dnorm, NULL, 0) == FFTCONV_INVALID_ARG);
    expect("a limit of zero", fftconv_grad_clip(hd, 2, grads, sizes, types, out, 0.0f, (float *)dnorm, NULL, 0) == FFTCONV_INVALID_ARG);

    HIP_OK(hipDeviceSynchronize());
    fftconv_destroy(hd);
    printf(failed ? "%d checks failed\n" : "all checks passed\n", failed);
    return failed != 0;
}
