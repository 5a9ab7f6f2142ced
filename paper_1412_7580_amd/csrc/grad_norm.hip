// The 2-norm of many tensors taken together, and their scaling to a largest norm:
//
//   norm = sqrt(sum over all elements of g^2),   out = g * min(1, max_norm / norm)
//
// The norm reads every element once; clipping reads it once more and writes it once (the coefficient
// is known only when all have been read).  Squares and sums are held in 64 bits: no gradient's square
// leaves that range, and a thousand million terms lose nothing that the fp32 result could show.
// The tensors are cut into pieces of equal length; a block adds up one piece and leaves its sum in the
// workspace, and whoever needs the norm adds all of those in the same order: the result does not
// depend on the order in which blocks run.  The list of tensors travels in the kernel's arguments, so
// nothing is copied to the device and a captured call holds its list itself.
//
// 400 million bf16 elements: norm 175 us (4.6 TB/s), scaling 307 (1.6 GB, 5.2 TB/s: the last of what the norm read
// comes from the cache); a copy runs at 4.8.  (Adding up all pieces in every block costs their number squared: 6 of 24 ms
// for 50000 tensors, nothing for hundreds.)
//
// A norm that is zero, infinite in fp32 or not a number leaves the tensors as they are: the caller sees it in `norm`.
#include "operands.hpp"

namespace fc {
namespace {

constexpr int kThreads = 256;
constexpr int kPerLaunch = 128, kFew = 16;    // tensors in one launch's arguments (29 bytes each, of 4096), and in a short list's
constexpr long kPieces = 2048, kLeast = 8192;      // eight blocks a CU, none of them tiny

template <int CAP>
struct NormArgs {
    const void *in[CAP];
    void *out[CAP];
    long size[CAP];
    int first[CAP + 1];                  // number of the tensor's first piece within this launch
    unsigned char dtype[CAP];
    int count, base;                     // tensors, pieces of earlier launches
    long piece;                          // elements, a multiple of 8
    double *sums;
    float *norm;
    int pieces;                          // of all launches
    float max_norm;
};

template <int CAP>
__device__ __forceinline__ int tensor_of(const NormArgs<CAP> &a, int p) {
    int lo = 0, hi = a.count;            // the last tensor whose first piece is not behind p
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= p) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <class T>
__device__ __forceinline__ double squares(const T *p, long n) {
    double s = 0;
    constexpr int U = 4;
    long i = (long)threadIdx.x * 8;
    for (; i + (U - 1) * kThreads * 8L + 8 <= n; i += U * kThreads * 8L) {
        float f[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) load8(p + i + u * kThreads * 8L, 8, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fma((double)f[u][j], (double)f[u][j], s);
    }
    for (; i < n; i += kThreads * 8L) {
        float f[8];
        load8(p + i, (int)(n - i < 8 ? n - i : 8), f);
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fma((double)f[j], (double)f[j], s);
    }
    return s;
}

template <int CAP>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs<CAP> a) {
    __shared__ double lds[4];
    const int p = blockIdx.x, t = tensor_of(a, p);
    const long from = (long)(p - a.first[t]) * a.piece;
    const long n = a.size[t] - from < a.piece ? a.size[t] - from : a.piece;
    double s;
    if (a.dtype[t] == kF32) s = squares(static_cast<const float *>(a.in[t]) + from, n);
    else if (a.dtype[t] == kBF16) s = squares(static_cast<const __bf16 *>(a.in[t]) + from, n);
    else s = squares(static_cast<const _Float16 *>(a.in[t]) + from, n);
    s = block_sum(s, lds);
    if (threadIdx.x == 0) a.sums[a.base + p] = s;
}

__device__ __forceinline__ double total(const double *sums, int pieces, double *lds) {
    double s = 0;
    for (int i = threadIdx.x; i < pieces; i += kThreads) s += sums[i];
    return block_sum(s, lds);
}

__global__ __launch_bounds__(kThreads) void norm_end_kernel(const double *sums, int pieces, float *norm) {
    __shared__ double lds[4];
    const double s = total(sums, pieces, lds);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// WIDE: a factor below fp32's normal range (2^-126) would lose bits that the results have; it is multiplied in 64 bits.
template <bool WIDE>
__device__ __forceinline__ float product(float v, double factor) {
    return WIDE ? (float)((double)v * factor) : v * (float)factor;
}
template <bool WIDE, class T>
__device__ __forceinline__ void scaled(const T *in, T *out, long n, double factor) {
    constexpr int U = 4;
    long i = (long)threadIdx.x * 8;
    for (; i + (U - 1) * kThreads * 8L + 8 <= n; i += U * kThreads * 8L) {
        float f[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) load8(in + i + u * kThreads * 8L, 8, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[u][j] = product<WIDE>(f[u][j], factor);
            store8(out + i + u * kThreads * 8L, 8, f[u]);
        }
    }
    for (; i < n; i += kThreads * 8L) {
        const int m = (int)(n - i < 8 ? n - i : 8);
        float f[8];
        load8(in + i, m, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = product<WIDE>(f[j], factor);
        store8(out + i, m, f);
    }
}
template <class T>
__device__ __forceinline__ void scaled(const void *in, void *out, long from, long n, double factor) {
    const T *const i = static_cast<const T *>(in) + from;
    T *const o = static_cast<T *>(out) + from;
    if (factor < 0x1p-126) scaled<true>(i, o, n, factor);
    else scaled<false>(i, o, n, factor);
}

// The pieces are walked from the last one back: the end of what the norm read is still in the cache.
template <int CAP>
__global__ __launch_bounds__(kThreads) void clip_kernel(NormArgs<CAP> a) {
    __shared__ double lds[4];
    const double norm = sqrt(total(a.sums, a.pieces, lds));
    if (a.base == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    const bool clip = norm > (double)a.max_norm && (float)norm < INFINITY;
    const double factor = clip ? (double)a.max_norm / norm : 1.0;
    const int p = (int)(gridDim.x - 1 - blockIdx.x), t = tensor_of(a, p);
    if (!clip && a.in[t] == a.out[t]) return;
    const long from = (long)(p - a.first[t]) * a.piece;
    const long n = a.size[t] - from < a.piece ? a.size[t] - from : a.piece;
    if (a.dtype[t] == kF32) scaled<float>(a.in[t], a.out[t], from, n, factor);
    else if (a.dtype[t] == kBF16) scaled<__bf16>(a.in[t], a.out[t], from, n, factor);
    else scaled<_Float16>(a.in[t], a.out[t], from, n, factor);
}

long piece_length(int count, const long *sizes) {
    long total = 0;
    for (int i = 0; i < count; ++i) total += sizes[i];
    const long even = ceil_to((total + kPieces - 1) / kPieces, 2048);
    return even < kLeast ? kLeast : even;
}
long pieces_of(int count, const long *sizes, long piece) {
    long n = 0;
    for (int i = 0; i < count; ++i) n += (sizes[i] + piece - 1) / piece;
    return n;
}

template <int CAP>
hipError_t launch(int count, const void *const *grads, const long *sizes, const int *dtypes, void *const *out, float max_norm,
            float *norm, void *ws, long piece, long pieces, hipStream_t s) {
    NormArgs<CAP> a;
    a.piece = piece;
    a.sums = static_cast<double *>(ws);
    a.norm = norm;
    a.max_norm = max_norm;
    a.pieces = (int)pieces;
    for (int clip = 0; clip < (out ? 2 : 1); ++clip) {
        int base = 0;
        for (int i = 0; i < count;) {
            a.count = 0;
            a.base = base;
            int n = 0;
            for (; i < count && a.count < CAP; ++i) {
                if (sizes[i] == 0) continue;
                const int k = a.count++;
                a.in[k] = grads[i];
                a.out[k] = out ? out[i] : nullptr;
                a.size[k] = sizes[i];
                a.dtype[k] = (unsigned char)dtypes[i];
                a.first[k] = n;
                n += (int)((sizes[i] + piece - 1) / piece);
            }
            a.first[a.count] = n;
            if (!a.count) break;
            if (hipError_t e = run(clip ? clip_kernel<CAP> : norm_kernel<CAP>, dim3(n), kThreads, 0, s, a); e != hipSuccess) return e;
            base += n;
        }
    }
    return hipSuccess;
}

}  // namespace

size_t grad_norm_bytes(int count, const long *sizes) {
    return up((size_t)pieces_of(count, sizes, piece_length(count, sizes)) * sizeof(double), 256);
}

hipError_t launch_grad_norm(int count, const void *const *grads, const long *sizes, const int *dtypes, void *const *out,
                            float max_norm, float *norm, void *ws, hipStream_t s) {
    const long piece = piece_length(count, sizes), pieces = pieces_of(count, sizes, piece);
    const auto lists = count <= kFew ? launch<kFew> : launch<kPerLaunch>;
    if (hipError_t e = lists(count, grads, sizes, dtypes, out, max_norm, norm, ws, piece, pieces, s); e != hipSuccess) return e;
    if (out && pieces) return hipSuccess;
    return run(norm_end_kernel, dim3(1), kThreads, 0, s, static_cast<const double *>(ws), (int)pieces, norm);
}

}  // namespace fc
