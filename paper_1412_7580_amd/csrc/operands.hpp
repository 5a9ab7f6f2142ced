// What the operators around the convolution passes share: the three operand types, loads and stores of
// eight neighbouring elements, token reads, and the launch interface between step_api.hip and the
// kernel files.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace fc {

enum { kF32 = 0, kBF16 = 1, kF16 = 2 };
inline size_t type_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }
inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline long ceil_to(long v, long a) { return (v + a - 1) / a * a; }
// Whether one launch takes so many blocks: it has fewer than 2^32 threads.  (In floating point: sizes up to 2^30 multiply
// beyond 64 bits.)
inline bool grid_fits(double blocks, int threads) { return blocks * threads < 0x1p32; }

// One launch and its own error, whatever an earlier HIP call of the caller's left.  What follows reads what it writes: a
// chain of launches ends with the first that fails.
template <class P> struct Same { typedef P type; };
template <class... P>
hipError_t run(void (*kernel)(P...), dim3 grid, int threads, size_t lds, hipStream_t s, const typename Same<P>::type &...p) {
    void *args[] = {const_cast<void *>(static_cast<const void *>(&p))...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), args, lds, s);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }

// Eight neighbouring elements of a row of which the first n exist (the others are zero).  Rows of odd
// length start at any multiple of the element, so nothing is assumed of the address: gfx950 takes
// 16-byte accesses at any of them.
template <class T>
__device__ __forceinline__ void load8(const T *p, int n, float (&f)[8]) {
    if (n >= 8) {
        T t[8];
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? to_float(p[i]) : 0.f;
    }
}
template <class T>
__device__ __forceinline__ void raw8(const T *p, int n, T (&t)[8]) {
    if (n >= 8) __builtin_memcpy(t, p, sizeof(t));
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : (T)0.f;
}
template <class T>
__device__ __forceinline__ void store8(T *p, int n, const float (&f)[8]) {
    if (n >= 8) {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (T)f[i];
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (T)f[i];
    }
}

// Token n of an int32 or int64 array; -1 for everything outside 0 .. V-1.
struct Tokens {
    const void *p;
    int wide;       // int64
    int V;
    __device__ __forceinline__ int operator()(long n) const {
        const long t = wide ? static_cast<const long *>(p)[n] : (long)static_cast<const int *>(p)[n];
        return t >= 0 && t < V ? (int)t : -1;
    }
};

// Row n of features that lie as rows [N, D] (T = 0) or as planes [N / T, D, T].
struct RowsOf {
    int D, T;
    __device__ __forceinline__ size_t offset(long n) const {
        if (T == 0) return (size_t)n * D;
        const long s = n / T;
        return (size_t)s * D * T + (size_t)(n - s * T);
    }
};

// ---- embedding.hip
size_t embedding_accgrad_bytes(int dtype, long N, int D, int V, int T);
bool embedding_fits(bool accgrad, int dtype, long N, int D, int V, int T);   // whether one launch takes each of its grids
hipError_t launch_embedding_fprop(int dtype, const void *table, Tokens tok, void *y, long N, int D, int T, float scale, hipStream_t s);
hipError_t launch_embedding_accgrad(int dtype, const void *gy, Tokens tok, void *gtable, long N, int D, int T, float scale,
                                    bool accumulate, void *ws, hipStream_t s);

// ---- grad_norm.hip
size_t grad_norm_bytes(int count, const long *sizes);
hipError_t launch_grad_norm(int count, const void *const *grads, const long *sizes, const int *dtypes, void *const *out,
                            float max_norm, float *norm, void *ws, hipStream_t s);

// ---- xent_f32.hip, xent_bf16.hip, xent_f16.hip
struct XentCall {
    int dtype;
    const void *x, *wt;
    Tokens tok;
    long N;
    int D, V, T;
    float *loss;                // fprop
    float *lse;                 // fprop writes it, backward reads it
    const float *gloss;         // backward
    void *gx, *gw;
    float scale;
    bool mean, accumulate;
};
// aligned: the weights start at a multiple of 16 bytes (others are copied).
size_t xent_bytes(bool backward, int dtype, long N, int D, int V, bool aligned);
bool xent_fits(bool backward, int dtype, long N, int D, int V, int T);      // whether one launch takes each of its grids
hipError_t xent_fprop_f32(const XentCall &c, void *ws, hipStream_t s);
hipError_t xent_fprop_bf16(const XentCall &c, void *ws, hipStream_t s);
hipError_t xent_fprop_f16(const XentCall &c, void *ws, hipStream_t s);
hipError_t xent_backward_f32(const XentCall &c, void *ws, hipStream_t s);
hipError_t xent_backward_bf16(const XentCall &c, void *ws, hipStream_t s);
hipError_t xent_backward_f16(const XentCall &c, void *ws, hipStream_t s);

}  // namespace fc
