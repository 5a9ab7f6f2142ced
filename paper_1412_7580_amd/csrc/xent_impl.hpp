// Softmax cross entropy of a linear classifier, without its scores ever standing in memory:
//
//   z[n, v]  = x[n] . w[v]
//   lse[n]   = log sum over v of exp(z[n, v]),      loss[n] = lse[n] - z[n, target[n]]
//   G[n, v]  = (exp(z[n, v] - lse[n]) - [v = target[n]]) * dL/dloss[n]
//   gx[n]    = sum over v of G[n, v] w[v],          gw[v] = sum over n of G[n, v] x[n]
//
// fprop is one product whose tiles leave a maximum and a sum of exponentials per row, joined by a small
// second kernel.  backward takes the vocabulary in pieces: a piece of G is formed from the product
// and the saved lse, and both gradients' products read it before the next piece overwrites it.
// All three products are matrix-core work: 2 N V D operations each, four of them in a training step with
// the scores formed twice, which costs a third more operations and saves 4 N V bytes written and read.
//
// Rows without a target are taken out before anything else: the rows that have one are packed, so a
// padded batch costs what its filled part costs, and nothing of the other rows is read (whatever
// they hold).  How many there are is only known on the device: grids cover all rows, and what
// lies behind the count ends at once.
//
// G is held in the operands' type (fp32: in three terms): one rounding of each element, half a step
// of its own size, beside the one rounding of the gradients.  fp16 holds it times a power of two
// that lifts the largest dL/dloss to 2^13 .. 2^14: what underflows is below 2^-37 of it.
#pragma once
#include "xent_gemm.hpp"
#include <type_traits>

namespace fc {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------- rows with a target
struct ScanArgs {
    Tokens tok;
    long N;
    int *row_of, *pos, *target;     // by packed row, by row, by packed row
    int *count;
    uint4 *zeros;                   // what the products read in place of columns that are not there
    float *loss, *lse;              // fprop: zero for rows without a target
    const float *lse_in, *gloss;    // backward
    float *lse_out, *coef, *alpha;
    float scale;
    int mean, half_range;           // half_range: G is held in fp16
};

__global__ __launch_bounds__(1024) void xent_scan_kernel(ScanArgs a) {
    constexpr int E = 8;
    __shared__ int waves[16];
    __shared__ float tops[16];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int base = 0;
    float top = 0.f;
    for (long n0 = 0; n0 < a.N; n0 += 1024 * E) {
        int t[E], mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const long n = n0 + tid * E + e;
            t[e] = n < a.N ? a.tok(n) : -1;
            mine += t[e] >= 0;
        }
        int upto = mine;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int v = __shfl_up(upto, m);
            if (lane >= m) upto += v;
        }
        __syncthreads();
        if (lane == 63) waves[w] = upto;
        __syncthreads();
        int at = base + upto - mine, all = 0;
        for (int q = 0; q < 16; ++q) {
            at += q < w ? waves[q] : 0;
            all += waves[q];
        }
        base += all;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const long n = n0 + tid * E + e;
            if (n >= a.N) break;
            const bool has = t[e] >= 0;
            if (a.pos) a.pos[n] = has ? at : -1;
            if (has) {
                a.row_of[at] = (int)n;
                a.target[at] = t[e];
                if (a.gloss) top = fmaxf(top, fabsf(a.gloss[n]));
                ++at;
            } else if (a.loss) {
                a.loss[n] = 0.f;
                a.lse[n] = 0.f;
            }
        }
    }
    if (tid == 0) { *a.count = base; *a.zeros = make_uint4(0, 0, 0, 0); }
    if (!a.coef) return;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) tops[w] = top;
    __syncthreads();
    for (int q = 0; q < 16; ++q) top = fmaxf(top, tops[q]);
    int e = 0;
    if (a.half_range) {
        if (!a.gloss) top = 1.f;
        if (top > 0.f && top < INFINITY) e = 14 - (ilogbf(top) + 1);
        e = e < -100 ? -100 : e > 100 ? 100 : e;
    }
    const float up = ldexpf(1.f, e);
    for (long c = tid; c < base; c += 1024) {
        const int n = a.row_of[c];
        a.lse_out[c] = a.lse_in[n];
        a.coef[c] = (a.gloss ? a.gloss[n] : 1.f) * up;
    }
    if (tid == 0) *a.alpha = base ? ldexpf(a.mean ? a.scale / (float)base : a.scale, -e) : 0.f;
}

// ---------------------------------------------------------------------------------- packing
template <class S, class T, bool SPLIT>
struct PackArgs {
    const S *from;
    T *to;                    // [rows][terms][ld]
    const int *row_of, *count;    // null: rows as they are
    long rows;                // rows behind the count are written as zeros
    int D, ld, T_;            // ld: a multiple of 8, filled with zeros
};

template <class T, bool SPLIT>
__device__ __forceinline__ void put8(T *to, long term, const float (&f)[8]) {
    if constexpr (SPLIT) {
        uint4 h, m, l;
        split2(f[0], f[1], h.x, m.x, l.x);
        split2(f[2], f[3], h.y, m.y, l.y);
        split2(f[4], f[5], h.z, m.z, l.z);
        split2(f[6], f[7], h.w, m.w, l.w);
        *reinterpret_cast<uint4 *>(to) = h;
        *reinterpret_cast<uint4 *>(to + term) = m;
        *reinterpret_cast<uint4 *>(to + 2 * term) = l;
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (T)f[i];
        __builtin_memcpy(__builtin_assume_aligned(to, 16), t, 16);
    }
}

template <class S, class T, bool SPLIT>
__global__ __launch_bounds__(kThreads) void xent_pack_kernel(PackArgs<S, T, SPLIT> a) {
    const long count = a.count ? *a.count : a.rows;
    const int cpr = a.ld / 8;
    const size_t total = (size_t)a.rows * cpr;
    for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < total; c += (size_t)gridDim.x * kThreads) {
        const long r = (long)(c / cpr);
        const int d = (int)(c - (size_t)r * cpr) * 8;
        float f[8] = {};
        if (r < count) load8(a.from + (size_t)(a.row_of ? a.row_of[r] : r) * a.D + d, a.D - d, f);
        put8<T, SPLIT>(a.to + (size_t)r * a.ld * (SPLIT ? 3 : 1) + d, a.ld, f);
    }
}

template <class S, class T, bool SPLIT>
__global__ __launch_bounds__(kThreads) void xent_pack_planes_kernel(PackArgs<S, T, SPLIT> a) {
    __shared__ float tile[64][65];
    const long count = *a.count;
    const unsigned tiles_d = (a.D + 63) / 64;
    const long r0 = (long)(blockIdx.x / tiles_d) * 64;
    const int d0 = (int)(blockIdx.x % tiles_d) * 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long r = r0 + lane;
    if (r < count) {
        const RowsOf at{a.D, a.T_};
        const S *p = a.from + at.offset(a.row_of[r]);
        for (int i = w; i < 64; i += 4) tile[i][lane] = d0 + i < a.D ? to_float(p[(size_t)(d0 + i) * a.T_]) : 0.f;
    } else {
        for (int i = w; i < 64; i += 4) tile[i][lane] = 0.f;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int q = c >> 3, dd = (c & 7) * 8;
        if (d0 + dd >= a.ld || r0 + q >= a.rows) continue;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = tile[dd + i][q];
        put8<T, SPLIT>(a.to + (size_t)(r0 + q) * a.ld * (SPLIT ? 3 : 1) + d0 + dd, a.ld, f);
    }
}

// ---------------------------------------------------------------------------------- ends
struct LossArgs {
    const float2 *part;       // [tiles][ld]
    long ld;
    int tiles;
    const float *hit;
    const int *row_of, *count;
    float *loss, *lse;
};

// 64 rows a block; sixteen threads a row join its tiles' maxima and sums.
__global__ __launch_bounds__(1024) void xent_loss_kernel(LossArgs a) {
    __shared__ float2 both[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, count = *a.count;
    const long m = (long)blockIdx.x * 64 + lane;
    if ((long)blockIdx.x * 64 >= count) return;
    float2 v = make_float2(-INFINITY, 0.f);
    auto join = [](float2 x, float2 y) {
        const float top = fmaxf(x.x, y.x), base = top == -INFINITY ? 0.f : top;
        return make_float2(top, x.y * __expf(x.x - base) + y.y * __expf(y.x - base));
    };
    if (m < count)
        for (int t = w; t < a.tiles; t += 16) v = join(v, a.part[t * a.ld + m]);
    both[w][lane] = v;
    __syncthreads();
    if (w == 0 && m < count) {
        for (int q = 1; q < 16; ++q) v = join(v, both[q][lane]);
        const float lse = v.x + logf(v.y);
        const int n = a.row_of[m];
        a.lse[n] = lse;
        a.loss[n] = lse - a.hit[m];
    }
}

template <class S>
struct RowsOutArgs {
    const float *partial;     // [splits][M][ld]
    const int *pos;           // by row
    const float *alpha;
    S *gx;
    long N, M, ld;
    int splits, D, T_;
};

template <class S>
__device__ __forceinline__ void sum8(const RowsOutArgs<S> &a, int c, int d, float alpha, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
    if (c < 0) return;
    for (int s = 0; s < a.splits; ++s) {
        float v[8];
        load8(a.partial + ((size_t)s * a.M + c) * a.ld + d, a.D - d, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= alpha;
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_rows_out_kernel(RowsOutArgs<S> a) {
    const int cpr = (a.D + 7) / 8;
    const size_t total = (size_t)a.N * cpr;
    const float alpha = *a.alpha;
    for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < total; c += (size_t)gridDim.x * kThreads) {
        const long n = (long)(c / cpr);
        const int d = (int)(c - (size_t)n * cpr) * 8;
        float f[8];
        sum8(a, a.pos[n], d, alpha, f);
        store8(a.gx + (size_t)n * a.D + d, a.D - d, f);
    }
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_planes_out_kernel(RowsOutArgs<S> a) {
    __shared__ float tile[64][65];
    const unsigned tiles_d = (a.D + 63) / 64, tiles_t = (a.T_ + 63) / 64;
    const unsigned per = tiles_d * tiles_t, s = blockIdx.x / per, rest = blockIdx.x - s * per;
    const int t0 = (int)(rest % tiles_t) * 64, d0 = (int)(rest / tiles_t) * 64;
    const float alpha = *a.alpha;
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int q = c >> 3, dd = (c & 7) * 8;
        float f[8] = {};
        if (t0 + q < a.T_ && d0 + dd < a.D) sum8(a, a.pos[(long)s * a.T_ + t0 + q], d0 + dd, alpha, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[dd + i][q] = f[i];
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (t0 + lane < a.T_)
        for (int i = w; i < 64 && d0 + i < a.D; i += 4)
            a.gx[((size_t)s * a.D + d0 + i) * a.T_ + t0 + lane] = (S)tile[i][lane];
}

template <class S>
struct ClassesOutArgs {
    const float *partial;     // [splits][M][ld]
    const float *alpha;
    S *gw;                    // the piece's first row
    long M, ld;
    int splits, D, add;
};

template <class S>
__global__ __launch_bounds__(kThreads) void xent_classes_out_kernel(ClassesOutArgs<S> a) {
    const int cpr = (a.D + 7) / 8;
    const size_t total = (size_t)a.M * cpr;
    const float alpha = *a.alpha;
    for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < total; c += (size_t)gridDim.x * kThreads) {
        const long m = (long)(c / cpr);
        const int d = (int)(c - (size_t)m * cpr) * 8;
        float f[8] = {};
        for (int s = 0; s < a.splits; ++s) {
            float v[8];
            load8(a.partial + ((size_t)s * a.M + m) * a.ld + d, a.D - d, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] += v[i];
        }
        float old[8] = {};
        if (a.add) load8(a.gw + (size_t)m * a.D + d, a.D - d, old);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fmaf(f[i], alpha, old[i]);
        store8(a.gw + (size_t)m * a.D + d, a.D - d, f);
    }
}

// ---------------------------------------------------------------------------------- plan
struct Shape { int big, tiles_m, tiles_n, splits; };
constexpr long kBigPlaces = 256, kSmallPlaces = 512;     // blocks the chip holds at once

// 256x256 tiles where they fill the chip (one block a CU), 128x128 ones (two a CU) where they do not.
// Where the reduction may be split, it is, until there is a block for every place.
Shape shape_of(long M, long N, long K, bool split) {
    const long m2 = (M + 255) / 256, n2 = (N + 255) / 256, m1 = (M + 127) / 128, n1 = (N + 127) / 128;
    const long steps = (K + kStep - 1) / kStep;
    Shape s{};
    const long most = split ? steps / 8 < 1 ? 1 : steps / 8 : 1;
    s.big = m2 * n2 * most >= 192;
    s.tiles_m = (int)(s.big ? m2 : m1);
    s.tiles_n = (int)(s.big ? n2 : n1);
    s.splits = 1;
    if (split) {
        const long tiles = (long)s.tiles_m * s.tiles_n, places = s.big ? kBigPlaces : kSmallPlaces;
        long want = places / tiles;
        if (want > most) want = most;
        if (want > 64) want = 64;
        s.splits = (int)(want < 1 ? 1 : want);
    }
    return s;
}

struct XentPlan {
    long Np;                  // rows, up to a multiple of 256
    int Dp, Dc;               // features, up to a multiple of 8 and of 4
    int terms;
    bool pack_w;
    int piece, pieces;        // classes a piece
    Shape score, rows, classes;
    size_t row_of, pos, target, count, lse, coef, hit, part, x, w, G, gx, gw, total;
};

constexpr size_t kPieceBytes = (size_t)256 << 20;

inline XentPlan xent_plan(bool backward, int dtype, long N, int D, int V, bool aligned) {
    XentPlan p{};
    p.Np = ceil_to(N, 256);
    p.Dp = (int)ceil_to(D, 8);
    p.Dc = (int)ceil_to(D, 4);
    p.terms = dtype == kF32 ? 3 : 1;
    p.pack_w = dtype == kF32 || D % 8 || !aligned;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = up(at + bytes, 256); return o; };
    p.row_of = take((size_t)N * 4);
    p.target = take((size_t)p.Np * 4);                   // (the products read the rows' values a tile at a time)
    p.count = take(32);                                  // count, alpha, and from 16 on zeros
    p.x = take((size_t)p.Np * p.terms * p.Dp * 2);
    p.w = take(p.pack_w ? (size_t)V * p.terms * p.Dp * 2 : 0);
    if (!backward) {
        p.score = shape_of(N, V, D, false);
        p.hit = take((size_t)N * 4);
        p.part = take((size_t)p.score.tiles_n * p.Np * 8);
    } else {
        p.pos = take((size_t)N * 4);
        p.lse = take((size_t)p.Np * 4);
        p.coef = take((size_t)p.Np * 4);
        long most = (long)(kPieceBytes / ((size_t)p.Np * 2 * p.terms)) / 256 * 256;
        if (most < 2048) most = 2048;
        p.pieces = (int)(((long)V + most - 1) / most);
        p.piece = (int)ceil_to(((long)V + p.pieces - 1) / p.pieces, 256);
        p.pieces = (int)(((long)V + p.piece - 1) / p.piece);
        const long widest = p.piece < V ? p.piece : V;
        p.score = shape_of(N, widest, D, false);
        p.rows = shape_of(N, D, widest, true);
        p.classes = shape_of(widest, D, N, true);
        p.G = take((size_t)p.Np * p.terms * ceil_to(widest, 64) * 2);
        p.gx = take((size_t)p.rows.splits * p.Np * p.Dc * 4);
        p.gw = take(p.classes.splits > 1 ? (size_t)p.classes.splits * widest * p.Dc * 4 : 0);
    }
    p.total = at;
    return p;
}

template <class T, int END, bool SPLIT>
hipError_t product(GemmArgs &g, const Shape &sh, hipStream_t s) {
    g.tiles_m = sh.tiles_m; g.tiles_n = sh.tiles_n; g.splits = sh.splits;
    const long tiles = (long)sh.tiles_m * sh.tiles_n * sh.splits, places = sh.big ? kBigPlaces : kSmallPlaces;
    if (tiles > 0x7fffffffL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(tiles < places ? tiles : places));
    if (sh.big) {
        auto k = xent_gemm_kernel<T, 4, 8, 4, 2, END, SPLIT>;
        constexpr int lds = xent_lds_bytes(256, 256, 2);
        if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(k), lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(k, grid, dim3(512), lds, s, g);
    } else {
        auto k = xent_gemm_kernel<T, 4, 4, 2, 2, END, SPLIT>;
        constexpr int lds = xent_lds_bytes(128, 128, 2);
        if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(k), lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(k, grid, dim3(256), lds, s, g);
    }
    return hipGetLastError();
}

inline unsigned blocks_for(size_t chunks) {
    const size_t b = (chunks + kThreads - 1) / kThreads;
    return (unsigned)(b < 1 ? 1 : b < 8192 ? b : 8192);
}

// S: the operands' type in memory; T: the type the matrix cores take.
template <class S, class T, bool SPLIT>
struct Xent {
    const XentCall &c;
    const XentPlan p;
    char *ws;
    hipStream_t s;

    static bool aligned(const void *q) { return ((size_t)q & 15) == 0; }
    Xent(const XentCall &call, bool backward, void *w, hipStream_t st)
        : c(call), p(xent_plan(backward, call.dtype, call.N, call.D, call.V, aligned(call.wt))), ws(static_cast<char *>(w)), s(st) {}

    template <class P> P *at(size_t o) const { return reinterpret_cast<P *>(ws + o); }
    const void *zeros() const { return ws + p.count + 16; }

    hipError_t pack() {
        PackArgs<S, T, SPLIT> a{static_cast<const S *>(c.x), at<T>(p.x), at<int>(p.row_of), at<int>(p.count), p.Np, c.D, p.Dp, c.T};
        if (c.T) {
            const long blocks = p.Np / 64 * ((c.D + 63) / 64);
            if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
            hipLaunchKernelGGL((xent_pack_planes_kernel<S, T, SPLIT>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
        } else {
            hipLaunchKernelGGL((xent_pack_kernel<S, T, SPLIT>), dim3(blocks_for((size_t)p.Np * p.Dp / 8)), dim3(kThreads), 0, s, a);
        }
        if (p.pack_w) {
            PackArgs<S, T, SPLIT> b{static_cast<const S *>(c.wt), at<T>(p.w), nullptr, nullptr, c.V, c.D, p.Dp, 0};
            hipLaunchKernelGGL((xent_pack_kernel<S, T, SPLIT>), dim3(blocks_for((size_t)c.V * p.Dp / 8)), dim3(kThreads), 0, s, b);
        }
        return hipGetLastError();
    }
    GemmSide features() const { return GemmSide{at<T>(p.x), (long)p.terms * p.Dp, p.Dp, p.Np, p.Dp}; }
    GemmSide weights(long v0) const {
        const long ld = (long)p.terms * p.Dp;
        const T *w = p.pack_w ? at<T>(p.w) : static_cast<const T *>(c.wt);
        return GemmSide{w + v0 * ld, ld, p.Dp, c.V - v0, p.Dp};
    }

    hipError_t fprop() {
        ScanArgs sc{};
        sc.tok = c.tok; sc.N = c.N;
        sc.row_of = at<int>(p.row_of); sc.target = at<int>(p.target); sc.count = at<int>(p.count); sc.zeros = at<uint4>(p.count + 16);
        sc.loss = c.loss; sc.lse = c.lse;
        hipLaunchKernelGGL(xent_scan_kernel, dim3(1), dim3(1024), 0, s, sc);
        if (hipError_t e = pack(); e != hipSuccess) return e;
        GemmArgs g{};
        g.P = features(); g.Q = weights(0);
        g.count = sc.count; g.zeros = zeros();
        g.M = (int)p.Np; g.N = c.V; g.K = c.D;
        g.target = sc.target; g.part = at<float2>(p.part); g.part_ld = p.Np; g.hit = at<float>(p.hit);
        if (hipError_t e = product<T, kStats, SPLIT>(g, p.score, s); e != hipSuccess) return e;
        const LossArgs l{g.part, p.Np, p.score.tiles_n, g.hit, sc.row_of, sc.count, c.loss, c.lse};
        hipLaunchKernelGGL(xent_loss_kernel, dim3((unsigned)(p.Np / 64)), dim3(1024), 0, s, l);
        return hipGetLastError();
    }

    hipError_t backward() {
        ScanArgs sc{};
        sc.tok = c.tok; sc.N = c.N;
        sc.row_of = at<int>(p.row_of); sc.pos = at<int>(p.pos); sc.target = at<int>(p.target); sc.count = at<int>(p.count); sc.zeros = at<uint4>(p.count + 16);
        sc.lse_in = c.lse; sc.gloss = c.gloss;
        sc.lse_out = at<float>(p.lse); sc.coef = at<float>(p.coef);
        sc.alpha = reinterpret_cast<float *>(sc.count + 1);
        sc.scale = c.scale; sc.mean = c.mean; sc.half_range = c.dtype == kF16;
        hipLaunchKernelGGL(xent_scan_kernel, dim3(1), dim3(1024), 0, s, sc);
        if (hipError_t e = pack(); e != hipSuccess) return e;
        for (int i = 0; i < p.pieces; ++i) {
            const long v0 = (long)i * p.piece;
            const int width = (int)(c.V - v0 < p.piece ? c.V - v0 : p.piece);
            const long ld = ceil_to(width, 64);
            const GemmSide G{at<T>(p.G), p.terms * ld, ld, p.Np, (int)ld};
            GemmArgs g{};
            g.P = features(); g.Q = weights(v0);
            g.count = sc.count; g.zeros = zeros();
            g.M = (int)p.Np; g.N = width; g.K = c.D;
            g.target = sc.target; g.lse = sc.lse_out; g.coef = sc.coef;
            g.n0 = (int)v0;
            g.G = at<T>(p.G); g.g_ld = ld; g.g_term = ld;
            if (hipError_t e = product<T, kGrad, SPLIT>(g, tiles(p.score, c.N, width), s); e != hipSuccess) return e;
            if (c.gx) {
                GemmArgs r{};
                r.P = G; r.Q = weights(v0);
                r.count = sc.count; r.zeros = zeros();
                r.M = (int)p.Np; r.N = c.D; r.K = width;
                r.partial = at<float>(p.gx); r.part_cols = p.Dc; r.add = i > 0;
                r.alpha_scale = sc.alpha;
                if (hipError_t e = product<T, kRows, SPLIT>(r, p.rows, s); e != hipSuccess) return e;
            }
            if (c.gw) {
                GemmArgs w{};
                w.P = G; w.Q = features();
                w.count = sc.count; w.zeros = zeros();
                w.M = width; w.N = c.D; w.K = (int)c.N;
                w.alpha_scale = sc.alpha;
                S *gw = static_cast<S *>(c.gw) + v0 * c.D;
                const Shape sh = tiles(p.classes, width, c.D);
                if (sh.splits > 1) { w.partial = at<float>(p.gw); w.part_cols = p.Dc; }
                else { w.out = gw; w.out_ld = c.D; w.add = c.accumulate; }
                if (hipError_t e = product<T, kClasses, SPLIT>(w, sh, s); e != hipSuccess) return e;
                if (sh.splits > 1) {
                    const ClassesOutArgs<S> o{at<float>(p.gw), sc.alpha, gw, width, p.Dc, sh.splits, c.D, c.accumulate};
                    hipLaunchKernelGGL(xent_classes_out_kernel<S>, dim3(blocks_for((size_t)width * ((c.D + 7) / 8))), dim3(kThreads), 0, s, o);
                }
            }
        }
        if (c.gx) {
            const RowsOutArgs<S> o{at<float>(p.gx), sc.pos, sc.alpha, static_cast<S *>(c.gx), c.N, p.Np, p.Dc, p.rows.splits, c.D, c.T};
            if (c.T) {
                const long blocks = c.N / c.T * ((c.T + 63) / 64) * ((c.D + 63) / 64);
                if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
                hipLaunchKernelGGL(xent_planes_out_kernel<S>, dim3((unsigned)blocks), dim3(kThreads), 0, s, o);
            } else {
                hipLaunchKernelGGL(xent_rows_out_kernel<S>, dim3(blocks_for((size_t)c.N * ((c.D + 7) / 8))), dim3(kThreads), 0, s, o);
            }
        }
        return hipGetLastError();
    }
    // The last piece may be narrower than the plan's.
    static Shape tiles(Shape sh, long M, long N) {
        const long t = sh.big ? 256 : 128;
        sh.tiles_m = (int)((M + t - 1) / t);
        sh.tiles_n = (int)((N + t - 1) / t);
        return sh;
    }
};

}  // namespace
}  // namespace fc
