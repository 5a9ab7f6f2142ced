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
// With 8192 rows, 2048 features and 65536 classes in bf16 the step takes 6.9 ms: 1270 TFLOP/s over all four,
// where a library product of that size and layout reaches 1300 (1270 and 1090 for the gradients' layouts).
//
// Rows without a target are taken out before anything else: the rows that have one are packed, so a
// padded batch costs what its filled part costs, and nothing of the other rows is read (whatever
// they hold).  How many there are is only known on the device: grids cover all rows, and what
// lies behind the count ends at once.
//
// G is held in the operands' type (fp32: in three terms): one rounding of each element, half a step
// of its own size, beside the one rounding of the gradients; a few rows bring what it left as well.  fp16 holds it times a power of two
// that lifts the largest dL/dloss to 2^13 .. 2^14: what underflows is below 2^-37 of it.
#pragma once
#include "xent_gemm.hpp"
#include <type_traits>

namespace fc {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------- rows with a target
// The rows that have a target, packed in their order: blocks of 1024 rows place theirs behind those of the
// blocks before them.  Up to kScanInline blocks each counts all rows itself; beyond that the blocks' counts
// come from a launch of their own.  (15488 rows: 38 us by one block, 22 by blocks that count all, 10 by two
// launches.)
constexpr int kScanRows = 1024, kScanInline = 4;

struct ScanArgs {
    Tokens tok;
    long N;
    int blocks;
    int *counts;                    // by block
    float *tops;                    // by block: the largest |dL/dloss|
    int *row_of, *pos, *target;     // by packed row, by row, by packed row
    int *count;
    uint4 *zeros;                   // what the products read in place of columns that are not there
    float *loss, *lse;              // fprop: zero for rows without a target
    const float *lse_in, *gloss;    // backward
    float *lse_out, *coef, *alpha;
    float scale;
    int mean, half_range;           // half_range: G is held in fp16
    int copies;                     // packed rows to a row
};

struct ScanRows { int t[4], mine, upto; float top; };
__device__ __forceinline__ ScanRows scan_rows(const ScanArgs &a, long n0) {
    ScanRows r;
    r.mine = 0; r.top = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const long n = n0 + threadIdx.x * 4 + e;
        r.t[e] = n < a.N ? a.tok(n) : -1;
        r.mine += r.t[e] >= 0;
        if (r.t[e] >= 0 && a.gloss) r.top = fmaxf(r.top, fabsf(a.gloss[n]));
    }
    r.upto = r.mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int v = __shfl_up(r.upto, m);
        if ((threadIdx.x & 63) >= m) r.upto += v;
        r.top = fmaxf(r.top, __shfl_xor(r.top, m));
    }
    return r;
}

__global__ __launch_bounds__(kThreads) void xent_count_kernel(ScanArgs a) {
    __shared__ int counts[4];
    __shared__ float tops[4];
    const ScanRows r = scan_rows(a, (long)blockIdx.x * kScanRows);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane == 63) { counts[w] = r.upto; tops[w] = r.top; }
    __syncthreads();
    if (threadIdx.x == 0) {
        a.counts[blockIdx.x] = counts[0] + counts[1] + counts[2] + counts[3];
        a.tops[blockIdx.x] = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    }
}

__global__ __launch_bounds__(kThreads) void xent_place_kernel(ScanArgs a) {
    __shared__ int waves[4], before[4], all[4];
    __shared__ float tops[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const long n0 = (long)blockIdx.x * kScanRows;
    const ScanRows r = scan_rows(a, n0);
    int b4 = 0, sum = 0;
    float top = r.top;
    if (a.blocks <= kScanInline)
#pragma unroll
        for (int i = 0; i < kScanInline * 4; ++i) {
            const long n = (long)i * kThreads + tid;
            const bool has = n < a.N && a.tok(n) >= 0;
            b4 += has && n < n0;
            sum += has;
            if (has && a.gloss) top = fmaxf(top, fabsf(a.gloss[n]));
        }
    else
        for (int b = tid; b < a.blocks; b += kThreads) {
            const int c = a.counts[b];
            b4 += b < (int)blockIdx.x ? c : 0;
            sum += c;
            top = fmaxf(top, a.tops[b]);
        }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        b4 += __shfl_xor(b4, m);
        sum += __shfl_xor(sum, m);
        top = fmaxf(top, __shfl_xor(top, m));
    }
    if (lane == 63) { waves[w] = r.upto; before[w] = b4; all[w] = sum; tops[w] = top; }
    __syncthreads();
    int at = r.upto - r.mine, total = 0;
    for (int q = 0; q < 4; ++q) {
        at += before[q] + (q < w ? waves[q] : 0);
        total += all[q];
        top = fmaxf(top, tops[q]);
    }
    int e2 = 0;
    if (a.half_range) {
        if (!a.gloss) top = 1.f;
        if (top > 0.f && top < INFINITY) e2 = 14 - (ilogbf(top) + 1);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const long n = n0 + tid * 4 + e;
        if (n >= a.N) break;
        const bool has = r.t[e] >= 0;
        if (a.pos) a.pos[n] = has ? at * a.copies : -1;
        if (has) {
            for (int q = at * a.copies; q < (at + 1) * a.copies; ++q) {
                a.row_of[q] = (int)n;
                a.target[q] = r.t[e];
                if (a.coef) {
                    a.lse_out[q] = a.lse_in[n];
                    a.coef[q] = ldexpf(a.gloss ? a.gloss[n] : 1.f, e2);
                }
            }
            ++at;
        } else if (a.loss) {
            a.loss[n] = 0.f;
            a.lse[n] = 0.f;
        }
    }
    if (blockIdx.x == 0 && tid == 0) {
        *a.count = total * a.copies;
        *a.zeros = make_uint4(0, 0, 0, 0);
        // (in 64 bits: a scale of 2^-140 is still whole when 2^140 comes to it)
        if (a.alpha) *a.alpha = total ? (float)ldexp(a.mean ? (double)a.scale / total : (double)a.scale, -e2) : 0.f;
    }
}

// ---------------------------------------------------------------------------------- packing
// Operands as the products read them: whole rows of a multiple of 8 elements, filled with zeros, the rows that
// have a target only, and fp32 cut into terms.
template <class S>
struct PackArgs {
    const S *from;
    S *to;                    // [rows][ld], or null
    __bf16 *three;            // fp32: [rows][3][ld], where the gradients' products follow
    const int *row_of, *count;    // null: rows as they are
    long rows;                // rows behind the count are written as zeros
    int D, ld, T_;            // ld: a multiple of 8, filled with zeros
};

// (a, b) = h + m + l as split2 cuts them, where a value whose nearest bf16 is infinite goes toward zero: a weight of
// the type's lowest value is multiplied by gradients of zero.
__device__ __forceinline__ unsigned finite_high(float v, unsigned h) {
    const float s = fabsf(v);
    return s >= 0x1.ffp127f && s < INFINITY ? __builtin_bit_cast(unsigned, v) >> 16 : h;
}
__device__ __forceinline__ void cut2(float a, float b, unsigned &h, unsigned &m, unsigned &l) {
    h = pack_bf16(a, b);
    h = finite_high(a, h & 0xffff) | finite_high(b, h >> 16) << 16;
    const float ra = a - low_of(h), rb = b - high_of(h);
    m = pack_bf16(ra, rb);
    l = pack_bf16(ra - low_of(m), rb - high_of(m));
}

// Eight elements of row r from d on, to where they go.
template <class S>
__device__ __forceinline__ void put8(const PackArgs<S> &a, long r, int d, const S (&t)[8]) {
    if (a.to) __builtin_memcpy(__builtin_assume_aligned(a.to + (size_t)r * a.ld + d, 16), t, sizeof(t));
    if constexpr (sizeof(S) == 4)
        if (a.three) {
            uint4 c[3];
            cut2(t[0], t[1], c[0].x, c[1].x, c[2].x);
            cut2(t[2], t[3], c[0].y, c[1].y, c[2].y);
            cut2(t[4], t[5], c[0].z, c[1].z, c[2].z);
            cut2(t[6], t[7], c[0].w, c[1].w, c[2].w);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(a.three + (size_t)r * 3 * a.ld + (size_t)q * a.ld + d) = c[q];
        }
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_pack_kernel(PackArgs<S> a) {
    const long count = a.count ? *a.count : a.rows;
    const int cpr = a.ld / 8;
    const size_t total = (size_t)a.rows * cpr;
    for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < total; c += (size_t)gridDim.x * kThreads) {
        const long r = (long)(c / cpr);
        const int d = (int)(c - (size_t)r * cpr) * 8;
        S t[8] = {};
        if (r < count) raw8(a.from + (size_t)(a.row_of ? a.row_of[r] : r) * a.D + d, a.D - d, t);
        put8(a, r, d, t);
    }
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_pack_planes_kernel(PackArgs<S> a) {
    __shared__ S tile[64][sizeof(S) == 4 ? 65 : 66];
    const long count = *a.count;
    const unsigned tiles_d = (a.D + 63) / 64;
    const long r0 = (long)(blockIdx.x / tiles_d) * 64;
    const int d0 = (int)(blockIdx.x % tiles_d) * 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long r = r0 + lane;
    if (r < count) {
        const RowsOf at{a.D, a.T_};
        const S *p = a.from + at.offset(a.row_of[r]);
        S v[16];                                             // (all asked for before the first is stored)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int d = d0 + i * 4 + w;
            v[i] = p[(size_t)(d < a.D ? d : a.D - 1) * a.T_];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) tile[i * 4 + w][lane] = d0 + i * 4 + w < a.D ? v[i] : (S)0.f;
    } else {
        for (int i = w; i < 64; i += 4) tile[i][lane] = (S)0.f;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int q = c >> 3, dd = (c & 7) * 8;
        if (d0 + dd >= a.ld || r0 + q >= a.rows) continue;
        S t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = tile[dd + i][q];
        put8(a, r0 + q, d0 + dd, t);
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

// (maximum, sum of exponentials less that maximum) of two sets of scores taken together.
__device__ __forceinline__ float2 joined(float2 x, float2 y) {
    const float top = fmaxf(x.x, y.x), base = base_of(top);
    return make_float2(top, x.y * __expf(x.x - base) + y.y * __expf(y.x - base));
}

// 64 rows a block; sixteen threads a row join its tiles' maxima and sums.
constexpr int kLossThreads = 1024;
__global__ __launch_bounds__(kLossThreads) void xent_loss_kernel(LossArgs a) {
    __shared__ float2 both[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, count = *a.count;
    const long m = (long)blockIdx.x * 64 + lane;
    if ((long)blockIdx.x * 64 >= count) return;
    float2 v = make_float2(-INFINITY, 0.f);
    if (m < count)
        for (int t = w; t < a.tiles; t += 16) v = joined(v, a.part[t * a.ld + m]);
    both[w][lane] = v;
    __syncthreads();
    if (w == 0 && m < count) {
        for (int q = 1; q < 16; ++q) v = joined(v, both[q][lane]);
        const float lse = v.x + logf(v.y);
        const int n = a.row_of[m];
        a.lse[n] = lse;
        a.loss[n] = lse - a.hit[m];
    }
}

template <class S>
struct RowsOutArgs {
    const float *partial;     // [splits][rows of live tiles][ld]
    const int *pos, *count;   // pos: by row
    const float *alpha;
    S *gx;
    long N, ld;
    int bm, tiles_n, places, most, D, T_;
    int copies;               // rows of partial to a row
};

// The sum of parts from, from + 1, ... below to, eight of them asked for at a time.
__device__ __forceinline__ void sum_parts(const float *p, size_t stride, int from, int to, int n, float (&f)[8]) {
    constexpr int U = 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
    for (int s = from; s < to; s += U) {
        float v[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < to) load8(p + (s + u) * stride, n, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < to)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += v[u][i];
    }
}

struct RowParts { int splits; size_t stride; };
// Parts from, ... below to, of packed row `at` and of what the rounding of its G left.
template <class S>
__device__ __forceinline__ void sum_row(const RowsOutArgs<S> &a, const RowParts &parts, int at, int d, int from, int to, float (&f)[8]) {
    sum_parts(a.partial + (size_t)at * a.ld + d, parts.stride, from, to, a.D - d, f);
    if (a.copies == 1) return;
    float rest[8];
    sum_parts(a.partial + (size_t)(at + 1) * a.ld + d, parts.stride, from, to, a.D - d, rest);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += rest[i];
}
template <class S>
__device__ __forceinline__ RowParts parts_of(const RowsOutArgs<S> &a) {
    const int tiles_m = (*a.count + a.bm - 1) / a.bm;
    return RowParts{rows_splits((long)tiles_m * a.tiles_n, a.places, a.most), (size_t)tiles_m * a.bm * a.ld};
}

// G threads share a piece of eight columns where there are many parts and few rows.
template <class S, int G>
__global__ __launch_bounds__(kThreads) void xent_rows_out_kernel(RowsOutArgs<S> a) {
    __shared__ float sums[G > 1 ? kThreads : 1][9];
    constexpr int B = kThreads / G;
    const int cpr = (a.D + 7) / 8, g = threadIdx.x / B;
    const size_t total = (size_t)a.N * cpr;
    const float alpha = *a.alpha;
    const RowParts parts = parts_of(a);
    const int each = (parts.splits + G - 1) / G, from = g * each, to = from + each < parts.splits ? from + each : parts.splits;
    for (size_t c0 = (size_t)blockIdx.x * B; c0 < total; c0 += (size_t)gridDim.x * B) {
        const size_t c = c0 + threadIdx.x % B;
        const long n = (long)(c / cpr);
        const int d = (int)(c - (size_t)n * cpr) * 8, at = c < total ? a.pos[n] : -1;
        float f[8] = {};
        if (at >= 0) sum_row(a, parts, at, d, from, to, f);
        if constexpr (G > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = f[i];
            __syncthreads();
            if (g > 0) continue;
            for (int q = 1; q * each < parts.splits; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += sums[q * B + threadIdx.x][i];
        }
        if (at >= 0)                                         // (else zero, whatever the scale)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= alpha;
        if (c < total) store8(a.gx + (size_t)n * a.D + d, a.D - d, f);
    }
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_planes_out_kernel(RowsOutArgs<S> a) {
    __shared__ float tile[64][65];
    const unsigned tiles_d = (a.D + 63) / 64, tiles_t = (a.T_ + 63) / 64;
    const unsigned per = tiles_d * tiles_t, s = blockIdx.x / per, rest = blockIdx.x - s * per;
    const int t0 = (int)(rest % tiles_t) * 64, d0 = (int)(rest / tiles_t) * 64;
    const float alpha = *a.alpha;
    const RowParts parts = parts_of(a);
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int q = c >> 3, dd = (c & 7) * 8;
        float f[8] = {};
        if (t0 + q < a.T_ && d0 + dd < a.D) {
            const int at = a.pos[(long)s * a.T_ + t0 + q];
            if (at >= 0) {
                sum_row(a, parts, at, d0 + dd, 0, parts.splits, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= alpha;
            }
        }
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
        float f[8];
        sum_parts(a.partial + (size_t)m * a.ld + d, (size_t)a.M * a.ld, 0, a.splits, a.D - d, f);
        float old[8] = {};
        if (a.add) load8(a.gw + (size_t)m * a.D + d, a.D - d, old);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fmaf(f[i], alpha, old[i]);
        store8(a.gw + (size_t)m * a.D + d, a.D - d, f);
    }
}

// ---------------------------------------------------------------------------------- few rows
// Up to a few tiles of rows the product is a read of the weights.  A block keeps its rows in LDS, whole, and
// its waves walk the classes 16 at a time, from memory straight to the matrix cores: 16 bytes a lane, two
// batches of eight loads in flight, the next tile's behind this one's, and no barrier on the way.  A lane
// keeps the running maximum and sum of its own classes; lanes, waves and blocks are joined at the end.  Rows
// need no packing: one without a target is zeros in LDS.  fp32 is multiplied in fp32 (16x16x4).
template <class S> struct Thin;
template <> struct Thin<float> {
    typedef floatx4 frag;
    static constexpr int k = 16;                             // of the reduction per 16 bytes of four lanes
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = Mfma<float>::mul(a, b, c, i);
        return c;
    }
};
template <> struct Thin<__bf16> : Mfma<__bf16> { static constexpr int k = 32; };
template <> struct Thin<_Float16> : Mfma<_Float16> { static constexpr int k = 32; };

constexpr int kThinThreads = 512, kThinWaves = 8;
constexpr int kThinLds = 140 * 1024;

template <class S>
struct ThinArgs {
    const S *x, *wt;
    Tokens tok;
    long N;
    int D, V, T_, blocks;     // blocks: of one group of rows
    float2 *part;             // [N][blocks]
    float *hit;
    float *loss, *lse;
};

template <class S, int NT>
__global__ __launch_bounds__(kThinThreads, NT < 4 ? 4 : 2) void xent_thin_kernel(ThinArgs<S> a) {
    typedef typename Thin<S>::frag F;
    constexpr int E = 16 / sizeof(S), KS = Thin<S>::k, R = NT * 16;   // elements of 16 bytes, k of one load, rows
    constexpr int AHEAD = 8;
    extern __shared__ __align__(16) char lds[];
    float2 (*const both)[R] = reinterpret_cast<float2 (*)[R]>(lds);                // [waves]
    int *const live = reinterpret_cast<int *>(lds + kThinWaves * R * 8);
    S *const xs = reinterpret_cast<S *>(lds + kThinWaves * R * 8 + R * 4);
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
    const long r0 = (long)blockIdx.y * R;
    const int steps = (a.D + KS - 1) / KS, batches = (steps + AHEAD - 1) / AHEAD, pitch = steps * KS + E;
    const int tiles = (a.V + 15) / 16, stride = a.blocks * kThinWaves;

    auto load = [&](F (&f)[AHEAD], int tile, int batch) {
        int v = tile * 16 + (lane & 15);
        if (v >= a.V) v = a.V - 1;
        const S *p = a.wt + (size_t)v * a.D + batch * AHEAD * KS + g * E;
        const int left = a.D - batch * AHEAD * KS;           // of the reduction
        if (left >= AHEAD * KS) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) __builtin_memcpy(&f[i], p + i * KS, 16);
        } else {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (left >= (i + 1) * KS) __builtin_memcpy(&f[i], p + i * KS, 16);
                else if (left > i * KS) {
                    S t[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) t[e] = i * KS + g * E + e < left ? p[i * KS + e] : (S)0.f;
                    __builtin_memcpy(&f[i], t, 16);
                }
            }
        }
    };
    int tile = blockIdx.x * kThinWaves + w, batch = 0;
    F now[AHEAD], next[AHEAD];
    if (tile < tiles) load(now, tile, 0);

    if (tid < R) live[tid] = r0 + tid < a.N && a.tok(r0 + tid) >= 0;
    __syncthreads();
    if (a.T_ == 0) {
        const int pieces = steps * KS / E, all = R * pieces;
        constexpr int U = 4;
        for (int c0 = tid; c0 < all; c0 += U * kThinThreads) {
            F f[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * kThinThreads, r = c / pieces, k = (c - r * pieces) * E;
                f[u] = F{};
                if (c >= all || !live[r]) continue;
                const S *p = a.x + (size_t)(r0 + r) * a.D + k;
                if (k + E <= a.D) __builtin_memcpy(&f[u], p, 16);
                else {
                    S t[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) t[e] = k + e < a.D ? p[e] : (S)0.f;
                    __builtin_memcpy(&f[u], t, 16);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * kThinThreads, r = c / pieces, k = (c - r * pieces) * E;
                if (c < all) __builtin_memcpy(__builtin_assume_aligned(&xs[r * pitch + k], 16), &f[u], 16);
            }
        }
    } else {
        const RowsOf at{a.D, a.T_};
        for (int c = tid; c < R * steps * KS; c += kThinThreads) {
            const int r = c % R, k = c / R;
            xs[r * pitch + k] = live[r] && k < a.D ? a.x[at.offset(r0 + r) + (size_t)k * a.T_] : (S)0.f;
        }
    }
    __syncthreads();

    int target[NT];
    float top[NT], sum[NT];
    floatx4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const long n = r0 + t * 16 + (lane & 15);
        target[t] = n < a.N ? a.tok(n) : -1;
        top[t] = -INFINITY; sum[t] = 0.f;
        acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const S *const xl = xs + (lane & 15) * pitch + g * E;
    while (tile < tiles) {
        int next_tile = tile, next_batch = batch + 1;
        if (next_batch == batches) { next_batch = 0; next_tile += stride; }
        if (next_tile < tiles) load(next, next_tile, next_batch);
        const S *const xk = xl + batch * AHEAD * KS;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (batch * AHEAD + i >= steps) break;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                F f;
                __builtin_memcpy(&f, __builtin_assume_aligned(xk + t * 16 * pitch + i * KS, 16), 16);
                acc[t] = Thin<S>::mul(now[i], f, acc[t]);
            }
        }
        if (next_batch == 0) {
            // a lane holds row lane & 15 of each tile of rows and the four classes from 4 (lane >> 4) on
            const int v0 = tile * 16 + g * 4;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int rel = target[t] - v0;
                if (rel >= 0 && rel < 4) {
                    float z = 0.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) z = rel == r ? acc[t][r] : z;
                    a.hit[r0 + t * 16 + (lane & 15)] = z;
                }
                float high = -INFINITY;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (v0 + r >= a.V) acc[t][r] = -INFINITY;
                    high = fmaxf(high, acc[t][r]);
                }
                const float m = fmaxf(top[t], high), base = base_of(m);
                float s = sum[t] * __expf(top[t] - base);
#pragma unroll
                for (int r = 0; r < 4; ++r) s += __expf(acc[t][r] - base);
                top[t] = m; sum[t] = s;
                acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) now[i] = next[i];
        tile = next_tile; batch = next_batch;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float2 v = make_float2(top[t], sum[t]);
        v = joined(v, make_float2(__shfl_xor(v.x, 16), __shfl_xor(v.y, 16)));
        v = joined(v, make_float2(__shfl_xor(v.x, 32), __shfl_xor(v.y, 32)));
        if (lane < 16) both[w][t * 16 + lane] = v;
    }
    __syncthreads();
    if (tid < R && r0 + tid < a.N) {
        float2 v = both[0][tid];
        for (int q = 1; q < kThinWaves; ++q) v = joined(v, both[q][tid]);
        a.part[(size_t)(r0 + tid) * a.blocks + blockIdx.x] = v;
    }
}

template <class S>
__global__ __launch_bounds__(kThreads) void xent_thin_loss_kernel(ThinArgs<S> a) {
    __shared__ float2 both[4];
    const long n = blockIdx.x;
    if (a.tok(n) < 0) {
        if (threadIdx.x == 0) { a.loss[n] = 0.f; a.lse[n] = 0.f; }
        return;
    }
    float2 v = make_float2(-INFINITY, 0.f);
    for (int b = threadIdx.x; b < a.blocks; b += kThreads) v = joined(v, a.part[(size_t)n * a.blocks + b]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = joined(v, make_float2(__shfl_xor(v.x, m), __shfl_xor(v.y, m)));
    if ((threadIdx.x & 63) == 0) both[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        v = joined(joined(both[0], both[1]), joined(both[2], both[3]));
        const float lse = v.x + logf(v.y);
        a.lse[n] = lse;
        a.loss[n] = lse - a.hit[n];
    }
}

// ---------------------------------------------------------------------------------- plan
struct Shape { int bm, bn, tiles_m, tiles_n, splits, most; };     // most: what the reduction's length allows of splits
constexpr long kBigPlaces = 256, kSmallPlaces = 512;     // blocks the chip holds at once
inline long places(const Shape &s) { return s.bm == 256 ? kBigPlaces : kSmallPlaces; }

// Tiles of 256x256 where they fill the chip (one block a CU), of 128x128 (two a CU) where they do not.
// Where the reduction may be split, it is, until there is a block for every place; such products take
// tiles 192 columns wide where that covers the columns with less (384 columns: 97 -> 75 us for 15488 rows
// and 1000 classes in fp32).  fp32 scores take the small tiles: at a sixteenth of the 16-bit rate nothing but the matrix
// instructions bounds them, and with four to a fragment the large ones spill.
inline Shape shape_of(long M, long N, long K, int terms, bool split, bool small = false) {
    const long steps = (K + kStep - 1) / kStep, parts = steps * (terms == 3 ? 6 : 1) / 6;      // of six products at least
    Shape s{};
    s.most = split ? (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts) : 1;
    const auto tiles = [](long n, long t) { return (n + t - 1) / t; };
    s.bm = 256;
    s.bn = split && tiles(N, 192) * 192 < tiles(N, 256) * 256 ? 192 : 256;
    if (small || tiles(M, s.bm) * tiles(N, s.bn) * s.most < 192) s.bm = s.bn = 128;
    s.tiles_m = (int)tiles(M, s.bm);
    s.tiles_n = (int)tiles(N, s.bn);
    s.splits = rows_splits((long)s.tiles_m * s.tiles_n, (int)places(s), s.most);
    return s;
}

struct XentPlan {
    int copies;               // packed rows to a row
    long R, Np;               // packed rows at most, and up to a multiple of 256
    int Dp, Dc;               // features, up to a multiple of 8 and of 4
    int terms;                // of fp32 in the gradients' products
    bool pack_w;
    int thin_tiles, thin_blocks, thin_lds;    // tiles of 16 rows in a block (0: not that path), blocks of a group of rows
    int piece, pieces;        // classes a piece
    Shape score, rows, classes;
    int scan_blocks;
    size_t row_of, pos, target, count, counts, tops, lse, coef, hit, part, x, w, x3, w3, G, gx, gw, total;
};

// Few rows: as many tiles of 16 of them as a block's LDS holds, four at most.  More groups of rows than one
// read the weights again; the other path reads them once, but packs the rows, wastes most of a 128-row tile and
// copies weights whose rows are no whole 16 bytes.  32000 classes of 1024 features,
// us by this path and the other: bf16 18 and 32 (1 row), 27 and 33 (128, two groups), 39 and 37 (192); fp32 27 and
// 86 (1), 57 and 85 (64, two groups), 100 and 85 (128, four groups; 34 and 80 with 5000 classes).  20001 classes of 333 (256 rows,
// four groups): bf16 35 and 36, fp32 51 and 78.
inline void thin_plan(XentPlan &p, int dtype, long N, int D, int V) {
    const int s = (int)type_bytes(dtype), ks = dtype == kF32 ? 16 : 32;
    const long row = (ceil_to(D, ks) + 16 / s) * s, groups_most = dtype == kF32 || D % 8 ? 4 : 2;
    int t = N <= 16 ? 1 : N <= 32 ? 2 : 4;
    while (t > 1 && t * 16 * row > kThinLds) t /= 2;
    if (t * 16 * row > kThinLds || N > groups_most * t * 16) return;
    p.thin_tiles = t;
    p.thin_lds = (int)(t * 16 * (row + kThinWaves * 8 + 4));
    const long groups = (N + t * 16 - 1) / (t * 16), waves = ((long)V + 15) / 16;
    const long places = (p.thin_lds <= kThinLds / 2 ? 512 : 256) / groups;     // two blocks a CU, or one
    const long want = (waves + kThinWaves - 1) / kThinWaves;
    p.thin_blocks = (int)(want < places ? want : places);
}

// A piece of G.  Fewer pieces add to the features' gradient in fewer rounds: 256 MB, which the last-level cache
// holds, cost 1 .. 11 % more than 640 (16384 rows of 768 features, 50257 classes: 4.44 ms and 3.99).
constexpr size_t kPieceBytes = (size_t)640 << 20;

// Gradients of up to so many rows of a 16-bit type take each row twice, the second time with what the rounding of
// its G left.  Over more rows these roundings average out: 1.2 times the error of the results' own rounding.  Over
// one to four a row's gradient is its target's coefficient times a vector, and that one rounding made it up to 2.6
// times as far off.  All of them fit one tile of the products; a call takes 3 us more (8 rows of 1024 features,
// 32000 classes: 81 and 85; of 256 features, 1000 classes: 32 and 35).
constexpr long kPairedRows = 8;

inline XentPlan xent_plan(bool backward, int dtype, long N, int D, int V, bool aligned) {
    XentPlan p{};
    p.copies = backward && dtype != kF32 && N <= kPairedRows ? 2 : 1;
    p.R = N * p.copies;
    p.Np = ceil_to(p.R, 256);
    p.Dp = (int)ceil_to(D, 8);
    p.Dc = (int)ceil_to(D, 4);
    p.terms = dtype == kF32 ? 3 : 1;
    p.pack_w = D % (16 / (int)type_bytes(dtype)) || !aligned;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = up(at + bytes, 256); return o; };
    if (!backward) thin_plan(p, dtype, N, D, V);
    if (p.thin_tiles) {
        p.hit = take((size_t)N * 4);
        p.part = take((size_t)p.thin_blocks * N * 8);
        p.total = at;
        return p;
    }
    p.row_of = take((size_t)p.R * 4);
    p.target = take((size_t)p.Np * 4);                   // (the products read the rows' values a tile at a time)
    p.count = take(32);                                  // count, alpha, and from 16 on zeros
    p.scan_blocks = (int)((N + kScanRows - 1) / kScanRows);
    p.counts = take((size_t)p.scan_blocks * 4);
    p.tops = take((size_t)p.scan_blocks * 4);
    p.x = take((size_t)p.Np * p.Dp * type_bytes(dtype));
    p.w = take(p.pack_w ? (size_t)V * p.Dp * type_bytes(dtype) : 0);
    p.x3 = take(backward && dtype == kF32 ? (size_t)p.Np * 3 * p.Dp * 2 : 0);
    p.w3 = take(backward && dtype == kF32 ? (size_t)V * 3 * p.Dp * 2 : 0);
    if (!backward) {
        p.score = shape_of(N, V, D, p.terms, false, dtype == kF32);
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
        p.score = shape_of(p.R, widest, D, p.terms, false, dtype == kF32 || p.copies == 2);
        p.rows = shape_of(p.R, D, widest, p.terms, true);
        p.classes = shape_of(widest, D, p.R, p.terms, true);
        p.G = take((size_t)p.Np * p.terms * ceil_to(widest, 64) * 2);
        // the rows product splits by the tiles of rows that have a target: the fewer, the more parts, but never more
        // tiles in all than places, or than one part of all rows
        const long parts = places(p.rows) / p.rows.tiles_n;
        p.gx = take((size_t)(parts > p.rows.tiles_m ? parts : p.rows.tiles_m) * p.rows.bm * p.Dc * 4);
        p.gw = take(p.classes.splits > 1 ? (size_t)p.classes.splits * widest * p.Dc * 4 : 0);
    }
    p.total = at;
    return p;
}

template <class T, int END, int TERMS>
hipError_t product(GemmArgs &g, const Shape &sh, hipStream_t s) {
    g.tiles_m = sh.tiles_m; g.tiles_n = sh.tiles_n; g.splits = sh.splits;
    g.places = (int)places(sh); g.most = sh.most;
    const long tiles = (long)sh.tiles_m * sh.tiles_n * (END == kRows ? sh.most : sh.splits);
    const dim3 grid((unsigned)(tiles < g.places ? tiles : g.places));
    const auto launch = [&](auto kernel, int threads, int lds) {
        if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(kernel), lds); e != hipSuccess) return e;
        return run(kernel, grid, threads, lds, s, g);
    };
    if constexpr (END == kRows || END == kClasses)
        if (sh.bn == 192) return launch(xent_gemm_kernel<T, 4, 6, 4, 2, END, TERMS>, 512, xent_lds_bytes(256, 192, 2));
    if constexpr (sizeof(T) == 2)
        if (sh.bm == 256) return launch(xent_gemm_kernel<T, 4, 8, 4, 2, END, TERMS>, 512, xent_lds_bytes(256, 256, 2));
    return launch(xent_gemm_kernel<T, 4, 4, 2, 2, END, TERMS>, 256, xent_lds_bytes(128, 128, 2));
}

inline unsigned blocks_for(size_t chunks) {
    const size_t b = (chunks + kThreads - 1) / kThreads;
    return (unsigned)(b < 1 ? 1 : b < 8192 ? b : 8192);
}

// Whether every launch of a call takes its grid.
inline bool xent_launchable(const XentPlan &p, bool backward, long N, int D, int T) {
    if (p.thin_tiles) return true;                           // (a thousand rows at most)
    if (T && !grid_fits((double)(p.Np / 64) * ((D + 63) / 64), kThreads)) return false;
    const auto product = [&](const Shape &s) { return (double)s.tiles_m * s.tiles_n * s.most <= 0x7fffffff; };      // (counted by its blocks)
    if (!backward) return product(p.score) && grid_fits((double)(p.Np / 64), kLossThreads);
    if (T && !grid_fits((double)(N / T) * ((T + 63) / 64) * ((D + 63) / 64), kThreads)) return false;
    return product(p.score) && product(p.rows) && product(p.classes);
}

// S: the operands' type in memory and in the scores' product.  The gradients' take Grad, in so many terms.
template <class S> struct Cores { typedef S Grad; static constexpr int terms = 1; };
template <> struct Cores<float> { typedef __bf16 Grad; static constexpr int terms = 3; };

template <class S>
struct Xent {
    typedef typename Cores<S>::Grad Grad;
    static constexpr int kGradTerms = Cores<S>::terms, kHalves = sizeof(S) / 2;      // 16-bit values in an element
    const XentCall &c;
    const XentPlan p;
    char *ws;
    hipStream_t s;

    static bool aligned(const void *q) { return ((size_t)q & 15) == 0; }
    Xent(const XentCall &call, bool backward, void *w, hipStream_t st)
        : c(call), p(xent_plan(backward, call.dtype, call.N, call.D, call.V, aligned(call.wt))), ws(static_cast<char *>(w)), s(st) {}

    template <class P> P *at(size_t o) const { return reinterpret_cast<P *>(ws + o); }
    const void *zeros() const { return ws + p.count + 16; }

    hipError_t scan(ScanArgs &sc) {
        sc.tok = c.tok; sc.N = c.N; sc.blocks = p.scan_blocks; sc.copies = p.copies;
        sc.counts = at<int>(p.counts); sc.tops = at<float>(p.tops);
        sc.row_of = at<int>(p.row_of); sc.target = at<int>(p.target); sc.count = at<int>(p.count); sc.zeros = at<uint4>(p.count + 16);
        if (sc.blocks > kScanInline)
            if (hipError_t e = run(xent_count_kernel, dim3(sc.blocks), kThreads, 0, s, sc); e != hipSuccess) return e;
        return run(xent_place_kernel, dim3(sc.blocks), kThreads, 0, s, sc);
    }
    hipError_t pack(bool backward) {
        PackArgs<S> a{};
        a.from = static_cast<const S *>(c.x); a.row_of = at<int>(p.row_of); a.count = at<int>(p.count);
        a.rows = p.Np; a.D = c.D; a.ld = p.Dp; a.T_ = c.T;
        a.to = at<S>(p.x);
        PackArgs<S> b{};
        b.from = static_cast<const S *>(c.wt); b.rows = c.V; b.D = c.D; b.ld = p.Dp;
        if (p.pack_w) b.to = at<S>(p.w);
        if (kGradTerms == 3 && backward) { a.three = at<__bf16>(p.x3); b.three = at<__bf16>(p.w3); }
        const hipError_t e = c.T ? run(xent_pack_planes_kernel<S>, dim3((unsigned)(p.Np / 64 * ((c.D + 63) / 64))), kThreads, 0, s, a)
                                 : run(xent_pack_kernel<S>, dim3(blocks_for((size_t)p.Np * p.Dp / 8)), kThreads, 0, s, a);
        if (e != hipSuccess || (!b.to && !b.three)) return e;
        return run(xent_pack_kernel<S>, dim3(blocks_for((size_t)c.V * p.Dp / 8)), kThreads, 0, s, b);
    }
    // Features and weights (from class v0 on) as the scores' product reads them, and as the gradients' do.
    GemmSide features() const { return GemmSide{at<S>(p.x), (long)kHalves * p.Dp, 0, p.Np, kHalves * p.Dp}; }
    GemmSide weights(long v0) const {
        const S *const w = p.pack_w ? at<S>(p.w) : static_cast<const S *>(c.wt);
        const int ld = p.pack_w ? p.Dp : c.D;
        return GemmSide{w + v0 * ld, (long)kHalves * ld, 0, c.V - v0, kHalves * ld};
    }
    GemmSide grad_features() const { return kGradTerms == 1 ? features() : GemmSide{at<Grad>(p.x3), 3L * p.Dp, p.Dp, p.Np, p.Dp}; }
    GemmSide grad_weights(long v0) const {
        return kGradTerms == 1 ? weights(v0) : GemmSide{at<Grad>(p.w3) + v0 * 3 * p.Dp, 3L * p.Dp, p.Dp, c.V - v0, p.Dp};
    }

    template <int NT>
    hipError_t thin_tiles(const ThinArgs<S> &a) {
        auto k = xent_thin_kernel<S, NT>;
        if (hipError_t e = allow_big_lds(reinterpret_cast<const void *>(k), p.thin_lds); e != hipSuccess) return e;
        const dim3 grid(p.thin_blocks, (unsigned)((c.N + NT * 16 - 1) / (NT * 16)));
        if (hipError_t e = run(k, grid, kThinThreads, p.thin_lds, s, a); e != hipSuccess) return e;
        return run(xent_thin_loss_kernel<S>, dim3((unsigned)c.N), kThreads, 0, s, a);
    }
    hipError_t thin() {
        const ThinArgs<S> a{static_cast<const S *>(c.x), static_cast<const S *>(c.wt), c.tok, c.N, c.D, c.V, c.T, p.thin_blocks,
                            at<float2>(p.part), at<float>(p.hit), c.loss, c.lse};
        return p.thin_tiles == 1 ? thin_tiles<1>(a) : p.thin_tiles == 2 ? thin_tiles<2>(a) : thin_tiles<4>(a);
    }
    hipError_t fprop() {
        if (p.thin_tiles) return thin();
        ScanArgs sc{};
        sc.loss = c.loss; sc.lse = c.lse;
        if (hipError_t e = scan(sc); e != hipSuccess) return e;
        if (hipError_t e = pack(false); e != hipSuccess) return e;
        GemmArgs g{};
        g.P = features(); g.Q = weights(0);
        g.count = sc.count; g.zeros = zeros();
        g.M = (int)p.Np; g.N = c.V; g.K = kHalves * c.D;
        g.target = sc.target; g.part = at<float2>(p.part); g.part_ld = p.Np; g.hit = at<float>(p.hit);
        if (hipError_t e = product<S, kStats, 1>(g, p.score, s); e != hipSuccess) return e;
        const LossArgs l{g.part, p.Np, p.score.tiles_n, g.hit, sc.row_of, sc.count, c.loss, c.lse};
        return run(xent_loss_kernel, dim3((unsigned)(p.Np / 64)), kLossThreads, 0, s, l);
    }

    hipError_t backward() {
        ScanArgs sc{};
        sc.pos = at<int>(p.pos);
        sc.lse_in = c.lse; sc.gloss = c.gloss;
        sc.lse_out = at<float>(p.lse); sc.coef = at<float>(p.coef);
        sc.alpha = at<float>(p.count + 4);
        sc.scale = c.scale; sc.mean = c.mean; sc.half_range = c.dtype == kF16;
        if (hipError_t e = scan(sc); e != hipSuccess) return e;
        if (hipError_t e = pack(true); e != hipSuccess) return e;
        for (int i = 0; i < p.pieces; ++i) {
            const long v0 = (long)i * p.piece;
            const int width = (int)(c.V - v0 < p.piece ? c.V - v0 : p.piece);
            const long ld = ceil_to(width, 64);
            const GemmSide G{at<Grad>(p.G), p.terms * ld, ld, p.Np, (int)ld};
            GemmArgs g{};
            g.P = features(); g.Q = weights(v0);
            g.count = sc.count; g.zeros = zeros();
            g.M = (int)p.Np; g.N = width; g.K = kHalves * c.D;
            g.target = sc.target; g.lse = sc.lse_out; g.coef = sc.coef;
            g.n0 = (int)v0;
            g.G = at<Grad>(p.G); g.g_ld = ld; g.g_term = ld; g.twice = p.copies == 2;
            if (hipError_t e = product<S, kGrad, 1>(g, tiles(p.score, p.R, width), s); e != hipSuccess) return e;
            if (c.gx) {
                GemmArgs r{};
                r.P = G; r.Q = grad_weights(v0);
                r.count = sc.count; r.zeros = zeros();
                r.M = (int)p.Np; r.N = c.D; r.K = width;
                r.partial = at<float>(p.gx); r.part_cols = p.Dc; r.add = i > 0;
                r.alpha_scale = sc.alpha;
                if (hipError_t e = product<Grad, kRows, kGradTerms>(r, p.rows, s); e != hipSuccess) return e;
            }
            if (c.gw) {
                GemmArgs w{};
                w.P = G; w.Q = grad_features();
                w.count = sc.count; w.zeros = zeros();
                w.M = width; w.N = c.D; w.K = (int)p.R;
                w.alpha_scale = sc.alpha;
                S *gw = static_cast<S *>(c.gw) + v0 * c.D;
                const Shape sh = tiles(p.classes, width, c.D);
                if (sh.splits > 1) { w.partial = at<float>(p.gw); w.part_cols = p.Dc; }
                else { w.out = gw; w.out_ld = c.D; w.add = c.accumulate; }
                if (hipError_t e = product<Grad, kClasses, kGradTerms>(w, sh, s); e != hipSuccess) return e;
                if (sh.splits > 1) {
                    const ClassesOutArgs<S> o{at<float>(p.gw), sc.alpha, gw, width, p.Dc, sh.splits, c.D, c.accumulate};
                    const dim3 grid(blocks_for((size_t)width * ((c.D + 7) / 8)));
                    if (hipError_t e = run(xent_classes_out_kernel<S>, grid, kThreads, 0, s, o); e != hipSuccess) return e;
                }
            }
        }
        if (!c.gx) return hipSuccess;
        const RowsOutArgs<S> o{at<float>(p.gx), sc.pos, sc.count, sc.alpha, static_cast<S *>(c.gx), c.N, p.Dc,
                               p.rows.bm, p.rows.tiles_n, (int)places(p.rows), p.rows.most, c.D, c.T, p.copies};
        if (c.T) {
            const long blocks = c.N / c.T * ((c.T + 63) / 64) * ((c.D + 63) / 64);
            return run(xent_planes_out_kernel<S>, dim3((unsigned)blocks), kThreads, 0, s, o);
        }
        const size_t pieces = (size_t)c.N * ((c.D + 7) / 8);
        if (p.rows.splits > 8) return run(xent_rows_out_kernel<S, 8>, dim3(blocks_for(pieces * 8)), kThreads, 0, s, o);
        return run(xent_rows_out_kernel<S, 1>, dim3(blocks_for(pieces)), kThreads, 0, s, o);
    }
    // The last piece may be narrower than the plan's.
    static Shape tiles(Shape sh, long M, long N) {
        sh.tiles_m = (int)((M + sh.bm - 1) / sh.bm);
        sh.tiles_n = (int)((N + sh.bn - 1) / sh.bn);
        return sh;
    }
};

}  // namespace
}  // namespace fc
