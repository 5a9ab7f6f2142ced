// The matrix products of the linear cross entropy, as one kernel with four ends:
//
//   C[m, n] = sum over k of P(m, k) Q(n, k)
//
//   stats   P = features [rows, D],  Q = weights [V, D]: the scores of a tile of rows and classes; only
//           their maximum and the sum of their exponentials leave the tile, by row
//   grad    the same product again, and from it G[row, class] = (softmax - target) * coef[row]
//   rows    P = G,            Q = weights (K = classes): the features' gradient, in fp32
//   classes P = G (K = rows), Q = features:              the weights' gradient
//
// Every operand is a row-major array of 16-bit values.  Where the reduction runs along its rows ("K
// inside") a tile is staged as 64 k of each of its rows; where it runs across them ("K outside") as
// 64 whole rows, and the transposing LDS reads turn them on their way to the matrix cores.  So G is
// written once and nothing is transposed in memory.
//
// fp32 operands are three bf16 terms each (their cut is exact, see split2), side by side in the row: the
// K loop walks six products of terms per 64 k, the small ones first.  What is left out is below 2^-24 of
// the product of the two.
//
// A tile is staged with direct global-to-LDS loads of 16 bytes a lane, one K step ahead, in two
// buffers.  LDS is written in lane order, so the swizzle that spreads a column of 16-byte pieces over
// the banks is applied to the addresses that are read: piece c of row r holds what belongs to
// c ^ (r & 7) (K inside), or c ^ 2 (r & 3) (K outside).
#pragma once
#include "operands.hpp"
#include "kernels.hpp"
#include "bf16_split.hpp"
#include <type_traits>

#pragma clang diagnostic ignored "-Winline-asm"     // m0 as a clobber: nothing else here keeps a value in it

namespace fc {

enum { kStats = 0, kGrad = 1, kRows = 2, kClasses = 3 };
constexpr int kStep = 64;            // k per step

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

// A row-major operand.  Rows beyond `rows` and columns beyond `cols` (a multiple of 8) are never read: K
// inside, columns beyond read as zero; elsewhere their place is taken by what lies before them, and the
// results that come of it are not kept.
struct GemmSide {
    const void *p;
    long ld;             // elements from row to row
    long term;           // elements from one term of an fp32 value to the next
    long rows;
    int cols;
};

struct GemmArgs {
    GemmSide P, Q;
    const int *count;        // rows that have a target; limits M (stats, grad, rows) or K (classes)
    const void *zeros;       // 16 bytes
    int M, N, K;             // what the grid covers
    int tiles_m, tiles_n, splits;
    // stats, grad
    const int *target;       // by row
    float2 *part;            // [tiles_n][part_ld]: maximum and sum of a row's scores in a tile
    float *hit;              // the target's score, by row
    const float *lse, *coef; // by row
    int n0;                  // class of column 0
    void *G;
    long g_ld, g_term;
    long part_ld;
    // rows, classes
    float *partial;          // [splits][M][part_cols], or null: straight to `out`
    long part_cols;
    int add;                 // add to what `partial` or `out` holds
    void *out;
    long out_ld;
    const float *alpha_scale;    // factor on the device
    float alpha;
};

__device__ __forceinline__ void lds_load16(const char *from, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void landed_and_met() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <class T> struct Mfma;
template <> struct Mfma<__bf16> {
    typedef bf16x8 frag;
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<_Float16> {
    typedef f16x8 frag;
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// One operand's tile: R rows of the result's side by 64 k, R * 128 bytes, moved by W waves.
template <int R, int W, bool KIN>
struct Tile {
    static constexpr int kLoads = R * 128 / 1024 / W;        // 1 KB a wave
    static constexpr int kPieces = R / 8;                    // 16-byte pieces in a row of 64 (K outside)
    const char *at[kLoads];                                  // K inside: the lane's place in step 0
    int col[kLoads];                                         // K inside: its column there; K outside: its k
    long across;                                             // K outside: its byte column

    // first: the tile's first row of the result's side.  KIN: rows of memory, else columns.
    __device__ __forceinline__ void begin(const GemmSide &g, long first, int w, int lane) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = (i * W + w) * 64 + lane;       // of 16 bytes, in LDS order
            if (KIN) {
                const int r = piece >> 3, c = (piece & 7) ^ (r & 7);
                long row = first + r;
                if (row >= g.rows) row = g.rows - 1;
                col[i] = c * 8;
                at[i] = static_cast<const char *>(g.p) + (row * g.ld + c * 8) * 2;
            } else {
                const int k = piece / kPieces, c = (piece % kPieces) ^ (2 * (k & 3));
                col[i] = k;
                long x = first + c * 8;
                if (x >= g.cols) x = 0;
                at[i] = static_cast<const char *>(g.p) + x * 2;
            }
        }
    }
    __device__ __forceinline__ void load(const GemmSide &g, const void *zeros, int k0, int term, unsigned lds, int w) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const char *from;
            if (KIN) {
                from = at[i] + ((long)k0 + term * g.term) * 2;
                if (col[i] + k0 >= g.cols) from = static_cast<const char *>(zeros);
            } else {
                long row = (long)k0 + col[i];
                if (row >= g.rows) row = g.rows - 1;
                from = at[i] + (row * g.ld + term * g.term) * 2;
            }
            lds_load16(from, lds + (i * W + w) * 1024);
        }
    }
    // The 16 rows from r0 on, 32 k from 32 ks on, as the matrix cores take them: lane l holds row
    // l & 15 and the eight k from 8 (l >> 4) on.
    template <class F>
    static __device__ __forceinline__ F frag(const char *lds, int r0, int ks, int lane) {
        if (KIN) {
            const int r = r0 + (lane & 15), c = ks * 4 + (lane >> 4);
            return *reinterpret_cast<const F *>(lds + r * 128 + ((c ^ (r & 7)) << 4));
        } else {
            const int i = lane & 15;
            union { short4v half[2]; F f; } u;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = ks * 32 + (lane >> 4) * 8 + h * 4 + (i >> 2);
                const int c = ((r0 >> 3) + ((i & 3) >> 1)) ^ (2 * (k & 3));
                const char *p = lds + k * (R * 2) + c * 16 + (i & 1) * 8;
                u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)(p));
            }
            return u.f;
        }
    }
};

// Tile of FM*WM*16 rows (m) by FN*WN*16 columns (n); a wave has FM*16 by FN*16 of it.
template <class T, int FM, int FN, int WM, int WN, int END, bool SPLIT>
__global__ __launch_bounds__(WM *WN * 64) void xent_gemm_kernel(GemmArgs a) {
    constexpr int BM = FM * WM * 16, BN = FN * WN * 16, W = WM * WN;
    constexpr bool PIN = END != kClasses, QIN = END == kStats || END == kGrad;
    typedef typename Mfma<T>::frag F;
    extern __shared__ __align__(1024) char lds[];
    constexpr int kBytes = (BM + BN) * 128;

    const int count = *a.count;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / WN, wn = w % WN;

    // Neighbouring blocks go to different XCDs: each XCD takes a contiguous eighth of the tiles, walked
    // in columns of four tiles so that what its L2 holds is used several times.
    const int total = a.tiles_m * a.tiles_n;
    const int split = blockIdx.x / total;
    int id = blockIdx.x - split * total;
    {
        const int per = total / 8, more = total % 8, x = id % 8;
        id = x * per + (x < more ? x : more) + id / 8;
    }
    constexpr int GN = 4;
    const int group = id / (GN * a.tiles_m), in = id - group * GN * a.tiles_m;
    const int gn = a.tiles_n - group * GN < GN ? a.tiles_n - group * GN : GN;
    const int tm = in / gn, tn = group * GN + in % gn;
    const long m0 = (long)tm * BM, n0 = (long)tn * BN;
    if (END != kClasses && m0 >= count) return;

    const int K = END == kClasses ? count : a.K;
    int steps = (K + kStep - 1) / kStep, begin = 0;
    if (a.splits > 1) {
        const int each = (steps + a.splits - 1) / a.splits;
        begin = split * each;
        steps = steps < begin + each ? steps : begin + each;
    }

    Tile<BM, W, PIN> tp;
    Tile<BN, W, QIN> tq;
    tp.begin(a.P, m0, w, lane);
    tq.begin(a.Q, n0, w, lane);
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char *)lds;

    constexpr int kTerms = SPLIT ? 6 : 1;
    floatx4 acc[FM][FN] = {};
    const int first = begin * kTerms, last = steps * kTerms;
    auto stage = [&](int s) {
        const int k0 = (SPLIT ? s / 6 : s) * kStep;
        int tp_ = 0, tq_ = 0;                                // terms: l h, h l, m m, m h, h m, h h
        if (SPLIT) {
            const int t = s % 6;
            tp_ = t == 0 ? 2 : t == 2 || t == 3 ? 1 : 0;
            tq_ = t == 1 ? 2 : t == 2 || t == 4 ? 1 : 0;
        }
        const unsigned to = lds0 + (s & 1) * kBytes;
        tp.load(a.P, a.zeros, k0, tp_, to, w);
        tq.load(a.Q, a.zeros, k0, tq_, to + BM * 128, w);
    };
    if (first < last) stage(first);
    for (int s = first; s < last; ++s) {
        landed_and_met();
        if (s + 1 < last) stage(s + 1);
        const char *p = lds + (s & 1) * kBytes, *q = p + BM * 128;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            F fp[FM], fq[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) fq[j] = Tile<BN, W, QIN>::template frag<F>(q, (wn * FN + j) * 16, ks, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i) fp[i] = Tile<BM, W, PIN>::template frag<F>(p, (wm * FM + i) * 16, ks, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<T>::mul(fq[j], fp[i], acc[i][j]);
        }
    }

    // A lane holds, of each 16x16 tile, row lane & 15 and the four columns from 4 (lane >> 4) on.
    const int row = lane & 15, quad = (lane >> 4) * 4;
    if constexpr (END == kStats) {
        landed_and_met();                                     // (the tiles in LDS are done with)
        float2 *both = reinterpret_cast<float2 *>(lds);      // [WN][BM]
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const long m = m0 + (wm * FM + i) * 16 + row;
            const int t = m < count ? a.target[m] : -1;
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const long n = n0 + (wn * FN + j) * 16 + quad + r;
                    if (n >= a.N) acc[i][j][r] = -INFINITY;
                    else if (n == t) a.hit[m] = acc[i][j][r];
                    top = fmaxf(top, acc[i][j][r]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.f : top;  // (nothing but -inf: the sum is 0)
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __expf(acc[i][j][r] - base);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (lane < 16) both[wn * BM + (wm * FM + i) * 16 + row] = make_float2(top, sum);
        }
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += W * 64) {
            float2 v = both[r];
#pragma unroll
            for (int q = 1; q < WN; ++q) {
                const float2 o = both[q * BM + r];
                const float top = fmaxf(v.x, o.x), base = top == -INFINITY ? 0.f : top;
                v = make_float2(top, v.y * __expf(v.x - base) + o.y * __expf(o.x - base));
            }
            if (m0 + r < count) a.part[tn * a.part_ld + m0 + r] = v;
        }
    } else if constexpr (END == kGrad) {
        T *G = static_cast<T *>(a.G);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const long m = m0 + (wm * FM + i) * 16 + row;
            const bool live = m < count;
            const int t = live ? a.target[m] - a.n0 : -1;
            const float lse = live ? a.lse[m] : 0.f, coef = live ? a.coef[m] : 0.f;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const long n = n0 + (wn * FN + j) * 16 + quad;
                if (n >= a.g_ld) continue;
                float g[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __expf(acc[i][j][r] - lse);
                    g[r] = live && n + r < a.N ? (p - (n + r == t ? 1.f : 0.f)) * coef : 0.f;
                }
                if (m >= a.M) continue;
                T *to = G + m * (SPLIT ? 3 * a.g_term : a.g_ld) + n;
                if constexpr (SPLIT) {
                    uint2 h, l1, l2;
                    split4(g[0], g[1], g[2], g[3], h, l1, l2);
                    *reinterpret_cast<uint2 *>(to) = h;
                    *reinterpret_cast<uint2 *>(to + a.g_term) = l1;
                    *reinterpret_cast<uint2 *>(to + 2 * a.g_term) = l2;
                } else {
                    T v[4] = {(T)g[0], (T)g[1], (T)g[2], (T)g[3]};
                    __builtin_memcpy(__builtin_assume_aligned(to, 8), v, 8);
                }
            }
        }
    } else {
        const float alpha = a.partial ? 1.f : a.alpha * *a.alpha_scale;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const long m = m0 + (wm * FM + i) * 16 + row;
            if (m >= a.M || (END == kRows && m >= count)) continue;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const long n = n0 + (wn * FN + j) * 16 + quad;
                if (n >= a.N) continue;
                floatx4 v = acc[i][j];
                if (a.partial) {
                    floatx4 *to = reinterpret_cast<floatx4 *>(a.partial + ((size_t)split * a.M + m) * a.part_cols + n);
                    *to = a.add ? *to + v : v;               // (part_cols is a multiple of four)
                } else {
                    const int left = (int)(a.N - n);
                    auto put = [&](auto *out) {
                        typedef typename std::remove_pointer<decltype(out)>::type O;
                        out += m * a.out_ld + n;
                        float f[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) f[r] = v[r] * alpha;
                        if (a.add)
#pragma unroll
                            for (int r = 0; r < 4; ++r) if (r < left) f[r] += to_float(out[r]);
                        O t[4] = {(O)f[0], (O)f[1], (O)f[2], (O)f[3]};
                        if (left >= 4) __builtin_memcpy(out, t, sizeof(t));
                        else
#pragma unroll
                            for (int r = 0; r < 4; ++r) if (r < left) out[r] = t[r];
                    };
                    if constexpr (SPLIT) put(static_cast<float *>(a.out));
                    else put(static_cast<T *>(a.out));
                }
            }
        }
    }
}

}  // namespace fc
