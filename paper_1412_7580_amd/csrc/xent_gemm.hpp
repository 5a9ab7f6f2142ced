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
// fp32 operands:
//
//  - The scores are multiplied in fp32 (16x16x4): what a mask puts into a weight (-1e9, the type's lowest value, an
//    infinity) leaves the other features of its class as they are, which terms of fewer bits do not.  The
//    tiles are staged as rows of twice as many 16-bit values.  (4096 rows of 1024 features, 32000 classes: 135 TFLOP/s
//    with all of the call; a library product 153.)
//  - The gradients' products take three bf16 terms side by side in the row, whose cut is exact (see split2); the K
//    loop walks six products of terms per 64 k.  What is left out is below 2^-24 of the product of the two.
//
// A tile is staged with direct global-to-LDS loads of 16 bytes a lane, one K step ahead, in two
// buffers.  LDS is written in lane order, so the swizzle that spreads a column of 16-byte pieces over
// the banks is applied to the addresses that are read: piece c of row r holds what belongs to
// c ^ (r & 7) (K inside), or c ^ (2 (r & 3) | (r & 8)) (K outside, whole 256 bytes a row).
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
    long term;           // elements from one of three terms to the next
    long rows;
    int cols;
};

struct GemmArgs {
    GemmSide P, Q;
    const int *count;        // rows that have a target; limits M (stats, grad, rows) or K (classes)
    const void *zeros;       // 16 bytes
    int M, N, K;             // what the grid covers
    int tiles_m, tiles_n, splits;
    int places, most;        // rows: blocks the chip holds, steps-bound of the splits; they follow from the live rows
    // stats, grad
    const int *target;       // by row
    float2 *part;            // [tiles_n][part_ld]: maximum and sum of a row's scores in a tile
    float *hit;              // the target's score, by row
    const float *lse, *coef; // by row
    int n0;                  // class of column 0
    void *G;                 // (from fp32 operands: in three terms)
    int twice;               // (small tiles) rows come in pairs: an odd one holds what the rounding of the even one's G left
    long g_ld, g_term;
    long part_ld;
    // rows, classes
    float *partial;          // [splits][M, or the rows of live tiles][part_cols], or null: straight to `out`
    long part_cols;
    int add;                 // add to what `partial` or `out` holds
    void *out;
    long out_ld;
    const float *alpha_scale;    // factor of `out`, on the device
};

// Into how many parts the rows product's reduction is split: until there is a block for every place.
__host__ __device__ inline int rows_splits(long tiles, int places, int most) {
    const long s = places / (tiles < 1 ? 1 : tiles);
    return (int)(s < 1 ? 1 : s > most ? most : s);
}

// Loads from memory to LDS, in lane order from m0 on.  As assembly, so that an LDS read waits for the step that it
// needs (landed_and_met) and not for all that is on its way; no register is written.
__device__ __forceinline__ void lds_load16(const char *from, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ const char *uniform(const char *p) {
    const unsigned long u = (unsigned long)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)u), hi = __builtin_amdgcn_readfirstlane((unsigned)(u >> 32));
    return (const char *)((unsigned long)hi << 32 | lo);
}
__device__ __forceinline__ void lds_load16(const char *base, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(const void *base, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_written_and_met() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// Every wave's staging loads but its last N have landed, its LDS reads are done, and all waves are here.
template <int N>
__device__ __forceinline__ void landed_and_met() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// What a lane and its partners 16 and 32 lanes on hold, by vector moves (the four sixteens' largest, or their sum).
__device__ __forceinline__ float2 both16(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return make_float2(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float2 both32(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return make_float2(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float sixteens_max(float x) {
    const float2 a = both16(x);
    const float2 b = both32(fmaxf(a.x, a.y));
    return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float sixteens_sum(float x) {
    const float2 a = both16(x);
    const float2 b = both32(a.x + a.y);
    return b.x + b.y;
}

// What exponentials are taken less of.  Where the largest score is infinite, nothing: sums of nothing but -inf are 0, those with +inf
// infinite, and so is their logarithm.
__device__ __forceinline__ float base_of(float top) { return fabsf(top) < INFINITY ? top : 0.f; }

// parts: matrix instructions for what 16 bytes a lane hold of the reduction.
template <class T> struct Mfma;
template <> struct Mfma<float> {
    typedef floatx4 frag;
    static constexpr int parts = 4;
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c, int part) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a[part], b[part], c, 0, 0, 0); }
};
template <> struct Mfma<__bf16> {
    typedef bf16x8 frag;
    static constexpr int parts = 1;
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c, int = 0) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<_Float16> {
    typedef f16x8 frag;
    static constexpr int parts = 1;
    static __device__ __forceinline__ floatx4 mul(frag a, frag b, floatx4 c, int = 0) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// One operand's tile: R rows of the result's side by 64 k, R * 128 bytes, moved by W waves.
template <int R, int W, bool KIN>
struct Tile {
    static constexpr int kLoads = R * 128 / 1024 / W;        // 1 KB a wave
    static constexpr int kPieces = R / 8;                    // 16-byte pieces in a row of 64 (K outside)
    const char *base;                                        // first row of the result's side, k = 0
    unsigned off[kLoads];                                    // the lane's bytes from there

    // (rows of 384 bytes already alternate between the halves of the banks)
    static __device__ __forceinline__ int swizzle(int k) { return kPieces % 16 == 0 ? 2 * (k & 3) | (k & 8) : (k & 2) | (k & 8) >> 1; }
    // Row (K inside) or k (K outside) and column of the lane's piece i.
    static __device__ __forceinline__ void place(int i, int w, int lane, int &r, int &c) {
        const int piece = (i * W + w) * 64 + lane;           // of 16 bytes, in LDS order
        if (KIN) { r = piece >> 3; c = ((piece & 7) ^ (r & 7)) * 8; }
        else { r = piece / kPieces; c = ((piece % kPieces) ^ swizzle(r)) * 8; }
    }
    // first: the tile's first row of the result's side.  KIN: rows of memory, else columns.
    __device__ __forceinline__ void begin(const GemmSide &g, long first, int w, int lane) {
        base = static_cast<const char *>(g.p) + (KIN ? first * g.ld : first) * 2;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int r, c;
            place(i, w, lane, r, c);
            if (KIN) { if (first + r >= g.rows) r = (int)(g.rows - 1 - first); }
            else if (first + c >= g.cols) c = 0;
            off[i] = (unsigned)(((long)r * g.ld + c) * 2);
        }
    }
    __device__ __forceinline__ void load(const GemmSide &g, const void *zeros, int k0, int term, unsigned lds, int w, int lane) const {
        const char *from = uniform(base + (KIN ? k0 : k0 * g.ld) * 2 + term * g.term * 2);
        if (k0 + kStep <= (KIN ? (long)g.cols : g.rows)) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) lds_load16(from, off[i], lds + (i * W + w) * 1024);
        } else {
            asm volatile("" : "+v"(lane));                   // (what follows from it is formed here, not kept in registers)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int r, c;
                place(i, w, lane, r, c);
                const char *at = from + off[i];
                if (KIN) { if (k0 + c >= g.cols) at = static_cast<const char *>(zeros); }
                else if (k0 + r >= g.rows) at += (g.rows - 1 - k0 - r) * g.ld * 2;
                lds_load16(at, lds + (i * W + w) * 1024);
            }
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
                const int c = ((r0 >> 3) + ((i & 3) >> 1)) ^ swizzle(k);
                const char *p = lds + k * (R * 2) + c * 16 + (i & 1) * 8;
                u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)(p));
            }
            return u.f;
        }
    }
};

constexpr int xent_lds_bytes(int bm, int bn, int wn) { return 2 * (bm + bn) * 128 + 2 * 3 * bm * 4 + wn * bm * 8; }

// Tiles of FM*WM*16 rows (m) by FN*WN*16 columns (n); a wave has FM*16 by FN*16 of one.  256x256 tiles of eight
// waves: 128 of a wave's 256 registers are sums, two half steps of fragments 96.  (Four waves of 128x128 spill;
// two blocks a CU of 128x256 tiles in steps of 32 k hide each other's ends but stage half as much again: 7.9 ms
// instead of 6.97 for the step of 8192 rows; 32x32 matrix instructions 8 % slower, and wave priorities 5 %.)  A block takes
// tiles until there are none left: the next one's first two steps are on their way while the
// last one's end is computed.
template <class T, int FM, int FN, int WM, int WN, int END, int TERMS>
__global__ __launch_bounds__(WM *WN * 64) void xent_gemm_kernel(GemmArgs a) {
    constexpr int BM = FM * WM * 16, BN = FN * WN * 16, W = WM * WN;
    constexpr bool PIN = END != kClasses, QIN = END == kStats || END == kGrad;
    constexpr bool SCORES = END == kStats || END == kGrad;
    constexpr int kProducts = TERMS == 3 ? 6 : 1;
    typedef typename Mfma<T>::frag F;
    typedef Tile<BM, W, PIN> TP;
    typedef Tile<BN, W, QIN> TQ;
    extern __shared__ __align__(1024) char lds[];
    constexpr int kBytes = (BM + BN) * 128;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char *)lds;
    constexpr int kValues = 3 * BM;                                           // of a tile's rows: target, lse, coef
    char *const values = lds + 2 * kBytes;                                    // [2][kValues]
    float2 *const both = reinterpret_cast<float2 *>(values + 2 * kValues * 4);    // [WN][BM]

    const int count = *a.count;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / WN, wn = w % WN;
    const int live_m = (count + BM - 1) / BM;
    const int tiles_m = END == kClasses || a.tiles_m < live_m ? a.tiles_m : live_m;
    const int total = tiles_m * a.tiles_n;
    const int splits = END == kRows ? rows_splits(total, a.places, a.most) : a.splits, units = total * splits;
    const int K = END == kClasses ? count : a.K, steps = (K + kStep - 1) / kStep;
    TP tp;
    TQ tq;
    long m0, n0;
    int tn, split, first, last;
    // Neighbouring blocks go to different XCDs: each XCD takes a contiguous eighth of the tiles (all of a
    // split's before the next one's), walked in columns of four tiles so that what its L2 holds is used
    // several times.
    auto place = [&](int u) {
        const int per = units / 8, more = units % 8, x = u % 8;
        int id = x * per + (x < more ? x : more) + u / 8;
        split = id / total;
        id -= split * total;
        constexpr int GN = 4;
        const int group = id / (GN * tiles_m), in = id - group * GN * tiles_m;
        const int gn = a.tiles_n - group * GN < GN ? a.tiles_n - group * GN : GN;
        tn = group * GN + in % gn;
        m0 = (long)(in / gn) * BM;
        n0 = (long)tn * BN;
        const int each = (steps + splits - 1) / splits, begin = split * each;
        first = begin * kProducts;
        last = (steps < begin + each ? steps : begin + each) * kProducts;
        tp.begin(a.P, m0, w, lane);
        tq.begin(a.Q, n0, w, lane);
    };
    auto stage = [&](int s) {
        const int t = s % kProducts, k0 = s / kProducts * kStep;
        int tp_ = 0, tq_ = 0;
        if (TERMS == 3) {                                    // l h, h l, m m, m h, h m, h h
            tp_ = t == 0 ? 2 : t == 2 || t == 3 ? 1 : 0;
            tq_ = t == 1 ? 2 : t == 2 || t == 4 ? 1 : 0;
        }
        const unsigned to = lds0 + (s & 1) * kBytes;
        tp.load(a.P, a.zeros, k0, tp_, to, w, lane);
        tq.load(a.Q, a.zeros, k0, tq_, to + BM * 128, w, lane);
    };
    // The first two steps, and before them the values that the tile's rows bring along.
    auto stage_first = [&](int parity) {
        if constexpr (SCORES) {
            const auto fetch = [&](const void *from, int n, int to) {         // n values, 64 a wave and load
                for (int i = w; i < n / 64; i += W)
                    lds_load4(uniform(static_cast<const char *>(from)), (i * 64 + lane) * 4, lds0 + 2 * kBytes + (parity * kValues + to + i * 64) * 4);
            };
            fetch(a.target + m0, BM, 0);
            if (END == kGrad) {
                fetch(a.lse + m0, BM, BM);
                fetch(a.coef + m0, BM, 2 * BM);
            }
        }
        if (first < last) stage(first);
        if (first + 1 < last) stage(first + 1);
    };
    struct Frags { F p[FM], q[FN]; };
    floatx4 acc[FM][FN];
    auto read = [&](Frags &f, int s, int ks) {
        const char *p = lds + (s & 1) * kBytes, *q = p + BM * 128;
#pragma unroll
        for (int j = 0; j < FN; ++j) f.q[j] = TQ::template frag<F>(q, (wn * FN + j) * 16, ks, lane);
#pragma unroll
        for (int i = 0; i < FM; ++i) f.p[i] = TP::template frag<F>(p, (wm * FM + i) * 16, ks, lane);
    };
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int part = 0; part < Mfma<T>::parts; ++part)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<T>::mul(f.q[j], f.p[i], acc[i][j], part);
    };
    // Reads of one half step between the matrix instructions of the other.
    auto interleave = [&]() {
        constexpr int reads = FM * (PIN ? 1 : 2) + FN * (QIN ? 1 : 2), all = FM * FN * Mfma<T>::parts, each = all / reads;
#pragma unroll
        for (int r = 0; r < reads; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, each, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, all - reads * each, 0);
    };

    int u = blockIdx.x, parity = 0;
    if (u >= units) return;
    place(u);
    stage_first(0);
    for (;;) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        // A step's second half is read while its first is multiplied; then the next step has landed, this
        // one's buffer is free for the step after it, and the next step's first half is read while
        // the second half is multiplied.
        if (first < last) {
            Frags even, odd;
            if (first + 1 < last) landed_and_met<TP::kLoads + TQ::kLoads>();
            else landed_and_met<0>();
            read(even, first, 0);
            for (int s = first; s + 1 < last; ++s) {
                read(odd, s, 1);
                multiply(even);
                interleave();
                landed_and_met<0>();
                if (s + 2 < last) stage(s + 2);
                read(even, s + 1, 0);
                multiply(odd);
                interleave();
            }
            read(odd, last - 1, 1);
            multiply(even);
            multiply(odd);
        }

        const long m_at = m0, n_at = n0;
        const int tn_at = tn, split_at = split;
        landed_and_met<0>();                                 // (the row values too, where there was no step)
        u += gridDim.x;
        const bool more = u < units;
        if (more) {
            place(u);
            stage_first(parity ^ 1);
        }

        // A lane holds, of each 16x16 tile, row lane & 15 and the four columns from 4 (lane >> 4) on.  (The ends are
        // vector work, 6 us of a tile's 35 at 1024 features, half of it exponentials.)
        int own = lane;
        asm volatile("" : "+v"(own));
        const int row = own & 15, quad = (own >> 4) * 4;
        const int *targets = reinterpret_cast<const int *>(values + parity * kValues * 4);
        const float *lses = reinterpret_cast<const float *>(targets) + BM, *coefs = lses + BM;
        if constexpr (END == kStats) {
            const bool edge = n_at + BN > a.N;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int lm = (wm * FM + i) * 16 + row;
                const long m = m_at + lm;
                const int rel = targets[lm] - (int)n_at - wn * FN * 16 - quad;
                const bool hit = m < count && rel >= 0 && rel < FN * 16 && (rel & 12) == 0;
                if (__any(hit)) {
                    float z = 0.f;
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) z = rel == j * 16 + r ? acc[i][j][r] : z;
                    if (hit) a.hit[m] = z;
                }
                if (edge) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n_at + (wn * FN + j) * 16 + quad + r >= a.N) acc[i][j][r] = -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < FN; ++j) top = fmaxf(fmaxf(fmaxf(top, acc[i][j][0]), acc[i][j][1]), fmaxf(acc[i][j][2], acc[i][j][3]));
                top = sixteens_max(top);
                const float base = base_of(top);
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum += __expf(acc[i][j][r] - base);
                sum = sixteens_sum(sum);
                if (lane < 16) both[wn * BM + lm] = make_float2(top, sum);
            }
            lds_written_and_met();
            for (int r = threadIdx.x; r < BM; r += W * 64) {
                float2 v = both[r];
#pragma unroll
                for (int q = 1; q < WN; ++q) {
                    const float2 o = both[q * BM + r];
                    const float top = fmaxf(v.x, o.x), base = base_of(top);
                    v = make_float2(top, v.y * __expf(v.x - base) + o.y * __expf(o.x - base));
                }
                if (m_at + r < count) a.part[tn_at * a.part_ld + m_at + r] = v;
            }
        } else if constexpr (END == kGrad) {
            constexpr int GT = sizeof(T) == 4 ? 3 : 1;        // G's terms
            unsigned short *G = static_cast<unsigned short *>(a.G);
            const bool edge = n_at + BN > a.N || m_at + BM > count;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int lm = (wm * FM + i) * 16 + row;
                const long m = m_at + lm;
                const int rel = targets[lm] - a.n0 - (int)n_at - wn * FN * 16 - quad;
                const float lse = lses[lm], coef = coefs[lm];
                const bool hit = m < count && rel >= 0 && rel < FN * 16 && (rel & 12) == 0;
                const bool any = __any(hit);
                // Two column tiles at a time: lanes of odd sixteens trade theirs of the first tile for the second's of
                // the sixteen before, after which a lane holds eight neighbouring columns of one of them.
                const long m_ld = m * (GT == 3 ? 3 * a.g_term : a.g_ld);
#pragma unroll
                for (int j = 0; j < FN; j += 2) {
                    uint2 t[GT][2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float g[4];
                        // (the difference first: it is exact where the two are close, and so is a probability of one)
#pragma unroll
                        for (int r = 0; r < 4; ++r) g[r] = __expf(acc[i][j + h][r] - lse);
                        if (any)
#pragma unroll
                            for (int r = 0; r < 4; ++r) g[r] -= hit && rel == (j + h) * 16 + r ? 1.f : 0.f;
#pragma unroll
                        for (int r = 0; r < 4; ++r) g[r] *= coef;
                        if (edge) {
                            const long n = n_at + (wn * FN + j + h) * 16 + quad;
#pragma unroll
                            for (int r = 0; r < 4; ++r) g[r] = m < count && n + r < a.N ? g[r] : 0.f;
                        }
                        if constexpr (GT == 3) {
                            split4(g[0], g[1], g[2], g[3], t[0][h], t[1][h], t[2][h]);
                        } else {
                            if (BM == 128 && a.twice && (lm & 1))
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    const float held = (float)(T)g[r];
                                    g[r] = fabsf(held) < INFINITY ? g[r] - held : 0.f;
                                }
                            T v[4] = {(T)g[0], (T)g[1], (T)g[2], (T)g[3]};
                            __builtin_memcpy(&t[0][h], v, 8);
                        }
                    }
                    const long n = n_at + (wn * FN + j + (own >> 4 & 1)) * 16 + (own >> 5) * 8;
                    if (edge && (m >= a.M || n >= a.g_ld)) continue;
#pragma unroll
                    for (int q = 0; q < GT; ++q) {
                        const auto x = __builtin_amdgcn_permlane16_swap(t[q][0].x, t[q][1].x, false, false);
                        const auto y = __builtin_amdgcn_permlane16_swap(t[q][0].y, t[q][1].y, false, false);
                        *reinterpret_cast<uint4 *>(G + m_ld + q * a.g_term + n) = make_uint4(x[0], y[0], x[1], y[1]);
                    }
                }
            }
        } else {
            const float alpha = a.partial ? 1.f : *a.alpha_scale;
            if constexpr (END == kClasses && TERMS == 1) {
                // straight to 16-bit weights' gradients, 16 bytes a lane where their rows allow it
                if (!a.partial && !a.add && a.out_ld % 8 == 0 && ((unsigned long)a.out & 15) == 0 && n_at + BN <= a.N) {
#pragma unroll
                    for (int i = 0; i < FM; ++i) {
                        const long m = m_at + (wm * FM + i) * 16 + row;
                        T *to = static_cast<T *>(a.out) + m * a.out_ld + n_at + (wn * FN + (own >> 4 & 1)) * 16 + (own >> 5) * 8;
#pragma unroll
                        for (int j = 0; j < FN; j += 2) {
                            uint2 t[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                T v[4];
#pragma unroll
                                for (int r = 0; r < 4; ++r) v[r] = (T)(acc[i][j + h][r] * alpha);
                                __builtin_memcpy(&t[h], v, 8);
                            }
                            const auto x = __builtin_amdgcn_permlane16_swap(t[0].x, t[1].x, false, false);
                            const auto y = __builtin_amdgcn_permlane16_swap(t[0].y, t[1].y, false, false);
                            if (m < a.M) *reinterpret_cast<uint4 *>(to + j * 16) = make_uint4(x[0], y[0], x[1], y[1]);
                        }
                    }
                    goto done;
                }
            }
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const long m = m_at + (wm * FM + i) * 16 + row;
                if (m >= a.M || (END == kRows && m >= count)) continue;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const long n = n_at + (wn * FN + j) * 16 + quad;
                    if (n >= a.N) continue;
                    floatx4 v = acc[i][j];
                    if (a.partial) {
                        floatx4 *to = reinterpret_cast<floatx4 *>(a.partial + ((size_t)split_at * (END == kRows ? tiles_m * BM : a.M) + m) * a.part_cols + n);
                        *to = a.add ? *to + v : v;           // (part_cols is a multiple of four)
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
                        if constexpr (TERMS == 3) put(static_cast<float *>(a.out));
                        else put(static_cast<T *>(a.out));
                    }
                }
            }
        }
    done:
        if (!more) return;
        parity ^= 1;
    }
}

}  // namespace fc
