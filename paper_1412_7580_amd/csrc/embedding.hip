// Rows of a table by token, and the table's gradient.
//
//   fprop     y[n] = scale * table[token[n]]              (zero where n has no token)
//   accGrad   gtable[v] = scale * sum over n with token[n] = v of gy[n]   (+ what was there)
//
// Both move bytes and compute next to nothing: fprop reads and writes each row once, accGrad reads
// each row of gy once and writes each row of the table once.
//
// accGrad adds a token's rows in the order of n, whatever the launch: the tokens are sorted by a
// stable radix sort (least significant digit first), the sorted list is cut into chunks of equal
// length, and each chunk adds up its runs of equal tokens in fp32 registers.  A run that ends inside its
// chunk is written straight to the table; what a chunk holds of a run that crosses its borders goes to the
// workspace in fp32, and a second launch joins those parts, again in order.  So a token that half
// of the text consists of costs what any other rows cost, and two calls give the same bits.
// 16384 rows of 1024 bf16 features into a table of 32000: 50 us, of which sorting and clearing the table 24, the
// sums 17, joining 12; the 99 MB that have to move are 21 us at a copy's rate.  What is over that are six launches
// and their chains of dependent reads.
#include "operands.hpp"

namespace fc {
namespace {

constexpr int kThreads = 256, kWaves = 4;

// ---------------------------------------------------------------------------------- fprop
template <class T>
struct FpropArgs {
    const T *table;
    Tokens tok;
    T *y;
    long N;
    int D, rows, cpr;     // rows per block, chunks of 8 elements per row
    float scale;
};

template <class T>
__global__ __launch_bounds__(kThreads) void embedding_rows_kernel(FpropArgs<T> a) {
    const long n0 = (long)blockIdx.x * a.rows;
    const int rows = (int)(a.N - n0 < a.rows ? a.N - n0 : a.rows);
    const unsigned total = (unsigned)rows * a.cpr;
    for (unsigned c = threadIdx.x; c < total; c += kThreads) {
        const unsigned r = c / (unsigned)a.cpr;
        const int d = (int)(c - r * a.cpr) * 8, n = a.D - d;
        const int t = a.tok(n0 + r);
        float f[8] = {};
        if (t >= 0) {                                        // (else zero, whatever the scale)
            load8(a.table + (size_t)t * a.D + d, n, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= a.scale;
        }
        store8(a.y + (size_t)(n0 + r) * a.D + d, n, f);
    }
}

// Planes: a tile of 64 positions by 64 features turns in LDS, so that rows are read along their features
// and planes written along their positions.  (65536 positions of 512 bf16 features, in planes of 729: 31 us; of 16, where most of
// a tile's positions are not there, 54, and of 4, 178.)
template <class T>
struct PlaneArgs {
    const T *table;
    Tokens tok;
    T *y;
    int D, T_, tiles_t, tiles_d;
    float scale;
};

template <class T>
__global__ __launch_bounds__(kThreads) void embedding_planes_kernel(PlaneArgs<T> a) {
    __shared__ float tile[64][65];
    const unsigned per = (unsigned)a.tiles_t * a.tiles_d;
    const unsigned s = blockIdx.x / per, rest = blockIdx.x - s * per;
    const int t0 = (int)(rest % a.tiles_t) * 64, d0 = (int)(rest / a.tiles_t) * 64;
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int r = c >> 3, d = d0 + (c & 7) * 8;
        float f[8] = {};
        if (t0 + r < a.T_ && d < a.D) {
            const int v = a.tok((long)s * a.T_ + t0 + r);
            if (v >= 0) {
                load8(a.table + (size_t)v * a.D + d, a.D - d, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= a.scale;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[(c & 7) * 8 + i][r] = f[i];
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (t0 + lane < a.T_)
        for (int i = w; i < 64 && d0 + i < a.D; i += kWaves)
            a.y[((size_t)s * a.D + d0 + i) * a.T_ + t0 + lane] = (T)tile[i][lane];
}

// The turn back: planes of gy to rows, for accGrad (rows without a token are not needed and skipped).
template <class T>
struct TurnArgs {
    const T *gy;
    Tokens tok;
    T *rows;
    int D, T_, tiles_t, tiles_d;
};

template <class T>
__global__ __launch_bounds__(kThreads) void planes_to_rows_kernel(TurnArgs<T> a) {
    __shared__ float tile[64][65];
    const unsigned per = (unsigned)a.tiles_t * a.tiles_d;
    const unsigned s = blockIdx.x / per, rest = blockIdx.x - s * per;
    const int t0 = (int)(rest % a.tiles_t) * 64, d0 = (int)(rest / a.tiles_t) * 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (t0 + lane < a.T_) {
        T v[64 / kWaves];                                    // (all asked for before the first is stored)
#pragma unroll
        for (int i = 0; i < 64 / kWaves; ++i) {
            const int d = d0 + i * kWaves + w;
            v[i] = a.gy[((size_t)s * a.D + (d < a.D ? d : a.D - 1)) * a.T_ + t0 + lane];
        }
#pragma unroll
        for (int i = 0; i < 64 / kWaves; ++i) tile[i * kWaves + w][lane] = to_float(v[i]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
        const int r = c >> 3, dd = (c & 7) * 8, n = a.D - d0 - dd;
        if (t0 + r >= a.T_ || n <= 0) continue;
        const long row = (long)s * a.T_ + t0 + r;
        if (a.tok(row) < 0) continue;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? tile[dd + i][r] : 0.f;
        store8(a.rows + (size_t)row * a.D + d0 + dd, n, f);
    }
}

// ---------------------------------------------------------------------------------- sort
// Least significant digit first, stable.  A block's waves take neighbouring stretches of its items, 64 at a
// time; among those a lane's rank is the number of lower lanes with its digit, found by a ballot for each bit.
// The launches are short of work for the chip: blocks behind the sorting ones write the table's zeros meanwhile
// (a 32000x1024 bf16 table: 4 us more in four launches, 9 less in the sums').
//  - Up to 4096 items one block sorts them in LDS, all digits in one launch (500 items: 5 us; 16384 of them
//    would take 42, beside 21 for the launches of the other way).
//  - More are sorted by blocks of 1024 with two launches a digit: counts by block, then places.  Where a
//    digit of a block begins follows from all blocks' counts: up to kInline blocks add those up themselves,
//    beyond that a launch turns counts into places.
constexpr int kSortThreads = 1024, kSortWaves = 16;
constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;
constexpr int kOneBlock = 4096;
constexpr int kItems = kSortThreads, kInline = 32;

struct SortPlan {
    bool one;
    int passes, bits;     // digits, bits of one
    int blocks;
};
SortPlan sort_plan(long N, int V) {
    int bits = 1;
    while (bits < 31 && (1L << bits) < V) ++bits;
    SortPlan p;
    p.one = N <= kOneBlock;
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.blocks = (int)((N + kItems - 1) / kItems);
    return p;
}

struct SortArgs {
    Tokens tok;               // the first pass reads these,
    const int *key_in, *idx_in;   // the others these
    int *key_out, *idx_out;
    int *hist, *totals;       // [blocks][digits] and [digits]: counts, or places where there are totals
    int *count;               // how many rows have a token
    char *zero_from, *zero_to;    // what this launch's other blocks clear
    long N;
    int shift, bits, passes, blocks;
    int first, placed;
};

__device__ __forceinline__ int sort_key(const SortArgs &a, long at, long n) {
    return at < n ? a.first ? a.tok(at) : a.key_in[at] : -1;
}
// The work of the blocks behind the sorting ones: kZeroBytes each.
constexpr int kZeroBytes = kSortThreads * 16 * 4;
__device__ __forceinline__ void write_zeros(const SortArgs &a, int block) {
    char *const from = a.zero_from + (size_t)block * kZeroBytes;
    const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        char *const p = from + (i * kSortThreads + threadIdx.x) * 16;
        if (p + 16 <= a.zero_to) __builtin_memcpy(p, &zero, 16);
        else
            for (char *q = p; q < a.zero_to; q += 2) *reinterpret_cast<unsigned short *>(q) = 0;
    }
}

// Rank of each of a lane's items among its wave's with the same digit; `mine` (the wave's counts by digit, zero
// before) holds how many there are of each afterwards.  Items without a token (key < 0) take no part.
template <int R>
__device__ __forceinline__ void rank_items(const int (&key)[R], int shift, int bits, int *mine, int (&rank)[R]) {
    const int lane = threadIdx.x & 63, mask = (1 << bits) - 1;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool has = key[i] >= 0;
        const int digit = (key[i] >> shift) & mask;
        unsigned long long same = __ballot(has);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int lower = __popcll(same & ((1ull << lane) - 1));
        int before = 0;
        if (has) before = mine[digit];
        __builtin_amdgcn_wave_barrier();
        if (has && lower == 0) mine[digit] = before + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        rank[i] = before + lower;
    }
}

// Exclusive sum over a block's threads.
__device__ __forceinline__ int sum_before(int mine, int *part, int *all) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int upto = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int v = __shfl_up(upto, m);
        if (lane >= m) upto += v;
    }
    if (lane == 63) part[w] = upto;
    __syncthreads();
    int before = upto - mine;
    *all = 0;
#pragma unroll
    for (int q = 0; q < kSortWaves; ++q) {
        before += q < w ? part[q] : 0;
        *all += part[q];
    }
    return before;
}

// counts [waves][digits] -> places, given where each digit begins
__device__ __forceinline__ void places_of(int *counts, int digit, int at) {
#pragma unroll
    for (int q = 0; q < kSortWaves; ++q) {
        const int c = counts[q * kDigits + digit];
        counts[q * kDigits + digit] = at;
        at += c;
    }
}

template <int R>
__global__ __launch_bounds__(kSortThreads) void sort_block_kernel(SortArgs a) {
    if (blockIdx.x > 0) return write_zeros(a, blockIdx.x - 1);
    __shared__ int keys[R * kSortThreads];
    __shared__ unsigned short rows[R * kSortThreads];
    __shared__ int counts[kSortWaves * kDigits];
    __shared__ int part[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, begin = w * R * 64 + lane;
    int key[R], row[R], rank[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        row[i] = begin + i * 64;
        key[i] = sort_key(a, row[i], a.N);
    }
    int n = 0;
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.bits;
        for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        rank_items<R>(key, shift, a.bits, counts + w * kDigits, rank);
        __syncthreads();
        int sum = 0;
        if (tid < kDigits)
#pragma unroll
            for (int q = 0; q < kSortWaves; ++q) sum += counts[q * kDigits + tid];
        const int at = sum_before(sum, part, &n);
        if (tid < kDigits) places_of(counts, tid, at);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (key[i] >= 0) {
                const int to = counts[w * kDigits + ((key[i] >> shift) & ((1 << a.bits) - 1))] + rank[i];
                keys[to] = key[i];
                rows[to] = (unsigned short)row[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool has = begin + i * 64 < n;
            key[i] = has ? keys[begin + i * 64] : -1;
            row[i] = has ? rows[begin + i * 64] : 0;
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (key[i] >= 0) {
            a.key_out[begin + i * 64] = key[i];
            a.idx_out[begin + i * 64] = row[i];
        }
    if (tid == 0) *a.count = n;
}

// Text is made of few tokens: the digit of the first lane that has one is counted by all lanes at once, the
// others by an atomic each.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs a) {
    if ((int)blockIdx.x >= a.blocks) return write_zeros(a, blockIdx.x - a.blocks);
    __shared__ int h[kDigits];
    const int nd = 1 << a.bits, tid = threadIdx.x;
    if (tid < nd) h[tid] = 0;
    __syncthreads();
    const long begin = (long)blockIdx.x * kItems, n = a.first ? a.N : (long)*a.count;
    const int key = sort_key(a, begin + tid, n), digit = (key >> a.shift) & (nd - 1);
    if (const unsigned long long any = __ballot(key >= 0)) {
        const int common = __builtin_amdgcn_readlane(digit, __ffsll(any) - 1);
        const unsigned long long same = __ballot(key >= 0 && digit == common);
        if (key >= 0 && digit != common) atomicAdd(&h[digit], 1);
        if ((tid & 63) == 0) atomicAdd(&h[common], __popcll(same));
    }
    __syncthreads();
    if (tid < nd) a.hist[(size_t)blockIdx.x * nd + tid] = h[tid];
}

// Counts to places, by digit: 64 digits a block, 16 threads walk the blocks of one.
__global__ __launch_bounds__(kSortThreads) void sort_columns_kernel(SortArgs a) {
    __shared__ int sums[16][64];
    const int nd = 1 << a.bits, lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
    const int each = (a.blocks + 15) / 16, from = w * each, to = from + each < a.blocks ? from + each : a.blocks;
    int sum = 0;
    if (d < nd)
        for (int b = from; b < to; ++b) sum += a.hist[(size_t)b * nd + d];
    sums[w][lane] = sum;
    __syncthreads();
    int at = 0, all = 0;
    for (int q = 0; q < 16; ++q) {
        at += q < w ? sums[q][lane] : 0;
        all += sums[q][lane];
    }
    if (d < nd) {
        for (int b = from; b < to; ++b) {
            const int c = a.hist[(size_t)b * nd + d];
            a.hist[(size_t)b * nd + d] = at;
            at += c;
        }
        if (w == 0) a.totals[d] = all;
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortArgs a) {
    if ((int)blockIdx.x >= a.blocks) return write_zeros(a, blockIdx.x - a.blocks);
    __shared__ int counts[kSortWaves * kDigits];
    __shared__ int part[kSortWaves];
    const int nd = 1 << a.bits, tid = threadIdx.x, w = tid >> 6;
    const long n = a.first ? a.N : (long)*a.count;
    const long item = (long)blockIdx.x * kItems + tid;
    const int key[1] = {sort_key(a, item, n)}, row = a.first || item >= n ? (int)item : a.idx_in[item];
    int rank[1];
    for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) counts[i] = 0;
    int sum = 0, before = 0;             // of digit tid: in all blocks, in the blocks before this one
    if (tid < nd) {
        if (a.placed) {
            sum = a.totals[tid];
            before = a.hist[(size_t)blockIdx.x * nd + tid];
        } else {
#pragma unroll 16
            for (int b = 0; b < a.blocks; ++b) {
                const int h = a.hist[(size_t)b * nd + tid];
                sum += h;
                before += b < (int)blockIdx.x ? h : 0;
            }
        }
    }
    __syncthreads();
    rank_items<1>(key, a.shift, a.bits, counts + w * kDigits, rank);
    int all;
    const int at = sum_before(sum, part, &all) + before;      // (its barrier: the waves' counts are there)
    if (a.first && blockIdx.x == 0 && tid == 0) *a.count = all;
    if (tid < nd) places_of(counts, tid, at);
    __syncthreads();
    if (key[0] >= 0) {
        const int to = counts[w * kDigits + ((key[0] >> a.shift) & (nd - 1))] + rank[0];
        a.key_out[to] = key[0];
        a.idx_out[to] = row;
    }
}

// ---------------------------------------------------------------------------------- sums
constexpr int kMostChunk = 64;

template <class T>
struct SumArgs {
    const T *gy;
    const int *key, *idx;     // sorted
    const int *count;
    T *gtable;
    float *head, *tail;       // [chunks][D]: a chunk's part of the run that began before it / that goes on after it
    long chunks;
    int D, C;                 // C: sorted positions per chunk
    int lanes;                // threads of one row: a power of two, 8 elements each
    int slices;               // pieces of 8 * lanes elements in a row
    float scale;
    int accumulate;
};

template <class T>
__device__ __forceinline__ void finish_row(const SumArgs<T> &a, int key, int d, int n, const float (&acc)[8]) {
    T *to = a.gtable + (size_t)key * a.D + d;
    float f[8];
    if (a.accumulate) {
        load8(to, n, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += acc[i] * a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = acc[i] * a.scale;
    }
    store8(to, n, f);
}

template <class T>
__global__ __launch_bounds__(kThreads) void embedding_sum_kernel(SumArgs<T> a) {
    const int tid = threadIdx.x;
    // the chunk's tokens and rows first, so that its rows can be asked for at once
    __shared__ int keys[kThreads * kMostChunk / 8], rows[kThreads * kMostChunk / 8];
    const int groups = kThreads / a.lanes, g = tid / a.lanes, l = tid % a.lanes;
    const long unit = (long)blockIdx.x * groups + g;
    const long chunk = unit / a.slices;
    const int d = ((int)(unit - chunk * a.slices) * a.lanes + l) * 8, n = a.D - d;
    const long cnt = *a.count, begin = chunk * a.C;
    const int len = (int)(begin + a.C < cnt ? a.C : cnt > begin ? cnt - begin : 0);
    int *const key_of = keys + g * a.C, *const row_of = rows + g * a.C;
    for (int i = l; i < len; i += a.lanes) {
        key_of[i] = a.key[begin + i];
        row_of[i] = a.idx[begin + i];
    }
    const int before = begin > 0 && len ? a.key[begin - 1] : -1, after = begin + len < cnt && len ? a.key[begin + len] : -1;
    __syncthreads();
    if (len == 0 || n <= 0) return;
    int key = key_of[0];
    float acc[8] = {};
    constexpr int U = 8;
    for (int p = 0; p < len; p += U) {
        T row[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) raw8(a.gy + (size_t)row_of[p + u < len ? p + u : len - 1] * a.D + d, n, row[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= len) break;
            const int k = key_of[p + u];
            if (k != key) {
                if (key == before) store8(a.head + (size_t)chunk * a.D + d, n, acc);
                else finish_row(a, key, d, n, acc);
                key = k;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += to_float(row[u][i]);
        }
    }
    if (key == before) store8(a.head + (size_t)chunk * a.D + d, n, acc);
    else if (key == after) store8(a.tail + (size_t)chunk * a.D + d, n, acc);
    else finish_row(a, key, d, n, acc);
}

// Joins the parts of the runs that cross chunks: a block for each chunk in which a run begins that the
// chunk does not end (the others end at once).
template <class T>
__global__ __launch_bounds__(kThreads) void embedding_join_kernel(SumArgs<T> a) {
    __shared__ float sums[kThreads][9];
    const long chunk = blockIdx.x, cnt = *a.count, begin = chunk * a.C, end = begin + a.C;
    if (end >= cnt) return;                              // (nothing after it)
    const int key = a.key[end - 1];
    if (a.key[end] != key || (begin > 0 && a.key[begin - 1] == key)) return;
    long last = chunk;                                   // the chunk it ends in: the last that begins with its token
    for (int more = kThreads; more == kThreads; last += more) {      // (all ask at once: a search is a chain of reads, 10 us of them)
        const long at = (last + 1 + threadIdx.x) * a.C;
        more = __syncthreads_count(at < cnt && a.key[at] == key);
    }
    const int groups = kThreads / a.lanes, g = threadIdx.x / a.lanes, l = threadIdx.x % a.lanes;
    // group g adds the parts of a stretch of neighbouring chunks, then the stretches are added in order
    const long parts = last - chunk + 1, each = (parts + groups - 1) / groups;
    const long from = chunk + g * each, to = from + each <= last + 1 ? from + each : last + 1;
    for (int s = 0; s < a.slices; ++s) {
        const int d = (s * a.lanes + l) * 8, n = a.D - d;
        float acc[8] = {};
        if (n > 0) {
            constexpr int U = 8;
            for (long c = from; c < to; c += U) {
                float f[U][8];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long at = c + u < to ? c + u : to - 1;
                    load8((at == chunk ? a.tail : a.head) + (size_t)at * a.D + d, n, f[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c + u < to)
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[i] += f[u][i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = acc[i];
        __syncthreads();
        if (g == 0 && n > 0) {
            for (int q = 1; q * each < parts; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += sums[q * a.lanes + l][i];
            finish_row(a, key, d, n, acc);
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void zero_kernel(T *p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (size_t)gridDim.x * kThreads) p[i] = (T)0.f;
}

struct GradPlan {
    SortPlan sort;
    int lanes, slices, C;
    long chunks;
    size_t rows, key[2], idx[2], hist, totals, count, head, tail, total;
};
GradPlan grad_plan(int dtype, long N, int D, int V, int T) {
    GradPlan p;
    p.sort = sort_plan(N, V);
    const int cpr = (D + 7) / 8;
    p.lanes = 1;
    while (p.lanes < cpr && p.lanes < kThreads) p.lanes *= 2;
    if (p.lanes < 8) p.lanes = 8;
    p.slices = (cpr + p.lanes - 1) / p.lanes;
    // chunks short enough for 128k threads, long enough that the parts they leave are few
    const long c = N * (long)cpr / 131072, least = N <= 8192 ? 4 : 16;
    p.C = (int)(c < least ? least : c > kMostChunk ? kMostChunk : c);
    p.chunks = (N + p.C - 1) / p.C;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = up(at + bytes, 256); return o; };
    p.rows = take(T ? (size_t)N * D * type_bytes(dtype) : 0);
    for (int i = 0; i < 2; ++i) { p.key[i] = take((size_t)N * 4); p.idx[i] = take((size_t)N * 4); }
    p.hist = take(p.sort.one ? 0 : (size_t)p.sort.blocks * (4u << p.sort.bits));
    p.totals = take(4u << p.sort.bits);
    p.count = take(4);
    p.head = take((size_t)p.chunks * D * 4);
    p.tail = take((size_t)p.chunks * D * 4);
    p.total = at;
    return p;
}

// Of the rows' kernel: four chunks a thread, but no fewer than a thousand blocks for it.
int rows_per_block(long N, int cpr) {
    const long most = 1024 / cpr, share = (N + 1023) / 1024;
    return (int)(most < 1 ? 1 : most < share ? most : share);
}
long sum_blocks(const GradPlan &p) {
    const long groups = kThreads / p.lanes;
    return (p.chunks * p.slices + groups - 1) / groups;
}
template <class T>
hipError_t fprop(const void *table, Tokens tok, void *y, long N, int D, int Tn, float scale, hipStream_t s) {
    if (Tn) {
        PlaneArgs<T> a{static_cast<const T *>(table), tok, static_cast<T *>(y), D, Tn, (Tn + 63) / 64, (D + 63) / 64, scale};
        const long blocks = N / Tn * a.tiles_t * a.tiles_d;
        return run(embedding_planes_kernel<T>, dim3((unsigned)blocks), kThreads, 0, s, a);
    }
    FpropArgs<T> a{static_cast<const T *>(table), tok, static_cast<T *>(y), N, D, rows_per_block(N, (D + 7) / 8), (D + 7) / 8, scale};
    return run(embedding_rows_kernel<T>, dim3((unsigned)((N + a.rows - 1) / a.rows)), kThreads, 0, s, a);
}

template <class T>
hipError_t accgrad(int dtype, const void *gy, Tokens tok, void *gtable, long N, int D, int Tn, float scale, bool accumulate,
                   char *ws, hipStream_t s) {
    const int V = tok.V;
    const GradPlan p = grad_plan(dtype, N, D, V, Tn);
    const T *rows = static_cast<const T *>(gy);
    if (Tn) {
        TurnArgs<T> t{rows, tok, reinterpret_cast<T *>(ws + p.rows), D, Tn, (Tn + 63) / 64, (D + 63) / 64};
        const long blocks = N / Tn * t.tiles_t * t.tiles_d;
        if (hipError_t e = run(planes_to_rows_kernel<T>, dim3((unsigned)blocks), kThreads, 0, s, t); e != hipSuccess) return e;
        rows = t.rows;
    }
    SortArgs so{};
    so.tok = tok;
    so.count = reinterpret_cast<int *>(ws + p.count);
    so.hist = reinterpret_cast<int *>(ws + p.hist); so.totals = reinterpret_cast<int *>(ws + p.totals);
    so.N = N; so.bits = p.sort.bits; so.passes = p.sort.passes; so.blocks = p.sort.blocks;
    so.placed = p.sort.blocks > kInline;
    so.key_out = reinterpret_cast<int *>(ws + p.key[0]);
    so.idx_out = reinterpret_cast<int *>(ws + p.idx[0]);
    // the table's bytes, in as many parts as launches clear them
    char *const begin = static_cast<char *>(gtable);
    const size_t bytes = accumulate ? 0 : (size_t)V * D * sizeof(T), launches = p.sort.one ? 1 : 2 * p.sort.passes;
    const auto clear = [&](size_t i) {
        so.zero_from = begin + bytes / 16 * i / launches * 16;
        so.zero_to = i + 1 == launches ? begin + bytes : begin + bytes / 16 * (i + 1) / launches * 16;
        return (unsigned)((so.zero_to - so.zero_from + kZeroBytes - 1) / kZeroBytes);
    };
    if (p.sort.one) {
        so.first = 1;
        const unsigned grid = 1 + clear(0);
        const auto kernel = N <= 1024 ? sort_block_kernel<1> : sort_block_kernel<4>;
        if (hipError_t e = run(kernel, dim3(grid), kSortThreads, 0, s, so); e != hipSuccess) return e;
    } else {
        for (int i = 0; i < p.sort.passes; ++i) {
            so.first = i == 0;
            so.shift = i * p.sort.bits;
            so.key_in = reinterpret_cast<int *>(ws + p.key[(i + 1) & 1]);
            so.idx_in = reinterpret_cast<int *>(ws + p.idx[(i + 1) & 1]);
            so.key_out = reinterpret_cast<int *>(ws + p.key[i & 1]);
            so.idx_out = reinterpret_cast<int *>(ws + p.idx[i & 1]);
            unsigned grid = so.blocks + clear(2 * i);
            if (hipError_t e = run(sort_count_kernel, dim3(grid), kSortThreads, 0, s, so); e != hipSuccess) return e;
            if (so.placed)
                if (hipError_t e = run(sort_columns_kernel, dim3(((1 << so.bits) + 63) / 64), kSortThreads, 0, s, so); e != hipSuccess) return e;
            grid = so.blocks + clear(2 * i + 1);
            if (hipError_t e = run(sort_place_kernel, dim3(grid), kSortThreads, 0, s, so); e != hipSuccess) return e;
        }
    }
    SumArgs<T> a{};
    a.gy = rows;
    a.key = so.key_out; a.idx = so.idx_out; a.count = so.count;
    a.gtable = static_cast<T *>(gtable);
    a.head = reinterpret_cast<float *>(ws + p.head);
    a.tail = reinterpret_cast<float *>(ws + p.tail);
    a.chunks = p.chunks; a.D = D; a.C = p.C; a.lanes = p.lanes; a.slices = p.slices;
    a.scale = scale; a.accumulate = accumulate;
    if (hipError_t e = run(embedding_sum_kernel<T>, dim3((unsigned)sum_blocks(p)), kThreads, 0, s, a); e != hipSuccess) return e;
    return p.chunks > 1 ? run(embedding_join_kernel<T>, dim3((unsigned)p.chunks), kThreads, 0, s, a) : hipSuccess;
}

}  // namespace

size_t embedding_accgrad_bytes(int dtype, long N, int D, int V, int T) { return N ? grad_plan(dtype, N, D, V, T).total : 0; }

bool embedding_fits(bool accgrad, int dtype, long N, int D, int V, int T) {
    if (N == 0) return true;
    if (T && !grid_fits((double)(N / T) * ((T + 63) / 64) * ((D + 63) / 64), kThreads)) return false;
    if (!accgrad) {
        const int rows = rows_per_block(N, (D + 7) / 8);
        return T || grid_fits((double)((N + rows - 1) / rows), kThreads);
    }
    const GradPlan p = grad_plan(dtype, N, D, V, T);
    // (a sorting launch clears its share of the table: this many blocks and up to one for what does not divide)
    const double clearing = (double)V * D * type_bytes(dtype) / kZeroBytes / (p.sort.one ? 1 : 2 * p.sort.passes) + 1;
    return grid_fits((p.sort.one ? 1 : p.sort.blocks) + clearing, kSortThreads) && grid_fits((double)sum_blocks(p), kThreads) &&
           grid_fits((double)p.chunks, kThreads);
}

hipError_t launch_embedding_fprop(int dtype, const void *table, Tokens tok, void *y, long N, int D, int T, float scale, hipStream_t s) {
    if (N == 0) return hipSuccess;
    if (dtype == kF32) return fprop<float>(table, tok, y, N, D, T, scale, s);
    if (dtype == kBF16) return fprop<__bf16>(table, tok, y, N, D, T, scale, s);
    return fprop<_Float16>(table, tok, y, N, D, T, scale, s);
}

hipError_t launch_embedding_accgrad(int dtype, const void *gy, Tokens tok, void *gtable, long N, int D, int T, float scale,
                                    bool accumulate, void *ws, hipStream_t s) {
    if (N == 0) {
        if (accumulate) return hipSuccess;
        const size_t n = (size_t)tok.V * D;
        const unsigned blocks = (unsigned)(n / kThreads + 1 < 4096 ? n / kThreads + 1 : 4096);
        if (dtype == kF32) return run(zero_kernel<float>, dim3(blocks), kThreads, 0, s, static_cast<float *>(gtable), n);
        return run(zero_kernel<__bf16>, dim3(blocks), kThreads, 0, s, static_cast<__bf16 *>(gtable), n);
    }
    char *w = static_cast<char *>(ws);
    if (dtype == kF32) return accgrad<float>(dtype, gy, tok, gtable, N, D, T, scale, accumulate, w, s);
    if (dtype == kBF16) return accgrad<__bf16>(dtype, gy, tok, gtable, N, D, T, scale, accumulate, w, s);
    return accgrad<_Float16>(dtype, gy, tok, gtable, N, D, T, scale, accumulate, w, s);
}

}  // namespace fc
