// Token sampling of libimm (sm_100a) and its C ABI (declared in imm.h).
//
//   imm_sample   one token per row of logits: temperature, top-k, top-p and min-p filters, and the entry
//                at which the cumulative weight passes u times the weight the filters leave
//
// The mathematics.  With M the row's maximum, the weight of an entry is w = exp((x - M) / T).  Order the
// entries by (x descending, index ascending).  Each of the three filters keeps a prefix of that order, so
// what they leave together is a prefix too, and a prefix is given by one value and one index: the entries
// with x > X, and those with x == X and index <= I.  The draw then needs the kept weights in index order.
//
// Which entry the filters end at and which one is drawn are comparisons of sums of up to 10^5 weights with
// a border; sums in 32 bits would answer them differently for about one row in a hundred, so weights and
// sums are held in 64 bits, added in an order that the row's partition fixes: its alignment, and on the general path the
// number of blocks that share it.
//
// A row is taken by the blocks of a thread-block cluster.  One pass reads it from HBM; what a second pass needs again
// comes from L2 (the rows in flight stay below its size):
//   a strided sample of the row gives a reference M0 near the maximum and the spread of the values;
//   pass 1: the maximum of every sub-chunk of 4 KiB; the weights' sum of every sub-chunk, where all of them
//   count (no filter, or top-p); counts of the entries over 2048 bins of the value, for top-p and a large top-k
//   (integer atomics, whose order does not matter);
//   where the prefix ends: for a small top-k, the k-th largest of the sub-chunks' maxima is a bound with k entries or
//   a few more above it.  By count the bins are exact.  By mass, a bin's mass lies between its count times the weights
//   at its two edges, added up from the top or taken from the whole from the bottom;
//   pass 2, over the sub-chunks whose maximum says so: entries certainly kept are added up by sub-chunk, those of
//   the undecided bins go to a short list in shared memory, which block 0 sorts and finishes;
//   the draw: prefix sums over the sub-chunks, then over the entries of one of them.
// The blocks store what they find into block 0's shared memory and leave; only block 0 finishes the row.
// Rows that do not fit this (thousands of equal values at the border, spreads that the sample does not show, a
// top-k beyond the list, weights that the reference does not hold, temperatures next to float32's end) are answered by
// the general path: the same prefix found coarse to fine, 256 bins a pass.
//
// Weights: exp in float64 by a table of 2^(j/16) and a polynomial of degree 5 on the remainder (table-driven
// exponential, P. T. P. Tang 1989; Taylor coefficients): relative error below 2e-13.  Sixteen entries are all that
// fits the banks of shared memory side by side: no lane waits for another one's.
//
// Bound by chains of dependent float64 operations where rows are many (31 instructions per entry of pass 1, 10.5 of them
// float64, 89 in both passes of top-p; issue slots 57 % busy, the largest stall waits for a result; measured at 512 x 151936
// bf16 unfiltered: 117 us, 1.3 TB/s; 1024 x 128256 float32 with top-p 0.95: 565 us), by latency for few (1 x 128256, top-k 20:
// 11 us on the GPU, a tenth of it loads from HBM).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_sample_ns {

namespace cg = cooperative_groups;

constexpr int NT = 256;                        // threads per block
constexpr int NW = NT / 32;
constexpr int MAX_CLUSTER = 16;
constexpr int BLOCKS_PER_SM = 4;
constexpr int SUB = 256;                       // 16-byte vectors of a sub-chunk: eight per lane of a warp
constexpr int MAX_SUB = IMM_LDD_MAX_N / 4 / SUB + 1;
constexpr int BINS = 2048;                     // bins of pass 1
constexpr int BPT = BINS / NT;
constexpr int LIST = 1536;                     // longest list
constexpr int LPT = LIST / NT;
constexpr int SHORT = 1024;                    // rows that go to the list whole (16 us; a few such rows have no usable bins: 90 us and more)
constexpr int SMALL = 128;                     // longest list that one warp finishes
constexpr int NB = NT;                         // bins of the general path (one per thread in its scans)
constexpr float SPAN = 24.f;                   // its first histogram covers weights down to e^-24
constexpr float NEG_INF = -INFINITY;
constexpr float LOWEST = -3.402823466e+38f;    // the lowest finite value
constexpr int NONE = 0x7FFFFFFF;

struct Args {
    const void* logits;
    int64_t n, ld;
    const double* u;
    const float *temperature_row, *top_p_row, *min_p_row;
    const int32_t* top_k_row;
    float temperature, top_p, min_p;
    int32_t top_k;
    int32_t* token;
    float* logprob;
    int32_t *kept, *status;
};

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// order-preserving integer of a float (larger value, larger key); both zeros have one key
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

template <typename T> struct Vec;                       // a 16-byte vector of logits
template <> struct Vec<float> {
    static constexpr int V = 4;
    __device__ static void unpack(uint4 r, float (&f)[4])
    {
        f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
    }
    __device__ static void mask(uint4& r, int e) { (&r.x)[e] = 0xFF800000u; }          // -inf
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int V = 8;
    __device__ static void unpack(uint4 r, float (&f)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; i++) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    __device__ static void mask(uint4& r, int e)
    {
        uint32_t* w = &r.x + (e >> 1);
        *w = (e & 1) ? (*w & 0x0000FFFFu) | 0xFF800000u : (*w & 0xFFFF0000u) | 0x0000FF80u;
    }
};
template <> struct Vec<__half> {
    static constexpr int V = 8;
    __device__ static void unpack(uint4 r, float (&f)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = p.x; f[2 * i + 1] = p.y;
        }
    }
    __device__ static void mask(uint4& r, int e)
    {
        uint32_t* w = &r.x + (e >> 1);
        *w = (e & 1) ? (*w & 0x0000FFFFu) | 0xFC000000u : (*w & 0xFFFF0000u) | 0x0000FC00u;
    }
};

struct Publish { double mass; uint32_t count, ties; };

struct Params {
    float temperature, top_p, min_p;
    int top_k;
    double factor;                             // of Weight
    double u, min_gap;                         // min-p on the logits: x - M >= min_gap
};
// what a row needs: MASS, HIST: sums and counts in pass 1; TOPS: the bound of a small top-k
enum { FINE = 1, GREEDY = 2, USE_K = 4, USE_P = 8, LONG_K = 16, HIST = 32, MASS = 64, TOPS = 128 };

struct Shared {
    alignas(128) double table[16];             // 2^(j/16)
    Params prm;
    int flags;
    alignas(16) uint32_t hist[BINS];           // pass 1, later the list's; the general path uses it as two copies of NB bins
    uint32_t tops[MAX_CLUSTER], listed[MAX_CLUSTER];           // keys of the blocks' maxima, their entries in the list: stored here by every block
    uint32_t low, lows[MAX_CLUSTER];           // this block has a finite entry near the floor of the weights; every block's, stored alike
    uint32_t hits;                             // this block's entries in the list
    Publish pub[2];                            // this block's share of a cluster-wide sum (two copies: the other blocks may still read the last one)
    double warp_d[2][NW];
    uint32_t warp_u[2][NW];
    float warp_f[NW];
    double sum_d, before_d;                    // cluster totals, and what the blocks before this one hold
    uint32_t sum_u, before_u, sum_t, before_t;
    int first_bin, pick;
    uint32_t edge[2];
    int32_t answer_i;                          // an index found by one block, stored into every block
    // block 0: the short list.  First (~key, index) pairs, ascending: best entry first; later (index, rank) pairs.
    uint32_t list_count;
    unsigned long long list[LIST], moved[LIST];
    double list_w[LIST];
};
static_assert(2 * NB <= BINS && BPT == 8 && LIST % NT == 0 && LIST <= BINS, "bins and lists are whole shares of the threads");

// By sub-chunk of the whole row, behind Shared: block 0's copy is what all blocks fill.  (The general path uses a block's
// own copy for its own sub-chunks.)
struct Subs {
    double *mass, *kept;                       // weights; weights of what the filters certainly keep
    uint32_t *count, *kept_count, *top;        // finite entries; kept ones; key of the maximum (in every block)
};
__host__ __device__ constexpr size_t subs_bytes(int nsub) { return (size_t)nsub * (2 * sizeof(double) + 3 * sizeof(uint32_t)); }

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xFFFFFFFFu, v); }
// what the lanes before hold, from their inclusive sums: the sum less the lane's own would lose what is small beside it
__device__ __forceinline__ double lanes_before(double inclusive, int lane)
{
    const double t = __shfl_up_sync(0xFFFFFFFFu, inclusive, 1);
    return lane ? t : 0.0;
}
template <typename V> __device__ __forceinline__ V warp_scan(V v, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const V t = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += t; }
    return v;
}

// A row as its 16-byte vectors; the first may begin before the row and the last end behind it (always inside the
// 16-byte granules that the row touches).
template <typename T>
struct Row {
    static constexpr int V = Vec<T>::V;
    const uint4* stream;
    int shift;                                 // entries of the first vector that lie before the row
    int n, nv;                                 // entries, vectors
    int s0, s1;                                // this block's sub-chunks

    __device__ __forceinline__ uint4 raw(int v) const          // entries outside the row read as -inf
    {
        uint4 r = __ldg(stream + v);
        const int e0 = v * V - shift;
        if (e0 < 0 || e0 + V > n) {
            for (int e = 0; e < V; e++)
                if (e0 + e < 0 || e0 + e >= n) Vec<T>::mask(r, e);
        }
        return r;
    }
    // vector j (0..7) of a lane in sub-chunk s; `in`: the sub-chunk lies inside the row
    __device__ __forceinline__ bool inner(int s) const { return s > 0 && (s + 1) * SUB < nv; }
    __device__ __forceinline__ uint4 vec(int s, int lane, int j, bool in) const
    {
        const int v = s * SUB + 32 * j + lane;
        if (in) return __ldg(stream + v);
        if (v < nv) return raw(v);
        uint4 r = make_uint4(0, 0, 0, 0);
        for (int e = 0; e < V; e++) Vec<T>::mask(r, e);        // past the row: -inf
        return r;
    }
    __device__ __forceinline__ float entry(int i) const        // 0 <= i < n
    {
        const T v = __ldg(reinterpret_cast<const T*>(stream) + shift + i);
        return (float)v;
    }
    // one cache line per lane: a whole sub-chunk on its way to L2
    __device__ __forceinline__ void prefetch(int s, int lane) const
    {
        const int v = s * SUB + 8 * lane;
        if (s < s1 && v < nv) asm volatile("prefetch.global.L2 [%0];" ::"l"(stream + v));
    }
    // calls f(x, first index) for every vector of sub-chunk s that this lane holds.  Two vectors a step, the next two
    // on their way: short code (a pass over few sub-chunks waits for instructions otherwise) with enough loads in flight.
    template <typename F>
    __device__ __forceinline__ void vectors(int s, int lane, F&& f) const
    {
        const bool in = inner(s);
        uint4 a = vec(s, lane, 0, in), b = vec(s, lane, 1, in);
#pragma unroll 1
        for (int j = 0; j < 8; j += 2) {
            uint4 a2 = a, b2 = b;
            if (j < 6) { a2 = vec(s, lane, j + 2, in); b2 = vec(s, lane, j + 3, in); }
            const int i0 = (s * SUB + 32 * j + lane) * V - shift;
            float x[V];
            Vec<T>::unpack(a, x);
            f(x, i0);
            Vec<T>::unpack(b, x);
            f(x, i0 + 32 * V);
            a = a2; b = b2;
        }
    }
    // ... with all eight loads at once, for passes with little work per entry
    template <typename F>
    __device__ __forceinline__ void vectors_at_once(int s, int lane, F&& f) const
    {
        const bool in = inner(s);
        uint4 r[8];
#pragma unroll
        for (int j = 0; j < 8; j++) r[j] = vec(s, lane, j, in);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            float x[V];
            Vec<T>::unpack(r[j], x);
            f(x, j);
        }
    }
    // calls f(value, index) for the entries of sub-chunk s that this lane holds
    template <typename F>
    __device__ __forceinline__ void each_in(int s, int lane, F&& f) const
    {
        vectors(s, lane, [&](const float (&x)[V], int i0) {
#pragma unroll
            for (int e = 0; e < V; e++) f(x[e], i0 + e);
        });
    }
    // ... of all sub-chunks of this block that the warp takes
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const
    {
        for (int s = s0 + (int)(threadIdx.x >> 5); s < s1; s += NW) each_in(s, threadIdx.x & 31, f);
    }
};

// exp(x / T) up to a factor of the row, in float64: with y = x 16 log2(e) / T, K the nearest integer to y and r = y - K
// (one fused operation: exact up to the rounding of the factor), 2^((K - R)/16) * 2^(r/16); R, the integer nearest to the
// reference's y, keeps the range.  The large constant that rounds y carries -R as well.
struct Weight {
    double factor, least, bias;                // least: -689 T; bias = 1.5 * 2^52 - R: the sum's low word is K - R
    float floor;                               // lower values count as this one (e^-690 of the reference)
    const double* table;

    __device__ __forceinline__ void set(float reference, const Params& prm, const double* tab)
    {
        const float temperature = prm.temperature;
        factor = prm.factor;                                               // 16 log2(e) / T
        least = -689.0 * (double)temperature;
        bias = 6755399441055744.0 - rint((double)reference * factor);
        floor = (float)fmax((double)reference - 690.0 * (double)temperature, (double)LOWEST);
        table = tab;
    }
    __device__ __forceinline__ double finish(double r, int K) const        // 2^(K/16) 2^(r/16)
    {
        // (ln 2 / 16)^k / k!
        constexpr double L = 0.043321698784996581838;
        constexpr double c1 = L, c2 = L * L / 2, c3 = L * L * L / 6, c4 = L * L * L * L / 24, c5 = L * L * L * L * L / 120;
        double p = fma(c5, r, c4);
        p = fma(p, r, c3);
        p = fma(p, r, c2);
        p = fma(p, r, c1);
        p = fma(p, r, 1.0);
        const double w = p * table[K & 15];
        return __hiloint2double(__double2hiint(w) + (int)((uint32_t)(K & ~15) << 16), __double2loint(w));
    }
    __device__ __forceinline__ double operator()(float value) const        // (NaN and -inf: as `floor`)
    {
        const double x = (double)fmaxf(value, floor);
        const double km = fma(x, factor, bias);
        return finish(fma(x, factor, bias - km), __double2loint(km));
    }
    // exp(d / T) for a gap d <= 0 itself, exactly 1 for d = 0, down to float64's smallest value and 0 below it
    __device__ __forceinline__ double of_gap(double d) const
    {
        const double MAGIC = 6755399441055744.0;
        const double e = fmax(d, 2.0 * least);
        const double km = fma(e, factor, MAGIC);
        const int K = __double2loint(km);
        const bool far = K < -15900;           // the power of two in two factors, the second of which rounds
        const double w = finish(fma(e, factor, MAGIC - km), far ? K + 16000 : K);
        return far ? w * 0x1p-1000 : w;
    }
};

// Bins of a value: round(c - x scale), 0 at the top, the last one takes everything below.  c is an integer of less than
// 2^22, so adding 1.5 * 2^23 makes the fused operation round exactly there.
struct Grid {
    float c, scale;
    static constexpr float MAGIC = 12582912.f;
    static constexpr int BASE = 0x4B400000;    // its bits
    __device__ __forceinline__ int raw(float x) const { return max(__float_as_int(fmaf(x, -scale, c + MAGIC)), BASE); }
    __device__ __forceinline__ int of(float x) const { return min(raw(x) - BASE, BINS - 1); }
};
// the general path's: linear from the top
struct Linear {
    float top, scale;
    __device__ __forceinline__ int of(float x) const { return (int)fminf(fmaxf((top - x) * scale, 0.f), (float)(NB - 1)); }
};

// Everything the paths share: the block's view of the row, and block-wide helpers (all threads call them).
template <typename T>
struct Work {
    Row<T> row;
    Shared& sh;
    Subs subs;                                 // this block's copies
    cg::cluster_group cluster;
    int nc, c, tid, lane, warp;
    int flip, hflip;                           // which copy of pub / of the general path's histogram is in use
    float M;

    // memory of block b: the block's own is addressed directly, so that block barriers order it
    template <typename P> __device__ __forceinline__ P* at(P* p, int b) const { return b == c ? p : cluster.map_shared_rank(p, b); }
    __device__ __forceinline__ Shared* of(int b) { return at(&sh, b); }
    __device__ __forceinline__ void sync_all()
    {
        if (nc == 1) __syncthreads();
        else cluster.sync();
    }
    // sums of (mass, count, ties) over the cluster: totals, and what the blocks before hold
    __device__ void exchange(double mass, uint32_t count, uint32_t ties)
    {
        mass = warp_sum(mass); count = warp_sum(count); ties = warp_sum(ties);
        __syncthreads();                       // (the last exchange's values have been read)
        if (lane == 0) { sh.warp_d[0][warp] = mass; sh.warp_u[0][warp] = count; sh.warp_u[1][warp] = ties; }
        __syncthreads();
        if (tid == 0) {
            double s = 0.0; uint32_t k = 0, t = 0;
            for (int w = 0; w < NW; w++) { s += sh.warp_d[0][w]; k += sh.warp_u[0][w]; t += sh.warp_u[1][w]; }
            sh.pub[flip].mass = s; sh.pub[flip].count = k; sh.pub[flip].ties = t;
        }
        sync_all();
        if (tid == 0) {
            double s = 0.0, sb = 0.0; uint32_t k = 0, kb = 0, t = 0, tb = 0;
            for (int b = 0; b < nc; b++) {
                const Publish p = of(b)->pub[flip];
                if (b == c) { sb = s; kb = k; tb = t; }
                s += p.mass; k += p.count; t += p.ties;
            }
            sh.sum_d = s; sh.before_d = sb; sh.sum_u = k; sh.before_u = kb; sh.sum_t = t; sh.before_t = tb;
        }
        __syncthreads();
        flip ^= 1;
    }
    // inclusive scans over the block's threads, and the total
    __device__ uint32_t scan_u(uint32_t v, uint32_t* total = nullptr)
    {
        uint32_t s = warp_scan(v, lane);
        __syncthreads();
        if (lane == 31) sh.warp_u[0][warp] = s;
        __syncthreads();
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < NW; w++) { const uint32_t x = sh.warp_u[0][w]; s += w < warp ? x : 0u; all += x; }
        if (total) *total = all;
        return s;
    }
    __device__ double scan_d(double v, int slot, double* total = nullptr, bool exclusive = false)
    {
        double s = warp_scan(v, lane);
        __syncthreads();
        if (lane == 31) sh.warp_d[slot][warp] = s;
        if (exclusive) s = lanes_before(s, lane);
        __syncthreads();
        double before = 0.0, all = 0.0;
#pragma unroll
        for (int w = 0; w < NW; w++) { const double x = sh.warp_d[slot][w]; before += w < warp ? x : 0.0; all += x; }
        if (total) *total = all;
        return before + s;
    }
    // the sum over the threads before
    __device__ double before_d(double v, int slot, double* total = nullptr) { return scan_d(v, slot, total, true); }
    __device__ int first_of(int candidate, int none)       // the smallest candidate over the block, at most `none`
    {
        const int m = __reduce_min_sync(0xFFFFFFFFu, candidate);
        __syncthreads();
        if (lane == 0) sh.warp_u[1][warp] = (uint32_t)m;
        __syncthreads();
        int best = none;
#pragma unroll
        for (int w = 0; w < NW; w++) best = min(best, (int)sh.warp_u[1][w]);
        return best;
    }
    __device__ int first_true(bool yes, int none) { return first_of(yes ? tid : NONE, none); }

    // khi: the largest key whose value falls into a bin >= b1; klo: the smallest one with a bin <= b2 (bins fall
    // with rising keys).  A search with 32 probes a round, by two warps.
    template <typename G>
    __device__ void bin_edges(const G& g, int b1, int b2, uint32_t& khi, uint32_t& klo)
    {
        __syncthreads();
        if (warp < 2) {
            uint64_t lo = key_of(LOWEST), hi = key_of(M);                  // the answers lie in [lo, hi]
            while (lo < hi) {
                const uint64_t gap = hi - lo, off = min(gap, (gap / 32 + 1) * lane);
                const uint64_t probe = warp == 0 ? hi - off : lo + off;
                const int b = g.of(value_of((uint32_t)probe));
                const unsigned hits = __ballot_sync(0xFFFFFFFFu, warp == 0 ? b >= b1 : b <= b2);       // monotone in the lane
                if (!hits) {                                               // beyond the last probe
                    const uint64_t last = __shfl_sync(0xFFFFFFFFu, probe, 31);
                    if (warp == 0) { if (last == lo) break; hi = last - 1; } else { if (last == hi) break; lo = last + 1; }
                } else {                                                   // at the first hit or between it and the probe before
                    const int f = __ffs(hits) - 1;
                    const uint64_t at = __shfl_sync(0xFFFFFFFFu, probe, f), prev = __shfl_sync(0xFFFFFFFFu, probe, f > 0 ? f - 1 : 0);
                    if (warp == 0) { lo = at; hi = f > 0 ? prev - 1 : at; } else { hi = at; lo = f > 0 ? prev + 1 : at; }
                }
            }
            if (lane == 0) sh.edge[warp] = (uint32_t)(warp == 0 ? hi : lo);
        }
        __syncthreads();
        khi = sh.edge[0]; klo = sh.edge[1];
    }
    // the smallest value that min-p leaves: x - M >= gap (M itself always stays)
    __device__ float min_p_value(double gap_allowed)
    {
        __syncthreads();
        if (warp == 0) {
            uint64_t lo = key_of(LOWEST), hi = key_of(M);
            while (lo < hi) {
                const uint64_t gap = hi - lo, probe = lo + min(gap, (gap / 32 + 1) * lane);
                const unsigned hits = __ballot_sync(0xFFFFFFFFu, (double)value_of((uint32_t)probe) - (double)M >= gap_allowed);
                if (!hits) { lo = __shfl_sync(0xFFFFFFFFu, probe, 31) + 1; continue; }
                const int f = __ffs(hits) - 1;
                const uint64_t at = __shfl_sync(0xFFFFFFFFu, probe, f), prev = __shfl_sync(0xFFFFFFFFu, probe, f > 0 ? f - 1 : 0);
                hi = at;
                lo = f > 0 ? prev + 1 : at;
            }
            if (lane == 0) sh.edge[0] = (uint32_t)hi;
        }
        __syncthreads();
        return value_of(sh.edge[0]);
    }
    // Sorts sh.list[0..m) (distinct pairs) by a counting sort over BINS bins of the upper word, then by rank within a
    // bin; a short list by rank alone.
    __device__ void sort_list(int m)
    {
        unsigned long long mine[LPT];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < LPT; q++) mine[q] = tid + q * NT < m ? sh.list[tid + q * NT] : 0ull;
        if (m <= 64) {
            int r = 0;
            if (tid < m) for (int j = 0; j < m; j++) r += sh.list[j] < mine[0] ? 1 : 0;
            __syncthreads();
            if (tid < m) sh.list[r] = mine[0];
            __syncthreads();
            return;
        }
        uint32_t lowest = ~0u, highest = 0;
#pragma unroll
        for (int q = 0; q < LPT; q++)
            if (tid + q * NT < m) { lowest = min(lowest, (uint32_t)(mine[q] >> 32)); highest = max(highest, (uint32_t)(mine[q] >> 32)); }
        lowest = __reduce_min_sync(0xFFFFFFFFu, lowest);
        highest = __reduce_max_sync(0xFFFFFFFFu, highest);
        if (lane == 0) { sh.warp_u[0][warp] = lowest; sh.warp_u[1][warp] = highest; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; w++) { lowest = min(lowest, sh.warp_u[0][w]); highest = max(highest, sh.warp_u[1][w]); }
        int s = 0;
        while (((highest - lowest) >> s) >= BINS) s++;
        uint4* bins = reinterpret_cast<uint4*>(sh.hist) + 2 * tid;
        bins[0] = bins[1] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        int slot[LPT];
#pragma unroll
        for (int q = 0; q < LPT; q++)
            if (tid + q * NT < m) slot[q] = (int)atomicAdd(&sh.hist[((uint32_t)(mine[q] >> 32) - lowest) >> s], 1u);
        __syncthreads();
        uint32_t h[BPT], part = 0;
#pragma unroll
        for (int q = 0; q < BPT; q++) { h[q] = sh.hist[tid * BPT + q]; part += h[q]; }
        uint32_t before = scan_u(part) - part;
#pragma unroll
        for (int q = 0; q < BPT; q++) { const uint32_t n = h[q]; sh.hist[tid * BPT + q] = before; before += n; }       // where every bin begins
        __syncthreads();
#pragma unroll
        for (int q = 0; q < LPT; q++)
            if (tid + q * NT < m) sh.moved[sh.hist[((uint32_t)(mine[q] >> 32) - lowest) >> s] + slot[q]] = mine[q];
        __syncthreads();
#pragma unroll 1
        for (int q = 0; q < LPT; q++)
            if (tid + q * NT < m) {
                const uint32_t b = ((uint32_t)(mine[q] >> 32) - lowest) >> s, first = sh.hist[b], end = b + 1 < BINS ? sh.hist[b + 1] : (uint32_t)m;
                uint32_t r = first;
                for (uint32_t j = first; j < end; j++) r += sh.moved[j] < mine[q] ? 1 : 0;
                sh.list[r] = mine[q];
            }
        __syncthreads();
    }
};

__device__ __forceinline__ void answer(const Args& a, int64_t step, int token, double logprob, uint32_t kept)
{
    a.token[step] = token; a.logprob[step] = (float)logprob; a.kept[step] = (int32_t)kept; a.status[step] = IMM_OK;
}

// The draw within sub-chunk s, by the whole block, a vector per thread: the entries of the prefix (X, I) in index order,
// `before` the weight of everything before the sub-chunk, `aim` the weight to pass.  An entry at which the sum does not
// grow is never drawn: the sum before it passes `aim` as well, or neither does.
template <typename T, typename F>
__device__ __forceinline__ void draw_in_sub(const Args& a, int64_t step, Work<T>& k, F&& weight, int s, float X, int I, double before,
                            double aim, double total, uint32_t kept)
{
    constexpr int V = Row<T>::V;
    static_assert(SUB == NT, "a vector per thread");
    const int v = s * SUB + k.tid, i0 = v * V - k.row.shift;
    float x[V];
    if (v < k.row.nv) Vec<T>::unpack(k.row.raw(v), x);
    double w[V], mine = 0.0;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const float y = v < k.row.nv ? x[e] : NEG_INF;
        w[e] = y > X || (y == X && i0 + e <= I) ? weight(y) : 0.0;         // 0: not kept
        mine += w[e];
    }
    double run = before + k.before_d(mine, 0);
    int at = -1, grown = -1, last = -1;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const double next = run + w[e];
        if (w[e] > 0.0) last = e;
        if (next > run) {
            grown = e;
            if (at < 0 && next > aim) at = e;
        }
        run = next;
    }
    int winner = k.first_true(at >= 0, NT);
    if (winner == NT) {
        // rounding hides the entry: the last one at which the sum grows (or the last one with a weight, in a sub-chunk
        // at which it grows by all of them together)
        const int best = -k.first_of(grown >= 0 ? -(k.tid + NT) : last >= 0 ? -k.tid : 1, 1);
        at = best >= NT ? grown : last;
        winner = best >= NT ? best - NT : best;
    }
    if (k.tid == winner) {
        double mass = 0.0;
#pragma unroll
        for (int e = 0; e < V; e++) if (e == at) mass = w[e];
        answer(a, step, i0 + at, log(mass / total), kept);
    }
}

// ------------------------------------------------------------------------------------------
// The general path: a prefix found coarse to fine, whatever the values are
// ------------------------------------------------------------------------------------------

template <typename T>
struct General {
    Work<T>& k;
    const Params& prm;
    Weight scale;
    float X;                                   // the prefix: x > X, or x == X and index <= I
    int I;

    __device__ __forceinline__ double weight(float x) const { return scale.of_gap((double)x - (double)k.M); }
    __device__ __forceinline__ bool inside(float x, int i) const { return x > X || (x == X && i <= I); }
    __device__ __forceinline__ uint32_t* bins(int copy) { return k.sh.hist + copy * NB; }

    __device__ uint32_t merged_bin()           // bin `tid` summed over the cluster
    {
        k.sync_all();
        uint32_t s = 0;
        for (int b = 0; b < k.nc; b++) s += (k.of(b)->hist + k.hflip * NB)[k.tid];
        k.hflip ^= 1;
        bins(k.hflip)[k.tid] = 0;              // the other copy was last read before this barrier
        __syncthreads();
        return s;
    }

    // index of the j-th (j >= 1) entry of value x in index order (`ties`: its entries inside the prefix so far)
    __device__ int tie_index(float x, uint32_t j)
    {
        // entries by sub-chunk, then prefix sums over this block's sub-chunks
        for (int s = k.row.s0 + k.warp; s < k.row.s1; s += NW) {
            uint32_t cnt = 0;
            k.row.each_in(s, k.lane, [&](float y, int i) { cnt += (y == x && inside(y, i)) ? 1u : 0u; });
            cnt = warp_sum(cnt);
            if (k.lane == 0) k.subs.count[s - k.row.s0] = cnt;
        }
        __syncthreads();
        uint32_t mine = 0;
        for (int s = k.row.s0 + k.tid; s < k.row.s1; s += NT) mine += k.subs.count[s - k.row.s0];
        k.exchange(0.0, 0, mine);
        const uint32_t own = k.sh.pub[k.flip ^ 1].ties;
        if (j > k.sh.before_t && j <= k.sh.before_t + own && k.warp == 0) {
            uint32_t want = j - k.sh.before_t;
            int s = k.row.s0;
            while (want > k.subs.count[s - k.row.s0]) want -= k.subs.count[s++ - k.row.s0];
            const int v0 = s * SUB + 8 * k.lane;           // a lane takes eight neighbouring vectors
            constexpr int V = Row<T>::V;
            uint32_t cnt = 0;
            for (int q = 0; q < 8 && v0 + q < k.row.nv; q++) {
                float f[V];
                Vec<T>::unpack(k.row.raw(v0 + q), f);
#pragma unroll
                for (int e = 0; e < V; e++) cnt += (f[e] == x) ? 1u : 0u;
            }
            uint32_t run = cnt;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, run, o); if (k.lane >= o) run += t; }
            if (cnt && want > run - cnt && want <= run) {
                uint32_t left = want - (run - cnt);
                int at = -1;
                for (int q = 0; q < 8 && v0 + q < k.row.nv; q++) {
                    float f[V];
                    Vec<T>::unpack(k.row.raw(v0 + q), f);
#pragma unroll
                    for (int e = 0; e < V; e++) if (f[e] == x && left && --left == 0) at = (v0 + q) * V - k.row.shift + e;
                }
                for (int b = 0; b < k.nc; b++) k.of(b)->answer_i = at;
            }
        }
        k.sync_all();
        return k.sh.answer_i;
    }

    // Refines [klo, khi] (keys) until one value is left that holds the end of the prefix, then sets X and I.  By count:
    // the prefix has `want` entries, `above` of which have keys over khi.  By mass: it is the shortest whose mass reaches
    // `target`; entries with keys over khi and not over khi_known are not in mass_above yet.
    __device__ void refine(bool by_mass, uint32_t khi, uint32_t klo, uint32_t khi_known, uint32_t above, uint32_t want, double target)
    {
        double mass_above = 0.0;
        for (int level = 0; level < 64; level++) {             // (11 levels at most: every one leaves an eighth or less)
            int s = 0;
            while (((khi - klo) >> s) >= NB) s++;
            const bool last = khi == klo;
            double mass = 0.0;
            uint32_t ties = 0;
            uint32_t* hist = bins(k.hflip);
            k.row.each([&](float x, int i) {
                if (!inside(x, i)) return;
                const uint32_t key = key_of(x);
                if (key > khi) {
                    if (by_mass && key <= khi_known) mass += weight(x);
                } else if (key >= klo) {
                    if (last) ties++;
                    else atomicAdd(&hist[(khi - key) >> s], 1u);
                }
            });
            if (by_mass || last) { k.exchange(mass, 0, ties); mass_above += k.sh.sum_d; khi_known = khi; }
            if (last) {
                const float x = value_of(khi);
                const uint32_t all = k.sh.sum_t;
                uint32_t j = want - above;
                if (by_mass) {
                    const double w = weight(x);
                    double guess = ceil((target - mass_above) / w);
                    if (!(guess >= 1.0)) guess = 1.0;
                    if (guess > (double)all) guess = (double)all;
                    j = (uint32_t)guess;
                    for (int t = 0; t < 4 && j > 1 && mass_above + (double)(j - 1) * w >= target; t++) j--;
                    for (int t = 0; t < 4 && j < all && mass_above + (double)j * w < target; t++) j++;
                }
                const int at = j >= all ? (x == X ? I : 0x7FFFFFFF) : tie_index(x, j);
                X = x; I = at;
                return;
            }
            const uint32_t mine = merged_bin();
            int b1, b2;
            const uint32_t cum = k.scan_u(mine);
            if (by_mass) {
                const uint32_t top = khi - ((uint32_t)k.tid << s);
                const bool real = ((uint32_t)k.tid << s) <= khi - klo;
                const uint32_t bottom = top - klo < (1u << s) ? klo : top - ((1u << s) - 1u);
                const double hi = real ? (double)mine * weight(value_of(top)) : 0.0;
                const double lo = real ? (double)mine * weight(value_of(bottom)) : 0.0;
                const double upper = k.scan_d(hi, 0), lower = k.scan_d(lo, 1);
                const int end = (int)((khi - klo) >> s);
                b1 = k.first_true(mass_above + upper * (1.0 + 1e-12) >= target * (1.0 - 1e-12), end);
                b2 = k.first_true(mass_above + lower * (1.0 - 1e-12) >= target * (1.0 + 1e-12), end);
                // bounds too wide to help (weights that differ much within a bin), or the border nearer to a key's
                // mass than they resolve: halve the bins by their exact mass
                while (b2 > b1 && (s == 0 || b2 - b1 > NB / 8)) {
                    const int mid = (b1 + b2) >> 1;
                    const uint32_t split = khi - (((uint32_t)mid << s) + ((1u << s) - 1u));     // lowest key of bin `mid`
                    double part = 0.0;
                    k.row.each([&](float x, int i) {
                        const uint32_t key = key_of(x);
                        if (key >= split && key <= khi_known && inside(x, i)) part += weight(x);
                    });
                    k.exchange(part, 0, 0);
                    if (mass_above + k.sh.sum_d >= target) b2 = mid;
                    else { b1 = mid + 1; mass_above += k.sh.sum_d; khi_known = split - 1; }
                }
            } else {
                b1 = b2 = k.first_true(above + cum >= want, NB - 1);
                __syncthreads();
                if (k.tid == b1) k.sh.first_bin = (int)(cum - mine);
                __syncthreads();
                above += (uint32_t)k.sh.first_bin;
            }
            const uint32_t depth = ((uint32_t)b2 << s) + ((1u << s) - 1u);
            const uint32_t new_lo = depth >= khi - klo ? klo : khi - depth;
            khi = khi - ((uint32_t)b1 << s);
            klo = new_lo;
        }
    }

    __device__ void run(const Args& a, int64_t step)
    {
        const float M = k.M, t = prm.temperature;
        X = LOWEST; I = 0x7FFFFFFF;            // every finite entry
        k.sync_all();                          // the other blocks have read what pass 1 left here
        bins(0)[k.tid] = 0; bins(1)[k.tid] = 0;
        k.hflip = 0;
        k.sync_all();
        const Linear grid{M, fmaxf(fminf((float)NB / (SPAN * t), 1e30f), 1e-30f)};
        const double inv_t = 1.0 / (double)t, width = 1.0 / (double)grid.scale;

        if (prm.top_k > 0 && prm.top_k < k.row.n) {
            uint32_t count = 0;
            uint32_t* hist = bins(k.hflip);
            k.row.each([&](float x, int) {
                if (x > NEG_INF) { count++; atomicAdd(&hist[grid.of(x)], 1u); }
            });
            k.exchange(0.0, count, 0);
            const uint32_t total = k.sh.sum_u, mine = merged_bin();
            if (total > (uint32_t)prm.top_k) {             // (else all are kept)
                const uint32_t cum = k.scan_u(mine);
                const int b1 = k.first_true(cum >= (uint32_t)prm.top_k, NB - 1);
                __syncthreads();
                if (k.tid == b1) k.sh.first_bin = (int)(cum - mine);
                __syncthreads();
                const uint32_t above = (uint32_t)k.sh.first_bin;
                uint32_t khi, klo;
                k.bin_edges(grid, b1, b1, khi, klo);
                refine(false, khi, klo, khi, above, (uint32_t)prm.top_k, 0.0);
            }
        }
        if (prm.top_p < 1.f) {                 // the mass and the first histogram in one pass
            double mass = 0.0;
            uint32_t* hist = bins(k.hflip);
            k.row.each([&](float x, int i) {
                if (!inside(x, i)) return;
                mass += weight(x);
                atomicAdd(&hist[grid.of(x)], 1u);
            });
            k.exchange(mass, 0, 0);
            const double target = (double)prm.top_p * k.sh.sum_d;
            const uint32_t mine = merged_bin();
            // bounds of a bin's mass: the weights at its edges, a thousandth of a bin outwards for the rounding of Grid::of
            const double hi = (double)mine * exp(-fmax(0.0, (double)k.tid - 1e-3) * width * inv_t);
            const double lo = k.tid == NB - 1 ? 0.0 : (double)mine * exp(-((double)k.tid + 1.001) * width * inv_t);
            const double upper = k.scan_d(hi, 0), lower = k.scan_d(lo, 1);
            const int b1 = k.first_true(upper >= target * (1.0 - 1e-9), NB - 1), b2 = k.first_true(lower >= target * (1.0 + 1e-9), NB - 1);
            uint32_t khi, klo;
            k.bin_edges(grid, b1, b2, khi, klo);
            refine(true, khi, klo, key_of(M), 0, 0, target);
        }
        if (prm.min_p > 0.f) {
            const float x = k.min_p_value(prm.min_gap);
            if (x > X) { X = x; I = 0x7FFFFFFF; }
        }
        // the draw: kept weights by sub-chunk of this block, the block, the sub-chunk, the entry
        for (int s = k.row.s0 + k.warp; s < k.row.s1; s += NW) {
            double mass = 0.0;
            uint32_t count = 0;
            k.row.each_in(s, k.lane, [&](float x, int i) { if (inside(x, i)) { mass += weight(x); count++; } });
            mass = warp_sum(mass); count = warp_sum(count);
            if (k.lane == 0) { k.subs.mass[s - k.row.s0] = mass; k.subs.count[s - k.row.s0] = count; }
        }
        __syncthreads();
        double mass = 0.0;
        uint32_t count = 0;
        for (int s = k.row.s0 + k.tid; s < k.row.s1; s += NT) { mass += k.subs.mass[s - k.row.s0]; count += k.subs.count[s - k.row.s0]; }
        k.exchange(mass, count, 0);
        const double total = k.sh.sum_d, aim = prm.u * total;
        const uint32_t kept = k.sh.sum_u;
        int owner = -1, last_block = 0;
        double reached = 0.0;
        for (int b = 0; b < k.nc; b++) {
            const double next = reached + k.of(b)->pub[k.flip ^ 1].mass;
            if (next > reached) {
                last_block = b;
                if (owner < 0 && next > aim) owner = b;
            }
            reached = next;
        }
        if (owner < 0) owner = last_block;     // (rounding may hide the last one at which the sum grows)
        if (owner == k.c) {
            double before = k.sh.before_d, at_last = before;
            int s = k.row.s0, last_sub = s;
            bool found = false, grown = false;
            for (; s < k.row.s1; s++) {
                const double m = k.subs.mass[s - k.row.s0], next = before + m;
                if (next > before || (m > 0.0 && !grown)) {    // (the sum may grow by all of them together only)
                    last_sub = s; at_last = before;
                    grown = next > before;
                    if (grown && next > aim) { found = true; break; }
                }
                before = next;
            }
            if (!found) { s = last_sub; before = at_last; }
            draw_in_sub<T>(a, step, k, [&](float x) { return weight(x); }, s, X, I, before, aim, total, kept);
        }
    }
};

template <typename T>
__device__ __noinline__ void general_row(const Args& a, int64_t step, Work<T>& k, const Params& prm)
{
    General<T> g{k, prm};
    g.scale.set(k.M, prm, k.sh.table);
    g.run(a, step);
}

// ------------------------------------------------------------------------------------------
// The kernel: two passes and a short list
// ------------------------------------------------------------------------------------------

// Pass 1 over this block's sub-chunks.  SUMS: sums of weights and counts of finite entries; COUNTS: the histogram.
// What it finds goes to block 0's copy of the sub-chunks; the maxima to all blocks' copies.  The sums count masked entries,
// those beside the row and any other below the floor at its weight: at most 1e-273 of the maximum's, together less than 1e-267
// of the row's.  That moves no draw but those with the smallest numbers u; for these, a finite entry less than 60 T above the
// floor is reported (where there is none, the sums are off by less than e^-50 of themselves).
template <typename T, bool SUMS, bool COUNTS>
__device__ __forceinline__ uint32_t first_pass(const Work<T>& k, const Subs& all, const Weight& weight, const Grid& grid)
{
    const Row<T>& row = k.row;
    Shared& sh = k.sh;
    const int lane = k.lane, warp = k.warp;
    uint32_t* tops = lane < k.nc ? k.at(k.subs.top, lane) : nullptr;       // a lane for every block
    uint32_t top = 0;
    row.prefetch(row.s0 + warp, lane);
    for (int s = row.s0 + warp; s < row.s1; s += NW) {
        row.prefetch(s + NW, lane);
        float best = NEG_INF, least = INFINITY;
        double mass = 0.0;
        if (!SUMS && !COUNTS)
            row.vectors_at_once(s, lane, [&](const float (&x)[Row<T>::V], int) {
#pragma unroll
                for (int e = 0; e < Row<T>::V; e++) best = max_nan(best, x[e]);
            });
        else row.each_in(s, lane, [&](float x, int) {
            best = max_nan(best, x);
            if (SUMS) { mass += weight(x); least = fminf(least, x); }
            if (COUNTS) {
                const int b = grid.raw(x);
                if (b < Grid::BASE + BINS - 1) atomicAdd(&sh.hist[b - Grid::BASE], 1u);
            }
        });
        const uint32_t key = __reduce_max_sync(0xFFFFFFFFu, key_of(best));             // (the NaN of max.NaN has the largest key)
        top = max(top, key);
        uint32_t count = 0;
        if (SUMS) {
            mass = warp_sum(mass);
            count = SUB * Row<T>::V;
            const float bottom = sh.prm.u < 1e-260 ? weight.floor + 60.f * sh.prm.temperature : NEG_INF;
            if (__any_sync(0xFFFFFFFFu, least <= bottom)) {                            // masked entries, or the row's ends: count
                uint32_t mine = 0;
                row.each_in(s, lane, [&](float x, int) {
                    mine += x > NEG_INF ? 1u : 0u;
                    if (x > NEG_INF && x <= bottom) sh.low = 1;
                });
                count = warp_sum(mine);
                if (count == 0) mass = 0.0;            // masked as a whole: none of it can be drawn
            }
        }
        if (tops) tops[s] = key;
        if (SUMS && lane == 0) { all.mass[s] = mass; all.count[s] = count; }
    }
    return top;
}

// A list of at most 32 Q entries, finished by one warp, Q entries per lane.  `mass`: what top-p refers to, or negative:
// the first top_k entries' (weights are then taken from the list's own maximum).
template <typename T, int Q>
__device__ __forceinline__ void finish_small(const Args& a, int64_t step, Work<T>& k, const Weight& weight, int m, bool use_p, double mass,
                                             float minimum)
{
    Shared& sh = k.sh;
    const int lane = k.lane;
    const Params& prm = sh.prm;
    unsigned long long e[Q];
    int rank[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) { e[q] = lane + 32 * q < m ? sh.list[lane + 32 * q] : ~0ull; rank[q] = 0; }
#pragma unroll 2
    for (int j = 0; j < m; j++) {
        const unsigned long long o = sh.list[j];
#pragma unroll
        for (int q = 0; q < Q; q++) rank[q] += o < e[q] ? 1 : 0;
    }
#pragma unroll
    for (int q = 0; q < Q; q++) if (lane + 32 * q < m) sh.moved[rank[q]] = e[q];
    __syncwarp();
    const bool self = mass < 0.0;
    if (self && prm.top_k > 0) m = min(m, prm.top_k);
    double w[Q], run = 0.0;
    float x[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int r = lane * Q + q;
        w[q] = 0.0;
        if (r < m) {
            e[q] = sh.moved[r];
            x[q] = value_of(~(uint32_t)(e[q] >> 32));
            w[q] = self ? weight.of_gap((double)x[q] - (double)k.M) : weight(x[q]);
        }
        run += w[q];
    }
    double reached = warp_scan(run, lane);
    if (self) mass = __shfl_sync(0xFFFFFFFFu, reached, 31);
    const double target = (double)prm.top_p * mass;
    reached -= run;
    int end = NONE, cut = NONE;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int r = lane * Q + q;
        reached += w[q];
        if (r < m) {
            if (end == NONE && reached >= target) end = r + 1;
            if (cut == NONE && x[q] < minimum) cut = r;
        }
    }
    end = __reduce_min_sync(0xFFFFFFFFu, end);
    cut = __reduce_min_sync(0xFFFFFFFFu, cut);
    if (use_p) m = min(m, end);
    m = min(m, cut);
    // in index order
    __syncwarp();
#pragma unroll
    for (int q = 0; q < Q; q++) rank[q] = 0;
#pragma unroll 2
    for (int j = 0; j < m; j++) {
        const uint32_t o = (uint32_t)sh.moved[j];
#pragma unroll
        for (int q = 0; q < Q; q++) rank[q] += o < (uint32_t)e[q] ? 1 : 0;
    }
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (lane * Q + q < m) { sh.list[rank[q]] = e[q] & 0xFFFFFFFFull; sh.list_w[rank[q]] = w[q]; }
    __syncwarp();
    run = 0.0;
#pragma unroll
    for (int q = 0; q < Q; q++) { const int r = lane * Q + q; w[q] = r < m ? sh.list_w[r] : 0.0; run += w[q]; }
    double sum = warp_scan(run, lane);
    const double total = __shfl_sync(0xFFFFFFFFu, sum, 31), aim = prm.u * total;
    sum = lanes_before(sum, lane);
    int drawn = NONE, last = -1;               // last: where the sum grows for the last time, if rounding hides the entry
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const double next = sum + w[q];        // (nothing behind the m-th)
        if (drawn == NONE && next > sum) {
            last = lane * Q + q;
            if (next > aim) drawn = last;
        }
        sum = next;
    }
    drawn = __reduce_min_sync(0xFFFFFFFFu, drawn);
    if (drawn == NONE) drawn = __reduce_max_sync(0xFFFFFFFFu, last);
    if (lane == 0) answer(a, step, (int)sh.list[drawn], log(sh.list_w[drawn] / total), (uint32_t)m);
}

template <typename T>
__global__ void __launch_bounds__(NT, BLOCKS_PER_SM)
sample_kernel(const Args a, int per_block)
{
    extern __shared__ uint4 dynamic_shared[];
    Shared& sh = *reinterpret_cast<Shared*>(dynamic_shared);
    constexpr int V = Vec<T>::V;
    cg::cluster_group cluster = cg::this_cluster();
    Work<T> k{{}, sh, {}, cluster};
    k.nc = (int)cluster.num_blocks(); k.c = (int)cluster.block_rank();
    k.tid = threadIdx.x; k.lane = k.tid & 31; k.warp = k.tid >> 5;
    k.flip = 0; k.hflip = 0;
    const int tid = k.tid, lane = k.lane, warp = k.warp, c = k.c, nc = k.nc;
    // the other blocks' shared memory may be used once they have begun: asked for here, waited for before pass 1
    if (nc > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;");
    const int64_t step = blockIdx.x / nc;
    Row<T>& row = k.row;
    const char* p = (const char*)a.logits + step * a.ld * (int64_t)sizeof(T);
    row.shift = (int)(((uintptr_t)p & 15) / sizeof(T));
    row.stream = (const uint4*)((uintptr_t)p & ~(uintptr_t)15);
    row.n = (int)a.n;
    row.nv = (row.shift + row.n + V - 1) / V;
    const int nsub = (row.nv + SUB - 1) / SUB;
    row.s0 = min(nsub, c * per_block);
    row.s1 = min(nsub, row.s0 + per_block);
    {
        double* d = reinterpret_cast<double*>(&sh + 1);
        k.subs.mass = d; k.subs.kept = d + nsub;
        uint32_t* u = reinterpret_cast<uint32_t*>(d + 2 * nsub);
        k.subs.count = u; k.subs.kept_count = u + nsub; k.subs.top = u + 2 * nsub;
    }
    const Subs all{k.at(k.subs.mass, 0), k.at(k.subs.kept, 0), k.at(k.subs.count, 0), k.at(k.subs.kept_count, 0), k.subs.top};

    // ---- a sample of the row (used where weights or bins are needed), and the row's parameters
    const int at = row.nv <= NT ? tid : (int)((int64_t)tid * row.nv / NT);
    uint4 sampled = make_uint4(0, 0, 0, 0);
    if (at < row.nv) sampled = row.raw(at);
    if (tid == 0) {
        Params q;
        q.temperature = a.temperature_row ? a.temperature_row[step] : a.temperature;
        q.top_p = a.top_p_row ? a.top_p_row[step] : a.top_p;
        q.min_p = a.min_p_row ? a.min_p_row[step] : a.min_p;
        q.top_k = a.top_k_row ? a.top_k_row[step] : a.top_k;
        q.u = a.u[step];
        int f = 0;
        if (q.temperature >= 0.f && q.temperature < INFINITY && q.top_p > 0.f && q.min_p >= 0.f && q.min_p <= 1.f && q.u >= 0.0 && q.u < 1.0)
            f = FINE;                          // (not with a NaN in any of them)
        if (!(q.temperature > 0.f)) { f |= GREEDY; q.temperature = 1.f; }
        else {
            if (q.top_k > 0 && q.top_k < row.n) {
                f |= USE_K;
                // the sub-chunks' maxima bound a top-k that is below their number: some two thirds of it, or twice it, are above
                if (row.n <= SHORT) f |= TOPS;
                else if (nsub <= NT && q.top_k <= nsub - nsub / 8) f |= TOPS;
                else f |= q.top_k > LIST - 64 ? LONG_K : HIST;
            }
            if (q.top_p < 1.f) f |= f & USE_K ? USE_P : row.n <= SHORT ? USE_P | TOPS : USE_P | HIST | MASS;   // (of the top-k entries' mass, or of all)
            else if (!(f & USE_K) && q.min_p == 0.f) f |= MASS;
        }
        q.min_gap = -INFINITY;
        if (q.min_p > 0.f) q.min_gap = (double)q.temperature * log((double)q.min_p);
        q.factor = 23.083120654223414219 / (double)q.temperature;
        sh.prm = q;
        sh.flags = f & FINE ? f : f & GREEDY;
        sh.list_count = 0; sh.hits = 0; sh.low = 0; sh.answer_i = -1;
    }
    if (tid >= 32 && tid < 48) sh.table[tid - 32] = exp2((double)(tid - 32) * 0.0625);
    {
        uint4* h = reinterpret_cast<uint4*>(sh.hist) + 2 * tid;
        h[0] = h[1] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    const Params& prm = sh.prm;
    const int flags = sh.flags;
    const float t = prm.temperature;
    bool general = flags & LONG_K;
    float M0 = 0.f;
    Weight weight;
    weight.set(0.f, prm, sh.table);
    Grid grid{0.f, 1.f};
    if (flags & (MASS | HIST)) {
        float x[V], x0 = NEG_INF;
        int seen = 0;
        if (at < row.nv) {
            Vec<T>::unpack(sampled, x);
#pragma unroll
            for (int e = 0; e < V; e++) { x0 = fmaxf(x0, x[e]); seen += x[e] > NEG_INF ? 1 : 0; }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, o));
        seen = __reduce_add_sync(0xFFFFFFFFu, seen);
        if (lane == 0) { sh.warp_f[warp] = x0; sh.warp_u[1][warp] = (uint32_t)seen; }
        __syncthreads();
        // the largest of the warps' maxima, and the middle one of those that are finite
        const float mine = lane < NW ? sh.warp_f[lane] : NEG_INF;
        int rank = 0, alive = 0;
        uint32_t finite_seen = 0;
        float lowest = INFINITY;
        M0 = NEG_INF;
#pragma unroll
        for (int w = 0; w < NW; w++) {
            const float o = sh.warp_f[w];
            M0 = fmaxf(M0, o);
            if (o > NEG_INF) lowest = fminf(lowest, o);
            finite_seen += sh.warp_u[1][w];
            alive += o > NEG_INF ? 1 : 0;
            rank += (o > mine || (o == mine && w < lane)) ? 1 : 0;
        }
        const unsigned who = __ballot_sync(0xFFFFFFFFu, lane < NW && rank == alive / 2);
        float middle = __shfl_sync(0xFFFFFFFFu, mine, who ? __ffs(who) - 1 : 0);
        if (!(M0 > NEG_INF) || !(M0 < INFINITY)) M0 = middle = lowest = 0.f;
        float spread = M0 - middle;
        if (!(spread >= 0.f && spread < 1e30f)) spread = 0.f;
        weight.set(M0, prm, sh.table);
        if (fabs((double)M0 * weight.factor) > 1e12) general = true;       // (weights would lose their last bits)
        // Bins.  For normally spread values the sample's maximum lies some 3.3 deviations above the middle and a warp's
        // about 2.5, the lowest of the warps' 2: by count the largest entries are enough, eight times the distance to the
        // lowest (or four times the one to the middle, where a mask's values are lowest); by mass 20 T or, if less, 24 times the distance to the lowest one.
        const float finite = (float)finite_seen / (float)(min(row.nv, NT) * V) * (float)row.n;         // entries not masked
        float range = flags & USE_K ? ((float)prm.top_k * 8.f > finite ? 24.f : 8.f) * (spread > 0.f ? fminf(4.f * spread, M0 - lowest) : M0 - lowest) : fminf(20.f * t, 24.f * (M0 - lowest));
        if (!(range > 0.f)) range = flags & USE_K ? 1.f : fminf(20.f * t, 1e30f);
        grid.scale = fmaxf(fminf((float)BINS / range, 1e30f), 1e-30f);
        grid.c = rintf((M0 + 0.15f * range) * grid.scale);
        if (!(fabsf(grid.c) < 4e6f)) { grid.c = 0.f; grid.scale = 1.f; if (flags & HIST) general = true; }    // values far larger than their spread
    }

    // ---- pass 1
    if (nc > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    uint32_t top;
    switch (flags & (MASS | HIST)) {
    case MASS | HIST: top = first_pass<T, true, true>(k, all, weight, grid); break;
    case MASS: top = first_pass<T, true, false>(k, all, weight, grid); break;
    case HIST: top = first_pass<T, false, true>(k, all, weight, grid); break;
    default: top = first_pass<T, false, false>(k, all, weight, grid); break;
    }
    __syncthreads();
    if (lane == 0) sh.warp_u[0][warp] = top;
    __syncthreads();
    if (tid < nc) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < NW; w++) m = max(m, sh.warp_u[0][w]);
        k.of(tid)->tops[c] = m;
        k.of(tid)->lows[c] = sh.low;
    }
    k.sync_all();
    bool deep = false;                         // a finite entry near the floor, for a number u that it matters to
    {
        uint32_t m = 0;
        for (int b = 0; b < nc; b++) { m = max(m, sh.tops[b]); deep |= sh.lows[b] != 0; }
        k.M = m > key_of(INFINITY) ? NAN : value_of(m);
    }
    const float M = k.M;
    if (!(flags & FINE) || !(M > NEG_INF) || !(M < INFINITY)) {
        if (c == 0 && tid == 0) { a.token[step] = -1; a.logprob[step] = NAN; a.kept[step] = 0; a.status[step] = IMM_ERR_ARG; }
        return;
    }
    const bool use_k = flags & USE_K, use_p = flags & USE_P;

    if (flags & GREEDY) {                      // the lowest index of the maximum: the first sub-chunk that has it
        if (c == 0) {
            const uint32_t key = key_of(M);
            int s = NONE;
            for (int i = nsub - 1 - tid; i >= 0; i -= NT) if (all.top[i] == key) s = i;
            s = k.first_of(s, nsub - 1);
            int first = NONE;
            const int v = s * SUB + tid;
            if (v < row.nv) {
                float x[V];
                Vec<T>::unpack(row.raw(v), x);
#pragma unroll
                for (int e = V - 1; e >= 0; e--) if (x[e] == M) first = v * V - row.shift + e;
            }
            first = k.first_of(first, NONE);
            if (tid == 0) answer(a, step, first, 0.0, 1);
        }
        return;
    }

    if (flags & MASS) {
        // Weights relative to M0 have to hold M's (650 T above it at most).  M lies below M0 only where the sample saw
        // nothing but masked entries and M0 is 0: 60 T below it M still weighs e^630 times what an entry at the floor does.  For
        // the smallest u, 60 T above it: what weighs something beside M0 weighs something beside M then.
        const double above = ((double)M - (double)M0) * weight.factor;     // in 16 log2(e)
        if (above > (prm.u < 1e-260 ? 1385.0 : 15000.0) || above < -1385.0) general = true;
    } else {
        weight.set(M, prm, sh.table);
        if (fabs((double)M * weight.factor) > 1e12) general = true;
    }
    // From temperatures of 5e35 on the floor would lie below the lowest value, which weighs too much then.
    if (!use_k && !(flags & TOPS) && (deep || !(weight.floor > LOWEST))) general = true;
    float X = LOWEST;                          // the prefix: x > X, or x == X and index <= I
    int I = NONE;
    float minimum = LOWEST;                    // the smallest value that min-p leaves
    if (!general && prm.min_p > 0.f) minimum = k.min_p_value(prm.min_gap);

    // What pass 2 does: entries over `sure` are kept and added up, those from `low` to `sure` go to the list.
    float low = LOWEST, sure = INFINITY;
    double target = 0.0, whole = -1.0;
    bool second = false, by_list = false, whole_list = false;
    if (general) {
    } else if (flags & TOPS) {
        if (row.n > SHORT) {                   // the top_k-th largest of the sub-chunks' maxima; short rows go to the list whole
            uint32_t* tops = sh.hist;              // (not used by this kind of row)
            const uint32_t mine = tid < nsub ? all.top[tid] : 0u;
            tops[tid] = mine;
            __syncthreads();
            int rank = 0;
            for (int j = 0; j < nsub; j += 4) {
                const uint4 o = *reinterpret_cast<const uint4*>(tops + j);     // (0 behind the last)
                rank += (o.x > mine || (o.x == mine && j < tid)) + (o.y > mine || (o.y == mine && j + 1 < tid)) +
                        (o.z > mine || (o.z == mine && j + 2 < tid)) + (o.w > mine || (o.w == mine && j + 3 < tid));
        }
            if (tid < nsub && rank == prm.top_k - 1) sh.edge[0] = mine;
            __syncthreads();
            low = value_of(max(sh.edge[0], key_of(LOWEST)));
        }
        second = by_list = whole_list = true;
    } else if (!(flags & HIST)) {
        if (prm.min_p > 0.f) {                 // min-p alone: the prefix is known
            second = true;
            X = low = minimum;
        }
    } else {
        uint32_t mine[BPT] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
        for (int b = 0; b < nc; b++) {
            const uint4* h = reinterpret_cast<const uint4*>(k.of(b)->hist) + 2 * tid;
            const uint4 h0 = h[0], h1 = h[1];
            mine[0] += h0.x; mine[1] += h0.y; mine[2] += h0.z; mine[3] += h0.w;
            mine[4] += h1.x; mine[5] += h1.y; mine[6] += h1.z; mine[7] += h1.w;
        }
        uint32_t part = 0, held;
#pragma unroll
        for (int q = 0; q < BPT; q++) part += mine[q];
        const uint32_t before = k.scan_u(part, &held) - part;
        int b1 = 0, b2;                        // the undecided bins: entries in bins before b1 are kept, behind b2 are not
        uint32_t finite = 0;
        if (use_k) {
            int found = NONE;
            uint32_t cum = before;
#pragma unroll
            for (int q = 0; q < BPT; q++) { cum += mine[q]; if (found == NONE && cum >= (uint32_t)prm.top_k) found = tid * BPT + q; }
            b2 = k.first_of(found, BINS);
        } else {
            double m = 0.0;                    // the row's mass: in an order that does not depend on the cluster
            for (int s = tid; s < nsub; s += NT) { m += all.mass[s]; finite += all.count[s]; }
            k.scan_d(m, 0, &whole);
            k.scan_u(finite, &finite);
            target = (double)prm.top_p * whole;
            // A bin's mass lies between its count times the weights at its edges; a few units of float32's last place are
            // left for the exponentials.  Prefix sums from the top, and the whole less the sums from the bottom; what the
            // last bin would hold was not counted: its weights are at most those at its upper edge.
            const double width = 1.0 / (double)grid.scale, octave = weight.factor * 0.0625;
            const double base = ((double)grid.c + 0.5) * width * octave + (weight.bias - 6755399441055744.0) * 0.0625;
            auto edge = [&](int b) { return (double)exp2f((float)(base - (double)b * width * octave)); };      // at bin b's upper edge
            double hi[BPT], lo[BPT], hi_sum = 0.0, lo_sum = 0.0, upper = edge(tid * BPT);
            if (tid == 0) upper = weight(M) * (1.0 + 1e-5);    // (the first bin has no other upper edge)
#pragma unroll
            for (int q = 0; q < BPT; q++) {
                const double lower = edge(tid * BPT + q + 1);
                hi[q] = mine[q] ? (double)mine[q] * (upper * (1.0 + 2e-5)) : 0.0;
                lo[q] = mine[q] ? (double)mine[q] * (lower * (1.0 - 2e-5)) : 0.0;
                hi_sum += hi[q]; lo_sum += lo[q];
                upper = lower;
            }
            double hi_all, lo_all;
            double hi_run = k.scan_d(hi_sum, 0, &hi_all) - hi_sum, lo_run = k.scan_d(lo_sum, 1, &lo_all) - lo_sum;
            const double below = (double)(finite - held) * edge(BINS - 1) * (1.0 + 2e-5), slack = 1e-11 * whole;
            int f1 = NONE, f2 = NONE;
#pragma unroll
            for (int q = 0; q < BPT; q++) {
                hi_run += hi[q]; lo_run += lo[q];
                // the prefix up to this bin: at most / at least
                const double most = fmin(hi_run, whole - (lo_all - lo_run)) + slack;
                const double least = fmax(lo_run, whole - (hi_all - hi_run) - below) - slack;
                if (f1 == NONE && most >= target) f1 = tid * BPT + q;
                if (f2 == NONE && least >= target) f2 = tid * BPT + q;
            }
            b1 = k.first_of(f1, BINS);
            b2 = k.first_of(f2, BINS);
        }
        if (b2 >= BINS - 1) general = true;    // not within the bins
        else {
            // entries in the bins up to b2, and before b1
            __syncthreads();
            uint32_t cum = before;
#pragma unroll
            for (int q = 0; q < BPT; q++) {
                if (tid * BPT + q == b1) sh.before_u = cum;
                cum += mine[q];
                if (tid * BPT + q == b2) sh.sum_u = cum;
            }
            __syncthreads();
            const uint32_t upto = sh.sum_u, above = sh.before_u;
            if (upto <= LIST) {                // the whole prefix fits the list
                second = by_list = whole_list = true;
                b1 = 0;
                if (!use_k && upto == finite) whole = -1.0;    // so does the row: its mass is taken from the list
            } else if (use_k || upto - above > LIST) general = true;
            else {
                second = true;
                by_list = !(minimum > LOWEST && grid.of(minimum) < b1);
                if (!by_list) X = low = minimum;               // min-p alone decides
            }
            if (by_list) {
                uint32_t khi, klo;
                k.bin_edges(grid, b1, b2, khi, klo);
                low = value_of(klo);
                if (!whole_list) sure = value_of(khi);
            }
        }
    }
    if (second && !by_list) {
        const uint32_t key = key_of(low);      // entries >= low: over the value below it (no key is -0's)
        sure = value_of(key - (key == 0x80000000u ? 2u : 1u));
    }

    // ---- pass 2
    Shared* s0 = k.of(0);
    if (second && !general) {
        const uint32_t low_key = key_of(low);
        // entries of a sub-chunk for the list: a bit per entry of the lane, one reservation for the warp
        auto append = [&](int s, uint64_t hits) {
            const uint32_t mine = (uint32_t)__popcll(hits), upto = warp_scan(mine, lane);
            const uint32_t count = __shfl_sync(0xFFFFFFFFu, upto, 31);
            if (!count) return;
            uint32_t slot = 0;
            if (lane == 31) { slot = atomicAdd(&s0->list_count, count); atomicAdd(&sh.hits, count); }
            slot = __shfl_sync(0xFFFFFFFFu, slot, 31) + upto - mine;
            while (hits) {
                const int bit = __ffsll((long long)hits) - 1;
                hits &= hits - 1;
                const int i = (s * SUB + 32 * (bit / V) + lane) * V + bit % V - row.shift;
                if (slot < LIST) s0->list[slot] = ((unsigned long long)(~key_of(row.entry(i))) << 32) | (uint32_t)i;
                slot++;
            }
        };
        for (int s = row.s0 + warp; s < row.s1; s += NW) {
            const bool visit = k.subs.top[s] >= low_key;
            uint64_t hits = 0;
            double mass = 0.0;
            uint32_t count = 0;
            if (visit && whole_list) {
                row.vectors_at_once(s, lane, [&](const float (&x)[V], int j) {
                    unsigned listed = 0;
#pragma unroll
                    for (int e = 0; e < V; e++) listed |= x[e] >= low ? 1u << e : 0u;
                    hits |= (uint64_t)listed << (j * V);
                });
            } else if (visit) {
                // (Stacking a lane's kept values to take only their weights cost more than the weights saved: 65 against 51
                // thousand cycles a row, at a fifth of the entries kept.)
                int bit = 0;
                row.vectors(s, lane, [&](const float (&x)[V], int) {
                    unsigned taken = 0, listed = 0;
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const bool take = x[e] > sure;
                        mass += weight(take ? x[e] : LOWEST);  // (the weight of LOWEST is e^-690 of the reference's at most)
                        taken |= take ? 1u << e : 0u;
                        listed |= x[e] >= low ? 1u << e : 0u;
                    }
                    count += __popc(taken);
                    hits |= (uint64_t)(listed & ~taken) << bit;
                    bit += V;
                });
                mass = warp_sum(mass); count = warp_sum(count);
                if (count == 0) mass = 0.0;            // (entries not taken have added the weight of LOWEST)
            }
            if (by_list && visit) append(s, hits);
            if (!whole_list && lane == 0) { all.kept[s] = mass; all.kept_count[s] = count; }
        }
        if (flags & TOPS) {                    // every block's number of entries, to every block: more than the list holds?
            __syncthreads();
            if (tid < nc) k.of(tid)->listed[c] = sh.hits;
        }
        k.sync_all();
        if (flags & TOPS) {
            uint32_t n = 0;
            for (int b = 0; b < nc; b++) n += sh.listed[b];
            general = n > LIST;                // (ties at the bound)
        }
    }
    if (general) {
        Work<T> own = k;                       // (a copy: what a function takes by reference lives in memory)
        general_row<T>(a, step, own, prm);
        if (nc > 1) cluster.sync();            // nobody leaves while another block reads its shared memory
        return;
    }
    if (c != 0) return;                        // (nothing of this block is read any more)

    // ---- block 0: masses and counts of the sub-chunks, a few neighbours per thread
    if (whole_list && sh.list_count <= SMALL) {
        if (warp == 0) {
            const int n = (int)sh.list_count;
            if (n <= 32) finish_small<T, 1>(a, step, k, weight, n, use_p, use_k ? -1.0 : whole, minimum);
            else finish_small<T, SMALL / 32>(a, step, k, weight, n, use_p, use_k ? -1.0 : whole, minimum);
        }
        return;
    }
    constexpr int SPT = (MAX_SUB + NT - 1) / NT;
    const int spt = (nsub + NT - 1) / NT;      // one for rows of up to 256 of them
    double sub_mass[SPT], mass_sum = 0.0;
    uint32_t count_sum = 0;
#pragma unroll
    for (int q = 0; q < SPT; q++) {
        const int s = tid * spt + q;
        sub_mass[q] = 0.0;
        if (q < spt && s < nsub && !whole_list) {
            sub_mass[q] = second ? all.kept[s] : all.mass[s];
            count_sum += second ? all.kept_count[s] : all.count[s];
        }
        mass_sum += sub_mass[q];
    }
    int m = 0;                                 // kept entries of the list
    if (by_list) {
        double sure_mass = 0.0;
        if (!whole_list) k.scan_d(mass_sum, 0, &sure_mass);
        m = (int)min(sh.list_count, (uint32_t)LIST);
        const bool self = use_k || whole < 0.0;
        k.sort_list(m);
        if (use_k) m = min(m, prm.top_k);
        double w[LPT], run = 0.0;              // neighbours of the list per thread
#pragma unroll
        for (int q = 0; q < LPT; q++) {
            const int r = tid * LPT + q;
            w[q] = 0.0;
            if (r < m) {
                const float x = value_of(~(uint32_t)(sh.list[r] >> 32));
                w[q] = self ? weight.of_gap((double)x - (double)M) : weight(x);
            }
            run += w[q];
        }
        double all_w;
        double reached = k.scan_d(run, 1, &all_w) - run + sure_mass;
        if (self) target = (double)prm.top_p * all_w;
        int end = NONE, cut = NONE;
#pragma unroll
        for (int q = 0; q < LPT; q++) {
            const int r = tid * LPT + q;
            reached += w[q];
            if (r < m) {
                if (end == NONE && reached >= target) end = r + 1;
                if (cut == NONE && value_of(~(uint32_t)(sh.list[r] >> 32)) < minimum) cut = r;
            }
        }
        if (use_p) m = k.first_of(end, m);
        // (X, I) is the last entry that top-p keeps, unless min-p cuts before it
        const unsigned long long edge = sh.list[m - 1];
        X = value_of(~(uint32_t)(edge >> 32)); I = (int)(uint32_t)edge;
        if (prm.min_p > 0.f) {
            m = k.first_of(cut, m);
            if (minimum > X) { X = minimum; I = NONE; }
        }
        // the kept ones in index order, with the running sum of their weights
        unsigned long long by_index[LPT];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < LPT; q++) {
            const int r = tid * LPT + q;
            by_index[q] = r < m ? ((sh.list[r] & 0xFFFFFFFFull) << 32) | (uint32_t)r : 0ull;
            if (r < m) sh.list_w[r] = w[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < LPT; q++) if (tid * LPT + q < m) sh.list[tid * LPT + q] = by_index[q];
        k.sort_list(m);
        run = 0.0;
#pragma unroll
        for (int q = 0; q < LPT; q++) {
            const int r = tid * LPT + q;
            w[q] = r < m ? sh.list_w[(uint32_t)sh.list[r]] : 0.0;
            run += w[q];
        }
        double total;
        double sum = k.before_d(run, 0, &total);
        if (whole_list) {                      // nothing but the list
            const double aim = prm.u * total;
            int drawn = NONE, last = -1;       // last: where the sum grows for the last time, if rounding hides the entry
#pragma unroll
            for (int q = 0; q < LPT; q++) {
                const double next = sum + w[q];                            // (nothing behind the m-th)
                if (drawn == NONE && next > sum) {
                    last = tid * LPT + q;
                    if (next > aim) drawn = last;
                }
                sum = next;
            }
            drawn = k.first_of(drawn, NONE);
            if (drawn == NONE) drawn = -k.first_of(last >= 0 ? -last : 1, 1);
#pragma unroll
            for (int q = 0; q < LPT; q++)
                if (tid * LPT + q == drawn) answer(a, step, (int)(sh.list[drawn] >> 32), log(w[q] / total), (uint32_t)m);
            return;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < LPT; q++) {
            sum += w[q];
            if (tid * LPT + q < m) sh.list_w[tid * LPT + q] = sum;         // inclusive, by position in index order
        }
        __syncthreads();
        // the list's share of every sub-chunk
        auto upto = [&](int border) -> double {                            // weight of the list's entries before index `border`
            int lo = 0, hi = m;
            while (lo < hi) { const int mid = (lo + hi) >> 1; if ((int)(sh.list[mid] >> 32) < border) lo = mid + 1; else hi = mid; }
            return lo ? sh.list_w[lo - 1] : 0.0;
        };
        mass_sum = 0.0;
        double from = tid * spt < nsub ? upto(tid * spt * SUB * V - row.shift) : 0.0;
#pragma unroll 1
        for (int q = 0; q < spt; q++) {
            const int s = tid * spt + q;
            if (s < nsub) {
                const double to = upto((s + 1) * SUB * V - row.shift);
#pragma unroll
                for (int z = 0; z < SPT; z++) if (z == q) { sub_mass[z] += to - from; mass_sum += sub_mass[z]; }
                from = to;
            }
        }
    }
    // ---- the draw: the sub-chunk, then the entry
    double total;
    uint32_t kept;
    double run = k.before_d(mass_sum, 1, &total);
    k.scan_u(count_sum, &kept);
    const double aim = prm.u * total;
    int hit = NONE, last = -1;                 // the first sub-chunk that passes the aim; the last one at which the sum grows
    double before = 0.0;                       // the sum before the former, or else the latter
#pragma unroll
    for (int q = 0; q < SPT; q++) {
        const double next = run + sub_mass[q];
        if (hit == NONE && next > run) {
            last = tid * spt + q; before = run;
            if (next > aim) hit = last;
        }
        run = next;
    }
    int s = k.first_of(hit, NONE);
    if (s == NONE) {                           // rounding hides it
        s = -k.first_of(last >= 0 ? -last : 1, 1);
        hit = last;
    }
    __syncthreads();
    if (hit == s) sh.before_d = before;
    __syncthreads();
    before = sh.before_d;
    draw_in_sub<T>(a, step, k, weight, s, X, I, before, aim, total, kept + (uint32_t)m);
}

template <typename T>
cudaError_t launch(const Args& a, int64_t steps, cudaStream_t st)
{
    constexpr int V = Vec<T>::V;
    const int64_t nv = (a.n + 2 * V - 2) / V;              // vectors of a row, wherever it begins
    const int nsub = (int)((nv + SUB - 1) / SUB);
    auto kernel = sample_kernel<T>;
    // once per device: permission for the shared memory and for large clusters, and the largest cluster it can hold
    static std::atomic<int> largest[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    int most = dev < 64 ? largest[dev].load(std::memory_order_relaxed) : 0;
    if (most == 0) {
        const int bytes = (int)(sizeof(Shared) + subs_bytes(MAX_SUB));
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t ask;
        memset(&ask, 0, sizeof(ask));
        ask.gridDim = dim3(MAX_CLUSTER);
        ask.blockDim = dim3(NT);
        ask.dynamicSmemBytes = (size_t)bytes;
        e = cudaOccupancyMaxPotentialClusterSize(&most, kernel, &ask);
        if (e != cudaSuccess) return e;
        most = most >= MAX_CLUSTER ? MAX_CLUSTER : most >= 8 ? 8 : 1;
        if (dev < 64) largest[dev].store(most, std::memory_order_relaxed);
    }
    // Blocks per row: more while the rows leave places on the GPU and every warp still has a sub-chunk, and where the
    // rows in flight would outgrow L2 between the two passes.  Rows of one pass are all alike: two blocks for a place
    // even out the SMs (512 x 151936 bf16: 114 us against 127 with one; rows with filters differ, 66 us against 74).
    const int64_t slots = (int64_t)BLOCKS_PER_SM * imm::sm_count();
    const bool one_pass = !a.top_k_row && !a.top_p_row && !a.min_p_row && a.top_k <= 0 && a.top_p >= 1.f && a.min_p == 0.f;
    int nc = 1;
    while (nc < most && nsub > nc * NW &&
           (steps * nc * 2 <= (one_pass ? 2 : 1) * slots || (!one_pass && nc < 8 && slots / nc * nv * 16 > ((int64_t)80 << 20)))) nc *= 2;
    const int per = (nsub + nc - 1) / nc;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(steps * nc));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = sizeof(Shared) + subs_bytes(nsub);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    memset(&attr, 0, sizeof(attr));
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)nc;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, per);
}

}  // namespace imm_sample_ns

extern "C" int imm_sample(const imm_sample_desc* desc_host, void* stream)
{
    using namespace imm_sample_ns;
    if (!desc_host || desc_host->reserved) return IMM_ERR_ARG;
    const imm_sample_desc& d = *desc_host;
    if (d.steps > 0 && (!d.d_logits || !d.d_u || !d.d_token || !d.d_logprob || !d.d_kept || !d.d_status)) return IMM_ERR_ARG;
    if (d.dtype != IMM_F32 && d.dtype != IMM_BF16 && d.dtype != IMM_F16) return IMM_ERR_ARG;
    if (d.steps < 0 || d.n <= 0 || d.ld < d.n || d.n > IMM_LDD_MAX_N || d.steps > IMM_LDD_MAX_STEPS) return IMM_ERR_SHAPE;
    if ((uintptr_t)d.d_logits % (d.dtype == IMM_F32 ? 4 : 2) || (uintptr_t)d.d_u % 8 || (uintptr_t)d.d_token % 4 || (uintptr_t)d.d_logprob % 4 ||
        (uintptr_t)d.d_kept % 4 || (uintptr_t)d.d_status % 4 || (uintptr_t)d.d_temperature % 4 || (uintptr_t)d.d_top_k % 4 ||
        (uintptr_t)d.d_top_p % 4 || (uintptr_t)d.d_min_p % 4)
        return IMM_ERR_ALIGN;
    if (d.steps == 0) return IMM_OK;
    Args a{};
    a.logits = d.d_logits; a.n = d.n; a.ld = d.ld; a.u = d.d_u;
    a.temperature_row = d.d_temperature; a.top_p_row = d.d_top_p; a.min_p_row = d.d_min_p; a.top_k_row = d.d_top_k;
    a.temperature = d.temperature; a.top_p = d.top_p; a.min_p = d.min_p; a.top_k = d.top_k;
    a.token = d.d_token; a.logprob = d.d_logprob; a.kept = d.d_kept; a.status = d.d_status;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == IMM_F32 ? launch<float>(a, d.steps, st)
                          : d.dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, d.steps, st) : launch<__half>(a, d.steps, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
