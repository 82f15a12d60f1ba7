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
// sums are held in 64 bits, added in an order that is fixed by the row's partition.
//
// A row is cut into slices, one per block of a thread-block cluster; a slice is read from HBM once and stays
// in shared memory (in the logits' own type) for the passes that follow.  Finding a prefix:
//   by count or by mass, coarse to fine: a histogram of the entries over 512 bins of the value (counts only:
//   integer atomics, whose order does not matter), merged over the cluster.  For a prefix that holds a share
//   of the mass, a bin's mass lies between its count times the weights at its two edges; that bounds the bins
//   in which the prefix can end.  Entries above those bins are certainly kept: their exact mass is added up in
//   the next pass, which also splits the remaining bins into 512 finer ones, until a single value is left.
//   Equal values are then taken in index order.
//   When only a short list of candidates is left (top-k with a small k, a confident row), it is gathered into
//   one block and finished there by ranking.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_sample_ns {

namespace cg = cooperative_groups;

constexpr int NT = 512;                        // threads per block
constexpr int NW = NT / 32;
constexpr int NB = NT;                         // histogram bins (one per thread in the scans)
constexpr int MAX_CLUSTER = 8;
constexpr int CAP = 512;                       // longest list that is finished by ranking (one entry per thread)
constexpr int SLICE_BYTES = 65536;             // of a row per block, before the cluster cap
constexpr int CACHE_MAX = 196608;              // shared memory a slice may take; longer rows are read again (from L2)
constexpr float SPAN = 24.f;                   // the first histogram covers weights down to e^-24
constexpr float NEG_INF = -INFINITY;

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
    int64_t per;                               // 16-byte vectors per slice
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
    static constexpr uint32_t LOWEST = 0xFF800000u;     // -inf
    __device__ static void mask(uint4& r, int e) { (&r.x)[e] = LOWEST; }
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

struct Publish { double mass; uint32_t count, ties; float top; uint32_t spare; };

struct Shared {
    uint32_t hist[2][NB];                      // this block's bins (two copies: the other blocks may still read the last one)
    Publish pub[2];                            // this block's share of a cluster-wide sum (two copies, likewise)
    double warp_d[2][NW];
    uint32_t warp_u[2][NW];
    float warp_f[NW];
    double sum_d, before_d;                    // cluster totals, and what the blocks before this one hold
    uint32_t sum_u, before_u, sum_t, before_t;
    int first_bin, last_bin, pick;
    uint32_t edge[2];
    // block 0: the short list
    uint32_t list_key[CAP];
    int32_t list_idx[CAP];
    uint32_t list_rank_key[CAP];
    int32_t list_rank_idx[CAP];
    double list_w[CAP];
    uint32_t list_count;
    int32_t answer_i;                          // an index found by one block, stored into every block
    double answer_d;
};

// ---- block-wide helpers (every thread of the block calls them) ----

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xFFFFFFFFu, v); }

template <typename T, bool CACHED>
struct Row {
    using VT = Vec<T>;
    static constexpr int V = VT::V;
    const uint4* stream;                       // the row's 16-byte vectors; the first may begin before the row
    const uint4* cache;                        // this block's slice of them in shared memory
    int shift;                                 // entries of the first vector that lie before the row
    int64_t n, v0, v1;                         // this block's vectors
    int64_t w0, w1;                            // this warp's

    __device__ __forceinline__ uint4 raw(int64_t v) const
    {
        uint4 r = __ldg(stream + v);
        const int64_t e0 = v * V - shift;
        if (e0 < 0 || e0 + V > n) {            // the row's first or last vector
            for (int e = 0; e < V; e++)
                if (e0 + e < 0 || e0 + e >= n) VT::mask(r, e);
        }
        return r;
    }
    __device__ __forceinline__ void get(int64_t v, float (&f)[V]) const
    {
        if (CACHED) VT::unpack(cache[v - v0], f);
        else VT::unpack(raw(v), f);
    }
    // calls f(value, index) for the entries of this warp's chunk, lanes side by side
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const
    {
        for (int64_t v = w0 + (threadIdx.x & 31); v < w1; v += 32) {
            float x[V];
            get(v, x);
            const int i0 = (int)(v * V - shift);
#pragma unroll
            for (int e = 0; e < V; e++) f(x[e], i0 + e);
        }
    }
};

template <typename T, bool CACHED>
__global__ void __launch_bounds__(NT)
sample_kernel(const Args a)
{
    extern __shared__ uint4 slice[];
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int nc = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
    const int64_t step = blockIdx.x / nc;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int V = Vec<T>::V;
    int flip = 0;                              // which copy of hist / pub is in use

    Row<T, CACHED> row;
    {
        const char* p = (const char*)a.logits + step * a.ld * (int64_t)sizeof(T);
        row.shift = (int)(((uintptr_t)p & 15) / sizeof(T));
        row.stream = (const uint4*)((uintptr_t)p & ~(uintptr_t)15);
        row.n = a.n;
        const int64_t nv = (row.shift + a.n + V - 1) / V;
        row.v0 = min(nv, (int64_t)c * a.per);
        row.v1 = min(nv, row.v0 + a.per);
        const int64_t chunk = (a.per + NW - 1) / NW;
        row.w0 = min(row.v1, row.v0 + warp * chunk);
        row.w1 = min(row.v1, row.w0 + chunk);
        row.cache = slice;
    }

    // ---- the slice into shared memory, and the row's maximum
    float best = NEG_INF;
    for (int64_t v = row.w0 + lane; v < row.w1; v += 32) {
        const uint4 r = row.raw(v);
        if (CACHED) slice[v - row.v0] = r;
        float f[V];
        Vec<T>::unpack(r, f);
#pragma unroll
        for (int e = 0; e < V; e++) best = max_nan(best, f[e]);
    }
    if (CACHED) __syncwarp();                  // a warp reads only what it stored itself
    const float thread_best = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max_nan(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
    if (lane == 0) sh.warp_f[warp] = best;
    sh.hist[0][tid] = 0; sh.hist[1][tid] = 0;
    if (tid == 0) { sh.list_count = 0; sh.answer_i = -1; sh.pick = -1; }
    __syncthreads();
    if (tid == 0) {
        float m = NEG_INF;
        for (int w = 0; w < NW; w++) m = max_nan(m, sh.warp_f[w]);
        sh.pub[flip].top = m;
    }
    cluster.sync();
    float M = NEG_INF;
    for (int b = 0; b < nc; b++) M = max_nan(M, cluster.map_shared_rank(&sh.pub[flip], b)->top);
    flip ^= 1;

    const float temperature = a.temperature_row ? a.temperature_row[step] : a.temperature;
    const float top_p = a.top_p_row ? a.top_p_row[step] : a.top_p;
    const float min_p = a.min_p_row ? a.min_p_row[step] : a.min_p;
    const int64_t top_k = a.top_k_row ? a.top_k_row[step] : a.top_k;
    const double u = a.u[step];
    const bool fine = M > NEG_INF && M < INFINITY && temperature >= 0.f && temperature < INFINITY && top_p > 0.f &&
                      min_p >= 0.f && min_p <= 1.f && u >= 0.0 && u < 1.0;            // (false for a NaN in any of them)
    if (!fine) {
        if (c == 0 && tid == 0) {
            a.token[step] = -1; a.logprob[step] = NAN; a.kept[step] = 0; a.status[step] = IMM_ERR_ARG;
        }
        cluster.sync();
        return;
    }

    const double m64 = (double)M, inv_t = 1.0 / (double)(temperature > 0.f ? temperature : 1.f);
    auto weight = [&](float x) { return exp(((double)x - m64) * inv_t); };
    // min-p on the logits: w >= min_p where x - M >= T log(min_p) (weights next to 1 would round to it)
    const double min_gap = min_p > 0.f ? (double)temperature * log((double)min_p) : -INFINITY;

    // Sums of (mass, count, ties) over the cluster: totals, and what the blocks and warps before hold.
    // Every thread returns with sh.sum_* and sh.before_* set; warp-level values stay in sh.warp_*[0..1].
    auto exchange = [&](double mass, uint32_t count, uint32_t ties) {
        mass = warp_sum(mass); count = warp_sum(count); ties = warp_sum(ties);
        __syncthreads();                       // (the last exchange's values have been read)
        if (lane == 0) { sh.warp_d[0][warp] = mass; sh.warp_u[0][warp] = count; sh.warp_u[1][warp] = ties; }
        __syncthreads();
        if (tid == 0) {
            double s = 0.0; uint32_t k = 0, t = 0;
            for (int w = 0; w < NW; w++) { s += sh.warp_d[0][w]; k += sh.warp_u[0][w]; t += sh.warp_u[1][w]; }
            sh.pub[flip].mass = s; sh.pub[flip].count = k; sh.pub[flip].ties = t;
        }
        cluster.sync();
        if (tid == 0) {
            double s = 0.0, sb = 0.0; uint32_t k = 0, kb = 0, t = 0, tb = 0;
            for (int b = 0; b < nc; b++) {
                const Publish p = *cluster.map_shared_rank(&sh.pub[flip], b);
                if (b == c) { sb = s; kb = k; tb = t; }
                s += p.mass; k += p.count; t += p.ties;
            }
            sh.sum_d = s; sh.before_d = sb; sh.sum_u = k; sh.before_u = kb; sh.sum_t = t; sh.before_t = tb;
        }
        __syncthreads();
        flip ^= 1;
    };
    // merged histogram: bin `tid` summed over the cluster (hist[hflip] of every block)
    int hflip = 0;
    auto merged_bin = [&]() -> uint32_t {
        cluster.sync();                        // (also a block barrier: every block's bins are complete)
        uint32_t s = 0;
        for (int b = 0; b < nc; b++) s += cluster.map_shared_rank(&sh.hist[hflip][0], b)[tid];
        hflip ^= 1;
        sh.hist[hflip][tid] = 0;               // the other copy was last read before this barrier
        __syncthreads();
        return s;
    };
    // inclusive scans over the block's threads
    auto scan_u = [&](uint32_t v) -> uint32_t {
        uint32_t s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
        __syncthreads();
        if (lane == 31) sh.warp_u[0][warp] = s;
        __syncthreads();
        for (int w = 0; w < warp; w++) s += sh.warp_u[0][w];
        return s;
    };
    auto scan_d = [&](double v, int slot) -> double {
        double s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const double t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
        __syncthreads();
        if (lane == 31) sh.warp_d[slot][warp] = s;
        __syncthreads();
        double before = 0.0;
        for (int w = 0; w < warp; w++) before += sh.warp_d[slot][w];
        return before + s;
    };
    auto first_true = [&](bool yes, int none) -> int {     // lowest thread for which `yes` holds, at most `none`
        __syncthreads();
        if (tid == 0) sh.pick = none;
        __syncthreads();
        if (yes) atomicMin(&sh.pick, tid);
        __syncthreads();
        return sh.pick;
    };

    // the first histogram's bins: linear in the value
    const float scale = fmaxf(fminf((float)NB / (SPAN * (temperature > 0.f ? temperature : 1.f)), 1e30f), 1e-30f);
    auto bin_of = [&](float x) -> int { return (int)fminf((M - x) * scale, (float)(NB - 1)); };
    // largest (smallest) key whose value falls into a bin >= b1 (<= b2): bins fall with rising keys
    auto bin_edges = [&](int b1, int b2, uint32_t& khi, uint32_t& klo) {
        __syncthreads();
        if (warp < 2) {
            // warp 0: the largest key with bin >= b1; warp 1: the smallest key with bin <= b2
            uint64_t lo = key_of(-3.402823466e+38f), hi = key_of(M);       // bin(hi) = 0; the answers lie in [lo, hi]
            while (lo < hi) {
                const uint64_t gap = hi - lo, stepk = gap / 32 + 1;
                const uint64_t probe = warp == 0 ? hi - min(gap, stepk * lane) : lo + min(gap, stepk * lane);
                const int b = bin_of(value_of((uint32_t)probe));
                const bool ok = warp == 0 ? b >= b1 : b <= b2;
                const unsigned hits = __ballot_sync(0xFFFFFFFFu, ok);      // monotone in the lane
                if (!hits) {                                               // beyond the last probe
                    const uint64_t last = __shfl_sync(0xFFFFFFFFu, probe, 31);
                    if (warp == 0) { if (last == lo) break; hi = last - 1; } else { if (last == hi) break; lo = last + 1; }
                } else {
                    const int f = __ffs(hits) - 1;
                    const uint64_t at = __shfl_sync(0xFFFFFFFFu, probe, f);
                    const uint64_t prev = __shfl_sync(0xFFFFFFFFu, probe, f > 0 ? f - 1 : 0);
                    if (warp == 0) { lo = at; hi = f > 0 ? prev - 1 : at; } else { hi = at; lo = f > 0 ? prev + 1 : at; }
                    if (f == 0) break;
                    // the answer lies in [lo, hi]: `at` itself or a key between it and the probe before
                }
            }
            if (lane == 0) sh.edge[warp] = (uint32_t)(warp == 0 ? hi : lo);
        }
        __syncthreads();
        khi = sh.edge[0]; klo = sh.edge[1];
    };

    // ---- the prefix that is left: x > X, or x == X and index <= I
    float X = NEG_INF;
    int I = 0x7FFFFFFF;
    auto inside = [&](float x, int i) { return x > X || (x == X && i <= I); };
    X = -3.402823466e+38f;                     // every finite entry

    // Index of the j-th (j >= 1) entry of value `x` in index order; `mine` ties in this thread's chunk, warp and
    // block totals as the last exchange left them.
    auto tie_index = [&](float x, uint32_t j) -> int {
        const bool here = j > sh.before_t && j <= sh.before_t + sh.pub[flip ^ 1].ties;
        if (here) {                            // (uniform over the block)
            uint32_t want = j - sh.before_t;
            int w = 0;
            while (want > sh.warp_u[1][w]) want -= sh.warp_u[1][w++];
            if (warp == w) {
                for (int64_t v0 = row.w0; v0 < row.w1; v0 += 32) {
                    const int64_t v = v0 + lane;
                    float f[V];
                    uint32_t cnt = 0;
                    if (v < row.w1) {
                        row.get(v, f);
#pragma unroll
                        for (int e = 0; e < V; e++) cnt += f[e] == x ? 1u : 0u;
                    }
                    uint32_t s = cnt;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
                    const uint32_t total = __shfl_sync(0xFFFFFFFFu, s, 31);
                    if (want <= total) {
                        if (cnt && want > s - cnt && want <= s) {
                            uint32_t left = want - (s - cnt);
                            int at = -1;
#pragma unroll
                            for (int e = 0; e < V; e++) if (f[e] == x && --left == 0) at = (int)(v * V - row.shift) + e;
                            for (int b = 0; b < nc; b++) *cluster.map_shared_rank(&sh.answer_i, b) = at;
                        }
                        break;
                    }
                    want -= total;
                }
            }
        }
        cluster.sync();
        const int at = sh.answer_i;
        return at;
    };

    // ---- finish with a short list: every entry with x >= low goes to block 0.  cut_k: it holds the top-k prefix,
    // whose mass top-p refers to; otherwise that mass is `mass`.
    auto finish_list = [&](float low, bool cut_k, double mass) {
        Shared* s0 = cluster.map_shared_rank(&sh, 0);
        row.each([&](float x, int i) {
            if (x >= low) {
                const uint32_t slot = atomicAdd(&s0->list_count, 1u);
                if (slot < CAP) { s0->list_key[slot] = key_of(x); s0->list_idx[slot] = i; }
            }
        });
        cluster.sync();
        if (c != 0) return;
        int m = (int)min(sh.list_count, (uint32_t)CAP);
        if (tid < m) {
            const uint32_t k = sh.list_key[tid];
            const int32_t i = sh.list_idx[tid];
            int r = 0;
            for (int j = 0; j < m; j++) r += (sh.list_key[j] > k || (sh.list_key[j] == k && sh.list_idx[j] < i)) ? 1 : 0;
            sh.list_rank_key[r] = k; sh.list_rank_idx[r] = i;
        }
        __syncthreads();
        if (cut_k) m = (int)min((int64_t)m, top_k);
        double w = tid < m ? weight(value_of(sh.list_rank_key[tid])) : 0.0;
        double reached = scan_d(w, 0);
        if (cut_k) {
            __syncthreads();
            if (tid == NT - 1) sh.sum_d = reached;
            __syncthreads();
            mass = sh.sum_d;
        }
        if (top_p < 1.f) m = min(m, first_true(tid < m && reached >= (double)top_p * mass, m - 1) + 1);
        if (min_p > 0.f) m = min(m, first_true(tid >= m || (double)value_of(sh.list_rank_key[tid]) - m64 < min_gap, m));
        // the kept entries in index order
        __syncthreads();
        if (tid < m) {
            const int32_t i = sh.list_rank_idx[tid];
            int r = 0;
            for (int j = 0; j < m; j++) r += sh.list_rank_idx[j] < i ? 1 : 0;
            sh.list_idx[r] = i; sh.list_w[r] = w;
        }
        __syncthreads();
        const double wi = tid < m ? sh.list_w[tid] : 0.0;
        reached = scan_d(wi, 1);
        __syncthreads();
        if (tid == m - 1) sh.sum_d = reached;
        __syncthreads();
        const double total = sh.sum_d;
        const int at = first_true(tid < m && reached > u * total, m - 1);
        if (tid == 0) {
            a.token[step] = sh.list_idx[at];
            a.logprob[step] = (float)log(sh.list_w[at] / total);
            a.kept[step] = m; a.status[step] = IMM_OK;
        }
    };

    // ---- greedy: the lowest index of the maximum
    if (temperature == 0.f) {
        uint32_t lowest = 0x7FFFFFFFu;
        row.each([&](float x, int i) { if (x == M) lowest = min(lowest, (uint32_t)i); });
        lowest = __reduce_min_sync(0xFFFFFFFFu, lowest);
        if (lane == 0) atomicMin((uint32_t*)&cluster.map_shared_rank(&sh, 0)->answer_i, lowest);   // (starts at -1 = 2^32 - 1)
        cluster.sync();
        if (c == 0 && tid == 0) {
            a.token[step] = sh.answer_i; a.logprob[step] = 0.f; a.kept[step] = 1; a.status[step] = IMM_OK;
        }
        return;
    }

    // Refines [klo, khi] (keys) until one value is left that holds the end of the prefix; then X and I are
    // set.  By count: the prefix has `k` entries, `above` of which have keys over khi.  By mass: it is the shortest
    // whose mass reaches `target`; entries with keys over khi and not over `khi_known` are not in `mass_above` yet.
    auto refine = [&](bool by_mass, uint32_t khi, uint32_t klo, uint32_t khi_known, uint32_t above, uint32_t k, double mass_above,
                      double target) {
        for (int level = 0; level < 64; level++) {             // (11 levels at most: every one leaves an eighth or less)
            int s = 0;
            while (((khi - klo) >> s) >= NB) s++;
            const bool last = khi == klo;
            double mass = 0.0;
            uint32_t ties = 0;
            row.each([&](float x, int i) {
                if (!inside(x, i)) return;
                const uint32_t key = key_of(x);
                if (key > khi) {
                    if (by_mass && key <= khi_known) mass += weight(x);
                } else if (key >= klo) {
                    if (last) ties++;
                    else atomicAdd(&sh.hist[hflip][(khi - key) >> s], 1u);
                }
            });
            if (by_mass || last) { exchange(mass, 0, ties); mass_above += sh.sum_d; khi_known = khi; }
            if (last) {
                const float x = value_of(khi);
                uint32_t j;
                if (by_mass) {
                    const double w = weight(x);
                    double want = ceil((target - mass_above) / w);
                    if (!(want >= 1.0)) want = 1.0;
                    if (want > (double)sh.sum_t) want = (double)sh.sum_t;
                    j = (uint32_t)want;
                    while (j > 1 && mass_above + (double)(j - 1) * w >= target) j--;
                    while (j < sh.sum_t && mass_above + (double)j * w < target) j++;
                } else {
                    j = k - above;
                }
                const bool all = j >= sh.sum_t;
                const int at = all ? (x == X ? I : 0x7FFFFFFF) : tie_index(x, j);
                X = x; I = at;
                return;
            }
            const uint32_t mine = merged_bin();
            int b1, b2;
            const uint32_t cum = scan_u(mine);
            if (by_mass) {
                const uint32_t top = khi - ((uint32_t)tid << s);
                const bool real = ((uint32_t)tid << s) <= khi - klo;
                const uint32_t bottom = top - klo < (1u << s) ? klo : top - ((1u << s) - 1u);
                const double hi = real ? (double)mine * weight(value_of(top)) : 0.0;
                const double lo = real ? (double)mine * weight(value_of(bottom)) : 0.0;
                const double upper = scan_d(hi, 0), lower = scan_d(lo, 1);
                const int end = (int)((khi - klo) >> s);
                b1 = first_true(mass_above + upper * (1.0 + 1e-12) >= target * (1.0 - 1e-12), end);
                b2 = first_true(mass_above + lower * (1.0 - 1e-12) >= target * (1.0 + 1e-12), end);
                b1 = min(b1, end); b2 = min(b2, end);
                // bounds too wide to help (weights that differ much within a bin), or the border nearer to a key's
                // mass than they resolve: halve the bins by their exact mass
                while (b2 > b1 && (s == 0 || b2 - b1 > NB / 8)) {
                    const int mid = (b1 + b2) >> 1;
                    const uint32_t split = khi - (((uint32_t)mid << s) + ((1u << s) - 1u));     // lowest key of bin `mid`
                    double part = 0.0;
                    row.each([&](float x, int i) {
                        const uint32_t key = key_of(x);
                        if (key >= split && key <= khi_known && inside(x, i)) part += weight(x);
                    });
                    exchange(part, 0, 0);
                    if (mass_above + sh.sum_d >= target) b2 = mid;
                    else { b1 = mid + 1; mass_above += sh.sum_d; khi_known = split - 1; }
                }
            } else {
                b1 = b2 = first_true(above + cum >= k, NB - 1);
                __syncthreads();
                if (tid == b1) sh.first_bin = (int)(cum - mine);
                __syncthreads();
                above += (uint32_t)sh.first_bin;
            }
            const uint32_t bottom = ((uint32_t)b2 << s) + ((1u << s) - 1u);
            const uint32_t new_lo = bottom >= khi - klo ? klo : khi - bottom;
            khi = khi - ((uint32_t)b1 << s);
            klo = new_lo;
        }
    };

    // ---- top-k
    bool cut_k = top_k > 0 && top_k < a.n;
    if (cut_k) {
        // A bound from the threads' maxima: if k of them lie in the first bins, so do the k largest entries.
        if (thread_best > NEG_INF) atomicAdd(&sh.hist[hflip][bin_of(thread_best)], 1u);
        uint32_t mine = merged_bin();
        const int b = first_true((int64_t)scan_u(mine) >= top_k, NB);
        if (b < NB - 1) {
            uint32_t khi, klo;
            bin_edges(0, b, khi, klo);
            const float low = value_of(klo);
            uint32_t count = 0;
            row.each([&](float x, int) { count += x >= low ? 1u : 0u; });
            exchange(0.0, count, 0);
            if (sh.sum_u <= CAP) { finish_list(low, true, 0.0); return; }
        }
        uint32_t count = 0;
        row.each([&](float x, int) {
            if (x > NEG_INF) { count++; atomicAdd(&sh.hist[hflip][bin_of(x)], 1u); }
        });
        exchange(0.0, count, 0);
        const uint32_t total = sh.sum_u;
        mine = merged_bin();
        if (total <= (uint64_t)top_k) cut_k = false;       // fewer entries than k: all are kept
        else {
            const uint32_t cum = scan_u(mine);
            const int b1 = first_true((int64_t)cum >= top_k, NB - 1);
            __syncthreads();
            if (tid == b1) sh.first_bin = (int)(cum - mine);
            __syncthreads();
            const uint32_t above = (uint32_t)sh.first_bin;
            uint32_t khi, klo;
            bin_edges(b1, b1, khi, klo);
            refine(false, khi, klo, khi, above, (uint32_t)top_k, 0.0, 0.0);
        }
    }

    // ---- top-p: the mass and the first histogram in one pass
    if (top_p < 1.f) {
        double mass = 0.0;
        row.each([&](float x, int i) {
            if (!inside(x, i)) return;
            mass += weight(x);
            atomicAdd(&sh.hist[hflip][bin_of(x)], 1u);
        });
        exchange(mass, 0, 0);
        const double whole = sh.sum_d, target = (double)top_p * whole;
        const uint32_t mine = merged_bin();
        // bounds of a bin's mass: the weights at its edges, with room for the rounding of bin_of (below 1e-5)
        const double width = 1.0 / (double)scale;
        const double hi = (double)mine * exp(-(double)tid * width * inv_t) * (1.0 + 1e-4);
        const double lo = tid == NB - 1 ? 0.0 : (double)mine * exp(-(double)(tid + 1) * width * inv_t) * (1.0 - 1e-4);
        const double upper = scan_d(hi, 0), lower = scan_d(lo, 1);
        const int b1 = first_true(upper >= target, NB - 1), b2 = first_true(lower >= target * (1.0 + 1e-9), NB - 1);
        const uint32_t cum = scan_u(mine);
        __syncthreads();
        if (tid == b2) sh.last_bin = (int)cum;
        uint32_t khi, klo;
        bin_edges(b1, b2, khi, klo);
        const uint32_t candidates = (uint32_t)sh.last_bin;
        if (candidates <= CAP && !cut_k) { finish_list(value_of(klo), false, whole); return; }
        refine(true, khi, klo, key_of(M), 0, 0, 0.0, target);
    }

    // ---- min-p: the smallest value that it leaves (M itself always stays)
    if (min_p > 0.f) {
        __syncthreads();
        if (warp == 0) {
            uint64_t lo = key_of(-3.402823466e+38f), hi = key_of(M);       // the answer lies in [lo, hi]
            while (lo < hi) {
                const uint64_t gap = hi - lo, probe = lo + min(gap, (gap / 32 + 1) * lane);
                const unsigned hits = __ballot_sync(0xFFFFFFFFu, (double)value_of((uint32_t)probe) - m64 >= min_gap);
                if (!hits) { lo = __shfl_sync(0xFFFFFFFFu, probe, 31) + 1; continue; }
                const int f = __ffs(hits) - 1;
                const uint64_t at = __shfl_sync(0xFFFFFFFFu, probe, f), prev = __shfl_sync(0xFFFFFFFFu, probe, f > 0 ? f - 1 : 0);
                hi = at;
                lo = f > 0 ? prev + 1 : at;
            }
            if (lane == 0) sh.edge[0] = (uint32_t)hi;
        }
        __syncthreads();
        const float x = value_of(sh.edge[0]);
        if (x > X) { X = x; I = 0x7FFFFFFF; }
    }

    // ---- the draw, in index order
    {
        double mass = 0.0;
        uint32_t count = 0;
        row.each([&](float x, int i) { if (inside(x, i)) { mass += weight(x); count++; } });
        exchange(mass, count, 0);
        const double total = sh.sum_d, aim = u * total;
        const uint32_t kept = sh.sum_u;
        // the block in which the cumulative weight passes `aim`; the last one with kept entries if rounding hides it
        int owner = -1, last_block = 0;
        double reached = 0.0;
        for (int b = 0; b < nc; b++) {
            const Publish p = *cluster.map_shared_rank(&sh.pub[flip ^ 1], b);
            reached += p.mass;
            if (p.count) last_block = b;
            if (owner < 0 && reached > aim) owner = b;
        }
        if (owner < 0) owner = last_block;
        if (owner == c) {
            double before = sh.before_d;
            int w = -1, last_warp = 0;
            double at_warp = before;
            for (int i = 0; i < NW; i++) {
                if (sh.warp_u[0][i]) last_warp = i;
                if (w < 0 && before + sh.warp_d[0][i] > aim) { w = i; at_warp = before; }
                before += sh.warp_d[0][i];
            }
            if (w < 0) {
                w = last_warp;
                at_warp = sh.before_d;
                for (int i = 0; i < w; i++) at_warp += sh.warp_d[0][i];
            }
            if (warp == w) {
                double acc = at_warp, w_found = 0.0, w_last = 0.0;
                int found = -1, last_kept = -1;
                for (int64_t v0 = row.w0; v0 < row.w1 && found < 0; v0 += 32) {
                    const int64_t v = v0 + lane;
                    float f[V];
                    double wt[V], mine = 0.0;
                    if (v < row.w1) row.get(v, f);
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        wt[e] = (v < row.w1 && inside(f[e], (int)(v * V - row.shift) + e)) ? weight(f[e]) : -1.0;
                        if (wt[e] > 0.0) mine += wt[e];
                    }
                    double s = mine;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) { const double t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
                    double run = acc + (s - mine);
                    int at = -1, lk = -1;
                    double wf = 0.0, wl = 0.0;
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        if (wt[e] >= 0.0) {
                            run += wt[e];
                            lk = (int)(v * V - row.shift) + e; wl = wt[e];
                            if (at < 0 && run > aim) { at = lk; wf = wl; }
                        }
                    }
                    const unsigned hits = __ballot_sync(0xFFFFFFFFu, at >= 0), some = __ballot_sync(0xFFFFFFFFu, lk >= 0);
                    if (hits) {
                        const int l = __ffs(hits) - 1;
                        found = __shfl_sync(0xFFFFFFFFu, at, l); w_found = __shfl_sync(0xFFFFFFFFu, wf, l);
                    }
                    if (some) {
                        const int l = 31 - __clz(some);
                        last_kept = __shfl_sync(0xFFFFFFFFu, lk, l); w_last = __shfl_sync(0xFFFFFFFFu, wl, l);
                    }
                    acc += __shfl_sync(0xFFFFFFFFu, s, 31);
                }
                if (found < 0) { found = last_kept; w_found = w_last; }
                if (lane == 0) {
                    a.token[step] = found; a.logprob[step] = (float)log(w_found / total);
                    a.kept[step] = (int32_t)kept; a.status[step] = IMM_OK;
                }
            }
        }
        cluster.sync();                        // nobody leaves while another block still reads its shared memory
    }
}

template <typename T>
cudaError_t launch(const Args& args, int64_t steps, cudaStream_t st)
{
    Args a = args;
    constexpr int V = Vec<T>::V;
    const int64_t nv = (a.n + 2 * V - 2) / V;              // vectors of a row, wherever it begins
    int nc = 1;
    while (nc < MAX_CLUSTER && (nv * 16 + nc - 1) / nc > SLICE_BYTES) nc *= 2;
    a.per = (nv + nc - 1) / nc;
    const bool cached = a.per * 16 <= CACHE_MAX;
    const size_t smem = cached ? (size_t)a.per * 16 : 0;
    auto kernel = cached ? sample_kernel<T, true> : sample_kernel<T, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, CACHE_MAX);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(steps * nc));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    memset(&attr, 0, sizeof(attr));
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)nc;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace imm_sample_ns

extern "C" int imm_sample(const void* d_logits, int dtype, int64_t steps, int64_t n, int64_t ld, const double* d_u,
                          const imm_sample_params* params_host, int32_t* d_token, float* d_logprob, int32_t* d_kept,
                          int32_t* d_status, void* stream)
{
    using namespace imm_sample_ns;
    if (!params_host || (steps > 0 && (!d_logits || !d_u || !d_token || !d_logprob || !d_kept || !d_status))) return IMM_ERR_ARG;
    if (dtype != IMM_F32 && dtype != IMM_BF16 && dtype != IMM_F16) return IMM_ERR_ARG;
    if (steps < 0 || n <= 0 || ld < n || n > IMM_LDD_MAX_N || steps > IMM_LDD_MAX_STEPS) return IMM_ERR_SHAPE;
    const imm_sample_params& p = *params_host;
    if ((uintptr_t)d_logits % (dtype == IMM_F32 ? 4 : 2) || (uintptr_t)d_u % 8 || (uintptr_t)d_token % 4 || (uintptr_t)d_logprob % 4 ||
        (uintptr_t)d_kept % 4 || (uintptr_t)d_status % 4 || (uintptr_t)p.d_temperature % 4 || (uintptr_t)p.d_top_k % 4 ||
        (uintptr_t)p.d_top_p % 4 || (uintptr_t)p.d_min_p % 4)
        return IMM_ERR_ALIGN;
    if (steps == 0) return IMM_OK;
    Args a{};
    a.logits = d_logits; a.n = n; a.ld = ld; a.u = d_u;
    a.temperature_row = p.d_temperature; a.top_p_row = p.d_top_p; a.min_p_row = p.d_min_p; a.top_k_row = p.d_top_k;
    a.temperature = p.temperature; a.top_p = p.top_p; a.min_p = p.min_p; a.top_k = p.top_k;
    a.token = d_token; a.logprob = d_logprob; a.kept = d_kept; a.status = d_status;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == IMM_F32 ? launch<float>(a, steps, st)
                          : dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, steps, st) : launch<__half>(a, steps, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
