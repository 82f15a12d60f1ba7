// Verification of drafted tokens (sm_100a), and the call's C ABI (declared in imm.h).
//
//   imm_verify_draft   takes drafted tokens while u q(d) < p(d), and draws the token behind them
//
// The mathematics (speculative sampling, Leviathan, Kalman, Matias 2023).  With w = exp((x - M) / T) and Z their sum, p = w / Z.
// A drafted token is taken where u q(d) < p(d); the first that is not is replaced by a draw from max(p - q, 0): the
// lowest index at which the running sum passes u' times the whole.  Both are comparisons next to borders, so weights and
// sums are float64, as in the draw without a draft.  exp: table of 2^(j/16) and a polynomial of degree 5 (table-driven
// exponential, P. T. P. Tang 1989; Taylor coefficients), relative error below 2e-13.
//
// A request is taken by the blocks of a thread-block cluster, row by row until a token is not taken: rows more than one
// behind it are not read (the next is asked for while one is summed).  A row (and its draft's) takes one pass in float32 against an
// entry of its own, whose sum is within 1e-5 or so of exact (the bound grows with the distance of the entries that matter); the
// blocks' sums meet in every block's shared memory, so that all come to the same decision.  Where u q(d) and p(d) are nearer to each
// other than that, the rows are summed in float64; rows in which a block's first entries are all masked (filters that leave a few
// of many) are summed so throughout, after the float32 pass.  The answer's rows take one more pass (from
// L2): p's sum in float64, for the logarithm, and the sums of max(p - q, 0) by sub-chunk in float32; an answer that lies nearer
// to a border than those can tell (one in ten, where the tail of the distribution holds a tenth) is drawn again in float64.
//
// Measured (B200): one request of 4 drafts and 128256 float32 entries 21 us, 64 of them in bfloat16 105 us.  What bounds it is
// latency: a row waits for the one before it, 11 thousand cycles a row (5 thousand of them exponentials, the rest loads and a
// cluster barrier), 25 thousand for the answer (float64 sums, two barriers), and requests of different lengths leave a third of
// the multiprocessors idle at the end.
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

namespace imm_verify_ns {

namespace cg = cooperative_groups;

constexpr int NT = 256;
constexpr int NW = NT / 32;
constexpr int MAX_CLUSTER = 16;
constexpr int BLOCKS_PER_SM = 2;              // resident: 128 registers (three with 80: 115 us for 64 x 4 of 128256 bf16, two: 103)
constexpr int PIECES = 64;                    // 16-byte pieces of a sub-chunk: two per lane of a warp
constexpr int MOST_SUBS = IMM_LDD_MAX_N / 4 / PIECES;     // sub-chunks of the longest row (4 entries to a piece at least)
constexpr float NEG_INF = -INFINITY;
constexpr double RANGE = 690.0;               // entries below the maximum by more temperatures count as 0

struct Args {
    const void *target, *draft;
    const int32_t* tokens;
    const int64_t* offsets;
    const double* u;
    const float* temperature_of;
    int32_t *accepted, *token;
    float* logprob;
    int32_t* status;
    int64_t rows, drafts, n, ldt, ldd;
    float temperature;
};

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <typename T> __device__ __forceinline__ void unpack(uint4 r, float (&f)[16 / sizeof(T)])
{
    const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); i++) f[i] = (float)e[i];
}

// A row of logits by pieces of 16 bytes, counted from its first entry wherever that lies.
template <typename T, bool ALIGNED> struct Row {           // ALIGNED: begins on a 16-byte boundary
    static constexpr int V = 16 / sizeof(T);
    const T* p;
    int n;
    // Piece i (entries V i .. V i + V - 1) as the one or two 16-byte granules that hold it, so that it can be asked for before it
    // is wanted; granules without an entry of the row are not read, and entries behind the row are -inf.
    struct Raw { uint4 lo, hi; };
    __device__ __forceinline__ Raw ask(int i) const
    {
        Raw r;
        const uintptr_t at = (uintptr_t)(p + (int64_t)i * V), last = (uintptr_t)(p + min(n, i * V + V)) - 1;
        const uint4* a = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
        r.lo = __ldg(a);
        r.hi = r.lo;
        if (!ALIGNED && (at ^ last) & ~(uintptr_t)15) r.hi = __ldg(a + 1);
        return r;
    }
    __device__ __forceinline__ void get(const Raw& raw, int i, float (&f)[V]) const
    {
        uint4 r = raw.lo;
        const uint32_t sh = (uint32_t)(uintptr_t)p & 15u;              // (V entries are 16 bytes: alike for all pieces)
        if (!ALIGNED && sh) {
            const uint32_t bits = 8 * (sh & 3u), w[8] = {raw.lo.x, raw.lo.y, raw.lo.z, raw.lo.w, raw.hi.x, raw.hi.y, raw.hi.z, raw.hi.w};
            uint32_t s[5];
#pragma unroll
            for (int k = 0; k < 5; k++) s[k] = (sh >> 2) == 0 ? w[k] : (sh >> 2) == 1 ? w[k + 1] : (sh >> 2) == 2 ? w[k + 2] : w[k + 3 < 8 ? k + 3 : 7];
            r = make_uint4(__funnelshift_r(s[0], s[1], bits), __funnelshift_r(s[1], s[2], bits), __funnelshift_r(s[2], s[3], bits),
                           __funnelshift_r(s[3], s[4], bits));
        }
        unpack<T>(r, f);
        if (i * V + V > n) {
#pragma unroll
            for (int e = 0; e < V; e++) if (i * V + e >= n) f[e] = NEG_INF;
        }
    }
    __device__ __forceinline__ T entry(int i) const { return __ldg(p + i); }
    // pieces [i0, i1) on their way to L2: whole granules that hold an entry of the row
    __device__ __forceinline__ void prefetch(int i0, int i1) const
    {
        const int64_t e0 = (int64_t)i0 * V, e1 = min((int64_t)n, (int64_t)i1 * V);
        if (e0 >= e1) return;
        const uintptr_t from = (uintptr_t)(p + e0) & ~(uintptr_t)15, to = ((uintptr_t)(p + e1) + 15) & ~(uintptr_t)15;
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((uint32_t)(to - from)) : "memory");
    }
};

// The same by the granules that hold it, for sums that need no common index: entry 0 lies at `head` of the first one.
template <typename T> struct Granules {
    static constexpr int V = 16 / sizeof(T);
    using Raw = uint4;
    const uint4* p;
    int head, n;                               // n: head and entries
    __device__ __forceinline__ Granules(const T* row, int entries)
        : p(reinterpret_cast<const uint4*>((uintptr_t)row & ~(uintptr_t)15)), head((int)((uintptr_t)row & 15) / (int)sizeof(T)), n(entries + head) {}
    __device__ __forceinline__ Raw ask(int i) const { return __ldg(p + i); }
    __device__ __forceinline__ void get(const Raw& raw, int i, float (&f)[V]) const
    {
        unpack<T>(raw, f);
        if (i == 0 || i * V + V > n) {
#pragma unroll
            for (int e = 0; e < V; e++) if (i * V + e < head || i * V + e >= n) f[e] = NEG_INF;
        }
    }
};

// exp(d / T) in float64
struct Weight {
    double factor, least;                     // 16 log2(e) / T, -RANGE * T
    const double* table;
    // d from -RANGE T to RANGE T
    __device__ __forceinline__ double of(double d) const
    {
        constexpr double MAGIC = 6755399441055744.0;
        constexpr double L = 0.043321698784996581838;          // ln(2) / 16
        constexpr double c1 = L, c2 = L * L / 2, c3 = L * L * L / 6, c4 = L * L * L * L / 24, c5 = L * L * L * L * L / 120;
        const double km = fma(d, factor, MAGIC);
        const int K = __double2loint(km);
        const double r = fma(d, factor, MAGIC - km);
        double q = fma(c5, r, c4);
        q = fma(q, r, c3);
        q = fma(q, r, c2);
        q = fma(q, r, c1);
        q = fma(q, r, 1.0);
        const double w = q * table[K & 15];
        return __hiloint2double(__double2hiint(w) + (int)((uint32_t)(K & ~15) << 16), __double2loint(w));
    }
    __device__ __forceinline__ double operator()(float x, float M) const          // 0 below the range
    {
        const double d = (double)x - (double)M;
        return d < least ? 0.0 : of(fmin(d, -least));
    }
};

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// This thread's pieces of the block's [p0, p1) of ROWS rows, BATCH pieces (NT apart) at a time, the next ones on their way; what
// lies behind the block's pieces is -inf
template <int ROWS, int BATCH, typename R> struct Batches {
    static constexpr int V = R::V;
    const R &a, &b;
    int i0, end[ROWS];
    typename R::Raw raw[ROWS][BATCH];
    __device__ __forceinline__ void ask()
    {
#pragma unroll
        for (int w = 0; w < ROWS; w++)
#pragma unroll
            for (int u = 0; u < BATCH; u++)
                if (i0 + u * NT < end[w]) raw[w][u] = (w ? b : a).ask(i0 + u * NT);
    }
    __device__ __forceinline__ Batches(const R& a_, const R& b_, int p0, int p1) : a(a_), b(b_)
    {
        asm volatile("" : "+r"(p0), "+r"(p1)); // (nothing of the loop is worth keeping in registers from one row to the next)
#pragma unroll
        for (int w = 0; w < ROWS; w++) end[w] = min(p1, ((w ? b : a).n + V - 1) / V);
        i0 = p0 + (int)threadIdx.x;
        ask();
    }
    __device__ __forceinline__ void get(float (&x)[ROWS][BATCH][V]) const
    {
#pragma unroll
        for (int w = 0; w < ROWS; w++)
#pragma unroll
            for (int u = 0; u < BATCH; u++)
                if (i0 + u * NT < end[w]) (w ? b : a).get(raw[w][u], i0 + u * NT, x[w][u]);
                else {
#pragma unroll
                    for (int e = 0; e < V; e++) x[w][u][e] = NEG_INF;
                }
    }
    // f(piece, entries)
    template <typename F> __device__ __forceinline__ void each(F&& f)
    {
#pragma unroll 1
        while (i0 < max(end[0], end[ROWS - 1])) {
            float x[ROWS][BATCH][V];
            get(x);
            const int at = i0;
            i0 += BATCH * NT;
            ask();
            f(at, x);
        }
    }
};

// The sum of a row's float32 weights relative to `ref`, an entry of it
struct Quick { float z, ref; };

struct Stat { double z; float top; int32_t index; };          // sum of the weights relative to the maximum, maximum, its lowest index

struct Shared {
    double table[16];
    Quick quick[2][2][MAX_CLUSTER];           // [which copy][target, draft][block]
    Stat stat[2][MAX_CLUSTER];
    double sums[MAX_CLUSTER];                 // the blocks' shares of the draw's mass
    double warp_d[NW];
    uint32_t mass[MOST_SUBS / 32];            // a bit per sub-chunk of the block: its sum is not 0
    float warp_f[2][NW];
    uint32_t warp_u[NW];
    int32_t hit, unsure;
};

// Of this block's sub-chunks [s0, s1), against the largest of the entries that its threads meet first.  With y = (x - ref) log2(e) / T
// a weight is off by three roundings of 2^-24 |y| ln(2) each and the 2^-22 of the exponential: off_by(y) of it.  What lies 2^40 below
// the reference holds n 2^-40 of the sum at most, and what lies 2^126 below and is 0, n 2^-126; so a sum with weights up to 2^k is off by
// off_by(max(40, k)), and by its additions: of a thread's entries in four parts, a quarter of them half-steps; of parts, lanes, warps and
// blocks, 2 + 5 + 8 + 4.  A row whose sum is not a positive finite number is left to float64 (a block that meets masked entries only,
// entries 2^127 above the reference, NaN, infinity).
__device__ __forceinline__ float off_by(float y) { return fmaf(fminf(fabsf(y), 512.f), 2.1f * 0x1p-24f, 0x1p-22f); }
__device__ __forceinline__ float additions(int entries_per_thread) { return (float)(entries_per_thread / 4 + 20) * 0x1p-24f; }
// ... relative to another entry, and what it is off by (but for its additions).  The sum's exponent k goes into the exponential: beside a
// reference 2^127 below the row's largest entries the sum is as large, and would be lost where the other entry lies 2^126 above.
__device__ __forceinline__ float share_of(const Quick& x, float ref, float factor, float& off)
{
    const uint32_t bits = __float_as_uint(x.z);            // (1 or more: the reference's own weight is in it)
    off = 0.f;
    if (x.z == 0.f || bits >= 0x7F800000u) return x.z;     // no pieces; infinity, NaN
    const float k = (float)((int)(bits >> 23) - 127), y = (x.ref - ref) * factor;
    const float share = __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u) * exp2_fast(y + k);
    // (the sum itself; y, y + k, the exponential and the product; blocks of less than 2^-40 hold 2^-36 of the row together)
    if (share > 0x1p-40f) off = off_by(fmaxf(40.f, k + 1.f) + fabsf(y) + fabsf(y + k)) + 0x1p-21f;
    return share;
}
template <int ROWS, typename R>
__device__ __forceinline__ void quick_stat(const R target, const R draft, int p0, int p1, float factor, Quick& first, Quick& second, Shared& sh)
{
    constexpr int V = R::V, BATCH = 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float ref[ROWS], sum[ROWS][4], z[ROWS];
#pragma unroll
    for (int w = 0; w < ROWS; w++) { ref[w] = NEG_INF; sum[w][0] = sum[w][1] = sum[w][2] = sum[w][3] = 0.f; }
    Batches<ROWS, BATCH, R> batches(target, draft, p0, p1);
    {
        float x[ROWS][BATCH][V];
        batches.get(x);
#pragma unroll
        for (int w = 0; w < ROWS; w++)
#pragma unroll
            for (int u = 0; u < BATCH; u++)
#pragma unroll
                for (int e = 0; e < V; e++) ref[w] = fmaxf(ref[w], x[w][u][e]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int w = 0; w < ROWS; w++) ref[w] = fmaxf(ref[w], __shfl_xor_sync(0xFFFFFFFFu, ref[w], o));
    __syncthreads();
    if (lane == 0) {
#pragma unroll
        for (int w = 0; w < ROWS; w++) sh.warp_f[w][warp] = ref[w];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < ROWS; w++)
#pragma unroll
        for (int k = 0; k < NW; k++) ref[w] = fmaxf(ref[w], sh.warp_f[w][k]);
    batches.each([&](int, const float (&x)[ROWS][BATCH][V]) {
#pragma unroll
        for (int w = 0; w < ROWS; w++)
#pragma unroll
            for (int u = 0; u < BATCH; u++)
#pragma unroll
                for (int e = 0; e < V; e++) sum[w][e & 3] += exp2_fast((x[w][u][e] - ref[w]) * factor);
    });
#pragma unroll
    for (int w = 0; w < ROWS; w++) z[w] = (sum[w][0] + sum[w][1]) + (sum[w][2] + sum[w][3]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int w = 0; w < ROWS; w++) z[w] += __shfl_xor_sync(0xFFFFFFFFu, z[w], o);
    __syncthreads();
    if (lane == 0) {
#pragma unroll
        for (int w = 0; w < ROWS; w++) sh.warp_f[w][warp] = z[w];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < ROWS; w++) {
        float all = 0.f;
#pragma unroll
        for (int k = 0; k < NW; k++) all += sh.warp_f[w][k];
        (w ? second : first) = Quick{p0 < p1 ? all : 0.f, p0 < p1 ? ref[w] : NEG_INF};        // (a block without pieces has nothing)
    }
}

// The block's maximum and its lowest index from the threads', and the threads' sums (relative to `ref`) relative to the maximum
__device__ __forceinline__ Stat block_join(float top, int index, float ref, double z, const Weight& weight, Shared& sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float all = top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all = max_nan(all, __shfl_xor_sync(0xFFFFFFFFu, all, o));
    __syncthreads();
    if (lane == 0) sh.warp_f[0][warp] = all;
    __syncthreads();
    all = sh.warp_f[0][0];
#pragma unroll
    for (int k = 1; k < NW; k++) all = max_nan(all, sh.warp_f[0][k]);
    const uint32_t first = __reduce_min_sync(0xFFFFFFFFu, top == all ? (uint32_t)index : 0x7FFFFFFFu);
    const double mine = warp_sum(ref > NEG_INF && all < INFINITY ? z * weight(ref, all) : 0.0);
    if (lane == 0) { sh.warp_u[warp] = first; sh.warp_d[warp] = mine; }
    __syncthreads();
    Stat r{0.0, all, 0x7FFFFFFF};
#pragma unroll
    for (int k = 0; k < NW; k++) { r.z += sh.warp_d[k]; r.index = min(r.index, (int32_t)sh.warp_u[k]); }
    return r;
}

// A thread's float64 sum relative to an entry of its own, which it leaves for one that lies far above
struct Running {
    float top, ref, slack;
    double z;
    __device__ __forceinline__ explicit Running(const Weight& weight) : top(NEG_INF), ref(NEG_INF), slack((float)fmin(-0.4 * weight.least, 3e38)), z(0.0) {}
    template <int V> __device__ __forceinline__ void add(const float (&x)[V], const Weight& weight)
    {
        float most = x[0];
#pragma unroll
        for (int e = 1; e < V; e++) most = max_nan(most, x[e]);
        top = max_nan(top, most);
        if (!(most > NEG_INF && most < INFINITY)) return;
        if (!(most - ref <= slack)) {          // (the first, too)
            z = ref == NEG_INF ? 0.0 : z * weight(ref, most);
            ref = most;
        }
#pragma unroll
        for (int e = 0; e < V; e++) z += weight.of(fmax((double)x[e] - (double)ref, weight.least));       // (a masked entry: e^-690)
    }
};

// Maximum and float64 sum of this block's sub-chunks of a row
template <typename R>
__device__ __forceinline__ Stat exact_stat(const R row, int s0, int s1, const Weight weight, Shared& sh)
{
    Running run(weight);
    Batches<1, 1, R>(row, row, s0 * PIECES, s1 * PIECES).each([&](int, const float (&x)[1][1][R::V]) { run.add(x[0][0], weight); });
    return block_join(run.top, 0x7FFFFFFF, run.ref, run.z, weight, sh);
}
// ... maximum and its lowest index
template <typename R>
__device__ __forceinline__ Stat greedy_stat(const R row, int s0, int s1, const Weight weight, Shared& sh)
{
    float top = NEG_INF;
    int index = 0x7FFFFFFF;
    Batches<1, 2, R>(row, row, s0 * PIECES, s1 * PIECES).each([&](int i, const float (&x)[1][2][R::V]) {
        float most = NEG_INF;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int e = 0; e < R::V; e++) most = max_nan(most, x[0][u][e]);
        if (most > top) {
#pragma unroll
            for (int u = 1; u >= 0; u--)
#pragma unroll
                for (int e = R::V - 1; e >= 0; e--) if (x[0][u][e] == most) index = (i + u * NT) * R::V + e;
        }
        top = max_nan(top, most);
    });
    return block_join(top, index, NEG_INF, 0.0, weight, sh);
}

// What the draw is made from, in float64: max(p - q, 0), without entry `without`; iq = 0: p alone.  (Nothing is contracted: an entry
// is the same number wherever it is worked out, so a sub-chunk whose sum is not 0 holds one that is not 0.)
template <typename R> struct Rest {
    R target, draft;
    Weight weight;
    double ip, iq;                             // 1 / Z
    float p, q;                                // maxima
    int without;
    __device__ __forceinline__ void operator()(int i, double (&r)[R::V]) const
    {
        float x[R::V], y[R::V];
        const typename R::Raw rx = target.ask(i), ry = iq != 0.0 ? draft.ask(i) : rx;
        target.get(rx, i, x);
        if (iq != 0.0) draft.get(ry, i, y);
#pragma unroll
        for (int e = 0; e < R::V; e++) {
            r[e] = __dmul_rn(weight(x[e], p), ip);
            if (iq != 0.0) r[e] = fmax(__dsub_rn(r[e], __dmul_rn(weight(y[e], q), iq)), 0.0);
            if (i * R::V + e == without) r[e] = 0.0;
        }
    }
};
// ... in float32, against the references of the quick sums
template <typename R> struct QuickRest {
    R target, draft;
    float factor, ip, iq, p, q;
    int without;
    __device__ __forceinline__ void rest(int i, const float (&x)[R::V], const float (&y)[R::V], double (&r)[R::V]) const
    {
#pragma unroll
        for (int e = 0; e < R::V; e++) {
            float v = exp2_fast((x[e] - p) * factor) * ip;
            if (iq != 0.f) v = fmaxf(fmaf(exp2_fast((y[e] - q) * factor), -iq, v), 0.f);
            r[e] = i * R::V + e == without ? 0.f : v;
        }
    }
    __device__ __forceinline__ void operator()(int i, double (&r)[R::V]) const
    {
        float x[R::V], y[R::V];
        const typename R::Raw rx = target.ask(i), ry = iq != 0.f ? draft.ask(i) : rx;
        target.get(rx, i, x);
        if (iq != 0.f) draft.get(ry, i, y);
        rest(i, x, y, r);
    }
};
// float64 sums over the block's sub-chunks
template <typename R>
__device__ __forceinline__ void rest_sums(const Rest<R> rest, int s0, int s1, double* sub_sum)
{
    const int lane = threadIdx.x & 31;
    for (int s = s0 + (int)(threadIdx.x >> 5); s < s1; s += NW) {
        double part = 0.0;
#pragma unroll
        for (int h = 0; h < PIECES / 32; h++) {
            const int i = s * PIECES + h * 32 + lane;
            if (i * R::V >= rest.target.n) continue;
            double r[R::V];
            rest(i, r);
#pragma unroll
            for (int e = 0; e < R::V; e++) part += r[e];
        }
        part = warp_sum(part);
        if (lane == 0) sub_sum[s - s0] = part;
    }
}
// float32 sums over the block's sub-chunks (a lane's 2 V entries, then the lanes': 20 half-steps at most), and the target's float64 sum
template <typename R>
__device__ __forceinline__ Stat quick_sums(const QuickRest<R> quick, int s0, int s1, const Weight weight, double* sub_sum, Shared& sh)
{
    constexpr int V = R::V, H = PIECES / 32;
    const int lane = threadIdx.x & 31;
    Running run(weight);
    typename R::Raw rx[H], ry[H], next_x[H], next_y[H];
    auto ask = [&](int s) {
#pragma unroll
        for (int h = 0; h < H; h++) {
            const int i = s * PIECES + h * 32 + lane;
            if (s >= s1 || i * V >= quick.target.n) continue;
            next_x[h] = quick.target.ask(i);
            if (quick.iq != 0.f) next_y[h] = quick.draft.ask(i);
        }
    };
    ask(s0 + (int)(threadIdx.x >> 5));
    for (int s = s0 + (int)(threadIdx.x >> 5); s < s1; s += NW) {
#pragma unroll
        for (int h = 0; h < H; h++) { rx[h] = next_x[h]; ry[h] = next_y[h]; }
        ask(s + NW);
        float part = 0.f;
#pragma unroll
        for (int h = 0; h < H; h++) {
            const int i = s * PIECES + h * 32 + lane;
            if (i * V >= quick.target.n) continue;
            float x[V], y[V];
            quick.target.get(rx[h], i, x);
            if (quick.iq != 0.f) quick.draft.get(ry[h], i, y);
            double r[V];
            quick.rest(i, x, y, r);
#pragma unroll
            for (int e = 0; e < V; e++) part += (float)r[e];
            run.add(x, weight);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
        if (lane == 0) sub_sum[s - s0] = part;
    }
    return block_join(run.top, 0x7FFFFFFF, run.ref, run.z, weight, sh);
}

// The entry at which the running sum of the rests passes `aim`, by one warp of the block that holds it: `before` is what lies before
// sub-chunk s.  Where rounding hides it, the last entry at which the sum grows.  sure: it lies further than `doubt` from its borders.
template <typename F, int V>
__device__ __forceinline__ int entry_of(const F& rest, int s, int n, double before, double aim, double doubt, bool& sure)
{
    const int lane = threadIdx.x & 31;
    double r[2][V], mine = 0.0;
#pragma unroll
    for (int h = 0; h < 2; h++) {              // two neighbouring pieces per lane
        const int i = s * PIECES + 2 * lane + h;
#pragma unroll
        for (int e = 0; e < V; e++) r[h][e] = 0.0;
        if (i * V < n) rest(i, r[h]);
#pragma unroll
        for (int e = 0; e < V; e++) mine += r[h][e];
    }
    double upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const double w = __shfl_up_sync(0xFFFFFFFFu, upto, o); if (lane >= o) upto += w; }
    const double lower = __shfl_up_sync(0xFFFFFFFFu, upto, 1);
    double at = before + (lane ? lower : 0.0), left = 0.0;
    int hit = 0x7FFFFFFF, end = -1;
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int e = 0; e < V; e++)
            if (r[h][e] > 0.0) {
                const double from = at;
                at += r[h][e];
                end = (s * PIECES + 2 * lane + h) * V + e;
                if (at > aim && hit == 0x7FFFFFFF) { hit = end; left = fmin(at - aim, aim - from); }
            }
    int answer = (int)__reduce_min_sync(0xFFFFFFFFu, (uint32_t)hit);
    sure = __any_sync(0xFFFFFFFFu, hit == answer && hit != 0x7FFFFFFF && left > doubt);
    const int behind = __reduce_max_sync(0xFFFFFFFFu, end);
    return answer == 0x7FFFFFFF ? behind : answer;
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(NT, BLOCKS_PER_SM) verify_kernel(const Args a)
{
    using R = Row<T, ALIGNED>;
    constexpr int V = R::V;
    extern __shared__ double sub_sum[];       // of this block's sub-chunks
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int nc = (int)cluster.num_blocks(), c = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t request = blockIdx.x / nc;
    const int64_t o0 = __ldg(a.offsets + request), o1 = __ldg(a.offsets + request + 1);
    const float t = a.temperature_of ? __ldg(a.temperature_of + request) : a.temperature;
    const int n = (int)a.n;
    if (tid < 16) sh.table[tid] = exp2((double)tid * 0.0625);
    bool wrong = !(o0 >= 0 && o1 > o0 && o1 <= a.rows) || !(t >= 0.f && t < INFINITY);
    if (a.draft) wrong |= o0 < request || o1 - 1 - request > a.drafts;
    if (!wrong) {
        for (int64_t i = o0 + tid; i < o1; i += NT) {
            const double u = __ldg(a.u + i);
            const int32_t d = i > o0 ? __ldg(a.tokens + i) : 0;
            wrong |= !(u >= 0.0 && u < 1.0) || d < 0 || d >= n;
        }
    }
    const int nsub = ((n + V - 1) / V + PIECES - 1) / PIECES, per = (nsub + nc - 1) / nc;
    const int s0 = min(nsub, c * per), s1 = min(nsub, s0 + per);
    const bool two_rows = a.draft && t != 0.f;
    // (a row is asked for while the one before it is summed: it is read in vain where that one's token is not taken, but a request's
    // rows otherwise wait for HBM one after the other)
    auto prefetch = [&](int64_t row, bool tested) {
        if (tid == 0) R{(const T*)a.target + row * a.ldt, n}.prefetch(s0 * PIECES, s1 * PIECES);
        if (tid == 32 && tested && two_rows) R{(const T*)a.draft + (row - request) * a.ldd, n}.prefetch(s0 * PIECES, s1 * PIECES);
    };
    if (!wrong) prefetch(o0, o1 - o0 > 1);
    wrong = __syncthreads_or(wrong);
    cluster.sync();                           // (all blocks run before one stores into another's memory)
    const bool greedy = t == 0.f;
    Weight weight;
    weight.factor = greedy ? 0.0 : 23.083120654223414219 / (double)t;
    weight.least = -RANGE * (double)t;
    weight.table = sh.table;
    // float32 serves temperatures that are not near its ends
    const float factor = (float)(weight.factor * 0.0625);
    const bool quick = !greedy && factor > 1e-30f && factor < 1e30f;
    const float added = additions((per * PIECES + NT) / NT * V);

    int taken = 0, copy = 0, fresh = 0;
    Stat p{}, q{};
    Quick qp{}, qq{};
    float doubt_p = 0.f, doubt_q = 0.f;        // what their sums are off by, relative
    bool refused = false, quick_done = false;             // the answer replaces a drafted token; its rows have float32 sums
    R target{nullptr, n}, draft{nullptr, n};
    const int k = wrong ? 0 : (int)(o1 - o0 - 1);
    int d = 0;

    // a row's maximum and sum from all blocks, which every warp puts together alike, a lane per block
    auto put = [&](const Stat& mine) {
        if (tid < nc) cluster.map_shared_rank(&sh, tid)->stat[copy][c] = mine;
    };
    auto together = [&](Stat& r) {             // (behind a cluster barrier)
        const Stat x = lane < nc ? sh.stat[copy][lane] : Stat{0.0, NEG_INF, 0x7FFFFFFF};
        r.top = x.top;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) r.top = max_nan(r.top, __shfl_xor_sync(0xFFFFFFFFu, r.top, o));
        r.index = (int32_t)__reduce_min_sync(0xFFFFFFFFu, x.top == r.top ? (uint32_t)x.index : 0x7FFFFFFFu);
        r.z = warp_sum(x.top > NEG_INF && r.top < INFINITY ? x.z * weight(x.top, r.top) : 0.0);
        copy ^= 1;
        wrong |= !(r.top > NEG_INF && r.top < INFINITY);
    };
    auto gather = [&](const Stat& mine, Stat& r) {
        put(mine);
        cluster.sync();
        together(r);
    };
    auto exact = [&](bool one, bool two) {
        if (one) gather(exact_stat(target, s0, s1, weight, sh), p);
        if (two) gather(exact_stat(draft, s0, s1, weight, sh), q);
    };

    while (!wrong) {
        const int64_t row = o0 + taken;
        const bool tested = taken < k;
        // (at temperature 0 nothing asks for it.  `&& !greedy` here as well, a factor that the branches below hold anyway, made nvcc 12.9
        // sum the target's row alone: its front end from -Xcicc -O1 on, whatever ptxas did, right at -O0)
        const bool drafted = tested && a.draft != nullptr;
        target.p = (const T*)a.target + row * a.ldt;
        draft.p = drafted ? (const T*)a.draft + (row - request) * a.ldd : target.p;
        d = tested ? __ldg(a.tokens + row + 1) : 0;
        const double u = __ldg(a.u + row);
        const T xd = target.entry(d), yd = draft.entry(d);            // (float32 where they are used: nothing waits for them here)
        if (tested) prefetch(row + 1, taken + 1 < k);
        bool take = false, sure = false;
        quick_done = false;
        if (greedy) {
            gather(greedy_stat(target, s0, s1, weight, sh), p);
            take = d == p.index;
            sure = true;
        } else if (quick) {
            Quick first, second;
            // (a row that begins inside a granule may have one more of them: the last block's)
            const int p0 = s0 * PIECES, p1 = s1 == nsub && s0 < s1 ? 0x7FFFFFFF : s1 * PIECES;
            const Granules<T> tg(target.p, n), dg(draft.p, n);
            if (drafted) quick_stat<2>(tg, dg, p0, p1, factor, first, second, sh);
            else {
                quick_stat<1>(tg, dg, p0, p1, factor, first, second, sh);
                second = first;
            }
            if (tid < nc) {
                Shared* there = cluster.map_shared_rank(&sh, tid);
                there->quick[fresh][0][c] = first;
                there->quick[fresh][1][c] = second;
            }
            cluster.sync();
#pragma unroll
            for (int w = 0; w < 2; w++) {
                const Quick x = lane < nc ? sh.quick[fresh][w][lane] : Quick{0.f, NEG_INF};
                Quick r{0.f, x.ref};
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) r.ref = fmaxf(r.ref, __shfl_xor_sync(0xFFFFFFFFu, r.ref, o));
                float off;
                r.z = share_of(x, r.ref, factor, off);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) r.z += __shfl_xor_sync(0xFFFFFFFFu, r.z, o);
                (w ? qq : qp) = r;
                (w ? doubt_q : doubt_p) = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(off))) + added;
            }
            fresh ^= 1;
            quick_done = qp.z > 0.f && qp.z < INFINITY && qq.z > 0.f && qq.z < INFINITY;
            if (quick_done && tested) {
                const float yp = ((float)xd - qp.ref) * factor, yq = drafted ? ((float)yd - qq.ref) * factor : 0.f;
                const float pd = exp2_fast(yp) / qp.z, limit = drafted ? (float)u * (exp2_fast(yq) / qq.z) : (float)u;
                // (two more half-steps for either side; the exponentials give 0 below 2^-126)
                const float margin = fmaf(off_by(yp) + doubt_p + 0x1p-23f, pd, fmaf((drafted ? off_by(yq) + doubt_q : 0.f) + 0x1p-23f, limit, 0x1p-124f));
                take = limit < pd;
                sure = fabsf(limit - pd) > margin;                     // (false for NaN, and where both are 0)
            }
        }
        if (!sure && tested && !wrong) {
            exact(true, drafted);
            // (quotients: where the two rows are the same, u q < q holds after rounding for every u below 1)
            const double pd = weight((float)xd, p.top) / p.z;
            take = (drafted ? u * (weight((float)yd, q.top) / q.z) : u) < pd;
        }
        if (wrong || !tested) break;
        if (!take) { refused = true; break; }
        taken++;
    }

    // ---- the draw
    const bool drafted = refused && a.draft;
    const int without = refused && !a.draft ? d : -1;     // a proposal without a distribution: d alone is left out
    const double u = wrong || greedy ? 0.0 : __ldg(a.u + o1 - 1);
    double total = 0.0, before = 0.0;
    int answer = -1;
    // from the sums of the sub-chunks: the block and the sub-chunk of the aim; false: none here.  Every block finds the same total.
    auto place = [&](int& sub, double& from) {
        double sum = 0.0;
        __syncthreads();
        if (warp == 0) {                       // inclusive sums over the block's sub-chunks, 32 at a time
            for (int base = 0; base < s1 - s0; base += 32) {
                double v = base + lane < s1 - s0 ? sub_sum[base + lane] : 0.0;
                const uint32_t some = __ballot_sync(0xFFFFFFFFu, v > 0.0);
                if (lane == 0) sh.mass[base / 32] = some;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const double w = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += w; }
                v += sum;
                if (base + lane < s1 - s0) sub_sum[base + lane] = v;
                sum = __shfl_sync(0xFFFFFFFFu, v, 31);
            }
            if (lane < nc) cluster.map_shared_rank(&sh, lane)->sums[c] = sum;
        }
        if (tid == 0) sh.unsure = 0;
        cluster.sync();
        total = 0.0;
        for (int b = 0; b < nc; b++) { if (b == c) before = total; total += sh.sums[b]; }
        const double aim = u * total;
        int block = -1, last = 0;
        double run = 0.0;
        for (int b = 0; b < nc; b++) {
            const double next = run + sh.sums[b];
            if (next > run) { last = b; if (block < 0 && next > aim) block = b; }
            run = next;
        }
        if ((block < 0 ? last : block) != c) return false;
        // the first sub-chunk with mass that passes the aim, or the last one with mass (neighbouring sums are added up in different
        // orders, so that they may differ where nothing was added)
        const int count = s1 - s0;
        int first = 0x7FFFFFFF, grows = 0;
        for (int i = tid; i < count; i += NT) {
            if (sh.mass[i >> 5] >> (i & 31) & 1) {
                grows = i;
                if (before + sub_sum[i] > aim) first = min(first, i);
            }
        }
        if (tid == 0) { sh.hit = 0x7FFFFFFF; sh.warp_u[0] = 0; }
        __syncthreads();
        if (first != 0x7FFFFFFF) atomicMin(&sh.hit, first);
        if (grows) atomicMax(&sh.warp_u[0], (uint32_t)grows);
        __syncthreads();
        sub = sh.hit == 0x7FFFFFFF ? (int)sh.warp_u[0] : sh.hit;
        from = before + (sub ? sub_sum[sub - 1] : 0.0);
        return true;
    };
    auto finish = [&]() {                      // (one thread)
        a.accepted[request] = taken;
        a.token[request] = answer;
        a.logprob[request] = (float)(((double)(float)target.entry(answer) - (double)p.top) / (double)t - log(p.z));
        a.status[request] = IMM_OK;
    };
    bool done = wrong || greedy;
    if (!done && quick_done) {
        const QuickRest<R> rest{target, draft, factor, 1.f / qp.z, drafted ? 1.f / qq.z : 0.f, qp.ref, qq.ref, without};
        put(quick_sums(rest, s0, s1, weight, sub_sum, sh));
        int sub;
        double from;
        const bool mine = place(sub, from);
        together(p);
        if (!wrong) {
            if (mine && warp == 0) {
                // Running sum less aim are the rests up to there times 1 - u, less those behind times u: off by no more than the rests are
                // together, each by its weight (log2 of which is that of the sum at most), three half-steps, and twenty of its sub-chunk's
                // sum, of p and of q.  What 1 / Z is off by is the same factor of p everywhere, and matters beside q's only.
                const float of_p = off_by(fmaxf(40.f, log2f(qp.z))) + 23 * 0x1p-24f, of_q = off_by(fmaxf(40.f, log2f(qq.z))) + 23 * 0x1p-24f;
                const float off = drafted ? of_p + doubt_p + of_q + doubt_q : of_p;
                bool sure;
                answer = entry_of<QuickRest<R>, V>(rest, s0 + sub, n, from, u * total, (double)off, sure);
                if (sure) { if (lane == 0) finish(); }
                else if (lane < nc) cluster.map_shared_rank(&sh, lane)->unsure = 1;
            }
            cluster.sync();
            done = sh.unsure == 0;            // (cleared behind the next barrier of the block)
        }
    }
    if (!done && !wrong) {
        exact(!quick_done, drafted);
        if (!wrong) {
            Rest<R> rest{target, draft, weight, 1.0 / p.z, drafted ? 1.0 / q.z : 0.0, p.top, q.top, without};
            int sub;
            double from;
            bool mine;
            for (;;) {
                rest_sums(rest, s0, s1, sub_sum);
                mine = place(sub, from);
                if (total > 0.0 || (rest.iq == 0.0 && rest.without < 0)) break;
                rest.iq = 0.0;                // p and q differ by rounding only: the draw is p's
                rest.without = -1;
                cluster.sync();               // (the sums have been read)
            }
            if (mine && warp == 0) {
                bool sure;
                answer = entry_of<Rest<R>, V>(rest, s0 + sub, n, from, u * total, 0.0, sure);
                if (lane == 0) finish();
            }
        }
    }
    if ((wrong || greedy) && c == 0 && tid == 0) {
        a.accepted[request] = wrong ? 0 : taken;
        a.token[request] = wrong ? -1 : p.index;
        a.logprob[request] = wrong ? NAN : 0.f;
        a.status[request] = wrong ? IMM_ERR_ARG : IMM_OK;
    }
    cluster.sync();                           // (no block leaves while another may store into its memory, or read it)
}

template <typename T, bool ALIGNED>
cudaError_t launch(const Args& a, int64_t requests, cudaStream_t st)
{
    constexpr int V = Row<T, ALIGNED>::V;
    const int nsub = (int)(((a.n + V - 1) / V + PIECES - 1) / PIECES);
    auto kernel = verify_kernel<T, ALIGNED>;
    constexpr int MOST = (IMM_LDD_MAX_N / V + PIECES - 1) / PIECES;
    static_assert(MOST <= MOST_SUBS, "a bit per sub-chunk");
    static_assert(MOST * sizeof(double) + sizeof(Shared) <= 48 * 1024, "sums of the longest row in one block");
    // once per device: permission for large clusters, and the largest it can hold
    static std::atomic<int> largest[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    int most = dev < 64 ? largest[dev].load(std::memory_order_relaxed) : 0;
    if (most == 0) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t ask;
        memset(&ask, 0, sizeof(ask));
        ask.gridDim = dim3(MAX_CLUSTER);
        ask.blockDim = dim3(NT);
        ask.dynamicSmemBytes = MOST * sizeof(double);
        e = cudaOccupancyMaxPotentialClusterSize(&most, kernel, &ask);
        if (e != cudaSuccess) return e;
        most = most >= MAX_CLUSTER ? MAX_CLUSTER : most >= 8 ? 8 : 1;
        if (dev < 64) largest[dev].store(most, std::memory_order_relaxed);
    }
    // blocks per request: more while the requests leave places on the GPU and every warp still has a sub-chunk
    // (requests differ in the rows they read: twice as many blocks as are resident even that out)
    const int64_t slots = 2 * (int64_t)BLOCKS_PER_SM * imm::sm_count();
    int nc = 1;
    // (sixteen only for a few: many clusters of sixteen do not fit the GPU at once)
    while (nc < (requests * MAX_CLUSTER > imm::sm_count() && most > 8 ? 8 : most) && nsub > nc * NW && requests * nc * 2 <= slots) nc *= 2;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(requests * nc));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = (size_t)((nsub + nc - 1) / nc) * sizeof(double);
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

}  // namespace imm_verify_ns

extern "C" int imm_verify_draft(const imm_verify_desc* desc_host, void* stream)
{
    using namespace imm_verify_ns;
    if (!desc_host || desc_host->reserved || desc_host->reserved2) return IMM_ERR_ARG;
    const imm_verify_desc& d = *desc_host;
    if (d.dtype != IMM_F32 && d.dtype != IMM_BF16 && d.dtype != IMM_F16) return IMM_ERR_ARG;
    if (d.requests > 0 && (!d.d_offsets || !d.d_accepted || !d.d_token || !d.d_logprob || !d.d_status)) return IMM_ERR_ARG;
    if (d.requests > 0 && d.tokens > 0 && (!d.d_target || !d.d_tokens || !d.d_u)) return IMM_ERR_ARG;
    if (d.requests < 0 || d.requests > (1 << 20) || d.tokens < 0 || d.tokens > IMM_LDD_MAX_STEPS || d.drafts < 0 || d.n <= 0 || d.n > IMM_LDD_MAX_N || d.ldt < d.n ||
        (d.d_draft && d.ldd < d.n))
        return IMM_ERR_SHAPE;
    const uintptr_t es = d.dtype == IMM_F32 ? 4 : 2;
    if ((uintptr_t)d.d_target % es || (uintptr_t)d.d_draft % es || (uintptr_t)d.d_tokens % 4 || (uintptr_t)d.d_offsets % 8 || (uintptr_t)d.d_u % 8 ||
        (uintptr_t)d.d_temperature % 4 || (uintptr_t)d.d_accepted % 4 || (uintptr_t)d.d_token % 4 || (uintptr_t)d.d_logprob % 4 ||
        (uintptr_t)d.d_status % 4)
        return IMM_ERR_ALIGN;
    if (d.requests == 0) return IMM_OK;
    Args a{};
    a.target = d.d_target; a.draft = d.d_draft; a.tokens = d.d_tokens; a.offsets = d.d_offsets; a.u = d.d_u;
    a.temperature_of = d.d_temperature; a.accepted = d.d_accepted; a.token = d.d_token; a.logprob = d.d_logprob; a.status = d.d_status;
    a.rows = d.tokens; a.drafts = d.drafts; a.n = d.n; a.ldt = d.ldt; a.ldd = d.ldd; a.temperature = d.temperature;
    const bool aligned = ((uintptr_t)d.d_target | (uintptr_t)(es * d.ldt) | (uintptr_t)d.d_draft | (uintptr_t)(d.d_draft ? es * d.ldd : 0)) % 16 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (d.dtype == IMM_F32) e = aligned ? launch<float, true>(a, d.requests, st) : launch<float, false>(a, d.requests, st);
    else if (d.dtype == IMM_BF16) e = aligned ? launch<__nv_bfloat16, true>(a, d.requests, st) : launch<__nv_bfloat16, false>(a, d.requests, st);
    else e = aligned ? launch<__half, true>(a, d.requests, st) : launch<__half, false>(a, d.requests, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
