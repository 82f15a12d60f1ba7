// Root-mean-square norm with residual addition and int8 output (sm_100a) and its C ABI (declared in imm.h).
//
//   imm_rmsnorm_quant   h = x + residual;  t = h * weight;  q = round(127 t / max|t|);  scale = max|t| r / 127
//
// One streaming pass over the rows (x and residual read, h and q written, each once), bound by HBM: a block
// takes a row and keeps it in registers between the reductions and the rounding.  Measured with a residual: 8192 x 4096
// bf16 42.8 us (5.5 TB/s, 0.84 of the copy rate); 2047 x 14336 float32 in groups of 128 columns 82.5 us (4.6 TB/s).
//
// The rounding.  q is defined on the exact products in float64 (reproducible anywhere); 127 t / a in float32 is
// off by less than 127 * 2^-22 < 3.1e-5, so only values that near to a border between two integers -- one entry in
// fifteen thousand -- are worked out again in float64.  Products of two 16-bit floats are exact in float32, so
// their maximum is too; with float32 factors the exact maximum is taken, where an entry needs it, over the vectors
// whose float32 maximum is the row's.  Rows whose maximum is so large or small that float32 products may overflow
// or vanish take the float64 path altogether.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_norm {

struct Args {
    const void *x, *residual, *weight;
    void* h;
    int8_t* q;
    float* scale;
    int64_t rows, ldx, ldr, ldh, ldq;
    int32_t cols, group;
    double eps;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ double max_nan(double a, double b) { return a != a ? a : b != b ? b : fmax(a, b); }
// float32 products neither overflow nor lose bits that matter while the largest is in this range (false for a NaN)
__device__ __forceinline__ bool in_range(float top) { return top >= 0x1p-60f && top <= 0x1p100f; }

// The exact maximum of a group's products; dead: the group or its row is not finite.
struct Peak { double wide; bool dead; };

__device__ __forceinline__ Peak make_peak(double wide, bool row_fine) { return Peak{wide, !row_fine || !(wide < (double)INFINITY)}; }

// the definition, for the few entries that float32 does not decide
__device__ __noinline__ int8_t round_wide(float h, float w, const Peak& p)
{
    if (p.dead || p.wide == 0.0) return 0;
    return (int8_t)(int)rint((double)h * (double)w * 127.0 / p.wide);
}

__device__ __forceinline__ float group_scale(const Peak& p, double inverse)
{
    if (p.dead) return NAN;
    return p.wide == 0.0 ? 0.f : (float)(p.wide * inverse / 127.0);
}

// V entries of a row as they lie in memory (16 bytes; V = 1: a single entry, for rows that are not 16-byte aligned)
template <typename T, int V> struct Raw { uint4 w; };
template <typename T> struct Raw<T, 1> { T w; };

template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_raw(const T* p) { return *reinterpret_cast<const Raw<T, V>*>(p); }
template <typename T, int V> __device__ __forceinline__ void store_raw(T* p, const Raw<T, V>& r) { *reinterpret_cast<Raw<T, V>*>(p) = r; }

template <typename T, int V> __device__ __forceinline__ void unpack(const Raw<T, V>& r, float (&f)[V])
{
    if constexpr (V == 1) f[0] = to_f(r.w);
    else {
        const uint32_t w[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(w[i]);
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                f[2 * i] = p.x; f[2 * i + 1] = p.y;
            }
        }
    }
}
// each value rounded to T once
template <typename T, int V> __device__ __forceinline__ Raw<T, V> pack(const float (&f)[V])
{
    Raw<T, V> r;
    if constexpr (V == 1) r.w = from_f<T>(f[0]);
    else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&p);
            } else {
                const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
        }
        r.w = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}
// V weights of any type
template <typename W, int V> __device__ __forceinline__ void load_weights(const W* p, float (&f)[V])
{
    if constexpr (V * sizeof(W) == 32) {
        float a[4], b[4];
        unpack<W, 4>(load_raw<W, 4>(p), a);
        unpack<W, 4>(load_raw<W, 4>(p + 4), b);
#pragma unroll
        for (int i = 0; i < 4; i++) { f[i] = a[i]; f[4 + i] = b[i]; }
    } else unpack<W, V>(load_raw<W, V>(p), f);
}

// float32's error of 127 t / a, a little more than it: four roundings, or two where products are exact (127 * 2^-22 or 2^-23)
template <typename T, typename W> constexpr float BORDER = sizeof(T) == 2 && sizeof(W) == 2 ? 0.5f - 1.6e-5f : 0.5f - 3.1e-5f;
constexpr float MAGIC = 12582912.f;            // 1.5 * 2^23: v + MAGIC has round(v) in its low bits

// q of V products; returns the largest distance of a value to its rounding (over BORDER: doubtful)
template <int V> __device__ __forceinline__ float round_store(int8_t* q, const float (&prod)[V], float inv)
{
    uint32_t word[V >= 4 ? V / 4 : 1] = {};
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const float v = prod[e] * inv, m = v + MAGIC;
        off = fmaxf(off, fabsf(v - (m - MAGIC)));
        const uint32_t b = __float_as_uint(m);
        if constexpr (V == 1) word[0] = b;
        else if (e % 4 == 0) word[e / 4] = b & 0xFFu;
        else word[e / 4] = __byte_perm(word[e / 4], b, e % 4 == 1 ? 0x3240 : e % 4 == 2 ? 0x3410 : 0x4210);
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(word[0], word[1]);
    else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(q) = word[0];
    else q[0] = (int8_t)word[0];
    return off;
}

// h = x + residual of V entries, rounded to T and written; products with the weights; the sum of squares goes on
template <typename T, typename W, int V>
__device__ __forceinline__ float take(const Raw<T, V>& hx, const Raw<T, V>& hr, bool more, T* hout, const W* w, float (&prod)[V], float& sum)
{
    float h[V], wt[V], peak = 0.f;
    load_weights<W, V>(w, wt);
    unpack<T, V>(hx, h);
    Raw<T, V> kept = hx;
    if (more) {
        float add[V];
        unpack<T, V>(hr, add);
#pragma unroll
        for (int e = 0; e < V; e++) h[e] += add[e];
        kept = pack<T, V>(h);
        unpack<T, V>(kept, h);
    }
    if (hout) store_raw<T, V>(hout, kept);
#pragma unroll
    for (int e = 0; e < V; e++) {
        sum = fmaf(h[e], h[e], sum);
        prod[e] = h[e] * wt[e];
        peak = max_nan(peak, fabsf(prod[e]));
    }
    return peak;                               // the largest |product|, or NaN
}

// Vectors of a row that does not begin on a 16-byte boundary (x, residual and h all at the same distance from one): the row's
// aligned 16-byte granules, of which the first and the last belong to it in part.  `first`, `last`: the entries of a vector
// that do.
__device__ __forceinline__ float weight_at(const float* p) { return *p; }
__device__ __forceinline__ float weight_at(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float weight_at(const __half* p) { return __half2float(*p); }

template <typename W, int V> __device__ __forceinline__ void load_weights_anywhere(const W* p, int first, int last, float (&f)[V])
{
    if (first == 0 && last == V) {
        constexpr int STEP = 16 / (int)sizeof(W);
#pragma unroll
        for (int b = 0; b < V; b += STEP) {    // 16 bytes from the two aligned vectors that they lie in
            const uint32_t sh = (uint32_t)(uintptr_t)(p + b) & 15u;
            const uint4* a = reinterpret_cast<const uint4*>((uintptr_t)(p + b) & ~(uintptr_t)15);
            const uint4 lo = __ldg(a), hi = sh ? __ldg(a + 1) : lo;
            const uint32_t src[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, bits = 8 * (sh & 3u);
            uint32_t w[5];
#pragma unroll
            for (int i = 0; i < 5; i++) {      // (the shift is the same for all lanes)
                w[i] = src[i];
                if (sh >= 12) w[i] = src[i + 3 < 8 ? i + 3 : 7];
                else if (sh >= 8) w[i] = src[i + 2];
                else if (sh >= 4) w[i] = src[i + 1];
            }
            Raw<W, STEP> r;
            r.w = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                             __funnelshift_r(w[3], w[4], bits));
            float g[STEP];
            unpack<W, STEP>(r, g);
#pragma unroll
            for (int e = 0; e < STEP; e++) f[b + e] = g[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = e >= first && e < last ? weight_at(p + e) : 0.f;
    }
}

template <typename T, typename W, int V>
__device__ __forceinline__ float take_anywhere(const Raw<T, V>& hx, const Raw<T, V>& hr, bool more, T* hout, const W* w, int first, int last,
                                               float (&prod)[V], float& sum)
{
    float h[V], wt[V], peak = 0.f;
    load_weights_anywhere<W, V>(w, first, last, wt);
    unpack<T, V>(hx, h);
    Raw<T, V> kept = hx;
    if (more) {
        float add[V];
        unpack<T, V>(hr, add);
#pragma unroll
        for (int e = 0; e < V; e++) h[e] += add[e];
        kept = pack<T, V>(h);
        unpack<T, V>(kept, h);
    }
    const bool whole = first == 0 && last == V;
    if (hout) {
        if (whole) store_raw<T, V>(hout, kept);
        else {
#pragma unroll
            for (int e = 0; e < V; e++) if (e >= first && e < last) hout[e] = from_f<T>(h[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < V; e++) {
        if (!whole && (e < first || e >= last)) h[e] = 0.f;                // (another row's, whatever it is)
        sum = fmaf(h[e], h[e], sum);
        prod[e] = h[e] * wt[e];
        peak = max_nan(peak, fabsf(prod[e]));
    }
    return peak;
}

template <int V> __device__ __forceinline__ float round_store_anywhere(int8_t* q, const float (&prod)[V], float inv, int first, int last)
{
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const float v = prod[e] * inv, m = v + MAGIC;
        off = fmaxf(off, fabsf(v - (m - MAGIC)));
        if (e >= first && e < last) q[e] = (int8_t)__float_as_uint(m);
    }
    return off;
}

// The entries of a vector that float32 does not decide, or all of them, by the definition
template <typename T, typename W, int V>
__device__ __forceinline__ void redo(int8_t* q, const T* held, const W* w, float inv, bool all, const Peak& p, int first = 0, int last = V)
{
#pragma unroll 1
    for (int e = first; e < last; e++) {
        const float h = to_f(held[e]), wt = to_f(w[e]), v = h * wt * inv;
        if (all || fabsf(v - rintf(v)) > BORDER<T, W>) q[e] = round_wide(h, wt, p);
    }
}

// A row per block, or per warp (WARP: short rows).  A thread holds the products of VPT vectors in registers, vector
// i * nt + tid being its i-th, from the pass that reads x and writes h to the rounding.  Sums of squares: float32
// within a thread (at most 64 terms), float64 above; a sum that leaves float32's range is taken again in float64.
// Entries next to a border are found by one maximum per vector and redone after the others, from h as it was written.
// Four vectors a thread measured best for 4096 bf16 columns (45 us for 8192 rows; one 66, two 49, eight 53).
constexpr int ROWS = 8;                        // rows per block of the warp form

template <typename T, typename W, int V, int VPT, bool WARP, bool SHIFTED>
__global__ void __launch_bounds__(WARP ? 32 * ROWS : VPT * V <= 16 ? 1024 : 512) norm_rows_kernel(const Args a)
{
    constexpr bool EXACT = sizeof(T) == 2 && sizeof(W) == 2;               // products are exact in float32
    __shared__ double s_sum[32];
    __shared__ float s_seen[32];
    __shared__ unsigned long long s_wide;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tid = WARP ? lane : threadIdx.x, nt = WARP ? 32 : blockDim.x, nw = nt >> 5;
    const int64_t r = WARP ? (int64_t)blockIdx.x * ROWS + warp : blockIdx.x;
    if (WARP && r >= a.rows) return;
    const T* x = (const T*)a.x + r * a.ldx;
    const T* res = a.residual ? (const T*)a.residual + r * a.ldr : nullptr;
    T* hout = a.h ? (T*)a.h + r * a.ldh : nullptr;
    const T* held = hout ? hout : x;           // h in memory, once it is written
    const W* w = (const W*)a.weight;
    int8_t* q = a.q + r * a.ldq;
    // entries of the first vector that lie before the row
    const int shift = SHIFTED ? (int)(((uintptr_t)x & 15) / sizeof(T)) : 0;
    const int nvec = SHIFTED ? (shift + a.cols + V - 1) / V : a.cols / V;
    auto first_of = [&](int c) { return SHIFTED ? max(0, -c) : 0; };
    auto last_of = [&](int c) { return SHIFTED ? min(V, a.cols - c) : V; };
    if (!WARP && tid == 0) s_wide = 0;
    auto total = [&](double v) {               // over the row's threads, the same for all of them
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if (!WARP) {
            __syncthreads();
            if (lane == 0) s_sum[warp] = v;
            __syncthreads();
            v = 0.0;
            for (int i = 0; i < nw; i++) v += s_sum[i];
        }
        return v;
    };

    Raw<T, V> hx[VPT], hr[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++)
        if (i * nt + tid < nvec) {
            hx[i] = load_raw<T, V>(x + (i * nt + tid) * V - shift);
            if (res) hr[i] = load_raw<T, V>(res + (i * nt + tid) * V - shift);
        }
    float prod[VPT][V], peak[VPT], sum = 0.f, seen = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        peak[i] = 0.f;
        const int c = (i * nt + tid) * V - shift;
        if (i * nt + tid < nvec) {
            if constexpr (SHIFTED)
                peak[i] = take_anywhere<T, W, V>(hx[i], hr[i], res != nullptr, hout ? hout + c : nullptr, w + c, first_of(c), last_of(c), prod[i], sum);
            else peak[i] = take<T, W, V>(hx[i], hr[i], res != nullptr, hout ? hout + c : nullptr, w + c, prod[i], sum);
        }
        seen = max_nan(seen, peak[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) seen = max_nan(seen, __shfl_xor_sync(0xFFFFFFFFu, seen, o));
    if (!WARP && lane == 0) s_seen[warp] = seen;
    double wide_sum = total((double)sum);
    if (!WARP) for (int i = 0; i < nw; i++) seen = max_nan(seen, s_seen[i]);
    if (!(wide_sum < 1e37) || wide_sum < 1e-25) {              // squares beyond float32, or lost below it: once more in float64
        double again = 0.0;
#pragma unroll 1
        for (int i = 0; i < VPT; i++)
            if (i * nt + tid < nvec) {
                const int c = (i * nt + tid) * V - shift;
                for (int e = first_of(c); e < last_of(c); e++) { const double v = (double)to_f(held[c + e]); again += v * v; }
            }
        wide_sum = total(again);
    }
    const bool row_fine = wide_sum < (double)INFINITY, out = !in_range(seen);

    unsigned doubtful = 0;                     // bit i: an entry of vector i next to a border, or a row out of range
    const float inv = 127.f / seen;
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        const int c = (i * nt + tid) * V - shift;
        if (c >= a.cols) continue;
        float off;
        if constexpr (SHIFTED) off = round_store_anywhere<V>(q + c, prod[i], inv, first_of(c), last_of(c));
        else off = round_store<V>(q + c, prod[i], inv);
        if (off > BORDER<T, W> || out || !row_fine) doubtful |= 1u << i;
    }

    // the entries that float32 does not decide, and rows outside its range: by the definition
    double wide = (double)seen;
    if (WARP ? __any_sync(0xFFFFFFFFu, doubtful != 0) : __syncthreads_or((int)doubtful)) {
        if (!EXACT || out) {
            // the largest product exactly: among the vectors whose float32 maximum is the row's, or among all
            double mine = 0.0;
#pragma unroll 1
            for (int i = 0; i < VPT; i++) {
                float top = 0.f;
#pragma unroll
                for (int z = 0; z < VPT; z++) if (z == i) top = peak[z];
                const int c = (i * nt + tid) * V - shift;
                if (c < a.cols && (out || top == seen))
                    for (int e = first_of(c); e < last_of(c); e++) mine = max_nan(mine, fabs((double)to_f(held[c + e]) * (double)to_f(w[c + e])));
            }
            if (WARP) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) mine = max_nan(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, o));
                wide = mine;
            } else {
                // (bits of doubles that are not negative are ordered as they are; NaN above infinity)
                if (mine > 0.0 || mine != mine) atomicMax(&s_wide, (unsigned long long)__double_as_longlong(fabs(mine)));
                __syncthreads();
                wide = __longlong_as_double((long long)s_wide);
            }
        }
        const Peak p = make_peak(wide, row_fine);
#pragma unroll 1
        for (int i = 0; i < VPT; i++) {
            const int c = (i * nt + tid) * V - shift;
            if ((doubtful >> i) & 1u) redo<T, W, V>(q + c, held + c, w + c, inv, out || !row_fine, p, first_of(c), last_of(c));
        }
    }
    if (tid == 0) {                            // (a float64 root and a division, by one warp)
        const Peak p = make_peak(wide, row_fine);
        a.scale[r] = p.dead ? NAN : wide == 0.0 ? 0.f : (float)(wide / (sqrt(wide_sum / (double)a.cols + a.eps) * 127.0));
    }
}

// Groups of 128 columns: the rounding needs the group's maximum only, so a row streams through its block (a thread's next vector
// on its way while one is worked on) and nothing of it is held.  A group's maximum waits in its scale's place until
// the row's sum is known; groups outside float32's range are marked there and worked out again at the end.
template <typename T, typename W, int V, int NT>
__global__ void __launch_bounds__(NT, 1280 / NT) norm_groups_kernel(const Args a)
{
    constexpr bool EXACT = sizeof(T) == 2 && sizeof(W) == 2;
    constexpr int GL = 128 / V, NW = NT / 32;        // lanes of a group
    constexpr float MARK = -1.f;
    __shared__ double s_sum[NW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned mates = GL == 32 ? 0xFFFFFFFFu : 0xFFFFu << (lane & 16);
    const int64_t r = blockIdx.x;
    const T* x = (const T*)a.x + r * a.ldx;
    const T* res = a.residual ? (const T*)a.residual + r * a.ldr : nullptr;
    T* hout = a.h ? (T*)a.h + r * a.ldh : nullptr;
    const T* held = hout ? hout : x;
    const W* w = (const W*)a.weight;
    int8_t* q = a.q + r * a.ldq;
    float* scale = a.scale + r * (a.cols / 128);
    const int nvec = a.cols / V, rounds = (nvec + NT - 1) / NT;
    // the exact maximum of the group of vector v, by its lanes
    auto widest = [&](int c, bool live) {
        double wide = 0.0;
        if (live)
            for (int e = 0; e < V; e++) wide = max_nan(wide, fabs((double)to_f(held[c + e]) * (double)to_f(w[c + e])));
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1) wide = max_nan(wide, __shfl_xor_sync(mates, wide, o));
        return wide;
    };

    Raw<T, V> hx, hr, nx, nr;
    auto fetch = [&](int i) {
        const int v = i * NT + tid;
        if (v < nvec) {
            nx = load_raw<T, V>(x + v * V);
            if (res) nr = load_raw<T, V>(res + v * V);
        }
    };
    fetch(0);
    double wide_sum = 0.0;
    for (int i = 0; i < rounds; i++) {
        hx = nx; hr = nr;
        fetch(i + 1);                          // (two vectors ahead, with fewer blocks per SM, measured slower)
        const int v = i * NT + tid, c = v * V;
        const bool live = v < nvec;
        float prod[V], peak = 0.f, sum = 0.f;
        if (live) peak = take<T, W, V>(hx, hr, res != nullptr, hout ? hout + c : nullptr, w + c, prod, sum);
        if (!(sum < 1e37f) || sum < 1e-25f) {              // squares beyond float32, or lost below it
            double again = 0.0;
            if (live)
                for (int e = 0; e < V; e++) { const double h = (double)to_f(held[c + e]); again += h * h; }
            wide_sum += again;
        } else wide_sum += (double)sum;
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1) peak = max_nan(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, o));
        if (!live) continue;
        const bool out = !in_range(peak);
        const float inv = 127.f / peak;
        const bool doubt = round_store<V>(q + c, prod, inv) > BORDER<T, W> || out;
        if (__any_sync(mates, doubt)) {                    // (groups are whole: live or not together)
            double wide = (double)peak;
            if (!EXACT || out) wide = widest(c, true);
            const Peak p = make_peak(wide, true);
            if (doubt) redo<T, W, V>(q + c, held + c, w + c, inv, out, p);
        }
        if (lane % GL == 0) scale[c / 128] = out ? MARK : peak;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wide_sum += __shfl_xor_sync(0xFFFFFFFFu, wide_sum, o);
    if (lane == 0) s_sum[warp] = wide_sum;
    __syncthreads();
    wide_sum = 0.0;
#pragma unroll
    for (int i = 0; i < NW; i++) wide_sum += s_sum[i];
    const bool row_fine = wide_sum < (double)INFINITY;
    const double factor = 1.0 / (sqrt(wide_sum / (double)a.cols + a.eps) * 127.0);
    for (int i = 0; i < rounds; i++) {         // (a thread reads only scales that it wrote itself)
        const int v = i * NT + tid, c = v * V;
        if (v >= nvec) break;
        const float peak = __shfl_sync(mates, lane % GL == 0 ? scale[c / 128] : 0.f, lane & ~(GL - 1));
        double wide = (double)peak;
        if (peak == MARK) wide = widest(c, true);
        if (!row_fine)
            for (int e = 0; e < V; e++) q[c + e] = 0;
        const Peak p = make_peak(wide, row_fine);
        if (lane % GL == 0) scale[c / 128] = p.dead ? NAN : wide == 0.0 ? 0.f : (float)(wide * factor);
    }
}

// Rows too long for a block's registers: read again in the second pass (h from where it was written).
template <typename T, typename W, int NT>
__global__ void __launch_bounds__(NT) norm_long_kernel(const Args a)
{
    constexpr int NW = NT / 32;
    __shared__ double s_sum[NW], s_peak[NW];
    __shared__ float s_top[NW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t r = blockIdx.x;
    const T* x = (const T*)a.x + r * a.ldx;
    const T* res = a.residual ? (const T*)a.residual + r * a.ldr : nullptr;
    T* hout = a.h ? (T*)a.h + r * a.ldh : nullptr;
    const W* w = (const W*)a.weight;
    int8_t* q = a.q + r * a.ldq;

    double sum = 0.0, peak = 0.0;
    float top = 0.f;
    for (int j = tid; j < a.cols; j += NT) {
        float v = to_f(x[j]);
        if (res) v = to_f(from_f<T>(v + to_f(res[j])));
        if (hout) hout[j] = from_f<T>(v);
        const float wt = to_f(w[j]);
        sum += (double)v * (double)v;
        peak = fmax(peak, fabs((double)v * (double)wt));
        top = max_nan(top, fabsf(v * wt));
    }
    double bsum = sum, bpeak = peak;
    float btop = top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        bsum += __shfl_xor_sync(0xFFFFFFFFu, bsum, o);
        bpeak = fmax(bpeak, __shfl_xor_sync(0xFFFFFFFFu, bpeak, o));
        btop = max_nan(btop, __shfl_xor_sync(0xFFFFFFFFu, btop, o));
    }
    if (lane == 0) { s_sum[warp] = bsum; s_peak[warp] = bpeak; s_top[warp] = btop; }
    __syncthreads();
    bsum = 0.0; bpeak = 0.0; btop = 0.f;
    for (int i = 0; i < NW; i++) { bsum += s_sum[i]; bpeak = fmax(bpeak, s_peak[i]); btop = max_nan(btop, s_top[i]); }
    const bool row_fine = bsum < (double)INFINITY;
    const double inverse = 1.0 / sqrt(bsum / (double)a.cols + a.eps);
    const T* again = hout ? hout : x;

    if (a.group == 0) {
        const Peak p = make_peak(btop == btop ? bpeak : (double)NAN, row_fine);
        for (int j = tid; j < a.cols; j += NT) q[j] = round_wide(to_f(again[j]), to_f(w[j]), p);
        if (tid == 0) a.scale[r] = group_scale(p, inverse);
    } else {
        // groups of 128 columns: NT is a multiple of 128, so a group is four neighbouring warps at one i
        const int groups = a.cols / a.group;
        __shared__ double g_peak[NW];
        __shared__ float g_top[NW];
        const int rounds = (a.cols + NT - 1) / NT;
        for (int i = 0; i < rounds; i++) {
            const int j = tid + i * NT;
            float v = 0.f, wt = 0.f;
            if (j < a.cols) { v = to_f(again[j]); wt = to_f(w[j]); }
            double gp = fabs((double)v * (double)wt);
            float gt = fabsf(v * wt);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                gp = fmax(gp, __shfl_xor_sync(0xFFFFFFFFu, gp, o));
                gt = max_nan(gt, __shfl_xor_sync(0xFFFFFFFFu, gt, o));
            }
            __syncthreads();
            if (lane == 0) { g_peak[warp] = gp; g_top[warp] = gt; }
            __syncthreads();
            const int w0 = warp & ~3;
            gp = 0.0; gt = 0.f;
            for (int k = 0; k < 4; k++) { gp = fmax(gp, g_peak[w0 + k]); gt = max_nan(gt, g_top[w0 + k]); }
            const Peak p = make_peak(gt == gt ? gp : (double)NAN, row_fine);
            if (j < a.cols) {
                q[j] = round_wide(v, wt, p);
                if ((j & 127) == 0) a.scale[r * groups + j / 128] = group_scale(p, inverse);
            }
        }
    }
}


template <typename T, typename W, int V, int VPT, bool SHIFTED = false>
cudaError_t launch_rows(const Args& a, int nt, cudaStream_t st)
{
    norm_rows_kernel<T, W, V, VPT, false, SHIFTED><<<(unsigned)a.rows, nt, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, typename W, int V, int VPT, bool SHIFTED = false>
cudaError_t launch_warps(const Args& a, cudaStream_t st)
{
    norm_rows_kernel<T, W, V, VPT, true, SHIFTED><<<(unsigned)((a.rows + ROWS - 1) / ROWS), 32 * ROWS, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t launch(const Args& a, cudaStream_t st)
{
    constexpr int V = 16 / (int)sizeof(T);
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.h | (uintptr_t)a.weight | (uintptr_t)(a.ldx * sizeof(T)) |
                          (a.residual ? (uintptr_t)(a.ldr * sizeof(T)) : 0) | (a.h ? (uintptr_t)(a.ldh * sizeof(T)) : 0);
    const bool vec = all % 16 == 0 && ((uintptr_t)a.q | (uintptr_t)a.ldq) % V == 0 && a.cols % V == 0;
    auto odd = [](const void* p, const void* o) { return p && (((uintptr_t)p ^ (uintptr_t)o) & 15); };
    const bool even = !odd(a.residual, a.x) && !odd(a.h, a.x) && (!a.residual || (a.ldr - a.ldx) * (int64_t)sizeof(T) % 16 == 0) &&
                      (!a.h || (a.ldh - a.ldx) * (int64_t)sizeof(T) % 16 == 0);
    const int nvec = vec ? a.cols / V : a.cols;
    const bool few = a.rows <= imm::sm_count();            // then a row's time counts: many threads for it
    auto threads = [&](int per) { return ((nvec + per - 1) / per + 31) / 32 * 32; };
    if (a.group) {
        if (vec) {
            // short rows: a smaller block, so that its last round is not mostly empty
            if (nvec <= 512 && !few) norm_groups_kernel<T, W, V, 64><<<(unsigned)a.rows, 64, 0, st>>>(a);
            else if (nvec <= 1024 && !few) norm_groups_kernel<T, W, V, 128><<<(unsigned)a.rows, 128, 0, st>>>(a);
            else norm_groups_kernel<T, W, V, 256><<<(unsigned)a.rows, 256, 0, st>>>(a);
            return cudaGetLastError();
        }
    } else if (vec) {
        if (few && threads(1) <= 1024) return launch_rows<T, W, V, 1>(a, threads(1), st);
        if (nvec <= 32) return launch_warps<T, W, V, 1>(a, st);
        if (nvec <= 64) return launch_warps<T, W, V, 2>(a, st);
        if (nvec <= 128) return launch_warps<T, W, V, 4>(a, st);
        if (threads(4) <= (V == 8 ? 512 : 1024)) return launch_rows<T, W, V, 4>(a, threads(4), st);
        if constexpr (V == 8)                  // (up to 4096 vectors, which four a thread take of 4-byte entries)
            if (threads(8) <= 512) return launch_rows<T, W, V, 8>(a, threads(8), st);
    } else if (even) {
        // rows at odd addresses, all three alike: their aligned granules (one more than the entries fill)
        const int grains = a.cols / V + 2;
        auto lanes = [&](int per) { return ((grains + per - 1) / per + 31) / 32 * 32; };
        if (few && lanes(1) <= 1024) return launch_rows<T, W, V, 1, true>(a, lanes(1), st);
        if (grains <= 32) return launch_warps<T, W, V, 1, true>(a, st);
        if (grains <= 64) return launch_warps<T, W, V, 2, true>(a, st);
        if (grains <= 128) return launch_warps<T, W, V, 4, true>(a, st);
        if (lanes(4) <= (V == 8 ? 512 : 1024)) return launch_rows<T, W, V, 4, true>(a, lanes(4), st);
        if constexpr (V == 8)
            if (lanes(8) <= 512) return launch_rows<T, W, V, 8, true>(a, lanes(8), st);
    } else {
        if (nvec <= 128 && !few) return launch_warps<T, W, 1, 4>(a, st);
        if (nvec <= 512 && !few) return launch_warps<T, W, 1, 16>(a, st);
        if (few && threads(4) <= 1024) return launch_rows<T, W, 1, 4>(a, threads(4), st);
        if (threads(16) <= 1024) return launch_rows<T, W, 1, 16>(a, threads(16), st);
    }
    norm_long_kernel<T, W, 512><<<(unsigned)a.rows, 512, 0, st>>>(a);
    return cudaGetLastError();
}

size_t elem(int dtype) { return dtype == IMM_F32 ? 4 : 2; }

}  // namespace imm_norm

extern "C" int imm_rmsnorm_quant(const imm_norm_desc* desc_host, void* stream)
{
    using namespace imm_norm;
    if (!desc_host || desc_host->reserved) return IMM_ERR_ARG;
    const auto [d_x, d_residual, d_weight, d_h, d_q, d_scale, rows, cols, ldx, ldr, ldh, ldq, eps, dtype, wdtype, group, reserved] = *desc_host;
    if (rows > 0 && (!d_x || !d_weight || !d_q || !d_scale || (d_residual && !d_h))) return IMM_ERR_ARG;
    if (dtype != IMM_F32 && dtype != IMM_BF16 && dtype != IMM_F16) return IMM_ERR_ARG;
    if (wdtype != dtype && wdtype != IMM_F32) return IMM_ERR_ARG;
    if (!(eps >= 0.0) || eps > 1e300 || (group != 0 && group != 128)) return IMM_ERR_ARG;
    if (rows < 0 || rows > ((int64_t)1 << 30) || cols <= 0 || cols > IMM_NORM_MAX_COLS) return IMM_ERR_SHAPE;
    if (ldx < cols || ldq < cols || (d_residual && ldr < cols) || (d_h && ldh < cols)) return IMM_ERR_SHAPE;
    if (group && cols % group) return IMM_ERR_SHAPE;
    const size_t es = elem(dtype);
    if ((uintptr_t)d_x % es || (uintptr_t)d_residual % es || (uintptr_t)d_h % es || (uintptr_t)d_weight % elem(wdtype) ||
        (uintptr_t)d_scale % 4)
        return IMM_ERR_ALIGN;
    if (rows == 0) return IMM_OK;
    const Args a{d_x, d_residual, d_weight, d_h, d_q, d_scale, rows, ldx, ldr, ldh, ldq, (int32_t)cols, group, eps};
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == IMM_F32) e = launch<float, float>(a, st);
    else if (dtype == IMM_BF16) e = wdtype == IMM_F32 ? launch<__nv_bfloat16, float>(a, st) : launch<__nv_bfloat16, __nv_bfloat16>(a, st);
    else e = wdtype == IMM_F32 ? launch<__half, float>(a, st) : launch<__half, __half>(a, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
