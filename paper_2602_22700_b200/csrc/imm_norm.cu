// Root-mean-square norm with residual addition and int8 output (sm_100a) and its C ABI (declared in imm.h).
//
//   imm_rmsnorm_quant   h = x + residual;  t = h * weight;  q = round(127 t / max|t|);  scale = max|t| r / 127
//
// One streaming pass over the rows (x and residual read, h and q written, each once), bound by HBM: a block
// takes a row and keeps it in registers between the reductions and the rounding.
//
// The rounding.  q is defined on the exact products in float64 (reproducible anywhere); 127 t / a in float32 is
// off by less than 127 * 2^-22 < 3.1e-5, so only values within 5e-5 of a border between two integers -- one entry
// in ten thousand -- are worked out again in float64.  Products of two 16-bit floats are exact in float32, so
// their maximum is too; with float32 factors the rounding error of the product is carried along (a fused
// multiply-add gives it exactly).  Rows whose maximum is so large or small that float32 products may overflow or
// vanish take the float64 path altogether.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

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

// What the rounding of one group needs: its maximum in both widths, and which path it takes.
struct Peak { double wide; float inv; bool slow, dead; };

__device__ __forceinline__ Peak make_peak(double wide, float narrow, bool row_fine)
{
    Peak p;
    p.wide = wide;
    p.dead = !row_fine || !(wide < (double)INFINITY);          // not finite, or NaN
    p.slow = !in_range(narrow);
    p.inv = p.slow ? 0.f : 127.f / (float)wide;
    return p;
}

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

// A block per row, the row in registers.  A thread holds VPT vectors of V entries (16 bytes; V = 1: single entries, for
// rows that are not 16-byte aligned), vector i * blockDim.x + tid being its i-th.  Sums of squares: float32 within
// a thread (at most 64 terms), float64 above; a sum that leaves float32's range is taken again in float64.
template <typename T, int V> struct Raw { T v[V]; };
template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_raw(const T* p)
{
    Raw<T, V> r;
    if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4*>(&r) = *reinterpret_cast<const uint4*>(p);
    else if constexpr (V * sizeof(T) == 32) {
        reinterpret_cast<uint4*>(&r)[0] = reinterpret_cast<const uint4*>(p)[0];
        reinterpret_cast<uint4*>(&r)[1] = reinterpret_cast<const uint4*>(p)[1];
    } else r.v[0] = *p;
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_raw(T* p, const Raw<T, V>& r)
{
    if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&r);
    else *p = r.v[0];
}

constexpr int MAX_NT = 1024;

template <typename T, typename W, int V, int VPT, bool GROUPS>
__global__ void __launch_bounds__(VPT * V * (int)sizeof(T) <= 64 ? MAX_NT : MAX_NT / 2) norm_rows_kernel(const Args a)
{
    constexpr bool EXACT = sizeof(T) == 2 && sizeof(W) == 2;               // products are exact in float32
    constexpr float NEAR = 5e-5f;              // 127 * 2^-22 < 3.1e-5
    constexpr float MAGIC = 12582912.f;        // 1.5 * 2^23: v + MAGIC has round(v) in its low bits
    __shared__ double s_sum[MAX_NT / 32], s_wide[MAX_NT / 32];
    __shared__ float s_seen[MAX_NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, nw = nt >> 5;
    const int64_t r = blockIdx.x;
    const T* x = (const T*)a.x + r * a.ldx;
    const T* res = a.residual ? (const T*)a.residual + r * a.ldr : nullptr;
    T* hout = a.h ? (T*)a.h + r * a.ldh : nullptr;
    const W* w = (const W*)a.weight;
    int8_t* q = a.q + r * a.ldq;
    const int nvec = a.cols / V;

    Raw<T, V> h[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        const int c = (i * nt + tid) * V;
        if (i * nt + tid < nvec) h[i] = load_raw<T, V>(x + c);
        else
            for (int e = 0; e < V; e++) h[i].v[e] = from_f<T>(0.f);
    }
    if (res) {
        Raw<T, V> more[VPT];
#pragma unroll
        for (int i = 0; i < VPT; i++)
            if (i * nt + tid < nvec) more[i] = load_raw<T, V>(res + (i * nt + tid) * V);
#pragma unroll
        for (int i = 0; i < VPT; i++)
            if (i * nt + tid < nvec) {
#pragma unroll
                for (int e = 0; e < V; e++) h[i].v[e] = from_f<T>(to_f(h[i].v[e]) + to_f(more[i].v[e]));
            }
    }
    float sum = 0.f, seen = 0.f, top = 0.f, low = 0.f;         // seen: the largest |product| in float32, or NaN
    float gseen[GROUPS ? VPT : 1], glow[GROUPS ? VPT : 1];     // top + low: the largest one exactly (of one vector with groups)
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        if (GROUPS) { gseen[i] = 0.f; glow[i] = 0.f; seen = 0.f; top = 0.f; low = 0.f; }
        if (i * nt + tid < nvec) {
            const int c = (i * nt + tid) * V;
            if (hout) store_raw<T, V>(hout + c, h[i]);
            const Raw<W, V> wt = load_raw<W, V>(w + c);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float hv = to_f(h[i].v[e]), wv = to_f(wt.v[e]);
                sum = fmaf(hv, hv, sum);
                const float p = fabsf(hv * wv);
                seen = max_nan(seen, p);
                if (!EXACT) {
                    const float rest = fmaf(fabsf(hv), fabsf(wv), -p);
                    if (p > top || (p == top && rest > low)) { top = p; low = rest; }
                }
            }
        }
        if (GROUPS) { gseen[i] = seen; glow[i] = top == seen ? low : 0.f; }
    }
    double wide_sum = (double)sum, wide = EXACT ? 0.0 : (double)top + (double)low;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        wide_sum += __shfl_xor_sync(0xFFFFFFFFu, wide_sum, o);
        if (!GROUPS) {
            seen = max_nan(seen, __shfl_xor_sync(0xFFFFFFFFu, seen, o));
            if (!EXACT) wide = fmax(wide, __shfl_xor_sync(0xFFFFFFFFu, wide, o));
        }
    }
    if (lane == 0) { s_sum[warp] = wide_sum; s_seen[warp] = seen; s_wide[warp] = wide; }
    __syncthreads();
    wide_sum = 0.0;
    for (int i = 0; i < nw; i++) wide_sum += s_sum[i];
    if (!(wide_sum < 1e37) || wide_sum < 1e-25) {              // squares beyond float32, or lost below it: once more in float64
        double again = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; i++)
#pragma unroll
            for (int e = 0; e < V; e++) again += (double)to_f(h[i].v[e]) * (double)to_f(h[i].v[e]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) again += __shfl_xor_sync(0xFFFFFFFFu, again, o);
        __syncthreads();
        if (lane == 0) s_sum[warp] = again;
        __syncthreads();
        wide_sum = 0.0;
        for (int i = 0; i < nw; i++) wide_sum += s_sum[i];
    }
    const bool row_fine = wide_sum < (double)INFINITY;
    // (a float64 root and two divisions: taken last, by the threads that write a scale)
    auto inverse = [&]() { return 1.0 / sqrt(wide_sum / (double)a.cols + a.eps); };

    Peak p{0.0, 0.f, false, false};
    float peak_of[GROUPS ? VPT : 1];           // the groups' maxima, until their scales are written
    if (!GROUPS) peak_of[0] = 0.f;
    if (!GROUPS) {
        seen = 0.f; wide = 0.0;
        for (int i = 0; i < nw; i++) { seen = max_nan(seen, s_seen[i]); wide = fmax(wide, s_wide[i]); }
        if (EXACT) wide = (double)seen;
        if (!in_range(seen)) {                 // products beyond float32 or lost below it, or NaN: the maximum in float64
            wide = 0.0;
#pragma unroll 1
            for (int j = tid; j < a.cols; j += nt) {
                const float hv = to_f(hout ? hout[j] : x[j]);              // (stored before the barrier; x or residual may be h)
                wide = max_nan(wide, fabs((double)hv * (double)to_f(w[j])));
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) wide = max_nan(wide, __shfl_xor_sync(0xFFFFFFFFu, wide, o));
            __syncthreads();
            if (lane == 0) s_wide[warp] = wide;
            __syncthreads();
            wide = 0.0;
            for (int i = 0; i < nw; i++) wide = max_nan(wide, s_wide[i]);
        }
        p = make_peak(wide, seen, row_fine);
    }
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        const bool live = i * nt + tid < nvec;
        const int c = (i * nt + tid) * V;
        Raw<W, V> wt;
        if (live) wt = load_raw<W, V>(w + c);
        if (GROUPS) {                          // 128 columns: 128 / V neighbouring lanes
            constexpr int GL = V == 1 ? 32 : 128 / V;
            float gs = gseen[i];
            double gw = EXACT ? 0.0 : (double)gs + (double)glow[i];
#pragma unroll
            for (int o = GL / 2; o > 0; o >>= 1) {
                gs = max_nan(gs, __shfl_xor_sync(0xFFFFFFFFu, gs, o));
                if (!EXACT) gw = fmax(gw, __shfl_xor_sync(0xFFFFFFFFu, gw, o));
            }
            if (EXACT) gw = (double)gs;
            if (!in_range(gs)) {               // (whole groups of lanes)
                gw = 0.0;
                if (live) {
#pragma unroll
                    for (int e = 0; e < V; e++) gw = max_nan(gw, fabs((double)to_f(h[i].v[e]) * (double)to_f(wt.v[e])));
                }
                const unsigned mates = GL == 32 ? 0xFFFFFFFFu : 0xFFFFu << (lane & 16);
#pragma unroll
                for (int o = GL / 2; o > 0; o >>= 1) gw = max_nan(gw, __shfl_xor_sync(mates, gw, o));
            }
            p = make_peak(gw, gs, row_fine);
            peak_of[i] = p.dead ? NAN : (float)p.wide;
            if (p.slow && !p.dead && live && lane % GL == 0) a.scale[r * (a.cols / 128) + c / 128] = group_scale(p, inverse());
        }
        if (!live) continue;
        uint32_t word[V >= 4 ? V / 4 : 1] = {};
        unsigned near = 0;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float v = to_f(h[i].v[e]) * to_f(wt.v[e]) * p.inv, m = v + MAGIC;
            if (fabsf(fabsf(v - (m - MAGIC)) - 0.5f) <= NEAR) near |= 1u << e;
            word[e / 4] |= (__float_as_uint(m) & 0xFFu) << (8 * (e % 4));
        }
        if (p.slow || p.dead) near = (1u << V) - 1u;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(word[0], word[1]);
        else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(q + c) = word[0];
        else q[c] = (int8_t)word[0];
        if (near) {
#pragma unroll
            for (int e = 0; e < V; e++)
                if ((near >> e) & 1u) q[c + e] = round_wide(to_f(h[i].v[e]), to_f(wt.v[e]), p);
        }
    }
    if (!GROUPS) {
        if (tid == 0) a.scale[r] = group_scale(p, inverse());
    } else {
        constexpr int GL = V == 1 ? 32 : 128 / V;
        const double factor = inverse() / 127.0;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int v = i * nt + tid;
            // (a maximum outside float32's safe range has been written above)
            if (v < nvec && lane % GL == 0 && !(in_range(peak_of[i]) == false && peak_of[i] == peak_of[i]))
                a.scale[r * (a.cols / 128) + v / GL] = (float)((double)peak_of[i] * factor);
        }
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
        const Peak p = make_peak(btop == btop ? bpeak : (double)NAN, btop, row_fine);
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
            const Peak p = make_peak(gt == gt ? gp : (double)NAN, gt, row_fine);
            if (j < a.cols) {
                q[j] = round_wide(v, wt, p);
                if ((j & 127) == 0) a.scale[r * groups + j / 128] = group_scale(p, inverse);
            }
        }
    }
}


template <typename T, typename W, int V, int VPT>
cudaError_t launch_rows(const Args& a, int nt, cudaStream_t st)
{
    if constexpr (V > 1) {
        if (a.group) {
            norm_rows_kernel<T, W, V, VPT, true><<<(unsigned)a.rows, nt, 0, st>>>(a);
            return cudaGetLastError();
        }
    }
    norm_rows_kernel<T, W, V, VPT, false><<<(unsigned)a.rows, nt, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T, typename W>
cudaError_t launch(const Args& a, cudaStream_t st)
{
    constexpr int V = 16 / (int)sizeof(T);
    const uintptr_t all = (uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.h | (uintptr_t)a.weight | (uintptr_t)(a.ldx * sizeof(T)) |
                          (a.residual ? (uintptr_t)(a.ldr * sizeof(T)) : 0) | (a.h ? (uintptr_t)(a.ldh * sizeof(T)) : 0);
    const bool vec = all % 16 == 0 && ((uintptr_t)a.q | (uintptr_t)a.ldq) % V == 0 && a.cols % V == 0;
    const int nvec = vec ? a.cols / V : a.cols;
    auto threads = [&](int per) { return ((nvec + per - 1) / per + 31) / 32 * 32; };
    if (vec) {
        // four vectors a thread when there are rows enough for the GPU; one, the quickest for a row, when there are few
        if (a.rows <= imm::sm_count() && threads(1) <= MAX_NT) return launch_rows<T, W, V, 1>(a, threads(1), st);
        if (threads(2) <= 128) return launch_rows<T, W, V, 2>(a, threads(2), st);
        if (threads(4) <= MAX_NT) return launch_rows<T, W, V, 4>(a, threads(4), st);
        if (threads(8) <= MAX_NT / 2) return launch_rows<T, W, V, 8>(a, threads(8), st);
    } else if (!a.group) {
        if (threads(4) <= 128) return launch_rows<T, W, 1, 4>(a, threads(4), st);
        if (threads(16) <= MAX_NT) return launch_rows<T, W, 1, 16>(a, threads(16), st);
        if (threads(32) <= MAX_NT / 2) return launch_rows<T, W, 1, 32>(a, threads(32), st);
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
