// Root-mean-square norm with residual addition and int8 output (sm_100a) and its C ABI (declared in imm.h).
//
//   imm_rmsnorm_quant   h = x + residual;  t = h * weight;  q = round(127 t / max|t|);  scale = max|t| r / 127
//
// One streaming pass over the rows (x and residual read, h and q written, each once), bound by HBM: a block
// takes a row and keeps it in registers between the reductions and the rounding.
//
// The rounding.  q is defined on the exact products in float64 (reproducible anywhere); 127 t / a in float32 is
// off by less than 127 * 2^-22 < 4e-5, so only values within 1e-4 of a border between two integers -- two entries
// in ten thousand -- are worked out again in float64.  Products of two 16-bit floats are exact in float32, so
// their maximum is too; with float32 factors the maximum is taken over float64 products.  Rows whose maximum
// is so large or small that float32 products may overflow or vanish take the float64 path altogether.
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

// What the rounding of one group needs: its maximum in both widths, and which path it takes.
struct Peak { double wide; float inv; bool slow, dead; };

__device__ __forceinline__ Peak make_peak(double wide, float narrow, bool row_fine)
{
    Peak p;
    p.wide = wide;
    p.dead = !row_fine || !(wide < (double)INFINITY);          // not finite, or NaN
    // float32 products neither overflow nor lose bits that matter while the maximum is in this range
    p.slow = !(narrow >= 0x1p-60f && narrow <= 0x1p100f);
    p.inv = p.slow ? 0.f : 127.f / (float)wide;
    return p;
}

__device__ __forceinline__ int quantise(float h, float w, const Peak& p)
{
    if (p.dead) return 0;
    if (!p.slow) {
        const float v = h * w * p.inv;
        const float n = rintf(v);
        if (fabsf(fabsf(v - n) - 0.5f) > 1e-4f) return (int)n;
    }
    if (p.wide == 0.0) return 0;
    return (int)rint((double)h * (double)w * 127.0 / p.wide);
}

__device__ __forceinline__ float group_scale(const Peak& p, double inverse)
{
    if (p.dead) return NAN;
    return p.wide == 0.0 ? 0.f : (float)(p.wide * inverse / 127.0);
}

// A block per row.  Each thread holds up to ITEMS entries (its columns tid, tid + NT, ...) as float32.
// Longer rows are read again in the second pass (h from where it was written).
template <typename T, typename W, int NT, int ITEMS>
__global__ void __launch_bounds__(NT) norm_rows_kernel(const Args a)
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

    float held[ITEMS];
    double sum = 0.0, peak = 0.0;
    float top = 0.f;
    auto take = [&](int j) -> float {
        float v = to_f(x[j]);
        if (res) v = to_f(from_f<T>(v + to_f(res[j])));
        if (hout) hout[j] = from_f<T>(v);
        const float wt = to_f(w[j]);
        sum += (double)v * (double)v;
        peak = fmax(peak, fabs((double)v * (double)wt));
        top = max_nan(top, fabsf(v * wt));
        return v;
    };
#pragma unroll
    for (int i = 0; i < ITEMS; i++) {
        const int j = tid + i * NT;
        held[i] = j < a.cols ? take(j) : 0.f;
    }
    for (int j = tid + ITEMS * NT; j < a.cols; j += NT) take(j);
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
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int j = tid + i * NT;
            if (j < a.cols) q[j] = (int8_t)quantise(held[i], to_f(w[j]), p);
        }
        for (int j = tid + ITEMS * NT; j < a.cols; j += NT) q[j] = (int8_t)quantise(to_f(again[j]), to_f(w[j]), p);
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
            if (j < a.cols) { v = to_f(again[j]); if (!hout && res) v = 0.f; wt = to_f(w[j]); }
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
                q[j] = (int8_t)quantise(v, wt, p);
                if ((j & 127) == 0) a.scale[r * groups + j / 128] = group_scale(p, inverse);
            }
        }
    }
}

template <typename T, typename W>
cudaError_t launch(const Args& a, cudaStream_t st)
{
    norm_rows_kernel<T, W, 256, 16><<<(unsigned)a.rows, 256, 0, st>>>(a);
    return cudaGetLastError();
}

size_t elem(int dtype) { return dtype == IMM_F32 ? 4 : 2; }

}  // namespace imm_norm

extern "C" int imm_rmsnorm_quant(const void* d_x, const void* d_residual, const void* d_weight, int dtype, int wdtype,
                                 int64_t rows, int64_t cols, int64_t ldx, int64_t ldr, int64_t ldh, int64_t ldq, double eps,
                                 int group, void* d_h, int8_t* d_q, float* d_scale, void* stream)
{
    using namespace imm_norm;
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
