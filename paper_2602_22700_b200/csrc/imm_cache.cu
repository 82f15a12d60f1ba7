// Rows of keys and values into a paged int8 cache (sm_100a), and the call's C ABI (declared in imm.h).
//
//   imm_kv_append   rounds the new rows of every sequence to int8 under one scale per page and head
//
// The mathematics.  A page holds `page` positions of one sequence; scale = the largest magnitude of a head's entries in
// it / 127, so far.  New rows may raise it, then the entries that the page holds already are rounded again:
//     s' = max(s, max |x| / 127),   q = rint(x / s'),   earlier entries q <- rint(q s / s').
// Quotients are those of float64 on exact operands, so anyone who holds the rows repeats every entry bit for bit; a
// float32 quotient is off by less than 2^-15 here (127 times three half-steps of 2^-24) and decides all entries that
// are not that near to a half.
//
// A block takes the pages that begin in its share of the new rows, for one head of the keys or the values: one pass over
// a page's rows for the maximum, a second (from L1 and L2) that rounds.  No block waits for another.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_cache {

constexpr int NT = 128;
constexpr int NW = NT / 32;

struct Args {
    const void* x[2];                         // rows of keys, of values
    int64_t ld[2], hs[2];                     // strides of a row and of a head (entries)
    int8_t* cache[2];
    float* scale[2];
    int64_t page_stride[2];
    const int32_t* table;
    const int64_t* offsets;
    const int32_t* length;
    int32_t* status;
    int64_t tokens, ld_table, pages;
    int32_t batch, max_pages, kv_heads, dim, page, page_log, share;
};

// Rows of sequence b; false: they do not lie in the call, or its length has no room for them
__device__ __forceinline__ bool sequence(const Args& a, int b, int64_t& first, int64_t& rows, int64_t& length)
{
    first = a.offsets[b];
    rows = a.offsets[b + 1] - first;
    length = a.length[b];
    return first >= 0 && rows >= 0 && first + rows <= a.tokens && length >= rows && length <= (int64_t)a.max_pages * a.page;
}

template <typename T, int N> struct alignas(N * sizeof(T)) Pack { T v[N]; };

// x / s rounded to the nearest integer, half to even, as float64 has it; inverse: float32's 1 / s
__device__ __forceinline__ int rounded(float x, float s, float inverse)
{
    const float y = x * inverse;
    float r = rintf(y);
    if (!(fabsf(fabsf(y - r) - 0.5f) > 1e-4f)) r = (float)rint((double)x / (double)s);
    return (int)fminf(fmaxf(r, -127.f), 127.f);
}

// N entries at a time, N * sizeof(T) = 16 bytes where rows are aligned to them
template <typename T, int N>
__global__ void __launch_bounds__(NT) append_kernel(const Args a)
{
    __shared__ float peak[NW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t shares = (a.tokens + a.share - 1) / a.share;
    if (blockIdx.x >= shares) {               // the last blocks look the sequences over, a warp each
        if (blockIdx.y || blockIdx.z) return;
        const int b = (int)(blockIdx.x - shares) * NW + warp;
        if (b >= a.batch) return;
        int64_t first, rows, length;
        bool good = sequence(a, b, first, rows, length);
        if (good && rows > 0) {
            const int64_t p0 = (length - rows) >> a.page_log, p1 = (length - 1) >> a.page_log;
            for (int64_t p = p0 + lane; p <= p1; p += 32) {
                const int32_t at = a.table[b * a.ld_table + p];
                good &= at >= 0 && at < a.pages;
            }
        }
        good = __all_sync(0xFFFFFFFFu, good);
        if (lane == 0) a.status[b] = good ? IMM_OK : IMM_ERR_ARG;
        return;
    }
    const int head = blockIdx.y, which = blockIdx.z, dim = a.dim;
    const T* x = (const T*)a.x[which] + (int64_t)head * a.hs[which];
    const int64_t ld = a.ld[which];
    const int pieces = dim / N;               // of a row
    for (int64_t t = (int64_t)blockIdx.x * a.share, end = min(a.tokens, t + a.share); t < end;) {
        // the sequence of row t: the number of those that end before it
        int b = 0;
        for (int i = 0; i < a.batch; i += NT) b += __syncthreads_count(i + tid < a.batch && a.offsets[i + tid + 1] <= t);
        if (b >= a.batch) return;             // rows behind the last sequence
        int64_t first, rows, length;
        if (!sequence(a, b, first, rows, length) || t < first || t >= first + rows) { t++; continue; }       // (offsets may be anything)
        const int64_t place = length - rows + (t - first);
        const int slot = (int)(place & (a.page - 1));
        if (slot && t > first) {              // inside a page that another share begins
            t += min(min((int64_t)(a.page - slot), first + rows - t), end - t);
            continue;
        }
        const int count = (int)min((int64_t)(a.page - slot), first + rows - t);
        const int32_t number = a.table[b * a.ld_table + (place >> a.page_log)];
        if (number >= 0 && number < a.pages) {
            int8_t* out = a.cache[which] + number * a.page_stride[which] + (int64_t)head * a.page * dim;
            float* scale = a.scale[which] + (int64_t)number * a.kv_heads + head;
            const T* mine = x + t * ld;
            float top = 0.f;
            bool finite = true;
            for (int i = tid; i < count * pieces; i += NT) {
                const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(mine + (i / pieces) * ld + (i % pieces) * N);
#pragma unroll
                for (int e = 0; e < N; e++) {
                    const float f = fabsf((float)v.v[e]);
                    finite &= f < INFINITY;
                    top = fmaxf(top, f);
                }
            }
            top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));       // (not negative: ordered like integers)
            if (lane == 0) peak[warp] = top;
            finite = __syncthreads_and(finite);
#pragma unroll
            for (int w = 0; w < NW; w++) top = fmaxf(top, peak[w]);
            const float old = slot ? *scale : 0.f;
            const float fresh = __fdiv_rn(top, 127.f);
            const float s = !finite || isnan(old) ? NAN : fmaxf(old, fresh);
            const float inverse = s > 0.f && s < INFINITY ? __frcp_rn(s) : 0.f;
            const bool usable = s > 0.f && inverse < INFINITY;           // (1 / s of the smallest scales is not a float32)
            if (slot && s > old && old > 0.f) {
                for (int i = tid; i < slot * dim / 16; i += NT) {
                    Pack<int8_t, 16> v = *reinterpret_cast<Pack<int8_t, 16>*>(out + i * 16);
#pragma unroll
                    for (int e = 0; e < 16; e++) v.v[e] = (int8_t)rint((double)v.v[e] * (double)old / (double)s);
                    *reinterpret_cast<Pack<int8_t, 16>*>(out + i * 16) = v;
                }
            }
            for (int i = tid; i < count * pieces; i += NT) {
                const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(mine + (i / pieces) * ld + (i % pieces) * N);
                Pack<int8_t, N> q;
#pragma unroll
                for (int e = 0; e < N; e++) {
                    const float f = (float)v.v[e];
                    q.v[e] = (int8_t)(usable ? rounded(f, s, inverse) : s > 0.f ? (int)fmin(fmax(rint((double)f / (double)s), -127.0), 127.0) : 0);
                }
                *reinterpret_cast<Pack<int8_t, N>*>(out + ((int64_t)(slot + i / pieces) * dim + (i % pieces) * N)) = q;
            }
            __syncthreads();                  // (the scale and the peaks have been read)
            if (tid == 0) *scale = s;
        }
        t += min((int64_t)count, end - t);
    }
}

template <typename T>
cudaError_t launch(const Args& a, bool aligned, dim3 grid, cudaStream_t st)
{
    if (aligned) append_kernel<T, 16 / sizeof(T)><<<grid, NT, 0, st>>>(a);
    else append_kernel<T, 1><<<grid, NT, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace imm_cache

extern "C" int imm_kv_append(const imm_kv_append_desc* desc_host, void* stream)
{
    using namespace imm_cache;
    if (!desc_host || desc_host->reserved) return IMM_ERR_ARG;
    const imm_kv_append_desc& d = *desc_host;
    if (d.dtype != IMM_F32 && d.dtype != IMM_BF16 && d.dtype != IMM_F16) return IMM_ERR_ARG;
    if (d.batch < 0 || d.tokens < 0) return IMM_ERR_SHAPE;
    if (d.batch > 0 && (!d.d_offsets || !d.d_length || !d.d_status)) return IMM_ERR_ARG;
    if (d.batch > 0 && d.tokens > 0 && (!d.d_k || !d.d_v || !d.d_k_cache || !d.d_v_cache || !d.d_k_scale || !d.d_v_scale || !d.d_table))
        return IMM_ERR_ARG;
    int log = 4;
    while (log < 7 && (1 << log) != d.page) log++;
    if ((1 << log) != d.page || d.dim <= 0 || d.dim > IMM_KV_MAX_DIM || d.dim % 16) return IMM_ERR_SHAPE;
    if (d.kv_heads <= 0 || d.kv_heads > IMM_KV_MAX_HEADS || d.batch > IMM_KV_MAX_BATCH || d.tokens > IMM_KV_MAX_TOKENS || d.max_pages <= 0 ||
        d.max_pages > IMM_KV_MAX_LENGTH / d.page || d.pages <= 0 || d.pages > 0x7FFFFFFF || d.ld_table < d.max_pages)
        return IMM_ERR_SHAPE;
    const int64_t entries = (int64_t)d.kv_heads * d.page * d.dim;
    if (d.hsk < d.dim || d.hsv < d.dim || d.ldk < d.dim || d.ldv < d.dim || d.k_page_stride < entries || d.v_page_stride < entries) return IMM_ERR_SHAPE;
    if (d.k_page_stride % 16 || d.v_page_stride % 16) return IMM_ERR_ALIGN;
    const uintptr_t es = d.dtype == IMM_F32 ? 4 : 2;
    if ((uintptr_t)d.d_k % es || (uintptr_t)d.d_v % es || (uintptr_t)d.d_k_cache % 16 || (uintptr_t)d.d_v_cache % 16 || (uintptr_t)d.d_k_scale % 4 ||
        (uintptr_t)d.d_v_scale % 4 || (uintptr_t)d.d_table % 4 || (uintptr_t)d.d_offsets % 8 || (uintptr_t)d.d_length % 4 || (uintptr_t)d.d_status % 4)
        return IMM_ERR_ALIGN;
    if (d.batch == 0) return IMM_OK;
    Args a{};
    a.x[0] = d.d_k; a.x[1] = d.d_v;
    a.ld[0] = d.ldk; a.ld[1] = d.ldv;
    a.hs[0] = d.hsk; a.hs[1] = d.hsv;
    a.cache[0] = d.d_k_cache; a.cache[1] = d.d_v_cache;
    a.scale[0] = d.d_k_scale; a.scale[1] = d.d_v_scale;
    a.page_stride[0] = d.k_page_stride; a.page_stride[1] = d.v_page_stride;
    a.table = d.d_table; a.offsets = d.d_offsets; a.length = d.d_length; a.status = d.d_status;
    a.tokens = d.tokens; a.ld_table = d.ld_table; a.pages = d.pages;
    a.batch = d.batch; a.max_pages = d.max_pages; a.kv_heads = d.kv_heads; a.dim = d.dim; a.page = d.page; a.page_log = log;
    // a block for every row while that fills the GPU's places about twice over, for a page's rows at most
    const int64_t room = 32 * (int64_t)imm::sm_count();
    int64_t share = (2 * d.tokens * d.kv_heads + room - 1) / room;
    share = share < 1 ? 1 : share > d.page ? d.page : share;
    a.share = (int32_t)share;
    const int64_t blocks = (d.tokens + share - 1) / share + (d.batch + NW - 1) / NW;
    const dim3 grid((unsigned)blocks, (unsigned)d.kv_heads, 2);
    const uintptr_t all = (uintptr_t)d.d_k | (uintptr_t)d.d_v | (uintptr_t)(es * d.ldk) | (uintptr_t)(es * d.ldv) | (uintptr_t)(es * d.hsk) | (uintptr_t)(es * d.hsv);
    const bool aligned = all % 16 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == IMM_F32 ? launch<float>(a, aligned, grid, st)
                          : d.dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, aligned, grid, st) : launch<__half>(a, aligned, grid, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
