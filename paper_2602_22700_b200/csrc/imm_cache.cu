// Rows of keys and values into a paged int8 cache (sm_100a), and the call's C ABI (declared in imm.h).
//
//   imm_kv_append   rounds the new rows of every sequence to int8 under one scale per page and head
//
// The mathematics.  A page holds `page` positions of one sequence; scale = the largest magnitude of a head's entries in
// it / 127, so far.  New rows may raise it, then the entries that the page holds already are rounded again:
//     s' = max(s, max |x| / 127),   q = rint(x / s'),   earlier entries q <- rint(q s / s').
// Quotients are those of float64 on exact operands, so anyone who holds the rows repeats every entry bit for bit; a
// float32 quotient is off by less than 2^-16 here (127 times two half-steps of 2^-24) and decides all entries that
// are not that near to a half.
//
// A block takes the pages that begin in its share of the new rows, for one head of the keys or the values: a page's rows
// stay in registers between the maximum and the rounding (what does not fit there is read again, from L2).  No block waits for
// another.  What bounds it is latency: a page is a chain of dependent loads (sequence, table, scale, rows), so blocks are small
// and many.  Measured (B200, bfloat16, 8 heads of 128): 64 rows 5.1 us, 11000 rows in five prompts of up to 3000 38 us (33 in
// float16).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_cache {

// pieces of a page's rows that a thread holds between the maximum and the rounding: few where a page gets few rows, since every
// step of the unrolled loops is paid for (1000 sequences of a row each: 8 pieces 37 us, 2 24;
// 100 of 20 rows: 8 pieces in 64 threads 20 us, 4 15)
__host__ __device__ constexpr int held_by(int threads) { return threads == 32 ? 2 : threads == 64 ? 4 : 8; }

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

// The sequence of row t: the number of those that end before it, found by a warp, 32 probes a step
__device__ __forceinline__ int sequence_of(const Args& a, int64_t t, int lane)
{
    int low = 0, size = a.batch;
    while (size > 0) {
        const int step = (size + 31) / 32, at = low + min((lane + 1) * step, size) - 1;
        const int past = __popc(__ballot_sync(0xFFFFFFFFu, lane * step < size && __ldg(a.offsets + at + 1) <= t));
        const int skipped = min(past * step, size);
        low += skipped;
        size = step == 1 ? 0 : min(step - 1, size - skipped);          // (the last of a part was probed)
    }
    return low;
}

template <typename T, int N> struct alignas(N * sizeof(T)) Pack { T v[N]; };

// N entries / s rounded to the nearest integers, half to even, by float64's quotients; 0 for s = 0 and NaN.  (No part of the kernel's
// code: copies of it in every unrolled step cost more in instruction fetches than the calls.)
template <typename T, int N>
__device__ __noinline__ Pack<int8_t, N> rounded_slowly(const Pack<T, N> x, float s)
{
    Pack<int8_t, N> q;
#pragma unroll 4
    for (int e = 0; e < N; e++) q.v[e] = (int8_t)(s > 0.f ? (int)fmin(fmax(rint((double)(float)x.v[e] / (double)s), -127.0), 127.0) : 0);
    return q;
}
// ... by float32's where that decides: x * inverse, with inverse float32's 1 / s, is off by 127 * 2^-24 = 7.6e-6 at most.  The large
// constant rounds it to its low bits; what is left over (2^-25 off) says how near to a half it was.
template <typename T, int N>
__device__ __forceinline__ Pack<int8_t, N> rounded(const Pack<T, N>& x, float s, float inverse, bool usable)
{
    constexpr float MAGIC = 12582912.f;       // 1.5 * 2^23
    Pack<int8_t, N> q;
    float worst = usable ? 0.f : 1.f;
#pragma unroll
    for (int e = 0; e < N; e++) {
        const float t = fmaf((float)x.v[e], inverse, MAGIC);
        worst = fmaxf(worst, fabsf(fmaf((float)x.v[e], inverse, MAGIC - t)));
        q.v[e] = (int8_t)__float_as_int(t);
    }
    if (worst > 0.49999f) q = rounded_slowly(x, s);
    return q;
}
// 16 entries times old / s, the same way (not inlined either)
__device__ __noinline__ Pack<int8_t, 16> rescaled_slowly(const Pack<int8_t, 16> x, float old, float s)
{
    Pack<int8_t, 16> q;
#pragma unroll 4
    for (int e = 0; e < 16; e++) q.v[e] = (int8_t)rint((double)x.v[e] * (double)old / (double)s);
    return q;
}

// N entries at a time, N * sizeof(T) = 16 bytes where rows are aligned to them
template <typename T, int N, int NT>
__global__ void __launch_bounds__(NT) append_kernel(const Args a)
{
    constexpr int NW = NT / 32, HELD = held_by(NT);
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
        const int b = sequence_of(a, t, lane);
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
            const int total = count * pieces, row0 = tid / pieces, piece0 = tid - row0 * pieces, dr = NT / pieces, dp = NT - dr * pieces;
            uint32_t top = 0;                  // (magnitudes order like integers, infinity and NaN above)
            Pack<T, N> held[HELD];
            // pieces tid, tid + NT, ... : HELD of them on their way at once, and kept if there are no more
            int row = row0, piece = piece0;
            for (int i0 = tid; i0 - tid < total; i0 += HELD * NT) {
#pragma unroll
                for (int k = 0; k < HELD; k++) {
                    if (i0 + k * NT < total) held[k] = *reinterpret_cast<const Pack<T, N>*>(mine + row * ld + piece * N);
                    row += dr;
                    piece += dp;
                    if (piece >= pieces) { piece -= pieces; row++; }
                }
#pragma unroll
                for (int k = 0; k < HELD; k++)
                    if (i0 + k * NT < total) {
#pragma unroll
                        for (int e = 0; e < N; e++) top = max(top, __float_as_uint(fabsf((float)held[k].v[e])));
                    }
            }
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            __syncthreads();                  // (the last page's peaks and scale have been read)
            if (lane == 0) peak[warp] = __uint_as_float(top);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; w++) top = max(top, __float_as_uint(peak[w]));
            const bool finite = top < 0x7F800000u;
            const float old = slot ? *scale : 0.f;
            const float fresh = __fdiv_rn(__uint_as_float(top), 127.f);
            const float s = !finite || isnan(old) ? NAN : fmaxf(old, fresh);
            const float inverse = s > 0.f && s < INFINITY ? __frcp_rn(s) : 0.f;
            const bool usable = s > 0.f && inverse < INFINITY;           // (1 / s of the smallest scales is not a float32)
            if (slot && s > old && old > 0.f) {
                for (int i = tid; i < slot * dim / 16; i += NT) {
                    Pack<int8_t, 16> v = *reinterpret_cast<Pack<int8_t, 16>*>(out + i * 16);
                    const Pack<int8_t, 16> w = v;
                    float worst = usable ? 0.f : 1.f;
                    const float ratio = old * inverse;               // (old < s: two half-steps off, 127 * 2^-23 = 1.5e-5)
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        const float t = fmaf((float)w.v[e], ratio, 12582912.f);
                        worst = fmaxf(worst, fabsf(fmaf((float)w.v[e], ratio, 12582912.f - t)));
                        v.v[e] = (int8_t)__float_as_int(t);
                    }
                    if (worst > 0.49998f) v = rescaled_slowly(w, old, s);
                    *reinterpret_cast<Pack<int8_t, 16>*>(out + i * 16) = v;
                }
            }
            row = row0;
            piece = piece0;
            const bool kept = total <= HELD * NT;
            for (int i0 = tid; i0 - tid < total; i0 += HELD * NT) {
#pragma unroll
                for (int k = 0; k < HELD; k++) {
                    if (i0 + k * NT < total) {
                        if (!kept) held[k] = *reinterpret_cast<const Pack<T, N>*>(mine + row * ld + piece * N);
                        *reinterpret_cast<Pack<int8_t, N>*>(out + ((slot + row) * dim + piece * N)) = rounded(held[k], s, inverse, usable);
                    }
                    row += dr;
                    piece += dp;
                    if (piece >= pieces) { piece -= pieces; row++; }
                }
            }
            __syncthreads();                  // (the scale has been read)
            if (tid == 0) *scale = s;
        }
        t += min((int64_t)count, end - t);
    }
}

template <typename T, int N>
cudaError_t launch(const Args& a, int threads, dim3 grid, cudaStream_t st)
{
    if (threads == 32) append_kernel<T, N, 32><<<grid, 32, 0, st>>>(a);
    else if (threads == 64) append_kernel<T, N, 64><<<grid, 64, 0, st>>>(a);
    else if (threads == 128) append_kernel<T, N, 128><<<grid, 128, 0, st>>>(a);
    else append_kernel<T, N, 256><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch(const Args& a, bool aligned, int threads, dim3 grid, cudaStream_t st)
{
    return aligned ? launch<T, 16 / (int)sizeof(T)>(a, threads, grid, st) : launch<T, 1>(a, threads, grid, st);
}

}  // namespace imm_cache

extern "C" int imm_kv_append(const imm_kv_append_desc* desc_host, void* stream)
{
    using namespace imm_cache;
    if (!desc_host || desc_host->reserved || desc_host->reserved2) return IMM_ERR_ARG;
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
    // rows of a block: a page's where sequences have so many, else one while that leaves no more blocks than run at once or so
    const int64_t room = 32 * (int64_t)imm::sm_count();
    int64_t share = (2 * d.tokens * d.kv_heads + room - 1) / room;
    share = d.tokens / d.batch >= d.page || share > d.page ? d.page : share < 1 ? 1 : share;
    a.share = (int32_t)share;
    const uintptr_t all = (uintptr_t)d.d_k | (uintptr_t)d.d_v | (uintptr_t)(es * d.ldk) | (uintptr_t)(es * d.ldv) | (uintptr_t)(es * d.hsk) | (uintptr_t)(es * d.hsv);
    const bool aligned = all % 16 == 0;
    // threads that hold a page's rows (as many of them as a sequence has on average) in their registers: blocks are bound by the
    // latency of a chain of loads, so many small ones beat few large ones (prompts of 3000: 256 threads 59 us, 128 of them 36)
    const int64_t rows = d.tokens / d.batch + 1 < d.page ? d.tokens / d.batch + 1 : d.page;
    const int64_t pieces = rows * d.dim / (aligned ? 16 / (int64_t)es : 1);
    int threads = 32;
    while (threads < 256 && pieces > threads * held_by(threads)) threads *= 2;
    const int64_t blocks = (d.tokens + share - 1) / share + (d.batch + threads / 32 - 1) / (threads / 32);
    const dim3 grid((unsigned)blocks, (unsigned)d.kv_heads, 2);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == IMM_F32 ? launch<float>(a, aligned, threads, grid, st)
                          : d.dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, aligned, threads, grid, st) : launch<__half>(a, aligned, threads, grid, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
