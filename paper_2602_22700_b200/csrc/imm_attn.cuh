// What the kernels of the attention over the int8 cache share: arguments, the sequences' share of the work, and the
// layout of partial results.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/imm.h"

namespace imm_attn {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NOTHING = -1e30f;             // running maximum of a row that has seen nothing
// Weights are kept as 2^(x - m): a new m puts the largest at 2^BIAS, and m stays until one passes 2^(BIAS + SLACK).  Both
// stay below float16's 2^16, and BIAS keeps the small weights away from its smallest values.
constexpr float BIAS = 6.f, SLACK = 8.f;

struct Args {
    const void* q;
    const int8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    const int32_t* table;
    const int64_t* offsets;
    const int32_t* length;
    void* out;
    float* lse;
    float* parts;                             // partial results: two slots per block
    int64_t tokens, ldq, hsq, ldo, hso, pages, k_page_stride, v_page_stride, ld_table;
    int32_t batch, heads, kv_heads, group, dim, page_log, window, sinks;
    int32_t q_aligned;                        // rows of q begin on 16-byte boundaries
    int64_t max_length;
    float scale;                              // times log2(e)
};

// A sequence's work: key tiles of TILE keys that some row sees (the first ones, then those of the window and the
// history), the same for each of kv_heads * row tiles.
struct Sequence {
    int64_t first;                            // first row
    int32_t rows, length;
    int32_t low, sink, tiles;                 // first tile of the window; tiles of the first tokens before it; tiles in all
    int32_t row_tiles;
    bool bad;                                 // a length that no table holds
    __device__ __forceinline__ int64_t work(int kv_heads) const { return (int64_t)kv_heads * row_tiles * tiles; }
};

template <int TILE, int ROWS>
__device__ __forceinline__ Sequence sequence(const Args& a, int b)
{
    Sequence s;
    const int64_t o0 = __ldg(a.offsets + b), o1 = __ldg(a.offsets + b + 1);
    s.length = __ldg(a.length + b);
    s.first = o0;
    s.rows = o0 >= 0 && o1 >= o0 && o1 <= a.tokens ? (int)(o1 - o0) : 0;
    s.bad = s.length < 0 || s.length > a.max_length;
    s.row_tiles = (int)(((int64_t)s.rows * a.group + ROWS - 1) / ROWS);
    s.low = s.sink = s.tiles = 0;
    if (s.bad || s.rows == 0) return s;
    if (a.window) {
        const int low = max(0, max(0, s.length - s.rows) - a.window + 1);
        s.low = low / TILE;
        s.sink = min((min(a.sinks, s.length) + TILE - 1) / TILE, s.low);
    }
    s.tiles = s.sink + (s.length + TILE - 1) / TILE - s.low;
    return s;
}

// block sum and scan of 64-bit counts; `sh`: a word per warp
template <int NT> __device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* sh, int64_t& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int64_t t = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += t; }
    __syncthreads();
    if (lane == 31) sh[warp] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; w++) { if (w < warp) before += sh[w]; total += sh[w]; }
    return before + v;                        // inclusive
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <typename T> __device__ __forceinline__ T to(float x);
template <> __device__ __forceinline__ float to<float>(float x) { return x; }
template <> __device__ __forceinline__ __half to<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// two bytes of w (those that `pick` names) as two float16 values: 1024 + (x + 128) has the byte in its low bits
__device__ __forceinline__ uint32_t halves(uint32_t biased, uint32_t pick)
{
    const uint32_t r = __byte_perm(biased, 0x64646464u, pick);
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&r), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&v);
}

// The factors of a page and head: of x (k's scale), and v's scale as mantissa * 2^exponent.  The exponent joins x, so that
// the largest weight, not the largest scale, sets the range of the float16 weights; its inverse leaves the sum of weights.
struct Factors { float k, exponent, inverse, mantissa; };
__device__ __forceinline__ Factors factors(float ks, float vs)
{
    Factors f;
    const bool good = ks >= 0.f && ks < INFINITY && vs >= 0.f && vs < INFINITY;
    const bool small = vs < 0x1p-100f;
    const int e = !good ? 0 : small ? -100 : (int)(__float_as_uint(vs) >> 23) - 127;
    f.k = good ? ks : NAN;
    f.exponent = (float)e;
    f.inverse = e == 127 ? 0x1p-127f : __uint_as_float((uint32_t)(127 - e) << 23);
    f.mantissa = !good ? 1.f : small ? 0.f : vs * f.inverse;
    return f;
}

}  // namespace imm_attn
