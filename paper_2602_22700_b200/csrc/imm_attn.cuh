// What the kernels of the attention over the int8 cache share: arguments, the sequences' share of the work, and the
// layout of partial results.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/imm.h"

namespace imm_attn {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NOTHING = -3.402823466e38f;   // running maximum of a row that has seen nothing: no score lies below it
// Weights are kept as 2^(x - m): a new m puts the largest at 2^BIAS, and m stays until one passes 2^(BIAS + SLACK).  Both
// stay below float16's 2^16, and BIAS keeps the small weights away from its smallest values.
constexpr float BIAS = 6.f, SLACK = 8.f;
// what x may be beside m: never above m + BIAS + SLACK, where a rounding step of m is larger than these
__device__ __forceinline__ float limit_of(float m) { return __fadd_rd(m, BIAS + SLACK); }

struct Args {
    const void* q;
    const int8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    const int32_t* table;
    const int64_t* offsets;
    const int32_t* length;
    void* out;
    float* lse;
    struct Record* records;                   // one per block of the first launch
    float* parts;                             // partial results: two slots per block
    int64_t tokens, ldq, hsq, ldo, hso, pages, k_page_stride, v_page_stride, ld_table;
    int32_t batch, heads, kv_heads, group, dim, page_log, window, sinks;
    int32_t steps;                            // products of a block's streams at most (tests end them early)
    int32_t q_aligned, out_aligned;           // rows of q, of the output begin on 16-byte boundaries
    int64_t max_length, patience;             // patience: cycles that a wait inside a block may take
    float scale;                              // times log2(e)
    float per_group;                          // 1 / group
};

// Row t0 * group + h0 + w of a sequence and key head: its query and its head in the group.  h0 + w is below 2^11, so that the
// quotient's error stays far below the half step that keeps it away from the next integer.
struct Place { int query, head; };
__device__ __forceinline__ Place place_of(const Args& a, int t0, int h0, int w)
{
    const int x = h0 + w, t = (int)(((float)x + 0.5f) * a.per_group);
    return {t0 + t, x - t * a.group};
}

// A sequence's work: key tiles of TILE keys that some row sees (the first ones, then those of the window and the
// history), the same for each of kv_heads * row tiles.
struct Sequence {
    int64_t first;                            // first row
    int32_t rows, length;
    int32_t low, sink, tiles;                 // first tile of the window; tiles of the first tokens before it; tiles in all
    int32_t row_tiles;
    bool bad;                                 // a length that no table holds
    __device__ __forceinline__ int64_t work(int kv_heads, int setup) const { return tiles ? (int64_t)kv_heads * row_tiles * (setup + tiles) : 0; }
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

// A sum of weights l times 2^d, in two steps, since 2^d by itself may be 0: beside a maximum that a page of large values sets, the sum of
// the others is large.
__device__ __forceinline__ float scaled(float l, float d)
{
    const float half = ex2(0.5f * d);
    return l * half * half;
}
// Where the value scale of a page lies 2^FAR below another's that the row has seen, the weights that the values are multiplied by are too
// small for the sum: its keys enter that by exponentials of their own.  (Less far, what is lost lies 2^-60 below the largest weight.)
constexpr float FAR = 40.f;

// An item that begins in a block's share and goes on behind it: its partial results lie in slot `slot` of that block and in
// slot 0 of the next parts - 1 ones.  parts = 0: none.
struct alignas(16) Record {
    int64_t first;                            // the sequence's first row
    int32_t kvh, r0, rows;                    // rows r0 .. r0 + rows - 1 of key head kvh (row r: query r / group, head r % group)
    int32_t parts, slot, reserved;
};
// a slot: outputs [ROWS][DT], then m[ROWS], l[ROWS]
template <int DT, int ROWS> __host__ __device__ constexpr int slot_floats() { return ROWS * (DT + 2); }

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

// rows that see nothing
template <typename T>
__device__ __forceinline__ void blank(const Args& a, int64_t first, int64_t rows, bool bad, int tid, int threads)
{
    const T value = to<T>(bad ? NAN : 0.f);
    const int64_t per = (int64_t)a.heads * a.dim;
    for (int64_t i = tid; i < rows * per; i += threads) {
        const int64_t row = first + i / per;
        const int h = (int)(i % per) / a.dim, d = (int)(i % per) % a.dim;
        ((T*)a.out)[row * a.ldo + h * a.hso + d] = value;
        if (d == 0 && a.lse) a.lse[row * a.heads + h] = bad ? NAN : -INFINITY;
    }
}

constexpr int JOIN_ROWS = 32;                 // blocks per item at most (prompt of 4096: a block per row 247 us, 32 blocks 214)
constexpr int JOIN_ALONE = 8;                 // parts that one warp adds up by itself
// The second launch: the blocks of a number add up the parts of the item that the first launch's block of that number began,
// always in the same order.  Few parts of a row are added up by one warp; of more of them a block's warps take theirs in turn, and
// their sums are added up at the end.
template <typename T, int DT, int ROWS>
__global__ void __launch_bounds__(128) join_kernel(const Args a)
{
    constexpr int N = DT / 32;
    __shared__ float sh_m[4], sh_l[4], sh_o[4][DT];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    cudaGridDependencySynchronize();          // (every block: the call ends after the first launch)
    const Record rec = a.records[blockIdx.x];
    if (rec.parts == 0) return;
    auto part = [&](int p) { return a.parts + ((int64_t)(blockIdx.x + p) * 2 + (p ? 0 : rec.slot)) * slot_floats<DT, ROWS>(); };
    // parts first, first + step, ... of row r: a lane each for maxima and sums, 32 at a time, then the outputs
    float top, lsum, acc[N];
    auto add_up = [&](int r, int first, int step) {
        top = NOTHING;
        lsum = 0.f;
#pragma unroll
        for (int i = 0; i < N; i++) acc[i] = 0.f;
        const int count = rec.parts > first ? (rec.parts - first + step - 1) / step : 0;
        for (int k0 = 0; k0 < count; k0 += 32) {
            const bool in = k0 + lane < count;
            const float* p = part(in ? step * (k0 + lane) + first : 0);
            const float pm = in ? p[ROWS * DT + r] : NOTHING, pl = in ? p[ROWS * DT + ROWS + r] : 0.f;
            float next = fmaxf(top, pm);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) next = fmaxf(next, __shfl_xor_sync(0xFFFFFFFFu, next, o));
            const float down = ex2(top - next), weight = ex2(pm - next);
            float add = scaled(pl, pm - next);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) add += __shfl_xor_sync(0xFFFFFFFFu, add, o);
            lsum = scaled(lsum, top - next) + add;
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] *= down;
            top = next;
            const int n = min(32, count - k0);
            for (int k = 0; k < n; k += 4) {   // four at once
                float v[4][N];
#pragma unroll
                for (int z = 0; z < 4; z++)
#pragma unroll
                    for (int i = 0; i < N; i++) v[z][i] = part(step * (k0 + min(k + z, n - 1)) + first)[r * DT + i * 32 + lane];
#pragma unroll
                for (int z = 0; z < 4; z++) {
                    const float w = __shfl_sync(0xFFFFFFFFu, weight, min(k + z, 31));
                    if (k + z < n) {
#pragma unroll
                        for (int i = 0; i < N; i++) acc[i] = fmaf(w, v[z][i], acc[i]);
                    }
                }
            }
        }
    };
    const int t0 = rec.r0 / a.group, h0 = rec.r0 - t0 * a.group;
    int64_t row;
    int head;
    auto find = [&](int r) {
        const Place at = place_of(a, t0, h0, r);
        head = rec.kvh * a.group + at.head;
        row = rec.first + at.query;
    };
    auto write = [&](int d, float y) { ((T*)a.out)[row * a.ldo + (int64_t)head * a.hso + d] = to<T>(lsum == 0.f ? 0.f : y / lsum); };
    auto write_lse = [&]() { if (a.lse) a.lse[row * a.heads + head] = lsum == 0.f ? -INFINITY : (top + log2f(lsum)) * LN2; };
    if (rec.parts <= JOIN_ALONE) {
        for (int r = blockIdx.y * 4 + warp; r < rec.rows; r += gridDim.y * 4) {
            add_up(r, 0, 1);
            find(r);
#pragma unroll
            for (int i = 0; i < N; i++) if (i * 32 + lane < a.dim) write(i * 32 + lane, acc[i]);
            if (lane == 0) write_lse();
        }
        return;
    }
    for (int r = blockIdx.y; r < rec.rows; r += gridDim.y) {
        add_up(r, warp, 4);
        if (lane == 0) { sh_m[warp] = top; sh_l[warp] = lsum; }
#pragma unroll
        for (int i = 0; i < N; i++) sh_o[warp][i * 32 + lane] = acc[i];
        __syncthreads();
        top = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
        lsum = 0.f;
        float weight[4];
#pragma unroll
        for (int w = 0; w < 4; w++) { weight[w] = ex2(sh_m[w] - top); lsum += scaled(sh_l[w], sh_m[w] - top); }
        find(r);
        for (int d = tid; d < a.dim; d += 128) {
            float y = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) y = fmaf(weight[w], sh_o[w][d], y);
            write(d, y);
        }
        if (tid == 0) write_lse();
        __syncthreads();
    }
}
template <typename T, int DT, int ROWS>
cudaError_t launch_join(const Args& a, int grid, cudaStream_t st)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)grid, ROWS < JOIN_ROWS ? ROWS : JOIN_ROWS);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    memset(&attr, 0, sizeof(attr));
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, join_kernel<T, DT, ROWS>, a);
}

constexpr size_t HEADER = 64 * 1024;          // the records: more blocks than any launch has
constexpr int MANY_ROWS = 256;                // rows of an item where sequences have many (imm_attn_many.cu)
constexpr int MANY_BATCH = 1024;              // sequences that its plan holds
constexpr int64_t MANY_PATIENCE = 4000000000LL;      // limit on its waits in cycles (about two seconds)

// Whether sequences have so many rows that the products are worth tiles of 128 of them.  At 32 rows the two are about even: 32
// sequences of up to 6000 keys, heads of 128 in float16 152 us here, 131 there; bfloat16 133 and 132; heads of 64 89 and 109; 100
// sequences of up to 200 keys 57 and 77
inline bool use_many(int64_t tokens, int batch, int group, int dim, size_t bytes)
{
    return bytes == 2 && dim <= 128 && batch <= MANY_BATCH && tokens * group > 32 * (int64_t)batch;
}
template <typename T> cudaError_t launch_many(const Args& a, cudaStream_t st);

}  // namespace imm_attn
