// Expert dispatch and combine (sm_100a) and their C ABI (declared in imm.h).
//
//   imm_moe_dispatch   rows of the tokens sorted by expert: the ragged left operands of the experts' products
//   imm_moe_combine    the experts' output rows back in token order, weighted and added up
//
// Both move rows of some KiB and are bound by HBM.  The order is a stable counting sort of the (token, slot) pairs:
// pairs are cut into runs of RUN; a counting launch writes how many pairs of every run go to every expert (no such
// launch when there is one run only); a moving launch then gives every block a few neighbouring tokens: the block
// works out the first row of its pairs from the counts of the runs before and by counting the pairs of its own run
// that come first, so no scan launch and no waiting between blocks is needed.  Counting uses integer atomics in
// shared memory, whose order does not matter; ranks among the pairs of one expert follow the pair's number (32 pairs
// a step, matched within a warp), so the result is the same on every run.
//
// Measured: dispatch of 16384 x 4096 int8, top-2 of 8 (198 MB): 44 us, 4.5 TB/s, the moving launch alone 35 us; combine of
// 4096 x 4096 int32 to bf16, top-2 (168 MB): 36.9 us, 4.6 TB/s (8 columns per lane and one row at a time: 47 us).
//
// Rows need not be aligned to 16 bytes: stores are, and a 16-byte piece of a row that begins anywhere is put
// together from the two aligned vectors that it touches.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/imm.h"
#include "imm_kernels.h"

namespace imm_moe {

constexpr int NT = 256;
constexpr int NW = NT / 32;
constexpr int RUN = 2048;                     // pairs per counted run, or a multiple of it for calls with more than MAX_RUNS of them
constexpr int MAX_RUNS = 256;                 // (every moving block reads the counts of all runs, and counts its own run up to its
                                              // first pair: with runs that grow, 18 ms for 2^26 pairs against 0.06 for 2^19)
constexpr int MAX_E = IMM_MOE_MAX_EXPERTS;
constexpr int MAX_PAIRS = 512;                // pairs per moving block (a token's may exceed none of them: top <= 64)

struct Dispatch {
    const char* x;
    const float* scale;
    const int32_t* expert;
    char* out;
    float* out_scale;
    int64_t* offsets;
    int32_t *position, *status;
    int32_t* counts;                          // nruns x experts, then one word per run: an expert that does not exist (nullptr: one run)
    int64_t tokens, pairs, ldx, ldo;          // ld in bytes
    int64_t row_bytes, run;                   // run: pairs per run
    int32_t top, experts, nruns;
    int32_t tokens_per_block;
};

// 16 bytes that begin at any address; only aligned vectors that hold some of them are read
__device__ __forceinline__ uint4 load16(const char* p)
{
    const uint32_t sh = (uint32_t)(uintptr_t)p & 15u;
    const uint4* a = reinterpret_cast<const uint4*>((uintptr_t)p & ~(uintptr_t)15);
    const uint4 lo = __ldg(a);
    if (sh == 0) return lo;
    const uint4 hi = __ldg(a + 1);
    const uint32_t bits = 8 * (sh & 3u);
    uint32_t w0, w1, w2, w3, w4;
    switch (sh >> 2) {                        // (the same for all lanes of a row)
    case 0: w0 = lo.x; w1 = lo.y; w2 = lo.z; w3 = lo.w; w4 = hi.x; break;
    case 1: w0 = lo.y; w1 = lo.z; w2 = lo.w; w3 = hi.x; w4 = hi.y; break;
    case 2: w0 = lo.z; w1 = lo.w; w2 = hi.x; w3 = hi.y; w4 = hi.z; break;
    default: w0 = lo.w; w1 = hi.x; w2 = hi.y; w3 = hi.z; w4 = hi.w; break;
    }
    return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits),
                      __funnelshift_r(w3, w4, bits));
}

// f(p, expert of pair p) for p in [b, end), RUN of them at a time: all loads of a thread on their way at once
template <typename F> __device__ __forceinline__ void each_pair(const int32_t* expert, int64_t b, int64_t end, F&& f)
{
    for (; b < end; b += RUN) {
        int e[RUN / NT];
#pragma unroll
        for (int q = 0; q < RUN / NT; q++) { const int64_t p = b + q * NT + threadIdx.x; e[q] = p < end ? expert[p] : -1; }
#pragma unroll
        for (int q = 0; q < RUN / NT; q++) { const int64_t p = b + q * NT + threadIdx.x; if (p < end) f(p, e[q]); }
    }
}

__global__ void __launch_bounds__(NT) count_kernel(const Dispatch d)
{
    __shared__ int hist[MAX_E];
    cudaTriggerProgrammaticLaunchCompletion();        // (the moving blocks may take their places; they wait for the counts)
    for (int e = threadIdx.x; e < d.experts; e += NT) hist[e] = 0;
    __syncthreads();
    const int64_t b = (int64_t)blockIdx.x * d.run;
    int wrong = 0;
    each_pair(d.expert, b, min(d.pairs, b + d.run), [&](int64_t, int e) {
        if (e >= 0 && e < d.experts) atomicAdd(&hist[e], 1);
        else wrong |= e != -1;
    });
    wrong = __syncthreads_or(wrong);
    int32_t* mine = d.counts + (int64_t)blockIdx.x * d.experts;
    for (int e = threadIdx.x; e < d.experts; e += NT) mine[e] = hist[e];
    if (threadIdx.x == 0) d.counts[(int64_t)d.nruns * d.experts + blockIdx.x] = wrong;
}

// ALIGNED: every row of x and out begins and ends on a 16-byte boundary.
template <bool ALIGNED>
__global__ void __launch_bounds__(NT) move_kernel(const Dispatch d)
{
    __shared__ int total[MAX_E], before[MAX_E];       // pairs of an expert in all runs / before the pairs of this block
    __shared__ int first[MAX_E];                      // first output row of an expert
    __shared__ int rows[MAX_PAIRS];
    __shared__ int warp_sum[NW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = d.experts;
    const int64_t t0 = (int64_t)blockIdx.x * d.tokens_per_block;
    const int ntok = (int)min((int64_t)d.tokens_per_block, d.tokens - t0);     // (0 for a call without tokens)
    const int64_t p0 = t0 * d.top;
    const int np = ntok * d.top;
    const int run = (int)(p0 / d.run);
    for (int e = tid; e < E; e += NT) { total[e] = 0; before[e] = 0; }
    __syncthreads();
    int wrong = 0;
    if (d.counts) {
        each_pair(d.expert, run * d.run, p0, [&](int64_t, int e) { if (e >= 0 && e < E) atomicAdd(&before[e], 1); });
        cudaGridDependencySynchronize();
        // counts of the runs: a few threads per expert
        const int lanes = E <= NT / 8 ? 8 : E <= NT / 2 ? 2 : 1;
        for (int i = tid; i < E * lanes; i += NT) {
            const int e = i / lanes;
            int s = 0, b = 0;
            for (int r = i % lanes; r < d.nruns; r += lanes) {
                const int c = d.counts[(int64_t)r * E + e];
                if (r < run) b += c;
                s += c;
            }
            if (s) atomicAdd(&total[e], s);
            if (b) atomicAdd(&before[e], b);
        }
        if (blockIdx.x == 0) for (int r = tid; r < d.nruns; r += NT) wrong |= d.counts[(int64_t)d.nruns * E + r];
    } else {
        each_pair(d.expert, 0, d.pairs, [&](int64_t p, int e) {
            if (e >= 0 && e < E) {
                atomicAdd(&total[e], 1);
                if (p < p0) atomicAdd(&before[e], 1);
            } else wrong |= e != -1;
        });
    }
    __syncthreads();
    // exclusive scan of the totals: first rows
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += NT) {
        const int e = e0 + tid;
        const int v = e < E ? total[e] : 0;
        int s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= o) s += t; }
        if (lane == 31) warp_sum[warp] = s;
        __syncthreads();
        int base = carry, all = 0;
#pragma unroll
        for (int w = 0; w < NW; w++) { if (w < warp) base += warp_sum[w]; all += warp_sum[w]; }
        if (e < E) first[e] = base + s - v;
        carry += all;
        __syncthreads();
    }
    if (blockIdx.x == 0) {
        for (int e = tid; e < E; e += NT) d.offsets[e] = first[e];
        wrong = __syncthreads_or(wrong);
        if (tid == 0) { d.offsets[E] = carry; *d.status = wrong ? IMM_ERR_ARG : IMM_OK; }
    }
    // output rows of the block's pairs
    if (warp == 0)
        for (int i0 = 0; i0 < np; i0 += 32) {
            const int i = i0 + lane;
            int e = -1;
            if (i < np) {
                e = d.expert[p0 + i];
                if (e < 0 || e >= E) e = -1;
            }
            const unsigned mates = __match_any_sync(0xFFFFFFFFu, e);
            int row = -1;
            if (e >= 0) row = first[e] + before[e] + __popc(mates & ((1u << lane) - 1u));
            __syncwarp();
            if (e >= 0 && lane == __ffs(mates) - 1) before[e] += __popc(mates);
            __syncwarp();
            if (i < np) {
                rows[i] = row;
                d.position[p0 + i] = row;
                if (row >= 0 && d.out_scale) d.out_scale[row] = d.scale[t0 + i / d.top];
            }
        }
    __syncthreads();
    // Rows: long ones by the whole block, a token at a time, short ones by a warp each.
    const bool together = ALIGNED && d.row_bytes >= 16 * NT * 2;
    if (ALIGNED) {
        const int who = together ? tid : lane, step = together ? NT : 32;
        const int words = (int)(d.row_bytes / 16), parts = !together && words >= 64 ? 2 : 1, share = (words + parts - 1) / parts;
        for (int u = together ? 0 : warp; u < ntok * parts; u += together ? 1 : NW) {
            const int t = u / parts, w0 = (u % parts) * share, w1 = min(words, w0 + share);
            const uint4* src = reinterpret_cast<const uint4*>(d.x + (t0 + t) * d.ldx);
            const int* mine = rows + t * d.top;
            int i = w0 + who;
            for (; i + 3 * step < w1; i += 4 * step) {
                uint4 v[4];
#pragma unroll
                for (int q = 0; q < 4; q++) v[q] = __ldg(src + i + q * step);
                for (int k = 0; k < d.top; k++) {
                    const int r = mine[k];
                    if (r < 0) continue;
                    uint4* dst = reinterpret_cast<uint4*>(d.out + r * d.ldo);
#pragma unroll
                    for (int q = 0; q < 4; q++) dst[i + q * step] = v[q];
                }
            }
            for (; i < w1; i += step) {
                const uint4 v = __ldg(src + i);
                for (int k = 0; k < d.top; k++)
                    if (mine[k] >= 0) reinterpret_cast<uint4*>(d.out + mine[k] * d.ldo)[i] = v;
            }
        }
    } else {
        for (int t = warp; t < ntok; t += NW) {
            const char* src = d.x + (t0 + t) * d.ldx;
            const int* mine = rows + t * d.top;
            for (int k = 0; k < d.top; k++) {
                const int r = mine[k];
                if (r < 0) continue;
                char* dst = d.out + r * d.ldo;
                const int64_t head = min(d.row_bytes, (int64_t)((16 - ((uintptr_t)dst & 15)) & 15));
                const int64_t words = (d.row_bytes - head) / 16, tail = head + 16 * words;
                if (lane < head) dst[lane] = src[lane];
                for (int64_t i = lane; i < words; i += 32) *reinterpret_cast<uint4*>(dst + head + 16 * i) = load16(src + head + 16 * i);
                if (tail + lane < d.row_bytes) dst[tail + lane] = src[tail + lane];
            }
        }
    }
}

// ---- combine ----

struct Combine {
    const void* y;
    const float* row_scale;
    const int32_t* position;
    const float* weight;
    void* out;
    int64_t tokens, y_rows, ldy, ldo;
    int32_t top, cols;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(int32_t v) { return (float)v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }

// A warp takes 512 columns of a token, PIECES of them per lane in pieces of V = 16 / sizeof(T).  Pieces are laid so that
// their stores are aligned; the columns before the first and behind the last whole piece are taken one by one.
constexpr int PIECES = 16;

template <typename T, typename O>
__global__ void __launch_bounds__(NT) combine_kernel(const Combine c, int segments)
{
    constexpr int V = 16 / (int)sizeof(T), C = PIECES / V;
    constexpr int STORE = V * (int)sizeof(O) < 16 ? V * (int)sizeof(O) : 16;   // bytes a store is aligned to
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * NW + (threadIdx.x >> 5);
    const int64_t t = item / segments;
    if (t >= c.tokens) return;                        // (whole warp)
    const int seg = (int)(item % segments);
    O* out = (O*)c.out + t * c.ldo;
    const int head = min(c.cols, (int)(((STORE - ((uintptr_t)out & (STORE - 1))) & (STORE - 1)) / sizeof(O)));
    const int whole = (c.cols - head) / V, p0 = seg * (32 * C);

    // rows and factors: one slot per lane, 32 at a time
    float acc[C][V], edge = 0.f;
#pragma unroll
    for (int q = 0; q < C; q++)
#pragma unroll
        for (int e = 0; e < V; e++) acc[q][e] = 0.f;
    // the columns outside the pieces: lanes of the first segment
    const int rest = c.cols - whole * V;              // head, then the columns behind the last piece
    const int col = lane < head ? lane : whole * V + lane;
    const bool odd = seg == 0 && lane < rest;
    for (int k0 = 0; k0 < c.top; k0 += 32) {
        int r = -1;
        float f = 0.f;
        if (k0 + lane < c.top) {
            r = c.position[t * c.top + k0 + lane];
            if (r >= c.y_rows) r = -1;
            if (r >= 0) {
                f = c.weight ? c.weight[t * c.top + k0 + lane] : 1.f;
                if (c.row_scale) f *= c.row_scale[r];
            }
        }
        const int n = min(32, c.top - k0);
        for (int k = 0; k < n; k += 2) {       // two rows' pieces on their way together; added in the order of the slots
            uint4 raw[2][C];
            const T* y[2];
            float fk[2];
#pragma unroll
            for (int z = 0; z < 2; z++) {
                const int rk = __shfl_sync(0xFFFFFFFFu, r, (k + z) & 31);
                fk[z] = __shfl_sync(0xFFFFFFFFu, f, (k + z) & 31);
                y[z] = (rk < 0 || k + z >= n) ? nullptr : (const T*)c.y + (int64_t)rk * c.ldy;
#pragma unroll
                for (int q = 0; q < C; q++)
                    if (y[z] && p0 + 32 * q + lane < whole) raw[z][q] = load16((const char*)(y[z] + head + (p0 + 32 * q + lane) * V));
            }
#pragma unroll
            for (int z = 0; z < 2; z++)
                if (y[z]) {
#pragma unroll
                    for (int q = 0; q < C; q++)
                        if (p0 + 32 * q + lane < whole) {
                            const T* v = reinterpret_cast<const T*>(&raw[z][q]);
#pragma unroll
                            for (int e = 0; e < V; e++) acc[q][e] = fmaf(to_f(v[e]), fk[z], acc[q][e]);
                        }
                    if (odd) edge = fmaf(to_f(y[z][col]), fk[z], edge);
                }
        }
    }
#pragma unroll
    for (int q = 0; q < C; q++) {
        const int piece = p0 + 32 * q + lane;
        if (piece >= whole) continue;
        alignas(16) O o[V];
#pragma unroll
        for (int e = 0; e < V; e++) put(o + e, acc[q][e]);
        O* to = out + head + piece * V;
        if constexpr (V * sizeof(O) == 8) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(o);
        else
#pragma unroll
            for (int e = 0; e < V * (int)sizeof(O) / 16; e++) reinterpret_cast<uint4*>(to)[e] = reinterpret_cast<const uint4*>(o)[e];
    }
    if (odd) put(out + col, edge);
}

template <typename T>
cudaError_t launch_combine(const Combine& c, int out_dtype, cudaStream_t st)
{
    constexpr int SEG = 32 * PIECES;
    const int segments = (c.cols + SEG - 1) / SEG;
    const int64_t blocks = (c.tokens * segments + NW - 1) / NW;
    const unsigned grid = (unsigned)blocks;
    if (out_dtype == IMM_F32) combine_kernel<T, float><<<grid, NT, 0, st>>>(c, segments);
    else if (out_dtype == IMM_BF16) combine_kernel<T, __nv_bfloat16><<<grid, NT, 0, st>>>(c, segments);
    else combine_kernel<T, __half><<<grid, NT, 0, st>>>(c, segments);
    return cudaGetLastError();
}

bool valid(int64_t tokens, int top, int experts)
{
    return tokens >= 0 && top > 0 && top <= IMM_MOE_MAX_TOP && experts > 0 && experts <= IMM_MOE_MAX_EXPERTS &&
           tokens <= IMM_MOE_MAX_PAIRS / top;
}

int64_t run_length(int64_t pairs) { return (pairs / ((int64_t)RUN * MAX_RUNS) + 1) * RUN; }
int runs_of(int64_t pairs) { return (int)((pairs + run_length(pairs) - 1) / run_length(pairs)); }

}  // namespace imm_moe

extern "C" {

size_t imm_moe_dispatch_workspace(int64_t tokens, int top, int experts)
{
    using namespace imm_moe;
    if (!valid(tokens, top, experts)) return 0;
    const int n = runs_of(tokens * top);
    return n > 1 ? (size_t)n * (experts + 1) * sizeof(int32_t) : 0;
}

int imm_moe_dispatch(const imm_dispatch_desc* desc_host, void* stream)
{
    using namespace imm_moe;
    if (!desc_host || desc_host->reserved) return IMM_ERR_ARG;
    const auto [d_x, d_scale, d_expert, d_out, d_out_scale, d_offsets, d_position, d_status, d_ws, ws_bytes, tokens, cols, ldx, ldo, out_rows,
                top, experts, elem_bytes, reserved] = *desc_host;
    if (!d_offsets || !d_status || (tokens > 0 && (!d_x || !d_expert || !d_out || !d_position))) return IMM_ERR_ARG;
    if ((d_scale == nullptr) != (d_out_scale == nullptr)) return IMM_ERR_ARG;
    if (elem_bytes != 1 && elem_bytes != 2 && elem_bytes != 4) return IMM_ERR_ARG;
    if (!valid(tokens, top, experts)) return IMM_ERR_SHAPE;
    if (cols <= 0 || cols > IMM_NORM_MAX_COLS || ldx < cols || ldo < cols || out_rows < tokens * top) return IMM_ERR_SHAPE;
    if ((uintptr_t)d_x % elem_bytes || (uintptr_t)d_out % elem_bytes || (uintptr_t)d_scale % 4 || (uintptr_t)d_out_scale % 4 ||
        (uintptr_t)d_expert % 4 || (uintptr_t)d_offsets % 8 || (uintptr_t)d_position % 4 || (uintptr_t)d_status % 4 || (uintptr_t)d_ws % 16)
        return IMM_ERR_ALIGN;
    const size_t need = imm_moe_dispatch_workspace(tokens, top, experts);
    if (need && (!d_ws || ws_bytes < need)) return IMM_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    Dispatch d{};
    d.x = (const char*)d_x; d.scale = d_scale; d.expert = d_expert; d.out = (char*)d_out; d.out_scale = d_out_scale;
    d.offsets = d_offsets; d.position = d_position; d.status = d_status; d.counts = need ? (int32_t*)d_ws : nullptr;
    d.tokens = tokens; d.pairs = tokens * top; d.ldx = ldx * elem_bytes; d.ldo = ldo * elem_bytes; d.row_bytes = cols * elem_bytes;
    d.top = top; d.experts = experts; d.nruns = runs_of(d.pairs); d.run = run_length(d.pairs);
    // tokens per block: four blocks per SM, one token each for short calls, within the block's list of pairs
    const int64_t blocks = 4 * (int64_t)imm::sm_count();
    d.tokens_per_block = (int32_t)((tokens + blocks - 1) / blocks);
    if (d.tokens_per_block > MAX_PAIRS / top) d.tokens_per_block = MAX_PAIRS / top;
    if (d.tokens_per_block < 1) d.tokens_per_block = 1;
    const int64_t grid = tokens ? (tokens + d.tokens_per_block - 1) / d.tokens_per_block : 1;
    const uintptr_t all = (uintptr_t)d_x | (uintptr_t)d_out | (uintptr_t)d.ldx | (uintptr_t)d.ldo | (uintptr_t)d.row_bytes;
    auto kernel = all % 16 == 0 ? move_kernel<true> : move_kernel<false>;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(NT);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    memset(&attr, 0, sizeof(attr));
    if (need) {                               // launched while the counts are made; waits for them itself
        count_kernel<<<(unsigned)d.nruns, NT, 0, st>>>(d);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return imm::cuda_failed(e);
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    }
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, d);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}

int imm_moe_combine(const imm_combine_desc* desc_host, void* stream)
{
    using namespace imm_moe;
    if (!desc_host || desc_host->reserved) return IMM_ERR_ARG;
    const auto [d_y, d_row_scale, d_position, d_weight, d_out, tokens, cols, y_rows, ldy, ldo, top, dtype, out_dtype, reserved] = *desc_host;
    if (tokens > 0 && (!d_position || !d_out || (y_rows > 0 && !d_y))) return IMM_ERR_ARG;
    if (dtype != IMM_I32 && dtype != IMM_F32 && dtype != IMM_BF16 && dtype != IMM_F16) return IMM_ERR_ARG;
    if (out_dtype != IMM_F32 && out_dtype != IMM_BF16 && out_dtype != IMM_F16) return IMM_ERR_ARG;
    if (!valid(tokens, top, 1)) return IMM_ERR_SHAPE;
    if (cols <= 0 || cols > IMM_NORM_MAX_COLS || y_rows < 0 || y_rows > IMM_MOE_MAX_PAIRS || ldy < cols || ldo < cols) return IMM_ERR_SHAPE;
    const uintptr_t es = dtype == IMM_I32 || dtype == IMM_F32 ? 4 : 2, os = out_dtype == IMM_F32 ? 4 : 2;
    if ((uintptr_t)d_y % es || (uintptr_t)d_out % os || (uintptr_t)d_row_scale % 4 || (uintptr_t)d_position % 4 || (uintptr_t)d_weight % 4)
        return IMM_ERR_ALIGN;
    if (tokens > ((int64_t)1 << 33) / ((cols + 511) / 512)) return IMM_ERR_SHAPE;          // more pieces than a launch has
    if (tokens == 0) return IMM_OK;
    const Combine c{d_y, d_row_scale, d_position, d_weight, d_out, tokens, y_rows, ldy, ldo, top, (int32_t)cols};
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == IMM_I32) e = launch_combine<int32_t>(c, out_dtype, st);
    else if (dtype == IMM_F32) e = launch_combine<float>(c, out_dtype, st);
    else if (dtype == IMM_BF16) e = launch_combine<__nv_bfloat16>(c, out_dtype, st);
    else e = launch_combine<__half>(c, out_dtype, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}

}  // extern "C"
