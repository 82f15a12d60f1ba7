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
// A request is taken by the blocks of a thread-block cluster, row by row until a token is not taken: rows behind it are
// not read.  A row (and its draft's) takes one pass: a thread keeps its weights relative to an entry of its own, so no
// pass for the maximum comes first; the blocks' maxima and sums meet in every block's shared memory, in the order of
// the blocks, so that all come to the same decision.  The draw reads its rows (from L2) once more: sums of max(p - q, 0) by
// sub-chunk, then the entries of one sub-chunk.
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
constexpr int BLOCKS_PER_SM = 3;
constexpr int PIECES = 64;                    // 16-byte pieces of a sub-chunk: two per lane of a warp
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
    int32_t aligned;                          // all rows begin on 16-byte boundaries
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
template <typename T> struct Row {
    static constexpr int V = 16 / sizeof(T);
    const T* p;
    int n;
    bool aligned;
    // entries V i .. V i + V - 1; those behind the row are -inf.  Only 16-byte granules that hold some of the row are read.
    __device__ __forceinline__ void piece(int i, float (&f)[V]) const
    {
        const T* at = p + (int64_t)i * V;
        if (i * V + V <= n) {
            uint4 r;
            const uint32_t sh = (uint32_t)(uintptr_t)at & 15u;
            const uint4* a = reinterpret_cast<const uint4*>((uintptr_t)at & ~(uintptr_t)15);
            r = __ldg(a);
            if (!aligned && sh) {
                const uint4 h = __ldg(a + 1);
                const uint32_t bits = 8 * (sh & 3u), w[8] = {r.x, r.y, r.z, r.w, h.x, h.y, h.z, h.w};
                uint32_t s[5];
#pragma unroll
                for (int k = 0; k < 5; k++) s[k] = (sh >> 2) == 0 ? w[k] : (sh >> 2) == 1 ? w[k + 1] : (sh >> 2) == 2 ? w[k + 2] : w[k + 3 < 8 ? k + 3 : 7];
                r = make_uint4(__funnelshift_r(s[0], s[1], bits), __funnelshift_r(s[1], s[2], bits), __funnelshift_r(s[2], s[3], bits),
                               __funnelshift_r(s[3], s[4], bits));
            }
            unpack<T>(r, f);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) f[e] = i * V + e < n ? (float)__ldg(at + e) : NEG_INF;
        }
    }
    __device__ __forceinline__ float entry(int i) const { return (float)__ldg(p + i); }
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

struct Stat { double z; float top; int32_t index; };          // sum of the weights relative to the maximum, maximum, its lowest index

struct Shared {
    double table[16];
    Stat stat[2][2][MAX_CLUSTER];             // [which copy][target, draft][block]
    double sums[MAX_CLUSTER];                 // the blocks' shares of the draw's mass
    double warp_d[NW];
    float warp_f[NW];
    uint32_t warp_u[NW];
    int32_t hit;
    double before;
};

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// of this block's sub-chunks [s0, s1) of a row; every thread returns the block's
template <typename T>
__device__ Stat block_stat(const Row<T>& row, int s0, int s1, bool greedy, const Weight& weight, Shared& sh)
{
    constexpr int V = Row<T>::V;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float top = NEG_INF, ref = NEG_INF;
    int index = 0x7FFFFFFF;
    double z = 0.0;
    const float slack = (float)fmin(-0.4 * weight.least, 3e38);
    for (int s = s0 + warp; s < s1; s += NW)
#pragma unroll
        for (int h = 0; h < PIECES / 32; h++) {
            const int i = s * PIECES + h * 32 + lane;
            if (i * V >= row.n) continue;
            float f[V];
            row.piece(i, f);
            float most = f[0];
#pragma unroll
            for (int e = 1; e < V; e++) most = max_nan(most, f[e]);
            if (!(most <= top)) {              // (also for NaN)
                if (most > top) {
                    index = 0x7FFFFFFF;
#pragma unroll
                    for (int e = V - 1; e >= 0; e--) if (f[e] == most) index = i * V + e;
                }
                top = max_nan(top, most);
            }
            if (greedy || !(most > NEG_INF && most < INFINITY)) continue;
            if (ref == NEG_INF || most - ref > slack) {
                z = ref == NEG_INF ? 0.0 : z * weight(ref, most);
                ref = most;
            }
#pragma unroll
            for (int e = 0; e < V; e++) z += weight.of(fmax((double)f[e] - (double)ref, weight.least));
        }
    // the block's maximum, then sums relative to it; among equal maxima the lowest index
    float all = top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all = max_nan(all, __shfl_xor_sync(0xFFFFFFFFu, all, o));
    __syncthreads();
    if (lane == 0) sh.warp_f[warp] = all;
    __syncthreads();
    all = sh.warp_f[0];
#pragma unroll
    for (int w = 1; w < NW; w++) all = max_nan(all, sh.warp_f[w]);
    const uint32_t first = __reduce_min_sync(0xFFFFFFFFu, top == all ? (uint32_t)index : 0x7FFFFFFFu);
    const double mine = warp_sum(ref > NEG_INF && all < INFINITY ? z * weight(ref, all) : 0.0);
    if (lane == 0) { sh.warp_d[warp] = mine; sh.warp_u[warp] = first; }
    __syncthreads();
    Stat r{0.0, all, 0x7FFFFFFF};
#pragma unroll
    for (int w = 0; w < NW; w++) { r.z += sh.warp_d[w]; r.index = min(r.index, (int32_t)sh.warp_u[w]); }
    return r;
}

template <typename T>
__global__ void __launch_bounds__(NT, BLOCKS_PER_SM) verify_kernel(const Args a)
{
    constexpr int V = Row<T>::V;
    extern __shared__ double sub_sum[];       // of this block's sub-chunks
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int nc = (int)cluster.num_blocks(), c = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t request = blockIdx.x / nc;
    if (tid < 16) sh.table[tid] = exp2((double)tid * 0.0625);
    const int64_t o0 = __ldg(a.offsets + request), o1 = __ldg(a.offsets + request + 1);
    const float t = a.temperature_of ? __ldg(a.temperature_of + request) : a.temperature;
    const int n = (int)a.n;
    bool wrong = !(o0 >= 0 && o1 > o0 && o1 <= a.rows) || !(t >= 0.f && t < INFINITY);
    if (a.draft) wrong |= o0 < request || o1 - 1 - request > a.drafts;
    if (!wrong) {
        for (int64_t i = o0 + tid; i < o1; i += NT) {
            const double u = __ldg(a.u + i);
            const int32_t d = i > o0 ? __ldg(a.tokens + i) : 0;
            wrong |= !(u >= 0.0 && u < 1.0) || d < 0 || d >= n;
        }
    }
    wrong = __syncthreads_or(wrong);
    cluster.sync();                           // (all blocks run before one stores into another's memory)
    const bool greedy = t == 0.f;
    Weight weight;
    weight.factor = greedy ? 0.0 : 23.083120654223414219 / (double)t;
    weight.least = -RANGE * (double)t;
    weight.table = sh.table;
    const int nsub = ((n + V - 1) / V + PIECES - 1) / PIECES, per = (nsub + nc - 1) / nc;
    const int s0 = min(nsub, c * per), s1 = min(nsub, s0 + per);

    int taken = 0, copy = 0;
    Stat p{}, q{};
    bool refused = false;                     // the answer replaces a drafted token
    Row<T> target{nullptr, n, a.aligned != 0}, draft{nullptr, n, a.aligned != 0};
    const int k = wrong ? 0 : (int)(o1 - o0 - 1);
    int d = 0;
    while (!wrong) {
        const int64_t row = o0 + taken;
        const bool tested = taken < k, drafted = tested && a.draft && !greedy;
        target.p = (const T*)a.target + row * a.ldt;
        draft.p = drafted ? (const T*)a.draft + (row - request) * a.ldd : nullptr;
        Stat both[2];
        both[0] = block_stat(target, s0, s1, greedy, weight, sh);
        if (drafted) both[1] = block_stat(draft, s0, s1, false, weight, sh);
        if (tid < 2 * nc && (tid < nc || drafted)) {
            Shared* there = cluster.map_shared_rank(&sh, tid < nc ? tid : tid - nc);
            there->stat[copy][tid < nc ? 0 : 1][c] = both[tid < nc ? 0 : 1];
        }
        cluster.sync();
        Stat* found[2] = {&p, &q};
        for (int which = 0; which < (drafted ? 2 : 1); which++) {
            Stat r{0.0, NEG_INF, 0x7FFFFFFF};
            for (int b = 0; b < nc; b++) r.top = max_nan(r.top, sh.stat[copy][which][b].top);
            for (int b = 0; b < nc; b++) {
                const Stat& x = sh.stat[copy][which][b];
                if (x.top == r.top) r.index = min(r.index, x.index);
                if (x.top > NEG_INF && r.top < INFINITY) r.z += x.z * weight(x.top, r.top);
            }
            *found[which] = r;
            wrong |= !(r.top > NEG_INF && r.top < INFINITY);
        }
        copy ^= 1;
        if (wrong || !tested) break;
        d = __ldg(a.tokens + row + 1);
        bool take;
        if (greedy) take = d == p.index;
        else {
            // (quotients: where the two rows are the same, u q < q holds after rounding for every u below 1)
            const double u = __ldg(a.u + row), pd = weight(target.entry(d), p.top) / p.z;
            take = drafted ? u * (weight(draft.entry(d), q.top) / q.z) < pd : u < pd;
        }
        if (!take) { refused = true; break; }
        taken++;
    }
    if (wrong || greedy) {
        if (c == 0 && tid == 0) {
            a.accepted[request] = wrong ? 0 : taken;
            a.token[request] = wrong ? -1 : p.index;
            a.logprob[request] = wrong ? NAN : 0.f;
            a.status[request] = wrong ? IMM_ERR_ARG : IMM_OK;
        }
        cluster.sync();                       // (no block leaves while another may store into its memory)
        return;
    }

    // ---- the draw
    const bool drafted = refused && a.draft;
    int without = refused && !a.draft ? d : -1;           // a proposal without a distribution: d alone is left out
    double ip = 1.0 / p.z, iq = drafted ? 1.0 / q.z : 0.0;
    auto rest = [&](int i, const float (&x)[V], double (&r)[V]) {
        float y[V];
        if (iq != 0.0) draft.piece(i, y);
#pragma unroll
        for (int e = 0; e < V; e++) {
            r[e] = weight(x[e], p.top) * ip;
            if (iq != 0.0) r[e] = fmax(r[e] - weight(y[e], q.top) * iq, 0.0);
            if (i * V + e == without) r[e] = 0.0;
        }
    };
    const double u = __ldg(a.u + o1 - 1);
    double total, before;
    for (;;) {
        double sum = 0.0;
        for (int s = s0 + warp; s < s1; s += NW) {
            double part = 0.0;
#pragma unroll
            for (int h = 0; h < PIECES / 32; h++) {
                const int i = s * PIECES + h * 32 + lane;
                if (i * V >= n) continue;
                float x[V];
                double r[V];
                target.piece(i, x);
                rest(i, x, r);
#pragma unroll
                for (int e = 0; e < V; e++) part += r[e];
            }
            part = warp_sum(part);
            if (lane == 0) sub_sum[s - s0] = part;
        }
        __syncthreads();
        if (warp == 0) {                       // inclusive sums over the block's sub-chunks, 32 at a time
            for (int base = 0; base < s1 - s0; base += 32) {
                double v = base + lane < s1 - s0 ? sub_sum[base + lane] : 0.0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const double w = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += w; }
                v += sum;
                if (base + lane < s1 - s0) sub_sum[base + lane] = v;
                sum = __shfl_sync(0xFFFFFFFFu, v, 31);
            }
            if (lane < nc) cluster.map_shared_rank(&sh, lane)->sums[c] = sum;
        }
        cluster.sync();
        total = before = 0.0;
        for (int b = 0; b < nc; b++) { if (b == c) before = total; total += sh.sums[b]; }
        if (total > 0.0 || (iq == 0.0 && without < 0)) break;
        iq = 0.0; without = -1;               // p and q differ by rounding only: the draw is p's
        cluster.sync();                       // (the sums have been read)
    }
    const double aim = u * total;
    // the block, then the sub-chunk, then the entry; where rounding hides it, the last one at which the sum grows
    int block = -1, last = 0;
    double run = 0.0;
    for (int b = 0; b < nc; b++) {
        const double next = run + sh.sums[b];
        if (next > run) { last = b; if (block < 0 && next > aim) block = b; }
        run = next;
    }
    if (block < 0) block = last;
    if (c == block) {
        const int count = s1 - s0;
        if (tid == 0) sh.hit = 0x7FFFFFFF;
        __syncthreads();
        for (int i = tid; i < count; i += NT) {
            const double from = i ? sub_sum[i - 1] : 0.0;
            if (sub_sum[i] > from && before + sub_sum[i] > aim) atomicMin(&sh.hit, i);
        }
        __syncthreads();
        int sub = sh.hit;
        __syncthreads();
        if (sub == 0x7FFFFFFF) {
            if (tid == 0) sh.hit = -1;
            __syncthreads();
            for (int i = tid; i < count; i += NT) if (sub_sum[i] > (i ? sub_sum[i - 1] : 0.0)) atomicMax(&sh.hit, i);
            __syncthreads();
            sub = max(sh.hit, 0);
        }
        if (warp == 0) {
            const double from = before + (sub ? sub_sum[sub - 1] : 0.0);
            double r[2][V], mine = 0.0;
            float x[V];
            for (int h = 0; h < 2; h++) {      // two neighbouring pieces per lane
                const int i = (s0 + sub) * PIECES + 2 * lane + h;
#pragma unroll
                for (int e = 0; e < V; e++) r[h][e] = 0.0;
                if (i * V < n) {
                    target.piece(i, x);
                    rest(i, x, r[h]);
                }
#pragma unroll
                for (int e = 0; e < V; e++) mine += r[h][e];
            }
            double upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const double w = __shfl_up_sync(0xFFFFFFFFu, upto, o); if (lane >= o) upto += w; }
            const double lower = __shfl_up_sync(0xFFFFFFFFu, upto, 1);
            double at = from + (lane ? lower : 0.0);
            int hit = 0x7FFFFFFF, end = -1;
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (r[h][e] > 0.0) {
                        at += r[h][e];
                        end = ((s0 + sub) * PIECES + 2 * lane + h) * V + e;
                        if (at > aim && hit == 0x7FFFFFFF) hit = end;
                    }
            int answer = (int)__reduce_min_sync(0xFFFFFFFFu, (uint32_t)hit);
            const int behind = __reduce_max_sync(0xFFFFFFFFu, end);
            if (answer == 0x7FFFFFFF) answer = behind;
            if (lane == 0) {
                a.accepted[request] = taken;
                a.token[request] = answer;
                a.logprob[request] = (float)(((double)target.entry(answer) - (double)p.top) / (double)t - log(p.z));
                a.status[request] = IMM_OK;
            }
        }
    }
    cluster.sync();                           // (no block leaves while another may read its sums)
}

template <typename T>
cudaError_t launch(const Args& a, int64_t requests, cudaStream_t st)
{
    constexpr int V = Row<T>::V;
    const int nsub = (int)(((a.n + V - 1) / V + PIECES - 1) / PIECES);
    auto kernel = verify_kernel<T>;
    constexpr int MOST = (IMM_LDD_MAX_N / V + PIECES - 1) / PIECES;
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
    const int64_t slots = (int64_t)BLOCKS_PER_SM * imm::sm_count();
    int nc = 1;
    while (nc < most && nsub > nc * NW && requests * nc * 2 <= slots) nc *= 2;
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
    a.aligned = ((uintptr_t)d.d_target | (uintptr_t)(es * d.ldt) | (uintptr_t)d.d_draft | (uintptr_t)(d.d_draft ? es * d.ldd : 0)) % 16 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == IMM_F32 ? launch<float>(a, d.requests, st)
                          : d.dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, d.requests, st) : launch<__half>(a, d.requests, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}
