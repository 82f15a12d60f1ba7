// Attention over the paged int8 cache (sm_100a): few rows per key, and the call's C ABI (declared in imm.h).
//
//   imm_kv_attention   out = softmax(scale q k^T) v over the positions that a row sees, in one pass over the keys
//
// The mathematics.  With x_s = scale q k_s (times log2(e) throughout) and running m and l, every 16 keys add
// 2^(x_s - m) to l and 2^(x_s - m) v_s to the output; where some x_s passes m by more than a slack, m grows and what is
// there is scaled down.  An int8 is a float16 without rounding, and a row of q times a power of two is one (float32: two
// terms), so the products are exact and the sums float32.  The scale of a page's values is mantissa * 2^exponent: the
// exponent is added to x_s, so that the weights that multiply the values are always near 1 for the keys that matter, and
// comes out of l again by its inverse (far below another page's, where the weight may be 0, by an exponential of its own).
//
// Layout.  Few rows see many keys (a decode step), so the product is turned round: 16 keys are the rows of the matrix
// instruction (m16n8k16) and 8 rows of q its columns.  (The tcgen05 instructions take it turned round as well, 128 keys by 16 columns or
// more, which is not built.)  Every key is used by one warp only: its tiles of 16 keys wait in a ring of its own in shared memory
// (asynchronous copies of whole lines, three tiles ahead), no warp waits for another one within an item, and as the order
// of the contracted index is free, a lane takes whole 16-byte pieces of a key and of the values of four keys.
//
// Work.  A sequence has kv_heads x row tiles items of the same number of 64-key tiles; the tiles of all items, and what
// beginning an item costs, lie in one line that is cut into equal shares, one per block, whatever the lengths are.  A block that
// holds an item whole writes its output; the others write partial results, which a second launch adds up in the order of the
// blocks (it is started while the first one runs, by programmatic dependent launch).
//
// Measured (B200, int8 pages of 8 heads of 128, 4 query heads each): 64 sequences of up to 32000 keys 383 us at 1965 MHz, 5.7 TB/s of the
// 6.5 that a copy reaches, and 445 us at the 1700 MHz that the power limit leaves a GPU that does nothing else: the time goes with
// the multiprocessors' clock, so it is their issue slots (500 instructions a tile of 16 keys and warp) and latencies that bound it.  One
// of 100001 48 us (the same, and the start); one of 2000 10 us and other short ones (latency: 20 thousand cycles, of which a tile is
// two thousand); float32, heads of 80 in a window of 2047: 93 us (650 instructions, issue slots 58 % busy).
#include <atomic>
#include <type_traits>

#include "imm_attn.cuh"
#include "imm_kernels.h"

namespace imm_attn {

constexpr int NW = 4;                         // warps per block
constexpr int NT = NW * 32;
constexpr int TILE = 16 * NW;                 // keys of a tile: 16 per warp
constexpr int LEAST = 2;                      // tiles that a block takes at least: parts of one tile cost more to join than they save (22 us against 11 for 2000 keys)

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transpose(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// DT: 64, 128 or 256, the width of dim's tile.  NQ: tiles of 8 rows.
template <typename T, int DT, int NQ>
struct Few {
    static constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;              // of a row of q
    // of a weight: bf16 outputs have 8 bits, one term of 11 is enough; float16's rounding of an output would be joined by
    // that of the weights (error 1.4 times as large, measured), so they have two terms like float32's
    static constexpr int PTERMS = std::is_same<T, __nv_bfloat16>::value ? 1 : 2;
    static constexpr int ROWS = 8 * NQ;
    static constexpr int KC = DT / 64;        // 16-byte pieces of a key that a lane takes
    static constexpr int VW = DT / 32;        // words of a key's values that it takes
    static constexpr int MT = DT / 16;        // tiles of 16 dims
    static constexpr int CH = DT / 16;        // 16-byte pieces of a key
    static constexpr int BLOCKS = DT == 256 || NQ > 2 ? 2 : 3;        // per SM
    static constexpr int STAGES = 4;          // tiles of a warp in shared memory: one in use, the others on their way (64 requests: three and
                                              // four blocks 419 us, four and three 399)
    static constexpr int HALF = 16 * DT;      // bytes of 16 keys
    static constexpr int RING = STAGES * 2 * HALF;
    struct Shared {
        float m[NW][ROWS], l[NW][ROWS];
        float4 weight[ROWS];
        float inverse[ROWS];
        int64_t at[ROWS];
        int64_t scan[NW];
        int64_t before;
        int seq;
    };
    static constexpr int BYTES = NW * RING + (int)sizeof(Shared);
    static constexpr int PITCH = ROWS * (DT + 4) * 4 <= RING ? DT + 4 : DT;
    static_assert(ROWS * PITCH * 4 <= RING, "a warp's results take the place of its tiles");
    static constexpr int SETUP = 2 + 2 * NQ;  // what beginning an item costs, in tiles (64 requests of up to 2000 keys, one row each: 45 us, not counted 77)
    // where piece c of key r lies in a tile (in pieces): the lanes that read together hit different banks; for key r + z 32 / CH (r below 32 / CH)
    // the place changes by z 32 and these bits
    static __device__ constexpr uint32_t k_turn(int z) { return DT == 64 ? 0 : DT == 128 ? (z & 1) << 1 : z & 3; }
    static __device__ constexpr uint32_t v_turn(int z) { return DT == 64 ? 0 : DT == 128 ? (z & 1) << 2 : (z & 1) | (z >> 1 & 1) << 2; }
    static __device__ __forceinline__ int k_piece(int r, int c) { return r * CH + (DT == 64 ? c : c ^ ((r & 1) << 2 | (r >> 1 & 3))); }
    static __device__ __forceinline__ int v_piece(int r, int c)
    {
        return r * CH + (c ^ (DT == 64 ? (r >> 1 & 1) << 1 : DT == 128 ? (r >> 1 & 3) << 1 : (r >> 1 & 1) | (r >> 2 & 1) << 2));
    }
};

template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool real)       // zeros where there is nothing
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}

template <typename T, int DT, int NQ>
__global__ void __launch_bounds__(NT, Few<T, DT, NQ>::BLOCKS) few_kernel(const Args a)
{
    using F = Few<T, DT, NQ>;
    constexpr int TERMS = F::TERMS, PTERMS = F::PTERMS, ROWS = F::ROWS, KC = F::KC, VW = F::VW, MT = F::MT, CH = F::CH, STAGES = F::STAGES, SETUP = F::SETUP;
    extern __shared__ __align__(1024) uint4 few_shared[];
    typename F::Shared& sh = *reinterpret_cast<typename F::Shared*>(reinterpret_cast<uint8_t*>(few_shared) + NW * F::RING);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    uint8_t* const ring = reinterpret_cast<uint8_t*>(few_shared) + warp * F::RING;
    float* const results = reinterpret_cast<float*>(few_shared);           // a warp's at warp * RING
    const bool packed = a.dim == DT;
    cudaTriggerProgrammaticLaunchCompletion();

    // ---- this block's share of the tiles (a sequence per thread, NT of them at a time)
    auto work_of = [&](int b) { return b < a.batch ? sequence<TILE, ROWS>(a, b).work(a.kv_heads, SETUP) : 0; };
    int64_t total;
    const int64_t first_mine = work_of(tid), first_upto = block_scan<NT>(first_mine, sh.scan, total);
    const int64_t first_total = total;
    for (int i = NT; i < a.batch; i += NT) {
        int64_t part;
        block_scan<NT>(work_of(i + tid), sh.scan, part);
        total += part;
    }
    const int64_t share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)LEAST);
    int64_t x = blockIdx.x * share;
    const int64_t end = min(total, x + share);

    // ---- sequences that see nothing: zeros, or NaN where their length is none
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        const Sequence s = sequence<TILE, ROWS>(a, b);
        if (s.rows && s.tiles == 0) blank<T>(a, s.first, s.rows, s.bad, tid, NT);
    }
    if (tid == 0) a.records[blockIdx.x].parts = 0;
    if (x >= end) return;
    {
        int64_t mine = first_mine, upto = first_upto, carry = first_total;
        for (int i = 0;;) {
            if (x < upto && x >= upto - mine) { sh.seq = i + tid; sh.before = upto - mine; }
            if (carry > x) break;
            int64_t part;
            i += NT;
            mine = work_of(i + tid);
            upto = carry + block_scan<NT>(mine, sh.scan, part);
            carry += part;
        }
    }
    __syncthreads();
    int b = sh.seq;
    int64_t before = sh.before;
    Sequence s = sequence<TILE, ROWS>(a, b);
    const int64_t begin = x;

    while (x < end) {
        while (x >= before + s.work(a.kv_heads, SETUP)) { before += s.work(a.kv_heads, SETUP); s = sequence<TILE, ROWS>(a, ++b); }
        const int64_t item = (x - before) / (SETUP + s.tiles), item_begin = before + item * (SETUP + s.tiles) + SETUP;
        const int j0 = (int)max((int64_t)0, x - item_begin), j1 = (int)min((int64_t)s.tiles, end - item_begin);
        const int slot = x == begin ? 0 : 1;
        x = item_begin + s.tiles;
        if (j1 <= j0) continue;                // (its tiles begin in the next share)
        const int kvh = (int)(item / s.row_tiles), r0 = (int)(item - (int64_t)kvh * s.row_tiles) * ROWS;
        const int nrows = (int)min((int64_t)ROWS, (int64_t)s.rows * a.group - r0);
        const int place0 = s.length - s.rows;                          // position of the sequence's first row

        // ---- the keys: the first ones are on their way while the rows of q are read
        const int count = j1 - j0;
        const int32_t* table = a.table + b * a.ld_table;
        const int64_t head_entries = (int64_t)a.dim << a.page_log;
        auto key_of = [&](int i) { const int j = j0 + i; return (j < s.sink ? j : s.low + j - s.sink) * TILE + 16 * warp; };
        int32_t pages = -1;                    // of the 32 tiles around the one asked for, a lane each, and their scales; those of the 32 before
        float ks = NAN, vs = NAN, former_ks = NAN, former_vs = NAN;
        auto refill = [&](int base) {
            const int i = base + lane;
            pages = -1;
            former_ks = ks; former_vs = vs;
            ks = vs = NAN;
            if (i < count) {
                const int k0 = key_of(i);
                if (k0 < s.length) {
                    const int32_t at = __ldg(table + (k0 >> a.page_log));
                    if (at >= 0 && at < a.pages) {
                        pages = at;
                        ks = __ldg(a.k_scale + (int64_t)at * a.kv_heads + kvh);
                        vs = __ldg(a.v_scale + (int64_t)at * a.kv_heads + kvh);
                    }
                }
            }
        };
        const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
        const uint32_t k_lane = ring_at + 16 * F::k_piece(lane / CH, lane % CH), v_lane = ring_at + F::HALF + 16 * F::v_piece(lane / CH, lane % CH);
        auto ask = [&](int i) {                // tile i into its stage, whole lines at a time
            if (i < count) {
                if ((i & 31) == 0) refill(i);
                const int32_t page = __shfl_sync(0xFFFFFFFFu, pages, i & 31);
                const int64_t at = kvh * head_entries + (int64_t)(key_of(i) & ((1 << a.page_log) - 1)) * a.dim;
                const int8_t *k = a.k_cache + (page >= 0 ? (int64_t)page * a.k_page_stride + at : 0), *v = a.v_cache + (page >= 0 ? (int64_t)page * a.v_page_stride + at : 0);
                const uint32_t to_k = k_lane + i % STAGES * (2 * F::HALF), to_v = v_lane + i % STAGES * (2 * F::HALF);
                if (packed) {                  // (16 keys in a row: all offsets are constants)
                    k += page >= 0 ? lane * 16 : 0;
                    v += page >= 0 ? lane * 16 : 0;
#pragma unroll
                    for (int z = 0; z < CH / 2; z++) {
                        copy16((to_k ^ F::k_turn(z) * 16) + z * 512, k + z * 512, page >= 0);
                        copy16((to_v ^ F::v_turn(z) * 16) + z * 512, v + z * 512, page >= 0);
                    }
                } else {
                    const bool real = page >= 0 && lane % CH * 16 < a.dim;
                    const int from = real ? lane / CH * a.dim + lane % CH * 16 : 0, next = real ? 32 / CH * a.dim : 0;
#pragma unroll
                    for (int z = 0; z < CH / 2; z++) {
                        copy16((to_k ^ F::k_turn(z) * 16) + z * 512, k + (from + z * next), real);
                        copy16((to_v ^ F::v_turn(z) * 16) + z * 512, v + (from + z * next), real);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; i++) ask(i);
        // ---- rows of q: column g of tile n; word w of piece c of a lane holds the dims 64 c + 16 t + 4 w + (0..3), or (where dim does
        // not fill its tile, so that steps without a dim can be left out) 64 c + 16 w + 4 t + (0..3)
        uint32_t qf[NQ][TERMS][KC * 4][2];
        float factor[NQ][2], m[NQ][2], l[NQ][2];
        int place[NQ][2];
        const int t0 = r0 / a.group, h0 = r0 - t0 * a.group;
        Four<T> raw[NQ][KC * 4];
        // (what lies behind the last row or dim is read inside them, and cleared)
        auto dim_of = [&](int w) { return packed ? 64 * (w >> 2) + 16 * t + 4 * (w & 3) : 16 * w + 4 * t; };
#pragma unroll
        for (int n = 0; n < NQ; n++) {
            const Place at = place_of(a, t0, h0, min(n * 8 + g, nrows - 1));
            const T* const row = (const T*)a.q + (s.first + at.query) * a.ldq + (int64_t)(kvh * a.group + at.head) * a.hsq;
            if (a.q_aligned) {
#pragma unroll
                for (int w = 0; w < KC * 4; w++) raw[n][w] = *reinterpret_cast<const Four<T>*>(row + min(dim_of(w), a.dim - 4));
            } else {
#pragma unroll
                for (int w = 0; w < KC * 4; w++)
#pragma unroll
                    for (int i = 0; i < 4; i++) raw[n][w].v[i] = row[min(dim_of(w), a.dim - 4) + i];
            }
        }
#pragma unroll
        for (int n = 0; n < NQ; n++) {
            float v[KC * 16];
            float top = 0.f;
            bool finite = true;
#pragma unroll
            for (int w = 0; w < KC * 4; w++) {
                const bool real = n * 8 + g < nrows && dim_of(w) < a.dim;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    float& y = v[w * 4 + i];
                    y = real ? (float)raw[n][w].v[i] : 0.f;
                    top = fmaxf(top, fabsf(y));
                    finite &= fabsf(y) < INFINITY;
                }
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                finite &= (bool)__shfl_xor_sync(0xFFFFFFFFu, (int)finite, o);
            }
            // the row times 2^(13 - e): its largest magnitude lies in [2^13, 2^14)
            const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100);
            const float up = finite ? __uint_as_float((uint32_t)(127 + 13 - e) << 23) : 0.f;
            const float f = finite ? a.scale * __uint_as_float((uint32_t)(127 - 13 + e) << 23) : NAN;
#pragma unroll
            for (int w = 0; w < KC * 4; w++) {
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; i++) y[i] = finite ? v[w * 4 + i] * up : 0.f;
                qf[n][0][w][0] = pack(y[0], y[1]);
                qf[n][0][w][1] = pack(y[2], y[3]);
                if (TERMS == 2) {
                    const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&qf[n][0][w][0]));
                    const float2 h1 = __half22float2(*reinterpret_cast<const __half2*>(&qf[n][0][w][1]));
                    qf[n][TERMS - 1][w][0] = pack(y[0] - h0.x, y[1] - h0.y);
                    qf[n][TERMS - 1][w][1] = pack(y[2] - h1.x, y[3] - h1.y);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                factor[n][i] = __shfl_sync(0xFFFFFFFFu, f, (2 * t + i) * 4);
                const int w = n * 8 + 2 * t + i;
                place[n][i] = w < nrows ? place0 + place_of(a, t0, h0, w).query : -1;
                m[n][i] = NOTHING;
                l[n][i] = 0.f;
            }
        }
        float widest = -INFINITY;              // exponent of the largest value scale so far
        const int place_first = place0 + t0, place_last = place0 + place_of(a, t0, h0, nrows - 1).query;
        float o[NQ][MT][4];
#pragma unroll
        for (int n = 0; n < NQ; n++)
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int z = 0; z < 4; z++) o[n][i][z] = 0.f;

        for (int i = 0; i < count; i++) {
            const int k0 = key_of(i);
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                      // (tile i is there for all lanes, and tile i - 1 has been read)
            ask(i + STAGES - 1);
            const uint4* const tile_k = reinterpret_cast<const uint4*>(ring + i % STAGES * (2 * F::HALF));
            const uint4* const tile_v = tile_k + F::HALF / 16;
            const bool ahead = (i & ~31) != (min(i + STAGES - 1, count - 1) & ~31);           // the latest scales are of the next tiles
            const Factors f = factors(__shfl_sync(0xFFFFFFFFu, ahead ? former_ks : ks, i & 31), __shfl_sync(0xFFFFFFFFu, ahead ? former_vs : vs, i & 31));
            // two sums that do not wait for each other: of every other step, or of the two terms (the second's products would be cut off
            // beside the first one's)
            float sc[NQ][4], low[NQ][4];
#pragma unroll
            for (int n = 0; n < NQ; n++)
#pragma unroll
                for (int z = 0; z < 4; z++) sc[n][z] = low[n][z] = 0.f;
            auto scores = [&](int w, uint32_t k_lo, uint32_t k_hi) {               // words of keys g and g + 8
                const uint32_t lo = k_lo ^ 0x80808080u, hi = k_hi ^ 0x80808080u;
                const uint32_t am[4] = {halves(lo, 0x4140), halves(hi, 0x4140), halves(lo, 0x4342), halves(hi, 0x4342)};
#pragma unroll
                for (int n = 0; n < NQ; n++) {
                    mma(TERMS == 1 && (w & 1) ? low[n] : sc[n], am, qf[n][0][w]);
                    if (TERMS == 2) mma(low[n], am, qf[n][TERMS - 1][w]);
                }
            };
            if (packed) {
#pragma unroll
                for (int c = 0; c < KC; c++) {
                    const uint4 k_lo = tile_k[F::k_piece(g, 4 * c + t)], k_hi = tile_k[F::k_piece(g + 8, 4 * c + t)];
#pragma unroll
                    for (int w = 0; w < 4; w++) scores(c * 4 + w, (&k_lo.x)[w], (&k_hi.x)[w]);
                }
            } else {
#pragma unroll
                for (int w = 0; w < KC * 4; w++)
                    if (16 * w < a.dim)
                        scores(w, reinterpret_cast<const uint32_t*>(tile_k + F::k_piece(g, w))[t], reinterpret_cast<const uint32_t*>(tile_k + F::k_piece(g + 8, w))[t]);
            }
            const bool full = k0 + 15 <= place_first && (a.window == 0 || place_last - k0 < a.window || k0 + 15 < a.sinks);
            const bool far = widest - f.exponent > FAR;
            widest = fmaxf(widest, f.exponent);
            bool grown = far;
#pragma unroll
            for (int n = 0; n < NQ; n++)
#pragma unroll
                for (int z = 0; z < 4; z++) {
                    float& y = sc[n][z];
                    y += low[n][z];
                    y = fmaf(y, factor[n][z & 1] * f.k, f.exponent);
                    if (!full) {
                        const int k = k0 + g + (z & 2) * 4, p = place[n][z & 1];
                        if (!(k <= p && (a.window == 0 || p - k < a.window || k < a.sinks))) y = -INFINITY;
                    }
                    grown |= y > limit_of(m[n][z & 1]);
                }
            if (__any_sync(0xFFFFFFFFu, grown)) {
#pragma unroll
                for (int n = 0; n < NQ; n++)
#pragma unroll
                    for (int z = 0; z < 2; z++) {
                        float top = fmaxf(sc[n][z], sc[n][z + 2]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                        const float next = fmaxf(m[n][z], top - BIAS);
                        const float half = ex2(0.5f * (m[n][z] - next)), down = half * half;
                        m[n][z] = next;
                        l[n][z] = l[n][z] * half * half;         // (scaled(): down may be 0)
#pragma unroll
                        for (int d = 0; d < MT; d++) { o[n][d][z] *= down; o[n][d][z + 2] *= down; }
                        if (far) l[n][z] += ex2(sc[n][z] - m[n][z] - f.exponent) + ex2(sc[n][z + 2] - m[n][z] - f.exponent);
                    }
            }
            const float inverse = far ? 0.f : f.inverse;
            uint32_t pb[NQ][PTERMS][2];
#pragma unroll
            for (int n = 0; n < NQ; n++) {
                float p[4];
#pragma unroll
                for (int z = 0; z < 4; z++) {
                    p[z] = ex2(sc[n][z] - m[n][z & 1]);
                    l[n][z & 1] = fmaf(p[z], inverse, l[n][z & 1]);
                    p[z] *= f.mantissa;
                }
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    const uint32_t hi = pack(p[2 * z], p[2 * z + 1]);
                    pb[n][0][z] = transpose(hi);
                    if (PTERMS == 2) {
                        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                        pb[n][PTERMS - 1][z] = transpose(pack(p[2 * z] - h.x, p[2 * z + 1] - h.y));
                    }
                }
            }
            // word w of a lane: dims g DT / 8 + 4 w + (0..3), or 32 w + 4 g + (0..3)
            auto values = [&](int w, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
                v0 ^= 0x80808080u; v1 ^= 0x80808080u; v2 ^= 0x80808080u; v3 ^= 0x80808080u;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t ab = __byte_perm(v0, v1, h ? 0x7362 : 0x5140), cd = __byte_perm(v2, v3, h ? 0x7362 : 0x5140);
                    const uint32_t am[4] = {halves(ab, 0x4140), halves(ab, 0x4342), halves(cd, 0x4140), halves(cd, 0x4342)};
#pragma unroll
                    for (int n = 0; n < NQ; n++)
#pragma unroll
                        for (int z = 0; z < PTERMS; z++) mma(o[n][2 * w + h], am, pb[n][z]);
                }
            };
            if (packed && DT == 64) {
                uint2 v[4];
#pragma unroll
                for (int z = 0; z < 4; z++) v[z] = reinterpret_cast<const uint2*>(tile_v + F::v_piece(2 * t + (z & 1) + (z & 2) * 4, g >> 1))[g & 1];
                values(0, v[0].x, v[1].x, v[2].x, v[3].x);
                values(1, v[0].y, v[1].y, v[2].y, v[3].y);
            } else if (packed) {
#pragma unroll
                for (int c = 0; c < VW / 4; c++) {
                    uint4 v[4];
#pragma unroll
                    for (int z = 0; z < 4; z++) v[z] = tile_v[F::v_piece(2 * t + (z & 1) + (z & 2) * 4, g * (VW / 4) + c)];
#pragma unroll
                    for (int w = 0; w < 4; w++) values(4 * c + w, (&v[0].x)[w], (&v[1].x)[w], (&v[2].x)[w], (&v[3].x)[w]);
                }
            } else {
#pragma unroll
                for (int w = 0; w < VW; w++)
                    if (32 * w < a.dim) {
                        uint32_t v[4];
#pragma unroll
                        for (int z = 0; z < 4; z++) v[z] = reinterpret_cast<const uint32_t*>(tile_v + F::v_piece(2 * t + (z & 1) + (z & 2) * 4, 2 * w + (g >> 2)))[g & 3];
                        values(w, v[0], v[1], v[2], v[3]);
                    }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();                          // (the warp's results take the place of its tiles)

        // ---- the warps' results together
#pragma unroll
        for (int n = 0; n < NQ; n++)
#pragma unroll
            for (int z = 0; z < 2; z++) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][z] += __shfl_xor_sync(0xFFFFFFFFu, l[n][z], d);
                const int r = n * 8 + 2 * t + z;
                if (g == 0) { sh.m[warp][r] = m[n][z]; sh.l[warp][r] = l[n][z]; }
#pragma unroll
                for (int i = 0; i < MT; i++)
                    *reinterpret_cast<float2*>(results + warp * (F::RING / 4) + r * F::PITCH + (packed ? g * (DT / 8) + 2 * i : 32 * (i >> 1) + 4 * g + 2 * (i & 1))) =
                        make_float2(o[n][i][z], o[n][i][z + 2]);
            }
        __syncthreads();
        const bool whole = count == s.tiles;
        float* part = a.parts + ((int64_t)blockIdx.x * 2 + slot) * slot_floats<DT, ROWS>();
        if (!whole && j0 == 0 && tid == 0)
            a.records[blockIdx.x] = Record{s.first, kvh, r0, nrows, (int)(1 + (s.tiles - count + share - 1) / share), slot, 0};
        if (tid < ROWS) {                      // a row's weights of the warps' results
            const int r = tid;
            float top = sh.m[0][r], weight[NW], lsum = 0.f;
#pragma unroll
            for (int w = 1; w < NW; w++) top = fmaxf(top, sh.m[w][r]);
#pragma unroll
            for (int w = 0; w < NW; w++) { weight[w] = ex2(sh.m[w][r] - top); lsum += scaled(sh.l[w][r], sh.m[w][r] - top); }
            sh.weight[r] = make_float4(weight[0], weight[1], weight[2], weight[3]);
            if (!whole) {
                part[ROWS * DT + r] = top;
                part[ROWS * DT + ROWS + r] = lsum;
            } else if (r < nrows) {
                const Place at = place_of(a, t0, h0, r);
                const int head = kvh * a.group + at.head;
                const int64_t row = s.first + at.query;
                sh.inverse[r] = lsum == 0.f ? 0.f : 1.f / lsum;
                sh.at[r] = row * a.ldo + (int64_t)head * a.hso;
                if (a.lse) a.lse[row * a.heads + head] = lsum == 0.f ? -INFINITY : (top + log2f(lsum)) * LN2;
            }
        }
        __syncthreads();
        static_assert(NW == 4, "weights in a float4");
#pragma unroll 2
        for (int idx = tid; idx < ROWS * (DT / 4); idx += NT) {
            const int r = idx / (DT / 4), d = idx % (DT / 4) * 4;
            const float4 weight = sh.weight[r];
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < NW; w++) {
                const float4 v = *reinterpret_cast<const float4*>(results + w * (F::RING / 4) + r * F::PITCH + d);
                const float by = (&weight.x)[w];
                y.x = fmaf(by, v.x, y.x); y.y = fmaf(by, v.y, y.y); y.z = fmaf(by, v.z, y.z); y.w = fmaf(by, v.w, y.w);
            }
            if (!whole) {
                *reinterpret_cast<float4*>(part + r * DT + d) = y;
            } else if (r < nrows && d < a.dim) {
                const float inverse = sh.inverse[r];
                const Four<T> four{to<T>(y.x * inverse), to<T>(y.y * inverse), to<T>(y.z * inverse), to<T>(y.w * inverse)};
                T* const out = (T*)a.out + sh.at[r] + d;
                if (a.out_aligned) *reinterpret_cast<Four<T>*>(out) = four;
                else {
#pragma unroll
                    for (int i = 0; i < 4; i++) out[i] = four.v[i];
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, int DT, int NQ>
cudaError_t launch_few(const Args& a, cudaStream_t st)
{
    using F = Few<T, DT, NQ>;
    const int grid = F::BLOCKS * imm::sm_count();
    // once per device: permission for the shared memory
    static std::atomic<int> allowed[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(few_kernel<T, DT, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::BYTES);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(1, std::memory_order_relaxed);
    }
    few_kernel<T, DT, NQ><<<grid, NT, F::BYTES, st>>>(a);
    e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_join<T, DT, F::ROWS>(a, grid, st);
}

template <typename T>
cudaError_t launch(const Args& a, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2) {
        if (use_many(a.tokens, a.batch, a.group, a.dim, sizeof(T))) return launch_many<T>(a, st);
    }
    // Tiles of 8 rows at once: as many as a sequence has on average.  Three go with two blocks per multiprocessor instead of three,
    // and still win where they save reading the keys twice (20 rows of 32 sequences of up to 6000 keys, when this was
    // chosen: 110 us, two tiles 133); 32 rows take two tiles twice (158 us, three tiles 190)
    const int64_t rows = a.tokens * a.group;
    const int tiles = rows <= 8 * (int64_t)a.batch ? 1 : rows > 16 * (int64_t)a.batch && rows <= 24 * (int64_t)a.batch ? 3 : 2;
    if (a.dim > 128) return launch_few<T, 256, 1>(a, st);
    if constexpr (sizeof(T) == 2) {
        if (a.dim > 64) return tiles == 1 ? launch_few<T, 128, 1>(a, st) : tiles == 2 ? launch_few<T, 128, 2>(a, st) : launch_few<T, 128, 3>(a, st);
        return tiles == 1 ? launch_few<T, 64, 1>(a, st) : tiles == 2 ? launch_few<T, 64, 2>(a, st) : launch_few<T, 64, 3>(a, st);
    } else {
        return a.dim > 64 ? launch_few<T, 128, 1>(a, st) : launch_few<T, 64, 1>(a, st);
    }
}

size_t workspace(int64_t tokens, int batch, int heads, int kv_heads, int dim, int dtype)
{
    // two slots per block of the first launch: at most three blocks of 16 rows or two of 24 per SM; one block of MANY_ROWS rows
    const size_t wide = dim > 128 ? 256 : dim > 64 ? 128 : 64;
    const int rows = use_many(tokens, batch, heads / kv_heads, dim, dtype == IMM_F32 ? 4 : 2) ? MANY_ROWS : 48;
    return HEADER + (size_t)imm::sm_count() * 2 * rows * (wide + 2) * sizeof(float);
}

bool valid(int64_t tokens, int batch, int heads, int kv_heads, int dim, int dtype)
{
    return (dtype == IMM_F32 || dtype == IMM_BF16 || dtype == IMM_F16) && tokens >= 0 && tokens <= IMM_KV_MAX_TOKENS && batch >= 0 &&
           batch <= IMM_KV_MAX_BATCH && kv_heads > 0 && heads > 0 && heads <= IMM_KV_MAX_HEADS && heads % kv_heads == 0 && dim > 0 &&
           dim <= IMM_KV_MAX_DIM && dim % 16 == 0 && tokens * (heads / kv_heads) <= IMM_KV_MAX_ROWS;
}

}  // namespace imm_attn

extern "C" {

size_t imm_kv_attention_workspace(int64_t tokens, int batch, int heads, int kv_heads, int dim, int dtype)
{
    using namespace imm_attn;
    if (!valid(tokens, batch, heads, kv_heads, dim, dtype)) return 0;
    return workspace(tokens, batch, heads, kv_heads, dim, dtype);
}

int imm_kv_attention(const imm_kv_attention_desc* desc_host, void* stream)
{
    return imm_kv_attention_limited(desc_host, imm_attn::MANY_PATIENCE, 0x7FFFFFFF, stream);
}

int imm_kv_attention_limited(const imm_kv_attention_desc* desc_host, int64_t cycles, int steps, void* stream)
{
    using namespace imm_attn;
    if (!desc_host || desc_host->reserved || desc_host->reserved2) return IMM_ERR_ARG;
    const imm_kv_attention_desc& d = *desc_host;
    if (d.dtype != IMM_F32 && d.dtype != IMM_BF16 && d.dtype != IMM_F16) return IMM_ERR_ARG;
    if (!(d.scale > 0.f) || !(d.scale < INFINITY) || d.window < 0 || d.sinks < 0) return IMM_ERR_ARG;
    if (!valid(d.tokens, d.batch, d.heads, d.kv_heads, d.dim, d.dtype)) return IMM_ERR_SHAPE;
    const bool any = d.batch > 0 && d.tokens > 0;
    if (any && (!d.d_q || !d.d_k_cache || !d.d_v_cache || !d.d_k_scale || !d.d_v_scale || !d.d_table || !d.d_offsets || !d.d_length || !d.d_out))
        return IMM_ERR_ARG;
    int log = 4;
    while (log < 7 && (1 << log) != d.page) log++;
    if ((1 << log) != d.page) return IMM_ERR_SHAPE;
    if (d.max_pages <= 0 || d.max_pages > IMM_KV_MAX_LENGTH / d.page || d.pages <= 0 || d.pages > 0x7FFFFFFF || d.ld_table < d.max_pages) return IMM_ERR_SHAPE;
    const int64_t entries = (int64_t)d.kv_heads * d.page * d.dim;
    if (d.hsq < d.dim || d.hso < d.dim || d.ldq < d.dim || d.ldo < d.dim || d.k_page_stride < entries || d.v_page_stride < entries) return IMM_ERR_SHAPE;
    if (d.k_page_stride % 16 || d.v_page_stride % 16) return IMM_ERR_ALIGN;
    const uintptr_t es = d.dtype == IMM_F32 ? 4 : 2;
    if ((uintptr_t)d.d_q % es || (uintptr_t)d.d_out % es || (uintptr_t)d.d_k_cache % 16 || (uintptr_t)d.d_v_cache % 16 || (uintptr_t)d.d_k_scale % 4 ||
        (uintptr_t)d.d_v_scale % 4 || (uintptr_t)d.d_table % 4 || (uintptr_t)d.d_offsets % 8 || (uintptr_t)d.d_length % 4 || (uintptr_t)d.d_lse % 4 ||
        (uintptr_t)d.d_ws % 16)
        return IMM_ERR_ALIGN;
    if (!any) return IMM_OK;
    if (!d.d_ws || d.ws_bytes < imm_kv_attention_workspace(d.tokens, d.batch, d.heads, d.kv_heads, d.dim, d.dtype)) return IMM_ERR_WORKSPACE;
    Args a{};
    a.q = d.d_q; a.k_cache = d.d_k_cache; a.v_cache = d.d_v_cache; a.k_scale = d.d_k_scale; a.v_scale = d.d_v_scale;
    a.table = d.d_table; a.offsets = d.d_offsets; a.length = d.d_length; a.out = d.d_out; a.lse = d.d_lse;
    a.records = (Record*)d.d_ws; a.parts = (float*)((char*)d.d_ws + HEADER);
    a.tokens = d.tokens; a.ldq = d.ldq; a.hsq = d.hsq; a.ldo = d.ldo; a.hso = d.hso; a.pages = d.pages;
    a.k_page_stride = d.k_page_stride; a.v_page_stride = d.v_page_stride; a.ld_table = d.ld_table;
    a.batch = d.batch; a.heads = d.heads; a.kv_heads = d.kv_heads; a.group = d.heads / d.kv_heads; a.dim = d.dim; a.page_log = log;
    a.window = d.window; a.sinks = d.window ? d.sinks : 0;
    a.q_aligned = ((uintptr_t)d.d_q | (uintptr_t)(es * d.ldq) | (uintptr_t)(es * d.hsq)) % 16 == 0;
    a.out_aligned = ((uintptr_t)d.d_out | (uintptr_t)(es * d.ldo) | (uintptr_t)(es * d.hso)) % 16 == 0;
    a.max_length = (int64_t)d.max_pages * d.page;
    a.patience = cycles;
    a.steps = steps;
    a.scale = d.scale * LOG2E;
    a.per_group = 1.f / (float)a.group;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = d.dtype == IMM_F32 ? launch<float>(a, st) : d.dtype == IMM_BF16 ? launch<__nv_bfloat16>(a, st) : launch<__half>(a, st);
    return e == cudaSuccess ? IMM_OK : imm::cuda_failed(e);
}

}  // extern "C"
