// Attention over the paged int8 cache (sm_100a): many rows per key (prompts, drafted tokens), on the tensor cores' tcgen05
// instructions.
//
// The mathematics is that of imm_attn.cu: running maximum m and sum l per row, weights 2^(x - m) with the exponent of a
// page's value scale inside x (log2 of the whole scale here), m moved only when a weight passes a slack.  Tiles without masked
// keys, whose scores are small enough for one rounding of x - m and whose value scales lie near each other, take fewer steps.
//
// A block (one per SM) takes items of up to 256 rows, against tiles of 128 keys.  Its warps have roles:
//   converters (4 warps)   int8 tiles from HBM through registers to float16 in shared memory, in the 128-byte swizzle that
//                          the matrix instructions read; keys and values alike (the values are the operand's other major)
//   two warps              the factors of the next tiles' pages, for either stream
//   one issuing thread     S = Q K^T into tensor memory; O += P V with P from tensor memory
//   softmax (2 x 4 warps)  a thread per row: its row of q (once per item), S to registers, weights as float16 back over S;
//                          rescales O in tensor memory where m moves, which is rare; the output
// The two groups of softmax warps work on two streams in turn, so that the tensor cores compute one stream's products while
// the other's weights are made.  An item of more than 128 rows gives the streams 128 rows each and every tile of keys to
// both; one of fewer gives both the same rows, and the tiles in turn (their results are added up at the end).
//
// Work: the tiles that some row of an item sees, and what an item costs besides, over all items, in equal shares (imm_attn.cu).
// The tensor cores need 2048 cycles for a tile of keys and 256 rows of 128 dims, and the exponentials as many; converting takes
// about 400 issue slots of them.  Measured (B200): a prompt of 4096 with 32 heads of 128 218 us, 630 TFLOP/s of the causal
// products.  What bounds it is each stream's chain of products, softmax (2900 cycles) and products again (1500): about 4600
// cycles per tile pair, and 17 thousand per item for its rows of q and its output, which nothing overlaps.
//
// Every wait is bounded: a block whose wait runs out writes NaN for the rows that it holds and those that were still to come, and leaves.
#include <atomic>
#include <type_traits>

#include "imm_attn.cuh"
#include "imm_kernels.h"

namespace imm_attn {

namespace {

constexpr int NT = 512;                       // softmax 0-127, 128-255; converters 256-383; issuer 384; factors from 416 and 448 on
constexpr int TILE = 128;                     // keys of a tile
constexpr int STAGES = 4;
constexpr int SETUP = 4;                      // what an item costs besides its tiles, in tiles (prompt of 4096, when this was added: 247 us, not counted 366)
constexpr uint32_t HALF_TILE = 128 * 128;     // bytes of 128 rows x 64 float16

__device__ __forceinline__ uint32_t smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem(b)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem(b)) : "memory"); }
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem(b)), "r"(parity) : "memory");
    return ok;
}
// a block's limit on its waits, in cycles, and whether one ran out
struct Limit { long long patience; int stop; };
__device__ __forceinline__ bool bar_wait_long(uint64_t* b, uint32_t parity, volatile Limit* stop)
{
    const long long begin = clock64();
    while (!bar_try(b, parity)) {
        if (stop->stop) return false;
        if (clock64() - begin > stop->patience) { stop->stop = 1; return false; }
    }
    return true;
}
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile Limit* stop)
{
    return bar_try(b, parity) || bar_wait_long(b, parity, stop);
}
// after generic writes to shared memory that the tensor cores read
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* b) { asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem(b)) : "memory"); }

__device__ __forceinline__ bool elect()       // one lane of a warp
{
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r;
}

// shared memory operand: 128-byte swizzle; lbo, sbo in bytes
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((address >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 | 1ull << 46 | 2ull << 61;
}
// float16 operands, float32 sums, 128 rows, n columns; the second operand by columns (its contiguous index is n) or not
__device__ __forceinline__ constexpr uint32_t shape(int n, bool by_columns)
{
    return 1u << 4 | (by_columns ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (128u / 16) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
#define IMM_R8(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3]), "=r"(a[i + 4]), "=r"(a[i + 5]), "=r"(a[i + 6]), "=r"(a[i + 7])
#define IMM_W8(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3]), "r"(a[i + 4]), "r"(a[i + 5]), "r"(a[i + 6]), "r"(a[i + 7])
// 32 columns of this thread's lane
__device__ __forceinline__ void load32(uint32_t (&v)[32], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
                 "%29,%30,%31}, [%32];" : IMM_R8(v, 0), IMM_R8(v, 8), IMM_R8(v, 16), IMM_R8(v, 24) : "r"(at));
}
__device__ __forceinline__ void load16(uint32_t (&v)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : IMM_R8(v, 0), IMM_R8(v, 8) : "r"(at));
}
__device__ __forceinline__ void store16(uint32_t at, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), IMM_W8(v, 0), IMM_W8(v, 8) : "memory");
}
// (the registers pass through, so that nothing that reads them moves in front of the wait)
#define IMM_P8(a, i) "+r"(a[i]), "+r"(a[i + 1]), "+r"(a[i + 2]), "+r"(a[i + 3]), "+r"(a[i + 4]), "+r"(a[i + 5]), "+r"(a[i + 6]), "+r"(a[i + 7])
__device__ __forceinline__ void wait_load(uint32_t (&v)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : IMM_P8(v, 0), IMM_P8(v, 8)::"memory"); }
__device__ __forceinline__ void wait_load(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : IMM_P8(v, 0), IMM_P8(v, 8), IMM_P8(v, 16), IMM_P8(v, 24)::"memory");
}
__device__ __forceinline__ void wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// two float32 at once
__device__ __forceinline__ uint64_t pair(float lo, float hi) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z)); return r; }
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y)); return r; }

__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// An item: MANY_ROWS rows of one key head of a sequence, and the tiles that some of them sees
struct Item {
    int64_t first;
    int32_t rows, length, kvh, r0, nrows;     // of the sequence; of the item
    int32_t t0, h0;                           // r0's query and head of the group
    int32_t low, sink, tiles;
    bool split;                               // 128 rows at most: the streams share the tiles
};
__device__ __forceinline__ int tiles_of(const Args& a, int rows, int length, int r0, int& low, int& sink)
{
    const int64_t all = (int64_t)rows * a.group;
    const int place = length - rows, p0 = max(place + r0 / a.group, 0);
    const int p1 = max(place + (int)((min(all, (int64_t)r0 + MANY_ROWS) - 1) / a.group), 0);
    low = a.window ? max(0, p0 - a.window + 1) / TILE : 0;
    sink = a.window ? min((min(a.sinks, p1 + 1) + TILE - 1) / TILE, low) : 0;
    return sink + p1 / TILE + 1 - low;
}
struct Rows { int64_t first; int32_t rows, length, row_tiles; bool bad; };
__device__ __forceinline__ Rows rows_of(const Args& a, int b)
{
    Rows s;
    const int64_t o0 = __ldg(a.offsets + b), o1 = __ldg(a.offsets + b + 1);
    s.length = __ldg(a.length + b);
    s.first = o0;
    s.rows = o0 >= 0 && o1 >= o0 && o1 <= a.tokens ? (int)(o1 - o0) : 0;
    s.bad = s.length < 0 || s.length > a.max_length;
    s.row_tiles = s.bad || s.length == 0 ? 0 : (int)(((int64_t)s.rows * a.group + MANY_ROWS - 1) / MANY_ROWS);
    return s;
}

// A block's way through its share; every role goes it by itself
struct Cursor {
    int32_t b, kvh, rt, u0;                   // u0: where in the next item's SETUP + tiles units the share begins
    int64_t left;
    // the next item; its tiles from .. from + count - 1 are this block's
    __device__ __forceinline__ bool next(const Args& a, Item& it, int& from, int& count)
    {
        if (left <= 0) return false;
        Rows s = rows_of(a, b);
        while (rt >= s.row_tiles) {
            rt = 0;
            if (s.row_tiles == 0 || ++kvh == a.kv_heads) { kvh = 0; s = rows_of(a, ++b); }
        }
        it.first = s.first; it.rows = s.rows; it.length = s.length; it.kvh = kvh; it.r0 = rt * MANY_ROWS;
        it.t0 = it.r0 / a.group; it.h0 = it.r0 - it.t0 * a.group;
        it.nrows = (int)min((int64_t)MANY_ROWS, (int64_t)s.rows * a.group - it.r0);
        it.tiles = tiles_of(a, s.rows, s.length, it.r0, it.low, it.sink);
        it.split = it.nrows <= 128;
        const int u1 = (int)min((int64_t)(SETUP + it.tiles), u0 + left);
        from = max(0, u0 - SETUP);
        count = max(0, u1 - SETUP) - from;
        left -= u1 - u0;
        u0 = 0;
        rt++;
        return count > 0;                      // (or the share ends before the item's tiles)
    }
};
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ int tile_at(const Item& it, int j) { return j < it.sink ? j : it.low + j - it.sink; }

template <int DT> struct Layout {
    static constexpr int HALVES = DT / 64;
    static constexpr uint32_t OPERAND = HALVES * HALF_TILE;      // bytes of 128 rows
    static constexpr uint32_t Q = 0, RING = 2 * OPERAND, END = RING + STAGES * OPERAND;
    static constexpr uint32_t S = 0, O = 256;                    // columns of tensor memory: stream s at S + 128 s, O + 128 s
};

constexpr int FACTORS = 4;                    // tiles whose factors wait for the softmax warps of a stream
struct Control {
    // of a tile's groups of 16 keys: k's scale, log2 of v's, its inverse (0: far below another's), 0 where the values count as 0
    float4 factors[2][FACTORS][8];
    float largest[2][FACTORS];                // the tile's largest scale of keys; infinity where some values count as 0 or lie far below
    uint64_t f_full[2][FACTORS], f_empty[2][FACTORS];
    uint64_t q_full[2], s_full[2], p_full[2], full[STAGES], empty[STAGES], o_full, hand[2], last;
    struct { Cursor cursor; Item item; int32_t from, count; } now[8];      // a softmax warp's item (kept here: its registers are for S)
    float row_factor[8][32];
    int64_t work[MANY_BATCH];                 // units of a sequence and key head: SETUP and the tiles of each item
    int64_t share, left;
    int32_t b, kvh, rt, u0;
    uint32_t tmem;
    Limit limit;
};

template <typename T, int DT>
__global__ void __launch_bounds__(NT, 1) many_kernel(const Args a)
{
    using L = Layout<DT>;
    extern __shared__ uint8_t raw_shared[];
    uint8_t* const base = raw_shared + (1024 - (smem(raw_shared) & 1023)) % 1024;
    Control& c = *reinterpret_cast<Control*>(base + L::END);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile Limit* const stop = &c.limit;
    cudaTriggerProgrammaticLaunchCompletion();

    // ---- setup: barriers, tensor memory, this block's share
    if (tid == 0) {
        for (int i = 0; i < 2; i++) { bar_init(&c.q_full[i], 128); bar_init(&c.s_full[i], 1); bar_init(&c.p_full[i], 128); bar_init(&c.hand[i], 128); }
        for (int i = 0; i < STAGES; i++) { bar_init(&c.full[i], 128); bar_init(&c.empty[i], 1); }
        for (int i = 0; i < 2 * FACTORS; i++) { bar_init(&c.f_full[0][i], 1); bar_init(&c.f_empty[0][i], 128); }
        bar_init(&c.o_full, 1);
        bar_init(&c.last, 1);
        c.limit.patience = a.patience;
        c.limit.stop = 0;
        c.left = 0;
        a.records[blockIdx.x].parts = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 12) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem(&c.tmem)) : "memory");
    for (int b = warp; b < a.batch; b += NT / 32) {
        const Rows s = rows_of(a, b);
        if (s.rows && s.row_tiles == 0 && b % gridDim.x == blockIdx.x) blank<T>(a, s.first, s.rows, s.bad, lane, 32);
        long long sum = 0;
        for (int rt = lane; rt < s.row_tiles; rt += 32) { int low, sink; sum += SETUP + tiles_of(a, s.rows, s.length, rt * MANY_ROWS, low, sink); }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) c.work[b] = sum;
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 0) {
        const int per = (a.batch + 31) / 32, b0 = min(a.batch, lane * per), b1 = min(a.batch, b0 + per);
        long long mine = 0;
        for (int b = b0; b < b1; b++) mine += c.work[b] * a.kv_heads;
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xFFFFFFFFu, upto, o); if (lane >= o) upto += t; }
        const long long total = __shfl_sync(0xFFFFFFFFu, upto, 31), share = (total + gridDim.x - 1) / gridDim.x, x = blockIdx.x * share;
        if (x < total) {
            if (x >= upto - mine && x < upto) {
                long long before = upto - mine;
                int b = b0;
                while (x >= before + c.work[b] * a.kv_heads) before += c.work[b++] * a.kv_heads;
                c.b = b;
                c.kvh = (int)((x - before) / c.work[b]);
                c.left = min(share, total - x);
                c.share = (x - before) % c.work[b];                   // (for the search below)
            }
            __syncwarp();
            const int b = c.b;
            long long rest = c.share;
            const Rows s = rows_of(a, b);
            int rt = 0;
            for (int r = 0;; r += 32) {
                int low, sink;
                const long long n = r + lane < s.row_tiles ? SETUP + tiles_of(a, s.rows, s.length, (r + lane) * MANY_ROWS, low, sink) : 0;
                long long sum = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xFFFFFFFFu, sum, o); if (lane >= o) sum += t; }
                const uint32_t found = __ballot_sync(0xFFFFFFFFu, sum > rest);
                if (found) {
                    const int at = __ffs(found) - 1;
                    rest -= __shfl_sync(0xFFFFFFFFu, sum - n, at);
                    rt = r + at;
                    break;
                }
                rest -= __shfl_sync(0xFFFFFFFFu, sum, 31);
                if (r >= s.row_tiles) break;                           // (not reached: rest lies below the sequence's work)
            }
            if (lane == 0) { c.rt = rt; c.u0 = (int)rest; c.share = share; }
        }
    }
    __syncthreads();
    const uint32_t tmem = c.tmem;
    Cursor cursor{c.b, c.kvh, c.rt, c.u0, c.left};
    Item it;
    int from, count;

    if (warp < 8) {
        // ---- softmax: thread = row of stream s
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int s = warp >> 2, r = tid & 127;
        const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21);           // this warp's lanes
        const uint32_t s_at = mine + L::S + 128 * s, o_at = mine + L::O + 128 * s;
        uint32_t s_phase = 0, o_phase = 0, h_phase = 0, tile = 0;
        bool first_item = true, ok = true;
        auto& now = c.now[warp];
        if (lane == 0) now.cursor = cursor;
        __syncwarp();
        while (ok) {
            {
                Cursor here = now.cursor;
                Item item;
                int i0, n;
                const bool more = here.next(a, item, i0, n);
                __syncwarp();
                if (!more) break;
                if (lane == 0) { now.cursor = here; now.item = item; now.from = i0; now.count = n; }
                __syncwarp();
            }
            const Item& it = now.item;
            const int row = it.split ? r : 128 * s + r;
            const bool real = row < it.nrows, some = (row & ~31) < it.nrows;           // this row; some row of this warp
            const int place0 = it.length - it.rows, place = real ? place0 + place_of(a, it.t0, it.h0, row).query : -1;
            // ---- rows of q times a power of two, float16, swizzled: this warp's 32, a row in DT / 8 lanes
            float factor;
            {
                constexpr int LANES = DT / 8, TURNS = LANES / 2;       // 32 / LANES rows a turn, 16 rows in TURNS of them
                const int piece = lane % LANES, nrows = it.nrows;      // (copies: the stores below could change shared memory)
                const Place p = place_of(a, it.t0, it.h0, min(row, nrows - 1));
                // (what lies behind the last row or dim is read inside them, and cleared)
                const T* const src = (const T*)a.q + (it.first + p.query) * a.ldq + (int64_t)(it.kvh * a.group + p.head) * a.hsq;
                const int dim0 = min(piece * 8, a.dim - 8);
                uint8_t* const q_at = base + L::Q + s * L::OPERAND + (r & ~31) * 128 + (piece >> 3) * HALF_TILE;
#pragma unroll 1
                for (int z0 = 0; z0 < 32; z0 += 16) {
                    uint4 v[TURNS];
                    const T* at_row[TURNS];
#pragma unroll
                    for (int k = 0; k < TURNS; k++)
                        at_row[k] = reinterpret_cast<const T*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)src, z0 + k * (32 / LANES) + lane / LANES)) + dim0;
                    if (a.q_aligned) {
#pragma unroll
                        for (int k = 0; k < TURNS; k++) v[k] = __ldg(reinterpret_cast<const uint4*>(at_row[k]));
                    } else {
#pragma unroll
                        for (int k = 0; k < TURNS; k++) {
                            const uint16_t* u = reinterpret_cast<const uint16_t*>(at_row[k]);
#pragma unroll
                            for (int e = 0; e < 4; e++) (&v[k].x)[e] = (uint32_t)__ldg(u + 2 * e) | (uint32_t)__ldg(u + 2 * e + 1) << 16;
                        }
                    }
                    uint32_t top[TURNS];
#pragma unroll
                    for (int k = 0; k < TURNS; k++) {
                        const int z = z0 + k * (32 / LANES) + lane / LANES;
                        if (row - lane + z >= nrows || piece * 8 >= a.dim) v[k] = make_uint4(0, 0, 0, 0);
                        const T* x = reinterpret_cast<const T*>(&v[k]);
                        top[k] = 0;
#pragma unroll
                        for (int e = 0; e < 8; e++) top[k] = max(top[k], __float_as_uint(fabsf((float)x[e])));         // (infinity and NaN order above)
                    }
#pragma unroll
                    for (int o = 1; o < LANES; o <<= 1)
#pragma unroll
                        for (int k = 0; k < TURNS; k++) top[k] = max(top[k], __shfl_xor_sync(0xFFFFFFFFu, top[k], o));
#pragma unroll
                    for (int k = 0; k < TURNS; k++) {
                        const int z = z0 + k * (32 / LANES) + lane / LANES;
                        const T* x = reinterpret_cast<const T*>(&v[k]);
                        const bool finite = top[k] < 0x7F800000u;
                        const int e = max((int)(top[k] >> 23) - 127, -100);
                        const float up = __uint_as_float((uint32_t)(127 + 13 - (finite ? e : 0)) << 23);
                        uint4 w;
#pragma unroll
                        for (int e2 = 0; e2 < 4; e2++) (&w.x)[e2] = finite ? pack((float)x[2 * e2] * up, (float)x[2 * e2 + 1] * up) : 0u;
                        *reinterpret_cast<uint4*>(q_at + z * 128 + ((piece ^ z) & 7) * 16) = w;
                        if (piece == 0) c.row_factor[warp][z] = finite ? a.scale * __uint_as_float((uint32_t)(127 - 13 + e) << 23) : NAN;
                    }
                }
                __syncwarp();
                factor = real ? c.row_factor[warp][lane] : 0.f;
            }
            fence_async();
            bar_arrive(&c.q_full[s]);
            // Sums of products lie below 2^14 127 128, 2^28 of them: below 2^22, where a rounding of a score is 2^-3 of a binary order at most,
            // no weight passes float16's range for one that its maximum has and it has not
            const float most_factor = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(factor)));

            const int row_first = it.r0 + (it.split ? 0 : 128 * s), row_last = min(it.r0 + it.nrows - 1, row_first + 127);
            const int place_first = place0 + place_of(a, it.t0, it.h0, row_first - it.r0).query, place_last = place0 + place_of(a, it.t0, it.h0, row_last - it.r0).query;
            const int step = it.split ? 2 : 1, j_begin = now.from + (it.split ? s : 0), j_end = now.from + now.count;
            float m = NOTHING, l = 0.f;
            for (int j = j_begin; ok && j < j_end; j += step, tile++) {
                ok = bar_wait(&c.f_full[s][tile % FACTORS], tile / FACTORS & 1, stop);
                const float4* const f_at = c.factors[s][tile % FACTORS];
                ok = ok && bar_wait(&c.s_full[s], s_phase, stop);
                ok = __all_sync(0xFFFFFFFFu, ok);
                s_phase ^= 1;
                if (!ok) break;
                fence_after();
                if (some) {
                    const int k0 = tile_at(it, j) * TILE;
                    const bool full = k0 + TILE - 1 <= place_first && (a.window == 0 || place_last - k0 < a.window || k0 + TILE - 1 < a.sinks);
                    // MASKED: keys that a row does not see, or large scores.  FAR_APART: value scales of 0, or far from each other, too.
                    auto weights = [&](auto masked, auto far_apart) {
                        constexpr bool MASKED = decltype(masked)::value, FAR_APART = decltype(far_apart)::value;
                        // the keys of chunk i (32 of them) that the row sees
                        auto seen = [&](int i) {
                            const int k = k0 + 32 * i;
                            uint32_t bits = first_bits(place + 1 - k);
                            if (a.window) bits &= ~first_bits(place - a.window + 1 - k) | first_bits(a.sinks - k);
                            return bits;
                        };
                        uint32_t x[2][32];
                        // the largest x: of a group of 16 keys, the largest product's (factors are not negative)
                        float top = -INFINITY;
                        load32(x[0], s_at);
#pragma unroll 1
                        for (int i2 = 0; i2 < 4; i2 += 2)
#pragma unroll
                        for (int i1 = 0; i1 < 2; i1++) {
                            const int i = i2 + i1;
                            wait_load(x[i1]);
                            load32(x[1 - i1], s_at + 32 * ((i + 1) & 3));          // (after the last, the first once more: for the weights)
                            const uint32_t bits = MASKED ? seen(i) : 0;
#pragma unroll
                            for (int h = 0; h < 2; h++) {
                                const float2 f = *reinterpret_cast<const float2*>(f_at + 2 * i + h);
                                float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
                                for (int k = 0; k < 16; k++) {
                                    const float y = __uint_as_float(x[i1][16 * h + k]);
                                    most[k & 1] = fmaxf(most[k & 1], !MASKED || (bits >> (16 * h + k) & 1) ? y : -INFINITY);
                                }
                                most[0] = fmaxf(most[0], most[1]);
                                if (!MASKED || most[0] > -INFINITY) top = fmaxf(top, fmaf(most[0], factor * f.x, f.y));
                            }
                        }
                        if (__any_sync(0xFFFFFFFFu, top > limit_of(m))) {
                            const float next = top > limit_of(m) ? top - BIAS : m, half = ex2(0.5f * (m - next)), down = half * half;
                            m = next;
                            l = l * half * half;               // (scaled(): down may be 0)
                            if (j > j_begin) { // what O holds; the products before this S are complete
#pragma unroll 1
                                for (int i = 0; i < DT / 16; i++) {
                                    uint32_t o[16];
                                    load16(o, o_at + 16 * i);
                                    wait_load(o);
#pragma unroll
                                    for (int k = 0; k < 16; k++) o[k] = __float_as_uint(__uint_as_float(o[k]) * down);
                                    store16(o_at + 16 * i, o);
                                }
                            }
                        }
#pragma unroll 1
                        for (int i2 = 0; i2 < 4; i2 += 2)
#pragma unroll
                        for (int i1 = 0; i1 < 2; i1++) {
                            const int i = i2 + i1;
                            wait_load(x[i1]);
                            if (i < 3) load32(x[1 - i1], s_at + 32 * (i + 1));
                            const uint32_t bits = MASKED ? seen(i) : 0;
                            uint32_t p[16];
#pragma unroll
                            for (int h = 0; h < 2; h++) {
                                const float4 f = f_at[2 * i + h];
                                const uint64_t fk = pair(factor * f.x, factor * f.x);
                                // once; twice where the keys enter the sum by exponentials of their own
#pragma unroll 1
                                for (int turn = FAR_APART && f.z == 0.f ? 0 : 1; turn < 2; turn++) {
                                    // (not masked: product and maximum in one rounding.  Masked: rounded like the maximum's own, first)
                                    const float shift = MASKED ? f.y : f.y - m, last = turn ? 0.f : -f.y;
                                    const uint64_t lm = pair(shift, shift);
                                    uint64_t sum[2] = {0, 0};
#pragma unroll
                                    for (int k = 0; k < 16; k += 2) {
                                        float y0, y1;
                                        uint64_t y = fma2(pair(__uint_as_float(x[i1][16 * h + k]), __uint_as_float(x[i1][16 * h + k + 1])), fk, lm);
                                        if (MASKED) y = add2(y, pair(-m, -m));
                                        if (FAR_APART) y = add2(y, pair(last, last));
                                        unpair(y, y0, y1);
                                        if (MASKED) {
                                            y0 = bits >> (16 * h + k) & 1 ? y0 : -INFINITY;
                                            y1 = bits >> (16 * h + k + 1) & 1 ? y1 : -INFINITY;
                                        }
                                        y0 = ex2(y0);
                                        y1 = ex2(y1);
                                        sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], pair(y0, y1));
                                        p[8 * h + k / 2] = FAR_APART && f.w == 0.f ? 0u : pack(y0, y1);
                                    }
                                    float y0, y1;
                                    unpair(add2(sum[0], sum[1]), y0, y1);
                                    l = fmaf(y0 + y1, turn ? f.z : 1.f, l);
                                }
                            }
                            // weights of 32 keys over 16 columns of S that have been read: the next 32 are on their way
                            store16(s_at + 16 * i, p);
                        }
                    };
                    const float largest = c.largest[s][tile % FACTORS];
                    if (full && largest * most_factor < 0x1p-6f) weights(std::false_type(), std::false_type());
                    else if (largest < INFINITY) weights(std::true_type(), std::false_type());
                    else weights(std::true_type(), std::true_type());
                    wait_store();
                }
                fence_before();
                bar_arrive(&c.p_full[s]);
                bar_arrive(&c.f_empty[s][tile % FACTORS]);
            }
            // ---- the output
            asm volatile("" ::: "memory");    // (what follows is read and worked out again)
            const Item mi = now.item;
            const int own = mi.split ? r : 128 * s + r;
            const Place own_at = place_of(a, mi.t0, mi.h0, min(own, mi.nrows - 1));
            const int head = mi.kvh * a.group + own_at.head;
            const bool is = own < mi.nrows, any = (own & ~31) < mi.nrows;
            const int64_t out_row = mi.first + own_at.query;
            T* const out = (T*)a.out + out_row * a.ldo + (int64_t)head * a.hso;
            if (ok) ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.o_full, o_phase, stop));
            o_phase ^= 1;
            fence_after();
            const bool whole = now.from == 0 && now.count == mi.tiles;
            const int slot = first_item ? 0 : 1;
            float* part = a.parts + ((int64_t)blockIdx.x * 2 + slot) * slot_floats<DT, MANY_ROWS>();
            if (!whole && now.from == 0 && tid == 0)
                a.records[blockIdx.x] = Record{mi.first, mi.kvh, mi.r0, mi.nrows, (int)(1 + (mi.tiles - now.count + c.share - 1) / c.share), slot, 0};
            first_item = false;
            const bool empty = now.count <= s;                    // the second stream of a single tile
            float* const other = reinterpret_cast<float*>(base + L::Q);    // the second stream's O, by column; its m and l behind the control block
            float* const other_m = reinterpret_cast<float*>(base + L::END + sizeof(Control));
            if (mi.split && s == 1) {
                if (ok) {
#pragma unroll 1
                    for (int i = 0; i < DT / 32; i++) {
                        uint32_t o[32];
                        if (any && !empty) load32(o, o_at + 32 * i);
                        wait_load(o);
#pragma unroll
                        for (int k = 0; k < 32; k++) other[(32 * i + k) * 128 + r] = is && !empty ? __uint_as_float(o[k]) : 0.f;
                    }
                }
                other_m[r] = m;
                other_m[128 + r] = ok ? l : NAN;
                bar_arrive(&c.hand[0]);
                ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.hand[1], h_phase, stop)) && ok;          // (its rows of q may be overwritten)
                h_phase ^= 1;
                continue;
            }
            float weight = 1.f, other_weight = 0.f;
            if (mi.split) {
                ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.hand[0], h_phase, stop)) && ok;
                if (ok) {
                    const float om = other_m[r], next = fmaxf(m, om);
                    weight = ex2(m - next);
                    other_weight = ex2(om - next);
                    l = scaled(l, m - next) + scaled(other_m[128 + r], om - next);
                    m = next;
                }
            }
            const float inverse = !ok ? NAN : !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
            if (any) {
                // By way of the warp's own rows of q (2 DT bytes each: DT entries of the output, or DT / 2 floats of a partial result, at a
                // time), so that rows are written in whole lines.  Where the streams share rows, shared memory holds the other's
                // results and the rows are few: a thread writes its own.
                constexpr int UNITS = DT / 8;                          // of 16 bytes
                const int turn = whole ? DT : DT / 2;
                auto unit_at = [&](int row_at, int u) {
                    return reinterpret_cast<uint4*>(base + L::Q + s * L::OPERAND + (u >> 3) * HALF_TILE + row_at * 128 + ((u ^ row_at) & 7) * 16);
                };
#pragma unroll 1
                for (int i = 0; i < DT / 32; i++) {
                    uint32_t o[32];
                    load32(o, o_at + 32 * i);
                    wait_load(o);
                    float y[32];
#pragma unroll
                    for (int k = 0; k < 32; k++) {
                        y[k] = __uint_as_float(o[k]) * weight;
                        if (mi.split) y[k] = fmaf(other[(32 * i + k) * 128 + r], other_weight, y[k]);
                        y[k] *= inverse;
                    }
                    if (mi.split) {
                        if (is && !whole) {
#pragma unroll
                            for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(part + (int64_t)own * DT + 32 * i + k) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
                        } else if (is) {
                            const bool wide = ((uintptr_t)out & 15) == 0;
#pragma unroll
                            for (int k = 0; k < 32; k += 8) {
                                if (32 * i + k >= a.dim) break;
                                alignas(16) T t[8];
#pragma unroll
                                for (int z = 0; z < 8; z++) t[z] = to<T>(y[k + z]);
                                if (wide) *reinterpret_cast<uint4*>(out + 32 * i + k) = *reinterpret_cast<const uint4*>(t);
                                else {
#pragma unroll
                                    for (int z = 0; z < 8; z++) out[32 * i + k + z] = t[z];
                                }
                            }
                        }
                        __syncwarp();
                        continue;
                    }
                    const int in = 32 * i % turn;
                    if (whole) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            alignas(16) T t[8];
#pragma unroll
                            for (int z = 0; z < 8; z++) t[z] = to<T>(y[k + z]);
                            *unit_at(r, (in + k) / 8) = *reinterpret_cast<const uint4*>(t);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *unit_at(r, (in + k) / 4) = make_uint4(__float_as_uint(y[k]), __float_as_uint(y[k + 1]), __float_as_uint(y[k + 2]), __float_as_uint(y[k + 3]));
                    }
                    if (in + 32 < turn) continue;
                    __syncwarp();
                    const int u = lane % UNITS, w0 = own & ~31;
#pragma unroll 4
                    for (int z = lane / UNITS; z < 32; z += 32 / UNITS) {
                        T* const to_row = reinterpret_cast<T*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)out, z)) + u * 8;
                        const uint4 v = *unit_at((r & ~31) + z, u);
                        if (w0 + z >= mi.nrows) continue;
                        if (!whole) {
                            *reinterpret_cast<uint4*>(part + (int64_t)(w0 + z) * DT + (32 * i - in) + u * 4) = v;
                        } else if (u * 8 < a.dim) {
                            if (((uintptr_t)to_row & 15) == 0) *reinterpret_cast<uint4*>(to_row) = v;
                            else {
                                const T* t = reinterpret_cast<const T*>(&v);
#pragma unroll
                                for (int k = 0; k < 8; k++) to_row[k] = t[k];
                            }
                        }
                    }
                    __syncwarp();
                }
                if (is) {
                    if (!ok) l = NAN;
                    if (!whole) { part[MANY_ROWS * DT + own] = m; part[MANY_ROWS * DT + MANY_ROWS + own] = l; }
                    else if (a.lse) a.lse[out_row * a.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
                }
            }
            fence_before();                   // (O and S are read: the next item's products may overwrite them)
            if (mi.split) {                   // (the other rows' results are read: the next rows of q may be written over them)
                bar_arrive(&c.hand[1]);
                ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.hand[1], h_phase, stop)) && ok;
                h_phase ^= 1;
            }
        }
        if (!ok) {                             // a wait ran out: the rows that were still to come
            Cursor here = now.cursor;
            Item item;
            int i0, n;
            while (here.next(a, item, i0, n)) {
                const bool whole = i0 == 0 && n == item.tiles;
                const int slot = first_item ? 0 : 1, own = item.split ? r : 128 * s + r;
                if (!whole && i0 == 0 && tid == 0)
                    a.records[blockIdx.x] = Record{item.first, item.kvh, item.r0, item.nrows, (int)(1 + (item.tiles - n + c.share - 1) / c.share), slot, 0};
                first_item = false;
                if (own >= item.nrows || (item.split && s == 1)) continue;
                if (whole) {
                    const Place at = place_of(a, item.t0, item.h0, own);
                    const int head = item.kvh * a.group + at.head;
                    const int64_t row = item.first + at.query;
                    for (int d = 0; d < a.dim; d++) ((T*)a.out)[row * a.ldo + (int64_t)head * a.hso + d] = to<T>(NAN);
                    if (a.lse) a.lse[row * a.heads + head] = NAN;
                } else {                      // (a sum that is NaN makes the row's outputs NaN)
                    float* const part = a.parts + ((int64_t)blockIdx.x * 2 + slot) * slot_floats<DT, MANY_ROWS>();
                    part[MANY_ROWS * DT + own] = 0.f;
                    part[MANY_ROWS * DT + MANY_ROWS + own] = NAN;
                }
            }
        }
    } else if (warp < 12) {
        // ---- converters: 16-byte pieces of a key's 64 dims in four neighbouring lanes, eight keys per warp
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        const int cw = warp - 8, piece = lane & 3, sub = lane >> 2;
        const int64_t head_entries = (int64_t)a.dim << a.page_log;
        uint32_t unit = 0;                    // tiles converted
        bool ok = true;
        while (ok && cursor.next(a, it, from, count)) {
            const int32_t* table = a.table + (int64_t)cursor.b * a.ld_table;
            // the order in which the products want their tiles: K0 V0 K1 V1 ..., or K0 K1 V0 K2 V1 ... where the streams share them
            auto what = [&](int i, bool& values) {
                if (!it.split) { values = i & 1; return i >> 1; }
                if (i == 0) { values = false; return 0; }
                if (i & 1) { const int k = (i + 1) >> 1; values = k >= count; return values ? count - 1 : k; }
                values = true;
                return (i - 2) >> 1;
            };
            auto pages = [&](int i, int (&p)[2]) {
                bool values;
                const int key = tile_at(it, from + what(i, values)) * TILE + cw * 32;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    p[h] = -1;
                    if (i < 2 * count && key + 16 * h < it.length) p[h] = __ldg(table + ((key + 16 * h) >> a.page_log));
                    if (p[h] >= a.pages) p[h] = -1;
                }
            };
            uint4 v[4][L::HALVES];
            auto load = [&](int i, const int (&p)[2], int q) {
                bool values;
                const int key = tile_at(it, from + what(i, values)) * TILE + cw * 32 + q * 8;
                const int8_t* cache = values ? a.v_cache : a.k_cache;
                const int64_t stride = values ? a.v_page_stride : a.k_page_stride;
                const int slot = (key & ((1 << a.page_log) - 1)) + sub;
                const int8_t* src = cache + p[q >> 1] * stride + it.kvh * head_entries + (int64_t)slot * a.dim + piece * 16;
#pragma unroll
                for (int h = 0; h < L::HALVES; h++)
                    v[q][h] = p[q >> 1] >= 0 && h * 64 + piece * 16 < a.dim ? __ldg(reinterpret_cast<const uint4*>(src + h * 64)) : make_uint4(0, 0, 0, 0);
            };
            int now[2], later[2];
            pages(0, now);
#pragma unroll
            for (int q = 0; q < 4; q++) load(0, now, q);
            pages(1, now);
            for (int i = 0; i < 2 * count; i++) {
                pages(i + 2, later);
                const uint32_t stage = unit % STAGES;
                ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.empty[stage], (unit / STAGES & 1) ^ 1, stop));
                if (!ok) break;
                uint8_t* const at = base + L::RING + stage * L::OPERAND;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int r = cw * 32 + q * 8 + sub;
#pragma unroll
                    for (int h = 0; h < L::HALVES; h++) {
#pragma unroll
                        for (int z = 0; z < 2; z++) {
                            const uint32_t b0 = (&v[q][h].x)[2 * z] ^ 0x80808080u, b1 = (&v[q][h].x)[2 * z + 1] ^ 0x80808080u;
                            const uint4 w = make_uint4(halves(b0, 0x4140), halves(b0, 0x4342), halves(b1, 0x4140), halves(b1, 0x4342));
                            *reinterpret_cast<uint4*>(at + h * HALF_TILE + r * 128 + ((piece * 2 + z) ^ sub) * 16) = w;
                        }
                    }
                    if (i + 1 < 2 * count) load(i + 1, now, q);
                }
                fence_async();
                bar_arrive(&c.full[stage]);
                unit++;
                now[0] = later[0]; now[1] = later[1];
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (warp == 12) {
            // ---- the products: the warp goes through the waits together (addresses stay in its uniform registers), one lane issues
            uint32_t unit = 0, q_phase = 0, p_phase = 0, k_stage = 0, v_stage = 0;
            bool ok = true;
            int left = a.steps;               // products that a test leaves the block
            const uint32_t at = smem(base);
            const uint64_t q_op = operand(at + L::Q, 16, 1024), k_op = operand(at + L::RING, 16, 1024), v_op = operand(at + L::RING, HALF_TILE, 1024);
            auto wait = [&](uint64_t* b, uint32_t parity) { ok = __all_sync(0xFFFFFFFFu, ok && bar_wait(b, parity, stop)); };
            auto take = [&]() {               // the next converted tile
                const uint32_t stage = unit % STAGES;
                wait(&c.full[stage], unit / STAGES & 1);
                unit++;
                return stage;
            };
            while (ok && cursor.next(a, it, from, count)) {
                const int steps = it.split ? count : 2 * count;
                auto scores = [&](int u) {
                    const int s = u & 1;
                    if (it.split || s == 0) k_stage = take();
                    if (u < 2) wait(&c.q_full[s], q_phase);
                    if (!ok) return;
                    fence_after();
                    const uint64_t q = q_op + s * (L::OPERAND >> 4), k = k_op + k_stage * (L::OPERAND >> 4);
                    const uint32_t d = tmem + L::S + 128 * s;
                    if (elect()) {
#pragma unroll
                        for (int i = 0; i < DT / 16; i++) {
                            const uint32_t off = ((i >> 2) * HALF_TILE + (i & 3) * 32) >> 4;
                            mma_ss(d, q + off, k + off, shape(128, false), i > 0);
                        }
                        commit(&c.s_full[s]);
                        if (it.split || s == 1) commit(&c.empty[k_stage]);
                    }
                    __syncwarp();
                };
                scores(0);
                if (steps > 1) scores(1);
                else wait(&c.q_full[1], q_phase);                      // (no product of the second stream)
                for (int u = 0; ok && u < steps; u++) {
                    const int s = u & 1;
                    if (left-- <= 0) { ok = false; break; }
                    if (it.split || s == 0) v_stage = take();
                    wait(&c.p_full[s], p_phase >> s & 1);
                    p_phase ^= 1u << s;
                    if (!ok) break;
                    fence_after();
                    const uint64_t v = v_op + v_stage * (L::OPERAND >> 4);
                    const uint32_t d = tmem + L::O + 128 * s, p = tmem + L::S + 128 * s;
                    if (elect()) {
#pragma unroll
                        for (int i = 0; i < TILE / 16; i++) mma_ts(d, p + 8 * i, v + i * (2048 >> 4), shape(DT, true), u > 1 || i > 0);
                        if (it.split || s == 1) commit(&c.empty[v_stage]);
                        if (u + 1 == steps) commit(&c.o_full);
                    }
                    __syncwarp();
                    if (u + 2 < steps) scores(u + 2);
                }
                q_phase ^= 1;
            }
            if (elect()) commit(&c.last);     // whatever was issued is complete before tensor memory is given back
            __syncwarp();
            const long long begin = clock64();
            while (!bar_try(&c.last, 0) && clock64() - begin < MANY_PATIENCE) {}
        }
        if (warp == 13 || warp == 14) {
            // ---- a stream's factors: a lane per group of 16 keys; pages two tiles ahead, scales one
            const int s = warp - 13;
            uint32_t tile = 0;
            bool ok = true;
            while (ok && cursor.next(a, it, from, count)) {
                const int32_t* table = a.table + (int64_t)cursor.b * a.ld_table;
                const int step = it.split ? 2 : 1, j_begin = from + (it.split ? s : 0), j_end = from + count;
                auto page_of = [&](int j) {
                    const int key = tile_at(it, min(j, j_end - 1)) * TILE + lane * 16;
                    return lane < 8 && j < j_end && key < it.length ? __ldg(table + (key >> a.page_log)) : -1;
                };
                float ks = NAN, vs = NAN, widest = -INFINITY;          // widest: log2 of the largest value scale so far
                auto scales_of = [&](int page) {
                    ks = vs = NAN;
                    if (page >= 0 && page < a.pages) {
                        ks = __ldg(a.k_scale + (int64_t)page * a.kv_heads + it.kvh);
                        vs = __ldg(a.v_scale + (int64_t)page * a.kv_heads + it.kvh);
                    }
                };
                scales_of(page_of(j_begin));
                int page = page_of(j_begin + step);
                for (int j = j_begin; j < j_end; j += step, tile++) {
                    const bool good = ks >= 0.f && ks < INFINITY && vs >= 0.f && vs < INFINITY;
                    const float v = fmaxf(vs, 0x1p-100f);
                    float4 f = make_float4(good ? ks : NAN, good ? log2f(v) : 0.f, good ? 1.f / v : 1.f, good && vs < 0x1p-100f ? 0.f : 1.f);
                    float most = lane < 8 ? f.y : -INFINITY;
#pragma unroll
                    for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
                    widest = fmaxf(widest, most);
                    if (good && widest - f.y > FAR) f.z = 0.f;
                    const bool behind = tile_at(it, j) * TILE + lane * 16 >= it.length;            // (keys that no row sees)
                    float largest = behind ? 0.f : good && f.z != 0.f && f.w != 0.f ? ks : INFINITY;
#pragma unroll
                    for (int o = 1; o < 8; o <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, o));
                    scales_of(page);
                    page = page_of(j + 2 * step);
                    ok = __all_sync(0xFFFFFFFFu, bar_wait(&c.f_empty[s][tile % FACTORS], (tile / FACTORS & 1) ^ 1, stop));
                    if (!ok) break;
                    if (lane < 8) c.factors[s][tile % FACTORS][lane] = f;
                    if (lane == 0) c.largest[s][tile % FACTORS] = largest;
                    __syncwarp();
                    if (lane == 0) bar_arrive(&c.f_full[s][tile % FACTORS]);
                }
            }
        }
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 12) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <typename T, int DT>
cudaError_t run(const Args& a, cudaStream_t st)
{
    constexpr int bytes = Layout<DT>::END + sizeof(Control) + 2 * 128 * sizeof(float) + 1024;
    static_assert(bytes <= 227 * 1024, "shared memory of an SM");
    auto kernel = many_kernel<T, DT>;
    // once per device: permission for the shared memory
    static std::atomic<int> allowed[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(1, std::memory_order_relaxed);
    }
    const int grid = imm::sm_count();
    kernel<<<grid, NT, bytes, st>>>(a);
    e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_join<T, DT, MANY_ROWS>(a, grid, st);
}

}  // namespace

template <typename T> cudaError_t launch_many(const Args& a, cudaStream_t st)
{
    return a.dim > 64 ? run<T, 128>(a, st) : run<T, 64>(a, st);
}
template cudaError_t launch_many<__half>(const Args&, cudaStream_t);
template cudaError_t launch_many<__nv_bfloat16>(const Args&, cudaStream_t);

}  // namespace imm_attn
