// The 4-bit product for many rows, on the tensor cores.
//
// A CTA computes 128 outputs x 64, 128 or 256 rows: the weights are the M operand, unpacked by warps from
// shared memory into tensor memory (integers q - z, exact in bf16 and f16), the rows of x are the
// N operand in shared memory.  The accumulator of one group of inputs is complete after group / 16
// instructions; it is then read back, scaled in fp32 and added to the running sums in registers,
// while the next one (the other half of the rows, or the next group) accumulates in another buffer.
// Weights are therefore never rounded, and a thread needs one scale per group, because its
// accumulator lane is one output.
//
// With too few tiles for the SMs the CTAs of a cluster split K (SPLIT: one tile per cluster, the sums
// meet through distributed shared memory in the order of the slices).
//
// Bound by the tensor cores with groups of 128 (8192 x 8192 x 4096 in 432 us, 1.27 PFLOP/s),
// by scaling with groups of 64 and 32 (622 to 640 and 1115 us; of 4096 x 4096 x 4096 the tensor pipe is busy for 59, 39 and 22 % of the
// cycles with groups of 128, 64 and 32).  The forms with two halves spill 20 bytes of registers.
//
// Roles: warps 0-3 unpack, warps 4-11 scale and store, one thread of warp 12 loads (TMA for x, bulk
// copies for the weight tile and its scales and zero points), one thread of warp 13 issues the
// products.  Every wait on an mbarrier is bounded by the clock: one that gives up latches BLS_ST_ETIMEOUT, all
// roles wind down and tensor memory is released.  A wait gives up lane by lane, but the instructions on tensor
// memory and the barriers want whole warps: the lanes finish what they do, with whatever lies in the
// buffers, and a vote in every step lets the warp go on or leave as a whole (2 % of the time of 16 000 rows over 32 matrices).
// The cluster barriers of the split form have no limit of their own: every role of every CTA arrives at both, at
// the end of its loop or after a wait that gave up.
#include "bls_tc.cuh"
#include "bls_w4.cuh"
#include "bls_w4_gemm.h"

namespace {

constexpr int GM_SLOTS = 2;                                   // tensor-memory slots of unpacked weights
constexpr int GM_THREADS = 16 * 32;                           // warps 14 and 15 only fill the fourth warpgroup
constexpr unsigned GM_TMEM_COLS = 512, GM_A_COL = GM_TMEM_COLS - GM_SLOTS * 64;       // accumulators, then the weights' slots of 64 columns
constexpr int GM_MAX_E = 1024;

struct GmRest {
    unsigned long long bars[2 * 8 + 2 * GM_SLOTS + 2 * 6];        // at most 8 stages and 6 accumulators
    int tile_end[GM_MAX_E];                                       // row tiles of the matrices up to and including this one
    int scan[16];
    unsigned tmem_slot;
};

// A tile has HALVES times COLS rows of x, COLS being the rows per product instruction (its N).  With one half of
// 128 rows there are three accumulators, with one of 64 there are six: few rows make short products,
// and more of them have to be under way.  A stage of 128 inputs: x, the weight tile, the scales and the zero points of its groups.
template <int GROUP, int COLS, int HALVES> struct GmStage {
    static constexpr int COUNT = HALVES == 2 ? 3 : COLS == 128 ? 5 : 8;                                     // what fits into 227 KB
    static constexpr int BUFFERS = GM_A_COL / COLS;
    static constexpr unsigned HALF = COLS * W4_TILE * 2, W = HALVES * HALF, BYTES = W + W4_TILE_BYTES;      // x (two boxes of 64 inputs), weights
    // after all stages: scales and zero points, 64-byte rows of results for each of the eight storing warps, and the rest
    static constexpr int GPT = W4_TILE / GROUP, STORE_ROWS = HALVES == 2 && GROUP == 32 ? 4 : 8;
    static constexpr unsigned SCALE = COUNT * BYTES, ZERO = GPT * W4_TILE * 2, SIDE = GPT * W4_TILE * 3,
                              STORE = SCALE + COUNT * SIDE, REST = STORE + 8 * STORE_ROWS * 64, ALL = REST + sizeof(GmRest);
    static_assert(ALL <= 232448, "shared memory of a CTA");
};

struct GmTile { int e, row0, rows, nt; };                     // matrix, first row, rows of x in the tile, output tile

// A in tensor memory, B in shared memory.
__device__ __forceinline__ void umma_f16_ta(unsigned d_tmem, unsigned a_tmem, unsigned long long db, unsigned idesc, unsigned acc)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(db), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_st16(unsigned taddr, const unsigned (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
// 16 columns of this warp's lanes; the registers hold them after tmem_wait_ld().
__device__ __forceinline__ void tmem_ld16(unsigned taddr, unsigned (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
// The registers pass through, so that nothing that uses them is moved before the wait.
__device__ __forceinline__ void tmem_wait_ld(unsigned (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
__device__ __forceinline__ bool elect_one()
{
    unsigned p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// Registers move to the warps that hold the running sums: 512 threads start with 128 each (512 per four
// threads, one of each warpgroup); 64 + 2 x 208 + 32 = 512.
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// a * s + c on two fp32 values at once
__device__ __forceinline__ unsigned long long fma2(unsigned long long s, unsigned a0, unsigned a1, unsigned long long c)
{
    unsigned long long r;
    asm("{\n\t.reg .b64 a;\n\tmov.b64 a, {%2, %3};\n\tfma.rn.f32x2 %0, %1, a, %4;\n\t}" : "=l"(r) : "l"(s), "r"(a0), "r"(a1), "l"(c));
    return r;
}
template <class T> __device__ __forceinline__ unsigned gm_idesc(int n)
{
    constexpr unsigned f = W4Pairs<T>::MAGIC == 0x43004300u ? 1u : 0u;                        // 1 bf16, 0 f16
    return (1u << 4) | (f << 7) | (f << 10) | ((unsigned)(n >> 3) << 17) | ((unsigned)(128 >> 4) << 24);
}

// 32 results of one output, one per row of x, from `at` on.
template <class Y>
__device__ __forceinline__ void gm_store(Y *at, long long ldy, int rows, const float (&v)[32])
{
    #pragma unroll
    for (int c = 0; c < 32; c++) {
        if (c < rows) *at = from_float<Y>(v[c]);
        at += ldy;
    }
}

// The same in 16 bits for the 32 outputs of a warp, from y's `at` on for output 0: ROWS rows of 64 bytes at a time go
// through the warp's shared memory, so that a thread stores 16 bytes.  `outs`: outputs that exist (a multiple of 8).
template <class Y, int ROWS>
__device__ __forceinline__ void gm_store_rows(Y *at, long long ldy, int rows, int outs, unsigned char *stage, int lane, const float (&v)[32])
{
    const int r = lane >> 2, piece = lane & 3;
    #pragma unroll
    for (int c0 = 0; c0 < 32; c0 += ROWS) {
        #pragma unroll
        for (int c = 0; c < ROWS; c++) *(Y *)(stage + c * 64 + lane * 2) = from_float<Y>(v[c0 + c]);
        __syncwarp();
        if (r < ROWS && c0 + r < rows && piece * 8 < outs) *(uint4 *)(at + (c0 + r) * ldy + piece * 8) = *(const uint4 *)(stage + lane * 16);
        __syncwarp();
    }
}

// The .aligned barrier wants whole warps, and callers come out of code that goes lane by lane.
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// grid: persistent, one CTA per SM at most; tiles are numbered over (matrix, row tile, output tile).
// SPLIT: one cluster of `slices` CTAs per tile, every CTA a slice of K.
template <class T, int GROUP, int COLS, int HALVES, bool SPLIT>
__global__ void __launch_bounds__(GM_THREADS, 1) bls_w4_tiles_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ W4Args a, int slices)
{
    using Stage = GmStage<GROUP, COLS, HALVES>;
    constexpr int STAGES = Stage::COUNT, BUFS = Stage::BUFFERS, GPT = W4_TILE / GROUP, ROWS = HALVES * COLS, CHUNKS = COLS / 64;
    constexpr unsigned HALF = Stage::HALF;
    extern __shared__ __align__(1024) unsigned char gm_smem[];    // the swizzle pattern repeats every 1024 bytes
    GmRest &rest = *(GmRest *)(gm_smem + Stage::REST);
    int *tile_end = rest.tile_end, *scan = rest.scan;
    unsigned &tmem_slot = rest.tmem_slot;
    const unsigned smem = s_addr(gm_smem);
    const unsigned full = s_addr(rest.bars), empty = full + 8 * STAGES, a_full = empty + 8 * STAGES, a_empty = a_full + 8 * GM_SLOTS,
                   d_full = a_empty + 8 * GM_SLOTS, d_empty = d_full + 8 * BUFS;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const W4Weights &w = a.w;
    // this CTA's first tile, the step to the next one, and its tiles of K
    const int KT = w.KT, rank = SPLIT ? blockIdx.x % slices : 0, first_tile = SPLIT ? blockIdx.x / slices : blockIdx.x,
              step = SPLIT ? gridDim.x / slices : gridDim.x, per = SPLIT ? (KT + slices - 1) / slices : KT,
              k0 = SPLIT ? min(rank * per, KT) : 0, k1 = SPLIT ? min(k0 + per, KT) : KT;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
        for (int s = 0; s < STAGES; s++) { mb_init(full + 8 * s, 1); mb_init(empty + 8 * s, 1 + 4 + 8); }
        for (int s = 0; s < GM_SLOTS; s++) { mb_init(a_full + 8 * s, 4); mb_init(a_empty + 8 * s, 1); }
        for (int s = 0; s < BUFS; s++) { mb_init(d_full + 8 * s, 1); mb_init(d_empty + 8 * s, 8); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_addr(&tmem_slot)), "r"(GM_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    stream_order_enter();
    // row tiles of every matrix, summed up in chunks of one matrix per thread
    int carry = 0;
    for (int e0 = 0; e0 < w.E; e0 += GM_THREADS) {
        const int e = e0 + threadIdx.x;
        int c = 0;
        if (e < w.E) {
            int lo, hi;
            w4_rows(a, e, lo, hi);
            c = (hi - lo + ROWS - 1) / ROWS;
        }
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(~0u, c, d);
            if (lane >= d) c += o;
        }
        if (lane == 31) scan[warp] = c;
        __syncthreads();
        int before = carry;
        #pragma unroll
        for (int i = 0; i < 16; i++) {
            if (i < warp) before += scan[i];
            carry += scan[i];
        }
        if (e < w.E) tile_end[e] = before + c;
        __syncthreads();
    }
    if (a.offsets) {                                               // rows of no matrix become 0
        for (int row = min(max(a.offsets[w.E], 0), a.rows) + blockIdx.x; row < a.rows; row += gridDim.x)
            for (int n = threadIdx.x; n < w.N; n += GM_THREADS) w4_store(a.y, (size_t)row * a.ldy + n, a.y_dtype, 0.f);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const unsigned tmem = *(volatile unsigned *)&tmem_slot;
    const int tiles = carry * w.NT;

    auto tile_of = [&](int i) {
        const int m = i / w.NT;
        int lo = 0, hi = w.E - 1;                                  // the first matrix whose tiles end past m
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (tile_end[mid] > m) hi = mid; else lo = mid + 1;
        }
        GmTile t;
        t.e = lo;
        t.nt = i % w.NT;
        int r0, r1;
        w4_rows(a, lo, r0, r1);
        t.row0 = r0 + (m - (lo ? tile_end[lo - 1] : 0)) * ROWS;
        t.rows = min(ROWS, r1 - t.row0);
        return t;
    };

    if (warp >= 12) {
        regs_down<32>();
        if (warp == 12 && lane == 0) {
            unsigned s = 0, ph = 0, issued = 0;
            bool ok = true;
            for (int i = first_tile; i < tiles && ok; i += step) {
                const GmTile t = tile_of(i);
                const uint8_t *q = w.q + (((size_t)t.e * w.NT + t.nt) * KT + k0) * W4_TILE_BYTES;
                size_t g = ((size_t)t.e * KT + k0) * GPT * w.NT * W4_TILE + t.nt * W4_TILE;
                const bool two = HALVES == 2 && t.rows > COLS;
                const unsigned bytes = W4_TILE_BYTES + (two ? 2 : 1) * HALF + GPT * W4_TILE * (w.zero ? 3 : 2);
                for (int kt = k0; kt < k1; kt++) {
                    ok = mb_wait(empty + 8 * s, ph ^ 1, a.status);
                    if (!ok) break;
                    const unsigned dst = smem + s * Stage::BYTES, side = smem + Stage::SCALE + s * Stage::SIDE, bar = full + 8 * s;
                    mb_expect_tx(bar, bytes);
                    bulk_load(dst + Stage::W, q, W4_TILE_BYTES, bar);
                    q += W4_TILE_BYTES;
                    tma_load_2d(dst, &map_x, bar, kt * W4_TILE, t.row0);
                    tma_load_2d(dst + HALF / 2, &map_x, bar, kt * W4_TILE + 64, t.row0);
                    if (two) {
                        tma_load_2d(dst + HALF, &map_x, bar, kt * W4_TILE, t.row0 + COLS);
                        tma_load_2d(dst + HALF + HALF / 2, &map_x, bar, kt * W4_TILE + 64, t.row0 + COLS);
                    }
                    #pragma unroll
                    for (int gi = 0; gi < GPT; gi++) {
                        bulk_load(side + gi * W4_TILE * 2, w.scale + g, W4_TILE * 2, bar);
                        if (w.zero) bulk_load(side + Stage::ZERO + gi * W4_TILE, w.zero + g, W4_TILE, bar);
                        g += (size_t)w.NT * W4_TILE;
                    }
                    issued++;
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                }
            }
            // the copies still in flight write to this CTA's shared memory: see them land before leaving
            for (unsigned b = issued > STAGES ? issued - STAGES : 0; b < issued; b++) mb_wait(full + 8 * (b % STAGES), (b / STAGES) & 1, a.status);
        } else if (warp == 13) {
            // the whole warp follows, one thread of it issues
            const bool leader = elect_one();
            unsigned s = 0, ph = 0, j = 0, jph = 0, used = 0, b = 0;                  // used: how often all accumulators have been filled
            bool ok = true;
            for (int i = first_tile; i < tiles && ok; i += step) {
                const GmTile t = tile_of(i);
                for (int kt = k0; kt < k1 && ok; kt++) {
                    ok = mb_wait(full + 8 * s, ph, a.status) && mb_wait(a_full + 8 * j, jph, a.status);
                    const unsigned long long base = umma_desc(smem + s * Stage::BYTES);
                    const unsigned at = tmem + GM_A_COL + j * 64;
                    #pragma unroll
                    for (int gi = 0; gi < GPT; gi++) {
                        #pragma unroll
                        for (int h = 0; h < HALVES; h++) {
                            const int rows = min(COLS, t.rows - h * COLS);
                            if (rows <= 0) continue;
                            ok = ok && mb_wait(d_empty + 8 * b, (used & 1) ^ 1, a.status);
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            if (leader && ok) {
                                const unsigned idesc = gm_idesc<T>((rows + 15) & ~15);
                                #pragma unroll
                                for (int k = 0; k < GROUP / 16; k++) {
                                    const int ks = gi * (GROUP / 16) + k;     // step of 16 inputs: box ks / 4, 32 bytes each
                                    umma_f16_ta(tmem + b * COLS, at + ks * 8,
                                                base + (h * HALF + (ks >> 2) * (HALF / 2) + (ks & 3) * 32) / 16, idesc, k ? 1u : 0u);
                                }
                                umma_commit(d_full + 8 * b);
                            }
                            if (++b == BUFS) { b = 0; used++; }
                        }
                    }
                    if (leader && ok) {
                        umma_commit(a_empty + 8 * j);
                        umma_commit(empty + 8 * s);
                    }
                    ok = __all_sync(~0u, ok);
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                    if (++j == GM_SLOTS) { j = 0; jph ^= 1; }
                }
            }
        }
    } else if (warp < 4) {
        regs_down<64>();
        // unpack: thread = output row of the weight tile = lane of tensor memory
        const int r = warp * 32 + lane;
        const unsigned swz = (unsigned)((r >> 1) & 3);
        unsigned s = 0, ph = 0, j = 0, jph = 0;
        bool ok = true;
        for (int i = first_tile; i < tiles && ok; i += step) {
            for (int kt = k0; kt < k1; kt++) {
                ok = mb_wait(full + 8 * s, ph, a.status);
                const unsigned src = smem + s * Stage::BYTES + Stage::W + r * 64;
                unsigned word[4][4];                                      // [quarter][block of 32 inputs]
                #pragma unroll
                for (int p = 0; p < 4; p++)
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(word[p][0]), "=r"(word[p][1]), "=r"(word[p][2]), "=r"(word[p][3]) : "r"(src + ((p ^ swz) * 16)));
                unsigned zp[GPT];
                #pragma unroll
                for (int gi = 0; gi < GPT; gi++) {
                    unsigned z = 8;
                    if (w.zero) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(z) : "r"(smem + Stage::SCALE + s * Stage::SIDE + Stage::ZERO + gi * W4_TILE + r));
                    zp[gi] = w4_zero_pair<T>(z & 15);
                }
                ok = ok && mb_wait(a_empty + 8 * j, jph ^ 1, a.status);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const unsigned dst = tmem + ((unsigned)(warp * 32) << 16) + GM_A_COL + j * 64;
                #pragma unroll
                for (int b = 0; b < 4; b++) {
                    unsigned o[16];
                    #pragma unroll
                    for (int p = 0; p < 4; p++) {
                        unsigned v[4];
                        w4_unpack<T>(word[p][b], zp[b * 32 / GROUP], v);
                        #pragma unroll
                        for (int c = 0; c < 4; c++) o[p * 4 + c] = v[c];
                    }
                    tmem_st16(dst + b * 16, o);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                ok = __all_sync(~0u, ok);
                if (lane == 0) {
                    mb_arrive(a_full + 8 * j);
                    mb_arrive(empty + 8 * s);
                }
                if (!ok) break;
                if (++s == STAGES) { s = 0; ph ^= 1; }
                if (++j == GM_SLOTS) { j = 0; jph ^= 1; }
            }
        }
    } else {
        regs_up<208>();
        // scale and store: thread = output, half of the rows of x of every half of the tile
        const int q4 = warp & 3, part = (warp - 4) >> 2, r = q4 * 32 + lane;
        const unsigned lanes = (unsigned)(q4 * 32) << 16;
        unsigned s = 0, ph = 0, used = 0, b = 0;
        bool ok = true;
        for (int i = first_tile; i < tiles && ok; i += step) {
            const GmTile t = tile_of(i);
            unsigned long long tot[HALVES][CHUNKS][16];                         // two rows each
            #pragma unroll
            for (int h = 0; h < HALVES; h++)
                #pragma unroll
                for (int c = 0; c < CHUNKS * 16; c++) tot[h][c >> 4][c & 15] = 0ull;
            for (int kt = k0; kt < k1; kt++) {
                ok = ok && mb_wait(full + 8 * s, ph, a.status);            // the scales have arrived
                unsigned sc[GPT];
                #pragma unroll
                for (int gi = 0; gi < GPT; gi++)
                    asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tmov.b32 %0, {0, h};\n\t}" : "=r"(sc[gi])
                                 : "r"(smem + Stage::SCALE + s * Stage::SIDE + gi * W4_TILE * 2 + r * 2));      // bf16 -> fp32
                ok = __all_sync(~0u, ok);
                if (!ok) break;
                if (lane == 0) mb_arrive(empty + 8 * s);
                #pragma unroll
                for (int gi = 0; gi < GPT; gi++) {
                    const unsigned long long s2 = (unsigned long long)sc[gi] << 32 | sc[gi];
                    #pragma unroll
                    for (int h = 0; h < HALVES; h++) {
                        if (h * COLS >= t.rows) continue;
                        ok = ok && mb_wait(d_full + 8 * b, used & 1, a.status);
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const bool busy = h * COLS + part * (COLS / 2) < t.rows;     // the whole warp alike
                        const unsigned src = tmem + lanes + b * COLS + part * (COLS / 2);
                        // all of this thread's columns are read at once, so that the accumulator is free as early as possible
                        constexpr int PARTS = COLS / 32;
                        unsigned v[PARTS][16];
                        if (busy) {
                            #pragma unroll
                            for (int p = 0; p < PARTS; p++) tmem_ld16(src + p * 16, v[p]);
                            #pragma unroll
                            for (int p = 0; p < PARTS; p++) tmem_wait_ld(v[p]);
                        }
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mb_arrive(d_empty + 8 * b);
                        if (busy) {
                            #pragma unroll
                            for (int p = 0; p < PARTS; p++)
                                #pragma unroll
                                for (int c = 0; c < 8; c++)
                                    tot[h][p >> 1][(p & 1) * 8 + c] = fma2(s2, v[p][2 * c], v[p][2 * c + 1], tot[h][p >> 1][(p & 1) * 8 + c]);
                        }
                        if (++b == BUFS) { b = 0; used++; }
                    }
                }
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            ok = __all_sync(~0u, ok);
            const int n = t.nt * W4_TILE + r;
            if (SPLIT) {
                // the slice's sums, [row][output], over the stages: every copy has arrived and every product has been read
                #pragma unroll
                for (int c = 0; c < COLS / 2; c++)
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem + ((part * (COLS / 2) + c) * W4_TILE + r) * 4),
                                 "r"((unsigned)(tot[0][c >> 5][c >> 1 & 15] >> (32 * (c & 1)))) : "memory");
                continue;
            }
            if (!ok) continue;
            const float bias = a.bias && n < w.N ? a.bias[(size_t)t.e * w.N + n] : 0.f;
            const int n0 = t.nt * W4_TILE + q4 * 32;                       // the warp's outputs
            unsigned char *stage = gm_smem + Stage::STORE + (warp - 4) * Stage::STORE_ROWS * 64;
            #pragma unroll
            for (int h = 0; h < HALVES; h++)
                #pragma unroll
                for (int p = 0; p < CHUNKS; p++) {
                    const int row = h * COLS + part * (COLS / 2) + p * 32;
                    if (row >= t.rows) continue;
                    const int left = t.rows - row;
                    const size_t at = (size_t)(t.row0 + row) * a.ldy + n0;
                    float v[32];
                    #pragma unroll
                    for (int c = 0; c < 32; c++) v[c] = __uint_as_float((unsigned)(tot[h][p][c >> 1] >> (32 * (c & 1)))) + bias;
                    if (a.act == 1) {
                        #pragma unroll
                        for (int c = 0; c < 32; c++) v[c] = w4_act(v[c], 1);
                    } else if (a.act == 2) {
                        #pragma unroll
                        for (int c = 0; c < 32; c++) v[c] = w4_act(v[c], 2);
                    }
                    if (a.y_pieces) {
                        if (a.y_dtype == BLS_BF16) gm_store_rows<__nv_bfloat16, Stage::STORE_ROWS>((__nv_bfloat16 *)a.y + at, a.ldy, left, w.N - n0, stage, lane, v);
                        else gm_store_rows<__half, Stage::STORE_ROWS>((__half *)a.y + at, a.ldy, left, w.N - n0, stage, lane, v);
                    } else if (n < w.N) {
                        if (a.y_dtype == BLS_F32) gm_store((float *)a.y + at + lane, a.ldy, left, v);
                        else if (a.y_dtype == BLS_BF16) gm_store((__nv_bfloat16 *)a.y + at + lane, a.ldy, left, v);
                        else gm_store((__half *)a.y + at + lane, a.ldy, left, v);
                    }
                }
        }
        if (SPLIT) {
            cluster_sync();
            if (first_tile < tiles) {
                // four outputs at a time: every CTA finishes its share of the 32 fours of a row
                const GmTile t = tile_of(first_tile);
                const int four0 = 32 * rank / slices, fours = 32 * (rank + 1) / slices - four0;
                for (int i = threadIdx.x - 128; i < t.rows * fours; i += 256) {
                    const int row = i / fours, o = (four0 + i % fours) * 4, n = t.nt * W4_TILE + o;
                    const unsigned at = smem + (row * W4_TILE + o) * 4;
                    float p[8][4], v[4] = {0.f, 0.f, 0.f, 0.f};
                    #pragma unroll
                    for (int sl = 0; sl < 8; sl++)
                        if (sl < slices)
                            asm volatile("{\n\t.reg .u32 t;\n\tmapa.shared::cluster.u32 t, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [t];\n\t}"
                                         : "=f"(p[sl][0]), "=f"(p[sl][1]), "=f"(p[sl][2]), "=f"(p[sl][3]) : "r"(at), "r"(sl) : "memory");
                    #pragma unroll
                    for (int sl = 0; sl < 8; sl++)
                        #pragma unroll
                        for (int c = 0; c < 4; c++)
                            if (sl < slices) v[c] += p[sl][c];
                    #pragma unroll
                    for (int c = 0; c < 4; c++)
                        if (n + c < w.N)
                            w4_store(a.y, (size_t)(t.row0 + row) * a.ldy + n + c, a.y_dtype,
                                     w4_act(v[c] + (a.bias ? a.bias[(size_t)t.e * w.N + n + c] : 0.f), a.act));
                }
            }
            cluster_sync();                                                // nobody reads this CTA's sums any more
        }
    }
    if (SPLIT && (warp < 4 || warp >= 12)) {
        cluster_sync();
        cluster_sync();
    }
    __syncwarp();                                                          // the loader and the lanes that waited for it
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 13) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(GM_TMEM_COLS) : "memory");
    }
}

// Rows of x copied to 16-byte boundaries, padded with zeros: [rows][ldo], ldo a multiple of 8.
__global__ void __launch_bounds__(256) bls_w4_align_kernel(const unsigned short *x, long long ldx, int K, int rows, unsigned short *o, int ldo)
{
    stream_order_enter();
    const int per = ldo / 8;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)rows * per; i += (long long)gridDim.x * blockDim.x) {
        const long long r = i / per;
        const int c = (int)(i % per) * 8;
        unsigned v[4] = {0, 0, 0, 0};
        #pragma unroll
        for (int j = 0; j < 8; j++)
            if (c + j < K) v[j >> 1] |= (unsigned)x[r * ldx + c + j] << (16 * (j & 1));
        *(uint4 *)(o + r * ldo + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

int sm_count()
{
    static int n = 0;                                              // of the first device used: all are alike
    if (!n) {
        int dev = 0, v = 0;
        if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) n = v;
    }
    return n > 0 ? n : 148;
}

template <class T, int GROUP, int COLS, int HALVES, bool SPLIT>
cudaError_t launch_tiles_h(const W4Args &a, int grid, int slices, cudaStream_t s)
{
    CUtensorMap map;
    if (!tc_make_map(&map, a.x, a.rows, a.w.K, a.ldx, COLS)) return cudaErrorInvalidValue;
    const size_t smem = GmStage<GROUP, COLS, HALVES>::ALL;
    auto kernel = bls_w4_tiles_kernel<T, GROUP, COLS, HALVES, SPLIT>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_serialised_cluster(kernel, dim3(grid), dim3(GM_THREADS), slices, smem, s, map, a, slices);
}

// One half of COLS rows per tile; K is split while that leaves an SM for every slice of two tiles or more.
template <class T, int GROUP, int COLS>
cudaError_t launch_tiles_c(const W4Args &a, long long tiles, cudaStream_t s)
{
    const int slices = (int)max(1ll, min(min(8ll, sm_count() / tiles), a.w.KT / 2ll));
    if (slices > 1) return launch_tiles_h<T, GROUP, COLS, 1, true>(a, (int)tiles * slices, slices, s);
    return launch_tiles_h<T, GROUP, COLS, 1, false>(a, (int)min(tiles, (long long)sm_count()), 1, s);
}

template <class T, int GROUP>
cudaError_t launch_tiles_g(const W4Args &a, cudaStream_t s)
{
    // upper bounds of the tiles: every matrix may end in a part of one
    const long long layers = min((long long)a.w.E, (long long)a.rows), ends = a.offsets ? layers : 0;
    const auto tiles = [&](int rows) { return ((a.rows + rows - 1ll) / rows + ends) * a.w.NT; };
    // tiles of 256 rows unpack every weight for twice as many products; they are taken where enough of them remain: 256 of
    // them take 61 us where 512 of 128 rows take 73 (2048 x 4096 x 4096), 192 take 36 and the smaller ones 33 (8 x 375 rows)
    if ((a.rows + 255ll) / 256 * a.w.NT * 2 >= 3ll * sm_count())
        return launch_tiles_h<T, GROUP, 128, 2, false>(a, (int)min(tiles(256), (long long)sm_count()), 1, s);
    // 64 rows on average: 32 x 64 rows take 25 us in tiles of 64 and 31 in tiles of 128, 32 x 125 rows 41 and 35
    if (a.rows <= 64 * layers) return launch_tiles_c<T, GROUP, 64>(a, tiles(64), s);
    return launch_tiles_c<T, GROUP, 128>(a, tiles(128), s);
}

template <class T>
cudaError_t launch_tiles(const W4Args &a, cudaStream_t s)
{
    return a.w.group == 32 ? launch_tiles_g<T, 32>(a, s) : a.w.group == 64 ? launch_tiles_g<T, 64>(a, s) : launch_tiles_g<T, 128>(a, s);
}

}  // namespace

size_t w4_tiles_bytes(const W4Weights &w, const void *x, long long ldx, long long rows)
{
    if (((uintptr_t)x & 15) == 0 && ldx % 8 == 0) return 0;
    return ((size_t)rows * ((w.K + 7) / 8 * 8) * 2 + 255) / 256 * 256;
}

cudaError_t w4_tiles(W4Args a, int x_dtype, void *workspace, cudaStream_t s)
{
    if (!a.x_pieces) {
        const int ldo = (a.w.K + 7) / 8 * 8;
        const long long items = (long long)a.rows * (ldo / 8);
        cudaError_t e = launch_serialised(bls_w4_align_kernel, dim3((unsigned)min((items + 255) / 256, 148ll * 16)), dim3(256), s,
                                          (const unsigned short *)a.x, a.ldx, a.w.K, a.rows, (unsigned short *)workspace, ldo);
        if (e != cudaSuccess) return e;
        a.x = workspace; a.ldx = ldo; a.x_pieces = 1;
    }
    return x_dtype == BLS_BF16 ? launch_tiles<__nv_bfloat16>(a, s) : launch_tiles<__half>(a, s);
}
