// The 4-bit product for many rows, on the tensor cores.
//
// A CTA computes 128 outputs x 128 rows: the weights are the M operand, unpacked by warps from
// shared memory into tensor memory (integers q - z, exact in bf16 and f16), the rows of x are the
// N operand in shared memory.  The accumulator of one group of inputs is complete after group / 16
// instructions; it is then read back, scaled in fp32 and added to the running sums in registers,
// while the next group accumulates in a second buffer.  Weights are therefore never rounded, and
// a thread needs one scale per group, because its accumulator lane is one output.
//
// Roles: warps 0-7 unpack (two sets of four take the stages in turn), warps 8-15 scale and
// store, one thread of warp 16 loads (TMA for x, one bulk copy per stored weight tile), one thread
// of warp 17 issues the products.  Every wait is bounded by the clock: one that gives up latches
// BLS_ST_ETIMEOUT, all roles wind down and tensor memory is released.
#include "bls_tc.cuh"
#include "bls_w4.cuh"
#include "bls_w4_gemm.h"

namespace {

constexpr int GM_ROWS = 128;                                  // rows of x per tile (N of the instruction)
constexpr int GM_STAGES = 5;                                  // shared-memory stages of 128 inputs
constexpr int GM_SLOTS = 4;                                   // tensor-memory slots of unpacked weights
constexpr unsigned GM_X_BYTES = GM_ROWS * W4_TILE * 2, GM_STAGE_BYTES = GM_X_BYTES + W4_TILE_BYTES;
constexpr int GM_THREADS = 20 * 32;                            // warps 18 and 19 only fill the fifth warpgroup
constexpr unsigned GM_TMEM_COLS = 512, GM_A_COL = 256;        // accumulators: columns 0..127 and 128..255; weights: 4 x 64 columns
constexpr int GM_MAX_E = 1024;

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
__device__ __forceinline__ void mb_arrive(unsigned bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(unsigned dst, const void *src, unsigned bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Registers move from the loading and unpacking warps to those that hold the running sums.  640 threads
// start with 96 each (480 per five threads, one of each warpgroup); 2 x 80 + 2 x 136 + 40 = 472.
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
    constexpr unsigned f = sizeof(T) == 2 && W4Pairs<T>::MAGIC == 0x43004300u ? 1u : 0u;      // 1 bf16, 0 f16
    return (1u << 4) | (f << 7) | (f << 10) | ((unsigned)(n >> 3) << 17) | ((unsigned)(128 >> 4) << 24);
}

// grid: persistent, one CTA per SM at most; tiles are numbered over (matrix, row tile, output tile).
template <class T>
__global__ void __launch_bounds__(GM_THREADS, 1) bls_w4_tiles_kernel(const __grid_constant__ CUtensorMap map_x, W4Args a)
{
    extern __shared__ unsigned char gm_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * GM_STAGES + 2 * GM_SLOTS + 4];
    __shared__ unsigned tmem_slot;
    __shared__ int tile_end[GM_MAX_E];                            // row tiles of the matrices up to and including this one
    __shared__ int scan[32];
    const unsigned smem = (s_addr(gm_smem) + 1023u) & ~1023u;
    const unsigned full = s_addr(&bars[0]), empty = full + 8 * GM_STAGES, a_full = empty + 8 * GM_STAGES, a_empty = a_full + 8 * GM_SLOTS,
                   d_full = a_empty + 8 * GM_SLOTS, d_empty = d_full + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const W4Weights &w = a.w;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
        for (int s = 0; s < GM_STAGES; s++) { mb_init(full + 8 * s, 1); mb_init(empty + 8 * s, 1 + 4); }
        for (int s = 0; s < GM_SLOTS; s++) { mb_init(a_full + 8 * s, 4); mb_init(a_empty + 8 * s, 1); }
        for (int s = 0; s < 2; s++) { mb_init(d_full + 8 * s, 1); mb_init(d_empty + 8 * s, 8); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_addr(&tmem_slot)), "r"(GM_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    stream_order_enter();
    // row tiles of every matrix, summed up: the first E threads count, a scan over chunks of 512 adds
    int carry = 0;
    for (int e0 = 0; e0 < w.E; e0 += 512) {
        const int e = e0 + threadIdx.x;
        int c = 0;
        if (threadIdx.x < 512 && e < w.E) {
            int lo, hi;
            w4_rows(a, e, lo, hi);
            c = (hi - lo + GM_ROWS - 1) / GM_ROWS;
        }
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(~0u, c, d);
            if (lane >= d) c += o;
        }
        if (lane == 31) scan[warp] = c;
        __syncthreads();
        int before = carry, all = carry;
        for (int i = 0; i < 16; i++) {
            if (i < warp) before += scan[i];
            all += scan[i];
        }
        if (threadIdx.x < 512 && e < w.E) tile_end[e] = before + c;
        carry = all;
        __syncthreads();
    }
    if (a.offsets) {                                               // rows of no matrix become 0
        const int first = min(max(a.offsets[w.E], 0), a.rows);
        for (long long i = (long long)blockIdx.x * GM_THREADS + threadIdx.x; i < (long long)(a.rows - first) * w.N; i += (long long)gridDim.x * GM_THREADS)
            w4_store(a.y, (size_t)(first + i / w.N) * a.ldy + i % w.N, a.y_dtype, 0.f);
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
        t.row0 = r0 + (m - (lo ? tile_end[lo - 1] : 0)) * GM_ROWS;
        t.rows = min(GM_ROWS, r1 - t.row0);
        return t;
    };
    const int gpt = W4_TILE / w.group;

    if (warp >= 16) regs_down<40>();
    if (warp == 16) {
        if (lane == 0) {
            unsigned it = 0;
            bool ok = true;
            for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
                const GmTile t = tile_of(i);
                const uint8_t *q = w.q + ((size_t)t.e * w.NT + t.nt) * w.KT * W4_TILE_BYTES;
                for (int kt = 0; kt < w.KT; kt++, it++) {
                    const unsigned s = it % GM_STAGES;
                    ok = mb_wait(empty + 8 * s, ((it / GM_STAGES) & 1) ^ 1, a.status);
                    if (!ok) break;
                    const unsigned dst = smem + s * GM_STAGE_BYTES, bar = full + 8 * s;
                    mb_expect_tx(bar, GM_STAGE_BYTES);
                    bulk_load(dst + GM_X_BYTES, q + (size_t)kt * W4_TILE_BYTES, W4_TILE_BYTES, bar);
                    tma_load_2d(dst, &map_x, bar, kt * W4_TILE, t.row0);
                    tma_load_2d(dst + GM_X_BYTES / 2, &map_x, bar, kt * W4_TILE + 64, t.row0);
                }
            }
            // the copies still in flight write to this CTA's shared memory: see them land before leaving
            for (unsigned b = it > GM_STAGES ? it - GM_STAGES : 0; b < it; b++) mb_wait(full + 8 * (b % GM_STAGES), (b / GM_STAGES) & 1, a.status);
        }
    } else if (warp == 17) {
        if (lane == 0) {
            unsigned it = 0, g = 0;
            bool ok = true;
            for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
                const GmTile t = tile_of(i);
                const unsigned idesc = gm_idesc<T>((t.rows + 15) & ~15);
                for (int kt = 0; kt < w.KT && ok; kt++, it++) {
                    const unsigned s = it % GM_STAGES, j = it % GM_SLOTS;
                    ok = mb_wait(full + 8 * s, (it / GM_STAGES) & 1, a.status) && mb_wait(a_full + 8 * j, (it / GM_SLOTS) & 1, a.status);
                    if (!ok) break;
                    for (int gi = 0; gi < gpt && ok; gi++, g++) {
                        ok = mb_wait(d_empty + 8 * (g & 1), ((g >> 1) & 1) ^ 1, a.status);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const int steps = w.group / 16;
                        for (int k = 0; k < steps; k++) {
                            const int ks = gi * steps + k;            // step of 16 inputs in the stage: half-tile ks / 4, 32 bytes each
                            umma_f16_ta(tmem + (g & 1) * 128, tmem + GM_A_COL + j * 64 + ks * 8,
                                        umma_desc(smem + s * GM_STAGE_BYTES + (ks >> 2) * (GM_X_BYTES / 2) + (ks & 3) * 32), idesc, k ? 1u : 0u);
                        }
                        umma_commit(d_full + 8 * (g & 1));
                    }
                    umma_commit(a_empty + 8 * j);
                    umma_commit(empty + 8 * s);
                }
            }
        }
    } else if (warp < 8) {
        regs_down<80>();
        // unpack: thread = output row of the weight tile = lane of tensor memory
        const int q4 = warp & 3, set = warp >> 2, r = q4 * 32 + lane;
        const unsigned swz = (unsigned)((r >> 1) & 3);
        unsigned it = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
            const GmTile t = tile_of(i);
            const size_t z0 = (size_t)t.e * w.KT * gpt * w.NT * W4_TILE + t.nt * W4_TILE + r;
            // the zero points of this set's next stage are on their way while a stage is unpacked
            unsigned zn[4] = {8, 8, 8, 8};
            auto fetch_zeros = [&](int kt) {
                #pragma unroll
                for (int b = 0; b < 4; b++)
                    if (w.zero && kt < w.KT) zn[b] = w.zero[z0 + (size_t)(kt * gpt + b * 32 / w.group) * w.NT * W4_TILE];
            };
            fetch_zeros((it & 1) == (unsigned)set ? 0 : 1);
            for (int kt = 0; kt < w.KT; kt++, it++) {
                if ((it & 1) != (unsigned)set) continue;
                unsigned zp[4];
                #pragma unroll
                for (int b = 0; b < 4; b++) zp[b] = w4_zero_pair<T>(zn[b] & 15);
                fetch_zeros(kt + 2);
                const unsigned s = it % GM_STAGES, j = it % GM_SLOTS;
                ok = mb_wait(full + 8 * s, (it / GM_STAGES) & 1, a.status) && mb_wait(a_empty + 8 * j, ((it / GM_SLOTS) & 1) ^ 1, a.status);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const unsigned src = smem + s * GM_STAGE_BYTES + GM_X_BYTES + r * 64;
                unsigned word[4][4];                                      // [quarter][block of 32 inputs]
                #pragma unroll
                for (int p = 0; p < 4; p++)
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(word[p][0]), "=r"(word[p][1]), "=r"(word[p][2]), "=r"(word[p][3]) : "r"(src + ((p ^ swz) * 16)));
                const unsigned dst = tmem + ((unsigned)(q4 * 32) << 16) + GM_A_COL + j * 64;
                #pragma unroll
                for (int b = 0; b < 4; b++) {
                    unsigned o[16];
                    #pragma unroll
                    for (int p = 0; p < 4; p++) {
                        unsigned v[4];
                        w4_unpack<T>(word[p][b], zp[b], v);
                        #pragma unroll
                        for (int c = 0; c < 4; c++) o[p * 4 + c] = v[c];
                    }
                    tmem_st16(dst + b * 16, o);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mb_arrive(a_full + 8 * j);
                    mb_arrive(empty + 8 * s);
                }
            }
        }
    } else if (warp < 16) {
        regs_up<136>();
        // scale and store: thread = output, 64 rows of x each
        const int q4 = warp & 3, half = (warp - 8) >> 2;
        unsigned g = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
            const GmTile t = tile_of(i);
            const int n = t.nt * W4_TILE + q4 * 32 + lane;
            const unsigned short *sc = (const unsigned short *)w.scale + (size_t)t.e * w.KT * gpt * w.NT * W4_TILE + n;
            const int groups = w.KT * gpt;
            const bool busy = half * 64 < t.rows;                          // the whole warp alike
            unsigned long long tot[32];                                    // two rows each
            #pragma unroll
            for (int c = 0; c < 32; c++) tot[c] = 0ull;
            // scales of the next four groups are on their way while four groups are added
            unsigned short nx[4];
            auto fetch_scales = [&](int gi) {
                #pragma unroll
                for (int b = 0; b < 4; b++)
                    nx[b] = gi + b < groups ? __ldg(sc + (size_t)(gi + b) * w.NT * W4_TILE) : (unsigned short)0;
            };
            fetch_scales(0);
            for (int g4 = 0; g4 < groups && ok; g4 += 4) {
                unsigned short cur[4];
                #pragma unroll
                for (int b = 0; b < 4; b++) cur[b] = nx[b];
                fetch_scales(g4 + 4);
                #pragma unroll
                for (int b = 0; b < 4; b++) {
                    if (g4 + b >= groups) break;
                    const unsigned si = (unsigned)cur[b] << 16;                   // bf16 -> fp32
                    const unsigned long long s2 = (unsigned long long)si << 32 | si;
                    ok = mb_wait(d_full + 8 * (g & 1), (g >> 1) & 1, a.status);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (busy) {
                        const unsigned src = tmem + ((unsigned)(q4 * 32) << 16) + (g & 1) * 128 + half * 64;
                        #pragma unroll
                        for (int h = 0; h < 2; h++) {
                            unsigned r[32];
                            tmem_ld32(src + h * 32, r);
                            if (h == 1) {
                                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                                __syncwarp();
                                if (lane == 0) mb_arrive(d_empty + 8 * (g & 1));
                            }
                            #pragma unroll
                            for (int c = 0; c < 16; c++) tot[h * 16 + c] = fma2(s2, r[2 * c], r[2 * c + 1], tot[h * 16 + c]);
                        }
                    } else if (lane == 0) {
                        mb_arrive(d_empty + 8 * (g & 1));
                    }
                    g++;
                }
            }
            if (!ok || !busy || n >= w.N) continue;
            const float bias = a.bias ? a.bias[(size_t)t.e * w.N + n] : 0.f;
            #pragma unroll
            for (int c = 0; c < 64; c++) {
                const int row = half * 64 + c;
                if (row < t.rows) w4_store(a.y, (size_t)(t.row0 + row) * a.ldy + n, a.y_dtype, w4_act(__uint_as_float((unsigned)(tot[c >> 1] >> (32 * (c & 1)))) + bias, a.act));
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 17) {
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

template <class T>
cudaError_t launch_tiles(const CUtensorMap &map, const W4Args &a, cudaStream_t s)
{
    const size_t smem = 1024 + (size_t)GM_STAGES * GM_STAGE_BYTES;
    cudaError_t e = cudaFuncSetAttribute(bls_w4_tiles_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    // an upper bound of the tiles: every matrix may end in a part of one
    const long long row_tiles = a.offsets ? min((long long)a.rows, (a.rows + GM_ROWS - 1) / GM_ROWS + (long long)a.w.E) : (a.rows + GM_ROWS - 1) / GM_ROWS;
    const int grid = (int)min(row_tiles * a.w.NT, (long long)sm_count());
    return launch_serialised_smem(bls_w4_tiles_kernel<T>, dim3(grid), dim3(GM_THREADS), smem, s, map, a);
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
    CUtensorMap map;
    if (!tc_make_map(&map, a.x, a.rows, a.w.K, a.ldx, GM_ROWS)) return cudaErrorInvalidValue;
    return x_dtype == BLS_BF16 ? launch_tiles<__nv_bfloat16>(map, a, s) : launch_tiles<__half>(map, a, s);
}
