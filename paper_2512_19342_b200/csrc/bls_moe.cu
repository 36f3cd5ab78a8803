// The movements of an expert stage: slots sorted by expert, rows moved to their experts and
// back as a weighted sum, and the gradients of both moves.
//
// Routing is a stable counting sort.  A tile of consecutive slots is counted per warp, an
// exclusive scan over (expert, tile, warp) gives every warp its first position for every
// expert, and inside a warp the position of a slot is the number of lower lanes with the same
// expert.  Up to ROUTE_ONE slots one block does it all; more take a kernel that counts
// the tiles and one in which every block adds up the counts before its own (tiles x E integers
// from L2) and sorts its tile.  Positions depend on scans only: the result is the unique stable sort, the
// same in every run.
//
// The moves are bound by memory: every row is read and written once, sums are fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "bls_device.cuh"
#include "bls_internal.h"

namespace {

constexpr int ROUTE_THREADS = 1024;
constexpr int ROUTE_WARPS = ROUTE_THREADS / 32;
constexpr int ROUTE_ONE = 4096;              // slots that one block sorts alone
constexpr int MOE_MAX_EXPERTS = 1024;
constexpr int MOVE_THREADS = 256;

// Inclusive scan over the block of one value per thread; scratch holds 32 words.
__device__ __forceinline__ int block_scan(int v, int *scratch)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    #pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, v, d);
        if (lane >= d) v += o;
    }
    if (lane == 31) scratch[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int s = scratch[lane];
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(~0u, s, d);
            if (lane >= d) s += o;
        }
        scratch[lane] = s;
    }
    __syncthreads();
    return v + (warp ? scratch[warp - 1] : 0);
}

// The lanes whose expert is this lane's, found bit by bit: 1 + log2(E) votes, a few instructions each (the warp's match instruction
// takes a turn for every different value, 400 cycles for 32 random experts).
__device__ __forceinline__ unsigned same_expert(int e, int bits)
{
    unsigned same = ~0u;
    for (int b = 0; b < bits; b++) {
        const bool set = (e >> b) & 1;
        const unsigned v = __ballot_sync(~0u, set);
        same &= set ? v : ~v;
    }
    return same;
}

// Counts of a tile's experts: row blockIdx.x of count [tiles][E].
__global__ void __launch_bounds__(ROUTE_THREADS) bls_moe_count_kernel(const int *expert, int n, int E, int tile, int *count)
{
    stream_order_enter();
    extern __shared__ int hist[];
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) hist[e] = 0;
    __syncthreads();
    const int lo = blockIdx.x * tile, hi = min(lo + tile, n);
    for (int i = lo + threadIdx.x; i < hi; i += ROUTE_THREADS) {
        const int e = expert[i];
        if ((unsigned)e < (unsigned)E) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) count[(size_t)blockIdx.x * E + e] = hist[e];
}

// Sorts tile blockIdx.x of the slots.  TILED: count holds the counts of all tiles, and the block adds up
// what lies before it; otherwise there is one block, which counts for itself.
// hist [ROUTE_WARPS][E]: counts, then first positions, of every warp; TILED: two more rows.
template <bool TILED>
__global__ void __launch_bounds__(ROUTE_THREADS) bls_moe_route_kernel(const int *expert, int n, int E, int tile, const int *count,
                                                                      int *order, int *place, int *offsets)
{
    stream_order_enter();
    extern __shared__ int hist[];
    __shared__ int scratch[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t0 = TILED ? blockIdx.x * tile : 0, t1 = min(t0 + tile, n);
    int *all = hist + ROUTE_WARPS * E, *before = all + E;
    for (int i = threadIdx.x; i < (ROUTE_WARPS + (TILED ? 2 : 0)) * E; i += ROUTE_THREADS) hist[i] = 0;
    __syncthreads();
    const int per = ((t1 - t0 + ROUTE_WARPS - 1) / ROUTE_WARPS + 31) & ~31;   // consecutive slots of a warp
    const int lo = min(t0 + warp * per, t1), hi = min(lo + per, t1);
    int *mine = hist + warp * E;
    const int bits = 32 - __clz(E);
    for (int i = lo; i < hi; i += 32) {
        const int e = i + lane < hi ? expert[i + lane] : -1;
        if ((unsigned)e < (unsigned)E) atomicAdd(&mine[e], 1);
    }
    if (TILED) {
        // every thread adds up one expert over a part of the tiles
        const int parts = E < ROUTE_THREADS ? ROUTE_THREADS / E : 1;
        const int e = threadIdx.x % E, part = threadIdx.x / E;
        if (part < parts) {
            int sum = 0, low = 0;
            #pragma unroll 8
            for (int t = part; t < (int)gridDim.x; t += parts) {
                const int c = count[(size_t)t * E + e];
                sum += c;
                low += t < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(&all[e], sum);
            atomicAdd(&before[e], low);
        }
    }
    __syncthreads();
    int total = 0;
    if (threadIdx.x < E) {
        if (TILED) total = all[threadIdx.x];
        else for (int w = 0; w < ROUTE_WARPS; w++) total += hist[w * E + threadIdx.x];
    }
    const int incl = block_scan(total, scratch);
    if (threadIdx.x < E) {
        int at = incl - total;
        if (blockIdx.x == 0) {
            offsets[threadIdx.x] = at;
            if (threadIdx.x == E - 1) offsets[E] = incl;
        }
        if (TILED) at += before[threadIdx.x];
        for (int w = 0; w < ROUTE_WARPS; w++) {
            const int c = hist[w * E + threadIdx.x];
            hist[w * E + threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int i = lo; i < hi; i += 32) {
        const int e = i + lane < hi ? expert[i + lane] : -1;
        const bool kept = (unsigned)e < (unsigned)E;
        const unsigned same = same_expert(kept ? e : E, bits);
        const int first = kept ? mine[e] : 0;
        __syncwarp();
        if (kept) {
            const int at = first + __popc(same & ((1u << lane) - 1));
            order[at] = i + lane;
            place[i + lane] = at;
            if (lane == __ffs(same) - 1) mine[e] = first + __popc(same);
        } else if (i + lane < hi) {
            place[i + lane] = -1;
        }
        __syncwarp();
    }
    // scratch[31] still holds the number of kept slots: order past it is -1
    for (int i = max(t0, scratch[31]) + threadIdx.x; i < t1; i += ROUTE_THREADS) order[i] = -1;
}

// Tiles of the slots, of about 1024 slots at least (832 of 4097); one up to ROUTE_ONE slots (one block and one launch: 4000 slots take 6.4 us, two
// kernels 5.4 us and another launch; 8000 slots 10.3 and 5.4).  74 tiles, half the SMs: every block reads the counts of all tiles, and
// 400k slots over 256 experts take 13.7 us with 74 tiles, 18.3 with 148, 16.1 with 50.
void route_tiles(long long n, int &tiles, int &tile)
{
    if (n <= ROUTE_ONE) { tiles = 1; tile = (int)n; return; }
    const long long want = min((n + 1023) / 1024, 74ll);
    tile = (int)(((n + want - 1) / want + 31) & ~31ll);
    tiles = (int)((n + tile - 1) / tile);
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// V elements of T that move as one piece: 16 bytes, or one element where rows do not allow it.  Pieces are kept as
// they were loaded and taken apart as fp32 only where they are summed.
template <class T, int V> struct Piece {
    using Raw = T;
    static __device__ __forceinline__ void floats(const Raw &r, float (&f)[V]) { f[0] = to_f(r); }
    static __device__ __forceinline__ Raw from(const float (&f)[V]) { return from_f<T>(f[0]); }
};
template <> struct Piece<float, 4> {
    using Raw = float4;
    static __device__ __forceinline__ void floats(const Raw &r, float (&f)[4]) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    static __device__ __forceinline__ Raw from(const float (&f)[4]) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Piece<__nv_bfloat16, 8> {
    using Raw = uint4;
    static __device__ __forceinline__ void floats(const Raw &r, float (&f)[8])
    {
        const unsigned u[4] = {r.x, r.y, r.z, r.w};
        #pragma unroll
        for (int i = 0; i < 4; i++) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ Raw from(const float (&f)[8])
    {
        unsigned u[4];
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            u[i] = *reinterpret_cast<unsigned *>(&h);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Piece<__half, 8> {
    using Raw = uint4;
    static __device__ __forceinline__ void floats(const Raw &r, float (&f)[8])
    {
        const unsigned u[4] = {r.x, r.y, r.z, r.w};
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 g = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
            f[2 * i] = g.x; f[2 * i + 1] = g.y;
        }
    }
    static __device__ __forceinline__ Raw from(const float (&f)[8])
    {
        unsigned u[4];
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            u[i] = *reinterpret_cast<unsigned *>(&h);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};

struct MoveArgs {
    const void *a;              // dispatch: x; combine: y; gradient: dout
    const void *b;              // gradient: y
    void *o;                    // dispatch: y; combine: out; gradient: dy
    long long lda, ldb, ldo;
    const int *place, *total;   // total: number of sorted rows (device)
    const float *w;
    float *dw;
    int tokens, rows, k;
    int pieces;                 // pieces of a row
    int lanes_log;              // threads of a token (of a slot)
};

// Who does what: 1 << lanes_log neighbouring threads take a token, its pieces `lane`, `lane` + lanes, .. .  Blocks
// share the tokens and, along the other axis, the turns of a long row (the gradient: the slots), so that no
// index is divided.
struct MoveLane {
    int token, step, lane, lanes;
    __device__ __forceinline__ MoveLane(const MoveArgs &m, int block, int blocks)
    {
        lanes = 1 << m.lanes_log;
        lane = threadIdx.x & (lanes - 1);
        const int per = MOVE_THREADS >> m.lanes_log;                          // tokens of a block
        token = block * per + (threadIdx.x >> m.lanes_log);
        step = blocks * per;
    }
};

template <class T, int V> using MP = typename Piece<T, V>::Raw;

// Sets the rows of o from *total on to zero; the blocks of the grid share them.
template <class T, int V>
__device__ __forceinline__ void zero_tail(const MoveArgs &m, const MoveLane &l, int part, int parts)
{
    const float none[V] = {};
    const MP<T, V> z = Piece<T, V>::from(none);
    const long long first = max(0, *m.total);
    for (long long r = first + l.token; r < m.rows; r += l.step)
        for (int p = part * l.lanes + l.lane; p < m.pieces; p += parts * l.lanes)
            *(MP<T, V> *)((T *)m.o + r * m.ldo + (long long)p * V) = z;
}

// A thread reads U pieces of a token and writes them to the token's k places: x is read once.  Bound by memory:
// 16384 x 8 x 2048 bf16 in 100 us (6.0 TB/s).  Rows that no whole piece divides (V = 1) are bound by issue: 75 % busy in
// 3001 x 3 x 1531, fp32 or bf16.
template <class T, int V>
__global__ void __launch_bounds__(MOVE_THREADS) bls_moe_dispatch_kernel(const __grid_constant__ MoveArgs m)
{
    stream_order_enter();
    constexpr int U = V == 1 ? 4 : 1;
    const MoveLane l(m, blockIdx.y, gridDim.y);
    for (long long t = l.token; t < m.tokens; t += l.step) {
        const int *place = m.place + t * m.k;
        for (int p0 = blockIdx.x * l.lanes * U + l.lane; p0 < m.pieces; p0 += gridDim.x * l.lanes * U) {
            MP<T, V> v[U];
            #pragma unroll
            for (int u = 0; u < U; u++)
                if (p0 + u * l.lanes < m.pieces) v[u] = *(const MP<T, V> *)((const T *)m.a + t * m.lda + (long long)(p0 + u * l.lanes) * V);
            for (int j = 0; j < m.k; j++) {
                const int at = __ldg(place + j);
                if ((unsigned)at >= (unsigned)m.rows) continue;
                T *o = (T *)m.o + at * m.ldo + (long long)p0 * V;
                #pragma unroll
                for (int u = 0; u < U; u++)
                    if (p0 + u * l.lanes < m.pieces) *(MP<T, V> *)(o + (long long)u * l.lanes * V) = v[u];
            }
        }
    }
    zero_tail<T, V>(m, l, blockIdx.x, gridDim.x);
}

// A thread sums U pieces of a token over its k rows, several rows' pieces on their way at a time, in the order of the slots.
// Bound by memory: 16384 x 8 x 2048 bf16 in 94 us (6.3 TB/s); eight rows on their way instead of four: 151.  With V = 1 by
// issue: 58 % busy with fp32, 66 % with bf16.
template <class T, int V>
__global__ void __launch_bounds__(MOVE_THREADS) bls_moe_combine_kernel(const __grid_constant__ MoveArgs m)
{
    stream_order_enter();
    constexpr int U = V == 1 ? 4 : 1, J = 4;
    const MoveLane l(m, blockIdx.y, gridDim.y);
    for (long long t = l.token; t < m.tokens; t += l.step) {
        const int *place = m.place + t * m.k;
        const float *weight = m.w + t * m.k;
        for (int p0 = blockIdx.x * l.lanes * U + l.lane; p0 < m.pieces; p0 += gridDim.x * l.lanes * U) {
            float acc[U][V];
            #pragma unroll
            for (int u = 0; u < U; u++)
                #pragma unroll
                for (int e = 0; e < V; e++) acc[u][e] = 0.f;
            for (int j0 = 0; j0 < m.k; j0 += J) {
                MP<T, V> v[J][U];
                int at[J];
                float w[J];
                #pragma unroll
                for (int j = 0; j < J; j++) {
                    at[j] = j0 + j < m.k ? __ldg(place + j0 + j) : -1;
                    w[j] = m.w && j0 + j < m.k ? __ldg(weight + j0 + j) : 1.f;
                }
                #pragma unroll
                for (int j = 0; j < J; j++)
                    if ((unsigned)at[j] < (unsigned)m.rows)
                        #pragma unroll
                        for (int u = 0; u < U; u++)
                            if (p0 + u * l.lanes < m.pieces)
                                v[j][u] = *(const MP<T, V> *)((const T *)m.a + at[j] * m.lda + (long long)(p0 + u * l.lanes) * V);
                #pragma unroll
                for (int j = 0; j < J; j++)
                    if ((unsigned)at[j] < (unsigned)m.rows)
                        #pragma unroll
                        for (int u = 0; u < U; u++) {
                            float f[V];
                            Piece<T, V>::floats(v[j][u], f);
                            #pragma unroll
                            for (int e = 0; e < V; e++) acc[u][e] = fmaf(w[j], f[e], acc[u][e]);
                        }
            }
            #pragma unroll
            for (int u = 0; u < U; u++) {
                if (p0 + u * l.lanes >= m.pieces) break;
                *(MP<T, V> *)((T *)m.o + t * m.ldo + (long long)(p0 + u * l.lanes) * V) = Piece<T, V>::from(acc[u]);
            }
        }
    }
}

// The lanes of a token take its slots (blockIdx.y: which of them): dy = w * dout and dw = <dout, y> in one pass over the
// row, U pieces at a time.  Bound by memory: 16384 x 8 x 2048 bf16 in 191 us (5.9 TB/s).
template <class T, int V>
__global__ void __launch_bounds__(MOVE_THREADS) bls_moe_combine_grad_kernel(const __grid_constant__ MoveArgs m)
{
    stream_order_enter();
    constexpr int U = V == 1 ? 8 : 4;
    const MoveLane l(m, blockIdx.x, gridDim.x);
    // all lanes of a warp take the same number of turns (the sums below are shuffled over the warp)
    const int sub = threadIdx.x % 32 >> m.lanes_log;
    for (long long t0 = l.token - sub; t0 < m.tokens; t0 += l.step) {
        const long long t = t0 + sub;
        const T *d = (const T *)m.a + t * m.lda;
        for (int j = blockIdx.y; j < m.k; j += gridDim.y) {
            const long long s = t * m.k + j;
            const int at = t < m.tokens ? __ldg(m.place + s) : -1;
            const bool kept = (unsigned)at < (unsigned)m.rows;
            float dot = 0.f;
            if (kept) {
                const float w = m.w ? __ldg(m.w + s) : 1.f;
                const T *y = (const T *)m.b + at * m.ldb;
                T *o = (T *)m.o + at * m.ldo;
                for (int p0 = l.lane; p0 < m.pieces; p0 += l.lanes * U) {
                    MP<T, V> g[U], v[U];
                    #pragma unroll
                    for (int u = 0; u < U; u++)
                        if (p0 + u * l.lanes < m.pieces) {
                            g[u] = *(const MP<T, V> *)(d + (long long)(p0 + u * l.lanes) * V);
                            if (m.dw) v[u] = *(const MP<T, V> *)(y + (long long)(p0 + u * l.lanes) * V);
                        }
                    #pragma unroll
                    for (int u = 0; u < U; u++)
                        if (p0 + u * l.lanes < m.pieces) {
                            float f[V], h[V];
                            Piece<T, V>::floats(g[u], f);
                            if (m.dw) {
                                Piece<T, V>::floats(v[u], h);
                                #pragma unroll
                                for (int e = 0; e < V; e++) dot = fmaf(f[e], h[e], dot);
                            }
                            #pragma unroll
                            for (int e = 0; e < V; e++) f[e] *= w;
                            *(MP<T, V> *)(o + (long long)(p0 + u * l.lanes) * V) = Piece<T, V>::from(f);
                        }
                }
            }
            if (m.dw) {
                for (int x = l.lanes >> 1; x; x >>= 1) dot += __shfl_xor_sync(~0u, dot, x);
                if (l.lane == 0 && t < m.tokens) m.dw[s] = kept ? dot : 0.f;
            }
        }
    }
    zero_tail<T, V>(m, l, blockIdx.y, gridDim.y);
}

bool whole_pieces(const void *p, long long ld, int dim, int elem)
{
    return ((uintptr_t)p & 15) == 0 && (ld * elem) % 16 == 0 && (dim * (long long)elem) % 16 == 0;
}

enum { MOVE_DISPATCH, MOVE_COMBINE, MOVE_GRAD };

template <class T, int V>
cudaError_t launch_move_v(int what, MoveArgs m, int dim, cudaStream_t s)
{
    m.pieces = dim / V;
    // no more threads than a row has pieces; a slot's gradient is summed inside a warp, and single elements are
    // taken by warps with more of them each
    m.lanes_log = what == MOVE_GRAD || V == 1 ? 5 : 8;
    while (m.lanes_log > 2 && 1 << (m.lanes_log - 1) >= m.pieces) m.lanes_log--;
    const long long per = MOVE_THREADS >> m.lanes_log, most = 148 * 32;
    const unsigned blocks = (unsigned)max(1ll, min((m.tokens + per - 1) / per, most));
    const int turn = (V == 1 ? 4 : 1) << m.lanes_log;
    const dim3 grid = what == MOVE_GRAD ? dim3(blocks, (unsigned)max(1ll, min((long long)m.k, most / blocks))) :
                                         dim3((unsigned)min((m.pieces + turn - 1) / turn, 1024), blocks);
    void (*kernel)(MoveArgs) = what == MOVE_DISPATCH ? bls_moe_dispatch_kernel<T, V> :
                               what == MOVE_COMBINE ? bls_moe_combine_kernel<T, V> : bls_moe_combine_grad_kernel<T, V>;
    return launch_serialised(kernel, grid, dim3(MOVE_THREADS), s, m);
}

bls_status_t launch_move(int what, const MoveArgs &m, int dtype, int dim, bool whole, cudaStream_t s)
{
    cudaError_t e;
    switch (dtype) {
    case BLS_F32: e = whole ? launch_move_v<float, 4>(what, m, dim, s) : launch_move_v<float, 1>(what, m, dim, s); break;
    case BLS_BF16: e = whole ? launch_move_v<__nv_bfloat16, 8>(what, m, dim, s) : launch_move_v<__nv_bfloat16, 1>(what, m, dim, s); break;
    default: e = whole ? launch_move_v<__half, 8>(what, m, dim, s) : launch_move_v<__half, 1>(what, m, dim, s); break;
    }
    return e == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

bool slots_ok(int64_t tokens, int k, int n_experts)
{
    return tokens >= 0 && k >= 1 && k <= 1024 && n_experts >= 1 && n_experts <= MOE_MAX_EXPERTS && tokens <= (1 << 30) / k;
}
bool move_ok(int dtype, int64_t tokens, int k, int dim, int64_t rows, int64_t ld0, int64_t ld1)
{
    return dtype >= 0 && dtype <= 2 && slots_ok(tokens, k, 1) && dim >= 1 && rows >= 0 && rows <= (1 << 30) && ld0 >= dim && ld1 >= dim;
}
int elem_bytes(int dtype) { return dtype == BLS_F32 ? 4 : 2; }

}  // namespace

extern "C" {

bls_status_t bls_moe_bytes(int64_t tokens, int k, int n_experts, size_t *bytes)
{
    if (!bytes || !slots_ok(tokens, k, n_experts)) return BLS_EINVAL;
    int tiles, tile;
    route_tiles(tokens * k, tiles, tile);
    *bytes = tiles == 1 ? 0 : (sizeof(int) * tiles * n_experts + 255) / 256 * 256;
    return BLS_OK;
}

bls_status_t bls_moe_route(const int32_t *expert, int64_t tokens, int k, int n_experts, int32_t *order, int32_t *place,
                           int32_t *offsets, void *workspace, size_t bytes, void *cuda_stream)
{
    size_t need = 0;
    if (bls_moe_bytes(tokens, k, n_experts, &need) != BLS_OK || !offsets || (tokens && (!expert || !order || !place))) return BLS_EINVAL;
    if (bytes < need) return BLS_ENOSPC;
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return BLS_EINVAL;
    const int n = (int)(tokens * k);
    int tiles, tile;
    route_tiles(n, tiles, tile);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    int *count = (int *)workspace;
    auto kernel = tiles == 1 ? bls_moe_route_kernel<false> : bls_moe_route_kernel<true>;
    const size_t smem = sizeof(int) * (ROUTE_WARPS + (tiles == 1 ? 0 : 2)) * n_experts;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return BLS_ECUDA;
    if (tiles > 1 && launch_serialised_smem(bls_moe_count_kernel, dim3(tiles), dim3(ROUTE_THREADS), sizeof(int) * n_experts, s, expert, n,
                                            n_experts, tile, count) != cudaSuccess)
        return BLS_ECUDA;
    return launch_serialised_smem(kernel, dim3(tiles), dim3(ROUTE_THREADS), smem, s, expert, n, n_experts, tile, (const int *)count, order,
                                  place, offsets) == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

bls_status_t bls_moe_dispatch(const void *x, int64_t ldx, int dtype, const int32_t *place, const int32_t *offsets,
                              int n_experts, int64_t tokens, int k, int dim, void *y, int64_t ldy, int64_t rows,
                              void *cuda_stream)
{
    if (!move_ok(dtype, tokens, k, dim, rows, ldx, ldy) || n_experts < 1 || n_experts > MOE_MAX_EXPERTS || !offsets ||
        (tokens && (!x || !place)) || (rows && !y))
        return BLS_EINVAL;
    if (rows == 0) return BLS_OK;
    MoveArgs m = {};
    m.a = x; m.lda = ldx; m.o = y; m.ldo = ldy; m.place = place; m.total = offsets + n_experts;
    m.tokens = (int)tokens; m.rows = (int)rows; m.k = k;
    const int eb = elem_bytes(dtype);
    return launch_move(MOVE_DISPATCH, m, dtype, dim, whole_pieces(x, ldx, dim, eb) && whole_pieces(y, ldy, dim, eb), (cudaStream_t)cuda_stream);
}

bls_status_t bls_moe_combine(const void *y, int64_t ldy, int64_t rows, int dtype, const int32_t *place, const float *w,
                             int64_t tokens, int k, int dim, void *out, int64_t ldo, void *cuda_stream)
{
    if (!move_ok(dtype, tokens, k, dim, rows, ldy, ldo) || (tokens && (!place || !out)) || (rows && !y)) return BLS_EINVAL;
    if (tokens == 0) return BLS_OK;
    MoveArgs m = {};
    m.a = y; m.lda = ldy; m.o = out; m.ldo = ldo; m.place = place; m.w = w;
    m.tokens = (int)tokens; m.rows = (int)rows; m.k = k;
    const int eb = elem_bytes(dtype);
    return launch_move(MOVE_COMBINE, m, dtype, dim, whole_pieces(y, ldy, dim, eb) && whole_pieces(out, ldo, dim, eb), (cudaStream_t)cuda_stream);
}

bls_status_t bls_moe_combine_grad(const void *dout, int64_t ldd, const void *y, int64_t ldy, int64_t rows, int dtype,
                                  const int32_t *place, const int32_t *offsets, int n_experts, const float *w,
                                  int64_t tokens, int k, int dim, void *dy, int64_t lddy, float *dw, void *cuda_stream)
{
    if (!move_ok(dtype, tokens, k, dim, rows, ldd, lddy) || n_experts < 1 || n_experts > MOE_MAX_EXPERTS || !offsets ||
        (tokens && (!dout || !place)) || (rows && !dy) || (dw && rows && (!y || ldy < dim)))
        return BLS_EINVAL;
    if (rows == 0 && !(dw && tokens)) return BLS_OK;
    MoveArgs m = {};
    m.a = dout; m.lda = ldd; m.b = y; m.ldb = ldy; m.o = dy; m.ldo = lddy; m.place = place; m.total = offsets + n_experts;
    m.w = w; m.dw = dw; m.tokens = (int)tokens; m.rows = (int)rows; m.k = k;
    const int eb = elem_bytes(dtype);
    const bool whole = whole_pieces(dout, ldd, dim, eb) && whole_pieces(dy, lddy, dim, eb) && (!dw || whole_pieces(y, ldy, dim, eb));
    return launch_move(MOVE_GRAD, m, dtype, dim, whole, (cudaStream_t)cuda_stream);
}

}  // extern "C"
