// Linear layers with 4-bit weights: the product for few rows, quantisation and its inverse, and
// the host side.
//
// y[r][n] = act(bias[n] + sum_g s[n][g] * sum_{c in g} (q[n][c] - z[n][g]) x[r][c]).
// With few rows the product is bound by reading the weights (K / 2 bytes for 2 K operations per
// row).  The weights are the A operand of mma.m16n8k16 (16 outputs x 16 inputs), 8 rows of x the
// B operand: an instruction then takes 256 weights for one word per lane, which leaves the ALUs
// only the unpacking.  The order of the inputs inside a product is free, so a lane
// takes the inputs that one stored 16-byte piece holds, and reads the same 8 neighbouring x values per word.
#include "bls_w4.cuh"
#include "bls_w4_gemm.h"

namespace {

constexpr int MV_WARPS = 8;                  // the warps of a block share 16 outputs and split K

__device__ __forceinline__ void mma_16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight x values from input k on, zeros past K.
template <class T>
__device__ __forceinline__ uint4 load_x8(const W4Args &a, long long row, int k)
{
    const unsigned short *p = (const unsigned short *)a.x + row * a.ldx + k;
    if (a.x_pieces && k + 8 <= a.w.K) return *(const uint4 *)p;
    unsigned v[4] = {0, 0, 0, 0};
    #pragma unroll
    for (int i = 0; i < 8; i++)
        if (k + i < a.w.K) v[i >> 1] |= (unsigned)p[i] << (16 * (i & 1));
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// grid (ceil(N / 16), E + 1): 16 outputs of one matrix; the last layer of blocks clears the rows
// that belong to no matrix.
template <class T, int NT>
__global__ void __launch_bounds__(MV_WARPS * 32) bls_w4_rows_kernel(W4Args a)
{
    stream_order_enter();
    __shared__ float part[MV_WARPS][16][8 * NT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int n0 = blockIdx.x * 16, e = blockIdx.y;
    const W4Weights &w = a.w;
    if (e == w.E) {
        if (!a.offsets) return;
        const int first = min(max(a.offsets[w.E], 0), a.rows);
        for (long long i = threadIdx.x; i < (long long)(a.rows - first) * 16; i += blockDim.x) {
            const int n = n0 + (int)(i & 15);
            if (n < w.N) w4_store(a.y, (size_t)(first + (i >> 4)) * a.ldy + n, a.y_dtype, 0.f);
        }
        return;
    }
    int lo, hi;
    w4_rows(a, e, lo, hi);
    const int r0 = n0 % W4_TILE + gid;                                   // this lane's outputs in the tile: r0, r0 + 8
    const int groups = w.KT * W4_TILE / w.group, gpt = W4_TILE / w.group;
    const uint8_t *q = w.q + ((size_t)e * w.NT + n0 / W4_TILE) * w.KT * W4_TILE_BYTES + r0 * 64;
    const int p0 = (tig ^ ((r0 >> 1) & 3)) * 16, p1 = 512 + (tig ^ (((r0 + 8) >> 1) & 3)) * 16;
    const size_t s0 = (size_t)e * groups * w.NT * W4_TILE + n0 + gid;
    for (int base = lo; base < hi; base += 8 * NT) {
        float tot[NT][4], acc[NT][4];
        #pragma unroll
        for (int j = 0; j < NT; j++)
            #pragma unroll
            for (int c = 0; c < 4; c++) tot[j][c] = acc[j][c] = 0.f;
        for (int kt = warp; kt < w.KT; kt += MV_WARPS) {
            const uint4 qa = *(const uint4 *)(q + (size_t)kt * W4_TILE_BYTES + p0);
            const uint4 qb = *(const uint4 *)(q + (size_t)kt * W4_TILE_BYTES + p1);
            const unsigned wa[4] = {qa.x, qa.y, qa.z, qa.w}, wb[4] = {qb.x, qb.y, qb.z, qb.w};
            #pragma unroll
            for (int b = 0; b < 4; b++) {
                const int g = kt * gpt + b * 32 / w.group;
                const size_t sg = s0 + (size_t)g * w.NT * W4_TILE;
                const unsigned z0 = w4_zero_pair<T>(w.zero ? w.zero[sg] & 15 : 8), z1 = w4_zero_pair<T>(w.zero ? w.zero[sg + 8] & 15 : 8);
                unsigned pa[4], pb[4];
                w4_unpack<T>(wa[b], z0, pa);
                w4_unpack<T>(wb[b], z1, pb);
                const unsigned f0[4] = {pa[0], pb[0], pa[1], pb[1]}, f1[4] = {pa[2], pb[2], pa[3], pb[3]};
                #pragma unroll
                for (int j = 0; j < NT; j++) {
                    const int row = base + j * 8 + gid;
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (row < hi) x = load_x8<T>(a, row, kt * W4_TILE + b * 32 + tig * 8);
                    mma_16816(acc[j], f0, x.x, x.y, T());
                    mma_16816(acc[j], f1, x.z, x.w, T());
                }
                if ((b + 1) * 32 % w.group == 0) {                        // the group's sum is complete: scale it
                    const float sc0 = __bfloat162float(w.scale[sg]), sc1 = __bfloat162float(w.scale[sg + 8]);
                    #pragma unroll
                    for (int j = 0; j < NT; j++) {
                        tot[j][0] = fmaf(sc0, acc[j][0], tot[j][0]);
                        tot[j][1] = fmaf(sc0, acc[j][1], tot[j][1]);
                        tot[j][2] = fmaf(sc1, acc[j][2], tot[j][2]);
                        tot[j][3] = fmaf(sc1, acc[j][3], tot[j][3]);
                        #pragma unroll
                        for (int c = 0; c < 4; c++) acc[j][c] = 0.f;
                    }
                }
            }
        }
        __syncthreads();                                                  // the previous chunk's sums have been read
        #pragma unroll
        for (int j = 0; j < NT; j++) {
            part[warp][gid][j * 8 + tig * 2] = tot[j][0];
            part[warp][gid][j * 8 + tig * 2 + 1] = tot[j][1];
            part[warp][gid + 8][j * 8 + tig * 2] = tot[j][2];
            part[warp][gid + 8][j * 8 + tig * 2 + 1] = tot[j][3];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * 8 * NT; i += blockDim.x) {
            const int o = i & 15, r = i >> 4, n = n0 + o, row = base + r;
            if (n >= w.N || row >= hi) continue;
            float v = 0.f;
            #pragma unroll
            for (int k = 0; k < MV_WARPS; k++) v += part[k][o][r];
            if (a.bias) v += a.bias[(size_t)e * w.N + n];
            w4_store(a.y, (size_t)row * a.ldy + n, a.y_dtype, w4_act(v, a.act));
        }
    }
}

__device__ __forceinline__ float w4_load(const void *p, size_t i, int dtype)
{
    if (dtype == BLS_F32) return ((const float *)p)[i];
    if (dtype == BLS_BF16) return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
    return __half2float(((const __half *)p)[i]);
}

// grid (KT, NT, E): one tile.  A warp takes an output row, a lane four neighbouring inputs, so that a
// group is 8, 16 or 32 neighbouring lanes and a stored word two lanes.
__global__ void __launch_bounds__(256) bls_w4_quantize_kernel(const void *w, int dtype, long long ldw, W4Weights d, uint8_t *q,
                                                              __nv_bfloat16 *scale, uint8_t *zero)
{
    stream_order_enter();
    __shared__ __nv_bfloat16 s_sc[4][W4_TILE];
    __shared__ uint8_t s_z[4][W4_TILE];
    const int kt = blockIdx.x, nt = blockIdx.y, e = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int gpt = W4_TILE / d.group, lanes = d.group / 4;
    uint8_t *tile = q + (((size_t)e * d.NT + nt) * d.KT + kt) * W4_TILE_BYTES;
    for (int r = warp; r < W4_TILE; r += 8) {
        const int n = nt * W4_TILE + r, k = kt * W4_TILE + lane * 4;
        float v[4], lo = 0.f, hi = 0.f;
        bool bad = false;
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            v[i] = n < d.N && k + i < d.K ? w4_load(w, ((size_t)e * d.N + n) * ldw + k + i, dtype) : 0.f;
            bad |= !isfinite(v[i]);
            lo = fminf(lo, v[i]);
            hi = fmaxf(hi, v[i]);
        }
        for (int o = 1; o < lanes; o <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
            bad |= __shfl_xor_sync(~0u, (int)bad, o) != 0;
        }
        const __nv_bfloat16 sb = bad ? __float2bfloat16_rn(__int_as_float(0x7fc00000)) :
                                 __float2bfloat16_rn(zero ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(hi, -lo), 7.f));
        const float s = __bfloat162float(sb);
        const bool usable = s > 0.f && isfinite(s);
        const float z = !zero || n >= d.N ? 8.f : usable ? fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 0.f;
        unsigned word = 0;
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            const float c = usable ? rintf(__fdiv_rn(v[i], s)) : 0.f;
            const unsigned u = (unsigned)fminf(fmaxf(c + z, 0.f), 15.f);
            word |= u << (4 * (((i >> 1) | ((lane & 1) << 1)) + 4 * (i & 1)));    // input i + 4 (lane mod 2) of the word
        }
        word |= __shfl_xor_sync(~0u, word, 1);
        const int b = lane >> 3, t = (lane >> 1) & 3;
        if ((lane & 1) == 0) *(unsigned *)(tile + r * 64 + (t ^ ((r >> 1) & 3)) * 16 + b * 4) = word;
        if (lane % lanes == 0) {
            s_sc[lane / lanes][r] = sb;
            s_z[lane / lanes][r] = (uint8_t)z;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < gpt * W4_TILE; i += blockDim.x) {
        const int g = i / W4_TILE, r = i % W4_TILE;
        const size_t at = ((size_t)e * d.KT * gpt + kt * gpt + g) * d.NT * W4_TILE + nt * W4_TILE + r;
        scale[at] = s_sc[g][r];
        if (zero) zero[at] = s_z[g][r];
    }
}

// grid (KT, NT, E): the inverse, with the same lanes.
__global__ void __launch_bounds__(256) bls_w4_dequantize_kernel(W4Weights d, void *w, int dtype, long long ldw)
{
    stream_order_enter();
    const int kt = blockIdx.x, nt = blockIdx.y, e = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int gpt = W4_TILE / d.group;
    const uint8_t *tile = d.q + (((size_t)e * d.NT + nt) * d.KT + kt) * W4_TILE_BYTES;
    for (int r = warp; r < W4_TILE; r += 8) {
        const int n = nt * W4_TILE + r, k = kt * W4_TILE + lane * 4;
        if (n >= d.N || k >= d.K) continue;
        const int b = lane >> 3, t = (lane >> 1) & 3;
        const unsigned word = *(const unsigned *)(tile + r * 64 + (t ^ ((r >> 1) & 3)) * 16 + b * 4);
        const size_t sg = ((size_t)e * d.KT * gpt + kt * gpt + lane * 4 / d.group) * d.NT * W4_TILE + n;
        const float s = __bfloat162float(d.scale[sg]);
        const int z = d.zero ? d.zero[sg] & 15 : 8;
        #pragma unroll
        for (int i = 0; i < 4; i++) {
            const int u = (word >> (4 * (((i >> 1) | ((lane & 1) << 1)) + 4 * (i & 1)))) & 15;
            if (k + i < d.K) w4_store(w, ((size_t)e * d.N + n) * ldw + k + i, dtype, (float)(u - z) * s);
        }
    }
}

bool w4_shape(int E, int N, int K, int group, W4Weights &w)
{
    if (E < 1 || E > 1024 || N < 1 || N > (1 << 20) || K < 1 || K > (1 << 20) || (group != 32 && group != 64 && group != 128)) return false;
    w.E = E; w.N = N; w.K = K; w.group = group;
    w.NT = (N + W4_TILE - 1) / W4_TILE;
    w.KT = (K + W4_TILE - 1) / W4_TILE;
    return true;
}

// Which kernel: by the rows that a matrix gets on average.
bool many_rows(const W4Weights &w, int64_t rows) { return rows > 32ll * w.E; }

template <class T, int NT>
cudaError_t launch_rows(const W4Args &a, cudaStream_t s)
{
    return launch_serialised(bls_w4_rows_kernel<T, NT>, dim3((a.w.N + 15) / 16, a.w.E + (a.offsets ? 1 : 0)), dim3(MV_WARPS * 32), s, a);
}
template <class T>
cudaError_t launch_linear4(const W4Args &a, cudaStream_t s)
{
    if (a.rows <= 8) return launch_rows<T, 1>(a, s);
    if (a.rows <= 16) return launch_rows<T, 2>(a, s);
    return launch_rows<T, 4>(a, s);
}

}  // namespace

extern "C" {

bls_status_t bls_w4_sizes(int E, int N, int K, int group, int64_t *q_bytes, int64_t *scale_elems)
{
    W4Weights w;
    if (!q_bytes || !scale_elems || !w4_shape(E, N, K, group, w)) return BLS_EINVAL;
    *q_bytes = (int64_t)E * w.NT * w.KT * W4_TILE_BYTES;
    *scale_elems = (int64_t)E * w.NT * w.KT * W4_TILE * (W4_TILE / group);
    return BLS_OK;
}

bls_status_t bls_w4_quantize(const void *w, int dtype, int64_t ldw, int E, int N, int K, int group, uint8_t *q, void *scale,
                             uint8_t *zero, void *cuda_stream)
{
    W4Weights d = {};
    if (!w || !q || !scale || ((uintptr_t)q & 15) || dtype < 0 || dtype > 2 || ldw < K || !w4_shape(E, N, K, group, d)) return BLS_EINVAL;
    if (d.NT > 65535) return BLS_EINVAL;
    return launch_serialised(bls_w4_quantize_kernel, dim3(d.KT, d.NT, E), dim3(256), (cudaStream_t)cuda_stream, w, dtype, ldw, d, q,
                             (__nv_bfloat16 *)scale, zero) == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

bls_status_t bls_w4_dequantize(const uint8_t *q, const void *scale, const uint8_t *zero, int E, int N, int K, int group,
                               void *w, int dtype, int64_t ldw, void *cuda_stream)
{
    W4Weights d = {};
    if (!w || !q || !scale || ((uintptr_t)q & 15) || dtype < 0 || dtype > 2 || ldw < K || !w4_shape(E, N, K, group, d)) return BLS_EINVAL;
    d.q = q; d.scale = (const __nv_bfloat16 *)scale; d.zero = zero;
    return launch_serialised(bls_w4_dequantize_kernel, dim3(d.KT, d.NT, E), dim3(256), (cudaStream_t)cuda_stream, d, w, dtype, ldw) ==
           cudaSuccess ? BLS_OK : BLS_ECUDA;
}

bls_status_t bls_w4_bytes(int E, int N, int K, const void *x, int64_t ldx, int64_t rows, size_t *bytes)
{
    W4Weights d;
    if (!bytes || rows < 0 || rows > (1 << 30) || !w4_shape(E, N, K, 32, d)) return BLS_EINVAL;
    *bytes = many_rows(d, rows) ? w4_tiles_bytes(d, x, ldx, rows) : 0;
    return BLS_OK;
}

bls_status_t bls_w4_linear(const uint8_t *q, const void *scale, const uint8_t *zero, int E, int N, int K, int group,
                           const void *x, int x_dtype, int64_t ldx, int64_t rows, const int32_t *offsets,
                           const float *bias, int act, void *y, int y_dtype, int64_t ldy, void *workspace, size_t bytes,
                           int32_t *status, void *cuda_stream)
{
    W4Args a = {};
    size_t need = 0;
    if (!q || !scale || ((uintptr_t)q & 15) || !w4_shape(E, N, K, group, a.w) || bls_w4_bytes(E, N, K, x, ldx, rows, &need) != BLS_OK ||
        (x_dtype != BLS_BF16 && x_dtype != BLS_F16) || y_dtype < 0 || y_dtype > 2 || act < 0 || act > 2 || ldx < K || ldy < N ||
        (!offsets && E != 1) || (rows && (!x || !y)) || !status)
        return BLS_EINVAL;
    if (bytes < need) return BLS_ENOSPC;
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return BLS_EINVAL;
    if (rows == 0) return BLS_OK;
    a.w.q = q; a.w.scale = (const __nv_bfloat16 *)scale; a.w.zero = zero;
    a.x = x; a.ldx = ldx; a.rows = (int)rows; a.x_pieces = ((uintptr_t)x & 15) == 0 && ldx % 8 == 0;
    a.offsets = offsets; a.bias = bias; a.act = act; a.y = y; a.y_dtype = y_dtype; a.ldy = ldy; a.status = status;
    cudaError_t r = many_rows(a.w, rows) ? w4_tiles(a, x_dtype, workspace, (cudaStream_t)cuda_stream) :
                    x_dtype == BLS_BF16 ? launch_linear4<__nv_bfloat16>(a, (cudaStream_t)cuda_stream) : launch_linear4<__half>(a, (cudaStream_t)cuda_stream);
    return r == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

}  // extern "C"
