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

// The scales of two outputs and of all groups of a tile: one word per lane (lanes 8 g .. 8 g + 7: group g, outputs
// 2 (lane mod 8) and the next one of the 16), taken apart by shuffles when they are needed.
template <int GROUP> struct RowsSide { unsigned scale, zero; };

// Adds the products of up to 8 * NT rows of x with 16 * MT outputs over the tiles warp, warp + MV_WARPS, ..
// of 128 inputs.  A thread asks for the weights of U tiles before it uses the first.
template <class T, int GROUP, int MT, int NT, int U>
__device__ __forceinline__ void rows_product(const W4Args &a, const uint8_t *q, size_t side, int warp, int lane, int base, int hi,
                                             float (&tot)[MT][NT][4])
{
    constexpr int GPT = W4_TILE / GROUP;
    const W4Weights &w = a.w;
    const int gid = lane >> 2, tig = lane & 3, KT = w.KT;
    const size_t np = (size_t)w.NT * W4_TILE;
    // a lane's piece of output gid (and gid + 8, 512 bytes on, where the same swizzle holds): 64 bytes per output
    const uint8_t *mine = q + gid * 64 + ((tig ^ ((gid >> 1) & 3)) * 16);
    const unsigned *scale = (const unsigned *)(w.scale + side + (size_t)(lane >> 3) * np + (lane & 7) * 2);
    const unsigned short *zero = (const unsigned short *)(w.zero + side + (size_t)(lane >> 3) * np + (lane & 7) * 2);
    const bool holds = lane < 8 * GPT;
    for (int kt0 = warp; kt0 < KT; kt0 += MV_WARPS * U) {
        uint4 qw[U][MT][2];
        RowsSide<GROUP> sd[U][MT];
        #pragma unroll
        for (int u = 0; u < U; u++) {
            const int kt = kt0 + u * MV_WARPS;
            #pragma unroll
            for (int m = 0; m < MT; m++) {
                qw[u][m][0] = qw[u][m][1] = make_uint4(0, 0, 0, 0);
                sd[u][m].scale = 0; sd[u][m].zero = 0x0808;
                if (kt < KT) {
                    const uint8_t *p = mine + (size_t)kt * W4_TILE_BYTES + m * 1024;
                    qw[u][m][0] = __ldcs((const uint4 *)p);                        // read once: nothing else has to leave L2 for it
                    qw[u][m][1] = __ldcs((const uint4 *)(p + 512));
                    if (holds) {
                        sd[u][m].scale = __ldg(scale + ((size_t)kt * GPT * np + m * 16) / 2);
                        if (w.zero) sd[u][m].zero = __ldg(zero + ((size_t)kt * GPT * np + m * 16) / 2);
                    }
                }
            }
        }
        #pragma unroll
        for (int u = 0; u < U; u++) {
            const int kt = kt0 + u * MV_WARPS;
            if (kt >= KT) break;
            float acc[MT][NT][4];
            #pragma unroll
            for (int b = 0; b < 4; b++) {
                if (b * 32 % GROUP == 0) {
                    #pragma unroll
                    for (int m = 0; m < MT; m++)
                        #pragma unroll
                        for (int j = 0; j < NT; j++)
                            #pragma unroll
                            for (int c = 0; c < 4; c++) acc[m][j][c] = 0.f;
                }
                uint4 x[NT];
                #pragma unroll
                for (int j = 0; j < NT; j++) {
                    const int row = base + j * 8 + gid;
                    x[j] = make_uint4(0, 0, 0, 0);
                    if (row < hi) x[j] = load_x8<T>(a, row, kt * W4_TILE + b * 32 + tig * 8);
                }
                const int from = b * 32 / GROUP * 8 + (gid >> 1);
                #pragma unroll
                for (int m = 0; m < MT; m++) {
                    const unsigned za = __shfl_sync(~0u, sd[u][m].zero, from), zb = __shfl_sync(~0u, sd[u][m].zero, from + 4);
                    const unsigned z0 = w4_zero_pair<T>(za >> (8 * (gid & 1)) & 15), z1 = w4_zero_pair<T>(zb >> (8 * (gid & 1)) & 15);
                    const unsigned wa = b == 0 ? qw[u][m][0].x : b == 1 ? qw[u][m][0].y : b == 2 ? qw[u][m][0].z : qw[u][m][0].w;
                    const unsigned wb = b == 0 ? qw[u][m][1].x : b == 1 ? qw[u][m][1].y : b == 2 ? qw[u][m][1].z : qw[u][m][1].w;
                    unsigned pa[4], pb[4];
                    w4_unpack<T>(wa, z0, pa);
                    w4_unpack<T>(wb, z1, pb);
                    const unsigned f0[4] = {pa[0], pb[0], pa[1], pb[1]}, f1[4] = {pa[2], pb[2], pa[3], pb[3]};
                    #pragma unroll
                    for (int j = 0; j < NT; j++) {
                        mma_16816(acc[m][j], f0, x[j].x, x[j].y, T());
                        mma_16816(acc[m][j], f1, x[j].z, x[j].w, T());
                    }
                    if ((b + 1) * 32 % GROUP == 0) {                              // the group's sum is complete: scale it
                        const unsigned sa = __shfl_sync(~0u, sd[u][m].scale, from), sb = __shfl_sync(~0u, sd[u][m].scale, from + 4);
                        const float s0 = __uint_as_float(gid & 1 ? sa & 0xffff0000u : sa << 16), s1 = __uint_as_float(gid & 1 ? sb & 0xffff0000u : sb << 16);
                        #pragma unroll
                        for (int j = 0; j < NT; j++) {
                            tot[m][j][0] = fmaf(s0, acc[m][j][0], tot[m][j][0]);
                            tot[m][j][1] = fmaf(s0, acc[m][j][1], tot[m][j][1]);
                            tot[m][j][2] = fmaf(s1, acc[m][j][2], tot[m][j][2]);
                            tot[m][j][3] = fmaf(s1, acc[m][j][3], tot[m][j][3]);
                        }
                    }
                }
            }
        }
    }
}

// 8 * NT rows of x from `base` on: the warps' parts of the sums meet in shared memory, in the order of the warps.
template <class T, int GROUP, int MT, int NT>
__device__ __forceinline__ void rows_chunk(const W4Args &a, const uint8_t *q, size_t side, int e, int n0, int base, int hi, float *part)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    constexpr int O = 16 * MT, R = 8 * NT;
    float tot[MT][NT][4];
    #pragma unroll
    for (int m = 0; m < MT; m++)
        #pragma unroll
        for (int j = 0; j < NT; j++)
            #pragma unroll
            for (int c = 0; c < 4; c++) tot[m][j][c] = 0.f;
    rows_product<T, GROUP, MT, NT, 2>(a, q, side, warp, lane, base, hi, tot);
    __syncthreads();                                                      // the previous chunk's sums have been read
    float *mine = part + warp * O * R;
    #pragma unroll
    for (int m = 0; m < MT; m++)
        #pragma unroll
        for (int j = 0; j < NT; j++)
            #pragma unroll
            for (int c = 0; c < 4; c++) mine[(j * 8 + tig * 2 + (c & 1)) * O + m * 16 + gid + (c >> 1) * 8] = tot[m][j][c];
    __syncthreads();
    for (int i = threadIdx.x; i < O * R; i += MV_WARPS * 32) {
        const int n = n0 + i % O, row = base + i / O;
        if (n >= a.w.N || row >= hi) continue;
        float v = 0.f;
        #pragma unroll
        for (int k = 0; k < MV_WARPS; k++) v += part[k * O * R + i];
        if (a.bias) v += a.bias[(size_t)e * a.w.N + n];
        w4_store(a.y, (size_t)row * a.ldy + n, a.y_dtype, w4_act(v, a.act));
    }
}

// grid (ceil(N / (16 MT)), min(E, rows), + 1 with offsets): 16 MT outputs of one matrix that has rows; with fewer rows
// than matrices the y-th one that has any.  The last layer of blocks clears the rows that belong to no matrix.
template <class T, int GROUP, int MT, int NT>
__global__ void __launch_bounds__(MV_WARPS * 32) bls_w4_rows_kernel(const __grid_constant__ W4Args a)
{
    stream_order_enter();
    __shared__ float part[MV_WARPS * 16 * MT * 8 * NT];
    __shared__ int found;
    const int n0 = blockIdx.x * 16 * MT;
    const W4Weights &w = a.w;
    const int layers = min(w.E, a.rows);
    int e = blockIdx.y;
    if (e == layers) {
        const int first = min(max(a.offsets[w.E], 0), a.rows);
        for (long long i = threadIdx.x; i < (long long)(a.rows - first) * 16 * MT; i += blockDim.x) {
            const int n = n0 + (int)(i % (16 * MT));
            if (n < w.N) w4_store(a.y, (size_t)(first + i / (16 * MT)) * a.ldy + n, a.y_dtype, 0.f);
        }
        return;
    }
    if (a.offsets && layers < w.E) {
        // the matrices that have rows are counted by the first warp, 32 at a time
        if (threadIdx.x < 32) {
            int seen = 0, at = -1;
            for (int e0 = 0; e0 < w.E && at < 0; e0 += 32) {
                int lo = 0, hi = 0;
                if (e0 + (int)threadIdx.x < w.E) w4_rows(a, e0 + threadIdx.x, lo, hi);
                unsigned some = __ballot_sync(~0u, hi > lo);
                const int c = __popc(some);
                if (seen + c > e) at = e0 + __fns(some, 0, e - seen + 1);
                seen += c;
            }
            if (threadIdx.x == 0) found = at;
        }
        __syncthreads();
        e = found;
        if (e < 0) return;
    }
    int lo, hi;
    w4_rows(a, e, lo, hi);
    const uint8_t *q = w.q + ((size_t)e * w.NT + n0 / W4_TILE) * w.KT * W4_TILE_BYTES + n0 % W4_TILE * 64;
    const size_t side = (size_t)e * (w.KT * (W4_TILE / GROUP)) * w.NT * W4_TILE + n0;
    for (int base = lo; base < hi; ) {
        const int left = hi - base;
        if (NT >= 4 && left > 16) { rows_chunk<T, GROUP, MT, NT >= 4 ? 4 : 1>(a, q, side, e, n0, base, hi, part); base += 32; }
        else if (NT >= 2 && left > 8) { rows_chunk<T, GROUP, MT, NT >= 2 ? 2 : 1>(a, q, side, e, n0, base, hi, part); base += 16; }
        else { rows_chunk<T, GROUP, MT, 1>(a, q, side, e, n0, base, hi, part); base += 8; }
    }
}

template <int DT> struct W4Elem;
template <> struct W4Elem<BLS_F32> { using type = float; };
template <> struct W4Elem<BLS_BF16> { using type = __nv_bfloat16; };
template <> struct W4Elem<BLS_F16> { using type = __half; };
template <class T> struct alignas(16) W4Eight { T v[8]; };

// Eight elements as loaded (16 or 32 bytes), and as fp32.
template <class T> struct W4Raw { uint4 u[sizeof(T) / 2]; };
template <class T, bool WHOLE>
__device__ __forceinline__ W4Raw<T> w4_load8(const T *p, int avail)
{
    W4Raw<T> r;
    if (WHOLE && avail >= 8) {
        #pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; i++) r.u[i] = ((const uint4 *)p)[i];
        return r;
    }
    unsigned v[sizeof(T) * 2];
    #pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; i++) v[i] = 0;
    #pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < avail) {
            if (sizeof(T) == 4) v[i] = ((const unsigned *)p)[i];
            else v[i >> 1] |= (unsigned)((const unsigned short *)p)[i] << (16 * (i & 1));
        }
    #pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) r.u[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    return r;
}
__device__ __forceinline__ void w4_floats(const W4Raw<float> &r, float (&v)[8])
{
    #pragma unroll
    for (int i = 0; i < 2; i++) {
        v[4 * i] = __uint_as_float(r.u[i].x); v[4 * i + 1] = __uint_as_float(r.u[i].y);
        v[4 * i + 2] = __uint_as_float(r.u[i].z); v[4 * i + 3] = __uint_as_float(r.u[i].w);
    }
}
__device__ __forceinline__ void w4_floats(const W4Raw<__nv_bfloat16> &r, float (&v)[8])
{
    const unsigned u[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
    #pragma unroll
    for (int i = 0; i < 4; i++) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ void w4_floats(const W4Raw<__half> &r, float (&v)[8])
{
    const unsigned u[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
    #pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// grid (KT, NT, E): one tile.  A lane takes the eight inputs of one stored word, half a warp an output row; a
// group is 4, 8 or 16 neighbouring lanes.  A thread asks for four rows' pieces before it uses the
// first.  WHOLE: rows of w start at 16-byte boundaries.
//
// The floor is reading w once, which leaves about 20 instructions per element.  So rint(w / s) of the
// correctly rounded quotient comes from two products, with 1 / s made smaller and larger by 2^-19: a product is
// within 1.5 2^-23 of the quotient relatively, so where both round to the same number it is the
// right one.  Where they differ, fp32 inputs are divided.  16-bit inputs are then exactly halfway (w and
// s have few bits; a quotient up to 15 that is no half stays 1e-4 away from one), which happens
// often, and the even one of the two is right.  Adding 1.5 2^23 rounds a product to a whole number and
// leaves it in the low bits; the constant's bits leave the sum of the eight nibbles at the end.
template <int DT, bool WHOLE, bool ZERO>
__global__ void __launch_bounds__(256) bls_w4_quantize_kernel(const void *wv, long long ldw, W4Weights d, uint8_t *q,
                                                              __nv_bfloat16 *scale, uint8_t *zero)
{
    using T = typename W4Elem<DT>::type;
    stream_order_enter();
    __shared__ __nv_bfloat16 s_sc[4][W4_TILE];
    __shared__ uint8_t s_z[4][W4_TILE];
    const int kt = blockIdx.x, nt = blockIdx.y, e = blockIdx.z;
    const int l = threadIdx.x & 15;
    const int gpt = W4_TILE / d.group, lanes = d.group / 8;
    const int k = kt * W4_TILE + l * 8;
    const T *w = (const T *)wv + ((size_t)e * d.N + nt * W4_TILE) * ldw + k;
    uint8_t *tile = q + (((size_t)e * d.NT + nt) * d.KT + kt) * W4_TILE_BYTES;
    #pragma unroll 1
    for (int r0 = threadIdx.x >> 4; r0 < W4_TILE; r0 += 64) {
        W4Raw<T> p[4];
        #pragma unroll
        for (int u = 0; u < 4; u++) {
            const int r = r0 + u * 16;
            p[u] = w4_load8<T, WHOLE>(w + r * ldw, nt * W4_TILE + r < d.N ? d.K - k : 0);
        }
        #pragma unroll
        for (int u = 0; u < 4; u++) {
            const int r = r0 + u * 16;
            float v[8], lo = 0.f, hi = 0.f, bad = 0.f;                       // bad: NaN after a value that is not finite
            w4_floats(p[u], v);
            #pragma unroll
            for (int i = 0; i < 8; i++) {
                bad = fmaf(v[i], 0.f, bad);
                if (ZERO) lo = fminf(lo, v[i]);
                hi = fmaxf(hi, ZERO ? v[i] : fabsf(v[i]));
            }
            if (bad != 0.f) hi = __int_as_float(0x7f800000);
            for (int o = 1; o < lanes; o <<= 1) {
                if (ZERO) lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
            }
            float s = __bfloat162float(__float2bfloat16_rn(ZERO ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(hi, 7.f)));
            if (!isfinite(s)) s = __int_as_float(0x7fc00000);                // the whole group becomes NaN
            const __nv_bfloat16 sb = __float2bfloat16_rn(s);
            const bool usable = s > 0.f;
            const int z = !ZERO || nt * W4_TILE + r >= d.N ? 8 : usable ? (int)fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 0;
            // above 1e37 the reciprocal would be subnormal and lose bits
            const float inv = usable && s < 1e37f ? __fdividef(1.f, s) : __int_as_float(0x7fc00000);
            const float below = inv * (1.f - 0x1p-19f), above = inv * (1.f + 0x1p-19f);
            constexpr float ROUND = 12582912.f;                              // 1.5 2^23
            constexpr unsigned BITS = 0x4b400000u;                           // its bits
            unsigned word = (unsigned)z * 0x11111111u - BITS * 0x11111111u, differ = 0;
            #pragma unroll
            for (int i = 0; i < 8; i++) {
                unsigned t = __float_as_uint(fmaf(v[i], below, ROUND));
                const unsigned t2 = __float_as_uint(fmaf(v[i], above, ROUND));
                if (DT == BLS_F32) differ |= t ^ t2;
                else if (t & 1) t = t2;
                if (ZERO) t = min(t, BITS + 15u - z);                        // rint(w / s) + z is at least 0, but can reach 16
                word += t << (4 * ((i >> 1) + 4 * (i & 1)));
            }
            if (differ || !(fmaxf(hi, -lo) * inv < (ZERO ? 15.5f : 7.5f))) {      // !(..): also where inv is NaN
                word = 0;
                #pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int c = usable ? (int)rintf(__fdiv_rn(v[i], s)) : 0;
                    word |= (unsigned)min(max(c + z, 0), 15) << (4 * ((i >> 1) + 4 * (i & 1)));
                }
            }
            *(unsigned *)(tile + r * 64 + ((l & 3) ^ ((r >> 1) & 3)) * 16 + (l >> 2) * 4) = word;
            if (l % lanes == 0) {
                s_sc[l / lanes][r] = sb;
                s_z[l / lanes][r] = (uint8_t)z;
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < gpt * W4_TILE; i += blockDim.x) {
        const int g = i / W4_TILE, r = i % W4_TILE;
        const size_t at = ((size_t)e * d.KT * gpt + kt * gpt + g) * d.NT * W4_TILE + nt * W4_TILE + r;
        scale[at] = s_sc[g][r];
        if (ZERO) zero[at] = s_z[g][r];
    }
}

// grid (KT, NT, E): the inverse, with the same lanes; bound by writing w once.
template <int DT, bool WHOLE>
__global__ void __launch_bounds__(256) bls_w4_dequantize_kernel(W4Weights d, void *wv, long long ldw)
{
    using T = typename W4Elem<DT>::type;
    stream_order_enter();
    __shared__ float s_sc[4][W4_TILE];
    __shared__ int s_z[4][W4_TILE];
    const int kt = blockIdx.x, nt = blockIdx.y, e = blockIdx.z;
    const int l = threadIdx.x & 15, gpt = W4_TILE / d.group;
    const int k = kt * W4_TILE + l * 8, g = l * 8 / d.group;
    const uint8_t *tile = d.q + (((size_t)e * d.NT + nt) * d.KT + kt) * W4_TILE_BYTES;
    unsigned word[8];
    #pragma unroll
    for (int u = 0; u < 8; u++) {
        const int r = (threadIdx.x >> 4) + u * 16;
        word[u] = __ldg((const unsigned *)(tile + r * 64 + ((l & 3) ^ ((r >> 1) & 3)) * 16 + (l >> 2) * 4));
    }
    for (int i = threadIdx.x; i < gpt * W4_TILE; i += blockDim.x) {
        const size_t at = ((size_t)e * d.KT * gpt + kt * gpt + i / W4_TILE) * d.NT * W4_TILE + nt * W4_TILE + i % W4_TILE;
        s_sc[i / W4_TILE][i % W4_TILE] = __bfloat162float(d.scale[at]);
        s_z[i / W4_TILE][i % W4_TILE] = d.zero ? d.zero[at] & 15 : 8;
    }
    __syncthreads();
    T *w = (T *)wv + ((size_t)e * d.N + nt * W4_TILE) * ldw + k;
    #pragma unroll
    for (int u = 0; u < 8; u++) {
        const int r = (threadIdx.x >> 4) + u * 16;
        if (nt * W4_TILE + r >= d.N) break;
        const float s = s_sc[g][r];
        const int z = s_z[g][r];
        W4Eight<T> o;
        #pragma unroll
        for (int i = 0; i < 8; i++) o.v[i] = T((float)((int)((word[u] >> (4 * ((i >> 1) + 4 * (i & 1)))) & 15) - z) * s);
        if (WHOLE && k + 8 <= d.K) {
            *(W4Eight<T> *)(w + r * ldw) = o;
        } else {
            #pragma unroll
            for (int i = 0; i < 8; i++)
                if (k + i < d.K) w[r * ldw + i] = o.v[i];
        }
    }
}

// A kernel of one type with or without whole 16-byte pieces.
#define W4_PICK(KERNEL, dtype, whole, ...)                                                                                        \
    ((dtype) == BLS_F32 ? ((whole) ? KERNEL<BLS_F32, true __VA_ARGS__> : KERNEL<BLS_F32, false __VA_ARGS__>) :                        \
     (dtype) == BLS_BF16 ? ((whole) ? KERNEL<BLS_BF16, true __VA_ARGS__> : KERNEL<BLS_BF16, false __VA_ARGS__>) :                     \
                           ((whole) ? KERNEL<BLS_F16, true __VA_ARGS__> : KERNEL<BLS_F16, false __VA_ARGS__>))
#define W4_COMMA ,

bool w4_whole(const void *w, int dtype, long long ldw) { return ((uintptr_t)w & 15) == 0 && ldw * (dtype == BLS_F32 ? 4 : 2) % 16 == 0; }

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

template <class T, int GROUP, int MT>
cudaError_t launch_rows_m(const W4Args &a, cudaStream_t s)
{
    const dim3 grid((a.w.N + 16 * MT - 1) / (16 * MT), min(a.w.E, a.rows) + (a.offsets ? 1 : 0)), block(MV_WARPS * 32);
    return a.rows <= 8 ? launch_serialised(bls_w4_rows_kernel<T, GROUP, MT, 1>, grid, block, s, a) :
           a.rows <= 16 ? launch_serialised(bls_w4_rows_kernel<T, GROUP, MT, 2>, grid, block, s, a) :
                          launch_serialised(bls_w4_rows_kernel<T, GROUP, MT, 4>, grid, block, s, a);
}
template <class T, int GROUP>
cudaError_t launch_rows_g(const W4Args &a, cudaStream_t s)
{
    const long long blocks = (long long)((a.w.N + 31) / 32) * min(a.w.E, a.rows);
    return blocks >= 2 * 148 ? launch_rows_m<T, GROUP, 2>(a, s) : launch_rows_m<T, GROUP, 1>(a, s);
}
template <class T>
cudaError_t launch_rows(const W4Args &a, cudaStream_t s)
{
    return a.w.group == 32 ? launch_rows_g<T, 32>(a, s) : a.w.group == 64 ? launch_rows_g<T, 64>(a, s) : launch_rows_g<T, 128>(a, s);
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
    return launch_serialised(zero ? W4_PICK(bls_w4_quantize_kernel, dtype, w4_whole(w, dtype, ldw), W4_COMMA true) :
                                    W4_PICK(bls_w4_quantize_kernel, dtype, w4_whole(w, dtype, ldw), W4_COMMA false), dim3(d.KT, d.NT, E), dim3(256),
                             (cudaStream_t)cuda_stream, w, (long long)ldw, d, q,
                             (__nv_bfloat16 *)scale, zero) == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

bls_status_t bls_w4_dequantize(const uint8_t *q, const void *scale, const uint8_t *zero, int E, int N, int K, int group,
                               void *w, int dtype, int64_t ldw, void *cuda_stream)
{
    W4Weights d = {};
    if (!w || !q || !scale || ((uintptr_t)q & 15) || dtype < 0 || dtype > 2 || ldw < K || !w4_shape(E, N, K, group, d)) return BLS_EINVAL;
    d.q = q; d.scale = (const __nv_bfloat16 *)scale; d.zero = zero;
    return launch_serialised(W4_PICK(bls_w4_dequantize_kernel, dtype, w4_whole(w, dtype, ldw)), dim3(d.KT, d.NT, E), dim3(256),
                             (cudaStream_t)cuda_stream, d, w, (long long)ldw) ==
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
    if (!q || !scale || (((uintptr_t)q | (uintptr_t)scale | (uintptr_t)zero) & 15) || !w4_shape(E, N, K, group, a.w) || bls_w4_bytes(E, N, K, x, ldx, rows, &need) != BLS_OK ||
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
                    x_dtype == BLS_BF16 ? launch_rows<__nv_bfloat16>(a, (cudaStream_t)cuda_stream) : launch_rows<__half>(a, (cudaStream_t)cuda_stream);
    return r == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

}  // extern "C"
