// Linear layers with 4-bit weights: the product for few rows, quantisation and its inverse, and
// the host side.
//
// y[r][n] = act(bias[n] + sum_g s[n][g] * sum_{c in g} (q[n][c] - z[n][g]) x[r][c]).
// With few rows the product is bound by reading the weights (K / 2 bytes for 2 K operations per
// row).  The weights are the A operand of mma.m16n8k16 (16 outputs x 16 inputs), 8 rows of x the
// B operand: an instruction then takes 256 weights for one word per lane, which leaves the ALUs
// only the unpacking.  The order of the inputs inside a product is free, so a lane
// takes the inputs that one stored 16-byte piece holds, and the same 8 neighbouring x values per word.
//
// At this size a layer is a few such steps per warp, so what counts is that all loads are on their way
// at once and that many warps share the unpacking: the 16 warps of a block split K (and, where K is short
// or there is plenty of work, also the outputs), and their sums meet in shared memory in the order of the slices.
// One row: 4096 x 4096 in 5.3 us, 8192 x 8192 in 15 us (2.2 TB/s); 64 matrices of 2048 x 1024 with a row each in 25 us (2.7 TB/s).
// Neither memory (23 % of its rate, 8192 x 8192) nor issue (50 %; 7.5 M instructions are 6.4 of the 15 us) is full: a warp asks for its
// next tiles only after it has used the ones it has, and the block meets twice a round for x.  So a round costs
// a memory latency and then its instructions, 179 for 16 x 128 weights.
// 64 registers per thread, for two blocks on an SM; 10 of the 12 forms spill 4 to 12 bytes of them.
#include "bls_w4.cuh"
#include "bls_w4_gemm.h"

namespace {

constexpr int FR_WARPS = 16;
constexpr int FR_U = 2;                              // tiles of weights a warp has on their way

__device__ __forceinline__ void mma_16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, bool first, __nv_bfloat16)
{
    if (first) {                                     // known when compiled: c = a b
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
        return;
    }
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, bool first, __half)
{
    if (first) {                                     // known when compiled: c = a b
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
        return;
    }
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight x values of a row from input k on, zeros past K.
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

// grid (blocks of 16 * OW outputs, min(E, rows), + 1 with offsets), OW = 16 >> kw_log: the outputs of one matrix that
// has rows; with fewer rows than matrices the y-th one that has any.  KW = 1 << kw_log warps split K.
// The last layer of blocks clears the rows that belong to no matrix.
template <class T, int GROUP, bool ZERO>
__global__ void __launch_bounds__(FR_WARPS * 32, 2) bls_w4_rows_kernel(const __grid_constant__ W4Args a, int kw_log)
{
    stream_order_enter();
    constexpr int GPT = W4_TILE / GROUP;
    extern __shared__ __align__(16) unsigned char fr_smem[];
    __shared__ int found;
    const W4Weights &w = a.w;
    const int KW = 1 << kw_log, outs = 16 * (FR_WARPS >> kw_log);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int layers = min(w.E, a.rows);
    int e = blockIdx.y;
    if (e == layers) {
        const int first = min(max(a.offsets[w.E], 0), a.rows);
        for (long long i = threadIdx.x; i < (long long)(a.rows - first) * outs; i += blockDim.x) {
            const int n = blockIdx.x * outs + (int)(i % outs);
            if (n < w.N) w4_store(a.y, (size_t)(first + i / outs) * a.ldy + n, a.y_dtype, 0.f);
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
    const int kw = warp & (KW - 1), n0 = blockIdx.x * outs + (warp >> kw_log) * 16, KT = w.KT;
    const bool live = n0 < w.N;
    // a lane's piece of output gid (and gid + 8, 512 bytes on, where the same swizzle holds): 64 bytes per output
    const uint8_t *q = w.q + ((size_t)e * w.NT + n0 / W4_TILE) * KT * W4_TILE_BYTES + (n0 % W4_TILE + gid) * 64 + ((tig ^ ((gid >> 1) & 3)) * 16);
    // scales and zero points of a tile are held by lanes 8 g .. 8 g + 7 (and the lanes 8 GPT on): group g, outputs
    // 2 (lane mod 8) and the next one
    const size_t np = (size_t)w.NT * W4_TILE, side = (size_t)e * KT * GPT * np + n0 + (size_t)(lane >> 3 & (GPT - 1)) * np + (lane & 7) * 2;
    const int round = KW * FR_U, pitch = round * W4_TILE * 2 + 64;            // 64 past a multiple of 128: two rows fill the banks
    const int pieces_log = kw_log + 5;                                        // 16-byte pieces of a row in a round: KW * 2 * 16
    const size_t gstep = (size_t)KW * GPT * np;                               // scales from a tile to this warp's next one
    const int piece = threadIdx.x & ((1 << pieces_log) - 1), row0 = threadIdx.x >> pieces_log;
    for (int base = lo; base < hi; base += 8) {
        const int cnt = min(8, hi - base);
        float tot[4] = {0.f, 0.f, 0.f, 0.f};
        const uint8_t *qk = q + (size_t)kw * W4_TILE_BYTES;
        const __nv_bfloat16 *sk = w.scale + side + (size_t)(kw * GPT) * np;
        const uint8_t *zk = w.zero + side + (size_t)(kw * GPT) * np;
        for (int k0 = 0; k0 < KT; k0 += round) {
            const int mine = live ? KT - k0 - kw : 0;                         // > u * KW: this warp has tile u of the round
            uint4 qw[FR_U][2];
            unsigned sc[FR_U], zr[FR_U];
            #pragma unroll
            for (int u = 0; u < FR_U; u++) {
                sc[u] = 0; zr[u] = 0x0808;
                if (mine > u * KW) {
                    qw[u][0] = __ldcs((const uint4 *)qk);
                    qw[u][1] = __ldcs((const uint4 *)(qk + 512));
                    sc[u] = __ldg((const unsigned *)sk);
                    if (ZERO) zr[u] = __ldg((const unsigned short *)zk);
                }
                qk += KW * W4_TILE_BYTES;
                sk += gstep;
                if (ZERO) zk += gstep;
            }
            if (k0) __syncthreads();                                          // the previous round's x has been used
            if (k0 * (W4_TILE / 8) + piece < KT * (W4_TILE / 8))
                for (int r = row0; r < cnt; r += FR_WARPS * 32 >> pieces_log)
                    *(uint4 *)(fr_smem + r * pitch + piece * 16) = load_x8(a, base + r, k0 * W4_TILE + piece * 8);
            __syncthreads();
            // rows past cnt take the last one's x: a column of the product depends on its own row alone, and theirs are not stored
            #pragma unroll
            for (int u = 0; u < FR_U; u++) {
                if (mine <= u * KW) break;
                const unsigned char *xs = fr_smem + min(gid, cnt - 1) * pitch + (u * KW + kw) * W4_TILE * 2 + tig * 16;
                const unsigned wa[4] = {qw[u][0].x, qw[u][0].y, qw[u][0].z, qw[u][0].w}, wb[4] = {qw[u][1].x, qw[u][1].y, qw[u][1].z, qw[u][1].w};
                float acc[2][4];                                              // two chains of products
                #pragma unroll
                for (int b = 0; b < 4; b++) {
                    const uint4 x = *(const uint4 *)(xs + b * 64);
                    const int from = b * 32 / GROUP * 8 + (gid >> 1);
                    unsigned z0 = w4_zero_pair<T>(8), z1 = z0;
                    if (ZERO) {
                        z0 = w4_zero_pair<T>(__shfl_sync(~0u, zr[u], from) >> (8 * (gid & 1)) & 15);
                        z1 = w4_zero_pair<T>(__shfl_sync(~0u, zr[u], from + 4) >> (8 * (gid & 1)) & 15);
                    }
                    unsigned pa[4], pb[4];
                    w4_unpack<T>(wa[b], z0, pa);
                    w4_unpack<T>(wb[b], z1, pb);
                    const unsigned f0[4] = {pa[0], pb[0], pa[1], pb[1]}, f1[4] = {pa[2], pb[2], pa[3], pb[3]};
                    mma_16816(acc[0], f0, x.x, x.y, b * 32 % GROUP == 0, T());
                    mma_16816(acc[1], f1, x.z, x.w, b * 32 % GROUP == 0, T());
                    if ((b + 1) * 32 % GROUP == 0) {                          // the group's sum is complete: scale it
                        const unsigned sa = __shfl_sync(~0u, sc[u], from), sb = __shfl_sync(~0u, sc[u], from + 4);
                        const float s0 = __uint_as_float(gid & 1 ? sa & 0xffff0000u : sa << 16), s1 = __uint_as_float(gid & 1 ? sb & 0xffff0000u : sb << 16);
                        tot[0] = fmaf(s0, acc[0][0] + acc[1][0], tot[0]);
                        tot[1] = fmaf(s0, acc[0][1] + acc[1][1], tot[1]);
                        tot[2] = fmaf(s1, acc[0][2] + acc[1][2], tot[2]);
                        tot[3] = fmaf(s1, acc[0][3] + acc[1][3], tot[3]);
                    }
                }
            }
        }
        // tot: outputs gid, gid + 8 of rows 2 tig, 2 tig + 1
        __syncthreads();                                                      // x has been used
        float *part = (float *)fr_smem;                                       // [KW][8 rows][outs]
        #pragma unroll
        for (int c = 0; c < 4; c++) part[(kw * 8 + tig * 2 + (c & 1)) * outs + (warp >> kw_log) * 16 + gid + (c >> 1) * 8] = tot[c];
        __syncthreads();
        const int outs_log = 8 - kw_log;
        for (int i = threadIdx.x; i < cnt << outs_log; i += FR_WARPS * 32) {
            const int n = blockIdx.x * outs + (i & (outs - 1)), r = i >> outs_log;
            if (n >= w.N) continue;
            float v = 0.f;
            for (int k = 0; k < KW; k++) v += part[(k << (outs_log + 3)) + i];
            if (a.bias) v += a.bias[(size_t)e * w.N + n];
            w4_store(a.y, (size_t)(base + r) * a.ldy + n, a.y_dtype, w4_act(v, a.act));
        }
        if (base + 8 < hi) __syncthreads();
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

// (span + more) / STEPS rounded once to bfloat16; more: what the rounded span leaves out.  A tie of bfloat16 times STEPS has few
// enough bits for fp32, so the span and the quotient are rounded to one side of a tie or onto it, never past it.
// On a tie the remainder, exact in fp32, says on which side the quotient lies, and the low bit of the fp32 quotient keeps it there.
template <int STEPS>
__device__ __forceinline__ float w4_scale(float span, float more)
{
    unsigned s = __float_as_uint(__fdiv_rn(span, (float)STEPS));
    if ((s & 0xffffu) == 0x8000u) {
        float rest = fmaf(-(float)STEPS, __uint_as_float(s), span);
        if (rest == 0.f) rest = more;
        s += rest > 0.f ? 1u : rest < 0.f ? ~0u : 0u;
    }
    return __bfloat162float(__float2bfloat16_rn(__uint_as_float(s)));
}
// The same for hi - lo, hi >= 0 >= lo.  A difference past fp32's range is taken in halves.
__device__ __forceinline__ float w4_scale_between(float lo, float hi)
{
    const float part = isinf(hi - lo) ? 0.5f : 1.f;
    hi *= part; lo *= part;
    const float span = hi - lo, b = span - hi;
    return w4_scale<15>(span, (hi - (span - b)) - (lo + b)) / part;
}

// grid (KT, NT, E): one tile.  A lane takes the sixteen inputs of two stored words, eight lanes an output row; a
// group is 2, 4 or 8 neighbouring lanes.  A thread asks for two rows' pieces before it uses the
// first.  WHOLE: rows of w start at 16-byte boundaries.
//
// The floor, reading w once and writing q, leaves 14 instructions per weight of 16 bits; 19 are used, with the issue slots 78 % busy.
// A division per weight would take many more, so rint(w / s) of the correctly rounded quotient comes from two products, with 1 / s made smaller and larger by 2^-19: a product is
// within 1.5 2^-23 of the quotient relatively, so where both round to the same number it is the
// right one.  Where they differ, fp32 inputs are divided.  16-bit inputs are then exactly halfway (w and
// s have few bits; a quotient up to 15 that is no half stays 1e-4 away from one), which happens
// often, and the even one of the two is right.  Adding 1.5 2^23 rounds a product to a whole number and
// leaves it in the low bits; the constant's bits leave the sum of the eight nibbles at the end.
// 16 matrices of 4096 x 2048 bf16 take 85 us (4.0 TB/s, floor 51); a division per weight took 390.
template <int DT, bool WHOLE, bool ZERO>
__global__ void __launch_bounds__(256) bls_w4_quantize_kernel(const void *wv, long long ldw, W4Weights d, uint8_t *q,
                                                              __nv_bfloat16 *scale, uint8_t *zero)
{
    using T = typename W4Elem<DT>::type;
    stream_order_enter();
    __shared__ __nv_bfloat16 s_sc[4][W4_TILE];
    __shared__ uint8_t s_z[4][W4_TILE];
    const int kt = blockIdx.x, nt = blockIdx.y, e = blockIdx.z;
    const int l = threadIdx.x & 7;
    const int gpt = W4_TILE / d.group, lanes = d.group / 16;
    const int k = kt * W4_TILE + l * 16;
    const T *w = (const T *)wv + ((size_t)e * d.N + nt * W4_TILE) * ldw + k;
    uint8_t *tile = q + (((size_t)e * d.NT + nt) * d.KT + kt) * W4_TILE_BYTES;
    #pragma unroll 1
    for (int r0 = threadIdx.x >> 3; r0 < W4_TILE; r0 += 64) {
        W4Raw<T> p[2][2];
        #pragma unroll
        for (int u = 0; u < 2; u++) {
            const int r = r0 + u * 32, avail = nt * W4_TILE + r < d.N ? d.K - k : 0;
            p[u][0] = w4_load8<T, WHOLE>(w + r * ldw, avail);
            p[u][1] = w4_load8<T, WHOLE>(w + r * ldw + 8, avail - 8);
        }
        #pragma unroll
        for (int u = 0; u < 2; u++) {
            const int r = r0 + u * 32;
            float v[2][8], lo = 0.f, hi = 0.f, bad = 0.f;                       // bad: NaN after a value that is not finite
            w4_floats(p[u][0], v[0]);
            w4_floats(p[u][1], v[1]);
            #pragma unroll
            for (int j = 0; j < 2; j++)
                #pragma unroll
                for (int i = 0; i < 8; i++) {
                    bad = fmaf(v[j][i], 0.f, bad);
                    if (ZERO) lo = fminf(lo, v[j][i]);
                    hi = fmaxf(hi, ZERO ? v[j][i] : fabsf(v[j][i]));
                }
            if (bad != 0.f) hi = __int_as_float(0x7f800000);
            for (int o = 1; o < lanes; o <<= 1) {
                if (ZERO) lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
            }
            float s = ZERO ? w4_scale_between(lo, hi) : w4_scale<7>(hi, 0.f);
            if (!isfinite(s)) s = __int_as_float(0x7fc00000);                // the whole group becomes NaN
            const __nv_bfloat16 sb = __float2bfloat16_rn(s);
            const bool usable = s > 0.f;
            const int z = !ZERO || nt * W4_TILE + r >= d.N ? 8 : usable ? (int)fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 0;
            // above 1e37 the reciprocal would be subnormal and lose bits, below 2^-126 the fast division is not defined
            const float inv = s >= 0x1p-126f && s < 1e37f ? __fdividef(1.f, s) : __int_as_float(0x7fc00000);
            const float below = inv * (1.f - 0x1p-19f), above = inv * (1.f + 0x1p-19f);
            constexpr float ROUND = 12582912.f;                              // 1.5 2^23
            constexpr unsigned BITS = 0x4b400000u;                           // its bits
            unsigned word[2], differ = 0;
            #pragma unroll
            for (int j = 0; j < 2; j++) {
                word[j] = (unsigned)z * 0x11111111u - BITS * 0x11111111u;
                #pragma unroll
                for (int i = 0; i < 8; i++) {
                    unsigned t = __float_as_uint(fmaf(v[j][i], below, ROUND));
                    const unsigned t2 = __float_as_uint(fmaf(v[j][i], above, ROUND));
                    if (DT == BLS_F32) differ |= t ^ t2;
                    else if (t & 1) t = t2;
                    if (ZERO) t = min(t, BITS + 15u - z);                    // rint(w / s) + z is at least 0, but can reach 16
                    word[j] += t << (4 * ((i >> 1) + 4 * (i & 1)));
                }
            }
            if (differ || !(fmaxf(hi, -lo) * inv < (ZERO ? 15.5f : 7.5f))) {      // !(..): also where inv is NaN
                #pragma unroll
                for (int j = 0; j < 2; j++) {
                    word[j] = 0;
                    #pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const int c = usable ? (int)rintf(__fdiv_rn(v[j][i], s)) : 0;
                        word[j] |= (unsigned)min(max(c + z, 0), 15) << (4 * ((i >> 1) + 4 * (i & 1)));
                    }
                }
            }
            #pragma unroll
            for (int j = 0; j < 2; j++) {
                const int m = 2 * l + j;                                     // eight inputs: block m / 4 of 32, quarter m mod 4
                *(unsigned *)(tile + r * 64 + ((m & 3) ^ ((r >> 1) & 3)) * 16 + (m >> 2) * 4) = word[j];
            }
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

// grid (KT, NT, E): the inverse, eight inputs per lane; bound by writing w once (57 us for the same, 5.9 TB/s).
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

// Which kernel: by the rows that a matrix gets on average, since the offsets are on the device.  4096 x 4096: 8 rows 6.9 us here,
// 9 rows 9.8 us in tiles and 10.2 here, 16 rows 9.8 and 11.6; 8192 x 8192: 8 rows 20 us here, 16 rows 20 in tiles and 38 here.
// With many matrices the average is a fair guide for even loads alone.  64 matrices of 2048 x 1024 (groups of 64): 128 rows over
// all of them take 26 us here and 39 in tiles, 512 rows 44 and 39; but 512 rows of 16, 4 and 1 of the matrices take 80, 188 and
// 459 us here and 14, 14 and 9 in tiles, because a matrix's rows are taken eight at a time, one after the other.
bool many_rows(const W4Weights &w, int64_t rows) { return rows > 8ll * w.E; }

template <class T, int GROUP>
cudaError_t launch_rows_g(const W4Args &a, cudaStream_t s)
{
    const int layers = min(a.w.E, a.rows);
    // K is split over as many warps as have two tiles each, or fewer where the outputs alone keep 32 warps on every SM busy
    int kw_log = 4;
    while (kw_log > 0 && ((a.w.KT < FR_U << kw_log) || (((long long)(a.w.N + 15) / 16 * layers) << kw_log) > 2 * 32 * 148)) kw_log--;
    const int outs = 16 * (FR_WARPS >> kw_log), rows = min(8, a.rows);
    const size_t smem = max((size_t)rows * ((FR_U << kw_log) * W4_TILE * 2 + 64), (size_t)FR_WARPS * 16 * 8 * sizeof(float));
    auto kernel = a.w.zero ? bls_w4_rows_kernel<T, GROUP, true> : bls_w4_rows_kernel<T, GROUP, false>;
    cudaError_t e = smem <= 48 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_serialised_smem(kernel, dim3((a.w.N + outs - 1) / outs, layers + (a.offsets ? 1 : 0)), dim3(FR_WARPS * 32), smem, s, a, kw_log);
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
    a.y_pieces = y_dtype != BLS_F32 && ((uintptr_t)y & 15) == 0 && ldy % 8 == 0 && N % 8 == 0;
    cudaError_t r = many_rows(a.w, rows) ? w4_tiles(a, x_dtype, workspace, (cudaStream_t)cuda_stream) :
                    x_dtype == BLS_BF16 ? launch_rows<__nv_bfloat16>(a, (cudaStream_t)cuda_stream) : launch_rows<__half>(a, (cudaStream_t)cuda_stream);
    return r == cudaSuccess ? BLS_OK : BLS_ECUDA;
}

}  // extern "C"
