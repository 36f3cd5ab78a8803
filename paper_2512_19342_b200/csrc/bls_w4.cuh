// The 4-bit weight format, and what the kernels that read it share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "bls_device.cuh"
#include "bls_internal.h"

constexpr int W4_TILE = 128;                 // outputs and inputs of a stored tile
constexpr int W4_TILE_BYTES = 128 * 64;

struct W4Weights {
    const uint8_t *q;                        // [E][NT][KT][128][64]
    const __nv_bfloat16 *scale;              // [E][KT * 128 / group][NT * 128]
    const uint8_t *zero;                     // like scale, or NULL
    int E, N, K, NT, KT, group;
};

struct W4Args {
    W4Weights w;
    const void *x;                           // [rows][ldx], bf16 or f16
    long long ldx;
    int rows;
    int x_pieces;                            // rows of x start at 16-byte boundaries
    const int *offsets;                      // [E + 1] or NULL (one matrix, all rows)
    const float *bias;                       // [E][N] or NULL
    int act;
    void *y;
    int y_dtype;
    int y_pieces;                            // 16-bit rows of y (and N) are whole 16-byte pieces
    long long ldy;
    int *status;
};

__device__ __forceinline__ float w4_act(float v, int act)
{
    if (act == 1) return v < 0.f ? 0.f : v;                  // a NaN stays one
    if (act == 2) return 1.f / (1.f + expf(-v));
    return v;
}

template <class Y> __device__ __forceinline__ Y from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void w4_store(void *y, size_t i, int dtype, float v)
{
    if (dtype == BLS_F32) ((float *)y)[i] = v;
    else if (dtype == BLS_BF16) ((__nv_bfloat16 *)y)[i] = __float2bfloat16_rn(v);
    else ((__half *)y)[i] = __float2half_rn(v);
}

// First and last row of matrix e; a broken offsets array cannot lead outside x and y.
__device__ __forceinline__ void w4_rows(const W4Args &a, int e, int &lo, int &hi)
{
    lo = 0; hi = a.rows;
    if (a.offsets) {
        lo = min(max(a.offsets[e], 0), a.rows);
        hi = min(max(a.offsets[e + 1], lo), a.rows);
    }
}

// Four pairs of neighbouring inputs (k0,k1) .. (k6,k7) of one stored word, as x's type, minus the
// zero point.  The number q in the low bits of the constant's mantissa is 128 + q in bf16 (1024 + q in
// f16) exactly, and so is the difference with 128 + z (1024 + z).  The difference is one packed
// multiply-add per pair (v * 1 - zero); the header's subtraction compiles to more.
template <class T> struct W4Pairs;
template <> struct W4Pairs<__nv_bfloat16> {
    static constexpr unsigned MAGIC = 0x43004300u;
    static __device__ __forceinline__ unsigned add(unsigned a, unsigned z)
    {
        unsigned r;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(0x3f803f80u), "r"(z));
        return r;
    }
};
template <> struct W4Pairs<__half> {
    static constexpr unsigned MAGIC = 0x64006400u;
    static __device__ __forceinline__ unsigned add(unsigned a, unsigned z)
    {
        unsigned r;
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(0x3c003c00u), "r"(z));
        return r;
    }
};
// minus the pair of the zero point z
template <class T>
__device__ __forceinline__ unsigned w4_zero_pair(int z) { return (W4Pairs<T>::MAGIC | 0x80008000u) | (unsigned)z | ((unsigned)z << 16); }
template <class T>
__device__ __forceinline__ void w4_unpack(unsigned word, unsigned zero_pair, unsigned (&p)[4])
{
    #pragma unroll
    for (int j = 0; j < 4; j++) {
        unsigned v;
        asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(v) : "r"(word >> (4 * j)), "r"(W4Pairs<T>::MAGIC));   // (a & b) | c
        p[j] = W4Pairs<T>::add(v, zero_pair);
    }
}
