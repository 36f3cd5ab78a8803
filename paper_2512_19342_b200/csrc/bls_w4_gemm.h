// The many-rows kernel of the 4-bit product, as its host side calls it.
#pragma once
#include "bls_w4.cuh"

// Workspace it needs (rows of x that do not start at 16-byte boundaries are copied first).
size_t w4_tiles_bytes(const W4Weights &w, const void *x, long long ldx, long long rows);
cudaError_t w4_tiles(W4Args a, int x_dtype, void *workspace, cudaStream_t s);
