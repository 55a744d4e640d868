// Pieces that the tiled kernels of MX4 products share.
#pragma once

#include "hlq_mx4_gemm.h"
#include "hlq_mfma_common.h"

// A lane of the matrix core holds 16 bytes of a row.  In LDS a row's panel is four such pieces, piece p at place p ^ key(row):
// reading one piece of 8 or of 16 successive rows then meets every bank once.
__device__ __forceinline__ int piece_key(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 1); }

// as dma_16B_per_lane, 4 bytes a lane
__device__ __forceinline__ void dma_4B_per_lane(const void *gptr, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(gptr), "s"(lds_base) : "memory", "m0");
}
