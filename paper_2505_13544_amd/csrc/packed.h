// Packed pages: complete pages of the slot storage with their latents in 4 bits (gfx950).
//
// A row's latents are E2M1 numbers (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times one power of two per 32 of them, the
// MX format's block: v_cvt_scalef32_pk_bf16_fp4 turns two of them into bf16 with the scale applied, exactly (a number has two
// significant bits, and the scale's exponent is bf16's own).  RoPE keys stay bf16: they are a ninth of a row, and they alone place a slot in time.
// Everything of 16 slots lies together in the order in which the matrix cores take it, 16 bytes of slot 0, of slot 1, ...:
//   codes   [page][tile of 16 slots][r / 32][16 slots][16 bytes]   32 latents: the even ones in the low nibbles
//   scales  [page][tile][r / 32][16 slots]                         the power of two's exponent + 127; 255: the block is NaN
//   keys    [page][tile][d_rope / 8][16 slots][8]                  bf16
// so that a wavefront's load of a column slice of 16 slots is one run of bytes.
#pragma once
#include "mtla_kernels.h"
#include "packed_scale.h"

namespace mtla {

constexpr int kPackTile = 16;    // slots
constexpr int kPackBlock = 32;   // latents with one scale

// Bytes of one tile's codes, scales and keys.
__host__ __device__ constexpr size_t packed_code_bytes(int r) { return (size_t)r * 8; }
__host__ __device__ constexpr size_t packed_scale_bytes(int r) { return (size_t)r / 2; }
__host__ __device__ constexpr size_t packed_key_bytes(int d_rope) { return (size_t)d_rope * 32; }

__host__ __device__ inline int clamp_page(int page, int n_pages) { return page < 0 ? 0 : (page < n_pages ? page : n_pages - 1); }

}  // namespace mtla
