// Complete pages between the bf16 pool and packed pages (the format: packed.h).
//
// One workgroup takes the 16 slots of a tile: rows come in whole, 16 bytes a lane, four lanes to a block of 32 latents, which find
// the block's largest magnitude among themselves, round their eight numbers with v_cvt_scalef32_pk_fp4_bf16 (nearest, ties to the even
// code, beyond 6 to 6) and put the four bytes into LDS, where the tile's codes get the packed order; they leave as whole lines.  The way back is the
// same in the other direction and exact.  Nothing but bytes bounds either: 2 (r + d_R) bytes of a slot on one side, r / 2 + r / 32 + 2 d_R on the other.
// At r = 512, d_R = 64: 245500 slots, 283 MB on one side and 98 MB on the other, into packed pages 103 us (3.7 TB/s, where a large sum reads 4.0) and back 64 us (packed
// pages just written are still in the last-level cache); 500 slots of 16 sequences at r = 256 3.0 and 2.7 us, launches.
#include "bounds.h"
#include "mtla_device.h"
#include "packed.h"

namespace mtla {

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_of_quad(uint32_t v) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true);  // lane ^ 1
  v = v > o ? v : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true);           // lane ^ 2
  return v > o ? v : o;
}

struct PackTile {  // where a tile's parts lie in both forms
  uint16_t* lat;
  uint16_t* key;
  uint8_t* codes;
  uint8_t* scales;
  uint16_t* keys;
};

__device__ __forceinline__ PackTile pack_tile(const PackArgs& a, int b, int page, int tile) {
  const size_t at = (size_t)b * a.pages.max_pages + page;
  const int tiles = 1 << (a.pages.shift - 4);
  const size_t row = ((size_t)clamp_page(a.pages.table[at], a.pages.n_pages) << a.pages.shift) + kPackTile * tile;
  const size_t pt = (size_t)clamp_page(a.pk.table[at], a.pk.n_pages) * tiles + tile;
  return PackTile{reinterpret_cast<uint16_t*>(a.cache_c) + row * a.r, reinterpret_cast<uint16_t*>(a.cache_kr) + row * a.d_rope,
                  a.pk.codes + pt * packed_code_bytes(a.r), a.pk.scales + pt * packed_scale_bytes(a.r), a.pk.keys + pt * (packed_key_bytes(a.d_rope) / 2)};
}

// grid = (pages_each * tiles of a page, batch): further pages of a sequence are taken in turns
template <bool PACK, int R>
__global__ __launch_bounds__(kBlock) void pack_kernel(PackArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char s_codes[R * 8];
  __shared__ __attribute__((aligned(16))) unsigned char s_scales[R / 2];
  const int tid = threadIdx.x, b = blockIdx.y;
  const int tiles_log = a.pages.shift - 4, tile = blockIdx.x & ((1 << tiles_log) - 1);
  const int first = pages_inside(a.first ? a.first[b] : 0, a.pages.max_pages), end = pages_inside(a.end[b], a.pages.max_pages);
  constexpr int RP = R / 8, kPieces = kPackTile * RP;         // 16-byte pieces of a row and of the tile
  constexpr int kOwn = (kPieces + kBlock - 1) / kBlock;       // of a thread: all of them asked for at once
  const int kp = a.d_rope / 8, n_keys = kPackTile * kp;
  for (int page = first + (int)(blockIdx.x >> tiles_log); page < end; page += a.pages_each) {
    const PackTile t = pack_tile(a, b, page, tile);
    if constexpr (PACK) {
      uint4 v[kOwn];
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int i = tid + k * kBlock;
        if (i < kPieces) v[k] = *reinterpret_cast<const uint4*>(t.lat + (size_t)8 * i);  // (the tile's rows lie one behind the other)
      }
      for (int i = tid; i < n_keys; i += kBlock) {
        const int unit = i / kPackTile, row = i % kPackTile;
        *reinterpret_cast<uint4*>(t.keys + 8 * i) = *reinterpret_cast<const uint4*>(t.key + (size_t)row * a.d_rope + 8 * unit);
      }
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int i = tid + k * kBlock, row = i / RP, piece = i % RP;
        if (i >= kPieces) break;
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
          top = top > lo ? top : lo;
          top = top > hi ? top : hi;
        }
        top = max_of_quad(top);  // (as integers: magnitudes order as their bits do, and a NaN is above them all)
        const uint32_t sc = packed_scale_of(top);
        const float scale = __uint_as_float(sc << 23);
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[0]), scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[1]), scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[2]), scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[3]), scale, 3);
        const int at = (piece >> 2) * kPackTile + row;
        *reinterpret_cast<uint32_t*>(s_codes + at * 16 + 4 * (piece & 3)) = code;
        if ((piece & 3) == 0) s_scales[at] = (unsigned char)sc;
      }
      __syncthreads();
      for (int i = tid; i < kPieces / 4; i += kBlock) *reinterpret_cast<uint4*>(t.codes + 16 * i) = *reinterpret_cast<const uint4*>(s_codes + 16 * i);
      for (int i = tid; i < R / 8; i += kBlock) *reinterpret_cast<uint32_t*>(t.scales + 4 * i) = *reinterpret_cast<const uint32_t*>(s_scales + 4 * i);
    } else {
      for (int i = tid; i < kPieces / 4; i += kBlock) *reinterpret_cast<uint4*>(s_codes + 16 * i) = *reinterpret_cast<const uint4*>(t.codes + 16 * i);
      for (int i = tid; i < R / 8; i += kBlock) *reinterpret_cast<uint32_t*>(s_scales + 4 * i) = *reinterpret_cast<const uint32_t*>(t.scales + 4 * i);
      for (int i = tid; i < n_keys; i += kBlock) {
        const int unit = i / kPackTile, row = i % kPackTile;
        *reinterpret_cast<uint4*>(t.key + (size_t)row * a.d_rope + 8 * unit) = *reinterpret_cast<const uint4*>(t.keys + 8 * i);
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int i = tid + k * kBlock, row = i / RP, piece = i % RP, at = (piece >> 2) * kPackTile + row;
        if (i >= kPieces) break;
        const uint32_t code = *reinterpret_cast<const uint32_t*>(s_codes + at * 16 + 4 * (piece & 3));
        const float scale = __uint_as_float((uint32_t)s_scales[at] << 23);
        uint4 v;
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
        *reinterpret_cast<uint4*>(t.lat + (size_t)8 * i) = v;
      }
    }
    __syncthreads();  // the next page's codes take the same place
  }
}

template <bool PACK>
hipError_t launch_as(PackArgs a, hipStream_t st) {
  // pages_each is what the caller expects of a sequence; the grid stays a grid whatever it says
  const long long tiles = 1LL << (a.pages.shift - 4), most = (1LL << 20) / tiles;
  long long each = a.pages_each < a.pages.max_pages ? a.pages_each : a.pages.max_pages;
  each = each < 1 ? 1 : (each > most && most > 0 ? most : each);
  a.pages_each = (int)each;
  const dim3 grid((unsigned)(each * tiles), a.batch);
  switch (a.r) {
    case 64: hipLaunchKernelGGL((pack_kernel<PACK, 64>), grid, dim3(kBlock), 0, st, a); break;
    case 128: hipLaunchKernelGGL((pack_kernel<PACK, 128>), grid, dim3(kBlock), 0, st, a); break;
    case 256: hipLaunchKernelGGL((pack_kernel<PACK, 256>), grid, dim3(kBlock), 0, st, a); break;
    case 512: hipLaunchKernelGGL((pack_kernel<PACK, 512>), grid, dim3(kBlock), 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const PackArgs& a, hipStream_t st) { return launch_as<true>(a, st); }
hipError_t launch_unpack(const PackArgs& a, hipStream_t st) { return launch_as<false>(a, st); }

}  // namespace mtla
