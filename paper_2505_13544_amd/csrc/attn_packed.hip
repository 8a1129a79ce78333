// Decode attention over packed pages (packed.h) and, behind them, pages of the bf16 pool (gfx950).
//
// Eq. (with-rope), incremental case, per tile of 16 slots and 16 heads:
//     S^T[slot, head] = [C_hat | K_hat^R][slot, :] . [q~ | q^R][head, :]
//     O^T[col,  head] += C_hat^T[col, slot] . P^T[slot, head]
// Workgroup = (sequence, 16 heads, chunk of slots); where the packed slots end inside a chunk, what the chunk holds behind them is another workgroup's (open_piece:
// in one the open page's two barriers a step came on top, 47 us instead of 43 over 256 lengths from 256 to 2048 slots, 26 instead of 22.7 over 131071).
// A wavefront owns 128 latent columns (all 64 at r = 64): CG = r / 128 of them share the slots of a step (64 at r = 512, else 32), and the W / CG groups take
// different slots (W = 4; 8 for few long sequences at r = 512: packed_wide).  Every byte of the cache is loaded once per 16 heads.
//   logits   the codes go into the matrix cores as they are: v_mfma_scale_f32_16x16x128_f8f6f4 takes a lane's 32 codes of a slot with the block's power of
//            two, against the query as four planes of 6-bit floats (E2M3), each with a power of two per 32 columns of a head.  Plane after plane takes what
//            the ones before left: off by 2^-18 of the block's largest number after four (QueryPlanes).  64 cycles a tile, against 128 for two bf16 planes
//            behind a conversion of the codes.  The RoPE columns are bf16 on either side (two planes of the query).
//   weights  the group's shares of S^T meet in LDS; every wavefront makes the weights of its own tiles, as two bf16 planes, which all read.
//   values   the codes go through the wavefront's own LDS as they are and come back transposed by bytes; behind that they become bf16 pairs and operands.
//            Converted first, as bf16 rows, they were four times the bytes there: of a step's 1900 cycles LDS was busy with 960 (13 a 16-byte store of a wavefront).
// The packed cache is a third of the bytes of the bf16 one, so the matrix cores have time for the second plane of the weights: the output's error is its own
// rounding to bf16 (one plane would add as much again).  The normaliser sums the unrounded weights, and the chunks' sums meet as fp32: latents reach from 2^-124
// to 6 x 2^125, and a half, for all that it is half the bytes to join, holds 11 bits of numbers from 2^-14 to 65504.
//
// Between two barriers a wavefront forms the values of step i - 1, the weights of step i and the logits of step i + 1.  What bounds it, r = 512, 16 heads:
//   512 x 1024 slots (two workgroups a unit)  54 us, 3.8 TB/s: half the time VALU, a quarter MFMA, and the memory (50 us with all pages in L2)
//   256 x 1024 slots, chunks of 512           34 us, 3.0 TB/s: a step of 64 slots is 1.7 us alone on a unit, 2.4 beside another workgroup's
//   256 x 32 slots                            9 us: the launch, two reads that wait for each other (0.7 us each, 1.6 with all units reading), an open step (2.3)
// Tried and left: an equal share of all steps for each of 512 workgroups (ahead of the above 47 us instead of 49 where 256 lengths range from 256 to 2048 slots, but 37
// instead of 32 where all are 1024: its scan of the lengths is one more read to wait for); the open page in front of the packed ones, its rows asked for early (no gain).
#include "bounds.h"
#include "decode_schedule.h"
#include "lds_stream.h"
#include "mtla_device.h"
#include "packed.h"

#include <type_traits>

namespace mtla {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t* lds_int2_ptr;
typedef uint32_t u32x6_t __attribute__((ext_vector_type(6)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x32_t __attribute__((ext_vector_type(32)));

constexpr int kTile = kPackTile;   // slots of an operand tile
constexpr float kRebase = 40.f;

template <int R_, int DR_, int W_>
struct PackCfg {
  static constexpr int R = R_, DR = DR_, W = W_;      // W wavefronts
  static constexpr int E = R + DR;
  static constexpr int CG = R >= 128 ? R / 128 : 1;   // wavefronts that share a group's slots
  static constexpr int SG = W / CG;                   // groups
  static constexpr int RW = R / CG;                   // latent columns of a wavefront: 128, or 64
  static constexpr int NB = RW / kPackBlock;          // blocks of a slot: one in each of the lanes g < NB
  static constexpr int DRW = DR / CG;                 // RoPE columns of a wavefront: 8 to 64
  static constexpr int KR = (DRW + 31) / 32;          // K steps over them
  static constexpr int MT = RW / 16;                  // column tiles of its sums
  static constexpr int PC = RW / 8;                   // 16-byte pieces of a parked row
  static constexpr int TL = CG == 4 ? 4 : 2;          // tiles of a group's step
  static constexpr int STEP = TL * kTile;
  static constexpr int U = TL / CG;                   // of them a wavefront's own: it makes their weights
  // a wavefront's rows in LDS: the codes of a step and behind them the scales, in two places, or bf16 rows of two tiles
  static constexpr int tile_bytes = NB * kTile * 16, place_bytes = TL * (tile_bytes + kWave * 4);
  static constexpr int wave_bytes = 2 * place_bytes > 2 * kTile * RW * 2 ? 2 * place_bytes : 2 * kTile * RW * 2;
  static constexpr size_t park_bytes = (size_t)W * wave_bytes;
  static constexpr size_t share_bytes = (size_t)SG * TL * (CG - 1) * kWave * 16;            // [group][tile][other wavefront][lane][4 slots]
  static constexpr size_t weight_bytes = CG > 1 ? (size_t)SG * TL * kWave * 16 : 0;         // [group][pair of tiles][plane][lane][4 slots of either tile]
  static constexpr size_t loop_bytes = park_bytes + 2 * share_bytes + 2 * weight_bytes;
  static constexpr int OS = R + 4;                                                          // row stride of the groups' sums when they are merged (floats)
  static constexpr size_t merge_bytes = SG > 1 ? (size_t)SG * 16 * OS * 4 : 0;
  static constexpr size_t body_bytes = loop_bytes > merge_bytes ? loop_bytes : merge_bytes;
  static constexpr size_t top_bytes = (size_t)W * 16 * 4;                                   // [wavefront][head]
  static constexpr size_t lds_bytes = body_bytes + 2 * top_bytes + 2 * W * 4;               // and whether a wavefront's weights need another reference
};

// Where a wavefront's and a lane's part of everything is: constant for the kernel.
template <class C>
struct LaneMap {
  int lane, l16, g, wv, cg, sg;
  int col;                      // the lane's first latent column (of a lane that has none: another's)
  int rope[C::KR];              // its first RoPE column in a K step (likewise)
  bool has_lat, has_rope[C::KR];
  // a step's tile that is this wavefront's h-th: its own U first, and h = 0, 1 and h = 2, 3 a pair of neighbours
  __device__ __forceinline__ int tile(int h) const { return C::CG == 1 ? h : (C::U * cg) ^ h; }
  __device__ __forceinline__ int pair(int k) const { return tile(2 * k) >> 1; }
  __device__ __forceinline__ LaneMap(int lane_, int wv_) : lane(lane_), l16(lane_ & 15), g(lane_ >> 4), wv(wv_), cg(wv_ % C::CG), sg(wv_ / C::CG) {
    has_lat = g < C::NB;
    col = cg * C::RW + kPackBlock * (g % C::NB);
#pragma unroll
    for (int t = 0; t < C::KR; ++t) {
      const int c = 32 * t + 8 * g;
      has_rope[t] = c < C::DRW;
      rope[t] = cg * C::DRW + (has_rope[t] ? c : 0);
    }
  }
};

// The table entries of 64 pages, one a lane, clamped into the pool that they belong to.  A lookup is a
// v_readlane: as a load it would be one more in flight in front of the tile's own, and every wait for a tile one for all of them.
struct ChunkPages {
  int at, entry;
};

template <class C>
struct PackedTile {  // as loaded
  u32x4_t code;
  uint32_t scale;    // of four slots (a byte would be widened where the registers go round, a wait for a load just issued)
  u32x4_t xr[C::KR];
};
template <class C>
struct OpenTile {
  u32x4_t xc[4];     // 32 latents
  u32x4_t xr[C::KR];
};
struct Source {  // of one sequence
  const uint8_t* codes;
  const uint8_t* scales;
  const uint16_t* keys;
  const uint16_t* lat;   // the bf16 pool
  const uint16_t* key;
  const int32_t* table;  // the sequence's rows of both tables
  const int32_t* table4;
  int n_packed, n_pages, n_pages4, shift, last_entry;
};

// (Both tables are read: which one counts need not be known yet.)
struct PageEntries {
  int packed, open;
  __device__ __forceinline__ void load(const Source& s, int at, int lane) {
    const int k = at + lane < s.last_entry ? at + lane : s.last_entry;
    packed = s.table4[k];
    open = s.table[k];
  }
};
__device__ __forceinline__ ChunkPages chunk_pages(const PageEntries& e, const Source& s, int at, int lane) {
  const int k = at + lane < s.last_entry ? at + lane : s.last_entry;
  const bool packed = k < s.n_packed;
  return ChunkPages{at, clamp_page(packed ? e.packed : e.open, packed ? s.n_pages4 : s.n_pages)};
}
// Tile of the pool (in units of 16 slots) that holds slot s0 (wavefront-uniform, a multiple of 16).
__device__ __forceinline__ uint32_t pool_tile(const ChunkPages& p, const Source& s, int s0) {
  const int e = __builtin_amdgcn_readlane(p.entry, (s0 >> s.shift) - p.at);
  return ((uint32_t)e << (s.shift - 4)) + (uint32_t)((s0 & ((1 << s.shift) - 1)) >> 4);
}

template <class C>
__device__ __forceinline__ void load_tile(PackedTile<C>& t, const Source& s, uint32_t tile, const LaneMap<C>& m) {
  const uint32_t unit = (uint32_t)(m.col / kPackBlock) * kTile + m.l16;
  t.code = *reinterpret_cast<const u32x4_t*>(s.codes + (size_t)tile * packed_code_bytes(C::R) + unit * 16);
  t.scale = *reinterpret_cast<const uint32_t*>(s.scales + (size_t)tile * packed_scale_bytes(C::R) + (unit & ~3u));
#pragma unroll
  for (int k = 0; k < C::KR; ++k)
    t.xr[k] = *reinterpret_cast<const u32x4_t*>(s.keys + (size_t)tile * (packed_key_bytes(C::DR) / 2) + ((uint32_t)(m.rope[k] / 8) * kTile + m.l16) * 8);
}
template <class C>
__device__ __forceinline__ void load_tile(OpenTile<C>& t, const Source& s, uint32_t tile, const LaneMap<C>& m) {
  const size_t row = (size_t)tile * kTile + m.l16;
#pragma unroll
  for (int i = 0; i < 4; ++i) t.xc[i] = *reinterpret_cast<const u32x4_t*>(s.lat + row * C::R + m.col + 8 * i);
#pragma unroll
  for (int k = 0; k < C::KR; ++k) t.xr[k] = *reinterpret_cast<const u32x4_t*>(s.key + row * C::DR + m.rope[k]);
}

// Slots that are none of the sequence's count as zeros, whatever their bytes are.  `live`: of the tile's slots.
template <class C>
__device__ __forceinline__ void drop(PackedTile<C>& t, int live, const LaneMap<C>& m) {
  if (m.l16 >= live) {
    t.code = u32x4_t{0, 0, 0, 0};
    t.scale = 0x7f7f7f7fu;
#pragma unroll
    for (int k = 0; k < C::KR; ++k) t.xr[k] = u32x4_t{0, 0, 0, 0};
  }
}
template <class C>
__device__ __forceinline__ void drop(OpenTile<C>& t, int live, const LaneMap<C>& m) {
  if (m.l16 >= live) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t.xc[i] = u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < C::KR; ++k) t.xr[k] = u32x4_t{0, 0, 0, 0};
  }
}

// Heads past the last one are copies of it and never stored.
template <class C>
__device__ __forceinline__ const uint16_t* query_row(const uint16_t* rows, int n_heads, const LaneMap<C>& m) {
  return rows + (size_t)(m.l16 < n_heads ? m.l16 : n_heads - 1) * C::E;
}
// The RoPE columns: two bf16 planes; a lane without a column holds zeros.
template <class C>
struct QueryRope {
  u32x4_t hi[C::KR], lo[C::KR];
  __device__ __forceinline__ void load(const uint16_t* rows, size_t plane, int n_heads, const LaneMap<C>& m) {
#pragma unroll
    for (int k = 0; k < C::KR; ++k) {
      const uint16_t* from = query_row<C>(rows, n_heads, m) + C::R + m.rope[k];
      const uint32_t mask = m.has_rope[k] ? 0xffffffffu : 0u;
      hi[k] = *reinterpret_cast<const u32x4_t*>(from) & mask;
      lo[k] = *reinterpret_cast<const u32x4_t*>(from + plane) & mask;
    }
  }
};
// The latent columns, for bf16 rows: the planes as they are.
template <class C>
struct QueryRows {
  u32x4_t hi[4], lo[4];
  __device__ __forceinline__ void load(const uint16_t* rows, size_t plane, int n_heads, const LaneMap<C>& m) {
    const uint32_t mask = m.has_lat ? 0xffffffffu : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t* from = query_row<C>(rows, n_heads, m) + m.col + 8 * i;
      hi[i] = *reinterpret_cast<const u32x4_t*>(from) & mask;
      lo[i] = *reinterpret_cast<const u32x4_t*>(from + plane) & mask;
    }
  }
};
// The latent columns, for codes: a lane's 32 numbers (a head's block) as four planes of E2M3 numbers (steps of 1/8 below 2, 1/4 below 4, 1/2 up to 7.5).  With
// s the smallest power of two of which the largest is at most 7.5 times: the first plane is off by s / 4 at most; the second, in units of s / 16, sees
// numbers up to 4 and is off by 1/8 of its unit, s / 128; so on in units of s / 512 and s / 2^14: s 2^-17, the largest number times 2^-18.9, at the end.
template <class C>
struct QueryPlanes {
  u32x6_t plane[4];
  uint32_t scale;  // the planes' exponents, a byte each
  __device__ __forceinline__ void make(const QueryRows<C>& q) {
    f32x16_t even, odd;
    float top = 0.f, nan = 0.f;  // (fmaxf drops a NaN; it and an infinity make the block's logits NaN)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4_t hi = q.hi[i], lo = q.lo[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = __uint_as_float(hi[j] << 16) + __uint_as_float(lo[j] << 16), y = __uint_as_float(hi[j] & 0xffff0000u) + __uint_as_float(lo[j] & 0xffff0000u);
        top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
        nan = fmaf(0.f, x, fmaf(0.f, y, nan));
        even[4 * i + j] = x;
        odd[4 * i + j] = y;
      }
    }
    const uint32_t tb = __float_as_uint(top);
    int e = (int)(tb >> 23) - 2 + ((tb & 0x7fffffu) > 0x700000u ? 1 : 0);
    e = nan == 0.f ? (e < 16 ? 16 : e) : 255;
    constexpr int kDown[4] = {0, 4, 9, 14};
    scale = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t ep = (uint32_t)(e == 255 ? 255 : e - kDown[p]);
      scale |= ep << (8 * p);
      const float unit = __uint_as_float(ep << 23);
      // packed number 2i is the first operand's i-th, 2i + 1 the second's
      u32x6_t code = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, unit);
      asm volatile("" : "+v"(code) : "v"(even), "v"(odd), "v"(unit));  // (else the compiler lets the result overlap the operands, which the instruction reads to its end)
      plane[p] = code;
      if (p < 3) {
        f32x32_t back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(code, unit);
        asm volatile("" : "+v"(back) : "v"(code), "v"(unit));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          even[i] -= back[2 * i];
          odd[i] -= back[2 * i + 1];
        }
      }
    }
  }
};

// The state of one wavefront and what it does with it.
template <class C>
struct Worker {
  static constexpr int MT = C::MT, CG = C::CG, U = C::U, TL = C::TL;
  const LaneMap<C>& m;
  unsigned char* smem;
  int k1;                       // end of the slots that are attended here
  float m_ref;                  // head l16's softmax reference, the same in all wavefronts of the group
  float l_run;                  // normaliser, of the lane's slots of this wavefront's weights only
  float4_t o[MT];               // sums over this wavefront's columns
  float4_t sh[TL];              // this wavefront's share of a step's logits
  float4_t sv[U], pw[U];        // its own tiles' logits (log2 units: the query is pre-scaled) and weights
  struct Weights {              // two tiles' weights as operands
    bf16x8_t hi, lo;
  };
  Weights own;                  // CG = 1: those of the step

  __device__ __forceinline__ Worker(const LaneMap<C>& m_, unsigned char* smem_) : m(m_), smem(smem_), k1(0), m_ref(-INFINITY), l_run(0.f) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ float4_t* shares(int par) const {
    return reinterpret_cast<float4_t*>(smem + C::park_bytes + par * C::share_bytes) + m.sg * (TL * (CG - 1) * kWave) + m.lane;
  }
  __device__ __forceinline__ u32x4_t* weights(int par) const {
    return reinterpret_cast<u32x4_t*>(smem + C::park_bytes + 2 * C::share_bytes + par * C::weight_bytes) + m.sg * TL * kWave + m.lane;
  }
  __device__ __forceinline__ float* tops() const { return reinterpret_cast<float*>(smem + C::body_bytes); }
  __device__ __forceinline__ int* flags(int par) const { return reinterpret_cast<int*>(smem + C::body_bytes + 2 * C::top_bytes) + par * C::W; }

  __device__ __forceinline__ void barrier() const {  // of the wavefronts that share slots
    if constexpr (CG > 1) __syncthreads();
  }

  // ---- logits of a step: rows in a lane's registers against the query
  __device__ __forceinline__ void rope_logits(const u32x4_t (&xr)[C::KR], const QueryRope<C>& q, int h) {
#pragma unroll
    for (int k = 0; k < C::KR; ++k) {
      const bf16x8_t x = __builtin_bit_cast(bf16x8_t, xr[k]);
      sh[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8_t, q.hi[k]), sh[h], 0, 0, 0);
      sh[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8_t, q.lo[k]), sh[h], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void logits(const PackedTile<C> (&t)[TL], const QueryPlanes<C>& q, const QueryRope<C>& qr) {
#pragma unroll
    for (int h = 0; h < TL; ++h) {
      const i32x8_t a = {(int)t[h].code[0], (int)t[h].code[1], (int)t[h].code[2], (int)t[h].code[3], 0, 0, 0, 0};
      const int sa = (int)(t[h].scale >> (8 * (m.l16 & 3)));  // (the lowest byte counts)
      auto plane = [&](auto p_, float4_t c) __attribute__((always_inline)) {
        constexpr int p = decltype(p_)::value;
        const u32x6_t b = q.plane[p];
        const i32x8_t bv = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], (int)b[4], (int)b[5], 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, bv, c, /*A: E2M1*/ 4, /*B: E2M3*/ 2, 0, sa, p, (int)q.scale);
      };
      sh[h] = plane(std::integral_constant<int, 0>{}, float4_t{0.f, 0.f, 0.f, 0.f});
      sh[h] = plane(std::integral_constant<int, 1>{}, sh[h]);
      sh[h] = plane(std::integral_constant<int, 2>{}, sh[h]);
      sh[h] = plane(std::integral_constant<int, 3>{}, sh[h]);
      rope_logits(t[h].xr, qr, h);
    }
  }
  __device__ __forceinline__ void logits(const OpenTile<C> (&t)[TL], const QueryRows<C>& q, const QueryRope<C>& qr, int base) {
#pragma unroll
    for (int h = 0; h < TL; ++h) {
      sh[h] = float4_t{0.f, 0.f, 0.f, 0.f};
      if (base + m.tile(h) * kTile >= k1) continue;  // (uniform: a page of a sequence is half empty)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8_t x = __builtin_bit_cast(bf16x8_t, t[h].xc[i]);
        sh[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8_t, q.hi[i]), sh[h], 0, 0, 0);
        sh[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8_t, q.lo[i]), sh[h], 0, 0, 0);
      }
      rope_logits(t[h].xr, qr, h);
    }
  }
  template <class Tile>
  __device__ __forceinline__ void drop_dead(Tile (&t)[TL], int base) const {
    if (base + C::STEP > k1) {  // (uniform; the last step's at most)
#pragma unroll
      for (int h = 0; h < TL; ++h) drop<C>(t[h], k1 - base - m.tile(h) * kTile, m);
    }
  }

  // ---- the group's shares meet
  __device__ __forceinline__ void put_shares(int par) const {
    float4_t* to = shares(par);
#pragma unroll
    for (int h = U; h < TL; ++h) to[(m.tile(h) * (CG - 1) + h / U - 1) * kWave] = sh[h];
  }
  // this wavefront's own tiles (its share of them is still in `sh`)
  __device__ __forceinline__ void get_logits(int par, float4_t (&to)[U]) const {
    const float4_t* from = shares(par);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to[u] = sh[u];
#pragma unroll
      for (int w = 0; w < CG - 1; ++w) to[u] += from[(m.tile(u) * (CG - 1) + w) * kWave];
    }
  }
  __device__ __forceinline__ int any_flag(int par) const {
    if constexpr (CG == 1) return 0;
    const int4* at = reinterpret_cast<const int4*>(flags(par));
    int4 f = at[0];
    if constexpr (C::W == 8) f = make_int4(f.x | at[1].x, f.y | at[1].y, f.z | at[1].z, f.w | at[1].w);
    return f.x | f.y | f.z | f.w;
  }

  // ---- weights of a step, relative to a reference that is fixed at the first live step and moved only where a step tops it by more than 2^kRebase
  __device__ __forceinline__ float top() const {
    float t = fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[0][2], sv[0][3]));
    if constexpr (U == 2) t = fmaxf(t, fmaxf(fmaxf(sv[1][0], sv[1][1]), fmaxf(sv[1][2], sv[1][3])));
    return t;
  }
  __device__ __forceinline__ void put_weights(int par) {
    const float ref = m_ref == -INFINITY ? 0.f : m_ref;
    u32x4_t h = {}, l = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int v = 0; v < 4; ++v) pw[u][v] = __builtin_amdgcn_exp2f(sv[u][v] - ref);
      split_bf16x2(pw[u][0], pw[u][1], hi[0], lo[0]);
      split_bf16x2(pw[u][2], pw[u][3], hi[1], lo[1]);
      if constexpr (CG == 1) {
        h[2 * u] = hi[0], h[2 * u + 1] = hi[1];
        l[2 * u] = lo[0], l[2 * u + 1] = lo[1];
      } else {
        const int t = m.tile(u);
        uint2* to = reinterpret_cast<uint2*>(weights(par) + (t >> 1) * (2 * kWave)) + (t & 1);
        to[0] = make_uint2(hi[0], hi[1]);
        to[2 * kWave] = make_uint2(lo[0], lo[1]);
      }
    }
    if constexpr (CG == 1) {
      own.hi = __builtin_bit_cast(bf16x8_t, h);
      own.lo = __builtin_bit_cast(bf16x8_t, l);
    }
  }
  __device__ __forceinline__ void add_weights() {
#pragma unroll
    for (int u = 0; u < U; ++u) l_run += (pw[u][0] + pw[u][1]) + (pw[u][2] + pw[u][3]);
  }
  __device__ __forceinline__ void move_ref(float to) {
    const float alpha = m_ref == to ? 1.f : __builtin_amdgcn_exp2f(m_ref - to);
    m_ref = to;
    l_run *= alpha;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] *= alpha;
  }
  // Logits `sv` of the step at `base` -> weights, in the place `par`.  CG = 1: the reference moves at once (everything formed with the old one is in `o`);
  // else a wavefront that sees that it has to says so, and settle() forms the group's weights again, behind a barrier.
  __device__ __forceinline__ void make_weights(int par, int base) {
    if (base + C::STEP > k1) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (base + m.tile(u) * kTile + 4 * m.g + v >= k1) sv[u][v] = -INFINITY;
    }
    const float t = top();
    const bool moves = m_ref == -INFINITY ? t > -INFINITY : t - m_ref > kRebase;
    if constexpr (CG == 1) {
      if (__any(moves)) move_ref(fmaxf(m_ref, quarter_reduce(t, LaneMax())));
    } else {
      flags(par)[m.wv] = __any(moves) ? 1 : 0;
    }
    put_weights(par);
  }
  // Behind the barrier after make_weights(par), with any_flag(par): true weights in their place.  All wavefronts of the workgroup take the same way.
  __device__ __forceinline__ bool settle(int par, int flag) {  // whether they changed
    if constexpr (CG > 1) {
      if (__builtin_amdgcn_readfirstlane(flag)) {
        const float t = quarter_reduce(top(), LaneMax());
        if (m.g == 0) tops()[m.wv * 16 + m.l16] = t;
        __syncthreads();
        float to = m_ref;
#pragma unroll
        for (int w = 0; w < CG; ++w) to = fmaxf(to, tops()[(m.sg * CG + w) * 16 + m.l16]);
        move_ref(to);
        put_weights(par);
        __syncthreads();
        add_weights();
        return true;
      }
    }
    add_weights();
    return false;
  }
  __device__ __forceinline__ Weights get_weights(int par, int pair) const {
    if constexpr (CG == 1) return own;
    return Weights{__builtin_bit_cast(bf16x8_t, weights(par)[pair * 2 * kWave]), __builtin_bit_cast(bf16x8_t, weights(par)[pair * 2 * kWave + kWave])};
  }

  // ---- values of codes.  A tile's codes lie in LDS as in memory, [block][slot][16 bytes].  A transposing read of bytes gives lane (l16, g) byte l16, that is
  // columns 2 l16 and 2 l16 + 1 of a block, of the eight slots whose weights it holds; they become bf16 pairs (v_cvt_scalef32_pk_bf16_fp4, exact; of the scale
  // operand only the exponent counts, so a shift brings a slot's byte there), and two slots' pairs one dword of either column's operand.
  // Column of o[2 nb + par][i] of lane (l16, g): 32 nb + 8 g + 2 i + par.
  __device__ __forceinline__ unsigned char* codes_at(int par) const { return smem + m.wv * C::wave_bytes + par * C::place_bytes; }
  __device__ __forceinline__ void park(const PackedTile<C> (&t)[TL], int par) const {
    unsigned char* to = codes_at(par);
#pragma unroll
    for (int h = 0; h < TL; ++h) {
      if (m.has_lat) *reinterpret_cast<u32x4_t*>(to + m.tile(h) * C::tile_bytes + m.lane * 16) = t[h].code;
      // [tile][block][slot], exponents of floats
      reinterpret_cast<uint32_t*>(to + TL * C::tile_bytes)[m.tile(h) * kWave + m.lane] = (t[h].scale >> (8 * (m.l16 & 3))) << 23;
    }
  }
  struct CodeRows {  // of a block of two tiles
    i32x2_t code;
    u32x4_t scale[2];
  };
  __device__ __forceinline__ void get_codes(CodeRows& x, int par, int pair, int nb) const {
    const unsigned char* from = codes_at(par);
    const int row = m.l16 >> 1;
    const unsigned char* at = from + (2 * pair + (row >> 2)) * C::tile_bytes + (4 * m.g + (row & 3)) * 16 + 8 * (m.l16 & 1);
    x.code = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2_ptr)(const int*)(at + nb * (kTile * 16)));
#pragma unroll
    for (int h = 0; h < 2; ++h)
      x.scale[h] = *reinterpret_cast<const u32x4_t*>(from + TL * C::tile_bytes + ((2 * pair + h) * kWave + nb * kTile + 4 * m.g) * 4);
  }
  __device__ __forceinline__ void add_codes(const CodeRows& x, const Weights& p, int nb) {
    u32x4_t even, odd;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t c = (uint32_t)x.code[h];
      const u32x4_t e = x.scale[h];
      const uint32_t s0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, __uint_as_float(e[0]), 0));
      const uint32_t s1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, __uint_as_float(e[1]), 1));
      const uint32_t s2 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, __uint_as_float(e[2]), 2));
      const uint32_t s3 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, __uint_as_float(e[3]), 3));
      even[2 * h] = __builtin_amdgcn_perm(s1, s0, 0x05040100u);
      odd[2 * h] = __builtin_amdgcn_perm(s1, s0, 0x07060302u);
      even[2 * h + 1] = __builtin_amdgcn_perm(s3, s2, 0x05040100u);
      odd[2 * h + 1] = __builtin_amdgcn_perm(s3, s2, 0x07060302u);
    }
    const bf16x8_t a = __builtin_bit_cast(bf16x8_t, even), b = __builtin_bit_cast(bf16x8_t, odd);
    o[2 * nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.hi, o[2 * nb], 0, 0, 0);
    o[2 * nb + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, p.hi, o[2 * nb + 1], 0, 0, 0);
    o[2 * nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.lo, o[2 * nb], 0, 0, 0);
    o[2 * nb + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, p.lo, o[2 * nb + 1], 0, 0, 0);
  }
  __device__ __forceinline__ void add_value(int mt, bf16x8_t x) {
    o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, own.hi, o[mt], 0, 0, 0);
    o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, own.lo, o[mt], 0, 0, 0);
  }

  // ---- values of bf16 rows, through the wavefront's own LDS too: a block's even columns in front of its odd ones (the order of the sums).  Piece p of row i lies at
  // place p ^ f(i): the 16 rows' writes of one piece go to all banks (f takes 16 values), and so do the transposing reads, 32 bytes of each of 8 rows.
  __device__ __forceinline__ static int place(int row) { return (((row & 7) << 1) | ((row >> 3) & 1)) & (C::PC - 1); }
  __device__ __forceinline__ void park_rows(const OpenTile<C> (&t)[TL], int k) const {
#pragma unroll
    for (int h = 2 * k; h < 2 * k + 2; ++h) park_row(t[h].xc, m.tile(h) & 1);
  }
  __device__ __forceinline__ void park_row(const u32x4_t (&x)[4], int h) const {
    if (m.has_lat) {
      unsigned char* to = smem + m.wv * C::wave_bytes + (h * kTile + m.l16) * (C::RW * 2);
      const int p0 = (m.g % C::NB) * 4, f = place(m.l16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4_t &a = x[2 * (i & 1)], &b = x[2 * (i & 1) + 1];
        const uint32_t sel = i < 2 ? 0x05040100u : 0x07060302u;
        *reinterpret_cast<u32x4_t*>(to + 16 * ((p0 + i) ^ f)) = u32x4_t{__builtin_amdgcn_perm(a[1], a[0], sel), __builtin_amdgcn_perm(a[3], a[2], sel),
                                                                       __builtin_amdgcn_perm(b[1], b[0], sel), __builtin_amdgcn_perm(b[3], b[2], sel)};
      }
    }
  }
  __device__ __forceinline__ void add_rows() {
    const int row = 4 * m.g + (m.l16 >> 2), f = place(row);
    const unsigned char* at = smem + m.wv * C::wave_bytes + row * (C::RW * 2) + 8 * (m.l16 & 1);
    const int piece = (m.l16 >> 1) & 1;  // of the two that a column tile has
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const unsigned char* from = at + 16 * ((2 * mt + piece) ^ f);
      const short4_t c0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(const short*)from);
      const short4_t c1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(const short*)(from + kTile * C::RW * 2));
      add_value(mt, __builtin_bit_cast(bf16x8_t, (short8_t)__builtin_shufflevector(c0, c1, 0, 1, 2, 3, 4, 5, 6, 7)));
    }
  }
};

// The tiles of a step of this wavefront's group, from slot `base` on; slots past `last` become copies of its tile.
template <class C, int H0 = 0, int H1 = C::TL, class Tile>
__device__ __forceinline__ void load_step(Tile (&t)[C::TL], const Source& s, ChunkPages& pages, int base, int last, const LaneMap<C>& m) {
  constexpr int kAll = C::STEP * C::SG;
  const int first = base - C::STEP * m.sg, to = ((first + kAll - 1 < last ? first + kAll - 1 : last) >> s.shift) - pages.at;
  if (__builtin_amdgcn_readfirstlane(to) >= kWave) {  // (the next 64 pages)
    pages.at = __builtin_amdgcn_readfirstlane((first < last ? first : last) >> s.shift);
    PageEntries e;
    e.load(s, pages.at, m.lane);
    pages = chunk_pages(e, s, pages.at, m.lane);
  }
#pragma unroll
  for (int h = H0; h < H1; ++h) {
    const int s0 = base + m.tile(h) * kTile, s1 = s0 < last ? s0 : last;
    load_tile<C>(t[h], s, pool_tile(pages, s, __builtin_amdgcn_readfirstlane(s1)), m);
  }
  __builtin_amdgcn_sched_barrier(0);  // in this order everywhere: the waits count the loads issued since
}

// Packed slots [k0, k1), k0 a multiple of 16, k0 < k1.  Between two barriers: values of step i - 1, weights of step i and logits of step i + 1 (of a step past the
// last one: of copies, and nobody reads them).  The codes of step i + 1 take the place of those of step i - 1, behind their reads.
template <class C>
__device__ __forceinline__ void stream_packed(Worker<C>& w, const Source& s, ChunkPages& pages, const QueryRows<C>& rows, const QueryRope<C>& qr, int k0,
                                              int k1) {
  const LaneMap<C>& m = w.m;
  constexpr int kAll = C::STEP * C::SG;  // slots of a step of all groups
  w.k1 = k1;
  const int first = k0 + C::STEP * m.sg, last = (k1 - 1) & ~(kTile - 1), n = (k1 - k0 + kAll - 1) / kAll;
  PackedTile<C> t[C::TL];
  load_step<C>(t, s, pages, first, last, m);
  QueryPlanes<C> q;
  q.make(rows);  // (1.6 us: the first step's bytes come in meanwhile)
  auto logits = [&](int step) __attribute__((always_inline)) {
    w.drop_dead(t, first + step * kAll);
    w.logits(t, q, qr);
    w.park(t, step & 1);
    load_step<C>(t, s, pages, first + (step + 1) * kAll, last, m);
  };
  // A block (of two tiles) after the other, the reads of the next two under way: left to itself the compiler puts every read in front of its use, ten waits a step.
  auto values = [&](int step) __attribute__((always_inline)) {
    constexpr int NB = C::NB, kBlocks = NB * C::TL / 2, kAhead = 2;
    const int par = step & 1, flag = w.any_flag(par);
    typename Worker<C>::Weights p = w.get_weights(par, 0), p_next = p;
    typename Worker<C>::CodeRows x[kAhead + 1];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) w.get_codes(x[j], par, j / NB, j % NB);
    __builtin_amdgcn_sched_barrier(0);
    if (w.settle(par, flag)) p = w.get_weights(par, 0);
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      const int next = j + kAhead;
      if (next < kBlocks) {
        w.get_codes(x[next % (kAhead + 1)], par, next / NB, next % NB);
        if (next % NB == 0) p_next = w.get_weights(par, next / NB);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (j > 0 && j % NB == 0) p = p_next;
      w.add_codes(x[j % (kAhead + 1)], p, j % NB);
    }
  };
  auto weights = [&](int step) __attribute__((always_inline)) {
    w.get_logits(step & 1, w.sv);
    w.make_weights(step & 1, first + step * kAll);
  };
  auto meet = [&](int step) __attribute__((always_inline)) {
    w.put_shares(step & 1);
    w.barrier();
  };
  logits(0);
  meet(0);
  for (int i = 0; i < n; ++i) {
    if (i > 0) values(i - 1);
    weights(i);
    logits(i + 1);
    meet(i + 1);
  }
  values(n - 1);
}

// Slots [k0, k1) of the bf16 pool, k0 a multiple of 16, k0 < k1: the few behind the packed ones, one step after the other.
template <class C>
struct OpenStep {
  OpenTile<C> t[C::TL];
  QueryRows<C> q;
};
template <class C, int H0, int H1>
__device__ __forceinline__ void load_open(OpenStep<C>& o, const Source& s, ChunkPages& pages, int base, int k1, const LaneMap<C>& m) {
  load_step<C, H0, H1>(o.t, s, pages, base + C::STEP * m.sg, (k1 - 1) & ~(kTile - 1), m);
}
template <class C>
__device__ __forceinline__ void stream_open(Worker<C>& w, const Source& s, ChunkPages& pages, OpenStep<C>& o, const QueryRope<C>& qr, int k0, int k1) {
  const LaneMap<C>& m = w.m;
  constexpr int kAll = C::STEP * C::SG;
  w.k1 = k1;
  for (int at = k0; at < k1; at += kAll) {
    const int base = at + C::STEP * m.sg;
    const bool more = at + kAll < k1;
    w.drop_dead(o.t, base);
    w.logits(o.t, o.q, qr, base);
    w.put_shares(0);
    const auto live = [&](int k) { return base + 2 * m.pair(k) * kTile < k1; };
    if (live(0)) w.park_rows(o.t, 0);
    if (more) load_open<C, 0, 2>(o, s, pages, at + kAll, k1, m);
    w.barrier();
    w.get_logits(0, w.sv);
    w.make_weights(0, base);
    w.barrier();
    w.settle(0, w.any_flag(0));
    if (live(0)) {
      w.own = w.get_weights(0, m.pair(0));
      w.add_rows();
    }
    if constexpr (C::TL > 2) {
      if (live(1)) w.park_rows(o.t, 1);
      if (more) load_open<C, 2, C::TL>(o, s, pages, at + kAll, k1, m);
      if (live(1)) {
        w.own = w.get_weights(0, m.pair(1));
        w.add_rows();
      }
    }
  }
}

struct Run {  // slots [k0, k1) of sequence b, k0 < k1, k0 a multiple of 16: all of them packed, or none
  int b, k0, k1, piece;
  int packed;  // the sequence's slots that lie in packed pages
};

// What a run asks for ahead of everything that it has to know first.
template <class C>
struct RunHead {
  PageEntries entries;
  QueryRope<C> qr;
  QueryRows<C> q;
};
template <class C>
__device__ __forceinline__ Source source_of(const AttnPackedArgs& a, int b) {
  Source s;
  s.codes = a.pk.codes;
  s.scales = a.pk.scales;
  s.keys = a.pk.keys;
  s.lat = reinterpret_cast<const uint16_t*>(a.at.lat);
  s.key = reinterpret_cast<const uint16_t*>(a.at.key);
  s.table = a.at.pages.table + (size_t)b * a.at.pages.max_pages;
  s.table4 = a.pk.table + (size_t)b * a.at.pages.max_pages;
  s.n_pages = a.at.pages.n_pages;
  s.n_pages4 = a.pk.n_pages;
  s.shift = a.at.pages.shift;
  s.last_entry = a.at.pages.max_pages - 1;
  return s;
}
template <class C>
__device__ __forceinline__ const uint16_t* query_rows(const AttnArgs& at, int b, int h0) {
  return reinterpret_cast<const uint16_t*>(at.qcat) + ((size_t)b * at.n_heads + h0) * C::E;
}
template <class C>
__device__ __forceinline__ void load_head(RunHead<C>& h, const AttnPackedArgs& a, const Source& s, int b, int k0, const LaneMap<C>& m, int h0, int heads) {
  h.entries.load(s, k0 >> s.shift, m.lane);
  h.q.load(query_rows<C>(a.at, b, h0), a.at.q_plane, heads, m);
  h.qr.load(query_rows<C>(a.at, b, h0), a.at.q_plane, heads, m);
}

template <class C>
__device__ __forceinline__ void attend_run(const AttnPackedArgs& a, const Run& run, RunHead<C>& head, Source& s, const LaneMap<C>& m, int h0, int heads, unsigned char* smem) {
  constexpr int R = C::R;
  const AttnArgs& at = a.at;
  const int k0 = run.k0, k1 = run.k1, tid = threadIdx.x, wv = m.wv;
  const QueryRope<C>& qr = head.qr;
  Worker<C> w(m, smem);
  ChunkPages pages = chunk_pages(head.entries, s, k0 >> s.shift, m.lane);
  if (run.packed > k0) {
    stream_packed<C>(w, s, pages, head.q, qr, k0, k1);
  } else {
    OpenStep<C> o;
    o.q.load(query_rows<C>(at, run.b, h0), at.q_plane, heads, m);
    load_open<C, 0, C::TL>(o, s, pages, k0, k1, m);
    stream_open<C>(w, s, pages, o, qr, k0, k1);
  }

  // ---- normalisers and references of the groups
  float* part_l = w.tops();                            // [wavefront][head]
  float* refs = part_l + C::W * 16;                    // [group][head]
  w.barrier();  // (the tops' place may have been in use)
  const float l_wave = quarter_reduce(w.l_run, LaneSum());
  if (m.g == 0) part_l[wv * 16 + m.l16] = l_wave;
  if (m.g == 0 && m.cg == 0) refs[m.sg * 16 + m.l16] = w.m_ref;
  const size_t piece = run.piece;
  if constexpr (C::SG == 1) {
    __syncthreads();
    // ---- the chunk's partial: lane holds head l16, columns 32nb + 8g .. + 7
    float l = 0.f;
#pragma unroll
    for (int cg = 0; cg < C::CG; ++cg) l += part_l[cg * 16 + m.l16];
    if (m.l16 < heads) {
      const size_t oh = piece * at.n_heads + h0 + m.l16, col = oh * R + m.cg * C::RW + 8 * m.g;
#pragma unroll
      for (int nb = 0; nb < C::NB; ++nb) {
        const float4_t a0 = w.o[2 * nb], a1 = w.o[2 * nb + 1];
        *reinterpret_cast<float4_t*>(at.part_o + col + 32 * nb) = float4_t{a0[0], a1[0], a0[1], a1[1]};
        *reinterpret_cast<float4_t*>(at.part_o + col + 32 * nb + 4) = float4_t{a0[2], a1[2], a0[3], a1[3]};
      }
      if (wv == 0 && m.g == 0) *reinterpret_cast<float2*>(at.part_ml + oh * 2) = make_float2(w.m_ref, l);
    }
  } else {
    // ---- the groups' sums meet
    float* sums = reinterpret_cast<float*>(smem);  // [group][head][OS]
    __syncthreads();  // the parked rows' place
    float* to = sums + (m.sg * 16 + m.l16) * C::OS + m.cg * C::RW + 8 * m.g;
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb) {
      const float4_t a0 = w.o[2 * nb], a1 = w.o[2 * nb + 1];
      *reinterpret_cast<float4_t*>(to + 32 * nb) = float4_t{a0[0], a1[0], a0[1], a1[1]};
      *reinterpret_cast<float4_t*>(to + 32 * nb + 4) = float4_t{a0[2], a1[2], a0[3], a1[3]};
    }
    __syncthreads();
    constexpr int R4 = R / 4;
    for (int i = tid; i < heads * R4; i += C::W * kWave) {
      const int h = i / R4, c4 = i - h * R4;
      float ref[C::SG], top = -INFINITY, l = 0.f;
#pragma unroll
      for (int sg = 0; sg < C::SG; ++sg) {
        ref[sg] = refs[sg * 16 + h];
        top = fmaxf(top, ref[sg]);
      }
      float4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int sg = 0; sg < C::SG; ++sg) {
        const float f = __builtin_amdgcn_exp2f(ref[sg] - top);  // 0 for a group that saw no slot
        sum += f * *reinterpret_cast<const float4_t*>(sums + (sg * 16 + h) * C::OS + 4 * c4);
#pragma unroll
        for (int cg = 0; cg < C::CG; ++cg) l += f * part_l[(sg * C::CG + cg) * 16 + h];
      }
      const size_t oh = piece * at.n_heads + h0 + h, col = oh * R + 4 * c4;
      *reinterpret_cast<float4_t*>(at.part_o + col) = sum;
      if (c4 == 0) *reinterpret_cast<float2*>(at.part_ml + oh * 2) = make_float2(top, l);
    }
  }
}

// grid = (sequences, tiles of 16 heads, chunks and the piece behind the packed slots): the head tiles of a chunk run side by side and find its bytes in the
// caches (32 heads in one workgroup need twice the registers, and few long sequences have too few workgroups); sequences side by side go to different XCDs.
template <int R, int DR, int W>
__global__ __launch_bounds__(W * kWave, 2) void attn_packed_kernel(AttnPackedArgs a) {
  using C = PackCfg<R, DR, W>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), h0 = blockIdx.y * 16;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const LaneMap<C> m(lane, wv);
  const AttnArgs& at = a.at;
  const int heads = at.n_heads - h0 < 16 ? at.n_heads - h0 : 16;
  Run run;
  run.b = blockIdx.x;
  const int len = load_uniform_i32(at.seq_len, run.b), n_packed = load_uniform_i32(a.pk.n_packed, run.b);
  const bool behind = (int)blockIdx.z == at.n_splits - 1;  // what lies behind the packed slots in their chunk
  int live = 0;
  if (behind) {
    live = live_slots(len, at.stride, at.max_slots);
    run.packed = packed_slots(n_packed, at.pages.max_pages, at.pages.shift, live);
    if (!open_piece(run.packed, live, at.chunk)) return;
    run.k0 = run.packed;
  } else {
    run.k0 = blockIdx.z * at.chunk;
  }
  Source s = source_of<C>(a, run.b);
  RunHead<C> head;
  load_head<C>(head, a, s, run.b, run.k0, m, h0, heads);
  if (behind) {
    const int chunk_end = at.chunk - run.packed % at.chunk;  // (slots from k0 on)
    run.k1 = live - run.k0 < chunk_end ? live : run.k0 + chunk_end;
    run.piece = run.b * at.n_splits + chunks_of(live, at.chunk);
  } else {
    live = live_slots(len, at.stride, at.max_slots);
    if (run.k0 >= live) return;
    run.packed = packed_slots(n_packed, at.pages.max_pages, at.pages.shift, live);
    run.k1 = live - run.k0 < at.chunk ? live : run.k0 + at.chunk;
    if (run.packed > run.k0 && run.packed < run.k1) run.k1 = run.packed;
    run.piece = run.b * at.n_splits + blockIdx.z;
  }
  s.n_packed = run.packed >> at.pages.shift;  // (whole pages, or all that live)
  if (run.packed & ((1 << at.pages.shift) - 1)) ++s.n_packed;
  attend_run<C>(a, run, head, s, m, h0, heads, smem);
}

template <int R, int DR, int W>
hipError_t launch_one(const AttnPackedArgs& a, hipStream_t st, const EventPair& ev) {
  using C = PackCfg<R, DR, W>;
  static DeviceSet lds_allowed;
  const hipError_t e = allow_lds(&attn_packed_kernel<R, DR, W>, C::lds_bytes, lds_allowed);
  if (e != hipSuccess) return e;
  const dim3 grid(a.at.batch, (a.at.n_heads + 15) / 16, a.at.n_splits);
  launch_timed(attn_packed_kernel<R, DR, W>, grid, dim3(W * kWave), C::lds_bytes, st, ev, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_packed(const AttnPackedArgs& a, hipStream_t st, const EventPair& ev) {
  if (a.at.r == 512 && packed_wide(a.at.r, a.at.batch, a.at.n_heads, a.at.n_splits - 1, a.at.chunk))
    return a.at.d_rope == 32 ? launch_one<512, 32, 8>(a, st, ev) : launch_one<512, 64, 8>(a, st, ev);
#define MTLA_CASE(RR, DD)                       \
  if (a.at.r == RR && a.at.d_rope == DD)        \
    return launch_one<RR, DD, 4>(a, st, ev);
  MTLA_CASE(64, 32)
  MTLA_CASE(64, 64)
  MTLA_CASE(128, 32)
  MTLA_CASE(128, 64)
  MTLA_CASE(256, 32)
  MTLA_CASE(256, 64)
  MTLA_CASE(512, 32)
  MTLA_CASE(512, 64)
#undef MTLA_CASE
  return hipErrorInvalidValue;
}

}  // namespace mtla
