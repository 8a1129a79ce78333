// Decode attention over packed pages (packed.h) and, behind them, pages of the bf16 pool (gfx950).
//
// Eq. (with-rope), incremental case, per 32 slots and 16 heads:
//     S^T[slot, head] = [C_hat | K_hat^R][slot, :] . [q~ | q^R][head, :]
//     O^T[col,  head] += C_hat^T[col, slot] . P^T[slot, head]
// Workgroup = (chunk of slots, sequence); wavefront w owns latent columns [w r/4, (w+1) r/4) and a quarter of the RoPE columns, as in the column-split
// kernel for bf16 rows: every byte of the cache is loaded once whatever the number of heads, the wavefronts' shares of S^T meet in LDS, all form the same
// weights, and each ends with its own columns of the sums.  A lane loads the codes of r / 16 latents of one slot (at r = 512 a whole block of
// 32 with its scale), turns them into bf16 (exact: packed.h) and has them in the A operand's layout of v_mfma_f32_16x16x32_bf16 at once: the order
// of a contraction's terms is free, so the query is brought into the order in which the codes lie.  The same registers go through LDS and
// come back transposed for the value product.
// The query comes as two bf16 planes (hi + lo), and so do the weights here: the packed cache is a third of the bytes of the bf16 one, the matrix cores have
// time for the second product, and the output's error is its own rounding to bf16 (one plane of weights would add as much again).
// The normaliser sums the unrounded weights.
#include "bounds.h"
#include "lds_stream.h"
#include "mtla_device.h"
#include "packed.h"

namespace mtla {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = kBlock / kWave;
constexpr int kTile = kPackTile;   // slots of an operand tile
constexpr int kStep = 2 * kTile;   // slots of a step: the contraction of the value product

template <int R_, int DR_, int NHT_>
struct PackCfg {
  static constexpr int R = R_, DR = DR_, NHT = NHT_;
  static constexpr int E = R + DR;
  static constexpr int RW = R / kWaves;               // latent columns of a wavefront
  static constexpr bool kMixed = RW < 32;             // r = 64: one K step holds the latents (lanes g < 2) and the RoPE columns
  static constexpr int LN = kMixed ? 8 : RW / 4;      // latent columns of a lane
  static constexpr int KC = kMixed ? 0 : RW / 32;     // K steps of latents alone
  static constexpr int KQ = KC + 1;                   // and the one with the RoPE columns (lanes without any hold zeros)
  static constexpr int DRW = DR / kWaves;             // RoPE columns of a wavefront: 8 or 16
  static constexpr int MT = RW / 16;                  // column tiles of its sums
  static constexpr int TS = RW + 16;                  // row stride of the parked slice
  static constexpr int CW = LN / 8;                   // words of codes of a lane
  static constexpr size_t park_bytes = (size_t)kWaves * kStep * TS * 2;
  static constexpr size_t share_bytes = (size_t)kWaves * 2 * NHT * kWave * 16;
  static constexpr size_t lds_bytes = park_bytes + 2 * share_bytes;
};

// What a lane has to do with a tile: constant for the kernel.
template <class C>
struct LaneMap {
  int l16, g, wv;
  int col;                 // its first latent column
  int rope;                // its first RoPE column (of a lane that has none: a readable one)
  bool has_lat, has_rope;
  __device__ __forceinline__ LaneMap(int lane, int wv_) : l16(lane & 15), g(lane >> 4), wv(wv_) {
    has_lat = !C::kMixed || g < 2;
    col = wv * C::RW + (C::kMixed ? 8 * (g & 1) : C::LN * g);
    const int rg = C::kMixed ? g - 2 : g;
    has_rope = rg >= 0 && 8 * rg < C::DRW;
    rope = wv * C::DRW + (has_rope ? 8 * rg : 0);
  }
};

// The table entries of 64 pages from `at` on, one a lane, clamped into the pool that they belong to.
struct Pages64 {
  int at, entry;
};

template <class C>
struct PackedTile {  // as loaded
  uint32_t code[C::CW];
  uint32_t scale;
  u32x4_t xr;
};
template <class C>
struct OpenTile {
  u32x4_t xc[C::CW];
  u32x4_t xr;
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

__device__ __forceinline__ void fetch_pages(Pages64& p, const Source& s, int at, int lane) {
  const int k = at + lane < s.last_entry ? at + lane : s.last_entry;
  const bool packed = k < s.n_packed;
  p.at = at;
  p.entry = clamp_page(packed ? s.table4[k] : s.table[k], packed ? s.n_pages4 : s.n_pages);
}
// Tile of the pool (in units of 16 slots) that holds slot s0 (wavefront-uniform, a multiple of 16).
__device__ __forceinline__ uint32_t pool_tile(Pages64& p, const Source& s, int s0, int lane) {
  const int k = s0 >> s.shift;
  if (k - p.at >= kWave) fetch_pages(p, s, k, lane);
  const int e = __builtin_amdgcn_readlane(p.entry, k - p.at);
  return ((uint32_t)e << (s.shift - 4)) + (uint32_t)((s0 & ((1 << s.shift) - 1)) >> 4);
}

template <class C>
__device__ __forceinline__ void load_tile(PackedTile<C>& t, const Source& s, uint32_t tile, const LaneMap<C>& m) {
  const uint8_t* c = s.codes + (size_t)tile * packed_code_bytes(C::R);
  const uint32_t unit = (uint32_t)(m.col / kPackBlock) * kTile + m.l16;
  const uint8_t* from = c + unit * 16 + (m.col % kPackBlock) / 2;
  if constexpr (C::CW == 4) {
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(from);
    t.code[0] = v[0], t.code[1] = v[1], t.code[2] = v[2], t.code[3] = v[3];
  } else if constexpr (C::CW == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(from);
    t.code[0] = v.x, t.code[1] = v.y;
  } else {
    t.code[0] = *reinterpret_cast<const uint32_t*>(from);
  }
  t.scale = s.scales[(size_t)tile * packed_scale_bytes(C::R) + unit];
  t.xr = *reinterpret_cast<const u32x4_t*>(s.keys + (size_t)tile * (packed_key_bytes(C::DR) / 2) + ((uint32_t)(m.rope / 8) * kTile + m.l16) * 8);
}
template <class C>
__device__ __forceinline__ void load_tile(OpenTile<C>& t, const Source& s, uint32_t tile, const LaneMap<C>& m) {
  const size_t row = (size_t)tile * kTile + m.l16;
  const uint16_t* c = s.lat + row * C::R + m.col;
#pragma unroll
  for (int i = 0; i < C::CW; ++i) t.xc[i] = *reinterpret_cast<const u32x4_t*>(c + 8 * i);
  t.xr = *reinterpret_cast<const u32x4_t*>(s.key + row * C::DR + m.rope);
}

template <class C>
struct Operand {  // a lane's latents, 8 a piece, and its RoPE columns as bf16
  u32x4_t lat[C::CW], rope;
  __device__ __forceinline__ u32x4_t step(int kk, const LaneMap<C>& m) const {
    if constexpr (C::kMixed) {
      u32x4_t v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = m.has_lat ? lat[0][i] : rope[i];
      return v;
    } else {
      return kk < C::KC ? lat[kk < C::KC ? kk : 0] : rope;
    }
  }
};

// live: whether the lane's slot is one of the sequence's; a dead one counts as zeros whatever its bytes are
template <class C>
__device__ __forceinline__ void to_operand(Operand<C>& x, const PackedTile<C>& t, bool live) {
  const float scale = __uint_as_float((live ? t.scale : 127u) << 23);
#pragma unroll
  for (int i = 0; i < C::CW; ++i) {
    const uint32_t c = live ? t.code[i] : 0u;
    x.lat[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
    x.lat[i][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
    x.lat[i][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
    x.lat[i][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x.rope[i] = live ? t.xr[i] : 0u;
}
template <class C>
__device__ __forceinline__ void to_operand(Operand<C>& x, const OpenTile<C>& t, bool live) {
#pragma unroll
  for (int i = 0; i < C::CW; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) x.lat[i][j] = live ? t.xc[i][j] : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.rope[i] = live ? t.xr[i] : 0u;
}

template <class C>
struct Query {
  u32x4_t hi[C::NHT][C::KQ], lo[C::NHT][C::KQ];
};
// Heads past the last one are copies of it and never stored; lanes without a column of a step hold zeros, whatever their rows hold.
template <class C>
__device__ __forceinline__ void load_query(Query<C>& q, const uint16_t* rows, size_t plane, int n_heads, const LaneMap<C>& m) {
#pragma unroll
  for (int ht = 0; ht < C::NHT; ++ht) {
    const int h = 16 * ht + m.l16 < n_heads ? 16 * ht + m.l16 : n_heads - 1;
    const uint16_t* row = rows + (size_t)h * C::E;
#pragma unroll
    for (int kk = 0; kk < C::KQ; ++kk) {
      const bool rope_step = kk == C::KC;
      const uint16_t* from = rope_step ? (C::kMixed && m.has_lat ? row + m.col : row + C::R + m.rope) : row + m.col + 8 * kk;
      const uint32_t mask = !rope_step || m.has_rope || (C::kMixed && m.has_lat) ? 0xffffffffu : 0u;
      q.hi[ht][kk] = *reinterpret_cast<const u32x4_t*>(from) & mask;
      q.lo[ht][kk] = *reinterpret_cast<const u32x4_t*>(from + plane) & mask;
    }
  }
}

template <class C>
struct Sums {  // m_ref: the same in all wavefronts; l_run: this lane's slots only; o: this wavefront's columns
  float m_ref[C::NHT], l_run[C::NHT];
  float4_t o[C::NHT][C::MT];
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int ht = 0; ht < C::NHT; ++ht) {
      m_ref[ht] = -INFINITY;
      l_run[ht] = 0.f;
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt) o[ht][mt] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// Slots [k0, k1) of one kind of page, k0 a multiple of 16 and k0 < k1.
template <class C, class Tile, int NS>
__device__ __forceinline__ void stream(const Source& s, Pages64& pages, const Query<C>& q, Sums<C>& ws, unsigned char* smem, int k0, int k1, int& par,
                                       const LaneMap<C>& m, int lane) {
  uint16_t* park = reinterpret_cast<uint16_t*>(smem) + m.wv * kStep * C::TS;
  const int last = (k1 - 1) & ~(kTile - 1);  // the last tile with a live slot: beyond it, copies of it are loaded and count as dead
  Tile t[NS][2];
  auto load = [&](Tile (&to)[2], int base) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s0 = base + h * kTile < last ? base + h * kTile : last;
      load_tile<C>(to[h], s, pool_tile(pages, s, __builtin_amdgcn_readfirstlane(s0), lane), m);
    }
  };
#pragma unroll
  for (int st = 0; st < NS; ++st) load(t[st], k0 + st * kStep);
  for (int base = k0; base < k1;) {
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      if (base >= k1) break;
      float4_t* shares = reinterpret_cast<float4_t*>(smem + C::park_bytes + (size_t)par * C::share_bytes);
      // ---- this wavefront's share of the logits (log2 units: the query is pre-scaled), and its slice of the latents for the value product
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Operand<C> x;
        to_operand<C>(x, t[st][h], base + h * kTile + m.l16 < k1);
#pragma unroll
        for (int ht = 0; ht < C::NHT; ++ht) {
          float4_t s0 = float4_t{0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
          for (int kk = 0; kk < C::KQ; ++kk) {
            const bf16x8_t xv = __builtin_bit_cast(bf16x8_t, x.step(kk, m));
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, __builtin_bit_cast(bf16x8_t, q.hi[ht][kk]), s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, __builtin_bit_cast(bf16x8_t, q.lo[ht][kk]), s1, 0, 0, 0);
          }
          shares[((m.wv * 2 + h) * C::NHT + ht) * kWave + lane] = s0 + s1;
        }
        if (m.has_lat) {
          uint16_t* to = park + (h * kTile + m.l16) * C::TS + (m.col - m.wv * C::RW);
#pragma unroll
          for (int i = 0; i < C::CW; ++i) *reinterpret_cast<u32x4_t*>(to + 8 * i) = x.lat[i];
        }
      }
      load(t[st], base + NS * kStep);
      __syncthreads();  // all shares are in LDS
      // ---- weights: lane holds head l16 of a head tile and slots 4g .. 4g + 3 of both tiles
      bf16x8_t ph[C::NHT], pl[C::NHT];
#pragma unroll
      for (int ht = 0; ht < C::NHT; ++ht) {
        float sv[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4_t sum = shares[(h * C::NHT + ht) * kWave + lane];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) sum += shares[((w * 2 + h) * C::NHT + ht) * kWave + lane];
#pragma unroll
          for (int v = 0; v < 4; ++v) sv[4 * h + v] = base + h * kTile + 4 * m.g + v < k1 ? sum[v] : -INFINITY;
        }
        // relative to a reference that is fixed at the first live step and moved only where a step tops it by more than 2^kRebase
        constexpr float kRebase = 40.f;
        float top = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
        if (__any(ws.m_ref[ht] == -INFINITY || top - ws.m_ref[ht] > kRebase)) {
          top = quarter_reduce(top, LaneMax());
          if (ws.m_ref[ht] == -INFINITY) {
            ws.m_ref[ht] = top;
          } else if (top - ws.m_ref[ht] > kRebase) {
            const float alpha = __builtin_amdgcn_exp2f(ws.m_ref[ht] - top);
            ws.m_ref[ht] = top;
            ws.l_run[ht] *= alpha;
#pragma unroll
            for (int mt = 0; mt < C::MT; ++mt) ws.o[ht][mt] *= alpha;
          }
        }
        const float ref = ws.m_ref[ht] == -INFINITY ? 0.f : ws.m_ref[ht];
        u32x4_t hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p0 = __builtin_amdgcn_exp2f(sv[2 * j] - ref), p1 = __builtin_amdgcn_exp2f(sv[2 * j + 1] - ref);
          uint32_t a, b;
          split_bf16x2(p0, p1, a, b);
          hi[j] = a;
          lo[j] = b;
          ws.l_run[ht] += p0 + p1;
        }
        ph[ht] = __builtin_bit_cast(bf16x8_t, hi);
        pl[ht] = __builtin_bit_cast(bf16x8_t, lo);
      }
      // ---- O^T[col, head] += C_hat^T[col, slot] P^T[slot, head]: a transposing read hands a lane four slots of a column, two of them the operand
      const uint16_t* trow = park + (4 * m.g + (m.l16 >> 2)) * C::TS + 4 * (m.l16 & 3);
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt) {
        const short4_t c0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(trow + 16 * mt));
        const short4_t c1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(trow + kTile * C::TS + 16 * mt));
        typedef short short8_t __attribute__((ext_vector_type(8)));
        const bf16x8_t cv = __builtin_bit_cast(bf16x8_t, (short8_t)__builtin_shufflevector(c0, c1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int ht = 0; ht < C::NHT; ++ht) {
          ws.o[ht][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cv, ph[ht], ws.o[ht][mt], 0, 0, 0);
          ws.o[ht][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cv, pl[ht], ws.o[ht][mt], 0, 0, 0);
        }
      }
      par ^= 1;
      base += kStep;
    }
  }
}

// grid = (chunks, sequences, groups of up to 32 heads)
template <int R, int DR, int NHT>
__global__ __launch_bounds__(kBlock) void attn_packed_kernel(AttnPackedArgs a) {
  using C = PackCfg<R, DR, NHT>;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int split = blockIdx.x, b = blockIdx.y, h0 = blockIdx.z * 32;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const LaneMap<C> m(lane, wv);
  const AttnArgs& at = a.at;
  const int heads = at.n_heads - h0 < 32 ? at.n_heads - h0 : 32;

  const int live = live_slots(load_uniform_i32(at.seq_len, b), at.stride, at.max_slots);
  int n_packed = load_uniform_i32(a.pk.n_packed, b);
  const int k0 = split * at.chunk, k1 = live < k0 + at.chunk ? live : k0 + at.chunk;
  if (k0 >= k1) return;
  n_packed = n_packed < 0 ? 0 : (n_packed < at.pages.max_pages ? n_packed : at.pages.max_pages);
  Source s;
  s.codes = a.pk.codes;
  s.scales = a.pk.scales;
  s.keys = a.pk.keys;
  s.lat = reinterpret_cast<const uint16_t*>(at.lat);
  s.key = reinterpret_cast<const uint16_t*>(at.key);
  s.table = at.pages.table + (size_t)b * at.pages.max_pages;
  s.table4 = a.pk.table + (size_t)b * at.pages.max_pages;
  s.n_packed = n_packed;
  s.n_pages = at.pages.n_pages;
  s.n_pages4 = a.pk.n_pages;
  s.shift = at.pages.shift;
  s.last_entry = at.pages.max_pages - 1;

  Pages64 pages;
  fetch_pages(pages, s, k0 >> s.shift, lane);
  Query<C> q;
  load_query<C>(q, reinterpret_cast<const uint16_t*>(at.qcat) + ((size_t)b * at.n_heads + h0) * C::E, at.q_plane, heads, m);
  Sums<C> ws;
  ws.reset();
  const long long packed_slots = (long long)n_packed << s.shift;
  const int kp = (int)(packed_slots < k1 ? packed_slots : k1);  // slots below it come out of packed pages
  int par = 0;
  if (kp > k0) stream<C, PackedTile<C>, 2>(s, pages, q, ws, smem, k0, kp, par, m, lane);
  const int ko = kp > k0 ? kp : k0;
  if (k1 > ko) stream<C, OpenTile<C>, 1>(s, pages, q, ws, smem, ko, k1, par, m, lane);

  // ---- the chunk's partial: lane holds head l16, columns 16mt + 4g .. + 3
  const size_t piece = (size_t)b * at.n_splits + split;
#pragma unroll
  for (int ht = 0; ht < NHT; ++ht) {
    const float l = quarter_reduce(ws.l_run[ht], LaneSum());
    if (16 * ht + m.l16 < heads) {
      const size_t oh = piece * at.n_heads + h0 + 16 * ht + m.l16;
      const size_t col = oh * R + wv * C::RW + 4 * m.g;
      if (at.part_f16) {
        const float inv = 1.f / l;
        uint16_t* po = reinterpret_cast<uint16_t*>(at.part_o) + col;
#pragma unroll
        for (int mt = 0; mt < C::MT; ++mt)
          *reinterpret_cast<uint2*>(po + 16 * mt) = make_uint2(pack_f16x2(ws.o[ht][mt][0] * inv, ws.o[ht][mt][1] * inv),
                                                               pack_f16x2(ws.o[ht][mt][2] * inv, ws.o[ht][mt][3] * inv));
      } else {
#pragma unroll
        for (int mt = 0; mt < C::MT; ++mt) *reinterpret_cast<float4_t*>(at.part_o + col + 16 * mt) = ws.o[ht][mt];
      }
      if (wv == 0 && m.g == 0) *reinterpret_cast<float2*>(at.part_ml + oh * 2) = make_float2(ws.m_ref[ht], l);
    }
  }
}

template <int R, int DR, int NHT>
hipError_t launch_one(const AttnPackedArgs& a, hipStream_t st, const EventPair& ev) {
  using C = PackCfg<R, DR, NHT>;
  static DeviceSet lds_allowed;
  const hipError_t e = allow_lds(&attn_packed_kernel<R, DR, NHT>, C::lds_bytes, lds_allowed);
  if (e != hipSuccess) return e;
  const dim3 grid(a.at.n_splits, a.at.batch, (a.at.n_heads + 31) / 32);
  launch_timed(attn_packed_kernel<R, DR, NHT>, grid, dim3(kBlock), C::lds_bytes, st, ev, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_packed(const AttnPackedArgs& a, hipStream_t st, const EventPair& ev) {
#define MTLA_CASE(RR, DD)                       \
  if (a.at.r == RR && a.at.d_rope == DD)        \
    return a.at.n_heads <= 16 ? launch_one<RR, DD, 1>(a, st, ev) : launch_one<RR, DD, 2>(a, st, ev);
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
