// Page tables made to fit the sequences' lengths, on the device: which pages every sequence holds, the ring of free pages, and the rows that
// new tokens go to.  What csrc/pages.hip does on the host for callers that may synchronise, for those that replay their steps as a graph.
//
// A sequence holds entries first .. end - 1 of its table row.  What it should hold follows from its length, so the pages that it lacks and
// those that it has no use for are two intervals each, and where they are taken from and go to in the ring are running sums over the sequences:
//   packed pool   [0, max(len / s / P - keep, 0))                    complete pages (P slots a page)
//   bf16 pool     [end of the packed ones, ceil(ceil((len + n) / s) / P))
// A sequence gets all that it lacks or, if the ring does not hold what it and those before it lack together, nothing.  Given back pages can be
// handed out from the next call on: the packing behind this call still reads them.
//
// A wavefront takes 16 or 64 sequences, one a lane; the three beside it help to carry long intervals.  Up to 64 sequences that is one launch.  Beyond, a launch in
// front adds up what every group takes and gives, and if the rings hold all of it, a workgroup a group goes on from the sums before its own; if not, one workgroup
// goes through all in order (who gets nothing depends on who came before).  The calls are chains of reads that wait for each other and of some 2000
// instructions a wavefront, not of bytes.  us, beside one workgroup of 1024 threads and the slot map in a launch of its own:
//   16 sequences, a token each        5.0, 7.2 + 2.6
//   256 that take 40 pages each       2.3 + 7.3 (groups of 64: 1.9 + 11.5), 13.5
//   3001, drafts of 8, two pools      3.2 + 7.5, 25.2 + 5.1
#include "bounds.h"
#include "decode_schedule.h"
#include "mtla_device.h"
#include "packed.h"

namespace mtla {

namespace {

constexpr int kFitWaves = kBlock / kWave;
constexpr int kBatch = 4;       // long intervals that a wavefront has under way
constexpr int kOwnTokens = 8;   // new tokens of a sequence whose rows its thread finds itself
constexpr int kOwnEntries = 2;  // entries of an interval that its sequence's thread moves itself; longer ones are dealt to the wavefronts

// Running sums that stay at `cap` once they reach it: what is above is refused (or dropped) whatever its size, and no length in a caller's
// array makes a sum overflow (cap <= 2^28).
__device__ __forceinline__ int add_upto(int a, int b, int cap) {
  const int s = a + b;
  return s < cap ? s : cap;
}
__device__ __forceinline__ int row_scan_upto(int v, int cap) {  // inclusive, over 16 lanes
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true), cap);
  return add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true), cap);
}
__device__ __forceinline__ int wave_scan_upto(int v, int cap) {
  v = row_scan_upto(v, cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false), cap);
  return add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false), cap);
}

// A lane's sum in front of its own `v`, over the wavefront and, through `carry`, the rounds before.
__device__ __forceinline__ int sum_before(int v, int cap, int& carry, int lane) {
  const int inc = wave_scan_upto(v < cap ? v : cap, cap), prev = __shfl_up(inc, 1, kWave);
  const int before = lane == 0 ? carry : add_upto(carry, prev, cap);
  carry = add_upto(carry, __builtin_amdgcn_readlane(inc, kWave - 1), cap);
  return before;
}

// What a sequence lacks of [wf, we) and what it has beside it, where it holds [f, e): two intervals each, the lower one first (a lower
// one to take leaves none to give there, and so above: two moves in all).
struct Change {
  int take_lo, n_take_lo, take_hi, n_take_hi;
  int give_lo, n_give_lo, give_hi, n_give_hi;
  __device__ __forceinline__ int n_take() const { return n_take_lo + n_take_hi; }
  __device__ __forceinline__ int n_give() const { return n_give_lo + n_give_hi; }
};
__device__ __forceinline__ int above0(int v) { return v > 0 ? v : 0; }
__device__ __forceinline__ Change change_of(int f, int e, int wf, int we) {
  Change c;
  if (f >= e) {
    c = Change{wf, 0, wf, above0(we - wf), f, 0, f, 0};
  } else {
    c.take_lo = wf;
    c.n_take_lo = above0((f < we ? f : we) - wf);
    c.take_hi = e > wf ? e : wf;
    c.n_take_hi = above0(we - c.take_hi);
    c.give_lo = f;
    c.n_give_lo = above0((e < wf ? e : wf) - f);
    c.give_hi = f > we ? f : we;
    c.n_give_hi = above0(e - c.give_hi);
  }
  return c;
}

// One interval of table entries and its places in the ring.
struct Move {
  int32_t* entries;  // of the table row
  int n, at;         // the first one's place in the ring
  int give;          // 1: entries -> ring, 0: ring -> entries, 2: the spill page -> entries
};

__device__ __forceinline__ int wrapped(long long at, int n) { return (int)(at < n ? at : at - n); }

__device__ __forceinline__ int32_t moved(const FitPool& p, const Move& m, int i) {  // the page that entry i of an interval moves
  return m.give == 1 ? m.entries[i] : (m.give == 0 ? p.ring[wrapped((long long)m.at + i, p.n_pages)] : p.spill);
}
__device__ __forceinline__ void put_moved(const FitPool& p, const Move& m, int i, int32_t page) {
  *(m.give == 1 ? p.ring + wrapped((long long)m.at + i, p.n_pages) : m.entries + i) = page;
}

// Two intervals to take and two to give of either pool.
constexpr int kMoves = 8;
struct FitShared {
  int n_long;
  Move longs[kMoves / 2 * kWave];  // (of a pool's four intervals two at most are not empty)
  unsigned char of_packed[kMoves / 2 * kWave];
};

// What a round needs of a sequence.
struct Held {
  int len, n, f, e, f4, e4;
};
__device__ __forceinline__ Held held_by(const FitArgs& a, bool two, int b) {
  Held h{0, 0, 0, 0, 0, 0};
  if (b < a.batch) {
    h.len = a.seq_len[b];
    h.n = a.n_new ? a.n_new[b] : a.n_new_max;
    h.f = a.pool.first[b];
    h.e = a.pool.end[b];
    if (two) {
      h.f4 = a.packed.first[b];
      h.e4 = a.packed.end[b];
    }
  }
  return h;
}

// What it holds and what it should hold, in entries of its table row.
struct Needs {
  int have, n, f, e, f4, e4;
  int reach, complete;  // end of the entries that its tokens reach, of those that complete pages have
};
__device__ __forceinline__ Needs needs_of(const FitArgs& a, const Held& h, bool in) {
  Needs s;
  s.f = pages_inside(h.f, a.max_pages);
  s.e = pages_inside(h.e, a.max_pages);
  s.f4 = pages_inside(h.f4, a.max_pages);
  s.e4 = pages_inside(h.e4, a.max_pages);
  s.n = new_rows(h.n, a.n_new_max);
  // tokens before and after; a length outside 0 .. max_slots * stride counts as the nearer end
  const long long room = (long long)a.max_slots * a.stride;
  s.have = h.len < 0 ? 0 : (int)(h.len < room ? h.len : room);
  const long long after = (long long)s.have + s.n < room ? (long long)s.have + s.n : room;
  s.reach = in ? (live_slots((int)after, a.stride, a.max_slots) + (1 << a.shift) - 1) >> a.shift : 0;
  s.complete = in ? above0((int)((unsigned)s.have / (unsigned)a.stride >> a.shift) - a.keep_pages) : 0;
  return s;
}

// A ring as it is, whatever its words hold.
struct Ring {
  int head, count;
};
__device__ __forceinline__ Ring ring_of(const FitPool& p) {
  Ring r{p.state[0], p.state[1]};
  r.head = r.head < 0 || r.head >= p.n_pages ? 0 : r.head;
  r.count = r.count < 0 ? 0 : (r.count < p.n_pages ? r.count : p.n_pages);
  return r;
}
__device__ __forceinline__ void put_ring(const FitPool& p, const Ring& r, int taken, int given, int refused) {
  const int room = p.n_pages - r.count;
  p.state[0] = wrapped((long long)r.head + taken, p.n_pages);
  p.state[1] = r.count - taken + (given < room ? given : room);
  p.state[2] = refused;
}

// What a group of sequences takes and gives if nobody is refused.
struct Sums {
  int take4, take, give, give4;
};
static_assert(sizeof(Sums) == 16, "fit_scratch_bytes");
constexpr int kSumCap = 1 << 29;  // (more than any pool has pages)

// sums[i] of the i-th `group` (16 or 64) sequences, and behind them the rings
__global__ __launch_bounds__(kBlock) void pages_sums_kernel(FitArgs a, Sums* sums, int n_sums, int group) {
  const bool two = a.packed.table != nullptr;
  const int b = blockIdx.x * kBlock + threadIdx.x, last = group - 1;
  const bool in = b < a.batch;
  const Needs h = needs_of(a, held_by(a, two, b), in);
  const Change c4 = change_of(h.f4, h.e4, 0, two ? h.complete : 0);
  const int end4 = two ? h.complete : 0;
  const Change c = change_of(h.f, h.e, end4, h.reach > end4 ? h.reach : end4);
  const int v[4] = {in && two ? c4.n_take() : 0, in ? c.n_take() : 0, in ? c.n_give() : 0, in && two ? c4.n_give() : 0};
  int sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = group == kWave ? wave_scan_upto(v[k], kSumCap) : row_scan_upto(v[k], kSumCap);
  if ((b & last) == last && b / group < n_sums) sums[b / group] = Sums{sum[0], sum[1], sum[2], sum[3]};
  if (b == 0) {
    const Ring r = ring_of(a.pool), r4 = two ? ring_of(a.packed) : Ring{0, 0};
    sums[n_sums] = Sums{r.head, r.count, r4.head, r4.count};
  }
}

// Where token `t` behind a sequence's `len` goes in the bf16 pool: entry `k` of its table row (-1: nowhere), and the slot of the page.
struct TokenPlace {
  int k, in_page;
};
__device__ __forceinline__ TokenPlace place_of(const FitArgs& a, int t, int n, int len, int f, int e) {
  const long long at = (long long)len + t;
  TokenPlace r{-1, 0};
  if (t < n && len >= 0 && at < (long long)a.max_slots * a.stride) {
    const int slot = (int)((unsigned)at / (unsigned)a.stride), k = slot >> a.shift;
    if (k >= f && k < e) r = TokenPlace{k, slot & ((1 << a.shift) - 1)};
  }
  return r;
}

// Rows of four tokens, `step` apart: their table entries are asked for together.
__device__ __forceinline__ void put_rows(const FitArgs& a, int64_t* out, const int32_t* row, int t0, int step, int n, int len, int f, int e) {
  TokenPlace to[4];
  int32_t at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    to[i] = place_of(a, t0 + i * step, n, len, f, e);
    at[i] = to[i].k >= 0 ? row[to[i].k] : 0;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + i * step < a.n_new_max) out[t0 + i * step] = to[i].k >= 0 ? ((int64_t)at[i] << a.shift) + to[i].in_page : -1;
}

// `sums` (may be NULL: one workgroup): of pages_sums_kernel; `own_map`: a sequence's lane writes its part of the slot map too.
__global__ __launch_bounds__(kBlock) void pages_fit_kernel(FitArgs a, const Sums* sums, int n_sums, int group, int own_map) {
  __shared__ FitShared s;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool two = a.packed.table != nullptr;
  const int P = a.max_pages;

  Ring r{0, 0}, r4{0, 0};
  // takes stop at what the ring holds, gives at the places that it has left
  Sums carry{0, 0, 0, 0}, all{0, 0, 0, 0};
  bool side_by_side = false;
  Held next = held_by(a, two, (sums ? blockIdx.x : 0) * group + lane);
  if (sums) {
    const Sums rings = sums[n_sums];
    r = Ring{rings.take4, rings.take};
    r4 = Ring{rings.give, rings.give4};
    for (int i = lane; i < n_sums; i += kWave) {
      const Sums x = sums[i];
      const bool before = i < (int)blockIdx.x;
      auto add = [&](int Sums::* k) {
        all.*k = add_upto(all.*k, x.*k, kSumCap);
        if (before) carry.*k = add_upto(carry.*k, x.*k, kSumCap);
      };
      add(&Sums::take4);
      add(&Sums::take);
      add(&Sums::give);
      add(&Sums::give4);
    }
    auto whole = [&](int Sums::* k) {
      all.*k = __builtin_amdgcn_readlane(wave_scan_upto(all.*k, kSumCap), kWave - 1);
      carry.*k = __builtin_amdgcn_readlane(wave_scan_upto(carry.*k, kSumCap), kWave - 1);
    };
    whole(&Sums::take4);
    whole(&Sums::take);
    whole(&Sums::give);
    whole(&Sums::give4);
    side_by_side = all.take <= r.count && all.give <= a.pool.n_pages - r.count && (!two || (all.take4 <= r4.count && all.give4 <= a.packed.n_pages - r4.count));
    if (!side_by_side) {
      if (blockIdx.x > 0) return;
      carry = Sums{0, 0, 0, 0};
    }
  } else {
    r = ring_of(a.pool);
    if (two) r4 = ring_of(a.packed);
  }
  const Sums cap{r4.count + 1, r.count + 1, a.pool.n_pages - r.count + 1, two ? a.packed.n_pages - r4.count + 1 : 1};
  int taken = 0, taken4 = 0, refused = 0, refused4 = 0;

  const int width = side_by_side ? group : kWave, b_end = side_by_side ? ((int)blockIdx.x + 1) * group : a.batch;
  for (int b0 = side_by_side ? blockIdx.x * group : 0; b0 < b_end; b0 += width) {
    const int b = b0 + lane;
    const bool in = lane < width && b < a.batch;
    int nf = 0, ne = 0;
    Needs h{};
    const Held held = next;
    if (tid == 0) s.n_long = 0;
    if (wv == 0) {
      if (!side_by_side) next = held_by(a, two, b + kWave);
      h = needs_of(a, held, in);
      if (in && a.pool.was_end) a.pool.was_end[b] = h.e;
      if (in && two && a.packed.was_end) a.packed.was_end[b] = h.e4;

      // ---- packed pool: complete pages
      const Change c4 = change_of(h.f4, h.e4, 0, two ? h.complete : 0);
      int first4 = 0, end4 = 0, rank4 = 0;
      bool ok4 = true;
      if (two) {
        const int n4 = in ? c4.n_take() : 0;
        rank4 = sum_before(n4, cap.take4, carry.take4, lane);
        ok4 = n4 == 0 || (long long)rank4 + n4 <= r4.count;
        end4 = h.complete;
        if (!ok4) {  // refused: what it holds of what it should hold stays (a packed pool's rows start at 0)
          first4 = h.f4 < h.complete ? h.f4 : h.complete;
          end4 = h.e4 < h.complete ? h.e4 : h.complete;
          end4 = end4 > first4 ? end4 : first4;
        }
      }

      // ---- bf16 pool: from there on
      const int want_end = h.reach > end4 ? h.reach : end4;
      const Change c = change_of(h.f, h.e, end4, want_end);
      const int n_take = in ? c.n_take() : 0, n_give = in ? c.n_give() : 0, n_give4 = in && two ? c4.n_give() : 0;
      const int rank = sum_before(n_take, cap.take, carry.take, lane), given = sum_before(n_give, cap.give, carry.give, lane);
      const int given4 = two ? sum_before(n_give4, cap.give4, carry.give4, lane) : 0;
      const bool ok = n_take == 0 || (long long)rank + n_take <= r.count;

      // ---- entries: out of the ring (or the spill page), and back behind its last page
      struct {
        int from, n, at;  // first entry, entries, the first one's place in the ring
      } mv[kMoves] = {};
      int32_t* row = a.pool.table + (size_t)(in ? b : 0) * P;
      int32_t* row4 = two ? a.packed.table + (size_t)(in ? b : 0) * P : row;
      auto move = [&](int k) {
        const bool packed = k >= kMoves / 2;
        return Move{(packed ? row4 : row) + mv[k].from, mv[k].n, mv[k].at, (k & 2) ? 1 : (packed || ok ? 0 : 2)};
      };
      if (in) {
        if (ok) {
          const int at = wrapped((long long)r.head + rank, a.pool.n_pages);
          mv[0] = {c.take_lo, c.n_take_lo, at};
          mv[1] = {c.take_hi, c.n_take_hi, wrapped((long long)at + c.n_take_lo, a.pool.n_pages)};
          taken += n_take;
        } else {
          ++refused;
          if (a.pool.spill >= 0) {
            mv[0] = {c.take_lo, c.n_take_lo, 0};
            mv[1] = {c.take_hi, c.n_take_hi, 0};
          }
        }
        if (n_give > 0 && (long long)given + n_give <= a.pool.n_pages - r.count) {  // (always, unless the arrays name more pages than there are)
          const int at = wrapped(wrapped((long long)r.head + r.count, a.pool.n_pages) + (long long)given, a.pool.n_pages);
          mv[2] = {c.give_lo, c.n_give_lo, at};
          mv[3] = {c.give_hi, c.n_give_hi, wrapped((long long)at + c.n_give_lo, a.pool.n_pages)};
        }
        // refused: it keeps what it holds of what it should hold
        nf = ok ? end4 : (h.f > end4 ? (h.f < want_end ? h.f : want_end) : end4);
        ne = ok ? want_end : (h.e < want_end ? h.e : want_end);
        ne = ne > nf ? ne : nf;
        a.pool.first[b] = nf;
        a.pool.end[b] = ne;
        if (two) {
          if (ok4) {
            const int at = wrapped((long long)r4.head + rank4, a.packed.n_pages);
            mv[4] = {c4.take_lo, c4.n_take_lo, at};
            mv[5] = {c4.take_hi, c4.n_take_hi, wrapped((long long)at + c4.n_take_lo, a.packed.n_pages)};
            taken4 += c4.n_take();
          } else {
            ++refused4;
          }
          if (n_give4 > 0 && (long long)given4 + n_give4 <= a.packed.n_pages - r4.count) {
            const int at = wrapped(wrapped((long long)r4.head + r4.count, a.packed.n_pages) + (long long)given4, a.packed.n_pages);
            mv[6] = {c4.give_lo, c4.n_give_lo, at};
            mv[7] = {c4.give_hi, c4.n_give_hi, wrapped((long long)at + c4.n_give_lo, a.packed.n_pages)};
          }
          a.packed.first[b] = first4;
          a.packed.end[b] = end4;
        }
      }
      // What an interval does depends on no other, so all pages of the short ones are asked for before the first is put down.
      int32_t page[kMoves][kOwnEntries];
#pragma unroll
      for (int k = 0; k < kMoves; ++k) {
        if (mv[k].n > kOwnEntries) {
          const int at = atomicAdd(&s.n_long, 1);
          s.longs[at] = move(k);
          s.of_packed[at] = k >= kMoves / 2;
        }
#pragma unroll
        for (int i = 0; i < kOwnEntries; ++i)
          if (i < mv[k].n && mv[k].n <= kOwnEntries) page[k][i] = moved(k < kMoves / 2 ? a.pool : a.packed, move(k), i);
      }
#pragma unroll
      for (int k = 0; k < kMoves; ++k)
#pragma unroll
        for (int i = 0; i < kOwnEntries; ++i)
          if (i < mv[k].n && mv[k].n <= kOwnEntries) put_moved(k < kMoves / 2 ? a.pool : a.packed, move(k), i, page[k][i]);
    }
    __syncthreads();
    const int n_long = s.n_long;
    for (int k = wv; k < n_long; k += kBatch * kFitWaves) {  // a wavefront has the first entries of several under way
      int32_t first[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int at = k + j * kFitWaves;
        if (at < n_long && lane < s.longs[at].n) first[j] = moved(s.of_packed[at] ? a.packed : a.pool, s.longs[at], lane);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int at = k + j * kFitWaves;
        if (at >= n_long) break;
        const Move m = s.longs[at];
        const FitPool& p = s.of_packed[at] ? a.packed : a.pool;
        if (lane < m.n) put_moved(p, m, lane, first[j]);
        for (int i = kWave + lane; i < m.n; i += kWave) put_moved(p, m, i, moved(p, m, i));
      }
    }
    __syncthreads();  // the list is filled anew; a sequence's entries are in place
    if (own_map && wv == 0 && in) {
      const int32_t* row = a.pool.table + (size_t)b * P;
      int64_t* out = a.slot_map + (size_t)b * a.n_new_max;
#pragma unroll 1
      for (int t0 = 0; t0 < a.n_new_max; t0 += 4) put_rows(a, out, row, t0, 1, h.n, held.len, nf, ne);
    }
  }

  // ---- the rings
  if (side_by_side) {
    if (blockIdx.x == 0 && tid == 0) {
      put_ring(a.pool, r, all.take, all.give, 0);
      if (two) put_ring(a.packed, r4, all.take4, all.give4, 0);
    }
  } else if (wv == 0) {
    auto sum = [&](int v) { return __builtin_amdgcn_readlane(wave_scan_upto(v, kSumCap), kWave - 1); };
    taken = sum(taken);
    taken4 = sum(taken4);
    refused = sum(refused);
    refused4 = sum(refused4);
    if (lane == 0) {
      put_ring(a.pool, r, taken, carry.give, refused);
      if (two) put_ring(a.packed, r4, taken4, carry.give4, refused4);
      if (refused || refused4) *a.status = 3;  // MTLA_ERR_CAPACITY
    }
  }
}

// Rows of the bf16 pool that the new tokens go to; -1 for padding and where the sequence holds no page.  grid = (pieces of the tokens, batch)
__global__ __launch_bounds__(kBlock) void slot_map_kernel(FitArgs a) {
  const int b = blockIdx.y;
  const int n = new_rows(a.n_new ? a.n_new[b] : a.n_new_max, a.n_new_max);
  const int len = a.seq_len[b], f = a.pool.first[b], e = a.pool.end[b];
  const int32_t* row = a.pool.table + (size_t)b * a.max_pages;
  int64_t* out = a.slot_map + (size_t)b * a.n_new_max;
  for (int t = blockIdx.x * 4 * kBlock + threadIdx.x; t < a.n_new_max; t += gridDim.x * 4 * kBlock) put_rows(a, out, row, t, kBlock, n, len, f, e);
}

}  // namespace

hipError_t launch_pages_fit(const FitArgs& a, hipStream_t st) {
  const bool own_map = a.slot_map && a.n_new_max <= kOwnTokens;
  const int group = fit_group(a.batch), n = fit_groups(a.batch);
  Sums* sums = n > 1 ? reinterpret_cast<Sums*>(a.scratch) : nullptr;
  if (sums) {
    hipLaunchKernelGGL(pages_sums_kernel, dim3((a.batch + kBlock - 1) / kBlock), dim3(kBlock), 0, st, a, sums, n, group);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(pages_fit_kernel, dim3(n), dim3(kBlock), 0, st, a, (const Sums*)sums, n, group, own_map ? 1 : 0);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.slot_map || own_map) return e;
  const int parts = (a.n_new_max + 4 * kBlock - 1) / (4 * kBlock);
  hipLaunchKernelGGL(slot_map_kernel, dim3(parts, a.batch), dim3(kBlock), 0, st, a);
  return hipGetLastError();
}

}  // namespace mtla
