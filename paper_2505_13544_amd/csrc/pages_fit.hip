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
// One workgroup, a sequence per thread and 1024 of them at a time: the call is a chain of latencies (lengths, two scans, ring, tables), not of
// bytes, and everything that would have to cross workgroups would be another launch.
#include "bounds.h"
#include "mtla_device.h"
#include "packed.h"

namespace mtla {

namespace {

constexpr int kFitBlock = 1024, kFitWaves = kFitBlock / kWave;
constexpr int kOwnEntries = 2;  // entries of an interval that its sequence's thread moves itself; longer ones are dealt to the wavefronts

// Running sums that stay at `cap` once they reach it: what is above is refused (or dropped) whatever its size, and no length in a caller's
// array makes a sum overflow (cap <= 2^28).
__device__ __forceinline__ int add_upto(int a, int b, int cap) {
  const int s = a + b;
  return s < cap ? s : cap;
}
__device__ __forceinline__ int wave_scan_upto(int v, int cap) {  // inclusive
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false), cap);
  v = add_upto(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false), cap);
  return v;
}

// Sums over the workgroup's sequences of this round and, through `carry`, of the rounds before: the sum in front of this thread's `v`.
template <int N>
struct Scan {
  int before[N];
};
template <int N>
__device__ __forceinline__ Scan<N> block_scan(const int (&v)[N], const int (&cap)[N], int (&carry)[N], int* s_tot /*[N][kFitWaves]*/, int lane, int wv) {
  Scan<N> r;
  int inc[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    inc[k] = wave_scan_upto(v[k] < cap[k] ? v[k] : cap[k], cap[k]);
    if (lane == kWave - 1) s_tot[k * kFitWaves + wv] = inc[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    int sum = carry[k], all = carry[k];
#pragma unroll
    for (int w = 0; w < kFitWaves; ++w) {
      const int t = s_tot[k * kFitWaves + w];
      if (w < wv) sum = add_upto(sum, t, cap[k]);
      all = add_upto(all, t, cap[k]);
    }
    // (the sum in front of this lane's own: of the lane before)
    const int prev = __shfl_up(inc[k], 1, kWave);
    r.before[k] = lane == 0 ? sum : add_upto(sum, prev, cap[k]);
    carry[k] = all;
  }
  __syncthreads();  // the totals' place is used again
  return r;
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

__device__ __forceinline__ void move_one(const FitPool& p, const Move& m, int i) {
  const int place = wrapped((long long)m.at + i, p.n_pages);
  if (m.give == 1) p.ring[place] = m.entries[i];
  else m.entries[i] = m.give == 0 ? p.ring[place] : p.spill;
}

struct FitShared {
  int tot[3 * kFitWaves];
  int n_long;
  Move longs[4 * kFitBlock];  // two intervals of each pool
  unsigned char of_packed[4 * kFitBlock];
};

// Carries one interval out, or leaves it to all wavefronts.
__device__ __forceinline__ void do_move(const FitPool& p, const Move& m, bool packed, FitShared& s) {
  if (m.n <= 0) return;
  if (m.n > kOwnEntries) {
    const int at = atomicAdd(&s.n_long, 1);  // (what an interval does depends on no other: any order)
    s.longs[at] = m;
    s.of_packed[at] = packed;
    return;
  }
  for (int i = 0; i < m.n; ++i) move_one(p, m, i);
}

__global__ __launch_bounds__(kFitBlock) void pages_fit_kernel(FitArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  FitShared& s = *reinterpret_cast<FitShared*>(smem);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid >> 6;
  const bool two = a.packed.table != nullptr;
  const int P = a.max_pages, ps_mask = (1 << a.shift) - 1;

  // the rings as they are, whatever the words hold
  auto ring_of = [](const FitPool& p, int& head, int& count) {
    head = p.state[0];
    count = p.state[1];
    head = head < 0 || head >= p.n_pages ? 0 : head;
    count = count < 0 ? 0 : (count < p.n_pages ? count : p.n_pages);
  };
  int head, count, head4 = 0, count4 = 0;
  ring_of(a.pool, head, count);
  if (two) ring_of(a.packed, head4, count4);
  // takes stop at what the ring holds, gives at the places that it has left
  int carry4[1] = {0}, carry[3] = {0, 0, 0};
  const int cap4[1] = {count4 + 1};
  const int cap[3] = {count + 1, a.pool.n_pages - count + 1, two ? a.packed.n_pages - count4 + 1 : 1};
  int taken = 0, taken4 = 0, refused = 0, refused4 = 0;

  for (int b0 = 0; b0 < a.batch; b0 += kFitBlock) {
    const int b = b0 + tid;
    const bool in = b < a.batch;
    if (tid == 0) s.n_long = 0;
    int len = 0, n = 0, f = 0, e = 0, f4 = 0, e4 = 0;
    if (in) {
      len = a.seq_len[b];
      n = a.n_new ? a.n_new[b] : a.n_new_max;
      f = a.pool.first[b];
      e = a.pool.end[b];
      if (two) {
        f4 = a.packed.first[b];
        e4 = a.packed.end[b];
      }
    }
    auto inside = [&](int v) { return v < 0 ? 0 : (v < P ? v : P); };
    f = inside(f);
    e = inside(e);
    f4 = inside(f4);
    e4 = inside(e4);
    n = new_rows(n, a.n_new_max);
    if (in && a.pool.was_end) a.pool.was_end[b] = e;
    if (in && two && a.packed.was_end) a.packed.was_end[b] = e4;
    // tokens before and after; a length outside 0 .. max_slots * stride counts as the nearer end
    const long long room = (long long)a.max_slots * a.stride;
    const int have = len < 0 ? 0 : (int)(len < room ? len : room);
    const long long after = (long long)have + n < room ? (long long)have + n : room;
    const int reach = in ? (live_slots((int)after, a.stride, a.max_slots) + ps_mask) >> a.shift : 0;
    const int complete = in ? above0((int)((unsigned)have / (unsigned)a.stride >> a.shift) - a.keep_pages) : 0;

    // ---- packed pool: complete pages
    Change c4 = change_of(f4, e4, 0, two ? complete : 0);
    int end4 = 0, rank4 = 0;
    bool ok4 = true;
    if (two) {
      const int v[1] = {in ? c4.n_take() : 0};
      const Scan<1> sc = block_scan<1>(v, cap4, carry4, s.tot, lane, wv);
      rank4 = sc.before[0];
      ok4 = v[0] == 0 || (long long)rank4 + v[0] <= count4;
      // refused: what it holds of what it should hold stays (a packed pool's rows start at 0)
      end4 = ok4 ? complete : (e4 < complete ? e4 : complete);
      if (!ok4) {
        const int first4 = f4 < complete ? f4 : complete;
        end4 = end4 > first4 ? end4 : first4;
        f4 = first4;
      } else {
        f4 = 0;
      }
    }

    // ---- bf16 pool: from there on
    const int want_end = reach > end4 ? reach : end4;
    const Change c = change_of(f, e, end4, want_end);
    const int v[3] = {in ? c.n_take() : 0, in ? c.n_give() : 0, in && two ? c4.n_give() : 0};
    const Scan<3> sc = block_scan<3>(v, cap, carry, s.tot, lane, wv);
    const bool ok = v[0] == 0 || (long long)sc.before[0] + v[0] <= count;

    // ---- entries: out of the ring, and back behind its last page
    if (in) {
      int32_t* row = a.pool.table + (size_t)b * P;
      if (ok) {
        const int at = wrapped((long long)head + sc.before[0], a.pool.n_pages);
        if (v[0] > 0) {
          do_move(a.pool, Move{row + c.take_lo, c.n_take_lo, at, 0}, false, s);
          do_move(a.pool, Move{row + c.take_hi, c.n_take_hi, wrapped((long long)at + c.n_take_lo, a.pool.n_pages), 0}, false, s);
          taken += v[0];
        }
      } else {
        ++refused;
        if (a.pool.spill >= 0) {
          do_move(a.pool, Move{row + c.take_lo, c.n_take_lo, 0, 2}, false, s);
          do_move(a.pool, Move{row + c.take_hi, c.n_take_hi, 0, 2}, false, s);
        }
      }
      if (v[1] > 0 && (long long)sc.before[1] + v[1] <= a.pool.n_pages - count) {  // (always, unless the arrays name more pages than there are)
        const int at = wrapped(wrapped((long long)head + count, a.pool.n_pages) + (long long)sc.before[1], a.pool.n_pages);
        do_move(a.pool, Move{row + c.give_lo, c.n_give_lo, at, 1}, false, s);
        do_move(a.pool, Move{row + c.give_hi, c.n_give_hi, wrapped((long long)at + c.n_give_lo, a.pool.n_pages), 1}, false, s);
      }
      // refused: it keeps what it holds of what it should hold
      const int nf = ok ? end4 : (f > end4 ? (f < want_end ? f : want_end) : end4);
      const int ne = ok ? want_end : (e < want_end ? e : want_end);
      a.pool.first[b] = nf;
      a.pool.end[b] = ne > nf ? ne : nf;
      if (two) {
        int32_t* row4 = a.packed.table + (size_t)b * P;
        if (ok4) {
          const int at = wrapped((long long)head4 + rank4, a.packed.n_pages);
          if (c4.n_take() > 0) {
            do_move(a.packed, Move{row4 + c4.take_lo, c4.n_take_lo, at, 0}, true, s);
            do_move(a.packed, Move{row4 + c4.take_hi, c4.n_take_hi, wrapped((long long)at + c4.n_take_lo, a.packed.n_pages), 0}, true, s);
            taken4 += c4.n_take();
          }
        } else {
          ++refused4;
        }
        if (v[2] > 0 && (long long)sc.before[2] + v[2] <= a.packed.n_pages - count4) {
          const int at = wrapped(wrapped((long long)head4 + count4, a.packed.n_pages) + (long long)sc.before[2], a.packed.n_pages);
          do_move(a.packed, Move{row4 + c4.give_lo, c4.n_give_lo, at, 1}, true, s);
          do_move(a.packed, Move{row4 + c4.give_hi, c4.n_give_hi, wrapped((long long)at + c4.n_give_lo, a.packed.n_pages), 1}, true, s);
        }
        a.packed.first[b] = f4;
        a.packed.end[b] = end4;
      }
    }
    __syncthreads();
    const int n_long = s.n_long;
    for (int k = wv; k < n_long; k += kFitWaves) {
      const Move m = s.longs[k];
      const FitPool& p = s.of_packed[k] ? a.packed : a.pool;
      for (int i = lane; i < m.n; i += kWave) move_one(p, m, i);
    }
    __syncthreads();  // the list is filled anew; a sequence's entries are in place
  }

  // ---- the rings
  const int lane_sums[4] = {taken, taken4, refused, refused4};
  int* s_sum = s.tot;
  if (tid < 4) s_sum[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (lane_sums[k]) atomicAdd(s_sum + k, lane_sums[k]);
  __syncthreads();
  if (tid == 0) {
    auto put = [](const FitPool& p, int head_, int count_, int taken_, int given, int refused_) {
      const int room_ = p.n_pages - count_;
      p.state[0] = wrapped((long long)head_ + taken_, p.n_pages);
      p.state[1] = count_ - taken_ + (given < room_ ? given : room_);
      p.state[2] = refused_;
    };
    put(a.pool, head, count, s_sum[0], carry[1], s_sum[2]);
    if (two) put(a.packed, head4, count4, s_sum[1], carry[2], s_sum[3]);
    if (s_sum[2] || s_sum[3]) *a.status = 3;  // MTLA_ERR_CAPACITY
  }
}

// Rows of the bf16 pool that the new tokens go to; -1 for padding and where the sequence holds no page.  grid = (pieces of the tokens, batch)
__global__ __launch_bounds__(kBlock) void slot_map_kernel(FitArgs a) {
  const int b = blockIdx.y;
  const int n = new_rows(a.n_new ? a.n_new[b] : a.n_new_max, a.n_new_max);
  const int len = a.seq_len[b], f = a.pool.first[b], e = a.pool.end[b];
  const int32_t* row = a.pool.table + (size_t)b * a.max_pages;
  int64_t* out = a.slot_map + (size_t)b * a.n_new_max;
  for (int t = blockIdx.x * kBlock + threadIdx.x; t < a.n_new_max; t += gridDim.x * kBlock) {
    const long long at = (long long)len + t;
    long long v = -1;
    if (t < n && len >= 0 && at < (long long)a.max_slots * a.stride) {
      const int slot = (int)((unsigned)at / (unsigned)a.stride), k = slot >> a.shift;
      if (k >= f && k < e) v = ((long long)row[k] << a.shift) + (slot & ((1 << a.shift) - 1));
    }
    out[t] = v;
  }
}

}  // namespace

hipError_t launch_pages_fit(const FitArgs& a, hipStream_t st) {
  static DeviceSet lds_allowed;
  hipError_t e = allow_lds(&pages_fit_kernel, sizeof(FitShared), lds_allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_fit_kernel, dim3(1), dim3(kFitBlock), sizeof(FitShared), st, a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.slot_map) return e;
  const int parts = (a.n_new_max + 4 * kBlock - 1) / (4 * kBlock);
  hipLaunchKernelGGL(slot_map_kernel, dim3(parts, a.batch), dim3(kBlock), 0, st, a);
  return hipGetLastError();
}

}  // namespace mtla
