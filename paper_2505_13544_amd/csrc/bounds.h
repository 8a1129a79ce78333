// What lengths and starts out of the caller's arrays count as.  They are read on the device, where nothing can return an error
// in front of the launch, so every kernel takes them through the functions here and all of them agree.
#pragma once

namespace mtla {

// The live slots of a sequence of `len` tokens.  A length outside 0 .. max_slots * stride counts as the nearer end.
[[gnu::always_inline]] constexpr int live_slots(int len, int stride, int max_slots) {
  const int n = len > 0 ? (int)((unsigned)(len - 1) / (unsigned)stride) + 1 : 0;
  return n < max_slots ? n : max_slots;
}

// Chunks that `live` slots have, for any two ints (a caller's chunk may be the largest multiple of 32).
[[gnu::always_inline]] constexpr int chunks_of(int live, int chunk) { return live / chunk + (live % chunk != 0 ? 1 : 0); }

// A page count or a page's place in its table row, as the nearest that the row has or ends with.  (Also in front of any sum: max_pages and a
// launch's pages together stay far from what an int holds, a caller's word does not.)
[[gnu::always_inline]] constexpr int pages_inside(int page, int max_pages) { return page < 0 ? 0 : (page < max_pages ? page : max_pages); }

// Slots of a sequence that lie in packed pages: `n_packed` pages of 2^shift slots, taken as [0, max_pages].
[[gnu::always_inline]] constexpr int packed_slots(int n_packed, int max_pages, int shift, int live) {
  const long long end = (long long)pages_inside(n_packed, max_pages) << shift;
  return end < live ? (int)end : live;
}
// Whether they end inside a chunk: what the chunk holds behind them is a piece of its own then, behind those of the chunks.
[[gnu::always_inline]] constexpr bool open_piece(int packed, int live, int chunk) { return packed > 0 && packed < live && packed % chunk != 0; }

// May `n` tokens be appended to a sequence of `len`?  0, or the status that refuses them (the sequence is left untouched):
// 1 (MTLA_ERR_INVALID_ARG) for a length below zero, 3 (MTLA_ERR_CAPACITY) for more than the capacity holds.
[[gnu::always_inline]] constexpr int append_status(int len, int n, int stride, int max_slots) {
  return len < 0 ? 1 : ((long long)len + n > (long long)max_slots * stride ? 3 : 0);
}

// The slots in front of a sequence's new rows.  A start outside the `past` slots that the call declared counts as all of them
// (the front launch raises the status word): no kernel leaves its arrays, and the sequence's rows are meaningless.  (As an
// unsigned number a start below zero lies above every slot that past * stride < 2^31 tokens can have.)
[[gnu::always_inline]] constexpr int slots_inside(int pos0, int stride, int past) {
  const unsigned k = (unsigned)pos0 / (unsigned)stride;
  return k < (unsigned)past ? (int)k : past;
}
// The tokens in front of them: the start itself, or those of the whole past.
[[gnu::always_inline]] constexpr int start_inside(int pos0, int stride, int past) {
  return pos0 >= 0 && (unsigned)pos0 / (unsigned)stride <= (unsigned)past ? pos0 : past * stride;
}

// The new rows of a sequence, of at most T.  A sequence's part of past + T rows then has slots_inside(..) + new_rows(..) in use.
[[gnu::always_inline]] constexpr int new_rows(int n_new, int T) { return n_new < 0 ? 0 : (n_new < T ? n_new : T); }

}  // namespace mtla
