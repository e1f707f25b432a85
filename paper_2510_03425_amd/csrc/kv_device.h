// Device-side view of the paged cache (KvPages, KvRows): which rows and pages a sequence has.
#pragma once
#include "device_common.h"
#include "mebp_internal.h"

namespace mebp {

// Row, count and first position of sequence s: never outside the call's rows, whatever `start` holds.
struct KvSeq {
  int row, n, past;
};
DEV KvSeq kv_seq(const KvRows& b, int s) {
  const int lo = min(max(b.start[s], 0), b.rows), hi = min(max(b.start[s + 1], lo), b.rows);
  // (positions and the ends of their tiles stay below 2^31)
  const int past = min(max(b.past[s], 0), 0x7fffff00 - b.max_new);
  return KvSeq{lo, min(hi - lo, b.max_new), past};
}

// Page of 16-token block `blk` of sequence s, or -1 where the table has none for it.
DEV int kv_page(const KvPages& c, const KvRows& b, int s, int blk) {
  const int col = blk >> c.log_blocks;
  if ((unsigned)col >= (unsigned)b.cols) return -1;
  const int p = b.table[s * b.table_ld + col];
  return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}
// The same in two steps, for lookups ahead of their use: what the table says (of its nearest column), and what
// that is worth.
DEV int kv_entry(const KvPages& c, const KvRows& b, int s, int blk) {
  return b.table[s * b.table_ld + min(blk >> c.log_blocks, b.cols - 1)];
}
DEV int kv_page_of(const KvPages& c, const KvRows& b, int entry, int blk) {
  return (blk >> c.log_blocks) < b.cols && (unsigned)entry < (unsigned)c.n_pages ? entry : -1;
}
// Index of a block of head h among all blocks of the pool, fewer than 2^31 (its bytes take 64 bits).
DEV uint32_t kv_block(const KvPages& c, int page, int h, int blk) {
  return (((uint32_t)page * c.heads + h) << c.log_blocks) + (blk & ((1 << c.log_blocks) - 1));
}

}  // namespace mebp
