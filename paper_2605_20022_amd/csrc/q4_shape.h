// How the attention over a 4-bit cache is cut into pieces, and what the host has to reserve for them (internal; plain C++).
#pragma once
#include <stddef.h>

namespace fd {

constexpr int Q4_TK = 32;                 // keys of a block
constexpr int Q4_ROWS = 128;              // tile rows of an item
constexpr int Q4_SLOTS = 512;             // work-groups that run at once: two a compute unit
// Units a compute unit up to which it takes one piece (one sequence of 32 768 keys, 64 rows, 99 units: 25.6 us a call, in twice as many pieces 29.1;
// 4 of 8192 to 16 384, 146: 31.3 and 33.1; one of 8192, 272 rows, 420: 60.8 and 58.6).
constexpr int Q4_ALONE = 192;
constexpr int Q4_PIECES = 512;            // pieces aimed at where there are Q4_SLOTS items or more
constexpr int Q4_CLASSES = 4;             // lengths of pieces that are told apart
// A block of own rows takes as long as Q4_OWN of cached ones, the first Q4_OWN_START more (1 sequence of 16 new rows 15.4 us a call, 2 of 272 in 17
// blocks 67.7; counted as cached ones 17.0 and 70.0, the first 6 more 16.0 and 70.0).
constexpr int Q4_OWN = 3, Q4_OWN_START = 4;
constexpr int Q4_MIN_PIECE = 8;           // blocks of a piece, at least, but for the last of a short item (1 sequence of 1024 keys 14.2 us; 6: 15.0, 12: 14.5)
constexpr int Q4_KEPT = 4;                // rounds of 64 sequences whose lengths a wave keeps in LDS

// Items of the largest sequence, partial slots and work-groups that there can be, and the workspace.
struct Q4Shape { long long items, partials, wgs, max_pieces; int rt_max, fixed, unit_shift; size_t off_ml, off_entries, total; };
inline Q4Shape q4_shape(int batch, int num_kv_heads, int group, int total_rows, int max_kv_len, int max_new_rows, int kv_chunk, int head_dim) {
  Q4Shape z;
  const long long tile_rows = (long long)max_new_rows * group;
  z.rt_max = (int)((tile_rows + Q4_ROWS - 1) / Q4_ROWS);
  if (z.rt_max < 1) z.rt_max = 1;
  z.fixed = kv_chunk / Q4_TK;
  const long long seqs = batch < total_rows ? batch : total_rows;       // sequences that have rows
  z.items = seqs * num_kv_heads * z.rt_max;
  const long long blocks = ((long long)max_kv_len + Q4_TK - 1) / Q4_TK + Q4_OWN_START + Q4_OWN * ((max_new_rows + Q4_TK - 1) / Q4_TK);
  // Units of one head's work, a sum in 32 bits over all sequences on the device.  Not even rows that contradict total_rows may make it more than is counted
  // on here (a sum that wraps would cut thousands of pieces an item, with slots outside the workspace): every sequence as many rows and keys as one may have.
  const double rows = max_new_rows < total_rows ? max_new_rows : total_rows;
  const double units = (double)batch * (rows * group / 32 + 2) * 2 * (double)blocks;
  z.unit_shift = 0;
  while (units / (double)(1ll << z.unit_shift) >= 1073741824.0) ++z.unit_shift;
  z.max_pieces = blocks / (z.fixed > 0 ? z.fixed : Q4_MIN_PIECE) + 1;
  if (z.fixed > 0) {
    z.wgs = z.items * z.max_pieces;
    z.partials = z.wgs;
  } else {
    // pieces - 1 of an item are density x units at most, which sum to Q4_PIECES over all items (Q4_SLOTS in one round)
    static_assert(Q4_SLOTS <= Q4_PIECES, "what one round takes is within the bounds of several");
    // (work-groups without a piece are not free, 0.8 us for 528 of them: none where one round is sure to do)
    const bool one_round = z.items < Q4_SLOTS && batch <= 64 * Q4_KEPT;
    z.wgs = one_round ? Q4_SLOTS : z.items + Q4_PIECES;
    z.partials = one_round ? Q4_SLOTS : 2 * Q4_PIECES;                  // an item in c >= 2 pieces: c <= 2 (c - 1)
    const long long most = z.items * z.max_pieces;
    if (most < z.wgs) z.wgs = most;
    if (most < z.partials) z.partials = most;
  }
  auto round = [](size_t x) { return (x + 255) / 256 * 256; };
  z.off_ml = round((size_t)z.partials * Q4_ROWS * head_dim * sizeof(float));
  z.off_entries = z.off_ml + round((size_t)z.partials * Q4_ROWS * 2 * sizeof(float));
  z.total = z.off_entries + round((size_t)(batch > 0 ? batch : 1) * num_kv_heads * z.rt_max * 2 * sizeof(int));
  return z;
}

}  // namespace fd
