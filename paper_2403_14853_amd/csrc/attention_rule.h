// How the attention's passes share the heads out over lanes (attention.h): host arithmetic only, so that the rules can be checked without a device.
#pragma once
#include <stdint.h>

namespace isp_dev {

// Lanes that hold a head of dh columns, w of them to a lane: a power of two, for the sums over them.
inline int att_lanes_per_head(int dh, int w) {
  int l = 1;
  while (l * w < dh) l *= 2;
  return l;
}

// Query heads of a key head that a lane takes at once: as many of `most` (4 or 2) as divide them.  The forward and the columns' pass take four, which reads
// the gathered rows once for all; the rows' pass two, as four of them need 220 registers in 16 bits and 270 in fp32.  us with four / two: 1 M rows, 17 M entries, 8 query
// heads on 2 of 16, bf16: forward 720 / 884, rows 1113 / 1142, columns 1294 / 2364 (in two passes); rows, fp16 1094 / 1140; 169 k, 2.4 M, fp32 325 / 249; 60 k, 6 M, 4 on 1 of 64, bf16 568 / 517, fp32
// 1010 / 695.
inline int att_share(int group, int most) { return group % 4 == 0 && most == 4 ? 4 : group % 2 == 0 ? 2 : 1; }

// Passes over 16-bit operands with one query head to a key head give a lane eight columns instead of four where that leaves eight lanes to a group and rows average 16
// entries: half the lanes, so twice the entries per step, and half the exponentials, for 30 registers more.  The columns' pass then keeps two steps in flight instead of four
// (8 of 16 on 6 M entries 301 / 237 us with four / two, 2 of 128 631 / 491).
// us with four / eight, bf16, forward, rows, columns: R-MAT, 169 k rows, 2.4 M entries: 8 heads of 8 72 / 62, 87 / 81, 88 / 86; 8 of 16 117 / 108, 134 / 121, 157 / 150; 3 of 20 110 / 94, 130 / 111, 149 / 138; 1 of
// 64 68 / 60, 83 / 76, 89 / 85; 1 of 256, fp16 268 / 242, 301 / 256, 350 / 293; 60 k, 6 M: 8 of 16 238 / 173, 265 / 211, 322 / 237; 2 of 128 519 / 348, 585 / 412, 706 / 491; 1 of 50 146 / 118, 163 / 147, 180 / 165; 1 M,
// 17 M: 8 of 16 826 / 813, 948 / 866, 1155 / 1078; 233 k, 40 M: 3 of 20, fp16 1383 / 867, 1622 / 1215, 1984 / 1515; 20 k, 400 k: 3 of 20 22.8 / 17.9, 25.8 / 24.8, 31.3 / 30.3.  Forward with four lanes to a group: 169 k,
// 2.4 M: 2 of 16 52.1 / 53.9; uniform, 10 entries a row, 100 k, 1 M: 8 of 8 47.3 / 49.0, 4 of 32 87.4 / 90.2.  fp32 operands wait for their gathers (forward, 8 of 16 251 / 251, 8 of 8 110 / 112; 60 k, 6 M: 8 of 16
// 334 / 351, 1 of 64 157 / 170).
// live_rows: rows with entries, of the matrix whose rows the pass goes over.
inline bool att_wide(int element_bytes, int group, int kv_heads, int dh, int64_t nnz, int64_t live_rows) {
  return element_bytes == 2 && group == 1 && dh >= 8 && att_lanes_per_head(dh, 8) * kv_heads >= 5 && nnz >= 16 * live_rows;
}

// The forward copies K and V next to each other into rows of whole lines (pitch: att_packed_pitch) where that saves its gathers more than it costs.
// A row of x bytes lies on ceil(x / 128) lines where rows start on lines, else on x / 128 + 1 on average; the copy moves its bytes at 4.5 TB/s, and its launch is 4 us.
// A line less per entry saves 1 ps where the launch is bound by the vector ALU or L2 has the rows, up to 6 where gathers miss; the rule takes 1.5.  us with K and V as they
// lie / side by side, and the copy: 233 k columns, 40 M entries: 3 heads of 20, 16-bit 981 / 837, 30; 1 of 16 459 / 358, 14; 200 k, 10 M: 4 of 7, fp32 257 / 162, 25; uniform, 100 k, 6 M: 1 of
// 32, 16-bit 149 / 84, 10; 60 k, 6 M: 1 of 50, 16-bit 127 / 108, 10; not taken: 1 M, 17 M: 2 key heads of 16, 16-bit 640 / 629, 64, and 1 of 32 337 / 241, 64; 169 k, 2.4 M: 3 of 20, 16-bit 95 / 82, 23, and 2 of
// 50, fp32 237 / 204, 68; 60 k, 6 M: 3 of 33, fp32 434 / 434, 27.
constexpr int ATT_LINE = 128;
inline int64_t att_packed_pitch(int64_t row_bytes) { return (2 * row_bytes + ATT_LINE - 1) / ATT_LINE * ATT_LINE; }
// whole: rows of K and V start on lines
inline bool att_packs(int64_t row_bytes, bool whole, int64_t nnz, int64_t n_cols) {
  const double lines = whole ? (double)((row_bytes + ATT_LINE - 1) / ATT_LINE) : (double)row_bytes / ATT_LINE + 1.;
  const double saved = 2. * lines - (double)(att_packed_pitch(row_bytes) / ATT_LINE);
  return 1.5e-6 * saved * (double)nnz > 4. + (double)n_cols * (double)(2 * row_bytes + att_packed_pitch(row_bytes)) / 4.5e6;
}

}  // namespace isp_dev
