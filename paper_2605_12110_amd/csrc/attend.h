// Dense attention of new rows over the paged cache: what the host plans and the kernels in attend.hip take.
#pragma once
#include "common.h"

namespace absb {

// Work-groups of 256 threads that a launch can have: its threads are counted in 32 bits.
constexpr int64_t MAX_WGS = (int64_t(1) << 24) - 1;

// A phase of a call: the rows of "owners" against the keys that an owner holds.  Own keys: an owner is a request.  Shared keys: an
// owner is a group of requests, its keys the group's prefix.  An owner's rows, n tokens of G query heads a KV head, are cut
// into tiles; tiles have slots, owner after owner.  A wave adds up the tiles of DENSE_OWNERS owners; with more of them owner o's
// are slots floor(row_off[o] * G / tile) + o and on, which leaves room for all of them and can be searched; a slot without rows
// leaves at once.  (Slots without rows upset the order in which work-groups find places: of 544 with tiles of 4096 keys, 512 on
// the chip at a time, some that had room in the first round went in the second: 209 us, and 164 without.)
constexpr int DENSE_OWNERS = 63;
struct AttendPhase {
  int32_t owners;
  int32_t log2_tile;  // rows (token, query head of the group) of a work-group: 128, or 32 that its four waves share
  int32_t splits;  // of a tile's keys, a work-group each
  int32_t chunk;   // keys of a split of the longest tile, a multiple of 128; a tile's own are divided evenly
  int32_t stream;  // 1: rows are read past the caches
  int64_t slots;   // tiles, empty ones included
  int64_t whole;   // of them, the last: not cut, their results written straight to the output.  (All cut or none, but for equal
                   // tiles that fill the chip and a bit: then the few that would have it to themselves afterwards are.)
};

// Of a partial result: maximum in log2 units, sums of the weights as rounded for the product with V and before rounding.
struct PartSums {
  float m, l, lx;
};

struct AttendPlan {
  AttendPhase shared, own;  // shared.owners = 0: no such phase
  int32_t parts;            // partial results of a row: shared.splits + own.splits
  int64_t rows;
  int64_t cut_rows;         // rows of q up to the last that has partial results
  size_t ws_part_ml, ws_bytes;  // ws_bytes = 0: one part, written straight to the output
};

struct AttendParams {
  const uint16_t* q;
  const char *k, *v;
  const int32_t *page_table, *seq_lens, *row_off;
  const int32_t *first, *len;  // groups: first request, shared tokens (null: none)
  const int32_t *prefix_lens, *doc_start;
  const float* slopes;
  uint16_t* out;
  float* lse;
  float* part_o;   // [cut rows][Hq][parts][128], not normalised
  float* part_ml;  // [cut rows][Hq][parts] PartSums
  int64_t s_page, s_head, s_tok;  // bytes
  int32_t groups, pt_stride, Hq, Hkv, G, log2_page;
  int32_t inv_G;                  // 2^16 / G, rounded up
  int32_t window, parts;
  float scale_log2;               // sm_scale * log2(e)
  float cap_log2, cap_in;         // cap * log2(e), 2 log2(e) sm_scale / cap (capped only)
  uint32_t shared_units;          // work-groups of the first phase, ahead of the second's
  AttendPhase shared, own;
};

ABSB_HIDDEN int launch_attend(const AttendParams& p, const AttendPlan& plan, int dtype, float softcap, hipStream_t stream);

}  // namespace absb
