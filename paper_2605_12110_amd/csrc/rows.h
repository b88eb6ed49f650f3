// Arguments of the kernels in rows.hip.
#pragma once
#include "common.h"

namespace absb {

struct MapParams {
  const int32_t* before;
  const int32_t* after;
  int32_t* page_table;
  int32_t* ring;  // null: no pages change hands
  const int64_t* cursors;
  int64_t* cursors_out;
  int32_t* row_off;
  int32_t* row_pos;
  int64_t* row_slot;
  int32_t batch, pt_stride, capacity, max_rows, log2_page;
};
ABSB_HIDDEN int launch_map_rows(const MapParams& p, hipStream_t stream);

struct RotateParams {
  const uint16_t *q, *k, *v;
  uint16_t *q_out, *k_cache, *v_cache;
  int64_t q_stride, k_stride, v_stride;  // elements between rows
  int64_t s_page, s_head, s_tok;         // of the caches
  const int32_t* pos;
  const int64_t* slot;
  const double* freq;
  float amplitude;
  int32_t n_rows, nq, nkv;  // nq, nkv: heads to do (0: none)
  int32_t rot, halves, log2_page;
  int32_t parts, heads_per_part;  // a token's heads, cut for as many waves
};
ABSB_HIDDEN int launch_rotate(RotateParams p, int dtype, hipStream_t stream);

}  // namespace absb
