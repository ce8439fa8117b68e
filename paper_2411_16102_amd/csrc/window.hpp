// Kernels of bs_window_attention and bs_rope_append (see blendstep_stream.h).
#pragma once
#include <stdint.h>
#include <hip/hip_runtime.h>
#include "attn.hpp"

namespace bs {

// One unit of narrow work: a run of pages seen by at most 16 / group rows of one sequence (a wavefront per unit and
// KV head).  Tokens are counted from the run's first page; sink pages and window pages stand one behind the other in it.
struct WindowItem {
  int32_t row0, n_rows;
  int32_t page_off, n_pages;  // its part of item_pages; at most 64
  int32_t at;                 // where row0 stands
  int32_t sinks;              // tokens below this are seen whatever the window
  int32_t state;              // partial state of row0 (one per row behind it), or -1: the unit has everything its rows see
  int32_t pad;
};

struct WindowArgs {
  AttnShape s;
  const WindowItem *items;
  const int32_t *item_pages;
  int n_items, window;
  const uint16_t *q, *kv_pool;
  uint16_t *out;
  int64_t q_stride, out_stride;  // elements of a row
  const int32_t *joins;          // [n_joins][4] = (row, first state, states between two of a row, states)
  int n_joins;
  float *part_acc, *part_m, *part_l;  // [states][Hq][dh], [states][Hq]
};
hipError_t launch_window_units(const WindowArgs &a, hipStream_t stream);
hipError_t launch_window_join(const WindowArgs &a, hipStream_t stream);

// Rows of one sequence whose keys and values go to one page, at most 16, or rows that append nothing (page -1).
struct RopeItem {
  int32_t row0, n_rows, page, slot0;
};

struct RopeArgs {
  int n_rows, n_items, n_q_heads, n_kv_heads, head_dim;
  bool whole;                      // eight pairs from a multiple of eight on share an axis
  const RopeItem *items;
  const float *cos, *sin;          // [max_positions][head_dim / 2]
  const int32_t *positions;        // [n_axes][n_rows]
  const int32_t *axis_of_pair;     // [head_dim / 2]
  const uint16_t *qkv;
  uint16_t *q, *kv_pool;
  int64_t qkv_stride, q_stride;
};
hipError_t launch_rope_append(const RopeArgs &a, hipStream_t stream);

}  // namespace bs
