// Kernels of bs_window_attention and bs_rope_append (see blendstep_stream.h).
#pragma once
#include <stdint.h>
#include <hip/hip_runtime.h>
#include "attn.hpp"

namespace bs {

// One unit of narrow work: a run of pages seen by at most 16 / group rows of one sequence (a workgroup per unit and
// KV head).  Tokens are counted from the run's first page; sink pages and window pages stand one behind the other in it.
struct WindowItem {
  int32_t row0, n_rows;
  int32_t page_off, n_pages;  // its part of item_pages
  int32_t at;                 // where row0 stands
  int32_t sinks;              // tokens below this are seen whatever the window
  int32_t state;              // partial state of this unit, or -1: it has everything that its rows see
  int32_t group;              // units with the same rows: first state | number of states << 20
};
constexpr int WINDOW_STATE_BITS = 20;

struct WindowArgs {
  AttnShape s;
  const WindowItem *items;
  const int32_t *item_pages;
  int n_items, window;
  int waves;                     // of a workgroup: 1, 2, 4 or 8, which share its run of pages
  int heads;                     // KV heads of a workgroup (a cache in four bits, see kv4_attn.hip: 1 or 2)
  const uint16_t *q, *kv_pool;
  uint16_t *out;
  int64_t q_stride, out_stride;  // elements of a row
  float *parts;                  // [states][Hkv / heads][dh / 16 + 1][64 lanes][4]: accumulators as the lanes hold them, then (m, l) of a column
  unsigned *counters;            // [states][Hkv / heads], zero between launches
};
hipError_t launch_window_units(const WindowArgs &a, hipStream_t stream);
// Narrow and wide work of a step in one launch (a.waves is 4).
hipError_t launch_window_step(const WindowArgs &a, const WindowPrefillArgs &f, int heads, hipStream_t stream);

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
