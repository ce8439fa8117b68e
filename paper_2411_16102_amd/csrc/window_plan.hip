// Entry points of the window operators: validation, the plan of a step, and the launches that work from it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>
#include <vector>

#include "../../include/blendstep_bits.h"
#include "context.hpp"
#include "kv4.hpp"
#include "misc.hpp"
#include "window.hpp"

using namespace bs;

namespace {

constexpr int PAGE = 16;
constexpr int MOST_STATES = 4095;        // of rows whose pages are split (see WindowItem::group)
constexpr int MAX_AXES = 8;
constexpr int32_t MAX_LEN = 1 << 30;    // of lengths and rows, so that sums of two stay in 32 bits
constexpr long STAGE_WORDS = 1 << 16;   // of the plan's pinned memory at first (it grows with the plans)

// What the kernels of a planned step need to know beside the arrays on the device.
struct Planned {
  bool made = false, has_angles = false, whole_axes = true;
  int n_rows = 0, n_rope = 0, n_items = 0, waves = 1, heads = 1, window = 1, sinks = 0;
  int n_work = 0, n_cut = 0, wide_blocks = 0;   // wide work: workgroups per group of heads, blocks of rows that several share, all blocks
  int32_t longest = 0, split_rows = 0;
  long states = 0, cut_states = 0, pages = 0;
  long off_items = 0, off_pages = 0, off_rope = 0, off_positions = 0, off_axis = 0, words = 0;
  long off_work = 0, off_cut = 0, off_row_start = 0, off_kv_len = 0, off_page_start = 0, off_page_ids = 0;
  long at_cut_acc = 0, at_cut_m = 0, at_cut_l = 0, state_floats = 0;  // partial states, in floats
  long off_wide = 0;
  int n_wide = 0;                               // wide units over a cache in four bits
};

}  // namespace

struct bs_window {
  bs_ctx *ctx = nullptr;
  int group = 0;  // channels of a group of the cache in four bits that plans are for; 0: a cache in bf16
  Planned p;
  Staging<HipRuntime> stage;
  int32_t *d_words = nullptr;
  long cap_words = 0;
  float *d_states = nullptr;
  long cap_states = 0;
  unsigned *d_counters = nullptr;
  long cap_counters = 0;
  // host scratch reused across plans
  std::vector<int32_t> words, refs, item_pages, cut, wide_start, wide_pages;
  std::vector<WindowItem> items;
  std::vector<RopeItem> rope;
  struct Rows { int seq, first, n, pages; };  // rows of narrow work that share their units
  std::vector<Rows> rows, wide_rows;          // wide_rows: of wide work over a cache in four bits, two blocks of columns each
  std::vector<WindowItem> wide_items;
  struct Work { int blocks, seq, block, t0, t1, state; };
  std::vector<Work> work;
};

namespace {

int check_batch(bs_ctx *c, const bs_batch *b, int64_t n_pages) {
  if (!b) return ctx_fail(c, BS_EINVAL, "batch is NULL");
  if (b->n_seq < 0 || b->n_rows < 0 || b->n_rows > MAX_LEN) return ctx_fail(c, BS_EINVAL, "bad counts: n_seq=%d n_rows=%d", b->n_seq, b->n_rows);
  if (n_pages < 0 || n_pages > (int64_t)0x7fffffff) return ctx_fail(c, BS_EINVAL, "n_pages=%lld out of range", (long long)n_pages);
  if (b->n_seq == 0) return b->n_rows == 0 ? BS_OK : ctx_fail(c, BS_EINVAL, "n_rows=%d with no sequences", b->n_rows);
  if (!b->row_start || !b->kv_len || !b->page_start) return ctx_fail(c, BS_EINVAL, "a required array is NULL");
  if (b->row_start[0] != 0 || b->page_start[0] != 0) return ctx_fail(c, BS_EINVAL, "CSR arrays must start at 0");
  for (int s = 0; s < b->n_seq; ++s) {
    const int64_t rows = (int64_t)b->row_start[s + 1] - b->row_start[s], pages = (int64_t)b->page_start[s + 1] - b->page_start[s];
    if (rows < 0 || b->row_start[s + 1] > b->n_rows) return ctx_fail(c, BS_EINVAL, "row_start not monotone within n_rows at sequence %d", s);
    if (pages < 0) return ctx_fail(c, BS_EINVAL, "page_start not monotone at sequence %d", s);
    if (b->kv_len[s] < 0 || b->kv_len[s] > MAX_LEN) return ctx_fail(c, BS_EINVAL, "sequence %d: kv_len %d out of range", s, b->kv_len[s]);
    if (pages * PAGE < b->kv_len[s]) return ctx_fail(c, BS_EINVAL, "sequence %d: kv_len %d exceeds its %lld pages", s, b->kv_len[s], (long long)pages);
  }
  if (b->row_start[b->n_seq] != b->n_rows) return ctx_fail(c, BS_EINVAL, "row_start ends at %d, n_rows is %d", b->row_start[b->n_seq], b->n_rows);
  if (b->page_start[b->n_seq] > 0 && !b->page_ids) return ctx_fail(c, BS_EINVAL, "a required array is NULL");
  for (int i = 0; i < b->page_start[b->n_seq]; ++i)
    if (b->page_ids[i] != BS_PAGE_NONE && (b->page_ids[i] < 0 || b->page_ids[i] >= n_pages))
      return ctx_fail(c, BS_EINVAL, "page_ids[%d]=%d outside the pool of %lld pages", i, b->page_ids[i], (long long)n_pages);
  return BS_OK;
}

// pages that a step appends to are there, and named once (refs: zero between calls, so that a plan costs what it names, not what the pool has)
int check_appends(bs_window *w, const bs_batch *b, int64_t n_pages) {
  const int named = b->n_seq > 0 ? b->page_start[b->n_seq] : 0;
  if (w->refs.size() < (size_t)n_pages) w->refs.resize((size_t)n_pages, 0);
  const auto count = [&](int by) {
    for (int i = 0; i < named; ++i)
      if (b->page_ids[i] >= 0) w->refs[b->page_ids[i]] += by;
  };
  const auto check = [&]() -> int {
    for (int s = 0; s < b->n_seq; ++s) {
      const int rows = b->row_start[s + 1] - b->row_start[s];
      if (rows == 0 || b->kv_len[s] == 0) continue;
      for (int pg = std::max(0, b->kv_len[s] - rows) / PAGE; pg <= (b->kv_len[s] - 1) / PAGE; ++pg) {
        const int id = b->page_ids[b->page_start[s] + pg];
        if (id < 0) return ctx_fail(w->ctx, BS_EINVAL, "sequence %d appends to page %d of its table, which was given up", s, pg);
        if (w->refs[id] != 1) return ctx_fail(w->ctx, BS_EINVAL, "sequence %d appends into page %d, which is referenced more than once", s, id);
      }
    }
    return BS_OK;
  };
  count(1);
  const int rc = check();
  count(-1);
  return rc;
}

// The pages that rows at positions [p0, p1] see: the first n_sink, then [first, last].
struct Seen {
  int n_sink, first, last;
  int pages() const { return n_sink + last - first + 1; }
  int left_out() const { return PAGE * (first - n_sink); }  // tokens between the two parts
  int page(int i) const { return i < n_sink ? i : first + i - n_sink; }
};
Seen seen_by(int p0, int p1, int window, int sinks) {
  if (p1 < 0) return {0, 0, -1};
  const int first = std::max(0, p0 - window + 1) / PAGE;
  return {std::min((int)(((int64_t)sinks + PAGE - 1) / PAGE), first), first, p1 / PAGE};
}

int check_seen(bs_window *w, int seq, const int32_t *table, const Seen &seen) {
  for (int i = 0; i < seen.pages(); ++i) {
    const int pg = seen.page(i);
    if (table[pg] < 0) return ctx_fail(w->ctx, BS_EINVAL, "sequence %d: a row sees page %d of its table, which was given up", seq, pg);
  }
  return BS_OK;
}

int too_large(bs_window *w) { return ctx_fail(w->ctx, BS_EUNSUPPORTED, "the step is too large for one plan"); }

// Rows [j, end) of a sequence as narrow work, at most `per_unit` in a unit.
int add_rows(bs_window *w, const bs_batch *b, int s, int j, int end, int per_unit, std::vector<bs_window::Rows> *to = nullptr) {
  const int rows = b->row_start[s + 1] - b->row_start[s];
  for (; j < end; j += per_unit) {
    const int n = std::min(per_unit, end - j), p0 = b->kv_len[s] - rows + j;
    const Seen seen = seen_by(p0, p0 + n - 1, w->p.window, w->p.sinks);
    if (const int rc = check_seen(w, s, b->page_ids + b->page_start[s], seen)) return rc;
    (to ? *to : w->rows).push_back({s, j, n, seen.pages()});
  }
  return BS_OK;
}

// How narrow work is cut: wavefronts of a workgroup, pages of a unit, and the microseconds that are expected of it.  Timed for 1 to 256 streams
// of four head layouts, windows of 64 to 4096, each with 1 to 8 wavefronts and 4 to 256 pages: within 2 % of the best of them on
// average, 11 % at worst (one stream, window 1024, 8 KV heads: 6 units of 12 pages 9.2 us, one of 66 on eight wavefronts 18; 64 of window 4096: whole
// on eight 169, halves 187).  84 batches of 200 to 2048 streams of 1 to 1100 pages, most of them unequal: 2.6 % on average, 10 %
// at worst (one stream of 100 pages beside 255 of 4, 8 KV heads: whole 38.4 us, cut 20.0; one of 256 beside 255 of 32: 139 and 101; 256 of 64 each: 163
// whole, halves 190).
struct Division {
  int waves, pages;
  double us;
  int heads = 1;  // KV heads of a workgroup
};
Division divide(const std::vector<bs_window::Rows> &rows, int hkv, int dh, int n_cu) {
  int64_t all = 0, once = 0;  // pages of all units; without those that rows of the same sequence have seen before
  int longest = 0, last = -1;
  for (const bs_window::Rows &r : rows) {
    all += r.pages;
    once += r.seq == last ? std::min(r.pages, 1) : r.pages;
    last = r.seq;
    longest = std::max(longest, r.pages);
  }
  // A CU streams 36 GB/s of pages however many ask, a unit's pages go through one; a join waits for a round trip and one more for every
  // eight units or so.
  // Where units are many, each is one wavefront's, which takes as long beside others as the memory keeps it waiting.
  const double us_alone = dh == 128 ? 0.27 : 0.22;
  const double us_per_page = dh == 128 ? 0.23 : 0.13, all_us = (double)once * hkv * dh * (4.0 * PAGE / 5.9e6);
  double best = 0;
  Division div = {1, std::max(2, longest), 0.0};
  int64_t n_units = (int64_t)rows.size() * hkv;
  for (int n : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
    const int pages = std::max(2, 2 * ((longest + 2 * n - 1) / (2 * n)));
    if (n > 1 && pages < 4) break;
    int64_t units = 0, joined = 0;
    for (const bs_window::Rows &r : rows) {
      const int k = std::max(1, (r.pages + pages - 1) / pages);
      units += k;
      joined += k > 1 ? k : 0;
    }
    units *= hkv;
    joined *= hkv;
    double cost;
    if (units <= 4 * (int64_t)n_cu) {
      const double rounds = (double)((units + n_cu - 1) / n_cu);
      cost = std::max(all_us, us_per_page * pages * rounds) + (n > 1 ? 2.0 + 0.25 * n + 0.004 * (double)units : 0.0);
    } else {
      cost = std::max({all_us, us_per_page * (0.5 * pages + (double)all * hkv / n_cu), us_alone * std::min(pages, longest) + 0.7 * all_us}) +
             (joined ? 2.0 + 0.25 * n + 0.0045 * (double)joined : 0.0);
    }
    if (n == 1 || cost < best) {
      best = cost;
      div.pages = std::max(2, pages);
      n_units = units;
    }
  }
  // Wavefronts of a workgroup: about 16 to 32 pages each, and no more than two for a SIMD.
  div.waves = div.pages <= 2 ? 1 : div.pages <= 64 ? 2 : div.pages <= 128 ? 4 : 8;
  while (div.waves > 1 && n_units * div.waves > 12 * (int64_t)n_cu) div.waves /= 2;
  div.us = best;
  return div;
}

// Narrow work over a cache in four bits: microseconds that the chip's SIMDs compute for so many pages of units (rows that share their pages, which the caches then hold, are bound by it)
double compute4_us(const bs_layer_cfg &g, int group, int heads, int64_t pages, int n_cu) {
  return ((g.head_dim == 128 ? 0.27 : 0.16) + 0.055 * (g.head_dim / group)) * (heads == 2 ? 0.75 : 1.0) * (double)pages * g.n_kv_heads / (4.0 * n_cu);
}
constexpr double UNITS4_US = 3.36;  // of any division

// The division over a cache in four bits, whose units read less and compute more: KV heads that share a wavefront too, where the columns of two have
// room (see kv4_attn.hip).  A wavefront takes `step` microseconds a page; what its registers allow is on the chip at a time, in rounds; or the bytes
// are longer.  Fitted to 4000 batches of 1 to 300 streams (up to 16000 tokens, equal and unequal, five head layouts, all groups) timed in every
// division with 1, 2 and 4 wavefronts: 3.4 % off the best on average, 15 % for one in twenty, 34 % at worst; the division of the cache in bf16 is 29 % off.
Division divide4(const std::vector<bs_window::Rows> &rows, const bs_layer_cfg &g, int group, int n_cu) {
  int64_t once = 0, every = 0;
  int longest = 0, last = -1, most_rows = 1;
  for (const bs_window::Rows &r : rows) {
    every += r.pages;
    once += r.seq == last ? std::min(r.pages, 1) : r.pages;
    last = r.seq;
    longest = std::max(longest, r.pages);
    most_rows = std::max(most_rows, r.n);
  }
  const int hkv = g.n_kv_heads, dh = g.head_dim;
  const bool two = most_rows * (g.n_q_heads / hkv) <= 8 && hkv % 2 == 0;
  const double bytes_us = 0.133e-6 * (double)once * hkv * kv4_head_bytes(dh, group);
  Division best = {1, std::max(2, longest), 0.0, 1};
  bool any = false;
  for (int n : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128}) {
    const int pages = std::max(2, 2 * ((longest + 2 * n - 1) / (2 * n)));
    if (n > 1 && pages < 4) break;
    int64_t all = 0, joined = 0;
    int most = 0;
    for (const bs_window::Rows &r : rows) {
      const int k = std::max(1, (r.pages + pages - 1) / pages);
      all += k;
      joined += k > 1 ? k : 0;
      most = std::max(most, k);
    }
    for (int waves : {1, 2, 4}) {
      if (waves > 1 && pages < 2 * waves) break;
      int64_t steps = 0;  // pages that the first wavefront of every unit takes
      int longest_steps = 0;
      for (const bs_window::Rows &r : rows) {
        const int k = std::max(1, (r.pages + pages - 1) / pages), s = ((r.pages + k - 1) / k + 2 * waves - 1) / (2 * waves) * 2;
        steps += (int64_t)k * s;
        longest_steps = std::max(longest_steps, s);
      }
      for (int heads = 1; heads <= (two ? 2 : 1); ++heads) {
        const double step = (0.272 + 0.043 * (dh / group)) * (dh == 128 ? 1.0 : 0.707) * (heads == 2 ? 1.34 : 1.0);
        const double units = (double)all * hkv / heads, slots = 4.0 * n_cu * kv4_resident(dh, group, heads) / waves;
        const double alone = 1.44 + step * longest_steps, mean = 2.91 + 1.18 * step * (double)steps / std::max<int64_t>(1, all);
        const double load = std::max(compute4_us(g, group, heads, every, n_cu), mean * (units / slots + 0.31 * (std::ceil(units / slots) - units / slots)));
        const double us = UNITS4_US + std::max({bytes_us + 0.087 * alone, alone, load}) + 0.54 * std::min(bytes_us, load) +
                          (joined ? 0.75 + 0.22 * most + 0.0011 * (double)joined * hkv / heads : 0.0);
        if (!any || us < best.us) best = {waves, pages, us, heads};
        any = true;
      }
    }
  }
  return best;
}

// The units of the rows of narrow work.
int add_units(bs_window *w, const bs_batch *b, const Division &div) {
  Planned &p = w->p;
  p.waves = div.waves;
  for (const bs_window::Rows &r : w->rows) {
    const int r0 = b->row_start[r.seq], p0 = b->kv_len[r.seq] - (b->row_start[r.seq + 1] - r0) + r.first;
    const int32_t *table = b->page_ids + b->page_start[r.seq];
    const Seen seen = seen_by(p0, p0 + r.n - 1, p.window, p.sinks);
    int n_units = std::max(1, (r.pages + div.pages - 1) / div.pages);
    n_units = std::min(n_units, MOST_STATES);
    if (n_units > 1 && p.states + n_units >= 1L << WINDOW_STATE_BITS) n_units = 1;
    for (int k = 0; k < n_units; ++k) {
      // whole pairs of pages, in nearly equal shares
      const int64_t pairs = (r.pages + 1) / 2;
      const int lo = (int)(2 * (pairs * k / n_units)), hi = std::min(r.pages, (int)(2 * (pairs * (k + 1) / n_units)));
      WindowItem it{};
      it.row0 = r0 + r.first;
      it.n_rows = r.n;
      it.page_off = (int32_t)w->item_pages.size();
      it.n_pages = hi - lo;
      it.at = p0 - seen.left_out() - PAGE * lo;
      it.sinks = std::max(0, std::min(p.sinks - PAGE * lo, PAGE * (hi - lo)));
      it.state = n_units > 1 ? (int32_t)(p.states + k) : -1;
      it.group = n_units > 1 ? (int32_t)((uint32_t)p.states | (uint32_t)n_units << WINDOW_STATE_BITS) : 0;
      w->items.push_back(it);
      for (int i = lo; i < hi; ++i) w->item_pages.push_back(table[seen.page(i)]);
      p.longest = std::max(p.longest, it.n_pages);
    }
    if (n_units > 1) {
      p.states += n_units;
      p.split_rows += r.n;
    }
    if (w->item_pages.size() > (size_t)MAX_LEN || w->items.size() > (size_t)MAX_LEN) return too_large(w);
  }
  // longest first: the short ones then fill the end of the launch
  std::stable_sort(w->items.begin(), w->items.end(), [](const auto &x, const auto &y) { return x.n_pages > y.n_pages; });
  // wide units over a cache in four bits
  w->wide_items.clear();
  for (const bs_window::Rows &r : w->wide_rows) {
    const int r0 = b->row_start[r.seq], p0 = b->kv_len[r.seq] - (b->row_start[r.seq + 1] - r0) + r.first;
    const Seen seen = seen_by(p0, p0 + r.n - 1, p.window, p.sinks);
    WindowItem it{};
    it.row0 = r0 + r.first;
    it.n_rows = r.n;
    it.page_off = (int32_t)w->item_pages.size();
    it.n_pages = r.pages;
    it.at = p0 - seen.left_out();
    it.sinks = std::max(0, std::min(p.sinks, PAGE * r.pages));
    it.state = -1;
    w->wide_items.push_back(it);
    for (int i = 0; i < r.pages; ++i) w->item_pages.push_back(b->page_ids[b->page_start[r.seq] + seen.page(i)]);
    if (w->item_pages.size() > (size_t)MAX_LEN) return too_large(w);
  }
  std::stable_sort(w->wide_items.begin(), w->wide_items.end(), [](const auto &x, const auto &y) { return x.n_pages > y.n_pages; });
  return BS_OK;
}

// How a step's rows are divided between the two kinds of work.
struct Route {
  int per_unit;   // rows of a narrow unit
  int heads, rows;  // of a wide workgroup: query heads of one KV group, query rows
  int per_wide;     // rows of a wide unit over a cache in four bits
};
Route route_of(const bs_layer_cfg &g) {
  const int grp = g.n_q_heads / g.n_kv_heads, heads = grp % 4 == 0 ? 4 : grp % 2 == 0 ? 2 : 1;
  return {std::max(1, 16 / grp), heads, 64 * (4 / heads), 4 * std::max(1, 16 * KV4_ROW_BLOCKS / grp)};
}

// The rows of a longer segment as blocks for wide workgroups; rows of blocks that stand wholly in front of their sequence see nothing:
// units without pages.
int add_blocks(bs_window *w, const bs_batch *b, int s, const Route &r) {
  Planned &p = w->p;
  const int rows = b->row_start[s + 1] - b->row_start[s];
  const int32_t *table = b->page_ids + b->page_start[s];
  for (int k = 0; k * r.rows < rows; ++k) {
    const int j = k * r.rows, end = std::min(rows, j + r.rows), p0 = b->kv_len[s] - rows + j, p1 = b->kv_len[s] - rows + end - 1;
    if (p1 < 0) {
      if (const int rc = add_rows(w, b, s, j, end, r.per_unit)) return rc;
      continue;
    }
    const Seen seen = seen_by(p0, p1, p.window, p.sinks);
    if (const int rc = check_seen(w, s, table, seen)) return rc;
    w->work.push_back({(seen.pages() + 1) / 2, s, k, 0, 0, -1});
    p.pages += seen.pages();
    ++p.wide_blocks;
  }
  return BS_OK;
}

// How the blocks of wide work are cut into ranges of their pages, workgroups of their own: 32-token blocks of a range (0: not cut), and the
// microseconds that are expected.  A workgroup takes 1.25 us per 32 tokens (64-wide heads: 1.15, two to a CU) and two such
// to begin; states and their merge cost 10 us and 0.02 for every workgroup.  Timed for segments of 6 to 300 rows, 1 to 16 of them, windows of
// 1024 to 4096: 64 rows behind 4096 tokens, 8 KV heads, 165 us whole, 28 in ranges of 8; four segments of 300 rows 149 whole, 168 in halves.
struct Cut {
  int blocks;
  double us;
};
Cut cut_choice(const std::vector<bs_window::Work> &work, int wg_per_work, int dh, int rows, int n_cu) {
  const double us = dh == 64 ? 1.15 : 1.25;
  const int64_t slots = dh == 64 ? 2 * n_cu : n_cu;
  int64_t all = 0;
  int longest = 0;
  for (const bs_window::Work &k : work) {
    all += k.blocks + 2;
    longest = std::max(longest, k.blocks);
  }
  Cut best = {0, us * std::max((double)(longest + 2), (double)(all * wg_per_work) / slots)};
  for (int t : {4, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96}) {
    if (t >= longest || longest >= 65536) break;
    int64_t ranges = 0, states = 0;
    for (const bs_window::Work &k : work) {
      const int n = (k.blocks + t - 1) / t;
      ranges += n;
      states += n > 1 ? n : 0;
    }
    if (states * rows > MAX_LEN / 64) continue;
    const int64_t wgs = ranges * wg_per_work;
    const double cost = us * (t + 2) * (double)((wgs + slots - 1) / slots) + 10.0 + 0.02 * (double)wgs;
    if (cost < best.us) best = {t, cost};
  }
  return best;
}

// The microseconds that are expected of wide units over a cache in four bits: what all of them take of the chip's SIMDs, or the longest.
// Fitted to 23 100 batches of 1 to 16 sequences of 5 to 3000 rows behind up to 8000 tokens, timed as narrow and as wide work: 7 % off on average,
// and the kind that is chosen 0.23 % off the shorter, 8 % for one in a hundred.  (All of them as narrow work: 2.3 %; the largest 20 to 40 %.)
double wide4_us(const std::vector<bs_window::Rows> &rows, const bs_layer_cfg &g, int group, int n_cu) {
  if (rows.empty()) return 0.0;
  int64_t pages = 0;
  int longest = 0;
  for (const bs_window::Rows &r : rows) {
    pages += r.pages;
    longest = std::max(longest, r.pages);
  }
  const double step = g.head_dim == 128 ? 1.77 : 0.856 + 0.228 * (64 / group), per_simd = g.n_kv_heads / (4.0 * n_cu);
  const double all = per_simd * (0.89 * (double)pages + 10.0 * (double)rows.size()), alone = 0.407 * longest;
  return 6.5 + step * std::pow(std::pow(all, 2.9) + std::pow(alone, 2.9), 1.0 / 2.9);
}

void cut_blocks(bs_window *w, int most) {
  Planned &p = w->p;
  if (most == 0) return;
  std::vector<bs_window::Work> whole;
  whole.swap(w->work);
  for (const bs_window::Work &k : whole) {
    const int n = (k.blocks + most - 1) / most;
    if (n == 1) {
      w->work.push_back(k);
      continue;
    }
    w->cut.insert(w->cut.end(), {k.seq, k.block, (int32_t)p.cut_states, n});
    for (int i = 0; i < n; ++i) {
      const int t0 = (int)((int64_t)k.blocks * i / n), t1 = (int)((int64_t)k.blocks * (i + 1) / n);
      w->work.push_back({t1 - t0, k.seq, k.block, t0, i + 1 < n ? t1 : 0, (int)p.cut_states + i});
    }
    p.cut_states += n;
  }
}

// Sorts the rows of every sequence into the two kinds of work: wide that of sequences with more than most_narrow rows.
int sort_rows(bs_window *w, const bs_batch *b, const Route &r, int most_narrow) {
  Planned &p = w->p;
  w->rows.clear();
  w->work.clear();
  w->wide_start.assign((size_t)b->n_seq + 1, 0);
  w->wide_pages.clear();
  w->wide_rows.clear();
  p.wide_blocks = 0;
  p.pages = 0;
  for (int s = 0; s < b->n_seq; ++s) {
    const int rows = b->row_start[s + 1] - b->row_start[s];
    w->wide_start[s] = (int32_t)w->wide_pages.size();
    if (rows > most_narrow) {
      if (w->group) {
        if (const int rc = add_rows(w, b, s, 0, rows, r.per_wide, &w->wide_rows)) return rc;
        continue;
      }
      if (const int rc = add_blocks(w, b, s, r)) return rc;
      w->wide_pages.insert(w->wide_pages.end(), b->page_ids + b->page_start[s], b->page_ids + b->page_start[s + 1]);
    } else if (const int rc = add_rows(w, b, s, 0, rows, r.per_unit)) {
      return rc;
    }
  }
  w->wide_start[b->n_seq] = (int32_t)w->wide_pages.size();
  return BS_OK;
}

// Whether all rows as narrow work over a cache in four bits are expected to take `us` or more, whatever their division: what they compute alone.  (A segment
// of more rows than a unit is among them, whose units leave no room for a second KV head.)
bool narrow4_takes(const bs_window *w, const bs_batch *b, const Route &r, const bs_layer_cfg &g, int n_cu, double us) {
  int64_t pages = 0;
  for (int s = 0; s < b->n_seq; ++s) {
    const int rows = b->row_start[s + 1] - b->row_start[s];
    for (int j = 0; j < rows; j += r.per_unit) {
      const int p0 = b->kv_len[s] - rows + j;
      pages += seen_by(p0, p0 + std::min(r.per_unit, rows - j) - 1, w->p.window, w->p.sinks).pages();
    }
    if (UNITS4_US + compute4_us(g, w->group, 1, pages, n_cu) >= us) return true;
  }
  return false;
}

int plan_work(bs_window *w, const bs_batch *b, const Route &r, const bs_layer_cfg &g, int n_cu) {
  Planned &p = w->p;
  w->items.clear();
  w->item_pages.clear();
  w->cut.clear();
  // Sequences with more rows than a unit, or than four, are wide work, or none is: whichever is expected to be shortest.  A few blocks of
  // rows are shorter as narrow work, whose units spread over the chip: four segments of 32 rows, window 1024, 8 KV heads 18.6 us
  // against 25, sixteen of 64 rows, 16 heads without groups 79 against 44.
  int rows_of[3] = {std::numeric_limits<int>::max(), 4 * r.per_unit, r.per_unit}, most = 0, next = 0;
  for (int s = 0; s < b->n_seq; ++s) {
    const int n = b->row_start[s + 1] - b->row_start[s];
    most = std::max(most, n);
    if (n > r.per_unit && n <= 4 * r.per_unit) next = 1;
  }
  Division div = {1, 2, 0.0};
  Cut cut = {0, 0.0};
  double best = -1.0;
  int chosen = rows_of[0];
  for (int k = 2; k >= 0; --k) {
    const int rows = rows_of[k];
    if (rows < most ? (k == 2 && !next) : k != 0) continue;  // (the same as another)
    if (k && w->group && !kv4_has_rows(g.head_dim, w->group)) continue;
    if (k == 0 && best >= 0.0 && w->group) {
      if (narrow4_takes(w, b, r, g, n_cu, best)) continue;
    } else if (k == 0 && best >= 0.0) {  // many rows as narrow work: more pages than could be worth it
      int64_t pages = 0;
      for (const bs_window::Work &x : w->work) pages += (int64_t)x.blocks * (r.rows / r.per_unit);
      if (pages * g.n_kv_heads * 0.1 > 2.0 * best * n_cu) continue;
    }
    if (const int rc = sort_rows(w, b, r, rows)) return rc;
    const Division d = w->group ? divide4(w->rows, g, w->group, n_cu) : divide(w->rows, g.n_kv_heads, g.head_dim, n_cu);
    const Cut c = w->work.empty() ? Cut{0, 0.0} : cut_choice(w->work, g.n_q_heads / r.heads, g.head_dim, r.rows, n_cu);
    const double us = d.us + c.us + wide4_us(w->wide_rows, g, w->group, n_cu);
    if (best < 0.0 || us < best) {
      best = us;
      div = d;
      cut = c;
      chosen = rows;
    }
  }
  if (const int rc = sort_rows(w, b, r, chosen)) return rc;
  if (!w->work.empty()) {
    cut_blocks(w, cut.blocks);
    div = {4, std::max(div.pages, 8), 0.0};  // (one launch for both kinds, of workgroups of four wavefronts)
  }
  p.heads = div.heads;
  if (const int rc = add_units(w, b, div)) return rc;
  p.n_items = (int)w->items.size();
  p.pages += (long)w->item_pages.size();
  // longest first: the short ones then fill the end of the launch
  std::stable_sort(w->work.begin(), w->work.end(), [](const auto &x, const auto &y) { return x.blocks > y.blocks; });
  p.n_work = (int)w->work.size();
  p.n_wide = (int)w->wide_items.size();
  p.n_cut = (int)w->cut.size() / 4;
  return BS_OK;
}

// Runs of rows whose keys and values go to one page.
void plan_appends(bs_window *w, const bs_batch *b) {
  w->rope.clear();
  for (int s = 0; s < b->n_seq; ++s) {
    const int r0 = b->row_start[s], rows = b->row_start[s + 1] - r0, first = b->kv_len[s] - rows;
    for (int j = 0; j < rows;) {
      const int at = first + j, n = std::min(rows - j, at < 0 ? std::min(PAGE, -at) : PAGE - at % PAGE);
      w->rope.push_back({r0 + j, n, at < 0 ? -1 : b->page_ids[b->page_start[s] + at / PAGE], at < 0 ? 0 : at % PAGE});
      j += n;
    }
  }
  w->p.n_rope = (int)w->rope.size();
}

template <class T>
int grow(bs_ctx *c, T **at, long *cap, long want, size_t each) {
  if (want <= *cap) return BS_OK;
  const long room = want + want / 4 + 1024;
  if (*at) CTX_HIP_TRY(c, hipFree(*at));
  *at = nullptr;
  *cap = 0;
  const hipError_t e = hipMalloc(reinterpret_cast<void **>(at), (size_t)room * each);
  if (e != hipSuccess) {
    *at = nullptr;
    return ctx_fail(c, BS_ENOMEM, "hipMalloc of %zu bytes: %s", (size_t)room * each, hipGetErrorString(e));
  }
  *cap = room;
  return BS_OK;
}

int stream_is_capturing(bs_ctx *c, hipStream_t st, bool *yes) {
  if (const int e = HipRuntime().capturing(st, yes)) return ctx_fail(c, BS_EHIP, "hipStreamIsCapturing: %s", hipGetErrorString((hipError_t)e));
  return BS_OK;
}

AttnShape shape_of(const bs_layer_cfg &g) {
  AttnShape s;
  s.n_q_heads = g.n_q_heads; s.n_kv_heads = g.n_kv_heads; s.head_dim = g.head_dim; s.page_size = g.page_size;
  s.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)g.head_dim));
  return s;
}

bool aligned(const void *p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0; }

// the checks that every call on a plan makes first
int check_call(bs_window *w, const char *what) {
  if (ctx_view(w->ctx).device == BS_DEVICE_NONE) return ctx_fail(w->ctx, BS_EINVAL, "host-only context");
  if (!w->p.made) return ctx_fail(w->ctx, BS_EINVAL, "%s: nothing is planned", what);
  return BS_OK;
}

}  // namespace

extern "C" {

int bs_window_create(bs_ctx *c, bs_window **out) {
  if (out) *out = nullptr;
  if (!c) return BS_EINVAL;
  return ctx_guarded(c, [&]() -> int {
    if (!out) return ctx_fail(c, BS_EINVAL, "out is NULL");
    bs_window *w = new bs_window();
    w->ctx = c;
    const CtxView v = ctx_view(c);
    if (v.device != BS_DEVICE_NONE) {
      hipError_t e = hipSetDevice(v.device);
      if (e == hipSuccess) e = (hipError_t)w->stage.open(STAGE_WORDS, 16);
      if (e != hipSuccess) {
        w->stage.close();
        delete w;
        return ctx_fail(c, e == hipErrorOutOfMemory ? BS_ENOMEM : BS_EHIP, "pinned memory of a plan: %s", hipGetErrorString(e));
      }
    }
    *out = w;
    return BS_OK;
  });
}

void bs_window_destroy(bs_window *w) {
  if (!w) return;
  const int device = ctx_view(w->ctx).device;
  if (device != BS_DEVICE_NONE) {
    (void)hipSetDevice(device);
    (void)hipDeviceSynchronize();
    if (w->d_words) (void)hipFree(w->d_words);
    if (w->d_states) (void)hipFree(w->d_states);
    if (w->d_counters) (void)hipFree(w->d_counters);
    w->stage.close();
  }
  delete w;
}

int bs_window_cache(bs_window *w, int32_t bits, int32_t group) {
  if (!w) return BS_EINVAL;
  return ctx_guarded(w->ctx, [&]() -> int {
    if (bits == 4 ? bs_kv4_page_bytes(w->ctx, group) == 0 : bits != 16 || group != 0)
      return ctx_fail(w->ctx, BS_EINVAL, "bs_window_cache: %d bits, groups of %d channels (16 and 0, or 4 and 32, 64 or 128, at most head_dim)", bits, group);
    w->p = Planned();
    w->group = group;
    return BS_OK;
  });
}

int bs_window_plan(bs_window *w, const bs_batch *b, int64_t n_pages, int32_t window, int32_t sinks, int32_t n_axes,
                   const int32_t *positions, const int32_t *axis_of_pair, void *stream) {
  if (!w) return BS_EINVAL;
  bs_ctx *c = w->ctx;
  return ctx_guarded(c, [&]() -> int {
    const CtxView v = ctx_view(c);
    const bs_layer_cfg &g = *v.cfg;
    const hipStream_t st = (hipStream_t)stream;
    w->p = Planned();
    if (window < 1 || sinks < 0) return ctx_fail(c, BS_EINVAL, "window %d must be at least 1 and sinks %d at least 0", window, sinks);
    if (n_axes < 0 || n_axes > MAX_AXES || (n_axes > 0) != (positions != nullptr) || (n_axes > 0) != (axis_of_pair != nullptr))
      return ctx_fail(c, BS_EINVAL, "n_axes %d: 1 to %d with positions and axis_of_pair, or 0 without", n_axes, MAX_AXES);
    if (const int rc = check_batch(c, b, n_pages)) return rc;
    if (const int rc = check_appends(w, b, n_pages)) return rc;
    const int half = g.head_dim / 2, rows = b->n_rows;
    for (int i = 0; n_axes > 0 && i < half; ++i)
      if (axis_of_pair[i] < 0 || axis_of_pair[i] >= n_axes) return ctx_fail(c, BS_EINVAL, "axis_of_pair[%d]=%d of %d axes", i, axis_of_pair[i], n_axes);
    for (int64_t i = 0; i < (int64_t)n_axes * rows; ++i)
      if (positions[i] < 0 || positions[i] >= g.max_positions)
        return ctx_fail(c, BS_EINVAL, "positions[%lld]=%d outside [0, %d)", (long long)i, positions[i], g.max_positions);

    Planned &p = w->p;
    p.n_rows = rows;
    // (longer windows and more sinks than any length change nothing)
    p.window = std::min(window, MAX_LEN);
    p.sinks = std::min(sinks, MAX_LEN);
    const auto fail_with = [&](int rc) { w->p = Planned(); return rc; };
    const Route route = route_of(g);
    if (const int rc = plan_work(w, b, route, g, v.n_cu)) return fail_with(rc);
    plan_appends(w, b);
    // (grids count units of a KV head, workgroups of some heads, and shares of the heads of a run)
    if ((int64_t)p.n_items * g.n_kv_heads > 0x7fffffff || (int64_t)p.n_work * g.n_q_heads > 0x7fffffff ||
        (int64_t)p.n_rope * (g.n_kv_heads + 1) + 4096 > 0x7fffffff || (int64_t)p.n_wide * g.n_kv_heads > 0x7fffffff)
      return fail_with(too_large(w));

    for (int i = 0; n_axes > 0 && i < half; ++i) p.whole_axes = p.whole_axes && axis_of_pair[i] == axis_of_pair[i & ~7];
    const int axes = std::max(1, n_axes);
    const long n_item_pages = (long)w->item_pages.size(), n_wide_pages = (long)w->wide_pages.size();
    p.off_pages = 8L * p.n_items;
    p.off_work = p.off_pages + whole_units(n_item_pages);
    p.off_cut = p.off_work + 4L * p.n_work;
    p.off_row_start = p.off_cut + 4L * p.n_cut;
    const long n_tab = p.n_work ? b->n_seq + 1 : 0;
    p.off_kv_len = p.off_row_start + n_tab;
    p.off_page_start = p.off_kv_len + n_tab;
    p.off_page_ids = p.off_page_start + n_tab;
    p.off_wide = whole_units(p.off_page_ids + n_wide_pages);
    p.off_rope = p.off_wide + 8L * p.n_wide;
    p.off_axis = p.off_rope + 4L * p.n_rope;
    p.off_positions = p.off_axis + half;
    p.words = whole_units(p.off_positions + (long)axes * rows);
    std::vector<int32_t> &words = w->words;
    words.assign((size_t)p.words, 0);
    if (p.n_items) std::memcpy(&words[p.off_items], w->items.data(), sizeof(WindowItem) * p.n_items);
    if (n_item_pages) std::memcpy(&words[p.off_pages], w->item_pages.data(), sizeof(int32_t) * n_item_pages);
    for (int i = 0; i < p.n_work; ++i) {
      const bs_window::Work &k = w->work[i];
      int32_t *to = &words[p.off_work + 4L * i];
      to[0] = k.seq;
      to[1] = k.block;
      to[2] = (int32_t)((uint32_t)k.t0 | (uint32_t)k.t1 << 16);
      to[3] = k.state;
    }
    if (p.n_cut) std::memcpy(&words[p.off_cut], w->cut.data(), sizeof(int32_t) * w->cut.size());
    if (p.n_work) {
      std::memcpy(&words[p.off_row_start], b->row_start, sizeof(int32_t) * n_tab);
      std::memcpy(&words[p.off_kv_len], b->kv_len, sizeof(int32_t) * b->n_seq);
      std::memcpy(&words[p.off_page_start], w->wide_start.data(), sizeof(int32_t) * n_tab);
      if (n_wide_pages) std::memcpy(&words[p.off_page_ids], w->wide_pages.data(), sizeof(int32_t) * n_wide_pages);
    }
    if (p.n_wide) std::memcpy(&words[p.off_wide], w->wide_items.data(), sizeof(WindowItem) * p.n_wide);
    if (p.n_rope) std::memcpy(&words[p.off_rope], w->rope.data(), sizeof(RopeItem) * p.n_rope);
    p.has_angles = true;
    for (int s = 0; n_axes == 0 && s < b->n_seq; ++s) {
      const int r0 = b->row_start[s], n = b->row_start[s + 1] - r0;
      if (n > 0 && b->kv_len[s] > g.max_positions) p.has_angles = false;
      for (int j = 0; j < n; ++j) words[p.off_positions + r0 + j] = std::max(0, b->kv_len[s] - n + j);
    }
    if (n_axes > 0) {
      std::memcpy(&words[p.off_positions], positions, sizeof(int32_t) * (size_t)n_axes * rows);
      std::memcpy(&words[p.off_axis], axis_of_pair, sizeof(int32_t) * half);
    }
    if (v.device == BS_DEVICE_NONE) { p.made = true; return BS_OK; }

    bool capturing = false;
    if (hipError_t e = hipSetDevice(v.device)) return fail_with(ctx_fail(c, BS_EHIP, "hipSetDevice: %s", hipGetErrorString(e)));
    if (const int rc = stream_is_capturing(c, st, &capturing)) return fail_with(rc);
    if (capturing) return fail_with(ctx_fail(c, BS_EINVAL, "bs_window_plan cannot be captured: plan first, then capture the calls that use the plan"));
    if (const int rc = grow(c, &w->d_words, &w->cap_words, p.words, sizeof(int32_t))) return fail_with(rc);
    const long n_cut = p.cut_states * route.rows * g.n_q_heads;  // state rows of a head of wide work
    p.at_cut_acc = p.states * g.n_kv_heads * (g.head_dim / 16 + 1) * 256;
    p.at_cut_m = p.at_cut_acc + n_cut * g.head_dim;
    p.at_cut_l = p.at_cut_m + n_cut;
    p.state_floats = p.at_cut_l + n_cut;
    if (p.at_cut_acc > (1L << 29)) return fail_with(too_large(w));  // (offsets of the joins: 32 bits of bytes)
    if (const int rc = grow(c, &w->d_states, &w->cap_states, p.state_floats, sizeof(float))) return fail_with(rc);
    if (p.states * g.n_kv_heads > w->cap_counters) {
      if (const int rc = grow(c, &w->d_counters, &w->cap_counters, p.states * g.n_kv_heads, sizeof(unsigned))) return fail_with(rc);
      if (hipError_t e = hipMemsetAsync(w->d_counters, 0, sizeof(unsigned) * (size_t)w->cap_counters, st)) {
        w->cap_counters = 0;
        return fail_with(ctx_fail(c, BS_EHIP, "hipMemsetAsync: %s", hipGetErrorString(e)));
      }
    }
    int32_t *pinned = nullptr;
    if (const int e = w->stage.place(p.words, st, &pinned))
      return fail_with(ctx_fail(c, e == hipErrorOutOfMemory ? BS_ENOMEM : BS_EHIP, "pinned memory of a plan: %s", hipGetErrorString((hipError_t)e)));
    std::memcpy(pinned, words.data(), sizeof(int32_t) * (size_t)p.words);
    Upload up;
    up.src = reinterpret_cast<const uint4 *>(pinned);
    up.dst = reinterpret_cast<uint4 *>(w->d_words);
    up.n16 = (int)(p.words / 4);
    up.blocks = (up.n16 + 255) / 256;
    if (hipError_t e = launch_upload(up, st)) return fail_with(ctx_fail(c, BS_EHIP, "the plan's upload: %s", hipGetErrorString(e)));
    p.made = true;
    return BS_OK;
  });
}

int bs_rope_append(bs_window *w, const void *qkv, int64_t qkv_stride, void *q, int64_t q_stride, void *kv_pool, void *stream) {
  if (!w) return BS_EINVAL;
  bs_ctx *c = w->ctx;
  return ctx_guarded(c, [&]() -> int {
    if (const int rc = check_call(w, "bs_rope_append")) return rc;
    const Planned &p = w->p;
    const CtxView v = ctx_view(c);
    const bs_layer_cfg &g = *v.cfg;
    if (p.n_rows == 0) return BS_OK;
    if (!p.has_angles) return ctx_fail(c, BS_EINVAL, "bs_rope_append: a row stands beyond max_positions %d: plan with positions of its own", g.max_positions);
    if (!qkv || !q || !kv_pool) return ctx_fail(c, BS_EINVAL, "bs_rope_append: NULL pointer");
    const int64_t q_row = (int64_t)g.n_q_heads * g.head_dim, qkv_row = q_row + 2 * (int64_t)g.n_kv_heads * g.head_dim;
    if (qkv_stride < qkv_row || q_stride < q_row || !aligned(qkv, qkv_stride) || !aligned(q, q_stride) || !aligned(kv_pool, 0))
      return ctx_fail(c, BS_EINVAL, "bs_rope_append: rows of %lld and %lld elements at strides %lld and %lld (16-byte aligned, strides multiples of 8)",
                      (long long)qkv_row, (long long)q_row, (long long)qkv_stride, (long long)q_stride);
    if (q == qkv && q_stride != qkv_stride) return ctx_fail(c, BS_EINVAL, "bs_rope_append: in place, but with another stride");
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    RopeArgs a{};
    a.n_rows = p.n_rows; a.n_items = p.n_rope; a.n_q_heads = g.n_q_heads; a.n_kv_heads = g.n_kv_heads; a.head_dim = g.head_dim;
    a.cos = v.rope_cos; a.sin = v.rope_sin;
    a.positions = w->d_words + p.off_positions;
    a.axis_of_pair = w->d_words + p.off_axis;
    a.whole = p.whole_axes;
    a.items = reinterpret_cast<const RopeItem *>(w->d_words + p.off_rope);
    a.qkv = (const uint16_t *)qkv; a.q = (uint16_t *)q; a.kv_pool = (uint16_t *)kv_pool;
    a.qkv_stride = qkv_stride; a.q_stride = q_stride;
    CTX_HIP_TRY(c, w->group ? launch_rope_append4(a, w->group, (hipStream_t)stream) : launch_rope_append(a, (hipStream_t)stream));
    return BS_OK;
  });
}

int bs_window_attention(bs_window *w, const void *q, int64_t q_stride, void *out, int64_t out_stride, const void *kv_pool, void *stream) {
  if (!w) return BS_EINVAL;
  bs_ctx *c = w->ctx;
  return ctx_guarded(c, [&]() -> int {
    if (const int rc = check_call(w, "bs_window_attention")) return rc;
    const Planned &p = w->p;
    const CtxView v = ctx_view(c);
    const bs_layer_cfg &g = *v.cfg;
    if (p.n_rows == 0) return BS_OK;
    if (!q || !out || (!kv_pool && p.pages > 0)) return ctx_fail(c, BS_EINVAL, "bs_window_attention: NULL pointer");
    const int64_t row = (int64_t)g.n_q_heads * g.head_dim;
    if (q_stride < row || out_stride < row || !aligned(q, q_stride) || !aligned(out, out_stride) || !aligned(kv_pool, 0))
      return ctx_fail(c, BS_EINVAL, "bs_window_attention: rows of %lld elements at strides %lld and %lld (16-byte aligned, strides multiples of 8)",
                      (long long)row, (long long)q_stride, (long long)out_stride);
    if (q == out && q_stride != out_stride) return ctx_fail(c, BS_EINVAL, "bs_window_attention: in place, but with another stride");
    CTX_HIP_TRY(c, hipSetDevice(v.device));
    const hipStream_t st = (hipStream_t)stream;
    WindowArgs a{};
    a.s = shape_of(g);
    a.items = reinterpret_cast<const WindowItem *>(w->d_words + p.off_items);
    a.item_pages = w->d_words + p.off_pages;
    a.n_items = p.n_items; a.window = p.window;
    a.q = (const uint16_t *)q; a.kv_pool = (const uint16_t *)kv_pool; a.out = (uint16_t *)out;
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.waves = p.waves;
    a.heads = p.heads;
    a.parts = w->d_states;
    a.counters = w->d_counters;
    if (p.n_work) {
      const Route route = route_of(g);
      WindowPrefillArgs f{};
      f.s = a.s;
      f.work = w->d_words + p.off_work;
      f.n_work = p.n_work;
      f.cut = p.n_cut > 0;
      f.part_acc = w->d_states + p.at_cut_acc; f.part_m = w->d_states + p.at_cut_m; f.part_l = w->d_states + p.at_cut_l;
      f.row_start = w->d_words + p.off_row_start; f.kv_len = w->d_words + p.off_kv_len;
      f.page_start = w->d_words + p.off_page_start; f.page_ids = w->d_words + p.off_page_ids;
      f.q = a.q; f.kv_pool = a.kv_pool; f.out = a.out;
      f.window = p.window; f.sinks = p.sinks; f.q_stride = q_stride; f.out_stride = out_stride;
      if (p.n_items > 0) CTX_HIP_TRY(c, launch_window_step(a, f, route.heads, st));
      else CTX_HIP_TRY(c, launch_window_prefill(f, route.heads, st));
      if (p.n_cut) {
        WindowMergeArgs m{};
        m.s = a.s;
        m.row_start = f.row_start;
        m.out = a.out; m.out_stride = out_stride;
        m.cut = w->d_words + p.off_cut; m.n_cut = p.n_cut; m.cut_heads = route.heads; m.cut_rows = route.rows;
        m.cut_acc = f.part_acc; m.cut_m = f.part_m; m.cut_l = f.part_l;
        CTX_HIP_TRY(c, launch_window_merge(m, st));
      }
      if (p.n_items > 0) return BS_OK;
    }
    if (!w->group) {
      CTX_HIP_TRY(c, launch_window_units(a, st));
      return BS_OK;
    }
    if (p.n_wide) {
      WindowArgs wide = a;
      wide.items = reinterpret_cast<const WindowItem *>(w->d_words + p.off_wide);
      wide.n_items = p.n_wide;
      CTX_HIP_TRY(c, launch_window_rows4(wide, w->group, st));
    }
    CTX_HIP_TRY(c, launch_window_units4(a, w->group, st));
    return BS_OK;
  });
}

int bs_window_division(const bs_window *w, bs_window_parts *out) {
  if (!w) return BS_EINVAL;
  if (!out) return ctx_fail(w->ctx, BS_EINVAL, "out is NULL");
  if (!w->p.made) return ctx_fail(w->ctx, BS_EINVAL, "bs_window_division: nothing is planned");
  const Planned &p = w->p;
  *out = {p.n_items, p.longest, p.split_rows, w->group ? p.n_wide : p.wide_blocks, p.n_cut, p.waves, p.pages};
  return BS_OK;
}

}  // extern "C"
