// Paged window memory: what its translation units share (not public).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fademem.h"

namespace fademem {

constexpr int kPagedMaxSeqs = 1024;   // one thread of the plan kernel per sequence
constexpr int kPagedMaxGroups = 512;  // workgroups of one attention launch at most

// Attention work of a step.  The rows of a tile are (token, head of the group)
// pairs of one sequence and one key head, token-major: row r is token r / G,
// head r % G of the key head's G query heads, so that a tile of K and V serves
// all of them.  A tile's keys come in units of `unit_keys`: first the units
// that cover the sinks, then those that cover the window.  A task is a tile of a
// key head; tasks are numbered in the order (sequence, key head, tile).  The units
// of all tasks lie on one line, each task with its overhead before it, and the
// line is dealt to the workgroups in equal runs: a run may end one task's units,
// take some tasks whole and begin another's.  Units of a task that several
// workgroups share leave partial results in their slots (0: a run's first units,
// which continue a task; 1: its last units, which begin one).
struct WorkStart {
  int32_t task, unit;  // unit: within the task
};

// Tile and key-unit shapes of an attention kernel.
struct TileShape {
  int rows;       // query rows of a tile
  int unit_keys;  // keys of a unit
  int groups;     // workgroups at most: those resident at once
  int overhead;   // key units that a task costs beside its own: first loads, last results
  int min_part;   // key units of a part at least
  int even;       // 1: equal tasks may be dealt evenly (EvenPlan)
};
// (Overheads of 2, 4, 6, 8 of the wide bf16 kernel: 24 ragged sequences 85.0, 76.0,
// 74.9, 73.7 us, one chunk of 12 heads x 4680 rows 648, 640, 636, 627 us.  Least
// parts of 1, 2, 4 units of the narrow one: 5 sequences x 32 heads over up to 5000
// tokens 16.2, 18.0, 20.6 us.  At D = 64 two workgroups of 128 rows share a CU, one
// computing while the other begins or ends a task: 24 ragged sequences 80 us with
// 256 rows, 76 so, 64 short ones 60 and 50, 32 whole prompts of 1024 tokens 160 and
// 148, one long chunk 1057 and 1070; overheads of 2, 4, 6, 8 there 83, 76, 78, 80.)
constexpr TileShape kPagedWideBf16 = {256, 64, 256, 8, 6, 1};
constexpr TileShape kPagedWideBf16D64 = {128, 64, 512, 4, 6, 1};
__host__ __device__ constexpr TileShape paged_wide_bf16_shape(int head_dim) {
  return head_dim == 64 ? kPagedWideBf16D64 : kPagedWideBf16;
}
constexpr TileShape kPagedNarrowBf16 = {32, 128, 512, 1, 1, 0};
constexpr TileShape kPagedWideF32 = {128, 64, 256, 1, 2, 1};
constexpr TileShape kPagedNarrowF32 = {32, 128, 256, 1, 1, 0};
constexpr int kPagedMinTileRows = 32;

// Floats of a partial result of a tile: O of every row, then row max and row sum.
__host__ __device__ constexpr size_t paged_slot_floats(int rows, int head_dim) {
  return size_t(rows) * size_t(head_dim + 2);
}

// Where all tiles of a step have equally many units and all sequences equally
// many tiles (chunks of a video), the tiles are dealt so that workgroups run the
// same keys at the same time, which their XCD's L2 then serves: task i of the
// first rounds * groups goes to workgroup i % groups, whole; each of the `rem`
// left is cut into `heads` parts of head_len units together and a tail of
// tail_len, part j of the i-th going to workgroup j * rem + i, the tails to the
// workgroups left over, tails_per each.  Part j of tile i leaves its partial
// result in slot j * rem + i, its tail in slot heads * rem + i.
struct EvenPlan {
  int32_t even;       // 0: the line above
  int32_t groups;     // workgroups of a round
  int32_t rounds, rem, heads, head_len, tail_len, tails_per;
  int32_t units;      // of a tile
};

// The even dealing of `total` tiles of `units` key units (EvenPlan); returns the
// workgroups with work.  Head parts: as many as the groups allow, none shorter
// than the shape's least.  Tails for the groups left over: a tail costs its
// group the overhead of a tile again, counted as half of shape.overhead beyond a
// head part's own; tails that take less than two units off every head part are
// left out.
constexpr int kMinTailSaves = 2;
__host__ __device__ inline int even_plan(int total, int units, TileShape shape, EvenPlan* e) {
  e->even = 1;
  e->groups = shape.groups;
  e->units = units;
  e->rounds = total / shape.groups;
  e->rem = total - e->rounds * shape.groups;
  e->heads = e->tails_per = 1;
  e->tail_len = 0;
  if (e->rem > 0) {
    const int most = shape.groups / e->rem, long_enough = units / shape.min_part, heads = most < long_enough ? most : long_enough;
    e->heads = heads > 1 ? heads : 1;
    const int left = shape.groups - e->heads * e->rem;
    if (left > 0 && units >= shape.min_part) {
      e->tails_per = (e->rem + left - 1) / left;
      const int over = (shape.overhead + 1) / 2 * (e->tails_per - 1) * e->heads;
      const int len = units > over ? (units - over) / (e->tails_per * e->heads + 1) : 0;
      if (len >= kMinTailSaves * e->heads) e->tail_len = len;
    }
  }
  e->head_len = units - e->tail_len;
  if (e->rounds > 0) return shape.groups;
  return e->heads * e->rem + (e->tail_len > 0 ? (e->rem + e->tails_per - 1) / e->tails_per : 0);
}

// Unit at which part j of the first `len` units begins, cut into `parts`: j * len / parts, whose product passes 32 bits
// from 2^31 / parts units on (one tile over 2^28 keys at 512 workgroups).
__host__ __device__ inline int32_t even_cut(int32_t len, int32_t parts, int32_t j) {
  const int32_t q = len / parts;
  return j * q + j * (len - q * parts) / parts;
}

// Segments of workgroup g, and the k-th of them: task, units, slot of its partial result or -1.
struct EvenSegment {
  int32_t task, u0, u1, slot;
};
__host__ __device__ inline int32_t even_segments(const EvenPlan& e, int32_t g) {
  const int32_t i0 = (g - e.heads * e.rem) * e.tails_per, left = e.rem - i0;
  return e.rounds + (g < e.heads * e.rem ? 1 : e.tail_len > 0 && left > 0 ? (left < e.tails_per ? left : e.tails_per) : 0);
}
__host__ __device__ inline EvenSegment even_segment(const EvenPlan& e, int32_t g, int32_t k) {
  const int32_t base = e.rounds * e.groups, head_groups = e.heads * e.rem;
  EvenSegment s = {k * e.groups + g, 0, e.units, -1};
  if (k >= e.rounds && g < head_groups) {
    const int32_t j = g / e.rem;
    s.task = base + g - j * e.rem;
    s.u0 = even_cut(e.head_len, e.heads, j);
    s.u1 = even_cut(e.head_len, e.heads, j + 1);
    if (e.heads > 1 || e.tail_len > 0) s.slot = g;
  } else if (k >= e.rounds) {
    s.task = base + (g - head_groups) * e.tails_per + k - e.rounds;
    s.u0 = e.head_len;
    s.slot = head_groups + s.task - base;
  }
  return s;
}

struct PagedHeader {
  int32_t free;    // free pages
  int32_t groups;  // workgroups with work (attention)
  int32_t tiles;   // row tiles of the step
  int32_t refused; // 1: some sequence was not admitted
  int32_t rows;    // rows and most new tokens that the step was planned with: a call
  int32_t max_new; // made for others (a replayed graph's, say) does nothing
  EvenPlan even;
  int32_t again;   // 1: since the plan, some attention marked rows that are to be worked out again (PagedView::redo)
};

// The store as kernels see it.
struct PagedView {
  char* pool;
  PagedHeader* header;
  int32_t* held;       // [seqs] tokens held
  int32_t* gone;       // [seqs] first page behind the sinks' that is still mapped
  int32_t* status;     // [seqs]
  int32_t* first;      // [seqs] position of the step's first new token
  int32_t* added;      // [seqs] new tokens of the step that were admitted
  int32_t* q_start;    // [seqs + 1]
  uint32_t* bitmap;    // [words] bit = 1: the page is free
  int32_t* table;      // [seqs][width]
  int64_t* slots;      // [max_rows]
  int32_t* pos;        // [max_rows][3]
  int32_t* tile0;      // [seqs + 1] first row tile of each sequence
  int64_t* cost_end;   // [tiles] cost of one head up to and with each tile, in key units
  WorkStart* starts;   // [groups + 1]
  int32_t* tile_seq;   // [tiles] sequence of each tile
  int32_t* joins;      // [groups]: parts of the tile that this workgroup is the first to begin inside, or 0
  uint64_t* redo;      // [tasks]: byte w != 0: rows 32 w.. of the tile have to be worked out again
  float* scratch;      // attention partials
  char* pages;         // layer 0
  size_t layer_bytes;
  int64_t n_pages;
  int64_t max_tokens;
  uint32_t page_bytes;
  int32_t block;       // B
  int32_t window;      // W, 0: everything
  int32_t sink_tokens; // S * B (0 without a window)
  int32_t seqs, heads, kv_heads, group, head_dim;
  int32_t page_tokens, width;
  int32_t front;       // pages that hold sinks
  int32_t grid_h, grid_w;
  int32_t align;       // a window's first tile begins at a multiple of this, a power of two that keeps it in the
                       // page of its first key: 64 or 32 where pages are multiples of that, P where P divides 32, or 1
  uint32_t page_magic;  // key / page_tokens = (key * page_magic >> 31) >> page_shift for keys below 2^31
  int32_t page_shift;
};

// 2^(31+L) / P rounded up, 2^L >= P: the product is off by less than key / 2^(31+L) < 1/P.
inline void set_page_division(PagedView* v, int64_t P) {
  int shift = 31;
  while ((int64_t(1) << (shift - 31)) < P) ++shift;
  v->page_shift = shift - 31;
  v->page_magic = uint32_t(((uint64_t(1) << shift) + uint64_t(P) - 1) / uint64_t(P));
}

// Page of a token (or of a sequence's end, 2^30 at most).
__host__ __device__ inline int32_t page_of(const PagedView& v, int32_t key) {
  return int32_t(uint32_t((uint64_t(uint32_t(key) << 1) * v.page_magic) >> 32) >> v.page_shift);
}

// First key of the window of a query at position p, and the end of what it sees.
__host__ __device__ inline int32_t paged_low(const PagedView& v, int32_t p) {
  if (v.window == 0) return 0;
  const int32_t b = int32_t(uint32_t(p) / uint32_t(v.block)) - v.window + 1;
  return b > 0 ? b * v.block : 0;
}
__host__ __device__ inline int32_t paged_high(const PagedView& v, int32_t p, int32_t held) {
  const uint32_t e = (uint32_t(p) / uint32_t(v.block) + 1u) * uint32_t(v.block);  // at most p + block, below 2^31
  return e < uint32_t(held) ? int32_t(e) : held;
}

// Key units of the tokens at positions p0..p1 of a sequence that holds `held`:
// units 0..n_sink-1 cover [0, sinks), the others [from, end).  Where the sinks
// reach the window, one range from 0 covers both.
struct TileSpan {
  int32_t n_sink, n_units;
  int32_t from, end, sinks;
};
__host__ __device__ inline TileSpan tile_span(const PagedView& v, int32_t p0, int32_t p1, int32_t held, int unit_keys) {
  TileSpan t;
  const int32_t low = paged_low(v, p0) & ~(v.align - 1);
  t.end = paged_high(v, p1, held);
  const bool apart = v.sink_tokens < low;
  t.sinks = apart ? v.sink_tokens : 0;
  t.from = apart ? low : 0;
  t.n_sink = (t.sinks + unit_keys - 1) / unit_keys;
  t.n_units = t.n_sink + (t.end - t.from + unit_keys - 1) / unit_keys;
  return t;
}

struct PagedAttendArgs {
  PagedView v;
  const char* q;
  char* out;
  float* lse;
  const char* pages;       // of the layer
  size_t q_pitch, out_pitch;  // bytes between rows
  int64_t rows, max_new;
  float scale;
};

// Attention of one kernel shape (paged_bf16.hip, paged_f32.hip), and the
// kernel behind it that joins what workgroups shared and works out again what
// an infinity or NaN of a hidden key may have reached (paged_attend.hip).
hipError_t launch_paged_bf16(const PagedAttendArgs& a, bool narrow, hipStream_t stream);
hipError_t launch_paged_f32(const PagedAttendArgs& a, bool narrow, hipStream_t stream);
hipError_t launch_paged_finish(const PagedAttendArgs& a, bool bf16, TileShape shape, hipStream_t stream);

}  // namespace fademem
