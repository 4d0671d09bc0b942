// Paged attention: what its kernels share on the device.
#pragma once

#include "attend_tile.h"
#include "paged_internal.h"

#define CONST_AS __attribute__((address_space(4)))

namespace fademem {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Plan arrays, which the attention kernels only read: the constant address
// space lets wave-uniform reads go through the scalar cache.
template <class T>
__device__ __forceinline__ const CONST_AS T* plan_array(const T* p) {
  return (const CONST_AS T*)p;
}

__device__ __forceinline__ int32_t safe_page(const PagedView& v, int32_t id) {
  return int32_t(min(uint32_t(id), uint32_t(v.n_pages) - 1u));
}

// Waits until at most N of the wave's loads are in flight (they land in order),
// respectively for its LDS reads.  The compiler does not wait for loads into LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "a 6-bit count");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_sched_barrier(0);
}

// Units [u0, u1) of a task: the work of one segment.
struct Segment {
  int u0, u1;
  int slot;                // scratch slot of its partial result, or -1: it has all units
  int task, seq, head;
  int row0, rows;          // of the sequence's (token, head of the group) rows
  int first, held, q_start;
  TileSpan span;
};

// Workgroups with work; none if the plan on the device is another step's.
__device__ __forceinline__ int planned_groups(const PagedAttendArgs& a) {
  const CONST_AS int32_t* h = plan_array(&a.v.header->groups);
  return h[3] == a.rows && h[4] == a.max_new ? h[0] : 0;
}

// How the plan deals equal tiles.
__device__ __forceinline__ EvenPlan planned_even(const PagedView& v) {
  const CONST_AS int32_t* e = plan_array(&v.header->even.even);
  return {e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7], e[8]};
}

// What follows from a segment's task.
__device__ __forceinline__ void describe(const PagedView& v, TileShape shape, Segment& s) {
  s.seq = plan_array(v.tile_seq)[s.task / v.kv_heads];  // a sequence's tasks are kv_heads times its tiles, as is their first
  const int t0 = plan_array(v.tile0)[s.seq], tiles = plan_array(v.tile0)[s.seq + 1] - t0;
  s.first = plan_array(v.first)[s.seq];
  s.held = plan_array(v.held)[s.seq];
  s.q_start = plan_array(v.q_start)[s.seq];
  const int added = plan_array(v.added)[s.seq], r = s.task - t0 * v.kv_heads;
  s.head = r / tiles;
  s.row0 = (r - s.head * tiles) * shape.rows;
  s.rows = min(shape.rows, added * v.group - s.row0);
  s.span = tile_span(v, s.first + s.row0 / v.group, s.first + (s.row0 + s.rows - 1) / v.group, s.held, shape.unit_keys);
}

// A workgroup's segments, described by its threads side by side, kSegBatch at a
// time, in LDS: walking the plan's arrays segment by segment took three dependent
// reads each time.
constexpr int kSegBatch = 64;
struct SegmentList {
  int32_t x[kSegBatch][16];
};

// Segments of workgroup g.
__device__ __forceinline__ int count_segments(const PagedView& v, TileShape shape, int g) {
  const EvenPlan e = planned_even(v);
  if (shape.even && e.even) return even_segments(e, g);
  const CONST_AS int32_t* w = plan_array(reinterpret_cast<const int32_t*>(v.starts + g));
  return w[2] - w[0] + (w[3] > 0 && (w[2] > w[0] || w[3] > w[1]) ? 1 : 0);
}

// Describes segments first .. first + kSegBatch - 1 of `n`; a barrier has to follow.
__device__ __forceinline__ void list_segments(const PagedView& v, TileShape shape, int g, int first, int n,
                                              SegmentList& list) {
  const int i = int(threadIdx.x), k = first + i;
  if (i >= kSegBatch || k >= n) return;
  Segment s;
  const EvenPlan e = planned_even(v);
  if (shape.even && e.even) {
    const EvenSegment x = even_segment(e, g, k);
    s.task = x.task;
    s.u0 = x.u0;
    s.u1 = x.u1;
    s.slot = x.slot;
    describe(v, shape, s);
  } else {
    s.u0 = 0;
    const CONST_AS int32_t* w = plan_array(reinterpret_cast<const int32_t*>(v.starts + g));
    s.task = w[0] + k;
    describe(v, shape, s);
    if (k == 0) s.u0 = w[1];
    s.u1 = s.task == w[2] ? w[3] : s.span.n_units;
    s.slot = s.u0 > 0 ? 2 * g : s.u1 < s.span.n_units ? 2 * g + 1 : -1;
  }
  const int32_t x[16] = {s.u0,    s.u1,   s.slot,    s.task,        s.seq,         s.head,     s.row0,      s.rows,
                         s.first, s.held, s.q_start, s.span.n_sink, s.span.n_units, s.span.from, s.span.end, s.span.sinks};
#pragma unroll
  for (int j = 0; j < 16; ++j) list.x[i][j] = x[j];
}

// Segment i of the list, in scalar registers.
__device__ __forceinline__ Segment read_segment(const SegmentList& list, int i) {
  const int32_t x = list.x[i][threadIdx.x & 15];
  auto get = [&](int j) { return int(__builtin_amdgcn_readlane(x, j)); };
  Segment s;
  s.u0 = get(0);
  s.u1 = get(1);
  s.slot = get(2);
  s.task = get(3);
  s.seq = get(4);
  s.head = get(5);
  s.row0 = get(6);
  s.rows = get(7);
  s.first = get(8);
  s.held = get(9);
  s.q_start = get(10);
  s.span.n_sink = get(11);
  s.span.n_units = get(12);
  s.span.from = get(13);
  s.span.end = get(14);
  s.span.sinks = get(15);
  return s;
}

// Runs `f` over workgroup g's segments.
template <class F>
__device__ __forceinline__ void for_segments(const PagedView& v, TileShape shape, int g, SegmentList& list, F f) {
  const int n = count_segments(v, shape, g);
  for (int k0 = 0; k0 < n; k0 += kSegBatch) {
    __syncthreads();
    list_segments(v, shape, g, k0, n, list);
    __syncthreads();
    for (int i = 0; i < min(kSegBatch, n - k0); ++i) f(read_segment(list, i));
  }
}

// A query row of a segment: its token's position, what it sees, where it lies.
struct QueryRow {
  int low, high;     // window [low, high)
  int row, head;     // row of q and out, query head
};
__device__ __forceinline__ QueryRow query_row(const PagedView& v, const Segment& s, int r) {
  const int t = (s.row0 + r) / v.group, g = s.row0 + r - t * v.group;
  QueryRow q;
  q.low = paged_low(v, s.first + t);
  q.high = paged_high(v, s.first + t, s.held);
  q.row = s.q_start + t;
  q.head = s.head * v.group + g;
  return q;
}

// Page numbers of a wave's next tiles of 32 keys, which begin at multiples of 32 or
// (a window's) of PagedView::align.
// Lane j holds page j % n of tile batch + j / n, n pages at most lying under a
// tile; a row's lane fetches its page's number from there.  A table read per tile
// would have to be waited for behind the tile loads issued before it.
struct PageBatch {
  int n_under, per_batch, batch;
  int32_t ids;
  __device__ __forceinline__ PageBatch(const PagedView& v) {
    const int P = v.page_tokens;
    n_under = P % 32 == 0 ? 1 : 32 % P == 0 ? 32 / P : 31 / P + 2;
    per_batch = 64 / n_under;
  }
  // A segment that begins with unit u0.
  __device__ __forceinline__ void begin(int u0) {
    batch = u0 - per_batch;
    ids = 0;
  }
  // Byte offsets, from the key head's first row in page 0, of the rows that this lane loads of unit u's tile: row
  // row_of(i) for load i, rows of `row_bytes`.  keys_of(u): the wave's first key of unit u and the end of its keys.
  template <int N, class Keys, class RowOf>
  __device__ __forceinline__ void place(const PagedView& v, const int32_t* table, int u, int u1, Keys keys_of,
                                        RowOf row_of, uint32_t row_bytes, size_t (&at)[N]) {
    const int P = v.page_tokens;
    const auto k = keys_of(u);
    if (k.key0 >= k.lim) return;
    if (u - batch >= per_batch) {
      batch = u;
      const int lane = threadIdx.x & 63, t = lane / n_under;
      const auto kl = keys_of(min(u + t, u1 - 1));
      const int page = page_of(v, max(0, min(kl.key0, kl.lim - 1))) + lane - t * n_under;
      ids = safe_page(v, table[min(page, page_of(v, kl.lim - 1))]);
      asm volatile("" : "+v"(ids));  // waited for here, once a batch
    }
    const int page0 = page_of(v, k.key0), off0 = k.key0 - page0 * P, first = (u - batch) * n_under, last = k.lim - 1 - k.key0;
    if (n_under == 1) {
      const size_t base = size_t(uint32_t(__builtin_amdgcn_readlane(ids, first))) * v.page_bytes;
#pragma unroll
      for (int i = 0; i < N; ++i) at[i] = base + uint32_t(off0 + min(row_of(i), last)) * row_bytes;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int x = off0 + min(row_of(i), last), under = page_of(v, x);
        const uint32_t id = __builtin_amdgcn_ds_bpermute((first + under) * 4, ids);
        at[i] = size_t(id) * v.page_bytes + uint32_t(x - under * P) * row_bytes;
      }
    }
  }
};

}  // namespace
}  // namespace fademem
