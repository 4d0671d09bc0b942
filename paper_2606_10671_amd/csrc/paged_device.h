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

__device__ __forceinline__ int page_of(const PagedView& v, int key) {
  return int((uint64_t(uint32_t(key)) * v.page_magic) >> v.page_shift);
}
__device__ __forceinline__ int32_t safe_page(const PagedView& v, int32_t id) {
  return min(max(id, 0), int32_t(v.n_pages) - 1);
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

// Units [u0, u1) of a row tile: the work of one segment.
struct Segment {
  int seq, head, tile;     // tile: over all sequences
  int u0, u1;
  int row0, rows;          // of the sequence's (token, head of the group) rows
  int first, held, q_start;
  TileSpan span;
  __device__ bool whole() const { return u0 == 0 && u1 == span.n_units; }
  // Slot of a partial result of workgroup g.
  __device__ int slot(int g) const { return 2 * g + (u0 == 0 ? 1 : 0); }
};

// Runs `f` over workgroup g's segments.
template <class F>
__device__ __forceinline__ void for_segments(const PagedView& v, TileShape shape, int g, F f) {
  const CONST_AS int32_t* starts = plan_array(reinterpret_cast<const int32_t*>(v.starts + g));
  const CONST_AS int32_t* tile0 = plan_array(v.tile0);
  int seq = starts[0], head = starts[1], tile = starts[2], unit = starts[3];
  const int e_seq = starts[4], e_head = starts[5], e_tile = starts[6], e_unit = starts[7];
  for (;;) {
    const bool last = seq == e_seq && head == e_head && tile == e_tile;
    if (last && unit >= e_unit) return;
    Segment s;
    s.seq = seq;
    s.head = head;
    s.tile = tile;
    s.first = plan_array(v.first)[seq];
    s.held = plan_array(v.held)[seq];
    s.q_start = plan_array(v.q_start)[seq];
    const int t0 = tile0[seq], t1 = tile0[seq + 1];
    s.row0 = (tile - t0) * shape.rows;
    s.rows = min(shape.rows, plan_array(v.added)[seq] * v.group - s.row0);
    s.span = tile_span(v, s.first + s.row0 / v.group, s.first + (s.row0 + s.rows - 1) / v.group, s.held, shape.unit_keys);
    s.u0 = unit;
    s.u1 = last ? e_unit : s.span.n_units;
    f(s);
    if (last) return;
    unit = 0;
    if (++tile == t1) {
      tile = t0;
      if (++head == v.kv_heads) {
        head = 0;
        tile = t1;
        do ++seq;
        while (seq < v.seqs && tile0[seq + 1] == t1);
      }
    }
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

// Page numbers of a wave's next tiles of 32 keys, which begin at multiples of 32.
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
