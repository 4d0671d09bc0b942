// Paged window memory: pool layout, the C ABI, the step's plan (block tables,
// slot maps, positions, the attention's work list) and the insertion of keys
// and values into pages.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <new>

#include "paged_internal.h"
#include "rotary_device.h"

using namespace fademem;

struct fademem_paged {
  fademem_paged_config cfg;
  PagedView view;
  int device;
  bool planned;
  int64_t rows, max_new;  // of the planned step
  bool serialize;
  int last_hip_error;
};

namespace {

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int hip_fail(fademem_paged* c, hipError_t e) {
  c->last_hip_error = int(e);
  return FADEMEM_EHIP;
}

// The end of an asynchronous call: its launch status; in serialize mode also its work's.
int finish(fademem_paged* c, void* stream) {
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && c->serialize) {
    e = hipStreamSynchronize(as_stream(stream));
    if (e == hipSuccess) e = hipGetLastError();
  }
  return e == hipSuccess ? FADEMEM_OK : hip_fail(c, e);
}

// The start of one: the store's device has to be the current one.
int enter(fademem_paged* c) {
  int dev = -1;
  (void)hipGetLastError();
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(c, e);
  return dev == c->device ? FADEMEM_OK : FADEMEM_EINVAL;
}

// ---------------------------------------------------------------------------
// Layout
// ---------------------------------------------------------------------------

constexpr uint64_t kMaxPool = uint64_t(1) << 46;

// Row tiles of a step at most, whatever the kernel.
int64_t max_tiles(const fademem_paged_config& c) {
  return c.max_rows * (c.heads / c.kv_heads) / kPagedMinTileRows + c.seqs;
}

// Fills `v` with offsets from `pool` (NULL: sizes only); false: too large.
bool lay_out(const fademem_paged_config& c, char* pool, PagedView* v, size_t* total) {
  unsigned __int128 at = 0;
  auto take = [&](unsigned __int128 bytes) {
    const unsigned __int128 here = at;
    at += (bytes + 255) / 256 * 256;
    return pool + size_t(here);
  };
  memset(v, 0, sizeof *v);
  const int64_t P = c.page_tokens, width = (c.max_tokens + P - 1) / P;
  const size_t elt = c.dtype == FADEMEM_BF16 ? 2 : 4;
  const unsigned __int128 seqs = unsigned(c.seqs);
  const unsigned __int128 page = (unsigned __int128)2 * unsigned(c.kv_heads) * uint64_t(P) * unsigned(c.head_dim) * elt;
  const unsigned __int128 layer = page * uint64_t(c.pages);
  if (page > (uint64_t(1) << 31) || layer * unsigned(c.layers) > kMaxPool || seqs * uint64_t(width) * 4 > kMaxPool) return false;
  const TileShape wide = c.dtype == FADEMEM_BF16 ? paged_wide_bf16_shape(c.head_dim) : kPagedWideF32;
  const TileShape narrow = c.dtype == FADEMEM_BF16 ? kPagedNarrowBf16 : kPagedNarrowF32;
  v->pool = pool;
  v->header = reinterpret_cast<PagedHeader*>(take(sizeof(PagedHeader)));
  v->held = reinterpret_cast<int32_t*>(take(seqs * 4));
  v->gone = reinterpret_cast<int32_t*>(take(seqs * 4));
  v->status = reinterpret_cast<int32_t*>(take(seqs * 4));
  v->first = reinterpret_cast<int32_t*>(take(seqs * 4));
  v->added = reinterpret_cast<int32_t*>(take(seqs * 4));
  v->q_start = reinterpret_cast<int32_t*>(take((seqs + 1) * 4));
  v->bitmap = reinterpret_cast<uint32_t*>(take(uint64_t((c.pages + 31) / 32) * 4));
  v->table = reinterpret_cast<int32_t*>(take(seqs * uint64_t(width) * 4));
  v->slots = reinterpret_cast<int64_t*>(take(uint64_t(c.max_rows) * 8));
  v->pos = reinterpret_cast<int32_t*>(take(uint64_t(c.max_rows) * 12));
  v->tile0 = reinterpret_cast<int32_t*>(take((seqs + 1) * 4));
  v->cost_end = reinterpret_cast<int64_t*>(take(uint64_t(max_tiles(c)) * 8));
  v->starts = reinterpret_cast<WorkStart*>(take((kPagedMaxGroups + 1) * sizeof(WorkStart)));
  v->tile_seq = reinterpret_cast<int32_t*>(take(uint64_t(max_tiles(c)) * 4));
  v->joins = reinterpret_cast<int32_t*>(take(kPagedMaxGroups * sizeof(int32_t)));
  v->redo = reinterpret_cast<uint64_t*>(take((unsigned __int128)uint64_t(max_tiles(c)) * unsigned(c.kv_heads) * 8));
  const size_t wide_slots = 2 * size_t(wide.groups) * paged_slot_floats(wide.rows, c.head_dim);
  const size_t narrow_slots = 2 * size_t(narrow.groups) * paged_slot_floats(narrow.rows, c.head_dim);
  v->scratch = reinterpret_cast<float*>(take((wide_slots > narrow_slots ? wide_slots : narrow_slots) * 4));
  v->pages = take(layer * unsigned(c.layers));
  v->page_bytes = uint32_t(page);
  v->layer_bytes = size_t(layer);
  v->n_pages = c.pages;
  v->max_tokens = c.max_tokens;
  v->block = int32_t(c.block_tokens);
  v->window = int32_t(c.window);
  const int64_t most = int64_t(1) << 30;  // beyond every sequence
  v->sink_tokens = int32_t(c.window == 0 ? 0 : c.sinks > most / c.block_tokens ? most : c.sinks * c.block_tokens);
  v->seqs = c.seqs;
  v->heads = c.heads;
  v->kv_heads = c.kv_heads;
  v->group = c.heads / c.kv_heads;
  v->head_dim = c.head_dim;
  v->page_tokens = int32_t(P);
  v->width = int32_t(width);
  v->front = int32_t((v->sink_tokens + P - 1) / P);
  v->align = P % 64 == 0 ? 64 : P % 32 == 0 ? 32 : 32 % P == 0 ? int32_t(P) : 1;
  set_page_division(v, P);
  v->grid_h = c.grid_h;
  v->grid_w = c.grid_w;
  if (at > kMaxPool) return false;
  *total = size_t(at);
  return true;
}

bool valid_config(const fademem_paged_config* c) {
  const int64_t most = int64_t(1) << 30;
  if (!c) return false;
  if (c->seqs < 1 || c->seqs > kPagedMaxSeqs || c->layers < 1 || c->layers > 4096) return false;
  if (c->kv_heads < 1 || c->heads < c->kv_heads || c->heads > 4096 || c->heads % c->kv_heads) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->dtype != FADEMEM_F32 && c->dtype != FADEMEM_BF16) return false;
  if (c->page_tokens < 1 || c->page_tokens > 65536 || c->pages < 1 || c->pages > (int64_t(1) << 24)) return false;
  if (c->max_tokens < 1 || c->max_tokens > most || c->max_rows < 1 || c->max_rows > (int64_t(1) << 23)) return false;
  if (c->max_rows * (c->heads / c->kv_heads) > most || max_tiles(*c) * c->kv_heads > most) return false;
  if (c->block_tokens < 1 || c->block_tokens > most || c->window < 0 || c->window > most) return false;
  if (c->sinks < 0) return false;
  if (c->grid_h < 1 || c->grid_w < 1 || int64_t(c->grid_h) * c->grid_w > most) return false;
  return true;
}

// ---------------------------------------------------------------------------
// Kernels
// ---------------------------------------------------------------------------

__global__ void paged_init_kernel(PagedView v, int64_t words, int64_t entries) {
  const int64_t step = int64_t(gridDim.x) * blockDim.x, i0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i0 == 0) {
    v.header->free = int32_t(v.n_pages);
    v.header->groups = v.header->tiles = v.header->refused = v.header->rows = v.header->max_new = v.header->again = 0;
    v.q_start[v.seqs] = 0;
  }
  for (int64_t i = i0; i < v.seqs; i += step) {
    v.held[i] = v.status[i] = v.first[i] = v.added[i] = v.q_start[i] = 0;
    v.gone[i] = v.front;
  }
  for (int64_t i = i0; i < words; i += step) {
    const int64_t left = v.n_pages - i * 32;
    v.bitmap[i] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
  }
  for (int64_t i = i0; i < entries; i += step) v.table[i] = -1;
}

constexpr int kPlanThreads = 1024;
constexpr int64_t kFillInPlan = 4 * kPlanThreads;  // rows up to which the plan's block fills them itself
constexpr int kPlanWaves = kPlanThreads / 64;

// Inclusive prefix sum of a value below 2^25 over the wave: four shifts within rows
// of 16 lanes, then the rows' last lanes broadcast to the rows behind them.  On
// the vector ALU; through LDS permutes a scan of the block took 1.9 us.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The same over the block, with the total.  red: kPlanWaves values of LDS that the
// next call of this function does not use (calls alternate between two).
struct Scan {
  int64_t x, sum;
};
__device__ __forceinline__ Scan block_scan(uint32_t x, uint32_t* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan(x);
  if (lane == 63) red[wave] = x;  // below 2^31
  __syncthreads();
  int64_t before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; w += 4) {
    const uint4 y = *reinterpret_cast<const uint4*>(red + w);
    const uint32_t v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      before += w + i < wave ? v[i] : 0u;
      sum += v[i];
    }
  }
  return {before + int64_t(x), sum};
}

// Position of the k-th (from 0) set bit.
__device__ __forceinline__ int nth_bit(uint32_t bits, int k) {
  int at = 0;
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) {
    const int c = __popc((bits >> at) & ((1u << w) - 1u));
    if (k >= c) {
      k -= c;
      at += w;
    }
  }
  return at;
}

// Last i in [0, n) with a[i] <= x (a[0] <= x, a not decreasing).
template <class T>
__device__ __forceinline__ int last_at_most(const T* a, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

constexpr int kCostsInLds = 4096;  // tiles whose costs the search for the workgroups' starts finds in LDS

struct PlanArgs {
  PagedView v;
  const int32_t* kept;
  const int32_t* added;
  int64_t rows, max_new;
  TileShape shape;
  int fill;       // 1: this kernel also writes the rows' slots and positions
};

// Slot and position of row i, o tokens behind the sequence's first new one.
__device__ __forceinline__ void write_row(const PagedView& v, int64_t i, bool live, int s, int32_t p) {
  int64_t slot = -1;
  int32_t t = 0, y = 0, x = 0;
  if (live) {
    const int32_t frame = v.grid_h * v.grid_w, page = page_of(v, p);
    slot = int64_t(v.table[size_t(s) * v.width + page]) * v.page_tokens + (p - page * v.page_tokens);
    t = p / frame;
    y = (p - t * frame) / v.grid_w;
    x = p - t * frame - y * v.grid_w;
  }
  v.slots[i] = slot;
  v.pos[3 * i] = t;
  v.pos[3 * i + 1] = y;
  v.pos[3 * i + 2] = x;
}

// The step's plan, one block: thread s has sequence s.  What each sequence gives
// back and needs follows from its lengths alone; prefix sums over the sequences
// say where its rows, pages and row tiles begin.  Pages are bits of a map, so
// "the lowest free page" does not depend on the order in which pages came back.
// Bound by latency: the chain is lengths -> two prefix sums -> pages -> two
// prefix sums over the row tiles -> the workgroups' starts.
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PlanArgs a) {
  const PagedView& v = a.v;
  __shared__ __attribute__((aligned(16))) uint32_t red_a[kPlanWaves], red_b[kPlanWaves];
  __shared__ uint32_t word_s[kPlanThreads], word_pre[kPlanThreads];
  __shared__ int64_t pre[kPagedMaxSeqs + 1];  // prefix sums of what the phase deals out
  __shared__ int32_t r1_lo[kPagedMaxSeqs], r1_n[kPagedMaxSeqs], r2_lo[kPagedMaxSeqs];
  __shared__ int32_t row_start[kPagedMaxSeqs + 1];
  __shared__ WorkStart starts[kPagedMaxGroups + 1];
  __shared__ int64_t cost_s[kCostsInLds], base_s[kPagedMaxSeqs + 1];
  __shared__ int32_t even_tiles, even_units;  // of the first sequence with tiles, of the first tile
  const int tid = threadIdx.x, s = tid, seqs = v.seqs;
  const bool live = s < seqs;
  const int64_t P = v.page_tokens;
  const int64_t free0 = v.header->free;

  // Lengths, checked.
  const int64_t k = live ? a.kept[s] : 0, n = live ? a.added[s] : 0, held = live ? v.held[s] : 0;
  const int32_t gone = live ? v.gone[s] : 0;
  const int64_t want_rows = live && n > 0 ? n : 0;
  const Scan rows = block_scan(uint32_t(min(want_rows, a.rows + 1)), red_a);
  int32_t code = FADEMEM_OK;
  if (k < 0 || n < 0 || n > a.max_new || k > held || k + n > v.max_tokens || (n > 0 && rows.x > a.rows))
    code = FADEMEM_EINVAL;
  const int32_t front = v.front;
  const int32_t k32 = code ? 0 : int32_t(k), n32 = code ? 0 : int32_t(n);
  const int32_t low_page = page_of(v, paged_low(v, k32));
  const bool restart = gone > front && k <= front * P;  // all that is kept lies in the sinks' pages
  if (!code && gone > front && !restart && low_page < gone) code = FADEMEM_ESTATE;
  const bool ok = live && code == FADEMEM_OK;

  // Pages that go (two ranges) and pages needed, for `m` new tokens.
  const int32_t top = max(low_page, front);
  auto pages_of = [&](int32_t tokens) { return tokens > 0 ? page_of(v, tokens - 1) + 1 : 0; };
  const int32_t np_old = pages_of(int32_t(held));
  int32_t lo1 = 0, n1 = 0, lo2 = 0, n2 = 0, need = 0, from = 0;
  auto pages_for = [&](int32_t m) {
    const int32_t np = pages_of(k32 + m);
    n1 = n2 = need = 0;
    if (!ok) return;
    if (restart) {
      lo1 = np;
      n1 = max(0, min(front, np_old) - np);
      lo2 = gone;
      n2 = max(0, np_old - gone);
      from = front;
    } else {
      lo1 = gone;
      n1 = max(0, min(top, np_old) - gone);
      lo2 = np;
      n2 = max(0, np_old - np);
      from = np_old;
    }
    need = min(max(0, np - from), int32_t(v.n_pages) + 1);  // more never fit
  };
  pages_for(n32);
  Scan going = block_scan(uint32_t(n1 + n2), red_b), taken = block_scan(uint32_t(need), red_a);
  if (taken.sum > free0 + going.sum) {  // not all fit: the sequences from the first that does not on take none
    if (ok && need > 0 && taken.x > free0 + going.sum) {
      code = FADEMEM_ENOMEM;
      pages_for(0);
    }
    going = block_scan(uint32_t(n1 + n2), red_b);
    taken = block_scan(uint32_t(need), red_a);
  }
  const bool admitted = ok && code == FADEMEM_OK;
  const int refused = __syncthreads_or(live && !admitted);
  const int64_t released = going.sum, given = taken.sum;

  // Release.
  if (released > 0) {
    if (live) {
      pre[s] = going.x - n1 - n2;
      r1_lo[s] = lo1;
      r1_n[s] = n1;
      r2_lo[s] = lo2;
    }
    __syncthreads();
    for (int64_t i = tid; i < released; i += kPlanThreads) {
      const int q = last_at_most<int64_t>(pre, seqs, i);
      const int32_t o = int32_t(i - pre[q]);
      const int32_t idx = o < r1_n[q] ? r1_lo[q] + o : r2_lo[q] + o - r1_n[q];
      int32_t* e = v.table + size_t(q) * v.width + idx;
      const int32_t page = *e;
      *e = -1;
      if (page >= 0 && page < v.n_pages) atomicOr(v.bitmap + (page >> 5), 1u << (page & 31));
    }
    __syncthreads();
  }

  // Allocation: the i-th lowest free page is the i-th needed one.
  if (given > 0) {
    if (live) {
      pre[s] = taken.x - need;
      r1_lo[s] = from;
    }
    __syncthreads();
    const int64_t words = (v.n_pages + 31) / 32;
    int64_t done = 0;
    for (int64_t w0 = 0; w0 < words && done < given; w0 += kPlanThreads) {
      const int64_t w = w0 + tid;
      const uint32_t bits = w < words ? __hip_atomic_load(v.bitmap + w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
      const int cnt = __popc(bits);
      const Scan upto = block_scan(cnt, red_b);
      const int64_t first = upto.x - cnt;  // rank of the word's first free page in this round
      word_s[tid] = bits;
      word_pre[tid] = uint32_t(first);
      const int64_t take = min(upto.sum, given - done);  // of this round
      const int m = int(max(int64_t(0), min(int64_t(cnt), take - first)));
      if (m > 0)
        __hip_atomic_store(v.bitmap + w, m == cnt ? 0u : bits & (0xffffffffu << nth_bit(bits, m)), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      for (int64_t r = tid; r < take; r += kPlanThreads) {
        const int i = last_at_most<uint32_t>(word_pre, kPlanThreads, uint32_t(r));
        const int q = last_at_most<int64_t>(pre, seqs, done + r);
        v.table[size_t(q) * v.width + r1_lo[q] + int32_t(done + r - pre[q])] =
            int32_t((w0 + i) * 32 + nth_bit(word_s[i], int(r - word_pre[i])));
      }
      done += take;
      __syncthreads();
    }
  }

  // State.
  const int64_t fresh = admitted ? n : 0;
  const int32_t row0 = int32_t(min(rows.x - min(want_rows, a.rows + 1), a.rows)), row_last = int32_t(min(rows.sum, a.rows));
  if (live) {
    v.status[s] = code;
    v.first[s] = int32_t(ok ? k : 0);
    v.added[s] = int32_t(fresh);
    v.q_start[s] = row0;
    if (ok) {
      v.held[s] = int32_t(k + fresh);
      v.gone[s] = top;
    }
  }
  if (tid == 0) {
    v.q_start[seqs] = row_last;
    v.header->free = int32_t(free0 + released - given);
  }

  // The attention's work: row tiles, their costs in key units, where each workgroup starts.
  const int G = v.group;
  const int tiles_s = (int(fresh) * G + a.shape.rows - 1) / a.shape.rows;
  const Scan tiles = block_scan(tiles_s, red_b);
  const int64_t n_tiles = tiles.sum;
  if (live) {
    if (tiles_s > 0 && tiles.x == tiles_s) even_tiles = tiles_s;
    pre[s] = tiles.x - tiles_s;
    v.tile0[s] = int32_t(tiles.x - tiles_s);
    r1_lo[s] = int32_t(k);
    r2_lo[s] = int32_t(fresh);
    row_start[s] = row0;
  }
  if (tid == 0) {
    pre[seqs] = n_tiles;
    v.tile0[seqs] = int32_t(n_tiles);
    row_start[seqs] = row_last;
  }
  __syncthreads();
  bool even = a.shape.even && (tiles_s == 0 || tiles_s == even_tiles);
  const bool one_each = !a.shape.even;
  int64_t cost0 = 0;
  for (int64_t t0 = 0; t0 < n_tiles; t0 += kPlanThreads) {
    // Narrow tiles: one for every sequence with new tokens, worked out by the sequence's thread.
    const int64_t t = one_each ? pre[min(s, seqs)] : t0 + tid;
    const bool has = one_each ? tiles_s > 0 : t < n_tiles;
    int64_t cost = 0;
    int q = 0;
    if (has) {
      q = one_each ? s : last_at_most<int64_t>(pre, seqs, t);
      const int first_row = int(t - pre[q]) * a.shape.rows, row1 = min(first_row + a.shape.rows, r2_lo[q] * G);
      const int32_t p = r1_lo[q];
      cost = a.shape.overhead + tile_span(v, p + first_row / G, p + (row1 - 1) / G, p + r2_lo[q], a.shape.unit_keys).n_units;
    }
    const int32_t units = int32_t(cost) - a.shape.overhead;
    if (t == 0) even_units = units;
    const Scan upto = block_scan(uint32_t(cost), t0 / kPlanThreads % 2 ? red_b : red_a);
    even = even && (!has || units == even_units);
    if (has) {
      v.cost_end[t] = cost0 + upto.x;
      v.tile_seq[t] = q;
      if (t < kCostsInLds) cost_s[t] = cost0 + upto.x;
    }
    cost0 += upto.sum;
  }
  __syncthreads();
  even = __syncthreads_and(even);
  const int64_t all = cost0 * v.kv_heads;
  const int min_cost = a.shape.overhead + a.shape.min_part;
  int groups = all >= int64_t(a.shape.groups) * min_cost ? a.shape.groups : (int(all) + min_cost - 1) / min_cost;
  auto cost_end = [&](int64_t t) { return t < kCostsInLds ? cost_s[t] : v.cost_end[t]; };
  if (even) {
    groups = 0;
  } else {
    if (s <= seqs) base_s[s] = pre[s] > 0 ? cost_end(pre[s] - 1) : 0;  // where each sequence's tiles begin
    if (seqs == kPlanThreads && tid == 0) base_s[seqs] = cost0;
    __syncthreads();
  }
  if (tid <= groups && groups > 0) {
    WorkStart w = {int32_t(n_tiles) * v.kv_heads, 0};
    if (tid < groups) {
      const int64_t at = int64_t(double(all) * double(tid) / double(groups));  // rises with tid and stays below `all`
      // The last sequence that begins at or before `at`: it has tiles.
      int lo = 0, hi = seqs;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (base_s[mid] * v.kv_heads <= at) lo = mid;
        else hi = mid;
      }
      const int64_t base = base_s[lo], per_head = base_s[lo + 1] - base, local = at - base * v.kv_heads;
      int head = int(double(local) / double(per_head));  // within one of the quotient; made exact
      head += (head + 1) * per_head <= local ? 1 : 0;
      head -= head * per_head > local ? 1 : 0;
      const int64_t x = base + local - head * per_head;  // on the line of the sequence's tiles
      int64_t t = pre[lo], e = pre[lo + 1];              // first tile that ends behind x
      while (t < e) {
        const int64_t mid = (t + e) >> 1;
        if (cost_end(mid) > x) e = mid;
        else t = mid + 1;
      }
      const int64_t n = pre[lo + 1] - pre[lo];
      w.task = int32_t(pre[lo] * v.kv_heads + head * n + t - pre[lo]);
      w.unit = int32_t(max(int64_t(0), x - (t > 0 ? cost_end(t - 1) : 0) - a.shape.overhead));
    }
    v.starts[tid] = w;
    starts[tid] = w;
  }
  if (tid == 0) {
    EvenPlan e = {};
    int launched = groups;
    if (even && n_tiles > 0) launched = even_plan(int(n_tiles * v.kv_heads), even_units, a.shape, &e);
    v.header->groups = launched;
    v.header->tiles = int32_t(n_tiles);
    v.header->refused = refused;
    v.header->rows = int32_t(a.rows);
    v.header->max_new = int32_t(a.max_new);
    v.header->even = e;
    v.header->again = 0;
  }
  __syncthreads();
  // Workgroup g is the first that begins inside its tile: the tile has parts from g - 1 on.
  if (tid < groups) {
    const WorkStart w = starts[tid];
    int parts = 0;
    if (w.unit > 0 && (starts[tid - 1].unit == 0 || starts[tid - 1].task != w.task)) {
      parts = 2;
      for (int i = tid + 1; i < groups && starts[i].unit > 0 && starts[i].task == w.task; ++i)
        ++parts;
    }
    v.joins[tid] = parts;
  }

  if (a.fill) {
    for (int64_t i = tid; i < a.rows; i += kPlanThreads) {
      const int q = last_at_most<int32_t>(row_start, seqs, int32_t(i));
      const int32_t o = int32_t(i) - row_start[q];
      write_row(v, i, i < row_last && o < r2_lo[q], q, r1_lo[q] + o);
    }
  }
}

// Slot and position of every row of the step.
constexpr int kFillThreads = 256;
__global__ __launch_bounds__(kFillThreads) void paged_rows_kernel(PagedView v, int64_t rows) {
  __shared__ int32_t start[kPagedMaxSeqs + 1];
  for (int i = threadIdx.x; i <= v.seqs; i += kFillThreads) start[i] = v.q_start[i];
  __syncthreads();
  const int64_t i = int64_t(blockIdx.x) * kFillThreads + threadIdx.x;
  if (i >= rows) return;
  const int s = last_at_most<int32_t>(start, v.seqs, int32_t(i));
  const int32_t o = int32_t(i) - start[s];
  write_row(v, i, i < start[v.seqs] && o < v.added[s], s, v.first[s] + o);
}

struct PagedInsertArgs {
  const char* k;
  const char* v;
  size_t k_pitch, v_pitch;  // bytes between rows
  char* pages;              // of the layer
  size_t page_bytes;
  int64_t n_slots;          // pages * page_tokens
  const PagedHeader* header;
  const int64_t* slots;
  const int32_t* pos;
  int64_t rows, max_new;    // of the step
  int kv_heads, head_dim, page_tokens;
  int per_block;            // rows of a block
  RotaryArg rot;            // pairs = 0: keys as they are
};

// Rows into the pages of their slots.  As rope_kernel, with the keys' units
// first and the values' behind them; a unit goes to
// [page][K|V][head][offset][element].  Bound by memory (4 x 4680 rows of 12 x 128
// in bf16: 230 MB in 40 us, 5.7 TB/s), few rows by latency (256 rows of 8 x 128: 4.3 us).
template <bool BF16, bool HALVES>
__global__ __launch_bounds__(kRotThreads) void paged_insert_kernel(PagedInsertArgs a) {
  extern __shared__ __attribute__((aligned(16))) double2 cs[];
  constexpr int kElts = BF16 ? 8 : 4;
  if (a.header->rows != a.rows || a.header->max_new != a.max_new) return;  // another step is planned
  const int64_t row0 = int64_t(blockIdx.x) * a.per_block;
  const int n = int(min(int64_t(a.per_block), a.rows - row0));
  if (a.rot.pairs > 0) {
    rotary_angles(a.rot, a.pos, row0, n, cs);
    __syncthreads();
  }
  const int head_units = a.head_dim / kElts, half = head_units / 2;
  const int k_head = HALVES ? half : head_units;
  const int k_row = a.kv_heads * k_head, v_row = a.kv_heads * head_units, per_row = k_row + v_row;
  const size_t head_pitch = size_t(a.page_tokens) * head_units;  // units between heads of a page
  for (int i = threadIdx.x; i < n * per_row; i += kRotThreads) {
    const int t = i / per_row;
    int r = i - t * per_row;
    const int64_t slot = a.slots[row0 + t];
    if (slot < 0 || slot >= a.n_slots) continue;
    const int64_t page = slot / a.page_tokens, off = slot - page * a.page_tokens;
    rot_u32x4* base = reinterpret_cast<rot_u32x4*>(a.pages + size_t(page) * a.page_bytes) + off * head_units;
    if (r < k_row) {
      const int h = r / k_head, u = r - h * k_head;
      const rot_u32x4* src = reinterpret_cast<const rot_u32x4*>(a.k + size_t(row0 + t) * a.k_pitch) + h * head_units + u;
      rot_u32x4* dst = base + h * head_pitch + u;
      const double2* c = cs + t * a.rot.pairs;
      if constexpr (HALVES) {
        rot_u32x4 p = src[0], q = src[half];
        rotate_halves<BF16>(p, q, c, u * kElts, a.rot.pairs);
        dst[0] = p;
        dst[half] = q;
      } else {
        dst[0] = rotate_unit<BF16>(src[0], c, u * (kElts / 2), a.rot.pairs);
      }
    } else {
      r -= k_row;
      const int h = r / head_units, u = r - h * head_units;
      base[(a.kv_heads + h) * head_pitch + u] =
          reinterpret_cast<const rot_u32x4*>(a.v + size_t(row0 + t) * a.v_pitch)[h * head_units + u];
    }
  }
}

// The step's attention kernel: narrow where every sequence's rows fit one narrow tile.
// A sequence of 32 rows costs about the same either way (256 sequences over 500
// tokens: narrow 118, wide 135 us; 8 over 8000: 64, 51), fewer rows are the narrow
// kernel's (12 heads of one row over 4000 tokens: 13.6, 20.5), and with more rows it
// would read the keys once for every 32 of them.
bool narrow_step(const fademem_paged* c) { return c->max_new * c->view.group <= kPagedNarrowBf16.rows; }
TileShape step_shape(const fademem_paged* c) {
  return c->cfg.dtype == FADEMEM_BF16 ? (narrow_step(c) ? kPagedNarrowBf16 : paged_wide_bf16_shape(c->cfg.head_dim))
                                      : (narrow_step(c) ? kPagedNarrowF32 : kPagedWideF32);
}

}  // namespace

// ---------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------

extern "C" {

int fademem_paged_bytes(const fademem_paged_config* cfg, size_t* bytes) {
  PagedView v;
  size_t total = 0;
  if (!bytes || !valid_config(cfg) || !lay_out(*cfg, nullptr, &v, &total)) return FADEMEM_EINVAL;
  *bytes = total;
  return FADEMEM_OK;
}

int fademem_paged_create(const fademem_paged_config* cfg, void* dev_pool, size_t pool_bytes, void* stream,
                         fademem_paged** out) {
  if (!out) return FADEMEM_EINVAL;
  *out = nullptr;
  PagedView v;
  size_t total = 0;
  if (!valid_config(cfg) || !dev_pool || !aligned(dev_pool, 256)) return FADEMEM_EINVAL;
  if (!lay_out(*cfg, static_cast<char*>(dev_pool), &v, &total)) return FADEMEM_EINVAL;
  if (pool_bytes < total) return FADEMEM_ENOMEM;
  fademem_paged* c = new (std::nothrow) fademem_paged();
  if (!c) return FADEMEM_ENOMEM;
  c->cfg = *cfg;
  c->view = v;
  c->planned = false;
  c->rows = c->max_new = 0;
  const char* ser = getenv("FADEMEM_SERIALIZE");
  c->serialize = ser && ser[0] && strcmp(ser, "0") != 0;
  c->last_hip_error = 0;
  (void)hipGetLastError();
  if (hipGetDevice(&c->device) != hipSuccess) {
    delete c;
    return FADEMEM_EHIP;
  }
  const int64_t words = (cfg->pages + 31) / 32, entries = int64_t(cfg->seqs) * v.width;
  const int64_t blocks = (entries + 255) / 256;
  hipLaunchKernelGGL(paged_init_kernel, dim3(unsigned(blocks < 1024 ? blocks : 1024)), dim3(256), 0, as_stream(stream),
                     v, words, entries);
  if (int rc = finish(c, stream)) {
    delete c;
    return rc;
  }
  *out = c;
  return FADEMEM_OK;
}

int fademem_paged_destroy(fademem_paged* paged) {
  delete paged;
  return FADEMEM_OK;
}

int fademem_paged_last_hip_error(const fademem_paged* paged) { return paged ? paged->last_hip_error : 0; }

int fademem_paged_plan(fademem_paged* c, const int32_t* kept, const int32_t* added, int64_t rows, int64_t max_new,
                       void* stream) {
  if (!c || !kept || !added || !aligned(kept, 4) || !aligned(added, 4)) return FADEMEM_EINVAL;
  if (rows < 0 || rows > c->cfg.max_rows || max_new < 0 || max_new > rows) return FADEMEM_EINVAL;
  if (int rc = enter(c)) return rc;
  c->rows = rows;
  c->max_new = max_new;
  PlanArgs a;
  a.v = c->view;
  a.kept = kept;
  a.added = added;
  a.rows = rows;
  a.max_new = max_new;
  a.shape = step_shape(c);
  a.fill = rows <= kFillInPlan;
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, as_stream(stream), a);
  if (!a.fill)
    hipLaunchKernelGGL(paged_rows_kernel, dim3(unsigned((rows + kFillThreads - 1) / kFillThreads)), dim3(kFillThreads), 0,
                       as_stream(stream), c->view, rows);
  const int rc = finish(c, stream);
  c->planned = rc == FADEMEM_OK;
  return rc;
}

int fademem_paged_array(const fademem_paged* c, int32_t which, int32_t layer, void** ptr, int64_t* count) {
  if (!c || !ptr) return FADEMEM_EINVAL;
  const PagedView& v = c->view;
  void* p = nullptr;
  int64_t n = 0;
  switch (which) {
    case FADEMEM_PAGED_Q_START: p = v.q_start; n = v.seqs + 1; break;
    case FADEMEM_PAGED_SLOTS: p = v.slots; n = c->cfg.max_rows; break;
    case FADEMEM_PAGED_POSITIONS: p = v.pos; n = c->cfg.max_rows * 3; break;
    case FADEMEM_PAGED_STATUS: p = v.status; n = v.seqs; break;
    case FADEMEM_PAGED_HELD: p = v.held; n = v.seqs; break;
    case FADEMEM_PAGED_TABLE: p = v.table; n = int64_t(v.seqs) * v.width; break;
    case FADEMEM_PAGED_FREE: p = &v.header->free; n = 1; break;
    case FADEMEM_PAGED_PAGES:
      if (layer < 0 || layer >= c->cfg.layers) return FADEMEM_EINVAL;
      p = v.pages + size_t(layer) * v.layer_bytes;
      n = int64_t(v.layer_bytes / (c->cfg.dtype == FADEMEM_BF16 ? 2 : 4));
      break;
    default: return FADEMEM_EINVAL;
  }
  *ptr = p;
  if (count) *count = n;
  return FADEMEM_OK;
}

int fademem_paged_insert(fademem_paged* c, int32_t layer, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, const fademem_rope* rope, void* stream) {
  if (!c || layer < 0 || layer >= c->cfg.layers) return FADEMEM_EINVAL;
  const int elt = c->cfg.dtype == FADEMEM_BF16 ? 2 : 4;
  const int64_t row = int64_t(c->cfg.kv_heads) * c->cfg.head_dim;
  PagedInsertArgs a;
  memset(&a.rot, 0, sizeof a.rot);
  if (rope) {
    if (int rc = rotary_arg(rope, 0, &a.rot)) return rc;
    if (a.rot.head_dim != c->cfg.head_dim) return FADEMEM_EINVAL;
  }
  for (int64_t s : {k_stride, v_stride})
    if (s < row || s > (int64_t(1) << 32) || s * elt % 16) return FADEMEM_EINVAL;
  if (!c->planned) return FADEMEM_ESTATE;
  if (c->rows == 0) return FADEMEM_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return FADEMEM_EINVAL;
  if (int rc = enter(c)) return rc;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.k_pitch = size_t(k_stride) * elt;
  a.v_pitch = size_t(v_stride) * elt;
  a.pages = c->view.pages + size_t(layer) * c->view.layer_bytes;
  a.page_bytes = c->view.page_bytes;
  a.n_slots = c->cfg.pages * c->cfg.page_tokens;
  a.header = c->view.header;
  a.slots = c->view.slots;
  a.pos = c->view.pos;
  a.rows = c->rows;
  a.max_new = c->max_new;
  a.kv_heads = c->cfg.kv_heads;
  a.head_dim = c->cfg.head_dim;
  a.page_tokens = c->cfg.page_tokens;
  a.per_block = rows_per_block(a.rows, int(2 * row * elt / 16), a.rot.pairs);
  const bool bf16 = c->cfg.dtype == FADEMEM_BF16, halves = rope && a.rot.halves;
  auto kernel = bf16 ? (halves ? paged_insert_kernel<true, true> : paged_insert_kernel<true, false>)
                     : (halves ? paged_insert_kernel<false, true> : paged_insert_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned((a.rows + a.per_block - 1) / a.per_block)), dim3(kRotThreads),
                     size_t(a.per_block) * a.rot.pairs * sizeof(double2), as_stream(stream), a);
  return finish(c, stream);
}

int fademem_paged_attend(fademem_paged* c, int32_t layer, const void* q, int64_t q_stride, float scale, void* out,
                         int64_t out_stride, float* lse, void* stream) {
  if (!c || layer < 0 || layer >= c->cfg.layers) return FADEMEM_EINVAL;
  if (!(scale >= 0.0f) || !isfinite(scale)) return FADEMEM_EINVAL;
  const int elt = c->cfg.dtype == FADEMEM_BF16 ? 2 : 4;
  const int64_t row = int64_t(c->cfg.heads) * c->cfg.head_dim;
  for (int64_t s : {q_stride, out_stride})
    if (s < row || s > (int64_t(1) << 32) || s * elt % 16) return FADEMEM_EINVAL;
  if (!c->planned) return FADEMEM_ESTATE;
  if (c->rows == 0) return FADEMEM_OK;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return FADEMEM_EINVAL;
  if (!rows_apart(static_cast<const char*>(q), size_t(q_stride) * elt, static_cast<const char*>(out),
                  size_t(out_stride) * elt, c->rows, size_t(row) * elt))
    return FADEMEM_EINVAL;
  if (int rc = enter(c)) return rc;
  PagedAttendArgs a;
  a.v = c->view;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.pages = c->view.pages + size_t(layer) * c->view.layer_bytes;
  a.q_pitch = size_t(q_stride) * elt;
  a.out_pitch = size_t(out_stride) * elt;
  a.rows = c->rows;
  a.max_new = c->max_new;
  a.scale = scale == 0.0f ? 1.0f / sqrtf(float(c->cfg.head_dim)) : scale;
  const bool bf16 = c->cfg.dtype == FADEMEM_BF16, narrow = narrow_step(c);
  hipError_t e = bf16 ? launch_paged_bf16(a, narrow, as_stream(stream)) : launch_paged_f32(a, narrow, as_stream(stream));
  if (e == hipSuccess) e = launch_paged_finish(a, bf16, step_shape(c), as_stream(stream));
  if (e != hipSuccess) return hip_fail(c, e);
  return finish(c, stream);
}

}  // extern "C"
