// Paged attention, fp32 in and out, on the fp32 matrix cores
// (v_mfma_f32_32x32x2_f32: fp32 products and sums throughout).
//
// The arithmetic of a block of 32 rows and 32 keys is the unpaged fp32 kernel's:
// S^T = K Q^T leaves 16 keys of one row in each lane; the summed index of a step
// is d = 8 j + 4 (l / 32) + e, so that a lane's K operands of four steps are one
// 16-byte LDS read; scores run in two chains; a tile's O^T is summed from zero
// and added to the running one; the queries carry only the scale's power of two,
// the rest of it enters in the one rounding that takes a score's distance to the
// row max.  Bound by the matrix cores (2 x 64 MFMAs of 64 cycles per block at
// D = 128) and by the softmax between them, which on a SIMD does not run beside fp32
// MFMAs: 2 x 1170 rows of 12 heads over 5850 keys, 84 GFLOP in 769 to 836 us from one card to another, matrix cores
// busy 73% of the cycles.  (1170 rows are nine tiles and 18 rows: the tenth costs as much as the others, for the work
// of one wave of each split.)  Narrow tiles of few rows by those too, or by reading K and V.  The wide kernel at
// D = 128 spills 16 registers around a segment's start and end, none inside the loop over its keys.
#include "paged_device.h"

namespace fademem {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // keys of a tile

template <int D>
struct Row {
  static constexpr int CH = D / 4;  // 16-byte chunks
  static constexpr int DB = D / 32;
  static constexpr int TILE = kTile * D;  // floats
};

// Scale in the log2 domain as a power of two, which the queries take, and a factor in [1, 2).
struct Scale {
  float power, rest;
  __device__ explicit Scale(float scale) {
    const float c2 = scale * kLog2e;
    power = fmaxf(__uint_as_float(__float_as_uint(c2) & 0x7f800000u), 0x1p-126f);
    rest = c2 / power;
  }
};

// One tile of one wave: scores, weights, running max m and sum l (of this lane's
// keys), O.  hide(key of the tile): true where the lane's row does not see it;
// `hides`: some row of the wave does not see the whole tile.
// `after_k` runs once the K tile is read, `before_v` before V is.
template <int D, class Hide, class AfterK, class BeforeV>
__device__ __forceinline__ void tile_f32(const f32x4 (&q)[D / 8], const float* kb, const float* vb, float rest, bool hides,
                                         Hide hide, AfterK after_k, BeforeV before_v, float& m, float& l,
                                         f32x16 (&o)[D / 32]) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
  const float* kr = kb + l32 * D;
  int swz = (l32 & 15) ^ hh;  // worked out anew for each tile: kept, the addresses would cost registers
  asm volatile("" : "+v"(swz));
  f32x16 zero;
#pragma unroll
  for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
  f32x16 s, s1;
#pragma unroll
  for (int j = 0; j < D / 8; ++j) {
    const f32x4 kf = *reinterpret_cast<const f32x4*>(kr + ((2 * j) ^ swz) * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e % 2 == 0) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q[j][e], j + e == 0 ? zero : s, 0, 0, 0);
      else s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q[j][e], j + e == 1 ? zero : s1, 0, 0, 0);
    }
  }
  after_k();
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] += s1[r];
  if (hides) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (hide(8 * (r >> 2) + 4 * hh + (r & 3))) s[r] = -INFINITY;
  }
  float mx = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mx = __builtin_elementwise_maximum(mx, s[r]);
  const float m_new = __builtin_elementwise_maximum(m, pair_max(mx) * rest);
  const float m_ref = m_new == -INFINITY ? 0.0f : m_new;  // no score above -inf so far: weights 0, not NaN
  const float alpha = exp2f(m - m_ref);
  m = m_new;
  float least = 0.0f, sum = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = __builtin_fmaf(s[r], rest, -m_ref);
    least = fminf(least, s[r]);
  }
  // The instruction alone makes weights below 2^-126 zero, exp2f does not.  (Tiles with a hidden key take exp2f too:
  // to tell them apart would cost every tile two instructions a score.)
  if (__any(least < -126.0f)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = exp2f(s[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r]);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) sum += s[r];
  l = l * alpha + sum;
  before_v();
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const float* vp = vb + 4 * hh * D + 32 * db + l32;
    f32x16 t;
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      t = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[(8 * (r >> 2) + (r & 3)) * D], s[r], t, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = __builtin_fmaf(o[db][r], alpha, t[r]);
    __builtin_amdgcn_sched_barrier(0);  // the next block's V reads stay behind: the registers do not hold them too
  }
}

// ---------------------------------------------------------------------------
// Narrow tiles: 32 rows, four waves that share out the keys, 32 of a unit of 128
// each, through LDS buffers of their own without barriers: K(t+1) is on its way
// while the scores of t are worked out, V(t+1) from P V(t) on.
// ---------------------------------------------------------------------------

constexpr int kNarrowThreads = 256;
constexpr int kNarrowWaves = kNarrowThreads / 64;

template <int D>
__device__ __forceinline__ void paged_narrow_f32_body(const PagedAttendArgs& a) {
  using R = Row<D>;
  constexpr int kLoads = R::TILE * 4 / 1024;
  __shared__ __attribute__((aligned(16))) float k_lds[kNarrowWaves * R::TILE];
  __shared__ __attribute__((aligned(16))) float v_lds[kNarrowWaves * R::TILE];
  __shared__ float m_s[kNarrowWaves][32], l_s[kNarrowWaves][32];
  __shared__ SegmentList segments;
  const PagedView& v = a.v;
  const int groups = planned_groups(a);
  if (int(blockIdx.x) >= groups) return;
  const int g = xcd_group(blockIdx.x, groups);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* const kb = k_lds + wave * R::TILE;
  float* const vb = v_lds + wave * R::TILE;
  const Scale scale(a.scale);
  const int P = v.page_tokens;
  const size_t v_off = size_t(v.kv_heads) * P * D * 4;
  PageBatch pages_under(v);

  for_segments(v, kPagedNarrowF32, g, segments, [&](const Segment& s) {
    const QueryRow qr = query_row(v, s, min(l32, s.rows - 1));
    f32x4 q[D / 8];
    {
      const char* qp = a.q + size_t(qr.row) * a.q_pitch + size_t(qr.head) * D * 4;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        q[j] = *reinterpret_cast<const f32x4*>(qp + 32 * j + 16 * hh) * scale.power;
        asm volatile("" : "+v"(q[j]));  // waited for here, not behind the tile loads
      }
    }
    const QueryRow qa = query_row(v, s, 0), qz = query_row(v, s, s.rows - 1);
    const int all_low = __builtin_amdgcn_readfirstlane(qz.low), all_high = __builtin_amdgcn_readfirstlane(qa.high);
    const int32_t* table = v.table + size_t(s.seq) * v.width;
    const char* pages = a.pages + size_t(s.head) * P * D * 4;
    struct Keys {
      int key0, lim;
    };
    auto keys_of = [&](int u) {
      Keys k;
      const bool sink = u < s.span.n_sink;
      k.key0 = (sink ? u * 128 : s.span.from + (u - s.span.n_sink) * 128) + wave * kTile;
      k.lim = sink ? s.span.sinks : s.span.end;
      return k;
    };
    size_t row_at[kLoads];
    pages_under.begin(s.u0);
    auto place = [&](int u) {
      pages_under.place(v, table, u, s.u1, keys_of, [&](int i) { return (i * 64 + lane) / R::CH; }, D * 4, row_at);
    };
    auto load_k = [&] {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int c = i * 64 + lane;
        __builtin_amdgcn_global_load_lds(pages + row_at[i] + ((c % R::CH) ^ ((c / R::CH) & 15)) * 16,
                                         (LDS_AS void*)(kb + i * 256), 16, 0, 0);
      }
    };
    auto load_v = [&] {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_global_load_lds(pages + v_off + row_at[i] + ((i * 64 + lane) % R::CH) * 16,
                                         (LDS_AS void*)(vb + i * 256), 16, 0, 0);
    };

    f32x16 o[R::DB];
#pragma unroll
    for (int db = 0; db < R::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    __syncthreads();  // the last segment's results have been read
    place(s.u0);
    if (keys_of(s.u0).key0 < keys_of(s.u0).lim) {
      load_k();
      load_v();
    }
    for (int u = s.u0; u < s.u1; ++u) {
      const Keys k = keys_of(u);
      const bool work = k.key0 < k.lim, next = u + 1 < s.u1 && keys_of(u + 1).key0 < keys_of(u + 1).lim;
      if (u + 1 < s.u1) place(u + 1);
      if (work) {
        const int e = k.key0 + kTile, high = min(qr.high, k.lim);
        const bool hides = !(e <= k.lim && e <= all_high && (k.key0 >= all_low || e <= v.sink_tokens));
        wait_loads<kLoads>();  // K(u) has landed; the loads behind it are V(u)'s
        tile_f32<D>(
            q, kb, vb, scale.rest, hides,
            [&](int j) {
              const int key = k.key0 + j;
              return !(key < high && (key >= qr.low || key < v.sink_tokens));
            },
            [&] {
              wait_lds();  // K(u) is read: its buffer takes the next tile
              if (next) load_k();
            },
            [&] {
              if (next) wait_loads<kLoads>();  // V(u) has landed; behind it, K(u+1)'s loads
              else wait_loads<0>();
            },
            m, l, o);
        wait_lds();
        if (next) load_v();
      } else if (next) {
        load_k();
        load_v();
      }
    }

    // Join the waves: O row by row in the tile buffers, waves 0-1 in K's, 2-3 in V's.
    constexpr int kO = 32 * D;
    static_assert(2 * kO <= kNarrowWaves * R::TILE, "two waves' O fit the K buffers");
    l = pair_sum(l);
    __syncthreads();
    float* mine = (wave < 2 ? k_lds : v_lds) + (wave & 1) * kO + l32 * D + 4 * hh;
    if (l32 < s.rows) {
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
          *reinterpret_cast<f32x4*>(mine + 32 * db + 8 * g4) =
              f32x4{o[db][4 * g4], o[db][4 * g4 + 1], o[db][4 * g4 + 2], o[db][4 * g4 + 3]};
      if (hh == 0) {
        m_s[wave][l32] = m;
        l_s[wave][l32] = l;
      }
    }
    __syncthreads();
    const bool whole = s.slot < 0;
    bool bad = false;
    float* slot = v.scratch + size_t(max(s.slot, 0)) * paged_slot_floats(32, D);
    constexpr int kLanes = D / 4;
    for (int i = tid; i < s.rows * kLanes; i += kNarrowThreads) {
      const int r = i / kLanes, c = 4 * (i % kLanes);
      float mm = m_s[0][r];
#pragma unroll
      for (int w = 1; w < kNarrowWaves; ++w) mm = __builtin_elementwise_maximum(mm, m_s[w][r]);
      const float ref = mm == -INFINITY ? 0.0f : mm;
      float ll = 0.0f;
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kNarrowWaves; ++w) {
        const float f = exp2f(m_s[w][r] - ref);
        ll += f * l_s[w][r];
        x += f * *reinterpret_cast<const f32x4*>((w < 2 ? k_lds : v_lds) + (w & 1) * kO + r * D + c);
      }
      if (!whole) {
        *reinterpret_cast<f32x4*>(slot + r * D + c) = x;
        if (c == 0) {
          slot[32 * D + r] = mm;
          slot[32 * D + 32 + r] = ll;
        }
      } else {
        const QueryRow out = query_row(v, s, r);
        const float inv = 1.0f / ll;
        *reinterpret_cast<f32x4*>(a.out + size_t(out.row) * a.out_pitch + (size_t(out.head) * D + c) * 4) = x * inv;
        if (a.lse && c == 0) a.lse[size_t(out.head) * a.rows + out.row] = (mm + log2f(ll)) * kLn2;
        const float all = (x[0] + x[1]) + (x[2] + x[3]) + inv;
        bad = bad || !(__builtin_fabsf(all) < INFINITY);
      }
    }
    bad = __syncthreads_or(bad);
    if (s.u0 == 0 && tid == 0) {
      v.redo[s.task] = whole && bad ? ~uint64_t(0) : 0;
      if (whole && bad) v.header->again = 1;
    }
  });
}

// ---------------------------------------------------------------------------
// Wide tiles: 128 rows; four waves x 32 rows share a K/V tile, two such splits
// take a unit's two tiles of 32 keys.  Two tile buffers per split, one barrier
// per unit.
// ---------------------------------------------------------------------------

constexpr int kWideThreads = 512;
constexpr int kQW = 4, kKS = 2;

template <int D>
__device__ __forceinline__ void paged_wide_f32_body(const PagedAttendArgs& a) {
  using R = Row<D>;
  constexpr int kLoads = kTile * R::CH / (64 * kQW);
  constexpr int kObj = kKS * R::TILE;              // floats of an LDS object
  constexpr int kArea = 64 * (16 * R::DB + 2);     // floats that a wave of split 1 leaves
  static_assert(kArea <= kObj, "one area per object");
  __shared__ __attribute__((aligned(16))) float k_lds0[kObj];
  __shared__ __attribute__((aligned(16))) float v_lds0[kObj];
  __shared__ __attribute__((aligned(16))) float k_lds1[kObj];
  __shared__ __attribute__((aligned(16))) float v_lds1[kObj];
  __shared__ SegmentList segments;
  const PagedView& v = a.v;
  const int groups = planned_groups(a);
  if (int(blockIdx.x) >= groups) return;
  const int g = xcd_group(blockIdx.x, groups);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qw = wave % kQW, split = wave / kQW;
  const Scale scale(a.scale);
  const int P = v.page_tokens;
  const size_t v_off = size_t(v.kv_heads) * P * D * 4;

  for_segments(v, kPagedWideF32, g, segments, [&](const Segment& s) {
    const int32_t* table = v.table + size_t(s.seq) * v.width;
    const char* pages = a.pages + size_t(s.head) * P * D * 4;
    const bool active = 32 * qw < s.rows;  // the wave has a row
    const int r_last = min(32 * qw + 31, s.rows - 1);
    const QueryRow qr = query_row(v, s, min(32 * qw + l32, max(r_last, 0)));
    const int all_low = paged_low(v, s.first + (s.row0 + max(r_last, 0)) / v.group);
    const int all_high = paged_high(v, s.first + (s.row0 + min(32 * qw, s.rows - 1)) / v.group, s.held);
    f32x4 q[D / 8];
    {
      const char* qp = a.q + size_t(qr.row) * a.q_pitch + size_t(qr.head) * D * 4;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) q[j] = *reinterpret_cast<const f32x4*>(qp + 32 * j + 16 * hh) * scale.power;
    }
    f32x16 o[R::DB];
#pragma unroll
    for (int db = 0; db < R::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    auto key0_of = [&](int u) {
      return (u < s.span.n_sink ? u * 64 : s.span.from + (u - s.span.n_sink) * 64) + split * kTile;
    };
    auto lim_of = [&](int u) { return u < s.span.n_sink ? s.span.sinks : s.span.end; };
    auto ld_row = [&](int i) { return ((i * kQW + qw) * 64 + lane) / R::CH; };
    int32_t id[kLoads];  // pages of the rows that this lane loads next
    auto find = [&](int u) {
      const int key0 = key0_of(u), lim = lim_of(u);
      if (key0 >= lim) return;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) id[i] = table[page_of(v, min(key0 + ld_row(i), lim - 1))];
    };
    auto issue = [&](int u, float* kb, float* vb) {
      const int key0 = key0_of(u), lim = lim_of(u);
      if (key0 < lim) {
        int chunk = lane % R::CH;
        // Offsets worked out anew for each unit: kept, they spill at D = 128 (24 ragged sequences 620 us, so 573; at
        // D = 64, where they fit, one chunk of 16 heads 1582 us kept and 1608 anew).
        if constexpr (D == 128) asm volatile("" : "+v"(chunk));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = ld_row(i), key = min(key0 + row, lim - 1);
          const char* src = pages + size_t(uint32_t(safe_page(v, id[i]))) * v.page_bytes +
                            uint32_t(key - page_of(v, key) * P) * uint32_t(D * 4);
          __builtin_amdgcn_global_load_lds(src + (chunk ^ (row & 15)) * 16,
                                           (LDS_AS void*)(kb + split * R::TILE + (i * kQW + qw) * 256), 16, 0, 0);
          __builtin_amdgcn_global_load_lds(src + v_off + chunk * 16,
                                           (LDS_AS void*)(vb + split * R::TILE + (i * kQW + qw) * 256), 16, 0, 0);
        }
      }
      if (u + 1 < s.u1) find(u + 1);
    };
    // Unit u, and the loads of the next one: at its start in split 0, behind the scores in split 1, so that of two
    // waves on a SIMD one has products for the matrix cores while the other works out addresses (one chunk of 24 heads
    // 15.85 ms with all loads at the start, 15.37 so; at D = 64 8.39, 8.15).
    auto compute = [&](int u, const float* kb, const float* vb, float* kb_next, float* vb_next) {
      const int key0 = key0_of(u), lim = lim_of(u);
      const bool more = u + 1 < s.u1, work = key0 < lim && active;
      if (more && (split == 0 || !work)) issue(u + 1, kb_next, vb_next);
      if (!work) return;
      const int e = key0 + kTile, high = min(qr.high, lim);
      const bool hides = !(e <= lim && e <= all_high && (key0 >= all_low || e <= v.sink_tokens));
      tile_f32<D>(
          q, kb + split * R::TILE, vb + split * R::TILE, scale.rest, hides,
          [&](int j) {
            const int key = key0 + j;
            return !(key < high && (key >= qr.low || key < v.sink_tokens));
          },
          [&] {
            if (more && split > 0) issue(u + 1, kb_next, vb_next);
          },
          [] {}, m, l, o);
    };

    __syncthreads();  // the last segment's reads are done
    find(s.u0);
    issue(s.u0, k_lds0, v_lds0);
    for (int u = s.u0; u < s.u1; u += 2) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();  // unit u's tiles landed for every wave; the other buffers are free
      compute(u, k_lds0, v_lds0, k_lds1, v_lds1);
      if (u + 1 >= s.u1) break;
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      compute(u + 1, k_lds1, v_lds1, k_lds0, v_lds0);
    }

    // Join the splits: split 1 leaves its registers, one object per wave.
    l = pair_sum(l);
    float* area = (qw == 0 ? k_lds0 : qw == 1 ? v_lds0 : qw == 2 ? k_lds1 : v_lds1) + lane;
    __syncthreads();
    if (split > 0) {
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) area[64 * (16 * db + r)] = o[db][r];
      area[64 * 16 * R::DB] = m;
      area[64 * (16 * R::DB + 1)] = l;
    }
    __syncthreads();
    uint8_t* redo = reinterpret_cast<uint8_t*>(v.redo + s.task);
    if (split > 0) {
      if (s.u0 == 0 && lane == 0) redo[4 + qw] = 0;
      return;
    }
    if (!active) {
      if (s.u0 == 0 && lane == 0) redo[qw] = 0;
      return;
    }
    {
      const float m_o = area[64 * 16 * R::DB], l_o = area[64 * (16 * R::DB + 1)];
      const float m_new = __builtin_elementwise_maximum(m, m_o), ref = m_new == -INFINITY ? 0.0f : m_new;
      const float x = exp2f(m - ref), y = exp2f(m_o - ref);
      l = l * x + l_o * y;
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = o[db][r] * x + area[64 * (16 * db + r)] * y;
      m = m_new;
    }
    const int r = 32 * qw + l32;
    auto write = [&](float* row, float f) {
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<f32x4*>(row + 32 * db + 2 * j + 4 * hh) =
              f32x4{o[db][j] * f, o[db][j + 1] * f, o[db][j + 2] * f, o[db][j + 3] * f};
    };
    if (s.slot < 0) {
      const float inv = 1.0f / l;
      float all = inv;
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) all += o[db][j];
      if (r < s.rows) {
        write(reinterpret_cast<float*>(a.out + size_t(qr.row) * a.out_pitch + size_t(qr.head) * D * 4), inv);
        if (a.lse && hh == 0) a.lse[size_t(qr.head) * a.rows + qr.row] = (m + log2f(l)) * kLn2;
      }
      const bool bad = __any(r < s.rows && !(__builtin_fabsf(all) < INFINITY));
      if (lane == 0) {
        redo[qw] = bad ? 1 : 0;
        if (bad) v.header->again = 1;
      }
    } else {
      float* slot = v.scratch + size_t(max(s.slot, 0)) * paged_slot_floats(kPagedWideF32.rows, D);
      if (r < s.rows) {
        write(slot + size_t(r) * D, 1.0f);
        if (hh == 0) {
          slot[128 * D + r] = m;
          slot[128 * (D + 1) + r] = l;
        }
      }
      if (s.u0 == 0 && lane == 0) redo[qw] = 0;
    }
  });
}

template <int D>
__global__ __launch_bounds__(kNarrowThreads, 1) void paged_narrow_f32(PagedAttendArgs a) {
  paged_narrow_f32_body<D>(a);
}
template <int D>
__global__ __launch_bounds__(kWideThreads, 1) void paged_wide_f32(PagedAttendArgs a) {
  paged_wide_f32_body<D>(a);
}

}  // namespace

hipError_t launch_paged_f32(const PagedAttendArgs& a, bool narrow, hipStream_t stream) {
  const bool d128 = a.v.head_dim == 128;
  auto kernel = narrow ? (d128 ? paged_narrow_f32<128> : paged_narrow_f32<64>)
                       : (d128 ? paged_wide_f32<128> : paged_wide_f32<64>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(narrow ? kPagedNarrowF32.groups : kPagedWideF32.groups)),
                     dim3(narrow ? kNarrowThreads : kWideThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace fademem
