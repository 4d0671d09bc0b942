// Paged attention, bf16 in, fp32 accumulation, on v_mfma_f32_32x32x16_bf16.
//
// Two kernels share the arithmetic of a 32-row block: S^T = K Q^T leaves 16 keys
// of one row in each lane (row = lane % 32), so row max and sum take one
// exchange between the halves of the wave, and the weights P leave the
// accumulator in the operand layout of O^T = V^T P^T.  K is read from LDS with
// 16-byte loads, V with the transposing LDS read; both lie XOR-swizzled by row.
// Pages are [head][token][element], so a run of keys inside a page is one run
// of bytes.
//
// Rows are (token, head of the key head's group) pairs: a step of one token with
// G heads per key head is one block of G rows.
//
// Scores, row maxima, sums and O are fp32.  Rounded to fewer bits are the weights P,
// to bf16 (2^-8 of each at most): the matrix cores take P and V in one type, and
// products of fp32 operands run at an eighth of the rate.  The row sum is that of
// the weights before this rounding, whose errors average out over the keys: against
// fp64 the output is off by its own rounding (24 ragged sequences: 1.70e-3 of the
// output's root mean square, 1.65e-3 with weights in fp32).  The exponent
// instruction makes a weight below 2^-126 zero, where the row's largest is 1 to 2^8.
#include <type_traits>

#include "paged_device.h"

namespace fademem {
namespace {

template <int D>
struct Row {
  static constexpr int CH = D / 8;         // 16-byte chunks
  static constexpr int KB = D / 16;        // k-steps of S^T = K Q^T
  static constexpr int DB = D / 32;        // 32-row blocks of O^T
  static constexpr int RPB = 256 / (2 * D);  // rows per 256 bytes of LDS
};

// Swizzles: LDS 16-byte position of chunk c of row n is c ^ swz(n).
template <int D>
__device__ __forceinline__ int kswz(int n) {
  return (n / Row<D>::RPB) % Row<D>::CH;
}
template <int D>
__device__ __forceinline__ int vswz(int n) {
  return 4 * ((n / Row<D>::RPB) % (4 / Row<D>::RPB));
}

// Per-lane LDS offsets of the operand reads within a buffer of rows of D.
//   K fragment (row 32 nb + l32, chunk 2 kb + hh): kswz(32 nb + l32) = kswz(l32).
//   V^T transposing read (row 16 ks + 8 second + 4 hh + sl/4, d = 32 db +
//   16 (g & 1) + 4 (sl & 3)): vswz of that row depends on the lane only.
template <int D>
struct ReadOffsets {
  int k[Row<D>::KB], v[Row<D>::DB];
  __device__ __forceinline__ explicit ReadOffsets(int lane) {
    const int l32 = lane & 31, hh = lane >> 5, g16 = lane >> 4, sl = lane & 15;
#pragma unroll
    for (int kb = 0; kb < Row<D>::KB; ++kb) k[kb] = l32 * D * 2 + (((2 * kb + hh) ^ kswz<D>(l32)) * 16);
    const int n = 4 * hh + (sl >> 2), vs = vswz<D>(n);
#pragma unroll
    for (int db = 0; db < Row<D>::DB; ++db) {
      const int d = 32 * db + 16 * (g16 & 1) + 4 * (sl & 3);
      v[db] = n * D * 2 + (((d >> 3) ^ vs) * 16) + ((d >> 2) & 1) * 8;
    }
  }
};

// V^T fragment of k-step ks, 32-row block db (two transposing reads).
template <int D>
__device__ __forceinline__ bf16x8 read_v(const char* buf, const ReadOffsets<D>& rd, int ks, int db) {
  bf16x8 a;
#pragma unroll
  for (int second = 0; second < 2; ++second) {
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (LDS_AS s16x4*)((LDS_AS const char*)(buf) + rd.v[db] + (16 * ks + 8 * second) * D * 2));
    const bf16x4 vb = __builtin_bit_cast(bf16x4, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) a[4 * second + e] = vb[e];
  }
  return a;
}

// ---------------------------------------------------------------------------
// Narrow tiles: 32 rows.  Bound by reading K and V once (a tile of 32 keys is
// 16 KB and 16 MFMAs at D = 128).  Four waves share out the keys, 32 of a unit of
// 128 each, and stream them through LDS buffers of their own without barriers:
// K(t+1) is on its way while the scores of t are worked out, V(t+1) from P V(t)
// on, so that half a workgroup's 64 KB are in flight at any time.  Two workgroups
// share a CU, so that one streams while the other begins or ends a tile.  At the
// end the waves' results are joined through LDS.  64 sequences of up to 16 000
// tokens, 32 heads over 8: 999 MB in 180 us, 5.55 TB/s where a large copy reaches 5.07.
// ---------------------------------------------------------------------------

constexpr int kNarrowKeys = 32;
constexpr int kNarrowThreads = 256;
constexpr int kNarrowWaves = kNarrowThreads / 64;
static_assert(kPagedNarrowBf16.unit_keys == kNarrowWaves * kNarrowKeys, "a tile per wave");

template <int D>
__device__ __forceinline__ void paged_narrow_body(const PagedAttendArgs& a) {
  using R = Row<D>;
  constexpr int kBuf = kNarrowKeys * D * 2;        // bytes of a wave's K (or V) buffer
  constexpr int kLoads = kBuf / 1024;              // 16-byte loads per lane
  constexpr int kO = 32 * D;                       // floats of a wave's O
  static_assert(2 * kO * 4 == kNarrowWaves * kBuf, "two waves' O fit the K buffers, two the V buffers");
  __shared__ __attribute__((aligned(16))) char k_lds[kNarrowWaves * kBuf];
  __shared__ __attribute__((aligned(16))) char v_lds[kNarrowWaves * kBuf];
  __shared__ float m_s[kNarrowWaves][32], l_s[kNarrowWaves][32];
  __shared__ SegmentList segments;
  const PagedView& v = a.v;
  const int groups = planned_groups(a);
  if (int(blockIdx.x) >= groups) return;
  const int g = xcd_group(blockIdx.x, groups);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* const kb_lds = k_lds + wave * kBuf;
  char* const vb_lds = v_lds + wave * kBuf;
  const ReadOffsets<D> rd(lane);
  const float c2 = a.scale * kLog2e;
  const int P = v.page_tokens;
  const size_t v_off = size_t(v.kv_heads) * P * D * 2;  // from a key's row to its value's
  PageBatch pages_under(v);

  for_segments(v, kPagedNarrowBf16, g, segments, [&](const Segment& s) {
    const QueryRow qr = query_row(v, s, min(l32, s.rows - 1));
    bf16x8 qf[R::KB];
    {
      const char* q = a.q + size_t(qr.row) * a.q_pitch + size_t(qr.head) * D * 2;
#pragma unroll
      for (int kb = 0; kb < R::KB; ++kb) qf[kb] = *reinterpret_cast<const bf16x8*>(q + (16 * kb + 8 * hh) * 2);
    }
#pragma unroll
    for (int kb = 0; kb < R::KB; ++kb) asm volatile("" : "+v"(qf[kb]));  // waited for here, not behind the tile loads
    // Keys that every row sees need no mask.
    const QueryRow qa = query_row(v, s, 0), qz = query_row(v, s, s.rows - 1);
    const int all_low = __builtin_amdgcn_readfirstlane(qz.low), all_high = __builtin_amdgcn_readfirstlane(qa.high);
    const int32_t* table = v.table + size_t(s.seq) * v.width;
    const char* pages = a.pages + size_t(s.head) * P * D * 2;

    // The wave's keys of unit u: from key0 on, those below lim exist.
    struct Keys {
      int key0, lim;
    };
    auto keys_of = [&](int u) {
      Keys k;
      const bool sink = u < s.span.n_sink;
      k.key0 = (sink ? u * 128 : s.span.from + (u - s.span.n_sink) * 128) + wave * kNarrowKeys;
      k.lim = sink ? s.span.sinks : s.span.end;
      return k;
    };
    size_t row_at[kLoads];
    pages_under.begin(s.u0);
    auto place = [&](int u) {
      pages_under.place(v, table, u, s.u1, keys_of, [&](int i) { return (i * 64 + lane) / R::CH; }, D * 2, row_at);
    };
    auto load_k = [&] {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int q = i * 64 + lane;
        __builtin_amdgcn_global_load_lds(pages + row_at[i] + ((q % R::CH) ^ kswz<D>(q / R::CH)) * 16,
                                         (LDS_AS void*)(kb_lds + i * 1024), 16, 0, 0);
      }
    };
    auto load_v = [&] {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int q = i * 64 + lane;
        __builtin_amdgcn_global_load_lds(pages + v_off + row_at[i] + ((q % R::CH) ^ vswz<D>(q / R::CH)) * 16,
                                         (LDS_AS void*)(vb_lds + i * 1024), 16, 0, 0);
      }
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
      u32x4 p[2];
      if (work) {
        f32x16 sc;
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.0f;
        wait_loads<kLoads>();  // K(u) has landed; the loads behind it are V(u)'s
#pragma unroll
        for (int kb = 0; kb < R::KB; ++kb)
          sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kb_lds + rd.k[kb]), qf[kb], sc, 0,
                                                       0, 0);
        wait_lds();  // K(u) is read: its buffer takes the next tile
        if (next) load_k();
        const bool seen = k.key0 + kNarrowKeys <= k.lim && k.key0 + kNarrowKeys <= all_high &&
                          (k.key0 >= all_low || k.key0 + kNarrowKeys <= v.sink_tokens);
        if (!seen) {
          const int high = min(qr.high, k.lim);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = k.key0 + 8 * (r >> 2) + 4 * hh + (r & 3);
            if (!(key < high && (key >= qr.low || key < v.sink_tokens))) sc[r] = -INFINITY;
          }
        }
        float mx = sc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = __builtin_elementwise_maximum(mx, sc[r]);
        mx = pair_max(mx);
        if (__any(!(mx <= m))) {
          const float m_new = __builtin_elementwise_maximum(m, mx);
          const float alpha = __builtin_amdgcn_exp2f((m - (m_new == -INFINITY ? 0.0f : m_new)) * c2);
          m = m_new;
          l *= alpha;
#pragma unroll
          for (int db = 0; db < R::DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
        }
        const float mc = (m == -INFINITY ? 0.0f : m) * c2;  // no key so far: weights 0, not NaN
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c2, -mc));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r + 1], c2, -mc));
          sum += p0 + p1;
          p[r >> 3][(r & 7) >> 1] = round_pair(p0, p1);
        }
        l += sum;
        if (next) wait_loads<kLoads>();  // V(u) has landed; behind it, K(u+1)'s loads
        else wait_loads<0>();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int db = 0; db < R::DB; ++db)
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v<D>(vb_lds, rd, ks, db),
                                                            __builtin_bit_cast(bf16x8, p[ks]), o[db], 0, 0, 0);
        wait_lds();
        if (next) load_v();
      } else if (next) {
        load_k();
        load_v();
      }
    }

    // Join the waves: O row by row in the tile buffers, waves 0-1 in K's, 2-3 in V's.
    l = pair_sum(l);
    __syncthreads();
    float* mine = reinterpret_cast<float*>(wave < 2 ? k_lds : v_lds) + (wave & 1) * kO + l32 * D + 4 * hh;
    if (l32 < s.rows) {
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
          *reinterpret_cast<float4*>(mine + 32 * db + 8 * g4) =
              make_float4(o[db][4 * g4], o[db][4 * g4 + 1], o[db][4 * g4 + 2], o[db][4 * g4 + 3]);
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
      float ll = 0.0f, x[4] = {};
#pragma unroll
      for (int w = 0; w < kNarrowWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f((m_s[w][r] - ref) * c2);
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w < 2 ? k_lds : v_lds) +
                                                          (w & 1) * kO + r * D + c);
        ll += f * l_s[w][r];
        x[0] += f * y.x;
        x[1] += f * y.y;
        x[2] += f * y.z;
        x[3] += f * y.w;
      }
      if (!whole) {
        *reinterpret_cast<float4*>(slot + r * D + c) = make_float4(x[0], x[1], x[2], x[3]);
        if (c == 0) {
          slot[32 * D + r] = mm * c2;
          slot[32 * D + 32 + r] = ll;
        }
      } else {
        const QueryRow out = query_row(v, s, r);
        const float inv = 1.0f / ll;
        uint2 y = {round_pair(x[0] * inv, x[1] * inv), round_pair(x[2] * inv, x[3] * inv)};
        *reinterpret_cast<uint2*>(a.out + size_t(out.row) * a.out_pitch + (size_t(out.head) * D + c) * 2) = y;
        if (a.lse && c == 0) a.lse[size_t(out.head) * a.rows + out.row] = (mm * c2 + __log2f(ll)) * kLn2;
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
// Wide tiles: 8 waves x 32 rows, or 4 at D = 64, where a CU has LDS for two such
// workgroups.  Bound by the matrix cores.  The pipeline
// is the one of the unpaged attention: K/V tiles of 64 keys go from the pages
// straight into three-deep LDS rings, two tiles ahead, one barrier per tile;
// iteration t runs S(t+1) = K(t+1) Q^T beside the exponentials of S(t)'s second
// half, then O += V(t) P(t) beside those of S(t+1)'s first half, in fenced steps
// of two MFMAs.  Weights stand against a stale row max; a tile with a weight
// above 2^8 is redone against the exact one.
// The keys are two ranges (sinks, window), so a tile's first key comes from the
// unit's number; a tile that some row of the wave does not see whole is masked,
// row by row; addresses come from the page table, read one tile before the loads
// that need it.
// 40 heads x 10 800 rows over 54 000 keys: 1.09 to 1.20 PFLOP/s from one card to another, where a
// product of two 8192 x 8192 matrices reaches 1.22; 12 x 4680 rows over 23 400 keys 1.05 to 1.13, the matrix cores
// busy 61% of the cycles.  Many short tasks are bound by what each costs beside its units, first
// loads and last results (24 ragged sequences, 16 heads of 64 over 4: 28 GFLOP in
// 62 us).
// ---------------------------------------------------------------------------

constexpr float kRescaleBound = 256.0f;
constexpr int kKeys = 64;

// WHOLE: pages are multiples of 64 tokens, so a tile lies in one page.
template <int D, bool WHOLE>
__device__ __forceinline__ void paged_wide_body(const PagedAttendArgs& a) {
  using R = Row<D>;
  constexpr TileShape kShape = paged_wide_bf16_shape(D);
  constexpr int kWaves = kShape.rows / 32, kThreads = 64 * kWaves;
  constexpr int kTileBytes = kKeys * D * 2;
  constexpr int kLoads = kKeys * R::CH / kThreads;  // 16-byte loads per lane and tile, for K and for V
  __shared__ __attribute__((aligned(16))) char k_lds0[kTileBytes];
  __shared__ __attribute__((aligned(16))) char k_lds1[kTileBytes];
  __shared__ __attribute__((aligned(16))) char k_lds2[kTileBytes];
  __shared__ __attribute__((aligned(16))) char v_lds0[kTileBytes];
  __shared__ __attribute__((aligned(16))) char v_lds1[kTileBytes];
  __shared__ __attribute__((aligned(16))) char v_lds2[kTileBytes];
  char* const kbuf[3] = {k_lds0, k_lds1, k_lds2};
  char* const vbuf[3] = {v_lds0, v_lds1, v_lds2};
  __shared__ SegmentList segments;
  const PagedView& v = a.v;
  const int groups = planned_groups(a);
  if (int(blockIdx.x) >= groups) return;
  const int g = xcd_group(blockIdx.x, groups);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ReadOffsets<D> rd(lane);
  const float c2 = a.scale * kLog2e;
  const int P = v.page_tokens;
  const size_t v_off = size_t(v.kv_heads) * P * D * 2;

  // Load i of a tile writes destination chunk (i * waves + wave) * 64 + lane.
  auto ld_row = [&](int i) { return ((i * kWaves + wave) * 64 + lane) / R::CH; };
  auto ld_kch = [&](int i) {
    const int q = (i * kWaves + wave) * 64 + lane;
    return uint32_t(((q % R::CH) ^ kswz<D>(q / R::CH)) * 16);
  };
  auto ld_vch = [&](int i) {
    const int q = (i * kWaves + wave) * 64 + lane;
    return uint32_t(((q % R::CH) ^ vswz<D>(q / R::CH)) * 16);
  };
  uint32_t ld_koff[kLoads], ld_voff[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    ld_koff[i] = uint32_t(ld_row(i) * D * 2) + ld_kch(i);
    ld_voff[i] = uint32_t(ld_row(i) * D * 2) + ld_vch(i);
  }

  for_segments(v, kShape, g, segments, [&](const Segment& s) {
    const CONST_AS int32_t* table = plan_array(v.table + size_t(s.seq) * v.width);
    const char* pages = a.pages + size_t(s.head) * P * D * 2;
    const int n_sink = s.span.n_sink, end = s.span.end, from = s.span.from, sinks = s.span.sinks;
    auto key0_of = [&](int t) { return t < n_sink ? t * kKeys : from + (t - n_sink) * kKeys; };
    auto lim_of = [&](int t) { return t < n_sink ? sinks : end; };

    // The page (or each load's row's page) of the next tile to load.
    int32_t next_id[kLoads];
    auto find = [&](int t) {
      const int key0 = key0_of(t);
      if constexpr (WHOLE) {
        next_id[0] = table[page_of(v, key0)];
      } else {
        const int lim = lim_of(t);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) next_id[i] = v.table[size_t(s.seq) * v.width + page_of(v, min(key0 + ld_row(i), lim - 1))];
      }
    };
    // All loads of tile t, whose pages `find` has; then the pages of tile t + 1.
    auto load_tile = [&](int t, char* kb_lds, char* vb_lds) {
      const int key0 = key0_of(t), valid = lim_of(t) - key0;
      if constexpr (WHOLE) {
        const int off = key0 - page_of(v, key0) * P;
        const char* base = pages + size_t(uint32_t(safe_page(v, next_id[0]))) * v.page_bytes + size_t(off) * (D * 2);
        const char* kbase = uniform_ptr(base);
        const char* vbase = uniform_ptr(base + v_off);
        if (valid >= kKeys) {
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const int j = i * kWaves + wave;
            __builtin_amdgcn_global_load_lds(kbase + ld_koff[i], (LDS_AS void*)(kb_lds + j * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(vbase + ld_voff[i], (LDS_AS void*)(vb_lds + j * 1024), 16, 0, 0);
          }
        } else {  // rows past the last key load it again
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const int j = i * kWaves + wave;
            const uint32_t row = uint32_t(min(ld_row(i), valid - 1)) * (D * 2);
            __builtin_amdgcn_global_load_lds(kbase + (row + ld_kch(i)), (LDS_AS void*)(kb_lds + j * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(vbase + (row + ld_vch(i)), (LDS_AS void*)(vb_lds + j * 1024), 16, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int j = i * kWaves + wave;
          const int key = key0 + min(ld_row(i), valid - 1);
          const char* row = pages + size_t(uint32_t(safe_page(v, next_id[i]))) * v.page_bytes +
                            uint32_t(key - page_of(v, key) * P) * uint32_t(D * 2);
          __builtin_amdgcn_global_load_lds(row + ld_kch(i), (LDS_AS void*)(kb_lds + j * 1024), 16, 0, 0);
          __builtin_amdgcn_global_load_lds(row + v_off + ld_vch(i), (LDS_AS void*)(vb_lds + j * 1024), 16, 0, 0);
        }
      }
      if (t + 1 < s.u1) find(t + 1);
    };

    // The wave's share of the task's eight bytes.
    auto mark = [&](int bad) {
      uint8_t* marks = reinterpret_cast<uint8_t*>(v.redo + s.task);
      marks[wave] = uint8_t(bad);
      if (bad) v.header->again = 1;
      if constexpr (kWaves == 4) marks[4 + wave] = 0;
    };
    // A wave without rows (a sequence's last tile is usually partial) only
    // issues its share of the loads and meets the barriers.
    if (wave * 32 >= s.rows) {
      __syncthreads();
      find(s.u0);
      load_tile(s.u0, kbuf[0], vbuf[0]);
      if (s.u0 + 1 < s.u1) load_tile(s.u0 + 1, kbuf[1], vbuf[1]);
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      int b = 2;
      for (int t = s.u0; t < s.u1; ++t) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (t + 2 < s.u1)
          load_tile(t + 2, b == 0 ? kbuf[0] : b == 1 ? kbuf[1] : kbuf[2], b == 0 ? vbuf[0] : b == 1 ? vbuf[1] : vbuf[2]);
        b = b == 2 ? 0 : b + 1;
      }
      if (s.u0 == 0 && lane == 0) mark(0);
      return;
    }

    const int r_last = min(wave * 32 + 31, s.rows - 1);
    const QueryRow qr = query_row(v, s, min(wave * 32 + l32, r_last));
    // Keys that every row of the wave sees need no mask.
    const int all_low = paged_low(v, s.first + (s.row0 + r_last) / v.group);
    const int all_high = paged_high(v, s.first + (s.row0 + wave * 32) / v.group, s.held);
    bf16x8 qf[R::KB];
    {
      const char* q = a.q + size_t(qr.row) * a.q_pitch + size_t(qr.head) * D * 2;
#pragma unroll
      for (int kb = 0; kb < R::KB; ++kb) qf[kb] = *reinterpret_cast<const bf16x8*>(q + (16 * kb + 8 * hh) * 2);
    }
    auto hides = [&](int t) {
      const int key0 = key0_of(t), e = key0 + kKeys;
      return !(e <= lim_of(t) && e <= all_high && (key0 >= all_low || e <= v.sink_tokens));
    };
    auto mask = [&](int t, f32x16 (&sc)[2]) {
      const int key0 = key0_of(t), high = min(qr.high, lim_of(t));
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + 32 * nb + 8 * (r >> 2) + 4 * hh + (r & 3);
          if (!(key < high && (key >= qr.low || key < v.sink_tokens))) sc[nb][r] = -INFINITY;
        }
    };

    f32x16 o[R::DB];
#pragma unroll
    for (int db = 0; db < R::DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.0f;
    float m = -INFINITY, l = 0.0f;  // running (possibly stale) max of raw scores; this lane's partial sum of weights
    f32x16 s_cur[2];                // S^T of the current tile, 32 keys each
    u32x4 p_cur[4];                 // its weights, bf16 pairs, 16 keys each
    float ps_cur;                   // this lane's sum of them so far

    constexpr int kPairs = 16, kPairsB = 8;  // score pairs of a tile; those exponentiated in block B
    auto exp_pair = [&](const f32x16 (&sc)[2], u32x4 (&p)[4], float& ps, int pi) {
      const int nb = pi / 8, r = 2 * (pi % 8);
      const float mc = m * c2;
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nb][r], c2, -mc));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nb][r + 1], c2, -mc));
      ps = ps + (p0 + p1);
      const uint32_t w = round_pair(p0, p1);
      asm volatile("" ::"v"(w));  // keep the weight in its pipeline step
      p[2 * nb + (r >> 3)][(r & 7) >> 1] = w;
    };
    auto row_max = [&](const f32x16 (&sc)[2]) {
      float m0 = sc[0][0], m1 = sc[1][0];
#pragma unroll
      for (int r = 1; r < 15; r += 2) {
        m0 = __builtin_elementwise_maximum(m0, __builtin_elementwise_maximum(sc[0][r], sc[0][r + 1]));
        m1 = __builtin_elementwise_maximum(m1, __builtin_elementwise_maximum(sc[1][r], sc[1][r + 1]));
      }
      return pair_max(__builtin_elementwise_maximum(
          m0, __builtin_elementwise_maximum(m1, __builtin_elementwise_maximum(sc[0][15], sc[1][15]))));
    };
    auto qk_tile = [&](int t, const char* kb_lds, f32x16 (&sc)[2]) {
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[nb][r] = 0.0f;
#pragma unroll
      for (int kb = 0; kb < R::KB; ++kb) {
        const bf16x8 k0 = *reinterpret_cast<const bf16x8*>(kb_lds + rd.k[kb]);
        const bf16x8 k1 = *reinterpret_cast<const bf16x8*>(kb_lds + rd.k[kb] + 32 * D * 2);
        sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qf[kb], sc[0], 0, 0, 0);
        sc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qf[kb], sc[1], 0, 0, 0);
      }
      if (hides(t)) mask(t, sc);
    };
    // A tile again against the exact running max: its scores from its K buffer,
    // new m, O and l rescaled, all weights anew.
    auto redo_tile = [&](int t, const char* kb_lds, u32x4 (&p)[4], float& ps) {
      f32x16 sc[2];
      qk_tile(t, kb_lds, sc);
      const float m_new = __builtin_elementwise_maximum(m, row_max(sc));
      const float alpha = __builtin_amdgcn_exp2f((m - m_new) * c2);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      ps = 0.0f;
#pragma unroll
      for (int pi = 0; pi < kPairs; ++pi) exp_pair(sc, p, ps, pi);
    };
    auto close_tile = [&](int t, const char* kb_lds, u32x4 (&p)[4], float& ps) {
      if (__any(!(ps <= kRescaleBound))) redo_tile(t, kb_lds, p, ps);
      l += ps;
    };
    auto read_k = [&](const char* kb_lds, int kb, bf16x8 (&kf)[2]) {
      kf[0] = *reinterpret_cast<const bf16x8*>(kb_lds + rd.k[kb]);
      kf[1] = *reinterpret_cast<const bf16x8*>(kb_lds + rd.k[kb] + 32 * D * 2);
    };
    constexpr int kStepsB = 2 * R::DB;  // block B steps: (16 keys, pair of 32-row blocks)
    constexpr int kPrefetch = D == 64 ? 2 : 1;  // steps between an LDS read and its MFMA

    // Iteration of tile t: kb_cur, vb_cur its buffers, kb_next tile t+1's K,
    // kb_load, vb_load the free ones.  LOAD: tile t+2 exists; NEXT: tile t+1 does.
    auto iteration = [&](int t, const char* kb_cur, const char* vb_cur, const char* kb_next, char* kb_load, char* vb_load,
                         auto load_c, auto next_c) {
      constexpr bool LOAD = decltype(load_c)::value;
      constexpr bool NEXT = decltype(next_c)::value;
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();  // tiles t, t+1 landed for every wave; tile t-1's buffers are free
      f32x16 s_next[2];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s_next[nb][r] = 0.0f;
      bf16x8 kring[kPrefetch + 1][2];
      bf16x8 vring[kPrefetch + 1][2];
      if constexpr (NEXT) {
#pragma unroll
        for (int j = 0; j < kPrefetch && j < R::KB; ++j) read_k(kb_next, j, kring[j]);
      }
#pragma unroll
      for (int st = 0; st < R::KB; ++st) {
        if constexpr (NEXT) {
          if (st + kPrefetch < R::KB) read_k(kb_next, st + kPrefetch, kring[(st + kPrefetch) % (kPrefetch + 1)]);
        }
        {
          const int j = st + kPrefetch - R::KB;  // block B step to prefetch
          if (j >= 0 && j < kStepsB) {
#pragma unroll
            for (int d = 0; d < 2; ++d)
              vring[j % (kPrefetch + 1)][d] = read_v<D>(vb_cur, rd, j / (R::DB / 2), (j % (R::DB / 2)) * 2 + d);
          }
        }
        if constexpr (LOAD) {
          if (st == 0) load_tile(t + 2, kb_load, vb_load);
        }
        if constexpr (NEXT) {
#pragma unroll
          for (int nb = 0; nb < 2; ++nb)
            s_next[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kring[st % (kPrefetch + 1)][nb], qf[st], s_next[nb], 0, 0, 0);
        }
#pragma unroll
        for (int pi = kPairsB; pi < kPairs; ++pi)
          if (st == (pi - kPairsB) * R::KB / (kPairs - kPairsB)) exp_pair(s_cur, p_cur, ps_cur, pi);
        __builtin_amdgcn_sched_barrier(0);
      }
      close_tile(t, kb_cur, p_cur, ps_cur);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (NEXT) {
        if (hides(t + 1)) mask(t + 1, s_next);
      }
      u32x4 p_next[4];
      float ps_next = 0.0f;
#pragma unroll
      for (int st = 0; st < kStepsB; ++st) {
        const int ks = st / (R::DB / 2), db0 = (st % (R::DB / 2)) * 2;
        if (st + kPrefetch < kStepsB) {
          const int j = st + kPrefetch;
#pragma unroll
          for (int d = 0; d < 2; ++d)
            vring[j % (kPrefetch + 1)][d] = read_v<D>(vb_cur, rd, j / (R::DB / 2), (j % (R::DB / 2)) * 2 + d);
        }
#pragma unroll
        for (int d = 0; d < 2; ++d)
          o[db0 + d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vring[st % (kPrefetch + 1)][d],
                                                               __builtin_bit_cast(bf16x8, p_cur[ks]), o[db0 + d], 0, 0, 0);
        if constexpr (NEXT) {
#pragma unroll
          for (int pi = 0; pi < kPairsB; ++pi)
            if (st == pi * kStepsB / kPairsB) exp_pair(s_next, p_next, ps_next, pi);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (NEXT) {
        s_cur[0] = s_next[0];
        s_cur[1] = s_next[1];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) p_cur[ks] = p_next[ks];
        ps_cur = ps_next;
      }
    };

    __syncthreads();  // the last segment's reads of the buffers are done
    find(s.u0);
    load_tile(s.u0, kbuf[0], vbuf[0]);
    if (s.u0 + 1 < s.u1) load_tile(s.u0 + 1, kbuf[1], vbuf[1]);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    qk_tile(s.u0, kbuf[0], s_cur);
    m = row_max(s_cur);
    // No visible key yet: weights 0 against a finite max below any score
    // (against minus infinity they would be NaN), which a later tile redoes.
    if (m == -INFINITY) m = -1e30f;
    ps_cur = 0.0f;
#pragma unroll
    for (int pi = 0; pi < kPairsB; ++pi) exp_pair(s_cur, p_cur, ps_cur, pi);

    using T = std::true_type;
    using F = std::false_type;
    int t = s.u0, b = 0;
    while (t + 2 < s.u1) {
      iteration(t, kbuf[0], vbuf[0], kbuf[1], kbuf[2], vbuf[2], T{}, T{});
      ++t;
      b = 1;
      if (t + 2 >= s.u1) break;
      iteration(t, kbuf[1], vbuf[1], kbuf[2], kbuf[0], vbuf[0], T{}, T{});
      ++t;
      b = 2;
      if (t + 2 >= s.u1) break;
      iteration(t, kbuf[2], vbuf[2], kbuf[0], kbuf[1], vbuf[1], T{}, T{});
      ++t;
      b = 0;
    }
    auto buf_of = [&](char* const (&buf)[3], int i) -> const char* { return i == 0 ? buf[0] : i == 1 ? buf[1] : buf[2]; };
    if (t + 1 < s.u1) {
      const int n = b == 2 ? 0 : b + 1;
      iteration(t, buf_of(kbuf, b), buf_of(vbuf, b), buf_of(kbuf, n), nullptr, nullptr, F{}, T{});
      ++t;
      b = n;
    }
    iteration(t, buf_of(kbuf, b), buf_of(vbuf, b), nullptr, nullptr, nullptr, F{}, F{});

    l = pair_sum(l);
    const int r = wave * 32 + l32;
    if (s.slot < 0) {
      const float inv = 1.0f / l;
      float all = inv;
      char* out = a.out + size_t(qr.row) * a.out_pitch + size_t(qr.head) * D * 2;
#pragma unroll
      for (int db = 0; db < R::DB; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const float x0 = o[db][4 * g4] * inv, x1 = o[db][4 * g4 + 1] * inv, x2 = o[db][4 * g4 + 2] * inv,
                      x3 = o[db][4 * g4 + 3] * inv;
          all += (x0 + x1) + (x2 + x3);
          if (r < s.rows) {
            uint2 y = {round_pair(x0, x1), round_pair(x2, x3)};
            *reinterpret_cast<uint2*>(out + (32 * db + 8 * g4 + 4 * hh) * 2) = y;
          }
        }
      if (a.lse && hh == 0 && r < s.rows) a.lse[size_t(qr.head) * a.rows + qr.row] = (m * c2 + __log2f(l)) * kLn2;
      const bool bad = __any(r < s.rows && !(__builtin_fabsf(all) < INFINITY));
      if (lane == 0) mark(bad ? 1 : 0);
    } else {
      float* slot = v.scratch + size_t(max(s.slot, 0)) * paged_slot_floats(kShape.rows, D);
      if (r < s.rows) {
        float* row = slot + size_t(r) * D + 4 * hh;
#pragma unroll
        for (int db = 0; db < R::DB; ++db)
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4)
            *reinterpret_cast<float4*>(row + 32 * db + 8 * g4) =
                make_float4(o[db][4 * g4], o[db][4 * g4 + 1], o[db][4 * g4 + 2], o[db][4 * g4 + 3]);
        if (hh == 0) {
          slot[kShape.rows * D + r] = m * c2;
          slot[kShape.rows * (D + 1) + r] = l;
        }
      }
      if (s.u0 == 0 && lane == 0) mark(0);
    }
  });
}

template <int D>
__global__ __launch_bounds__(kNarrowThreads, 2) void paged_narrow_bf16(PagedAttendArgs a) {
  paged_narrow_body<D>(a);
}
template <int D, bool WHOLE>
__global__ __launch_bounds__(2 * paged_wide_bf16_shape(D).rows, 2 - paged_wide_bf16_shape(D).rows / 256) void paged_wide_bf16(PagedAttendArgs a) {
  paged_wide_body<D, WHOLE>(a);
}

}  // namespace

hipError_t launch_paged_bf16(const PagedAttendArgs& a, bool narrow, hipStream_t stream) {
  const bool d128 = a.v.head_dim == 128, whole = a.v.page_tokens % kKeys == 0;
  const TileShape wide = paged_wide_bf16_shape(a.v.head_dim);
  auto kernel = narrow ? (d128 ? paged_narrow_bf16<128> : paged_narrow_bf16<64>)
                : whole ? (d128 ? paged_wide_bf16<128, true> : paged_wide_bf16<64, true>)
                        : (d128 ? paged_wide_bf16<128, false> : paged_wide_bf16<64, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(narrow ? kPagedNarrowBf16.groups : wide.groups)),
                     dim3(narrow ? kNarrowThreads : 2 * wide.rows), 0, stream, a);
  return hipGetLastError();
}

}  // namespace fademem
