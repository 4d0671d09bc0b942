// Paged attention: what follows the kernels of paged_bf16.hip and paged_f32.hip.
//
// paged_finish_kernel
// * joins the partial results of row tiles whose keys several workgroups shared,
//   in the order of the workgroups: O = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i;
// * works out again, key by key, rows whose result is not finite.  The matrix
//   kernels give a hidden key the weight 0, and 0 times an infinite or NaN value
//   is NaN: such a row is only right if it saw that value.  attend_row adds up
//   the keys that the row sees and no others;
// * writes 0 (and an LSE of minus infinity) to the rows of sequences that were
//   not admitted to the step.
#include "paged_device.h"

namespace fademem {
namespace {

constexpr int kFinishThreads = 256;
constexpr int kFinishWaves = kFinishThreads / 64;

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Address of key `key` of a sequence in key head hk's K rows.
__device__ __forceinline__ const char* key_row(const PagedAttendArgs& a, const int32_t* table, int key, int hk,
                                               int row_bytes) {
  const int page = page_of(a.v, key), off = key - page * a.v.page_tokens;
  return a.pages + size_t(safe_page(a.v, table[page])) * a.v.page_bytes +
         (size_t(hk) * a.v.page_tokens + off) * row_bytes;
}

// One row of one head by one wave: a lane takes one key of 64, then D/64
// elements of the output.  q_s: the wave's D floats of LDS.
template <bool BF16, int D>
__device__ void attend_row(const PagedAttendArgs& a, int s, const QueryRow& qr, float* q_s) {
  constexpr int kPer = D / 64;  // output elements per lane
  constexpr int kElt = BF16 ? 2 : 4;
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 63, hk = qr.head / v.group;
  const char* q = a.q + size_t(qr.row) * a.q_pitch + size_t(qr.head) * D * kElt;
  for (int d = lane; d < D; d += 64)
    q_s[d] = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(q)[d]) << 16)
                  : reinterpret_cast<const float*>(q)[d];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int32_t* table = v.table + size_t(s) * v.width;
  const int sinks = min(v.sink_tokens, min(qr.low, qr.high));
  const float c2 = a.scale * kLog2e;
  const char* const v0 = a.pages;
  float m = -INFINITY, l = 0.0f, o[kPer] = {};
  bool dead = false;
  for (int part = 0; part < 2; ++part) {
    const int end = part ? qr.high : sinks;
    for (int k0 = part ? qr.low : 0; k0 < end; k0 += 64) {
      const int key = k0 + lane, n = min(64, end - k0);
      uint64_t v_at = 0;
      float x = -INFINITY;
      if (key < end) {
        const char* krow = key_row(a, table, key, hk, D * kElt);
        v_at = uint64_t(krow - v0) + size_t(v.kv_heads) * v.page_tokens * D * kElt;
        x = 0.0f;
        for (int d = 0; d < D; d += 16 / kElt) {
          const uint4 w = *reinterpret_cast<const uint4*>(krow + d * kElt);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (BF16) {
              x = __builtin_fmaf(q_s[d + 2 * e], __uint_as_float(ws[e] << 16), x);
              x = __builtin_fmaf(q_s[d + 2 * e + 1], __uint_as_float(ws[e] & 0xffff0000u), x);
            } else {
              x = __builtin_fmaf(q_s[d + e], __uint_as_float(ws[e]), x);
            }
          }
        }
        x *= c2;
      }
      const float m_new = fmaxf(m, wave_max(x));
      const float ref = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = exp2f(m - ref);
      const float p = key < end ? exp2f(x - ref) : 0.0f;
      m = m_new;
      l = l * alpha + wave_sum(p);
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] *= alpha;
      // A key at a time for all of V's elements, four of them in flight.
      auto add = [&](int j) {
        const float pj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), j));
        const char* vr = v0 + ((uint64_t(uint32_t(__builtin_amdgcn_readlane(uint32_t(v_at >> 32), j))) << 32) |
                               uint32_t(__builtin_amdgcn_readlane(uint32_t(v_at), j)));
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int d = lane * kPer + e;
          const float x1 = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(vr)[d]) << 16)
                                : reinterpret_cast<const float*>(vr)[d];
          o[e] = __builtin_fmaf(pj, x1, o[e]);
        }
      };
      if (!dead) {
        int j = 0;
        for (; j + 4 <= n; j += 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) add(j + i);
        }
        for (; j < n; ++j) add(j);
        bool nan = true;
#pragma unroll
        for (int e = 0; e < kPer; ++e) nan = nan && o[e] != o[e];
        dead = __all(nan);  // every element is NaN and stays it
      }
      if (dead && !a.lse) break;
      if (l != l) break;  // a NaN score: every element is NaN
    }
    if (l != l || (dead && !a.lse)) break;
  }
  char* out = a.out + size_t(qr.row) * a.out_pitch + size_t(qr.head) * D * kElt;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const float y = l != l ? l : o[e] / l;
    if constexpr (BF16) reinterpret_cast<__bf16*>(out)[lane * kPer + e] = (__bf16)y;
    else reinterpret_cast<float*>(out)[lane * kPer + e] = y;
  }
  if (a.lse && lane == 0) a.lse[size_t(qr.head) * a.rows + qr.row] = (m + log2f(l)) * kLn2;
}

// grid = (groups at most, chunks of a tile's rows): a block joins ROWS rows of the
// tile that workgroup blockIdx.x is the first to begin inside.  Bound by latency:
// kernel arguments, plan, partial results (beside the sequence's lengths), results;
// 8 to 11 us, 16 to 18 where every workgroup shares a tile of 256 x 128.
// SLICED = false (wide tiles, few parts): a thread takes four elements of several
// rows, two parts at a time.  SLICED (narrow tiles, up to hundreds of parts): the
// block's threads share out the parts of ROWS rows, AHEAD of them in flight per
// thread, and add up through LDS.  Each keeps a running max.
template <bool BF16, int D, bool SLICED, int ROWS, int AHEAD>
__global__ __launch_bounds__(kFinishThreads) void paged_finish_kernel(PagedAttendArgs a, TileShape shape, int rows_used) {
  constexpr int kLanes = D / 4, kSlices = kFinishThreads / kLanes;  // threads of a row; rows (or parts) side by side
  constexpr int kPer = SLICED ? ROWS : ROWS / kSlices;  // rows of a thread
  __shared__ float q_s[kFinishWaves][D];
  __shared__ int list[kFinishThreads + 1], n_list;
  __shared__ float4 o_s[SLICED ? ROWS : 1][SLICED ? kFinishThreads : 1];
  __shared__ float2 ml_s[SLICED ? ROWS : 1][kSlices];
  const PagedView& v = a.v;
  const int tid = threadIdx.x, wave = tid >> 6, g = blockIdx.x;
  const CONST_AS int32_t* h = plan_array(&v.header->groups);
  const CONST_AS int32_t* start = plan_array(reinterpret_cast<const int32_t*>(v.starts + g));
  const int groups = h[0], tiles = h[1], refused = h[2], join = plan_array(v.joins)[g];
  const int start_task = start[0];
  const EvenPlan even = {h[5], h[6], h[7], h[8], h[9], h[10], h[11], h[12], h[13]};
  const bool is_even = shape.even && even.even;
  if (h[3] != a.rows || h[4] != a.max_new) return;  // another step is planned
  // Parts: group g - 1's last units, then the first units of groups g, g + 1, ...; of an even plan, those of tile g
  // of the tiles left over.
  int parts = 0;
  if (is_even) {
    if (g < even.rem) parts = even.heads + (even.tail_len > 0 ? 1 : 0);
  } else if (g > 0 && g < groups) {
    parts = join;
  }
  static_assert(offsetof(PagedHeader, again) == offsetof(PagedHeader, groups) + 14 * sizeof(int32_t), "h[14]");
  const bool marks = h[14] != 0;
  Segment mine = {};
  bool again = false;
  if (parts > 1) {
    Segment s;
    const int slot0 = is_even ? g : 2 * g - 1, slot1 = is_even ? g + even.rem : 2 * g, step = is_even ? even.rem : 2;
    const int lane = tid % kLanes, c = 4 * lane, slice = tid / kLanes, base = blockIdx.y * ROWS;
    const size_t slot = paged_slot_floats(shape.rows, D);
    auto part = [&](int p) { return v.scratch + size_t(p == 0 ? slot0 : slot1 + (p - 1) * step) * slot; };
    auto find = [&] {
      s.task = is_even ? even.rounds * even.groups + g : start_task;
      describe(v, shape, s);
    };
    bool bad = false;
    auto store = [&](int r, float m, float l, const float4& o) {
      const int t = (s.row0 + r) / v.group, head = s.head * v.group + s.row0 + r - t * v.group, row = s.q_start + t;
      const float inv = 1.0f / l;
      char* out = a.out + size_t(row) * a.out_pitch + (size_t(head) * D + c) * (BF16 ? 2 : 4);
      if constexpr (BF16) {
        const uint2 y = {round_pair(o.x * inv, o.y * inv), round_pair(o.z * inv, o.w * inv)};
        *reinterpret_cast<uint2*>(out) = y;
      } else {
        *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      }
      if (a.lse && c == 0) a.lse[size_t(head) * a.rows + row] = (m + log2f(l)) * kLn2;
      const float sum = (o.x + o.y) + (o.z + o.w) + inv;
      bad = bad || !(__builtin_fabsf(sum) < INFINITY);
    };
    // Rows of this thread, and its parts: all of them, or every kSlices-th.  Rows below the host's bound are read
    // before the sequence's lengths are known.
    auto row_of = [&](int i) { return SLICED ? base + i : base + slice + i * kSlices; };
    float4 o[kPer];
    float m[kPer], l[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      o[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      m[i] = -INFINITY;
      l[i] = 0.0f;
    }
    constexpr int kStep = SLICED ? kSlices : 1;
    for (int p0 = SLICED ? slice : 0; p0 < parts; p0 += kStep * AHEAD) {
      float4 y[AHEAD][kPer];
      float my[AHEAD][kPer], ly[AHEAD][kPer];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int p = p0 + j * kStep;
        const float* x = part(min(p, parts - 1));
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int row = min(row_of(i), rows_used - 1);
          y[j][i] = *reinterpret_cast<const float4*>(x + size_t(row) * D + c);
          my[j][i] = p < parts ? x[shape.rows * D + row] : -INFINITY;
          ly[j][i] = x[shape.rows * (D + 1) + row];
        }
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        float top = m[i];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) top = __builtin_elementwise_maximum(top, my[j][i]);
        const float ref = top == -INFINITY ? 0.0f : top, f0 = exp2f(m[i] - ref);
        m[i] = top;
        l[i] *= f0;
        o[i] = make_float4(o[i].x * f0, o[i].y * f0, o[i].z * f0, o[i].w * f0);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          if (p0 + j * kStep >= parts) continue;
          const float f = exp2f(my[j][i] - ref);
          l[i] += f * ly[j][i];
          o[i].x += f * y[j][i].x;
          o[i].y += f * y[j][i].y;
          o[i].z += f * y[j][i].z;
          o[i].w += f * y[j][i].w;
        }
      }
    }
    find();
    if constexpr (!SLICED) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (row_of(i) < s.rows) store(row_of(i), m[i], l[i], o[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        o_s[i][tid] = o[i];
        if (lane == 0) ml_s[i][slice] = make_float2(m[i], l[i]);
      }
      __syncthreads();
      for (int i = tid; i < min(ROWS, s.rows - base) * kLanes; i += kFinishThreads) {  // kLanes divides the step
        const int r = i / kLanes;
        float top = ml_s[r][0].x;
#pragma unroll
        for (int k = 1; k < kSlices; ++k) top = __builtin_elementwise_maximum(top, ml_s[r][k].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float ls = 0.0f;
#pragma unroll
        for (int k = 0; k < kSlices; ++k) {
          const float2 ml = ml_s[r][k];
          const float f = exp2f(ml.x - ref);
          const float4 z = o_s[r][k * kLanes + lane];
          ls += f * ml.y;
          sum.x += f * z.x;
          sum.y += f * z.y;
          sum.z += f * z.z;
          sum.w += f * z.w;
        }
        store(base + r, top, ls, sum);
      }
    }
    again = __syncthreads_or(bad);
    mine = s;
  }

  // Rows again: this block's, if joining them gave something that is not finite, and rows of whole tiles that the
  // attention marked.  An infinity or NaN that every row sees marks them all, and key by key a row costs 115 times
  // what it does by matrix (4680 rows of 12 heads over 23 400 keys: 74 ms), so they are spread over all blocks: 512
  // tiles of 128 rows over 640 keys 1.7 ms, 895 with 256 tiles to a block.
  if (again || marks) {
    // Blocks of 32 rows of whole tiles, none if no attention since the plan marked any: thread t of block b looks at
    // number b, and t times as many as there are blocks behind it, so that marked ones lying together go to different blocks.
    const int per_shift = shape.rows == 32 ? 0 : shape.rows == 128 ? 2 : 3;  // 32-row blocks of a tile
    const int64_t jobs = marks ? (int64_t(tiles) * v.kv_heads) << per_shift : 0, blocks = int64_t(gridDim.x) * gridDim.y;
    const int64_t job0 = int64_t(blockIdx.y) * gridDim.x + g;
    for (int64_t j0 = job0; again || j0 < jobs; j0 += blocks * kFinishThreads) {
      const int64_t at = j0 + tid * blocks;
      const int mark =
          at < jobs ? reinterpret_cast<const uint8_t*>(v.redo)[(at >> per_shift) * 8 + (at & ((1 << per_shift) - 1))] : 0;
      if (!__syncthreads_or(mark) && !again) continue;
      if (tid == 0) {
        n_list = again;
        list[0] = -1;
      }
      __syncthreads();
      if (mark) list[atomicAdd(&n_list, 1)] = tid;
      __syncthreads();
      for (int i = 0; i < n_list; ++i) {
        Segment s = mine;
        int r0 = blockIdx.y * ROWS, r1 = min(r0 + ROWS, mine.rows);
        if (list[i] >= 0) {
          const int64_t job = j0 + list[i] * blocks;
          s.task = int(job >> per_shift);
          describe(v, shape, s);
          r0 = 32 * int(job & ((1 << per_shift) - 1));
          r1 = min(r0 + 32, s.rows);
        }
        for (int r = r0 + wave; r < r1; r += kFinishWaves) attend_row<BF16, D>(a, s.seq, query_row(v, s, r), q_s[wave]);
      }
      again = false;
      __syncthreads();
    }
  }
  if (blockIdx.y > 0 || !refused) return;

  // Rows of sequences that were not admitted.
  for (int s = g; s < v.seqs; s += gridDim.x) {
    if (v.status[s] == FADEMEM_OK) continue;
    const int r0 = v.q_start[s], r1 = v.q_start[s + 1];
    const int units = v.heads * D * (BF16 ? 2 : 4) / 16;
    for (int64_t i = tid; i < int64_t(r1 - r0) * units; i += kFinishThreads) {
      const int64_t row = r0 + i / units;
      reinterpret_cast<uint4*>(a.out + size_t(row) * a.out_pitch)[i % units] = make_uint4(0, 0, 0, 0);
    }
    if (a.lse)
      for (int64_t i = tid; i < int64_t(r1 - r0) * v.heads; i += kFinishThreads)
        a.lse[(i / (r1 - r0)) * a.rows + r0 + i % (r1 - r0)] = -INFINITY;
  }
}

using FinishKernel = void (*)(PagedAttendArgs, TileShape, int);

// The kernel whose blocks join `rows` rows.
template <bool BF16, int D>
FinishKernel finish_kernel(int rows) {
  return rows == 32 ? paged_finish_kernel<BF16, D, false, 32, 2>
         : rows == 1 ? paged_finish_kernel<BF16, D, true, 1, 4>
                     : paged_finish_kernel<BF16, D, true, 4, 2>;
}

}  // namespace

hipError_t launch_paged_finish(const PagedAttendArgs& a, bool bf16, TileShape shape, hipStream_t stream) {
  const int64_t most = a.max_new * a.v.group;  // rows of a sequence
  const int rows_used = int(most < 1 ? 1 : most < shape.rows ? most : shape.rows);
  // Narrow tiles: a block per row or, from five rows on, per four (32 rows of 32 tiles over 8000 tokens: a block per
  // row 104 us a call, per four 64); wide ones: a block per 32.
  const bool d128 = a.v.head_dim == 128, narrow = shape.rows == kPagedMinTileRows;
  const int rows = !narrow ? 32 : rows_used <= 4 ? 1 : 4;
  const FinishKernel kernel = bf16 ? (d128 ? finish_kernel<true, 128>(rows) : finish_kernel<true, 64>(rows))
                                   : (d128 ? finish_kernel<false, 128>(rows) : finish_kernel<false, 64>(rows));
  hipLaunchKernelGGL(kernel, dim3(unsigned(shape.groups), unsigned((rows_used + rows - 1) / rows)), dim3(kFinishThreads), 0,
                     stream, a, shape, rows_used);
  return hipGetLastError();
}

}  // namespace fademem
