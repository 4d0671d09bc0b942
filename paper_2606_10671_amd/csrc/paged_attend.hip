// Attention of a step's queries over the paged window memory.
//
// O = softmax(scale Q K^T) V over the keys that a row sees: the sinks [0, S) and
// the window [low, high) of its position.
#include "bf16_round.h"
#include "paged_internal.h"

namespace fademem {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRowWaves = 4;

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

// Byte address of key (or value) `key` of sequence table `table`, key head hk.
__device__ __forceinline__ const char* key_row(const PagedAttendArgs& a, const int32_t* table, int key, int hk, int kv,
                                               int row_bytes) {
  const int page = key / a.v.page_tokens, off = key - page * a.v.page_tokens;
  const int32_t id = min(max(table[page], 0), int32_t(a.v.n_pages) - 1);
  return a.pages + size_t(id) * a.v.page_bytes + (size_t(kv * a.v.kv_heads + hk) * a.v.page_tokens + off) * row_bytes;
}

// One row of one head by one wave: a lane takes a key of 64, then two (or one)
// elements of the output.  q_s: the wave's D floats of LDS.
template <bool BF16, int D>
__device__ void attend_row(const PagedAttendArgs& a, int s, int row, int h, float* q_s) {
  constexpr int kPer = D / 64;  // output elements per lane
  constexpr int kElt = BF16 ? 2 : 4;
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 63, hk = h / v.group;
  const char* q = a.q + size_t(row) * a.q_pitch + size_t(h) * D * kElt;
  for (int d = lane; d < D; d += 64)
    q_s[d] = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(q)[d]) << 16)
                  : reinterpret_cast<const float*>(q)[d];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int32_t* table = v.table + size_t(s) * v.width;
  const int pos = v.first[s] + row - v.q_start[s], held = v.held[s];
  const int low = int(paged_low(v, pos)), high = v.added[s] > 0 ? int(paged_high(v, pos, held)) : 0;
  const int sinks = int(min(v.sink_tokens, int64_t(min(low, high))));
  const float c2 = a.scale * kLog2e;
  float m = -INFINITY, l = 0.0f, o[kPer] = {};
  for (int part = 0; part < 2; ++part) {
    const int end = part ? high : sinks;
    for (int k0 = part ? low : 0; k0 < end; k0 += 64) {
      const int key = k0 + lane, n = min(64, end - k0);
      const char* vrow = nullptr;
      float x = -INFINITY;
      if (key < end) {
        const char* krow = key_row(a, table, key, hk, 0, D * kElt);
        vrow = krow + size_t(v.kv_heads) * v.page_tokens * D * kElt;
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
      for (int j = 0; j < n; ++j) {
        const float pj = __shfl(p, j);
        const char* vr = reinterpret_cast<const char*>(__shfl(reinterpret_cast<unsigned long long>(vrow), j));
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int d = lane * kPer + e;
          const float x1 = BF16 ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(vr)[d]) << 16)
                                : reinterpret_cast<const float*>(vr)[d];
          o[e] = __builtin_fmaf(pj, x1, o[e]);
        }
      }
      if (l != l) k0 = end, part = 2;  // a NaN score: every element is NaN
    }
  }
  char* out = a.out + size_t(row) * a.out_pitch + size_t(h) * D * kElt;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const float y = l != l ? l : high > 0 ? o[e] / l : 0.0f;
    if constexpr (BF16) reinterpret_cast<__bf16*>(out)[lane * kPer + e] = (__bf16)y;
    else reinterpret_cast<float*>(out)[lane * kPer + e] = y;
  }
  if (a.lse && lane == 0) a.lse[size_t(h) * a.rows + row] = high > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
}

template <bool BF16, int D>
__global__ __launch_bounds__(64 * kRowWaves) void paged_attend_rows_kernel(PagedAttendArgs a) {
  __shared__ float q_s[kRowWaves][D];
  const int wave = threadIdx.x >> 6;
  const int64_t i = int64_t(blockIdx.x) * kRowWaves + wave;
  const int row = int(i / a.v.heads), h = int(i - int64_t(row) * a.v.heads);
  if (row >= a.v.q_start[a.v.seqs]) return;
  int lo = 0, hi = a.v.seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.v.q_start[mid] <= row) lo = mid;
    else hi = mid;
  }
  attend_row<BF16, D>(a, lo, row, h, q_s[wave]);
}

}  // namespace

hipError_t launch_paged_attend(const PagedAttendArgs& a, bool bf16, bool narrow, hipStream_t stream) {
  (void)narrow;
  auto kernel = a.v.head_dim == 128 ? (bf16 ? paged_attend_rows_kernel<true, 128> : paged_attend_rows_kernel<false, 128>)
                                    : (bf16 ? paged_attend_rows_kernel<true, 64> : paged_attend_rows_kernel<false, 64>);
  const int64_t blocks = (a.rows * a.v.heads + kRowWaves - 1) / kRowWaves;
  if (blocks > int64_t(0x7fffffff)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kernel, dim3(unsigned(blocks)), dim3(64 * kRowWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace fademem
