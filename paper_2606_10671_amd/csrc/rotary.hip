// Rotary positions with several axes on rows of heads (rotary_device.h has the
// mathematics).
//
// A block takes a few rows: the angles' cos and sin of each (row, pair) are made
// once, in LDS, and serve every head of the row; then every thread turns
// 16-byte units (for half-split pairs: two of them).  Reads and writes each
// element once.  Bound by memory where the call is large (fp32 10 007 rows of
// 24 x 64: 123 MB in 20 us, 6.1 TB/s), below that by the chain of launch, angles and
// one round of loads (bf16 4680 rows of 12 x 128: 28.8 MB in 9.5 us; 16 rows 3.6).
#include <math.h>

#include "rotary_device.h"

namespace fademem {

namespace {

struct RopeArgs {
  const char* x;
  char* y;
  size_t x_pitch, y_pitch;  // bytes between rows
  const int32_t* pos;
  int64_t rows;
  int heads;
  int per_block;            // rows of a block
  RotaryArg rot;
};

template <bool BF16, bool HALVES>
__global__ __launch_bounds__(kRotThreads) void rope_kernel(RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) double2 cs[];
  constexpr int kElts = BF16 ? 8 : 4;  // elements per 16-byte unit
  const int64_t row0 = int64_t(blockIdx.x) * a.per_block;
  const int n = int(min(int64_t(a.per_block), a.rows - row0));
  const int head_units = a.rot.head_dim / kElts, half = head_units / 2;
  const int per_head = HALVES ? half : head_units;
  const int per_row = a.heads * per_head, items = n * per_row;
  rotary_angles(a.rot, a.pos, row0, n, cs);
  __syncthreads();
  for (int i = threadIdx.x; i < items; i += kRotThreads) {
    const int t = i / per_row, r = i - t * per_row;
    const int h = r / per_head, u = r - h * per_head;
    const rot_u32x4* src = reinterpret_cast<const rot_u32x4*>(a.x + size_t(row0 + t) * a.x_pitch) + h * head_units + u;
    rot_u32x4* dst = reinterpret_cast<rot_u32x4*>(a.y + size_t(row0 + t) * a.y_pitch) + h * head_units + u;
    const double2* c = cs + t * a.rot.pairs;
    if constexpr (HALVES) {
      rot_u32x4 p = src[0], q = src[half];
      rotate_halves<BF16>(p, q, c, u * kElts, a.rot.pairs);
      dst[0] = p;
      dst[half] = q;
    } else {
      dst[0] = rotate_unit<BF16>(src[0], c, u * (kElts / 2), a.rot.pairs);
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

bool rows_apart(const char* x, size_t x_pitch, const char* y, size_t y_pitch, int64_t rows, size_t row) {
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), x1 = x0 + size_t(rows - 1) * x_pitch + row;
  const uintptr_t y0 = reinterpret_cast<uintptr_t>(y), y1 = y0 + size_t(rows - 1) * y_pitch + row;
  if (x1 <= y0 || y1 <= x0) return true;
  if (x_pitch != y_pitch) return false;
  const size_t gap = (x0 > y0 ? x0 - y0 : y0 - x0) % x_pitch;  // slices of one row, side by side
  return gap >= row && gap + row <= x_pitch;
}

int rotary_arg(const fademem_rope* r, int inverse, RotaryArg* out) {
  if (!r || (inverse != 0 && inverse != 1)) return FADEMEM_EINVAL;
  if (r->head_dim < 16 || r->head_dim > 2 * FADEMEM_ROPE_MAX_PAIRS || r->head_dim % 16) return FADEMEM_EINVAL;
  if (r->layout != FADEMEM_ROPE_INTERLEAVED && r->layout != FADEMEM_ROPE_HALVES) return FADEMEM_EINVAL;
  int64_t n = 0;
  for (int p : r->pairs) {
    if (p < 0) return FADEMEM_EINVAL;
    n += p;
  }
  if (n < 1 || n > r->head_dim / 2) return FADEMEM_EINVAL;
  for (int i = 0; i < n; ++i)
    if (!isfinite(r->freq[i])) return FADEMEM_EINVAL;
  out->head_dim = r->head_dim;
  out->pairs = int(n);
  out->end_t = r->pairs[0];
  out->end_h = r->pairs[0] + r->pairs[1];
  out->halves = r->layout == FADEMEM_ROPE_HALVES;
  out->sign = inverse ? -1.0 : 1.0;
  for (int i = 0; i < FADEMEM_ROPE_MAX_PAIRS; ++i) out->freq[i] = i < n ? r->freq[i] : 0.0;
  return FADEMEM_OK;
}

}  // namespace fademem

using namespace fademem;

extern "C" {

int fademem_rope_init(fademem_rope* rope, int32_t head_dim, int32_t layout, int32_t pairs_t, int32_t pairs_h,
                      int32_t pairs_w, double theta) {
  if (!rope || !(theta > 1.0 && theta < 1e300)) return FADEMEM_EINVAL;
  fademem_rope r = {};
  r.head_dim = head_dim;
  r.layout = layout;
  r.pairs[0] = pairs_t;
  r.pairs[1] = pairs_h;
  r.pairs[2] = pairs_w;
  RotaryArg checked;
  if (int rc = rotary_arg(&r, 0, &checked)) return rc;
  int i = 0;
  for (int p : r.pairs)
    for (int k = 0; k < p; ++k) r.freq[i++] = pow(theta, -double(k) / double(p));
  *rope = r;
  return FADEMEM_OK;
}

int fademem_rope_apply(const fademem_rope* rope, int32_t dtype, const int32_t* pos, int64_t rows, int32_t heads,
                       const void* x, int64_t x_stride, void* y, int64_t y_stride, int32_t inverse, void* stream) {
  RopeArgs a;
  if (int rc = rotary_arg(rope, inverse, &a.rot)) return rc;
  if (dtype != FADEMEM_F32 && dtype != FADEMEM_BF16) return FADEMEM_EINVAL;
  if (rows < 0 || rows > (int64_t(1) << 23) || heads < 1 || heads > 4096) return FADEMEM_EINVAL;
  const int elt = dtype == FADEMEM_BF16 ? 2 : 4;
  const int64_t row = int64_t(heads) * rope->head_dim;
  for (int64_t s : {x_stride, y_stride})
    if (s < row || s > (int64_t(1) << 32) || s * elt % 16) return FADEMEM_EINVAL;
  if (rows == 0) return FADEMEM_OK;
  if (!pos || reinterpret_cast<uintptr_t>(pos) % 4 || !x || !y || !aligned16(x) || !aligned16(y)) return FADEMEM_EINVAL;
  a.x = static_cast<const char*>(x);
  a.y = static_cast<char*>(y);
  a.x_pitch = size_t(x_stride) * elt;
  a.y_pitch = size_t(y_stride) * elt;
  const bool in_place = x == y && x_stride == y_stride;
  if (!in_place && !rows_apart(a.x, a.x_pitch, a.y, a.y_pitch, rows, size_t(row) * elt)) return FADEMEM_EINVAL;
  a.pos = pos;
  a.rows = rows;
  a.heads = heads;
  a.per_block = rows_per_block(rows, int(row * elt / 16), a.rot.pairs);
  const int64_t blocks = (rows + a.per_block - 1) / a.per_block;
  const bool bf16 = dtype == FADEMEM_BF16, halves = a.rot.halves != 0;
  auto kernel = bf16 ? (halves ? rope_kernel<true, true> : rope_kernel<true, false>)
                     : (halves ? rope_kernel<false, true> : rope_kernel<false, false>);
  (void)hipGetLastError();
  hipLaunchKernelGGL(kernel, dim3(unsigned(blocks)), dim3(kRotThreads), size_t(a.per_block) * a.rot.pairs * sizeof(double2),
                     reinterpret_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? FADEMEM_OK : FADEMEM_EHIP;
}

}  // extern "C"
