// Rotary positions with several axes: what the kernels that rotate share.
//
// Pair p of a head turns by pos[axis(p)] * freq[p]:
//   (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos),
// products and sums in fp64 and one rounding to the storage type, as the
// re-indexed views of the memory are made.  The gradient of the rotation is the
// rotation by the negative angle.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bf16_round.h"
#include "fademem.h"

namespace fademem {

constexpr int kRotThreads = 256;
constexpr int kRotMaxRows = 16;  // rows of a block at most

// Kernel argument: the rotation as the kernels use it.
struct RotaryArg {
  int head_dim;
  int pairs;       // pairs that turn, over all axes
  int end_t;       // pairs [0, end_t) follow axis 0, [end_t, end_h) axis 1, the rest axis 2
  int end_h;
  int halves;      // 0: pair p = elements (2p, 2p+1); 1: (p, p + head_dim/2)
  double sign;     // 1, or -1 for the inverse
  double freq[FADEMEM_ROPE_MAX_PAIRS];
};

typedef uint32_t rot_u32x4 __attribute__((ext_vector_type(4)));

// cos and sin of the pairs of rows [row0, row0 + n) into cs[(row, pair)], row
// by row; the angle in fp64 (positions far from zero), reduced there.
__device__ __forceinline__ void rotary_angles(const RotaryArg& r, const int32_t* pos, int64_t row0, int n,
                                              double2* cs) {
  for (int i = threadIdx.x; i < n * r.pairs; i += blockDim.x) {
    const int t = i / r.pairs, p = i - t * r.pairs;
    const int axis = (p >= r.end_t ? 1 : 0) + (p >= r.end_h ? 1 : 0);
    double s, c;
    sincos(double(pos[(row0 + t) * 3 + axis]) * r.freq[p], &s, &c);
    cs[i] = make_double2(c, r.sign * s);
  }
}

// Eight fp64 values rounded once to bf16.  Rounding by way of fp32 is off only
// where the fp32 value is a tie between two bf16 values and the fp64 one is not:
// those few go through round-to-odd, which costs three times as much (a chunk of
// 4680 rows of 12 x 128: 10.8 us with it everywhere, 9.5 so).
__device__ __forceinline__ void pack_unit(const double (&y)[8], rot_u32x4& out) {
  bool tie = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float lo = float(y[2 * w]), hi = float(y[2 * w + 1]);
    tie = tie || (__float_as_uint(lo) & 0xffffu) == 0x8000u || (__float_as_uint(hi) & 0xffffu) == 0x8000u;
    bf16x2_t v;
    v[0] = (__bf16)lo;
    v[1] = (__bf16)hi;
    out[w] = __builtin_bit_cast(uint32_t, v);
  }
  if (tie) {
#pragma unroll
    for (int w = 0; w < 4; ++w) out[w] = pack_bf16_rne(y[2 * w], y[2 * w + 1]);
  }
}

// The elements of a unit that turn, in place of those of `x`; the others keep their bits.
__device__ __forceinline__ rot_u32x4 keep_rest(rot_u32x4 turned, rot_u32x4 x, int elements) {
#pragma unroll
  for (int w = 0; w < 4; ++w)
    turned[w] = 2 * w + 1 < elements ? turned[w] : 2 * w < elements ? (turned[w] & 0xffffu) | (x[w] & 0xffff0000u) : x[w];
  return turned;
}

// One 16-byte unit of interleaved pairs: its first pair is pair k.
template <bool BF16>
__device__ __forceinline__ rot_u32x4 rotate_unit(rot_u32x4 x, const double2* cs, int k, int pairs) {
#pragma clang fp contract(off)
  if (k >= pairs) return x;
  if constexpr (BF16) {
    double y[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const double2 t = cs[min(k + w, pairs - 1)];
      const double a = bf16_lo(x[w]), b = bf16_hi(x[w]);
      y[2 * w] = a * t.x - b * t.y;
      y[2 * w + 1] = a * t.y + b * t.x;
    }
    rot_u32x4 r;
    pack_unit(y, r);
    return k + 4 <= pairs ? r : keep_rest(r, x, 2 * (pairs - k));
  } else {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (k + w < pairs) {
        const double2 t = cs[k + w];
        const double a = double(__uint_as_float(x[2 * w])), b = double(__uint_as_float(x[2 * w + 1]));
        x[2 * w] = __float_as_uint(float(a * t.x - b * t.y));
        x[2 * w + 1] = __float_as_uint(float(a * t.y + b * t.x));
      }
    }
    return x;
  }
}

// Two 16-byte units of half-split pairs: a holds the first elements of pairs
// k, k+1, ..., b their second ones.
template <bool BF16>
__device__ __forceinline__ void rotate_halves(rot_u32x4& a, rot_u32x4& b, const double2* cs, int k, int pairs) {
#pragma clang fp contract(off)
  if (k >= pairs) return;
  if constexpr (BF16) {
    double p[8], q[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const double2 t = cs[min(k + 2 * w, pairs - 1)], u = cs[min(k + 2 * w + 1, pairs - 1)];
      const double x0 = bf16_lo(a[w]), x1 = bf16_hi(a[w]), y0 = bf16_lo(b[w]), y1 = bf16_hi(b[w]);
      p[2 * w] = x0 * t.x - y0 * t.y;
      p[2 * w + 1] = x1 * u.x - y1 * u.y;
      q[2 * w] = x0 * t.y + y0 * t.x;
      q[2 * w + 1] = x1 * u.y + y1 * u.x;
    }
    rot_u32x4 r, s;
    pack_unit(p, r);
    pack_unit(q, s);
    a = k + 8 <= pairs ? r : keep_rest(r, a, pairs - k);
    b = k + 8 <= pairs ? s : keep_rest(s, b, pairs - k);
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (k + w < pairs) {
        const double2 t = cs[k + w];
        const double x = double(__uint_as_float(a[w])), y = double(__uint_as_float(b[w]));
        a[w] = __float_as_uint(float(x * t.x - y * t.y));
        b[w] = __float_as_uint(float(x * t.y + y * t.x));
      }
    }
  }
}

// Rows of a block: about four 16-byte units per thread, no more than still leave
// two blocks per CU, and whole rounds of the block's threads over their angles.
inline int rows_per_block(int64_t rows, int units_per_row, int pairs) {
  int64_t per = 4 * kRotThreads / units_per_row;
  if (per > (rows + 511) / 512) per = (rows + 511) / 512;
  const int round = pairs > 0 ? kRotThreads / pairs : 1;
  if (round > 1 && per > round) per = per / round * round;
  return int(per < 1 ? 1 : per > kRotMaxRows ? kRotMaxRows : per);
}

// Checks a rotation and turns it into the kernels' argument.
int rotary_arg(const fademem_rope* r, int inverse, RotaryArg* out);

// Rows of x and of y, `row` bytes each, their pitches apart, share no byte.
bool rows_apart(const char* x, size_t x_pitch, const char* y, size_t y_pitch, int64_t rows, size_t row);

}  // namespace fademem
