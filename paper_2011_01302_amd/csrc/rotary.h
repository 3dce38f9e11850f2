// The rotation of a head's pairs of values by their token's position.
#pragma once

#include "decoder.h"

namespace ios {

// Cosine and sine of a position's angle, times the amplitude, rounded once from 64 bits: the angle less a multiple of
// pi / 2 (which two numbers hold to 107 bits), then the series of both up to x^13 and x^14, off by at most 2e-14 up to
// pi / 4.  So they round to what the definition says but for a few in 10^6, also at positions where 32 bits have lost
// the angle.  About 30 operations in 64 bits, as fast here as single ones in 32.
__device__ __forceinline__ float2 turn_of(int pos, double freq, double amplitude) {
  const double angle = (double)pos * freq, n = __builtin_rint(angle * 0.63661977236758134308);
  const double x = fma(-n, 6.12323399573676603587e-17, fma(-n, 1.57079632679489655800, angle)), y = x * x;
  double s = fma(y, 1.0 / 6227020800.0, -1.0 / 39916800.0);
  s = fma(s, y, 1.0 / 362880.0);
  s = fma(s, y, -1.0 / 5040.0);
  s = fma(s, y, 1.0 / 120.0);
  s = fma(s, y, -1.0 / 6.0);
  s = fma(s * y, x, x);
  double c = fma(y, -1.0 / 87178291200.0, 1.0 / 479001600.0);
  c = fma(c, y, -1.0 / 3628800.0);
  c = fma(c, y, 1.0 / 40320.0);
  c = fma(c, y, -1.0 / 720.0);
  c = fma(c, y, 1.0 / 24.0);
  c = fma(c, y, -0.5);
  c = fma(c, y, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return float2{(float)(amplitude * (quarter == 1 || quarter == 2 ? -a : a)), (float)(amplitude * (quarter >= 2 ? -b : b))};
}

// A pair turned: each product and their sum rounded by itself (no fused operation), so that the values are defined to
// the bit.
__device__ __forceinline__ void turn(float &a, float &b, float2 cs) {
#pragma clang fp contract(off)
  const float ac = a * cs.x, bs = b * cs.y, as = a * cs.y, bc = b * cs.x;
  a = ac - bs;
  b = as + bc;
}

// Values of a head are turned in units that no two threads share, so that a tensor can be turned in place: 8 values of
// each half, 8 values of neighbours, 8 values that stay, or, where a half is not a multiple of 8, single pairs and values.
struct RotaryUnits {
  int dim, half;                          // of a head, of its rotated part
  bool interleaved, single;
  int turned, all;                        // units of a head that are turned, and in all
  __host__ __device__ RotaryUnits(const ios_rotary &r, int head_dim)
      : dim(head_dim), half(r.dim / 2), interleaved(r.interleaved != 0), single(!interleaved && half % 8 != 0) {
    turned = single ? half : interleaved ? (2 * half + 7) / 8 : half / 8;
    all = turned + (single ? head_dim - 2 * half : interleaved ? head_dim / 8 - turned : (head_dim - 2 * half) / 8);
  }
};

template <class T>
struct alignas(16) Octet8 {
  T v[8];
};

// What a thread holds of one unit between its loads and its stores.
template <class T>
struct RotaryUnit {
  Octet8<T> a, b;
  __device__ __forceinline__ void load(const RotaryUnits &u, const T *row, int at) {
    if (u.single) {
      a.v[0] = row[at < u.half ? at : at + u.half];
      if (at < u.half) b.v[0] = row[at + u.half];
    } else {
      a = *(const Octet8<T> *)(row + 8 * (u.interleaved || at < u.turned ? at : at + u.turned));
      if (!u.interleaved && at < u.turned) b = *(const Octet8<T> *)(row + 8 * at + u.half);
    }
  }
  __device__ __forceinline__ void turn_by(const RotaryUnits &u, const float2 *cs, int at) {
    if (at >= u.turned) return;
    auto pair = [&](T &x, T &y, float2 c) {
      float f = (float)x, g = (float)y;
      turn(f, g, c);
      x = (T)f;
      y = (T)g;
    };
    if (u.single) {
      pair(a.v[0], b.v[0], cs[at]);
    } else if (u.interleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * at + e < u.half) pair(a.v[2 * e], a.v[2 * e + 1], cs[4 * at + e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) pair(a.v[e], b.v[e], cs[8 * at + e]);
    }
  }
  __device__ __forceinline__ void store(const RotaryUnits &u, T *row, int at) const {
    if (u.single) {
      row[at < u.half ? at : at + u.half] = a.v[0];
      if (at < u.half) row[at + u.half] = b.v[0];
    } else {
      *(Octet8<T> *)(row + 8 * (u.interleaved || at < u.turned ? at : at + u.turned)) = a;
      if (!u.interleaved && at < u.turned) *(Octet8<T> *)(row + 8 * at + u.half) = b;
    }
  }
};

}  // namespace ios
