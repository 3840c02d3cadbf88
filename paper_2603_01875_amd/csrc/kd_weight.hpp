// The weights that sampling adds up: w = exp((z - largest) / temperature) in 64 bits.  Plain arithmetic, compiled for the host as well.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace kd {

// ------------------------------------------------------------------------------------------------
// w = 2^t in 64 bits, t <= 2^-45
//
// t = n + x with a whole number n and |x| <= 1/2; 2^x is the polynomial of degree 8 that meets it at the Chebyshev nodes of [-1/2, 1/2] (1 at 0; off by
// 2^-39.7 at most), 2^n is added to its exponent.  n comes out of the low bits of t + 1.5 2^52: no conversion, no table.  13 instructions in 64 bits; an exp
// in 32 bits would be off by 2^-24 in every sum that a uniform number is compared with: one token in some thousand would be another one.
// ------------------------------------------------------------------------------------------------
constexpr double kLog2e = 1.44269504088896340736;
constexpr int kChunkBits = 48;         // a chunk's sums: 2^14 entries of at most 2^48 (0x1p48 below)

typedef uint32_t halves_t __attribute__((vector_size(8)));      // of a double, the low one first
__host__ __device__ inline __attribute__((always_inline)) uint64_t double_bits(double x) { return __builtin_bit_cast(uint64_t, x); }

__host__ __device__ inline __attribute__((always_inline)) double weight(double t) {
  t = fmax(t, -80.);                                   // (2^-80 and less count as nothing; also for a NaN, where a chunk is empty)
  const double m = t + 0x1.8p52, x = t - (m - 0x1.8p52);
  double p = 0x1.63d1363930791p-20;
  p = fma(p, x, 0x1.00dc4a53395d3p-16);
  p = fma(p, x, 0x1.4308ac85a7718p-13);
  p = fma(p, x, 0x1.5d8745a72831bp-10);
  p = fma(p, x, 0x1.3b2ab7181b778p-7);
  p = fma(p, x, 0x1.c6b08dd6fd236p-5);
  p = fma(p, x, 0x1.ebfbdff823cedp-3);
  p = fma(p, x, 0x1.62e42fef84cf0p-1);
  p = fma(p, x, 1.);
  halves_t bits = __builtin_bit_cast(halves_t, p);
  bits[1] += __builtin_bit_cast(halves_t, m)[0] << 20;
  return __builtin_bit_cast(double, bits);
}
// A weight (or a sum of some) as a whole number of 2^-bits.
__host__ __device__ inline __attribute__((always_inline)) uint64_t whole(double w, int bits) { return (uint64_t)rint(ldexp(w, bits)); }
// The same of a single one (less than 2^52 of them, so that they are the low bits of what 2^52 is added to); scale = 2^bits.
__host__ __device__ inline __attribute__((always_inline)) uint64_t whole_one(double w, double scale) {
  return double_bits(fma(w, scale, 0x1p52)) - double_bits(0x1p52);
}

// Exponents of a chunk's weights: (z - top) scale, one multiply-add each.  Where |top scale| is below 256, as z scale - zero with zero = top scale, rounded by 2^-46 at
// most: nothing beside the polynomial's error.  Where it is more, zero's rounding would be more than that (at 1e16 more than 1: no weight at all), and z - top is taken
// first, in 32 bits: exact for every z whose weight counts, because (top - z) scale < 80 makes top - z less than a third of |top|, and a
// difference of numbers within a factor of two of each other is not rounded.  (Always z - top in 64 bits: one more of 21 instructions for each entry.)
struct Exponents { float base; double scale, zero; };
__host__ __device__ inline __attribute__((always_inline)) Exponents exponents_of(float top, double scale) {
  const double zero = (double)top * scale;
  const bool far = fabs(zero) >= 256.;
  return Exponents{far ? top : 0.f, scale, far ? 0. : zero};
}
__host__ __device__ inline __attribute__((always_inline)) double exponent(const Exponents& e, float z) { return fma((double)(z - e.base), e.scale, -e.zero); }
// The factor from weights relative to `from`, a chunk's largest entry, to those relative to `to`.
__host__ __device__ inline __attribute__((always_inline)) double rescale(double from, double to, double scale) { return exp2((from - to) * scale); }

}  // namespace kd
