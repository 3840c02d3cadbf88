// Rows of logits: the top logits of each (kd_top_logits), one token sampled from each (kd_sample).
//
// Both read the logits once.  A first kernel, a workgroup to a piece of a row (a chunk), leaves the chunk's sum of w = exp((z - largest of
// the chunk) / tau) and, per thread, the largest entry of its share (a group).  A second, a workgroup to a row, works on these: the
// G-th largest of the groups' largest entries is a bound that at least G entries reach, and only groups that reach it hold entries
// that do, so that a few hundred groups are read again, and a short list is sorted.  Sampling from all of a row needs the sums alone: the
// chunk in which the sum of w passes u times the whole is read again.  A list that does not fit, or does not reach far enough (thousands of
// equal entries, a flat distribution under top-p), sends its row down the slow way: passes over the row that narrow the last kept
// entry down by eight bits of its key at a time.
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_launch.h"
#include "kd_unaligned.hpp"

namespace kd {

constexpr uint32_t kKeyMinusInf = 0x007fffffu, kKeyInf = 0xff800000u, kKeyNaN = 0xffffffffu;

// Order of keys = order of values, -0 = +0, NaN above all.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  const uint32_t k = u & 0x80000000u ? ~u : u | 0x80000000u;
  return z == 0.f ? 0x80000000u : z != z ? kKeyNaN : k;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <bool F32>
__device__ __forceinline__ float logit(const void* row, int64_t i) {
  return F32 ? ((const float*)row)[i] : bf16_float(((const uint16_t*)row)[i]);
}
template <bool F32>
__device__ __forceinline__ const void* row_of(const RowsArgs& a, int64_t t) {
  return (const char*)a.logits + t * a.ld * (F32 ? 4 : 2);
}

// ------------------------------------------------------------------------------------------------
// w = 2^(t / 32) in 64 bits, as a whole number of 2^-bits
//
// t / 32 = n / 32 + r with a whole number n and |r| <= 1/64: 2^(n / 32) is one of 32 table entries (256 bytes of LDS: every bank once, any 64 lanes read
// them without a conflict) and a shift, 2^r four terms of its series, off by (ln 2 / 64)^5 / 120 = 2^-39.6 at most.  Adding 2^52 leaves the rounded whole
// number in the low bits.  (An exp in 32 bits would be off by 2^-24 in every sum that a uniform number is compared with: one token in some
// thousand would be another one.)
// ------------------------------------------------------------------------------------------------
constexpr double kLn2 = 0.693147180559945309417, kLog2e = 1.44269504088896340736;
constexpr double kC1 = kLn2 / 32, kC2 = kC1 * kC1 / 2, kC3 = kC2 * kC1 / 3, kC4 = kC3 * kC1 / 4;
constexpr int kChunkBits = 48;         // a chunk's sums: 2^14 entries of at most 2^48

__device__ __forceinline__ void fill_table(double* tab) {
  if (threadIdx.x < 32) tab[threadIdx.x] = exp2((double)threadIdx.x / 32);
  __syncthreads();
}
__device__ __forceinline__ uint64_t weight(double t, const double* tab, int bits) {
  t = fmax(t, -2560.);                                 // 2^-80 and less: 0 (also for a NaN, where a chunk is empty)
  const double n = rint(t), r = t - n;
  const int k = (int)n;
  double p = fma(r, kC4, kC3);
  p = fma(r, p, kC2);
  p = fma(r, p, kC1);
  p = fma(r, p, 1.);
  const double v = ldexp(p * tab[k & 31], (k >> 5) + bits);
  return __double_as_longlong(v + 0x1p52) - 0x4330000000000000ll;
}

// ------------------------------------------------------------------------------------------------
// first kernel
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ float row_temperature(const RowsArgs& a, int64_t t) { return a.temperature_rows ? a.temperature_rows[t] : a.tau; }

template <bool F32, int E, bool SAMPLE>
__global__ __launch_bounds__(kRowThreads) void rows_scan_kernel(const RowsArgs a) {
  constexpr int VE = F32 ? 4 : 8, J = E / VE, NT = kRowThreads, NW = NT / 64;
  static_assert(E % VE == 0, "whole loads");
  __shared__ double tab[32];
  __shared__ uint32_t keys[NW];
  __shared__ uint64_t sums[NW];
  const int64_t piece = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, t = piece / a.chunks;
  if (t >= a.T) return;                // (the last row of a large grid)
  const int c = (int)(piece - t * a.chunks), tid = threadIdx.x;
  const void* const row = row_of<F32>(a, t);
  const int64_t at = (int64_t)c * (NT * E) + tid * VE;
  float z[E];
  if ((int64_t)(c + 1) * (NT * E) <= a.V) {
    u32x4_t v[J];
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = load16((const char*)row + (at + j * (NT * VE)) * (F32 ? 4 : 2));
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (F32) z[j * VE + i] = __uint_as_float(v[j][i]);
        else {
          z[j * VE + (2 * i) % VE] = __uint_as_float(v[j][i] << 16);
          z[j * VE + (2 * i + 1) % VE] = __uint_as_float(v[j][i] & 0xffff0000u);
        }
      }
  } else {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int64_t k = at + j * (NT * VE) + i;
        z[j * VE + i] = k < a.V ? logit<F32>(row, k) : -__builtin_inff();
      }
  }
  float m = z[0];
  bool nan = m != m;
#pragma unroll
  for (int i = 1; i < E; ++i) {
    nan |= z[i] != z[i];
    m = fmaxf(m, z[i]);
  }
  uint32_t key = nan ? kKeyNaN : key_of(m);
  a.group[t * ((int64_t)a.chunks * NT) + c * NT + tid] = key;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
  if ((tid & 63) == 0) keys[tid >> 6] = key;
  if (SAMPLE) fill_table(tab);         // (and the barrier)
  else __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) key = max(key, keys[w]);
  const float top = value_of(key);
  RowChunk out{0, 0.f, key};
  if (SAMPLE) {
    const float tau = row_temperature(a, t);
    uint64_t s = 0;
    if (tau > 0.f) {
      const double scale = 32 * kLog2e / (double)tau, zero = (double)top;
#pragma unroll
      for (int i = 0; i < E; ++i) s += weight(((double)z[i] - zero) * scale, tab, kChunkBits);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor((unsigned long long)s, o, 64);
    if ((tid & 63) == 0) sums[tid >> 6] = s;
    __syncthreads();
    out.sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) out.sum += sums[w];
  } else {
    const float scale = (float)(kLog2e / (double)a.tau);
    float s = 0.f;
    if (key > kKeyMinusInf)
#pragma unroll
      for (int i = 0; i < E; ++i) s += __builtin_amdgcn_exp2f((z[i] - top) * scale);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
    if ((tid & 63) == 0) sums[tid >> 6] = __float_as_uint(s);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) out.part += __uint_as_float((uint32_t)sums[w]);
  }
  if (tid == 0) a.chunk[t * a.chunks + c] = out;
}

// ------------------------------------------------------------------------------------------------
// second kernel: pieces
// ------------------------------------------------------------------------------------------------
constexpr int kSelect = 512;           // threads
constexpr int kList = 8192;            // entries of the list at most
constexpr int kTile = kSelect * 8;     // entries that a pass of the slow way takes at a time
constexpr int kSlots = 4096;           // tiles of a row at most
// Sampling: groups that the list takes, for a top-k of at most kReach as many, else (top-p and min-p, mostly) kReachAll.
constexpr int kReach = 1024, kReachAll = 512;

struct SelectLds {
  union {
    uint64_t list[kList];              // key, complement of the index: descending order is the order of the entries
    uint64_t mass[kSlots];             // chunks' or tiles' sums
  };
  uint64_t scan[kSelect / 64 + 1];
  uint64_t bin_mass[256];
  uint32_t bin[256];
  uint32_t count;
  uint64_t value[2];
  double tab[32];
};

// Exclusive prefix sum over the workgroup; total to all.
__device__ __forceinline__ uint64_t prefix(uint64_t v, uint64_t& total, SelectLds& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();                     // (what an earlier call left has been read)
  if (lane == 63) s.scan[wave] = x;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) {
    if (w < wave) before += s.scan[w];
    all += s.scan[w];
  }
  total = all;
  return before + x - v;
}

// The 16 high bits of the G-th largest of n keys (at least G keys reach them).
__device__ __forceinline__ uint32_t bound_of(const uint32_t* group, int64_t n, uint32_t G, SelectLds& s) {
  uint32_t high = 0;
#pragma unroll 1
  for (int level = 0; level < 2; ++level) {
    const int shift = 24 - 8 * level;
    for (int i = threadIdx.x; i < 256; i += kSelect) s.bin[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < n; i += kSelect) {
      const uint32_t k = group[i];
      if (level == 0 || k >> 24 == high >> 24) atomicAdd(&s.bin[k >> shift & 255], 1u);
    }
    __syncthreads();
    // bins from the largest down: thread i < 256 has bin 255 - i
    const uint32_t mine = threadIdx.x < 256 ? s.bin[255 - threadIdx.x] : 0;
    uint64_t all;
    const uint64_t before = prefix(mine, all, s);
    if (threadIdx.x < 256 && before < G && before + mine >= G) {
      s.value[0] = 255 - threadIdx.x;
      s.value[1] = before;
    }
    __syncthreads();
    high |= (uint32_t)s.value[0] << shift;
    G -= (uint32_t)s.value[1];
  }
  return high;
}

// Entries of the row that reach `bound` into the list; their number, which may be more than fit.
template <bool F32>
__device__ __forceinline__ uint32_t gather(const RowsArgs& a, int64_t t, uint32_t bound, SelectLds& s) {
  constexpr int VE = F32 ? 4 : 8;
  const void* const row = row_of<F32>(a, t);
  const int64_t n = (int64_t)a.chunks * kRowThreads;
  const uint32_t* const group = a.group + t * n;
  const int J = a.per_thread / VE;
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  for (int64_t g = threadIdx.x; g < n; g += kSelect) {
    if (group[g] < bound) continue;
    const int64_t at = g / kRowThreads * ((int64_t)kRowThreads * a.per_thread) + g % kRowThreads * VE;
    for (int j = 0; j < J; ++j)
      for (int i = 0; i < VE; ++i) {
        const int64_t k = at + (int64_t)j * (kRowThreads * VE) + i;
        if (k >= a.V) break;
        const uint32_t key = key_of(logit<F32>(row, k));
        if (key < bound) continue;
        const uint32_t to = atomicAdd(&s.count, 1u);
        if (to < (uint32_t)kList) s.list[to] = (uint64_t)key << 32 | (uint32_t)~(uint32_t)k;
      }
  }
  __syncthreads();
  return s.count;
}

// Sorts list[0 .. n) in descending order (n at most kList; filled up to a power of two with 0).
__device__ __forceinline__ void sort_list(uint32_t n, SelectLds& s) {
  uint32_t size = 2;
  while (size < n) size <<= 1;
  for (uint32_t i = n + threadIdx.x; i < size; i += kSelect) s.list[i] = 0;
  __syncthreads();
  for (uint32_t k = 2; k <= size; k <<= 1)
    for (uint32_t j = k >> 1; j; j >>= 1) {
      for (uint32_t i = threadIdx.x; i < size / 2; i += kSelect) {
        const uint32_t lo = 2 * i - (i & (j - 1)), hi = lo + j;
        const uint64_t x = s.list[lo], y = s.list[hi];
        if ((x < y) == ((lo & k) == 0)) {
          s.list[lo] = y;
          s.list[hi] = x;
        }
      }
      __syncthreads();
    }
}

// ---- the slow way: the last kept entry, as its key and the last index that counts among entries of that key ----
struct Cut { uint32_t key; int64_t last; };

__device__ __forceinline__ bool inside(const Cut& c, uint32_t key, int64_t i) { return key > c.key || (key == c.key && i <= c.last); }

// Index of the e-th entry (from 1) of this key.
template <bool F32>
__device__ __forceinline__ int64_t place_of(const void* row, int64_t V, uint32_t key, uint64_t e, SelectLds& s) {
  for (int64_t base = 0;; base += kTile) {
    const int64_t at = base + threadIdx.x * 8;
    uint32_t hits = 0;
    for (int i = 0; i < 8; ++i)
      if (at + i < V && key_of(logit<F32>(row, at + i)) == key) hits |= 1u << i;
    uint64_t all;
    const uint64_t before = prefix(__popc(hits), all, s);
    if (e <= all || base + kTile >= V) {
      if (threadIdx.x == 0) s.value[0] = V - 1;
      __syncthreads();
      if (before < e && e <= before + __popc(hits)) {
        uint64_t left = e - before;
        for (int i = 0; i < 8; ++i)
          if (hits >> i & 1 && --left == 0) s.value[0] = at + i;
      }
      __syncthreads();
      const int64_t found = s.value[0];
      __syncthreads();
      return found;
    }
    e -= all;
  }
}

// The last entry of the fewest, in descending order, whose number (MASS: sum of w) is at least `want` (which the whole row reaches).
template <bool F32, bool MASS>
__device__ __forceinline__ Cut narrow(const void* row, int64_t V, uint64_t want, double zero, double scale, int bits, SelectLds& s) {
  uint32_t high = 0;
#pragma unroll 1
  for (int level = 0; level < 4; ++level) {
    const int shift = 24 - 8 * level;
    for (int i = threadIdx.x; i < 256; i += kSelect) s.bin_mass[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < V; i += kSelect) {
      const float z = logit<F32>(row, i);
      const uint32_t k = key_of(z);
      if (level && (k ^ high) >> (shift + 8)) continue;
      atomicAdd((unsigned long long*)&s.bin_mass[k >> shift & 255],
                (unsigned long long)(MASS ? weight(((double)z - zero) * scale, s.tab, bits) : 1));
    }
    __syncthreads();
    const uint64_t mine = threadIdx.x < 256 ? s.bin_mass[255 - threadIdx.x] : 0;
    uint64_t all;
    const uint64_t before = prefix(mine, all, s);
    if (threadIdx.x < 256 && before < want && before + mine >= want) {
      s.value[0] = 255 - threadIdx.x;
      s.value[1] = before;
    }
    __syncthreads();
    high |= (uint32_t)s.value[0] << shift;
    want -= s.value[1];
    __syncthreads();
  }
  uint64_t e = want;
  if (MASS) {
    const uint64_t w = weight(((double)value_of(high) - zero) * scale, s.tab, bits);
    e = (want + w - 1) / w;
  }
  return Cut{high, place_of<F32>(row, V, high, e, s)};
}

// ------------------------------------------------------------------------------------------------
// top logits
// ------------------------------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ void put_top(const RowsArgs& a, int64_t t, int at, uint32_t key, int64_t index) {
  const bool there = key > kKeyMinusInf;
  const int64_t to = t * a.K + at;
  const float z = there ? (F32 ? ((const float*)row_of<true>(a, t))[index] : 0.f) : -__builtin_inff();
  if (F32) ((float*)a.top)[to] = z;
  else ((uint16_t*)a.top)[to] = there ? ((const uint16_t*)row_of<false>(a, t))[index] : (uint16_t)0xff80;
  if (a.index64) ((int64_t*)a.index)[to] = there ? index : -1;
  else ((int32_t*)a.index)[to] = there ? (int32_t)index : -1;
}

template <bool F32>
__global__ __launch_bounds__(kSelect) void top_select_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const int64_t n = (int64_t)a.chunks * kRowThreads;
  const void* const row = row_of<F32>(a, t);
  if (a.lse) {
    // the chunks' sums at the row's largest entry, in a fixed order
    uint32_t key = 0;
    for (int c = tid; c < a.chunks; c += kSelect) key = max(key, a.chunk[t * a.chunks + c].key);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
    if ((tid & 63) == 0) s.bin[tid >> 6] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelect / 64; ++w) key = max(key, s.bin[w]);
    __syncthreads();
    const double top = value_of(key);
    double sum = 0;
    for (int c = tid; c < a.chunks; c += kSelect) {
      const RowChunk& r = a.chunk[t * a.chunks + c];
      if (r.key > kKeyMinusInf) sum += (double)r.part * exp(((double)value_of(r.key) - top) / (double)a.tau);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) s.tab[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
      sum = 0;
      for (int w = 0; w < kSelect / 64; ++w) sum += s.tab[w];
      a.lse[t] = key == kKeyNaN ? __builtin_nanf("") : key == kKeyInf ? __builtin_inff() : key <= kKeyMinusInf ? -__builtin_inff()
                 : (float)(top / (double)a.tau + log(sum));
    }
  }
  // (entries of minus infinity are no entries: the lowest bound is above them)
  uint32_t bound = kKeyMinusInf + 1;
  if ((int64_t)a.K < n) bound = max(bound, bound_of(a.group + t * n, n, (uint32_t)a.K, s));
  const uint32_t found = gather<F32>(a, t, bound, s);
  if (found <= (uint32_t)kList) {
    sort_list(found, s);
    for (int i = tid; i < a.K; i += kSelect) {
      const uint64_t x = i < (int)found ? s.list[i] : 0;
      put_top<F32>(a, t, i, (uint32_t)(x >> 32), (int64_t)(uint32_t)~(uint32_t)x);
    }
    return;
  }
  const Cut cut = narrow<F32, false>(row, a.V, (uint64_t)a.K, 0, 0, 0, s);
  if (tid == 0) s.count = 0;
  __syncthreads();
  for (int64_t i = tid; i < a.V; i += kSelect) {
    const uint32_t key = key_of(logit<F32>(row, i));
    if (key <= kKeyMinusInf || !inside(cut, key, i)) continue;
    s.list[atomicAdd(&s.count, 1u)] = (uint64_t)key << 32 | (uint32_t)~(uint32_t)i;
  }
  __syncthreads();
  const uint32_t kept = s.count;
  sort_list(kept, s);
  for (int i = tid; i < a.K; i += kSelect) {
    const uint64_t x = i < (int)kept ? s.list[i] : 0;
    put_top<F32>(a, t, i, (uint32_t)(x >> 32), (int64_t)(uint32_t)~(uint32_t)x);
  }
}

// ------------------------------------------------------------------------------------------------
// sampling
// ------------------------------------------------------------------------------------------------
// The largest whole number that is not above u total.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const uint64_t x = (uint64_t)((double)u * (double)total);
  return x < total ? x : total - 1;
}

template <bool F32>
__global__ __launch_bounds__(kSelect) void sample_select_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const int64_t t = blockIdx.x, n = (int64_t)a.chunks * kRowThreads, V = a.V;
  const int tid = threadIdx.x;
  const void* const row = row_of<F32>(a, t);
  const float u = a.u[t], tau = row_temperature(a, t);
  const float top_p = a.top_p_rows ? a.top_p_rows[t] : a.top_p, min_p = a.min_p_rows ? a.min_p_rows[t] : a.min_p;
  const int64_t top_k = a.top_k_rows ? a.top_k_rows[t] : a.top_k;
  const bool greedy = tau == 0.f, all_k = !greedy && (top_k == 0 || top_k >= V);
  fill_table(s.tab);
  // the row's largest entry
  uint32_t key = 0;
  for (int c = tid; c < a.chunks; c += kSelect) key = max(key, a.chunk[t * a.chunks + c].key);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
  if ((tid & 63) == 0) s.bin[tid >> 6] = key;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) key = max(key, s.bin[w]);
  __syncthreads();
  auto answer = [&](int64_t token, float logp) {
    if (a.index64) ((int64_t*)a.token)[t] = token;
    else ((int32_t*)a.token)[t] = (int32_t)token;
    if (a.logp) a.logp[t] = logp;
  };
  const bool valid = u >= 0.f && u < 1.f && (tau == 0.f || (tau >= 1e-6f && tau <= 1e6f)) && top_k >= 0 && top_p > 0.f && top_p <= 1.f &&
                     min_p >= 0.f && min_p <= 1.f && key > kKeyMinusInf && key < kKeyInf;
  if (!valid) {
    if (tid == 0) answer(-1, __builtin_nanf(""));
    return;
  }
  const double top = value_of(key), scale = 32 * kLog2e / (greedy ? 1. : (double)tau);
  const int row_bits = min(kChunkBits, 62 - (64 - __clzll((unsigned long long)V)));      // V entries of at most 2^row_bits
  auto log_p = [&](int64_t token, uint64_t total, int bits) {
    return greedy ? 0.f : (float)(((double)logit<F32>(row, token) - top) / (double)tau - log(ldexp((double)total, -bits)));
  };

  uint64_t row_total = 0;
  if (all_k) {
    // chunks' sums at the row's largest entry
    uint64_t part = 0;
    const int per = (a.chunks + kSelect - 1) / kSelect, c0 = tid * per;
    auto chunk_mass = [&](int c) {
      const RowChunk& r = a.chunk[t * a.chunks + c];
      if (r.key <= kKeyMinusInf) return (uint64_t)0;
      return (uint64_t)rint(ldexp((double)r.sum, row_bits - kChunkBits) * exp2(((double)value_of(r.key) - top) * (scale / 32)));
    };
    for (int c = c0; c < c0 + per && c < a.chunks; ++c) part += chunk_mass(c);
    const uint64_t before = prefix(part, row_total, s);
    if (top_p == 1.f && min_p == 0.f) {
      const uint64_t target = target_of(u, row_total);
      if (before <= target && target < before + part) {
        uint64_t x = before;
        for (int c = c0; c < c0 + per && c < a.chunks; ++c) {
          const uint64_t m = chunk_mass(c);
          if (target < x + m) {
            s.value[0] = c;
            s.value[1] = target - x;
            break;
          }
          x += m;
        }
      }
      __syncthreads();
      const int c = (int)s.value[0];
      const RowChunk r = a.chunk[t * a.chunks + c];
      // that chunk again, with its own sums
      const double zero = value_of(r.key);
      const double inner = ldexp((double)s.value[1], kChunkBits - row_bits) * exp2((top - zero) * (scale / 32));
      const uint64_t want = inner < (double)r.sum ? (uint64_t)inner : r.sum - 1;
      const int64_t begin = (int64_t)c * kRowThreads * a.per_thread, end = min(V, begin + (int64_t)kRowThreads * a.per_thread);
      const int each = (int)((end - begin + kSelect - 1) / kSelect);
      const int64_t i0 = begin + (int64_t)tid * each;
      uint64_t mine = 0;
      for (int i = 0; i < each; ++i)
        if (i0 + i < end) mine += weight(((double)logit<F32>(row, i0 + i) - zero) * scale, s.tab, kChunkBits);
      uint64_t all;
      const uint64_t ahead = prefix(mine, all, s);
      if (ahead <= want && want < ahead + mine) {
        uint64_t x = ahead;
        for (int i = 0; i < each; ++i) {
          x += weight(((double)logit<F32>(row, i0 + i) - zero) * scale, s.tab, kChunkBits);
          if (x > want) {
            answer(i0 + i, log_p(i0 + i, row_total, row_bits));
            break;
          }
        }
      }
      return;
    }
  }

  // a short list of the largest entries
  const int64_t k = greedy ? 1 : all_k ? V : top_k;
  const uint32_t reach = (uint32_t)(k <= kReach ? k : kReachAll);
  uint32_t bound = kKeyMinusInf + 1;
  if ((int64_t)reach < n) bound = max(bound, bound_of(a.group + t * n, n, reach, s));
  const bool whole = bound == kKeyMinusInf + 1;
  const uint32_t found = gather<F32>(a, t, bound, s);
  if (found <= (uint32_t)kList) {
    sort_list(found, s);
    if (greedy) {
      if (tid == 0) answer((int64_t)(uint32_t)~(uint32_t)s.list[0], 0.f);
      return;
    }
    const uint32_t limit = k < (int64_t)found ? (uint32_t)k : found;
    // thread i has entries i per .. + per - 1 of the list
    const uint32_t per = (found + kSelect - 1) / kSelect, i0 = tid * per;
    const double floor_w = ldexp((double)min_p, kChunkBits);
    auto w_at = [&](uint32_t i) { return weight(((double)value_of((uint32_t)(s.list[i] >> 32)) - top) * scale, s.tab, kChunkBits); };
    uint64_t part = 0;
    for (uint32_t i = i0; i < i0 + per && i < limit; ++i) part += w_at(i);
    uint64_t listed;
    uint64_t x = prefix(part, listed, s);
    const bool reaches_k = whole || k <= (int64_t)found;
    // sum over the first top_k
    const double base = all_k ? ldexp((double)row_total, kChunkBits - row_bits) : (double)listed;
    const bool p_known = top_p == 1.f || all_k || reaches_k;
    const double nucleus = top_p == 1.f ? __builtin_inf() : (double)top_p * base;
    // an entry is kept if what is in front of it is less than the nucleus and its own w is not too small
    uint32_t kept = 0;
    for (uint32_t i = i0; i < i0 + per && i < limit; ++i) {
      const uint64_t w = w_at(i);
      if ((double)x < nucleus && (double)w >= floor_w) ++kept;
      x += w;
    }
    uint64_t n_kept;
    prefix(kept, n_kept, s);
    // the list says it all if it is the whole row, or holds the first top_k, or an entry of it that is not kept
    if (p_known && (reaches_k || n_kept < found)) {
      // kept entries in order of their index
      for (uint32_t i = tid; i < n_kept; i += kSelect) {
        const uint64_t e = s.list[i];
        s.list[i] = (e & 0xffffffffu) << 32 | e >> 32;           // (complement of the index: descending is reversed below)
      }
      __syncthreads();
      sort_list((uint32_t)n_kept, s);
      const uint32_t m = (uint32_t)n_kept, each = (m + kSelect - 1) / kSelect, j0 = tid * each;
      auto w_of = [&](uint32_t j) { return weight(((double)value_of((uint32_t)s.list[j]) - top) * scale, s.tab, kChunkBits); };
      uint64_t mine = 0, total;
      for (uint32_t j = j0; j < j0 + each && j < m; ++j) mine += w_of(j);
      uint64_t y = prefix(mine, total, s);
      const uint64_t target = target_of(u, total);
      if (y <= target && target < y + mine)
        for (uint32_t j = j0; j < j0 + each && j < m; ++j) {
          y += w_of(j);
          if (y > target) {
            const int64_t token = (int64_t)(uint32_t)~(uint32_t)(s.list[j] >> 32);
            answer(token, log_p(token, total, kChunkBits));
            break;
          }
        }
      return;
    }
  }

  // the slow way
  Cut cut{0, V};
  if (k < V) cut = narrow<F32, false>(row, V, (uint64_t)k, 0, 0, 0, s);
  if (top_p < 1.f) {
    uint64_t mine = 0, total;
    for (int64_t i = tid; i < V; i += kSelect) {
      const float z = logit<F32>(row, i);
      if (inside(cut, key_of(z), i)) mine += weight(((double)z - top) * scale, s.tab, row_bits);
    }
    prefix(mine, total, s);
    const uint64_t want = (uint64_t)ceil((double)top_p * (double)total);
    const Cut p = narrow<F32, true>(row, V, want < 1 ? 1 : want < total ? want : total, top, scale, row_bits, s);
    if (p.key > cut.key || (p.key == cut.key && p.last < cut.last)) cut = p;
  }
  const double floor_w = ldexp((double)min_p, row_bits);
  auto w_kept = [&](int64_t i) {
    const float z = logit<F32>(row, i);
    if (!inside(cut, key_of(z), i)) return (uint64_t)0;
    const uint64_t w = weight(((double)z - top) * scale, s.tab, row_bits);
    return (double)w >= floor_w ? w : (uint64_t)0;
  };
  // the tile in which the sum passes the target, and the entry in the tile
  const int64_t tiles = (V + kTile - 1) / kTile;
  uint64_t total = 0;
  __syncthreads();
  for (int64_t b = 0; b < tiles; ++b) {
    uint64_t mine = 0, all;
    for (int i = 0; i < 8; ++i) {
      const int64_t at = b * kTile + i * kSelect + tid;
      if (at < V) mine += w_kept(at);
    }
    prefix(mine, all, s);
    if (tid == 0) s.mass[b] = all;
    total += all;
  }
  __syncthreads();
  uint64_t target = target_of(u, total);
  const uint64_t sum = total;
  int64_t b = 0;
  while (b + 1 < tiles && target >= s.mass[b]) target -= s.mass[b++];
  const int64_t at = b * kTile + tid * 8;
  uint64_t mine = 0, all;
  for (int i = 0; i < 8; ++i)
    if (at + i < V) mine += w_kept(at + i);
  uint64_t y = prefix(mine, all, s);
  if (y <= target && target < y + mine)
    for (int i = 0; i < 8; ++i) {
      if (at + i >= V) break;
      y += w_kept(at + i);
      if (y > target) {
        answer(at + i, log_p(at + i, sum, row_bits));
        break;
      }
    }
}

// ------------------------------------------------------------------------------------------------
// launchers
// ------------------------------------------------------------------------------------------------
template <bool F32, bool SAMPLE>
static hipError_t scan(const RowsArgs& r, hipStream_t st) {
  const FlatGrid g = flat_grid(r.T * r.chunks);
  const dim3 grid(g.x, g.y);
  switch (r.per_thread) {
    case 8: hipLaunchKernelGGL((rows_scan_kernel<F32, 8, SAMPLE>), grid, dim3(kRowThreads), 0, st, r); break;
    case 16: hipLaunchKernelGGL((rows_scan_kernel<F32, 16, SAMPLE>), grid, dim3(kRowThreads), 0, st, r); break;
    case 32: hipLaunchKernelGGL((rows_scan_kernel<F32, 32, SAMPLE>), grid, dim3(kRowThreads), 0, st, r); break;
    default: hipLaunchKernelGGL((rows_scan_kernel<F32, 64, SAMPLE>), grid, dim3(kRowThreads), 0, st, r);
  }
  return hipGetLastError();
}

hipError_t launch_top_logits(const RowsArgs& r, hipStream_t st) {
  const hipError_t e = r.f32 ? scan<true, false>(r, st) : scan<false, false>(r, st);
  if (e != hipSuccess) return e;
  if (r.f32) hipLaunchKernelGGL(top_select_kernel<true>, dim3((uint32_t)r.T), dim3(kSelect), 0, st, r);
  else hipLaunchKernelGGL(top_select_kernel<false>, dim3((uint32_t)r.T), dim3(kSelect), 0, st, r);
  return hipGetLastError();
}

hipError_t launch_sample(const RowsArgs& r, hipStream_t st) {
  const hipError_t e = r.f32 ? scan<true, true>(r, st) : scan<false, true>(r, st);
  if (e != hipSuccess) return e;
  if (r.f32) hipLaunchKernelGGL(sample_select_kernel<true>, dim3((uint32_t)r.T), dim3(kSelect), 0, st, r);
  else hipLaunchKernelGGL(sample_select_kernel<false>, dim3((uint32_t)r.T), dim3(kSelect), 0, st, r);
  return hipGetLastError();
}

}  // namespace kd
