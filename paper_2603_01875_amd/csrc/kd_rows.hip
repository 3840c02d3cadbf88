// Rows of logits: the top logits of each (kd_top_logits), one token sampled from each (kd_sample).
//
// Both read the logits once.  A first kernel, a workgroup to a piece of a row (a chunk), leaves the chunk's sum of w = exp((z - largest of
// the chunk) / tau) and, per thread, the largest entry of its share (a group).  The last, a workgroup to a row, works on these: the
// G-th largest of the groups' largest entries is a bound that at least G entries reach, and only groups that reach it hold entries
// that do, so that a few hundred groups are read again, and a short list is sorted.  Sampling from all of a row needs the sums alone: the
// chunk in which the sum of w passes u times the whole is read again.
// Sampling under top-p or min-p without a top-k may keep any number of entries.  There two kernels come between, again many workgroups
// to a row (wide): one adds up w by bins of the logit, the other the w above the bin in which the sum passes top-p of the whole, tile by tile, and
// lists that bin's entries.
// A list that does not fit (thousands of equal entries) and a top-k of more than kReach go the slow way: passes of the last kernel over the row that narrow the
// last kept entry down (top-k 3000 in 64 rows of 128256 fp32: 281 us, beside 43 for 1000).
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_launch.h"
#include "kd_unaligned.hpp"
#include "kd_weight.hpp"

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
// first kernel
//
// All of a thread's loads are on their way at once, and only then used.  Top logits: bound by memory, 4096 x 151936 bf16 212 to 243 us (5.1 to 5.9 TB/s).  Sampling: by
// the exponentials in 64 bits, 21 instructions an entry issued at 90 % of the rate, 512 x 151936 bf16 61 us (2.5 TB/s).
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ float row_temperature(const RowsArgs& a, int64_t t) { return a.temperature_rows ? a.temperature_rows[t] : a.tau; }

template <bool F32, int E, bool SAMPLE>
__global__ __launch_bounds__(kRowThreads) void rows_scan_kernel(const RowsArgs a) {
  constexpr int VE = F32 ? 4 : 8, J = E / VE, NT = kRowThreads, NW = NT / 64;
  static_assert(E % VE == 0, "whole loads");
  __shared__ uint32_t keys[NW];
  __shared__ uint64_t sums[NW];
  const int64_t piece = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, t = piece / a.chunks;
  if (t >= a.T) return;                // (the last row of a large grid)
  const int c = (int)(piece - t * a.chunks), tid = threadIdx.x;
  const void* const row = row_of<F32>(a, t);
  const int64_t at = (int64_t)c * (NT * E) + tid * VE;
  float z[E];
  auto unpack = [&](int j, const u32x4_t& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (F32) z[j * VE + i] = __uint_as_float(v[i]);
      else {
        z[j * VE + (2 * i) % VE] = __uint_as_float(v[i] << 16);
        z[j * VE + (2 * i + 1) % VE] = __uint_as_float(v[i] & 0xffff0000u);
      }
    }
  };
  if ((int64_t)(c + 1) * (NT * E) <= a.V) {
    u32x4_t v[J];
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = load16((const char*)row + (at + j * (NT * VE)) * (F32 ? 4 : 2));
#pragma unroll
    for (int j = 0; j < J; ++j) unpack(j, v[j]);
  } else {
    // the row's end: whole loads as far as they go (an address that is surely there where they do not), then the entries behind the last one,
    // all under way together as well
    u32x4_t v[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int64_t k = at + j * (NT * VE);
      v[j] = a.V >= VE ? load16((const char*)row + (k + VE <= a.V ? k : 0) * (F32 ? 4 : 2)) : u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int64_t k = at + j * (NT * VE);
      unpack(j, v[j]);
      if (k + VE > a.V)
#pragma unroll
        for (int i = 0; i < VE; ++i) z[j * VE + i] = -__builtin_inff();
      if (k < a.V && k + VE > a.V) {
        float e[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) e[i] = logit<F32>(row, k + i < a.V ? k + i : a.V - 1);
#pragma unroll
        for (int i = 0; i < VE; ++i) z[j * VE + i] = k + i < a.V ? e[i] : -__builtin_inff();
      }
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
  if (!SAMPLE || a.group) a.group[t * ((int64_t)a.chunks * NT) + c * NT + tid] = key;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
  if ((tid & 63) == 0) keys[tid >> 6] = key;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) key = max(key, keys[w]);
  if (SAMPLE && a.wide && c == 0 && t < kWideRows) {   // (the wide kernels add to these; of later rows: wide_clear_kernel)
    for (int i = tid; i < kWideBins; i += NT) a.wide[t].bins[i] = 0;
    if (tid == 0) a.wide[t].count = 0;
  }
  const float top = value_of(key);
  RowChunk out{0, 0.f, key};
  if (SAMPLE) {
    const float tau = row_temperature(a, t);
    uint64_t s = 0;
    if (tau > 0.f) {
      const Exponents x = exponents_of(top, kLog2e / (double)tau);
      if (x.base != 0.f)
#pragma unroll
        for (int i = 0; i < E; ++i) z[i] -= x.base;
      double w = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) w += weight(fma((double)z[i], x.scale, -x.zero));
      s = whole(w, kChunkBits);
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
constexpr int kList = kWideList;       // entries of the list at most
constexpr int kGroups = 1536;          // groups that are read again at most
constexpr int kNear = 1792;            // bins by the distance from the largest key
constexpr int kFlat = kWideBins;       // bins by the distance from the largest value
constexpr int kTile = kWideTile, kEach = kTile / kSelect;      // entries whose sum the slow way keeps
// Sampling: groups that the list takes, for a top-k of at most kReach as many, else (top-p and min-p, mostly) kReachAll.
constexpr int kReach = 1024, kReachAll = 512;
static_assert(kList / kSelect == kEach, "a thread's entries of a list and of a tile");

struct SelectLds {
  union {
    uint64_t list[kList];              // key, complement of the index: descending order is the order of the entries
    uint64_t mass[kList];              // chunks' or tiles' sums
    uint64_t flat[kFlat];
  };
  union {
    uint32_t groups[kGroups];
    uint32_t near_[kNear];
    uint64_t bin_mass[256];
  };
  uint64_t scan[kSelect / 64 + 1];
  uint32_t word[kSelect / 64];
  double part[kSelect / 64];
  uint32_t count;
  uint64_t value[2];
};

// v of the lane that a DPP control names, 0 where there is none (or the row mask leaves it out).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t lane_from(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (uint64_t)hi << 32 | lo;
}
// Inclusive prefix sum over the wave: within rows of 16 lanes, then the rows' sums (a shuffle through LDS for each step took five times as long).
__device__ __forceinline__ uint64_t wave_prefix(uint64_t v) {
  v += lane_from<0x111, 0xf>(v);       // row_shr 1, 2, 4, 8
  v += lane_from<0x112, 0xf>(v);
  v += lane_from<0x114, 0xf>(v);
  v += lane_from<0x118, 0xf>(v);
  v += lane_from<0x142, 0xa>(v);       // row_bcast 15, into rows 1 and 3
  v += lane_from<0x143, 0xc>(v);       // row_bcast 31, into rows 2 and 3
  return v;
}

// Exclusive prefix sum over the workgroup; total to all.
__device__ __forceinline__ uint64_t prefix(uint64_t v, uint64_t& total, SelectLds& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t x = wave_prefix(v);
  __syncthreads();                     // (what an earlier call left has been read)
  if (lane == 63) s.scan[wave] = x;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) {
    const uint64_t y = s.scan[w];
    before += w < wave ? y : 0;
    all += y;
  }
  total = all;
  return before + x - v;
}

// The row's largest key.
__device__ __forceinline__ uint32_t largest_key(const RowsArgs& a, int64_t t, SelectLds& s) {
  uint32_t key = 0;
  for (int c = threadIdx.x; c < a.chunks; c += kSelect) key = max(key, a.chunk[t * a.chunks + c].key);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) key = max(key, (uint32_t)__shfl_xor((int)key, o, 64));
  if ((threadIdx.x & 63) == 0) s.word[threadIdx.x >> 6] = key;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) key = max(key, s.word[w]);
  __syncthreads();
  return key;
}

// A thread's entries of a tile; minus infinity behind the row.
template <bool F32>
__device__ __forceinline__ void load_tile(float (&z)[kEach], const void* row, int64_t V, int64_t at) {
  static_assert(kEach == 8, "one or two loads");
  if (at + kEach <= V) {
#pragma unroll
    for (int h = 0; h < (F32 ? 2 : 1); ++h) {
      const u32x4_t v = load16((const char*)row + at * (F32 ? 4 : 2) + 16 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (F32) z[4 * h + i] = __uint_as_float(v[i]);
        else {
          z[2 * i] = __uint_as_float(v[i] << 16);
          z[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) z[i] = at + i < V ? logit<F32>(row, at + i) : -__builtin_inff();
  }
}

// Bin of a key by its distance from the row's largest: 64 bins to a doubling, so fine near the top whatever the logits' scale.
__device__ __forceinline__ uint32_t near_bin(uint32_t distance) {
  if (distance < 64) return distance;
  const int e = 31 - __clz((int)distance);
  return (uint32_t)(e - 5) << 6 | (distance >> (e - 6) & 63);
}
// The largest distance of a bin.
__device__ __forceinline__ uint32_t near_end(uint32_t bin) {
  if (bin < 64) return bin;
  const int e = (int)(bin >> 6) + 5;
  return (((bin & 63) + 65) << (e - 6)) - 1;
}

// Keys of a row's groups (a multiple of 256), 16 bytes a thread and several of them in flight: put(four keys, number of the first).
template <class Put>
__device__ __forceinline__ void for_groups(const uint32_t* group, int64_t n, Put&& put) {
  constexpr int U = 4, STEP = kSelect * 4;
  for (int64_t base = (int64_t)threadIdx.x * 4; base < n; base += U * STEP) {
    u32x4_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *(const u32x4_t*)(group + (base + u * STEP < n ? base + u * STEP : base));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (base + u * STEP < n) put(v[u], (uint32_t)(base + u * STEP));
  }
}

// A key that at least G of the row's n groups reach, and not many more if the largest are spread a little.
__device__ __forceinline__ uint32_t bound_of(const uint32_t* group, int64_t n, uint32_t G, uint32_t top, SelectLds& s) {
  constexpr int PER = (kNear + kSelect - 1) / kSelect;
  for (int i = threadIdx.x; i < kNear; i += kSelect) s.near_[i] = 0;
  __syncthreads();
  for_groups(group, n, [&](const u32x4_t& keys, uint32_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) atomicAdd(&s.near_[near_bin(top - keys[i])], 1u);
  });
  __syncthreads();
  uint32_t mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    mine[i] = b < kNear ? s.near_[b] : 0;
    sum += mine[i];
  }
  uint64_t all;
  uint64_t before = prefix(sum, all, s);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < G && before + mine[i] >= G) s.value[0] = threadIdx.x * PER + i;
    before += mine[i];
  }
  __syncthreads();
  const uint32_t end = near_end((uint32_t)s.value[0]);
  __syncthreads();
  return end < top ? top - end : 0;
}

// Places in a list for what the lanes have to put, N things each: one addition to the count for a wave.
template <int N>
__device__ __forceinline__ void places_in(uint32_t* count, const bool (&put)[N], uint32_t (&to)[N]) {
  uint64_t lanes[N];
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lanes[i] = __ballot(put[i]);
    to[i] = all + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes[i], 0));
    all += (uint32_t)__popcll(lanes[i]);
  }
  if (!all) return;
  uint32_t first = 0;
  const int leader = __ffsll((unsigned long long)__ballot(1)) - 1;
  if ((int)(threadIdx.x & 63) == leader) first = atomicAdd(count, all);
  first = (uint32_t)__builtin_amdgcn_readlane((int)first, leader);
#pragma unroll
  for (int i = 0; i < N; ++i) to[i] += first;
}

// Entries of the row that reach `bound` into the list; their number, which may be more than fit (then the list is not whole).
template <bool F32>
__device__ __forceinline__ uint32_t gather(const RowsArgs& a, int64_t t, uint32_t bound, SelectLds& s) {
  constexpr int VE = F32 ? 4 : 8;
  const void* const row = row_of<F32>(a, t);
  const int64_t n = (int64_t)a.chunks * kRowThreads;
  const uint32_t* const group = a.group + t * n;
  const int J = a.per_thread / VE;
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  for_groups(group, n, [&](const u32x4_t& keys, uint32_t g) {
    bool put[4];
    uint32_t to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) put[i] = keys[i] >= bound;
    places_in(&s.count, put, to);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (put[i] && to[i] < (uint32_t)kGroups) s.groups[to[i]] = g + i;
  });
  __syncthreads();
  const uint32_t groups = s.count;
  __syncthreads();
  if (groups > (uint32_t)kGroups) return ~0u;
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  // 16 bytes of a group a thread, U of them in flight
  constexpr int U = 4;
  const int shift = 31 - __clz(J);                     // (J is a power of two)
  const uint32_t pieces = groups << shift;
  for (uint32_t q0 = threadIdx.x; q0 - threadIdx.x < pieces; q0 += U * kSelect) {
    u32x4_t v[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t q = q0 + u * kSelect < pieces ? q0 + u * kSelect : 0;
      const uint32_t g = s.groups[q >> shift], j = q & (J - 1);
      at[u] = ((int64_t)(g / kRowThreads) * a.per_thread + j * VE) * kRowThreads + g % kRowThreads * VE;
      if (q0 + u * kSelect >= pieces) at[u] = a.V;
      v[u] = a.V >= VE ? load16((const char*)row + (at[u] + VE <= a.V ? at[u] : 0) * (F32 ? 4 : 2)) : u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float z[VE];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (F32) z[i] = __uint_as_float(v[u][i]);
        else {
          z[(2 * i) % VE] = __uint_as_float(v[u][i] << 16);
          z[(2 * i + 1) % VE] = __uint_as_float(v[u][i] & 0xffff0000u);
        }
      }
      if (at[u] + VE > a.V)
#pragma unroll
        for (int i = 0; i < VE; ++i) z[i] = at[u] + i < a.V ? logit<F32>(row, at[u] + i) : -__builtin_inff();
      bool put[VE];
      uint32_t key[VE], to[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        key[i] = key_of(z[i]);
        put[i] = key[i] >= bound;
      }
      places_in(&s.count, put, to);
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (put[i] && to[i] < (uint32_t)kList) s.list[to[i]] = (uint64_t)key[i] << 32 | (uint32_t)~(uint32_t)(at[u] + i);
    }
  }
  __syncthreads();
  const uint32_t found = s.count;
  __syncthreads();
  return found;
}

// Prefix sums over near_ in place (a bin's first place), the same for all threads afterwards.
__device__ __forceinline__ void starts_of_bins(SelectLds& s) {
  constexpr int PER = (kNear + kSelect - 1) / kSelect;
  uint32_t mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    mine[i] = b < kNear ? s.near_[b] : 0;
    sum += mine[i];
  }
  uint64_t all;
  uint32_t before = (uint32_t)prefix(sum, all, s);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    if (b < kNear) s.near_[b] = before;
    before += mine[i];
  }
  __syncthreads();
}

// Sorts list[0 .. n) in descending order, n at most half a list (no entry twice); top: its largest key.  By bins of the distance from the top
// into the list's other half, then each entry counts the larger ones of its bin: n^2 steps for n equal logits, so that 2000 of them at the top of each of 64 rows make the top 50
// take 185 us instead of 18 (600: 44).
__device__ __forceinline__ void sort_by_bins(uint32_t n, uint32_t top, SelectLds& s) {
  constexpr int HELD = kList / 2 / kSelect;
  for (int i = threadIdx.x; i < kNear; i += kSelect) s.near_[i] = 0;
  __syncthreads();
  uint64_t mine[HELD];
  uint32_t bin[HELD], at[HELD];
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const uint32_t i = threadIdx.x + h * kSelect;
    if (i >= n) continue;
    mine[h] = s.list[i];
    bin[h] = near_bin(top - (uint32_t)(mine[h] >> 32));
    at[h] = atomicAdd(&s.near_[bin[h]], 1u);
  }
  __syncthreads();
  starts_of_bins(s);
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (threadIdx.x + h * kSelect < n) s.list[kList / 2 + s.near_[bin[h]] + at[h]] = mine[h];
  __syncthreads();
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    if (threadIdx.x + h * kSelect >= n) continue;
    const uint32_t first = s.near_[bin[h]], last = bin[h] + 1 < (uint32_t)kNear ? s.near_[bin[h] + 1] : n;
    uint32_t rank = first;
#pragma unroll 4
    for (uint32_t i = first; i < last; ++i) rank += s.list[kList / 2 + i] > mine[h];
    s.list[rank] = mine[h];
  }
  __syncthreads();
}

// The same for any n.  Short lists: each entry counts the larger ones.  More than half a list: by exchanges.
__device__ __forceinline__ void sort_list(uint32_t n, uint32_t top, SelectLds& s) {
  if (n <= 128) {
    uint64_t mine = 0;
    uint32_t rank = 0;
    if (threadIdx.x < n) {
      mine = s.list[threadIdx.x];
#pragma unroll 8
      for (uint32_t i = 0; i < n; ++i) rank += s.list[i] > mine;
    }
    __syncthreads();
    if (threadIdx.x < n) s.list[rank] = mine;
    __syncthreads();
    return;
  }
  if (n <= kList / 2) {
    sort_by_bins(n, top, s);
    return;
  }
  uint32_t size = 512;
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
      // pairs up to 64 apart lie in 128 entries that one wave has from step to step: it waits for itself alone
      const uint32_t after = j > 1 ? j >> 1 : k;
      if (j > 64 || after > 64) __syncthreads();
      else {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
      }
    }
  __syncthreads();
}

struct Row {
  const void* p;
  int64_t V;
  float top;             // largest entry
  double scale;          // t = (z - top) scale
  float bins;            // flat bins to a unit of the logits
  double one;            // 2^bits, a weight of 1
};
__device__ __forceinline__ uint64_t row_weight(const Row& r, float z) { return whole_one(weight(((double)z - (double)r.top) * r.scale), r.one); }
// Bin of an entry by its distance from the largest, all of the entries with a weight of 2^-44 and more in kFlat - 1 of them.
__device__ __forceinline__ uint32_t flat_bin(const Row& r, float z) {
  const float x = (r.top - z) * r.bins;
  return x < (float)(kFlat - 1) ? (uint32_t)x : kFlat - 1;
}
// An entry: its key, the complement of its index.  Descending order is the order of the entries.
__device__ __forceinline__ uint64_t entry_of(float z, uint32_t i) { return (uint64_t)key_of(z) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float entry_value(uint64_t e) { return value_of((uint32_t)(e >> 32)); }
__device__ __forceinline__ uint32_t entry_index(uint64_t e) { return ~(uint32_t)e; }

// Entries that the threads hold (0: none).
constexpr int kHeld = kList / kSelect;
__device__ __forceinline__ void hold(uint64_t (&held)[kHeld], const uint64_t* list, uint32_t n) {
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const uint32_t i = threadIdx.x + h * kSelect;
    held[h] = i < n ? list[i] : 0;
  }
}

// The last entry of the fewest, in descending order and not behind `limit`, of those that are held or of the whole row, whose number (by_weight: sum
// of w) is at least `want`, which all of them reach; want > 0.  By 11, 11, 10 bits of the key and 12, 12 of the index at a time, the
// sums over a digit's values in LDS (overwrites the list).  One piece of code for all who ask: this kernel runs through each of its
// parts once, and what it waits for is its own instructions (198 KB of them, with a copy of everything for each use, took twice as long).
template <bool F32>
__device__ __forceinline__ uint64_t last_of(const uint64_t (&held)[kHeld], bool whole_row, const Row& r, uint64_t limit, uint64_t want, bool by_weight,
                                            SelectLds& s) {
  constexpr int PER = 4096 / kSelect;
  uint64_t high = 0;
#pragma unroll 1
  for (int level = 0; level < 5; ++level) {
    const int shift = level == 0 ? 53 : level == 1 ? 42 : level == 2 ? 32 : level == 3 ? 12 : 0, bits = level < 2 ? 11 : level == 2 ? 10 : 12;
    const uint64_t above = level == 3 ? ~0ull << 32 : level ? ~0ull << (shift + bits) : 0;      // (an index has 24 bits, their complement 8 ones in front)
    const int bins = 1 << bits;
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kSelect) s.mass[i] = 0;
    __syncthreads();
    int64_t at = (int64_t)threadIdx.x * kEach;
#pragma unroll 1
    for (;;) {
      uint64_t e[kHeld], w[kHeld];
      bool in[kHeld], any = false;
      if (whole_row) {
        float z[kEach];
        load_tile<F32>(z, r.p, r.V, at);
#pragma unroll
        for (int h = 0; h < kHeld; ++h) e[h] = at + h < r.V ? entry_of(z[h], (uint32_t)(at + h)) : 0;
      } else {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) e[h] = held[h];
      }
#pragma unroll
      for (int h = 0; h < kHeld; ++h) {
        in[h] = e[h] && e[h] >= limit && ((e[h] ^ high) & above) == 0;
        any |= in[h];
        w[h] = 1;
      }
      if (any && by_weight)
#pragma unroll
        for (int h = 0; h < kHeld; ++h) w[h] = row_weight(r, entry_value(e[h]));
#pragma unroll
      for (int h = 0; h < kHeld; ++h)
        if (in[h] && w[h]) atomicAdd((unsigned long long*)&s.mass[e[h] >> shift & (bins - 1)], (unsigned long long)w[h]);
      at += kTile;
      if (!whole_row || at - (int64_t)threadIdx.x * kEach >= r.V) break;
    }
    __syncthreads();
    // bins from the largest down, PER of them a thread
    uint64_t sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = bins - 1 - ((int)threadIdx.x * PER + i);
      sum += b >= 0 ? s.mass[b] : 0;
    }
    uint64_t before = prefix(sum, all, s);
    if (before < want && before + sum >= want)
      for (int i = 0; i < PER; ++i) {
        const int b = bins - 1 - ((int)threadIdx.x * PER + i);
        const uint64_t m = b >= 0 ? s.mass[b] : 0;
        if (before + m >= want) {
          s.value[0] = b;
          s.value[1] = before;
          break;
        }
        before += m;
      }
    __syncthreads();
    high |= s.value[0] << shift;
    if (level >= 3) high |= 0xff000000ull;
    want -= s.value[1];
  }
  __syncthreads();
  return high;
}

// ------------------------------------------------------------------------------------------------
// top logits
//
// Four workgroups of eight waves a CU, which wait for each other's LDS and groups: 4096 rows of 151936, 64 of each, 78 to 93 us; 7 rows 9.
// Where V / 8 is no more than K every entry is listed, and a row of more entries than a list goes the slow way: top 1024 of 512 rows of 8192 fp32 47 us,
// of 9000 70, of 12288, which take the short one, 35.
// ------------------------------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ void put_top(const RowsArgs& a, int64_t t, int at, uint64_t entry) {
  const uint32_t key = (uint32_t)(entry >> 32), index = ~(uint32_t)entry;
  const bool there = key > kKeyMinusInf;
  const int64_t to = t * a.K + at;
  if (F32) ((float*)a.top)[to] = there ? ((const float*)row_of<true>(a, t))[index] : -__builtin_inff();
  else ((uint16_t*)a.top)[to] = there ? ((const uint16_t*)row_of<false>(a, t))[index] : (uint16_t)0xff80;
  if (a.index64) ((int64_t*)a.index)[to] = there ? (int64_t)index : -1;
  else ((int32_t*)a.index)[to] = there ? (int32_t)index : -1;
}

template <bool F32>
__global__ __launch_bounds__(kSelect, 8) void top_select_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const int64_t n = (int64_t)a.chunks * kRowThreads;
  const uint32_t key = largest_key(a, t, s);
  if (a.lse) {
    // the chunks' sums at the row's largest entry, in a fixed order
    const double top = value_of(key);
    double sum = 0;
    for (int c = tid; c < a.chunks; c += kSelect) {
      const RowChunk& r = a.chunk[t * a.chunks + c];
      if (r.key > kKeyMinusInf) sum += (double)r.part * exp(((double)value_of(r.key) - top) / (double)a.tau);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) s.part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
      sum = 0;
      for (int w = 0; w < kSelect / 64; ++w) sum += s.part[w];
      a.lse[t] = key == kKeyNaN ? __builtin_nanf("") : key == kKeyInf ? __builtin_inff() : key <= kKeyMinusInf ? -__builtin_inff()
                 : (float)(top / (double)a.tau + log(sum));
    }
  }
  // (entries of minus infinity are no entries: the lowest bound is above them)
  uint32_t bound = kKeyMinusInf + 1;
  if ((int64_t)a.K < n) bound = max(bound, bound_of(a.group + t * n, n, (uint32_t)a.K, key, s));
  uint32_t found = gather<F32>(a, t, bound, s);
  if (found > (uint32_t)kList) {
    const Row r{row_of<F32>(a, t), a.V, 0.f, 0, 0.f, 0.};
    const uint64_t none[kHeld] = {}, last = last_of<F32>(none, true, r, 0, (uint64_t)a.K, false, s);
    if (tid == 0) s.count = 0;
    __syncthreads();
#pragma unroll 1
    for (int64_t at = (int64_t)tid * kEach; at - (int64_t)tid * kEach < a.V; at += kTile) {
      float z[kEach];
      load_tile<F32>(z, r.p, a.V, at);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const uint64_t e = entry_of(z[i], (uint32_t)(at + i));
        if (at + i < a.V && e >= last && (uint32_t)(e >> 32) > kKeyMinusInf) s.list[atomicAdd(&s.count, 1u)] = e;
      }
    }
    __syncthreads();
    found = s.count;
  }
  sort_list(found, key, s);
  for (int i = tid; i < a.K; i += kSelect) put_top<F32>(a, t, i, i < (int)found ? s.list[i] : 0);
}

// ------------------------------------------------------------------------------------------------
// sampling
//
// Bins and tiles read the row again (10 and 12 us for 64 rows of 128256 fp32), and the select kernel is a chain of short steps of one workgroup a row, each some
// thousand cycles of latency: 14 to 15 us for 512 rows without a filter, 16 for one row with a short list, 37 where lists of a thousand are sorted.
// ------------------------------------------------------------------------------------------------
// A row's settings, and whether it can be drawn from.
struct Draw {
  float u, tau, top_p, min_p;
  int64_t top_k;
  bool greedy, all_k, valid;
  // top-p and min-p over all entries, for which the wide kernels work
  __device__ __forceinline__ bool wide() const { return valid && all_k && (top_p < 1.f || min_p > 0.f); }
};
__device__ __forceinline__ Draw draw_of(const RowsArgs& a, int64_t t, uint32_t key) {
  Draw d;
  d.u = a.u[t];
  d.tau = row_temperature(a, t);
  d.top_p = a.top_p_rows ? a.top_p_rows[t] : a.top_p;
  d.min_p = a.min_p_rows ? a.min_p_rows[t] : a.min_p;
  d.top_k = a.top_k_rows ? a.top_k_rows[t] : a.top_k;
  d.greedy = d.tau == 0.f;
  d.all_k = !d.greedy && (d.top_k == 0 || d.top_k >= a.V);
  d.valid = d.u >= 0.f && d.u < 1.f && (d.greedy || (d.tau >= 1e-6f && d.tau <= 1e6f)) && d.top_k >= 0 && d.top_p > 0.f && d.top_p <= 1.f &&
            d.min_p >= 0.f && d.min_p <= 1.f && key > kKeyMinusInf && key < kKeyInf;
  return d;
}
// Bits of a weight in sums of chunks' sums: V entries of at most 2^bits.
__device__ __forceinline__ int bits_of_row(int64_t V) { return min(kChunkBits, 62 - (64 - __clzll((unsigned long long)V))); }
// Bits of a weight in sums over the row's entries, each of them rounded: as many as the row's sum leaves of 62, and no more than whole_one takes.  (As many as V equal
// entries leave would be 44 at V = 151936 and 37 at 2^24: a tail of small weights, all rounded the same way, would be off by V halves of that.)  The chunks'
// sums in 32 bits, in a fixed order and with no operation that a compiler may fuse or not: whichever kernel asks for a row gets the same bits.
constexpr int kMostBits = 51;
__device__ __forceinline__ int bits_of_sum(const RowsArgs& a, int64_t t, float top, double scale, SelectLds& s) {
  float sum = 0.f;
  for (int c = threadIdx.x; c < a.chunks; c += kSelect) {
    const RowChunk& q = a.chunk[t * a.chunks + c];
    if (q.key > kKeyMinusInf) sum = fmaf((float)q.sum, __builtin_amdgcn_exp2f((value_of(q.key) - top) * (float)scale), sum);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = sum;
  __syncthreads();
  double all = 0;
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) all += s.part[w];
  __syncthreads();
  int e;                               // (the sum is less than 2^e)
  frexp(fmax(ldexp(all, -kChunkBits), 1.), &e);
  return min(kMostBits, 62 - e);
}
__device__ __forceinline__ Row row_for(const void* row, int64_t V, float top, double scale, int bits) {
  return Row{row, V, top, scale, (float)((kFlat - 1) / 44. * scale), ldexp(1., bits)};
}

// The part of a row that a workgroup of the wide kernels has: tiles first .. last - 1.
struct Part { int64_t t; int first, last; };      // (t >= a.rows_end: none)
__device__ __forceinline__ Part part_of(const RowsArgs& a) {
  const int64_t piece = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int tiles = (int)((a.V + kTile - 1) / kTile);
  Part p;
  p.t = a.row0 + piece / a.wide_parts;
  const int i = (int)(piece % a.wide_parts), per = (tiles + a.wide_parts - 1) / a.wide_parts;
  p.first = i * per;
  p.last = min(tiles, p.first + per);
  return p;
}

__global__ __launch_bounds__(256) void wide_clear_kernel(const RowsArgs a) {
  for (int i = threadIdx.x; i < kWideBins; i += 256) a.wide[blockIdx.x].bins[i] = 0;
  if (threadIdx.x == 0) a.wide[blockIdx.x].count = 0;
}

// w by bins, added to the row's (which the first kernel has cleared): whole numbers, so in any order.
template <bool F32>
__global__ __launch_bounds__(kSelect) void sample_bins_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const Part p = part_of(a);
  if (p.t >= a.rows_end || p.first >= p.last) return;
  const int tid = threadIdx.x;
  const uint32_t key = largest_key(a, p.t, s);
  const Draw d = draw_of(a, p.t, key);
  if (!d.wide() || d.top_p == 1.f) return;
  const double scale = kLog2e / (double)d.tau;
  const Row r = row_for(row_of<F32>(a, p.t), a.V, value_of(key), scale, bits_of_sum(a, p.t, value_of(key), scale, s));
  for (int i = tid; i < kFlat; i += kSelect) s.flat[i] = 0;
  __syncthreads();
  for (int b = p.first; b < p.last; ++b) {
    float z[kEach];
    uint64_t w[kEach];
    load_tile<F32>(z, r.p, a.V, (int64_t)b * kTile + tid * kEach);
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = row_weight(r, z[i]);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (w[i]) atomicAdd((unsigned long long*)&s.flat[flat_bin(r, z[i])], (unsigned long long)w[i]);
  }
  __syncthreads();
  for (int i = tid; i < kFlat; i += kSelect)
    if (s.flat[i]) atomicAdd((unsigned long long*)&a.wide[p.t - a.row0].bins[i], (unsigned long long)s.flat[i]);
}

// The bin in which the sum over the bins passes `share` of the whole, and what is left to reach in it.
struct Border { uint32_t bin; uint64_t left; };
__device__ __forceinline__ Border border_of(const uint64_t* bins, double share, SelectLds& s) {
  constexpr int PER = kFlat / kSelect;
  uint64_t mine[PER], sum = 0, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += mine[i] = bins[threadIdx.x * PER + i];
  uint64_t before = prefix(sum, all, s);
  uint64_t want = (uint64_t)ceil(share * (double)all);
  want = want < 1 ? 1 : want < all ? want : all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < want && before + mine[i] >= want) {
      s.value[0] = threadIdx.x * PER + i;
      s.value[1] = want - before;
    }
    before += mine[i];
  }
  __syncthreads();
  const Border b{(uint32_t)s.value[0], s.value[1]};
  __syncthreads();
  return b;
}

// Each tile's sum of the kept w above that bin, and the bin's entries (as many as there is room for, and their number).
template <bool F32>
__global__ __launch_bounds__(kSelect) void sample_tiles_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const Part p = part_of(a);
  if (p.t >= a.rows_end || p.first >= p.last) return;
  const int tid = threadIdx.x;
  const uint32_t key = largest_key(a, p.t, s);
  const Draw d = draw_of(a, p.t, key);
  if (!d.wide()) return;
  const double scale = kLog2e / (double)d.tau;
  const Row r = row_for(row_of<F32>(a, p.t), a.V, value_of(key), scale, bits_of_sum(a, p.t, value_of(key), scale, s));
  const uint32_t bin = d.top_p < 1.f ? border_of(a.wide[p.t - a.row0].bins, (double)d.top_p, s).bin : ~0u;
  const uint64_t least = (uint64_t)ceil((double)d.min_p * r.one);
  for (int b = p.first; b < p.last; ++b) {
    const int64_t at = (int64_t)b * kTile + tid * kEach;
    float z[kEach];
    load_tile<F32>(z, r.p, a.V, at);
    uint64_t sum = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint64_t w = row_weight(r, z[i]);
      sum += (flat_bin(r, z[i]) < bin) & (w >= least) ? w : 0;
    }
    if (bin != ~0u) {
      uint32_t hits = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) hits |= (uint32_t)(flat_bin(r, z[i]) == bin && at + i < a.V) << i;
      if (hits) {
        uint32_t to = atomicAdd(&a.wide[p.t - a.row0].count, (uint32_t)__popc(hits));
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (hits >> i & 1) {
            if (to < (uint32_t)kWideList) a.wide[p.t - a.row0].list[to] = (uint64_t)key_of(z[i]) << 32 | (uint32_t)~(uint32_t)(at + i);
            ++to;
          }
      }
    }
    prefix(sum, all, s);
    if (tid == 0) a.wide_mass[(p.t - a.row0) * ((a.V + kTile - 1) / kTile) + b] = all;
  }
}

// The largest whole number that is not above u total, and less than it.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const uint64_t x = (uint64_t)((double)u * (double)total);
  return x < total ? x : total - 1;
}

template <bool F32>
__global__ __launch_bounds__(kSelect, 4) void sample_select_kernel(const RowsArgs a) {
  __shared__ SelectLds s;
  const int64_t t = a.row0 + blockIdx.x, n = (int64_t)a.chunks * kRowThreads, V = a.V;
  const int tid = threadIdx.x;
  const uint32_t key = largest_key(a, t, s);
  const Draw d = draw_of(a, t, key);
  auto answer = [&](int64_t token, float logp) {
    if (a.index64) ((int64_t*)a.token)[t] = token;
    else ((int32_t*)a.token)[t] = (int32_t)token;
    if (a.logp) a.logp[t] = logp;
  };
  if (!d.valid) {
    if (tid == 0) answer(-1, __builtin_nanf(""));
    return;
  }
  const double top = value_of(key), scale = kLog2e / (d.greedy ? 1. : (double)d.tau);
  const int tiles = (int)((V + kTile - 1) / kTile);
  auto log_p = [&](float z, double sum) { return d.greedy ? 0.f : (float)(((double)z - top) / (double)d.tau - log(sum)); };

  if (d.all_k && d.top_p == 1.f && d.min_p == 0.f) {
    // chunks' sums at the row's largest entry
    const int row_bits = bits_of_row(V);
    const void* const row = row_of<F32>(a, t);
    uint64_t part = 0, row_total;
    const int per = (a.chunks + kSelect - 1) / kSelect, c0 = tid * per;
    auto chunk_mass = [&](int c) {
      const RowChunk& q = a.chunk[t * a.chunks + c];
      if (q.key <= kKeyMinusInf) return (uint64_t)0;
      return whole((double)q.sum * rescale(value_of(q.key), top, scale), row_bits - kChunkBits);
    };
    if (tid == 0) s.value[0] = s.value[1] = 0;      // (a thread's share holds the target, whatever it is; were it not so, chunk 0 would be read)
#pragma unroll 1
    for (int c = c0; c < c0 + per && c < a.chunks; ++c) part += chunk_mass(c);
    const uint64_t before = prefix(part, row_total, s);
    const uint64_t target = target_of(d.u, row_total);
    if (before <= target && target < before + part) {
      uint64_t x = before;
#pragma unroll 1
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
    const float z0 = value_of(a.chunk[t * a.chunks + c].key);
    const Exponents ex = exponents_of(z0, scale);
    const double inner = ldexp((double)s.value[1], kChunkBits - row_bits) * rescale(top, z0, scale);
    // that chunk again, with its own sums; thread i has `each` entries from the i-th on, VE at a time
    constexpr int VE = F32 ? 4 : 8, MOST = 32 / VE;
    const int each = max(VE, a.per_thread * kRowThreads / kSelect), entries = kRowThreads * a.per_thread;
    const int64_t i0 = (int64_t)c * entries + (int64_t)tid * each;
    const bool here = (tid + 1) * each <= entries;
    auto load = [&](float (&z)[VE], int j) {
      const int64_t at = i0 + j * VE;
      const bool in = here && j * VE < each && at + VE <= V;
      const u32x4_t v = V >= VE ? load16((const char*)row + (in ? at : 0) * (F32 ? 4 : 2)) : u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (F32) z[i] = __uint_as_float(v[i]);
        else {
          z[(2 * i) % VE] = __uint_as_float(v[i] << 16);
          z[(2 * i + 1) % VE] = __uint_as_float(v[i] & 0xffff0000u);
        }
      }
      if (!in)
#pragma unroll
        for (int i = 0; i < VE; ++i) z[i] = here && j * VE < each && at + i < V ? logit<F32>(row, at + i) : -__builtin_inff();
    };
    auto w_of = [&](float v) { return whole_one(weight(exponent(ex, v)), 0x1p48); };
    float z[MOST][VE];
    uint64_t sums[MOST], mine = 0, all;
#pragma unroll
    for (int j = 0; j < MOST; ++j) load(z[j], j);
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      sums[j] = 0;
#pragma unroll
      for (int i = 0; i < VE; ++i) sums[j] += w_of(z[j][i]);
      mine += sums[j];
    }
    uint64_t x = prefix(mine, all, s);
    const uint64_t want = inner < (double)all ? (uint64_t)inner : all - 1;
    if (x <= want && want < x + mine) {
      int at = 0;
      bool past = false;
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        past |= want < x + sums[j];
        if (!past) {
          x += sums[j];
          at = j + 1;
        }
      }
      float v[VE];
      load(v, at);
      past = false;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        x += w_of(v[i]);
        if (x > want && !past) {
          answer(i0 + at * VE + i, log_p(v[i], ldexp((double)row_total, -row_bits)));
          past = true;
        }
      }
    }
    return;
  }

  // (the sums of a list, of no more than kList entries, have room for all bits that a weight may have)
  static_assert(kList <= 1 << (63 - kMostBits), "64 bits");
  const bool wide = a.wide && d.wide();
  Row r = row_for(row_of<F32>(a, t), V, (float)top, scale, wide ? bits_of_sum(a, t, (float)top, scale, s) : kMostBits);
  const int64_t k = d.greedy ? 1 : d.all_k ? V : d.top_k;
  uint64_t held[kHeld], limit = 1;      // entries; the last kept one
  uint32_t found = 0;
  enum { WIDE, LIST, ROW } from = ROW;  // where the kept entries are: above a bin and in its list; in a list of the largest; anywhere
  if (wide) {
    found = d.top_p < 1.f ? a.wide[t - a.row0].count : 0;
    if (found <= (uint32_t)kList) {
      from = WIDE;
      hold(held, a.wide[t - a.row0].list, found);
    }
  } else {
    const uint32_t reach = (uint32_t)(k <= kReach ? k : kReachAll);
    uint32_t bound = kKeyMinusInf + 1;
    if ((int64_t)reach < n) bound = max(bound, bound_of(a.group + t * n, n, reach, key, s));
    found = gather<F32>(a, t, bound, s);
    if (found <= (uint32_t)kList) {
      const bool listed = bound == kKeyMinusInf + 1 || k <= (int64_t)found;      // the whole row, or the first top_k
      hold(held, s.list, found);
      if (d.greedy) {
        uint64_t most = held[0];
#pragma unroll
        for (int h = 1; h < kHeld; ++h) most = max(most, held[h]);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, o, 64));
        __syncthreads();
        if ((tid & 63) == 0) s.scan[tid >> 6] = most;
        __syncthreads();
        if (tid == 0) {
          for (int v = 1; v < kSelect / 64; ++v) most = max(most, s.scan[v]);
          answer(entry_index(most), 0.f);
        }
        return;
      }
      if (listed && found <= 128) {
        const uint64_t least = (uint64_t)ceil((double)d.min_p * r.one);
        // one entry a thread: what is in front of it in descending order, then what is kept in front of it in order of the index
        uint64_t* const w = s.list + 128;
        const uint64_t mine = held[0], my_w = mine ? row_weight(r, entry_value(mine)) : 0;
        __syncthreads();
        if (tid < 128) w[tid] = my_w;
        __syncthreads();
        uint32_t rank = 0;
        uint64_t before = 0, sum, total;
        if (tid < (int)found)
#pragma unroll 8
          for (uint32_t i = 0; i < found; ++i) {
            const bool larger = s.list[i] > mine;
            rank += larger;
            before += larger ? w[i] : 0;
          }
        prefix(mine && (int64_t)rank < k ? my_w : 0, sum, s);      // over the first top_k
        const bool keep = mine && (int64_t)rank < k && (d.top_p == 1.f || (double)before < (double)d.top_p * (double)sum) && my_w >= least;
        prefix(keep ? my_w : 0, total, s);
        if (tid < 128) w[tid] = keep ? my_w : 0;
        __syncthreads();
        const uint64_t target = target_of(d.u, total);
        if (keep) {
          uint64_t y = 0;
#pragma unroll 8
          for (uint32_t i = 0; i < found; ++i) y += entry_index(s.list[i]) < entry_index(mine) ? w[i] : 0;
          if (y <= target && target < y + my_w) answer(entry_index(mine), log_p(entry_value(mine), (double)total / r.one));
        }
        return;
      }
      if (listed) from = LIST;
    }
  }

  if (from == ROW && !wide) r.one = ldexp(1., bits_of_sum(a, t, (float)top, scale, s));
  const uint64_t least = (uint64_t)ceil((double)d.min_p * r.one);
  // A list of up to half a list is sorted, and its sums are those of places.  (64 rows of 128256 fp32, us, so and by the digits below: top-k 300 29 and 38, 1000 43 and 45,
  // 1000 with top-p 0.9 43 and 58.  A wide bin's entries lie close to each other, which is where sorting is slow: one row of 151936 bf16, top-p 0.9, 31 and 38; but
  // lists of up to 2048 of 64 rows of 128256 fp32 82 and 66.)
  const bool sorts = from == LIST ? found <= (uint32_t)kList / 2 && (k < (int64_t)found || d.top_p < 1.f) : from == WIDE && d.top_p < 1.f && found <= (uint32_t)kSelect;
  if (sorts) {
    constexpr int PER = kList / 2 / kSelect;
    uint64_t want = 0;
    if (from == WIDE) {
      want = border_of(a.wide[t - a.row0].bins, (double)d.top_p, s).left;
      s.list[tid] = held[0];
      __syncthreads();
    }
    sort_by_bins(found, key, s);
    uint64_t w[PER], sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      w[i] = at < (int)found && at < k ? row_weight(r, entry_value(s.list[at])) : 0;
      sum += w[i];
    }
    uint64_t before = prefix(sum, all, s);
    if (from == LIST) {
      want = (uint64_t)ceil((double)d.top_p * (double)all);
      want = want < 1 ? 1 : want < all ? want : all;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < want && before + w[i] >= want) s.value[0] = s.list[tid * PER + i];
      before += w[i];
    }
    __syncthreads();
    limit = d.top_p < 1.f ? s.value[0] : s.list[k - 1];
  }
  // the last of the first top_k, then of those the last of the nucleus
#pragma unroll 1
  for (int pass = sorts ? 2 : 0; pass < 2; ++pass) {
    uint64_t want = (uint64_t)k;
    if (pass == 0) {
      if (from == WIDE || (from == LIST && k >= (int64_t)found) || k >= V) continue;
    } else {
      if (d.top_p == 1.f) continue;
      if (from == WIDE) {
        want = border_of(a.wide[t - a.row0].bins, (double)d.top_p, s).left;
      } else {
        uint64_t sum = 0, all;
#pragma unroll 1
        for (int64_t at = (int64_t)tid * kEach;; at += kTile) {
          float z[kEach];
          if (from == ROW) load_tile<F32>(z, r.p, V, at);
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const uint64_t e = from == ROW ? (at + i < V ? entry_of(z[i], (uint32_t)(at + i)) : 0) : held[i];
            const uint64_t w = row_weight(r, entry_value(e));
            sum += e && e >= limit ? w : 0;
          }
          if (from != ROW || at + kTile - (int64_t)tid * kEach >= V) break;
        }
        prefix(sum, all, s);
        want = (uint64_t)ceil((double)d.top_p * (double)all);
        want = want < 1 ? 1 : want < all ? want : all;
      }
    }
    limit = last_of<F32>(held, from == ROW, r, limit, want, pass == 1, s);
  }

  // each tile's sum of the kept w: of the entries, of what the wide kernel summed and the entries, or of the row
  __syncthreads();
  for (int i = tid; i < tiles; i += kSelect) s.mass[i] = from == WIDE ? a.wide_mass[(t - a.row0) * tiles + i] : 0;
  __syncthreads();
  if (from == ROW) {
#pragma unroll 1
    for (int b = 0; b < tiles; ++b) {
      const int64_t at = (int64_t)b * kTile + tid * kEach;
      float z[kEach];
      uint64_t sum = 0;
      load_tile<F32>(z, r.p, V, at);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const uint64_t w = row_weight(r, z[i]);
        sum += (entry_of(z[i], (uint32_t)(at + i)) >= limit) & (w >= least) ? w : 0;
      }
      sum = wave_prefix(sum);
      if ((tid & 63) == 63 && sum) atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)sum);
    }
  } else if (from == LIST || d.top_p < 1.f) {
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
      if (!held[h] || held[h] < limit) continue;
      const uint64_t w = row_weight(r, entry_value(held[h]));
      if (w >= least) atomicAdd((unsigned long long*)&s.mass[entry_index(held[h]) / kTile], (unsigned long long)w);
    }
  }
  __syncthreads();
  // the tile in which the sum passes the target (one thread's share holds it; were it not so, tile 0 would be read), and the entry in the tile
  if (tid == 0) s.value[0] = s.value[1] = 0;
  const int per = (tiles + kSelect - 1) / kSelect, b0 = tid * per;
  uint64_t part = 0, total;
  for (int b = b0; b < b0 + per && b < tiles; ++b) part += s.mass[b];
  uint64_t x = prefix(part, total, s);
  const uint64_t target = target_of(d.u, total);
  if (x <= target && target < x + part)
    for (int b = b0; b < b0 + per && b < tiles; ++b) {
      if (target < x + s.mass[b]) {
        s.value[0] = b;
        s.value[1] = target - x;
        break;
      }
      x += s.mass[b];
    }
  __syncthreads();
  const int64_t at = (int64_t)s.value[0] * kTile + tid * kEach;
  const uint64_t want = s.value[1];
  float z[kEach];
  uint64_t w[kEach], mine = 0, all;
  load_tile<F32>(z, r.p, V, at);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    w[i] = row_weight(r, z[i]);
    w[i] = (entry_of(z[i], (uint32_t)(at + i)) >= limit) & (w[i] >= least) ? w[i] : 0;
    mine += w[i];
  }
  uint64_t y = prefix(mine, all, s);
  if (y <= want && want < y + mine) {
    bool done = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      y += w[i];
      if (y > want && !done) {
        answer(at + i, log_p(z[i], (double)total / r.one));
        done = true;
      }
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

// With wide kernels kWideRows rows at a time, which share what those leave.
template <bool F32>
static hipError_t sample(RowsArgs r, hipStream_t st) {
  hipError_t e = scan<F32, true>(r, st);
  if (e != hipSuccess) return e;
  const int64_t rows = r.wide ? kWideRows : r.T;
  for (r.row0 = 0; r.row0 < r.T; r.row0 += rows) {
    r.rows_end = r.row0 + rows < r.T ? r.row0 + rows : r.T;
    const int64_t n = r.rows_end - r.row0;
    if (r.wide) {
      const FlatGrid g = flat_grid(n * r.wide_parts);
      if (r.row0) {
        hipLaunchKernelGGL(wide_clear_kernel, dim3((uint32_t)n), dim3(256), 0, st, r);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
      if (r.top_p_rows || r.top_p < 1.f) {
        hipLaunchKernelGGL(sample_bins_kernel<F32>, dim3(g.x, g.y), dim3(kSelect), 0, st, r);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
      hipLaunchKernelGGL(sample_tiles_kernel<F32>, dim3(g.x, g.y), dim3(kSelect), 0, st, r);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(sample_select_kernel<F32>, dim3((uint32_t)n), dim3(kSelect), 0, st, r);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_sample(const RowsArgs& r, hipStream_t st) { return r.f32 ? sample<true>(r, st) : sample<false>(r, st); }

}  // namespace kd
