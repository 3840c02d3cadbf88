// Product of two matrices of e4m3 in blocks (kd_matmul_e4m3, kd_linear_e4m3):
//   out[m][n] = sum_j a_scale[m][j] b_scale[n or n / 128][j] sum_{k in block j} a[m][k] b[n][k]
//
// Rows of b are the register axis of the matrix instructions, rows of a the lane axis, so that a lane has one a's scale.
// A bf16 result takes the e4m3 pipe (16x16x128: one instruction is one block's sum).  That pipe aligns the products of a group of eight to the
// largest of them and cuts off what lies 2^-13 below: 1.5e-5 of a result of normal numbers, nothing beside its rounding to bf16
// (1.7e-3), but not what fp32 stands for.  An fp32 result takes the codes to bf16, which holds them exactly, and the bf16 pipe at
// half the rate (CUT false).
#include <hip/hip_runtime.h>

#include "kd_beside.h"
#include "kd_blocks.hpp"
#include "kd_common.hpp"
#include "kd_launch.h"
#include "kd_unaligned.hpp"

namespace kd {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// eight codes as bf16
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A lane's 32 codes of a row as the matrix instructions take them.
template <bool CUT> struct Codes { i32x8 v; };
template <> struct Codes<false> { bf16x8 v[4]; };
template <bool CUT>
__device__ __forceinline__ Codes<CUT> codes_from(const u32x4& lo, const u32x4& hi) {
  Codes<CUT> c;
  if constexpr (CUT) {
    c.v = __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    c.v[0] = widen(lo[0], lo[1]);
    c.v[1] = widen(lo[2], lo[3]);
    c.v[2] = widen(hi[0], hi[1]);
    c.v[3] = widen(hi[2], hi[3]);
  }
  return c;
}
// sum over a block of 16 rows by 16 rows
template <bool CUT>
__device__ __forceinline__ f32x4 block_product(const Codes<CUT>& x, const Codes<CUT>& y) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  if constexpr (CUT) {
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.v, y.v, c, 0, 0, 0, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[i], y.v[i], c, 0, 0, 0);
  }
  return c;
}

// four results of one row m, columns n .. n + 3 (at most N), as a lane has them
__device__ __forceinline__ void store4(const ProductArgs& p, int64_t m, int64_t n, f32x4 v) {
  const int64_t at = m * p.N + n;
  if (n + 4 <= p.N) {
    if (p.out_f32) {
      const global_t o = (global_t)((float*)p.out + at);
      if (p.accumulate) {
        const u32x4_t w = load16((const float*)p.out + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(w[i]);
      }
      store16(o, u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    } else {
      const global_t o = (global_t)((uint16_t*)p.out + at);
      if (p.accumulate) {
        const u32x2_t w = ((const Bytes8*)((uint16_t*)p.out + at))->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += bf16_float((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
      }
      store8(o, u32x2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])});
    }
    return;
  }
  for (int i = 0; i < 4 && n + i < p.N; ++i) {
    if (p.out_f32) {
      float* const o = (float*)p.out + at + i;
      *o = v[i] + (p.accumulate ? *o : 0.f);
    } else {
      uint16_t* const o = (uint16_t*)p.out + at + i;
      *o = bf16_bits(v[i] + (p.accumulate ? bf16_float(*o) : 0.f));
    }
  }
}

// 16 bytes of results of row m from column n on, as far as they are in the matrix
template <bool F32>
__device__ __forceinline__ void store_row(const ProductArgs& p, int64_t m, int64_t n, u32x4_t v) {
  constexpr int VE = F32 ? 4 : 8;
  if (m >= p.M || n >= p.N) return;
  const global_t o = (global_t)p.out + (m * p.N + n) * (F32 ? 4 : 2);
  if (n + VE <= p.N) {
    store16(o, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    if (n + i >= p.N) break;
    if (F32) ((KD_GLOBAL uint32_t*)o)[i] = v[i % 4];
    else ((KD_GLOBAL uint16_t*)o)[i] = (uint16_t)(v[i / 2 % 4] >> (16 * (i & 1)));
  }
}

// ------------------------------------------------------------------------------------------------
// tiles
//
// (K in parts: a workgroup does its part of one tile and leaves fp32 sums, which product_join_kernel adds in the parts' order.)
// WN x WM waves, each with NB x MB blocks of 16 x 16 results.  A k-step is one block of 128: the tile's rows of b and a, 128 bytes each, and
// their scales, loaded straight into LDS while the step before is multiplied (two stages).  16-byte chunks of a row are permuted by
// XOR with bits of its number, and a lane takes chunks g and g + 4 (which of a block's codes an instruction contracts together does not
// matter), so that the lanes that LDS serves at once read from different banks, in whichever order it takes them.  (Chunks 2 g and 2 g + 1: 25 k of 137 k
// cycles in conflicts.)  4096 x 4096 x 4096 with scales by tiles of b 65 us, 2.1 PFLOP/s, of 2.5 for a library product of 8192^3 with one scale; by rows of b, where each result
// has a product of two scales to make, 81; 4096 x 151936 x 4096 2370 us; fp32 results 4096 x 4096 x 4096 135 us, 1.0 PFLOP/s.
// ------------------------------------------------------------------------------------------------
template <int NB_, int MB_, int WN_, int WM_>
struct ProductTile {
  static constexpr int NB = NB_, MB = MB_, WN = WN_, WM = WM_, NT = 64 * WN * WM, BN = 16 * NB * WN, BM = 16 * MB * WM;
  static constexpr int LOAD_ROWS = NT / 8;                                  // rows of one 16-byte load a thread
  static constexpr int N_LOADS = BN / LOAD_ROWS, M_LOADS = BM / LOAD_ROWS;
  static constexpr int SCALES = BN + BM, SCALE_LOADS = (SCALES + NT - 1) / NT;
  static constexpr int STAGE = (BN + BM) * 128 + SCALE_LOADS * NT * 4;
  static constexpr int OUT_ROW = 144, OUT = 16 * OUT_ROW, SMEM = 2 * STAGE + WN * WM * OUT;      // OUT: where a wave turns results into rows
  static_assert(BN % LOAD_ROWS == 0 && BM % LOAD_ROWS == 0 && LOAD_ROWS % 16 == 0, "whole loads, one permutation a thread");
  static_assert(SMEM <= 160 * 1024, "LDS");
};

// Tile number q: rows of a in panels of 16 tiles, a panel's rows of b in strips of eight tiles, a strip four by eight after four by eight
// (group_decode).  32 numbers, the workgroups of an XCD, so share what they load through its L2, and 256 of them, all workgroups,
// 16 + 16 tiles' rows through the last-level cache: a b of any size comes from memory once for 4096 rows of a.
__device__ __forceinline__ void tile_of(int q, int n_mt, int n_nt, int& tm, int& tn) {
  const int panel = q / (16 * n_nt), m_first = panel * 16, m = n_mt - m_first < 16 ? n_mt - m_first : 16;
  q -= panel * 16 * n_nt;
  const int strip = q / (8 * m), n_first = strip * 8, n = n_nt - n_first < 8 ? n_nt - n_first : 8;
  group_decode(q - strip * 8 * m, m, n, tm, tn);
  tm += m_first;
  tn += n_first;
}

// The tile that comes `round` rounds of the grid after a workgroup's first: its rows and what loads them.
template <class Tile>
struct TileRows {
  int64_t n0, m0;
  rsrc_t b, a, scales;      // scales: of b's or of a's rows, by the wave
};

template <class Tile, bool CUT, bool B_TILE>
__device__ __forceinline__ void product_tiles(const ProductArgs& p, char* smem) {
  constexpr int NB = Tile::NB, MB = Tile::MB, NT = Tile::NT, BN = Tile::BN, BM = Tile::BM;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wn = wave % Tile::WN, wm = wave / Tile::WN;
  const int l = lane & 15, g = lane >> 4;
  const int n_mt = (int)((p.M + BM - 1) / BM), n_nt = (int)((p.N + BN - 1) / BN), tiles = n_mt * n_nt;
  const int ld = (int)((p.K + 15) / 16 * 16), nk = (int)((p.K + 127) / 128);
  const int part = blockIdx.x % p.parts, grid = gridDim.x / p.parts, part_steps = (nk + p.parts - 1) / p.parts, k0 = part * part_steps;
  const int last = nk - k0 < part_steps ? nk - k0 : part_steps, steps = last < 2 ? 2 : last;      // (behind nk: 0; a part that is not the last has two)
  const int my = xcd_logical_id(blockIdx.x / p.parts, grid), mine = (tiles - my + grid - 1) / grid;      // (the grid is not larger)
  const bool b_scales = wave * 64 < BN;
  static_assert(BN % 64 == 0 && Tile::SCALE_LOADS == 1, "a wave loads scales of one matrix");

  auto rows_of = [&](int round) {
    TileRows<Tile> r;
    int tm, tn;
    tile_of(my + round * grid, n_mt, n_nt, tm, tn);
    r.n0 = (int64_t)tn * BN;
    r.m0 = (int64_t)tm * BM;
    const int64_t n = p.N - r.n0 < BN ? p.N - r.n0 : BN, m = p.M - r.m0 < BM ? p.M - r.m0 : BM;
    r.b = make_rsrc(p.b + r.n0 * ld, (uint32_t)(n * ld));
    r.a = make_rsrc(p.a + r.m0 * ld, (uint32_t)(m * ld));
    if (b_scales) r.scales = make_rsrc(p.b_scales + (B_TILE ? r.n0 / 128 : r.n0) * nk, (uint32_t)((B_TILE ? (n + 127) / 128 : n) * nk * 4));
    else r.scales = make_rsrc(p.a_scales + r.m0 * nk, (uint32_t)(m * nk * 4));
    return r;
  };

  // Loads of a step: thread tid has chunk tid % 8 (as stored) of rows tid / 8 + j LOAD_ROWS.  Rows behind the matrix and chunks behind a row's
  // end are 0, and so are scales behind either.
  constexpr uint32_t BEHIND = 0x80000000u;
  const int row = tid >> 3, chunk = (tid & 7) ^ ((row >> 1) & 7);
  const uint32_t at = (uint32_t)row * ld + chunk * 16, step = (uint32_t)Tile::LOAD_ROWS * ld;
  const int scale_row = b_scales ? (B_TILE ? tid / 128 : tid) : tid - BN;
  const uint32_t scale_at = scale_row < (b_scales ? BN : BM) ? (uint32_t)scale_row * (nk * 4) : BEHIND;
  auto load = [&](int stage, const TileRows<Tile>& r, int step_k) {
    const int k = k0 + step_k;
    char* const to = smem + stage * Tile::STAGE + wave * 1024;
    const uint32_t from = at | (k * 128 + chunk * 16 < ld ? 0u : BEHIND);
#pragma unroll
    for (int j = 0; j < Tile::N_LOADS; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r.b, (lds_void_t*)(to + j * (NT * 16)), 16, from + j * step, k * 128, 0, 0);
#pragma unroll
    for (int j = 0; j < Tile::M_LOADS; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r.a, (lds_void_t*)(to + BN * 128 + j * (NT * 16)), 16, from + j * step, k * 128, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r.scales, (lds_void_t*)(smem + stage * Tile::STAGE + (BN + BM) * 128 + wave * 256), 4,
                                             scale_at | (k < nk ? 0u : BEHIND), k * 4, 0, 0);
  };

  f32x4 acc[NB][MB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int sw = (l >> 1) & 7, c0 = (g ^ sw) * 16, c1 = ((g + 4) ^ sw) * 16;
  auto read = [&](const char* rows, int block) {
    const char* const r = rows + (block * 16 + l) * 128;
    return codes_from<CUT>(*(const u32x4*)(r + c0), *(const u32x4*)(r + c1));
  };
  // What a step multiplies by: codes and scales of the wave's rows of a, and 16 rows of b after the other.
  Codes<CUT> y[MB], x[2];
  float s[MB], s_next[MB];
  constexpr int PRODUCTS = NB * MB, LATE = 3, TS = MB - 1 + LATE < 2 * MB ? 2 : 4;      // TS: a block's scales stay until its last result is added
  static_assert(NB % TS == 0 && MB - 1 + LATE < TS * MB, "places of t");
  f32x4 t[TS];
  auto read_a = [&](const char* base, int j) {
    const float* const scales = (const float*)(base + (BN + BM) * 128);
    y[j] = read(base + BN * 128 + wm * (MB * 16 * 128), j);
    s_next[j] = scales[BN + wm * (MB * 16) + j * 16 + l];
    if (B_TILE) s_next[j] *= scales[wn * (NB * 16)];
  };
  auto read_b = [&](const char* base, int i) { x[i & 1] = read(base + wn * (NB * 16 * 128), i); };
  auto read_t = [&](const char* base, int i) {
    if (!B_TILE) t[i % TS] = *(const f32x4*)((const float*)(base + (BN + BM) * 128) + wn * (NB * 16) + i * 16 + 4 * g);
  };
  // A product's result is scaled and added three products later, so that nothing waits for the matrix pipe.
  static_assert(NB % 2 == 0 && PRODUCTS % 4 == 0 && PRODUCTS > 4, "places of x and c");
  f32x4 c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < TS; ++i) t[i] = c[0];
  auto add = [&](int q) {
    const int i = q / MB, j = q % MB;
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(c[q & 3][r], B_TILE ? s[j] : s[j] * t[i % TS][r], acc[i][j][r]);
  };

  int stage = 0;
  // One step; the loads of the one after the next go where it was.
  auto multiply = [&](const TileRows<Tile>& r, int k_load) {
    const char* const base = smem + stage * Tile::STAGE;
    const char* const next = smem + (stage ^ 1) * Tile::STAGE;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (i < NB - 1) {
        if (i) read_t(base, i);
      } else {
        // the step's last rows: all of it has been read, and the next one has landed
        read_t(base, i);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        load(stage, r, k_load);
        read_b(next, 0);
      }
#pragma unroll
      for (int j = 0; j < MB; ++j) {
        const int q = i * MB + j;
        c[q & 3] = block_product<CUT>(x[i & 1], y[j]);
        add((q + PRODUCTS - LATE) % PRODUCTS);
        if (q == LATE - 1) {
#pragma unroll
          for (int n = 0; n < MB; ++n) s[n] = s_next[n];
          read_t(base, 0);
        }
        if (i == NB - 1) read_a(next, j);
        else if (j == 0) read_b(base, i + 1);
        __builtin_amdgcn_sched_barrier(0);             // (in this order: a place is free once it is used)
      }
    }
    stage ^= 1;
  };

  TileRows<Tile> rows = rows_of(0);
  load(0, rows, 0);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  load(1, rows, 1);
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    read_a(smem, j);
    s[j] = 0.f;
  }
  read_b(smem, 0);
  for (int round = 0; round < mine; ++round) {
    for (int k = 2; k < steps; ++k) multiply(rows, k);
    const int64_t n0 = rows.n0, m0 = rows.m0;
    if (round + 1 < mine) rows = rows_of(round + 1);   // (behind the last tile its own first steps again)
    multiply(rows, 0);
    multiply(rows, 1);
#pragma unroll
    for (int q = PRODUCTS - LATE; q < PRODUCTS; ++q) {
      add(q);
      c[q & 3] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // (what the next tile's first sums add is 0 times these, which may be NaN)
#pragma unroll
    for (int j = 0; j < MB; ++j) s[j] = 0.f;
#pragma unroll
    for (int i = 0; i < TS; ++i) t[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (p.accumulate || p.parts > 1) {
      ProductArgs to = p;
      if (p.parts > 1) {
        to.out = p.sums + part * p.M * p.N;
        to.out_f32 = 1;
        to.accumulate = 0;
      }
#pragma unroll
      for (int j = 0; j < MB; ++j)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int64_t m = m0 + wm * (MB * 16) + j * 16 + l, n = n0 + wn * (NB * 16) + i * 16 + 4 * g;
          if (m < p.M && n < p.N) store4(to, m, n, acc[i][j]);
        }
    } else {
      // 16 rows at a time through LDS, so that 128 bytes of a row go out together (32 at a time, as a lane has them, cost 340 of 2520 us
      // at T = 4096, H = 4096, V = 151936)
      constexpr int BLOCKS = CUT ? 4 : 2, VE = CUT ? 8 : 4;
      char* const turn = smem + 2 * Tile::STAGE + wave * Tile::OUT;
      const int64_t m = m0 + wm * (MB * 16) + (lane >> 3), n = n0 + wn * (NB * 16) + (lane & 7) * VE;
#pragma unroll
      for (int j = 0; j < MB; ++j)
#pragma unroll
        for (int h = 0; h < NB; h += BLOCKS) {
#pragma unroll
          for (int i = 0; i < BLOCKS; ++i) {
            const f32x4& v = acc[h + i][j];
            if (CUT) *(u32x2_t*)(turn + l * Tile::OUT_ROW + i * 32 + g * 8) = u32x2_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            else *(f32x4*)(turn + l * Tile::OUT_ROW + i * 64 + g * 16) = v;
          }
#pragma unroll
          for (int r = 0; r < 2; ++r)
            store_row<!CUT>(p, m + j * 16 + r * 8, n + h * 16, *(const u32x4_t*)(turn + ((lane >> 3) + 8 * r) * Tile::OUT_ROW + (lane & 7) * 16));
        }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (loads behind the end still write to this workgroup's LDS)
}

template <class Tile, bool CUT, bool B_TILE>
__global__ __launch_bounds__(Tile::NT) void product_tile_kernel(const ProductArgs p) {
  extern __shared__ __attribute__((aligned(128))) char smem[];
  product_tiles<Tile, CUT, B_TILE>(p, smem);
}

// out = the parts' sums one after the other, four columns a thread
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void product_join_kernel(const ProductArgs p) {
  const int64_t quads = (p.N + 3) / 4, i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x, m = i / quads, n = (i - m * quads) * 4;
  if (m >= p.M) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int part = 0; part < p.parts; ++part) {
    const float* const from = p.sums + (part * p.M + m) * p.N + n;
    if (n + 4 <= p.N) {
      const u32x4_t w = load16(from);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] += __uint_as_float(w[r]);
    } else {
      for (int r = 0; n + r < p.N; ++r) v[r] += from[r];
    }
  }
  store4(p, m, n, v);
}

template <class Tile> static int64_t tiles_of(int64_t M, int64_t N) { return (M + Tile::BM - 1) / Tile::BM * ((N + Tile::BN - 1) / Tile::BN); }
template <class Tile> constexpr int kResident = 160 * 1024 / Tile::SMEM * kNumCU;      // workgroups

template <class Tile, bool CUT>
static hipError_t launch_tiles(ProductArgs p, hipStream_t st, int parts = 1) {
  const int64_t tiles = tiles_of<Tile>(p.M, p.N);
  if (tiles > INT32_MAX / 2) return hipErrorInvalidValue;
  p.parts = parts;
  const int grid = parts * (tiles < kResident<Tile> ? (int)tiles : kResident<Tile>);
  void* args = &p;
  const hipError_t e = p.b_tile ? launch_big<product_tile_kernel<Tile, CUT, true>>(grid, Tile::NT, Tile::SMEM, st, args)
                                : launch_big<product_tile_kernel<Tile, CUT, false>>(grid, Tile::NT, Tile::SMEM, st, args);
  if (e != hipSuccess || parts == 1) return e;
  product_join_kernel<<<dim3((unsigned)((p.M * ((p.N + 3) / 4) + kJoinThreads - 1) / kJoinThreads)), dim3(kJoinThreads), 0, st>>>(p);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// few rows of a (at most 16 MB)
//
// b is read once, straight into registers, each wave 16 rows of it and a lane 32 codes of a block at a time; a's codes lie in LDS,
// quantised by the workgroup itself where they are few (QUANT).  WK of the workgroup's eight waves share the blocks of 16 rows of b
// and join their sums through LDS in a fixed order.  Bound by memory: 1 x 151936 x 4096 113 us, 5.5 TB/s; 16 rows 130; 8 x 1024 x 1024, where it waits for
// one load after the other, 5.6.
// ------------------------------------------------------------------------------------------------
constexpr int kFewWaves = 8, kFewBlocks = 4;      // waves; blocks of b that a wave has in flight
constexpr int kFewSmem = 128 * 1024;              // most LDS
struct FewArgs {
  ProductArgs p;
  const void* x;                                  // QUANT: a in bf16 or fp32
  int x_f32, wk;
};
inline int64_t few_row(int64_t K) { return (K + 127) / 128 * 128 + 16; }      // (16 rows' reads of a chunk fall into different banks)
inline int64_t few_smem(int64_t M, int64_t K, int mb) {
  const int64_t blocks = (K + 127) / 128, codes = M * few_row(K), scales = (M * blocks * 4 + 15) / 16 * 16;
  return codes + scales + kFewWaves * mb * 1024;
}

template <int MB, bool CUT, bool B_TILE, bool QUANT>
__global__ __launch_bounds__(64 * kFewWaves) void product_few_kernel(const FewArgs f) {
  extern __shared__ __attribute__((aligned(128))) char smem[];
  const ProductArgs& p = f.p;
  constexpr int NT = 64 * kFewWaves, U = kFewBlocks;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l = lane & 15, g = lane >> 4;
  const int M = (int)p.M, ld = (int)((p.K + 15) / 16 * 16), nk = (int)((p.K + 127) / 128), row = nk * 128 + 16;
  char* const codes = smem;
  float* const scales = (float*)(smem + M * row);
  char* const joined = smem + M * row + (M * nk * 4 + 15) / 16 * 16;
  if (QUANT) {
    // 16 lanes a block of 128, eight values each
    for (int i = tid / 16; i < M * nk; i += NT / 16) {
      const int m = i / nk, j = i - m * nk, c = j * 128 + (tid & 15) * 8;
      float x[8];
      if (f.x_f32) load_row8<true>(x, (const float*)f.x + (int64_t)m * p.K, c, p.K);
      else load_row8<false>(x, (const uint16_t*)f.x + (int64_t)m * p.K, c, p.K);
      uint32_t top = kLeastBlock;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, magnitude(x[e]));
      top = row_max(top);
      const Divisor d = divisor_of(top);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = quotient<true>(x[e], d);
      *(uint2*)(codes + m * row + c) = codes_of(x);
      if ((tid & 15) == 0) scales[i] = scale_of(top);
    }
  } else {
    for (int i = tid; i < M * nk * 8; i += NT) {
      const int m = i / (nk * 8), c = (i - m * nk * 8) * 16;
      *(u32x4_t*)(codes + m * row + c) = c < ld ? *(const u32x4_t*)(p.a + (int64_t)m * ld + c) : u32x4_t{0, 0, 0, 0};
    }
    for (int i = tid; i < M * nk; i += NT) scales[i] = p.a_scales[i];
  }
  __syncthreads();

  const int wk = f.wk, wn = kFewWaves / wk, my_k = wave % wk, my_n = wave / wk;
  const int64_t groups = (p.N + 15) / 16;
  const int64_t group = (int64_t)blockIdx.x * wn + my_n;
  const int64_t n0 = (group < groups ? group : groups - 1) * 16;
  const uint8_t* const b = p.b + (n0 + l < p.N ? n0 + l : p.N - 1) * ld + g * 16;
  const float* const sb = p.b_scales + (B_TILE ? n0 / 128 : n0) * nk;
  const int parts = (nk + U - 1) / U;
  f32x4 acc[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 next[2 * U];
  auto fetch = [&](int part) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (part * U + u) * 128 + h * 64;
        next[2 * u + h] = k + g * 16 < ld ? *(const u32x4*)(b + k) : u32x4{0, 0, 0, 0};
      }
  };
  int a_row[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) a_row[i] = i * 16 + l < M ? i * 16 + l : M - 1;
  fetch(my_k < parts ? my_k : parts - 1);
  for (int part = my_k; part < parts; part += wk) {
    u32x4 now[2 * U];
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) now[u] = next[u];
    if (part + wk < parts) fetch(part + wk);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = part * U + u;
      if (k >= nk) break;
      const Codes<CUT> x = codes_from<CUT>(now[2 * u], now[2 * u + 1]);
      f32x4 t;
      if (!B_TILE)
#pragma unroll
        for (int r = 0; r < 4; ++r) t[r] = sb[(n0 + 4 * g + r < p.N ? 4 * g + r : 0) * nk + k];
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const char* const a = codes + a_row[i] * row + k * 128 + g * 16;
        const f32x4 c = block_product<CUT>(x, codes_from<CUT>(*(const u32x4*)a, *(const u32x4*)(a + 64)));
        float s = scales[a_row[i] * nk + k];
        if (B_TILE) s *= sb[k];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][r] = fmaf(c[r], B_TILE ? s : s * t[r], acc[i][r]);
      }
    }
  }
  if (wk > 1) {
    f32x4* const to = (f32x4*)joined;
#pragma unroll
    for (int i = 0; i < MB; ++i) to[(wave * MB + i) * 64 + lane] = acc[i];
    __syncthreads();
    if (my_k) return;
    for (int w = 1; w < wk; ++w)
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const f32x4 v = to[((wave + w) * MB + i) * 64 + lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][r] += v[r];
      }
  }
  if (group >= groups) return;
#pragma unroll
  for (int i = 0; i < MB; ++i)
    if (i * 16 + l < M && n0 + 4 * g < p.N) store4(p, i * 16 + l, n0 + 4 * g, acc[i]);
}

template <int MB, bool CUT>
static hipError_t launch_few_of(const FewArgs& f, int grid, int smem, hipStream_t st) {
  void* args = const_cast<FewArgs*>(&f);
  if (f.x) return launch_big<product_few_kernel<MB, CUT, true, true>>(grid, 64 * kFewWaves, smem, st, args, kFewSmem);
  return f.p.b_tile ? launch_big<product_few_kernel<MB, CUT, true, false>>(grid, 64 * kFewWaves, smem, st, args, kFewSmem)
                    : launch_big<product_few_kernel<MB, CUT, false, false>>(grid, 64 * kFewWaves, smem, st, args, kFewSmem);
}

static hipError_t launch_few(const ProductArgs& p, const void* x, int x_f32, hipStream_t st) {
  const int mb = p.M <= 16 ? 1 : 2;
  const int64_t groups = (p.N + 15) / 16;
  // As many waves to 16 rows of b as there are kFewBlocks blocks for; where workgroups are many (more than four a CU), as leave each wave four times that.
  // (1 x 151936 x 4096 with one, two, four and eight: 119, 113, 113, 125 us; 16 rows of a 140, 130, 142, 173; 8 x 151936 x 2048 56, 60, 71, 71;
  // 8 x 40000 x 4096 with two and eight 31 and 38.)
  int wk = kFewWaves;
  while (wk > 1 && ((groups * wk > 4 * kNumCU * kFewWaves && wk * 4 * kFewBlocks * 128 > p.K) || (wk / 2) * kFewBlocks * 128 >= p.K)) wk >>= 1;
  const FewArgs f{p, x, x_f32, wk};
  const int wn = kFewWaves / wk, grid = (int)((groups + wn - 1) / wn), smem = (int)few_smem(p.M, p.K, mb);
  if (mb == 1) return p.out_f32 ? launch_few_of<1, false>(f, grid, smem, st) : launch_few_of<1, true>(f, grid, smem, st);
  return p.out_f32 ? launch_few_of<2, false>(f, grid, smem, st) : launch_few_of<2, true>(f, grid, smem, st);
}

// (us as few rows and in tiles, bf16 results: 1 x 4096 x 4096 5.5 and 10.2, 16 8.1 and 10.7, 24 10.2 and 11.0; 32 x 20000 x 1024 8.9 and 7.5, 32 x 512 x 3000 12 and 14.5,
// 24 x 151936 x 2048 65 and 100)
bool product_is_few(int64_t M, int64_t K) { return M <= 32 && few_smem(M, K, M <= 16 ? 1 : 2) <= kFewSmem; }
// (every workgroup anew, or a launch in front: 1 x 4096 x 4096 6.0 and 7.5, 4 x 4096 x 4096 7.3 and 7.8, 8 x 4096 x 4096 10.6 and 8.9, 8 x 151936 x 4096 138 and 131)
bool product_quantises(int64_t M, int64_t K) { return product_is_few(M, K) && M * K <= 16384; }
hipError_t launch_linear_few(const ProductArgs& p, const void* x, int x_f32, hipStream_t st) { return launch_few(p, x, x_f32, st); }

using TileBig = ProductTile<8, 4, 2, 4>;        // 256 x 256
using TileMid = ProductTile<4, 4, 2, 2>;        // 128 x 128
using TileSmall = ProductTile<4, 2, 2, 2>;      // 64 rows of a x 128 of b

// At 4096 x 4096 x 4096 (bf16 results, us) 256 x 256 takes 65, 128 x 128 87 and 64 x 128 102; but a CU wants a tile: 2048 x 4096 x 4096
// takes 64, 45 and 57.  128 x 128 pays with two tiles a CU, as many as fit, and where 64 x 128 would not save rows: two of those
// take 1.25 times as long (fp32 results: 4096 x 4096 x 4096 135 and 168; 777 x 5003 x 1008 23.7 and 20.1; 300 x 1000 x 4096 41 and 27).
static bool takes_big(int64_t M, int64_t N, int out_f32) { return !out_f32 && tiles_of<TileBig>(M, N) >= kNumCU; }
static bool takes_mid(int64_t M, int64_t N) {
  const int64_t mid = tiles_of<TileMid>(M, N);
  return mid >= kResident<TileMid> && 8 * mid <= 5 * tiles_of<TileSmall>(M, N);
}

// Few tiles of many steps: K in parts, workgroups of their own, with eight steps or more each.  (us with one part, with this many and with parts of four steps:
// 256 x 4096 x 16384 98, 51, 51 for fp32 and 67, 35, 35 for bf16 results; 48 x 4096 x 4096 27, 14, 15; 300 x 1000 x 4096 27, 16, 18;
// 1024 x 1024 x 1024 12, 12, 15: the join is a launch.)
int product_parts(int64_t M, int64_t N, int64_t K, int out_f32) {
  if (product_is_few(M, K) || takes_big(M, N, out_f32) || takes_mid(M, N)) return 1;
  const int64_t tiles = tiles_of<TileSmall>(M, N), nk = (K + 127) / 128;
  int parts = 1;
  while (parts < 16 && 2 * parts * tiles <= kResident<TileSmall> && nk >= 16 * parts) parts *= 2;
  return parts;
}

hipError_t launch_product(const ProductArgs& p, hipStream_t st) {
  if (product_is_few(p.M, p.K)) return launch_few(p, nullptr, 0, st);
  if (takes_big(p.M, p.N, p.out_f32)) return launch_tiles<TileBig, true>(p, st);
  if (takes_mid(p.M, p.N)) return p.out_f32 ? launch_tiles<TileMid, false>(p, st) : launch_tiles<TileMid, true>(p, st);
  const int parts = product_parts(p.M, p.N, p.K, p.out_f32);
  return p.out_f32 ? launch_tiles<TileSmall, false>(p, st, parts) : launch_tiles<TileSmall, true>(p, st, parts);
}

}  // namespace kd
