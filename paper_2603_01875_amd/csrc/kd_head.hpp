// The logit tiles of the one-head losses: work map and epilogues on the strip loop (kd_strip.hpp) with one accumulator.
//
// Both losses are a divergence of p = softmax(h W / tau) from a distribution q that lives on a short list of vocabulary entries per
// token (a label: one entry), beside a constant U elsewhere (label smoothing) or one more category for all the rest:
//   l = sum_list q (log q - log p) + r (log r - log p_rest) - U sum_v z + z_loss lse^2
//   dl/dz_v = A_in p_v - q_v - U on the list,  A_in p_v - r p_v / p_rest - U beside it
// The list is left out of the running sums of a tile and its logits are stored instead, so that p_rest is a sum of what lies beside
// the list and never a difference from 1 (which a student that is sure of the list would lose), and so that dl/dz on the list is
// written from fp32 values with one rounding.  Beside the list, where there is a rest, dl/dz is (A_in p_rest - r) 2^(z c - lse_rest): with the
// rest's own log-sum-exp both factors stay in a float's range, also where p_v and p_rest (by themselves) are far below it.
#pragma once
#include "kd_common.hpp"
#include "kd_logit_math.hpp"

namespace kd {

// 256 (vocabulary) x 256 (token) tiles: one accumulator leaves the registers for twice 128 rows.
struct HeadCfg : StripShape<kHeadRows / 16, 4> {
  static constexpr int HELD_V = 16, HELD_A = 12;     // (of two accumulators: unused)
  static constexpr int SHORT = 64;                   // a workgroup's last tile, if it has at most so many rows: see StripCfg
  // behind the stages: 32 bytes per token of what lasts from tile to tile, and 32 bytes per token of which rows of the tile are listed
  // ... and the entries of its list that come next
  static constexpr int AHEAD = 16;
  static constexpr int STATE_AT = SMEM_BYTES, LISTED_AT = STATE_AT + 32 * BN, NEXT_AT = LISTED_AT + 32 * BN;
  static constexpr int STATE_SMEM_BYTES = NEXT_AT + 4 * (AHEAD + 1) * BN;
  static_assert(STATE_SMEM_BYTES <= 160 * 1024, "LDS of a gfx950 CU");
};

struct HeadArgs {
  const bf16_t* W; const bf16_t* h;    // as the kernels read them
  int T, V, K, ld;         // K: contraction; ld: elements from row to row of the head; T: kd_head_few.hip only
  const int* meta;
  int v0, v_end;           // vocabulary rows of this launch
  int T_pad;
  float c;                 // log2(e) / tau
  int last_chunk;
  // statistics
  float* partials;         // [ranges][2, or 3 with the sum of the logits][T_pad]
  const int* rowmap;
  const int* list;         // Targets
  int n_list;
  float* z;
  float* kept;             // all logits, in the order of dz_chunk, where there are few enough (null otherwise)
  // gradient
  const f32x4* rowinfo;    // [T_pad]: {log-sum-exp (base 2), factor beside the list, U if there is label smoothing, else the logarithm (base 2) that
                           // goes with that factor: the log-sum-exp beside the list, if the teacher has a rest, or of all logits; A_in}
  bf16_t* dz;
  int ldz, sets;
};

struct TargetArgs {
  Targets t;
  int T, V;
  double inv_tau;
  int identity;            // few tokens: there is no row map; this launch writes that every token is its own row
  int *meta, *rowmap, *inv;
};

// What the row map leaves behind (make_rowmap, kd_kernels.hip), for tokens that all keep their places: inv says which count.
__device__ __forceinline__ void keep_places(const TargetArgs& a, int t, bool counts) {
  if (!a.identity) return;
  a.rowmap[t] = t;
  a.inv[t] = counts ? t : -1;
  if (t == 0) {
    a.meta[META_N_VALID] = a.T;
    a.meta[META_N_TT] = 1;
    a.meta[META_T_EFF] = (a.T + 63) / 64 * 64;
    a.meta[META_N_SPLIT] = a.meta[META_G_SPLIT] = a.meta[META_G_SPLIT_LAST] = 1;
  }
  for (int i = a.T + t; i < kTileN; i += a.T) a.rowmap[i] = a.T - 1;
}

// A label's entry, kNoEntry where there is none.  One past the vocabulary makes its token NaN: it is never read, and the loss says so.
__device__ __forceinline__ int64_t label_of(const TargetArgs& a, int t) {
  return a.t.index64 ? ((const int64_t*)a.t.index)[t] : (int64_t)((const int*)a.t.index)[t];
}
__device__ __forceinline__ int label_row(const TargetArgs& a, int t) {
  const int64_t y = label_of(a, t);
  return y >= 0 && y < a.V ? (int)y : kNoEntry;
}
// ... written down as what later kernels take
__device__ __forceinline__ int label_target(const TargetArgs& a, int t) {
  const int64_t y = label_of(a, t);
  const bool out = y >= a.V, counts = y >= 0 && (!a.t.mask || a.t.mask[t]);
  const int row = y >= 0 && !out ? (int)y : kNoEntry;
  a.t.valid[t] = counts;
  keep_places(a, t, counts);
  a.t.list[t] = row;
  a.t.q[t] = 1.f - a.t.smoothing;
  double* const info = a.t.info + (int64_t)t * kTargetInfo;
  info[0] = out ? __builtin_nan("") : 1.0;
  info[1] = info[2] = 0.0;
  info[3] = out ? 0.0 : 1.0 - (double)a.t.smoothing;
  return row;
}
TargetArgs target_args(const HeadProblem& h);  // kd_head.hip

// One workgroup: see StripWork (kd_logits.hpp), with tiles of four units.
template <bool HV>
struct HeadWork {
  const HeadArgs& a;
  int n_tt, tt, split, row0, row1, cnt, L, G, n_vt;
  __device__ HeadWork(const HeadArgs& a_, int n_split) : a(a_) {
    n_tt = meta_get(a.meta, META_N_TT);
    tt = split = row0 = row1 = cnt = L = n_vt = 0;
    G = 1;
    if (n_split == 0) {
      G = min((int)gridDim.x, kNumCU);
      n_vt = (a.v_end - a.v0 + HeadCfg::BM - 1) / HeadCfg::BM;
      if ((int)blockIdx.x >= G) return;
      L = xcd_logical_id(blockIdx.x, G);
      cnt = L < n_tt * n_vt ? (n_tt * n_vt - L + G - 1) / G : 0;
      return;
    }
    const int active = n_tt * n_split;               // the grid is sized for the unmasked worst case
    if ((int)blockIdx.x >= active) return;
    group_decode(xcd_logical_id(blockIdx.x, active), n_tt, n_split, tt, split);
    const int units = (a.v_end - a.v0 + 63) / 64;
    row0 = a.v0 + 64 * (int)(((int64_t)split * units) / n_split);
    row1 = min(a.v_end, a.v0 + 64 * (int)(((int64_t)(split + 1) * units) / n_split));
    cnt = (row1 - row0 + HeadCfg::BM - 1) / HeadCfg::BM;
  }
  __device__ int n_items() const { return cnt; }
  __device__ StripItem item(int i) const {
    const auto p = kernel_args<HeadArgs>();
    StripItem it;
    int m0 = row0 + i * HeadCfg::BM, n0 = tt * HeadCfg::BN, end = row1;
    if (n_vt > 0) {
      const int q = i * G + L, n_four = n_tt / 4, grp = q / (4 * n_vt), w = q - grp * 4 * n_vt;
      const int g = grp < n_four ? 4 : n_tt - 4 * n_four;
      const int vt = w / g;
      n0 = (4 * grp + w - vt * g) * HeadCfg::BN;
      m0 = p->v0 + vt * HeadCfg::BM;
      end = p->v_end;
    }
    it.a_rows = min(HeadCfg::BM, end - m0);
    it.out_rows = (it.a_rows + 63) / 64 * 64;
    it.m0 = m0;
    it.n0 = n0;
    it.k0 = it.k1 = p->K;
    it.lda0 = it.lda1 = 2 * p->ld;
    it.ldb0 = it.ldb1 = 128 * p->K;
    it.A0 = it.A1 = (const char*)p->W + (int64_t)m0 * (HV ? 2 : it.lda1);
    it.B0 = it.B1 = (const char*)p->h + (int64_t)n0 * (2 * p->K);
    it.aux = it.b_blocks = 0;
    return it;
  }
};

// First of `n` ascending entries that is not below `row`; sixteen probes a level, whose loads are in flight together.
__device__ __forceinline__ int first_entry(const int* list, int n, int row) {
  int at = 0;
  while (n > 0) {                          // the answer lies in at .. at + n
    const int step = (n + 15) >> 4;
    int below = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = i * step + step - 1, v = list[at + min(k, n - 1)];
      below += (int)(k < n) & (int)(v < row);
    }
    at += below * step;
    n = min(step - 1, n - below * step);
  }
  return at;
}

// Whether a logit is one of a row that exists beside the list: those of others are NEG_BIG, give or take a logit (kd_strip.hpp).  (What is
// lower still is: minus infinity counts.)
__device__ __forceinline__ bool counts_in(float z) { return !(fabsf(z - NEG_BIG) <= -0.9f * NEG_BIG); }

struct HeadGeo {
  int wave, lane;
  __device__ HeadGeo() : wave(threadIdx.x >> 6), lane(threadIdx.x & 63) {}
  __device__ __forceinline__ int n(int j) const { return HeadCfg::acc_n(j, lane, wave); }
};

// Running max and sum of what lies beside the lists, and the logits on them.  As in StripStatsEpi the state lives in LDS, [token][8]:
// max, sum, sum of logits; next entry of the list, its place in it, that place at the tile's start, the token.
// Which rows of the tile are listed: [token][4] words of 64 bits, bit 4 i + r of word g for row 16 i + 4 g + r, so that a lane finds
// its own rows in one word.  Thread i keeps the list of token i of the tile, which is its own wave's: no barrier.
// x, or the logit of what does not exist where bit B of `word` is set: the bit, spread over a word, picks one of the two.  (Pinned: with
// all of a column's words made at once they are spilled.)
template <int B>
__device__ __forceinline__ float left_out(float x, uint32_t word) {
  int32_t on;
  asm volatile("v_bfe_i32 %1, %2, %3, 1\n\tv_bfi_b32 %0, %1, %4, %0" : "+v"(x), "=&v"(on) : "v"(word), "n"(B), "v"(NEG_BIG));
  return x;
}

// KEPT: all logits are stored (HeadArgs::kept), so those on the lists need not be picked out: they are only taken out of the sums.
template <bool SMOOTH, bool KEPT>
struct HeadStatsEpi {
  static constexpr int NV = SMOOTH ? 3 : 2;
  HeadGeo geo;
  const HeadArgs& a;
  float* all;
  uint64_t* listed;
  int* ahead;              // [AHEAD][token]: entry k of the list in row k mod AHEAD; behind them the first that is not there
  __device__ HeadStatsEpi(const HeadArgs& a_, char* smem, int tt, int row0) : a(a_) {
    all = (float*)(smem + HeadCfg::STATE_AT);
    listed = (uint64_t*)(smem + HeadCfg::LISTED_AT);
    ahead = (int*)(smem + HeadCfg::NEXT_AT) + threadIdx.x;
    float* const own = all + threadIdx.x * 8;
    int* const owni = (int*)own;
    *(f32x4*)own = f32x4{M_FLOOR, 0.f, 0.f, 0.f};
    const int j = tt * HeadCfg::BN + threadIdx.x;
    int next = kNoEntry, at = 0, token = 0;
    if (j < meta_get(a.meta, META_N_VALID)) {
      token = a.rowmap[j];
      const int* const list = a.list + (int64_t)token * a.n_list;
      at = first_entry(list, a.n_list, row0);
      next = fetch(list, at);
    }
    owni[4] = next; owni[5] = owni[6] = at; owni[7] = token;
  }
  // Entries at .. of the list into the ring; the first of them.  (Read when it is needed, an entry costs a tile the time of a load and of
  // all that are in flight.)
  __device__ __forceinline__ int fetch(const int* list, int at) const {
    int v[HeadCfg::AHEAD];
#pragma unroll
    for (int i = 0; i < HeadCfg::AHEAD; ++i) v[i] = list[min(at + i, a.n_list - 1)];
#pragma unroll
    for (int i = 0; i < HeadCfg::AHEAD; ++i) ahead[((at + i) % HeadCfg::AHEAD) * HeadCfg::BN] = at + i < a.n_list ? v[i] : kNoEntry;
    ahead[HeadCfg::AHEAD * HeadCfg::BN] = at + HeadCfg::AHEAD;
    return at < a.n_list ? v[0] : kNoEntry;
  }
  __device__ __forceinline__ void begin_item(const StripItem& it) {
    int* const own = (int*)(all + threadIdx.x * 8);
    uint32_t* const bits = (uint32_t*)(listed + threadIdx.x * 4);
    *(u32x4*)bits = u32x4{0u, 0u, 0u, 0u};
    *(u32x4*)(bits + 4) = u32x4{0u, 0u, 0u, 0u};
    int next = own[4], at = own[5];
    own[6] = at;
    const int end = it.m0 + it.a_rows;
    if (next < end) {
      do {
        const int row = next - it.m0, e = 4 * (row >> 4) + (row & 3), g = (row >> 2) & 3;
        bits[2 * g + (e >> 5)] |= 1u << (e & 31);
        ++at;
        next = at < ahead[HeadCfg::AHEAD * HeadCfg::BN] ? ahead[(at % HeadCfg::AHEAD) * HeadCfg::BN]
                                                        : fetch(a.list + (int64_t)own[7] * a.n_list, at);
      } while (next < end);
      own[4] = next; own[5] = at;
    }
  }
  // Stores the logits of this lane's listed rows, one row a time, and takes them out of the tile.
  template <int NE>
  __device__ __forceinline__ void take(const StripItem& it, int n, uint64_t mine, float (&T)[NE]) {
    const int g = geo.lane >> 4;
    while (__any(mine != 0)) {
      const int e = mine ? __builtin_ctzll(mine) : 4096, block = e >> 2, r = e & 3;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < NE / 16; ++q)
        if (__any((e >> 4) == q)) {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const bool it = e == 16 * q + k;
            v = it ? T[16 * q + k] : v;
            T[16 * q + k] = it ? NEG_BIG : T[16 * q + k];
          }
        }
      if (mine) {
        int rank = ((const int*)all)[n * 8 + 6];       // entries of the list in front of this row
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int below = 4 * block + (w < g ? 4 : w == g ? r : 0);
          rank += __popcll(listed[n * 4 + w] & (below < 64 ? (1ull << below) - 1 : ~0ull));
        }
        a.z[(int64_t)(it.n0 + n) * a.n_list + rank] = v;
        mine &= mine - 1;
      }
    }
  }
  template <class J, int NE>
  __device__ __forceinline__ void column(const StripItem& it, J, float (&T)[NE]) {
    const int n = geo.n(J::value);
    if constexpr (KEPT) {
      const int64_t panel = uniform((it.n0 >> 6) + geo.wave);
      const rsrc_t to = make_rsrc(a.kept + panel * 64 * a.ldz, 256u * (uint32_t)a.ldz);
#pragma unroll
      for (int u = 0; u < NE / 8; ++u) {
        if (32 * u >= it.out_rows) break;
        const uint32_t sub = 8192u * (uint32_t)((it.m0 >> 5) + u) + 2048u * J::value;      // (as dz_chunk, elements of four bytes)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{T[8 * u], T[8 * u + 1], T[8 * u + 2], T[8 * u + 3]}), to, 32 * geo.lane, sub, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{T[8 * u + 4], T[8 * u + 5], T[8 * u + 6], T[8 * u + 7]}), to, 32 * geo.lane + 16, sub, 0);
      }
    }
    const uint64_t mine = listed[n * 4 + (geo.lane >> 4)];
    float* const at = all + n * 8;
    const f32x4 old = *(const f32x4*)at;
    // logit(IntC<e>): entry e of the column, as it counts
    auto add = [&](auto&& logit) {
      float top = NEG_BIG;
      static_for<0, NE>([&](auto ec) { top = fmaxf(top, logit(ec)); });
      const float m = fmaxf(old[0], quad_max(top) * a.c);
      float s = 0.f, zs = 0.f;
      static_for<0, NE>([&](auto ec) {
        const float z = logit(ec);
        s += fexp2(fmaf(z, a.c, -m));
        if (SMOOTH) zs += counts_in(z) ? z : 0.f;
      });
      *(f32x4*)at = f32x4{m, fmaf(old[1], fexp2(old[0] - m), quad_sum(s)), SMOOTH ? old[2] + quad_sum(zs) : 0.f, 0.f};
    };
    if constexpr (KEPT) {
      if (__any(mine != 0)) {                // (taken out twice: a column that has been changed does not stay in accumulation registers)
        const uint32_t half[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
        add([&](auto ec) { return left_out<decltype(ec)::value & 31>(T[decltype(ec)::value], half[decltype(ec)::value >> 5]); });
        return;
      }
    } else {
      if (__any(mine != 0)) take(it, n, mine, T);
    }
    add([&](auto ec) { return T[decltype(ec)::value]; });
  }
  __device__ void write(int tt, int split) {
    const float* const own = all + threadIdx.x * 8;
    float* p = a.partials + (int64_t)split * NV * a.T_pad + tt * HeadCfg::BN + threadIdx.x;
#pragma unroll
    for (int i = 0; i < NV; ++i) p[(int64_t)i * a.T_pad] = own[i];
  }
};

// Eight neighbours of dL/dz (beside the lists) to `to` and, in parts, to the copies of the token axis, `stride` elements apart.
template <int PARTS>
__device__ __forceinline__ void store_dz(float (&x)[8], bf16_t* to, int64_t stride, int sets) {
  if constexpr (PARTS == 1) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16_t)x[e];
    *(bf16x8*)to = o;
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = (bf16_t)x[e];
        x[e] -= (float)o[e];
      }
      const int first = sets == 3 ? q : q == 0 ? 0 : q == 1 ? 3 : 5, n = sets == 3 ? 1 : 3 - q;
      for (int s = 0; s < n; ++s) *(bf16x8*)(to + (first + s) * stride) = o;
    }
  }
}
// (a token of zeros beside infinite weights: 0 x infinity is NaN, and the larger of that and a number the number.  A token that counts
// keeps its NaN through the factor.)
__device__ __forceinline__ float unlisted_dz(float factor, float base, float z, float c, float u) {
  return fmaf(factor, fexp2(fmaxf(fmaf(z, c, -base), -1.0e38f)), -u);
}

__device__ __forceinline__ float listed_dz(const f32x4& ri, float z, float c, float q, float u) {
  return fmaf(ri[3], fexp2(fmaxf(fmaf(z, c, -ri[0]), -1.0e38f)), -q) - u;
}

// dL/dz of a tile beside the lists, without its common factor (Targets::scale), in bf16 (PARTS 1), or as three bf16 parts that hold 24 bits,
// each in the copies of the token axis that multiply it (`sets`: 3, parts 0 1 2; 6, parts 0 0 0 1 1 2).  What is listed is written over
// by head_listed_kernel.  Rows that do not exist give 0; panels of 64 tokens without a valid one are left out.
template <bool SMOOTH, int PARTS>
struct HeadGradEpi {
  HeadGeo geo;
  const HeadArgs& a;
  f32x4* info;
  int n0, panels;
  __device__ HeadGradEpi(const HeadArgs& a_, char* smem) : a(a_), n0(-1) {
    info = (f32x4*)(smem + HeadCfg::STATE_AT);
    panels = meta_get(a.meta, META_T_EFF) >> 6;
  }
  __device__ __forceinline__ void begin_item(const StripItem& it) {
    if (n0 != it.n0) info[threadIdx.x] = a.rowinfo[it.n0 + threadIdx.x];
    n0 = it.n0;
  }
  template <class J, int NE>
  __device__ __forceinline__ void column(const StripItem& it, J, float (&T)[NE]) {
    constexpr int j = J::value;
    const int panel = (it.n0 >> 6) + geo.wave, m0 = it.m0 - a.v0;
    if (panel >= panels) return;
    const f32x4 ri = info[geo.n(j)];
#pragma unroll
    for (int p = 0; p < NE / 16; ++p) {
      if (64 * p >= it.out_rows) break;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = T[16 * p + 8 * u + e];
          x[e] = SMOOTH ? unlisted_dz(ri[1], ri[0], z, a.c, counts_in(z) ? ri[2] : 0.f) : unlisted_dz(ri[1], ri[2], z, a.c, 0.f);
        }
        store_dz<PARTS>(x, a.dz + dz_chunk(a.ldz, panel, (m0 >> 5) + 2 * p + u, j, geo.lane), (int64_t)panels * 64 * a.ldz, a.sets);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Drives an epilogue from strip_loop.
template <class Epi>
struct HeadDrive {
  static constexpr bool WHOLE = false;
  Epi& epi;
  __device__ HeadDrive(Epi& e) : epi(e) {}
  __device__ __forceinline__ void begin_item(const StripItem& it) { epi.begin_item(it); }
  __device__ float pad(int) const { return NEG_BIG; }
  template <class J, int NM>
  __device__ __forceinline__ void column(const StripItem& it, J jc, f32x4 (&)[NM], f32x4 (&T4)[NM]) {
    float T[4 * NM];
#pragma unroll
    for (int e = 0; e < 4 * NM; ++e) T[e] = T4[e >> 2][e & 3];
    epi.column(it, jc, T);
  }
};

HeadArgs head_args(const HeadProblem& h);      // kd_head.hip

// Statistics: per token max and sum of e^(z/tau) beside the list, and sum z.  A workgroup has one token tile and a range of the vocabulary,
// so that a token's running sums stay in its LDS and partial sums leave once a range.  Bound by the matrix pipe (T = 4096, 15 tiles computed,
// H = 1024, V = 151936: 866 us, 1.38 PFLOP/s beside 2.3 TB/s; with lists of 64 1004 us, of which the difference is taking their logits out,
// one listed row of a lane at a time), with one token tile by memory as much (T = 200, H = 2048, V = 151936, storing the logits: 206 us, 649 MB
// read and 156 written, 3.9 TB/s, and 0.77 PFLOP/s on the whole tile).
template <bool HV, bool SMOOTH, bool KEPT>
KD_STRIP_KERNEL void head_stats_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  HeadWork<HV> work(a, meta_get(a.meta, META_N_SPLIT));
  HeadStatsEpi<SMOOTH, KEPT> epi(a, smem, work.tt, work.row0);
  HeadDrive<HeadStatsEpi<SMOOTH, KEPT>> drive(epi);
  strip_loop<1, true, HeadCfg, HV ? A_KMAJOR_DZ : A_ROWS>(work, drive, smem);
  if (work.cnt > 0) epi.write(work.tt, work.split);
}

// dL/dz of a chunk: the logits again, four token tiles by all of the chunk's rows at a time, so that the head's come from L2.  Bound by the
// matrix pipe, and by a tile's stores, for which its one wave per SIMD waits (the same size: 1048 us in five chunks, 1.15 PFLOP/s).
template <bool HV, bool SMOOTH, int PARTS>
KD_STRIP_KERNEL void head_grad_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  HeadWork<HV> work(a, meta_get(a.meta, a.last_chunk ? META_G_SPLIT_LAST : META_G_SPLIT));
  HeadGradEpi<SMOOTH, PARTS> epi(a, smem);
  HeadDrive<HeadGradEpi<SMOOTH, PARTS>> drive(epi);
  strip_loop<1, false, HeadCfg, HV ? A_KMAJOR_DZ : A_ROWS>(work, drive, smem);
}

}  // namespace kd
