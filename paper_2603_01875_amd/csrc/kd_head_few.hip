// Statistics of the one-head losses with few tokens (one token tile).  The head streams through once and nothing of it is shared, so
// what bounds these kernels is how much of it is in flight: a wave has 64 of a tile's 256 rows to itself and loads them straight into
// registers, R k-steps ahead; the tokens, 16 MB of them, go through the LDS for all four waves, as far ahead.  (Vector memory operations
// are waited for in order, so nothing may be issued with less lead than the rest.)
#include "kd_head.hpp"

namespace kd {

template <int MB_>
struct FewCfg {
  static constexpr int MB = MB_, NB = 4;
  static constexpr int R = 4;                        // k-steps of the head in flight; of the tokens one less
  static constexpr int BM = 16 * MB, BN = 256;       // tokens, rows of the head
  static constexpr int STAGE_BYTES = BM * 128, STAGES = R, A_LOADS = BM / 32;
  // behind the stages: [wave][token] max, sum, sum of logits; [token] next entry of the list, its place, the token; twice: which
  // rows are listed ([token][wave], 64 bits) and the place of the first of them
  static constexpr int SUMS_AT = STAGES * STAGE_BYTES, LIST_AT = SUMS_AT + 4 * 16 * BM, LISTED_AT = LIST_AT + 16 * BM, START_AT = LISTED_AT + 2 * 32 * BM;
  static constexpr int ALL_SMEM_BYTES = START_AT + 2 * 4 * BM;
  static_assert(ALL_SMEM_BYTES <= 160 * 1024, "LDS of a gfx950 CU");
};

struct FewArgs {
  HeadArgs h;
  TargetArgs t;            // labels are taken as they are, lists have been made of top logits
};

// A range of the vocabulary, in units of 32 rows, in tiles of 256.
struct FewItem { int n0, rows; };                      // first row, rows that exist
struct FewWork {
  int row0, row1;
  __device__ FewWork(const HeadArgs& a) {
    const int units = (a.V + 31) / 32, L = xcd_logical_id(blockIdx.x, gridDim.x);
    row0 = 32 * (int)((int64_t)L * units / gridDim.x);
    row1 = min(a.V, 32 * (int)((int64_t)(L + 1) * units / gridDim.x));
  }
  __device__ int n_items() const { return (row1 - row0 + 255) / 256; }
  __device__ FewItem item(int i) const { return FewItem{row0 + 256 * i, min(256, row1 - row0 - 256 * i)}; }
};

// epi.begin_item(item), T = all products of the tile (block MB j + i: rows 16 j of the wave's x tokens 16 i), epi.tile(item, T).
// A tile's k-steps are rounded up to whole groups of R, so that the ring's registers have fixed numbers; those behind the last load
// nothing (an offset past the buffer gives 0) and multiply tokens that are there with 0.
template <int MB, class Epi>
__device__ __forceinline__ void few_loop(const HeadArgs& a, const FewWork& work, Epi& epi, char* smem) {
  typedef FewCfg<MB> C;
  constexpr int R = C::R, NB = C::NB;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, frow = lane & 15;
  const int n_items = work.n_items(), nk = a.K >> 6, groups = (nk + R - 1) / R;
  // Rows are a power of two apart more often than not, and what all workgroups load at a time would lie behind the same few memory
  // channels: each starts at another k-step (H = 2048, V = 151936, T = 1 167 -> 131 us a call; H = 1024 and 4096 the same).
  const int turn = (int)(blockIdx.x * 3u % (uint32_t)nk);
  // tokens: direct load j of the workgroup fills bytes 4096 j .. of a stage; 128 bytes per token, its eight chunks permuted by row bits
  const rsrc_t ra = make_rsrc(a.h, (uint32_t)a.T * (uint32_t)a.K * 2u);
  uint32_t voff[C::A_LOADS];
  const int slot = threadIdx.x, lrow = slot >> 3, lchunk = (slot & 7) ^ ((lrow >> 1) & 7);
#pragma unroll
  for (int j = 0; j < C::A_LOADS; ++j) voff[j] = (uint32_t)min(lrow + 32 * j, a.T - 1) * (uint32_t)a.K * 2u + lchunk * 16;
  // the head: row 16 j + frow of the wave's, 16 bytes at k = 8 g of a sub-step
  uint32_t woff[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) woff[j] = (uint32_t)(16 * j + frow) * (uint32_t)a.ld * 2u + g * 16;
  rsrc_t rw;
  int l_item = 0, l_k = 0, t_k = 0;      // load cursors: of the head, of the tokens
  auto set_rows = [&](int i) {
    const FewItem it = work.item(min(i, n_items - 1));
    const int rows = i < n_items ? min(max(it.rows - 64 * wave, 0), 64) : 0;
    rw = make_rsrc(a.W + (int64_t)(it.n0 + min(64 * wave, it.rows)) * a.ld, (uint32_t)rows * (uint32_t)a.ld * 2u);
  };
  u32x4 W[R][2][NB];
  auto load_tokens = [&](int stage) {
    const int k = min(t_k, nk - 1), at = k + turn < nk ? k + turn : k + turn - nk;
#pragma unroll
    for (int j = 0; j < C::A_LOADS; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void_t*)(smem + stage * C::STAGE_BYTES + wave * 1024 + j * 4096), 16, voff[j], at * 128, 0, 0);
    t_k = t_k + 1 == groups * R ? 0 : t_k + 1;
  };
  auto load_rows = [&](u32x4 (&w)[NB], int s) {      // sub-step s of the cursor's k-step
    const int at = l_k >= nk ? (int)0x80000000 : (l_k + turn < nk ? l_k + turn : l_k + turn - nk) * 128;
#pragma unroll
    for (int j = 0; j < NB; ++j) w[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, woff[j] + s * 64, at, 0));
    if (s == 1 && ++l_k == groups * R) {
      l_k = 0;
      set_rows(++l_item);
    }
  };
  set_rows(0);
  static_for<0, R>([&](auto rc) {
    constexpr int r = decltype(rc)::value;
    load_rows(W[r][0], 0);
    load_rows(W[r][1], 1);
    if constexpr (r < R - 1) load_tokens(r);
  });
  const int fsw = (frow >> 1) & 7, fk0 = (g ^ fsw) << 4, fk1 = ((4 + g) ^ fsw) << 4;
  int stage = 0;
  const char* const frag = smem + frow * 128;
  for (int i = 0; i < n_items; ++i) {
    const FewItem it = work.item(i);
    epi.begin_item(it);
    f32x4 T[MB * NB];
#pragma unroll
    for (int e = 0; e < MB * NB; ++e) T[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    strip_settle<true, MB * NB>(T);
    for (int k = 0; k < groups; ++k)
      static_for<0, R>([&](auto rc) {
        constexpr int r = decltype(rc)::value;
        // this step's tokens have landed for every wave (issued since: rows, and R - 2 whole steps), and every wave has read the step
        // before, whose stage is refilled
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * NB + (R - 2) * (C::A_LOADS + 2 * NB)) : "memory");
        load_tokens(stage == 0 ? R - 1 : stage - 1);
        __builtin_amdgcn_sched_barrier(0);
        const char* const at = frag + stage * C::STAGE_BYTES;
        auto read = [&](int n) { return *(const u32x4*)(at + (n % MB) * 2048 + (n < MB ? fk0 : fk1)); };
        asm volatile("s_nop 1");           // whatever the compiler moved between steps, an MFMA may read now
        // (pinned: left to itself the compiler reads all fragments first and has no registers for them)
        u32x4 x[2] = {read(0), read(1)};
        static_for<0, 2 * MB>([&](auto nc) {
          constexpr int n = decltype(nc)::value, s = n / MB, m = n % MB;
          const u32x4 now = x[n & 1];
#pragma unroll
          for (int j = 0; j < NB; ++j)
            strip_mfma_a(T[MB * j + m], W[r][s][j], now);
          if constexpr (n + 2 < 2 * MB) x[n & 1] = read(n + 2);
          if constexpr (m == MB - 1) load_rows(W[r][s], s);
          __builtin_amdgcn_sched_barrier(0);
        });
        stage = stage == R - 1 ? 0 : stage + 1;
        __builtin_amdgcn_sched_barrier(0);
      });
    strip_settle<true, MB * NB>(T);
    epi.tile(it, T);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the loads issued past the end still target this workgroup's LDS
}

template <int MB, bool SMOOTH>
struct FewEpi {
  typedef FewCfg<MB> C;
  static constexpr int NV = SMOOTH ? 3 : 2;
  const HeadArgs& a;
  char* const smem;
  int lane, wave, flip, n_valid, panels;
  __device__ FewEpi(const FewArgs& k, char* s, int row0) : a(k.h), smem(s), lane(threadIdx.x & 63), wave(uniform(threadIdx.x >> 6)), flip(1) {
    n_valid = a.T;
    panels = (a.T + 63) >> 6;
    for (int i = threadIdx.x; i < 4 * C::BM; i += 256) *(f32x4*)(smem + C::SUMS_AT + 16 * i) = f32x4{M_FLOOR, 0.f, 0.f, 0.f};
    const int j = threadIdx.x;
    if (j >= C::BM) return;
    int next = kNoEntry, at = 0, token = 0;
    if (j < n_valid) {
      token = j;
      if (k.t.t.ce) {                        // (the first workgroup writes lists of them, for what comes later)
        const int y = blockIdx.x == 0 ? label_target(k.t, j) : label_row(k.t, j);
        if (y >= row0) next = y;
      } else {
        const int* const list = a.list + (int64_t)token * a.n_list;
        at = first_entry(list, a.n_list, row0);
        if (at < a.n_list) next = list[at];
      }
    }
    int* const own = (int*)(smem + C::LIST_AT) + 4 * j;
    own[0] = next; own[1] = at; own[2] = token;
  }
  // Thread i marks the listed rows of token i: bit 16 g + 4 j + r of word w for row 64 w + 16 j + 4 g + r.  All waves read them behind the
  // tile's k-steps, whose barriers lie between; the words of the tile before may still be read, so there are two sets.
  __device__ __forceinline__ void begin_item(const FewItem& it) {
    flip ^= 1;
    const int t = threadIdx.x;
    if (t >= C::BM) return;
    int* const own = (int*)(smem + C::LIST_AT) + 4 * t;
    uint32_t* const bits = (uint32_t*)(smem + C::LISTED_AT) + (flip * C::BM + t) * 8;
    *(u32x4*)bits = u32x4{0u, 0u, 0u, 0u};
    *(u32x4*)(bits + 4) = u32x4{0u, 0u, 0u, 0u};
    int next = own[0], at = own[1];
    ((int*)(smem + C::START_AT))[flip * C::BM + t] = at;
    const int end = it.n0 + it.rows;
    if (next < end) {
      const int* const list = a.list + (int64_t)own[2] * a.n_list;
      do {
        const int row = next - it.n0, e = 16 * ((row >> 2) & 3) + 4 * ((row >> 4) & 3) + (row & 3);
        bits[2 * (row >> 6) + (e >> 5)] |= 1u << (e & 31);
        ++at;
        next = at < a.n_list ? list[at] : kNoEntry;
      } while (next < end);
      own[0] = next; own[1] = at;
    }
  }
  // as HeadStatsEpi::take, for the 16 rows that a lane has of a token
  __device__ __forceinline__ void take(int n, uint32_t mine, float (&z)[16]) const {
    const int g = lane >> 4;
    while (__any(mine != 0)) {
      const int e = mine ? __builtin_ctz(mine) : 16;
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v = e == i ? z[i] : v;
        z[i] = e == i ? NEG_BIG : z[i];
      }
      if (mine) {
        const uint64_t* const words = (const uint64_t*)(smem + C::LISTED_AT) + (flip * C::BM + n) * 4;
        int rank = ((const int*)(smem + C::START_AT))[flip * C::BM + n];
        for (int w = 0; w < wave; ++w) rank += __popcll(words[w]);
        uint64_t below = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) below |= (uint64_t)((1u << (4 * (e >> 2) + (q < g ? 4 : q == g ? e & 3 : 0))) - 1) << (16 * q);
        rank += __popcll(words[wave] & below);
        a.z[(int64_t)n * a.n_list + rank] = v;
        mine &= mine - 1;
      }
    }
  }
  __device__ __forceinline__ void tile(const FewItem& it, f32x4 (&T)[4 * MB]) const {
    const int left = it.rows - 64 * wave, g = lane >> 4;
    if (left <= 0) return;
    static_for<0, MB>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      if (16 * i < n_valid) {
        const int n = 16 * i + (lane & 15);
        float z[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = T[MB * (e >> 2) + i][e & 3];
        if (left < 64)
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e] = 16 * (e >> 2) + 4 * g + (e & 3) < left ? z[e] : NEG_BIG;
        if (a.kept && (i >> 2) < panels) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
            if (32 * u < left) {
              f32x4* const to = (f32x4*)(a.kept + dz_chunk(a.ldz, i >> 2, (it.n0 >> 5) + 2 * wave + u, i & 3, lane));
              to[0] = f32x4{z[8 * u], z[8 * u + 1], z[8 * u + 2], z[8 * u + 3]};
              to[1] = f32x4{z[8 * u + 4], z[8 * u + 5], z[8 * u + 6], z[8 * u + 7]};
            }
        }
        const uint32_t mine = ((const uint16_t*)(smem + C::LISTED_AT))[((flip * C::BM + n) * 4 + wave) * 4 + g];
        if (__any(mine != 0)) {
          if (a.kept)                        // (they are there among the others)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = mine >> e & 1 ? NEG_BIG : z[e];
          else
            take(n, mine, z);
        }
        f32x4* const at = (f32x4*)(smem + C::SUMS_AT) + wave * C::BM + n;
        const f32x4 old = *at;
        float top = NEG_BIG;
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, z[e]);
        const float m = fmaxf(old[0], quad_max(top) * a.c);
        float s = 0.f, zs = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s += fexp2(fmaf(z[e], a.c, -m));
          if (SMOOTH) zs += counts_in(z[e]) ? z[e] : 0.f;
        }
        *at = f32x4{m, fmaf(old[1], fexp2(old[0] - m), quad_sum(s)), SMOOTH ? old[2] + quad_sum(zs) : 0.f, 0.f};
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  __device__ void write(int split) const {
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= C::BM) return;
    f32x4 v[4];
    float m = M_FLOOR, s = 0.f, zs = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      v[w] = *((const f32x4*)(smem + C::SUMS_AT) + w * C::BM + t);
      m = fmaxf(m, v[w][0]);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      s = fmaf(v[w][1], fexp2(v[w][0] - m), s);
      zs += v[w][2];
    }
    float* const p = a.partials + (int64_t)split * NV * a.T_pad + t;
    p[0] = m;
    p[a.T_pad] = s;
    if (SMOOTH) p[2 * a.T_pad] = zs;
  }
};

// Statistics (head_stats_kernel) of at most 128 tokens, each workgroup a range of the vocabulary.  Bound by memory: H = 1024, V = 151936 one
// token 61 us, 5.1 TB/s (by the strip loop 85), 128 tokens, whose logits are kept, 102 us, 3.8 TB/s of reads and stores (129); H = 2048,
// V = 128256, 48 tokens 101 us, 5.2 TB/s (129).  More than 128 tokens leave no registers for as many rows in flight: the strip loop is
// ahead there, or as fast.
template <int MB, bool SMOOTH>
KD_STRIP_KERNEL void head_few_kernel(const FewArgs k) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  FewWork work(k.h);
  FewEpi<MB, SMOOTH> epi(k, smem, work.row0);
  few_loop<MB>(k.h, work, epi, smem);
  epi.write(blockIdx.x);
}

hipError_t launch_head_few(const HeadProblem& h, hipStream_t st) {
  FewArgs a{head_args(h), target_args(h)};
  a.h.T = h.p.T;
  const bool smooth = h.t.smoothing > 0.f;
#define KD_FEW(MB) (smooth ? launch_big<head_few_kernel<MB, true>>(h.parts, 256, FewCfg<MB>::ALL_SMEM_BYTES, st, &a) \
                           : launch_big<head_few_kernel<MB, false>>(h.parts, 256, FewCfg<MB>::ALL_SMEM_BYTES, st, &a))
  static_assert(kFewHeadTokens == 128, "tokens of the larger one");
  return h.p.T <= 64 ? KD_FEW(4) : KD_FEW(8);
#undef KD_FEW
}

}  // namespace kd
