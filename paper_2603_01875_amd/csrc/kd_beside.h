// Host-side interface of what stands beside the losses: kd_blocks.hip (e4m3 in blocks), kd_rows.hip (rows of logits), kd_norm.hip
// (gradient norm), called by kd_beside_api.hip.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace kd {

// ---- e4m3 in blocks ----
struct BlocksArgs {
  const void* src;
  int64_t rows, cols, ld;
  int src_f32, tile;
  uint8_t *codes, *codes_t;
  float *scales, *scales_t;
};
hipError_t launch_quantize_blocks(const BlocksArgs& a, hipStream_t st);

struct ProductArgs {
  const uint8_t *a, *b;
  const float *a_scales, *b_scales;
  void* out;
  int64_t M, N, K;
  int out_f32, b_tile, accumulate;
  float* sums;                  // [product_parts][M][N], if that is more than one
  int parts;                    // (launch_product's own)
};
int product_parts(int64_t M, int64_t N, int64_t K, int out_f32);
hipError_t launch_product(const ProductArgs& p, hipStream_t st);
// whether a is so small that the product's workgroups quantise it themselves; p.a and p.a_scales are then not read
bool product_quantises(int64_t M, int64_t K);
hipError_t launch_linear_few(const ProductArgs& p, const void* x, int x_f32, hipStream_t st);

// ---- rows of logits ----
// A workgroup of the first kernel reads kRowThreads * per_thread entries of a row, a chunk.  Each thread leaves the largest key of its
// entries (a group), the workgroup the chunk's.
constexpr int kRowThreads = 256;
struct RowChunk {
  uint64_t sum;      // sampling: of w relative to the chunk's largest entry, in fixed point
  float part;        // top logits: the same in fp32
  uint32_t key;      // the largest entry's
};
// Sampling under top-p or min-p alone from rows of more than a list, kWideRows of them at a time: sums by bins, sums of tiles (kWideTile entries), and the
// entries of the bin in which the last kept one lies.
constexpr int kWideRows = 1024, kWideBins = 2048, kWideList = 4096, kWideTile = 4096;
struct RowWide {
  uint64_t bins[kWideBins], list[kWideList];
  uint32_t count, reserved[3];
};
struct RowsArgs {
  const void* logits;
  int64_t T, V, ld;
  int f32, index64;
  int per_thread, chunks;     // entries per thread; chunks per row
  float tau;                  // top logits; sampling: the temperature of all rows
  // top logits
  int K;
  void *top, *index;
  float* lse;
  // sampling
  const float *u, *temperature_rows, *top_p_rows, *min_p_rows;
  const int32_t* top_k_rows;
  int top_k;
  float top_p, min_p;
  void* token;
  float* logp;
  // workspace
  RowChunk* chunk;            // [T][chunks]
  uint32_t* group;            // [T][chunks * kRowThreads]
  RowWide* wide;              // [kWideRows at most], null unless the wide kernels are launched
  uint64_t* wide_mass;        // [kWideRows at most][tiles]
  int64_t row0, rows_end;     // rows of this launch
  int wide_parts;             // workgroups a row
};
hipError_t launch_top_logits(const RowsArgs& r, hipStream_t st);
hipError_t launch_sample(const RowsArgs& r, hipStream_t st);

// ---- gradient norm ----
constexpr int kGradsPerLaunch = 160;
constexpr int kNormGroups = 2048;      // workgroups of a launch
// Elements of a piece.  (Norm and clipped copy, us, each repeated by itself on arrays with allocations of their own, with 2048, 8192 and 32768: 3.2 million fp32 in 24 arrays 9.3 + 6.7, 7.3 + 6.1, 7.5 + 6.7; 30 million bf16 39 + 26,
// 17 + 22, 14 + 21; 1.7 billion 1802 + 1505, 587 + 1338, 573 + 1313: finding a piece's array costs as much as some thousand elements.)
constexpr int kPieceElements = 32768;
struct GradTable {
  int n;                               // arrays of this launch
  uint32_t chunks;                     // pieces of all arrays of this launch
  uint64_t in[kGradsPerLaunch];        // address, bit 0: fp32
  uint64_t count[kGradsPerLaunch];
  uint32_t first[kGradsPerLaunch];     // first piece of the array
};
struct ClipTable {
  GradTable t;
  uint64_t out[kGradsPerLaunch];       // address, bit 0: fp32
};
hipError_t launch_grad_norm(const GradTable& t, int max_norm_kind, double* partials, int groups, hipStream_t st);
hipError_t launch_grad_total(const double* partials, int64_t n, int max_norm_kind, double* total, hipStream_t st);
hipError_t launch_grad_clip(const ClipTable& t, int max_norm_kind, const double* total, double max_norm, float* norm, hipStream_t st);

}  // namespace kd
