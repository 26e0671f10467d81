// fp32 product of the linear layer, C[m][n] = sum_k A(m,k) B(n,k), with its epilogue.  The forms are
// those of the bf16 product: an operand lies with k contiguous ("row form") or with its row index
// contiguous ("transposed form").  Any sizes, any strides.
//
// What bounds it: the fp32 matrix rate, 256 flop per clock and CU, a sixteenth of bf16's.  A slice of 32
// k of a 128 x 128 tile is 4096 clocks of products against 32 KB to load and 64 KB of operands to
// read from LDS, so loads go through registers (no alignment asked for; rows past an edge are repeated, k past the
// end is zero), LDS holds two slices, and one barrier separates them.  The loads cost a seventh: 140 TFLOP/s without.
// v_mfma_f32_16x16x4_f32: lane (i16, gq) holds row i16 (column i16), k = gq.  Step s of 16 k takes k = 4 gq + s of both
// operands, so that a lane of a row-form operand reads its four steps at once.  n is on the matrix row axis:
// a lane ends up with four consecutive n of one row m, as in the bf16 product.  (4096^3: 124
// TFLOP/s, a library product 154; 2000 x 2048 x 768, 64 x 64 tiles: 63 us, 128 x 128 71.)
// LDS: row form [rows][32], 16-byte chunks permuted by (row / 2) % 8; transposed form [32 k][rows + 4] (the quarters of
// a wave, four k apart, lie 16 banks apart): no bank conflicts in either.
#include "epilogue.h"

#include <type_traits>

namespace mhffn {
namespace {

constexpr int kFK = 32, kFThreads = 256;
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct GemmF32Args {
  const float* A;      // m side
  const float* B;      // n side
  int64_t M, N, K, lda, ldb;
  int64_t tiles_n, n_items;
  int splits;
  int64_t k_per_split; // a multiple of kFK
};

template <bool TR, int ROWS>
struct OperandF32 {
  static constexpr int kLd = TR ? ROWS + 4 : kFK;
  static constexpr int kFloats = TR ? kFK * kLd : ROWS * kLd;
  static constexpr int kVecs = ROWS * kFK / 4 / kFThreads;   // 16-byte pieces per thread and slice
  // piece q of a thread: (row, k) of its first element
  static __device__ __forceinline__ void place(int q, int tid, int& row, int& k) {
    const int i = q * kFThreads + tid;
    if constexpr (TR) { k = i / (ROWS / 4); row = i % (ROWS / 4) * 4; }
    else { row = i / (kFK / 4); k = i % (kFK / 4) * 4; }
  }
  // Offsets of a thread's pieces from the tile's first element, in floats.  Rows past the edge repeat the last
  // piece (their products are never stored).
  static __device__ __forceinline__ void offsets(int64_t ld, int64_t rows, int tid, unsigned (&off)[kVecs]) {
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      int row, k;
      place(q, tid, row, k);
      const int64_t r = row < rows ? row : TR ? (rows - 1) & ~3 : rows - 1;
      off[q] = (unsigned)(TR ? k * ld + r : r * ld + k);
    }
  }
  // src: the tile's first element of this slice; rows, ks: how many rows and k of the slice exist
  static __device__ __forceinline__ void load(const float* src, const unsigned (&off)[kVecs], int64_t rows, int64_t ks, int tid, f32x4 (&v)[kVecs]) {
    const bool cut = TR && rows < ROWS && (rows & 3) != 0;   // the last piece of a k row is not whole
    if (ks >= kFK && !cut) {
#pragma unroll
      for (int q = 0; q < kVecs; ++q) v[q] = *reinterpret_cast<const f32x4_any*>(src + off[q]);
    } else if (ks >= kFK) {   // element by element, the last one repeated (no load waits for another)
#pragma unroll
      for (int q = 0; q < kVecs; ++q) {
        int row, k;
        place(q, tid, row, k);
        row = row < rows ? row : (int)(rows - 1) & ~3;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[q][j] = src[off[q] + min(j, (int)rows - 1 - row)];
      }
    } else {
#pragma unroll
      for (int q = 0; q < kVecs; ++q) {
        int row, k;
        place(q, tid, row, k);
        if (TR) row = row < rows ? row : (int)(rows - 1) & ~3;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[q][j] = (TR ? k < ks && row + j < rows : k + j < ks) ? src[off[q] + j] : 0.f;
      }
    }
  }
  static __device__ __forceinline__ void store(float* lds, int tid, const f32x4 (&v)[kVecs]) {
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      int row, k;
      place(q, tid, row, k);
      *reinterpret_cast<f32x4*>(lds + (TR ? k * kLd + row : row * kLd + (k ^ (((row >> 1) & 7) << 2)))) = v[q];
    }
  }
  // the four steps of k = 16 j .. 16 j + 15 of row `row`
  static __device__ __forceinline__ f32x4 read(const float* lds, int row, int j, int gq) {
    const int k = 16 * j + 4 * gq;
    if constexpr (TR) {
      f32x4 v;
#pragma unroll
      for (int s = 0; s < 4; ++s) v[s] = lds[(k + s) * kLd + row];
      return v;
    } else {
      return *reinterpret_cast<const f32x4*>(lds + row * kLd + (k ^ (((row >> 1) & 7) << 2)));
    }
  }
};

template <bool A_TR, bool B_TR, int TILE>
__device__ __forceinline__ void gemm_f32_tile(const GemmF32Args& a, Epilogue e, int64_t item, unsigned char* smem) {
  constexpr int W = TILE / 2, I = W / 16;     // four waves of W x W
  using OA = OperandF32<A_TR, TILE>;
  using OB = OperandF32<B_TR, TILE>;
  constexpr int kStage = OA::kFloats + OB::kFloats;
  float* const lds = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, gq = lane >> 4;
  const int split = (int)(item % a.splits);
  const int64_t tile = item / a.splits, m0 = tile / a.tiles_n * TILE, n0 = tile % a.tiles_n * TILE;
  const int64_t k0 = split * a.k_per_split, k1 = k0 + a.k_per_split < a.K ? k0 + a.k_per_split : a.K;
  const int wm = (wave >> 1) * W, wn = (wave & 1) * W;

  f32x4 acc[I][I];
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < I; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  unsigned oa[OA::kVecs], ob[OB::kVecs];
  OA::offsets(a.lda, a.M - m0, tid, oa);
  OB::offsets(a.ldb, a.N - n0, tid, ob);
  const float* const pa = a.A + (A_TR ? m0 : m0 * a.lda);
  const float* const pb = a.B + (B_TR ? n0 : n0 * a.ldb);
  f32x4 va[OA::kVecs], vb[OB::kVecs];
  auto load = [&](int64_t k) {
    OA::load(pa + (A_TR ? k * a.lda : k), oa, a.M - m0, k1 - k, tid, va);
    OB::load(pb + (B_TR ? k * a.ldb : k), ob, a.N - n0, k1 - k, tid, vb);
  };
  auto store = [&](int stage) {
    OA::store(lds + stage * kStage, tid, va);
    OB::store(lds + stage * kStage + OA::kFloats, tid, vb);
  };
  load(k0);
  store(0);
  __syncthreads();
  int stage = 0;
  for (int64_t k = k0; k < k1; k += kFK) {
    if (k + kFK < k1) load(k + kFK);
    const float* const la = lds + stage * kStage;
    const float* const lb = la + OA::kFloats;
    stage ^= 1;
#pragma unroll
    for (int j = 0; j < kFK / 16; ++j) {
      f32x4 fa[I], fb[I];
#pragma unroll
      for (int i = 0; i < I; ++i) {
        fa[i] = OA::read(la, wm + 16 * i + i16, j, gq);
        fb[i] = OB::read(lb, wn + 16 * i + i16, j, gq);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
          for (int n = 0; n < I; ++n)
            acc[n][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[n][s], fa[i][s], acc[n][i], 0, 0, 0);
    }
    if (k + kFK < k1) store(stage);
    __syncthreads();   // (everyone has read the slice that the next store overwrites)
  }
  if (a.splits > 1) e.Y = static_cast<float*>(e.Y) + split * a.M * e.ldy;   // partial sums
  wave_epilogue_by<float, I / 2, I / 2>(
      [&](auto IM_, unsigned char* piece) __attribute__((always_inline)) {
        constexpr int im = decltype(IM_)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int jn = 0; jn < I; ++jn) put_sums<I / 2>(piece, 16 * h + i16, 4 * jn + gq, acc[jn][2 * im + h]);
      },
      smem + wave * (32 * W * 4), m0 + wm, n0 + wn, lane, e);
}

template <bool A_TR, bool B_TR, int TILE>
__global__ __launch_bounds__(kFThreads, 2) void gemm_f32_kernel(GemmF32Args a, Epilogue e) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int64_t item = xcd_work_item(blockIdx.x, a.n_items);
  if (item < a.n_items) gemm_f32_tile<A_TR, B_TR, TILE>(a, e, item, smem);
}
// Two products of a backward at once, dW (both transposed) and dX (both row form): neither fills the chip
// with the three or four workgroups a CU that hide a slice's latency (us a backward, together | apart: 1500 x 1001 x 515 64 |
// 83, 1024 x 1024 x 1024 56 | 87, 2048 x 2048 x 2048 323 | 340).
constexpr int kPairTile = 64;
__global__ __launch_bounds__(kFThreads, 2) void gemm_f32_pair_kernel(GemmF32Args w, Epilogue ew, GemmF32Args x, Epilogue ex, unsigned grid_w) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  if (blockIdx.x < grid_w) {
    const int64_t item = xcd_work_item(blockIdx.x, w.n_items);
    if (item < w.n_items) gemm_f32_tile<true, true, kPairTile>(w, ew, item, smem);
  } else {
    const int64_t item = xcd_work_item(blockIdx.x - grid_w, x.n_items);
    if (item < x.n_items) gemm_f32_tile<false, false, kPairTile>(x, ex, item, smem);
  }
}

// Tile and split of the contraction.  The workgroups of a CU share its matrix rate: with n of them a slice takes
// kAlone + n kSlice microseconds (measured; what n hides is the latency of a slice), and 2 + n lie around the
// slices; the sum over the splits is a launch of 6 and 3 MB a us, written and read
// (2048^3: 157 us in 64 x 64 tiles, 168 in 128 x 128 with four splits).
struct F32Plan { int tile, splits; int64_t k_per_split; double cost; };
constexpr int kMostSplits = 16;
constexpr double kAlone[2] = {1.02, 0.42}, kSlice[2] = {1.88, 0.53};   // of tiles of 128, 64
int64_t tiles_of(int64_t M, int64_t N, int tile) { return ((M + tile - 1) / tile) * ((N + tile - 1) / tile); }
// k of a share if `want` of them make sense, else 0
int64_t share_of(int64_t K, int want) {
  const int64_t per = ((K + want - 1) / want + kFK - 1) / kFK * kFK;
  return want == 1 || (per >= 2 * kFK && (K + per - 1) / per == want) ? per : 0;
}
double sum_cost(int64_t M, int64_t N, int splits) { return splits > 1 ? 6 + (double)splits * M * N * 4 / 3e6 : 0; }
F32Plan plan_f32(int64_t M, int64_t N, int64_t K) {
  F32Plan best{128, 1, K, 0.0};
  for (int t = 0; t < 2; ++t) {
    const int tile = 128 >> t;
    const int64_t tiles = tiles_of(M, N, tile);
    for (int want = 1; want <= kMostSplits; ++want) {
      const int64_t per = share_of(K, want);
      if (!per || !launch_holds(tiles * want, kFThreads)) continue;
      const double n = (double)((tiles * want + 255) / 256);
      const double cost = (double)(per / kFK) * (kAlone[t] + kSlice[t] * n) + 2 + n + sum_cost(M, N, want);
      if (best.cost == 0.0 || cost < best.cost) best = {tile, want, per, cost};
    }
  }
  return best;
}
// The two products of a backward in one launch, by the longest share and the mean of the slices of a CU
struct F32Pair { bool worth; F32Plan x, w; };
F32Pair plan_f32_pair(int64_t M, int64_t N, int64_t K) {   // the layer's sizes
  const F32Plan x = plan_f32(M, K, N), w = plan_f32(K, N, M);
  F32Pair best{false, x, w};
  double least = x.cost + w.cost;
  const int64_t tx = tiles_of(M, K, kPairTile), tw = tiles_of(K, N, kPairTile);
  for (int sx = 1; sx <= kMostSplits; ++sx) {
    const int64_t px = share_of(N, sx);
    for (int sw = 1; px && sw <= kMostSplits; ++sw) {
      const int64_t pw = share_of(M, sw);
      if (!pw || !launch_holds(tx * sx + tw * sw, kFThreads)) continue;
      const double longest = (double)((px > pw ? px : pw) / kFK), mean = (double)(tx * sx * px + tw * sw * pw) / kFK / 256;
      const double cost = longest * kAlone[1] + (0.5 * longest + mean) * kSlice[1] + 2 + (double)(tx * sx + tw * sw) / 256 +
                          sum_cost(M, K, sx) + sum_cost(K, N, sw);
      if (cost < least) { least = cost; best = {true, {kPairTile, sx, px, cost}, {kPairTile, sw, pw, cost}}; }
    }
  }
  return best;
}

int64_t partial_ld(int64_t N) { return (N + 3) & ~(int64_t)3; }   // rows of 16-byte pieces

template <bool A_TR, bool B_TR, int TILE>
constexpr int lds_of() {
  constexpr int kStages = 2 * (OperandF32<A_TR, TILE>::kFloats + OperandF32<B_TR, TILE>::kFloats) * 4, kOut = 4 * 32 * (TILE / 2) * 4;
  return kStages > kOut ? kStages : kOut;
}
template <bool A_TR, bool B_TR, int TILE>
int launch_tile(const GemmF32Args& a, const Epilogue& e, hipStream_t stream) {
  constexpr int kLds = lds_of<A_TR, B_TR, TILE>();
  if (hipError_t e0 = LdsLimit<&gemm_f32_kernel<A_TR, B_TR, TILE>, kLds>::ensure(); e0 != hipSuccess) return (int)e0;
  hipLaunchKernelGGL((gemm_f32_kernel<A_TR, B_TR, TILE>), dim3((unsigned)xcd_grid_size(a.n_items)), dim3(kFThreads), kLds,
                     stream, a, e);
  return (int)hipGetLastError();
}
template <int TILE>
int launch_form(bool a_tr, bool b_tr, const GemmF32Args& a, const Epilogue& e, hipStream_t stream) {
  if (!a_tr && b_tr) return launch_tile<false, true, TILE>(a, e, stream);
  if (!a_tr && !b_tr) return launch_tile<false, false, TILE>(a, e, stream);
  if (a_tr && b_tr) return launch_tile<true, true, TILE>(a, e, stream);
  return -1;   // transposed A with row-form B: no caller
}

size_t partials(int64_t M, int64_t N, const F32Plan& p) {
  return p.splits > 1 ? (size_t)p.splits * M * partial_ld(N) * sizeof(float) : 0;
}
GemmF32Args args_of(const Product& p, const F32Plan& plan) {
  const int64_t tiles_n = (p.N + plan.tile - 1) / plan.tile;
  return {static_cast<const float*>(p.A), static_cast<const float*>(p.B), p.M, p.N, p.K, p.lda, p.ldb, tiles_n,
          (p.M + plan.tile - 1) / plan.tile * tiles_n * plan.splits, plan.splits, plan.k_per_split};
}
Epilogue epilogue_of(const Product& p, const F32Plan& plan, void* ws) {
  if (plan.splits == 1) return p.e;
  Epilogue e = {};
  e.Y = ws; e.ldy = partial_ld(p.N); e.M = p.M; e.N = p.N;
  return e;
}
LinearSums left_of(const Product& p, const F32Plan& plan, void* ws) {
  return plan.splits == 1 ? LinearSums{} : LinearSums{static_cast<float*>(ws), p.M, partial_ld(p.N), plan.splits};
}
std::string text_of(const F32Plan& p) {
  return std::to_string(p.tile) + "x" + std::to_string(p.tile) + " splits=" + std::to_string(p.splits);
}

}  // namespace

std::string linear_f32_plan(int64_t M, int64_t N, int64_t K) { return text_of(plan_f32(M, N, K)); }
std::string linear_f32_pair_plan(int64_t M, int64_t N, int64_t K) {
  const F32Pair p = plan_f32_pair(M, N, K);
  return "dX " + text_of(p.x) + (p.worth ? " with dW " : "; dW ") + text_of(p.w);
}

size_t linear_f32_workspace_bytes(int64_t M, int64_t N, int64_t K) { return partials(M, N, plan_f32(M, N, K)); }
bool linear_f32_pair(int64_t M, int64_t N, int64_t K, size_t& dX_bytes, size_t& dW_bytes) {
  const F32Pair p = plan_f32_pair(M, N, K);
  dX_bytes = partials(M, K, p.x);
  dW_bytes = partials(K, N, p.w);
  return p.worth;
}

int launch_linear_f32(const Product& p, void* ws, LinearSums& left, void* stream) {
  const F32Plan plan = plan_f32(p.M, p.N, p.K);
  const GemmF32Args a = args_of(p, plan);
  const Epilogue e = epilogue_of(p, plan, ws);
  left = left_of(p, plan, ws);
  hipStream_t st = static_cast<hipStream_t>(stream);
  return plan.tile == 128 ? launch_form<128>(p.a_tr, p.b_tr, a, e, st) : launch_form<64>(p.a_tr, p.b_tr, a, e, st);
}

int launch_linear_f32_pair(const Product& x, const Product& w, void* ws_x, void* ws_w, LinearSums& left_x, LinearSums& left_w,
                           void* stream) {
  constexpr int kLdsW = lds_of<true, true, kPairTile>(), kLdsX = lds_of<false, false, kPairTile>(), kLds = kLdsW > kLdsX ? kLdsW : kLdsX;
  const F32Pair plan = plan_f32_pair(x.M, x.K, x.N);
  const GemmF32Args aw = args_of(w, plan.w), ax = args_of(x, plan.x);
  const unsigned grid_w = w.e.Y ? (unsigned)xcd_grid_size(aw.n_items) : 0, grid_x = x.e.Y ? (unsigned)xcd_grid_size(ax.n_items) : 0;
  left_x = x.e.Y ? left_of(x, plan.x, ws_x) : LinearSums{};
  left_w = w.e.Y ? left_of(w, plan.w, ws_w) : LinearSums{};
  if (hipError_t e0 = LdsLimit<&gemm_f32_pair_kernel, kLds>::ensure(); e0 != hipSuccess) return (int)e0;
  hipLaunchKernelGGL(gemm_f32_pair_kernel, dim3(grid_w + grid_x), dim3(kFThreads), kLds, static_cast<hipStream_t>(stream), aw,
                     epilogue_of(w, plan.w, ws_w), ax, epilogue_of(x, plan.x, ws_x), grid_w);
  return (int)hipGetLastError();
}

}  // namespace mhffn
