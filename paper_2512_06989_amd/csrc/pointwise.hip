// Kernels of the linear layer and of dropout that touch every element once: the epilogue over
// partial products, dZ with the sums of its columns, dropout alone, and operands packed for the
// product.  All of them move pieces of eight columns (epilogue.h) and are bound by memory.
#include "epilogue.h"

namespace mhffn {
namespace {

constexpr int kThreads = kSumThreads;

// A thread's pieces of a [rows][cols] array, in row order: piece -> (row, first column)
struct Pieces {
  int64_t total;      // rows * per_row
  uint32_t per_row;
  Divisor div;
};
Pieces make_pieces(int64_t rows, int64_t cols) {
  const uint32_t per = (uint32_t)((cols + 7) / 8);
  return {rows * (int64_t)per, per, make_divisor(per ? per : 1)};
}
__device__ __forceinline__ void piece_at(const Pieces& p, int64_t i, int64_t& row, int64_t& col) {
  row = p.total <= 0xFFFFFFFFll ? (int64_t)divide((uint32_t)i, p.div) : i / p.per_row;
  col = 8 * (i - row * p.per_row);
}
// (a launch holds fewer than 2^32 threads: past that a thread takes several pieces)
unsigned piece_blocks(int64_t pieces) {
  const int64_t blocks = (pieces + kThreads - 1) / kThreads;
  return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
}

template <typename T>
__device__ __forceinline__ void linear_sum(const LinearSums& s, const Epilogue& e, const Pieces& p, int64_t i, const DropKey& key) {
  int64_t row, col;
  piece_at(p, i, row, col);
  const int cols = (int)(s.ldp - col < 8 ? s.ldp - col : 8);
  float v[8];
  load8(s.P + row * s.ldp + col, cols, v);
  for (int k = 1; k < s.splits; ++k) {
    float w[8];
    load8(s.P + ((int64_t)k * s.rows + row) * s.ldp + col, cols, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
  }
  epilogue8<T>(v, row, col, e, key);
}
// What one or two products left (pieces of the first, then of the second), and in the first `blocks_c` workgroups sums of columns
template <typename T>
__global__ __launch_bounds__(kSumThreads) void linear_sums_kernel(LinearSums a, Epilogue ea, Pieces pa, LinearSums b, Epilogue eb, Pieces pb,
                                                                  ColumnSums c, unsigned blocks_c) {
  __shared__ float sums[kSumThreads];
  if (blockIdx.x < blocks_c) {
    column_sums<T>(c, blockIdx.x, sums);
    return;
  }
  const DropKey key = drop_key(ea.drop);   // (the second is a gradient: no dropout)
  for (int64_t i = (int64_t)(blockIdx.x - blocks_c) * kThreads + threadIdx.x; i < pa.total + pb.total;
       i += (int64_t)(gridDim.x - blocks_c) * kThreads) {
    if (i < pa.total) linear_sum<T>(a, ea, pa, i, key);
    else linear_sum<T>(b, eb, pb, i - pa.total, DropKey{});
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* X, int64_t ldx, Epilogue e, Pieces p) {
  const DropKey key = drop_key(e.drop);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < p.total; i += (int64_t)gridDim.x * kThreads) {
    int64_t row, col;
    piece_at(p, i, row, col);
    float v[8];
    load8(X + row * ldx + col, (int)(e.N - col < 8 ? e.N - col : 8), v);
    epilogue8<T>(v, row, col, e, key);
  }
}

// One launch packs both operands of a product: pieces of the first, then of the second
template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackJob a, Pieces pa, PackJob b, Pieces pb) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < pa.total + pb.total; i += (int64_t)gridDim.x * kThreads) {
    const bool first = i < pa.total;
    const PackJob& j = first ? a : b;
    int64_t row, col;
    piece_at(first ? pa : pb, first ? i : i - pa.total, row, col);
    Raw8<T> v = {};
    if (row < j.rows && col < j.cols) v = load_raw8(static_cast<const T*>(j.src) + row * j.ld + col, (int)(j.cols - col < 8 ? j.cols - col : 8));
    store_raw8(static_cast<T*>(j.dst) + row * j.cols_to + col, (int)(j.cols_to - col < 8 ? j.cols_to - col : 8), v);
  }
}

// dZ is rounded to the storage type, as the operand of two products (in bf16: the MFMA's operand; the columns' sums take it
// unrounded).  The dropout's scale is left to the products' sums: without an activation, or with relu, dZ is dY or 0 and
// the rounding costs nothing; with a slope it is a second rounding of the gradients (bf16, GELU: 2.35e-3 of their norm in place of 1.66e-3;
// products of both halves of a split dZ would cost twice the matrix time).
// Lane t of a workgroup takes piece column t % lanes of rows t / lanes, + rows_at_once, ..: the
// workgroup's share of dZ, and the sums of its eight columns per lane, which meet in LDS in row
// order and go out as one partial sum per column and row block.
struct DzGrid {
  int lane_shift;        // log2 of the piece columns a workgroup spans
  int64_t pieces;        // piece columns, padding of dZ among them
  int64_t rows_per_block;
};
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_dz_kernel(LinearDz a, DzGrid g) {
  __shared__ float sums[kThreads * 8];
  const DropKey key = drop_key(a.drop);
  const int lanes = 1 << g.lane_shift, at_once = kThreads >> g.lane_shift;
  const int lane = threadIdx.x & (lanes - 1), first = threadIdx.x >> g.lane_shift;
  const int64_t piece = (int64_t)blockIdx.x * lanes + lane, col = 8 * piece;
  const int64_t r0 = (int64_t)blockIdx.y * g.rows_per_block;
  const int64_t r1 = r0 + g.rows_per_block < a.M ? r0 + g.rows_per_block : a.M;
  const int64_t per_row = (a.N + 7) >> 3;
  const int cols = (int)(a.N - col < 8 ? a.N - col : 8);   // (0 or less: padding)
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (piece < g.pieces) {
    for (int64_t row = r0 + first; row < r1; row += at_once) {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (cols > 0) {
        load8(static_cast<const T*>(a.dY) + row * a.ldy + col, cols, v);
        if (a.act) {
          float z[8];
          load8(static_cast<const T*>(a.Z) + row * a.N + col, cols, z);
          slope8<T>(v, z, a.act);
        }
        drop8(v, (uint64_t)row * per_row + piece, a.drop, key, 1.f);   // (last: a dropped element may hold anything in Z and dY)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
      }
      if (a.dZ) store8(static_cast<T*>(a.dZ) + row * a.ldz + col, (int)(a.ldz - col < 8 ? a.ldz - col : 8), v);
    }
  }
  if (!a.dbias) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[threadIdx.x * 8 + j] = acc[j];
  __syncthreads();
  for (int t = threadIdx.x; t < 8 * lanes; t += kThreads) {
    float sum = 0.f;
    for (int k = 0; k < at_once; ++k) sum += sums[k * 8 * lanes + t];
    const int64_t c = (int64_t)blockIdx.x * 8 * lanes + t;
    if (c < a.N) a.partials[(int64_t)blockIdx.y * a.N + c] = sum * a.drop.scale;
  }
}

DzGrid dz_grid(int64_t M, int64_t N, int64_t cols_to) {
  DzGrid g;
  g.pieces = ((cols_to > N ? cols_to : N) + 7) / 8;
  g.lane_shift = 0;
  while (g.lane_shift < 5 && (1 << g.lane_shift) < (N + 7) / 8) ++g.lane_shift;
  const int64_t blocks = linear_column_blocks(M, N);
  g.rows_per_block = (M + blocks - 1) / blocks;
  return g;
}

}  // namespace

int64_t linear_column_blocks(int64_t M, int64_t N) {
  const int64_t across = (N + 255) / 256, want = 2048 / across > 1 ? 2048 / across : 1;
  const int64_t most = (M + 7) / 8;
  return most < want ? (most > 0 ? most : 1) : want;
}

int launch_linear_sums(int dtype, const LinearSums& a, const Epilogue& ea, const LinearSums& b, const Epilogue& eb,
                       const ColumnSums& c, void* stream) {
  const Pieces pa = a.splits ? make_pieces(ea.M, ea.N) : make_pieces(0, 0), pb = b.splits ? make_pieces(eb.M, eb.N) : make_pieces(0, 0);
  const unsigned blocks_c = column_sum_blocks(c), blocks = piece_blocks(pa.total + pb.total);
  if (blocks_c + blocks == 0) return 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == 1)
    hipLaunchKernelGGL(linear_sums_kernel<uint16_t>, dim3(blocks_c + blocks), dim3(kSumThreads), 0, st, a, ea, pa, b, eb, pb, c, blocks_c);
  else
    hipLaunchKernelGGL(linear_sums_kernel<float>, dim3(blocks_c + blocks), dim3(kSumThreads), 0, st, a, ea, pa, b, eb, pb, c, blocks_c);
  return (int)hipGetLastError();
}

int launch_dropout(int dtype, const void* X, int64_t ldx, const Epilogue& e, void* stream) {
  const Pieces p = make_pieces(e.M, e.N);
  if (p.total == 0) return 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == 1)
    hipLaunchKernelGGL(dropout_kernel<uint16_t>, dim3(piece_blocks(p.total)), dim3(kThreads), 0, st,
                       static_cast<const uint16_t*>(X), ldx, e, p);
  else
    hipLaunchKernelGGL(dropout_kernel<float>, dim3(piece_blocks(p.total)), dim3(kThreads), 0, st,
                       static_cast<const float*>(X), ldx, e, p);
  return (int)hipGetLastError();
}

int launch_pack(int dtype, const PackJob& a, const PackJob& b, void* stream) {
  const Pieces pa = make_pieces(a.rows_to, a.cols_to), pb = make_pieces(b.rows_to, b.cols_to);
  if (pa.total + pb.total == 0) return 0;
  const dim3 grid(piece_blocks(pa.total + pb.total));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == 1) hipLaunchKernelGGL(pack_kernel<uint16_t>, grid, dim3(kThreads), 0, st, a, pa, b, pb);
  else hipLaunchKernelGGL(pack_kernel<float>, grid, dim3(kThreads), 0, st, a, pa, b, pb);
  return (int)hipGetLastError();
}

int launch_linear_dz(int dtype, const LinearDz& a, ColumnSums& left, void* stream) {
  left = {};
  if (!a.dZ && !a.dbias) return 0;
  const DzGrid g = dz_grid(a.M, a.N, a.dZ ? a.ldz : a.N);
  const int64_t blocks = linear_column_blocks(a.M, a.N);
  const dim3 grid((unsigned)((g.pieces + (1 << g.lane_shift) - 1) >> g.lane_shift), (unsigned)blocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == 1) hipLaunchKernelGGL(linear_dz_kernel<uint16_t>, grid, dim3(kThreads), 0, st, a, g);
  else hipLaunchKernelGGL(linear_dz_kernel<float>, grid, dim3(kThreads), 0, st, a, g);
  if (a.dbias) left = {a.partials, blocks, a.N, a.dbias};
  return (int)hipGetLastError();
}

}  // namespace mhffn
