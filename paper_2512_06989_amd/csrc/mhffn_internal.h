// Host-side declarations shared by the C-ABI layer (api.cpp) and the kernel
// translation units.  Every launcher enqueues on `stream`, never synchronises,
// and returns the hipError_t of the launch as an int (0 = success).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <string>

namespace mhffn {

// Problem description after validation; strides are always filled in.
struct Problem {
  int64_t N;        // tokens
  int H, dh, E, de; // heads, head width, sub-networks per head, sub-network width
  int64_t ldx, ldy; // row strides (elements) of X/dX and Y/dY
  int route_mode;   // 0: route = W_r (gating parameters), 1: route = R (weights)
  float eps;
};

// ---- fused forward ---------------------------------------------------------
// bf16, d_h in {64, 128, 256}, d_e % 32 == 0, E <= kFwdBf16MaxSub, LDS within the limit.
constexpr int kFwdBf16MaxSub = 96;
size_t fwd_bf16_lds_bytes(const Problem& p);
// Scratch of the bf16 forward: 0 unless the token tiles cannot fill the chip and the
// intermediate dimension is split over workgroups (fp32 partial outputs).
size_t fwd_bf16_workspace_bytes(const Problem& p);
int launch_fwd_bf16(const Problem& p, const void* X, const void* Wg, const void* Wu,
                    const void* Wd, const void* route, void* Y, void* ws, void* stream);
// fp32, d_h % 4 == 0, d_h <= 256.  The workspace is optional: with fwd_f32_workspace_bytes of
// it the shares of the intermediate dimension run on workgroups of their own, with less (or
// none) one after the other on one, with the same result.
int launch_fwd_f32(const Problem& p, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, const void* route, void* Y, void* ws, size_t ws_bytes, void* stream);
size_t fwd_f32_workspace_bytes(const Problem& p);
size_t fwd_f32_lds_bytes(const Problem& p);
constexpr size_t kLdsBytesPerWorkgroup = 160 * 1024;

// ---- fused backward --------------------------------------------------------
// bf16 limits of the backward kernels for a shape (d_h in {64, 128, 256})
int bwd_bf16_max_sub(const Problem& p);
size_t bwd_bf16_lds_bytes(const Problem& p);
size_t bwd_workspace_bytes(const Problem& p, int dtype);
int launch_bwd(const Problem& p, int dtype, const void* X, const void* Wg, const void* Wu,
               const void* Wd, const void* route, const void* dY, void* dX, void* dWg,
               void* dWu, void* dWd, void* d_route, void* ws, void* stream,
               void* const* phase_events = nullptr, int n_phase_events = 0);
// Phases of the fused backward, in launch order (see mhffn_backward_phases).
constexpr int kBwdPhases = 3;
// fp32 companion (d_h % 4 == 0, d_h <= 256, tiles must fit in LDS)
size_t bwd_f32_lds_bytes(const Problem& p);
size_t bwd_f32_workspace_bytes(const Problem& p);
int launch_bwd_f32(const Problem& p, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, const void* route, const void* dY, void* dX, void* dWg,
                   void* dWu, void* dWd, void* d_route, void* ws, void* stream);

// Last step of a token-major backward that shared its sub-networks out (bwd_finish.hip)
struct BwdFinish {
  const float* P;      // partial dX: fp32 path [shares][N][H*dh]; bf16 path [shares][unit][32 tokens],
                       // each as a wave's registers hold it (bwd.hip)
  const float* R;      // [H][E][N] gating weights
  float* DP;           // [H][E][N] dr_e in, dp_e out (params mode)
  const float* Zinv;   // [H][N] 1 / (Z + eps) (params mode)
  const void* Wr;      // [H][dh][E], storage type (params mode)
  void* dX;            // may be NULL
  int64_t N, ldx;
  int H, dh, E, shares;
  bool params;
  // units: token blocks of block_tokens, head by head, from block first_unit on
  int block_tokens;
  uint32_t first_unit, n_units;
};
int launch_bwd_tok_finish(int dtype, const BwdFinish& a, void* stream);

// ---- unfused baseline ------------------------------------------------------
size_t unfused_workspace_bytes(const Problem& p, int dtype, bool backward);
int launch_unfused(const Problem& p, int dtype, const void* X, const void* Wg,
                   const void* Wu, const void* Wd, const void* route, void* Y,
                   const void* dY, void* dX, void* dWg, void* dWu, void* dWd,
                   void* d_route, void* ws, void* stream);

// Zero `bytes` (a multiple of 4) of device memory with a fill kernel (safe under graph capture).
int launch_fill_zero(void* p, size_t bytes, void* stream);

// Plain strided product C[m][n] = sum_k A(m,k) B(n,k) on the generic MFMA GEMM of the
// unfused baseline (element strides; n is contiguous in C).  M, N or K of 0 launches nothing
// (K = 0 leaves C untouched: callers zero-fill themselves).
int launch_gemm(int dtype, const void* A, int64_t a_ms, int64_t a_ks, const void* B, int64_t b_ns,
                int64_t b_ks, void* C, int64_t c_ms, int64_t M, int64_t N, int64_t K, void* stream);

// Tuned bf16 product C[m][n] = sum_k A(m,k) B(n,k) (C row-major, ldc).  a_tr / b_tr: the
// operand is stored with its row index contiguous ([K][rows], leading dimension = row
// stride of k) instead of k contiguous ([rows][K]).  Forms: (false,true), (false,false),
// (true,true).  gemm_bf16_supported() says whether sizes and alignment fit the kernel.
bool gemm_bf16_supported(bool a_tr, bool b_tr, const void* A, int64_t lda, const void* B,
                         int64_t ldb, const void* C, int64_t ldc, int64_t M, int64_t N, int64_t K);
// Scratch (fp32 partial outputs, 256-byte aligned) when the contraction is split over
// workgroups because the output tiles alone cannot fill the chip; 0 otherwise.
size_t gemm_bf16_workspace_bytes(int64_t M, int64_t N, int64_t K);
int launch_gemm_bf16(bool a_tr, bool b_tr, const void* A, int64_t lda, const void* B, int64_t ldb,
                     void* C, int64_t ldc, int64_t M, int64_t N, int64_t K, void* ws, void* stream,
                     bool accumulate = false);
// ---- linear layer with its epilogue, dropout ---------------------------------
// Dropout after validation: an element stays where its 16 random bits reach `threshold`
// (0: all stay, the generator is not read; 65536: none does).
struct Dropout {
  uint32_t threshold;
  float scale;           // 65536 / (65536 - threshold)
  uint64_t call;
  const uint64_t* rng;   // device: seed, offset
};
// Y = residual + D(act(product + bias)), Z = product + bias where kept
struct Epilogue {
  const void* bias;      // [N]; may be NULL, like residual and Z
  const void* residual;
  void* Z;
  void* Y;
  int64_t ldr, ldz, ldy, M, N;
  int act;               // mhffn_activation
  Dropout drop;
  float scale = 1.f;     // of the product (a backward's dropout)
};
struct Linear {
  int64_t M;             // rows
  int64_t K, N;          // features in and out
  int64_t ldx, ldy, ldr; // row strides of X / dX, Y / dY, residual
  int dtype, act;
  Dropout drop;
};
size_t linear_workspace_bytes(const Linear& p, bool backward);
int launch_linear_forward(const Linear& p, const void* X, const void* W, const void* bias,
                          const void* residual, void* Y, void* Z, void* ws, void* stream);
int launch_linear_backward(const Linear& p, const void* X, const void* W, const void* Z,
                           const void* dY, void* dX, void* dW, void* dbias, void* ws, void* stream);
// Y = residual + D(X), X [M][N]; Y may be X or the residual
int launch_dropout(int dtype, const void* X, int64_t ldx, const Epilogue& e, void* stream);
// Kernels of pointwise.hip behind the host code of linear.cpp
struct LinearSums {   // `splits` partial products P [splits][rows][ldp] that an epilogue goes over (splits = 0: none)
  const float* P;
  int64_t rows, ldp;   // of the product, padding among them: at least the epilogue's
  int splits;
};
struct ColumnSums {   // out[N] = the sum of partials [blocks][N] (blocks = 0: none)
  const float* partials;
  int64_t blocks, N;
  void* out;
};
// C[m][n] = sum_k A(m,k) B(n,k) of the forms that launch_gemm_bf16 takes, and its epilogue: in the product's
// kernel where it is not split (`left` is none), to be gone over partial sums in `ws` otherwise
struct Product {
  bool a_tr, b_tr;
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb, M, N, K;
  Epilogue e;
};
// A launch holds fewer than 2^32 threads: tall outputs in small tiles may have more (2^28 x 320 in 64 x 64: 5.4e9)
inline bool launch_holds(int64_t workgroups, int threads) { return (workgroups + 16) * threads < (int64_t)1 << 32; }   // (16: grids of whole eights)
// bf16: N % 8 == 0 (e.N of the columns exist); row-form operands hold K % 32 == 0
size_t linear_bf16_workspace_bytes(bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K);
int launch_linear_bf16(const Product& p, void* ws, LinearSums& left, void* stream);
// Its kernels for a few rows (gemm_bf16.hip): N % 32 == 0, K % 64 == 0; `any`: transposed weights, K and N from 8,
// wherever they lie
constexpr int kFewRows = 16, kFewCols = 16;   // of a workgroup
int launch_linear_few_rows(const Product& p, bool any, void* stream);
// fp32: any sizes, any strides
size_t linear_f32_workspace_bytes(int64_t M, int64_t N, int64_t K);
int launch_linear_f32(const Product& p, void* ws, LinearSums& left, void* stream);
// dX [M][K] = dZ W^T and dW [K][N] = X^T dZ of a layer in one launch.  Returns whether that is worth it at these
// sizes (without launching: the bytes of both's partial sums).  e.Y = NULL: that one is not wanted
bool linear_f32_pair(int64_t M, int64_t N, int64_t K, size_t& dX_bytes, size_t& dW_bytes);
int launch_linear_f32_pair(const Product& dX, const Product& dW, void* dX_ws, void* dW_ws, LinearSums& dX_left, LinearSums& dW_left, void* stream);
// bf16: neither is split, and the sums are made in the same launch
bool linear_bf16_pair(int64_t M, int64_t N, int64_t K, int64_t Np);
int launch_linear_bf16_pair(const Product& dX, const Product& dW, const ColumnSums& c, void* stream);
// What is left of one or two products and the sums of columns, in one launch
int launch_linear_sums(int dtype, const LinearSums& a, const Epilogue& ea, const LinearSums& b, const Epilogue& eb, const ColumnSums& c, void* stream);
// [rows][cols] (row stride ld) -> dense [rows_to][cols_to], zero outside; two at once (none: rows_to = 0)
struct PackJob {
  const void* src;
  int64_t ld, rows, cols;
  void* dst;
  int64_t rows_to, cols_to;
};
int launch_pack(int dtype, const PackJob& a, const PackJob& b, void* stream);
// dZ = D(dY act'(Z)) without D's scale into dZ [M][ldz] (zero past column N; may be NULL), its column sums, scaled, into
// dbias (may be NULL) by way of `partials` (linear_column_blocks(M, N) x N floats)
struct LinearDz {
  const void* dY;
  const void* Z;
  void* dZ;
  void* dbias;
  float* partials;
  int64_t M, N, ldy, ldz;
  int act;
  Dropout drop;
};
int64_t linear_column_blocks(int64_t M, int64_t N);
int launch_linear_dz(int dtype, const LinearDz& a, ColumnSums& left, void* stream);

// ---- whole module: projections around the fused path -------------------------
// Problem::ldx / ldy are the row strides of the module's input X (dX) and output O (dO);
// Q and S are dense [N][H*d_h].
struct Residual {   // the branch O = R + D(S W_out); `rows` may be NULL
  const void* rows;
  int64_t ld;
  Dropout drop;
};
size_t module_residual_workspace_bytes(const Problem& p, int dtype, bool backward);
size_t module_workspace_bytes(const Problem& p, int dtype, bool backward);
int launch_module_forward(const Problem& p, int dtype, const void* X, const void* W_in,
                          const void* Wg, const void* Wu, const void* Wd, const void* Wr,
                          const void* W_out, void* O, void* Q, void* S, void* ws, size_t ws_bytes,
                          void* stream, const Residual* residual = nullptr);
int launch_module_backward(const Problem& p, int dtype, const void* X, const void* W_in,
                           const void* Wg, const void* Wu, const void* Wd, const void* Wr,
                           const void* W_out, const void* Q, const void* S, const void* dO,
                           void* dX, void* dW_in, void* dWg, void* dWu, void* dWd, void* dWr,
                           void* dW_out, void* ws, void* stream);
int launch_module_residual_backward(const Problem& p, int dtype, const void* X, const void* W_in,
                                    const void* Wg, const void* Wu, const void* Wd, const void* Wr,
                                    const void* W_out, const void* Q, const void* S, const void* dO,
                                    const Dropout& drop, void* dX, void* dW_in, void* dWg, void* dWu,
                                    void* dWd, void* dWr, void* dW_out, void* ws, void* stream);

// ---- what a call would launch, as text (host only; for tests) ------------------
// Kernel, tile shape and how the work is shared out, e.g. "pair256 shares=2"; products by form
// (nn, nt, tn), e.g. "256x128 splits=4".
std::string fwd_bf16_plan(const Problem& p);
std::string fwd_f32_plan(const Problem& p);
std::string bwd_plan(const Problem& p, int dtype);
std::string bwd_f32_plan(const Problem& p);
std::string gemm_bf16_plan(bool a_tr, int64_t M, int64_t N, int64_t K);
// columns of C per workgroup of the few-rows kernel that an unaccumulated product takes (0: none)
int gemm_bf16_few_columns(bool b_tr, int64_t M, int64_t N, int64_t K);
std::string module_plan(const Problem& p, int dtype, bool backward);
std::string linear_plan(const Linear& p, bool backward);
std::string linear_bf16_plan(bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K);
std::string linear_bf16_pair_plan();
std::string linear_f32_plan(int64_t M, int64_t N, int64_t K);
std::string linear_f32_pair_plan(int64_t M, int64_t N, int64_t K);

}  // namespace mhffn
