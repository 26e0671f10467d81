// The linear layer Y = R + D(act(X W + b)) and its backward, composed on the host from the
// library's products and the kernels of pointwise.hip.  Nothing is allocated: operands that the
// product cannot read where they lie (widths or row strides it does not take) are packed into the
// workspace, zero-padded, and dZ and the partial products live there too.
#include "mhffn_internal.h"

namespace mhffn {
namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
size_t elt(int dtype) { return dtype == 1 ? 2 : 4; }
constexpr int64_t kMostLd = 1 << 22;   // (lane offsets inside a tile are 32-bit)

// Workspace, handed out front to back; a null base only adds up
struct Arena {
  unsigned char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    void* p = base ? base + used : nullptr;
    used += align256(bytes);
    return p;
  }
};

// What has to be packed, and the padded sizes of what is
struct Operands {
  bool x, w, dz;          // packed X [M][Kp], packed W [Kp][Np], dZ [M][Np] in the workspace
  bool few;               // a few rows whose operands are read as they lie
  int64_t Kp, Np;
  Operands(const Linear& p, bool backward) {
    const bool bf16 = p.dtype == 1;
    Kp = bf16 ? up(p.K, 32) : p.K;
    Np = bf16 ? up(p.N, 32) : p.N;
    const bool y_fits = p.ldy <= kMostLd && (!bf16 || p.ldy % 8 == 0);
    x = p.ldx > kMostLd || (bf16 && ((backward ? p.K % 8 : p.K % 32) != 0 || p.ldx % 8 != 0));
    w = bf16 && (backward ? p.K % 8 != 0 || p.N % 32 != 0 : p.K % 32 != 0 || p.N % 8 != 0);
    // A width that nothing divides and few rows: the kernel for few rows reads the operands as they lie.  Instead of packing
    // with up to 16 rows, or few rounds of one workgroup a CU; instead of tiles with one round.  (us, as they lie | packed:
    // 1 x 1001 x 515 5.4 | 9.5, 16 x 2048 x 5001 15 | 22, 1 x 2048 x 50257 61 | 140, 64 x 1001 x 1001 6.5 | 10.2, 130 x 520 x
    // 1000 7.6 | 10.4, 300 x 520 x 1000 11.2 | 10.5; | tiles: 1 x 4096 x 1000 6.3 | 12.0, 1 x 4128 x 4104 15.6 | 13.7.)  By sizes alone:
    // the bits of a result do not depend on row strides.
    const int64_t rounds = (up(p.M, kFewRows) / kFewRows * (up(p.N, kFewCols) / kFewCols) + 255) / 256;
    few = !backward && bf16 && p.K >= 8 && p.N >= 8 &&
          (p.K % 32 != 0 || p.N % 8 != 0 ? p.M <= kFewRows || rounds == 1 || rounds * (p.K + 300) <= 2500
                                         : (p.K % 64 != 0 || p.N % 32 != 0) && rounds == 1);
    if (few) x = w = false;
    dz = backward && (p.act != 0 || p.drop.threshold != 0 || !y_fits || (bf16 && p.N % 32 != 0));
  }
};

size_t partial_bytes(int dtype, bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K) {
  return dtype == 1 ? linear_bf16_workspace_bytes(a_tr, b_tr, M, N, K) : linear_f32_workspace_bytes(M, N, K);
}

// Columns that the forward's product works on: with W packed its padding is there for the asking
int64_t forward_columns(const Linear& p, const Operands& o) { return p.dtype != 1 || o.few ? p.N : o.w ? o.Np : up(p.N, 8); }

PackJob pack_x(const Linear& p, const Operands& o, const void* X, void* Xp) {
  return o.x ? PackJob{X, p.ldx, p.M, p.K, Xp, p.M, o.Kp} : PackJob{};
}
PackJob pack_w(const Linear& p, const Operands& o, const void* W, void* Wp) {
  return o.w ? PackJob{W, p.N, p.K, p.N, Wp, o.Kp, o.Np} : PackJob{};
}

Epilogue plain(void* Y, int64_t ldy, int64_t M, int64_t N, float scale = 1.f) {
  Epilogue e = {};
  e.Y = Y; e.ldy = ldy; e.M = M; e.N = N;
  e.scale = scale;
  return e;
}

int forward(const Linear& p, const void* X, const void* W, const void* bias, const void* residual, void* Y, void* Z,
            void* ws, size_t* bytes, void* stream) {
  const Operands o(p, false);
  const bool bf16 = p.dtype == 1;
  Arena arena{static_cast<unsigned char*>(ws)};
  void* const Xp = o.x ? arena.take((size_t)p.M * o.Kp * elt(p.dtype)) : nullptr;
  void* const Wp = o.w ? arena.take((size_t)o.Kp * o.Np * 2) : nullptr;
  const int64_t K = bf16 && (o.x || o.w) ? o.Kp : p.K, N = forward_columns(p, o);
  void* const P = o.few ? nullptr : arena.take(partial_bytes(p.dtype, false, true, p.M, N, K));
  if (bytes) {
    *bytes = arena.used;
    return 0;
  }
  int rc = launch_pack(p.dtype, pack_x(p, o, X, Xp), pack_w(p, o, W, Wp), stream);
  if (rc) return rc;
  Epilogue e = plain(Y, p.ldy, p.M, p.N);
  e.bias = bias;
  e.residual = residual; e.ldr = p.ldr;
  e.Z = Z; e.ldz = p.N;
  e.act = p.act;
  e.drop = p.drop;
  const Product y = {false, true, o.x ? Xp : X, o.x ? o.Kp : p.ldx, o.w ? Wp : W, o.w ? o.Np : p.N, p.M, N, K, e};
  if (o.few) return launch_linear_few_rows(y, true, stream);
  LinearSums left;
  rc = (bf16 ? launch_linear_bf16 : launch_linear_f32)(y, P, left, stream);
  return rc ? rc : launch_linear_sums(p.dtype, left, e, {}, {}, {}, stream);
}

int backward(const Linear& p, const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW,
             void* dbias, void* ws, size_t* bytes, void* stream) {
  const Operands o(p, true);
  const bool bf16 = p.dtype == 1;
  Arena arena{static_cast<unsigned char*>(ws)};
  void* const Xp = o.x ? arena.take((size_t)p.M * o.Kp * elt(p.dtype)) : nullptr;
  void* const Wp = o.w ? arena.take((size_t)o.Kp * o.Np * 2) : nullptr;
  const int64_t ldz = o.Np, K8 = bf16 ? up(p.K, 8) : p.K, N8 = bf16 ? up(p.N, 8) : p.N;
  void* const dZ = o.dz ? arena.take((size_t)p.M * ldz * elt(p.dtype)) : nullptr;
  float* const sums = static_cast<float*>(arena.take((size_t)linear_column_blocks(p.M, p.N) * p.N * 4));
  // Both products at once, or one after the other; what is split is added up at the end
  size_t px = 0, pw = 0;
  const bool pair = bf16 ? linear_bf16_pair(p.M, N8, K8, o.Np) : linear_f32_pair(p.M, p.N, p.K, px, pw);
  if (!pair) {
    px = partial_bytes(p.dtype, false, false, p.M, K8, o.Np);
    pw = partial_bytes(p.dtype, true, true, K8, N8, p.M);
  }
  void* const Px = arena.take(px);
  void* const Pw = arena.take(pw);
  if (bytes) {
    *bytes = arena.used;
    return 0;
  }
  LinearDz z = {dY, Z, dX || dW ? dZ : nullptr, dbias, sums, p.M, p.N, p.ldy, ldz, p.act, p.drop};
  ColumnSums columns;
  int rc = launch_linear_dz(p.dtype, z, columns, stream);
  if (rc) return rc;
  const void* const G = o.dz ? dZ : dY;
  const int64_t ldg = o.dz ? ldz : p.ldy;
  rc = launch_pack(p.dtype, dW ? pack_x(p, o, X, Xp) : PackJob{}, dX ? pack_w(p, o, W, Wp) : PackJob{}, stream);
  if (rc) return rc;
  const Product x = {false, false, G, ldg, o.w ? Wp : W, o.w ? o.Np : p.N, p.M, K8, o.Np, plain(dX, p.ldx, p.M, p.K, p.drop.scale)};
  const Product w = {true, true, o.x ? Xp : X, o.x ? o.Kp : p.ldx, G, ldg, K8, N8, p.M, plain(dW, p.N, p.K, p.N, p.drop.scale)};
  LinearSums left_x = {}, left_w = {};
  if (pair && (dX || dW)) {   // (one alone too: its bits do not depend on what else is asked for)
    if (bf16) return launch_linear_bf16_pair(x, w, columns, stream);
    rc = launch_linear_f32_pair(x, w, Px, Pw, left_x, left_w, stream);
  } else {
    const auto launch = bf16 ? launch_linear_bf16 : launch_linear_f32;
    if (dX) rc = launch(x, Px, left_x, stream);
    if (!rc && dW) rc = launch(w, Pw, left_w, stream);
  }
  return rc ? rc : launch_linear_sums(p.dtype, left_x, x.e, left_w, w.e, columns, stream);
}

}  // namespace

std::string linear_plan(const Linear& p, bool back) {
  const Operands o(p, back);
  std::string s = o.x ? "packed X " : "";
  if (o.w) s += "packed W ";
  if (o.dz) s += "dZ ";
  if (p.dtype != 1) return s + (back ? linear_f32_pair_plan(p.M, p.N, p.K) : linear_f32_plan(p.M, p.N, p.K));
  const int64_t K8 = up(p.K, 8), N8 = up(p.N, 8);
  if (o.few) return s + "few rows as they lie";
  if (!back) return s + linear_bf16_plan(false, true, p.M, forward_columns(p, o), o.x || o.w ? o.Kp : p.K);
  if (linear_bf16_pair(p.M, N8, K8, o.Np)) return s + linear_bf16_pair_plan();
  return s + "dX " + linear_bf16_plan(false, false, p.M, K8, o.Np) + "; dW " + linear_bf16_plan(true, true, K8, N8, p.M);
}

size_t linear_workspace_bytes(const Linear& p, bool back) {
  size_t bytes = 0;
  if (p.M == 0) return 0;
  if (back) backward(p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, &bytes, nullptr);
  else forward(p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, &bytes, nullptr);
  return bytes;
}

int launch_linear_forward(const Linear& p, const void* X, const void* W, const void* bias, const void* residual,
                          void* Y, void* Z, void* ws, void* stream) {
  return p.M == 0 ? 0 : forward(p, X, W, bias, residual, Y, Z, ws, nullptr, stream);
}

int launch_linear_backward(const Linear& p, const void* X, const void* W, const void* Z, const void* dY, void* dX,
                           void* dW, void* dbias, void* ws, void* stream) {
  if (p.M > 0) return backward(p, X, W, Z, dY, dX, dW, dbias, ws, nullptr, stream);
  // no rows: the parameters' gradients are zero
  return launch_pack(p.dtype, dW ? PackJob{nullptr, 0, 0, 0, dW, p.K, p.N} : PackJob{},
                     dbias ? PackJob{nullptr, 0, 0, 0, dbias, 1, p.N} : PackJob{}, stream);
}

}  // namespace mhffn
