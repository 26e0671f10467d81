// What follows a matrix product in a linear layer, element by element, and the generator of its
// dropout:
//   z = x W + b;   y = r + D(act(z));   D(v) = v * scale where the element stays, 0 elsewhere.
// Everything works on pieces of eight neighbouring columns of one row (columns 8 c .. 8 c + 7):
// 16 bytes of bf16, and exactly what one call of the generator decides.
//
// The generator is Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as
// 1, 2, 3", 2011): ten rounds of two 32 x 32 -> 64 products over a counter of 128 bits.  Key = the
// seed; counter = (piece, offset + call), both 64 bits, low word first; piece = row * ceil(n / 8) + c.
// Column 8 c + j stays where half j of the four words (16 bits, low half first) reaches the
// threshold rint(65536 p).  So an element's fate depends on the seed, the offset and its place
// alone: whoever needs the mask again computes it again, in any tiling, and it is never stored.
#pragma once

#include "mhffn_device.h"
#include "mhffn_internal.h"

#include <type_traits>

namespace mhffn {

// ---- dropout ----------------------------------------------------------------------------------
struct DropKey { uint32_t k0, k1, c2, c3; };

// (read on the device: a captured graph draws new numbers when the caller advances the offset)
__device__ __forceinline__ DropKey drop_key(const Dropout& d) {
  DropKey k = {0, 0, 0, 0};
  if (d.threshold == 0 || d.threshold > 65535) return k;
  const uint64_t seed = d.rng[0], step = d.rng[1] + d.call;
  k.k0 = (uint32_t)seed; k.k1 = (uint32_t)(seed >> 32);
  k.c2 = (uint32_t)step; k.c3 = (uint32_t)(step >> 32);
  return k;
}

__device__ __forceinline__ u32x4 philox4x32_10(uint64_t piece, const DropKey& key) {
  uint32_t c0 = (uint32_t)piece, c1 = (uint32_t)(piece >> 32), c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// A dropped element is 0 whatever it held, infinities and NaN among it.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t piece, const Dropout& d, const DropKey& key, float scale) {
  if (d.threshold == 0) return;
  if (d.threshold > 65535) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    return;
  }
  const u32x4 w = philox4x32_10(piece, key);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t half = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
    v[j] = half >= d.threshold ? v[j] * scale : 0.f;
  }
}

// ---- activations (ACT: mhffn_activation) --------------------------------------------------------
// Phi(-|z|) and exp(-z^2 / 2) for bf16 results: Abramowitz and Stegun, Handbook of Mathematical
// Functions, 7.1.26, good to 1.5e-7 absolute, with the one exponential that the slope needs too.
// |z| stops at 30, where both are 0 in fp32.  Relative to itself the tail is good to 1e-4 at z = -3 and a bf16 half step (0.4 %) at
// -6, where z Phi(z) is 6e-9.
struct NormalTail { float a, q, e; };
__device__ __forceinline__ NormalTail normal_tail(float z) {
  NormalTail n;
  n.a = fminf(fabsf(z), 30.f);
  n.e = __builtin_amdgcn_exp2f(-0.5f * MHFFN_LOG2E * n.a * n.a);
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678118654752f * n.a);
  float p = 0.5f * 1.061405429f;
  p = p * t - 0.5f * 1.453152027f;
  p = p * t + 0.5f * 1.421413741f;
  p = p * t - 0.5f * 0.284496736f;
  p = p * t + 0.5f * 0.254829592f;
  n.q = p * t * n.e;
  return n;
}
// NaN stays NaN in each, infinities give the limits: a factor z next to one that has vanished is held to a finite value (128
// for silu, 30 for gelu; past them the other factor is 0 or 1).  Results of type T: fp32 takes the library's erfc (its products are
// sixteen times as long; 1 + erf would cancel for negative z: a digit is left at -5; a forward of 2000 x 768 x 2048 67.0 us, with erf 65.0), bf16 the tail above.
template <int ACT, typename T>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == 1) return z < 0.f ? 0.f : z;
  else if constexpr (ACT == 2) return fmaxf(z, -128.f) * sigmoid_fast(z);
  else if constexpr (ACT == 3 && sizeof(T) == 4) return 0.5f * fmaxf(z, -30.f) * erfcf(-0.70710678118654752f * z);
  else if constexpr (ACT == 3) {
    const NormalTail n = normal_tail(z);
    return (z < 0.f ? 0.f : z) - n.a * n.q;   // z Phi(z)
  } else return z;
}
// act'(z)
template <int ACT, typename T>
__device__ __forceinline__ float slope(float z) {
  if constexpr (ACT == 1) return z <= 0.f ? 0.f : 1.f;
  else if constexpr (ACT == 2) {
    const float s = sigmoid_fast(z);
    return s + fminf(fmaxf(z, -128.f), 128.f) * s * (1.f - s);
  } else if constexpr (ACT == 3 && sizeof(T) == 4) {
    return 0.5f * erfcf(-0.70710678118654752f * z) +
           fminf(fmaxf(z, -30.f), 30.f) * (0.39894228040143268f * __builtin_amdgcn_exp2f(-0.5f * MHFFN_LOG2E * z * z));
  } else if constexpr (ACT == 3) {
    const NormalTail n = normal_tail(z);
    return (z < 0.f ? n.q : 1.f - n.q) + (fabsf(z) > 30.f ? 0.f : z) * (0.39894228040143268f * n.e);
  } else return 1.f;
}
template <int ACT, typename T>
__device__ __forceinline__ void activate8(float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = activate<ACT, T>(v[j]);
}
template <typename T>
__device__ __forceinline__ void activate8(float (&v)[8], int act) {
  if (act == 1) activate8<1, T>(v);
  else if (act == 2) activate8<2, T>(v);
  else if (act == 3) activate8<3, T>(v);
}
template <int ACT, typename T>
__device__ __forceinline__ void slope8(float (&v)[8], const float (&z)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= slope<ACT, T>(z[j]);
}
template <typename T>
__device__ __forceinline__ void slope8(float (&v)[8], const float (&z)[8], int act) {
  if (act == 1) slope8<1, T>(v, z);
  else if (act == 2) slope8<2, T>(v, z);
  else if (act == 3) slope8<3, T>(v, z);
}

// ---- pieces of eight columns in memory -----------------------------------------------------------
// `cols`: how many of the eight exist (at least one).  A whole piece moves 16 bytes at a time wherever it lies: such
// an access needs no more than its elements' alignment, and rows need none (an element at a time, fp32
// rows of 1001 took twice the time).
template <typename T> struct Raw8 { u32x4 w[sizeof(T) / 2]; };   // a piece as it lies in memory
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void unpack8(const Raw8<uint16_t>& r, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t two = r.w[0][j];
    v[2 * j] = __builtin_bit_cast(float, two << 16);
    v[2 * j + 1] = __builtin_bit_cast(float, two & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t bits = r.w[j >> 2][j & 3];
    v[j] = __builtin_bit_cast(float, bits);
  }
}
__device__ __forceinline__ Raw8<uint16_t> pack8(const float (&v)[8], uint16_t) {
  return {{u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}}};
}
__device__ __forceinline__ Raw8<float> pack8(const float (&v)[8], float) {
  Raw8<float> r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r.w[j >> 2][j & 3] = __builtin_bit_cast(uint32_t, v[j]);
  return r;
}
__device__ __forceinline__ Raw8<uint16_t> load_raw8(const uint16_t* p, int cols) {
  Raw8<uint16_t> r;
  if (cols >= 8) {
    r.w[0] = *reinterpret_cast<const u32x4_any2*>(p);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      r.w[0][j] = (2 * j < cols ? (uint32_t)p[2 * j] : 0u) | (2 * j + 1 < cols ? (uint32_t)p[2 * j + 1] << 16 : 0u);
  }
  return r;
}
__device__ __forceinline__ Raw8<float> load_raw8(const float* p, int cols) {
  Raw8<float> r;
  if (cols >= 8) {
    r.w[0] = reinterpret_cast<const u32x4_any4*>(p)[0];
    r.w[1] = reinterpret_cast<const u32x4_any4*>(p)[1];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j >> 2][j & 3] = j < cols ? __builtin_bit_cast(uint32_t, p[j]) : 0u;
  }
  return r;
}
__device__ __forceinline__ void store_raw8(uint16_t* p, int cols, const Raw8<uint16_t>& r) {
  if (cols >= 8) {
    *reinterpret_cast<u32x4_any2*>(p) = r.w[0];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < cols) p[j] = (uint16_t)(j & 1 ? r.w[0][j >> 1] >> 16 : r.w[0][j >> 1] & 0xFFFFu);
  }
}
__device__ __forceinline__ void store_raw8(float* p, int cols, const Raw8<float>& r) {
  if (cols >= 8) {
    reinterpret_cast<u32x4_any4*>(p)[0] = r.w[0];
    reinterpret_cast<u32x4_any4*>(p)[1] = r.w[1];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = r.w[j >> 2][j & 3];
      if (j < cols) p[j] = __builtin_bit_cast(float, bits);
    }
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, int cols, float (&v)[8]) { unpack8(load_raw8(p, cols), v); }
template <typename T>
__device__ __forceinline__ void store8(T* p, int cols, const float (&v)[8]) { store_raw8(p, cols, pack8(v, T{})); }

// ---- the epilogue of pieces in one column of pieces -------------------------------------------------
// Columns col .. col + 7 of any row, whose bias is read once.  residual() before finish(), by the
// same thread: Y may be the residual itself.  Rows and columns that do not exist are left alone.
template <typename T>
struct EpilogueColumns {
  int64_t col;
  int cols;            // how many of the eight exist (0 or less: none)
  float bias[8];
  __device__ __forceinline__ EpilogueColumns(const Epilogue& e, int64_t col_) : col(col_) {
    cols = (int)(e.N - col < 8 ? e.N - col : 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) bias[j] = 0.f;
    if (e.bias && cols > 0) load8(static_cast<const T*>(e.bias) + col, cols, bias);
  }
  __device__ __forceinline__ Raw8<T> residual(int64_t row, const Epilogue& e) const {
    if (e.residual && row < e.M && cols > 0) return load_raw8(static_cast<const T*>(e.residual) + row * e.ldr + col, cols);
    return Raw8<T>{};
  }
  __device__ __forceinline__ void store(const float (&v)[8], int64_t row, const Epilogue& e) const {
    if (row < e.M && cols > 0) store8(static_cast<T*>(e.Y) + row * e.ldy + col, cols, v);
  }
  // v: the product's eight sums
  __device__ __forceinline__ void finish(float (&v)[8], int64_t row, const Raw8<T>& res, const Epilogue& e, const DropKey& key) const {
    if (row >= e.M || cols <= 0) return;
    if (e.scale != 1.f) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= e.scale;
    }
    if (e.bias) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += bias[j];
    }
    if (e.Z) store8(static_cast<T*>(e.Z) + row * e.ldz + col, cols, v);
    activate8<T>(v, e.act);
    drop8(v, (uint64_t)row * (uint64_t)((e.N + 7) >> 3) + (uint64_t)(col >> 3), e.drop, key, e.drop.scale);
    if (e.residual) {
      float r[8];
      unpack8(res, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    store8(static_cast<T*>(e.Y) + row * e.ldy + col, cols, v);
  }
};
template <typename T>
__device__ __forceinline__ void epilogue8(float (&v)[8], int64_t row, int64_t col, const Epilogue& e, const DropKey& key) {
  const EpilogueColumns<T> ec(e, col);
  const Raw8<T> r = ec.residual(row, e);
  ec.finish(v, row, r, e, key);
}

// A wave's piece of a product, 32 IM rows m by 32 IN columns n.  The sums pass through LDS in fp32, 32 rows at a time
// (`piece`, the wave's own 32 x 32 IN floats), so that a lane holds eight columns of one row: whole rows of
// the residual, Z and Y move, and a call of the generator serves the lane that makes it.
// `put`(im, piece), im a compile-time constant, stores rows 32 im .. + 31 with put_sums: four columns 4 c .. + 3 of a row, the 16-byte
// chunks of a row permuted by the row (no bank meets two lanes on either side).
template <int IN>
__device__ __forceinline__ int sums_off(int row, int c) { return row * (128 * IN) + ((c ^ (row & (8 * IN - 1))) << 4); }
template <int IN>
__device__ __forceinline__ void put_sums(unsigned char* piece, int row, int c, f32x4 v) {
  *reinterpret_cast<f32x4*>(piece + sums_off<IN>(row, c)) = v;
}
// The residual is asked for one group of rows ahead.  The loops stay loops (only `put` needs its row block
// at compile time): unrolled, an epilogue of 128 x 128 is 150 KB of code.
template <int I, int N, typename F>
__device__ __forceinline__ void at_index(int i, F&& f) {
  if constexpr (I < N) {
    if (i == I) {   // (the marks keep the compiler from making one block of all, which would index registers)
      asm volatile("; %0" ::"n"(I));
      f(std::integral_constant<int, I>{});
      asm volatile("; %0" ::"n"(I));
    } else {
      at_index<I + 1, N>(i, f);
    }
  }
}
// SUMS: store what is there and nothing else (partial sums).
template <typename T, int IM, int IN, bool SUMS = false, typename Put>
__device__ __forceinline__ void wave_epilogue_by(Put&& put, unsigned char* piece, int64_t m, int64_t n, int lane, const Epilogue& e) {
  constexpr int LPR = 4 * IN, RPP = 64 / LPR, PASSES = 32 / RPP, GS = PASSES < 4 ? PASSES : 4;   // lanes per row, rows per pass
  const DropKey key = SUMS ? DropKey{} : drop_key(e.drop);
  const int lrow = lane / LPR, c = 2 * (lane % LPR);
  const EpilogueColumns<T> ec(e, n + 8 * (lane % LPR));
  int64_t row = m + lrow;
  Raw8<T> res[GS];
#pragma unroll
  for (int q = 0; q < GS; ++q) res[q] = SUMS ? Raw8<T>{} : ec.residual(row + q * RPP, e);
#pragma unroll 1
  for (int im = 0; im < IM; ++im) {
    at_index<0, IM>(im, [&](auto I_) __attribute__((always_inline)) { put(I_, piece); });
    __builtin_amdgcn_wave_barrier();   // (one wave: its reads follow its writes in the same queue)
#pragma unroll 1
    for (int p = 0; p < PASSES; p += GS) {
      Raw8<T> next[GS];
      const bool more = !SUMS && (im + 1 < IM || p + GS < PASSES);
      if (more) {
#pragma unroll
        for (int q = 0; q < GS; ++q) next[q] = ec.residual(row + (GS + q) * RPP, e);
      }
#pragma unroll
      for (int q = 0; q < GS; ++q) {
        const int r = (p + q) * RPP + lrow;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(piece + sums_off<IN>(r, c));
        const f32x4 hi = *reinterpret_cast<const f32x4*>(piece + sums_off<IN>(r, c + 1));
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if constexpr (SUMS) ec.store(v, row + q * RPP, e);
        else ec.finish(v, row + q * RPP, res[q], e, key);
      }
      row += GS * RPP;
      if (more) {
#pragma unroll
        for (int q = 0; q < GS; ++q) res[q] = next[q];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}
// ---- sums of columns --------------------------------------------------------------------------------
// 32 columns a workgroup of 256: thread (column t % 32, t / 32) adds up every eighth row, the eight sums meet
// in LDS (one thread a column waited for each of its loads: 128 rows of 1024 columns took 31 us)
constexpr int kSumThreads = 256;
inline unsigned column_sum_blocks(const ColumnSums& c) { return c.blocks ? (unsigned)((c.N + 31) / 32) : 0; }
template <typename T>
__device__ __forceinline__ void column_sums(const ColumnSums& s, int64_t block, float* sums) {
  const int64_t c = block * 32 + (threadIdx.x & 31);
  float sum = 0.f;
  if (c < s.N) {
#pragma unroll 8
    for (int64_t b = threadIdx.x >> 5; b < s.blocks; b += 8) sum += s.partials[b * s.N + c];
  }
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x >= 32 || c >= s.N) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) sum += sums[32 * k + threadIdx.x];
  if constexpr (sizeof(T) == 2) static_cast<uint16_t*>(s.out)[c] = (uint16_t)pack_bf16(sum, 0.f);
  else static_cast<float*>(s.out)[c] = sum;
}

// ---- division by a number that the host knows ----------------------------------------------------------
// x / d for x < 2^32: m = ceil(2^64 / d) (d > 1), the product's upper 64 bits
struct Divisor { uint32_t d, m_hi, m_lo; };
inline Divisor make_divisor(uint32_t d) {
  const uint64_t m = d > 1 ? ~(uint64_t)0 / d + 1 : 0;
  return {d, (uint32_t)(m >> 32), (uint32_t)m};
}
__device__ __forceinline__ uint32_t divide(uint32_t x, const Divisor& v) {
  if (v.d == 1) return x;
  return (uint32_t)(((uint64_t)x * v.m_hi + (((uint64_t)x * v.m_lo) >> 32)) >> 32);
}

}  // namespace mhffn
