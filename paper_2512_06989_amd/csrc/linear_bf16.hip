// bf16 product of the linear layer with its epilogue, C[m][n] = sum_k A(m,k) B(n,k), for outputs of many tiles
// (fewer: the kernels of gemm_bf16.hip).  Forms as there: an operand lies with k contiguous ("row form") or with
// its row index contiguous ("transposed form").
//
// A workgroup of eight waves owns a BM x BN tile, one workgroup per CU.  Waves w and w + 4 share a SIMD and run
// half a step apart: while one reads the operands of a slice of 32 k from LDS, the other multiplies, all
// operands in registers, and a barrier ends each half, so that the matrix pipe waits neither for LDS nor for
// memory.  What was measured for it:
//   * Products of 16 x 16 x 32, not 32 x 32 x 16: an MFMA loop fed from LDS with random operands reaches 1625
//     TFLOP/s against 1470 (from registers 1906 | 1692), since power sets the clock and the smaller product
//     moves fewer accumulator bytes (constant operands: 2107 | 2134).
//   * Direct loads of 64-byte pieces of rows come at 69 bytes a ns and CU, of 128 bytes and more at 124; a slice of
//     256 + 256 rows is 32 KB in 427 ns of products.  So a row-form operand moves in units of 64 k (whole
//     lines); a transposed one, rows of 256 bytes as they are, in units of 32.
// Waves 0-3 (early) request the n side, waves 4-7 (late) the m side, each into a ring of its own.
// n sits on the MFMA row axis: a lane ends up with four consecutive n of one row m.
//   * Beside 16 x 16 x 32 products every VALU instruction of the wave that reads costs the other one about four
//     clocks of the matrix pipe (two a read, to place it, cost the form with both operands transposed 15 %):
//     the loop over slices is unrolled over the rings' places, and reads and requests are a register and a constant.
// LDS images, 128-byte rows of eight 16-byte chunks.  Row form [rows][64 k], chunks permuted by (row / 2) % 8.
// Transposed form [32 k][64] per 64 columns, pairs of chunks permuted by bits 1 and 3 of k.  Both are free of bank
// conflicts for their reads (16 rows, 16 bytes of each; eight k rows, 32 bytes of each, a half wave at a time).
#include "epilogue.h"

#include <type_traits>

namespace mhffn {
namespace {

constexpr int kSlice = 32;      // k per half step
constexpr uint32_t kBand = 4;   // tiles along n that are worked on side by side

struct LinearGemmArgs {
  const uint16_t* A;   // m side
  const uint16_t* B;   // n side
  int64_t M, N, K, lda, ldb;
  int64_t n_items, tiles_n;
  int splits;                 // each tile is shared out over `splits` workgroups,
  int64_t slices_per_split;   // slices of k each; they leave fp32 partial sums
};

template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    static_for<B + 1, E>(f);
  }
}

template <bool TR, int ROWS, int SLOTS>
struct Ring {
  static constexpr int kK = TR ? 32 : 64;                  // k of a unit
  static constexpr int kUnit = ROWS * kK * 2, kSlots = SLOTS, kBytes = SLOTS * kUnit;
  static constexpr int kLoads = kUnit / 1024 / 4;          // 1 KB loads per unit of each of four waves
  static_assert(kLoads * 4096 == kUnit && ROWS % 64 == 0, "whole loads");
};
// Output tile, waves along m and n, and the rings: four units of a transposed operand; of a row-form one two on the
// n side (weights: near) and three on the m side
template <bool A_TR, bool B_TR, int BM_, int BN_, int WM_, int WN_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, TM = BM / WM, TN = BN / WN, IM = TM / 16, IN = TN / 16;
  using A = Ring<A_TR, BM, A_TR ? 4 : 3>;
  using B = Ring<B_TR, BN, B_TR ? 4 : 2>;
  static constexpr int kOut = 8 * 32 * TN * 4;             // the epilogue's pieces
  static constexpr int kLds = A::kBytes + B::kBytes > kOut ? A::kBytes + B::kBytes : kOut;
  static_assert(WM * WN == 8 && kLds <= (int)kLdsBytesPerWorkgroup, "eight waves, 160 KB");
  static_assert((!A_TR || TM % 64 == 0) && (!B_TR || TN % 64 == 0), "whole column blocks per wave");
};

// A pointer that is the same in every lane, in scalar registers
__device__ __forceinline__ const unsigned char* uniform(const unsigned char* p) {
  const uint64_t v = (uint64_t)p;
  return (const unsigned char*)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) |
                                (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
// global_to_lds_16B to an LDS address (the same in every lane)
__device__ __forceinline__ void load_to_lds(const void* gptr, unsigned to) {
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) const void*)gptr,
                                   (__attribute__((address_space(3))) void*)(uintptr_t)to, 16, 0, 0);
}
// byte offset of 16-byte chunk `chunk` of `row` in a row-form unit
__device__ __forceinline__ int row_unit_off(int row, int chunk) { return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4); }
// the chunk bits that k row `kr` of a transposed unit flips
__device__ __forceinline__ int tr_flip(int kr) { return (kr & 2) | ((kr >> 1) & 4); }

// T: what the epilogue stores (fp32: partial sums)
template <bool A_TR, bool B_TR, typename G, typename T>
__global__ __launch_bounds__(512, 2) void linear_gemm_kernel(LinearGemmArgs a, Epilogue e) {
  constexpr int IM = G::IM, IN = G::IN;
  using RA = typename G::A;
  using RB = typename G::B;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, gq = lane >> 4;
  const int w4 = wave & 3, wm = wave / G::WN, wn = wave % G::WN;
  const bool late = wave >= 4;
  const int64_t item = xcd_work_item(blockIdx.x, a.n_items);
  if (item >= a.n_items) return;
  // An XCD's share of the list runs over the tiles of one share of k, in bands of kBand tiles along n: the 32
  // workgroups that run at once there form a patch of about 4 x 8 tiles, whose 12 panels meet in its L2.
  const uint32_t n_tiles = (uint32_t)(a.n_items / a.splits), t = (uint32_t)(item % n_tiles);
  const int split = (int)(item / n_tiles);
  const uint32_t tiles_n = (uint32_t)a.tiles_n, tiles_m = n_tiles / tiles_n, band = t / (tiles_m * kBand);
  const uint32_t width = min(kBand, tiles_n - band * kBand), in_band = t - band * (tiles_m * kBand);
  const int64_t m0 = (int64_t)(in_band / width) * G::BM, n0 = (int64_t)(band * kBand + in_band % width) * G::BN;
  const int64_t K = a.K, KT_all = (K + kSlice - 1) / kSlice;
  const int64_t kbase = split * a.slices_per_split;           // first slice of this workgroup
  const int64_t kend = kbase + a.slices_per_split < KT_all ? kbase + a.slices_per_split : KT_all;
  const int KT = (int)(kend - kbase);                         // its number of slices (>= 1)

  // ---- requests: a wave has one side, and of its units the 1 KB images 4 q + w4 ----------------
  // An image is eight rows of 128 bytes, lane l -> row l / 8, physical chunk l % 8.  Row form: the last unit may
  // hold 32 k only, its second half fetches the first again.  Transposed form: image i = k rows 8 (i % 4) .. + 7
  // of column block i / 4.  Rows and columns past the edge are clamped (never stored), k rows past K too
  // (their slots are cleared before use).  A request is a wave-uniform base and a 32-bit offset per lane.
  constexpr int kMostLoads = RA::kLoads > RB::kLoads ? RA::kLoads : RB::kLoads;
  const int64_t ld = late ? a.lda : a.ldb, row0 = late ? m0 : n0, rows = late ? a.M : a.N;
  const int64_t k_left = K - (KT_all - 1) * kSlice;
  unsigned goff[kMostLoads];
  auto place = [&](auto TR_, int q, int64_t most_k) -> unsigned {   // most_k: k of the unit that exist
    const int img = 4 * q + w4;
    if constexpr (!decltype(TR_)::value) {
      const int row = 8 * img + (lane >> 3);
      int chunk = (lane & 7) ^ ((row >> 1) & 7);
      if (most_k <= kSlice) chunk &= 3;
      const int64_t gr = row0 + row < rows ? row : rows - 1 - row0;
      return (unsigned)(gr * ld * 2 + (chunk << 4));
    } else {
      int64_t kr = 8 * (img & 3) + (lane >> 3);
      int64_t gc = row0 + 64 * (img >> 2) + (((lane & 7) ^ tr_flip((int)kr)) << 3);
      gc = (gc + 8 <= rows ? gc : rows - 8) - row0;
      kr = kr < most_k ? kr : most_k - 1;
      return (unsigned)((kr * ld + gc) * 2);
    }
  };
  using TA = std::integral_constant<bool, A_TR>;
  using TB = std::integral_constant<bool, B_TR>;
  if (late) {
#pragma unroll
    for (int q = 0; q < RA::kLoads; ++q) goff[q] = place(TA{}, q, 64);
  } else {
#pragma unroll
    for (int q = 0; q < RB::kLoads; ++q) goff[q] = place(TB{}, q, 64);
  }
  const unsigned char* const gbase = uniform(reinterpret_cast<const unsigned char*>(
      late ? a.A + (A_TR ? m0 + kbase * kSlice * a.lda : m0 * a.lda + kbase * kSlice)
           : a.B + (B_TR ? n0 + kbase * kSlice * a.ldb : n0 * a.ldb + kbase * kSlice)));
  const int64_t gstep = late ? (A_TR ? a.lda : 1) * (RA::kK * 2) : (B_TR ? a.ldb : 1) * (RB::kK * 2);
  const unsigned ring_a = lds_addr_of(smem), ring_b = ring_a + RA::kBytes;   // LDS addresses
  auto request_side = [&](auto TR_, auto ring_, unsigned ring, int unit, int slot) {
    using R = typename decltype(ring_)::type;
    constexpr bool TR = decltype(TR_)::value;
    const unsigned char* const p = gbase + unit * gstep;
    const unsigned to = ring + slot * R::kUnit + w4 * 1024;
    const bool cut = TR ? A_TR && k_left < kSlice && kbase + unit == KT_all - 1 : kbase + 2 * unit + 1 >= KT_all;
    if (__builtin_expect(cut, 0)) {   // (this side's last request: its offsets are overwritten)
#pragma unroll
      for (int q = 0; q < R::kLoads; ++q) {
        goff[q] = place(TR_, q, k_left);
        asm volatile("" : "+v"(goff[q]));   // (computed here and not ahead of the loop)
      }
    }
#pragma unroll
    for (int q = 0; q < R::kLoads; ++q) load_to_lds(p + goff[q], to + q * 4096);
  };
  struct SideA { using type = RA; };
  struct SideB { using type = RB; };
  const int units = (late ? A_TR : B_TR) ? KT : (KT + 1) / 2;      // of this wave's side
  const int slots = late ? RA::kSlots : RB::kSlots;
  auto request = [&](int unit, int slot) {
    if (late) request_side(TA{}, SideA{}, ring_a, unit, slot);
    else request_side(TB{}, SideB{}, ring_b, unit, slot);
  };
  // waits until `unit` has landed: slots - 2 units are requested behind it, none near the end
  auto landed = [&](int unit) {
    constexpr int kA = RA::kLoads * (RA::kSlots - 2), kB = RB::kLoads * (RB::kSlots - 2);
    static_assert(kA < 64 && kB < 64, "vmcnt holds six bits");
    if (unit + slots - 2 >= units) __builtin_amdgcn_s_waitcnt(0x0F70);
    else if (late) __builtin_amdgcn_s_waitcnt(0x0F70 | (kA & 15) | ((kA >> 4) << 14));
    else __builtin_amdgcn_s_waitcnt(0x0F70 | (kB & 15) | ((kB >> 4) << 14));
  };

  // ---- operands: 16 rows of a side, 32 k ---------------------------------------------------------
  // Lane (i16, gq) holds row i16, k = 8 gq .. 8 gq + 7.  Row form: one 16-byte read; the half of the unit flips
  // a chunk bit (a register each), 16 rows are 2048 bytes.  Transposed form: two transposing reads of four k rows
  // each, 512 bytes apart; 16 columns are a pair of chunks (a register each of four), 64 columns 4096 bytes.
  constexpr int kRegs = 4;
  unsigned at[2][kRegs];   // [m side]
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const unsigned base = side ? ring_a : ring_b, wrow = side ? G::TM * wm : G::TN * wn;
    const int kr = 8 * gq + (i16 >> 2);
#pragma unroll
    for (int x = 0; x < kRegs; ++x)
      at[side][x] = (side ? A_TR : B_TR)
                        ? base + (wrow >> 6) * 4096 + kr * 128 + (((2 * x + ((i16 >> 1) & 1)) ^ tr_flip(kr)) << 4) + 8 * (i16 & 1)
                        : base + row_unit_off(wrow + i16, gq + 4 * (x & 1));
  }

  f32x4 acc[IN][IM];
#pragma unroll
  for (int i = 0; i < IN; ++i)
#pragma unroll
    for (int j = 0; j < IM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  constexpr int OPS = IN + IM;
  s16x4 lo[OPS], hi[OPS];
  bf16x8 full[OPS];
  auto barrier = [] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  int slot_a = 0, slot_r = slots - 1;   // (row form on the m side) the unit being read; the place to fill next
  auto slice = [&](int kt, auto PH_) {  // PH: kt % 4, the place of a transposed unit, half and place of a row-form one
    constexpr int PH = decltype(PH_)::value, HALF = PH & 1;
    unsigned row_a = at[1][HALF];
    if constexpr (!A_TR) row_a += slot_a * RA::kUnit;
    static_for<0, OPS>([&](auto C_) {
      constexpr int c = decltype(C_)::value, side = c < IN ? 0 : 1, idx = side ? c - IN : c;
      if constexpr (side ? A_TR : B_TR) {
        constexpr int off = PH * (side ? RA::kUnit : RB::kUnit) + (idx >> 2) * 4096;
        lo[c] = lds_read_tr16_untracked<off>(at[side][idx & 3]);
        hi[c] = lds_read_tr16_untracked<off + 512>(at[side][idx & 3]);
      } else if constexpr (side) {
        full[c] = lds_read_b128_untracked<2048 * idx>(row_a);
      } else {
        full[c] = lds_read_b128_untracked<(PH >> 1) * RB::kUnit + 2048 * idx>(at[0][HALF]);
      }
    });
    const bool row_form = !(late ? A_TR : B_TR);
    if (!row_form || HALF == 0) {
      const int unit = (row_form ? kt >> 1 : kt) + slots - 1;
      if (unit < units) request(unit, slot_r);
      slot_r = slot_r + 1 == slots ? 0 : slot_r + 1;
    }
    // Early waves read slice kt + 1 right after their products of slice kt: the parts of it that this wave
    // requested must have landed by then (row form: only where it begins a unit)
    const bool fresh = !row_form || HALF == 1;
    const int next_unit = row_form ? (kt + 1) >> 1 : kt + 1;
    if (late && fresh) landed(next_unit);
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, OPS>([&](auto C_) {   // (one wait; the others only tie their registers to it)
      constexpr int c = decltype(C_)::value;
      if constexpr (c < IN ? B_TR : A_TR) {
        if constexpr (c == 0) lds_wait<0>(lo[c], hi[c]);
        else asm volatile("" : "+v"(lo[c]), "+v"(hi[c]));
      } else {
        if constexpr (c == 0) lds_wait<0>(full[c]);
        else asm volatile("" : "+v"(full[c]));
      }
    });
    barrier();
    const bool ragged_last = A_TR && (kbase + kt == KT_all - 1) && k_left < kSlice;
    if constexpr (A_TR) {
      if (ragged_last) {   // k rows past K were clamped: clear their slots
        static_for<0, OPS>([&](auto C_) {
          constexpr int c = decltype(C_)::value;
#pragma unroll
          for (int sl = 0; sl < 4; ++sl) {
            if (8 * gq + sl >= k_left) lo[c][sl] = 0;
            if (8 * gq + 4 + sl >= k_left) hi[c][sl] = 0;
          }
        });
      }
    }
    __builtin_amdgcn_s_setprio(1);
    static_for<0, OPS>([&](auto C_) {
      constexpr int c = decltype(C_)::value;
      if constexpr (c < IN ? B_TR : A_TR) full[c] = join_tr(lo[c], hi[c]);
      if constexpr (c >= IN) {
#pragma unroll
        for (int jn = 0; jn < IN; ++jn) acc[jn][c - IN] = mfma16(full[jn], full[c], acc[jn][c - IN]);
      }
    });
    __builtin_amdgcn_s_setprio(0);
    if (!late && fresh) landed(next_unit);
    barrier();
    if (!A_TR && HALF == 1) slot_a = slot_a == 2 ? 0 : slot_a + 1;
  };

  for (int i = 0; i < slots - 1 && i < units; ++i) request(i, i);
  landed(0);
  barrier();
  if (late) barrier();
  for (int kt = 0; kt < KT; kt += 4) {
    slice(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < KT) slice(kt + 1, std::integral_constant<int, 1>{});
    if (kt + 2 < KT) slice(kt + 2, std::integral_constant<int, 2>{});
    if (kt + 3 < KT) slice(kt + 3, std::integral_constant<int, 3>{});
  }
  if (!late) barrier();
  __syncthreads();   // the rings are done with
  if (sizeof(T) == 4) e.Y = static_cast<float*>(e.Y) + (int64_t)split * a.M * a.N;
  wave_epilogue_by<T, IM / 2, IN / 2, sizeof(T) == 4>(
      [&](auto IM_, unsigned char* piece) __attribute__((always_inline)) {
        constexpr int im = decltype(IM_)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int jn = 0; jn < IN; ++jn) put_sums<IN / 2>(piece, 16 * h + i16, 4 * jn + gq, acc[jn][2 * im + h]);
      },
      smem + wave * (32 * G::TN * 4), m0 + G::TM * wm, n0 + G::TN * wn, lane, e);
}

template <bool A_TR, bool B_TR, int BM, int BN, int WM, int WN, typename T>
int launch_tile(LinearGemmArgs a, const Epilogue& e, hipStream_t stream) {
  using G = Tile<A_TR, B_TR, BM, BN, WM, WN>;
  a.tiles_n = (a.N + BN - 1) / BN;
  a.n_items = (a.M + BM - 1) / BM * a.tiles_n * a.splits;
  if (hipError_t e0 = LdsLimit<&linear_gemm_kernel<A_TR, B_TR, G, T>, G::kLds>::ensure(); e0 != hipSuccess) return (int)e0;
  hipLaunchKernelGGL((linear_gemm_kernel<A_TR, B_TR, G, T>), dim3((unsigned)xcd_grid_size(a.n_items)), dim3(512), G::kLds,
                     stream, a, e);
  return (int)hipGetLastError();
}
template <bool A_TR, bool B_TR, typename T>
int launch_form(const LinearGemmArgs& a, const Epilogue& e, bool wide, hipStream_t stream) {
  return wide ? launch_tile<A_TR, B_TR, 256, 256, 2, 4, T>(a, e, stream) : launch_tile<A_TR, B_TR, 256, 128, 4, 2, T>(a, e, stream);
}
template <typename T>
int launch(bool a_tr, bool b_tr, const LinearGemmArgs& a, const Epilogue& e, bool wide, hipStream_t stream) {
  if (!a_tr && b_tr) return launch_form<false, true, T>(a, e, wide, stream);
  if (!a_tr && !b_tr) return launch_form<false, false, T>(a, e, wide, stream);
  return a_tr && b_tr ? launch_form<true, true, T>(a, e, wide, stream) : -1;   // transposed A with row-form B: no caller
}

}  // namespace

int launch_linear_tiles(bool a_tr, bool b_tr, bool wide, const void* A, int64_t lda, const void* B, int64_t ldb, int64_t M,
                        int64_t N, int64_t K, int splits, int64_t slices_per_split, const Epilogue& e, void* P, void* stream) {
  LinearGemmArgs a = {static_cast<const uint16_t*>(A), static_cast<const uint16_t*>(B), M, N, K, lda, ldb, 0, 0, splits,
                      slices_per_split};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (splits == 1) return launch<uint16_t>(a_tr, b_tr, a, with_vec(e, 1), wide, st);
  Epilogue sums = {};
  sums.Y = P; sums.ldy = N; sums.M = M; sums.N = N;   // (N % 8 == 0)
  return launch<float>(a_tr, b_tr, a, with_vec(sums, 0), wide, st);
}

}  // namespace mhffn
