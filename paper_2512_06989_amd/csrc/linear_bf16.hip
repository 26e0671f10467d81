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

constexpr int kStep = 32;      // k per half step
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

// A workgroup's tile and share of k.  An XCD's share of the list runs over the tiles of one share of k, in bands
// of kBand tiles along n: the 32 workgroups that run at once there form a patch of about 4 x 8 tiles, whose 12
// panels meet in its L2.
template <typename G>
__device__ __forceinline__ bool place_of(const LinearGemmArgs& a, int64_t block, int64_t& m0, int64_t& n0, int& split, int64_t& kbase, int64_t& kend) {
  const int64_t item = xcd_work_item(block, a.n_items);
  if (item >= a.n_items) return false;
  const uint32_t n_tiles = (uint32_t)(a.n_items / a.splits), t = (uint32_t)(item % n_tiles);
  split = (int)(item / n_tiles);
  const uint32_t tiles_n = (uint32_t)a.tiles_n, tiles_m = n_tiles / tiles_n, band = t / (tiles_m * kBand);
  const uint32_t width = min(kBand, tiles_n - band * kBand), in_band = t - band * (tiles_m * kBand);
  m0 = (int64_t)(in_band / width) * G::BM;
  n0 = (int64_t)(band * kBand + in_band % width) * G::BN;
  const int64_t KT_all = (a.K + kStep - 1) / kStep;
  kbase = split * a.slices_per_split;
  kend = kbase + a.slices_per_split < KT_all ? kbase + a.slices_per_split : KT_all;
  return true;
}

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
  int64_t m0, n0, kbase, kend;   // tile, slices of k
  int split;
  if (!place_of<G>(a, blockIdx.x, m0, n0, split, kbase, kend)) return;
  const int64_t K = a.K, KT_all = (K + kStep - 1) / kStep;
  const int KT = (int)(kend - kbase);                         // its number of slices (>= 1)

  // ---- requests: a wave has one side, and of its units the 1 KB images 4 q + w4 ----------------
  // An image is eight rows of 128 bytes, lane l -> row l / 8, physical chunk l % 8.  Row form: the last unit may
  // hold 32 k only, its second half fetches the first again.  Transposed form: image i = k rows 8 (i % 4) .. + 7
  // of column block i / 4.  Rows and columns past the edge are clamped (never stored), k rows past K too
  // (their slots are cleared before use).  A request is a wave-uniform base and a 32-bit offset per lane.
  constexpr int kMostLoads = RA::kLoads > RB::kLoads ? RA::kLoads : RB::kLoads;
  const int64_t ld = late ? a.lda : a.ldb, row0 = late ? m0 : n0, rows = late ? a.M : a.N;
  const int64_t k_left = K - (KT_all - 1) * kStep;
  unsigned goff[kMostLoads];
  auto place = [&](auto TR_, int q, int64_t most_k) -> unsigned {   // most_k: k of the unit that exist
    const int img = 4 * q + w4;
    if constexpr (!decltype(TR_)::value) {
      const int row = 8 * img + (lane >> 3);
      int chunk = (lane & 7) ^ ((row >> 1) & 7);
      if (most_k <= kStep) chunk &= 3;
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
      late ? a.A + (A_TR ? m0 + kbase * kStep * a.lda : m0 * a.lda + kbase * kStep)
           : a.B + (B_TR ? n0 + kbase * kStep * a.ldb : n0 * a.ldb + kbase * kStep)));
  const int64_t gstep = late ? (A_TR ? a.lda : 1) * (RA::kK * 2) : (B_TR ? a.ldb : 1) * (RB::kK * 2);
  const unsigned ring_a = lds_addr_of(smem), ring_b = ring_a + RA::kBytes;   // LDS addresses
  auto request_side = [&](auto TR_, auto ring_, unsigned ring, int unit, int slot) {
    using R = typename decltype(ring_)::type;
    constexpr bool TR = decltype(TR_)::value;
    const unsigned char* const p = gbase + unit * gstep;
    const unsigned to = ring + slot * R::kUnit + w4 * 1024;
    const bool cut = TR ? A_TR && k_left < kStep && kbase + unit == KT_all - 1 : kbase + 2 * unit + 1 >= KT_all;
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
    const bool ragged_last = A_TR && (kbase + kt == KT_all - 1) && k_left < kStep;
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

// ---------------------------------------------------------------------------
// Smaller tiles, for outputs that would leave CUs without one: two rows of waves, k in units of 64.  Such products wait
// for memory, so what counts is bytes in flight: units lie in a ring of 48 KB (64 x 64) .. 160 KB (128 x 128), all but
// one of them under way, and up to three workgroups share a CU, so that one's first loads and epilogue lie under
// another's products (1000 x 1024 x 2816: 14.9 us; 64 x 64 with all of LDS to itself 24.4, 128 x 128 16.0).  A wave
// multiplies a unit's operands from registers and between the products reads the next one's from LDS and requests
// another, an instruction at a time; one wait for LDS and one barrier per unit (two steps of 32 with a wait each:
// 730 clocks a unit of 64 x 64).  Images and operands as above, a transposed unit [64 k][64] per 64 columns.
// ---------------------------------------------------------------------------
template <int BM_, int BN_, int WN_, int PER_CU>
struct SmallTile {
  static constexpr int BM = BM_, BN = BN_, WN = WN_, NW = 2 * WN, TM = BM / 2, TN = BN / WN, IM = TM / 16, IN = TN / 16;
  static constexpr int kK = 64;                            // k of a unit
  static constexpr int kUnitA = BM * 128, kUnitB = BN * 128, kUnit = kUnitA + kUnitB;
  static constexpr int kPerCu = PER_CU, kSlots = (int)kLdsBytesPerWorkgroup / PER_CU / kUnit, kLds = kSlots * kUnit;
  static constexpr int kLoadsA = kUnitA / 1024 / NW, kLoadsB = kUnitB / 1024 / NW, kLoads = kLoadsA + kLoadsB;   // 1 KB loads per unit of each wave
  static_assert(BM % 64 == 0 && BN % 64 == 0 && TN % 32 == 0 && kSlots > 1 && kLds >= NW * 32 * TN * 4 && kLoads * (kSlots - 1) < 64, "");
  static_assert(kLoadsA * NW * 1024 == kUnitA && kLoads * NW * 1024 == kUnit, "whole loads");
};

template <bool A_TR, bool B_TR, typename G, typename T>
__device__ __forceinline__ void linear_small_tile(const LinearGemmArgs& a, Epilogue e, int64_t block, unsigned char* smem) {
  constexpr int IM = G::IM, IN = G::IN, OPS = IM + IN, NM = IM * IN, S = G::kSlots, NS = 2;   // operands and products of 32 k, of which a unit has NS
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, gq = lane >> 4;
  const int wm = wave / G::WN, wn = wave % G::WN;
  int64_t m0, n0, kbase, kend;
  int split;
  if (!place_of<G>(a, block, m0, n0, split, kbase, kend)) return;
  const int64_t K = a.K, k0 = kbase * kStep, k_own = (kend * kStep < K ? kend * kStep : K) - k0;
  const int units = (int)((kend - kbase + NS - 1) / NS);

  // ---- requests: of a side's 1 KB images wave w moves NW q + w -------------------------------------
  // k past the product's end: row form fetches the first 32 of 64 again, k rows repeat the last.
  unsigned ga[G::kLoadsA], gb[G::kLoadsB];
  auto place = [&](bool tr, int q, int64_t ld, int64_t row0, int64_t rows, int64_t left) __attribute__((always_inline)) -> unsigned {
    const int i = G::NW * q + wave;
    if (!tr) {
      const int row = 8 * i + (lane >> 3);
      int chunk = (lane & 7) ^ ((row >> 1) & 7);
      if (left <= kStep) chunk &= 3;
      const int64_t gr = row0 + row < rows ? row : rows - 1 - row0;
      return (unsigned)(gr * ld * 2 + (chunk << 4));
    }
    int64_t kr = 8 * (i & 7) + (lane >> 3);
    int64_t gc = row0 + 64 * (i >> 3) + (((lane & 7) ^ tr_flip((int)kr)) << 3);
    gc = (gc + 8 <= rows ? gc : rows - 8) - row0;
    kr = kr < left ? kr : left - 1;
    return (unsigned)((kr * ld + gc) * 2);
  };
  auto offsets = [&](int64_t left) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < G::kLoadsA; ++q) ga[q] = place(A_TR, q, a.lda, m0, a.M, left);
#pragma unroll
    for (int q = 0; q < G::kLoadsB; ++q) gb[q] = place(B_TR, q, a.ldb, n0, a.N, left);
  };
  const unsigned char* pa = uniform(reinterpret_cast<const unsigned char*>(a.A + (A_TR ? m0 + k0 * a.lda : m0 * a.lda + k0)));
  const unsigned char* pb = uniform(reinterpret_cast<const unsigned char*>(a.B + (B_TR ? n0 + k0 * a.ldb : n0 * a.ldb + k0)));
  const int64_t step_a = (A_TR ? a.lda : 1) * (2 * G::kK), step_b = (B_TR ? a.ldb : 1) * (2 * G::kK);
  const unsigned ring = lds_addr_of(smem);
  unsigned to = ring + wave * 1024;
  auto begin = [&](int unit) __attribute__((always_inline)) {
    const int64_t left = K - k0 - G::kK * (int64_t)unit;
    if (__builtin_expect(left < G::kK, 0)) {   // (the last request: its offsets take the place of the others')
      offsets(left);
#pragma unroll
      for (int q = 0; q < G::kLoadsA; ++q) asm volatile("" : "+v"(ga[q]));   // (computed here and not ahead of the loop)
#pragma unroll
      for (int q = 0; q < G::kLoadsB; ++q) asm volatile("" : "+v"(gb[q]));
    }
  };
  auto load = [&](auto Q_) __attribute__((always_inline)) {
    constexpr int q = decltype(Q_)::value;
    if constexpr (q < G::kLoadsA) load_to_lds(pa + ga[q], to + q * (1024 * G::NW));
    else load_to_lds(pb + gb[q - G::kLoadsA], to + G::kUnitA + (q - G::kLoadsA) * (1024 * G::NW));
  };
  auto end = [&]() __attribute__((always_inline)) {
    pa += step_a;
    pb += step_b;
    to = to == ring + (S - 1) * G::kUnit + wave * 1024 ? ring + wave * 1024 : to + G::kUnit;
  };
  offsets(G::kK);

  // ---- operands (see above); a transposed unit's halves of k are 4096 bytes apart -----------------------
  constexpr int RA = A_TR ? IM : 2, RB = B_TR ? IN : 2;
  unsigned at_a[RA], at_b[RB];
  auto first = [&](bool tr, unsigned base, unsigned wrow, int x) __attribute__((always_inline)) -> unsigned {
    const int kr = 8 * gq + (i16 >> 2);
    return tr ? base + (wrow >> 6) * 8192 + kr * 128 + (((2 * (((wrow & 63) >> 4) + x) + ((i16 >> 1) & 1)) ^ tr_flip(kr)) << 4) + 8 * (i16 & 1)
              : base + row_unit_off(wrow + i16, gq + 4 * x);
  };
#pragma unroll
  for (int x = 0; x < RA; ++x) at_a[x] = first(A_TR, ring, G::TM * wm, x);
#pragma unroll
  for (int x = 0; x < RB; ++x) at_b[x] = first(B_TR, ring + G::kUnitA, G::TN * wn, x);
  int slot = 0;
  auto next_unit = [&]() __attribute__((always_inline)) {
    const unsigned by = slot == S - 1 ? 0u - (S - 1) * G::kUnit : (unsigned)G::kUnit;
    slot = slot == S - 1 ? 0 : slot + 1;
#pragma unroll
    for (int x = 0; x < RA; ++x) at_a[x] += by;
#pragma unroll
    for (int x = 0; x < RB; ++x) at_b[x] += by;
  };

  f32x4 acc[IN][IM];
#pragma unroll
  for (int i = 0; i < IN; ++i)
#pragma unroll
    for (int j = 0; j < IM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  struct Operands {   // of a unit, 32 k after 32 k
    s16x4 lo[NS * OPS], hi[NS * OPS];
    bf16x8 full[NS * OPS];
  };
  Operands f0, f1;
  auto read = [&](auto C_, Operands& f) __attribute__((always_inline)) {
    constexpr int c = decltype(C_)::value, HALF = c / OPS, o = c % OPS, idx = o < IN ? o : o - IN;
    if constexpr (o < IN ? B_TR : A_TR) {
      const unsigned at = o < IN ? at_b[B_TR ? idx : 0] : at_a[A_TR ? idx : 0];
      f.lo[c] = lds_read_tr16_untracked<HALF * 4096>(at);
      f.hi[c] = lds_read_tr16_untracked<HALF * 4096 + 512>(at);
    } else {
      f.full[c] = lds_read_b128_untracked<2048 * idx>(o < IN ? at_b[HALF] : at_a[HALF]);
    }
  };
  auto arrived = [&](Operands& f, int unit) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, NS * OPS>([&](auto C_) __attribute__((always_inline)) {   // (one wait; the others only tie their registers to it)
      constexpr int c = decltype(C_)::value;
      if constexpr (c % OPS < IN ? B_TR : A_TR) {
        if constexpr (c == 0) lds_wait<0>(f.lo[c], f.hi[c]);
        else asm volatile("" : "+v"(f.lo[c]), "+v"(f.hi[c]));
      } else {
        if constexpr (c == 0) lds_wait<0>(f.full[c]);
        else asm volatile("" : "+v"(f.full[c]));
      }
    });
    // k past the share's end was repeated or is another share's: clear those slots, on both sides (infinities)
    const int64_t left = k_own - G::kK * (int64_t)unit;
    if (__builtin_expect(left < G::kK, 0)) {
      static_for<0, NS * OPS>([&](auto C_) __attribute__((always_inline)) {
        constexpr int c = decltype(C_)::value, k = c / OPS * kStep;
        if constexpr (c % OPS < IN ? B_TR : A_TR) {
#pragma unroll
          for (int sl = 0; sl < 4; ++sl) {
            if (k + 8 * gq + sl >= left) f.lo[c][sl] = 0;
            if (k + 8 * gq + 4 + sl >= left) f.hi[c][sl] = 0;
          }
        } else {
          if (k >= left) f.full[c] = bf16x8{0};   // (row form: K % 32 == 0)
        }
      });
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // The products of a unit; between the first half of them the next one's reads, and the requests of another
  auto multiply = [&](Operands& f, Operands& next, bool more, auto LAST_) __attribute__((always_inline)) {
    static_for<0, NS * NM>([&](auto I_) __attribute__((always_inline)) {
      constexpr int i = decltype(I_)::value, h = i / NM, jn = i % IN, c = h * OPS + IN + i % NM / IN, cn = h * OPS + jn;
      if constexpr (jn == 0 && A_TR) f.full[c] = join_tr(f.lo[c], f.hi[c]);
      if constexpr (i % NM < IN && B_TR) f.full[cn] = join_tr(f.lo[cn], f.hi[cn]);
      acc[jn][i % NM / IN] = mfma16(f.full[cn], f.full[c], acc[jn][i % NM / IN]);
      if constexpr (!decltype(LAST_)::value) {
        static_for<0, NS * OPS>([&](auto C_) __attribute__((always_inline)) {
          if constexpr (decltype(C_)::value * NM / (2 * OPS) == i) read(C_, next);
        });
        constexpr int kPer = (G::kLoads + NS * NM - 1) / (NS * NM), q0 = i * kPer < G::kLoads ? i * kPer : G::kLoads;
        if (more) static_for<q0, (q0 + kPer < G::kLoads ? q0 + kPer : G::kLoads)>(load);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };
  auto request = [&](int unit) __attribute__((always_inline)) {
    begin(unit);
    static_for<0, G::kLoads>(load);
    end();
  };
  // waits until unit `unit` has landed: S - 1 units are requested behind unit `unit` - 1, none near the end
  auto landed = [&](int unit) __attribute__((always_inline)) {
    constexpr int kBehind = G::kLoads * (S - 2);
    if (unit + S - 2 < units) __builtin_amdgcn_s_waitcnt(0x0F70 | (kBehind & 15) | ((kBehind >> 4) << 14));
    else __builtin_amdgcn_s_waitcnt(0x0F70);
  };

  for (int i = 0; i < S - 1 && i < units; ++i) request(i);
  landed(0);
  __syncthreads();
  static_for<0, NS * OPS>([&](auto C_) __attribute__((always_inline)) { read(C_, f0); });
  if (S - 1 < units) request(S - 1);
  arrived(f0, 0);
  auto unit = [&](int j, Operands& f, Operands& next) __attribute__((always_inline)) {
    // Unit j is in registers, and unit j + 1 has to have landed: behind it the ring's other S - 2 units are under way
    landed(j + 1);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const bool more = j + S < units;
    if (more) begin(j + S);
    next_unit();
    multiply(f, next, more, std::false_type{});
    if (more) end();
    arrived(next, j + 1);   // (here: no read may be under way where paths meet and registers are renamed)
  };
  auto last = [&](Operands& f) __attribute__((always_inline)) { multiply(f, f, false, std::true_type{}); };
  int j = 0;
  for (; j + 2 < units; j += 2) {
    unit(j, f0, f1);
    unit(j + 1, f1, f0);
  }
  if (j + 1 < units) {
    unit(j, f0, f1);
    last(f1);
  } else {
    last(f0);
  }
  __syncthreads();   // the ring is done with
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

template <bool A_TR, bool B_TR, typename G, typename T>
__global__ __launch_bounds__(64 * G::NW, G::kPerCu * G::NW / 4) void linear_small_kernel(LinearGemmArgs a, Epilogue e) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  linear_small_tile<A_TR, B_TR, G, T>(a, e, blockIdx.x, smem);
}
// A backward of few tiles: dX, dW and the sums of columns in one launch.  Workgroups start in order: the longer
// product's come first.
using PairTile = SmallTile<64, 64, 2, 3>;
__global__ __launch_bounds__(64 * PairTile::NW, PairTile::kPerCu * PairTile::NW / 4) void linear_pair_kernel(
    LinearGemmArgs x, Epilogue ex, LinearGemmArgs w, Epilogue ew, ColumnSums c, unsigned grid_x, unsigned grid_w, bool x_first) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  static_assert(64 * PairTile::NW == kSumThreads, "");
  const unsigned from_x = x_first ? 0 : grid_w, from_w = x_first ? grid_x : 0;
  if (blockIdx.x >= grid_x + grid_w) column_sums<uint16_t>(c, blockIdx.x - grid_x - grid_w, reinterpret_cast<float*>(smem));
  else if (blockIdx.x - from_x < grid_x) linear_small_tile<false, false, PairTile, uint16_t>(x, ex, blockIdx.x - from_x, smem);
  else linear_small_tile<true, true, PairTile, uint16_t>(w, ew, blockIdx.x - from_w, smem);
}

template <typename G>
unsigned set_tiles(LinearGemmArgs& a) {   // returns the grid
  a.tiles_n = (a.N + G::BN - 1) / G::BN;
  a.n_items = (a.M + G::BM - 1) / G::BM * a.tiles_n * a.splits;
  return (unsigned)xcd_grid_size(a.n_items);
}
template <bool SMALL, bool A_TR, bool B_TR, typename G, typename T>
int launch_tile(LinearGemmArgs a, const Epilogue& e, hipStream_t stream) {
  const dim3 grid(set_tiles<G>(a));
  if constexpr (SMALL) {
    if (hipError_t e0 = LdsLimit<&linear_small_kernel<A_TR, B_TR, G, T>, G::kLds>::ensure(); e0 != hipSuccess) return (int)e0;
    hipLaunchKernelGGL((linear_small_kernel<A_TR, B_TR, G, T>), grid, dim3(64 * G::NW), G::kLds, stream, a, e);
  } else {
    if (hipError_t e0 = LdsLimit<&linear_gemm_kernel<A_TR, B_TR, G, T>, G::kLds>::ensure(); e0 != hipSuccess) return (int)e0;
    hipLaunchKernelGGL((linear_gemm_kernel<A_TR, B_TR, G, T>), grid, dim3(512), G::kLds, stream, a, e);
  }
  return (int)hipGetLastError();
}
template <bool A_TR, bool B_TR, typename T>
int launch_form(const LinearGemmArgs& a, const Epilogue& e, int shape, hipStream_t stream) {
  switch (shape) {
    case 0: return launch_tile<false, A_TR, B_TR, Tile<A_TR, B_TR, 256, 256, 2, 4>, T>(a, e, stream);
    case 1: return launch_tile<false, A_TR, B_TR, Tile<A_TR, B_TR, 256, 128, 4, 2>, T>(a, e, stream);
    case 2: return launch_tile<true, A_TR, B_TR, SmallTile<128, 128, 4, 1>, T>(a, e, stream);
    case 3: return launch_tile<true, A_TR, B_TR, SmallTile<64, 128, 2, 2>, T>(a, e, stream);
    default: return launch_tile<true, A_TR, B_TR, PairTile, T>(a, e, stream);
  }
}
template <typename T>
int launch(bool a_tr, bool b_tr, const LinearGemmArgs& a, const Epilogue& e, int shape, hipStream_t stream) {
  if (!a_tr && b_tr) return launch_form<false, true, T>(a, e, shape, stream);
  if (!a_tr && !b_tr) return launch_form<false, false, T>(a, e, shape, stream);
  return a_tr && b_tr ? launch_form<true, true, T>(a, e, shape, stream) : -1;   // transposed A with row-form B: no caller
}

// Tile shape and split of the contraction.  Microseconds measured, with n tiles on the fullest CU: a slice of k takes
// kSliceUs[0] + n kSliceUs[1] (what is shared by the workgroups of a CU hides a latency), what lies around the slices
// kAroundUs[0] + n kAroundUs[1]; the sum over the splits is a launch of 4 and moves 5.7 MB a us.  The kernels for
// few rows: up to 16 (weights in row form: 8) 16 columns a workgroup and 4.2 MB of weights a us at most, above 32 x 32 in one
// round of one workgroup a CU (which also keeps their row blocks within a grid's second dimension, however narrow the layer).
// (us, few rows | the best of tiles and splits: 24 x 2048 x 1024 5.7 | 9.1, 64 x 5632 x 2048 18.0 | 13.2, one round 8192 x 64 x 32
// 4.1 | 4.0, 8192 x 1024 x 32 5.2 | 7.9, 2048 x 256 x 64 3.9 | 4.6, two 16384 x 64 x 32 5.9 | 4.2, 16384 x 1024 x 32 8.7 | 8.4, 8192 x
// 512 x 64 7.6 | 5.8, 64 x 2048 x 5632 18.5 | 12.9, 128 rounds 1048576 x 64 x 64 581 | 65.)
struct Plan { int shape, splits; int64_t slices_per_split; double cost; };   // shape -1: the kernels for few rows
constexpr int kShapes = 5, kShapeM[kShapes] = {256, 256, 128, 64, 64}, kShapeN[kShapes] = {256, 128, 128, 128, 64};
constexpr int kShapeThreads[kShapes] = {512, 512, 512, 256, 256};
constexpr double kSliceUs[kShapes][2] = {{0, 0.72}, {0, 0.48}, {0, 0.277}, {0.045, 0.128}, {0.04, 0.08}};
constexpr double kAroundUs[kShapes][2] = {{1, 12}, {3, 6}, {2, 4}, {3.5, 1.6}, {3.3, 0.73}};
int64_t tiles_of(int sh, int64_t M, int64_t N) { return ((M + kShapeM[sh] - 1) / kShapeM[sh]) * ((N + kShapeN[sh] - 1) / kShapeN[sh]); }
Plan plan_of(bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K) {
  const int64_t KT = (K + kStep - 1) / kStep;
  Plan best{0, 1, KT, 0.0};
  for (int sh = 0; sh < kShapes; ++sh) {
    const int64_t tiles = tiles_of(sh, M, N);
    for (int want = 1; want <= 16; ++want) {
      const int64_t per = (KT + want - 1) / want;
      if (want > 1 && (per < 8 || (KT + per - 1) / per != want)) continue;   // at least eight slices per workgroup
      if (!launch_holds(tiles * want, kShapeThreads[sh])) continue;
      const double n = (double)((tiles * want + 255) / 256);
      double cost = (double)per * (kSliceUs[sh][0] + kSliceUs[sh][1] * n) + kAroundUs[sh][0] + kAroundUs[sh][1] * n;
      if (want > 1) cost += 4 + (double)want * M * N * 4 / 5.7e6;
      if (best.cost == 0.0 || cost < best.cost) best = {sh, want, per, cost};
    }
  }
  const bool few = M <= (b_tr ? 16 : 8);
  const int64_t wgs = few ? N / 16 : (M + 31) / 32 * (N / 32);
  if (!a_tr && N % 32 == 0 && K % 64 == 0 && (few || wgs <= 256)) {
    const double slices = (double)((wgs + 255) / 256) * (double)(K / 64) * (few ? 0.065 : 0.13), weights = (double)K * N * 2 / 4.2e6;
    const double cost = 3.3 + (few && weights > slices ? weights : slices);
    if (cost < best.cost) best = {-1, 1, KT, cost};
  }
  return best;
}
Plan pair_plan(int64_t K) { return {kShapes - 1, 1, (K + kStep - 1) / kStep, 0.0}; }
LinearGemmArgs args_of(const Product& p, const Plan& plan) {
  return {static_cast<const uint16_t*>(p.A), static_cast<const uint16_t*>(p.B), p.M, p.N, p.K, p.lda, p.ldb, 0, 0, plan.splits,
          plan.slices_per_split};
}

}  // namespace

std::string linear_bf16_plan(bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K) {
  const Plan p = plan_of(a_tr, b_tr, M, N, K);
  if (p.shape < 0) return "few rows";
  return std::to_string(kShapeM[p.shape]) + "x" + std::to_string(kShapeN[p.shape]) + " splits=" + std::to_string(p.splits);
}

std::string linear_bf16_pair_plan() { return "dX 64x64 splits=1 with dW 64x64 splits=1"; }

size_t linear_bf16_workspace_bytes(bool a_tr, bool b_tr, int64_t M, int64_t N, int64_t K) {
  const int splits = plan_of(a_tr, b_tr, M, N, K).splits;
  return splits > 1 ? (size_t)splits * M * N * sizeof(float) : 0;
}

int launch_linear_bf16(const Product& p, void* ws, LinearSums& left, void* stream) {
  const Plan plan = plan_of(p.a_tr, p.b_tr, p.M, p.N, p.K);
  left = {};
  if (plan.shape < 0) return launch_linear_few_rows(p, false, stream);
  const LinearGemmArgs a = args_of(p, plan);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (plan.splits == 1) return launch<uint16_t>(p.a_tr, p.b_tr, a, p.e, plan.shape, st);
  Epilogue sums = {};
  sums.Y = ws; sums.ldy = p.N; sums.M = p.M; sums.N = p.N;   // (N % 8 == 0)
  left = {static_cast<float*>(ws), p.M, p.N, plan.splits};
  return launch<float>(p.a_tr, p.b_tr, a, sums, plan.shape, st);
}

// By the longer product and the mean of a CU's slices; apart, they are another launch or two of 6.  (us, a backward
// with an activation, together | apart: 1024 x 1024 x 1024 16 | 24, 4096 x 1024 x 1024 39 | 51, 2048 x 2048 x 2048 64 | 60.)
bool linear_bf16_pair(int64_t M, int64_t N, int64_t K, int64_t Np) {
  constexpr int kTile = kShapes - 1;
  const double kx = (double)pair_plan(Np).slices_per_split, kw = (double)pair_plan(M).slices_per_split, longest = kx > kw ? kx : kw;
  const double tx = (double)tiles_of(kTile, M, K), tw = (double)tiles_of(kTile, K, N);
  if (!launch_holds(tiles_of(kTile, M, K) + tiles_of(kTile, K, N) + N, kShapeThreads[kTile])) return false;   // (N: more than the columns' workgroups)
  const double cost = longest * kSliceUs[kTile][0] + (longest / 2 + (tx * kx + tw * kw) / 256) * kSliceUs[kTile][1] + kAroundUs[kTile][0] +
                      kAroundUs[kTile][1] * (tx + tw) / 256;
  return cost < 6 + plan_of(false, false, M, K, Np).cost + plan_of(true, true, K, N, M).cost;
}

int launch_linear_bf16_pair(const Product& x, const Product& w, const ColumnSums& c, void* stream) {
  LinearGemmArgs ax = args_of(x, pair_plan(x.K)), aw = args_of(w, pair_plan(w.K));
  const unsigned grid_w = w.e.Y ? set_tiles<PairTile>(aw) : 0, grid_x = x.e.Y ? set_tiles<PairTile>(ax) : 0;
  if (hipError_t e0 = LdsLimit<&linear_pair_kernel, PairTile::kLds>::ensure(); e0 != hipSuccess) return (int)e0;
  hipLaunchKernelGGL(linear_pair_kernel, dim3(grid_w + grid_x + column_sum_blocks(c)), dim3(64 * PairTile::NW), PairTile::kLds,
                     static_cast<hipStream_t>(stream), ax, x.e, aw, w.e, c, grid_x, grid_w, x.K > w.K);
  return (int)hipGetLastError();
}

}  // namespace mhffn
