// product.hip -- y = x W^T of FP8 operands with one scale per 128 elements of
// x's rows and per 128 x 128 block of W.
//
// Computed transposed, y^T = W x^T: W's rows are the A operand and x's rows
// the B operand of v_mfma_f32_16x16x128_f8f6f4, so a lane of a 16 x 16 result
// holds ONE token (column) and four consecutive outputs.  One instruction sums
// a whole scale block; its result then enters the fp32 accumulators with one
// FMA a value, whose factor x_scale w_scale is one number a lane: the token is
// the lane's own and the weight's scale is the same for all 128 outputs of a
// wave.  (Factors past fp32's normal range lose what lies past it: a second
// multiplication by the other scale would stand beside every product, where the
// FMAs already hold the matrix cores up.)
//
// acrl_linear_fp8 is the same product with an epilogue: bias, activation and
// residual enter the fp32 sums before their one rounding.
#include <type_traits>

#include "activation.h"
#include "entry.h"

namespace acrl {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;  // elements (bytes) of K per scale

// Results of type T by way of the epilogue.
template <typename T>
struct Fused {};
struct ProductParams {
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  void* y;
  int64_t ldy;
  int M, N, K;
  int kb;                  // scale blocks of a row, ceil(K / 128)
  int n_mtiles, n_ntiles;
  int vec, whole;          // y's rows take stores of four values; of 16 bytes
};
struct LinearParams : ProductParams {
  const void* bias;        // [N] or NULL
  const void* res;         // [M, N], rows ldr apart, or NULL
  int64_t ldr;
  int act;
  int bias_f32, res_f32;   // else bf16
  int res_vec;             // the residual's rows take loads of four values, and of as many as a 16-byte store has
};
template <typename OUT>
struct Result {
  using type = OUT;
  using params = ProductParams;
  static constexpr bool fused = false;
};
template <typename T>
struct Result<Fused<T>> {
  using type = T;
  using params = LinearParams;
  static constexpr bool fused = true;
};
template <typename OUT>
using Params = typename Result<OUT>::params;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, int64_t bytes) {
  const uint32_t n = bytes > 0xFFFFFFFFll ? 0xFFFFFFFFu : (uint32_t)bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)n, 0x00020000);
}
// SIZE bytes a lane from a buffer into LDS: lane l writes lds_wave_base + SIZE l.
template <int SIZE>
__device__ __forceinline__ void buffer_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t voffset, uint32_t soffset,
                                              uint8_t* lds_wave_base) {
  auto* l = (__attribute__((address_space(3))) void*)lds_wave_base;
  if constexpr (SIZE == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, l, 16, (int)voffset, (int)soffset, 0, 0);
  else if constexpr (SIZE == 4) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, l, 4, (int)voffset, (int)soffset, 0, 0);
  else static_assert(SIZE == 16, "size must be 4 or 16");
}
// Workgroup barrier once this wave's loads (all but the N youngest) and LDS
// reads are complete.
template <int N>
__device__ __forceinline__ void wait_loads_and_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The same with the loads into registers still under way.
__device__ __forceinline__ void read_lds_and_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A block's sum, from zero.  The instruction aligns the 128 products to the
// largest before it adds them and so keeps fewer bits than fp32 sums would: over
// K = 4096 .. 13824, y before its rounding is 1.4e-5 off for normally distributed
// operands and 2.4e-5 .. 2.7e-5 where every 61st column is ten times as large,
// relative to its size, with no bias (toward 0 or from it: below 4e-8).  A bf16 y
// is rounded by far more: 1.6608e-3 from the exact one, 1.6606e-3 with fp32 sums.
// The FP8 instructions of 32 products have half its published rate.
__device__ __forceinline__ f32x4 mfma(const i32x8& a, const i32x8& b) {
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 127, 0, 127);
}

__device__ __forceinline__ void add(f32x4& acc, const f32x4& t, float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = fmaf(t[e], s, acc[e]);
}

// The sums stand here: the compiler would move the last products into the
// stores' branches, one after another.
template <int A, int B>
__device__ __forceinline__ void settle(f32x4 (&acc)[A][B]) {
#pragma unroll
  for (int i = 0; i < A; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) asm volatile("" : "+v"(acc[i][j]));
}

template <typename OUT>
using out4 = OUT __attribute__((ext_vector_type(4)));

// C consecutive values of an array of fp32 or bf16, as they are read.  Those that are not there count -0: added to any
// value, that leaves it as it is.
template <int C>
struct Piece {
  uint32_t raw[C];
  __device__ __forceinline__ float value(int e, bool f32) const {
    const float h = e % 2 ? bf16_hi(raw[e / 2]) : bf16_lo(raw[e / 2]);
    return f32 ? __uint_as_float(raw[e]) : h;
  }
  // values at .. at + C - 1, the first `left` of them
  __device__ __forceinline__ void read(const void* base, bool f32, int64_t at, int left, bool vec) {
    constexpr uint32_t kNone = 0x80000000u;
    if (base && left >= C && vec) {
      const uint32_t* q = static_cast<const uint32_t*>(base) + (f32 ? at : at / 2);
      using words = uint32_t __attribute__((ext_vector_type(C / 2)));  // (half a piece of fp32, a piece of bf16)
      const words u = *reinterpret_cast<const words*>(q);
#pragma unroll
      for (int i = 0; i < C / 2; ++i) raw[i] = u[i];
      if (f32) {
        const words v = *reinterpret_cast<const words*>(q + C / 2);
#pragma unroll
        for (int i = 0; i < C / 2; ++i) raw[C / 2 + i] = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < C; ++i) raw[i] = f32 || i % 2 ? kNone : kNone | kNone >> 16;
      if (!base) return;
      if (f32) {
#pragma unroll
        for (int i = 0; i < C; ++i)
          if (i < left) raw[i] = static_cast<const uint32_t*>(base)[at + i];
      } else {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
          const uint16_t* q = static_cast<const uint16_t*>(base) + at + 2 * i;
          const uint32_t lo = 2 * i < left ? q[0] : kNone >> 16, hi = 2 * i + 1 < left ? q[1] : kNone >> 16;
          raw[i] = hi << 16 | lo;
        }
      }
    }
  }
  // the residual's values n .. n + C - 1 of token m
  __device__ __forceinline__ void read(const LinearParams& p, int m, int n) {
    read(m < p.M ? p.res : nullptr, p.res_f32, (int64_t)m * p.ldr + n, p.N - n, p.res_vec);
  }
};

template <int C>
__device__ __forceinline__ void read_bias(const LinearParams& p, int n, float (&v)[C]) {
  Piece<C> b;
  b.read(p.bias, p.bias_f32, n, p.N - n, true);
#pragma unroll
  for (int e = 0; e < C; ++e) v[e] = b.value(e, p.bias_f32);
}

// Four consecutive outputs n .. n + 3 of token m.
template <typename RES>
__device__ __forceinline__ void store4(const Params<RES>& p, int m, int n, f32x4 v) {
  using OUT = typename Result<RES>::type;
  if (m >= p.M || n >= p.N) return;
  if constexpr (Result<RES>::fused) {
    // (in fp32.  A residual that is y itself is read by the lane that writes it, before it does)
    Piece<4> r;
    r.read(p, m, n);
    float b[4];
    read_bias(p, n, b);
    for_activation(p.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = activate<decltype(act)::value, std::is_same<OUT, float>::value>(v[e] + b[e]) + r.value(e, p.res_f32);
    });
  }
  OUT* y = static_cast<OUT*>(p.y) + (int64_t)m * p.ldy + n;
  const out4<OUT> o = __builtin_convertvector(v, out4<OUT>);
  if (p.vec && n + 3 < p.N) {
    *reinterpret_cast<out4<OUT>*>(y) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.N) y[i] = o[i];
  }
}

// The sums of a TM x TN tile (WM x WN waves) to y by way of LDS: a wave's
// lanes hold 16 tokens and write 8 or 16 bytes of each, which costs twice the
// time of rows written whole (4096 x 4096 of K = 256: 23 us, 9 without stores).
// With an epilogue they pass as fp32, and it runs where rows are written: its
// arrays are then read as wide as y is written, and its code stands once.
template <typename RES, int TN, int TM, int WN, int WM, int PARTS, int A, int B>
__device__ __forceinline__ void store_tile(const Params<RES>& p, uint8_t* lds, int m0, int n0, int wm, int wn,
                                           const f32x4 (&acc)[A][B]) {
  using OUT = typename Result<RES>::type;
  using IN = typename std::conditional<Result<RES>::fused, float, OUT>::type;
  constexpr int kPitch = TN * sizeof(IN) + 16, kPiece = 16 / sizeof(OUT), kPieces = TN / kPiece;  // (16: other banks)
  constexpr int kThreads = 64 * WN * WM, kRows = TM / PARTS;
  static_assert(WM % PARTS == 0 && kRows * kPieces % kThreads == 0, "whole parts");
  const int lane = threadIdx.x & 63, q = lane >> 4;
  // A lane's column is the same in every row it writes: its bias comes once, and the residual's pieces of a part are
  // under way while the sums pass through LDS (8192 x 13824 x 5120 and a bf16 residual: 545 us; each piece read where it is
  // added cost 40 more).
  constexpr int kIter = kRows * kPieces / kThreads;
  static_assert(!Result<RES>::fused || kThreads % kPieces == 0, "a lane keeps its column");
  const int c = threadIdx.x % kPieces, n = n0 + c * kPiece;
  float bias[kPiece];
  Piece<kPiece> res[Result<RES>::fused ? kIter : 1];
  if constexpr (Result<RES>::fused) read_bias<kPiece>(p, n, bias);
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
    if constexpr (Result<RES>::fused) {
#pragma unroll
      for (int k = 0; k < kIter; ++k) res[k].read(p, m0 + part * kRows + (k * kThreads + (int)threadIdx.x) / kPieces, n);
    }
    read_lds_and_barrier();
    if (wm / (WM / PARTS) == part) {
#pragma unroll
      for (int j = 0; j < B; ++j)
#pragma unroll
        for (int i = 0; i < A; ++i)
          *reinterpret_cast<out4<IN>*>(lds + (wm % (WM / PARTS) * (TM / WM) + j * 16 + (lane & 15)) * kPitch +
                                       (wn * (TN / WN) + i * 16 + 4 * q) * sizeof(IN)) =
              __builtin_convertvector(acc[i][j], out4<IN>);
    }
    __syncthreads();
    if constexpr (Result<RES>::fused) {
      const auto row = [&](auto act, int k) {
        const int r = (k * kThreads + threadIdx.x) / kPieces, m = m0 + part * kRows + r;
        if (m >= p.M || n >= p.N) return;
        const f32x4* from = reinterpret_cast<const f32x4*>(lds + r * kPitch + c * kPiece * sizeof(float));
        float v[kPiece];
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
          v[e] = activate<decltype(act)::value, std::is_same<OUT, float>::value>(from[e / 4][e % 4] + bias[e]);
        if (p.res) {
#pragma unroll
          for (int e = 0; e < kPiece; ++e) v[e] += res[k].value(e, p.res_f32);
        }
        using values = float __attribute__((ext_vector_type(kPiece)));
        using results = OUT __attribute__((ext_vector_type(kPiece)));
        const results o = __builtin_convertvector(__builtin_bit_cast(values, v), results);  // (two values an instruction)
        OUT* y = static_cast<OUT*>(p.y) + (int64_t)m * p.ldy + n;
        if (p.whole && n + kPiece <= p.N) {
          *reinterpret_cast<i32x4*>(y) = __builtin_bit_cast(i32x4, o);
        } else {
#pragma unroll
          for (int e = 0; e < kPiece; ++e)
            if (n + e < p.N) y[e] = o[e];
        }
      };
      for_activation(p.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kIter; ++k) row(act, k);
      });
      continue;
    }
#pragma unroll
    for (int k = 0; k < kRows * kPieces / kThreads; ++k) {
      const int at = k * kThreads + threadIdx.x, r = at / kPieces, c = at % kPieces;
      const int m = m0 + part * kRows + r, n = n0 + c * kPiece;
      const uint8_t* from = lds + r * kPitch + c * 16;
      OUT* y = static_cast<OUT*>(p.y) + (int64_t)m * p.ldy + n;
      if (m < p.M && n + kPiece <= p.N) *reinterpret_cast<i32x4*>(y) = *reinterpret_cast<const i32x4*>(from);
      else if (m < p.M)
        for (int e = 0; e < kPiece && n + e < p.N; ++e) y[e] = reinterpret_cast<const OUT*>(from)[e];
    }
  }
}

// The workgroup's tile.  Consecutive workgroups go to the 8 XCDs in turn; each
// XCD takes a contiguous range of tiles, ordered in bands of 8 token tiles
// with the output tile as the slow index, so that the 32 tiles its CUs work
// on at a time share 8 token tiles and 4 output tiles in its L2.
constexpr int kXcds = 8, kBand = 8;
__device__ __forceinline__ void tile_of(const ProductParams& p, int block, int& mt, int& nt) {
  const int tiles = p.n_mtiles * p.n_ntiles, per = tiles / kXcds, more = tiles % kXcds;
  const int xcd = block % kXcds, t = xcd * per + min(xcd, more) + block / kXcds;
  const int band = t / (kBand * p.n_ntiles), rest = t - band * kBand * p.n_ntiles;
  const int high = min(kBand, p.n_mtiles - band * kBand);
  nt = rest / high;
  mt = band * kBand + rest - nt * high;
}

// Tile of TN outputs x TM tokens a workgroup, WN x WM waves for each of KG
// groups.  K passes through LDS in ST stages of KG scale blocks, one a group
// (buffer -> LDS loads; W's rows of all groups, then x's), and the groups' sums
// are added at the end in their order.  Piece c (16 bytes) of row r lies at
// position c ^ (r / 2 mod 8) of the row's 128 bytes, and lane group q of a
// fragment takes pieces q and q + 4 (the products of a block may be summed in
// any order of k, as long as both operands have the same): LDS then serves a
// fragment's reads without bank conflicts.
//
// A stage's place is loaded again, one load behind each product, from the
// barrier on that ends its reads.  That barrier stands, row by row (AHEAD
// false), where a wave has its last operands of a turn in registers and a row
// of products still to issue, with the next turn's first operands read under
// those; or (AHEAD) at the turn's start, with all operands of the next turn read
// under this one's products, which takes twice their registers (128 x 128, 700 x
// 5120 x 13824: 64 us for 72; tiles of 64 and less gain nothing).  The
// loops have no branches: the compiler would move products past them, away from
// the reads of their operands.  The scales come C blocks at a time, between the
// turns.
//
// What bounds it.  A wave issues its instructions one by one, and address
// arithmetic beside the products counts in full: with descriptor, row group and
// bounds of each load known when it is compiled or once a turn, a turn of a
// 128 x 128 tile went from 158 instructions to 103, and times fell by 3 to 12 % at
// nearly all sizes.  Large tiles (16384 x 5120 x 13824: 952 us in a run of calls, 916 to
// 980, 2440 TFLOP/s; 1000 to 1020 on average of 25 from a cold start; counters): the
// matrix cores are busy for 2048 of a turn's 3250 cycles, at 1.83 GHz,
// to which the power limit brings the clock (2.4 without load); the four FMAs
// beside each product let it take 37 cycles for 32.  Smaller ones: loads alone,
// without products, take the same time while there are two stages (128 x 128
// tiles of two groups, 49 us for 0.4 GB by way of L2 at 700 x 4096 x 8192; 36 if
// all hit there), hence four stages (42; where all hit, loads reach 120 bytes a ns
// and CU with 32 KB under way).  Measured without gain (946 us): two or four loads
// behind a product (975, 980; a wave waits while the address unit is taken), one
// behind every second (946); waves that only load (0.6 to 1.08 of the speed);
// lines touched a turn or more ahead; bands of 4 or 16 token tiles; priorities.
template <typename OUT, int TN, int TM, int WN, int WM, int KG, int ST, int C, bool AHEAD>
__device__ __forceinline__ void tile_product(Params<OUT> p) {
  constexpr int NW = WN * WM * KG, AN = TN / WN / 16, BM = TM / WM / 16, kSteps = AN * BM;  // fragments of a wave
  constexpr int kRows = TN + TM, kStage = kRows * kBlock * KG, kLoads = kRows * KG / 8 / NW;
  constexpr int kStepLoads = (kLoads + kSteps - 1) / kSteps;  // behind each product
  constexpr int kStepReads = (AN + BM + kSteps * 3 / 4 - 1) / (kSteps * 3 / 4);  // (AHEAD) so that the last are early
  // the scales of C blocks lie in LDS at a time, twice: x's [TM][C], W's [TN / 128][C]; 64 floats a load
  constexpr int kParts = TM * C / 64, kChunk = (kParts + 1) * 256, kChunkTurns = C / KG;
  static_assert(kRows * KG % (8 * NW) == 0 && TN % 16 == 0 && TM * C % 64 == 0 && kRows % 16 == 0, "whole loads");
  static_assert((TN + kBlock - 1) / kBlock * C <= 64 && C % KG == 0, "one load of W's scales");
  // (they are older than ST - 2 stages' loads when they are read, so that no barrier need count them)
  static_assert(kChunkTurns >= ST && kChunkTurns % 2 == 0, "the next scales are there in time");
  static_assert(kBlock % (TN / WN) == 0, "a wave's outputs lie in one scale block");
  // (rows of products take W's operand from two places in turn: an even number of them ends where it began)
  static_assert(AN >= 2 && AN % 2 == 0 && kSteps % 4 == 0, "operands and products in turn");
  static_assert(KG == 1 || KG * TN * TM * 4 <= ST * kStage, "the groups' sums fit the stages");
  constexpr int kLds = ST * kStage + 2 * kChunk + 256;
  __shared__ __align__(1024) uint8_t lds[kLds];
  uint8_t* const lds_s = lds + ST * kStage;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wm = wave / WN % WM, g = wave / (WN * WM);
  int mt, nt;
  tile_of(p, blockIdx.x, mt, nt);
  const int n0 = nt * TN, m0 = mt * TM;
  const int last = p.kb - 1, tail = p.K - last * kBlock;  // bytes of the last block
  const int last_turn = (p.kb + KG - 1) / KG - 1;
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.w + (int64_t)n0 * p.K, (int64_t)(p.N - n0) * p.K);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x + (int64_t)m0 * p.K, (int64_t)(p.M - m0) * p.K);
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(p.xs + (int64_t)m0 * p.kb, (int64_t)(p.M - m0) * p.kb * 4);
  const int nb0 = n0 / kBlock, nb_last = (p.N - 1) / kBlock;
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.ws + (int64_t)nb0 * p.kb, (int64_t)(nb_last + 1 - nb0) * p.kb * 4);
  // Rows past the matrix repeat its last one (their results are not stored).  The last block is read as the row's last
  // 128 bytes, and blocks past it too; what of those belongs to the block before is cleared in the fragments (of a row
  // shorter than a block: the pieces past its end, which repeat its last one).  A lane's piece is the same in every load.
  constexpr int kSpan = 8 * NW, kWLoads = KG * TN / kSpan;  // rows of a load of all waves; loads of W
  static_assert(KG * TN % kSpan == 0 && KG * TM % kSpan == 0 && (TN % kSpan == 0 || kSpan % TN == 0) &&
                (TM % kSpan == 0 || kSpan % TM == 0), "a load is of W or of x, of whole groups or of one");
  const int piece = (lane & 7) ^ ((wave * 8 + (lane >> 3)) >> 1 & 7);
  const int last_at = max(p.K - kBlock, 0);
  uint32_t off[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const bool is_w = i < kWLoads;
    const int r = ((is_w ? i : i - kWLoads) * kSpan + wave * 8 + (lane >> 3)) % (is_w ? TN : TM);
    off[i] = (uint32_t)min(r, (is_w ? p.N - n0 : p.M - m0) - 1) * (uint32_t)p.K + min(16 * piece, p.K - 16);
  }
  uint8_t* const lds_w = lds + wave * 1024;
  auto load = [&](int turn, int at, int i) {  // into the stage `at` bytes from the first
    const bool is_w = i < kWLoads;
    const int k = is_w ? i : i - kWLoads, T = is_w ? TN : TM;
    const int group = T % kSpan == 0 ? k * kSpan / T : k * (kSpan / T) + wave * 8 / T;
    buffer_to_lds<16>(is_w ? rw : rx, off[i], min((turn * KG + group) * kBlock, last_at), lds_w + at + i * (kSpan * kBlock));
  };
  // The scales of blocks C c .. C c + C - 1, in parts of 64: x's, then W's; past those, into no one's place
  auto load_scales = [&](int c) {
#pragma unroll
    for (int i = 0; i <= kParts / NW; ++i) {
      const int part = i * NW + wave, k = min(C * c + lane % C, last);
      const bool is_w = part >= kParts;
      const int row = is_w ? min(lane / C, nb_last - nb0) : min(part * (64 / C) + lane / C, p.M - 1 - m0);
      buffer_to_lds<4>(is_w ? rv : rs, (uint32_t)(row * p.kb + k) * 4, 0,
                       part <= kParts ? lds_s + (c & 1) * kChunk + part * 256 : lds_s + 2 * kChunk);
    }
  };

  f32x4 acc[AN][BM] = {};
  const int q = lane >> 4, f = (lane >> 1) & 7;
  const int lo = (lane & 15) * kBlock + ((q ^ f) << 4), hi = lo ^ 64;  // pieces q and q + 4
  const int a_at = (g * TN + wn * (TN / WN)) * kBlock, b_at = (KG * TN + g * TM + wm * (TM / WM)) * kBlock;
  const int s_at = (wm * (TM / WM) + (lane & 15)) * C + g, w_at = TM * C + wn * (TN / WN) / kBlock * C + g;
  auto fragment = [&](int at) {
    const i32x4 u = *reinterpret_cast<const i32x4*>(lds + at + lo), v = *reinterpret_cast<const i32x4*>(lds + at + hi);
    return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  f32x4 t[4];          // the last products, which enter the sums three products later
  float s[BM], s_new[BM], w_new;
  auto scales = [&](int at) {
    const float* ss = reinterpret_cast<const float*>(lds_s + at);
#pragma unroll
    for (int j = 0; j < BM; ++j) s_new[j] = ss[s_at + j * 16 * C];
    w_new = ss[w_at];
  };
  auto next_scales = [&](int turn, int at) {  // where the scales of the turn after `turn` lie; at: its own
    return (turn + 1) % kChunkTurns == 0 ? (at >= kChunk ? 0 : kChunk) : at + KG * 4;
  };
  // in the last turn
  const bool mine = last_turn * KG + g <= last, cut_here = last_turn * KG + g == last, one = p.K < kBlock;
  const bool no_lo = cut_here & (one ? 16 * q >= tail : 16 * q < kBlock - tail);
  const bool no_hi = cut_here & (one ? 16 * q + 64 >= tail : 16 * q + 64 < kBlock - tail);
  auto cut = [&](i32x8 v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = no_lo ? 0 : v[e];
      v[e + 4] = no_hi ? 0 : v[e + 4];
    }
    return v;
  };
  if constexpr (AHEAD) {
    i32x8 a[2][AN], b[2][BM];
    // The products of a turn, whose operands are in a[P] and b[P]; MORE: with the reads of the next turn's
    auto block = [&](int turn, int st, int st_next, int ss_next, auto more, auto parity) {
      constexpr bool MORE = decltype(more)::value;
      constexpr int P = decltype(parity)::value;
      // this wave's reads of the turn's stage are done, all waves' and the loads of the next
      wait_loads_and_barrier<(ST - 2) * kLoads>();
#pragma unroll
      for (int i = 0; i < AN; ++i) asm volatile("" : "+v"(a[P][i]));
#pragma unroll
      for (int j = 0; j < BM; ++j) asm volatile("" : "+v"(b[P][j]));
      if (!MORE) {
#pragma unroll
        for (int i = 0; i < AN; ++i) a[P][i] = cut(a[P][i]);
#pragma unroll
        for (int j = 0; j < BM; ++j) b[P][j] = cut(b[P][j]);
      }
#pragma unroll
      for (int n = 0; n < kSteps; ++n) {
        const int i = n / BM, j = n % BM, d = (n + kSteps - 3) % kSteps;
        t[n & 3] = mfma(a[P][i], b[P][j]);
        add(acc[d / BM][d % BM], t[(n + 1) & 3], s[d % BM]);
        if (n == 2) {
#pragma unroll
          for (int k = 0; k < BM; ++k) s[k] = MORE || mine ? s_new[k] * w_new : 0.0f;
          if (MORE) scales(ss_next);
        }
        if (MORE) {
#pragma unroll
          for (int k = 0; k < kStepReads; ++k) {
            const int f = n * kStepReads + k;
            if (f < BM) b[P ^ 1][f] = fragment(st_next + b_at + f * 16 * kBlock);
            else if (f < BM + AN) a[P ^ 1][f - BM] = fragment(st_next + a_at + (f - BM) * 16 * kBlock);
          }
#pragma unroll
          for (int k = 0; k < kStepLoads; ++k)
            if (n * kStepLoads + k < kLoads) load(turn + ST, st, n * kStepLoads + k);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    load_scales(0);
#pragma unroll
    for (int k = 0; k < ST; ++k)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(k, k * kStage, i);
    wait_loads_and_barrier<(ST - 1) * kLoads>();
#pragma unroll
    for (int i = 0; i < AN; ++i) a[0][i] = fragment(a_at + i * 16 * kBlock);
#pragma unroll
    for (int j = 0; j < BM; ++j) b[0][j] = fragment(b_at + j * 16 * kBlock);
    scales(0);
#pragma unroll
    for (int j = 0; j < BM; ++j) s[j] = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = f32x4{};
    int st = 0, ss = 0, turn = 0;
    auto next = [&](int k) { return k == (ST - 1) * kStage ? 0 : k + kStage; };
    while (turn + 2 <= last_turn) {
      load_scales(turn / kChunkTurns + 1);
      for (const int end = min(last_turn, turn + kChunkTurns); turn + 2 <= end; turn += 2) {
        const int s1 = next(st), s2 = next(s1), ss1 = ss + KG * 4, ss2 = next_scales(turn + 1, ss1);
        block(turn, st, s1, ss1, std::true_type{}, std::integral_constant<int, 0>{});
        block(turn + 1, s1, s2, ss2, std::true_type{}, std::integral_constant<int, 1>{});
        st = s2;
        ss = ss2;
      }
    }
    if (turn < last_turn) {
      block(turn, st, next(st), ss + KG * 4, std::true_type{}, std::integral_constant<int, 0>{});
      block(last_turn, next(st), 0, 0, std::false_type{}, std::integral_constant<int, 1>{});
    } else {
      block(last_turn, st, 0, 0, std::false_type{}, std::integral_constant<int, 0>{});
    }
  } else {
    i32x8 a[2], b[BM];
    // The products of a turn, whose b and a[0] are there; MORE: with the reads of the next turn's, else it is the last
    auto block = [&](int turn, int st_prev, int st, int st_next, int ss_next, auto more) {
      constexpr bool MORE = decltype(more)::value;
      if (!MORE) {
        a[0] = cut(a[0]);
#pragma unroll
        for (int j = 0; j < BM; ++j) b[j] = cut(b[j]);
      }
#pragma unroll
      for (int i = 0; i < AN; ++i) {
        if (MORE && i == AN - 1) {
          // all waves' loads of the next turn and reads of this one are done
          wait_loads_and_barrier<(ST - 2) * kLoads>();
          a[0] = fragment(st_next + a_at);
        }
#pragma unroll
        for (int j = 0; j < BM; ++j) {
          const int n = i * BM + j, d = (n + kSteps - 3) % kSteps;  // the product made, and the one added (n < 3: the turn before's)
          t[n & 3] = mfma(a[i & 1], b[j]);
          if (j == 0 && i + 1 < AN) {
            const i32x8 v = fragment(st + a_at + (i + 1) * 16 * kBlock);
            a[(i + 1) & 1] = MORE ? v : cut(v);
          }
          add(acc[d / BM][d % BM], t[(n + 1) & 3], s[d % BM]);
          if (n == 2) {
#pragma unroll
            for (int k = 0; k < BM; ++k) s[k] = MORE || mine ? s_new[k] * w_new : 0.0f;
          }
          if (MORE && i == AN - 1) b[j] = fragment(st_next + b_at + j * 16 * kBlock);
          if (MORE && n == kSteps - 1) scales(ss_next);
          // into this turn's place, the loads of turn + ST from the barrier on
          if (MORE) {
#pragma unroll
            for (int k = 0; k < kStepLoads; ++k) {
              const int at = ((n + BM) % kSteps) * kStepLoads + k;
              if (at < kLoads) i == AN - 1 ? load(turn + ST, st, at) : load(turn + ST - 1, st_prev, at);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    load_scales(0);
#pragma unroll
    for (int k = 0; k < ST - 1; ++k)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(k, k * kStage, i);
    wait_loads_and_barrier<(ST - 2) * kLoads>();
#pragma unroll
    for (int i = 0; i < (BM * kStepLoads < kLoads ? BM * kStepLoads : kLoads); ++i) load(ST - 1, (ST - 1) * kStage, i);
    a[0] = fragment(a_at);
#pragma unroll
    for (int j = 0; j < BM; ++j) b[j] = fragment(b_at + j * 16 * kBlock);
    scales(0);
#pragma unroll
    for (int j = 0; j < BM; ++j) s[j] = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = f32x4{};
    int st_prev = (ST - 1) * kStage, st = 0, ss = 0;
    for (int turn = 0; turn < last_turn;) {
      load_scales(turn / kChunkTurns + 1);
      for (const int end = min(last_turn, turn + kChunkTurns); turn < end; ++turn) {
        const int st_next = st == (ST - 1) * kStage ? 0 : st + kStage;
        ss = next_scales(turn, ss);
        block(turn, st_prev, st, st_next, ss, std::true_type{});
        st_prev = st;
        st = st_next;
      }
    }
    block(last_turn, st_prev, st, 0, 0, std::false_type{});
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) add(acc[(kSteps - 3 + e) / BM][(kSteps - 3 + e) % BM], t[(kSteps - 3 + e) & 3], s[(kSteps - 3 + e) % BM]);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads past the last turn are still under way into LDS)
  settle(acc);
  if constexpr (KG > 1) {
    // the groups' sums through LDS: wave w adds every NW-th of the WN WM AN BM blocks of 16 x 16
    constexpr int kBlocks = WN * WM * AN * BM;
    f32x4* const red = reinterpret_cast<f32x4*>(lds);
    wait_loads_and_barrier<0>();
#pragma unroll
    for (int i = 0; i < AN; ++i)
#pragma unroll
      for (int j = 0; j < BM; ++j)
        red[((g * kBlocks) + ((wm * WN + wn) * AN + i) * BM + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int e = wave; e < kBlocks; e += NW) {
      f32x4 v = red[e * 64 + lane];
#pragma unroll
      for (int h = 1; h < KG; ++h) v += red[(h * kBlocks + e) * 64 + lane];
      const int j = e % BM, i = e / BM % AN, n = e / (BM * AN) % WN, m = e / (BM * AN * WN);
      store4<OUT>(p, m0 + m * (TM / WM) + j * 16 + (lane & 15), n0 + n * (TN / WN) + i * 16 + 4 * q, v);
    }
  } else if (Result<OUT>::fused || p.whole) {
    constexpr int kValue = Result<OUT>::fused ? 4 : (int)sizeof(OUT);
    constexpr int kParted = TM * (TN * kValue + 16) <= kLds ? 1 : 2;
    static_assert(TM / kParted * (TN * kValue + 16) <= kLds, "a part of the tile fits");
    store_tile<OUT, TN, TM, WN, WM, kParted>(p, lds, m0, n0, wm, wn, acc);
  } else {
#pragma unroll
    for (int j = 0; j < BM; ++j) {
      const int m = m0 + wm * (TM / WM) + j * 16 + (lane & 15);
#pragma unroll
      for (int i = 0; i < AN; ++i) store4<OUT>(p, m, n0 + wn * (TN / WN) + i * 16 + 4 * q, acc[i][j]);
    }
  }
}
template <typename OUT, int TN, int TM, int WN, int WM, int KG, int ST, int C, bool AHEAD>
__global__ __launch_bounds__(64 * WN * WM * KG, 2) void product_tile_kernel(ProductParams p) {
  tile_product<OUT, TN, TM, WN, WM, KG, ST, C, AHEAD>(p);
}
template <typename OUT, int TN, int TM, int WN, int WM, int KG, int ST, int C, bool AHEAD>
__global__ __launch_bounds__(64 * WN * WM * KG, 2) void linear_tile_kernel(LinearParams p) {
  tile_product<Fused<OUT>, TN, TM, WN, WM, KG, ST, C, AHEAD>(p);
}

// Up to 16 tokens: the weights' stream is the whole work (16 x 24576 x 4096: 26.2 us,
// 3.9 TB/s from HBM, 22.3 where the weights lie in the 256 MB cache; 1 x 4096 x 4096: 6.3
// us, 2.7 TB/s, and 4.6: two rounds of loads for each wave), and a workgroup takes
// 16 AN outputs so that many of them share it out.  Its NW waves take every
// NW-th scale block each, U of them at a time, straight into registers: 16-byte
// pieces q and q + 4 of a row's 128 bytes for lane group q, so that a load takes
// 64 contiguous bytes of each row (the products of a block may be summed in any
// order of k, as long as both operands have the same).  The waves' sums are added
// through LDS in their order.
template <typename OUT, int AN, int NW, int U>
__device__ __forceinline__ void rows_product(Params<OUT> p) {
  __shared__ f32x4 red[NW][AN][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16 * AN, q = lane >> 4;
  const int last = p.kb - 1, tail = p.K - last * kBlock;
  const uint8_t* pw[AN];
#pragma unroll
  for (int i = 0; i < AN; ++i) pw[i] = p.w + (int64_t)min(n0 + 16 * i + (lane & 15), p.N - 1) * p.K;
  const int64_t m = min(lane & 15, p.M - 1);
  const uint8_t* const px = p.x + m * p.K;
  const float* const ps = p.xs + m * p.kb;
  const float* const ws = p.ws + (int64_t)(n0 / kBlock) * p.kb;  // (16 AN divides 128)
  f32x4 acc[AN] = {};
  for (int k0 = wave; k0 < p.kb; k0 += NW * U) {
    i32x4 a[U][AN][2], b[U][2];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // blocks past the last repeat it, pieces past its end its first; neither is used
      const int kb = min(k0 + u * NW, last);
      const int o0 = kb * kBlock + (kb == last && 16 * q >= tail ? 0 : 16 * q);
      const int o1 = kb * kBlock + (kb == last && 16 * q + 64 >= tail ? 0 : 16 * q + 64);
#pragma unroll
      for (int i = 0; i < AN; ++i) {
        a[u][i][0] = *reinterpret_cast<const i32x4*>(pw[i] + o0);
        a[u][i][1] = *reinterpret_cast<const i32x4*>(pw[i] + o1);
      }
      b[u][0] = *reinterpret_cast<const i32x4*>(px + o0);
      b[u][1] = *reinterpret_cast<const i32x4*>(px + o1);
      s[u] = ps[kb] * ws[kb];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = k0 + u * NW;
      if (kb > last) break;
      const bool no0 = kb == last && 16 * q >= tail, no1 = kb == last && 16 * q + 64 >= tail;
      auto operand = [&](i32x4 (&h)[2]) {
        const i32x4 zero = {0, 0, 0, 0};
        return __builtin_shufflevector(no0 ? zero : h[0], no1 ? zero : h[1], 0, 1, 2, 3, 4, 5, 6, 7);
      };
      const i32x8 bf = operand(b[u]);
#pragma unroll
      for (int i = 0; i < AN; ++i) add(acc[i], mfma(operand(a[u][i]), bf), s[u]);
    }
  }
#pragma unroll
  for (int i = 0; i < AN; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  for (int t = wave; t < AN; t += NW) {
    f32x4 v = red[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += red[w][t][lane];
    store4<OUT>(p, lane & 15, n0 + 16 * t + 4 * q, v);
  }
}
template <typename OUT, int AN, int NW, int U>
__global__ __launch_bounds__(64 * NW, 2) void product_rows_kernel(ProductParams p) {
  rows_product<OUT, AN, NW, U>(p);
}
template <typename OUT, int AN, int NW, int U>
__global__ __launch_bounds__(64 * NW, 2) void linear_rows_kernel(LinearParams p) {
  rows_product<Fused<OUT>, AN, NW, U>(p);
}

template <typename OUT, int AN, int NW, int U>
hipError_t launch_rows(const Params<OUT>& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.N + 16 * AN - 1) / (16 * AN)));
  using T = typename Result<OUT>::type;
  if constexpr (Result<OUT>::fused) hipLaunchKernelGGL((linear_rows_kernel<T, AN, NW, U>), grid, dim3(64 * NW), 0, s, p);
  else hipLaunchKernelGGL((product_rows_kernel<T, AN, NW, U>), grid, dim3(64 * NW), 0, s, p);
  return hipGetLastError();
}

template <typename OUT, int TN, int TM, int WN, int WM, int KG, int ST, int C, bool AHEAD>
hipError_t launch_tiles(Params<OUT> p, hipStream_t s) {
  p.n_ntiles = (p.N + TN - 1) / TN;
  p.n_mtiles = (p.M + TM - 1) / TM;
  const dim3 grid((unsigned)(p.n_ntiles * (int64_t)p.n_mtiles)), threads(64 * WN * WM * KG);
  using T = typename Result<OUT>::type;
  if constexpr (Result<OUT>::fused)
    hipLaunchKernelGGL((linear_tile_kernel<T, TN, TM, WN, WM, KG, ST, C, AHEAD>), grid, threads, 0, s, p);
  else
    hipLaunchKernelGGL((product_tile_kernel<T, TN, TM, WN, WM, KG, ST, C, AHEAD>), grid, threads, 0, s, p);
  return hipGetLastError();
}

// The tilings and what they take: `turn` us for KG scale blocks of every tile
// of a round (a tile a CU), `round` us beside them: fits to the times of 60
// sizes (M 24 .. 4096; N x K 4096 x 4096, 24576 x 4096, 5120 x 13824, 1024 x 5120,
// 2048 x 2048), at each of which but one they choose the fastest of the seven.
// How far apart those are: 64 x 4096 x 4096 6.9 us by the first, 17.4 by the
// fifth; 700 x 4096 x 4096 20.5 by the fifth, 50 by the last; 1500 x 4096 x 4096 32.5
// by the sixth, 51 by the last; 4096 x 4096 x 4096 60 by the last, 72 by the sixth, 173
// by the third.  Of the same N x K at M 17, 20, 23, 32, 48 and 64, with weights from the
// cache and from HBM, they choose the fastest at all but 5120 x 13824 of up to 32 tokens
// from the cache (16.9 us by the second, 19.7 by the first, which is the faster one
// from HBM: 25.1 to 27.5).
template <typename OUT>
struct Variant {
  int tn, tm, kg;
  float turn, round;
  hipError_t (*launch)(Params<OUT>, hipStream_t);
};
constexpr int kCus = 256;
template <typename OUT>
float cost(const Variant<OUT>& v, const ProductParams& p) {
  const int64_t tiles = (int64_t)((p.N + v.tn - 1) / v.tn) * ((p.M + v.tm - 1) / v.tm);
  return (float)((tiles + kCus - 1) / kCus) * ((float)((p.kb + v.kg - 1) / v.kg) * v.turn + v.round);
}

template <typename OUT>
hipError_t launch_product(const Params<OUT>& p, hipStream_t s) {
  // Up to 16 tokens: 16 outputs a workgroup while that is needed to have workgroups for the CUs, 32 from there on.
  // With 16 / 32, M 1, 8 and 16, K 2048, 4096 and 13824, weights from the cache: N = 4096, K = 4096 4.8 / 6.4, 6.0 / 7.8,
  // 7.0 / 8.9 us; N = 5120, K = 13824 18.2 / 16.3, 24.5 / 19.0, 29.8 / 21.8; every K and N 1024 .. 24576, from HBM too,
  // goes the same way or is within 5 %, but N = 12288 of up to 8 tokens (1 x 12288 x 13824: 26.8 / 32.9)
  if (p.M <= 16) return p.N < 20 * kCus ? launch_rows<OUT, 1, 8, 2>(p, s) : launch_rows<OUT, 2, 8, 2>(p, s);
  static const Variant<OUT> variants[] = {
      {32, 32, 8, 1.179f, 2.13f, launch_tiles<OUT, 32, 32, 1, 1, 8, 2, 32, false>},
      {64, 32, 4, 0.680f, 2.42f, launch_tiles<OUT, 64, 32, 2, 1, 4, 3, 16, false>},
      {64, 64, 2, 0.487f, 2.92f, launch_tiles<OUT, 64, 64, 2, 2, 2, 4, 16, false>},
      {128, 64, 2, 0.756f, 2.59f, launch_tiles<OUT, 128, 64, 2, 2, 2, 3, 8, false>},
      {128, 128, 1, 0.541f, 3.06f, launch_tiles<OUT, 128, 128, 2, 4, 1, 4, 8, true>},
      {256, 128, 1, 0.878f, 4.04f, launch_tiles<OUT, 256, 128, 4, 2, 1, 3, 8, false>},
      {256, 256, 1, 1.531f, 3.54f, launch_tiles<OUT, 256, 256, 2, 4, 1, 2, 8, false>},
  };
  const Variant<OUT>* best = variants;
  for (const Variant<OUT>& v : variants)
    if (cost(v, p) < cost(*best, p)) best = &v;
  return best->launch(p, s);
}

acrl_status validate_product(const acrl_matmul_desc* d) {
  ACRL_REQUIRE(d, "desc is NULL");
  ACRL_REQUIRE(d->M >= 0 && d->M < ((int64_t)1 << 26), "M = %lld out of range", (long long)d->M);
  ACRL_REQUIRE(d->N > 0 && d->N < ((int64_t)1 << 26), "N = %lld out of range", (long long)d->N);
  ACRL_REQUIRE(d->K > 0 && d->K % 32 == 0 && d->K <= ((int64_t)1 << 22),
               "K = %lld must be a positive multiple of 32, at most 2^22", (long long)d->K);
  ACRL_REQUIRE(d->ldy >= d->N, "ldy = %lld must be >= N", (long long)d->ldy);
  ACRL_REQUIRE(d->y_type == ACRL_OUT_BF16 || d->y_type == ACRL_OUT_F32, "y_type %d unknown", d->y_type);
  // a launch holds fewer than 2^32 threads
  ACRL_REQUIRE(((d->M + 127) / 128) * ((d->N + 127) / 128) < ((int64_t)1 << 23), "M x N too large");
  ACRL_REQUIRE(d->wq && d->w_scales, "wq and w_scales are required");
  ACRL_REQUIRE(aligned16(d->wq) && ((uintptr_t)d->w_scales & 3u) == 0, "wq or w_scales is misaligned");
  if (d->M > 0) {
    ACRL_REQUIRE(d->xq && d->x_scales && d->y, "xq, x_scales and y are required");
    ACRL_REQUIRE(aligned16(d->xq) && aligned16(d->y) && ((uintptr_t)d->x_scales & 3u) == 0,
                 "xq, y or x_scales is misaligned");
  }
  return ACRL_OK;
}

template <typename P>
P product_params(const acrl_matmul_desc* d) {
  P p{};
  p.x = static_cast<const uint8_t*>(d->xq);
  p.xs = d->x_scales;
  p.w = static_cast<const uint8_t*>(d->wq);
  p.ws = d->w_scales;
  p.y = d->y;
  p.ldy = d->ldy;
  p.M = (int)d->M;
  p.N = (int)d->N;
  p.K = (int)d->K;
  p.kb = (int)((d->K + kBlock - 1) / kBlock);
  p.vec = d->ldy % 4 == 0;
  p.whole = d->ldy % (d->y_type == ACRL_OUT_BF16 ? 8 : 4) == 0;
  return p;
}

}  // namespace
}  // namespace acrl

extern "C" {

acrl_status acrl_matmul_fp8(const acrl_matmul_desc* d, void* stream) {
  acrl_status st = acrl::validate_product(d);
  if (st == ACRL_OK) st = acrl::check_device();
  if (st != ACRL_OK || d->M == 0) return st;
  const acrl::ProductParams p = acrl::product_params<acrl::ProductParams>(d);
  const hipStream_t s = (hipStream_t)stream;
  return acrl::hip_status(
      d->y_type == ACRL_OUT_BF16 ? acrl::launch_product<__bf16>(p, s) : acrl::launch_product<float>(p, s),
      "acrl_matmul_fp8 launch");
}

acrl_status acrl_linear_fp8(const acrl_linear_desc* l, void* stream) {
  ACRL_REQUIRE(l, "desc is NULL");
  const acrl_matmul_desc* d = &l->product;
  acrl_status st = acrl::validate_product(d);
  if (st != ACRL_OK) return st;
  ACRL_REQUIRE(l->activation >= ACRL_ACT_NONE && l->activation <= ACRL_ACT_GELU_TANH, "activation %d unknown", l->activation);
  if (l->bias) {
    ACRL_REQUIRE(l->bias_type == ACRL_OUT_BF16 || l->bias_type == ACRL_OUT_F32, "bias_type %d unknown", l->bias_type);
    ACRL_REQUIRE(acrl::aligned16(l->bias), "bias must be 16-byte aligned");
  }
  if (l->residual) {
    ACRL_REQUIRE(l->residual_type == ACRL_OUT_BF16 || l->residual_type == ACRL_OUT_F32, "residual_type %d unknown",
                 l->residual_type);
    const int64_t most = (int64_t)1 << 34;  // (so that bytes of whole matrices fit 63 bits)
    ACRL_REQUIRE(l->ldr >= d->N && l->ldr < most && d->ldy < most, "ldr = %lld must lie in [N, 2^34), ldy = %lld below it",
                 (long long)l->ldr, (long long)d->ldy);
    ACRL_REQUIRE(acrl::aligned16(l->residual), "residual must be 16-byte aligned");
    ACRL_REQUIRE(!acrl::overlaps(l->residual, l->ldr, l->residual_type, d->y, d->ldy, d->y_type, d->M, d->N),
                 "the residual overlaps y without being y itself");
  }
  st = acrl::check_device();
  if (st != ACRL_OK || d->M == 0) return st;
  acrl::LinearParams p = acrl::product_params<acrl::LinearParams>(d);
  p.bias = l->bias;
  p.bias_f32 = l->bias_type == ACRL_OUT_F32;
  p.res = l->residual;
  p.ldr = l->ldr;
  p.res_f32 = l->residual_type == ACRL_OUT_F32;
  p.res_vec = l->ldr % (p.res_f32 ? 4 : 8) == 0;
  p.act = l->activation;
  const hipStream_t s = (hipStream_t)stream;
  return acrl::hip_status(d->y_type == ACRL_OUT_BF16 ? acrl::launch_product<acrl::Fused<__bf16>>(p, s)
                                                     : acrl::launch_product<acrl::Fused<float>>(p, s),
                          "acrl_linear_fp8 launch");
}

void acrl_abi_operator_struct_sizes(size_t* matmul_desc, size_t* policy_loss_desc, size_t* preference_desc) {
  if (matmul_desc) *matmul_desc = sizeof(acrl_matmul_desc);
  if (policy_loss_desc) *policy_loss_desc = sizeof(acrl_policy_loss_desc);
  if (preference_desc) *preference_desc = sizeof(acrl_preference_desc);
}

void acrl_abi_decode_struct_sizes(size_t* linear_desc, size_t* moe_desc, size_t* beam_desc, size_t* reorder_desc) {
  if (linear_desc) *linear_desc = sizeof(acrl_linear_desc);
  if (moe_desc) *moe_desc = sizeof(acrl_moe_desc);
  if (beam_desc) *beam_desc = sizeof(acrl_beam_desc);
  if (reorder_desc) *reorder_desc = sizeof(acrl_reorder_desc);
}

}  // extern "C"
