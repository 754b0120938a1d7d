// product.hip -- y = x W^T of FP8 operands with one scale per 128 elements of
// x's rows and per 128 x 128 block of W.
//
// Computed transposed, y^T = W x^T: W's rows are the A operand and x's rows
// the B operand of v_mfma_f32_16x16x128_f8f6f4, so a lane of a 16 x 16 result
// holds ONE token (column) and four consecutive outputs.  One instruction sums
// a whole scale block; its result then enters the fp32 accumulators with one
// FMA a value, whose factor x_scale w_scale is one number a lane: the token is
// the lane's own and the weight's scale is the same for all 128 outputs of a
// wave.
#include "entry.h"

namespace acrl {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;  // elements (bytes) of K per scale

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
  int vec;                 // y's rows take the vector stores
};

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

__device__ __forceinline__ f32x4 mfma(const i32x8& a, const i32x8& b) {
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 127, 0, 127);
}

__device__ __forceinline__ uint32_t bf16_rne(float f) {  // NaN stays NaN (quiet)
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (u >> 16) | 0x40u;
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// Four consecutive outputs n .. n + 3 of token m.
template <typename OUT>
__device__ __forceinline__ void store4(const ProductParams& p, int m, int n, const f32x4& v) {
  if (m >= p.M || n >= p.N) return;
  OUT* y = static_cast<OUT*>(p.y) + (int64_t)m * p.ldy + n;
  if constexpr (sizeof(OUT) == 2) {
    if (p.vec && n + 3 < p.N) {
      *reinterpret_cast<uint2*>(y) = make_uint2(bf16_rne(v[0]) | bf16_rne(v[1]) << 16, bf16_rne(v[2]) | bf16_rne(v[3]) << 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < p.N) y[i] = (OUT)bf16_rne(v[i]);
    }
  } else {
    if (p.vec && n + 3 < p.N) {
      *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < p.N) y[i] = v[i];
    }
  }
}

// Tile of TN outputs x TM tokens a workgroup, WN x WM waves, K in blocks of
// 128 bytes through two stages of LDS (buffer -> LDS loads, one barrier a
// block).  Piece c (16 bytes) of row r lies at position c ^ (r / 2 mod 8) of
// the row's 128 bytes: the 16 rows of a fragment then read 16 different
// 16-byte columns of LDS's 64 banks.
template <typename OUT, int TN, int TM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM) void product_tile_kernel(ProductParams p) {
  constexpr int NW = WN * WM, AN = TN / WN / 16, BM = TM / WM / 16;  // 16-row fragments of a wave
  constexpr int kStage = (TN + TM) * kBlock, kLoads = (TN + TM) / 8 / NW;
  static_assert(kBlock % (TN / WN) == 0, "a wave's outputs lie in one scale block");
  __shared__ __align__(1024) uint8_t lds[2 * kStage + 2 * TM * 4];
  float* const lds_s = reinterpret_cast<float*>(lds + 2 * kStage);  // x's scales of the two stages
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const int nt = blockIdx.x % p.n_ntiles, mt = blockIdx.x / p.n_ntiles;
  const int n0 = nt * TN, m0 = mt * TM;
  const int last = p.kb - 1, tail = p.K - last * kBlock;  // bytes of the last block

  const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.w + (int64_t)n0 * p.K, (int64_t)(p.N - n0) * p.K);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x + (int64_t)m0 * p.K, (int64_t)(p.M - m0) * p.K);
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(p.xs + (int64_t)m0 * p.kb, (int64_t)(p.M - m0) * p.kb * 4);
  // rows past the matrix repeat its last one; their results are not stored
  uint32_t off[kLoads];
  int piece[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = (i * NW + wave) * 8 + (lane >> 3);  // row of the stage: W's TN, then x's TM
    const int row = r < TN ? min(r, p.N - 1 - n0) : min(r - TN, p.M - 1 - m0);
    piece[i] = (lane & 7) ^ ((r >> 1) & 7);
    off[i] = (uint32_t)row * (uint32_t)p.K + 16 * piece[i];
  }
  const uint32_t s_off = (uint32_t)min((int)(threadIdx.x % TM), p.M - 1 - m0) * (uint32_t)p.kb * 4;

  auto load = [&](int kb) {
    uint8_t* stage = lds + (kb & 1) * kStage;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      // pieces past the row's end (last block) read its block's first one; the fragments there are cleared
      const uint32_t o = kb == last && 16 * piece[i] >= tail ? off[i] - 16 * piece[i] : off[i];
      const bool is_w = (i * NW + wave) * 8 < TN;
      buffer_to_lds<16>(is_w ? rw : rx, o, kb * kBlock, stage + (i * NW + wave) * 1024);
    }
    if (wave < TM / 64)
      buffer_to_lds<4>(rs, s_off, kb * 4, lds + 2 * kStage + (kb & 1) * TM * 4 + wave * 256);
  };

  f32x4 acc[AN][BM] = {};
  const int q = lane >> 4, f = (lane >> 1) & 7;
  const int lo = (lane & 15) * kBlock + (((2 * q) ^ f) << 4), hi = (lane & 15) * kBlock + (((2 * q + 1) ^ f) << 4);
  const float* const ws = p.ws + (int64_t)min((n0 + wn * (TN / WN)) / kBlock, (p.N - 1) / kBlock) * p.kb;
  load(0);
  for (int kb = 0; kb < p.kb; ++kb) {
    wait_loads_and_barrier<0>();
    if (kb < last) load(kb + 1);
    const uint8_t* sw = lds + (kb & 1) * kStage + wn * (TN / WN) * kBlock;
    const uint8_t* sx = lds + (kb & 1) * kStage + (TN + wm * (TM / WM)) * kBlock;
    const bool empty = kb == last && 32 * q >= tail;  // (K is a multiple of 32: a lane's 32 bytes are all in or all out)
    auto fragment = [&](const uint8_t* rows) {
      const i32x4 u = *reinterpret_cast<const i32x4*>(rows + lo), v = *reinterpret_cast<const i32x4*>(rows + hi);
      i32x8 r = __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
      if (empty) r = i32x8{};
      return r;
    };
    const float w_scale = ws[kb];
    i32x8 b[BM];
    float s[BM];
#pragma unroll
    for (int j = 0; j < BM; ++j) {
      b[j] = fragment(sx + j * 16 * kBlock);
      s[j] = lds_s[(kb & 1) * TM + wm * (TM / WM) + j * 16 + (lane & 15)] * w_scale;
    }
#pragma unroll
    for (int i = 0; i < AN; ++i) {
      const i32x8 a = fragment(sw + i * 16 * kBlock);
#pragma unroll
      for (int j = 0; j < BM; ++j) {
        const f32x4 t = mfma(a, b[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[e], s[j], acc[i][j][e]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < BM; ++j) {
    const int m = m0 + wm * (TM / WM) + j * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < AN; ++i) store4<OUT>(p, m, n0 + wn * (TN / WN) + i * 16 + 4 * q, acc[i][j]);
  }
}

template <typename OUT>
hipError_t launch_product(ProductParams p, hipStream_t s) {
  constexpr int TN = 128, TM = 128;
  p.n_ntiles = (p.N + TN - 1) / TN;
  p.n_mtiles = (p.M + TM - 1) / TM;
  hipLaunchKernelGGL((product_tile_kernel<OUT, TN, TM, 2, 2>), dim3((unsigned)(p.n_ntiles * (int64_t)p.n_mtiles)),
                     dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace
}  // namespace acrl

extern "C" {

acrl_status acrl_matmul_fp8(const acrl_matmul_desc* d, void* stream) {
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
  ACRL_REQUIRE(acrl::aligned16(d->wq) && ((uintptr_t)d->w_scales & 3u) == 0, "wq or w_scales is misaligned");
  if (d->M > 0) {
    ACRL_REQUIRE(d->xq && d->x_scales && d->y, "xq, x_scales and y are required");
    ACRL_REQUIRE(acrl::aligned16(d->xq) && acrl::aligned16(d->y) && ((uintptr_t)d->x_scales & 3u) == 0,
                 "xq, y or x_scales is misaligned");
  }
  acrl_status st = acrl::check_device();
  if (st != ACRL_OK || d->M == 0) return st;
  acrl::ProductParams p{};
  p.x = static_cast<const uint8_t*>(d->xq);
  p.xs = d->x_scales;
  p.w = static_cast<const uint8_t*>(d->wq);
  p.ws = d->w_scales;
  p.y = d->y;
  p.ldy = d->ldy;
  p.M = (int)d->M;
  p.N = (int)d->N;
  p.K = (int)d->K;
  p.kb = (int)((d->K + acrl::kBlock - 1) / acrl::kBlock);
  p.vec = d->ldy % 4 == 0;
  const hipStream_t s = (hipStream_t)stream;
  return acrl::hip_status(
      d->y_type == ACRL_OUT_BF16 ? acrl::launch_product<uint16_t>(p, s) : acrl::launch_product<float>(p, s),
      "acrl_matmul_fp8 launch");
}

void acrl_abi_operator_struct_sizes(size_t* matmul_desc, size_t* policy_loss_desc, size_t* preference_desc) {
  if (matmul_desc) *matmul_desc = sizeof(acrl_matmul_desc);
  if (policy_loss_desc) *policy_loss_desc = sizeof(acrl_policy_loss_desc);
  if (preference_desc) *preference_desc = sizeof(acrl_preference_desc);
}

}  // extern "C"
