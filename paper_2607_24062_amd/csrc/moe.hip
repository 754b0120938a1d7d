// moe.hip -- a mixture-of-experts layer for a few tokens: router, choice of the
// experts, their gated products and the weighted sum.
//
//   l = R x (64 bits), s = softmax(l) or sigmoid(l), the top_k largest s + bias
//   y = residual + sum_j w_j Wout[e_j] (act(Wgate[e_j] x) * (Wup[e_j] x))
//
// The experts' FP8 weights are the bytes that count: each is read once, straight
// into registers, by the experts that a token chose alone.  Activations stay
// bf16 (x) and bf16 + bf16 (what lies between the two products): with a few
// columns in each product the matrix cores are idle, so nothing is gained by
// quantizing them.  E4M3 codes become bf16 exactly, products of 128 columns are
// summed by bf16 matrix instructions from zero and enter the fp32 sums with the
// block's scale by one FMA each.
#include "activation.h"
#include "entry.h"

namespace acrl {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;        // columns per scale
constexpr int kMaxTokens = 128, kMaxK = 16, kMaxExperts = 512;
constexpr int kMaxPairs = kMaxTokens * kMaxK;
constexpr int kWaves = 8;          // of the products' workgroups

struct MoeParams {
  const uint16_t* x;
  int64_t ldx;
  const uint16_t* router;          // NULL: ids and weights are given
  const float* bias;               // [E] or NULL
  const uint8_t* mask;             // [T] or NULL
  const uint8_t* w_in;
  const float* s_in;
  const uint8_t* w_out;
  const float* s_out;
  const void* res;
  int64_t ldr;
  int res_f32;
  void* y;
  int64_t ldy;
  int32_t* ids;
  float* weights;
  int T, d, E, k, F;
  int score, renormalize, act;
  float scale;
  int kb_d, kb_f;                  // scale blocks of a row of Win, of Wout
  int n_lists;                     // min(E, T k): experts that may be chosen
  int up_wk, down_wk;              // waves that share a tile's K
  // workspace
  double* logits;                  // [T][E]
  int* arrived;
  int* lists;                      // number of chosen experts, then (expert, first position, pairs) of each
  int* pairs;                      // [T k] pairs t k + j by expert
  uint16_t* hi;                    // [T k][F] by position in `pairs`
  uint16_t* lo;
  float* part;                     // [T k][d] by pair
};

__device__ __forceinline__ bool live(const MoeParams& p, int t) { return !p.mask || p.mask[t]; }

// ------------------------------------------------------------------ router
__device__ __forceinline__ double shfl_xor_f64(double v, int m) {
  return __hiloint2double(__shfl_xor(__double2hiint(v), m), __shfl_xor(__double2loint(v), m));
}

// The router's logits in 64 bits, so that which of two experts is chosen does not
// hang on the order of the sum: a wave takes one expert and NT tokens, 8 columns
// a lane at a time, each router value converted once for all of them.
template <int NT>
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeParams p) {
  const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + (threadIdx.x >> 6), t0 = blockIdx.y * NT;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.arrived = 0;  // (of the kernel behind this one)
  if (e >= p.E) return;
  const uint16_t* const r = p.router + (int64_t)e * p.d;
  double acc[NT] = {};
#pragma unroll 2
  for (int c = 8 * lane; c < p.d; c += 512) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(r + c);
    u32x4 v[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t] = *reinterpret_cast<const u32x4*>(p.x + min(t0 + t, p.T - 1) * p.ldx + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double a = bf16_lo(w[i]), b = bf16_hi(w[i]);
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = fma(b, (double)bf16_hi(v[t][i]), fma(a, (double)bf16_lo(v[t][i]), acc[t]));
    }
  }
  // halves of the tokens to halves of the lanes, until a lane has one token (NT = 8: by its upper three bits)
  int m = 32;
#pragma unroll
  for (int n = NT; n > 1; n /= 2, m /= 2)
#pragma unroll
    for (int t = 0; t < NT / 2; ++t)
      if (t < n / 2) {
        const double give = lane & m ? acc[t] : acc[t + n / 2], keep = lane & m ? acc[t + n / 2] : acc[t];
        acc[t] = keep + shfl_xor_f64(give, m);
      }
  for (; m; m /= 2) acc[0] += shfl_xor_f64(acc[0], m);
  const int t = t0 + (NT == 1 ? 0 : lane / (64 / NT));
  if (lane % (64 / NT) == 0 && t < p.T) p.logits[(int64_t)t * p.E + e] = acc[0];
}

// Choice of a token's experts by one wave: lane l has the experts l, l + 64, ..
__device__ __forceinline__ void choose(const MoeParams& p, int t, int lane) {
  constexpr int kEach = kMaxExperts / 64;
  if (!live(p, t)) {
    if (lane < p.k) {
      p.ids[t * p.k + lane] = -1;
      p.weights[t * p.k + lane] = 0.0f;
    }
    return;
  }
  double s[kEach], by[kEach];  // the score, what the choice goes by (NaN counts as the lowest)
  double top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = 64 * i + lane;
    s[i] = e < p.E ? p.logits[(int64_t)t * p.E + e] : -INFINITY;
    by[i] = s[i];
    if (s[i] > top) top = s[i];
  }
  if (p.score == ACRL_MOE_SOFTMAX) {
    for (int m = 32; m; m /= 2) {
      const double o = shfl_xor_f64(top, m);
      if (o > top) top = o;
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (64 * i + lane < p.E) {
        s[i] = exp(s[i] - top);
        sum += s[i];
      }
    for (int m = 32; m; m /= 2) sum += shfl_xor_f64(sum, m);
#pragma unroll
    for (int i = 0; i < kEach; ++i) s[i] /= sum;
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (64 * i + lane < p.E) s[i] = 1.0 / (1.0 + exp(-s[i]));
  }
  uint32_t open = 0;  // the lane's experts that are not chosen yet
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = 64 * i + lane;
    if (e < p.E) open |= 1u << i;
    if (p.bias && e < p.E) by[i] = s[i] + (double)p.bias[e];
    if (by[i] != by[i]) by[i] = -INFINITY;
  }
  double mine = 0.0, total = 0.0;  // lane j: the score of the j-th choice
  int mine_id = 0;
  for (int j = 0; j < p.k; ++j) {
    double best = -INFINITY, best_s = 0.0;
    int id = kMaxExperts;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if ((open >> i & 1) && (id == kMaxExperts || by[i] > best)) {
        best = by[i];
        best_s = s[i];
        id = 64 * i + lane;
      }
    for (int m = 32; m; m /= 2) {
      const double o = shfl_xor_f64(best, m), os = shfl_xor_f64(best_s, m);
      const int oid = __shfl_xor(id, m);
      if (oid < kMaxExperts && (id == kMaxExperts || o > best || (o == best && oid < id))) {
        best = o;
        best_s = os;
        id = oid;
      }
    }
    if (id % 64 == lane) open &= ~(1u << (id / 64));
    if (lane == j) {
      mine = best_s;
      mine_id = id;
    }
    total += best_s;
  }
  if (lane < p.k) {
    if (p.renormalize) mine = total == 0.0 ? 0.0 : mine / total;
    p.ids[t * p.k + lane] = mine_id;
    p.weights[t * p.k + lane] = (float)(mine * (double)p.scale);
  }
}

// The pairs (token, choice) by expert, in their own order within one: by 256
// threads.  Pairs whose expert is out of range, and those of masked tokens, are
// in no list.
struct ListScratch {
  uint8_t count[kMaxPairs / 64][kMaxExperts];  // of a wave's 64 pairs, by expert
  int first[kMaxExperts];
};
__device__ __forceinline__ void make_lists(const MoeParams& p, ListScratch& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, P = p.T * p.k, chunks = (P + 63) / 64;
  for (int i = threadIdx.x; i < chunks * kMaxExperts / 4; i += 256) reinterpret_cast<uint32_t*>(s.count)[i] = 0;
  __syncthreads();
  auto expert = [&](int pair) {
    if (pair >= P || !live(p, pair / p.k)) return -1;
    const int e = __hip_atomic_load(p.ids + pair, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return e >= 0 && e < p.E ? e : -1;
  };
  auto same = [&](int e) {  // the lanes with the same expert
    uint64_t m = __ballot(e >= 0);
#pragma unroll
    for (int b = 0; b < 9; ++b) {
      const uint64_t set = __ballot(e >> b & 1);
      m &= e >> b & 1 ? set : ~set;
    }
    return m;
  };
  const uint64_t before = (1ull << lane) - 1;
  for (int c = wave; c < chunks; c += 4) {
    const int e = expert(64 * c + lane);
    const uint64_t m = same(e);
    if (e >= 0 && !(m & before)) s.count[c][e] = (uint8_t)__popcll(m);
  }
  __syncthreads();
  if (wave == 0) {
    int at = 0, n = 0;
    for (int e0 = 0; e0 < p.E; e0 += 64) {
      const int e = e0 + lane;
      int total = 0;
      if (e < p.E)
        for (int c = 0; c < chunks; ++c) total += s.count[c][e];
      int sum = total;
      for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(sum, o);
        if (lane >= o) sum += v;
      }
      const uint64_t any = __ballot(total > 0);
      const int first = at + sum - total;
      if (e < p.E) s.first[e] = first;
      if (total) {
        int* l = p.lists + 1 + 3 * (n + __popcll(any & before));
        l[0] = e;
        l[1] = first;
        l[2] = total;
      }
      at += __shfl(sum, 63);
      n += __popcll(any);
    }
    if (lane == 0) p.lists[0] = n;
  }
  __syncthreads();
  for (int c = wave; c < chunks; c += 4) {
    const int e = expert(64 * c + lane);
    const uint64_t m = same(e);
    if (e < 0) continue;
    int at = s.first[e] + __popcll(m & before);
    for (int b = 0; b < c; ++b) at += s.count[b][e];
    p.pairs[at] = 64 * c + lane;
  }
}

// Four tokens' choices a workgroup; the one that ends last makes the lists.
__global__ __launch_bounds__(256) void moe_choose_kernel(MoeParams p) {
  __shared__ ListScratch scratch;
  __shared__ int last;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t < p.T) choose(p, t, threadIdx.x & 63);
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.arrived, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  make_lists(p, scratch);
}

// The lists of given choices.
__global__ __launch_bounds__(256) void moe_lists_kernel(MoeParams p) {
  __shared__ ListScratch scratch;
  make_lists(p, scratch);
}

// ------------------------------------------------------------------ products
// Sixteen E4M3 codes as two operands of eight bf16 values (exact).
__device__ __forceinline__ void widen(const i32x4& c, bf16x8 (&o)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[2 * h + i], 1.0f, false);
      const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[2 * h + i], 1.0f, true);
      o[h][4 * i] = a[0];
      o[h][4 * i + 1] = a[1];
      o[h][4 * i + 2] = b[0];
      o[h][4 * i + 3] = b[1];
    }
}
__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A lane's part of a row's scale block: pieces q and q + 4 of 16 columns (any order of k will do that both operands
// have).  What lies past the row's end is read as its first columns and then cleared.
struct Place {
  int at[2];
  bool no[2];
};
__device__ __forceinline__ Place place(int kb, int K, int q) {
  Place r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = kb * kBlock + 16 * (q + 4 * h);
    r.no[h] = k >= K;
    r.at[h] = r.no[h] ? 0 : k;
  }
  return r;
}
// The codes of a block of a row of weights / the bf16 values of a column as four operands.
__device__ __forceinline__ void load_codes(const uint8_t* row, const Place& l, i32x4 (&c)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) c[h] = *reinterpret_cast<const i32x4*>(row + l.at[h]);
}
__device__ __forceinline__ void codes(const i32x4 (&c)[2], const Place& l, bf16x8 (&o)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const i32x4 zero = {0, 0, 0, 0};
    widen(l.no[h] ? zero : c[h], reinterpret_cast<bf16x8(&)[2]>(o[2 * h]));
  }
}
__device__ __forceinline__ void load_column(const uint16_t* col, const Place& l, i32x4 (&c)[4]) {
#pragma unroll
  for (int h = 0; h < 4; ++h) c[h] = *reinterpret_cast<const i32x4*>(col + l.at[h / 2] + 8 * (h % 2));
}
__device__ __forceinline__ bf16x8 column(const i32x4 (&c)[4], const Place& l, int h) {
  const i32x4 zero = {0, 0, 0, 0};
  return __builtin_bit_cast(bf16x8, l.no[h / 2] ? zero : c[h]);
}

__device__ __forceinline__ void add(f32x4& acc, const f32x4& t, float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = fmaf(t[e], s, acc[e]);
}

// The gated products of an expert's tokens: a tile of 16 gate rows and the 16 up
// rows that meet them, times CB blocks of 16 tokens, by up_wk waves that take
// every up_wk-th scale block of K, U at a time; their sums meet in LDS in their
// order.  h = act(gate) * up goes out as two bf16, within 2^-16 of h.
template <int CB, int U>
__global__ __launch_bounds__(64 * kWaves, 2) void moe_up_kernel(MoeParams p) {
  __shared__ f32x4 red[kWaves][2][CB][64];
  if ((int)blockIdx.y >= p.lists[0]) return;
  const int* l = p.lists + 1 + 3 * blockIdx.y;
  const int e = l[0], first = l[1], n = l[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int wk = p.up_wk, tiles = kWaves / wk, kw = wave % wk;
  const int f0 = (blockIdx.x * tiles + wave / wk) * 16;
  const uint8_t *gate = p.w_in, *up = p.w_in;
  const float *s_gate = p.s_in, *s_up = p.s_in;
  if (f0 < p.F) {
    const int row = f0 + (lane & 15), blocks = (2 * p.F + kBlock - 1) / kBlock;
    gate += ((int64_t)e * 2 * p.F + row) * p.d;
    up = gate + (int64_t)p.F * p.d;
    s_gate += ((int64_t)e * blocks + f0 / kBlock) * p.kb_d;
    s_up += ((int64_t)e * blocks + (p.F + f0) / kBlock) * p.kb_d;
  }
  for (int c0 = 0; c0 < n; c0 += 16 * CB) {
    const uint16_t* col[CB];
#pragma unroll
    for (int j = 0; j < CB; ++j) col[j] = p.x + p.pairs[first + min(c0 + 16 * j + (lane & 15), n - 1)] / p.k * p.ldx;
    f32x4 g[CB] = {}, u[CB] = {};
    if (f0 < p.F)
      for (int k0 = kw; k0 < p.kb_d; k0 += wk * U) {
        i32x4 a[U][2][2];
        Place at[U];
        float s[U][2];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int kb = min(k0 + i * wk, p.kb_d - 1);
          at[i] = place(kb, p.d, q);
          load_codes(gate, at[i], a[i][0]);
          load_codes(up, at[i], a[i][1]);
          s[i][0] = s_gate[kb];
          s[i][1] = s_up[kb];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (k0 + i * wk >= p.kb_d) break;
          bf16x8 wg[4], wu[4];
          codes(a[i][0], at[i], wg);
          codes(a[i][1], at[i], wu);
#pragma unroll
          for (int j = 0; j < CB; ++j) {
            if (j && c0 + 16 * j >= n) break;
            i32x4 b[4];
            load_column(col[j], at[i], b);
            f32x4 tg = {}, tu = {};
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const bf16x8 v = column(b, at[i], h);
              tg = mfma(wg[h], v, tg);
              tu = mfma(wu[h], v, tu);
            }
            add(g[j], tg, s[i][0]);
            add(u[j], tu, s[i][1]);
          }
        }
      }
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      red[wave][0][j][lane] = g[j];
      red[wave][1][j][lane] = u[j];
    }
    __syncthreads();
    for (int t = wave; t < tiles * CB; t += kWaves) {
      const int j = t % CB, tile = t / CB, c = c0 + 16 * j + (lane & 15), f = (blockIdx.x * tiles + tile) * 16 + 4 * q;
      f32x4 vg = red[tile * wk][0][j][lane], vu = red[tile * wk][1][j][lane];
      for (int w = 1; w < wk; ++w) {
        vg += red[tile * wk + w][0][j][lane];
        vu += red[tile * wk + w][1][j][lane];
      }
      if (c >= n || f >= p.F) continue;
      float h[4];
      for_activation(p.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = activate<decltype(act)::value, true>(vg[i]) * vu[i];
      });
      bf16x2 hi[2], lo[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __bf16 r = (__bf16)h[i];
        hi[i / 2][i % 2] = r;
        lo[i / 2][i % 2] = fabsf((float)r) < INFINITY ? (__bf16)(h[i] - (float)r) : (__bf16)0.0f;
      }
      const int64_t to = (int64_t)(first + c) * p.F + f;
      *reinterpret_cast<u32x2*>(p.hi + to) = __builtin_bit_cast(u32x2, hi);
      *reinterpret_cast<u32x2*>(p.lo + to) = __builtin_bit_cast(u32x2, lo);
    }
    __syncthreads();
  }
}

// Wout h of an expert's tokens: tiles of 16 rows, split as above, to one fp32 row a pair.
template <int CB, int U>
__global__ __launch_bounds__(64 * kWaves, 2) void moe_down_kernel(MoeParams p) {
  __shared__ f32x4 red[kWaves][CB][64];
  if ((int)blockIdx.y >= p.lists[0]) return;
  const int* l = p.lists + 1 + 3 * blockIdx.y;
  const int e = l[0], first = l[1], n = l[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int wk = p.down_wk, tiles = kWaves / wk, kw = wave % wk;
  const int r0 = (blockIdx.x * tiles + wave / wk) * 16;
  const uint8_t* row = p.w_out;
  const float* s_row = p.s_out;
  if (r0 < p.d) {
    row += ((int64_t)e * p.d + r0 + (lane & 15)) * p.F;
    s_row += ((int64_t)e * ((p.d + kBlock - 1) / kBlock) + r0 / kBlock) * p.kb_f;
  }
  for (int c0 = 0; c0 < n; c0 += 16 * CB) {
    int64_t col[CB];
#pragma unroll
    for (int j = 0; j < CB; ++j) col[j] = (int64_t)(first + min(c0 + 16 * j + (lane & 15), n - 1)) * p.F;
    f32x4 acc[CB] = {};
    if (r0 < p.d)
      for (int k0 = kw; k0 < p.kb_f; k0 += wk * U) {
        i32x4 a[U][2];
        Place at[U];
        float s[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int kb = min(k0 + i * wk, p.kb_f - 1);
          at[i] = place(kb, p.F, q);
          load_codes(row, at[i], a[i]);
          s[i] = s_row[kb];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (k0 + i * wk >= p.kb_f) break;
          bf16x8 w[4];
          codes(a[i], at[i], w);
#pragma unroll
          for (int j = 0; j < CB; ++j) {
            if (j && c0 + 16 * j >= n) break;
            i32x4 bh[4], bl[4];
            load_column(p.hi + col[j], at[i], bh);
            load_column(p.lo + col[j], at[i], bl);
            f32x4 t = {};
#pragma unroll
            for (int h = 0; h < 4; ++h) t = mfma(w[h], column(bl, at[i], h), t);
#pragma unroll
            for (int h = 0; h < 4; ++h) t = mfma(w[h], column(bh, at[i], h), t);
            add(acc[j], t, s[i]);
          }
        }
      }
#pragma unroll
    for (int j = 0; j < CB; ++j) red[wave][j][lane] = acc[j];
    __syncthreads();
    for (int t = wave; t < tiles * CB; t += kWaves) {
      const int j = t % CB, tile = t / CB, c = c0 + 16 * j + (lane & 15), r = (blockIdx.x * tiles + tile) * 16 + 4 * q;
      f32x4 v = red[tile * wk][j][lane];
      for (int w = 1; w < wk; ++w) v += red[tile * wk + w][j][lane];
      if (c < n && r < p.d) *reinterpret_cast<f32x4*>(p.part + (int64_t)p.pairs[first + c] * p.d + r) = v;
    }
    __syncthreads();
  }
}

// y of a token: its pairs' rows by their weights, in the order of its choices, and the residual.
template <typename OUT>
__global__ __launch_bounds__(256) void moe_sum_kernel(MoeParams p) {
  const int t = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= p.d) return;
  f32x4 v = {};
  if (live(p, t))
    for (int j = 0; j < p.k; ++j) {
      const int pair = t * p.k + j, e = p.ids[pair];
      if (e < 0 || e >= p.E) continue;
      add(v, *reinterpret_cast<const f32x4*>(p.part + (int64_t)pair * p.d + c), p.weights[pair]);
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (p.res) {
      const int64_t at = t * p.ldr + c + i;
      v[i] += p.res_f32 ? static_cast<const float*>(p.res)[at] : bf16_lo(static_cast<const uint16_t*>(p.res)[at]);
    }
    static_cast<OUT*>(p.y)[t * p.ldy + c + i] = (OUT)v[i];
  }
}

// ------------------------------------------------------------------ host
size_t lay_out(MoeParams& p, uint8_t* base) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* r = base + at;
    at += (bytes + 255) / 256 * 256;
    return r;
  };
  const size_t P = (size_t)p.T * p.k;
  p.logits = reinterpret_cast<double*>(take((size_t)p.T * p.E * 8));
  p.arrived = reinterpret_cast<int*>(take(4));
  p.lists = reinterpret_cast<int*>(take((1 + 3 * (size_t)p.E) * 4));
  p.pairs = reinterpret_cast<int*>(take(P * 4));
  p.hi = reinterpret_cast<uint16_t*>(take(P * p.F * 2));
  p.lo = reinterpret_cast<uint16_t*>(take(P * p.F * 2));
  p.part = reinterpret_cast<float*>(take(P * p.d * 4));
  return at;
}

// Waves that share a tile's K: as many as leave each a round of loads.
int share(int kb, int each) {
  int wk = 1;
  while (wk < kWaves && wk * each < kb) wk *= 2;
  return wk;
}

template <int CB, int U>
hipError_t launch_products(const MoeParams& p, hipStream_t s) {
  const int up = (p.F / 16 + kWaves / p.up_wk - 1) / (kWaves / p.up_wk);
  hipLaunchKernelGGL((moe_up_kernel<CB, U>), dim3(up, p.n_lists), dim3(64 * kWaves), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int down = (p.d / 16 + kWaves / p.down_wk - 1) / (kWaves / p.down_wk);
  hipLaunchKernelGGL((moe_down_kernel<CB, U>), dim3(down, p.n_lists), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_moe(MoeParams p, int y_type, hipStream_t s) {
  p.up_wk = share(p.kb_d, 2);
  p.down_wk = share(p.kb_f, 2);
  hipError_t e;
  if (p.router) {
    const dim3 grid((p.E + 3) / 4, p.T == 1 ? 1 : (p.T + 7) / 8);
    if (p.T == 1) hipLaunchKernelGGL((moe_logits_kernel<1>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((moe_logits_kernel<8>), grid, dim3(256), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(moe_choose_kernel, dim3((p.T + 3) / 4), dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL(moe_lists_kernel, dim3(1), dim3(256), 0, s, p);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  e = p.T <= 16 ? launch_products<1, 2>(p, s) : p.T <= 32 ? launch_products<2, 2>(p, s) : launch_products<4, 2>(p, s);
  if (e != hipSuccess) return e;
  const dim3 grid((p.d / 4 + 255) / 256, p.T);
  if (y_type == ACRL_OUT_BF16) hipLaunchKernelGGL(moe_sum_kernel<__bf16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(moe_sum_kernel<float>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

acrl_status validate_sizes(int64_t T, int64_t d, int64_t E, int64_t k, int64_t F) {
  ACRL_REQUIRE(T >= 0 && T <= kMaxTokens, "T = %lld must lie in [0, %d]", (long long)T, kMaxTokens);
  ACRL_REQUIRE(d > 0 && d % 32 == 0 && d <= 65536, "d = %lld must be a positive multiple of 32, at most 65536", (long long)d);
  ACRL_REQUIRE(F > 0 && F % 32 == 0 && F <= 65536, "F = %lld must be a positive multiple of 32, at most 65536", (long long)F);
  ACRL_REQUIRE(E > 0 && E <= kMaxExperts, "E = %lld must lie in [1, %d]", (long long)E, kMaxExperts);
  ACRL_REQUIRE(k > 0 && k <= kMaxK && k <= E, "top_k = %lld must lie in [1, min(E, %d)]", (long long)k, kMaxK);
  return ACRL_OK;
}

}  // namespace
}  // namespace acrl

extern "C" {

acrl_status acrl_moe_workspace_size(int64_t T, int64_t d, int64_t E, int64_t top_k, int64_t F, size_t* bytes) {
  ACRL_REQUIRE(bytes, "bytes is NULL");
  acrl_status st = acrl::validate_sizes(T, d, E, top_k, F);
  if (st != ACRL_OK) return st;
  acrl::MoeParams p{};
  p.T = (int)T;
  p.d = (int)d;
  p.E = (int)E;
  p.k = (int)top_k;
  p.F = (int)F;
  *bytes = T ? acrl::lay_out(p, nullptr) : 0;
  return ACRL_OK;
}

acrl_status acrl_moe_fp8(const acrl_moe_desc* m, void* stream) {
  using acrl::aligned16;
  ACRL_REQUIRE(m, "desc is NULL");
  acrl_status st = acrl::validate_sizes(m->T, m->d, m->E, m->top_k, m->F);
  if (st != ACRL_OK) return st;
  const int64_t most = (int64_t)1 << 34;
  ACRL_REQUIRE(m->score == ACRL_MOE_SOFTMAX || m->score == ACRL_MOE_SIGMOID, "score %d unknown", m->score);
  ACRL_REQUIRE(m->activation >= ACRL_ACT_NONE && m->activation <= ACRL_ACT_GELU_TANH, "activation %d unknown", m->activation);
  ACRL_REQUIRE(m->y_type == ACRL_OUT_BF16 || m->y_type == ACRL_OUT_F32, "y_type %d unknown", m->y_type);
  ACRL_REQUIRE(!m->router || (m->scale > -1e30f && m->scale < 1e30f), "scale must be finite, below 1e30 in size");
  ACRL_REQUIRE(m->ldx >= m->d && m->ldx < most && m->ldx % 8 == 0, "ldx = %lld must be a multiple of 8 in [d, 2^34)",
               (long long)m->ldx);
  ACRL_REQUIRE(m->ldy >= m->d && m->ldy < most, "ldy = %lld must lie in [d, 2^34)", (long long)m->ldy);
  ACRL_REQUIRE(m->w_in && m->s_in && m->w_out && m->s_out, "w_in, s_in, w_out and s_out are required");
  ACRL_REQUIRE(aligned16(m->w_in) && aligned16(m->w_out), "w_in and w_out must be 16-byte aligned");
  ACRL_REQUIRE((((uintptr_t)m->s_in | (uintptr_t)m->s_out | (uintptr_t)m->select_bias) & 3u) == 0,
               "s_in, s_out or select_bias is misaligned");
  ACRL_REQUIRE(aligned16(m->router), "router must be 16-byte aligned");
  if (m->residual) {
    ACRL_REQUIRE(m->residual_type == ACRL_OUT_BF16 || m->residual_type == ACRL_OUT_F32, "residual_type %d unknown",
                 m->residual_type);
    ACRL_REQUIRE(m->ldr >= m->d && m->ldr < most, "ldr = %lld must lie in [d, 2^34)", (long long)m->ldr);
    ACRL_REQUIRE(((uintptr_t)m->residual & 3u) == 0, "residual is misaligned");
    ACRL_REQUIRE(!acrl::overlaps(m->residual, m->ldr, m->residual_type, m->y, m->ldy, m->y_type, m->T, m->d),
                 "the residual overlaps y without being y itself");
  }
  if (m->T > 0) {
    ACRL_REQUIRE(m->x && m->y && m->ids && m->weights, "x, y, ids and weights are required");
    ACRL_REQUIRE(aligned16(m->x), "x must be 16-byte aligned");
    ACRL_REQUIRE((((uintptr_t)m->y | (uintptr_t)m->ids | (uintptr_t)m->weights) & 3u) == 0, "y, ids or weights is misaligned");
  }
  acrl::MoeParams p{};
  p.x = static_cast<const uint16_t*>(m->x);
  p.ldx = m->ldx;
  p.router = static_cast<const uint16_t*>(m->router);
  p.bias = m->select_bias;
  p.mask = static_cast<const uint8_t*>(m->mask);
  p.w_in = static_cast<const uint8_t*>(m->w_in);
  p.s_in = m->s_in;
  p.w_out = static_cast<const uint8_t*>(m->w_out);
  p.s_out = m->s_out;
  p.res = m->residual;
  p.ldr = m->ldr;
  p.res_f32 = m->residual_type == ACRL_OUT_F32;
  p.y = m->y;
  p.ldy = m->ldy;
  p.ids = m->ids;
  p.weights = m->weights;
  p.T = (int)m->T;
  p.d = (int)m->d;
  p.E = (int)m->E;
  p.k = (int)m->top_k;
  p.F = (int)m->F;
  p.score = m->score;
  p.renormalize = m->renormalize != 0;
  p.act = m->activation;
  p.scale = m->scale;
  p.kb_d = (p.d + acrl::kBlock - 1) / acrl::kBlock;
  p.kb_f = (p.F + acrl::kBlock - 1) / acrl::kBlock;
  p.n_lists = p.T * p.k < p.E ? p.T * p.k : p.E;
  const size_t need = p.T ? acrl::lay_out(p, static_cast<uint8_t*>(m->workspace)) : 0;
  if (need && (!m->workspace || m->workspace_bytes < need)) {
    acrl::set_error("acrl_moe_fp8 needs %zu workspace bytes, got %zu", need, m->workspace_bytes);
    return ACRL_ERR_WORKSPACE;
  }
  ACRL_REQUIRE(aligned16(m->workspace), "workspace must be 16-byte aligned");
  st = acrl::check_device();
  if (st != ACRL_OK || p.T == 0) return st;
  return acrl::hip_status(acrl::launch_moe(p, m->y_type, (hipStream_t)stream), "acrl_moe_fp8 launch");
}

}  // extern "C"
