// moe.hip -- a mixture-of-experts layer for a few tokens: router, choice of the
// experts, their gated products and the weighted sum.
//
//   l = R x (64 bits), s = softmax(l) or sigmoid(l), the top_k largest s + bias
//   y = residual + sum_j w_j Wout[e_j] (act(Wgate[e_j] x) * (Wup[e_j] x))
//
// The experts' FP8 weights are the bytes that count.  They go straight into
// registers, and those of experts that no token chose are not read.  One pass over an
// expert's weights serves the tokens that its blocks of 16 columns hold, 16, 32 or 64
// (column_blocks); the next ones take another pass.  The kernels for few tokens read
// them for every pair, and workgroups of pairs that turn out not to be their expert's
// first have read one block.  Activations stay
// bf16 (x) and two or three bf16 parts (what lies between the two products): with a few
// columns in each product the matrix cores are idle, so nothing is gained by
// quantizing them.  E4M3 codes become bf16 exactly, products of 128 columns are
// summed by bf16 matrix instructions from zero and enter the fp32 sums with the
// block's scale by one FMA each.
#include <algorithm>

#include "activation.h"
#include "entry.h"
#include "lanes.h"

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
constexpr int kWaves = 4;          // of the products' workgroups (7 tokens, 60 experts: 37 us, 46 with eight)
constexpr int kFewWaves = 8;       // of those for few tokens, a wave at least for each
constexpr int kFewPairs = 16;      // up to so many, the second products and their sum are one kernel, a wave each

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
  int by_pair;                     // there are fewer pairs than experts
  int up_wk, down_wk;              // waves that share a tile's K
  int splits;                      // workgroups that share it in the second products
  // workspace
  double* logits;                  // [T][E]
  uint16_t* h[3];                  // [T k][F] by pair t k + j: h in two bf16 parts, or three
  int parts;
  float* part;                     // [splits][T k][d]
};

__device__ __forceinline__ bool live(const MoeParams& p, int t) { return !p.mask || p.mask[t]; }
// Whether the ids of token t count: those that the router made are -1 where the mask takes it out.
__device__ __forceinline__ bool has_pairs(const MoeParams& p, int t) { return p.router || live(p, t); }

// ------------------------------------------------------------------ router
// The router's logits in 64 bits, so that which of two experts is chosen does not
// hang on the order of the sum: a wave takes one expert and NT tokens, 8 columns
// a lane at a time, each router value converted once for all of them.
template <int NT>
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeParams p) {
  const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + (threadIdx.x >> 6), t0 = blockIdx.y * NT;
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
  // halves of the tokens to halves of the lanes, until a lane has one token (by its upper bits)
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

// Choice of a token's experts by one wave, lane j getting the j-th: lane l looks at the experts l, l + 64, .. (EACH).
// Without WEIGHTS, the ids alone, of the first n.  (Experts that no lane has are passed by: 2 tokens, 8 of 256, 24.3 us, 28.3
// without; with two a lane that would cost 0.5 us.)
struct Choice {
  int id;
  float weight;
};
template <int EACH, bool WEIGHTS>
__device__ __forceinline__ Choice choose(const MoeParams& p, int t, int lane, int n) {
  double s[EACH];     // the score
  float bias[EACH];
  uint64_t by[EACH];  // what the choice goes by, in order (NaN counts as the lowest; 0: chosen)
  double top = -INFINITY;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {  // (all that is read, before any of it is looked at)
    if (EACH > 2 && 64 * i >= p.E) break;
    const int e = min(64 * i + lane, p.E - 1);
    s[i] = p.logits[(int64_t)t * p.E + e];
    bias[i] = p.bias ? p.bias[e] : 0.0f;
  }
  if (!live(p, t)) return {-1, 0.0f};
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (EACH > 2 && 64 * i >= p.E) break;
    if (64 * i + lane >= p.E) s[i] = -INFINITY;
    by[i] = score_key(s[i] == s[i] ? s[i] : -INFINITY);
    if (s[i] > top) top = s[i];
  }
  if (!WEIGHTS && !p.bias) {
  } else if (p.score == ACRL_MOE_SOFTMAX) {
    top = score_of(largest(score_key(top)));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (EACH > 2 && 64 * i >= p.E) break;
      if (64 * i + lane < p.E) {
        s[i] = exp(s[i] - top);
        sum += s[i];
      }
    }
    for (int m = 32; m; m /= 2) sum += shfl_xor_f64(sum, m);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (EACH > 2 && 64 * i >= p.E) break;
      s[i] /= sum;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (EACH > 2 && 64 * i >= p.E) break;
      if (64 * i + lane < p.E) s[i] = 1.0 / (1.0 + exp(-s[i]));
    }
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (EACH > 2 && 64 * i >= p.E) break;
    const int e = 64 * i + lane;
    if (p.bias && e < p.E) {
      const double v = s[i] + (double)bias[i];
      by[i] = score_key(v == v ? v : -INFINITY);
    }
    if (e >= p.E) by[i] = 0;
  }
  double mine = 0.0, total = 0.0;  // lane j: the score of the j-th choice
  int mine_id = 0;
  for (int j = 0; j < n; ++j) {
    uint64_t best = by[0];
    double best_s = s[0];
    int id = lane;
#pragma unroll
    for (int i = 1; i < EACH; ++i) {
      if (EACH > 2 && 64 * i >= p.E) break;
      if (by[i] > best) {
        best = by[i];
        best_s = s[i];
        id = 64 * i + lane;
      }
    }
    const uint64_t most = largest(best);
    uint64_t same = __ballot(best == most);
    int who = lowest(same);
    for (same &= same - 1; same; same &= same - 1)  // equal ones: the lowest index
      if (read_lane(id, lowest(same)) < read_lane(id, who)) who = lowest(same);
    id = read_lane(id, who);
    best_s = read_lane(best_s, who);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (EACH > 2 && 64 * i >= p.E) break;
      by[i] = 64 * i + lane == id ? 0 : by[i];
    }
    if (lane == j) {
      mine = best_s;
      mine_id = id;
    }
    total += best_s;
  }
  if (!WEIGHTS) return {mine_id, 0.0f};
  if (p.renormalize) mine = total == 0.0 ? 0.0 : mine / total;
  return {mine_id, (float)(mine * (double)p.scale)};
}
template <int EACH>
__device__ __forceinline__ void write_choice(const MoeParams& p, int t, int lane) {
  const Choice c = choose<EACH, true>(p, t, lane, p.k);
  if (lane < p.k) {
    p.ids[t * p.k + lane] = c.id;
    p.weights[t * p.k + lane] = c.weight;
  }
}
template <int EACH>
__global__ __launch_bounds__(64) void moe_choose_kernel(MoeParams p) {
  write_choice<EACH>(p, blockIdx.x, threadIdx.x);
}

// The pairs (token, choice) of the workgroup's expert, in their order: `pairs`
// holds n of them.  Row y of the grid is expert y, or, where there are fewer pairs
// than experts, the expert of pair y if that is its first pair.  Every workgroup
// looks through all ids (8 KB at most): lists made once for all of them took 10 us
// more behind the choice, for one token and for 64.
struct Tokens {
  uint16_t pairs[kMaxPairs];
  int counts[kWaves];
};
// ids: all tokens' choices
template <bool BY_PAIR>
__device__ __forceinline__ int expert_of(const MoeParams& p, const int* ids) {
  const int y = blockIdx.y;
  if (!BY_PAIR) return y;
  const int e = ids[y];
  return e >= 0 && e < p.E && has_pairs(p, y / p.k) ? e : -1;
}
template <bool BY_PAIR>
__device__ __forceinline__ int find_tokens(const MoeParams& p, const int* ids, int e, Tokens& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, P = p.T * p.k;
  int n = 0, next = (int)threadIdx.x < P ? ids[threadIdx.x] : -1;
  for (int first = 0; first < P; first += 64 * kWaves) {
    const int pair = first + threadIdx.x, id = next;
    next = pair + 64 * kWaves < P ? ids[pair + 64 * kWaves] : -1;
    const bool hit = id == e && has_pairs(p, pair / p.k);
    const uint64_t m = __ballot(hit);
    if (lane == 0) s.counts[wave] = __popcll(m);
    lds_barrier();
    int at = n + __popcll(m & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s.counts[w];
      at += w < wave ? c : 0;
      n += c;
    }
    if (hit) s.pairs[at] = (uint16_t)pair;
    lds_barrier();
  }
  return BY_PAIR && n && s.pairs[0] != blockIdx.y ? 0 : n;
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
__device__ __forceinline__ bf16x8 cleared(const i32x4& c, bool no) {
  const i32x4 zero = {0, 0, 0, 0};
  return __builtin_bit_cast(bf16x8, no ? zero : c);
}
// The codes of a block of a row as four operands.
__device__ __forceinline__ void codes(const i32x4 (&c)[2], const Place& l, bf16x8 (&o)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const i32x4 zero = {0, 0, 0, 0};
    widen(l.no[h] ? zero : c[h], reinterpret_cast<bf16x8(&)[2]>(o[2 * h]));
  }
}

__device__ __forceinline__ void add(f32x4& acc, const f32x4& t, float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = fmaf(t[e], s, acc[e]);
}

// h as bf16 parts, the largest first; an infinity has none behind its first.
__device__ __forceinline__ void store_parts(const MoeParams& p, int64_t to, float (&h)[4]) {
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    if (c == p.parts) break;
    bf16x2 o[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __bf16 r = (__bf16)h[i];
      o[i / 2][i % 2] = r;
      h[i] = fabsf((float)r) < INFINITY ? h[i] - (float)r : 0.0f;
    }
    *reinterpret_cast<u32x2*>(p.h[c] + to) = __builtin_bit_cast(u32x2, o);
  }
}

// Scales of rows: the same for a wave, so they are read by scalar loads, whose addresses and results take no vector
// registers (nine fewer in the products, which brings the second ones from two waves a SIMD to three: 64 tokens, 8 of 128
// experts of 2048 x 1536: 229 us for 238).
using Scales = const __attribute__((address_space(4))) float*;
__device__ __forceinline__ Scales scales_at(const float* base, int64_t at) { return (Scales)(base + at); }

// R tiles of 16 rows of an expert (their codes at `row`, scales at `scale`) times
// CB blocks of 16 columns of PARTS bf16 each (their sum), over the scale blocks
// kw, kw + wk, .. of K.  A block's codes are loaded one block ahead, its columns
// (from the caches) right before the codes that are ahead of them: loads come back
// in their order.  (Codes two blocks ahead, columns behind the products: 202 us for
// 150 at 64 tokens, 8 of 128 experts of 2048 x 768; two blocks of both at a time: 165.)
// Lanes of columns that are not there load nothing.
template <int R, int CB, int PARTS>
struct Stream {
  using Codes = i32x4[R][2];
  const uint8_t* row[R];
  Scales scale[R];
  const uint16_t* col[CB][PARTS];
  bool there[CB];
  int K, kb, kw, wk, q;

  __device__ __forceinline__ void load(Codes& x, int k) const {
    const Place at = place(min(k, kb - 1), K, q);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) x[i][h] = *reinterpret_cast<const i32x4*>(row[i] + at.at[h]);
  }
  __device__ __forceinline__ void step(Codes& now, Codes& ahead, int k, f32x4 (&acc)[R][CB]) const {
    const Place at = place(k, K, q);
    float s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] = scale[i][k];
    constexpr int G = CB == 1 || CB + PARTS == 7 ? 1 : 2;  // blocks of columns at a time, as registers allow
#pragma unroll
    for (int j0 = 0; j0 < CB; j0 += G) {
      i32x4 b[G][PARTS][4] = {};
#pragma unroll
      for (int j = 0; j < G; ++j)
        if (there[j0 + j]) {
#pragma unroll
          for (int c = 0; c < PARTS; ++c)
#pragma unroll
            for (int h = 0; h < 4; ++h)
              b[j][c][h] = *reinterpret_cast<const i32x4*>(col[j0 + j][c] + at.at[h / 2] + 8 * (h % 2));
        }
      if (j0 + G == CB) load(ahead, k + wk);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        bf16x8 w[4];
        codes(now[i], at, w);
#pragma unroll
        for (int j = 0; j < G; ++j) {
          f32x4 t = {};
#pragma unroll
          for (int c = PARTS - 1; c >= 0; --c)  // (the smaller part first)
#pragma unroll
            for (int h = 0; h < 4; ++h) t = mfma(w[h], cleared(b[j][c][h], at.no[h / 2]), t);
          add(acc[i][j0 + j], t, s[i]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // first: the codes of block kw
  __device__ __forceinline__ void run(Codes& first, f32x4 (&acc)[R][CB]) const {
    if (kw >= kb) return;
    Codes other;
    int k = kw;
    for (; k + wk < kb; k += 2 * wk) {
      step(first, other, k, acc);
      step(other, first, k + wk, acc);
    }
    if (k < kb) step(first, other, k, acc);
  }
};

// The gated products of an expert's tokens: a tile of 16 gate rows and the 16 up
// rows that meet them, times CB blocks of 16 tokens, by up_wk waves that share K;
// their sums meet in LDS in their order.  h = act(gate) * up goes out as two bf16,
// within 2^-16 of h (7 % of the time of 16 tokens, d = 4096, F = 14336 over one, which
// would be as far off as y's own rounding), or, where y is fp32, as three, exactly.
template <int CB, int R, bool BY_PAIR>
__global__ __launch_bounds__(64 * kWaves, CB == 1 && R == 2 ? 4 : CB == 1 ? 3 : 2) void moe_up_kernel(MoeParams p) {
  __shared__ f32x4 red[kWaves][R][CB][64];
  __shared__ Tokens tokens;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int e = __builtin_amdgcn_readfirstlane(expert_of<BY_PAIR>(p, p.ids));
  if (e < 0) return;
  const int wk = p.up_wk, tiles = kWaves / wk;
  constexpr int H = R / 2, kRows = 16 * H;  // tiles of gate rows
  const int f0 = min((int)(blockIdx.x * tiles + wave / wk) * kRows, p.F - kRows);  // (tiles past the last repeat it)
  const int blocks = (2 * p.F + kBlock - 1) / kBlock;
  Stream<R, CB, 1> st;
  st.K = p.d;
  st.kb = p.kb_d;
  st.kw = wave % wk;
  st.wk = wk;
  st.q = q;
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int f = f0 + 16 * i;
    st.row[i] = p.w_in + ((int64_t)e * 2 * p.F + f + (lane & 15)) * p.d;
    st.row[H + i] = st.row[i] + (int64_t)p.F * p.d;
    st.scale[i] = scales_at(p.s_in, ((int64_t)e * blocks + f / kBlock) * p.kb_d);
    st.scale[H + i] = scales_at(p.s_in, ((int64_t)e * blocks + (p.F + f) / kBlock) * p.kb_d);
  }
  typename Stream<R, CB, 1>::Codes first;
  if (BY_PAIR) st.load(first, st.kw);  // (while it looks for the tokens: the expert is chosen)
  const int n = find_tokens<BY_PAIR>(p, p.ids, e, tokens);
  for (int c0 = 0; c0 < n;) {
    if (!BY_PAIR) st.load(first, st.kw);
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int c = c0 + 16 * j + (lane & 15);
      st.there[j] = c < n;
      st.col[j][0] = p.x + tokens.pairs[min(c, n - 1)] / p.k * p.ldx;
    }
    f32x4 acc[R][CB] = {};
    st.run(first, acc);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) red[wave][i][j][lane] = acc[i][j];
    lds_barrier();
    for (int t = wave; t < tiles * H * CB; t += kWaves) {
      const int j = t % CB, i = t / CB % H, tile = t / CB / H, c = c0 + 16 * j + (lane & 15);
      const int f = (blockIdx.x * tiles + tile) * kRows + 16 * i + 4 * q;
      f32x4 vg = red[tile * wk][i][j][lane], vu = red[tile * wk][H + i][j][lane];
      for (int w = 1; w < wk; ++w) {
        vg += red[tile * wk + w][i][j][lane];
        vu += red[tile * wk + w][H + i][j][lane];
      }
      if (c >= n || f >= p.F) continue;
      float h[4];
      for_activation(p.act, [&](auto act) {
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = activate<decltype(act)::value, true>(vg[v]) * vu[v];
      });
      store_parts(p, (int64_t)tokens.pairs[c] * p.F + f, h);
    }
    lds_barrier();
    c0 += 16 * CB;
    if (BY_PAIR && c0 < n) st.load(first, st.kw);
  }
}

// Wout h of an expert's tokens: tiles of 16 R rows, K shared as above and by workgroups, to an fp32 row a pair for each.
template <int CB, int R, int PARTS, bool BY_PAIR>
__global__ __launch_bounds__(64 * kWaves, CB + PARTS + R == 5 ? 4 : 2) void moe_down_kernel(MoeParams p) {
  __shared__ f32x4 red[kWaves][R][CB][64];
  __shared__ Tokens tokens;
  const int e = __builtin_amdgcn_readfirstlane(expert_of<BY_PAIR>(p, p.ids));
  if (e < 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int wk = p.down_wk, tiles = kWaves / wk;
  const int r0 = min((int)(blockIdx.x * tiles + wave / wk) * 16 * R, p.d - 16 * R);
  Stream<R, CB, PARTS> st;
  st.K = p.F;
  st.kb = p.kb_f;
  st.kw = blockIdx.z * wk + wave % wk;
  st.wk = wk * p.splits;
  st.q = q;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + 16 * i;
    st.row[i] = p.w_out + ((int64_t)e * p.d + r + (lane & 15)) * p.F;
    st.scale[i] = scales_at(p.s_out, ((int64_t)e * ((p.d + kBlock - 1) / kBlock) + r / kBlock) * p.kb_f);
  }
  float* const part = p.part + (int64_t)blockIdx.z * p.T * p.k * p.d;
  typename Stream<R, CB, PARTS>::Codes first;
  if (BY_PAIR) st.load(first, st.kw);
  const int n = find_tokens<BY_PAIR>(p, p.ids, e, tokens);
  for (int c0 = 0; c0 < n;) {
    if (!BY_PAIR) st.load(first, st.kw);
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      const int c = c0 + 16 * j + (lane & 15);
      st.there[j] = c < n;
      const int64_t at = (int64_t)tokens.pairs[min(c, n - 1)] * p.F;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) st.col[j][i] = p.h[i] + at;
    }
    f32x4 acc[R][CB] = {};
    st.run(first, acc);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) red[wave][i][j][lane] = acc[i][j];
    lds_barrier();
    for (int t = wave; t < tiles * R * CB; t += kWaves) {
      const int j = t % CB, i = t / CB % R, tile = t / CB / R, c = c0 + 16 * j + (lane & 15);
      const int r = (blockIdx.x * tiles + tile) * 16 * R + 16 * i + 4 * q;
      f32x4 v = red[tile * wk][i][j][lane];
      for (int w = 1; w < wk; ++w) v += red[tile * wk + w][i][j][lane];
      if (c < n && r < p.d) *reinterpret_cast<f32x4*>(part + (int64_t)tokens.pairs[c] * p.d + r) = v;
    }
    lds_barrier();
    c0 += 16 * CB;
    if (BY_PAIR && c0 < n) st.load(first, st.kw);
  }
}

__device__ __forceinline__ float residual(const MoeParams& p, int t, int c) {
  const int64_t at = t * p.ldr + c;
  return p.res_f32 ? static_cast<const float*>(p.res)[at] : bf16_lo(static_cast<const uint16_t*>(p.res)[at]);
}

// The same for few tokens that hardly share experts, where what counts is how many
// loads wait for another: every workgroup chooses its pair's expert by itself (2 us
// of 22 for one token, 2048 x 768, 8 of 128 experts; weights are made by a workgroup
// apart), and the codes and columns of two blocks are under way together.  One pair a
// workgroup and 16 gate and up rows, K shared by its waves.
template <int EACH>
__global__ __launch_bounds__(64 * kFewWaves) void moe_up_few_kernel(MoeParams p) {
  __shared__ f32x4 red[kFewWaves][2][4];
  __shared__ int chosen;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int pair = (int)blockIdx.y - 1, f0 = blockIdx.x * 16;
  if (pair < 0) {  // (first, since it takes as long as any)
    if (blockIdx.x == 0 && wave < p.T) write_choice<EACH>(p, wave, lane);
    return;
  }
  if (wave == 0) {
    const int id = choose<EACH, false>(p, pair / p.k, lane, pair % p.k + 1).id;
    if (lane == pair % p.k) chosen = id;
  }
  lds_barrier();
  const int e = __builtin_amdgcn_readfirstlane(chosen), blocks = (2 * p.F + kBlock - 1) / kBlock;
  if (e < 0) return;
  const uint16_t* const x = p.x + pair / p.k * p.ldx;
  const uint8_t* const gate = p.w_in + ((int64_t)e * 2 * p.F + f0 + (lane & 15)) * p.d;
  const uint8_t* const row[2] = {gate, gate + (int64_t)p.F * p.d};
  const Scales scale[2] = {scales_at(p.s_in, ((int64_t)e * blocks + f0 / kBlock) * p.kb_d),
                           scales_at(p.s_in, ((int64_t)e * blocks + (p.F + f0) / kBlock) * p.kb_d)};
  f32x4 acc[2] = {};
  constexpr int U = 2;
  for (int k0 = wave; k0 < p.kb_d; k0 += U * kFewWaves) {
    i32x4 a[U][2][2], b[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const Place at = place(min(k0 + u * kFewWaves, p.kb_d - 1), p.d, q);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) a[u][i][h] = *reinterpret_cast<const i32x4*>(row[i] + at.at[h]);
#pragma unroll
      for (int h = 0; h < 4; ++h) b[u][h] = *reinterpret_cast<const i32x4*>(x + at.at[h / 2] + 8 * (h % 2));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kFewWaves;
      if (k >= p.kb_d) break;
      const Place at = place(k, p.d, q);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        bf16x8 w[4];
        codes(a[u][i], at, w);
        f32x4 t = {};
#pragma unroll
        for (int h = 0; h < 4; ++h) t = mfma(w[h], cleared(b[u][h], at.no[h / 2]), t);
        add(acc[i], t, scale[i][k]);
      }
    }
  }
  if ((lane & 15) == 0) {  // (all columns are the one token)
    red[wave][0][q] = acc[0];
    red[wave][1][q] = acc[1];
  }
  lds_barrier();
  if (threadIdx.x >= 4) return;
  f32x4 vg = red[0][0][threadIdx.x], vu = red[0][1][threadIdx.x];
#pragma unroll
  for (int w = 1; w < kFewWaves; ++w) {
    vg += red[w][0][threadIdx.x];
    vu += red[w][1][threadIdx.x];
  }
  float h[4];
  for_activation(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = activate<decltype(act)::value, true>(vg[i]) * vu[i];
  });
  store_parts(p, (int64_t)pair * p.F + f0 + 4 * threadIdx.x, h);
}

// Wout h and the sum over a token's experts, for few pairs: 16 rows of y a
// workgroup, each wave a pair, or a share of its K where there are fewer pairs than
// waves.  h passes through LDS, 512 columns of a wave at a time, so that no load
// waits for another but by these (columns read where they are used: 9.5 us for one
// token, 2048 x 768, 8 experts).
template <typename OUT>
__global__ __launch_bounds__(64 * kFewPairs) void moe_down_few_kernel(MoeParams p) {
  constexpr int PARTS = std::is_same<OUT, float>::value ? 3 : 2, U = 4;
  __shared__ i32x4 columns[kFewPairs][PARTS][64];
  __shared__ float part[kFewPairs][16];  // by pair and share of K
  __shared__ float weight[kFewPairs];    // of the pairs that count
  __shared__ bool counts[kFewPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const int r0 = blockIdx.x * 16, P = p.T * p.k, wk = p.down_wk, pair = wave / wk;
  const int e = pair < P ? __builtin_amdgcn_readfirstlane(p.ids[pair]) : -1;
  const int t = threadIdx.x / 16, r = threadIdx.x % 16;  // of the sum
  float res = -0.0f;
  if (p.res && t < p.T) res = residual(p, t, r0 + r);
  if ((int)threadIdx.x < P) {
    const int id = p.ids[threadIdx.x];
    counts[threadIdx.x] = id >= 0 && id < p.E && has_pairs(p, threadIdx.x / p.k);
    weight[threadIdx.x] = p.weights[threadIdx.x];
  }
  if (e >= 0 && e < p.E && has_pairs(p, pair / p.k)) {
    const int each = (p.kb_f + wk - 1) / wk, k1 = min(p.kb_f, (wave % wk + 1) * each);
    const uint8_t* const row = p.w_out + ((int64_t)e * p.d + r0 + (lane & 15)) * p.F;
    const Scales scale = scales_at(p.s_out, ((int64_t)e * ((p.d + kBlock - 1) / kBlock) + r0 / kBlock) * p.kb_f);
    f32x4 acc = {};
    for (int k0 = wave % wk * each; k0 < k1; k0 += U) {
      i32x4 a[U][2], h[PARTS];
      const int c = k0 * kBlock + 8 * lane;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        h[i] = i32x4{0, 0, 0, 0};
        if (c < p.F) h[i] = *reinterpret_cast<const i32x4*>(p.h[i] + (int64_t)pair * p.F + c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k0 + u >= k1) break;
        const Place at = place(k0 + u, p.F, q);
#pragma unroll
        for (int i = 0; i < 2; ++i) a[u][i] = *reinterpret_cast<const i32x4*>(row + at.at[i]);
      }
#pragma unroll
      for (int i = 0; i < PARTS; ++i) columns[wave][i][lane] = h[i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k0 + u >= k1) break;
        const Place at = place(k0 + u, p.F, q);
        bf16x8 w[4];
        codes(a[u], at, w);
        f32x4 t = {};
#pragma unroll
        for (int i = PARTS - 1; i >= 0; --i)  // (the smaller part first)
#pragma unroll
          for (int m = 0; m < 4; ++m)
            t = mfma(w[m], cleared(columns[wave][i][16 * u + 2 * (q + 4 * (m / 2)) + m % 2], at.no[m / 2]), t);
        add(acc, t, scale[k0 + u]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if ((lane & 15) == 0) *reinterpret_cast<f32x4*>(&part[wave][4 * q]) = acc;
  }
  __syncthreads();
  if (t >= p.T) return;
  float v = 0.0f;
  for (int j = 0; j < p.k; ++j) {
    const int i = t * p.k + j;
    if (!counts[i]) continue;
    float s = part[i * wk][r];
    for (int w = 1; w < wk; ++w) s += part[i * wk + w][r];
    v = fmaf(s, weight[i], v);
  }
  if (p.res) v += res;
  static_cast<OUT*>(p.y)[t * p.ldy + r0 + r] = (OUT)v;
}

// y of a token: its pairs' rows by their weights, in the order of its choices (no atomics: equal calls give equal bits),
// and the residual.  All rows are under way together (one after another: 6.0 us for 4.6 at 64 tokens, 8 pairs each, d =
// 2048).
template <typename OUT>
__global__ __launch_bounds__(256) void moe_sum_kernel(MoeParams p) {
  const int t = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4, j = threadIdx.x & 63;
  int id = -1;
  float weight = 0.0f;
  if (j < p.k && has_pairs(p, t)) {  // lane j has the j-th pair's
    id = p.ids[t * p.k + j];
    weight = p.weights[t * p.k + j];
  }
  const uint64_t pairs = __ballot(id >= 0 && id < p.E);
  if (c >= p.d) return;
  f32x4 rows[kMaxK], v = {};
  float res[4];
#pragma unroll
  for (int n = 0; n < kMaxK; ++n)
    if (pairs >> n & 1) rows[n] = *reinterpret_cast<const f32x4*>(p.part + (int64_t)(t * p.k + n) * p.d + c);
  for (int z = 1; z < p.splits; ++z)
#pragma unroll
    for (int n = 0; n < kMaxK; ++n)
      if (pairs >> n & 1) rows[n] += *reinterpret_cast<const f32x4*>(p.part + ((int64_t)z * p.T * p.k + t * p.k + n) * p.d + c);
#pragma unroll
  for (int i = 0; i < 4; ++i) res[i] = p.res ? residual(p, t, c + i) : 0.0f;
#pragma unroll
  for (int n = 0; n < kMaxK; ++n)
    if (pairs >> n & 1) add(v, rows[n], __int_as_float(read_lane(__float_as_int(weight), n)));
#pragma unroll
  for (int i = 0; i < 4; ++i) static_cast<OUT*>(p.y)[t * p.ldy + c + i] = (OUT)(p.res ? v[i] + res[i] : v[i]);
}

// ------------------------------------------------------------------ host
// Waves that share a tile's K: until there are four rounds of waves for the CUs (16 each), with two blocks each at
// least; and one, while there is less than a round.
int share(int64_t tiles, int kb) {
  constexpr int64_t kRound = 256 * 16;
  int wk = 1;
  while (wk < kWaves && ((tiles * wk * 2 <= 4 * kRound && wk * 4 <= kb) || (tiles * wk < kRound && wk < kb))) wk *= 2;
  return wk;
}

// Blocks of 16 columns by the tokens an expert has on average; where it has more than they hold, its weights are read
// again (128 tokens, 2 of 8 experts of 4096 x 14336: 871 us with one block, 502 with two, 619 with four, which leave
// registers for two tiles of rows alone; 1 of 4 of 1024 x 4096: 51 with two, 45 with four).  At those 502 us that is most
// of the way to the floor of 284: three of the eight experts have 33 to 43 tokens and theirs come twice, so that the
// products fetch 1.39 and 1.45 times what they fetch for 64 tokens, in 339 us.
int column_blocks(const MoeParams& p) {
  const int P = p.T * p.k;
  return P <= 10 * p.E || p.T <= 16 ? 1 : P <= 40 * p.E || p.T <= 32 ? 2 : 4;
}

// The second products of few pairs and their sum as one kernel, where its waves, 16 a workgroup of 16 rows, have not much
// more of K each than those of the others (2 tokens, 6 of 8 experts of 928 x 8800: 76 us in all, 46 the other way).
int few_share(const MoeParams& p) {
  int wk = 1;
  while (wk * 2 * p.T * p.k <= kFewPairs && wk * 2 <= p.kb_f) wk *= 2;
  return wk;
}
bool few_down(const MoeParams& p) {
  return p.T * p.k <= kFewPairs && (p.kb_f + few_share(p) - 1) / few_share(p) <= p.kb_f / kWaves + 8;
}

// What follows from the sizes.
void plan(MoeParams& p) {
  p.kb_d = (p.d + kBlock - 1) / kBlock;
  p.kb_f = (p.F + kBlock - 1) / kBlock;
  p.by_pair = p.T * p.k < p.E;
  // K of the second products is shared by workgroups until there are two a CU, with four blocks a wave at least (8 tokens, 2
  // of 8 experts of 2048 x 8224: 99 us in all, 131 without; 4 of 4 of 384 x 10432: 36 and 50)
  const int rows = column_blocks(p) <= 2 && !p.by_pair && p.d % 64 == 0 ? 64 : 32, tiles = p.d / rows, y = p.by_pair ? p.T * p.k : p.E;
  const int wk = share((int64_t)tiles * y, p.kb_f), each = kWaves / wk;
  p.splits = std::max(1, std::min(512 / std::max(1, (tiles + each - 1) / each * y), p.kb_f / (4 * wk)));
}

size_t lay_out(MoeParams& p, uint8_t* base) {
  plan(p);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* r = base + at;
    at += (bytes + 255) / 256 * 256;
    return r;
  };
  const size_t P = (size_t)p.T * p.k;
  p.logits = reinterpret_cast<double*>(take((size_t)p.T * p.E * 8));
  for (uint16_t*& h : p.h) h = reinterpret_cast<uint16_t*>(take(P * p.F * 2));
  p.part = reinterpret_cast<float*>(take(p.splits * P * p.d * 4));
  return at;
}

// R tiles of 16 rows a wave: four, which columns are read for once; two where there are few pairs, and with four blocks of
// columns, whose sums take the registers.  (With two, in workgroups of eight waves: 64 tokens, 8 of 128 experts of 2048 x
// 768 149 us for 143, 16 tokens, 2 of 8 of 4096 x 14336 293 for 267.  With two and two blocks of columns: 64 tokens of the
// latter 429 us for 339, 128 tokens, 4 of 32 of 2048 x 1024 86 for 70.)
template <int CB, int R, bool BY_PAIR>
hipError_t launch_up_tiles(MoeParams p, hipStream_t s) {
  const int y = BY_PAIR ? p.T * p.k : p.E, tiles = p.F / (8 * R);
  p.up_wk = share((int64_t)tiles * y, p.kb_d);
  const int each = kWaves / p.up_wk;
  hipLaunchKernelGGL((moe_up_kernel<CB, R, BY_PAIR>), dim3((tiles + each - 1) / each, y), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}
template <int CB, int R, int PARTS, bool BY_PAIR>
hipError_t launch_down_tiles(MoeParams p, hipStream_t s) {
  const int y = BY_PAIR ? p.T * p.k : p.E, tiles = p.d / (16 * R);
  p.down_wk = share((int64_t)tiles * y, p.kb_f);
  const int each = kWaves / p.down_wk;
  hipLaunchKernelGGL((moe_down_kernel<CB, R, PARTS, BY_PAIR>), dim3((tiles + each - 1) / each, y, p.splits), dim3(64 * kWaves), 0, s, p);
  return hipGetLastError();
}

template <int CB>
hipError_t launch_up(const MoeParams& p, hipStream_t s) {
  if constexpr (CB > 1) return launch_up_tiles<CB, CB == 2 ? 4 : 2, false>(p, s);  // (fewer pairs than experts are few an expert)
  else if (p.by_pair) return launch_up_tiles<1, 2, true>(p, s);
  else return launch_up_tiles<1, 4, false>(p, s);
}

template <int CB, int PARTS>
hipError_t launch_down(const MoeParams& p, hipStream_t s) {
  if constexpr (CB == 4) return launch_down_tiles<4, 2, PARTS, false>(p, s);
  else if constexpr (CB == 2) return p.d % 64 == 0 ? launch_down_tiles<2, 4, PARTS, false>(p, s) : launch_down<4, PARTS>(p, s);
  else if (p.by_pair) return launch_down_tiles<1, 2, PARTS, true>(p, s);
  else if (p.d % 64 == 0) return launch_down_tiles<1, 4, PARTS, false>(p, s);
  else return launch_down_tiles<1, 2, PARTS, false>(p, s);
}

template <typename OUT>
hipError_t launch_moe(MoeParams p, hipStream_t s) {
  constexpr int PARTS = std::is_same<OUT, float>::value ? 3 : 2;
  const int P = p.T * p.k;
  p.parts = PARTS;
  const int blocks = column_blocks(p);
  hipError_t e;
  if (p.router) {
    const int nt = p.T <= 16 ? 1 : 2;  // (7 tokens, 60 experts: 46 us with 2, 48 with 8; 64 tokens: 1 us more with 8)
    const dim3 grid((p.E + 3) / 4, (p.T + nt - 1) / nt);
    if (nt == 1) hipLaunchKernelGGL((moe_logits_kernel<1>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((moe_logits_kernel<2>), grid, dim3(256), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  // (3 tokens, 8 of 128 experts of 2048 x 768: 38.2 us, 40.2 the other way; 4 tokens, 2 of them: 19.8 and 23.1; but 8 tokens, 8
  // of them, 70.4 and 67.2; 4 tokens, 2 of 8 experts of 4096 x 14336: 237 and 208, 2 tokens: 132 and 117)
  if (p.router && (p.T == 1 || (p.T <= kFewWaves && 4 * P <= p.E))) {
    const dim3 grid(p.F / 16, P + 1);
    if (p.E <= 128) hipLaunchKernelGGL(moe_up_few_kernel<2>, grid, dim3(64 * kFewWaves), 0, s, p);
    else hipLaunchKernelGGL(moe_up_few_kernel<8>, grid, dim3(64 * kFewWaves), 0, s, p);
    e = hipGetLastError();
  } else {
    if (p.router) {
      if (p.E <= 64) hipLaunchKernelGGL(moe_choose_kernel<1>, dim3(p.T), dim3(64), 0, s, p);
      else if (p.E <= 128) hipLaunchKernelGGL(moe_choose_kernel<2>, dim3(p.T), dim3(64), 0, s, p);
      else hipLaunchKernelGGL(moe_choose_kernel<8>, dim3(p.T), dim3(64), 0, s, p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    e = blocks == 1 ? launch_up<1>(p, s) : blocks == 2 ? launch_up<2>(p, s) : launch_up<4>(p, s);
  }
  if (e != hipSuccess) return e;
  if (few_down(p)) {
    p.down_wk = few_share(p);
    hipLaunchKernelGGL(moe_down_few_kernel<OUT>, dim3(p.d / 16), dim3(64 * kFewPairs), 0, s, p);
    return hipGetLastError();
  }
  e = blocks == 1 ? launch_down<1, PARTS>(p, s) : blocks == 2 ? launch_down<2, PARTS>(p, s) : launch_down<4, PARTS>(p, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(moe_sum_kernel<OUT>, dim3((p.d / 4 + 255) / 256, p.T), dim3(256), 0, s, p);
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
  const size_t need = p.T ? acrl::lay_out(p, static_cast<uint8_t*>(m->workspace)) : 0;
  if (need && (!m->workspace || m->workspace_bytes < need)) {
    acrl::set_error("acrl_moe_fp8 needs %zu workspace bytes, got %zu", need, m->workspace_bytes);
    return ACRL_ERR_WORKSPACE;
  }
  ACRL_REQUIRE(aligned16(m->workspace), "workspace must be 16-byte aligned");
  st = acrl::check_device();
  if (st != ACRL_OK || p.T == 0) return st;
  const hipStream_t s = (hipStream_t)stream;
  return acrl::hip_status(m->y_type == ACRL_OUT_BF16 ? acrl::launch_moe<__bf16>(p, s) : acrl::launch_moe<float>(p, s),
                          "acrl_moe_fp8 launch");
}

}  // extern "C"
