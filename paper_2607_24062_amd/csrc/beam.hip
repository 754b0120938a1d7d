// beam.hip -- beam search: the choice of the next tokens over beams and
// vocabulary, and the states of the chosen beams.
//
// The choice compares scores of different beams, score_j + z - lse_j, so a
// normaliser that is off by an fp32 rounding would now and then choose another
// candidate: exponentials and sums are fp64.  Within a beam the order is that of
// the logits alone.
#include <float.h>

#include <algorithm>
#include <iterator>
#include <type_traits>
#include <utility>

#include "entry.h"
#include "lanes.h"

namespace acrl {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kMaxBeams = 64, kMaxOut = 64;
constexpr int kScanWaves = 8, kEach = 8, kTile = 64 * kEach;  // logits of a lane, of a wave at a time
constexpr int notes_left(int N) { return 32 + 2 * N; }  // notes of a workgroup between tiles, at most
constexpr int kNotes = notes_left(kMaxOut) + kScanWaves * kTile;
static_assert(notes_left(kMaxOut) <= 64 * kScanWaves, "a thread ranks one");
constexpr int kPickWaves = 4, kMaxLists = 64 * kPickWaves, kMaxStaged = 6144;
constexpr int kNone = 0x7FFFFFFF;

struct BeamParams {
  const void* logits;
  int64_t ldl;
  const float* scores;
  const uint8_t* finished;  // or NULL
  int B, K, V, N, eos;
  float inv_t;
  double c, least, reach;   // inv_t log2 e, -1000 / c, 400 / c
  int S;                    // segments of a row, each one workgroup's
  int seg_tiles;            // tiles of a segment
  int32_t* ids;
  int32_t* parents;
  float* out;
  // workspace, by row and segment
  double* norm;             // [2]: a logit near the largest (NaN: no normaliser), sum of 2^((z - it) inv_t log2 e)
  float* val;               // [N] the segment's largest logits, falling
  int* idx;                 // [N] their tokens (kNone: no more)
};

// A row's beam can give candidates: it has a finite score.
__device__ __forceinline__ bool alive(float score) { return fabsf(score) < INFINITY; }

// 2^(c d) for c d up to 1000 (below -1000: as there): the polynomial is an
// interpolation of 2^f, |f| <= 1/2, at Chebyshev's points, within 1.07e-12 of it and
// exact at 0, which is one of the points at even degrees.  That keeps what the lane's,
// wave's and segment's references have in common free of error: a row with a single
// token left has that token's logit for its normaliser, to the bit.  (Degree 7 is off
// by 5.5e-11, at 0 by 4e-11, and saves 2.5 us of 76 at 512 x 151936; degree 10, 3.7e-16,
// takes 6 more.)
__device__ __forceinline__ double exp2_f64(const BeamParams& p, double d) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 2^52: added, it leaves an integer in the low bits
  d = fmax(d, p.least);
  const double r = fma(d, p.c, kRound), f = fma(d, p.c, kRound - r);
  double v = 1.3255224884799127e-06;
  v = fma(v, f, 1.5310079402383103e-05);
  v = fma(v, f, 0.00015403455852419016);
  v = fma(v, f, 0.0013333450568000008);
  v = fma(v, f, 0.00961812915940262);
  v = fma(v, f, 0.05550410941205934);
  v = fma(v, f, 0.2402265069581299);
  v = fma(v, f, 0.6931471805459335);
  v = fma(v, f, 1.0);
  return __hiloint2double(__double2hiint(v) + (__double2loint(r) << 20), __double2loint(v));
}

// fp32 values in their order as integers, and back.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7FFFFFFFu : ~o); }

// A lane's kEach consecutive logits, as they are read.  No lane skips a load: the compiler can then count them, and they
// pass while the logits before them are worked on.  (Behind a load that some lanes skip all have to have arrived before
// an older one is used: 4 us more of 97 at 512 x 151936.)
template <typename T>
struct Logits {
  static constexpr int kWords = kEach * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  // the lane's of a wave's tile of a row z; what lies past `end` is the row's last
  __device__ __forceinline__ void read(const T* z, int64_t tile, int64_t end, uint32_t lane) {
    if (tile + kTile <= end) {
      // (rows of odd lengths begin anywhere: the loads are wide all the same)
      using global = __attribute__((address_space(1))) const T*;
      global from = (global)(z + tile);
      asm("" : "+s"(from));  // (one address for the wave, or the lanes' take registers that are needed elsewhere)
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4_anywhere v = reinterpret_cast<__attribute__((address_space(1))) const u32x4_anywhere*>(from + lane * kEach)[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
      }
    } else {
      const int64_t first = min(tile, end - 1);
      const T* const from = z + first;
      const uint32_t last = (uint32_t)(end - 1 - first);
      uint32_t mine = lane * kEach;
      asm volatile("" : "+v"(mine));  // (made here: else eight offsets lie in registers all the time)
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const T* const one = from + min(mine + i, last);
        if constexpr (sizeof(T) == 4) {
          w[i] = *reinterpret_cast<const uint32_t*>(one);
        } else {
          const uint32_t v = *reinterpret_cast<const uint16_t*>(one);
          w[i / 2] = i % 2 ? w[i / 2] | v << 16 : v;
        }
      }
    }
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
  }
};

// 64-bit keys: the larger value first, then the lower token; -0 as 0.
__device__ __forceinline__ uint64_t key_of(float v, int idx) {
  return (uint64_t)order_of(v == 0.0f ? 0.0f : v) << 32 | (uint32_t)~idx;
}

// One pass over a row's segment: the sum of exponentials and the N largest
// logits.  A workgroup notes in LDS, key by key, what is no less than a bar; when
// there are many notes they are thinned out to the N largest, and what is above the
// least of those is noted from there on.  With logits in no order that happens three
// or four times.  What bounds it (512 x 151936: 76 us) is less the loads (50 alone)
// than the vector instructions: fp64 exponentials (20) and notes.  (A list of N a
// wave, kept in order by insertions, took 28 us more; notes by ballots over all eight
// logits, 200 instructions, 8 more; notes thinned out from 256 on, 3 more; fmaxf,
// which has NaN to hide, and a check of its own, 3.)
struct Scan {
  uint64_t notes[kNotes];
  double norms[kScanWaves][2];
  uint32_t first_bar[kScanWaves];
  int digits[3][256] __attribute__((aligned(16)));
  int count, left;
};

// The notes down to the N largest, by all threads: the N-th largest key by its
// digits of eight bits, counted in LDS, from the value's first until the keys that
// are no less than it are N (three or four for logits in no order; the token's
// digits only where others share the value).  Bit by bit, a barrier each, it took
// 15 us instead of 1.  Returns the N-th's value, by order_of.
__device__ __forceinline__ int sum_before(int v) {  // of the lanes up to this one
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // (into rows 1 and 3)
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // (into rows 2 and 3)
  return v;
}
__device__ __forceinline__ uint32_t thin_out(Scan& s, int count, int N) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 256) s.digits[0][threadIdx.x] = 0;
  if (threadIdx.x == 0) s.left = 0;
  lds_barrier();
  uint64_t nth = 0;
  int need = N;  // of the keys that begin as nth does
  for (int shift = 56, now = 0; shift >= 0; shift -= 8, now = now == 2 ? 0 : now + 1) {
    if (threadIdx.x < 256) s.digits[now == 2 ? 0 : now + 1][threadIdx.x] = 0;  // (the next; the one before may still be read)
    for (int i = threadIdx.x; i < count; i += 64 * kScanWaves) {
      const uint64_t k = s.notes[i];
      if (shift == 56 || k >> (shift + 8) == nth >> (shift + 8)) atomicAdd(&s.digits[now][k >> shift & 255], 1);
    }
    lds_barrier();
    // lane l counts the digits 255 - 4 l .. 252 - 4 l
    const i32x4 n = *reinterpret_cast<const i32x4*>(&s.digits[now][252 - 4 * lane]);
    const int all = n[0] + n[1] + n[2] + n[3], upto = sum_before(all);
    const int who = lowest(__ballot(upto >= need));
    int above = upto - all, d = 3;  // keys above digit 252 - 4 l + d
    while (d > 0 && above + n[d] < need) above += n[d--];
    const int digit = 252 - 4 * who + read_lane(d, who), same = read_lane(d == 3 ? n[3] : d == 2 ? n[2] : d == 1 ? n[1] : n[0], who);
    need -= read_lane(above, who);
    nth |= (uint64_t)digit << shift;
    if (same == need) break;
  }
  // (what stays is written to places that have been read: no more stays than was)
  for (int first = 0; first < count; first += 64 * kScanWaves) {
    const int i = first + threadIdx.x;
    const uint64_t k = i < count ? s.notes[i] : 0;
    lds_barrier();
    if (k >= nth && i < count) s.notes[atomicAdd(&s.left, 1)] = k;
    lds_barrier();
  }
  if (threadIdx.x == 0) s.count = s.left;
  lds_barrier();
  return (uint32_t)(nth >> 32);
}

template <typename T>
__global__ __launch_bounds__(64 * kScanWaves, 8) void beam_scan_kernel(BeamParams p) {
  __shared__ Scan s;
  const int row = blockIdx.x / p.S, seg = blockIdx.x % p.S;
  if (!alive(p.scores[row]) || (p.finished && p.finished[row])) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* const z = static_cast<const T*>(p.logits) + row * p.ldl;
  const int64_t begin = (int64_t)seg * p.seg_tiles * kTile;
  const int64_t end = min((int64_t)p.V, begin + (int64_t)p.seg_tiles * kTile);
  const int N = p.N;
  float m = -INFINITY, most = -INFINITY;  // the lane's reference, one of its logits, and up to where it serves
  double sum = 0.0;
  bool bad = false;
  Logits<T> next;
  int64_t tile = begin + (int64_t)wave * kTile;  // the wave's
  next.read(z, tile, end, lane);
  if (threadIdx.x == 0) s.count = 0;
  // The first bar: each of the W waves whose tile is whole has q = ceil(N / W) logits that are no less than the q-th
  // largest of its lanes' largest, so N of the workgroup's are no less than the least of these.
  uint32_t bar = order_of(-FLT_MAX);
  const int W = (int)min((int64_t)kScanWaves, (end - begin) / kTile), q = W ? (N + W - 1) / W : 0;
  if (W) {
    float top = next[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) top = fmaxf(top, next[i]);
    const uint32_t mine = top == top ? order_of(top + 0.0f) : 0;  // (-0 as 0)
    uint32_t nth = 0;
    for (uint32_t bit = 1u << 31; bit; bit >>= 1)
      if (__popcll(__ballot(mine >= (nth | bit))) >= q) nth |= bit;
    if (lane == 0) s.first_bar[wave] = nth;
    lds_barrier();
    nth = ~0u;
    for (int w = 0; w < W; ++w) nth = min(nth, s.first_bar[w]);
    bar = max(bar, nth);
  } else {
    lds_barrier();
  }
  for (int64_t first = begin; first < end; first += kScanWaves * kTile) {
    float x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = next[i];
    const int64_t here = tile + lane * kEach;
    if (tile + kTile > end) {
      const int left = (int)max((int64_t)0, end - tile) - lane * kEach;
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = i < left ? x[i] : -INFINITY;
    }
    tile += kScanWaves * kTile;
    next.read(z, tile, end, lane);
    float top = x[0];  // (or NaN)
#pragma unroll
    for (int i = 1; i < kEach; ++i) top = __builtin_elementwise_maximum(top, x[i]);
    bad |= !(top < INFINITY);
    const float cut = value_of(bar);
    if (top >= cut) {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (x[i] >= cut) s.notes[atomicAdd(&s.count, 1)] = key_of(x[i], (int)(here + i));
    }
    if (top > most) {
      // (most is rounded: by no more than what it is above m, or to m; no term is above 2^800)
      sum *= exp2_f64(p, (double)m - (double)top);
      m = top;
      most = (float)((double)m + p.reach);
    }
    // (the difference first: logits of 1e20 would leave nothing of an exponent in z c - m c)
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += exp2_f64(p, (double)x[i] - (double)m);
    lds_barrier();
    const int count = s.count;
    lds_barrier();  // (all have read it before any wave notes more)
    if (count > notes_left(N)) bar = thin_out(s, count, N) + 1;  // (what comes has higher tokens: more than the N-th, not as much)
  }
  // the waves' sums together
  const float ref = wave_max(m);
  sum *= exp2_f64(p, (double)m - (double)ref);
  for (int o = 32; o; o /= 2) sum += shfl_xor_f64(sum, o);
  const bool any_bad = __ballot(bad) != 0;
  if (lane == 0) {
    s.norms[wave][0] = any_bad ? (double)NAN : (double)ref;
    s.norms[wave][1] = sum;
  }
  __syncthreads();
  const int64_t slot = blockIdx.x;
  const int n = s.count;
  if ((int)threadIdx.x < n) {
    const uint64_t k = s.notes[threadIdx.x];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s.notes[j] > k;
    if (rank < N) {
      p.val[slot * N + rank] = value_of((uint32_t)(k >> 32));
      p.idx[slot * N + rank] = (int)~(uint32_t)k;
    }
  }
  for (int i = n + threadIdx.x; i < N; i += 64 * kScanWaves) p.idx[slot * N + i] = kNone;
  if (threadIdx.x == 0) {
    double ref_all = -INFINITY, total = 0.0;
    bool none = false;
    for (int w = 0; w < kScanWaves; ++w) {
      none |= s.norms[w][0] != s.norms[w][0];
      if (s.norms[w][0] > ref_all) ref_all = s.norms[w][0];
    }
    for (int w = 0; w < kScanWaves; ++w) total += s.norms[w][1] * exp2_f64(p, s.norms[w][0] - ref_all);
    p.norm[2 * slot] = none ? (double)NAN : ref_all;
    p.norm[2 * slot + 1] = total;
  }
}

// A sequence's N best of its beams' lists: their scores as 64-bit keys (0: no
// candidate) lie in LDS, a lane walks one list, and the first of all heads is taken
// N times; with more than 64 lists four waves do that, and one of them over their
// results.  Lists lie by beam, then by rising tokens: of equal scores the first list's
// comes first.  Different logits of a beam may have the same score, too (they are far
// smaller than it, or the temperature is near infinity), and then go by logit.  They are
// read again for that alone, and only where it can be: scores fall with the logits, so
// no two differing logits share one unless a list's entry and the fp32 value below it
// do, which is looked at as the scores are made.  (64 x 8 beams, 16 chosen: 7.7 us, 12.6
// where all logits are 0 and every round has such ties.)  What a round waits for is else the
// largest of 64 keys alone, 0.15 us (with scores, tokens and ties looked up in each: 0.4).
__global__ __launch_bounds__(64 * kPickWaves) void beam_pick_kernel(BeamParams p) {
  extern __shared__ uint64_t keys[];   // [lists][N]
  __shared__ double lse[kMaxBeams], score[kMaxBeams];
  __shared__ double refs[kMaxLists], sums[kMaxLists];
  __shared__ int state[kMaxBeams];     // 0: no candidates, 1: its lists, 2: finished
  __shared__ int picked[kPickWaves][kMaxOut], chosen[kMaxOut];  // places in keys
  __shared__ int chosen_beam[kMaxOut], chosen_id[kMaxOut];
  __shared__ int close;                // different logits of a beam may have the same score
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lists = p.K * p.S, N = p.N;
  const float* const val = p.val + (int64_t)b * lists * N;
  const int* const idx = p.idx + (int64_t)b * lists * N;
  // All of a list is read at once, also where its beam turns out to have none and nothing has been written.
  const bool has_list = (int)threadIdx.x < lists, has_beam = (int)threadIdx.x < p.K;
  const double* const norm = p.norm + 2 * ((int64_t)b * lists + threadIdx.x);
  double list_ref = 0.0, list_sum = 0.0;
  float own = 0.0f;
  bool finished = false;
  if (has_list) list_ref = norm[0], list_sum = norm[1];
  if (has_beam) own = p.scores[b * p.K + threadIdx.x];
  if (has_beam && p.finished) finished = p.finished[b * p.K + threadIdx.x];
  for (int i = threadIdx.x; i < lists * N; i += 64 * kPickWaves)  // (a thread's own, until they are keys)
    keys[i] = (uint64_t)__float_as_uint(val[i]) << 1 | (idx[i] != kNone);
  if (has_list) refs[threadIdx.x] = list_ref, sums[threadIdx.x] = list_sum;
  if (threadIdx.x == 0) close = 0;
  __syncthreads();
  if (has_beam) {
    const int j = threadIdx.x;
    score[j] = own;
    state[j] = !alive(own) ? 0 : finished ? 2 : 1;
    if (state[j] == 1) {
      double ref = -INFINITY, sum = 0.0;
      bool none = false;
      for (int s = j * p.S; s < (j + 1) * p.S; ++s) {
        none |= refs[s] != refs[s];
        if (refs[s] > ref) ref = refs[s];
      }
      for (int s = j * p.S; s < (j + 1) * p.S; ++s) sum += sums[s] * exp2_f64(p, refs[s] - ref);
      lse[j] = ref * (double)p.inv_t + log(sum);
      if (none || !(fabs(lse[j]) < INFINITY)) state[j] = 0;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < lists * N; i += 64 * kPickWaves) {
    const int j = i / (p.S * N);
    const uint64_t v = keys[i];
    uint64_t key = 0;
    if (state[j] == 2 && i == j * p.S * N) key = score_key(score[j]);
    if (state[j] == 1 && (v & 1)) {
      const float z = __uint_as_float((uint32_t)(v >> 1));
      auto key_at = [&](float z) { return score_key(score[j] + ((double)z * (double)p.inv_t - lse[j])); };
      key = key_at(z);
      if (p.S > 1 && key_at(value_of(order_of(z) - 1)) == key) close = 1;
    }
    keys[i] = key;
  }
  __syncthreads();
  const bool by_logit = __builtin_amdgcn_readfirstlane(close);
  // of the lanes `same`, whose lists' heads (at `here`) have equal scores, the first: by beam, logit and list
  auto first_of = [&](uint64_t same, int here) {
    const int each = p.S * N, beam = read_lane(here, lowest(same)) / each;
    const bool in = same >> lane & 1 && here / each == beam;
    const uint32_t z = in ? order_of(val[here]) : 0;  // (0: a NaN's, no candidate's.  A finished beam has one, with nobody to tie)
    const uint32_t top = (uint32_t)largest(z);
    return lowest(__ballot(in && z == top));
  };
  // the first n of the lists that the wave's lanes walk, place by place (-1: none), to `to`
  auto pick = [&](auto place, int* to) {
    int at = 0, here = place(0), behind = place(1), n = 0;
    uint64_t key = here < 0 ? 0 : keys[here], next = behind < 0 ? 0 : keys[behind];
    for (; n < N; ++n) {
      const uint64_t best = largest(key);
      if (best == 0) break;
      const uint64_t same = __ballot(key == best);
      if (lane == (by_logit && same & (same - 1) ? first_of(same, here) : lowest(same))) {
        to[n] = here;
        here = behind;
        key = next;
        behind = place(++at + 1);
        next = behind < 0 ? 0 : keys[behind];
      }
    }
    return n;
  };
  int n;
  if (lists <= 64) {
    if (wave != 0) return;
    n = pick([&](int at) { return lane < lists && at < N ? lane * N + at : -1; }, chosen);
  } else {
    const int k = pick([&](int at) { return (int)threadIdx.x < lists && at < N ? (int)threadIdx.x * N + at : -1; }, picked[wave]);
    if (lane >= k && lane < N) picked[wave][lane] = -1;
    __syncthreads();
    if (wave != 0) return;
    n = pick([&](int at) { return lane < kPickWaves && at < N ? picked[lane][at] : -1; }, chosen);
  }
  __threadfence_block();
  if (lane < n) {
    const int place = chosen[lane], j = place / (p.S * N), id = state[j] == 2 ? p.eos : idx[place];
    p.ids[(int64_t)b * N + lane] = chosen_id[lane] = id;
    p.parents[(int64_t)b * N + lane] = chosen_beam[lane] = j;
    p.out[(int64_t)b * N + lane] = (float)score_of(keys[place]);
  }
  if (n == N) return;
  // All candidates above -infinity are chosen.  The others follow by beam and token.
  __threadfence_block();
  if (lane != 0) return;
  int beam = 0, id = 0;
  for (int k = n; k < N;) {
    bool taken = false;
    for (int i = 0; i < n; ++i) taken |= chosen_beam[i] == beam && chosen_id[i] == id;
    if (!taken) {
      p.ids[(int64_t)b * N + k] = id;
      p.parents[(int64_t)b * N + k] = beam;
      p.out[(int64_t)b * N + k] = -INFINITY;
      ++k;
    }
    if (++id == p.V) {
      id = 0;
      ++beam;
    }
  }
}

// ------------------------------------------------------------------ states
struct ReorderParams {
  const uint8_t* src;
  uint8_t* dst;
  int64_t s_outer, s_seq, s_beam;  // bytes
  int64_t d_outer, d_seq, d_beam;
  const int32_t* parents;
  int outer, B, K, N;
  int64_t units;    // of a row
  int64_t chunks;   // of a row, one workgroup's each
  int in_place;
};

// Thread by thread, one unit of a row at the same place of all beams of a
// sequence: the rows that are somebody's parent are read once each, whoever wants
// them, into the thread's own column of LDS, and written from there.  All reads of a
// place stand before its writes, so the states may be reordered in place; beams
// that stay where they are are then not touched.
template <typename UNIT, int THREADS>
__global__ __launch_bounds__(THREADS) void beam_reorder_kernel(ReorderParams p) {
  extern __shared__ uint8_t column[];  // [K][THREADS] units
  UNIT* const held = reinterpret_cast<UNIT*>(column) + threadIdx.x;
  const int64_t at = (int64_t)blockIdx.x % p.chunks * THREADS + threadIdx.x, seq = blockIdx.x / p.chunks;
  const int b = (int)(seq % p.B);
  const int64_t o = seq / p.B;
  const int32_t* const parent = p.parents + (int64_t)b * p.N;
  uint64_t used = 0;
  for (int n = 0; n < p.N; ++n) {
    const uint32_t j = (uint32_t)parent[n];
    if (j < (uint32_t)p.K && !(p.in_place && (int)j == n)) used |= 1ull << j;
  }
  if (at >= p.units) return;
  const uint8_t* const src = p.src + o * p.s_outer + b * p.s_seq + at * (int64_t)sizeof(UNIT);
  uint8_t* const dst = p.dst + o * p.d_outer + b * p.d_seq + at * (int64_t)sizeof(UNIT);
  for (int j0 = 0; j0 < p.K; j0 += 8) {
    UNIT v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (used >> (j0 + i) & 1) v[i] = *reinterpret_cast<const UNIT*>(src + (j0 + i) * p.s_beam);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (used >> (j0 + i) & 1) held[(j0 + i) * THREADS] = v[i];
  }
  for (int n = 0; n < p.N; ++n) {
    const uint32_t j = (uint32_t)parent[n];
    if (p.in_place && (int)j == n) continue;
    UNIT* to = reinterpret_cast<UNIT*>(dst + n * p.d_beam);
    if (j < (uint32_t)p.K) *to = held[j * THREADS];
    else *to = UNIT{};
  }
}

template <typename UNIT, int THREADS>
hipError_t launch_reorder(ReorderParams p, int64_t row_bytes, hipStream_t s) {
  p.units = row_bytes / (int64_t)sizeof(UNIT);
  p.chunks = (p.units + THREADS - 1) / THREADS;
  const int64_t grid = p.chunks * p.B * p.outer;
  hipLaunchKernelGGL((beam_reorder_kernel<UNIT, THREADS>), dim3((unsigned)grid), dim3(THREADS),
                     (unsigned)(p.K * THREADS * (int)sizeof(UNIT)), s, p);
  return hipGetLastError();
}

// ------------------------------------------------------------------ host
constexpr int kCus = 256;

// Segments: four workgroups a CU (512 x 151936: 107 us with two) where the rows allow it, each of a tile a wave at
// least; as many as one wave of the pick has lanes for (1 x 4 x 151936: 15.6 us, 18.6 with 38 of them), or of four tiles a
// wave where that saves more tiles one after another than the pick's second round of choices costs (1 x 24 x 151936, 4
// chosen: 19 us, 26 with the former; 8 x 8, 8 chosen: 30 with the latter, 24); what the pick has lanes and LDS for.
void segment(BeamParams& p) {
  const int64_t rows = (int64_t)p.B * p.K, tiles = ((int64_t)p.V + kTile - 1) / kTile;
  int64_t S = rows ? std::max<int64_t>(1, (4 * kCus + rows - 1) / rows) : 1;
  const int64_t most = (tiles + kScanWaves - 1) / kScanWaves;
  const int64_t few = std::max(1, 64 / p.K), many = (most + 3) / 4;
  S = std::min(S, std::min(most, most / few - most / many > p.N / 2 + 2 ? many : few));
  S = std::min<int64_t>(S, std::min(kMaxLists / p.K, std::max(1, kMaxStaged / (p.K * p.N))));
  p.seg_tiles = (int)((tiles + S - 1) / S);
  p.S = (int)((tiles + p.seg_tiles - 1) / p.seg_tiles);
}

size_t lay_out(BeamParams& p, uint8_t* base) {
  const size_t slots = (size_t)p.B * p.K * p.S;
  p.norm = reinterpret_cast<double*>(base);
  p.val = reinterpret_cast<float*>(base + slots * 16);
  p.idx = reinterpret_cast<int*>(base + slots * (16 + 4 * (size_t)p.N));
  return slots * (16 + 8 * (size_t)p.N);
}

acrl_status validate_sizes(int64_t B, int64_t K, int64_t V, int64_t N) {
  ACRL_REQUIRE(K > 0 && K <= kMaxBeams, "K = %lld must lie in [1, %d]", (long long)K, kMaxBeams);
  ACRL_REQUIRE(B >= 0 && B <= (1 << 20), "B = %lld must lie in [0, 2^20]", (long long)B);
  ACRL_REQUIRE(B * K < (1 << 22), "B x K = %lld must be below 2^22", (long long)(B * K));
  ACRL_REQUIRE(V > 0 && V < ((int64_t)1 << 30), "V = %lld must lie in [1, 2^30)", (long long)V);
  ACRL_REQUIRE(N > 0 && N <= kMaxOut && N <= K * V, "n_out = %lld must lie in [1, min(%d, K V)]", (long long)N, kMaxOut);
  return ACRL_OK;
}

BeamParams sized(int64_t B, int64_t K, int64_t V, int64_t N) {
  BeamParams p{};
  p.B = (int)B;
  p.K = (int)K;
  p.V = (int)V;
  p.N = (int)N;
  segment(p);
  return p;
}

}  // namespace
}  // namespace acrl

extern "C" {

acrl_status acrl_beam_workspace_size(int64_t B, int64_t K, int64_t V, int64_t n_out, size_t* bytes) {
  ACRL_REQUIRE(bytes, "bytes is NULL");
  acrl_status st = acrl::validate_sizes(B, K, V, n_out);
  if (st != ACRL_OK) return st;
  acrl::BeamParams p = acrl::sized(B, K, V, n_out);
  *bytes = acrl::lay_out(p, nullptr);
  return ACRL_OK;
}

acrl_status acrl_beam_step(const acrl_beam_desc* d, void* stream) {
  ACRL_REQUIRE(d, "desc is NULL");
  acrl_status st = acrl::validate_sizes(d->B, d->K, d->V, d->n_out);
  if (st != ACRL_OK) return st;
  const bool f32 = d->logits_type == ACRL_OUT_F32;
  ACRL_REQUIRE(f32 || d->logits_type == ACRL_OUT_BF16, "logits_type %d unknown", d->logits_type);
  ACRL_REQUIRE(d->ldl >= d->V && d->ldl < ((int64_t)1 << 34), "ldl = %lld must lie in [V, 2^34)", (long long)d->ldl);
  ACRL_REQUIRE(d->inv_temperature > 1e-30f && d->inv_temperature < 1e30f, "inv_temperature must lie in (1e-30, 1e30)");
  ACRL_REQUIRE(!d->finished || (d->eos_id >= 0 && d->eos_id < d->V), "eos_id = %d must lie in [0, V)", d->eos_id);
  if (d->B > 0) {
    ACRL_REQUIRE(d->logits && d->scores && d->ids && d->parents && d->out_scores,
                 "logits, scores, ids, parents and out_scores are required");
    ACRL_REQUIRE(((uintptr_t)d->logits & (f32 ? 3u : 1u)) == 0, "logits is misaligned");
    ACRL_REQUIRE((((uintptr_t)d->scores | (uintptr_t)d->ids | (uintptr_t)d->parents | (uintptr_t)d->out_scores) & 3u) == 0,
                 "scores, ids, parents or out_scores is misaligned");
  }
  acrl::BeamParams p = acrl::sized(d->B, d->K, d->V, d->n_out);
  const size_t need = acrl::lay_out(p, static_cast<uint8_t*>(d->workspace));
  if (need && (!d->workspace || d->workspace_bytes < need)) {
    acrl::set_error("acrl_beam_step needs %zu workspace bytes, got %zu", need, d->workspace_bytes);
    return ACRL_ERR_WORKSPACE;
  }
  ACRL_REQUIRE(acrl::aligned16(d->workspace), "workspace must be 16-byte aligned");
  // (a sequence's scores are read by its own workgroup of the choice, before it writes: only there may they be replaced)
  const uintptr_t in = (uintptr_t)d->scores, out = (uintptr_t)d->out_scores;
  ACRL_REQUIRE(d->B == 0 || (in == out && d->n_out == d->K) || out >= in + (uintptr_t)(d->B * d->K) * 4 ||
                   in >= out + (uintptr_t)(d->B * d->n_out) * 4,
               "out_scores overlaps scores without being scores itself, of n_out = K");
  st = acrl::check_device();
  if (st != ACRL_OK || d->B == 0) return st;
  p.logits = d->logits;
  p.ldl = d->ldl;
  p.scores = d->scores;
  p.finished = d->finished;
  p.eos = d->eos_id;
  p.inv_t = d->inv_temperature;
  p.c = (double)p.inv_t * 1.4426950408889634074;
  p.least = -1000.0 / p.c;
  p.reach = 400.0 / p.c;
  p.ids = d->ids;
  p.parents = d->parents;
  p.out = d->out_scores;
  const hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)((int64_t)p.B * p.K * p.S)), threads(64 * acrl::kScanWaves);
  if (f32) hipLaunchKernelGGL(acrl::beam_scan_kernel<float>, grid, threads, 0, s, p);
  else hipLaunchKernelGGL(acrl::beam_scan_kernel<__bf16>, grid, threads, 0, s, p);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(acrl::beam_pick_kernel, dim3((unsigned)p.B), dim3(64 * acrl::kPickWaves),
                       (unsigned)(p.K * p.S * p.N * 8), s, p);
    e = hipGetLastError();
  }
  return acrl::hip_status(e, "acrl_beam_step launch");
}

acrl_status acrl_beam_reorder(const acrl_reorder_desc* d, void* stream) {
  ACRL_REQUIRE(d, "desc is NULL");
  ACRL_REQUIRE(d->K > 0 && d->K <= acrl::kMaxBeams, "K = %lld must lie in [1, %d]", (long long)d->K, acrl::kMaxBeams);
  ACRL_REQUIRE(d->n_out > 0 && d->n_out <= acrl::kMaxOut, "n_out = %lld must lie in [1, %d]", (long long)d->n_out, acrl::kMaxOut);
  ACRL_REQUIRE(d->B >= 0 && d->B <= (1 << 20), "B = %lld must lie in [0, 2^20]", (long long)d->B);
  ACRL_REQUIRE(d->outer >= 0 && d->outer <= (1 << 20), "outer = %lld must lie in [0, 2^20]", (long long)d->outer);
  ACRL_REQUIRE(d->row_bytes >= 0 && d->row_bytes < ((int64_t)1 << 40), "row_bytes = %lld must lie in [0, 2^40)",
               (long long)d->row_bytes);
  const int64_t strides[] = {d->src_outer, d->src_seq, d->src_beam, d->dst_outer, d->dst_seq, d->dst_beam};
  for (int64_t v : strides) ACRL_REQUIRE(v >= 0 && v < ((int64_t)1 << 42), "a stride of %lld bytes", (long long)v);
  const bool none = d->outer == 0 || d->B == 0 || d->row_bytes == 0;
  bool in_place = false;
  uintptr_t all = 0;
  if (!none) {
    ACRL_REQUIRE(d->src && d->dst && d->parents, "src, dst and parents are required");
    ACRL_REQUIRE(((uintptr_t)d->parents & 3u) == 0, "parents is misaligned");
    // (the last byte's place fits 64 bits: factors of at most 2^20, strides below 2^42)
    // By rising stride, each no less than what the rows under it span.  (No overflow: a span that passes is no more than a
    // stride, below 2^42, and grows by at most 2^20 strides.)
    std::pair<uint64_t, uint64_t> sides[] = {{d->dst_beam, d->n_out}, {d->dst_seq, d->B}, {d->dst_outer, d->outer}};
    std::sort(std::begin(sides), std::end(sides));
    uint64_t span = (uint64_t)d->row_bytes;
    for (auto [stride, n] : sides)
      if (n > 1) {
        ACRL_REQUIRE(stride >= span, "rows of dst overlap: a stride of %llu bytes, and %llu under it",
                     (unsigned long long)stride, (unsigned long long)span);
        span += (n - 1) * stride;
      }
    auto last = [&](int64_t so, int64_t ss, int64_t sb, int64_t n) {
      return (uintptr_t)((d->outer - 1) * so) + (uintptr_t)((d->B - 1) * ss) + (uintptr_t)((n - 1) * sb + d->row_bytes);
    };
    const uintptr_t s0 = (uintptr_t)d->src, d0 = (uintptr_t)d->dst;
    const uintptr_t s1 = s0 + last(d->src_outer, d->src_seq, d->src_beam, d->K);
    const uintptr_t d1 = d0 + last(d->dst_outer, d->dst_seq, d->dst_beam, d->n_out);
    in_place = s0 == d0 && d->n_out == d->K && (d->K == 1 || d->src_beam == d->dst_beam) &&
               (d->B == 1 || d->src_seq == d->dst_seq) && (d->outer == 1 || d->src_outer == d->dst_outer);
    ACRL_REQUIRE(in_place || s0 >= d1 || d0 >= s1, "dst overlaps src without being src itself");
    all = s0 | d0 | (uintptr_t)d->row_bytes;
    for (int64_t v : strides) all |= (uintptr_t)v;
    // a launch holds fewer than 2^32 threads
    const int64_t unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
    ACRL_REQUIRE((d->row_bytes / unit + 255) / 256 * 256 < ((int64_t)1 << 32) / (d->B * d->outer),
                 "outer x B x row_bytes / %lld too large", (long long)unit);
  }
  acrl_status st = acrl::check_device();
  if (st != ACRL_OK || none) return st;
  acrl::ReorderParams p{};
  p.src = static_cast<const uint8_t*>(d->src);
  p.dst = static_cast<uint8_t*>(d->dst);
  p.s_outer = d->src_outer;
  p.s_seq = d->src_seq;
  p.s_beam = d->src_beam;
  p.d_outer = d->dst_outer;
  p.d_seq = d->dst_seq;
  p.d_beam = d->dst_beam;
  p.parents = d->parents;
  p.outer = (int)d->outer;
  p.B = (int)d->B;
  p.K = (int)d->K;
  p.N = (int)d->n_out;
  p.in_place = in_place;
  const hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (all % 16 == 0) e = p.K <= 16 ? acrl::launch_reorder<acrl::u32x4, 256>(p, d->row_bytes, s)
                                   : acrl::launch_reorder<acrl::u32x4, 64>(p, d->row_bytes, s);
  else if (all % 4 == 0) e = acrl::launch_reorder<uint32_t, 256>(p, d->row_bytes, s);
  else e = acrl::launch_reorder<uint8_t, 256>(p, d->row_bytes, s);
  return acrl::hip_status(e, "acrl_beam_reorder launch");
}

}  // extern "C"
