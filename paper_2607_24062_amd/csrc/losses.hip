// losses.hip -- the clipped policy loss with a KL term and the loss of
// preferred / rejected pairs, each with its gradient with respect to the new
// policy's log-probs (the coef that acrl_lm_head_backward takes).
//
// Layout: slots [B, L] row-major.  A slot's log-probs, weight and advantage are
// read once, its mask twice (for the counts or sums that a coef waits for, and
// with the coef); the terms and sums are fp64, the sums by fixed trees
// (deterministic).
#include "entry.h"
#include "slots.h"

namespace acrl {
namespace {

// e = exp(x); returns exp(x) - 1 - x without cancellation.  x = k ln 2 + r with
// |r| <= ln 2 / 2 (ln 2 in two parts, the first of 33 bits, so that k times it
// is exact), exp(r) = 1 + r + r^2 q(r) with the Taylor series of q to r^11, whose
// next term is below 2^-57: 22 fp64 operations for both values (errors over
// x of 1e-6 .. 200 in size: exp 1.5e-16, the difference 2.8e-15, relative).
__device__ __forceinline__ double exp_rest(double x, double& e) {
  const double c = x < -746.0 ? -746.0 : x > 710.0 ? 710.0 : x;  // (0 and infinity from there on; a NaN stays)
  const double k = rint(c * 1.4426950408889634);
  const double r = fma(k, -1.9082149292705877e-10, fma(k, -0.6931471803691238, c));
  double q = 1.0 / 6227020800.0;
  q = fma(q, r, 1.0 / 479001600.0);
  q = fma(q, r, 1.0 / 39916800.0);
  q = fma(q, r, 1.0 / 3628800.0);
  q = fma(q, r, 1.0 / 362880.0);
  q = fma(q, r, 1.0 / 40320.0);
  q = fma(q, r, 1.0 / 5040.0);
  q = fma(q, r, 1.0 / 720.0);
  q = fma(q, r, 1.0 / 120.0);
  q = fma(q, r, 1.0 / 24.0);
  q = fma(q, r, 1.0 / 6.0);
  q = fma(q, r, 0.5);
  const double rest = r * r * q;
  e = ldexp(1.0 + (r + rest), (int)k);
  return k == 0.0 ? rest : e < INFINITY ? e - 1.0 - x : e;  // (infinite like e, where x is too)
}

// ------------------------------------------------------------------ policy loss
// Sums of a unit of slots: policy term, KL term, clipped, at the dual clip,
// moved, valid (the first two before a_t).
constexpr int kPolicySums = 6;

struct PolicyWs {
  int32_t* n;        // [B] valid slots of a response (-1: its group id is out of range)
  double* share;     // [B] a_t of the response's slots
  int32_t* live;     // [n_groups] non-empty responses of a group
  double* part;      // [kPolicySums][units]
  int64_t bytes;
};
constexpr int kUnitThreads = 256;
constexpr int kOneRows = 1024;  // responses, and groups, whose counts one workgroup holds
constexpr int64_t kMaxResponses = (int64_t)1 << 22;
constexpr int64_t kOneSlots = 4096;  // of a batch that one workgroup does
inline bool one_policy(int64_t B, int64_t L, int64_t n_groups) {
  return B * L <= kOneSlots && B <= kOneRows && n_groups <= kOneRows;
}
// Slots of a workgroup: four a thread, in two turns in a large batch (policy_main_kernel and policy_sum_kernel of 512
// responses of 16384 slots, 1 / 2 / 4 turns: 34.8 + 7.8, 33.4 + 4.9, 35.6 + 4.3 us).
constexpr int64_t kManySlots = (int64_t)1 << 20;
inline int unit_turns(int64_t B, int64_t L) { return B * L <= kManySlots ? 1 : 2; }
inline int unit_slots(int64_t B, int64_t L) { return kUnitThreads * kSlots * unit_turns(B, L); }
inline int64_t units_of_response(int64_t B, int64_t L) {
  const int64_t u = unit_slots(B, L);
  return (L + u - 1) / u;
}
PolicyWs policy_ws(void* base, int64_t B, int64_t L, int64_t n_groups) {
  uint8_t* b = static_cast<uint8_t*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align_up(bytes, 256);
    return b + at;
  };
  PolicyWs w;
  w.n = reinterpret_cast<int32_t*>(take((size_t)B * sizeof(int32_t)));
  w.share = reinterpret_cast<double*>(take((size_t)B * sizeof(double)));
  w.live = reinterpret_cast<int32_t*>(take((size_t)n_groups * sizeof(int32_t)));
  w.part = reinterpret_cast<double*>(take((size_t)B * units_of_response(B, L) * kPolicySums * sizeof(double)));
  w.bytes = (int64_t)off;
  return w;
}

// a_t of a response of n valid slots (-1: of no group); v = {valid slots,
// non-empty responses or groups} of the batch, live = those of its group.
__device__ __forceinline__ double share_of(const acrl_policy_loss_desc& p, int n, int live, const double (&v)[2]) {
  if (n < 0) return __builtin_nan("");
  if (n == 0) return 0.0;
  switch (p.aggregate) {
    case ACRL_AGG_GROUP: return 1.0 / (v[1] * live * n);
    case ACRL_AGG_SEQUENCE: return 1.0 / (v[1] * n);
    case ACRL_AGG_TOKEN: return 1.0 / v[0];
    default: return 1.0 / (double)p.norm;
  }
}

// Nonzero bytes of the L bytes at m, by the lanes of a group of NT threads
// (their sum is the count): 16-byte loads of what lies 16-byte aligned.
__device__ __forceinline__ int nonzero_bytes(uint32_t x) {
  return __popc((((x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | x) & 0x80808080u);
}
template <int NT>
__device__ __forceinline__ int count_valid(const uint8_t* __restrict__ m, int64_t L, int lane) {
  const int64_t head = min((int64_t)(-(uintptr_t)m & 15), L), body = (L - head) / 16, tail = head + 16 * body;
  int c = lane < head ? m[lane] != 0 : 0;
  const uint4* v = reinterpret_cast<const uint4*>(m + head);
#pragma unroll 4
  for (int64_t j = lane; j < body; j += NT) {
    const uint4 x = v[j];
    c += nonzero_bytes(x.x) + nonzero_bytes(x.y) + nonzero_bytes(x.z) + nonzero_bytes(x.w);
  }
  if (tail + lane < L) c += m[tail + lane] != 0;  // (fewer than 16)
  return c;
}
__device__ __forceinline__ int lane_sum_int(int c) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) c += __shfl_xor(c, s);
  return c;
}
__device__ __forceinline__ bool in_no_group(const acrl_policy_loss_desc& p, int64_t i) {
  return p.aggregate == ACRL_AGG_GROUP && (p.group_of_seq[i] < 0 || p.group_of_seq[i] >= p.n_groups);
}

// Valid slots of each response: a wavefront each.
__global__ __launch_bounds__(kUnitThreads) void policy_count_kernel(acrl_policy_loss_desc p, int32_t* n) {
  const int64_t i = (int64_t)blockIdx.x * (kUnitThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (i >= p.B) return;
  const int c = lane_sum_int(count_valid<64>(p.mask + i * p.L, p.L, lane));
  if (lane == 0) n[i] = in_no_group(p, i) ? -1 : c;
}

// a_t of every response, by one workgroup (more responses or groups than the
// main kernel's workgroups look through themselves).
__global__ __launch_bounds__(1024) void policy_share_kernel(acrl_policy_loss_desc p, PolicyWs ws) {
  __shared__ BlockShared<2, 1024> sh;
  const bool groups = p.aggregate == ACRL_AGG_GROUP;
  double v[2] = {0, 0}, unused = 0.0;  // tokens, non-empty responses (groups)
  if (groups) {
    for (int64_t g = threadIdx.x; g < p.n_groups; g += 1024) ws.live[g] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < p.B; i += 1024)
      if (ws.n[i] > 0) atomicAdd(&ws.live[p.group_of_seq[i]], 1);
    __syncthreads();
    for (int64_t g = threadIdx.x; g < p.n_groups; g += 1024)
      if (atomicAdd(&ws.live[g], 0) > 0) v[1] += 1.0;
  } else {
    for (int64_t i = threadIdx.x; i < p.B; i += 1024) {
      v[0] += ws.n[i];
      v[1] += ws.n[i] > 0 ? 1.0 : 0.0;
    }
  }
  block_stats<2, 1024>(v, unused, sh);
  for (int64_t i = threadIdx.x; i < p.B; i += 1024)
    ws.share[i] = share_of(p, ws.n[i], groups && ws.n[i] > 0 ? atomicAdd(&ws.live[p.group_of_seq[i]], 0) : 0, v);
}

// a_t of response i by a workgroup of the main kernel, from the counts of all.
__device__ __forceinline__ double own_share(const acrl_policy_loss_desc& p, const int32_t* n, int64_t i) {
  __shared__ BlockShared<2, kUnitThreads> sh;
  __shared__ int live[kOneRows];
  const bool groups = p.aggregate == ACRL_AGG_GROUP;
  double v[2] = {0, 0}, unused = 0.0;
  if (groups) {
    for (int g = threadIdx.x; g < p.n_groups; g += kUnitThreads) live[g] = 0;
    __syncthreads();
  }
  for (int j = threadIdx.x; j < p.B; j += kUnitThreads) {
    const int c = n[j];
    if (c <= 0) continue;
    v[0] += c;
    if (groups) atomicAdd(&live[p.group_of_seq[j]], 1);
    else v[1] += 1.0;
  }
  if (groups) {
    __syncthreads();
    for (int g = threadIdx.x; g < p.n_groups; g += kUnitThreads) v[1] += live[g] > 0 ? 1.0 : 0.0;
  }
  block_stats<2, kUnitThreads>(v, unused, sh);
  return share_of(p, n[i], groups && n[i] > 0 ? live[p.group_of_seq[i]] : 0, v);
}

// One slot: its terms added to v, its d(-w m + kl_coef k) / d logp_new returned.
__device__ __forceinline__ double policy_slot(const acrl_policy_loss_desc& p, double ln, double lo, double lr,
                                              double A, double w, double (&v)[kPolicySums]) {
  const double delta = ln - lo, lo_r = 1.0 - (double)p.eps_low, hi_r = 1.0 + (double)p.eps_high;
  double r;
  v[4] += exp_rest(delta, r);
  const bool over = A > 0 && r > hi_r, under = A < 0 && r < lo_r;
  const bool dual = p.dual_clip > 0.0f && A < 0 && r > (double)p.dual_clip;
  const double eff = over ? hi_r : under ? lo_r : dual ? (double)p.dual_clip : r;
  v[0] -= w * (eff * A);
  v[2] += over || under ? 1.0 : 0.0;
  v[3] += dual ? 1.0 : 0.0;
  v[5] += 1.0;
  double g = over || under || dual ? 0.0 : -w * (r * A);
  if (p.logp_ref) {
    const double q = lr - ln;
    double k, dk;
    if (p.kl_estimator == ACRL_KL_K1) {
      k = -q;
      dk = 1.0;
    } else if (p.kl_estimator == ACRL_KL_K2) {
      k = 0.5 * q * q;
      dk = -q;
    } else {
      double e;
      k = exp_rest(q, e);
      dk = q < -1.0 ? 1.0 - e : -(k + q);  // 1 - exp(q): k + q loses it below, 1 - e next to 0
    }
    v[1] += k;
    if (p.kl_coef > 0.0f) g += (double)p.kl_coef * dk;  // (no 0 * infinity)
  }
  return g;
}

// Where the main kernel has a_t from.
enum ShareFrom { kShareNorm, kShareOwn, kShareWs };

// One unit of a response's slots: coef, and the unit's sums.  Where a thread's
// mask leaves nothing, nothing else is loaded.  512 responses of up to 16384
// slots (126 MB): 33.4 us, 3.8 TB/s; the fp64 operations alone are 20 us of the
// SIMDs' time (12.4 M wavefront instructions), and cover the loads in part.
// (The sums added up by the workgroup that ends last, behind a device-wide
// fence, instead of by policy_sum_kernel: 216 us, 14.4 for 7.4 at 64 x 4096.)
template <int TURNS, bool VEC>
__global__ __launch_bounds__(kUnitThreads) void policy_main_kernel(acrl_policy_loss_desc p, PolicyWs ws,
                                                                   int64_t units, int from) {
  __shared__ BlockShared<kPolicySums, kUnitThreads> sh;
  const int64_t i = blockIdx.x / units, u = blockIdx.x - i * units;
  const int64_t base = i * p.L;
  const double a = from == kShareNorm ? 1.0 / (double)p.norm : from == kShareOwn ? own_share(p, ws.n, i) : ws.share[i];
  double v[kPolicySums] = {}, unused = 0.0;
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int64_t j = (u * TURNS + t) * kUnitThreads * kSlots + first_slot<kUnitThreads, VEC>();
    if (j >= p.L) break;
    uint8_t m[kSlots];
    float ln[kSlots] = {}, lo[kSlots] = {}, lr[kSlots] = {}, w[kSlots] = {1.0f, 1.0f, 1.0f, 1.0f}, A[kSlots] = {}, c[kSlots] = {};
    load_mask<kUnitThreads, VEC>(p.mask, base, j, p.L, m);
    if (m[0] | m[1] | m[2] | m[3]) {
      load_slots<kUnitThreads, VEC>(p.logp_new, base, j, p.L, ln);
      load_slots<kUnitThreads, VEC>(p.logp_old, base, j, p.L, lo);
      if (p.logp_ref) load_slots<kUnitThreads, VEC>(p.logp_ref, base, j, p.L, lr);
      if (p.weight) load_slots<kUnitThreads, VEC>(p.weight, base, j, p.L, w);
      if (p.adv_per_token) {
        load_slots<kUnitThreads, VEC>(p.adv, base, j, p.L, A);
      } else {
#pragma unroll
        for (int k = 0; k < kSlots; ++k) A[k] = p.adv[i];
      }
#pragma unroll
      for (int k = 0; k < kSlots; ++k)
        if (m[k]) c[k] = (float)(a * policy_slot(p, ln[k], lo[k], lr[k], A[k], w[k], v));
    }
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(p.coef + base + j) = make_float4(c[0], c[1], c[2], c[3]);
    } else {
#pragma unroll
      for (int k = 0; k < kSlots; ++k)
        if (j + k * kUnitThreads < p.L) p.coef[base + j + k * kUnitThreads] = c[k];
    }
  }
  block_stats<kPolicySums, kUnitThreads>(v, unused, sh);
  if (threadIdx.x == 0) {
    const bool in = a == a;  // (a response of no group enters nothing)
    const int64_t n = gridDim.x;
#pragma unroll
    for (int k = 0; k < kPolicySums; ++k) ws.part[k * n + blockIdx.x] = in ? (k < 2 ? a * v[k] : v[k]) : 0.0;
  }
}

__device__ __forceinline__ void policy_finish(const acrl_policy_loss_desc& p, const double (&v)[kPolicySums]) {
  p.loss[0] = p.kl_coef > 0.0f ? v[0] + (double)p.kl_coef * v[1] : v[0];
  if (!p.stats) return;
  const double inv = v[5] > 0 ? 1.0 / v[5] : 0.0;
  p.stats[ACRL_PSTAT_POLICY] = v[0];
  p.stats[ACRL_PSTAT_KL] = v[1];
  p.stats[ACRL_PSTAT_CLIPPED] = v[2] * inv;
  p.stats[ACRL_PSTAT_DUAL] = v[3] * inv;
  p.stats[ACRL_PSTAT_MOVED] = v[4] * inv;
  p.stats[ACRL_PSTAT_N_TOKENS] = v[5];
}

// loss and stats from the units' sums, by one workgroup.
__global__ __launch_bounds__(1024) void policy_sum_kernel(acrl_policy_loss_desc p, PolicyWs ws, int64_t n) {
  __shared__ BlockShared<kPolicySums, 1024> sh;
  double v[kPolicySums] = {}, unused = 0.0;
#pragma unroll 4
  for (int64_t u = threadIdx.x; u < n; u += 1024) {
#pragma unroll
    for (int k = 0; k < kPolicySums; ++k) v[k] += ws.part[k * n + u];
  }
  block_stats<kPolicySums, 1024>(v, unused, sh);
  if (threadIdx.x == 0) policy_finish(p, v);
}

// All of it in one workgroup, a slot a thread and turn: a small batch is
// launches and waits (4 responses of 64 slots 5.7 us; 14.5 by the four kernels).
__global__ __launch_bounds__(1024) void policy_one_kernel(acrl_policy_loss_desc p) {
  __shared__ BlockShared<2, 1024> sh2;
  __shared__ BlockShared<kPolicySums, 1024> sh;
  __shared__ int n[kOneRows], live[kOneRows];
  __shared__ double share[kOneRows];
  const int t = threadIdx.x, B = (int)p.B, L = (int)p.L, slots = B * L;
  const bool groups = p.aggregate == ACRL_AGG_GROUP;
  n[t] = live[t] = 0;
  __syncthreads();
  for (int j = t; j < slots; j += 1024)
    if (p.mask[j]) atomicAdd(&n[j / L], 1);
  __syncthreads();
  int g = -1;
  if (t < B) {
    if (groups) g = p.group_of_seq[t];
    if (in_no_group(p, t)) n[t] = g = -1;
    else if (groups && n[t] > 0) atomicAdd(&live[g], 1);
  }
  __syncthreads();
  double c[2] = {t < B ? (double)max(n[t], 0) : 0.0, (groups ? live[t] : n[t]) > 0 ? 1.0 : 0.0}, unused = 0.0;
  block_stats<2, 1024>(c, unused, sh2);
  if (t < B) share[t] = share_of(p, n[t], g >= 0 ? live[g] : 0, c);
  __syncthreads();
  double v[kPolicySums] = {};
  for (int j = t; j < slots; j += 1024) {
    float out = 0.0f;
    if (p.mask[j]) {
      const int i = j / L;
      const double a = share[i];
      double one[kPolicySums] = {};
      out = (float)(a * policy_slot(p, p.logp_new[j], p.logp_old[j], p.logp_ref ? p.logp_ref[j] : 0.0f,
                                    p.adv_per_token ? p.adv[j] : p.adv[i], p.weight ? p.weight[j] : 1.0f, one));
      if (a == a) {
#pragma unroll
        for (int k = 0; k < kPolicySums; ++k) v[k] += k < 2 ? a * one[k] : one[k];
      }
    }
    p.coef[j] = out;
  }
  unused = 0.0;
  block_stats<kPolicySums, 1024>(v, unused, sh);
  if (t == 0) policy_finish(p, v);
}

hipError_t launch_policy_loss(const acrl_policy_loss_desc& p, hipStream_t s) {
  const PolicyWs ws = policy_ws(p.workspace, p.B, p.L, p.n_groups);
  const int64_t units = units_of_response(p.B, p.L), n = p.B * units;
  if (n > 0 && one_policy(p.B, p.L, p.n_groups)) {
    hipLaunchKernelGGL(policy_one_kernel, dim3(1), dim3(1024), 0, s, p);
    return hipGetLastError();
  }
  if (n > 0) {
    int from = kShareNorm;
    if (p.aggregate != ACRL_AGG_CONSTANT) {
      const int per = kUnitThreads / 64;
      hipLaunchKernelGGL(policy_count_kernel, dim3((unsigned)((p.B + per - 1) / per)), dim3(kUnitThreads), 0, s, p, ws.n);
      // (a few workgroups look through the counts of all responses sooner than a launch of its own does; of many, 512
      // responses of 16384 slots, each would do so again: policy_main_kernel 38.7 us, 33.4 + 2.7 with the launch)
      from = p.B * p.L <= kManySlots && p.B <= kOneRows && p.n_groups <= kOneRows ? kShareOwn : kShareWs;
      if (from == kShareWs) hipLaunchKernelGGL(policy_share_kernel, dim3(1), dim3(1024), 0, s, p, ws);
    }
    const bool vec = p.L % kSlots == 0 && aligned(p.mask, 4) && aligned(p.logp_new, 16) && aligned(p.logp_old, 16) &&
                     aligned(p.logp_ref, 16) && aligned(p.weight, 16) && aligned(p.coef, 16) &&
                     (!p.adv_per_token || aligned(p.adv, 16));
    auto go = [&](auto turns, auto v) {
      hipLaunchKernelGGL((policy_main_kernel<decltype(turns)::value, decltype(v)::value>), dim3((unsigned)n),
                         dim3(kUnitThreads), 0, s, p, ws, units, from);
    };
    auto with = [&](auto turns) { vec ? go(turns, std::true_type{}) : go(turns, std::false_type{}); };
    if (unit_turns(p.B, p.L) == 1) with(std::integral_constant<int, 1>{});
    else with(std::integral_constant<int, 2>{});
  }
  hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(1024), 0, s, p, ws, n);
  return hipGetLastError();
}

// ------------------------------------------------------------------ preference loss
struct PrefRec {
  double x, each;  // x_i (mean_logp applied); d x_i / d logp_new of a valid slot
};
// Every response's workgroup looks through all pairs: 65536 responses of 65536 pairs take 2.9 ms, 2^20 of 2^20 would
// 1.1 s: from there on they are refused.
constexpr int64_t kMaxPairs = (int64_t)1 << 24, kMaxPairLooks = (int64_t)1 << 40;
constexpr int kPrefOne = 256;  // responses, and pairs, of a batch that one workgroup does
inline bool one_preference(int64_t B, int64_t L, int64_t P) {
  return B * L <= kOneSlots && B <= kPrefOne && P <= kPrefOne;
}
size_t pref_ws_bytes(int64_t B) { return align_up((size_t)B * sizeof(PrefRec), 256) + 256; }

// Workgroup size: 1024 threads from the second turn on while that leaves a few
// workgroups a CU (512 responses of up to 16384 slots 10.3 us, 14.9 with 256
// threads; 256 of 4096 3.6 / 4.2; 2048 of 2048 10.3 / 5.9).
inline int pref_threads(int64_t B, int64_t L) {
  if (L <= 64 * kSlots) return 64;
  return L > kRedThreads * kSlots && B <= 1024 ? 1024 : kRedThreads;
}

// x_i of each response, one workgroup per response.
template <int NT, bool VEC>
__global__ __launch_bounds__(NT) void pref_seq_kernel(acrl_preference_desc p, PrefRec* rec) {
  __shared__ BlockShared<2, NT> sh;
  const int64_t i = blockIdx.x;
  const int64_t base = i * p.L;
  double v[2] = {0, 0}, unused = 0.0;  // n, x
  for (int64_t j = first_slot<NT, VEC>(); j < p.L; j += NT * kSlots) {
    uint8_t m[kSlots];
    float ln[kSlots], lr[kSlots] = {};
    load_mask<NT, VEC>(p.mask, base, j, p.L, m);
    if (!(m[0] | m[1] | m[2] | m[3])) continue;
    load_slots<NT, VEC>(p.logp_new, base, j, p.L, ln);
    if (p.logp_ref) load_slots<NT, VEC>(p.logp_ref, base, j, p.L, lr);
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      if (!m[k]) continue;
      v[0] += 1.0;
      v[1] += (double)ln[k] - (double)lr[k];
    }
  }
  block_stats<2, NT>(v, unused, sh);
  if (threadIdx.x == 0) {
    const double each = p.mean_logp ? (v[0] > 0 ? 1.0 / v[0] : 0.0) : 1.0;
    rec[i] = PrefRec{v[1] * each, each};
  }
}

// The loss of pair `at` and u l'(h) beta / n_pairs; NaN for an index outside
// the batch.
__device__ __forceinline__ double pref_pair(const acrl_preference_desc& p, const PrefRec* rec, int64_t at, int32_t c,
                                            int32_t r, double& loss) {
  const double nan = __builtin_nan("");
  const double xc = c >= 0 && c < p.B ? rec[c].x : nan, xr = r >= 0 && r < p.B ? rec[r].x : nan;
  const double beta = p.beta, h = beta * (xc - xr) - (double)p.margin;
  double l, d;
  if (p.form == ACRL_PREF_SIGMOID) {
    const double e = p.label_smoothing, t = exp(-fabs(h)), soft = log1p(t);
    // sigmoid(h) and sigmoid(-h), each without cancellation
    const double big = 1.0 / (1.0 + t), small = t * big, up = h >= 0 ? big : small, down = h >= 0 ? small : big;
    l = (1.0 - e) * (soft + fmax(-h, 0.0)) + (e > 0 ? e * (soft + fmax(h, 0.0)) : 0.0);
    d = h == h ? e * up - (1.0 - e) * down : nan;
    if (!(h == h)) l = nan;  // (fmax drops a NaN)
  } else if (p.form == ACRL_PREF_HINGE) {
    l = h == h ? fmax(1.0 - h, 0.0) : nan;
    d = h == h ? (h < 1.0 ? -1.0 : 0.0) : nan;
  } else {
    const double z = (h - 0.5) / beta;
    l = z * z;
    d = 2.0 * z / beta;
  }
  const double u = p.pair_weight ? (double)p.pair_weight[at] : 1.0;
  loss = u * l;
  return u * d * beta / (double)p.n_pairs;
}

__device__ __forceinline__ void pref_rewards(const acrl_preference_desc& p, const PrefRec* rec, int64_t at, int32_t c,
                                             int32_t r) {
  if (!p.rewards) return;
  const float nan = __builtin_nanf("");
  p.rewards[at] = c >= 0 && c < p.B ? (float)((double)p.beta * rec[c].x) : nan;
  p.rewards[p.n_pairs + at] = r >= 0 && r < p.B ? (float)((double)p.beta * rec[r].x) : nan;
}

// coef of one response's slots: its pairs' slopes, then one value for every
// valid slot (512 responses of up to 16384 slots: 10.1 us, 4.1 TB/s;
// pref_seq_kernel 10.2 us, 4.4 TB/s).  The last workgroup sums the loss and writes
// the rewards.
template <bool VEC>
__global__ __launch_bounds__(kUnitThreads) void pref_coef_kernel(acrl_preference_desc p, const PrefRec* rec) {
  __shared__ BlockShared<1, kUnitThreads> sh;
  double v[1] = {0}, unused = 0.0;
  const int64_t i = blockIdx.x;
  for (int64_t at = threadIdx.x; at < p.n_pairs; at += kUnitThreads) {
    const int32_t c = p.chosen[at], r = p.rejected[at];
    double l;
    if (i == p.B) {
      pref_pair(p, rec, at, c, r, l);
      v[0] += l;
      pref_rewards(p, rec, at, c, r);
    } else if ((c == i) != (r == i)) {  // (a response against itself: its slopes cancel)
      const double g = pref_pair(p, rec, at, c, r, l);
      v[0] += c == i ? g : -g;
    }
  }
  block_stats<1, kUnitThreads>(v, unused, sh);
  if (i == p.B) {
    if (threadIdx.x == 0) p.loss[0] = p.n_pairs > 0 ? v[0] / (double)p.n_pairs : 0.0;
    return;
  }
  const float c = (float)(v[0] * rec[i].each);
  const int64_t base = i * p.L;
  if constexpr (VEC) {
#pragma unroll 4
    for (int64_t j = threadIdx.x * kSlots; j < p.L; j += kUnitThreads * kSlots) {
      uint8_t m[kSlots];
      load_mask<kUnitThreads, true>(p.mask, base, j, p.L, m);
      *reinterpret_cast<float4*>(p.coef + base + j) =
          make_float4(m[0] ? c : 0.0f, m[1] ? c : 0.0f, m[2] ? c : 0.0f, m[3] ? c : 0.0f);
    }
  } else {
    for (int64_t j = threadIdx.x; j < p.L; j += kUnitThreads) p.coef[base + j] = p.mask[base + j] ? c : 0.0f;
  }
}

// All of it in one workgroup: a wavefront a response for the sums, a thread a
// pair for the slopes, a thread a response for its coef (8 responses of 67
// slots 4.1 us; 6.9 by the two kernels).
__global__ __launch_bounds__(1024) void pref_one_kernel(acrl_preference_desc p) {
  __shared__ BlockShared<1, 1024> sh;
  __shared__ PrefRec rec[kPrefOne];
  __shared__ double slope[kPrefOne];
  __shared__ int32_t chosen[kPrefOne], rejected[kPrefOne];
  __shared__ float coef[kPrefOne];
  const int t = threadIdx.x, lane = t & 63, B = (int)p.B, L = (int)p.L, P = (int)p.n_pairs;
  for (int i = t >> 6; i < B; i += 16) {
    double n = 0, x = 0;
    for (int j = lane; j < L; j += 64)
      if (p.mask[i * L + j]) {
        n += 1.0;
        x += (double)p.logp_new[i * L + j] - (p.logp_ref ? (double)p.logp_ref[i * L + j] : 0.0);
      }
    n = lane_sum<64>(n);
    x = lane_sum<64>(x);
    const double each = p.mean_logp ? (n > 0 ? 1.0 / n : 0.0) : 1.0;
    if (lane == 0) rec[i] = PrefRec{x * each, each};
  }
  __syncthreads();
  double v[1] = {0}, unused = 0.0;
  if (t < P) {
    chosen[t] = p.chosen[t];
    rejected[t] = p.rejected[t];
    slope[t] = pref_pair(p, rec, t, chosen[t], rejected[t], v[0]);
    pref_rewards(p, rec, t, chosen[t], rejected[t]);
  }
  block_stats<1, 1024>(v, unused, sh);
  if (t == 0) p.loss[0] = P > 0 ? v[0] / (double)P : 0.0;
  if (t < B) {
    double c = 0.0;
    for (int k = 0; k < P; ++k) {
      const bool up = chosen[k] == t, down = rejected[k] == t;
      if (up != down) c += up ? slope[k] : -slope[k];
    }
    coef[t] = (float)(c * rec[t].each);
  }
  __syncthreads();
  for (int j = t; j < B * L; j += 1024) p.coef[j] = p.mask[j] ? coef[j / L] : 0.0f;
}

hipError_t launch_preference_loss(const acrl_preference_desc& p, hipStream_t s) {
  if (one_preference(p.B, p.L, p.n_pairs)) {
    hipLaunchKernelGGL(pref_one_kernel, dim3(1), dim3(1024), 0, s, p);
    return hipGetLastError();
  }
  PrefRec* rec = static_cast<PrefRec*>(p.workspace);
  if (p.B > 0) {
    const bool vec = p.L % kSlots == 0 && aligned(p.mask, 4) && aligned(p.logp_new, 16) && aligned(p.logp_ref, 16);
    launch_seq(pref_threads(p.B, p.L), vec, [&](auto nt, auto v) {
      constexpr int NT = decltype(nt)::value;
      hipLaunchKernelGGL((pref_seq_kernel<NT, decltype(v)::value>), dim3((unsigned)p.B), dim3(NT), 0, s, p, rec);
    });
  }
  const bool vec = p.L % kSlots == 0 && aligned(p.mask, 4) && aligned(p.coef, 16);
  if (vec) hipLaunchKernelGGL((pref_coef_kernel<true>), dim3((unsigned)p.B + 1), dim3(kUnitThreads), 0, s, p, (const PrefRec*)rec);
  else hipLaunchKernelGGL((pref_coef_kernel<false>), dim3((unsigned)p.B + 1), dim3(kUnitThreads), 0, s, p, (const PrefRec*)rec);
  return hipGetLastError();
}

bool finite(float v) { return v - v == 0.0f; }

}  // namespace
}  // namespace acrl

using acrl::set_error;

extern "C" {

acrl_status acrl_policy_loss_workspace_size(int64_t B, int64_t L, int64_t n_groups, size_t* bytes) {
  ACRL_REQUIRE(bytes, "bytes is NULL");
  ACRL_REQUIRE(B >= 0 && L >= 0 && n_groups >= 0, "B, L and n_groups must be >= 0");
  // a launch holds fewer than 2^32 threads
  ACRL_REQUIRE(B < acrl::kMaxResponses && L < INT32_MAX && n_groups < INT32_MAX, "B must be < 2^22, L and n_groups < 2^31 - 1");
  ACRL_REQUIRE(B * acrl::units_of_response(B, L) < 4 * acrl::kMaxResponses, "B ceil(L / 2048) must be < 2^24");
  *bytes = acrl::one_policy(B, L, n_groups) ? 0 : (size_t)acrl::policy_ws(nullptr, B, L, n_groups).bytes;
  return ACRL_OK;
}

acrl_status acrl_policy_loss(const acrl_policy_loss_desc* d, void* stream) {
  ACRL_REQUIRE(d, "desc is NULL");
  size_t need = 0;
  acrl_status st = acrl_policy_loss_workspace_size(d->B, d->L, d->n_groups, &need);
  if (st != ACRL_OK) return st;
  ACRL_REQUIRE(d->aggregate >= ACRL_AGG_GROUP && d->aggregate <= ACRL_AGG_CONSTANT, "aggregate %d unknown",
               d->aggregate);
  ACRL_REQUIRE(d->kl_estimator >= ACRL_KL_K1 && d->kl_estimator <= ACRL_KL_K3, "kl_estimator %d unknown",
               d->kl_estimator);
  ACRL_REQUIRE(d->eps_low >= 0.0f && d->eps_low < 1.0f, "eps_low must lie in [0, 1) (got %g)", (double)d->eps_low);
  ACRL_REQUIRE(d->eps_high >= 0.0f && d->eps_high < 1e30f, "eps_high must lie in [0, 1e30) (got %g)", (double)d->eps_high);
  ACRL_REQUIRE(d->dual_clip == 0.0f || (d->dual_clip > 1.0f && d->dual_clip < 1e30f),
               "dual_clip must be 0 or lie in (1, 1e30) (got %g)", (double)d->dual_clip);
  ACRL_REQUIRE(d->kl_coef >= 0.0f && d->kl_coef < 1e30f, "kl_coef must lie in [0, 1e30) (got %g)", (double)d->kl_coef);
  ACRL_REQUIRE(d->logp_ref || d->kl_coef == 0.0f || d->B == 0 || d->L == 0, "kl_coef needs logp_ref");
  if (d->aggregate == ACRL_AGG_CONSTANT)
    ACRL_REQUIRE(d->norm > 0.0f && acrl::finite(d->norm), "norm must be positive and finite (got %g)", (double)d->norm);
  ACRL_REQUIRE(d->loss, "loss is required");
  if (d->B > 0 && d->aggregate == ACRL_AGG_GROUP)
    ACRL_REQUIRE(d->n_groups > 0 && d->group_of_seq, "group_of_seq and n_groups > 0 are required");
  if (d->B > 0 && d->L > 0)
    ACRL_REQUIRE(d->mask && d->logp_new && d->logp_old && d->adv && d->coef,
                 "mask, logp_new, logp_old, adv and coef are required");
  if (need > 0 && (!d->workspace || d->workspace_bytes < need)) {
    set_error("acrl_policy_loss needs %zu workspace bytes, got %zu", need, d->workspace_bytes);
    return ACRL_ERR_WORKSPACE;
  }
  ACRL_REQUIRE(acrl::aligned16(d->workspace), "workspace must be 16-byte aligned");
  st = acrl::check_device();
  if (st != ACRL_OK) return st;
  return acrl::hip_status(acrl::launch_policy_loss(*d, (hipStream_t)stream), "acrl_policy_loss launch");
}

acrl_status acrl_preference_loss_workspace_size(int64_t B, int64_t L, int64_t n_pairs, size_t* bytes) {
  ACRL_REQUIRE(bytes, "bytes is NULL");
  ACRL_REQUIRE(B >= 0 && L >= 0 && n_pairs >= 0, "B, L and n_pairs must be >= 0");
  ACRL_REQUIRE(B < acrl::kMaxResponses && L < INT32_MAX && n_pairs < acrl::kMaxPairs, "B must be < 2^22, L < 2^31 - 1, n_pairs < 2^24");
  ACRL_REQUIRE(B * n_pairs < acrl::kMaxPairLooks, "B n_pairs must be < 2^40");
  *bytes = acrl::one_preference(B, L, n_pairs) ? 0 : acrl::pref_ws_bytes(B);
  return ACRL_OK;
}

acrl_status acrl_preference_loss(const acrl_preference_desc* d, void* stream) {
  ACRL_REQUIRE(d, "desc is NULL");
  size_t need = 0;
  acrl_status st = acrl_preference_loss_workspace_size(d->B, d->L, d->n_pairs, &need);
  if (st != ACRL_OK) return st;
  ACRL_REQUIRE(d->form >= ACRL_PREF_SIGMOID && d->form <= ACRL_PREF_SQUARED, "form %d unknown", d->form);
  ACRL_REQUIRE(d->mean_logp == 0 || d->mean_logp == 1, "mean_logp must be 0 or 1");
  ACRL_REQUIRE(d->beta > 0.0f && d->beta < 1e30f, "beta must lie in (0, 1e30) (got %g)", (double)d->beta);
  ACRL_REQUIRE(acrl::finite(d->margin), "margin must be finite");
  ACRL_REQUIRE(d->label_smoothing >= 0.0f && d->label_smoothing < 1.0f, "label_smoothing must lie in [0, 1) (got %g)",
               (double)d->label_smoothing);
  ACRL_REQUIRE(d->form == ACRL_PREF_SIGMOID || d->label_smoothing == 0.0f, "label_smoothing goes with SIGMOID only");
  ACRL_REQUIRE(d->loss, "loss is required");
  if (d->B > 0 && d->L > 0) ACRL_REQUIRE(d->mask && d->logp_new && d->coef, "mask, logp_new and coef are required");
  if (d->n_pairs > 0) ACRL_REQUIRE(d->chosen && d->rejected, "chosen and rejected are required");
  if (need > 0 && (!d->workspace || d->workspace_bytes < need)) {
    set_error("acrl_preference_loss needs %zu workspace bytes, got %zu", need, d->workspace_bytes);
    return ACRL_ERR_WORKSPACE;
  }
  ACRL_REQUIRE(acrl::aligned16(d->workspace), "workspace must be 16-byte aligned");
  st = acrl::check_device();
  if (st != ACRL_OK) return st;
  return acrl::hip_status(acrl::launch_preference_loss(*d, (hipStream_t)stream), "acrl_preference_loss launch");
}

}  // extern "C"
