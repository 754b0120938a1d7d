/*
 * Host-side driver of the argument validation of the block-scaled FP8
 * operators and the losses, and of the reduce's and the surrogate's calls that
 * tests/host_validation.c leaves out, built with AddressSanitizer on the host
 * code (tests/test_host_asan_operators.py).  Every call below is out of contract
 * (or a size query), so it returns before any HIP call: no device is needed
 * and none is touched.  Exit status = number of unexpected results.
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "acrl.h"

static int failures = 0;

static void expect(const char* what, acrl_status got, acrl_status want) {
  if (got != want) {
    printf("FAIL %s: status %d, expected %d (%s)\n", what, got, want, acrl_last_error());
    ++failures;
  }
}

static unsigned char buf[1 << 16] __attribute__((aligned(256)));
static void* const p = buf;

static void quantize_blocks(void) {
  size_t nb = 7;
  for (int s = ACRL_SCALE_ROW128; s <= ACRL_SCALE_BLOCK128; ++s) {
    expect("blocks ws", acrl_quantize_workspace_size(4, 64, s, &nb), ACRL_OK);
    if (nb != 0) ++failures;
    expect("blocks cols", acrl_quantize_fp8(p, 4, 33, 64, s, 0, p, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks rows", acrl_quantize_fp8(p, -1, 64, 64, s, 0, p, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks ld", acrl_quantize_fp8(p, 4, 64, 68, s, 0, p, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks rounding", acrl_quantize_fp8(p, 4, 64, 64, s, 7, p, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks scales", acrl_quantize_fp8(p, 4, 64, 64, s, 0, p, NULL, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks x", acrl_quantize_fp8(NULL, 4, 64, 64, s, 0, p, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    expect("blocks misaligned", acrl_quantize_fp8(p, 4, 64, 64, s, 0, buf + 8, p, NULL, 0, NULL), ACRL_ERR_INVALID_ARG);
    /* the scorers know the first three scalings only */
    expect("blocks score", acrl_score_workspace_size(4, 256, 1000, s, &nb), ACRL_ERR_INVALID_ARG);
    expect("blocks packed", acrl_packed_weights_size(1000, 256, s, &nb), ACRL_ERR_INVALID_ARG);
  }
  expect("blocks scaling", acrl_quantize_workspace_size(4, 64, ACRL_SCALE_BLOCK128 + 1, &nb), ACRL_ERR_INVALID_ARG);
}

static acrl_matmul_desc matmul(void) {
  acrl_matmul_desc d;
  memset(&d, 0, sizeof d);
  d.M = 4; d.N = 64; d.K = 256; d.xq = p; d.x_scales = (float*)p; d.wq = p; d.w_scales = (float*)p; d.y = p; d.ldy = 64;
  return d;
}

static void products(void) {
  acrl_matmul_desc d;
  expect("matmul null", acrl_matmul_fp8(NULL, NULL), ACRL_ERR_INVALID_ARG);
  memset(&d, 0, sizeof d);
  expect("matmul zero", acrl_matmul_fp8(&d, NULL), ACRL_ERR_INVALID_ARG);
#define BAD(change) \
  do { d = matmul(); change; expect("matmul " #change, acrl_matmul_fp8(&d, NULL), ACRL_ERR_INVALID_ARG); } while (0)
  BAD(d.M = -1); BAD(d.M = (int64_t)1 << 26); BAD(d.M = INT64_MAX); BAD(d.N = 0); BAD(d.N = INT64_MIN);
  BAD(d.N = d.ldy = (int64_t)1 << 26); BAD(d.K = 0); BAD(d.K = 100); BAD(d.K = ((int64_t)1 << 22) + 32);
  BAD(d.K = INT64_MIN); BAD(d.ldy = 63); BAD(d.y_type = 2); BAD(d.y_type = -1); BAD(d.xq = NULL); BAD(d.x_scales = NULL);
  BAD(d.wq = NULL); BAD(d.w_scales = NULL); BAD(d.y = NULL); BAD(d.xq = buf + 8); BAD(d.wq = buf + 4); BAD(d.y = buf + 2);
  BAD(d.x_scales = (const float*)(buf + 2)); BAD(d.w_scales = (const float*)(buf + 1));
  BAD((d.M = (int64_t)1 << 25, d.N = d.ldy = (int64_t)1 << 20));
#undef BAD
}

static acrl_policy_loss_desc policy(void) {
  acrl_policy_loss_desc d;
  memset(&d, 0, sizeof d);
  d.B = 2; d.L = 4096; d.n_groups = 1; d.mask = p; d.group_of_seq = (int32_t*)p; d.logp_new = (float*)p;
  d.logp_old = (float*)p; d.logp_ref = (float*)p; d.adv = (float*)p; d.eps_low = 0.2f; d.eps_high = 0.2f;
  d.kl_coef = 0.1f; d.kl_estimator = ACRL_KL_K3; d.coef = (float*)p; d.loss = (double*)p; d.workspace = p;
  d.workspace_bytes = sizeof buf;
  return d;
}

static void linears(void) {
  acrl_linear_desc d;
  size_t sz[4] = {0};
  acrl_abi_decode_struct_sizes(&sz[0], &sz[1], &sz[2], &sz[3]);
  acrl_abi_decode_struct_sizes(NULL, NULL, NULL, NULL);
  if (sz[0] != sizeof d || sz[1] != sizeof(acrl_moe_desc) || sz[2] != sizeof(acrl_beam_desc) ||
      sz[3] != sizeof(acrl_reorder_desc))
    ++failures;
  expect("linear null", acrl_linear_fp8(NULL, NULL), ACRL_ERR_INVALID_ARG);
#define BAD_LINEAR(change)                                                                      \
  do {                                                                                          \
    memset(&d, 0, sizeof d);                                                                    \
    d.product = matmul(); d.bias = p; d.residual = buf + 4096; d.ldr = 64;                      \
    change;                                                                                     \
    expect("linear " #change, acrl_linear_fp8(&d, NULL), ACRL_ERR_INVALID_ARG);                 \
  } while (0)
  BAD_LINEAR(d.product.K = 100);
  BAD_LINEAR(d.product.y = NULL);
  BAD_LINEAR(d.activation = ACRL_ACT_GELU_TANH + 1);
  BAD_LINEAR(d.activation = -1);
  BAD_LINEAR(d.bias_type = 2);
  BAD_LINEAR(d.bias = buf + 8);
  BAD_LINEAR(d.residual_type = -1);
  BAD_LINEAR(d.residual = buf + 4100);
  BAD_LINEAR(d.ldr = 63);
  BAD_LINEAR(d.ldr = (int64_t)1 << 34);
  BAD_LINEAR(d.product.ldy = (int64_t)1 << 34);
  BAD_LINEAR(d.residual = buf + 64);                           /* inside y's rows */
  BAD_LINEAR(d.residual = buf + 128);                          /* y's second row */
  BAD_LINEAR(d.residual = p; d.ldr = 128);                     /* y with other rows */
  BAD_LINEAR(d.residual = p; d.residual_type = ACRL_OUT_F32);  /* y as another type */
}

static void experts(void) {
  acrl_moe_desc d;
  size_t nb = 0;
  expect("moe ws", acrl_moe_workspace_size(4, 64, 8, 2, 32, &nb), ACRL_OK);
  if (nb < 4 * 2 * 64 * 4) ++failures;
  expect("moe ws none", acrl_moe_workspace_size(0, 64, 8, 2, 32, &nb), ACRL_OK);
  if (nb != 0) ++failures;
  expect("moe ws null", acrl_moe_workspace_size(4, 64, 8, 2, 32, NULL), ACRL_ERR_INVALID_ARG);
  expect("moe ws T", acrl_moe_workspace_size(129, 64, 8, 2, 32, &nb), ACRL_ERR_INVALID_ARG);
  expect("moe ws d", acrl_moe_workspace_size(4, 65568, 8, 2, 32, &nb), ACRL_ERR_INVALID_ARG);
  expect("moe ws E", acrl_moe_workspace_size(4, 64, 513, 2, 32, &nb), ACRL_ERR_INVALID_ARG);
  expect("moe ws k", acrl_moe_workspace_size(4, 64, 8, 9, 32, &nb), ACRL_ERR_INVALID_ARG);
  expect("moe ws F", acrl_moe_workspace_size(4, 64, 8, 2, 48, &nb), ACRL_ERR_INVALID_ARG);
  expect("moe null", acrl_moe_fp8(NULL, NULL), ACRL_ERR_INVALID_ARG);
#define MOE(change, status)                                                                      \
  do {                                                                                           \
    memset(&d, 0, sizeof d);                                                                     \
    d.T = 4; d.d = 64; d.E = 8; d.top_k = 2; d.F = 32; d.x = p; d.ldx = 64; d.router = p;        \
    d.w_in = p; d.s_in = (float*)p; d.w_out = p; d.s_out = (float*)p; d.y = p; d.ldy = 64;       \
    d.residual = buf + 4096; d.ldr = 64; d.ids = (int32_t*)p; d.weights = (float*)p;             \
    d.scale = 1.0f; d.workspace = p; d.workspace_bytes = 1 << 30;                                \
    change;                                                                                      \
    expect("moe " #change, acrl_moe_fp8(&d, NULL), status);                                      \
  } while (0)
#define BAD_MOE(change) MOE(change, ACRL_ERR_INVALID_ARG)
  BAD_MOE(d.T = -1);
  BAD_MOE(d.T = 129);
  BAD_MOE(d.d = 48);
  BAD_MOE(d.top_k = 17; d.E = 32);
  BAD_MOE(d.score = 2);
  BAD_MOE(d.activation = 5);
  BAD_MOE(d.y_type = 2);
  BAD_MOE(d.scale = (float)NAN);
  BAD_MOE(d.ldx = 60);
  BAD_MOE(d.ldx = 68);
  BAD_MOE(d.ldy = 63);
  BAD_MOE(d.ldr = (int64_t)1 << 40);
  BAD_MOE(d.x = NULL);
  BAD_MOE(d.w_in = NULL);
  BAD_MOE(d.s_out = NULL);
  BAD_MOE(d.ids = NULL);
  BAD_MOE(d.weights = NULL);
  BAD_MOE(d.y = NULL);
  BAD_MOE(d.w_out = buf + 8);
  BAD_MOE(d.x = buf + 8);
  BAD_MOE(d.router = buf + 2);
  BAD_MOE(d.residual = buf + 64);
  BAD_MOE(d.residual_type = 7);
  BAD_MOE(d.workspace = buf + 8);
  MOE(d.workspace = NULL, ACRL_ERR_WORKSPACE);
  MOE(d.workspace_bytes = 64, ACRL_ERR_WORKSPACE);
}

static void beams(void) {
  acrl_beam_desc d;
  acrl_reorder_desc r;
  size_t nb = 0;
  expect("beam ws", acrl_beam_workspace_size(2, 3, 1000, 4, &nb), ACRL_OK);
  if (nb < 6 * 4 * 8) ++failures;
  expect("beam ws null", acrl_beam_workspace_size(2, 3, 1000, 4, NULL), ACRL_ERR_INVALID_ARG);
  expect("beam ws K", acrl_beam_workspace_size(2, 65, 1000, 4, &nb), ACRL_ERR_INVALID_ARG);
  expect("beam ws BK", acrl_beam_workspace_size(1 << 20, 4, 1000, 4, &nb), ACRL_ERR_INVALID_ARG);
  expect("beam ws n", acrl_beam_workspace_size(2, 2, 3, 7, &nb), ACRL_ERR_INVALID_ARG);
  expect("beam null", acrl_beam_step(NULL, NULL), ACRL_ERR_INVALID_ARG);
#define BEAM(change, status)                                                                     \
  do {                                                                                           \
    memset(&d, 0, sizeof d);                                                                     \
    d.B = 2; d.K = 3; d.V = 1000; d.n_out = 4; d.logits = p; d.ldl = 1000; d.scores = (float*)p; \
    d.finished = p; d.eos_id = 5; d.inv_temperature = 1.0f; d.ids = (int32_t*)p;                 \
    d.parents = (int32_t*)p; d.out_scores = (float*)p; d.workspace = p;                          \
    d.workspace_bytes = 1 << 30;                                                                 \
    change;                                                                                      \
    expect("beam " #change, acrl_beam_step(&d, NULL), status);                                   \
  } while (0)
#define BAD_BEAM(change) BEAM(change, ACRL_ERR_INVALID_ARG)
  BAD_BEAM(d.B = -1);
  BAD_BEAM(d.V = (int64_t)1 << 30; d.ldl = d.V);
  BAD_BEAM(d.n_out = 65);
  BAD_BEAM(d.ldl = 999);
  BAD_BEAM(d.logits_type = 2);
  BAD_BEAM(d.eos_id = -1);
  BAD_BEAM(d.eos_id = 1000);
  BAD_BEAM(d.inv_temperature = 0.0f);
  BAD_BEAM(d.inv_temperature = (float)NAN);
  BAD_BEAM(d.logits = NULL);
  BAD_BEAM(d.logits = buf + 1);
  BAD_BEAM(d.parents = NULL);
  BAD_BEAM(d.scores = (float*)(buf + 2));
  BAD_BEAM(d.workspace = buf + 8);
  BEAM(d.workspace = NULL, ACRL_ERR_WORKSPACE);
  BEAM(d.workspace_bytes = 8, ACRL_ERR_WORKSPACE);
  expect("reorder null", acrl_beam_reorder(NULL, NULL), ACRL_ERR_INVALID_ARG);
#define BAD_REORDER(change)                                                                      \
  do {                                                                                           \
    memset(&r, 0, sizeof r);                                                                     \
    r.outer = 2; r.B = 2; r.K = 3; r.n_out = 3; r.row_bytes = 64; r.src = p; r.src_outer = 384;  \
    r.src_seq = 192; r.src_beam = 64; r.dst = buf + 4096; r.dst_outer = 384; r.dst_seq = 192;    \
    r.dst_beam = 64; r.parents = (int32_t*)p;                                                    \
    change;                                                                                      \
    expect("reorder " #change, acrl_beam_reorder(&r, NULL), ACRL_ERR_INVALID_ARG);               \
  } while (0)
  BAD_REORDER(r.K = 0);
  BAD_REORDER(r.K = 65);
  BAD_REORDER(r.n_out = 65);
  BAD_REORDER(r.B = -1);
  BAD_REORDER(r.outer = (1 << 20) + 1);
  BAD_REORDER(r.row_bytes = -1);
  BAD_REORDER(r.row_bytes = (int64_t)1 << 40);
  BAD_REORDER(r.src_beam = -64);
  BAD_REORDER(r.dst_outer = (int64_t)1 << 42);
  BAD_REORDER(r.src = NULL);
  BAD_REORDER(r.parents = NULL);
  BAD_REORDER(r.parents = (int32_t*)(buf + 2));
  BAD_REORDER(r.dst_beam = 63);
  BAD_REORDER(r.dst_seq = 63);
  BAD_REORDER(r.dst = buf + 64);
  BAD_REORDER(r.dst = p; r.dst_beam = 128);
  BAD_REORDER(r.dst = p; r.n_out = 2);
  BAD_REORDER(r.row_bytes = (int64_t)1 << 36; r.dst_beam = (int64_t)1 << 37; r.dst_seq = (int64_t)1 << 39;
              r.dst_outer = (int64_t)1 << 40; r.dst = (void*)((int64_t)1 << 44));
}

static void policy_losses(void) {
  acrl_policy_loss_desc d;
  size_t nb = 0;
  expect("policy null", acrl_policy_loss(NULL, NULL), ACRL_ERR_INVALID_ARG);
  memset(&d, 0, sizeof d);
  expect("policy zero", acrl_policy_loss(&d, NULL), ACRL_ERR_INVALID_ARG);
#define BAD(change) \
  do { d = policy(); change; expect("policy " #change, acrl_policy_loss(&d, NULL), ACRL_ERR_INVALID_ARG); } while (0)
  BAD(d.B = -1); BAD(d.L = -1); BAD(d.n_groups = -1); BAD(d.n_groups = 0); BAD(d.group_of_seq = NULL); BAD(d.mask = NULL);
  BAD(d.logp_new = NULL); BAD(d.logp_old = NULL); BAD(d.adv = NULL); BAD(d.coef = NULL); BAD(d.loss = NULL);
  BAD(d.logp_ref = NULL); BAD(d.eps_low = 1.0f); BAD(d.eps_low = -0.1f); BAD(d.eps_low = NAN); BAD(d.eps_high = -0.1f);
  BAD(d.eps_high = INFINITY); BAD(d.dual_clip = 1.0f); BAD(d.dual_clip = NAN); BAD(d.kl_coef = -1.0f);
  BAD(d.kl_coef = INFINITY); BAD(d.kl_estimator = 3); BAD(d.kl_estimator = -1); BAD(d.aggregate = 4); BAD(d.aggregate = -1);
  BAD((d.aggregate = ACRL_AGG_CONSTANT, d.norm = 0.0f)); BAD((d.aggregate = ACRL_AGG_CONSTANT, d.norm = INFINITY));
  BAD(d.B = (int64_t)1 << 22); BAD(d.B = INT64_MAX); BAD(d.L = INT64_MAX); BAD(d.n_groups = INT64_MAX);
  BAD((d.B = (int64_t)1 << 21, d.L = (int64_t)1 << 20)); BAD(d.workspace = buf + 8);
#undef BAD
  d = policy(); d.workspace = NULL;
  expect("policy workspace", acrl_policy_loss(&d, NULL), ACRL_ERR_WORKSPACE);
  d = policy(); d.workspace_bytes = 16;
  expect("policy workspace bytes", acrl_policy_loss(&d, NULL), ACRL_ERR_WORKSPACE);
  expect("policy ws", acrl_policy_loss_workspace_size(64, 4096, 8, &nb), ACRL_OK);
  expect("policy ws most", acrl_policy_loss_workspace_size(((int64_t)1 << 22) - 1, 4096, INT32_MAX - 1, &nb), ACRL_OK);
  expect("policy ws null", acrl_policy_loss_workspace_size(64, 4096, 8, NULL), ACRL_ERR_INVALID_ARG);
  expect("policy ws B", acrl_policy_loss_workspace_size(INT64_MIN, 4096, 8, &nb), ACRL_ERR_INVALID_ARG);
}

static acrl_preference_desc preference(void) {
  acrl_preference_desc d;
  memset(&d, 0, sizeof d);
  d.B = 2; d.L = 4096; d.n_pairs = 1; d.mask = p; d.logp_new = (float*)p; d.logp_ref = (float*)p; d.chosen = (int32_t*)p;
  d.rejected = (int32_t*)p; d.beta = 0.1f; d.coef = (float*)p; d.loss = (double*)p; d.workspace = p;
  d.workspace_bytes = sizeof buf;
  return d;
}

static void preference_losses(void) {
  acrl_preference_desc d;
  size_t nb = 0;
  expect("preference null", acrl_preference_loss(NULL, NULL), ACRL_ERR_INVALID_ARG);
  memset(&d, 0, sizeof d);
  expect("preference zero", acrl_preference_loss(&d, NULL), ACRL_ERR_INVALID_ARG);
#define BAD(change)                                                                                  \
  do { d = preference(); change; expect("preference " #change, acrl_preference_loss(&d, NULL),       \
                                        ACRL_ERR_INVALID_ARG); } while (0)
  BAD(d.B = -1); BAD(d.L = -1); BAD(d.n_pairs = -1); BAD(d.mask = NULL); BAD(d.logp_new = NULL); BAD(d.coef = NULL);
  BAD(d.loss = NULL); BAD(d.chosen = NULL); BAD(d.rejected = NULL); BAD(d.beta = 0.0f); BAD(d.beta = NAN);
  BAD(d.beta = INFINITY); BAD(d.margin = NAN); BAD(d.margin = INFINITY); BAD(d.label_smoothing = 1.0f);
  BAD(d.label_smoothing = NAN); BAD((d.form = ACRL_PREF_HINGE, d.label_smoothing = 0.1f)); BAD(d.form = 3); BAD(d.form = -1);
  BAD(d.mean_logp = 2); BAD(d.B = (int64_t)1 << 22); BAD(d.L = INT64_MAX); BAD(d.n_pairs = INT64_MAX);
  BAD(d.n_pairs = (int64_t)1 << 24); BAD((d.B = (int64_t)1 << 20, d.n_pairs = (int64_t)1 << 20)); BAD(d.workspace = buf + 8);
#undef BAD
  d = preference(); d.workspace = NULL;
  expect("preference workspace", acrl_preference_loss(&d, NULL), ACRL_ERR_WORKSPACE);
  d = preference(); d.workspace_bytes = 16;
  expect("preference workspace bytes", acrl_preference_loss(&d, NULL), ACRL_ERR_WORKSPACE);
  expect("preference ws", acrl_preference_loss_workspace_size(64, 4096, 8, &nb), ACRL_OK);
  expect("preference ws null", acrl_preference_loss_workspace_size(64, 4096, 8, NULL), ACRL_ERR_INVALID_ARG);
  expect("preference ws B", acrl_preference_loss_workspace_size(INT64_MIN, 4096, 8, &nb), ACRL_ERR_INVALID_ARG);
}

static void reduces(void) {
  acrl_reduce_desc d;
  size_t nb = 0;
  expect("reduce ws", acrl_reduce_workspace_size(2, 4, 1, &nb), ACRL_OK);
  expect("reduce ws null", acrl_reduce_workspace_size(2, 4, 1, NULL), ACRL_ERR_INVALID_ARG);
  expect("reduce ws B", acrl_reduce_workspace_size(-1, 4, 1, &nb), ACRL_ERR_INVALID_ARG);
  expect("surrogate ws", acrl_surrogate_workspace_size(2, 1, &nb), ACRL_OK);
  expect("surrogate ws null", acrl_surrogate_workspace_size(2, 1, NULL), ACRL_ERR_INVALID_ARG);
  expect("surrogate ws groups", acrl_surrogate_workspace_size(2, -1, &nb), ACRL_ERR_INVALID_ARG);
  expect("reduce noalloc null", acrl_discrepancy_reduce_noalloc(NULL, NULL), ACRL_ERR_INVALID_ARG);
  memset(&d, 0, sizeof d);
  d.B = -1; d.stats = (double*)p;
  expect("reduce noalloc B", acrl_discrepancy_reduce_noalloc(&d, NULL), ACRL_ERR_INVALID_ARG);
  d.B = 1 << 20; d.L = 4; d.n_groups = 1; d.logp_pi = (float*)p; d.logp_mu = (float*)p; d.mask = p;
  d.group_of_seq = (const int32_t*)p; d.seq_mean_d = (float*)p; d.group_y = (float*)p;
  expect("reduce noalloc size", acrl_discrepancy_reduce_noalloc(&d, NULL), ACRL_ERR_WORKSPACE);
}

int main(void) {
  size_t sz[3] = {0};
  acrl_abi_operator_struct_sizes(&sz[0], &sz[1], &sz[2]);
  acrl_abi_operator_struct_sizes(NULL, NULL, NULL);
  if (sz[0] != sizeof(acrl_matmul_desc) || sz[1] != sizeof(acrl_policy_loss_desc) || sz[2] != sizeof(acrl_preference_desc))
    ++failures;
  quantize_blocks();
  products();
  linears();
  experts();
  beams();
  policy_losses();
  preference_losses();
  reduces();
  printf("%d unexpected results\n", failures);
  return failures;
}
