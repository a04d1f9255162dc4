// echo_ops.h -- operators of a training step: what their entry points (echo_ops.cpp) need of
// a context (echo_host.cpp) and the launches of their kernels.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>
#include <functional>
#include <string>

#include "echo.h"

namespace echo {

// -- a context as the operators see it (defined in echo_host.cpp) ---------------------------
struct OpContext {
  int device, sms;
  cudaStream_t stream;
  long long wait_limit;  // bound of every device-side wait, in SM clock cycles
  int skip;              // failure injection for tests (-1: none)
  int64_t head_piece;    // scratch of a head's gradient for a piece of the vocabulary, at most
};
// Makes the context's device current; an echo_status.
int op_context(echo_ctx *c, OpContext *o);
// The same for an operator: ECHO_E_TIMEOUT where a kernel of an earlier call gave up.
int op_begin(echo_ctx *c, OpContext *o);
// Waits for the context's stream; ECHO_E_TIMEOUT as above.
int op_wait(echo_ctx *c);
int op_error(echo_ctx *c, int code, const std::string &msg);
int op_cuda_error(echo_ctx *c, cudaError_t e, const char *what);
// Memory of the context that lasts until a later call's, or as long as the context where a graph
// is captured: at least `bytes`, 256-byte aligned.
int op_scratch(echo_ctx *c, size_t bytes, void **p);
// Whether p is memory of the context's device.
bool op_device_memory(echo_ctx *c, const void *p);
// Word of the context in host memory that kernels set when a wait gives up.
int op_status(echo_ctx *c, int32_t **p);
// Runs a launch, between two events while the context is profiled and its stream not captured.
cudaError_t op_launch(echo_ctx *c, const char *name, const std::function<cudaError_t()> &launch);

// -- launches ------------------------------------------------------------------------------
// Runs a launch under a name: op_launch with its context (for calls of several kernels).
using OpTimer = std::function<cudaError_t(const char *, const std::function<cudaError_t()> &)>;

struct EmbedArgs {
  int64_t n, H, V, v0;      // tokens, row length, rows of the shard, its first id
  const void *ids;
  int id64;
  const void *table;
  void *out;
  int64_t table_stride, out_stride;
  int table_type, out_type;
  float scale;
};
cudaError_t launch_embed(const EmbedArgs &a, int sms, cudaStream_t st);

// Embedding gradient: the tokens of the shard sorted by row (stable), then the sums.
struct EmbedGradArgs {
  int64_t n, H, V, v0;
  const void *ids;
  int id64;
  const void *dy;
  void *dtable;
  int64_t dy_stride, dtable_stride;
  int dy_type, dtable_type, accumulate;
  float scale;
  // scratch: two (row, token) arrays of n entries each; the number of tokens of the shard; the
  // partial sums of rows that windows cut, [windows][2][H]
  uint32_t *key[2], *tok[2];
  int32_t *count;
  float *part;
  int window;               // sorted tokens a warp sums
};
int embed_grad_window(int64_t n, int64_t H, int sms);
cudaError_t launch_embed_sort(const EmbedGradArgs &a, cudaStream_t st);
// (and, unless it accumulates, zeros to the rows without tokens)
cudaError_t launch_embed_sum(const EmbedGradArgs &a, cudaStream_t st);
cudaError_t launch_embed_join(const EmbedGradArgs &a, cudaStream_t st);

struct NormArgs {
  int64_t rows, H;
  const void *x;
  void *y;
  const void *w, *b;
  float *mean, *rstd;
  int64_t x_stride, y_stride;
  int x_type, p_type;
  float eps;
};
cudaError_t launch_layer_norm(const NormArgs &a, int sms, cudaStream_t st);

struct NormGradArgs {
  int64_t rows, H;
  const void *dy, *x, *w;
  const float *mean, *rstd;
  void *dx, *dw, *db;
  int64_t dy_stride, x_stride, dx_stride;
  int x_type, p_type, accumulate;
  float *part;              // scratch: [parts][2][H] partial sums of dw and db, or null without them
  int parts;
};
// Partial sums that the call below writes (rows > 0).
int layer_norm_grad_parts(const NormGradArgs &a, int sms);
cudaError_t launch_layer_norm_grad(const NormGradArgs &a, int sms, const OpTimer &timed, cudaStream_t st);

// Orthogonalised update: m <= n are the smaller and the larger side, `tall` whether the
// matrices have n rows (the others are taken transposed).
struct OrthoArgs {
  int64_t batch, m, n;
  bool tall;
  const void *g;
  void *o;
  int64_t g_stride, g_batch_stride, o_stride, o_batch_stride;
  int type, steps;
  float a, b, c, eps, scale;
  void *scratch;
  int32_t *status;          // of op_status
  long long wait_limit;     // bound of every wait of the kernels, in SM clock cycles
  int skip;                 // failure injection for tests (ProductArgs)
};
size_t ortho_scratch_bytes(const OrthoArgs &a, int sms);
cudaError_t launch_orthogonalize(const OrthoArgs &a, int sms, const OpTimer &timed, cudaStream_t st);

// Losses of a head and their gradients (echo_ops_head.cu): a list of K targets a token, labels
// (K = 1, no logits) or a teacher's top logits.
struct HeadArgs {
  bool grad;
  int64_t n, H, V, v0;      // tokens, row length, rows of the shard, its first id
  const void *x, *w;
  int64_t x_stride, w_stride;
  int type;
  const void *ids;
  int id64, K;
  const void *logits;
  int logits_type;
  const float *teacher_lse;
  float scale, tau;
  float *loss, *lse, *part;                // forward; `part`: sum of q z over the shard's targets
  const float *dloss, *dlse, *lse_in;      // backward
  void *dx, *dw;
  int64_t dx_stride, dw_stride;
  int dw_type, accumulate;
  int64_t piece_bytes;      // of scratch for a piece of the vocabulary
  void *scratch;
  int32_t *status;          // of op_status
  long long wait_limit;     // bound of every wait of the kernels, in SM clock cycles
  int skip;                 // failure injection for tests
};
int64_t head_piece_bytes();
int head_most_targets();
size_t head_scratch_bytes(const HeadArgs &a, int sms);
cudaError_t launch_head(const HeadArgs &a, int sms, const OpTimer &timed, cudaStream_t st);

// Rotary positions of up to two arrays [batch][tokens][heads][dim] (strides in elements).
constexpr int kRotaryPairs = 256;
struct RotaryArgs {
  int64_t batch, tokens, heads[2];
  const void *x[2];
  void *out[2];
  int64_t x_batch[2], x_token[2], x_head[2], out_batch[2], out_token[2], out_head[2];
  const void *positions;
  int64_t positions_batch;
  int id64, dim, rot, type, interleaved;
  bool back;                // the turn back
  float scale;
  uint64_t turns[kRotaryPairs];  // of a position, times 2^64
};
uint64_t rotary_turns(double frequency);
cudaError_t launch_rotary(const RotaryArgs &a, int sms, cudaStream_t st);

}  // namespace echo
