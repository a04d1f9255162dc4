// echo_ops.cpp -- entry points of the operators of a training step (include/echo.h): argument
// checks, scratch memory, launches.
#include "echo_ops.h"

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <exception>
#include <utility>

namespace {

using echo::OpContext;

constexpr int64_t kMaxHidden = (int64_t)1 << 30;

bool known_type(int t) { return t == ECHO_F32 || t == ECHO_BF16 || t == ECHO_F16; }
int type_size(int t) { return t == ECHO_F32 ? 4 : 2; }

// Collects what is wrong with a call's arguments: the first complaint.
struct Checks {
  echo_ctx *c;
  int rc = ECHO_OK;
  int fail(int code, const char *msg) { return rc ? rc : rc = echo::op_error(c, code, msg); }
  void need(bool ok, const char *msg) {
    if (!ok) fail(ECHO_E_INVALID_ARG, msg);
  }
  void supported(bool ok, const char *msg) {
    if (!ok) fail(ECHO_E_UNSUPPORTED, msg);
  }
  void array(const void *p, int size, const char *what) {
    if (rc) return;
    const std::string name(what);
    if (!p) {
      rc = echo::op_error(c, ECHO_E_INVALID_ARG, name + " is NULL");
    } else if (reinterpret_cast<uintptr_t>(p) % size) {
      rc = echo::op_error(c, ECHO_E_INVALID_ARG, name + " is not at a multiple of its element size");
    } else if (!echo::op_device_memory(c, p)) {
      rc = echo::op_error(c, ECHO_E_INVALID_ARG, name + " is not memory of the context's device");
    }
  }
  // rows of `length` elements whose last one has to lie within the address space
  void matrix(const void *p, int type, int64_t rows, int64_t length, int64_t stride, bool out, const char *what) {
    need(known_type(type), "unknown element type");
    if (rc) return;
    array(p, type_size(type), what);
    need(stride >= 0 && (!out || rows <= 1 || stride >= length), "a stride is negative, or an output's is less than its row");
    need(rows <= 1 || stride <= ((int64_t)1 << 58) / (rows - 1), "a matrix does not fit the address space");
  }
};

// Runs an entry point: no C++ exception leaves it.
template <typename F>
int guarded(F &&body) {
  try {
    return body();
  } catch (const std::exception &) {
    return ECHO_E_OOM;
  }
}
// The entry point of an operator.
template <typename F>
int entry(echo_ctx *c, const void *d, F &&body) {
  return guarded([&]() -> int {
    OpContext o;
    if (const int rc = echo::op_begin(c, &o)) return rc;
    if (!d) return echo::op_error(c, ECHO_E_INVALID_ARG, "an argument is NULL");
    return body(o);
  });
}

#define RUN(call, name)                                                                       \
  do {                                                                                        \
    const cudaError_t _e = echo::op_launch(c, name, [&] { return call; });                    \
    if (_e != cudaSuccess) return echo::op_cuda_error(c, _e, name);                           \
  } while (0)

echo::OpTimer timer(echo_ctx *c) {
  return [c](const char *name, const std::function<cudaError_t()> &f) { return echo::op_launch(c, name, f); };
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// -- losses of a head ----------------------------------------------------------------------------
template <typename D>
echo::HeadArgs head_of(const OpContext &o, const D &d) {
  echo::HeadArgs a{};
  a.n = d.n_tokens, a.H = d.hidden, a.V = d.vocab_rows, a.v0 = d.vocab_start;
  a.x = d.x, a.w = d.weight, a.x_stride = d.x_stride, a.w_stride = d.weight_stride, a.type = d.type;
  a.id64 = d.id_bits == 64 ? 1 : d.id_bits == 32 ? 0 : -1;
  a.scale = d.scale;
  a.wait_limit = o.wait_limit, a.skip = o.skip, a.piece_bytes = o.head_piece;
  return a;
}

template <typename D>
int teacher_of(Checks &k, echo::HeadArgs &a, const D &d) {
  a.ids = d.ids, a.logits = d.logits, a.logits_type = d.logits_type, a.teacher_lse = d.teacher_lse, a.tau = d.temperature;
  k.need(d.n_top >= 1, "no targets");
  k.supported(d.n_top <= echo::head_most_targets(), "more than 256 targets a token");
  k.need(std::isfinite(d.temperature) && d.temperature > 0.f, "the temperature is not positive and finite");
  k.need(known_type(d.logits_type), "unknown element type");
  a.K = k.rc ? 1 : (int)d.n_top;
  if (!k.rc && a.n > 0) {
    k.array(d.logits, type_size(d.logits_type), "logits");
    if (d.teacher_lse) k.array(d.teacher_lse, 4, "teacher_lse");
  }
  return k.rc;
}

// What all of them ask for.
void check_head(Checks &k, const echo::HeadArgs &a) {
  k.need(a.n >= 0 && a.V >= 0 && a.v0 >= 0 && a.H >= 1, "negative sizes, or no elements in a row");
  k.supported(a.H <= (int64_t)1 << 24, "rows of more than 2^24 elements");
  k.supported(a.n <= (int64_t)1 << 30 && a.V <= (int64_t)1 << 30, "more than 2^30 tokens or rows");
  k.need(a.id64 >= 0, "id_bits is neither 32 nor 64");
  k.need(known_type(a.type), "unknown element type");
  k.need(std::isfinite(a.scale), "the scale is not finite");
  if (k.rc || a.n == 0) return;
  k.matrix(a.x, a.type, a.n, a.H, a.x_stride, false, "x");
  if (a.V) k.matrix(a.w, a.type, a.V, a.H, a.w_stride, false, "weight");
  k.array(a.ids, a.id64 ? 8 : 4, a.logits ? "ids" : "labels");
}

int head_run(echo_ctx *c, const OpContext &o, echo::HeadArgs &a, const char *name) {
  if (const int rc = echo::op_status(c, &a.status)) return rc;
  if (const int rc = echo::op_scratch(c, echo::head_scratch_bytes(a, o.sms), &a.scratch)) return rc;
  const cudaError_t e = echo::launch_head(a, o.sms, timer(c), o.stream);
  if (e != cudaSuccess) return echo::op_cuda_error(c, e, name);
  return (int)ECHO_OK;
}

int head_forward(echo_ctx *c, const OpContext &o, echo::HeadArgs &a, const char *part) {
  Checks k{c};
  check_head(k, a);
  if (k.rc || a.n == 0) return k.rc;
  if (a.loss) k.array(a.loss, 4, "loss");
  if (a.lse) k.array(a.lse, 4, "lse");
  if (a.part) k.array(a.part, 4, part);
  if (k.rc) return k.rc;
  return head_run(c, o, a, a.logits ? "distill" : "cross_entropy");
}

template <typename D>
int head_backward(echo_ctx *c, const OpContext &o, echo::HeadArgs &a, const D &d) {
  Checks k{c};
  a.grad = true;
  a.dloss = d.dloss, a.dlse = d.dlse, a.lse_in = d.lse;
  a.dx = a.n ? d.dx : nullptr, a.dw = a.V ? d.dweight : nullptr;  // (empty ones are not touched)
  a.dx_stride = d.dx_stride, a.dw_stride = d.dweight_stride, a.dw_type = d.dweight_type, a.accumulate = d.accumulate != 0;
  check_head(k, a);
  k.need(known_type(d.dweight_type), "unknown element type");
  if (k.rc) return k.rc;
  if (a.n) {
    k.array(a.dloss, 4, "dloss");
    if (a.dlse) k.array(a.dlse, 4, "dlse");
    k.array(a.lse_in, 4, "lse");
  }
  if (a.dx) k.matrix(a.dx, a.type, a.n, a.H, a.dx_stride, true, "dx");
  if (a.dw) k.matrix(a.dw, a.dw_type, a.V, a.H, a.dw_stride, true, "dweight");
  if (k.rc) return k.rc;
  const char *name = a.logits ? "distill_grad" : "cross_entropy_grad";
  auto zeros = [&](void *p, int type, int64_t rows, int64_t stride) {
    const size_t size = type_size(type);
    const cudaError_t e = rows <= 1 || stride == a.H ? cudaMemsetAsync(p, 0, (size_t)rows * a.H * size, o.stream)
                                                     : cudaMemset2DAsync(p, (size_t)stride * size, 0, (size_t)a.H * size, (size_t)rows, o.stream);
    return e == cudaSuccess ? (int)ECHO_OK : echo::op_cuda_error(c, e, name);
  };
  if (a.n == 0) return a.dw && !a.accumulate ? zeros(a.dw, a.dw_type, a.V, a.dw_stride) : (int)ECHO_OK;
  if (a.V == 0) return a.dx ? zeros(a.dx, a.type, a.n, a.dx_stride) : (int)ECHO_OK;
  if (!a.dx && !a.dw) return (int)ECHO_OK;
  return head_run(c, o, a, name);
}

// -- rotary positions ------------------------------------------------------------------------------
int rotary(echo_ctx *c, const echo_rotary_desc *d, bool back, const char *name) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->n_batch >= 0 && d->n_tokens >= 0 && d->heads[0] >= 0 && d->heads[1] >= 0, "negative sizes");
    k.need(d->dim >= 1 && d->rot >= 2 && d->rot % 2 == 0 && d->rot <= d->dim, "rot is odd, or not 2 to a head's length");
    k.supported(d->dim <= 65536 && d->rot <= 2 * echo::kRotaryPairs, "heads of more than 65536 elements, or more than 512 turned");
    k.supported(d->heads[0] <= 65535 && d->heads[1] <= 65535 - d->heads[0], "more than 65535 heads");
    k.need(d->id_bits == 32 || d->id_bits == 64, "id_bits is neither 32 nor 64");
    k.need(known_type(d->type), "unknown element type");
    k.need(std::isfinite(d->scale), "the scale is not finite");
    k.need(d->frequencies, "frequencies is NULL");
    if (k.rc) return k.rc;
    echo::RotaryArgs a{};
    for (int i = 0; i < d->rot / 2; ++i) {
      k.need(std::fabs(d->frequencies[i]) <= 0x1p32, "a frequency is not within 2^32");  // (or a NaN)
      if (k.rc) return k.rc;
      a.turns[i] = echo::rotary_turns(d->frequencies[i]);
    }
    const int64_t tokens = d->n_batch == 0 ? 0 : d->n_tokens;
    k.supported(tokens == 0 || d->n_batch <= (((int64_t)1 << 31) - 1) / tokens, "more than 2^31 - 1 tokens");
    if (k.rc || tokens == 0 || d->heads[0] + d->heads[1] == 0) return k.rc;
    k.array(d->positions, d->id_bits / 8, "positions");
    const int64_t most = (int64_t)1 << 58, batches = d->n_batch - 1;
    k.need(d->positions_stride >= 0 && (batches == 0 || d->positions_stride <= most / batches), "a stride is negative, or an array does not fit the address space");
    for (int i = 0; i < 2; ++i) {
      if (k.rc || d->heads[i] == 0) continue;
      k.array(d->x[i], type_size(d->type), i ? "x[1]" : "x[0]");
      k.array(d->out[i], type_size(d->type), i ? "out[1]" : "out[0]");
      // a head at a time along each of the three: counts and strides of those that there is more than one of
      const int64_t count[3] = {d->n_batch, d->n_tokens, d->heads[i]};
      const int64_t in[3] = {d->x_batch_stride[i], d->x_stride[i], d->x_head_stride[i]}, out[3] = {d->out_batch_stride[i], d->out_stride[i], d->out_head_stride[i]};
      std::pair<int64_t, int64_t> at[3];  // stride, count
      int dims = 0;
      for (int j = 0; j < 3; ++j) {
        k.need(in[j] >= 0 && out[j] >= 0 && (count[j] == 1 || std::max(in[j], out[j]) <= most / (count[j] - 1)),
               "a stride is negative, or an array does not fit the address space");
        if (count[j] > 1) at[dims++] = {out[j], count[j]};
      }
      if (k.rc) return k.rc;
      // an output's heads are apart: each stride is at least what the smaller ones span
      std::sort(at, at + dims);
      int64_t span = d->dim;
      for (int j = 0; j < dims; ++j) {
        k.need(at[j].first >= span, "an output's heads overlap");
        span += at[j].first * (at[j].second - 1);
      }
    }
    if (k.rc) return k.rc;
    a.batch = d->n_batch, a.tokens = d->n_tokens;
    for (int i = 0; i < 2; ++i) {
      a.heads[i] = d->heads[i], a.x[i] = d->x[i], a.out[i] = d->out[i];
      // (a stride that nothing takes may be any)
      const bool b = a.batch > 1, t = a.tokens > 1, h = a.heads[i] > 1;
      a.x_batch[i] = b ? d->x_batch_stride[i] : 0, a.x_token[i] = t ? d->x_stride[i] : 0, a.x_head[i] = h ? d->x_head_stride[i] : 0;
      a.out_batch[i] = b ? d->out_batch_stride[i] : 0, a.out_token[i] = t ? d->out_stride[i] : 0, a.out_head[i] = h ? d->out_head_stride[i] : 0;
    }
    a.positions = d->positions, a.positions_batch = d->positions_stride, a.id64 = d->id_bits == 64;
    a.dim = d->dim, a.rot = d->rot, a.type = d->type, a.interleaved = d->interleaved != 0, a.back = back, a.scale = d->scale;
    RUN(echo::launch_rotary(a, o.sms, o.stream), name);
    return (int)ECHO_OK;
  });
}

}  // namespace

extern "C" {

int echo_stream_get(echo_ctx *c, void **cuda_stream) {
  return guarded([&]() -> int {
    OpContext o;
    if (const int rc = echo::op_context(c, &o)) return rc;
    if (!cuda_stream) return echo::op_error(c, ECHO_E_INVALID_ARG, "an argument is NULL");
    *cuda_stream = o.stream;
    return ECHO_OK;
  });
}

int echo_wait(echo_ctx *c) {
  return guarded([&] { return echo::op_wait(c); });
}

int echo_embed(echo_ctx *c, const echo_embed_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->n_tokens >= 0 && d->vocab_rows >= 0 && d->vocab_start >= 0 && d->hidden >= 1, "negative sizes, or no elements in a row");
    k.supported(d->hidden <= kMaxHidden, "rows of more than 2^30 elements");
    k.need(d->id_bits == 32 || d->id_bits == 64, "id_bits is neither 32 nor 64");
    k.need(known_type(d->table_type) && known_type(d->out_type), "unknown element type");
    if (k.rc || d->n_tokens == 0) return k.rc;
    k.array(d->ids, d->id_bits / 8, "ids");
    if (d->vocab_rows) k.matrix(d->table, d->table_type, d->vocab_rows, d->hidden, d->table_stride, false, "table");
    k.matrix(d->out, d->out_type, d->n_tokens, d->hidden, d->out_stride, true, "out");
    if (k.rc) return k.rc;
    const echo::EmbedArgs a{d->n_tokens, d->hidden, d->vocab_rows, d->vocab_start, d->ids, d->id_bits == 64, d->table, d->out,
                            d->table_stride, d->out_stride, d->table_type, d->out_type, d->scale};
    RUN(echo::launch_embed(a, o.sms, o.stream), "embed");
    return (int)ECHO_OK;
  });
}

int echo_embed_grad(echo_ctx *c, const echo_embed_grad_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->n_tokens >= 0 && d->vocab_rows >= 0 && d->vocab_start >= 0 && d->hidden >= 1, "negative sizes, or no elements in a row");
    k.supported(d->hidden <= kMaxHidden, "rows of more than 2^30 elements");
    k.supported(d->n_tokens < ((int64_t)1 << 31) && d->vocab_rows < ((int64_t)1 << 31) - 1, "more than 2^31 - 1 tokens or 2^31 - 2 rows");
    k.need(d->id_bits == 32 || d->id_bits == 64, "id_bits is neither 32 nor 64");
    k.need(known_type(d->dy_type) && known_type(d->dtable_type), "unknown element type");
    if (k.rc || d->vocab_rows == 0 || (d->n_tokens == 0 && d->accumulate)) return k.rc;
    if (d->n_tokens) {
      k.array(d->ids, d->id_bits / 8, "ids");
      k.matrix(d->dy, d->dy_type, d->n_tokens, d->hidden, d->dy_stride, false, "dy");
    }
    k.matrix(d->dtable, d->dtable_type, d->vocab_rows, d->hidden, d->dtable_stride, true, "dtable");
    if (k.rc) return k.rc;
    echo::EmbedGradArgs a{};
    a.n = d->n_tokens, a.H = d->hidden, a.V = d->vocab_rows, a.v0 = d->vocab_start;
    a.ids = d->ids, a.id64 = d->id_bits == 64, a.dy = d->dy, a.dtable = d->dtable;
    a.dy_stride = d->dy_stride, a.dtable_stride = d->dtable_stride, a.dy_type = d->dy_type, a.dtable_type = d->dtable_type;
    a.accumulate = d->accumulate != 0, a.scale = d->scale;
    a.window = echo::embed_grad_window(a.n, a.H, o.sms);
    const int64_t windows = (a.n + a.window - 1) / a.window;
    if (windows * ((a.H + 31) / 32) / 8 + a.V / 32 >= INT32_MAX) return echo::op_error(c, ECHO_E_UNSUPPORTED, "too many sums for one launch");
    const size_t list = up256((size_t)a.n * 4);
    void *scratch = nullptr;
    if (const int rc = echo::op_scratch(c, 4 * list + 256 + (size_t)windows * 2 * a.H * sizeof(float), &scratch)) return rc;
    char *at = static_cast<char *>(scratch);
    for (int i = 0; i < 2; ++i) {
      a.key[i] = reinterpret_cast<uint32_t *>(at + 2 * i * list);
      a.tok[i] = reinterpret_cast<uint32_t *>(at + (2 * i + 1) * list);
    }
    a.count = reinterpret_cast<int32_t *>(at + 4 * list);
    a.part = reinterpret_cast<float *>(at + 4 * list + 256);
    RUN(echo::launch_embed_sort(a, o.stream), "embed_sort");
    RUN(echo::launch_embed_sum(a, o.stream), "embed_sum");
    if (a.n == 0) return (int)ECHO_OK;
    RUN(echo::launch_embed_join(a, o.stream), "embed_join");
    return (int)ECHO_OK;
  });
}

int echo_layer_norm(echo_ctx *c, const echo_layer_norm_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->rows >= 0 && d->hidden >= 1, "negative rows, or no elements in a row");
    k.supported(d->hidden <= kMaxHidden, "rows of more than 2^30 elements");
    k.need(known_type(d->x_type) && known_type(d->param_type), "unknown element type");
    k.need(d->eps >= 0.f && std::isfinite(d->eps), "eps is negative or not finite");
    if (k.rc || d->rows == 0) return k.rc;
    k.matrix(d->x, d->x_type, d->rows, d->hidden, d->x_stride, false, "x");
    k.matrix(d->y, d->x_type, d->rows, d->hidden, d->y_stride, true, "y");
    if (d->weight) k.array(d->weight, type_size(d->param_type), "weight");
    if (d->bias) k.array(d->bias, type_size(d->param_type), "bias");
    if (d->mean) k.array(d->mean, 4, "mean");
    if (d->rstd) k.array(d->rstd, 4, "rstd");
    if (k.rc) return k.rc;
    const echo::NormArgs a{d->rows, d->hidden, d->x, d->y, d->weight, d->bias, d->mean, d->rstd,
                           d->x_stride, d->y_stride, d->x_type, d->param_type, d->eps};
    RUN(echo::launch_layer_norm(a, o.sms, o.stream), "layer_norm");
    return (int)ECHO_OK;
  });
}

int echo_layer_norm_grad(echo_ctx *c, const echo_layer_norm_grad_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->rows >= 0 && d->hidden >= 1, "negative rows, or no elements in a row");
    k.supported(d->hidden <= kMaxHidden, "rows of more than 2^30 elements");
    k.need(known_type(d->x_type) && known_type(d->param_type), "unknown element type");
    if (k.rc) return k.rc;
    const bool params = d->dweight || d->dbias;
    if (d->rows) {
      k.matrix(d->dy, d->x_type, d->rows, d->hidden, d->dy_stride, false, "dy");
      k.matrix(d->x, d->x_type, d->rows, d->hidden, d->x_stride, false, "x");
      k.array(d->mean, 4, "mean");
      k.array(d->rstd, 4, "rstd");
      if (d->dx) k.matrix(d->dx, d->x_type, d->rows, d->hidden, d->dx_stride, true, "dx");
      if (d->weight) k.array(d->weight, type_size(d->param_type), "weight");
    }
    if (d->dweight) k.array(d->dweight, type_size(d->param_type), "dweight");
    if (d->dbias) k.array(d->dbias, type_size(d->param_type), "dbias");
    if (k.rc || (d->rows == 0 && (!params || d->accumulate))) return k.rc;
    echo::NormGradArgs a{d->rows, d->hidden, d->dy, d->x, d->weight, d->mean, d->rstd, d->dx, d->dweight, d->dbias,
                         d->dy_stride, d->x_stride, d->dx_stride, d->x_type, d->param_type, d->accumulate != 0, nullptr, 0};
    if (params) {
      a.parts = d->rows ? echo::layer_norm_grad_parts(a, o.sms) : 0;
      void *scratch = nullptr;
      if (const int rc = echo::op_scratch(c, (size_t)a.parts * 2 * a.H * sizeof(float), &scratch)) return rc;
      a.part = static_cast<float *>(scratch);
    }
    const cudaError_t e = echo::launch_layer_norm_grad(a, o.sms, timer(c), o.stream);
    if (e != cudaSuccess) return echo::op_cuda_error(c, e, "layer_norm_grad");
    return (int)ECHO_OK;
  });
}

int echo_orthogonalize(echo_ctx *c, const echo_orthogonalize_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    Checks k{c};
    k.need(d->batch >= 0 && d->rows >= 1 && d->cols >= 1, "negative batch, or a matrix without elements");
    k.supported(d->rows <= 65536 && d->cols <= 65536, "matrices of more than 65536 rows or columns");
    k.supported(d->batch < ((int64_t)1 << 31), "more than 2^31 - 1 matrices");
    k.need(d->steps >= 0 && d->steps <= 64, "steps is not 0 to 64");
    k.need(std::isfinite(d->a) && std::isfinite(d->b) && std::isfinite(d->c) && std::isfinite(d->scale), "a coefficient or the scale is not finite");
    k.need(d->eps >= 0.f && std::isfinite(d->eps), "eps is negative or not finite");
    k.need(known_type(d->type), "unknown element type");
    if (k.rc || d->batch == 0) return k.rc;
    k.matrix(d->g, d->type, d->rows, d->cols, d->g_stride, false, "g");
    k.matrix(d->o, d->type, d->rows, d->cols, d->o_stride, true, "o");
    const int64_t o_span = (d->rows - 1) * d->o_stride + d->cols;  // of a matrix
    k.need(d->g_batch_stride >= 0 && d->o_batch_stride >= 0 && (d->batch == 1 || d->o_batch_stride >= o_span),
           "a batch stride is negative, or the output's less than a matrix");
    k.need(d->batch == 1 || std::max(d->g_batch_stride, d->o_batch_stride) <= ((int64_t)1 << 58) / (d->batch - 1), "a batch does not fit the address space");
    if (k.rc) return k.rc;
    echo::OrthoArgs a{d->batch, std::min(d->rows, d->cols), std::max(d->rows, d->cols), d->rows >= d->cols, d->g, d->o,
                      d->g_stride, d->g_batch_stride, d->o_stride, d->o_batch_stride, d->type, d->steps,
                      d->a, d->b, d->c, d->eps, d->scale, nullptr, nullptr, o.wait_limit, o.skip};
    if (const int rc = echo::op_status(c, &a.status)) return rc;
    if (const int rc = echo::op_scratch(c, echo::ortho_scratch_bytes(a, o.sms), &a.scratch)) return rc;
    const cudaError_t e = echo::launch_orthogonalize(a, o.sms, timer(c), o.stream);
    if (e != cudaSuccess) return echo::op_cuda_error(c, e, "orthogonalize");
    return (int)ECHO_OK;
  });
}

int echo_cross_entropy(echo_ctx *c, const echo_cross_entropy_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    echo::HeadArgs a = head_of(o, *d);
    a.ids = d->labels, a.K = 1, a.tau = 1.f;
    a.loss = d->loss, a.lse = d->lse, a.part = d->target;
    return head_forward(c, o, a, "target");
  });
}

int echo_distill(echo_ctx *c, const echo_distill_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    echo::HeadArgs a = head_of(o, *d);
    Checks k{c};
    if (const int rc = teacher_of(k, a, *d)) return rc;
    a.loss = d->loss, a.lse = d->lse, a.part = d->cross;
    return head_forward(c, o, a, "cross");
  });
}

int echo_cross_entropy_grad(echo_ctx *c, const echo_cross_entropy_grad_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    echo::HeadArgs a = head_of(o, *d);
    a.ids = d->labels, a.K = 1, a.tau = 1.f;
    return head_backward(c, o, a, *d);
  });
}

int echo_distill_grad(echo_ctx *c, const echo_distill_grad_desc *d) {
  return entry(c, d, [&](const OpContext &o) {
    echo::HeadArgs a = head_of(o, *d);
    Checks k{c};
    if (const int rc = teacher_of(k, a, *d)) return rc;
    return head_backward(c, o, a, *d);
  });
}

int echo_rotary(echo_ctx *c, const echo_rotary_desc *d) { return rotary(c, d, false, "rotary"); }

int echo_rotary_grad(echo_ctx *c, const echo_rotary_desc *d) { return rotary(c, d, true, "rotary_grad"); }

}  // extern "C"
