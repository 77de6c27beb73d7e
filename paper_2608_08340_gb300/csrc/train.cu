// C entry points of the operators that train a query encoder against an index
// (declared in include/oprag.h): argument checks, then the launch.
#include <cfloat>
#include <cmath>

#include "oprag.h"
#include "internal.h"
#include "overlap.h"

using namespace oprag;

namespace {

bool is_dtype(int32_t d) { return d == OPRAG_F32 || d == OPRAG_BF16; }
int dtype_of(int32_t d) { return d == OPRAG_BF16 ? kBF16 : kF32; }
int64_t size_of(int32_t d) { return d == OPRAG_BF16 ? 2 : 4; }
bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

Rows rows_of(const void* at, int64_t rows, int64_t bytes, int64_t stride) {
  return {reinterpret_cast<uintptr_t>(at), rows, bytes, stride};
}

// Whether out, `bytes` long, lies over a gradient of texts x tokens rows (strides in bytes,
// any of them 0).
bool over_gradient(const void* out, int64_t bytes, const void* grad, int64_t texts, int64_t tokens,
                   int64_t row, int64_t text_stride, int64_t token_stride) {
  if (texts < 1 || tokens < 1) return false;
  const Rows to = rows_of(out, 1, bytes, bytes);
  // A text's rows, one block where they touch.
  const int64_t text = (tokens - 1) * token_stride + row;
  Rows part = token_stride > row ? rows_of(grad, tokens, row, token_stride)
                                 : rows_of(grad, 1, text, text);
  const int64_t whole = (texts - 1) * text_stride + text;
  if (!overlap(to, rows_of(grad, 1, whole, whole))) return false;
  for (int64_t b = 0; b < (text_stride == 0 ? 1 : texts); ++b, part.at += text_stride)
    if (overlap(to, part)) return true;
  return false;
}

}  // namespace

extern "C" {

int oprag_embed_lookup(const void* table, int32_t table_dtype, int64_t vocab, int32_t dim,
                       int64_t row_stride, const void* ids, int32_t ids_64, int64_t count,
                       float scale, void* out, int32_t out_dtype, void* stream) {
  if (!is_dtype(table_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "table dtype %d", table_dtype);
  if (!is_dtype(out_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "output dtype %d", out_dtype);
  if (vocab < 1 || vocab > INT32_MAX)
    return fail(OPRAG_ERR_INVALID_ARG, "vocab %lld outside [1, 2^31)", static_cast<long long>(vocab));
  if (dim < 8 || dim % 8 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "dim %d is not a positive multiple of 8", dim);
  if (row_stride < dim || row_stride * size_of(table_dtype) % 16 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "row stride %lld: at least dim, and whole 16 bytes",
                static_cast<long long>(row_stride));
  if (count < 0 || count > INT32_MAX)
    return fail(OPRAG_ERR_INVALID_ARG, "count %lld outside [0, 2^31)", static_cast<long long>(count));
  if (count == 0) return ok();
  if (!table || !ids || !out) return fail(OPRAG_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(table) || !aligned(out))
    return fail(OPRAG_ERR_INVALID_ARG, "table and out must be 16-byte aligned");
  const int64_t size = size_of(table_dtype), bytes = count * dim * size_of(out_dtype);
  if (overlap(rows_of(out, 1, bytes, bytes), rows_of(table, vocab, dim * size, row_stride * size)))
    return fail(OPRAG_ERR_INVALID_ARG, "out overlaps table");
  const LookupArgs a{table, dtype_of(table_dtype), vocab, row_stride, dim, ids, ids_64 != 0, count,
                     scale, out, dtype_of(out_dtype)};
  const cudaError_t e = launch_embed_lookup(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ok() : cuda_fail(e, "embedding lookup");
}

int oprag_embed_lookup_grad_workspace(int64_t count, int64_t vocab, int32_t dim, int64_t* bytes) {
  if (!bytes) return fail(OPRAG_ERR_INVALID_ARG, "bytes is NULL");
  if (count < 0 || count > INT32_MAX || vocab < 1 || vocab >= INT32_MAX || dim < 8 || dim % 8 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "need count >= 0, vocab >= 1, dim a positive multiple of 8");
  *bytes = embed_lookup_grad_workspace(count, vocab, dim);
  return ok();
}

int oprag_embed_lookup_grad(const void* grad, int32_t grad_dtype, int64_t texts, int64_t tokens,
                            int32_t dim, int64_t text_stride, int64_t token_stride, const void* ids,
                            int32_t ids_64, int64_t vocab, float scale, void* out,
                            int32_t out_dtype, void* workspace, int64_t workspace_bytes,
                            void* stream) {
  if (!is_dtype(grad_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "gradient dtype %d", grad_dtype);
  if (!is_dtype(out_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "output dtype %d", out_dtype);
  if (vocab < 1 || vocab >= INT32_MAX)
    return fail(OPRAG_ERR_INVALID_ARG, "vocab %lld outside [1, 2^31 - 1)",
                static_cast<long long>(vocab));
  if (dim < 8 || dim % 8 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "dim %d is not a positive multiple of 8", dim);
  if (texts < 0 || tokens < 0 || (tokens > 0 && texts > INT32_MAX / tokens))
    return fail(OPRAG_ERR_INVALID_ARG, "texts * tokens outside [0, 2^31)");
  const int64_t size = size_of(grad_dtype);
  if (text_stride < 0 || token_stride < 0 || text_stride * size % 16 != 0 ||
      token_stride * size % 16 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "strides must not be negative and be whole 16 bytes");
  const int64_t count = texts * tokens;
  const int64_t need = embed_lookup_grad_workspace(count, vocab, dim);
  if (!out || (count > 0 && (!grad || !ids)) || (need > 0 && !workspace))
    return fail(OPRAG_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(out) || (count > 0 && !aligned(grad)) || (need > 0 && !aligned(workspace)))
    return fail(OPRAG_ERR_INVALID_ARG, "grad, out and workspace must be 16-byte aligned");
  if (workspace_bytes < need)
    return fail(OPRAG_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed",
                static_cast<long long>(workspace_bytes), static_cast<long long>(need));
  if (over_gradient(out, vocab * dim * size_of(out_dtype), grad, texts, tokens, dim * size,
                    text_stride * size, token_stride * size))
    return fail(OPRAG_ERR_INVALID_ARG, "out overlaps grad");
  const LookupGradArgs a{grad, dtype_of(grad_dtype), count, tokens, text_stride, token_stride, dim,
                         ids, ids_64 != 0, vocab, scale, out, dtype_of(out_dtype), workspace};
  const cudaError_t e = launch_embed_lookup_grad(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ok() : cuda_fail(e, "gradient of the embedding lookup");
}

int oprag_embed_pool_train(const void* hidden, int32_t hidden_dtype, int32_t batch, int32_t tokens,
                           int32_t dim, const uint8_t* mask, void* out, int32_t out_dtype,
                           float* mean, void* stream) {
  if (!is_dtype(hidden_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "hidden dtype %d", hidden_dtype);
  if (!is_dtype(out_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "output dtype %d", out_dtype);
  if (batch < 0 || tokens < 1 || dim < 8 || dim % 8 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "need batch >= 0, tokens >= 1, dim a positive multiple of 8");
  if (dim > (hidden_dtype == OPRAG_BF16 ? 16384 : 8192))
    return fail(OPRAG_ERR_INVALID_ARG, "dim %d too large", dim);
  if (batch == 0) return ok();
  if (!hidden || !mask || !out || !mean) return fail(OPRAG_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(hidden) || !aligned(out) || !aligned(mean))
    return fail(OPRAG_ERR_INVALID_ARG, "hidden, out and mean must be 16-byte aligned");
  const cudaError_t e =
      launch_embed_pool(dtype_of(hidden_dtype), hidden, batch, tokens, dim, mask,
                        dtype_of(out_dtype), out, mean, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ok() : cuda_fail(e, "embedding tail kernel");
}

int oprag_embed_pool_grad(const void* grad, int32_t grad_dtype, const float* mean, int32_t batch,
                          int32_t tokens, int32_t dim, const uint8_t* mask, void* out,
                          int32_t out_dtype, int32_t per_token, void* stream) {
  if (!is_dtype(grad_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "gradient dtype %d", grad_dtype);
  if (!is_dtype(out_dtype)) return fail(OPRAG_ERR_INVALID_ARG, "output dtype %d", out_dtype);
  if (batch < 0 || tokens < 1 || dim < 8 || dim % 8 != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "need batch >= 0, tokens >= 1, dim a positive multiple of 8");
  if (dim > 16384) return fail(OPRAG_ERR_INVALID_ARG, "dim %d too large", dim);
  if (batch == 0) return ok();
  if (!grad || !mean || !mask || !out) return fail(OPRAG_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(grad) || !aligned(mean) || !aligned(out))
    return fail(OPRAG_ERR_INVALID_ARG, "grad, mean and out must be 16-byte aligned");
  const cudaError_t e =
      launch_embed_pool_grad(grad, dtype_of(grad_dtype), mean, batch, tokens, dim, mask, out,
                             dtype_of(out_dtype), per_token != 0, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ok() : cuda_fail(e, "gradient of the embedding tail");
}

int oprag_distill(const void* logits, int32_t dtype, int64_t row_stride, int32_t q, int32_t n,
                  const int64_t* teacher_ids, const float* teacher_scores, int32_t k,
                  float temperature, const float* weight, float* loss, void* grad,
                  int64_t grad_stride, void* stream) {
  if (!is_dtype(dtype)) return fail(OPRAG_ERR_INVALID_ARG, "dtype %d", dtype);
  if (q < 0 || n < 1) return fail(OPRAG_ERR_INVALID_ARG, "need q >= 0, n >= 1");
  if (k < 1 || k > OPRAG_K_MAX)
    return fail(OPRAG_ERR_INVALID_ARG, "k = %d outside [1, %d]", k, OPRAG_K_MAX);
  if (!(temperature >= FLT_MIN) || std::isinf(temperature))   // (1 / temperature is finite too)
    return fail(OPRAG_ERR_INVALID_ARG, "temperature %g is not positive, normal and finite", temperature);
  if (row_stride < n || (grad && grad_stride < n))
    return fail(OPRAG_ERR_INVALID_ARG, "row strides must be at least n");
  if (q == 0) return ok();
  if (!logits || !teacher_ids || !teacher_scores || !loss)
    return fail(OPRAG_ERR_INVALID_ARG, "NULL argument");
  const uintptr_t bits = reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(grad);
  if (bits % size_of(dtype) != 0)
    return fail(OPRAG_ERR_INVALID_ARG, "logits and grad must be aligned to their values");
  const int64_t size = size_of(dtype);
  if (grad && !(grad == logits && (q == 1 || grad_stride == row_stride)) &&
      overlap(rows_of(logits, q, n * size, row_stride * size),
              rows_of(grad, q, n * size, grad_stride * size)))
    return fail(OPRAG_ERR_INVALID_ARG,
                "grad overlaps logits: it may be logits itself, with its stride, or lie apart");
  const DistillArgs a{logits, dtype_of(dtype), row_stride, q, n, k, teacher_ids, teacher_scores,
                      temperature, weight, loss, grad, grad_stride};
  const cudaError_t e = launch_distill(a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ok() : cuda_fail(e, "distillation kernel");
}

}  // extern "C"
