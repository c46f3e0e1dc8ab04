// C ABI of the output head: argument checks of each entry point.
#include "head.hpp"

using namespace embbag;

namespace {

constexpr int64_t kInt32Max = 2147483647;
constexpr int64_t kMaxRowsX = (int64_t(1) << 23) - 1;  // rows of x, dy: m * k / 128 < 2^31
constexpr int64_t kMaxMatrix = int64_t(1) << 40;       // elements of a matrix of logits
constexpr size_t kWsAlign = 256;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? EMBBAG_OK : EMBBAG_ERR_HIP; }

bool type_ok(int32_t t) { return t == EMBBAG_F32 || t == EMBBAG_BF16; }
size_t type_size(int32_t t) { return t == EMBBAG_BF16 ? 2 : 4; }

bool dim_ok(int32_t dim) { return dim >= 4 && dim <= kMxMaxDim && dim % 4 == 0; }

// Rows that are read and written 4 elements at a time.
bool rows_ok(const void* p, int32_t type, int64_t stride, int32_t dim) {
  return type_ok(type) && stride >= dim && stride % 4 == 0 && p != nullptr &&
         aligned(p, 4 * type_size(type));
}

// Rows of any alignment.
bool matrix_ok(const void* p, int32_t type, int64_t stride, int64_t cols) {
  return type_ok(type) && stride >= cols && p != nullptr && aligned(p, type_size(type));
}

bool table_ok(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t dim) {
  return dim_ok(dim) && rows >= 1 && rows <= kInt32Max && codes != nullptr && scales != nullptr &&
         aligned(codes, 16) && aligned(scales, 4);
}

bool product_ok(int32_t m, int64_t n, int32_t k) {
  return m >= 0 && m <= kMaxRowsX && n >= 1 && n <= kInt32Max && dim_ok(k) && m * n <= kMaxMatrix;
}

// A list per row (offsets, entries) of n entries, fewer than 2^30: occurrences are counted in
// 30 bits.
int check_list(int32_t rows, const int32_t* offsets, const void* entries, int64_t n) {
  if (n < 0 || n >= (int64_t(1) << 30)) return EMBBAG_ERR_INVALID_ARG;
  if (offsets == nullptr) return n == 0 && entries == nullptr ? EMBBAG_OK : EMBBAG_ERR_INVALID_ARG;
  if (n > 0 && entries == nullptr) return EMBBAG_ERR_INVALID_ARG;
  if (rows == 0 && n > 0) return EMBBAG_ERR_OFFSETS;
  return EMBBAG_OK;
}

}  // namespace

extern "C" {

int embbag_mx4_quantize(const void* src, int32_t src_type, int64_t src_stride, int64_t rows,
                        int32_t dim, const int32_t* row_ids, int64_t num_ids, uint8_t* codes,
                        uint8_t* scales, int32_t* d_status, hipStream_t stream) {
  if (!table_ok(codes, scales, rows, dim) || !rows_ok(src, src_type, src_stride, dim))
    return EMBBAG_ERR_INVALID_ARG;
  if (num_ids < 0 || num_ids > kInt32Max || (row_ids == nullptr && num_ids != 0))
    return EMBBAG_ERR_INVALID_ARG;
  return hip_status(launch_mx4_quantize(src, src_type == EMBBAG_BF16, src_stride, rows, dim,
                                        row_ids, num_ids, codes, scales, d_status, stream));
}

int embbag_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t dim,
                          void* dst, int32_t dst_type, int64_t dst_stride, hipStream_t stream) {
  if (!table_ok(codes, scales, rows, dim) || !rows_ok(dst, dst_type, dst_stride, dim))
    return EMBBAG_ERR_INVALID_ARG;
  return hip_status(launch_mx4_dequantize({codes, scales, rows, dim}, dst,
                                          dst_type == EMBBAG_BF16, dst_stride, stream));
}

int embbag_mx4_forward(const embbag_mx4_tables_t* tables, int32_t batch, const int32_t* indices,
                       const int32_t* offsets, int64_t num_indices,
                       const float* per_sample_weights, int32_t pooling, void* pooled_out,
                       int32_t out_type, int32_t* d_status, hipStream_t stream) {
  if (tables == nullptr || tables->rows == nullptr || tables->codes == nullptr ||
      tables->scales == nullptr || !type_ok(out_type))
    return EMBBAG_ERR_INVALID_ARG;
  const int32_t T = tables->num_tables;
  if (T < 1 || T > kMaxTables || !dim_ok(tables->dim) || tables->dim > 1024)
    return EMBBAG_ERR_INVALID_ARG;
  PoolArgs pool;
  if (pooling == EMBBAG_POOL_SUM)
    pool.mode = per_sample_weights != nullptr ? kPoolWeighted : kPoolPlain;
  else if (pooling == EMBBAG_POOL_MEAN && per_sample_weights == nullptr)
    pool.mode = kPoolMean;
  else
    return EMBBAG_ERR_INVALID_ARG;
  pool.weights = per_sample_weights;
  TableDesc d = {};
  int64_t total = 0;
  for (int t = 0; t < T; ++t) {
    if (!table_ok(tables->codes[t], tables->scales[t], tables->rows[t], tables->dim))
      return EMBBAG_ERR_INVALID_ARG;
    d.w[t] = tables->codes[t];
    d.lo[t] = tables->scales[t];
    d.rows[t] = uint32_t(tables->rows[t]);
    d.rowbase[t] = uint32_t(total);
    total += tables->rows[t];
    if (total > kInt32Max) return EMBBAG_ERR_INVALID_ARG;
  }
  d.rowbase[T] = uint32_t(total);
  d.num_tables = T;
  d.dim = tables->dim;
  if (batch < 0 || num_indices < 0 || num_indices > kInt32Max || offsets == nullptr ||
      int64_t(T) * batch + 1 > kInt32Max || (num_indices > 0 && indices == nullptr))
    return EMBBAG_ERR_INVALID_ARG;
  if (int64_t(T) * batch == 0 && num_indices > 0) return EMBBAG_ERR_OFFSETS;
  if (int64_t(T) * batch > 0 && (pooled_out == nullptr || !aligned(pooled_out, 4 * type_size(out_type))))
    return EMBBAG_ERR_INVALID_ARG;
  return hip_status(launch_mx4_forward(d, batch, indices, offsets, num_indices, pooled_out,
                                       out_type == EMBBAG_BF16, d_status, pool, stream));
}

size_t embbag_mx4_matmul_workspace_bytes(int32_t m, int64_t n, int32_t k) {
  return product_ok(m, n, k) ? mx4_matmul_workspace(m, n, k) : 0;
}

int embbag_mx4_matmul(const void* x, int32_t x_type, int64_t x_stride, int32_t m,
                      const uint8_t* codes, const uint8_t* scales, int64_t n, int32_t k, void* out,
                      int32_t out_type, int64_t out_stride, void* workspace,
                      size_t workspace_bytes, hipStream_t stream) {
  if (!product_ok(m, n, k) || !table_ok(codes, scales, n, k)) return EMBBAG_ERR_INVALID_ARG;
  if (!type_ok(x_type) || !type_ok(out_type)) return EMBBAG_ERR_INVALID_ARG;
  if (m > 0 && (!rows_ok(x, x_type, x_stride, k) || !matrix_ok(out, out_type, out_stride, n)))
    return EMBBAG_ERR_INVALID_ARG;
  if (workspace_bytes < mx4_matmul_workspace(m, n, k) || !aligned(workspace, kWsAlign) ||
      (workspace == nullptr && mx4_matmul_workspace(m, n, k) > 0))
    return EMBBAG_ERR_WORKSPACE;
  return hip_status(launch_mx4_matmul(x, x_type == EMBBAG_BF16, x_stride, m, {codes, scales, n, k},
                                      out, out_type == EMBBAG_BF16, out_stride,
                                      static_cast<char*>(workspace), stream));
}

size_t embbag_mx4_matmul_grad_workspace_bytes(int32_t m, int64_t n, int32_t k) {
  return product_ok(m, n, k) ? mx4_matmul_grad_workspace(m, n, k) : 0;
}

int embbag_mx4_matmul_grad(const void* dy, int32_t dy_type, int64_t dy_stride, int32_t m,
                           const uint8_t* codes, const uint8_t* scales, int64_t n, int32_t k,
                           void* dx, int32_t dx_type, int64_t dx_stride, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  if (!product_ok(m, n, k) || !table_ok(codes, scales, n, k)) return EMBBAG_ERR_INVALID_ARG;
  if (!type_ok(dy_type) || !type_ok(dx_type)) return EMBBAG_ERR_INVALID_ARG;
  if (m > 0 && (!matrix_ok(dy, dy_type, dy_stride, n) || !rows_ok(dx, dx_type, dx_stride, k)))
    return EMBBAG_ERR_INVALID_ARG;
  if (workspace_bytes < mx4_matmul_grad_workspace(m, n, k) || !aligned(workspace, kWsAlign) ||
      (workspace == nullptr && mx4_matmul_grad_workspace(m, n, k) > 0))
    return EMBBAG_ERR_WORKSPACE;
  return hip_status(launch_mx4_matmul_grad(dy, dy_type == EMBBAG_BF16, dy_stride, m,
                                           {codes, scales, n, k}, dx, dx_type == EMBBAG_BF16,
                                           dx_stride, static_cast<char*>(workspace), stream));
}

int embbag_logits_process(const embbag_logits_t* args, int32_t* d_status, hipStream_t stream) {
  if (args == nullptr) return EMBBAG_ERR_INVALID_ARG;
  const embbag_logits_t& a = *args;
  if (a.rows < 0 || a.vocab < 1 || !type_ok(a.type) || int64_t(a.rows) * a.vocab > kMaxMatrix)
    return EMBBAG_ERR_INVALID_ARG;
  if (a.rows > 0 && (!matrix_ok(a.logits, a.type, a.logits_stride, a.vocab) ||
                     !matrix_ok(a.out, a.type, a.out_stride, a.vocab)))
    return EMBBAG_ERR_INVALID_ARG;
  if (a.rows > 1 && a.out == a.logits && a.out_stride != a.logits_stride)
    return EMBBAG_ERR_INVALID_ARG;
  int rc = check_list(a.rows, a.seen_offsets, a.seen, a.num_seen);
  if (rc) return rc;
  rc = check_list(a.rows, a.bias_offsets, a.bias_ids, a.num_biases);
  if (rc) return rc;
  if (a.bias_offsets != nullptr && a.num_biases > 0 && a.biases == nullptr)
    return EMBBAG_ERR_INVALID_ARG;
  if (a.seen_offsets == nullptr && (a.prompt_lens != nullptr || a.repetition != nullptr ||
                                    a.frequency != nullptr || a.presence != nullptr))
    return EMBBAG_ERR_INVALID_ARG;
  if (a.masks != nullptr) {
    if (a.num_masks < 1 || a.mask_stride < (int64_t(a.vocab) + 31) / 32 || !aligned(a.masks, 4))
      return EMBBAG_ERR_INVALID_ARG;
    if (a.mask_ids == nullptr && a.num_masks < a.rows) return EMBBAG_ERR_INVALID_ARG;
  } else if (a.mask_ids != nullptr) {
    return EMBBAG_ERR_INVALID_ARG;
  }
  return hip_status(launch_logits(a, d_status, stream));
}

size_t embbag_distill_workspace_bytes(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 0 || vocab < 1 || top < 1 || top > kMaxTeacher || int64_t(rows) * vocab > kMaxMatrix)
    return 0;
  return distill_workspace(rows, vocab, top);
}

int embbag_distill(const embbag_distill_t* args, void* workspace, size_t workspace_bytes,
                   int32_t* d_status, hipStream_t stream) {
  if (args == nullptr) return EMBBAG_ERR_INVALID_ARG;
  const embbag_distill_t& a = *args;
  if (a.rows < 0 || a.vocab < 1 || !type_ok(a.type) || !type_ok(a.teacher_type) || a.top < 1 ||
      a.top > kMaxTeacher || int64_t(a.rows) * a.vocab > kMaxMatrix)
    return EMBBAG_ERR_INVALID_ARG;
  if (!(a.temperature >= 1e-6f && a.temperature <= 1e6f)) return EMBBAG_ERR_INVALID_ARG;
  if (a.rows > 0) {
    if (!matrix_ok(a.logits, a.type, a.logits_stride, a.vocab) || a.ids == nullptr ||
        a.teacher == nullptr || a.loss == nullptr)
      return EMBBAG_ERR_INVALID_ARG;
    if (a.grad != nullptr && !matrix_ok(a.grad, a.type, a.grad_stride, a.vocab))
      return EMBBAG_ERR_INVALID_ARG;
    if (a.rows > 1 && a.grad == a.logits && a.grad_stride != a.logits_stride)
      return EMBBAG_ERR_INVALID_ARG;
  }
  const size_t need = distill_workspace(a.rows, a.vocab, a.top);
  if (workspace_bytes < need || !aligned(workspace, kWsAlign) || (workspace == nullptr && need > 0))
    return EMBBAG_ERR_WORKSPACE;
  return hip_status(launch_distill(a, static_cast<char*>(workspace), d_status, stream));
}

}  // extern "C"
