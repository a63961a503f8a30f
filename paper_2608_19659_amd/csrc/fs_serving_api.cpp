// fs_serving_api.cpp -- C entries of the serving operators: argument checks,
// workspace sizes and launches on the caller's stream.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <vector>

#include "fs_host.h"
#include "fs_serving.h"

namespace {

using fs::DeviceGuard;
using fs::fail;
using fs::hip_fail;

constexpr int64_t kMost = 0x7fffffff;

bool element_type(fs_dtype t) { return t == FS_F32 || t == FS_F16 || t == FS_BF16; }

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

fs_status check_product(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || N < 0 || K < 0 || M > kMost || N > kMost || K > kMost)
    return fail(FS_ERR_INVALID_ARGUMENT, "M, N and K must be in [0, 2^31)");
  if (K > FS_MAX_INNER)
    return fail(FS_ERR_UNSUPPORTED, "K must be at most " + std::to_string(FS_MAX_INNER) + " (32-bit sums)");
  return FS_OK;
}

// Codes of M rows for fs_linear: rows an odd number of lines of 128 bytes apart,
// so that the same columns of neighbouring rows, which all tiles read together,
// do not meet in a few channels of L2.  (2048 x 5120 x 5120 78 to 80 us a call
// and 79 with rows of 5120 bytes on one card, 80 and 84 on another; 64 rows 12.3
// either way.)
int64_t padded(int64_t K) { return ((K + 127) / 128 | 1) * 128; }

size_t linear_codes(int64_t M, int64_t K) { return align256((size_t)(M * padded(K))); }

fs_status check_cache(const fs_kv_cache *c) {
  if (!c) return fail(FS_ERR_INVALID_ARGUMENT, "cache is NULL");
  if (c->n_pages < 0 || c->n_heads < 1 || c->head_dim < 1 || c->page_size < 1)
    return fail(FS_ERR_INVALID_ARGUMENT, "cache sizes must be positive (n_pages >= 0)");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(FS_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64)
    return fail(FS_ERR_UNSUPPORTED, "page_size must be 16, 32 or 64");
  if (c->n_heads > 4096) return fail(FS_ERR_UNSUPPORTED, "n_heads must be at most 4096");
  if ((int64_t)c->n_pages * c->page_size > kMost)
    return fail(FS_ERR_UNSUPPORTED, "the cache's slots must number less than 2^31");
  return FS_OK;
}

fs_status check_cache_memory(const fs_kv_cache *c) {
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || c->n_pages < 1)
    return fail(FS_ERR_INVALID_ARGUMENT, "the cache has no memory");
  if (((uintptr_t)c->k | (uintptr_t)c->v) & 15)
    return fail(FS_ERR_INVALID_ARGUMENT, "the cache's codes must start on multiples of 16 bytes");
  return FS_OK;
}

fs::Cache to_cache(const fs_kv_cache *c) {
  return fs::Cache{c->k,       c->v,       c->k_scale, c->v_scale, c->n_pages, c->n_heads, c->head_dim,
                   c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : 6};
}

// FS_VALIDATE=1: launches a check on cleared counters, waits and reads them.
std::mutex g_checking;  // the counters are the device's

template <class Launch>
fs_status checked(Launch launch, hipStream_t stream, const char *what, const char *const (&texts)[2]) {
  std::lock_guard<std::mutex> lock(g_checking);
  int32_t *flag = nullptr, counted[2] = {0, 0};
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(stream, &capture);
  if (e == hipSuccess && capture != hipStreamCaptureStatusNone)  // refused while nothing is enqueued
    return fail(FS_ERR_DEVICE, std::string(what) + ": FS_VALIDATE=1 waits for the stream, which is being captured");
  if (e == hipSuccess) e = fs::flag_address(&flag);
  if (e == hipSuccess) e = fs::launch_clear_flag(flag, stream);
  if (e == hipSuccess) e = launch(flag);
  if (e == hipSuccess) e = hipMemcpyAsync(counted, flag, sizeof(counted), hipMemcpyDeviceToHost, stream);
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  if (e != hipSuccess) return hip_fail(e, what);
  for (int i = 0; i < 2; ++i)
    if (counted[i])
      return fail(FS_ERR_INVALID_ARGUMENT, std::string(what) + ": " + std::to_string(counted[i]) + " " + texts[i]);
  return FS_OK;
}

// FS_VALIDATE=1: a page may have one run of tokens.  A block enters a page for
// each token that does not follow the one before it, so two of them in one page
// would write its scale and codes at the same time.
fs_status check_pages(const fs::Cache &c, const int32_t *d_slots, int64_t n_tokens, hipStream_t stream, const char *what) {
  try {
    std::vector<int32_t> slots((size_t)n_tokens), pages;
    hipError_t e = hipMemcpyAsync(slots.data(), d_slots, slots.size() * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    if (e != hipSuccess) return hip_fail(e, what);
    const int32_t in_page = (1 << c.page_shift) - 1;
    for (size_t t = 0; t < slots.size(); ++t)
      if (slots[t] >= 0 && (!(slots[t] & in_page) || t == 0 || slots[t - 1] != slots[t] - 1))
        pages.push_back(slots[t] >> c.page_shift);
    const size_t runs = pages.size();
    std::sort(pages.begin(), pages.end());
    pages.erase(std::unique(pages.begin(), pages.end()), pages.end());
    if (runs != pages.size())
      return fail(FS_ERR_INVALID_ARGUMENT, std::string(what) + ": " + std::to_string(runs - pages.size()) +
                                               " tokens that do not follow in their page");
    return FS_OK;
  } catch (const std::bad_alloc &) {
    return fail(FS_ERR_INTERNAL, std::string(what) + ": no host memory for the check");
  }
}

fs_status too_many_tiles() { return fail(FS_ERR_UNSUPPORTED, "the product has more tiles than a launch: split the call"); }

fs_status matmul(const fs::MatmulArgs &A, hipStream_t stream) {
  const hipError_t e = fs::launch_scaled_matmul(A, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "matrix product launch");
}

// Codes and scales of the rows, counts and sums of the product's parts.
fs_status project_workspace_size(int64_t M, int64_t w_rows, int64_t K, size_t *bytes) {
  const fs_status st = fs_linear_workspace_size(M, w_rows, K, bytes);
  if (st != FS_OK) return st;
  const fs::PartsRoom parts = fs::parts_room(M, w_rows, K);
  *bytes += align256(parts.counts) + align256(parts.sums);
  return FS_OK;
}

// fs_project and fs_gated_project.
fs_status project(fs_context *ctx, const fs_norm *norm, int64_t w_rows, bool gated, fs::QuantizeArgs rows,
                  fs::MatmulArgs product, int64_t M, int64_t N, int64_t K, void *d_workspace, size_t workspace_bytes,
                  hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  size_t need = 0;
  const fs_status st = project_workspace_size(M, w_rows, K, &need);
  if (st != FS_OK) return st;
  if (!element_type((fs_dtype)rows.type) || !element_type((fs_dtype)product.out_type))
    return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (product.activation < FS_ACT_NONE || product.activation > FS_ACT_SILU)
    return fail(FS_ERR_INVALID_ARGUMENT, "unknown activation");
  if (norm && !(norm->eps >= 0x1p-80f && norm->eps <= 0x1p80f))
    return fail(FS_ERR_INVALID_ARGUMENT, "the norm's eps must be in [2^-80, 2^80]");
  if (rows.x_stride < K || product.w_stride < K || product.out_stride < N || (product.residual && product.residual_stride < N))
    return fail(FS_ERR_INVALID_ARGUMENT, "row strides must be at least the rows' lengths");
  if (M == 0 || N == 0) return FS_OK;
  if (!product.w_scale || !product.out || (K > 0 && (!rows.x || !product.w)))
    return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if (K > 0 && rows.x == product.out) return fail(FS_ERR_INVALID_ARGUMENT, "out may not be x");
  if (product.residual == product.out && product.residual_stride != product.out_stride)
    return fail(FS_ERR_INVALID_ARGUMENT, "a residual that is out must have out's stride");
  if (!d_workspace) return fail(FS_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (workspace_bytes < need)
    return fail(FS_ERR_WORKSPACE_TOO_SMALL, "workspace needs " + std::to_string(need) + " bytes");
  if ((uintptr_t)d_workspace & 15) return fail(FS_ERR_INVALID_ARGUMENT, "the workspace must start on a multiple of 16 bytes");
  if (!fs::project_fits(M, w_rows, K)) return too_many_tiles();
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  rows.codes = (int8_t *)d_workspace;
  rows.scale = (float *)(rows.codes + linear_codes(M, K));
  rows.code_stride = product.a_stride = padded(K);
  rows.rows = product.M = (int32_t)M;
  rows.cols = product.K = (int32_t)K;
  product.N = (int32_t)N;
  product.a = rows.codes;
  product.a_scale = rows.scale;
  product.a_padded = 1;
  uint8_t *const counts = (uint8_t *)rows.scale + align256(4 * (size_t)M);
  fs::plan_project(M, w_rows, K, counts, counts + align256(fs::parts_room(M, w_rows, K).counts), &rows, &product);
  if (norm) {
    rows.normed = 1;
    rows.gain = norm->gain;
    rows.eps = norm->eps;
  }
  hipError_t e = hipSuccess;
  if (fs::launch_project_few(rows, product, gated, stream, &e)) return e == hipSuccess ? FS_OK : hip_fail(e, "projection launch");
  e = norm ? fs::launch_quantize_normed(rows, stream) : fs::launch_quantize_rows(rows, stream);
  if (e != hipSuccess) return hip_fail(e, "quantize launch");
  e = fs::launch_project(product, gated, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "projection launch");
}

}  // namespace

extern "C" {

fs_status fs_quantize_rows(fs_context *ctx, const void *d_x, fs_dtype type, int64_t rows, int64_t cols,
                           int64_t x_stride, int8_t *d_codes, int64_t code_stride, float *d_scale,
                           hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  if (!element_type(type)) return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (rows < 0 || cols < 0 || rows > kMost || cols > kMost)
    return fail(FS_ERR_INVALID_ARGUMENT, "rows and cols must be in [0, 2^31)");
  if (x_stride < cols || code_stride < cols) return fail(FS_ERR_INVALID_ARGUMENT, "row strides must be at least cols");
  if (rows == 0) return FS_OK;
  if (!d_scale || (cols > 0 && (!d_x || !d_codes))) return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  const hipError_t e = fs::launch_quantize_rows(
      {d_x, d_codes, d_scale, x_stride, code_stride, (int32_t)rows, (int32_t)cols, (int32_t)type}, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "quantize launch");
}

fs_status fs_scaled_matmul_workspace_size(int64_t M, int64_t N, int64_t K, size_t *bytes) {
  if (!bytes) return fail(FS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  const fs_status st = check_product(M, N, K);
  if (st != FS_OK) return st;
  *bytes = 0;  // no product has parts
  return FS_OK;
}

fs_status fs_scaled_matmul(fs_context *ctx, const int8_t *d_a, int64_t a_stride, const float *d_a_scale,
                           const int8_t *d_w, int64_t w_stride, const float *d_w_scale, const float *d_bias,
                           int64_t M, int64_t N, int64_t K, void *d_out, fs_dtype out_type, int64_t out_stride,
                           void *, size_t, hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  const fs_status st = check_product(M, N, K);
  if (st != FS_OK) return st;
  if (!element_type(out_type)) return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (a_stride < K || w_stride < K || out_stride < N)
    return fail(FS_ERR_INVALID_ARGUMENT, "row strides must be at least the rows' lengths");
  if (M == 0 || N == 0) return FS_OK;
  if (!d_a_scale || !d_w_scale || !d_out || (K > 0 && (!d_a || !d_w)))
    return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if (!fs::matmul_fits((int32_t)M, (int32_t)N, (int32_t)K)) return too_many_tiles();
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  return matmul({d_a, d_w, d_a_scale, d_w_scale, d_bias, d_out, a_stride, w_stride, out_stride, (int32_t)M, (int32_t)N,
                 (int32_t)K, (int32_t)out_type, 0},
                stream);
}

fs_status fs_linear_workspace_size(int64_t M, int64_t N, int64_t K, size_t *bytes) {
  const fs_status st = fs_scaled_matmul_workspace_size(M, N, K, bytes);
  if (st != FS_OK) return st;
  *bytes = linear_codes(M, K) + align256(4 * (size_t)M);
  return FS_OK;
}

fs_status fs_linear(fs_context *ctx, const void *d_x, fs_dtype type, int64_t x_stride, const int8_t *d_w,
                    int64_t w_stride, const float *d_w_scale, const float *d_bias, int64_t M, int64_t N, int64_t K,
                    void *d_out, fs_dtype out_type, int64_t out_stride, void *d_workspace, size_t workspace_bytes,
                    hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  size_t need = 0;
  const fs_status st = fs_linear_workspace_size(M, N, K, &need);
  if (st != FS_OK) return st;
  if (!element_type(type) || !element_type(out_type)) return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (x_stride < K || w_stride < K || out_stride < N)
    return fail(FS_ERR_INVALID_ARGUMENT, "row strides must be at least the rows' lengths");
  if (M == 0 || N == 0) return FS_OK;
  if (!d_w_scale || !d_out || (K > 0 && (!d_x || !d_w))) return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if (!d_workspace) return fail(FS_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (workspace_bytes < need)
    return fail(FS_ERR_WORKSPACE_TOO_SMALL, "workspace needs " + std::to_string(need) + " bytes");
  if ((uintptr_t)d_workspace & 15) return fail(FS_ERR_INVALID_ARGUMENT, "the workspace must start on a multiple of 16 bytes");
  if (!fs::matmul_fits((int32_t)M, (int32_t)N, (int32_t)K)) return too_many_tiles();
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  int8_t *const codes = (int8_t *)d_workspace;
  float *const scale = (float *)(codes + linear_codes(M, K));
  const fs::QuantizeArgs rows{d_x, codes, scale, x_stride, padded(K), (int32_t)M, (int32_t)K, (int32_t)type};
  const fs::MatmulArgs product{codes, d_w, scale, d_w_scale, d_bias, d_out, padded(K), w_stride, out_stride, (int32_t)M,
                               (int32_t)N, (int32_t)K, (int32_t)out_type, 1};
  hipError_t e = hipSuccess;
  if (fs::launch_linear_few(rows, product, stream, &e))
    return e == hipSuccess ? FS_OK : hip_fail(e, "linear launch");
  e = fs::launch_quantize_rows(rows, stream);
  if (e != hipSuccess) return hip_fail(e, "quantize launch");
  return matmul(product, stream);
}

fs_status fs_project_workspace_size(int64_t M, int64_t N, int64_t K, size_t *bytes) {
  return project_workspace_size(M, N, K, bytes);
}

fs_status fs_project(fs_context *ctx, const void *d_x, fs_dtype type, int64_t x_stride, const fs_norm *norm,
                     const int8_t *d_w, int64_t w_stride, const float *d_w_scale, const float *d_bias,
                     fs_activation activation, const void *d_residual, int64_t residual_stride, int64_t M, int64_t N,
                     int64_t K, void *d_out, fs_dtype out_type, int64_t out_stride, void *d_workspace,
                     size_t workspace_bytes, hipStream_t stream) {
  fs::QuantizeArgs rows{};
  rows.x = d_x;
  rows.type = (int32_t)type;
  rows.x_stride = x_stride;
  fs::MatmulArgs product{};
  product.w = d_w;
  product.w_stride = w_stride;
  product.w_scale = d_w_scale;
  product.bias = d_bias;
  product.activation = (int32_t)activation;
  product.residual = d_residual;
  product.residual_stride = residual_stride;
  product.out = d_out;
  product.out_type = (int32_t)out_type;
  product.out_stride = out_stride;
  return project(ctx, norm, N, false, rows, product, M, N, K, d_workspace, workspace_bytes, stream);
}

fs_status fs_gated_project_workspace_size(int64_t M, int64_t N, int64_t K, size_t *bytes) {
  if (N < 0 || N > kMost / 2) return fail(FS_ERR_INVALID_ARGUMENT, "2 N must be in [0, 2^31)");
  return project_workspace_size(M, 2 * N, K, bytes);
}

fs_status fs_gated_project(fs_context *ctx, const void *d_x, fs_dtype type, int64_t x_stride, const fs_norm *norm,
                           const int8_t *d_w, int64_t w_stride, const float *d_w_scale, const float *d_bias,
                           fs_activation activation, int64_t M, int64_t N, int64_t K, void *d_out, fs_dtype out_type,
                           int64_t out_stride, void *d_workspace, size_t workspace_bytes, hipStream_t stream) {
  if (N < 0 || N > kMost / 2) return fail(FS_ERR_INVALID_ARGUMENT, "2 N must be in [0, 2^31)");
  fs::QuantizeArgs rows{};
  rows.x = d_x;
  rows.type = (int32_t)type;
  rows.x_stride = x_stride;
  fs::MatmulArgs product{};
  product.w = d_w;
  product.w_stride = w_stride;
  product.w_scale = d_w_scale;
  product.bias = d_bias;
  product.activation = (int32_t)activation;
  product.out = d_out;
  product.out_type = (int32_t)out_type;
  product.out_stride = out_stride;
  return project(ctx, norm, 2 * N, true, rows, product, M, N, K, d_workspace, workspace_bytes, stream);
}

fs_status fs_cache_append(fs_context *ctx, const fs_kv_cache *cache, const void *d_k, int64_t k_stride,
                          const void *d_v, int64_t v_stride, const void *d_q, int64_t q_stride, int32_t n_q_heads,
                          fs_dtype type, int64_t n_tokens, const int32_t *d_slots, const int32_t *d_positions,
                          const float *d_cos, const float *d_sin, int32_t n_positions, int32_t rotary_dim,
                          void *d_q_out, hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  fs_status st = check_cache(cache);
  if (st != FS_OK) return st;
  if (!element_type(type)) return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (n_tokens < 0 || n_tokens > kMost) return fail(FS_ERR_INVALID_ARGUMENT, "n_tokens must be in [0, 2^31)");
  if (rotary_dim < 0 || rotary_dim > cache->head_dim || rotary_dim % 2)
    return fail(FS_ERR_INVALID_ARGUMENT, "rotary_dim must be even and in [0, head_dim]");
  const int64_t width = (int64_t)cache->n_heads * cache->head_dim;
  if (k_stride < width || v_stride < width)
    return fail(FS_ERR_INVALID_ARGUMENT, "token strides must be at least the rows' lengths");
  if (d_q) {
    if (n_q_heads < 1 || n_q_heads > 65536) return fail(FS_ERR_INVALID_ARGUMENT, "n_q_heads must be in [1, 65536]");
    if (q_stride < (int64_t)n_q_heads * cache->head_dim)
      return fail(FS_ERR_INVALID_ARGUMENT, "token strides must be at least the rows' lengths");
    if (!d_q_out && n_tokens > 0) return fail(FS_ERR_INVALID_ARGUMENT, "q_out is NULL");
  }
  if (n_tokens == 0) return FS_OK;
  st = check_cache_memory(cache);
  if (st != FS_OK) return st;
  if (!d_k || !d_v || !d_slots) return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if (rotary_dim && (!d_positions || !d_cos || !d_sin || n_positions < 1))
    return fail(FS_ERR_INVALID_ARGUMENT, "a rotation needs positions and tables");
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  const fs::Cache c = to_cache(cache);
  if (fs::env_validate()) {
    st = checked(
        [&](int32_t *flag) {
          return fs::launch_check_slots(c, d_slots, rotary_dim ? d_positions : nullptr, n_positions, (int32_t)n_tokens,
                                        1, flag, stream);
        },
        stream, "fs_cache_append", {"slots outside the cache", "positions outside the tables"});
    if (st == FS_OK) st = check_pages(c, d_slots, n_tokens, stream, "fs_cache_append");
    if (st != FS_OK) return st;
  }
  const hipError_t e = fs::launch_cache_append(
      {c, d_k, d_v, d_q, d_q_out, d_slots, d_positions, d_cos, d_sin, k_stride, v_stride, q_stride, (int32_t)n_tokens,
       d_q ? n_q_heads : 0, (int32_t)type, n_positions, rotary_dim / 2},
      stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "append launch");
}

fs_status fs_cache_read(fs_context *ctx, const fs_kv_cache *cache, int64_t n_tokens, const int32_t *d_slots,
                        void *d_k_out, void *d_v_out, fs_dtype type, hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  fs_status st = check_cache(cache);
  if (st != FS_OK) return st;
  if (!element_type(type)) return fail(FS_ERR_INVALID_ARGUMENT, "unknown element type");
  if (n_tokens < 0 || n_tokens > kMost) return fail(FS_ERR_INVALID_ARGUMENT, "n_tokens must be in [0, 2^31)");
  if (n_tokens == 0 || (!d_k_out && !d_v_out)) return FS_OK;
  st = check_cache_memory(cache);
  if (st != FS_OK) return st;
  if (!d_slots) return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  const fs::Cache c = to_cache(cache);
  if (fs::env_validate()) {
    st = checked(
        [&](int32_t *flag) {
          return fs::launch_check_slots(c, d_slots, nullptr, 0, (int32_t)n_tokens, 0, flag, stream);
        },
        stream, "fs_cache_read", {"slots outside the cache", ""});
    if (st != FS_OK) return st;
  }
  const hipError_t e =
      fs::launch_cache_read({c, d_slots, d_k_out, d_v_out, (int32_t)n_tokens, (int32_t)type}, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "cache read launch");
}

static fs_status check_heads(const fs_kv_cache *cache, int32_t n_q_heads, int64_t n_tokens, int32_t n_seqs) {
  const fs_status st = check_cache(cache);
  if (st != FS_OK) return st;
  if (n_q_heads < 1 || n_q_heads % cache->n_heads)
    return fail(FS_ERR_INVALID_ARGUMENT, "n_q_heads must be a positive multiple of the cache's heads");
  if (n_q_heads > 65536 / 2) return fail(FS_ERR_UNSUPPORTED, "n_q_heads must be at most 32768");
  if (n_tokens < 0 || n_tokens > kMost || n_tokens * n_q_heads > kMost)
    return fail(FS_ERR_INVALID_ARGUMENT, "n_tokens * n_q_heads must be in [0, 2^31)");
  if (n_seqs < 0) return fail(FS_ERR_INVALID_ARGUMENT, "n_seqs must be >= 0");
  if (n_seqs > FS_MAX_SEQUENCES)
    return fail(FS_ERR_UNSUPPORTED, "n_seqs must be at most " + std::to_string(FS_MAX_SEQUENCES));
  return FS_OK;
}

fs_status fs_cache_attention_workspace_size(const fs_kv_cache *cache, int32_t n_q_heads, int64_t n_tokens,
                                            int32_t n_seqs, size_t *bytes) {
  if (!bytes) return fail(FS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  const fs_status st = check_heads(cache, n_q_heads, n_tokens, n_seqs);
  if (st != FS_OK) return st;
  *bytes = align256(fs::attention_workspace(to_cache(cache), n_q_heads, n_tokens, n_seqs));
  return FS_OK;
}

fs_status fs_cache_attention(fs_context *ctx, const fs_kv_cache *cache, const void *d_q, int64_t q_stride,
                             fs_dtype type, int32_t n_q_heads, int64_t n_tokens, int32_t n_seqs,
                             const int32_t *d_cu_q, const int32_t *d_ctx_lens, const int32_t *d_block_table,
                             int64_t table_width, int32_t max_q, float scale, int32_t window, void *d_out,
                             void *d_workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  size_t need = 0;
  fs_status st = fs_cache_attention_workspace_size(cache, n_q_heads, n_tokens, n_seqs, &need);
  if (st != FS_OK) return st;
  if (type != FS_F16 && type != FS_BF16) return fail(FS_ERR_UNSUPPORTED, "queries must be FS_F16 or FS_BF16");
  if (q_stride < (int64_t)n_q_heads * cache->head_dim)
    return fail(FS_ERR_INVALID_ARGUMENT, "token strides must be at least the rows' lengths");
  if (table_width < 0 || table_width > kMost) return fail(FS_ERR_INVALID_ARGUMENT, "table_width must be in [0, 2^31)");
  if (max_q < 0) return fail(FS_ERR_INVALID_ARGUMENT, "max_q must be >= 0");
  if (window < 0) return fail(FS_ERR_INVALID_ARGUMENT, "window must be >= 0");
  if (!std::isfinite(scale)) return fail(FS_ERR_INVALID_ARGUMENT, "scale must be finite");
  if (n_tokens == 0 || n_seqs == 0) return FS_OK;
  st = check_cache_memory(cache);
  if (st != FS_OK) return st;
  if (!d_q || !d_cu_q || !d_ctx_lens || !d_out || (table_width > 0 && !d_block_table))
    return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if (need && !d_workspace) return fail(FS_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (workspace_bytes < need)
    return fail(FS_ERR_WORKSPACE_TOO_SMALL, "workspace needs " + std::to_string(need) + " bytes");
  if ((uintptr_t)d_workspace & 15) return fail(FS_ERR_INVALID_ARGUMENT, "the workspace must start on a multiple of 16 bytes");
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  const int32_t group = n_q_heads / cache->n_heads;
  const fs::AttendArgs A{to_cache(cache), d_q, d_out, d_cu_q, d_ctx_lens, d_block_table, q_stride, table_width,
                         (int32_t)n_tokens, n_seqs, n_q_heads, max_q, window, (int32_t)type, scale,
                         (uint32_t)((0x100000000ull + (uint64_t)group - 1) / (uint64_t)group)};
  if (!fs::attention_fits(A, ctx->attention))
    return fail(FS_ERR_UNSUPPORTED, "more than 2^31 tiles of rows and tokens: split the call");
  if (fs::env_validate()) {
    st = checked([&](int32_t *flag) { return fs::launch_check_attention(A, flag, stream); }, stream,
                 "fs_cache_attention", {"sequences with lengths out of range", "pages outside the cache"});
    if (st != FS_OK) return st;
  }
  const hipError_t e = fs::launch_cache_attention(A, ctx->attention, d_workspace, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "attention launch");
}

static fs_status check_pool(const fs_state_pool *pool, int32_t n_q_heads, int64_t n_tokens, int32_t n_seqs) {
  if (!pool) return fail(FS_ERR_INVALID_ARGUMENT, "pool is NULL");
  if (pool->n_states < 0 || pool->n_heads < 1)
    return fail(FS_ERR_INVALID_ARGUMENT, "the pool's heads must be positive (n_states >= 0)");
  if (pool->head_dim != 64 && pool->head_dim != 128) return fail(FS_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (pool->n_heads > 4096) return fail(FS_ERR_UNSUPPORTED, "n_heads must be at most 4096");
  if (n_q_heads < 1 || n_q_heads % pool->n_heads)
    return fail(FS_ERR_INVALID_ARGUMENT, "n_q_heads must be a positive multiple of the pool's heads");
  if (n_q_heads > 65536 / 2) return fail(FS_ERR_UNSUPPORTED, "n_q_heads must be at most 32768");
  if (n_tokens < 0 || n_tokens > kMost || n_tokens * n_q_heads > kMost)
    return fail(FS_ERR_INVALID_ARGUMENT, "n_tokens * n_q_heads must be in [0, 2^31)");
  if (n_seqs < 0) return fail(FS_ERR_INVALID_ARGUMENT, "n_seqs must be >= 0");
  if (n_seqs > FS_MAX_SEQUENCES)
    return fail(FS_ERR_UNSUPPORTED, "n_seqs must be at most " + std::to_string(FS_MAX_SEQUENCES));
  return FS_OK;
}

fs_status fs_state_attention_workspace_size(const fs_state_pool *pool, int32_t n_q_heads, int64_t n_tokens,
                                            int32_t n_seqs, size_t *bytes) {
  if (!bytes) return fail(FS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  const fs_status st = check_pool(pool, n_q_heads, n_tokens, n_seqs);
  if (st != FS_OK) return st;
  *bytes = align256(fs::state_workspace(pool->n_heads, pool->head_dim, n_tokens, n_seqs));
  return FS_OK;
}

fs_status fs_state_attention(fs_context *ctx, const fs_state_pool *pool, const void *d_q, int64_t q_stride,
                             const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride, fs_dtype type,
                             int32_t n_q_heads, int64_t n_tokens, int32_t n_seqs, const int32_t *d_cu_q,
                             const int32_t *d_ctx_lens, const int32_t *d_state_index, int32_t max_q,
                             const float *d_log_decay, float scale, void *d_out, void *d_workspace,
                             size_t workspace_bytes, hipStream_t stream) {
  if (!ctx) return fail(FS_ERR_INVALID_ARGUMENT, "context is NULL");
  size_t need = 0;
  fs_status st = fs_state_attention_workspace_size(pool, n_q_heads, n_tokens, n_seqs, &need);
  if (st != FS_OK) return st;
  if (type != FS_F16 && type != FS_BF16) return fail(FS_ERR_UNSUPPORTED, "queries, keys and values must be FS_F16 or FS_BF16");
  const int64_t width = (int64_t)pool->n_heads * pool->head_dim;
  if (q_stride < (int64_t)n_q_heads * pool->head_dim || k_stride < width || v_stride < width)
    return fail(FS_ERR_INVALID_ARGUMENT, "token strides must be at least the rows' lengths");
  if (max_q < 0) return fail(FS_ERR_INVALID_ARGUMENT, "max_q must be >= 0");
  if (!std::isfinite(scale)) return fail(FS_ERR_INVALID_ARGUMENT, "scale must be finite");
  if (n_tokens == 0 || n_seqs == 0 || max_q == 0) return FS_OK;
  if (!d_q || !d_k || !d_v || !d_cu_q || !d_ctx_lens || !d_state_index || !d_log_decay || !d_out ||
      (pool->n_states > 0 && !pool->s))
    return fail(FS_ERR_INVALID_ARGUMENT, "array is NULL");
  if ((uintptr_t)pool->s & 15) return fail(FS_ERR_INVALID_ARGUMENT, "the pool must start on a multiple of 16 bytes");
  if (need && !d_workspace) return fail(FS_ERR_INVALID_ARGUMENT, "workspace is NULL");
  if (workspace_bytes < need)
    return fail(FS_ERR_WORKSPACE_TOO_SMALL, "workspace needs " + std::to_string(need) + " bytes");
  if ((uintptr_t)d_workspace & 15) return fail(FS_ERR_INVALID_ARGUMENT, "the workspace must start on a multiple of 16 bytes");
  DeviceGuard dg(ctx->device);
  if (dg.err != hipSuccess) return hip_fail(dg.err, "hipSetDevice");
  const fs::StateArgs A{pool->s,      d_q,          d_k,           d_v,      d_out,          d_cu_q,
                        d_ctx_lens,   d_state_index, d_log_decay,  (float *)d_workspace,     q_stride,
                        k_stride,     v_stride,     pool->n_states, pool->n_heads,           pool->head_dim,
                        n_q_heads,    (int32_t)n_tokens, n_seqs,   max_q,    (int32_t)type,  scale,
                        0,            0,            0};
  if (fs::env_validate()) {
    st = checked([&](int32_t *flag) { return fs::launch_check_state(A, flag, stream); }, stream, "fs_state_attention",
                 {"sequences with lengths or states out of range", "decays that are not at most 0"});
    if (st != FS_OK) return st;
  }
  const hipError_t e = fs::launch_state_attention(A, stream);
  return e == hipSuccess ? FS_OK : hip_fail(e, "state attention launch");
}

}  // extern "C"
