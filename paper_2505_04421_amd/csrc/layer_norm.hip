// Layer norm of token rows and its backward pass (longer_layer_norm, longer_layer_norm_backward): argument checks and dispatch.
#include "layer_norm.h"

#include <algorithm>
#include <cfloat>

namespace longer {
namespace ln {

// out[c] = sum over the workgroups of part[.][c], 32 columns a workgroup, 32 shares of the sum in a fixed order.  Latency for narrow rows (2
// us), memory for wide ones (6 us at width 8191, 17 MB).
__global__ __launch_bounds__(1024) void join_kernel(const float* part, int slices, int n, float* out) {
  __shared__ float lds[32][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), share = threadIdx.x >> 5;
  float s = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int i = share; i < slices; i += 32) s += part[(size_t)i * n + c];
  }
  lds[share][threadIdx.x & 31] = s;
  __syncthreads();
  if (share || c >= n) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += lds[i][threadIdx.x];
  out[c] = s;
}

// ------------------------------------------------------------------------------------ host
constexpr int kGradGroups = 512;                    // most workgroups of a backward launch: two for each compute unit

static int check_sizes(int B, int L, int d) {
  if (B <= 0 || L <= 0 || (int64_t)B * L >= ((int64_t)1 << 31) - (1 << 21)) return api_error(LONGER_ERR_ARG, "B=%d L=%d: at least 1 each, B * L below 2^31 - 2^21", B, L);
  if (d <= 0 || d > LONGER_MAX_NORM_WIDTH) return api_error(LONGER_ERR_ARG, "d=%d: 1 to %d", d, LONGER_MAX_NORM_WIDTH);
  return 0;
}

// column sums of every workgroup (of one alone: in their place at once)
static size_t workspace_bytes(int B, int L, int d) {
  return ((size_t)std::min<int64_t>((int64_t)B * L, kGradGroups) * 2 * d * 4 + 255) & ~(size_t)255;
}

static int size_of(int dtype) { return dtype == LONGER_F32 ? 4 : dtype == LONGER_BF16 ? 2 : 0; }

static int check_rows(const longer_rows* r, const char* name, int B, int L, int d, bool written) {
  if (!r || !r->data) return api_error(LONGER_ERR_ARG, "%s is NULL", name);
  const int e = size_of(r->dtype);
  if (!e) return api_error(LONGER_ERR_ARG, "%s: dtype %d unknown", name, r->dtype);
  if ((uintptr_t)r->data % e) return api_error(LONGER_ERR_ARG, "%s is not aligned to its elements", name);
  const int64_t su = r->user_stride, sr = r->row_stride, most = (int64_t)1 << 40;
  if ((B > 1 && (su < 0 || su > most)) || (L > 1 && (sr < 0 || sr > most))) return api_error(LONGER_ERR_ARG, "%s: strides %lld, %lld out of range", name, (long long)su, (long long)sr);
  if (written) {
    // users apart and rows apart inside one user, or the other way round
    const bool rows_inside = (L == 1 || sr >= d) && (B == 1 || su >= (__int128)(L - 1) * (L > 1 ? sr : 0) + d);
    const bool users_inside = (B == 1 || su >= d) && (L == 1 || sr >= (__int128)(B - 1) * (B > 1 ? su : 0) + d);
    if (!rows_inside && !users_inside) return api_error(LONGER_ERR_ARG, "%s: rows of an output overlap (strides %lld, %lld)", name, (long long)su, (long long)sr);
  }
  return 0;
}

static Rows rows_of(const longer_rows* r, int B, int L) { return {(char*)r->data, B > 1 ? r->user_stride : 0, L > 1 ? r->row_stride : 0}; }

static bool same(const longer_rows* a, const longer_rows* b, int B, int L) {
  return a->data == b->data && a->dtype == b->dtype && (B == 1 || a->user_stride == b->user_stride) && (L == 1 || a->row_stride == b->row_stride);
}


// An output's buffer may hold other rows between its own (those of another tensor too), so extents that cross say
// nothing; equal first values under another layout do.
static int check_alias(const longer_rows* in, const longer_rows* out, const char* what, int B, int L) {
  if (in->data == out->data && !same(in, out, B, L)) return api_error(LONGER_ERR_ARG, "%s: the same memory under other strides or types", what);
  return 0;
}

static int check_vector(const void* p, int dtype, const char* name) {
  if (!p) return api_error(LONGER_ERR_ARG, "%s is NULL", name);
  if ((uintptr_t)p % size_of(dtype)) return api_error(LONGER_ERR_ARG, "%s is not aligned to its elements", name);
  return 0;
}

static int launched(const char* what) {
  return hipGetLastError() == hipSuccess ? 0 : api_error(LONGER_ERR_HIP, "%s launch failed", what);
}

}  // namespace ln
}  // namespace longer

using namespace longer;

extern "C" {

int longer_layer_norm(const longer_rows* x, const void* ln_g, const void* ln_b, const int32_t* lens,
                      int B, int L, int d, float eps, const longer_rows* y, void* stream) {
  int rc = ln::check_sizes(B, L, d);
  if (!rc) rc = ln::check_rows(x, "x", B, L, d, false);
  if (!rc) rc = ln::check_rows(y, "y", B, L, d, true);
  if (!rc) rc = ln::check_vector(ln_g, x->dtype, "ln_g");
  if (!rc) rc = ln::check_vector(ln_b, x->dtype, "ln_b");
  if (!rc && x->dtype != y->dtype) rc = api_error(LONGER_ERR_ARG, "x and y have one dtype");
  if (!rc) rc = ln::check_alias(x, y, "x and y", B, L);
  if (!rc && !(eps >= FLT_MIN && eps <= FLT_MAX)) rc = api_error(LONGER_ERR_ARG, "eps must be positive (a normal number)");
  if (!rc && ((uintptr_t)lens & 3)) rc = api_error(LONGER_ERR_ARG, "lens is not aligned");
  if (rc) return rc;
  ln::Params p = {ln::rows_of(x, B, L), {}, ln::rows_of(y, B, L), ln_g, ln_b, lens, B * L, L, d, 0, 0, 0, eps, 1.f / d, nullptr};
  if (x->dtype == LONGER_F32) ln::norm_f32(p, (hipStream_t)stream);
  else ln::norm_bf16(p, (hipStream_t)stream);
  return ln::launched("layer norm");
}

size_t longer_layer_norm_backward_workspace_bytes(int B, int L, int d) {
  return ln::check_sizes(B, L, d) ? 0 : ln::workspace_bytes(B, L, d);
}

int longer_layer_norm_backward(const longer_rows* x, const void* ln_g, const longer_rows* dy, const int32_t* lens,
                               int B, int L, int d, float eps, const longer_rows* dx, float* grads_out,
                               void* ws, size_t ws_bytes, void* stream) {
  int rc = ln::check_sizes(B, L, d);
  if (!rc) rc = ln::check_rows(x, "x", B, L, d, false);
  if (!rc) rc = ln::check_rows(dy, "dy", B, L, d, false);
  if (!rc) rc = ln::check_rows(dx, "dx", B, L, d, true);
  if (!rc) rc = ln::check_vector(ln_g, x->dtype, "ln_g");
  if (!rc) rc = ln::check_vector(grads_out, LONGER_F32, "grads_out");
  if (!rc && (dy->dtype != dx->dtype || (dy->dtype != LONGER_F32 && dy->dtype != x->dtype)))
    rc = api_error(LONGER_ERR_ARG, "dy and dx are both fp32 or both of x's dtype");
  if (!rc) rc = ln::check_alias(dy, dx, "dy and dx", B, L);
  if (!rc && x->data == dx->data) rc = api_error(LONGER_ERR_ARG, "dx may not be x");
  if (!rc && !(eps >= FLT_MIN && eps <= FLT_MAX)) rc = api_error(LONGER_ERR_ARG, "eps must be positive (a normal number)");
  if (!rc && ((uintptr_t)lens & 3)) rc = api_error(LONGER_ERR_ARG, "lens is not aligned");
  if (!rc && (!ws || ((uintptr_t)ws & 255))) rc = api_error(LONGER_ERR_ARG, "ws must be 256-byte aligned and not NULL");
  if (rc) return rc;
  const size_t need = ln::workspace_bytes(B, L, d);
  if (ws_bytes < need) return api_error(LONGER_ERR_WS, "workspace too small: %zu < %zu bytes", ws_bytes, need);
  ln::Params p = {ln::rows_of(x, B, L), ln::rows_of(dy, B, L), ln::rows_of(dx, B, L), ln_g, nullptr, lens, B * L, L, d, 0, 0, 0, eps, 1.f / d,
                  (float*)ws};
  hipStream_t st = (hipStream_t)stream;
  const unsigned groups = x->dtype == LONGER_F32 ? ln::grad_f32(p, ln::kGradGroups, grads_out, st)
                          : dy->dtype == LONGER_F32 ? ln::grad_bf16_f32(p, ln::kGradGroups, grads_out, st)
                                                    : ln::grad_bf16(p, ln::kGradGroups, grads_out, st);
  if (groups > 1) ln::join_kernel<<<(2 * d + 31) / 32, 1024, 0, st>>>((const float*)ws, (int)groups, 2 * d, grads_out);
  return ln::launched("layer norm gradient");
}

}  // extern "C"
