// Layer norm of token rows and its backward pass (longer_layer_norm, longer_layer_norm_backward).
#include "../../include/longer.h"
#include "device.h"

namespace longer {

int api_error(int code, const char* fmt, ...);   // longer_api.hip

namespace ln {

struct Rows { char* data; int64_t user, row; };      // strides in elements

struct Params {
  Rows x, dy, out;                  // out: y, or dx
  const void *g, *b;
  const int32_t* lens;
  int rows, L, d;
  float eps;
  float* stats;                     // [rows][2], mean and 1 / sqrt(var + eps)
};

template <typename T> __device__ __forceinline__ T* row_of(const Rows& r, int u, int l) { return (T*)r.data + u * r.user + l * r.row; }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// a wave per row
template <typename T>
__global__ __launch_bounds__(256) void norm_kernel(Params p) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= p.rows) return;
  const int u = r / p.L, l = r - u * p.L;
  T* y = row_of<T>(p.out, u, l);
  if (p.lens && l >= p.lens[u]) {
    for (int c = lane; c < p.d; c += 64) y[c] = (T)0.f;
    return;
  }
  const T* x = row_of<T>(p.x, u, l);
  float s = 0.f;
  for (int c = lane; c < p.d; c += 64) s += (float)x[c];
  const float mean = wave_sum(s) / p.d;
  s = 0.f;
  for (int c = lane; c < p.d; c += 64) { const float v = (float)x[c] - mean; s += v * v; }
  const float rs = 1.f / sqrtf(wave_sum(s) / p.d + p.eps);
  for (int c = lane; c < p.d; c += 64) y[c] = (T)(((float)x[c] - mean) * rs * (float)((const T*)p.g)[c] + (float)((const T*)p.b)[c]);
}

template <typename T>
__global__ __launch_bounds__(256) void stats_kernel(Params p) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= p.rows) return;
  const int u = r / p.L, l = r - u * p.L;
  if (p.lens && l >= p.lens[u]) return;
  const T* x = row_of<T>(p.x, u, l);
  float s = 0.f;
  for (int c = lane; c < p.d; c += 64) s += (float)x[c];
  const float mean = wave_sum(s) / p.d;
  s = 0.f;
  for (int c = lane; c < p.d; c += 64) { const float v = (float)x[c] - mean; s += v * v; }
  const float rs = 1.f / sqrtf(wave_sum(s) / p.d + p.eps);
  if (lane == 0) { p.stats[2 * (size_t)r] = mean; p.stats[2 * (size_t)r + 1] = rs; }
}

// (after the column sums: dx may be dy)
template <typename T, typename U>
__global__ __launch_bounds__(256) void grad_kernel(Params p) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= p.rows) return;
  const int u = r / p.L, l = r - u * p.L;
  U* dx = row_of<U>(p.out, u, l);
  if (p.lens && l >= p.lens[u]) {
    for (int c = lane; c < p.d; c += 64) dx[c] = (U)0.f;
    return;
  }
  const T* x = row_of<T>(p.x, u, l);
  const U* dy = row_of<U>(p.dy, u, l);
  const float mean = p.stats[2 * (size_t)r], rs = p.stats[2 * (size_t)r + 1];
  float q1 = 0.f, q2 = 0.f;
  for (int c = lane; c < p.d; c += 64) {
    const float q = (float)dy[c] * (float)((const T*)p.g)[c];
    q1 += q;
    q2 += q * (((float)x[c] - mean) * rs);
  }
  q1 = wave_sum(q1) / p.d;
  q2 = wave_sum(q2) / p.d;
  for (int c = lane; c < p.d; c += 64) {
    const float q = (float)dy[c] * (float)((const T*)p.g)[c];
    dx[c] = (U)(rs * (q - q1 - (((float)x[c] - mean) * rs) * q2));
  }
}

// column sums over a slice of the rows: a lane per column, a wave per row
template <typename T, typename U>
__global__ __launch_bounds__(256) void param_kernel(Params p, float* part) {
  __shared__ float sum[2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float dg = 0.f, db = 0.f;
  for (int r = blockIdx.y * 4 + wave; r < p.rows; r += gridDim.y * 4) {
    const int u = r / p.L, l = r - u * p.L;
    if ((p.lens && l >= p.lens[u]) || c >= p.d) continue;
    const float dy = (float)row_of<U>(p.dy, u, l)[c];
    dg += dy * (((float)row_of<T>(p.x, u, l)[c] - p.stats[2 * (size_t)r]) * p.stats[2 * (size_t)r + 1]);
    db += dy;
  }
  sum[0][wave][lane] = dg;
  sum[1][wave][lane] = db;
  __syncthreads();
  if (wave < 2 && c < p.d) {
    float s = 0.f;
    for (int w = 0; w < 4; ++w) s += sum[wave][w][lane];
    part[((size_t)blockIdx.y * 2 + wave) * p.d + c] = s;
  }
}

__global__ __launch_bounds__(256) void join_kernel(const float* part, int slices, int n, float* out) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n) return;
  float s = 0.f;
  for (int i = 0; i < slices; ++i) s += part[(size_t)i * n + c];
  out[c] = s;
}

// ------------------------------------------------------------------------------------ host
constexpr int kSlices = 64;

struct Workspace { size_t stats, part, total; };
static Workspace workspace(int B, int L, int d) {
  Workspace w;
  w.stats = 0;
  w.part = ((size_t)B * L * 8 + 255) & ~(size_t)255;
  w.total = (w.part + (size_t)kSlices * 2 * d * 4 + 255) & ~(size_t)255;
  return w;
}

static int check_sizes(int B, int L, int d) {
  if (B <= 0 || L <= 0 || (int64_t)B * L >= ((int64_t)1 << 31)) return api_error(LONGER_ERR_ARG, "B=%d L=%d: at least 1 each, B * L below 2^31", B, L);
  if (d <= 0 || d > LONGER_MAX_NORM_WIDTH) return api_error(LONGER_ERR_ARG, "d=%d: 1 to %d", d, LONGER_MAX_NORM_WIDTH);
  return 0;
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

template <typename T, typename U>
static int backward(const Params& p, float* part, float* grads, hipStream_t st) {
  const unsigned grid = (unsigned)(((int64_t)p.rows + 3) / 4);
  stats_kernel<T><<<grid, 256, 0, st>>>(p);
  param_kernel<T, U><<<dim3((p.d + 63) / 64, kSlices), 256, 0, st>>>(p, part);
  join_kernel<<<(2 * p.d + 255) / 256, 256, 0, st>>>(part, kSlices, 2 * p.d, grads);
  grad_kernel<T, U><<<grid, 256, 0, st>>>(p);
  return launched("layer norm gradient");
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
  if (!rc && !(eps > 0.f)) rc = api_error(LONGER_ERR_ARG, "eps must be positive");
  if (!rc && ((uintptr_t)lens & 3)) rc = api_error(LONGER_ERR_ARG, "lens is not aligned");
  if (rc) return rc;
  const ln::Params p = {ln::rows_of(x, B, L), {}, ln::rows_of(y, B, L), ln_g, ln_b, lens, B * L, L, d, eps, nullptr};
  const unsigned grid = (unsigned)(((int64_t)B * L + 3) / 4);
  if (x->dtype == LONGER_F32) ln::norm_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(p);
  else ln::norm_kernel<__bf16><<<grid, 256, 0, (hipStream_t)stream>>>(p);
  return ln::launched("layer norm");
}

size_t longer_layer_norm_backward_workspace_bytes(int B, int L, int d) {
  return ln::check_sizes(B, L, d) ? 0 : ln::workspace(B, L, d).total;
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
  if (!rc && !(eps > 0.f)) rc = api_error(LONGER_ERR_ARG, "eps must be positive");
  if (!rc && ((uintptr_t)lens & 3)) rc = api_error(LONGER_ERR_ARG, "lens is not aligned");
  if (!rc && (!ws || ((uintptr_t)ws & 255))) rc = api_error(LONGER_ERR_ARG, "ws must be 256-byte aligned and not NULL");
  if (rc) return rc;
  const ln::Workspace w = ln::workspace(B, L, d);
  if (ws_bytes < w.total) return api_error(LONGER_ERR_WS, "workspace too small: %zu < %zu bytes", ws_bytes, w.total);
  const ln::Params p = {ln::rows_of(x, B, L), ln::rows_of(dy, B, L), ln::rows_of(dx, B, L), ln_g, nullptr, lens, B * L, L, d, eps,
                        (float*)((char*)ws + w.stats)};
  float* part = (float*)((char*)ws + w.part);
  hipStream_t st = (hipStream_t)stream;
  if (x->dtype == LONGER_F32) return ln::backward<float, float>(p, part, grads_out, st);
  if (dy->dtype == LONGER_F32) return ln::backward<__bf16, float>(p, part, grads_out, st);
  return ln::backward<__bf16, __bf16>(p, part, grads_out, st);
}

}  // extern "C"
