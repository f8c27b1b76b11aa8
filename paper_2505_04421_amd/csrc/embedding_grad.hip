// Gradient of a table of embeddings by sorted tokens (longer_embedding_backward).
//
// The order's tokens are cut into ranges of S.  A group of lanes takes a range (and a chunk of at most 512 columns, 8 a lane) and adds up
// its rows of dE in registers, one run after the other; where a run ends, its row is complete and goes out, scaled once.  A run that
// crosses ranges leaves a sum in each: [range][0] the run that began earlier, [range][1] the one that begins in the range and goes on;
// the join adds them up in order, in the range where the run begins.
#include "embedding.h"

namespace longer {
namespace emb {

constexpr int kChunk = 512;                          // columns of a group: 64 lanes of 8

struct GradParams {
  Rows de;
  Divider by_L;
  uint32_t n, L;                                     // tokens of the batch
  int d, shift, chunks;
  uint32_t range;                                    // S
  float factor;
  Mask mask;
  longer_order order;
  int dense;
  uint32_t out_rows;
  float *grads, *norms;
  float* part;                                       // [ranges][2][d]
  double* squares;                                   // [runs][chunks], where there is more than one chunk
};

__device__ __forceinline__ uint32_t tokens_of(const GradParams& p) { return min((uint32_t)max(p.order.counts[1], 0), p.n); }

__device__ __forceinline__ void store_sums(float* to, int n, const float (&a)[8]) {
  Piece<float, 8> v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = a[j];
  if (n >= 8) *(Piece<float, 8>*)to = v;
  else
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < n) to[j] = v[j];
}

// A run's sums are complete: its row, and its norm's squares.  All lanes of the group are here.
__device__ __forceinline__ void finish(const GradParams& p, uint32_t run, int c, int chunk, int lane, const float (&acc)[8]) {
  const uint32_t row = p.dense ? (uint32_t)p.order.rows[run] : run;
  if (row >= p.out_rows) return;
  float g[8];
  double s = 0.;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] = c + j < p.d ? p.factor * acc[j] : 0.f;
    s = fma((double)g[j], (double)g[j], s);
  }
  if (c < p.d) store_sums(p.grads + (size_t)row * p.d + c, p.d - c, g);
  if (!p.norms) return;
  for (int o = 1; o < 1 << p.shift; o *= 2) s += __shfl_xor(s, o);
  if (lane == 0) {
    if (p.chunks == 1) p.norms[row] = (float)sqrt(s);
    else p.squares[(size_t)run * p.chunks + chunk] = s;
  }
}

template <typename T, bool DROP>
__global__ __launch_bounds__(256) void grad_kernel(GradParams p) {
  constexpr int U = 8;
  const int lanes = 1 << p.shift, lane = threadIdx.x & (lanes - 1), chunk = blockIdx.y, c = chunk * kChunk + lane * 8, width = p.d - c;
  const uint32_t n = tokens_of(p), range = blockIdx.x * (256 >> p.shift) + (threadIdx.x >> p.shift);
  const uint64_t from = (uint64_t)range * p.range;
  if (from >= n) return;
  const uint32_t begin = (uint32_t)from, end = min(begin + p.range, n);
  const Key key = DROP ? load_key(p.mask) : Key{};
  float acc[8] = {};
  int run = p.order.runs[begin];
  bool earlier = begin && p.order.runs[begin - 1] == run;
  float* part = p.part + (size_t)range * 2 * p.d + c;
  for (uint32_t at = begin; at < end; at += U) {
    uint32_t token[U];
    int runs[U];
    Piece<T, 8> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = at + u < end;
      token[u] = in ? (uint32_t)p.order.tokens[at + u] : p.n;
      runs[u] = in ? p.order.runs[at + u] : run;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (token[u] < p.n && width > 0) {
        const uint32_t b = p.by_L(token[u]), l = token[u] - b * p.L;
        x[u] = load8((const T*)p.de.data + (int64_t)b * p.de.user + (int64_t)l * p.de.row + c, width);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at + u >= end) break;
      if (runs[u] != run) {
        if (earlier) { if (width > 0) store_sums(part, width, acc); }
        else finish(p, run, c, chunk, lane, acc);
        run = runs[u];
        earlier = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
      }
      if (token[u] < p.n && width > 0) {
        Piece<float, 8> y;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = (float)x[u][j];
        if (DROP) drop8(p.mask, key, token[u], c / 8, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += y[j];
      }
    }
  }
  const bool on = end < n && p.order.runs[end] == run;
  if (earlier) { if (width > 0) store_sums(part, width, acc); }
  else if (on) { if (width > 0) store_sums(part + p.d, width, acc); }
  else finish(p, run, c, chunk, lane, acc);
}

constexpr int kJoinThreads = 1024, kJoinAlone = 32;

// The runs that cross ranges, each by the group whose range it begins in, and by the whole workgroup where it crosses more than
// kJoinAlone: group k takes every groups-th of its sums, which then meet in pairs.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(GradParams p) {
  __shared__ float lds[kJoinThreads * 8];
  __shared__ uint32_t list[kJoinThreads][2], listed;
  const int lanes = 1 << p.shift, lane = threadIdx.x & (lanes - 1), chunk = blockIdx.y, c = chunk * kChunk + lane * 8, width = p.d - c;
  const uint32_t group = threadIdx.x >> p.shift, groups = kJoinThreads >> p.shift, n = tokens_of(p);
  const int32_t* runs = p.order.runs;
  const uint32_t ranges = (n + p.range - 1) / p.range;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  const uint32_t g = blockIdx.x * groups + group;
  uint32_t last = 0;                                 // the last range that the run of this one reaches (0: it ends here, or began earlier)
  if (g + 1 < ranges) {
    const uint32_t begin = g * p.range, end = begin + p.range;
    const int run = runs[end];
    if (runs[end - 1] == run && !(begin && runs[begin - 1] == run)) {
      uint32_t lo = g + 1, hi = ranges - 1;          // runs ascend: the last range that begins with it
      while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (runs[(size_t)mid * p.range] == run) lo = mid;
        else hi = mid - 1;
      }
      last = lo;
    }
  }
  const size_t step = (size_t)2 * p.d;
  float acc[8] = {};
  if (last && last - g <= kJoinAlone) {
    if (width > 0) {
      const float* at = p.part + g * step + c;
      Piece<float, 8> x = load8(at + p.d, width);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = x[j];
      for (uint32_t h = g + 1; h <= last; ++h) {
        x = load8(p.part + h * step + c, width);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += x[j];
      }
    }
    finish(p, runs[(size_t)last * p.range], c, chunk, lane, acc);
  }
  if (last && last - g > kJoinAlone && lane == 0) {
    const uint32_t i = atomicAdd(&listed, 1u);       // (the order of the list is that of the work alone)
    list[i][0] = g;
    list[i][1] = last;
  }
  __syncthreads();
  for (uint32_t i = 0; i < listed; ++i) {
    const uint32_t a = list[i][0], b = list[i][1];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (width > 0)
      for (uint32_t h = a + group; h <= b; h += groups) {
        const Piece<float, 8> x = load8(p.part + h * step + (h == a ? p.d : 0) + c, width);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += x[j];
      }
    for (uint32_t half = groups / 2; half; half /= 2) {
      __syncthreads();
      if (group >= half && group < 2 * half)
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[(threadIdx.x - (half << p.shift)) * 8 + j] = acc[j];
      __syncthreads();
      if (group < half)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += lds[threadIdx.x * 8 + j];
    }
    if (group == 0) finish(p, runs[(size_t)b * p.range], c, chunk, lane, acc);
  }
}

// zeros in grads and norms (dense), or in norms behind the last row
__global__ __launch_bounds__(256) void zero_kernel(GradParams p) {
  const size_t first = (size_t)blockIdx.x * 256 + threadIdx.x, step = (size_t)gridDim.x * 256;
  if (p.dense) {
    const size_t values = (size_t)p.out_rows * p.d, pieces = values / 8;
    for (size_t i = first; i < pieces; i += step) __builtin_nontemporal_store(Piece<float, 8>(0.f), (Piece<float, 8>*)p.grads + i);
    if (first < values % 8) p.grads[pieces * 8 + first] = 0.f;
  }
  if (p.norms)
    for (size_t i = first + (p.dense ? 0 : (uint32_t)max(p.order.counts[0], 0)); i < p.out_rows; i += step) p.norms[i] = 0.f;
}

// a row's norm from its chunks' squares
__global__ __launch_bounds__(256) void norm_kernel(GradParams p) {
  const uint32_t runs = min((uint32_t)max(p.order.counts[0], 0), p.n);
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < runs; i += gridDim.x * 256) {
    const uint32_t row = p.dense ? (uint32_t)p.order.rows[i] : i;
    if (row >= p.out_rows) continue;
    double s = 0.;
    for (int k = 0; k < p.chunks; ++k) s += p.squares[(size_t)i * p.chunks + k];
    p.norms[row] = (float)sqrt(s);
  }
}

// ------------------------------------------------------------------------------------ host
// Tokens of a range: as many as leave 4096 waves, 8 to 128.
static uint32_t range_of(int64_t n, int shift, int chunks) {
  uint32_t s = 128;
  while (s > 8 && (n / s * chunks << shift) < (int64_t)4096 * 64) s /= 2;
  return s;
}

struct GradPlan { int shift, chunks; uint32_t range, ranges; size_t squares, bytes; };

static GradPlan grad_plan(int B, int L, int d) {
  const int64_t n = (int64_t)B * L;
  GradPlan g = {};
  g.chunks = (d + kChunk - 1) / kChunk;
  g.shift = lanes_shift((std::min(d, kChunk) + 7) / 8, 6);
  g.range = range_of(n, g.shift, g.chunks);
  g.ranges = (uint32_t)((n + g.range - 1) / g.range);
  g.squares = align256((size_t)g.ranges * 2 * d * 4);
  g.bytes = g.squares + (g.chunks > 1 ? align256((size_t)n * g.chunks * 8) : 0);
  return g;
}

}  // namespace emb
}  // namespace longer

using namespace longer;

extern "C" {

size_t longer_embedding_backward_workspace_bytes(int B, int L, int d) {
  return check_tokens(B, L) || emb::check_width(d) ? 0 : emb::grad_plan(B, L, d).bytes;
}

int longer_embedding_backward(const longer_order* order, const longer_rows* de, int B, int L, int d, float scale,
                              const longer_dropout_mask* drop, int dense, int64_t out_rows, float* grads_out, float* norms_out,
                              void* ws, size_t ws_bytes, void* stream) {
  int rc = check_tokens(B, L);
  if (!rc) rc = emb::check_width(d);
  if (!rc) rc = emb::check_order(order);
  if (!rc) rc = check_rows(de, "de", B, L, d, false);
  if (!rc) rc = emb::check_mask(drop);
  if (!rc && dense != 0 && dense != 1) rc = api_error(LONGER_ERR_ARG, "dense=%d: 0 or 1", dense);
  if (!rc) rc = check_table_rows(out_rows);
  if (!rc) rc = check_vector(grads_out, LONGER_F32, "grads_out");
  if (!rc && ((uintptr_t)norms_out & 3)) rc = api_error(LONGER_ERR_ARG, "norms_out is not aligned");
  if (!rc && (de->data == grads_out || grads_out == norms_out)) rc = api_error(LONGER_ERR_ARG, "two of de, grads_out, norms_out are the same memory");
  const double factor = scale * emb::kept(rc ? nullptr : drop);
  if (!rc && !std::isfinite((float)factor)) rc = api_error(LONGER_ERR_ARG, "scale=%g: not an fp32 number", scale);
  if (!rc && (!ws || ((uintptr_t)ws & 255))) rc = api_error(LONGER_ERR_ARG, "ws must be 256-byte aligned and not NULL");
  if (rc) return rc;
  const emb::GradPlan g = emb::grad_plan(B, L, d);
  if (ws_bytes < g.bytes) return api_error(LONGER_ERR_WS, "workspace too small: %zu < %zu bytes", ws_bytes, g.bytes);
  hipStream_t st = (hipStream_t)stream;
  const emb::GradParams p = {emb::rows_of(de, B, L), emb::divider(L), (uint32_t)B * L, (uint32_t)L, d, g.shift, g.chunks, g.range, (float)factor, emb::mask_of(drop), *order,
                             dense, (uint32_t)out_rows, grads_out, norms_out, (float*)ws, (double*)((char*)ws + g.squares)};
  if (dense || norms_out) {
    const size_t pieces = dense ? (size_t)out_rows * d / 8 : (size_t)out_rows / 8;
    emb::zero_kernel<<<(unsigned)std::min<size_t>(pieces / 256 + 1, 2048), 256, 0, st>>>(p);
  }
  const unsigned per_group = 256u >> g.shift, per_join = (unsigned)emb::kJoinThreads >> g.shift;
  const dim3 grid((g.ranges + per_group - 1) / per_group, g.chunks);
  if (de->dtype == LONGER_F32) {
    if (p.mask.drop) emb::grad_kernel<float, true><<<grid, 256, 0, st>>>(p);
    else emb::grad_kernel<float, false><<<grid, 256, 0, st>>>(p);
  } else {
    if (p.mask.drop) emb::grad_kernel<__bf16, true><<<grid, 256, 0, st>>>(p);
    else emb::grad_kernel<__bf16, false><<<grid, 256, 0, st>>>(p);
  }
  if (g.ranges > 1) emb::join_kernel<<<dim3((g.ranges + per_join - 1) / per_join, g.chunks), emb::kJoinThreads, 0, st>>>(p);
  if (norms_out && g.chunks > 1) emb::norm_kernel<<<std::min((p.n + 255) / 256, 2048u), 256, 0, st>>>(p);
  return launched("embedding gradient");
}

}  // extern "C"
