// Gradient of a table of embeddings by sorted tokens (longer_embedding_backward).
//
// The order's tokens are cut into ranges.  A group of lanes takes a range (and a chunk of at most 512 columns, 8 a lane) and adds up
// its rows of dE in registers, one run of equal ids after the other; where a run ends, its row is complete and goes out, scaled once.  A
// run that crosses ranges leaves a sum in each: they meet in LDS inside a workgroup, and the workgroups' sums, [workgroup][0] of the
// run that began before it, [workgroup][1] of the run that begins in it and goes on, in a second launch.  However long a run is, no
// group has more than its range to read; the order of a sum follows from the sizes alone.
#include "embedding.h"

namespace longer {
namespace emb {

constexpr int kChunk = 512;                          // columns of a group: 64 lanes of 8

struct GradParams {
  Rows de;
  Divider by_L;
  uint32_t n, L;                                     // tokens of the batch
  int d, shift, chunks;
  uint32_t range, block;                             // tokens of a group and of a workgroup
  float factor;
  Mask mask;
  longer_order order;
  int dense;
  uint32_t out_rows;
  float *grads, *norms;
  float* part;                                       // [workgroups][2][d]
  double* squares;                                   // [runs][chunks], where there is more than one chunk
};

__device__ __forceinline__ uint32_t tokens_of(const GradParams& p) { return min((uint32_t)max(p.order.counts[1], 0), p.n); }
__device__ __forceinline__ uint32_t runs_of(const GradParams& p) { return min((uint32_t)max(p.order.counts[0], 0), p.n); }

// (these rows are read again, by the join or the update)
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

struct Lane { Part at; int lane, chunk; };           // a lane's columns (n <= 0: it has none)
template <bool WHOLE>
__device__ __forceinline__ Lane lane_of(const GradParams& p) {
  const int lane = threadIdx.x & ((1 << p.shift) - 1), chunk = blockIdx.y, c = chunk * kChunk + lane * 8;
  if (c >= p.d) return {{0, 0, 0}, lane, chunk};
  return {part_of<WHOLE>((uint32_t)c / 8, p.d, p.d >= 8), lane, chunk};
}

template <int CTRL> __device__ __forceinline__ double with_dpp(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(bits >> 32), CTRL, 0xF, 0xF, true);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// sum over the 2^shift lanes of a group (all of them are here, other groups may not be: lanes take from their own group's alone)
__device__ __forceinline__ double group_sum(double v, int shift) {
  if (shift >= 1) v = with_dpp<0xB1>(v);             // the neighbour's
  if (shift >= 2) v = with_dpp<0x4E>(v);             // the other pair's
  if (shift >= 3) v = with_dpp<0x141>(v);            // mirrored in 8
  if (shift >= 4) v = with_dpp<0x140>(v);            // mirrored in 16
  if (shift >= 5) v += __shfl_xor(v, 16);
  if (shift >= 6) v += __shfl_xor(v, 32);
  return v;
}

// The root of a sum of squares, rounded: in fp32 (off by 1.5 half steps) where the sum is a normal number of fp32
__device__ __forceinline__ float root(double s) { return s > 1e-37 && s < 1e38 ? sqrtf((float)s) : (float)sqrt(s); }

// A run's sums are complete: its row, and its norm's squares.  All lanes of the group are here.
__device__ __forceinline__ void finish(const GradParams& p, uint32_t run, uint32_t row, const Lane& me, const float (&acc)[8]) {
  if (row >= p.out_rows) return;
  float g[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = p.factor * acc[j];
  if (me.at.n > 0) store_sums(p.grads + (size_t)row * p.d + me.at.c, me.at.n, g);
  if (!p.norms) return;
  double s = 0.;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const double v = j >= me.at.twice && j < me.at.n ? g[j] : 0.f;
    s = fma(v, v, s);
  }
  s = group_sum(s, p.shift);
  if (me.lane == 0) {
    if (p.chunks == 1) p.norms[row] = root(s);
    else p.squares[(size_t)run * p.chunks + me.chunk] = s;
  }
}
__device__ __forceinline__ uint32_t row_of(const GradParams& p, uint32_t run) { return p.dense ? (uint32_t)p.order.rows[run] : run; }

template <typename T, bool DROP, bool WHOLE>
__global__ __launch_bounds__(256, 4) void grad_kernel(GradParams p) {
  constexpr int U = 8;
  constexpr uint32_t kLead = 1, kOn = 2;             // a group's first run began before it; that run goes on behind it
  __shared__ float lead[256 * 8];
  __shared__ uint32_t flags[256];
  const Lane me = lane_of<WHOLE>(p);
  const int c = me.at.c, width = me.at.n;
  const uint32_t n = tokens_of(p), group = threadIdx.x >> p.shift, groups = 256 >> p.shift;
  if (p.norms && blockIdx.y == 0 && !p.dense)        // zeros behind the last row's norm
    for (uint64_t i = (uint64_t)runs_of(p) + blockIdx.x * 256 + threadIdx.x; i < p.out_rows; i += (uint64_t)gridDim.x * 256) p.norms[i] = 0.f;
  if ((uint64_t)blockIdx.x * p.block >= n) return;
  const uint32_t first = blockIdx.x * p.block, begin = min(first + group * p.range, n), end = min(begin + p.range, n);
  const Key key = DROP ? load_key(p.mask) : Key{};
  float acc[8] = {};
  uint32_t run = 0, row = 0;
  bool earlier = false, on = false;
  if (begin < end) {
    run = p.order.runs[begin];
    row = row_of(p, run);
    earlier = begin && (uint32_t)p.order.runs[begin - 1] == run;
    const uint32_t behind = end < n ? (uint32_t)p.order.runs[end] : ~0u;
    if (me.lane == 0) flags[group] = earlier ? kLead : 0;
    for (uint32_t at = begin; at < end; at += U) {
      uint32_t token[U], runs[U], rows[U];
      Piece<T, 8> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t i = min(at + u, end - 1);
        token[u] = (uint32_t)p.order.tokens[i];
        runs[u] = (uint32_t)p.order.runs[i];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        rows[u] = row_of(p, runs[u]);
        if (at + u < end && token[u] < p.n && width > 0) {
          const uint32_t b = p.by_L(token[u]), l = token[u] - b * p.L;
          x[u] = load8((const T*)p.de.data + (int64_t)b * p.de.user + (int64_t)l * p.de.row + c, width);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (at + u >= end) break;
        if (runs[u] != run) {
          if (earlier) {
#pragma unroll
            for (int j = 0; j < 8; ++j) lead[threadIdx.x * 8 + j] = acc[j];
          } else {
            finish(p, run, row, me, acc);
          }
          run = runs[u];
          row = rows[u];
          earlier = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
        if (token[u] < p.n && width > 0) {
          Piece<float, 8> y;
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = (float)x[u][j];
          if (DROP) drop8<WHOLE>(p.mask, key, token[u], c, y);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += y[j];
        }
      }
    }
    on = behind == run;
    if (earlier) {
#pragma unroll
      for (int j = 0; j < 8; ++j) lead[threadIdx.x * 8 + j] = acc[j];
      if (me.lane == 0) flags[group] = kLead | (on ? kOn : 0);
    } else if (!on) {
      finish(p, run, row, me, acc);
    }
  }
  __syncthreads();
  // a run that goes on: the group where it begins (or the workgroup's first, where it began before) adds up the sums of those behind
  const bool owner = begin < end && on && !earlier, before = group == 0 && flags[0] & kLead;
  if (!owner && !before) return;
  float* part = p.part + (size_t)blockIdx.x * 2 * p.d + c;
  if (before) {
    float sum[8];
    bool more = true;
    for (uint32_t h = 0; h < groups && more; ++h) {
      more = flags[h] & kOn;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = (h ? sum[j] : 0.f) + lead[((h << p.shift) + me.lane) * 8 + j];
    }
    if (width > 0) store_sums(part, width, sum);
  }
  if (owner) {
    bool more = true;
    for (uint32_t h = group + 1; h < groups && more; ++h) {
      more = flags[h] & kOn;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += lead[((h << p.shift) + me.lane) * 8 + j];
    }
    if (!more) finish(p, run, row, me, acc);
    else if (width > 0) store_sums(part + p.d, width, acc);
  }
}

constexpr int kJoinThreads = 1024, kJoinAlone = 16;

// The runs that cross workgroups' stretches, each by the group of the stretch that it begins in, and by the whole workgroup where it
// goes on for more than kJoinAlone: group k takes every groups-th of its sums, which then meet in two steps.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(GradParams p) {
  constexpr int U = 4;
  __shared__ float lds[kJoinThreads * 8];
  __shared__ uint32_t list[kJoinThreads], listed;
  const Lane me = lane_of<false>(p);
  const int c = me.at.c, width = me.at.n;
  const uint32_t group = threadIdx.x >> p.shift, groups = kJoinThreads >> p.shift, n = tokens_of(p), blocks = (n + p.block - 1) / p.block;
  const int32_t* runs = p.order.runs;
  if (blockIdx.x * groups >= blocks) return;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  const size_t step = (size_t)2 * p.d;
  // adds the sums of stretches h, h + by, ... below `to` that begin with `run`; says whether the last one did
  auto add = [&](float (&acc)[8], uint32_t h, uint32_t by, uint32_t to, uint32_t run) {
    bool more = true;
    for (; more && h < to; h += U * by) {
      bool goes[U];
      Piece<float, 8> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t i = min(h + u * by, blocks - 1);
        goes[u] = h + u * by < to && (uint32_t)runs[(size_t)i * p.block] == run;
        x[u] = load8(p.part + i * step + c, max(width, 0));
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        more &= goes[u];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += more ? x[u][j] : 0.f;
      }
    }
  };
  const uint32_t g = blockIdx.x * groups + group;
  if (g + 1 < blocks) {
    const uint32_t begin = g * p.block, end = begin + p.block, run = (uint32_t)runs[end], row = row_of(p, run);
    if ((uint32_t)runs[end - 1] == run && !(begin && (uint32_t)runs[begin - 1] == run)) {
      if (g + kJoinAlone + 1 < blocks && (uint32_t)runs[(size_t)(g + kJoinAlone + 1) * p.block] == run) {
        if (me.lane == 0) list[atomicAdd(&listed, 1u)] = g;          // (the order of the list is that of the work alone)
      } else {
        float acc[8];
        const Piece<float, 8> x = load8(p.part + g * step + p.d + c, max(width, 0));
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = x[j];
        add(acc, g + 1, 1, blocks, run);
        finish(p, run, row, me, acc);
      }
    }
  }
  __syncthreads();
  for (uint32_t i = 0; i < listed; ++i) {
    const uint32_t a = list[i], run = (uint32_t)runs[(size_t)(a + 1) * p.block];
    float acc[8] = {};
    if (group == 0) {
      const Piece<float, 8> x = load8(p.part + a * step + p.d + c, max(width, 0));
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = x[j];
    }
    add(acc, a + 1 + group, groups, blocks, run);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[threadIdx.x * 8 + j] = acc[j];
    __syncthreads();
    if (group < 8) {                                 // (at least 16 groups)
#pragma unroll 4
      for (uint32_t h = group + 8; h < groups; h += 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += lds[((h << p.shift) + me.lane) * 8 + j];
    }
    __syncthreads();
    if (group < 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) lds[threadIdx.x * 8 + j] = acc[j];
    __syncthreads();
    if (group == 0)
      for (uint32_t h = 1; h < 8; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += lds[((h << p.shift) + me.lane) * 8 + j];
    if (group == 0) finish(p, run, row_of(p, run), me, acc);
  }
}

// zeros in grads and norms of a dense gradient (1 GiB in ... us)
__global__ __launch_bounds__(256) void zero_kernel(GradParams p) {
  const size_t first = (size_t)blockIdx.x * 256 + threadIdx.x, step = (size_t)gridDim.x * 256;
  const size_t values = (size_t)p.out_rows * p.d, pieces = values / 4;
  for (size_t i = first; i < pieces; i += step) __builtin_nontemporal_store(Piece<float, 4>(0.f), (Piece<float, 4>*)p.grads + i);
  if (first < values % 4) p.grads[pieces * 4 + first] = 0.f;
  if (p.norms)
    for (size_t i = first; i < p.out_rows; i += step) p.norms[i] = 0.f;
}

// a row's norm from its chunks' squares
__global__ __launch_bounds__(256) void norm_kernel(GradParams p) {
  const uint32_t runs = runs_of(p);
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < runs; i += gridDim.x * 256) {
    const uint32_t row = p.dense ? (uint32_t)p.order.rows[i] : i;
    if (row >= p.out_rows) continue;
    double s = 0.;
    for (int k = 0; k < p.chunks; ++k) s += p.squares[(size_t)i * p.chunks + k];
    p.norms[row] = root(s);
  }
}

// ------------------------------------------------------------------------------------ host
// Tokens of a range: as many as leave 4096 waves, 8 to 64.
static uint32_t range_of(int64_t n, int shift, int chunks) {
  uint32_t s = 64;
  while (s > 8 && (n / s * chunks << shift) < (int64_t)4096 * 64) s /= 2;
  return s;
}

struct GradPlan { int shift, chunks; uint32_t range, block, blocks; size_t squares, bytes; };

static GradPlan grad_plan(int B, int L, int d) {
  const int64_t n = (int64_t)B * L;
  GradPlan g = {};
  g.chunks = (d + kChunk - 1) / kChunk;
  g.shift = lanes_shift((std::min(d, kChunk) + 7) / 8, 6);
  g.range = range_of(n, g.shift, g.chunks);
  g.block = g.range * (256 >> g.shift);
  g.blocks = (uint32_t)((n + g.block - 1) / g.block);
  g.squares = align256((size_t)g.blocks * 2 * d * 4);
  g.bytes = g.squares + (g.chunks > 1 ? align256((size_t)n * g.chunks * 8) : 0);
  return g;
}

template <typename T>
static void grad(const GradParams& p, dim3 grid, hipStream_t st) {
  if (p.d % 8 == 0) {
    if (p.mask.drop) grad_kernel<T, true, true><<<grid, 256, 0, st>>>(p);
    else grad_kernel<T, false, true><<<grid, 256, 0, st>>>(p);
  } else {
    if (p.mask.drop) grad_kernel<T, true, false><<<grid, 256, 0, st>>>(p);
    else grad_kernel<T, false, false><<<grid, 256, 0, st>>>(p);
  }
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
  const emb::GradParams p = {emb::rows_of(de, B, L), emb::divider(L), (uint32_t)B * L, (uint32_t)L, d, g.shift, g.chunks, g.range, g.block, (float)factor,
                             emb::mask_of(drop), *order, dense, (uint32_t)out_rows, grads_out, norms_out, (float*)ws, (double*)((char*)ws + g.squares)};
  if (dense) emb::zero_kernel<<<(unsigned)std::min<size_t>((size_t)out_rows * d / 1024 + 1, 4096), 256, 0, st>>>(p);
  const dim3 grid(g.blocks, g.chunks);
  if (de->dtype == LONGER_F32) emb::grad<float>(p, grid, st);
  else emb::grad<__bf16>(p, grid, st);
  const unsigned per_join = (unsigned)emb::kJoinThreads >> g.shift;
  if (g.blocks > 1) emb::join_kernel<<<dim3((g.blocks + per_join - 1) / per_join, g.chunks), emb::kJoinThreads, 0, st>>>(p);
  if (norms_out && g.chunks > 1) emb::norm_kernel<<<std::min((p.n + 255) / 256, 2048u), 256, 0, st>>>(p);
  return launched("embedding gradient");
}

}  // extern "C"
