// Behind the gradients: their global norm and clipping, and the AdamW update of whole tensors and of the rows that a batch names
// (longer_grad_norm, longer_clip_gradients, longer_adamw_step, longer_adamw_rows).
#include "embedding.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>

namespace longer {
namespace upd {

// A launch takes its tensors in its arguments (under 4 KB of them), so a call needs no table in device memory and
// keeps none.  (Arrays of 4 and 8 byte elements only: beside a byte array the compiler takes the others by scalar loads from a base
// that is off a multiple of 4, and scalar loads drop the two low bits of each part of their address.)  Each tensor is cut into
// pieces, numbered over the launch's list; a workgroup takes one.
struct Piece { int t; int64_t begin; };

// the last of `count` ascending numbers at first[0], first[STRIDE], ... that is not above b: the tensor of piece b, by the number of its
// first piece (an empty tensor is not in the list)
template <int N, int STRIDE>
__device__ __forceinline__ int find_piece(const uint32_t* first, int count, uint32_t b) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int k = 0; k < N; k += 64) {
    const int i = k + lane;
    n += __popcll(__ballot(i < count && first[i * STRIDE] <= b));         // (count is at most N)
  }
  return n - 1;
}
template <int N>
__device__ __forceinline__ Piece find_piece(const uint32_t (&first)[N], int count, uint32_t b, int64_t values) {
  const int t = find_piece<N, 1>(first, count, b);
  return {t, (b - first[t]) * values};
}

// 16 bytes of a tensor, aligned to its element only
template <typename T> struct Line_ { typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };
template <typename T> using Line = typename Line_<T>::type;
template <typename T> struct Four_ { typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T)))); };
template <typename T> using Four = typename Four_<T>::type;

constexpr int kNormList = 248, kClipList = 166;
// Values of a piece.  An update has five streams to keep going and a clip two: with small pieces, in the list's order, what is under
// way at one time is one stretch of each, in few memory pages (128 million parameters, an update in pieces of 1024 / 2048 / 4096 /
// 8192 / 32768 values by 256 threads: 725 / 765 / 808 / 830 / 890 us; four values a thread in workgroups of 256 / 512 / 1024: 725 /
// 720 / 711; 260 million values clipped in pieces of 1024 / 2048 / 4096 / 8192 / 65536: 364 / 362 / 390 / 420 / 420).  The norm's
// pieces, each of which leaves a sum to be joined, are as large as keeps every compute unit busy (at 2048 in all instead of 4096:
// 180 us for 171).
constexpr int kStepPiece = 4096, kClipPiece = 2048;
constexpr uint32_t kHalf = 1u << 31;                // in an entry's size: its values are bf16

struct NormArgs {
  const void* data[kNormList];
  uint32_t n[kNormList];
  uint32_t first[kNormList];
  int count;
  uint32_t pieces;
  int64_t piece;
};
struct ClipArgs {
  const void* in[kClipList];
  void* out[kClipList];
  uint32_t n[kClipList];
  uint32_t first[kClipList];
  const float* norm;
  int count;
};
// An update's list.  Tensors whose p, m, v, g and w each lie in one buffer, at the same place, as a training program keeps them, share
// the buffers' addresses: a tensor is an entry of kEntry words from the front of the list (its place in values, 64 bits; its values; its first
// piece; lr * decay; its buffers and types), the buffers are kBuffers words from the end: 155 tensors of common buffers to a launch,
// or 58 with buffers of their own.
constexpr int kStepWords = 940, kEntry = 6, kBuffers = 10, kStepList = (kStepWords - kBuffers) / kEntry;
constexpr uint32_t kHalfG = 1u << 16, kHalfW = 1u << 17, kCopy = 1u << 18, kGroup = 0xffff;
struct How { float beta1, one_beta1, beta2, one_beta2, rate, root, eps; };   // rate = lr / (1 - beta1^t), root = 1 / sqrt(1 - beta2^t)
struct StepArgs {
  uint32_t list[kStepWords];
  int count;
  const float* norm;
  How how;
};

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
  return v;
}

// sum of squares in 64 bits: exact squares, nothing to scale, and no time beside the loads
template <typename T>
__device__ __forceinline__ double squares(const T* g, uint32_t n) {
  constexpr int V = 16 / sizeof(T), U = 4;
  const uint32_t lines = n / V;
  double s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] = 0.;
  uint32_t i = threadIdx.x;
  for (; i + 256 * (U - 1) < lines; i += 256 * U) {
    Line<T> x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = *(const Line<T>*)(g + (size_t)(i + 256 * k) * V);
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) { const double v = (float)x[k][j]; s[j] = fma(v, v, s[j]); }
  }
  for (; i < lines; i += 256) {
    const Line<T> x = *(const Line<T>*)(g + (size_t)i * V);
#pragma unroll
    for (int j = 0; j < V; ++j) { const double v = (float)x[j]; s[j] = fma(v, v, s[j]); }
  }
  if (lines * V + threadIdx.x < n) { const double v = (float)g[lines * V + threadIdx.x]; s[0] = fma(v, v, s[0]); }
#pragma unroll
  for (int j = 1; j < V; ++j) s[0] += s[j];
  return s[0];
}

// Bound by memory: 260 million fp32 values in 171 to 177 us, 5.9 TB/s or more, 129 million bf16 values in 48, 5.4; 1.2 million in 98 tensors: 4.6 us, and 2 for the sums' join (of
// 4096 sums 4.7).
// (from the list's end to its start: what is read last is what a pass behind this one reads first, and may still be near: 128 million
// parameters, norm and update 858 us for 929)
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a, double* part) {
  __shared__ double lds[4];
  const uint32_t b = a.pieces - 1 - blockIdx.x;
  const Piece w = find_piece(a.first, a.count, b, a.piece);
  const uint32_t n = (uint32_t)min((a.n[w.t] & ~kHalf) - w.begin, a.piece);
  double s = a.n[w.t] & kHalf ? squares((const __bf16*)a.data[w.t] + w.begin, n) : squares((const float*)a.data[w.t] + w.begin, n);
  s = block_sum<256>(s, lds);
  if (threadIdx.x == 0) part[b] = s;
}

__global__ __launch_bounds__(1024) void norm_join_kernel(const double* part, uint32_t n, float max_norm, float* norm) {
  __shared__ double lds[16];
  double s = 0.;
  for (uint32_t i = threadIdx.x; i < n; i += 4096) {          // (four at a time: a list's 4096 sums in one trip to memory)
    double v[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) v[k] = i + 1024 * k < n ? part[i + 1024 * k] : 0.;
    s += (v[0] + v[1]) + (v[2] + v[3]);
  }
  s = block_sum<1024>(s, lds);
  if (threadIdx.x) return;
  const float v = (float)sqrt(s);
  norm[0] = v;
  norm[1] = !isfinite(v) ? 0.f : v <= max_norm ? 1.f : max_norm / v;
}

// Bound by memory: 260 million fp32 values in 358 to 364 us, 5.7 TB/s, two lines of 16 bytes a lane.
template <typename T>
__device__ __forceinline__ void clip_piece(const T* in, T* out, uint32_t n, float c, bool finite) {
  constexpr uint32_t V = 16 / sizeof(T), U = kClipPiece / 256 / V;
  if (n == kClipPiece) {
    Line<T> x[U];
#pragma unroll
    for (uint32_t k = 0; k < U; ++k) x[k] = *(const Line<T>*)(in + (threadIdx.x + 256 * k) * V);
#pragma unroll
    for (uint32_t k = 0; k < U; ++k) {
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) x[k][j] = (T)(finite ? (float)x[k][j] * c : 0.f);
      __builtin_nontemporal_store(x[k], (Line<T>*)(out + (threadIdx.x + 256 * k) * V));
    }
  } else {
    for (uint32_t i = threadIdx.x; i < n; i += 256) out[i] = (T)(finite ? (float)in[i] * c : 0.f);
  }
}

__global__ __launch_bounds__(256) void clip_kernel(ClipArgs a) {
  const Piece w = find_piece(a.first, a.count, blockIdx.x, kClipPiece);
  const float c = a.norm[1];
  const bool finite = isfinite(a.norm[0]);
  if (c == 1.f && a.in[w.t] == a.out[w.t]) return;
  const uint32_t n = (uint32_t)min((a.n[w.t] & ~kHalf) - w.begin, (int64_t)kClipPiece);
  if (a.n[w.t] & kHalf) clip_piece((const __bf16*)a.in[w.t] + w.begin, (__bf16*)a.out[w.t] + w.begin, n, c, finite);
  else clip_piece((const float*)a.in[w.t] + w.begin, (float*)a.out[w.t] + w.begin, n, c, finite);
}

struct Place { float *p, *m, *v; const void* g; void* w; };

// one value (one copy of the formula for whole vectors and tails: the same bits whatever the piece)
__device__ __forceinline__ void step_value(const How& a, float decay, float g, float& p, float& m, float& v) {
  m = fmaf(a.beta1, m, a.one_beta1 * g);
  v = fmaf(a.beta2, v, a.one_beta2 * (g * g));
  p -= fmaf(decay, p, a.rate * (m / fmaf(sqrtf(v), a.root, a.eps)));
}

// Bound by memory: 128 million values in 704 us, 5.4 TB/s; the square root and the quotient are the exact ones, which hide behind the
// loads.  Four values a lane.  Moments, parameters and their copy pass by once: nontemporal, they leave the last cache to the
// gradients that the norm has just read, and to the next norm's (128 million parameters in pieces of 2048: norm 87 us for 150, both
// together 858 us for 916; a reading of times, the traffic itself was not counted).
template <typename G, typename W, bool COPY>
__device__ __forceinline__ void step_piece(const StepArgs& a, const Place& t, uint32_t n, float c, float decay) {
  const G* gs = (const G*)t.g;
  W* ws = (W*)t.w;
  const uint32_t i = threadIdx.x * 4;
  if (i + 4 <= n) {
    const Four<G> g = *(const Four<G>*)(gs + i);
    Four<float> m = __builtin_nontemporal_load((const Four<float>*)(t.m + i));
    Four<float> v = __builtin_nontemporal_load((const Four<float>*)(t.v + i));
    Four<float> p = __builtin_nontemporal_load((const Four<float>*)(t.p + i));
    Four<W> w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float pj = p[j], mj = m[j], vj = v[j];
      step_value(a.how, decay, c * (float)g[j], pj, mj, vj);
      p[j] = pj;
      m[j] = mj;
      v[j] = vj;
      w[j] = (W)pj;
    }
    __builtin_nontemporal_store(m, (Four<float>*)(t.m + i));
    __builtin_nontemporal_store(v, (Four<float>*)(t.v + i));
    __builtin_nontemporal_store(p, (Four<float>*)(t.p + i));
    if (COPY) __builtin_nontemporal_store(w, (Four<W>*)(ws + i));
  } else {
    for (uint32_t k = i; k < n; ++k) {
      float p = t.p[k], m = t.m[k], v = t.v[k];
      step_value(a.how, decay, c * (float)gs[k], p, m, v);
      t.p[k] = p;
      t.m[k] = m;
      t.v[k] = v;
      if (COPY) ws[k] = (W)p;
    }
  }
}

__device__ __forceinline__ uint64_t two_words(const uint32_t* w) { return w[0] | (uint64_t)w[1] << 32; }

template <typename G>
__device__ __forceinline__ void step_piece(const StepArgs& a, const uint32_t* buffers, int64_t at, uint32_t kind, uint32_t n, float c, float decay) {
  Place t = {(float*)two_words(buffers) + at, (float*)two_words(buffers + 2) + at, (float*)two_words(buffers + 4) + at,
             (const G*)two_words(buffers + 6) + at, nullptr};
  if (!(kind & kCopy)) return step_piece<G, float, false>(a, t, n, c, decay);
  if (kind & kHalfW) {
    t.w = (__bf16*)two_words(buffers + 8) + at;
    return step_piece<G, __bf16, true>(a, t, n, c, decay);
  }
  t.w = (float*)two_words(buffers + 8) + at;
  step_piece<G, float, true>(a, t, n, c, decay);
}

__global__ __launch_bounds__(kStepPiece / 4) void step_kernel(StepArgs a) {
  float c = 1.f;
  if (a.norm) {
    if (!isfinite(a.norm[0])) return;
    c = a.norm[1];
  }
  const uint32_t* e = a.list + kEntry * find_piece<kStepList, kEntry>(a.list + 3, a.count, blockIdx.x);
  const uint32_t begin = (blockIdx.x - e[3]) * kStepPiece, n = min(e[2] - begin, (uint32_t)kStepPiece), kind = e[5];
  const int64_t at = (int64_t)two_words(e) + begin;
  const uint32_t* buffers = a.list + kStepWords - kBuffers * ((kind & kGroup) + 1);
  const float decay = __uint_as_float(e[4]);
  if (kind & kHalfG) step_piece<__bf16>(a, buffers, at, kind, n, c, decay);
  else step_piece<float>(a, buffers, at, kind, n, c, decay);
}

// The rows of a table that a batch names: row i of g is the gradient of row rows[i].  A lane holds four values of a row.
// Bound by memory: 400 thousand rows of 128 in 301 us, 5.1 TB/s, p, m, v and w past the caches (312 with ordinary accesses), g, which the gradient's pass
// has left there, not.  The grid is as large as pays where the count, which is on the GPU, turns out small (2048 / 16384 / 65536 workgroups: 138 thousand rows
// of a batch of 512000 tokens 99.5 / 95.6 / 102 us; 400 thousand 312 / 301 / 294).
struct RowsArgs {
  float *p, *m, *v;
  void* w;
  const float* g;
  const int32_t *rows, *counts;
  const float* norm;
  uint32_t most, table_rows;                          // rows of g at most, rows of the table
  int d;
  emb::Deal deal;
  float decay;                                        // lr * decay
  How how;
};

template <bool PAST>
__device__ __forceinline__ Four<float> load_four(const float* p) { return PAST ? __builtin_nontemporal_load((const Four<float>*)p) : *(const Four<float>*)p; }
template <bool PAST, typename T>
__device__ __forceinline__ void store_four(T* p, Four<T> v) {
  if (PAST) __builtin_nontemporal_store(v, (Four<T>*)p);
  else *(Four<T>*)p = v;
}

template <typename W, bool COPY, bool PAST>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
  float c = 1.f;
  if (a.norm) {
    if (!isfinite(a.norm[0])) return;
    c = a.norm[1];
  }
  const uint32_t count = min((uint32_t)max(a.counts[0], 0), a.most);
  const emb::Seat me = emb::seat(a.deal);
  if (!me.taken) return;
  for (uint32_t i = blockIdx.x * a.deal.per_turn + me.row; i < count; i += gridDim.x * a.deal.per_turn) {
    const uint32_t row = (uint32_t)a.rows[i];
    if (row >= a.table_rows) continue;
    const size_t at = (size_t)row * a.d;
    const float* gs = a.g + (size_t)i * a.d;
    W* ws = (W*)a.w;
    for (int k = (blockIdx.y * a.deal.lanes + me.lane) * 4; k < a.d; k += gridDim.y * a.deal.lanes * 4) {
      if (k + 4 <= a.d) {
        const Four<float> g = *(const Four<float>*)(gs + k);
        Four<float> m = load_four<PAST>(a.m + at + k), v = load_four<PAST>(a.v + at + k), p = load_four<PAST>(a.p + at + k);
        Four<W> w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float pj = p[j], mj = m[j], vj = v[j];
          step_value(a.how, a.decay, c * g[j], pj, mj, vj);
          p[j] = pj;
          m[j] = mj;
          v[j] = vj;
          w[j] = (W)pj;
        }
        store_four<PAST>(a.m + at + k, m);
        store_four<PAST>(a.v + at + k, v);
        store_four<PAST>(a.p + at + k, p);
        if (COPY) store_four<PAST>(ws + at + k, w);
      } else {
        for (int j = k; j < a.d; ++j) {
          float p = a.p[at + j], m = a.m[at + j], v = a.v[at + j];
          step_value(a.how, a.decay, c * gs[j], p, m, v);
          a.p[at + j] = p;
          a.m[at + j] = m;
          a.v[at + j] = v;
          if (COPY) ws[at + j] = (W)p;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t kMostEntry = (int64_t)1 << 30;     // values of one place in a launch's list
constexpr int64_t kMostValues = (int64_t)1 << 40;    // of a list: more than a GPU's memory holds

static int check_tensor(const void* p, int64_t n, int dtype, int i, const char* name) {
  if (n < 0 || n > kMostValues) return api_error(LONGER_ERR_ARG, "tensor %d: n=%lld out of range", i, (long long)n);
  if (!size_of(dtype)) return api_error(LONGER_ERR_ARG, "tensor %d: dtype %d of %s unknown", i, dtype, name);
  if (n && !p) return api_error(LONGER_ERR_ARG, "tensor %d: %s is NULL", i, name);
  if ((uintptr_t)p % size_of(dtype)) return api_error(LONGER_ERR_ARG, "tensor %d: %s is not aligned to its elements", i, name);
  return 0;
}

static int check_list(const longer_tensor* t, int count, int64_t* values) {
  if (!t || count <= 0) return api_error(LONGER_ERR_ARG, "an empty list of tensors");
  int64_t sum = 0;
  for (int i = 0; i < count; ++i) {
    if (int rc = check_tensor(t[i].data, t[i].n, t[i].dtype, i, "data")) return rc;
    sum += t[i].n;
    if (sum > kMostValues) return api_error(LONGER_ERR_ARG, "a list of more than 2^40 values");
  }
  *values = sum;
  return 0;
}

static int check_how(const longer_adamw* how, How* h) {
  if (!how) return api_error(LONGER_ERR_ARG, "how is NULL");
  if (!(how->lr >= 0.) || !std::isfinite(how->lr)) return api_error(LONGER_ERR_ARG, "lr=%g: not negative, finite", how->lr);
  if (!(how->beta1 >= 0. && how->beta1 < 1.) || !(how->beta2 >= 0. && how->beta2 < 1.)) return api_error(LONGER_ERR_ARG, "beta1=%g beta2=%g: 0 to below 1", how->beta1, how->beta2);
  if (!(how->eps >= FLT_MIN && how->eps <= FLT_MAX)) return api_error(LONGER_ERR_ARG, "eps=%g must be positive (a normal fp32 number)", how->eps);
  if (how->step < 1) return api_error(LONGER_ERR_ARG, "step=%lld: counts from 1", (long long)how->step);
  const double rate = how->lr / (1. - std::pow(how->beta1, (double)how->step));
  if (!(rate <= FLT_MAX)) return api_error(LONGER_ERR_ARG, "lr=%g: lr / (1 - beta1^step) is beyond fp32", how->lr);
  *h = {(float)how->beta1, (float)(1. - how->beta1), (float)how->beta2, (float)(1. - how->beta2), (float)rate,
        (float)(1. / std::sqrt(1. - std::pow(how->beta2, (double)how->step))), (float)how->eps};
  return 0;
}

// The norm's pieces: about 4096 in all (sixteen workgroups for each compute unit), of at least 2048 values, so that a short list has as
// many workgroups as it can feed.
static int64_t norm_piece(int64_t values) {
  int64_t piece = 2048;
  while (piece * 4096 < values) piece *= 2;
  return piece;
}
static uint32_t pieces(int64_t n, int64_t piece) { return (uint32_t)((n + piece - 1) / piece); }

static uint32_t list_pieces(const longer_tensor* t, int count, int64_t piece) {
  uint32_t k = 0;
  for (int i = 0; i < count; ++i) k += pieces(t[i].n, piece);
  return k;
}
static size_t norm_bytes(uint32_t n) { return ((size_t)(n ? n : 1) * 8 + 255) & ~(size_t)255; }

// Cuts a list into launches: `add(j, i, begin, n, first)` puts values [begin, begin + n) of tensor i in place j of a launch, their
// pieces numbered from `first`, or says that the launch has no room for them; `go(entries, pieces)` launches.  A launch ends full or at
// `most_pieces` workgroups (the grid counts threads in 32 bits); a tensor may go on in the next place.
template <typename Size, typename Add, typename Go>
static void launches(int count, int64_t piece, uint32_t most_pieces, Size size, Add add, Go go) {
  int64_t begin = 0;
  for (int i = 0; i < count;) {
    int entries = 0;
    uint32_t k = 0;
    while (i < count && k < most_pieces) {
      const int64_t left = size(i) - begin;
      const int64_t room = std::min((most_pieces - k) * piece, kMostEntry);
      const int64_t n = std::min(left, room);
      if (n) {
        if (!add(entries, i, begin, n, k)) break;
        ++entries;
        k += pieces(n, piece);
      }
      begin += n;
      if (n == left) { ++i; begin = 0; }
    }
    if (k) go(entries, k);
  }
}

}  // namespace upd
}  // namespace longer

using namespace longer;

extern "C" {

size_t longer_grad_norm_workspace_bytes(const longer_tensor* grads, int count) {
  int64_t values;
  if (upd::check_list(grads, count, &values)) return 0;
  return upd::norm_bytes(upd::list_pieces(grads, count, upd::norm_piece(values)));
}

int longer_grad_norm(const longer_tensor* grads, int count, float max_norm, float* norm_out,
                     void* ws, size_t ws_bytes, void* stream) {
  int64_t values;
  if (int rc = upd::check_list(grads, count, &values)) return rc;
  if (!norm_out || !ws) return api_error(LONGER_ERR_ARG, "null pointer argument");
  if ((uintptr_t)norm_out & 3) return api_error(LONGER_ERR_ARG, "norm_out is not aligned");
  if ((uintptr_t)ws & 255) return api_error(LONGER_ERR_ARG, "ws must be 256-byte aligned");
  if (!(max_norm > 0.f)) return api_error(LONGER_ERR_ARG, "max_norm must be positive");
  const int64_t piece = upd::norm_piece(values);
  const uint32_t all = upd::list_pieces(grads, count, piece);
  if (ws_bytes < upd::norm_bytes(all)) return api_error(LONGER_ERR_WS, "workspace too small: %zu < %zu bytes", ws_bytes, upd::norm_bytes(all));
  hipStream_t st = (hipStream_t)stream;
  uint32_t done = 0;
  upd::NormArgs a;
  a.piece = piece;
  upd::launches(count, piece, 1u << 23, [&](int i) { return grads[i].n; },
                [&](int j, int i, int64_t begin, int64_t n, uint32_t first) {
                  if (j == upd::kNormList) return false;
                  const bool half = grads[i].dtype == LONGER_BF16;
                  a.data[j] = (const char*)grads[i].data + begin * (half ? 2 : 4);
                  a.n[j] = (uint32_t)n | (half ? upd::kHalf : 0);
                  a.first[j] = first;
                  return true;
                },
                [&](int entries, uint32_t k) {
                  a.count = entries;
                  a.pieces = k;
                  upd::norm_kernel<<<k, 256, 0, st>>>(a, (double*)ws + done);
                  done += k;
                });
  upd::norm_join_kernel<<<1, 1024, 0, st>>>((const double*)ws, done, max_norm, norm_out);
  return launched("gradient norm");
}

int longer_clip_gradients(const longer_tensor* grads, const longer_tensor* out, int count, const float* norm, void* stream) {
  int64_t values;
  if (int rc = upd::check_list(grads, count, &values)) return rc;
  if (out) {
    if (int rc = upd::check_list(out, count, &values)) return rc;
    for (int i = 0; i < count; ++i)
      if (out[i].n != grads[i].n || out[i].dtype != grads[i].dtype) return api_error(LONGER_ERR_ARG, "tensor %d: out has another size or dtype", i);
  }
  if (!norm || ((uintptr_t)norm & 3)) return api_error(LONGER_ERR_ARG, "norm is NULL or not aligned");
  hipStream_t st = (hipStream_t)stream;
  upd::ClipArgs a;
  a.norm = norm;
  upd::launches(count, upd::kClipPiece, 1u << 23, [&](int i) { return grads[i].n; },
                [&](int j, int i, int64_t begin, int64_t n, uint32_t first) {
                  if (j == upd::kClipList) return false;
                  const bool half = grads[i].dtype == LONGER_BF16;
                  a.in[j] = (const char*)grads[i].data + begin * (half ? 2 : 4);
                  a.out[j] = (char*)(out ? out[i].data : grads[i].data) + begin * (half ? 2 : 4);
                  a.n[j] = (uint32_t)n | (half ? upd::kHalf : 0);
                  a.first[j] = first;
                  return true;
                },
                [&](int entries, uint32_t k) {
                  a.count = entries;
                  upd::clip_kernel<<<k, 256, 0, st>>>(a);
                });
  return launched("gradient clipping");
}

int longer_adamw_step(const longer_adamw_tensor* t, int count, const longer_adamw* how, const float* norm, void* stream) {
  if (!t || count <= 0) return api_error(LONGER_ERR_ARG, "an empty list of tensors");
  upd::How h;
  if (int rc = upd::check_how(how, &h)) return rc;
  if ((uintptr_t)norm & 3) return api_error(LONGER_ERR_ARG, "norm is not aligned");
  int64_t values = 0;
  for (int i = 0; i < count; ++i) {
    int rc = upd::check_tensor(t[i].p, t[i].n, LONGER_F32, i, "p");
    if (!rc) rc = upd::check_tensor(t[i].m, t[i].n, LONGER_F32, i, "m");
    if (!rc) rc = upd::check_tensor(t[i].v, t[i].n, LONGER_F32, i, "v");
    if (!rc) rc = upd::check_tensor(t[i].g, t[i].n, t[i].g_dtype, i, "g");
    if (!rc && t[i].w) rc = upd::check_tensor(t[i].w, t[i].n, t[i].w_dtype, i, "w");
    if (rc) return rc;
    if (!(t[i].decay >= 0.) || !(how->lr * t[i].decay <= FLT_MAX)) return api_error(LONGER_ERR_ARG, "tensor %d: decay=%g: not negative, lr decay an fp32 number", i, t[i].decay);
    const void* at[5] = {t[i].p, t[i].m, t[i].v, t[i].g, t[i].w};
    for (int j = 0; j < 5; ++j)
      for (int k = 0; k < j; ++k)
        if (t[i].n && at[j] && at[j] == at[k]) return api_error(LONGER_ERR_ARG, "tensor %d: two of p, m, v, g, w are the same memory", i);
    values += t[i].n;
    if (values > upd::kMostValues) return api_error(LONGER_ERR_ARG, "a list of more than 2^40 values");
  }
  hipStream_t st = (hipStream_t)stream;
  upd::StepArgs a;
  a.norm = norm;
  a.how = h;
  int groups = 0;                                     // of the launch at hand, and the last one's buffers, where place 0 would be
  uint64_t last[5];
  uint32_t last_kind = 0;
  upd::launches(count, upd::kStepPiece, 1u << 21, [&](int i) { return t[i].n; },
                [&](int j, int i, int64_t begin, int64_t n, uint32_t first) {
                  if (j == 0) groups = 0;
                  const bool half_g = t[i].g_dtype == LONGER_BF16, half_w = t[i].w && t[i].w_dtype == LONGER_BF16;
                  const uint32_t kind = (half_g ? upd::kHalfG : 0) | (half_w ? upd::kHalfW : 0) | (t[i].w ? upd::kCopy : 0);
                  const uint64_t at[5] = {(uint64_t)t[i].p, (uint64_t)t[i].m, (uint64_t)t[i].v, (uint64_t)t[i].g, (uint64_t)t[i].w};
                  const int64_t size[5] = {4, 4, 4, half_g ? 2 : 4, half_w ? 2 : 4};
                  int64_t place = groups ? ((int64_t)(at[0] - last[0])) / 4 : 0;
                  bool joins = groups && kind == last_kind;
                  for (int k = 0; joins && k < (t[i].w ? 5 : 4); ++k) joins = (int64_t)(at[k] - last[k]) == place * size[k];
                  if (upd::kEntry * (j + 1) + upd::kBuffers * (groups + !joins) > upd::kStepWords) return false;
                  if (!joins) {
                    uint32_t* b = a.list + upd::kStepWords - upd::kBuffers * ++groups;
                    for (int k = 0; k < 5; ++k) {
                      last[k] = at[k];
                      b[2 * k] = (uint32_t)at[k];
                      b[2 * k + 1] = (uint32_t)(at[k] >> 32);
                    }
                    last_kind = kind;
                    place = 0;
                  }
                  place += begin;
                  const float decay = (float)(how->lr * t[i].decay);
                  uint32_t* e = a.list + upd::kEntry * j;
                  e[0] = (uint32_t)place;
                  e[1] = (uint32_t)((uint64_t)place >> 32);
                  e[2] = (uint32_t)n;
                  e[3] = first;
                  std::memcpy(e + 4, &decay, 4);
                  e[5] = kind | (uint32_t)(groups - 1);
                  return true;
                },
                [&](int entries, uint32_t k) {
                  a.count = entries;
                  upd::step_kernel<<<k, upd::kStepPiece / 4, 0, st>>>(a);
                });
  return launched("AdamW update");
}

int longer_adamw_rows(const longer_adamw_table* t, const longer_order* order, int B, int L, const float* g,
                      const longer_adamw* how, const float* norm, void* stream) {
  int rc = check_tokens(B, L);
  if (!rc) rc = emb::check_order(order);
  if (!rc && !t) rc = api_error(LONGER_ERR_ARG, "table is NULL");
  if (!rc) rc = emb::check_width(t->d);
  if (!rc) rc = check_table_rows(t->rows);
  if (!rc) rc = check_vector(t->p, LONGER_F32, "p");
  if (!rc) rc = check_vector(t->m, LONGER_F32, "m");
  if (!rc) rc = check_vector(t->v, LONGER_F32, "v");
  if (!rc) rc = check_vector(g, LONGER_F32, "g");
  if (!rc && t->w && !size_of(t->w_dtype)) rc = api_error(LONGER_ERR_ARG, "dtype %d of w unknown", t->w_dtype);
  if (!rc && t->w) rc = check_vector(t->w, t->w_dtype, "w");
  if (rc) return rc;
  const void* at[5] = {t->p, t->m, t->v, g, t->w};
  for (int j = 0; j < 5; ++j)
    for (int k = 0; k < j; ++k)
      if (at[j] == at[k]) return api_error(LONGER_ERR_ARG, "two of p, m, v, g, w are the same memory");
  upd::How h;
  if ((rc = upd::check_how(how, &h))) return rc;
  if (!(t->decay >= 0.) || !(how->lr * t->decay <= FLT_MAX)) return api_error(LONGER_ERR_ARG, "decay=%g: not negative, lr decay an fp32 number", t->decay);
  if ((uintptr_t)norm & 3) return api_error(LONGER_ERR_ARG, "norm is not aligned");
  const uint32_t most = (uint32_t)std::min<int64_t>((int64_t)B * L, t->rows);
  const upd::RowsArgs a = {t->p, t->m, t->v, t->w, g, order->rows, order->counts, norm, most, (uint32_t)t->rows, t->d, emb::deal((t->d + 3) / 4),
                           (float)(how->lr * t->decay), h};
  const unsigned groups = std::min((most + a.deal.per_turn - 1) / a.deal.per_turn, 16384u);
  // Few rows of several turns: a workgroup for each turn (300 rows of 8192 in 17.1 us for 19.1; 4606 of 3486 in 115 either way; 12000 of 4096 in 294 for 284).
  const unsigned parts = most <= 8192 ? (t->d + 1023) / 1024 : 1;
  hipStream_t st = (hipStream_t)stream;
  // Whole lines of 128 bytes go past the caches; rows of other widths through them, where the lines that two rows share may meet (138 thousand rows of
  // 33 / 40 / 100 / 129 values, 12397 of 4099: 98.6 / 67.3 / 126 / 190 / 365 us past, 63.7 / 65 / 135 / 174 / 353 through; of 128 95.4, 113).
  const bool past = t->d % 32 == 0 && !(((uintptr_t)t->p | (uintptr_t)t->m | (uintptr_t)t->v) & 127);
  auto go = [&](auto kernel) { kernel<<<dim3(groups, parts), 256, 0, st>>>(a); };
  if (!t->w) past ? go(upd::rows_kernel<float, false, true>) : go(upd::rows_kernel<float, false, false>);
  else if (t->w_dtype == LONGER_BF16) past ? go(upd::rows_kernel<__bf16, true, true>) : go(upd::rows_kernel<__bf16, true, false>);
  else past ? go(upd::rows_kernel<float, true, true>) : go(upd::rows_kernel<float, true, false>);
  return launched("AdamW update of rows");
}

}  // extern "C"
