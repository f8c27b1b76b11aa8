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

constexpr int kThreads = 256, kThreadBits = 8;
constexpr int kValues = 8;                           // of a lane where rows are added up; a group has 512 columns at most (4 values of fp32 rows: 80 us for 74)

// What of a workgroup's sums crosses its borders: the run that began before it, the run that begins in it and goes on, and that run's row
// of the gradient (kNone: there is none).
constexpr uint32_t kNone = ~0u;
struct alignas(16) Border { uint32_t lead, tail, row, unused; };

struct GradParams {
  Rows de;
  Divider by_L, by_d;
  uint32_t n, L;                                     // tokens of the batch
  int d, shift, chunks;
  uint32_t range, block;                             // tokens of a group and of a workgroup
  float factor;
  Mask mask;
  longer_order order;
  int dense;
  uint32_t out_rows, blocks, zero_rows, zero_shares; // blocks: workgroups with tokens; the others write zeros, in shares of zero_rows of a dense gradient
  float *grads, *norms;
  float* part;                                       // [workgroups][2][d]
  Border* borders;                                   // [workgroups]
  double* squares;                                   // [runs][chunks], where there is more than one chunk
  int part_bits;                                     // 2^part_bits workgroups share the columns of a run of many stretches
  uint32_t* arrivals;                                // [workgroups][chunks]: of them, how many are done with the run that begins there
  double* part_squares;                              // [workgroups][chunks][parts]
};

__device__ __forceinline__ uint32_t tokens_of(const GradParams& p) { return min((uint32_t)max(p.order.counts[1], 0), p.n); }
__device__ __forceinline__ uint32_t runs_of(const GradParams& p) { return min((uint32_t)max(p.order.counts[0], 0), p.n); }

// (these rows are read again, by the join or the update, and go through the caches: past them the gradient of 512000 tokens of 128 takes 71 us for 74, but
// with the update behind it 235 for 228)
template <Kind KIND, int V>
__device__ __forceinline__ void store_sums(float* to, int n, const float (&a)[V]) {
  Piece<float, V> v;
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = a[j];
  if (KIND != VALUES || n >= V) *(Piece<float, V>*)to = v;
  else
#pragma unroll
    for (int j = 0; j < V - 1; ++j)
      if (j < n) to[j] = v[j];
}

struct Lane { Part at; uint32_t piece; int lane, chunk, shift; };    // a lane's columns (n <= 0: it has none), of the 2^shift lanes of its group
template <Kind KIND, int V>
__device__ __forceinline__ Lane lane_of(const GradParams& p, int shift, uint32_t part = 0) {
  const int lane = threadIdx.x & ((1 << shift) - 1), chunk = blockIdx.y, c = (chunk * 64 + (part << shift) + lane) * V;
  if (c >= p.d) return {{0, 0, 0}, 0, lane, chunk, shift};
  return {part_of<KIND, V>((uint32_t)c / V, p.d), (uint32_t)c / V, lane, chunk, shift};
}

template <int CTRL> __device__ __forceinline__ float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int CTRL> __device__ __forceinline__ double from_lane(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(bits >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// sum over the 2^shift lanes of a group (all of them are here, other groups may not be: lanes take from their own group's alone)
template <typename V>
__device__ __forceinline__ V group_sum(V v, int shift) {
  if (shift >= 1) v += from_lane<0xB1>(v);           // the neighbour's
  if (shift >= 2) v += from_lane<0x4E>(v);           // the other pair's
  if (shift >= 3) v += from_lane<0x141>(v);          // mirrored in 8
  if (shift >= 4) v += from_lane<0x140>(v);          // mirrored in 16
  if (shift >= 5) v += __shfl_xor(v, 16);
  if (shift >= 6) v += __shfl_xor(v, 32);
  return v;
}

// A run's sums are complete: its row goes out, and the squares of its values, which are added up in 64 bits so that a row of any size has its norm, rounded
// once, are returned.  All lanes of the group are here.
template <Kind KIND, int V>
__device__ __forceinline__ double put_row(const GradParams& p, uint32_t row, const Lane& me, const float (&acc)[V]) {
  float g[V];
#pragma unroll
  for (int j = 0; j < V; ++j) g[j] = p.factor * acc[j];
  if (row < p.out_rows && me.at.n > 0) store_sums<KIND, V>(p.grads + (size_t)row * p.d + me.at.c, me.at.n, g);
  double squares = 0.;
  if (!p.norms) return squares;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const double x = KIND == WHOLE ? (me.at.n ? g[j] : 0.f) : j >= me.at.twice && j < me.at.n ? g[j] : 0.f;
    squares = fma(x, x, squares);
  }
  return group_sum(squares, me.shift);
}

__device__ __forceinline__ void put_norm(const GradParams& p, uint32_t run, uint32_t row, int chunk, double squares) {
  if (row >= p.out_rows) return;
  if (p.chunks > 1) p.squares[(size_t)run * p.chunks + chunk] = squares;
  else p.norms[row] = (float)sqrt(squares);
}

template <Kind KIND, int V>
__device__ __forceinline__ void finish(const GradParams& p, uint32_t run, uint32_t row, const Lane& me, const float (&acc)[V]) {
  const double squares = put_row<KIND, V>(p, row, me, acc);
  if (p.norms && me.lane == 0) put_norm(p, run, row, me.chunk, squares);
}

// The first of `count` ascending numbers that is not below `from`: 64 places at a time.
__device__ __forceinline__ uint32_t lower_bound(const int32_t* rows, uint32_t count, uint32_t from) {
  uint32_t lo = 0, hi = count;
  while (lo < hi) {
    const uint32_t step = (hi - lo + 63) / 64, at = lo + (threadIdx.x & 63) * step;
    const uint32_t below = __popcll(__ballot(at < hi && (uint32_t)rows[min(at, hi - 1)] < from));
    if (!below) break;
    hi = min(hi, lo + below * step);
    lo += (below - 1) * step + 1;
  }
  return lo;
}

// Zeros in the rows of a dense gradient that no token names, and in their norms, beside the workgroups that add up the others': the named rows of a
// share come from the order.  16 KB to a share, a workgroup each while the grid has room for them (300007 rows of 96, 256000 tokens, shares of 4 / 16 / 32 / 64 KB: 47 / 30 / 35 / 36 us
// in all; zeros in a launch of their own: 35 and that launch's time; 1000003 rows of 128: 103 us for 97 and the launch).
constexpr uint32_t kMostZeroRows = 2048;
__device__ __forceinline__ void zero_rows(const GradParams& p, uint32_t share, uint8_t* named) {
  const uint32_t a = share * p.zero_rows, b = min(a + p.zero_rows, p.out_rows), count = min(runs_of(p), p.out_rows);
  for (uint32_t i = threadIdx.x; i < p.zero_rows; i += kThreads) named[i] = 0;
  const uint32_t first = lower_bound(p.order.rows, count, a);
  __syncthreads();
  for (uint32_t i = first + threadIdx.x; i < count; i += kThreads) {
    const uint32_t row = (uint32_t)p.order.rows[i];
    if (row >= b) break;
    if (row >= a) named[row - a] = 1;
  }
  __syncthreads();
  // the share's values in pieces of four, whatever row they are of (row by row: 1000438 rows of 33 in 56 us for 30, 145146 of 282 in 44 for 30)
  const uint32_t values = (b - a) * p.d;
  float* to = p.grads + (size_t)a * p.d;
  for (uint32_t i = 4 * threadIdx.x; i < values; i += 4 * kThreads) {
    const uint32_t first_row = p.by_d(i), last_row = p.d % 4 ? p.by_d(min(i + 4, values) - 1) : first_row;
    uint32_t any = i + 4 > values;
    for (uint32_t row = first_row; row <= last_row; ++row) any |= named[row];
    if (!any) __builtin_nontemporal_store(Piece<float, 4>(0.f), (Piece<float, 4>*)(to + i));
    else
      for (uint32_t k = i; k < min(i + 4, values); ++k)
        if (!named[p.by_d(k)]) to[k] = 0.f;
  }
  if (p.norms)
    for (uint32_t row = a + threadIdx.x; row < b; row += kThreads)
      if (!named[row - a]) p.norms[row] = 0.f;
}

// LDS of a workgroup's tokens: where their rows of dE lie, their runs (with the neighbours' on both sides), the runs' rows, their numbers
__host__ __device__ inline size_t staged_bytes(uint32_t block, bool drop) { return (size_t)block * (drop ? 20 : 16) + 8; }

template <typename T, bool DROP, Kind KIND>
__global__ __launch_bounds__(kThreads, 4) void grad_kernel(GradParams p) {
  constexpr int V = kValues, U = 2;
  constexpr uint32_t kLead = 1, kOn = 2;             // a group's first run began before it; that run goes on behind it
  extern __shared__ int64_t staged[];
  __shared__ float lead[kThreads * V];
  __shared__ uint32_t flags[kThreads];
  int64_t* from = staged;
  uint32_t *runs = (uint32_t*)(from + p.block) + 1, *rows = runs + p.block + 1, *tokens = rows + p.block;
  if (blockIdx.x >= p.blocks) {
    static_assert(kMostZeroRows <= sizeof(lead), "a byte for each row");
    if (blockIdx.y) return;
    uint32_t share = blockIdx.x - p.blocks;
    zero_rows(p, share, (uint8_t*)lead);
    while ((share += gridDim.x - p.blocks) < p.zero_shares) {
      __syncthreads();                               // (a share's marks go where the last one's are read; behind the last share nobody waits)
      zero_rows(p, share, (uint8_t*)lead);
    }
    return;
  }
  const Lane me = lane_of<KIND, V>(p, p.shift);
  const int c = me.at.c, width = me.at.n;
  const uint32_t group = threadIdx.x >> p.shift, groups = kThreads >> p.shift, first = blockIdx.x * p.block;
  // (read before it is known how many of them the order holds; its arrays are as long as the batch)
  const uint32_t at = min(first + threadIdx.x, p.n - 1);
  const uint32_t token0 = (uint32_t)p.order.tokens[at], run0 = (uint32_t)p.order.runs[at];
  const uint32_t run_before = (uint32_t)p.order.runs[max(first, 1u) - 1], run_behind = (uint32_t)p.order.runs[min(first + p.block, p.n - 1)];
  const uint32_t n = tokens_of(p);
  if (p.norms && blockIdx.y == 0 && !p.dense)        // zeros behind the last row's norm
    for (uint64_t i = (uint64_t)runs_of(p) + blockIdx.x * kThreads + threadIdx.x; i < p.out_rows; i += (uint64_t)p.blocks * kThreads) p.norms[i] = 0.f;
  if (p.part_bits && threadIdx.x == 0) p.arrivals[blockIdx.x * p.chunks + blockIdx.y] = 0;
  if (first >= n) {
    if (blockIdx.y == 0 && threadIdx.x == 0) p.borders[blockIdx.x] = {kNone, kNone, 0, 0};
    return;
  }
  const uint32_t count = min(p.block, n - first);
  const Key key = DROP ? load_key(p.mask) : Key{};
  // (whatever the order holds, nothing outside the buffers is read or written: rows ascend, so that a run has no row below its number)
  const uint32_t most = min(p.n, p.out_rows);
  for (uint32_t i = threadIdx.x; i < count; i += kThreads) {
    const uint32_t token = i == threadIdx.x ? token0 : (uint32_t)p.order.tokens[first + i], run = i == threadIdx.x ? run0 : (uint32_t)p.order.runs[first + i];
    const uint32_t b = p.by_L(token), l = token - b * p.L;
    from[i] = token < p.n ? (int64_t)b * p.de.user + (int64_t)l * p.de.row : 0;
    runs[i] = run;
    rows[i] = run >= most ? kNone : p.dense ? (uint32_t)p.order.rows[run] : run;
    if (DROP) tokens[i] = token;
  }
  if (threadIdx.x == 0) {
    runs[-1] = first ? run_before : kNone;
    runs[count] = first + count < n ? run_behind : kNone;
  }
  __syncthreads();
  if (blockIdx.y == 0 && threadIdx.x == 0) {
    const bool leads = runs[0] == runs[-1], goes = runs[count - 1] == runs[count];
    p.borders[blockIdx.x] = {leads ? runs[0] : kNone, goes && !(leads && runs[count - 1] == runs[0]) ? runs[count - 1] : kNone, rows[count - 1], 0};
  }
  const uint32_t begin = min(group * p.range, count), end = min(begin + p.range, count);
  float acc[V] = {};
  uint32_t run = kNone;
  bool earlier = false, on = false;
  if (begin < end) {
    struct Batch { Piece<T, V> x[U]; uint32_t run[U], token[U]; } batch[2];
    // The rows of one batch are under way while another is added up.  Loads are unconditional (behind the range, its last row again): a
    // load in a branch makes the compiler wait for all that are under way.
    auto load = [&](Batch& to, uint32_t at) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t i = min(at + u, end - 1);
        to.x[u] = load_piece<T, KIND, V>((const T*)p.de.data + from[i] + c, width);
        to.run[u] = runs[i];
        if (DROP) to.token[u] = tokens[i];
      }
    };
    // a run that began here is complete with token i, whose place in dE nobody asks for any more: its norm's squares wait there
    auto done = [&](uint32_t i) {
      const double squares = put_row<KIND, V>(p, rows[i], me, acc);
      if (p.norms && me.lane == 0) from[i] = __builtin_bit_cast(int64_t, squares);
    };
    auto take = [&](const Batch& in, uint32_t at) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (at + u >= end) return;
        if (in.run[u] != run) {
          if (earlier) {
#pragma unroll
            for (int j = 0; j < V; ++j) lead[threadIdx.x * V + j] = acc[j];
          } else {
            done(at + u - 1);
          }
          run = in.run[u];
          earlier = false;
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] = 0.f;
        }
        Piece<float, V> y;
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = (float)in.x[u][j];
        if (DROP) drop_piece<KIND, V>(p.mask, key, in.token[u], me.piece, me.lane == 0, p.d, y);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += y[j];
      }
    };
    run = runs[begin];
    earlier = runs[(int)begin - 1] == run;
    if (me.lane == 0) flags[group] = earlier ? kLead : 0;
    load(batch[0], begin);
    for (uint32_t k = 0; k < p.range; k += 2 * U) {
      load(batch[1], begin + k + U);
      take(batch[0], begin + k);
      if (k + 2 * U < p.range) load(batch[0], begin + k + 2 * U);
      take(batch[1], begin + k + U);
    }
    on = runs[end] == run;
    if (earlier) {
#pragma unroll
      for (int j = 0; j < V; ++j) lead[threadIdx.x * V + j] = acc[j];
      if (me.lane == 0) flags[group] = kLead | (on ? kOn : 0);
    } else if (!on) {
      done(end - 1);
    }
  }
  __syncthreads();
  // the norms of the runs that began and ended in one range, a thread each (by a group at each run's end: 512000 tokens of 129 in 102 us for 89, of 128 75 for 74,
  // of 33 38 for 34)
  if (p.norms)
    for (uint32_t i = threadIdx.x; i < count; i += kThreads)
      if (runs[i] != runs[i + 1] && runs[i] != runs[(int)(i & ~(p.range - 1)) - 1]) put_norm(p, runs[i], rows[i], me.chunk, __builtin_bit_cast(double, from[i]));
  // Runs that go on: where a wave has eight groups or more, what each of them has of the run that began before it first becomes the sum over the groups from it
  // on, as far as that run goes in the wave, doubling the distance at every step (163 thousand tokens of 537 rows of 16 / 32 / 64: 11 / 10 / 12 us, 19 / 14 / 13
  // group after group; of 128 16.6, 16.4).
  const int per_step = p.shift <= 3 ? 64 >> p.shift : 1;
  if (per_step > 1) {
    const uint32_t flag = begin < end ? flags[group] : 0;
    bool more = flag & kOn;                          // whether the run goes on behind them
    if (__any(more)) {
      float x[V];
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = flag & kLead ? lead[threadIdx.x * V + j] : 0.f;
      for (int by = 1; by < per_step; by *= 2) {
        const bool there = (threadIdx.x & 63) + (by << p.shift) < 64;
        const int behind = __shfl_down((int)more, by << p.shift);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float y = __shfl_down(x[j], by << p.shift);
          x[j] += there && more ? y : 0.f;
        }
        more &= !there || behind;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) lead[threadIdx.x * V + j] = x[j];
      if (me.lane == 0) flags[group] = (flag & kLead) | (more ? kOn : 0);
    }
    __syncthreads();
  }
  // Then the group where a run begins (or the workgroup's first, where it began before) adds up those sums.
  const bool owner = begin < end && on && !earlier, before = group == 0 && flags[0] & kLead;
  if (!owner && !before) return;
  float* part = p.part + (size_t)blockIdx.x * 2 * p.d + c;
  auto add_sums = [&](float (&sum)[V], uint32_t h) {
    bool on = true;
    for (; h < groups && on; h = (h / per_step + 1) * per_step) {
      on = flags[h] & kOn;
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += lead[((h << p.shift) + me.lane) * V + j];
    }
    return on;
  };
  if (before) {
    float sum[V] = {};
    add_sums(sum, 0);
    if (width > 0) store_sums<KIND, V>(part, width, sum);
  }
  if (owner) {
    if (!add_sums(acc, group + 1)) finish<KIND, V>(p, run, rows[end - 1], me, acc);
    else if (width > 0) store_sums<KIND, V>(part + p.d, width, acc);
  }
}

constexpr uint32_t kLong = 256;

// The sums of stretches h, h + by, ..., U of them under way at once, while they go on with the run; says whether the last one did.  (A
// stretch that does not has left nothing to read: what is there is not used.)
template <Kind KIND, int V, uint32_t U>
__device__ __forceinline__ bool add_leads(const GradParams& p, float (&acc)[V], uint32_t h, uint32_t by, uint32_t run, int c, int width) {
  uint32_t lead[U];
  Piece<float, V> x[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t i = min(h + u * by, p.blocks - 1);
    lead[u] = h + u * by < p.blocks ? p.borders[i].lead : kNone;
    x[u] = load_piece<float, KIND, V>(p.part + (size_t)i * 2 * p.d + c, width);
  }
  bool more = true;
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    more &= lead[u] == run;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += more ? x[u][j] : 0.f;
  }
  return more;
}

// The runs that cross workgroups' stretches, each by the group of the stretch that it begins in, and by the whole workgroup where it
// goes on for more than ALONE.  Then group k takes every groups-th of its sums, which meet in two steps; of more than kLong, workgroups z = 0, 1, ... take a part
// of its columns each, as one item may have most of the tokens, and one compute unit reads 2 MB in 26 us.  The last of them to be done adds up what the
// others left for the norm, in the order of the parts: nobody waits.  Bound by its loads' latency (512000
// tokens of 128, 8 values a lane: 10.6 us with ALONE 4, 11.8 with 8; 230 thousand tokens of one item: 11.4 us with 8 sums of a group under way, 14.2 with 4).
template <Kind KIND, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void join_kernel(GradParams p) {
  constexpr uint32_t ALONE = 4;
  __shared__ float lds[THREADS * V];
  constexpr uint32_t kShared = 1u << 31;             // of a list's entry: the run is shared among the workgroups z
  __shared__ uint32_t list[THREADS], listed;
  const size_t step = (size_t)2 * p.d;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  {
    const Lane me = lane_of<KIND, V>(p, p.shift);
    const int c = me.at.c, width = max(me.at.n, 0);
    const uint32_t group = threadIdx.x >> p.shift, groups = THREADS >> p.shift, g = blockIdx.x * groups + group;
    if (g < p.blocks) {
      const Border own = p.borders[g];
      const Piece<float, V> x = load_piece<float, KIND, V>(p.part + g * step + p.d + c, width);
      float acc[V];
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = x[j];
      const uint32_t after = g + ALONE + 1 < p.blocks ? p.borders[g + ALONE + 1].lead : kNone;
      const bool is_long = p.part_bits && (g + kLong < p.blocks ? p.borders[g + kLong].lead : kNone) == own.tail;
      if (own.tail != kNone) {
        if (after == own.tail) {
          if (me.lane == 0 && (is_long || blockIdx.z == 0)) list[atomicAdd(&listed, 1u)] = is_long ? g | kShared : g;      // (the order of the list is that of the work alone)
        } else if (blockIdx.z == 0) {
          add_leads<KIND, V, ALONE>(p, acc, g + 1, 1, own.tail, c, width);
          finish<KIND, V>(p, own.tail, own.row, me, acc);
        }
      }
    }
  }
  __syncthreads();
  for (uint32_t i = 0; i < listed; ++i) {
    const bool shared = list[i] & kShared;
    const uint32_t a = list[i] & ~kShared;
    const int shift = shared ? p.shift - p.part_bits : p.shift;
    const Lane me = lane_of<KIND, V>(p, shift, blockIdx.z);
    const int c = me.at.c, width = max(me.at.n, 0);
    const uint32_t group = threadIdx.x >> shift, groups = THREADS >> shift;
    const Border own = p.borders[a];
    float acc[V] = {};
    constexpr uint32_t MANY = 64 / V;
    for (uint32_t h = a + 1 + group; add_leads<KIND, V, MANY>(p, acc, h, groups, own.tail, c, width); h += MANY * groups) {}
    if (group == 0) {
      const Piece<float, V> x = load_piece<float, KIND, V>(p.part + a * step + p.d + c, width);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += x[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) lds[threadIdx.x * V + j] = acc[j];
    __syncthreads();
    if (group < 8) {                                 // (at least 8 groups)
#pragma unroll 4
      for (uint32_t h = group + 8; h < groups; h += 8)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += lds[((h << shift) + me.lane) * V + j];
    }
    __syncthreads();
    if (group < 8)
#pragma unroll
      for (int j = 0; j < V; ++j) lds[threadIdx.x * V + j] = acc[j];
    __syncthreads();
    if (group == 0) {
      for (uint32_t h = 1; h < 8; ++h)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += lds[((h << shift) + me.lane) * V + j];
      double squares = put_row<KIND, V>(p, own.row, me, acc);
      if (p.norms && me.lane == 0) {
        const uint32_t parts = 1u << p.part_bits;
        bool last = true;
        if (shared) {
          const size_t at = (size_t)a * p.chunks + me.chunk;
          double* all = p.part_squares + at * parts;
          __hip_atomic_store(all + blockIdx.z, squares, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          last = __hip_atomic_fetch_add(p.arrivals + at, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
          if (last) {
            squares = 0.;
            for (uint32_t k = 0; k < parts; ++k) squares += __hip_atomic_load(all + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          }
        }
        if (last) put_norm(p, own.tail, own.row, me.chunk, squares);
      }
    }
  }
}

// a row's norm from its chunks' squares
__global__ __launch_bounds__(256) void norm_kernel(GradParams p) {
  const uint32_t runs = min(runs_of(p), p.out_rows);
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < runs; i += gridDim.x * 256) {
    const uint32_t row = p.dense ? (uint32_t)p.order.rows[i] : i;
    if (row >= p.out_rows) continue;
    double s = 0.;
    for (int k = 0; k < p.chunks; ++k) s += p.squares[(size_t)i * p.chunks + k];
    p.norms[row] = (float)sqrt(s);
  }
}

// ------------------------------------------------------------------------------------ host
// Tokens of a range: 32 where that leaves 8192 waves (and a workgroup at most 2048), down to 8 for as many, 4 where 8 leave less than 4096.
// (512000 tokens of 128, ranges of 8 / 16 / 32: 74 / 82 / 85 us; 2.6 million: 312 / 320 / 330, but crossings 20 / 18 / 13, and of one item in
// most places 170 / 85 / 50; 4503 tokens of 4099, 4 / 8 / 16: with the crossings 21.7 / 19.3 / 19.0.)
static uint32_t range_of(int64_t n, int shift, int chunks) {
  auto waves = [&](uint32_t s) { return (n / s * chunks << shift) / 64; };
  uint32_t s = std::min(32u, 2048u >> (kThreadBits - shift));
  while (s > 8 && waves(s) < 8192) s /= 2;
  if (s == 8 && waves(s) < 4096) s = 4;
  return s;
}

// A run that goes on for more than kLong of a workgroup's stretches is shared among 2^kPartBits workgroups, where the rows are wide enough (512000 tokens of 128: most of
// one item in 16 us for 26, popular in 8.3 for 7.8, also where 8 share it 17 and 13; shared from 128 on: 9.6; 23 thousand tokens of 512, most of one: 16 for 34).
constexpr int kPartBits = 2;
struct GradPlan { int shift, chunks, part_bits; uint32_t range, block, blocks; size_t borders, squares, arrivals, part_squares, bytes; };

static GradPlan grad_plan(int B, int L, int d) {
  const int64_t n = (int64_t)B * L;
  GradPlan g = {};
  const int pieces = (d + kValues - 1) / kValues;
  g.chunks = (pieces + 63) / 64;
  g.shift = lanes_shift(std::min(pieces, 64), 6);
  g.range = range_of(n, g.shift, g.chunks);
  g.block = g.range * (kThreads >> g.shift);
  g.blocks = (uint32_t)((n + g.block - 1) / g.block);
  g.borders = align256((size_t)g.blocks * 2 * d * 4);
  g.squares = g.borders + align256((size_t)g.blocks * sizeof(Border));
  g.arrivals = g.squares + (g.chunks > 1 ? align256((size_t)n * g.chunks * 8) : 0);
  g.part_bits = d > 64 && g.blocks > kLong ? kPartBits : 0;
  g.part_squares = g.arrivals + (g.part_bits ? align256((size_t)g.blocks * g.chunks * 4) : 0);
  g.bytes = g.part_squares + (g.part_bits ? align256((size_t)g.blocks * g.chunks * 8 << g.part_bits) : 0);
  return g;
}

template <typename T>
static void grad(const GradParams& p, dim3 grid, hipStream_t st) {
  const size_t lds = staged_bytes(p.block, p.mask.drop);
  auto go = [&](auto kind) {
    constexpr Kind KIND = decltype(kind)::value;
    if (p.mask.drop) grad_kernel<T, true, KIND><<<grid, kThreads, lds, st>>>(p);
    else grad_kernel<T, false, KIND><<<grid, kThreads, lds, st>>>(p);
  };
  with_kind(kind_of(p.d, kValues), go);
}

// V: values of a lane.  4 where a wave holds a row so, which is one chunk either way (512000 tokens of 128, few / most of one item: 7.8 / 26.6 us, 10.6 / 27.2
// with 8).  Groups: as many as 512 threads have, 128 threads' where these are at least 8, so that fewer of a batch's popular items meet in one workgroup, one
// behind the other (512000 tokens of 32, popular / most of one item: 6.9 / 10.0 us, 13.4 / 5.5 with 512 threads; of 64: 5.9, 11.3).
template <int V, int THREADS>
static void join(GradParams p, hipStream_t st) {
  p.shift = lanes_shift(std::min((p.d + V - 1) / V, 64), 6);
  const uint32_t groups = (uint32_t)THREADS >> p.shift;
  const dim3 grid((p.blocks + groups - 1) / groups, p.chunks, 1 << p.part_bits);
  with_kind(kind_of(p.d, V), [&](auto kind) { join_kernel<decltype(kind)::value, V, THREADS><<<grid, THREADS, 0, st>>>(p); });
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
  uint32_t zero_rows = std::max(4096u / (uint32_t)d, 1u);
  if (d % 4) zero_rows = (zero_rows + 3) & ~3u;                       // (shares begin where pieces of 16 bytes do)
  zero_rows = std::min(zero_rows, emb::kMostZeroRows);
  const uint32_t zero_shares = dense ? ((uint32_t)out_rows + zero_rows - 1) / zero_rows : 0;
  const emb::GradParams p = {emb::rows_of(de, B, L), emb::divider(L), emb::divider(d), (uint32_t)B * L, (uint32_t)L, d, g.shift, g.chunks, g.range, g.block, (float)factor,
                             emb::mask_of(drop), *order, dense, (uint32_t)out_rows, g.blocks, zero_rows, zero_shares, grads_out, norms_out, (float*)ws, (emb::Border*)((char*)ws + g.borders), (double*)((char*)ws + g.squares), g.part_bits, (uint32_t*)((char*)ws + g.arrivals), (double*)((char*)ws + g.part_squares)};
  // (a grid counts threads in 32 bits; at most 2^24 - 2^14 workgroups have tokens)
  static_assert(emb::kThreads == 256, "2^24 workgroups");
  const dim3 grid(g.blocks + std::min(zero_shares, (1u << 24) - 1 - g.blocks), g.chunks);
  if (de->dtype == LONGER_F32) emb::grad<float>(p, grid, st);
  else emb::grad<__bf16>(p, grid, st);
  if (g.blocks > 1) d <= 64 ? emb::join<4, 128>(p, st) : d <= 256 ? emb::join<4, 512>(p, st) : emb::join<emb::kValues, 512>(p, st);
  if (norms_out && g.chunks > 1) emb::norm_kernel<<<std::min((p.n + 255) / 256, 2048u), 256, 0, st>>>(p);
  return launched("embedding gradient");
}

}  // extern "C"
