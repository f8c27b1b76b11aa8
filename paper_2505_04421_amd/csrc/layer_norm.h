// Layer norm of token rows and its backward pass: one read of a row, everything else in registers.
//
// A row of d values is cut into pieces of V values, at most 16 bytes of the narrower type; LPR lanes hold it, NV pieces each (piece
// lane + LPR i), so a wave holds 64 / LPR rows at once and a row wider than a wave's pieces has a workgroup's lanes.  The statistics
// take two sums in lanes, the mean and then the centred squares: no cancellation, and the row is there already.  A lane divides its
// at most 32 squares by d before lanes meet: at any width they leave fp32 only where single values do, not where d of them would (a
// value within 1e18 of the row's mean is within 2e18 of its wave's: 32 * 4e36 < 3.4e38).
//
// Widths that no piece divides: the last piece is moved back to end with the row, so that every access is whole and inside it; its
// first values (below `lo`) are also its neighbour's, take no part in sums, and are computed and stored twice, to the same bits.
// Loads and stores are aligned to the element only, which the memory path takes at any address.
#pragma once
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
  int spread;                       // workgroups' groups in turn, not each workgroup's side by side
  int step_u, step_l;               // rows from one of a workgroup's turns to its next, as users and rows
  float eps, inv_d;
  float* part;                      // backward: [workgroups][2][d] column sums
};

enum { FULL, PIECES, VALUES };      // what is masked: nothing, whole pieces past the row, values of the last piece too

template <typename T, int V> struct Piece_ { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <typename T, int V> using Piece = typename Piece_<T, V>::type;

template <int CTRL> __device__ __forceinline__ float with_dpp(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// sum over groups of LPR adjacent lanes, in every lane (every lane of the wave takes part)
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (LPR >= 2) v = with_dpp<0xB1>(v);       // the neighbour's
  if constexpr (LPR >= 4) v = with_dpp<0x4E>(v);       // the other pair's
  if constexpr (LPR >= 8) v = with_dpp<0x141>(v);      // mirrored in 8
  if constexpr (LPR >= 16) v = with_dpp<0x140>(v);     // mirrored in 16
  if constexpr (LPR >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned lo = r[0], hi = r[1];           // (named: a bit cast of a vector's element takes the first one)
    v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
  }
  if constexpr (LPR >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned lo = r[0], hi = r[1];           // (named: a bit cast of a vector's element takes the first one)
    v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
  }
  return v;
}

// Rows of several waves.  Each wave centres its values on its own mean; then one barrier a row brings the waves' sums together:
// with n_w values, mean m_w and e_w = m_w - mean, the row's centred squares are sum of (wave's + n_w e_w^2), its sum of q (x - mean)
// is sum of (wave's q (x - m_w) + e_w wave's q), none of which cancels.  Squares are divided by d before they meet.  Two places in LDS in turn: a wave that writes one again has
// passed the other's barrier, which every wave reaches after its reads.
struct Shares { float s, squares, q, qx; };
template <int LPR, int THREADS, bool SEVERAL = (LPR > 64)>
struct Meeting {                    // (rows of one wave: nothing)
  struct Memory {};
  __device__ __forceinline__ Meeting(Memory&, int) {}
};
template <int LPR, int THREADS>
struct Meeting<LPR, THREADS, true> {
  static constexpr int W = THREADS / 64, S = LPR / 64;
  struct Memory { Shares at[2][W]; float n[W], inv_n[W]; };
  Memory& m;
  float inv_n;
  int turn = 0;
  __device__ __forceinline__ Meeting(Memory& memory, int own) : m(memory) {      // own: values of the row that the lane has
    const float n = lanes_sum<64>((float)own);
    inv_n = n > 0.f ? 1.f / n : 0.f;
    if ((threadIdx.x & 63) == 0) { m.n[threadIdx.x / 64] = n; m.inv_n[threadIdx.x / 64] = inv_n; }
  }
  // the wave's shares (s: its sum) to the row's; gives the row's mean, the same bits in every wave (two may hold the same value)
  __device__ __forceinline__ float join(Shares& v, float inv_d) {
    const int wave = threadIdx.x / 64;
    if ((threadIdx.x & 63) == 0) m.at[turn][wave] = v;
    __syncthreads();
    const int other = wave / S * S + threadIdx.x % S;
    Shares o = m.at[turn][other];
    turn ^= 1;
    const float mean = lanes_sum<S>(o.s) * inv_d, e = o.s * m.inv_n[other] - mean;
    v.squares = lanes_sum<S>(fmaf(m.n[other] * inv_d * e, e, o.squares));
    v.q = lanes_sum<S>(o.q);
    v.qx = lanes_sum<S>(fmaf(e, o.q, o.qx));
    return mean;
  }
};

// A lane's columns
template <int V, int LPR, int NV, int MODE>
struct Columns {
  int col[NV], lo[NV];              // first column; first value that is its own (V: the piece is past the row)
  __device__ __forceinline__ Columns(int lane, int d) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + LPR * i) * V;
      col[i] = MODE == FULL ? c : min(c, d - V);
      lo[i] = MODE == FULL ? 0 : min(c - col[i], V);
    }
  }
  __device__ __forceinline__ bool there(int i) const { return MODE == FULL || lo[i] < V; }
  // whether some lane of the wave has values that are not its own: only there sums leave values out
  __device__ __forceinline__ bool masked() const {
    if (MODE == FULL) return false;
    bool some = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) some |= lo[i] > 0;
    return __builtin_amdgcn_ballot_w64(some) != 0;
  }
  __device__ __forceinline__ int owned() const {
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) n += MODE == FULL ? V : V - lo[i];
    return n;
  }
  __device__ __forceinline__ bool own(int i, int j) const { return MODE == FULL || (MODE == PIECES ? lo[i] < V : j >= lo[i]); }
};

// A row's lanes, or a wave's rows side by side, are a group.  A workgroup's groups of a turn are neighbours (rows that share a cache
// line are then one die's); where rows may be padding, which comes in long stretches, the workgroups' first groups are neighbours,
// then their second ones, so that every compute unit has its share (gradients of 512 users of up to 5000 rows of 128: 479 us for 499;
// but of 128000 dense rows of 255: 99 for 91).
template <int LPR> constexpr int kGroupRows = LPR < 64 ? 64 / LPR : 1;
template <int LPR, int THREADS>
__device__ __forceinline__ int first_turn(const Params& p) {
  constexpr int RPW = kGroupRows<LPR>, GROUPS = THREADS / LPR / RPW;
  if (LPR > 64 && GROUPS == 1) return blockIdx.x;
  const int group = threadIdx.x / (LPR * RPW);
  return (p.spread ? group * gridDim.x + blockIdx.x : blockIdx.x * GROUPS + group) * RPW;
}

// (of its first group, which has the most turns: what waves go by that meet at barriers)
template <int LPR, int THREADS>
__device__ __forceinline__ int first_of_workgroup(const Params& p) {
  return p.spread ? blockIdx.x : blockIdx.x * (THREADS / LPR);
}

// A workgroup's walk over the rows: its next turns' places, and the lengths of their users asked for one turn ahead of the rows.
struct Walk {
  int r, u, l, n;
  __device__ __forceinline__ Walk(const Params& p, int first) {
    r = first;
    u = (unsigned)first / (unsigned)p.L;
    l = first - u * p.L;
    n = p.L;
    ask(p);
  }
  // no kernel writes lengths: where a workgroup's lanes share the row it is a scalar load
  __device__ __forceinline__ void ask(const Params& p) {
    typedef const __attribute__((address_space(4))) int32_t* fixed;
    if (p.lens) n = r < p.rows ? ((fixed)p.lens)[u] : 0;
  }
  __device__ __forceinline__ bool valid(const Params& p) const { return r < p.rows && l < n; }
  __device__ __forceinline__ Walk next(const Params& p, int step) const {
    Walk w = *this;
    w.r = r + step;                           // (at most two turns past the last row: the host keeps that below 2^31)
    w.u += p.step_u;
    w.l += p.step_l;
    if (w.l >= p.L) { w.l -= p.L; ++w.u; }
    w.ask(p);
    return w;
  }
};

template <typename T, int V, int LPR, int NV, int MODE>
__device__ __forceinline__ void load_row(Piece<T, V> (&x)[NV], const Rows& r, const Walk& at, bool ok, const Columns<V, LPR, NV, MODE>& c) {
  const T* row = (const T*)r.data + at.u * r.user + at.l * r.row;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    x[i] = (Piece<T, V>)(T)0.f;
    if (ok && c.there(i)) x[i] = *(const Piece<T, V>*)(row + c.col[i]);
  }
}

// Waits for a row that is under way.  In front of a turn's stores, which are under conditions: behind them the wait would be for the
// stores as well, each turn.
template <typename T, int V, int NV>
__device__ __forceinline__ void landed(Piece<T, V> (&x)[NV]) {
  if constexpr (sizeof(T) * V >= 16) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * V / 4)));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      words w = __builtin_bit_cast(words, x[i]);
      asm volatile("" : "+v"(w) : : "memory");
      x[i] = __builtin_bit_cast(Piece<T, V>, w);
    }
  }
}

template <typename T, int V, int NV, int LPR, int MODE>
__device__ __forceinline__ void load_vector(float (&v)[NV][V], const void* p, const Columns<V, LPR, NV, MODE>& c) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    Piece<T, V> w = (Piece<T, V>)(T)0.f;
    if (c.there(i)) w = *(const Piece<T, V>*)((const T*)p + c.col[i]);
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] = (float)w[j];
  }
}

// y = (x - mean) / sqrt(var + eps) g + b.  Bound by memory: x once, y once, at the rate of a copy (512000 rows of 128 bf16: 49.6 us, 5.3
// TB/s; 8000 of 8192: 50.5, 5.2; of 8191, whose every other row is off the words' alignment: 62, 4.2; 4503 of 4099 fp32: 31, 4.8).
template <typename T, int V, int LPR, int NV, int MODE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(Params p) {
  constexpr int RPB = THREADS / LPR;
  typedef Meeting<LPR, THREADS> Waves;
  __shared__ typename Waves::Memory lds;
  const Columns<V, LPR, NV, MODE> c(threadIdx.x % LPR, p.d);
  Waves waves(lds, c.owned());
  const bool masked = c.masked();
  float g[NV][V], b[NV][V];
  load_vector<T>(g, p.g, c);
  load_vector<T>(b, p.b, c);
  const int step = gridDim.x * RPB;
  const int first_row = first_turn<LPR, THREADS>(p);
  Walk at(p, first_row + (LPR < 64 ? threadIdx.x % 64 / LPR : 0));
  bool ok = at.valid(p);
  Piece<T, V> x[NV];
  load_row<T>(x, p.x, at, ok, c);
  Walk ahead = at.next(p, step);
  for (int first = LPR > 64 ? first_of_workgroup<LPR, THREADS>(p) : first_row; first < p.rows; first += step) {
    // the next turn's rows, and the length for the one after it, are under way while this one's are worked on
    const Walk ahead2 = ahead.next(p, step);
    const bool ok_ahead = ahead.valid(p);
    Piece<T, V> x_ahead[NV];
    load_row<T>(x_ahead, p.x, ahead, ok_ahead, c);
    float y[NV][V];
    // (no row of the wave counts: nothing to do; rows of several waves meet at barriers, which their whole workgroup has to reach)
    if (LPR <= 64 ? __builtin_amdgcn_ballot_w64(ok) != 0 : RPB > 1 || ok) {
      Shares s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) y[i][j] = (float)x[i][j];
      auto sum = [&](auto all) {
        s.s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) s.s += decltype(all)::value || c.own(i, j) ? y[i][j] : 0.f;
      };
      // (a piece past the row holds zeros)
      if (MODE == VALUES && masked) sum(std::false_type()); else sum(std::true_type());
      s.s = lanes_sum<(LPR < 64 ? LPR : 64)>(s.s);
      float share = p.inv_d;
      if constexpr (LPR > 64) share = waves.inv_n;
      const float mean = s.s * share;              // the row's, or of several waves the wave's
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) y[i][j] -= mean;
      auto squares = [&](auto all) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float own = decltype(all)::value || c.own(i, j) ? y[i][j] : 0.f;
            s.squares = fmaf(own, own, s.squares);
          }
      };
      if (masked) squares(std::false_type()); else squares(std::true_type());
      s.squares = lanes_sum<(LPR < 64 ? LPR : 64)>(s.squares * p.inv_d);
      if constexpr (LPR > 64) {
        const float row_mean = waves.join(s, p.inv_d);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) y[i][j] = (float)x[i][j] - row_mean;
      }
      const float r = __builtin_amdgcn_rsqf(s.squares + p.eps);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) y[i][j] = fmaf(y[i][j] * r, g[i][j], b[i][j]);
    }
    if (at.r < p.rows) {
      T* row = (T*)p.out.data + at.u * p.out.user + at.l * p.out.row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!c.there(i)) continue;
        Piece<T, V> w;
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = (T)(ok ? y[i][j] : 0.f);
        *(Piece<T, V>*)(row + c.col[i]) = w;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = x_ahead[i];
    at = ahead;
    ok = ok_ahead;
    ahead = ahead2;
  }
}

// dx = r (q - mean(q) - xh mean(q xh)), q = dy g, and the workgroup's share of sum dy xh and sum dy: x and dy are read once for both.
// Bound by memory (512000 rows of 128, x bf16, gradients fp32: 125 us, 5.2 TB/s; 7161 of 8192: 112, 5.2; gradients bf16: 81, 4.3, where a
// row's arithmetic no longer hides; widths of 16 values a lane: 5461 of 12288, gradients fp32, 138, 4.9; 4096 of 16383, 164, 4.1, one of
// three kernels that spill, 3 to 9 registers a lane: bf16 rows off a piece past 8192, fp32 rows past 12288 but for 16384).  Workgroups stay for the whole launch, so the column sums leave the chip once for each: 16 waves
// in one keep those few (256 pairs of rows at width 8192: 17 MB written and read).  Beside the centred squares a
// row's sums of q and q (x - mean) are taken.
template <typename T, typename U, int V, int LPR, int NV, int MODE>
__global__ __launch_bounds__(1024) void grad_kernel(Params p) {
  constexpr int THREADS = 1024, RPB = THREADS / LPR, GROUPS = LPR < 64 ? THREADS / 64 : RPB, WIDE = LPR * NV * V;
  constexpr bool AHEAD = NV * V <= 8;                    // room for the next turn's rows beside this one's (16 waves leave 128 registers each)
  typedef Meeting<LPR, THREADS> Waves;
  __shared__ typename Waves::Memory lds;
  __shared__ float sums[GROUPS > 1 ? GROUPS * WIDE : 1];
  const Columns<V, LPR, NV, MODE> c(threadIdx.x % LPR, p.d);
  Waves waves(lds, c.owned());
  const bool masked = c.masked();
  float g[NV][V], dg[NV][V], db[NV][V];
  load_vector<T>(g, p.g, c);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.f;
  const int step = gridDim.x * RPB;
  const int first_row = first_turn<LPR, THREADS>(p);
  Walk at(p, first_row + (LPR < 64 ? threadIdx.x % 64 / LPR : 0));
  bool ok = at.valid(p);
  Piece<T, V> x[NV];
  Piece<U, V> dy[NV];
  load_row<T>(x, p.x, at, ok, c);
  load_row<U>(dy, p.dy, at, ok, c);
  Walk ahead = at.next(p, step);
  for (int first = LPR > 64 ? first_of_workgroup<LPR, THREADS>(p) : first_row; first < p.rows; first += step) {
    const Walk ahead2 = ahead.next(p, step);
    const bool ok_ahead = ahead.valid(p);
    Piece<T, V> x_ahead[NV];
    Piece<U, V> dy_ahead[NV];
    if constexpr (AHEAD) {
      load_row<T>(x_ahead, p.x, ahead, ok_ahead, c);
      load_row<U>(dy_ahead, p.dy, ahead, ok_ahead, c);
    }
    float xc[NV][V];
    if (LPR <= 64 ? __builtin_amdgcn_ballot_w64(ok) != 0 : RPB > 1 || ok) {
      constexpr int WAVE = LPR < 64 ? LPR : 64;
      Shares s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) xc[i][j] = (float)x[i][j];
      auto sum = [&](auto all) {
        s.s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) s.s += decltype(all)::value || c.own(i, j) ? xc[i][j] : 0.f;
      };
      if (MODE == VALUES && masked) sum(std::false_type()); else sum(std::true_type());
      s.s = lanes_sum<WAVE>(s.s);
      float share = p.inv_d;
      if constexpr (LPR > 64) share = waves.inv_n;
      const float mean = s.s * share;              // the row's, or of several waves the wave's
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) xc[i][j] -= mean;
      auto sums = [&](auto all) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const bool mine = decltype(all)::value || c.own(i, j);
            const float own = mine ? xc[i][j] : 0.f, q = mine ? (float)dy[i][j] * g[i][j] : 0.f;
            s.squares = fmaf(own, own, s.squares);
            s.q += q;
            s.qx = fmaf(q, own, s.qx);
          }
      };
      if (masked) sums(std::false_type()); else sums(std::true_type());
      s.squares = lanes_sum<WAVE>(s.squares * p.inv_d);
      s.q = lanes_sum<WAVE>(s.q);
      s.qx = lanes_sum<WAVE>(s.qx);
      if constexpr (LPR > 64) {
        const float row_mean = waves.join(s, p.inv_d);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) xc[i][j] = (float)x[i][j] - row_mean;
      }
      const float r = __builtin_amdgcn_rsqf(s.squares + p.eps);
      const float k1 = -(s.qx * p.inv_d) * r * r * r, k2 = -(s.q * p.inv_d) * r;       // dx = r q + k1 (x - mean) + k2
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float v = (float)dy[i][j], rv = r * v;                  // (a row that does not count: v = 0, x - mean = 0)
          db[i][j] += v;
          dg[i][j] = fmaf(rv, xc[i][j], dg[i][j]);
          xc[i][j] = fmaf(rv, g[i][j], fmaf(k1, xc[i][j], k2));
        }
    }
    if constexpr (AHEAD) {
      landed<T, V>(x_ahead);
      landed<U, V>(dy_ahead);
    }
    if (at.r < p.rows) {
      U* row = (U*)p.out.data + at.u * p.out.user + at.l * p.out.row;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!c.there(i)) continue;
        Piece<U, V> w;
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = (U)(ok ? xc[i][j] : 0.f);
        *(Piece<U, V>*)(row + c.col[i]) = w;
      }
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < NV; ++i) { x[i] = x_ahead[i]; dy[i] = dy_ahead[i]; }
    } else {
      load_row<T>(x, p.x, ahead, ok_ahead, c);
      load_row<U>(dy, p.dy, ahead, ok_ahead, c);
    }
    // Rows of one wave, gradients in 32 bits: until the stores are done no wave asks for more, which the memory rewards (512000 rows
    // of 128: 127 us for 131, of 77: 81 for 89; rows of several waves, which barriers hold together: 106 for 88, gradients in 16
    // bits: 81 for 79).
    if constexpr (LPR <= 64 && sizeof(U) == 4) __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    at = ahead;
    ok = ok_ahead;
    ahead = ahead2;
  }
  // columns: the rows of a wave, then the workgroup's groups of rows
  float* part = p.part + (size_t)blockIdx.x * 2 * p.d;
  auto leave = [&](float (&v)[NV][V], float* out) {
    if constexpr (GROUPS == 1) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (c.own(i, j)) out[c.col[i] + j] = v[i][j];
    } else {
      if constexpr (LPR < 64) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j)
#pragma unroll
            for (int o = LPR; o < 64; o <<= 1) v[i][j] += __shfl_xor(v[i][j], o);
      }
      float* mine = sums + threadIdx.x / (LPR < 64 ? 64 : LPR) * WIDE;
      if (LPR >= 64 || (threadIdx.x & 63) < LPR)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (c.own(i, j)) mine[c.col[i] + j] = v[i][j];
      __syncthreads();
      for (int i = threadIdx.x; i < p.d; i += THREADS) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) t += sums[k * WIDE + i];
        out[i] = t;
      }
    }
  };
  leave(dg, part);
  __syncthreads();
  leave(db, part + p.d);
}

// ------------------------------------------------------------------------------------ host
struct Shape { int lpr, nv, mode, v; };

// Lanes and pieces of a row, for pieces of `v` values: up to `most` pieces a lane, as few places for pieces as hold the row; at equal
// count as few lanes.  A row wider than 1024 lanes hold that way has as many a lane as it needs.
constexpr Shape shape(int d, int v, int most) {
  if (d < v) return {8, 1, PIECES, 1};
  const int pieces = (d + v - 1) / v;
  Shape s = {1, 1, 0, v};
  while (s.lpr < pieces && s.lpr < 64) s.lpr *= 2;
  if (pieces > 64) {
    s.lpr = 1024;
    s.nv = (pieces + 1023) / 1024;
    for (int lpr = 512; lpr >= 64; lpr /= 2) {
      const int nv = (pieces + lpr - 1) / lpr;
      if (nv <= most && lpr * nv <= s.lpr * s.nv) { s.lpr = lpr; s.nv = nv; }
    }
  }
  s.mode = d % v ? VALUES : pieces == s.lpr * s.nv ? FULL : PIECES;
  return s;
}

// pieces a lane: in the forward pass four in one wave before a row takes several, which meet in LDS (64 million bf16 values in rows of 2500: 53
// us for 58 with up to two, 58 with one; of 520: 67, 66, 80; of 4096 or 8192 50, 50, 51); in the backward pass 8 or 12 values,
// beside their column sums and the next turn's, more only where a workgroup's lanes are too few
constexpr int most_pieces(int v, bool backward) { return !backward ? 4 : v == 4 ? 3 : 1; }

// whether some width has this shape: every launch below asserts it, so that nothing is built that no call reaches
constexpr bool reached(int v, bool backward, int lpr, int nv, int mode, int per_piece) {
  for (int pieces = lpr * nv; pieces > 0; --pieces)
    for (int d = pieces * v; d > 0 && d >= pieces * v - 1; --d) {
      const Shape s = shape(d, v, most_pieces(v, backward));
      if (d <= LONGER_MAX_NORM_WIDTH && s.lpr == lpr && s.nv == nv && s.mode == mode && s.v == per_piece) return true;
    }
  return false;
}

// Workgroups of a launch: as many as the card holds at once, each with its share of the turns (a few more than it holds would take
// a second round for themselves), or a turn each.
template <typename K>
inline unsigned resident(K kernel, int threads) {
  int n = 0;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0) != hipSuccess || n < 1) n = 1;
  return 256u * n;
}

inline void set_step(Params& p, unsigned grid, int rows_per_turn, bool spread) {
  p.spread = spread;
  const int64_t step = (int64_t)grid * rows_per_turn;
  p.step_u = (int)(step / p.L);
  p.step_l = (int)(step % p.L);
}

template <typename T, int V, int LPR, int NV, int MODE>
inline void launch_norm(Params& p, hipStream_t st) {
  static_assert(reached(16 / sizeof(T), false, LPR, NV, MODE, V), "no width takes this kernel");
  constexpr int THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
  static const unsigned most = resident(norm_kernel<T, V, LPR, NV, MODE, THREADS>, THREADS);
  const unsigned turns = ((unsigned)p.rows + RPB - 1) / RPB;
  unsigned grid = turns < most ? turns : most;
  // ragged users: shares of eight turns, dealt as workgroups end, where a workgroup has 32 turns or more (users of up to 5000 bf16 rows,
  // 1.3 / 2.5 million of 128: 93 / 176 us for 99 / 190, 500000 of 512: 141 for 151, 5 million of 32: 90 for 94; from 8 turns on: 1
  // million of 128 73 for 75, but 500000 of 128 40.5 for 39.5 and 1.3 million of 32 29 for 26)
  const bool dealt = p.lens && turns >= 32 * most && p.rows < (1 << 30);      // (two steps past the last row stay below 2^31)
  if (dealt) grid = turns / 8;
  set_step(p, grid, RPB, p.lens && !dealt);
  norm_kernel<T, V, LPR, NV, MODE, THREADS><<<grid, THREADS, 0, st>>>(p);
}
template <typename T, int V, int LPR, int NV>
inline void launch_norm(Params& p, int mode, hipStream_t st) {
  // (with one lane or two every lane has its piece, and one lane's is whole)
  if constexpr (LPR > 2) if (mode == PIECES) return launch_norm<T, V, LPR, NV, PIECES>(p, st);
  if constexpr (LPR > 1) if (mode == VALUES) return launch_norm<T, V, LPR, NV, VALUES>(p, st);
  launch_norm<T, V, LPR, NV, FULL>(p, st);
}

template <typename T, int V>
inline void norm(Params& p, hipStream_t st) {
  const Shape s = shape(p.d, V, most_pieces(V, false));
  if (s.v == 1) return launch_norm<T, 1, 8, 1, PIECES>(p, st);
  switch (s.lpr * 8 + s.nv) {
    case 1 * 8 + 1: return launch_norm<T, V, 1, 1>(p, s.mode, st);
    case 2 * 8 + 1: return launch_norm<T, V, 2, 1>(p, s.mode, st);
    case 4 * 8 + 1: return launch_norm<T, V, 4, 1>(p, s.mode, st);
    case 8 * 8 + 1: return launch_norm<T, V, 8, 1>(p, s.mode, st);
    case 16 * 8 + 1: return launch_norm<T, V, 16, 1>(p, s.mode, st);
    case 32 * 8 + 1: return launch_norm<T, V, 32, 1>(p, s.mode, st);
    case 64 * 8 + 1: return launch_norm<T, V, 64, 1>(p, s.mode, st);
    case 64 * 8 + 2: return launch_norm<T, V, 64, 2>(p, s.mode, st);
    case 64 * 8 + 3: return launch_norm<T, V, 64, 3>(p, s.mode, st);
    case 64 * 8 + 4: return launch_norm<T, V, 64, 4>(p, s.mode, st);
    case 128 * 8 + 3: return launch_norm<T, V, 128, 3>(p, s.mode, st);
    case 128 * 8 + 4: return launch_norm<T, V, 128, 4>(p, s.mode, st);
    case 256 * 8 + 3: return launch_norm<T, V, 256, 3>(p, s.mode, st);
    case 256 * 8 + 4: return launch_norm<T, V, 256, 4>(p, s.mode, st);
    case 512 * 8 + 3: return launch_norm<T, V, 512, 3>(p, s.mode, st);
    case 512 * 8 + 4: return launch_norm<T, V, 512, 4>(p, s.mode, st);
  }
  if constexpr (V == 4) {
    if (s.nv == 3) launch_norm<T, V, 1024, 3>(p, s.mode, st);
    else launch_norm<T, V, 1024, 4>(p, s.mode, st);
  }
}

// The backward launch; the workgroups that it takes (at most `most`), each of which leaves its column sums.
template <typename T, typename U, int V, int LPR, int NV, int MODE>
inline unsigned launch_grad(Params& p, unsigned most, float* only, hipStream_t st) {
  static_assert(reached(16 / sizeof(T), true, LPR, NV, MODE, V), "no width takes this kernel");
  static const unsigned held = resident(grad_kernel<T, U, V, LPR, NV, MODE>, 1024);
  const unsigned turns = ((unsigned)p.rows + 1024 / LPR - 1) / (1024 / LPR);
  unsigned grid = turns < held ? turns : held;
  if (grid > most) grid = most;
  // (up to two turns one workgroup takes alone, and leaves the sums themselves: two turns of rows of 32 to 8192 values, 7.6 to 8.0 us a
  // call for 9.9 to 10.4, 4.3 to 6.5 for 5.2 to 7.5 in a graph; of four turns 7.7 to 9.4 for 10.2 to 10.6, but 6.5 to 9.4 for 5.2 to
  // 7.6 in a graph)
  if (turns <= 2) grid = 1;
  set_step(p, grid, 1024 / LPR, p.lens != nullptr);
  if (grid == 1) p.part = only;
  grad_kernel<T, U, V, LPR, NV, MODE><<<grid, 1024, 0, st>>>(p);
  return grid;
}
template <typename T, typename U, int V, int LPR, int NV>
inline unsigned launch_grad(Params& p, int mode, unsigned most, float* only, hipStream_t st) {
  if constexpr (LPR > 2) if (mode == PIECES) return launch_grad<T, U, V, LPR, NV, PIECES>(p, most, only, st);
  if constexpr (LPR > 1) if (mode == VALUES) return launch_grad<T, U, V, LPR, NV, VALUES>(p, most, only, st);
  return launch_grad<T, U, V, LPR, NV, FULL>(p, most, only, st);
}

template <typename T, typename U, int V>
inline unsigned grad(Params& p, unsigned most, float* only, hipStream_t st) {
  const Shape s = shape(p.d, V, most_pieces(V, true));
  if (s.v == 1) return launch_grad<T, U, 1, 8, 1, PIECES>(p, most, only, st);
  switch (s.lpr * 8 + s.nv) {
    case 1 * 8 + 1: return launch_grad<T, U, V, 1, 1>(p, s.mode, most, only, st);
    case 2 * 8 + 1: return launch_grad<T, U, V, 2, 1>(p, s.mode, most, only, st);
    case 4 * 8 + 1: return launch_grad<T, U, V, 4, 1>(p, s.mode, most, only, st);
    case 8 * 8 + 1: return launch_grad<T, U, V, 8, 1>(p, s.mode, most, only, st);
    case 16 * 8 + 1: return launch_grad<T, U, V, 16, 1>(p, s.mode, most, only, st);
    case 32 * 8 + 1: return launch_grad<T, U, V, 32, 1>(p, s.mode, most, only, st);
    case 64 * 8 + 1: return launch_grad<T, U, V, 64, 1>(p, s.mode, most, only, st);
  }
  if constexpr (V == 4) {
    switch (s.lpr * 8 + s.nv) {
      case 64 * 8 + 2: return launch_grad<T, U, V, 64, 2>(p, s.mode, most, only, st);
      case 64 * 8 + 3: return launch_grad<T, U, V, 64, 3>(p, s.mode, most, only, st);
      case 128 * 8 + 2: return launch_grad<T, U, V, 128, 2>(p, s.mode, most, only, st);
      case 128 * 8 + 3: return launch_grad<T, U, V, 128, 3>(p, s.mode, most, only, st);
      case 256 * 8 + 2: return launch_grad<T, U, V, 256, 2>(p, s.mode, most, only, st);
      case 256 * 8 + 3: return launch_grad<T, U, V, 256, 3>(p, s.mode, most, only, st);
      case 512 * 8 + 2: return launch_grad<T, U, V, 512, 2>(p, s.mode, most, only, st);
      case 512 * 8 + 3: return launch_grad<T, U, V, 512, 3>(p, s.mode, most, only, st);
      case 1024 * 8 + 2: return launch_grad<T, U, V, 1024, 2>(p, s.mode, most, only, st);
      case 1024 * 8 + 3: return launch_grad<T, U, V, 1024, 3>(p, s.mode, most, only, st);
      default: return launch_grad<T, U, V, 1024, 4>(p, s.mode, most, only, st);
    }
  } else {
    switch (s.lpr * 8 + s.nv) {
      case 128 * 8 + 1: return launch_grad<T, U, V, 128, 1>(p, s.mode, most, only, st);
      case 256 * 8 + 1: return launch_grad<T, U, V, 256, 1>(p, s.mode, most, only, st);
      case 512 * 8 + 1: return launch_grad<T, U, V, 512, 1>(p, s.mode, most, only, st);
      case 1024 * 8 + 1: return launch_grad<T, U, V, 1024, 1>(p, s.mode, most, only, st);
      default: return launch_grad<T, U, V, 1024, 2>(p, s.mode, most, only, st);
    }
  }
}

// inst_norm_*.hip
void norm_f32(Params& p, hipStream_t st);
void norm_bf16(Params& p, hipStream_t st);
unsigned grad_f32(Params& p, unsigned most, float* only, hipStream_t st);
unsigned grad_bf16_f32(Params& p, unsigned most, float* only, hipStream_t st);
unsigned grad_bf16(Params& p, unsigned most, float* only, hipStream_t st);

}  // namespace ln
}  // namespace longer
