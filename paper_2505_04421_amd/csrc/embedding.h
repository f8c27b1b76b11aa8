// What the embedding's kernels share: rows of tokens, pieces of a row, and the mask that a counter-based generator gives.
#pragma once
#include "device.h"
#include "rows.h"

#include <algorithm>
#include <cmath>

namespace longer {
namespace emb {

struct Rows { char* data; int64_t user, row; };      // strides in elements

// n / by for n below 2^31: mul = ceil(2^(31 + shift) / by) is off by less than by <= 2^shift, which n times is below one step
struct Divider {
  uint32_t mul, shift;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> (31 + shift)); }
};
inline Divider divider(uint32_t by) {
  uint32_t shift = 0;
  while (((uint64_t)1 << shift) < by) ++shift;
  return {(uint32_t)((((uint64_t)1 << (31 + shift)) + by - 1) / by), shift};
}

// The lanes of a workgroup of 256 that hold a row, a piece each: as many as it has pieces (a wider row: all of them, in turns), so that no power of two
// has to be filled; what is left over of a workgroup idles.  A lane's piece is the same in all its rows.
struct Deal { Divider by_lanes; uint32_t lanes, per_turn; };
struct Seat { uint32_t lane, row; bool taken; };
__device__ __forceinline__ Seat seat(const Deal& d) {
  const uint32_t row = d.by_lanes(threadIdx.x);
  return {threadIdx.x - row * d.lanes, row, row < d.per_turn};
}
inline Deal deal(uint32_t pieces) {
  const uint32_t lanes = std::min(pieces, 256u);
  return {divider(lanes), lanes, 256 / lanes};
}

// The 2^k lanes, at most `most` = 2^m, that hold a row in pieces of 8 values
inline int lanes_shift(int pieces, int m) {
  int k = 0;
  while (k < m && (1 << k) < pieces) ++k;
  return k;
}

template <typename T, int V> struct Piece_ { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <typename T, int V> using Piece = typename Piece_<T, V>::type;

// A lane's piece of a row: 8 values from column c on.  Widths that 8 does not divide: the last piece is moved back to end with the row, so that
// every access is whole and inside it; its first `twice` values are its neighbour's too, and are computed and stored by both, to the
// same bits.  That asks for a row of 8 values, and for nobody who reads behind the neighbour's store (in place: no); otherwise the last piece is
// taken value by value.  Accesses are aligned to the element only, which the memory path takes at any address.
enum Kind { WHOLE, BACK, VALUES };                   // rows of whole pieces; the last piece is moved back; the last piece is taken value by value
struct Part { int c, n, twice; };                    // n: values of the row from c on, 8 or more: a whole piece
template <Kind KIND, int V = 8>
__device__ __forceinline__ Part part_of(uint32_t piece, int d) {
  const int c = piece * V;
  if (KIND == WHOLE) return {c, V, 0};
  if (KIND == VALUES) return {c, d - c, 0};
  return {min(c, d - V), V, max(c - (d - V), 0)};
}
template <typename Go>
inline void with_kind(Kind kind, Go go) {
  if (kind == WHOLE) go(std::integral_constant<Kind, WHOLE>());
  else if (kind == BACK) go(std::integral_constant<Kind, BACK>());
  else go(std::integral_constant<Kind, VALUES>());
}
inline Kind kind_of(int d, int V = 8, bool in_place = false) { return d % V == 0 ? WHOLE : d > V && !in_place ? BACK : VALUES; }

template <typename T, Kind KIND, int V = 8>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p, int n) {
  if (KIND != VALUES || n >= V) return *(const Piece<T, V>*)p;
  Piece<T, V> x;
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] = j < n ? p[j] : (T)0.f;
  return x;
}
// written once and read by another kernel: past the caches
template <typename T, Kind KIND, int V = 8>
__device__ __forceinline__ void store_piece(T* p, int n, const Piece<T, V>& x) {
  if (KIND != VALUES || n >= V) {
    __builtin_nontemporal_store(x, (Piece<T, V>*)p);
    return;
  }
#pragma unroll
  for (int j = 0; j < V - 1; ++j)
    if (j < n) p[j] = x[j];
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011): ten rounds of two 32 x 32 -> 64 bit
// products on a counter of four words under a key of two.  Half a word decides about one value: 8 values, 16 bytes of bf16, to a
// call, and a share that is a multiple of 2^-16.  A wave's call takes 187 cycles of its SIMD with the words joined in one instruction
// (275 with two exclusive ors): 65 million values in 10 us of the whole chip, of a lookup's 29 in bf16.
struct Mask { const uint64_t* key; uint32_t site, drop; };      // site: in place; drop: half-words below it drop their value (0: there is no mask)
struct Key { uint32_t k0, k1, c2, c3; };

__device__ __forceinline__ Key load_key(const Mask& m) {
  const uint64_t seed = m.key[0], step = m.key[1];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

__device__ __forceinline__ void words(const Mask& m, const Key& key, uint32_t row, uint32_t block, uint32_t (&c)[4]) {
  uint32_t k0 = key.k0, k1 = key.k1;
  c[0] = m.site | block;
  c[1] = row;
  c[2] = key.c2;
  c[3] = key.c3;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = xor3((uint32_t)(b >> 32), c[1], k0);
    c[1] = (uint32_t)b;
    c[2] = xor3((uint32_t)(a >> 32), c[3], k1);
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// x[j] where the value is kept, zero (whatever x[j] is) where it is not, for the V values of a lane's piece.  A last piece that was moved back begins in the
// words of the piece before it, which the lane before has (512000 rows of 100 in bf16 looked up: 34 us, 39 with a second call of the generator for them);
// only where that lane is of another wave or turn they are drawn again.
template <Kind KIND, int V, typename X>
__device__ __forceinline__ void drop_piece(const Mask& m, const Key& key, uint32_t row, uint32_t piece, bool first, int d, X& x) {
  constexpr int W = V / 2;
  uint32_t w[4];
  auto draw = [&](uint32_t i) {                      // the W words of piece i
    words(m, key, row, i * V / 8, w);
    if (V == 4 && (i & 1)) {
      w[0] = w[2];
      w[1] = w[3];
    }
  };
  draw(piece);
  if (KIND == BACK) {
    const bool last = (int)(piece + 1) * V > d;
    const uint32_t by = (uint32_t)d % V;             // half-words to pass over
    uint32_t v[2 * W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      v[W + k] = w[k];
      v[k] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[k], 0x138, 0xF, 0xF, true);       // the lane before
    }
    if (last && (first || (threadIdx.x & 63) == 0)) {
      draw(piece - 1);
#pragma unroll
      for (int k = 0; k < W; ++k) v[k] = w[k];
    }
#pragma unroll
    for (int step = W / 2; step; step /= 2)
      if (by & 2 * step)
#pragma unroll
        for (int k = 0; k + step < 2 * W; ++k) v[k] = v[k + step];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if (by & 1) v[k] = __builtin_amdgcn_alignbit(v[k + 1], v[k], 16);
      w[k] = last ? v[k] : w[k];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] = (w[j / 2] >> 16 * (j & 1) & 0xffff) >= m.drop ? x[j] : 0.f;
}

// ------------------------------------------------------------------------------------ host
inline int check_mask(const longer_dropout_mask* d) {
  if (!d) return 0;
  if (!(d->p >= 0. && d->p < 1.) || std::lround(65536. * d->p) > 65535) return api_error(LONGER_ERR_ARG, "p=%g: 0 to below 1 - 2^-17", d->p);
  if (d->site < 0 || d->site > 65535) return api_error(LONGER_ERR_ARG, "site=%d: 0 to 65535", d->site);
  if (!d->key || ((uintptr_t)d->key & 7)) return api_error(LONGER_ERR_ARG, "key is NULL or not aligned to 8 bytes");
  return 0;
}

inline Mask mask_of(const longer_dropout_mask* d) {
  return d ? Mask{d->key, (uint32_t)d->site << 16, (uint32_t)std::lround(65536. * d->p)} : Mask{nullptr, 0, 0};
}

// what a kept value counts
inline double kept(const longer_dropout_mask* d) { return d ? 65536. / (65536 - std::lround(65536. * d->p)) : 1.; }

inline int check_width(int d) {
  if (d <= 0 || d > LONGER_MAX_EMBEDDING_WIDTH) return api_error(LONGER_ERR_ARG, "d=%d: 1 to %d", d, LONGER_MAX_EMBEDDING_WIDTH);
  return 0;
}

inline Rows rows_of(const longer_rows* r, int B, int L) { return {(char*)r->data, B > 1 ? r->user_stride : 0, L > 1 ? r->row_stride : 0}; }

// an order's arrays (what they hold is the caller's contract, but for what a kernel checks)
inline int check_order(const longer_order* o) {
  if (!o || !o->tokens || !o->runs || !o->rows || !o->counts) return api_error(LONGER_ERR_ARG, "order: a NULL pointer");
  if (o->tokens == o->runs || o->tokens == o->rows || o->tokens == o->counts || o->runs == o->rows || o->runs == o->counts || o->rows == o->counts)
    return api_error(LONGER_ERR_ARG, "order: two of its arrays are the same memory");
  if (((uintptr_t)o->tokens | (uintptr_t)o->runs | (uintptr_t)o->rows | (uintptr_t)o->counts) & 3) return api_error(LONGER_ERR_ARG, "order is not aligned to its elements");
  return 0;
}

}  // namespace emb
}  // namespace longer
