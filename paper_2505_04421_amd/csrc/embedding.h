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

// The 2^k lanes, at most `most` = 2^m, that hold a row in pieces of 8 values
inline int lanes_shift(int pieces, int m) {
  int k = 0;
  while (k < m && (1 << k) < pieces) ++k;
  return k;
}

template <typename T, int V> struct Piece_ { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <typename T, int V> using Piece = typename Piece_<T, V>::type;

// 8 values of a row, of which `n` are the row's (the others come as zeros and are not stored)
template <typename T>
__device__ __forceinline__ Piece<T, 8> load8(const T* p, int n) {
  if (n >= 8) return *(const Piece<T, 8>*)p;
  Piece<T, 8> x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j < n ? p[j] : (T)0.f;
  return x;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const Piece<T, 8>& x) {
  if (n >= 8) {
    __builtin_nontemporal_store(x, (Piece<T, 8>*)p);
    return;
  }
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < n) p[j] = x[j];
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011): ten rounds of two 32 x 32 -> 64 bit
// products on a counter of four words under a key of two.  Half a word decides about one value: 8 values, 16 bytes of bf16, to a
// call, and a share that is a multiple of 2^-16.
struct Mask { const uint64_t* key; uint32_t site, drop; };      // site: in place; drop: half-words below it drop their value (0: there is no mask)
struct Key { uint32_t k0, k1, c2, c3; };

__device__ __forceinline__ Key load_key(const Mask& m) {
  const uint64_t seed = m.key[0], step = m.key[1];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
}

// x[j] where value j of the piece is kept, zero (whatever x[j] is) where it is not
template <typename V>
__device__ __forceinline__ void drop8(const Mask& m, const Key& key, uint32_t row, uint32_t piece, V& x) {
  uint32_t c[4] = {m.site | piece, row, key.c2, key.c3}, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)b;
    c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (c[j / 2] >> 16 * (j & 1) & 0xffff) >= m.drop ? x[j] : 0.f;
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
  if (((uintptr_t)o->tokens | (uintptr_t)o->runs | (uintptr_t)o->rows | (uintptr_t)o->counts) & 3) return api_error(LONGER_ERR_ARG, "order is not aligned to its elements");
  return 0;
}

}  // namespace emb
}  // namespace longer
