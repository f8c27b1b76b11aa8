// Rows of a table by item id, with scaling and dropout (longer_embedding), and dropout of token rows (longer_dropout).
#include "embedding.h"

namespace longer {
namespace emb {

struct Ids { const char* data; int64_t user, row; const int32_t* lens; uint32_t table_rows; int wide; };

struct LookupParams {
  const char* table;
  int64_t stride;
  Ids ids;
  Rows out;
  Divider by_L;
  uint32_t n, L;
  int d;
  Deal deal;
  float factor;
  Mask mask;
};

// the row of the table that token (b, l) names, or -1
__device__ __forceinline__ int64_t item(const Ids& ids, uint32_t b, uint32_t l) {
  if (ids.lens && (int)l >= ids.lens[b]) return -1;
  const int64_t at = (int64_t)b * ids.user + (int64_t)l * ids.row;
  const int64_t id = ids.wide ? ((const int64_t*)ids.data)[at] : ((const int32_t*)ids.data)[at];
  return (uint64_t)id < ids.table_rows ? id : -1;
}

// Values of a lane's piece: 16 bytes of what is written, so that a store of the wave is one stretch without holes (fp32 rows in two stores of 16 bytes a lane,
// every other 16 to each: 512000 rows of 128 from a bf16 table in 110 us for 49, from one of 500009 fp32 rows 71 for 57, dropout 102 for 91; from 1000003
// fp32 rows, whose reads bound it, 74 for 76).
template <typename O> constexpr int kPiece = 16 / sizeof(O);

// E[r] = factor * mask * table[id of r], zeros where r is padding or names no row.  A thread finds where a row's values come from and go to, for all
// lanes that hold the row; four rows of a lane are under way at once.
template <typename T, typename O, bool DROP, Kind KIND>
__global__ __launch_bounds__(256) void lookup_kernel(LookupParams p) {
  constexpr uint32_t U = 4;
  constexpr int V = kPiece<O>;
  struct alignas(16) Way { int64_t from, to; };      // from < 0: nowhere
  __shared__ Way way[256 * U];
  const uint32_t per_turn = p.deal.per_turn, per_group = per_turn * U;
  const Seat me = seat(p.deal);
  const Key key = DROP ? load_key(p.mask) : Key{};
  for (uint32_t first = blockIdx.x * per_group; first < p.n; first += gridDim.x * per_group) {
    const uint32_t rows = min(per_group, p.n - first);
    if (first != blockIdx.x * per_group) __syncthreads();
    for (uint32_t i = threadIdx.x; i < rows; i += 256) {
      const uint32_t b = p.by_L(first + i), l = first + i - b * p.L;
      const int64_t id = item(p.ids, b, l);
      way[i] = {id < 0 ? -1 : id * p.stride, (int64_t)b * p.out.user + (int64_t)l * p.out.row};
    }
    __syncthreads();
    if (me.taken)
      for (uint32_t piece = me.lane; (int)piece * V < p.d; piece += p.deal.lanes) {
        const Part at = part_of<KIND, V>(piece, p.d);
        Way w[U];
        Piece<T, V> x[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) w[u] = way[min(me.row + u * per_turn, rows - 1)];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)             // (a token that names no row loads the table's first: no branch around a load)
          x[u] = load_piece<T, KIND, V>((const T*)p.table + max(w[u].from, (int64_t)0) + at.c, at.n);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          const uint32_t r = me.row + u * per_turn;
          if (r >= rows) break;
          Piece<float, V> y;
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = (float)x[u][j] * p.factor;
          if (DROP) drop_piece<KIND, V>(p.mask, key, first + r, piece, me.lane == 0, p.d, y);
          Piece<O, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = w[u].from >= 0 ? (O)y[j] : (O)0.f;
          store_piece<O, KIND, V>((O*)p.out.data + w[u].to + at.c, at.n, o);
        }
      }
  }
}

struct DropParams {
  Rows x, residual, out;
  const int32_t* lens;
  Divider by_L;
  uint32_t n, L;
  int d;
  Deal deal;
  Kind kind;
  float factor;
  Mask mask;
};

// Y[r] = residual[r] + factor * mask * X[r]; padding zeros, not read.  Rows' places as in the lookup.
template <typename T, bool ADD, Kind KIND>
__global__ __launch_bounds__(256) void dropout_kernel(DropParams p) {
  constexpr uint32_t U = 2;
  constexpr int V = kPiece<T>;
  struct alignas(16) Way { int64_t from, to; };      // from < 0: padding
  __shared__ Way way[256 * U];
  __shared__ int64_t add_from[ADD ? 256 * U : 1];
  const uint32_t per_turn = p.deal.per_turn, per_group = per_turn * U;
  const Seat me = seat(p.deal);
  const Key key = load_key(p.mask);
  for (uint32_t first = blockIdx.x * per_group; first < p.n; first += gridDim.x * per_group) {
    const uint32_t rows = min(per_group, p.n - first);
    if (first != blockIdx.x * per_group) __syncthreads();
    for (uint32_t i = threadIdx.x; i < rows; i += 256) {
      const uint32_t b = p.by_L(first + i), l = first + i - b * p.L;
      const bool there = !p.lens || (int)l < p.lens[b];
      way[i] = {there ? (int64_t)b * p.x.user + (int64_t)l * p.x.row : -1, (int64_t)b * p.out.user + (int64_t)l * p.out.row};
      if (ADD) add_from[i] = (int64_t)b * p.residual.user + (int64_t)l * p.residual.row;
    }
    __syncthreads();
    if (me.taken)
      for (uint32_t piece = me.lane; (int)piece * V < p.d; piece += p.deal.lanes) {
        const Part at = part_of<KIND, V>(piece, p.d);
        Way w[U];
        Piece<T, V> x[U], add[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          const uint32_t i = min(me.row + u * per_turn, rows - 1);
          w[u] = way[i];
          if (w[u].from >= 0) {
            x[u] = load_piece<T, KIND, V>((const T*)p.x.data + w[u].from + at.c, at.n);
            if (ADD) add[u] = load_piece<T, KIND, V>((const T*)p.residual.data + add_from[i] + at.c, at.n);
          }
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          const uint32_t r = me.row + u * per_turn;
          if (r >= rows) break;
          Piece<float, V> y = 0.f;
          if (w[u].from >= 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = (float)x[u][j] * p.factor;
            drop_piece<KIND, V>(p.mask, key, first + r, piece, me.lane == 0, p.d, y);
            if (ADD)
#pragma unroll
              for (int j = 0; j < V; ++j) y[j] += (float)add[u][j];
          }
          Piece<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = (T)y[j];
          store_piece<T, KIND, V>((T*)p.out.data + w[u].to + at.c, at.n, o);
        }
      }
  }
}

// ------------------------------------------------------------------------------------ host
static unsigned groups(uint32_t n, const Deal& deal, uint32_t turns) {
  return std::min((n + deal.per_turn * turns - 1) / (deal.per_turn * turns), 1u << 22);      // (a grid counts threads in 32 bits)
}

template <typename T, typename O>
static void lookup(const LookupParams& p, hipStream_t st) {
  const unsigned g = groups(p.n, p.deal, 4);
  auto go = [&](auto kind) {
    constexpr Kind KIND = decltype(kind)::value;
    if (p.mask.drop) lookup_kernel<T, O, true, KIND><<<g, 256, 0, st>>>(p);
    else lookup_kernel<T, O, false, KIND><<<g, 256, 0, st>>>(p);
  };
  with_kind(kind_of(p.d, kPiece<O>), go);
}

template <typename T>
static void dropout(const DropParams& p, hipStream_t st) {
  const unsigned g = groups(p.n, p.deal, 2);
  auto go = [&](auto kind) {
    constexpr Kind KIND = decltype(kind)::value;
    if (p.residual.data) dropout_kernel<T, true, KIND><<<g, 256, 0, st>>>(p);
    else dropout_kernel<T, false, KIND><<<g, 256, 0, st>>>(p);
  };
  with_kind(p.kind, go);
}

}  // namespace emb
}  // namespace longer

using namespace longer;

extern "C" {

int longer_embedding(const longer_table* table, const longer_ids* ids, const int32_t* lens, int B, int L, int d, float scale,
                     const longer_dropout_mask* drop, const longer_rows* e, void* stream) {
  int rc = check_tokens(B, L);
  if (!rc) rc = emb::check_width(d);
  if (!rc) rc = check_ids(ids, lens, B, L);
  if (!rc && (!table || !table->data)) rc = api_error(LONGER_ERR_ARG, "table is NULL");
  if (!rc && !size_of(table->dtype)) rc = api_error(LONGER_ERR_ARG, "table: dtype %d unknown", table->dtype);
  if (!rc && (uintptr_t)table->data % size_of(table->dtype)) rc = api_error(LONGER_ERR_ARG, "table is not aligned to its elements");
  if (!rc) rc = check_table_rows(table->rows);
  if (!rc && (table->row_stride < 0 || table->row_stride > (int64_t)1 << 40)) rc = api_error(LONGER_ERR_ARG, "table: row stride %lld out of range", (long long)table->row_stride);
  if (!rc) rc = check_rows(e, "e", B, L, d, true);
  if (!rc && e->data == table->data) rc = api_error(LONGER_ERR_ARG, "e may not be the table");
  if (!rc) rc = emb::check_mask(drop);
  const double factor = scale * emb::kept(rc ? nullptr : drop);
  if (!rc && !std::isfinite((float)factor)) rc = api_error(LONGER_ERR_ARG, "scale=%g: not an fp32 number", scale);
  if (rc) return rc;
  const emb::LookupParams p = {(const char*)table->data, table->row_stride,
                               {(const char*)ids->data, B > 1 ? ids->user_stride : 0, L > 1 ? ids->row_stride : 0, lens, (uint32_t)table->rows, ids->type == LONGER_I64},
                               emb::rows_of(e, B, L), emb::divider(L), (uint32_t)B * L, (uint32_t)L, d, emb::deal(e->dtype == LONGER_F32 ? (d + 3) / 4 : (d + 7) / 8), (float)factor, emb::mask_of(drop)};
  hipStream_t st = (hipStream_t)stream;
  if (table->dtype == LONGER_F32) e->dtype == LONGER_F32 ? emb::lookup<float, float>(p, st) : emb::lookup<float, __bf16>(p, st);
  else e->dtype == LONGER_F32 ? emb::lookup<__bf16, float>(p, st) : emb::lookup<__bf16, __bf16>(p, st);
  return launched("embedding");
}

int longer_dropout(const longer_rows* x, const longer_rows* residual, const int32_t* lens, int B, int L, int d,
                   const longer_dropout_mask* drop, const longer_rows* y, void* stream) {
  int rc = check_tokens(B, L);
  if (!rc) rc = emb::check_width(d);
  if (!rc) rc = check_rows(x, "x", B, L, d, false);
  if (!rc && residual) rc = check_rows(residual, "residual", B, L, d, false);
  if (!rc) rc = check_rows(y, "y", B, L, d, true);
  if (!rc && (x->dtype != y->dtype || (residual && residual->dtype != y->dtype))) rc = api_error(LONGER_ERR_ARG, "x, residual and y have one dtype");
  if (!rc) rc = check_alias(x, y, "x and y", B, L);
  if (!rc && residual) rc = check_alias(residual, y, "residual and y", B, L);
  if (!rc && ((uintptr_t)lens & 3)) rc = api_error(LONGER_ERR_ARG, "lens is not aligned");
  if (!rc && !drop) rc = api_error(LONGER_ERR_ARG, "drop is NULL");
  if (!rc) rc = emb::check_mask(drop);
  if (rc) return rc;
  const emb::DropParams p = {emb::rows_of(x, B, L), residual ? emb::rows_of(residual, B, L) : emb::Rows{}, emb::rows_of(y, B, L), lens, emb::divider(L), (uint32_t)B * L,
                             (uint32_t)L, d, emb::deal(x->dtype == LONGER_F32 ? (d + 3) / 4 : (d + 7) / 8), emb::kind_of(d, x->dtype == LONGER_F32 ? 4 : 8, x->data == y->data || (residual && residual->data == y->data)), (float)emb::kept(drop), emb::mask_of(drop)};
  if (x->dtype == LONGER_F32) emb::dropout<float>(p, (hipStream_t)stream);
  else emb::dropout<__bf16>(p, (hipStream_t)stream);
  return launched("dropout");
}

}  // extern "C"
