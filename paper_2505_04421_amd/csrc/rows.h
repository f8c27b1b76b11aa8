// Host checks that the entry points on token rows (layer norm, embeddings, dropout, updates) share.
#pragma once
#include "../../include/longer.h"

#include <hip/hip_runtime.h>

namespace longer {

int api_error(int code, const char* fmt, ...);   // longer_api.hip

inline int size_of(int dtype) { return dtype == LONGER_F32 ? 4 : dtype == LONGER_BF16 ? 2 : 0; }

inline int check_tokens(int B, int L) {
  if (B <= 0 || L <= 0 || (int64_t)B * L >= ((int64_t)1 << 31) - (1 << 21)) return api_error(LONGER_ERR_ARG, "B=%d L=%d: at least 1 each, B * L below 2^31 - 2^21", B, L);
  return 0;
}

inline int check_strides(const char* name, int64_t su, int64_t sr, int B, int L) {
  const int64_t most = (int64_t)1 << 40;
  if ((B > 1 && (su < 0 || su > most)) || (L > 1 && (sr < 0 || sr > most))) return api_error(LONGER_ERR_ARG, "%s: strides %lld, %lld out of range", name, (long long)su, (long long)sr);
  return 0;
}

inline int check_rows(const longer_rows* r, const char* name, int B, int L, int d, bool written) {
  if (!r || !r->data) return api_error(LONGER_ERR_ARG, "%s is NULL", name);
  const int e = size_of(r->dtype);
  if (!e) return api_error(LONGER_ERR_ARG, "%s: dtype %d unknown", name, r->dtype);
  if ((uintptr_t)r->data % e) return api_error(LONGER_ERR_ARG, "%s is not aligned to its elements", name);
  const int64_t su = r->user_stride, sr = r->row_stride;
  if (int rc = check_strides(name, su, sr, B, L)) return rc;
  if (written) {
    // users apart and rows apart inside one user, or the other way round
    const bool rows_inside = (L == 1 || sr >= d) && (B == 1 || su >= (__int128)(L - 1) * (L > 1 ? sr : 0) + d);
    const bool users_inside = (B == 1 || su >= d) && (L == 1 || sr >= (__int128)(B - 1) * (B > 1 ? su : 0) + d);
    if (!rows_inside && !users_inside) return api_error(LONGER_ERR_ARG, "%s: rows of an output overlap (strides %lld, %lld)", name, (long long)su, (long long)sr);
  }
  return 0;
}

inline bool same(const longer_rows* a, const longer_rows* b, int B, int L) {
  return a->data == b->data && a->dtype == b->dtype && (B == 1 || a->user_stride == b->user_stride) && (L == 1 || a->row_stride == b->row_stride);
}

// An output's buffer may hold other rows between its own (those of another tensor too), so extents that cross say
// nothing; equal first values under another layout do.
inline int check_alias(const longer_rows* in, const longer_rows* out, const char* what, int B, int L) {
  if (in->data == out->data && !same(in, out, B, L)) return api_error(LONGER_ERR_ARG, "%s: the same memory under other strides or types", what);
  return 0;
}

inline int check_vector(const void* p, int dtype, const char* name) {
  if (!p) return api_error(LONGER_ERR_ARG, "%s is NULL", name);
  if ((uintptr_t)p % size_of(dtype)) return api_error(LONGER_ERR_ARG, "%s is not aligned to its elements", name);
  return 0;
}

inline int check_ids(const longer_ids* ids, const int32_t* lens, int B, int L) {
  if (!ids || !ids->data) return api_error(LONGER_ERR_ARG, "ids is NULL");
  if (ids->type != LONGER_I32 && ids->type != LONGER_I64) return api_error(LONGER_ERR_ARG, "ids: type %d unknown", ids->type);
  if ((uintptr_t)ids->data % (ids->type == LONGER_I64 ? 8 : 4)) return api_error(LONGER_ERR_ARG, "ids is not aligned to its elements");
  if ((uintptr_t)lens & 3) return api_error(LONGER_ERR_ARG, "lens is not aligned");
  return check_strides("ids", ids->user_stride, ids->row_stride, B, L);
}

inline int check_table_rows(int64_t rows) {
  if (rows < 1 || rows >= (int64_t)1 << 31) return api_error(LONGER_ERR_ARG, "a table of %lld rows: 1 to below 2^31", (long long)rows);
  return 0;
}

inline int launched(const char* what) {
  return hipGetLastError() == hipSuccess ? 0 : api_error(LONGER_ERR_HIP, "%s launch failed", what);
}

}  // namespace longer
