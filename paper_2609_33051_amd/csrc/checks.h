// Argument checks that the operators' entry points share (mixer_abi.hip, attention_abi.hip).
#pragma once

#include "../../include/sketchssm_mixer.h"

#include "host.h"
#include "mixer.h"

namespace skssm {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;

inline int elem(int dtype) { return dtype == SKSSM_F32 ? 4 : dtype == SKSSM_BF16 ? 2 : 1; }

// A row stride in elements of e bytes: at least the row, whole 16-byte pieces.
inline int check_stride(const char* what, const char* name, int64_t ld, int64_t row, int e) {
  if (ld < row) return fail(SKSSM_EINVAL, "%s: %s stride %lld is less than its row of %lld", what, name, (long long)ld, (long long)row);
  if ((ld * e) & 15) return fail(SKSSM_EALIGN, "%s: %s stride %lld is not a multiple of 16 bytes", what, name, (long long)ld);
  return SKSSM_OK;
}

// Bytes from the first to past the last element of `rows` rows.
inline size_t span(int64_t rows, int64_t ld, int64_t row, int e) { return rows > 0 ? (size_t)(((rows - 1) * ld + row) * e) : 0; }

// Arrays by address and bytes (NULL or 0 bytes: none); whether one of the first overlaps one of the second.
struct Range { const void* p; size_t n; };
template <size_t N, size_t M> bool any_overlap(const Range (&a)[N], const Range (&b)[M]) {
  for (const Range& x : a)
    for (const Range& y : b)
      if (x.n && y.n && overlap(x.p, x.n, y.p, y.n)) return true;
  return false;
}

inline int check_packed(const char* what, int batch, int64_t tokens, const int32_t* offsets) {
  if (batch < 1) return fail(SKSSM_EINVAL, "%s: batch must be >= 1", what);
  if (tokens < 0 || tokens > kMaxTokens)
    return fail(tokens < 0 ? SKSSM_EINVAL : SKSSM_EUNSUPPORTED, "%s: %lld tokens: 0 to 2^30", what, (long long)tokens);
  if (!offsets && tokens % batch) return fail(SKSSM_EINVAL, "%s: %lld tokens are not %d equal sequences (offsets is NULL)", what, (long long)tokens, batch);
  if (reinterpret_cast<uintptr_t>(offsets) & 3u) return fail(SKSSM_EALIGN, "%s: offsets not aligned", what);
  return SKSSM_OK;
}

inline Sequences sequences(int batch, int64_t tokens, const int32_t* offsets) {
  Sequences q;
  q.offsets = offsets;
  q.batch = batch;
  q.tokens = (int)tokens;
  q.each = (int)(tokens / batch);
  return q;
}

}  // namespace skssm
