// Strided tensors of heads, [batch][token][head][D] with the elements of a head beside one another: host-side checks.
#pragma once
#include "common.h"

namespace dat {

struct HeadsShape { int64_t batch, tokens, heads, D; };

// The dimensions of a tensor from the widest stride to the narrowest; false where some of its elements lie on one another (or may).
struct HeadsDims { int64_t stride[3], count[3], inner[3]; bool apart; };   // inner: elements from the first to behind the last of what lies inside
inline HeadsDims heads_dims(const dat_heads& t, const HeadsShape& s) {
  HeadsDims d;
  const int64_t stride[3] = {t.batch, t.token, t.head}, count[3] = {s.batch, s.tokens, s.heads};
  int order[3] = {0, 1, 2};
  auto wider = [&](int a, int b) { return (count[a] > 1 ? stride[a] : 0) > (count[b] > 1 ? stride[b] : 0); };
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j) if (wider(order[j], order[i])) { const int x = order[i]; order[i] = order[j]; order[j] = x; }
  int64_t inner = s.D;
  d.apart = true;
  for (int i = 2; i >= 0; --i) {
    d.count[i] = count[order[i]];
    d.stride[i] = d.count[i] > 1 ? stride[order[i]] : 0;
    d.inner[i] = inner;
    if (d.count[i] > 1 && d.stride[i] < inner) d.apart = false;
    if (d.count[i] > 1) inner += d.stride[i] * (d.count[i] - 1);
  }
  return d;
}
inline int64_t heads_extent(const dat_heads& t, const HeadsShape& s) {
  const HeadsDims d = heads_dims(t, s);
  return d.inner[0] + (d.count[0] > 1 ? d.stride[0] * (d.count[0] - 1) : 0);
}

// Whether elements of two tensors with the same strides, the second (b) `delta` elements behind the first (a), are the same one.
inline bool nested_overlap(int64_t delta, const HeadsDims& a, const HeadsDims& b, int level, int64_t D) {
  if (level == 3) return delta < D && -delta < D;
  const int64_t s = a.stride[level] ? a.stride[level] : b.stride[level];     // a's index less b's: above -b's count, below a's
  if (a.count[level] <= 1 && b.count[level] <= 1) return nested_overlap(delta, a, b, level + 1, D);
  int64_t i = delta / s;
  if (delta < 0 && i * s != delta) --i;                 // floor
  for (int64_t k = i; k <= i + 1; ++k)
    if (k < a.count[level] && -k < b.count[level] && nested_overlap(delta - k * s, a, b, level + 1, D)) return true;
  return false;
}

// Whether two tensors share an element: exact where their strides agree (parts of one tensor), by their extents elsewhere.
inline bool heads_overlap(const dat_heads& x, const HeadsShape& sx, const dat_heads& y, const HeadsShape& sy, size_t width) {
  if (sx.batch * sx.tokens * sx.heads == 0 || sy.batch * sy.tokens * sy.heads == 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.data), b = reinterpret_cast<uintptr_t>(y.data);
  const uintptr_t ea = a + (uintptr_t)heads_extent(x, sx) * width, eb = b + (uintptr_t)heads_extent(y, sy) * width;
  if (ea <= b || eb <= a) return false;
  const HeadsDims dx = heads_dims(x, sx), dy = heads_dims(y, sy);
  const int64_t gap = (int64_t)(b - a);
  bool same = dx.apart && dy.apart && gap % (int64_t)width == 0;
  for (int i = 0; i < 3; ++i) same = same && (dx.count[i] <= 1 || dy.count[i] <= 1 || dx.stride[i] == dy.stride[i]);
  for (int i = 0; i < 3; ++i)                           // a level's stride has to reach over what lies inside in either tensor
    if (dx.count[i] > 1 || dy.count[i] > 1) {
      const int64_t s = dx.stride[i] ? dx.stride[i] : dy.stride[i];
      same = same && s >= dx.inner[i] && s >= dy.inner[i];
    }
  return same ? nested_overlap(gap / (int64_t)width, dx, dy, 0, sx.D) : true;
}

// Alignment of 16-byte vectors; strides at least 0 (that of a dimension of one is not looked at).
inline bool heads_vectors(const dat_heads& t, const HeadsShape& s, size_t width) {
  const int64_t v = 16 / (int64_t)width;
  auto fine = [&](int64_t count, int64_t stride) { return count <= 1 || (stride >= 0 && stride % v == 0); };
  return t.data && aligned(t.data, 16) && fine(s.batch, t.batch) && fine(s.tokens, t.token) && fine(s.heads, t.head);
}

}  // namespace dat
