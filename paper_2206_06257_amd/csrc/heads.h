// Strided tensors of heads, [batch][token][head][D] with the elements of a head beside one another: host-side checks.
#pragma once
#include "common.h"

namespace dat {

struct HeadsShape { int64_t batch, tokens, heads, D; };

// Whether a tensor's elements are apart: each dimension's stride reaches over what lies inside it, from the widest stride to the narrowest.
inline bool heads_apart(const dat_heads& t, const HeadsShape& s) {
  int64_t stride[3] = {t.batch, t.token, t.head}, count[3] = {s.batch, s.tokens, s.heads};
  for (int i = 0; i < 3; ++i) if (count[i] <= 1) stride[i] = 0;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] > stride[i]) { const int64_t x = stride[i], n = count[i]; stride[i] = stride[j]; count[i] = count[j]; stride[j] = x; count[j] = n; }
  int64_t inner = s.D;
  for (int i = 2; i >= 0; --i) {
    if (count[i] <= 1) continue;
    if (stride[i] < inner) return false;
    inner += stride[i] * (count[i] - 1);
  }
  return true;
}
inline int64_t heads_extent(const dat_heads& t, const HeadsShape& s) {
  const int64_t stride[3] = {t.batch, t.token, t.head}, count[3] = {s.batch, s.tokens, s.heads};
  int64_t extent = s.D;
  for (int i = 0; i < 3; ++i) if (count[i] > 1) extent += stride[i] * (count[i] - 1);
  return extent;
}

// A dimension (batch, token or head) of two tensors that step through it alike; a dimension of one has no stride.
struct SharedDim { int64_t stride, a, b; };             // and how many the first has of it, and the second

// Whether elements of two tensors, the second `delta` elements behind the first, are the same one; dimensions from the widest stride to the
// narrowest, each reaching over what lies inside it in either tensor.
inline bool nested_overlap(int64_t delta, const SharedDim* d, int left, int64_t D) {
  if (left == 0) return delta < D && -delta < D;
  if (d->a <= 1 && d->b <= 1) return nested_overlap(delta, d + 1, left - 1, D);
  int64_t i = delta / d->stride;                        // the first's index less the second's: above -b, below a
  if (delta < 0 && i * d->stride != delta) --i;         // floor
  for (int64_t k = i; k <= i + 1; ++k)
    if (k < d->a && -k < d->b && nested_overlap(delta - k * d->stride, d + 1, left - 1, D)) return true;
  return false;
}

// Whether two tensors share an element: exact where they step through each dimension alike (parts of one tensor), by their extents elsewhere.
inline bool heads_overlap(const dat_heads& x, const HeadsShape& sx, const dat_heads& y, const HeadsShape& sy, size_t width) {
  if (sx.batch * sx.tokens * sx.heads == 0 || sy.batch * sy.tokens * sy.heads == 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.data), b = reinterpret_cast<uintptr_t>(y.data);
  const uintptr_t ea = a + (uintptr_t)heads_extent(x, sx) * width, eb = b + (uintptr_t)heads_extent(y, sy) * width;
  if (ea <= b || eb <= a) return false;
  const int64_t gap = (int64_t)(b - a), xs[3] = {x.batch, x.token, x.head}, ys[3] = {y.batch, y.token, y.head};
  const int64_t xn[3] = {sx.batch, sx.tokens, sx.heads}, yn[3] = {sy.batch, sy.tokens, sy.heads};
  SharedDim dims[3];
  bool alike = gap % (int64_t)width == 0;
  for (int i = 0; i < 3; ++i) {                         // dimension by dimension, then sorted by what both step by: a tensor's own order may differ
    dims[i] = SharedDim{xn[i] > 1 ? xs[i] : yn[i] > 1 ? ys[i] : 0, xn[i], yn[i]};
    alike = alike && (xn[i] <= 1 || yn[i] <= 1 || xs[i] == ys[i]);
  }
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j) if (dims[j].stride > dims[i].stride) { const SharedDim d = dims[i]; dims[i] = dims[j]; dims[j] = d; }
  int64_t inner_a = sx.D, inner_b = sy.D;               // elements from the first to behind the last of what lies inside
  for (int i = 2; i >= 0; --i) {
    const SharedDim& d = dims[i];
    if (d.a <= 1 && d.b <= 1) continue;
    alike = alike && d.stride >= inner_a && d.stride >= inner_b;
    inner_a += d.stride * (d.a - 1);
    inner_b += d.stride * (d.b - 1);
  }
  return alike ? nested_overlap(gap / (int64_t)width, dims, 3, sx.D) : true;
}

// A block of memory beside tensors of heads (rows' statistics, scales, positions).
struct Block { const void* data; uint64_t bytes; };
inline bool blocks_overlap(const Block& x, const Block& y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.data), b = reinterpret_cast<uintptr_t>(y.data);
  return x.data && y.data && x.bytes && y.bytes && a < b + y.bytes && b < a + x.bytes;
}
// What a tensor reaches over, from its first element to behind its last.
inline Block heads_block(const dat_heads* t, const HeadsShape& s, size_t width) {
  if (!t || s.batch * s.tokens * s.heads == 0) return Block{nullptr, 0};
  return Block{t->data, (uint64_t)heads_extent(*t, s) * width};
}

// Alignment of 16-byte vectors; strides at least 0 (that of a dimension of one is not looked at).
inline bool heads_vectors(const dat_heads& t, const HeadsShape& s, size_t width) {
  const int64_t v = 16 / (int64_t)width;
  auto fine = [&](int64_t count, int64_t stride) { return count <= 1 || (stride >= 0 && stride % v == 0); };
  return t.data && aligned(t.data, 16) && fine(s.batch, t.batch) && fine(s.tokens, t.token) && fine(s.heads, t.head);
}

}  // namespace dat
