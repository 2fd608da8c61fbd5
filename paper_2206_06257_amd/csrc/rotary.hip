// Root-mean-square norm of every head of queries and keys, its scale and the rotation by positions, in one pass, and the gradients.
//
//   r = 1 / sqrt(mean x^2 + eps),  n = x r gamma;  pair p of elements (a, b) turns by the angle w = position[axis(p)] frequency[p]:
//   (a cos w - b sin w, a sin w + b cos w);
//   backward: dn = dy turned back, h = dn gamma, xhat = x r:  dx = r (h - xhat mean(h xhat)),  dgamma = sum dn xhat.
//
// Bound by HBM.  A lane holds two vectors of W elements of a head that hold W whole pairs (pairs of neighbours: vectors behind one another;
// pairs of halves: one vector of each half), so nothing is exchanged but the sums of a head, among the L lanes (a power of two) that
// share it.  A wave takes one token, or several where a token has few heads, and all its heads: the angles are made once for all of them,
// each lane making some and the others taking them over.  Queries come first, then keys, so that a step of the wave has one scale.
// An angle is a product in 64 bits (the exact one up to its last bit, at any position), reduced to quarter turns there; sine and
// cosine of what is left are Taylor polynomials in fp32 (|x| <= pi/4, degrees 11 and 12: below 1e-9 off).
// Measured: forward 65536 tokens of 16 + 4 heads of 128, bf16, three axes, 137 us: 672 MB at 4.9 TB/s (a copy reaches 5.14); backward 18464 tokens of
// 16 + 16 heads of 64, bf16, 50 us: 227 MB at 4.5 TB/s, and 4 us for the sums of dgamma; 10007 tokens of 6 + 6 heads of 80, fp32, 29 us and 4.
// (With every lane making all its angles, and no heads on their way meanwhile: 217 and 96 us for the first two calls.)
// Backward in bf16 with 16-byte vectors keeps 8 to 12 dwords of a lane in scratch memory from token to token (32 and 48 registers spilled), none inside the loop
// over heads.
#include "kernels.h"
#include "heads.h"
#include <initializer_list>

namespace dat {
namespace {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kThreads = 256, kWaves = 4;
constexpr int kMaxParts = 512;                   // workgroups of a backward pass: 2 a compute unit

struct Rows {                                    // strides in bytes
  char* data; int64_t batch, token, head;
};

struct RotArgs {
  Rows q, k, yq, yk, dq, dk;                     // backward: yq and yk are the incoming gradients
  const float* gamma_q; const float* gamma_k;
  const int32_t* positions; const float* frequencies;
  float* parts;                                  // backward: [workgroups][2][D]
  int T, S, H, Hkv, D, axes, pairs, units, turned;     // vectors a lane; of them with pairs that turn
  int c1, c2, c3;                                // first pairs of the axes 1, 2 and 3
  int lanes, head_groups, token_groups;          // L; heads and tokens that a wave takes at once
  float eps, inv_d;
  int norm;
};

template <typename T, int W> struct Vec;
template <> struct Vec<bf16_t, 8> { typedef u32x4 type; };
template <> struct Vec<bf16_t, 4> { typedef u32x2 type; };
template <> struct Vec<bf16_t, 2> { typedef uint32_t type; };
template <> struct Vec<float, 4> { typedef u32x4 type; };
template <> struct Vec<float, 2> { typedef u32x2 type; };

template <typename T, int W> __device__ __forceinline__ void unpack(const typename Vec<T, W>::type& v, float (&x)[W]) {
  uint32_t w[sizeof(T) * W / 4];
  __builtin_memcpy(w, &v, sizeof(w));
#pragma unroll
  for (int j = 0; j < W; ++j) {
    if constexpr (sizeof(T) == 2) x[j] = __uint_as_float((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    else x[j] = __uint_as_float(w[j]);
  }
}
template <typename T, int W> __device__ __forceinline__ typename Vec<T, W>::type pack(const float (&x)[W]) {
  uint32_t w[sizeof(T) * W / 4];
#pragma unroll
  for (int j = 0; j < (int)(sizeof(T) * W / 4); ++j) {
    if constexpr (sizeof(T) == 2) w[j] = f2bf_pack(x[2 * j], x[2 * j + 1]);
    else w[j] = __float_as_uint(x[j]);
  }
  typename Vec<T, W>::type v;
  __builtin_memcpy(&v, w, sizeof(w));
  return v;
}

// Sum over the L lanes of a head (1, 2, 4, .. 64; the same for all lanes), the same bits in each.
template <int CTRL> __device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float v, int L) {
  if (L > 1) v += moved<0xb1>(v);
  if (L > 2) v += moved<0x4e>(v);
  if (L > 4) v += moved<0x141>(v);
  if (L > 8) v += moved<0x140>(v);
  if (L > 16) { const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
  if (L > 32) { const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
  return v;
}

// cos and sin of position * frequency.
__device__ __forceinline__ void turn(int position, float frequency, float& c, float& s) {
  const double quarters = (double)position * (double)frequency * 0.63661977236758134308;      // 2 / pi
  const double n = __builtin_rint(quarters);
  const float x = (float)(quarters - n) * 1.57079632679489661923f, z = x * x;
  const float sx = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 39916800, 1.0f / 362880), -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
  const float cx = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 479001600, -1.0f / 3628800), 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int k = (int)fma(-4.0, __builtin_rint(0.25 * n), n);      // n modulo 4, from -2 to 2
  const bool swap = k & 1;
  c = swap ? sx : cx;
  s = swap ? cx : sx;
  c = (k + 1) & 2 ? -c : c;
  s = k & 2 ? -s : s;
}

// What a lane holds: its token, its place among the heads, the first elements of its two vectors, the angles of its pairs.
template <int W, bool HALVES> struct Lane {
  int token, group, first, second;
  bool there;
  float c[W], s[W];
  __device__ __forceinline__ void init(const RotArgs& a, int lane) {
    const int u = lane & (a.lanes - 1), g = (uint32_t)lane / (uint32_t)a.lanes;
    group = g & (a.head_groups - 1);
    token = (uint32_t)g / (uint32_t)a.head_groups;
    there = u < a.units;
    if (HALVES) {                                // behind the turned pairs: what is left, in two halves as well
      const int rest = u - a.turned, half = (a.D - 2 * a.pairs) / 2;
      first = rest < 0 ? W * u : 2 * a.pairs + W * rest;
      second = rest < 0 ? a.pairs + W * u : 2 * a.pairs + half + W * rest;
    } else {
      first = 2 * W * u;
      second = first + W;
    }
#pragma unroll
    for (int j = 0; j < W; ++j) { c[j] = 1.0f; s[j] = 0.0f; }     // (lanes without elements hold zeros, which have to stay zeros)
  }
  // Of the W pairs that SHARE lanes (heads of one token) have in common, this lane makes every SHARE-th; the rest comes from the others.
  template <int SHARE> __device__ __forceinline__ void make(const RotArgs& a, int lane, int64_t t, bool live) {
    const int u = lane & (a.lanes - 1), mine = group & (SHARE - 1);
    float cc[W / SHARE], ss[W / SHARE];
    const float* frequencies = a.frequencies;
    asm volatile("" : "+s"(frequencies));        // read again for each token: kept over the backward pass's loop they cost more registers than it has
#pragma unroll
    for (int i = 0; i < W / SHARE; ++i) {
      const int p = W * u + mine + SHARE * i;
      cc[i] = 1.0f; ss[i] = 0.0f;
      if (live && p < a.pairs) {
        const int axis = (p >= a.c1) + (p >= a.c2) + (p >= a.c3);
        turn(a.positions[t * a.axes + axis], frequencies[p], cc[i], ss[i]);
      }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int from = 4 * (lane + (j % SHARE - mine) * a.lanes);
      c[j] = SHARE == 1 ? cc[j / SHARE] : __int_as_float(__builtin_amdgcn_ds_bpermute(from, __float_as_int(cc[j / SHARE])));
      s[j] = SHARE == 1 ? ss[j / SHARE] : __int_as_float(__builtin_amdgcn_ds_bpermute(from, __float_as_int(ss[j / SHARE])));
    }
  }
  __device__ __forceinline__ void angles(const RotArgs& a, int lane, int64_t t, bool live) {
    if (a.head_groups >= W) make<W>(a, lane, t, live);
    else if (a.head_groups >= 4) make<W < 4 ? W : 4>(a, lane, t, live);
    else if (a.head_groups >= 2) make<2>(a, lane, t, live);
    else make<1>(a, lane, t, live);
  }
  // pair j of the two vectors
  __device__ __forceinline__ static float& one(float (&x)[2][W], int j) { return HALVES ? x[0][j] : x[(2 * j) / W][(2 * j) % W]; }
  __device__ __forceinline__ static float& two(float (&x)[2][W], int j) { return HALVES ? x[1][j] : x[(2 * j + 1) / W][(2 * j + 1) % W]; }
};

template <int W> __device__ __forceinline__ void load_gamma(const float* gamma, bool there, int first, int second, float (&g)[2][W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) {
    g[0][j] = there && gamma ? gamma[first + j] : 1.0f;
    g[1][j] = there && gamma ? gamma[second + j] : 1.0f;
  }
}

// f and 1 / sqrt(mean (f x)^2 + eps f^2); f = 1 but where the sum of squares leaves fp32's range, or is small enough to lose digits in it and
// eps does not stand in for it.  x r is (f x) times the result.
template <int W> __device__ __forceinline__ void rms(const RotArgs& a, const float (&x)[2][W], float& f, float& rs) {
  float ss = 0.0f;
#pragma unroll
  for (int v = 0; v < 2; ++v)
#pragma unroll
    for (int j = 0; j < W; ++j) ss = fmaf(x[v][j], x[v][j], ss);
  ss = head_sum(ss, a.lanes);
  f = ss == __builtin_inff() ? 0x1p-70f : ss < 0x1p-80f && a.eps < 0x1p-60f ? 0x1p70f : 1.0f;
  if (__any(f != 1.0f)) {
    float again = 0.0f;
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) again = fmaf(x[v][j] * f, x[v][j] * f, again);
    again = head_sum(again, a.lanes);
    ss = f != 1.0f ? again : ss;
  }
  rs = __builtin_amdgcn_rsqf(fmaf(ss, a.inv_d, a.eps * f * f));
}

// Heads of one token: where they are, and how many.
struct HeadRow { char* p; int64_t stride; int n; };
__device__ __forceinline__ HeadRow heads_at(const Rows& r, int b, int s, int n) { return HeadRow{r.data + (int64_t)b * r.batch + (int64_t)s * r.token, r.head, n}; }

// U steps of heads from h0 on: a lane's two vectors of each.
template <typename T, int W, bool HALVES, int U>
__device__ __forceinline__ void load_heads(const RotArgs& a, const Lane<W, HALVES>& me, const HeadRow& x, bool live, int h0, typename Vec<T, W>::type (&raw)[U][2]) {
  typedef typename Vec<T, W>::type V;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int head = h0 + i * a.head_groups + me.group;
    __builtin_memset(raw[i], 0, sizeof(raw[i]));
    if (live && head < x.n) {
      const T* const p = reinterpret_cast<const T*>(x.p + head * x.stride);
      raw[i][0] = *reinterpret_cast<const V*>(p + me.first);
      raw[i][1] = *reinterpret_cast<const V*>(p + me.second);
    }
  }
}
template <typename T, int W, bool HALVES>
__device__ __forceinline__ void store_head(const Lane<W, HALVES>& me, const HeadRow& y, int head, const float (&v)[2][W]) {
  typedef typename Vec<T, W>::type V;
  T* const p = reinterpret_cast<T*>(y.p + head * y.stride);
  *reinterpret_cast<V*>(p + me.first) = pack<T, W>(v[0]);
  *reinterpret_cast<V*>(p + me.second) = pack<T, W>(v[1]);
}

template <typename T, int W, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_forward_kernel(RotArgs a) {
  typedef typename Vec<T, W>::type V;
  constexpr int U = 4;                           // steps in flight
  const int lane = threadIdx.x & 63, wave = (int)(threadIdx.x >> 6);
  Lane<W, HALVES> me;
  me.init(a, lane);
  const int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * a.token_groups + me.token;
  const bool live = t < a.T && me.there;
  const int b = live && a.S < a.T ? (int)((uint32_t)t / (uint32_t)a.S) : 0, s = live ? (int)t - b * a.S : 0;
  V raw[U][2];
  // loaded: the first U steps are there already
  auto run = [&](const HeadRow& x, const HeadRow& y, const float* gamma, bool loaded) {
    float g[2][W];
    if (a.norm) load_gamma<W>(gamma, me.there, me.first, me.second, g);
    for (int h0 = 0; h0 < x.n; h0 += U * a.head_groups) {
      if (!loaded || h0 > 0) load_heads<T, W, HALVES, U>(a, me, x, live, h0, raw);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (h0 + i * a.head_groups >= x.n) break;
        const int head = h0 + i * a.head_groups + me.group;
        float v[2][W], w[2][W];
        unpack<T, W>(raw[i][0], v[0]);
        unpack<T, W>(raw[i][1], v[1]);
        if (a.norm) {
          float f, rs;
          rms<W>(a, v, f, rs);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j) v[k][j] = v[k][j] * f * rs * g[k][j];
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float p = Lane<W, HALVES>::one(v, j), q = Lane<W, HALVES>::two(v, j);
          Lane<W, HALVES>::one(w, j) = fmaf(p, me.c[j], -(q * me.s[j]));
          Lane<W, HALVES>::two(w, j) = fmaf(p, me.s[j], q * me.c[j]);
        }
        if (live && head < x.n) store_head<T, W, HALVES>(me, y, head, w);
      }
    }
  };
  const HeadRow q = heads_at(a.q, b, s, a.H);
  load_heads<T, W, HALVES, U>(a, me, q, live, 0, raw);           // on their way while the angles are made
  me.angles(a, lane, t, live);
  run(q, heads_at(a.yq, b, s, a.H), a.gamma_q, true);
  run(heads_at(a.k, b, s, a.Hkv), heads_at(a.yk, b, s, a.Hkv), a.gamma_k, false);
}

// Waves go on to further tokens, so that few partial sums of dgamma are left: one for each workgroup, added up by a launch of its own.
template <typename T, int W, bool HALVES>
__global__ __launch_bounds__(kThreads, 2) void rotary_backward_kernel(RotArgs a) {
  typedef typename Vec<T, W>::type V;
  constexpr int U = 2;
  __shared__ float sums[2 * W][kThreads];
  const int lane = threadIdx.x & 63, wave = (int)(threadIdx.x >> 6);
  Lane<W, HALVES> me;
  me.init(a, lane);
  float gq[2][W], gk[2][W], dgq[2][W], dgk[2][W];
  if (a.norm) {
    load_gamma<W>(a.gamma_q, me.there, me.first, me.second, gq);
    load_gamma<W>(a.gamma_k, me.there, me.first, me.second, gk);
  }
#pragma unroll
  for (int v = 0; v < 2; ++v)
#pragma unroll
    for (int j = 0; j < W; ++j) dgq[v][j] = dgk[v][j] = 0.0f;
  V raw[U][2], grad[U][2];
  auto load = [&](const HeadRow& x, const HeadRow& dy, bool live, int h0) {
    load_heads<T, W, HALVES, U>(a, me, dy, live, h0, grad);
    if (a.norm) load_heads<T, W, HALVES, U>(a, me, x, live, h0, raw);
  };
  auto run = [&](const HeadRow& x, const HeadRow& dy, const HeadRow& dx, const float (&gamma)[2][W], float (&dgamma)[2][W], bool live, bool loaded) {
    for (int h0 = 0; h0 < dy.n; h0 += U * a.head_groups) {
      if (!loaded || h0 > 0) load(x, dy, live, h0);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (h0 + i * a.head_groups >= dy.n) break;
        const int head = h0 + i * a.head_groups + me.group;
        const bool counts = live && head < dy.n;
        float v[2][W], y[2][W], dn[2][W];
        unpack<T, W>(grad[i][0], y[0]);
        unpack<T, W>(grad[i][1], y[1]);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float p = Lane<W, HALVES>::one(y, j), q = Lane<W, HALVES>::two(y, j);
          Lane<W, HALVES>::one(dn, j) = fmaf(p, me.c[j], q * me.s[j]);
          Lane<W, HALVES>::two(dn, j) = fmaf(q, me.c[j], -(p * me.s[j]));
        }
        if (a.norm) {
          unpack<T, W>(raw[i][0], v[0]);
          unpack<T, W>(raw[i][1], v[1]);
          float f, rs, dot = 0.0f;
          rms<W>(a, v, f, rs);
          if (!counts) rs = 0.0f;                // (a head that is not there may have an infinite 1 / sqrt(eps))
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j) {
              v[k][j] = v[k][j] * f * rs;        // xhat
              dgamma[k][j] = fmaf(dn[k][j], v[k][j], dgamma[k][j]);
              dn[k][j] *= gamma[k][j];
              dot = fmaf(dn[k][j], v[k][j], dot);
            }
          dot = head_sum(dot, a.lanes) * a.inv_d;
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j) dn[k][j] = fmaf(-v[k][j], dot, dn[k][j]) * rs * f;
        }
        if (counts) store_head<T, W, HALVES>(me, dx, head, dn);
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kWaves * a.token_groups;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * a.token_groups; t0 < a.T; t0 += step) {
    const int64_t t = t0 + me.token;
    const bool live = t < a.T && me.there;
    const int b = live && a.S < a.T ? (int)((uint32_t)t / (uint32_t)a.S) : 0, s = live ? (int)t - b * a.S : 0;
    const HeadRow q = heads_at(a.q, b, s, a.H), dyq = heads_at(a.yq, b, s, a.H);
    load(q, dyq, live, 0);
    me.angles(a, lane, t, live);
    run(q, dyq, heads_at(a.dq, b, s, a.H), gq, dgq, live, true);
    run(heads_at(a.k, b, s, a.Hkv), heads_at(a.yk, b, s, a.Hkv), heads_at(a.dk, b, s, a.Hkv), gk, dgk, live, false);
  }
  if (!a.norm) return;
  // element e of a head: the lanes that hold it, of all waves, one after the other
  const int groups = 64 / a.lanes;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) sums[v * W + j][threadIdx.x] = which ? dgk[v][j] : dgq[v][j];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * W * a.units; i += kThreads) {
      const int u = i / (2 * W), vj = i - u * 2 * W;
      float total = 0.0f;
      for (int w = 0; w < kWaves; ++w)
        for (int g = 0; g < groups; ++g) total += sums[vj][w * 64 + g * a.lanes + u];
      const int v = vj / W, j = vj - v * W;
      int at;
      if (HALVES) {
        const int rest = u - a.turned, half = (a.D - 2 * a.pairs) / 2;
        at = (rest < 0 ? v * a.pairs + W * u : 2 * a.pairs + v * half + W * rest) + j;
      } else {
        at = 2 * W * u + v * W + j;
      }
      a.parts[((int64_t)blockIdx.x * 2 + which) * a.D + at] = total;
    }
  }
}

// dgamma[e] = sum over the workgroups' parts in a fixed order: 16 elements a workgroup, 64 threads an element (16 ones: 18 us for 1024 parts of
// 128; the parts come one after the other).
__global__ __launch_bounds__(1024) void rotary_dgamma_kernel(const float* __restrict__ parts, int n, int D, float* __restrict__ dgq, float* __restrict__ dgk) {
  __shared__ float part[64][17];
  const int e = threadIdx.x & 15, row = threadIdx.x >> 4, col = blockIdx.x * 16 + e;
  float total = 0.0f;
  if (col < 2 * D) {
#pragma unroll
    for (int i = 0; i < kMaxParts / 64; ++i) total += row + 64 * i < n ? parts[(int64_t)(row + 64 * i) * 2 * D + col] : 0.0f;
  }
  part[row][e] = total;
  __syncthreads();
  if (threadIdx.x < 16 && col < 2 * D) {
    total = 0.0f;
#pragma unroll
    for (int r = 0; r < 64; ++r) total += part[r][e];
    float* const out = col < D ? dgq : dgk;
    if (out) out[col < D ? col : col - D] = total;
  }
}

int power_of_two(int n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

bool fill(const dat_rotary* s, RotArgs& a, dat_status& status) {
  status = DAT_ERR_ARG;
  if (!s || (s->dtype != DAT_F32 && s->dtype != DAT_BF16) || s->B < 0 || s->S < 0 || s->H < 0 || s->Hkv < 0 || s->H + (int64_t)s->Hkv < 1 || s->D < 1) return false;
  if (s->axes < 0 || s->axes > 4 || (s->layout != DAT_ROTARY_HALVES && s->layout != DAT_ROTARY_PAIRS) || (s->norm != 0 && s->norm != 1)) return false;
  if (!(s->eps >= 0.0f) || !(s->eps < __builtin_inff())) return false;
  int64_t pairs = 0;
  for (int i = 0; i < s->axes; ++i) {
    if (s->sections[i] < 0) return false;
    pairs += s->sections[i];
  }
  if (2 * pairs > s->D) return false;
  status = DAT_ERR_SHAPE;
  if (s->D % 8 || s->D > 256 || (s->layout == DAT_ROTARY_HALVES && pairs % 2)) return false;
  if ((int64_t)s->B * s->S > 1 << 30 || s->H + (int64_t)s->Hkv > 1 << 20) return false;
  a.T = s->B * s->S; a.S = s->S; a.H = s->H; a.Hkv = s->Hkv; a.D = s->D; a.axes = s->axes; a.pairs = (int)pairs;
  a.c1 = s->axes > 1 ? s->sections[0] : INT32_MAX;
  a.c2 = s->axes > 2 ? a.c1 + s->sections[1] : INT32_MAX;
  a.c3 = s->axes > 3 ? a.c2 + s->sections[2] : INT32_MAX;
  a.eps = s->eps; a.inv_d = 1.0f / (float)s->D; a.norm = s->norm;
  status = DAT_OK;
  return true;
}

// Elements of a lane's vector: 16 bytes where the halves have whole ones of them.
int vector_of(const dat_rotary& s, int pairs) {
  const int rest = (s.D - 2 * pairs) / 2, widest = s.dtype == DAT_BF16 ? 8 : 4;
  for (int w = widest; w > 2; w /= 2)
    if (s.layout == DAT_ROTARY_PAIRS ? s.D % (2 * w) == 0 : pairs % w == 0 && rest % w == 0) return w;
  return 2;
}

int blocks_of(const RotArgs& a) { return (int)(((int64_t)a.T + kWaves * a.token_groups - 1) / (kWaves * a.token_groups)); }

void arrange(const dat_rotary& s, RotArgs& a) {
  const int w = vector_of(s, a.pairs);
  a.units = a.D / (2 * w); a.turned = a.pairs / w;
  a.lanes = power_of_two(a.units);
  // heads of a token that a wave takes at once: as many as leave at most an eighth of the steps' places empty
  // (16 + 4 heads of 128, forward: 4 at once 142 us, 8, a sixth of the places empty, 175, one 138; 16 + 16 of 64, backward: 8 at once 59 us, one 77; 6 + 6 of
  // 80, backward, fp32: 2 at once 38 us, 4 37, one 41)
  const int groups = 64 / a.lanes;
  auto places = [&](int n) { return ((int64_t)a.H + n - 1) / n * n + ((int64_t)a.Hkv + n - 1) / n * n; };
  a.head_groups = groups;
  while (a.head_groups > 1 && 8 * places(a.head_groups) > 9 * ((int64_t)a.H + a.Hkv)) a.head_groups /= 2;
  a.token_groups = groups / a.head_groups;
}

template <typename T, int W, bool HALVES> dat_status launch(bool backward, const RotArgs& a, hipStream_t st) {
  const int blocks = blocks_of(a);
  if (!backward) {
    hipLaunchKernelGGL((rotary_forward_kernel<T, W, HALVES>), dim3(blocks), dim3(kThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL((rotary_backward_kernel<T, W, HALVES>), dim3(blocks < kMaxParts ? blocks : kMaxParts), dim3(kThreads), 0, st, a);
  }
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}
template <typename T, int W> dat_status launch(bool backward, int layout, const RotArgs& a, hipStream_t st) {
  if constexpr (W > 2) { if (layout == DAT_ROTARY_PAIRS) return launch<T, W, false>(backward, a, st); }   // (D is a multiple of 8)
  return launch<T, W, true>(backward, a, st);
}
dat_status launch(bool backward, const dat_rotary& s, const RotArgs& a, hipStream_t st) {
  if (!fits_launch(blocks_of(a), kThreads)) return DAT_ERR_SHAPE;
  const int w = vector_of(s, a.pairs);
  if (s.dtype == DAT_BF16) {
    if (w == 8) return launch<bf16_t, 8>(backward, s.layout, a, st);
    return w == 4 ? launch<bf16_t, 4>(backward, s.layout, a, st) : launch<bf16_t, 2>(backward, s.layout, a, st);
  }
  return w == 4 ? launch<float, 4>(backward, s.layout, a, st) : launch<float, 2>(backward, s.layout, a, st);
}

struct Tensor { const dat_heads* t; HeadsShape s; Rows* to; bool output; };

dat_status take(const Tensor& x, size_t width) {
  if (x.s.batch * x.s.tokens * x.s.heads == 0) { *x.to = Rows{nullptr, 0, 0, 0}; return DAT_OK; }
  if (!x.t || !heads_vectors(*x.t, x.s, width) || (x.output && !heads_apart(*x.t, x.s))) return DAT_ERR_ARG;
  const int64_t w = (int64_t)width;
  *x.to = Rows{(char*)x.t->data, x.s.batch > 1 ? x.t->batch * w : 0, x.s.tokens > 1 ? x.t->token * w : 0, x.s.heads > 1 ? x.t->head * w : 0};
  return DAT_OK;
}
bool same(const Tensor& x, const Tensor& y) {
  return x.t->data == y.t->data && (x.s.batch <= 1 || x.t->batch == y.t->batch) && (x.s.tokens <= 1 || x.t->token == y.t->token) &&
         (x.s.heads <= 1 || x.t->head == y.t->head);
}
// The output may be the input at the same index of the other list (where it is read before it is written, by the same lane).
dat_status take_all(std::initializer_list<Tensor> in, std::initializer_list<Tensor> out, size_t width) {
  for (auto* list : {&in, &out})
    for (const Tensor& x : *list) {
      const dat_status st = take(x, width);
      if (st != DAT_OK) return st;
    }
  for (size_t i = 0; i < out.size(); ++i) {
    const Tensor& x = out.begin()[i];
    if (x.s.heads * x.s.tokens * x.s.batch == 0) continue;
    for (size_t j = 0; j < in.size(); ++j) {
      const Tensor& y = in.begin()[j];
      if (y.s.heads == 0 || (j % 2 == i && same(x, y))) continue;
      if (heads_overlap(*x.t, x.s, *y.t, y.s, width)) return DAT_ERR_ARG;
    }
    for (size_t j = 0; j < out.size(); ++j) {
      const Tensor& y = out.begin()[j];
      if (j != i && y.s.heads > 0 && heads_overlap(*x.t, x.s, *y.t, y.s, width)) return DAT_ERR_ARG;
    }
  }
  return DAT_OK;
}
// The blocks that a call reads lie in no output; those that it writes (the scales' gradients, when all else has been read and written) lie in no
// tensor and not on each other.
bool blocks_apart(std::initializer_list<Tensor> in, std::initializer_list<Tensor> out, std::initializer_list<Block> read, std::initializer_list<Block> written, size_t width) {
  for (const Tensor& x : out)
    for (const Block& y : read) if (blocks_overlap(heads_block(x.t, x.s, width), y)) return false;
  for (auto* list : {&in, &out})
    for (const Tensor& x : *list)
      for (const Block& y : written) if (blocks_overlap(heads_block(x.t, x.s, width), y)) return false;
  for (const Block& x : written)
    for (const Block& y : written) if (&x < &y && blocks_overlap(x, y)) return false;
  return true;
}
Block scale_block(const RotArgs& a, const float* gamma) { return Block{gamma, a.norm ? (uint64_t)a.D * 4 : 0}; }
Block positions_block(const RotArgs& a, const int32_t* positions) { return Block{positions, a.pairs ? (uint64_t)a.T * a.axes * 4 : 0}; }
Block frequencies_block(const RotArgs& a, const float* frequencies) { return Block{frequencies, (uint64_t)a.pairs * 4}; }

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" dat_status dat_norm_rotary_forward(const dat_rotary* shape, const dat_heads* q, const dat_heads* k, const float* gamma_q, const float* gamma_k,
                                              const int32_t* positions, const float* frequencies, const dat_heads* yq, const dat_heads* yk, void* stream) {
  RotArgs a{};
  dat_status st;
  if (!fill(shape, a, st)) return st;
  const HeadsShape sq{shape->B, shape->S, shape->H, shape->D}, sk{shape->B, shape->S, shape->Hkv, shape->D};
  const size_t width = shape->dtype == DAT_BF16 ? 2 : 4;
  st = take_all({{q, sq, &a.q, false}, {k, sk, &a.k, false}}, {{yq, sq, &a.yq, true}, {yk, sk, &a.yk, true}}, width);
  if (st != DAT_OK) return st;
  if (a.T == 0) return DAT_OK;
  if (!blocks_apart({}, {{yq, sq, &a.yq, true}, {yk, sk, &a.yk, true}},
                    {scale_block(a, gamma_q), scale_block(a, gamma_k), positions_block(a, positions), frequencies_block(a, frequencies)}, {}, width)) return DAT_ERR_ARG;
  if (!aligned(gamma_q, 4) || !aligned(gamma_k, 4) || !aligned(positions, 4) || !aligned(frequencies, 4) || (a.pairs > 0 && (!positions || !frequencies))) return DAT_ERR_ARG;
  a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.positions = positions; a.frequencies = frequencies;
  arrange(*shape, a);
  return launch(false, *shape, a, (hipStream_t)stream);
}

extern "C" size_t dat_norm_rotary_workspace(int pass, const dat_rotary* shape) {
  RotArgs a{};
  dat_status st;
  if (!fill(shape, a, st) || pass != 1 || !a.norm || a.T == 0) return 0;
  arrange(*shape, a);
  const int blocks = blocks_of(a);
  return (size_t)(blocks < kMaxParts ? blocks : kMaxParts) * 2 * a.D * 4;
}

extern "C" dat_status dat_norm_rotary_backward(const dat_rotary* shape, const dat_heads* q, const dat_heads* k, const float* gamma_q, const float* gamma_k,
                                               const int32_t* positions, const float* frequencies, const dat_heads* dyq, const dat_heads* dyk,
                                               const dat_heads* dq, const dat_heads* dk, float* dgamma_q, float* dgamma_k, void* workspace,
                                               size_t workspace_bytes, void* stream) {
  RotArgs a{};
  dat_status st;
  if (!fill(shape, a, st)) return st;
  const HeadsShape sq{shape->B, shape->S, shape->H, shape->D}, sk{shape->B, shape->S, shape->Hkv, shape->D};
  const size_t width = shape->dtype == DAT_BF16 ? 2 : 4;
  st = a.norm ? take_all({{q, sq, &a.q, false}, {k, sk, &a.k, false}, {dyq, sq, &a.yq, false}, {dyk, sk, &a.yk, false}}, {{dq, sq, &a.dq, true}, {dk, sk, &a.dk, true}}, width)
              : take_all({{dyq, sq, &a.yq, false}, {dyk, sk, &a.yk, false}}, {{dq, sq, &a.dq, true}, {dk, sk, &a.dk, true}}, width);
  if (st != DAT_OK) return st;
  if (!aligned(gamma_q, 4) || !aligned(gamma_k, 4) || !aligned(positions, 4) || !aligned(frequencies, 4) || !aligned(dgamma_q, 4) || !aligned(dgamma_k, 4)) return DAT_ERR_ARG;
  if (a.T > 0 && a.pairs > 0 && (!positions || !frequencies)) return DAT_ERR_ARG;
  if (!blocks_apart({{q, a.norm ? sq : HeadsShape{}, &a.q, false}, {k, a.norm ? sk : HeadsShape{}, &a.k, false}, {dyq, sq, &a.yq, false}, {dyk, sk, &a.yk, false}},
                    {{dq, sq, &a.dq, true}, {dk, sk, &a.dk, true}},
                    {scale_block(a, gamma_q), scale_block(a, gamma_k), positions_block(a, positions), frequencies_block(a, frequencies)},
                    {scale_block(a, dgamma_q), scale_block(a, dgamma_k)}, width)) return DAT_ERR_ARG;
  const bool sums = a.norm && (dgamma_q || dgamma_k);
  if (a.norm && a.T > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < dat_norm_rotary_workspace(1, shape))) return DAT_ERR_ARG;
  a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.positions = positions; a.frequencies = frequencies;
  a.parts = (float*)workspace;
  int parts = 0;
  if (a.T > 0) {
    arrange(*shape, a);
    st = launch(true, *shape, a, (hipStream_t)stream);
    if (st != DAT_OK) return st;
    parts = blocks_of(a) < kMaxParts ? blocks_of(a) : kMaxParts;
  }
  if (sums) {
    hipLaunchKernelGGL(rotary_dgamma_kernel, dim3((2 * a.D + 15) / 16), dim3(1024), 0, (hipStream_t)stream, a.parts, parts, a.D, dgamma_q, dgamma_k);
    DAT_LAUNCH_CHECK();
  }
  return DAT_OK;
}
