// Group normalisation with an activation, channels last, forward and backward.
//
// An image is P pixels of C channels; a thread owns one 16-byte vector of channels (VE of them) at several pixels, so its scale,
// shift and statistics are registers and a wavefront reads whole pixel rows.  Every sum runs in a fixed order (thread, LDS,
// partial sums in memory): the same bits on every call.  Variances are sums of squared deviations from a mean, taken from values
// that are still in registers; where bf16 takes a difference of sums instead, it holds little rounding error (below).
//
// Two ways, both bound by HBM:
//   resident  one workgroup holds a slice of whole groups of one image in registers: every tensor is moved once.
//   split     an image's slice is too large for that: partial sums over ranges of pixels, a small kernel that joins them, and a
//             second pass over the tensors, from the last image to the first: the last-level cache still holds what the first
//             pass read last.
// Forward, resident: 256 x 56 x 56 x 256 bf16 200 us = 4.1 TB/s (one workgroup a compute unit: nothing moves while it joins its
// sums), 512 x 32 x 32 x 64 28 us = 4.8 TB/s; split (256 x 112 x 112 x 64) 260 us, three passes at 4.7 TB/s.
// Backward, resident: 256 x 28 x 28 x 512 bf16 144 us = 4.3 TB/s; split: 85 x 112 x 112 x 64 with SiLU 158 us, five passes at
// 4.3 TB/s (sums 70 us = 3.9 TB/s, the vector units issuing for half of it; apply 79 us = 5.2 TB/s).
#include <type_traits>
#include "kernels.h"
#include "lanes.h"

namespace dat {
namespace {

struct GnArgs {
  const void* x; const void* dy; const float* gamma; const float* beta; const float* mean_in; const float* rstd_in;
  void* out; float* mean; float* rstd; float* part;
  int B, P, C, G, Cg;
  int nv;            // vectors of a pixel's channels
  int sv, slices;    // vectors of a slice, slices of a pixel
  int chunk, chunks; // split: pixels of a range, ranges of an image
  float eps;
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename T, int VE> struct Vec;          // VE channels as they lie in memory
template <> struct Vec<float, 4> { typedef u32x4 type; };
template <> struct Vec<bf16_t, 8> { typedef u32x4 type; };
template <> struct Vec<float, 1> { typedef float type; };
template <> struct Vec<bf16_t, 1> { typedef bf16_t type; };

template <typename T, int VE> __device__ __forceinline__ void unpack(const typename Vec<T, VE>::type& v, float (&f)[VE]) {
  if constexpr (VE == 1 && sizeof(T) == 4) f[0] = v;
  else if constexpr (VE == 1) f[0] = bf2f(v);
  else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = __uint_as_float(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < VE; j += 2) { f[j] = __uint_as_float(v[j / 2] << 16); f[j + 1] = __uint_as_float(v[j / 2] & 0xffff0000u); }
  }
}
template <typename T, int VE> __device__ __forceinline__ typename Vec<T, VE>::type pack(const float (&f)[VE]) {
  typename Vec<T, VE>::type v;
  if constexpr (VE == 1 && sizeof(T) == 4) v = f[0];
  else if constexpr (VE == 1) v = f2bf(f[0]);
  else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = __float_as_uint(f[j]);
  } else {
#pragma unroll
    for (int j = 0; j < VE; j += 2) v[j / 2] = f2bf_pack(f[j], f[j + 1]);
  }
  return v;
}
// Channels h .. h+3 of a 16-byte vector.
template <typename T> __device__ __forceinline__ void unpack4(const u32x4& v, int h, float (&f)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) f[j] = __uint_as_float(v[j]);
    else f[j] = __uint_as_float(j % 2 ? v[(h + j) / 2] & 0xffff0000u : v[(h + j) / 2] << 16);
  }
}
template <typename T> __device__ __forceinline__ void pack4(const float (&f)[4], int h, u32x4& v) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) v[j] = __float_as_uint(f[j]);
    else if (j % 2) v[(h + j) / 2] = f2bf_pack(f[j - 1], f[j]);
  }
}
// Held vectors are unpacked anew in every pass: without this the compiler unpacks them where they are loaded, or keeps the
// unpacked values of one pass for the next, twice the registers, and spills.  (With 1024 threads, 128 registers each, two forms
// spill all the same: bf16 forward with four groups to a vector 29 registers, backward with eight and an activation 6.)
__device__ __forceinline__ void forget(u32x4& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void forget(float& v) { asm volatile("" : "+v"(v)); }

// acc + a.lo b.lo + a.hi b.hi of two pairs of bf16
__device__ __forceinline__ float dot_pairs(uint32_t a, uint32_t b, float acc) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), acc, false);
}

// Buffer descriptors: a lane beyond the range reads zeros and writes nothing, so no load or store stands behind a branch, where
// it would be waited for together with everything else in flight.  All of the offset is in the vector register: with a scalar
// register for the part that all lanes share, the compiler takes the registers of a store's data as free at once, and on gfx950
// what it computed into them next came out in memory (single lanes, now and then).  The wait states after a store keep its data
// where it is until it has been read; the empty statements of forget() would be counted as some.
typedef __amdgpu_buffer_rsrc_t BufRsrc;
constexpr uint32_t kOob = 0xfffffff0u;
__device__ __forceinline__ void buffer_load(BufRsrc r, uint32_t off, u32x4& v) { v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0); }
__device__ __forceinline__ void buffer_store(BufRsrc r, uint32_t off, const u32x4& v) { __builtin_amdgcn_raw_buffer_store_b128(v, r, (int)off, 0, 0); }
__device__ __forceinline__ void after_store() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 3");
  __builtin_amdgcn_sched_barrier(0);
}

// z = xhat gamma + beta of the ReLU's derivative: one rounding per operation, as dat.h says.
__device__ __forceinline__ float gn_z(float xm, float rstd, float gamma, float beta) {
  return __fadd_rn(__fmul_rn(__fmul_rn(xm, rstd), gamma), beta);
}
// 1 / (1 + e^-z) from the hardware's exponential and reciprocal (1 unit of 2^-23 each).  fp32 outputs: the rounding error of the
// exponent z log2(e) goes back in, or it would grow with |z|: as a factor, not as a sum, which would be infinity less infinity below
// z = -88.7, where e^-z is infinite.  The sigmoid is 0 there (it has to be, beside a z of any size).
template <typename T> __device__ __forceinline__ float sigmoid(float z) {
  constexpr float kLog2e = 1.44269504088896340736f, kLog2eLow = 1.92596299112661746887e-8f, kLn2 = 0.69314718055994530942f;
  if (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z));
  const float y = -__builtin_amdgcn_fmed3f(z, -126.0f, 126.0f), t = y * kLog2e;
  const float low = fmaf(y, kLog2eLow, fmaf(y, kLog2e, -t)), e = __builtin_amdgcn_exp2f(t);
  return __builtin_amdgcn_rcpf(fmaf(e, fmaf(kLn2, low, 1.0f), 1.0f));
}
template <typename T, int ACT> __device__ __forceinline__ float act_of(float z) {
  if (ACT == DAT_ACT_RELU) return __builtin_elementwise_maximum(z, 0.0f);      // NaN stays
  if (ACT == DAT_ACT_SILU) return z * sigmoid<T>(z);
  return z;
}
template <typename T> __device__ __forceinline__ float silu_dz(float z, float dy) {
  const float s = sigmoid<T>(z);
  return dy * fmaf(z * s, 1.0f - s, s);
}
// dz of one channel.  xm = x - mean, scale = rstd gamma.
template <typename T, int ACT>
__device__ __forceinline__ float gn_dz(float xm, float dy, float rstd, float gamma, float scale, float beta) {
  if (ACT == DAT_ACT_RELU) return gn_z(xm, rstd, gamma, beta) > 0.0f ? dy : 0.0f;
  if (ACT == DAT_ACT_SILU) return silu_dz<T>(fmaf(xm, scale, beta), dy);
  return dy;
}
__device__ __forceinline__ float rstd_of(float var, float eps) { return __fdiv_rn(1.0f, sqrtf(var + eps)); }

// The scale and shift of a thread's channels.
template <int VE> struct Affine {
  float gamma[VE], beta[VE];
  __device__ __forceinline__ Affine(const GnArgs& a, int c) {
#pragma unroll
    for (int j = 0; j < VE; ++j) { gamma[j] = a.gamma ? a.gamma[c + j] : 1.0f; beta[j] = a.gamma ? a.beta[c + j] : 0.0f; }
  }
};

// Groups of a thread's vector of VE channels, GV of them: 1 (the vector lies in one), VE/Cg where Cg divides VE, else VE (one
// for each channel).  of(j): which of the GV entries channel j uses; find(c, Cg, g): the group of each entry.
template <int VE, int GV> struct Groups {
  static constexpr int of(int j) { return j * GV / VE; }
  static __device__ __forceinline__ void find(int c, int Cg, int (&g)[GV]) {
    if (GV < VE || GV == 1) {
      const int g0 = GV == 1 ? c / Cg : c / (VE / GV);
#pragma unroll
      for (int k = 0; k < GV; ++k) g[k] = g0 + k;
      return;
    }
    int g0 = c / Cg, r = c - g0 * Cg;
#pragma unroll
    for (int k = 0; k < GV; ++k) { g[k] = g0; if (++r == Cg) { r = 0; ++g0; } }
  }
  // columns of one group where a vector has GV columns
  static __device__ __forceinline__ int columns(int Cg) { return GV == 1 ? Cg / VE : GV < VE ? 1 : Cg; }
};

// ---- resident ----------------------------------------------------------------------------------------------------------
// Tile: slice of an image.  Neighbouring slices share cache lines: they go to workgroups of one XCD (workgroups are dealt to the
// eight XCDs in turn).
constexpr int kXcds = 8;
__device__ __forceinline__ int tiles_per_xcd(int tiles) { return (tiles + kXcds - 1) / kXcds; }

// Thread tid = ty*sv + tx holds vector tx of the slice at pixels ty, ty + rows, ...: at most VPT of them.
template <typename T, int VE, int NT> struct Tile {
  typedef typename Vec<T, VE>::type V;
  bool valid;
  int b, sv, rows, tx, ty, c_slice, c;     // image, width, threads along the pixels, first channels of the slice and the thread
  int full;                                // rounds in which every thread has a pixel
  int64_t base;                            // bytes: first pixel of the slice
  uint32_t size, step;                     // bytes: from there to the image's end (0: no tile); distance of a thread's pixels
  uint32_t off, off_last;                  // bytes: the thread's first pixel, for the full rounds and for the one after them
  __device__ __forceinline__ Tile(const GnArgs& a, int index, int tiles) {
    const int per = tiles_per_xcd(tiles), i = index / kXcds, tile = (index - i * kXcds) * per + i;
    valid = i < per && tile < tiles;
    b = valid ? tile / a.slices : 0;
    const int slice = valid ? tile - b * a.slices : 0;
    sv = min(a.sv, a.nv - slice * a.sv);
    rows = NT / sv;
    ty = threadIdx.x / sv; tx = threadIdx.x - ty * sv;
    full = a.P / rows;
    const int v = slice * a.sv + tx, left = a.P - full * rows;
    c_slice = slice * a.sv * VE;
    c = v * VE;
    constexpr uint32_t kBytes = sizeof(V);
    base = ((int64_t)b * a.P * a.nv + slice * a.sv) * kBytes;
    size = valid ? ((uint32_t)a.P * (uint32_t)a.nv - (uint32_t)(slice * a.sv)) * kBytes : 0u;
    step = (uint32_t)rows * (uint32_t)a.nv * kBytes;
    const uint32_t own = ((uint32_t)ty * (uint32_t)a.nv + (uint32_t)tx) * kBytes;
    off = ty < rows ? own : kOob;
    off_last = ty < left ? own : kOob;
  }
  __device__ __forceinline__ BufRsrc buffer(const void* p) const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(p)) + base, 0, (int)size, 0x00020000);
  }
  // (one select a round instead of a register for each of them from the loads to the stores)
  __device__ __forceinline__ void forget_rounds() { asm volatile("" : "+v"(off), "+v"(off_last)); }
  __device__ __forceinline__ bool own(int i) const { return (i < full ? off : i == full ? off_last : kOob) != kOob; }
  __device__ __forceinline__ uint32_t round(int i) const {     // (kOob stays beyond every range: the sum saturates)
    return __builtin_elementwise_add_sat(i < full ? off : i == full ? off_last : kOob, (uint32_t)i * step);
  }
  __device__ __forceinline__ void load(BufRsrc r, int i, V& v) const { buffer_load(r, round(i), v); }
  // the same, but where the thread has no pixel its vector of the first one, not zeros
  __device__ __forceinline__ void load_values(BufRsrc r, int i, V& v) const { buffer_load(r, own(i) ? round(i) : (uint32_t)(tx * sizeof(V)), v); }
  __device__ __forceinline__ void store(BufRsrc r, int i, const V& v) const { buffer_store(r, round(i), v); after_store(); }
};

// Threads hold M sets of N columns each, thread ty*sv + tx those of vector tx; brings the sums over ty to s_red[set][row][sv*N],
// NT*N floats a set, with as few rows as the return value says.  Lanes of a wavefront that share a vector are joined in registers.
template <int NT, int M, int N>
__device__ __forceinline__ int lay_columns(float (&v)[M][N], int sv, int rows, float* s_red) {
  __syncthreads();                 // what was in s_red has been read
  int at = threadIdx.x;
  bool lay = true;
  if (sv < 64 && (sv & (sv - 1)) == 0) {
    for (int d = 32; d >= sv; d >>= 1) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < N; ++j) v[m][j] += __shfl_xor(v[m][j], d);
    }
    const int lane = threadIdx.x & 63;
    lay = lane < sv;
    at = (threadIdx.x >> 6) * sv + lane;
    rows = NT / 64;
  }
  if (lay) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < N; ++j) s_red[(m * NT + at) * N + j] = v[m][j];
  }
  __syncthreads();
  return rows;
}
// Sums of ng groups of ncol neighbouring columns over the rows of width w, of M sets `set` floats apart; done(g, sums) by one
// thread of each.
template <int NT, int M, typename F>
__device__ __forceinline__ void sum_columns(const float* s_red, int set, int w, int rows, int ncol, int ng, F done) {
  int lanes = 64;
  while (lanes > 1 && lanes * ng > NT) lanes >>= 1;
  while (lanes > 1 && lanes >= 2 * rows * ncol) lanes >>= 1;
  const int k = threadIdx.x & (lanes - 1);
  for (int g0 = 0; g0 < ng; g0 += NT / lanes) {
    const int g = g0 + threadIdx.x / lanes;
    float sum[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      sum[m] = 0.0f;
      if (g < ng) {
        const float* col = s_red + m * set + g * ncol;
        if (ncol >= lanes) { for (int c = k; c < ncol; c += lanes) for (int r = 0; r < rows; ++r) sum[m] += col[r * w + c]; }
        else { for (int r = k; r < rows; r += lanes) for (int c = 0; c < ncol; ++c) sum[m] += col[r * w + c]; }
      }
      for (int d = lanes >> 1; d >= 1; d >>= 1) sum[m] += __shfl_xor(sum[m], d);
    }
    if (g < ng && k == 0) done(g, sum);
  }
}

constexpr int kMaxSliceGroups = 512, kMaxSlice = 256;     // of a slice: groups, vectors

// bf16 with two channels or more to a group: sums and sums of squares in one pass by dot products of pairs, exact products added
// in fp32, and var = E x^2 - mean^2 where mean^2 <= 4 var.  With sums that are off by a share d of their terms' magnitudes, that is off
// by at most 14 d var: E x^2 = var + mean^2 <= 5 var by 5 d var, mean^2 by 2 |mean| d E|x| <= 2 (2 sd) d (sqrt 5 sd) = 9 d var.  A slice
// with a group whose mean is farther out takes the deviations from the mean (d var), as all others do (fp32 has half the
// arithmetic for its bytes).
template <typename T, int ACT, int GV, int NT, int VPT>
__global__ __launch_bounds__(NT) void gn_forward_resident_kernel(GnArgs a) {
  constexpr int VE = 16 / sizeof(T);
  constexpr bool kPairs = sizeof(T) == 2 && GV < VE;
  typedef Tile<T, VE, NT> Tl;
  typedef Groups<VE, GV> Gr;
  __shared__ float s_red[NT * GV * (kPairs ? 2 : 1)], s_mean[kMaxSliceGroups], s_rstd[kMaxSliceGroups];
  Tl t(a, blockIdx.x, a.B * a.slices);
  if (!t.valid) return;            // (the number of tiles is rounded up to the XCDs)
  typename Tl::V v[VPT];
  {
    const BufRsrc x = t.buffer(a.x);
#pragma unroll
    for (int i = 0; i < VPT; ++i) t.load(x, i, v[i]);
  }
  // A thread adds VPT VE values at most, as 2^-7 of them (exact, so the same bits), and what it hands on is its share of the mean: sums
  // would leave the range before the mean does.
  static_assert(VPT * VE <= 128, "of 2^-7 of their size");
  constexpr float kPart = 0x1p-7f;
  const float share = 1.0f / ((float)a.P * (float)a.Cg);
  const int ncol = Gr::columns(a.Cg);
  const int ng = t.sv * VE / a.Cg, g_first = t.c_slice / a.Cg, w = t.sv * GV;
  float* out_mean = a.mean + (int64_t)t.b * a.G + g_first;
  float* out_rstd = a.rstd + (int64_t)t.b * a.G + g_first;
  int g[GV];
  Gr::find(t.c - t.c_slice, a.Cg, g);
  float mean[GV], f[VE];
  bool far = false;
  if constexpr (kPairs) {
    float acc[2][GV];
#pragma unroll
    for (int k = 0; k < GV; ++k) acc[0][k] = acc[1][k] = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {            // (past the end: zeros)
      forget(v[i]);
#pragma unroll
      for (int j = 0; j < VE; j += 2) {
        const int k = Gr::of(j);
        acc[0][k] = dot_pairs(v[i][j / 2], 0x3c003c00u, acc[0][k]);      // kPart
        acc[1][k] = dot_pairs(v[i][j / 2], v[i][j / 2], acc[1][k]);
      }
    }
#pragma unroll
    for (int k = 0; k < GV; ++k) { acc[0][k] *= share / kPart; acc[1][k] *= share; }
    const int rows = lay_columns<NT, 2, GV>(acc, t.sv, t.rows, s_red);
    sum_columns<NT, 2>(s_red, NT * GV, w, rows, ncol, ng, [&](int k, const float (&sum)[2]) {
      const float mu = sum[0], var = fmaf(-mu, mu, sum[1]), r = rstd_of(var, a.eps);
      if (!(mu * mu <= 4.0f * var) || !(var < __builtin_inff())) far = true;      // (too far out, squares out of range, or no numbers)
      s_mean[k] = mu; s_rstd[k] = r;
      out_mean[k] = mu; out_rstd[k] = r;
    });
    far = __syncthreads_or(far);
  } else {
    float acc[1][GV];
#pragma unroll
    for (int k = 0; k < GV; ++k) acc[0][k] = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {            // (past the end: zeros)
      forget(v[i]);
      unpack<T, VE>(v[i], f);
      float s[GV];
#pragma unroll
      for (int k = 0; k < GV; ++k) s[k] = 0.0f;
#pragma unroll
      for (int j = 0; j < VE; ++j) s[Gr::of(j)] = fmaf(f[j], kPart, s[Gr::of(j)]);
#pragma unroll
      for (int k = 0; k < GV; ++k) acc[0][k] += s[k];
    }
#pragma unroll
    for (int k = 0; k < GV; ++k) acc[0][k] *= share / kPart;
    const int rows = lay_columns<NT, 1, GV>(acc, t.sv, t.rows, s_red);
    sum_columns<NT, 1>(s_red, 0, w, rows, ncol, ng, [&](int k, const float (&sum)[1]) { s_mean[k] = sum[0]; });
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < GV; ++k) mean[k] = s_mean[g[k]];
  if (!kPairs || far) {
    float acc[1][GV];
#pragma unroll
    for (int k = 0; k < GV; ++k) acc[0][k] = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      forget(v[i]);
      unpack<T, VE>(v[i], f);
      float s[GV];
#pragma unroll
      for (int k = 0; k < GV; ++k) s[k] = 0.0f;
#pragma unroll
      for (int j = 0; j < VE; ++j) { const float d = f[j] - mean[Gr::of(j)]; s[Gr::of(j)] = fmaf(d, d, s[Gr::of(j)]); }
      const bool own = t.own(i);               // (a select, no factor 0: the mean's square may be out of range)
#pragma unroll
      for (int k = 0; k < GV; ++k) acc[0][k] += own ? s[k] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < GV; ++k) acc[0][k] *= share;
    const int rows = lay_columns<NT, 1, GV>(acc, t.sv, t.rows, s_red);
    sum_columns<NT, 1>(s_red, 0, w, rows, ncol, ng, [&](int k, const float (&sum)[1]) {
      const float r = rstd_of(sum[0], a.eps);
      s_rstd[k] = r;
      out_mean[k] = s_mean[k]; out_rstd[k] = r;
    });
    __syncthreads();
  }
  // z = (x - mean) (rstd gamma) + beta
  Affine<VE> af(a, t.c);
#pragma unroll
  for (int j = 0; j < VE; ++j) af.gamma[j] *= s_rstd[g[Gr::of(j)]];
  const BufRsrc y = t.buffer(a.out);
  t.forget_rounds();
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    forget(v[i]);
    unpack<T, VE>(v[i], f);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = act_of<T, ACT>(fmaf(f[j] - mean[Gr::of(j)], af.gamma[j], af.beta[j]));
    t.store(y, i, pack<T, VE>(f));
  }
}

// part[0][b][c] = sum dz, part[1][b][c] = sum dz xhat.  A vector's channels go four at a time: unpacked values of eight (bf16) do not
// fit beside the held vectors and the channels' constants.  (Vectors of four bf16 channels fit, but twice the loads cost more:
// 256 x 28 x 28 x 512 174 us against 148.)
template <typename T, int ACT, int GV, int NT, int VPT>
__global__ __launch_bounds__(NT) void gn_backward_resident_kernel(GnArgs a) {
  constexpr int VE = 16 / sizeof(T);
  typedef Tile<T, VE, NT> Tl;
  typedef Groups<VE, GV> Gr;
  __shared__ float s_red[2 * NT * VE], s_c[2][kMaxSlice * VE], s_g[2][kMaxSliceGroups];
  Tl t(a, blockIdx.x, a.B * a.slices);
  if (!t.valid) return;
  typename Tl::V vx[VPT], vd[VPT];
  {
    const BufRsrc x = t.buffer(a.x), dy = t.buffer(a.dy);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      // (SiLU' is taken past the end as well, where dy = 0: beside an x that is none of the image's, its z may be infinite, and 0 times
      // what comes of that is NaN.  A select behind it costs 2 to 5 % of the kernel.)
      if (ACT == DAT_ACT_SILU) t.load_values(x, i, vx[i]); else t.load(x, i, vx[i]);
      t.load(dy, i, vd[i]);
    }
  }
  const float n = (float)a.P * (float)a.Cg;
  const int w = t.sv * VE, ng = w / a.Cg, g_first = t.c_slice / a.Cg;
  int g[GV];
  Gr::find(t.c, a.Cg, g);
  float mean[GV], rstd[GV], s[2][VE];
  const Affine<VE> af(a, t.c);
#pragma unroll
  for (int k = 0; k < GV; ++k) { mean[k] = a.mean_in[(int64_t)t.b * a.G + g[k]]; rstd[k] = a.rstd_in[(int64_t)t.b * a.G + g[k]]; }
#pragma unroll
  for (int j = 0; j < VE; ++j) s[0][j] = s[1][j] = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {          // (past the end: dy = 0)
    forget(vx[i]);
    forget(vd[i]);
#pragma unroll
    for (int h = 0; h < VE; h += 4) {
      float f[4], d[4];
      unpack4<T>(vx[i], h, f);
      if constexpr (ACT == DAT_ACT_RELU) {     // dy becomes dz where it is held: the second pass needs no z
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool on = gn_z(f[j] - mean[Gr::of(h + j)], rstd[Gr::of(h + j)], af.gamma[h + j], af.beta[h + j]) > 0.0f;
          const uint32_t whole = 0xffffffffu, half = j % 2 ? 0x0000ffffu : 0xffff0000u;   // what stays if it is off
          vd[i][sizeof(T) == 4 ? h + j : (h + j) / 2] &= on ? whole : sizeof(T) == 4 ? 0u : half;
        }
      }
      unpack4<T>(vd[i], h, d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = Gr::of(h + j);
        const float xm = f[j] - mean[k];
        if constexpr (ACT == DAT_ACT_SILU) d[j] = silu_dz<T>(fmaf(xm, rstd[k] * af.gamma[h + j], af.beta[h + j]), d[j]);
        s[0][h + j] += d[j]; s[1][h + j] = fmaf(d[j], xm, s[1][h + j]);
      }
      __builtin_amdgcn_sched_barrier(0);       // (the scheduler would unpack them all first, and spill)
    }
    if (ACT == DAT_ACT_RELU) forget(vd[i]);    // (masked here, not where it is read)
  }
#pragma unroll
  for (int j = 0; j < VE; ++j) { s[1][j] *= rstd[Gr::of(j)]; forget(s[1][j]); }   // (here, not sunk below the first barrier)
  float* part = a.part + (int64_t)t.b * a.C + t.c_slice;
  const int rows = lay_columns<NT, 2, VE>(s, t.sv, t.rows, s_red);
  sum_columns<NT, 2>(s_red, NT * VE, w, rows, 1, w, [&](int c, const float (&sum)[2]) {
    const float gamma = a.gamma ? a.gamma[t.c_slice + c] : 1.0f;
    part[c] = sum[0]; part[(int64_t)a.B * a.C + c] = sum[1];
    s_c[0][c] = gamma * sum[0]; s_c[1][c] = gamma * sum[1];
  });
  __syncthreads();
  sum_columns<NT, 2>(s_c[0], kMaxSlice * VE, 0, 1, a.Cg, ng, [&](int k, const float (&sum)[2]) {
    s_g[0][k] = __fdiv_rn(sum[0], n); s_g[1][k] = __fdiv_rn(sum[1], n);
  });
  __syncthreads();
  // dx = rstd (gamma dz - c1 - xhat c2) = (rstd gamma) dz + ((x - mean) (-rstd^2 c2) - rstd c1).  A group of one value does not depend on
  // it: the terms cancel but for their rounding, and with rstd = 0 altogether (x - mean is 0, z = beta all the same; images of one pixel
  // take the smallest tile).
  float q1[GV], q2[GV];
  if (VPT == 2 && n == 1.0f) {
#pragma unroll
    for (int k = 0; k < GV; ++k) rstd[k] = 0.0f;
  }
#pragma unroll
  for (int k = 0; k < GV; ++k) { q1[k] = -rstd[k] * s_g[0][g[k] - g_first]; q2[k] = -(rstd[k] * rstd[k]) * s_g[1][g[k] - g_first]; }
  float scale[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) scale[j] = rstd[Gr::of(j)] * af.gamma[j];
  const BufRsrc dx = t.buffer(a.out);
  t.forget_rounds();
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    forget(vx[i]);
    forget(vd[i]);
#pragma unroll
    for (int h = 0; h < VE; h += 4) {
      float f[4], d[4];
      unpack4<T>(vx[i], h, f);
      unpack4<T>(vd[i], h, d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = Gr::of(h + j);
        const float xm = f[j] - mean[k];
        if constexpr (ACT == DAT_ACT_SILU) d[j] = silu_dz<T>(fmaf(xm, scale[h + j], af.beta[h + j]), d[j]);
        f[j] = fmaf(scale[h + j], d[j], fmaf(xm, q2[k], q1[k]));
      }
      pack4<T>(f, h, vx[i]);
    }
    t.store(dx, i, vx[i]);
  }
}

// ---- split -------------------------------------------------------------------------------------------------------------
// Workgroup: image, range of `chunk` pixels, block of vectors of channels; the threads of one vector take pixels in turn.
constexpr int kT = 256;
constexpr int kHeld = 8;          // pixels a thread of the forward statistics holds: chunk = kHeld * rows

template <typename T, int VE, bool BACK> struct Range {   // BACK: images from the last to the first
  typedef typename Vec<T, VE>::type V;
  int sv, rows, tx, ty, c, p0, p1;           // p0: own first pixel; p1: end of the range
  int64_t base;                              // vectors of the image's first pixel, own channels
  int b, chunk;
  __device__ __forceinline__ Range(const GnArgs& a) {
    const int per = a.chunks * a.slices;
    b = blockIdx.x / per;
    const int rest = blockIdx.x - b * per, slice = rest / a.chunks;
    chunk = rest - slice * a.chunks;
    if (BACK) b = a.B - 1 - b;
    sv = min(a.sv, a.nv - slice * a.sv);
    rows = kT / sv;
    ty = threadIdx.x / sv; tx = threadIdx.x - ty * sv;
    const int v = slice * a.sv + tx;
    c = v * VE;
    p1 = min(a.P, (chunk + 1) * a.chunk);
    p0 = ty < rows ? chunk * a.chunk + ty : p1;
    base = (int64_t)b * a.P * a.nv + v;
  }
};

// Every channel's mean and sum of squared deviations within the range: part[(b, chunk)][0..1][c].  A range has kHeld kT pixels at most:
// as 2^-11 of their size (exact) their sum stays in range.
static_assert(kHeld * kT <= 2048, "of 2^-11 of their size");
constexpr float kRangePart = 0x1p-11f;
template <typename T, int VE>
__global__ __launch_bounds__(kT) void gn_stats_kernel(GnArgs a) {
  __shared__ float s_red[VE * kT], s_mean[VE * 32];      // (a slice has at most 32 vectors)
  const Range<T, VE, false> r(a);
  const typename Range<T, VE, false>::V* x = reinterpret_cast<const typename Range<T, VE, false>::V*>(a.x) + r.base;
  typename Range<T, VE, false>::V v[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) v[i] = x[(int64_t)min(r.p0 + i * r.rows, a.P - 1) * a.nv];
  float acc[1][VE], f[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) acc[0][j] = 0.0f;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (r.p0 + i * r.rows < r.p1) {
      unpack<T, VE>(v[i], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) acc[0][j] = fmaf(f[j], kRangePart, acc[0][j]);
    }
  const float n = (float)(r.p1 - r.chunk * a.chunk) * kRangePart;
  const int w = r.sv * VE;
  float* part = a.part + ((int64_t)r.b * a.chunks + r.chunk) * 2 * a.C + (r.c - r.tx * VE);
  int rows = lay_columns<kT, 1, VE>(acc, r.sv, r.rows, s_red);
  sum_columns<kT, 1>(s_red, 0, w, rows, 1, w, [&](int c, const float (&sum)[1]) { s_mean[c] = part[c] = __fdiv_rn(sum[0], n); });
  __syncthreads();
  float mean[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) { mean[j] = s_mean[r.tx * VE + j]; acc[0][j] = 0.0f; }
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (r.p0 + i * r.rows < r.p1) {
      unpack<T, VE>(v[i], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) { const float d = f[j] - mean[j]; acc[0][j] = fmaf(d, d, acc[0][j]); }
    }
  rows = lay_columns<kT, 1, VE>(acc, r.sv, r.rows, s_red);
  sum_columns<kT, 1>(s_red, 0, w, rows, 1, w, [&](int c, const float (&sum)[1]) { part[a.C + c] = sum[0]; });
}

// The joining kernels: one workgroup per image and group.  Threads lie along the group's channels, as many as it has up to kT (in
// powers of two), and what is left of them along the ranges.
struct JoinLanes {
  int width, rows, c, k;
  __device__ __forceinline__ explicit JoinLanes(int Cg) {
    width = 1;
    while (width < Cg && width < kT) width <<= 1;
    rows = kT / width; c = threadIdx.x & (width - 1); k = threadIdx.x / width;
  }
};
__device__ __forceinline__ float block_sum(float v, float* s) {
  v = lanes_sum<64>(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Means and squared deviations of a group's ranges and channels into one, by the deviations of the means from their own mean.
__global__ __launch_bounds__(kT) void gn_join_stats_kernel(GnArgs a) {
  __shared__ float s_sum[kT / 64];
  const int b = blockIdx.x / a.G, g = blockIdx.x - b * a.G;
  const float* part = a.part + (int64_t)b * a.chunks * 2 * a.C + g * a.Cg;
  const JoinLanes l(a.Cg);
  const float share = 1.0f / ((float)a.P * (float)a.Cg);
  float s = 0.0f;
  for (int c = l.c; c < a.Cg; c += l.width)
#pragma unroll 4
    for (int k = l.k; k < a.chunks; k += l.rows)
      s = fmaf((float)(min(a.P, (k + 1) * a.chunk) - k * a.chunk) * share, part[(int64_t)k * 2 * a.C + c], s);
  const float mean = block_sum(s, s_sum);
  s = 0.0f;
  for (int c = l.c; c < a.Cg; c += l.width)
#pragma unroll 4
    for (int k = l.k; k < a.chunks; k += l.rows) {
      const float* q = part + (int64_t)k * 2 * a.C + c;
      const float d = q[0] - mean;
      s = fmaf(q[a.C], share, fmaf((float)(min(a.P, (k + 1) * a.chunk) - k * a.chunk) * share * d, d, s));
    }
  s = block_sum(s, s_sum);
  if (threadIdx.x == 0) {
    a.mean[(int64_t)b * a.G + g] = mean;
    a.rstd[(int64_t)b * a.G + g] = rstd_of(s, a.eps);
  }
}

template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_apply_kernel(GnArgs a) {
  const Range<T, VE, true> r(a);
  if (r.p0 >= r.p1) return;
  typedef typename Range<T, VE, true>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  V* y = reinterpret_cast<V*>(a.out) + r.base;
  Affine<VE> w(a, r.c);
  float mean[VE], f[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean[g]; w.gamma[j] *= a.rstd[g];
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack<T, VE>(x[(int64_t)p * a.nv], f);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = act_of<T, ACT>(fmaf(f[j] - mean[j], w.gamma[j], w.beta[j]));
    y[(int64_t)p * a.nv] = pack<T, VE>(f);
  }
}

// Sums of dz and dz xhat of every channel within the range: ranges[(image of the batch, chunk)][0..1][c].
template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_grad_sums_kernel(GnArgs a, float* ranges) {
  __shared__ float s_red[2 * VE * kT];
  const Range<T, VE, false> r(a);
  typedef typename Range<T, VE, false>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  const V* dy = reinterpret_cast<const V*>(a.dy) + r.base;
  const Affine<VE> w(a, r.c);
  float mean[VE], rstd[VE], s[2][VE], f[VE], d[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean_in[g]; rstd[j] = a.rstd_in[g];
    s[0][j] = s[1][j] = 0.0f;
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack<T, VE>(x[(int64_t)p * a.nv], f);
    unpack<T, VE>(dy[(int64_t)p * a.nv], d);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float xm = f[j] - mean[j], dz = gn_dz<T, ACT>(xm, d[j], rstd[j], w.gamma[j], rstd[j] * w.gamma[j], w.beta[j]);
      s[0][j] += dz; s[1][j] = fmaf(dz, xm, s[1][j]);
    }
  }
#pragma unroll
  for (int j = 0; j < VE; ++j) s[1][j] *= rstd[j];
  float* out = ranges + ((int64_t)r.b * a.chunks + r.chunk) * 2 * a.C + (r.c - r.tx * VE);
  const int cols = r.sv * VE, rows = lay_columns<kT, 2, VE>(s, r.sv, r.rows, s_red);
  sum_columns<kT, 2>(s_red, kT * VE, cols, rows, 1, cols, [&](int c, const float (&sum)[2]) { out[c] = sum[0]; out[a.C + c] = sum[1]; });
}

// Sums over the ranges: of every channel to part[0][b][c] and [1][b][c] (as the resident kernel leaves them), and of the group, as
// means, to join[(b, g)][0..1].
__global__ __launch_bounds__(kT) void gn_join_grad_kernel(GnArgs a, const float* ranges, float* join) {
  __shared__ float s_sum[kT / 64], s_row[2][kT];
  const int b = blockIdx.x / a.G, g = blockIdx.x - b * a.G;
  const float* q = ranges + (int64_t)b * a.chunks * 2 * a.C + g * a.Cg;
  const JoinLanes l(a.Cg);
  float c1 = 0.0f, c2 = 0.0f;
  for (int c0 = 0; c0 < a.Cg; c0 += l.width) {
    const int c = c0 + l.c;
    float s1 = 0.0f, s2 = 0.0f;
    if (c < a.Cg) {
#pragma unroll 4
      for (int k = l.k; k < a.chunks; k += l.rows) { s1 += q[(int64_t)k * 2 * a.C + c]; s2 += q[(int64_t)k * 2 * a.C + a.C + c]; }
    }
    s_row[0][threadIdx.x] = s1; s_row[1][threadIdx.x] = s2;
    __syncthreads();
    if (l.k == 0 && c < a.Cg) {
      for (int r = 1; r < l.rows; ++r) { s1 += s_row[0][r * l.width + l.c]; s2 += s_row[1][r * l.width + l.c]; }
      float* part = a.part + (int64_t)b * a.C + g * a.Cg + c;
      part[0] = s1; part[(int64_t)a.B * a.C] = s2;
      const float gamma = a.gamma ? a.gamma[g * a.Cg + c] : 1.0f;
      c1 = fmaf(gamma, s1, c1); c2 = fmaf(gamma, s2, c2);
    }
    __syncthreads();
  }
  const float n = (float)a.P * (float)a.Cg;
  c1 = block_sum(c1, s_sum) / n;
  c2 = block_sum(c2, s_sum) / n;
  if (threadIdx.x == 0) { join[((int64_t)b * a.G + g) * 2] = c1; join[((int64_t)b * a.G + g) * 2 + 1] = c2; }
}

template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_grad_apply_kernel(GnArgs a, const float* join) {
  const Range<T, VE, true> r(a);
  if (r.p0 >= r.p1) return;
  typedef typename Range<T, VE, true>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  const V* dy = reinterpret_cast<const V*>(a.dy) + r.base;
  V* dx = reinterpret_cast<V*>(a.out) + r.base;
  const Affine<VE> w(a, r.c);
  float mean[VE], rstd[VE], q1[VE], q2[VE], f[VE], d[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean_in[g]; rstd[j] = a.P * a.Cg == 1 ? 0.0f : a.rstd_in[g];      // (as in the resident kernel)
    q1[j] = -rstd[j] * join[2 * g]; q2[j] = -(rstd[j] * rstd[j]) * join[2 * g + 1];
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack<T, VE>(x[(int64_t)p * a.nv], f);
    unpack<T, VE>(dy[(int64_t)p * a.nv], d);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float xm = f[j] - mean[j], dz = gn_dz<T, ACT>(xm, d[j], rstd[j], w.gamma[j], rstd[j] * w.gamma[j], w.beta[j]);
      f[j] = fmaf(rstd[j] * w.gamma[j], dz, fmaf(xm, q2[j], q1[j]));
    }
    dx[(int64_t)p * a.nv] = pack<T, VE>(f);
  }
}

// dbeta[c] and dgamma[c]: the sums over the images of part[0][b][c] and part[1][b][c].
constexpr int kParamRows = 16;
__global__ __launch_bounds__(64 * kParamRows) void gn_param_kernel(const float* part, int B, int C, float* dgamma, float* dbeta) {
  __shared__ float s[2][kParamRows][64];
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s1 = 0.0f, s2 = 0.0f;
  if (c < C)
#pragma unroll 8
    for (int b = row; b < B; b += kParamRows) { s1 += part[(int64_t)b * C + c]; s2 += part[(int64_t)(B + b) * C + c]; }
  s[0][row][lane] = s1; s[1][row][lane] = s2;
  __syncthreads();
  if (row == 0 && c < C) {
#pragma unroll
    for (int i = 1; i < kParamRows; ++i) { s1 += s[0][i][lane]; s2 += s[1][i][lane]; }
    dbeta[c] = s1; dgamma[c] = s2;
  }
}

// ---- which way ---------------------------------------------------------------------------------------------------------
int gcd(int a, int b) { while (b) { const int r = a % b; a = b; b = r; } return a; }

struct Plan {
  int ve;              // channels per vector: 16 bytes, or 1
  int nv, sv, slices;
  int nt, vpt;         // resident: threads, vectors each; nt = 0: split
  int chunk, chunks;   // split
};

Plan plan_of(bool backward, dat_dtype dtype, bool vectors, int B, int P, int C, int G) {
  Plan p{};
  const int width = dtype == DAT_BF16 ? 2 : 4, whole = 16 / width, Cg = C / G;
  p.ve = vectors && C % whole == 0 ? whole : 1;
  p.nv = C / p.ve;
  if (p.ve > 1) {
    const int unit = Cg / gcd(Cg, whole);              // vectors of the smallest slice of whole groups
    // Tiles of up to 16 vectors a thread (backward: 8 of x and 8 of dy), in the smallest workgroup that takes them: several on a
    // compute unit, each at its own stage.  Rows of a slice: 128 bytes forward (512 x 32 x 32 x 64 bf16 28.6 us against 35.6 with
    // 64, 128 x 32 x 32 x 160 fp32 48.6 against 60.5, 256 x 40 x 40 x 256 101.3 against 101.1), 64 where the image does not fit
    // so, and backward, where the workgroup that takes 128 is alone on its unit (256 x 28 x 28 x 512 146 us against 189).  Wider
    // where the image is small (256 x 7 x 7 x 2048 41 -> 23 us), narrower where there would be few tiles for 256 compute units, but not
    // where 64 bytes do not fit: such maps (bf16 backward from 56 x 56 up) go the split way, slices of 32 or 16 are not tried.
    static const int fwd[][2] = {{256, 2}, {256, 8}, {256, 16}, {512, 16}, {1024, 16}}, bwd[][2] = {{256, 2}, {256, 8}, {512, 8}, {1024, 8}};
    const int (*sizes)[2] = backward ? bwd : fwd;
    const int count = backward ? 4 : 5, nv = p.nv;
    auto fits = [&](int sv, int i) { return sv <= sizes[i][0] && (P + sizes[i][0] / sv - 1) / (sizes[i][0] / sv) <= sizes[i][1]; };
    int sv = unit, i = 0;
    while (sv * 16 < 64 && 2 * sv <= nv) sv *= 2;
    if (!backward && sv * 16 < 128 && 2 * sv <= nv && fits(2 * sv, count - 1)) sv *= 2;
    const int least = sv;
    while (2 * sv <= nv && fits(2 * sv, backward ? 1 : 2) && (int64_t)B * (nv / (2 * sv)) >= 1024) sv *= 2;
    if (sv == least) while (sv > unit && (int64_t)B * ((nv + sv - 1) / sv) < 512) sv /= 2;
    while (i < count && !fits(sv, i)) ++i;
    if (i < count && sv <= kMaxSlice && sv * whole / Cg <= kMaxSliceGroups && (int64_t)P * C * width < kOob) {
      p.sv = sv; p.nt = sizes[i][0]; p.vpt = sizes[i][1];
    }
    if (p.nt) { p.slices = (p.nv + p.sv - 1) / p.sv; return p; }
  }
  p.slices = (p.nv + 31) / 32;                          // at most 32 vectors wide: at least 64 pixels to a range
  p.sv = (p.nv + p.slices - 1) / p.slices;
  p.slices = (p.nv + p.sv - 1) / p.sv;
  p.chunk = kHeld * (kT / p.sv);
  p.chunks = (P + p.chunk - 1) / p.chunk;
  return p;
}

dat_status check(dat_dtype dtype, int B, int H, int W, int C, int groups) {
  if ((dtype != DAT_F32 && dtype != DAT_BF16) || B < 0 || H < 1 || W < 1 || C < 1 || groups < 1 || C % groups) return DAT_ERR_ARG;
  constexpr int64_t most = 1 << 30;
  if ((int64_t)H * W > most || (int64_t)H * W * C > most || (int64_t)B * C > most) return DAT_ERR_SHAPE;
  return DAT_OK;
}

size_t workspace_of(const Plan& p, bool backward, int B, int C, int G) {
  if (backward) return p.nt ? (size_t)B * C * 8 : ((size_t)B * C + (size_t)B * G + (size_t)B * p.chunks * C) * 8;
  return p.nt ? 0 : (size_t)B * p.chunks * C * 8;
}

#define DAT_GN_ACT(act, ...)                                                              \
  do {                                                                                    \
    if (act == DAT_ACT_RELU) { constexpr int ACT = DAT_ACT_RELU; __VA_ARGS__; }           \
    else if (act == DAT_ACT_SILU) { constexpr int ACT = DAT_ACT_SILU; __VA_ARGS__; }      \
    else { constexpr int ACT = DAT_ACT_NONE; __VA_ARGS__; }                               \
  } while (0)

bool fits_launches(const Plan& p, int B, int G) {
  if (p.nt) return fits_launch((int64_t)B * p.slices + kXcds, p.nt);
  return fits_launch((int64_t)B * p.chunks * p.slices, kT) && fits_launch((int64_t)B * G, kT);
}

inline unsigned tiles_of(const GnArgs& a) { return (unsigned)(((int64_t)a.B * a.slices + kXcds - 1) / kXcds * kXcds); }

template <typename T, int GV> void launch_forward_resident(const Plan& p, const GnArgs& a, dat_act act, hipStream_t st) {
  const dim3 grid(tiles_of(a));
#define DAT_GN_SIZE(NT, VPT) if (p.nt == NT && p.vpt == VPT) DAT_GN_ACT(act, hipLaunchKernelGGL((gn_forward_resident_kernel<T, ACT, GV, NT, VPT>), grid, dim3(NT), 0, st, a))
  DAT_GN_SIZE(256, 2); DAT_GN_SIZE(256, 8); DAT_GN_SIZE(256, 16); DAT_GN_SIZE(512, 16); DAT_GN_SIZE(1024, 16);
#undef DAT_GN_SIZE
}
template <typename T, int GV> void launch_backward_resident(const Plan& p, const GnArgs& a, dat_act act, hipStream_t st) {
  const dim3 grid(tiles_of(a));
#define DAT_GN_SIZE(NT, VPT) if (p.nt == NT && p.vpt == VPT) DAT_GN_ACT(act, hipLaunchKernelGGL((gn_backward_resident_kernel<T, ACT, GV, NT, VPT>), grid, dim3(NT), 0, st, a))
  DAT_GN_SIZE(256, 2); DAT_GN_SIZE(256, 8); DAT_GN_SIZE(512, 8); DAT_GN_SIZE(1024, 8);
#undef DAT_GN_SIZE
}
template <int VE, typename F> void with_groups(int Cg, F f) {
  const int gv = Cg % VE == 0 ? 1 : Cg > 1 && VE % Cg == 0 ? VE / Cg : VE;
  if (gv == 1) f(std::integral_constant<int, 1>());
  else if (gv == 2) f(std::integral_constant<int, 2>());
  else if (gv == 4) f(std::integral_constant<int, 4>());
  else if constexpr (VE == 8) f(std::integral_constant<int, 8>());
}
template <typename T> void launch_resident(bool backward, const Plan& p, const GnArgs& a, dat_act act, hipStream_t st) {
  with_groups<16 / sizeof(T)>(a.Cg, [&](auto gv) {
    if (backward) launch_backward_resident<T, decltype(gv)::value>(p, a, act, st);
    else launch_forward_resident<T, decltype(gv)::value>(p, a, act, st);
  });
}
template <typename T, int VE> void launch_forward_split(const GnArgs& a, dat_act act, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.chunks * a.slices));
  hipLaunchKernelGGL((gn_stats_kernel<T, VE>), grid, dim3(kT), 0, st, a);
  hipLaunchKernelGGL(gn_join_stats_kernel, dim3((unsigned)((int64_t)a.B * a.G)), dim3(kT), 0, st, a);
  DAT_GN_ACT(act, hipLaunchKernelGGL((gn_apply_kernel<T, VE, ACT>), grid, dim3(kT), 0, st, a));
}
template <typename T, int VE> void launch_backward_split(const GnArgs& a, dat_act act, float* join, float* ranges, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.chunks * a.slices));
  DAT_GN_ACT(act, hipLaunchKernelGGL((gn_grad_sums_kernel<T, VE, ACT>), grid, dim3(kT), 0, st, a, ranges));
  hipLaunchKernelGGL(gn_join_grad_kernel, dim3((unsigned)((int64_t)a.B * a.G)), dim3(kT), 0, st, a, (const float*)ranges, join);
  DAT_GN_ACT(act, hipLaunchKernelGGL((gn_grad_apply_kernel<T, VE, ACT>), grid, dim3(kT), 0, st, a, (const float*)join));
}

}  // namespace
}  // namespace dat

using namespace dat;

// (The larger of the two needs: buffers that are not 16-byte aligned take the path of single elements.)
extern "C" size_t dat_group_norm_workspace(int pass, dat_dtype dtype, int B, int H, int W, int C, int groups) {
  if (check(dtype, B, H, W, C, groups) != DAT_OK || (pass != 0 && pass != 1) || B == 0) return 0;
  size_t most = 0;
  for (int v = 0; v < 2; ++v) {
    const size_t s = workspace_of(plan_of(pass == 1, dtype, v == 1, B, H * W, C, groups), pass == 1, B, C, groups);
    if (s > most) most = s;
  }
  return most;
}

extern "C" dat_status dat_group_norm_forward(const void* x, const float* gamma, const float* beta, dat_dtype dtype, int B, int H,
                                             int W, int C, int groups, float eps, dat_act act, void* y, float* mean, float* rstd,
                                             void* workspace, size_t workspace_bytes, void* stream) {
  const dat_status s = check(dtype, B, H, W, C, groups);
  if (s != DAT_OK) return s;
  if (!gamma != !beta || !(eps >= 0.0f) || (unsigned)act > DAT_ACT_SILU || (B > 0 && (!x || !y || !mean || !rstd))) return DAT_ERR_ARG;
  const size_t width = dtype == DAT_BF16 ? 2 : 4, need = dat_group_norm_workspace(0, dtype, B, H, W, C, groups);
  if (!aligned(x, width) || !aligned(y, width) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return DAT_ERR_ARG;
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return DAT_ERR_ARG;
  if (overlaps(x, y, (size_t)B * H * W * C * width)) return DAT_ERR_ARG;
  if (B == 0) return DAT_OK;
  const Plan p = plan_of(false, dtype, aligned(x, 16) && aligned(y, 16), B, H * W, C, groups);
  GnArgs a{x, nullptr, gamma, beta, nullptr, nullptr, y, mean, rstd, (float*)workspace, B, H * W, C, groups, C / groups,
           p.nv, p.sv, p.slices, p.chunk, p.chunks, eps};
  if (!fits_launches(p, B, groups)) return DAT_ERR_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  if (p.nt) {
    if (dtype == DAT_BF16) launch_resident<bf16_t>(false, p, a, act, st); else launch_resident<float>(false, p, a, act, st);
    DAT_LAUNCH_CHECK();
    return DAT_OK;
  }
  if (dtype == DAT_BF16) { if (p.ve > 1) launch_forward_split<bf16_t, 8>(a, act, st); else launch_forward_split<bf16_t, 1>(a, act, st); }
  else { if (p.ve > 1) launch_forward_split<float, 4>(a, act, st); else launch_forward_split<float, 1>(a, act, st); }
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

extern "C" dat_status dat_group_norm_backward(const void* x, const void* dy, const float* gamma, const float* beta,
                                              const float* mean, const float* rstd, dat_dtype dtype, int B, int H, int W, int C,
                                              int groups, dat_act act, void* dx, float* dgamma, float* dbeta, void* workspace,
                                              size_t workspace_bytes, void* stream) {
  const dat_status s = check(dtype, B, H, W, C, groups);
  if (s != DAT_OK) return s;
  if (!gamma != !beta || !dgamma != !dbeta || (unsigned)act > DAT_ACT_SILU || (B > 0 && (!x || !dy || !dx || !mean || !rstd))) return DAT_ERR_ARG;
  const size_t width = dtype == DAT_BF16 ? 2 : 4, need = dat_group_norm_workspace(1, dtype, B, H, W, C, groups);
  if (!aligned(x, width) || !aligned(dy, width) || !aligned(dx, width) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return DAT_ERR_ARG;
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return DAT_ERR_ARG;
  if (overlaps(x, dx, (size_t)B * H * W * C * width) || overlaps(dy, dx, (size_t)B * H * W * C * width)) return DAT_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const Plan p = plan_of(true, dtype, aligned(x, 16) && aligned(dy, 16) && aligned(dx, 16), B, H * W, C, groups);
  GnArgs a{x, dy, gamma, beta, mean, rstd, dx, nullptr, nullptr, (float*)workspace, B, H * W, C, groups, C / groups,
           p.nv, p.sv, p.slices, p.chunk, p.chunks, 0.0f};
  if (!fits_launches(p, B, groups) || !fits_launch((C + 63) / 64, 64 * kParamRows)) return DAT_ERR_SHAPE;
  if (p.nt && B > 0) {
    if (dtype == DAT_BF16) launch_resident<bf16_t>(true, p, a, act, st); else launch_resident<float>(true, p, a, act, st);
    DAT_LAUNCH_CHECK();
  } else if (B > 0) {
    float *join = a.part + (int64_t)B * C * 2, *ranges = join + (int64_t)B * groups * 2;
    if (dtype == DAT_BF16) { if (p.ve > 1) launch_backward_split<bf16_t, 8>(a, act, join, ranges, st); else launch_backward_split<bf16_t, 1>(a, act, join, ranges, st); }
    else { if (p.ve > 1) launch_backward_split<float, 4>(a, act, join, ranges, st); else launch_backward_split<float, 1>(a, act, join, ranges, st); }
    DAT_LAUNCH_CHECK();
  }
  if (dgamma) {
    hipLaunchKernelGGL(gn_param_kernel, dim3((C + 63) / 64), dim3(64 * kParamRows), 0, st, (const float*)workspace, B, C, dgamma, dbeta);
    DAT_LAUNCH_CHECK();
  }
  return DAT_OK;
}
