// Group normalisation with an activation, channels last, forward and backward.
//
// An image is P pixels of C channels; a thread owns one 16-byte vector of channels (VE of them) at several pixels, so its scale,
// shift and statistics are registers and a wavefront reads whole pixel rows.  Every sum runs in a fixed order (thread, LDS,
// partial sums in memory): the same bits on every call.  Variances are sums of squared deviations from a mean, taken from values
// that are still in registers, never a difference of two large sums.
//
// Two ways, both bound by HBM:
//   resident  one workgroup holds a slice of whole groups of one image in registers: every tensor is moved once.
//   split     an image's slice is too large for that: partial sums over ranges of pixels, a small kernel that joins them, and a
//             second pass over the tensors.  Images go in batches whose tensors fit into the last-level cache, where the second
//             pass finds them.
#include "kernels.h"

namespace dat {
namespace {

struct GnArgs {
  const void* x; const void* dy; const float* gamma; const float* beta; const float* mean_in; const float* rstd_in;
  void* out; float* mean; float* rstd; float* part;
  int B, P, C, G, Cg;
  int nv;            // vectors of a pixel's channels
  int sv, slices;    // vectors of a slice, slices of a pixel
  int chunk, chunks; // split: pixels of a range, ranges of an image
  int b0;            // split: first image of the batch
  float eps;
};

template <typename T, int VE> struct Vec;
template <> struct Vec<float, 4> { typedef float4 type; };
template <> struct Vec<bf16_t, 8> { typedef uint4 type; };
template <> struct Vec<float, 1> { typedef float type; };
template <> struct Vec<bf16_t, 1> { typedef bf16_t type; };

__device__ __forceinline__ void unpack(const float4& v, float (&f)[4]) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void unpack(const float& v, float (&f)[1]) { f[0] = v; }
__device__ __forceinline__ void unpack(const bf16_t& v, float (&f)[1]) { f[0] = bf2f(v); }
__device__ __forceinline__ void pack(const float (&f)[4], float4* v) { *v = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void pack(const float (&f)[8], uint4* v) {
  *v = make_uint4(f2bf_pack(f[0], f[1]), f2bf_pack(f[2], f[3]), f2bf_pack(f[4], f[5]), f2bf_pack(f[6], f[7]));
}
__device__ __forceinline__ void pack(const float (&f)[1], float* v) { *v = f[0]; }
__device__ __forceinline__ void pack(const float (&f)[1], bf16_t* v) { *v = f2bf(f[0]); }

__device__ __forceinline__ float gn_xhat(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }
__device__ __forceinline__ float gn_z(float xhat, float gamma, float beta) { return __fadd_rn(__fmul_rn(xhat, gamma), beta); }
// 1 / (1 + e^-z).  The results that leave in bf16 take the hardware's exponential and reciprocal, a few units of 2^-23 off.
template <typename T> __device__ __forceinline__ float sigmoid(float z) {
  if (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  return 1.0f / (1.0f + expf(-z));
}
template <typename T, int ACT> __device__ __forceinline__ float act_of(float z) {
  if (ACT == DAT_ACT_RELU) return z <= 0.0f ? 0.0f : z;      // NaN stays
  if (ACT == DAT_ACT_SILU) return z * sigmoid<T>(z);
  return z;
}
template <typename T, int ACT> __device__ __forceinline__ float act_grad(float z, float dy) {
  if (ACT == DAT_ACT_RELU) return z > 0.0f ? dy : 0.0f;
  if (ACT == DAT_ACT_SILU) { const float s = sigmoid<T>(z); return dy * (s * (1.0f + z * (1.0f - s))); }
  return dy;
}
__device__ __forceinline__ float rstd_of(float sum, float n, float eps) { return __fdiv_rn(1.0f, sqrtf(__fdiv_rn(sum, n) + eps)); }

// The scale and shift of a thread's channels.
template <int VE> struct Affine {
  float gamma[VE], beta[VE];
  __device__ __forceinline__ Affine(const GnArgs& a, int c) {
#pragma unroll
    for (int j = 0; j < VE; ++j) { gamma[j] = a.gamma ? a.gamma[c + j] : 1.0f; beta[j] = a.gamma ? a.beta[c + j] : 0.0f; }
  }
};

// ---- resident ----------------------------------------------------------------------------------------------------------
// Thread tid = ty*sv + tx holds vector tx of the slice at pixels ty, ty + rows, ...: at most VPT of them.
template <typename T, int NT, int VPT> struct Tile {
  static constexpr int VE = 16 / sizeof(T);
  typedef typename Vec<T, VE>::type V;
  int sv, rows, tx, ty, count, c;            // width of this slice, threads along the pixels, own pixels, first channel
  int64_t at, step;                          // first vector, distance to the next one (vectors)
  __device__ __forceinline__ Tile(const GnArgs& a, int b, int slice) {
    sv = min(a.sv, a.nv - slice * a.sv);
    rows = NT / sv;
    ty = threadIdx.x / sv; tx = threadIdx.x - ty * sv;
    count = ty < rows && ty < a.P ? (a.P - ty + rows - 1) / rows : 0;
    const int v = slice * a.sv + tx;
    c = v * VE;
    at = ((int64_t)b * a.P + min(ty, a.P - 1)) * a.nv + v;
    step = (int64_t)rows * a.nv;
  }
  // Pixels past the end: the last own one again (the first, for a thread without any), not used.
  __device__ __forceinline__ void load(const void* p, V (&v)[VPT]) const {
    const V* src = reinterpret_cast<const V*>(p) + at;
#pragma unroll
    for (int i = 0; i < VPT; ++i) v[i] = src[min(i, max(count - 1, 0)) * step];
  }
};

// Joins what the threads of a slice hold for SUB columns each, columns of a group being ncol neighbours: the groups' sums in
// s_out.  Lanes of a group take rows (or columns, where there are more of these) in turn.
template <int NT, int SUB>
__device__ __forceinline__ void group_sums(const float (&v)[SUB], int sv, int rows, int ncol, int ng, float* s_red, float* s_out) {
  __syncthreads();                 // s_red and s_out of the round before have been read
#pragma unroll
  for (int j = 0; j < SUB; ++j) s_red[threadIdx.x * SUB + j] = v[j];
  __syncthreads();
  int lanes = 64;
  while (lanes > 1 && lanes * ng > NT) lanes >>= 1;
  const int k = threadIdx.x & (lanes - 1), w = sv * SUB;
  for (int g0 = 0; g0 < ng; g0 += NT / lanes) {
    const int g = g0 + threadIdx.x / lanes;
    float sum = 0.0f;
    if (g < ng) {
      const float* col = s_red + g * ncol;
      if (ncol >= lanes) { for (int c = k; c < ncol; c += lanes) for (int r = 0; r < rows; ++r) sum += col[r * w + c]; }
      else { for (int r = k; r < rows; r += lanes) for (int c = 0; c < ncol; ++c) sum += col[r * w + c]; }
    }
    for (int d = lanes >> 1; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (g < ng && k == 0) s_out[g] = sum;
  }
  __syncthreads();
}

constexpr int kMaxSliceGroups = 512;

// SUB = 1: a vector lies inside one group; SUB = VE: columns are single channels.
template <typename T, int ACT, bool WHOLE, int NT, int VPT>
__global__ __launch_bounds__(NT) void gn_forward_resident_kernel(GnArgs a) {
  typedef Tile<T, NT, VPT> Tl;
  constexpr int VE = Tl::VE, SUB = WHOLE ? 1 : VE;
  __shared__ float s_red[NT * SUB], s_mean[kMaxSliceGroups], s_rstd[kMaxSliceGroups];
  const int b = blockIdx.x / a.slices, slice = blockIdx.x - b * a.slices;
  const Tl t(a, b, slice);
  typename Tl::V v[VPT];
  t.load(a.x, v);
  const int ng = t.sv * VE / a.Cg, g_first = slice * a.sv * VE / a.Cg, ncol = WHOLE ? a.Cg / VE : a.Cg;
  const float n = (float)a.P * (float)a.Cg;
  float acc[SUB], f[VE];
#pragma unroll
  for (int j = 0; j < SUB; ++j) acc[j] = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (i < t.count) {
      unpack(v[i], f);
      if (WHOLE) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < VE; ++j) s += f[j];
        acc[0] += s;
      } else {
#pragma unroll
        for (int j = 0; j < SUB; ++j) acc[j] += f[j];
      }
    }
  group_sums<NT, SUB>(acc, t.sv, t.rows, ncol, ng, s_red, s_mean);
  float mean[SUB], rstd[SUB];
  const int c0 = t.tx * VE;
#pragma unroll
  for (int j = 0; j < SUB; ++j) { mean[j] = t.count ? __fdiv_rn(s_mean[(c0 + j) / a.Cg], n) : 0.0f; acc[j] = 0.0f; }
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (i < t.count) {
      unpack(v[i], f);
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float d = f[j] - mean[WHOLE ? 0 : j];
        if (WHOLE) s = fmaf(d, d, s); else acc[j] = fmaf(d, d, acc[j]);
      }
      if (WHOLE) acc[0] += s;
    }
  group_sums<NT, SUB>(acc, t.sv, t.rows, ncol, ng, s_red, s_rstd);
  for (int g = threadIdx.x; g < ng; g += NT) {
    a.mean[(int64_t)b * a.G + g_first + g] = __fdiv_rn(s_mean[g], n);
    a.rstd[(int64_t)b * a.G + g_first + g] = rstd_of(s_rstd[g], n, a.eps);
  }
  if (t.count == 0) return;
#pragma unroll
  for (int j = 0; j < SUB; ++j) rstd[j] = rstd_of(s_rstd[(c0 + j) / a.Cg], n, a.eps);
  const Affine<VE> w(a, t.c);
  typename Tl::V* y = reinterpret_cast<typename Tl::V*>(a.out) + t.at;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (i < t.count) {
      unpack(v[i], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] = act_of<T, ACT>(gn_z(gn_xhat(f[j], mean[WHOLE ? 0 : j], rstd[WHOLE ? 0 : j]), w.gamma[j], w.beta[j]));
      pack(f, y + i * t.step);
    }
}

// s1[c] = sum dz, s2[c] = sum dz xhat of the slice's channels, joined over the pixels; written to part as well.
template <int NT, int VE>
__device__ __forceinline__ void channel_sums(const float (&v)[VE], int sv, int rows, float* s_red, float* s_out, float* part) {
  __syncthreads();
#pragma unroll
  for (int j = 0; j < VE; ++j) s_red[threadIdx.x * VE + j] = v[j];
  __syncthreads();
  const int w = sv * VE;
  int lanes = 64;
  while (lanes > 1 && lanes * w > NT) lanes >>= 1;
  const int k = threadIdx.x & (lanes - 1);
  for (int c0 = 0; c0 < w; c0 += NT / lanes) {
    const int c = c0 + threadIdx.x / lanes;
    float sum = 0.0f;
    if (c < w) for (int r = k; r < rows; r += lanes) sum += s_red[r * w + c];
    for (int d = lanes >> 1; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    if (c < w && k == 0) { s_out[c] = sum; part[c] = sum; }
  }
}

// part[0][b][c] = sum dz, part[1][b][c] = sum dz xhat.
template <typename T, int ACT, int NT, int VPT>
__global__ __launch_bounds__(NT) void gn_backward_resident_kernel(GnArgs a) {
  typedef Tile<T, NT, VPT> Tl;
  constexpr int VE = Tl::VE;
  __shared__ float s_red[NT * VE];
  __shared__ float s_c[2][NT * VE];
  const int b = blockIdx.x / a.slices, slice = blockIdx.x - b * a.slices;
  const Tl t(a, b, slice);
  typename Tl::V vx[VPT], vd[VPT];
  t.load(a.x, vx);
  t.load(a.dy, vd);
  float mean[VE], rstd[VE], s1[VE], s2[VE], f[VE], d[VE];
  const Affine<VE> w(a, t.c);
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)b * a.G + (t.c + j) / a.Cg;
    mean[j] = a.mean_in[g]; rstd[j] = a.rstd_in[g];
    s1[j] = s2[j] = 0.0f;
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (i < t.count) {
      unpack(vx[i], f);
      unpack(vd[i], d);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float xhat = gn_xhat(f[j], mean[j], rstd[j]);
        const float dz = act_grad<T, ACT>(gn_z(xhat, w.gamma[j], w.beta[j]), d[j]);
        s1[j] += dz; s2[j] = fmaf(dz, xhat, s2[j]);
      }
    }
  float* part = a.part + (int64_t)b * a.C + slice * a.sv * VE;
  channel_sums<NT, VE>(s1, t.sv, t.rows, s_red, s_c[0], part);
  channel_sums<NT, VE>(s2, t.sv, t.rows, s_red, s_c[1], part + (int64_t)a.B * a.C);
  __syncthreads();
  if (t.count == 0) return;
  const float n = (float)a.P * (float)a.Cg;
  const int c_slice = slice * a.sv * VE;
  float c1[VE], c2[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int first = (t.c + j) / a.Cg * a.Cg;
    if (j > 0 && (t.c + j) % a.Cg) { c1[j] = c1[j - 1]; c2[j] = c2[j - 1]; continue; }
    float u1 = 0.0f, u2 = 0.0f;
    for (int c = first; c < first + a.Cg; ++c) {
      const float gamma = a.gamma ? a.gamma[c] : 1.0f;
      u1 = fmaf(gamma, s_c[0][c - c_slice], u1); u2 = fmaf(gamma, s_c[1][c - c_slice], u2);
    }
    c1[j] = u1 / n; c2[j] = u2 / n;
  }
  typename Tl::V* dx = reinterpret_cast<typename Tl::V*>(a.out) + t.at;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (i < t.count) {
      unpack(vx[i], f);
      unpack(vd[i], d);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float xhat = gn_xhat(f[j], mean[j], rstd[j]);
        const float dz = act_grad<T, ACT>(gn_z(xhat, w.gamma[j], w.beta[j]), d[j]);
        f[j] = rstd[j] * ((dz * w.gamma[j] - c1[j]) - xhat * c2[j]);
      }
      pack(f, dx + i * t.step);
    }
}

// ---- split -------------------------------------------------------------------------------------------------------------
// Workgroup: image, range of `chunk` pixels, block of vectors of channels; the threads of one vector take pixels in turn.
constexpr int kT = 256;
constexpr int kHeld = 8;          // pixels a thread of the forward statistics holds: chunk = kHeld * rows

template <typename T, int VE> struct Range {
  typedef typename Vec<T, VE>::type V;
  int sv, rows, tx, ty, c, p0, p1;           // p0: own first pixel; p1: end of the range
  int64_t base;                              // vectors of the image's first pixel, own channels
  int b, chunk;
  __device__ __forceinline__ Range(const GnArgs& a) {
    const int per = a.chunks * a.slices;
    b = blockIdx.x / per;
    const int rest = blockIdx.x - b * per, slice = rest / a.chunks;
    chunk = rest - slice * a.chunks;
    b += a.b0;
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

// Sums of VE values over the threads of a vector; result in the threads with ty = 0.
template <int VE> __device__ __forceinline__ void range_sums(float (&v)[VE], int sv, int rows, int tx, int ty, float* s_red) {
  __syncthreads();
#pragma unroll
  for (int j = 0; j < VE; ++j) s_red[j * kT + threadIdx.x] = v[j];
  __syncthreads();
  if (ty == 0) {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      float s = 0.0f;
      for (int r = 0; r < rows; ++r) s += s_red[j * kT + r * sv + tx];
      v[j] = s;
    }
  }
}

// Every channel's mean and sum of squared deviations within the range: part[(b, chunk)][0..1][c].
template <typename T, int VE>
__global__ __launch_bounds__(kT) void gn_stats_kernel(GnArgs a) {
  __shared__ float s_red[VE * kT], s_mean[VE * kT];
  const Range<T, VE> r(a);
  const typename Range<T, VE>::V* x = reinterpret_cast<const typename Range<T, VE>::V*>(a.x) + r.base;
  typename Range<T, VE>::V v[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) v[i] = x[(int64_t)min(r.p0 + i * r.rows, a.P - 1) * a.nv];
  float acc[VE], f[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) acc[j] = 0.0f;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (r.p0 + i * r.rows < r.p1) {
      unpack(v[i], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) acc[j] += f[j];
    }
  range_sums<VE>(acc, r.sv, r.rows, r.tx, r.ty, s_red);
  const float n = (float)(r.p1 - r.chunk * a.chunk);
  if (r.ty == 0) {
#pragma unroll
    for (int j = 0; j < VE; ++j) { acc[j] = __fdiv_rn(acc[j], n); s_mean[j * kT + r.tx] = acc[j]; }
  }
  __syncthreads();
  float mean[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) { mean[j] = s_mean[j * kT + r.tx]; acc[j] = 0.0f; }
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (r.p0 + i * r.rows < r.p1) {
      unpack(v[i], f);
#pragma unroll
      for (int j = 0; j < VE; ++j) { const float d = f[j] - mean[j]; acc[j] = fmaf(d, d, acc[j]); }
    }
  range_sums<VE>(acc, r.sv, r.rows, r.tx, r.ty, s_red);
  if (r.ty == 0) {
    float* part = a.part + ((int64_t)(r.b - a.b0) * a.chunks + r.chunk) * 2 * a.C + r.c;
#pragma unroll
    for (int j = 0; j < VE; ++j) { part[j] = mean[j]; part[a.C + j] = acc[j]; }
  }
}

// One wavefront per image and group: means and squared deviations of its ranges and channels into one, by the deviations of the
// means from their own mean.
__global__ __launch_bounds__(64) void gn_join_stats_kernel(GnArgs a) {
  const int b = blockIdx.x / a.G, g = blockIdx.x - b * a.G, entries = a.chunks * a.Cg;
  const float* part = a.part + (int64_t)b * a.chunks * 2 * a.C + g * a.Cg;
  const float n = (float)a.P * (float)a.Cg;
  float s = 0.0f;
  for (int e = threadIdx.x; e < entries; e += 64) {
    const int k = e / a.Cg, c = e - k * a.Cg;
    s = fmaf((float)(min(a.P, (k + 1) * a.chunk) - k * a.chunk), part[(int64_t)k * 2 * a.C + c], s);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
  const float mean = __fdiv_rn(s, n);
  s = 0.0f;
  for (int e = threadIdx.x; e < entries; e += 64) {
    const int k = e / a.Cg, c = e - k * a.Cg;
    const float* q = part + (int64_t)k * 2 * a.C + c;
    const float d = q[0] - mean;
    s += fmaf((float)(min(a.P, (k + 1) * a.chunk) - k * a.chunk) * d, d, q[a.C]);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
  if (threadIdx.x == 0) {
    a.mean[(int64_t)(a.b0 + b) * a.G + g] = mean;
    a.rstd[(int64_t)(a.b0 + b) * a.G + g] = rstd_of(s, n, a.eps);
  }
}

template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_apply_kernel(GnArgs a) {
  const Range<T, VE> r(a);
  if (r.p0 >= r.p1) return;
  typedef typename Range<T, VE>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  V* y = reinterpret_cast<V*>(a.out) + r.base;
  const Affine<VE> w(a, r.c);
  float mean[VE], rstd[VE], f[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean[g]; rstd[j] = a.rstd[g];
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack(x[(int64_t)p * a.nv], f);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = act_of<T, ACT>(gn_z(gn_xhat(f[j], mean[j], rstd[j]), w.gamma[j], w.beta[j]));
    pack(f, y + (int64_t)p * a.nv);
  }
}

// Sums of dz and dz xhat of every channel within the range: part[(b, chunk)][0..1][c].
template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_grad_sums_kernel(GnArgs a) {
  __shared__ float s_red[VE * kT];
  const Range<T, VE> r(a);
  typedef typename Range<T, VE>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  const V* dy = reinterpret_cast<const V*>(a.dy) + r.base;
  const Affine<VE> w(a, r.c);
  float mean[VE], rstd[VE], s1[VE], s2[VE], f[VE], d[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean_in[g]; rstd[j] = a.rstd_in[g];
    s1[j] = s2[j] = 0.0f;
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack(x[(int64_t)p * a.nv], f);
    unpack(dy[(int64_t)p * a.nv], d);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float xhat = gn_xhat(f[j], mean[j], rstd[j]);
      const float dz = act_grad<T, ACT>(gn_z(xhat, w.gamma[j], w.beta[j]), d[j]);
      s1[j] += dz; s2[j] = fmaf(dz, xhat, s2[j]);
    }
  }
  range_sums<VE>(s1, r.sv, r.rows, r.tx, r.ty, s_red);
  range_sums<VE>(s2, r.sv, r.rows, r.tx, r.ty, s_red);
  if (r.ty == 0) {
    float* part = a.part + ((int64_t)r.b * a.chunks + r.chunk) * 2 * a.C + r.c;
#pragma unroll
    for (int j = 0; j < VE; ++j) { part[j] = s1[j]; part[a.C + j] = s2[j]; }
  }
}

// One wavefront per image and group: the two means of the group, to join[(b, g)][0..1].
__global__ __launch_bounds__(64) void gn_join_grad_kernel(GnArgs a, float* join) {
  const int b = a.b0 + blockIdx.x / a.G, g = blockIdx.x % a.G, entries = a.chunks * a.Cg;
  const float* part = a.part + (int64_t)b * a.chunks * 2 * a.C + g * a.Cg;
  float c1 = 0.0f, c2 = 0.0f;
  for (int e = threadIdx.x; e < entries; e += 64) {
    const int k = e / a.Cg, c = e - k * a.Cg;
    const float gamma = a.gamma ? a.gamma[g * a.Cg + c] : 1.0f;
    const float* q = part + (int64_t)k * 2 * a.C + c;
    c1 = fmaf(gamma, q[0], c1); c2 = fmaf(gamma, q[a.C], c2);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) { c1 += __shfl_xor(c1, d); c2 += __shfl_xor(c2, d); }
  const float n = (float)a.P * (float)a.Cg;
  if (threadIdx.x == 0) { join[((int64_t)b * a.G + g) * 2] = c1 / n; join[((int64_t)b * a.G + g) * 2 + 1] = c2 / n; }
}

template <typename T, int VE, int ACT>
__global__ __launch_bounds__(kT) void gn_grad_apply_kernel(GnArgs a, const float* join) {
  const Range<T, VE> r(a);
  if (r.p0 >= r.p1) return;
  typedef typename Range<T, VE>::V V;
  const V* x = reinterpret_cast<const V*>(a.x) + r.base;
  const V* dy = reinterpret_cast<const V*>(a.dy) + r.base;
  V* dx = reinterpret_cast<V*>(a.out) + r.base;
  const Affine<VE> w(a, r.c);
  float mean[VE], rstd[VE], c1[VE], c2[VE], f[VE], d[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int64_t g = (int64_t)r.b * a.G + (r.c + j) / a.Cg;
    mean[j] = a.mean_in[g]; rstd[j] = a.rstd_in[g]; c1[j] = join[2 * g]; c2[j] = join[2 * g + 1];
  }
#pragma unroll 4
  for (int p = r.p0; p < r.p1; p += r.rows) {
    unpack(x[(int64_t)p * a.nv], f);
    unpack(dy[(int64_t)p * a.nv], d);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float xhat = gn_xhat(f[j], mean[j], rstd[j]);
      const float dz = act_grad<T, ACT>(gn_z(xhat, w.gamma[j], w.beta[j]), d[j]);
      f[j] = rstd[j] * ((dz * w.gamma[j] - c1[j]) - xhat * c2[j]);
    }
    pack(f, dx + (int64_t)p * a.nv);
  }
}

// dbeta[c] = sum of part[k][c], dgamma[c] = sum of part[k][second + c] over k < n, `stride` floats apart.
constexpr int kParamRows = 16;
__global__ __launch_bounds__(64 * kParamRows) void gn_param_kernel(const float* part, int n, int64_t stride, int64_t second, int C,
                                                                   float* dgamma, float* dbeta) {
  __shared__ float s[2][kParamRows][64];
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s1 = 0.0f, s2 = 0.0f;
  if (c < C)
    for (int k = row; k < n; k += kParamRows) { s1 += part[k * stride + c]; s2 += part[k * stride + second + c]; }
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
  int batch;           // split: images at a time
};

constexpr int64_t kCacheBytes = 128ll << 20;   // of the 256 MiB last-level cache, for the tensors of a batch

Plan plan_of(bool backward, dat_dtype dtype, bool vectors, int B, int P, int C, int G) {
  Plan p{};
  const int width = dtype == DAT_BF16 ? 2 : 4, whole = 16 / width, Cg = C / G;
  p.ve = vectors && C % whole == 0 ? whole : 1;
  p.nv = C / p.ve;
  if (p.ve > 1) {
    const int unit = Cg / gcd(Cg, whole);              // vectors of the smallest slice of whole groups
    static const int sizes[][2] = {{256, 2}, {256, 8}, {512, 8}, {1024, 8}, {1024, 16}};
    const int most = backward ? 4 : 5;
    // rows of 128 bytes if they fit, else 64; narrower where there would be few workgroups
    for (int want = 8; want >= 4 && !p.nt; want >>= 1) {
      int sv = unit * ((want + unit - 1) / unit);
      while (sv > unit && (int64_t)B * ((p.nv + sv - 1) / sv) < 512) sv = sv / 2 / unit * unit >= unit ? sv / 2 / unit * unit : unit;
      if (sv > p.nv) sv = p.nv;
      if (sv * whole / Cg > kMaxSliceGroups) break;
      for (int i = 0; i < most; ++i) {
        const int nt = sizes[i][0], vpt = sizes[i][1];
        if (sv <= nt && (P + nt / sv - 1) / (nt / sv) <= vpt) { p.sv = sv; p.nt = nt; p.vpt = vpt; break; }
      }
    }
    if (p.nt) { p.slices = (p.nv + p.sv - 1) / p.sv; return p; }
  }
  p.slices = (p.nv + 31) / 32;                          // at most 32 vectors wide: at least 64 pixels to a range
  p.sv = (p.nv + p.slices - 1) / p.slices;
  p.slices = (p.nv + p.sv - 1) / p.sv;
  p.chunk = kHeld * (kT / p.sv);
  p.chunks = (P + p.chunk - 1) / p.chunk;
  const int64_t image = (int64_t)P * C * width * (backward ? 2 : 1);
  p.batch = (int)(kCacheBytes / image < 1 ? 1 : kCacheBytes / image > B ? B : kCacheBytes / image);
  if (p.batch < 1) p.batch = 1;
  return p;
}

dat_status check(dat_dtype dtype, int B, int H, int W, int C, int groups) {
  if ((dtype != DAT_F32 && dtype != DAT_BF16) || B < 0 || H < 1 || W < 1 || C < 1 || groups < 1 || C % groups) return DAT_ERR_ARG;
  constexpr int64_t most = 1 << 30;
  if ((int64_t)H * W > most || (int64_t)H * W * C > most || (int64_t)B * C > most) return DAT_ERR_SHAPE;
  return DAT_OK;
}

size_t workspace_of(const Plan& p, bool backward, int B, int C, int G) {
  if (backward) return p.nt ? (size_t)B * C * 8 : ((size_t)B * p.chunks * C + (size_t)B * G) * 8;
  return p.nt ? 0 : (size_t)p.batch * p.chunks * C * 8;
}

#define DAT_GN_ACT(act, ...)                                                              \
  do {                                                                                    \
    if (act == DAT_ACT_RELU) { constexpr int ACT = DAT_ACT_RELU; __VA_ARGS__; }           \
    else if (act == DAT_ACT_SILU) { constexpr int ACT = DAT_ACT_SILU; __VA_ARGS__; }      \
    else { constexpr int ACT = DAT_ACT_NONE; __VA_ARGS__; }                               \
  } while (0)

template <typename T, bool WHOLE> void launch_forward_resident(const Plan& p, const GnArgs& a, dat_act act, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.slices));
#define DAT_GN_SIZE(NT, VPT) if (p.nt == NT && p.vpt == VPT) DAT_GN_ACT(act, hipLaunchKernelGGL((gn_forward_resident_kernel<T, ACT, WHOLE, NT, VPT>), grid, dim3(NT), 0, st, a))
  DAT_GN_SIZE(256, 2); DAT_GN_SIZE(256, 8); DAT_GN_SIZE(512, 8); DAT_GN_SIZE(1024, 8); DAT_GN_SIZE(1024, 16);
#undef DAT_GN_SIZE
}
template <typename T> void launch_backward_resident(const Plan& p, const GnArgs& a, dat_act act, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.slices));
#define DAT_GN_SIZE(NT, VPT) if (p.nt == NT && p.vpt == VPT) DAT_GN_ACT(act, hipLaunchKernelGGL((gn_backward_resident_kernel<T, ACT, NT, VPT>), grid, dim3(NT), 0, st, a))
  DAT_GN_SIZE(256, 2); DAT_GN_SIZE(256, 8); DAT_GN_SIZE(512, 8); DAT_GN_SIZE(1024, 8);
#undef DAT_GN_SIZE
}
template <typename T, int VE> void launch_forward_split(const GnArgs& a, int images, dat_act act, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)images * a.chunks * a.slices));
  hipLaunchKernelGGL((gn_stats_kernel<T, VE>), grid, dim3(kT), 0, st, a);
  hipLaunchKernelGGL(gn_join_stats_kernel, dim3((unsigned)((int64_t)images * a.G)), dim3(64), 0, st, a);
  DAT_GN_ACT(act, hipLaunchKernelGGL((gn_apply_kernel<T, VE, ACT>), grid, dim3(kT), 0, st, a));
}
template <typename T, int VE> void launch_backward_split(const GnArgs& a, int images, dat_act act, float* join, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)images * a.chunks * a.slices));
  DAT_GN_ACT(act, hipLaunchKernelGGL((gn_grad_sums_kernel<T, VE, ACT>), grid, dim3(kT), 0, st, a));
  hipLaunchKernelGGL(gn_join_grad_kernel, dim3((unsigned)((int64_t)images * a.G)), dim3(64), 0, st, a, join);
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
  if (B == 0) return DAT_OK;
  const Plan p = plan_of(false, dtype, aligned(x, 16) && aligned(y, 16), B, H * W, C, groups);
  GnArgs a{x, nullptr, gamma, beta, nullptr, nullptr, y, mean, rstd, (float*)workspace, B, H * W, C, groups, C / groups,
           p.nv, p.sv, p.slices, p.chunk, p.chunks, 0, eps};
  if ((int64_t)(p.nt ? B : p.batch) * p.slices * (p.nt ? 1 : p.chunks) > INT32_MAX) return DAT_ERR_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  if (p.nt) {
    const bool whole = a.Cg % p.ve == 0;
    if (dtype == DAT_BF16) { if (whole) launch_forward_resident<bf16_t, true>(p, a, act, st); else launch_forward_resident<bf16_t, false>(p, a, act, st); }
    else { if (whole) launch_forward_resident<float, true>(p, a, act, st); else launch_forward_resident<float, false>(p, a, act, st); }
    DAT_LAUNCH_CHECK();
    return DAT_OK;
  }
  for (a.b0 = 0; a.b0 < B; a.b0 += p.batch) {
    const int images = B - a.b0 < p.batch ? B - a.b0 : p.batch;
    if (dtype == DAT_BF16) { if (p.ve > 1) launch_forward_split<bf16_t, 8>(a, images, act, st); else launch_forward_split<bf16_t, 1>(a, images, act, st); }
    else { if (p.ve > 1) launch_forward_split<float, 4>(a, images, act, st); else launch_forward_split<float, 1>(a, images, act, st); }
    DAT_LAUNCH_CHECK();
  }
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
  hipStream_t st = (hipStream_t)stream;
  const Plan p = plan_of(true, dtype, aligned(x, 16) && aligned(dy, 16) && aligned(dx, 16), B, H * W, C, groups);
  GnArgs a{x, dy, gamma, beta, mean, rstd, dx, nullptr, nullptr, (float*)workspace, B, H * W, C, groups, C / groups,
           p.nv, p.sv, p.slices, p.chunk, p.chunks, 0, 0.0f};
  if ((int64_t)(p.nt ? B : p.batch) * p.slices * (p.nt ? 1 : p.chunks) > INT32_MAX) return DAT_ERR_SHAPE;
  if (p.nt && B > 0) {
    if (dtype == DAT_BF16) launch_backward_resident<bf16_t>(p, a, act, st); else launch_backward_resident<float>(p, a, act, st);
    DAT_LAUNCH_CHECK();
  } else if (B > 0) {
    float* join = a.part + (int64_t)B * p.chunks * 2 * C;
    for (a.b0 = 0; a.b0 < B; a.b0 += p.batch) {
      const int images = B - a.b0 < p.batch ? B - a.b0 : p.batch;
      if (dtype == DAT_BF16) { if (p.ve > 1) launch_backward_split<bf16_t, 8>(a, images, act, join, st); else launch_backward_split<bf16_t, 1>(a, images, act, join, st); }
      else { if (p.ve > 1) launch_backward_split<float, 4>(a, images, act, join, st); else launch_backward_split<float, 1>(a, images, act, join, st); }
      DAT_LAUNCH_CHECK();
    }
  }
  if (dgamma) {
    const int n = p.nt ? B : B * p.chunks;
    hipLaunchKernelGGL(gn_param_kernel, dim3((C + 63) / 64), dim3(64 * kParamRows), 0, st, (const float*)workspace, B == 0 ? 0 : n,
                       (int64_t)(p.nt ? C : 2 * C), p.nt ? (int64_t)B * C : (int64_t)C, C, dgamma, dbeta);
    DAT_LAUNCH_CHECK();
  }
  return DAT_OK;
}
