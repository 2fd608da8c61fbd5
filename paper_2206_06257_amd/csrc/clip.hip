// The norm of many gradient tensors together, and all of them scaled down to a largest norm.
//
//   norm = sqrt(sum g^2),  c = largest / norm where norm > largest, else 1;  g <- g c.
//
// Squares are formed and added in 64 bits: exact products, no overflow, and no loss however many elements there are; beside the memory
// that costs nothing.  Bound by HBM: one read and, where c < 1, one more read and a write.  Tensors are cut into blocks of kBlock elements; block j
// of tensor t has the slot off[t] / kBlock + t + j (strictly increasing in (t, j)), and a workgroup takes a range of slots, in the
// second pass from its end, which is what the last-level cache still holds.
// Measured: 236 M elements, bf16 matrices and fp32 vectors (472 MB), 292 us where they are scaled: 91 to 106 us for the sum (4.5 to 5.2 TB/s, part of it
// from the cache), 154 us for the scaling (945 MB at 6.1 TB/s).
#include "kernels.h"
#include "tensor_table.h"

namespace dat {
namespace {

constexpr int kThreads = 256, kBlock = 8192;
constexpr int kMaxParts = 2048;                    // workgroups of a pass: 8 a compute unit
constexpr int kAloneThreads = 1024;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
struct __attribute__((packed, aligned(4))) Vec4 { uint32_t w[4]; };      // 16 bytes from an address that is aligned to an element only
struct __attribute__((packed, aligned(2))) Vec2 { uint32_t w[4]; };

struct ClipArgs {
  const uint64_t* pointers; const uint8_t* types; const int64_t* off;
  int T, slots, per;                               // slots of a workgroup
  float largest;
  double* parts; float* norm;
};

__device__ __forceinline__ int64_t first_slot(const int64_t* off, int t) { return off[t] / kBlock + t; }
__device__ __forceinline__ int tensor_of_slot(const int64_t* off, int T, int64_t slot) {
  int lo = 0, hi = T;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_slot(off, mid) <= slot) lo = mid; else hi = mid;
  }
  return lo;
}

// The elements of a slot: their address, type and number (0: none).
struct Block { char* p; bool half; int n; };
__device__ __forceinline__ Block block_of(const ClipArgs& a, int slot, int t) {
  const int64_t e = (slot - first_slot(a.off, t)) * kBlock, left = a.off[t + 1] - a.off[t] - e;
  Block b;
  b.half = a.types[t] == DAT_BF16;
  b.p = reinterpret_cast<char*>(a.pointers[t]) + e * (b.half ? 2 : 4);
  b.n = (int)max((int64_t)0, min((int64_t)kBlock, left));
  return b;
}

// c as a product of two factors, the second 1 but where c is too small for fp32 (gradients far beyond its square root's range); a norm that
// is NaN makes everything NaN, an infinite one zero (and what is infinite NaN).
struct Factor { float c, rest; };
__device__ __forceinline__ Factor factor(double norm, float largest) {
  const double c = norm <= (double)largest ? 1.0 : (double)largest / norm;
  return c < 0x1p-100 && c > 0.0 ? Factor{(float)(c * 0x1p120), 0x1p-120f} : Factor{(float)c, 1.0f};
}

__device__ __forceinline__ void add_squares(const uint32_t (&w)[4], bool half, double& sum) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (half) {
      const double x = (double)__uint_as_float(w[i] << 16), y = (double)__uint_as_float(w[i] & 0xffff0000u);
      sum = fma(x, x, sum);
      sum = fma(y, y, sum);
    } else {
      const double x = (double)__uint_as_float(w[i]);
      sum = fma(x, x, sum);
    }
  }
}
__device__ __forceinline__ void scale(uint32_t (&w)[4], bool half, const Factor& f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (half) w[i] = f2bf_pack(__uint_as_float(w[i] << 16) * f.c * f.rest, __uint_as_float(w[i] & 0xffff0000u) * f.c * f.rest);
    else w[i] = __float_as_uint(__uint_as_float(w[i]) * f.c * f.rest);
  }
}

// A type's passes over a block by LANES threads, this one being the `at`-th: whole vectors, then the elements behind the last one.
template <typename V, bool HALF, int LANES> __device__ __forceinline__ void squares_of(const Block& b, int at, double& sum) {
  constexpr int E = HALF ? 8 : 4, N = kBlock / E / LANES;
  const V* const v = reinterpret_cast<const V*>(b.p);
  if (N <= 8 && b.n == kBlock) {
    V x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = v[at + i * LANES];
#pragma unroll
    for (int i = 0; i < N; ++i) add_squares(x[i].w, HALF, sum);
  } else {
    const int whole = b.n / E;
    for (int i = at; i < whole; i += LANES) { const V x = v[i]; add_squares(x.w, HALF, sum); }
    const int e = whole * E + at;
    if (e < b.n) {
      double x;
      if constexpr (HALF) x = (double)bf2f(reinterpret_cast<const bf16_t*>(b.p)[e]); else x = (double)reinterpret_cast<const float*>(b.p)[e];
      sum = fma(x, x, sum);
    }
  }
}
template <typename V, bool HALF, int LANES> __device__ __forceinline__ void scale_block(const Block& b, int at, const Factor& f) {
  constexpr int E = HALF ? 8 : 4, N = kBlock / E / LANES;
  V* const v = reinterpret_cast<V*>(b.p);
  if (N <= 8 && b.n == kBlock) {
    V x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = v[at + i * LANES];
#pragma unroll
    for (int i = 0; i < N; ++i) { scale(x[i].w, HALF, f); v[at + i * LANES] = x[i]; }
  } else {
    const int whole = b.n / E;
    for (int i = at; i < whole; i += LANES) { V x = v[i]; scale(x.w, HALF, f); v[i] = x; }
    const int e = whole * E + at;
    if (e < b.n) {
      if constexpr (HALF) { bf16_t* const p = reinterpret_cast<bf16_t*>(b.p) + e; *p = f2bf(bf2f(*p) * f.c * f.rest); }
      else { float* const p = reinterpret_cast<float*>(b.p) + e; *p = *p * f.c * f.rest; }
    }
  }
}

// Sum over the workgroup in a fixed order, in every thread.
template <int THREADS> __device__ __forceinline__ double workgroup_sum(double x, double* s) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) x += s[w];
  return x;
}
template <typename F> __device__ __forceinline__ void each_block(const ClipArgs& a, int first, int last, int step, bool backwards, F f) {
  if (first >= last) return;
  int t = tensor_of_slot(a.off, a.T, backwards ? last - 1 : first);
  for (int i = first; i < last; i += step) {
    const int slot = backwards ? last - 1 - (i - first) : i;
    if (backwards) { while (t > 0 && first_slot(a.off, t) > slot) --t; }
    else { while (t + 1 < a.T && first_slot(a.off, t + 1) <= slot) ++t; }
    f(block_of(a, slot, t));
  }
}

// pass 0: partial sums of squares; 1: norm from them, and the scaling; 2: both, by a single workgroup whose waves take a slot each.
template <int PASS> __global__ __launch_bounds__(PASS == 2 ? kAloneThreads : kThreads) void clip_kernel(ClipArgs a, int parts, int write) {
  constexpr int THREADS = PASS == 2 ? kAloneThreads : kThreads, LANES = PASS == 2 ? 64 : kThreads, STEP = THREADS / LANES;
  __shared__ double s[THREADS / 64];
  const int at = threadIdx.x % LANES;
  const int start = min((int)blockIdx.x * a.per, a.slots), last = min(start + a.per, a.slots), first = PASS == 2 ? start + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : start;
  double sum = 0.0;
  if (PASS != 1) {
    each_block(a, first, last, STEP, false, [&](const Block& b) { if (b.half) squares_of<Vec2, true, LANES>(b, at, sum); else squares_of<Vec4, false, LANES>(b, at, sum); });
    sum = workgroup_sum<THREADS>(sum, s);
    if (PASS == 0) {
      if (threadIdx.x == 0) a.parts[blockIdx.x] = sum;
      return;
    }
  } else {
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += a.parts[i];
    sum = workgroup_sum<THREADS>(sum, s);
  }
  const double norm = sqrt(sum);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)norm;
  const Factor f = factor(norm, a.largest);
  if (!write || f.c == 1.0f) return;
  each_block(a, first, last, STEP, PASS == 1, [&](const Block& b) { if (b.half) scale_block<Vec2, true, LANES>(b, at, f); else scale_block<Vec4, false, LANES>(b, at, f); });
}

int64_t slots_of(int64_t total, int T) { return total / kBlock + T; }
int parts_of(int64_t slots) { return (int)(slots < kMaxParts ? slots : kMaxParts); }

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" size_t dat_clip_gradients_workspace(int num_tensors, int64_t total) {
  if (num_tensors < 1 || total < 0 || slots_of(total, num_tensors) > INT32_MAX) return 0;
  return (size_t)parts_of(slots_of(total, num_tensors)) * 8;
}

extern "C" dat_status dat_clip_gradients(const uint64_t* pointers_dev, const uint8_t* types_dev, const int64_t* offsets_dev, int num_tensors, int64_t total,
                                         float largest, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (num_tensors < 1 || total < 0 || !(largest >= 0.0f)) return DAT_ERR_ARG;
  if (!pointers_dev || !types_dev || !offsets_dev || !norm || !aligned(pointers_dev, 8) || !aligned(offsets_dev, 8) || !aligned(norm, 4)) return DAT_ERR_ARG;
  const int64_t slots = slots_of(total, num_tensors);
  if (slots > INT32_MAX) return DAT_ERR_SHAPE;
  if (!workspace || !aligned(workspace, 8) || workspace_bytes < dat_clip_gradients_workspace(num_tensors, total)) return DAT_ERR_ARG;
  const hipStream_t st = (hipStream_t)stream;
  ClipArgs a{pointers_dev, types_dev, offsets_dev, num_tensors, (int)slots, 0, largest, (double*)workspace, norm};
  const int write = largest < __builtin_inff();
  // Few small tensors: one launch of one workgroup, a slot to each of its waves (12 tensors of 170 to 2700 elements 8.5 to 9.1 us with the host's
  // part, two launches 11.5; 4 tensors of 8000 12.7 against 11.4, 16 of 1000 in 17 slots 11.4 against 11.6).
  if (slots <= kAloneThreads / 64 && total <= (int64_t)num_tensors * (kBlock / 2)) {
    a.per = (int)slots;
    hipLaunchKernelGGL(clip_kernel<2>, dim3(1), dim3(kAloneThreads), 0, st, a, 0, write);
    DAT_LAUNCH_CHECK();
    return DAT_OK;
  }
  int parts = parts_of(slots);
  a.per = (int)((slots + parts - 1) / parts);
  parts = (int)((slots + a.per - 1) / a.per);
  hipLaunchKernelGGL(clip_kernel<0>, dim3(parts), dim3(kThreads), 0, st, a, 0, 0);
  DAT_LAUNCH_CHECK();
  hipLaunchKernelGGL(clip_kernel<1>, dim3(write ? parts : 1), dim3(kThreads), 0, st, a, parts, write);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}
