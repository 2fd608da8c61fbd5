// AdamW over a tensor table, moments in 32 or in 8 bits (the format is described in dat.h).
//
// Both widths walk the same slots: block j of 256 elements of tensor t has the slot off[t]/256 + t + j, strictly increasing in
// (t, j) because floor((a+n)/256) + 1 >= floor(a/256) + ceil(n/256); a wavefront takes a slot, a lane four consecutive elements.
// Streaming, bound by HBM: 28 bytes an element with 32-bit moments, 16 with 8-bit ones (+2 for the bf16 copy).  46.2 M parameters
// with the copy, 32 bits: 270 us = 5.1 TB/s; 25.6 M, 8 bits: 98 us = 4.7 TB/s (beside the memory 117 vector instructions an
// element, 77 % of the cycles: IEEE square root and quotient, a quarter of a Philox block).  One block a wavefront: four behind one search of the
// table take 129 and 340 us.
#include "kernels.h"
#include "tensor_table.h"
#include "philox.h"
#include "lanes.h"

namespace dat {
namespace {

constexpr int kT = 256, kWaves = kT / 64;
constexpr int kBlock = 256;                  // elements of a block: four per lane
constexpr uint32_t kRandomStream = 2;        // Philox stream (0: the quantizer, 1: the random start)
constexpr int kTopM = 127, kTopV = 255;      // codes of the largest magnitude

struct AdamwArgs {
  float* theta; const void* g; void* m; void* v; int16_t* scales;
  const int64_t* off; const float* decay; bf16_t* copy;
  int T; int slots; uint64_t seed;
  AdamwParams hp;
};

// Four elements from an address that is aligned to one of them only: global memory takes such vector accesses whole.
struct __attribute__((packed, aligned(4))) Float4U { float x[4]; };
struct __attribute__((packed, aligned(2))) Half4U { bf16_t x[4]; };
struct __attribute__((packed, aligned(1))) Byte4U { uint8_t x[4]; };

template <typename V, typename E> __device__ __forceinline__ void load4(const E* p, int count, E (&x)[4]) {
  if (count >= 4) {
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v.x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < count ? p[i] : E(0);
  }
}
template <typename V, typename E> __device__ __forceinline__ void store4(E* p, const E (&x)[4], int count) {
  if (count >= 4) {
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.x[i] = x[i];
    *reinterpret_cast<V*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < count) p[i] = x[i];
  }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return (uint32_t)lanes_reduce<64>((int)x, [](int a, int b) { return (int)max((uint32_t)a, (uint32_t)b); });
}

// s of a block: one above T(largest), so that rounding up stays in range; -1 where a value is not finite.
__device__ __forceinline__ int block_scale(uint32_t largest) { return largest >= 0x7f800000u ? -1 : (int)(largest >> 20) + 1; }

__device__ __forceinline__ float decode(int code, int s, int top) {
  const int t = code + s - top;
  const float x = __uint_as_float(code > 0 && t > 0 ? (uint32_t)t << 20 : 0u);
  return s < 0 ? __builtin_nanf("") : x;
}
__device__ __forceinline__ float decode_m(uint8_t c, int s) { const float x = decode(c & 127, s, kTopM); return c & 128 ? -x : x; }
__device__ __forceinline__ float decode_v(uint8_t c, int s) { return decode(c, s, kTopV); }

// (bits + 16 r + 8) >> 20, less the block's s: the random number fills the bits that are cut off.
__device__ __forceinline__ int steps(uint32_t bits, uint32_t r, int s, int top) {
  return max(min((int)((bits + (r << 4) + 8u) >> 20), 0x7f7) - s + top, 0);
}
__device__ __forceinline__ uint8_t encode_m(float m, uint32_t r, int s) {
  return (uint8_t)(steps(abs_bits(m), r, s, kTopM) | (m < 0.0f ? 128 : 0));
}
__device__ __forceinline__ uint8_t encode_v(float v, uint32_t r, int s) {
  const uint32_t bits = abs_bits(v);
  return (uint8_t)(max(steps(bits, r, s, kTopV), bits ? 1 : 0));
}

__device__ __forceinline__ int64_t first_slot(const int64_t* off, int t) { return off[t] / kBlock + t; }

// Tensor of a slot: the largest t whose first slot is not above it.
__device__ __forceinline__ int tensor_of_slot(const int64_t* off, int T, int64_t slot) {
  int lo = 0, hi = T;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_slot(off, mid) <= slot) lo = mid; else hi = mid;
  }
  return lo;
}

// One block; WHOLE: all of its 256 elements are there, so that no load stands behind a branch, where the next would wait for it.
template <int BITS, bool WHOLE, typename G, typename GV>
__device__ __forceinline__ void adamw_block(const AdamwArgs& a, int slot, int t, int64_t e0, int64_t left, int lane) {
  const int64_t e = e0 + 4 * lane;
  const int count = WHOLE ? 4 : (int)max((int64_t)0, min((int64_t)4, left - 4 * lane));
  const AdamwParams& hp = a.hp;
  const float wd = a.decay ? __fmul_rn(hp.wd, a.decay[t]) : hp.wd;
  float th[4], m[4], v[4];
  G g4[4];
  load4<Float4U>(a.theta + e, count, th);
  load4<GV>((const G*)a.g + e, count, g4);
  if constexpr (BITS == 8) {
    const int sm = a.scales[2 * (int64_t)slot], sv = a.scales[2 * (int64_t)slot + 1];
    uint8_t cm[4], cv[4];
    load4<Byte4U>((const uint8_t*)a.m + e, count, cm);
    load4<Byte4U>((const uint8_t*)a.v + e, count, cv);
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = i < count ? decode_m(cm[i], sm) : 0.0f; v[i] = i < count ? decode_v(cv[i], sv) : 0.0f; }
  } else {
    load4<Float4U>((const float*)a.m + e, count, m);
    load4<Float4U>((const float*)a.v + e, count, v);
  }
  bf16_t half[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float g;
    if constexpr (sizeof(G) == 2) g = bf2f(g4[i]); else g = g4[i];
    m[i] = __fadd_rn(__fmul_rn(hp.b1, m[i]), __fmul_rn(hp.om1, g));
    v[i] = __fadd_rn(__fmul_rn(hp.b2, v[i]), __fmul_rn(hp.om2, __fmul_rn(g, g)));
    const float u = __fdiv_rn(__fmul_rn(m[i], hp.c1), __fadd_rn(sqrtf(__fmul_rn(v[i], hp.c2)), hp.eps));
    th[i] = __fsub_rn(th[i], __fmul_rn(hp.lr, __fadd_rn(u, __fmul_rn(wd, th[i]))));
    half[i] = f2bf(th[i]);
  }
  store4<Float4U>(a.theta + e, th, count);
  if (a.copy) store4<Half4U>(a.copy + e, half, count);
  if constexpr (BITS == 8) {
    uint32_t bm = 0, bv = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < count) { bm = max(bm, abs_bits(m[i])); bv = max(bv, abs_bits(v[i])); }
    const int sm = block_scale(wave_max(bm)), sv = block_scale(wave_max(bv));
    const PhiloxWords w = philox_block((uint64_t)slot * 64 + lane, a.seed, kRandomStream);
    const uint32_t word[4] = {w.w0, w.w1, w.w2, w.w3};
    uint8_t cm[4], cv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { cm[i] = encode_m(m[i], word[i] & 0xffffu, sm); cv[i] = encode_v(v[i], word[i] >> 16, sv); }
    store4<Byte4U>((uint8_t*)a.m + e, cm, count);
    store4<Byte4U>((uint8_t*)a.v + e, cv, count);
    if (lane == 0) { a.scales[2 * (int64_t)slot] = (int16_t)sm; a.scales[2 * (int64_t)slot + 1] = (int16_t)sv; }
  } else {
    store4<Float4U>((float*)a.m + e, m, count);
    store4<Float4U>((float*)a.v + e, v, count);
  }
}

template <int BITS, typename G, typename GV>
__global__ __launch_bounds__(kT) void adamw_kernel(AdamwArgs a) {
  const int lane = threadIdx.x & 63;
  const int slot = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6));
  if (slot >= a.slots) return;
  const int t = tensor_of_slot(a.off, a.T, slot);
  const int64_t e0 = a.off[t] + (slot - first_slot(a.off, t)) * kBlock;
  const int64_t left = a.off[t + 1] - e0;
  if (left >= kBlock) adamw_block<BITS, true, G, GV>(a, slot, t, e0, left, lane);
  else if (left > 0) adamw_block<BITS, false, G, GV>(a, slot, t, e0, left, lane);
}

template <bool WHOLE>
__device__ __forceinline__ void moments_block(const uint8_t* m, const uint8_t* v, const int16_t* scales, int slot, int64_t e0, int64_t left,
                                              int lane, float* m_out, float* v_out) {
  const int64_t e = e0 + 4 * lane;
  const int count = WHOLE ? 4 : (int)max((int64_t)0, min((int64_t)4, left - 4 * lane));
  const int sm = scales[2 * (int64_t)slot], sv = scales[2 * (int64_t)slot + 1];
  uint8_t cm[4], cv[4];
  float fm[4], fv[4];
  load4<Byte4U>(m + e, count, cm);
  load4<Byte4U>(v + e, count, cv);
#pragma unroll
  for (int i = 0; i < 4; ++i) { fm[i] = decode_m(cm[i], sm); fv[i] = decode_v(cv[i], sv); }
  store4<Float4U>(m_out + e, fm, count);
  store4<Float4U>(v_out + e, fv, count);
}

__global__ __launch_bounds__(kT) void adamw_moments_kernel(const uint8_t* __restrict__ m, const uint8_t* __restrict__ v,
                                                           const int16_t* __restrict__ scales, const int64_t* __restrict__ off,
                                                           int T, int slots, float* __restrict__ m_out, float* __restrict__ v_out) {
  const int lane = threadIdx.x & 63;
  const int slot = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6));
  if (slot >= slots) return;
  const int t = tensor_of_slot(off, T, slot);
  const int64_t e0 = off[t] + (slot - first_slot(off, t)) * kBlock;
  const int64_t left = off[t + 1] - e0;
  if (left >= kBlock) moments_block<true>(m, v, scales, slot, e0, left, lane, m_out, v_out);
  else if (left > 0) moments_block<false>(m, v, scales, slot, e0, left, lane, m_out, v_out);
}

inline int64_t blocks_for(int64_t slots) { return (slots + kWaves - 1) / kWaves; }

}  // namespace

bool adamw_params(float lr, float beta1, float beta2, float eps, float weight_decay, int t, AdamwParams* hp) {
  if (!(lr >= 0.0f) || !(eps >= 0.0f) || !(weight_decay >= 0.0f) || t < 1) return false;
  if (!(beta1 >= 0.0f && beta1 < 1.0f) || !(beta2 >= 0.0f && beta2 < 1.0f)) return false;
  hp->lr = lr; hp->b1 = beta1; hp->b2 = beta2; hp->eps = eps; hp->wd = weight_decay;
  hp->om1 = (float)(1.0 - (double)beta1); hp->om2 = (float)(1.0 - (double)beta2);
  hp->c1 = (float)(1.0 / (1.0 - pow((double)beta1, t))); hp->c2 = (float)(1.0 / (1.0 - pow((double)beta2, t)));
  return true;
}

dat_status launch_adamw(float* theta, const void* g, int g_dtype, const int64_t* off, int T, int64_t d, int bits, void* m, void* v,
                        int16_t* scales, uint64_t seed, const AdamwParams& hp, const float* decay, bf16_t* copy, hipStream_t st) {
  const int64_t slots = dat_adamw_slots(d, T);
  AdamwArgs a{theta, g, m, v, scales, off, decay, copy, T, (int)slots, seed, hp};
  const dim3 grid((unsigned)blocks_for(slots)), block(kT);
  if (bits == 8 && g_dtype == DAT_BF16) hipLaunchKernelGGL((adamw_kernel<8, bf16_t, Half4U>), grid, block, 0, st, a);
  else if (bits == 8) hipLaunchKernelGGL((adamw_kernel<8, float, Float4U>), grid, block, 0, st, a);
  else if (g_dtype == DAT_BF16) hipLaunchKernelGGL((adamw_kernel<32, bf16_t, Half4U>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((adamw_kernel<32, float, Float4U>), grid, block, 0, st, a);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

}  // namespace dat

using namespace dat;

extern "C" int64_t dat_adamw_slots(int64_t d, int num_tensors) { return d < 0 || num_tensors < 1 ? 0 : d / kBlock + num_tensors; }

extern "C" dat_status dat_adamw_update(float* theta, const void* grads, dat_dtype grad_dtype, const int64_t* offsets_dev,
                                       int num_tensors, int64_t d, int state_bits, void* m, void* v, int16_t* scales,
                                       uint64_t seed, float lr, float beta1, float beta2, float eps, float weight_decay,
                                       const float* decay, int t, uint16_t* theta_bf16, void* stream) {
  AdamwParams hp;
  if (num_tensors < 1 || d < 0) return DAT_ERR_ARG;
  if ((grad_dtype != DAT_F32 && grad_dtype != DAT_BF16) || (state_bits != 8 && state_bits != 32)) return DAT_ERR_ARG;
  if (!adamw_params(lr, beta1, beta2, eps, weight_decay, t, &hp)) return DAT_ERR_ARG;
  if (d == 0) return DAT_OK;
  if (!theta || !grads || !offsets_dev || !m || !v || (state_bits == 8 && !scales)) return DAT_ERR_ARG;
  if (!aligned(theta, 4) || !aligned(grads, grad_dtype == DAT_BF16 ? 2 : 4) || !aligned(offsets_dev, 8) || !aligned(scales, 2) ||
      !aligned(decay, 4) || !aligned(theta_bf16, 2) || (state_bits == 32 && (!aligned(m, 4) || !aligned(v, 4)))) return DAT_ERR_ARG;
  if (!fits_launch(blocks_for(dat_adamw_slots(d, num_tensors)), kT)) return DAT_ERR_ARG;
  if (decay) hp.wd = 1.0f;
  return launch_adamw(theta, grads, grad_dtype, offsets_dev, num_tensors, d, state_bits, m, v, scales, seed, hp, decay, theta_bf16,
                      (hipStream_t)stream);
}

extern "C" dat_status dat_adamw_moments(const uint8_t* m, const uint8_t* v, const int16_t* scales, const int64_t* offsets_dev,
                                        int num_tensors, int64_t d, float* m_out, float* v_out, void* stream) {
  if (num_tensors < 1 || d < 0) return DAT_ERR_ARG;
  if (d == 0) return DAT_OK;
  if (!m || !v || !scales || !offsets_dev || !m_out || !v_out) return DAT_ERR_ARG;
  if (!aligned(scales, 2) || !aligned(offsets_dev, 8) || !aligned(m_out, 4) || !aligned(v_out, 4)) return DAT_ERR_ARG;
  const int64_t slots = dat_adamw_slots(d, num_tensors);
  if (!fits_launch(blocks_for(slots), kT)) return DAT_ERR_ARG;
  hipLaunchKernelGGL(adamw_moments_kernel, dim3((unsigned)blocks_for(slots)), dim3(kT), 0, (hipStream_t)stream, m, v, scales, offsets_dev,
                     num_tensors, (int)slots, m_out, v_out);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}
