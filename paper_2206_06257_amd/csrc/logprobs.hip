// Log probabilities of given labels over rows of logits, with entropies and the largest alternatives, and the gradient.
//
// One pass with a running maximum M and the sums s = sum e^(x-M), w = sum (x-M) e^(x-M):  lse = M + log s,
// logp_y = (x_y - M) - log s,  H = log s - w / s.  Alternatives are ordered by one 64-bit key, the logit (as an ordered integer)
// above the complement of the index, so that equal logits go by ascending index and no two keys are equal.
#include "kernels.h"

namespace dat {
namespace {

constexpr float kInf = __builtin_inff();

template <typename T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f2bf(v); }

// Running softmax statistics.  bad: a NaN or +inf was met.  m = -inf: nothing allowed so far (s = w = 0).
struct Stats { float m, s, w; uint32_t bad; };

__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m);
  // (x - m_new) e^(x-m_new) = ((x - m_old) + d) e^(x-m_old) e^d, d = m_old - m_new; an empty side adds nothing
  const float da = a.m == m ? 0.0f : a.m - m, db = b.m == m ? 0.0f : b.m - m;
  const float ea = expf(da), eb = expf(db);
  const float wa = a.s > 0.0f && ea > 0.0f ? ea * fmaf(da, a.s, a.w) : 0.0f;
  const float wb = b.s > 0.0f && eb > 0.0f ? eb * fmaf(db, b.s, b.w) : 0.0f;
  return Stats{m, fmaf(a.s, ea, b.s * eb), wa + wb, a.bad | b.bad};
}
__device__ __forceinline__ void add(Stats& st, float x) {
  if (!(x < kInf)) { st.bad = 1; return; }
  if (x == -kInf) return;
  if (x > st.m) {
    const float d = st.m - x, e = expf(d);      // d = -inf at the first value: e = 0
    st.w = e > 0.0f ? e * fmaf(d, st.s, st.w) : 0.0f;
    st.s = fmaf(st.s, e, 1.0f);
    st.m = x;
  } else {
    const float d = x - st.m, e = expf(d);
    st.s += e;
    if (e > 0.0f) st.w = fmaf(d, e, st.w);
  }
}

// Ordered key of a logit: larger logit first, then the lower index.  0 is below every allowed logit's key.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x + 0.0f);                       // -0 counts as 0
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return x > -kInf ? ((uint64_t)o << 32) | (0xffffffffu - index) : 0;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int32_t key_index(uint64_t k) { return (int32_t)(0xffffffffu - (uint32_t)k); }

struct LogProbsArgs {
  const void* x; int64_t N, V, ld; const int32_t* labels; int top;
  float *logp, *entropy, *lse, *top_logp; int32_t* top_index;
};

template <int WAVES> __device__ Stats block_stats(Stats st, Stats* s_st) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1)
    st = merge(st, Stats{__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.w, d), (uint32_t)__shfl_xor((int)st.bad, d)});
  if ((threadIdx.x & 63) == 0) s_st[threadIdx.x >> 6] = st;
  __syncthreads();
  st = s_st[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) st = merge(st, s_st[i]);
  return st;
}
__device__ __forceinline__ uint64_t wave_max_key(uint64_t k) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) { const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)k, d); k = o > k ? o : k; }
  return k;
}

// The row's results, by one thread.
template <typename T> __device__ void write_stats(const LogProbsArgs& a, int64_t n, const Stats& st) {
  const bool empty = st.m == -kInf;
  const float ls = empty ? -kInf : logf(st.s), nan = __builtin_nanf("");
  if (a.lse) a.lse[n] = st.bad ? nan : empty ? -kInf : st.m + ls;
  if (a.entropy) a.entropy[n] = st.bad ? nan : empty ? 0.0f : fmaxf(ls - st.w / st.s, 0.0f);
  if (a.logp) {
    const int y = a.labels[n];
    const bool ok = (unsigned)y < (unsigned)a.V && !st.bad;
    a.logp[n] = !ok ? nan : empty ? -kInf : (load1((const T*)a.x + n * a.ld + y) - st.m) - ls;
  }
}
__device__ void write_top(const LogProbsArgs& a, int64_t n, int r, uint64_t key, const Stats& st) {
  const bool none = key == 0;
  a.top_index[n * a.top + r] = none || st.bad ? -1 : key_index(key);
  a.top_logp[n * a.top + r] = st.bad ? __builtin_nanf("") : none ? -kInf : (key_value(key) - st.m) - logf(st.s);
}

constexpr int kRowT = 256;
template <typename T>
__global__ __launch_bounds__(kRowT) void log_probs_row_kernel(LogProbsArgs a) {
  __shared__ Stats s_st[kRowT / 64];
  __shared__ uint64_t s_key[kRowT / 64];
  const int64_t n = blockIdx.x;
  const T* x = (const T*)a.x + n * a.ld;
  Stats st{-kInf, 0.0f, 0.0f, 0};
  for (int64_t i = threadIdx.x; i < a.V; i += kRowT) add(st, load1(x + i));
  st = block_stats<kRowT / 64>(st, s_st);
  if (threadIdx.x == 0) write_stats<T>(a, n, st);
  uint64_t below = ~0ull;
  for (int r = 0; r < a.top; ++r) {
    uint64_t best = 0;
    for (int64_t i = threadIdx.x; i < a.V; i += kRowT) {
      const uint64_t k = key_of(load1(x + i), (uint32_t)i);
      best = k < below && k > best ? k : best;
    }
    best = wave_max_key(best);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_key[threadIdx.x >> 6] = best;
    __syncthreads();
    best = s_key[0];
#pragma unroll
    for (int i = 1; i < kRowT / 64; ++i) best = s_key[i] > best ? s_key[i] : best;
    if (threadIdx.x == 0) write_top(a, n, r, best, st);
    below = best;
  }
}

struct LogProbsGradArgs {
  const void* x; int64_t N, V, ld, ldd; const int32_t* labels; const float *lse, *entropy, *dlogp, *dentropy; void* dx;
};

// One row's constants, and its gradient: a ([i = y] - p) - b p (log p + H).
struct RowGrad { float lse, a, b, H; int y; };
__device__ __forceinline__ RowGrad row_grad(const LogProbsGradArgs& g, int64_t n) {
  RowGrad r;
  r.lse = g.lse[n];
  r.a = g.dlogp ? g.dlogp[n] : 0.0f;
  r.y = g.dlogp ? g.labels[n] : -1;
  r.b = g.dentropy ? g.dentropy[n] : 0.0f;
  r.H = g.dentropy ? g.entropy[n] : 0.0f;
  if (r.lse == -kInf) { r.a = r.b = r.H = 0.0f; r.lse = kInf; r.y = -1; }     // nothing allowed: p = 0 everywhere
  return r;
}
__device__ __forceinline__ float grad1(float x, int64_t i, const RowGrad& r) {
  const float q = x - r.lse, p = expf(q);
  const float d = r.a * ((i == r.y ? 1.0f : 0.0f) - p);
  return p == 0.0f ? d : fmaf(-r.b * p, q + r.H, d);
}

constexpr int kGradT = 256;
template <typename T>
__global__ __launch_bounds__(kGradT) void log_probs_grad_kernel(LogProbsGradArgs g) {
  const int64_t n = blockIdx.x;
  const RowGrad r = row_grad(g, n);
  const T* x = (const T*)g.x + n * g.ld;
  T* dx = (T*)g.dx + n * g.ldd;
  for (int64_t i = threadIdx.x; i < g.V; i += kGradT) store1(dx + i, grad1(load1(x + i), i, r));
}

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" size_t dat_log_probs_workspace(int64_t, int64_t, int) { return 0; }

namespace {
dat_status check_rows(const void* x, dat_dtype dtype, int64_t N, int64_t V, int64_t ld) {
  if ((!x && N != 0) || (dtype != DAT_F32 && dtype != DAT_BF16) || N < 0 || V < 1 || ld < V) return DAT_ERR_ARG;
  if (!aligned(x, dtype == DAT_BF16 ? 2 : 4)) return DAT_ERR_ARG;
  if (V > (1ll << 30) || N > INT32_MAX || (N > 0 && ld > INT64_MAX / 8 / N)) return DAT_ERR_SHAPE;
  return DAT_OK;
}
}  // namespace

extern "C" dat_status dat_log_probs(const void* logits, dat_dtype dtype, int64_t N, int64_t V, int64_t ld, const int32_t* labels,
                                    int top, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_index,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  const dat_status s = check_rows(logits, dtype, N, V, ld);
  if (s != DAT_OK) return s;
  if (top < 0 || top > DAT_MAX_TOP) return DAT_ERR_ARG;
  if (N == 0) return DAT_OK;
  if ((logp && !labels) || (top > 0 && (!top_logp || !top_index))) return DAT_ERR_ARG;
  if (!aligned(labels, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_logp, 4) || !aligned(top_index, 4)) return DAT_ERR_ARG;
  const size_t need = dat_log_probs_workspace(N, V, top);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return DAT_ERR_ARG;
  LogProbsArgs a{logits, N, V, ld, labels, top, logp, entropy, lse, top_logp, top_index};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == DAT_BF16) hipLaunchKernelGGL(log_probs_row_kernel<bf16_t>, dim3((unsigned)N), dim3(kRowT), 0, st, a);
  else hipLaunchKernelGGL(log_probs_row_kernel<float>, dim3((unsigned)N), dim3(kRowT), 0, st, a);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

extern "C" dat_status dat_log_probs_backward(const void* logits, dat_dtype dtype, int64_t N, int64_t V, int64_t ld,
                                             const int32_t* labels, const float* lse, const float* entropy, const float* dlogp,
                                             const float* dentropy, void* dlogits, int64_t ldd, void* stream) {
  dat_status s = check_rows(logits, dtype, N, V, ld);
  if (s == DAT_OK) s = check_rows(dlogits, dtype, N, V, ldd);
  if (s != DAT_OK) return s;
  if (N == 0) return DAT_OK;
  if (!lse || !dlogp != !labels || !entropy != !dentropy || (dlogits == logits && ldd != ld)) return DAT_ERR_ARG;
  if (!aligned(labels, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4)) return DAT_ERR_ARG;
  LogProbsGradArgs g{logits, N, V, ld, ldd, labels, lse, entropy, dlogp, dentropy, dlogits};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == DAT_BF16) hipLaunchKernelGGL(log_probs_grad_kernel<bf16_t>, dim3((unsigned)N), dim3(kGradT), 0, st, g);
  else hipLaunchKernelGGL(log_probs_grad_kernel<float>, dim3((unsigned)N), dim3(kGradT), 0, st, g);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}
