// Log probabilities of given labels over rows of logits, with entropies and the largest alternatives, and the gradient.
//
// With M = max x, s = sum 2^t and w = sum t 2^t, t = (x - M) log2 e:  lse = M + ln s,  logp_y = (x_y - M) - ln s,
// H = ln s - ln 2 w / s.  The logits are read once: a workgroup holds its row, or a part of it, in registers; what comes of the
// parts of a row is joined by a second, small kernel.  Bound by HBM (one read) and the vector units, twenty instructions a logit in
// bf16, alternatives included: 2039 x 50021 bf16 with eight of them 57 us = 3.6 TB/s, issuing for 82 % of it (two workgroups of 1024
// threads on a compute unit; 64 us with two of 512 that hold twice as much).  Few long rows are latency: 3 x 131075 with 20 alternatives 12.4 us
// in two launches.
//
// Alternatives are ordered by one 64-bit key, the logit (as an ordered integer) above the complement of the index, so that equal
// logits go by ascending index and no two keys are equal.  The k-th largest of 64 groups' maxima is no larger than the k-th
// largest logit: what is not below it, a few more than k, goes to a list in LDS and is ranked there.  A list that would not fit
// (many equal logits) is replaced by k searches for the next key.
#include "kernels.h"
#include "lanes.h"

namespace dat {
namespace {

constexpr float kInf = __builtin_inff(), kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kTiny = -150.0f;             // 2^-150 is 0 in fp32: stands for all smaller exponents

template <typename T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f2bf(v); }

__device__ __forceinline__ float minus_inf_to_zero(float m) { return m == -kInf ? 0.0f : m; }
// Adds one logit to the sums for the maximum m (finite).
__device__ __forceinline__ void add(float x, float m, float& s, float& w) {
  const float t = fmaxf((x - m) * kLog2e, kTiny), e = __builtin_amdgcn_exp2f(t);
  s += e;
  w = fmaf(t, e, w);
}
// The sums of maximum m as sums of maximum M >= m (m = -inf: nothing there).
__device__ __forceinline__ void rescale(float m, float M, float& s, float& w) {
  const float d = m == M ? 0.0f : fmaxf((m - M) * kLog2e, kTiny), e = __builtin_amdgcn_exp2f(d);
  w = e * fmaf(d, s, w);
  s *= e;
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

struct Part { float m, s, w, pad; };         // of one part of a row
struct LogProbsArgs {
  const void* x; int64_t N, V, ld; const int32_t* labels; int top;
  float *logp, *entropy, *lse, *top_logp; int32_t* top_index;
  int parts, part_vectors;                   // parts of a row, 16-byte vectors of a part
  Part* part; uint64_t* keys;                // [N][parts], [N][parts][top]
};

__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) { const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)k, d); k = o > k ? o : k; }
  return k;
}

// The row's results from its maximum and sums, by one thread.  M: NaN or +inf for a row that holds such, -inf for an empty one.
template <typename T> __device__ void write_stats(const LogProbsArgs& a, int64_t n, float M, float s, float w) {
  const bool bad = !(M < kInf), empty = M == -kInf;
  const float ls = logf(s), nan = __builtin_nanf("");
  if (a.lse) a.lse[n] = bad ? nan : empty ? -kInf : M + ls;
  if (a.entropy) a.entropy[n] = bad ? nan : empty ? 0.0f : fmaxf(ls - kLn2 * w / s, 0.0f);
  if (a.logp) {
    const int y = a.labels[n];
    const bool ok = (unsigned)y < (unsigned)a.V && !bad;
    a.logp[n] = !ok ? nan : empty ? -kInf : (load1((const T*)a.x + n * a.ld + y) - M) - ls;
  }
}
__device__ __forceinline__ void write_top(const LogProbsArgs& a, int64_t n, int r, uint64_t key, float M, float s) {
  const bool bad = !(M < kInf), none = key == 0;
  a.top_index[n * a.top + r] = none || bad ? -1 : key_index(key);
  a.top_logp[n * a.top + r] = bad ? __builtin_nanf("") : none ? -kInf : (key_value(key) - M) - logf(s);
}

// ---- short rows: L lanes a row, E logits a lane ---------------------------------------------------------------------------
constexpr int kShortT = 256;
template <typename T, int L, int E>
__global__ __launch_bounds__(kShortT) void log_probs_short_kernel(LogProbsArgs a) {
  const int64_t n = (int64_t)blockIdx.x * (kShortT / L) + threadIdx.x / L;
  const int lane = threadIdx.x & (L - 1), V = (int)a.V;
  const bool row = n < a.N;                      // (lanes of a row that is not there take part in the exchanges of their wavefront)
  const T* x = (const T*)a.x + (row ? n : 0) * a.ld;
  float v[E], m = -kInf, s = 0.0f, w = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) { const int i = lane + L * e; v[e] = i < V ? load1(x + i) : -kInf; }
#pragma unroll
  for (int e = 0; e < E; ++e) m = maximum(m, v[e]);
  const float M = lanes_max<L>(m), base = minus_inf_to_zero(M);
#pragma unroll
  for (int e = 0; e < E; ++e) add(v[e], base, s, w);
  s = lanes_sum<L>(s); w = lanes_sum<L>(w);
  if (row && lane == 0) write_stats<T>(a, n, M, s, w);
  if (a.top == 0) return;
  // a lane offers its largest logit that is not taken; among equal ones the lowest index goes first
  uint32_t taken = 0;
  float best;
  int at;
  auto offer = [&]() {
    best = -kInf; at = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) if (v[e] > best && !(taken >> e & 1)) { best = v[e]; at = e; }
  };
  offer();
  for (int r = 0; r < a.top; ++r) {
    const float top = lanes_max<L>(best);
    const int own = lane + L * at, index = lanes_min<L>(best == top ? own : 0x7fffffff);
    if (row && lane == 0) write_top(a, n, r, top > -kInf ? key_of(top, index) : 0, M, s);
    if (best == top && own == index) { taken |= 1u << at; offer(); }
  }
}

// ---- long rows -----------------------------------------------------------------------------------------------------------
constexpr int kList = 512;                       // candidates that the list in LDS holds
template <int NT> struct Selection {             // shared memory of one workgroup
  float s_v[NT / 64], s_s[NT / 64], s_w[NT / 64];
  float s_group[64], s_bound;
  uint64_t s_list[kList], s_wave[NT / 64];
  int s_count;
};

// The k-th largest of the maxima of 64 groups of threads (or less), k >= 1, in every thread; -inf where fewer hold anything.
template <int NT> __device__ __forceinline__ float lower_bound_of_top(float best, int k, Selection<NT>& sh) {
  constexpr int G = NT / 64;
  if (G >= 2) best = fmaxf(best, __int_as_float(dpp<0xb1, 0xf>(__float_as_int(best))));
  if (G >= 4) best = fmaxf(best, __int_as_float(dpp<0x4e, 0xf>(__float_as_int(best))));
  if (G >= 8) best = fmaxf(best, __int_as_float(dpp<0x141, 0xf>(__float_as_int(best))));
  if (G >= 16) best = fmaxf(best, __int_as_float(dpp<0x140, 0xf>(__float_as_int(best))));
  if (threadIdx.x % G == 0) sh.s_group[threadIdx.x / G] = best;
  if (threadIdx.x == 0) sh.s_count = 0;
  __syncthreads();
  if (threadIdx.x < 64) {                        // (by one wavefront: the others' turn on the vector units is another workgroup's)
    const float own = sh.s_group[threadIdx.x];
    int above = 0;
#pragma unroll
    for (int g = 0; g < 64; ++g) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(own), g)) > own;
    const float bound = -lanes_max<64>(above < k ? -own : -kInf);
    if (threadIdx.x == 0) sh.s_bound = bound;
  }
  __syncthreads();
  return sh.s_bound;
}
template <int NT> __device__ __forceinline__ void append(uint64_t key, Selection<NT>& sh) {
  const int at = atomicAdd(&sh.s_count, 1);      // (the order of the list does not matter)
  if (at < kList) sh.s_list[at] = key;
}
// done(r, key) for the k largest keys in order, by one thread each.  The list holds every key from the k-th largest up; where it
// did not fit, next_below(key) finds a thread's largest key below one, k times.
template <int NT, typename N, typename D>
__device__ __forceinline__ void select_top(int k, Selection<NT>& sh, N next_below, D done) {
  __syncthreads();
  const int count = sh.s_count;
  if (count <= kList) {
    for (int i = threadIdx.x; i < count; i += NT) {
      const uint64_t own = sh.s_list[i];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += sh.s_list[j] > own;
      if (rank < k) done(rank, own);
    }
    for (int r = count + threadIdx.x; r < k; r += NT) done(r, 0);
    return;
  }
  uint64_t below = ~0ull;
  for (int r = 0; r < k; ++r) {
    const uint64_t best = wave_max(next_below(below));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.s_wave[threadIdx.x >> 6] = best;
    __syncthreads();
    below = sh.s_wave[0];
    for (int i = 1; i < NT / 64; ++i) below = sh.s_wave[i] > below ? sh.s_wave[i] : below;
    if (threadIdx.x == 0) done(r, below);
  }
}

// A workgroup's maximum and sums from those of its threads.
template <int NT> __device__ __forceinline__ void block_stats(float m, float& M, float& s, float& w, Selection<NT>& sh) {
  M = lanes_max<64>(m);
  if ((threadIdx.x & 63) == 0) sh.s_v[threadIdx.x >> 6] = M;
  __syncthreads();
  M = sh.s_v[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) M = maximum(M, sh.s_v[i]);
  rescale(m, M, s, w);
  s = lanes_sum<64>(s); w = lanes_sum<64>(w);
  if ((threadIdx.x & 63) == 0) { sh.s_s[threadIdx.x >> 6] = s; sh.s_w[threadIdx.x >> 6] = w; }
  __syncthreads();
  s = sh.s_s[0]; w = sh.s_w[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) { s += sh.s_s[i]; w += sh.s_w[i]; }
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename T> __device__ __forceinline__ float element(const u32x4& v, int j) {
  if (sizeof(T) == 4) return __uint_as_float(v[j]);
  return __uint_as_float(j % 2 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16);
}

// (Held vectors are unpacked anew in every pass: the compiler would keep the unpacked values, and spill.)
__device__ __forceinline__ void forget(u32x4& v) { asm volatile("" : "+v"(v)); }

// Rows start at any element: vectors are those of the 16-byte blocks that the row touches, what lies beside the row in the first
// and the last counts as -inf.  (Such a block holds an element of the row, so all of it can be read.)
template <typename T, int NT, int VPT, bool WHOLE>
__global__ __launch_bounds__(NT) void log_probs_long_kernel(LogProbsArgs a) {
  constexpr int VE = 16 / sizeof(T);
  __shared__ Selection<NT> sh;
  const int64_t n = WHOLE ? blockIdx.x : blockIdx.x / (unsigned)a.parts;
  const int p = WHOLE ? 0 : (int)(blockIdx.x - n * a.parts), V = (int)a.V;
  const uintptr_t row = reinterpret_cast<uintptr_t>((const T*)a.x + n * a.ld);
  const int head = (int)(row & 15) / (int)sizeof(T), vectors = (head + V + VE - 1) / VE;
  const int first = p * a.part_vectors, own = WHOLE ? vectors : max(0, min(a.part_vectors, vectors - first));
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((row & ~(uintptr_t)15) + (uintptr_t)first * 16), 0,
                                                                     own * 16, 0x00020000);
  u32x4 v[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(threadIdx.x + i * NT) * 16, 0, 0);
  const int e0 = (first + (int)threadIdx.x) * VE - head;        // index of the thread's first element in the row
  float m = -kInf, s = 0.0f, w = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int at = e0 + i * NT * VE;
    // elements from..to of the vector belong to the row and the part
    int from = max(-at, 0), to = (int)threadIdx.x + i * NT < own ? min(V - at, VE) : 0;
    asm volatile("" : "+v"(from), "+v"(to));     // (the compiler would follow the conditions from vector to vector)
    if (from > 0 || to < VE) {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const uint32_t gone = j < from || j >= to ? 0xffffffffu : 0u;
        if (sizeof(T) == 4) v[i][j] = (v[i][j] & ~gone) | (gone & 0xff800000u);
        else { const uint32_t half = gone & (j % 2 ? 0xffff0000u : 0xffffu); v[i][j / 2] = (v[i][j / 2] & ~half) | (half & 0xff80ff80u); }
      }
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) m = maximum(m, element<T>(v[i], j));
    __builtin_amdgcn_sched_barrier(0);
  }
  const float base = minus_inf_to_zero(m);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    forget(v[i]);
    float si = 0.0f, wi = 0.0f;
#pragma unroll
    for (int j = 0; j < VE; ++j) add(element<T>(v[i], j), base, si, wi);
    s += si; w += wi;
    __builtin_amdgcn_sched_barrier(0);
  }
  float M;
  block_stats<NT>(m, M, s, w, sh);
  if (threadIdx.x == 0) {
    if (WHOLE) write_stats<T>(a, n, M, s, w);
    else a.part[n * a.parts + p] = Part{M, s, w, 0.0f};
  }
  if (a.top == 0) return;
  // values only: elements equal to the bound go to the list as well
  const float least = lower_bound_of_top<NT>(m, a.top, sh);
  const T* x = reinterpret_cast<const T*>(row);
  const int lo = max(0, first * VE - head), hi = min(V, (first + own) * VE - head);      // the part's elements
  if (m >= least && m > -kInf) {
    uint32_t hits = 0;                           // vectors that reach the bound: one or two, read again element by element
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      forget(v[i]);
      float top = element<T>(v[i], 0);
#pragma unroll
      for (int j = 1; j < VE; ++j) top = fmaxf(top, element<T>(v[i], j));
      hits |= top >= least ? 1u << i : 0u;
    }
#pragma nounroll
    for (; hits; hits &= hits - 1) {
      const int at = e0 + (__ffs(hits) - 1) * NT * VE;
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float f = at + j >= lo && at + j < hi ? load1(x + at + j) : -kInf;
        if (f >= least && f > -kInf) append<NT>(key_of(f, at + j), sh);
      }
    }
  }
  select_top<NT>(a.top, sh,
    [&](uint64_t below) {
      uint64_t best = 0;
      for (int i = lo + (int)threadIdx.x; i < hi; i += NT) { const uint64_t k = key_of(load1(x + i), i); best = k < below && k > best ? k : best; }
      return best;
    },
    [&](int k, uint64_t key) {
      if (WHOLE) write_top(a, n, k, key, M, s);
      else a.keys[(n * a.parts + p) * a.top + k] = key;
    });
}

// Joins the parts of a row.
constexpr int kJoinT = 256;
template <typename T>
__global__ __launch_bounds__(kJoinT) void log_probs_join_kernel(LogProbsArgs a) {
  __shared__ Selection<kJoinT> sh;
  const int64_t n = blockIdx.x;
  const Part* part = a.part + n * a.parts;
  float m = -kInf, M, s = 0.0f, w = 0.0f;
  for (int p = threadIdx.x; p < a.parts; p += kJoinT) m = maximum(m, part[p].m);
  for (int p = threadIdx.x; p < a.parts; p += kJoinT) {
    float ps = part[p].s, pw = part[p].w;
    rescale(part[p].m, m, ps, pw);
    s += ps; w += pw;
  }
  block_stats<kJoinT>(m, M, s, w, sh);
  if (threadIdx.x == 0) write_stats<T>(a, n, M, s, w);
  if (a.top == 0) return;
  const uint64_t* keys = a.keys + n * a.parts * a.top;
  const int count = a.parts * a.top;
  uint64_t best = 0;
  for (int i = threadIdx.x; i < count; i += kJoinT) best = keys[i] > best ? keys[i] : best;
  const float least = lower_bound_of_top<kJoinT>(best ? key_value(best) : -kInf, a.top, sh);
  for (int i = threadIdx.x; i < count; i += kJoinT) if (keys[i] && key_value(keys[i]) >= least) append<kJoinT>(keys[i], sh);
  select_top<kJoinT>(a.top, sh,
    [&](uint64_t below) {
      uint64_t k = 0;
      for (int i = threadIdx.x; i < count; i += kJoinT) k = keys[i] < below && keys[i] > k ? keys[i] : k;
      return k;
    },
    [&](int k, uint64_t key) { write_top(a, n, k, key, M, s); });
}

// Which kernel.  As few lanes a row as hold it, 4 to 16 logits (2^20 x 10 fp32 17.2 us against 55.1 with 16 lanes), 16 to 64 (65536 x 64
// 6.4 against 16.9 with 64) and, where there are more than 1024 rows, to 256 (65536 x 100 with three alternatives 18.8 against 37.9;
// 2048 x 100 5.0 against 4.3), then a wavefront to 1024 (8192 x 1000 with five alternatives 17.4 against 20.6 for a workgroup a
// row, 4096 x 300 bf16 9.9 against 13.4; even at 2048 rows).  With fewer rows a workgroup each (256 x 1000 4.7 against 6.0 for a
// wavefront, 256 x 100 4.8 against 5.8, 1024 x 300 5.3 against 6.2), and for longer ones; in parts where a row is longer than 1024
// threads hold, and where there are at most 32 rows of more than 2^15 logits, when a second launch costs less than a row's time in
// one workgroup (bf16: 3 x 131075 with 20 alternatives 12.4 us against 25.0, 8 x 50021 9.2 against 10.5, 32 x 131000 11.9 against
// 18.3, 48 x 50021 13.2 against 10.9; fp32: 1 x 33000 7.7 against 10.8, 32 x 65000 10.1 against 11.5, 48 x 65000 12.7 against
// 11.8, 4 x 20000 8.0 against 7.5).
struct LogProbsPlan { int lanes, nt, vpt, parts, part_vectors; };     // lanes = 0: nt threads, vpt vectors each, else vpt logits a lane
LogProbsPlan log_probs_plan(int width, int64_t N, int64_t V) {
  if (V <= 16) return {4, 0, 4, 1, 0};
  if (V <= 64) return {16, 0, 4, 1, 0};
  if (V <= 256 && N > 1024) return {16, 0, 16, 1, 0};
  if (V <= 1024 && N > 1024) return {64, 0, 16, 1, 0};
  static const int sizes[][2] = {{256, 1}, {256, 4}, {256, 8}, {512, 8}, {1024, 8}, {1024, 16}};
  const int64_t vectors = V * width / 16 + 2;            // at most, with the row's start anywhere
  int64_t parts = (vectors + 1024 * 16 - 1) / (1024 * 16);
  if (N * parts <= 32 && V > 32768) {
    const int64_t want = (256 + N - 1) / N, most = (vectors + 255) / 256;
    if (parts < want) parts = want < most ? want : most;
  }
  const int64_t each = (vectors + parts - 1) / parts;
  int i = 0;
  while (sizes[i][0] * sizes[i][1] < each) ++i;
  return {0, sizes[i][0], sizes[i][1], (int)parts, (int)each};
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
__device__ __forceinline__ float grad1(float x, int i, const RowGrad& r) {
  const float q = x - r.lse, p = __builtin_amdgcn_exp2f(maximum(q * kLog2e, kTiny));   // (NaN where lse is)
  const float d = r.a * ((i == r.y ? 1.0f : 0.0f) - p);
  return p == 0.0f ? d : fmaf(-r.b * p, q + r.H, d);
}

// Streaming, bound by HBM (one read, one write): 1021 x 32771 fp32 51 us = 5.2 TB/s.  A thread takes vectors of 16 bytes from the
// row's start, at any alignment: global memory takes them whole.
constexpr int kGradT = 256, kGradV = 4;      // vectors a thread
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Vector { T x[16 / sizeof(T)]; };

// An lse far from zero has lost what it knows of the sum (at 1e6 it is rounded to sixteenths, at the type's lowest value nothing is
// left), and p = e^(x - lse) with it.  Up to 64 its rounding moves p by at most 2^-19; beyond, maximum and sum are taken from the row again,
// p = e^((x - M) - ln s), by the threads of one workgroup or the lanes of a short row: a second read, for such rows alone (all rows
// at lse = 100: 1021 x 32771 fp32 90 us against 45, 16384 x 1000 37 against 21, 64 x 262144 379 against 21).
// (By its bits, as numbers of a scalar register: finite, and more than 64 in size.)
__device__ __forceinline__ bool is_far(const RowGrad& r) {
  constexpr uint32_t k64 = 0x42800000u, kInfinite = 0x7f800000u;
  return (__float_as_uint(r.lse) & 0x7fffffffu) - (k64 + 1) < kInfinite - (k64 + 1);
}

// use(index, vector, elements) for the vectors of a row that are thread `lane`'s of L, in long rows four loads at a time; a vector at the row's
// end has -inf behind it.
template <typename T, int L, typename F> __device__ __forceinline__ void each_vector(const T* x, int V, int lane, F use) {
  constexpr int VE = 16 / sizeof(T), N = L < 64 ? 1 : 4;      // (short rows have four at most, and would pay with registers)
  int i = lane * VE;
  for (; i <= V - VE - (N - 1) * L * VE; i += N * L * VE) {
    Vector<T> v[N];
    float f[N][VE];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = *reinterpret_cast<const Vector<T>*>(x + i + k * L * VE);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int j = 0; j < VE; ++j) f[k][j] = load1(&v[k].x[j]);
#pragma unroll
    for (int k = 0; k < N; ++k) use(i + k * L * VE, f[k]);
  }
  for (; i < V; i += L * VE) {
    Vector<T> v;
    float f[VE];
    if (i + VE <= V) v = *reinterpret_cast<const Vector<T>*>(x + i);
    else {
#pragma unroll
      for (int j = 0; j < VE; ++j) v.x[j] = x[min(i + j, V - 1)];
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = i + j < V ? load1(&v.x[j]) : -kInf;
    use(i, f);
  }
}
// Gradient of a far row by L threads, `lane` of them; max_of and sum_of join a value of theirs.  dx may be x: after the joins a thread reads
// what it alone writes.
template <typename T, int L, typename M, typename S>
__device__ __forceinline__ void far_row(const T* x, T* dx, int V, int lane, RowGrad r, M max_of, S sum_of) {
  constexpr int VE = 16 / sizeof(T);
  float m = -kInf, s = 0.0f;
  auto scale = [](float from, float to) { return __builtin_amdgcn_exp2f(fmaxf((from - to) * kLog2e, kTiny)); };   // (-inf less -inf: 0)
  each_vector<T, L>(x, V, lane, [&](int, const float (&f)[VE]) {
    float top = m;
#pragma unroll
    for (int j = 0; j < VE; ++j) top = fmaxf(top, f[j]);
    if (top > m) { s *= scale(m, top); m = top; }
#pragma unroll
    for (int j = 0; j < VE; ++j) s += scale(f[j], m);
  });
  const float top = max_of(m);
  r.lse = logf(sum_of(s * (m == top ? 1.0f : scale(m, top))));
  each_vector<T, L>(x, V, lane, [&](int i, const float (&f)[VE]) {
    if (i + VE <= V) {
      Vector<T> v;
#pragma unroll
      for (int j = 0; j < VE; ++j) store1(&v.x[j], grad1(f[j] - top, i + j, r));
      *reinterpret_cast<Vector<T>*>(dx + i) = v;
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) if (i + j < V) store1(dx + i + j, grad1(f[j] - top, i + j, r));
    }
  });
}

template <typename T>
__global__ __launch_bounds__(kGradT) void log_probs_grad_kernel(LogProbsGradArgs g, unsigned blocks) {
  constexpr int VE = 16 / sizeof(T);
  const int64_t n = blockIdx.x / blocks;
  const int V = (int)g.V, first = (int)(blockIdx.x - n * blocks) * (kGradT * kGradV * VE) + (int)threadIdx.x * VE;
  const RowGrad r = row_grad(g, n);
  const T* x = (const T*)g.x + n * g.ld;
  T* dx = (T*)g.dx + n * g.ldd;
  Vector<T> v[kGradV];
#pragma unroll
  for (int k = 0; k < kGradV; ++k) {
    const int i = first + k * kGradT * VE;
    if (i + VE <= V) v[k] = *reinterpret_cast<const Vector<T>*>(x + i);
  }
  if (is_far(r)) {                           // (all of the row by its first workgroup: dx may be x)
    __shared__ float s_wave[2][kGradT / 64];
    if (blockIdx.x != n * blocks) return;
    auto joined = [&](float (&s)[kGradT / 64], float v) { if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v; __syncthreads(); };
    far_row<T, kGradT>(x, dx, V, threadIdx.x, r,
      [&](float m) { joined(s_wave[0], lanes_max<64>(m)); return fmaxf(fmaxf(s_wave[0][0], s_wave[0][1]), fmaxf(s_wave[0][2], s_wave[0][3])); },
      [&](float s) { joined(s_wave[1], lanes_sum<64>(s)); return (s_wave[1][0] + s_wave[1][1]) + (s_wave[1][2] + s_wave[1][3]); });
    return;
  }
#pragma unroll
  for (int k = 0; k < kGradV; ++k) {
    const int i = first + k * kGradT * VE;
    if (i + VE <= V) {
#pragma unroll
      for (int j = 0; j < VE; ++j) store1(&v[k].x[j], grad1(load1(&v[k].x[j]), i + j, r));
      *reinterpret_cast<Vector<T>*>(dx + i) = v[k];
    } else {
      for (int j = i; j < V; ++j) store1(dx + j, grad1(load1(x + j), j, r));
    }
  }
}

// Short rows: L lanes a row, kGradV vectors a lane at most.
template <typename T, int L>
__global__ __launch_bounds__(kGradT) void log_probs_grad_short_kernel(LogProbsGradArgs g) {
  constexpr int VE = 16 / sizeof(T);
  const int64_t n = (int64_t)blockIdx.x * (kGradT / L) + threadIdx.x / L;
  if (n >= g.N) return;
  const int V = (int)g.V, first = (int)(threadIdx.x % L) * VE;
  const RowGrad r = row_grad(g, n);
  const T* x = (const T*)g.x + n * g.ld;
  T* dx = (T*)g.dx + n * g.ldd;
  if (is_far(r)) {                           // (all lanes of the row, those without an element as well, for the exchanges)
    far_row<T, L>(x, dx, V, threadIdx.x % L, r, [](float m) { return lanes_max<L>(m); }, [](float s) { return lanes_sum<L>(s); });
    return;
  }
  if (first >= V) return;
  Vector<T> v[kGradV];
#pragma unroll
  for (int k = 0; k < kGradV; ++k) {
    const int i = first + k * L * VE;
    if (i + VE <= V) v[k] = *reinterpret_cast<const Vector<T>*>(x + i);
    else {
#pragma unroll
      for (int j = 0; j < VE; ++j) if (i + j < V) v[k].x[j] = x[i + j];
    }
  }
#pragma unroll
  for (int k = 0; k < kGradV; ++k) {
    const int i = first + k * L * VE;
    if (i >= V) break;
#pragma unroll
    for (int j = 0; j < VE; ++j) store1(&v[k].x[j], i + j < V ? grad1(load1(&v[k].x[j]), i + j, r) : 0.0f);
    if (i + VE <= V) *reinterpret_cast<Vector<T>*>(dx + i) = v[k];
    else {
#pragma unroll
      for (int j = 0; j < VE; ++j) if (i + j < V) dx[i + j] = v[k].x[j];
    }
  }
}

template <typename T> void launch_log_probs(const LogProbsPlan& p, const LogProbsArgs& a, hipStream_t st) {
  const unsigned rows = (unsigned)a.N;
#define DAT_LP_SHORT(L, E)                                                                                                          \
  if (p.lanes == L && p.vpt == E) {                                                                                                 \
    hipLaunchKernelGGL((log_probs_short_kernel<T, L, E>), dim3((rows + kShortT / L - 1) / (kShortT / L)), dim3(kShortT), 0, st, a); \
    return;                                                                                                                         \
  }
  DAT_LP_SHORT(4, 4) DAT_LP_SHORT(16, 4) DAT_LP_SHORT(16, 16) DAT_LP_SHORT(64, 16)
#undef DAT_LP_SHORT
#define DAT_LP_SIZE(NT, VPT)                                                                                                        \
  if (p.nt == NT && p.vpt == VPT) {                                                                                                 \
    if (p.parts == 1) hipLaunchKernelGGL((log_probs_long_kernel<T, NT, VPT, true>), dim3(rows), dim3(NT), 0, st, a);                \
    else hipLaunchKernelGGL((log_probs_long_kernel<T, NT, VPT, false>), dim3(rows * (unsigned)p.parts), dim3(NT), 0, st, a);        \
  }
  DAT_LP_SIZE(256, 1) DAT_LP_SIZE(256, 4) DAT_LP_SIZE(256, 8) DAT_LP_SIZE(512, 8) DAT_LP_SIZE(1024, 8) DAT_LP_SIZE(1024, 16)
#undef DAT_LP_SIZE
  if (p.parts > 1) hipLaunchKernelGGL(log_probs_join_kernel<T>, dim3(rows), dim3(kJoinT), 0, st, a);
}

// Lanes a row of the gradient, 0: workgroups of one row.  2^20 x 10 fp32 20.8 us with 4 lanes, 64.1 with 16, 894 with a workgroup;
// 16384 x 256 9.3 with 16, 14.0 with a workgroup; 256 x 100 3.2 and 2.7; longer rows: 16384 x 1000 24.9 with 64 lanes, 22.1 with a
// workgroup.
int log_probs_grad_lanes(int width, int64_t V) {
  const int64_t vectors = (V * width + 15) / 16;
  return vectors <= 4 * kGradV ? 4 : vectors <= 16 * kGradV ? 16 : 0;
}
template <typename T> void launch_log_probs_grad(int lanes, unsigned blocks, unsigned each, const LogProbsGradArgs& g, hipStream_t st) {
  if (lanes == 4) hipLaunchKernelGGL((log_probs_grad_short_kernel<T, 4>), dim3(blocks), dim3(kGradT), 0, st, g);
  else if (lanes == 16) hipLaunchKernelGGL((log_probs_grad_short_kernel<T, 16>), dim3(blocks), dim3(kGradT), 0, st, g);
  else hipLaunchKernelGGL(log_probs_grad_kernel<T>, dim3(blocks), dim3(kGradT), 0, st, g, each);
}

}  // namespace
}  // namespace dat

using namespace dat;

namespace {
size_t workspace_of(const LogProbsPlan& p, int64_t N, int top) {
  return p.parts > 1 ? (size_t)N * p.parts * (sizeof(Part) + sizeof(uint64_t) * (size_t)top) : 0;
}
}  // namespace

// (The larger of the types' needs.)
extern "C" size_t dat_log_probs_workspace(int64_t N, int64_t V, int top) {
  if (N < 1 || V < 1 || V > (1ll << 30) || N > INT32_MAX || top < 0 || top > DAT_MAX_TOP) return 0;
  const size_t a = workspace_of(log_probs_plan(2, N, V), N, top), b = workspace_of(log_probs_plan(4, N, V), N, top);
  return a > b ? a : b;
}

namespace {
dat_status check_rows(const void* x, dat_dtype dtype, int64_t N, int64_t V, int64_t ld) {
  if ((!x && N != 0) || (dtype != DAT_F32 && dtype != DAT_BF16) || N < 0 || V < 1 || ld < V) return DAT_ERR_ARG;
  if (!aligned(x, dtype == DAT_BF16 ? 2 : 4)) return DAT_ERR_ARG;
  if (V > (1ll << 30) || N > INT32_MAX || (N > 0 && ld > INT64_MAX / 8 / N)) return DAT_ERR_SHAPE;
  return DAT_OK;
}

// N rows of `row` bytes, `step` bytes apart, at p and at q: share some bytes, but not all.  (step N < 2^63: check_rows.)
bool rows_overlap(const void* p, const void* q, uint64_t N, uint64_t row, uint64_t step) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  const uint64_t d = a > b ? a - b : b - a;
  if (d == 0 || d >= (N - 1) * step + row) return false;
  return d % step < row || (step - d % step < row && d < (N - 1) * step);      // beside the same row, and beside the next one
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
  const LogProbsPlan p = log_probs_plan(dtype == DAT_BF16 ? 2 : 4, N, V);
  LogProbsArgs a{logits, N, V, ld, labels, top, logp, entropy, lse, top_logp, top_index, p.parts, p.part_vectors, (Part*)workspace, nullptr};
  if (p.parts > 1) a.keys = reinterpret_cast<uint64_t*>(a.part + N * p.parts);
  const int64_t lanes = p.lanes ? p.lanes : (int64_t)p.parts * p.nt;
  if (!fits_launch((N * lanes + kShortT - 1) / kShortT, kShortT) || (p.parts > 1 && !fits_launch(N, kJoinT))) return DAT_ERR_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == DAT_BF16) launch_log_probs<bf16_t>(p, a, st); else launch_log_probs<float>(p, a, st);
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
  const int lanes = log_probs_grad_lanes(dtype == DAT_BF16 ? 2 : 4, V);
  const int64_t per = kGradT * kGradV * 16 / (dtype == DAT_BF16 ? 2 : 4), each = lanes ? 1 : (V + per - 1) / per;
  const int64_t blocks = lanes ? (N + kGradT / lanes - 1) / (kGradT / lanes) : N * each;
  if (!fits_launch(blocks, kGradT)) return DAT_ERR_SHAPE;
  const uint64_t width = dtype == DAT_BF16 ? 2 : 4;
  if (ld == ldd && rows_overlap(logits, dlogits, N, V * width, ld * width)) return DAT_ERR_ARG;
  if (dtype == DAT_BF16) launch_log_probs_grad<bf16_t>(lanes, (unsigned)blocks, (unsigned)each, g, st);
  else launch_log_probs_grad<float>(lanes, (unsigned)blocks, (unsigned)each, g, st);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}
