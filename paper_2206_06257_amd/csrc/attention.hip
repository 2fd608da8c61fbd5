// Attention and its gradients on the matrix cores, probabilities never in memory.
//
//   S = scale q k^T,  lse_i = log sum_j exp S_ij,  P = exp(S - lse),  o = P v;
//   D_i = sum_d do o,  dP = do v^T,  dS = P (dP - D),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T do.
//
// A wavefront owns 32 rows of the result (queries; keys for dk and dv) and walks along the other axis in tiles that the
// workgroup's waves share in LDS.  Every product is made transposed, so that a lane holds a single row: 32x32x16 MFMA leaves in lane l
// column l % 32 and rows 8 (r / 4) + 4 (l / 32) + r % 4 (r = 0..15), and row statistics need one exchange between the halves of a
// wave.  The k index of an MFMA may be assigned to (lane half, element) as one likes if both operands agree: the second product takes
// P or dS as its B operand from the registers the first one left it in (elements 0-3 of half h are rows 4h.., elements 4-7 rows
// 8 + 4h..), and reads its A operand from LDS in that order, transposed.  fp32 runs the same code: a 32x32x16 product is eight
// 32x32x2 ones that take the eight elements of a lane one after the other.
#include "kernels.h"
#include "heads.h"
#include <initializer_list>

namespace dat {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef short v4s16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef __amdgpu_buffer_rsrc_t BufRsrc;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();
constexpr int kFar = 1 << 30;                    // lengths stay below it: a window side without a limit
constexpr uint32_t kOob = 0xfffffff0u;           // an offset behind every descriptor's range: the load delivers zeros
constexpr int kTile = 64;                        // rows of an LDS tile
constexpr int kPatience = 8;                     // steps of 2 that the running maximum may fall behind

struct HeadsArg { char* data; int64_t batch, token, head; };    // strides in bytes

struct AttnArgs {
  HeadsArg q, k, v, o, d_o, dq, dk, dv;
  const float* lse_in; float* lse; float* stats;         // stats: [2][rows] lse / ln 2 and D
  const int32_t* off_q; const int32_t* off_k;
  int B, Sq, Sk, H, Hkv, G, D, left, right;
  float scale, c;                                        // c = scale / ln 2
  int rows_per_group, groups, xcd;                       // tiles of a group of heads; groups; 1: a contiguous share of the work for each XCD
  int64_t items, rows;                                   // rows = B * H * Sq (H * Sq packed)
};

// One tile of a result: sequence, heads and rows.
struct Place { int b, hk, g, row0, q0, k0, Lq, Lk; };

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Packed sequences: rows off[b] .. off[b + 1] - 1, clamped to the tensor, so that no offset leads out of it.
__device__ __forceinline__ void sequence(const int32_t* off, int b, int T, int& start, int& len) {
  start = clampi(off[b], 0, T);
  len = max(clampi(off[b + 1], 0, T) - start, 0);
}

// Work item -> place.  The tiles of a group (the query heads of one key head, of one sequence or of all packed ones) follow one another,
// late rows first, which see the most keys where a window is causal.  BM rows a tile; PER: items of a tile (query heads that are
// handled apart).
template <int BM, bool QUERIES>
__device__ __forceinline__ bool find_place(const AttnArgs& a, int per, Place& p) {
  int64_t item = blockIdx.x;
  if (a.xcd) item = (int64_t)(blockIdx.x & 7) * ((a.items + 7) >> 3) + (blockIdx.x >> 3);
  if (item >= a.items) return false;
  const int t = (int)(item / per);
  p.g = (int)(item - (int64_t)t * per);
  const int group = t / a.rows_per_group;
  int tile = a.rows_per_group - 1 - (t - group * a.rows_per_group);
  if (!QUERIES) tile = t - group * a.rows_per_group;      // early keys are seen by the most queries
  if (a.off_q) {
    p.hk = group;
    const int32_t* off = QUERIES ? a.off_q : a.off_k;
    const int T = QUERIES ? a.Sq : a.Sk;
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (clampi(off[mid], 0, T) / BM + mid <= tile) lo = mid; else hi = mid;
    }
    p.b = lo;
    sequence(a.off_q, p.b, a.Sq, p.q0, p.Lq);
    sequence(a.off_k, p.b, a.Sk, p.k0, p.Lk);
    const int j = tile - ((QUERIES ? p.q0 : p.k0) / BM + p.b);
    if (j < 0 || (int64_t)j * BM >= (QUERIES ? p.Lq : p.Lk)) return false;
    p.row0 = j * BM;
  } else {
    p.b = group / a.Hkv;
    p.hk = group - p.b * a.Hkv;
    p.row0 = tile * BM;
    p.q0 = p.k0 = 0; p.Lq = a.Sq; p.Lk = a.Sk;
  }
  return true;
}

// First row of a head of the place's sequence (packed tensors have no batch stride).
__device__ __forceinline__ char* rows_of(const HeadsArg& t, int b, int first, int head) {
  return t.data + (int64_t)b * t.batch + (int64_t)first * t.token + (int64_t)head * t.head;
}
__device__ __forceinline__ int64_t stat_row(const AttnArgs& a, const Place& p, int head) {
  return a.off_q ? (int64_t)head * a.Sq + p.q0 : ((int64_t)p.b * a.H + head) * a.Sq;
}
__device__ __forceinline__ BufRsrc buffer_at(const char* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, (int)0x80000000u, 0x00020000);
}

// ---- fragments: eight elements of a lane ---------------------------------------------------------------------------------
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { u32x4 u; };
template <> struct Frag<float> { float f[8]; };

__device__ __forceinline__ void mma(f32x16& acc, const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.u), __builtin_bit_cast(bf16x8, b.u), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& acc, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[j], b.f[j], acc, 0, 0, 0);
}
__device__ __forceinline__ void zero(f32x16& acc) {
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
}
// Registers 8 kk .. 8 kk + 7 of a result as the B operand of the next product (bf16: rounded to nearest).
template <typename T> __device__ __forceinline__ Frag<T> operand(const f32x16& x, int kk) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f.u[j] = f2bf_pack(x[8 * kk + 2 * j], x[8 * kk + 2 * j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.f[j] = x[8 * kk + j];
  }
  return f;
}
__device__ __forceinline__ float element(const Frag<bf16_t>& f, int j) { return __uint_as_float((j & 1) ? f.u[j >> 1] & 0xffff0000u : f.u[j >> 1] << 16); }
__device__ __forceinline__ float element(const Frag<float>& f, int j) { return f.f[j]; }

// x and its counterpart in the other half of the wave, the lower half's first.
__device__ __forceinline__ void halves(float x, float& low, float& high) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  low = __uint_as_float(r[0]); high = __uint_as_float(r[1]);
}
__device__ __forceinline__ float both_sum(float x) { float a, b; halves(x, a, b); return a + b; }
__device__ __forceinline__ float both_max(float x) { float a, b; halves(x, a, b); return fmaxf(a, b); }

// ---- LDS tiles ---------------------------------------------------------------------------------------------------------------
// A tile holds kTile rows of a head as they are in memory, rows of 128, 256 or 512 bytes (what lies behind D is zero), their 16-byte
// slots permuted: slot s of row r is at s ^ flip(r).  Row fragments (16 bytes of each of 32 rows) then spread over all banks, and so
// do the transposing reads, whose half-waves take 64 bytes of each of four consecutive rows.
template <int ROWB> __device__ __forceinline__ int flip(int r) {
  if (ROWB == 128) return (r & 1) | ((r >> 2 & 1) << 1) | ((r >> 1 & 1) << 2);
  if (ROWB == 256) return ((r & 3) << 2) | (r >> 2 & 3);
  return r & 7;
}

// Loads of a tile straight into LDS: a wave's instruction fills 1 KB, the lane that fills slot p of row r fetches slot p ^ flip(r).
template <int ROWB, int NW> struct TileLoad {
  static constexpr int NS = ROWB / 16, N = kTile * NS / 64 / NW, RPI = 64 / NS;
  uint32_t off[N];
  __device__ __forceinline__ static int row(int i, int wave, int lane) { return (i * NW + wave) * RPI + lane / NS; }
  __device__ __forceinline__ void init(int wave, int lane, int64_t stride, int row_bytes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i, wave, lane), slot = (lane % NS) ^ flip<ROWB>(r);
      off[i] = slot * 16 < row_bytes ? (uint32_t)(r * stride + slot * 16) : kOob;
    }
  }
  __device__ __forceinline__ void load(const char* base, int rows, unsigned char* tile, int wave, int lane) const {
    const BufRsrc r = buffer_at(base);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t at = off[i];
      if (rows < kTile) at = row(i, wave, lane) < rows ? at : kOob;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_ptr)(tile + (i * NW + wave) * 1024), 16, (int)at, 0, 0, 0);
    }
  }
};

// Row fragment: elements 16 kk + 8 (lane / 32) .. + 7 of row `r0` + lane % 32.
template <typename T, int ROWB> struct RowReader {
  int base, mask;
  __device__ __forceinline__ void init(int lane) { base = (lane & 31) * ROWB; mask = flip<ROWB>(lane & 31) << 4 ^ ((lane >> 5) * 8 * (int)sizeof(T)); }
  __device__ __forceinline__ Frag<T> read(const unsigned char* tile, int r0, int kk) const {
    Frag<T> f;
    const unsigned char* p = tile + r0 * ROWB + base;
    if constexpr (sizeof(T) == 2) {
      f.u = *reinterpret_cast<const u32x4*>(p + (mask ^ (kk * 32)));
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(p + (mask ^ (kk * 64))), b = *reinterpret_cast<const u32x4*>(p + (mask ^ (kk * 64 + 16)));
#pragma unroll
      for (int j = 0; j < 4; ++j) { f.f[j] = __uint_as_float(a[j]); f.f[4 + j] = __uint_as_float(b[j]); }
    }
    return f;
  }
};

// Transposed fragment: element 32 blk + lane % 32 of rows r0 + 4 h + 0..3 and r0 + 8 + 4 h + 0..3 (h = lane / 32).  bf16: inside every
// group of 16 lanes the transposing read hands lane i element i % 4 of the 8-byte chunks named by lanes i / 4 + 0, 4, 8, 12.
template <typename T, int ROWB> struct ColReader {
  int base[2], mask[2];
  __device__ __forceinline__ void init(int lane) {
    const int g = lane >> 4, s = lane & 15;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * e + 4 * (g >> 1) + (s >> 2);            // (rows r0 = 0, 16, .. leave the flip as it is)
      base[e] = r * ROWB;
      mask[e] = (flip<ROWB>(r) << 4) ^ ((g & 1) * 32 + (s & 3) * 8);
    }
  }
  __device__ __forceinline__ Frag<T> read(const unsigned char* tile, int r0, int blk, int lane) const {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const v4s16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s16*)(tile + r0 * ROWB + base[e] + (mask[e] ^ (blk * 64))));
        const u32x2 y = __builtin_bit_cast(u32x2, x);
        f.u[2 * e] = y[0]; f.u[2 * e + 1] = y[1];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = r0 + 8 * (j >> 2) + 4 * (lane >> 5) + (j & 3), d = 32 * blk + (lane & 31);
        f.f[j] = *reinterpret_cast<const float*>(tile + r * ROWB + (((d >> 2) ^ flip<ROWB>(r)) << 4) + (d & 3) * 4);
      }
    }
    return f;
  }
};

// Fragments of 32 rows in memory as an operand whose columns are rows: elements 16 kk + 8 (lane / 32) .. of row lane % 32.
template <typename T> __device__ __forceinline__ Frag<T> load_row(BufRsrc r, uint32_t row_off, bool there, int kk, int lane, int D) {
  Frag<T> f;
  const int d = 16 * kk + 8 * (lane >> 5);
  const uint32_t at = there && d < D ? row_off + (uint32_t)(d * (int)sizeof(T)) : kOob;
  if constexpr (sizeof(T) == 2) {
    f.u = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0);
  } else {
    const u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0), b = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at + (at == kOob ? 0 : 16)), 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) { f.f[j] = __uint_as_float(a[j]); f.f[4 + j] = __uint_as_float(b[j]); }
  }
  return f;
}

// Writes a transposed result: lane's row, elements 32 blk + 8 (r / 4) + 4 (lane / 32) + r % 4, each times `factor`, rounded once.
template <typename T, int NB> __device__ __forceinline__ void store_rows(char* row, bool there, const f32x16 (&acc)[NB], float factor, int lane, int D) {
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {                     // the halves exchange: each lane then has eight elements beside one another
        uint32_t x[2], y[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          x[j] = f2bf_pack(acc[blk][8 * b + 2 * j] * factor, acc[blk][8 * b + 2 * j + 1] * factor);
          y[j] = f2bf_pack(acc[blk][8 * b + 4 + 2 * j] * factor, acc[blk][8 * b + 5 + 2 * j] * factor);
        }
        const auto r0 = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false), r1 = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
        const int d = 32 * blk + 16 * b + 8 * (lane >> 5);
        if (there && d < D) *reinterpret_cast<u32x4*>(row + d * 2) = u32x4{r0[0], r1[0], r0[1], r1[1]};
      }
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int d = 32 * blk + 8 * b + 4 * (lane >> 5);
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(acc[blk][4 * b + j] * factor);
        if (there && d < D) *reinterpret_cast<u32x4*>(row + d * 4) = v;
      }
    }
  }
}

template <int NB> __device__ __forceinline__ bool any_nan(const f32x16 (&acc)[NB]) {
  bool nan = false;
#pragma unroll
  for (int blk = 0; blk < NB; ++blk)
#pragma unroll
    for (int r = 0; r < 16; ++r) nan |= acc[blk][r] != acc[blk][r];
  return nan;
}

// What is not finite in a row that a window hides must not reach a row that does not see it (0 times a NaN), and every such case leaves a
// NaN in the accumulators.  They are then made once more with the second product reading a copy of the tiles in which such elements are
// zero, and spoil() puts NaN where a row sees one.
template <typename T> __device__ __forceinline__ bool finite_bits(uint32_t u) {
  if constexpr (sizeof(T) == 2) return (u & 0x7f80u) != 0x7f80u && (u & 0x7f800000u) != 0x7f800000u;
  return (u & 0x7f800000u) != 0x7f800000u;
}
template <typename T, int BYTES, int NT> __device__ __forceinline__ void copy_finite(const unsigned char* from, unsigned char* to, int tid) {
#pragma unroll 1
  for (int at = tid * 16; at < BYTES; at += NT * 16) {
    u32x4 v = *reinterpret_cast<const u32x4*>(from + at);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (sizeof(T) == 4) v[j] = finite_bits<T>(v[j]) ? v[j] : 0u;
      else v[j] = (finite_bits<T>(v[j] & 0xffffu) ? v[j] & 0xffffu : 0u) | (finite_bits<T>(v[j] & 0xffff0000u) ? v[j] & 0xffff0000u : 0u);
    }
    *reinterpret_cast<u32x4*>(to + at) = v;
  }
}
template <typename T, int NB> __device__ __forceinline__ void spoil(f32x16 (&acc)[NB], const char* base, int64_t stride, int lo, int hi, int lane, int D) {
#pragma unroll 1
  for (int j = lo; j <= hi; ++j) {
    const T* const row = reinterpret_cast<const T*>(base + (int64_t)j * stride);
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int d = 32 * blk + 8 * b + 4 * (lane >> 5);
        if (d < D) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t u;
            if constexpr (sizeof(T) == 2) u = row[d + x]; else u = __float_as_uint(row[d + x]);
            acc[blk][4 * b + x] = finite_bits<T>(u) ? acc[blk][4 * b + x] : __builtin_nanf("");
          }
        }
      }
  }
}

// Keys that rows [first, last] of the queries see: [lo, hi] (hi < lo: none).
__device__ __forceinline__ void keys_seen(const AttnArgs& a, const Place& p, int first, int last, int& lo, int& hi) {
  const int c0 = first + p.Lk - p.Lq, c1 = last + p.Lk - p.Lq;
  lo = max(0, c0 - a.left);
  hi = min(p.Lk - 1, c1 + a.right);
}
__device__ __forceinline__ void wait_tile() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
}

template <typename T, int NB> constexpr int row_bytes() { return (NB <= 2 ? 64 : 128) * (int)sizeof(T); }

// ---- forward -----------------------------------------------------------------------------------------------------------------
// The running maximum m (in scores) is raised only where one passes it by kPatience / c: what is summed then stays below 2^kPatience
// times the sum that the true maximum would give, and few tiles rescale the accumulators.
template <typename T, int NB, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_fwd_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), KK = 2 * NB, BM = 32 * NW, STAGE = 2 * kTile * ROWB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  Place p;
  if (!find_place<BM, true>(a, a.G, p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = p.hk * a.G + p.g, half = lane >> 5;
  const int i0 = p.row0 + 32 * wave, i = i0 + (lane & 31);
  const bool there = i < p.Lq;
  const char* const kbase = rows_of(a.k, p.b, p.k0, p.hk);
  const char* const vbase = rows_of(a.v, p.b, p.k0, p.hk);

  Frag<T> q[KK];
  {
    const BufRsrc r = buffer_at(rows_of(a.q, p.b, p.q0 + p.row0, head));
    const uint32_t at = (uint32_t)((32 * wave + (lane & 31)) * a.q.token);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = load_row<T>(r, at, there, kk, lane, a.D);
  }
  TileLoad<ROWB, NW> kload, vload;
  kload.init(wave, lane, a.k.token, a.D * (int)sizeof(T));
  vload.init(wave, lane, a.v.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB> rows;
  ColReader<T, ROWB> cols;
  rows.init(lane);
  cols.init(lane);

  int lo, hi, wlo, whi;                        // keys that the workgroup's and the wave's rows see
  keys_seen(a, p, p.row0, min(p.row0 + BM, p.Lq) - 1, lo, hi);
  keys_seen(a, p, i0, min(i0 + 32, p.Lq) - 1, wlo, whi);
  if (i0 >= p.Lq) whi = -1;
  const int c = i + p.Lk - p.Lq, mylo = max(0, c - a.left), myhi = min(p.Lk - 1, c + a.right);
  // keys that every row of the wave sees
  const int alllo = max(0, min(i0 + 32, p.Lq) - 1 + p.Lk - p.Lq - a.left), allhi = min(p.Lk - 1, i0 + p.Lk - p.Lq + a.right);
  const int first = lo / kTile, last = hi / kTile;
  const bool any = hi >= lo;

  f32x16 acc[NB];
  float m, l;
  auto walk = [&](bool careful) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) zero(acc[blk]);
    m = -kInf; l = 0.0f;
    if (!any) return;
    auto fetch = [&](int t, int stage) {
      unsigned char* s = lds + stage * STAGE;
      kload.load(kbase + (int64_t)t * kTile * a.k.token, p.Lk - t * kTile, s, wave, lane);
      vload.load(vbase + (int64_t)t * kTile * a.v.token, p.Lk - t * kTile, s + kTile * ROWB, wave, lane);
    };
    if (!careful) fetch(first, first & 1);
    for (int t = first; t <= last; ++t) {
      wait_tile();                             // this tile is there, and no wave reads the other stage any more
      if (careful) {
        fetch(t, 0);
        wait_tile();
        copy_finite<T, kTile * ROWB, NW * 64>(lds + kTile * ROWB, lds + STAGE, tid);
        __syncthreads();
      } else if (t < last) {
        fetch(t + 1, t + 1 & 1);
      }
      const int j0 = t * kTile;
      if (j0 > whi || j0 + kTile <= wlo) continue;
      const unsigned char* const kt = lds + (careful ? 0 : (t & 1) * STAGE);
      const unsigned char* const vt = careful ? lds + STAGE : kt + kTile * ROWB;
      f32x16 s[2];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) {
        zero(s[nb]);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) mma(s[nb], rows.read(kt, 32 * nb, kk), q[kk]);
      }
      const bool border = j0 < alllo || j0 + kTile - 1 > allhi;
      if (border) {
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + 32 * nb + 8 * (r >> 2) + 4 * half + (r & 3);
            const bool see = j >= mylo && j <= myhi;
            s[nb][r] = see ? s[nb][r] : -kInf;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[nb][r]);
      top = both_max(top);
      const bool rise = top > m + (float)kPatience / a.c;        // (row by row: no row's rounding depends on another's values)
      if (__any(rise)) {
        const float up = rise ? top : m, f = rise ? __builtin_amdgcn_exp2f((m - up) * a.c) : 1.0f;
        m = up; l *= f;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[blk][r] *= f;
      }
      const float mc = m == -kInf ? 0.0f : m * a.c;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[nb][r] = __builtin_amdgcn_exp2f(fmaf(s[nb][r], a.c, -mc));
          l += s[nb][r];
        }
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const Frag<T> pk = operand<T>(s[nb], kk);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) mma(acc[blk], cols.read(vt, 32 * nb + 16 * kk, blk, lane), pk);
        }
    }
  };
  // a NaN may come from a value that a window hides (0 times what is not finite): once more then, with the tiles on a border taken apart
  bool careful = false;
  for (;;) {
    walk(careful);
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(acc))) break;
    careful = true;
  }
  if (careful && there) spoil<T, NB>(acc, vbase, a.v.token, mylo, myhi, lane, a.D);
  l = both_sum(l);
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  store_rows<T, NB>(rows_of(a.o, p.b, p.q0 + i, head), there, acc, inv, lane, a.D);
  if (there && half == 0) a.lse[stat_row(a, p, head) + i] = l > 0.0f || l != l ? (m * a.c + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
}

// ---- gradient by the queries; D and lse / ln 2 for the pass over the keys ---------------------------------------------------
template <typename T, int NB, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_dq_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), KK = 2 * NB, BM = 32 * NW, STAGE = 2 * kTile * ROWB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  Place p;
  if (!find_place<BM, true>(a, a.G, p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = p.hk * a.G + p.g, half = lane >> 5;
  const int i0 = p.row0 + 32 * wave, i = i0 + (lane & 31);
  const bool there = i < p.Lq;
  const char* const kbase = rows_of(a.k, p.b, p.k0, p.hk);
  const char* const vbase = rows_of(a.v, p.b, p.k0, p.hk);

  Frag<T> q[KK], g[KK];
  float delta = 0.0f;
  {
    const BufRsrc rq = buffer_at(rows_of(a.q, p.b, p.q0 + p.row0, head)), rg = buffer_at(rows_of(a.d_o, p.b, p.q0 + p.row0, head)),
                  ro = buffer_at(rows_of(a.o, p.b, p.q0 + p.row0, head));
    const int row = 32 * wave + (lane & 31);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      q[kk] = load_row<T>(rq, (uint32_t)(row * a.q.token), there, kk, lane, a.D);
      g[kk] = load_row<T>(rg, (uint32_t)(row * a.d_o.token), there, kk, lane, a.D);
      const Frag<T> o = load_row<T>(ro, (uint32_t)(row * a.o.token), there, kk, lane, a.D);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(element(g[kk], j), element(o, j), delta);
    }
  }
  delta = both_sum(delta);
  const int64_t at = stat_row(a, p, head) + i;
  const float lse = there ? a.lse_in[at] : -kInf;
  const float l2 = lse == -kInf ? kInf : lse * kLog2e;            // (a row that sees nothing: no probability)
  if (there && half == 0) { a.stats[at] = l2; a.stats[a.rows + at] = delta; }

  TileLoad<ROWB, NW> kload, vload;
  kload.init(wave, lane, a.k.token, a.D * (int)sizeof(T));
  vload.init(wave, lane, a.v.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB> rows;
  ColReader<T, ROWB> cols;
  rows.init(lane);
  cols.init(lane);

  int lo, hi, wlo, whi;
  keys_seen(a, p, p.row0, min(p.row0 + BM, p.Lq) - 1, lo, hi);
  keys_seen(a, p, i0, min(i0 + 32, p.Lq) - 1, wlo, whi);
  if (i0 >= p.Lq) whi = -1;
  const int c = i + p.Lk - p.Lq, mylo = max(0, c - a.left), myhi = min(p.Lk - 1, c + a.right);
  const int alllo = max(0, min(i0 + 32, p.Lq) - 1 + p.Lk - p.Lq - a.left), allhi = min(p.Lk - 1, i0 + p.Lk - p.Lq + a.right);
  const int first = lo / kTile, last = hi / kTile;
  const bool any = hi >= lo;

  f32x16 acc[NB];
  auto walk = [&](bool careful) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) zero(acc[blk]);
    if (!any) return;
    auto fetch = [&](int t, int stage) {
      unsigned char* s = lds + stage * STAGE;
      kload.load(kbase + (int64_t)t * kTile * a.k.token, p.Lk - t * kTile, s, wave, lane);
      vload.load(vbase + (int64_t)t * kTile * a.v.token, p.Lk - t * kTile, s + kTile * ROWB, wave, lane);
    };
    if (!careful) fetch(first, first & 1);
    for (int t = first; t <= last; ++t) {
      wait_tile();
      if (careful) {
        fetch(t, 0);
        wait_tile();
        copy_finite<T, kTile * ROWB, NW * 64>(lds, lds + STAGE, tid);
        __syncthreads();
      } else if (t < last) {
        fetch(t + 1, t + 1 & 1);
      }
      const int j0 = t * kTile;
      if (j0 > whi || j0 + kTile <= wlo) continue;
      const unsigned char* const kt = lds + (careful ? 0 : (t & 1) * STAGE);
      const unsigned char* const vt = kt + kTile * ROWB;
      const unsigned char* const ct = careful ? lds + STAGE : kt;
      const bool border = j0 < alllo || j0 + kTile - 1 > allhi;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) {
        f32x16 s, dp;
        zero(s);
        zero(dp);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) mma(s, rows.read(kt, 32 * nb, kk), q[kk]);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) mma(dp, rows.read(vt, 32 * nb, kk), g[kk]);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -l2)) * (dp[r] - delta);
        if (border) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + 32 * nb + 8 * (r >> 2) + 4 * half + (r & 3);
            const bool see = j >= mylo && j <= myhi;
            s[r] = see ? s[r] : 0.0f;
          }
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const Frag<T> ds = operand<T>(s, kk);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) mma(acc[blk], cols.read(ct, 32 * nb + 16 * kk, blk, lane), ds);
        }
      }
    }
  };
  bool careful = false;
  for (;;) {
    walk(careful);
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(acc))) break;
    careful = true;
  }
  if (careful && there) spoil<T, NB>(acc, kbase, a.k.token, mylo, myhi, lane, a.D);
  store_rows<T, NB>(rows_of(a.dq, p.b, p.q0 + i, head), there, acc, a.scale, lane, a.D);
}

// ---- gradients by keys and values -------------------------------------------------------------------------------------------
// A wave owns 32 keys, its lanes a key each, and walks over the queries of every head of its group: no sum leaves the workgroup, and the
// order is always the same.
template <typename T, int NB, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_dkv_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), KK = 2 * NB, BN = 32 * NW, TILE = kTile * ROWB, STAGE = 2 * TILE + 2 * kTile * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  Place p;
  if (!find_place<BN, false>(a, 1, p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int j0 = p.row0 + 32 * wave, j = j0 + (lane & 31);
  const bool there = j < p.Lk;

  Frag<T> k[KK], v[KK];
  {
    const BufRsrc rk = buffer_at(rows_of(a.k, p.b, p.k0 + p.row0, p.hk)), rv = buffer_at(rows_of(a.v, p.b, p.k0 + p.row0, p.hk));
    const int row = 32 * wave + (lane & 31);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      k[kk] = load_row<T>(rk, (uint32_t)(row * a.k.token), there, kk, lane, a.D);
      v[kk] = load_row<T>(rv, (uint32_t)(row * a.v.token), there, kk, lane, a.D);
    }
  }
  TileLoad<ROWB, NW> qload, gload;
  qload.init(wave, lane, a.q.token, a.D * (int)sizeof(T));
  gload.init(wave, lane, a.d_o.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB> rows;
  ColReader<T, ROWB> cols;
  rows.init(lane);
  cols.init(lane);

  // query i sees key j from i = j - right - (Lk - Lq) to i = j + left - (Lk - Lq)
  const int ahead = p.Lk - p.Lq;
  const int lo = max(0, p.row0 - a.right - ahead), hi = min(p.Lq - 1, min(p.row0 + BN, p.Lk) - 1 + a.left - ahead);
  const int wlo = max(0, j0 - a.right - ahead), whi = j0 < p.Lk ? min(p.Lq - 1, min(j0 + 32, p.Lk) - 1 + a.left - ahead) : -1;
  const int mylo = max(0, j - a.right - ahead), myhi = min(p.Lq - 1, j + a.left - ahead);
  const int alllo = max(0, min(j0 + 32, p.Lk) - 1 - a.right - ahead), allhi = j0 + a.left - ahead;      // rows behind Lq add nothing anyway
  const int first = lo / kTile, last = hi / kTile, tiles = hi >= lo ? last - first + 1 : 0;

  f32x16 dk[NB], dv[NB];
  auto walk = [&](bool careful) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) { zero(dk[blk]); zero(dv[blk]); }
    const int steps = tiles * a.G;
    if (steps == 0) return;
    int ft = first, fg = 0;                              // the next tile to fetch
    auto fetch = [&](int stage) {
      unsigned char* s = lds + stage * STAGE;
      const int head = p.hk * a.G + fg, row = ft * kTile, left = p.Lq - row;
      qload.load(rows_of(a.q, p.b, p.q0 + row, head), left, s, wave, lane);
      gload.load(rows_of(a.d_o, p.b, p.q0 + row, head), left, s + TILE, wave, lane);
      if (wave == 0) {                                   // rows that are not there: lse 0 and D 0 beside do = 0
        const float* st = a.stats + stat_row(a, p, head) + row;
        const BufRsrc r0 = buffer_at((const char*)st), r1 = buffer_at((const char*)(st + a.rows));
        const int off = lane < left ? lane * 4 : (int)kOob;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r0, (lds_void_ptr)(s + 2 * TILE), 4, off, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r1, (lds_void_ptr)(s + 2 * TILE + kTile * 4), 4, off, 0, 0, 0);
      }
      if (++ft > last) { ft = first; ++fg; }
    };
    if (!careful) fetch(0);
    int t = first;
    for (int n = 0; n < steps; ++n, t = t == last ? first : t + 1) {
      wait_tile();
      if (careful) {
        fetch(0);
        wait_tile();
        copy_finite<T, 2 * TILE, NW * 64>(lds, lds + STAGE, tid);
        __syncthreads();
      } else if (n + 1 < steps) {
        fetch(n + 1 & 1);
      }
      const int i0 = t * kTile;
      if (i0 > whi || i0 + kTile <= wlo) continue;
      const unsigned char* const qt = lds + (careful ? 0 : (n & 1) * STAGE);
      const unsigned char* const gt = qt + TILE;
      const unsigned char* const ct = careful ? lds + STAGE : qt;
      const float* const st = reinterpret_cast<const float*>(qt + 2 * TILE);
      const bool border = i0 < alllo || i0 + kTile - 1 > allhi;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) {
        f32x16 s, dp;
        zero(s);
        zero(dp);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) mma(s, rows.read(qt, 32 * nb, kk), k[kk]);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) mma(dp, rows.read(gt, 32 * nb, kk), v[kk]);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float4 l2 = *reinterpret_cast<const float4*>(st + 32 * nb + 8 * b + 4 * half);
          const float4 de = *reinterpret_cast<const float4*>(st + kTile + 32 * nb + 8 * b + 4 * half);
          const float l4[4] = {l2.x, l2.y, l2.z, l2.w}, d4[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int r = 4 * b + x;
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -l4[x]));
            dp[r] = s[r] * (dp[r] - d4[x]);
          }
        }
        if (border) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int i = i0 + 32 * nb + 8 * (r >> 2) + 4 * half + (r & 3);
            const bool see = i >= mylo && i <= myhi;
            s[r] = see ? s[r] : 0.0f;
            dp[r] = see ? dp[r] : 0.0f;
          }
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const Frag<T> pk = operand<T>(s, kk), ds = operand<T>(dp, kk);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) {
            mma(dv[blk], cols.read(ct + TILE, 32 * nb + 16 * kk, blk, lane), pk);
            mma(dk[blk], cols.read(ct, 32 * nb + 16 * kk, blk, lane), ds);
          }
        }
      }
    }
  };
  bool careful = false;
  for (;;) {
    walk(careful);
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(dk) || any_nan<NB>(dv))) break;
    careful = true;
  }
  if (careful && there)
    for (int g = 0; g < a.G; ++g) {
      spoil<T, NB>(dk, rows_of(a.q, p.b, p.q0, p.hk * a.G + g), a.q.token, mylo, myhi, lane, a.D);
      spoil<T, NB>(dv, rows_of(a.d_o, p.b, p.q0, p.hk * a.G + g), a.d_o.token, mylo, myhi, lane, a.D);
    }
  store_rows<T, NB>(rows_of(a.dk, p.b, p.k0 + j, p.hk), there, dk, a.scale, lane, a.D);
  store_rows<T, NB>(rows_of(a.dv, p.b, p.k0 + j, p.hk), there, dv, 1.0f, lane, a.D);
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
enum { kForward, kGradQ, kGradKV };

// Tiles and items of a launch; false where it has too many.
template <int BM, bool QUERIES> bool plan(AttnArgs& a, int per) {
  const int S = QUERIES ? a.Sq : a.Sk;
  const int64_t tiles = a.off_q ? (int64_t)S / BM + a.B : ((int64_t)S + BM - 1) / BM;
  a.groups = a.off_q ? a.Hkv : a.B * a.Hkv;
  a.rows_per_group = (int)tiles;
  a.items = tiles * a.groups * per;
  // a share of the work for each XCD, whose L2 then holds the keys of few heads; under a window the shares are only alike if each has
  // whole groups
  a.xcd = a.groups % 8 == 0 || (a.left >= kFar && a.right >= kFar);
  return tiles <= INT32_MAX && a.items + 7 <= INT32_MAX;
}

template <typename T, int NB, int NW, int OCC> dat_status launch(int pass, AttnArgs a, hipStream_t st) {
  constexpr int BM = 32 * NW;
  if (!(pass == kGradKV ? plan<BM, false>(a, 1) : plan<BM, true>(a, a.G)) || !fits_launch(a.items + 7, NW * 64)) return DAT_ERR_SHAPE;
  if (a.items == 0) return DAT_OK;
  const dim3 grid((unsigned)(a.xcd ? (a.items + 7) / 8 * 8 : a.items)), block(NW * 64);
  if (pass == kForward) hipLaunchKernelGGL((attn_fwd_kernel<T, NB, NW, OCC>), grid, block, 0, st, a);
  else if (pass == kGradQ) hipLaunchKernelGGL((attn_dq_kernel<T, NB, NW, OCC>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((attn_dkv_kernel<T, NB, NW, OCC>), grid, block, 0, st, a);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

template <typename T> dat_status launch_heads(int pass, const AttnArgs& a, hipStream_t st) {
  switch ((a.D + 31) / 32) {
    case 1: return launch<T, 1, 4, 2>(pass, a, st);
    case 2: return launch<T, 2, 4, 2>(pass, a, st);
    case 3: return launch<T, 3, 4, 1>(pass, a, st);
    default: return launch<T, 4, 4, 1>(pass, a, st);
  }
}

bool fill(const dat_attention* s, AttnArgs& a, dat_status& status) {
  status = DAT_ERR_ARG;
  if (!s || (s->dtype != DAT_F32 && s->dtype != DAT_BF16) || s->B < 0 || s->Sq < 0 || s->Sk < 0 || s->H < 1 || s->Hkv < 1 || s->H % s->Hkv || s->D < 1) return false;
  if (!(s->scale > 0.0f) || !(s->scale < kInf) || !(s->scale * kLog2e < kInf) || s->left < -1 || s->right < -1) return false;
  if (!s->offsets_q != !s->offsets_k || !aligned(s->offsets_q, 4) || !aligned(s->offsets_k, 4)) return false;
  status = DAT_ERR_SHAPE;
  if (s->D % 8 || s->D > 128 || s->Sq >= kFar || s->Sk >= kFar) return false;
  const int64_t batches = s->offsets_q ? 1 : s->B;
  if (batches * s->H * (int64_t)s->Sq >= (int64_t)1 << 40 || (int64_t)s->B * s->Hkv > INT32_MAX) return false;
  a.off_q = s->offsets_q; a.off_k = s->offsets_k;
  a.B = s->B; a.Sq = s->Sq; a.Sk = s->Sk; a.H = s->H; a.Hkv = s->Hkv; a.G = s->H / s->Hkv; a.D = s->D;
  a.left = s->left < 0 ? kFar : s->left < kFar ? s->left : kFar;
  a.right = s->right < 0 ? kFar : s->right < kFar ? s->right : kFar;
  a.scale = s->scale; a.c = s->scale * kLog2e;
  a.rows = batches * s->H * (int64_t)s->Sq;
  status = DAT_OK;
  return true;
}

// Checks a tensor and turns its strides into bytes.
dat_status take(const dat_heads* t, const HeadsShape& s, size_t width, bool output, HeadsArg& out) {
  if (!t) return DAT_ERR_ARG;
  if (s.batch * s.tokens * s.heads == 0) { out = HeadsArg{(char*)t->data, 0, 0, 0}; return DAT_OK; }
  if (!heads_vectors(*t, s, width) || (output && !heads_dims(*t, s).apart)) return DAT_ERR_ARG;
  const int64_t w = (int64_t)width, token = s.tokens > 1 ? t->token * w : 0;
  if (token >= (int64_t)1 << 23) return DAT_ERR_SHAPE;             // the offsets in a tile of up to 256 rows are 31 bits
  out = HeadsArg{(char*)t->data, s.batch > 1 ? t->batch * w : 0, token, s.heads > 1 ? t->head * w : 0};
  return DAT_OK;
}

struct Tensor { const dat_heads* t; HeadsShape s; HeadsArg* to; bool output; };

dat_status take_all(std::initializer_list<Tensor> list, size_t width) {
  for (const Tensor& x : list) {
    const dat_status st = take(x.t, x.s, width, x.output, *x.to);
    if (st != DAT_OK) return st;
  }
  for (const Tensor& x : list)
    if (x.output)
      for (const Tensor& y : list) if (&x != &y && heads_overlap(*x.t, x.s, *y.t, y.s, width)) return DAT_ERR_ARG;
  return DAT_OK;
}

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" dat_status dat_attention_forward(const dat_attention* shape, const dat_heads* q, const dat_heads* k, const dat_heads* v,
                                            const dat_heads* o, float* lse, void* stream) {
  AttnArgs a{};
  dat_status st;
  if (!fill(shape, a, st)) return st;
  const int64_t B = a.off_q ? (a.B > 0) : a.B;
  const HeadsShape sq{B, a.Sq, a.H, a.D}, sk{B, a.Sk, a.Hkv, a.D};
  const size_t width = shape->dtype == DAT_BF16 ? 2 : 4;
  st = take_all(std::initializer_list<Tensor>{{q, sq, &a.q, false}, {k, sk, &a.k, false}, {v, sk, &a.v, false}, {o, sq, &a.o, true}}, width);
  if (st != DAT_OK) return st;
  if (B == 0 || a.Sq == 0) return DAT_OK;
  if (!lse || !aligned(lse, 4)) return DAT_ERR_ARG;
  a.lse = lse;
  return width == 2 ? launch_heads<bf16_t>(kForward, a, (hipStream_t)stream) : launch_heads<float>(kForward, a, (hipStream_t)stream);
}

extern "C" size_t dat_attention_workspace(int pass, const dat_attention* shape) {
  AttnArgs a{};
  dat_status st;
  if (!fill(shape, a, st) || pass != 1) return 0;
  return (size_t)(2 * a.rows * 4 + 15) / 16 * 16;
}

extern "C" dat_status dat_attention_backward(const dat_attention* shape, const dat_heads* q, const dat_heads* k, const dat_heads* v,
                                             const dat_heads* o, const float* lse, const dat_heads* d_o, const dat_heads* dq,
                                             const dat_heads* dk, const dat_heads* dv, void* workspace, size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  dat_status st;
  if (!fill(shape, a, st)) return st;
  const int64_t B = a.off_q ? (a.B > 0) : a.B;
  const HeadsShape sq{B, a.Sq, a.H, a.D}, sk{B, a.Sk, a.Hkv, a.D};
  const size_t width = shape->dtype == DAT_BF16 ? 2 : 4;
  st = take_all(std::initializer_list<Tensor>{{q, sq, &a.q, false}, {k, sk, &a.k, false}, {v, sk, &a.v, false}, {o, sq, &a.o, false}, {d_o, sq, &a.d_o, false},
                                              {dq, sq, &a.dq, true}, {dk, sk, &a.dk, true}, {dv, sk, &a.dv, true}}, width);
  if (st != DAT_OK) return st;
  if (B == 0) return DAT_OK;
  if (a.Sq > 0) {
    if (!lse || !aligned(lse, 4) || !workspace || !aligned(workspace, 16) || workspace_bytes < dat_attention_workspace(1, shape)) return DAT_ERR_ARG;
    a.lse_in = lse;
    a.stats = (float*)workspace;
    st = width == 2 ? launch_heads<bf16_t>(kGradQ, a, (hipStream_t)stream) : launch_heads<float>(kGradQ, a, (hipStream_t)stream);
    if (st != DAT_OK) return st;
  }
  if (a.Sk == 0) return DAT_OK;
  return width == 2 ? launch_heads<bf16_t>(kGradKV, a, (hipStream_t)stream) : launch_heads<float>(kGradKV, a, (hipStream_t)stream);
}
