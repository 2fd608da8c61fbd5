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
//
// Bound by the matrix cores and the vector instructions of the softmax beside them: 64 keys for 32 queries are 32 products of 32 cycles at D = 128
// and about 150 vector instructions, a third of them exponentials and their arguments (at D = 64 16 products, and the vector work is the
// longer).  The waves of different workgroups on a SIMD fill each other's gaps; inside a wave fragments are read ahead of their
// products.  Memory: a tile of 64 rows comes in once for 128 rows of the result, 4 to 5 TB/s out of the L2s, and nothing of S x S size is
// written.  Measured over several cards, operations that the mask leaves: forward 1 x 8192 tokens, 32 heads of 128 on 8, causal 497 to 525 us (1107 to
// 1047 TFLOP/s; a plain product of 8192^3 reaches 1216 here); 32 x 1024 tokens, 16 heads of 64 188 us (730); 2 x 4096 tokens 165 us (833).
// bf16 calls round P and dS to bf16 where they enter a product (fp32 ones run at an eighth of the rate): outputs are then 2.1e-3 to 2.5e-3 of their norm
// off, where the one rounding at the end leaves 1.7e-3.  Nothing else is rounded to less than fp32.
// Why 32 rows a wave and 128 a workgroup: 64 rows a wave halve the reads of LDS, but need 512 registers, one wave a SIMD (causal
// 302 -> 392 us at 32 x 1024 x 16 x 128); 256 rows a workgroup (8 waves) 504 -> 493 us on the 8192 tokens, slower on all shorter ones.
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
typedef __amdgpu_buffer_rsrc_t BufRsrc;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff(), kLargest = 0x1.fffffep127f;
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
  int parts;                                             // workgroups that share the walk of a tile
  int items;
  int64_t rows, key_rows;                                // rows = B * H * Sq (H * Sq packed), key_rows = B * Hkv * Sk
  float* part;                                           // their results in fp32: [parts][rows][D], then [parts][rows][2] (forward: m c and l)
};

// One tile of a result: sequence, heads and rows.
struct Place { int b, hk, g, part, row0, q0, k0, Lq, Lk; };

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
  uint32_t item = blockIdx.x;
  if (a.xcd) item = (blockIdx.x & 7) * (((uint32_t)a.items + 7) >> 3) + (blockIdx.x >> 3);
  if (item >= (uint32_t)a.items) return false;
  const int each = per * a.parts, t = (int)(item / (uint32_t)each), within = (int)item - t * each;
  p.g = (uint32_t)within / (uint32_t)a.parts;
  p.part = within - p.g * a.parts;
  const int group = (int)((uint32_t)t / (uint32_t)a.rows_per_group);
  int tile = a.rows_per_group - 1 - (t - group * a.rows_per_group);
  if (!QUERIES) tile = t - group * a.rows_per_group;      // early keys are seen by the most queries
  if (a.off_q) {
    p.hk = group;
    const int32_t* off = QUERIES ? a.off_q : a.off_k;
    const int T = QUERIES ? a.Sq : a.Sk;
    int lo = 0, hi = a.B;                                // the last sequence whose first slot is not behind the tile's: the lanes try 64 places at once
    while (hi - lo > 1) {
      const int stride = (hi - lo + 63) >> 6, at = lo + (int)(threadIdx.x & 63) * stride;
      const uint64_t before = __ballot(at < hi && clampi(off[min(at, hi - 1)], 0, T) / BM + at <= tile);
      lo += max(__popcll(before) - 1, 0) * stride;
      hi = min(lo + stride, hi);
    }
    p.b = lo;
    sequence(a.off_q, p.b, a.Sq, p.q0, p.Lq);
    sequence(a.off_k, p.b, a.Sk, p.k0, p.Lk);
    const int j = tile - ((QUERIES ? p.q0 : p.k0) / BM + p.b);
    if (j < 0 || (int64_t)j * BM >= (QUERIES ? p.Lq : p.Lk)) return false;
    p.row0 = j * BM;
  } else {
    p.b = (int)((uint32_t)group / (uint32_t)a.Hkv);
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
__device__ __forceinline__ int64_t key_row(const AttnArgs& a, const Place& p) {
  return a.off_q ? (int64_t)p.hk * a.Sk + p.k0 : ((int64_t)p.b * a.Hkv + p.hk) * a.Sk;
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

__device__ __forceinline__ u32x4 descriptor(const char* p) {      // (buffer_at's, as four dwords)
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, 0x80000000u, 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_at(const unsigned char* p) { return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char*)p); }

// Loads straight into LDS, lane l's bytes at `to` + l * BYTES.  Written as one asm statement because the compiler otherwise waits for all such
// loads in flight before the next LDS read, the next tile's too; wait_tile() waits for them.  M0 (which the compiler reserves: no list of
// overwritten registers holds it) is left as it was.  The instructions before the load give a descriptor just written by a vector instruction
// the five wait states that it needs, and M0 the one.
template <int BYTES> __device__ __forceinline__ void load_to_lds(const u32x4& d, uint32_t off, uint32_t to) {
  static_assert(BYTES == 4 || BYTES == 16, "one or four dwords a lane");
  uint32_t m0;
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 2\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n\ts_mov_b32 m0, %0" : "=&s"(m0) : "v"(off), "s"(d), "s"(to) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 2\n\tbuffer_load_dword %1, %2, 0 offen lds\n\ts_mov_b32 m0, %0" : "=&s"(m0) : "v"(off), "s"(d), "s"(to) : "memory");
}

// ---- LDS tiles ---------------------------------------------------------------------------------------------------------------
// A tile holds kTile rows of a head as they are in memory (what lies between D and 32 NB is zero), their 16-byte slots permuted: slot s of row r
// is at s ^ flip(r).  The 16 rows that a row fragment's read takes at once then lie in 16 different places of the 256 bytes that the banks
// cover, and so do the 64 bytes of each of four consecutive rows that half a wave's transposing read takes.
template <int ROWB> __device__ __forceinline__ int flip(int r) {
  constexpr int apart = ROWB / 16 % 16;            // from row to row, in slots, around the banks
  if (apart == 4 || apart == 12) return r >> 2 & 3;                                                   // every fourth row on the same place
  if (apart == 8) return ROWB == 128 ? ((r >> 1 & 1) << 2) | ((r >> 2 & 1) << 1) | (r >> 3 & 1) : r >> 1 & 7;  // every other one
  return ROWB == 256 ? ((r & 3) << 2) | (r >> 2 & 3) : r & 15;
}

// Loads of a tile straight into LDS: a wave's instruction fills 1 KB, the lane that fills slot p of row r fetches slot p ^ flip(r).
template <int ROWB, int NW> struct TileLoad {
  static constexpr int NS = ROWB / 16, N = kTile * NS / 64 / NW;
  static_assert(kTile * NS % (64 * NW) == 0, "whole instructions of every wave");
  uint32_t off[N];
  __device__ __forceinline__ static int row(int i, int wave, int lane) { return (uint32_t)((i * NW + wave) * 64 + lane) / (uint32_t)NS; }
  __device__ __forceinline__ void init(int wave, int lane, int64_t stride, int row_bytes) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i, wave, lane), slot = ((i * NW + wave) * 64 + lane - r * NS) ^ flip<ROWB>(r);
      off[i] = slot * 16 < row_bytes ? (uint32_t)r * (uint32_t)stride + slot * 16 : kOob;
    }
  }
  __device__ __forceinline__ void load(const char* base, int rows, uint32_t tile, int wave, int lane) const {
    const u32x4 r = descriptor(base);
    if (rows >= kTile) {                       // (a branch of its own: no comparisons for whole tiles)
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds<16>(r, off[i], tile + (i * NW + wave) * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds<16>(r, row(i, wave, lane) < rows ? off[i] : kOob, tile + (i * NW + wave) * 1024);
    }
  }
};

// Readers hold LDS addresses, one for each k-step or block (the permutation is an XOR, which no offset can stand in for); the stage, the
// tile and the rows go into the instruction's offset.
template <typename V> __device__ __forceinline__ V lds_read(uint32_t at, int offset) {
  return *((__attribute__((address_space(3))) const V*)(uintptr_t)(at + (uint32_t)offset));
}

// Row fragment: elements 16 kk + 8 (lane / 32) .. + 7 of the row lane % 32 behind `offset`.
template <typename T, int ROWB, int KK> struct RowReader {
  uint32_t at[KK];
  __device__ __forceinline__ void init(uint32_t lds, int lane) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      at[kk] = lds + (lane & 31) * ROWB + ((flip<ROWB>(lane & 31) << 4) ^ ((lane >> 5) * 8 * (int)sizeof(T)) ^ (kk * 16 * (int)sizeof(T)));
  }
  __device__ __forceinline__ Frag<T> read(int offset, int kk) const {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      f.u = lds_read<u32x4>(at[kk], offset);
    } else {
      const u32x4 a = lds_read<u32x4>(at[kk], offset), b = lds_read<u32x4>(at[kk] ^ 16, offset);
#pragma unroll
      for (int j = 0; j < 4; ++j) { f.f[j] = __uint_as_float(a[j]); f.f[4 + j] = __uint_as_float(b[j]); }
    }
    return f;
  }
};

// Transposed fragment: element 32 blk + lane % 32 of the rows 4 h + 0..3 and 8 + 4 h + 0..3 (h = lane / 32) behind `offset` (a multiple of
// 16 rows, which leaves the permutation as it is).  bf16: inside every group of 16 lanes the transposing read hands lane i element i % 4 of
// the 8-byte chunks named by lanes i / 4 + 0, 4, 8, 12.
template <typename T, int ROWB, int NB> struct ColReader {
  uint32_t at[2][sizeof(T) == 2 ? NB : 4];
  __device__ __forceinline__ void init(uint32_t lds, int lane) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (sizeof(T) == 2) {
        const int g = lane >> 4, s = lane & 15, r = 8 * e + 4 * (g >> 1) + (s >> 2);
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) at[e][blk] = lds + r * ROWB + ((flip<ROWB>(r) << 4) ^ ((g & 1) * 32 + (s & 3) * 8) ^ (blk * 64));
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = 8 * e + 4 * (lane >> 5) + x;
          at[e][x] = lds + r * ROWB + ((((lane & 31) >> 2) ^ flip<ROWB>(r)) << 4) + (lane & 3) * 4;
        }
      }
    }
  }
  __device__ __forceinline__ void shift(int by) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 0; x < (sizeof(T) == 2 ? NB : 4); ++x) at[e][x] += by;
  }
  __device__ __forceinline__ Frag<T> read(int offset, int blk) const {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s16*)(uintptr_t)(at[e][blk] + (uint32_t)offset)));
        f.u[2 * e] = y[0]; f.u[2 * e + 1] = y[1];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {           // (rows of 384 bytes: the permutation stays within 128, and the rows do not begin at multiples of 256)
        const uint32_t row = at[j >> 2][j & 3];
        f.f[j] = lds_read<float>(ROWB == 384 ? row + blk * 128 : row ^ (blk * 128), offset);
      }
    }
    return f;
  }
};

// Fragments that are read ahead of their use (the matrix cores are busy 32 cycles with a bf16 product, 512 with an fp32 one; an LDS read
// takes over a hundred).
template <typename T> constexpr int fragments_ahead() { return sizeof(T) == 2 ? 8 : 2; }

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
// The loads of a wave's own rows, waited for once: where the compiler does not see them done before the loop it waits for them in there, and for
// the tiles in flight with them.
__device__ __forceinline__ void wait_own() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void wait_tile() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");               // (the barrier alone does not hold reads of LDS back)
}

template <int N> struct Stage { static constexpr int value = N; };
template <typename T, int NB> constexpr int row_bytes() { return 32 * NB * (int)sizeof(T); }

// ---- the walk along a tile's other axis --------------------------------------------------------------------------------------
// Two stages of LDS: while the waves compute on one, the other fills.  step(stage, n) computes tile n of the walk from a stage known at
// compile time; fetch(n, stage) loads it.  Careful: every tile into the first stage, copy() makes the finite copy of it in the
// second, and the columns are read from there.
template <typename F, typename S, typename C> __device__ __forceinline__ void walk_tiles(int from, int to, bool careful, F fetch, S step, C copy) {
  for (int n = from; n < to;) {
    wait_tile();                               // this tile is there, and no wave reads the other stage any more
    if (careful) {
      fetch(n, 0);
      wait_tile();
      copy();
      __syncthreads();
    } else if (n + 1 < to) {
      fetch(n + 1, 1);
    }
    step(Stage<0>{}, n);
    ++n;
    if (careful || n >= to) continue;
    wait_tile();
    if (n + 1 < to) fetch(n + 1, 0);
    step(Stage<1>{}, n);
    ++n;
  }
}
__device__ __forceinline__ int share(int n, int part, int parts) { return parts == 1 ? n * part : (int)((int64_t)n * part / parts); }

// ---- forward -----------------------------------------------------------------------------------------------------------------
// The running maximum m (in scores) is raised only where one passes it by kPatience / c: what is summed then stays below 2^kPatience
// times the sum that the true maximum would give, and few tiles rescale the accumulators.
// A tile costs a wave, at D = 128, 16 + 16 products, 32 exponentials and the reads of 32 KB from LDS.  Timing with parts left out (32 x 1024 tokens,
// 16 heads of 128): 311 us; without the tiles' loads 256, without the fragments' reads 276, without both 212.
template <typename T, int NB, int KK, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_fwd_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), BM = 32 * NW, TILE = kTile * ROWB, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  Place p;
  if (!find_place<BM, true>(a, a.G, p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = p.hk * a.G + p.g, half = lane >> 5;
  const int i0 = p.row0 + 32 * wave, i = i0 + (lane & 31);
  const bool there = i < p.Lq;
  const char* const kbase = rows_of(a.k, p.b, p.k0, p.hk);
  const char* const vbase = rows_of(a.v, p.b, p.k0, p.hk);

  TileLoad<ROWB, NW> kload, vload;
  kload.init(wave, lane, a.k.token, a.D * (int)sizeof(T));
  vload.init(wave, lane, a.v.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB, KK> rows;
  ColReader<T, ROWB, NB> cols;
  rows.init(lds_at(lds), lane);
  cols.init(lds_at(lds) + TILE, lane);

  int lo, hi, wlo, whi;                        // keys that the workgroup's and the wave's rows see
  keys_seen(a, p, p.row0, min(p.row0 + BM, p.Lq) - 1, lo, hi);
  keys_seen(a, p, i0, min(i0 + 32, p.Lq) - 1, wlo, whi);
  if (i0 >= p.Lq) whi = -1;
  const int c = i + p.Lk - p.Lq, mylo = max(0, c - a.left), myhi = min(p.Lk - 1, c + a.right);
  // keys that every row of the wave sees
  const int alllo = max(0, min(i0 + 32, p.Lq) - 1 + p.Lk - p.Lq - a.left), allhi = min(p.Lk - 1, i0 + p.Lk - p.Lq + a.right);
  const int tile0 = lo / kTile, tiles = hi >= lo ? hi / kTile - tile0 + 1 : 0;
  const int from = tile0 + share(tiles, p.part, a.parts), to = tile0 + share(tiles, p.part + 1, a.parts);

  auto fetch = [&](int t, int stage) {
    const uint32_t s = lds_at(lds) + stage * STAGE;
    kload.load(kbase + (int64_t)t * kTile * a.k.token, p.Lk - t * kTile, s, wave, lane);
    vload.load(vbase + (int64_t)t * kTile * a.v.token, p.Lk - t * kTile, s + TILE, wave, lane);
  };
  if (from < to) fetch(from, 0);               // under way while the wave's own rows come
  Frag<T> q[KK];
  {
    const BufRsrc r = buffer_at(rows_of(a.q, p.b, p.q0 + p.row0, head));
    const uint32_t at = (uint32_t)(32 * wave + (lane & 31)) * (uint32_t)a.q.token;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = load_row<T>(r, at, there, kk, lane, a.D);
  }
  wait_own();

  f32x16 acc[NB];
  float m, l;
  const float patience = fminf((float)kPatience / a.c, kLargest);   // finite: m rises from -inf at any scale
  auto step = [&](auto stage, int t) {
    constexpr int AT = decltype(stage)::value * STAGE;
    const int j0 = t * kTile;
    if (j0 > whi || j0 + kTile <= wlo) return;
    f32x16 s[2];
    Frag<T> buf[fragments_ahead<T>()];
    // the keys' rows (block nb, k-step kk), then the values' columns (16 keys, block blk): the first of these are read under the
    // last products of the scores and are there when the exponentials are
    constexpr int NK = 2 * KK, NV = 4 * NB, ALL = NK + NV, P = fragments_ahead<T>();
    auto fragment = [&](int n) {
      return n < NK ? rows.read(AT + 32 * (n / KK) * ROWB, n % KK) : cols.read(AT + 16 * ((n - NK) / NB) * ROWB, (n - NK) % NB);
    };
#pragma unroll
    for (int n = 0; n < P; ++n) if (n < ALL) buf[n] = fragment(n);
    zero(s[0]);
    zero(s[1]);
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      mma(s[n / KK], buf[n % P], q[n % KK]);
      if (n + P < ALL) buf[n % P] = fragment(n + P);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (j0 < alllo || j0 + kTile - 1 > allhi) {
      const int first = mylo - j0 - 4 * half, behind = myhi - j0 - 4 * half;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = 32 * nb + 8 * (r >> 2) + (r & 3);
          s[nb][r] = j >= first && j <= behind ? s[nb][r] : -kInf;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[nb][r]);
    top = both_max(top);
    const bool rise = top > m + patience;      // (row by row: no row's rounding depends on another's values)
    if (__any(rise)) {
      const float up = rise ? top : m, f = rise ? __builtin_amdgcn_exp2f((m - up) * a.c) : 1.0f;
      m = up; l *= f;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[blk][r] *= f;
    }
    const float mc = m == -kInf ? 0.0f : m * a.c;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[nb][r] = __builtin_amdgcn_exp2f(fmaf(s[nb][r], a.c, -mc));
        sum[r & 1] += s[nb][r];
      }
    l += sum[0] + sum[1];
    Frag<T> pk;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if (n % NB == 0) pk = operand<T>(s[n / NB / 2], n / NB % 2);
      mma(acc[n % NB], buf[(NK + n) % P], pk);
      if (n + P < NV) buf[(NK + n) % P] = fragment(NK + n + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // a NaN may come from a value that a window hides (0 times what is not finite): once more then, with the values' finite copy
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) zero(acc[blk]);
    m = -kInf; l = 0.0f;
    walk_tiles(from, to, careful, fetch, step, [&] { copy_finite<T, TILE, NW * 64>(lds + TILE, lds + STAGE + TILE, tid); });
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(acc))) break;
    careful = true;
    cols.shift(STAGE);
  }
  if (careful && there) spoil<T, NB>(acc, vbase, a.v.token, max(mylo, from * kTile), min(myhi, to * kTile - 1), lane, a.D);
  l = both_sum(l);
  const int64_t at = stat_row(a, p, head) + i;
  if (a.parts > 1) {
    const int64_t row = p.part * a.rows + at;
    store_rows<float, NB>((char*)(a.part + row * a.D), there, acc, 1.0f, lane, a.D);
    if (there && half == 0) {
      float* const ml = a.part + a.parts * a.rows * a.D + 2 * row;
      ml[0] = m * a.c; ml[1] = l;
    }
    return;
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  store_rows<T, NB>(rows_of(a.o, p.b, p.q0 + i, head), there, acc, inv, lane, a.D);
  if (there && half == 0) a.lse[at] = l > 0.0f || l != l ? (m * a.c + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
}

// ---- gradient by the queries; -D and lse / ln 2 for the pass over the keys --------------------------------------------------
// The rows of o and d_o are here anyway, so D is made here and no launch of its own reads them.  Three products a pair of tiles; keys by halves of a
// tile, which needs 32 registers less than both at once and leaves room for two or three workgroups a compute unit.  2 x 6001 tokens, 16
// heads of 128 on 4, causal: 397 to 419 us, 1110 to 1050 TFLOP/s, matrix cores busy 54 to 57 % of the time; 32 x 577 tokens, 16 heads of 64: 93 to 100 us, 700 to
// 650 TFLOP/s (640 keys in tiles for 577).
// (A half tile that no row sees left out: 1112 -> 1147 us for the whole gradient, the test breaks the order of the loads.)
template <typename T, int NB, int KK, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_dq_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), BM = 32 * NW, TILE = kTile * ROWB, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];
  Place p;
  if (!find_place<BM, true>(a, a.G, p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = p.hk * a.G + p.g, half = lane >> 5;
  const int i0 = p.row0 + 32 * wave, i = i0 + (lane & 31);
  const bool there = i < p.Lq;
  const char* const kbase = rows_of(a.k, p.b, p.k0, p.hk);
  const char* const vbase = rows_of(a.v, p.b, p.k0, p.hk);

  TileLoad<ROWB, NW> kload, vload;
  kload.init(wave, lane, a.k.token, a.D * (int)sizeof(T));
  vload.init(wave, lane, a.v.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB, KK> rows;
  ColReader<T, ROWB, NB> cols;
  rows.init(lds_at(lds), lane);
  cols.init(lds_at(lds), lane);

  int lo, hi, wlo, whi;
  keys_seen(a, p, p.row0, min(p.row0 + BM, p.Lq) - 1, lo, hi);
  keys_seen(a, p, i0, min(i0 + 32, p.Lq) - 1, wlo, whi);
  if (i0 >= p.Lq) whi = -1;
  const int c = i + p.Lk - p.Lq, mylo = max(0, c - a.left), myhi = min(p.Lk - 1, c + a.right);
  const int alllo = max(0, min(i0 + 32, p.Lq) - 1 + p.Lk - p.Lq - a.left), allhi = min(p.Lk - 1, i0 + p.Lk - p.Lq + a.right);
  const int tile0 = lo / kTile, tiles = hi >= lo ? hi / kTile - tile0 + 1 : 0;
  const int from = tile0 + share(tiles, p.part, a.parts), to = tile0 + share(tiles, p.part + 1, a.parts);

  auto fetch = [&](int t, int stage) {
    const uint32_t s = lds_at(lds) + stage * STAGE;
    kload.load(kbase + (int64_t)t * kTile * a.k.token, p.Lk - t * kTile, s, wave, lane);
    vload.load(vbase + (int64_t)t * kTile * a.v.token, p.Lk - t * kTile, s + TILE, wave, lane);
  };
  if (from < to) fetch(from, 0);
  Frag<T> q[KK], g[KK];
  float delta = 0.0f;
  {
    const BufRsrc rq = buffer_at(rows_of(a.q, p.b, p.q0 + p.row0, head)), rg = buffer_at(rows_of(a.d_o, p.b, p.q0 + p.row0, head)),
                  ro = buffer_at(rows_of(a.o, p.b, p.q0 + p.row0, head));
    const int row = 32 * wave + (lane & 31);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      q[kk] = load_row<T>(rq, (uint32_t)row * (uint32_t)a.q.token, there, kk, lane, a.D);
      g[kk] = load_row<T>(rg, (uint32_t)row * (uint32_t)a.d_o.token, there, kk, lane, a.D);
      const Frag<T> o = load_row<T>(ro, (uint32_t)row * (uint32_t)a.o.token, there, kk, lane, a.D);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(element(g[kk], j), element(o, j), delta);
    }
  }
  delta = both_sum(delta);
  const int64_t at = stat_row(a, p, head) + i;
  const float lse = there ? a.lse_in[at] : -kInf;
  const float l2 = lse == -kInf ? kInf : lse * kLog2e;            // (a row that sees nothing: no probability)
  if (there && half == 0 && p.part == 0) { a.stats[at] = l2; a.stats[a.rows + at] = -delta; }
  wait_own();

  f32x16 acc[NB];
  auto step = [&](auto stage, int t) {
    constexpr int AT = decltype(stage)::value * STAGE;
    const int j0 = t * kTile;
    if (j0 > whi || j0 + kTile <= wlo) return;
    const bool border = j0 < alllo || j0 + kTile - 1 > allhi;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      f32x16 s, dp;
      Frag<T> buf[fragments_ahead<T>()];
      // rows of the keys, rows of the values, columns of the keys
      constexpr int N1 = 2 * KK, N2 = 2 * NB, ALL = N1 + N2, P = fragments_ahead<T>();
      auto fragment = [&](int n) {
        return n < N1 ? rows.read(AT + (n < KK ? 0 : TILE) + 32 * nb * ROWB, n % KK) : cols.read(AT + (32 * nb + 16 * ((n - N1) / NB)) * ROWB, (n - N1) % NB);
      };
#pragma unroll
      for (int n = 0; n < P; ++n) if (n < ALL) buf[n] = fragment(n);
      zero(s);
      zero(dp);
  #pragma unroll
      for (int n = 0; n < N1; ++n) {
        if (n < KK) mma(s, buf[n % P], q[n]); else mma(dp, buf[n % P], g[n - KK]);
        if (n + P < ALL) buf[n % P] = fragment(n + P);
        __builtin_amdgcn_sched_barrier(0);
      }
  #pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -l2)) * (dp[r] - delta);
      if (border) {
        const int first = mylo - j0 - 4 * half, behind = myhi - j0 - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = 32 * nb + 8 * (r >> 2) + (r & 3);
          s[r] = j >= first && j <= behind ? s[r] : 0.0f;
        }
      }
      Frag<T> ds;
  #pragma unroll
      for (int n = 0; n < N2; ++n) {
        if (n % NB == 0) ds = operand<T>(s, n / NB);
        mma(acc[n % NB], buf[(N1 + n) % P], ds);
        if (n + P < N2) buf[(N1 + n) % P] = fragment(N1 + n + P);
        __builtin_amdgcn_sched_barrier(0);
      }
      }
  };
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) zero(acc[blk]);
    walk_tiles(from, to, careful, fetch, step, [&] { copy_finite<T, TILE, NW * 64>(lds, lds + STAGE, tid); });
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(acc))) break;
    careful = true;
    cols.shift(STAGE);
  }
  if (careful && there) spoil<T, NB>(acc, kbase, a.k.token, max(mylo, from * kTile), min(myhi, to * kTile - 1), lane, a.D);
  const float factor = mylo == myhi ? 0.0f : a.scale;             // the softmax of one score has no gradient, and what rounding leaves of dP - D is none
  if (a.parts > 1) store_rows<float, NB>((char*)(a.part + (p.part * a.rows + at) * a.D), there, acc, factor, lane, a.D);
  else store_rows<T, NB>(rows_of(a.dq, p.b, p.q0 + i, head), there, acc, factor, lane, a.D);
}

// ---- gradients by keys and values -------------------------------------------------------------------------------------------
// A wave owns 32 keys, its lanes a key each, and walks over the queries of every head of its group: no sum leaves the workgroup (or the
// parts, which are added in their order), and the order is always the same.
// Four products a pair of tiles; two accumulators and two own operands of 128 elements take 192 of the 512 registers that one wave a SIMD
// has at D > 64, so little runs beside its vector work, waits and barriers: 2 x 6001 tokens as above 650 to 737 us by card and clock, 900 to 800 TFLOP/s,
// matrix cores busy 37 % of the time; 32 x 577 tokens, 16 heads of 64, two waves a SIMD: 122 to 141 us, 715 to 620 TFLOP/s.  Forming one block's probabilities
// under the other's products gave 2 % there and lost 20 % at D = 64 (registers); more fragments ahead gave nothing.
template <typename T, int NB, int KK, int NW, int OCC>
__global__ __launch_bounds__(NW * 64, OCC) void attn_dkv_kernel(AttnArgs a) {
  constexpr int ROWB = row_bytes<T, NB>(), BN = 32 * NW, TILE = kTile * ROWB, STATS = 2 * TILE, STAGE = STATS + 2 * kTile * 4;
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
      k[kk] = load_row<T>(rk, (uint32_t)row * (uint32_t)a.k.token, there, kk, lane, a.D);
      v[kk] = load_row<T>(rv, (uint32_t)row * (uint32_t)a.v.token, there, kk, lane, a.D);
    }
  }
  wait_own();
  TileLoad<ROWB, NW> qload, gload;
  qload.init(wave, lane, a.q.token, a.D * (int)sizeof(T));
  gload.init(wave, lane, a.d_o.token, a.D * (int)sizeof(T));
  RowReader<T, ROWB, KK> rows;
  ColReader<T, ROWB, NB> cols;
  rows.init(lds_at(lds), lane);
  cols.init(lds_at(lds), lane);
  const uint32_t stats_at = lds_at(lds) + STATS + 16 * half;

  // query i sees key j from i = j - right - (Lk - Lq) to i = j + left - (Lk - Lq)
  const int ahead = p.Lk - p.Lq;
  const int lo = max(0, p.row0 - a.right - ahead), hi = min(p.Lq - 1, min(p.row0 + BN, p.Lk) - 1 + a.left - ahead);
  const int wlo = max(0, j0 - a.right - ahead), whi = j0 < p.Lk ? min(p.Lq - 1, min(j0 + 32, p.Lk) - 1 + a.left - ahead) : -1;
  const int mylo = max(0, j - a.right - ahead), myhi = min(p.Lq - 1, j + a.left - ahead);
  // Rows between these see every key of the wave and no row that sees one key alone is among them: query -right - ahead sees key 0 alone and no
  // other key of that wave; where left = 0 the last query sees the last key alone, which may be its wave's only one.
  const int alllo = max(0, min(j0 + 32, p.Lk) - 1 - a.right - ahead), allhi = min(p.Lq - 1 - (a.left == 0), j0 + a.left - ahead);
  const int tile0 = lo / kTile, tiles = hi >= lo ? hi / kTile - tile0 + 1 : 0;
  const int from = share(tiles * a.G, p.part, a.parts), to = share(tiles * a.G, p.part + 1, a.parts);      // of the tiles of all heads, one after the other

  const int from_head = tiles > 0 ? from / tiles : 0, from_tile = from - from_head * tiles;
  int fetched_head = from_head, fetched_tile = from_tile, tile = from_tile;      // the next ones
  auto fetch = [&](int, int stage) {
    const uint32_t s = lds_at(lds) + stage * STAGE;
    const int head = p.hk * a.G + fetched_head, row = (tile0 + fetched_tile) * kTile, left = p.Lq - row;
    qload.load(rows_of(a.q, p.b, p.q0 + row, head), left, s, wave, lane);
    gload.load(rows_of(a.d_o, p.b, p.q0 + row, head), left, s + TILE, wave, lane);
    if (wave == 0) {                                   // (zeros for rows that are not there)
      const float* st = a.stats + stat_row(a, p, head) + row;
      const uint32_t off = lane < left ? lane * 4 : kOob;
      load_to_lds<4>(descriptor((const char*)st), off, s + STATS);
      load_to_lds<4>(descriptor((const char*)(st + a.rows)), off, s + STATS + kTile * 4);
    }
    if (++fetched_tile == tiles) { fetched_tile = 0; ++fetched_head; }
  };
  if (from < to) fetch(from, 0);

  f32x16 dk[NB], dv[NB];
  auto step = [&](auto stage, int) {
    constexpr int AT = decltype(stage)::value * STAGE;
    const int i0 = (tile0 + tile) * kTile;
    if (++tile == tiles) tile = 0;
    if (i0 > whi || i0 + kTile <= wlo) return;
    const bool border = i0 < alllo || i0 + kTile - 1 > allhi;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      f32x16 s, dp;
      Frag<T> buf[fragments_ahead<T>()];
      // rows of the queries, rows of d_o, columns of d_o and of the queries
      constexpr int N1 = 2 * KK, N2 = 4 * NB, ALL = N1 + N2, P = fragments_ahead<T>();
      auto fragment = [&](int n) {
        return n < N1 ? rows.read(AT + (n < KK ? 0 : TILE) + 32 * nb * ROWB, n % KK)
                      : cols.read(AT + ((n - N1) % (2 * NB) < NB ? TILE : 0) + (32 * nb + 16 * ((n - N1) / (2 * NB))) * ROWB, (n - N1) % NB);
      };
#pragma unroll
      for (int n = 0; n < P; ++n) if (n < ALL) buf[n] = fragment(n);
#pragma unroll
      for (int b = 0; b < 4; ++b) {                    // dP - D: the product starts from -D
        const u32x4 d = lds_read<u32x4>(stats_at, AT + kTile * 4 + (32 * nb + 8 * b) * 4);
#pragma unroll
        for (int x = 0; x < 4; ++x) dp[4 * b + x] = __uint_as_float(d[x]);
      }
      zero(s);
  #pragma unroll
      for (int n = 0; n < N1; ++n) {
        if (n < KK) mma(s, buf[n % P], k[n]); else mma(dp, buf[n % P], v[n - KK]);
        if (n + P < ALL) buf[n % P] = fragment(n + P);
        __builtin_amdgcn_sched_barrier(0);
      }
  #pragma unroll
      for (int b = 0; b < 4; ++b) {
        const u32x4 l2 = lds_read<u32x4>(stats_at, AT + (32 * nb + 8 * b) * 4);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = 4 * b + x;
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.c, -__uint_as_float(l2[x])));
          dp[r] *= s[r];
        }
      }
      if (border) {
        int at = lane;
        if constexpr (NB > 2) asm volatile("" : "+v"(at));     // (made again for each border: kept over the loop this costs registers that D > 96 does not have)
        const int key = j0 + (at & 31), base = i0 + 4 * (at >> 5);
        const int first = max(0, key - a.right - ahead) - base, behind = min(p.Lq - 1, key + a.left - ahead) - base;
        const int alone = max(key == 0 ? -a.right - ahead : key == p.Lk - 1 && a.left == 0 ? p.Lq - 1 : -1, -1) - base;     // the query that sees no other key
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int i = 32 * nb + 8 * (r >> 2) + (r & 3);
          const bool see = i >= first && i <= behind;
          s[r] = see ? s[r] : 0.0f;
          dp[r] = see ? i == alone ? 0.0f * dp[r] : dp[r] : 0.0f;      // (one score has no gradient; a NaN stays one)
        }
      }
      Frag<T> pk, ds;
  #pragma unroll
      for (int n = 0; n < N2; ++n) {
        if (n % (2 * NB) == 0) { pk = operand<T>(s, n / (2 * NB)); ds = operand<T>(dp, n / (2 * NB)); }
        if (n % (2 * NB) < NB) mma(dv[n % NB], buf[(N1 + n) % P], pk); else mma(dk[n % NB], buf[(N1 + n) % P], ds);
        if (n + P < N2) buf[(N1 + n) % P] = fragment(N1 + n + P);
        __builtin_amdgcn_sched_barrier(0);
      }
      }
  };
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) { zero(dk[blk]); zero(dv[blk]); }
    walk_tiles(from, to, careful, fetch, step, [&] { copy_finite<T, 2 * TILE, NW * 64>(lds, lds + STAGE, tid); });
    if (careful || (a.left >= kFar && a.right >= kFar) || !__syncthreads_or(any_nan<NB>(dk) || any_nan<NB>(dv))) break;
    careful = true;
    cols.shift(STAGE);
    fetched_head = from_head;
    tile = fetched_tile = from_tile;
  }
  if (careful && there)
    for (int g = 0; g < a.G; ++g) {
      const int t0 = max(from - g * tiles, 0), t1 = min(to - g * tiles, tiles);        // of this head
      const int r0 = max(mylo, (tile0 + t0) * kTile), r1 = min(myhi, (tile0 + t1) * kTile - 1);
      spoil<T, NB>(dk, rows_of(a.q, p.b, p.q0, p.hk * a.G + g), a.q.token, r0, r1, lane, a.D);
      spoil<T, NB>(dv, rows_of(a.d_o, p.b, p.q0, p.hk * a.G + g), a.d_o.token, r0, r1, lane, a.D);
    }
  const float factor = p.Lk == 1 || (a.left | a.right) == 0 ? 0.0f : a.scale;       // (no query sees more than one key; single ones among others: at the border, above)
  if (a.parts > 1) {
    const int64_t row = p.part * a.key_rows + key_row(a, p) + j;
    store_rows<float, NB>((char*)(a.part + row * a.D), there, dk, factor, lane, a.D);
    store_rows<float, NB>((char*)(a.part + (a.parts * a.key_rows + row) * a.D), there, dv, 1.0f, lane, a.D);
  } else {
    store_rows<T, NB>(rows_of(a.dk, p.b, p.k0 + j, p.hk), there, dk, factor, lane, a.D);
    store_rows<T, NB>(rows_of(a.dv, p.b, p.k0 + j, p.hk), there, dv, 1.0f, lane, a.D);
  }
}

// ---- parts into one result ---------------------------------------------------------------------------------------------------
// Bound by HBM or, where it is used most, by its launch: 20 us for dk and dv of 2 x 6001 x 4 x 128 in two parts (98 MB in, 25 MB out, 6 TB/s from the
// cache), 4.5 us for 8 x 197 x 6 x 64.  Eight elements a thread, the parts in their order.  Forward: weighted by exp2(m c - the largest m c), over the weighted sum of the l.
struct JoinArgs {
  const float* part; const float* ml; HeadsArg out, second; float* lse;      // second: of the parts behind these (dv behind dk)
  const int32_t* off; int B, S, H, D, parts;
  int64_t rows;
};
template <typename T> __global__ __launch_bounds__(256) void attn_join_kernel(JoinArgs a) {
  const int vectors = a.D / 8;
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, row = n / vectors;
  if (row >= a.rows) return;
  const int d = (int)(n - row * vectors) * 8;
  int64_t first = row / a.S;
  const int i = (int)(row - first * a.S), b = a.off ? 0 : (int)(first / a.H), h = (int)(first - (int64_t)b * a.H);
  if (a.off && (i < clampi(a.off[0], 0, a.S) || i >= clampi(a.off[a.B], 0, a.S))) return;      // in no sequence
  const float* const parts = a.part + (int64_t)blockIdx.y * a.parts * a.rows * a.D;
  float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, top = -kInf, l = 0.0f, factor = 1.0f;
  if (a.ml) {
    for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.ml[2 * (p * a.rows + row)]);
  }
  for (int p = 0; p < a.parts; ++p) {
    const float* const src = parts + (p * a.rows + row) * a.D + d;
    float w = 1.0f;
    if (a.ml) {
      const float m = a.ml[2 * (p * a.rows + row)];
      w = m == -kInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
      l += w * a.ml[2 * (p * a.rows + row) + 1];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float4 v = *reinterpret_cast<const float4*>(src + 4 * j);
      x[4 * j] += w * v.x; x[4 * j + 1] += w * v.y; x[4 * j + 2] += w * v.z; x[4 * j + 3] += w * v.w;
    }
  }
  if (a.ml) {
    const bool some = l > 0.0f || l != l;
    factor = some ? 1.0f / l : 0.0f;
    if (d == 0) a.lse[row] = some ? (top + __builtin_amdgcn_logf(l)) * kLn2 : -kInf;
  }
  T* const out = reinterpret_cast<T*>(rows_of(blockIdx.y ? a.second : a.out, b, i, h)) + d;
  if constexpr (sizeof(T) == 2) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = f2bf_pack(x[2 * j] * factor, x[2 * j + 1] * factor);
    *reinterpret_cast<u32x4*>(out) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) *reinterpret_cast<float4*>(out + 4 * j) = make_float4(x[4 * j] * factor, x[4 * j + 1] * factor, x[4 * j + 2] * factor, x[4 * j + 3] * factor);
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
enum { kForward, kGradQ, kGradKV };
constexpr int kWavesOf = 4, kRows = 32 * kWavesOf, kUnits = 256, kMostParts = 32;

// Workgroups of a pass that a compute unit holds at least (one wave of each on every SIMD): what their registers leave room for without spilling
// in the loops over tiles.  Three where 168 a lane are enough (bf16 heads of up to 64, forward and dq), two with 256, one with 512.  Outside these loops heads of
// 112 and more spill: 17 registers in dq (bf16, 128) and in dk and dv (bf16, 128), 49 and 67 there in fp32.
constexpr int occupancy(bool half_width, int nb, int pass) {
  return pass == kGradKV ? (half_width && nb <= 2 ? 2 : 1) : half_width && nb <= 2 ? 3 : half_width || nb <= 2 ? 2 : 1;
}

int64_t tiles_of(const AttnArgs& a, int pass) {
  const int S = pass == kGradKV ? a.Sk : a.Sq;
  return a.off_q ? (int64_t)S / kRows + a.B : ((int64_t)S + kRows - 1) / kRows;
}

// In how many parts a pass walks: where the tiles are too few for the compute units, or too unlike, several workgroups share the walk of each and a
// launch adds up what they leave.  The estimate is in tiles of the walk (about 1 us in bf16, 8 in fp32): those that the busiest unit takes, the
// start of a workgroup (3 us), and for the launch that adds up 7 us and its traffic at 4 TB/s.  Measured: 2 x 6001 tokens, 16 heads of
// 128 on 4 key heads, causal: dk and dv 861 us in one part (376 unlike tiles on 256 units), 698 + 22 us in two.
int parts_of(const dat_attention& s, const AttnArgs& a, int pass) {
  const int64_t tiles = tiles_of(a, pass), groups = a.off_q ? a.Hkv : (int64_t)a.B * a.Hkv;
  const int64_t items = tiles * groups * (pass == kGradKV ? 1 : a.G), slots = (int64_t)kUnits * occupancy(s.dtype == DAT_BF16, (s.D + 31) / 32, pass);
  if (items == 0 || items > 8 * slots || tiles > 65536) return 1;
  const int seqs = a.off_q ? (a.B > 0 ? a.B : 1) : 1;
  const int64_t Lq = (a.Sq + seqs - 1) / seqs, Lk = (a.Sk + seqs - 1) / seqs;     // (packed: as if all were alike)
  int64_t total = 0, most = 0;
  const int64_t own = pass == kGradKV ? Lk : Lq;
  for (int64_t r = 0; r < own; r += kRows) {
    const int64_t end = (r + kRows < own ? r + kRows : own) - 1;
    int64_t lo, hi;
    if (pass == kGradKV) { lo = r - a.right - (Lk - Lq); hi = end + a.left - (Lk - Lq); lo = lo > 0 ? lo : 0; hi = hi < Lq - 1 ? hi : Lq - 1; }
    else { lo = r + Lk - Lq - a.left; hi = end + Lk - Lq + a.right; lo = lo > 0 ? lo : 0; hi = hi < Lk - 1 ? hi : Lk - 1; }
    const int64_t n = hi >= lo ? (hi / kTile - lo / kTile + 1) * (pass == kGradKV ? a.G : 1) : 0;
    total += n;
    most = n > most ? n : most;
  }
  total *= seqs * groups * (pass == kGradKV ? 1 : a.G);
  const bool alike = a.left >= kFar && a.right >= kFar && !a.off_q;
  const double us = s.dtype == DAT_BF16 ? 1.0 : 8.0, traffic = 2.0 * (pass == kGradKV ? 2 * a.key_rows : a.rows) * a.D * 4 / 4e6;
  int best = 1;
  double least = 0;
  for (int p = 1; p <= kMostParts && (p == 1 || p <= most); ++p) {
    const int64_t rounds = (items * p + slots - 1) / slots, longest = (most + p - 1) / p;
    const double even = (double)total / slots;
    double t = us * (alike ? (double)rounds * longest : even > longest ? even : longest) + 3.0 * rounds;
    if (p > 1) t += 7.0 + p * traffic;
    if (p == 1 || t < least) { best = p; least = t; }
  }
  return best;
}
size_t part_bytes(const AttnArgs& a, int pass, int parts) {
  if (parts <= 1) return 0;
  return (size_t)parts * (pass == kGradKV ? 2 * a.key_rows * a.D : a.rows * (a.D + (pass == kForward ? 2 : 0))) * 4;
}

template <typename T, int NB, int KK> dat_status launch(int pass, AttnArgs a, hipStream_t st) {
  constexpr int NW = kWavesOf;
  const int64_t tiles = tiles_of(a, pass), groups = a.off_q ? a.Hkv : (int64_t)a.B * a.Hkv;
  a.groups = (int)groups;
  a.rows_per_group = (int)tiles;
  const int64_t items = tiles * groups * (pass == kGradKV ? 1 : a.G) * a.parts;
  a.items = (int)items;
  // A share of the work for each XCD, whose L2 then holds the keys of few heads; under a window the shares of few groups are too unlike.  Measured with
  // and without, causal: 8 groups 511 / 593 us forward and 1070 / 1321 us backward (the cases named above), 36 groups 366 / 494, 11 300 / 327, 6
  // 287 / 358 (backward), 12 64 / 66, 9 241 / 230, 5 140 / 137, 3 296 / 251 (forward); no window, 64 sequences of 4 to 1024 tokens 260 / 308.
  a.xcd = a.groups >= 6 || (a.left >= kFar && a.right >= kFar);
  if (tiles > INT32_MAX || !fits_launch(items + 7, NW * 64)) return DAT_ERR_SHAPE;
  if (items == 0) return DAT_OK;
  const dim3 grid((unsigned)(a.xcd ? (items + 7) / 8 * 8 : items)), block(NW * 64);
  if (pass == kForward) hipLaunchKernelGGL((attn_fwd_kernel<T, NB, KK, NW, occupancy(sizeof(T) == 2, NB, kForward)>), grid, block, 0, st, a);
  else if (pass == kGradQ) hipLaunchKernelGGL((attn_dq_kernel<T, NB, KK, NW, occupancy(sizeof(T) == 2, NB, kGradQ)>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((attn_dkv_kernel<T, NB, KK, NW, occupancy(sizeof(T) == 2, NB, kGradKV)>), grid, block, 0, st, a);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

// Adds up the parts of a pass.
template <typename T> dat_status join(int pass, const AttnArgs& a, hipStream_t st) {
  const bool keys = pass == kGradKV;
  const int64_t rows = keys ? a.key_rows : a.rows;
  JoinArgs j{a.part, pass == kForward ? a.part + a.parts * a.rows * a.D : nullptr, pass == kForward ? a.o : keys ? a.dk : a.dq, a.dv, a.lse, keys ? a.off_k : a.off_q, a.B,
             keys ? a.Sk : a.Sq, keys ? a.Hkv : a.H, a.D, a.parts, rows};
  const int64_t blocks = (rows * (a.D / 8) + 255) / 256;
  if (!fits_launch(blocks, 256)) return DAT_ERR_SHAPE;
  hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)blocks, keys ? 2 : 1), dim3(256), 0, st, j);
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

template <typename T> dat_status launch_heads(int pass, const AttnArgs& a, hipStream_t st) {
  switch ((a.D + 15) / 16) {          // steps of 16 in the products over a head, blocks of 32 in its results
    case 1: return launch<T, 1, 1>(pass, a, st);
    case 2: return launch<T, 1, 2>(pass, a, st);
    case 3: return launch<T, 2, 3>(pass, a, st);
    case 4: return launch<T, 2, 4>(pass, a, st);
    case 5: return launch<T, 3, 5>(pass, a, st);
    case 6: return launch<T, 3, 6>(pass, a, st);
    case 7: return launch<T, 4, 7>(pass, a, st);
    default: return launch<T, 4, 8>(pass, a, st);
  }
}
template <typename T> dat_status run_pass(int pass, const AttnArgs& a, hipStream_t st) {
  const dat_status r = launch_heads<T>(pass, a, st);
  return r != DAT_OK || a.parts <= 1 ? r : join<T>(pass, a, st);
}
dat_status run_pass(int pass, dat_dtype dtype, const AttnArgs& a, hipStream_t st) {
  return dtype == DAT_BF16 ? run_pass<bf16_t>(pass, a, st) : run_pass<float>(pass, a, st);
}
size_t stats_bytes(const AttnArgs& a) { return (size_t)(2 * a.rows * 4 + 15) / 16 * 16; }

bool fill(const dat_attention* s, AttnArgs& a, dat_status& status) {
  status = DAT_ERR_ARG;
  if (!s || (s->dtype != DAT_F32 && s->dtype != DAT_BF16) || s->B < 0 || s->Sq < 0 || s->Sk < 0 || s->H < 1 || s->Hkv < 1 || s->H % s->Hkv || s->D < 1) return false;
  if (!(s->scale > 0.0f) || !(s->scale < kInf) || !(s->scale * kLog2e < kInf) || s->left < -1 || s->right < -1) return false;
  if (!s->offsets_q != !s->offsets_k || !aligned(s->offsets_q, 4) || !aligned(s->offsets_k, 4)) return false;
  status = DAT_ERR_SHAPE;
  if (s->D % 8 || s->D > 128 || s->Sq >= kFar || s->Sk >= kFar) return false;
  const int64_t batches = s->offsets_q ? 1 : s->B;
  if (batches * s->H * (int64_t)s->Sq >= (int64_t)1 << 40 || batches * s->Hkv * (int64_t)s->Sk >= (int64_t)1 << 40 || (int64_t)s->B * s->Hkv > INT32_MAX) return false;
  if (((int64_t)s->Sq / kTile + 1) * (s->H / s->Hkv) > INT32_MAX) return false;       // tiles of a key head's queries are counted in 32 bits
  a.off_q = s->offsets_q; a.off_k = s->offsets_k;
  a.B = s->B; a.Sq = s->Sq; a.Sk = s->Sk; a.H = s->H; a.Hkv = s->Hkv; a.G = s->H / s->Hkv; a.D = s->D;
  a.left = s->left < 0 ? kFar : s->left < kFar ? s->left : kFar;
  a.right = s->right < 0 ? kFar : s->right < kFar ? s->right : kFar;
  a.scale = s->scale; a.c = s->scale * kLog2e;
  a.rows = batches * s->H * (int64_t)s->Sq;
  a.key_rows = batches * s->Hkv * (int64_t)s->Sk;
  status = DAT_OK;
  return true;
}

// Checks a tensor and turns its strides into bytes.
dat_status take(const dat_heads* t, const HeadsShape& s, size_t width, bool output, HeadsArg& out) {
  if (!t) return DAT_ERR_ARG;
  if (s.batch * s.tokens * s.heads == 0) { out = HeadsArg{(char*)t->data, 0, 0, 0}; return DAT_OK; }
  if (!heads_vectors(*t, s, width) || (output && !heads_apart(*t, s))) return DAT_ERR_ARG;
  const int64_t w = (int64_t)width, token = s.tokens > 1 ? t->token * w : 0;
  if (token >= (int64_t)1 << 23) return DAT_ERR_SHAPE;             // the offsets in a tile of up to 256 rows are 31 bits
  out = HeadsArg{(char*)t->data, s.batch > 1 ? t->batch * w : 0, token, s.heads > 1 ? t->head * w : 0};
  return DAT_OK;
}

struct Tensor { const dat_heads* t; HeadsShape s; HeadsArg* to; bool output; };
enum { kStatsRead, kStatsWritten };

// The tensors, and beside them the rows' statistics that a call reads or writes (fp32, none where there are no rows) and the offsets.
dat_status take_all(std::initializer_list<Tensor> list, size_t width, const AttnArgs& a, const float* lse, int stats) {
  for (const Tensor& x : list) {
    const dat_status st = take(x.t, x.s, width, x.output, *x.to);
    if (st != DAT_OK) return st;
  }
  for (const Tensor& x : list)
    if (x.output)
      for (const Tensor& y : list) if (&x != &y && heads_overlap(*x.t, x.s, *y.t, y.s, width)) return DAT_ERR_ARG;
  const Block rows{lse, a.B > 0 ? (uint64_t)a.rows * 4 : 0}, offsets_q{a.off_q, (uint64_t)a.B * 4 + 4}, offsets_k{a.off_k, (uint64_t)a.B * 4 + 4};
  for (const Tensor& x : list) {
    const Block block = heads_block(x.t, x.s, width);
    if ((x.output || stats == kStatsWritten) && blocks_overlap(block, rows)) return DAT_ERR_ARG;
    if (x.output && (blocks_overlap(block, offsets_q) || blocks_overlap(block, offsets_k))) return DAT_ERR_ARG;
  }
  if (stats == kStatsWritten && (blocks_overlap(rows, offsets_q) || blocks_overlap(rows, offsets_k))) return DAT_ERR_ARG;
  return DAT_OK;
}

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" size_t dat_attention_workspace(int pass, const dat_attention* shape) {
  AttnArgs a{};
  dat_status st;
  if (!fill(shape, a, st) || (pass != 0 && pass != 1)) return 0;
  if (pass == 0) return part_bytes(a, kForward, parts_of(*shape, a, kForward));
  // D and lse / ln 2, then the parts of one pass after those of the other
  const size_t q = part_bytes(a, kGradQ, parts_of(*shape, a, kGradQ)), kv = part_bytes(a, kGradKV, parts_of(*shape, a, kGradKV));
  return stats_bytes(a) + (q > kv ? q : kv);
}

extern "C" dat_status dat_attention_forward(const dat_attention* shape, const dat_heads* q, const dat_heads* k, const dat_heads* v,
                                            const dat_heads* o, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  dat_status st;
  if (!fill(shape, a, st)) return st;
  const int64_t B = a.off_q ? (a.B > 0) : a.B;
  const HeadsShape sq{B, a.Sq, a.H, a.D}, sk{B, a.Sk, a.Hkv, a.D};
  const size_t width = shape->dtype == DAT_BF16 ? 2 : 4;
  st = take_all({{q, sq, &a.q, false}, {k, sk, &a.k, false}, {v, sk, &a.v, false}, {o, sq, &a.o, true}}, width, a, lse, kStatsWritten);
  if (st != DAT_OK) return st;
  if (B == 0 || a.Sq == 0) return DAT_OK;
  if (!lse || !aligned(lse, 4)) return DAT_ERR_ARG;
  a.parts = parts_of(*shape, a, kForward);
  const size_t need = part_bytes(a, kForward, a.parts);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return DAT_ERR_ARG;
  a.lse = lse;
  a.part = (float*)workspace;
  return run_pass(kForward, shape->dtype, a, (hipStream_t)stream);
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
  st = take_all({{q, sq, &a.q, false}, {k, sk, &a.k, false}, {v, sk, &a.v, false}, {o, sq, &a.o, false}, {d_o, sq, &a.d_o, false},
                 {dq, sq, &a.dq, true}, {dk, sk, &a.dk, true}, {dv, sk, &a.dv, true}}, width, a, lse, kStatsRead);
  if (st != DAT_OK) return st;
  if (B == 0) return DAT_OK;
  if (a.Sq > 0 && (!lse || !aligned(lse, 4))) return DAT_ERR_ARG;
  const size_t need = dat_attention_workspace(1, shape);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return DAT_ERR_ARG;
  a.lse_in = lse;
  a.stats = (float*)workspace;
  a.part = (float*)((char*)workspace + stats_bytes(a));
  if (a.Sq > 0) {
    a.parts = parts_of(*shape, a, kGradQ);
    st = run_pass(kGradQ, shape->dtype, a, (hipStream_t)stream);
    if (st != DAT_OK) return st;
  }
  if (a.Sk == 0) return DAT_OK;
  a.parts = parts_of(*shape, a, kGradKV);
  return run_pass(kGradKV, shape->dtype, a, (hipStream_t)stream);
}
