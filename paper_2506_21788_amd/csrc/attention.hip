// hgnn_graph_attention_fwd / _bwd: attention over the atoms of each graph with a learned bias per head and pair bucket.
//
//   s_ij = scale q_i . k_j + bias[h][bucket_ij],   p_ij = exp(s_ij - max) / sum,   o_i = sum_j p_ij v_j
//   D_i = g_i . o_i,   ds_ij = p_ij (g_i . v_j - D_i),   g_q_i = scale sum_j ds_ij k_j,   g_k_j = scale sum_i ds_ij q_i,
//   g_v_j = sum_i p_ij g_i,   g_bias[h][b] = sum of ds over the pairs of bucket b
//
// One wavefront works alone on 32 rows (queries; keys in k_attn_dkv) and walks the other side in tiles of 32, with the running
// maximum and sum of the softmax: nothing of the size of a graph's pairs is stored. Every score tile is formed transposed,
// S^T[key][query], on 32 x 32 matrix-core tiles. A lane then holds 16 scores of ONE query: the sums over keys are within the
// lane but for one exchange with the other half, the scale factors of a row are one register, and the packed weights are, as
// they stand, the operand of the next product (O^T = V^T P^T, the order of its contraction being free). The rows of the first
// operand are permuted (tile_row) so that the 16 keys of a lane are neighbours: their buckets are one 16-byte load. The bias
// of a bucket, in units of the product (bias / scale), is read from a table of 256 in LDS straight into the accumulators that the
// product adds to; the table holds -inf past the last bucket, so a pair that is left out costs nothing.
// Operands that a product needs by columns go through LDS once, row by row, and come back through transposing reads (bf16)
// or as single values (float32, matrix-core products of float32).
//
// Bound by the vector units forward, by waits in reverse. 20,000 atoms in one graph, 4 heads of 32, bf16: forward 0.83 ms (247 TFLOP/s),
// reverse 1.17 + 0.97 ms. A tile of 1,024 scores takes a SIMD 1,110 cycles in k_attn_fwd, 79 % of them vector instructions (the three
// terms of the weights 350, exponentials 128, places in the table of biases 64) and 23 % the matrix cores; 1,750 in k_attn_dq (vector units 56 %,
// LDS 35, matrix cores 11) and 1,400 in k_attn_dkv (LDS 55, vector units 48, matrix cores 18) at 2.5 wavefronts a SIMD. In batches of small
// graphs a wavefront has some four tiles, and its first loads and its end cost as much as two more: 390 graphs of 5 to 200 atoms,
// 8 heads of 32 on 2, bf16, take 40 us forward (vector units 57 % busy) and 53 + 48 us in reverse (k_attn_dq: vector units 42 %, LDS 28).
//
// The sums of the reverse pass are split in two kernels (one owns queries, one keys) rather than added with atomics, so that
// their order is fixed: the scores are formed twice. g_bias is collected in LDS, a column per lane and bucket (in long graphs lanes i and
// i + 32 share one and add in turn), over all tiles that a wavefront takes, and then added up over the wavefronts in order.
//
// A pair that is left out must not be touched by what its atoms hold, but a matrix product multiplies it by zero, and 0 * inf is
// no number. So a wavefront whose result is not finite forms its rows again, pair by pair over the pairs that count.
#include <climits>

#include "common.h"
#include "devmath.h"
#include "pairs.h"
#include "prof.h"

namespace hgnn {
namespace {

typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr int ATTN_BUCKETS = 64;   // most buckets: a wavefront's sums of g_bias are 64 lanes x buckets words of LDS

struct AttnArgs {
  int N, G, nh, nkv, dh, nb;
  int nw;        // wavefronts of a workgroup: 1, or (SPLIT) those that share a tile of rows and deal out the other side's tiles
  int per_head;  // workgroups per head of k_attn_dq
  int near;      // see item_of
  float scale, c, inv;   // c = scale log2 e, inv = 1 / scale
  PairPlan plan;
  const uint8_t* pairs;
  const void* qkv;
  const float* bias;
  void* out;
  float2* stat;   // [nh][N] largest score / scale, log2 of the sum of exp(score - largest); 0 and +inf for a row without pairs
  float* o32;     // [N][nh][dh] the output before its rounding (bf16), else null
  const void* g_out;
  void* g_qkv;
  float* delta;   // [nh][N]
  float* partial; // [nh][per_head][nb]
  float* g_bias;
};

// row of the tile that row m of a first operand holds: lane half g ends up with accumulator registers 0..15 = rows 16 g + 0..15
__device__ __forceinline__ int tile_row(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

__device__ __forceinline__ void lds_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); __builtin_amdgcn_wave_barrier(); }

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// 16-byte piece `piece` of row `row` of a bf16 tile in LDS. Rows are a multiple of 64 bytes long and 64 or 192 bytes apart (mod 256), so that a
// transposing read (four rows of 64 bytes at a time) meets every bank once; within each 64 bytes the pieces are exchanged by
// the row's place, so that sixteen rows read at one piece (in either order of rows) do too.
__device__ __forceinline__ int piece_at(int row, int piece, int pitch) {
  return row * pitch + ((piece ^ ((row >> 2) & 3) ^ ((row >> 4) * 2)) * 8);
}

// One row of DP (dh and zeros) per lane pair, as the operand of a product that contracts over it.
// bf16: dims 16 k + 8 g + 0..7 of step k. float32: dims g DP/2 + s of step s.
template <bool BF, int DP>
struct Row;
template <int DP>
struct Row<true, DP> {
  static constexpr int PITCH = DP == 32 ? 32 : DP + 32;   // elements from row to row in LDS
  using T = unsigned short;
  u32x4_t f[DP / 16];
  __device__ __forceinline__ void load(const T* p, int dh, int g) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      const int d = 16 * k + 8 * g;
      f[k] = u32x4_t{0, 0, 0, 0};
      if (d < dh) f[k] = *reinterpret_cast<const u32x4_t*>(p + d);
    }
  }
  __device__ __forceinline__ void from_lds(const T* tile, int row, int g) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) f[k] = *reinterpret_cast<const u32x4_t*>(tile + piece_at(row, 2 * k + g, PITCH));
  }
  __device__ __forceinline__ void negate_if(bool yes) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) f[k] ^= yes ? 0x80008000u : 0u;
  }
  __device__ __forceinline__ static f32x16_t dot(const Row& a, const Row& b, f32x16_t acc) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.f[k]), __builtin_bit_cast(bf16x8_t, b.f[k]), acc, 0, 0, 0);
    return acc;
  }
  // sum over the row's own dims of a product with float32 values in the same place
  __device__ __forceinline__ float dot32(const float* p, int dh, int g) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      const int d = 16 * k + 8 * g;
      if (d < dh) {
        const float4 x = *reinterpret_cast<const float4*>(p + d), y = *reinterpret_cast<const float4*>(p + d + 4);
        s = fmaf(__uint_as_float(f[k][0] << 16), x.x, s); s = fmaf(__uint_as_float(f[k][0] & 0xffff0000u), x.y, s);
        s = fmaf(__uint_as_float(f[k][1] << 16), x.z, s); s = fmaf(__uint_as_float(f[k][1] & 0xffff0000u), x.w, s);
        s = fmaf(__uint_as_float(f[k][2] << 16), y.x, s); s = fmaf(__uint_as_float(f[k][2] & 0xffff0000u), y.y, s);
        s = fmaf(__uint_as_float(f[k][3] << 16), y.z, s); s = fmaf(__uint_as_float(f[k][3] & 0xffff0000u), y.w, s);
      }
    }
    return s;
  }
};
template <int DP>
struct Row<false, DP> {
  static constexpr int PITCH = DP + 4;
  using T = float;
  float f[DP / 2];
  __device__ __forceinline__ void load(const T* p, int dh, int g) {
#pragma unroll
    for (int k = 0; k < DP / 8; ++k) {
      const int d = g * (DP / 2) + 4 * k;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (d < dh) v = *reinterpret_cast<const float4*>(p + d);
      f[4 * k] = v.x; f[4 * k + 1] = v.y; f[4 * k + 2] = v.z; f[4 * k + 3] = v.w;
    }
  }
  __device__ __forceinline__ void from_lds(const T* tile, int row, int g) {
#pragma unroll
    for (int k = 0; k < DP / 8; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(tile + row * PITCH + g * (DP / 2) + 4 * k);
      f[4 * k] = v.x; f[4 * k + 1] = v.y; f[4 * k + 2] = v.z; f[4 * k + 3] = v.w;
    }
  }
  __device__ __forceinline__ void negate_if(bool yes) {
#pragma unroll
    for (int s = 0; s < DP / 2; ++s) f[s] = yes ? -f[s] : f[s];
  }
  __device__ __forceinline__ static f32x16_t dot(const Row& a, const Row& b, f32x16_t acc) {
#pragma unroll
    for (int s = 0; s < DP / 2; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[s], b.f[s], acc, 0, 0, 0);
    return acc;
  }
  __device__ __forceinline__ float dot32(const float* p, int dh, int g) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 8; ++k) {
      const int d = g * (DP / 2) + 4 * k;
      if (d < dh) {
        const float4 x = *reinterpret_cast<const float4*>(p + d);
        s = fmaf(f[4 * k], x.x, s); s = fmaf(f[4 * k + 1], x.y, s); s = fmaf(f[4 * k + 2], x.z, s); s = fmaf(f[4 * k + 3], x.w, s);
      }
    }
    return s;
  }
};

// 32 rows on their way from memory to LDS, in pieces of 16 bytes: neighbouring lanes hold neighbouring pieces of a row. (Loaded as
// operands, a lane its own row, every lane's piece was an access of its own to the cache: 320 a tile and wavefront, the
// vector cache 64 % busy with looking them up; so it is a quarter of that.)
template <bool BF, int DP>
struct Tile {
  using T = typename Row<BF, DP>::T;
  static constexpr int EP = 16 / sizeof(T), NP = DP / EP;   // elements of a piece, pieces of a row
  u32x4_t f[NP / 2];
  // p: the tile's first row (uniform); rows: how many exist (the last one stands for those behind it, and a row's last piece for
  // those behind that: the operand that meets it in a product has zeros there, and result columns past dh are not stored)
  __device__ __forceinline__ void load(const T* p, unsigned ld, int rows, int dh, int lane) {
#pragma unroll
    for (int u = 0; u < NP / 2; ++u) {
      const int row = (u * 64 + lane) / NP, d = min((u * 64 + lane) % NP * EP, dh - EP);
      f[u] = *reinterpret_cast<const u32x4_t*>(p + (unsigned)(min(row, rows - 1) * ld + d));
    }
  }
  __device__ __forceinline__ void to_lds(T* tile, int lane) const {
#pragma unroll
    for (int u = 0; u < NP / 2; ++u) {
      const int row = (u * 64 + lane) / NP, piece = (u * 64 + lane) % NP;
      T* at;
      if constexpr (BF) at = tile + piece_at(row, piece, Row<BF, DP>::PITCH);
      else at = tile + row * Row<BF, DP>::PITCH + piece * EP;
      *reinterpret_cast<u32x4_t*>(at) = f[u];
    }
  }
};

__device__ __forceinline__ bf16x8_t read_tr(const unsigned short* lo, const unsigned short* hi) {
  const s16x4_t l = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lo));
  const s16x4_t h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(hi));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7));
}
// rows 16 g + 8 t + 0..7 of column 32 b + lane & 31 of a tile in LDS
__device__ __forceinline__ bf16x8_t read_col(const unsigned short* tile, int pitch, int b, int t, int lane) {
  const int row = 16 * (lane >> 5) + 8 * t + ((lane & 15) >> 2);   // (row / 4 is 2 t mod 4, and 2 t + 1 for the rows behind)
  const int piece = (((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) ^ ((lane >> 5) * 2), within = (lane & 1) * 4;
  const unsigned short* p = tile + row * pitch + 32 * b + within;
  return read_tr(p + (piece ^ (2 * t & 3)) * 8, p + 4 * pitch + (piece ^ ((2 * t + 1) & 3)) * 8);
}

// sixteen weights of a lane's query (rows 16 g + v), packed as the second operand of a product over those rows
template <bool BF>
struct Weights;
template <>
struct Weights<true> {
  bf16x8_t w[2];
  __device__ __forceinline__ explicit Weights(const f32x16_t& p) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4_t u = {pack_bf16x2(p[8 * t], p[8 * t + 1]), pack_bf16x2(p[8 * t + 2], p[8 * t + 3]), pack_bf16x2(p[8 * t + 4], p[8 * t + 5]),
                         pack_bf16x2(p[8 * t + 6], p[8 * t + 7])};
      w[t] = __builtin_bit_cast(bf16x8_t, u);
    }
  }
};
// the same as three terms that add up to the weights exactly: the high 16 bits, those of the remainder, and what is left (8 bits)
struct Weights3 {
  bf16x8_t w[3][2];
  __device__ __forceinline__ explicit Weights3(const f32x16_t& p) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4_t u[3];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float x = p[8 * t + 2 * k], y = p[8 * t + 2 * k + 1];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          u[q][k] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
          x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
          y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
        }
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) w[q][t] = __builtin_bit_cast(bf16x8_t, u[q]);
    }
  }
};
template <>
struct Weights<false> {
  f32x16_t w;
  __device__ __forceinline__ explicit Weights(const f32x16_t& p) : w(p) {}
};

// acc[b][d][query] += sum over the tile's rows of tile[row][32 b + d] w[row]
template <bool BF, int DP>
__device__ __forceinline__ void add_cols(const typename Row<BF, DP>::T* tile, const Weights<BF>& w, f32x16_t (&acc)[DP / 32], int lane) {
  constexpr int PITCH = Row<BF, DP>::PITCH;
#pragma unroll
  for (int b = 0; b < DP / 32; ++b) {
    if constexpr (BF) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_col(tile, PITCH, b, t, lane), w.w[t], acc[b], 0, 0, 0);
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[(16 * (lane >> 5) + v) * PITCH + 32 * b + (lane & 31)], w.w[v], acc[b], 0, 0, 0);
    }
  }
}
// the same with weights of three bf16 terms, smallest first
template <int DP>
__device__ __forceinline__ void add_cols3(const unsigned short* tile, const Weights3& w, f32x16_t (&acc)[DP / 32], int lane) {
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8_t c = read_col(tile, Row<true, DP>::PITCH, b, t, lane);
#pragma unroll
      for (int q = 2; q >= 0; --q) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c, w.w[q][t], acc[b], 0, 0, 0);
    }
}
// the same where both operands are tiles in LDS: acc[b][d][col] += sum over rows of tile[row][32 b + d] w[row][col]
template <bool BF, int DP>
__device__ __forceinline__ void add_cols_lds(const typename Row<BF, DP>::T* tile, const typename Row<BF, DP>::T* w, f32x16_t (&acc)[DP / 32], int lane) {
  constexpr int PITCH = Row<BF, DP>::PITCH, WP = Row<BF, 32>::PITCH;
  if constexpr (BF) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8_t o = read_col(w, WP, 0, t, lane);
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_col(tile, PITCH, b, t, lane), o, acc[b], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = 16 * (lane >> 5) + v;
      const float o = w[r * WP + (lane & 31)];
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[r * PITCH + 32 * b + (lane & 31)], o, acc[b], 0, 0, 0);
    }
  }
}
// a lane's sixteen weights as row lane & 31 of a tile in LDS, columns 16 g + 0..15
template <bool BF>
__device__ __forceinline__ void weights_to_lds(const Weights<BF>& w, typename Row<BF, 32>::T* tile, int lane) {
  if constexpr (BF) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      *reinterpret_cast<u32x4_t*>(tile + piece_at(lane & 31, 2 * (lane >> 5) + t, Row<BF, 32>::PITCH)) = __builtin_bit_cast(u32x4_t, w.w[t]);
  } else {
    typename Row<BF, 32>::T* p = tile + (lane & 31) * Row<BF, 32>::PITCH + 16 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<float4*>(p + 4 * t) = make_float4(w.w[4 * t], w.w[4 * t + 1], w.w[4 * t + 2], w.w[4 * t + 3]);
  }
}

// byte v of a lane's sixteen buckets, shifted left by SH: the place of its entry in a table of 4- or 8-byte entries (one instruction)
template <int SH>
__device__ __forceinline__ unsigned entry_of(const u32x4_t& w, int v) {
  const unsigned x = w[v >> 2], sh = SH;
  unsigned r;
  switch (v & 3) {
    case 0: asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(sh), "v"(x)); break;
    case 1: asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(sh), "v"(x)); break;
    case 2: asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(sh), "v"(x)); break;
    default: asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(sh), "v"(x)); break;
  }
  return r;
}
// LDS by its address (the kernels have no LDS but the dynamic one, which begins at 0)
template <class V>
using Lds = __attribute__((address_space(3))) V;
typedef float f32x2v_t __attribute__((ext_vector_type(2)));
template <class V>
__device__ __forceinline__ Lds<V>& lds(unsigned at) { return *(Lds<V>*)(uintptr_t)at; }

// the buckets of the keys j0 + 16 g + 0..15 of a row; those past the graph's last atom become HGNN_PAIR_NONE
__device__ __forceinline__ u32x4_t load_buckets(const uint8_t* at, int j0, int n, int g) {
  u32x4_t w = *reinterpret_cast<const u32x4_t*>(at);
  if (j0 + 32 > n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int left = n - (j0 + 16 * g + 4 * k);   // valid bytes of this word
      if (left < 4) w[k] |= left <= 0 ? 0xffffffffu : 0xffffffffu << (8 * left);
    }
  }
  return w;
}

// The table of one head's biases in units of the product: 256 entries, -inf for what is no bucket (a wavefront fills its own, or the
// same as the others). A finite bias stays finite: a row of the lowest values is still a softmax over its pairs. In two
// steps, so that the wait for the biases does not hold up the loads behind it.
__device__ __forceinline__ float read_bias(const float* bias, int nb, int lane) { return bias[min(lane, nb - 1)]; }   // (nb <= 64)
__device__ __forceinline__ void fill_table(float* table, float x, int nb, float inv, int lane) {
  const float v = fabsf(x) < __builtin_inff() ? fminf(fmaxf(x * inv, -3.4028235e38f), 3.4028235e38f) : x;
  table[lane] = lane < nb ? v : -__builtin_inff();
#pragma unroll
  for (int k = 1; k < 4; ++k) table[k * 64 + lane] = -__builtin_inff();
}
__device__ __forceinline__ f32x16_t biases(unsigned table, const u32x4_t& w) {
  f32x16_t t;
#pragma unroll
  for (int i = 0; i < 16; ++i) t[i] = lds<const float>(entry_of<2>(w, i) + table);
  return t;
}

// weights of sixteen scores (in units of the product): 2^(c (s - m) - l). Where every c m is small the exponent is one multiply-add;
// a large one would lose its low places there (a bias of -1e9 as a mask), and s - m comes first.
__device__ __forceinline__ void weights_of(f32x16_t& s, float c, float m, float l) {
  const float cm = c * m;
  if (__all(fabsf(cm) <= 64.f)) {
    const float e = -cm - l;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, e));
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i] - m, c, -l));
  }
}

template <bool BF>
__device__ __forceinline__ float value(const void* p, size_t i) {
  if constexpr (BF) return __uint_as_float((unsigned)static_cast<const unsigned short*>(p)[i] << 16);
  else return static_cast<const float*>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void put(void* p, size_t i, float v) {
  if constexpr (BF) static_cast<unsigned short*>(p)[i] = (unsigned short)f2bf_bits(v);
  else static_cast<float*>(p)[i] = v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// four neighbouring dims of a row (accumulator registers 4 q .. 4 q + 3 of block b), times f
template <bool BF>
__device__ __forceinline__ void store4(void* base, size_t i, const f32x16_t& a, int q, float f) {
  if constexpr (BF) {
    const uint2 u = make_uint2(pack_bf16x2(a[4 * q] * f, a[4 * q + 1] * f), pack_bf16x2(a[4 * q + 2] * f, a[4 * q + 3] * f));
    *reinterpret_cast<uint2*>(static_cast<unsigned short*>(base) + i) = u;
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(base) + i) = make_float4(a[4 * q] * f, a[4 * q + 1] * f, a[4 * q + 2] * f, a[4 * q + 3] * f);
  }
}

// whether every value is finite, over the wavefront
template <int NB>
__device__ __forceinline__ bool all_finite(const f32x16_t (&acc)[NB], float more, bool counts) {
  float z = more * 0.f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int v = 0; v < 16; ++v) z = fmaf(acc[b][v], 0.f, z);
  return __all(!counts || z == 0.f);
}

// Item of a workgroup: tile (or share of the tiles) i and head h of `heads`. Workgroups are dealt to the 8 XCDs in turn. near: ITEM_TILES
// consecutive tiles with all their heads go to one XCD, so that the heads of an atom, parts of one line of qkv, out and the
// gradients, meet in one L2 (the next to the next XCD: graphs may be sorted by size). Else, in long graphs, the heads of a tile
// go to different XCDs: each gets few heads, whose keys and values its L2 can hold.
constexpr unsigned ITEM_TILES = 4;
__device__ __forceinline__ void item_of(int near, unsigned block, unsigned heads, int& i, int& h) {
  if (near) {
    const unsigned place = block >> 3, run = place / (ITEM_TILES * heads), r = place - run * (ITEM_TILES * heads);
    i = (run * 8 + (block & 7)) * ITEM_TILES + r / heads;
    h = r % heads;
  } else {
    i = block / heads;
    h = block - i * heads;
  }
}
// workgroups for n items a head
int64_t item_blocks(int near, int64_t n, int heads) { return near ? (n + 8 * ITEM_TILES - 1) / (8 * ITEM_TILES) * (8 * ITEM_TILES) * heads : n * heads; }

// where a workgroup's rows are (t: uniform)
struct Where {
  int lo, n, i0;           // the graph's first atom, its atoms, first row of the tile
  int64_t pitch;
  const uint8_t* pairs;    // the graph's matrix
};
__device__ __forceinline__ Where tile_where(const AttnArgs& a, int t) {
  const PairTile r = a.plan.tile[t < a.plan.max_tiles ? t : a.plan.max_tiles - 1];   // (also asked for before t is known to exist)
  Where w;
  w.lo = r.lo;
  w.n = r.n;
  w.i0 = r.i0;
  w.pitch = pair_pitch(r.n);
  w.pairs = a.pairs + r.off;
  return w;
}

// LDS: the tables first, then each wavefront's tiles (and over them, when they have been used, its share of a join)
template <bool BF, int DP>
constexpr int tile_bytes() { return 32 * Row<BF, DP>::PITCH * (BF ? 2 : 4); }
constexpr int TABLE = 1024;
template <bool BF, int DP>
__host__ __device__ constexpr int fwd_wave_bytes() { return 2 * tile_bytes<BF, DP>() + 256; }
template <bool BF, int DP, int COLS>
__host__ __device__ constexpr int dq_wave_bytes(int nb) { return 2 * tile_bytes<BF, DP>() + (nb + 1) * COLS * 4; }
template <bool BF, int DP>
constexpr int dkv_wave_bytes() { return 2 * tile_bytes<BF, DP>() + 2 * tile_bytes<BF, 32>(); }

// x of the wavefronts of a workgroup, added in order: the sum is wavefront 0's. room: that of wavefront 0; the others' are `stride`
// bytes on. The barriers around it keep what lies there before and after.
template <int NB>
__device__ __forceinline__ void join_sum(f32x16_t (&x)[NB], char* room, int stride, int nw, int wave, int lane) {
  __syncthreads();
  if (wave) {
    float* mine = reinterpret_cast<float*>(room + wave * stride);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(b * 16 + i) * 64 + lane] = x[b][i];
  }
  __syncthreads();
  if (wave == 0) {
    for (int k = 1; k < nw; ++k) {
      const float* theirs = reinterpret_cast<const float*>(room + k * stride);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[b][i] += theirs[(b * 16 + i) * 64 + lane];
    }
  }
  __syncthreads();
}

// -------------------------------------------------------------------------------------------------------------------------
template <bool BF, int DP, bool SPLIT>
__global__ void __launch_bounds__(256, DP == 128 ? 1 : 2) k_attn_fwd(AttnArgs a) {
  using T = typename Row<BF, DP>::T;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, wave = SPLIT ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, g = lane >> 5;
  int t, h;
  item_of(a.near, blockIdx.x, a.nh, t, h);
  const int ntiles = *a.plan.count;
  const Where w = tile_where(a, t);
  asm volatile("" ::"s"(w.lo));   // both loads before either is waited for
  if (t >= ntiles) return;   // uniform over the workgroup
  float* table = reinterpret_cast<float*>(smem);
  T* tk = reinterpret_cast<T*>(smem + TABLE + wave * fwd_wave_bytes<BF, DP>());
  T* tv = tk + 32 * Row<BF, DP>::PITCH;
  const float my_bias = read_bias(a.bias + (size_t)h * a.nb, a.nb, lane);

  const int hk = h / (a.nh / a.nkv);
  const unsigned ld = (unsigned)(a.nh + 2 * a.nkv) * a.dh;   // elements of an atom's q, k, v
  const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
  const int qi = w.i0 + (lane & 31), ql = min(lane & 31, w.n - 1 - w.i0);
  Row<BF, DP> q, k;
  q.load(base + (size_t)w.i0 * ld + (size_t)h * a.dh + ql * ld, a.dh, g);
  const T* kbase = base + (size_t)(a.nh + hk) * a.dh;
  const T* vbase = kbase + (size_t)a.nkv * a.dh;
  const uint8_t* prow = w.pairs + w.i0 * w.pitch;
  const unsigned pl = (unsigned)ql * (unsigned)w.pitch + 16 * g;
  Tile<BF, DP> kt, vt;
  u32x4_t bk;
  auto fetch = [&](int j0) {   // (addresses: a uniform one and a lane's offset within the tile)
    kt.load(kbase + (size_t)j0 * ld, ld, w.n - j0, a.dh, lane);
    vt.load(vbase + (size_t)j0 * ld, ld, w.n - j0, a.dh, lane);
    bk = load_buckets(prow + j0 + pl, j0, w.n, g);
  };

  float m = -__builtin_inff(), l = 0.f;   // m in units of the product
  f32x16_t o[DP / 32] = {};
  const int step = SPLIT ? a.nw * PAIR_T : PAIR_T;
  const float slack = 8.f / a.c;
  int j0 = wave * PAIR_T;
  if (j0 < w.n) fetch(j0);
  fill_table(table, my_bias, a.nb, a.inv, lane);   // (SPLIT: the same values by every wavefront)
  for (; j0 < w.n; j0 += step) {
    lds_order();
    kt.to_lds(tk, lane);
    vt.to_lds(tv, lane);
    f32x16_t s = biases(0, bk);
    lds_order();
    if (j0 + step < w.n) fetch(j0 + step);
    k.from_lds(tk, tile_row(lane & 31), g);
    s = Row<BF, DP>::dot(k, q, s);
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(top, other_half(top));
    // the sums are rescaled only where a maximum has grown by 2^8: weights up to that size lose nothing
    if (__any(top > m + slack || (m == -__builtin_inff() && top > m))) {
      const float mn = fmaxf(m, top), f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.c);
      m = mn;
      l *= f;
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
    }
    weights_of(s, a.c, m == -__builtin_inff() ? 0.f : m, 0.f);
    float l4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
    for (int i = 4; i < 16; ++i) l4[i & 3] += s[i];
    l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
    // bf16: the weights enter as they are, as three terms. The reverse pass takes D from the output, and a rounding of the weights
    // there is more than the bias gradient, a sum of differences over all pairs, can bear (two terms: off by 1e-6 to 7e-6 where
    // float32 is off by 1e-7 to 2e-6)
    if constexpr (BF) add_cols3<DP>(tv, Weights3(s), o, lane);
    else add_cols<BF, DP>(tv, Weights<BF>(s), o, lane);
  }
  l += other_half(l);

  if constexpr (SPLIT) {   // the wavefronts' shares, in order
    constexpr int WB = fwd_wave_bytes<BF, DP>();
    __syncthreads();
    if (wave) {
      float* mine = reinterpret_cast<float*>(smem + TABLE + wave * WB);
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine[(b * 16 + i) * 64 + lane] = o[b][i];
      if (lane < 32) { mine[DP * 32 + lane] = m; mine[DP * 32 + 32 + lane] = l; }
    }
    __syncthreads();
    if (wave) return;
    for (int k2 = 1; k2 < a.nw; ++k2) {   // (a sum that is no number stays one)
      const float* jo = reinterpret_cast<const float*>(smem + TABLE + k2 * WB);
      const float m2 = jo[DP * 32 + (lane & 31)], l2 = jo[DP * 32 + 32 + (lane & 31)], mn = fmaxf(m, m2);
      const float f1 = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.c);
      const float f2 = m2 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m2 - mn) * a.c);
      l = l * f1 + l2 * f2;
      m = mn;
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = o[b][i] * f1 + jo[(b * 16 + i) * 64 + lane] * f2;
    }
  }

  const size_t orow = ((size_t)w.lo + qi) * a.nh + h;   // row of out
  if (all_finite<DP / 32>(o, l, qi < w.n)) {
    if (qi < w.n) {
      const float f = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = 32 * b + 8 * r + 4 * g;
          if (d < a.dh) {
            store4<BF>(a.out, orow * a.dh + d, o[b], r, f);
            if (BF && a.o32) store4<false>(a.o32, orow * a.dh + d, o[b], r, f);
          }
        }
      if (a.stat && g == 0) a.stat[(size_t)h * a.N + w.lo + qi] = l > 0.f ? make_float2(m, __log2f(l)) : make_float2(0.f, __builtin_inff());
    }
    return;
  }
  // pair by pair: lanes are dims (lane and lane + 64)
  const bool d0 = lane < a.dh, d1 = lane + 64 < a.dh;
  for (int r = 0; r < PAIR_T && w.i0 + r < w.n; ++r) {
    const size_t at = ((size_t)w.lo + w.i0 + r) * ld + (size_t)h * a.dh;
    const float q0 = d0 ? value<BF>(a.qkv, at + lane) : 0.f, q1 = d1 ? value<BF>(a.qkv, at + lane + 64) : 0.f;
    const uint8_t* row = w.pairs + (w.i0 + r) * w.pitch;
    float mr = -__builtin_inff(), lr = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j = 0; j < w.n; ++j) {
      const float b = table[row[j]];
      if (b == -__builtin_inff()) continue;
      const size_t kj = ((size_t)w.lo + j) * ld + (size_t)(a.nh + hk) * a.dh, vj = kj + (size_t)a.nkv * a.dh;
      const float k0 = d0 ? value<BF>(a.qkv, kj + lane) : 0.f, k1 = d1 ? value<BF>(a.qkv, kj + lane + 64) : 0.f;
      const float v0 = d0 ? value<BF>(a.qkv, vj + lane) : 0.f, v1 = d1 ? value<BF>(a.qkv, vj + lane + 64) : 0.f;
      const float s = wave_sum(fmaf(q0, k0, q1 * k1)) + b;
      if (s == -__builtin_inff()) continue;
      const float mn = fmaxf(mr, s), f = mr == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((mr - mn) * a.c), p = __builtin_amdgcn_exp2f((s - mn) * a.c);
      mr = mn;
      lr = lr * f + p;
      o0 = o0 * f + p * v0;
      o1 = o1 * f + p * v1;
    }
    const size_t out = (((size_t)w.lo + w.i0 + r) * a.nh + h) * a.dh;
    const float f = lr == 0.f ? 0.f : 1.0f / lr;
    if (d0) { put<BF>(a.out, out + lane, o0 * f); if (BF && a.o32) a.o32[out + lane] = o0 * f; }
    if (d1) { put<BF>(a.out, out + lane + 64, o1 * f); if (BF && a.o32) a.o32[out + lane + 64] = o1 * f; }
    if (a.stat && lane == 0) a.stat[(size_t)h * a.N + w.lo + w.i0 + r] = lr == 0.f ? make_float2(0.f, __builtin_inff()) : make_float2(mr, __log2f(lr));
  }
}

// The sums of g_bias of a wavefront: COLS words of LDS per bucket, and as many more for the pairs that are left out. 64: a column per
// lane. 32, in long graphs: lanes i and i + 32 share one and take turns, and twice as many wavefronts fit a compute unit.
template <int COLS>
__device__ __forceinline__ float hist_sum(const float* hist, int b) {   // (a lane per bucket: the columns from its own on, so that no bank is hit twice)
  float s[8] = {};
#pragma unroll
  for (int k = 0; k < COLS; ++k) s[k & 7] += hist[b * COLS + ((k + b) & (COLS - 1))];
  return ((s[0] + s[4]) + (s[1] + s[5])) + ((s[2] + s[6]) + (s[3] + s[7]));
}

// Adds to this lane's words, HB at a time: they are read together, and one that is named twice takes up what the earlier one has
// made of it. (Adding in LDS itself, ds_add_f32, took 210 cycles of the compute unit for 64 words; four at a time, with six
// comparisons, were slower than two.)
constexpr int HB = 2;
template <int COLS>
__device__ __forceinline__ void hist_at(const u32x4_t& bk, int i, int nb, unsigned col, unsigned (&at)[HB]) {
#pragma unroll
  for (int k = 0; k < HB; ++k) at[k] = min(entry_of<COLS == 64 ? 8 : 7>(bk, i + k), (unsigned)nb * (COLS * 4)) + col;
}
__device__ __forceinline__ void hist_read(const unsigned (&at)[HB], float (&v)[HB]) {
#pragma unroll
  for (int k = 0; k < HB; ++k) v[k] = lds<float>(at[k]);
}
__device__ __forceinline__ void hist_add(const unsigned (&at)[HB], float (&v)[HB], const f32x16_t& x, int i) {
#pragma unroll
  for (int k = 0; k < HB; ++k) {
#pragma unroll
    for (int u = 0; u < k; ++u) v[k] = at[k] == at[u] ? v[u] : v[k];
    v[k] += x[i + k];
  }
#pragma unroll
  for (int k = 0; k < HB; ++k) lds<float>(at[k]) = v[k];
}
// bytes of w that differ from those of v
__device__ __forceinline__ int bytes_unlike(unsigned w, unsigned v) {
  const unsigned t = w ^ v;
  return __popc((((t & 0x7f7f7f7fu) + 0x7f7f7f7fu) | t) & 0x80808080u);
}

// wavefronts that a SIMD's registers hold of the reverse kernel over queries
constexpr int dq_waves(bool bf16, int dp) { return dp == 128 || (!bf16 && dp == 64) ? 1 : bf16 && dp == 32 ? 3 : 2; }

// -------------------------------------------------------------------------------------------------------------------------
// g_q of 32 queries, D of theirs, and g_bias. A workgroup of head h takes tiles me, me + per_head, ...
// LONG (graphs of 1,024 atoms and more, SPLIT): nearly all pairs of most tiles are in the last bucket. Those are added up in a register,
// the few others one by one in LDS, where an addition takes some three cycles a lane that takes part.
template <bool BF, int DP, bool SPLIT, bool LONG>
__global__ void __launch_bounds__(256, dq_waves(BF, DP)) k_attn_dq(AttnArgs a) {
  using T = typename Row<BF, DP>::T;
  constexpr int COLS = LONG ? 32 : 64;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, wave = SPLIT ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, g = lane >> 5;
  int me, h;
  item_of(a.near, blockIdx.x, a.nh, me, h);
  if (me >= a.per_head) return;   // uniform over the workgroup
  const int wave_bytes = dq_wave_bytes<BF, DP, COLS>(a.nb);
  float* table = reinterpret_cast<float*>(smem);
  T* tk = reinterpret_cast<T*>(smem + TABLE + wave * wave_bytes);
  T* tv = tk + 32 * Row<BF, DP>::PITCH;
  const unsigned hist0 = TABLE + wave * wave_bytes + 2 * tile_bytes<BF, DP>();
  float* hist = reinterpret_cast<float*>(smem + hist0);
  const float my_bias = read_bias(a.bias + (size_t)h * a.nb, a.nb, lane);
  for (int b = lane; b < (a.nb + 1) * COLS; b += 64) hist[b] = 0.f;
  const unsigned col = hist0 + (lane & (COLS - 1)) * 4;
  float far_sum = 0.f;
  const int hk = h / (a.nh / a.nkv);
  const unsigned ld = (unsigned)(a.nh + 2 * a.nkv) * a.dh, lo_ = (unsigned)a.nh * a.dh;
  const int ntiles = *a.plan.count;
  // The matrix cores' sums of bf16 products are low by a hundredth of a step (6e-10 for 32 terms of size 1, measured), whatever their sign.
  // In g_bias the rows would add that up (20,000 rows: 1.2e-5, half of its error), so every other wavefront works with -g and -D, and
  // so with -ds, up to its sums.
  const bool minus = ((wave ^ me) & 1) != 0;

  for (int t = me; t < ntiles; t += a.per_head) {   // uniform over the workgroup
    const Where w = tile_where(a, t);
    const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
    const int qi = w.i0 + (lane & 31), ql = min(lane & 31, w.n - 1 - w.i0);
    const bool real = qi < w.n;
    Row<BF, DP> q, go, k, v;
    q.load(base + (size_t)w.i0 * ld + (size_t)h * a.dh + ql * ld, a.dh, g);
    const size_t orow = ((size_t)w.lo + w.i0) * lo_ + (size_t)h * a.dh;
    go.load(static_cast<const T*>(a.g_out) + orow + ql * lo_, a.dh, g);
    float2 st = a.stat[(size_t)h * a.N + w.lo + w.i0 + ql];
    const T* kbase = base + (size_t)(a.nh + hk) * a.dh;
    const uint8_t* prow = w.pairs + w.i0 * w.pitch;
    const T* vbase = kbase + (size_t)a.nkv * a.dh;
    const unsigned pl = (unsigned)ql * (unsigned)w.pitch + 16 * g;
    const unsigned none = real ? 0u : 0xffffffffu;   // a row past the last atom: no pairs
    Tile<BF, DP> kt, vt;
    u32x4_t bk;
    auto fetch = [&](int j0) {
      kt.load(kbase + (size_t)j0 * ld, ld, w.n - j0, a.dh, lane);
      vt.load(vbase + (size_t)j0 * ld, ld, w.n - j0, a.dh, lane);
      bk = load_buckets(prow + j0 + pl, j0, w.n, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) bk[i] |= none;
    };
    f32x16_t dq[DP / 32] = {};
    const int step = SPLIT ? a.nw * PAIR_T : PAIR_T;
    int j0 = wave * PAIR_T;
    if (j0 < w.n) fetch(j0);
    float D = go.dot32((BF ? a.o32 : static_cast<const float*>(a.out)) + orow + ql * lo_, a.dh, g);
    D += other_half(D);
    if (!real) st = make_float2(0.f, __builtin_inff());
    if (real && g == 0 && wave == 0) a.delta[(size_t)h * a.N + w.lo + qi] = D;
    if (t == me) fill_table(table, my_bias, a.nb, a.inv, lane);
    const float Ds = minus ? -D : D;
    go.negate_if(minus);
    for (; j0 < w.n; j0 += step) {
      lds_order();
      kt.to_lds(tk, lane);
      vt.to_lds(tv, lane);
      f32x16_t s = biases(0, bk);
      const u32x4_t bc = bk;
      bool far = false;
      if constexpr (LONG) {
        int others = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) others += bytes_unlike(bc[i], (a.nb - 1) * 0x01010101u);
        far = !__any(others > 3);
      }
      lds_order();
      if (j0 + step < w.n) fetch(j0 + step);
      k.from_lds(tk, tile_row(lane & 31), g);
      s = Row<BF, DP>::dot(k, q, s);
      v.from_lds(tv, tile_row(lane & 31), g);
      f32x16_t ds = Row<BF, DP>::dot(v, go, f32x16_t{});
      unsigned at[HB];
      float h2[HB];
      if (!LONG) {   // (the first words of the sums are on their way while the weights are formed, the next while the ones before are added)
        hist_at<COLS>(bc, 0, a.nb, col, at);
        hist_read(at, h2);
      }
      weights_of(s, a.c, st.x, st.y);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ds[i] = s[i] * (ds[i] - Ds);
        if (!LONG && i % HB == HB - 1) {
          hist_add(at, h2, ds, i - (HB - 1));
          if (i < 15) {
            hist_at<COLS>(bc, i + 1, a.nb, col, at);
            hist_read(at, h2);
          }
        }
      }
      if constexpr (LONG) {
        const unsigned last = (a.nb - 1) * 128u;
        if (far) {
          float tile = 0.f;   // (the tile's first: thousands of terms in one chain would lose places)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const unsigned e = entry_of<7>(bc, i);
            tile += e == last ? ds[i] : 0.f;
            if (__any(e < last)) {   // (the two lanes of a column, one after the other: the fences keep both turns apart, and from the next place's)
              if (e < last && g == 0) __hip_atomic_fetch_add(&lds<float>(e + col), ds[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
              lds_order();
              if (e < last && g == 1) __hip_atomic_fetch_add(&lds<float>(e + col), ds[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
              lds_order();
            }
          }
          far_sum += tile;
        } else {
          for (int half = 0; half < 2; ++half) {
            if (g == half) {
#pragma unroll
              for (int i = 0; i < 16; i += HB) {
                hist_at<COLS>(bc, i, a.nb, col, at);
                hist_read(at, h2);
                hist_add(at, h2, ds, i);
              }
            }
            lds_order();
          }
        }
      }
      add_cols<BF, DP>(tk, Weights<BF>(ds), dq, lane);
    }
    if (minus) {
#pragma unroll
      for (int b = 0; b < DP / 32; ++b) dq[b] = -dq[b];
    }
    if constexpr (SPLIT) {
      static_assert(DP * 128 <= 2 * tile_bytes<BF, DP>(), "room for the join");
      join_sum<DP / 32>(dq, smem + TABLE, wave_bytes, a.nw, wave, lane);
      if (wave) continue;
    }
    T* gq = static_cast<T*>(a.g_qkv) + (size_t)w.lo * ld + (size_t)h * a.dh;
    if (all_finite<DP / 32>(dq, 0.f, real)) {
      if (real) {
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 32 * b + 8 * r + 4 * g;
            if (d < a.dh) store4<BF>(gq, (size_t)qi * ld + d, dq[b], r, a.scale);
          }
      }
      continue;
    }
    const bool d0 = lane < a.dh, d1 = lane + 64 < a.dh;
    for (int r = 0; r < PAIR_T && w.i0 + r < w.n; ++r) {
      const size_t qa = ((size_t)w.lo + w.i0 + r) * ld + (size_t)h * a.dh, og = (((size_t)w.lo + w.i0 + r) * a.nh + h) * a.dh;
      const float q0 = d0 ? value<BF>(a.qkv, qa + lane) : 0.f, q1 = d1 ? value<BF>(a.qkv, qa + lane + 64) : 0.f;
      const float g0 = d0 ? value<BF>(a.g_out, og + lane) : 0.f, g1 = d1 ? value<BF>(a.g_out, og + lane + 64) : 0.f;
      const float mr = __shfl(st.x, r), lr = __shfl(st.y, r), Dr = __shfl(D, r);
      const uint8_t* row = w.pairs + (w.i0 + r) * w.pitch;
      float a0 = 0.f, a1 = 0.f;
      for (int j = 0; j < w.n; ++j) {
        const float b = table[row[j]];
        if (b == -__builtin_inff()) continue;
        const size_t kj = ((size_t)w.lo + j) * ld + (size_t)(a.nh + hk) * a.dh, vj = kj + (size_t)a.nkv * a.dh;
        const float k0 = d0 ? value<BF>(a.qkv, kj + lane) : 0.f, k1 = d1 ? value<BF>(a.qkv, kj + lane + 64) : 0.f;
        const float v0 = d0 ? value<BF>(a.qkv, vj + lane) : 0.f, v1 = d1 ? value<BF>(a.qkv, vj + lane + 64) : 0.f;
        const float p = __builtin_amdgcn_exp2f(fmaf(wave_sum(fmaf(q0, k0, q1 * k1)) + b - mr, a.c, -lr));
        const float d = p * (wave_sum(fmaf(g0, v0, g1 * v1)) - Dr);
        a0 = fmaf(d, k0, a0);
        a1 = fmaf(d, k1, a1);
      }
      if (d0) put<BF>(a.g_qkv, qa + lane, a0 * a.scale);
      if (d1) put<BF>(a.g_qkv, qa + lane + 64, a1 * a.scale);
    }
  }

  if constexpr (LONG) {
    far_sum += other_half(far_sum);
    if (g == 0) lds<float>((a.nb - 1) * 128u + col) += far_sum;
  }
  lds_order();
  if constexpr (SPLIT) __syncthreads();
  if (wave == 0 && lane < a.nb) {
    float s = 0.f;
    for (int k2 = 0; k2 < (SPLIT ? a.nw : 1); ++k2) {
      const float x = hist_sum<COLS>(reinterpret_cast<const float*>(smem + hist0 + k2 * wave_bytes), lane);
      s += (k2 ^ me) & 1 ? -x : x;
    }
    a.partial[((size_t)h * a.per_head + me) * a.nb + lane] = s;
  }
}

// g_bias of head h: the workgroups' partials in order, a run per group of threads (8 to 64, as many as there are buckets), then the runs, in
// double precision: a bucket's partials nearly cancel (20,000 atoms: to 3e-4 of the sum of |ds|)
__device__ __forceinline__ void bias_reduce(const AttnArgs& a, int h, double* sh) {
  const int w = a.nb <= 8 ? 8 : a.nb <= 16 ? 16 : a.nb <= 32 ? 32 : 64;
  const int b = threadIdx.x & (w - 1), run = threadIdx.x / w, runs = blockDim.x / w;
  const int per = (a.per_head + runs - 1) / runs, k1 = min(a.per_head, (run + 1) * per);
  double s = 0.0;
  if (b < a.nb) {
    const float* p = a.partial + (size_t)h * a.per_head * a.nb + b;
    for (int k = run * per; k < k1; k += 32) {   // 32 loads on their way at a time: the chain of their waits is the kernel's on small batches
      float v[32];
#pragma unroll
      for (int u = 0; u < 32; ++u) v[u] = p[(size_t)min(k + u, k1 - 1) * a.nb];
#pragma unroll
      for (int u = 0; u < 32; ++u) s += k + u < k1 ? v[u] : 0.f;
    }
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (run == 0 && b < a.nb) {
    for (int k = 1; k < runs; ++k) s += sh[k * w + b];
    if (a.bias[(size_t)h * a.nb + b] == -__builtin_inff()) s = 0.0;   // its pairs are left out
    a.g_bias[(size_t)h * a.nb + b] = (float)s;
  }
}

// -------------------------------------------------------------------------------------------------------------------------
// g_k and g_v of 32 keys, over the query heads that share them; the first nh workgroups add up g_bias
template <bool BF, int DP, bool SPLIT>
__global__ void __launch_bounds__(256, DP == 128 || (!BF && DP == 64) ? 1 : 2) k_attn_dkv(AttnArgs a) {
  using T = typename Row<BF, DP>::T;
  constexpr int PT = Row<BF, 32>::PITCH;
  extern __shared__ __align__(16) char smem[];
  if ((int)blockIdx.x < a.nh) {   // uniform over the workgroup
    bias_reduce(a, blockIdx.x, reinterpret_cast<double*>(smem));
    return;
  }
  const int lane = threadIdx.x & 63, wave = SPLIT ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, g = lane >> 5;
  const unsigned item = blockIdx.x - a.nh;
  int t, hk;
  item_of(a.near, item, a.nkv, t, hk);
  const int ntiles = *a.plan.count;
  const Where w = tile_where(a, t);
  asm volatile("" ::"s"(w.lo));   // (as in k_attn_fwd)
  if (t >= ntiles) return;
  // (tables: wavefronts of one workgroup may be at different heads, so each has its own)
  const unsigned table_at = wave * TABLE;
  float* table = reinterpret_cast<float*>(smem + table_at);
  T* tq = reinterpret_cast<T*>(smem + (SPLIT ? a.nw : 1) * TABLE + wave * dkv_wave_bytes<BF, DP>());
  T* tg = tq + 32 * Row<BF, DP>::PITCH;
  T* tp = tg + 32 * Row<BF, DP>::PITCH;
  T* ts = tp + 32 * PT;
  const int rep = a.nh / a.nkv;
  const unsigned ld = (unsigned)(a.nh + 2 * a.nkv) * a.dh, lo_ = (unsigned)a.nh * a.dh;
  const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
  const T* gbase = static_cast<const T*>(a.g_out) + (size_t)w.lo * lo_;
  Row<BF, DP> k, v, q, go;
  {
    const T* p = base + (size_t)(w.i0 + min(tile_row(lane & 31), w.n - 1 - w.i0)) * ld + (size_t)(a.nh + hk) * a.dh;
    k.load(p, a.dh, g);
    v.load(p + (size_t)a.nkv * a.dh, a.dh, g);
  }
  f32x16_t dk[DP / 32] = {}, dv[DP / 32] = {};
  // the tiles of queries of one head after the other; SPLIT: dealt out in turn
  const int step = SPLIT ? a.nw * PAIR_T : PAIR_T, span = (w.n + PAIR_T - 1) / PAIR_T * PAIR_T;
  int i0 = wave * PAIR_T;
  for (int r = 0; r < rep; ++r, i0 -= span) {
    if (i0 >= span) continue;
    const int h = hk * rep + r;
    const float my_bias = read_bias(a.bias + (size_t)h * a.nb, a.nb, lane);
    Tile<BF, DP> qt, gt;
    u32x4_t bk;
    float2 st;
    float D;
    auto fetch = [&](int i0) {
      const bool part = i0 + 32 > w.n;
      const unsigned il = part ? min(lane & 31, w.n - 1 - i0) : lane & 31;
      qt.load(base + (size_t)i0 * ld + (size_t)h * a.dh, ld, w.n - i0, a.dh, lane);
      gt.load(gbase + (size_t)i0 * lo_ + (size_t)h * a.dh, lo_, w.n - i0, a.dh, lane);
      bk = load_buckets(w.pairs + i0 * w.pitch + w.i0 + (il * (unsigned)w.pitch + 16 * g), w.i0, w.n, g);
      const size_t at = (size_t)h * a.N + w.lo + i0;
      st = a.stat[at + il];
      D = a.delta[at + il];
      if (part && (lane & 31) > (int)il) st = make_float2(0.f, __builtin_inff());   // a row past the last atom: weight 0
    };
    fetch(i0);
    lds_order();
    fill_table(table, my_bias, a.nb, a.inv, lane);
    for (; i0 < w.n; i0 += step) {
      lds_order();
      qt.to_lds(tq, lane);
      gt.to_lds(tg, lane);
      f32x16_t s = biases(table_at, bk);
      lds_order();
      const float2 sc = st;
      const float Dc = D;
      if (i0 + step < w.n) fetch(i0 + step);
      q.from_lds(tq, lane & 31, g);
      s = Row<BF, DP>::dot(k, q, s);
      go.from_lds(tg, lane & 31, g);
      f32x16_t ds = Row<BF, DP>::dot(v, go, f32x16_t{});
      weights_of(s, a.c, sc.x, sc.y);
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] = s[i] * (ds[i] - Dc);
      weights_to_lds<BF>(Weights<BF>(s), tp, lane);
      weights_to_lds<BF>(Weights<BF>(ds), ts, lane);
      lds_order();
      add_cols_lds<BF, DP>(tg, tp, dv, lane);
      add_cols_lds<BF, DP>(tq, ts, dk, lane);
    }
  }
  if constexpr (SPLIT) {
    char* room = smem + a.nw * TABLE;
    join_sum<DP / 32>(dk, room, dkv_wave_bytes<BF, DP>(), a.nw, wave, lane);
    join_sum<DP / 32>(dv, room, dkv_wave_bytes<BF, DP>(), a.nw, wave, lane);
    if (wave) return;
  }
  const int kj = w.i0 + (lane & 31);
  const size_t gk = (size_t)(a.nh + hk) * a.dh, gv = gk + (size_t)a.nkv * a.dh;
  T* gbase_out = static_cast<T*>(a.g_qkv) + (size_t)w.lo * ld;
  if (all_finite<DP / 32>(dk, 0.f, kj < w.n) && all_finite<DP / 32>(dv, 0.f, kj < w.n)) {
    if (kj < w.n) {
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = 32 * b + 8 * r + 4 * g;
          if (d < a.dh) {
            store4<BF>(gbase_out, (size_t)kj * ld + gk + d, dk[b], r, a.scale);
            store4<BF>(gbase_out, (size_t)kj * ld + gv + d, dv[b], r, 1.f);
          }
        }
    }
    return;
  }
  const bool d0 = lane < a.dh, d1 = lane + 64 < a.dh;
  for (int r = 0; r < PAIR_T && w.i0 + r < w.n; ++r) {
    const size_t at = ((size_t)w.lo + w.i0 + r) * ld;
    const float k0 = d0 ? value<BF>(a.qkv, at + gk + lane) : 0.f, k1 = d1 ? value<BF>(a.qkv, at + gk + lane + 64) : 0.f;
    const float v0 = d0 ? value<BF>(a.qkv, at + gv + lane) : 0.f, v1 = d1 ? value<BF>(a.qkv, at + gv + lane + 64) : 0.f;
    float a0 = 0.f, a1 = 0.f, b0 = 0.f, b1 = 0.f;
    for (int u = 0; u < rep; ++u) {
      const int h = hk * rep + u;
      lds_order();
      fill_table(table, read_bias(a.bias + (size_t)h * a.nb, a.nb, lane), a.nb, a.inv, lane);
      lds_order();
      for (int i = 0; i < w.n; ++i) {
        const float b = table[w.pairs[i * w.pitch + w.i0 + r]];
        if (b == -__builtin_inff()) continue;
        const size_t qa = ((size_t)w.lo + i) * ld + (size_t)h * a.dh, ga = (((size_t)w.lo + i) * a.nh + h) * a.dh;
        const float q0 = d0 ? value<BF>(a.qkv, qa + lane) : 0.f, q1 = d1 ? value<BF>(a.qkv, qa + lane + 64) : 0.f;
        const float g0 = d0 ? value<BF>(a.g_out, ga + lane) : 0.f, g1 = d1 ? value<BF>(a.g_out, ga + lane + 64) : 0.f;
        const float2 st = a.stat[(size_t)h * a.N + w.lo + i];
        const float p = __builtin_amdgcn_exp2f(fmaf(wave_sum(fmaf(q0, k0, q1 * k1)) + b - st.x, a.c, -st.y));
        const float d = p * (wave_sum(fmaf(g0, v0, g1 * v1)) - a.delta[(size_t)h * a.N + w.lo + i]);
        a0 = fmaf(d, q0, a0);
        a1 = fmaf(d, q1, a1);
        b0 = fmaf(p, g0, b0);
        b1 = fmaf(p, g1, b1);
      }
    }
    if (d0) { put<BF>(a.g_qkv, at + gk + lane, a0 * a.scale); put<BF>(a.g_qkv, at + gv + lane, b0); }
    if (d1) { put<BF>(a.g_qkv, at + gk + lane + 64, a1 * a.scale); put<BF>(a.g_qkv, at + gv + lane + 64, b1); }
  }
}

// -------------------------------------------------------------------------------------------------------------------------
// Wavefronts of a workgroup that share a tile, of `items` workgroups: one to four, whichever takes the least time by this count: a
// workgroup's time is its share of a tile, and a compute unit takes `fit` of them at a time, with half a turn idle at the end where
// there is more than one. simd: wavefronts that the registers of a SIMD hold. (Two where four need more than 64 KB: 4,000 atoms,
// 4 heads of 32, float32, reverse 598 us instead of 324. Four wherever they fit: 8 graphs of 700 atoms, 4 heads of 32, bf16, 64
// buckets, reverse 64 us instead of 42. Without the half turn three: 54 us there.)
constexpr int lds_pieces(int bytes) { return (bytes + 1279) / 1280; }   // LDS is given out in pieces of 1,280 bytes, 128 a compute unit
int waves_that_fit(int64_t items, int simd, int wave_bytes, int extra) {
  const double asked = (double)items / num_cus();
  int best = 1;
  double least = 0.0;
  for (int nw = 1; nw <= 4; ++nw) {
    const int lds = 128 / lds_pieces(wave_bytes * nw + extra), regs = 4 * simd / nw, fit = lds < regs ? lds : regs;
    if (fit == 0) break;
    const double time = (asked <= fit ? 1.0 : asked / fit + 0.5) / nw;
    if (nw == 1 || time <= least) { best = nw; least = time; }
  }
  return best;
}
template <class... A>
int32_t allow_lds(void (*kernel)(A...), int bytes) {
  if (bytes > 64 * 1024) HGNN_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  return HGNN_OK;
}

// Long graphs: see attn_split.
bool long_graphs(int64_t G, int64_t N) { return N >= 1024 * G; }

// Workgroups per head of k_attn_dq (each leaves one partial of g_bias): every tile its own while they are few, then as many as run
// at once, which registers and LDS decide. (40,041 atoms in 390 graphs, 8 heads,
// bf16, in runs of 20 passes: 62 us; 72 with a tenth more, 67 with half as many more, 72 with a workgroup per tile.) In long graphs, where a
// tile is a long chain, 4,096 and more are dealt out best.
int64_t dq_per_head(int64_t max_tiles, int32_t N, int32_t G, int nh, int dh, int nb, bool bf16) {
  int64_t at_once = 4096;
  if (!long_graphs(G, N)) {
    const int dp = dh <= 32 ? 32 : dh <= 64 ? 64 : 128;
    const int lds = TABLE + (bf16 ? dp == 32 ? dq_wave_bytes<true, 32, 64>(nb) : dp == 64 ? dq_wave_bytes<true, 64, 64>(nb) : dq_wave_bytes<true, 128, 64>(nb)
                                  : dp == 32 ? dq_wave_bytes<false, 32, 64>(nb) : dp == 64 ? dq_wave_bytes<false, 64, 64>(nb) : dq_wave_bytes<false, 128, 64>(nb));
    const int by_lds = 128 / lds_pieces(lds), by_registers = 4 * dq_waves(bf16, dp);
    at_once = (int64_t)num_cus() * (by_lds < by_registers ? by_lds : by_registers);
  }
  const int64_t most = at_once / nh;
  return max_tiles < most ? max_tiles : most;
}

struct AttnWs {
  float *delta, *partial;
  size_t bytes;
};
AttnWs carve_attn_ws(void* p, int N, int G, int nh, int dh, int nb, bool bf16) {
  Carver c(p);
  AttnWs w;
  w.delta = c.take<float>((size_t)nh * N);
  w.partial = c.take<float>((size_t)nh * dq_per_head(pair_plan_view(nullptr, N, G).max_tiles, N, G, nh, dh, nb, bf16) * nb);
  w.bytes = c.used();
  return w;
}
struct AttnSaved {
  float2* stat;
  float* o32;
  size_t bytes;
};
AttnSaved carve_attn_saved(void* p, int N, int nh, int dh, bool bf16) {
  Carver c(p);
  AttnSaved s;
  s.stat = c.take<float2>((size_t)nh * N);
  s.o32 = bf16 ? c.take<float>((size_t)N * nh * dh) : nullptr;
  s.bytes = c.used();
  return s;
}

constexpr int64_t MOST_THREADS = (int64_t)1 << 32;   // of a launch: it has to have fewer

int32_t check_attn(int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb, int32_t dtype) {
  HGNN_REQUIRE(N >= 0 && G >= 0, HGNN_ERR_BAD_SHAPE, "negative N or G");
  HGNN_REQUIRE(nh >= 1 && nh <= 64 && nkv >= 1 && nh % nkv == 0, HGNN_ERR_BAD_SHAPE,
               "graph_attention: 1..64 heads, a multiple of the key heads (got %d, %d)", nh, nkv);
  HGNN_REQUIRE(dh >= 8 && dh <= 128 && dh % 8 == 0, HGNN_ERR_BAD_SHAPE, "graph_attention: the head width must be a multiple of 8 in 8..128 (got %d)", dh);
  HGNN_REQUIRE(nb >= 1 && nb <= ATTN_BUCKETS, HGNN_ERR_BAD_SHAPE, "graph_attention: 1..%d buckets (got %d)", ATTN_BUCKETS, nb);
  HGNN_REQUIRE(dtype == HGNN_F32 || dtype == HGNN_BF16, HGNN_ERR_BAD_SHAPE, "unknown dtype %d", dtype);
  HGNN_REQUIRE(N < (1 << 28) && G < (1 << 28), HGNN_ERR_OVERFLOW, "graph_attention: N and G must be below 2^28");
  HGNN_REQUIRE((pair_plan_view(nullptr, N, G).max_tiles + 64) * nh < MOST_THREADS / 64, HGNN_ERR_OVERFLOW, "graph_attention: too many tiles for one launch");
  return HGNN_OK;
}

// The wavefronts of a workgroup share a tile of rows and deal out the other side's tiles in two cases. Few tiles: until there is a
// wavefront per SIMD this shortens the chain of tiles without taking a compute unit from anybody. Long graphs: 2,500
// wavefronts of 625 tiles each leave a fifth of the SIMDs idle at the end; four times as many of a quarter the length do not, and
// the join is small against their chains.
// Where keys are shared by query heads, k_attn_dkv has few and long chains as well. (Never where a launch could not hold four
// wavefronts a tile.)
bool attn_split(int64_t max_tiles, int heads, int64_t G, int64_t N, int rep) {
  if ((max_tiles + 64) * (heads * rep) >= MOST_THREADS / 256) return false;
  return (max_tiles * heads <= 4 * num_cus() && N * rep > 2 * PAIR_T * G) || long_graphs(G, N) || rep > 1;
}

template <bool BF, int DP, bool SPLIT>
int32_t launch_fwd(hipStream_t st, AttnArgs a) {
  constexpr int WB = fwd_wave_bytes<BF, DP>(), extra = TABLE;
  a.nw = SPLIT ? waves_that_fit(a.plan.max_tiles * a.nh, DP == 128 ? 1 : DP == 32 ? 4 : BF ? 3 : 2, WB, extra) : 1;
  HGNN_TRY(allow_lds(k_attn_fwd<BF, DP, SPLIT>, WB * a.nw + extra));
  k_attn_fwd<BF, DP, SPLIT><<<(unsigned)item_blocks(a.near, a.plan.max_tiles, a.nh), 64 * a.nw, WB * a.nw + extra, st>>>(a);
  HGNN_LAUNCH_CHECK("k_attn_fwd");
  return HGNN_OK;
}

template <bool BF, int DP, bool SPLIT, bool LONG>
int32_t launch_dq(hipStream_t st, AttnArgs a) {
  const int wb = dq_wave_bytes<BF, DP, LONG ? 32 : 64>(a.nb), extra = TABLE;
  a.nw = SPLIT ? waves_that_fit((int64_t)a.per_head * a.nh, dq_waves(BF, DP), wb, extra) : 1;
  HGNN_TRY(allow_lds(k_attn_dq<BF, DP, SPLIT, LONG>, wb * a.nw + extra));
  k_attn_dq<BF, DP, SPLIT, LONG><<<(unsigned)item_blocks(a.near, a.per_head, a.nh), 64 * a.nw, wb * a.nw + extra, st>>>(a);
  HGNN_LAUNCH_CHECK("k_attn_dq");
  return HGNN_OK;
}

template <bool BF, int DP, bool SPLIT>
int32_t launch_dkv(hipStream_t st, AttnArgs a) {
  constexpr int WB = TABLE + dkv_wave_bytes<BF, DP>();
  a.nw = SPLIT ? waves_that_fit(a.plan.max_tiles * a.nkv, dq_waves(BF, DP), WB, 0) : 1;
  HGNN_TRY(allow_lds(k_attn_dkv<BF, DP, SPLIT>, WB * a.nw));
  k_attn_dkv<BF, DP, SPLIT><<<(unsigned)(item_blocks(a.near, a.plan.max_tiles, a.nkv) + a.nh), 64 * a.nw, WB * a.nw, st>>>(a);
  HGNN_LAUNCH_CHECK("k_attn_dkv");
  return HGNN_OK;
}

template <bool BF, int DP>
int32_t run_width(hipStream_t st, AttnArgs a, bool fwd) {
  // (the keys and values of a graph of average length against the L2 of an XCD, 4 MB)
  a.near = 2.0 * a.N / a.G * a.nkv * a.dh * (BF ? 2 : 4) <= 2e6;
  const bool split = attn_split(a.plan.max_tiles, a.nh, a.G, a.N, 1);
  if (fwd) return split ? launch_fwd<BF, DP, true>(st, a) : launch_fwd<BF, DP, false>(st, a);
  if (long_graphs(a.G, a.N)) HGNN_TRY((launch_dq<BF, DP, true, true>(st, a)));
  else if (split) HGNN_TRY((launch_dq<BF, DP, true, false>(st, a)));
  else HGNN_TRY((launch_dq<BF, DP, false, false>(st, a)));
  return attn_split(a.plan.max_tiles, a.nkv, a.G, a.N, a.nh / a.nkv) ? launch_dkv<BF, DP, true>(st, a) : launch_dkv<BF, DP, false>(st, a);
}

template <bool BF>
int32_t run_attn(hipStream_t st, const AttnArgs& a, bool fwd) {
  if (a.dh <= 32) return run_width<BF, 32>(st, a, fwd);
  if (a.dh <= 64) return run_width<BF, 64>(st, a, fwd);
  return run_width<BF, 128>(st, a, fwd);
}

// (scores are kept in units of the product, biases divided by the scale)
int32_t check_scale(float scale) {
  HGNN_REQUIRE(scale >= 1e-6f && scale <= 1e6f, HGNN_ERR_BAD_SHAPE, "graph_attention: the scale must be in 1e-6..1e6 (got %g)", (double)scale);
  return HGNN_OK;
}

__global__ void k_zero_bias(float* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

}  // namespace
}  // namespace hgnn

using namespace hgnn;

extern "C" int32_t hgnn_graph_attention_workspace_bytes(int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb,
                                                        int32_t dtype, size_t* ws_bytes_host, size_t* saved_bytes_host) {
  HGNN_TRY(check_attn(N, G, nh, nkv, dh, nb, dtype));
  HGNN_REQUIRE(ws_bytes_host && saved_bytes_host, HGNN_ERR_NULLPTR, "null size pointer");
  *ws_bytes_host = carve_attn_ws(nullptr, N, G, nh, dh, nb, dtype == HGNN_BF16).bytes;
  *saved_bytes_host = carve_attn_saved(nullptr, N, nh, dh, dtype == HGNN_BF16).bytes;
  return HGNN_OK;
}

extern "C" int32_t hgnn_graph_attention_fwd(void* stream, int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb,
                                            int32_t dtype, float scale, const void* plan, size_t plan_bytes, const uint8_t* pairs,
                                            const void* qkv, const float* bias, void* out, void* saved, size_t saved_bytes) {
  HGNN_TRY(check_attn(N, G, nh, nkv, dh, nb, dtype));
  HGNN_TRY(check_scale(scale));
  if (N == 0) return HGNN_OK;
  HGNN_REQUIRE(plan && pairs && qkv && bias && out, HGNN_ERR_NULLPTR, "graph_attention_fwd: null pointer");
  AttnArgs a{};
  a.plan = pair_plan_view(plan, N, G);
  HGNN_REQUIRE(plan_bytes >= a.plan.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "pair plan: need %zu bytes, got %zu", a.plan.bytes, plan_bytes);
  const AttnSaved s = carve_attn_saved(saved, N, nh, dh, dtype == HGNN_BF16);
  HGNN_REQUIRE(!saved || saved_bytes >= s.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "graph_attention saved buffer: need %zu bytes, got %zu", s.bytes, saved_bytes);
  if (a.plan.max_tiles == 0) return HGNN_OK;   // (G == 0: no plan of N atoms exists)
  a.N = N; a.G = G; a.nh = nh; a.nkv = nkv; a.dh = dh; a.nb = nb;
  a.scale = scale; a.c = scale * LOG2E; a.inv = 1.0f / scale;
  a.pairs = pairs; a.qkv = qkv; a.bias = bias; a.out = out;
  a.stat = saved ? s.stat : nullptr;
  a.o32 = saved ? s.o32 : nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_ATTENTION, st);
  return dtype == HGNN_BF16 ? run_attn<true>(st, a, true) : run_attn<false>(st, a, true);
}

extern "C" int32_t hgnn_graph_attention_bwd(void* stream, int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb,
                                            int32_t dtype, float scale, const void* plan, size_t plan_bytes, const uint8_t* pairs,
                                            const void* qkv, const float* bias, const void* out, const void* saved, size_t saved_bytes,
                                            const void* g_out, void* g_qkv, float* g_bias, void* ws, size_t ws_bytes) {
  HGNN_TRY(check_attn(N, G, nh, nkv, dh, nb, dtype));
  HGNN_TRY(check_scale(scale));
  HGNN_REQUIRE(g_bias, HGNN_ERR_NULLPTR, "graph_attention_bwd: null pointer");
  hipStream_t st = static_cast<hipStream_t>(stream);
  AttnArgs a{};
  a.plan = pair_plan_view(plan, N, G);
  if (N == 0 || a.plan.max_tiles == 0) {
    k_zero_bias<<<(nh * nb + 255) / 256, 256, 0, st>>>(g_bias, nh * nb);
    HGNN_LAUNCH_CHECK("k_zero_bias");
    return HGNN_OK;
  }
  HGNN_REQUIRE(plan && pairs && qkv && bias && out && saved && g_out && g_qkv && ws, HGNN_ERR_NULLPTR, "graph_attention_bwd: null pointer");
  HGNN_REQUIRE(plan_bytes >= a.plan.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "pair plan: need %zu bytes, got %zu", a.plan.bytes, plan_bytes);
  const AttnSaved s = carve_attn_saved(const_cast<void*>(saved), N, nh, dh, dtype == HGNN_BF16);
  HGNN_REQUIRE(saved_bytes >= s.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "graph_attention saved buffer: need %zu bytes, got %zu", s.bytes, saved_bytes);
  const AttnWs w = carve_attn_ws(ws, N, G, nh, dh, nb, dtype == HGNN_BF16);
  HGNN_REQUIRE(ws_bytes >= w.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "graph_attention workspace: need %zu bytes, got %zu", w.bytes, ws_bytes);
  a.N = N; a.G = G; a.nh = nh; a.nkv = nkv; a.dh = dh; a.nb = nb;
  a.per_head = (int)dq_per_head(a.plan.max_tiles, N, G, nh, dh, nb, dtype == HGNN_BF16);
  a.scale = scale; a.c = scale * LOG2E; a.inv = 1.0f / scale;
  a.pairs = pairs; a.qkv = qkv; a.bias = bias; a.out = const_cast<void*>(out); a.stat = s.stat; a.o32 = s.o32;
  a.g_out = g_out; a.g_qkv = g_qkv; a.delta = w.delta; a.partial = w.partial; a.g_bias = g_bias;
  ProfScope ps(PT_ATTENTION, st);
  return dtype == HGNN_BF16 ? run_attn<true>(st, a, false) : run_attn<false>(st, a, false);
}
