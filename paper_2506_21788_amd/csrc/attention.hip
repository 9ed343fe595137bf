// hgnn_graph_attention_fwd / _bwd: attention over the atoms of each graph with a learned bias per head and pair bucket.
//
//   s_ij = scale q_i . k_j + bias[h][bucket_ij],   p_ij = exp(s_ij - lse_i),   o_i = sum_j p_ij v_j
//   D_i = g_i . o_i,   ds_ij = p_ij (g_i . v_j - D_i),   g_q_i = scale sum_j ds_ij k_j,   g_k_j = scale sum_i ds_ij q_i,
//   g_v_j = sum_i p_ij g_i,   g_bias[h][b] = sum of ds over the pairs of bucket b
//
// One wavefront works alone on 32 rows (queries; keys in k_attn_dkv) and walks the other side in tiles of 32, with the running
// maximum and sum of the softmax: nothing of the size of a graph's pairs is stored. Every score tile is formed transposed,
// S^T[key][query], on 32 x 32 matrix-core tiles. A lane then holds 16 scores of ONE query: the sums over keys are within the
// lane but for one exchange with the other half, the scale factors of a row are one register, and the packed weights are, as
// they stand, the operand of the next product (O^T = V^T P^T, the order of its contraction being free). The rows of the first
// operand are permuted (tile_row) so that the 16 keys of a lane are neighbours: their buckets are one 16-byte load. The bias
// of a bucket is read from a table of 256 in LDS, which holds -inf past the last bucket, so a pair that is left out costs nothing.
// Operands that a product needs by columns go through LDS once, row by row, and come back through transposing reads (bf16)
// or as single values (float32, matrix-core products of float32).
//
// The sums of the reverse pass are split in two kernels (one owns queries, one keys) rather than added with atomics, so that
// their order is fixed: the scores are formed twice. g_bias is collected in LDS, a column per lane and bucket (no two lanes
// share a word), over all tiles that a wavefront takes, and then added up over the wavefronts in order.
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
  int nw;        // wavefronts of a workgroup
  int split;     // 1: they share one tile of rows and deal the other side's tiles out, 0: a tile each
  int per_head;  // wavefronts (split: workgroups) per head
  float scale, c;   // c = scale log2 e
  PairPlan plan;
  const uint8_t* pairs;
  const void* qkv;
  const float* bias;
  void* out;
  float* lse;     // [nh][N] log2 of the sum of exp, +inf for a row without pairs
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

// One row of DP (dh and zeros) per lane pair, as the operand of a product that contracts over it.
// bf16: dims 16 k + 8 g + 0..7 of step k. float32: dims g DP/2 + s of step s.
template <bool BF, int DP>
struct Row;
template <int DP>
struct Row<true, DP> {
  static constexpr int PITCH = DP + 16;   // elements of a row in LDS: rows 0..3 in four different groups of banks
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
  __device__ __forceinline__ void to_lds(T* row, int g) const {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) *reinterpret_cast<u32x4_t*>(row + 16 * k + 8 * g) = f[k];
  }
  __device__ __forceinline__ static f32x16_t dot(const Row& a, const Row& b) {
    f32x16_t acc = {};
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
  __device__ __forceinline__ void to_lds(T* row, int g) const {
#pragma unroll
    for (int k = 0; k < DP / 8; ++k)
      *reinterpret_cast<float4*>(row + g * (DP / 2) + 4 * k) = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
  }
  __device__ __forceinline__ static f32x16_t dot(const Row& a, const Row& b) {
    f32x16_t acc = {};
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

__device__ __forceinline__ bf16x8_t read_tr(const unsigned short* lo, const unsigned short* hi) {
  const s16x4_t l = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(lo));
  const s16x4_t h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(hi));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7));
}
// rows 16 g + 8 t + 0..7 of column col0 + lane & 31 of a tile in LDS
__device__ __forceinline__ bf16x8_t read_col(const unsigned short* tile, int pitch, int col0, int t, int lane) {
  const unsigned short* p = tile + (16 * (lane >> 5) + 8 * t + ((lane & 15) >> 2)) * pitch + col0 + (lane & 16) + (lane & 3) * 4;
  return read_tr(p, p + 4 * pitch);
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
// what is left of them after that rounding
__device__ __forceinline__ Weights<true> remainder_of(const f32x16_t& p, const Weights<true>& w) {
  f32x16_t r;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const u32x4_t u = __builtin_bit_cast(u32x4_t, w.w[t]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r[8 * t + 2 * k] = p[8 * t + 2 * k] - __uint_as_float(u[k] << 16);
      r[8 * t + 2 * k + 1] = p[8 * t + 2 * k + 1] - __uint_as_float(u[k] & 0xffff0000u);
    }
  }
  return Weights<true>(r);
}
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
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_col(tile, PITCH, 32 * b, t, lane), w.w[t], acc[b], 0, 0, 0);
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[(16 * (lane >> 5) + v) * PITCH + 32 * b + (lane & 31)], w.w[v], acc[b], 0, 0, 0);
    }
  }
}
// the same with weights of two bf16 terms
template <int DP>
__device__ __forceinline__ void add_cols2(const unsigned short* tile, const Weights<true>& w, const Weights<true>& w2, f32x16_t (&acc)[DP / 32], int lane) {
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8_t c = read_col(tile, Row<true, DP>::PITCH, 32 * b, t, lane);
      acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c, w2.w[t], acc[b], 0, 0, 0);
      acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c, w.w[t], acc[b], 0, 0, 0);
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
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_col(tile, PITCH, 32 * b, t, lane), o, acc[b], 0, 0, 0);
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
  typename Row<BF, 32>::T* p = tile + (lane & 31) * Row<BF, 32>::PITCH + 16 * (lane >> 5);
  if constexpr (BF) {
#pragma unroll
    for (int t = 0; t < 2; ++t) *reinterpret_cast<u32x4_t*>(p + 8 * t) = __builtin_bit_cast(u32x4_t, w.w[t]);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<float4*>(p + 4 * t) = make_float4(w.w[4 * t], w.w[4 * t + 1], w.w[4 * t + 2], w.w[4 * t + 3]);
  }
}

// byte v of a lane's sixteen buckets
__device__ __forceinline__ unsigned bucket_of(const u32x4_t& w, int v) { return (w[v >> 2] >> (8 * (v & 3))) & 255u; }

// the buckets of the keys j0 + 16 g + 0..15 of a row; those past the graph's last atom become HGNN_PAIR_NONE
__device__ __forceinline__ u32x4_t load_buckets(const uint8_t* row, int j0, int n, int g) {
  const int j = j0 + 16 * g;
  u32x4_t w = *reinterpret_cast<const u32x4_t*>(row + j);
  if (j0 + 32 > n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int left = n - (j + 4 * k);   // valid bytes of this word
      if (left < 4) w[k] |= left <= 0 ? 0xffffffffu : 0xffffffffu << (8 * left);
    }
  }
  return w;
}

// bias table of one head in units of log2 e: 256 entries, -inf for what is no bucket (a wavefront fills its own). A bias of the
// lowest finite value stays finite: such a row is still a softmax over its pairs.
__device__ __forceinline__ void fill_table(float* table, const float* bias, int nb, int lane) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int b = k * 64 + lane;
    float v = -__builtin_inff();
    if (b < nb) {
      const float x = bias[b];
      v = x * LOG2E;
      if (fabsf(x) < __builtin_inff()) v = fminf(fmaxf(v, -3.4028235e38f), 3.4028235e38f);
    }
    table[b] = v;
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

// where a wavefront's rows are
struct Where {
  int g, lo, n, i0;        // graph, its first atom, its atoms, first row of the tile
  int64_t pitch;
  const uint8_t* pairs;    // the graph's matrix
};
__device__ __forceinline__ Where tile_where(const AttnArgs& a, int t) {
  Where w;
  w.g = __builtin_amdgcn_readfirstlane(a.plan.tile_graph[t]);
  w.lo = __builtin_amdgcn_readfirstlane(a.plan.graph_off[w.g]);
  w.n = __builtin_amdgcn_readfirstlane(a.plan.graph_off[w.g + 1]) - w.lo;
  w.i0 = (t - __builtin_amdgcn_readfirstlane(a.plan.tile_off[w.g])) * PAIR_T;
  w.pitch = pair_pitch(w.n);
  w.pairs = a.pairs + a.plan.pair_off[w.g];
  return w;
}

// bytes of LDS of one wavefront (tables first)
template <bool BF, int DP>
constexpr int tile_bytes() { return 32 * Row<BF, DP>::PITCH * (BF ? 2 : 4); }
template <bool BF, int DP>
constexpr int fwd_wave_bytes() { return 1024 + tile_bytes<BF, DP>(); }
template <bool BF, int DP>
int dq_wave_bytes(int nb) { return 1024 + tile_bytes<BF, DP>() + (nb + 1) * 256; }
template <bool BF, int DP>
constexpr int dkv_wave_bytes() { return 1024 + 2 * tile_bytes<BF, DP>() + 2 * tile_bytes<BF, 32>(); }
constexpr int join_bytes(int DP) { return DP * 32 * 4 + 512; }

// -------------------------------------------------------------------------------------------------------------------------
template <bool BF, int DP>
__global__ void __launch_bounds__(256) k_attn_fwd(AttnArgs a) {
  using T = typename Row<BF, DP>::T;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int group = blockIdx.x / a.nh, h = blockIdx.x - group * a.nh;
  const int t = a.split ? group : group * a.nw + wave;
  if (t >= a.plan.tile_off[a.G]) return;   // split: uniform over the workgroup
  const Where w = tile_where(a, t);
  char* mine = smem + wave * fwd_wave_bytes<BF, DP>();
  float* table = reinterpret_cast<float*>(mine);
  T* tv = reinterpret_cast<T*>(mine + 1024);
  fill_table(table, a.bias + (size_t)h * a.nb, a.nb, lane);

  const int hk = h / (a.nh / a.nkv);
  const size_t ld = (size_t)(a.nh + 2 * a.nkv) * a.dh;   // elements of an atom's q, k, v
  const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
  const int qi = w.i0 + (lane & 31), qc = qi < w.n ? qi : w.n - 1;
  Row<BF, DP> q, k, v;
  q.load(base + qc * ld + (size_t)h * a.dh, a.dh, g);
  const T* kbase = base + (size_t)(a.nh + hk) * a.dh;
  const T* vbase = kbase + (size_t)a.nkv * a.dh;
  const uint8_t* prow = w.pairs + qc * w.pitch;
  u32x4_t bk;
  auto fetch = [&](int j0) {
    const int jk = j0 + tile_row(lane & 31), jv = j0 + (lane & 31);
    k.load(kbase + (size_t)(jk < w.n ? jk : w.n - 1) * ld, a.dh, g);
    v.load(vbase + (size_t)(jv < w.n ? jv : w.n - 1) * ld, a.dh, g);
    bk = load_buckets(prow, j0, w.n, g);
  };

  float m = -__builtin_inff(), l = 0.f;
  f32x16_t o[DP / 32] = {};
  const int step = a.split ? a.nw * PAIR_T : PAIR_T;
  int j0 = a.split ? wave * PAIR_T : 0;
  if (j0 < w.n) fetch(j0);
  for (; j0 < w.n; j0 += step) {
    f32x16_t s = Row<BF, DP>::dot(k, q);
    lds_order();
    v.to_lds(tv + (lane & 31) * Row<BF, DP>::PITCH, g);
    lds_order();
    const u32x4_t bc = bk;
    if (j0 + step < w.n) fetch(j0 + step);
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = fmaf(s[i], a.c, table[bucket_of(bc, i)]);
      top = fmaxf(top, s[i]);
    }
    top = fmaxf(top, other_half(top));
    // the sums are rescaled only where a maximum has grown by 2^8: weights up to that size lose nothing
    if (__any(top > m + 8.f || (m == -__builtin_inff() && top > m))) {
      const float mn = fmaxf(m, top), f = mn == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
    }
    const float mu = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - mu);
      l += s[i];
    }
    const Weights<BF> p(s);
    // bf16: the weights enter as two terms. The reverse pass takes D from the output, and one rounding of the weights (2^-9) there
    // is more than the bias gradient, a sum of differences, can bear; two more products and 40 operations of some 180 a tile
    if constexpr (BF) add_cols2<DP>(tv, p, remainder_of(s, p), o, lane);
    else add_cols<BF, DP>(tv, p, o, lane);
  }
  l += other_half(l);

  if (a.split) {   // the wavefronts' shares, in order
    char* join = smem + a.nw * fwd_wave_bytes<BF, DP>();
    float* jo = reinterpret_cast<float*>(join);
    float* jm = reinterpret_cast<float*>(join + DP * 32 * 4);
    for (int k2 = 1; k2 < a.nw; ++k2) {
      __syncthreads();
      if (wave == k2) {
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) jo[(b * 16 + i) * 64 + lane] = o[b][i];
        if (lane < 32) { jm[lane] = m; jm[32 + lane] = l; }
      }
      __syncthreads();
      if (wave == 0) {
        const float m2 = jm[lane & 31], l2 = jm[32 + (lane & 31)];
        const float mn = fmaxf(m, m2);
        const float f1 = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - mn), f2 = m2 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m2 - mn);
        // (a sum that is no number stays one)
        l = l * f1 + l2 * f2;
        m = mn;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[b][i] = o[b][i] * f1 + jo[(b * 16 + i) * 64 + lane] * f2;
      }
    }
    if (wave) return;
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
      if (a.lse && g == 0) a.lse[(size_t)h * a.N + w.lo + qi] = l > 0.f ? m + __log2f(l) : __builtin_inff();
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
      const float s = fmaf(wave_sum(fmaf(q0, k0, q1 * k1)), a.c, b);
      if (s == -__builtin_inff()) continue;
      const float mn = fmaxf(mr, s), f = mr == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mr - mn), p = __builtin_amdgcn_exp2f(s - mn);
      mr = mn;
      lr = lr * f + p;
      o0 = o0 * f + p * v0;
      o1 = o1 * f + p * v1;
    }
    const size_t out = (((size_t)w.lo + w.i0 + r) * a.nh + h) * a.dh;
    const float f = lr == 0.f ? 0.f : 1.0f / lr;
    if (d0) { put<BF>(a.out, out + lane, o0 * f); if (BF && a.o32) a.o32[out + lane] = o0 * f; }
    if (d1) { put<BF>(a.out, out + lane + 64, o1 * f); if (BF && a.o32) a.o32[out + lane + 64] = o1 * f; }
    if (a.lse && lane == 0) a.lse[(size_t)h * a.N + w.lo + w.i0 + r] = lr == 0.f ? __builtin_inff() : mr + __log2f(lr);
  }
}

// sum of a bucket's 64 columns (a lane per bucket: the columns are taken in turn, from its own on, so that no bank is hit twice)
__device__ __forceinline__ float hist_sum(const float* hist, int b) {
  float s[8] = {};
#pragma unroll
  for (int k = 0; k < 64; ++k) s[k & 7] += hist[b * 64 + ((k + b) & 63)];
  return ((s[0] + s[4]) + (s[1] + s[5])) + ((s[2] + s[6]) + (s[3] + s[7]));
}

// adds x[k] to this lane's word at[k] of LDS, HB words at a time: they are read together, and one that is named twice takes up
// what the earlier one has made of it. (Adding in LDS itself, ds_add_f32, took 210 cycles of the compute unit for 64 words.)
constexpr int HB = 4;
__device__ __forceinline__ void hist_add(float* hist, const unsigned (&at)[HB], const float (&x)[HB]) {
  float v[HB];
#pragma unroll
  for (int k = 0; k < HB; ++k) v[k] = hist[at[k]];
#pragma unroll
  for (int k = 0; k < HB; ++k) {
#pragma unroll
    for (int u = 0; u < k; ++u) v[k] = at[k] == at[u] ? v[u] : v[k];
    v[k] += x[k];
  }
#pragma unroll
  for (int k = 0; k < HB; ++k) hist[at[k]] = v[k];
}

// -------------------------------------------------------------------------------------------------------------------------
// g_q of 32 queries, D of theirs, and g_bias. A wavefront (split: a workgroup) of head h takes tiles w, w + per_head, ...
template <bool BF, int DP>
__global__ void __launch_bounds__(256) k_attn_dq(AttnArgs a) {
  using T = typename Row<BF, DP>::T;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int group = blockIdx.x / a.nh, h = blockIdx.x - group * a.nh;
  const int me = a.split ? group : group * a.nw + wave;
  const int wave_bytes = 1024 + tile_bytes<BF, DP>() + (a.nb + 1) * 256;
  char* mine = smem + wave * wave_bytes;
  float* table = reinterpret_cast<float*>(mine);
  T* tk = reinterpret_cast<T*>(mine + 1024);
  float* hist = reinterpret_cast<float*>(mine + 1024 + tile_bytes<BF, DP>());
  fill_table(table, a.bias + (size_t)h * a.nb, a.nb, lane);
  for (int b = 0; b <= a.nb; ++b) hist[b * 64 + lane] = 0.f;
  const int hk = h / (a.nh / a.nkv);
  const size_t ld = (size_t)(a.nh + 2 * a.nkv) * a.dh, lo_ = (size_t)a.nh * a.dh;
  const int ntiles = a.plan.tile_off[a.G];

  for (int t = me < a.per_head ? me : ntiles; t < ntiles; t += a.per_head) {   // split: uniform over the workgroup
    const Where w = tile_where(a, t);
    const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
    const int qi = w.i0 + (lane & 31), qc = qi < w.n ? qi : w.n - 1;
    Row<BF, DP> q, go, k, v;
    q.load(base + qc * ld + (size_t)h * a.dh, a.dh, g);
    go.load(static_cast<const T*>(a.g_out) + ((size_t)w.lo + qc) * lo_ + (size_t)h * a.dh, a.dh, g);
    const float* o32 = BF ? a.o32 : static_cast<const float*>(a.out);
    float D = go.dot32(o32 + ((size_t)w.lo + qc) * lo_ + (size_t)h * a.dh, a.dh, g);
    D += other_half(D);
    const float lse = qi < w.n ? a.lse[(size_t)h * a.N + w.lo + qi] : __builtin_inff();
    if (qi < w.n && g == 0 && (!a.split || wave == 0)) a.delta[(size_t)h * a.N + w.lo + qi] = D;
    const T* kbase = base + (size_t)(a.nh + hk) * a.dh;
    const T* vbase = kbase + (size_t)a.nkv * a.dh;
    const uint8_t* prow = w.pairs + qc * w.pitch;
    u32x4_t bk;
    auto fetch = [&](int j0) {
      const int j = j0 + tile_row(lane & 31);
      const size_t r = (size_t)(j < w.n ? j : w.n - 1) * ld;
      k.load(kbase + r, a.dh, g);
      v.load(vbase + r, a.dh, g);
      bk = load_buckets(prow, j0, w.n, g);
    };
    f32x16_t dq[DP / 32] = {};
    const int step = a.split ? a.nw * PAIR_T : PAIR_T;
    int j0 = a.split ? wave * PAIR_T : 0;
    if (j0 < w.n) fetch(j0);
    for (; j0 < w.n; j0 += step) {
      f32x16_t s = Row<BF, DP>::dot(k, q), ds = Row<BF, DP>::dot(v, go);
      lds_order();
      k.to_lds(tk + tile_row(lane & 31) * Row<BF, DP>::PITCH, g);
      lds_order();
      const u32x4_t bc = bk;
      if (j0 + step < w.n) fetch(j0 + step);
      const bool real = qi < w.n;
#pragma unroll
      for (int i0 = 0; i0 < 16; i0 += HB) {
        unsigned at[HB];
        float x[HB];
#pragma unroll
        for (int k = 0; k < HB; ++k) {
          const int i = i0 + k;
          const unsigned b = bucket_of(bc, i);
          const float tb = table[b], p = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, tb) - lse);
          ds[i] = p * (ds[i] - D);
          at[k] = (real && tb > -__builtin_inff() ? b : (unsigned)a.nb) * 64 + lane;   // (a column for what is left out)
          x[k] = ds[i];
        }
        hist_add(hist, at, x);
      }
      add_cols<BF, DP>(tk, Weights<BF>(ds), dq, lane);
    }
    if (a.split) {
      float* jo = reinterpret_cast<float*>(smem + a.nw * wave_bytes);
      for (int k2 = 1; k2 < a.nw; ++k2) {
        __syncthreads();
        if (wave == k2) {
#pragma unroll
          for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) jo[(b * 16 + i) * 64 + lane] = dq[b][i];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) dq[b][i] += jo[(b * 16 + i) * 64 + lane];
        }
      }
      if (wave) continue;
    }
    T* gq = static_cast<T*>(a.g_qkv) + (size_t)w.lo * ld + (size_t)h * a.dh;
    if (all_finite<DP / 32>(dq, 0.f, qi < w.n)) {
      if (qi < w.n) {
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
      const size_t at = ((size_t)w.lo + w.i0 + r) * ld + (size_t)h * a.dh, og = (((size_t)w.lo + w.i0 + r) * a.nh + h) * a.dh;
      const float q0 = d0 ? value<BF>(a.qkv, at + lane) : 0.f, q1 = d1 ? value<BF>(a.qkv, at + lane + 64) : 0.f;
      const float g0 = d0 ? value<BF>(a.g_out, og + lane) : 0.f, g1 = d1 ? value<BF>(a.g_out, og + lane + 64) : 0.f;
      const float lr = __shfl(lse, r), Dr = __shfl(D, r);
      const uint8_t* row = w.pairs + (w.i0 + r) * w.pitch;
      float a0 = 0.f, a1 = 0.f;
      for (int j = 0; j < w.n; ++j) {
        const float b = table[row[j]];
        if (b == -__builtin_inff()) continue;
        const size_t kj = ((size_t)w.lo + j) * ld + (size_t)(a.nh + hk) * a.dh, vj = kj + (size_t)a.nkv * a.dh;
        const float k0 = d0 ? value<BF>(a.qkv, kj + lane) : 0.f, k1 = d1 ? value<BF>(a.qkv, kj + lane + 64) : 0.f;
        const float v0 = d0 ? value<BF>(a.qkv, vj + lane) : 0.f, v1 = d1 ? value<BF>(a.qkv, vj + lane + 64) : 0.f;
        const float p = __builtin_amdgcn_exp2f(fmaf(wave_sum(fmaf(q0, k0, q1 * k1)), a.c, b) - lr);
        const float d = p * (wave_sum(fmaf(g0, v0, g1 * v1)) - Dr);
        a0 = fmaf(d, k0, a0);
        a1 = fmaf(d, k1, a1);
      }
      if (d0) put<BF>(a.g_qkv, at + lane, a0 * a.scale);
      if (d1) put<BF>(a.g_qkv, at + lane + 64, a1 * a.scale);
    }
  }

  lds_order();
  if (!a.split) {
    if (me < a.per_head && lane < a.nb) a.partial[((size_t)h * a.per_head + me) * a.nb + lane] = hist_sum(hist, lane);
    return;
  }
  __syncthreads();
  if (wave == 0 && lane < a.nb) {
    float s = 0.f;
    for (int k2 = 0; k2 < a.nw; ++k2)
      s += hist_sum(reinterpret_cast<const float*>(smem + k2 * wave_bytes + 1024 + tile_bytes<BF, DP>()), lane);
    a.partial[((size_t)h * a.per_head + me) * a.nb + lane] = s;
  }
}

// g_bias of head h: the wavefronts' partials in order, a run per group of threads, then the runs
__device__ __forceinline__ void bias_reduce(const AttnArgs& a, int h, float* sh) {
  const int b = threadIdx.x & 63, run = threadIdx.x >> 6, runs = blockDim.x >> 6;
  const int per = (a.per_head + runs - 1) / runs, k1 = min(a.per_head, (run + 1) * per);
  float s = 0.f;
  if (b < a.nb) {
    const float* p = a.partial + (size_t)h * a.per_head * a.nb + b;
    for (int k = run * per; k < k1; k += 16) {   // sixteen loads on their way at a time
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = k + u < k1 ? p[(size_t)(k + u) * a.nb] : 0.f;
#pragma unroll
      for (int u = 0; u < 16; ++u) s += v[u];
    }
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (run == 0 && b < a.nb) {
    for (int k = 1; k < runs; ++k) s += sh[k * 64 + b];
    a.g_bias[(size_t)h * a.nb + b] = s;
  }
}

// -------------------------------------------------------------------------------------------------------------------------
// g_k and g_v of 32 keys, over the query heads that share them; the last nh workgroups add up g_bias
template <bool BF, int DP>
__global__ void __launch_bounds__(256) k_attn_dkv(AttnArgs a, int ngroups) {
  using T = typename Row<BF, DP>::T;
  constexpr int PT = Row<BF, 32>::PITCH;
  extern __shared__ __align__(16) char smem[];
  if ((int)blockIdx.x >= ngroups * a.nkv) {   // uniform over the workgroup
    bias_reduce(a, blockIdx.x - ngroups * a.nkv, reinterpret_cast<float*>(smem));
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int group = blockIdx.x / a.nkv, hk = blockIdx.x - group * a.nkv;
  const int t = a.split ? group : group * a.nw + wave;
  if (t >= a.plan.tile_off[a.G]) return;
  const Where w = tile_where(a, t);
  char* mine = smem + wave * dkv_wave_bytes<BF, DP>();
  float* table = reinterpret_cast<float*>(mine);
  T* tq = reinterpret_cast<T*>(mine + 1024);
  T* tg = tq + 32 * Row<BF, DP>::PITCH;
  T* tp = tg + 32 * Row<BF, DP>::PITCH;
  T* ts = tp + 32 * PT;
  const int rep = a.nh / a.nkv;
  const size_t ld = (size_t)(a.nh + 2 * a.nkv) * a.dh, lo_ = (size_t)a.nh * a.dh;
  const T* base = static_cast<const T*>(a.qkv) + (size_t)w.lo * ld;
  const T* gbase = static_cast<const T*>(a.g_out) + (size_t)w.lo * lo_;
  Row<BF, DP> k, v, q, go;
  {
    const int j = w.i0 + tile_row(lane & 31);
    const T* p = base + (size_t)(j < w.n ? j : w.n - 1) * ld + (size_t)(a.nh + hk) * a.dh;
    k.load(p, a.dh, g);
    v.load(p + (size_t)a.nkv * a.dh, a.dh, g);
  }
  f32x16_t dk[DP / 32] = {}, dv[DP / 32] = {};
  const int step = a.split ? a.nw * PAIR_T : PAIR_T;
  for (int r = 0; r < rep; ++r) {
    const int h = hk * rep + r;
    lds_order();
    fill_table(table, a.bias + (size_t)h * a.nb, a.nb, lane);
    lds_order();
    u32x4_t bk;
    float lse, D;
    auto fetch = [&](int i0) {
      const int i = i0 + (lane & 31), ic = i < w.n ? i : w.n - 1;
      q.load(base + (size_t)ic * ld + (size_t)h * a.dh, a.dh, g);
      go.load(gbase + (size_t)ic * lo_ + (size_t)h * a.dh, a.dh, g);
      bk = load_buckets(w.pairs + ic * w.pitch, w.i0, w.n, g);
      lse = i < w.n ? a.lse[(size_t)h * a.N + w.lo + i] : __builtin_inff();
      D = a.delta[(size_t)h * a.N + w.lo + ic];
    };
    int i0 = a.split ? wave * PAIR_T : 0;
    if (i0 < w.n) fetch(i0);
    for (; i0 < w.n; i0 += step) {
      f32x16_t s = Row<BF, DP>::dot(k, q), ds = Row<BF, DP>::dot(v, go);
      lds_order();
      q.to_lds(tq + (lane & 31) * Row<BF, DP>::PITCH, g);
      go.to_lds(tg + (lane & 31) * Row<BF, DP>::PITCH, g);
      const u32x4_t bc = bk;
      const float lc = lse, Dc = D;
      if (i0 + step < w.n) fetch(i0 + step);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, table[bucket_of(bc, i)]) - lc);
        s[i] = p;
        ds[i] = p * (ds[i] - Dc);
      }
      weights_to_lds<BF>(Weights<BF>(s), tp, lane);
      weights_to_lds<BF>(Weights<BF>(ds), ts, lane);
      lds_order();
      add_cols_lds<BF, DP>(tg, tp, dv, lane);
      add_cols_lds<BF, DP>(tq, ts, dk, lane);
    }
  }
  if (a.split) {
    float* jo = reinterpret_cast<float*>(smem + a.nw * dkv_wave_bytes<BF, DP>());
    for (int k2 = 1; k2 < a.nw; ++k2) {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        f32x16_t(&x)[DP / 32] = which ? dv : dk;
        __syncthreads();
        if (wave == k2) {
#pragma unroll
          for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) jo[(b * 16 + i) * 64 + lane] = x[b][i];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] += jo[(b * 16 + i) * 64 + lane];
        }
      }
    }
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
      fill_table(table, a.bias + (size_t)h * a.nb, a.nb, lane);
      lds_order();
      for (int i = 0; i < w.n; ++i) {
        const float b = table[w.pairs[i * w.pitch + w.i0 + r]];
        if (b == -__builtin_inff()) continue;
        const size_t qa = ((size_t)w.lo + i) * ld + (size_t)h * a.dh, ga = (((size_t)w.lo + i) * a.nh + h) * a.dh;
        const float q0 = d0 ? value<BF>(a.qkv, qa + lane) : 0.f, q1 = d1 ? value<BF>(a.qkv, qa + lane + 64) : 0.f;
        const float g0 = d0 ? value<BF>(a.g_out, ga + lane) : 0.f, g1 = d1 ? value<BF>(a.g_out, ga + lane + 64) : 0.f;
        const float p = __builtin_amdgcn_exp2f(fmaf(wave_sum(fmaf(q0, k0, q1 * k1)), a.c, b) - a.lse[(size_t)h * a.N + w.lo + i]);
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
constexpr int LDS_MOST = 64 * 1024;   // of a workgroup, so that two fit a compute unit and no attribute has to be set

int waves_that_fit(int wave_bytes, int extra) {
  int nw = (LDS_MOST - extra) / wave_bytes;
  return nw >= 4 ? 4 : nw >= 2 ? 2 : 1;
}

// wavefronts per head of the reverse kernel over queries: every tile its own while they are few, then as many as keep the chip
// busy (each leaves one partial of g_bias)
int64_t dq_per_head(int64_t max_tiles, int nh) {
  const int64_t most = (4096 + nh - 1) / nh;
  return max_tiles < most ? max_tiles : most;
}

struct AttnWs {
  float *delta, *partial;
  size_t bytes;
};
AttnWs carve_attn_ws(void* p, int N, int G, int nh, int nb) {
  Carver c(p);
  AttnWs w;
  w.delta = c.take<float>((size_t)nh * N);
  w.partial = c.take<float>((size_t)nh * dq_per_head(pair_plan_view(nullptr, N, G).max_tiles, nh) * nb);
  w.bytes = c.used();
  return w;
}
struct AttnSaved {
  float *lse, *o32;
  size_t bytes;
};
AttnSaved carve_attn_saved(void* p, int N, int nh, int dh, bool bf16) {
  Carver c(p);
  AttnSaved s;
  s.lse = c.take<float>((size_t)nh * N);
  s.o32 = bf16 ? c.take<float>((size_t)N * nh * dh) : nullptr;
  s.bytes = c.used();
  return s;
}

int32_t check_attn(int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb, int32_t dtype) {
  HGNN_REQUIRE(N >= 0 && G >= 0, HGNN_ERR_BAD_SHAPE, "negative N or G");
  HGNN_REQUIRE(nh >= 1 && nh <= 64 && nkv >= 1 && nh % nkv == 0, HGNN_ERR_BAD_SHAPE,
               "graph_attention: 1..64 heads, a multiple of the key heads (got %d, %d)", nh, nkv);
  HGNN_REQUIRE(dh >= 8 && dh <= 128 && dh % 8 == 0, HGNN_ERR_BAD_SHAPE, "graph_attention: the head width must be a multiple of 8 in 8..128 (got %d)", dh);
  HGNN_REQUIRE(nb >= 1 && nb <= ATTN_BUCKETS, HGNN_ERR_BAD_SHAPE, "graph_attention: 1..%d buckets (got %d)", ATTN_BUCKETS, nb);
  HGNN_REQUIRE(dtype == HGNN_F32 || dtype == HGNN_BF16, HGNN_ERR_BAD_SHAPE, "unknown dtype %d", dtype);
  HGNN_REQUIRE(N < (1 << 28) && G < (1 << 28), HGNN_ERR_OVERFLOW, "graph_attention: N and G must be below 2^28");
  HGNN_REQUIRE((pair_plan_view(nullptr, N, G).max_tiles + 64) * nh < INT_MAX, HGNN_ERR_OVERFLOW, "graph_attention: too many tiles for one launch");
  return HGNN_OK;
}

// Few tiles: the wavefronts of a workgroup share one tile and deal out the other side's. Until there is a wavefront per SIMD
// this shortens the chain of tiles without taking a compute unit from anybody.
bool attn_split(int64_t max_tiles, int nh, int G, int N) { return max_tiles * nh <= 4 * num_cus() && N > 2 * PAIR_T * (int64_t)G; }

template <bool BF, int DP>
int32_t launch_fwd(hipStream_t st, AttnArgs a) {
  constexpr int WB = fwd_wave_bytes<BF, DP>();
  a.split = attn_split(a.plan.max_tiles, a.nh, a.G, a.N);
  const int extra = a.split ? join_bytes(DP) : 0;
  a.nw = waves_that_fit(WB, extra);
  const int64_t groups = a.split ? a.plan.max_tiles : (a.plan.max_tiles + a.nw - 1) / a.nw;
  k_attn_fwd<BF, DP><<<(unsigned)(groups * a.nh), 64 * a.nw, WB * a.nw + extra, st>>>(a);
  HGNN_LAUNCH_CHECK("k_attn_fwd");
  return HGNN_OK;
}

template <bool BF, int DP>
int32_t launch_bwd(hipStream_t st, AttnArgs a) {
  a.split = attn_split(a.plan.max_tiles, a.nh, a.G, a.N);
  {
    const int wb = dq_wave_bytes<BF, DP>(a.nb), extra = a.split ? join_bytes(DP) : 0;
    a.nw = a.split ? waves_that_fit(wb, extra) : 1;   // (nothing is shared but in a split tile, and single wavefronts pack into LDS best)
    const int64_t groups = a.split ? a.per_head : (a.per_head + a.nw - 1) / a.nw;
    k_attn_dq<BF, DP><<<(unsigned)(groups * a.nh), 64 * a.nw, wb * a.nw + extra, st>>>(a);
    HGNN_LAUNCH_CHECK("k_attn_dq");
  }
  constexpr int WB = dkv_wave_bytes<BF, DP>();
  const int extra = a.split ? join_bytes(DP) : 0;
  a.nw = waves_that_fit(WB, extra);
  const int64_t groups = a.split ? a.plan.max_tiles : (a.plan.max_tiles + a.nw - 1) / a.nw;
  k_attn_dkv<BF, DP><<<(unsigned)(groups * a.nkv + a.nh), 64 * a.nw, WB * a.nw + extra, st>>>(a, (int)groups);
  HGNN_LAUNCH_CHECK("k_attn_dkv");
  return HGNN_OK;
}

template <bool BF>
int32_t run_attn(hipStream_t st, const AttnArgs& a, bool fwd) {
  if (a.dh <= 32) return fwd ? launch_fwd<BF, 32>(st, a) : launch_bwd<BF, 32>(st, a);
  if (a.dh <= 64) return fwd ? launch_fwd<BF, 64>(st, a) : launch_bwd<BF, 64>(st, a);
  return fwd ? launch_fwd<BF, 128>(st, a) : launch_bwd<BF, 128>(st, a);
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
  *ws_bytes_host = carve_attn_ws(nullptr, N, G, nh, nb).bytes;
  *saved_bytes_host = carve_attn_saved(nullptr, N, nh, dh, dtype == HGNN_BF16).bytes;
  return HGNN_OK;
}

extern "C" int32_t hgnn_graph_attention_fwd(void* stream, int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb,
                                            int32_t dtype, float scale, const void* plan, size_t plan_bytes, const uint8_t* pairs,
                                            const void* qkv, const float* bias, void* out, void* saved, size_t saved_bytes) {
  HGNN_TRY(check_attn(N, G, nh, nkv, dh, nb, dtype));
  if (N == 0) return HGNN_OK;
  HGNN_REQUIRE(plan && pairs && qkv && bias && out, HGNN_ERR_NULLPTR, "graph_attention_fwd: null pointer");
  AttnArgs a{};
  a.plan = pair_plan_view(plan, N, G);
  HGNN_REQUIRE(plan_bytes >= a.plan.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "pair plan: need %zu bytes, got %zu", a.plan.bytes, plan_bytes);
  const AttnSaved s = carve_attn_saved(saved, N, nh, dh, dtype == HGNN_BF16);
  HGNN_REQUIRE(!saved || saved_bytes >= s.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "graph_attention saved buffer: need %zu bytes, got %zu", s.bytes, saved_bytes);
  if (a.plan.max_tiles == 0) return HGNN_OK;   // (G == 0: no plan of N atoms exists)
  a.N = N; a.G = G; a.nh = nh; a.nkv = nkv; a.dh = dh; a.nb = nb;
  a.scale = scale; a.c = scale * LOG2E;
  a.pairs = pairs; a.qkv = qkv; a.bias = bias; a.out = out;
  a.lse = saved ? s.lse : nullptr;
  a.o32 = saved ? s.o32 : nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_MISC, st);
  return dtype == HGNN_BF16 ? run_attn<true>(st, a, true) : run_attn<false>(st, a, true);
}

extern "C" int32_t hgnn_graph_attention_bwd(void* stream, int32_t N, int32_t G, int32_t nh, int32_t nkv, int32_t dh, int32_t nb,
                                            int32_t dtype, float scale, const void* plan, size_t plan_bytes, const uint8_t* pairs,
                                            const void* qkv, const float* bias, const void* out, const void* saved, size_t saved_bytes,
                                            const void* g_out, void* g_qkv, float* g_bias, void* ws, size_t ws_bytes) {
  HGNN_TRY(check_attn(N, G, nh, nkv, dh, nb, dtype));
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
  const AttnWs w = carve_attn_ws(ws, N, G, nh, nb);
  HGNN_REQUIRE(ws_bytes >= w.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "graph_attention workspace: need %zu bytes, got %zu", w.bytes, ws_bytes);
  a.N = N; a.G = G; a.nh = nh; a.nkv = nkv; a.dh = dh; a.nb = nb;
  a.per_head = (int)dq_per_head(a.plan.max_tiles, nh);
  a.scale = scale; a.c = scale * LOG2E;
  a.pairs = pairs; a.qkv = qkv; a.bias = bias; a.out = const_cast<void*>(out); a.lse = s.lse; a.o32 = s.o32;
  a.g_out = g_out; a.g_qkv = g_qkv; a.delta = w.delta; a.partial = w.partial; a.g_bias = g_bias;
  ProfScope ps(PT_MISC, st);
  return dtype == HGNN_BF16 ? run_attn<true>(st, a, false) : run_attn<false>(st, a, false);
}
