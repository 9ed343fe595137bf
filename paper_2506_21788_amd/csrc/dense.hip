// hgnn_dense_fwd / _bwd: y = r + act(x W + b) and its gradients, x [M,K], W [K,N], and hgnn_round_bf16.
//
//   g_z = g_y act'(z),   g_x = g_z W^T,   gW = x^T g_z,   g_b = column sums of g_z
//
// Three products with operands in different orders, one kernel each way: a workgroup forms a tile of the result from slices
// of 32 of the contraction that it stages in LDS as bf16 while the next slice is on its way from memory. An operand whose
// neighbours in memory run along the contraction is staged row by row and read in 8-byte pieces, one whose neighbours run along
// the result through transposing reads; both give a lane the contraction places 4 g + 0..3 and 8 + 4 g + 0..3 of 16.
// float32 operands are staged as three bf16 terms and take six partial products (devmath.h): 2.7 times the rate of the float32
// matrix cores at their precision. The forward pass keeps act'(z) in float32, so that the reverse pass multiplies by it where
// it stages g_z: no tensor g_z exists. A bf16 call takes g_z = g_y act'(z) as two bf16 terms (terms_of_gz), 16 bits: one would add a rounding
// to g_x's own and leave gW, a float32 result, with 8. (A third in gW: both directions of 40,041 x 256 -> 512 take 7 % more time; with two
// its error there is 2.5e-6, that of a float32 sum over the rows 2.2e-6.)
//
// The two products with W (large calls): W is laid out once per call in the order in which the matrix cores take it (k_pack), a 1 KB fragment
// per 32 columns and 16 places, in the one or three bf16 terms, and goes from the L2 to registers without LDS. Staged by every
// workgroup, half of the LDS traffic and of the splitting was W's, and the LDS was what bound the kernel (128 x 128 x 64:
// 768 cycles of LDS against 512 of the matrix cores). The forward pass lays out W^T for the reverse pass as well, in `saved`.
//
// Bound by memory in bf16 (40,041 x 256 -> 512 with silu: 37 us forward, 36 and 33 in reverse, each moving 143 MB: 3.8 to 4.4 TB/s) and
// by waits in float32 (7,703 x 866 -> 889 with gelu: 96, 88 and 81 us, six products of 11.9 GFLOP each, 0.74 to 0.88 PFLOP/s: the matrix
// cores are busy 32 to 37 % of the time, 1.2 to 1.5 wavefronts a SIMD wait half of theirs).
//
// Small calls (few tiles) take k_dense_small: 32 x 32 results, the contraction dealt to the four wavefronts of a workgroup, operands
// straight from memory: nothing is staged, the chain is one load, some products and a join.
#include <climits>
#include <type_traits>

#include "common.h"
#include "devmath.h"
#include "prof.h"

namespace hgnn {
namespace {

typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct Operand {
  const void* p = nullptr;      // float32 or bf16
  const float* mul = nullptr;   // float32 factors in the same places (act'), or null
  int ld = 0;
};

struct DenseArgs {
  int I, J, C;           // result I x J, contraction C
  Operand a, b;          // a: [I][C] or [C][I], b: [J][C] or [C][J]
  int act;
  const float* bias;     // [J] or null
  const void* res;       // [I][J] added to the result, or null
  void* out;             // [I][J]
  float* dact;           // [I][J] act'(z) or null
  float* partial;        // weight gradient: [nsplit][I][J], then colsum [nsplit][J]
  float* colsum;         // [nsplit][J] column sums of b, or null
  const u32x4_t* packed; // k_dense_packed: operand b in fragments [term][32 columns][16 places][64 lanes]
  int pkb, pterm;        // fragments per 32 columns; of a term
  int nsplit, per_split; // contraction slices of a split (multiple of 32 places)
  int ti, tj;            // tiles
};

// Eight neighbouring values of an operand as they come from memory. Nothing is done to them before they are staged: an operation here
// would wait for the load that is meant to travel while a slice is multiplied.
template <bool BF, bool MUL>
struct Raw {
  u32x4_t w[BF ? 1 : 2];
  u32x4_t m[MUL ? 2 : 1];
  __device__ __forceinline__ void load(const Operand& o, size_t at) {
    if constexpr (BF) __builtin_memcpy(&w[0], static_cast<const unsigned short*>(o.p) + at, 16);
    else __builtin_memcpy(w, static_cast<const float*>(o.p) + at, 32);
    if constexpr (MUL) __builtin_memcpy(m, o.mul + at, 32);
  }
  // n of them exist, the others are zeros
  __device__ __forceinline__ void load(const Operand& o, size_t at, int n) {
    if (n >= 8) {
      load(o, at);
      return;
    }
#pragma unroll
    for (int k = 0; k < (BF ? 1 : 2); ++k) w[k] = u32x4_t{0, 0, 0, 0};
    if constexpr (MUL) m[0] = m[1] = u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k < n) {
        if constexpr (BF) w[0][k >> 1] |= (unsigned)static_cast<const unsigned short*>(o.p)[at + k] << (16 * (k & 1));
        else w[k >> 2][k & 3] = __float_as_uint(static_cast<const float*>(o.p)[at + k]);
        if constexpr (MUL) m[k >> 2][k & 3] = __float_as_uint(o.mul[at + k]);
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (BF) v[k] = __uint_as_float(k & 1 ? w[0][k >> 1] & 0xffff0000u : w[0][k >> 1] << 16);
      else v[k] = __uint_as_float(w[k >> 2][k & 3]);
      if constexpr (MUL) v[k] *= __uint_as_float(m[k >> 2][k & 3]);
    }
  }
};
template <bool BF, bool MUL>
__device__ __forceinline__ void load8(const Operand& o, size_t at, int n, float (&v)[8]) {
  Raw<BF, MUL> r;
  r.load(o, at, n);
  r.values(v);
}

// eight values as NT bf16 terms
template <int NT>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4_t (&o)[NT]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if constexpr (NT == 3) {
      unsigned p[3];
      split_bf16x3_pair(x[2 * t], x[2 * t + 1], p);
      o[0][t] = p[0]; o[1][t] = p[1]; o[2][t] = p[2];
    } else {
      const unsigned h = pack_bf16x2(x[2 * t], x[2 * t + 1]);
      o[0][t] = h;
      if constexpr (NT == 2) o[1][t] = pack_bf16x2(x[2 * t] - __uint_as_float(h << 16), x[2 * t + 1] - __uint_as_float(h & 0xffff0000u));
    }
  }
}

// acc[i][j] += a[i] b[j] over the terms that count, smallest first (three terms each: the six products of devmath.h; else one operand is of
// one term). Term by term over all accumulators: a product that adds to the one before waits for it twice as long as it takes.
template <int NA, int NB, int WI, int WJ>
__device__ __forceinline__ void mfma_terms(const bf16x8_t (&a)[WI][NA], const bf16x8_t (&b)[WJ][NB], f32x16_t (&acc)[WI][WJ]) {
  constexpr bool SIX = NA == 3 && NB == 3;
  static_assert(SIX || NA == 1 || NB == 1);
  constexpr int N = SIX ? 6 : NA > NB ? NA : NB;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const int ta = SIX ? (t == 0 ? 2 : t == 1 || t == 3 ? 1 : 0) : NA > 1 ? N - 1 - t : 0, tb = SIX ? (t == 2 ? 2 : t == 1 || t == 4 ? 1 : 0) : NB > 1 ? N - 1 - t : 0;
#pragma unroll
    for (int i = 0; i < WI; ++i)
#pragma unroll
      for (int j = 0; j < WJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i][ta], b[j][tb], acc[i][j], 0, 0, 0);
  }
}

__device__ __forceinline__ bf16x8_t cat(s16x4_t l, s16x4_t h) {
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A slice of an operand: E places along the result (E = 64 or 128) by BC along the contraction. KC: its neighbours in memory
// run along the contraction. NT bf16 terms, one plane each.
template <int E, bool KC, int NT, int BC>
struct Slice {
  static constexpr int PITCH = KC ? BC + 8 : E + 16;          // elements; rows of 16 bytes, in different groups of banks
  static constexpr int PLANE = (KC ? E : BC) * PITCH;
  static constexpr int BYTES = PLANE * NT * 2;
  static constexpr int CH = E * BC / 8 / 256;                 // chunks of 8 of a thread
  __device__ static __forceinline__ void place(int c, int& e, int& k) {   // of chunk c
    if (KC) { e = c / (BC / 8); k = c % (BC / 8) * 8; }
    else { k = c / (E / 8); e = c % (E / 8) * 8; }
  }
  // from place e0 of ne along the result and k0 of nk along the contraction. Places past nk are zeros; past ne anything may stand
  // (their results are not stored). Slices that lie inside take wide loads without a test; where neighbours run along the result,
  // a load past the end of a row reads on in the next one, so only the last of all rows (`all` places) needs the test.
  template <bool BF, bool MUL>
  __device__ static __forceinline__ void fetch(const Operand& o, int e0, int k0, int ne, int nk, int all, int tid, Raw<BF, MUL> (&v)[CH]) {
    const bool inside = k0 + BC <= nk && (KC || e0 + E <= ne || (k0 + BC < all && ne >= 8));   // uniform
    if (inside) {
#pragma unroll
      for (int u = 0; u < CH; ++u) {
        int e, k;
        place(tid + u * 256, e, k);
        if (KC) v[u].load(o, (size_t)min(e0 + e, ne - 1) * o.ld + k0 + k);
        else v[u].load(o, (size_t)(k0 + k) * o.ld + (e0 + e < ne ? e0 + e : 0));
      }
    } else {
#pragma unroll
      for (int u = 0; u < CH; ++u) {
        int e, k;
        place(tid + u * 256, e, k);
        e += e0;
        k += k0;
        if (KC) v[u].load(o, (size_t)min(e, ne - 1) * o.ld + (k < nk ? k : 0), nk - k);
        else v[u].load(o, (size_t)(k < nk ? k : 0) * o.ld + (e < ne ? e : 0), k < nk ? ne - e : 0);
      }
    }
  }
  // cs: running sums of the values along the contraction (KC: none)
  template <bool BF, bool MUL>
  __device__ static __forceinline__ void stage(unsigned short* lds, int tid, const Raw<BF, MUL> (&v)[CH], float (*cs)[8]) {
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      int e, k;
      place(tid + u * 256, e, k);
      u32x4_t t[NT];
      if constexpr (BF && !MUL && NT == 1) {
        t[0] = v[u].w[0];
        if (cs) {
          float x[8];
          v[u].values(x);
#pragma unroll
          for (int i = 0; i < 8; ++i) cs[u][i] += x[i];
        }
      } else {
        float x[8];
        v[u].values(x);
        if (cs) {
#pragma unroll
          for (int i = 0; i < 8; ++i) cs[u][i] += x[i];
        }
        split8<NT>(x, t);
      }
#pragma unroll
      for (int q = 0; q < NT; ++q) *reinterpret_cast<u32x4_t*>(lds + q * PLANE + (KC ? e * PITCH + k : k * PITCH + e)) = t[q];
    }
  }
  // operand of the 32 places from e on, contraction places 16 s + {4 g + 0..3, 8 + 4 g + 0..3}
  __device__ static __forceinline__ void read(const unsigned short* lds, int e, int s, int lane, bf16x8_t (&o)[NT]) {
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      if constexpr (KC) {
        const unsigned short* p = lds + q * PLANE + (e + (lane & 31)) * PITCH + 16 * s + 4 * (lane >> 5);
        o[q] = cat(*reinterpret_cast<const s16x4_t*>(p), *reinterpret_cast<const s16x4_t*>(p + 8));
      } else {
        const unsigned short* p = lds + q * PLANE + (16 * s + 4 * (lane >> 5) + ((lane & 15) >> 2)) * PITCH + e + (lane & 16) + (lane & 3) * 4;
        o[q] = cat(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p)),
                   __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p + 8 * PITCH)));
      }
    }
  }
};

// Operands of several terms only reach to the largest bf16 number, 3.39e38: a larger one, and an infinite one, has an infinite first
// term, and that is no number with a remainder of the other operand that is zero or of the other sign, or with its own. So where a
// wavefront's 32 x 32 results are not all finite, those that are not are formed again from the operands themselves, on the float32
// matrix cores: what the definition makes infinite is infinite, what it makes finite is finite. Results (i0 .., j0 ..), contraction places
// c .. c + run - 1 of every `step` up to c1. Such values are slow (40,041 x 256 -> 512 bf16 with silu, both
// directions: one infinite operand 0.74 ms, nothing but NaN 1.9 ms instead of 0.13); all others pay 16 operations for the test.
template <bool BF, bool KC, bool MUL>
__device__ __forceinline__ float value_at(const Operand& o, int e, int ne, int k, int nk) {
  if (e >= ne || k >= nk) return 0.f;
  const size_t at = KC ? (size_t)e * o.ld + k : (size_t)k * o.ld + e;
  float x;
  if constexpr (BF) x = __uint_as_float((unsigned)static_cast<const unsigned short*>(o.p)[at] << 16);
  else x = static_cast<const float*>(o.p)[at];
  if constexpr (MUL) x *= o.mul[at];
  return x;
}
template <bool BF, bool AKC, bool BKC, int NA, int NB, bool AMUL, bool BMUL>
__device__ __forceinline__ void form_again(const DenseArgs& a, int i0, int j0, int c, int run, int step, int c1, int lane, f32x16_t& acc) {
  if constexpr (NA > 1 || NB > 1) {   // (single terms are the operands themselves)
    float z = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) z = fmaf(acc[v], 0.f, z);
    if (__all(z == 0.f)) return;
    f32x16_t s = {};
#pragma unroll 1
    for (; c < c1; c += step)
#pragma unroll 1
      for (int k = c; k < c + run; k += 2)
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(value_at<BF, AKC, AMUL>(a.a, i0 + (lane & 31), a.I, k + (lane >> 5), c1),
                                                 value_at<BF, BKC, BMUL>(a.b, j0 + (lane & 31), a.J, k + (lane >> 5), c1), s, 0, 0, 0);
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = fabsf(acc[v]) < __builtin_inff() ? acc[v] : s[v];
  }
}

// act(z) and act'(z)
__device__ __forceinline__ void activate(int act, float z, float& y, float& dy) {
  if (act == HGNN_ACT_SILU) {
    const float e = __expf(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.0f + e), s = z < 0.f ? e * r : r;   // (no overflow on either side)
    y = z * s;
    dy = s * (1.0f + z * (1.0f - s));
  } else if (act == HGNN_ACT_GELU) {
    const float phi = 0.5f * erfcf(-0.70710678118654752f * z);
    y = z * phi;
    dy = fmaf(0.39894228040143268f * z, __expf(-0.5f * z * z), phi);
  } else {
    y = z;
    dy = 1.f;
  }
}

enum { EPI_Y = 0, EPI_GX = 1, EPI_GW = 2 };

// four neighbouring values at p[at ..], n of them exist
__device__ __forceinline__ void put4(float* p, size_t at, const float (&v)[4], int n) {
  if (n >= 4) {
    __builtin_memcpy(p + at, v, 16);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) p[at + k] = v[k];
  }
}
__device__ __forceinline__ void get4(const float* p, size_t at, float (&v)[4], int n) {
  if (n >= 4) {
    __builtin_memcpy(v, p + at, 16);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = k < n ? p[at + k] : 0.f;
  }
}
__device__ __forceinline__ void put4(unsigned short* p, size_t at, const float (&v)[4], int n) {
  const unsigned w[2] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  if (n >= 4) {
    __builtin_memcpy(p + at, w, 8);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) p[at + k] = (unsigned short)(w[k >> 1] >> (16 * (k & 1)));
  }
}
__device__ __forceinline__ void get4(const unsigned short* p, size_t at, float (&v)[4], int n) {
  unsigned short w[4] = {};
  if (n >= 4) {
    __builtin_memcpy(w, p + at, 8);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) w[k] = p[at + k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = __uint_as_float((unsigned)w[k] << 16);
}

// Finishes four neighbouring values of row i from column j on, n of them exist. bias, res: theirs (zeros without).
template <bool BF, int EPI>
__device__ __forceinline__ void finish4(const DenseArgs& a, int i, int j, float (&v)[4], int n, int split, const float (&bias)[4], const float (&res)[4]) {
  using T = typename std::conditional<BF, unsigned short, float>::type;
  const size_t at = (size_t)i * a.J + j;
  if constexpr (EPI == EPI_GW) {
    put4(a.partial + (size_t)split * a.I * a.J, at, v, n);
  } else {
    if constexpr (EPI == EPI_Y) {
      float d[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float y;
        activate(a.act, v[k] + bias[k], y, d[k]);
        v[k] = y;
      }
      if (a.dact) put4(a.dact, at, d, n);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += res[k];
    put4(static_cast<T*>(a.out), at, v, n);
  }
}

// tile of a workgroup: the tiles of a row block are neighbours on one XCD (workgroups are dealt to the 8 XCDs in turn), so its
// rows come from memory once
__device__ __forceinline__ bool tile_of(const DenseArgs& a, int& ti, int& tj, int& split) {
  const int n = a.ti * a.tj * a.nsplit, per = (n + 7) / 8;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || t >= n) return false;
  tj = t % a.tj;
  ti = t / a.tj % a.ti;
  split = t / (a.tj * a.ti);
  return true;
}

// The results of a workgroup: wavefront (wi, wj) of 2 x 2 has EI / 2 rows and EJ / 2 columns.
template <bool BF, int EPI, int EI, int EJ>
__device__ __forceinline__ void store_tile(const DenseArgs& a, const f32x16_t (&acc)[EI / 64][EJ / 64], const float (&bias)[4], int i0, int j0, int wave, int lane,
                                           char* smem) {
  constexpr int WI = EI / 64, WJ = EJ / 64;
  const int wi = wave >> 1, wj = wave & 1;
  // through LDS, 32 rows of a wavefront at a time, so that a lane ends up with four neighbours of a row (always the same columns): a
  // lane's own sixteen values lie in sixteen rows
  __syncthreads();
  using T = typename std::conditional<BF, unsigned short, float>::type;
  constexpr int COLS = EJ / 2, P = COLS + 4, LPRO = COLS / 4, RP = 64 / LPRO, PASS = 32 / RP;   // lanes of a row, rows of a pass, passes
  float* sh = reinterpret_cast<float*>(smem) + wave * 32 * P;
  const int q = j0 + wj * COLS + lane % LPRO * 4, nq = a.J - q;
#pragma unroll
  for (int i = 0; i < WI; ++i) {
    const int r0 = i0 + wi * (EI / 2) + i * 32 + lane / LPRO;
    auto residual = [&](int u, float (&t)[4]) {
      if (a.res && r0 + u * RP < a.I && nq > 0) get4(static_cast<const T*>(a.res), (size_t)(r0 + u * RP) * a.J + q, t, nq);
    };
    float res[4] = {}, next[4] = {};
    residual(0, res);
    if (i) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
    for (int j = 0; j < WJ; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) sh[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * P + j * 32 + (lane & 31)] = acc[i][j][v];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    // (not unrolled: the activations in line 64 times were 54 KB of instructions, run once a workgroup, and took longer than the product)
#pragma unroll 1
    for (int u = 0; u < PASS; ++u) {
      float v[4];
      *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(sh + (u * RP + lane / LPRO) * P + lane % LPRO * 4);
      if (u + 1 < PASS) residual(u + 1, next);
      if (r0 + u * RP < a.I && nq > 0) finish4<BF, EPI>(a, r0 + u * RP, q, v, nq, 0, bias, res);
#pragma unroll
      for (int k = 0; k < 4; ++k) res[k] = next[k];
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// contraction places of a slice: as many as leave room for three workgroups a compute unit (fewer barriers and longer loads)
constexpr int slice_places(int na, int nb) { return na + nb == 2 ? 64 : 32; }

// EI x EJ tile, 2 x 2 wavefronts. AKC / BKC: the operand's neighbours run along the contraction.
template <bool BF, int EPI, int EI, int EJ, bool AKC, bool BKC, int NA, int NB, bool AMUL, bool BMUL>
__global__ void __launch_bounds__(256, 2) k_dense(DenseArgs a) {
  constexpr int BC = slice_places(NA, NB);
  using SA = Slice<EI, AKC, NA, BC>;
  using SB = Slice<EJ, BKC, NB, BC>;
  extern __shared__ __align__(16) char smem[];
  unsigned short* la = reinterpret_cast<unsigned short*>(smem);
  unsigned short* lb = reinterpret_cast<unsigned short*>(smem + SA::BYTES);
  constexpr int WI = EI / 64, WJ = EJ / 64;   // 32-blocks of a wavefront
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wi = wave >> 1, wj = wave & 1;
  int ti, tj, split;
  if (!tile_of(a, ti, tj, split)) return;
  const int i0 = ti * EI, j0 = tj * EJ;
  const int c0 = split * a.per_split, c1 = min(a.C, c0 + a.per_split);
  f32x16_t acc[WI][WJ] = {};
  Raw<BF, AMUL> va[SA::CH];
  Raw<BF, BMUL> vb[SB::CH];
  float cs[SB::CH][8] = {};
  const bool sums = EPI == EPI_GW && a.colsum && ti == 0;
  float bias[4] = {};   // of the four columns that this lane finishes
  if (EPI == EPI_Y && a.bias) {
    const int q = j0 + wj * (EJ / 2) + lane % (EJ / 8) * 4;
    if (q < a.J) get4(a.bias, q, bias, a.J - q);
  }
  if (c0 < c1) {
    SA::template fetch<BF, AMUL>(a.a, i0, c0, a.I, c1, a.C, tid, va);
    SB::template fetch<BF, BMUL>(a.b, j0, c0, a.J, c1, a.C, tid, vb);
  }
  for (int c = c0; c < c1; c += BC) {
    __syncthreads();
    SA::template stage<BF, AMUL>(la, tid, va, nullptr);
    SB::template stage<BF, BMUL>(lb, tid, vb, EPI == EPI_GW && sums ? cs : nullptr);
    if (c + BC < c1) {
      SA::template fetch<BF, AMUL>(a.a, i0, c + BC, a.I, c1, a.C, tid, va);
      SB::template fetch<BF, BMUL>(a.b, j0, c + BC, a.J, c1, a.C, tid, vb);
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BC / 16; ++s) {
      bf16x8_t fa[WI][NA], fb[WJ][NB];
#pragma unroll
      for (int i = 0; i < WI; ++i) SA::read(la, wi * (EI / 2) + i * 32, s, lane, fa[i]);
#pragma unroll
      for (int j = 0; j < WJ; ++j) SB::read(lb, wj * (EJ / 2) + j * 32, s, lane, fb[j]);
      mfma_terms<NA, NB, WI, WJ>(fa, fb, acc);
    }
  }
#pragma unroll
  for (int i = 0; i < WI; ++i)
#pragma unroll
    for (int j = 0; j < WJ; ++j)
      form_again<BF, AKC, BKC, NA, NB, AMUL, BMUL>(a, i0 + wi * (EI / 2) + i * 32, j0 + wj * (EJ / 2) + j * 32, c0, BC, BC, c1, lane, acc[i][j]);
  if constexpr (EPI == EPI_GW) {
    if (sums) {   // the threads that took the same columns, in order (a column's chunks: threads q, q + EJ/8, ...)
      static_assert(!BKC, "the rows of the slice are contraction places");
      __syncthreads();
      float* sh = reinterpret_cast<float*>(smem);
      constexpr int Q = EJ / 8;   // threads of a row; 256 / Q rows at a time
#pragma unroll
      for (int u = 1; u < SB::CH; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) cs[0][k] += cs[u][k];
#pragma unroll
      for (int k = 0; k < 8; ++k) sh[tid / Q * EJ + (tid % Q) * 8 + k] = cs[0][k];
      __syncthreads();
      if (tid < EJ && j0 + tid < a.J) {
        float s = sh[tid];
        for (int k = 1; k < 256 / Q; ++k) s += sh[k * EJ + tid];
        a.colsum[(size_t)split * a.J + j0 + tid] = s;
      }
    }
  }
  if constexpr (EPI == EPI_GW) {   // (float32: 32 lanes are a line as they are)
    float* out = a.partial + (size_t)split * a.I * a.J;
#pragma unroll
    for (int i = 0; i < WI; ++i)
#pragma unroll
      for (int j = 0; j < WJ; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = i0 + wi * (EI / 2) + i * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
          const int q = j0 + wj * (EJ / 2) + j * 32 + (lane & 31);
          if (r < a.I && q < a.J) out[(size_t)r * a.J + q] = acc[i][j][v];
        }
    return;
  }
  store_tile<BF, EPI, EI, EJ>(a, acc, bias, i0, j0, wave, lane, smem);
}

// The result's tile of 128 x 128 where operand b is packed; a: neighbours along the contraction. The slice of a is in LDS twice: one is
// multiplied while the next is written, a barrier between.
template <bool BF, int EPI, int NA, int NB, bool MUL>
__global__ void __launch_bounds__(256, 2) k_dense_packed(DenseArgs a) {
  constexpr int BC = slice_places(NA, NB), KS = BC / 16;
  using SA = Slice<128, true, NA, BC>;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wi = wave >> 1, wj = wave & 1;
  int ti, tj, split;
  if (!tile_of(a, ti, tj, split)) return;
  const int i0 = ti * 128, j0 = tj * 128;
  f32x16_t acc[2][2] = {};
  Raw<BF, MUL> va[SA::CH];
  float bias[4] = {};
  if (EPI == EPI_Y && a.bias) {
    const int q = j0 + wj * 64 + lane % 16 * 4;
    if (q < a.J) get4(a.bias, q, bias, a.J - q);
  }
  const u32x4_t* pb = a.packed + ((size_t)(tj * 4 + wj * 2) * a.pkb) * 64 + lane;
  bf16x8_t fb[KS][2][NB];
  auto fetch_b = [&](int c, int s) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < NB; ++t) fb[s][j][t] = __builtin_bit_cast(bf16x8_t, pb[((size_t)t * a.pterm + (size_t)j * a.pkb + c / 16 + s) * 64]);
  };
  SA::template fetch<BF, MUL>(a.a, i0, 0, a.I, a.C, a.C, tid, va);
#pragma unroll
  for (int s = 0; s < KS; ++s) fetch_b(0, s);
  SA::template stage<BF, MUL>(reinterpret_cast<unsigned short*>(smem), tid, va, nullptr);
  if (BC < a.C) SA::template fetch<BF, MUL>(a.a, i0, BC, a.I, a.C, a.C, tid, va);
  __syncthreads();
  for (int c = 0, at = 0; c < a.C; c += BC, at ^= 1) {
    const unsigned short* la = reinterpret_cast<const unsigned short*>(smem + at * SA::BYTES);
    const bool more = c + BC < a.C;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      bf16x8_t fa[2][NA];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NA; ++t)
          fa[i][t] = *reinterpret_cast<const bf16x8_t*>(la + t * SA::PLANE + (wi * 64 + i * 32 + (lane & 31)) * SA::PITCH + 16 * s + 8 * (lane >> 5));
      mfma_terms<NA, NB, 2, 2>(fa, fb[s], acc);
      if (more) fetch_b(c + BC, s);
    }
    if (more) {
      SA::template stage<BF, MUL>(reinterpret_cast<unsigned short*>(smem + (at ^ 1) * SA::BYTES), tid, va, nullptr);
      if (c + 2 * BC < a.C) SA::template fetch<BF, MUL>(a.a, i0, c + 2 * BC, a.I, a.C, a.C, tid, va);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)   // (W [K][N] is operand b of y, and of g_x by its rows)
      form_again<BF, true, EPI == EPI_GX, NA, NB, MUL, false>(a, i0 + wi * 64 + i * 32, j0 + wj * 64 + j * 32, 0, BC, BC, a.C, lane, acc[i][j]);
  store_tile<BF, EPI, 128, 128>(a, acc, bias, i0, j0, wave, lane, smem);
}

// W [K][N] in fragments: lane (n = lane & 31, g) of fragment (32 columns jb, 16 places kb) holds B[16 kb + 8 g + 0..7][32 jb + n], in NT bf16
// terms; zeros past the edges. First B = W (nf fragments a term), then B = W^T.
struct PackArgs {
  const void* W;
  int K, N;
  u32x4_t* fwd;
  int fkb, fterm;   // fragments per 32 columns and of a term; 0: not wanted
  u32x4_t* bwd;
  int bkb, bterm;
};
template <bool BF>
__global__ void __launch_bounds__(256) k_pack(PackArgs a) {
  constexpr int NT = BF ? 1 : 3;
  long f = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const bool back = f >= a.fterm;
  if (back) f -= a.fterm;
  if (back && f >= a.bterm) return;
  const int nkb = back ? a.bkb : a.fkb, jb = (int)(f / nkb), kb = (int)(f % nkb);
  const int c0 = kb * 16 + 8 * (lane >> 5), j = jb * 32 + (lane & 31);   // contraction places and column
  const int C = back ? a.N : a.K, J = back ? a.K : a.N;
  const size_t sc = back ? 1 : a.N, sj = back ? a.N : 1;
  float v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const bool ok = c0 + k < C && j < J;
    const size_t at = ok ? (c0 + k) * sc + j * sj : 0;
    float x;
    if constexpr (BF) x = __uint_as_float((unsigned)static_cast<const unsigned short*>(a.W)[at] << 16);
    else x = static_cast<const float*>(a.W)[at];
    v[k] = ok ? x : 0.f;
  }
  u32x4_t o[NT];
  split8<NT>(v, o);
#pragma unroll
  for (int t = 0; t < NT; ++t) (back ? a.bwd : a.fwd)[((size_t)t * (back ? a.bterm : a.fterm) + f) * 64 + lane] = o[t];
}

// 32 x 32 of the result; wavefront w takes contraction places 16 w + 64 t + 0..15
template <bool BF, int EPI, bool AKC, bool BKC, int NA, int NB, bool AMUL, bool BMUL>
__global__ void __launch_bounds__(256) k_dense_small(DenseArgs a) {
  __shared__ float join[4][16][64];
  __shared__ float cjoin[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5;
  int ti, tj, split;
  if (!tile_of(a, ti, tj, split)) return;
  const int i = ti * 32 + (lane & 31), j = tj * 32 + (lane & 31);
  const int c0 = split * a.per_split, c1 = min(a.C, c0 + a.per_split);
  f32x16_t acc[1][1] = {};
  float cs = 0.f;
  float bias[4] = {};   // of the four columns that this thread finishes
  if (EPI == EPI_Y && a.bias) {
    const int q = tj * 32 + (threadIdx.x & 7) * 4;
    if (q < a.J) get4(a.bias, q, bias, a.J - q);
  }
  // the lane's eight contraction places c + 0..7 of row e of an operand
  auto get = [&](auto kc, auto mul, const Operand& o, int e, int ne, int c, float (&v)[8]) {
    if constexpr (decltype(kc)::value) {
      load8<BF, decltype(mul)::value>(o, (size_t)(e < ne ? e : 0) * o.ld + (c < c1 ? c : 0), e < ne ? c1 - c : 0, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool ok = c + k < c1 && e < ne;
        const size_t at = (size_t)(ok ? c + k : 0) * o.ld + (ok ? e : 0);
        float x;
        if constexpr (BF) x = __uint_as_float((unsigned)static_cast<const unsigned short*>(o.p)[at] << 16);
        else x = static_cast<const float*>(o.p)[at];
        if constexpr (decltype(mul)::value) x *= o.mul[at];
        v[k] = ok ? x : 0.f;
      }
    }
  };
  for (int c = c0 + wave * 16; c < c1; c += 64) {
    float x[8], y[8];
    get(std::bool_constant<AKC>{}, std::bool_constant<AMUL>{}, a.a, i, a.I, c + 8 * g, x);
    get(std::bool_constant<BKC>{}, std::bool_constant<BMUL>{}, a.b, j, a.J, c + 8 * g, y);
    u32x4_t ua[NA], ub[NB];
    split8<NA>(x, ua);
    split8<NB>(y, ub);
    bf16x8_t fa[1][NA], fb[1][NB];
#pragma unroll
    for (int q = 0; q < NA; ++q) fa[0][q] = __builtin_bit_cast(bf16x8_t, ua[q]);
#pragma unroll
    for (int q = 0; q < NB; ++q) fb[0][q] = __builtin_bit_cast(bf16x8_t, ub[q]);
    mfma_terms<NA, NB, 1, 1>(fa, fb, acc);
    if constexpr (EPI == EPI_GW) {
#pragma unroll
      for (int k = 0; k < 8; ++k) cs += y[k];
    }
  }
  form_again<BF, AKC, BKC, NA, NB, AMUL, BMUL>(a, ti * 32, tj * 32, c0 + wave * 16, 16, 64, c1, lane, acc[0][0]);
#pragma unroll
  for (int v = 0; v < 16; ++v) join[wave][v][lane] = acc[0][0][v];
  if constexpr (EPI == EPI_GW) cjoin[wave][lane] = cs;
  __syncthreads();
  if constexpr (EPI == EPI_GW) {
    if (wave == 0 && a.colsum && ti == 0 && lane < 32 && j < a.J) {
      float s = 0.f;
      for (int w = 0; w < 4; ++w) s += cjoin[w][lane] + cjoin[w][lane + 32];
      a.colsum[(size_t)split * a.J + j] = s;
    }
  }
  // the shares are added in the order of the wavefronts; a thread finishes four neighbours of a row
  {
    const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 4;
    const int r = ti * 32 + row, q = tj * 32 + col;
    if (r < a.I && q < a.J) {
      const int reg = 4 * (row >> 3) + (row & 3), l0 = 32 * ((row >> 2) & 1) + col;   // of the accumulators
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = ((join[0][reg][l0 + k] + join[1][reg][l0 + k]) + join[2][reg][l0 + k]) + join[3][reg][l0 + k];
      float res[4] = {};
      if (EPI != EPI_GW && a.res) get4(static_cast<const typename std::conditional<BF, unsigned short, float>::type*>(a.res), (size_t)r * a.J + q, res, a.J - q);
      finish4<BF, EPI>(a, r, q, v, a.J - q, split, bias, res);
    }
  }
}

// gW and g_b: the splits' partials in order
__global__ void __launch_bounds__(256) k_dense_reduce(const float* partial, const float* colsum, int nsplit, int64_t n, int J, float* gW, float* g_b) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const float* p;
  int64_t stride;
  float* out;
  if (t < n) {
    p = partial + t; stride = n; out = gW + t;
  } else if (colsum && t - n < J) {
    p = colsum + (t - n); stride = J; out = g_b + (t - n);
  } else {
    return;
  }
  float s = 0.f;
  for (int k = 0; k < nsplit; k += 8) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = p[min(k + u, nsplit - 1) * stride];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += k + u < nsplit ? v[u] : 0.f;
  }
  *out = s;
}

__global__ void k_dense_zero(float* gW, int64_t n, float* g_b, int J) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t < n) gW[t] = 0.f;
  if (g_b && t < J) g_b[t] = 0.f;
}

// float -> bf16, nearest even
__global__ void __launch_bounds__(256) k_round_bf16(int64_t n, const float* src, unsigned short* dst) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i + 8 <= n) {
    const float4 x = *reinterpret_cast<const float4*>(src + i), y = *reinterpret_cast<const float4*>(src + i + 4);
    const u32x4_t w = {pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w)};
    *reinterpret_cast<u32x4_t*>(dst + i) = w;
  } else {
    for (int64_t k = i; k < n; ++k) dst[k] = (unsigned short)f2bf_bits(src[k]);
  }
}

// -------------------------------------------------------------------------------------------------------------------------
// Tiles of 128 fill the matrix cores best, but only with a workgroup for most compute units; below, tiles of 64, and where even
// those would leave most of the chip idle, 32 x 32 with the contraction dealt out inside the workgroup.
enum { SIZE_32, SIZE_64, SIZE_128 };
int tile_size(int64_t I, int64_t J, int64_t splits) {
  const int64_t cu = num_cus();
  auto tiles = [&](int e) { return ((I + e - 1) / e) * ((J + e - 1) / e) * splits; };
  if (tiles(128) >= cu) return SIZE_128;
  return tiles(64) >= cu / 2 ? SIZE_64 : SIZE_32;
}

// Splits of the weight gradient's contraction (the rows): as many workgroups as run at once, two per compute unit, and no more (7,703 x 866 x
// 889 float32: 11 splits of 49 tiles, 539 workgroups, took a second turn of them), at least 128 rows each.
struct WSplit {
  int size, nsplit, per;
};
WSplit weight_split(int64_t M, int64_t K, int64_t N) {
  const int64_t cu = num_cus();
  for (int size : {SIZE_128, SIZE_64, SIZE_32}) {
    const int e = size == SIZE_128 ? 128 : size == SIZE_64 ? 64 : 32;
    const int64_t tiles = ((K + e - 1) / e) * ((N + e - 1) / e);
    const int64_t want = 2 * cu / tiles, most = (M + 127) / 128;
    int64_t s = want < most ? want : most;
    if (s < 1) s = 1;
    if (size != SIZE_32 && tiles * s < cu / 2) continue;   // a smaller tile makes more workgroups
    int64_t per = (M + s - 1) / s;
    per = (per + 63) / 64 * 64;
    return {size, (int)((M + per - 1) / per), (int)per};
  }
  return {SIZE_32, 1, (int)M};
}

template <bool BF, int EPI, int E, bool AKC, bool BKC, int NA, int NB, bool AMUL, bool BMUL>
int32_t launch_tile(hipStream_t st, const DenseArgs& a) {
  constexpr int BC = slice_places(NA, NB);
  const int lds_in = Slice<E, AKC, NA, BC>::BYTES + Slice<E, BKC, NB, BC>::BYTES, lds_out = EPI == EPI_GW ? 256 * 8 * 4 : 4 * 32 * (E / 2 + 4) * 4;
  const int64_t n = (int64_t)a.ti * a.tj * a.nsplit;
  k_dense<BF, EPI, E, E, AKC, BKC, NA, NB, AMUL, BMUL><<<(unsigned)((n + 7) / 8 * 8), 256, lds_in > lds_out ? lds_in : lds_out, st>>>(a);
  HGNN_LAUNCH_CHECK("k_dense");
  return HGNN_OK;
}

template <bool BF, int EPI, bool AKC, bool BKC, int NA, int NB, bool AMUL, bool BMUL>
int32_t launch_size(hipStream_t st, DenseArgs a, int size) {
  const int e = size == SIZE_128 ? 128 : size == SIZE_64 ? 64 : 32;
  a.ti = (a.I + e - 1) / e;
  a.tj = (a.J + e - 1) / e;
  if constexpr (EPI == EPI_GW) {   // (the products with W: k_dense_packed)
    if (size == SIZE_128) return launch_tile<BF, EPI, 128, AKC, BKC, NA, NB, AMUL, BMUL>(st, a);
  }
  if (size == SIZE_64) return launch_tile<BF, EPI, 64, AKC, BKC, NA, NB, AMUL, BMUL>(st, a);
  const int64_t n = (int64_t)a.ti * a.tj * a.nsplit;
  k_dense_small<BF, EPI, AKC, BKC, NA, NB, AMUL, BMUL><<<(unsigned)((n + 7) / 8 * 8), 256, 0, st>>>(a);
  HGNN_LAUNCH_CHECK("k_dense_small");
  return HGNN_OK;
}

int32_t check_dense(int64_t M, int32_t K, int32_t N, int32_t act, int32_t dtype) {
  HGNN_REQUIRE(M >= 0, HGNN_ERR_BAD_SHAPE, "negative number of rows");
  HGNN_REQUIRE(K >= 1 && K <= 8192 && N >= 1 && N <= 8192, HGNN_ERR_BAD_SHAPE, "dense: widths must be in 1..8192 (got %d, %d)", K, N);
  HGNN_REQUIRE(act == HGNN_ACT_NONE || act == HGNN_ACT_SILU || act == HGNN_ACT_GELU, HGNN_ERR_BAD_SHAPE, "unknown activation %d", act);
  HGNN_REQUIRE(dtype == HGNN_F32 || dtype == HGNN_BF16, HGNN_ERR_BAD_SHAPE, "unknown dtype %d", dtype);
  HGNN_REQUIRE(M <= (1 << 26), HGNN_ERR_OVERFLOW, "dense: at most 2^26 rows");
  return HGNN_OK;
}

// fragments of a packed operand of C places and J columns: whole slices, whole tiles
struct Packed {
  int kb, term;   // fragments per 32 columns, of a term
  size_t bytes;
};
Packed packed_of(int C, int J, bool bf16) {
  Packed p;
  p.kb = (C + 63) / 64 * 4;
  p.term = p.kb * ((J + 127) / 128 * 4);
  p.bytes = (size_t)p.term * 1024 * (bf16 ? 1 : 3);
  return p;
}

// saved: act'(z), then W^T packed for the reverse pass
struct DenseSaved {
  float* dact;
  u32x4_t* wt;
  size_t bytes;
};
DenseSaved carve_saved(void* p, int64_t M, int K, int N, int act, bool bf16) {
  Carver c(p);
  DenseSaved s;
  s.dact = act == HGNN_ACT_NONE ? nullptr : c.take<float>((size_t)M * N);
  s.wt = tile_size(M, K, 1) == SIZE_128 ? c.take<u32x4_t>(packed_of(N, K, bf16).bytes / 16) : nullptr;
  s.bytes = c.used();
  return s;
}
// workspace: of the forward pass W packed, of the reverse pass the splits' partials
size_t fwd_ws_bytes(int64_t M, int K, int N, bool bf16) { return tile_size(M, N, 1) == SIZE_128 ? packed_of(K, N, bf16).bytes : 0; }
size_t bwd_ws_bytes(int64_t M, int K, int N) {
  if (M == 0) return 0;
  const WSplit w = weight_split(M, K, N);
  return w.nsplit > 1 ? (size_t)w.nsplit * ((size_t)K * N + N) * sizeof(float) : 0;
}

// Terms of an operand with factors, g_z = g_y act'(z). A bf16 call takes two (one: g_x off by 2.3e-3 instead of 1.7e-3 at 40,041 x 512 -> 256, in
// the same time; 132 us instead of 140 for both directions at 8,400 x 866 -> 889, where the matrix cores are the limit).
constexpr int terms_of_gz(bool bf16, bool mul) { return !bf16 ? 3 : mul ? 2 : 1; }

template <bool BF, int EPI, bool MUL>
int32_t launch_packed(hipStream_t st, DenseArgs a, const u32x4_t* packed) {
  constexpr int NA = terms_of_gz(BF, MUL), NB = BF ? 1 : 3, lds_in = 2 * Slice<128, true, NA, slice_places(NA, NB)>::BYTES, lds_out = 4 * 32 * (64 + 4) * 4;
  const Packed p = packed_of(a.C, a.J, BF);
  a.packed = packed; a.pkb = p.kb; a.pterm = p.term;
  a.ti = (a.I + 127) / 128;
  a.tj = (a.J + 127) / 128;
  const int64_t n = (int64_t)a.ti * a.tj;
  k_dense_packed<BF, EPI, NA, NB, MUL><<<(unsigned)((n + 7) / 8 * 8), 256, lds_in > lds_out ? lds_in : lds_out, st>>>(a);
  HGNN_LAUNCH_CHECK("k_dense_packed");
  return HGNN_OK;
}

template <bool BF>
int32_t run_fwd(hipStream_t st, const DenseArgs& a, const void* W, u32x4_t* packed, u32x4_t* wt) {
  const bool large = tile_size(a.I, a.J, 1) == SIZE_128;
  if (large || wt) {
    PackArgs p{};
    p.W = W; p.K = a.C; p.N = a.J;
    if (large) {
      const Packed f = packed_of(a.C, a.J, BF);
      p.fwd = packed; p.fkb = f.kb; p.fterm = f.term;
    }
    if (wt) {
      const Packed f = packed_of(a.J, a.C, BF);
      p.bwd = wt; p.bkb = f.kb; p.bterm = f.term;
    }
    k_pack<BF><<<(unsigned)((p.fterm + p.bterm + 3) / 4), 256, 0, st>>>(p);
    HGNN_LAUNCH_CHECK("k_pack");
  }
  if (large) return launch_packed<BF, EPI_Y, false>(st, a, packed);
  return launch_size<BF, EPI_Y, true, false, BF ? 1 : 3, BF ? 1 : 3, false, false>(st, a, tile_size(a.I, a.J, 1));
}

template <bool BF, bool MUL>
int32_t run_bwd(hipStream_t st, int M, int K, int N, const void* x, const void* W, const u32x4_t* wt, const float* dact, const void* g_y,
                const void* r_x, void* g_x, float* gW, float* g_b, float* ws) {
  if (g_x) {
    DenseArgs a{};
    a.I = M; a.J = K; a.C = N;
    a.a = {g_y, dact, N};
    a.b = {W, nullptr, N};
    a.res = r_x; a.out = g_x; a.nsplit = 1; a.per_split = N;
    if (wt) HGNN_TRY((launch_packed<BF, EPI_GX, MUL>(st, a, wt)));
    else HGNN_TRY((launch_size<BF, EPI_GX, true, true, terms_of_gz(BF, MUL), BF ? 1 : 3, MUL, false>(st, a, tile_size(M, K, 1))));
  }
  const WSplit w = weight_split(M, K, N);
  DenseArgs a{};
  a.I = K; a.J = N; a.C = M;
  a.a = {x, nullptr, K};
  a.b = {g_y, dact, N};
  a.nsplit = w.nsplit; a.per_split = w.per;
  const int64_t n = (int64_t)K * N;
  a.partial = w.nsplit > 1 ? ws : gW;
  a.colsum = g_b ? (w.nsplit > 1 ? ws + (size_t)w.nsplit * n : g_b) : nullptr;
  HGNN_TRY((launch_size<BF, EPI_GW, false, false, BF ? 1 : 3, terms_of_gz(BF, MUL), false, MUL>(st, a, w.size)));
  if (w.nsplit > 1) {
    k_dense_reduce<<<(unsigned)((n + N + 255) / 256), 256, 0, st>>>(a.partial, a.colsum, w.nsplit, n, N, gW, g_b);
    HGNN_LAUNCH_CHECK("k_dense_reduce");
  }
  return HGNN_OK;
}

}  // namespace
}  // namespace hgnn

using namespace hgnn;

extern "C" int32_t hgnn_dense_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t act, int32_t dtype, size_t* ws_bytes_host,
                                              size_t* saved_bytes_host) {
  HGNN_TRY(check_dense(M, K, N, act, dtype));
  HGNN_REQUIRE(ws_bytes_host && saved_bytes_host, HGNN_ERR_NULLPTR, "null size pointer");
  const size_t f = fwd_ws_bytes(M, K, N, dtype == HGNN_BF16), b = bwd_ws_bytes(M, K, N);
  *ws_bytes_host = f > b ? f : b;
  *saved_bytes_host = carve_saved(nullptr, M, K, N, act, dtype == HGNN_BF16).bytes;
  return HGNN_OK;
}

extern "C" int32_t hgnn_dense_fwd(void* stream, int32_t M, int32_t K, int32_t N, int32_t act, int32_t dtype, const void* x, const void* W,
                                  const float* b, const void* r, void* y, void* saved, size_t saved_bytes, void* ws, size_t ws_bytes) {
  HGNN_TRY(check_dense(M, K, N, act, dtype));
  if (M == 0) return HGNN_OK;
  HGNN_REQUIRE(x && W && y, HGNN_ERR_NULLPTR, "dense_fwd: null pointer");
  const DenseSaved s = carve_saved(saved, M, K, N, act, dtype == HGNN_BF16);
  HGNN_REQUIRE(!saved || saved_bytes >= s.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "dense saved buffer: need %zu bytes, got %zu", s.bytes, saved_bytes);
  const size_t need = fwd_ws_bytes(M, K, N, dtype == HGNN_BF16);
  HGNN_REQUIRE(need == 0 || ws, HGNN_ERR_NULLPTR, "dense_fwd: null workspace");
  HGNN_REQUIRE(ws_bytes >= need, HGNN_ERR_WORKSPACE_TOO_SMALL, "dense workspace: need %zu bytes, got %zu", need, ws_bytes);
  DenseArgs a{};
  a.I = M; a.J = N; a.C = K;
  a.a = {x, nullptr, K};
  a.b = {W, nullptr, N};
  a.act = act; a.bias = b; a.res = r; a.out = y;
  a.dact = saved ? s.dact : nullptr;
  a.nsplit = 1; a.per_split = K;
  hipStream_t st = static_cast<hipStream_t>(stream);
  u32x4_t *pk = static_cast<u32x4_t*>(ws), *wt = saved ? s.wt : nullptr;
  ProfScope ps(PT_DENSE, st);
  return dtype == HGNN_BF16 ? run_fwd<true>(st, a, W, pk, wt) : run_fwd<false>(st, a, W, pk, wt);
}

extern "C" int32_t hgnn_dense_bwd(void* stream, int32_t M, int32_t K, int32_t N, int32_t act, int32_t dtype, const void* x, const void* W,
                                  const void* saved, size_t saved_bytes, const void* g_y, const void* r_x, void* g_x, float* gW, float* g_b,
                                  void* ws, size_t ws_bytes) {
  HGNN_TRY(check_dense(M, K, N, act, dtype));
  HGNN_REQUIRE(gW && (g_x || !r_x || M == 0), HGNN_ERR_NULLPTR, "dense_bwd: null pointer");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (M == 0) {
    const int64_t n = (int64_t)K * N;
    k_dense_zero<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(gW, n, g_b, N);
    HGNN_LAUNCH_CHECK("k_dense_zero");
    return HGNN_OK;
  }
  HGNN_REQUIRE(x && W && g_y, HGNN_ERR_NULLPTR, "dense_bwd: null pointer");
  const DenseSaved s = carve_saved(const_cast<void*>(saved), M, K, N, act, dtype == HGNN_BF16);
  const size_t wneed = bwd_ws_bytes(M, K, N);
  HGNN_REQUIRE(s.bytes == 0 || saved, HGNN_ERR_NULLPTR, "dense_bwd: null saved buffer");
  HGNN_REQUIRE(saved_bytes >= s.bytes || s.bytes == 0, HGNN_ERR_WORKSPACE_TOO_SMALL, "dense saved buffer: need %zu bytes, got %zu", s.bytes, saved_bytes);
  HGNN_REQUIRE(wneed == 0 || ws, HGNN_ERR_NULLPTR, "dense_bwd: null workspace");
  HGNN_REQUIRE(ws_bytes >= wneed, HGNN_ERR_WORKSPACE_TOO_SMALL, "dense workspace: need %zu bytes, got %zu", wneed, ws_bytes);
  float* w = static_cast<float*>(ws);
  ProfScope ps(PT_DENSE, st);
  if (dtype == HGNN_BF16)
    return act == HGNN_ACT_NONE ? run_bwd<true, false>(st, M, K, N, x, W, s.wt, nullptr, g_y, r_x, g_x, gW, g_b, w)
                                : run_bwd<true, true>(st, M, K, N, x, W, s.wt, s.dact, g_y, r_x, g_x, gW, g_b, w);
  return act == HGNN_ACT_NONE ? run_bwd<false, false>(st, M, K, N, x, W, s.wt, nullptr, g_y, r_x, g_x, gW, g_b, w)
                              : run_bwd<false, true>(st, M, K, N, x, W, s.wt, s.dact, g_y, r_x, g_x, gW, g_b, w);
}

extern "C" int32_t hgnn_round_bf16(void* stream, int64_t n, const float* src, void* dst) {
  HGNN_REQUIRE(n >= 0, HGNN_ERR_BAD_SHAPE, "negative count");
  HGNN_REQUIRE(n < (int64_t)1 << 41, HGNN_ERR_OVERFLOW, "round_bf16: n must be below 2^41");
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(src && dst, HGNN_ERR_NULLPTR, "round_bf16: null pointer");
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_DENSE, st);
  constexpr int64_t MOST = (int64_t)((1 << 24) - 1) * 2048;   // values of a launch, which has to have fewer than 2^32 threads
  for (int64_t at = 0; at < n; at += MOST) {
    const int64_t k = n - at < MOST ? n - at : MOST;
    k_round_bf16<<<(unsigned)((k + 2047) / 2048), 256, 0, st>>>(k, src + at, static_cast<unsigned short*>(dst) + at);
    HGNN_LAUNCH_CHECK("k_round_bf16");
  }
  return HGNN_OK;
}
