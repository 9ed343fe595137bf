// hgnn_block_norm_fwd / _bwd: the seam between two blocks in one pass over the rows,
//     x' = x + s * gamma(z) * N(b; w1, c1),   y = N(x'; w0, c0),
// N(u; w, c) = w (u - mu) r + c with r = (mean (u - mu)^2 + eps)^-1/2, mu = mean u (layer norm) or 0 (rms norm).
// Reverse, with g' = g_x' + r0 (t - [mean t] - xh mean(t xh)),  t = w0 g_y,  xh = (x' - mu0) r0:
//     g_x = g',  g_s += g' gamma u,  g_z = g' s u gamma (1 - gamma),  q = g' s gamma,  g_w1 += q bh,  g_c1 += q,
//     g_b = r1 (q w1 - [mean q w1] - bh mean(q w1 bh)),  g_w0 += g_y xh,  g_c0 += g_y.
// Bound by memory: 14 bytes an element forward and 22 in reverse with bf16 blocks and a gate per channel (x, x', g 4 bytes each), a few
// dozen operations. 40,041 x 256 in bf16: 29 and 48 us, 4.9 and 4.7 TB/s; 7,703 x 866 in float32: 24 and 37 us, 4.4 TB/s.
// A row stays in the registers of LPR lanes of one wavefront (LPR = 16, 32 or 64 by the width), so every
// tensor is read and written once and the sums of a row are lane exchanges; no shared memory, no barrier in the loop. The
// reverse pass keeps the five parameter gradients of its columns in registers over all rows that a workgroup takes and leaves
// one partial per workgroup, which a second launch adds up in order.
#include "common.h"
#include "devmath.h"
#include "prof.h"

namespace hgnn {
namespace {

struct NormArgs {
  int N, H;
  int first;                 // first row of a forward launch
  int layer, gate;
  float eps;
  const float *x, *P;
  const void *b, *z;
  float* x_out;
  void* y;
  float* saved;              // [N][4]: mu and r of b, mu and r of x'
  const float* g_x_out;
  const void* g_y;
  float *g_x, *gP, *partial;
  void *g_b, *g_z;
};

// V consecutive elements as floats (T: float, or unsigned short for bf16)
template <class T, int V>
__device__ __forceinline__ void load_v(const T* p, float (&o)[V]) {
  struct alignas(sizeof(T) * V) Pack { T e[V]; };
  const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4) o[i] = k.e[i];
    else o[i] = __uint_as_float((unsigned)k.e[i] << 16);
  }
}
template <class T, int V>
__device__ __forceinline__ void store_v(T* p, const float (&o)[V]) {
  struct alignas(sizeof(T) * V) Pack { T e[V]; } k;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4) k.e[i] = o[i];
    else k.e[i] = (T)f2bf_bits(o[i]);
  }
  *reinterpret_cast<Pack*>(p) = k;
}

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int m = LPR / 2; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// sigmoid with an exact quotient: 1 / (1 + exp(-z))
__device__ __forceinline__ float sigmoid_f(float z) { return 1.0f / (1.0f + __expf(-z)); }

// element c * LPR * V + lane * V + i of the row is u[c][i]; ok: chunks that exist
#define HGNN_EACH(...)                                  \
  _Pragma("unroll") for (int c = 0; c < NC; ++c) {      \
    if (col + c * LPR * V < a.H) {                      \
      _Pragma("unroll") for (int i = 0; i < V; ++i) {   \
        __VA_ARGS__                                     \
      }                                                 \
    }                                                   \
  }

template <int LPR, int V, int NC>
__device__ __forceinline__ void moments(const NormArgs& a, int col, const float (&u)[NC][V], float& mu, float& r) {
  float s = 0.f;
  mu = 0.f;
  if (a.layer) {
    HGNN_EACH(s += u[c][i];)
    mu = row_sum<LPR>(s) / a.H;
  }
  s = 0.f;
  HGNN_EACH(const float d = u[c][i] - mu; s = fmaf(d, d, s);)
  r = 1.0f / sqrtf(row_sum<LPR>(s) / a.H + a.eps);
}

template <class T, int LPR, int V, int NC>
__global__ void __launch_bounds__(256) k_norm_fwd(NormArgs a) {
  constexpr int RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, sub = lane / LPR;
  const long row = a.first + ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * RPW + sub;
  const int col = (lane % LPR) * V;
  if (row >= a.N) return;
  const long at = row * a.H + col;
  float x[NC][V] = {}, b[NC][V] = {}, w[NC][V], e[NC][V];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (col + c * LPR * V < a.H) load_v<float, V>(a.x + at + c * LPR * V, x[c]);
  float mu1 = 0.f, r1 = 0.f, mu0 = 0.f, r0 = 0.f;
  if (a.b) {
    float g[NC][V], s[NC][V];
    float ga = 1.f;
    if (a.gate == HGNN_GATE_ATOM) {
      float t[1];
      load_v<T, 1>(static_cast<const T*>(a.z) + row, t);
      ga = sigmoid_f(t[0]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (col + c * LPR * V < a.H) {
        const int o = col + c * LPR * V;
        load_v<T, V>(static_cast<const T*>(a.b) + at + c * LPR * V, b[c]);
        if (a.gate == HGNN_GATE_CHANNEL) load_v<T, V>(static_cast<const T*>(a.z) + at + c * LPR * V, g[c]);
        load_v<float, V>(a.P + o, s[c]);
        load_v<float, V>(a.P + a.H + o, w[c]);
        load_v<float, V>(a.P + 2 * a.H + o, e[c]);
      }
    moments<LPR, V, NC>(a, col, b, mu1, r1);
    HGNN_EACH(const float u = fmaf((b[c][i] - mu1) * r1, w[c][i], e[c][i]);
              const float gm = a.gate == HGNN_GATE_CHANNEL ? sigmoid_f(g[c][i]) : ga;
              x[c][i] = fmaf(s[c][i] * gm, u, x[c][i]);)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (col + c * LPR * V < a.H) store_v<float, V>(a.x_out + at + c * LPR * V, x[c]);
  }
  if (a.y) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (col + c * LPR * V < a.H) {
        load_v<float, V>(a.P + 3 * a.H + col + c * LPR * V, w[c]);
        load_v<float, V>(a.P + 4 * a.H + col + c * LPR * V, e[c]);
      }
    moments<LPR, V, NC>(a, col, x, mu0, r0);
    HGNN_EACH(x[c][i] = fmaf((x[c][i] - mu0) * r0, w[c][i], e[c][i]);)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (col + c * LPR * V < a.H) store_v<T, V>(static_cast<T*>(a.y) + at + c * LPR * V, x[c]);
  }
  if (a.saved && lane % LPR == 0) *reinterpret_cast<float4*>(a.saved + row * 4) = make_float4(mu1, r1, mu0, r0);
}

// Wavefronts per SIMD that the registers of the reverse kernel allow, by the values of a row that a lane holds; as many workgroups
// per compute unit are launched. (With two for all: 67 us at 40,041 x 256 bf16, and 56 at 7,703 x 866 with one.)
constexpr int norm_bwd_waves(int values) { return values <= 4 ? 4 : values <= 8 ? 3 : 2; }

template <class T, int LPR, int V, int NC>
__global__ void __launch_bounds__(256, norm_bwd_waves(V * NC)) k_norm_bwd(NormArgs a) {
  constexpr int RPW = 64 / LPR;
  constexpr bool LP = V * NC > 4;   // the parameters of a lane's columns are kept in LDS, not in registers
  __shared__ float sh[3][NC * LPR * V];
  __shared__ __align__(16) float sp[LP ? 4 * NC * LPR * V : 1];
  const int lane = threadIdx.x & 63, sub = lane / LPR, wave = threadIdx.x >> 6;
  const int col = (lane % LPR) * V;
  float acc[5][NC][V] = {};
  float own[LP ? 1 : 4][NC][V] = {};
  if constexpr (LP) {
    for (int k = 0; k < 4; ++k)
      for (int j = threadIdx.x; j < a.H; j += 256) sp[k * NC * LPR * V + j] = a.P[k * a.H + j];
    __syncthreads();
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (col + c * LPR * V < a.H) load_v<float, V>(a.P + k * a.H + col + c * LPR * V, own[k][c]);
  }
  // parameter k (s, w1, c1, w0) of the lane's column (c, i)
  auto par = [&](int k, int c, int i) {
    if constexpr (LP) return sp[k * NC * LPR * V + c * LPR * V + col + i];
    else return own[k][c][i];
  };
  const float inv = 1.0f / a.H;
  for (long row = ((long)blockIdx.x * 4 + wave) * RPW + sub; row < a.N; row += (long)gridDim.x * 4 * RPW) {
    const long at = row * a.H + col;
    const float4 st = *reinterpret_cast<const float4*>(a.saved + row * 4);
    float g[NC][V] = {}, b[NC][V], z[NC][V];
    float ga = 1.f;
    if (a.g_x_out) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (col + c * LPR * V < a.H) load_v<float, V>(a.g_x_out + at + c * LPR * V, g[c]);
    }
    if (a.b) {
      if (a.gate == HGNN_GATE_ATOM) {
        float t[1];
        load_v<T, 1>(static_cast<const T*>(a.z) + row, t);
        ga = sigmoid_f(t[0]);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (col + c * LPR * V < a.H) {
          load_v<T, V>(static_cast<const T*>(a.b) + at + c * LPR * V, b[c]);
          if (a.gate == HGNN_GATE_CHANNEL) load_v<T, V>(static_cast<const T*>(a.z) + at + c * LPR * V, z[c]);
        }
    }
    if (a.g_y) {
      float x[NC][V], t[NC][V];
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (col + c * LPR * V < a.H) {
          load_v<float, V>(a.x + at + c * LPR * V, x[c]);   // x'
          load_v<T, V>(static_cast<const T*>(a.g_y) + at + c * LPR * V, t[c]);
        }
      float m = 0.f, mx = 0.f;
      HGNN_EACH(x[c][i] = (x[c][i] - st.z) * st.w; acc[3][c][i] = fmaf(t[c][i], x[c][i], acc[3][c][i]); acc[4][c][i] += t[c][i];
                t[c][i] *= par(3, c, i); m += t[c][i]; mx = fmaf(t[c][i], x[c][i], mx);)
      m = a.layer ? row_sum<LPR>(m) * inv : 0.f;
      mx = row_sum<LPR>(mx) * inv;
      HGNN_EACH(g[c][i] += st.w * (t[c][i] - m - x[c][i] * mx);)
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (col + c * LPR * V < a.H) store_v<float, V>(a.g_x + at + c * LPR * V, g[c]);
    if (a.b) {
      float m = 0.f, mx = 0.f, gz = 0.f;
      HGNN_EACH(const float gm = a.gate == HGNN_GATE_CHANNEL ? sigmoid_f(z[c][i]) : ga;
                const float bh = (b[c][i] - st.x) * st.y, w1 = par(1, c, i), u = fmaf(bh, w1, par(2, c, i)), q = g[c][i] * par(0, c, i) * gm;
                acc[0][c][i] = fmaf(g[c][i] * gm, u, acc[0][c][i]); acc[1][c][i] = fmaf(q, bh, acc[1][c][i]); acc[2][c][i] += q;
                z[c][i] = q * u * (1.0f - gm); gz += z[c][i];
                const float t = q * w1; m += t; mx = fmaf(t, bh, mx); g[c][i] = t; b[c][i] = bh;)
      m = a.layer ? row_sum<LPR>(m) * inv : 0.f;
      mx = row_sum<LPR>(mx) * inv;
      HGNN_EACH(b[c][i] = st.y * (g[c][i] - m - b[c][i] * mx);)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (col + c * LPR * V < a.H) {
          store_v<T, V>(static_cast<T*>(a.g_b) + at + c * LPR * V, b[c]);
          if (a.gate == HGNN_GATE_CHANNEL) store_v<T, V>(static_cast<T*>(a.g_z) + at + c * LPR * V, z[c]);
        }
      if (a.gate == HGNN_GATE_ATOM) {
        float t[1] = {row_sum<LPR>(gz)};
        if (lane % LPR == 0) store_v<T, 1>(static_cast<T*>(a.g_z) + row, t);
      }
    }
  }
  // the rows of a wavefront's lane groups, then of the four wavefronts, in order
  float* out = gridDim.x == 1 ? a.gP : a.partial + (size_t)blockIdx.x * 5 * a.H;
#pragma unroll
  for (int k = 0; k < 5; ++k) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int m = LPR; m < 64; m <<= 1) acc[k][c][i] += __shfl_xor(acc[k][c][i], m);
    if (k) __syncthreads();
    if (wave && lane < LPR) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) sh[wave - 1][c * LPR * V + col + i] = acc[k][c][i];
    }
    __syncthreads();
    if (wave == 0 && lane < LPR) {
      HGNN_EACH(const int o = c * LPR * V + col + i;
                out[(size_t)k * a.H + o] = ((acc[k][c][i] + sh[0][o]) + sh[1][o]) + sh[2][o];)
    }
  }
}

// gP[j] = sum over the workgroups' partials, in order within each of 32 runs and then over the runs
__global__ void __launch_bounds__(1024) k_norm_reduce(const float* partial, int np, int n, float* gP) {
  __shared__ float sh[32][33];
  const int c = threadIdx.x & 31, s = threadIdx.x >> 5, j = blockIdx.x * 32 + c;
  const int per = (np + 31) / 32, k1 = min(np, (s + 1) * per);
  float v = 0.f;
  if (j < n)
    for (int k = s * per; k < k1; k += 8) {   // eight loads on their way at a time
      float t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) t[u] = partial[(size_t)min(k + u, k1 - 1) * n + j];
#pragma unroll
      for (int u = 0; u < 8; ++u) v += k + u < k1 ? t[u] : 0.f;
    }
  sh[s][c] = v;
  __syncthreads();
  if (s == 0 && j < n) {
    for (int k = 1; k < 32; ++k) v += sh[k][c];
    gP[j] = v;
  }
}

// values of a row that a lane holds, as launch_norm() chooses them
int norm_values(int H) {
  if (H % 4 == 0) return H <= 256 ? 4 : H <= 512 ? 8 : 16;
  if (H % 2 == 0) return H <= 128 ? 2 : H <= 256 ? 4 : H <= 512 ? 8 : 16;
  return H <= 64 ? 1 : H <= 256 ? 4 : H <= 512 ? 8 : 16;
}

// workgroups of the reverse pass: as many as run at once, fewer where each would have less than one round of rows
int norm_bwd_groups(int N, int H) {
  const int rpw = H % 4 == 0 && H <= 64 ? 4 : H % 4 == 0 && H <= 128 ? 2 : 1;
  const long need = ((long)N + 4 * rpw - 1) / (4 * rpw), most = (long)num_cus() * norm_bwd_waves(norm_values(H));
  return (int)(need < most ? need : most);
}

// the widest access that every row's start is aligned to, and the lanes and chunks that hold a row
template <class T, bool FWD>
void launch_norm(hipStream_t st, NormArgs a, int groups) {
  constexpr int MOST = (1 << 24) - 1;   // workgroups of a launch, which has to have fewer than 2^32 threads
#define HGNN_NORM(LPR, V, NC)                                                                                       \
  do {                                                                                                              \
    constexpr int ROWS = 4 * (64 / LPR);                                                                            \
    if (FWD) {                                                                                                      \
      for (int64_t left = a.N; left > 0; left -= (int64_t)MOST * ROWS) {                                            \
        const int64_t n = (left + ROWS - 1) / ROWS;                                                                 \
        a.first = (int)(a.N - left);                                                                                \
        k_norm_fwd<T, LPR, V, NC><<<(unsigned)(n < MOST ? n : MOST), 256, 0, st>>>(a);                              \
      }                                                                                                             \
    } else {                                                                                                        \
      k_norm_bwd<T, LPR, V, NC><<<groups, 256, 0, st>>>(a);                                                         \
    }                                                                                                               \
    return;                                                                                                         \
  } while (0)
  const int H = a.H;
  if (H % 4 == 0) {
    if (H <= 64) HGNN_NORM(16, 4, 1);
    if (H <= 128) HGNN_NORM(32, 4, 1);
    if (H <= 256) HGNN_NORM(64, 4, 1);
    if (H <= 512) HGNN_NORM(64, 4, 2);
    HGNN_NORM(64, 4, 4);
  }
  if (H % 2 == 0) {
    if (H <= 128) HGNN_NORM(64, 2, 1);
    if (H <= 256) HGNN_NORM(64, 2, 2);
    if (H <= 512) HGNN_NORM(64, 2, 4);
    HGNN_NORM(64, 2, 8);
  }
  if (H <= 64) HGNN_NORM(64, 1, 1);
  if (H <= 256) HGNN_NORM(64, 1, 4);
  if (H <= 512) HGNN_NORM(64, 1, 8);
  HGNN_NORM(64, 1, 16);
#undef HGNN_NORM
}

int32_t check_norm(int32_t N, int32_t H, int32_t norm, int32_t gate, int32_t dtype) {
  HGNN_REQUIRE(N >= 0, HGNN_ERR_BAD_SHAPE, "negative N");
  HGNN_REQUIRE(N < (1 << 26), HGNN_ERR_OVERFLOW, "block_norm: N must be below 2^26");
  HGNN_REQUIRE(H >= 1 && H <= 1024, HGNN_ERR_BAD_SHAPE, "block_norm: H must be in 1..1024 (got %d)", H);
  HGNN_REQUIRE(norm == HGNN_NORM_RMS || norm == HGNN_NORM_LAYER, HGNN_ERR_BAD_SHAPE, "unknown norm %d", norm);
  HGNN_REQUIRE(gate == HGNN_GATE_NONE || gate == HGNN_GATE_ATOM || gate == HGNN_GATE_CHANNEL, HGNN_ERR_BAD_SHAPE, "unknown gate %d", gate);
  HGNN_REQUIRE(dtype == HGNN_F32 || dtype == HGNN_BF16, HGNN_ERR_BAD_SHAPE, "unknown dtype %d", dtype);
  return HGNN_OK;
}

}  // namespace
}  // namespace hgnn

using namespace hgnn;

extern "C" int32_t hgnn_block_norm_workspace_bytes(int32_t N, int32_t H, size_t* ws_bytes_host, size_t* saved_bytes_host) {
  HGNN_TRY(check_norm(N, H, HGNN_NORM_RMS, HGNN_GATE_NONE, HGNN_F32));
  HGNN_REQUIRE(ws_bytes_host && saved_bytes_host, HGNN_ERR_NULLPTR, "null size pointer");
  *ws_bytes_host = (size_t)norm_bwd_groups(N, H) * 5 * H * sizeof(float);
  *saved_bytes_host = (size_t)N * 4 * sizeof(float);
  return HGNN_OK;
}

extern "C" int32_t hgnn_block_norm_fwd(void* stream, int32_t N, int32_t H, int32_t norm, int32_t gate, int32_t dtype, float eps,
                                       const float* x, const void* b, const void* z, const float* P, float* x_out, void* y,
                                       void* saved, size_t saved_bytes) {
  HGNN_TRY(check_norm(N, H, norm, gate, dtype));
  HGNN_REQUIRE(eps >= 0.f, HGNN_ERR_BAD_SHAPE, "block_norm: eps must not be negative");
  HGNN_REQUIRE(b || gate == HGNN_GATE_NONE, HGNN_ERR_BAD_SHAPE, "block_norm: a gate without a block (b is NULL)");
  if (N == 0) return HGNN_OK;
  HGNN_REQUIRE(x && P && (b || y), HGNN_ERR_NULLPTR, "block_norm_fwd: null pointer");
  HGNN_REQUIRE(!b || x_out, HGNN_ERR_NULLPTR, "block_norm_fwd: x_out is needed with b");
  HGNN_REQUIRE(gate == HGNN_GATE_NONE || z, HGNN_ERR_NULLPTR, "block_norm_fwd: the gate needs z");
  HGNN_REQUIRE(!saved || saved_bytes >= (size_t)N * 16, HGNN_ERR_WORKSPACE_TOO_SMALL, "block_norm saved buffer: need %zu bytes, got %zu",
               (size_t)N * 16, saved_bytes);
  NormArgs a{};
  a.N = N; a.H = H; a.layer = norm == HGNN_NORM_LAYER; a.gate = gate; a.eps = eps;
  a.x = x; a.b = b; a.z = z; a.P = P; a.x_out = x_out; a.y = y; a.saved = static_cast<float*>(saved);
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_BLOCK_NORM, st);
  if (dtype == HGNN_BF16) launch_norm<unsigned short, true>(st, a, 0);
  else launch_norm<float, true>(st, a, 0);
  HGNN_LAUNCH_CHECK("k_norm_fwd");
  return HGNN_OK;
}

extern "C" int32_t hgnn_block_norm_bwd(void* stream, int32_t N, int32_t H, int32_t norm, int32_t gate, int32_t dtype,
                                       const float* x_out, const void* b, const void* z, const float* P, const void* saved,
                                       size_t saved_bytes, const float* g_x_out, const void* g_y, float* g_x, void* g_b,
                                       void* g_z, float* gP, void* ws, size_t ws_bytes) {
  HGNN_TRY(check_norm(N, H, norm, gate, dtype));
  HGNN_REQUIRE(b || gate == HGNN_GATE_NONE, HGNN_ERR_BAD_SHAPE, "block_norm: a gate without a block (b is NULL)");
  HGNN_REQUIRE(P && gP, HGNN_ERR_NULLPTR, "block_norm_bwd: null pointer");
  const int groups = norm_bwd_groups(N, H);
  const size_t need = (size_t)groups * 5 * H * sizeof(float);
  HGNN_REQUIRE(ws_bytes >= need, HGNN_ERR_WORKSPACE_TOO_SMALL, "block_norm workspace: need %zu bytes, got %zu", need, ws_bytes);
  if (N > 0) {
    HGNN_REQUIRE(g_x && saved && ws && (g_x_out || g_y) && (!b || g_b), HGNN_ERR_NULLPTR, "block_norm_bwd: null pointer");
    HGNN_REQUIRE(!g_y || x_out, HGNN_ERR_NULLPTR, "block_norm_bwd: g_y needs x_out");
    HGNN_REQUIRE(gate == HGNN_GATE_NONE || (z && g_z), HGNN_ERR_NULLPTR, "block_norm_bwd: the gate needs z and g_z");
    HGNN_REQUIRE(saved_bytes >= (size_t)N * 16, HGNN_ERR_WORKSPACE_TOO_SMALL, "block_norm saved buffer: need %zu bytes, got %zu",
                 (size_t)N * 16, saved_bytes);
  }
  NormArgs a{};
  a.N = N; a.H = H; a.layer = norm == HGNN_NORM_LAYER; a.gate = gate;
  a.x = x_out; a.b = b; a.z = z; a.P = P; a.saved = const_cast<float*>(static_cast<const float*>(saved));
  a.g_x_out = g_x_out; a.g_y = g_y; a.g_x = g_x; a.g_b = g_b; a.g_z = g_z; a.gP = gP; a.partial = static_cast<float*>(ws);
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_BLOCK_NORM, st);
  if (N > 0) {
    if (dtype == HGNN_BF16) launch_norm<unsigned short, false>(st, a, groups);
    else launch_norm<float, false>(st, a, groups);
    HGNN_LAUNCH_CHECK("k_norm_bwd");
  }
  if (groups != 1) {   // (none: no row, zeros)
    k_norm_reduce<<<(5 * H + 31) / 32, 1024, 0, st>>>(a.partial, groups, 5 * H, gP);
    HGNN_LAUNCH_CHECK("k_norm_reduce");
  }
  return HGNN_OK;
}
