// hgnn_pair_plan and hgnn_pair_buckets: the matrix of distance buckets of every graph, one byte a pair.
//
// The distance is that of the nearest of the 27 images j + t, t = (s1 a + s2 b) + s3 c with s in {-1, 0, 1}^3, each formed in
// float32 with every operation rounded on its own (this file is compiled without contraction), so the bytes do not depend
// on how the work is cut: a minimum over values has no ties to break. 12 operations an image and pair, 324 a pair in a
// periodic graph and 12 otherwise, against one byte written: bound by the vector units. A thread takes four neighbouring pairs
// of a row (one 4-byte store), a workgroup eight rows, whose positions and images stay in registers and shared memory.
//
// In a cell more than twice as high as the last boundary R in every direction some ten operations rule out most pairs: an image vector
// r* shorter than R has fractional coordinates |f_k| <= |r*| / h_k < 1/2 (h_k: the cell's heights), so rounding the difference of the
// atoms' fractional coordinates to whole numbers s finds that image, and the rest |d_k| <= R / h_k in every direction. A pair
// that fails this is beyond every boundary. The others are few (all pairs of 20,000 atoms at 75 R^3 an atom: 4 %), so a wavefront lists
// them and forms their distances afterwards with full lanes: that of the image s where that is one of the 27 (every other image is
// longer than h_min - R > R), of all of them where it is not. The margins (1/1000 of R and of the cell) cover the rounding of the
// fractional coordinates, of which cells up to 16 times as long as high and coordinates up to 100 R are good to 5e-4; a pair with larger
// coordinates takes all images. A thread has the fractional coordinates of four atoms for eight rows. 20,000 atoms: 0.22 ms, 1.8 TB/s
// written; with 27 images a pair 2.8 ms.
#include "common.h"
#include "pairs.h"
#include "prof.h"

namespace hgnn {
namespace {

constexpr int PAIR_EDGES = 254;   // most boundaries: buckets 0..254, byte 255 is HGNN_PAIR_NONE

// One workgroup: running sums over the graphs, the check of the offsets, every tile's record, the total for the host. A thread writes the
// records of its graph's first tiles, a wavefront those of its long graphs.
__global__ void __launch_bounds__(1024) k_pair_plan(int N, int G, const int32_t* graph_off, PairPlan v, HostMail* mail) {
  constexpr int OWN = 8;
  __shared__ long long wb[16];
  __shared__ int wt[16], bad_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) bad_s = 0;
  __syncthreads();
  long long base_b = 0;
  int base_t = 0;
  int bad = 0;
  if (tid == 0) bad = graph_off[0] != 0 || graph_off[G] != N;
  for (int g0 = 0; g0 < G; g0 += 1024) {
    const int g = g0 + tid;
    long long bytes = 0;
    int tiles = 0;
    PairTile r{};
    if (g < G) {
      const int lo = graph_off[g], hi = graph_off[g + 1];
      if (lo < 0 || hi < lo || hi > N) bad = 1;
      else {
        r.lo = lo;
        r.n = hi - lo;
        r.g = g;
        bytes = r.n * pair_pitch(r.n);
        tiles = (r.n + PAIR_T - 1) / PAIR_T;
      }
    }
    long long ib = bytes;
    int it = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long ub = __shfl_up(ib, d);
      const int ut = __shfl_up(it, d);
      if (lane >= d) { ib += ub; it += ut; }
    }
    if (lane == 63) { wb[wave] = ib; wt[wave] = it; }
    __syncthreads();
    long long pb = base_b, tb = 0;
    int pt = base_t, tt = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) { pb += wb[w]; pt += wt[w]; }
      tb += wb[w];
      tt += wt[w];
    }
    r.off = pb + ib - bytes;
    const int t0 = pt + it - tiles;
    // (offsets that are refused below may name more tiles than there is room for)
    for (int k = 0; k < OWN && k < tiles; ++k) {
      r.i0 = k * PAIR_T;
      if ((unsigned)(t0 + k) < (unsigned)v.max_tiles) v.tile[t0 + k] = r;
    }
    for (unsigned long long m = __ballot(tiles > OWN); m; m &= m - 1) {
      const int l = __ffsll(m) - 1, s0 = __shfl(t0, l), ns = __shfl(tiles, l);
      PairTile q{};
      q.off = __shfl(r.off, l);
      q.lo = __shfl(r.lo, l);
      q.n = __shfl(r.n, l);
      q.g = __shfl(r.g, l);
      for (int k = OWN + lane; k < ns; k += 64) {
        q.i0 = k * PAIR_T;
        if ((unsigned)(s0 + k) < (unsigned)v.max_tiles) v.tile[s0 + k] = q;
      }
    }
    base_b += tb;
    base_t += tt;
    __syncthreads();
  }
  if (bad) atomicOr(&bad_s, 1);
  __syncthreads();
  if (tid == 0) {
    *v.count = bad_s ? 0 : base_t;
    post_mail(mail, base_b, bad_s);
  }
}

struct BucketArgs {
  int nedge, drop_far;
  int64_t first;          // first tile of this launch
  const float *pos, *cell, *edge2;
  const uint8_t* pbc;
  PairPlan plan;
  uint8_t* pairs;
};

// number of boundaries that do not exceed d2 (a d2 that is no number: all)
__device__ __forceinline__ int boundaries_below(const float* edge, int nedge, float d2) {
  int lo = 0, hi = nedge;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (d2 < edge[m]) hi = m;
    else lo = m + 1;
  }
  return lo;
}

// squared distance over the images m0 .. m1 - 1
__device__ __forceinline__ float nearest(const float4* img, int m0, int m1, float px, float py, float pz, float qx, float qy, float qz) {
  float best = __builtin_inff();
  for (int m = m0; m < m1; ++m) {
    const float4 t = img[m];
    const float x = px - (qx + t.x), y = py - (qy + t.y), z = pz - (qz + t.z);
    best = fminf(best, (x * x + y * y) + z * z);
  }
  return best;
}

constexpr int ROWS = 8, COLS = 256;   // of a workgroup; of a wavefront at a time

// what a roomy cell gives: columns of the inverse, the most that a rest may be in each direction (in 2^-32)
struct Roomy {
  float inv[9];
  unsigned rest[3];
  int yes;
};
__device__ __forceinline__ void fractional(const Roomy& c, const float (&p)[3], float (&f)[3]) {
#pragma unroll
  for (int d = 0; d < 3; ++d) f[d] = __builtin_fmaf(p[0], c.inv[d], __builtin_fmaf(p[1], c.inv[3 + d], p[2] * c.inv[6 + d]));
}
__device__ __forceinline__ bool moderate(const float (&p)[3], float most) {   // (false for what is no number)
  return fabsf(p[0]) < most && fabsf(p[1]) < most && fabsf(p[2]) < most;
}

// fractional part in 2^-32: differences of two wrap around as the rounding to the next whole number asks
__device__ __forceinline__ unsigned turns(float f) { return (unsigned)fminf((f - floorf(f)) * 4294967296.0f, 4294967040.0f); }

struct Rows {
  float4 f[ROWS];   // fractional coordinates; w: 1 where they are not to be used
  float4 p[ROWS];
  uint4 t[ROWS];    // f in turns, plus the most that a rest may be
};

// Pairs of ROWS rows of a roomy cell. A wavefront's items: COLS columns of all rows, or of some where there are few columns.
__device__ __forceinline__ void roomy_rows(const BucketArgs& a, const PairTile& w, int i0, const Roomy& cell, float last, const float4* img, const float* edge,
                                           Rows& rows, unsigned short* list, unsigned* out) {
  const int n = w.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nrows = min(ROWS, n - i0);
  const int64_t pitch = pair_pitch(n);
  const float most = 100.f * last;
  uint8_t* base = a.pairs + w.off + i0 * pitch;
  const float* pos = a.pos + (size_t)w.lo * 3;
  const unsigned far = a.drop_far ? (unsigned)HGNN_PAIR_NONE : (unsigned)a.nedge;
  const Roomy c = cell;
  if (lane < ROWS) {   // (the same by every wavefront)
    const float* s = pos + (size_t)min(i0 + lane, n - 1) * 3;
    const float p[3] = {s[0], s[1], s[2]};
    float f[3];
    fractional(c, p, f);
    rows.f[lane] = make_float4(f[0], f[1], f[2], moderate(p, most) ? 0.f : 1.f);
    rows.p[lane] = make_float4(p[0], p[1], p[2], 0.f);
    rows.t[lane] = make_uint4(turns(f[0]) + c.rest[0], turns(f[1]) + c.rest[1], turns(f[2]) + c.rest[2], 0);
  }
  auto order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); __builtin_amdgcn_wave_barrier(); };
  order();
  const bool wild_rows = __any(lane < ROWS && rows.f[lane & (ROWS - 1)].w != 0.f);
  const int chunks = (int)((pitch + COLS - 1) / COLS), parts = chunks >= 4 ? 1 : 4, per = ROWS / parts;
  for (int item = wave; item < chunks * parts; item += 4) {
    const int j0 = item / parts * COLS, r0 = item % parts * per, r1 = min(nrows, r0 + per), j = j0 + lane * 4;
    if (r0 >= r1) continue;
    unsigned u[4][3], word = 0;
    // a bit per pair, row after row from the highest of `bits` down; columns that exist; pairs to take whatever their coordinates
    const int bits = (r1 - r0) * 4;
    unsigned near = 0, exist = 0, wild = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* s = pos + (size_t)min(j + k, n - 1) * 3;
      const float q[3] = {s[0], s[1], s[2]};
      float f[3];
      fractional(c, q, f);
#pragma unroll
      for (int d = 0; d < 3; ++d) u[k][d] = turns(f[d]);
      const unsigned column = 0x88888888u >> k;
      exist |= j + k < n ? column : 0u;
      wild |= moderate(q, most) ? 0u : column;
      word |= (j + k < n ? far : (unsigned)HGNN_PAIR_NONE) << (8 * k);
    }
    order();
    for (int r = r0; r < r1; ++r) {
      const uint4 i = rows.t[r];
      out[r * 64 + lane] = word;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int close = (int)(i.x - u[k][0] <= 2 * c.rest[0]) & (int)(i.y - u[k][1] <= 2 * c.rest[1]) & (int)(i.z - u[k][2] <= 2 * c.rest[2]);
        near = near + near + close;
      }
    }
    if (wild_rows) {
      for (int r = r0; r < r1; ++r)
        if (rows.f[r].w != 0.f) wild |= 0xfu << (bits - 4 - (r - r0) * 4);
    }
    near = (near | wild) & exist & (0xffffffffu >> (32 - bits));
    int before = __popc(near);   // entries of the lanes up to this one, then of those before it
    const int mine = before;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int t = __shfl_up(before, d);
      if (lane >= d) before += t;
    }
    const int count = __shfl(before, 63);
    before -= mine;
    while (near) {
      const int at = bits - 1 - (31 - __clz(near));
      list[before++] = (unsigned short)((r0 + at / 4) * COLS + lane * 4 + at % 4);
      near &= ~(0x80000000u >> __clz(near));
    }
    order();
    for (int e = lane; e < count; e += 64) {
      const int at = list[e];
      const float4 i = rows.f[at / COLS], p = rows.p[at / COLS];
      const float* s = pos + (size_t)(j0 + at % COLS) * 3;
      const float q[3] = {s[0], s[1], s[2]};
      float g[3];
      fractional(c, q, g);
      const float s0 = rintf(i.x - g[0]), s1 = rintf(i.y - g[1]), s2 = rintf(i.z - g[2]);
      int m0 = 0, m1 = 27;
      if (i.w == 0.f && moderate(q, most) && fmaxf(fmaxf(fabsf(s0), fabsf(s1)), fabsf(s2)) <= 1.f) {
        m0 = 13 + (int)s0 * 9 + (int)s1 * 3 + (int)s2;
        m1 = m0 + 1;
      }
      const unsigned b = boundaries_below(edge, a.nedge, nearest(img, m0, m1, p.x, p.y, p.z, q[0], q[1], q[2]));
      reinterpret_cast<uint8_t*>(out)[at] = (uint8_t)(b == (unsigned)a.nedge ? far : b);
    }
    order();
    for (int e = lane; e < (r1 - r0) * (COLS / 16); e += 64) {
      const int r = r0 + e / (COLS / 16), piece = e % (COLS / 16);
      if (j0 + piece * 16 < pitch) *reinterpret_cast<uint4*>(base + r * pitch + j0 + piece * 16) = *reinterpret_cast<const uint4*>(out + r * 64 + piece * 4);
    }
  }
}

// workgroup: 8 rows of a tile. Cells that are not roomy: thread: row tid / 32, pairs 4 (tid % 32) .. + 3 of every 128
__global__ void __launch_bounds__(256) k_pair_buckets(BucketArgs a) {
  __shared__ float4 img[27];
  __shared__ float edge[PAIR_EDGES + 1];
  __shared__ Roomy cell;
  __shared__ Rows rows;
  __shared__ unsigned short list[4][ROWS * COLS];
  __shared__ __align__(16) unsigned words[4][ROWS * COLS / 4];
  const int64_t tile = a.first + (blockIdx.x >> 2);
  if (tile >= *a.plan.count) return;
  const PairTile w = a.plan.tile[tile];
  const int g = w.g, lo = w.lo, n = w.n, i0 = w.i0 + (blockIdx.x & 3) * ROWS;
  if (i0 >= n) return;
  const bool periodic = a.cell && a.pbc && a.pbc[g];
  const float last2 = a.nedge ? a.edge2[a.nedge - 1] : 0.f, last = sqrtf(last2);
  if (threadIdx.x < 27) {
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (periodic) {
      const float s1 = (int)threadIdx.x / 9 - 1, s2 = (int)threadIdx.x / 3 % 3 - 1, s3 = (int)threadIdx.x % 3 - 1;
      const float* c = a.cell + (size_t)g * 9;
      t.x = (s1 * c[0] + s2 * c[3]) + s3 * c[6];
      t.y = (s1 * c[1] + s2 * c[4]) + s3 * c[7];
      t.z = (s1 * c[2] + s2 * c[5]) + s3 * c[8];
    }
    img[threadIdx.x] = t;
  }
  if (threadIdx.x == 64) {
    bool roomy = periodic;
    if (periodic) {
      const float* c = a.cell + (size_t)g * 9;
      // columns of the inverse: cross products of the other two rows over the determinant; 1 / their lengths are the heights
      float x[3][3];
      for (int k = 0; k < 3; ++k) {
        const float *u = c + (k + 1) % 3 * 3, *v = c + (k + 2) % 3 * 3;
        x[k][0] = u[1] * v[2] - u[2] * v[1];
        x[k][1] = u[2] * v[0] - u[0] * v[2];
        x[k][2] = u[0] * v[1] - u[1] * v[0];
      }
      const float det = (c[0] * x[0][0] + c[1] * x[0][1]) + c[2] * x[0][2];
      float low = __builtin_inff(), size = 0.f;
      for (int k = 0; k < 3; ++k) {
        for (int d = 0; d < 3; ++d) {
          cell.inv[d * 3 + k] = x[k][d] / det;
          size = fmaxf(size, fabsf(c[3 * k + d]));
        }
        const float height = fabsf(det) / sqrtf((x[k][0] * x[k][0] + x[k][1] * x[k][1]) + x[k][2] * x[k][2]);
        roomy = roomy && height > 2.01f * last;   // (false for what is no number: a flat cell)
        cell.rest[k] = (unsigned)(fminf(1.001f * last / height + 0.001f, 0.4999f) * 4294967296.0f);   // (below 1/2 in a roomy cell)
        low = fminf(low, height);
      }
      // (in a cell much longer than high the fractional coordinates lose their accuracy)
      roomy = roomy && size < 16.f * low && size < 100.f * last;
    }
    cell.yes = roomy;
  }
  for (int e = threadIdx.x; e < a.nedge; e += 256) edge[e] = a.edge2[e];
  __syncthreads();
  if (cell.yes) {   // uniform over the workgroup
    const int wave = threadIdx.x >> 6;
    roomy_rows(a, w, i0, cell, last, img, edge, rows, list[wave], words[wave]);
    return;
  }
  const int i = i0 + (threadIdx.x >> 5);
  if (i >= n) return;
  const float* p = a.pos + ((size_t)lo + i) * 3;
  const float px = p[0], py = p[1], pz = p[2];
  const int64_t pitch = pair_pitch(n);
  uint8_t* row = a.pairs + w.off + i * pitch;
  const int first = periodic ? 0 : 13, past = periodic ? 27 : 14;
  for (int j = (threadIdx.x & 31) * 4; j < pitch; j += 128) {
    float q[4][3];
    if (j + 4 <= n) {
      __builtin_memcpy(q, a.pos + ((size_t)lo + j) * 3, 48);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* s = a.pos + ((size_t)lo + (j + k < n ? j + k : n - 1)) * 3;
        q[k][0] = s[0]; q[k][1] = s[1]; q[k][2] = s[2];
      }
    }
    unsigned out = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      unsigned b = boundaries_below(edge, a.nedge, nearest(img, first, past, px, py, pz, q[k][0], q[k][1], q[k][2]));
      if (j + k >= n || (a.drop_far && b == (unsigned)a.nedge)) b = HGNN_PAIR_NONE;
      out |= b << (8 * k);
    }
    *reinterpret_cast<unsigned*>(row + j) = out;
  }
}

}  // namespace
}  // namespace hgnn

using namespace hgnn;

static int32_t check_pair(int32_t N, int32_t G) {
  HGNN_REQUIRE(N >= 0 && G >= 0, HGNN_ERR_BAD_SHAPE, "negative N or G");
  HGNN_REQUIRE(N < (1 << 28) && G < (1 << 28), HGNN_ERR_OVERFLOW, "pair matrix: N and G must be below 2^28");
  return HGNN_OK;
}

extern "C" int32_t hgnn_pair_plan_workspace_bytes(int32_t N, int32_t G, size_t* plan_bytes_host) {
  HGNN_TRY(check_pair(N, G));
  HGNN_REQUIRE(plan_bytes_host, HGNN_ERR_NULLPTR, "null size pointer");
  *plan_bytes_host = pair_plan_view(nullptr, N, G).bytes;
  return HGNN_OK;
}

extern "C" int32_t hgnn_pair_plan(void* stream, int32_t N, int32_t G, const int32_t* graph_off, void* plan, size_t plan_bytes,
                                  int64_t* pair_bytes_host) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  HGNN_TRY(check_pair(N, G));
  HGNN_REQUIRE(graph_off && plan && pair_bytes_host, HGNN_ERR_NULLPTR, "pair_plan: null pointer");
  const PairPlan v = pair_plan_view(plan, N, G);
  HGNN_REQUIRE(plan_bytes >= v.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "pair plan: need %zu bytes, got %zu", v.bytes, plan_bytes);
  MailSlot mail;
  HGNN_TRY(mail.take(st));
  {
    ProfScope ps(PT_PAIRS, st);
    k_pair_plan<<<1, 1024, 0, st>>>(N, G, graph_off, v, mail.dev());
    HGNN_LAUNCH_CHECK("k_pair_plan");
  }
  HGNN_HIP(mail.wait());
  HGNN_REQUIRE(mail.status() == 0, HGNN_ERR_BAD_OFFSETS, "graph_off must start at 0, not decrease and end at N");
  *pair_bytes_host = mail.value();
  return HGNN_OK;
}

extern "C" int32_t hgnn_pair_buckets(void* stream, int32_t N, int32_t G, const void* plan, size_t plan_bytes, const float* pos,
                                     const float* cell, const uint8_t* pbc, int32_t nedge, const float* edge2,
                                     int32_t drop_far, uint8_t* pairs) {
  HGNN_TRY(check_pair(N, G));
  HGNN_REQUIRE(nedge >= 0 && nedge <= PAIR_EDGES, HGNN_ERR_BAD_SHAPE, "pair_buckets: 0..%d boundaries (got %d)", PAIR_EDGES, nedge);
  if (N == 0) return HGNN_OK;
  HGNN_REQUIRE(plan && pos && pairs && (edge2 || nedge == 0), HGNN_ERR_NULLPTR, "pair_buckets: null pointer");
  BucketArgs a{};
  a.plan = pair_plan_view(plan, N, G);
  HGNN_REQUIRE(plan_bytes >= a.plan.bytes, HGNN_ERR_WORKSPACE_TOO_SMALL, "pair plan: need %zu bytes, got %zu", a.plan.bytes, plan_bytes);
  a.nedge = nedge; a.drop_far = drop_far; a.pos = pos; a.cell = cell; a.edge2 = edge2; a.pbc = pbc; a.pairs = pairs;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProfScope ps(PT_PAIRS, st);
  constexpr int64_t MOST = (1 << 22) - 1;   // tiles of a launch, which has to have fewer than 2^32 threads
  for (a.first = 0; a.first < a.plan.max_tiles; a.first += MOST) {
    const int64_t left = a.plan.max_tiles - a.first;
    k_pair_buckets<<<(unsigned)((left < MOST ? left : MOST) * 4), 256, 0, st>>>(a);
    HGNN_LAUNCH_CHECK("k_pair_buckets");
  }
  return HGNN_OK;
}
