// The dense product's own kernels beside the GEMMs: the product of a few rows, fp32 operands as bf16
// planes, the gradient of the pre-activation with the bias gradient.
//   P = X W + b, Y = R + drop(act(P));   dP = drop(dY) act'(P), db = column sums of dP
#include <algorithm>

#include <cooperative_groups.h>

#include "act.cuh"
#include "common.cuh"
#include "kernels.h"

namespace ecmoe {
namespace {

namespace cg = cooperative_groups;

template <typename T>
constexpr bool kFast = sizeof(T) == 2;   // bf16 results: hardware exp2 and reciprocal

// ------------------------------------------------------------------ a few rows
// A row, or fp32 rows in groups of up to 8 (blockIdx.y): the weight is read once a group and the time is
// that stream's. A CTA takes 64 columns and a block of K, its threads 16 bytes of a weight row each (a
// 128-byte line of a bf16 row, two of an fp32 one, to 8 or 16 lanes), several rows in flight; the rows
// of X wait in shared memory in fp32, all of them for one k side by side. The blocks of K are the CTAs
// of a cluster: each leaves its sums in its shared memory, and each then adds up its share of the
// outputs over the cluster, in rank order, and finishes them: no partial sum goes through global
// memory and no second kernel runs. One bf16 row of K 2048, N 4096: 4.9 us of 16.8 MB, of which a launch
// and the cluster's barriers are 3.
constexpr int kRowsThreads = 256, kRowsCols = 64, kRowsSlab = 512;

template <typename T, int R>
__global__ void __launch_bounds__(kRowsThreads)
linear_rows_kernel(const T* __restrict__ X, const T* __restrict__ W, LinearEpi<T> ep, int rows, int K,
                   int N, int kper) {
  pdl_begin(X, W, ep.bias, ep.R, ep.drop.rng);
  constexpr int VN = Vec16<T>::n, COLS = kRowsCols, LPR = COLS / VN, RPW = 32 / LPR;
  constexpr int KP = kRowsThreads / 32 * RPW;       // k rows a pass of the CTA
  constexpr int U = R >= 8 ? 4 : 8;                 // passes in flight
  __shared__ float s_x[kRowsSlab * R];
  __shared__ float s_red[kRowsThreads / 32][R * COLS];
  __shared__ float s_out[R * COLS];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int strip = (int)blockIdx.x / S, row0 = (int)blockIdx.y * R;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int grp = warp * RPW + lane / LPR;
  const int col = strip * COLS + (lane % LPR) * VN;
  const bool col_ok = col < N;                      // N is a multiple of VN
  const int kb = min(K, rank * kper), ke = min(K, kb + kper);
  float acc[R][VN];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < VN; ++j) acc[r][j] = 0.f;
  for (int k0 = kb; k0 < ke; k0 += kRowsSlab) {
    const int len = min(kRowsSlab, ke - k0);
    __syncthreads();   // the last slab has been read
    for (int i = tid; i < R * kRowsSlab; i += kRowsThreads) {
      const int r = i / kRowsSlab, kk = i % kRowsSlab;
      if (kk < len) s_x[kk * R + r] = row0 + r < rows ? to_f32(X[(size_t)(row0 + r) * K + k0 + kk]) : 0.f;
    }
    __syncthreads();
    if (col_ok) {
      for (int kk = grp; kk < len; kk += KP * U) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          w[u] = make_uint4(0, 0, 0, 0);
          if (kk + u * KP < len)
            w[u] = __ldg(reinterpret_cast<const uint4*>(W + (size_t)(k0 + kk + u * KP) * N + col));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (kk + u * KP >= len) break;
          float f[VN];
          unpack16(w[u], f, T());
          const float* x = s_x + (kk + u * KP) * R;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float xr = x[r];
#pragma unroll
            for (int j = 0; j < VN; ++j) acc[r][j] = fmaf(xr, f[j], acc[r][j]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < VN; ++j)
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) acc[r][j] += __shfl_xor_sync(0xffffffffu, acc[r][j], o);
  if (lane < LPR)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VN; ++j) s_red[warp][r * COLS + lane * VN + j] = acc[r][j];
  __syncthreads();
  for (int o = tid; o < R * COLS; o += kRowsThreads) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kRowsThreads / 32; ++w) s += s_red[w][o];
    s_out[o] = s;
  }
  cluster.sync();
  const int share = R * COLS / S;
  for (int i = tid; i < share; i += kRowsThreads) {
    const int o = rank * share + i, r = o / COLS, n = strip * COLS + o % COLS;
    float s = 0.f;
    for (int q = 0; q < S; ++q) s += *cluster.map_shared_rank(s_out + o, q);
    if (row0 + r < rows && n < N) {
      const int64_t at = (int64_t)(row0 + r) * N + n;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      const int w = (int)(at & 3);
      float x = ep.bias ? s + to_f32(ep.bias[n]) : s;
      if (ep.P) ep.P[at] = from_f32<T>(x);
      act_all<1, kFast<T>>(&x, ep.act);
      if (ep.drop.rng) {
        v[w] = x;
        drop_n<4>(v, drop_key(ep.drop), ep.drop, (uint64_t)at >> 2);
        x = v[w];
      }
      if (ep.R) x += to_f32(ep.R[at]);
      ep.Y[at] = from_f32<T>(x);
    }
  }
  cluster.sync();   // no CTA leaves while another reads its sums
}

// ------------------------------------------------------------------ fp32 as three bf16 planes
// x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1); both differences are exact in fp32. Where x is
// not finite (or rounds to infinity) x1 = x2 = 0. The smallest bf16 is 2^-133: below 2^-109 x2 has fewer
// bits, below 2^-117 x1 too.
__device__ __forceinline__ void split3(float x, float* p) {
  p[0] = __bfloat162float(__float2bfloat16_rn(x));
  const float r = fabsf(p[0]) <= 3.4e38f ? x - p[0] : 0.f;
  p[1] = __bfloat162float(__float2bfloat16_rn(r));
  p[2] = r - p[1];
}
// Four neighbours' planes, `plane` elements apart; dst 8-byte aligned.
__device__ __forceinline__ void store_planes(bf16* dst, int64_t plane, const float* x) {
  float p[4][3];
#pragma unroll
  for (int j = 0; j < 4; ++j) split3(x[j], p[j]);
#pragma unroll
  for (int i = 0; i < 3; ++i)
    *reinterpret_cast<uint2*>(dst + i * plane) =
        make_uint2(pack_bf16x2(p[0][i], p[1][i]), pack_bf16x2(p[2][i], p[3][i]));
}

// The share of `cta` of `ctas` CTAs of 256 threads.
__device__ __forceinline__ void planes_of(const PlaneJob& j, int cta, int ctas) {
  const int nv = j.cols / 4, ld = (j.cols + 7) / 8 * 8;
  const int64_t n = (int64_t)j.rows * nv, plane = (int64_t)j.rows * ld;
  for (int64_t i = (int64_t)cta * 256 + threadIdx.x; i < n; i += (int64_t)ctas * 256) {
    const int64_t row = n < (int64_t)1 << 31 ? (int64_t)((uint32_t)i / (uint32_t)nv) : i / nv;
    const float4 v = __ldg(reinterpret_cast<const float4*>(j.src) + i);
    const float x[4] = {v.x, v.y, v.z, v.w};
    store_planes(j.dst + row * ld + 4 * (i - row * nv), plane, x);
  }
}
__global__ void __launch_bounds__(256) linear_planes_kernel(PlaneJobs jobs) {
  pdl_begin(jobs.a.src, jobs.b.src);
  planes_of(blockIdx.y ? jobs.b : jobs.a, blockIdx.x, gridDim.x);
}

// ------------------------------------------------------------------ gradient of the pre-activation
// dP = drop(dY) act'(P), written where asked for (fp32: as planes), and db, its column sums before dP is
// rounded. A CTA takes 32 vectors of columns and `rper` rows, a warp every eighth row of them; its sums go
// to colsum [row_blocks][N], and the last CTA of a strip of columns to finish adds up the strip's, in the
// order of the row blocks. P NULL: no activation; db NULL: no sums. Bounded by memory: 8192 x 8192 with
// gelu, 403 MB, 67 us (0.89 of a plain copy); 32768 x 2048 with dropout and no activation, 268 MB, 64 us,
// where the draws' instructions bound it (alone, without the sums, they take 51). fp32: the CTAs from row
// `row_blocks` of the grid on write the planes of X and W in the same launch.
constexpr int kDpreWarps = 8;
template <typename T, bool ACT, bool DROP>
__global__ void __launch_bounds__(kDpreWarps * 32, 3)
linear_dpre_kernel(const T* __restrict__ dY, const T* __restrict__ P, bf16* __restrict__ dP,
                   float* colsum, T* __restrict__ db, unsigned* ticket, int act, DropArgs drop, int rows,
                   int N, int rper, int row_blocks, PlaneJobs jobs) {
  pdl_begin(dY, P, drop.rng, jobs.a.src, jobs.b.src);
  if constexpr (sizeof(T) == 4)
    if ((int)blockIdx.y >= row_blocks) {
      const int cta = (int)((blockIdx.y - row_blocks) * gridDim.x + blockIdx.x);
      const int ctas = (int)((gridDim.y - row_blocks) * gridDim.x);
      planes_of(jobs.a, cta, ctas);
      if (jobs.b.src) planes_of(jobs.b, cta, ctas);
      return;
    }
  constexpr int VN = Vec16<T>::n, U = 4, COLS = 32 * VN;
  __shared__ float s_sum[kDpreWarps][COLS];
  __shared__ bool s_last;
  DropKey key{};
  if (DROP) key = drop_key(drop);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n = ((int)blockIdx.x * 32 + lane) * VN;
  const bool ok = n < N;                             // N is a multiple of VN
  const int r0 = (int)blockIdx.y * rper, r1 = min(rows, r0 + rper);
  const int ldp = (N + 7) / 8 * 8;                   // of the planes
  float sum[VN];
#pragma unroll
  for (int j = 0; j < VN; ++j) sum[j] = 0.f;
  if (ok)
    for (int r = r0 + warp; r < r1; r += kDpreWarps * U) {
      uint4 y[U], x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = r + u * kDpreWarps;
        if (ru < r1) {
          const int64_t at = (int64_t)ru * N + n;
          y[u] = __ldg(reinterpret_cast<const uint4*>(dY + at));
          if (ACT) x[u] = __ldg(reinterpret_cast<const uint4*>(P + at));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = r + u * kDpreWarps;
        if (ru >= r1) break;
        const int64_t at = (int64_t)ru * N + n;
        float g[VN], f[VN];
        unpack16(y[u], g, T());
        if (DROP) drop_n<VN>(g, key, drop, (uint64_t)at >> 2);
        if (ACT) {
          unpack16(x[u], f, T());
          act_grad_all<VN, kFast<T>>(g, f, act);
        }
        if (dP) {
          if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint4*>(dP + at) = pack16(g, T());
          else
            store_planes(dP + (int64_t)ru * ldp + n, (int64_t)rows * ldp, g);
        }
#pragma unroll
        for (int j = 0; j < VN; ++j) sum[j] += g[j];
      }
    }
  if (!db) return;
#pragma unroll
  for (int j = 0; j < VN; ++j) s_sum[warp][lane * VN + j] = sum[j];
  __syncthreads();
  const int c0 = (int)blockIdx.x * COLS;
  for (int i = tid; i < COLS; i += kDpreWarps * 32) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kDpreWarps; ++w) s += s_sum[w][i];
    if (c0 + i < N) colsum[(int64_t)blockIdx.y * N + c0 + i] = s;
  }
  if (!last_of(ticket + blockIdx.x, row_blocks, &s_last)) return;
  // COLS / 4 threads to a row block's sums, the row blocks dealt out over the rest of them
  constexpr int QC = COLS / 4, G = kDpreWarps * 32 / QC;
  const int q = tid % QC, grp = tid / QC, c = c0 + 4 * q;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < N)
    for (int b = grp; b < row_blocks; b += 8 * G) {
      float4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        x[u] = b + u * G < row_blocks
                   ? __ldcg(reinterpret_cast<const float4*>(colsum + (int64_t)(b + u * G) * N + c))
                   : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int u = 0; u < 8; ++u) s[0] += x[u].x, s[1] += x[u].y, s[2] += x[u].z, s[3] += x[u].w;
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) s_sum[grp][4 * q + j] = s[j];
  __syncthreads();
  for (int i = tid; i < COLS; i += kDpreWarps * 32) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) t += s_sum[w][i];
    if (c0 + i < N) db[c0 + i] = from_f32<T>(t);
  }
}

template <typename T, int R>
cudaError_t rows_go(const T* X, const T* W, const LinearEpi<T>& ep, int rows, int K, int N,
                    LaunchStream st) {
  const int strips = (N + kRowsCols - 1) / kRowsCols;
  // blocks of K: up to 8 (a portable cluster), of 64 rows at least, until four CTAs stand on every SM
  int S = 1;
  while (S < 8 && strips * S * 2 <= 4 * kSms && K / (S * 2) >= 64) S *= 2;
  const int kper = (K + S - 1) / S;
  return launch_kernel(linear_rows_kernel<T, R>, dim3(strips * S, (rows + R - 1) / R), kRowsThreads, 0,
                       st, S, X, W, ep, rows, K, N, kper);
}

}  // namespace

template <typename T>
cudaError_t launch_linear_rows(const T* X, const T* W, const LinearEpi<T>& ep, int rows, int K, int N,
                               LaunchStream st) {
  if constexpr (sizeof(T) == 4) {
    if (rows > 4) return rows_go<T, 8>(X, W, ep, rows, K, N, st);
    if (rows > 2) return rows_go<T, 4>(X, W, ep, rows, K, N, st);
    if (rows > 1) return rows_go<T, 2>(X, W, ep, rows, K, N, st);
  }
  return rows_go<T, 1>(X, W, ep, rows, K, N, st);
}

static unsigned planes_grid(const PlaneJobs& j) {
  const int64_t n = std::max((int64_t)j.a.rows * j.a.cols, j.b.src ? (int64_t)j.b.rows * j.b.cols : 0) / 4;
  return (unsigned)std::min<int64_t>((n + 255) / 256, (int64_t)kSms * 16);
}
cudaError_t launch_linear_planes(const PlaneJobs& jobs, LaunchStream st) {
  return launch_kernel(linear_planes_kernel, dim3(planes_grid(jobs), jobs.b.src ? 2 : 1), 256, 0, st, 1,
                       jobs);
}

// Row blocks of the pre-activation gradient: three CTAs to an SM over the strips of columns, of eight rows
// at least (one to a warp).
static int dpre_most(int strips) { return std::max(1, 3 * kSms / strips); }
static int dpre_rows(int rows, int strips) {
  const int most = dpre_most(strips);
  return std::max(8, ((rows + most - 1) / most + 7) / 8 * 8);
}
static int dpre_strips(int N, int es) { return (N * es + 511) / 512; }
LinearDpreSize linear_dpre_size(int rows, int N, int es) {
  // a call with fewer rows may have more row blocks, whose height is rounded: bounds for all of them
  const int strips = dpre_strips(N, es);
  return {(size_t)std::min((rows + 7) / 8, dpre_most(strips)) * N, strips};
}

template <typename T>
cudaError_t launch_linear_dpre(const T* dY, const T* P, bf16* dP, float* colsum, unsigned* ticket, T* db,
                               int act, const DropArgs& drop, int rows, int N, const PlaneJobs& jobs,
                               LaunchStream st) {
  const int strips = dpre_strips(N, sizeof(T)), per = dpre_rows(rows, strips);
  const int blocks = (rows + per - 1) / per;
  const int more = jobs.a.src ? ((int)planes_grid(jobs) + strips - 1) / strips : 0;
  auto go = [&](auto kern) {
    return launch_kernel(kern, dim3(strips, blocks + more), kDpreWarps * 32, 0, st, 1, dY, P, dP, colsum,
                         db, ticket, act, drop, rows, N, per, blocks, jobs);
  };
  if (P) return drop.rng ? go(linear_dpre_kernel<T, true, true>) : go(linear_dpre_kernel<T, true, false>);
  return drop.rng ? go(linear_dpre_kernel<T, false, true>) : go(linear_dpre_kernel<T, false, false>);
}

#define LINEAR_INST(T)                                                                             \
  template cudaError_t launch_linear_rows<T>(const T*, const T*, const LinearEpi<T>&, int, int, int, \
                                             LaunchStream);                                        \
  template cudaError_t launch_linear_dpre<T>(const T*, const T*, bf16*, float*, unsigned*, T*, int,   \
                                             const DropArgs&, int, int, const PlaneJobs&,           \
                                             LaunchStream);
LINEAR_INST(float)
LINEAR_INST(bf16)

}  // namespace ecmoe
