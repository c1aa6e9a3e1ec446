// Dense products of few output tiles: one tile to a cluster, the cluster's CTAs (or CTA pairs) taking
// blocks of the summed dimension K.
//
// The persistent GEMM keeps one CTA on an SM and hides a tile's epilogue behind the next tile's main loop;
// with fewer tiles than SMs there is no next tile and most SMs idle. Here the S blocks of K of a tile run
// at the same time on S CTAs (pairs), each CTA leaves its fp32 sums in its shared memory, and after a
// cluster barrier each adds up its share of the tile over the others' shared memory, in the order of the
// blocks, and finishes it: the epilogue of the whole product in one launch, with no partial sum in global
// memory. The shares are read and written along rows, so bias, residual and outputs are whole lines.
//
// Bounded by what an SM takes in from L2 and by the launch: 256 rows, K 2048, N 8192 with gelu 11.6 us
// (33.5 MB of weights, 100 MB out of L2), 24 rows of 2048 x 2048 6.0 us; the persistent kernel takes 15.3
// and 14.8.
//
// fp32 operands come as three bf16 planes each (linear.cu): a k-slice is then three slices of A and of B,
// of which six products are added, the smallest first; see kPlaneA. 4096 x 1024 x 1024 48 us with its planes
// (179 TFLOP/s of fp32, 1.07 PFLOP/s of bf16), 1000 x 1000 x 1000 19.5 us; with a plane's slice loaded for
// each of the products 69 and 30 us, by what an SM takes in.
#pragma once
#include <type_traits>

#include "gemm_tc_kernel.cuh"
#include "kernels.h"
#include "linear_tile.h"

namespace ecmoe {
namespace {

constexpr int kTileThreads = 256;

// The plane of A and of B in product s of a k-slice, smallest products first. x = x0 + x1 + x2 + r with
// |x1| <= 2^-8 |x|, |x2| <= 2^-16 |x| and |r| <= 2^-24 |x| (each plane is rounded to nearest); what is
// left out (x1 y2, x2 y1, x2 y2 and the remainders' products) is at most 2^-22 |x y|, four times an fp32
// product's rounding, and as a random sum well below that of the fp32 sums.
__device__ constexpr int kPlaneA[6] = {1, 0, 2, 0, 1, 0};
__device__ constexpr int kPlaneB[6] = {1, 2, 0, 1, 0, 0};

struct TileArgs {
  int M, N, blocks, splits, n_tiles;         // blocks: k-slices
  int stages, a_rows;                        // of the operand ring; rows of A in a stage
  bool beside;                               // TileProblem::beside
  int* status;
};

// W columns of a row, four or eight (eight fp32 ones: the second four behind `more`, for rows end after
// any multiple of four).
template <int W>
__device__ __forceinline__ void tile_load(const bf16* p, float* f, bool) {
  if constexpr (W == 8) {
    unpack16(__ldg(reinterpret_cast<const uint4*>(p)), f, bf16());
  } else {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
    f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xFFFF0000u);
    f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xFFFF0000u);
  }
}
template <int W>
__device__ __forceinline__ void tile_load(const float* p, float* f, bool more) {
  unpack16(__ldg(reinterpret_cast<const uint4*>(p)), f, 0.f);
  if (W == 8 && more) unpack16(__ldg(reinterpret_cast<const uint4*>(p) + 1), f + 4, 0.f);
}
template <int W>
__device__ __forceinline__ void tile_store(bf16* p, const float* f, bool) {
  if constexpr (W == 8)
    *reinterpret_cast<uint4*>(p) = pack16(f, bf16());
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
}
template <int W>
__device__ __forceinline__ void tile_store(float* p, const float* f, bool more) {
  *reinterpret_cast<uint4*>(p) = pack16(f, 0.f);
  if (W == 8 && more) *(reinterpret_cast<uint4*>(p) + 1) = pack16(f + 4, 0.f);
}
// P, Y of W columns at element `at` of the output from their sums f, bias b and residual res.
template <int W, typename T>
__device__ __forceinline__ void tile_finish(const LinearEpi<T>& ep, const DropKey& key, int64_t at,
                                            float* f, const float* b, const float* res, bool more) {
#pragma unroll
  for (int j = 0; j < W; ++j) f[j] += b[j];
  if (ep.P) tile_store<W>(ep.P + at, f, more);
  act_all<W, sizeof(T) == 2>(f, ep.act);
  if (ep.drop.rng)
#pragma unroll
    for (int h = 0; h < W / 4; ++h) drop_n<4>(f + 4 * h, key, ep.drop, ((uint64_t)at >> 2) + h);
  if (ep.R)
#pragma unroll
    for (int j = 0; j < W; ++j) f[j] += res[j];
  tile_store<W>(ep.Y + at, f, more);
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr));
  return v;
}

// The tensor cores add in fp32 but cut off what does not fit, so a long sum of one sign drifts: up to 1e-7 of
// its size for every 16 of K (2e-5 at K 8192, 1.7e-4 at 32768, 1.6e-3 at 262144). With SUMS an accumulator therefore takes few k-slices and
// is then added to sums in registers, rounded to nearest, by eight warps of their own, while the MMAs go
// on in a second accumulator:
// - fp32 results, always: one k-slice, in which only the last four steps add numbers of the sum's size.
//   Against 64 bits 1e-7 at K 1000, where the product of fp32 numbers, added one by one, has 5.7e-7. Above
//   kBlockSlices k-slices (SUMS 2) the register sums of so many are added up on a second level, so that
//   neither chain is long: 1e-7 to 2.4e-7 of a sum of one sign from K 1000 to 524288 (one chain of 32768
//   slices: 1.3e-6).
// - bf16 results, where an accumulator would take more than kLongSlices (both in linear_tile.h): kLongRun
//   k-slices, a drift of 2.6e-5 at most, a hundredth of half a bf16 step.
constexpr int kLongRun = 64;
template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
template <int SUMS>
constexpr int kTileBlock = kTileThreads + (SUMS ? 64 : 0);

template <int BN, bool A_MN, bool B_MN, bool PAIR, typename T, int SUMS>
__global__ void __launch_bounds__(kTileBlock<SUMS>, SUMS ? 1 : 2)
linear_tile_kernel(const __grid_constant__ CUtensorMap mA, const __grid_constant__ CUtensorMap mB,
                   LinearEpi<T> ep, TileArgs p) {
  constexpr int BNL = PAIR ? BN / 2 : BN;        // columns of B in this CTA's shared memory
  constexpr int NP = PAIR ? 2 : 1;
  constexpr int PL = kPlanes<T>;                 // of an operand
  constexpr int RUN = PL == 3 ? 1 : kLongRun;    // SUMS: k-slices an accumulator takes
  constexpr uint32_t B_BYTES = BNL * BK * 2;     // of one plane's slice
  const uint32_t a_bytes = (uint32_t)p.a_rows * BK * 2;
  constexpr uint32_t IDESC = instr_desc<BN, A_MN, B_MN, NP * BM>();
  constexpr int FIRST = SUMS ? 2 : 0;            // the first warp of the eight that finish the tile
  constexpr uint32_t TCOLS = SUMS ? 2 * BN : BN;
  extern __shared__ uint8_t smem_raw[];
  // barriers first, the ring (a multiple of 1024 bytes from its start on) behind them
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* smem = base + 1024;
  uint8_t* sA = smem;
  uint8_t* sB = smem + p.stages * PL * a_bytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(base);
  uint64_t* empty = full + kTileMaxStages;
  uint64_t* done = empty + kTileMaxStages;
  uint64_t* tfull = done + 1;    // SUMS: the two accumulators, full and free
  uint64_t* tempty = tfull + 2;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(tempty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // known to be one value for the warp
  const uint32_t rank = cluster_ctarank();
  const int half = PAIR ? (int)(rank & 1u) : 0, split = (int)rank / NP;
  const bool leader = half == 0;                 // of the pair: issues its MMAs
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(done, 1);
    for (int a = 0; SUMS && a < 2; ++a) {
      mbar_init(&tfull[a], 1);
      mbar_init(&tempty[a], NP * 8);
    }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_map(&mA);
    prefetch_map(&mB);
  }
  if (warp == 1) {
    if constexpr (PAIR) tmem_alloc_pair(tmem_holder, TCOLS);
    else tmem_alloc(tmem_holder, TCOLS);
  }
  tc_fence_before();
  __syncthreads();
  const bool alone = NP * p.splits == 1;   // no cluster
  if (!alone) cluster_sync();   // the peers' barriers are initialised before use
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  if (!p.beside) pdl_begin(ep.bias, ep.R, ep.drop.rng);

  const int tile = (int)blockIdx.x / (NP * p.splits);
  const int mt = tile / p.n_tiles, nt = tile - mt * p.n_tiles;
  const int row0 = mt * NP * BM + half * BM, n0 = nt * BN;
  const int kb0 = (int)((int64_t)p.blocks * split / p.splits);
  const int kb1 = (int)((int64_t)p.blocks * (split + 1) / p.splits);
  // every finishing warp reads a lane quarter of the accumulator, two warps to a quarter
  const int q = warp & 3, r = q * 32 + lane, part2 = (warp - FIRST) >> 2;
  float sum[SUMS ? BN / 64 : 1][32];
  if (warp == 0) {
    const bool one = elect_one();
    int s = 0;
    uint32_t ph = 0;
    const int nb = n0 + half * BNL;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(&empty[s], ph ^ 1u, abort_flag, p.status)) { ok = false; break; }
      const int k0 = kb * BK;
      uint8_t* a = sA + s * PL * a_bytes;
      uint8_t* b = sB + s * PL * B_BYTES;
      // completion goes to the pair's leader: it gates the pair's MMAs
      const uint32_t fb = PAIR ? mapa_shared(smem_u32(&full[s]), rank & ~1u) : 0u;
      if (one) {
        if (leader) mbar_arrive_expect_tx(&full[s], (a_bytes + B_BYTES) * PL * NP);
        auto load = [&](void* dst, const CUtensorMap* m, int c0, int c1, int plane) {
          if constexpr (PAIR) tma_load_3d_pair(dst, m, fb, c0, c1, plane);
          else tma_load_3d(dst, m, &full[s], c0, c1, plane);
        };
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) {
          if constexpr (!A_MN) {
            load(a, &mA, k0, row0, pl);
          } else {
#pragma unroll
            for (int j = 0; j < BM / 64; ++j) load(a + j * 8192, &mA, row0 + 64 * j, k0, pl);
          }
          if constexpr (!B_MN) {
            load(b, &mB, k0, nb, pl);
          } else {
#pragma unroll
            for (int j = 0; j < BNL / 64; ++j) load(b + j * 8192, &mB, nb + 64 * j, k0, pl);
          }
          a += a_bytes;
          b += B_BYTES;
        }
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; ph ^= 1u; }
    }
    if (!ok) {
      // let copies already issued land before the CTA leaves
      const unsigned long long t = globaltimer();
      while (globaltimer() - t < 1000000ull) {}
    }
    __syncwarp();
  } else if (warp == 1) {
    if (leader) {
      const bool one = elect_one();
      const uint16_t mask = PAIR ? (uint16_t)(0x3u << (rank & ~1u)) : (uint16_t)0;
      auto commit = [&](uint64_t* bar) {
        if constexpr (PAIR) mma_commit_pair(bar, mask);
        else mma_commit(bar);
      };
      const uint32_t da0 = desc_lo(smem_u32(sA), A_MN ? 8192 : 16);
      const uint32_t db0 = desc_lo(smem_u32(sB), B_MN ? 8192 : 16);
      int s = 0;
      uint32_t ph = 0;
      // the MMAs of ring slot s into accumulator d, which starts from zero where acc is 0
      auto issue = [&](uint32_t d, uint32_t acc) {
        const uint32_t a0 = da0 + s * PL * (a_bytes >> 4), b0 = db0 + s * PL * (B_BYTES >> 4);
#pragma unroll
        for (int g = 0; g < (PL == 3 ? 6 : 1); ++g) {
          const uint32_t ag = PL == 3 ? a0 + kPlaneA[g] * (a_bytes >> 4) : a0;
          const uint32_t bg = PL == 3 ? b0 + kPlaneB[g] * (B_BYTES >> 4) : b0;
#pragma unroll
          for (int j = 0; j < BK / 16; ++j) {
            const uint32_t ad = ag + j * (A_MN ? 2048 >> 4 : 32 >> 4);
            const uint32_t bd = bg + j * (B_MN ? 2048 >> 4 : 32 >> 4);
            const uint32_t on = g + j == 0 ? acc : 1u;
            if constexpr (PAIR) mma_bf16_pair(d, ad, bd, IDESC, on);
            else mma_bf16(d, ad, bd, IDESC, on);
          }
        }
        commit(&empty[s]);
      };
      if constexpr (SUMS == 0 || RUN == 1) {
        int a = 0;   // SUMS: the accumulator of the slice
        uint32_t acc = 0, free_ph = 1;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (SUMS && !mbar_wait_warp(&tempty[a], free_ph, abort_flag, p.status)) break;
          if (!mbar_wait_warp(&full[s], ph, abort_flag, p.status)) break;
          tc_fence_after();
          if (one) {
            issue(tmem + (SUMS ? a * BN : 0), SUMS ? 0u : acc);
            if (SUMS) commit(&tfull[a]);
          }
          __syncwarp();
          acc = 1;
          if (SUMS && (a ^= 1) == 0) free_ph ^= 1u;
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
      } else {
        // a loop over the slices of an accumulator as short as the one without register sums: with the
        // accumulator changing inside it a slice of 128 x 64 tiles took 0.226 us, so 0.172, as without
        bool good = true;
        for (int kb = kb0, c = 0; kb < kb1 && good; ++c) {
          const int end = min(kb + RUN, kb1);
          good = mbar_wait_warp(&tempty[c & 1], (uint32_t)(c >> 1 & 1) ^ 1u, abort_flag, p.status);
          const uint32_t d = tmem + (c & 1) * BN;
          uint32_t acc = 0;
          for (; kb < end && good; ++kb) {
            if (!mbar_wait_warp(&full[s], ph, abort_flag, p.status)) { good = false; break; }
            tc_fence_after();
            if (one) issue(d, acc);
            __syncwarp();
            acc = 1;
            if (++s == p.stages) { s = 0; ph ^= 1u; }
          }
          if (one) commit(&tfull[c & 1]);
          __syncwarp();
        }
      }
      // also where the loop gave up: the MMAs already issued end before TMEM is released
      if (one) commit(done);
      __syncwarp();
    }
    // the other warps wait at the barrier below, where they take no issue slots from the two at work
    mbar_wait_warp(done, 0, abort_flag, p.status);
  } else if constexpr (SUMS != 0) {
    float blocks[SUMS == 2 ? BN / 64 : 1][32];   // SUMS 2: what is closed of the sum
    auto close_block = [&] {
#pragma unroll
      for (int i = 0; i < BN / 64; ++i)
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          blocks[i][j] += sum[i][j];
          sum[i][j] = 0.f;
        }
    };
#pragma unroll
    for (int i = 0; i < BN / 64; ++i)
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        sum[i][j] = 0.f;
        if (SUMS == 2) blocks[i][j] = 0.f;
      }
    const int runs = (kb1 - kb0 + RUN - 1) / RUN;
    for (int c = 0; c < runs; ++c) {
      const int a = c & 1;
      if (!mbar_wait_warp(&tfull[a], (uint32_t)(c >> 1) & 1u, abort_flag, p.status)) break;
      tc_fence_after();
#pragma unroll
      for (int i = 0; i < BN / 64; ++i) {
        uint32_t v[32];
        tmem_ld32(tmem + (uint32_t)(a * BN + part2 * (BN / 2) + 32 * i) + ((uint32_t)(q * 32) << 16), v);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[i][j] += f32(v[j]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&tempty[a]), rank & ~(uint32_t)(NP - 1)));
      if constexpr (SUMS == 2)
        if (c % kBlockSlices == kBlockSlices - 1) close_block();
    }
    if constexpr (SUMS == 2) {
      close_block();
#pragma unroll
      for (int i = 0; i < BN / 64; ++i)
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[i][j] = blocks[i][j];
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const bool ok = *abort_flag == 0;
  const int valid = min(BM, p.M - row0);                 // rows of this CTA, <= 0 past the last
  float* part = reinterpret_cast<float*>(smem);
  const uint32_t part_addr = smem_u32(part);
  DropKey key{};
  if (ep.drop.rng) key = drop_key(ep.drop);
  const int rows = max(valid, 0);
  // this CTA's sums, 16-byte units of a row swizzled by the row so that a warp's stores spread
  if (!SUMS || warp >= FIRST) {
#pragma unroll
    for (int i = 0; i < BN / 64; ++i) {
      const int c = part2 * (BN / 2) + 32 * i;
      if constexpr (!SUMS) {
        uint32_t v[32];
        tmem_ld32(tmem + (uint32_t)c + ((uint32_t)(q * 32) << 16), v);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[0][j] = f32(v[j]);
      }
      const float* v = sum[SUMS ? i : 0];
      if (r < valid)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<float4*>(part + r * BN + (((c / 4 + j) ^ (r & 7)) << 2)) =
              make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
  }
  if (p.splits > 1) cluster_sync();
  else __syncthreads();
  const int ft = tid - 32 * FIRST;
  if (ft < 0) {
    // the two warps of the main loop rest
  } else if (p.splits == 1) {
    // a thread keeps eight columns and has several rows in flight
    constexpr int UNITS = BN / 8, ROWS = kTileThreads / UNITS, U = PAIR ? 2 : 4;
    const int unit = ft % UNITS, n = n0 + 8 * unit;
    const bool more = n + 4 < p.N;
    float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (ep.bias && n < p.N) tile_load<8>(ep.bias + n, b, more);
    for (int row = ft / UNITS; row < rows && n < p.N && ok; row += ROWS * U) {
      float f[U][8], res[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = min(row + u * ROWS, rows - 1);
        if (ep.R) tile_load<8>(ep.R + (int64_t)(row0 + ru) * p.N + n, res[u], more);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          unpack16(*reinterpret_cast<const uint4*>(part + ru * BN +
                                                   (((2 * unit + h) ^ (ru & 7)) << 2)),
                   f[u] + 4 * h, 0.f);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (row + u * ROWS >= rows) break;
        tile_finish<8>(ep, key, (int64_t)(row0 + row + u * ROWS) * p.N + n, f[u], b, res[u], more);
      }
    }
  } else {
    // this CTA's share of the rows: a thread keeps four columns, and has the sums of all S blocks of
    // 8 / S rows in flight, which it adds in the order of the blocks
    constexpr int UNITS = BN / 4, ROWS = kTileThreads / UNITS;
    const int unit = ft % UNITS, n = n0 + 4 * unit;
    const int r1 = rows * (split + 1) / p.splits;
    float b[4] = {0.f, 0.f, 0.f, 0.f};
    if (ep.bias && n < p.N) tile_load<4>(ep.bias + n, b, false);
    auto join = [&](auto blocks) {
      constexpr int S = decltype(blocks)::value, U = std::max((PAIR ? 4 : 8) / S, 1);
      for (int row = rows * split / S + ft / UNITS; row < r1; row += ROWS * U) {
        float4 x[U][S];
        float res[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int ru = row + u * ROWS;
          if (ru >= r1) break;
          if (ep.R) tile_load<4>(ep.R + (int64_t)(row0 + ru) * p.N + n, res[u], false);
          const uint32_t off = part_addr + (uint32_t)(ru * BN + ((unit ^ (ru & 7)) << 2)) * 4u;
#pragma unroll
          for (int s = 0; s < S; ++s)
            x[u][s] = ld_cluster4(mapa_shared(off, (uint32_t)(s * NP + half)));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int ru = row + u * ROWS;
          if (ru >= r1) break;
          float f[4] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w};
#pragma unroll
          for (int s = 1; s < S; ++s)
            f[0] += x[u][s].x, f[1] += x[u][s].y, f[2] += x[u][s].z, f[3] += x[u][s].w;
          tile_finish<4>(ep, key, (int64_t)(row0 + ru) * p.N + n, f, b, res[u], false);
        }
      }
    };
    if (n < p.N && ok) {
      if (p.splits == 2) join(std::integral_constant<int, 2>());
      else if (PAIR || p.splits == 4) join(std::integral_constant<int, 4>());
      else join(std::integral_constant<int, 8>());
    }
  }
  tc_fence_before();
  // the other CTAs have read this one's sums, and the pair's other half has left its TMEM
  if (alone) __syncthreads();
  else cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem, TCOLS);
    else tmem_dealloc(tmem, TCOLS);
  }
  // the kernel before ends before this one does, so what comes after waits for both
  if (p.beside) pdl_begin();
}

// Operand maps: A [planes][M][K] (A_MN: [planes][K][M]), B [planes][N][K] (B_MN: [planes][K][N]), rows
// `lda`, `ldb` elements apart.
cudaError_t tile_map(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t ld,
                     uint64_t planes, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return cudaErrorNotSupported;
  cuuint64_t dims[3] = {cols, rows, planes};
  cuuint64_t strides[2] = {ld * 2, ld * rows * 2};
  cuuint32_t box[3] = {64, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
                  estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int BN, bool A_MN, bool B_MN, bool PAIR, int SUMS, typename T>
cudaError_t tile_go(const TileProblem<T>& t, const TileChoice& c, LaunchStream st) {
  auto kern = linear_tile_kernel<BN, A_MN, B_MN, PAIR, T, SUMS>;
  constexpr int PL = kPlanes<T>;
  const int a_rows = tile_a_rows(c.form, !A_MN, t.M), stage = tile_stage(c.form, PL, a_rows);
  static PerDevice once;
  int set = 0;
  TC_TRY(once.get(&set, [&](int* v) {
    *v = 1;
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                kTileDeep + kTileExtra);
  }));
  CUtensorMap ma, mb;
  TC_TRY(A_MN ? tile_map(&ma, t.A, t.M, t.K, t.lda, PL, 64)
              : tile_map(&ma, t.A, t.K, t.M, t.lda, PL, a_rows));
  TC_TRY(B_MN ? tile_map(&mb, t.B, t.N, t.K, t.ldb, PL, 64)
              : tile_map(&mb, t.B, t.K, t.N, t.ldb, PL, PAIR ? BN / 2 : BN));
  TileArgs p;
  p.M = t.M; p.N = t.N;
  p.blocks = (t.K + BK - 1) / BK;
  p.splits = c.splits;
  p.n_tiles = (t.N + BN - 1) / BN;
  p.status = t.status;
  const int rows = PAIR ? 2 * BM : BM, cluster = c.splits * (PAIR ? 2 : 1);
  const int64_t ctas = (int64_t)((t.M + rows - 1) / rows) * p.n_tiles * cluster;
  p.stages = tile_ring(stage, SUMS || tile_deep(ctas, cluster));
  p.a_rows = a_rows;
  p.beside = t.beside;
  // the ring holds the sums afterwards, and the MMA's reads past the last rows of A end inside it
  const int sums = std::min(t.M, BM) * BN * 4;
  const int ring = std::max({p.stages * stage, sums, (p.stages * PL - 1) * a_rows * 128 + BM * 128});
  return launch_kernel(kern, (unsigned)ctas, kTileBlock<SUMS>, (size_t)ring + kTileExtra, st, cluster, ma,
                       mb, t.ep, p);
}

// The last form of kTileForms is for long sums of bf16 products alone.
template <bool A_MN, bool B_MN, int SUMS, typename T>
cudaError_t tile_form(const TileProblem<T>& t, const TileChoice& c, LaunchStream st) {
  switch (c.form) {
    case 0: return tile_go<64, A_MN, B_MN, false, SUMS>(t, c, st);
    case 1: return tile_go<128, A_MN, B_MN, false, SUMS>(t, c, st);
    case 2: return tile_go<128, A_MN, B_MN, true, SUMS>(t, c, st);
  }
  if constexpr (sizeof(T) == 2 && SUMS) return tile_go<256, A_MN, B_MN, true, SUMS>(t, c, st);
  return cudaErrorInvalidValue;
}

template <int SUMS, typename T>
cudaError_t tile_launch(const TileProblem<T>& t, const TileChoice& c, LaunchStream st) {
  switch (t.form) {
    case LIN_FWD: return tile_form<false, true, SUMS>(t, c, st);
    case LIN_DX: return tile_form<false, false, SUMS>(t, c, st);
    case LIN_DW: return tile_form<true, true, SUMS>(t, c, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace
}  // namespace ecmoe
