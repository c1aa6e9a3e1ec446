// Balance loss of a router, its per-expert counts and the gradient of the router's logits.
//
// Over the n tokens that the mask leaves, n_g of them in sequence g (w_g = E / (k n n_g)):
//   c[g][e] = choices of expert e by those tokens of g
//   L       = sum_g w_g sum_e c[g][e] sum_{t in g} S[t][e]
//   dL/dZ[t][e] = S[t][e] (f[g][e] - sum_e' S[t][e'] f[g][e']),   f[g][e] = w_g c[g][e]
// (the softmax Jacobian on the constant row f of the token's sequence; the counts carry no gradient).
//
// The tokens are cut into chunks of one sequence each (every sequence has one, if an empty one); a CTA
// takes a chunk, the last CTA of a sequence to finish joins the sequence's sums, and the last of those
// joins the sequences'. All sums run in an order that the sizes alone fix: the only atomics add
// integers and draw tickets, which say who joins and not what is added to what.
//
// The loss is bounded by latency: a launch, a chunk's reads and the joins' after them. 65536 tokens of 128
// experts in 33 sequences, with a mask: 11.0 us for 36 MB (3.3 TB/s), 32768 x 64: 8.1 us, 256 x 8: 5.8 us.
// The gradient is bounded by memory: 11.4 us for 67 MB (5.9 TB/s, 0.87 of a plain copy), 3.9 and 1.9 us.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace ecmoe {
namespace {

constexpr int kBalThreads = 512;
static_assert(kBalanceMaxE <= kBalThreads, "a thread for every expert");

__device__ __forceinline__ int block_sum_int(int v, int* s) {
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < kBalThreads / 32; ++w) t += s[w];
  __syncthreads();
  return t;
}

template <int V>
__device__ __forceinline__ void load_v(const float* p, float* x) {
  if constexpr (V == 4) {
    const float4 q = __ldg(reinterpret_cast<const float4*>(p));
    x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
  } else {
    x[0] = __ldg(p);
  }
}

// Column sums of S over a chunk's live tokens and the counts of their choices: V columns (one 16-byte
// load) to a thread, a row of the block's threads to a token; then the joins.
template <int V, bool MASK>
__global__ void __launch_bounds__(kBalThreads, 2)
balance_kernel(BalanceArgs p) {
  pdl_begin(p.S, p.choice, p.mask, p.chunk, p.chunk_off);
  __shared__ float s_acc[kBalThreads * V];
  __shared__ int s_cnt[kBalThreads];
  __shared__ int s_warp[kBalThreads / 32];
  __shared__ bool s_last;
  const int E = p.E, tid = threadIdx.x;
  const int4 ch = __ldg(p.chunk + blockIdx.x);
  const int g = ch.x, t0 = ch.y, t1 = ch.z;
  // a thread's first token: its mask and first choices are asked for before the scores, and counted
  // after them
  constexpr int NC = 8;
  auto token = [&](int t, int r0, int* e) {   // choices r0 .. r0 + NC - 1 of token t, -1 past the last
    const int* choice = p.choice + (size_t)t * p.k;
#pragma unroll
    for (int r = 0; r < NC; ++r) e[r] = r0 + r < p.k ? __ldg(choice + r0 + r) : -1;
  };
  int pre[NC];
  bool pre_live = t0 + tid < t1;
#pragma unroll
  for (int r = 0; r < NC; ++r) pre[r] = -1;
  if (pre_live) {
    token(t0 + tid, 0, pre);
    if (MASK) pre_live = __ldg(p.mask + t0 + tid) != 0;
  }
  s_cnt[tid] = 0;

  const int ncol = E / V, rows = kBalThreads / ncol, row = tid / ncol, col = tid - row * ncol;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  if (row < rows) {
    constexpr int U = 8;
    const float* src = p.S + (size_t)col * V;
    for (int t = t0 + row; t < t1; t += rows * U) {
      // all loads of a round without a condition, the chunk's last token again past its end, so that
      // they are in flight together; a masked token's scores are left out when they are added
      float x[U][V];
      uint32_t use[U];   // all ones or 0
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int tu = min(t + u * rows, t1 - 1);
        use[u] = t + u * rows < t1 && (!MASK || __ldg(p.mask + tu) != 0) ? 0xFFFFFFFFu : 0u;
        load_v<V>(src + (size_t)tu * E, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j)
          acc[j] += __uint_as_float(__float_as_uint(x[u][j]) & use[u]);
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) s_acc[tid * V + j] = acc[j];
  __syncthreads();   // s_cnt is cleared
  // an entry outside [0, E) is no choice
  auto add = [&](const int* e) {
#pragma unroll
    for (int r = 0; r < NC; ++r)
      if ((unsigned)e[r] < (unsigned)E) atomicAdd(s_cnt + e[r], 1);
  };
  int live = 0;
  for (int t = t0 + tid; t < t1; t += kBalThreads) {
    const bool first = t == t0 + tid;
    if (first ? !pre_live : MASK && __ldg(p.mask + t) == 0) continue;
    ++live;
    int e[NC];
    if (first) add(pre);
    else token(t, 0, e), add(e);
    for (int r = NC; r < p.k; r += NC) token(t, r, e), add(e);
  }
  live = block_sum_int(live, s_warp);   // and every count is in
  float sum = 0.f;
  if (tid < E)
#pragma unroll 8
    for (int r = 0; r < rows; ++r) sum += s_acc[r * E + tid];
  __syncthreads();
  int cnt = tid < E ? s_cnt[tid] : 0;
  const int b0 = __ldg(p.chunk_off + g), b1 = __ldg(p.chunk_off + g + 1);
  if (b1 - b0 > 1) {
    if (tid < E) {
      p.part[(size_t)blockIdx.x * E + tid] = sum;
      p.pcnt[(size_t)blockIdx.x * E + tid] = cnt;
    }
    if (tid == 0) p.live[blockIdx.x] = live;
    if (!last_of(p.ticket + 1 + g, b1 - b0, &s_last)) return;
    // the sequence's sums: a row of E threads to a chunk, then the rows
    const int jr = kBalThreads / E, jrow = tid / E, e = tid - jrow * E;
    sum = 0.f;
    cnt = live = 0;
    if (jrow < jr) {
      constexpr int U = 8;
      for (int b = b0 + jrow; b < b1; b += jr * U) {
        float x[U];
        int c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int bu = b + u * jr;
          x[u] = bu < b1 ? __ldcg(p.part + (size_t)bu * E + e) : 0.f;
          c[u] = bu < b1 ? __ldcg(p.pcnt + (size_t)bu * E + e) : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          sum += x[u];
          cnt += c[u];
        }
      }
    }
    for (int b = b0 + tid; b < b1; b += kBalThreads) live += __ldcg(p.live + b);
    live = block_sum_int(live, s_warp);
    s_acc[tid] = sum;
    s_cnt[tid] = cnt;
    __syncthreads();
    if (tid < E)
#pragma unroll 4
      for (int r = 1; r < jr; ++r) {
        sum += s_acc[r * E + tid];
        cnt += s_cnt[r * E + tid];
      }
  }
  // The sequence: its counts, its row f n less the mean (which follows the row), formed from integers so
  // that the small difference of nearly equal counts is exact, its part of n L.
  if (tid >= E) sum = 0.f, cnt = 0;
  const int total = block_sum_int(cnt, s_warp);
  const float w = live > 0 ? 1.f / ((float)p.k * (float)live) : 0.f;
  float* table = p.table + (size_t)g * p.table_ld;
  if (tid < E) {
    if (p.count) p.count[(size_t)g * E + tid] = cnt;
    table[tid] = w * (float)((int64_t)E * cnt - total);
  }
  const float l = warp_sum(w * (float)E * (float)cnt * sum);
  if ((tid & 31) == 0) s_acc[tid >> 5] = l;
  __syncthreads();
  if (tid == 0) {
    float loss = 0.f;
    for (int i = 0; i < kBalThreads / 32; ++i) loss += s_acc[i];
    table[p.table_ld - 4] = w * (float)total;
    p.gloss[g] = loss;
    p.glive[g] = live;
  }
  if (!last_of(p.ticket, p.G, &s_last)) return;
  int n = 0;
  for (int i = tid; i < p.G; i += kBalThreads) n += __ldcg(p.glive + i);
  n = block_sum_int(n, s_warp);
  if (tid < 32) {
    float loss = 0.f;
    for (int i = tid; i < p.G; i += 32) loss += __ldcg(p.gloss + i);
    loss = warp_sum(loss);
    if (tid == 0) {
      const float inv = n > 0 ? 1.f / (float)n : 0.f;
      *p.inv_n = inv;
      if (p.loss) *p.loss = loss * inv;
    }
  }
}

// dZ = dloss S (f' - <S, f'> + f0 (1 - sum S)) with f' = f - f0: the row's mean is taken out first,
// so that the difference of two nearly equal numbers of f0's size is not formed from rounded ones
// (with balanced experts f' is a few percent of f0, or a few thousandths). So that f0 (1 - sum S) does not
// err by 2^-24 f0 and more, a score is added up in two parts: what it has in multiples of 2^-22, whose sum
// is exact up to 4, and the rest, which goes with the small terms (3 to 7% of the time of scores that lie
// in L2). `lanes` lanes (a power of two) to a token, NV vectors of V experts to a lane; blockIdx.y: the
// parts of the chunk, each as many tokens as the block has in flight, dealt out to as many CTAs as make
// eight to an SM (65536 x 128: with a CTA to every part 6% longer, with four to an SM 14%).
constexpr int kGradThreads = 256, kGradCtas = 8;
template <int NV>
constexpr int kGradTokens = NV <= 2 ? 4 : NV <= 4 ? 2 : 1;   // tokens a thread has in flight
template <int V, int NV, bool MASK>
__global__ void __launch_bounds__(kGradThreads, 4)
balance_grad_kernel(BalanceArgs p, const float* dloss, float* dZ, int lanes) {
  pdl_begin(p.S, p.mask, p.chunk, p.table, p.inv_n, dloss);
  const int E = p.E, tid = threadIdx.x;
  const int per = kGradThreads / lanes, j = tid & (lanes - 1);
  constexpr int U = kGradTokens<NV>;
  const int4 ch = __ldg(p.chunk + blockIdx.x);
  const float* table = p.table + (size_t)ch.x * p.table_ld;
  const float f0 = __ldg(table + p.table_ld - 4);
  const float dl = (dloss ? __ldg(dloss) : 1.f) * __ldg(p.inv_n);
  float tab[NV][V];   // this lane's columns are the same for every token; 0 past the last expert
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const int e = (j + i * lanes) * V + q;
      tab[i][q] = e < E ? __ldg(table + e) : 0.f;
    }
  // every lane of a warp goes round equally often: the sums are taken by shuffles
  const int first = ch.y + (int)blockIdx.y * per * U;
  for (int tw = first; tw < ch.z; tw += (int)gridDim.y * per * U) {
    const int tb = tw + tid / lanes;
    float s[U][NV][V];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(tb + u * per, ch.z - 1);
      live[u] = tb + u * per < ch.z && (!MASK || __ldg(p.mask + t) != 0);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (j + i * lanes) * V;
        load_v<V>(p.S + (size_t)t * E + min(e, E - V), s[u][i]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = tb + u * per;
      float sum = 3.f, rest = 0.f, dot = 0.f;   // in [2, 4) sums are multiples of 2^-22
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if ((j + i * lanes) * V < E)
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const float x = s[u][i][q], next = sum + x;
            rest += x - (next - sum);
            sum = next;
            dot = fmaf(x, tab[i][q], dot);
          }
      }
      sum -= 3.f;
      dot = fmaf(f0, rest, dot);
      for (int o = lanes >> 1; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      const float c = fmaf(f0, 1.f - sum, -dot);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (j + i * lanes) * V;
        if (t >= ch.z || e >= E) continue;
        float z[V];
        // a masked token's gradient is 0 whatever its scores hold
#pragma unroll
        for (int q = 0; q < V; ++q) z[q] = live[u] ? dl * s[u][i][q] * (tab[i][q] + c) : 0.f;
        float* dst = dZ + (size_t)t * E + e;
        if constexpr (V == 4) *reinterpret_cast<float4*>(dst) = make_float4(z[0], z[1], z[2], z[3]);
        else *dst = z[0];
      }
    }
  }
}

}  // namespace

// Tokens to a chunk: as few as leave one chunk to an SM at most over all sequences (a second one on some
// of the SMs doubled the time of a ragged batch), where there are no more sequences than SMs, and no
// fewer than the block reads in one pass, or 32: a sequence of one chunk needs no join (256 x 8 in two
// sequences 8.8 us with chunks of 32, 6.1 us with whole ones).
int balance_chunk_tokens(int N, int E, int G, const int* group_off) {
  const int rows = kBalThreads / (E % 4 == 0 ? E / 4 : E);   // tokens of a pass
  int64_t t = std::max<int64_t>(std::max(32, rows), ((int64_t)N + kSms - 1) / kSms);
  t = (t + 7) / 8 * 8;
  for (int tries = 0; tries < 64 && G <= kSms; ++tries, t = (t + t / 16 + 15) / 8 * 8) {
    int64_t chunks = 0;
    for (int g = 0; g < G; ++g)
      chunks += std::max<int64_t>(1, (group_off[g + 1] - group_off[g] + t - 1) / t);
    if (chunks <= kSms) break;
  }
  return (int)std::min<int64_t>(t, std::max(N, 32));
}

cudaError_t launch_balance_forward(const BalanceArgs& p, LaunchStream st) {
  auto go = [&](auto kern) { return launch_kernel(kern, p.chunks, kBalThreads, 0, st, 1, p); };
  if (p.E % 4 == 0) return p.mask ? go(balance_kernel<4, true>) : go(balance_kernel<4, false>);
  return p.mask ? go(balance_kernel<1, true>) : go(balance_kernel<1, false>);
}

template <int V, int NV>
static cudaError_t grad_go(const BalanceArgs& p, const float* dloss, float* dZ, int lanes,
                           LaunchStream st) {
  const int tokens = kGradThreads / lanes * kGradTokens<NV>;
  const dim3 grid(p.chunks, std::min((p.chunk_tokens + tokens - 1) / tokens,
                                     (kGradCtas * kSms + p.chunks - 1) / p.chunks));
  // A grid of one wave of four CTAs to an SM takes shared memory that nobody uses, so that an SM takes no
  // fifth while another has three (32768 x 64: 3.4 us, without it 3.9; on larger grids it only takes L1
  // away, 131072 x 128: 22.7 us, without it 21.9).
  const size_t smem = (int64_t)grid.x * grid.y <= 4 * kSms ? 46 * 1024 : 0;
  auto go = [&](auto kern) {
    return launch_kernel(kern, grid, kGradThreads, smem, st, 1, p, dloss, dZ, lanes);
  };
  return p.mask ? go(balance_grad_kernel<V, NV, true>) : go(balance_grad_kernel<V, NV, false>);
}

cudaError_t launch_balance_backward(const BalanceArgs& p, const float* dloss, float* dZ,
                                    LaunchStream st) {
  const int v = p.E % 4 == 0 ? 4 : 1, nv = p.E / v;
  int lanes = 1;
  while (lanes < 32 && lanes < nv) lanes *= 2;
  const int per = (nv + lanes - 1) / lanes;   // vectors to a lane: up to 4 (V 4) or 16 (V 1)
  if (v == 4)
    return per <= 1   ? grad_go<4, 1>(p, dloss, dZ, lanes, st)
           : per <= 2 ? grad_go<4, 2>(p, dloss, dZ, lanes, st)
                      : grad_go<4, 4>(p, dloss, dZ, lanes, st);
  return per <= 1   ? grad_go<1, 1>(p, dloss, dZ, lanes, st)
         : per <= 2 ? grad_go<1, 2>(p, dloss, dZ, lanes, st)
         : per <= 4 ? grad_go<1, 4>(p, dloss, dZ, lanes, st)
                    : grad_go<1, 16>(p, dloss, dZ, lanes, st);
}

}  // namespace ecmoe
