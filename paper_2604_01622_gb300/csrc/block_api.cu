// C ABI of the operators around the experts: dropout, the balance loss, the dense product.
#include <algorithm>
#include <climits>
#include <new>

#include "ctx.h"
#include "gemm_tc.h"
#include "kernels.h"

using namespace ecmoe;

namespace {

struct Span {
  const void* p;
  size_t n;
};
bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
}

}  // namespace
namespace ecmoe {

ec_status balance_plan(BalanceTerm* b, int N, int E, int k, int G, const int32_t* group_off) {
  if (!group_off) return EC_ERR_INVALID_ARG;
  if (N < 0 || E <= 0 || G <= 0 || k < 1 || k > E) return EC_ERR_SHAPE;
  if (E > kBalanceMaxE || (int64_t)N * k > 1 << 30) return EC_ERR_UNSUPPORTED;   // counts in 32 bits
  if (group_off[0] != 0 || group_off[G] != N) return EC_ERR_SHAPE;
  for (int g = 0; g < G; ++g)
    if (group_off[g + 1] < group_off[g]) return EC_ERR_SHAPE;
  const int per = balance_chunk_tokens(N, E, G, group_off);
  try {
    b->group_off.assign(group_off, group_off + G + 1);
    b->chunk.clear();
    b->chunk_off.assign(1, 0);
    for (int g = 0; g < G; ++g) {
      int64_t t = group_off[g];
      do   // an empty sequence has one empty chunk: its CTA writes the zeros
        for (int v : {g, (int)t, (int)std::min<int64_t>(t + per, group_off[g + 1]), 0})
          b->chunk.push_back(v);
      while ((t += per) < group_off[g + 1]);
      b->chunk_off.push_back((int)(b->chunk.size() / 4));
    }
  } catch (const std::bad_alloc&) {
    return EC_ERR_UNSUPPORTED;
  }
  b->N = N; b->E = E; b->k = k; b->G = G; b->chunk_tokens = per;
  return EC_OK;
}

void balance_layout(BalanceTerm* b, Taker& take) {
  const size_t C = b->chunks(), E = b->E, G = b->G;
  b->o_ticket = take((1 + G) * 4);
  b->o_inv_n = take(4);
  b->o_off = take((G + 1) * 4);
  b->o_chunk = take(C * 16);
  b->o_chunk_off = take((G + 1) * 4);
  b->o_part = take(C * E * 4);
  b->o_pcnt = take(C * E * 4);
  b->o_live = take(C * 4);
  b->o_gloss = take(G * 4);
  b->o_glive = take(G * 4);
  b->o_table = take(G * (size_t)b->table_ld() * 4);
}

ec_status balance_upload(ec_ctx* c, const BalanceTerm& b) {
  EC_CUDA(cudaMemset(c->ws + b.o_ticket, 0, (size_t)(1 + b.G) * 4), "clear the balance tickets");
  EC_CUDA(cudaMemcpy(c->ws + b.o_off, b.group_off.data(), (size_t)(b.G + 1) * 4,
                     cudaMemcpyHostToDevice), "upload the sequence offsets");
  EC_CUDA(cudaMemcpy(c->ws + b.o_chunk_off, b.chunk_off.data(), (size_t)(b.G + 1) * 4,
                     cudaMemcpyHostToDevice), "upload the chunk offsets");
  EC_CUDA(cudaMemcpy(c->ws + b.o_chunk, b.chunk.data(), b.chunk.size() * 4, cudaMemcpyHostToDevice),
          "upload the chunks");
  return EC_OK;
}

ec_status linear_clear(ec_ctx* c) {
  if (c->lin.tickets)
    EC_CUDA(cudaMemset(c->ws + c->lin.o_ticket, 0, (size_t)c->lin.tickets * 4), "clear the tickets");
  return EC_OK;
}

BalanceArgs balance_args(ec_ctx* c, const BalanceTerm& b) {
  BalanceArgs p;
  p.chunk = at<int4>(c, b.o_chunk);
  p.chunk_off = at<int>(c, b.o_chunk_off);
  p.part = at<float>(c, b.o_part);
  p.pcnt = at<int>(c, b.o_pcnt);
  p.live = at<int>(c, b.o_live);
  p.gloss = at<float>(c, b.o_gloss);
  p.glive = at<int>(c, b.o_glive);
  p.inv_n = at<float>(c, b.o_inv_n);
  p.ticket = at<unsigned>(c, b.o_ticket);
  p.table = at<float>(c, b.o_table);
  p.E = b.E; p.k = b.k; p.G = b.G; p.chunks = b.chunks(); p.table_ld = b.table_ld();
  p.chunk_tokens = b.chunk_tokens;
  return p;
}

void block_layout(ec_ctx* c) {
  Taker take;
  c->o_status = take(256);
  if (c->kind == CTX_BALANCE) balance_layout(&c->bal, take);
  if (c->kind == CTX_LINEAR) {
    LinearPlan& l = c->lin;
    const size_t rows = l.rows, K = l.K, N = l.N;
    const bool f32 = c->dtype == EC_F32;
    // dP: dY itself is read where there is no activation and no dropout (bf16)
    const bool need_dP = l.train && (f32 || l.act != EC_ACT_NONE || c->drop_buf);
    l.o_dP = take(!need_dP ? 0 : f32 ? 3 * rows * plane_ld(l.N) * 2 : rows * N * 2);
    l.o_xpl = take(f32 ? 3 * rows * plane_ld(l.K) * 2 : 0);
    l.o_wpl = take(f32 ? 3 * K * plane_ld(l.N) * 2 : 0);
    const LinearDpreSize dp = linear_dpre_size(l.rows, l.N, (int)esize(c));
    l.o_ticket = take(l.train ? (size_t)dp.tickets * 4 : 0);
    l.tickets = l.train ? dp.tickets : 0;
    // last and in whole 256-byte units, so a write past it is one past the workspace
    l.o_colsum = take(l.train ? dp.floats * 4 : 0);
  }
  c->total = take.o;
}

}  // namespace ecmoe

namespace {

ec_ctx* new_ctx() { return new (std::nothrow) ec_ctx(); }

// ---------------------------------------------------------------- dense product
// Kernels overlap at their ends where the product is small. Forward and backward with gelu, us plain ->
// overlapped by rows K N: 1 G 31.5 -> 29.3, 9 G 56.3 -> 54.4, 17 G 87.3 -> 85.8; 34 G 149.2 -> 150.7
// (131072 rows of 512 x 512: 356 -> 364), 69 G 266 -> 272, 137 G 556 -> 582, 275 G 1086 -> 1108.
constexpr double kLinearOverlapMax = 2.5e10;
LaunchStream linear_stream(const ec_ctx* c, int rows, void* stream) {
  return LaunchStream(static_cast<cudaStream_t>(stream),
                      (double)rows * c->lin.K * c->lin.N <= kLinearOverlapMax);
}

template <typename T>
T* tp(const void* p) { return const_cast<T*>(static_cast<const T*>(p)); }

template <typename T>
LinearEpi<T> epilogue(const ec_ctx* c, const void* b, const void* R, void* P, void* Y) {
  LinearEpi<T> ep;
  ep.bias = tp<const T>(b);
  ep.R = tp<const T>(R);
  ep.P = tp<T>(P);
  ep.Y = tp<T>(Y);
  ep.act = c->lin.act;
  ep.drop = c->drop;
  return ep;
}

// The tile kernel's or the persistent one's product of `form`: bf16 operands, or fp32 ones as planes.
template <typename T>
TileProblem<T> problem(ec_ctx* c, LinearForm form, const void* A, int lda, const void* B, int ldb, int M,
                       int N, int K) {
  TileProblem<T> t;
  t.form = form;
  t.A = A; t.lda = lda; t.B = B; t.ldb = ldb;
  t.M = M; t.N = N; t.K = K;
  t.status = at<int>(c, c->o_status);
  return t;
}

template <typename T>
ec_status run_linear_forward(ec_ctx* c, int rows, const void* X, const void* W,
                             const LinearEpi<T>& ep, LaunchStream st) {
  const int K = c->lin.K, N = c->lin.N;
  if (linear_few_rows<T>(rows, K, N)) {
    EC_KERNEL("linear_rows", 1, launch_linear_rows<T>(tp<const T>(X), tp<const T>(W), ep, rows, K, N, st));
    return EC_OK;
  }
  int lda = K, ldb = N;
  if constexpr (sizeof(T) == 4) {
    bf16 *x = at<bf16>(c, c->lin.o_xpl), *w = at<bf16>(c, c->lin.o_wpl);
    EC_KERNEL("linear_planes", 1,
              launch_linear_planes({{tp<const float>(X), x, rows, K}, {tp<const float>(W), w, K, N}}, st));
    X = x; W = w;
    lda = plane_ld(K); ldb = plane_ld(N);
  }
  TileProblem<T> t = problem<T>(c, LIN_FWD, X, lda, W, ldb, rows, N, K);
  t.ep = ep;
  EC_KERNEL("linear_gemm", 1, tc_linear<T>(t, st));
  return EC_OK;
}

template <typename T>
ec_status run_linear_backward(ec_ctx* c, int rows, const void* dY, const void* X, const void* W,
                              const void* P, void* dX, void* dW, void* db, LaunchStream st) {
  const int K = c->lin.K, N = c->lin.N;
  const bool f32 = sizeof(T) == 4, act = c->lin.act != EC_ACT_NONE;
  // dP = dY where nothing stands between them; fp32 products read its planes all the same
  const bool pre = act || c->drop.rng || (f32 && (dX || dW));
  bf16* dP = pre ? at<bf16>(c, c->lin.o_dP) : nullptr;
  int ldn = N, ldk = K;
  PlaneJobs jobs;
  const void *xa = X, *wb = W;
  if constexpr (sizeof(T) == 4) {
    bf16 *x = at<bf16>(c, c->lin.o_xpl), *w = at<bf16>(c, c->lin.o_wpl);
    if (dW) jobs.a = PlaneJob{tp<const float>(X), x, rows, K};
    if (dX) (dW ? jobs.b : jobs.a) = PlaneJob{tp<const float>(W), w, K, N};
    xa = x; wb = w;
    ldn = plane_ld(N); ldk = plane_ld(K);
  }
  if (pre || db)
    EC_KERNEL("linear_dpre", 1,
              launch_linear_dpre<T>(tp<const T>(dY), act ? tp<const T>(P) : nullptr, dP,
                                    at<float>(c, c->lin.o_colsum), at<unsigned>(c, c->lin.o_ticket),
                                    tp<T>(db), c->lin.act, c->drop, rows, N, jobs, st));
  const void* g = pre ? dP : dY;
  if (dX) {
    TileProblem<T> t = problem<T>(c, LIN_DX, g, ldn, wb, ldn, rows, K, N);
    t.ep.Y = tp<T>(dX);
    EC_KERNEL("linear_dgrad", 1, tc_linear<T>(t, st));
  }
  if (dW) {
    TileProblem<T> t = problem<T>(c, LIN_DW, xa, ldk, g, ldn, K, N, rows);
    t.ep.Y = tp<T>(dW);
    t.beside = dX != nullptr;
    EC_KERNEL("linear_wgrad", 1, tc_linear<T>(t, st));
  }
  return EC_OK;
}

}  // namespace

// ====================================================================== C ABI
extern "C" {

ec_status ec_dropout(int32_t dtype, int64_t n, const void* X, const void* R, void* Y, double p,
                     const uint64_t* rng, uint32_t site, void* stream) {
  if (dtype != EC_F32 && dtype != EC_BF16) return EC_ERR_INVALID_ARG;
  if (n < 0) return EC_ERR_SHAPE;
  DropArgs d;
  if (!X || !Y || !rng || !drop_of(p, &d)) return EC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(Y) || !aligned16(R) || (reinterpret_cast<uintptr_t>(rng) & 7u))
    return EC_ERR_INVALID_ARG;
  if (n > (int64_t)1 << 40) return EC_ERR_UNSUPPORTED;
  const size_t bytes = (size_t)n * (dtype == EC_BF16 ? 2 : 4);
  for (const void* in : {X, R})
    if (in != Y && overlap({in, bytes}, {Y, bytes})) return EC_ERR_INVALID_ARG;
  if (overlap({rng, 16}, {Y, bytes})) return EC_ERR_INVALID_ARG;
  d.rng = reinterpret_cast<const unsigned long long*>(rng);
  d.site = site;
  const LaunchStream st(static_cast<cudaStream_t>(stream), true);
  const cudaError_t e =
      dtype == EC_BF16
          ? launch_dropout<bf16>(tp<const bf16>(X), tp<const bf16>(R), tp<bf16>(Y), n, d, st)
          : launch_dropout<float>(tp<const float>(X), tp<const float>(R), tp<float>(Y), n, d, st);
  return e == cudaSuccess ? EC_OK : EC_ERR_CUDA;
}

ec_status ec_balance_ctx_create(ec_ctx** out, int32_t N, int32_t E, int32_t k, int32_t G,
                                const int32_t* group_off) {
  if (!out) return EC_ERR_INVALID_ARG;
  *out = nullptr;
  ec_ctx* c = new_ctx();
  if (!c) return EC_ERR_UNSUPPORTED;
  c->kind = CTX_BALANCE;
  const ec_status s = balance_plan(&c->bal, N, E, k, G, group_off);
  if (s != EC_OK) { delete c; return s; }
  block_layout(c);
  *out = c;
  return EC_OK;
}

ec_status ec_balance_forward(ec_ctx* c, const float* S, const int32_t* choice, const uint8_t* mask,
                             float* loss, int32_t* count, void* stream) {
  EC_TRY(check_ready(c));
  EC_TRY(check_kind(c, CTX_BALANCE));
  if (!S || !choice || !loss) return fail(c, EC_ERR_INVALID_ARG, "S, choice and loss are required");
  if (!aligned16(S)) return fail(c, EC_ERR_INVALID_ARG, "S must be 16-byte aligned");
  for (const void* p : {(const void*)choice, (const void*)loss, (const void*)count})
    if (reinterpret_cast<uintptr_t>(p) & 3u)
      return fail(c, EC_ERR_INVALID_ARG, "choice, loss and count must be 4-byte aligned");
  // sequences are finished while others are still read
  const size_t N = c->bal.N, E = c->bal.E;
  const Span out[2] = {{loss, 4}, {count, (size_t)c->bal.G * E * 4}};
  for (const Span& o : out)
    if (overlap(o, {S, N * E * 4}) || overlap(o, {choice, N * c->bal.k * 4}) || overlap(o, {mask, N}))
      return fail(c, EC_ERR_INVALID_ARG, "loss and count may not overlap an input");
  if (overlap(out[0], out[1])) return fail(c, EC_ERR_INVALID_ARG, "loss may not overlap count");
  const LaunchStream st(static_cast<cudaStream_t>(stream), true);
  BalanceArgs p = balance_args(c, c->bal);
  p.S = S; p.choice = choice; p.mask = mask; p.loss = loss; p.count = count;
  c->have_fwd = false;
  EC_KERNEL("balance", 1, launch_balance_forward(p, st));
  mark(c, "end", st);
  c->have_fwd = true;
  return EC_OK;
}

ec_status ec_balance_backward(ec_ctx* c, const float* S, const uint8_t* mask, const float* dloss,
                              float* dZ, void* stream) {
  EC_TRY(check_ready(c));
  EC_TRY(check_kind(c, CTX_BALANCE));
  if (!c->have_fwd) return fail(c, EC_ERR_STATE, "the backward call needs a preceding forward");
  if (!S || !dZ) return fail(c, EC_ERR_INVALID_ARG, "S and dZ are required");
  if (!aligned16(S) || !aligned16(dZ) || (reinterpret_cast<uintptr_t>(dloss) & 3u))
    return fail(c, EC_ERR_INVALID_ARG, "S and dZ must be 16-byte, dloss 4-byte aligned");
  const size_t n = (size_t)c->bal.N * c->bal.E * 4;
  if (overlap({S, n}, {dZ, n}) || overlap({mask, (size_t)c->bal.N}, {dZ, n}) ||
      overlap({dloss, 4}, {dZ, n}))
    return fail(c, EC_ERR_INVALID_ARG, "dZ may not overlap an input");
  const LaunchStream st(static_cast<cudaStream_t>(stream), true);
  BalanceArgs p = balance_args(c, c->bal);
  p.S = S; p.mask = mask;
  EC_KERNEL("balance_grad", 1, launch_balance_backward(p, dloss, dZ, st));
  mark(c, "end", st);
  return EC_OK;
}

ec_status ec_linear_ctx_create(ec_ctx** out, int32_t rows, int32_t K, int32_t N, int32_t act,
                               int32_t dtype, int32_t train) {
  if (!out) return EC_ERR_INVALID_ARG;
  *out = nullptr;
  if (dtype != EC_F32 && dtype != EC_BF16) return EC_ERR_INVALID_ARG;
  if (act < EC_ACT_NONE || act > EC_ACT_SILU) return EC_ERR_INVALID_ARG;
  if (rows < 0 || K <= 0 || N <= 0) return EC_ERR_SHAPE;
  const int unit = dtype == EC_BF16 ? 8 : 4;
  if (K % unit || N % unit) return EC_ERR_UNSUPPORTED;
  // up to 2^16 x 2^14 tiles of 128 x 64: CTAs, too, are counted in 32 bits
  if (K > 1 << 20 || N > 1 << 20 || rows > 1 << 23) return EC_ERR_UNSUPPORTED;
  ec_ctx* c = new_ctx();
  if (!c) return EC_ERR_UNSUPPORTED;
  c->kind = CTX_LINEAR;
  c->dtype = dtype;
  c->lin.rows = rows; c->lin.K = K; c->lin.N = N; c->lin.act = act; c->lin.train = train != 0;
  block_layout(c);
  *out = c;
  return EC_OK;
}

ec_status ec_linear_forward(ec_ctx* c, int32_t rows, const void* X, const void* W, const void* b,
                            const void* R, void* P, void* Y, void* stream) {
  EC_TRY(check_ready(c));
  EC_TRY(check_kind(c, CTX_LINEAR));
  if (rows < 0 || rows > c->lin.rows)
    return fail(c, EC_ERR_SHAPE, "%d rows: the context has room for %d", rows, c->lin.rows);
  if (rows == 0) return EC_OK;
  if (!X || !W || !Y) return fail(c, EC_ERR_INVALID_ARG, "X, W and Y are required");
  for (const void* p : {X, W, b, R, (const void*)P, (const void*)Y})
    if (!aligned16(p)) return fail(c, EC_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const size_t es = esize(c), m = rows, K = c->lin.K, N = c->lin.N, out = m * N * es;
  const Span in[4] = {{X, m * K * es}, {W, K * N * es}, {b, N * es}, {R, out}};
  for (const Span& s : in)
    if (overlap(s, {Y, out}) || overlap(s, {P, out}))
      return fail(c, EC_ERR_INVALID_ARG, "Y and P may not overlap an input");
  if (overlap({P, out}, {Y, out})) return fail(c, EC_ERR_INVALID_ARG, "P may not overlap Y");
  const LaunchStream st = linear_stream(c, rows, stream);
  EC_TRY(c->dtype == EC_BF16
             ? run_linear_forward<bf16>(c, rows, X, W, epilogue<bf16>(c, b, R, P, Y), st)
             : run_linear_forward<float>(c, rows, X, W, epilogue<float>(c, b, R, P, Y), st));
  mark(c, "end", st);
  return EC_OK;
}

ec_status ec_linear_backward(ec_ctx* c, int32_t rows, const void* dY, const void* X, const void* W,
                             const void* P, void* dX, void* dW, void* db, void* stream) {
  EC_TRY(check_ready(c));
  EC_TRY(check_kind(c, CTX_LINEAR));
  if (!c->lin.train) return fail(c, EC_ERR_STATE, "the context was created for forward calls only");
  if (rows < 0 || rows > c->lin.rows)
    return fail(c, EC_ERR_SHAPE, "%d rows: the context has room for %d", rows, c->lin.rows);
  const bool act = c->lin.act != EC_ACT_NONE;
  if (rows && (!dY || (dX && !W) || (dW && !X) || (act && !P)))
    return fail(c, EC_ERR_INVALID_ARG,
                "dY is required, W for dX, X for dW and P where there is an activation");
  for (const void* p : {dY, X, W, P, (const void*)dX, (const void*)dW, (const void*)db})
    if (!aligned16(p)) return fail(c, EC_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const size_t es = esize(c), m = rows, K = c->lin.K, N = c->lin.N;
  const Span in[4] = {{dY, m * N * es}, {X, m * K * es}, {W, K * N * es}, {act ? P : nullptr, m * N * es}};
  const Span out[3] = {{dX, m * K * es}, {dW, K * N * es}, {db, N * es}};
  for (int i = 0; i < 3; ++i) {
    for (const Span& s : in)
      if (overlap(s, out[i])) return fail(c, EC_ERR_INVALID_ARG, "a gradient may not overlap an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(c, EC_ERR_INVALID_ARG, "gradients may not overlap");
  }
  const LaunchStream st = linear_stream(c, rows, stream);
  if (rows == 0) {
    if (dW) EC_CUDA(cudaMemsetAsync(dW, 0, K * N * es, st), "zero dW");
    if (db) EC_CUDA(cudaMemsetAsync(db, 0, N * es, st), "zero db");
    return EC_OK;
  }
  EC_TRY(c->dtype == EC_BF16
             ? run_linear_backward<bf16>(c, rows, dY, X, W, P, dX, dW, db, st)
             : run_linear_backward<float>(c, rows, dY, X, W, P, dX, dW, db, st));
  mark(c, "end", st);
  return EC_OK;
}

}  // extern "C"
