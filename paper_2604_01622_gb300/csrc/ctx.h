// A context of the C ABI and what its calls share: error text, phase marks, launch counts. Internal.
#pragma once
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "../../include/ecmoe.h"
#include "common.cuh"
#include "philox.cuh"

namespace ecmoe {

enum CtxKind { CTX_EC, CTX_TC, CTX_BALANCE, CTX_LINEAR };

// The balance loss over one set of sequences: of a balance context, or of a token-choice layer.
// chunk: (sequence, first token, end, 0) a chunk, chunk_off [G+1] a sequence's chunks.
struct BalanceTerm {
  int N = 0, E = 0, k = 0, G = 0;   // G = 0: none
  int chunk_tokens = 0;             // at most
  std::vector<int32_t> group_off, chunk, chunk_off;
  int chunks() const { return (int)chunk.size() / 4; }
  int table_ld() const { return (E + 3) / 4 * 4 + 4; }
  size_t o_ticket = 0, o_inv_n = 0, o_off = 0, o_chunk = 0, o_chunk_off = 0, o_part = 0, o_pcnt = 0,
         o_live = 0, o_gloss = 0, o_glive = 0, o_table = 0;
  // a layer's term: what ec_tc_balance set
  float coef = 0.f;
  const uint8_t* mask = nullptr;
  float* loss = nullptr;
  int32_t* count = nullptr;
  bool on = false;
};

// A dense product of up to `rows` rows.
struct LinearPlan {
  int rows = 0, K = 0, N = 0, act = 0;
  bool train = false;
  size_t o_dP = 0, o_xpl = 0, o_wpl = 0, o_colsum = 0, o_ticket = 0;
  int tickets = 0;
};

}  // namespace ecmoe

struct ec_ctx {
  ecmoe::CtxKind kind = ecmoe::CTX_EC;
  int N = 0, d = 0, E = 0, F = 0, G = 0, dtype = 0;
  int M_cap = 0, M = 0, max_group = 0;
  bool goff_aligned = false;   // every group of every score column starts on a 16-byte boundary
  std::vector<int32_t> group_off, k_g, k_off;
  char* ws = nullptr;
  size_t ws_bytes = 0;
  // workspace offsets (bytes)
  size_t o_status, o_goff, o_kg, o_koff, o_ST, o_S, o_idx, o_gate, o_slot, o_H, o_A, o_B, o_U,
      o_O, o_dO, o_dA, o_dB, o_dgate, o_dZ, o_dZb, o_wrpad, o_dXr, o_part, total;
  int wr_splits = 1;   // split-K factor of dWr = X^T dZ
  int dg_parts = 1;    // partial sums per gate gradient (tensor-core dU epilogue)
  size_t o_dgsum = 0;  // the gate gradients summed over their partials
  size_t o_colsum = 0; // partial column sums of dZ (router bias gradient)
  int Ep = 64;         // experts rounded up to 64 (tensor-core router operands)
  // per-kernel event timing (off by default) and kernel launch counter
  bool prof = false;
  std::vector<cudaEvent_t> ev;
  std::vector<const char*> ev_name;
  int ev_n = 0;
  bool nvtx_open = false;   // an NVTX range named after the current phase is open
  int64_t launches = 0;
  // state saved by the forward pass
  bool residual = false;   // Y = X + EC(X), dX = dY + EC input gradient
  int Fs = 0;              // shared experts: total hidden width (0 = none)
  size_t o_Ash = 0, o_Bsh = 0, o_Ush = 0, o_Osh = 0, o_dAsh = 0, o_dBsh = 0, o_shpart = 0;
  const void *Wgs = nullptr, *Wus = nullptr, *Wds = nullptr;
  float *dWgs = nullptr, *dWus = nullptr, *dWds = nullptr;
  bool have_fwd = false;
  const void *X = nullptr, *Wr = nullptr, *Wg = nullptr, *Wu = nullptr, *Wd = nullptr;
  const float* br = nullptr;
  // token choice (k > 0): k experts per token, per-expert cap (< 0: none), padded rows
  int tc_k = 0, tc_cap = -1;
  int64_t P_tc = 0;
  int tiles = EC_TILES_AUTO;   // expert-GEMM tile policy (ec_ctx_set_tiles)
  size_t o_choice = 0, o_tgate = 0, o_Zs = 0, o_count = 0, o_tiles = 0, o_kept = 0, o_tcscr = 0;
  ecmoe::BalanceTerm bal;
  ecmoe::LinearPlan lin;
  // dropout (ec_ctx_set_dropout): off while drop.rng is NULL; drop_buf: the workspace has room for it
  ecmoe::DropArgs drop;
  bool drop_buf = false;
  size_t o_drop = 0;
  int kept_status = 0;   // device status word of a workspace given up before anyone read it
  std::string err;
  ec_status err_status = EC_OK;   // status of the last failed call (ec_get_last_error)
};

namespace ecmoe {

inline ec_status fail(ec_ctx* c, ec_status s, const char* fmt, ...) {
  if (c) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    c->err = buf;
    c->err_status = s;
  }
  return s;
}

inline ec_status cuda_fail(ec_ctx* c, cudaError_t e, const char* where) {
  return fail(c, EC_ERR_CUDA, "%s: %s", where, cudaGetErrorString(e));
}

#define EC_CUDA(call, where)                         \
  do {                                               \
    cudaError_t _e = (call);                         \
    if (_e != cudaSuccess) return cuda_fail(c, _e, where); \
  } while (0)

// Phase marker: with profiling on, records an event named after the kernel about to be
// launched (or "end" after the last one) on the call's stream, and opens an NVTX range of
// the same name (closed at the next marker) for profilers that filter by range.
inline void mark(ec_ctx* c, const char* name, LaunchStream st) {
  if (!c->prof) return;
  if (c->nvtx_open) nvtxRangePop();
  c->nvtx_open = std::strcmp(name, "end") != 0;
  if (c->nvtx_open) nvtxRangePushA(name);
  if (c->ev_n == (int)c->ev.size()) {
    cudaEvent_t e;
    if (cudaEventCreate(&e) != cudaSuccess) return;
    c->ev.push_back(e);
    c->ev_name.push_back(nullptr);
  }
  cudaEventRecord(c->ev[c->ev_n], st);
  c->ev_name[c->ev_n] = name;
  ++c->ev_n;
}

// Launch `nk` kernels through `call` as one named phase.
#define EC_KERNEL(name, nk, call)            \
  do {                                       \
    mark(c, name, st);                       \
    c->launches += (nk);                     \
    EC_CUDA(call, name);                     \
  } while (0)

// One layout of a workspace: offsets in whole 256-byte units, the status word first.
struct Taker {
  size_t o = 0;
  size_t operator()(size_t bytes) {
    const size_t r = o;
    o = (o + bytes + 255) & ~size_t(255);
    return r;
  }
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename P>
P* at(ec_ctx* c, size_t off) { return reinterpret_cast<P*>(c->ws + off); }

inline size_t esize(const ec_ctx* c) { return c->dtype == EC_BF16 ? 2 : 4; }

inline ec_status check_ready(ec_ctx* c) {
  if (!c) return EC_ERR_INVALID_ARG;
  if (!c->ws) return fail(c, EC_ERR_WORKSPACE, "no workspace attached (ec_ctx_set_workspace)");
  return EC_OK;
}

// Threshold and scale of a drop probability; false where p is not in [0, 1).
inline bool drop_of(double p, DropArgs* d) {
  if (!(p >= 0.0 && p < 1.0)) return false;
  const double t = p * 4294967296.0 + 0.5;
  d->threshold = t < 4294967295.0 ? (uint32_t)t : 0xFFFFFFFFu;
  d->scale = (float)(1.0 / (1.0 - p));
  return true;
}

// Refuses a call made on a context of another kind.
inline ec_status check_kind(ec_ctx* c, CtxKind kind) {
  if (c->kind == kind) return EC_OK;
  switch (c->kind) {
    case CTX_TC:
      return fail(c, EC_ERR_STATE, "token-choice context: use ec_tc_forward / ec_tc_backward");
    case CTX_BALANCE:
      return fail(c, EC_ERR_STATE, "balance context: use ec_balance_forward / ec_balance_backward");
    case CTX_LINEAR:
      return fail(c, EC_ERR_STATE, "dense-product context: use ec_linear_forward / ec_linear_backward");
    default:
      return fail(c, EC_ERR_STATE, "expert-choice context: use ec_moe_forward / ec_moe_backward");
  }
}

// Parts that a layer's context shares with the contexts of its own kind (block_api.cu).
ec_status balance_plan(BalanceTerm* b, int N, int E, int k, int G, const int32_t* group_off);
void balance_layout(BalanceTerm* b, Taker& take);
ec_status balance_upload(ec_ctx* c, const BalanceTerm& b);
ec_status linear_clear(ec_ctx* c);   // a dense product's tickets in a new workspace
struct BalanceArgs;
BalanceArgs balance_args(ec_ctx* c, const BalanceTerm& b);
void block_layout(ec_ctx* c);   // workspace of a balance or dense-product context

#define EC_TRY(call)                  \
  do {                                \
    ec_status _s = (call);            \
    if (_s != EC_OK) return _s;       \
  } while (0)

}  // namespace ecmoe
