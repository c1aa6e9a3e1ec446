// Counter-based random words for dropout: Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011; ten rounds, the paper's multipliers and
// key increments).
//
// Element i of a tensor takes word i % 4 of the block with counter (i / 4 low, i / 4 high, step, site)
// under the key (seed low, seed high), so what an element draws depends on nothing but its place:
// the backward pass draws the same words again and no mask is stored, and a tensor may be cut among
// threads, CTAs and kernels in any way.
#pragma once
#include <stdint.h>

namespace ecmoe {

// What a kernel needs to draw: rng points to device memory {seed, step}; a word below `threshold` =
// round(p 2^32) drops its element, the others are scaled by 1 / (1 - p).
struct DropArgs {
  const unsigned long long* rng = nullptr;   // NULL: no dropout
  uint32_t threshold = 0, site = 0;
  float scale = 1.f;
};

struct DropKey {
  uint32_t k0, k1, step, site;
};
__device__ __forceinline__ DropKey drop_key(const DropArgs& d) {
  const unsigned long long seed = __ldg(d.rng), step = __ldg(d.rng + 1);
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, d.site};
}

constexpr uint32_t kPhiloxM0 = 0xD2511F53u, kPhiloxM1 = 0xCD9E8D57u;   // multipliers
constexpr uint32_t kPhiloxW0 = 0x9E3779B9u, kPhiloxW1 = 0xBB67AE85u;   // key increments

// Both halves of a product (dropout of 67 M bf16 values and its gradient 113 us; with a 64-bit product in C++,
// shifted and cut, 125).
__device__ __forceinline__ void mul_wide(uint32_t m, uint32_t x, uint32_t& hi, uint32_t& lo) {
  asm("{\n\t.reg .b64 t;\n\tmul.wide.u32 t, %2, %3;\n\tmov.b64 {%0, %1}, t;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(x), "r"(m));
}

// A round takes (x0, x1, x2, x3) to (hi(M1 x2) ^ x1 ^ k0, lo(M1 x2), hi(M0 x0) ^ x3 ^ k1, lo(M0 x0)).
// Of the first two rounds only two products depend on the block's low word; the rest is the same for
// every block with one high word, and is taken out of the loop here.
struct DropPrefix {
  uint32_t c1, c2, c3, c4;
};
__device__ __forceinline__ DropPrefix drop_prefix(const DropKey& k, uint32_t high) {
  const uint64_t b = (uint64_t)kPhiloxM1 * k.step;
  const uint32_t x0 = (uint32_t)(b >> 32) ^ high ^ k.k0;
  const uint64_t a = (uint64_t)kPhiloxM0 * x0;
  return {k.site ^ k.k1, (uint32_t)b ^ (k.k0 + kPhiloxW0), (uint32_t)(a >> 32) ^ (k.k1 + kPhiloxW1),
          (uint32_t)a};
}

// The four words of elements 4 block .. 4 block + 3, low: block's low word.
__device__ __forceinline__ uint4 drop_words(const DropKey& key, const DropPrefix& p, uint32_t low) {
  uint32_t ah, al, bh, bl;
  mul_wide(kPhiloxM0, low, ah, al);
  mul_wide(kPhiloxM1, ah ^ p.c1, bh, bl);
  uint32_t x0 = bh ^ p.c2, x1 = bl, x2 = al ^ p.c3, x3 = p.c4;
#pragma unroll
  for (uint32_t r = 2; r < 10; ++r) {
    mul_wide(kPhiloxM0, x0, ah, al);
    mul_wide(kPhiloxM1, x2, bh, bl);
    x0 = bh ^ x1 ^ (key.k0 + r * kPhiloxW0);
    x2 = ah ^ x3 ^ (key.k1 + r * kPhiloxW1);
    x1 = bl;
    x3 = al;
  }
  return make_uint4(x0, x1, x2, x3);
}

// v[0..3], four elements with their words, dropped or scaled. A dropped element is exactly 0, whatever
// it held (NaN and infinities too).
__device__ __forceinline__ void drop4(float* v, const uint4& w, const DropArgs& d) {
  v[0] = w.x >= d.threshold ? v[0] * d.scale : 0.f;
  v[1] = w.y >= d.threshold ? v[1] * d.scale : 0.f;
  v[2] = w.z >= d.threshold ? v[2] * d.scale : 0.f;
  v[3] = w.w >= d.threshold ? v[3] * d.scale : 0.f;
}
// The same for n elements (a multiple of 4) from block `block` on; no two of the n / 4 blocks differ in
// their high words where n / 4 divides the block's number.
template <int n>
__device__ __forceinline__ void drop_n(float* v, const DropKey& key, const DropArgs& d, uint64_t block) {
  const DropPrefix p = drop_prefix(key, (uint32_t)(block >> 32));
#pragma unroll
  for (int q = 0; q < n / 4; ++q) drop4(v + 4 * q, drop_words(key, p, (uint32_t)block + q), d);
}

}  // namespace ecmoe
