// How a wave takes tokens of an 8-bit cache (kv_fp8.h): in steps of 64, four pages of one KV head, with v_mfma_f32_16x16x32_bf16.  Lane
// l = 16*j + i.
//   A 16-byte load is 16 channels of a key or all 16 slots of a value's channel, so a step is as many bytes in flight as one of 32
// tokens of a bf16 cache.  Codes become bf16 where they enter a product: the keys' with their row's scale (the conversion takes one,
// exactly), the values' without: a value's scale multiplies the token's weight, exactly too, as it is a power of two.
//   scores:  D[token][query row] = K-tile (A operand) x Q^T (B operand), four tiles of 16 tokens.  A-row i of tile T is slot 4*T + i%4 of page
// i/4, so lane (i, j) ends with the scores of query row i for all 16 slots of page j.  A 16-byte load feeds two operands of 8 channels, in the
// order in which they lie there: the queries are loaded in that order (a sum over channels may take any).
//   output:  D[channel][query row] += V^T-tile (A operand) x P^T (B operand), 8 channel tiles, each in two halves of 32 tokens: slots 8*h .. +7 of
// the four pages, which lane (i, j) holds of page j in both operands: no data moves between the products.
#ifndef MARL_KV_STEP_H
#define MARL_KV_STEP_H
#include "kv_fp8.h"
#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {

constexpr int kStepTok = 64, kStepPages = 4;
// Ids of a step's pages.  of(x): page x / 4 of them.  (The reads by readfirstlane keep the choice one between scalar registers: else the
// compiler makes it one between addresses, and the ids go through memory.)
struct StepPages {
  int p0, p1, p2, p3;
  __device__ __forceinline__ uint32_t of(int x) const {
    const int a = __builtin_amdgcn_readfirstlane(p0), b = __builtin_amdgcn_readfirstlane(p1);
    const int c = __builtin_amdgcn_readfirstlane(p2), d = __builtin_amdgcn_readfirstlane(p3);
    return x < 8 ? (x < 4 ? a : b) : (x < 12 ? c : d);
  }
};
constexpr int kCodeBytes = kPage * kD;       // of a page's keys or values of one KV head
constexpr int kExponentBytes = 2 * kPage;    // of a page and KV head
constexpr float kNoMaximum = -3.402823466e38f;   // running maximum of a row without tokens (finite: differences of two are 0)

// First of the 8 channels that lane j holds of operand kk.
__device__ __forceinline__ int channel_of(int kk, int j) { return 64 * (kk >> 1) + 16 * j + 8 * (kk & 1); }

// The operand of eight codes times 2^e, given as that number.
__device__ __forceinline__ u32x4 bf16_of_codes(uint32_t lo, uint32_t hi, float two_to_e) {
  return u32x4{codes_to_bf16<false>(lo, two_to_e), codes_to_bf16<true>(lo, two_to_e),
               codes_to_bf16<false>(hi, two_to_e), codes_to_bf16<true>(hi, two_to_e)};
}

// 2^e of the lane's key row (slot 4*T + i%4) of tile T, `word`: the exponents of slots 4*T .. +3 of its page.
__device__ __forceinline__ float key_scale(uint32_t word, int i) {
  return __uint_as_float((uint32_t)(exponent_of(word, i & 3) << 23) + 0x3f800000u);
}

// Bytes of word d of a value's channel, slots 4*d .. +3, that belong to tokens: `left` slots of the page do.
__device__ __forceinline__ uint32_t value_mask(int left, int d) {
  const int n = left - 4 * d;
  return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : 0xffffffffu >> (32 - 8 * n);
}

// Two words of the second product's operand: four weights times their values' scales.  The product takes bf16: a weight loses up to 2^-8 of itself, as
// over a bf16 cache (its sum, the divisor, does not); held in two bf16 numbers each, weights would need twice the matrix instructions and registers.
__device__ __forceinline__ void scaled_weights(const float* p, uint32_t exponents, uint32_t& lo, uint32_t& hi) {
  float w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_ldexpf(p[e], exponent_of(exponents, e));
  lo = pack_bf16(w[0], w[1]);
  hi = pack_bf16(w[2], w[3]);
}

__device__ __forceinline__ float max4(f32x4 v) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }
__device__ __forceinline__ float sum8(const float* p) { return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])); }

// The registers of a wave's step, filled straight from memory.  kStream: as data that is read once (see wave_ops.h).
template <bool kStream>
struct StepRegisters {
  u32x4 kr[4][2], vr[8];
  u32x4 kx, vx;              // exponents of the 16 slots of the pages that the lane's keys and values are of
  const char* kbase;
  const char* vbase;
  const char* kxbase;
  const char* vxbase;
  uint32_t page_bytes;
  int i, j;

  __device__ __forceinline__ StepRegisters(const AttnArgs& a, int i_, int j_) : i(i_), j(j_) { page_bytes = (uint32_t)a.Hkv * kCodeBytes; }
  __device__ __forceinline__ void keys_of(const AttnArgs& a, int kvh) {
    kbase = reinterpret_cast<const char*>(a.k_pages) + (size_t)kvh * kCodeBytes + ((i & 3) * kD + j * 16);
    kxbase = reinterpret_cast<const char*>(a.exponents) + (size_t)kvh * kExponentBytes;
  }
  __device__ __forceinline__ void values_of(const AttnArgs& a, int kvh) {
    vbase = reinterpret_cast<const char*>(a.v_pages) + (size_t)kvh * kCodeBytes + i * kPage;
    vxbase = reinterpret_cast<const char*>(a.exponents) + (size_t)kvh * kExponentBytes + kPage;
  }
  __device__ __forceinline__ void issue_k(const StepPages& p) {
    const uint32_t page = p.of(i);
    const char* kp = kbase + (uint64_t)page * page_bytes;
    kx = *reinterpret_cast<const u32x4*>(kxbase + (uint64_t)page * (page_bytes / (kCodeBytes / kExponentBytes)));
#pragma unroll
    for (int T = 0; T < 4; ++T)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const char* at = kp + T * (4 * kD) + c * 64;
        kr[T][c] = kStream ? ld_stream_k(at) : *reinterpret_cast<const u32x4*>(at);
      }
  }
  __device__ __forceinline__ void issue_v(const StepPages& p) {
    const uint32_t page = p.of(4 * j);
    const char* vp = vbase + (uint64_t)page * page_bytes;
    vx = *reinterpret_cast<const u32x4*>(vxbase + (uint64_t)page * (page_bytes / (kCodeBytes / kExponentBytes)));
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const char* at = vp + ct * (16 * kPage);
      vr[ct] = kStream ? ld_stream(at) : *reinterpret_cast<const u32x4*>(at);
    }
  }
};

// Results of 16 query rows: lane (i, j) holds channels 16*ct + 4*j .. +3 of row i; l is the lane's part of the row's sum.
struct RowTile {
  f32x4 acc[8];
  float m, l;
  __device__ __forceinline__ RowTile() : m(kNoMaximum), l(0.f) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) acc[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
};

// One step of a wave for one row tile: the `left` tokens from the step's first on exist (all 64, if there are more; none, if <= 0).  refill_k and
// refill_v are called as soon as the registers of the keys and of the values are free again.
template <bool kStream, class RefillK, class RefillV>
__device__ __forceinline__ void attend_step(StepRegisters<kStream>& kv, const u32x4 (&q)[4], float sc, int left, RowTile& t, RefillK&& refill_k,
                                            RefillV&& refill_v) {
  f32x4 s[4];
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    s[T] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float scale = key_scale(kv.kx[T], kv.i);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      s[T] = mfma_16x16x32(bf16_of_codes(kv.kr[T][kk >> 1][2 * (kk & 1)], kv.kr[T][kk >> 1][2 * (kk & 1) + 1], scale), q[kk], s[T]);
  }
  refill_k();
  if (left < kStepTok) {   // wave-uniform
    // tokens past the end: score -inf (weight 0), and their value slots zero, which may hold anything (NaN included)
    const int mine = left - kPage * kv.j;
#pragma unroll
    for (int T = 0; T < 4; ++T)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * T + e >= mine) s[T][e] = -INFINITY;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t mask = value_mask(mine, d);
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) kv.vr[ct][d] &= mask;
    }
  }
  const float m_new = fmaxf(t.m, rows_allreduce_max(fmaxf(fmaxf(max4(s[0]), max4(s[1])), fmaxf(max4(s[2]), max4(s[3])))) * sc);
  const float alpha = __builtin_amdgcn_exp2f(t.m - m_new);
  float p[16];
#pragma unroll
  for (int T = 0; T < 4; ++T)
#pragma unroll
    for (int e = 0; e < 4; ++e) p[4 * T + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[T][e], sc, -m_new));
  if (__builtin_amdgcn_ballot_w64(m_new > t.m) != 0) {   // wave-uniform
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) t.acc[ct] *= alpha;
  }
  t.l = t.l * alpha + (sum8(p) + sum8(p + 8));
  t.m = m_new;
  u32x4 w[2];
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    uint32_t lo, hi;
    scaled_weights(p + 4 * T, kv.vx[T], lo, hi);
    w[T >> 1][2 * (T & 1)] = lo;
    w[T >> 1][2 * (T & 1) + 1] = hi;
  }
#pragma unroll
  for (int ct = 0; ct < 8; ++ct)
#pragma unroll
    for (int h = 0; h < 2; ++h) t.acc[ct] = mfma_16x16x32(bf16_of_codes(kv.vr[ct][2 * h], kv.vr[ct][2 * h + 1], 1.0f), w[h], t.acc[ct]);
  refill_v();
}

}  // namespace marl
#endif  // MARL_KV_STEP_H
