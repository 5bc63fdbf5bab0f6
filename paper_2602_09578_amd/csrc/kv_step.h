// How a wave takes the tokens of a cache in steps of the attention kernels, for a bf16 cache and for one in 8 bits (kv_fp8.h).  Lane
// l = 16*j + i; the operands of v_mfma_f32_16x16x32_bf16 in both cases.
//   bf16:  32 tokens (two pages) a step.  A 16-byte load is 8 channels of a key, or 8 tokens of a value's channel.
//   8 bit: 64 tokens (four pages) a step, the same bytes in flight.  A 16-byte load is 16 channels of a key, two operands' worth (a sum over channels may
// take them in any order, so the queries are loaded in the keys' order), or all 16 slots of a value's channel.  Codes become bf16
// where they enter a product: the keys' with their row's scale, which is exact, the values' without: a value's scale multiplies the token's weight,
// exactly too, as it is a power of two.
// Scores: tiles of 16 tokens, of which lane (i, j) holds those of query row i for tokens 4*tile .. +3 of its 8 (bf16) or 16 (8 bit:
// page j of the step), so that the weights are the next product's operand where they are.
#ifndef MARL_KV_STEP_H
#define MARL_KV_STEP_H
#include "kv_fp8.h"
#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {

template <bool kFp8>
struct KvStep {
  static constexpr int kHalves = kFp8 ? 2 : 1;         // of 32 tokens: operands of the second product
  static constexpr int kTok = kBlockTok * kHalves;
  static constexpr int kPages = kTok / kPage;
  static constexpr int kTiles = kTok / 16;             // of scores
  static constexpr int kLaneTok = kTok / 4;            // tokens of a lane
  static constexpr int kKeyLoads = kFp8 ? 2 : 4;       // 16-byte loads of a tile's keys
  static constexpr int kRowBytes = kD * (kFp8 ? 1 : 2);
  static constexpr int kPageBytes = kPage * kRowBytes; // of one KV head, keys or values
  // first of the 8 channels that lane j holds of operand kk
  static __device__ __forceinline__ int channel(int kk, int j) { return kFp8 ? 64 * (kk >> 1) + 16 * j + 8 * (kk & 1) : 8 * (4 * kk + j); }
};

// The operand of eight codes times 2^e, given as that number.
__device__ __forceinline__ u32x4 bf16_of_codes(uint32_t lo, uint32_t hi, float two_to_e) {
  return u32x4{codes_to_bf16<false>(lo, two_to_e), codes_to_bf16<true>(lo, two_to_e),
               codes_to_bf16<false>(hi, two_to_e), codes_to_bf16<true>(hi, two_to_e)};
}

// Scale of the lane's key row (slot 4*tile + i%4) of a tile, from its page's exponents.
__device__ __forceinline__ float key_scale(u32x4 exponents, int tile, int i) {
  return __uint_as_float((uint32_t)(exponent_of(exponents[tile], i & 3) << 23) + 0x3f800000u);
}

// Scores of a tile (keys of 16 tokens, `scale` their lane's row's power of two; bf16: not used) and 16 query rows.
template <bool kFp8>
__device__ __forceinline__ f32x4 tile_scores(const u32x4 (&keys)[KvStep<kFp8>::kKeyLoads], float scale, const u32x4 (&q)[4]) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    if constexpr (kFp8) s = mfma_16x16x32(bf16_of_codes(keys[kk >> 1][2 * (kk & 1)], keys[kk >> 1][2 * (kk & 1) + 1], scale), q[kk], s);
    else s = mfma_16x16x32(keys[kk], q[kk], s);
  }
  return s;
}

// Which slots of a lane's word d of a value's channel belong to tokens before `end`; `first`: the lane's first token of the step.
template <bool kFp8>
__device__ __forceinline__ uint32_t value_mask(int first, int end, int d) {
  if constexpr (kFp8) {
    const int n = end - (first + 4 * d);
    return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : 0xffffffffu >> (32 - 8 * n);
  } else {
    const int tok = first + 2 * d;
    return (tok < end ? 0x0000ffffu : 0u) | (tok + 1 < end ? 0xffff0000u : 0u);
  }
}

// The second product's operand of the 8 weights from p[0] on; `exponents` of an 8-bit cache: of those 8 tokens' values.
template <bool kFp8>
__device__ __forceinline__ u32x4 weight_operand(const float* p, uint32_t exponents0, uint32_t exponents1) {
  if constexpr (kFp8) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_ldexpf(p[e], exponent_of(e < 4 ? exponents0 : exponents1, e & 3));
    return u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])};
  } else {
    return u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
  }
}

// The first product's other operand of a value channel's slots, for half h of the step.
template <bool kFp8>
__device__ __forceinline__ u32x4 value_operand(u32x4 v, int h) {
  if constexpr (kFp8) return bf16_of_codes(v[2 * h], v[2 * h + 1], 1.0f);
  else return v;
}

// The registers of one wave's step, filled straight from memory.  kStream: as data that is read once (see wave_ops.h).
template <bool kFp8, bool kStream>
struct KvRegisters {
  typedef KvStep<kFp8> Step;
  u32x4 kr[Step::kTiles][Step::kKeyLoads], vr[8];
  u32x4 kx, vx;              // 8 bit: exponents of the 16 slots of the pages that the lane's keys and values are of
  const char* kbase;
  const char* vbase;
  const char* xbase;
  size_t page_bytes;
  int i, j;

  __device__ __forceinline__ KvRegisters(const AttnArgs& a, int kvh, int i_, int j_) : i(i_), j(j_) {
    page_bytes = (size_t)a.Hkv * Step::kPageBytes;
    const int row = kFp8 ? i & 3 : 8 * ((i >> 2) & 1) + (i & 3);   // of the page, in the first tile
    kbase = reinterpret_cast<const char*>(a.k_pages) + (size_t)kvh * Step::kPageBytes + (row * Step::kRowBytes + j * 16);
    vbase = reinterpret_cast<const char*>(a.v_pages) + (size_t)kvh * Step::kPageBytes + (kFp8 ? i * kPage : i * (kPage * 2) + (j & 1) * 16);
    if constexpr (kFp8) xbase = reinterpret_cast<const char*>(a.exponents) + (size_t)kvh * (2 * kPage);
  }
  __device__ __forceinline__ void issue_k(const int (&p)[Step::kPages]) {
    int page;
    if constexpr (kFp8) page = i < 8 ? (i < 4 ? p[0] : p[1]) : (i < 12 ? p[2] : p[3]);
    else page = i < 8 ? p[0] : p[1];
    const char* kp = kbase + (size_t)page * page_bytes;
    if constexpr (kFp8) kx = *reinterpret_cast<const u32x4*>(xbase + (size_t)page * (page_bytes >> 6));
#pragma unroll
    for (int T = 0; T < Step::kTiles; ++T)
#pragma unroll
      for (int kk = 0; kk < Step::kKeyLoads; ++kk) {
        const char* at = kp + T * (4 * Step::kRowBytes) + kk * 64;
        kr[T][kk] = kStream ? ld_stream_k(at) : *reinterpret_cast<const u32x4*>(at);
      }
  }
  __device__ __forceinline__ void issue_v(const int (&p)[Step::kPages]) {
    int page;
    if constexpr (kFp8) page = j < 2 ? (j < 1 ? p[0] : p[1]) : (j < 3 ? p[2] : p[3]);
    else page = j < 2 ? p[0] : p[1];
    const char* vp = vbase + (size_t)page * page_bytes;
    if constexpr (kFp8) vx = *reinterpret_cast<const u32x4*>(xbase + (size_t)page * (page_bytes >> 6) + kPage);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      const char* at = vp + ct * (16 * kPage * (kFp8 ? 1 : 2));
      vr[ct] = kStream ? ld_stream(at) : *reinterpret_cast<const u32x4*>(at);
    }
  }
  __device__ __forceinline__ f32x4 scores(int tile, const u32x4 (&q)[4]) const {
    return tile_scores<kFp8>(kr[tile], kFp8 ? key_scale(kx, tile, i) : 1.f, q);
  }
};

}  // namespace marl
#endif  // MARL_KV_STEP_H
