// What the decode attention kernels over a bf16 cache and over an 8-bit one have in common: how partial results are added and
// stored, and which workgroup of a small call takes what.
#ifndef MARL_ATTN_SHARED_H
#define MARL_ATTN_SHARED_H
#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {

constexpr int kAccRowFloats = kD + 4;   // of a row in LDS (the 16 rows that a wave instruction writes start in different banks)
constexpr int kSeqBlock = 8;            // sequences whose workgroups for one KV head and part run on one XCD

// Four channels of a final row.
__device__ __forceinline__ void store_row_piece(const AttnArgs& a, size_t at, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  if (a.out_dtype == MARL_OUT_F32) {
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at) = v;
  } else {
    *reinterpret_cast<bf16x4*>(reinterpret_cast<uint16_t*>(a.out) + at) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  }
}

// Workgroups are dealt to the eight XCDs in turn.  The workgroups of eight neighbouring sequences (usually samples of
// one prompt) for one KV head and part follow each other on one XCD, so that the prefix they share is read out
// of its L2: 64 groups of 4 samples, 16 / 2 heads, 2304 tokens: 67 -> 41 us against a plain order.  The last block of sequences
// comes after the others and is as wide as there are sequences left: with empty workgroups for those that are not there, the
// others met on a few CUs of the XCD (one sequence, 8 KV heads, 131072 tokens: 282 us, now 112; 4 KV heads, 16384: 25.7, now 16.9).
struct SmallGrid {
  int units;        // (KV head, part) pairs of a block of sequences
  int left;         // sequences of the last, narrower block
  int full_slots;   // of an XCD: workgroups for blocks of kSeqBlock sequences (the last eight units may be past the end)
  __host__ __device__ SmallGrid(const AttnArgs& a)
      : units(a.Hkv * a.splits), left(a.NS % kSeqBlock), full_slots((a.NS / kSeqBlock * units + 7) / 8 * kSeqBlock) {}
  __host__ __device__ int workgroups() const { return 8 * (full_slots + (units + 7) / 8 * left); }
  // what workgroup `index` takes; whether that is there (the last units may be past the end)
  __device__ __forceinline__ bool place(const AttnArgs& a, int index, int& s, int& kvh, int& part) const {
    const int xcd = index & 7, slot = index >> 3;
    int unit = slot / kSeqBlock * 8 + xcd, first = 0, at = slot % kSeqBlock, end = a.NS - left;
    if (slot >= full_slots) {   // workgroup-uniform
      unit = (slot - full_slots) / left * 8 + xcd;
      at = (slot - full_slots) % left;
      first = end;
      end = a.NS;
    }
    const int pair = unit / a.splits;
    part = unit % a.splits;
    s = first + pair / a.Hkv * kSeqBlock + at;
    kvh = pair % a.Hkv;
    return s < end;
  }
};

}  // namespace marl
#endif  // MARL_ATTN_SHARED_H
