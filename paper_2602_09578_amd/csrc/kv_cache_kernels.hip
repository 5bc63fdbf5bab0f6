// KV-cache maintenance that precedes attention in a decode iteration: appending each
// sequence's new token to its paged suffix, and copying pages when a sample is forked from
// another one.  The paper only says that rollout manages large KV caches (Section 4.1) and
// that prompts are expanded into several samples (Section 5.1); the operations are the
// plain scatter / copy stated in marl_decode.h.  Pure data movement: results are bit-exact.
//   Into an 8-bit cache (kv_fp8.h) the appended rows are quantised on their way, and whole pages are read back as bf16, for
// calls that take a bf16 cache (a further chunk of a prompt).
#include "kv_fp8.h"
#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {
namespace {

// One workgroup of 256 threads per sequence: a thread stores V channels (2 bytes each, the layout keeps
// a channel's 16 slots together) of up to four (head, channel) pairs at a time and one 16-byte piece of
// a key row.  Latency is all it costs at small batches, so everything of a round is requested before
// the first store (64 sequences, 8 KV heads: 5.2 us; one head after the other, each waiting for its
// loads, 7.8 us).  Every thread reads the old length before the barrier; thread 0 stores the new
// one after it.
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(KvAppendArgs a) {
  const int s = blockIdx.x;
  const int tid = threadIdx.x;
  const int pos = a.suffix_lens[s];
  const uint16_t* kn = a.k_new + (size_t)s * a.Hkv * kD;
  const uint16_t* vn = a.v_new + (size_t)s * a.Hkv * kD;
  int flag = 0;
  int page = -1;
  if (pos < 0 || pos >= a.max_sp * kPage) flag = MARL_FLAG_LEN_CLAMPED;          // no room in the table row
  else {
    page = a.suffix_table[(size_t)s * a.max_sp + (pos >> 4)];
    if ((unsigned)page >= (unsigned)a.num_pages) { flag = MARL_FLAG_BAD_PAGE; page = -1; }
  }
  const int slot = pos & (kPage - 1);
  for (int h0 = 0; h0 < a.Hkv; h0 += 4 * kAppendThreads / kD) {                  // eight heads per round
    const int n = min(a.Hkv - h0, 4 * kAppendThreads / kD) * kD;                 // (head, channel) pairs of the round
    uint16_t v[4];
    u32x4 k = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = tid + e * kAppendThreads < n ? vn[(size_t)h0 * kD + tid + e * kAppendThreads] : (uint16_t)0;
    if (tid < n / 8) k = *reinterpret_cast<const u32x4*>(kn + (size_t)h0 * kD + tid * 8);
    if (page >= 0) {
      const size_t blk = ((size_t)page * a.Hkv + h0) * (kPage * kD);             // elements
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int p = tid + e * kAppendThreads;
        if (p < n) a.v_pages[blk + (size_t)p * kPage + slot] = v[e];             // (channels of consecutive heads follow each other)
      }
      if (tid < n / 8)
        *reinterpret_cast<u32x4*>(a.k_pages + blk + (size_t)(tid >> 4) * (kPage * kD) + (size_t)slot * kD + (tid & 15) * 8) = k;
    }
  }
  if (flag && tid == 0 && a.flags) atomicOr(a.flags, flag);
  __syncthreads();
  if (page >= 0 && tid == 0) a.suffix_lens[s] = pos + 1;
}

// The append of an 8-bit cache.  16 lanes take a row (8 channels each), so 256 threads the keys and values of eight heads at a time.
// The codes of a key are contiguous; those of a value lie 16 bytes apart, one byte per channel.
__global__ __launch_bounds__(kAppendThreads) void kv_append_fp8_kernel(KvAppendFp8Args a) {
  constexpr int kHeads = kAppendThreads / 32;
  const int s = blockIdx.x;
  const int piece = threadIdx.x & 15, which = threadIdx.x >> 7, head = (threadIdx.x >> 4) & (kHeads - 1);
  const int pos = a.suffix_lens[s];
  const uint16_t* rows = (which ? a.v_new : a.k_new) + ((size_t)s * a.Hkv) * kD + piece * 8;
  int flag = 0;
  int page = -1;
  if (pos < 0 || pos >= a.max_sp * kPage) flag = MARL_FLAG_LEN_CLAMPED;          // no room in the table row
  else {
    page = a.suffix_table[(size_t)s * a.max_sp + (pos >> 4)];
    if ((unsigned)page >= (unsigned)a.num_pages) { flag = MARL_FLAG_BAD_PAGE; page = -1; }
  }
  const int slot = pos & (kPage - 1);
  for (int h0 = 0; h0 < a.Hkv; h0 += kHeads) {                                   // workgroup-uniform
    const int h = h0 + head;
    u32x4 w = {0u, 0u, 0u, 0u};
    if (h < a.Hkv) w = *reinterpret_cast<const u32x4*>(rows + (size_t)h * kD);
    int e;
    const u32x2 codes = quantize_row(w, e);
    if (page < 0 || h >= a.Hkv) continue;
    const size_t row = (size_t)page * a.Hkv + h;
    if (which == 0) {
      *reinterpret_cast<u32x2*>(a.k_pages + row * (kPage * kD) + slot * kD + piece * 8) = codes;
    } else {
      uint8_t* at = a.v_pages + row * (kPage * kD) + piece * 8 * kPage + slot;
#pragma unroll
      for (int i = 0; i < 8; ++i) at[i * kPage] = (uint8_t)(codes[i >> 2] >> (8 * (i & 3)));
    }
    if (piece == 0) a.exponents[row * (2 * kPage) + which * kPage + slot] = (int8_t)e;
  }
  if (flag && threadIdx.x == 0 && a.flags) atomicOr(a.flags, flag);
  __syncthreads();
  if (page >= 0 && threadIdx.x == 0) a.suffix_lens[s] = pos + 1;
}

// bf16 page dst[i] <- 8-bit page src[i]: one workgroup per (pair, KV head), a thread for eight codes of the keys and eight of the
// values, so that a wave stores 1 KB at a time.  The exponents of eight neighbouring slots of a value row are one load.
// What bounds it: memory, two thirds of it writes.  3001 pages x 8 heads, 296 MB: 45 us (6.6 TB/s) where the codes are still in the memory's
// own cache, 55 to 59 where they are not (a large copy reaches the same 5 TB/s); 2 to 16 us more with stores through the caches, and as
// much with two, four or eight (page, KV head) pairs a workgroup (2, 4, 11).  What the XCDs' caches (4 MB each) can hold goes through them to
// whoever reads it next.
constexpr long kReadCacheBytes = 32l << 20;
template <bool kPastCaches>
__global__ __launch_bounds__(kReadPagesThreads) void kv_read_pages_fp8_kernel(KvReadFp8Args a) {
  const int pair = blockIdx.x / a.Hkv, h = blockIdx.x - pair * a.Hkv, t = threadIdx.x;
  const int src = a.src[pair], dst = a.dst[pair];
  if ((unsigned)src >= (unsigned)a.num_pages || (unsigned)dst >= (unsigned)a.num_out_pages) {
    if (t == 0 && a.flags) atomicOr(a.flags, MARL_FLAG_BAD_PAGE);
    return;
  }
  const size_t from = (size_t)src * a.Hkv + h, to = ((size_t)dst * a.Hkv + h) * (kPage * kD) + t * 8;
  const int8_t* ex = a.exponents + from * (2 * kPage);
  const u32x2 k = *reinterpret_cast<const u32x2*>(a.k_codes + from * (kPage * kD) + t * 8);
  const u32x2 v = *reinterpret_cast<const u32x2*>(a.v_codes + from * (kPage * kD) + t * 8);
  const int ke = ex[t >> 4];
  const u32x2 ve = *reinterpret_cast<const u32x2*>(ex + kPage + (t & 1) * 8);
  u32x4 ko, vo;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float ks = pow2(max(ke, -126));
    ko[2 * i] = codes_to_bf16<false>(k[i], ks);
    ko[2 * i + 1] = codes_to_bf16<true>(k[i], ks);
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i], true);
    vo[2 * i] = pack_bf16(__builtin_amdgcn_ldexpf(lo[0], exponent_of(ve[i], 0)), __builtin_amdgcn_ldexpf(lo[1], exponent_of(ve[i], 1)));
    vo[2 * i + 1] = pack_bf16(__builtin_amdgcn_ldexpf(hi[0], exponent_of(ve[i], 2)), __builtin_amdgcn_ldexpf(hi[1], exponent_of(ve[i], 3)));
  }
  if constexpr (kPastCaches) {
    __builtin_nontemporal_store(ko, reinterpret_cast<u32x4*>(a.k_pages + to));
    __builtin_nontemporal_store(vo, reinterpret_cast<u32x4*>(a.v_pages + to));
  } else {
    *reinterpret_cast<u32x4*>(a.k_pages + to) = ko;
    *reinterpret_cast<u32x4*>(a.v_pages + to) = vo;
  }
}

// dst[i] <- src[i] for whole pages (all KV heads, K and V): one workgroup per (pair, K|V)
__global__ __launch_bounds__(256) void kv_copy_pages_kernel(KvCopyArgs a) {
  const int pair = blockIdx.x >> 1;
  uint16_t* base = (blockIdx.x & 1) ? a.v_pages : a.k_pages;
  const int src = a.src[pair], dst = a.dst[pair];
  if ((unsigned)src >= (unsigned)a.num_pages || (unsigned)dst >= (unsigned)a.num_pages) {
    if (threadIdx.x == 0 && a.flags) atomicOr(a.flags, MARL_FLAG_BAD_PAGE);
    return;
  }
  if (src == dst) return;
  const size_t page_vecs = (size_t)a.Hkv * (kPage * kD * 2 / 16);
  const u32x4* sp = reinterpret_cast<const u32x4*>(base) + (size_t)src * page_vecs;
  u32x4* dp = reinterpret_cast<u32x4*>(base) + (size_t)dst * page_vecs;
  for (size_t i = threadIdx.x; i < page_vecs; i += 256) dp[i] = sp[i];
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st) {
  if (a.NS == 0) return hipSuccess;
  hipLaunchKernelGGL(kv_append_kernel, dim3((unsigned)a.NS), dim3(kAppendThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv_append_fp8(const KvAppendFp8Args& a, hipStream_t st) {
  if (a.NS == 0) return hipSuccess;
  hipLaunchKernelGGL(kv_append_fp8_kernel, dim3((unsigned)a.NS), dim3(kAppendThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv_read_pages_fp8(const KvReadFp8Args& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const bool past_caches = (long)a.n * a.Hkv * (2 * kPage * kD * 2) > kReadCacheBytes;
  hipLaunchKernelGGL(past_caches ? kv_read_pages_fp8_kernel<true> : kv_read_pages_fp8_kernel<false>, dim3((unsigned)(a.n * a.Hkv)), dim3(kReadPagesThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv_copy_pages(const KvCopyArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(kv_copy_pages_kernel, dim3(2u * a.n), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace marl
