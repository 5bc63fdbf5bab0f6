// Decode attention over the 8-bit KV cache (kv_fp8.h), by the plan and with the partial results of attn_kernels.hip, whose work items these
// are: prefix items (a chunk of a group's prefix for a block of its query rows), suffix items (a chunk of a sequence's own tokens) of one KV
// head, a merge of the partials in slot order, and for small calls one kernel that takes everything of a (sequence, KV head) together.  How a wave
// takes tokens is described in kv_step.h.
//
// With half the bytes per token the fixed costs of an item weigh twice as much as over a bf16 cache, and the vector ALU has codes to
// convert: so items follow each other without a gap, and waves without a row tile of their own share the others' tokens.
//   Measured (a call; its plan, items and merge kernels): 128 sequences of 8192 to 24576 own tokens and 32 prefixes of 8192, 64 / 8 heads,
// 4932 MB: 794 us (7, 780, 11; 6.3 TB/s in the items kernel, where the loads alone reach 6.8 and a plain read 7.0).  512 of a median of 256 to
// 2048 (at most 8192) and 64 prefixes of 512 to 2048, 28 / 4 heads, 789 MB: 168 us (6, 149, 10).
#include <algorithm>
#include <type_traits>

#include "attn_shared.h"
#include "kv_step.h"
#include "marl_internal.h"
#include "plan_lds.h"
#include "wave_ops.h"

namespace marl {
namespace {

constexpr int NW = kAttnThreads / 64;
constexpr int kStride = NW * kStepTok;   // tokens that the waves of a workgroup take in turn
constexpr int kMaximaAtOnce = 8;         // of partials that are about to be added
constexpr int kEager = 4;                // partials of a row that are requested before the first is used
constexpr int kSpareBlocks = 128;        // workgroups of the merge kernel beside those for the rows

// The thread's index, as something that the compiler knows nothing of: what follows from it is formed where it is used, not once
// for all items in registers that an item needs (which had 20 of them in scratch memory, and a launch with scratch takes 10 us longer).
__device__ __forceinline__ int thread_index() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

__device__ __forceinline__ float scale_of(const AttnArgs& a) {
  // scores are kept in log2 units; a zero scale becomes a tiny one so that -inf * sc stays -inf
  const float sc = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1e-30f);
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(sc)));   // (one for all lanes: a scalar register)
}
__device__ __forceinline__ uint32_t sign_flip_of(const AttnArgs& a) { return a.scale < 0.f ? 0x80008000u : 0u; }

// Page ids of the step that starts at token t of a table row, of tokens up to `end` (wave-uniform, scalar loads).  Places past the last
// page repeat it.
__device__ __forceinline__ StepPages load_pages(const AttnArgs& a, const int32_t* row, int t, int end, int& bad_page) {
  const int last = (end - 1) >> 4, first = t >> 4;
  auto id = [&](int u) {
    int page = ld_uniform(row + min(first + u, last));
    if ((unsigned)page >= (unsigned)a.num_pages) { page = 0; bad_page = 1; }
    return page;
  };
  return StepPages{id(0), id(1), id(2), id(3)};
}

// Channels of query row `row` that lane j holds of the four operands.
__device__ __forceinline__ void load_query(const AttnArgs& a, int row, int j, u32x4 (&q)[4]) {
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) q[kk] = *reinterpret_cast<const u32x4*>(a.q + (size_t)row * kD + channel_of(kk, j));
}
__device__ __forceinline__ void flip_query(u32x4 (&q)[4], uint32_t flip) {
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) q[kk] ^= flip;
}

// What the waves of a workgroup leave of a row tile, to be added in wave order (the same bits in every run).
struct TileLds {
  float m[NW][16];
  float l[NW][16];
  __attribute__((aligned(16))) float acc[NW][16][kAccRowFloats];

  __device__ __forceinline__ void put(const RowTile& t, int wave, int i, int j) {
    const float sum = rows_allreduce_sum(t.l);   // the four lanes that share a row each hold a part
    if (j == 0) {
      m[wave][i] = t.m;
      l[wave][i] = sum;
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *reinterpret_cast<f32x4*>(&acc[wave][i][16 * ct + 4 * j]) = t.acc[ct];
  }
  // channels 4 c4 .. +3 of row r over waves first, first + stride ..
  __device__ __forceinline__ f32x4 sum(int r, int c4, int first, int stride, float& mm, float& ll) const {
    mm = kNoMaximum;
    for (int w = first; w < NW; w += stride) mm = fmaxf(mm, m[w][r]);
    ll = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = first; w < NW; w += stride) {
      const float f = __builtin_amdgcn_exp2f(m[w][r] - mm);
      ll = __builtin_fmaf(l[w][r], f, ll);
      o += *reinterpret_cast<const f32x4*>(&acc[w][r][4 * c4]) * f;
    }
    return o;
  }
};

__device__ __forceinline__ void store_partial(const AttnArgs& a, size_t slot, int c4, f32x4 o, float m, float l) {
  *reinterpret_cast<f32x4*>(a.partial_o + slot * kD + 4 * c4) = o;
  if (c4 == 0) a.partial_ml[slot] = make_float2(m, l);
}

// ---------------------------------------------------------------------------------------
// Suffix items of one workgroup, one after the other.  The four waves take the 64-token steps in turn, straight from memory into
// operand registers, refilled as soon as they are free; a wave without tokens in an item takes one masked step, so that what is in flight is
// the same on every way through the code.
//   The next item is known while this one runs (see the queue below): its record and page ids are fetched while a wave waits for its last
// step's data, and its first keys, queries and values are requested where the last step frees the registers, so that they are under way
// while the waves' results are added.
//   What bounds them: memory, 6.3 TB/s.  A step's registers are its only look-ahead (186 of the 256 that two waves of a SIMD have), which is
// as many bytes as the memory needs: the same items on pages that the caches hold take half the time.
// ---------------------------------------------------------------------------------------
struct SuffixItem {
  const int32_t* row;   // of the block table
  int begin, end, seq, kvh, chunks;
};
__device__ __forceinline__ SuffixItem suffix_item(const AttnArgs& a, int index) {
  const int at = index / a.Hkv;
  const int32_t* rec = reinterpret_cast<const int32_t*>(a.suffix_items + at);
  SuffixItem it;
  it.seq = ld_uniform(rec);
  it.begin = ld_uniform(rec + 1);
  it.end = ld_uniform(rec + 2);
  it.kvh = index - at * a.Hkv;
  it.row = a.suffix_table + (size_t)it.seq * a.max_sp;
  it.chunks = ld_uniform(a.seq_chunks + it.seq);
  return it;
}

// ---------------------------------------------------------------------------------------
// Prefix items.  The group's keys and values go once from memory into an LDS ring (global_load_lds, no registers), four steps of 16 KB, and
// every wave reads what it needs of them.
//   A block has up to eight row tiles of 16.  With five to eight, tile t belongs to wave t % 4, which takes all tokens.  With fewer, waves would idle or
// convert all codes for a single tile: three or four tiles are taken in pairs, and the two waves of a pair take half of each step's tokens
// (slots 0-7 or 8-15 of its pages); one or two tiles belong to all waves, a quarter of the tokens each.  The waves' parts
// are then added through the ring's LDS.  (All waves with the same tokens: 145 us instead of 110 for a call over 32 prefixes of 8192 tokens
// for 32 rows each, 8 KV heads.)
//   A row's reference maximum moves only when a lane's weights of that row in a step sum to more than kMaxWeight (none exceeds a sum that passes, and their
// rounding to bf16 is relative): in the first step and hardly ever after.  A lane takes four tokens at a time or more, so weights are at most 64 on the mean, and
// sums over 2^21 tokens finite for values below 2^100.
//   Blocks of up to 256 rows (kHalves): half of the tiles each for two workgroups that run on the same XCD, as in attn_kernels.hip; their
// keys and values are ordinary cached loads.
//   What bounds them: waits between two waves a SIMD.  No unit is full (of the busy time the vector ALU issues in 53 %, the matrix pipe works in 25 %, and in a
// third nothing is issued): waves stand at waits and barriers in 38 % of their cycles and wait for their turn in 24 %.  Memory is not the cause.  A step of a wave with two tiles is about 560
// instructions, 64 of these matrix instructions; a wave that has tiles converts all of a step's codes itself where there are five tiles or more.  16 prefixes
// of 4096 tokens for 224 rows, 4 KV heads, 30 GFLOP: 57 us in the items kernel (0.53 PFLOP/s), the same on pages that the caches hold.  Measured
// and left out: scores by products of 8-bit numbers (the queries as two of them each: 71 us a call instead of 74, but calls bound by memory
// 0.5 to 1 % slower), one half of a step's weights beside the other half's scores (3 % slower), chunks of twice the default (88 us).
//   LDS: keys as 64 token rows of 128 bytes, the 16-byte chunk index XOR-ed with bits 1, 4, 5 of the row (the 16 rows of an operand read differ
// in bits 0, 1, 4, 5, and two rows span the banks), undone on the source side; values as [page][channel][16 slots].
// ---------------------------------------------------------------------------------------
constexpr int kStages = 4;
constexpr int kStepBytes = 2 * kStepPages * kCodeBytes;
constexpr int kRingSteps = 256;   // whose block numbers are there: all of an item's but where a caller names chunks of more than 16128 tokens
constexpr float kMaxWeight = 256.0f;
constexpr int waitcnt_imm(int vm, int lgkm) { return (vm & 0xf) | ((vm >> 4) << 14) | (7 << 4) | ((lgkm & 0xf) << 8); }
struct RingLds {
  __attribute__((aligned(16))) char buf[kStages][kStepBytes];
  __attribute__((aligned(16))) char exponents[kStages][NW][kStepPages * kExponentBytes];   // one copy a wave
  __attribute__((aligned(16))) uint32_t blocks[kRingSteps * kStepPages];                   // of steps n at n modulo kRingSteps
};
typedef const char __attribute__((address_space(1))) * GlobalBytes;
typedef char __attribute__((address_space(3))) * LdsBytes;

union ItemLds {
  RingLds ring;
  TileLds tiles[2];
  struct {
    TileLds tile;
    int rows[NW][16];
  } prefix;
};

template <bool kHalves>
__device__ __forceinline__ void prefix_item(const AttnArgs& a, const int4 it, const int kvh, const int half, ItemLds& lds, int& bad_page) {
  constexpr int kLoads = 5;
  RingLds& ring_lds = lds.ring;
  const int tid = thread_index(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, j = lane >> 4;
  const int g = it.x, tok_begin = it.y, tok_end = it.z;
  constexpr int kBlockRows = kHalves ? kRowsPerQBlockWide : kRowsPerQBlock;
  const int nrows = ld_uniform(a.group_count + g) * a.R;
  const int gstart = ld_uniform(a.group_start + g);
  const int tiles_all = (min(kBlockRows, nrows - it.w) + 15) >> 4;
  const int tiles0 = tiles_all <= 2 * NW ? tiles_all : (tiles_all + 1) >> 1;   // (at most eight tiles are not divided)
  const int tiles = half ? tiles_all - tiles0 : tiles0;
  if (kHalves && tiles <= 0) return;                         // workgroup-uniform (a first half is never empty)
  const int row_begin = it.w + (half ? tiles0 * 16 : 0);
  // the wave's tiles first, first + stride, and its share of the tokens: `sharers` waves have the same tiles
  // (the rows of a group of more than 64 sequences lie in the order in which the plan met them: all its blocks add their tokens in the same way,
  // so that a row's bits do not depend on its place)
  const bool any_order = nrows > max(64 * a.R, kRowsPerQBlock);
  const int sharers = any_order ? 1 : tiles <= 2 ? 4 : tiles <= 4 ? 2 : 1;
  const int first_tile = sharers == 4 ? 0 : sharers == 2 ? 2 * (wave & 1) : wave, tile_stride = sharers == 1 ? NW : 1;
  const int nt = sharers == 1 ? (tiles > wave + NW ? 2 : tiles > wave ? 1 : 0) : min(2, tiles - first_tile);

  const int32_t* table_row = a.prefix_table + (size_t)g * a.max_pp;
  const int nsteps = (tok_end - tok_begin + kStepTok - 1) / kStepTok;
  const int first_page = tok_begin >> 4, last_page = (tok_end - 1) >> 4;
  // A block is a page's keys or values of one KV head; its number is that of its exponents too.  Numbers of the first steps come straight from
  // the block table, so that their data is requested at once; all of them go to LDS, checked, from where a step's are read an iteration before
  // they are used (a scalar load in the loop would be waited for with the next LDS read, and both are slower than that).  A slot past the end
  // repeats the last page: valid bytes that nobody uses, so that every wait knows how many loads are in flight.
  const int n_pages = last_page - first_page + 1;
  auto block_of = [&](int page) {
    if ((unsigned)page >= (unsigned)a.num_pages) { page = 0; bad_page = 1; }
    return (uint32_t)page * (uint32_t)a.Hkv + (uint32_t)kvh;
  };
  // what a wave takes of a step: the two blocks of its loads, and the one whose exponents the lane asks for
  struct Blocks {
    uint32_t b0, b1, mine;
  };
  const int half_step = wave >> 1, mine_at = (lane >> 1) & (kStepPages - 1);
  auto read_blocks = [&](int n) {
    const uint32_t* p = ring_lds.blocks + kStepPages * (n & (kRingSteps - 1));
    return Blocks{(uint32_t)__builtin_amdgcn_readfirstlane(p[half_step]), (uint32_t)__builtin_amdgcn_readfirstlane(p[2 + half_step]), p[mine_at]};
  };
  // A step is 1024 16-byte vectors: keys of pages 0 and 1, of 2 and 3, values likewise; a load of a wave is half a page.
  uint32_t src_off[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int pos = (wave & 1) * 64 + lane;   // vector of the page
    const int key = ((pos >> 4) & 1) | (wave >> 1) << 1 | (k & 1) << 2;
    src_off[k] = 16u * (uint32_t)((k >> 1) ? pos : pos ^ key);
  }
  auto issue = [&](uint32_t ring, const Blocks& blocks) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const GlobalBytes base = reinterpret_cast<GlobalBytes>(reinterpret_cast<uintptr_t>((k >> 1) ? a.v_pages : a.k_pages)) +
                               (uint64_t)(k & 1 ? blocks.b1 : blocks.b0) * kCodeBytes;
      char* dst = ring_lds.buf[0] + (ring + k * 4096 + wave * 1024);   // wave-uniform; lane l lands at dst + 16 l
      uint32_t at = src_off[k];
      asm volatile("" : "+v"(at));   // (an offset to a scalar base, not four 64-bit addresses kept for all steps)
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const __attribute__((address_space(1))) void*>(base + at),
          reinterpret_cast<__attribute__((address_space(3))) void*>((uint32_t)reinterpret_cast<uintptr_t>(dst)), 16, 0, kHalves ? 0 : 2);   // (2: non-temporal)
    }
    if (lane < 2 * kStepPages) {   // lane 2 u + x: the exponents of page u, keys (x = 0) or values
      const GlobalBytes src = reinterpret_cast<GlobalBytes>(reinterpret_cast<uintptr_t>(a.exponents)) +
                              (uint64_t)blocks.mine * kExponentBytes + (lane & 1) * kPage;
      char* dst = ring_lds.exponents[0][0] + (ring / kStepBytes * NW + wave) * (kStepPages * kExponentBytes);
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const __attribute__((address_space(1))) void*>(src),
          reinterpret_cast<__attribute__((address_space(3))) void*>((uint32_t)reinterpret_cast<uintptr_t>(dst)), 16, 0, 0);
    }
  };
  constexpr uint32_t kRingBytes = kStages * kStepBytes;
  static_assert((kRingBytes & (kRingBytes - 1)) == 0, "the ring wraps by a mask");
  // the first three steps are requested before the chain of dependent loads that leads to the query rows
  int page0[kStages - 1], page1[kStages - 1], page_mine[kStages - 1];
#pragma unroll
  for (int s0 = 0; s0 < kStages - 1; ++s0) {
    const int page = first_page + kStepPages * s0;
    page0[s0] = ld_uniform(table_row + min(page + half_step, last_page));
    page1[s0] = ld_uniform(table_row + min(page + 2 + half_step, last_page));
    page_mine[s0] = table_row[min(page + mine_at, last_page)];
  }
#pragma unroll
  for (int s0 = 0; s0 < kStages - 1; ++s0) issue(s0 * kStepBytes, Blocks{block_of(page0[s0]), block_of(page1[s0]), block_of(page_mine[s0])});
  auto store_blocks = [&](int from, int to) {   // of steps from .. to - 1
    for (int u = from * kStepPages + tid; u < to * kStepPages; u += NW * 64)
      ring_lds.blocks[u & (kRingSteps * kStepPages - 1)] = block_of(table_row[first_page + min(u, n_pages - 1)]);
  };
  store_blocks(0, min(nsteps + kStages, kRingSteps));

  const float sc = scale_of(a);
  const uint32_t sign_flip = sign_flip_of(a);
  const int nslot = a.NCp + a.NCs, slot = tok_begin / a.Cp;
  int row_index[2];
  u32x4 qreg[2][4];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const int rho = row_begin + (first_tile + qt * tile_stride) * 16 + i;
    int idx = -1;
    if (qt < nt && rho < nrows) idx = a.group_seqs[gstart + rho / a.R] * a.Hq + kvh * a.R + rho % a.R;
    row_index[qt] = idx;
    load_query(a, max(idx, 0), j, qreg[qt]);
    flip_query(qreg[qt], sign_flip);
  }
  // (waited for here, once: with loads pending at the top of the loop the compiler would wait in every step, and for the steps in
  // flight with them)
#pragma unroll
  for (int qt = 0; qt < 2; ++qt)
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qreg[qt][kk]));
  RowTile tile[2];

  const uint32_t k_rd = (16 * (i >> 2) + (i & 3)) * kD;
  const uint32_t v_rd = kStepPages * kCodeBytes + kCodeBytes * j + kPage * i;
  auto run = [&](auto nt_tag, auto sharers_tag) {
    constexpr int NTraw = decltype(nt_tag)::value, kSharers = decltype(sharers_tag)::value;
    constexpr int NT = NTraw > 0 ? NTraw : 1;   // (no zero-length arrays; a wave without tiles only moves data)
    constexpr int kTiles = kSharers == 4 ? 1 : 2;
    // 16 kTiles tokens: slots `slot0` .. of the step's pages; `left` tokens of the step exist
    auto take = [&](uint32_t ring, int slot0, int left) {
      const char* ex = ring_lds.exponents[0][0] + (ring / kStepBytes * NW + wave) * (kStepPages * kExponentBytes) + slot0;
      const char* buf = ring_lds.buf[0] + ring;
      typedef uint32_t Words __attribute__((ext_vector_type(kTiles)));   // (a word is four slots)
      u32x4 kr[kTiles][2];
      Words vr[8];
      const Words kx = *reinterpret_cast<const Words*>(ex + (i >> 2) * kExponentBytes);
      const Words vx = *reinterpret_cast<const Words*>(ex + j * kExponentBytes + kPage);
#pragma unroll
      for (int T = 0; T < kTiles; ++T)
#pragma unroll
        for (int c = 0; c < 2; ++c) kr[T][c] = *reinterpret_cast<const u32x4*>(buf + k_rd + (slot0 + 4 * T) * kD + (((4 * c + j) ^ (i >> 1)) << 4));
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) vr[ct] = *reinterpret_cast<const Words*>(buf + v_rd + slot0 + ct * (16 * kPage));
      f32x4 s[NT][kTiles];
#pragma unroll
      for (int T = 0; T < kTiles; ++T) {
        const float scale = key_scale(kx[T], i);
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) s[qt][T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const u32x4 k = bf16_of_codes(kr[T][kk >> 1][2 * (kk & 1)], kr[T][kk >> 1][2 * (kk & 1) + 1], scale);
#pragma unroll
          for (int qt = 0; qt < NT; ++qt) s[qt][T] = mfma_16x16x32(k, qreg[qt][kk], s[qt][T]);
        }
      }
      if (left < kStepTok) {   // wave-uniform: the ragged end of the chunk
        const int mine = left - kPage * j - slot0;
#pragma unroll
        for (int T = 0; T < kTiles; ++T) {
#pragma unroll
          for (int qt = 0; qt < NT; ++qt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (4 * T + e >= mine) s[qt][T][e] = -INFINITY;
          // value slots that no token owns may hold anything (NaN included): zero them
          const uint32_t mask = value_mask(mine, T);
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) vr[ct][T] &= mask;
        }
      }
      u32x4 w[NT];
#pragma unroll
      for (int qt = 0; qt < NT; ++qt) {
        RowTile& t = tile[qt];
        float p[4 * kTiles], psum;
        auto weights = [&] {
          psum = 0.f;
#pragma unroll
          for (int T = 0; T < kTiles; ++T) {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[4 * T + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][T][e], sc, -t.m));
            psum += (p[4 * T] + p[4 * T + 1]) + (p[4 * T + 2] + p[4 * T + 3]);
          }
        };
        weights();
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(psum > kMaxWeight) != 0, 0)) {   // wave-uniform
          float mx = max4(s[qt][0]);
          if constexpr (kTiles == 2) mx = fmaxf(mx, max4(s[qt][1]));
          // (to the maximum of the row's lanes with such sums: its neighbours in the tile have no say)
          const float m_new = fmaxf(t.m, rows_allreduce_max(psum > kMaxWeight ? mx : -INFINITY) * sc);
          const float alpha = __builtin_amdgcn_exp2f(t.m - m_new);        // 1 where the row did not move
          t.l *= alpha;
          t.m = m_new;
#pragma unroll
          for (int ct = 0; ct < 8; ++ct) t.acc[ct] *= alpha;
          weights();
        }
        t.l += psum;
        // (with 16 tokens half of the second product's operands are zeros)
#pragma unroll
        for (int T = 0; T < 2; ++T) {
          uint32_t lo = 0u, hi = 0u;
          if (T < kTiles) scaled_weights(p + 4 * (T < kTiles ? T : 0), vx[T < kTiles ? T : 0], lo, hi);
          w[qt][2 * T] = lo;
          w[qt][2 * T + 1] = hi;
        }
      }
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        u32x4 v = {codes_to_bf16<false>(vr[ct][0], 1.0f), codes_to_bf16<true>(vr[ct][0], 1.0f), 0u, 0u};
        if constexpr (kTiles == 2) {
          v[2] = codes_to_bf16<false>(vr[ct][1], 1.0f);
          v[3] = codes_to_bf16<true>(vr[ct][1], 1.0f);
        }
#pragma unroll
        for (int qt = 0; qt < NT; ++qt) tile[qt].acc[ct] = mfma_16x16x32(v, w[qt], tile[qt].acc[ct]);
      }
    };
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, 0));              // this wave's block numbers are in LDS
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Blocks next = read_blocks(kStages - 1);
    uint32_t ring = 0;
#pragma unroll 1
    for (int n = 0; n < nsteps; ++n) {
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(2 * kLoads, 15));   // slot n has landed
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();                              // ... for every wave; all have read slot n - 1
      asm volatile("" ::: "memory");
      if ((n & (kRingSteps / 2 - 1)) == 0 && n > 0) store_blocks(n + kRingSteps / 2, min(nsteps + kStages, n + kRingSteps));
      issue((ring + 3 * kStepBytes) & (kRingBytes - 1), next);
      next = read_blocks(n + kStages);
      if constexpr (NTraw > 0) {
        const int left = tok_end - tok_begin - n * kStepTok;
        if constexpr (kSharers == 1) {
#pragma unroll
          for (int h = 0; h < 2; ++h) take(ring, 8 * h, left);
        } else {
          take(ring, kSharers == 2 ? 8 * (wave >> 1) : 4 * wave, left);
        }
      }
      ring = (ring + kStepBytes) & (kRingBytes - 1);
    }
  };
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  constexpr std::integral_constant<int, 2> k2{};
  constexpr std::integral_constant<int, 4> k4{};
  if (sharers == 1) {   // workgroup-uniform; the wave's number of tiles is wave-uniform
    if (nt == 2) run(k2, k1);
    else if (nt == 1) run(k1, k1);
    else run(k0, k1);
  } else if (sharers == 2) {
    if (nt == 2) run(k2, k2);
    else run(k1, k2);
  } else {
    if (nt == 2) run(k2, k4);
    else run(k1, k4);
  }

  const int tid2 = thread_index(), i2 = tid2 & 15, j2 = (tid2 & 63) >> 4;
  if (sharers == 1) {   // workgroup-uniform
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const float l = rows_allreduce_sum(tile[qt].l);
      if (row_index[qt] >= 0) {
        const size_t ps = (size_t)row_index[qt] * nslot + slot;
        float* dst = a.partial_o + ps * kD + 4 * j2;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) *reinterpret_cast<f32x4*>(dst + 16 * ct) = tile[qt].acc[ct];
        if (j2 == 0) a.partial_ml[ps] = make_float2(tile[qt].m, l);
      }
    }
  }
  // the slots requested past the end write to LDS: what comes next there, or the end of the kernel, comes after
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 15));
  __syncthreads();
  if (sharers == 1) return;
  // the sharers' parts of a tile, added in wave order: all four waves' of one tile at a time, or those of one tile of each pair
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    if (qt >= min(2, tiles)) break;                              // workgroup-uniform
    lds.prefix.tile.put(tile[qt], wave, i2, j2);
    if (j2 == 0) lds.prefix.rows[wave][i2] = row_index[qt];
    __syncthreads();
    const int pairs = 4 / sharers;                               // tiles whose parts are there
    for (int e = tid2; e < pairs * 16 * (kD / 4); e += NW * 64) {
      const int pair = e / (16 * (kD / 4)), r16 = e / (kD / 4) % 16, c4 = e % (kD / 4);
      const int row = lds.prefix.rows[pair][r16];
      if (row < 0) continue;
      float m, l;
      const f32x4 o = lds.prefix.tile.sum(r16, c4, pair, pairs, m, l);
      store_partial(a, (size_t)row * nslot + slot, c4, o, m, l);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------
// Short suffix items (at most kShortTokens tokens): one per wave, without LDS, barrier or atomic.  kFinish = false: those of sequences with
// several chunks, as partials, before the other items; kFinish = true, in the merge kernel: those of sequences whose own tokens are that one
// item, finished with the group's prefix partials; the first of these is requested with the queries and, the values, in place of the last keys.
// ---------------------------------------------------------------------------------------
template <bool kFinish>
__device__ __forceinline__ void short_item(const AttnArgs& a, const int4 rec, const int kvh, const int n_prefix, int& bad_page) {
  const int lane = threadIdx.x & 63, i = lane & 15, j = lane >> 4;
  const int nslot = a.NCp + a.NCs, end = rec.z;
  const int32_t* row = a.suffix_table + (size_t)rec.x * a.max_sp;
  const int query = rec.x * a.Hq + kvh * a.R + min(i, a.R - 1);
  const float sc = scale_of(a);
  StepRegisters<true> kv(a, i, j);
  kv.keys_of(a, kvh);
  kv.values_of(a, kvh);
  u32x4 q[4];
  load_query(a, query, j, q);
  float2 first_ml[kEager];   // (places past the last partial repeat it)
#pragma unroll
  for (int k = 0; k < kEager; ++k) {
    first_ml[k] = make_float2(-INFINITY, 0.f);
    if (kFinish && n_prefix > 0) first_ml[k] = a.partial_ml[(size_t)query * nslot + min(k, n_prefix - 1)];   // wave-uniform
  }
  int t0 = rec.y;
  StepPages pages = load_pages(a, row, t0, end, bad_page);
  kv.issue_k(pages);
  kv.issue_v(pages);
  flip_query(q, sign_flip_of(a));
  RowTile t;
  for (; t0 + kStepTok < end; t0 += kStepTok) {
    pages = load_pages(a, row, t0 + kStepTok, end, bad_page);
    attend_step(kv, q, sc, end - t0, t, [&] { kv.issue_k(pages); }, [&] { kv.issue_v(pages); });
  }
  f32x4 o0[8];
  const float* first = a.partial_o + (size_t)query * nslot * kD + 4 * j;
  attend_step(kv, q, sc, end - t0, t, [&] {
    if (kFinish && n_prefix > 0) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o0[ct] = *reinterpret_cast<const f32x4*>(first + 16 * ct);
    }
  }, [] {});
  const float l = rows_allreduce_sum(t.l);
  if (i >= a.R) return;
  if constexpr (!kFinish) {
    const size_t ps = (size_t)query * nslot + a.NCp + rec.y / a.Cs;
    float* dst = a.partial_o + ps * kD + 4 * j;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *reinterpret_cast<f32x4*>(dst + 16 * ct) = t.acc[ct];
    if (j == 0) a.partial_ml[ps] = make_float2(t.m, l);
  } else {
    const size_t p0 = (size_t)query * nslot;
    float mstar = t.m;
#pragma unroll
    for (int k = 0; k < kEager; ++k) mstar = fmaxf(mstar, first_ml[k].x);
    for (int k = kEager; k < n_prefix; k += kMaximaAtOnce) {
      float mk[kMaximaAtOnce];
#pragma unroll
      for (int u = 0; u < kMaximaAtOnce; ++u) mk[u] = a.partial_ml[p0 + min(k + u, n_prefix - 1)].x;
#pragma unroll
      for (int u = 0; u < kMaximaAtOnce; ++u) mstar = fmaxf(mstar, mk[u]);
    }
    float denom = 0.f;
    f32x4 sum[8];
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) sum[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (n_prefix > 0) {
      const float f = __builtin_amdgcn_exp2f(first_ml[0].x - mstar);
      denom = first_ml[0].y * f;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) sum[ct] = o0[ct] * f;
    }
    constexpr int kAtOnce = kEager - 1;   // requested together: one after the other, three more partials a row cost 16 us instead of 15
    for (int k = 1; k < n_prefix; k += kAtOnce) {
      f32x4 ok[kAtOnce][8];
      float2 mlk[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const size_t at = p0 + min(k + u, n_prefix - 1);
        mlk[u] = a.partial_ml[at];
        const float* src = a.partial_o + at * kD + 4 * j;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) ok[u][ct] = *reinterpret_cast<const f32x4*>(src + 16 * ct);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const float f = k + u < n_prefix ? __builtin_amdgcn_exp2f(mlk[u].x - mstar) : 0.f;
        denom = __builtin_fmaf(mlk[u].y, f, denom);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) sum[ct] += ok[u][ct] * f;
      }
    }
    const float f = __builtin_amdgcn_exp2f(t.m - mstar);
    denom = __builtin_fmaf(l, f, denom);
    const float inv = denom > 0.f ? 1.0f / denom : 0.f;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) store_row_piece(a, (size_t)query * kD + 16 * ct + 4 * j, (sum[ct] + t.acc[ct] * f) * inv);
  }
}

template <bool kFinish>
__device__ __forceinline__ void short_suffix_items(const AttnArgs& a, int& bad_page) {
  const int n_long = a.counters[MARL_CTR_NUM_LONG_SUFFIX_ITEMS] * a.Hkv;
  const int n_work = a.counters[MARL_CTR_NUM_SUFFIX_ITEMS] * a.Hkv;
  const int stride = gridDim.x * NW;
  int cur = n_long + blockIdx.x * NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (cur >= n_work) return;
  int4 rec = a.suffix_items[cur / a.Hkv];
  while (cur < n_work) {
    const int nxt = cur + stride;
    const int4 nrec = nxt < n_work ? a.suffix_items[nxt / a.Hkv] : make_int4(0, 0, 0, 0);
    const int chunks = ld_uniform(a.seq_chunks + rec.x);
    if (((chunks >> 16) == 1) == kFinish) short_item<kFinish>(a, rec, cur % a.Hkv, chunks & 0xffff, bad_page);
    cur = nxt;
    rec = nrec;
  }
}

// ---------------------------------------------------------------------------------------
// Items kernel: prefix and suffix items of a call from one queue, in the order of attn_kernels.hip's: the head of the suffix list, the prefix
// items, the other suffix items.  A workgroup's first entry is its index, its second the mirror image of that in the next round (the list is
// sorted, longest first); it draws the one after the next while it works on one.  A sequence's long suffix item is left as a partial but where
// the sequence has no prefix and no other item.
//   Two workgroups a CU ask for more than the memory can bring, and an item gets a 512th of its rate: one that is much longer than the others
// then ends long after them.  Where the list says so (ends_late), one workgroup a CU, enough to keep the memory busy, takes the suffix items, each
// at twice the rate, and the other the prefix items, which leave the memory time.  512 sequences of a median of 256 to 2048 tokens, 8192 at most:
// 182 -> 169 us; 640 with a median of 600: 174 -> 159; 16 x 32 with a median of 512 and 256-row prefix items: 141 -> 128.  Where items are about as long, it would
// cost 5 % (1024 sequences of 200 to 1000 tokens: 130 -> 137) to 20 (32 x 12 short ones after prefixes of 1000 to 6000: 88 -> 108); asking costs 1 us.
// ---------------------------------------------------------------------------------------
// Tokens of an item, as the plan lists them (longest first).
__device__ __forceinline__ int tokens_of(const int4* item) {
  const int32_t* rec = reinterpret_cast<const int32_t*>(item);
  return ld_uniform(rec + 2) - ld_uniform(rec + 1);
}
// Whether the longest suffix item, at one workgroup's share of the memory's rate, would end after all others: its tokens against what each of
// `grid` workgroups takes, the mean by the items in the middle of the list's quarters.
__device__ __forceinline__ bool ends_late(const AttnArgs& a, int suffix_items, int prefix_items, int grid) {
  const int longest = tokens_of(a.suffix_items);
  int four = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) four += tokens_of(a.suffix_items + (int)((2 * k + 1) * (long)suffix_items / 8));
  const int prefix = prefix_items > 0 ? tokens_of(a.prefix_items + prefix_items / 2) * kPrefixTokenCost : 0;
  const float all = ((float)suffix_items * (float)four * 0.25f + (float)prefix_items * (float)prefix) * (float)a.Hkv;
  return (float)longest * (float)grid > all;
}

template <bool kWide>
__device__ __forceinline__ void items_kernel_body(const AttnArgs& a) {
  __shared__ ItemLds lds;
  __shared__ int drawn_entry[2];
  const int n_long = a.counters[MARL_CTR_NUM_LONG_SUFFIX_ITEMS] * a.Hkv;
  const int pairs = a.counters[MARL_CTR_NUM_PREFIX_ITEMS] * a.Hkv;
  // wide: entries come in groups of 16, the first halves of eight (item, KV head) pairs and their second halves: workgroups are dealt to the
  // eight XCDs in turn, so the halves of a pair meet on one of them
  const int n_prefix = kWide ? (pairs + 7) / 8 * 16 : pairs;
  // short items that become partials are entries in short lists, and taken by the waves first in long ones
  const bool partials = a.counters[MARL_CTR_NUM_SHORT_PARTIAL_ITEMS] > 0;
  const int n_all = a.counters[MARL_CTR_NUM_SUFFIX_ITEMS] * a.Hkv;
  const int grid = gridDim.x;
  const bool as_entries = partials && n_prefix + n_all <= grid + grid / 2;
  const int n_suffix = as_entries ? n_all : n_long;
  // (apart, a streamer has two suffix items at least)
  const int streamers = (grid + 1) / 2, others = grid - streamers;
  const bool apart = !as_entries && n_suffix >= 2 * streamers && ends_late(a, n_suffix / a.Hkv, pairs / a.Hkv, grid);
  const int head = apart ? 0 : a.counters[MARL_CTR_NUM_FIRST_SUFFIX_ITEMS] * a.Hkv;
  const int total = n_prefix + n_suffix;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float sc = scale_of(a);
  const uint32_t sign_flip = sign_flip_of(a);
  const int nslot = a.NCp + a.NCs;
  int bad_page = 0;
  if (partials && !as_entries) {
    short_suffix_items<false>(a, bad_page);
    __syncthreads();
  }

  auto is_prefix = [&](int e) { return e >= head && e < head + n_prefix; };
  auto suffix_index = [&](int e) { return e < head ? e : e - n_prefix; };
  // whether an entry is a suffix item to be taken here, and which (among the short ones of a short list some are left to the merge kernel)
  auto suffix_of = [&](int e, SuffixItem& it) {
    if (e >= total || is_prefix(e)) return false;
    it = suffix_item(a, suffix_index(e));
    return suffix_index(e) < n_long || it.chunks >> 16 != 1;
  };
  // The queue: the current entry and the next one.  The one after is drawn while the current item is worked on (its first thread asks
  // for it at the start and leaves it in LDS before the item's last barrier).
  // Apart, entries are the prefix items and then the suffix items, and the two kinds are drawn by themselves.
  const bool draws = apart || total > 2 * grid;
  int cur = blockIdx.x, next = 2 * grid - 1 - cur, parity = 0, drawn = 0;
  bool streams = false;   // (of the first thread: draws suffix items)
  if (apart) {
    streams = cur < streamers;
    const int at = streams ? cur : cur - streamers, mirror = 2 * (streams ? streamers : others) - 1 - at;
    cur = streams ? n_prefix + at : at < n_prefix ? at : total;
    next = streams ? n_prefix + mirror : mirror < n_prefix ? mirror : total;
  }
  auto draw_prefix = [&] { return 2 * others + atomicAdd(&a.counters[MARL_CTR_PREFIX_CURSOR], 1); };
  auto draw = [&] {
    if (!draws || threadIdx.x != 0) return;
    if (apart && !streams) drawn = draw_prefix();
    else drawn = (apart ? n_prefix + 2 * streamers : 2 * grid) + atomicAdd(&a.counters[MARL_CTR_SUFFIX_CURSOR], 1);
  };
  auto leave_drawn = [&] {
    if (!draws || threadIdx.x != 0) return;
    if (apart) {
      if (streams && drawn >= total) {   // no suffix item is left
        streams = false;
        drawn = draw_prefix();
      }
      if (!streams && drawn >= n_prefix) drawn = total;
    }
    drawn_entry[parity] = drawn;
  };
  auto advance = [&] {   // after the barrier
    cur = next;
    next = draws ? drawn_entry[parity] : total;
    parity ^= 1;
  };
  while (cur < total) {   // workgroup-uniform, as everything about entries
    SuffixItem it;
    if (suffix_of(cur, it)) {
      const int tid = thread_index(), lane = tid & 63, i = lane & 15, j = lane >> 4;
      StepRegisters<true> kv(a, i, j);
      u32x4 q[4];
      auto query_row = [&](const SuffixItem& x) { return x.seq * a.Hq + x.kvh * a.R + min(i, a.R - 1); };
      StepPages pages = load_pages(a, it.row, it.begin + wave * kStepTok, it.end, bad_page);
      kv.keys_of(a, it.kvh);
      kv.values_of(a, it.kvh);
      kv.issue_k(pages);
      load_query(a, query_row(it), j, q);
      kv.issue_v(pages);
      for (bool more = true; more;) {
        draw();
        int t0 = it.begin + wave * kStepTok;
        if (t0 + kStride < it.end) pages = load_pages(a, it.row, t0 + kStride, it.end, bad_page);
        flip_query(q, sign_flip);
        RowTile t;
        while (t0 + kStride < it.end) {
          attend_step(kv, q, sc, it.end - t0, t, [&] { kv.issue_k(pages); }, [&] { kv.issue_v(pages); });
          t0 += kStride;
          if (t0 + kStride < it.end) pages = load_pages(a, it.row, t0 + kStride, it.end, bad_page);
        }
        // the last step's registers are refilled for the next item (if there is none here, for this item's first step once more: as many
        // loads on either way)
        SuffixItem ahead = it;
        more = suffix_of(next, ahead);
        if (!more) ahead = it;
        pages = load_pages(a, ahead.row, ahead.begin + wave * kStepTok, ahead.end, bad_page);
        attend_step(kv, q, sc, it.end - t0, t,
                    [&] {
                      leave_drawn();   // (asked for before the keys that have just been waited for)
                      kv.keys_of(a, ahead.kvh);
                      kv.issue_k(pages);
                      load_query(a, query_row(ahead), j, q);
                    },
                    [&] {
                      kv.values_of(a, ahead.kvh);
                      kv.issue_v(pages);
                    });
        TileLds& tl = lds.tiles[parity];   // (two: while some threads still add one item's parts others may be done with the next item)
        tl.put(t, wave, i, j);
        __syncthreads();
        const bool finish = it.chunks == 1 << 16;   // no prefix, no other item
        for (int e = tid; e < a.R * (kD / 4); e += NW * 64) {
          const int r = e / (kD / 4), c4 = e % (kD / 4);
          const size_t row = (size_t)it.seq * a.Hq + it.kvh * a.R + r;
          float m, l;
          const f32x4 o = tl.sum(r, c4, 0, 1, m, l);
          if (finish) store_row_piece(a, row * kD + 4 * c4, o * (l > 0.f ? 1.0f / l : 0.f));
          else store_partial(a, row * nslot + a.NCp + it.begin / a.Cs, c4, o, m, l);
        }
        advance();
        it = ahead;
      }
      __syncthreads();   // (a prefix item's LDS is that of the sums)
    } else {
      draw();
      if (is_prefix(cur)) {
        const int qi = cur - head;
        if constexpr (kWide) {
          const int pair = (qi >> 4) * 8 + (qi & 7);
          if (pair < pairs) prefix_item<true>(a, a.prefix_items[pair / a.Hkv], pair % a.Hkv, (qi >> 3) & 1, lds, bad_page);
        } else {
          prefix_item<false>(a, a.prefix_items[qi / a.Hkv], qi % a.Hkv, 0, lds, bad_page);
        }
      }
      leave_drawn();
      __syncthreads();
      advance();
    }
  }
  if (bad_page) atomicOr(&a.counters[MARL_CTR_FLAGS], MARL_FLAG_BAD_PAGE);
}

__global__ __launch_bounds__(kAttnThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void items_fp8_kernel(AttnArgs a) { items_kernel_body<false>(a); }
__global__ __launch_bounds__(kAttnThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void items_fp8_kernel_wide(AttnArgs a) { items_kernel_body<true>(a); }

// The partials of one row, those of npc prefix chunks and nsc own ones, added in slot order; half a wave a row.
struct MergedRow {
  int row, npc, n;   // n < 0: not a row to be added
  float2 mlk[kEager];
  f32x4 ok[kEager];

  __device__ __forceinline__ int slot_of(const AttnArgs& a, int k) const { return k < npc ? k : a.NCp + (k - npc); }
  __device__ __forceinline__ size_t first_slot(const AttnArgs& a) const { return (size_t)row * (a.NCp + a.NCs); }
  // (channels 4*sub .. 4*sub+3 of the lane)
  __device__ __forceinline__ f32x4 load(const AttnArgs& a, int slot) const {
    return __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.partial_o + (first_slot(a) + slot) * kD + 4 * (threadIdx.x & 31)));
  }

  // Asks for the first ones.
  __device__ __forceinline__ void request(const AttnArgs& a, int r, bool here, int num_prefix, int num_own) {
    row = r;
    npc = num_prefix;
    n = here ? num_prefix + num_own : -1;
#pragma unroll
    for (int k = 0; k < kEager; ++k) {
      mlk[k] = make_float2(-INFINITY, 0.f);
      ok[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k < n) {
        const int sl = slot_of(a, k);
        mlk[k] = a.partial_ml[first_slot(a) + sl];
        ok[k] = load(a, sl);
      }
    }
  }
  // Adds all of them and stores the row.
  __device__ __forceinline__ void finish(const AttnArgs& a) {
    if (n < 0) return;
    float mstar = -INFINITY;
#pragma unroll
    for (int k = 0; k < kEager; ++k) mstar = fmaxf(mstar, mlk[k].x);
    for (int k = kEager; k < n; k += kMaximaAtOnce) {
      float mk[kMaximaAtOnce];
#pragma unroll
      for (int u = 0; u < kMaximaAtOnce; ++u) mk[u] = a.partial_ml[first_slot(a) + slot_of(a, min(k + u, n - 1))].x;
#pragma unroll
      for (int u = 0; u < kMaximaAtOnce; ++u) mstar = fmaxf(mstar, mk[u]);
    }
    float denom = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kEager; ++k) {
      const float f = (mlk[k].x == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(mlk[k].x - mstar);
      denom = __builtin_fmaf(mlk[k].y, f, denom);
      acc += ok[k] * f;
    }
    for (int k = kEager; k < n; k += kEager) {   // as many at once as before the first use
#pragma unroll
      for (int u = 0; u < kEager; ++u) {
        const int sl = slot_of(a, min(k + u, n - 1));
        mlk[u] = a.partial_ml[first_slot(a) + sl];
        ok[u] = load(a, sl);
      }
#pragma unroll
      for (int u = 0; u < kEager; ++u) {
        const float f = (mlk[u].x == -INFINITY || k + u >= n) ? 0.f : __builtin_amdgcn_exp2f(mlk[u].x - mstar);
        denom = __builtin_fmaf(mlk[u].y, f, denom);
        acc += ok[u] * f;
      }
    }
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (n > 0 && denom > 0.f) r = acc * (1.0f / denom);
    store_row_piece(a, (size_t)row * kD + 4 * (threadIdx.x & 31), r);
  }
};

// Merge kernel: first the sequences whose own tokens are one short item, then the other rows' partials, half a wave a row.
// What bounds it: chains of dependent loads (the lists' lengths, an item, its page ids, its keys, the prefix partials).  11 us for 8192 rows of up
// to five partials, 10 for 14336 of up to three, 15 for 2048 items of up to 64 tokens with four prefix partials each.  Two to four rows for half a wave
// at once were 1 to 3 us slower.
// The workgroups that have short items take rows last, and the grid has some to spare, so that a row hardly ever waits for an item: 1 to 2 us
// of a call.
constexpr int kRowsPerBlock = kAttnThreads / 32;
__global__ __launch_bounds__(kAttnThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void merge_fp8_kernel(AttnArgs a) {
  const int rows = a.NS * a.Hq, at = blockIdx.x, grid = gridDim.x;
  const int short_items = (a.counters[MARL_CTR_NUM_SUFFIX_ITEMS] - a.counters[MARL_CTR_NUM_LONG_SUFFIX_ITEMS]) * a.Hkv;
  const int takers = min((short_items + NW - 1) / NW, grid);
  const int row = (at >= takers ? at - takers : at + grid - takers) * kRowsPerBlock + (threadIdx.x >> 5);
  const int seq = min(row, rows - 1) / a.Hq;   // (loads without a branch, which would be waited for before the items)
  const int info = a.seq_chunks[seq];
  const int own = min(a.suffix_lens[seq], a.max_sp * kPage);
  int bad_page = 0;
  short_suffix_items<true>(a, bad_page);
  if (bad_page) atomicOr(&a.counters[MARL_CTR_FLAGS], MARL_FLAG_BAD_PAGE);
  const int npc = info & 0xffff, nsc = info >> 16;
  // (else finished above, or in the items kernel)
  const bool here = row < rows && !(nsc == 1 && (npc == 0 || own <= kShortTokens));
  MergedRow m;
  m.request(a, min(row, rows - 1), here, npc, nsc);
  m.finish(a);
}

// ---------------------------------------------------------------------------------------
// A small call: one workgroup takes the tokens, prefix and own, of one part of a (sequence, KV head), as in attn_small_kernel.hip.
//   What bounds it: one chain of loads (lengths, page ids, keys, values) and the launch.  16 sequences of 4 prompts of 256 tokens and up to 128 of
// their own, 8 / 2 heads: 6 us.
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ void small_item(const AttnArgs& a, const int s, const int kvh, const int part) {
  __shared__ TileLds lds;
  const int lane = threadIdx.x & 63, i = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float sc = scale_of(a);
  const int g = ld_uniform(a.group_of_seq + s);
  const int S = min(max(ld_uniform(a.suffix_lens + s), 0), a.max_sp * kPage);
  u32x4 q[4];
  load_query(a, s * a.Hq + kvh * a.R + min(i, a.R - 1), j, q);
  const bool grouped = (unsigned)g < (unsigned)a.NG;
  const int P = grouped ? min(max(ld_uniform(a.prefix_lens + g), 0), a.max_pp * kPage) : 0;
  const int32_t* prefix_row = a.prefix_table + (size_t)(grouped ? g : 0) * a.max_pp;
  const int32_t* suffix_row = a.suffix_table + (size_t)s * a.max_sp;
  // steps: those of the prefix, then those of the sequence's own tokens
  const int prefix_steps = (P + kStepTok - 1) / kStepTok, all_steps = prefix_steps + (S + kStepTok - 1) / kStepTok;
  const int first_step = (int)((long)all_steps * part / a.splits), steps = (int)((long)all_steps * (part + 1) / a.splits);
  StepRegisters<false> kv(a, i, j);
  kv.keys_of(a, kvh);
  kv.values_of(a, kvh);
  int bad_page = 0;   // (the plan's workgroup raises the flag)
  // page ids of step k; `left`: the tokens that are left from its first on
  auto step_pages = [&](int k, int& left) {
    const bool own = k >= prefix_steps;
    const int t = (own ? k - prefix_steps : k) * kStepTok;
    left = (own ? S : P) - t;
    return load_pages(a, own ? suffix_row : prefix_row, t, own ? S : P, bad_page);
  };
  int k = first_step + wave;
  RowTile t;
  if (k < steps) {   // wave-uniform
    int left, left_next = 0;
    StepPages pages = step_pages(k, left);
    kv.issue_k(pages);
    kv.issue_v(pages);
    if (k + NW < steps) pages = step_pages(k + NW, left_next);
    flip_query(q, sign_flip_of(a));
    while (k + NW < steps) {
      attend_step(kv, q, sc, left, t, [&] { kv.issue_k(pages); }, [&] { kv.issue_v(pages); });
      left = left_next;
      k += NW;
      if (k + NW < steps) pages = step_pages(k + NW, left_next);
    }
    attend_step(kv, q, sc, left, t, [] {}, [] {});
  }
  lds.put(t, wave, i, j);
  __syncthreads();
  for (int e = threadIdx.x; e < a.R * (kD / 4); e += NW * 64) {
    const int r = e / (kD / 4), c4 = e % (kD / 4);
    const size_t row = (size_t)s * a.Hq + kvh * a.R + r;
    float m, l;
    const f32x4 o = lds.sum(r, c4, 0, 1, m, l);
    if (a.splits > 1) store_partial(a, row * (a.NCp + a.NCs) + part, c4, o, m, l);
    else store_row_piece(a, row * kD + 4 * c4, o * (l > 0.f ? 1.0f / l : 0.f));   // (no token at all: zeros)
  }
}

__global__ __launch_bounds__(kAttnThreads) __attribute__((amdgpu_waves_per_eu(2, 3)))
void decode_small_fp8_kernel(AttnArgs a) {
  if (blockIdx.x == 0) {
    plan_in_lds<kAttnThreads, kSmallAttnSeqs, kSmallAttnSeqs, int, true>(a);
    return;
  }
  int s, kvh, part;
  if (SmallGrid(a).place(a, blockIdx.x - 1, s, kvh, part)) small_item(a, s, kvh, part);   // (the last units may be past the end)
}

auto items_kernel_of(bool wide) { return wide ? items_fp8_kernel_wide : items_fp8_kernel; }

}  // namespace

int items_fp8_blocks_per_cu(bool wide) {
  int n = 0;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, items_kernel_of(wide), kAttnThreads, 0) != hipSuccess || n < 1) n = 1;
  return n;
}

hipError_t launch_items_fp8(const AttnArgs& a, int grid, hipStream_t st) {
  hipLaunchKernelGGL(items_kernel_of(a.qblock_rows == kRowsPerQBlockWide), dim3(grid), dim3(kAttnThreads), 0, st, a);
  return hipGetLastError();
}

// (a wave for every short item)
static long merge_workgroups(const AttnArgs& a) {
  const long rows = (long)a.NS * a.Hq, waves = ((long)a.NS * a.Hkv + NW - 1) / NW;
  const long row_blocks = (rows + kRowsPerBlock - 1) / kRowsPerBlock;
  return std::max(row_blocks + std::min(waves, (long)kSpareBlocks), waves);
}

bool merge_fp8_fits(const AttnArgs& a) { return merge_workgroups(a) <= most_workgroups(kAttnThreads); }

hipError_t launch_merge_fp8(const AttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(merge_fp8_kernel, dim3((unsigned)merge_workgroups(a)), dim3(kAttnThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_small_attn_fp8(const AttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(decode_small_fp8_kernel, dim3(SmallGrid(a).workgroups() + 1), dim3(kAttnThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace marl
