// Norm of every query and key head and the rotation by position, in one pass over the heads, and its backward pass.
//
// With r = 1 / sqrt(mean(x^2) + eps) of a head's D channels, n = x r and y = n w, the rotation turns the pairs (y_a, y_b) by the
// position's angle: z_a = y_a cos - y_b sin, z_b = y_b cos + y_a sin; channels from rotary_dim on keep y.  Written for one channel d
// with its partner p: z_d = r (x_d A_d + x_p B_d), A_d = w_d cos, B_d = -+ w_p sin, where A and B are the same for all heads of a
// token.  Backward, the rotation's transpose turns dz into dy; then dw = sum of dy n over tokens and heads, and with g = dy w
//   dx = r (g - n mean(g n)).
// All of it in 32 bits, rounded once when it is stored.
//
// What bounds it: memory.  Every head is read once and written once, so a wave keeps as many rows under way as its registers
// hold: D / 8 lanes take a head (16 or 32 bytes a lane), a wave's step is 64 * 8 / D heads, and a wave has kSteps of them of one
// token, whose table row it needs once.  65543 tokens of 28 + 4 heads of 128 in bf16, 1075 MB: 178 us (6.0 TB/s); the gradient of 32771, 806 MB: 150 us.
// A step is of queries or of keys alone, so few small heads leave lanes without a row: 4 + 4 heads of 64 use half of them, 3.3 to 4.1 TB/s.  One list of both
// takes these from 182 to 151 us, their gradient from 300 to 228, but costs others 0.5 to 6 % (28 + 4 of 128, 8 + 2 of 64).
#include <algorithm>
#include <type_traits>

#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesPerBlock = kThreads / 64;
constexpr int kFinishThreads = 512, kFinishColumns = 16;

// Eight channels of a head as they lie in memory.
template <bool kF32>
struct Piece;
template <>
struct Piece<false> {
  u32x4 w;
  __device__ __forceinline__ void load(const char* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void load_once(const char* p) { w = ld_stream(p); }
  __device__ __forceinline__ void clear() { w = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ Piece of_lane(int lane) const {
    Piece o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.w[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)w[i]);
    return o;
  }
  template <bool kPastCaches>
  static __device__ __forceinline__ void store(char* p, const float (&v)[8]) {
    const u32x4 o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if constexpr (kPastCaches) __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = o;
  }
};
template <>
struct Piece<true> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const char* p) { a = *reinterpret_cast<const f32x4*>(p); b = *reinterpret_cast<const f32x4*>(p + 16); }
  __device__ __forceinline__ void load_once(const char* p) { load(p); }   // (two loads take turns in every line: through the caches)
  __device__ __forceinline__ void clear() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ Piece of_lane(int lane) const {
    Piece o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o.a[i] = __int_as_float(__builtin_amdgcn_ds_bpermute(4 * lane, __float_as_int(a[i])));
      o.b[i] = __int_as_float(__builtin_amdgcn_ds_bpermute(4 * lane, __float_as_int(b[i])));
    }
    return o;
  }
  template <bool kPastCaches>   // (a lane's two stores are half of a line each, which the caches put together)
  static __device__ __forceinline__ void store(char* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 16) = f32x4{v[4], v[5], v[6], v[7]};
  }
};

// Sum over the kLanes neighbouring lanes that share a head, in every one of them.
template <int kLanes>
__device__ __forceinline__ float head_sum(float v) {
  auto dpp = [](float x, auto ctrl_tag) {
    constexpr int ctrl = decltype(ctrl_tag)::value;
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, false));
  };
  v += dpp(v, std::integral_constant<int, 0xB1>{});                           // quad_perm [1, 0, 3, 2]
  v += dpp(v, std::integral_constant<int, 0x4E>{});                           // quad_perm [2, 3, 0, 1]
  v += dpp(v, std::integral_constant<int, 0x141>{});                          // row_half_mirror
  if constexpr (kLanes >= 16) v += dpp(v, std::integral_constant<int, 0x140>{});   // row_mirror
  if constexpr (kLanes == 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t s0 = s[0], s1 = s[1];
    v = __uint_as_float(s0) + __uint_as_float(s1);
  }
  return v;
}

// What a lane has to know of the rotation of its token: its eight channels' cosines and signed sines
// (z_d = y_d c_d + y_partner s_d; the transpose is dy_d = dz_d c_d - dz_partner s_d) and the lane that holds the partners.
template <bool kAdjacent>
struct Turn {
  float c[8], s[8];
  int partner;   // (halves) lane of the wave

  __device__ __forceinline__ Turn(const NormRopeArgs& a, int token, int lane, int sub, int& flag) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
    partner = lane;
    if (a.rotary_dim == 0) return;
    int pos = a.positions[token];
    if ((unsigned)pos >= (unsigned)a.max_positions) {
      flag = MARL_FLAG_BAD_POSITION;
      pos = pos < 0 ? 0 : a.max_positions - 1;
    }
    const int d = 8 * sub, half = a.rotary_dim >> 1;
    if (d >= a.rotary_dim) return;
    const float* row = a.cos_sin + (size_t)pos * a.rotary_dim;
    if constexpr (kAdjacent) {
      const f32x4 cv = *reinterpret_cast<const f32x4*>(row + (d >> 1)), sv = *reinterpret_cast<const f32x4*>(row + half + (d >> 1));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = cv[i >> 1];
        s[i] = i & 1 ? sv[i >> 1] : -sv[i >> 1];
      }
    } else {
      const bool second = d >= half;
      const float* at = row + (second ? d - half : d);
      const f32x4 c0 = *reinterpret_cast<const f32x4*>(at), c1 = *reinterpret_cast<const f32x4*>(at + 4);
      const f32x4 s0 = *reinterpret_cast<const f32x4*>(at + half), s1 = *reinterpret_cast<const f32x4*>(at + half + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float sv = i < 4 ? s0[i] : s1[i - 4];
        c[i] = i < 4 ? c0[i] : c1[i - 4];
        s[i] = second ? sv : -sv;
      }
      partner = second ? lane - half / 8 : lane + half / 8;
    }
  }
};

template <bool kF32>
__device__ __forceinline__ void load_weights(const void* w, int sub, float (&v)[8]) {
  Piece<kF32> p;
  if (w) p.load(static_cast<const char*>(w) + (size_t)sub * (kF32 ? 32 : 16));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = w ? p.at(i) : 1.f;
}

// Steps (64 * 8 / D heads each) of a token: first those of its queries, then those of its keys.
template <int D>
struct Steps {
  static constexpr int kHeads = 512 / D;
  int q, all;
  __device__ __forceinline__ explicit Steps(const NormRopeArgs& a) : q((a.Hq + kHeads - 1) / kHeads), all(q + (a.Hkv + kHeads - 1) / kHeads) {}
};

template <bool kF32, int D, bool kAdjacent, int kSteps, bool kPastCaches>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(NormRopeArgs a) {
  constexpr int kLanes = D / 8, kBytes = kF32 ? 4 : 2;
  const int lane = threadIdx.x & 63, sub = lane & (kLanes - 1), group = lane / kLanes;
  const Steps<D> steps(a);
  const int unit = blockIdx.x * kWavesPerBlock + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int token = unit / a.units_per_token, first = (unit - token * a.units_per_token) * kSteps;

  Piece<kF32> x[kSteps];
  auto head_of = [&](int step, bool& query, bool& there) {   // (query: wave-uniform)
    query = step < steps.q;
    const int h = (query ? step : step - steps.q) * Steps<D>::kHeads + group;
    there = step < steps.all && h < (query ? a.Hq : a.Hkv);
    return h;
  };
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    bool query, there;
    const int h = head_of(first + u, query, there);
    x[u].clear();
    if (there)
      x[u].load_once(static_cast<const char*>(query ? a.q : a.k) + ((size_t)token * (query ? a.q_stride : a.k_stride) + (size_t)h * D + 8 * sub) * kBytes);
  }
  int flag = 0;
  const Turn<kAdjacent> turn(a, token, lane, sub, flag);
  float A[8], B[8];
  auto factors = [&](const void* weight) {
    float w[8], wp[8];
    load_weights<kF32>(weight, sub, w);
    if constexpr (!kAdjacent) load_weights<kF32>(weight, turn.partner & (kLanes - 1), wp);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      A[i] = w[i] * turn.c[i];
      B[i] = (kAdjacent ? w[i ^ 1] : wp[i]) * turn.s[i];
    }
  };
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    bool query, there;
    const int h = head_of(first + u, query, there);
    if (first + u >= steps.all) break;                                       // wave-uniform
    if (u == 0 || first + u == steps.q) factors(query ? a.q_weight : a.k_weight);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[u].at(i), x[u].at(i), sum);
    const float r = rsqrtf(head_sum<kLanes>(sum) * (1.f / D) + a.eps);
    Piece<kF32> xp;
    if constexpr (!kAdjacent) xp = x[u].of_lane(turn.partner);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = r * __builtin_fmaf(x[u].at(i), A[i], (kAdjacent ? x[u].at(i ^ 1) : xp.at(i)) * B[i]);
    if (there)
      Piece<kF32>::template store<kPastCaches>(static_cast<char*>(query ? a.q_out : a.k_out) +
                         ((size_t)token * (query ? a.q_out_stride : a.k_out_stride) + (size_t)h * D + 8 * sub) * kBytes, z);
  }
  if (flag && a.flags) atomicOr(a.flags, flag);
}

// Backward.  The waves stay and take every so many-th unit, so that dw of the heads that a lane sees stays in its registers; a
// workgroup adds its waves' sums through LDS and leaves one row of 2 D numbers, which the second kernel adds in their order
// (no atomics: the same bits in every run).
template <bool kF32, int D, bool kAdjacent, int kSteps, bool kPastCaches>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_backward_kernel(NormRopeArgs a) {
  constexpr int kLanes = D / 8, kBytes = kF32 ? 4 : 2;
  __shared__ float sums[kWavesPerBlock][2][D];
  const int lane = threadIdx.x & 63, sub = lane & (kLanes - 1), group = lane / kLanes;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Steps<D> steps(a);
  float dwq[8] = {}, dwk[8] = {};
  int flag = 0;
  for (int unit = blockIdx.x * kWavesPerBlock + wave; unit < a.units; unit += gridDim.x * kWavesPerBlock) {   // wave-uniform
    const int token = unit / a.units_per_token, first = (unit - token * a.units_per_token) * kSteps;
    Piece<kF32> x[kSteps], dz[kSteps];
    auto head_of = [&](int step, bool& query, bool& there) {
      query = step < steps.q;
      const int h = (query ? step : step - steps.q) * Steps<D>::kHeads + group;
      there = step < steps.all && h < (query ? a.Hq : a.Hkv);
      return h;
    };
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      bool query, there;
      const int h = head_of(first + u, query, there);
      x[u].clear();
      dz[u].clear();
      if (there) {
        const size_t at = (size_t)h * D + 8 * sub;
        x[u].load_once(static_cast<const char*>(query ? a.q : a.k) + ((size_t)token * (query ? a.q_stride : a.k_stride) + at) * kBytes);
        dz[u].load_once(static_cast<const char*>(query ? a.dq_out : a.dk_out) + ((size_t)token * (query ? a.q_out_stride : a.k_out_stride) + at) * kBytes);
      }
    }
    const Turn<kAdjacent> turn(a, token, lane, sub, flag);
    float w[8];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      bool query, there;
      const int h = head_of(first + u, query, there);
      if (first + u >= steps.all) break;                                     // wave-uniform
      if (u == 0 || first + u == steps.q) load_weights<kF32>(query ? a.q_weight : a.k_weight, sub, w);
      Piece<kF32> dp;
      if constexpr (!kAdjacent) dp = dz[u].of_lane(turn.partner);
      float xx = 0.f, gx = 0.f, dy[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dy[i] = __builtin_fmaf(dz[u].at(i), turn.c[i], -(kAdjacent ? dz[u].at(i ^ 1) : dp.at(i)) * turn.s[i]);
        xx = __builtin_fmaf(x[u].at(i), x[u].at(i), xx);
        gx = __builtin_fmaf(dy[i] * w[i], x[u].at(i), gx);
      }
      const float r = there ? rsqrtf(head_sum<kLanes>(xx) * (1.f / D) + a.eps) : 0.f;   // (lanes without a head add nothing, eps 0 or not)
      const float along = head_sum<kLanes>(gx) * (1.f / D) * r * r;          // mean(g n) / r, n = x r
      float dx[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) dx[i] = r * __builtin_fmaf(-x[u].at(i), along, dy[i] * w[i]);
      if (query) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dwq[i] = __builtin_fmaf(dy[i], x[u].at(i) * r, dwq[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) dwk[i] = __builtin_fmaf(dy[i], x[u].at(i) * r, dwk[i]);
      }
      if (there)
        Piece<kF32>::template store<kPastCaches>(static_cast<char*>(query ? a.dq : a.dk) +
                           ((size_t)token * (query ? a.dq_stride : a.dk_stride) + (size_t)h * D + 8 * sub) * kBytes, dx);
    }
  }
  if (flag && a.flags) atomicOr(a.flags, flag);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int d = kLanes; d < 64; d <<= 1) {
      dwq[i] += __shfl_xor(dwq[i], d);
      dwk[i] += __shfl_xor(dwk[i], d);
    }
    if (group == 0) {
      sums[wave][0][8 * sub + i] = dwq[i];
      sums[wave][1][8 * sub + i] = dwk[i];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * D; e += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWavesPerBlock; ++k) v += sums[k][e / D][e % D];
    a.partials[(size_t)blockIdx.x * (2 * D) + e] = v;
  }
}

// dw of the queries (columns 0 .. D - 1) and of the keys: sums of the workgroups' rows, 16 columns a workgroup.  A thread requests
// eight rows before it adds the first (one after the other: 12 us for 1024 rows).
__global__ __launch_bounds__(kFinishThreads) void qk_norm_weight_grad_kernel(NormRopeArgs a, int rows, int D) {
  constexpr int kSlices = kFinishThreads / kFinishColumns, kAtOnce = 8;
  __shared__ float part[kSlices][kFinishColumns];
  const int c = threadIdx.x % kFinishColumns, column = blockIdx.x * kFinishColumns + c, slice = threadIdx.x / kFinishColumns;
  const float* from = a.partials + column;
  float sum[kAtOnce] = {};
  for (int r = slice; r < rows; r += kSlices * kAtOnce) {
    float v[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) v[u] = r + u * kSlices < rows ? from[(size_t)(r + u * kSlices) * (2 * D)] : 0.f;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) sum[u] += v[u];
  }
  part[slice][c] = ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
  __syncthreads();
  if (slice != 0) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < kSlices; ++k) v += part[k][c];
  float* out = column < D ? a.dq_weight : a.dk_weight;
  if (out) out[column < D ? column : column - D] = v;
}

// A wave's steps at once: four, where there are waves enough for the GPU's 256 CUs (eight: 177 instead of 180 us for 65543 tokens of 28
// + 4 heads of 128, two 161 instead of 151 for the gradient of 32771); few, where a call is small and waits for its loads.
constexpr int kManySteps = 4, kFewSteps = 2, kBackwardSteps = 4, kBackwardStepsF32 = 2;
constexpr long kEnoughUnits = 8192;
// bf16 results that the caches of the XCDs (4 MB each) cannot hold until somebody reads them are stored past them: 191 -> 180 us for the
// 65543 tokens, 162 -> 151 for the gradient of 32771.
constexpr long kCacheBytes = 32l << 20;
bool past_caches(const NormRopeArgs& a) { return !a.f32 && (long)a.T * (a.Hq + a.Hkv) * a.D * 2 > kCacheBytes; }

int steps_of(const NormRopeArgs& a) { const int heads = 512 / a.D; return (a.Hq + heads - 1) / heads + (a.Hkv + heads - 1) / heads; }

// Units of a forward call where a wave has `steps` steps at once.
long units_of(const NormRopeArgs& a, int steps) { return (long)a.T * ((steps_of(a) + steps - 1) / steps); }

template <bool kF32, int D, bool kAdjacent>
hipError_t launch_forward(NormRopeArgs a, hipStream_t st) {
  const long all = steps_of(a);
  const bool many = units_of(a, kManySteps) >= kEnoughUnits;
  const int steps = many ? kManySteps : kFewSteps;
  a.units_per_token = (int)((all + steps - 1) / steps);
  a.units = (int)((long)a.T * a.units_per_token);
  const dim3 grid((unsigned)((a.units + kWavesPerBlock - 1) / kWavesPerBlock));
  // (few steps: under 8192 units of four, so at most 32 MB in bf16)
  if (many && past_caches(a)) hipLaunchKernelGGL((qk_norm_rope_kernel<kF32, D, kAdjacent, kManySteps, !kF32>), grid, dim3(kThreads), 0, st, a);
  else if (many) hipLaunchKernelGGL((qk_norm_rope_kernel<kF32, D, kAdjacent, kManySteps, false>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<kF32, D, kAdjacent, kFewSteps, false>), grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

template <bool kF32, int D, bool kAdjacent>
hipError_t launch_backward(NormRopeArgs a, hipStream_t st) {
  constexpr int kSteps = kF32 ? kBackwardStepsF32 : kBackwardSteps;
  a.units_per_token = (steps_of(a) + kSteps - 1) / kSteps;
  a.units = (int)((long)a.T * a.units_per_token);
  const int blocks = std::min((a.units + kWavesPerBlock - 1) / kWavesPerBlock, kNormRopeMaxBlocks);
  if (blocks > 0) {
    if (past_caches(a)) hipLaunchKernelGGL((qk_norm_rope_backward_kernel<kF32, D, kAdjacent, kSteps, !kF32>), dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((qk_norm_rope_backward_kernel<kF32, D, kAdjacent, kSteps, false>), dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dq_weight && !a.dk_weight) return hipSuccess;
  hipLaunchKernelGGL(qk_norm_weight_grad_kernel, dim3(2 * D / kFinishColumns), dim3(kFinishThreads), 0, st, a, blocks, D);
  return hipGetLastError();
}

template <class F>
hipError_t by_type(const NormRopeArgs& a, F&& launch) {
  auto with_dim = [&](auto f32, auto adjacent) {
    switch (a.D) {
      case 64: return launch(f32, std::integral_constant<int, 64>{}, adjacent);
      case 128: return launch(f32, std::integral_constant<int, 128>{}, adjacent);
      default: return launch(f32, std::integral_constant<int, 256>{}, adjacent);
    }
  };
  auto with_pairs = [&](auto f32) { return a.adjacent ? with_dim(f32, std::true_type{}) : with_dim(f32, std::false_type{}); };
  return a.f32 ? with_pairs(std::true_type{}) : with_pairs(std::false_type{});
}

}  // namespace

bool qk_norm_rope_fits(const NormRopeArgs& a) { return units_of(a, kManySteps) <= most_workgroups(kThreads) * kWavesPerBlock; }

hipError_t launch_qk_norm_rope(const NormRopeArgs& a, hipStream_t st) {
  return by_type(a, [&](auto f32, auto dim, auto adjacent) {
    return launch_forward<decltype(f32)::value, decltype(dim)::value, decltype(adjacent)::value>(a, st);
  });
}

hipError_t launch_qk_norm_rope_backward(const NormRopeArgs& a, hipStream_t st) {
  return by_type(a, [&](auto f32, auto dim, auto adjacent) {
    return launch_backward<decltype(f32)::value, decltype(dim)::value, decltype(adjacent)::value>(a, st);
  });
}

}  // namespace marl
