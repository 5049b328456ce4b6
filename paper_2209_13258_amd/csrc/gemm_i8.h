// Products of 8-bit integers: Y[T x O] = bf16( (Xq . Wq^T) * s_t * s_o ), Xq [T x I] and Wq [O x I], both with the reduction contiguous.
#pragma once
#include <algorithm>

#include "osdp_internal.h"

namespace osdp {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Largest magnitude, as fp32 bits, of eight bf16 values (a NaN's is larger than any number's).
__device__ __forceinline__ uint32_t i8_largest(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m = max(m, max((w[j] << 16) & 0x7fff0000u, w[j] & 0x7fff0000u));
  return m;
}

// Four lower bytes side by side.
__device__ __forceinline__ uint32_t i8_pack(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// From the bits of a row's or column's largest magnitude: its scale and the rounding of its values to 8 bits.
struct I8Scale {
  float scale, up, r;
  __device__ __forceinline__ explicit I8Scale(uint32_t most) {
    const float amax = __uint_as_float(most);
    const bool number = most < 0x7f800000u;
    scale = number ? amax / 127.f : __uint_as_float(0x7fc00000u);
    up = amax < 0x1p-100f ? 0x1p100f : 1.f;  // (127 / amax would be no number; a power of two changes no quotient)
    r = number && most != 0u ? 127.f / (amax * up) * (1.f + 0x1p-21f) : 0.f;
  }
  __device__ __forceinline__ I8Scale(float ratio, float shift) : scale(0.f), up(shift), r(ratio) {}
  // Lower 8 bits.  A half with the number's sign is added and the fraction dropped; what is no number gives 0.
  __device__ __forceinline__ uint32_t round(float x) const {
    const float half = __uint_as_float((__float_as_uint(x) & 0x80000000u) | 0x3f000000u);
    const float t = fmaf(x * up, r, half);
    uint32_t q;  // (the instruction itself, which makes 0 of a NaN; to a cast in C++ that would be undefined)
    asm("v_cvt_i32_f32 %0, %1" : "=v"(q) : "v"(t));
    return q;
  }
  __device__ __forceinline__ uint2 round8(uint4 v) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = round(__uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16));
    return uint2{i8_pack(q[0], q[1], q[2], q[3]), i8_pack(q[4], q[5], q[6], q[7])};
  }
};

// Bytes from one row of Xq to the next: whole pieces of 128, which end in zeros.
constexpr int64_t i8_row_bytes(int64_t I) { return (I + 127) / 128 * 128; }

struct I8Problem {
  int32_t T, I, O, ldq;
  const uint8_t *xq;
  const float *x_scale;
  ShardTable shards;      // of Wq
  int64_t L;              // bytes of a shard
  int32_t rows_each;      // > 0: rows of Wq (output channels) to a shard; 0: rows may go on in the next shard
  const float *w_scale;
  uint16_t *y;
  int64_t ldy;
  void *sums;             // where parts of a reduction meet, and their counters, which are 0; NULL: nowhere
  uint32_t *arrived;
};

// Launches whose tiles do not fill the card share the reduction of a tile among workgroups (gemm_i8_w4.h), which meet in
// kI8SumBytes of memory with a counter for each of kI8MostTiles.
constexpr int64_t kI8MostTiles = 256;
constexpr size_t kI8SumBytes = 16 << 20;

// Up to kI8FewTokens the product reads the weight where it lies, however it is cut; from there on if every shard is
// a block of at least kI8ShardRows channels (tiles end with a shard); beyond kI8ManyTokens only if that is no slower than gathering.
constexpr int64_t kI8FewTokens = 64, kI8ShardRows = 32, kI8ManyTokens = 256;

// What the kernels for few tokens, of 512 threads for 16 channels, can be launched over: threads along a grid are counted in 32 bits.
constexpr int64_t kI8FewChannels = (int64_t{1} << 27) - 16;

// Eight sums as Y: both scales, then the rounding to bf16.
__device__ __forceinline__ void i8_store8(uint16_t *y, const int *sums, float st, const float *so) {
  uint32_t out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float lo = static_cast<float>(sums[2 * j]) * st * so[2 * j], hi = static_cast<float>(sums[2 * j + 1]) * st * so[2 * j + 1];
    out[j] = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) |
             static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
  }
  store_global16(y, uint4{out[0], out[1], out[2], out[3]});
}

// ---- few tokens -----------------------------------------------------------------------------------------------------
// One output channel's row of the weight.  kFlat: the row may go on in the next shard, and every piece of 16 bytes looks for its own.
template <bool kFlat>
struct I8Row {
  const uint8_t *row;
  const uint8_t *const *tab;
  int64_t off, L;
  int shard;
  __device__ __forceinline__ I8Row(const I8Problem &p, const uint8_t *const *shards, int o) : tab(shards), L(p.L) {
    if constexpr (kFlat) {
      const uint64_t f = static_cast<uint64_t>(o) * p.I;
      shard = static_cast<int>(f / static_cast<uint64_t>(p.L));
      off = static_cast<int64_t>(f - static_cast<uint64_t>(shard) * p.L);
    } else {
      shard = static_cast<int>(static_cast<uint32_t>(o) / static_cast<uint32_t>(p.rows_each));
      row = tab[shard] + static_cast<int64_t>(o - shard * p.rows_each) * p.I;
    }
  }
  __device__ __forceinline__ uint4 load(int k) const {
    if constexpr (!kFlat) return load_global16(row + k);
    int64_t f = off + k;
    int s = shard;
    while (f >= L) {
      f -= L;
      ++s;
    }
    return load_global16(tab[s] + f);
  }
};

// Rows of the weight that lie a multiple of 4 KB apart are asked for from the same few memory channels by all workgroups at a time, unless
// these begin at different places of the reduction and go round.
constexpr int kI8Turn = 4096;

// Where a workgroup of the kernels for few tokens begins, whose waves take kSpan bytes of a row together: 32 workgroups that follow one
// another, four to an XCD, at one place, the next 32 behind it.  One token, weight from memory: 4096 -> 16384 17.2 us, so 15.1; 8192 -> 32768 50.5
// and 47.0, 16384 -> 16384 55.4 and 53.3, 24576 -> 8192 46.5 and 42.2; where neighbours, which run on different XCDs, differ instead: 15.3, 54.5, 72.8 and 47.8.
template <int kSpan>
__device__ __forceinline__ int i8_first(int I) {
  return I % kI8Turn == 0 ? static_cast<int>(blockIdx.x >> 5) % ((I + kSpan - 1) / kSpan) * kSpan : 0;
}

// What the two kernels below have in common: a workgroup owns 16 output channels and 16 tokens; its kWaves waves share the
// reduction, 64 * kUnroll bytes of every row at a time, and add their sums up in LDS (integers: in any order).  Weights go from memory
// to registers, each lane 16 bytes of a row, the four lanes of a row 64 in sequence; nothing of them is used twice, so nothing is
// staged.  Both are bound by the weight's bytes.
//
// Tokens that are in 8 bits already.  4 tokens, 4096 -> 16384, rounded in a launch before it: 17.9 us in all with the weight from memory (3.7 TB/s), 22.4
// before workgroups began at different places.  Before that too, 32 or 64 channels to a
// workgroup, which read the tokens half or a quarter as often, took 22 and 25 us where 16 took 25 (16 tokens), but 20 to 31 instead of 15 for
// 10240 -> 2560, whose workgroups then leave half the card or more idle.
//
// MB: 16 * MB tokens to a workgroup, for rows of the weight that may run over the ends of shards, which no tile reads.  us by sixteens and with all
// tokens to a workgroup: 33 tokens 4096 -> 16392 in 16 shards 47.9 and 38.9, 64 tokens 8192 -> 32776 250 and 184, 48 tokens 16384 -> 4104 62.6 and 65.9.
template <int MB, int kWaves, int kUnroll, bool kFlat>
__global__ __launch_bounds__(kWaves * 64) void i8_few_kernel(I8Problem p) {
  constexpr int kStep = 64 * kUnroll, kSpan = kWaves * kStep;
  __shared__ const uint8_t *tab[OSDP_MAX_SHARDS];
  __shared__ int sums[MB * 16 * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, q4 = lane >> 4;
  if (tid < OSDP_MAX_SHARDS) tab[tid] = static_cast<const uint8_t *>(p.shards.p[tid]);
  for (int i = tid; i < MB * 16 * 16; i += kWaves * 64) sums[i] = 0;
  __syncthreads();
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MB);
  // (rows beyond the last repeat it; they are not stored)
  const I8Row<kFlat> weight(p, tab, min(n0 + l16, p.O - 1));
  const uint8_t *token[MB];
  i32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    token[b] = p.xq + static_cast<int64_t>(min(m0 + 16 * b + l16, p.T - 1)) * p.ldq;
    acc[b] = i32x4{0, 0, 0, 0};
  }
  auto step = [&](int k0) {
    uint4 w[kUnroll], x[kUnroll][MB];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = k0 + 64 * u + 16 * q4;
      w[u] = weight.load(k < p.I ? k : 0);  // beyond the row's end: any weights, the tokens are zeros there
#pragma unroll
      for (int b = 0; b < MB; ++b) x[u][b] = load_global16(token[b] + (k < p.ldq ? k : p.ldq - 16));
    }
    __builtin_amdgcn_sched_barrier(0);  // (all of them on their way before the first is waited for)
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        if (k0 + 64 * u + 16 * q4 >= p.ldq) x[u][b] = uint4{0u, 0u, 0u, 0u};
        acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w[u]), __builtin_bit_cast(i32x4, x[u][b]), acc[b], 0, 0, 0);
      }
  };
  const int first = i8_first<kSpan>(p.I);
  for (int k0 = first + wave * kStep; k0 < p.I; k0 += kSpan) step(k0);
  for (int k0 = wave * kStep; k0 < first; k0 += kSpan) step(k0);
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) atomicAdd(&sums[(16 * b + l16) * 16 + 4 * q4 + i], acc[b][i]);
  __syncthreads();
  if (tid < 32 * MB) {
    const int r = tid >> 1, c = (tid & 1) * 8, m = m0 + r, n = n0 + c;
    if (m < p.T && n < p.O) i8_store8(p.y + static_cast<int64_t>(m) * p.ldy + n, &sums[r * 16 + c], p.x_scale[m], p.w_scale + n);
  }
}

// The same with the tokens' rounding in the launch, for tokens of so few features that the bytes of 16 of them fit in LDS and
// that every workgroup may well round its 16 for itself: one launch instead of two, the first weights on their way meanwhile.
// One token, 4096 -> 16384, one call behind another: 15.1 us in one launch, 17.4 in two, with the weight from memory (4.4 TB/s); 12.5 and 15.4 from the
// last-level cache.
template <int kWaves, int kUnroll, bool kFlat>
__global__ __launch_bounds__(kWaves * 64) void i8_fused_kernel(I8Problem p, const uint16_t *__restrict__ x, int64_t ldx) {
  constexpr int kStep = 64 * kUnroll, kSpan = kWaves * kStep;
  extern __shared__ __attribute__((aligned(16))) uint8_t rows[];  // [T][ldq + 16]: 16 rows fall into 16 different bank groups
  __shared__ const uint8_t *tab[OSDP_MAX_SHARDS];
  __shared__ int sums[16 * 16];
  __shared__ uint32_t most[16][kWaves];
  __shared__ float scale[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, q4 = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16, pitch = p.ldq + 16, tokens = min(p.T - m0, 16);
  x += static_cast<int64_t>(m0) * ldx;
  if (tid < OSDP_MAX_SHARDS) tab[tid] = static_cast<const uint8_t *>(p.shards.p[tid]);
  for (int i = tid; i < 16 * 16; i += kWaves * 64) sums[i] = 0;
  __syncthreads();
  const I8Row<kFlat> weight(p, tab, min(n0 + l16, p.O - 1));
  auto load = [&](int k0, uint4 (&w)[kUnroll]) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = k0 + 64 * u + 16 * q4;
      w[u] = weight.load(k < p.I ? k : 0);  // beyond the row's end: any weights, the tokens are zeros there
    }
  };
  const int first = i8_first<kSpan>(p.I);
  uint4 w[kUnroll];
  load(first + wave * kStep, w);
  // tokens to 8 bits: a row to a wave, or (fewer tokens than waves) to as many waves as there are for it
  const int share = tokens >= kWaves ? 1 : kWaves / tokens, part = wave % share;
  for (int t = wave / share; t < tokens; t += kWaves / share) {
    uint32_t m = 0;
    for (int i = (part * 64 + lane) * 8; i < p.I; i += share * 512) m = max(m, i8_largest(load_global16(x + t * ldx + i)));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
    if (lane == 0) most[t][part] = m;
  }
  __syncthreads();
  for (int t = wave / share; t < tokens; t += kWaves / share) {
    uint32_t m = 0;
    for (int i = 0; i < share; ++i) m = max(m, most[t][i]);
    const I8Scale s(m);
    if (part == 0 && lane == 0) scale[t] = s.scale;
    for (int i = (part * 64 + lane) * 8; i < p.ldq; i += share * 512)
      *reinterpret_cast<uint2 *>(rows + t * pitch + i) = i < p.I ? s.round8(load_global16(x + t * ldx + i)) : uint2{0u, 0u};
  }
  __syncthreads();
  const uint8_t *token = rows + min(l16, tokens - 1) * pitch + 16 * q4;
  i32x4 acc = {0, 0, 0, 0};
  for (int at = first;;) {  // (the kSpan bytes that the waves are at)
    const int k0 = at + wave * kStep;
    at = at + kSpan < p.I ? at + kSpan : 0;
    uint4 next[kUnroll];
    if (at != first) load(at + wave * kStep, next);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (k0 + 64 * u >= p.I) break;
      const i32x4 a = *reinterpret_cast<const i32x4 *>(token + k0 + 64 * u);
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w[u]), a, acc, 0, 0, 0);
    }
    if (at == first) break;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) w[u] = next[u];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) atomicAdd(&sums[l16 * 16 + 4 * q4 + i], acc[i]);
  __syncthreads();
  if (tid < 32) {
    const int m = tid >> 1, c = (tid & 1) * 8, n = n0 + c;
    if (m < tokens && n < p.O) i8_store8(p.y + static_cast<int64_t>(m0 + m) * p.ldy + n, &sums[m * 16 + c], scale[m], p.w_scale + n);
  }
}

// (eight waves with 128 bytes of a row on their way in the one, 256 in the other: 4 or 16 waves, or 512 bytes, were within 3 % or slower)
hipError_t launch_fused(const I8Problem &p, const uint16_t *x, int64_t ldx, hipStream_t stream) {
  constexpr int kWaves = 8, kUnroll = 2;
  const unsigned lds = static_cast<unsigned>(std::min(p.T, 16) * (p.ldq + 16));
  const dim3 grid(static_cast<unsigned>((p.O + 15) / 16), static_cast<unsigned>((p.T + 15) / 16));
  if (p.rows_each > 0) hipLaunchKernelGGL((i8_fused_kernel<kWaves, kUnroll, false>), grid, dim3(kWaves * 64), lds, stream, p, x, ldx);
  else hipLaunchKernelGGL((i8_fused_kernel<kWaves, kUnroll, true>), grid, dim3(kWaves * 64), lds, stream, p, x, ldx);
  return hipGetLastError();
}

template <int MB, bool kFlat>
hipError_t launch_few(const I8Problem &p, hipStream_t stream) {
  constexpr int kWaves = 8, kUnroll = 4;
  const dim3 grid(static_cast<unsigned>((p.O + 15) / 16), static_cast<unsigned>((p.T + 16 * MB - 1) / (16 * MB)));
  hipLaunchKernelGGL((i8_few_kernel<MB, kWaves, kUnroll, kFlat>), grid, dim3(kWaves * 64), 0, stream, p);
  return hipGetLastError();
}
hipError_t launch_few(const I8Problem &p, hipStream_t stream) {
  static_assert(kI8FewTokens == 64, "rows that run over the ends of shards come with up to 64 tokens");
  if (p.rows_each > 0) return launch_few<1, false>(p, stream);
  if (p.T <= 16) return launch_few<1, true>(p, stream);
  if (p.T <= 32) return launch_few<2, true>(p, stream);
  if (p.T <= 48) return launch_few<3, true>(p, stream);
  return launch_few<4, true>(p, stream);
}

}  // namespace
}  // namespace osdp
