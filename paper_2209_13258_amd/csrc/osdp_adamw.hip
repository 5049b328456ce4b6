// AdamW over many tensors at once, the sum of squares of their gradients, and the values of moments in 8 bits.
//
// Everything here is one pass over memory with some arithmetic on the way.  Per element a step moves 28 bytes (bf16
// gradient, parameter written, fp32 master and moments), 16 with moments in 8 bits, 10 when there is no master copy either.
//
// A launch covers up to kBatch tensors, whose pointers travel by value in the kernel's arguments (nothing to allocate or
// upload, and a captured graph keeps them).  Tensors are cut into tiles of 2048 elements, one to a workgroup of 256 at a time: 8
// elements to a lane, so that a row of 16 lanes is one block of 128 that moments in 8 bits share a power of two over, and
// its largest magnitude is found without leaving the row (four DPP steps, no LDS, no barrier).
//
// What bounds it: memory with moments in fp32 (78.7 million elements, 2.2 GB: 402 us, 5.5 TB/s) and with a master copy and moments in 8
// bits (1.57 GB with their values read back: 283 us); without a master copy the 55 instructions that two codes, a random number and a
// rounded parameter cost an element keep the vector units as busy as its 10 bytes keep memory (201 million elements: 362 us, 5.6 TB/s).  More waves to a SIMD would have to spill: a bound of six costs 7 % there and 12 % with a master copy.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <limits>

#include "osdp_internal.h"

namespace osdp {
namespace {

constexpr int kThreads = 256;
constexpr int kPerLane = 8;
constexpr int kTile = kThreads * kPerLane;
constexpr int kBlock = 128;      // elements that share a power of two: kPerLane * 16 lanes
constexpr int kBatch = 56;       // tensors to a launch: 4 KB of kernel arguments
constexpr int64_t kMaxElements = int64_t{1} << 40;

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Tensor {
  const void *grad;
  void *param;
  float *master;
  void *m, *v;
  uint8_t *exps;
  int64_t n;
  float decay;          // weight_decay
};

struct Batch {
  Tensor t[kBatch];
  uint32_t end[kBatch]; // tiles of this and all earlier tensors of the batch
  uint64_t wide;        // bit i: tensor i is aligned for 16-byte accesses
  int32_t count;
  uint32_t first;       // place of t[0] in the caller's array
  uint32_t tiles;
  uint32_t run;         // tiles that a workgroup takes one after another
};

struct Step {
  double lr, beta1, beta2;
  int64_t step;
  const double *sumsq;
  const int64_t *step_device;
  const float *lr_device;
  double max_norm;
  uint32_t seed_lo, seed_hi;
  float b1, c1, b2, c2, eps;  // c: 1 - beta, taken in double
  float rate, root;           // lr / (1 - beta1^t) and 1 / sqrt(1 - beta2^t), where t and lr come from the host
};

enum Form { kMaster = 0, kBf16 = 1, kF32 = 2 };

// 32 bits stirred: multiplications by odd numbers and shifted sums without carry, each of them one to one.  The first number is 2^32 over the golden ratio
// (Knuth's multiplicative hashing); 0x2C1B3C6D and 0x297A2D39 were published by Chris Wellons, from a search for numbers that let every bit reach every other.
constexpr uint32_t kStir = 0x9E3779B1u;
__device__ __forceinline__ uint32_t stir(uint32_t x) {  // mix() behind its first product
  x ^= x >> 15;
  x *= 0x2C1B3C6Du;
  return x ^ (x >> 13);
}
__device__ __forceinline__ uint32_t mix(uint32_t x) { return stir(x * kStir); }

// base^n by squaring: the same in a kernel and on the host.
__host__ __device__ inline double power(double base, int64_t n) {
  double r = 1.0;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= base;
    base *= base;
  }
  return r;
}

// The tensor that a tile (the same in all lanes of a wave) belongs to: by halving, on the scalar unit.
__device__ __forceinline__ int tensor_of(const Batch &b, uint32_t tile) {
  int lo = 0, hi = b.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (tile < b.end[mid]) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// The same for sums of squares, which do little else: lane i holds the end of tensor i, and the ends that do not lie behind the tile are
// counted.  (The arguments come from memory when a launch begins, and halving waits for it up to six times: 20 small tensors 9.8 us, so
// 6.7.)  The step and the values, whose waves wait for more, are the slower for the register: 78.7 million elements with moments in fp32 407 us,
// with a held end 419; values of 201 million 200 and 207.
static_assert(kBatch <= 64, "a lane holds the end of a tensor");
struct Ends {
  uint32_t end;
  __device__ __forceinline__ explicit Ends(const Batch &b) {
    const int lane = threadIdx.x & 63;
    end = lane < b.count ? b.end[lane < kBatch ? lane : 0] : ~0u;
  }
  // *from: the tile's first element in it
  __device__ __forceinline__ int find(uint32_t tile, int64_t *from) const {
    const int i = __popcll(__ballot(tile >= end));
    const uint32_t start = i > 0 ? __builtin_amdgcn_readlane(end, i - 1) : 0u;
    *from = static_cast<int64_t>(tile - start) * kTile;
    return i;
  }
};

// Element j of the lane's eight: side by side where a tile is read 16 bytes at a time; otherwise the lanes of a row of 16
// take neighbouring elements, so that accesses of single elements still cover whole segments.  Either way a row is a block.
template <bool kWide>
__device__ __forceinline__ uint32_t element(int j) {
  const uint32_t row = (threadIdx.x & (kThreads - 1)) >> 4, lane = threadIdx.x & 15;
  return row * kBlock + (kWide ? lane * kPerLane + j : j * 16u + lane);
}

// A lane's eight elements as they lie in memory, asked for (load) apart from where they are taken to pieces (get), so that all of a
// tile's loads are on their way before the first of them is waited for.  Wide loads and stores are marked as used once: nothing here
// is touched again before far more than the caches hold has passed.  A step over 78.7 million elements with moments in fp32 took 407 us
// with the marks and 425 without, with moments in 8 bits 291 and 310; the sum of squares of 403 million 126 and 135.
// load_anywhere: 16 bytes at a time from any element on (global memory is read so at any address), and not marked, since neighbouring lanes meet
// in a cache line that would be fetched twice (sum of squares of 403 million fp32 values off by one element 257 us, marked 300).
template <class T, bool kWide>
struct Eight;

template <class T>
struct Eight<T, false> {
  T x[8];
  __device__ __forceinline__ void load(const void *p, int64_t at, uint32_t left) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = static_cast<const T *>(p)[at + min(element<false>(j), left - 1)];  // (no branches: all at once)
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = element<false>(j) < left ? x[j] : T{0};
  }
  __device__ __forceinline__ void get(float (&out)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 4) out[j] = x[j];
      else out[j] = __uint_as_float(static_cast<uint32_t>(x[j]) << 16);
    }
  }
  __device__ __forceinline__ void get(uint32_t (&out)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = static_cast<uint32_t>(x[j]);
  }
};

template <>
struct Eight<float, true> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void *p, int64_t at, uint32_t) {
    const f32x4 *q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at + element<true>(0));
    a = __builtin_nontemporal_load(q);
    b = __builtin_nontemporal_load(q + 1);
  }
  __device__ __forceinline__ void load_anywhere(const void *p, int64_t at) {
    typedef f32x4 Any __attribute__((aligned(4)));
    const Any *q = reinterpret_cast<const Any *>(static_cast<const float *>(p) + at + element<true>(0));
    a = q[0];
    b = q[1];
  }
  __device__ __forceinline__ void get(float (&out)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = a[j], out[4 + j] = b[j];
  }
};

template <>
struct Eight<uint16_t, true> {
  uint4 a;
  __device__ __forceinline__ void load(const void *p, int64_t at, uint32_t) {
    const osdp_u32x4 z = __builtin_nontemporal_load(reinterpret_cast<const osdp_u32x4 *>(static_cast<const uint16_t *>(p) + at + element<true>(0)));
    a = uint4{z[0], z[1], z[2], z[3]};
  }
  __device__ __forceinline__ void load_anywhere(const void *p, int64_t at) {
    typedef osdp_u32x4 Any __attribute__((aligned(2)));
    const osdp_u32x4 z = *reinterpret_cast<const Any *>(static_cast<const uint16_t *>(p) + at + element<true>(0));
    a = uint4{z[0], z[1], z[2], z[3]};
  }
  __device__ __forceinline__ void get(float (&out)[8]) const {  // bf16
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[2 * j] = __uint_as_float(w[j] << 16);
      out[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
};

template <>
struct Eight<uint8_t, true> {
  uint2 a;
  __device__ __forceinline__ void load(const void *p, int64_t at, uint32_t) {
    a = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(p) + at + element<true>(0));
  }
  __device__ __forceinline__ void get(uint32_t (&out)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[j] = (a.x >> (8 * j)) & 255u;
      out[4 + j] = (a.y >> (8 * j)) & 255u;
    }
  }
};

template <bool kWide>
__device__ __forceinline__ void store8(float *p, int64_t at, uint32_t left, const float (&x)[8]) {
  if constexpr (kWide) {
    f32x4 *q = reinterpret_cast<f32x4 *>(p + at + element<true>(0));
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, q);
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, q + 1);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (element<false>(j) < left) p[at + element<false>(j)] = x[j];
  }
}

// bf16 bit patterns in the upper halves of x
template <bool kWide>
__device__ __forceinline__ void store8(uint16_t *p, int64_t at, uint32_t left, const uint32_t (&x)[8]) {
  if constexpr (kWide) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (x[2 * j] >> 16) | (x[2 * j + 1] & 0xffff0000u);
    __builtin_nontemporal_store(osdp_u32x4{w[0], w[1], w[2], w[3]}, reinterpret_cast<osdp_u32x4 *>(p + at + element<true>(0)));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (element<false>(j) < left) p[at + element<false>(j)] = static_cast<uint16_t>(x[j] >> 16);
  }
}

// bytes, and the bits of low and high (four bytes each) besides
template <bool kWide>
__device__ __forceinline__ void store8(uint8_t *p, int64_t at, uint32_t left, const uint32_t (&x)[8], uint32_t low = 0, uint32_t high = 0) {
  if constexpr (kWide) {
    uint2 w = {low, high};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w.x |= x[j] << (8 * j);
      w.y |= x[4 + j] << (8 * j);
    }
    __builtin_nontemporal_store(osdp_u32x2{w.x, w.y}, reinterpret_cast<osdp_u32x2 *>(p + at + element<true>(0)));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (element<false>(j) < left) p[at + element<false>(j)] = static_cast<uint8_t>(x[j] | (j < 4 ? low : high) >> 8 * (j & 3));
  }
}

// Largest of a value over the 16 lanes of a row, in all of them.
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  auto turned = [](uint32_t v, auto ctrl) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = max(x, turned(x, std::integral_constant<int, 0x128>{}));  // row_ror:8, :4, :2, :1
  x = max(x, turned(x, std::integral_constant<int, 0x124>{}));
  x = max(x, turned(x, std::integral_constant<int, 0x122>{}));
  return max(x, turned(x, std::integral_constant<int, 0x121>{}));
}

// ---- moments in 8 bits: kTop is the largest exponent field (15: m, 31: v), kLow the least b -------------------------
// With its exponent field and fraction put where fp32 has them, a code is the value times a power of two; where the field
// is 0 fp32 reads them as it reads its own smallest numbers, which is what the format wants.  nan: a quiet NaN's bits for a block that is none, else 0.
template <int kTop>
__device__ __forceinline__ float decode(uint32_t code, uint32_t b, uint32_t nan) {
  const uint32_t placed = kTop == 15 ? static_cast<uint32_t>(static_cast<int32_t>(code << 24) >> 4) & 0x87f00000u : code << 20;
  return __builtin_amdgcn_ldexpf(__uint_as_float(placed | nan), static_cast<int>(b) - kTop);
}
__device__ __forceinline__ uint32_t nan_bits(uint32_t b) { return b == 255u ? 0x7fc00000u : 0u; }

// The power of two of a block whose largest magnitude has these bits: rounding up to 3 fraction bits may carry into the
// next binade, or (FLT_MAX) out of the numbers, like an infinity and a NaN, whatever its sign and payload.
template <int kLow>
__device__ __forceinline__ uint32_t block_exponent(uint32_t most) {
  return max((min(most, 0x7f800000u) + 0xfffffu) >> 23, static_cast<uint32_t>(kLow));
}

// Codes of eight values (magnitudes' bits) of a block, rounded with 16 random bits each, from bit kShift of h on.  Above the smallest
// binade the random bits are added below the last fraction bit and the sum is cut: a carry runs into the exponent as it should,
// and never beyond the block's own largest code.  A lane that has a value in the smallest binade (one in 10^4 of a bell curve's; zeros) takes
// the general way, which is three times as long: in units of its binade's step a magnitude is x in [0, 16), and x plus the fraction is cut.
// A block that is none (b = 255) has zeros for codes; true is returned where it has not.
template <int kTop, int kShift>
__device__ __forceinline__ bool encode8(const uint32_t (&size)[8], uint32_t b, const uint32_t (&h)[8], uint32_t (&code)[8]) {
  const uint32_t least = b - (kTop - 1);
  uint32_t smallest = size[0];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    smallest = min(smallest, size[j]);
    const uint32_t r = kShift ? (h[j] >> 12) & 0xffff0u : (h[j] & 0xffffu) << 4;
    code[j] = ((size[j] + r) >> 20) - (least - 1) * 8u;
  }
  const bool number = b != 255u;
  if (smallest < least << 23 || !number) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t e = max(size[j] >> 23, least);
      const float units = __builtin_amdgcn_ldexpf(__uint_as_float(size[j]), 130 - static_cast<int>(e));
      const uint32_t q = static_cast<uint32_t>(fmaf(static_cast<float>((h[j] >> kShift) & 0xffffu), 0x1p-16f, units));
      code[j] = (e - least) * 8u + q;
      if (kTop == 31) code[j] = max(code[j], min(size[j], 1u));  // (a positive v stays positive)
      if (!number) code[j] = 0u;
    }
  }
  return number;
}

// The upper bytes of four values: their signs, where codes have them, and other bits.
__device__ __forceinline__ uint32_t signs_of(const float *m) {
  const uint32_t low = __builtin_amdgcn_perm(__float_as_uint(m[1]), __float_as_uint(m[0]), 0x0c0c0703u);
  const uint32_t high = __builtin_amdgcn_perm(__float_as_uint(m[3]), __float_as_uint(m[2]), 0x07030c0cu);
  return low | high;
}

struct Scalars {
  float coef, rate, root, lr;
  uint32_t key;
};

// m and v as the formulas have them, every operation rounded by itself.
__device__ __forceinline__ void moments(const Step &s, float coef, float grad, float &m, float &v) {
#pragma clang fp contract(off)
  const float g = grad * coef;
  const float mb = m * s.b1, gc = g * s.c1, vb = v * s.b2, gg = (g * g) * s.c2;
  m = mb + gc;
  v = vb + gg;
}

template <class Grad, int kForm, bool kState8, bool kWide>
__device__ __forceinline__ void adamw_tile(const Tensor &t, const Step &s, const Scalars &k, int64_t at) {
  const int64_t rest = t.n - at;
  const uint32_t left = rest < kTile ? static_cast<uint32_t>(rest) : kTile;
  using State = std::conditional_t<kState8, uint8_t, float>;
  using Source = std::conditional_t<kForm == kBf16, uint16_t, float>;
  Eight<Grad, kWide> grad;
  Eight<Source, kWide> source;
  Eight<State, kWide> old_m, old_v;
  // the block's two powers; of a short last tile only those of blocks that there are
  uint16_t *const exps = reinterpret_cast<uint16_t *>(t.exps) + at / kBlock + (threadIdx.x >> 4);
  const bool block = kWide || (threadIdx.x >> 4) * kBlock < left;
  uint32_t shared = 0;
  old_m.load(t.m, at, left);
  old_v.load(t.v, at, left);
  if (kState8 && block) shared = *exps;
  grad.load(t.grad, at, left);
  source.load(kForm == kMaster ? static_cast<const void *>(t.master) : t.param, at, left);
  float g[8], p[8], m[8], v[8];
  uint32_t cm[8], cv[8];
  if constexpr (kState8) {
    old_m.get(cm);
    old_v.get(cv);
    const uint32_t bm = shared & 255u, bv = shared >> 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = decode<15>(cm[j], bm, nan_bits(bm));
      v[j] = decode<31>(cv[j], bv, nan_bits(bv));
    }
  } else {
    old_m.get(m);
    old_v.get(v);
  }
  grad.get(g);
  source.get(p);
  const float decay = k.lr * t.decay;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    moments(s, k.coef, g[j], m[j], v[j]);
    // (both approximations are within an ulp; the root of a number below fp32's normal range, 1e-19, is nothing beside eps)
    const float size = fmaf(__builtin_amdgcn_sqrtf(v[j]), k.root, s.eps);
    p[j] -= fmaf(m[j] * k.rate, __builtin_amdgcn_rcpf(size), decay * p[j]);
  }
  uint32_t h[8];
  if constexpr (kState8 || kForm == kBf16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = stir((k.key + static_cast<uint32_t>(at) + element<kWide>(0)) * kStir + static_cast<uint32_t>(kWide ? j : 16 * j) * kStir);
  }
  if constexpr (kState8) {
    uint32_t sm[8], sv[8], most_m = 0, most_v = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (!kWide && element<kWide>(j) >= left) m[j] = v[j] = 0.f;  // (0 * beta is NaN where the block was)
      sm[j] = __float_as_uint(m[j]) & 0x7fffffffu;
      sv[j] = __float_as_uint(v[j]);  // (no sign, but of a NaN)
      most_m = max(most_m, sm[j]);
      most_v = max(most_v, sv[j]);
    }
    most_m = row_max(most_m);
    most_v = row_max(most_v);
    const uint32_t bm = block_exponent<32>(most_m), bv = block_exponent<48>(most_v);
    const uint32_t signs = encode8<15, 0>(sm, bm, h, cm) ? 0x80808080u : 0u;
    encode8<31, 16>(sv, bv, h, cv);
    if ((threadIdx.x & 15) == 0 && block)
      *exps = static_cast<uint16_t>((most_m ? bm : 0u) | (most_v ? bv << 8 : 0u));
    store8<kWide>(static_cast<uint8_t *>(t.m), at, left, cm, signs_of(m) & signs, signs_of(m + 4) & signs);
    store8<kWide>(static_cast<uint8_t *>(t.v), at, left, cv);
  } else {
    store8<kWide>(static_cast<float *>(t.m), at, left, m);
    store8<kWide>(static_cast<float *>(t.v), at, left, v);
  }
  if constexpr (kForm == kMaster) store8<kWide>(t.master, at, left, p);
  if constexpr (kForm == kF32) {
    store8<kWide>(static_cast<float *>(t.param), at, left, p);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // without a master copy to one of its neighbours, the one above with the probability that keeps the mean (an infinity
      // keeps its upper half whatever is added, and so does a NaN whose lower half is 0, as any is that comes from bf16, from a
      // block or from the rate; another might not)
      if constexpr (kForm == kMaster) w[j] = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(p[j]))) << 16;
      else w[j] = __float_as_uint(p[j]) + ((kState8 && sizeof(Grad) == 2) || p[j] == p[j] ? (h[j] * 0x297A2D39u) >> 16 : 0u);
    }
    store8<kWide>(static_cast<uint16_t *>(t.param), at, left, w);
  }
}

// The number, or a NaN whose lower half is 0 for any NaN: what is rounded stochastically counts on that.
__device__ __forceinline__ float with_plain_nan(float x) {
  const uint32_t w = __float_as_uint(x);
  return __uint_as_float((w & 0x7fffffffu) > 0x7f800000u ? 0x7fc00000u : w);
}

// Scalars of a call: one for all lanes.
__device__ __forceinline__ bool scalars_of(const Step &s, Scalars *k) {
  k->coef = 1.f;
  if (s.sumsq) {
    const double sum = *s.sumsq;
    if (!(sum < std::numeric_limits<double>::infinity())) return false;  // (NaN too)
    if (s.max_norm > 0.0) {
      // (1 / sqrt(sum) to some 50 bits, by two steps of Newton's from the instruction's 23 or more, which every wave works out for
      // itself: a division and a root in double take three times the instructions)
      if (sum > s.max_norm * s.max_norm) {
        double y = __builtin_amdgcn_rsq(sum);
#pragma unroll
        for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-(sum * y), y, 1.0), y);
        k->coef = static_cast<float>(s.max_norm * y);
      }
    }
  }
  k->rate = s.rate;
  k->root = s.root;
  k->lr = static_cast<float>(s.lr);
  int64_t step = s.step;
  if (s.step_device || s.lr_device) {
    const double lr = s.lr_device ? static_cast<double>(with_plain_nan(*s.lr_device)) : s.lr;
    if (s.step_device) step = *s.step_device;
    if (step < 1) step = 1;
    k->lr = static_cast<float>(lr);
    k->rate = static_cast<float>(lr / (1.0 - power(s.beta1, step)));
    k->root = static_cast<float>(1.0 / sqrt(1.0 - power(s.beta2, step)));
  }
  k->key = mix(mix(mix(s.seed_lo) ^ s.seed_hi) ^ static_cast<uint32_t>(step));
  return true;
}

template <class Grad, int kForm, bool kState8>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Batch b, Step s) {
  Scalars k;
  if (!scalars_of(s, &k)) return;
  const uint32_t stirred = k.key;
  for (uint32_t first = blockIdx.x * b.run; first < b.tiles; first += gridDim.x * b.run) {
    const uint32_t end = min(first + b.run, b.tiles);
    for (uint32_t tile = first; tile < end; ++tile) {
      const int i = tensor_of(b, tile);
      const Tensor t = b.t[i];
      const int64_t at = static_cast<int64_t>(tile - (i > 0 ? b.end[i - 1] : 0u)) * kTile;
      k.key = mix(mix(stirred ^ (b.first + static_cast<uint32_t>(i))) ^ static_cast<uint32_t>(at >> 32));
      if (((b.wide >> i) & 1u) && t.n - at >= kTile) adamw_tile<Grad, kForm, kState8, true>(t, s, k, at);
      else adamw_tile<Grad, kForm, kState8, false>(t, s, k, at);
    }
  }
}

template <bool kWide>
__device__ __forceinline__ void values_tile(const Tensor &t, int64_t at) {
  const int64_t rest = t.n - at;
  const uint32_t left = rest < kTile ? static_cast<uint32_t>(rest) : kTile;
  uint32_t shared = 0, cm[8], cv[8], wm[8], wv[8];
  Eight<uint8_t, kWide> m, v;
  m.load(t.m, at, left);
  v.load(t.v, at, left);
  if (kWide || (threadIdx.x >> 4) * kBlock < left) shared = reinterpret_cast<const uint16_t *>(t.exps)[at / kBlock + (threadIdx.x >> 4)];
  m.get(cm);
  v.get(cv);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    wm[j] = __float_as_uint(decode<15>(cm[j], shared & 255u, nan_bits(shared & 255u)));
    wv[j] = __float_as_uint(decode<31>(cv[j], shared >> 8, nan_bits(shared >> 8)));
  }
  store8<kWide>(static_cast<uint16_t *>(t.param), at, left, wm);                          // (m's values)
  store8<kWide>(reinterpret_cast<uint16_t *>(t.master), at, left, wv);                    // (v's values)
}

__global__ __launch_bounds__(kThreads) void values_kernel(Batch b) {
  for (uint32_t tile = blockIdx.x; tile < b.tiles; tile += gridDim.x) {
    const int i = tensor_of(b, tile);
    const int64_t at = static_cast<int64_t>(tile - (i > 0 ? b.end[i - 1] : 0u)) * kTile;
    const Tensor t = b.t[i];
    if (((b.wide >> i) & 1u) && t.n - at >= kTile) values_tile<true>(t, at);
    else values_tile<false>(t, at);
  }
}

// ---- sum of squares -------------------------------------------------------------------------------------------
// Squares and sums are in double from the first product on (a bf16 gradient of 1e20 is one, its square in fp32 is not): the
// vector unit multiplies and adds them as fast as fp32, and the pass stays bound by memory.
constexpr int kSumBlocks = 1024;  // workgroups, and so partial sums, of a launch at most
constexpr int kSumTiles = 4;      // tiles that a workgroup has on their way at a time, where there are enough for all: 806 MB in 123 us
                                  // (6.6 TB/s); one tile at a time takes half as long again

template <int kThreads = osdp::kThreads>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[kThreads / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) sum += part[w];
  return sum;
}

// A lane's eight elements of a tile, which ones depending on the tile's length alone, not on where the tensor lies: the same gradients are summed
// in the same order in tensors of their own and packed side by side.
template <class Grad>
__device__ __forceinline__ void load_tile(const Tensor &t, int64_t from, bool wide, float (&g)[8]) {
  const int64_t rest = t.n - from;
  if (rest >= kTile) {
    Eight<Grad, true> x;
    if (wide) x.load(t.grad, from, kTile);
    else x.load_anywhere(t.grad, from);
    x.get(g);
  } else {
    Eight<Grad, false> x;
    x.load(t.grad, from, static_cast<uint32_t>(rest));
    x.get(g);
  }
}

// Tiles in runs of kSumTiles, or alone, one run after another to the workgroups.
template <class Grad>
__global__ __launch_bounds__(kThreads) void sumsq_kernel(Batch b, uint32_t run, double *__restrict__ out) {
  double sum = 0.0;
  auto add = [&](const float (&g)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fma(static_cast<double>(g[j]), static_cast<double>(g[j]), sum);
  };
  const Ends ends(b);
  for (uint32_t first = blockIdx.x * run; first < b.tiles; first += gridDim.x * run) {
    const uint32_t end = min(first + run, b.tiles);
    int64_t at;
    int i = ends.find(first, &at);
    float g[8];
    if (run == kSumTiles && first + kSumTiles <= b.tiles && ((b.wide >> i) & 1u) && b.t[i].n - at >= kSumTiles * kTile) {
      Eight<Grad, true> x[kSumTiles];
#pragma unroll
      for (int u = 0; u < kSumTiles; ++u) x[u].load(b.t[i].grad, at + u * kTile, kTile);
#pragma unroll
      for (int u = 0; u < kSumTiles; ++u) {
        x[u].get(g);
        add(g);
      }
      continue;
    }
    for (uint32_t tile = first; tile < end; ++tile) {
      int64_t from;
      i = ends.find(tile, &from);
      load_tile<Grad>(b.t[i], from, (b.wide >> i) & 1u, g);
      add(g);
    }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) out[blockIdx.x] = sum;
}

// All tiles of a small batch by one workgroup of four times the size, which has the sum itself: one launch instead of two.
constexpr int kSmallThreads = 4 * kThreads;
template <class Grad>
__global__ __launch_bounds__(kSmallThreads) void sumsq_small_kernel(Batch b, int32_t accumulate, double *__restrict__ out) {
  const Ends ends(b);
  double sum = 0.0;
  for (uint32_t first = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads); first < b.tiles; first += 4 * kSumTiles) {
    float g[kSumTiles][8];
#pragma unroll
    for (int u = 0; u < kSumTiles; ++u) {
      const uint32_t tile = min(first + 4 * u, b.tiles - 1);
      int64_t from;
      const int i = ends.find(tile, &from);
      load_tile<Grad>(b.t[i], from, (b.wide >> i) & 1u, g[u]);
    }
#pragma unroll
    for (int u = 0; u < kSumTiles; ++u)
      if (first + 4 * u < b.tiles) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma(static_cast<double>(g[u][j]), static_cast<double>(g[u][j]), sum);
      }
  }
  sum = block_sum<kSmallThreads>(sum);
  if (threadIdx.x == 0) *out = accumulate ? *out + sum : sum;
}

__global__ __launch_bounds__(kThreads) void sumsq_finish_kernel(const double *__restrict__ part, int32_t count, int32_t accumulate,
                                                                double *__restrict__ out) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < count; i += 4 * kThreads) {
    double x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = part[min(i + j * kThreads, count - 1)];  // (all four on their way at once)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += i + j * kThreads < count ? x[j] : 0.0;
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) *out = accumulate ? *out + sum : sum;
}

// ---- host ---------------------------------------------------------------------------------------------------
osdp_status fail(osdp_status st, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return report_error(st, buf);
}

osdp_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return OSDP_OK;
  return fail(OSDP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

osdp_status device_ok() {
  const hipError_t e = check_device();
  if (e == hipErrorInvalidDevice)
    return fail(OSDP_ERR_UNSUPPORTED, "the current device is not an MI355X (256 compute units in 8 XCDs), which the kernels are written for");
  return hip_status(e, "querying the device");
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

osdp_status check_count(const osdp_adamw_tensor *tensors, int32_t count) {
  if (count < 0) return fail(OSDP_ERR_INVALID_ARG, "count must be >= 0 (got %d)", count);
  if (count > 0 && !tensors) return fail(OSDP_ERR_INVALID_ARG, "tensors is NULL");
  for (int32_t i = 0; i < count; ++i)
    if (tensors[i].n < 0 || tensors[i].n >= kMaxElements)
      return fail(OSDP_ERR_INVALID_ARG, "tensors[%d] has %lld elements: 0 to 2^40 - 1 are possible", i, (long long)tensors[i].n);
  return OSDP_OK;
}

osdp_status check_array(const void *p, size_t align, int32_t i, const char *name) {
  if (!p) return fail(OSDP_ERR_INVALID_ARG, "tensors[%d].%s is NULL", i, name);
  if (!aligned(p, align)) return fail(OSDP_ERR_UNSUPPORTED, "tensors[%d].%s is not %zu-byte aligned", i, name, align);
  return OSDP_OK;
}

size_t size_of(int32_t type) { return type == OSDP_BF16 ? 2 : 4; }

// Calls launch(batch) for the tensors that have elements, up to kBatch at a time and at most `most` tiles where more would not
// do; fill(i, &tensor) sets what the kernel reads and says whether it may use 16-byte accesses.
template <class Fill, class Launch>
osdp_status for_batches(const osdp_adamw_tensor *tensors, int32_t count, Fill &&fill, Launch &&launch) {
  Batch b;
  b.count = 0; b.tiles = 0; b.wide = 0; b.run = 1;
  int32_t last = -1;  // place of the batch's last tensor: places within a batch are consecutive
  auto flush = [&]() -> osdp_status {
    if (b.count == 0) return OSDP_OK;
    const osdp_status st = launch(b);
    b.count = 0; b.tiles = 0; b.wide = 0;
    return st;
  };
  for (int32_t i = 0; i < count; ++i) {
    if (tensors[i].n == 0) continue;
    const uint64_t tiles = (static_cast<uint64_t>(tensors[i].n) + kTile - 1) / kTile;  // < 2^29
    if (b.count == kBatch || b.tiles + tiles >= (1ull << 31) || (b.count > 0 && i != last + 1)) {
      const osdp_status st = flush();
      if (st != OSDP_OK) return st;
    }
    if (b.count == 0) b.first = static_cast<uint32_t>(i);
    Tensor &t = b.t[b.count];
    t = Tensor{};
    t.n = tensors[i].n;
    if (fill(i, &t)) b.wide |= 1ull << b.count;
    b.tiles += static_cast<uint32_t>(tiles);
    b.end[b.count] = b.tiles;
    ++b.count;
    last = i;
  }
  return flush();
}

constexpr unsigned kMostBlocks = 1u << 20;
unsigned grid_of(const Batch &b, uint32_t run) { return std::min<unsigned>((b.tiles + run - 1) / run, kMostBlocks); }

template <class Grad, int kForm, bool kState8>
hipError_t launch_adamw(const Batch &b, const Step &s, hipStream_t stream) {
  // Every wave works the call's scalars out for itself, 40 to 250 operations.  Where arithmetic is the bound and there are workgroups enough
  // (from 6144 tiles on; fewer leave compute units idle at the end), one takes four tiles, so that they weigh less: 201 million elements in
  // 375 us, with the step on the device 406, one tile to a workgroup 458 and 535 (359 and 380 since codes take fewer operations).  The other forms are bound by memory and are the
  // slower for it (78.7 million elements, master copy: moments in 8 bits 312 us instead of 291, in fp32 425 instead of 402).
  // With moments in fp32 a launch asks for LDS that it does not use, so that no more than two workgroups run on a compute unit, or three where
  // the scalars, and with them the wait before a tile's loads, are longer (step or rate on the device): their loads keep memory busy, and
  // with more of them its reads and writes, to eight arrays, get in one another's way.  us with eight / three / two workgroups, and with the step on
  // the device: 201 million elements with master copies 1069 / 1035 / 992 and 1074 / 1028 / 1138, bf16 alone 947 / 846 / 809 and 945 / 828 / 949, fp32
  // parameters 983 / 951 / 921 and 986 / 937 / 1066; 78.7 million with master copies 415 / 403 / 402, 6.3 million 35 / 34 / 34 and 37 / 36 / 41.
  // With moments in 8 bits the arithmetic needs the five that registers leave room for.
  const unsigned lds = kState8 ? 0 : s.step_device || s.lr_device ? 52 << 10 : 64 << 10;
  Batch batch = b;
  batch.run = kForm == kBf16 && kState8 && b.tiles >= 6144 ? 4 : 1;
  hipLaunchKernelGGL((adamw_kernel<Grad, kForm, kState8>), dim3(grid_of(batch, batch.run)), dim3(kThreads), lds, stream, batch, s);
  return hipGetLastError();
}

template <class Grad>
hipError_t launch_adamw(int form, bool state8, const Batch &b, const Step &s, hipStream_t stream) {
  if (form == kMaster) return state8 ? launch_adamw<Grad, kMaster, true>(b, s, stream) : launch_adamw<Grad, kMaster, false>(b, s, stream);
  if (form == kBf16) return state8 ? launch_adamw<Grad, kBf16, true>(b, s, stream) : launch_adamw<Grad, kBf16, false>(b, s, stream);
  return state8 ? launch_adamw<Grad, kF32, true>(b, s, stream) : launch_adamw<Grad, kF32, false>(b, s, stream);
}

// Workgroups, and so partial sums, of the launch over a batch.
// A call of so few tiles, in one batch, is the small kernel's, at 16 tiles a round: us captured / called 32 tiles 4.7 / 4.8, two launches 4.4 / 7.1; 48 tiles 6.0 / 6.1
// and 4.4 / 7.0.
constexpr uint32_t kSmallTiles = 32;
uint32_t sum_run(const Batch &b) { return b.tiles >= kSumTiles * kSumBlocks ? kSumTiles : 1; }
unsigned sum_blocks(const Batch &b) { return std::min<unsigned>(b.tiles, kSumBlocks); }

// Partial sums of a call, and whether it is a small one.
osdp_status sumsq_parts(const osdp_adamw_tensor *tensors, int32_t count, int64_t *parts, bool *small) {
  *parts = 0;
  *small = false;
  int batches = 0;
  return for_batches(tensors, count, [](int32_t, Tensor *) { return false; }, [&](const Batch &b) {
    *parts += sum_blocks(b);
    *small = ++batches == 1 && b.tiles <= kSmallTiles;
    return OSDP_OK;
  });
}

}  // namespace
}  // namespace osdp

using namespace osdp;

extern "C" {

osdp_status osdp_adamw_step(const osdp_adamw_tensor *tensors, int32_t count, const osdp_adamw_options *o, void *stream) {
  osdp_status st = check_count(tensors, count);
  if (st != OSDP_OK) return st;
  if (!o) return fail(OSDP_ERR_INVALID_ARG, "options is NULL");
  if (o->grad_type != OSDP_BF16 && o->grad_type != OSDP_F32) return fail(OSDP_ERR_INVALID_ARG, "unknown grad_type %d", o->grad_type);
  if (o->param_type != OSDP_BF16 && o->param_type != OSDP_F32) return fail(OSDP_ERR_INVALID_ARG, "unknown param_type %d", o->param_type);
  if (o->state_bits != 32 && o->state_bits != 8) return fail(OSDP_ERR_INVALID_ARG, "state_bits must be 32 or 8 (got %d)", o->state_bits);
  if (!(o->lr >= 0.0) || !std::isfinite(o->lr)) return fail(OSDP_ERR_INVALID_ARG, "lr must be a number >= 0");
  if (!(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0))
    return fail(OSDP_ERR_INVALID_ARG, "beta1 and beta2 must lie in [0, 1)");
  if (!(o->eps >= 1e-12) || !(o->eps <= 1e30)) return fail(OSDP_ERR_INVALID_ARG, "eps must be at least 1e-12");
  if (!o->step_device && o->step < 1) return fail(OSDP_ERR_INVALID_ARG, "step must be >= 1 (got %lld)", (long long)o->step);
  if (!(o->max_norm >= 0.0)) return fail(OSDP_ERR_INVALID_ARG, "max_norm must be >= 0");
  if (o->max_norm > 0.0 && !o->grad_sumsq) return fail(OSDP_ERR_INVALID_ARG, "max_norm needs grad_sumsq");
  if (!aligned(o->grad_sumsq, 8) || !aligned(o->step_device, 8) || !aligned(o->lr_device, 4))
    return fail(OSDP_ERR_UNSUPPORTED, "grad_sumsq, step_device or lr_device is not aligned to its type");
  const bool state8 = o->state_bits == 8;
  int form = -1;
  for (int32_t i = 0; i < count; ++i) {
    const osdp_adamw_tensor &t = tensors[i];
    if (t.n == 0) continue;
    if ((st = check_array(t.grad, size_of(o->grad_type), i, "grad")) != OSDP_OK) return st;
    if ((st = check_array(t.param, size_of(o->param_type), i, "param")) != OSDP_OK) return st;
    if ((st = check_array(t.m, state8 ? 1 : 4, i, "m")) != OSDP_OK) return st;
    if ((st = check_array(t.v, state8 ? 1 : 4, i, "v")) != OSDP_OK) return st;
    if (state8 && (st = check_array(t.exps, 2, i, "exps")) != OSDP_OK) return st;
    if (t.master && (st = check_array(t.master, 4, i, "master")) != OSDP_OK) return st;
    if (!(t.weight_decay >= 0.0) || !std::isfinite(t.weight_decay)) return fail(OSDP_ERR_INVALID_ARG, "tensors[%d].weight_decay must be a number >= 0", i);
    const int f = o->param_type == OSDP_F32 ? kF32 : (t.master ? kMaster : kBf16);
    if (f == kF32 && t.master) return fail(OSDP_ERR_INVALID_ARG, "tensors[%d] has a master copy of fp32 parameters", i);
    if (form >= 0 && f != form) return fail(OSDP_ERR_INVALID_ARG, "some of the tensors have masters and some have none");
    form = f;
  }
  if ((st = device_ok()) != OSDP_OK) return st;
  Step s{};
  s.lr = o->lr; s.beta1 = o->beta1; s.beta2 = o->beta2;
  s.step = o->step_device ? 1 : o->step;
  s.sumsq = o->grad_sumsq; s.step_device = o->step_device; s.lr_device = o->lr_device;
  s.max_norm = o->max_norm;
  s.seed_lo = static_cast<uint32_t>(o->seed); s.seed_hi = static_cast<uint32_t>(o->seed >> 32);
  s.b1 = static_cast<float>(o->beta1); s.c1 = static_cast<float>(1.0 - o->beta1);
  s.b2 = static_cast<float>(o->beta2); s.c2 = static_cast<float>(1.0 - o->beta2);
  s.eps = static_cast<float>(o->eps);
  s.rate = static_cast<float>(o->lr / (1.0 - power(o->beta1, s.step)));
  s.root = static_cast<float>(1.0 / std::sqrt(1.0 - power(o->beta2, s.step)));
  return for_batches(
      tensors, count,
      [&](int32_t i, Tensor *t) {
        const osdp_adamw_tensor &u = tensors[i];
        t->grad = u.grad; t->param = u.param; t->master = u.master; t->m = u.m; t->v = u.v; t->exps = u.exps;
        t->decay = static_cast<float>(u.weight_decay);
        const size_t state = state8 ? 8 : 16;
        return aligned(u.grad, 16) && aligned(u.param, 16) && aligned(u.master, 16) && aligned(u.m, state) && aligned(u.v, state);
      },
      [&](const Batch &b) {
        const hipStream_t q = static_cast<hipStream_t>(stream);
        return hip_status(o->grad_type == OSDP_BF16 ? launch_adamw<uint16_t>(form, state8, b, s, q) : launch_adamw<float>(form, state8, b, s, q),
                          "launching the step");
      });
}

osdp_status osdp_adamw_grad_sumsq_workspace_bytes(const osdp_adamw_tensor *tensors, int32_t count, size_t *bytes) {
  osdp_status st = check_count(tensors, count);
  if (st != OSDP_OK) return st;
  if (!bytes) return fail(OSDP_ERR_INVALID_ARG, "bytes is NULL");
  int64_t parts = 0;
  bool small = false;
  if ((st = sumsq_parts(tensors, count, &parts, &small)) != OSDP_OK) return st;
  *bytes = static_cast<size_t>(parts) * sizeof(double);
  return OSDP_OK;
}

osdp_status osdp_adamw_grad_sumsq(const osdp_adamw_tensor *tensors, int32_t count, int32_t grad_type, int32_t accumulate,
                                  double *sumsq, void *workspace, size_t workspace_bytes, void *stream) {
  osdp_status st = check_count(tensors, count);
  if (st != OSDP_OK) return st;
  if (grad_type != OSDP_BF16 && grad_type != OSDP_F32) return fail(OSDP_ERR_INVALID_ARG, "unknown grad_type %d", grad_type);
  if (!sumsq) return fail(OSDP_ERR_INVALID_ARG, "sumsq is NULL");
  if (!aligned(sumsq, 8)) return fail(OSDP_ERR_UNSUPPORTED, "sumsq is not 8-byte aligned");
  for (int32_t i = 0; i < count; ++i)
    if (tensors[i].n > 0 && (st = check_array(tensors[i].grad, size_of(grad_type), i, "grad")) != OSDP_OK) return st;
  int64_t parts = 0;
  bool small = false;
  if ((st = sumsq_parts(tensors, count, &parts, &small)) != OSDP_OK) return st;
  if (parts > 0 && !workspace) return fail(OSDP_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned(workspace, 8)) return fail(OSDP_ERR_UNSUPPORTED, "workspace is not 8-byte aligned");
  if (workspace_bytes < static_cast<size_t>(parts) * sizeof(double))
    return fail(OSDP_ERR_WORKSPACE, "workspace holds %zu bytes, %zu needed", workspace_bytes, static_cast<size_t>(parts) * sizeof(double));
  if ((st = device_ok()) != OSDP_OK) return st;
  const hipStream_t q = static_cast<hipStream_t>(stream);
  double *part = static_cast<double *>(workspace);
  st = for_batches(
      tensors, count,
      [&](int32_t i, Tensor *t) {
        t->grad = tensors[i].grad;
        return aligned(t->grad, 16);
      },
      [&](const Batch &b) {
        const unsigned blocks = sum_blocks(b);
        if (small) {
          if (grad_type == OSDP_BF16) hipLaunchKernelGGL(sumsq_small_kernel<uint16_t>, dim3(1), dim3(kSmallThreads), 0, q, b, accumulate, sumsq);
          else hipLaunchKernelGGL(sumsq_small_kernel<float>, dim3(1), dim3(kSmallThreads), 0, q, b, accumulate, sumsq);
          return hip_status(hipGetLastError(), "launching the sum of squares");
        }
        if (grad_type == OSDP_BF16) hipLaunchKernelGGL(sumsq_kernel<uint16_t>, dim3(blocks), dim3(kThreads), 0, q, b, sum_run(b), part);
        else hipLaunchKernelGGL(sumsq_kernel<float>, dim3(blocks), dim3(kThreads), 0, q, b, sum_run(b), part);
        part += blocks;
        return hip_status(hipGetLastError(), "launching the sum of squares");
      });
  if (st != OSDP_OK || small) return st;
  hipLaunchKernelGGL(sumsq_finish_kernel, dim3(1), dim3(kThreads), 0, q, static_cast<const double *>(workspace),
                     static_cast<int32_t>(parts), accumulate, sumsq);
  return hip_status(hipGetLastError(), "launching the end of the sum of squares");
}

osdp_status osdp_adamw_state_values(const osdp_adamw_tensor *tensors, int32_t count, void *const *m_out, void *const *v_out,
                                    void *stream) {
  osdp_status st = check_count(tensors, count);
  if (st != OSDP_OK) return st;
  if (count > 0 && (!m_out || !v_out)) return fail(OSDP_ERR_INVALID_ARG, "m_out or v_out is NULL");
  for (int32_t i = 0; i < count; ++i) {
    if (tensors[i].n == 0) continue;
    if ((st = check_array(tensors[i].m, 1, i, "m")) != OSDP_OK) return st;
    if ((st = check_array(tensors[i].v, 1, i, "v")) != OSDP_OK) return st;
    if ((st = check_array(tensors[i].exps, 2, i, "exps")) != OSDP_OK) return st;
    if (!m_out[i] || !v_out[i]) return fail(OSDP_ERR_INVALID_ARG, "m_out[%d] or v_out[%d] is NULL", i, i);
    if (!aligned(m_out[i], 2) || !aligned(v_out[i], 2)) return fail(OSDP_ERR_UNSUPPORTED, "m_out[%d] or v_out[%d] is not 2-byte aligned", i, i);
  }
  if ((st = device_ok()) != OSDP_OK) return st;
  return for_batches(
      tensors, count,
      [&](int32_t i, Tensor *t) {
        t->m = tensors[i].m; t->v = tensors[i].v; t->exps = tensors[i].exps;
        t->param = m_out[i];
        t->master = static_cast<float *>(v_out[i]);
        return aligned(t->m, 8) && aligned(t->v, 8) && aligned(m_out[i], 16) && aligned(v_out[i], 16);
      },
      [&](const Batch &b) {
        hipLaunchKernelGGL(values_kernel, dim3(grid_of(b, 1)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), b);
        return hip_status(hipGetLastError(), "launching the values of the moments");
      });
}

}  // extern "C"
