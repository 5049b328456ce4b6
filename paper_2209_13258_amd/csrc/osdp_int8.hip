// The operator in 8-bit integers: weight shards to 8 bits, tokens to 8 bits, and the product of the two.
//
// Rounding.  q = round(x * 127 / amax), halves away from zero, for bf16 x and amax.  With r = 127 / amax (1 + 2^-21), rounded,
// trunc(|x| r + 1/2) is that number exactly: |x| r lies above |x| 127 / amax, by 2^-20 of it at most, so a half is never
// missed; and a quotient of two numbers of 8 significant bits that is not a half but below one by less than 127 2^-j
// stays away from it by 2^-8-j at least, which 2^7-j 2^-20 does not reach.  One multiplication and one addition a value
// then do what a division would.
//
// Sums of products of 8-bit integers are exact in 32 bits (I <= 131072), whatever their order, so every kernel, every split of the
// reduction and every cut of the weight gives the same bits.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "gemm_i8_w4.h"

namespace osdp {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxFeatures = 131072;
constexpr size_t kAlign = 256;

// ---- tokens to 8 bits -------------------------------------------------------------------------------------------
// kWaves waves a token: the row is read once, kept in registers (what lies beyond kHold vectors a lane is read again), its largest
// magnitude found, and written as bytes.  Rows of Xq are a multiple of 128 bytes long and end in zeros.  Rows of up to 4096 features
// take one wave, and no barrier.
constexpr int kHold = 8;

template <int kWaves>
__global__ __launch_bounds__(kThreads) void quantize_tokens_kernel(const uint16_t *__restrict__ x, int64_t ldx, int32_t features,
                                                                   int32_t ldq, int32_t tokens, uint8_t *__restrict__ q,
                                                                   float *__restrict__ scale, uint32_t *__restrict__ counters) {
  __shared__ uint32_t part[kThreads / 64];
  constexpr int kRows = kThreads / 64 / kWaves, kStep = kWaves * 64 * 8;
  if (counters && blockIdx.x == 0 && threadIdx.x < kI8MostTiles) counters[threadIdx.x] = 0;  // (of the product that follows)
  const int own = threadIdx.x % (kWaves * 64) * 8;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / (kWaves * 64); t < tokens; t += static_cast<int64_t>(gridDim.x) * kRows) {
    const uint16_t *row = x + t * ldx;
    uint4 held[kHold];
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < kHold; ++c) {
      const int i = c * kStep + own;
      held[c] = i < features ? load_global16(row + i) : uint4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int c = 0; c < kHold; ++c) most = max(most, i8_largest(held[c]));
    for (int i = kHold * kStep + own; i < features; i += kStep) most = max(most, i8_largest(load_global16(row + i)));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), d)));
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) most = max(most, part[w]);
      __syncthreads();
    }
    const I8Scale s(most);
    if (own == 0) scale[t] = s.scale;
    uint8_t *out = q + t * ldq;
#pragma unroll
    for (int c = 0; c < kHold; ++c) {
      const int i = c * kStep + own;
      if (i < ldq) *reinterpret_cast<uint2 *>(out + i) = s.round8(held[c]);
    }
    for (int i = kHold * kStep + own; i < ldq; i += kStep)
      *reinterpret_cast<uint2 *>(out + i) = i < features ? s.round8(load_global16(row + i)) : uint2{0u, 0u};
  }
}

hipError_t launch_quantize_tokens(const uint16_t *x, int64_t ldx, const I8Problem &p, uint8_t *xq, float *x_scale, hipStream_t stream) {
  const bool one = p.I <= kHold * 64 * 8;
  const int64_t rows = one ? kThreads / 64 : 1, groups = std::min<int64_t>((p.T + rows - 1) / rows, 1 << 20);
  if (one) hipLaunchKernelGGL(quantize_tokens_kernel<1>, dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0, stream, x, ldx, p.I, p.ldq, p.T, xq, x_scale, p.arrived);
  else hipLaunchKernelGGL(quantize_tokens_kernel<4>, dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0, stream, x, ldx, p.I, p.ldq, p.T, xq, x_scale, p.arrived);
  return hipGetLastError();
}

// ---- weight shards to 8 bits --------------------------------------------------------------------------------------
// Two passes: the largest magnitude of every column over the rows that a workgroup takes (into the workspace), 32 rows at a time,
// the workgroups' side by side, so that all of them move down the matrix together; then, over tiles of 128 x 128, their largest,
// the rounding, and the transposition through LDS.  The second pass begins at the bottom, where the first has left the last
// 256 MB in the last-level cache, and marks its own loads and stores as used once, which keeps them there until they are read: 8192 -> 32768
// (537 MB read twice, 268 written) takes 212 us, against 267 with ranges of rows to the workgroups and both passes from the top.
// Taking the columns in strips of what the cache holds, pass after pass, did not pay (298 us in strips of 128 MB, 307 of 96, 367 of 64).
struct WeightShards {
  ShardTable w, q;          // bf16 [I x O], 8 bits [O x I]: flat, cut after every L elements
  int64_t L;
  int32_t I, O;
};

constexpr int kColumns = 256;  // of a workgroup of the first pass: 8 to a lane, 32 lanes side by side, 8 rows at a time
constexpr int kAmaxRows = 32;  // of a step of the first pass: 8 rows at a time, four times
constexpr int kStrip = 128;    // rows and columns of a tile of the second pass

// A place in a flat matrix that is cut into shards.  One division finds a workgroup's first place; from there on places move
// ahead and shards are counted as they end.
struct Place {
  int32_t shard;
  int64_t off;
  __device__ __forceinline__ Place(int64_t flat, int64_t L) : shard(static_cast<int32_t>(flat / L)), off(flat - shard * L) {}
  __device__ __forceinline__ void ahead(int64_t by, int64_t L) {
    off += by;
    while (off >= L) {
      off -= L;
      ++shard;
    }
  }
};

__global__ __launch_bounds__(kThreads) void column_amax_kernel(WeightShards p, uint32_t *__restrict__ part) {
  __shared__ const uint16_t *tab[OSDP_MAX_SHARDS];
  __shared__ uint32_t most[8][kColumns];
  if (threadIdx.x < OSDP_MAX_SHARDS) tab[threadIdx.x] = static_cast<const uint16_t *>(p.w.p[threadIdx.x]);
  __syncthreads();
  const int lane = threadIdx.x & 31, line = threadIdx.x >> 5;
  const int c = blockIdx.x * kColumns + lane * 8;
  const int r0 = blockIdx.y * kAmaxRows + line, turn = gridDim.y * kAmaxRows;
  uint32_t m[8] = {};
  if (c < p.O) {
    Place at(static_cast<int64_t>(r0) * p.O + c, p.L);
    // (rows beyond the last repeat it, so that the loads of four steps go out together)
    for (int r = r0; r < p.I; r += turn) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u] = load_global16(tab[at.shard] + at.off);
        if (u < 3 && r + 8 * (u + 1) < p.I) at.ahead(static_cast<int64_t>(8) * p.O, p.L);
      }
      if (r + turn < p.I) at.ahead(static_cast<int64_t>(turn - 24) * p.O, p.L);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          m[2 * j] = max(m[2 * j], w[j] << 16 & 0x7fff0000u);
          m[2 * j + 1] = max(m[2 * j + 1], w[j] & 0x7fff0000u);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) most[line][lane * 8 + j] = m[j];
  __syncthreads();
  const int col = blockIdx.x * kColumns + threadIdx.x;
  uint32_t all = 0;
#pragma unroll
  for (int l = 0; l < 8; ++l) all = max(all, most[l][threadIdx.x]);
  if (col < p.O) part[static_cast<int64_t>(blockIdx.y) * p.O + col] = all;
}

__global__ __launch_bounds__(kThreads) void quantize_weight_kernel(WeightShards p, int32_t parts, const uint32_t *__restrict__ part,
                                                                   float *__restrict__ scale) {
  __shared__ const uint16_t *tab[OSDP_MAX_SHARDS];
  __shared__ uint8_t *q_tab[OSDP_MAX_SHARDS];
  __shared__ uint32_t most[2][kStrip];
  __shared__ float ratio[kStrip], up[kStrip];
  __shared__ uint32_t tile[kStrip][kStrip / 4 + 1];  // [o][i / 4]; two lanes to a bank (an order without that takes as long: memory is the bound)
  if (threadIdx.x < OSDP_MAX_SHARDS) {
    tab[threadIdx.x] = static_cast<const uint16_t *>(p.w.p[threadIdx.x]);
    q_tab[threadIdx.x] = static_cast<uint8_t *>(p.q.p[threadIdx.x]);
  }
  __syncthreads();
  // (from the bottom up; tiles that run together lie on a diagonal: their stores, a row of the result apart, then do not all meet the same memory
  // channels; 149 -> 142 us)
  const int ti = (gridDim.y - 1 - blockIdx.y + blockIdx.x / 4) % gridDim.y;
  const int o0 = blockIdx.x * kStrip, i0 = ti * kStrip;
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;  // 8 columns, 4 rows to a lane, twice
  uint4 v[2][4];  // (on their way while the columns' largest are looked up; beyond the edges anything, it is not stored)
  {
    const Place first(static_cast<int64_t>(i0) * p.O + o0, p.L);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        Place at = first;
        at.ahead(static_cast<int64_t>(min(half * 64 + rg * 4 + j, p.I - 1 - i0)) * p.O + min(cg * 8, p.O - 8 - o0), p.L);
        v[half][j] = load_global16_once(tab[at.shard] + at.off);
      }
  }
  {
    const int o = o0 + (threadIdx.x & (kStrip - 1)), first = threadIdx.x / kStrip;
    uint32_t m = 0;
    if (o < p.O) {
#pragma unroll 4
      for (int y = first; y < parts; y += 2) m = max(m, part[static_cast<int64_t>(y) * p.O + o]);
    }
    most[first][threadIdx.x & (kStrip - 1)] = m;
  }
  __syncthreads();
  if (threadIdx.x < kStrip) {
    const I8Scale s(max(most[0][threadIdx.x], most[1][threadIdx.x]));
    ratio[threadIdx.x] = s.r;
    up[threadIdx.x] = s.up;
    if (ti == 0 && o0 + static_cast<int>(threadIdx.x) < p.O) scale[o0 + threadIdx.x] = s.scale;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const I8Scale s(ratio[cg * 8 + j], up[cg * 8 + j]);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t pair = (&v[half][e].x)[j >> 1];
        q[e] = s.round(__uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16));
      }
      const uint32_t word = i8_pack(q[0], q[1], q[2], q[3]);
      tile[cg * 8 + j][half * 16 + rg] = word;
    }
  }
  __syncthreads();
  const int piece = threadIdx.x & 7;
  const Place out(static_cast<int64_t>(o0) * p.I + i0, p.L);
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int row = pass * 32 + (threadIdx.x >> 3), o = o0 + row, i = i0 + piece * 16;
    if (o < p.O && i < p.I) {
      const uint4 v = {tile[row][piece * 4], tile[row][piece * 4 + 1], tile[row][piece * 4 + 2], tile[row][piece * 4 + 3]};
      Place at = out;
      at.ahead(static_cast<int64_t>(row) * p.I + piece * 16, p.L);
      store_global16_once(q_tab[at.shard] + at.off, v);
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------
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
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct Weight {
  int64_t T, I, O, L;
  int32_t N, k;
  int64_t rows_each;  // output channels to a shard where N divides O, else 0
};

osdp_status check_weight(const osdp_shape *s, Weight *w) {
  if (!s) return fail(OSDP_ERR_INVALID_ARG, "shape is NULL");
  if (s->T < 0 || s->I <= 0 || s->O <= 0)
    return fail(OSDP_ERR_INVALID_ARG, "I, O must be positive and T non-negative (got T %lld, I %lld, O %lld)", (long long)s->T, (long long)s->I, (long long)s->O);
  if (s->N < 1) return fail(OSDP_ERR_INVALID_ARG, "N must be >= 1 (got %d)", s->N);
  if (s->N > OSDP_MAX_SHARDS) return fail(OSDP_ERR_UNSUPPORTED, "N = %d exceeds %d shards", s->N, OSDP_MAX_SHARDS);
  // (columns of the tile that ends last are counted too, up to 263 behind O)
  if (s->T >= (1ll << 31) || s->O > (1ll << 31) - 512) return fail(OSDP_ERR_UNSUPPORTED, "T must be below 2^31, O at most 2^31 - 512");
  if (s->I % 16 || s->I > kMaxFeatures)
    return fail(OSDP_ERR_UNSUPPORTED, "I must be a multiple of 16 and at most %lld (got %lld)", (long long)kMaxFeatures, (long long)s->I);
  if (s->O % 8) return fail(OSDP_ERR_UNSUPPORTED, "O must be a multiple of 8 (got %lld)", (long long)s->O);
  w->T = s->T; w->I = s->I; w->O = s->O; w->N = s->N;
  w->L = (s->I * s->O + s->N - 1) / s->N;
  if (w->L % 16) return fail(OSDP_ERR_UNSUPPORTED, "shard length %lld is not a multiple of 16", (long long)w->L);
  w->rows_each = s->O % s->N == 0 ? s->O / s->N : 0;
  return OSDP_OK;
}

osdp_status fill_table(const void *const *ptrs, int32_t N, const char *name, ShardTable *t) {
  if (!ptrs) return fail(OSDP_ERR_INVALID_ARG, "%s is NULL", name);
  std::memset(t, 0, sizeof *t);
  for (int32_t s = 0; s < N; ++s) {
    if (!ptrs[s]) return fail(OSDP_ERR_INVALID_ARG, "%s[%d] is NULL", name, s);
    if (!aligned(ptrs[s], 16)) return fail(OSDP_ERR_UNSUPPORTED, "%s[%d] is not 16-byte aligned", name, s);
    t->p[s] = const_cast<void *>(ptrs[s]);
  }
  return OSDP_OK;
}

osdp_status check_scale(const float *p) {
  if (!p) return fail(OSDP_ERR_INVALID_ARG, "w_scale is NULL");
  if (!aligned(p, 16)) return fail(OSDP_ERR_UNSUPPORTED, "w_scale is not 16-byte aligned");
  return OSDP_OK;
}

osdp_status check_matrix(const void *p, int64_t ld, int64_t cols, const char *name) {
  if (!p) return fail(OSDP_ERR_INVALID_ARG, "%s is NULL", name);
  if (ld < cols) return fail(OSDP_ERR_INVALID_ARG, "leading dimension of %s (%lld) is below its row length %lld", name, (long long)ld, (long long)cols);
  if (ld % 8) return fail(OSDP_ERR_UNSUPPORTED, "leading dimension of %s (%lld) is not a multiple of 8", name, (long long)ld);
  if (!aligned(p, 16)) return fail(OSDP_ERR_UNSUPPORTED, "%s is not 16-byte aligned", name);
  return OSDP_OK;
}

// Whether T rows of I elements, ldx apart, and T of O, ldy apart, share any.  Rows of one length apart meet where those of the one fall into
// columns of the other; of different lengths, anywhere (nobody lays matrices into one another so).
bool overlap(const void *x, int64_t ldx, int64_t I, const void *y, int64_t ldy, int64_t O, int64_t T) {
  const int64_t d = (static_cast<int64_t>(reinterpret_cast<uintptr_t>(y)) - static_cast<int64_t>(reinterpret_cast<uintptr_t>(x))) / 2;
  if (d >= (T - 1) * ldx + I || -d >= (T - 1) * ldy + O) return false;
  if (ldx != ldy || T == 1) return true;
  // rows i of X and j of Y meet where (i - j) ld lies in (d - I, d + O)
  auto floor_div = [ldx](int64_t a) { return a / ldx - (a % ldx < 0); };
  return std::max(floor_div(d - I) + 1, 1 - T) <= std::min(-floor_div(-d - O) - 1, T - 1);
}

osdp_status check_workspace(const void *ws, size_t bytes, size_t need) {
  if (!ws) return fail(OSDP_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned(ws, kAlign)) return fail(OSDP_ERR_UNSUPPORTED, "workspace is not 256-byte aligned");
  if (bytes < need) return fail(OSDP_ERR_WORKSPACE, "workspace holds %zu bytes, %zu needed", bytes, need);
  return OSDP_OK;
}

// Workgroups that share the rows of a strip of columns in the first pass: enough for the card, with at least one step each.
int32_t amax_parts(const Weight &w) {
  const int64_t strips = (w.O + kColumns - 1) / kColumns;
  return static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>((w.I + kAmaxRows - 1) / kAmaxRows, 1024 / std::min<int64_t>(strips, 1024))));
}

// ---- which kernel ---------------------------------------------------------------------------------------------------
enum class Kernel { kFew, k64, k128, k128Walk, k256Walk };
struct Choice {
  Kernel kernel;
  int parts;
  double us;  // estimated
};

// The kernel, and the parts of a tile's reduction, that are estimated fastest for T tokens and `shards` blocks of `rows`
// channels.  A launch takes `fixed` us, and for each round of workgroups over the card `start` and `block` for every 128 input
// features; a tile's parts cost `each` apiece, and `meet` for every 256 workgroups' worth of sums.  The constants were fitted to 181 random sizes
// (8 to 8192 tokens, 256 to 16384 input and output features), all of them timed with every kernel below and 1 to 8 parts, and those of the
// walking tiles to 60 more with the weight from memory: the choice is 0.8 and 0.4 % slower than the best of them in the geometric mean, 30 and 12 %
// at most.  us for 16 / 64 x 64 / 128 x 128 / walking 128 x 128 / walking 256 x 256:
//     30 tokens   400 -> 3456       6.1 /  7.4 /   9.5 /   9.6 /  15.5
//    162         1152 -> 1344      10.2 /  8.9 /  11.7 /  12.9 /  22.0
//    161        14448 ->  960      37.5 / 35.1 (four parts 21.2) / 55.4 (30.0) / 85.8 / 135
//   1000         4096 -> 4096       230 / 36.9 /  27.9 /  32.6 /  51.6
//    500         2560 -> 10240      186 / 31.9 /  31.9 /  27.4 /  38.0
//   3000         4096 -> 16384     2630 /  349 /   242 /   202 /   167
Choice choose(int64_t T, int64_t I, int64_t rows, int64_t shards, bool may_share) {
  struct Prices {
    Kernel kernel;
    int side, room;  // tiles of side x side; workgroups that the card holds
    double fixed, block, start, each, meet;
  };
  constexpr Prices kPrices[] = {{Kernel::kFew, 16, 1024, 5.05, 0.364, 0.81, 0, 0},
                                {Kernel::k64, 64, 512, 4.84, 0.429, 3.07, 0.83, 0.83},
                                {Kernel::k128, 128, 256, 2.63, 0.447, 6.37, 0.89, 4.43},
                                {Kernel::k128Walk, 128, 512, 5.44, 0.9, 5.73, 0, 0},
                                {Kernel::k256Walk, 256, 256, 0.95, 1.1, 15, 0, 0}};
  const int64_t blocks = (I + 127) / 128;
  Choice best = {Kernel::k256Walk, 1, -1.0};
  for (const Prices &v : kPrices) {
    const bool few = v.kernel == Kernel::kFew;
    const int64_t across = few ? (rows * shards + 15) / 16 : shards * i8_shard_tiles(rows, v.side);
    const int64_t tiles = across * ((T + v.side - 1) / v.side);
    if (few && (T > 4096 || rows * shards > kI8FewChannels)) continue;
    if ((v.kernel == Kernel::k64 || v.kernel == Kernel::k128) && tiles > (1 << 20)) continue;
    for (int asked : {1, 2, 3, 4, 6, 8}) {
      const int64_t each = (blocks + asked - 1) / asked, parts = (blocks + each - 1) / each, groups = tiles * parts;
      if (asked > 1 && (v.each == 0 || !may_share || each < 2 || tiles > kI8MostTiles ||
                        static_cast<size_t>(groups) * v.side * v.side * 4 > kI8SumBytes))
        break;
      double rounds = static_cast<double>((groups + v.room - 1) / v.room);
      if (few) rounds = std::max(static_cast<double>(groups) / v.room, groups > 256 ? 0.5 : T > 16 ? 0.35 : 0.25);
      else if (v.room == 512 && groups % 512 != 0) {  // (one workgroup to a CU is faster than two; with so few tokens that bytes are the bound,
                                                          // in proportion: 16 tokens 5120 -> 20480 38.3 us, so 31.0; 20480 -> 5120 37.5 and 34.4)
        const double part = static_cast<double>(groups % 512) / 512.0;
        rounds -= T <= 16 ? std::min(0.4, 0.5 - 0.5 * part) : part <= 0.5 ? 0.4 : 0.0;
      }
      // (up to 16 tokens all workgroups read the same ones, and with fewer than 16 a wave's 16 rows of them are fewer lines: us by 16 / by
      // 64 x 64 in four to eight parts, weight from memory: 16384 -> 4096 2 tokens 20.1 / 25.0, 10 22.1 / 25.5, 16 24.8 / 25.6; 12000 -> 1024
      // 2 tokens 11.1 / 15.8, 16 14.1 / 15.9; 16000 -> 1000 40 tokens 21.4 / 17.9)
      const double block = few && T < 16 ? v.block * (0.7 + 0.3 * static_cast<double>(T) / 16.0) : v.block;
      double us = v.fixed + rounds * (static_cast<double>(each) * block + v.start);
      if (parts > 1) us += v.each * static_cast<double>(parts) + v.meet * static_cast<double>(groups) / 256.0;
      if (best.us < 0.0 || us < best.us) best = {v.kernel, static_cast<int>(parts), us};
    }
  }
  return best;
}

hipError_t launch_product(const I8Problem &p, hipStream_t stream) {
  if (p.rows_each == 0) return launch_few(p, stream);
  const Choice c = choose(p.T, p.I, p.rows_each, p.O / p.rows_each, p.sums != nullptr);
  switch (c.kernel) {
    case Kernel::kFew: return launch_few(p, stream);
    case Kernel::k64: return launch_i8_tiles<2, 2, 4>(p, c.parts, stream);
    case Kernel::k128: return launch_i8_tiles<4, 4, 4>(p, c.parts, stream);
    case Kernel::k128Walk: return launch_i8_tiles<4, 4, 2>(p, 1, stream);
    case Kernel::k256Walk: return launch_i8_tiles<8, 8, 2>(p, 1, stream);
  }
  return hipErrorInvalidValue;
}

// Whether tokens are rounded inside the product's launch: every workgroup, of 16 tokens and 16 channels, does it again, which
// 2^14 values are quick enough for as long as there are not too many workgroups.  (One token is always: it is read by all of them anyway.)  us in
// two launches / one, one call behind another, and captured: 1 token 512 -> 512 8.9 / 6.8 and 4.7 / 3.4, 4096 -> 16384 17.4 / 15.1 and 16.7 / 14.6; 64 tokens
// 512 -> 1024 8.5 / 6.6 and 5.6 / 5.0; at the line 512 of 512 -> 512 8.8 / 8.9 and 7.0 / 8.3, 128 of 1024 -> 1024 8.5 / 7.7 and 7.2 / 7.6; beyond it 256 of
// 256 -> 2048 8.8 / 14.6 and 6.4 / 14.6, 3 of 4096 -> 16384 17.4 / 17.4 and 17.4 / 17.4.
bool rounds_inside(const Weight &w) {
  const int64_t values = std::min<int64_t>(w.T, 16) * w.I;
  if (values > (1 << 14) || w.O > kI8FewChannels) return false;
  if (w.T == 1) return true;
  return (w.T + 15) / 16 * ((w.O + 15) / 16) * std::max<int64_t>(values, 1 << 13) <= (1 << 23);
}

// Whether slices have to be gathered, and whether they may be: with many tokens the tiles that end with each shard can cost more than a
// dense copy of the weight does.  Cut within channels, us in place (up to 64 tokens) / gathered (65), 16 shards: 4096 -> 16392 33 tokens 39 / 47, 64
// 56 / 47; 8192 -> 32776 33 tokens 122 / 180, 64 185 / 180; 16384 -> 4104 48 tokens 66 / 53, 64 82 / 53: the line is right for wide weights, and
// too far for long ones.
bool has_to_gather(const Weight &w) { return (w.T > kI8FewTokens || w.O > kI8FewChannels) && w.rows_each < kI8ShardRows; }
bool may_gather(const Weight &w) { return has_to_gather(w) || (w.T > kI8ManyTokens && w.N > 1 && w.rows_each % 256 != 0); }

// Gathers where that is estimated faster: a gather reads and writes a slice at 5.5 TB/s and takes 6 us besides.  Eight shards of 320 channels,
// 16384 tokens: 2560 -> 2560 in place 167 us, gathered 144; 10240 -> 2560 565 and 474; of 125 channels, 4000 tokens 4096 -> 1000: 46 and 34.
bool gathers(const Weight &w) {
  if (!may_gather(w) || has_to_gather(w)) return has_to_gather(w);
  double us = 0.0;
  for (int64_t j = 0; j < w.k; ++j) {
    const int64_t wide = (j + 1) * w.O / w.k - j * w.O / w.k;
    us += choose(w.T, w.I, wide, 1, false).us + 2.0 * static_cast<double>(w.I * wide) / 5.5e6 + 6.0;
  }
  return us < 0.97 * choose(w.T, w.I, w.rows_each, w.N, false).us;
}

// The workspace up to the staging slot: [Xq][s_t][counters][sums of tiles whose reduction is shared].  The last two do not depend on
// T, so that what does for many tokens does for fewer.
bool may_share(const Weight &w) { return w.I > 3 * 128 && w.O <= 16384; }
size_t scale_offset(const Weight &w) { return round_up(static_cast<size_t>(w.T) * i8_row_bytes(w.I), kAlign); }
size_t counter_offset(const Weight &w) { return scale_offset(w) + round_up(static_cast<size_t>(w.T) * 4, kAlign); }
size_t token_bytes(const Weight &w) { return counter_offset(w) + (may_share(w) ? kI8MostTiles * 4 + kI8SumBytes : 0); }

osdp_status check_slices(const osdp_shape *s, Weight *w, int64_t *widest) {
  const int64_t k = s->k == 0 ? 1 : s->k;
  if (s->k < 0) return fail(OSDP_ERR_INVALID_ARG, "k must be >= 0 (got %d)", s->k);
  if (k > w->O) return fail(OSDP_ERR_INVALID_ARG, "k = %lld exceeds O = %lld", (long long)k, (long long)w->O);
  w->k = static_cast<int32_t>(k);
  *widest = 0;
  for (int64_t j = 0; j < k; ++j) {
    const int64_t c0 = j * w->O / k, c1 = (j + 1) * w->O / k;
    if (c0 % 8 || c1 % 8) return fail(OSDP_ERR_UNSUPPORTED, "slice %lld = [%lld, %lld) is not aligned to 8 columns", (long long)j, (long long)c0, (long long)c1);
    *widest = std::max(*widest, c1 - c0);
  }
  if (!may_gather(*w)) *widest = 0;
  return OSDP_OK;
}

}  // namespace
}  // namespace osdp

using namespace osdp;

extern "C" {

osdp_status osdp_split_linear_i8_quantize_workspace_bytes(const osdp_shape *shape, size_t *bytes) {
  Weight w;
  const osdp_status st = check_weight(shape, &w);
  if (st != OSDP_OK) return st;
  if (!bytes) return fail(OSDP_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = static_cast<size_t>(amax_parts(w)) * w.O * 4;
  return OSDP_OK;
}

osdp_status osdp_split_linear_i8_quantize(const osdp_shape *shape, const void *const *w_shards, void *const *q_shards,
                                          float *w_scale, void *workspace, size_t workspace_bytes, void *stream) {
  Weight w;
  osdp_status st = check_weight(shape, &w);
  if (st != OSDP_OK) return st;
  WeightShards p;
  if ((st = fill_table(w_shards, w.N, "w_shards", &p.w)) != OSDP_OK) return st;
  if ((st = fill_table(const_cast<const void *const *>(q_shards), w.N, "q_shards", &p.q)) != OSDP_OK) return st;
  if ((st = check_scale(w_scale)) != OSDP_OK) return st;
  const int32_t parts = amax_parts(w);
  if ((st = check_workspace(workspace, workspace_bytes, static_cast<size_t>(parts) * w.O * 4)) != OSDP_OK) return st;
  const int64_t tiles_i = (w.I + kStrip - 1) / kStrip, tiles_o = (w.O + kStrip - 1) / kStrip;
  if (tiles_o >= (1ll << 24)) return fail(OSDP_ERR_UNSUPPORTED, "O = %lld is too large", (long long)w.O);
  if ((st = device_ok()) != OSDP_OK) return st;
  p.L = w.L;
  p.I = static_cast<int32_t>(w.I); p.O = static_cast<int32_t>(w.O);
  const hipStream_t q = static_cast<hipStream_t>(stream);
  uint32_t *part = static_cast<uint32_t *>(workspace);
  hipLaunchKernelGGL(column_amax_kernel, dim3(static_cast<unsigned>((w.O + kColumns - 1) / kColumns), static_cast<unsigned>(parts)),
                     dim3(kThreads), 0, q, p, part);
  if ((st = hip_status(hipGetLastError(), "launching the columns' largest")) != OSDP_OK) return st;
  hipLaunchKernelGGL(quantize_weight_kernel, dim3(static_cast<unsigned>(tiles_o), static_cast<unsigned>(tiles_i)), dim3(kThreads), 0, q,
                     p, parts, part, w_scale);
  return hip_status(hipGetLastError(), "launching the quantization");
}

osdp_status osdp_split_linear_i8_workspace_bytes(const osdp_shape *shape, size_t *total, size_t *peak_weight_staging) {
  Weight w;
  osdp_status st = check_weight(shape, &w);
  if (st != OSDP_OK) return st;
  int64_t widest = 0;
  if ((st = check_slices(shape, &w, &widest)) != OSDP_OK) return st;
  const size_t slot = static_cast<size_t>(widest) * w.I;
  if (total) *total = token_bytes(w) + round_up(slot, kAlign);
  if (peak_weight_staging) *peak_weight_staging = slot;
  return OSDP_OK;
}

osdp_status osdp_split_linear_i8_fwd(const osdp_shape *shape, const void *X, int64_t ldx, const void *const *q_shards,
                                     const float *w_scale, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  Weight w;
  osdp_status st = check_weight(shape, &w);
  if (st != OSDP_OK) return st;
  int64_t widest = 0;
  if ((st = check_slices(shape, &w, &widest)) != OSDP_OK) return st;
  const bool no_tokens = w.T == 0;  // X and Y have no rows and may be NULL
  if (!no_tokens && (st = check_matrix(X, ldx, w.I, "X")) != OSDP_OK) return st;
  if (!no_tokens && (st = check_matrix(Y, ldy, w.O, "Y")) != OSDP_OK) return st;
  ShardTable tab;
  if ((st = fill_table(q_shards, w.N, "q_shards", &tab)) != OSDP_OK) return st;
  if ((st = check_scale(w_scale)) != OSDP_OK) return st;
  if (!no_tokens && (st = check_workspace(workspace, workspace_bytes, token_bytes(w) + round_up(static_cast<size_t>(widest) * w.I, kAlign))) != OSDP_OK) return st;
  if (!no_tokens && overlap(X, ldx, w.I, Y, ldy, w.O, w.T)) return fail(OSDP_ERR_INVALID_ARG, "Y overlaps X");
  if ((st = device_ok()) != OSDP_OK) return st;
  if (no_tokens) return OSDP_OK;
  const hipStream_t q = static_cast<hipStream_t>(stream);
  char *ws = static_cast<char *>(workspace);
  I8Problem p{};
  p.T = static_cast<int32_t>(w.T); p.I = static_cast<int32_t>(w.I); p.O = static_cast<int32_t>(w.O);
  p.ldq = static_cast<int32_t>(i8_row_bytes(w.I));
  p.shards = tab; p.L = w.L; p.rows_each = static_cast<int32_t>(w.rows_each);
  p.w_scale = w_scale; p.y = static_cast<uint16_t *>(Y); p.ldy = ldy;
  const uint16_t *x = static_cast<const uint16_t *>(X);
  if (rounds_inside(w)) return hip_status(launch_fused(p, x, ldx, q), "launching the product");
  uint8_t *xq = reinterpret_cast<uint8_t *>(ws);
  float *x_scale = reinterpret_cast<float *>(ws + scale_offset(w));
  p.xq = xq; p.x_scale = x_scale;
  if (may_share(w)) {
    p.arrived = reinterpret_cast<uint32_t *>(ws + counter_offset(w));
    p.sums = p.arrived + kI8MostTiles;
  }
  char *slot = ws + token_bytes(w);
  if ((st = hip_status(launch_quantize_tokens(x, ldx, p, xq, x_scale, q), "launching the tokens' quantization")) != OSDP_OK) return st;
  if (!gathers(w)) return hip_status(launch_product(p, q), "launching the product");
  ShardLayout lay{};  // (two bytes an element, as the gather counts)
  lay.O = w.I / 2; lay.L = w.L / 2; lay.N = w.N; lay.rows_per_shard = static_cast<int32_t>(w.rows_each);
  for (int64_t j = 0; j < w.k; ++j) {
    const int64_t c0 = j * w.O / w.k, c1 = (j + 1) * w.O / w.k;
    if ((st = hip_status(launch_gather(tab, lay, c0, c1 - c0, 0, w.I / 2, slot, q), "gathering a slice")) != OSDP_OK) return st;
    p.O = static_cast<int32_t>(c1 - c0);
    p.shards.p[0] = slot;
    p.rows_each = p.O;
    p.w_scale = w_scale + c0; p.y = static_cast<uint16_t *>(Y) + c0;
    if ((st = hip_status(launch_product(p, q), "launching the product")) != OSDP_OK) return st;
  }
  return OSDP_OK;
}

}  // extern "C"
