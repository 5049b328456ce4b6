// What stands around the products of the split operator:
//   forward   Z = X . W + b,  Y = act(Z) + R      in the product's epilogue (store_fused in gemm_common.h)
//   backward  dZ = dY * act'(Z),  db = sum over tokens of dZ      in one pass in front of the product's backward
// The products are the kernels of osdp_gemm.hip.  Two things are done for them that the calls without an epilogue do not do, whose
// order of additions is promised: shards are read in place for any number of tokens, and products of few output tiles run in parts
// of the reduction, so that every CU has some, with a launch that adds the parts' planes up and goes through the epilogue.
#include "gemm_launch.h"

namespace osdp {

namespace {
// Few tokens: rows of a tile, and the length of a part of the reduction.
// A workgroup streams 2 (rows + 64) bytes a unit of K at some 38 KB a us, where they come from a cache, and takes 8 us to start and
// to store; the weights come from memory once, at 5 TB/s; parts cost the planes' way out and back and a launch.  us in the parts
// that this finds / in one: 1 token 4096 -> 4096 15.1 / 21.3, 33 tokens 8192 -> 1024 15.2 / 34.3, 128 tokens 16384 -> 2560 44.9 / 82.5.
struct SkinnyPlan {
  int rows;
  int64_t k_per;
  double us;
};
// unit: what the length of a part is a multiple of (128: four waves' K blocks; dX: 256); I: one part.
SkinnyPlan skinny_plan(int64_t T, int64_t I, int64_t O, int64_t unit = 128) {
  SkinnyPlan best{16, I, 0.0};
  for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    const int64_t per = parts == 1 ? I : ((I + parts - 1) / parts + unit - 1) / unit * unit;
    if (parts > 1 && (per < 512 || unit == I)) break;
    for (int rows : {16, 32, 48, 64, 128}) {
      const int64_t groups = ((T + rows - 1) / rows) * ((O + 63) / 64) * ((I + per - 1) / per);
      const double stream = static_cast<double>((groups + kCUs - 1) / kCUs) * (static_cast<double>((rows + 64) * 2 * per) / 38.0e3 + 8.0);
      const double us = std::max(stream, 2.0 * static_cast<double>(I) * static_cast<double>(O) / 5.0e6) +
                        (parts > 1 ? 3.5 + 8.0 * parts * static_cast<double>(T) * static_cast<double>(O) / 4.0e6 : 0.0);
      if (best.us == 0.0 || us < best.us) best = SkinnyPlan{rows, per, us};
    }
  }
  return best;
}
}  // namespace

hipError_t launch_gemm_fused(const GemmProblem &q, hipStream_t stream, bool *carry) {
  GemmParams p;
  const hipError_t e = launch_params(q, *carry, &p);
  if (e != hipSuccess) return e;
  constexpr int kFused = static_cast<int>(Epilogue::kBf16Fused);
  return q.acc_in ? launch_planned<true, false, kFused, true>(p, stream, carry, nullptr, 0)
                  : launch_planned<true, false, kFused, false>(p, stream, carry, nullptr, 0);
}

hipError_t launch_combine_fused(const GemmProblem &q, int parts, const float *planes, hipStream_t stream) {
  return launch_combine<static_cast<int>(Epilogue::kBf16Fused)>(gemm_params(q), parts, planes, stream);
}

hipError_t launch_skinny_fused(const WeightMap &w, int64_t T, const void *X, int64_t ldx, void *Y, int64_t ldy,
                               const FusedEpilogue &fused, void *planes, hipStream_t stream) {
  SkinnyParams p = skinny_params(false, w, T, X, ldx, Y, ldy);
  p.fused = fused;
  const SkinnyPlan plan = skinny_plan(T, p.K, p.N);
  if (plan.k_per >= p.K) return launch_skinny_forward<SkinnyResult::kFused>(p, T <= kSkinnyMaxTokens ? skinny_rows(p.M, p.N) : plan.rows, stream);
  p.planes = static_cast<float *>(planes);
  p.k_per = plan.k_per;
  const hipError_t e = launch_skinny_forward<SkinnyResult::kPlanes>(p, plan.rows, stream);
  if (e != hipSuccess) return e;
  GemmParams c{};
  c.M = p.M; c.N = p.N;
  c.C = Y; c.ldc = ldy;
  c.fused = fused;
  return launch_combine<static_cast<int>(Epilogue::kBf16Fused)>(c, (p.K + plan.k_per - 1) / plan.k_per, p.planes, stream);
}

int64_t fused_k_per(int64_t M, int64_t K, int64_t N) {
  // Of 128 x 128 tiles, one to a CU: 0.0105 us a unit of K.  The parts' planes and the launch that adds them up: some 11 us.
  // us in parts / in one: forward 300 tokens 8192 -> 1024 20.5 / 61.7, 500 tokens 4096 -> 1024 21.0 / 39.3; backward (the
  // pass for db, dX and dW) 300 tokens 1024 -> 8192 35 / 75, 8192 tokens 512 -> 512 36 / 75, 16384 tokens 256 -> 1024 51 / 137.
  const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128);
  const int64_t parts = std::min<int64_t>({kCUs / std::max<int64_t>(tiles, 1), K / 512, 32});
  if (parts < 2 || K - K / parts < 1500) return K;
  return ((K + parts - 1) / parts + 63) / 64 * 64;
}

namespace {
size_t planes_of(int64_t M, int64_t K, int64_t N, int64_t k_per) {
  const int64_t parts = k_per > 0 ? (K + k_per - 1) / k_per : 0;
  return parts > 1 ? static_cast<size_t>(parts) * static_cast<size_t>(M) * static_cast<size_t>(N) * 4 : 0;
}
}  // namespace

// Where no shard is a whole number of K blocks only the few-token kernel reads the weights in place, at a third of the tiles'
// rate.  More tokens than its own are worth that while the copy and the tiles behind it, each one's latency, take longer: three
// quarters of what they would take one after the other, and the launches.  By T, I and O alone: the unsplit copy is what counts, so
// that Y is the same for every k.  us in place / staged: 200 tokens 1024 -> 1024 10.3 / 15.0, 1000 tokens 13.4 / 16.3, 160 tokens
// 8160 -> 1024 22.8 / 29.4, 300 tokens 2560 -> 2560 23.2 / 25.4; 400 tokens 4032 -> 4032 51 / 40.5.
// copied: not so where one shard holds the matrix, which tiles read as it lies (219 tokens 624 -> 512 8.6 / 12.0).
bool skinny_beats_copy(int64_t T, int64_t I, int64_t O, bool copied = true) {
  const int64_t tiles = ((T + 127) / 128) * ((O + 127) / 128), k_per = fused_k_per(T, I, O), parts = (I + k_per - 1) / k_per;
  const double flops = 2.0 * static_cast<double>(T) * static_cast<double>(I) * static_cast<double>(O);
  const double tile = std::max(flops / 0.9e9, 0.0105 * static_cast<double>(std::min(k_per, I)) * static_cast<double>((tiles * parts + kCUs - 1) / kCUs));
  const double copy = (copied ? 4.0 * static_cast<double>(I) * static_cast<double>(O) / 5.5e6 : 0.0) + 6.0;
  return skinny_plan(T, I, O).us < 0.75 * (copy + tile) + (parts > 1 ? 12.0 : 3.0);
}

bool fused_takes_skinny(int64_t T, int64_t ldx, const ShardLayout &lay, int64_t I) {
  if (skinny_takes(false, T, ldx, lay, I)) return true;
  const DebugOptions &d = debug_options();  // (the switches that pick a kernel or a schedule for staged products keep those)
  if (d.gemm_generic.load(std::memory_order_relaxed) != 0 || d.tile.load(std::memory_order_relaxed) >= 0 ||
      d.fwd_pair.load(std::memory_order_relaxed) >= 0 || d.fused_gather.load(std::memory_order_relaxed) >= 0 ||
      d.poison_staging.load(std::memory_order_relaxed) != 0)
    return false;
  return T > kSkinnyMaxTokens && !(lay.rows_per_shard > 0 && lay.rows_per_shard % 64 == 0) && ldx < kMaxLd && I < kMaxLd && lay.O < kMaxLd &&
         skinny_beats_copy(T, I, lay.O, lay.N > 1);
}

size_t fused_planes_bytes(int64_t T, int64_t I, int64_t O) {
  const size_t tiles = planes_of(T, I, O, fused_k_per(T, I, O));  // (for any N: with a copy the few-token kernel takes no fewer)
  if (T <= 0 || !(T <= kSkinnyMaxTokens || skinny_beats_copy(T, I, O))) return tiles;
  return std::max(tiles, planes_of(T, I, O, skinny_plan(T, I, O).k_per));
}

int64_t skinny_dx_per(int64_t T, int64_t I, int64_t O) {
  // (worth the sums' own launch, and one for dW that would otherwise share dX's.  us of a backward pass in parts / in one: 33 tokens
  // 1024 -> 8192 26.2 / 35.6, 100 tokens 2560 -> 16384 74 / 83)
  const SkinnyPlan plan = skinny_plan(T, O, I, 256), whole = skinny_plan(T, O, I, O);
  return plan.us + 6.0 < whole.us ? plan.k_per : O;
}

size_t bwd_planes_bytes(int64_t T, int64_t I, int64_t O) {
  if (T <= 0) return 0;
  size_t most = std::max(planes_of(T, O, I, fused_k_per(T, O, I)), planes_of(I, T, O, fused_k_per(I, T, O)));
  if (T <= kSkinnyMaxTokens) most = std::max(most, planes_of(T, O, I, skinny_dx_per(T, I, O)));
  return most;
}

hipError_t launch_skinny_dx_parts(const WeightMap &w, int64_t T, const void *dY, int64_t lddy, void *dX, int64_t lddx, void *planes,
                                  hipStream_t stream) {
  SkinnyParams p = skinny_params(true, w, T, dY, lddy, dX, lddx);
  const SkinnyPlan plan = skinny_plan(T, p.K, p.N, 256);
  p.planes = static_cast<float *>(planes);
  p.k_per = static_cast<int32_t>(plan.k_per);
  constexpr SkinnyResult kPlanes = SkinnyResult::kPlanes;
  const hipError_t e = plan.rows == 16   ? launch_skinny_as<16, 64, 64, 3, true, kPlanes>(p, stream)
                       : plan.rows == 32 ? launch_skinny_as<32, 64, 64, 3, true, kPlanes>(p, stream)
                       : plan.rows <= 64 ? launch_skinny_as<64, 64, 64, 2, true, kPlanes>(p, stream)
                                         : launch_skinny_as<128, 64, 32, 3, true, kPlanes>(p, stream);
  if (e != hipSuccess) return e;
  GemmParams c{};
  c.M = p.M; c.N = p.N;
  c.C = dX; c.ldc = lddx;
  return launch_combine<static_cast<int>(Epilogue::kBf16RowMajor)>(c, (p.K + p.k_per - 1) / p.k_per, p.planes, stream);
}

namespace {

// ---- dZ and db ------------------------------------------------------------------------------------------------
// A workgroup takes `lanes` x 8 columns (as many lanes side by side as the columns need, 64 at most) and a range of rows, 256 /
// lanes of them at a time; every lane keeps the sums of its 8 columns.  The sums of its row groups are added up through LDS in
// ascending order, and, where more than one workgroup shares a column, written to a plane of the workspace; sum_planes_kernel
// adds the planes in ascending order.  No atomics: the same inputs give the same bits.
// HBM bound, 6 bytes an element: 8192 x 4096, gelu, 37 us (5.4 TB/s, its vector units busy all the while); 16384 x 10240, gelu_tanh,
// 195 us (5.2 TB/s).  The sums cost 4 to 5 us beside that.
struct SlopeParams {
  int64_t T;
  int32_t O, lanes_log2, rows_per_group;
  const uint16_t *dY;
  int64_t lddy;
  const uint16_t *Z;
  int64_t ldz;
  uint16_t *dZ;
  int64_t lddz;
  float *planes;   // nullptr: db is stored
  void *db;
  int32_t db_f32;
};

__device__ __forceinline__ void store_sums(void *db, int db_f32, int n, const float (&s)[8]) {
  if (db_f32) {
    float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(db) + n);
    dst[0] = float4{s[0], s[1], s[2], s[3]};
    dst[1] = float4{s[4], s[5], s[6], s[7]};
  } else {
    store_global16(static_cast<uint16_t *>(db) + n, uint4{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]), pack_bf16x2(s[4], s[5]), pack_bf16x2(s[6], s[7])});
  }
}

template <int kAct, bool kSums>
__global__ __launch_bounds__(256) void slope_kernel(SlopeParams p) {
  constexpr bool kSlope = kAct != OSDP_ACT_NONE;
  constexpr int kAtOnce = 4;  // rows of a lane under way together
  __shared__ float s_sum[kSums ? 256 * 8 : 1];
  const int lanes = 1 << p.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> p.lanes_log2;
  const int groups = 256 >> p.lanes_log2;
  const int n = (static_cast<int>(blockIdx.x) * lanes + lane) * 8;
  const bool columns = n < p.O;
  const int64_t first = static_cast<int64_t>(blockIdx.y) * p.rows_per_group;
  const int64_t end = first + p.rows_per_group < p.T ? first + p.rows_per_group : p.T;
  float sum[8] = {};
  if (columns) {
    for (int64_t m0 = first + group; m0 < end; m0 += kAtOnce * groups) {
      uint4 dy[kAtOnce], z[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int64_t m = m0 + i * groups;
        if (m < end) {
          dy[i] = load_global16(p.dY + m * p.lddy + n);
          if constexpr (kSlope) z[i] = load_global16(p.Z + m * p.ldz + n);
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int64_t m = m0 + i * groups;
        if (m >= end) continue;
        const uint32_t d[4] = {dy[i].x, dy[i].y, dy[i].z, dy[i].w};
        float g[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[2 * e] = bf16_low(d[e]);
          g[2 * e + 1] = bf16_high(d[e]);
        }
        if constexpr (kSlope) {
          const uint32_t zw[4] = {z[i].x, z[i].y, z[i].z, z[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            g[2 * e] *= activation_slope<kAct>(bf16_low(zw[e]));
            g[2 * e + 1] *= activation_slope<kAct>(bf16_high(zw[e]));
          }
          store_global16(p.dZ + m * p.lddz + n, uint4{pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7])});
        }
        if constexpr (kSums)
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += g[e];
      }
    }
  }
  if constexpr (kSums) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s_sum[e * 256 + threadIdx.x] = sum[e];
    __syncthreads();
    if (group != 0 || !columns) return;
    for (int g = 1; g < groups; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += s_sum[e * 256 + (g << p.lanes_log2) + lane];
    if (!p.planes) {
      store_sums(p.db, p.db_f32, n, sum);
    } else {
      float4 *dst = reinterpret_cast<float4 *>(p.planes + static_cast<int64_t>(blockIdx.y) * p.O + n);
      dst[0] = float4{sum[0], sum[1], sum[2], sum[3]};
      dst[1] = float4{sum[4], sum[5], sum[6], sum[7]};
    }
  }
}

// db[n] = the sum over the planes: four waves take a quarter of them each, 64 columns to a workgroup.
__global__ __launch_bounds__(256) void sum_planes_kernel(const float *planes, int count, int O, void *db, int db_f32) {
  __shared__ float s_sum[256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 64 + lane;
  const int per = (count + 3) / 4, first = wave * per, end = first + per < count ? first + per : count;
  float sum = 0.0f;
  if (n < O) {
    const float *src = planes + static_cast<int64_t>(first) * O + n;
#pragma unroll 8
    for (int s = first; s < end; ++s, src += O) sum += *src;
  }
  s_sum[threadIdx.x] = sum;
  __syncthreads();
  if (wave != 0 || n >= O) return;
  for (int w = 1; w < 4; ++w) sum += s_sum[w * 64 + lane];
  if (db_f32) static_cast<float *>(db)[n] = sum;
  else static_cast<__bf16 *>(db)[n] = static_cast<__bf16>(sum);
}

// How rows and columns are dealt out.
struct SlopeGrid {
  int lanes_log2;
  int blocks;     // of columns
  int parts;      // of rows
  int rows;       // in a part
};
// Narrow blocks of many row groups: the sums of a block's rows meet in LDS, so that few planes are left to add up, and small
// problems spread over the CUs.  Up to 256 rows a block takes them all, in 128-byte pieces, and there is no second launch; beyond,
// 256-byte pieces, 4 rows to a lane at least, some 4096 workgroups.
SlopeGrid slope_grid(int64_t T, int64_t O) {
  SlopeGrid g{};
  const int most = T <= 256 ? 3 : 4;
  while (g.lanes_log2 < most && (int64_t{8} << g.lanes_log2) < O) ++g.lanes_log2;
  const int64_t columns = int64_t{8} << g.lanes_log2;
  const int64_t blocks = (O + columns - 1) / columns, least = (T <= 256 ? 8 : 4) * (256 >> g.lanes_log2);
  const int64_t wanted = std::max<int64_t>(1, 4096 / blocks), possible = std::max<int64_t>(1, (T + least - 1) / least);
  const int64_t parts = std::min<int64_t>({wanted, possible, 1024});
  g.blocks = static_cast<int>(blocks);
  g.rows = static_cast<int>(std::max<int64_t>(1, (T + parts - 1) / parts));
  g.parts = static_cast<int>(std::max<int64_t>(1, (T + g.rows - 1) / g.rows));
  return g;
}

template <int kAct>
void launch_slope_as(const SlopeParams &p, const SlopeGrid &g, hipStream_t stream) {
  const dim3 grid(g.blocks, g.parts);
  if (p.db) hipLaunchKernelGGL((slope_kernel<kAct, true>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((slope_kernel<kAct, false>), grid, dim3(256), 0, stream, p);
}

}  // namespace

size_t slope_workspace_bytes(int64_t T, int64_t O) {
  const SlopeGrid g = slope_grid(T, O);
  return g.parts > 1 ? static_cast<size_t>(g.parts) * static_cast<size_t>(O) * sizeof(float) : 0;
}

hipError_t launch_slope(const SlopeProblem &q, void *workspace, hipStream_t stream) {
  const SlopeGrid g = slope_grid(q.T, q.O);
  SlopeParams p{};
  p.T = q.T; p.O = static_cast<int32_t>(q.O);
  p.lanes_log2 = g.lanes_log2; p.rows_per_group = g.rows;
  p.dY = static_cast<const uint16_t *>(q.dY); p.lddy = q.lddy;
  p.Z = static_cast<const uint16_t *>(q.Z); p.ldz = q.ldz;
  p.dZ = static_cast<uint16_t *>(q.dZ); p.lddz = q.lddz;
  p.db = q.db; p.db_f32 = q.db_f32;
  p.planes = q.db && g.parts > 1 ? static_cast<float *>(workspace) : nullptr;
  switch (q.activation) {
    case OSDP_ACT_RELU: launch_slope_as<OSDP_ACT_RELU>(p, g, stream); break;
    case OSDP_ACT_GELU: launch_slope_as<OSDP_ACT_GELU>(p, g, stream); break;
    case OSDP_ACT_GELU_TANH: launch_slope_as<OSDP_ACT_GELU_TANH>(p, g, stream); break;
    case OSDP_ACT_SILU: launch_slope_as<OSDP_ACT_SILU>(p, g, stream); break;
    default:
      if (!q.db) return hipSuccess;  // dZ is dY, and nobody asks for its sums
      hipLaunchKernelGGL((slope_kernel<OSDP_ACT_NONE, true>), dim3(g.blocks, g.parts), dim3(256), 0, stream, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.planes) return e;
  hipLaunchKernelGGL(sum_planes_kernel, dim3((p.O + 63) / 64), dim3(256), 0, stream, p.planes, g.parts, p.O, p.db, p.db_f32);
  return hipGetLastError();
}

}  // namespace osdp
