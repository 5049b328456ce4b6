// Slice GEMMs of the operator-split linear layer (arXiv 2209.13258, Section 3.3):
//   forward   Y[:, slice]  = X . Ws          A K-contiguous, B N-contiguous
//   dW        dW[:, slice] = X^T . dY_slice  A M-contiguous, B N-contiguous
//   dX        dX (+)= dY_slice . Ws^T        A K-contiguous, B K-contiguous
// bf16 operands, fp32 accumulation on the gfx950 matrix cores
// (v_mfma_f32_16x16x32_bf16), bf16 round-to-nearest-even outputs.
//
// Every kernel in this file but the few-token one (gemm_skinny.h) feeds each output element the same sequence of
// MFMA operations: K is walked in ascending blocks of 32, and inside a block
// logical k = 8*q + e sits in lane group q, element e of both operands.  Tile
// shape therefore never changes a result bit, which is what makes Y and dW of
// a split operator bit-identical to the unsplit ones.
#include "gemm_launch.h"

namespace osdp {

namespace {
bool shards_are_k_blocks(const ShardLayout &lay) { return lay.rows_per_shard > 0 && lay.rows_per_shard % 64 == 0; }
}  // namespace

bool gemm_reads_shards(int64_t T, int64_t ld_act, const ShardLayout &lay, bool any_tokens, bool any_rows) {
  const DebugOptions &d = debug_options();
  const bool forced = d.gemm_generic.load(std::memory_order_relaxed) != 0 || d.tile.load(std::memory_order_relaxed) >= 0 ||
                      d.fwd_pair.load(std::memory_order_relaxed) >= 0 || d.fused_gather.load(std::memory_order_relaxed) >= 0 ||
                      d.poison_staging.load(std::memory_order_relaxed) != 0;  // (these ask for the staged schedule)
  const bool fits = shards_are_k_blocks(lay) || (lay.rows_per_shard > 0 && any_rows && (lay.N == 1 || lay.rows_per_shard % 8 == 0));
  return !forced && (any_tokens || T <= kShardReadMaxTokens) && fits && ld_act < kMaxLd && lay.O < kMaxLd;
}

int gemm_forward_parts(int64_t M, int64_t K) { return forward_k_parts(M, K); }

bool gemm_takes_two_segments(int64_t k_first, int64_t k_second) {
  return k_first > 0 && k_second > 0 && fast_path(static_cast<int>(k_first + k_second), static_cast<int>(k_first), 0);
}

bool gemm_takes_two_column_segments(int64_t n_first, int64_t n_second, int64_t K) {
  return n_first > 0 && n_second > 0 && fast_path(static_cast<int>(K), 0, static_cast<int>(n_first));
}

double gemm_estimate_us(int64_t M, int64_t N, int64_t K, bool forward_parts) {
  // one CU sustains about 5e6 flop per microsecond (1.3 PFLOP/s over 256 CUs) on 256 x 256 tiles
  // (one launch on its best tile: pricing the whole-rounds + remainder pair here instead was measured and made the
  // forward launch grouping of config 3 slightly worse)
  double cost = 0.0;
  if (M > 0 && fast_path(static_cast<int>(K), 0, 0)) {
    // (how slices are paired decides how much workspace a call asks for: it goes by the shapes that sizes were first given for)
    best_tile(static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), 0, 0, &cost, 1, TileUse::kFirstShapes);
    const int parts = forward_parts ? forward_k_parts(M, K) : 1;
    if (parts > 1) {
      best_tile(static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), 0, 0, &cost, parts, TileUse::kFirstShapes);
      return cost / parts * 2.0 * static_cast<double>(K) / 5.0e6 + combine_estimate_us(M, N, parts) + 6.0;
    }
    return cost * 2.0 * static_cast<double>(K) / 5.0e6 + 6.0;
  }
  const double tiles = static_cast<double>((M + GBM - 1) / GBM) * static_cast<double>((N + GBN - 1) / GBN);
  const double rounds = static_cast<double>(static_cast<long>((tiles + kCUs - 1) / kCUs));
  return rounds * GBM * GBN * 5.0 * 2.0 * static_cast<double>(K) / 5.0e6 + 6.0;  // the checked kernel is about 5x slower per tile
}

double gemm_planned_us(int64_t M, int64_t N, int64_t K, bool dx, bool acc_in) {
  if (M <= 0 || !fast_path(static_cast<int>(K), 0, 0)) return gemm_estimate_us(M, N, K);
  int axis, cut;
  const double cost = plan_launches(static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), dx ? 2 : 0, acc_in, &axis, &cut);
  return cost * 2.0 * static_cast<double>(K) / 5.0e6 + 6.0;
}

namespace {
thread_local int64_t t_persistent_launches = 0;
}  // namespace
double gemm_shards_dx_us(int64_t M, int64_t N, int64_t K, int64_t shard_rows) {
  int axis, cut;
  const double cost = plan_launches(static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), 2, false, &axis, &cut, static_cast<int>(shard_rows));
  return cost * 2.0 * static_cast<double>(K) / 5.0e6 + 6.0;
}

int64_t gemm_persistent_launches() { return t_persistent_launches; }
void gemm_count_persistent_launch() { t_persistent_launches += 1; }

size_t gemm_forward_parts_bytes(int64_t M, int64_t N, int64_t K) {
  const int parts = forward_k_parts(M, K);
  return parts > 1 && N > 0 ? static_cast<size_t>(parts) * static_cast<size_t>(M) * static_cast<size_t>(N) * 4 : 0;
}

hipError_t check_device() {
  static std::atomic<int8_t> verdict[kMaxDevices] = {};  // 0: not looked at, 1: fits, -1: does not
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  int8_t v = verdict[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    int cus = 0, xcds = 0;
    if ((e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev)) != hipSuccess) return e;
    if ((e = hipDeviceGetAttribute(&xcds, hipDeviceAttributeNumberOfXccs, dev)) != hipSuccess) return e;
    v = (cus == kCUs && xcds == kXcds) ? 1 : -1;
    verdict[dev].store(v, std::memory_order_relaxed);
  }
  return v > 0 ? hipSuccess : hipErrorInvalidDevice;
}

namespace {
hipError_t dispatch_gemm(const GemmProblem &q, hipStream_t stream, bool *carry) {
  GemmParams p;
  const hipError_t e = launch_params(q, *carry, &p);
  if (e != hipSuccess) return e;
  if ((p.k_split || p.n_split) && !q.a_kcontig) return hipErrorInvalidValue;  // dW never takes a second segment
  if (p.k_split && p.n_split) return hipErrorInvalidValue;
  float *planes = static_cast<float *>(q.parts);
  const size_t planes_bytes = q.parts_bytes;
  constexpr int kRow = static_cast<int>(Epilogue::kBf16RowMajor), kShard = static_cast<int>(Epilogue::kBf16ShardMajor),
                kF32 = static_cast<int>(Epilogue::kF32Workspace);
  const bool acc = q.acc_in != nullptr;
  if (q.epilogue == Epilogue::kBf16Fused) {
    if (!q.a_kcontig || q.b_kcontig) return hipErrorInvalidValue;
    if (acc || p.k_split || !planes || q.k_per <= 0 || q.k_per >= p.K) return launch_gemm_fused(q, stream, carry);
    const hipError_t ep = launch_parts<true, false>(p, q.k_per, planes, planes_bytes, stream, carry);
    return ep != hipSuccess ? ep : launch_combine_fused(q, (p.K + q.k_per - 1) / q.k_per, planes, stream);
  }
  if (q.k_per > 0) {  // (behind the pass for dZ: parts by the caller's rule, or none)
    if (acc || p.k_split || !planes || q.k_per >= p.K || q.a_kcontig != q.b_kcontig) {
      planes = nullptr;
    } else {
      const int parts = (p.K + q.k_per - 1) / q.k_per;
      const hipError_t ep = q.a_kcontig ? launch_parts<true, true>(p, q.k_per, planes, planes_bytes, stream, carry)
                                        : launch_parts<false, false>(p, q.k_per, planes, planes_bytes, stream, carry);
      if (ep != hipSuccess) return ep;
      if (q.epilogue == Epilogue::kBf16ShardMajor) return launch_combine<kShard>(p, parts, planes, stream);
      return q.epilogue == Epilogue::kBf16RowMajor ? launch_combine<kRow>(p, parts, planes, stream) : hipErrorInvalidValue;
    }
  }
  // The three GEMMs of the split linear layer, with the four accumulate forms for forward and dX, are the only combinations built.
  if (q.a_kcontig && !q.b_kcontig) {                                               // forward (accumulating when the reduction dimension is split)
    if (q.epilogue == Epilogue::kBf16RowMajor) return acc ? launch_planned<true, false, kRow, true>(p, stream, carry, planes, planes_bytes) : launch_planned<true, false, kRow, false>(p, stream, carry, planes, planes_bytes);
    if (q.epilogue == Epilogue::kF32Workspace) return acc ? launch_planned<true, false, kF32, true>(p, stream, carry, planes, planes_bytes) : launch_planned<true, false, kF32, false>(p, stream, carry, planes, planes_bytes);
  }
  if (!q.a_kcontig && !q.b_kcontig && !acc) {                                      // dW: into the shards, or (DP slice) a plain array
    if (q.epilogue == Epilogue::kBf16ShardMajor) return launch_planned<false, false, kShard, false>(p, stream, carry, planes, planes_bytes);
    if (q.epilogue == Epilogue::kBf16RowMajor) return launch_planned<false, false, kRow, false>(p, stream, carry, planes, planes_bytes);
  }
  if (q.a_kcontig && q.b_kcontig) {                                                // dX
    if (q.epilogue == Epilogue::kBf16RowMajor) return acc ? launch_planned<true, true, kRow, true>(p, stream, carry, planes, planes_bytes) : launch_planned<true, true, kRow, false>(p, stream, carry, planes, planes_bytes);
    if (q.epilogue == Epilogue::kF32Workspace) return acc ? launch_planned<true, true, kF32, true>(p, stream, carry, planes, planes_bytes) : launch_planned<true, true, kF32, false>(p, stream, carry, planes, planes_bytes);
  }
  return hipErrorInvalidValue;
}
}  // namespace

bool skinny_takes(bool dx, int64_t T, int64_t ld_act, const ShardLayout &lay, int64_t I) {
  // (the switches that pick a kernel or a tile for the staged products keep those)
  const DebugOptions &d = debug_options();
  if (T <= 0 || T > kSkinnyMaxTokens || ld_act >= kMaxLd || I >= kMaxLd || lay.O >= kMaxLd ||
      d.gemm_generic.load(std::memory_order_relaxed) != 0 || d.tile.load(std::memory_order_relaxed) >= 0)
    return false;
  const int64_t N = dx ? I : lay.O, K = dx ? lay.O : I;
  return !(T > kSkinnyMaxWideTokens && N > kSkinnyMaxColumns && shards_are_k_blocks(lay) && forward_k_parts(T, K) == 1);
}

hipError_t launch_skinny(bool dx, const WeightMap &w, int64_t T, const void *act, int64_t ld_act, void *out, int64_t ld_out,
                         hipStream_t stream) {
  const SkinnyParams p = skinny_params(dx, w, T, act, ld_act, out, ld_out);
  if (dx) {
    const int bm = skinny_rows(T, p.N);
    if (bm == 16) return launch_skinny_as<16, 64, 64, 3, true>(p, stream);
    if (bm == 32) return launch_skinny_as<32, 64, 64, 3, true>(p, stream);
    if (bm <= 64) return launch_skinny_as<64, 64, 64, 2, true>(p, stream);
    return launch_skinny_as<128, 64, 32, 3, true>(p, stream);
  }
  return launch_skinny_forward<SkinnyResult::kPlain>(p, skinny_rows(p.M, p.N), stream);
}

namespace {
template <int BM, int BK, int kStages>
hipError_t launch_backward_as(SkinnyParams dx, const GemmParams &dw, hipStream_t stream) {
  constexpr size_t lds_dx = static_cast<size_t>(kSkinnyWaves) * kStages * (BM + 64) * BK * sizeof(uint16_t);
  constexpr size_t lds_dw = 4 * (W4Operand<false, 4>::kElems + W4Operand<false, 4>::kElems) * sizeof(uint16_t);
  constexpr size_t lds = lds_dx > lds_dw ? lds_dx : lds_dw;
  static_assert(lds + 3 * OSDP_MAX_SHARDS * 8 <= 160 * 1024, "the rings do not fit the 160 KB of LDS");
  auto kernel = few_token_backward_kernel<BM, BK, kStages>;
  static bool configured[kMaxDevices] = {};
  const hipError_t e = allow_lds(kernel, lds, configured);
  if (e != hipSuccess) return e;
  dx.tiles_m = (dx.M + BM - 1) / BM;
  dx.by_lane = skinny_by_lane<64, BK, true>(dx.w);
  const int n_dx = dx.tiles_m * ((dx.N + 63) / 64), tiles_m = (dw.M + 127) / 128, tiles_n = (dw.N + 127) / 128;
  hipLaunchKernelGGL(kernel, dim3(n_dx + tiles_m * tiles_n), dim3(256), lds, stream, dx, dw, n_dx, tiles_m, tiles_n);
  return hipGetLastError();
}
}  // namespace

namespace {
// Rows of a workgroup's tile of dX beside n_dw tiles of dW: for the CUs that these leave, or a quarter of all where they leave
// fewer.  us for tiles chosen for a quarter / a half / all of the CUs: 128 tokens 1024 -> 3072 12.2 / 13.5 / 13.5, 1024 -> 4096 14.2 /
// 15.2 / 15.2; 64 tokens 3072 -> 768 7.2 / 7.4 / 9.9; 128 tokens 2048 -> 2048 12.8 / 11.3 / 18.4; over 90 calls of 16 to 128 tokens
// (two launches: 1) 0.72 / 0.70 / 0.74.
int beside_rows(int64_t T, int64_t N, int64_t n_dw) { return skinny_rows(T, N, static_cast<int>(std::max<int64_t>(kCUs - n_dw, kCUs / 4))); }
}  // namespace

// us, two launches / one: 128 tokens 256 -> 1024 10.7 / 5.8, 1536 -> 1536 12.3 / 8.6, 2048 -> 2048 13.9 / 12.4, 512 -> 8192
// 24.7 / 19.5, 16 tokens 1024 -> 4096 16.5 / 11.9.  Two launches are kept for more than 64 tokens and so many in-features that tiles of dX
// with all rows make more than one round with those of dW: 128 tokens 4096 -> 1024 13.7 against 15.7 for one launch with such tiles (of 64
// rows, as one launch has now, 10.4; 8192 -> 512 13.5 and 12.5: the line could move).
bool few_token_backward_takes(const GemmProblem &dw, int64_t T) {
  const DebugOptions &d = debug_options();
  const GemmParams p = gemm_params(dw);
  int axis = -1, cut = 0;
  if (dw.epilogue != Epilogue::kBf16ShardMajor || !fast_path(p.K, 0, 0) || !fits_offsets(p) || tile_count(p.M, p.N, 128, 128) > kCUs ||
      d.deep.load(std::memory_order_relaxed) == 0 || d.small_tile.load(std::memory_order_relaxed) == 1 ||
      best_tile(p.M, p.N, p.K, 0, 1, nullptr) != 3)
    return false;
  plan_launches(p.M, p.N, p.K, 1, false, &axis, &cut);
  if (axis >= 0) return false;
  const int64_t n_dw = tile_count(p.M, p.N, 128, 128), bm = beside_rows(T, p.M, n_dw);
  return bm <= 64 || n_dw + (T + bm - 1) / bm * ((p.M + 63) / 64) <= kCUs;
}

hipError_t launch_few_token_backward(const GemmProblem &dw, const WeightMap &w, int64_t T, const void *dY, int64_t lddy, void *dX,
                                     int64_t lddx, hipStream_t stream) {
  const SkinnyParams p = skinny_params(true, w, T, dY, lddy, dX, lddx);
  const GemmParams g = gemm_params(dw);
  const int bm = beside_rows(T, p.N, tile_count(g.M, g.N, 128, 128));
  if (bm == 16) return launch_backward_as<16, 64, 3>(p, g, stream);
  if (bm == 32) return launch_backward_as<32, 64, 3>(p, g, stream);
  // (never 128 rows: their tile is the longest of the launch by far.  us as two launches / one with 128 rows / one with 64, 128
  // tokens: 3072 -> 1024 13.4 / 16.3 / 10.0, 2560 -> 1280 14.0 / 18.3 / 10.5)
  return launch_backward_as<64, 64, 2>(p, g, stream);
}

hipError_t launch_gemm(const GemmProblem &q, hipStream_t stream) {
  if (q.M < 0 || q.N < 0 || q.K < 0) return hipErrorInvalidValue;
  const GatherRequest *g = q.carry;
  const bool has_gather = g && g->rows > 0 && g->w > 0;
  if (has_gather && !q.carried) return hipErrorInvalidValue;  // the caller must learn whether the gather is still to do
  bool carry = has_gather;
  if (q.M > 0 && q.N > 0) {  // else nothing to write; K == 0 still writes the empty sum
    const hipError_t e = dispatch_gemm(q, stream, &carry);
    if (e != hipSuccess) return e;
  }
  if (q.carried) *q.carried = has_gather && !carry;
  return hipSuccess;
}

}  // namespace osdp
