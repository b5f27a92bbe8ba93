// Host side of the GEMM (kernels: sp24_gemm_kernel.cuh): tensor maps, tile choice, argument checks, entry points.
#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <mutex>

#include "sp24_gemm.cuh"

namespace sp24 {
namespace {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  });
  return fn;
}

using EncodeIm2colFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const int*, const int*, cuuint32_t, cuuint32_t, const cuuint32_t*,
                                    CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                    CUtensorMapFloatOOBfill);

EncodeIm2colFn encode_im2col_fn() {
  static EncodeIm2colFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeIm2col", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeIm2colFn>(ptr);
  });
  return fn;
}

}  // namespace

// im2col tensor map over an NHWC activation for a 3x3, stride-1, pad-1 convolution: the bounding box
// of the filter's anchor starts one pixel before the image and ends one pixel before its far edge, so
// that anchor + tap (0..2) covers rows/columns -1 .. H, W with zeros outside.
sp24_status make_im2col_map(CUtensorMap* map, const void* x, int es, uint64_t nb, uint64_t h, uint64_t w, uint64_t c,
                            uint32_t channels_per_box, uint32_t pixels_per_box) {
  EncodeIm2colFn fn = encode_im2col_fn();
  if (!fn) return SP24_ERR_CUDA;
  cuuint64_t dims[4] = {c, w, h, nb};
  cuuint64_t strides[3] = {c * es, w * c * es, h * w * c * es};
  int lower[2] = {-1, -1}, upper[2] = {-1, -1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUtensorMapDataType dt = es == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  CUresult r = fn(map, dt, 4, const_cast<void*>(x), dims, strides, lower, upper, channels_per_box, pixels_per_box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SP24_OK : SP24_ERR_CUDA;
}

namespace {

sp24_status encode_map(CUtensorMap* map, const MapShape& m) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return SP24_ERR_CUDA;
  const cuuint64_t dims[3] = {m.dims[0], m.dims[1], m.dims[2]}, strides[2] = {m.strides[0], m.strides[1]};
  const cuuint32_t box[3] = {m.box[0], m.box[1], m.box[2]}, estr[3] = {1, 1, 1};
  CUtensorMapDataType dt = m.es == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32
                                     : (m.es == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8);
  CUtensorMapSwizzle sw = m.swizzle == kSwizzle128Atom32
                              ? CU_TENSOR_MAP_SWIZZLE_128B_ATOM_32B
                              : (m.swizzle == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE);
  CUresult r = fn(map, dt, m.dims[2] ? 3 : 2, const_cast<void*>(m.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SP24_OK : SP24_ERR_CUDA;
}

// Host-side cache of encoded tensor maps.  A map is a pure function of (address, shape, leading
// dimension, element size, box, swizzle): a layer that is multiplied again with the same buffers
// finds its maps (three, five with a staged epilogue) here instead of encoding them again.  One small table per host thread (no
// lock), replaced round-robin.
struct MapCache {
  static constexpr int kEntries = 32;
  MapShape keys[kEntries];
  CUtensorMap maps[kEntries];
  int used = 0, next = 0;
};

}  // namespace

sp24_status make_map(CUtensorMap* map, const MapShape& key) {
  static thread_local MapCache cache;
  for (int i = 0; i < cache.used; ++i)
    if (cache.keys[i] == key) {
      *map = cache.maps[i];
      return SP24_OK;
    }
  sp24_status st = encode_map(map, key);
  if (st != SP24_OK) return st;
  const int slot = cache.used < MapCache::kEntries ? cache.used++ : (cache.next++ % MapCache::kEntries);
  cache.keys[slot] = key;
  cache.maps[slot] = *map;
  return SP24_OK;
}

int sm_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 1;
  const bool cacheable = dev >= 0 && dev < 64;
  if (cacheable && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 1;
  if (cacheable) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

namespace {

// Process-wide settings: the benchmarking overrides (environment, read once, or sp24_set_tile_override)
// and the fault-path test hooks (sp24_test_set_fault_hooks only; never read from the environment).
struct Settings {
  std::atomic<int> ctas{0}, block_n{0}, mblk{0}, band{0}, log{0};
  std::atomic<long long> test_wait_cycles{0};
  std::atomic<int> test_skip_stage{0};
};
Settings& settings() {
  static Settings st;
  static std::once_flag once;
  std::call_once(once, [] {
    if (const char* env = getenv("SP24_TILE")) {
      int c = 0, n = 0, m = 1;
      if (sscanf(env, "%dx%dx%d", &c, &n, &m) >= 2) { st.ctas = c; st.block_n = n; st.mblk = m; }
    }
    if (const char* env = getenv("SP24_BAND")) st.band = atoi(env) > 0 ? atoi(env) : 0;
    if (const char* env = getenv("SP24_LOG")) st.log = atoi(env) != 0 || env[0] == '\0' ? 1 : 0;
  });
  return st;
}

}  // namespace

// Test hooks for the failure path (set through sp24_test_set_fault_hooks only): a shorter limit, and a
// pipeline that stalls by leaving out one k-block.  Nothing faults or hangs: the waits expire and the
// kernel returns.
void set_wait_limit(GemmParams& p) {
  Settings& cfg = settings();
  p.wait_limit = kWaitTimeoutCycles;
  const long long v = cfg.test_wait_cycles.load(std::memory_order_relaxed);
  if (v >= 1000000) p.wait_limit = v;
  p.test_skip_stage = cfg.test_skip_stage.load(std::memory_order_relaxed);
}

void forced_tile(int* ctas, int* block_n, int* mblk) {
  Settings& cfg = settings();
  *ctas = cfg.ctas.load(std::memory_order_relaxed);
  *block_n = cfg.block_n.load(std::memory_order_relaxed);
  *mblk = cfg.mblk.load(std::memory_order_relaxed);
}
}  // namespace sp24

using namespace sp24;

extern "C" size_t sp24_gemm_workspace_bytes(const sp24_gemm_desc* d) {
  (void)d;
  return 256;
}

// Whether tall tiles beat pairs of CTAs on `blocks` 128-row blocks and at most 128 columns.  They stream A better but
// nothing hides their epilogue, so they lose where the output is wide next to A.  `out`: bytes of an output row; with
// C or column-major, where a byte of it costs more, the limits are lower.  In one round of tiles the limits hardly
// depend on K (short: all of it is launch and epilogue either way; long: the stream decides); with more rounds each
// round's epilogue counts, least on a short K in two rounds of two blocks, and on a long K a last round that leaves
// SMs idle does.
// Measured over 19200..98304 rows x 16..128 columns x 512..12288, every kind, order and C (3960 calls, tall tiles and
// pairs on each; us, pairs against tall): bf16 -> bf16 49152 x 32 x 12288 123.8 / 104.1, 37888 x 64 x 512 11.4 / 7.5;
// bf16 -> f32 49152 x 128 x 512 row-major 13.7 / 14.2, with C 17.3 / 20.8; int8 -> int32 98304 x 128 x 1024 23.5 / 29.1;
// bf16 -> bf16 60000 x 128 x 12288 154.3 / 174.4, TF32 60000 x 96 x 1024 38.5 / 38.3,
// 49152 x 128 x 4096 94.3 / 86.9.  The rule is 0.5 % off the better of the two in the mean.
static bool tall_tiles_pay(const sp24_gemm_desc* d, bool has_c, int64_t blocks, int64_t sms, int mblk, int64_t chain) {
  const int64_t out = d->N * elem_bytes(d->cd_type), k_bytes = d->K * elem_bytes(d->ab_type);
  const bool plain = d->order_d == SP24_ROW_MAJOR && !has_c, short_k = k_bytes <= 2048;
  if (blocks <= sms * mblk) {  // one round
    if (k_bytes >= (plain ? 12288 : 24576) || (plain && short_k)) return out <= 512;
    return out <= (plain ? 384 : 256);
  }
  if (k_bytes >= 12288 && 5 * sms * chain > 6 * blocks) return false;  // the last round leaves SMs idle
  if (plain && k_bytes <= 8192 && chain <= 4) return out <= (short_k ? 512 : 384);
  if (elem_bytes(d->ab_type) == 1 && short_k && chain <= 4) return out <= 256;
  return d->N <= 96 && out <= (has_c ? 170 : 256);
}

// Tile choice.  At most 128 columns: see below.  Small problems: single CTAs, 128 x 128 tiles.  Otherwise a
// pair of CTAs, and among the pair shapes the one with the smallest estimated time = rounds of tiles over
// the pairs x time of one tile.  The tile times are measured ratios (unit: one 256 x 224 tile per unit of K;
// interleaved runs on 2048..8192-row problems with K = 4096..16384):
//   256 x 224, two accumulator buffers (epilogue overlapped)      K                 the reference
//   256 x 240, the same (16-bit kinds, 16-bit output)              1.04 K            operand bytes per k
//   256 x 256, one accumulator buffer (epilogue exposed)           1.09 K + 450
//   512 x 224, two m-blocks per CTA share a B tile (epilogue exposed): twice the work in
//              1.65 K + 1150 (16-bit kinds), 1.80 K + 820 (8-bit floats), 1.98 K + 200 (int8 -> int32)
// (224: two fp32 accumulators plus the metadata columns fit the 512 columns of tensor memory and 224 is a
// multiple of 32; 240 is the widest multiple of 16 that fits.)  The dense variant: two m-blocks from six
// waves of tiles on, 512 x 256 there (no metadata columns needed); below that the one-m-block width with
// the fewest rounds.
static void choose_tile(const sp24_gemm_desc* d, bool has_c, bool conv, int& ctas, int& block_n, int& mblk) {
  const int64_t n224 = (d->N + 223) / 224;
  const bool k_major_b = d->order_b == SP24_COL_MAJOR;
  ctas = 1; block_n = 128; mblk = 1;
  if (!d->a_is_dense && k_major_b && d->N <= 128) {
    // One column of tiles: all of A is streamed once, and what counts is how evenly its 128-row blocks are spread
    // over the SMs.  Up to one block per SM: single blocks (us: 12288 x 32 x 4096 bf16 14.9 against 16.0 with
    // pairs of CTAs, 12288 x 128 x 12288 40.6 against 43.1).  Beyond, if they pay: tall tiles of the two or three
    // blocks that give the fewest blocks in a row on one SM, three if equal (B is loaded once per tile).
    const int64_t sms = sm_count(), blocks = (d->M + kBlockM - 1) / kBlockM;
    if (blocks <= sms || conv) return;  // (tall tiles load no im2col view)
    const int64_t chain2 = 2 * ((blocks + 2 * sms - 1) / (2 * sms)), chain3 = 3 * ((blocks + 3 * sms - 1) / (3 * sms));
    const int tall = chain2 < chain3 ? 2 : 3;
    if (tall_tiles_pay(d, has_c, blocks, sms, tall, chain2 < chain3 ? chain2 : chain3)) {
      mblk = tall;
      return;
    }
  }
  if (d->M < 256 || (d->M / 256) * n224 < 32) return;
  ctas = 2; block_n = 224;
  const int64_t pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
  const bool bits16 = d->ab_type == SP24_F16 || d->ab_type == SP24_BF16;
  const bool has_240 = bits16 && k_major_b && elem_bytes(d->cd_type) == 2;
  if (d->a_is_dense) {
    if (d->M >= 512 && (d->M / 512) * n224 >= 444) {
      mblk = 2;
      // two 256-column accumulators fill tensor memory exactly: 9 % fewer operand bytes per flop than 512 x 224
      if (k_major_b && d->ab_type != SP24_F32) block_n = 256;
      return;
    }
    // one m-block: the width that needs the fewest rounds of tiles, operand bytes per k as the tie-break
    // (without metadata columns two 256-column accumulators fit, so 256 x 256 keeps its epilogue overlapped; with N contiguous
    // it loads the two 128-byte chunks of B to a CTA that 224 columns need as well: bf16 4096 x 2048 x 8192 114 -> 96 us)
    const int widths[3] = {224, has_240 ? 240 : 0, d->ab_type != SP24_F32 ? 256 : 0};
    double best = 0.0;
    for (const int bn : widths) {
      if (bn == 0) continue;
      const int64_t tiles = ((d->M + 255) / 256) * ((d->N + bn - 1) / bn);
      const double cost = (double)((tiles + pairs - 1) / pairs) * (256.0 + bn);
      if (best == 0.0 || cost < best) { best = cost; block_n = bn; }
    }
    return;
  }
  const double K = (double)d->K;
  const double two_a = d->ab_type == SP24_I8 ? 1.98 : (is_fp8(d->ab_type) ? 1.80 : 1.65);
  const double two_b = d->ab_type == SP24_I8 ? 200.0 : (is_fp8(d->ab_type) ? 820.0 : 1150.0);
  struct Candidate { int block_n, mblk; bool built; double tile_time; };
  const Candidate candidates[4] = {
      {224, 2, d->M >= 512, two_a * K + two_b},
      {224, 1, true, K},
      {240, 1, has_240, (144.0 + 240.0) / (144.0 + 224.0) * K},
      {256, 1, k_major_b && (bits16 || d->N <= 2048), (144.0 + 256.0) / (144.0 + 224.0) * K + 450.0},
  };
  double best = 0.0;
  for (const Candidate& c : candidates) {
    if (!c.built) continue;
    const int64_t rows = 256 * c.mblk;
    const int64_t tiles = ((d->M + rows - 1) / rows) * ((d->N + c.block_n - 1) / c.block_n);
    const double cost = (double)((tiles + pairs - 1) / pairs) * c.tile_time;
    if (best == 0.0 || cost < best) { best = cost; block_n = c.block_n; mblk = c.mblk; }
  }
}

// Clusters of 2^log single CTAs that the device holds at one time (a GPC may end in SMs that make no whole cluster), 0 if it
// holds none; every GEMM CTA fills its SM.  Asked once per device.  A query that fails is not an answer: -1, and the next call
// asks again.
__global__ void cluster_probe() {}
static int split_clusters(int log) {
  static std::atomic<int> known[64][4];  // the answer + 1
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return -1;
  const bool cacheable = dev >= 0 && dev < 64;
  if (cacheable && (n = known[dev][log].load(std::memory_order_relaxed)) > 0) return n - 1;
  constexpr int smem = 227 * 1024;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1u << log;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.gridDim = dim3(1u << log);
  cfg.blockDim = dim3(kNumThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cuda_status(cudaFuncSetAttribute(cluster_probe, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != SP24_OK ||
      cuda_status(cudaOccupancyMaxActiveClusters(&n, cluster_probe, &cfg)) != SP24_OK || n < 0)
    return -1;
  if (cacheable) known[dev][log].store(n + 1, std::memory_order_relaxed);
  return n;
}

// Time of a product with tiles of (128 * ctas * mblk) x tile_n, us on an idle chip: start, and per round of tiles the
// k-blocks (a fixed part and one per column, the same for all kinds: a k-block is 256 bytes of K), then the epilogue of a
// tile by its columns (4-byte results and C cost more; 256-column tiles and two m-blocks cannot overlap it).  Fitted to
// 170 random problems (256..16384 rows, 160..16384 columns, K 256..12288, every kind, with and without C), 11 to 17
// shapes of each, before stages held two k-blocks: it puts bf16 512 x 512 x 8192 at 16.5 us, which now takes 13.1.  On 100
// other problems of the same ranges the mean error of later kernels is 9 to 13 % per shape, 16 % for two m-blocks.  (An int8
// result counts as a 16-bit one: the fit is older than its arithmetic by pairs and its twelve warps.)
// split_log: the CTAs of a cluster share the k-blocks.
static double tile_time(const sp24_gemm_desc* d, bool has_c, int ctas, int block_n, int mblk, int tile_n, int split_log = 0) {
  const int bytes = elem_bytes(d->ab_type), cs = elem_bytes(d->cd_type);
  const int es = bytes > 0 ? bytes : 1;  // (a type that no product takes may still ask for its plan)
  const double k_blocks = (double)((((d->K * es + 255) >> 8) + (1 << split_log) - 1) >> split_log);
  const int64_t rows = 128 * ctas * mblk, slots = sm_count() / ctas > 0 ? sm_count() / ctas : 1;
  const int64_t tiles = ((d->M + rows - 1) / rows) * ((d->N + tile_n - 1) / tile_n);
  const double rounds = (double)((tiles + slots - 1) / slots), w = tile_n / 100.0;
  double loaded = w;  // with N contiguous, B comes in chunks of 128 bytes along N
  if (d->order_b == SP24_ROW_MAJOR) loaded = (double)((tile_n / ctas * es + 127) / 128 * (128 / es) * ctas) / 100.0;
  const double store = cs == 4 ? (has_c ? 2.0 : 1.0) : (has_c ? 1.4 : 0.6);
  if (ctas == 1) return 2.4 + rounds * (k_blocks * (0.18 + 0.11 * loaded) + 0.12 + store * w);
  if (mblk == 2) return 1.6 + 1.08 * rounds * (k_blocks * (es == 4 ? 0.68 : 0.59) + 0.6 + 2.6 * store * w);
  if (block_n == 256) return 1.5 + rounds * (k_blocks * 0.156 * w + (0.5 + store) * w);
  if (block_n == 240) return 2.2 + rounds * (k_blocks * 0.151 * w + 1.1 * store * w);
  return 2.6 + rounds * (k_blocks * (0.165 + 0.085 * loaded) + 0.1 + store * w);
}

// Columns of a tile.  choose_tile() knows the widest form of each shape; a problem that leaves SMs idle in a round of
// tiles is faster with narrower ones on more of them (us, device: f16 256 x 256 x 512 4.10 -> 3.23, f16 1184 x 736 x 1008
// with C 7.6 -> 5.8, int8 992 x 480 x 6176 14.9 -> 9.5, bf16 512 x 192 x 10464 31.2 -> 19.8).  Over 150 other random
// problems the choice below is 17 % faster in the mean than the widest tiles, one is slower by more than 2 % (int8 128 x
// 3808 x 352 4.5 -> 4.7 us); it is 1.5 % behind the best of the shapes over the 170 above, 2.3 % (at worst 22 %) over the 100.
// A pair keeps its shape unless the estimate says 3 %, its two m-blocks unless it says 15 %: it puts those 12 % too high.
//
// INT32 accumulators of single CTAs: a cluster of 2, 4 or 8 of them may share the k-blocks of a tile (split_log), which the
// estimate has as its k-blocks in so many parts and the exchange of the accumulators, by their columns.  Where few tiles
// have many k-blocks this uses SMs that have none; the sums are integers, the same in any order, so the result does not
// depend on it (those of floating-point kinds would).  Us, device, one CTA to a tile and the choice: 4096 x 32 x 4096 5.7, 4.5;
// 512 x 512 x 8192 9.0, 6.3; 256 x 256 x 12288 12.2, 5.9; 1056 x 32 x 10816 with C 11.4, 5.0; 2048 x 64 x 2048 4.2, 4.2.
// The exchange was set from a few shapes (0.7 us for 2 CTAs, 1.2 for 4, 1.5 for 8 at 32 columns), the 4 % so that nearly equal
// ones are not split.  Over 100 random int8 products (64..9000 rows, 32..2000 columns, K 512..12288, up to 74 tiles of 128 x 128,
// every result type), at every width and number of parts, the mean error of the estimate is 9 % for 2 parts and 11 % for 4 and
// 8 (one: 10 %); the choice is 0.9 % behind the best (at worst 14 %), and 1.20 times as fast as the best unsplit one in the mean.
// False if the device did not say how many clusters it holds: nothing is split then, and the choice is not to be kept.
static bool choose_width(const sp24_gemm_desc* d, bool has_c, bool conv, int& ctas, int& block_n, int& mblk, int& tile_n, int& split_log) {
  split_log = 0;
  bool answered = true;
  const int64_t n32 = (d->N + 31) / 32 * 32;
  auto widest = [&](int bn) { return n32 < bn ? (int)n32 : bn; };
  tile_n = widest(block_n);
  // Room for clusters.  Every INT8 product that has the kernels with the split beside its own asks, also where nothing will be
  // split: a program's first call, before it captures a stream, is then the one that loads the probe.
  int room[4] = {};
  if (d->ab_type == SP24_I8 && !d->a_is_dense && d->order_b == SP24_COL_MAJOR)
    for (int log = 1; log <= 3; ++log)
      if ((room[log] = split_clusters(log)) < 0) answered = false;
  if (ctas == 1 && mblk > 1) {  // tall tiles: all the columns there are
    if (d->N < tile_n) tile_n = (int)d->N;
    return answered;
  }
  if (ctas == 2 && (d->a_is_dense || d->N <= 128)) return answered;
  const double now = tile_time(d, has_c, ctas, block_n, mblk, ctas == 2 ? block_n : tile_n);
  double best = now * (ctas == 1 ? 1.0 : mblk == 2 ? 0.85 : 0.97);
  auto try_shape = [&](int c, int bn, int tn) {
    const double t = tile_time(d, has_c, c, bn, 1, tn);
    if (t < best) { best = t; ctas = c; block_n = bn; mblk = 1; tile_n = tn; split_log = 0; }
  };
  const bool pairs = !d->a_is_dense && d->N > 128 && d->M >= 256 && (d->M / 256) * ((d->N + 223) / 224) >= 4;
  const bool k_major_b = d->order_b == SP24_COL_MAJOR, one = ctas == 1;
  const bool has_240 = k_major_b && elem_bytes(d->ab_type) == 2 && elem_bytes(d->cd_type) == 2;
  if (d->ab_type == SP24_I8 && !d->a_is_dense && d->order_b == SP24_COL_MAJOR && !conv) {
    const int64_t blocks = (d->M + kBlockM - 1) / kBlockM, k_blocks = (d->K + 255) / 256;
    for (int w = widest(128); w > 0; w -= 32) {
      const int64_t tiles = blocks * ((d->N + w - 1) / w);
      for (int log = 1; log <= 3 && k_blocks >= 2 << log; ++log) {
        if (tiles > (sm_count() >> log) || tiles > room[log]) break;
        const double columns = w / 100.0, exchange = log == 1 ? 0.4 + columns : (log == 2 ? 0.5 : 0.9) + 2.0 * columns;
        const double t = 1.04 * (tile_time(d, has_c, 1, 128, 1, w, log) + exchange);
        if (t < best) { best = t; ctas = 1; block_n = 128; mblk = 1; tile_n = w; split_log = log; }
      }
    }
  }
  if (!one) try_shape(1, 128, widest(128));
  for (int w = 96; w >= 32; w -= 32)
    if (w < n32) try_shape(1, 128, w);
  if (!pairs) return answered;
  for (int w = 224; w >= 64; w -= 32) try_shape(2, 224, widest(w));
  if (has_240) try_shape(2, 240, 240);
  if (k_major_b) try_shape(2, 256, widest(256));
  return answered;
}

// The shape, width and split of a product, a pure function of what is compared here and of the device.  The last ones of a
// host thread are kept: the estimates take 0.3 to 0.8 us of host time, and a short call is bound by that (f16 256 x 256 x 512
// in a loop 5.36 -> 5.10; int8 4096 x 32 x 4096 5.57 -> 5.18).  These are loops over one product: a first call of a shape has
// the estimate as before, and a thread with more than sixteen in rotation the search as well (up to 0.1 us).
struct Choice {
  int device, ab, cd, order_b, order_d, dense, has_c, conv;
  int64_t M, N, K;
  bool operator==(const Choice& o) const {
    return M == o.M && N == o.N && K == o.K && ab == o.ab && cd == o.cd && order_b == o.order_b && order_d == o.order_d &&
           dense == o.dense && has_c == o.has_c && conv == o.conv && device == o.device;
  }
};
static TileShape choose(const sp24_gemm_desc* d, bool has_c, bool conv) {
  constexpr int kKept = 16;
  static thread_local struct {
    Choice key[kKept];
    TileShape shape[kKept];
    int used, next;
  } kept;
  Choice key = {-1, (int)d->ab_type, (int)d->cd_type, (int)d->order_b, (int)d->order_d, d->a_is_dense, has_c, conv, d->M, d->N, d->K};
  const bool known = cudaGetDevice(&key.device) == cudaSuccess;
  for (int i = 0; known && i < kept.used; ++i)
    if (kept.key[i] == key) return kept.shape[i];
  TileShape t;
  choose_tile(d, has_c, conv, t.ctas, t.block_n, t.mblk);
  const bool answered = choose_width(d, has_c, conv, t.ctas, t.block_n, t.mblk, t.tile_n, t.split_log);
  if (known && answered) {
    const int slot = kept.used < kKept ? kept.used++ : (kept.next++ % kKept);
    kept.key[slot] = key;
    kept.shape[slot] = t;
  }
  return t;
}

extern "C" sp24_status sp24_gemm_plan(const sp24_gemm_desc* d, int* ctas, int* block_n, int* mblk) {
  SP24_RETURN_IF(d == nullptr || ctas == nullptr || block_n == nullptr || mblk == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(d->M <= 0 || d->N <= 0 || d->K <= 0, SP24_ERR_SHAPE);
  const TileShape t = choose(d, false, false);
  *ctas = t.ctas;
  *block_n = t.block_n;
  *mblk = t.mblk;
  Settings& cfg = settings();
  if (const int c = cfg.ctas.load(std::memory_order_relaxed)) {
    *ctas = c;
    *block_n = cfg.block_n.load(std::memory_order_relaxed);
    *mblk = cfg.mblk.load(std::memory_order_relaxed);
  }
  return SP24_OK;
}

static sp24_status validate_gemm(const sp24_gemm_desc* d, const void* alpha, const void* A, const void* meta,
                                 const void* B, const void* beta, const void* C, void* D, void* ws, size_t ws_bytes,
                                 bool& has_c, float& falpha, float& fbeta, bool dequant = false,
                                 const sp24_linear_epilogue* linear = nullptr) {
  SP24_RETURN_IF(d == nullptr || (!dequant && !linear && (alpha == nullptr || beta == nullptr)), SP24_ERR_NULL);
  const bool tf32 = d->ab_type == SP24_F32;
  const bool f8 = is_fp8(d->ab_type);
  const bool fp = d->ab_type == SP24_F16 || d->ab_type == SP24_BF16 || tf32 || f8;
  SP24_RETURN_IF(!fp && d->ab_type != SP24_I8, SP24_ERR_DTYPE);
  SP24_RETURN_IF(tf32 && d->cd_type != SP24_F32, SP24_ERR_UNSUPPORTED);
  if (dequant)
    SP24_RETURN_IF(fp || (d->cd_type != SP24_BF16 && d->cd_type != SP24_F16 && d->cd_type != SP24_F32 &&
                          d->cd_type != SP24_I8),
                   SP24_ERR_DTYPE);
  else if (f8 || (linear && !fp)) SP24_RETURN_IF(d->cd_type != SP24_F16 && d->cd_type != SP24_BF16 && d->cd_type != SP24_F32, SP24_ERR_DTYPE);
  else if (fp) SP24_RETURN_IF(d->cd_type != d->ab_type && d->cd_type != SP24_F32, SP24_ERR_DTYPE);
  else SP24_RETURN_IF(d->cd_type != SP24_I32, SP24_ERR_DTYPE);
  const int64_t mult = elem_bytes(d->ab_type) == 1 ? 32 : 16;
  SP24_RETURN_IF(d->M < 0 || d->N < 0 || d->K <= 0, SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->M % mult || d->N % mult || d->K % mult, SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->M > (int64_t(1) << 30) || d->N > (int64_t(1) << 30) || d->K > (int64_t(1) << 30), SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->order_b != SP24_COL_MAJOR && d->order_b != SP24_ROW_MAJOR, SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(d->order_d != SP24_ROW_MAJOR && d->order_d != SP24_COL_MAJOR, SP24_ERR_UNSUPPORTED);
  if (dequant || linear) {
    falpha = 1.f;
    fbeta = linear && linear->residual ? 1.f : 0.f;
  } else if (fp) {
    falpha = *static_cast<const float*>(alpha);
    fbeta = *static_cast<const float*>(beta);
  } else {
    int32_t ia = *static_cast<const int32_t*>(alpha), ib = *static_cast<const int32_t*>(beta);
    SP24_RETURN_IF(ia != 1 || (ib != 0 && ib != 1), SP24_ERR_UNSUPPORTED);
    falpha = 1.f;
    fbeta = (float)ib;
  }
  has_c = fbeta != 0.f;
  // C is converted in place into D inside the epilogue's staging buffer: same order for both
  SP24_RETURN_IF(has_c && d->order_c != d->order_d, SP24_ERR_UNSUPPORTED);
  if (d->M == 0 || d->N == 0) return SP24_OK;
  SP24_RETURN_IF(A == nullptr || B == nullptr || D == nullptr || (has_c && C == nullptr), SP24_ERR_NULL);
  SP24_RETURN_IF(!d->a_is_dense && meta == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(ws == nullptr || ws_bytes < 256 || !aligned16(ws), SP24_ERR_WORKSPACE);
  const int es = elem_bytes(d->ab_type), cs = elem_bytes(d->cd_type);
  const int64_t a_cols = d->a_is_dense ? d->K : d->K / 2;
  const int64_t cd_width = d->order_d == SP24_COL_MAJOR ? d->M : d->N;
  SP24_RETURN_IF(d->lda < a_cols || d->ldb < (d->order_b == SP24_COL_MAJOR ? d->K : d->N) || d->ldd < cd_width ||
                     (has_c && d->ldc < cd_width),
                 SP24_ERR_STRIDE);
  SP24_RETURN_IF((d->lda * es) % 16 || (d->ldb * es) % 16 || (d->ldd * cs) % 16 || (has_c && (d->ldc * cs) % 16),
                 SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned16(A) || !aligned16(B) || !aligned16(D) || (has_c && !aligned16(C)) ||
                     (!d->a_is_dense && !aligned16(meta)),
                 SP24_ERR_ALIGN);
  if (linear) {
    SP24_RETURN_IF(linear->pre && (linear->ld_pre < cd_width || (linear->ld_pre * cs) % 16), SP24_ERR_STRIDE);
    const uintptr_t vectors = reinterpret_cast<uintptr_t>(linear->row_scale) | reinterpret_cast<uintptr_t>(linear->col_scale) |
                              reinterpret_cast<uintptr_t>(linear->bias);
    SP24_RETURN_IF(!aligned16(linear->pre) || (vectors & 3), SP24_ERR_ALIGN);
  }
  return SP24_OK;
}

struct ConvArgs {
  int64_t nb, h, w, c;
};

struct DequantArgs {
  const float* row_scale;
  const float* bias;
  int relu;
  float out_inv_scale;
};

static sp24_status run_gemm(const sp24_gemm_desc* d, const void* alpha, const void* A, const void* meta, const void* B,
                            const void* beta, const void* C, void* D, void* workspace, size_t workspace_bytes,
                            void* stream, const DequantArgs* dq, const ConvArgs* cv = nullptr, bool acc_f16 = false,
                            const sp24_linear_epilogue* linear = nullptr) {
  bool has_c = false;
  float falpha = 1.f, fbeta = 0.f;
  sp24_status st = validate_gemm(d, alpha, A, meta, B, beta, C, D, workspace, workspace_bytes, has_c, falpha, fbeta,
                                 dq != nullptr, linear);
  if (st != SP24_OK) return st;
  if (d->M == 0 || d->N == 0) return SP24_OK;
  if ((st = check_arch()) != SP24_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  GemmParams p = {};
  if (cv) {
    p.conv = 1;
    p.conv_h = (int)cv->h;
    p.conv_w = (int)cv->w;
    p.conv_c = (int)cv->c;
    p.by_image = FastDiv::by((uint32_t)(cv->h * cv->w));
    p.by_conv_w = FastDiv::by((uint32_t)cv->w);
  }
  p.acc_f16 = acc_f16 ? 1 : 0;
  if (dq) {
    p.dequant = 1;
    p.relu = dq->relu;
    p.row_scale = dq->row_scale;
    p.bias = dq->bias;
    p.out_inv_scale = dq->out_inv_scale;
  }
  if (linear) {
    p.linear = 1;
    p.act = (int)linear->act;
    p.row_scale = linear->row_scale;
    p.col_scale = linear->col_scale;
    p.bias = linear->bias;
    p.pre = linear->pre;
    p.ld_pre = linear->ld_pre;
  }
  p.M = d->M; p.N = d->N; p.K = d->K;
  p.ldc = d->ldc; p.ldd = d->ldd;
  p.C = has_c ? C : nullptr;
  p.D = D;
  p.status = static_cast<uint32_t*>(workspace);
  p.alpha = falpha; p.beta = fbeta;
  p.a_fmt = (d->ab_type == SP24_BF16 || d->ab_type == SP24_E5M2) ? 1 : 0;
  p.cd_type = (int)d->cd_type;
  p.has_c = has_c ? 1 : 0;
  set_wait_limit(p);
  Settings& cfg = settings();
  p.cd_col_major = d->order_d == SP24_COL_MAJOR ? 1 : 0;
  const bool sparse = !d->a_is_dense;
  const bool i8 = d->ab_type == SP24_I8, tf32 = d->ab_type == SP24_F32, f8 = is_fp8(d->ab_type);
  TileShape tile = choose(d, has_c, cv != nullptr);
  p.band = 16 / tile.mblk;
  if (const int c = cfg.ctas.load(std::memory_order_relaxed)) {
    tile.ctas = c;
    tile.block_n = cfg.block_n.load(std::memory_order_relaxed);
    tile.mblk = cfg.mblk.load(std::memory_order_relaxed);
    tile.tile_n = tile.ctas == 1 && tile.mblk > 1 && d->N < tile.block_n ? (int)d->N : tile.block_n;
    tile.split_log = 0;
  }
  SP24_RETURN_IF(cv && tile.ctas == 1 && tile.mblk != 1, SP24_ERR_UNSUPPORTED);  // a forced tall tile
  p.mblk = tile.mblk;
  if (const int b = cfg.band.load(std::memory_order_relaxed)) p.band = b;
  const bool b_mn = d->order_b == SP24_ROW_MAJOR;  // B stored N-contiguous
  if (cfg.log.load(std::memory_order_relaxed))
    fprintf(stderr, "sp24_gemm: M=%lld N=%lld K=%lld ab=%d cd=%d %s%s tile=%dx%dx%d columns=%d split=%d band=%d beta=%g%s%s\n", (long long)d->M,
            (long long)d->N, (long long)d->K, (int)d->ab_type, (int)d->cd_type, sparse ? "sparse" : "dense",
            b_mn ? " B:N-contiguous" : "", tile.ctas, tile.block_n, tile.mblk, tile.tile_n, 1 << tile.split_log, p.band, (double)fbeta, dq ? " dequant" : (linear ? " linear" : ""),
            cv ? " conv3x3" : (acc_f16 ? " fp16-accumulate" : ""));
  if (i8) return launch_gemm<1>(tile, sparse, b_mn, d, p, A, meta, B, s);
  if (tf32) return launch_gemm<2>(tile, sparse, b_mn, d, p, A, meta, B, s);
  if (f8) return launch_gemm<3>(tile, sparse, b_mn, d, p, A, meta, B, s);
  return launch_gemm<0>(tile, sparse, b_mn, d, p, A, meta, B, s);
}

extern "C" sp24_status sp24_gemm(const sp24_gemm_desc* d, const void* alpha, const void* A, const void* meta,
                                 const void* B, const void* beta, const void* C, void* D, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  return run_gemm(d, alpha, A, meta, B, beta, C, D, workspace, workspace_bytes, stream, nullptr);
}

extern "C" sp24_status sp24_gemm_f16acc(const sp24_gemm_desc* d, const void* alpha, const void* A, const void* meta,
                                        const void* B, const void* beta, const void* C, void* D, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(d->ab_type != SP24_F16 || (d->cd_type != SP24_F16 && d->cd_type != SP24_F32), SP24_ERR_DTYPE);
  return run_gemm(d, alpha, A, meta, B, beta, C, D, workspace, workspace_bytes, stream, nullptr, nullptr, true);
}

extern "C" sp24_status sp24_gemm_i8_dequant(const sp24_gemm_desc* d, const void* A, const void* meta, const void* B,
                                            const float* row_scale, const float* bias, int relu, float out_scale,
                                            void* D, void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(d->M > 0 && d->N > 0 && row_scale == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(d->cd_type == SP24_I8 && !(out_scale > 0.f), SP24_ERR_UNSUPPORTED);
  DequantArgs dq = {row_scale, bias, relu ? 1 : 0, d->cd_type == SP24_I8 ? 1.0f / out_scale : 1.0f};
  return run_gemm(d, nullptr, A, meta, B, nullptr, nullptr, D, workspace, workspace_bytes, stream, &dq);
}

extern "C" sp24_status sp24_linear(const sp24_gemm_desc* d, const sp24_linear_epilogue* e, const void* A, const void* meta, const void* B,
                                   void* D, void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr || e == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF((int)e->act < SP24_ACT_NONE || (int)e->act > SP24_ACT_GELU_TANH, SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(e->col_scale && elem_bytes(d->ab_type) != 1, SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(e->pre && (e->pre == D || e->pre == e->residual), SP24_ERR_UNSUPPORTED);
  return run_gemm(d, nullptr, A, meta, B, nullptr, e->residual, D, workspace, workspace_bytes, stream, nullptr, nullptr, false, e);
}

extern "C" sp24_status sp24_conv3x3_nhwc(const sp24_gemm_desc* d, int64_t Nb, int64_t H, int64_t W, int64_t Cin,
                                         const void* alpha, const void* A, const void* meta, const void* x,
                                         const void* beta, const void* C, void* D, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(Nb <= 0 || H <= 0 || W <= 0 || Cin <= 0, SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->N != Nb * H * W || d->K != 9 * Cin, SP24_ERR_SHAPE);
  SP24_RETURN_IF(!is_ab_type(d->ab_type), SP24_ERR_DTYPE);
  // a shared-memory stage holds 128 (16-bit) or 256 (int8) consecutive k = channels of ONE filter tap
  const int64_t per_stage = elem_bytes(d->ab_type) == 1 ? 256 : 128;
  SP24_RETURN_IF(Cin % per_stage != 0, SP24_ERR_SHAPE);
  SP24_RETURN_IF(H > 32767 || W > 32767 || Nb > (int64_t(1) << 30), SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->order_b != SP24_COL_MAJOR, SP24_ERR_UNSUPPORTED);
  // smaller activations trip a tensor-map restriction of current drivers
  SP24_RETURN_IF(Nb * H * W * Cin * elem_bytes(d->ab_type) < 131072, SP24_ERR_UNSUPPORTED);
  sp24_gemm_desc dd = *d;
  dd.ldb = d->K;  // not used by the im2col view, but keeps the generic checks meaningful
  ConvArgs cv = {Nb, H, W, Cin};
  return run_gemm(&dd, alpha, A, meta, x, beta, C, D, workspace, workspace_bytes, stream, nullptr, &cv);
}

extern "C" sp24_status sp24_gemm_status(void* workspace, void* stream) {
  SP24_RETURN_IF(workspace == nullptr, SP24_ERR_NULL);
  uint32_t host[4] = {0, 0, 0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  SP24_CUDA_CHECK(cudaMemcpyAsync(host, workspace, sizeof(host), cudaMemcpyDeviceToHost, s));
  SP24_CUDA_CHECK(cudaStreamSynchronize(s));
  if (host[0] == 0) return SP24_OK;
  // reported once: the record starts again from "ok" for the launches that follow
  SP24_CUDA_CHECK(cudaMemsetAsync(workspace, 0, sizeof(host), s));
  return SP24_ERR_TIMEOUT;
}

extern "C" sp24_status sp24_set_tile_override(int ctas, int block_n, int mblk, int band) {
  SP24_RETURN_IF(ctas < 0 || block_n < 0 || mblk < 0 || band < 0, SP24_ERR_SHAPE);
  Settings& cfg = settings();
  cfg.block_n.store(ctas ? block_n : 0, std::memory_order_relaxed);
  cfg.mblk.store(ctas ? (mblk ? mblk : 1) : 0, std::memory_order_relaxed);
  cfg.ctas.store(ctas, std::memory_order_relaxed);
  cfg.band.store(band, std::memory_order_relaxed);
  return SP24_OK;
}

extern "C" sp24_status sp24_test_set_fault_hooks(long long wait_cycles, int skip_stage) {
  Settings& cfg = settings();
  cfg.test_wait_cycles.store(wait_cycles, std::memory_order_relaxed);
  cfg.test_skip_stage.store(skip_stage < 0 ? 1 : skip_stage, std::memory_order_relaxed);
  return SP24_OK;
}

// ---------------------------------------------------------------------------------------------
// sp24_gemm_static_ws: sp24_gemm for callers that cannot allocate device memory.
//
// sp24_gemm needs a small device workspace (its status record) that the caller normally
// allocates.  Some callers cannot: a serving process whose framework allocator has already
// reserved all device memory (cudaMalloc then fails), or a latency-critical loop that must not
// pay cudaMalloc's implicit device-wide synchronisation.  For them the workspace lives in the
// file-scope device array below, which every GPU that loads this library holds until the
// process exits.  Inputs and outputs are still the caller's.
//
// The array's name is only a host-side stand-in in host code, not a device address, so the
// address is resolved with cudaGetSymbolAddress once per device (with that device current) on
// the first call made on that device; that first call should therefore come before any stream
// capture.  The entry points call no cudaMalloc, cudaFree or other allocating routine.
//
// All calls on a device share the one array.  It starts out zero-filled (static storage) and the
// kernels only ever write a non-zero code into it, so nothing has to be cleared between calls:
// the record keeps the first expired wait of any call until sp24_gemm_static_ws_status reads and
// clears it.  Calls that overlap on the GPU (different streams) share that one record, so a
// reported timeout cannot be attributed to one of them: serialise them, or use sp24_gemm with
// one workspace per stream.
// ---------------------------------------------------------------------------------------------
namespace {
constexpr size_t kStaticWorkspaceBytes = 4096;  // stated maximum; sp24_gemm currently needs 256
static __device__ __align__(256) unsigned char g_static_workspace[kStaticWorkspaceBytes];

constexpr int kMaxDevices = 64;
std::mutex g_static_ws_mutex;
void* g_static_ws_ptr[kMaxDevices] = {};

// device address of the array on the current device (looked up once per device)
sp24_status static_workspace(void** out) {
  int dev = 0;
  SP24_CUDA_CHECK(cudaGetDevice(&dev));
  SP24_RETURN_IF(dev < 0 || dev >= kMaxDevices, SP24_ERR_UNSUPPORTED);
  std::lock_guard<std::mutex> lock(g_static_ws_mutex);
  if (g_static_ws_ptr[dev] == nullptr) {
    void* ptr = nullptr;
    SP24_CUDA_CHECK(cudaGetSymbolAddress(&ptr, g_static_workspace));
    if (ptr == nullptr) return SP24_ERR_CUDA;
    g_static_ws_ptr[dev] = ptr;
  }
  *out = g_static_ws_ptr[dev];
  return SP24_OK;
}
}  // namespace

extern "C" sp24_status sp24_gemm_static_ws(const sp24_gemm_desc* d, const void* alpha, const void* A,
                                           const void* meta, const void* B, const void* beta, const void* C,
                                           void* D, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  // the problem's workspace need must fit the fixed array
  SP24_RETURN_IF(sp24_gemm_workspace_bytes(d) > kStaticWorkspaceBytes, SP24_ERR_WORKSPACE);
  void* ws = nullptr;
  sp24_status st = static_workspace(&ws);
  if (st != SP24_OK) return st;
  return sp24_gemm(d, alpha, A, meta, B, beta, C, D, ws, kStaticWorkspaceBytes, stream);
}

extern "C" sp24_status sp24_gemm_static_ws_status(void* stream) {
  void* ws = nullptr;
  sp24_status st = static_workspace(&ws);
  if (st != SP24_OK) return st;
  return sp24_gemm_status(ws, stream);
}
