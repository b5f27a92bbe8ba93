// Products of many experts: argument checks, tile choice, entry points.
#include "sp24_act.cuh"
#include "sp24_gemm.cuh"

namespace sp24 {
namespace {

constexpr int64_t kMostRows = int64_t(1) << 30;

bool whole16(int64_t ld, int bytes) { return ld * bytes % 16 == 0; }

sp24_status check_sizes(const sp24_expert_desc* d) {
  const int64_t mult = elem_bytes(d->ab_type) == 1 ? 32 : 16;
  SP24_RETURN_IF(d->E < 1 || d->E > kMostExperts || d->M <= 0 || d->K <= 0 || d->rows < 0, SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->M % mult || d->K % mult, SP24_ERR_SHAPE);
  SP24_RETURN_IF(d->M > kMostRows || d->K > kMostRows || d->rows > kMostRows || d->E * d->M >= int64_t(1) << 31, SP24_ERR_SHAPE);
  return SP24_OK;
}

GemmParams params(const sp24_expert_desc* d, const int32_t* offsets, void* D, void* workspace) {
  GemmParams p = {};
  p.D = D;
  p.status = static_cast<uint32_t*>(workspace);
  p.alpha = 1.f;
  p.a_fmt = d->ab_type == SP24_BF16 || d->ab_type == SP24_E5M2 ? 1 : 0;
  p.cd_type = (int)d->cd_type;
  p.offsets = offsets;
  p.experts = (int)d->E;
  p.rows = (int)d->rows;
  set_wait_limit(p);
  return p;
}

sp24_status run(int group, TileShape tile, bool sparse, const sp24_gemm_desc* d, GemmParams& p, const void* A, const void* meta, const void* B, void* stream) {
  p.M = d->M; p.N = d->N; p.K = d->K;
  p.ldd = d->ldd; p.ldc = d->ldc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d->ab_type == SP24_I8) return launch_experts<1>(group, tile, sparse, d, p, A, meta, B, s);
  if (is_fp8(d->ab_type)) return launch_experts<3>(group, tile, sparse, d, p, A, meta, B, s);
  return launch_experts<0>(group, tile, sparse, d, p, A, meta, B, s);
}

// Tests and benchmarks: the shape that sp24_set_tile_override names, of any number of columns (whole 32) that a built one has; ctas 0: none is named.
TileShape forced_shape(bool dense) {
  int ctas, columns, mblk;
  forced_tile(&ctas, &columns, &mblk);
  return {ctas, ctas == 1 ? 128 : dense ? 256 : 224, mblk, columns, 0};
}
bool is_built(const TileShape& t) { return (t.ctas == 1 || t.ctas == 2) && t.mblk == 1 && t.tile_n >= 32 && t.tile_n <= t.block_n && t.tile_n % 32 == 0; }

// Rows of an expert with rows, in the mean: what the tiles are chosen by.
int64_t mean_rows(const sp24_expert_desc* d) {
  const int64_t met = d->E < d->rows ? d->E : d->rows;
  return met ? (d->rows + met - 1) / met : 0;
}

// The tile with the smallest estimated time, if every expert with rows has the mean number of them.  Two parts, us: the weights' way from HBM (with a little more where
// an expert's rows take several tiles), and the tiles x time of one over the CTAs or pairs (k-blocks of 256 bytes of K, a fixed part and one per column each, then the
// epilogue by columns, longer where other matrices are read or written); the sum of their cubes is compared, which is near the longer one.  Tiles of an expert: half a
// tile more than the rows ask for; where one would do for the mean, from 0.4 of its columns on there are experts with twice the mean or more.
// Fitted to bf16 and int8 products of 6 shapes (E, M, K from 8, 512, 512 to 64, 4096, 4096), 1 to 1024 rows an expert in the mean, even and uneven, at every width: 3.3 % off
// the best in the mean over the 312, 37 % at worst (32 x 512 x 4096, 48 rows, uneven).  Tiles of two m-blocks, which long products of one problem take, were slower
// nearly everywhere (bf16 16 experts 8192 x 4096, 16384 rows: 568 us, 518 and less with one).
TileShape choose_expert_tile(const sp24_expert_desc* d, bool has_c, bool has_pre) {
  const int64_t mean = mean_rows(d), met = d->E < d->rows ? d->E : d->rows;
  const int cs = elem_bytes(d->cd_type), es = elem_bytes(d->ab_type);
  const double k_blocks = (double)((d->K * es + 255) / 256);
  const double store = (cs == 4 ? (has_c ? 2.0 : 1.0) : (has_c ? 1.4 : 0.6)) + (has_pre ? (cs == 4 ? 1.0 : 0.6) : 0.0);
  const double weights = (double)met * d->M * d->K * (0.5 * es + 0.125) / 6.6e6;
  TileShape best = {1, 128, 1, 32, 0};
  double least = 0.0;
  auto consider = [&](int ctas, int block_n, int tile_n, double tile) {
    const int64_t rows = 128 * ctas, slots = sm_count() / ctas > 0 ? sm_count() / ctas : 1;
    const double full = (double)mean / tile_n;
    const double of_expert = full >= 1.0 ? full + 0.5 : full > 0.4 ? 1.0 + 0.5 * (full - 0.4) / 0.6 : 1.0;
    const double rounds = (double)((d->M + rows - 1) / rows) * (double)met * of_expert / (double)slots;
    const double time = tile * (rounds < 1.0 ? 1.0 : rounds + 0.6), way = weights * (1.0 + 0.07 * (of_expert - 1.0));
    const double cost = time * time * time + way * way * way;
    if (least == 0.0 || cost < least) {
      least = cost;
      best = {ctas, block_n, 1, tile_n, 0};
    }
  };
  for (int n = 32; n <= 128; n += 32) consider(1, 128, n, k_blocks * (0.2 + 0.00095 * n) + 0.1 + store * 0.01 * n);
  if (d->M <= 128) return best;
  for (int n = 64; n <= 224; n += 32) consider(2, 224, n, k_blocks * (0.165 + 0.00085 * n) + 0.1 + store * 0.01 * n);
  return best;
}

// The same for dense weights (D and dX): M features of the result, K of the contraction.  Pairs of CTAs whatever the rows, if there are features for them; what a column
// of a tile costs next to its 256 rows was set so that up to 160 columns, with which the ring has four stages (three from 192 on), are taken where there are a few rounds of
// tiles and 256 where there are many.  Us, device, bf16 dX, widths 96, 128, 160, 256 and as chosen: 8 experts 2816 x 2048, 128 rows each 23, 17, 17, 19, 19; 528: 51, 48, 46, 54, 49;
// 1024: 95, 75, 78, 75, 75; 50 of 2336 x 1760, 16 rows 65, 65, 65, 68, 66, 1024 434, 405, 352, 363, 360.
TileShape choose_dense_tile(const sp24_expert_desc* d, int64_t M, int64_t K) {
  const int64_t mean = mean_rows(d), met = d->E < d->rows ? d->E : d->rows;
  const int es = elem_bytes(d->ab_type), ctas = M > 128 ? 2 : 1, most = ctas == 2 ? 256 : 128;
  const double k_blocks = (double)((K * es + 255) / 256), weights = (double)met * M * K * es / 6.6e6;
  const int64_t rows = 128 * ctas, slots = sm_count() / ctas > 0 ? sm_count() / ctas : 1;
  TileShape best = {ctas, most, 1, most, 0};
  double least = 0.0;
  for (int n = 64; n <= most; n += 32) {
    const double full = (double)mean / n;
    const double of_expert = full >= 1.0 ? full + 0.5 : full > 0.4 ? 1.0 + 0.25 * (full - 0.4) / 0.6 : 1.0;
    const double rounds = (double)((M + rows - 1) / rows) * (double)met * of_expert / (double)slots;
    const double time = (k_blocks * 0.0028 * (30 + n) + 0.5) * (rounds < 1.0 ? 1.0 : rounds + 0.3), way = weights * (1.0 + 0.07 * (of_expert - 1.0));
    const double cost = time * time * time + way * way * way;
    if (least == 0.0 || cost < least) {
      least = cost;
      best.tile_n = n;
    }
  }
  return best;
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" sp24_status sp24_expert_linear(const sp24_expert_desc* d, const sp24_expert_epilogue* e, const void* A, const void* meta, const void* X,
                                          const int32_t* offsets, void* D, void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr || e == nullptr, SP24_ERR_NULL);
  const bool f16 = d->ab_type == SP24_F16 || d->ab_type == SP24_BF16, one_byte = d->ab_type == SP24_I8 || is_fp8(d->ab_type);
  SP24_RETURN_IF(!f16 && !one_byte, SP24_ERR_DTYPE);
  SP24_RETURN_IF(f16 ? d->cd_type != d->ab_type && d->cd_type != SP24_F32
                     : d->cd_type != SP24_F16 && d->cd_type != SP24_BF16 && d->cd_type != SP24_F32, SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(e->act), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(e->col_scale && f16, SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(e->pre && (e->pre == D || e->pre == e->residual), SP24_ERR_UNSUPPORTED);
  const sp24_status sizes = check_sizes(d);
  SP24_RETURN_IF(sizes != SP24_OK, sizes);
  if (d->rows == 0) return SP24_OK;
  SP24_RETURN_IF(A == nullptr || X == nullptr || offsets == nullptr || D == nullptr || (!d->a_is_dense && meta == nullptr), SP24_ERR_NULL);
  SP24_RETURN_IF(workspace == nullptr || workspace_bytes < 256 || !aligned16(workspace), SP24_ERR_WORKSPACE);
  const int es = elem_bytes(d->ab_type), cs = elem_bytes(d->cd_type);
  SP24_RETURN_IF(d->lda < (d->a_is_dense ? d->K : d->K / 2) || d->ldx < d->K || d->ldd < d->M || (e->residual && d->ld_residual < d->M) ||
                     (e->pre && d->ld_pre < d->M), SP24_ERR_STRIDE);
  SP24_RETURN_IF(!whole16(d->lda, es) || !whole16(d->ldx, es) || !whole16(d->ldd, cs) || (e->residual && !whole16(d->ld_residual, cs)) ||
                     (e->pre && !whole16(d->ld_pre, cs)), SP24_ERR_STRIDE);
  const uintptr_t vectors = reinterpret_cast<uintptr_t>(e->row_scale) | reinterpret_cast<uintptr_t>(e->col_scale) | reinterpret_cast<uintptr_t>(e->bias) |
                            reinterpret_cast<uintptr_t>(offsets);
  SP24_RETURN_IF(!aligned16(A) || !aligned16(X) || !aligned16(D) || !aligned16(e->residual) || !aligned16(e->pre) || (!d->a_is_dense && !aligned16(meta)) ||
                     (vectors & 3), SP24_ERR_ALIGN);
  SP24_RETURN_IF(e->residual == D && d->rows > 1 && d->ld_residual != d->ldd, SP24_ERR_STRIDE);
  const RowsAt result = {D, d->rows, d->M * cs, d->ldd * cs}, pre = {e->pre, d->rows, d->M * cs, d->ld_pre * cs},
               residual = {e->residual, d->rows, d->M * cs, d->ld_residual * cs}, x = {X, d->rows, d->K * es, d->ldx * es},
               a = {A, d->E * d->M, (d->a_is_dense ? d->K : d->K / 2) * es, d->lda * es};
  SP24_RETURN_IF(overlap(result, x) || overlap(result, a) || overlap(result, pre) || (e->residual != D && overlap(result, residual)) || overlap(pre, x) ||
                     overlap(pre, a) || overlap(pre, residual), SP24_ERR_UNSUPPORTED);
  const TileShape forced = forced_shape(d->a_is_dense != 0);
  SP24_RETURN_IF(forced.ctas && !is_built(forced), SP24_ERR_UNSUPPORTED);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  GemmParams p = params(d, offsets, D, workspace);
  p.linear = 1;
  p.cd_col_major = 1;
  p.act = (int)e->act;
  p.row_scale = e->row_scale;
  p.col_scale = e->col_scale;
  p.bias = e->bias;
  p.pre = e->pre;
  p.ld_pre = d->ld_pre;
  p.C = e->residual;
  p.has_c = e->residual != nullptr;
  p.beta = p.has_c ? 1.f : 0.f;
  const sp24_gemm_desc g = {d->ab_type, d->cd_type, d->M, d->rows, d->K, d->lda, d->ldx, d->ld_residual, d->ldd, SP24_COL_MAJOR, SP24_COL_MAJOR, SP24_COL_MAJOR,
                            d->a_is_dense};
  const TileShape tile = forced.ctas ? forced : d->a_is_dense ? choose_dense_tile(d, d->M, d->K) : choose_expert_tile(d, e->residual != nullptr, e->pre != nullptr);
  return run(kColumnsByExpert, tile, !d->a_is_dense, &g, p, A, meta, X, stream);
}

// What the two products of the gradient ask of their arguments: dz, `other` of so many rows of K columns, and `out` alike
static sp24_status check_gradient(const sp24_expert_desc* d, const void* dz, const void* other, int64_t other_rows, int64_t ld_other, const int32_t* offsets, void* out,
                                  int64_t out_rows, int64_t ld_out, const void* workspace, size_t workspace_bytes) {
  SP24_RETURN_IF(offsets == nullptr || out == nullptr || (d->rows > 0 && (dz == nullptr || other == nullptr)), SP24_ERR_NULL);
  SP24_RETURN_IF(workspace == nullptr || workspace_bytes < 256 || !aligned16(workspace), SP24_ERR_WORKSPACE);
  SP24_RETURN_IF(d->ldd < d->M || ld_other < d->K || ld_out < d->K, SP24_ERR_STRIDE);
  SP24_RETURN_IF(!whole16(d->ldd, 2) || !whole16(ld_other, 2) || !whole16(ld_out, 2), SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned16(dz) || !aligned16(other) || !aligned16(out) || (reinterpret_cast<uintptr_t>(offsets) & 3), SP24_ERR_ALIGN);
  const RowsAt result = {out, out_rows, d->K * 2, ld_out * 2};
  SP24_RETURN_IF(overlap(result, {dz, d->rows, d->M * 2, d->ldd * 2}) || overlap(result, {other, other_rows, d->K * 2, ld_other * 2}), SP24_ERR_UNSUPPORTED);
  return SP24_OK;
}

extern "C" sp24_status sp24_expert_linear_dx(const sp24_expert_desc* d, const void* dz, const void* W, const int32_t* offsets, void* dX, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF((d->ab_type != SP24_F16 && d->ab_type != SP24_BF16) || d->cd_type != d->ab_type, SP24_ERR_DTYPE);
  sp24_status st = check_sizes(d);
  SP24_RETURN_IF(st != SP24_OK, st);
  if (d->rows == 0) return SP24_OK;
  st = check_gradient(d, dz, W, d->E * d->M, d->lda, offsets, dX, d->rows, d->ldx, workspace, workspace_bytes);
  SP24_RETURN_IF(st != SP24_OK, st);
  const TileShape forced = forced_shape(true);
  SP24_RETURN_IF(forced.ctas && !is_built(forced), SP24_ERR_UNSUPPORTED);
  st = check_arch();
  SP24_RETURN_IF(st != SP24_OK, st);
  GemmParams p = params(d, offsets, dX, workspace);
  p.cd_col_major = 1;
  // W_e, transposed, times rows of dz: the tokens are columns as in the product itself, so that an expert's last tile is as wide as its rows ask for
  const sp24_gemm_desc g = {d->ab_type, d->cd_type, d->K, d->rows, d->M, d->lda, d->ldd, 0, d->ldx, SP24_COL_MAJOR, SP24_COL_MAJOR, SP24_COL_MAJOR, 1};
  return run(kColumnsTransposed, forced.ctas ? forced : choose_dense_tile(d, d->K, d->M), false, &g, p, W, nullptr, dz, stream);
}

extern "C" sp24_status sp24_expert_linear_dw(const sp24_expert_desc* d, const void* dz, const void* X, const int32_t* offsets, const void* meta, void* dW,
                                             void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF((d->ab_type != SP24_F16 && d->ab_type != SP24_BF16) || d->cd_type != d->ab_type, SP24_ERR_DTYPE);
  sp24_status st = check_sizes(d);
  SP24_RETURN_IF(st != SP24_OK, st);
  st = check_gradient(d, dz, X, d->rows, d->ldx, offsets, dW, d->E * d->M, d->lda, workspace, workspace_bytes);
  SP24_RETURN_IF(st != SP24_OK, st);
  SP24_RETURN_IF(reinterpret_cast<uintptr_t>(meta) & 1, SP24_ERR_ALIGN);
  st = check_arch();
  SP24_RETURN_IF(st != SP24_OK, st);
  if (d->rows == 0) {  // no expert has any
    SP24_CUDA_CHECK(cudaMemset2DAsync(dW, (size_t)d->lda * 2, 0, (size_t)d->K * 2, (size_t)(d->E * d->M), static_cast<cudaStream_t>(stream)));
    return SP24_OK;
  }
  GemmParams p = params(d, offsets, dW, workspace);
  const sp24_gemm_desc g = {d->ab_type, d->cd_type, d->M, d->K, d->rows, d->ldd, d->ldx, 0, d->lda, SP24_ROW_MAJOR, SP24_ROW_MAJOR, SP24_ROW_MAJOR, 1};
  TileShape tile = {1, 128, 1, 128, 0};
  if (d->M > 128 && d->K > 128) tile = {2, 256, 1, 256, 0};
  p.keep = static_cast<const uint8_t*>(meta);
  p.keep_kb = (int)(2 * ((d->K + 255) / 256));
  return run(kKByExpert, tile, false, &g, p, dz, nullptr, X, stream);
}
