// Products of many experts: argument checks, tile choice, entry points.
#include "sp24_act.cuh"
#include "sp24_gemm.cuh"

namespace sp24 {
namespace {

constexpr int64_t kMostExperts = 1024, kMostRows = int64_t(1) << 30;
enum { kColumnsByExpert = 1, kRowsByExpert = 2, kKByExpert = 3 };  // as the kernel has them

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

// Rows of an expert with rows, in the mean: what the tiles are chosen by.
int64_t mean_rows(const sp24_expert_desc* d) {
  const int64_t met = d->E < d->rows ? d->E : d->rows;
  return met ? (d->rows + met - 1) / met : 0;
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
  const int64_t mean = mean_rows(d);
  TileShape tile = {1, 128, 1, 32, 0};
  if (mean > 128 && d->M > 128) {
    tile.ctas = 2;
    tile.block_n = tile.tile_n = d->a_is_dense ? 256 : 224;
  } else {
    while (tile.tile_n < 128 && tile.tile_n < mean) tile.tile_n += 32;
  }
  return run(kColumnsByExpert, tile, !d->a_is_dense, &g, p, A, meta, X, stream);
}

// What the two products of the gradient ask of their arguments: a matrix each of M, K and again K or M columns
static sp24_status check_gradient(const sp24_expert_desc* d, const void* in, int64_t ld_in, int64_t least_in, const void* other, int64_t ld_other, const int32_t* offsets,
                                  void* out, int64_t ld_out, const void* workspace, size_t workspace_bytes) {
  SP24_RETURN_IF(offsets == nullptr || out == nullptr || (d->rows > 0 && (in == nullptr || other == nullptr)), SP24_ERR_NULL);
  SP24_RETURN_IF(workspace == nullptr || workspace_bytes < 256 || !aligned16(workspace), SP24_ERR_WORKSPACE);
  SP24_RETURN_IF(ld_in < least_in || ld_other < d->K || ld_out < d->K, SP24_ERR_STRIDE);
  SP24_RETURN_IF(!whole16(ld_in, 2) || !whole16(ld_other, 2) || !whole16(ld_out, 2), SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned16(in) || !aligned16(other) || !aligned16(out) || (reinterpret_cast<uintptr_t>(offsets) & 3), SP24_ERR_ALIGN);
  return check_arch();
}

extern "C" sp24_status sp24_expert_linear_dx(const sp24_expert_desc* d, const void* dz, const void* W, const int32_t* offsets, void* dX, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF((d->ab_type != SP24_F16 && d->ab_type != SP24_BF16) || d->cd_type != d->ab_type, SP24_ERR_DTYPE);
  sp24_status st = check_sizes(d);
  SP24_RETURN_IF(st != SP24_OK, st);
  if (d->rows == 0) return SP24_OK;
  st = check_gradient(d, dz, d->ldd, d->M, W, d->lda, offsets, dX, d->ldx, workspace, workspace_bytes);
  SP24_RETURN_IF(st != SP24_OK, st);
  GemmParams p = params(d, offsets, dX, workspace);
  // rows of tokens times K: dz is the operand with rows, W_e the one with columns
  const sp24_gemm_desc g = {d->ab_type, d->cd_type, d->rows, d->K, d->M, d->ldd, d->lda, 0, d->ldx, SP24_ROW_MAJOR, SP24_ROW_MAJOR, SP24_ROW_MAJOR, 1};
  TileShape tile = {1, 128, 1, 128, 0};
  if (mean_rows(d) > 128 && d->K > 128) tile = {2, 256, 1, 256, 0};
  return run(kRowsByExpert, tile, false, &g, p, dz, nullptr, W, stream);
}

extern "C" sp24_status sp24_expert_linear_dw(const sp24_expert_desc* d, const void* dzt, int64_t lddzt, const void* X, const int32_t* offsets, void* dW,
                                             void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(d == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF((d->ab_type != SP24_F16 && d->ab_type != SP24_BF16) || d->cd_type != d->ab_type, SP24_ERR_DTYPE);
  sp24_status st = check_sizes(d);
  SP24_RETURN_IF(st != SP24_OK, st);
  st = check_gradient(d, dzt, lddzt, d->rows, X, d->ldx, offsets, dW, d->lda, workspace, workspace_bytes);
  SP24_RETURN_IF(st != SP24_OK, st);
  if (d->rows == 0) {  // no expert has any
    SP24_CUDA_CHECK(cudaMemset2DAsync(dW, (size_t)d->lda * 2, 0, (size_t)d->K * 2, (size_t)(d->E * d->M), static_cast<cudaStream_t>(stream)));
    return SP24_OK;
  }
  GemmParams p = params(d, offsets, dW, workspace);
  const sp24_gemm_desc g = {d->ab_type, d->cd_type, d->M, d->K, d->rows, lddzt, d->ldx, 0, d->lda, SP24_ROW_MAJOR, SP24_ROW_MAJOR, SP24_ROW_MAJOR, 1};
  TileShape tile = {1, 128, 1, 128, 0};
  if (d->M > 128 && d->K > 128) tile = {2, 256, 1, 256, 0};
  return run(kKByExpert, tile, false, &g, p, dzt, nullptr, X, stream);
}
