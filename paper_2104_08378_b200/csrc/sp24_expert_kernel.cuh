// The GEMM kernels over the problems of many experts, and their launches.
#pragma once

#include "sp24_gemm_kernel.cuh"

namespace sp24 {
namespace {

// The kernel is that of sp24_linear; only where a tile lies is looked up (a search in shared memory, in a table that every CTA makes of the
// offsets at its start) and the last dimension of the tensor maps is that of all experts.  Tiles of one m-block; the columns of a tile are its caller's choice.
template <int KIND, bool SPARSE, int BLOCK_N, int CTAS, int GROUP>
sp24_status launch_group(const TileShape& tile, const sp24_gemm_desc* d, const GemmParams& base, const void* A, const void* meta, const void* B, cudaStream_t stream) {
  constexpr bool kBMn = GROUP == kKByExpert, kLinear = GROUP == kColumnsByExpert;
  using C = Cfg<KIND, SPARSE, BLOCK_N, CTAS, 1, kBMn>;
  GemmParams p = base;
  const int tile_n = p.tile_n = tile.tile_n;
  const int cs = elem_bytes(d->cd_type), es = elem_bytes(d->ab_type);
  const uint32_t atom_elems = kAtomBytes / es;
  const uint64_t E = (uint64_t)p.experts, rows = (uint64_t)p.rows, a_cols = (uint64_t)(SPARSE ? d->K / 2 : d->K);
  // twelve epilogue warps for the weights' gradients, whose k-blocks are the few of an expert's rows (us, bf16, with the pattern, eight, twelve and sixteen: 50 experts
  // 2336 x 1760, 656 rows 119, 104, 142; 8 of 2048 x 1408, 4224 rows 30, 26, 26)
  constexpr int kWarps = GROUP == kKByExpert ? 12 : kEpiWarps;
  p.epi_bytes = kWarps * 2048;
  p.table_bytes = (8 * (p.experts + 1) + 1023) / 1024 * 1024;
  p.kps = C::k_blocks_of_a_stage(tile_n, p.epi_bytes + p.table_bytes, (int64_t)a_cols, false);
  p.stages = C::ring_stages(C::stage_bytes(tile_n) * p.kps, p.epi_bytes + p.table_bytes);
  constexpr int tile_m = kBlockM * CTAS;
  p.m_tiles = (int)((d->M + tile_m - 1) / tile_m);
  p.n_tiles = (int)((d->N + tile_n - 1) / tile_n);
  p.k_blocks = (int)((d->K + C::kKPerStage - 1) / C::kKPerStage);
  p.by_band = FastDiv::by((uint32_t)p.m_tiles);
  p.meta_kb = (int)(2 * ((d->K + 255) / 256));
  p.meta_blocks = (int)((d->M + kBlockM - 1) / kBlockM);
  // tiles there can be at most: every expert with rows has one that is not full
  const int64_t met = p.experts < p.rows ? p.experts : p.rows;
  int64_t tiles;
  if (columns_by_expert(GROUP)) tiles = p.m_tiles * (p.rows / tile_n + met);
  else tiles = (int64_t)p.m_tiles * p.n_tiles * p.experts;
  SP24_RETURN_IF(tiles >= int64_t(1) << 31, SP24_ERR_SHAPE);
  if (GROUP == kKByExpert) p.by_expert = FastDiv::by((uint32_t)(p.m_tiles * p.n_tiles));
  const uint32_t b_box_rows = (uint32_t)C::b_rows(tile_n);
  CUtensorMap map_a, map_b, map_e;
  sp24_status st;
  if (columns_by_expert(GROUP)) {
    if (GROUP == kColumnsTransposed)
      st = make_map(&map_a, MapShape{A, {(uint64_t)d->M, (uint64_t)d->K, E}, {(uint64_t)d->lda * es, (uint64_t)(d->K * d->lda) * es},
                                     {atom_elems, (uint32_t)C::kKPerStage, 1}, es, 128});
    else if (p.kps == 2)
      st = make_map(&map_a, MapShape{A, {atom_elems, E * d->M, a_cols / atom_elems}, {(uint64_t)d->lda * es, kAtomBytes}, {atom_elems, kBlockM, 2}, es, 128});
    else
      st = make_map(&map_a, A, es, E * d->M, a_cols, d->lda * es, atom_elems, kBlockM, 128);
    if (st != SP24_OK) return st;
    if (C::kBBoxes > 1 && d->K % atom_elems == 0) {
      p.b_3d = 1;
      st = make_map(&map_b, MapShape{B, {atom_elems, rows, (uint64_t)d->K / atom_elems}, {(uint64_t)d->ldb * es, kAtomBytes},
                                     {atom_elems, b_box_rows, (uint32_t)(C::kBBoxes * p.kps)}, es, 128});
    } else {
      st = make_map(&map_b, B, es, rows, d->K, d->ldb * es, atom_elems, b_box_rows, 128);
    }
  } else {
    st = make_map(&map_a, A, es, rows, d->M, d->lda * es, atom_elems, C::kKPerStage, 128);
    if (st != SP24_OK) return st;
    st = make_map(&map_b, B, es, rows, d->N, d->ldb * es, C::kBChunkElems, C::kKPerStage, 128);
  }
  if (st != SP24_OK) return st;
  if (SPARSE) {
    st = make_map(&map_e, MapShape{meta, {128, (uint64_t)p.meta_kb * 16, E * p.meta_blocks}, {128, (uint64_t)p.meta_kb * 2048},
                                   {128, (uint32_t)(16 * C::kEBlocks * p.kps), 1}, 1, 0});
    if (st != SP24_OK) return st;
  } else {
    map_e = map_a;
  }
  using Kernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, GemmParams);
  Kernel forms[4] = {};  // [with C][bytes]
#define SP24_FORM(CS_, C_) forms[2 * C_ + (CS_ >> 2)] = gemm_kernel<KIND, SPARSE, BLOCK_N, CTAS, 1, kBMn, CS_, columns_by_expert(GROUP), C_, false, kWarps, kLinear, GROUP>;
  SP24_FORM(2, false)
  if constexpr (kLinear) { SP24_FORM(2, true) SP24_FORM(4, false) SP24_FORM(4, true) }
#undef SP24_FORM
  const Kernel kernel = forms[2 * p.has_c + (cs >> 2)];
  if (kernel == nullptr) return SP24_ERR_UNSUPPORTED;
  {
    static std::atomic<bool> done[64];  // the shared-memory opt-in, of all forms at once (as in launch)
    int dev = 0;
    SP24_CUDA_CHECK(cudaGetDevice(&dev));
    const bool kept = dev >= 0 && dev < 64;
    if (!kept || !done[dev].load(std::memory_order_acquire)) {
      for (const Kernel k : forms)
        if (k) SP24_CUDA_CHECK(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes));
      if (kept) done[dev].store(true, std::memory_order_release);
    }
  }
  int64_t clusters = sm_count() / CTAS;
  if (clusters > tiles) clusters = tiles;
  return launch_overlapped(kernel, dim3((unsigned)(clusters * CTAS)), dim3(32 * (kFirstEpiWarp + kWarps)), C::kSmemBytes, stream, CTAS, map_a, map_b, map_e, map_a, map_a, p);
}

template <int KIND>
sp24_status launch_group_shape(int group, TileShape t, bool sparse, const sp24_gemm_desc* d, const GemmParams& p, const void* A, const void* meta, const void* B,
                               cudaStream_t s) {
  const bool one = t.ctas == 1 && t.block_n == 128, pair = t.ctas == 2 && t.block_n == 224, wide = t.ctas == 2 && t.block_n == 256;
  if (t.mblk != 1) return SP24_ERR_UNSUPPORTED;
  if (group == kColumnsByExpert) {
    if (one) return sparse ? launch_group<KIND, true, 128, 1, kColumnsByExpert>(t, d, p, A, meta, B, s) : launch_group<KIND, false, 128, 1, kColumnsByExpert>(t, d, p, A, meta, B, s);
    if (pair && sparse) return launch_group<KIND, true, 224, 2, kColumnsByExpert>(t, d, p, A, meta, B, s);
    if (wide && !sparse) return launch_group<KIND, false, 256, 2, kColumnsByExpert>(t, d, p, A, meta, B, s);
  }
  if constexpr (KIND == 0) {
    if (group == kColumnsTransposed && !sparse) {
      if (one) return launch_group<KIND, false, 128, 1, kColumnsTransposed>(t, d, p, A, meta, B, s);
      if (wide) return launch_group<KIND, false, 256, 2, kColumnsTransposed>(t, d, p, A, meta, B, s);
    }
    if (group == kKByExpert && !sparse) {
      if (one) return launch_group<KIND, false, 128, 1, kKByExpert>(t, d, p, A, meta, B, s);
      if (wide) return launch_group<KIND, false, 256, 2, kKByExpert>(t, d, p, A, meta, B, s);
    }
  }
  return SP24_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace sp24
