// Attention of trees of drafted tokens over the paged cache: kernel entry points.
//
// A tree's rows are an extend's whose mask is no interval: a node sees all that is
// resident before the tree, and of the tree its path to the root.  So the stages
// before the tree run as the biased extend's unmasked ones, and in the stages that
// hold nodes a row's interval of tokens meets its path, one bit per node
// (biased_body.h: TREE).
#include "biased_body.h"

namespace pa {
namespace {

using mfma::kWaves;

template <int D, bool CAP>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
tree_split_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kSplitLdsBytes<D> + biased::kTreeBytes<kBiasedTileRows>];
  biased::split_body<D, CAP, false, kLoadDefault, true>(p, blockIdx.x, (lds_u8_t*)smem);
}

template <int D, bool CAP>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
tree_big_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kBigLdsBytes<D> + biased::kTreeBytes<kBiasedWgRows>];
  biased::big_body<D, CAP, false, true>(p, blockIdx.x, (lds_u8_t*)smem);
}

constexpr int kMergeWaves = 8;
template <int D, int NW, int ROWS>
__global__ void __launch_bounds__(64 * (NW > 1 ? NW : kWaves)) tree_merge_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) float smem[NW > 1 ? NW * (D + 1) : 1];
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int64_t row = NW > 1 ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;
  if (row >= (int64_t)p.batch * p.tiles * p.num_kv_heads * p.tile_rows) return;
  biased::merge_body<D, NW, ROWS>(p, (int)(row / p.tile_rows), (int)(row % p.tile_rows), NW > 1 ? wave : 0,
                                  (lds_f32_t*)smem);
}

template <int D, int ROWS>
void launch_merge(const BiasedParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.batch * p.tiles * p.num_kv_heads * p.tile_rows;
  if (p.parts > biased::kGroup && rows <= 512)
    hipLaunchKernelGGL((tree_merge_kernel<D, kMergeWaves, ROWS>), dim3((unsigned)rows), dim3(64 * kMergeWaves), 0, stream,
                       p);
  else
    hipLaunchKernelGGL((tree_merge_kernel<D, 1, ROWS>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(64 * kWaves),
                       0, stream, p);
}

template <int D, bool CAP>
hipError_t launch_t(const BiasedParams& p, hipStream_t stream) {
  const int64_t tiles = (int64_t)p.batch * p.tiles * p.num_kv_heads;
  const dim3 grid((unsigned)(tiles * p.parts)), wg(64 * kWaves);
  if (p.big)
    hipLaunchKernelGGL((tree_big_kernel<D, CAP>), grid, wg, 0, stream, p);
  else
    hipLaunchKernelGGL((tree_split_kernel<D, CAP>), grid, wg, 0, stream, p);
  if (p.parts > 1) {
    if (p.big)
      launch_merge<D, kBiasedWgRows>(p, stream);
    else
      launch_merge<D, kBiasedTileRows>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree(const BiasedParams& p, hipStream_t stream) {
  if (p.head_dim == 128) return p.cap > 0.f ? launch_t<128, true>(p, stream) : launch_t<128, false>(p, stream);
  return p.cap > 0.f ? launch_t<64, true>(p, stream) : launch_t<64, false>(p, stream);
}

}  // namespace pa
