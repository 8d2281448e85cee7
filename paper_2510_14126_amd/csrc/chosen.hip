// Decode attention over chosen blocks, and with its weights added to totals:
// kernel entry points.  The algorithms live in chosen_body.h.
#include "chosen_body.h"

namespace pa {
namespace {

using mfma::kWaves;

template <int D, int GP, bool LISTED, bool WEIGHTS, int AUX>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
chosen_decode_kernel(const TokensParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[chosen::kChosenLdsBytes<D, GP, WEIGHTS>];
  chosen::decode_body<D, GP, LISTED, WEIGHTS, AUX>(p, blockIdx.x, (lds_u8_t*)smem);
}

template <int D>
__global__ void __launch_bounds__(64 * kWaves) chosen_merge_kernel(const TokensParams p) {
  const int64_t row = (int64_t)blockIdx.x * kWaves + wave_uniform(threadIdx.x >> 6);
  if (row < (int64_t)p.batch * p.num_q_heads) chosen::merge_row<D>(p, row);
}

// The weights, `chunks` workgroups per sequence, and behind them the rows' merge.
template <int D, int GP>
__global__ void __launch_bounds__(256) chosen_weights_kernel(const TokensParams p, int chunks) {
  __shared__ float lds[chosen::kHeads];
  const int64_t wg = blockIdx.x;
  const int64_t first = (int64_t)p.batch * chunks;
  if (wg < first) {
    chosen::weights_body<GP>(p, (int)(wg / chunks), (int)(wg % chunks), (lds_f32_t*)lds);
    return;
  }
  const int64_t row = (wg - first) * kWaves + wave_uniform(threadIdx.x >> 6);
  if (row < (int64_t)p.batch * p.num_q_heads) chosen::merge_row<D>(p, row);
}

unsigned grid_of(const TokensParams& p) {
  return (unsigned)((int64_t)p.batch * p.head_tiles * p.num_kv_heads * p.parts);
}
unsigned merge_grid(const TokensParams& p) { return (unsigned)(((int64_t)p.batch * p.num_q_heads + kWaves - 1) / kWaves); }

template <int D, int GP>
hipError_t selected_t(const TokensParams& p, hipStream_t stream) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid_of(p)), dim3(64 * kWaves), 0, stream, p);
  };
  if (p.stream_tiles)
    go(chosen_decode_kernel<D, GP, true, false, kLoadStreaming>);
  else
    go(chosen_decode_kernel<D, GP, true, false, kLoadDefault>);
  if (p.parts > 1) hipLaunchKernelGGL(chosen_merge_kernel<D>, dim3(merge_grid(p)), dim3(64 * kWaves), 0, stream, p);
  return hipGetLastError();
}

template <int D, int GP>
hipError_t weights_t(const TokensParams& p, hipStream_t stream) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid_of(p)), dim3(64 * kWaves), 0, stream, p);
  };
  if (p.stream_tiles)
    go(chosen_decode_kernel<D, GP, false, true, kLoadStreaming>);
  else
    go(chosen_decode_kernel<D, GP, false, true, kLoadDefault>);
  const int chunks = (p.max_ctx + 255) / 256;
  const unsigned grid = (unsigned)((int64_t)p.batch * chunks + (p.parts > 1 ? merge_grid(p) : 0));
  if (grid > 0) hipLaunchKernelGGL((chosen_weights_kernel<D, GP>), dim3(grid), dim3(256), 0, stream, p, chunks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_selected(const TokensParams& p, hipStream_t stream) {
  if (p.head_dim == 128) return p.tile_heads == 4 ? selected_t<128, 4>(p, stream) : selected_t<128, 8>(p, stream);
  return p.tile_heads == 4 ? selected_t<64, 4>(p, stream) : selected_t<64, 8>(p, stream);
}

hipError_t launch_weights(const TokensParams& p, hipStream_t stream) {
  if (p.head_dim == 128) return p.tile_heads == 4 ? weights_t<128, 4>(p, stream) : weights_t<128, 8>(p, stream);
  return p.tile_heads == 4 ? weights_t<64, 4>(p, stream) : weights_t<64, 8>(p, stream);
}

}  // namespace pa
