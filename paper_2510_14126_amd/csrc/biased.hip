// Attention with capped, biased or masked scores over the paged cache: kernel
// entry points.  The algorithms live in biased_body.h.
#include "biased_body.h"
#include "biased_decode.h"

namespace pa {
namespace {

using mfma::kWaves;

template <int D, bool CAP, bool BIAS, int AUX>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
biased_split_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kSplitLdsBytes<D>];
  biased::split_body<D, CAP, BIAS, AUX>(p, blockIdx.x, (lds_u8_t*)smem);
}

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
biased_big_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kBigLdsBytes<D>];
  biased::big_body<D, CAP, BIAS>(p, blockIdx.x, (lds_u8_t*)smem);
}

template <int D, int GP, bool CAP, bool BIAS, int AUX>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
biased_decode_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kDecodeLdsBytes<D, GP>];
  biased::decode_body<D, GP, CAP, BIAS, AUX>(p, blockIdx.x, (lds_u8_t*)smem);
}

// One row per workgroup, NW = 8 wavefronts on it, or four rows (NW = 1): eight
// where a row has more partitions than one wavefront loads together and the rows
// alone do not fill the GPU's wavefronts.  Whole decodes, one wavefront per row /
// eight, capped: 64 rows of 32 partitions (a sequence of 30011 tokens, 64 heads over
// 8) 27.3 / 25.1 us, 8 of 256 (100000 tokens, 8 over 1) 36.7 / 19.5; with at most eight
// partitions, or more rows, the same or slower: 128 rows of 8 (four of 16384, 32 over
// 8) 45.4 / 45.6, 1024 of 16 (sixteen of 32768, 64 over 8) 335.4 / 336.0.
constexpr int kMergeWaves = 8;
template <int D, int NW>
__global__ void __launch_bounds__(64 * (NW > 1 ? NW : kWaves)) biased_merge_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) float smem[NW > 1 ? NW * (D + 1) : 1];
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int64_t row = NW > 1 ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;
  if (row >= (int64_t)p.batch * p.tiles * p.num_kv_heads * p.tile_rows) return;
  biased::merge_body<D, NW>(p, (int)(row / p.tile_rows), (int)(row % p.tile_rows), NW > 1 ? wave : 0, (lds_f32_t*)smem);
}

template <int D, bool CAP, bool BIAS>
hipError_t launch_t(const BiasedParams& p, hipStream_t stream) {
  const int64_t tiles = (int64_t)p.batch * p.tiles * p.num_kv_heads;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles * p.parts)), dim3(64 * kWaves), 0, stream, p);
  };
  if (!p.q_start && p.group <= 4)
    go(p.stream_tiles ? biased_decode_kernel<D, 4, CAP, BIAS, kLoadStreaming>
                      : biased_decode_kernel<D, 4, CAP, BIAS, kLoadDefault>);
  else if (!p.q_start && p.group <= 8)
    go(p.stream_tiles ? biased_decode_kernel<D, 8, CAP, BIAS, kLoadStreaming>
                      : biased_decode_kernel<D, 8, CAP, BIAS, kLoadDefault>);
  else if (p.big)
    go(biased_big_kernel<D, CAP, BIAS>);
  else if (p.stream_tiles)
    go(biased_split_kernel<D, CAP, BIAS, kLoadStreaming>);
  else
    go(biased_split_kernel<D, CAP, BIAS, kLoadDefault>);
  if (p.parts > 1) {
    const int64_t rows = tiles * p.tile_rows;
    if (p.parts > biased::kGroup && rows <= 512)
      hipLaunchKernelGGL((biased_merge_kernel<D, kMergeWaves>), dim3((unsigned)rows), dim3(64 * kMergeWaves), 0, stream,
                         p);
    else
      hipLaunchKernelGGL((biased_merge_kernel<D, 1>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(64 * kWaves),
                         0, stream, p);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const BiasedParams& p, hipStream_t stream) {
  const bool cap = p.cap > 0.f, bias = p.slopes != nullptr;
  if (cap) return bias ? launch_t<D, true, true>(p, stream) : launch_t<D, true, false>(p, stream);
  return bias ? launch_t<D, false, true>(p, stream) : launch_t<D, false, false>(p, stream);
}

}  // namespace

hipError_t launch_biased(const BiasedParams& p, hipStream_t stream) {
  return p.head_dim == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace pa
