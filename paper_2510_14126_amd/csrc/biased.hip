// Attention with capped, biased or masked scores over the paged cache: kernel
// entry points.  The algorithms live in biased_body.h.
#include "biased_body.h"

namespace pa {
namespace {

using mfma::kWaves;

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
biased_split_kernel(const BiasedParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[biased::kSplitLdsBytes<D>];
  biased::split_body<D, CAP, BIAS>(p, blockIdx.x, (lds_u8_t*)smem);
}

template <int D>
__global__ void __launch_bounds__(256) biased_merge_kernel(const BiasedParams p) {
  biased::merge_body<D>(p, blockIdx.x);
}

template <int D, bool CAP, bool BIAS>
hipError_t launch_t(const BiasedParams& p, hipStream_t stream) {
  const int64_t tiles = (int64_t)p.batch * p.tiles * p.num_kv_heads;
  hipLaunchKernelGGL((biased_split_kernel<D, CAP, BIAS>), dim3((unsigned)(tiles * p.parts)), dim3(64 * kWaves), 0,
                     stream, p);
  if (p.parts > 1)
    hipLaunchKernelGGL(biased_merge_kernel<D>, dim3((unsigned)tiles), dim3(256), 0, stream, p);
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
