// Norm of each head's row and rotation to its token's position, for the q and
// k rows of a batch of tokens, in one pass; and the same with the k and v rows
// written into the paged cache.
//
// For a row x of head_dim D with weight w (none: y = x)
//     y_d = x_d w_d / sqrt(mean(x^2) + eps),
// and for the pairs (a, b) = (y_i, y_{i + r/2}) (half) or (y_{2i}, y_{2i+1})
// (interleaved), i < r/2, of its first r = rotary_dim values
//     (a, b) -> magnitude (a cos t - b sin t, b cos t + a sin t),
// t = position * f_i; the rest of the row stays.  Sums and products are fp32.
// The angle is formed in fp64 revolutions and reduced to [-1/2, 1/2] before it
// becomes fp32 (in fp32 a position of 10^6 would be off by up to 1/16 radian).
//
// Layout.  A row takes LP = D / 16 lanes (rounded up to a power of two), 16
// values each in two pieces of eight: pieces c and c + r/16 of a rotated half
// row, 2c and 2c + 1 of an interleaved one, so that both values of a pair and
// the eight angles 8c .. 8c+7 belong to one lane in either layout, and rows are
// read and written in 16-byte accesses.  A wavefront holds 64 / LP rows of one
// token at a time and computes that token's angles once, one per lane, into LDS.
//
// What bounds it: the bytes of the rows while tokens are many, the launch and
// the round trips to memory (for the append length, table entry, store) while
// they are few; the rows' loads are issued before the position is known.
#include "mfma_body.h"
#include "ops.h"
#include "paged_attn_ops.h"
#include "pa_device.h"

#include <algorithm>
#include <type_traits>

namespace pa {
namespace {

constexpr int kWaves = 4;

// The revolutions travel with the kernel's arguments, as many as LP lanes per
// row have pairs: the library owns no device memory, and a launch takes the host
// longer the more bytes of arguments it has (four tokens at D = 64, whole call: a
// fixed array of 128 pairs 5.1 us, these 32 4.8 us).
template <int PAIRS>
struct Turns {
  double of[PAIRS];
};

typedef __attribute__((address_space(3))) mfma::floatx4_t lds_f4_t;

struct Bf16 {
  static constexpr int kBytes = 2;
};
struct Fp16 {
  static constexpr int kBytes = 2;
};
struct Fp32 {
  static constexpr int kBytes = 4;
};

// Eight consecutive values as they are in memory.
template <typename T>
struct Piece {
  uint4 w[T::kBytes / 2];
};

template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const uint8_t* row, int piece) {
  Piece<T> x;
  const uint4* src = reinterpret_cast<const uint4*>(row + piece * 8 * T::kBytes);
#pragma unroll
  for (int i = 0; i < T::kBytes / 2; ++i) x.w[i] = src[i];
  return x;
}

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ void widen(const Piece<T>& x, float* y) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(x.w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (std::is_same_v<T, Fp32>)
      y[i] = __uint_as_float(w[i]);
    else if constexpr (std::is_same_v<T, Bf16>)
      y[i] = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    else
      y[i] = (float)__builtin_bit_cast(half2_t, w[i / 2])[i & 1];
  }
}

// Rounds to nearest even.
template <typename T>
__device__ __forceinline__ Piece<T> narrow(const float* y) {
  Piece<T> x;
  uint32_t* w = reinterpret_cast<uint32_t*>(x.w);
  if constexpr (std::is_same_v<T, Fp32>) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(y[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, Bf16>)
        w[i] = mfma::pack_bf16(y[2 * i], y[2 * i + 1]);
      else
        w[i] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)y[2 * i], (_Float16)y[2 * i + 1]});
    }
  }
  return x;
}

template <typename T>
__device__ __forceinline__ void store_piece(uint8_t* row, int piece, const Piece<T>& x) {
  uint4* dst = reinterpret_cast<uint4*>(row + piece * 8 * T::kBytes);
#pragma unroll
  for (int i = 0; i < T::kBytes / 2; ++i) dst[i] = x.w[i];
}

constexpr int kDppHalfMirror = 0x141;   // lane i <- 7 - i of each eight

// Sum over the LP lanes of a row; every lane receives it.
template <int LP>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<kDppQuadXor1>(x);
  x += dpp<kDppQuadXor2>(x);
  if constexpr (LP >= 8) x += dpp<kDppHalfMirror>(x);
  if constexpr (LP == 16) x += dpp<kDppRowRor8>(x);
  return x;
}

// Entries q_start[1 .. batch] that are at most t: the sequence of row t.  All
// lanes of the wavefront, 64 entries per step.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int batch, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = batch;
  while (len > 0) {
    const int step = (len + 63) >> 6;
    const bool has = lane * step < len;
    const bool past = has && q_start[lo + min((lane + 1) * step, len)] <= t;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(past));
    if (c * step >= len) return lo + len;
    lo += c * step;
    len = min(step, len - c * step) - 1;      // the segment's last entry is known to be past t
  }
  return lo;
}

template <typename T, int LP, bool INTERLEAVED, bool APPEND>
__global__ void __launch_bounds__(64 * kWaves) rope_kernel(const RopeParams p, const Turns<8 * LP> turns) {
  using Out = std::conditional_t<APPEND, Bf16, T>;
  constexpr int kMaxPairs = 8 * LP;
  __shared__ __attribute__((aligned(16))) float angles[kWaves][2][kMaxPairs];
  constexpr int kRows = 64 / LP;                  // rows of one step
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * kWaves + wave;
  const int token = (int)(w / p.waves);
  if (token >= p.tokens) return;                  // no barrier below spans wavefronts
  const int part = (int)(w % p.waves);
  const int c = lane % LP;
  const int D = p.head_dim;
  const int rot = p.rotary_dim / 16;              // lanes of a row that rotate
  const bool live = c < D / 16;
  const int total = p.num_q_heads + (APPEND ? 2 : 1) * p.num_kv_heads;
  const int steps = (total + kRows - 1) / kRows;
  int pa_, pb_;                                   // the lane's pieces
  if (INTERLEAVED) {
    pa_ = 2 * c;
    pb_ = 2 * c + 1;
  } else {
    pa_ = c < rot ? c : 2 * c;
    pb_ = c < rot ? c + rot : 2 * c + 1;
  }

  Piece<T> xa, xb;
  auto load = [&](int step) {
    const int r = step * kRows + lane / LP;
    if (!live || r >= total) return;
    const uint8_t* row;
    const size_t h = (size_t)D * T::kBytes;
    if (r < p.num_q_heads)
      row = static_cast<const uint8_t*>(p.q) + (int64_t)token * p.q_stride * T::kBytes + r * h;
    else if (!APPEND || r < p.num_q_heads + p.num_kv_heads)
      row = static_cast<const uint8_t*>(p.k) + (int64_t)token * p.k_stride * T::kBytes + (r - p.num_q_heads) * h;
    else
      row = static_cast<const uint8_t*>(p.v) + (int64_t)token * p.v_stride * T::kBytes +
            (r - p.num_q_heads - p.num_kv_heads) * h;
    xa = load_piece<T>(row, pa_);
    xb = load_piece<T>(row, pb_);
  };
  load(part);

  // Where the token goes and its position.
  int pos;
  size_t slot = 0;                                // of row 0 of its block's tile, KV head 0, in rows
  int row_in_block = 0;
  if constexpr (APPEND) {
    int b = token, i = 0, len = 1;
    if (p.q_start) b = sequence_of(p.q_start, p.batch, token);
    if (b >= p.batch) return;                     // behind the last sequence
    if (p.q_start) {
      const int s0 = max(p.q_start[b], 0);
      if (token < s0) return;
      i = token - s0;
      len = p.q_start[b + 1] - s0;
    }
    const int cap = 16 * p.bt_stride;
    int n = p.context_lens[b];
    n = n < 0 ? 0 : (n > cap ? cap : n);
    len = min(len, n);
    if (i >= len) return;                         // an empty sequence, or a chunk longer than its context
    const int t = n - len + i;
    int phys = p.block_tables[(size_t)b * p.bt_stride + (t >> 4)];
    phys = phys < 0 ? 0 : (phys >= p.num_blocks ? p.num_blocks - 1 : phys);
    slot = (size_t)phys * p.num_kv_heads * 16;
    row_in_block = t & 15;
    pos = p.positions ? p.positions[token] : t;
  } else {
    pos = p.positions[token];
  }

  float cs[8], sn[8];
  {
    lds_f32_t* mine = (lds_f32_t*)&angles[wave][0][0];
    for (int i = lane; i < p.rotary_dim / 2; i += 64) {
      const double turn = (double)pos * turns.of[i];
      float s, co;
      sincospif(2.0f * (float)(turn - rint(turn)), &s, &co);
      mine[i] = co * p.magnitude;
      mine[kMaxPairs + i] = s * p.magnitude;
    }
    __builtin_amdgcn_wave_barrier();
    if (c < rot) {
      const lds_f4_t* src = reinterpret_cast<const lds_f4_t*>(mine);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const mfma::floatx4_t x = src[2 * c + i], y = src[kMaxPairs / 4 + 2 * c + i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          cs[4 * i + e] = x[e];
          sn[4 * i + e] = y[e];
        }
      }
    }
  }

  float wa[8], wb[8];
  for (int step = part; step < steps; step += p.waves) {
    const int r = step * kRows + lane / LP;
    const bool is_q = r < p.num_q_heads;
    const bool is_v = APPEND && r >= p.num_q_heads + p.num_kv_heads;
    const bool has = live && r < total;
    float a[8], b[8];
    widen<T>(xa, a);
    widen<T>(xb, b);
    const Piece<T> ra = xa, rb = xb;
    load(step + p.waves);
    const float* weight = is_q ? p.q_weight : p.k_weight;
    if (has && weight && !is_v) {
      const float4* s = reinterpret_cast<const float4*>(weight);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 x = s[2 * pa_ + i], y = s[2 * pb_ + i];
        wa[4 * i] = x.x; wa[4 * i + 1] = x.y; wa[4 * i + 2] = x.z; wa[4 * i + 3] = x.w;
        wb[4 * i] = y.x; wb[4 * i + 1] = y.y; wb[4 * i + 2] = y.z; wb[4 * i + 3] = y.w;
      }
    }
    float sum = 0.f;
    if (has) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += a[i] * a[i] + b[i] * b[i];
    }
    sum = row_sum<LP>(sum);
    if (!has) continue;
    if (weight && !is_v) {
      const float inv = rsqrtf(sum / D + p.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] *= inv * wa[i];
        b[i] *= inv * wb[i];
      }
    }
    if (c < rot && !is_v) {
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = a[2 * i], x1 = a[2 * i + 1], y0 = b[2 * i], y1 = b[2 * i + 1];
          a[2 * i] = x0 * cs[i] - x1 * sn[i];
          a[2 * i + 1] = x1 * cs[i] + x0 * sn[i];
          b[2 * i] = y0 * cs[4 + i] - y1 * sn[4 + i];
          b[2 * i + 1] = y1 * cs[4 + i] + y0 * sn[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = a[i], y = b[i];
          a[i] = x * cs[i] - y * sn[i];
          b[i] = y * cs[i] + x * sn[i];
        }
      }
    }
    uint8_t* dst;
    const size_t h = (size_t)D * Out::kBytes;
    if (is_q)
      dst = static_cast<uint8_t*>(p.q_out) + (int64_t)token * p.q_out_stride * Out::kBytes + r * h;
    else if constexpr (APPEND)
      dst = reinterpret_cast<uint8_t*>(is_v ? p.v_pool : p.k_pool) +
            (slot + (size_t)((r - p.num_q_heads) % p.num_kv_heads) * 16 + row_in_block) * h;
    else
      dst = static_cast<uint8_t*>(p.k_out) + (int64_t)token * p.k_out_stride * Out::kBytes + (r - p.num_q_heads) * h;
    if constexpr (std::is_same_v<T, Out>) {
      // values that are neither normed nor rotated keep their bits
      const bool same = !weight || is_v;
      store_piece<Out>(dst, pa_, same && (is_v || c >= rot) ? ra : narrow<Out>(a));
      store_piece<Out>(dst, pb_, same && (is_v || c >= rot) ? rb : narrow<Out>(b));
    } else {
      store_piece<Out>(dst, pa_, narrow<Out>(a));
      store_piece<Out>(dst, pb_, narrow<Out>(b));
    }
  }
}

template <typename T, int LP>
hipError_t launch_t(RopeParams p, const double* host_turns, bool interleaved, bool append, hipStream_t stream) {
  const int total = p.num_q_heads + (append ? 2 : 1) * p.num_kv_heads;
  const int steps = (total * LP + 63) / 64;
  // Steps of one wavefront: one while tokens are few; more once the call fills
  // the GPU several times over, which saves angles and launches, but leaves an
  // uneven end if there are too few wavefronts.  Normed, rotated, D = 128, at
  // 16384 / 32768 / 65536 / 131072 / 262144 / 10^6 steps in flight: 8191 tokens of 72
  // rows 62.0 / 59.7 / 59.0 / 61.8 / 61.8 / 61.7 us (5.1 TB/s at best, a copy of the same
  // bytes reaches 5.2-5.4), append of 53.6K tokens of 48 rows 247.8 / 247.9 / 240.8 / 241.6 /
  // 238.8 / 285.3 us (5.5 TB/s).  Loads with the streaming hint: 57.9 and 257 us.
  constexpr int64_t kFill = 65536;
  const int64_t per_wave = std::min<int64_t>(steps, ((int64_t)steps * p.tokens + kFill - 1) / kFill);
  p.waves = (int)((steps + per_wave - 1) / per_wave);
  const int64_t grid = ((int64_t)p.tokens * p.waves + kWaves - 1) / kWaves;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  Turns<8 * LP> turns{};
  std::copy(host_turns, host_turns + p.rotary_dim / 2, turns.of);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWaves), 0, stream, p, turns);
  };
  if (append)
    interleaved ? go(rope_kernel<T, LP, true, true>) : go(rope_kernel<T, LP, false, true>);
  else
    interleaved ? go(rope_kernel<T, LP, true, false>) : go(rope_kernel<T, LP, false, false>);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_d(const RopeParams& p, const double* turns, bool interleaved, bool append, hipStream_t stream) {
  if (p.head_dim <= 64) return launch_t<T, 4>(p, turns, interleaved, append, stream);
  if (p.head_dim <= 128) return launch_t<T, 8>(p, turns, interleaved, append, stream);
  return launch_t<T, 16>(p, turns, interleaved, append, stream);
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, const double* turns, int dtype, bool interleaved, bool append,
                       hipStream_t stream) {
  if (dtype == PA_BF16) return launch_d<Bf16>(p, turns, interleaved, append, stream);
  if (dtype == PA_FP16) return launch_d<Fp16>(p, turns, interleaved, append, stream);
  return launch_d<Fp32>(p, turns, interleaved, append, stream);
}

}  // namespace pa
