// Dropout onto a residual, and its backward pass: Y = R + mask * scale * X, the mask drawn
// from a counter-based generator (dropout.h) and never stored.
//
// Memory bounds it: X, R and Y move once, and a block of draws costs some hundred
// instructions per eight elements, less than their 48 (bf16) or 96 bytes take.  Every access
// is 16 bytes a lane, a wave's contiguous, two of each tensor in flight per lane (measured,
// onto a residual: 16384 x 2048 bf16 29.1 us, 6.9 TB/s through the last-level cache, one in
// flight 32.4; 32768 x 4096 fp32 279 us, 5.8 TB/s; without a residual 183 us; eight
// consecutive fp32 elements a lane, whose two loads then each cover every other 16 bytes, 294
// and 206).  Streaming loads and stores and a grid of one round were level or slower.
#include "dropout.h"

namespace ec {

namespace {

constexpr int DR_U = 2;          // blocks of draws a lane takes at a time
constexpr int DR_WAVE = 512;     // elements of a wave per block a lane

__device__ __forceinline__ f32x4 load16(const void* p) { return *static_cast<const f32x4*>(p); }

// The eight elements of 16 bytes of bf16.
__device__ __forceinline__ void widen8(f32x4 x, float v[8]) {
  const u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_to_f32(w[i] & 0xffffu);
    v[2 * i + 1] = bf16_to_f32(w[i] >> 16);
  }
}

// The elements past the last 16 bytes, one a thread.
template <typename T>
__device__ __forceinline__ void dropout_tail(const T* X, const T* R, const Dropout& drop, T* Y,
                                             long first, long n, uint64_t seed, uint64_t offset) {
  const long e = first + threadIdx.x;
  if (blockIdx.x != 0 || e >= n) return;
  float x = Elem<T>::load1(X + e);
  if (drop.thr) {
    const u32x4 w = dropout_block((uint64_t)e >> 3, seed, offset);
    const int u = (int)(e & 7);
    const uint32_t word = u < 4 ? (u < 2 ? w[0] : w[1]) : (u < 6 ? w[2] : w[3]);
    x = ((u & 1) ? word >> 16 : word & 0xffffu) >= drop.thr ? x * drop.scale : 0.f;
  }
  Elem<T>::store1(Y + e, R ? x + Elem<T>::load1(R + e) : x);
}

// A lane's 16 bytes are a block of draws.
__global__ __launch_bounds__(256) void dropout_kernel(const bf16_t* X, const bf16_t* R,
                                                      Dropout drop, bf16_t* Y, long n) {
  const uint64_t seed = drop.thr ? drop.rng[0] : 0, offset = drop.thr ? drop.rng[1] : 0;
  const long whole = n / 8, stride = (long)gridDim.x * 256 * DR_U;
  for (long c0 = (long)blockIdx.x * 256 * DR_U + threadIdx.x; c0 < whole; c0 += stride) {
    f32x4 x[DR_U], r[DR_U];
#pragma unroll
    for (int u = 0; u < DR_U; ++u) {   // past the end: the last block again, not stored
      const long c = c0 + u * 256 < whole ? c0 + u * 256 : whole - 1;
      x[u] = load16(X + c * 8);
      if (R) r[u] = load16(R + c * 8);
    }
#pragma unroll
    for (int u = 0; u < DR_U; ++u) {
      const long c = c0 + u * 256;
      float v[8], q[8];
      widen8(x[u], v);
      if (drop.thr)
        dropout_apply(v, dropout_block((uint64_t)c, seed, offset), drop.thr, drop.scale);
      if (R) {
        widen8(r[u], q);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += q[i];
      }
      if (c < whole) Elem<bf16_t>::store8(Y + c * 8, v);
    }
  }
  dropout_tail(X, R, drop, Y, whole * 8, n, seed, offset);
}

// A lane's 16 bytes are half a block of draws: of a wave's 512 elements, lane l takes 4 l ..
// 4 l + 3 of both halves, an even lane draws for the first half's block that it shares with
// the next lane, an odd one for the second half's, and the two exchange.
__global__ __launch_bounds__(256) void dropout_kernel(const float* X, const float* R, Dropout drop,
                                                      float* Y, long n) {
  const uint64_t seed = drop.thr ? drop.rng[0] : 0, offset = drop.thr ? drop.rng[1] : 0;
  const int lane = threadIdx.x & 63;
  const bool odd = lane & 1;
  const long whole = n / 4 * 4, stride = (long)gridDim.x * 4 * DR_WAVE * DR_U;
  const long wave = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  for (long e0 = wave * DR_WAVE * DR_U; e0 < whole; e0 += stride) {
    f32x4 x[DR_U][2], r[DR_U][2];
#pragma unroll
    for (int u = 0; u < DR_U; ++u)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const long e = e0 + u * DR_WAVE + s * (DR_WAVE / 2) + lane * 4;
        const long at = e < whole ? e : whole - 4;
        x[u][s] = load16(X + at);
        if (R) r[u][s] = load16(R + at);
      }
#pragma unroll
    for (int u = 0; u < DR_U; ++u) {
      const long first = e0 + u * DR_WAVE;
      u32x4 w = {0, 0, 0, 0};
      if (drop.thr)
        w = dropout_block((uint64_t)(first / 8 + (odd ? DR_WAVE / 16 : 0) + (lane >> 1)), seed,
                          offset);
      // what the neighbour needs of this lane's block: its other half
      const uint32_t x0 = dpp_u32<0xB1>(odd ? w[0] : w[2]), x1 = dpp_u32<0xB1>(odd ? w[1] : w[3]);
      const uint32_t words[2][2] = {{odd ? x0 : w[0], odd ? x1 : w[1]},
                                    {odd ? w[2] : x0, odd ? w[3] : x1}};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const long e = first + s * (DR_WAVE / 2) + lane * 4;
        f32x4 v = x[u][s];
        if (drop.thr) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t d = words[s][i >> 1];
            v[i] = ((i & 1) ? d >> 16 : d & 0xffffu) >= drop.thr ? v[i] * drop.scale : 0.f;
          }
        }
        if (R) v += r[u][s];
        if (e < whole) *reinterpret_cast<f32x4*>(Y + e) = v;
      }
    }
  }
  dropout_tail(X, R, drop, Y, whole, n, seed, offset);
}

template <typename T>
hipError_t run_dropout(const T* X, const T* R, const Dropout& drop, T* Y, long n, hipStream_t st) {
  constexpr long per = 4l * DR_WAVE * DR_U;   // elements of a workgroup
  const long blocks = (n + per - 1) / per;
  // one dimension of a launch ends below 2^32 threads
  const long grid = blocks < (1l << 22) ? blocks : 1l << 22;
  dropout_kernel<<<dim3((unsigned)grid), 256, 0, st>>>(X, R, drop, Y, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int dtype, const void* X, const void* R, const Dropout& drop, void* Y,
                          long n, hipStream_t st) {
  if (n == 0) return hipSuccess;
  if (dtype == DT_F32)
    return run_dropout<float>((const float*)X, (const float*)R, drop, (float*)Y, n, st);
  return run_dropout<bf16_t>((const bf16_t*)X, (const bf16_t*)R, drop, (bf16_t*)Y, n, st);
}

}  // namespace ec
