// A tensor in eight bits with scales (mx.h): the layout in which the experts' weights are
// held for serving.
//
// Memory bounds it: 65536 x 2048 bf16 in 61.0 us, 6.7 TB/s (one piece of 16 bytes a lane on its
// way instead of four: 69.6; streaming loads save 2 of that).  640 x 1472 fp32, 4.7 MB: 2.7 us,
// the launch.
#include "mx.h"
#include "ec_kernels.h"

namespace ec {

namespace {

constexpr int MX_U = 4;      // pieces of 16 bytes that a lane has on their way

// A lane takes 16 bytes at a time, so 32 / VEC neighbouring lanes share a block, whose largest
// value goes round between them in registers.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ X,
                                                          uint8_t* __restrict__ Q,
                                                          uint8_t* __restrict__ scale, long n) {
  const long stride = (long)gridDim.x * 256 * VEC * MX_U;
  for (long e0 = ((long)blockIdx.x * 256 * MX_U + threadIdx.x) * VEC; e0 < n; e0 += stride) {
    Piece<T, VEC> x[MX_U];
#pragma unroll
    for (int u = 0; u < MX_U; ++u) {      // past the end: the first again, not stored
      const long e = e0 + u * 256 * VEC;
      x[u].load(X + (e < n ? e : e0));
    }
#pragma unroll
    for (int u = 0; u < MX_U; ++u) {
      const long e = e0 + u * 256 * VEC;
      if (e >= n) break;
      float v[VEC];
      x[u].get(v);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < VEC; ++i) top = max(top, magnitude(v[i]));
      const uint32_t byte = mx_byte(mx_block_max<VEC>(top));
      mx_store<VEC>(Q + e, v, mx_inverse(byte));
      if (e % MX_BLOCK == 0) scale[e / MX_BLOCK] = (uint8_t)byte;
    }
  }
}

template <typename T, int VEC>
hipError_t run_quantize(const T* X, uint8_t* Q, uint8_t* scale, long n, hipStream_t st) {
  constexpr long per = 256l * VEC * MX_U;
  const long blocks = (n + per - 1) / per;
  // one dimension of a launch ends below 2^32 threads
  const long grid = blocks < (1l << 22) ? blocks : 1l << 22;
  mx_quantize_kernel<T, VEC><<<dim3((unsigned)grid), 256, 0, st>>>(X, Q, scale, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(int dtype, const void* X, uint8_t* Q, uint8_t* scale, long n,
                              hipStream_t st) {
  if (n == 0) return hipSuccess;
  if (dtype == DT_F32) return run_quantize<float, 4>((const float*)X, Q, scale, n, st);
  return run_quantize<bf16_t, 8>((const bf16_t*)X, Q, scale, n, st);
}

}  // namespace ec
