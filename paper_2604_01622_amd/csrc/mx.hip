// A tensor in eight bits with scales (mx.h): the layout in which the experts' weights are
// held for serving.
#include "mx.h"
#include "ec_kernels.h"

namespace ec {

namespace {

// A lane takes 16 bytes at a time, so 32 / VEC neighbouring lanes share a block, whose largest
// value goes round between them in registers.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ X,
                                                          uint8_t* __restrict__ Q,
                                                          uint8_t* __restrict__ scale, long n) {
  const long stride = (long)gridDim.x * 256 * VEC;
  for (long e = ((long)blockIdx.x * 256 + threadIdx.x) * VEC; e < n; e += stride) {
    float v[VEC];
    load_vec<T, VEC>(X + e, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) top = max(top, magnitude(v[i]));
    const uint32_t byte = mx_byte(mx_block_max<VEC>(top));
    const float inverse = mx_inverse(byte);
    if constexpr (VEC == 8)
      *reinterpret_cast<uint2*>(Q + e) = make_uint2(mx_codes4(v, inverse), mx_codes4(v + 4, inverse));
    else
      *reinterpret_cast<uint32_t*>(Q + e) = mx_codes4(v, inverse);
    if (e % MX_BLOCK == 0) scale[e / MX_BLOCK] = (uint8_t)byte;
  }
}

template <typename T, int VEC>
hipError_t run_quantize(const T* X, uint8_t* Q, uint8_t* scale, long n, hipStream_t st) {
  const long blocks = (n / VEC + 255) / 256;
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
