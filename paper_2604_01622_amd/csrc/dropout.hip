// Dropout onto a residual, and its backward pass: Y = R + mask * scale * X, the mask drawn
// from a counter-based generator (dropout.h) and never stored.
#include "dropout.h"

namespace ec {

namespace {

// A thread takes chunks of eight elements (one block of draws), 16 bytes of bf16 or 32 of
// fp32, a workgroup's consecutive.  Memory bounds it.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* X, const T* R, Dropout drop, T* Y,
                                                      long n) {
  const uint64_t seed = drop.thr ? drop.rng[0] : 0, offset = drop.thr ? drop.rng[1] : 0;
  const long stride = (long)gridDim.x * 256;
  for (long c = (long)blockIdx.x * 256 + threadIdx.x; c < (n + 7) / 8; c += stride) {
    const bool whole = c * 8 + 8 <= n;
    const int tail = whole ? 8 : (int)(n - c * 8);
    float v[8], r[8];
    if (whole) {
      Elem<T>::load8(X + c * 8, v);
      if (R) Elem<T>::load8(R + c * 8, r);
    } else {
      for (int u = 0; u < 8; ++u) {
        v[u] = u < tail ? Elem<T>::load1(X + c * 8 + u) : 0.f;
        r[u] = u < tail && R ? Elem<T>::load1(R + c * 8 + u) : 0.f;
      }
    }
    if (drop.thr) dropout_apply(v, dropout_block((uint64_t)c, seed, offset), drop.thr, drop.scale);
    if (R)
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] += r[u];
    if (whole) {
      Elem<T>::store8(Y + c * 8, v);
    } else {
      for (int u = 0; u < 8; ++u)
        if (u < tail) Elem<T>::store1(Y + c * 8 + u, v[u]);
    }
  }
}

template <typename T>
hipError_t run_dropout(const T* X, const T* R, const Dropout& drop, T* Y, long n, hipStream_t st) {
  const long blocks = ((n + 7) / 8 + 255) / 256;
  // one dimension of a launch ends below 2^32 threads
  const long grid = blocks < (1l << 22) ? blocks : 1l << 22;
  dropout_kernel<T><<<dim3((unsigned)grid), 256, 0, st>>>(X, R, drop, Y, n);
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
