// Root-mean-square norm of rows, the residual added first, and its backward pass:
//   h = round(x + residual) (x without one),  r = (mean(h^2) + eps)^-1/2,  y = h r w;
//   dx = r (g - h r^2 mean(g h)) + dh,  g = w dy,  dw = sum over the rows of dy h r.
// The norm is that of the sum as it is stored, so that the backward pass needs h alone.
// Sums in fp32; y is rounded once, to the storage type or to eight bits (mx.h).
//
// Memory bounds both: every row moves once and is held in registers between its sum and its
// use.  A row belongs to TPR lanes, each of which takes V pieces of VEC elements (16 bytes, or
// one element where the row's length leaves its rows unaligned).
#include "mx.h"
#include "ec_kernels.h"

namespace ec {

namespace {

// Sum over a wave, the same bits in every lane.
__device__ __forceinline__ float wave_sum(float t) {
  t = row16_sum_even(t);
  const int i = __builtin_bit_cast(int, t);
  const auto at = [&](int l) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, l));
  };
  return (at(0) + at(16)) + (at(32) + at(48));
}

// Sums of NS values over a row's lanes: TPR / 64 waves.  `red` holds two sets of NS values a
// wave, taken in turn, so that one barrier a row is enough.
template <int TPR, int NS>
__device__ __forceinline__ void row_sums(float (&s)[NS], float* red, int turn) {
#pragma unroll
  for (int n = 0; n < NS; ++n) s[n] = wave_sum(s[n]);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    float* r = red + turn * NW * NS;
    const int w = threadIdx.x >> 6;
    if (wave_lane() == 0)
#pragma unroll
      for (int n = 0; n < NS; ++n) r[w * NS + n] = s[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) s[n] += r[i * NS + n];
    }
  }
}

template <int TPR>
constexpr int norm_threads() { return TPR < 256 ? 256 : TPR; }

// One row a group of TPR lanes and step; MX: eight bits out.
template <typename T, int VEC, int V, int TPR, bool MX>
__global__ __launch_bounds__(norm_threads<TPR>()) void rms_norm_kernel(
    const T* X, const T* R, const T* __restrict__ w, T* H, T* __restrict__ Y,
    uint8_t* __restrict__ Q, uint8_t* __restrict__ scale, long rows, int d, float eps) {
  constexpr int RB = norm_threads<TPR>() / TPR;
  __shared__ float red[2 * (TPR / 64)];
  const int t = threadIdx.x % TPR;
  const float inv_d = 1.0f / (float)d;
  int turn = 0;
  for (long row = (long)blockIdx.x * RB + threadIdx.x / TPR; row < rows;
       row += (long)gridDim.x * RB, turn ^= 1) {
    const long at = row * d;
    float h[V][VEC];
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c < d) {
        load_vec<T, VEC>(X + at + c, h[v]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[v][i] = 0.f;
      }
    }
    if (R) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * VEC;
        if (c < d) {
          float q[VEC];
          load_vec<T, VEC>(R + at + c, q);
#pragma unroll
          for (int i = 0; i < VEC; ++i) h[v][i] = round_to<T>(h[v][i] + q[i]);
        }
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[0] = fmaf(h[v][i], h[v][i], s[0]);
    row_sums<TPR, 1>(s, red, turn);
    const float r = 1.0f / sqrtf(fmaf(s[0], inv_d, eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c >= d) break;
      if (R) store_vec<T, VEC>(H + at + c, h[v]);
      float y[VEC], q[VEC];
      load_vec<T, VEC>(w + c, q);
#pragma unroll
      for (int i = 0; i < VEC; ++i) y[i] = h[v][i] * r * q[i];
      if constexpr (MX) {   // d is a multiple of 32: a block's lanes are all here
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = max(top, magnitude(y[i]));
        const uint32_t byte = mx_byte(mx_block_max<VEC>(top));
        const float inverse = mx_inverse(byte);
        if constexpr (VEC == 8)
          *reinterpret_cast<uint2*>(Q + at + c) =
              make_uint2(mx_codes4(y, inverse), mx_codes4(y + 4, inverse));
        else
          *reinterpret_cast<uint32_t*>(Q + at + c) = mx_codes4(y, inverse);
        if (c % MX_BLOCK == 0) scale[(at + c) / MX_BLOCK] = (uint8_t)byte;
      } else {
        store_vec<T, VEC>(Y + at + c, y);
      }
    }
  }
}

// A workgroup takes every gridDim.x-th set of rows and keeps its share of dw in registers;
// part [gridDim.x, d] (dw itself where one workgroup takes all rows).
template <typename T, int VEC, int V, int TPR>
__global__ __launch_bounds__(norm_threads<TPR>()) void rms_norm_backward_kernel(
    const T* H, const T* __restrict__ w, const T* dY, const T* dH, T* dX,
    float* __restrict__ part, long rows, int d, float eps) {
  constexpr int RB = norm_threads<TPR>() / TPR;
  __shared__ float red[4 * (TPR / 64)];
  const int t = threadIdx.x % TPR;
  const float inv_d = 1.0f / (float)d;
  float dw[V][VEC];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[v][i] = 0.f;
  int turn = 0;
  for (long row = (long)blockIdx.x * RB + threadIdx.x / TPR; row < rows;
       row += (long)gridDim.x * RB, turn ^= 1) {
    const long at = row * d;
    float h[V][VEC], g[V][VEC];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c < d) {
        load_vec<T, VEC>(H + at + c, h[v]);
        load_vec<T, VEC>(dY + at + c, g[v]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[v][i] = g[v][i] = 0.f;
      }
    }
    float wv[V][VEC];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c < d) load_vec<T, VEC>(w + c, wv[v]);
      else
#pragma unroll
        for (int i = 0; i < VEC; ++i) wv[v][i] = 0.f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        s[0] = fmaf(h[v][i], h[v][i], s[0]);
        s[1] = fmaf(g[v][i] * wv[v][i], h[v][i], s[1]);
      }
    }
    row_sums<TPR, 2>(s, red, turn);
    const float r = 1.0f / sqrtf(fmaf(s[0], inv_d, eps));
    const float k = r * r * (s[1] * inv_d);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c >= d) break;
      float x[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        dw[v][i] = fmaf(g[v][i], h[v][i] * r, dw[v][i]);
        x[i] = r * (g[v][i] * wv[v][i] - h[v][i] * k);
      }
      if (dH) {
        float q[VEC];
        load_vec<T, VEC>(dH + at + c, q);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] += q[i];
      }
      store_vec<T, VEC>(dX + at + c, x);
    }
  }
  float* out = part + (long)blockIdx.x * d;
  if constexpr (RB == 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * VEC;
      if (c < d) store_vec<float, VEC>(out + c, dw[v]);
    }
  } else {
    // the workgroup's row groups add to one another in turn
    __shared__ float sum[V * TPR * VEC];
    for (int b = 0; b < RB; ++b) {
      if ((int)threadIdx.x / TPR == b) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float* p = &sum[(v * TPR + t) * VEC + i];
            *p = b == 0 ? dw[v][i] : *p + dw[v][i];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < d; c += norm_threads<TPR>()) out[c] = sum[c];
  }
}

// dw[c] = sum of part[i, c]: 64 columns a workgroup, its 16 waves each every 16th row.
__global__ __launch_bounds__(1024) void rms_norm_dw_kernel(const float* __restrict__ part,
                                                           float* __restrict__ dw, int n, int d) {
  __shared__ float s[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), g = threadIdx.x >> 6;
  float t = 0.f;
  if (c < d)
    for (int i = g; i < n; i += 16) t += part[(long)i * d + c];
  s[g][threadIdx.x & 63] = t;
  __syncthreads();
  if (g == 0 && c < d) {
    t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
    dw[c] = t;
  }
}

constexpr int kNormGrid = 1 << 20;   // workgroups of a forward launch at most

// Calls body(VEC, V, TPR) as types with the smallest group of lanes that holds a row in at most
// four pieces each.
template <typename T, typename F>
hipError_t with_shape(int d, F body) {
  constexpr int W = 16 / sizeof(T);
  const auto ints = [&](auto vec, auto v, auto tpr) { return body(vec, v, tpr); };
#define EC_I(n) std::integral_constant<int, n>{}
  if (d % W == 0) {
    const int u = d / W;
    if (u <= 64) return ints(EC_I(W), EC_I(1), EC_I(64));
    if (u <= 128) return ints(EC_I(W), EC_I(2), EC_I(64));
    if (u <= 256) return ints(EC_I(W), EC_I(4), EC_I(64));
    if (u <= 512) return ints(EC_I(W), EC_I(2), EC_I(256));
    if (u <= 1024) return ints(EC_I(W), EC_I(4), EC_I(256));
    if (u <= 2048) return ints(EC_I(W), EC_I(2), EC_I(1024));
    return ints(EC_I(W), EC_I(4), EC_I(1024));
  }
  if (d <= 256) return ints(EC_I(1), EC_I(4), EC_I(64));
  if (d <= 1024) return ints(EC_I(1), EC_I(4), EC_I(256));
  if (d <= 4096) return ints(EC_I(1), EC_I(4), EC_I(1024));
  return ints(EC_I(1), EC_I(16), EC_I(1024));
#undef EC_I
}

template <typename T>
hipError_t run_norm(const void* X, const void* R, const void* w, void* H, void* Y, uint8_t* Q,
                    uint8_t* scale, long rows, int d, float eps, hipStream_t st) {
  return with_shape<T>(d, [&](auto vec, auto v, auto tpr) {
    constexpr int VEC = decltype(vec)::value, V = decltype(v)::value, TPR = decltype(tpr)::value;
    constexpr int RB = norm_threads<TPR>() / TPR;
    const long blocks = (rows + RB - 1) / RB;
    const dim3 grid((unsigned)(blocks < kNormGrid ? blocks : kNormGrid));
    if (Q) {
      if constexpr (VEC > 1)
        rms_norm_kernel<T, VEC, V, TPR, true><<<grid, norm_threads<TPR>(), 0, st>>>(
            (const T*)X, (const T*)R, (const T*)w, (T*)H, nullptr, Q, scale, rows, d, eps);
      else
        return hipErrorInvalidValue;
    } else {
      rms_norm_kernel<T, VEC, V, TPR, false><<<grid, norm_threads<TPR>(), 0, st>>>(
          (const T*)X, (const T*)R, (const T*)w, (T*)H, (T*)Y, nullptr, nullptr, rows, d, eps);
    }
    return hipGetLastError();
  });
}

template <typename T>
hipError_t run_norm_backward(const void* H, const void* w, const void* dY, const void* dH, void* dX,
                             float* dw, float* part, int blocks, long rows, int d, float eps,
                             hipStream_t st) {
  hipError_t e = with_shape<T>(d, [&](auto vec, auto v, auto tpr) {
    constexpr int VEC = decltype(vec)::value, V = decltype(v)::value, TPR = decltype(tpr)::value;
    rms_norm_backward_kernel<T, VEC, V, TPR>
        <<<dim3((unsigned)blocks), norm_threads<TPR>(), 0, st>>>(
            (const T*)H, (const T*)w, (const T*)dY, (const T*)dH, (T*)dX,
            blocks > 1 ? part : dw, rows, d, eps);
    return hipGetLastError();
  });
  if (e != hipSuccess || blocks <= 1) return e;
  rms_norm_dw_kernel<<<dim3((unsigned)((d + 63) / 64)), 1024, 0, st>>>(part, dw, blocks, d);
  return hipGetLastError();
}

}  // namespace

int rms_norm_backward_blocks(int dtype, long rows, int d) {
  long per = 1;   // rows of a workgroup's step
  const auto rows_of = [&](auto, auto, auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    per = norm_threads<TPR>() / TPR;
    return hipSuccess;
  };
  const hipError_t e =
      dtype == DT_F32 ? with_shape<float>(d, rows_of) : with_shape<bf16_t>(d, rows_of);
  const long steps = e == hipSuccess ? (rows + per - 1) / per : 1;
  return (int)(steps < 1 ? 1 : steps < 512 ? steps : 512);
}

hipError_t launch_rms_norm(int dtype, const void* X, const void* R, const void* w, void* H, void* Y,
                           uint8_t* Q, uint8_t* scale, long rows, int d, float eps,
                           hipStream_t st) {
  if (rows == 0) return hipSuccess;
  return dtype == DT_F32 ? run_norm<float>(X, R, w, H, Y, Q, scale, rows, d, eps, st)
                         : run_norm<bf16_t>(X, R, w, H, Y, Q, scale, rows, d, eps, st);
}

hipError_t launch_rms_norm_backward(int dtype, const void* H, const void* w, const void* dY,
                                    const void* dH, void* dX, float* dw, float* part, long rows,
                                    int d, float eps, hipStream_t st) {
  const int blocks = rms_norm_backward_blocks(dtype, rows, d);
  return dtype == DT_F32
             ? run_norm_backward<float>(H, w, dY, dH, dX, dw, part, blocks, rows, d, eps, st)
             : run_norm_backward<bf16_t>(H, w, dY, dH, dX, dw, part, blocks, rows, d, eps, st);
}

}  // namespace ec
