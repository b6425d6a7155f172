// The balance loss of token choice, its per-expert counts and its gradient, and the router's
// dZ of token-choice training.
//
// Group g of L tokens, k choices a token: c_j = number of tokens that chose expert j (before
// any capacity drops pairs), P_j = mean of S_ij over the group;
//   loss_g = E / (k L) sum_j c_j P_j      (1 when the load is even; 0 for an empty group),
// the counts being constants of the gradient: with b_j = dloss_g E c_j / (k L^2),
//   dZ_ij = S_ij (b_j - sum_m S_im b_m) / tau.
//
// Every kernel takes the tokens in chunks that do not cross groups, sixteen lanes a token:
// lane r holds experts 4 r + 64 q + {0, 1, 2, 3}.  Chunks' sums are added in a fixed order,
// no atomics.  Sums of S, the dot product and the difference are in 64 bits (under an even
// load the difference is far below its terms).
#include "ec_common.h"
#include "ec_kernels.h"

namespace ec {

namespace {

// The group of a chunk: the last g with seg[g] <= chunk (empty groups have no chunks).
__device__ __forceinline__ int chunk_group(const ChunkTable& tab, int chunk) {
  int lo = 0, hi = tab.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tab.seg[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double row16_sum_f64(double t) {
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) t += __shfl_xor(t, m, 16);
  return t;
}

// Experts 4 r + 64 q + c of a row of E floats; entries past E read `fill`.
template <int Q>
__device__ __forceinline__ void load_row(const float* row, int E, int r, float fill,
                                         float v[Q][4]) {
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = 64 * q + 4 * r + c;
      v[q][c] = j < E ? row[j] : fill;
    }
}

// Sums of S and choices per expert over one chunk of tokens.
template <int Q>
__global__ __launch_bounds__(256) void balance_partial_kernel(const float* __restrict__ S, int E,
                                                              int k, ChunkTable tab,
                                                              double* __restrict__ psum,
                                                              int32_t* __restrict__ pcnt) {
  __shared__ double ssum[16][64 * Q];
  __shared__ int scnt[16][64 * Q];
  const int g = chunk_group(tab, blockIdx.x);
  const int t0 = (blockIdx.x - tab.seg[g]) * tab.chunk;
  const int t1 = t0 + tab.chunk < tab.len[g] ? t0 + tab.chunk : tab.len[g];
  const int r = threadIdx.x & 15, grp = threadIdx.x >> 4;
  double sum[Q][4];
  int cnt[Q][4];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      sum[q][c] = 0.0;
      cnt[q][c] = 0;
    }
  for (int t = t0 + grp; t < t1; t += 16) {   // uniform over the sixteen lanes
    float v[Q][4];
    load_row<Q>(S + (size_t)(tab.off[g] + t) * E, E, r, -INFINITY, v);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (64 * q + 4 * r + c < E) sum[q][c] += (double)v[q][c];
    uint32_t taken = 0;   // bit 4 q + c
    for (int n = 0; n < k; ++n) {
      float bv = -INFINITY;
      int bj = 1 << 30;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int j = 64 * q + 4 * r + c;
          if (j < E && !((taken >> (4 * q + c)) & 1u) &&
              (v[q][c] > bv || (v[q][c] == bv && j < bj))) {
            bv = v[q][c];
            bj = j;
          }
        }
#pragma unroll
      for (int m = 8; m >= 1; m >>= 1) {
        const float ov = __shfl_xor(bv, m, 16);
        const int oj = __shfl_xor(bj, m, 16);
        if (ov > bv || (ov == bv && oj < bj)) {
          bv = ov;
          bj = oj;
        }
      }
      // none left but NaN, which nothing chooses: bj >= E
      if (bj < E && ((bj >> 2) & 15) == r) taken |= 1u << ((bj >> 6) * 4 + (bj & 3));
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) cnt[q][c] += (taken >> (4 * q + c)) & 1u;
  }
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      ssum[grp][64 * q + 4 * r + c] = sum[q][c];
      scnt[grp][64 * q + 4 * r + c] = cnt[q][c];
    }
  __syncthreads();
  for (int j = threadIdx.x; j < E; j += 256) {
    double s = 0.0;
    int n = 0;
    for (int w = 0; w < 16; ++w) {
      s += ssum[w][j];
      n += scnt[w][j];
    }
    psum[(size_t)blockIdx.x * E + j] = s;
    pcnt[(size_t)blockIdx.x * E + j] = n;
  }
}

// Counts and loss of a group from its chunks' sums, a workgroup a group.
__global__ __launch_bounds__(256) void balance_finish_kernel(const double* __restrict__ psum,
                                                             const int32_t* __restrict__ pcnt,
                                                             int E, int k, ChunkTable tab,
                                                             float* __restrict__ loss,
                                                             int32_t* __restrict__ counts,
                                                             int32_t* __restrict__ counts2) {
  __shared__ double part[4];
  const int g = blockIdx.x, j = threadIdx.x;
  double x = 0.0;
  if (j < E) {
    double s = 0.0;
    int n = 0;
    for (int c = tab.seg[g]; c < tab.seg[g + 1]; ++c) {
      s += psum[(size_t)c * E + j];
      n += pcnt[(size_t)c * E + j];
    }
    counts[(size_t)g * E + j] = n;
    if (counts2) counts2[(size_t)g * E + j] = n;
    x = s * (double)n;
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  if ((j & 63) == 0) part[j >> 6] = x;
  __syncthreads();
  if (j == 0) {
    const double L = tab.len[g];
    const double all = part[0] + part[1] + part[2] + part[3];
    loss[g] = tab.len[g] > 0 ? (float)(all * E / (L * L * k)) : 0.f;
  }
}

// dZ of the loss alone, fp32 [N, E].
template <int Q>
__global__ __launch_bounds__(256) void balance_backward_kernel(const float* __restrict__ S,
                                                               const int32_t* __restrict__ counts,
                                                               const float* __restrict__ dloss,
                                                               int E, int k, float inv_tau,
                                                               ChunkTable tab,
                                                               float* __restrict__ dZ) {
  const int g = chunk_group(tab, blockIdx.x);
  const int t0 = (blockIdx.x - tab.seg[g]) * tab.chunk;
  const int t1 = t0 + tab.chunk < tab.len[g] ? t0 + tab.chunk : tab.len[g];
  const int r = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const double L = tab.len[g];
  const double coef = (double)dloss[g] * E / (L * L * k) * inv_tau;
  double b[Q][4];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = 64 * q + 4 * r + c;
      b[q][c] = j < E ? coef * counts[(size_t)g * E + j] : 0.0;
    }
  for (int t = t0 + grp; t < t1; t += 16) {
    const size_t at = (size_t)(tab.off[g] + t) * E;
    float v[Q][4];
    load_row<Q>(S + at, E, r, 0.f, v);
    double dot = 0.0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) dot += (double)v[q][c] * b[q][c];
    dot = row16_sum_f64(dot);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = 64 * q + 4 * r + c;
        if (j < E) dZ[at + j] = (float)((double)v[q][c] * (b[q][c] - dot));
      }
  }
}

// The router's dZ of token-choice training.  Over the chosen experts C_i of a token the
// gates are a softmax of their logits, so with u_ij = g_ij dL/dg_ij (what the dA product's
// partials of a packed row sum to; 0 for a dropped pair)
//   dZ_ij = (u_ij - g_ij sum_m u_im) / tau,
// nothing elsewhere and nothing at all for one choice, whose gate is 1; plus the balance
// loss's term with dloss.
template <int Q, typename T>
__global__ __launch_bounds__(256) void tc_dz_kernel(const float* __restrict__ S,
                                                    const float* __restrict__ G,
                                                    const int32_t* __restrict__ slotT,
                                                    const float* __restrict__ dsp, int nparts,
                                                    const int32_t* __restrict__ counts,
                                                    const float* __restrict__ dloss,
                                                    T* __restrict__ dZ, int N, int E, int EP,
                                                    int k, int max_rows, float inv_tau,
                                                    ChunkTable tab) {
  const int g = chunk_group(tab, blockIdx.x);
  const int t0 = (blockIdx.x - tab.seg[g]) * tab.chunk;
  const int t1 = t0 + tab.chunk < tab.len[g] ? t0 + tab.chunk : tab.len[g];
  const int r = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const double L = tab.len[g];
  const double coef = dloss ? (double)dloss[g] * E / (L * L * k) : 0.0;
  double b[Q][4];
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = 64 * q + 4 * r + c;
      b[q][c] = dloss && j < E ? coef * counts[(size_t)g * E + j] : 0.0;
    }
  for (int t = t0 + grp; t < t1; t += 16) {
    const int i = tab.off[g] + t;
    float v[Q][4], gt[Q][4], u[Q][4];
    load_row<Q>(G + (size_t)i * E, E, r, 0.f, gt);
    float all = 0.f;
    double dot = 0.0;
    if (dloss) load_row<Q>(S + (size_t)i * E, E, r, 0.f, v);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = 64 * q + 4 * r + c;
        u[q][c] = 0.f;
        if (k > 1 && gt[q][c] != 0.f) {
          const int row = slotT[(size_t)j * N + i];
          if (row >= 0 && row < max_rows)
            for (int n = 0; n < nparts; ++n) u[q][c] += dsp[(size_t)row * nparts + n];
        }
        all += u[q][c];
        if (dloss) dot += (double)v[q][c] * b[q][c];
      }
    all = row16_sum(all);
    if (dloss) dot = row16_sum_f64(dot);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = 64 * q + 4 * r + c;
        float z = k > 1 ? u[q][c] - gt[q][c] * all : 0.f;
        if (dloss) z = (float)((double)z + (double)v[q][c] * (b[q][c] - dot));
        if (j < EP) Elem<T>::store1(dZ + (size_t)i * EP + j, z * inv_tau);
      }
  }
}

}  // namespace

// 1024 chunks of a large batch; 64 tokens at least.
int balance_chunk(int N) {
  const int c = (N + 1023) / 1024;
  return c <= 64 ? 64 : (c + 63) / 64 * 64;
}

#define EC_BY_WIDTH(E, CALL)         \
  do {                               \
    if ((E) <= 64) CALL(1);          \
    else if ((E) <= 128) CALL(2);    \
    else if ((E) <= 192) CALL(3);    \
    else CALL(4);                    \
  } while (0)

hipError_t launch_balance_partial(const float* S, int E, int k, const ChunkTable& tab,
                                  double* psum, int32_t* pcnt, hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
#define EC_CALL(Q) balance_partial_kernel<Q><<<grid, 256, 0, st>>>(S, E, k, tab, psum, pcnt)
  EC_BY_WIDTH(E, EC_CALL);
#undef EC_CALL
  return hipGetLastError();
}

hipError_t launch_balance_finish(const double* psum, const int32_t* pcnt, int E, int k,
                                 const ChunkTable& tab, float* loss, int32_t* counts,
                                 int32_t* counts2, hipStream_t st) {
  if (tab.n == 0) return hipSuccess;
  balance_finish_kernel<<<tab.n, 256, 0, st>>>(psum, pcnt, E, k, tab, loss, counts, counts2);
  return hipGetLastError();
}

hipError_t launch_balance_backward(const float* S, const int32_t* counts, const float* dloss,
                                   int E, int k, float inv_tau, const ChunkTable& tab, float* dZ,
                                   hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
#define EC_CALL(Q) \
  balance_backward_kernel<Q><<<grid, 256, 0, st>>>(S, counts, dloss, E, k, inv_tau, tab, dZ)
  EC_BY_WIDTH(E, EC_CALL);
#undef EC_CALL
  return hipGetLastError();
}

hipError_t launch_tc_router_dz(int dtype, const float* S, const float* G, const int32_t* slotT,
                               const float* dsp, int nparts, const int32_t* counts,
                               const float* dloss, void* dZ, int N, int E, int EP, int k,
                               int max_rows, float inv_tau, const ChunkTable& tab,
                               hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
#define EC_CALL(Q)                                                                              \
  do {                                                                                          \
    if (dtype == DT_F32)                                                                        \
      tc_dz_kernel<Q, float><<<grid, 256, 0, st>>>(S, G, slotT, dsp, nparts, counts, dloss,     \
                                                   (float*)dZ, N, E, EP, k, max_rows, inv_tau,  \
                                                   tab);                                        \
    else                                                                                        \
      tc_dz_kernel<Q, bf16_t><<<grid, 256, 0, st>>>(S, G, slotT, dsp, nparts, counts, dloss,    \
                                                    (bf16_t*)dZ, N, E, EP, k, max_rows,         \
                                                    inv_tau, tab);                              \
  } while (0)
  EC_BY_WIDTH(E, EC_CALL);
#undef EC_CALL
  return hipGetLastError();
}

}  // namespace ec
