// The balance loss of token choice, its per-expert counts and its gradient, and the router's
// dZ of token-choice training.
//
// Group g of L tokens, k choices a token: c_j = number of tokens that chose expert j (before
// any capacity drops pairs), P_j = mean of S_ij over the group;
//   loss_g = E / (k L) sum_j c_j P_j      (1 when the load is even; 0 for an empty group),
// the counts being constants of the gradient: with b_j = dloss_g E c_j / (k L^2),
//   dZ_ij = S_ij (b_j - sum_m S_im b_m) / tau.
//
// Every kernel takes the tokens in chunks that do not cross groups, sixteen lanes (a DPP row)
// a token: lane r holds experts 4 r + 64 q + {0, 1, 2, 3}, one 16-byte load a quarter row.
// Chunks' sums are added in a fixed order, no atomics.  Sums of S, the dot product and the
// difference are in 64 bits (under an even load the difference is far below its terms).
//
// Latency bounds all but the largest: 16384 tokens x 64 experts, top 8, 5.6 (sums), 4.2
// (finish) and 5.6 us (gradient) for 4.2, 0.2 and 8.4 MB.  65536 x 256, top 8: 26.7, 5.6 and 25.6
// us.  Of the sums' 26.7, some 15 are the issue of the instructions that choose (560 a wave for
// four tokens; a pass over all sixteen registers each round, without the sort, 32.1); a
// workgroup's twelve waves, one a CU, take its 256 tokens in six passes, the last a third full, and
// nothing runs beside the reduction over the waves at the end.  The gradient moves 134 MB at 5.2
// TB/s.
#include <type_traits>

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
  for (int q = 0; q < Q; ++q) {
    const int j0 = 64 * q + 4 * r;
    if (E % 4 == 0) {   // rows start at a multiple of 16 bytes
      const float4 x = *reinterpret_cast<const float4*>(row + (j0 < E ? j0 : 0));
      const bool in = j0 < E;
      v[q][0] = in ? x.x : fill;
      v[q][1] = in ? x.y : fill;
      v[q][2] = in ? x.z : fill;
      v[q][3] = in ? x.w : fill;
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float x = row[j0 + c < E ? j0 + c : 0];
        v[q][c] = j0 + c < E ? x : fill;
      }
    }
  }
}

template <int Q>
__device__ __forceinline__ void store_row(float* row, int E, int r, const float v[Q][4]) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int j0 = 64 * q + 4 * r;
    if (E % 4 == 0) {
      if (j0 < E)
        *reinterpret_cast<float4*>(row + j0) = make_float4(v[q][0], v[q][1], v[q][2], v[q][3]);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (j0 + c < E) row[j0 + c] = v[q][c];
    }
  }
}

// v[a] >= v[b] from now on.
__device__ __forceinline__ void order_pair(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}

// Eight keys in falling order (19 exchanges, odd-even merging of halves).
__device__ __forceinline__ void sort8(uint32_t x[8]) {
  constexpr uint8_t A[19] = {0, 2, 4, 6, 0, 1, 4, 5, 1, 5, 0, 1, 2, 3, 2, 3, 1, 3, 5};
  constexpr uint8_t B[19] = {1, 3, 5, 7, 2, 3, 6, 7, 2, 6, 4, 5, 6, 7, 4, 5, 2, 4, 6};
#pragma unroll
  for (int i = 0; i < 19; ++i) order_pair(x[A[i]], x[B[i]]);
}

// The eight largest of a lane's 4 Q keys in falling order, zeros behind fewer.
template <int Q>
__device__ __forceinline__ void top8(const uint32_t w[Q][4], uint32_t top[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top[i] = i < 4 * Q ? w[i / 4][i % 4] : 0;
  sort8(top);
  if constexpr (Q > 2) {   // the larger of the ends of two sorted lists are bitonic
    uint32_t more[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) more[i] = i + 8 < 4 * Q ? w[i / 4 + 2][i % 4] : 0;
    sort8(more);
#pragma unroll
    for (int i = 0; i < 8; ++i) top[i] = max(top[i], more[7 - i]);
#pragma unroll
    for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((i & s) == 0) order_pair(top[i], top[i + s]);
  }
}

// Takes the k largest entries out of the four rows that a wave holds (ties: the lower
// expert; NaN, also in the entries past E, is never taken); a taken entry's key ends as 0.
// Keys are integers in the scores' order (f32_order_key's; 0 for NaN), whose maxima take no care
// for NaN.  Every lane sorts its largest eight once; a round is a maximum over the lanes' first
// ones, and the lanes that held it go on to their next.  The k-th round's maximum is the
// smallest entry to take (a lane with more than eight entries may run out past eight rounds:
// then a round is a maximum, a compare and a select per entry).  Only where some row so loses
// more or fewer than k (equal scores among its largest, or not k numbers) does the wave
// start over, one lowest expert at a time.  Every lane takes part.
template <int Q>
__device__ __forceinline__ void take_largest(uint32_t w[Q][4], const float v[Q][4], int r, int k) {
  auto keys = [&] {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int u = __float_as_int(v[q][c] + 0.f);   // -0 equals 0
        w[q][c] = v[q][c] == v[q][c] ? (uint32_t)(u ^ (u >> 31 | (int)0x80000000)) : 0;
      }
  };
  auto row_max = [&]() -> uint32_t {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      m = max(m, max(w[q][0], w[q][1]));
      m = max(m, max(w[q][2], w[q][3]));
    }
    return row16_max_u32(m);
  };
  keys();
  if (Q <= 2 || k <= 8) {
    constexpr int L = Q == 1 ? 4 : 8;
    uint32_t top[8], m = 0;
    top8<Q>(w, top);
    for (int n = 0; n < k; ++n) {
      m = row16_max_u32(top[0]);
      const bool held = top[0] == m;
#pragma unroll
      for (int i = 0; i < L; ++i) {   // values, not places: a choice of places is an index
        const uint32_t stay = top[i], next = i + 1 < L ? top[i + 1] : 0;
        top[i] = held ? next : stay;
      }
    }
    int took = m == 0 ? -4 * Q : 0;   // no k numbers: less than any k in all
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool take = w[q][c] >= m;
        took += take;
        w[q][c] = take ? 0 : w[q][c];
      }
    if (!__any(row16_sum_i32(took) != k)) return;
  } else {
    for (int n = 0; n < k; ++n) {
      const uint32_t m = row_max();
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) w[q][c] = w[q][c] == m ? 0 : w[q][c];
    }
    int took = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) took += w[q][c] == 0 && v[q][c] == v[q][c];
    if (!__any(row16_sum_i32(took) != k)) return;
  }
  keys();
  for (int n = 0; n < k; ++n) {
    const uint32_t m = row_max();
    int first = 1 << 30;
    if (m != 0) {
#pragma unroll
      for (int q = Q - 1; q >= 0; --q)
#pragma unroll
        for (int c = 3; c >= 0; --c) first = w[q][c] == m ? 64 * q + 4 * r + c : first;
    }
    first = row16_min_i32(first);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) w[q][c] = 64 * q + 4 * r + c == first ? 0 : w[q][c];
  }
}

// Threads of a workgroup that sums: 1024, 768 where a row takes four quarters (more than 192
// experts), whose sums need more registers than a lane of 16 waves has.
template <int Q> constexpr int BL_THREADS = Q == 4 ? 768 : 1024;

__device__ __forceinline__ float group_loss(double sum, int E, int k, int len) {
  const double L = len;
  return len > 0 ? (float)(sum * E / (L * L * k)) : 0.f;
}

// The group's loss and counts from its sums: thread j < E holds expert j's.
__device__ __forceinline__ void finish_group(double sum, int count, int E, int k, int len, size_t g,
                                             double* red, float* loss, int32_t* counts) {
  const int j = threadIdx.x;
  if (j < E) counts[g * E + j] = count;
  double x = j < E ? sum * (double)count : 0.0;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  if ((j & 63) == 0 && j < 256) red[j >> 6] = x;   // E <= 256
  __syncthreads();
  if (j == 0) loss[g] = group_loss(red[0] + red[1] + red[2] + red[3], E, k, len);
}

// Sums of S and choices per expert over one chunk of tokens.  WHOLE: every group is one
// chunk, whose workgroup also finishes it.  TRAIN (chunks of TC_CHOOSE_CHUNK): also writes the
// gates of each token's choices (G [N, E], 0 elsewhere) and the choice flags flagT [E, N],
// transposed through LDS.
template <int Q, bool WHOLE, bool TRAIN>
__global__ __launch_bounds__(BL_THREADS<Q>) void balance_partial_kernel(
    const float* __restrict__ S, int E, int k, ChunkTable tab, double* __restrict__ psum,
    int32_t* __restrict__ pcnt, int32_t* __restrict__ done, float* __restrict__ loss,
    int32_t* __restrict__ counts, float* __restrict__ G, int32_t* __restrict__ flagT, int N) {
  constexpr int WAVES = BL_THREADS<Q> / 64;
  __shared__ double ssum[WAVES][64 * Q];
  __shared__ int scnt[WAVES][64 * Q];
  __shared__ double red[4];
  __shared__ uint8_t sflag[TRAIN ? TC_CHOOSE_CHUNK : 1][64 * Q + 4];
  const int g = WHOLE ? blockIdx.x : chunk_group(tab, blockIdx.x);
  const int t0 = WHOLE ? 0 : (blockIdx.x - tab.seg[g]) * tab.chunk;
  const int nt = min(tab.chunk, tab.len[g] - t0);   // tokens of the chunk
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15;
  double sum[Q][4];
  uint32_t cnt[Q][2];   // two counts a register: a lane has at most 65536 / 48 tokens
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      sum[q][c] = 0.0;
      cnt[q][c / 2] = 0;
    }
  // a wave's four tokens at a time, the next four's scores requested before these are chosen
  const int first = tab.off[g] + t0;
  float next[Q][4];
  auto request = [&](int tw) {
    const int t = tw + (lane >> 4);
    load_row<Q>(S + (size_t)(first + (t < nt ? t : nt - 1)) * E, E, r, __builtin_nanf(""), next);
  };
  if (wave * 4 < nt) request(wave * 4);
  for (int tw = wave * 4; tw < nt; tw += 4 * WAVES) {
    const int t = tw + (lane >> 4), i = first + (t < nt ? t : nt - 1);
    float v[Q][4];
    uint32_t w[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[q][c] = next[q][c];
    if (tw + 4 * WAVES < nt) request(tw + 4 * WAVES);
    take_largest<Q>(w, v, r, k);
    float inv = 1.f;
    if constexpr (TRAIN) {   // the gates' sum, the same in all lanes of the row
      float chosen = 0.f;
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          chosen += w[q][c] == 0 && v[q][c] == v[q][c] ? v[q][c] : 0.f;
      inv = 1.0f / row16_sum_even(chosen);
    }
    auto add = [&](auto all) {   // all: no row of the wave's four lies past the chunk
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const bool taken = w[q][c] == 0 && v[q][c] == v[q][c];
          if (decltype(all)::value || t < nt) {
            sum[q][c] += (double)v[q][c];
            cnt[q][c / 2] += taken ? 1u << (c % 2 * 16) : 0u;
          }
          if constexpr (TRAIN) {
            sflag[t][64 * q + 4 * r + c] = taken;   // t < TC_CHOOSE_CHUNK
            v[q][c] = taken ? v[q][c] * inv : 0.f;
          }
        }
    };
    // (training's has no registers for both forms)
    if (!TRAIN && tw + 4 <= nt) add(std::true_type{}); else add(std::false_type{});
    if constexpr (TRAIN) {
      if (t < nt) store_row<Q>(G + (size_t)i * E, E, r, v);
    }
  }
  // the four rows of a wave, then the waves in order
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      double s = sum[q][c];
      int n = (int)(c % 2 ? cnt[q][c / 2] >> 16 : cnt[q][c / 2] & 0xffffu);
      s += __shfl_xor(s, 16, 64);
      n += __shfl_xor(n, 16, 64);
      s += __shfl_xor(s, 32, 64);
      n += __shfl_xor(n, 32, 64);
      if (lane < 16) {
        ssum[wave][64 * q + 4 * r + c] = s;
        scnt[wave][64 * q + 4 * r + c] = n;
      }
    }
  __syncthreads();
  const int j = threadIdx.x;
  double s = 0.0;
  int n = 0;
  if (j < E) {
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      s += ssum[w][j];
      n += scnt[w][j];
    }
  }
  if constexpr (WHOLE) {
    finish_group(s, n, E, k, tab.len[g], g, red, loss, counts);
  } else {
    if (j < E) {
      psum[(size_t)blockIdx.x * E + j] = s;
      pcnt[(size_t)blockIdx.x * E + j] = n;
    }
    if (j == 0 && t0 == 0) done[g] = 0;
  }
  if constexpr (TRAIN) {
    for (int c = threadIdx.x; c < E * TC_CHOOSE_CHUNK; c += BL_THREADS<Q>) {
      const int e = c / TC_CHOOSE_CHUNK, t = c % TC_CHOOSE_CHUNK;
      if (t < nt) flagT[(size_t)e * N + first + t] = sflag[t][e];
    }
  }
}

// Counts and loss of a group from its chunks' sums, a workgroup for every 64 experts: its
// sixteen waves share the chunks out, 4 Q loads of each in flight (256 chunks of a group of 65536
// tokens and 256 experts: 5.6 us; one workgroup for all 256 experts 12.1, with a loop of single
// loads 272).  With more than one workgroup a group (Q > 1), the last to arrive adds their
// parts of the loss, in order: done [n] counts them and is 0 before (the sums' kernel clears it).
template <int Q>
__global__ __launch_bounds__(1024) void balance_finish_kernel(
    const double* __restrict__ psum, const int32_t* __restrict__ pcnt, int E, int k,
    ChunkTable tab, double* part, int32_t* done, float* __restrict__ loss,
    int32_t* __restrict__ counts, int32_t* __restrict__ counts2, int32_t* __restrict__ kept) {
  constexpr int WAVES = 16, B = 4 * Q;
  __shared__ double ssum[WAVES][64];
  __shared__ int scnt[WAVES][64];
  const int g = blockIdx.x / Q, quarter = blockIdx.x % Q;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = 64 * quarter + lane;
  const int begin = tab.seg[g], end = tab.seg[g + 1];
  double s = 0.0;
  int n = 0;
  if (j < E) {
    for (int c0 = begin + wave; c0 < end; c0 += B * WAVES) {
      double x[B];
      int y[B];
#pragma unroll
      for (int u = 0; u < B; ++u) {   // past the end: the last chunk again, not added
        const int c = c0 + u * WAVES < end ? c0 + u * WAVES : end - 1;
        x[u] = psum[(size_t)c * E + j];
        y[u] = pcnt[(size_t)c * E + j];
      }
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const bool in = c0 + u * WAVES < end;
        s += in ? x[u] : 0.0;
        n += in ? y[u] : 0;
      }
    }
  }
  ssum[wave][lane] = s;
  scnt[wave][lane] = n;
  __syncthreads();
  if (wave != 0) return;
  s = 0.0;
  n = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    s += ssum[w][lane];
    n += scnt[w][lane];
  }
  if (j < E) {
    const size_t at = (size_t)g * E + j;
    counts[at] = n;
    if (counts2) counts2[at] = n;
    if (kept) kept[at] = n < tab.cap[g] ? n : tab.cap[g];
  }
  double x = s * (double)n;   // 0 past the experts
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  if (lane != 0) return;
  if (begin == end) {   // no tokens, so no sums' workgroup that cleared done
    if (quarter == 0) loss[g] = 0.f;
    return;
  }
  if constexpr (Q > 1) {
    __hip_atomic_store(part + g * Q + quarter, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(done + g, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) != Q - 1)
      return;
    x = 0.0;
#pragma unroll
    for (int i = 0; i < Q; ++i)
      x += __hip_atomic_load(part + g * Q + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  loss[g] = group_loss(x, E, k, tab.len[g]);
}

// dZ of the loss alone, fp32 [N, E].
template <int Q>
__global__ __launch_bounds__(256) void balance_backward_kernel(const float* S,
                                                               const int32_t* __restrict__ counts,
                                                               const float* __restrict__ dloss,
                                                               int E, int k, float inv_tau,
                                                               ChunkTable tab, float* dZ) {
  const int g = chunk_group(tab, blockIdx.x);
  const int t0 = (blockIdx.x - tab.seg[g]) * tab.chunk;
  const int nt = min(tab.chunk, tab.len[g] - t0);   // tokens of the chunk
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
  // the next token's scores are requested before this one's are used (S may be dZ: rows of
  // other tokens)
  const size_t first = (size_t)(tab.off[g] + t0) * E;
  float next[Q][4];
  if (grp < nt) load_row<Q>(S + first + (size_t)grp * E, E, r, 0.f, next);
  for (int t = grp; t < nt; t += 16) {
    const size_t at = first + (size_t)t * E;
    float v[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[q][c] = next[q][c];
    if (t + 16 < nt) load_row<Q>(S + at + (size_t)16 * E, E, r, 0.f, next);
    double dot = 0.0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) dot += (double)v[q][c] * b[q][c];
    dot = row16_sum_f64(dot);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[q][c] = (float)((double)v[q][c] * (b[q][c] - dot));
    store_row<Q>(dZ + at, E, r, v);
  }
}

// The router's dZ of token-choice training.  Over the chosen experts C_i of a token the
// gates are a softmax of their logits, so with u_ij = g_ij dL/dg_ij (what the dA product's
// partials of a packed row sum to; 0 for a dropped pair)
//   dZ_ij = (u_ij - g_ij sum_m u_im) / tau,
// nothing elsewhere and nothing at all for one choice, whose gate is 1; plus the balance
// loss's term with dloss.  Latency bounds it: a token's loads depend on each other (gate,
// slot, partials), so a quarter row's four slots and then all their partials are requested
// together, whether chosen or not (row 0 stands in for what is not): 16384 tokens, top 8 of
// 64, 31.8 -> 10.6 us.  NP: partials of a row
// read as 16-byte vectors (4, 8, 16; 0: any count, one by one).
template <int Q, int NP, typename T>
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
  const int nt = min(tab.chunk, tab.len[g] - t0);   // tokens of the chunk
  const int r = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const bool gates = k > 1 && max_rows > 0;
  for (int t = grp; t < nt; t += 16) {
    const int i = tab.off[g] + t0 + t;
    float v[Q][4], gt[Q][4], u[Q][4];
    load_row<Q>(G + (size_t)i * E, E, r, 0.f, gt);
    if (dloss) load_row<Q>(S + (size_t)i * E, E, r, 0.f, v);
    float all = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      int row[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = 64 * q + 4 * r + c;
        const int at = slotT[(size_t)(gates && j < E ? j : 0) * N + i];
        row[c] = gates && gt[q][c] != 0.f && at < max_rows ? at : -1;
      }
      if constexpr (NP > 0) {
        float4 x[4][NP / 4];
        if (gates) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int w = 0; w < NP / 4; ++w)
              x[c][w] = *reinterpret_cast<const float4*>(
                  dsp + (size_t)(row[c] >= 0 ? row[c] : 0) * NP + 4 * w);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u[q][c] = 0.f;
          if (row[c] >= 0) {
#pragma unroll
            for (int w = 0; w < NP / 4; ++w) {
              u[q][c] += x[c][w].x; u[q][c] += x[c][w].y;
              u[q][c] += x[c][w].z; u[q][c] += x[c][w].w;
            }
          }
          all += u[q][c];
        }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u[q][c] = 0.f;
          if (row[c] >= 0)
            for (int n = 0; n < nparts; ++n) u[q][c] += dsp[(size_t)row[c] * nparts + n];
          all += u[q][c];
        }
      }
    }
    all = row16_sum(all);
    double b[Q][4], dot = 0.0;
    if (dloss) {
      const double L = tab.len[g], coef = (double)dloss[g] * E / (L * L * k);
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int j = 64 * q + 4 * r + c;
          b[q][c] = j < E ? coef * counts[(size_t)g * E + j] : 0.0;
          dot += (double)v[q][c] * b[q][c];
        }
      dot = row16_sum_f64(dot);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      float z[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        z[c] = gates ? u[q][c] - gt[q][c] * all : 0.f;
        if (dloss) z[c] = (float)((double)z[c] + (double)v[q][c] * (b[q][c] - dot));
        z[c] *= inv_tau;
      }
      // (rounded to bf16 as the operand of the router's two products)
      T* out = dZ + (size_t)i * EP + 64 * q + 4 * r;   // EP = 64 Q
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float4*>(out) = make_float4(z[0], z[1], z[2], z[3]);
      else
        *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]));
    }
  }
}

// The quarters of 64 experts that a row takes, as a constant: f(integral_constant).
template <typename F>
void by_width(int E, F f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 192) f(std::integral_constant<int, 3>{});
  else f(std::integral_constant<int, 4>{});
}

template <int Q, int NP>
void run_tc_dz(int dtype, const float* S, const float* G, const int32_t* slotT, const float* dsp,
               int nparts, const int32_t* counts, const float* dloss, void* dZ, int N, int E,
               int EP, int k, int max_rows, float inv_tau, const ChunkTable& tab, hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (dtype == DT_F32)
    tc_dz_kernel<Q, NP, float><<<grid, 256, 0, st>>>(S, G, slotT, dsp, nparts, counts, dloss,
                                                     (float*)dZ, N, E, EP, k, max_rows, inv_tau,
                                                     tab);
  else
    tc_dz_kernel<Q, NP, bf16_t><<<grid, 256, 0, st>>>(S, G, slotT, dsp, nparts, counts, dloss,
                                                      (bf16_t*)dZ, N, E, EP, k, max_rows, inv_tau,
                                                      tab);
}

}  // namespace

// Sums: 64 tokens a chunk, or so many that a batch has at most 256 chunks and its groups:
// 65536 for the most tokens, below 2^24.
int balance_chunk(int N) { return (N + 256 * 64 - 1) / (256 * 64) * 64; }

// Gradients: 16 tokens (one each) while the workgroups are at most 1024, else 64.
int balance_backward_chunk(int N) { return N <= 16384 ? 16 : 64; }

hipError_t launch_balance_partial(const float* S, int E, int k, const ChunkTable& tab, bool whole,
                                  const BalanceSums& sums, float* loss, int32_t* counts,
                                  hipStream_t st) {
  const int grid = whole ? tab.n : tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
  by_width(E, [&](auto w) {
    constexpr int Q = decltype(w)::value;
    if (whole)
      balance_partial_kernel<Q, true, false><<<grid, BL_THREADS<Q>, 0, st>>>(
          S, E, k, tab, nullptr, nullptr, nullptr, loss, counts, nullptr, nullptr, 0);
    else
      balance_partial_kernel<Q, false, false><<<grid, BL_THREADS<Q>, 0, st>>>(
          S, E, k, tab, sums.psum, sums.pcnt, sums.done, nullptr, nullptr, nullptr, nullptr, 0);
  });
  return hipGetLastError();
}

hipError_t launch_tc_choose(const float* S, int N, int E, int k, const ChunkTable& tab,
                            const BalanceSums& sums, float* G, int32_t* flagT, hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
  if (tab.chunk != TC_CHOOSE_CHUNK) return hipErrorInvalidValue;
  by_width(E, [&](auto w) {
    constexpr int Q = decltype(w)::value;
    balance_partial_kernel<Q, false, true><<<grid, BL_THREADS<Q>, 0, st>>>(
        S, E, k, tab, sums.psum, sums.pcnt, sums.done, nullptr, nullptr, G, flagT, N);
  });
  return hipGetLastError();
}

hipError_t launch_balance_finish(const BalanceSums& sums, int E, int k, const ChunkTable& tab,
                                 float* loss, int32_t* counts, int32_t* counts2, int32_t* kept,
                                 hipStream_t st) {
  if (tab.n == 0) return hipSuccess;
  by_width(E, [&](auto w) {
    constexpr int Q = decltype(w)::value;
    balance_finish_kernel<Q><<<tab.n * Q, 1024, 0, st>>>(sums.psum, sums.pcnt, E, k, tab, sums.part,
                                                         sums.done, loss, counts, counts2, kept);
  });
  return hipGetLastError();
}

hipError_t launch_balance_backward(const float* S, const int32_t* counts, const float* dloss,
                                   int E, int k, float inv_tau, const ChunkTable& tab, float* dZ,
                                   hipStream_t st) {
  const int grid = tab.seg[tab.n];
  if (grid == 0) return hipSuccess;
  by_width(E, [&](auto w) {
    balance_backward_kernel<decltype(w)::value><<<grid, 256, 0, st>>>(S, counts, dloss, E, k,
                                                                      inv_tau, tab, dZ);
  });
  return hipGetLastError();
}

hipError_t launch_tc_router_dz(int dtype, const float* S, const float* G, const int32_t* slotT,
                               const float* dsp, int nparts, const int32_t* counts,
                               const float* dloss, void* dZ, int N, int E, int EP, int k,
                               int max_rows, float inv_tau, const ChunkTable& tab,
                               hipStream_t st) {
  if (tab.seg[tab.n] == 0) return hipSuccess;
  by_width(E, [&](auto w) {
    constexpr int Q = decltype(w)::value;
    auto run = [&](auto np) {
      run_tc_dz<Q, decltype(np)::value>(dtype, S, G, slotT, dsp, nparts, counts, dloss, dZ, N, E,
                                        EP, k, max_rows, inv_tau, tab, st);
    };
    switch (nparts) {
      case 4: run(std::integral_constant<int, 4>{}); break;
      case 8: run(std::integral_constant<int, 8>{}); break;
      case 16: run(std::integral_constant<int, 16>{}); break;
      default: run(std::integral_constant<int, 0>{});
    }
  });
  return hipGetLastError();
}

}  // namespace ec
