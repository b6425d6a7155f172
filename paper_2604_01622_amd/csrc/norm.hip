// Root-mean-square norm of rows, the residual added first, and its backward pass:
//   h = round(x + residual) (x without one),  r = (mean(h^2) + eps)^-1/2,  y = h r w;
//   dx = r (g - h r^2 mean(g h)) + dh,  g = w dy,  dw = sum over the rows of dy h r.
// The norm is that of the sum as it is stored, so that the backward pass needs h alone.
// Sums in fp32; y is rounded once, to the storage type or to eight bits (mx.h).
//
// Memory bounds both: every row moves once and is held in registers between its sum and its
// use.  A row belongs to TPR lanes, each of which takes V pieces of 16 bytes.  Where d leaves rows
// unaligned (ODD) the pieces are too, and a row's last one ends with the row: what it shares
// with the piece before it is that one's (5000 x 4097 bf16: 37 us, backward 55; an element a lane 116
// and 316).  Forward, a group of lanes takes one row and leaves: many short workgroups keep more on
// its way than loops over rows with the next one requested ahead (16384 x 2048 bf16 with a
// residual: 44.3 us, 6.1 TB/s, against 51.2; eight bits out 40, 5.9 TB/s).  Backward, where a
// workgroup keeps its share of dw, the loop it needs requests ahead (43 us and 5 for the sum of the
// shares, 5.6 TB/s; a row in one wave, without: 64 and 11).  One row takes 2.0 us, the launch.  Of
// narrow rows most lanes of a wave have nothing to do (40000 x 64 bf16 13.7 us, 1.5 TB/s; x 256
// 19.0, 4.3; backward 15.4 + 3.9 and 18.6 + 4.0).
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
// wave of the workgroup, taken in turn, so that one barrier a row is enough.
template <int TPR, int NS>
__device__ __forceinline__ void row_sums(float (&s)[NS], float* red, int turn) {
#pragma unroll
  for (int n = 0; n < NS; ++n) s[n] = wave_sum(s[n]);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    const int w = threadIdx.x >> 6;
    float* r = red + turn * (int)(blockDim.x >> 6) * NS;
    if (wave_lane() == 0)
#pragma unroll
      for (int n = 0; n < NS; ++n) r[w * NS + n] = s[n];
    lds_barrier();
    r += w / NW * NW * NS;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) s[n] += r[i * NS + n];
    }
  }
}

// Where a lane's piece of a row stands, and how many of its first elements are not its own.
struct Place {
  int at, skip;
};
template <int VEC, bool ODD>
__device__ __forceinline__ Place place(int c, int d) {
  if (c >= d) return {0, VEC};
  if (!ODD) return {c, 0};
  const int at = min(c, d - VEC);
  return {at, c - at};
}

// A lane's pieces of a row of p.  live false: one place for all lanes instead, not used: a
// request in every turn lets the waits count.
template <typename T, int VEC, int V, bool ODD>
__device__ __forceinline__ void load_row(Piece<T, VEC, ODD> (&to)[V], const T* p, long row,
                                         const Place (&my)[V], int d, bool live) {
  const T* r = p + (live ? row * d : 0);
#pragma unroll
  for (int v = 0; v < V; ++v) to[v].load(r + (live ? my[v].at : 0));
}

// A piece's own elements into row r.
template <typename T, int VEC, bool ODD>
__device__ __forceinline__ void store_own(T* r, const Place& my, const float* v) {
  if (my.skip == 0) {
    store_vec<T, VEC, ODD>(r + my.at, v);
  } else if (ODD) {
#pragma unroll
    for (int e = 1; e < VEC; ++e)
      if (e >= my.skip) Elem<T>::store1(r + my.at + e, v[e]);
  }
}

// Rows that a lane holds at a time, in registers.
template <int VEC, int V>
constexpr int row_buffers() { return VEC * V > 8 ? 1 : 2; }

// Of a forward workgroup: four rows of a wave each, or one row, whose waves meet in barriers.
template <int TPR>
constexpr int norm_threads() { return TPR == 64 ? 256 : TPR; }

// One row a group of TPR lanes and step; MX: eight bits out.
template <typename T, int VEC, int V, int TPR, bool ODD, bool MX, bool RES>
__global__ __launch_bounds__(norm_threads<TPR>()) void rms_norm_kernel(
    const T* X, const T* R, const T* __restrict__ w, T* H, T* __restrict__ Y,
    uint8_t* __restrict__ Q, uint8_t* __restrict__ scale, long rows, int d, float eps) {
  constexpr int RB = norm_threads<TPR>() / TPR;
  __shared__ float red[2 * norm_threads<TPR>() / 64];
  Place my[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
    my[v] = place<VEC, ODD>((v * TPR + (int)threadIdx.x % TPR) * VEC, d);
  const float inv_d = 1.0f / (float)d;
  const long stride = (long)gridDim.x * RB;
  long row = (long)blockIdx.x * RB + threadIdx.x / TPR;
  if (row >= rows) return;          // a wave without barriers, or the whole workgroup
  int turn = 0;
  do {
    Piece<T, VEC, ODD> x[V], r[RES ? V : 1], pw[V];
    load_row<T, VEC, V>(x, X, row, my, d, true);
    if constexpr (RES) load_row<T, VEC, V>(r, R, row, my, d, true);
#pragma unroll          // the one operand of all workgroups (8192 x 8192 bf16 90 -> 85 us)
    for (int v = 0; v < V; ++v) pw[v].load_shared(w + my[v].at);
    __builtin_amdgcn_sched_barrier(0);      // all on their way before the first is used
    const long at = row * d;
    float h[V][VEC], s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v].get(h[v]);
      if constexpr (RES) {
        float q[VEC];
        r[v].get(q);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[v][e] = round_to<T>(h[v][e] + q[e]);
        store_own<T, VEC, ODD>(H + at, my[v], h[v]);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[0] = e >= my[v].skip ? fmaf(h[v][e], h[v][e], s[0]) : s[0];
    }
    row_sums<TPR, 1>(s, red, turn);
    const float rs = 1.0f / sqrtf(fmaf(s[0], inv_d, eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (my[v].skip == VEC) break;
      float y[VEC], q[VEC];
      pw[v].get(q);
#pragma unroll
      for (int e = 0; e < VEC; ++e) y[e] = h[v][e] * rs * q[e];
      if constexpr (MX) {   // d is a multiple of 32: a block's lanes are all here
        const int c = my[v].at;
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = max(top, magnitude(y[e]));
        const uint32_t byte = mx_byte(mx_block_max<VEC>(top));
        mx_store<VEC>(Q + at + c, y, mx_inverse(byte));
        if (c % MX_BLOCK == 0) scale[(at + c) / MX_BLOCK] = (uint8_t)byte;
      } else {
        store_own<T, VEC, ODD>(Y + at, my[v], y);
      }
    }
    row += stride;
    turn ^= 1;
  } while (row < rows);
}

constexpr int NB_THREADS = 1024;     // of a backward workgroup: 1024 / TPR rows at a time

// A workgroup takes every gridDim.x-th set of rows and keeps its share of dw in registers; of more
// than eight elements a lane (d above 8192) in LDS, with the weight and dH loaded again for a piece
// at a time: the registers would spill (2048 x 16384 fp32 105 us, 5.1 TB/s, instead of 161; bf16
// 62 and 76).
// part [gridDim.x, d] (dw itself where one workgroup takes all rows).
template <typename T, int VEC, int V, int TPR, bool ODD, bool DH>
__global__ __launch_bounds__(NB_THREADS) void rms_norm_backward_kernel(
    const T* H, const T* __restrict__ w, const T* dY, const T* dH, T* dX,
    float* __restrict__ part, long rows, int d, float eps) {
  constexpr int RB = NB_THREADS / TPR, BUF = row_buffers<VEC, V>();
  __shared__ float red[4 * NB_THREADS / 64];
  Place my[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
    my[v] = place<VEC, ODD>((v * TPR + (int)threadIdx.x % TPR) * VEC, d);
  const float inv_d = 1.0f / (float)d;
  const long stride = (long)gridDim.x * RB;
  long first = (long)blockIdx.x * RB;               // of the workgroup's rows
  const int mine = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  // long rows: in LDS, a lane's own
  __shared__ float long_dw[BUF == 1 ? V * TPR * VEC : 1];
  float dw[V][VEC];
  Piece<T, VEC, ODD> ph[BUF][V], pg[BUF][V], pd[BUF][DH ? V : 1], pw[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (BUF == 1) long_dw[(v * TPR + threadIdx.x) * VEC + e] = 0.f;
      else dw[v][e] = 0.f;
    }
  const auto request = [&](int i, long row) __attribute__((always_inline)) {
    const bool live = row < rows;
    load_row<T, VEC, V>(ph[i], H, row, my, d, live);
    load_row<T, VEC, V>(pg[i], dY, row, my, d, live);
    if constexpr (DH && BUF == 2) load_row<T, VEC, V>(pd[i], dH, row, my, d, live);
  };
  const auto step = [&](int turn) __attribute__((always_inline)) {
    const int i = BUF == 2 ? turn : 0;
    const long row = first + mine;
    if (BUF == 2) request(i ^ 1, row + stride);
    else request(0, row);
    __builtin_amdgcn_sched_barrier(0);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (BUF == 1) {
        __builtin_amdgcn_sched_barrier(0);
        pw[v].load_shared(w + my[v].at);
      }
      float h[VEC], g[VEC], q[VEC];
      ph[i][v].get(h);
      pg[i][v].get(g);
      pw[v].get(q);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const bool in = e >= my[v].skip;
        s[0] = in ? fmaf(h[e], h[e], s[0]) : s[0];
        s[1] = in ? fmaf(g[e] * q[e], h[e], s[1]) : s[1];
      }
    }
    row_sums<TPR, 2>(s, red, turn);
    const float r = 1.0f / sqrtf(fmaf(s[0], inv_d, eps));
    // r * r passes fp32's range for a subnormal eps; r 0: the squares passed it, k 0 as Y is, though
    // the other sum may have passed it too
    const float k = r == 0.f ? 0.f : r * (r * (s[1] * inv_d));
    if (row < rows) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (my[v].skip == VEC) break;
        if constexpr (BUF == 1) {
          __builtin_amdgcn_sched_barrier(0);
          pw[v].load_shared(w + my[v].at);
          if constexpr (DH) pd[0][v].load(dH + row * d + my[v].at);
        }
        float h[VEC], g[VEC], q[VEC], x[VEC];
        ph[i][v].get(h);
        pg[i][v].get(g);
        pw[v].get(q);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          float& t = BUF == 1 ? long_dw[(v * TPR + threadIdx.x) * VEC + e] : dw[v][e];
          t = fmaf(g[e], h[e] * r, t);
          x[e] = r * (g[e] * q[e] - h[e] * k);
        }
        if constexpr (DH) {
          pd[i][v].get(q);
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[e] += q[e];
        }
        store_own<T, VEC, ODD>(dX + row * d, my[v], x);
      }
    }
    first += stride;
    return first < rows;
  };
  if (rows > 0) {
    if (BUF == 2) request(0, first + mine);
    if constexpr (BUF == 2) {
      load_row<T, VEC, V>(pw, w, 0, my, d, true);
      while (step(0) && step(1)) {
      }
    } else {
      for (int turn = 0; step(turn); turn ^= 1) {
      }
    }
  }
  float* out = part + (long)blockIdx.x * d;
  if constexpr (RB == 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (BUF == 1)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[v][e] = long_dw[(v * TPR + threadIdx.x) * VEC + e];
      store_own<float, VEC, ODD>(out, my[v], dw[v]);
    }
  } else {
    // the workgroup's rows meet, in order
    constexpr int W = V * TPR * VEC;
    __shared__ float sum[RB * W];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e >= my[v].skip) sum[mine * W + my[v].at + e] = dw[v][e];
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += NB_THREADS) {
      float t = sum[c];
#pragma unroll
      for (int b = 1; b < RB; ++b) t += sum[b * W + c];
      out[c] = t;
    }
  }
}

// dw[c] = sum of part[i, c]: 16 columns a workgroup, its 16 groups of lanes each every 16th row,
// eight on their way.
__global__ __launch_bounds__(256) void rms_norm_dw_kernel(const float* __restrict__ part,
                                                          float* __restrict__ dw, int n, int d) {
  __shared__ float s[16][16];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), g = threadIdx.x >> 4;
  float t = 0.f;
  if (c < d)
    for (int i0 = g; i0 < n; i0 += 16 * 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = part[(long)min(i0 + j * 16, n - 1) * d + c];
#pragma unroll
      for (int j = 0; j < 8; ++j) t += i0 + j * 16 < n ? v[j] : 0.f;
    }
  s[g][threadIdx.x & 15] = t;
  __syncthreads();
  if (g == 0 && c < d) {
    t = s[0][threadIdx.x];
#pragma unroll
    for (int i = 1; i < 16; ++i) t += s[i][threadIdx.x];
    dw[c] = t;
  }
}

constexpr int NORM_GRID = 1 << 20;   // workgroups at most
constexpr int NB_GRID = 256;         // of a backward launch: one a CU (512: 45.7 us instead of 44.2)

// Calls body(VEC, V, TPR, ODD) as types with the smallest group of lanes that holds a row in one
// piece of 16 bytes each (past 1024 lanes more); rows shorter than a piece by elements.  Forward,
// of 513 to 1024 pieces, two a lane: two rows a CU wait for one another less than one would (8192 x
// 8192 bf16 90 us instead of 107, 16384 x 4096 fp32 201 and 218); of more in bf16 four
// (4096 x 8198 56 and 66, 4096 x 12000 64.6 and 64.7; in fp32 113 and 103).
template <typename T, bool BACK, typename F>
hipError_t with_shape(int d, F body) {
  constexpr int W = 16 / sizeof(T);
#define EC_I(n) std::integral_constant<int, n>{}
  if (d < W) return body(EC_I(1), EC_I(1), EC_I(64), std::false_type{});
  const int u = (d + W - 1) / W;
  const auto with = [&](auto odd) {
    if (u <= 64) return body(EC_I(W), EC_I(1), EC_I(64), odd);
    if (u <= 128) return body(EC_I(W), EC_I(1), EC_I(128), odd);
    if (u <= 256) return body(EC_I(W), EC_I(1), EC_I(256), odd);
    if (u <= 512) return body(EC_I(W), EC_I(1), EC_I(512), odd);
    if (u <= 1024 && BACK) return body(EC_I(W), EC_I(1), EC_I(1024), odd);
    if (u <= 1024) return body(EC_I(W), EC_I(2), EC_I(512), odd);
    if constexpr (W == 8 && !BACK) return body(EC_I(W), EC_I(4), EC_I(512), odd);
    if constexpr (W == 4)
      if (u > 2048) return body(EC_I(W), EC_I(4), EC_I(1024), odd);
    return body(EC_I(W), EC_I(2), EC_I(1024), odd);
  };
#undef EC_I
  return d % W == 0 ? with(std::false_type{}) : with(std::true_type{});
}

template <typename T>
hipError_t run_norm(const void* X, const void* R, const void* w, void* H, void* Y, uint8_t* Q,
                    uint8_t* scale, long rows, int d, float eps, hipStream_t st) {
  return with_shape<T, false>(d, [&](auto vec, auto v, auto tpr, auto odd) {
    constexpr bool ODD = decltype(odd)::value;
    constexpr int VEC = decltype(vec)::value, V = decltype(v)::value, TPR = decltype(tpr)::value;
    constexpr int RB = norm_threads<TPR>() / TPR;
    const long blocks = (rows + RB - 1) / RB;
    const dim3 grid((unsigned)(blocks < NORM_GRID ? blocks : NORM_GRID));
    const auto go = [&](auto mx, auto res) {
      rms_norm_kernel<T, VEC, V, TPR, ODD, decltype(mx)::value, decltype(res)::value>
          <<<grid, norm_threads<TPR>(), 0, st>>>((const T*)X, (const T*)R, (const T*)w, (T*)H,
                                                 (T*)Y, Q, scale, rows, d, eps);
    };
    if (Q) {
      if constexpr (VEC > 1 && !ODD) {
        if (R) go(std::true_type{}, std::true_type{});
        else go(std::true_type{}, std::false_type{});
      } else {
        return hipErrorInvalidValue;
      }
    } else {
      if (R) go(std::false_type{}, std::true_type{});
      else go(std::false_type{}, std::false_type{});
    }
    return hipGetLastError();
  });
}

template <typename T>
hipError_t run_norm_backward(const void* H, const void* w, const void* dY, const void* dH, void* dX,
                             float* dw, float* part, int blocks, long rows, int d, float eps,
                             hipStream_t st) {
  hipError_t e = with_shape<T, true>(d, [&](auto vec, auto v, auto tpr, auto odd) {
    constexpr bool ODD = decltype(odd)::value;
    constexpr int VEC = decltype(vec)::value, V = decltype(v)::value, TPR = decltype(tpr)::value;
    const auto go = [&](auto dh) {
      rms_norm_backward_kernel<T, VEC, V, TPR, ODD, decltype(dh)::value>
          <<<dim3((unsigned)blocks), NB_THREADS, 0, st>>>(
              (const T*)H, (const T*)w, (const T*)dY, (const T*)dH, (T*)dX,
              blocks > 1 ? part : dw, rows, d, eps);
    };
    if (dH) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
  });
  if (e != hipSuccess || blocks <= 1) return e;
  rms_norm_dw_kernel<<<dim3((unsigned)((d + 15) / 16)), 256, 0, st>>>(part, dw, blocks, d);
  return hipGetLastError();
}

}  // namespace

int rms_norm_backward_blocks(int dtype, long rows, int d) {
  long per = 1;   // rows of a workgroup's step
  const auto rows_of = [&](auto, auto, auto tpr, auto) {
    per = NB_THREADS / decltype(tpr)::value;
    return hipSuccess;
  };
  const hipError_t e =
      dtype == DT_F32 ? with_shape<float, true>(d, rows_of) : with_shape<bf16_t, true>(d, rows_of);
  const long steps = e == hipSuccess ? (rows + per - 1) / per : 1;
  return (int)(steps < 1 ? 1 : steps < NB_GRID ? steps : NB_GRID);
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
