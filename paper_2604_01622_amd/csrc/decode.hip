// The token-choice layer for a few tokens (a serving step): N <= 64 tokens, every one kept.
//   z = x Wg^T;  C = the top_k experts of z (equal logits: the lower index);
//   g = softmax over C of z / tau;
//   y = residual + sum over j in C of W2_j (g_j silu(W1_j x) * (W3_j x)) + the shared experts.
//
// The weights of the chosen experts bound it: each is read once, for at most 64 tokens, far
// below the operations that the matrix cores need to be the limit.  So weight rows are the MFMAs' A
// operand, streamed from memory straight into registers, and the tokens are its 16 columns.
// Four launches: logits, choice, W1/W3, W2.
//
// Weights come in the storage type or in eight bits with scales (mx.h), which turn into bf16
// exactly (four leading bits) on their way to the matrix cores; the tokens and activations
// that they meet are bf16, so eight bits cost no accuracy beyond the weights' own.
#include <hip/hip_runtime.h>

#include "ec_kernels.h"
#include "mx.h"

namespace ec {

namespace {

// What a lane holds of 64 consecutive k of its row (weight row or token lane & 15): the 16
// from 16 q, q = lane >> 4.  The MFMAs take them in an order of k that both operands share.
struct BOperand {
  u32x4 r[2];
  __device__ __forceinline__ void load(const bf16_t* p) {
    r[0] = *reinterpret_cast<const u32x4*>(p);
    r[1] = *reinterpret_cast<const u32x4*>(p + 8);
  }
};

struct WBf16 {
  typedef bf16_t T;       // tokens and activations
  typedef bf16_t Code;
  typedef BOperand B;
  static constexpr int UNITS = 8;   // units of 64 k in flight, both matrices together
  u32x4 r[2];
  __device__ __forceinline__ void load(const Code* p, const uint8_t*) {
    r[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    r[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 8));
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r[j]),
                                                    __builtin_bit_cast(bf16x8, b.r[j]), acc, 0, 0, 0);
  }
};

// Eight consecutive codes as bf16, times 2^(byte - 127).
__device__ __forceinline__ bf16x8 mx_widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte == MX_NAN ? 0x7fc00000u : byte << 23);
}

struct WMx {
  typedef bf16_t T;
  typedef uint8_t Code;
  typedef BOperand B;
  static constexpr int UNITS = 16;
  u32x4 r;
  uint32_t s;
  __device__ __forceinline__ void load(const Code* p, const uint8_t* scale) {
    r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    s = *scale;
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
    const float f = mx_scale(s);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx_widen8(r[2 * j], r[2 * j + 1], f),
                                                    __builtin_bit_cast(bf16x8, b.r[j]), acc, 0, 0, 0);
  }
};

struct WF32 {
  typedef float T;
  typedef float Code;
  struct B {
    f32x4 r[4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
      for (int m = 0; m < 4; ++m) r[m] = *reinterpret_cast<const f32x4*>(p + 4 * m);
    }
  };
  static constexpr int UNITS = 4;
  f32x4 r[4];
  __device__ __forceinline__ void load(const Code* p, const uint8_t*) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
      r[m] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4 * m));
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(r[m][j], b.r[m][j], acc, 0, 0, 0);
  }
};

// ---- logits --------------------------------------------------------------------------

constexpr int LG_WAVES = 16;

// Z [N, E] = X Wg^T: a workgroup takes 16 experts, its waves every 16th 64 of k; the sums meet
// in LDS in a fixed order.  Codes, scales: the tokens in eight bits, whose rows go to Xb as
// bf16 for the expert products (X is then unused).
template <class F, int TT, bool XMX>
__global__ __launch_bounds__(64 * LG_WAVES) void decode_logits_kernel(
    const typename F::T* __restrict__ X, const uint8_t* __restrict__ codes,
    const uint8_t* __restrict__ scales, const typename F::T* __restrict__ Wg,
    float* __restrict__ Z, bf16_t* __restrict__ Xb, int N, int d, int E) {
  __shared__ f32x4 red[LG_WAVES][TT][64];
  const int lane = wave_lane(), wave = threadIdx.x >> 6, q = lane >> 4;
  const int e0 = blockIdx.x * 16 + (lane & 15);
  const typename F::T* wp = Wg + (size_t)(e0 < E ? e0 : E - 1) * d + q * 16;
  int tok[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int i = t * 16 + (lane & 15);
    tok[t] = i < N ? i : N - 1;
  }
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int u = wave; u < d / 64; u += LG_WAVES) {
    F a;
    a.load(wp + u * 64, nullptr);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      typename F::B b;
      if constexpr (XMX) {
        const size_t at = (size_t)tok[t] * d + u * 64 + q * 16;
        const u32x4 c = *reinterpret_cast<const u32x4*>(codes + at);
        const float f = mx_scale(scales[at / MX_BLOCK]);
        b.r[0] = __builtin_bit_cast(u32x4, mx_widen8(c[0], c[1], f));
        b.r[1] = __builtin_bit_cast(u32x4, mx_widen8(c[2], c[3], f));
        if (blockIdx.x == 0 && t * 16 + (lane & 15) < N) {
          *reinterpret_cast<u32x4*>(Xb + at) = b.r[0];
          *reinterpret_cast<u32x4*>(Xb + at + 8) = b.r[1];
        }
      } else {
        b.load(X + (size_t)tok[t] * d + u * 64 + q * 16);
      }
      a.mma(acc[t], b);
    }
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) red[wave][t][lane] = acc[t];
  __syncthreads();
  if (wave < TT) {
    f32x4 s = red[0][wave][lane];
#pragma unroll
    for (int w = 1; w < LG_WAVES; ++w) s += red[w][wave][lane];
    const int i = wave * 16 + (lane & 15);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = blockIdx.x * 16 + q * 4 + r;
      if (i < N && e < E) Z[(size_t)i * E + e] = s[r];
    }
  }
}

// ---- choice --------------------------------------------------------------------------

// Orders logits as integers: numbers above NaN above nothing; -0 equals 0.
__device__ __forceinline__ uint32_t logit_key(float z) {
  return z != z ? 1u : f32_order_key(z + 0.0f);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  if (k == 1u) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// Sixteen lanes per token choose its experts (lane r holds experts r, r + 16, ...); then a wave
// an expert, its lanes the tokens, lists who chose it.
template <int NQ>
__global__ __launch_bounds__(1024) void decode_choose_kernel(const float* __restrict__ Z, int N,
                                                             int E, int k, float inv_tau,
                                                             int32_t* __restrict__ experts,
                                                             float* __restrict__ gates,
                                                             DecodePlan plan, uint32_t* zero,
                                                             int n_zero) {
  __shared__ uint16_t pick[256][DECODE_TOKENS];
  __shared__ int count[256];
  const int tid = threadIdx.x, i = tid >> 4, r = tid & 15;
  for (int c = tid; c < n_zero; c += 1024) zero[c] = 0;
  for (int c = tid; c < E * DECODE_TOKENS / 2; c += 1024) reinterpret_cast<uint32_t*>(pick)[c] = 0;
  if (tid < 256) count[tid] = 0;
  uint32_t key[NQ];
#pragma unroll
  for (int m = 0; m < NQ; ++m) {
    const int j = r + 16 * m;
    key[m] = (i < N && j < E) ? logit_key(Z[(size_t)i * E + j]) : 0u;
  }
  __syncthreads();
  if (i < N) {
    float z0 = 0.f, sum = 0.f;
    for (int c = 0; c < k; ++c) {
      uint32_t bk = 0;
      int bj = 0;
#pragma unroll
      for (int m = 0; m < NQ; ++m)
        if (key[m] > bk) {
          bk = key[m];
          bj = r + 16 * m;
        }
      const auto better = [&](uint32_t ok, uint32_t oj) {
        if (ok > bk || (ok == bk && (int)oj < bj)) {
          bk = ok;
          bj = (int)oj;
        }
      };
      better(dpp_u32<0x128>(bk), dpp_u32<0x128>((uint32_t)bj));
      better(dpp_u32<0x124>(bk), dpp_u32<0x124>((uint32_t)bj));
      better(dpp_u32<0x4E>(bk), dpp_u32<0x4E>((uint32_t)bj));
      better(dpp_u32<0xB1>(bk), dpp_u32<0xB1>((uint32_t)bj));
#pragma unroll
      for (int m = 0; m < NQ; ++m)
        if (bj == r + 16 * m) key[m] = 0;
      const float z = key_logit(bk);
      if (c == 0) z0 = z;
      const float ex = expf((z - z0) * inv_tau);
      sum += ex;
      if (r == (c & 15)) {
        experts[i * k + c] = bj;
        gates[i * k + c] = ex;
        pick[bj][i] = (uint16_t)(c + 1);
      }
    }
    for (int c = r; c < k; c += 16) gates[i * k + c] = gates[i * k + c] / sum;
  }
  __syncthreads();
  const int wave = tid >> 6, lane = tid & 63;
  for (int e = wave; e < E; e += 16) {
    const unsigned long long who = __ballot(pick[e][lane] != 0);
    if (lane == 0) count[e] = __popcll(who);
  }
  __syncthreads();
  unsigned long long used[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) used[m] = __ballot(count[lane + 64 * m] != 0);
  if (tid == 0)
    plan.active[0] = __popcll(used[0]) + __popcll(used[1]) + __popcll(used[2]) + __popcll(used[3]);
  for (int e = wave; e < E; e += 16) {
    const int n = count[e];
    if (n == 0) continue;
    int a = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      if (m * 64 + 64 <= e) a += __popcll(used[m]);
      else if (m * 64 <= e) a += __popcll(used[m] & ((1ull << (e - m * 64)) - 1));
    }
    const uint32_t p = pick[e][lane];
    const unsigned long long who = __ballot(p != 0);
    if (lane == 0) plan.list[a] = (uint32_t)e | (uint32_t)n << 16;
    plan.pick[a * DECODE_TOKENS + lane] = (uint16_t)p;
    if (p)
      plan.rows[a * DECODE_TOKENS + __popcll(who & ((1ull << lane) - 1))] =
          (uint32_t)lane << 16 | (p - 1);
  }
}

// ---- W1 and W3 -----------------------------------------------------------------------

constexpr int W13_WAVES = 4;

// A workgroup takes 16 hidden units of an expert, its waves every fourth 64 of k; the expert's
// tokens are the columns.  A [token k + pick, h] = gate silu(W1 x) (W3 x); the workgroups past
// those of the chosen experts take the shared experts' hidden units, for every token.
template <class F, int TT>
__global__ __launch_bounds__(64 * W13_WAVES) void decode_w13_kernel(
    const typename F::T* __restrict__ X, DecodeWeights w, const float* __restrict__ gates,
    DecodePlan plan, typename F::T* __restrict__ A, typename F::T* __restrict__ As, int N, int d,
    int h, int hs, int k, int routed) {
  typedef typename F::T T;
  typedef typename F::Code Code;
  __shared__ f32x4 red[W13_WAVES][2 * TT][64];
  const int lane = wave_lane(), wave = threadIdx.x >> 6, q = lane >> 4, col = lane & 15;
  int bid = blockIdx.x;
  const bool shared = bid >= routed;
  const Code *w1, *w3;
  const uint8_t *s1 = nullptr, *s3 = nullptr;
  T* out;
  int n, tile, width, slot = 0;
  size_t row;
  if (shared) {
    tile = bid - routed;
    n = N;
    width = hs;
    row = (size_t)tile * 16 + col;
    w1 = (const Code*)w.Ws1;
    w3 = (const Code*)w.Ws3;
    s1 = w.Ss1;
    s3 = w.Ss3;
    out = As;
  } else {
    slot = bid / (h / 16);
    tile = bid % (h / 16);
    if (slot >= plan.active[0]) return;
    const uint32_t e = plan.list[slot];
    n = (int)(e >> 16);
    width = h;
    row = (size_t)(e & 0xffffu) * h + tile * 16 + col;
    w1 = (const Code*)w.W1;
    w3 = (const Code*)w.W3;
    s1 = w.S1;
    s3 = w.S3;
    out = A;
  }
  w1 += row * d + q * 16;
  w3 += row * d + q * 16;
  if (F::UNITS == 16) {
    s1 += row * (d / MX_BLOCK) + (q >> 1);
    s3 += row * (d / MX_BLOCK) + (q >> 1);
  }
  // columns past the expert's tokens repeat its last one; nothing of them is stored
  const T* xp[TT];
  int at[TT];      // their rows of A
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    int c = t * 16 + col;
    c = c < n ? c : n - 1;
    int token = c;
    at[t] = c;
    if (!shared) {
      const uint32_t p = plan.rows[slot * DECODE_TOKENS + c];
      token = (int)(p >> 16);
      at[t] = token * k + (int)(p & 0xffffu);
    }
    xp[t] = X + (size_t)token * d + q * 16;
  }
  f32x4 acc[2][TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto step = [&](auto units, int u) {
    constexpr int U = decltype(units)::value;
    F a1[U], a3[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int o = (u + i * W13_WAVES) * 64;
      a1[i].load(w1 + o, s1 + o / MX_BLOCK);
      a3[i].load(w3 + o, s3 + o / MX_BLOCK);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      if (t * 16 >= n) break;
      typename F::B b[U];
#pragma unroll
      for (int i = 0; i < U; ++i) b[i].load(xp[t] + (u + i * W13_WAVES) * 64);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        a1[i].mma(acc[0][t], b[i]);
        a3[i].mma(acc[1][t], b[i]);
      }
    }
  };
  constexpr int U = F::UNITS / 2;
  int u = wave;
  for (; u + (U - 1) * W13_WAVES < d / 64; u += U * W13_WAVES)
    step(std::integral_constant<int, U>{}, u);
  for (; u < d / 64; u += W13_WAVES) step(std::integral_constant<int, 1>{}, u);
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    red[wave][2 * t][lane] = acc[0][t];
    red[wave][2 * t + 1][lane] = acc[1][t];
  }
  __syncthreads();
  static_assert(TT <= W13_WAVES, "");
  if (wave >= TT || wave * 16 + col >= n) return;
  f32x4 a = red[0][2 * wave][lane], b = red[0][2 * wave + 1][lane];
#pragma unroll
  for (int i = 1; i < W13_WAVES; ++i) {
    a += red[i][2 * wave][lane];
    b += red[i][2 * wave + 1][lane];
  }
  int r = at[0];
#pragma unroll
  for (int t = 1; t < TT; ++t)
    if (wave == t) r = at[t];
  const float gate = shared ? 1.0f : gates[r];
  T* o = out + (size_t)r * width + tile * 16 + q * 4;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = gate * (a[i] / (1.0f + expf(-a[i]))) * b[i];
  store4<T>(o, v);
}

// ---- W2 ------------------------------------------------------------------------------

constexpr int W2_WAVES = 8;

// A workgroup takes 16 columns of Y (rows of W2) over all chosen experts and the shared ones,
// its waves every eighth 64 of the concatenated hidden units.  The columns of its products are
// the tokens, those that did not choose the expert reading a row of zeros, so the experts' sum
// is that of the accumulators.
template <class F, int TT>
__global__ __launch_bounds__(64 * W2_WAVES) void decode_w2_kernel(
    const typename F::T* __restrict__ A, const typename F::T* __restrict__ As, DecodeWeights w,
    DecodePlan plan, const typename F::T* __restrict__ zero, const typename F::T* __restrict__ R,
    typename F::T* __restrict__ Y, int N, int d, int h, int hs, int k) {
  typedef typename F::T T;
  typedef typename F::Code Code;
  __shared__ union {
    uint16_t pick[256 * DECODE_TOKENS];
    f32x4 red[W2_WAVES][TT][64];
  } lds;
  const int lane = wave_lane(), q = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int active = plan.active[0];
  for (int c = threadIdx.x; c < active * DECODE_TOKENS / 2; c += 64 * W2_WAVES)
    reinterpret_cast<uint32_t*>(lds.pick)[c] = reinterpret_cast<const uint32_t*>(plan.pick)[c];
  __syncthreads();
  const size_t row = (size_t)blockIdx.x * 16 + col;
  const int hu = h / 64, units = active * hu + hs / 64;
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto step = [&](auto count, int u) {
    constexpr int U = decltype(count)::value;
    F a[U];
    int slot[U], o[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = u + i * W2_WAVES;
      slot[i] = at / hu;
      if (slot[i] > active) slot[i] = active;      // the shared experts' units
      o[i] = (at - slot[i] * hu) * 64;
      const bool sh = slot[i] == active;
      const int width = sh ? hs : h;
      const size_t wr = (sh ? row : (size_t)(plan.list[slot[i]] & 0xffffu) * d + row);
      const size_t off = wr * width + o[i] + q * 16;
      a[i].load((const Code*)(sh ? w.Ws2 : w.W2) + off, (sh ? w.Ss2 : w.S2) + off / MX_BLOCK);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int token = t * 16 + col;
      typename F::B b[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const T* p;
        if (slot[i] == active) {
          p = token < N ? As + (size_t)token * hs : zero;
        } else {
          const int c = lds.pick[slot[i] * DECODE_TOKENS + token];
          p = c ? A + (size_t)(token * k + c - 1) * h : zero;
        }
        b[i].load(p + o[i] + q * 16);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) a[i].mma(acc[t], b[i]);
    }
  };
  constexpr int U = F::UNITS;
  int u = wave;
  for (; u + (U - 1) * W2_WAVES < units; u += U * W2_WAVES)
    step(std::integral_constant<int, U>{}, u);
  for (; u < units; u += W2_WAVES) step(std::integral_constant<int, 1>{}, u);
  __syncthreads();
#pragma unroll
  for (int t = 0; t < TT; ++t) lds.red[wave][t][lane] = acc[t];
  __syncthreads();
  const int token = wave * 16 + col;
  if (wave >= TT || token >= N) return;
  f32x4 s = lds.red[0][wave][lane];
#pragma unroll
  for (int i = 1; i < W2_WAVES; ++i) s += lds.red[i][wave][lane];
  const size_t at = (size_t)token * d + (size_t)blockIdx.x * 16 + q * 4;
  float v[4] = {s[0], s[1], s[2], s[3]};
  if (R) {
    float x[4];
    load4<T>(R + at, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += x[i];
  }
  store4<T>(Y + at, v);
}

template <class F, int TT>
hipError_t run_decode(const DecodeCall& c, hipStream_t st) {
  typedef typename F::T T;
  typedef std::conditional_t<sizeof(T) == 4, WF32, WBf16> G;   // the router's weights
  const dim3 lg((unsigned)((c.E + 15) / 16));
  if (c.Xs) {
    if constexpr (sizeof(T) == 2)
      decode_logits_kernel<G, TT, true><<<lg, 64 * LG_WAVES, 0, st>>>(
          nullptr, (const uint8_t*)c.X, c.Xs, (const T*)c.Wg, c.Z, (bf16_t*)c.Xb, c.N, c.d, c.E);
    else
      return hipErrorInvalidValue;
  } else {
    decode_logits_kernel<G, TT, false><<<lg, 64 * LG_WAVES, 0, st>>>(
        (const T*)c.X, nullptr, nullptr, (const T*)c.Wg, c.Z, nullptr, c.N, c.d, c.E);
  }
  const int n_zero = (int)((c.h > c.hs ? c.h : c.hs) * sizeof(T) / 4);
  if (c.E <= 64)
    decode_choose_kernel<4><<<1, 1024, 0, st>>>(c.Z, c.N, c.E, c.k, c.inv_tau, c.experts, c.gates,
                                                c.plan, (uint32_t*)c.zero, n_zero);
  else
    decode_choose_kernel<16><<<1, 1024, 0, st>>>(c.Z, c.N, c.E, c.k, c.inv_tau, c.experts, c.gates,
                                                 c.plan, (uint32_t*)c.zero, n_zero);
  const T* X = (const T*)(c.Xs ? c.Xb : c.X);
  const int most = c.N * c.k < c.E ? c.N * c.k : c.E;    // chosen experts at most
  const int routed = most * (c.h / 16);
  decode_w13_kernel<F, TT><<<dim3((unsigned)(routed + c.hs / 16)), 64 * W13_WAVES, 0, st>>>(
      X, c.w, c.gates, c.plan, (T*)c.A, (T*)c.As, c.N, c.d, c.h, c.hs, c.k, routed);
  decode_w2_kernel<F, TT><<<dim3((unsigned)(c.d / 16)), 64 * W2_WAVES, 0, st>>>(
      (const T*)c.A, (const T*)c.As, c.w, c.plan, (const T*)c.zero, (const T*)c.R, (T*)c.Y, c.N,
      c.d, c.h, c.hs, c.k);
  return hipGetLastError();
}

template <class F>
hipError_t run_decode(const DecodeCall& c, hipStream_t st) {
  if (c.N <= 16) return run_decode<F, 1>(c, st);
  if (c.N <= 32) return run_decode<F, 2>(c, st);
  return run_decode<F, 4>(c, st);
}

}  // namespace

hipError_t launch_decode(const DecodeCall& c, hipStream_t st) {
  if (c.N == 0) return hipSuccess;
  if (c.dtype == DT_F32) return run_decode<WF32>(c, st);
  return c.w.S1 ? run_decode<WMx>(c, st) : run_decode<WBf16>(c, st);
}

}  // namespace ec
