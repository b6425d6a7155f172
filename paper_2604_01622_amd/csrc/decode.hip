// The token-choice layer for a few tokens (a serving step): N <= 64 tokens, every one kept.
//   z = x Wg^T;  C = the top_k experts of z (equal logits: the lower index);
//   g = softmax over C of z / tau;
//   y = residual + sum over j in C of W2_j (g_j silu(W1_j x) * (W3_j x)) + the shared experts.
//
// The weights of the chosen experts bound it: each is read once, for at most 64 tokens, far
// below the operations that the matrix cores need to be the limit.  So weight rows are the
// MFMAs' A operand, streamed from memory straight into registers, and the tokens that chose
// the expert are its 16 columns.  Launches: logits, (many tokens) choice, W1/W3, W2, sum.
//
// Weights come in the storage type or in eight bits with scales (mx.h), which turn into bf16
// exactly (four leading bits) on their way to the matrix cores; the tokens and activations
// that they meet are bf16, so eight bits cost no accuracy beyond the weights' own.
#include <hip/hip_runtime.h>

#include "ec_kernels.h"
#include "mx.h"

namespace ec {

namespace {

// What a lane holds of a unit, 64 consecutive k of its row (a weight row, or token lane & 15);
// q = lane >> 4 says which.  The MFMAs take the k in any order that both operands share.
//
// Eight codes as bf16, times 2^(byte - 127).
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

__device__ __forceinline__ f32x4 mma_bf16(u32x4 a, u32x4 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}

// bf16: 16 bytes at 16 q of both halves, so that an instruction takes 64 consecutive bytes of
// each of 16 rows.
struct WBf16 {
  typedef bf16_t T;       // tokens and activations
  typedef bf16_t Code;
  static constexpr int BURST = 4;     // units of one matrix that are requested at once
  static constexpr bool MX = false;
  struct B {
    u32x4 r[2];
    __device__ __forceinline__ void load(const bf16_t* row, int q) {
      r[0] = *reinterpret_cast<const u32x4*>(row + q * 8);
      r[1] = *reinterpret_cast<const u32x4*>(row + 32 + q * 8);
    }
  };
  u32x4 r[2];
  __device__ __forceinline__ void load(const Code* row, const uint8_t*, int q) {
    r[0] = *reinterpret_cast<const u32x4*>(row + q * 8);
    r[1] = *reinterpret_cast<const u32x4*>(row + 32 + q * 8);
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
    acc = mma_bf16(r[0], b.r[0], acc);
    acc = mma_bf16(r[1], b.r[1], acc);
  }
};

// Eight bits: the 16 codes at 16 q, which lie in one block.
struct WMx {
  typedef bf16_t T;
  typedef uint8_t Code;
  static constexpr int BURST = 4;
  static constexpr bool MX = true;
  struct B {
    u32x4 r[2];
    __device__ __forceinline__ void load(const bf16_t* row, int q) {
      r[0] = *reinterpret_cast<const u32x4*>(row + q * 16);
      r[1] = *reinterpret_cast<const u32x4*>(row + q * 16 + 8);
    }
  };
  u32x4 r;
  uint32_t s;
  __device__ __forceinline__ void load(const Code* row, const uint8_t* scale, int q) {
    r = *reinterpret_cast<const u32x4*>(row + q * 16);
    s = scale[q >> 1];
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
    const float f = mx_scale(s);
    acc = mma_bf16(__builtin_bit_cast(u32x4, mx_widen8(r[0], r[1], f)), b.r[0], acc);
    acc = mma_bf16(__builtin_bit_cast(u32x4, mx_widen8(r[2], r[3], f)), b.r[1], acc);
  }
};

// fp32: 16 bytes at 16 q of each quarter.
struct WF32 {
  typedef float T;
  typedef float Code;
  static constexpr int BURST = 2;
  static constexpr bool MX = false;
  struct B {
    f32x4 r[4];
    __device__ __forceinline__ void load(const float* row, int q) {
#pragma unroll
      for (int m = 0; m < 4; ++m) r[m] = *reinterpret_cast<const f32x4*>(row + m * 16 + q * 4);
    }
  };
  f32x4 r[4];
  __device__ __forceinline__ void load(const Code* row, const uint8_t*, int q) {
#pragma unroll
    for (int m = 0; m < 4; ++m) r[m] = *reinterpret_cast<const f32x4*>(row + m * 16 + q * 4);
  }
  __device__ __forceinline__ void mma(f32x4& acc, const B& b) const {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(r[m][j], b.r[m][j], acc, 0, 0, 0);
  }
};

// ---- choice --------------------------------------------------------------------------

// Orders logits as integers: numbers above NaN above nothing; -0 equals 0.
__device__ __forceinline__ uint32_t logit_key(float z) {
  return z != z ? 1u : f32_order_key(z + 0.0f);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  if (k == 1u) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// Sixteen lanes choose a token's experts: lane r holds the logits of r, r + 16, ... in z.
// put(c, expert, e^((z - z_max) / tau)) is called by lane c % 16; returns the sum of the latter.
template <int NQ, typename Put>
__device__ __forceinline__ float choose(const float (&z)[NQ], int E, int k, float inv_tau, int r,
                                        Put put) {
  uint32_t key[NQ];
#pragma unroll
  for (int m = 0; m < NQ; ++m) key[m] = r + 16 * m < E ? logit_key(z[m]) : 0u;
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
    const float zc = key_logit(bk);
    if (c == 0) z0 = zc;
    const float ex = expf((zc - z0) * inv_tau);
    sum += ex;
    if (r == (c & 15)) put(c, bj, ex);
  }
  return sum;
}

// Logits r, r + 16, ... of a token: the sums of the splits' shares, in order.
template <int NQ>
__device__ __forceinline__ void load_logits(float (&z)[NQ], const float* __restrict__ Z, int i, int r,
                                            int N, int E, int splits) {
#pragma unroll
  for (int m = 0; m < NQ; ++m) z[m] = 0.f;
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int m = 0; m < NQ; ++m)
      if (r + 16 * m < E) z[m] += Z[((size_t)s * N + i) * E + r + 16 * m];
}

constexpr int LG_WAVES = 8;
constexpr int LG_SPLITS = 8;     // splits of k at most

// Z [splits, N, E]: shares of X Wg^T.  A workgroup takes 16 experts and the units of split
// blockIdx.y, its waves every eighth; they meet in LDS in a fixed order.  XMX: the tokens come
// in eight bits; their rows go to Xb as bf16 for the expert products.
template <class F, int TT, bool XMX>
__global__ __launch_bounds__(64 * LG_WAVES) void decode_logits_kernel(
    const typename F::T* __restrict__ X, const uint8_t* __restrict__ codes,
    const uint8_t* __restrict__ scales, const typename F::T* __restrict__ Wg,
    float* __restrict__ Z, bf16_t* __restrict__ Xb, int N, int d, int E) {
  __shared__ f32x4 red[LG_WAVES][TT][64];
  const int lane = wave_lane(), wave = threadIdx.x >> 6, q = lane >> 4, col = lane & 15;
  const int e0 = blockIdx.x * 16 + col;
  const typename F::T* wp = Wg + (size_t)(e0 < E ? e0 : E - 1) * d;
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int units = d / 64;
  const int u1 = units * (blockIdx.y + 1) / gridDim.y;
  for (int u = units * blockIdx.y / gridDim.y + wave; u < u1; u += LG_WAVES) {
    F a;
    a.load(wp + u * 64, nullptr, q);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int i = min(t * 16 + col, N - 1);
      typename F::B b;
      if constexpr (XMX) {
        // the lane's k of a bf16 unit: 8 q and 32 + 8 q
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const size_t at = (size_t)i * d + u * 64 + m * 32 + q * 8;
          const uint2 c = *reinterpret_cast<const uint2*>(codes + at);
          b.r[m] = __builtin_bit_cast(u32x4, mx_widen8(c.x, c.y, mx_scale(scales[at / MX_BLOCK])));
          if (blockIdx.x == 0) *reinterpret_cast<u32x4*>(Xb + at) = b.r[m];
        }
      } else {
        b.load(X + (size_t)i * d + u * 64, q);
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
    const int i = wave * 16 + col, e = blockIdx.x * 16 + q * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (i < N && e + r < E) Z[((size_t)blockIdx.y * N + i) * E + e + r] = s[r];
  }
}

// ---- who chose an expert -------------------------------------------------------------

// The chosen experts in ascending order ("slots"): expert | tokens << 16, and by slot the tokens
// that chose it, ascending: token << 16 | pick.  TOK: tokens at most, lanes of an expert here.
// All of the workgroup's NT threads; pick [E, TOK] holds pick + 1 or 0, count [256] is scratch.
// Returns the number of slots.
template <int TOK, int NT, typename List, typename Rows>
__device__ __forceinline__ int list_tokens(const uint16_t (*pick)[TOK], int* count, int E, List list,
                                           Rows rows) {
  constexpr int PER = 64 / TOK;         // experts of a wave at a time
  const int lane = wave_lane(), wave = threadIdx.x >> 6;
  const int sub = lane / TOK, i = lane % TOK;
  const unsigned long long mask = TOK == 64 ? ~0ull : (1ull << TOK) - 1;
  const auto who_of = [&](int e) {
    const unsigned long long who = __ballot(e < E && pick[min(e, E - 1)][i] != 0);
    return (who >> (sub * TOK)) & mask;
  };
  for (int c = threadIdx.x; c < 256; c += NT) count[c] = 0;
  __syncthreads();
  for (int e0 = wave * PER; e0 < E; e0 += NT / 64 * PER) {
    const unsigned long long who = who_of(e0 + sub);
    if (i == 0 && e0 + sub < E) count[e0 + sub] = __popcll(who);
  }
  __syncthreads();
  unsigned long long used[4];
  int active = 0;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    used[m] = __ballot(count[lane + 64 * m] != 0);
    active += __popcll(used[m]);
  }
  for (int e0 = wave * PER; e0 < E; e0 += NT / 64 * PER) {
    const int e = e0 + sub;
    const unsigned long long who = who_of(e);
    if (who == 0) continue;
    int slot = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      if (m * 64 + 64 <= e) slot += __popcll(used[m]);
      else if (m * 64 <= e) slot += __popcll(used[m] & ((1ull << (e - m * 64)) - 1));
    }
    if (i == 0) list(slot, (uint32_t)e | (uint32_t)__popcll(who) << 16);
    const uint32_t p = pick[e][i];
    if (p) rows(slot, __popcll(who & ((1ull << i) - 1)), (uint32_t)i << 16 | (p - 1));
  }
  return active;
}

// The choice of more tokens than every workgroup of W1/W3 would make for itself: one workgroup,
// sixteen lanes a token.
template <int NQ>
__global__ __launch_bounds__(1024) void decode_choose_kernel(const float* __restrict__ Z, int N,
                                                             int E, int k, int splits,
                                                             float inv_tau,
                                                             int32_t* __restrict__ experts,
                                                             float* __restrict__ gates,
                                                             DecodePlan plan) {
  __shared__ uint16_t pick[256][DECODE_TOKENS];
  __shared__ int count[256];
  const int tid = threadIdx.x, i = tid >> 4, r = tid & 15;
  float z[NQ];
  if (i < N) load_logits<NQ>(z, Z, i, r, N, E, splits);
  for (int c = tid; c < E * DECODE_TOKENS / 2; c += 1024) reinterpret_cast<uint32_t*>(pick)[c] = 0;
  __syncthreads();
  if (i < N) {
    const float sum = choose<NQ>(z, E, k, inv_tau, r, [&](int c, int e, float ex) {
      experts[i * k + c] = e;
      gates[i * k + c] = ex;
      pick[e][i] = (uint16_t)(c + 1);
    });
    for (int c = r; c < k; c += 16) gates[i * k + c] = gates[i * k + c] / sum;
  }
  __syncthreads();
  const int active = list_tokens<DECODE_TOKENS, 1024>(
      pick, count, E, [&](int s, uint32_t v) { plan.list[s] = v; },
      [&](int s, int c, uint32_t v) { plan.rows[s * DECODE_TOKENS + c] = v; });
  if (tid == 0) plan.active[0] = active;
}

// ---- W1 and W3 -----------------------------------------------------------------------

constexpr int W13_WAVES = 4;
constexpr int W13_GRID = 512, W2_GRID = 512;    // workgroups at most: two a CU
constexpr int INLINE_TOKENS = 16;       // every workgroup of W1/W3 chooses for itself up to so
constexpr int INLINE_PAIRS = 256;       // many tokens, and pairs of token and expert

// Tiles of 16 hidden units: those of the chosen experts, slot after slot, then the shared
// experts' (for every token).  A workgroup takes a contiguous share of them, its waves a quarter
// of k each; the expert's tokens are the columns.  A burst's weights are requested before the one
// before it is used, over the ends of tiles and experts too, so that memory never waits.
//   A [token k + pick, h] = gate silu(W1 x) (W3 x).
// NQ > 0: the choice is made here, from the logits, by every workgroup (16 NQ experts at most),
// and the first writes it down.
template <class F, int TT, int NQ>
__global__ __launch_bounds__(64 * W13_WAVES, 2) void decode_w13_kernel(
    const typename F::T* __restrict__ X, DecodeWeights w, const float* __restrict__ Z, int splits,
    float inv_tau, int E, int32_t* __restrict__ experts, float* __restrict__ gates, DecodePlan plan,
    typename F::T* __restrict__ A, typename F::T* __restrict__ As, int N, int d, int h, int hs,
    int k) {
  typedef typename F::T T;
  typedef typename F::Code Code;
  constexpr int U = TT > 2 ? F::BURST / 2 : F::BURST;    // registers
  constexpr bool OWN = NQ > 0;
  constexpr int OT = OWN ? INLINE_TOKENS : 1;
  __shared__ f32x4 red[2][W13_WAVES][2 * TT][64];
  __shared__ uint16_t pick[OWN ? 256 : 1][OT];
  __shared__ int count[OWN ? 256 : 1];
  __shared__ uint32_t own_list[OWN ? 256 : 1], own_rows[OWN ? 256 : 1][OT];
  __shared__ float own_gates[OWN ? INLINE_PAIRS : 1];
  const int tid = threadIdx.x, lane = wave_lane(), q = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int active;
  if constexpr (OWN) {
    const int i = tid >> 4, r = tid & 15;
    float z[NQ];
    if (i < N) load_logits<NQ>(z, Z, i, r, N, E, splits);
    for (int c = tid; c < E * OT / 2; c += 64 * W13_WAVES) reinterpret_cast<uint32_t*>(pick)[c] = 0;
    __syncthreads();
    if (i < N) {
      const float sum = choose<NQ>(z, E, k, inv_tau, r, [&](int c, int e, float ex) {
        if (blockIdx.x == 0) experts[i * k + c] = e;
        own_gates[i * k + c] = ex;
        pick[e][i] = (uint16_t)(c + 1);
      });
      for (int c = r; c < k; c += 16) {
        const float g = own_gates[i * k + c] / sum;
        own_gates[i * k + c] = g;
        if (blockIdx.x == 0) gates[i * k + c] = g;
      }
    }
    __syncthreads();
    active = list_tokens<OT, 64 * W13_WAVES>(
        pick, count, E,
        [&](int s, uint32_t v) {
          own_list[s] = v;
          if (blockIdx.x == 0) plan.list[s] = v;
        },
        [&](int s, int c, uint32_t v) {
          own_rows[s][c] = v;
          if (blockIdx.x == 0) plan.rows[s * DECODE_TOKENS + c] = v;
        });
    if (blockIdx.x == 0 && tid == 0) plan.active[0] = active;
    __syncthreads();
  } else {
    active = plan.active[0];
  }
  const int ht = h / 16, routed = active * ht, tiles = routed + hs / 16;
  const int t1 = (int)((long)tiles * (blockIdx.x + 1) / gridDim.x);
  int tile = (int)((long)tiles * blockIdx.x / gridDim.x);
  if (tile >= t1) return;
  const int units = d / 64;
  const int u0 = units * wave / W13_WAVES, u1 = units * (wave + 1) / W13_WAVES, last = units - 1;

  // the weights of tile t, for the requests; columns of the tile in use
  const Code* rows[2];
  const uint8_t* scale[2];
  const auto aim = [&](int t) __attribute__((always_inline)) {
    const bool shared = t >= routed;
    size_t row;
    if (shared) {
      row = (size_t)(t - routed) * 16 + col;
    } else {
      const int s = t / ht;
      const uint32_t e = OWN ? own_list[s] : plan.list[s];
      row = (size_t)__builtin_amdgcn_readfirstlane(e & 0xffffu) * h + (t - s * ht) * 16 + col;
    }
    rows[0] = (const Code*)(shared ? w.Ws1 : w.W1) + row * d;
    rows[1] = (const Code*)(shared ? w.Ws3 : w.W3) + row * d;
    if (F::MX) {
      scale[0] = (shared ? w.Ss1 : w.S1) + row * (d / MX_BLOCK);
      scale[1] = (shared ? w.Ss3 : w.S3) + row * (d / MX_BLOCK);
    }
  };
  const auto request = [&](F (&to)[2][U], int u) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = min(u + i, last);     // past the end: the last unit again, not used
#pragma unroll
      for (int m = 0; m < 2; ++m)
        to[m][i].load(rows[m] + at * 64, F::MX ? scale[m] + at * 2 : nullptr, q);
    }
  };
  const T* x[TT];
  int at[TT], n = 0, slot = -1;
  float gate[TT];
  const auto columns = [&](int s) __attribute__((always_inline)) {
    slot = s;
    const bool shared = s >= active;
    n = shared ? N : __builtin_amdgcn_readfirstlane((OWN ? own_list[s] : plan.list[s]) >> 16);
    // columns past the last token repeat it; nothing of them is stored
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int c = min(t * 16 + col, n - 1);
      int token = c;
      at[t] = c;
      gate[t] = 1.0f;
      if (!shared) {
        const uint32_t p = OWN ? own_rows[s][c] : plan.rows[s * DECODE_TOKENS + c];
        token = (int)(p >> 16);
        at[t] = token * k + (int)(p & 0xffffu);
        gate[t] = OWN ? own_gates[at[t]] : gates[at[t]];
      }
      x[t] = X + (size_t)token * d;
    }
  };

  F a[2][2][U];
  f32x4 acc[2][TT];
  int u = u0, turn = 0;
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  aim(tile);
  request(a[0], u0);
  __builtin_amdgcn_sched_barrier(0);
  columns(tile < routed ? tile / ht : active);
  // one burst of the tile in use; false past the last tile
  const auto step = [&](F (&now)[2][U], F (&next)[2][U]) __attribute__((always_inline)) {
    typename F::B b[TT][U];
#pragma unroll
    for (int t = 0; t < TT; ++t)
      if (t == 0 || t * 16 < n)
#pragma unroll
        for (int i = 0; i < U; ++i) b[t][i].load(x[t] + min(u + i, last) * 64, q);
    const bool ends = u + U >= u1;
    if (!ends) {
      request(next, u + U);
    } else if (tile + 1 < t1) {
      aim(tile + 1);
      request(next, u0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (u + i < u1)
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t == 0 || t * 16 < n)
#pragma unroll
            for (int m = 0; m < 2; ++m) now[m][i].mma(acc[m][t], b[t][i]);
    if (!ends) {
      u += U;
      return true;
    }
    // the tile's end: the waves' shares meet
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      red[turn][wave][2 * t][lane] = acc[0][t];
      red[turn][wave][2 * t + 1][lane] = acc[1][t];
      acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    static_assert(TT <= W13_WAVES, "");
    const bool shared = tile >= routed;
    const int width = shared ? hs : h, unit = (shared ? tile - routed : tile % ht) * 16 + q * 4;
#pragma unroll
    for (int t = 0; t < TT; ++t)
      if (wave == t && t * 16 + col < n) {
        f32x4 f = red[turn][0][2 * t][lane], g = red[turn][0][2 * t + 1][lane];
#pragma unroll
        for (int i = 1; i < W13_WAVES; ++i) {
          f += red[turn][i][2 * t][lane];
          g += red[turn][i][2 * t + 1][lane];
        }
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gate[t] * (f[i] / (1.0f + expf(-f[i]))) * g[i];
        store4<T>((shared ? As : A) + (size_t)at[t] * width + unit, v);
      }
    turn ^= 1;
    u = u0;
    if (++tile >= t1) return false;
    const int s = tile < routed ? tile / ht : active;
    if (s != slot) columns(s);
    return true;
  };
  while (step(a[0], a[1]) && step(a[1], a[0])) {
  }
}

// ---- W2 ------------------------------------------------------------------------------

constexpr int W2_WAVES = 4;

// Tiles of 16 columns of Y (rows of W2), slot after slot, then the shared experts'.  Each wave
// streams a contiguous share of them by itself, as in W1/W3; the expert's tokens are the columns
// of the products, which go to O [token k + pick, d] in fp32 (the shared experts' to the rows
// from N k).
template <class F, int TT>
__global__ __launch_bounds__(64 * W2_WAVES, 2) void decode_w2_kernel(
    const typename F::T* __restrict__ A, const typename F::T* __restrict__ As, DecodeWeights w,
    DecodePlan plan, float* __restrict__ O, int N, int d, int h, int hs, int k) {
  typedef typename F::T T;
  typedef typename F::Code Code;
  constexpr int U = TT > 1 ? F::BURST : 2 * F::BURST;
  const int lane = wave_lane(), q = lane >> 4, col = lane & 15;
  const int active = plan.active[0];
  const int dt = d / 16, routed = active * dt, hu = h / 64, su = hs / 64;
  // shares of equal work, in units
  const long waves = (long)gridDim.x * W2_WAVES, total = (long)dt * (active * hu + su);
  const long g = (long)blockIdx.x * W2_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const auto tile_from = [&](long c) {
    const long r = (long)routed * hu;
    return (int)(c <= r ? (c + hu - 1) / hu : routed + (c - r + su - 1) / su);
  };
  int tile = tile_from(total * g / waves);
  const int t1 = tile_from(total * (g + 1) / waves);
  if (tile >= t1) return;
  const Code* row;
  const uint8_t* scale;
  const auto aim = [&](int t) __attribute__((always_inline)) {
    const bool shared = t >= routed;
    size_t r;
    if (shared) {
      r = (size_t)(t - routed) * 16 + col;
    } else {
      const int s = t / dt;
      r = (size_t)__builtin_amdgcn_readfirstlane(plan.list[s] & 0xffffu) * d + (t - s * dt) * 16 + col;
    }
    row = (const Code*)(shared ? w.Ws2 : w.W2) + r * (shared ? hs : h);
    if (F::MX) scale = (shared ? w.Ss2 : w.S2) + r * ((shared ? hs : h) / MX_BLOCK);
  };
  const auto request = [&](F (&to)[U], int u, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = min(u + i, last);
      to[i].load(row + at * 64, F::MX ? scale + at * 2 : nullptr, q);
    }
  };
  const T* x[TT];
  int at[TT], n = 0, slot = -1;
  const auto columns = [&](int s) __attribute__((always_inline)) {
    slot = s;
    const bool shared = s >= active;
    n = shared ? N : __builtin_amdgcn_readfirstlane(plan.list[s] >> 16);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int c = min(t * 16 + col, n - 1);
      if (shared) {
        x[t] = As + (size_t)c * hs;
        at[t] = N * k + c;
      } else {
        const uint32_t p = plan.rows[s * DECODE_TOKENS + c];
        at[t] = (int)(p >> 16) * k + (int)(p & 0xffffu);
        x[t] = A + (size_t)at[t] * h;
      }
    }
  };
  F a[2][U];
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  int u = 0, units = tile < routed ? hu : su;
  aim(tile);
  request(a[0], 0, units - 1);
  __builtin_amdgcn_sched_barrier(0);
  columns(tile < routed ? tile / dt : active);
  const auto step = [&](F (&now)[U], F (&next)[U]) __attribute__((always_inline)) {
    typename F::B b[TT][U];
#pragma unroll
    for (int t = 0; t < TT; ++t)
      if (t == 0 || t * 16 < n)
#pragma unroll
        for (int i = 0; i < U; ++i) b[t][i].load(x[t] + min(u + i, units - 1) * 64, q);
    const bool ends = u + U >= units;
    if (!ends) {
      request(next, u + U, units - 1);
    } else if (tile + 1 < t1) {
      aim(tile + 1);
      request(next, 0, (tile + 1 < routed ? hu : su) - 1);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (u + i < units)
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t == 0 || t * 16 < n) now[i].mma(acc[t], b[t][i]);
    if (!ends) {
      u += U;
      return true;
    }
    const int c = (tile < routed ? tile % dt : tile - routed) * 16 + q * 4;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      if (t * 16 + col < n) *reinterpret_cast<f32x4*>(O + (size_t)at[t] * d + c) = acc[t];
      acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    u = 0;
    if (++tile >= t1) return false;
    units = tile < routed ? hu : su;
    const int s = tile < routed ? tile / dt : active;
    if (s != slot) columns(s);
    return true;
  };
  while (step(a[0], a[1]) && step(a[1], a[0])) {
  }
}

// Y = R + the sum of a token's rows of O, in the order of the choice, the shared experts' last; four
// columns a lane.
template <typename T>
__global__ __launch_bounds__(64) void decode_sum_kernel(const float* __restrict__ O, const T* R,
                                                        T* Y, int N, int d, int k, int shared) {
  const int i = blockIdx.y, c = (blockIdx.x * 64 + threadIdx.x) * 4;
  if (c >= d) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  const float* o = O + (size_t)i * k * d + c;
#pragma unroll 8
  for (int j = 0; j < k; ++j) s += *reinterpret_cast<const f32x4*>(o + (size_t)j * d);
  if (shared) s += *reinterpret_cast<const f32x4*>(O + ((size_t)N * k + i) * d + c);
  float v[4] = {s[0], s[1], s[2], s[3]};
  if (R) {
    float x[4];
    load4<T>(R + (size_t)i * d + c, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += x[j];
  }
  store4<T>(Y + (size_t)i * d + c, v);
}

template <class F, int TT>
hipError_t run_decode(const DecodeCall& c, hipStream_t st) {
  typedef typename F::T T;
  typedef std::conditional_t<sizeof(T) == 4, WF32, WBf16> G;   // the router's weights
  const int splits = decode_splits(c.d);
  const dim3 lg((unsigned)((c.E + 15) / 16), (unsigned)splits);
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
  const T* X = (const T*)(c.Xs ? c.Xb : c.X);
  const int most = c.N * c.k < c.E ? c.N * c.k : c.E;    // chosen experts at most
  const long tiles13 = (long)most * (c.h / 16) + c.hs / 16;
  const long tiles2 = ((long)most + (c.hs ? 1 : 0)) * (c.d / 16);
  const auto w13 = [&](auto nq) {
    decode_w13_kernel<F, TT, decltype(nq)::value>
        <<<dim3((unsigned)(tiles13 < W13_GRID ? tiles13 : W13_GRID)), 64 * W13_WAVES, 0, st>>>(
            X, c.w, c.Z, splits, c.inv_tau, c.E, c.experts, c.gates, c.plan, (T*)c.A, (T*)c.As, c.N,
            c.d, c.h, c.hs, c.k);
  };
  bool chosen = false;
  if constexpr (TT == 1)
    if (c.N * c.k <= INLINE_PAIRS) {
      if (c.E <= 64) w13(std::integral_constant<int, 4>{});
      else w13(std::integral_constant<int, 16>{});
      chosen = true;
    }
  if (!chosen) {
    if (c.E <= 64)
      decode_choose_kernel<4><<<1, 1024, 0, st>>>(c.Z, c.N, c.E, c.k, splits, c.inv_tau, c.experts,
                                                  c.gates, c.plan);
    else
      decode_choose_kernel<16><<<1, 1024, 0, st>>>(c.Z, c.N, c.E, c.k, splits, c.inv_tau, c.experts,
                                                   c.gates, c.plan);
    w13(std::integral_constant<int, 0>{});
  }
  const long g2 = (tiles2 + W2_WAVES - 1) / W2_WAVES;
  decode_w2_kernel<F, TT><<<dim3((unsigned)(g2 < W2_GRID ? g2 : W2_GRID)), 64 * W2_WAVES, 0, st>>>(
      (const T*)c.A, (const T*)c.As, c.w, c.plan, c.O, c.N, c.d, c.h, c.hs, c.k);
  decode_sum_kernel<T><<<dim3((unsigned)((c.d + 255) / 256), (unsigned)c.N), 64, 0, st>>>(
      c.O, (const T*)c.R, (T*)c.Y, c.N, c.d, c.k, c.hs);
  return hipGetLastError();
}

template <class F>
hipError_t run_decode(const DecodeCall& c, hipStream_t st) {
  if (c.N <= 16) return run_decode<F, 1>(c, st);
  if (c.N <= 32) return run_decode<F, 2>(c, st);
  return run_decode<F, 4>(c, st);
}

}  // namespace

int decode_splits(int d) {
  const int most = (d / 64 + LG_WAVES - 1) / LG_WAVES;
  return most < LG_SPLITS ? most : LG_SPLITS;
}

hipError_t launch_decode(const DecodeCall& c, hipStream_t st) {
  if (c.N == 0) return hipSuccess;
  if (c.dtype == DT_F32) return run_decode<WF32>(c, st);
  return c.w.S1 ? run_decode<WMx>(c, st) : run_decode<WBf16>(c, st);
}

}  // namespace ec
