// The token-choice layer for a few tokens (a serving step): N <= 64 tokens, every one kept.
//   z = x Wg^T;  C = the top_k experts of z (equal logits: the lower index);
//   g = softmax over C of z / tau;
//   y = residual + sum over j in C of W2_j (g_j silu(W1_j x) * (W3_j x)) + the shared experts.
//
// The weights of the chosen experts bound it: each is read once, for at most 64 tokens, far
// below the operations that the matrix cores need to be the limit.  So weight rows are the
// MFMAs' A operand, streamed from memory into registers, and the tokens that chose the expert
// are its 16 columns.  Launches: logits, (past 16 tokens) choice, W1/W3, W2, sum.
//
// Measured, d 2048, 64 experts of 1024, top 8, bf16: 64 tokens 5.2 + 6.5 + 87 + 48 + 5.1 us for
// 806 MB (W1/W3 6.2 TB/s, W2 5.5), one token 3.0 + 16.6 + 8.8 + 3.8 for 101 MB.  In eight bits 16
// tokens 4.6 + 49 + 25 + 4.6 for 367 MB.  A kernel's first 2 to 4 us are its launch.  Slower by the
// byte: more than 16 tokens an expert, whose activations every tile reads (64 tokens, 16 such
// experts, W1/W3 34 and W2 26 us: 4.0 and 2.6 TB/s), shared experts beside 64 tokens (of 1024, W1/W3
// 124 and W2 88 us), and shares of whole tiles that do not come out even (one token, experts of
// 1088: W1/W3 21.4 us).
//
// Weights come in the storage type or in eight bits with scales (mx.h), which turn into bf16
// on their way to the matrix cores, exactly (four leading bits) for scale bytes 3 to 246: below,
// the last bit may lie under bf16's 2^-133, above, the value past its range.  The tokens and
// activations that they meet are bf16, so eight bits cost no accuracy beyond the weights' own.
#include <hip/hip_runtime.h>

#include "ec_kernels.h"
#include "mx.h"

namespace ec {

namespace {

// Loads that are known to be of global memory: a generic one waits together with LDS.
template <typename V>
__device__ __forceinline__ V load_global(const void* p) {
  return *(const __attribute__((address_space(1))) V*)p;
}
template <typename V>
__device__ __forceinline__ V stream_global(const void* p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) V*)p);
}

// Eight codes as bf16, times 2^(byte - 127).
__device__ __forceinline__ bf16x8 mx_widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The scale as widening takes it, by its exponent field alone: 0 there is 2^-127 too.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte == MX_NAN ? 0x7fc00000u : byte << 23);
}

__device__ __forceinline__ f32x4 mma_bf16(u32x4 a, u32x4 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}

// Weights come in chunks, 256 bytes of each of 16 rows: sixteen pieces of 16 bytes a row.  As
// the MFMAs' A operand a lane needs row lane & 15 and, of each quarter s of the chunk, piece
// 4 s + q, q = lane >> 4; the k of its column (a token) that they meet are B's.
//
// bf16: a chunk is 128 k, a piece 8 of them.
struct WBf16 {
  typedef bf16_t T;       // tokens and activations
  typedef bf16_t Code;
  static constexpr int K = 128;       // k of a chunk
  static constexpr bool MX = false;
  struct B {
    u32x4 r[4];
    // row: the token's, at the chunk; `left` k are there (a multiple of 64)
    __device__ __forceinline__ void load(const bf16_t* row, int q, int left) {
#pragma unroll
      for (int s = 0; s < 4; ++s) r[s] = load_global<u32x4>(row + min(s * 32, left - 32) + q * 8);
    }
  };
  static constexpr int WIDE = 4;      // 16-byte operands of a chunk
  static __device__ __forceinline__ void widen(u32x4 (&)[4], const uint2&, int) {}
  static __device__ __forceinline__ void mma(f32x4& acc, const u32x4 (&a)[4], const B& b, int left) {
    acc = mma_bf16(a[0], b.r[0], acc);
    acc = mma_bf16(a[1], b.r[1], acc);
    if (left < K) return;
    acc = mma_bf16(a[2], b.r[2], acc);
    acc = mma_bf16(a[3], b.r[3], acc);
  }
};

// Eight bits: a chunk is 256 k, a piece 16 of them, which lie in one block; a quarter is two.
struct WMx {
  typedef bf16_t T;
  typedef uint8_t Code;
  static constexpr int K = 256;
  static constexpr bool MX = true;
  struct B {
    u32x4 r[8];
    __device__ __forceinline__ void load(const bf16_t* row, int q, int left) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bf16_t* p = row + min(s * 64, left - 64) + q * 16;
        r[2 * s] = load_global<u32x4>(p);
        r[2 * s + 1] = load_global<u32x4>(p + 8);
      }
    }
  };
  static constexpr int WIDE = 8;
  // the first four as bf16; scale: the row's eight bytes of the chunk
  static __device__ __forceinline__ void widen(u32x4 (&a)[8], const uint2& scale, int q) {
#pragma unroll
    for (int s = 3; s >= 0; --s) {
      const uint32_t word = s < 2 ? scale.x : scale.y;
      const float f = mx_scale(__builtin_amdgcn_ubfe(word, (s & 1) * 16 + (q >> 1) * 8, 8));
      const u32x4 c = a[s];
      a[2 * s] = __builtin_bit_cast(u32x4, mx_widen8(c[0], c[1], f));
      a[2 * s + 1] = __builtin_bit_cast(u32x4, mx_widen8(c[2], c[3], f));
    }
  }
  static __device__ __forceinline__ void mma(f32x4& acc, const u32x4 (&a)[8], const B& b, int left) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s * 64 >= left) return;
      acc = mma_bf16(a[2 * s], b.r[2 * s], acc);
      acc = mma_bf16(a[2 * s + 1], b.r[2 * s + 1], acc);
    }
  }
};

// fp32: a chunk is 64 k, a piece four of them.
struct WF32 {
  typedef float T;
  typedef float Code;
  static constexpr int K = 64;
  static constexpr bool MX = false;
  struct B {
    f32x4 r[4];
    __device__ __forceinline__ void load(const float* row, int q, int) {
#pragma unroll
      for (int s = 0; s < 4; ++s) r[s] = load_global<f32x4>(row + s * 16 + q * 4);
    }
  };
  static constexpr int WIDE = 4;
  static __device__ __forceinline__ void widen(u32x4 (&)[4], const uint2&, int) {}
  static __device__ __forceinline__ void mma(f32x4& acc, const u32x4 (&a)[4], const B& b, int) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const f32x4 v = __builtin_bit_cast(f32x4, a[s]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], b.r[s][j], acc, 0, 0, 0);
    }
  }
};

// Of two values (of two variables that a lambda holds by reference, ?: would choose the address).
template <typename V>
__device__ __forceinline__ V either(bool first, V a, V b) { return first ? a : b; }

// A chunk on its way: from memory an instruction takes 256 consecutive bytes of four rows (64
// bytes of each of sixteen, the operand's own order, reach 5.1 to 6.1 TB/s where this reaches
// 6.6), so lane (q, c) holds piece c of rows 4 m + q, and the scales of quarter q of row c.
template <class F>
struct Chunk {
  struct Lds {
    u32x4 piece[16][16];
    uint2 scale[16];
  };
  u32x4 r[4];
  uint16_t scale;
  // w: row 0 of the tile at the chunk; row, srow: bytes of a row; left: k there, 0 for a chunk
  // that is not used (the same 16 bytes for every lane)
  __device__ __forceinline__ void load(const typename F::Code* w, uint32_t row, const uint8_t* s,
                                       uint32_t srow, int left) {
    const int lane = wave_lane(), q = lane >> 4, c = lane & 15;
    // pieces past the row's end: the last one again, not used
    const int piece = max(min(c, left * (int)sizeof(typename F::Code) / 16 - 1), 0);
    const uint32_t step = left > 0 ? row : 0;
    const char* p = reinterpret_cast<const char*>(w) + (q * step + piece * 16);
#pragma unroll
    for (int m = 0; m < 4; ++m) r[m] = stream_global<u32x4>(p + m * 4 * step);
    if (F::MX) scale = load_global<uint16_t>(s + (left > 0 ? c * srow : 0) + max(min(q, left / 64 - 1), 0) * 2);
  }
  // through LDS of the wave's own to the operand's order: piece c of row r at place c ^ r of
  // the row, so that neither side meets in a bank
  __device__ __forceinline__ void turn(Lds& lds, u32x4 (&a)[F::WIDE]) const {
    const int lane = wave_lane(), q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int m = 0; m < 4; ++m) lds.piece[4 * m + q][c ^ (4 * m + q)] = r[m];
    if (F::MX) reinterpret_cast<uint16_t*>(lds.scale)[c * 4 + q] = scale;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int s = 0; s < 4; ++s) a[s] = lds.piece[c][(4 * s + q) ^ c];
    uint2 scales = {0, 0};
    if (F::MX) scales = lds.scale[c];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    F::widen(a, scales, q);
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
  for (int c0 = 0; c0 < k; c0 += 16) {
    uint32_t mine = 0;
    int expert = 0;
    for (int c = c0; c < min(k, c0 + 16); ++c) {
      uint32_t top = key[0];
#pragma unroll
      for (int m = 1; m < NQ; ++m) top = max(top, key[m]);
      top = row16_max_u32(top);
      int j = 256;
#pragma unroll
      for (int m = NQ - 1; m >= 0; --m) j = key[m] == top ? r + 16 * m : j;
      j = row16_min_i32(j);
#pragma unroll
      for (int m = 0; m < NQ; ++m) key[m] = j == r + 16 * m ? 0u : key[m];
      if (c == 0) z0 = key_logit(top);
      if (r == c - c0) {
        mine = top;
        expert = j;
      }
    }
    if (c0 + r < k) {
      const float ex = expf((key_logit(mine) - z0) * inv_tau);
      sum += ex;
      put(c0 + r, expert, ex);
    }
  }
  return row16_sum_even(sum);
}

constexpr int LG_SPLITS = 8;     // splits of the logits' k at most

// Logits r, r + 16, ... of a token: the sums of the splits' shares, in order, requested together.
template <int NQ>
__device__ __forceinline__ void load_logits(float (&z)[NQ], const float* __restrict__ Z, int i, int r,
                                            int N, int E, int splits) {
  constexpr int S = NQ > 4 ? 2 : LG_SPLITS;     // registers
#pragma unroll
  for (int m = 0; m < NQ; ++m) z[m] = 0.f;
  for (int s0 = 0; s0 < splits; s0 += S) {
    float v[S][NQ];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int m = 0; m < NQ; ++m)
        v[s][m] = Z[((size_t)min(s0 + s, splits - 1) * N + i) * E + min(r + 16 * m, E - 1)];
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s0 + s < splits)
#pragma unroll
        for (int m = 0; m < NQ; ++m) z[m] += v[s][m];
  }
}

constexpr int LG_WAVES = 8;

// Z [splits, N, E]: shares of X Wg^T.  A workgroup takes 16 experts and the 64s of k of split
// blockIdx.y, its waves every eighth; they meet in LDS in a fixed order.  The few rows of Wg are
// loaded in the operand's order.  XMX: the tokens come in eight bits; their rows go to Xb as
// bf16 for the expert products.
template <typename T, int TT, bool XMX>
__global__ __launch_bounds__(64 * LG_WAVES) void decode_logits_kernel(
    const T* __restrict__ X, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
    const T* __restrict__ Wg, float* __restrict__ Z, bf16_t* __restrict__ Xb, int N, int d, int E) {
  __shared__ f32x4 red[LG_WAVES][TT][64];
  constexpr int L = 64 * sizeof(T) / 64;       // 16-byte loads of 64 k: 2 or 4
  constexpr int P = 16 / sizeof(T);            // k of one
  const int lane = wave_lane(), wave = threadIdx.x >> 6, q = lane >> 4, col = lane & 15;
  const int e0 = blockIdx.x * 16 + col;
  const T* wp = Wg + (size_t)(e0 < E ? e0 : E - 1) * d + q * P;
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int units = d / 64;
  const int u1 = units * (blockIdx.y + 1) / gridDim.y;
  for (int u = units * blockIdx.y / gridDim.y + wave; u < u1; u += LG_WAVES) {
    u32x4 a[L];
#pragma unroll
    for (int m = 0; m < L; ++m)
      a[m] = *reinterpret_cast<const u32x4*>(wp + u * 64 + m * 4 * P);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int i = min(t * 16 + col, N - 1);
#pragma unroll
      for (int m = 0; m < L; ++m) {
        const size_t at = (size_t)i * d + u * 64 + m * 4 * P + q * P;
        u32x4 b;
        if constexpr (XMX) {
          const uint2 c = *reinterpret_cast<const uint2*>(codes + at);
          b = __builtin_bit_cast(u32x4, mx_widen8(c.x, c.y, mx_scale(scales[at / MX_BLOCK])));
          if (blockIdx.x == 0) *reinterpret_cast<u32x4*>(Xb + at) = b;
        } else {
          b = *reinterpret_cast<const u32x4*>(X + at);
        }
        if constexpr (sizeof(T) == 2) {
          acc[t] = mma_bf16(a[m], b, acc[t]);
        } else {
          const f32x4 fa = __builtin_bit_cast(f32x4, a[m]), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[j], fb[j], acc[t], 0, 0, 0);
        }
      }
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

// The choice by expert (DecodePlan): used, bit j: some token chose expert j; pick [E, TOK] by
// token, pick + 1 or 0.  The chosen experts in ascending order are the "slots".
template <int TT>
constexpr int plan_tokens() { return TT == 1 ? 16 : DECODE_TOKENS; }

struct Used {
  unsigned long long w[4];
  __device__ __forceinline__ int count() const {
    return __popcll(w[0]) + __popcll(w[1]) + __popcll(w[2]) + __popcll(w[3]);
  }
  // the expert of a slot
  __device__ __forceinline__ int expert(int slot) const {
    const int lane = wave_lane();
    int found = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int rank = __popcll(w[m] & ((1ull << lane) - 1));
      const unsigned long long hit = __ballot(((w[m] >> lane) & 1) && rank == slot);
      if (hit) found = m * 64 + __builtin_ctzll(hit);
      slot -= __popcll(w[m]);
    }
    return __builtin_amdgcn_readfirstlane(found);
  }
};

// The columns of an expert's products: with 16 tokens at most each token is its own, else those
// that chose the expert move together.  p: the lane's token's entry of pick (lane % 16 with
// 16 tokens).  token, pick: of the columns of this lane, t 16 + lane % 16; mine: bit t, whether the
// column is a token's (another repeats one, and nothing of it is stored); returns their number.
template <int TT>
__device__ __forceinline__ int columns_of(uint32_t p, int (&token)[TT], int (&pick)[TT],
                                          uint32_t* mine) {
  const int lane = wave_lane(), col = lane & 15;
  const unsigned long long who = __ballot(p != 0);
  *mine = 0;
  if constexpr (TT == 1) {
    const int first = __builtin_ctz((uint32_t)who & 0xffffu);
    const uint32_t q = __builtin_amdgcn_readlane(p, first);
    token[0] = p ? col : first;
    pick[0] = (int)(p ? p : q) - 1;
    *mine = p != 0;
    return 16;
  } else {
    const int n = __popcll(who), before = __popcll(who & ((1ull << lane) - 1));
    const int to = p ? before : n + lane - before;
    const int moved = __builtin_amdgcn_ds_permute(to * 4, lane << 16 | (int)(p ? p - 1 : 0));
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int c = t * 16 + col;
      const int v = __shfl(moved, min(c, n - 1));
      token[t] = v >> 16;
      pick[t] = v & 0xffff;
      *mine |= (uint32_t)(c < n) << t;
    }
    return n;
  }
}

// The choice of more tokens than every workgroup of W1/W3 would make for itself: one workgroup,
// sixteen lanes a token.
template <int NQ, int TOK>
__global__ __launch_bounds__(16 * TOK) void decode_choose_kernel(const float* __restrict__ Z, int N,
                                                                 int E, int k, int splits,
                                                                 float inv_tau,
                                                                 int32_t* __restrict__ experts,
                                                                 float* __restrict__ gates,
                                                                 DecodePlan plan) {
  __shared__ uint32_t pick[256 * TOK / 2];
  __shared__ unsigned long long used[4];
  const int tid = threadIdx.x, i = tid >> 4, r = tid & 15;
  float z[NQ];
  if (i < N) load_logits<NQ>(z, Z, i, r, N, E, splits);
  for (int c = tid; c < E * TOK / 2; c += 16 * TOK) pick[c] = 0;
  if (tid < 4) used[tid] = 0;
  __syncthreads();
  if (i < N) {
    const float sum = choose<NQ>(z, E, k, inv_tau, r, [&](int c, int e, float ex) {
      experts[i * k + c] = e;
      gates[i * k + c] = ex;
      reinterpret_cast<uint16_t*>(pick)[e * TOK + i] = (uint16_t)(c + 1);
      atomicOr(&used[e >> 6], 1ull << (e & 63));
    });
    for (int c = r; c < k; c += 16) gates[i * k + c] = gates[i * k + c] / sum;
  }
  __syncthreads();
  for (int c = tid; c < E * TOK / 2; c += 16 * TOK) reinterpret_cast<uint32_t*>(plan.pick)[c] = pick[c];
  if (tid < 4) plan.used[tid] = used[tid];
}

// ---- W1 and W3 -----------------------------------------------------------------------

template <typename T>
constexpr int act_parts() { return sizeof(T) == 2 ? 2 : 1; }

constexpr int W13_WAVES = 4;
// Workgroups at most, two or four a CU (64 tokens: W1/W3 512 87.6 us, 1024 85.0, 2048 84.7, and 512
// are best where each of them chooses; W2 512 47.9, 1024 48.9, 2048 53.6).
constexpr int W13_GRID = 1024, W13_OWN_GRID = 512, W2_GRID = 512;
// Up to so many tokens, and pairs of token and expert, every workgroup of W1/W3 chooses for
// itself (3.3 us at its start; the choice in a launch of its own takes 6.1).
constexpr int INLINE_TOKENS = 16;
constexpr int INLINE_PAIRS = 256;
static_assert(INLINE_TOKENS == plan_tokens<1>(), "one tile of columns");

// Tiles of 16 hidden units: those of the chosen experts, slot after slot, then the shared
// experts' (for every token).  A workgroup takes a contiguous share of them, its waves a quarter
// of k each; the expert's tokens are the columns.  A chunk's weights are requested before the one
// before it is used, over the ends of tiles and experts too, so that memory never waits; every
// step requests, at the end what is not used, so that the waits can count.
//   A [token k + pick, h] = gate silu(W1 x) (W3 x), in bf16 as two rows: the value rounded and what
// that left, rounded.  With one the rounding would be as large as the output's own (2-norm 0.0024
// of Y, now 0.0017).
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
  constexpr int PARTS = act_parts<T>();
  constexpr int AHEAD = F::MX && TT > 2 ? 2 : TT;   // tiles of columns requested ahead: registers
  constexpr int TURNS = TT > 2 ? 1 : 2;     // LDS for two workgroups a CU
  constexpr bool OWN = NQ > 0;
  constexpr int PT = plan_tokens<TT>();
  __shared__ f32x4 red[TURNS][W13_WAVES][2 * TT][64];
  __shared__ typename Chunk<F>::Lds turned[W13_WAVES][2];
  __shared__ uint32_t own_pick[OWN ? 256 * PT / 2 : 1];
  __shared__ unsigned long long own_used[4];
  __shared__ float own_gates[OWN ? INLINE_PAIRS : 1];
  const int tid = threadIdx.x, lane = wave_lane(), q = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Used used;
  if constexpr (OWN) {
    const int i = tid >> 4, r = tid & 15;
    float z[NQ];
    if (i < N) load_logits<NQ>(z, Z, i, r, N, E, splits);
    for (int c = tid; c < E * PT / 2; c += 64 * W13_WAVES) own_pick[c] = 0;
    if (tid < 4) own_used[tid] = 0;
    __syncthreads();
    if (i < N) {
      const float sum = choose<NQ>(z, E, k, inv_tau, r, [&](int c, int e, float ex) {
        if (blockIdx.x == 0) experts[i * k + c] = e;
        own_gates[i * k + c] = ex;
        reinterpret_cast<uint16_t*>(own_pick)[e * PT + i] = (uint16_t)(c + 1);
        atomicOr(&own_used[e >> 6], 1ull << (e & 63));
      });
      for (int c = r; c < k; c += 16) {
        const float g = own_gates[i * k + c] / sum;
        own_gates[i * k + c] = g;
        if (blockIdx.x == 0) gates[i * k + c] = g;
      }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
      for (int c = tid; c < E * PT / 2; c += 64 * W13_WAVES)
        reinterpret_cast<uint32_t*>(plan.pick)[c] = own_pick[c];
      if (tid < 4) plan.used[tid] = own_used[tid];
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) used.w[m] = own_used[m];
  } else {
#pragma unroll
    for (int m = 0; m < 4; ++m) used.w[m] = plan.used[m];
  }
  const int active = used.count(), ht = h / 16, tiles = active * ht + hs / 16;
  const int t0 = (int)((long)tiles * blockIdx.x / gridDim.x);
  const int t1 = (int)((long)tiles * (blockIdx.x + 1) / gridDim.x);
  if (t0 >= t1) return;
  const int chunks = (d + F::K - 1) / F::K;
  const int u0 = chunks * wave / W13_WAVES, u1 = chunks * (wave + 1) / W13_WAVES;

  // the tile in use and, one ahead where it ends, the one that is requested: slot (active: the
  // shared experts) and tile of it
  int slot = min(t0 / ht, active), tile = t0 - slot * ht, left = t1 - t0;
  int rslot = slot, rtile = tile, expert = slot < active ? used.expert(slot) : 0;
  const auto request = [&](Chunk<F> (&to)[2], int u, bool live) __attribute__((always_inline)) {
    const bool shared = rslot == active;
    const size_t row = (size_t)expert * (shared ? 0 : h) + rtile * 16;
    const int k0 = min(u, chunks - 1) * F::K;
    const Code* w1 = (const Code*)either(shared, w.Ws1, w.W1) + (row * d + k0);
    const Code* w3 = (const Code*)either(shared, w.Ws3, w.W3) + (row * d + k0);
    const size_t at = row * (d / MX_BLOCK) + k0 / MX_BLOCK;
    to[0].load(w1, d * sizeof(Code), F::MX ? either(shared, w.Ss1, w.S1) + at : nullptr, d / MX_BLOCK,
               live ? d - k0 : 0);
    to[1].load(w3, d * sizeof(Code), F::MX ? either(shared, w.Ss3, w.S3) + at : nullptr, d / MX_BLOCK,
               live ? d - k0 : 0);
  };
  const T* x[TT];
  int at[TT], n = 0;
  uint32_t mine = 0;
  float gate[TT];
  const auto columns = [&]() __attribute__((always_inline)) {
    int token[TT], pick[TT];
    if (slot == active) {
      n = TT == 1 ? 16 : N;
      mine = 0;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        at[t] = token[t] = min(t * 16 + col, N - 1);
        gate[t] = 1.0f;
        mine |= (uint32_t)(t * 16 + col < N) << t;
      }
    } else {
      const int o = used.expert(slot) * PT + (PT == 16 ? col : lane);
      n = columns_of<TT>(OWN ? reinterpret_cast<const uint16_t*>(own_pick)[o] : plan.pick[o], token,
                         pick, &mine);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        at[t] = token[t] * k + pick[t];
        gate[t] = OWN ? own_gates[at[t]] : gates[at[t]];
      }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = X + (size_t)token[t] * d;
  };

  Chunk<F> a[2][2];
  f32x4 acc[2][TT];
  int u = u0, turn = 0;
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  request(a[0], u0, true);
  columns();
  // one chunk of the tile in use; false past the last tile
  const auto step = [&](Chunk<F> (&now)[2], Chunk<F> (&next)[2]) __attribute__((always_inline)) {
    const int k0 = min(u, chunks - 1) * F::K;
    typename F::B b[AHEAD];
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)     // before the request: memory answers in order
      if (t == 0 || t * 16 < n) b[t].load(x[t] + k0, q, d - k0);
    const bool ends = u + 1 >= u1;
    if (ends && left > 1 && ++rtile == (rslot < active ? ht : hs / 16)) {
      rtile = 0;
      expert = ++rslot < active ? used.expert(rslot) : 0;
    }
    request(next, ends ? u0 : u + 1, !ends || left > 1);
    __builtin_amdgcn_sched_barrier(0);
    if (u < u1) {                     // else more waves than chunks
      u32x4 op[2][F::WIDE];
#pragma unroll
      for (int m = 0; m < 2; ++m) now[m].turn(turned[wave][m], op[m]);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t > 0 && t * 16 >= n) break;
        typename F::B& bt = b[t % AHEAD];
        if (t >= AHEAD) bt.load(x[t] + k0, q, d - k0);
#pragma unroll
        for (int m = 0; m < 2; ++m) F::mma(acc[m][t], op[m], bt, d - k0);
      }
    }
    if (!ends) {
      ++u;
      return true;
    }
    // the tile's end: the waves' shares meet
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      red[turn][wave][2 * t][lane] = acc[0][t];
      red[turn][wave][2 * t + 1][lane] = acc[1][t];
      acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    lds_barrier();
    static_assert(TT <= W13_WAVES, "");
#pragma unroll
    for (int t = 0; t < TT; ++t)
      if (wave == t && ((mine >> t) & 1)) {
        f32x4 f = red[turn][0][2 * t][lane], g = red[turn][0][2 * t + 1][lane];
#pragma unroll
        for (int i = 1; i < W13_WAVES; ++i) {
          f += red[turn][i][2 * t][lane];
          g += red[turn][i][2 * t + 1][lane];
        }
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gate[t] * (f[i] / (1.0f + expf(-f[i]))) * g[i];
        const int width = slot < active ? h : hs;
        T* o = either(slot < active, A, As) + (size_t)at[t] * (PARTS * width) + tile * 16 + q * 4;
        store4<T>(o, v);
        if constexpr (PARTS == 2) {     // what the rounding left
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float hi = round_to<T>(v[i]);
            v[i] = fabsf(hi) < INFINITY ? v[i] - hi : 0.f;
          }
          store4<T>(o + width, v);
        }
      }
    if (TURNS == 1) lds_barrier();
    turn ^= TURNS - 1;
    u = u0;
    if (--left == 0) return false;
    tile = rtile;
    if (slot != rslot) {
      slot = rslot;
      columns();
    }
    return true;
  };
  while (step(a[0], a[1]) && step(a[1], a[0])) {
  }
}

// ---- W2 ------------------------------------------------------------------------------

constexpr int W2_WAVES = 4;

// k of a wave's share whose activations stay in its registers (64 of them) from tile to tile.
constexpr int W2_KEPT = 256;

// Tiles of 32 columns of Y (rows of W2), slot after slot, then the shared experts'.  A workgroup
// takes a contiguous share of them (of equal work), its waves a quarter of k each, streamed as in
// W1/W3, a chunk of both 16 rows a step; the expert's tokens are the columns of the products,
// which go to O [token k + pick, d] in fp32 (the shared experts' to the rows from N k).
// KEEP (both widths W2_WAVES W2_KEPT at most): the activations of the first 16 columns are loaded
// once a slot (64 tokens 58.0 -> 48.9 us, 16 in eight bits 32.6 -> 27.9).  Wider ones do not fit the
// registers (experts of 1088 beside 1024: 66 and 48 us, in eight bits 39 and 25).
template <class F, int TT, bool KEEP>
__global__ __launch_bounds__(64 * W2_WAVES, 2) void decode_w2_kernel(
    const typename F::T* __restrict__ A, const typename F::T* __restrict__ As, DecodeWeights w,
    DecodePlan plan, float* __restrict__ O, int N, int d, int h, int hs, int k) {
  typedef typename F::T T;
  typedef typename F::Code Code;
  constexpr int PARTS = act_parts<T>();
  constexpr int PT = plan_tokens<TT>();
  constexpr int TURNS = TT > 2 ? 1 : 2;
  constexpr int NK = KEEP ? W2_KEPT / F::K : 1;       // 2, 1 or 4 chunks
  // tiles of columns whose activations are requested before the next weights, as many as the
  // registers hold (64 tokens over 64 experts bf16, all four launches: 157.8 us with one, 153.4)
  constexpr int AHEAD = F::MX ? 1 : PARTS == 1 ? TT : KEEP && TT > 2 ? 2 : TT < 3 ? TT : 3;
  __shared__ f32x4 red[TURNS][W2_WAVES][2 * TT][64];
  __shared__ typename Chunk<F>::Lds turned[W2_WAVES][2];
  const int lane = wave_lane(), q = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Used used;
#pragma unroll
  for (int m = 0; m < 4; ++m) used.w[m] = plan.used[m];
  const int active = used.count(), dt = d / 32, routed = active * dt;
  const int hu = h / 64, su = hs / 64;
  const long total = (long)dt * (active * hu + su);
  const auto tile_from = [&](long c) {
    const long r = (long)routed * hu;
    return (int)(c <= r ? (c + hu - 1) / hu : routed + (c - r + su - 1) / su);
  };
  const int t0 = tile_from(total * blockIdx.x / gridDim.x);
  const int t1 = tile_from(total * (blockIdx.x + 1) / gridDim.x);
  if (t0 >= t1) return;
  int slot = min(t0 / dt, active), tile = t0 - slot * dt, left = t1 - t0;
  int rslot = slot, rtile = tile, expert = slot < active ? used.expert(slot) : 0;
  const auto chunks_of = [&](int s) { return ((s == active ? hs : h) + F::K - 1) / F::K; };
  const auto request = [&](Chunk<F> (&to)[2], int u, bool live) __attribute__((always_inline)) {
    const bool shared = rslot == active;
    const int wide = shared ? hs : h, k0 = live ? u * F::K : 0;
    const size_t at = ((size_t)expert * (shared ? 0 : d) + rtile * 32) * wide + k0;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const size_t r = at + (size_t)(m * 16) * wide;
      to[m].load((const Code*)either(shared, w.Ws2, w.W2) + r, wide * sizeof(Code),
                 F::MX ? either(shared, w.Ss2, w.S2) + r / MX_BLOCK : nullptr, wide / MX_BLOCK,
                 live ? wide - k0 : 0);
    }
  };
  const T* x[TT];
  int at[TT], n = 0, width = 0, u0 = 0, u1 = 0, chunks = 0;
  uint32_t mine = 0;
  typename F::B kept[NK][PARTS];
  const auto load_b = [&](typename F::B& b, int t, int u, int p) __attribute__((always_inline)) {
    const int k0 = min(u, chunks - 1) * F::K;
    b.load(x[t] + p * width + k0, q, width - k0);
  };
  const auto columns = [&]() __attribute__((always_inline)) {
    int token[TT], pick[TT];
    const bool shared = slot == active;
    width = shared ? hs : h;
    chunks = chunks_of(slot);
    u0 = chunks * wave / W2_WAVES;
    u1 = chunks * (wave + 1) / W2_WAVES;
    if (shared) {
      n = TT == 1 ? 16 : N;
      mine = 0;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int c = t * 16 + col;
        at[t] = min(c, N - 1);
        mine |= (uint32_t)(c < N) << t;
      }
    } else {
      n = columns_of<TT>(plan.pick[used.expert(slot) * PT + (PT == 16 ? col : lane)], token, pick,
                         &mine);
#pragma unroll
      for (int t = 0; t < TT; ++t) at[t] = token[t] * k + pick[t];
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      x[t] = either(shared, As, A) + (size_t)at[t] * (PARTS * width);
      if (shared) at[t] += N * k;
    }
    if constexpr (KEEP)
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int p = 0; p < PARTS; ++p) load_b(kept[i][p], 0, u0 + i, p);
  };
  Chunk<F> a[2][2];
  f32x4 acc[2][TT];
  int u = 0;        // of the wave's share
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[0][t] = acc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  {
    const int c = chunks_of(slot), first = c * wave / W2_WAVES;
    request(a[0], first, first < c * (wave + 1) / W2_WAVES);
  }
  columns();
  // one chunk of the tile in use, the I-th of the wave's share where it is kept; false past the
  // last tile
  const auto step = [&](auto now_of, auto kept_of) __attribute__((always_inline)) {
    constexpr int P = decltype(now_of)::value, I = decltype(kept_of)::value;
    typename F::B loaded[AHEAD][PARTS];
#pragma unroll
    for (int t = KEEP ? 1 : 0; t < AHEAD; ++t)    // before the request: memory answers in order
      if (t == 0 || t * 16 < n)
#pragma unroll
        for (int p = 0; p < PARTS; ++p) load_b(loaded[t][p], t, u0 + u, p);
    const int share = u1 - u0;
    const bool ends = KEEP ? I + 1 == NK : u + 1 >= share;
    int next = u0 + u + 1;
    bool live = u + 1 < share;
    if (ends) {
      if (left > 1 && ++rtile == dt) {
        rtile = 0;
        expert = ++rslot < active ? used.expert(rslot) : 0;
      }
      const int c = chunks_of(rslot);
      next = c * wave / W2_WAVES;
      live = left > 1 && next < c * (wave + 1) / W2_WAVES;
    }
    request(a[P ^ 1], next, live);
    __builtin_amdgcn_sched_barrier(0);
    if (u < share) {
      u32x4 op[2][F::WIDE];
#pragma unroll
      for (int m = 0; m < 2; ++m) a[P][m].turn(turned[wave][m], op[m]);
      const int there = width - (u0 + u) * F::K;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t > 0 && t * 16 >= n) break;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          typename F::B late;
          if (t >= AHEAD) load_b(late, t, u0 + u, p);
#pragma unroll
          for (int m = 0; m < 2; ++m)
            F::mma(acc[m][t], op[m],
                   t >= AHEAD ? late : KEEP && t == 0 ? kept[I][p] : loaded[t % AHEAD][p], there);
        }
      }
    }
    ++u;
    if (!ends) return true;
    // the tile's end: the waves' shares meet
    f32x4 (&sums)[W2_WAVES][2 * TT][64] = red[TURNS == 1 ? 0 : left & 1];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        sums[wave][2 * t + m][lane] = acc[m][t];
        acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    lds_barrier();
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        if (wave == (2 * t + m) % W2_WAVES && ((mine >> t) & 1)) {
          f32x4 v = sums[0][2 * t + m][lane];
#pragma unroll
          for (int i = 1; i < W2_WAVES; ++i) v += sums[i][2 * t + m][lane];
          *reinterpret_cast<f32x4*>(O + (size_t)at[t] * d + tile * 32 + m * 16 + q * 4) = v;
        }
    if (TURNS == 1) lds_barrier();
    u = 0;
    if (--left == 0) return false;
    tile = rtile;
    if (slot != rslot) {
      slot = rslot;
      columns();
    }
    return true;
  };
  using zero = std::integral_constant<int, 0>;
  using one = std::integral_constant<int, 1>;
  if constexpr (NK == 4) {
    while (step(zero{}, zero{}) && step(one{}, one{}) &&
           step(zero{}, std::integral_constant<int, 2>{}) &&
           step(one{}, std::integral_constant<int, 3>{})) {
    }
  } else {
    while (step(zero{}, zero{}) && step(one{}, std::integral_constant<int, NK - 1>{})) {
    }
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
  const int splits = decode_splits(c.d);
  const dim3 lg((unsigned)((c.E + 15) / 16), (unsigned)splits);
  if (c.Xs) {
    if constexpr (sizeof(T) == 2)
      decode_logits_kernel<T, TT, true><<<lg, 64 * LG_WAVES, 0, st>>>(
          nullptr, (const uint8_t*)c.X, c.Xs, (const T*)c.Wg, c.Z, (bf16_t*)c.Xb, c.N, c.d, c.E);
    else
      return hipErrorInvalidValue;
  } else {
    decode_logits_kernel<T, TT, false><<<lg, 64 * LG_WAVES, 0, st>>>(
        (const T*)c.X, nullptr, nullptr, (const T*)c.Wg, c.Z, nullptr, c.N, c.d, c.E);
  }
  const T* X = (const T*)(c.Xs ? c.Xb : c.X);
  const int most = c.N * c.k < c.E ? c.N * c.k : c.E;    // chosen experts at most
  const long tiles13 = (long)most * (c.h / 16) + c.hs / 16;
  const auto w13 = [&](auto nq) {
    constexpr long most_wgs = decltype(nq)::value ? W13_OWN_GRID : W13_GRID;
    decode_w13_kernel<F, TT, decltype(nq)::value>
        <<<dim3((unsigned)(tiles13 < most_wgs ? tiles13 : most_wgs)), 64 * W13_WAVES, 0, st>>>(
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
    constexpr int PT = plan_tokens<TT>();
    if (c.E <= 64)
      decode_choose_kernel<4, PT><<<1, 16 * PT, 0, st>>>(c.Z, c.N, c.E, c.k, splits, c.inv_tau,
                                                         c.experts, c.gates, c.plan);
    else
      decode_choose_kernel<16, PT><<<1, 16 * PT, 0, st>>>(c.Z, c.N, c.E, c.k, splits, c.inv_tau,
                                                          c.experts, c.gates, c.plan);
    w13(std::integral_constant<int, 0>{});
  }
  const long tiles2 = ((long)most + (c.hs ? 1 : 0)) * (c.d / 32);
  const dim3 g2((unsigned)(tiles2 < W2_GRID ? tiles2 : W2_GRID));
  // (in eight bits and four tiles of columns the registers hold no more)
  constexpr bool CAN_KEEP = !(F::MX && TT > 2);
  if (CAN_KEEP && (c.h > c.hs ? c.h : c.hs) <= W2_WAVES * W2_KEPT)
    decode_w2_kernel<F, TT, CAN_KEEP><<<g2, 64 * W2_WAVES, 0, st>>>(
        (const T*)c.A, (const T*)c.As, c.w, c.plan, c.O, c.N, c.d, c.h, c.hs, c.k);
  else
    decode_w2_kernel<F, TT, false><<<g2, 64 * W2_WAVES, 0, st>>>(
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

int decode_act_parts(int dtype) {
  return dtype == DT_F32 ? act_parts<float>() : act_parts<bf16_t>();
}

hipError_t launch_decode(const DecodeCall& c, hipStream_t st) {
  if (c.N == 0) return hipSuccess;
  if (c.dtype == DT_F32) return run_decode<WF32>(c, st);
  return c.w.S1 ? run_decode<WMx>(c, st) : run_decode<WBf16>(c, st);
}

}  // namespace ec
