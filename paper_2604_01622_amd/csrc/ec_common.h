// Device-side helpers shared by the expert-choice MoE kernels (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ec {

typedef uint16_t bf16_t;  // bf16 storage: the upper 16 bits of an fp32

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// fp32 -> bf16, round to nearest, ties to even (v_cvt_pk_bf16_f32; NaN stays NaN).
__device__ __forceinline__ uint32_t f32_to_bf16(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Storage-type traits: load/store 8 consecutive elements as fp32.
template <typename T> struct Elem;

template <> struct Elem<float> {
  struct Raw { float4 a, b; };
  static __device__ __forceinline__ Raw load_raw(const float* p) {
    return Raw{*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)};
  }
  static __device__ __forceinline__ void fma_raw(float acc[8], float g, const Raw& r) {
    acc[0] = fmaf(g, r.a.x, acc[0]); acc[1] = fmaf(g, r.a.y, acc[1]);
    acc[2] = fmaf(g, r.a.z, acc[2]); acc[3] = fmaf(g, r.a.w, acc[3]);
    acc[4] = fmaf(g, r.b.x, acc[4]); acc[5] = fmaf(g, r.b.y, acc[5]);
    acc[6] = fmaf(g, r.b.z, acc[6]); acc[7] = fmaf(g, r.b.w, acc[7]);
  }
  static __device__ __forceinline__ void load8(const float* p, float v[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    const float4 b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ __forceinline__ void store8(float* p, const float v[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
  static __device__ __forceinline__ float load1(const float* p) { return *p; }
  static __device__ __forceinline__ void store1(float* p, float v) { *p = v; }
};

template <> struct Elem<bf16_t> {
  typedef uint4 Raw;
  // a streaming (non-temporal) load: the combines read each expert row once
  // (measured: -6-7% on both)
  static __device__ __forceinline__ Raw load_raw(const bf16_t* p) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
  }
  static __device__ __forceinline__ void fma_raw(float acc[8], float g, const Raw& r) {
    acc[0] = fmaf(g, bf16_to_f32(r.x & 0xffffu), acc[0]); acc[1] = fmaf(g, bf16_to_f32(r.x >> 16), acc[1]);
    acc[2] = fmaf(g, bf16_to_f32(r.y & 0xffffu), acc[2]); acc[3] = fmaf(g, bf16_to_f32(r.y >> 16), acc[3]);
    acc[4] = fmaf(g, bf16_to_f32(r.z & 0xffffu), acc[4]); acc[5] = fmaf(g, bf16_to_f32(r.z >> 16), acc[5]);
    acc[6] = fmaf(g, bf16_to_f32(r.w & 0xffffu), acc[6]); acc[7] = fmaf(g, bf16_to_f32(r.w >> 16), acc[7]);
  }
  static __device__ __forceinline__ void load8(const bf16_t* p, float v[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    v[0] = bf16_to_f32(a.x & 0xffffu); v[1] = bf16_to_f32(a.x >> 16);
    v[2] = bf16_to_f32(a.y & 0xffffu); v[3] = bf16_to_f32(a.y >> 16);
    v[4] = bf16_to_f32(a.z & 0xffffu); v[5] = bf16_to_f32(a.z >> 16);
    v[6] = bf16_to_f32(a.w & 0xffffu); v[7] = bf16_to_f32(a.w >> 16);
  }
  static __device__ __forceinline__ void store8(bf16_t* p, const float v[8]) {
    uint4 a;
    a.x = pack_bf16x2(v[0], v[1]); a.y = pack_bf16x2(v[2], v[3]);
    a.z = pack_bf16x2(v[4], v[5]); a.w = pack_bf16x2(v[6], v[7]);
    // a streaming (non-temporal) store: no kernel re-reads its own output within
    // the same launch (later launches do: W2 and dW2 read A, dA reads H1/H3, the
    // combine reads O), and the hint keeps the written lines from displacing the
    // launch's operands in the caches (measured: combines -8-9%, dA -2%)
    __builtin_nontemporal_store(u32x4{a.x, a.y, a.z, a.w}, reinterpret_cast<u32x4*>(p));
  }
  static __device__ __forceinline__ float load1(const bf16_t* p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ void store1(bf16_t* p, float v) { *p = (bf16_t)f32_to_bf16(v); }
};

// 16 bytes at any element's address: the hardware takes them in one access all the same.
typedef u32x4 u32x4_odd __attribute__((aligned(2)));

// VEC elements as they are stored, read once by a streaming load (16384 x 2048 bf16, with and
// without: the norm's backward pass 48.0 and 49.1 us, forward with a residual 44.3 and 43.8, without
// one 26.3 and 22.4).  ODD: at any element's address, where neighbouring loads share lines that a
// streaming one would give up (norm of 5000 x 4097 bf16 with a residual: 50.5 us with, 37.2
// without), else aligned to their size.
template <typename T, int VEC, bool ODD = false>
struct Piece {
  std::conditional_t<VEC == 1, T, u32x4> raw;
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC == 1)
      raw = __builtin_nontemporal_load(p);
    else if constexpr (ODD)
      raw = *reinterpret_cast<const u32x4_odd*>(p);
    else
      raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  }
  // what other workgroups read too: kept in the caches
  __device__ __forceinline__ void load_shared(const T* p) {
    if constexpr (VEC == 1) raw = *p;
    else raw = *reinterpret_cast<const std::conditional_t<ODD, u32x4_odd, u32x4>*>(p);
  }
  __device__ __forceinline__ void get(float* v) const {
    if constexpr (VEC == 1 && sizeof(T) == 4) {
      v[0] = raw;
    } else if constexpr (VEC == 1) {
      v[0] = bf16_to_f32(raw);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_to_f32(raw[i] & 0xffffu);
        v[2 * i + 1] = bf16_to_f32(raw[i] >> 16);
      }
    }
  }
};

// VEC elements from fp32, 16 or (fp32, eight) 32 bytes.  bf16 at any element's address in streaming
// stores (norm of 5000 x 4097 with a residual: 50.2 us without, 37.2), else in plain ones (16384 x
// 2048: 46.0 and 44.3).
template <typename T, int VEC, bool ODD>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  typedef std::conditional_t<ODD, u32x4_odd, u32x4> V;
  if constexpr (VEC == 1) {
    Elem<T>::store1(p, v[0]);
  } else if constexpr (sizeof(T) == 2) {
    const u32x4 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                     pack_bf16x2(v[6], v[7])};
    if constexpr (ODD) __builtin_nontemporal_store(w, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4)
      *reinterpret_cast<V*>(p + i) = u32x4{__float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                                           __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
  }
}

// Four consecutive elements.
template <typename T>
__device__ __forceinline__ void load4(const T* p, float* v) {
  if constexpr (sizeof(T) == 2) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    v[0] = bf16_to_f32(a.x & 0xffffu); v[1] = bf16_to_f32(a.x >> 16);
    v[2] = bf16_to_f32(a.y & 0xffffu); v[3] = bf16_to_f32(a.y >> 16);
  } else {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  }
}

template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else
    store_vec<T, 4, false>(p, v);
}

// A barrier for LDS alone: __syncthreads() would wait for a wave's loads on their way too.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A value as the storage type holds it.
template <typename T>
__device__ __forceinline__ float round_to(float v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(f32_to_bf16(v));
  return v;
}

// Hardware exp2 and reciprocal (about 1 ulp each): the activations feed bf16
// stores or fp32 sums whose tolerance is far wider.
__device__ __forceinline__ float sigmoid_f(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

__device__ __forceinline__ float silu_f(float z) { return z * sigmoid_f(z); }

// Sum over the 16 lanes of a DPP row (lanes 16 r .. 16 r + 15); every lane of
// the row ends with the total.  Quad swaps (xor 1, xor 2) then row rotations
// by 4 and 8 lanes, all in registers (no LDS permute).
__device__ __forceinline__ float dpp_add(float t, int ctrl_id) {
  int v = __builtin_bit_cast(int, t);
  switch (ctrl_id) {
    case 0: v = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false); break;   // quad [1,0,3,2]
    case 1: v = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false); break;   // quad [2,3,0,1]
    case 2: v = __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false); break;  // row_ror:4
    default: v = __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false); break; // row_ror:8
  }
  return t + __builtin_bit_cast(float, v);
}
__device__ __forceinline__ float row16_sum(float t) {
  return dpp_add(dpp_add(dpp_add(dpp_add(t, 0), 1), 2), 3);
}

// The same total with the same bits in every lane: mirrors of half rows and rows pair each
// lane with one that adds the same two sums, where the rotations of row16_sum add the quads
// in another order in each of them.
template <int CTRL>
__device__ __forceinline__ float dpp_plus(float t) {
  return t + __builtin_bit_cast(
                 float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, t), CTRL, 0xF, 0xF,
                                                    false));
}
__device__ __forceinline__ float row16_sum_even(float t) {
  return dpp_plus<0x140>(dpp_plus<0x141>(dpp_plus<0x4E>(dpp_plus<0xB1>(t))));
}

// DPP move of a 32-bit value within rows of 16 lanes; lanes whose source is
// outside the row read 0 (bound_ctrl).  Controls used here: quad_perm
// [1,0,3,2] = 0xB1 and [2,3,0,1] = 0x4E, row_shl:n = 0x100 + n, row_ror:n = 0x120 + n.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
  return __builtin_bit_cast(float, dpp_u32<CTRL>(__builtin_bit_cast(uint32_t, v)));
}

// Maximum of unsigned integers over the 16 lanes of a DPP row; every lane ends with it.
__device__ __forceinline__ uint32_t row16_max_u32(uint32_t t) {
  t = max(t, dpp_u32<0xB1>(t));
  t = max(t, dpp_u32<0x4E>(t));
  t = max(t, dpp_u32<0x124>(t));
  return max(t, dpp_u32<0x128>(t));
}

// Sum of integers over the 16 lanes of a DPP row; every lane of the row ends with it.
__device__ __forceinline__ int row16_sum_i32(int t) {
  t += (int)dpp_u32<0xB1>((uint32_t)t);
  t += (int)dpp_u32<0x4E>((uint32_t)t);
  t += (int)dpp_u32<0x124>((uint32_t)t);
  return t + (int)dpp_u32<0x128>((uint32_t)t);
}

// Minimum over the 16 lanes of a DPP row; every lane of the row ends with it.
__device__ __forceinline__ int row16_min_i32(int t) {
  const auto low = [](int a, uint32_t b) { return a < (int)b ? a : (int)b; };
  t = low(t, dpp_u32<0xB1>((uint32_t)t));
  t = low(t, dpp_u32<0x4E>((uint32_t)t));
  t = low(t, dpp_u32<0x124>((uint32_t)t));
  return low(t, dpp_u32<0x128>((uint32_t)t));
}

// Maximum over the 16 lanes of a DPP row; every lane of the row ends with it.
__device__ __forceinline__ float row16_max(float t) {
  t = fmaxf(t, dpp_f32<0xB1>(t));
  t = fmaxf(t, dpp_f32<0x4E>(t));
  t = fmaxf(t, dpp_f32<0x124>(t));
  return fmaxf(t, dpp_f32<0x128>(t));
}

// Minimum and maximum of an unsigned value over the whole wave (uniform results).
__device__ __forceinline__ void wave_minmax_u32(uint32_t mn, uint32_t mx, uint32_t* out_mn,
                                                uint32_t* out_mx) {
  uint32_t a, b;
  a = dpp_u32<0xB1>(mn); mn = a < mn ? a : mn;  b = dpp_u32<0xB1>(mx); mx = b > mx ? b : mx;
  a = dpp_u32<0x4E>(mn); mn = a < mn ? a : mn;  b = dpp_u32<0x4E>(mx); mx = b > mx ? b : mx;
  a = dpp_u32<0x124>(mn); mn = a < mn ? a : mn; b = dpp_u32<0x124>(mx); mx = b > mx ? b : mx;
  a = dpp_u32<0x128>(mn); mn = a < mn ? a : mn; b = dpp_u32<0x128>(mx); mx = b > mx ? b : mx;
  uint32_t rmn = __builtin_amdgcn_readlane(mn, 0), rmx = __builtin_amdgcn_readlane(mx, 0);
#pragma unroll
  for (int r = 16; r < 64; r += 16) {
    const uint32_t c = __builtin_amdgcn_readlane(mn, r), d = __builtin_amdgcn_readlane(mx, r);
    rmn = c < rmn ? c : rmn;
    rmx = d > rmx ? d : rmx;
  }
  *out_mn = rmn;
  *out_mx = rmx;
}

// Exclusive suffix sum over the wave's lanes: the sum of v over lanes > lane.
__device__ __forceinline__ uint32_t wave_excl_suffix_u32(uint32_t v) {
  uint32_t x = v;                       // inclusive suffix within the row of 16
  x += dpp_u32<0x101>(x);
  x += dpp_u32<0x102>(x);
  x += dpp_u32<0x104>(x);
  x += dpp_u32<0x108>(x);
  const uint32_t t1 = __builtin_amdgcn_readlane(x, 16), t2 = __builtin_amdgcn_readlane(x, 32),
                 t3 = __builtin_amdgcn_readlane(x, 48);
  const int row = (threadIdx.x & 63) >> 4;
  const uint32_t later = row == 0 ? t1 + t2 + t3 : (row == 1 ? t2 + t3 : (row == 2 ? t3 : 0u));
  return x - v + later;
}

// Order-preserving map from fp32 to uint32 (larger float -> larger key).
__device__ __forceinline__ uint32_t f32_order_key(float f) {
  uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int wave_lane() { return threadIdx.x & 63; }

// Remap a linear workgroup id so that consecutive tile ids land on the same XCD.
// Workgroups are dispatched round-robin over the 8 XCDs; the launch pads the
// grid to a multiple of 8 and ids >= n_tiles exit.
__device__ __forceinline__ int xcd_tile_id(int bid, int grid) {
  const int per_xcd = grid >> 3;
  return (bid & 7) * per_xcd + (bid >> 3);
}

}  // namespace ec
