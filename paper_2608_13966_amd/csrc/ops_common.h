// ops_common.h -- device helpers of the operators of quasar_ops.h: pieces of
// eight elements at any alignment, reductions over a wavefront and a workgroup.
#pragma once

#include "device_common.h"

namespace quasar {

// element types of a tensor operand; kNone: no operand
enum ElemType : int { kElemF32 = 0, kElemBF16 = 1, kElemNone = 2, kElemE4M3 = 3 };
template <int T>
constexpr int elem_size() { return T == kElemF32 ? 4 : T == kElemE4M3 ? 1 : 2; }

// 16 bytes from or to an address of any alignment: one instruction
// (unaligned accesses to global memory are on under HSA), so rows whose
// stride or base is not a multiple of 16 bytes take the same code.
__device__ __forceinline__ uint4 ld16_any(const void* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
__device__ __forceinline__ void st16_any(void* p, uint4 v) { __builtin_memcpy(p, &v, 16); }
__device__ __forceinline__ uint2 ld8_any(const void* p) {
  uint2 v;
  __builtin_memcpy(&v, p, 8);
  return v;
}
__device__ __forceinline__ void st8_any(void* p, uint2 v) { __builtin_memcpy(p, &v, 8); }

// Element i of a tensor of run-time type (F32 or BF16).
__device__ __forceinline__ float elem(const void* p, int64_t i, bool bf16) {
  return bf16 ? as_f32((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16) : reinterpret_cast<const float*>(p)[i];
}
__device__ __forceinline__ uint16_t bf16_bits(float x) { return (uint16_t)pack_bf16x2(x, 0.0f); }
__device__ __forceinline__ void put_elem(void* p, int64_t i, float v, bool bf16) {
  if (bf16)
    reinterpret_cast<uint16_t*>(p)[i] = bf16_bits(v);
  else
    reinterpret_cast<float*>(p)[i] = v;
}

// Eight consecutive elements in their storage form; n of them exist (n >= 8:
// all), the rest read as 0.
template <int T>
struct Piece;
template <>
struct Piece<kElemBF16> {
  uint32_t d[4];
  __device__ __forceinline__ void load(const void* base, int64_t e, int n) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + e;
    if (n >= 8) {
      const uint4 t = ld16_any(p);
      d[0] = t.x; d[1] = t.y; d[2] = t.z; d[3] = t.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const uint32_t lo = 2 * i < n ? p[2 * i] : 0, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0;
        d[i] = lo | (hi << 16);
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    return (i & 1) ? as_f32(d[i >> 1] & 0xffff0000u) : as_f32(d[i >> 1] << 16);
  }
  // To the compiler the elements change here: what it formed from them before
  // is not kept in registers for a use after.
  __device__ __forceinline__ void refresh() { asm volatile("" : "+v"(d[0]), "+v"(d[1]), "+v"(d[2]), "+v"(d[3])); }
};
template <>
struct Piece<kElemF32> {
  float f[8];
  __device__ __forceinline__ void load(const void* base, int64_t e, int n) {
    const float* p = reinterpret_cast<const float*>(base) + e;
    if (n >= 8) {
      const uint4 a = ld16_any(p), b = ld16_any(p + 4);
      f[0] = as_f32(a.x); f[1] = as_f32(a.y); f[2] = as_f32(a.z); f[3] = as_f32(a.w);
      f[4] = as_f32(b.x); f[5] = as_f32(b.y); f[6] = as_f32(b.z); f[7] = as_f32(b.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] = i < n ? p[i] : 0.0f;
    }
  }
  __device__ __forceinline__ float get(int i) const { return f[i]; }
  __device__ __forceinline__ void refresh() {}
};

// Eight elements from each of N places on, the first n[i] of which exist (the
// others 0).  All loads are issued before the first is waited for.
template <int N>
__device__ __forceinline__ void load_floats(const void* base, const int64_t (&e)[N], const int (&n)[N], bool bf16,
                                            float (&v)[N][8]) {
  const auto load = [&](auto piece) {
    decltype(piece) p[N];
#pragma unroll
    for (int j = 0; j < N; j++) p[j].load(base, e[j], n[j]);
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
      for (int i = 0; i < 8; i++) v[j][i] = p[j].get(i);
  };
  if (bf16)
    load(Piece<kElemBF16>());
  else
    load(Piece<kElemF32>());
}
__device__ __forceinline__ void load_floats(const void* base, int64_t e, int n, bool bf16, float (&v)[8]) {
  const int64_t es[1] = {e};
  const int ns[1] = {n};
  float vs[1][8];
  load_floats(base, es, ns, bf16, vs);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = vs[0][i];
}

// Eight values to a tensor of fp32 or bf16 elements (nearest even), the first n of them.
template <bool BF16>
__device__ __forceinline__ void store_piece(void* base, int64_t e, const float (&v)[8], int n) {
  if constexpr (BF16) {
    uint16_t* p = reinterpret_cast<uint16_t*>(base) + e;
    if (n >= 8) {
      st16_any(p, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                             pack_bf16x2(v[6], v[7])));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < n) p[i] = bf16_bits(v[i]);
    }
  } else {
    float* p = reinterpret_cast<float*>(base) + e;
    if (n >= 8) {
      st16_any(p, make_uint4(as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3])));
      st16_any(p + 4, make_uint4(as_u32(v[4]), as_u32(v[5]), as_u32(v[6]), as_u32(v[7])));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < n) p[i] = v[i];
    }
  }
}
__device__ __forceinline__ void store_piece(void* base, int64_t e, const float (&v)[8], int n, bool bf16) {
  if (bf16)
    store_piece<true>(base, e, v, n);
  else
    store_piece<false>(base, e, v, n);
}

// Eight elements at byte `at` of a wavefront's buffer (wave_buffer in
// device_common.h): past its end loads give 0 and stores do nothing, without a
// branch.  The whole offset is the vector one: the check against the buffer's
// end is specified for that, not for a scalar offset beside it.
template <int T>
__device__ __forceinline__ void load_piece(Piece<T>& p, __amdgpu_buffer_rsrc_t b, int at) {
  if constexpr (T == kElemBF16) {
    const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0);
    p.d[0] = t.x; p.d[1] = t.y; p.d[2] = t.z; p.d[3] = t.w;
  } else {
    const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0);
    const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(b, at + 16, 0, 0);
    p.f[0] = as_f32(t.x); p.f[1] = as_f32(t.y); p.f[2] = as_f32(t.z); p.f[3] = as_f32(t.w);
    p.f[4] = as_f32(u.x); p.f[5] = as_f32(u.y); p.f[6] = as_f32(u.z); p.f[7] = as_f32(u.w);
  }
}
// For stores there is one more reason: after a 128-bit buffer store with
// a scalar offset register the compiler puts no wait state before an overwrite
// of the data's first register, and such stores wrote the overwriting value's
// dword here now and then.
template <bool BF16>
__device__ __forceinline__ void store_piece(__amdgpu_buffer_rsrc_t b, int at, const float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 t = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    __builtin_amdgcn_raw_buffer_store_b128(t, b, at, 0, 0);
  } else {
    const u32x4 t = {as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3])};
    const u32x4 u = {as_u32(v[4]), as_u32(v[5]), as_u32(v[6]), as_u32(v[7])};
    __builtin_amdgcn_raw_buffer_store_b128(t, b, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(u, b, at + 16, 0, 0);
  }
}

// Eight values as E4M3 bytes (nearest even; |v| <= 448 (1 + 2^-4) rounds
// inside the format, NaN gives its NaN).
__device__ __forceinline__ uint2 pack_e4m3x8(const float (&v)[8]) {
  int a = 0, b = 0;
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], a, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], a, true);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], b, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], b, true);
  return make_uint2((uint32_t)a, (uint32_t)b);
}

// ---- reductions -------------------------------------------------------------
// Over the wavefront's 64 lanes, every lane gets the same bits (the pairing
// of lanes is symmetric); no LDS.  A NaN is not kept by the maximum.
struct SumOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct MaxOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
template <typename Op>
__device__ __forceinline__ float wave_reduce(float x, Op op) {
  x = op(x, dpp_f32<kDppXor1>(x));
  x = op(x, dpp_f32<kDppXor2>(x));
  x = op(x, dpp_f32<kDppHalfMirror>(x));
  x = op(x, dpp_f32<kDppMirror>(x));
  x = pair_rows<16>(x, op);
  return pair_rows<32>(x, op);
}

// Over a workgroup of WAVES wavefronts; `s`: WAVES floats of LDS that nothing
// else uses and that the previous reduction through them is done with (one
// barrier in between is enough: each call has one of its own).
template <int WAVES, typename Op>
__device__ __forceinline__ float group_reduce(float x, float* s, Op op) {
  x = wave_reduce(x, op);
  if constexpr (WAVES == 1) return x;
  if ((threadIdx.x & 63) == 0) s[wave_index()] = x;
  __syncthreads();
  x = s[0];
#pragma unroll
  for (int i = 1; i < WAVES; i++) x = op(x, s[i]);
  return x;
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eRest = (float)(1.44269504088896340736 - (double)kLog2e);
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLn2Rest = (float)(0.69314718055994530942 - (double)kLn2);

// exp(x) and log(x) from the hardware's exponential and logarithm to base 2, the
// rounding of the argument (the result) and of the constant made good: 2 to 4 x
// 2^-24 relative.  x <= 0 or NaN; x >= 1, 0 or NaN.  (expf and logf hold registers
// for arguments that do not occur here: with them a kernel full of pieces spilled.)
__device__ __forceinline__ float exp_of(float x) {
  const float t = x * kLog2e, rest = __builtin_fmaf(x, kLog2e, -t) + x * kLog2eRest;
  const float e = __builtin_amdgcn_exp2f(t);
  return t < -150.0f ? 0.0f : __builtin_fmaf(e, rest * kLn2, e);
}
__device__ __forceinline__ float log_of(float x) {
  const float y = __builtin_amdgcn_logf(x), t = y * kLn2, rest = __builtin_fmaf(y, kLn2, -t) + y * kLn2Rest;
  return x == 0.0f ? t : t + rest;
}
// Quotients by the same number in every lane: its reciprocal in two parts.
struct Divisor {
  float hi, lo;
  __device__ __forceinline__ explicit Divisor(float d) {
    hi = uniform_f32(1.0f / d);
    lo = uniform_f32(__builtin_fmaf(-d, hi, 1.0f) * hi);
  }
  __device__ __forceinline__ float of(float x) const {
    return fabsf(x) == INFINITY ? x : __builtin_fmaf(x, hi, x * lo);
  }
};

}  // namespace quasar
