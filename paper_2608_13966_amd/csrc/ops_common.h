// ops_common.h -- device helpers of the operators of quasar_ops.h: pieces of
// eight elements at any alignment, reductions over a wavefront and a workgroup.
#pragma once

#include "device_common.h"
#include "quasar_ops.h"

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
// ... non-temporal: for what is read or written once and is too much for the caches to keep
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
__device__ __forceinline__ uint4 ld16_any_nt(const void* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)));
}
__device__ __forceinline__ void st16_any_nt(void* p, uint4 v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4_any, v), reinterpret_cast<u32x4_any*>(p));
}
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
  template <bool NT = false>
  __device__ __forceinline__ void load(const void* base, int64_t e, int n) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + e;
    if (n >= 8) {
      const uint4 t = NT ? ld16_any_nt(p) : ld16_any(p);
      d[0] = t.x; d[1] = t.y; d[2] = t.z; d[3] = t.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const uint32_t lo = 2 * i < n ? p[2 * i] : 0, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0;
        d[i] = lo | (hi << 16);
      }
    }
  }
  // The first `gone` elements (1 to 8) go, the rest move up, 0 behind them.
  __device__ __forceinline__ void drop(int gone) {
    const uint32_t odd = (uint32_t)(gone & 1) * 16u;
#pragma unroll
    for (int i = 0; i < 4; i++) d[i] = __builtin_amdgcn_alignbit(i < 3 ? d[i + 1] : 0u, d[i], odd);
#pragma unroll
    for (int by = 1; by <= 4; by *= 2)
      if (gone & (2 * by)) {
#pragma unroll
        for (int i = 0; i < 4; i++) d[i] = i + by < 4 ? d[i + by] : 0u;
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
  template <bool NT = false>
  __device__ __forceinline__ void load(const void* base, int64_t e, int n) {
    const float* p = reinterpret_cast<const float*>(base) + e;
    if (n >= 8) {
      const uint4 a = NT ? ld16_any_nt(p) : ld16_any(p), b = NT ? ld16_any_nt(p + 4) : ld16_any(p + 4);
      f[0] = as_f32(a.x); f[1] = as_f32(a.y); f[2] = as_f32(a.z); f[3] = as_f32(a.w);
      f[4] = as_f32(b.x); f[5] = as_f32(b.y); f[6] = as_f32(b.z); f[7] = as_f32(b.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) f[i] = i < n ? p[i] : 0.0f;
    }
  }
  __device__ __forceinline__ void drop(int gone) {
#pragma unroll
    for (int by = 1; by <= 8; by *= 2)
      if (gone & by) {
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = i + by < 8 ? f[i + by] : 0.0f;
      }
  }
  __device__ __forceinline__ float get(int i) const { return f[i]; }
  __device__ __forceinline__ void refresh() {}
};

// Eight elements of a row (it begins at element `row` and has `cols`) from column c on, the rest 0.  Where MODE says
// cut, a piece that the row's end cuts comes as the row's last eight, without a branch, so that the loads of several
// pieces run side by side (element by element each is waited for); cut() then moves what there is to its place.
enum CutMode : int { kCutNone = 0, kCutBF16 = 1, kCutAll = 2, kCutTiny = 4 };  // of elements so wide; rows of less than eight occur
template <int MODE, int T>
constexpr bool cuts() { return (MODE & 3) >= (T == kElemBF16 ? 1 : 2); }
template <int MODE, int T>
__device__ __forceinline__ void load_cut(Piece<T>& p, const void* base, int64_t row, int c, int cols) {
  if (!cuts<MODE, T>() || ((MODE & kCutTiny) && cols < 8))
    p.load(base, row + c, cols - c);
  else
    p.load(base, row + (c < cols - 8 ? c : cols - 8), 8);
}
template <int MODE, int T>
__device__ __forceinline__ void cut(Piece<T>& p, int c, int cols) {
  if constexpr (cuts<MODE, T>()) {
    const int left = cols - c;
    if (left < 8 && !((MODE & kCutTiny) && cols < 8)) p.drop(left > 0 ? 8 - left : 8);
  }
}
// The same, widened, N pieces at once.
template <int MODE, int N>
__device__ __forceinline__ void load_cut_floats(const void* base, int64_t row, const int (&c)[N], int cols, bool bf16,
                                                float (&v)[N][8]) {
  const auto load = [&](auto piece) {
    decltype(piece) p[N];
#pragma unroll
    for (int j = 0; j < N; j++) load_cut<MODE>(p[j], base, row, c[j], cols);
#pragma unroll
    for (int j = 0; j < N; j++) {
      cut<MODE>(p[j], c[j], cols);
#pragma unroll
      for (int i = 0; i < 8; i++) v[j][i] = p[j].get(i);
    }
  };
  if (bf16)
    load(Piece<kElemBF16>());
  else
    load(Piece<kElemF32>());
}

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

template <bool NT>
__device__ __forceinline__ void st16_as(void* p, uint4 v) {
  if constexpr (NT)
    st16_any_nt(p, v);
  else
    st16_any(p, v);
}

// Eight values to a tensor of fp32 or bf16 elements (nearest even), the first n of them.
template <bool BF16, bool NT = false>
__device__ __forceinline__ void store_piece(void* base, int64_t e, const float (&v)[8], int n) {
  if constexpr (BF16) {
    uint16_t* p = reinterpret_cast<uint16_t*>(base) + e;
    if (n >= 8) {
      st16_as<NT>(p, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                             pack_bf16x2(v[6], v[7])));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < n) p[i] = bf16_bits(v[i]);
    }
  } else {
    float* p = reinterpret_cast<float*>(base) + e;
    if (n >= 8) {
      st16_as<NT>(p, make_uint4(as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3])));
      st16_as<NT>(p + 4, make_uint4(as_u32(v[4]), as_u32(v[5]), as_u32(v[6]), as_u32(v[7])));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < n) p[i] = v[i];
    }
  }
}
template <bool NT = false>
__device__ __forceinline__ void store_piece(void* base, int64_t e, const float (&v)[8], int n, bool bf16) {
  if (bf16)
    store_piece<true, NT>(base, e, v, n);
  else
    store_piece<false, NT>(base, e, v, n);
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

// Eight bytes to an address of any alignment, the first n of them.
__device__ __forceinline__ void store_bytes(uint8_t* p, uint2 b, int n) {
  if (n >= 8) {
    st8_any(p, b);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = (uint8_t)((i < 4 ? b.x : b.y) >> (8 * (i & 3)));
  }
}

// Eight bytes from an address of any alignment; n of them exist (n >= 8: all), the rest read as 0.
__device__ __forceinline__ uint2 load_bytes(const uint8_t* p, int n) {
  uint2 b = make_uint2(0u, 0u);
  if (n >= 8) {
    b = ld8_any(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) (i < 4 ? b.x : b.y) |= (uint32_t)p[i] << (8 * (i & 3));
  }
  return b;
}
// Eight E4M3 bytes as fp32.
__device__ __forceinline__ void unpack_e4m3x8(uint2 b, float (&v)[8]) {
  const auto p = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.x, false), q = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.x, true);
  const auto r = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.y, false), t = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.y, true);
  v[0] = p[0]; v[1] = p[1]; v[2] = q[0]; v[3] = q[1];
  v[4] = r[0]; v[5] = r[1]; v[6] = t[0]; v[7] = t[1];
}

// Quotients of 31-bit numbers by the same divisor: a high product and shifts
// (Granlund and Montgomery's round-up method).
struct Divide {
  uint32_t by, mul;
  int first, rest;
  explicit Divide(uint32_t d) : by(d) {
    int l = 0;
    while (l < 32 && ((uint64_t)1 << l) < d) l++;
    mul = (uint32_t)((((((uint64_t)1 << l) - d) << 32) / d) + 1);
    first = l < 1 ? l : 1;
    rest = l > 1 ? l - 1 : 0;
  }
  __device__ __forceinline__ uint32_t of(uint32_t u) const {
    const uint32_t t = __umulhi(mul, u);
    return (t + ((u - t) >> first)) >> rest;
  }
};

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

// x / d rounded to nearest, inv = 1 / d rounded to nearest: the product's error is
// taken off twice (the remainders are exact), the first time to within one place,
// from where the second gives the rounded quotient (Markstein).  x inv alone puts
// a value at the edge between two bytes on the wrong one.  16384 x 4096 bf16, q alone
// and all in the last-level cache: 36 us, with the compiler's division for any divisor
// 42, with x inv 35; 524288 x 128: 174, 212, 151; with y and from memory no difference.
__device__ __forceinline__ float quotient(float x, float d, float inv) {
  float q = x * inv;
  q = __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
  return __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
}

// ---- activations ------------------------------------------------------------
// The upper tail of the normal distribution at u >= 0, erfc(u / sqrt 2) / 2 =
// exp(-u^2 / 2) t Q(t) with t = 1 / (1 + 0.32 u): Q is of degree 9, fitted over
// 0 < t <= 1 to the least relative error, 3.2e-8.  20 instructions without a
// branch, erff some 100.
__device__ __forceinline__ float normal_exp(float u) { return __builtin_amdgcn_exp2f(u * u * (-0.5f * kLog2e)); }
__device__ __forceinline__ float normal_tail(float u, float e) {  // e = normal_exp(u)
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.32f, u, 1.0f));
  constexpr float q[10] = {0.12766153f,  0.12766095f, 0.11462236f,  0.0878291f,  0.05865397f,
                           -0.00937758f, 0.06532805f, -0.14670749f, 0.09540728f, -0.02107818f};
  float p = q[9];
#pragma unroll
  for (int i = 8; i >= 0; i--) p = __builtin_fmaf(p, t, q[i]);
  return p * t * e;
}
__device__ __forceinline__ float normal_tail(float u) { return normal_tail(u, normal_exp(u)); }

// exp(-|v|) does not overflow.  Within 8 x 2^-24 of the result (v times the
// hardware's reciprocal and exponential alone: 62 x 2^-24 at v = -85).
__device__ __forceinline__ float silu(float v) {
  const float e = exp_of(-fabsf(v));
  return (v >= 0.0f ? v : v * e) / (1.0f + e);
}

// N values at once: one branch for all, and their chains run side by side
// (value by value, GELU took 7 of the 16 us of 80 x 843 x 256).
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  if (act == QUASAR_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = v[i] < 0.0f ? 0.0f : v[i];  // NaN stays
  } else if (act == QUASAR_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = silu(v[i]);
  } else if (act == QUASAR_ACT_GELU) {  // no cancellation for v < 0; at infinity as v (1 + erf) / 2 is
    float tail[N];
#pragma unroll
    for (int i = 0; i < N; i++) tail[i] = normal_tail(fabsf(v[i]));
#pragma unroll
    for (int i = 0; i < N; i++) {
      const float p = fabsf(v[i]) * tail[i];
      v[i] = v[i] > 0.0f ? v[i] - (tail[i] > 0.0f ? p : 0.0f) : -p;
    }
  }
}

// ---- tiles of large products ----------------------------------------------------
// 16 bytes per lane from global memory straight into LDS: lane l's go from
// from + off to to + 16 l (from and to: the same in every lane).  In assembly
// because the compiler makes every later LDS read wait for all such loads in
// flight; the kernel counts them itself (no register is written by them).
__device__ __forceinline__ void load_lds16(const char* from, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from) : "memory");
}

// The place of workgroup b among `total` that are handed out in stretches: each of
// the eight XCDs (workgroup b runs on XCD b % 8) takes neighbours.
__device__ __forceinline__ int stretch_of(int b, int total) {
  const int q = total >> 3, r = total & 7, xcd = b & 7;
  return xcd * q + (xcd < r ? xcd : r) + (b >> 3);
}
// Tile t of tiles_m x tiles_n, counted eight tiles of tokens wide, so that what
// an XCD's workgroups read together fits its L2.
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per = 8 * tiles_n, g = t / per, first = g * 8, wide = tiles_m - first < 8 ? tiles_m - first : 8;
  const int in = t - g * per;
  tm = first + in % wide;
  tn = in / wide;
}
// Tile `b` of a grid as (tm, tn).
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
  tile_at(stretch_of(b, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
}

}  // namespace quasar
