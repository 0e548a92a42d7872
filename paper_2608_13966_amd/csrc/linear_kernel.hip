// linear_kernel.hip -- the product from packed codes (quasar_ops.h):
// y = act(x_scale x r^T + bias) + residual with r formed from the codes.
//
// r is the bf16 reconstruction, bit for bit the one a layer was trained with:
// every form below makes the same 16-bit weights and accumulates exact bf16
// products in fp32 matrix instructions, so a token's result does not depend on
// how many others are in the call but for the order of the fp32 sums.
//
//  - few tokens (strip kernel): the codes are what has to be read.  They go
//    from memory to registers, become bf16 there and feed 16x16x32 matrix
//    instructions directly; nothing is written but y.
//  - many tokens (tile kernel): r is written out once in bf16 (unpack kernel),
//    then multiplied in LDS-staged tiles.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

struct Weights {  // what r is made from
  const uint8_t* codes;
  const void* scales;
  const float* zeros;
  const float* tensor_scale;
  int64_t rows, cols;
  int group;
};

// 32 consecutive weights of one row from element k on (k % 32 == 0), n of
// which exist (n >= 32: all; less only at a row's end: 16 for NVFP4, or <= 0,
// none).  load() issues the loads, chunk(i) gives weights 8i .. 8i+7 in bf16,
// 0 where none exists.
template <int FMT, int BITS>
struct Strip {
  uint32_t d[BITS];    // the codes: 32 * BITS bits
  float s[2], z;       // NVFP4: the scales of the two blocks
  uint32_t book[2];    // RUBIN: the eight E4M3 entries
  int n;

  __device__ __forceinline__ void load(const Weights& w, int64_t row, int k, int left) {
    n = left;
    s[0] = s[1] = z = 0.0f;
#pragma unroll
    for (int i = 0; i < BITS; i++) d[i] = 0u;
    if (n <= 0) return;
    if constexpr (FMT == QUASAR_RUBIN_INT3) {
      const int64_t block = (row >> 3) * (w.cols >> 6) + (k >> 6);
      const uint8_t* p = w.codes + block * 192 + (row & 7) * 24 + ((k & 63) >> 5) * 12;
      __builtin_memcpy(d, p, 12);
      const uint2 b = ld8_any(reinterpret_cast<const uint8_t*>(w.scales) + block * 8);
      book[0] = b.x;
      book[1] = b.y;
    } else {
      const uint8_t* p = w.codes + (row * w.cols + k) * BITS / 8;
      if (FMT != QUASAR_NVFP4 || n >= 32)
        __builtin_memcpy(d, p, 4 * BITS);
      else
        __builtin_memcpy(d, p, 8);
      if constexpr (FMT == QUASAR_NVFP4) {
        const uint8_t* e = reinterpret_cast<const uint8_t*>(w.scales) + row * (w.cols >> 4) + (k >> 4);
        const float st = w.tensor_scale[0];
        s[0] = st * __builtin_amdgcn_cvt_f32_fp8((int)e[0], 0);
        if (n >= 32) s[1] = st * __builtin_amdgcn_cvt_f32_fp8((int)e[1], 0);
      } else {
        const int64_t g = row * (w.cols / w.group) + k / w.group;
        s[0] = reinterpret_cast<const float*>(w.scales)[g];
        // symmetric codes are offset by 2^(b-1): s q = fma(s, q + 2^(b-1), -2^(b-1) s), rounded once either way
        z = FMT == QUASAR_INT ? w.zeros[g] : s[0] * (float)-(1 << (BITS - 1));
      }
    }
  }

  __device__ __forceinline__ uint4 chunk(int i) const {
    uint32_t o[4];
    if constexpr (FMT == QUASAR_NVFP4) {
      const float f = i < 2 ? s[0] : s[1];
#define QUASAR_E2M1(J)                                                              \
  {                                                                                 \
    const auto q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d[i], 1.0f, J);         \
    o[J] = pack_bf16x2(q[0] * f, q[1] * f);                                         \
  }
      QUASAR_E2M1(0) QUASAR_E2M1(1) QUASAR_E2M1(2) QUASAR_E2M1(3)
#undef QUASAR_E2M1
    } else if constexpr (FMT == QUASAR_RUBIN_INT3) {
      const uint32_t v = bits24(i);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const uint32_t u = v >> (12 * h);
        const uint32_t sel = (u & 7u) | ((u << 5) & 0x700u) | ((u << 10) & 0x70000u) | ((u << 15) & 0x7000000u);
        const int b = (int)__builtin_amdgcn_perm(book[1], book[0], sel);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(b, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(b, true);
        o[2 * h] = pack_bf16x2(lo[0], lo[1]);
        o[2 * h + 1] = pack_bf16x2(hi[0], hi[1]);
      }
      if (n <= 0) o[0] = o[1] = o[2] = o[3] = 0u;
    } else {
      float q[8];
      if constexpr (BITS == 4) {
        const uint32_t c = FMT == QUASAR_INT ? d[i] : d[i] ^ 0x88888888u;
        const uint32_t e = c & 0x0f0f0f0fu, f = (c >> 4) & 0x0f0f0f0fu;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          q[2 * j] = (float)((e >> (8 * j)) & 0xffu);
          q[2 * j + 1] = (float)((f >> (8 * j)) & 0xffu);
        }
      } else if constexpr (BITS == 2) {
        const uint32_t c = (FMT == QUASAR_INT ? d[i >> 1] : d[i >> 1] ^ 0xaaaaaaaau);
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const uint32_t m = (c >> (2 * j)) & 0x03030303u;
          q[j] = (float)((m >> (16 * (i & 1))) & 0xffu);
          q[4 + j] = (float)((m >> (16 * (i & 1) + 8)) & 0xffu);
        }
      } else {
        const uint32_t c = FMT == QUASAR_INT ? bits24(i) : bits24(i) ^ 0x924924u;
#pragma unroll
        for (int j = 0; j < 8; j++) q[j] = (float)((c >> (3 * j)) & 7u);
      }
#pragma unroll
      for (int j = 0; j < 4; j++)
        o[j] = pack_bf16x2(__builtin_fmaf(s[0], q[2 * j], z), __builtin_fmaf(s[0], q[2 * j + 1], z));
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }

  // bits 24 i .. 24 i + 23 of a 3-bit strip
  __device__ __forceinline__ uint32_t bits24(int i) const {
    if (i == 0) return d[0] & 0xffffffu;
    if (i == 1) return ((d[0] >> 24) | (d[1] << 8)) & 0xffffffu;
    if (i == 2) return ((d[1] >> 16) | (d[BITS - 1] << 16)) & 0xffffffu;
    return d[BITS - 1] >> 8;
  }
};

// Eight activations from element e of x in bf16.
template <int XT>
__device__ __forceinline__ uint4 load_x8(const void* x, int64_t e) {
  if constexpr (XT == kElemBF16) {
    return ld16_any(reinterpret_cast<const uint16_t*>(x) + e);
  } else {
    const uint2 b = ld8_any(reinterpret_cast<const uint8_t*>(x) + e);
    const auto p = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.x, false), q = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.x, true);
    const auto r = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.y, false), t = __builtin_amdgcn_cvt_pk_f32_fp8((int)b.y, true);
    return make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(q[0], q[1]), pack_bf16x2(r[0], r[1]),
                      pack_bf16x2(t[0], t[1]));
  }
}

__device__ __forceinline__ float activate(float v, int act) {
  if (act == QUASAR_ACT_RELU) return v < 0.0f ? 0.0f : v;  // NaN stays
  if (act == QUASAR_ACT_SILU) return v / (1.0f + __builtin_amdgcn_exp2f(-v * kLog2e));
  if (act == QUASAR_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752440f));
  return v;
}

// ---- few tokens ---------------------------------------------------------------
// A workgroup makes 16 outputs of r's rows for TT * 16 tokens; its wavefronts
// split the columns in steps of 128 and meet in LDS.  The lane of row l % 16
// and quarter l / 16 decodes the 32 weights of its quarter of a step; matrix
// instruction i takes the eighths i of all four quarters, x likewise (the
// order of the columns inside a sum is free).
constexpr int kStripWaves = 8;
template <int FMT, int BITS, int XT, int TT>
__global__ __launch_bounds__(64 * kStripWaves) void strip_kernel(Weights w, quasar_linear a) {
  __shared__ float red[kStripWaves][TT][4][64];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int r16 = lane & 15, quarter = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t t0 = (int64_t)blockIdx.y * (16 * TT);
  const int64_t row = n0 + r16 < w.rows ? n0 + r16 : w.rows - 1;
  const int K = (int)w.cols, steps = (K + 127) / 128, per = (steps + kStripWaves - 1) / kStripWaves;
  const int s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
  int64_t xe[TT];
#pragma unroll
  for (int t = 0; t < TT; t++) {
    const int64_t token = t0 + 16 * t + r16;
    xe[t] = (token < a.tokens ? token : a.tokens - 1) * a.x_stride;
  }
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; t++) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
  for (int s = s0; s < s1; s++) {
    const int k = s * 128 + quarter * 32;
    Strip<FMT, BITS> strip;
    strip.load(w, row, k, K - k);
    uint4 x[TT][4];
#pragma unroll
    for (int t = 0; t < TT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        x[t][i] = make_uint4(0u, 0u, 0u, 0u);
        if (k + 8 * i < K) x[t][i] = load_x8<XT>(a.x, xe[t] + k + 8 * i);
      }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const bf16x8 r = as_bf16x8(strip.chunk(i));
#pragma unroll
      for (int t = 0; t < TT; t++)
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r, as_bf16x8(x[t][i]), acc[t], 0, 0, 0);
    }
  }
#pragma unroll
  for (int t = 0; t < TT; t++)
#pragma unroll
    for (int i = 0; i < 4; i++) red[wave][t][i][lane] = acc[t][i];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * TT; o += 64 * kStripWaves) {
    const int n = o & 15, t = o >> 4;
    const int64_t token = t0 + t;
    if (n0 + n >= w.rows || token >= a.tokens) continue;
    float v = 0.0f;
#pragma unroll
    for (int q = 0; q < kStripWaves; q++) v += red[q][t >> 4][n & 3][(n >> 2) * 16 + (t & 15)];
    if (a.x_scale) v *= a.x_scale[token];
    if (a.bias) v += elem(a.bias, n0 + n, a.bias_dtype == QUASAR_BF16);
    v = activate(v, a.act);
    if (a.residual) v += elem(a.residual, token * a.residual_stride + n0 + n, a.residual_dtype == QUASAR_BF16);
    put_elem(a.y, token * a.y_stride + n0 + n, v, a.y_dtype == QUASAR_BF16);
  }
}

// ---- many tokens --------------------------------------------------------------
constexpr int kTileK = 64;  // columns a tile step takes: 128 bytes of a row

// r in bf16 [rows, kp], columns past the last zero; then (workgroups from
// weight_blocks on) x in bf16 [tokens, kp] likewise, where it is not used as
// it is.  A thread makes 32 weights, or 8 activations.
template <int FMT, int BITS, int XT>
__global__ __launch_bounds__(256) void unpack_kernel(Weights w, quasar_linear a, int kp, uint16_t* r, uint16_t* xo,
                                                     unsigned weight_blocks) {
  if (blockIdx.x < weight_blocks) {
    const int per = kp / 32;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / per;
    if (row >= w.rows) return;
    const int k = (int)(i - row * per) * 32;
    Strip<FMT, BITS> strip;
    const int left = (int)w.cols - k;
    strip.load(w, row, k, left);
#pragma unroll
    for (int c = 0; c < 4; c++) st128(r + row * kp + k + 8 * c, 8 * c < left ? strip.chunk(c) : make_uint4(0u, 0u, 0u, 0u));
  } else {
    const int per = kp / 8;
    const int64_t i = (int64_t)(blockIdx.x - weight_blocks) * 256 + threadIdx.x;
    const int64_t t = i / per;
    if (t >= a.tokens) return;
    const int k = (int)(i - t * per) * 8;
    st128(xo + t * kp + k, k < w.cols ? load_x8<XT>(a.x, t * a.x_stride + k) : make_uint4(0u, 0u, 0u, 0u));
  }
}

// 16 bytes per lane from global memory straight into LDS: lane l's go to
// to + 16 l (to: the same in every lane).
__device__ __forceinline__ void load_lds16(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// A workgroup makes BM tokens x BN outputs, WM x WN wavefronts of 32x32x16
// matrix instructions; LDS holds two steps of both operands, one filled while
// the other is used.  Row m's 16-byte chunk c of a step lies at chunk
// c ^ (m / 2 % 8) of its 128 bytes: the 32 rows that an operand read touches
// then spread over all banks.
template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(quasar_linear a, const uint16_t* x, int64_t x_stride,
                                                            const uint16_t* r, int64_t rows, int kp, int tiles_m,
                                                            int tiles_n) {
  constexpr int kWavesT = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kStage = (BM + BN) * kTileK;  // bf16 elements
  extern __shared__ __align__(16) uint16_t lds[];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int wm = wave / WN, wn = wave % WN;
  const int tm = blockIdx.x % (unsigned)tiles_m, tn = blockIdx.x / (unsigned)tiles_m;
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;

  // this lane's rows of the loads: 8 rows of 128 bytes a wavefront and instruction
  constexpr int kLoads = (BM + BN) / 8 / kWavesT;
  const char* src[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; i++) {
    const int lr = (wave * kLoads + i) * 8 + (lane >> 3);
    const int c = (lane & 7) ^ ((lr >> 1) & 7);
    const int64_t m = m0 + lr, n = n0 + lr - BM;
    src[i] = lr < BM ? reinterpret_cast<const char*>(x + (m < a.tokens ? m : a.tokens - 1) * x_stride) + 16 * c
                     : reinterpret_cast<const char*>(r + (n < rows ? n : rows - 1) * kp) + 16 * c;
  }
  const auto fill = [&](int stage) {
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
      load_lds16(src[i], lds + stage * kStage + (wave * kLoads + i) * 8 * kTileK);
      src[i] += 2 * kTileK;
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

  fill(0);
  const int steps = kp / kTileK;
  for (int s = 0; s < steps; s++) {
    // step s has landed, and every wavefront is done with step s - 1
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (s + 1 < steps) fill((s + 1) & 1);
    const uint16_t* as = lds + (s & 1) * kStage;
    const uint16_t* bs = as + BM * kTileK;
#pragma unroll
    for (int k = 0; k < kTileK / 16; k++) {
      bf16x8 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; i++) {
        const int m = wm * (BM / WM) + i * 32 + (lane & 31);
        fa[i] = as_bf16x8(*reinterpret_cast<const uint4*>(as + m * kTileK + 8 * ((2 * k + (lane >> 5)) ^ ((m >> 1) & 7))));
      }
#pragma unroll
      for (int j = 0; j < TN; j++) {
        const int n = wn * (BN / WN) + j * 32 + (lane & 31);
        fb[j] = as_bf16x8(*reinterpret_cast<const uint4*>(bs + n * kTileK + 8 * ((2 * k + (lane >> 5)) ^ ((n >> 1) & 7))));
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  }
  // The epilogue goes through LDS (each wavefront its own part of it), 32
  // tokens at a time, so that y is written 16 bytes a lane.
  __syncthreads();
  constexpr int kCols = BN / WN, kPitch = kCols + 4;
  static_assert(32 * kPitch * 4 * kWavesT <= 2 * kStage * 2, "the epilogue's stage fits the tiles'");
  float* st = reinterpret_cast<float*>(lds) + wave * 32 * kPitch;
  const bool yb = a.y_dtype == QUASAR_BF16;
#pragma unroll
  for (int i = 0; i < TM; i++) {
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++)
        st[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * kPitch + j * 32 + (lane & 31)] = acc[i][j][e];
    wave_lds_fence();
    constexpr int kLanes = kCols / 8;  // lanes a token's outputs take
#pragma unroll 1
    for (int p = 0; p < 32; p += 64 / kLanes) {
      const int tr = p + lane / kLanes, c = (lane % kLanes) * 8;
      const int64_t token = m0 + wm * (BM / WM) + i * 32 + tr, n = n0 + wn * kCols + c;
      if (token >= a.tokens || n >= rows) continue;
      const int left = (int)(rows - n < 8 ? rows - n : 8);
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] = st[tr * kPitch + c + q];
      if (a.x_scale) {
        const float f = a.x_scale[token];
#pragma unroll
        for (int q = 0; q < 8; q++) v[q] *= f;
      }
      const auto add = [&](const void* p, int64_t e, bool bf16) {
        if (bf16) {
          Piece<kElemBF16> b;
          b.load(p, e, left);
#pragma unroll
          for (int q = 0; q < 8; q++) v[q] += b.get(q);
        } else {
          Piece<kElemF32> b;
          b.load(p, e, left);
#pragma unroll
          for (int q = 0; q < 8; q++) v[q] += b.get(q);
        }
      };
      if (a.bias) add(a.bias, n, a.bias_dtype == QUASAR_BF16);
      if (a.act != QUASAR_ACT_NONE) {
#pragma unroll
        for (int q = 0; q < 8; q++) v[q] = activate(v[q], a.act);
      }
      if (a.residual) add(a.residual, token * a.residual_stride + n, a.residual_dtype == QUASAR_BF16);
      store_piece(a.y, token * a.y_stride + n, v, left, yb);
    }
    wave_lds_fence();
  }
}

constexpr int64_t kStripTokens = 64;  // the strip kernel serves up to this many

int padded_cols(const quasar_desc& d) { return (int)((d.cols + kTileK - 1) / kTileK * kTileK); }

// x goes through the workspace unless the tile kernel can load its rows in
// 16-byte pieces as they are.
bool x_direct(int64_t cols, int x_dtype, const void* x, int64_t stride) {
  return x_dtype == QUASAR_BF16 && cols % kTileK == 0 && stride % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
}

template <int FMT, int BITS, int XT>
hipError_t launch(const quasar_desc& d, const quasar_linear& a, hipStream_t stream) {
  Weights w{a.codes, a.scales, a.zeros, a.tensor_scale, d.rows, d.cols, FMT == QUASAR_NVFP4 ? 16 : d.group};
  if (a.tokens <= kStripTokens) {
    const dim3 block(64 * kStripWaves);
    const unsigned gx = (unsigned)((d.rows + 15) / 16);
    if (a.tokens <= 16)
      strip_kernel<FMT, BITS, XT, 1><<<dim3(gx), block, 0, stream>>>(w, a);
    else if (a.tokens <= 32)
      strip_kernel<FMT, BITS, XT, 2><<<dim3(gx), block, 0, stream>>>(w, a);
    else
      strip_kernel<FMT, BITS, XT, 4><<<dim3(gx), block, 0, stream>>>(w, a);
    return hipGetLastError();
  }
  const int kp = padded_cols(d);
  uint16_t* r = reinterpret_cast<uint16_t*>(a.workspace);
  uint16_t* xo = r + d.rows * kp;
  const bool direct = x_direct(d.cols, a.x_dtype, a.x, a.x_stride);
  const int64_t wb = (d.rows * (kp / 32) + 255) / 256, xb = direct ? 0 : (a.tokens * (kp / 8) + 255) / 256;
  unpack_kernel<FMT, BITS, XT><<<dim3((unsigned)(wb + xb)), dim3(256), 0, stream>>>(w, a, kp, r, xo, (unsigned)wb);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int BM = 128, BN = 128;
  const int tm = (int)((a.tokens + BM - 1) / BM), tn = (int)((d.rows + BN - 1) / BN);
  tile_kernel<BM, BN, 2, 2><<<dim3((unsigned)(tm * tn)), dim3(256), 2 * (BM + BN) * kTileK * 2, stream>>>(
      a, direct ? reinterpret_cast<const uint16_t*>(a.x) : xo, direct ? a.x_stride : kp, r, d.rows, kp, tm, tn);
  return hipGetLastError();
}

template <int FMT, int BITS>
hipError_t launch_x(const quasar_desc& d, const quasar_linear& a, hipStream_t stream) {
  return a.x_dtype == QUASAR_BF16 ? launch<FMT, BITS, kElemBF16>(d, a, stream) : launch<FMT, BITS, kElemE4M3>(d, a, stream);
}

}  // namespace

size_t linear_workspace(const quasar_desc& d, int64_t tokens, int x_dtype) {
  (void)x_dtype;
  if (tokens <= kStripTokens) return 0;
  const size_t kp = (size_t)padded_cols(d);
  return ((size_t)d.rows + (size_t)tokens) * kp * 2;
}

hipError_t launch_linear(const quasar_desc& d, const quasar_linear& a, hipStream_t stream) {
  switch (d.format) {
    case QUASAR_INT:
      return d.bits == 2   ? launch_x<QUASAR_INT, 2>(d, a, stream)
             : d.bits == 3 ? launch_x<QUASAR_INT, 3>(d, a, stream)
                           : launch_x<QUASAR_INT, 4>(d, a, stream);
    case QUASAR_INT_SYM:
      return d.bits == 2   ? launch_x<QUASAR_INT_SYM, 2>(d, a, stream)
             : d.bits == 3 ? launch_x<QUASAR_INT_SYM, 3>(d, a, stream)
                           : launch_x<QUASAR_INT_SYM, 4>(d, a, stream);
    case QUASAR_NVFP4: return launch_x<QUASAR_NVFP4, 4>(d, a, stream);
    default: return launch_x<QUASAR_RUBIN_INT3, 3>(d, a, stream);
  }
}

}  // namespace quasar
