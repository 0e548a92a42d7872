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
//  - more (fused kernel): r is formed in LDS, a tile's step at a time.
//  - many (tile kernel): r is written out once in bf16 (unpack kernel), then
//    multiplied in LDS-staged tiles.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

// fma(s, v, z) in fp32, v the fp16 number in the low or high half of x.  A code
// q at bit o of a half (q 2^o < 2^10) is the subnormal q 2^(o - 24), which the
// instruction takes exactly: with s 2^(24 - o) in s's place it is fma(s, q, z)
// without a conversion.
template <bool HIGH>
__device__ __forceinline__ float fma_half(float s, uint32_t x, float z) {
  float r;
  if constexpr (HIGH)
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,1,0] op_sel_hi:[0,1,0]" : "=v"(r) : "v"(s), "v"(x), "v"(z));
  else
    asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel_hi:[0,1,0]" : "=v"(r) : "v"(s), "v"(x), "v"(z));
  return r;
}

// Two E4M3 bytes (of the low or the high half of x) as packed bf16; exact.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t x) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HIGH));
}

struct Weights {  // what r is made from
  const uint8_t* codes;
  const void* scales;
  const float* zeros;
  const float* tensor_scale;
  int64_t rows, cols;
  int shift;  // a group is 2^shift columns (INT)
};

// floats from one token's partial sums to the next one's: whole pieces, aligned
__host__ __device__ constexpr int64_t part_pitch(int64_t rows) { return (rows + 7) & ~(int64_t)7; }

// Where one row's codes and parameters lie.
template <int FMT, int BITS>
struct WeightRow {
  const uint8_t* codes;
  const uint8_t* scales;
  const float* zeros;
  float tensor_scale;
  int shift;

  __device__ __forceinline__ WeightRow(const Weights& w, int64_t row) {
    shift = w.shift;
    if constexpr (FMT == QUASAR_RUBIN_INT3) {
      const int64_t block = (row >> 3) * (w.cols >> 6);
      codes = w.codes + block * 192 + (row & 7) * 24;
      scales = reinterpret_cast<const uint8_t*>(w.scales) + block * 8;
    } else if constexpr (FMT == QUASAR_NVFP4) {
      codes = w.codes + row * (w.cols >> 1);
      scales = reinterpret_cast<const uint8_t*>(w.scales) + row * (w.cols >> 4);
      tensor_scale = w.tensor_scale[0];
    } else {
      const int64_t g = row * (w.cols >> w.shift);
      codes = w.codes + row * (w.cols >> 3) * BITS;
      scales = reinterpret_cast<const uint8_t*>(w.scales) + 4 * g;
      if constexpr (FMT == QUASAR_INT) zeros = w.zeros + g;
    }
  }
};

// 32 consecutive weights of one row from element k on (k % 32 == 0), n of
// which exist (n >= 32: all; less only at a row's end: 16 for NVFP4, or <= 0,
// none).  load() issues the loads, ready() follows before the first chunk();
// chunk(i) gives weights 8i .. 8i+7 in bf16, 0 where none exists.
template <int FMT, int BITS>
struct Strip {
  static constexpr int kOffsets = 10 / BITS;  // codes of a half that are subnormals where they are
  uint32_t d[BITS];    // the codes: 32 * BITS bits
  uint32_t p[2];       // the parameters as loaded: s and z, the two E4M3 scales, or the eight E4M3 entries
  float s[5], z;       // INT: s 2^(24 - BITS i) and z; NVFP4: the blocks' scales

  // all 32 exist
  __device__ __forceinline__ void load(const WeightRow<FMT, BITS>& w, int k) {
    if constexpr (FMT == QUASAR_RUBIN_INT3) {
      __builtin_memcpy(d, w.codes + (k >> 6) * 192 + ((k >> 5) & 1) * 12, 12);
      __builtin_memcpy(p, w.scales + (k >> 6) * 8, 8);
    } else {
      __builtin_memcpy(d, w.codes + (k >> 3) * BITS, 4 * BITS);
      if constexpr (FMT == QUASAR_NVFP4) {
        uint16_t e;
        __builtin_memcpy(&e, w.scales + (k >> 4), 2);
        p[0] = e;
      } else {
        const int g = k >> w.shift;
        p[0] = reinterpret_cast<const uint32_t*>(w.scales)[g];
        p[1] = FMT == QUASAR_INT ? as_u32(w.zeros[g]) : 0u;
      }
    }
  }
  __device__ __forceinline__ void load(const WeightRow<FMT, BITS>& w, int k, int n) {
    p[0] = p[1] = 0u;
#pragma unroll
    for (int i = 0; i < BITS; i++) d[i] = 0u;
    if (n >= 32) {
      load(w, k);
    } else if (FMT == QUASAR_NVFP4 && n > 0) {
      __builtin_memcpy(d, w.codes + (k >> 1), 8);
      p[0] = w.scales[k >> 4];
    }
  }

  __device__ __forceinline__ void ready(float tensor_scale) {
    if constexpr (FMT == QUASAR_NVFP4) {
      s[0] = tensor_scale * __builtin_amdgcn_cvt_f32_fp8((int)p[0], 0);
      s[1] = tensor_scale * __builtin_amdgcn_cvt_f32_fp8((int)p[0], 1);
    } else if constexpr (FMT != QUASAR_RUBIN_INT3) {
      const float f = as_f32(p[0]);
      // symmetric codes are offset by 2^(b-1): s q = fma(s, q + 2^(b-1), -2^(b-1) s), rounded once either way
      z = FMT == QUASAR_INT_SYM ? f * (float)-(1 << (BITS - 1)) : as_f32(p[1]);
#pragma unroll
      for (int i = 0; i < kOffsets; i++) s[i] = f * (float)(1 << (24 - BITS * i));
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
        const uint32_t b = __builtin_amdgcn_perm(p[1], p[0], sel);
        o[2 * h] = e4m3_bf16<false>(b);
        o[2 * h + 1] = e4m3_bf16<true>(b);
      }
    } else {
      float v[8];
      if constexpr (BITS == 4) {
        const uint32_t c = FMT == QUASAR_INT ? d[i] : d[i] ^ 0x88888888u;
        pair<0>(c, v[0], v[4]);
        pair<1>(c, v[1], v[5]);
        pair<0>(c >> 8, v[2], v[6]);
        pair<1>(c >> 8, v[3], v[7]);
      } else if constexpr (BITS == 2) {
        // chunk 2 j is the low halves of dword j's, chunk 2 j + 1 the high ones
        const uint32_t c = FMT == QUASAR_INT ? d[i >> 1] : d[i >> 1] ^ 0xaaaaaaaau;
        if (i & 1) {
          half<0, true>(c, v[0]); half<1, true>(c, v[1]); half<2, true>(c, v[2]); half<3, true>(c, v[3]);
          half<4, true>(c, v[4]); half<0, true>(c >> 10, v[5]); half<1, true>(c >> 10, v[6]); half<2, true>(c >> 10, v[7]);
        } else {
          half<0, false>(c, v[0]); half<1, false>(c, v[1]); half<2, false>(c, v[2]); half<3, false>(c, v[3]);
          half<4, false>(c, v[4]); half<0, false>(c >> 10, v[5]); half<1, false>(c >> 10, v[6]); half<2, false>(c >> 10, v[7]);
        }
      } else {
        const uint32_t c = FMT == QUASAR_INT ? bits24(i) : bits24(i) ^ 0x924924u;
        const uint32_t e = (c & 0x7fffu) | ((c >> 15) << 16);  // codes 0 .. 4, and 5 .. 7 from bit 16 on
        pair<0>(e, v[0], v[5]);
        pair<1>(e, v[1], v[6]);
        pair<2>(e, v[2], v[7]);
        half<0, false>(e >> 9, v[3]);
        half<1, false>(e >> 9, v[4]);
      }
#pragma unroll
      for (int j = 0; j < 4; j++) o[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }

  // the weights of the codes that lie J codes from bit 0 of the halves of c
  template <int J>
  static constexpr uint32_t kMask = ((1u << BITS) - 1u) << (BITS * J) | ((1u << BITS) - 1u) << (BITS * J + 16);
  template <int J>
  __device__ __forceinline__ void pair(uint32_t c, float& lo, float& hi) const {
    lo = fma_half<false>(s[J], c & kMask<J>, z);
    hi = fma_half<true>(s[J], c & kMask<J>, z);
  }
  template <int J, bool HIGH>
  __device__ __forceinline__ void half(uint32_t c, float& v) const {
    v = fma_half<HIGH>(s[J], c & kMask<J>, z);
  }

  // bits 24 i .. 24 i + 23 of a 3-bit strip
  __device__ __forceinline__ uint32_t bits24(int i) const {
    if (i == 0) return d[0] & 0xffffffu;
    if (i == 1) return ((d[0] >> 24) | (d[1] << 8)) & 0xffffffu;
    if (i == 2) return ((d[1] >> 16) | (d[BITS - 1] << 16)) & 0xffffffu;
    return d[BITS - 1] >> 8;
  }
};

// Eight activations as fetched, and in bf16; all 0 where `has` is false.
template <int XT>
struct XChunk {
  uint32_t d[XT == kElemBF16 ? 4 : 2];
  __device__ __forceinline__ void load(const void* x, int64_t e) {
    if constexpr (XT == kElemBF16) {
      const uint4 t = ld16_any(reinterpret_cast<const uint16_t*>(x) + e);
      d[0] = t.x; d[1] = t.y; d[2] = t.z; d[3] = t.w;
    } else {
      const uint2 t = ld8_any(reinterpret_cast<const uint8_t*>(x) + e);
      d[0] = t.x; d[1] = t.y;
    }
  }
  __device__ __forceinline__ void load(const void* x, int64_t e, bool has) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(d) / 4); i++) d[i] = 0u;
    if (has) load(x, e);
  }
  __device__ __forceinline__ uint4 bf16() const {
    if constexpr (XT == kElemBF16) {
      return make_uint4(d[0], d[1], d[2], d[3]);
    } else {
      return make_uint4(e4m3_bf16<false>(d[0]), e4m3_bf16<true>(d[0]), e4m3_bf16<false>(d[1]), e4m3_bf16<true>(d[1]));
    }
  }
};

// ---- few tokens ---------------------------------------------------------------
// The codes and parameters of 16 rows x 128 columns in LDS, and how a
// wavefront brings them there: a lane's load is a 16-byte piece whose
// neighbours in memory are its neighbours' (loaded in the order in which the
// matrix instruction wants them, every lane's would be a cache access of its
// own: that took twice as long at one token).
template <int FMT, int BITS>
struct Block16 {
  static constexpr bool kRubin = FMT == QUASAR_RUBIN_INT3, kNv = FMT == QUASAR_NVFP4;
  static constexpr int kPieces = 16 * BITS;  // 16-byte pieces of codes
  static constexpr int kBytes = 16 * kPieces + 256;

  // Of the 16 rows from n0 on: where they lie (the same in every lane), and
  // this lane's piece and parameters from there.
  struct Place {
    const uint8_t *codes, *par, *zero;
    uint32_t piece, first;  // bytes
    int at;                 // LDS offset of the piece
    int shift;              // a group is 2^shift columns (INT)
    float tensor_scale;

    __device__ __forceinline__ Place(const Weights& w, int64_t n0, int lane) {
      shift = w.shift;
      const int last = (int)(w.rows - 1 - n0 < 15 ? w.rows - 1 - n0 : 15);  // rows past the matrix: its last one's
      if constexpr (kRubin) {
        const int b = lane / 12, i = lane - 12 * b;
        const uint32_t wide = (uint32_t)(w.cols >> 6);
        codes = w.codes + (n0 >> 3) * (w.cols >> 6) * 192;
        par = reinterpret_cast<const uint8_t*>(w.scales) + (n0 >> 3) * (w.cols >> 6) * 8;
        piece = (((b >> 1) & (last >> 3)) * wide + (b & 1)) * 192 + 16 * i;
        first = (((lane >> 1) & (last >> 3)) * wide + (lane & 1)) * 8;
        at = b * 192 + 16 * i;
      } else {
        const int r = BITS == 4 ? lane >> 2 : BITS == 2 ? lane >> 1 : lane / 3, i = lane - r * BITS;
        codes = w.codes + n0 * (w.cols >> 3) * BITS;
        piece = (uint32_t)(r < last ? r : last) * (uint32_t)(w.cols >> 3) * BITS + 16 * i;
        // four pieces a row: rows 4 apart use other banks
        at = BITS == 4 ? 64 * r + 16 * (i ^ ((r >> 2) & 3)) : (r * BITS + i) * 16;
        if constexpr (kNv) {
          par = reinterpret_cast<const uint8_t*>(w.scales) + n0 * (w.cols >> 4);
          first = (uint32_t)((lane & 15) < last ? lane & 15 : last) * (uint32_t)(w.cols >> 4);
          tensor_scale = w.tensor_scale[0];
        } else {
          const int per = 7 - shift, pr = (lane >> per) & 15;
          const int64_t e = n0 * (w.cols >> shift);
          par = reinterpret_cast<const uint8_t*>(w.scales) + 4 * e;
          first = 4 * ((uint32_t)(pr < last ? pr : last) * (uint32_t)(w.cols >> shift) + (lane & per));
          if constexpr (FMT == QUASAR_INT) zero = reinterpret_cast<const uint8_t*>(w.zeros + e);
        }
      }
    }
  };
  uint4 c;
  uint32_t p[2];

  // columns k .. k + 127
  __device__ __forceinline__ void load(const Place& w, int k, int lane) {
    if (kPieces == 64 || lane < kPieces) c = ld16_any(w.codes + (kRubin ? (k >> 6) * 192 : (k >> 3) * BITS) + w.piece);
    if constexpr (kRubin || kNv) {
      if (lane < (kRubin ? 4 : 16)) {
        const uint2 t = ld8_any(w.par + (kRubin ? (k >> 6) * 8 : k >> 4) + w.first);
        p[0] = t.x;
        p[1] = t.y;
      }
    } else if (lane < (16 << (7 - w.shift))) {
      p[0] = *reinterpret_cast<const uint32_t*>(w.par + 4 * (k >> w.shift) + w.first);
      if constexpr (FMT == QUASAR_INT) p[1] = *reinterpret_cast<const uint32_t*>(w.zero + 4 * (k >> w.shift) + w.first);
    }
  }

  __device__ __forceinline__ void put(const Place& w, char* lds, int lane) const {
    if (kPieces == 64 || lane < kPieces) *reinterpret_cast<uint4*>(lds + w.at) = c;
    uint32_t* q = reinterpret_cast<uint32_t*>(lds + 16 * kPieces);
    if constexpr (kRubin || kNv) {
      if (lane < (kRubin ? 4 : 16)) *reinterpret_cast<uint2*>(q + 2 * lane) = make_uint2(p[0], p[1]);
    } else if (lane < (16 << (7 - w.shift))) {
      q[lane] = p[0];
      if constexpr (FMT == QUASAR_INT) q[32 + lane] = p[1];
    }
  }

  // the 32 weights of row r and quarter q
  static __device__ __forceinline__ void get(const Place& w, const char* lds, int r, int q, Strip<FMT, BITS>& o) {
    const char* par = lds + 16 * kPieces;
    if constexpr (kRubin) {
      const int b = (r >> 3) * 2 + (q >> 1);
      const uint32_t* d = reinterpret_cast<const uint32_t*>(lds + b * 192 + (r & 7) * 24 + (q & 1) * 12);
      o.d[0] = d[0]; o.d[1] = d[1]; o.d[2] = d[2];
      const uint2 t = *reinterpret_cast<const uint2*>(par + 8 * b);
      o.p[0] = t.x;
      o.p[1] = t.y;
      o.ready(0.0f);
    } else {
      if constexpr (BITS == 4) {
        const uint4 t = *reinterpret_cast<const uint4*>(lds + 64 * r + 16 * (q ^ ((r >> 2) & 3)));
        o.d[0] = t.x; o.d[1] = t.y; o.d[2] = t.z; o.d[3] = t.w;
      } else if constexpr (BITS == 2) {
        const uint2 t = *reinterpret_cast<const uint2*>(lds + 32 * r + 8 * q);
        o.d[0] = t.x; o.d[1] = t.y;
      } else {
        const uint32_t* d = reinterpret_cast<const uint32_t*>(lds + 48 * r + 12 * q);
        o.d[0] = d[0]; o.d[1] = d[1]; o.d[2] = d[2];
      }
      if constexpr (kNv) {
        o.p[0] = *reinterpret_cast<const uint16_t*>(par + 8 * r + 2 * q);
        o.ready(w.tensor_scale);
      } else {
        const int per = 7 - w.shift, e = (r << per) + ((32 * q) >> w.shift);
        o.p[0] = reinterpret_cast<const uint32_t*>(par)[e];
        o.p[1] = FMT == QUASAR_INT ? reinterpret_cast<const uint32_t*>(par)[32 + e] : 0u;
        o.ready(0.0f);
      }
    }
  }
};

// A workgroup makes 16 NB outputs for up to 4 NX tokens (NX 1, 2, 4, or 8 for 32)
// over its share of the columns (split of 2^log_splits; the shares meet in
// part); its wavefronts split them in steps of 128 and meet in LDS.  The lane
// of row l % 16 and quarter l / 16 decodes the 32 weights of its quarter of a
// step; matrix instruction i takes the eighths i of all four quarters, x
// likewise (the order of the columns inside a sum is free).  Both operands go
// through the wavefront's own part of LDS; the next step's loads are in flight
// meanwhile.  (Two or four steps in flight, or 4 or 16 wavefronts, were up to
// 25% slower at 4096 x 4096 to 14336 x 4096 and 1 to 32 tokens: registers and
// LDS then hold fewer wavefronts.)  4096 x 4096, 4 bits, 1 token: 5.1 us, a
// launch (2.9) and the codes at 4.3 TB/s; 14336 x 4096, 2 bits, 8 tokens of 8 bits: 11.7
// us among others (one by one under a trace 11.6 to 13.4), of which the copy of the codes
// and parameters would be 4.3: bound by the decoding (VALU and LDS) between loads.
constexpr int kStripWaves = 8;
template <int FMT, int BITS, int XT, int NX, int NB>
__global__ __launch_bounds__(64 * kStripWaves) void strip_kernel(Weights w, quasar_linear a, int log_splits, float* part) {
  constexpr int kTokens = 4 * NX, TT = kTokens > 16 ? 2 : 1;
  constexpr int kBlock = Block16<FMT, BITS>::kBytes, kPart = NB * kBlock + kTokens * 256;
  __shared__ __align__(16) char lds[kStripWaves * kPart];
  constexpr int kSums = 64 + 4;  // from one register's sums to the next one's: their readers use all banks
  static_assert(kPart >= NB * TT * 16 * kSums, "the partial sums fit");
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int r16 = lane & 15, quarter = lane >> 4;
  char* const mine = lds + wave * kPart;
  char* const xs = mine + NB * kBlock;
  const int split = blockIdx.x & ((1u << log_splits) - 1u);
  const int64_t n0 = (int64_t)(blockIdx.x >> log_splits) * (16 * NB);
  const auto first = [&](int b) { return n0 + 16 * b < w.rows ? n0 + 16 * b : n0; };  // a block past the matrix: the one before again
  // whole steps, in shares that differ by one at the most; the columns past them are the last share's
  const int K = (int)w.cols, steps = K / 128, log_shares = 3 + log_splits;
  static_assert(kStripWaves == 1 << 3, "shares of a workgroup");
  const int share = split * kStripWaves + wave;
  const int s0 = (int)((uint32_t)steps * share >> log_shares), s1 = (int)((uint32_t)steps * (share + 1) >> log_shares);
  const typename Block16<FMT, BITS>::Place place0(w, n0, lane), place1(w, first(NB - 1), lane);
  const auto place = [&](int b) -> const auto& { return b == 0 ? place0 : place1; };
  struct Fetched {
    Block16<FMT, BITS> w[NB];
    XChunk<XT> x[NX];
  } f = {};
  // x: 8 columns a lane, 16 lanes a token; NX times 4 tokens
  const int kk = lane & 15, tokens = (int)a.tokens;
  int64_t xe[NX];  // tokens past the last are not read: they only reach outputs that are not stored
#pragma unroll
  for (int i = 0; i < NX; i++) xe[i] = (4 * i + (lane >> 4)) * a.x_stride + 8 * kk;
  const auto fetch = [&](Fetched& o, int s) {
#pragma unroll
    for (int b = 0; b < NB; b++) o.w[b].load(place(b), s * 128, lane);
#pragma unroll
    for (int i = 0; i < NX; i++)
      if (4 * i + (lane >> 4) < tokens) o.x[i].load(a.x, xe[i] + s * 128);
  };
  f32x4 acc[NB][TT];
#pragma unroll
  for (int b = 0; b < NB; b++)
#pragma unroll
    for (int t = 0; t < TT; t++) acc[b][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // token t's eighth e of a step lies at chunk e * kTokens + (t ^ e % kTokens): both sides without bank conflicts
  const auto multiply = [&](const Strip<FMT, BITS> (&strip)[NB]) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      bf16x8 r[NB];
#pragma unroll
      for (int b = 0; b < NB; b++) r[b] = as_bf16x8(strip[b].chunk(i));
#pragma unroll
      for (int t = 0; t < TT; t++) {
        const int e = 4 * quarter + i, col = (16 * t + r16) & (kTokens - 1);
        const uint4 x = *reinterpret_cast<const uint4*>(xs + 16 * (e * kTokens + (col ^ (e & (kTokens - 1)))));
#pragma unroll
        for (int b = 0; b < NB; b++)
          acc[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[b], as_bf16x8(x), acc[b][t], 0, 0, 0);
      }
    }
  };
  const auto put_x = [&](int i, const XChunk<XT>& x) {
    const int t = 4 * i + (lane >> 4);
    *reinterpret_cast<uint4*>(xs + 16 * (kk * kTokens + (t ^ (kk & (kTokens - 1))))) = x.bf16();
  };
  if (s0 < s1) fetch(f, s0);
  for (int s = s0; s < s1; s++) {
    wave_lds_fence();
#pragma unroll
    for (int b = 0; b < NB; b++) f.w[b].put(place(b), mine + b * kBlock, lane);
#pragma unroll
    for (int i = 0; i < NX; i++) put_x(i, f.x[i]);
    if (s + 1 < s1) fetch(f, s + 1);
    wave_lds_fence();
    Strip<FMT, BITS> strip[NB];
#pragma unroll
    for (int b = 0; b < NB; b++) Block16<FMT, BITS>::get(place(b), mine + b * kBlock, r16, quarter, strip[b]);
    multiply(strip);
  }
  if (share == (1 << log_shares) - 1 && steps * 128 < K) {
    const int k = steps * 128 + quarter * 32;
    Strip<FMT, BITS> strip[NB];
#pragma unroll
    for (int b = 0; b < NB; b++) {
      const int64_t n = n0 + 16 * b + r16;
      const WeightRow<FMT, BITS> row(w, n < w.rows ? n : w.rows - 1);
      strip[b].load(row, k, K - k);
      strip[b].ready(row.tensor_scale);
    }
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < NX; i++) {
      const int t = 4 * i + (lane >> 4);
      XChunk<XT> x;
      x.load(a.x, t * a.x_stride + steps * 128 + 8 * kk, t < tokens && steps * 128 + 8 * kk < K);
      put_x(i, x);
    }
    wave_lds_fence();
    multiply(strip);
  }
  wave_lds_fence();
  float* const sums = reinterpret_cast<float*>(mine);
#pragma unroll
  for (int b = 0; b < NB; b++)
#pragma unroll
    for (int t = 0; t < TT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) sums[(4 * (b * TT + t) + i) * kSums + lane] = acc[b][t][i];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * TT * NB; o += 64 * kStripWaves) {
    const int n = o & (16 * NB - 1), t = o / (16 * NB);
    if (n0 + n >= w.rows || t >= tokens) continue;
    float sum[1] = {0.0f}, &v = sum[0];
#pragma unroll
    for (int q = 0; q < kStripWaves; q++)
      v += reinterpret_cast<const float*>(lds + q * kPart)[(4 * ((n >> 4) * TT + (t >> 4)) + (n & 3)) * kSums + (n >> 2 & 3) * 16 + (t & 15)];
    if (part) {
      part[((int64_t)split * tokens + t) * part_pitch(w.rows) + n0 + n] = v;
      continue;
    }
    if (a.x_scale) v *= a.x_scale[t];
    if (a.bias) v += elem(a.bias, n0 + n, a.bias_dtype == QUASAR_BF16);
    activate(sum, a.act);
    if (a.residual) v += elem(a.residual, t * a.residual_stride + n0 + n, a.residual_dtype == QUASAR_BF16);
    put_elem(a.y, t * a.y_stride + n0 + n, v, a.y_dtype == QUASAR_BF16);
  }
}

// ---- tiles ----------------------------------------------------------------------
constexpr int kTileK = 64;  // columns a tile step takes: 128 bytes of a row in bf16

// In LDS, 16-byte chunk c of row m of a step lies at chunk c ^ (m / 2 % 8) of
// the row's 128 bytes: the 16 rows that an operand read or a store touches at
// one chunk then lie in 16 different groups of four banks.
__device__ __forceinline__ int chunk_at(int m, int c) { return m * kTileK + 8 * (c ^ ((m >> 1) & 7)); }

// What N tokens need to finish eight neighbouring outputs, from output n on,
// left[i] of which exist (0: none, no such token): asked for at once, ahead of
// the sums.
template <int N>
struct Finish {
  float scale[N], res[N][8];
  __device__ __forceinline__ Finish(const quasar_linear& a, const int64_t (&token)[N], int64_t n, const int (&left)[N]) {
    if (a.x_scale) {
#pragma unroll
      for (int i = 0; i < N; i++) scale[i] = a.x_scale[left[i] > 0 ? token[i] : 0];
    }
    if (a.residual) {
      int64_t e[N];
#pragma unroll
      for (int i = 0; i < N; i++) e[i] = token[i] * a.residual_stride + n;
      load_floats(a.residual, e, left, a.residual_dtype == QUASAR_BF16, res);
    }
  }
  static __device__ __forceinline__ void load_bias(const quasar_linear& a, int64_t n, int left, float (&bias)[8]) {
    if (a.bias) load_floats(a.bias, n, left, a.bias_dtype == QUASAR_BF16, bias);
  }
  // scale, bias, activation, residual, store
  __device__ __forceinline__ void store(const quasar_linear& a, int i, int64_t token, int64_t n, int left,
                                        const float (&bias)[8], float (&v)[8]) const {
    if (a.x_scale) {
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] *= scale[i];
    }
    if (a.bias) {
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] += bias[q];
    }
    activate(v, a.act);
    if (a.residual) {
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] += res[i][q];
    }
    if (left > 0) store_piece(a.y, token * a.y_stride + n, v, left, a.y_dtype == QUASAR_BF16);
  }
};

// A wavefront's tile of 16 TM tokens x 64 outputs from its accumulators
// (acc[i][j][e]: token 16 i + 4 (lane / 16) + e, output 16 j + lane % 16), 32
// tokens at a time through its part `st` of LDS (kSlab floats), so that y is
// written 16 bytes a lane.  part: the sums go there [tokens, part_pitch] instead.
constexpr int kSlabPitch = 64 + 4, kSlab = 32 * kSlabPitch;
template <int TM>
__device__ __forceinline__ void store_tile(const quasar_linear& a, int64_t rows, const f32x4 (&acc)[TM][4], int64_t m0,
                                           int64_t n0, float* st, float* part) {
  const int lane = threadIdx.x & 63, c = (lane & 7) * 8;
  const int64_t n = n0 + c;
  const int some = (int)(rows - n < 0 ? 0 : rows - n < 8 ? rows - n : 8);
  float bias[8];
  if (!part) Finish<2>::load_bias(a, n, some, bias);
#pragma unroll
  for (int s = 0; s < TM / 2; s++) {
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 4; j++)
#pragma unroll
        for (int e = 0; e < 4; e++)
          st[(16 * i + 4 * (lane >> 4) + e) * kSlabPitch + 16 * j + (lane & 15)] = acc[2 * s + i][j][e];
    wave_lds_fence();
#pragma unroll 1
    for (int p = 0; p < 32; p += 16) {
      const int tr[2] = {p + (lane >> 3), p + 8 + (lane >> 3)};
      const int64_t token[2] = {m0 + 32 * s + tr[0], m0 + 32 * s + tr[1]};
      const int left[2] = {token[0] < a.tokens ? some : 0, token[1] < a.tokens ? some : 0};
      float v[2][8];
      const auto sums = [&] {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int q = 0; q < 8; q++) v[i][q] = st[tr[i] * kSlabPitch + c + q];
      };
      if (part) {
        sums();
#pragma unroll
        for (int i = 0; i < 2; i++)
          if (left[i] > 0) store_piece<false>(part, token[i] * part_pitch(rows) + n, v[i], 8);
      } else {
        const Finish<2> f(a, token, n, left);
        sums();
#pragma unroll
        for (int i = 0; i < 2; i++) f.store(a, i, token[i], n, left[i], bias, v[i]);
      }
    }
    wave_lds_fence();
  }
}

// ---- a middling number of tokens -------------------------------------------------
// A workgroup makes BM tokens x 128 outputs over its share of the columns
// (split of splits), in steps of 128.  Each thread fetches its weights and
// activations of the next two steps into registers while this one is
// multiplied, and turns them into bf16 in LDS after it, so r is never written to memory.
// LDS holds one step: another workgroup of the CU multiplies meanwhile.  203
// tokens, 4096 x 14336, 3 bits: 47 us, 510 TFLOP/s (and 7 to join the shares);
// matrix units busy 34%, VALU and LDS as much, one after the other: the two
// workgroups overlap little.  (Groups of four wavefronts that decode and multiply
// in turn, 128 or 256 tokens a workgroup, took as long, as did each wavefront
// decoding right into its operands, at 1.4 times the LDS reads.)
// Chunk c of row m of a step lies at chunk c ^ 2 (c / 8) ^ m % 16 of the row's 256
// bytes: neither 8 rows' chunk c nor two rows' chunks i, 4 + i, 8 + i and 12 + i share banks.
constexpr int kFusedK = 128;
__device__ __forceinline__ int wide_at(int m, int c) { return m * kFusedK + 8 * (c ^ (c >> 3 << 1) ^ (m & 15)); }

template <int FMT, int BITS, int XT, int BM>
__global__ __launch_bounds__(256, 2) void fused_kernel(Weights w, quasar_linear a, int tiles_m, int splits, int steps_per,
                                                       float* part) {
  constexpr int TM = BM / 32, NX = BM / 16;  // 16-token tiles of a wavefront; chunks of x a thread fetches
  __shared__ __align__(16) uint16_t lds[(BM + 128) * kFusedK];
  static_assert(4 * kSlab * 4 <= (int)sizeof(lds), "the epilogue's stage fits");
  uint16_t* const xs = lds;
  uint16_t* const rs = lds + BM * kFusedK;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
  const int split = blockIdx.x % (unsigned)splits, tile = blockIdx.x / (unsigned)splits;
  const int64_t m0 = (int64_t)(tile % tiles_m) * BM, n0 = (int64_t)(tile / tiles_m) * 128;
  const int K = (int)w.cols, all = (K + kFusedK - 1) / kFusedK;
  const int s0 = split * steps_per, s1 = s0 + steps_per < all ? s0 + steps_per : all;

  // this thread's quarter of the step in rows tid / 4 and 64 + tid / 4 of r; its chunk of x in rows tid / 16 + 16 i
  const int wr = tid >> 2, wq = tid & 3, xr = tid >> 4, xc = tid & 15;
  const WeightRow<FMT, BITS> row0(w, n0 + wr < w.rows ? n0 + wr : w.rows - 1);
  const WeightRow<FMT, BITS> row1(w, n0 + 64 + wr < w.rows ? n0 + 64 + wr : w.rows - 1);
  const char* xp[NX];
#pragma unroll
  for (int i = 0; i < NX; i++) {
    const int64_t m = m0 + xr + 16 * i;
    xp[i] = reinterpret_cast<const char*>(a.x) + ((m < a.tokens ? m : a.tokens - 1) * a.x_stride + 8 * xc) * elem_size<XT>();
  }
  struct Fetched {
    Strip<FMT, BITS> w[2];
    XChunk<XT> x[NX];
  } f[2];
  const auto fetch = [&](Fetched& o, int s) {
    const int k = s * kFusedK;
    o.w[0].load(row0, k + 32 * wq);
    o.w[1].load(row1, k + 32 * wq);
#pragma unroll
    for (int i = 0; i < NX; i++) o.x[i].load(xp[i], k);
  };
  const auto stage = [&](Fetched& o) {
#pragma unroll
    for (int i = 0; i < NX; i++) *reinterpret_cast<uint4*>(xs + wide_at(xr + 16 * i, xc)) = o.x[i].bf16();
#pragma unroll
    for (int h = 0; h < 2; h++) {
      o.w[h].ready(row0.tensor_scale);
#pragma unroll
      for (int i = 0; i < 4; i++) *reinterpret_cast<uint4*>(rs + wide_at(wr + 64 * h, 4 * wq + i)) = o.w[h].chunk(i);
    }
  };
  const int wm = wave >> 1, wn = wave & 1;
  f32x4 acc[TM][4];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const auto meet = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // matrix instructions first, where the CU's other workgroup decodes meanwhile (5 to 8% at 512 tokens)
  const auto multiply = [&] {
    meet();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 4; k++) {
      bf16x8 mx[TM], mr[4];
#pragma unroll
      for (int i = 0; i < TM; i++)
        mx[i] = as_bf16x8(*reinterpret_cast<const uint4*>(xs + wide_at(wm * (BM / 2) + 16 * i + (lane & 15), 4 * k + (lane >> 4))));
#pragma unroll
      for (int j = 0; j < 4; j++)
        mr[j] = as_bf16x8(*reinterpret_cast<const uint4*>(rs + wide_at(wn * 64 + 16 * j + (lane & 15), 4 * k + (lane >> 4))));
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx[i], mr[j], acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    meet();  // every wavefront is done with the step
  };
  // Whole steps, two in flight.  The loop's fetches stand behind no branch (the compiler would make the first use
  // of any wait for all of them); the last two or three steps come after it.
  const int whole = K / kFusedK < s1 ? K / kFusedK : s1, n = whole - s0;
  if (n >= 2) {
    fetch(f[0], s0);
    fetch(f[1], s0 + 1);
    int s = s0;
    for (; s + 3 < whole; s += 2) {
      stage(f[0]);
      fetch(f[0], s + 2);
      multiply();
      stage(f[1]);
      fetch(f[1], s + 3);
      multiply();
    }
    stage(f[0]);
    if (s + 2 < whole) fetch(f[0], s + 2);
    multiply();
    stage(f[1]);
    multiply();
    if (s + 2 < whole) {
      stage(f[0]);
      multiply();
    }
  } else if (n == 1) {
    fetch(f[0], s0);
    stage(f[0]);
    multiply();
  }
  if (whole < s1) {  // the columns past the whole steps
    const int k = whole * kFusedK;
    f[0].w[0].load(row0, k + 32 * wq, K - k - 32 * wq);
    f[0].w[1].load(row1, k + 32 * wq, K - k - 32 * wq);
#pragma unroll
    for (int i = 0; i < NX; i++) f[0].x[i].load(xp[i], k, k + 8 * xc < K);
    stage(f[0]);
    multiply();
  }
  store_tile<TM>(a, w.rows, acc, m0 + wm * (BM / 2), n0 + wn * 64, reinterpret_cast<float*>(lds) + wave * kSlab,
                 part ? part + (int64_t)split * a.tokens * part_pitch(w.rows) : nullptr);
}

// y from the sums of `splits` shares of the columns, eight outputs a thread.
__global__ __launch_bounds__(256) void join_kernel(quasar_linear a, int64_t rows, const float* part, int splits) {
  const int64_t per = (rows + 7) / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t token = i / per, n = (i - token * per) * 8;
  if (token >= a.tokens) return;
  const int left = (int)(rows - n < 8 ? rows - n : 8);
  float v[8] = {}, bias[8];
  const int64_t tokens[1] = {token};
  const int lefts[1] = {left};
  Finish<1>::load_bias(a, n, left, bias);
  const Finish<1> f(a, tokens, n, lefts);
  for (int s = 0; s < splits; s += 8) {  // eight shares in flight at once
    Piece<kElemF32> p[8];
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) p[j].load(part, ((int64_t)(s + j) * a.tokens + token) * part_pitch(rows) + n, 8);
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) {
#pragma unroll
        for (int q = 0; q < 8; q++) v[q] += p[j].get(q);
      }
  }
  f.store(a, 0, token, n, left, bias, v);
}

// ---- many tokens --------------------------------------------------------------
// r in bf16 [rows, kp], columns past the last zero; then (workgroups from
// weight_blocks on) x in bf16 [tokens, kp] likewise, where it is not used as
// it is.  A thread makes 32 weights, which go through LDS so that a wavefront
// stores whole lines, or 8 activations.
template <int FMT, int BITS, int XT>
__global__ __launch_bounds__(256) void unpack_kernel(Weights w, quasar_linear a, int kp, uint16_t* r, uint16_t* xo,
                                                     unsigned weight_blocks) {
  if (blockIdx.x < weight_blocks) {
    __shared__ uint4 lds[256 * 4];
    const int lane = threadIdx.x & 63, per = kp / 32;
    uint4* const mine = lds + wave_index() * 256;
    const int64_t first = (int64_t)blockIdx.x * 256 + wave_index() * 64, i = first + lane, total = w.rows * per;
    const int64_t row = i < total ? i / per : 0;
    const int k = i < total ? (int)(i - row * per) * 32 : 0;
    const WeightRow<FMT, BITS> at(w, row);
    Strip<FMT, BITS> strip;
    const int left = (int)w.cols - k;
    strip.load(at, k, left);
    strip.ready(at.tensor_scale);
    // strip l's chunk c lies at 4 l + (c ^ l / 4 % 4): both sides without bank conflicts
#pragma unroll
    for (int c = 0; c < 4; c++)
      mine[4 * lane + (c ^ ((lane >> 2) & 3))] = 8 * c < left ? strip.chunk(c) : make_uint4(0u, 0u, 0u, 0u);
    wave_lds_fence();
    uint4* const out = reinterpret_cast<uint4*>(r) + first * 4;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const int chunk = 64 * j + lane, l = chunk >> 2;
      if (first + l < total) out[chunk] = mine[4 * l + ((chunk & 3) ^ ((l >> 2) & 3))];
    }
  } else {
    const int per = kp / 8;
    const int64_t total = a.tokens * per, step = (int64_t)(gridDim.x - weight_blocks) * 256;
    // more than once only past the threads that a grid takes
    for (int64_t i = (int64_t)(blockIdx.x - weight_blocks) * 256 + threadIdx.x; i < total; i += step) {
      const int64_t t = i / per;
      const int k = (int)(i - t * per) * 8;
      XChunk<XT> c;
      c.load(a.x, t * a.x_stride + k, k < w.cols);
      st128(xo + t * kp + k, c.bf16());
    }
  }
}

// A workgroup makes 256 tokens x 256 outputs with 8 wavefronts of 128 x 64.
// Both operands of a step lie in LDS as two halves each (x0: the first 64
// tokens of every wavefront's 128, r0: the first 32 outputs of its 64, x1 and
// r1 the rest), and a step has two phases, each with 32 matrix instructions a
// wavefront: x0 (r0 r1), x1 (r0 r1).  Two stages; a half is filled again as soon
// as both halves of the workgroup have read it.
//
// The wavefronts of a SIMD work in turn: those of wm = 1 run one barrier
// behind, so that while one multiplies the other reads its next operands.
// Barriers 2p and 2p + 1 end the reading and the multiplying of phase p for
// wm = 0, 2p + 1 and 2p + 2 for wm = 1; a wavefront has its operands before it
// comes to the barrier that ends the reading.  Hence
//  - a half filled in phase p may be one whose last reads were in phase p - 1
//    (x0, r0 and r1, read in a step's phase 0, are filled for the step after the
//    next in its phase 1; x1 in the next step's phase 0);
//  - what phase p reads has to have landed for every wavefront's own loads
//    before the barrier that ends its reading of phase p - 1: with two loads a
//    half, "at most 8 outstanding" then, either phase.
// Past the last step the loads repeat it, so that the counts hold.  (Four phases
// of 16 instructions, with twice the barriers, were 5% slower.)  At 8192 tokens,
// 14336 x 4096: 665 to 740 us as the clock goes, 1.3 to 1.45 PFLOP/s, matrix units
// busy 81% of the time.
__global__ __launch_bounds__(512, 2) void tile_kernel(quasar_linear a, const uint16_t* x, int64_t x_stride,
                                                      const uint16_t* r, int64_t rows, int kp, int tiles_m, int tiles_n,
                                                      int steps_per, float* part) {
  constexpr int kHalf = 128 * kTileK, kStage = 4 * kHalf;  // elements; halves x0, r0, r1, x1
  __shared__ __align__(16) uint16_t lds[2 * kStage];
  static_assert(8 * kSlab * 4 <= (int)sizeof(lds), "the epilogue's stage fits");
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int wm = wave >> 2, wn = wave & 3;
  int tm, tn;
  const int split = blockIdx.x / (unsigned)(tiles_m * tiles_n);
  tile_of(blockIdx.x - split * tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * 256, n0 = (int64_t)tn * 256;
  const int ms = (int)(a.tokens - m0 < 256 ? a.tokens - m0 : 256), ns = (int)(rows - n0 < 256 ? rows - n0 : 256);
  const int first = split * steps_per, left = kp / kTileK - first, steps = left < steps_per ? left : steps_per;

  // each wavefront loads 16 rows of a half, 8 an instruction; rows past the matrix repeat its last
  uint32_t off[4][2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int lr = wave * 16 + i * 8 + (lane >> 3);
    const uint32_t c = 16u * ((lane & 7) ^ ((lr >> 1) & 7));
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int m = (lr >> 6) * 128 + h * 64 + (lr & 63), n = (lr >> 5) * 64 + h * 32 + (lr & 31);
      off[h == 0 ? 0 : 3][i] = (uint32_t)(m < ms ? m : ms - 1) * (uint32_t)(x_stride * 2) + c;
      off[h == 0 ? 1 : 2][i] = (uint32_t)(n < ns ? n : ns - 1) * (uint32_t)(kp * 2) + c;
    }
  }
  const char* const xb = reinterpret_cast<const char*>(x + m0 * x_stride + first * kTileK);
  const char* const rb = reinterpret_cast<const char*>(r + n0 * kp + first * kTileK);
  const auto fill = [&](int h, int step) {
    const char* const from = (h == 0 || h == 3 ? xb : rb) + (step < steps ? step : steps - 1) * (2 * kTileK);
#pragma unroll
    for (int i = 0; i < 2; i++)
      load_lds16(from, off[h][i], lds0 + ((step & 1) * kStage + h * kHalf + (wave * 16 + i * 8) * kTileK) * 2);
  };
  f32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 fx[4][2], fr[2][2][2];
  const auto read_x = [&](int h, int stage) {
    const uint16_t* p = lds + stage * kStage + (h ? 3 : 0) * kHalf;
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
      for (int k = 0; k < 2; k++)
        fx[t][k] = as_bf16x8(*reinterpret_cast<const uint4*>(p + chunk_at(wm * 64 + 16 * t + (lane & 15), 4 * k + (lane >> 4))));
  };
  const auto read_r = [&](int h, int stage) {
    const uint16_t* p = lds + stage * kStage + (h ? 2 : 1) * kHalf;
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int k = 0; k < 2; k++)
        fr[h][t][k] = as_bf16x8(*reinterpret_cast<const uint4*>(p + chunk_at(wn * 32 + 16 * t + (lane & 15), 4 * k + (lane >> 4))));
  };
  // ends the phase's reading, multiplies by both halves of r, ends the phase
  const auto multiply = [&](int hx) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int hr = 0; hr < 2; hr++)
#pragma unroll
      for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
          for (int j = 0; j < 2; j++)
            acc[hx * 4 + i][hr * 2 + j] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i][k], fr[hr][j][k], acc[hx * 4 + i][hr * 2 + j], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto landed8 = [] { asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); };

  fill(0, 0);
  fill(1, 0);
  fill(2, 0);
  fill(3, 0);
  fill(0, 1);
  fill(1, 1);
  fill(2, 1);
  landed8();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (wm == 1) __builtin_amdgcn_s_barrier();
  for (int s = 0; s < steps; s++) {
    const int stage = s & 1;
    read_x(0, stage);
    read_r(0, stage);
    read_r(1, stage);
    fill(3, s + 1);
    landed8();
    multiply(0);
    read_x(1, stage);
    fill(0, s + 2);
    fill(1, s + 2);
    fill(2, s + 2);
    landed8();
    multiply(1);
  }
  if (wm == 0) __builtin_amdgcn_s_barrier();
  // LDS is the epilogue's once every wavefront's loads have landed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  store_tile<8>(a, rows, acc, m0 + wm * 128, n0 + wn * 64, reinterpret_cast<float*>(lds) + wave * kSlab,
                part ? part + (int64_t)split * a.tokens * part_pitch(rows) : nullptr);
}

enum Form : int { kStrip, kFused, kTile };
struct Choice {
  Form form;
  int splits, steps;  // shares of the columns, and (fused, tile) the steps of each
  size_t bytes;       // workspace
  int bm;             // fused: tokens a workgroup takes
};

int padded_cols(const quasar_desc& d) { return (int)((d.cols + kTileK - 1) / kTileK * kTileK); }

// Splits the steps of `tiles` tiles into shares while that makes no more than
// `most` workgroups, each of `least` steps or more.
void split_steps(Choice& c, int64_t tiles, int steps, int64_t most, int least) {
  while (c.splits < 32 && 2 * tiles * c.splits <= most && steps >= 2 * c.splits * least) c.splits *= 2;
}

// Tiles of 64 or 128 tokens and shares of the columns for the fused kernel: those of
// the least time, from what was measured of its parts.  A step of 128 tokens takes 1.8
// us where a CU has one workgroup, 2.35 where it has two (64 tokens: 1.15 and 1.8); a
// round of workgroups costs 2 more, the join of the shares 3 and what it and they move
// at 5.2 TB/s.  (With 16 shares at most, 84 tokens at 192 x 14336 took 19.5 us, not 17;
// with 64 they took 17 as well.  With shares in powers of two that fill the CUs once or
// twice: 179 tokens at 4113 x 11904 67 us, so 48; 250 at 9000 x 9088 95, so 74; 60 at
// 16000 x 1024 19, so 13; 900 at 1500 x 12288 69, so 61.  203 at 4096 x 14336: 59 in tiles of 64, 48
// in tiles of 128; 320 at 6000 x 2048: 23.7 in tiles of 64, 28 in tiles of 128.)
void choose_fused(Choice& c, int64_t tokens, int64_t rows, int steps) {
  double least = 0.0;
  for (int bm = 64; bm <= 128; bm += 64) {
    const double one = bm == 64 ? 1.15 : 1.8, two = bm == 64 ? 1.8 : 2.35;
    const int64_t tiles = ((tokens + bm - 1) / bm) * ((rows + 127) / 128);
    for (int s = 1, last = 0; s <= 32 && s <= steps && (s == 1 || tiles * s <= 4 * kCUs); s++) {
      const int per = (steps + s - 1) / s;
      if (per == last) continue;  // as many steps a share
      last = per;
      const int64_t groups = tiles * s, full = groups / (2 * kCUs), rest = groups % (2 * kCUs);
      const double us = full * (2.0 + per * two) + (rest == 0 ? 0.0 : 2.0 + per * (rest <= kCUs ? one : two)) +
                        (s == 1 ? 0.0 : 3.0 + (double)(tokens * part_pitch(rows)) * s * (8 / 5.2e6));
      if (c.bm == 0 || us < least) {
        c.bm = bm;
        c.splits = s;
        c.steps = per;
        least = us;
      }
    }
  }
}

// By the number of tokens (figures: us at rows x columns, INT4, this form against its neighbour):
//  - up to 32 the strip kernel: 32 tokens 7.6 against 13 at 4096 x 4096, 20 against 25 at 4096 x 14336.  A wavefront
//    of it with eight steps or more shares them with other workgroups, down to two, while the CUs are not full (192 x
//    14336: 1 token 6.8 against 8.8, 32 tokens 9.7 against 16; with four steps the join costs more: 6.0 against 4.6);
//  - the tile kernel where its 256 x 256 tiles come near to filling the CUs and there are tokens enough to pay for
//    writing r out (6000 tokens at 2000 x 4096, 192 tiles: 87 against 146; 768 at 14336 x 4096: 98 against 135; 2500 at
//    4096 x 2048, 160 tiles: 57 against 68, but 4000 at 2048 x 2048, 128 tiles, 58 against 46; at 128 tiles of 4096 columns
//    even: 2000 at 4096 x 4096 81 against 84, 2048 at 5000 x 4096 88 against 84), or where the columns are
//    many enough to be split (1500 at 4096 x 14336, 96 tiles: 186 against 235, but 1024 at 2048 x 16384, 32 tiles, 105
//    against 91);
//  - the fused kernel between them.
Choice choose(const quasar_desc& d, int64_t tokens) {
  Choice c{kStrip, 1, 0, 0, 0};
  int64_t tiles = (d.rows + 15) / 16;
  int steps = (int)(d.cols / 128 / kStripWaves);
  if (tokens <= 32) {
    if (steps >= 8) split_steps(c, tiles, steps, kCUs, 2);
    if (c.splits > 1) c.bytes = (size_t)c.splits * (size_t)tokens * (size_t)part_pitch(d.rows) * 4;
    return c;
  }
  tiles = ((tokens + 255) / 256) * ((d.rows + 255) / 256);
  if ((tokens >= 768 && tiles >= 160) || (tokens >= 1024 && d.cols >= 8192 && tiles >= 48)) {
    c.form = kTile;
    steps = padded_cols(d) / kTileK;
    split_steps(c, tiles, steps, kCUs, 16);
    c.steps = (steps + c.splits - 1) / c.splits;
    c.splits = (steps + c.steps - 1) / c.steps;
    c.bytes = (size_t)(d.rows + tokens) * (size_t)padded_cols(d) * 2;
  } else {
    c.form = kFused;
    choose_fused(c, tokens, d.rows, (int)((d.cols + kFusedK - 1) / kFusedK));
  }
  if (c.splits > 1) c.bytes += (size_t)c.splits * (size_t)tokens * (size_t)part_pitch(d.rows) * 4;
  return c;
}

// 32 outputs a workgroup of the strip kernel where there are many and x is what takes time: 24 and 32 tokens in bf16 at
// 14336 x 4096 18.4 and 19.7 against 23.3 and 24.5, at 8192 x 4096 10.5 and 11.4 against 12.1 and 12.5, at 4096 x 4096
// 9.7 and 9.9 against 7.3 and 7.5; 8 tokens at 14336 x 4096 12.2 against 11.6, 32 of 8 bits there 19.3 against 19.1.
bool strip_two(const quasar_desc& d, int64_t tokens, int x_dtype) {
  return x_dtype == QUASAR_BF16 && tokens > 16 && d.rows >= 8192;
}
int64_t strip_groups(const quasar_desc& d, const Choice& c, bool two) {
  return (d.rows + (two ? 31 : 15)) / (two ? 32 : 16) * c.splits;
}
int64_t tiles_of(const quasar_desc& d, int64_t tokens, int bm, int bn) {
  return ((tokens + bm - 1) / bm) * ((d.rows + bn - 1) / bn);
}
int64_t unpack_weight_groups(const quasar_desc& d) { return (d.rows * (padded_cols(d) / 32) + 255) / 256; }

// x goes through the workspace unless the tile kernel can load its rows in
// 16-byte pieces as they are.
bool x_direct(int64_t cols, int x_dtype, const void* x, int64_t stride) {
  return x_dtype == QUASAR_BF16 && cols % kTileK == 0 && stride % 8 == 0 && stride < (1 << 22) &&
         (reinterpret_cast<uintptr_t>(x) & 15) == 0;
}

template <int FMT, int BITS, int XT>
hipError_t launch(const quasar_desc& d, const quasar_linear& a, hipStream_t stream) {
  Weights w{a.codes, a.scales, a.zeros, a.tensor_scale, d.rows, d.cols, d.group == 64 ? 6 : 7};
  const Choice c = choose(d, a.tokens);
  float* part = nullptr;  // the sums of the shares, [splits, tokens, part_pitch(rows)]
  const auto join = [&] {
    const int64_t n = a.tokens * ((d.rows + 7) / 8);
    join_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream>>>(a, d.rows, part, c.splits);
    return hipGetLastError();
  };
  if (c.form == kStrip) {
    const bool two = strip_two(d, a.tokens, a.x_dtype);
    const unsigned gx = (unsigned)strip_groups(d, c, two);
    if (c.splits > 1) part = reinterpret_cast<float*>(a.workspace);
    const auto strip = [&](auto nx) {
      constexpr int NX = decltype(nx)::value, NB = NX == 8 && XT == kElemBF16 ? 2 : 1;
      const dim3 block(64 * kStripWaves);
      if (two)
        strip_kernel<FMT, BITS, XT, NX, NB><<<dim3(gx), block, 0, stream>>>(w, a, __builtin_ctz(c.splits), part);
      else
        strip_kernel<FMT, BITS, XT, NX, 1><<<dim3(gx), block, 0, stream>>>(w, a, __builtin_ctz(c.splits), part);
    };
    if (a.tokens <= 4)
      strip(std::integral_constant<int, 1>());
    else if (a.tokens <= 8)
      strip(std::integral_constant<int, 2>());
    else if (a.tokens <= 16)
      strip(std::integral_constant<int, 4>());
    else
      strip(std::integral_constant<int, 8>());
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || !part ? e : join();
  }
  if (c.form == kFused) {
    const int tm = (int)((a.tokens + c.bm - 1) / c.bm);
    if (c.splits > 1) part = reinterpret_cast<float*>(a.workspace);
    const dim3 grid((unsigned)(tiles_of(d, a.tokens, c.bm, 128) * c.splits));
    if (c.bm == 64)
      fused_kernel<FMT, BITS, XT, 64><<<grid, dim3(256), 0, stream>>>(w, a, tm, c.splits, c.steps, part);
    else
      fused_kernel<FMT, BITS, XT, 128><<<grid, dim3(256), 0, stream>>>(w, a, tm, c.splits, c.steps, part);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || !part ? e : join();
  }
  const int kp = padded_cols(d);
  uint16_t* r = reinterpret_cast<uint16_t*>(a.workspace);
  uint16_t* xo = r + d.rows * kp;
  if (c.splits > 1) part = reinterpret_cast<float*>(xo + a.tokens * kp);
  const bool direct = x_direct(d.cols, a.x_dtype, a.x, a.x_stride);
  const int64_t wb = unpack_weight_groups(d), most = most_groups(256) - wb;
  int64_t xb = direct ? 0 : (a.tokens * (kp / 8) + 255) / 256;
  if (xb > most) xb = most;
  unpack_kernel<FMT, BITS, XT><<<dim3((unsigned)(wb + xb)), dim3(256), 0, stream>>>(w, a, kp, r, xo, (unsigned)wb);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tm = (int)((a.tokens + 255) / 256), tn = (int)((d.rows + 255) / 256);
  tile_kernel<<<dim3((unsigned)(tm * tn * c.splits)), dim3(512), 0, stream>>>(
      a, direct ? reinterpret_cast<const uint16_t*>(a.x) : xo, direct ? a.x_stride : kp, r, d.rows, kp, tm, tn, c.steps,
      part);
  e = hipGetLastError();
  return e != hipSuccess || !part ? e : join();
}

template <int FMT, int BITS>
hipError_t launch_x(const quasar_desc& d, const quasar_linear& a, hipStream_t stream) {
  return a.x_dtype == QUASAR_BF16 ? launch<FMT, BITS, kElemBF16>(d, a, stream) : launch<FMT, BITS, kElemE4M3>(d, a, stream);
}

}  // namespace

size_t linear_workspace(const quasar_desc& d, int64_t tokens) { return choose(d, tokens).bytes; }

bool linear_fits(const quasar_desc& d, int64_t tokens, int x_dtype, size_t& workspace) {
  const Choice c = choose(d, tokens);
  workspace = c.bytes;
  if (c.form == kStrip) return strip_groups(d, c, strip_two(d, tokens, x_dtype)) <= most_groups(64 * kStripWaves);
  if (c.form == kFused) return tiles_of(d, tokens, c.bm, 128) * c.splits <= most_groups(256);
  return tiles_of(d, tokens, 256, 256) * c.splits <= most_groups(512) && unpack_weight_groups(d) < most_groups(256);
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
