// layer_norm_kernel.hip -- the layer norm with the residual's addition and its
// gradients (quasar_ops.h).
//
// Both directions are bound by memory.  A row is read once and kept in registers
// widened to fp32, eight consecutive elements (one 16-byte load in bf16) per lane
// and step: the mean, then the deviations from it and their squares, the row's
// largest |y| and the outputs all come from one read.  (sum(h^2) - cols mean^2 cancels
// where the mean is large; and the fp32 mean is itself off by roundings of its own
// size, so the deviations' mean, which is what it is off by, is taken off again:
// without that y of rows 1000 +- 2^-8 was off by 2e-2.)  67 M elements in bf16 with a residual, rows of
// 64 to 16384 columns: forward 94 to 99 us, 5.4 to 5.7 TB/s (a copy of 1 GiB: 5.0),
// with q beside y 109, q alone 85 at 4096; gradients 101 to 118, 4.5 to 5.3.  Taking
// the mean's error off costs 0 to 3%.  Odd widths cost more (1537 columns: 110 and 137),
// as do gradients past 16384 columns, whose shares spill (32768: 364).  One row of 4096
// takes 3.9 us.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {

// floats from one part of dweight or dbias to the next
__host__ __device__ constexpr int ln_pitch(int cols) { return (cols + 3) & ~3; }

namespace {

// Threads of a workgroup, and the rows that it works on at once, where TPR
// threads (8, 16 or 32 lanes, a wavefront, or a workgroup) work on one row.
template <int TPR>
struct Shape {
  static constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
  static __device__ __forceinline__ int lane() { return threadIdx.x & (TPR - 1); }
  static __device__ __forceinline__ int row() { return TPR == 64 ? wave_index() : TPR > 64 ? 0 : threadIdx.x / TPR; }
};

// Over the TPR threads of a row; s: LDS of its own for each call where they are
// several wavefronts.
template <int TPR, typename Op>
__device__ __forceinline__ float row_reduce(float x, float* s, Op op) {
  if constexpr (TPR < 64) {
    x = op(x, dpp_f32<kDppXor1>(x));
    x = op(x, dpp_f32<kDppXor2>(x));
    x = op(x, dpp_f32<kDppHalfMirror>(x));
    if constexpr (TPR >= 16) x = op(x, dpp_f32<kDppMirror>(x));
    if constexpr (TPR == 32) x = pair_rows<16>(x, op);
    return x;
  } else {
    return group_reduce<TPR / 64>(x, s, op);
  }
}
// Two sums, through one barrier.
template <int TPR>
__device__ __forceinline__ void row_sums(float& x, float& y, float* s, float* t) {
  if constexpr (TPR <= 64) {
    x = row_reduce<TPR>(x, s, SumOp());
    y = row_reduce<TPR>(y, t, SumOp());
  } else {
    x = wave_reduce(x, SumOp());
    y = wave_reduce(y, SumOp());
    if ((threadIdx.x & 63) == 0) {
      s[wave_index()] = x;
      t[wave_index()] = y;
    }
    __syncthreads();
    x = s[0];
    y = t[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; i++) {
      x += s[i];
      y += t[i];
    }
  }
}

template <int XT, int RT, int TPR, int NV>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void layer_norm_kernel(quasar_layer_norm a) {
  constexpr int kWaves = TPR < 64 ? 1 : TPR / 64;
  __shared__ float red[4][kWaves];
  const int t = Shape<TPR>::lane(), cols = (int)a.cols;
  const int64_t row = (int64_t)blockIdx.x * Shape<TPR>::kRows + Shape<TPR>::row();
  if (row >= a.rows) return;  // whole rows of 16 lanes; no barrier follows where there are several rows
  // us, element by element and cut: 500000 x 60 bf16 71, 60; 29626 x 198 15.4, 12.6; 4000 x 5313 27, 24.5; fp32 100000 x 129
  // 21, 24
  constexpr int kMode = TPR == 1024 && NV == 2 ? kCutNone : TPR >= 64 ? kCutAll : kCutBF16 | (TPR == 8 ? kCutTiny : 0);
  float h[NV][8];
  int col[NV];
  Piece<XT> px[NV];
  Piece<RT == kElemNone ? XT : RT> pr[NV];
  const int64_t ex = row * a.x_stride, er = row * a.residual_stride;
#pragma unroll
  for (int v = 0; v < NV; v++) {
    col[v] = (v * TPR + t) * 8;
    load_cut<kMode>(px[v], a.x, ex, col[v], cols);
    if constexpr (RT != kElemNone) load_cut<kMode>(pr[v], a.residual, er, col[v], cols);
  }
  // weight and bias are asked for beside the row where there are registers for them
  constexpr bool kEarly = NV <= 2 && TPR <= 256;
  float w[NV][8], b[NV][8] = {};
  const auto affine = [&] {
    load_cut_floats<kMode>(a.weight, 0, col, cols, a.weight_dtype == QUASAR_BF16, w);
    if (a.bias) load_cut_floats<kMode>(a.bias, 0, col, cols, a.bias_dtype == QUASAR_BF16, b);
  };
  if constexpr (kEarly) affine();
  float sum = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; v++) {
    cut<kMode>(px[v], col[v], cols);
    if constexpr (RT != kElemNone) cut<kMode>(pr[v], col[v], cols);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      h[v][i] = px[v].get(i);
      if constexpr (RT != kElemNone) h[v][i] += pr[v].get(i);
      sum += h[v][i];
    }
  }
  const float mean = row_reduce<TPR>(sum, red[0], SumOp()) / (float)cols;
  if constexpr (RT != kElemNone) {
    if (a.h) {
      const int64_t eh = row * a.h_stride;
#pragma unroll
      for (int v = 0; v < NV; v++) {
        const int c = (v * TPR + t) * 8;
        store_piece<RT == kElemBF16>(a.h, eh + c, h[v], cols - c);
      }
    }
  }
  float ss = 0.0f, rest = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int left = cols - (v * TPR + t) * 8;
#pragma unroll
    for (int i = 0; i < 8; i++) h[v][i] -= mean;
    if (left < 8) {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i >= left) h[v][i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      ss = __builtin_fmaf(h[v][i], h[v][i], ss);
      rest += h[v][i];
    }
  }
  row_sums<TPR>(ss, rest, red[1], red[2]);
  // what the mean is off by (0 where the squares are not finite), and the squares about the better one
  rest = ss < INFINITY ? rest / (float)cols : 0.0f;
  float var = __builtin_fmaf(-rest, rest, ss / (float)cols);
  var = var < 0.0f ? 0.0f : var;  // NaN stays
  const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean + rest;
    if (a.rstd) a.rstd[row] = rstd;
  }
  if constexpr (!kEarly) affine();
  float top = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; v++) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      h[v][i] = __builtin_fmaf((h[v][i] - rest) * rstd, w[v][i], b[v][i]);
      top = fmaxf(top, fabsf(h[v][i]));
    }
  }
  if (a.y) {
    const int64_t ey = row * a.y_stride;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8;
      store_piece(a.y, ey + c, h[v], cols - c, a.y_dtype == QUASAR_BF16);
    }
  }
  if (!a.q) return;
  top = row_reduce<TPR>(top, red[3], MaxOp());
  // NaN for a row that is not finite
  float scale = fmaxf(top / 448.0f, 0x1p-120f);
  if (!(ss < INFINITY)) scale = __builtin_nanf("");
  if (t == 0) a.scale[row] = scale;
  const int64_t eq = row * a.q_stride;
  const float inv = 1.0f / scale;
  const bool plain = !(scale >= 0x1p-80f && scale <= 0x1p100f);  // the remainders may not be exact, or nothing finite
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; i++) s[i] = quotient(h[v][i], scale, inv);
    if (plain) {
#pragma unroll
      for (int i = 0; i < 8; i++) s[i] = h[v][i] / scale;
    }
    store_bytes(a.q + eq + c, pack_e4m3x8(s), cols - c);
  }
}

// f(TPR, NV) for the widest-fitting shape.
template <typename F>
hipError_t with_shape(int64_t cols, F f) {
  using std::integral_constant;
#define QUASAR_SHAPE(T, N) \
  if (cols <= 8 * T * N) return f(integral_constant<int, T>(), integral_constant<int, N>())
  QUASAR_SHAPE(8, 1);
  QUASAR_SHAPE(16, 1);
  QUASAR_SHAPE(32, 1);
  QUASAR_SHAPE(64, 1);
  QUASAR_SHAPE(64, 2);
  QUASAR_SHAPE(64, 4);
  QUASAR_SHAPE(256, 2);
  QUASAR_SHAPE(256, 4);
  QUASAR_SHAPE(1024, 2);
  QUASAR_SHAPE(1024, 4);
#undef QUASAR_SHAPE
  return hipErrorInvalidValue;
}

// n rows from row r on
quasar_layer_norm rows_of(quasar_layer_norm a, int64_t r, int64_t n) {
  a.rows = n;
  a.x = rows_on(a.x, r, a.x_stride, size_of(a.x_dtype));
  a.residual = rows_on(a.residual, r, a.residual_stride, size_of(a.residual_dtype));
  a.h = rows_on(a.h, r, a.h_stride, size_of(a.residual_dtype));
  a.y = rows_on(a.y, r, a.y_stride, size_of(a.y_dtype));
  a.q = rows_on(a.q, r, a.q_stride, 1);
  a.scale = rows_on(a.scale, r, 1, 4);
  a.mean = rows_on(a.mean, r, 1, 4);
  a.rstd = rows_on(a.rstd, r, 1, 4);
  return a;
}

template <int XT, int RT>
hipError_t launch_types(const quasar_layer_norm& a, hipStream_t stream) {
  return with_shape(a.cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    constexpr int threads = Shape<TPR>::kThreads, rows = Shape<TPR>::kRows;
    constexpr int64_t most = most_groups(threads) * rows;
    for (int64_t r = 0; r < a.rows; r += most) {
      const quasar_layer_norm s = rows_of(a, r, a.rows - r < most ? a.rows - r : most);
      layer_norm_kernel<XT, RT, TPR, NV><<<dim3((unsigned)((s.rows + rows - 1) / rows)), dim3(threads), 0, stream>>>(s);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

// ---- backward ---------------------------------------------------------------
// Groups of TPR threads take rows in turn; a thread meets the same columns in
// every row, so its shares of dweight and dbias stay in registers.  The shares of
// a workgroup's groups meet in its wavefronts and in LDS, those of the workgroups
// in `parts` (ln_parts_kernel sums them), in a fixed order.
template <int GT, int HT, int TPR, int NV>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void layer_norm_backward_kernel(quasar_layer_norm_backward a, float* dw_out,
                                                                                   float* db_out, int64_t part_step) {
  constexpr int kWaves = TPR < 64 ? 1 : TPR / 64, kRows = Shape<TPR>::kRows;
  constexpr int kShares = TPR < 256 ? 4 : 1, kWide = TPR < 64 ? TPR : TPR < 256 ? 64 : 1;  // wavefronts with shares of their own
  __shared__ float red[2][2][kWaves];
  __shared__ float shares[kShares > 1 ? (kShares - 1) * kWide * NV * 8 : 1];
  const int t = Shape<TPR>::lane(), cols = (int)a.cols;
  // us, element by element and cut: 500000 x 60 bf16 92, 60; 29626 x 198 26, 18; 777 x 1537 fp32 11.9, 12.8; 65536 x 1024 bf16
  // 106, 125; past 4096 columns 4000 x 5313 45, 42, but 8192 x 8192 114, 116
  constexpr int kMode = TPR == 8 ? kCutBF16 | kCutTiny : TPR < 64 || TPR == 256 || TPR == 512 ? kCutBF16 : kCutNone;
  const float rcols = 1.0f / (float)cols;
  constexpr bool kKeep = NV < 4;  // the weight stays in registers
  float w[kKeep ? NV : 1][8], dw[NV][8] = {}, db[NV][8] = {};
  const auto weight = [&](int v) -> float (&)[8] {
    if constexpr (kKeep) {
      return w[v];
    } else {
      const int c[1] = {(v * TPR + t) * 8};
      load_cut_floats<kMode>(a.weight, 0, c, cols, a.weight_dtype == QUASAR_BF16, w);
      return w[0];
    }
  };
  int col[NV];
#pragma unroll
  for (int v = 0; v < NV; v++) col[v] = (v * TPR + t) * 8;
  if constexpr (kKeep) load_cut_floats<kMode>(a.weight, 0, col, cols, a.weight_dtype == QUASAR_BF16, w);
  int flip = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + Shape<TPR>::row(); row < a.rows; row += (int64_t)gridDim.x * kRows) {
    Piece<GT> pg[NV];
    Piece<HT> ph[NV];
    const int64_t eg = row * a.dy_stride, eh = row * a.h_stride, ed = row * a.dh_stride, ex = row * a.dx_stride;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8;
      load_cut<kMode>(pg[v], a.dy, eg, c, cols);
      load_cut<kMode>(ph[v], a.h, eh, c, cols);
    }
    // dh is asked for with the rest where there are registers for it
    constexpr bool kEarly = TPR <= 512 || NV == 1;
    float dh[kEarly ? NV : 1][8];
    if constexpr (kEarly) {
      if (a.dh) load_cut_floats<kMode>(a.dh, ed, col, cols, a.dx_dtype == QUASAR_BF16, dh);
    }
    const float rstd = a.rstd[row], mean = a.mean[row];
    float dot = 0.0f, sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      cut<kMode>(pg[v], (v * TPR + t) * 8, cols);
      cut<kMode>(ph[v], (v * TPR + t) * 8, cols);
      float(&wv)[8] = weight(v);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        // past the row's end g and w are 0
        const float n = (ph[v].get(i) - mean) * rstd, g = pg[v].get(i), u = g * wv[i];
        sum += u;
        dot = __builtin_fmaf(u, n, dot);
        dw[v][i] = __builtin_fmaf(g, n, dw[v][i]);
        db[v][i] += g;
      }
    }
    // two LDS rows in turn: a wavefront may be a row ahead of another's read
    if constexpr (TPR <= 64) {
      sum = row_reduce<TPR>(sum, nullptr, SumOp());
      dot = row_reduce<TPR>(dot, nullptr, SumOp());
    } else {
      sum = wave_reduce(sum, SumOp());
      dot = wave_reduce(dot, SumOp());
      if ((threadIdx.x & 63) == 0) {
        red[flip][0][wave_index()] = sum;
        red[flip][1][wave_index()] = dot;
      }
      __syncthreads();
      sum = red[flip][0][0];
      dot = red[flip][1][0];
#pragma unroll
      for (int i = 1; i < kWaves; i++) {
        sum += red[flip][0][i];
        dot += red[flip][1][i];
      }
      flip ^= 1;
    }
    const float m = dot * rcols, mu = sum * rcols;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8, n8 = cols - c;
      float dx[8];
      float(&wv)[8] = weight(v);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float n = (ph[v].get(i) - mean) * rstd;
        dx[i] = rstd * __builtin_fmaf(-m, n, __builtin_fmaf(pg[v].get(i), wv[i], -mu));
      }
      if (a.dh) {
        float(&d)[8] = dh[kEarly ? v : 0];
        if constexpr (!kEarly) {
          const int at[1] = {c};
          load_cut_floats<kMode>(a.dh, ed, at, cols, a.dx_dtype == QUASAR_BF16, dh);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) dx[i] += d[i];
      }
      store_piece(a.dx, ex + c, dx, n8, a.dx_dtype == QUASAR_BF16);
    }
  }
  // the groups of a wavefront, then the wavefronts
  const auto meet = [&](float (&s)[NV][8], float* out) {
    if constexpr (TPR < 64) {
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
          float x = s[v][i];
          if constexpr (TPR == 8) x += dpp_f32<kDppHalf>(x);
          if constexpr (TPR <= 16) x = pair_rows<16>(x, SumOp());
          s[v][i] = pair_rows<32>(x, SumOp());
        }
    }
    if constexpr (kShares > 1) {
      const int wave = wave_index();
      __syncthreads();  // the other sum's reads are done
      if (wave > 0 && (threadIdx.x & 63) < kWide) {
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
          for (int i = 0; i < 8; i++) shares[(((wave - 1) * NV + v) * 8 + i) * kWide + t] = s[v][i];
      }
      __syncthreads();
      if (threadIdx.x >= kWide) return;
#pragma unroll
      for (int j = 0; j < kShares - 1; j++)
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
          for (int i = 0; i < 8; i++) s[v][i] += shares[((j * NV + v) * 8 + i) * kWide + t];
    }
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8;
      store_piece<false>(out, blockIdx.x * part_step + c, s[v], cols - c);
    }
  };
  if (dw_out) meet(dw, dw_out);
  if (db_out) meet(db, db_out);
}

// dweight[c] (blockIdx.y = 0) or dbias[c] = sum of its parts: 16 columns a
// workgroup, four a thread, the parts shared out over 64 rows of threads whose
// sums meet in LDS.
__global__ __launch_bounds__(256) void ln_parts_kernel(const float* parts, int n, int cols, float* dw, float* db) {
  __shared__ float s[64][17];
  float* const out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  const int x = (threadIdx.x & 3) * 4, y = threadIdx.x >> 2, c = blockIdx.x * 16 + x, pitch = ln_pitch(cols);
  parts += blockIdx.y * pitch;
  float sum[4] = {};
  if (c < cols) {
#pragma unroll 8
    for (int i = y; i < n; i += 64) {
      const float4 v = *reinterpret_cast<const float4*>(parts + (int64_t)i * 2 * pitch + c);
      sum[0] += v.x;
      sum[1] += v.y;
      sum[2] += v.z;
      sum[3] += v.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; i++) s[y][x + i] = sum[i];
  __syncthreads();
  // four threads a column sum 16 each, then meet (they are a quad)
  if (threadIdx.x < 64) {
    const int col = threadIdx.x >> 2, q = threadIdx.x & 3;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) t += s[q * 16 + i][col];
    t += dpp_f32<kDppXor1>(t);
    t += dpp_f32<kDppXor2>(t);
    if (q == 0 && blockIdx.x * 16 + col < cols) out[blockIdx.x * 16 + col] = t;
  }
}

// f(TPR, NV): as few pieces a thread as there are threads for, since dweight's and dbias' shares take registers too.
template <typename F>
hipError_t with_backward_shape(int64_t cols, F f) {
  using std::integral_constant;
#define QUASAR_SHAPE(T, N) \
  if (cols <= 8 * T * N) return f(integral_constant<int, T>(), integral_constant<int, N>())
  QUASAR_SHAPE(8, 1);
  QUASAR_SHAPE(16, 1);
  QUASAR_SHAPE(32, 1);
  QUASAR_SHAPE(64, 1);
  QUASAR_SHAPE(64, 2);
  QUASAR_SHAPE(256, 1);
  QUASAR_SHAPE(512, 1);
  QUASAR_SHAPE(1024, 1);
  QUASAR_SHAPE(1024, 2);
  QUASAR_SHAPE(1024, 4);
#undef QUASAR_SHAPE
  return hipErrorInvalidValue;
}

// Workgroups of the backward pass, each with its shares of dweight and dbias: what runs at once, in whole rounds of rows.
// Where one or two rounds would do, fewer may be better, since their shares are written and summed too: a round is reckoned
// 1.1 us, a workgroup's shares 6.2e-6 us a column.  (777 x 1537 fp32: 256 workgroups 11.7 us, 96 14.9, 777 16.6; 1000 x 4096
// bf16: 256 16.0, 96 20.6, 512 18.5; 300 x 4096: 128 10.4, 300 13.7.)  One workgroup's need no second launch, 3.4 (fp32: 4 x
// 4096 6.1, else 7.5; 6 7.4, 7.5; past 8192 columns a round takes longer: 3 x 16384 11.4, 9.1).
int backward_groups(int64_t rows, int64_t cols) {
  const int64_t per = cols <= 64 ? 32 : cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1;  // rows a workgroup takes at once
  const int64_t most = (cols <= 2048 ? 4 : cols <= 4096 ? 2 : 1) * kCUs;
  const int64_t units = (rows + per - 1) / per, first = (units + most - 1) / most;
  int64_t groups = (units + first - 1) / first;
  const auto time = [&](int64_t n) { return (double)((units + n - 1) / n) * 1.1 + (double)(n * cols) * 6.2e-6 + (n == 1 && cols <= 8192 ? 0.0 : 3.4); };
  for (int64_t rounds = first + 1; first <= 2 && rounds <= 8 && rounds <= units; rounds++) {
    const int64_t n = (units + rounds - 1) / rounds;
    if (time(n) < time(groups)) groups = n;
  }
  return (int)groups;
}

template <int GT, int HT>
hipError_t launch_backward_types(const quasar_layer_norm_backward& a, hipStream_t stream) {
  return with_backward_shape(a.cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    const int n = backward_groups(a.rows, a.cols), pitch = ln_pitch((int)a.cols);
    float* const parts = n == 1 ? nullptr : reinterpret_cast<float*>(a.workspace);
    float* const dw = !a.dweight || n == 1 ? a.dweight : parts;
    float* const db = !a.dbias || n == 1 ? a.dbias : parts + pitch;
    layer_norm_backward_kernel<GT, HT, TPR, NV><<<dim3(n), dim3(Shape<TPR>::kThreads), 0, stream>>>(a, dw, db, 2 * pitch);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 1 || (!a.dweight && !a.dbias)) return e;
    ln_parts_kernel<<<dim3((unsigned)((a.cols + 15) / 16), 2), dim3(256), 0, stream>>>(parts, n, (int)a.cols, a.dweight,
                                                                                       a.dbias);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_layer_norm(const quasar_layer_norm& a, hipStream_t stream) {
  const bool xb = a.x_dtype == QUASAR_BF16, rb = a.residual_dtype == QUASAR_BF16;
  if (!a.residual) return xb ? launch_types<kElemBF16, kElemNone>(a, stream) : launch_types<kElemF32, kElemNone>(a, stream);
  if (rb) return xb ? launch_types<kElemBF16, kElemBF16>(a, stream) : launch_types<kElemF32, kElemBF16>(a, stream);
  return xb ? launch_types<kElemBF16, kElemF32>(a, stream) : launch_types<kElemF32, kElemF32>(a, stream);
}

size_t layer_norm_backward_workspace(int64_t rows, int64_t cols) {
  const int n = backward_groups(rows, cols);
  return n > 1 ? (size_t)n * 2 * ln_pitch((int)cols) * sizeof(float) : 0;
}

hipError_t launch_layer_norm_backward(const quasar_layer_norm_backward& a, hipStream_t stream) {
  const bool gb = a.dy_dtype == QUASAR_BF16, hb = a.h_dtype == QUASAR_BF16;
  if (gb) return hb ? launch_backward_types<kElemBF16, kElemBF16>(a, stream) : launch_backward_types<kElemBF16, kElemF32>(a, stream);
  return hb ? launch_backward_types<kElemF32, kElemBF16>(a, stream) : launch_backward_types<kElemF32, kElemF32>(a, stream);
}

}  // namespace quasar
