// Dropout (mask formed from the position, dp_dropout.h), and LayerNorm with the dropout and the residual sum in front of it, forward and
// backward, as operators of their own: rows of any width and stride.  Bound by memory: every operand is read once and every result written once, in
// accesses of eight columns a lane (16 bytes in bf16, 32 in fp32), which need no alignment beyond the element's; only the last group of a row whose
// width is not a multiple of eight goes element by element.  Sums and statistics are fp32, in a fixed order.
#include "dp_device.h"
#include "dp_dropout.h"
#include "dp_errors.h"
#include "dp_host.h"
#include "dp_kernels.h"
#include "dp_ktime.h"

#include <math.h>
#include <type_traits>

namespace dp {

// Eight columns, as they lie in memory: the vector type is aligned like its element (wide global accesses do not ask for more).
template <typename T> struct Row8;
template <> struct Row8<bf16> { typedef bf16x8 value; typedef bf16x8 packed __attribute__((aligned(2))); };
template <> struct Row8<float> { typedef __attribute__((ext_vector_type(8))) float value; typedef value packed __attribute__((aligned(4))); };

template <typename T> __device__ __forceinline__ typename Row8<T>::value row8_load(const T* p, int n) {      // n: columns there are, the others are zero
  if (n >= 8) return *reinterpret_cast<const typename Row8<T>::packed*>(p);
  typename Row8<T>::value v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : (T)0.f;
  return v;
}
template <typename T> __device__ __forceinline__ void row8_store(T* p, int n, const float (&x)[8]) {
  typename Row8<T>::value v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = from_f<T>(x[j]);
  if (n >= 8) {
    *reinterpret_cast<typename Row8<T>::packed*>(p) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = v[j];
}
template <typename T> __device__ __forceinline__ void row8_widen(const typename Row8<T>::value& v, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = to_f<T>(v[j]);
}

// ------------------------------------------------------------------ dropout
struct DropoutK {
  int rows, cols, groups;      // groups of eight columns in a row
  const void* x; int ldx;
  const void* residual; int ldr;
  void* y; int ldy;
  DropK drop;
};

// A thread takes eight columns of a row, the workgroup 256 consecutive such groups, rows one after the other.  Bytes bound it: 32768 x 1280 bf16 with a residual
// 46 us, 5.4 TB/s (a copy of 1 GiB runs at 5.05).  With two groups a thread nothing is gained; found in the caches, one and two: 38 and 38 us, 4096 x 1280 6.6 and 6.8, 2048 x 640 3.5 and 4.0.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutK a) {
  const uint64_t first = (uint64_t)blockIdx.x * 256;
  const uint32_t at = (uint32_t)(first % (uint32_t)a.groups) + threadIdx.x, over = at / (uint32_t)a.groups, row = (uint32_t)(first / (uint32_t)a.groups) + over;
  const int group = (int)(at - over * (uint32_t)a.groups), n = a.cols - 8 * group;
  const DropKey key = drop_key(a.drop);
  if (row >= (uint32_t)a.rows) return;
  const size_t c = 8 * (size_t)group;
  const auto xv = row8_load((const T*)a.x + (size_t)row * a.ldx + c, n);
  typename Row8<T>::value rv;
  if (a.residual) rv = row8_load((const T*)a.residual + (size_t)row * a.ldr + c, n);
  float v[8], r[8];
  row8_widen<T>(xv, v);
  drop8(a.drop, key, group, row, v);
  if (a.residual) {
    row8_widen<T>(rv, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += r[j];
  }
  row8_store((T*)a.y + (size_t)row * a.ldy + c, n, v);
}

// ------------------------------------------------------------------ rows of a LayerNorm
// L lanes share a row: 16, 32 or 64 of a wave, or a workgroup of 256, 512 or 1024; lane l has columns 8 (c L + l) .. + 7 for c = 0 .. NC - 1.
constexpr int NORM_MAX_D = 8192;
template <int L> constexpr int norm_threads = L < 256 ? 256 : L;
template <int L> __device__ __forceinline__ float norm_row_sum(float v, float* red) {      // red: a float per wave, for a row that several waves share
  if constexpr (L >= 64) v = reduce_halves(v, AddOp());
  if constexpr (L >= 32) v = reduce_row_pairs(v, AddOp());
  v = reduce_row(v, AddOp());
  if constexpr (L > 64) {
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v += red[w];
  }
  return v;
}

struct NormK {
  int rows, d;
  float eps;
  const void* x; int ldx;
  const void* residual; int ldr;
  const void* gamma; const void* beta;
  void* sum; int lds;
  void* y; int ldy;
  float* mean; float* rstd;
  DropK drop;
};

// y = LayerNorm(residual + dropout(x)).  32768 x 640, fp32 residual and sum: 50 us, 5.1 TB/s.  The statistics are those of the fp32 sum: what is stored of it may have been rounded to 16 bits.
template <typename T, typename S, int L, int NC>
__global__ void __launch_bounds__(norm_threads<L>) norm_fwd_kernel(const NormK a) {
  __shared__ float red[2][L > 64 ? L / 64 : 1];
  const int l = threadIdx.x % L, wanted = blockIdx.x * (norm_threads<L> / L) + threadIdx.x / L, row = min(wanted, a.rows - 1);
  const bool live = wanted < a.rows;
  const T* x = (const T*)a.x + (size_t)row * a.ldx;
  const S* res = (const S*)a.residual + (size_t)row * a.ldr;
  auto left = [&](int c) { return a.d - 8 * (c * L + l); };      // columns from this group on
  typename Row8<T>::value xv[NC], ga[NC], be[NC];
  typename Row8<S>::value rv[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (left(c) > 0) {
      xv[c] = row8_load(x + 8 * (c * L + l), left(c));
      if (a.residual) rv[c] = row8_load(res + 8 * (c * L + l), left(c));
    }
#pragma unroll
  for (int c = 0; c < NC; ++c)      // (behind the row, not behind the two reductions: few rows wait for each round trip)
    if (left(c) > 0 && a.gamma) {
      ga[c] = row8_load((const T*)a.gamma + 8 * (c * L + l), left(c));
      be[c] = row8_load((const T*)a.beta + 8 * (c * L + l), left(c));
    }
  const DropKey key = drop_key(a.drop);
  float v[NC][8], s = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (left(c) <= 0) continue;
    row8_widen<T>(xv[c], v[c]);
    drop8(a.drop, key, c * L + l, row, v[c]);
    if (a.residual) {
      float r[8];
      row8_widen<S>(rv[c], r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[c][j] += r[j];
    }
    if (a.sum && live) row8_store((S*)a.sum + (size_t)row * a.lds + 8 * (c * L + l), left(c), v[c]);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[c][j];
  }
  const float mu = norm_row_sum<L>(s, red[0]) / a.d;
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left(c)) {
        v[c][j] -= mu;
        q = fmaf(v[c][j], v[c][j], q);
      }
  const float rs = rsqrtf(norm_row_sum<L>(q, red[1]) / a.d + a.eps);
  if (!live) return;
  if (l == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = rs;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (left(c) <= 0) continue;
    float g[8], b[8];
    if (a.gamma) {
      row8_widen<T>(ga[c], g);
      row8_widen<T>(be[c], b);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[c][j] = a.gamma ? fmaf(v[c][j] * rs, g[j], b[j]) : v[c][j] * rs;
    row8_store((T*)a.y + (size_t)row * a.ldy + 8 * (c * L + l), left(c), v[c]);
  }
}

// ------------------------------------------------------------------ backward
struct NormBwdK {
  int rows, d;
  const void* dy; int lddy;
  const void* sum; int lds;
  const float* mean; const float* rstd;
  const void* gamma;
  const void* dsum_in; int ldi;
  void* dsum; int ldds;
  void* dx; int lddx;
  float* partial;      // [workgroup][2][d], or NULL
  DropK drop;
};

// With g = dy gamma and xh = (sum - mean) rstd: dsum = rstd (g - mean(g) - xh mean(g xh)) + dsum_in, dx = dropout of dsum, and the columns' sums of
// dy xh and dy.  A group of L lanes walks every G-th row, the next one's operands requested before the present one is used; a lane adds its columns of
// dy xh and dy in registers, and the groups' sums meet in LDS at the end.  32768 x 640, fp32 residual gradients: 67 us (5.0 TB/s) and 4.7 for the sums.
// Four waves a SIMD where a row has 256 lanes and more, which is what norm_bwd_workgroups counts on: in fp32 129 registers left three, and one workgroup a CU of 512 lanes instead of two
// (us: 1000 x 3000 22.3 -> 19.5, 2048 x 4096 34.9 -> 33.2, 16384 x 1536 117 -> 101, 8192 x 2048 75 -> 71, 8192 x 4096 131 and 132).
template <typename T, typename S, int L, int NC>
__global__ void __launch_bounds__(norm_threads<L>, L >= 256 ? 4 : 1) norm_bwd_kernel(const NormBwdK a) {
  constexpr int NT = norm_threads<L>, PER = NT / L;      // rows at a time
  __shared__ float red[2][2][L > 64 ? L / 64 : 1];
  __shared__ __attribute__((aligned(16))) float meet[PER > 1 ? NT * 8 : 8];
  const int l = threadIdx.x % L, sub = threadIdx.x / L, step = gridDim.x * PER;
  auto left = [&](int c) { return a.d - 8 * (c * L + l); };
  const DropKey key = drop_key(a.drop);
  float ga[NC][8], dg[NC][8], db[NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { ga[c][j] = 1.f; dg[c][j] = 0.f; db[c][j] = 0.f; }
    if (left(c) > 0 && a.gamma) row8_widen<T>(row8_load((const T*)a.gamma + 8 * (c * L + l), left(c)), ga[c]);
  }
  typename Row8<T>::value yv[NC];
  typename Row8<S>::value sv[NC], iv[NC];
  float mu, rs;
  auto fetch = [&](int row) {
    mu = a.mean[row];
    rs = a.rstd[row];
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (left(c) > 0) {
        const int col = 8 * (c * L + l);
        yv[c] = row8_load((const T*)a.dy + (size_t)row * a.lddy + col, left(c));
        sv[c] = row8_load((const S*)a.sum + (size_t)row * a.lds + col, left(c));
        if (a.dsum_in) iv[c] = row8_load((const S*)a.dsum_in + (size_t)row * a.ldi + col, left(c));
      }
  };
  // every wave makes as many turns as its workgroup's first row group: the row sums of a workgroup per row meet at barriers
  int row = blockIdx.x * PER + sub;
  fetch(min(row, a.rows - 1));
  int turn = 0;
  for (int base = blockIdx.x * PER; base < a.rows; base += step, row += step, turn ^= 1) {
    const bool live = row < a.rows;
    float g[NC][8], xh[NC][8], in[NC][8], s0 = 0.f, s1 = 0.f;
    const float r = rs;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (left(c) <= 0) continue;
      float sm[8];
      row8_widen<T>(yv[c], g[c]);
      row8_widen<S>(sv[c], sm);
      if (a.dsum_in) row8_widen<S>(iv[c], in[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool on = live && j < left(c);
        xh[c][j] = on ? (sm[j] - mu) * rs : 0.f;
        if (!live) g[c][j] = 0.f;
        dg[c][j] = fmaf(g[c][j], xh[c][j], dg[c][j]);
        db[c][j] += g[c][j];
        g[c][j] *= ga[c][j];
        s0 += g[c][j];
        s1 = fmaf(g[c][j], xh[c][j], s1);
      }
    }
    if (base + step < a.rows) fetch(min(row + step, a.rows - 1));
    const float m0 = norm_row_sum<L>(s0, red[turn][0]) / a.d, m1 = norm_row_sum<L>(s1, red[turn][1]) / a.d;
    if (!live) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (left(c) <= 0) continue;
      const int col = 8 * (c * L + l);
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = r * (g[c][j] - m0 - xh[c][j] * m1);
        if (a.dsum_in) o[j] += in[c][j];
      }
      if (a.dsum) row8_store((S*)a.dsum + (size_t)row * a.ldds + col, left(c), o);
      if (a.dx) {
        drop8(a.drop, key, c * L + l, row, o);
        row8_store((T*)a.dx + (size_t)row * a.lddx + col, left(c), o);
      }
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float (&v)[8] = which ? db[c] : dg[c];
      if constexpr (PER > 1) {      // lane l of the first group adds the groups' in their order
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; j += 4) *reinterpret_cast<f32x4*>(&meet[threadIdx.x * 8 + j]) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
        __syncthreads();
        if (sub == 0)
          for (int w = 1; w < PER; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += meet[(w * L + l) * 8 + j];
      }
      if (sub == 0 && left(c) > 0) row8_store(out + (size_t)which * a.d + 8 * (c * L + l), left(c), v);
    }
}

// Columns' sums of the workgroups' parts [parts][n]: 32 columns (a line of memory) and 32 shares of the parts a workgroup, the shares added in their order.
__global__ void __launch_bounds__(1024) norm_bwd_reduce_kernel(const float* __restrict__ partial, int parts, int d, float* __restrict__ dgamma,
                                                               float* __restrict__ dbeta, int accumulate) {
  __shared__ float meet[32][33];
  const int lane = threadIdx.x % 32, share = threadIdx.x / 32, col = blockIdx.x * 32 + lane, n = 2 * d;
  float s = 0.f;
  if (col < n) {
#pragma unroll 8
    for (int p = share; p < parts; p += 32) s += partial[(size_t)p * n + col];
  }
  meet[share][lane] = s;
  __syncthreads();
  if (share || col >= n) return;
  for (int w = 1; w < 32; ++w) s += meet[w][lane];
  float* out = col < d ? dgamma : dbeta;
  const int at = col < d ? col : col - d;
  if (!out) return;
  out[at] = accumulate ? out[at] + s : s;
}

// ------------------------------------------------------------------ host side
static int make_drop(float p, const uint64_t* rng, uint32_t site, uint32_t first_row, const char* who, DropK& k) {
  if (!(p >= 0.f) || !(p <= 1.f)) return set_errorf(DP_EINVAL, "%s: the probability must lie in [0, 1]", who);
  k = DropK{rng, (uint32_t)lrintf(p * 65536.f), site, first_row, 0.f};
  if (k.threshold < 65536) k.up = 65536.f / (float)(65536 - k.threshold);
  if (k.threshold == 0) return DP_OK;
  if (!rng) return set_errorf(DP_EINVAL, "%s: dropout needs the generator's state", who);
  if ((uintptr_t)rng % 8) return set_errorf(DP_EALIGN, "%s: the generator's state must be 8-byte aligned", who);
  return DP_OK;
}
static int check_rows(const void* p, int ld, int cols, const char* who, const char* what) {
  if (!p) return set_errorf(DP_EINVAL, "%s: %s is NULL", who, what);
  if ((uintptr_t)p % 16) return set_errorf(DP_EALIGN, "%s: %s is not 16-byte aligned", who, what);
  if (ld < cols) return set_errorf(DP_EINVAL, "%s: the row stride of %s is less than a row", who, what);
  return DP_OK;
}
static int check_vec(const void* p, const char* who, const char* what) {
  if ((uintptr_t)p % 16) return set_errorf(DP_EALIGN, "%s: %s is not 16-byte aligned", who, what);
  return DP_OK;
}
static int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DP_OK : set_errorf(DP_EHIP, "%s: launch failed (%s)", who, hipGetErrorString(e));
}

template <typename T> static int dropout_t(const DropoutK& k, hipStream_t s) {
  const uint64_t groups = (uint64_t)k.rows * k.groups;
  hipLaunchKernelGGL((dropout_kernel<T>), dim3((unsigned)((groups + 255) / 256)), dim3(256), 0, s, k);
  return launched("dp_op_dropout");
}

// f(lanes, chunks) by the width of a row: few lanes leave few steps of a sum between lanes, few chunks leave registers for rows in flight.  The backward keeps
// four more vectors of a row than the forward and goes to more lanes earlier.  us of the lines' two sides (bf16, fp32 residual and sum unless said):
//   forward   65536 x 128 (16, 1) 17.6, (32, 1) 19.9;  65536 x 256 (16, 2) 30.6, (32, 1) 30.8, (64, 1) 35.3;  16384 x 512 (32, 2) 16.9, (64, 1) 17.8, (16, 4) 18.5;
//             16384 x 768, bf16 sums (64, 2) 20.3, (32, 4) 20.4, (256, 1) 28.2;  8192 x 1152 (256, 1) 19.5, (64, 4) 21.8;  4096 x 2560 (256, 2) 21.8, (512, 1) 22.9;
//             4096 x 5000, bf16 sums (512, 2) 30.1, (256, 4) 31.5, (1024, 1) 35.0
//   backward  65536 x 128 (16, 1) 23.8, (32, 1) 29.1;  65536 x 256 (32, 1) 44.2, (16, 2) 46.0, (64, 1) 57.6;  32768 x 320 (64, 1) 29.8, (32, 2) 31.8, (16, 4) 45.9;
//             16384 x 512 (64, 1) 22.4, (32, 2) 24.9;  8192 x 1024 (64, 2) 25.0, (256, 1) 28.9, (32, 4) 38.4;  8192 x 1152 (256, 1) 25.6, (64, 3) 47.2
template <bool FORWARD, class F> static void norm_dispatch(int d, F f) {
  using std::integral_constant;
  auto with = [&](auto l, auto nc) { f(l, nc); };
  if (d <= 128) return with(integral_constant<int, 16>(), integral_constant<int, 1>());
  if (d > 512 && d <= 1024) return with(integral_constant<int, 64>(), integral_constant<int, 2>());
  if (d > 1024 && d <= 2048) return with(integral_constant<int, 256>(), integral_constant<int, 1>());
  if constexpr (FORWARD) {
    if (d <= 256) with(integral_constant<int, 16>(), integral_constant<int, 2>());
    else if (d <= 512) with(integral_constant<int, 32>(), integral_constant<int, 2>());
    else if (d <= 4096) with(integral_constant<int, 256>(), integral_constant<int, 2>());
    else with(integral_constant<int, 512>(), integral_constant<int, 2>());
  } else {
    if (d <= 256) with(integral_constant<int, 32>(), integral_constant<int, 1>());
    else if (d <= 512) with(integral_constant<int, 64>(), integral_constant<int, 1>());
    else if (d <= 4096) with(integral_constant<int, 512>(), integral_constant<int, 1>());
    else with(integral_constant<int, 1024>(), integral_constant<int, 1>());
  }
}
static int norm_rows_per_workgroup(int d) {
  int per = 1;
  norm_dispatch<false>(d, [&](auto l, auto) { per = norm_threads<l> / l; });
  return per;
}
static bool norm_too_many(int rows, int d) {      // a launch has less than 2^32 threads
  long lanes = 1;
  norm_dispatch<false>(d, [&](auto l, auto) { lanes = l; });
  return rows * lanes >= (1l << 31);
}
// Workgroups of the backward, hence parts to be added afterwards: as many as run at once.  That is two a CU where a lane has two groups of columns (half the
// registers of a SIMD each wave) or a row 512 lanes, four where it has 256, one for 1024; rows within a wave of one group take three, which leave fewer parts.  512 / 768 / 1024
// of them, us without the sum: 32768 x 320 29.6 / 27.8 / 28.0, 65536 x 256 43.1 / 42.2 / 43.6, 32768 x 640 67 / 81 / 69, 8192 x 640 21 / 23 / 23, 8192 x 1152 28 / 26 / 23; with the sum, 256
// or 512: 2048 x 8192 33 / 39, 1000 x 5000 fp32 23 / 29.  Few rows of a workgroup each would leave as many parts as rows: of 1 / 2 / 4 / 8 each, 512 x 1280 9.5 / 8.7 / 10.5 / 14.2, 1024 x
// 2048 15.7 / 12.6 / 12.3 / 16.4, 512 x 4096 15.8 / 13.2 / 13.7 / 18.3, 2048 x 2048 18.4 / 18.4 / 16.2 / 17.7; within a wave (1027 x 1001 fp32) 10.8 / 12.6 / 15.7.
static int norm_bwd_workgroups(int rows, int d, bool most = false) {      // (most: what this many rows or fewer leave)
  const int per = d <= 1024 || d > 4096 ? norm_rows_per_workgroup(d) : rows < 1024 || most ? 2 : 4;
  return std::min((rows + per - 1) / per, d <= 512 ? 768 : d <= 1024 ? 512 : d <= 2048 ? 1024 : d <= 4096 ? 512 : 256);
}
template <typename T, typename S> static int norm_fwd_t(const NormK& k, hipStream_t s) {
  norm_dispatch<true>(k.d, [&](auto l, auto nc) {
    constexpr int PER = norm_threads<l> / l;
    hipLaunchKernelGGL((norm_fwd_kernel<T, S, l, nc>), dim3((k.rows + PER - 1) / PER), dim3(norm_threads<l>), 0, s, k);
  });
  return launched("dp_op_layernorm_fwd");
}
template <typename T, typename S> static int norm_bwd_t(const NormBwdK& k, int workgroups, hipStream_t s) {
  norm_dispatch<false>(k.d, [&](auto l, auto nc) { hipLaunchKernelGGL((norm_bwd_kernel<T, S, l, nc>), dim3(workgroups), dim3(norm_threads<l>), 0, s, k); });
  return launched("dp_op_layernorm_bwd");
}

}  // namespace dp

using namespace dp;

extern "C" {

int dp_op_dropout(int dtype, int rows, int cols, const void* x, int ldx, const void* residual, int ldr, float p, const uint64_t* rng, uint32_t site,
                  uint32_t first_row, void* y, int ldy, void* hip_stream) {
  const char* who = "dp_op_dropout";
  if (dtype != DP_F32 && dtype != DP_BF16) return set_error(DP_EINVAL, "unknown dtype");
  if (rows < 0 || cols <= 0) return set_errorf(DP_EINVAL, "%s: bad size", who);
  DropoutK k{rows, cols, cols / 8 + (cols % 8 != 0), x, ldx, residual, ldr, y, ldy, {}};
  DP_TRY(make_drop(p, rng, site, first_row, who, k.drop));
  if (rows == 0) return DP_OK;
  DP_TRY(check_rows(x, ldx, cols, who, "x"));
  DP_TRY(check_rows(y, ldy, cols, who, "y"));
  if (residual) DP_TRY(check_rows(residual, ldr, cols, who, "residual"));
  if ((uint64_t)rows * k.groups >= (1ull << 31)) return set_errorf(DP_EUNSUPPORTED, "%s: 2^34 elements and more", who);      // (a launch has less than 2^32 threads)
  const int es = dtype == DP_BF16 ? 2 : 4;
  KScope ks(KK_OTHER, 0.0, (double)rows * cols * es * (residual ? 3 : 2), (hipStream_t)hip_stream, rows, cols);
  return dtype == DP_BF16 ? dropout_t<bf16>(k, (hipStream_t)hip_stream) : dropout_t<float>(k, (hipStream_t)hip_stream);
}

int dp_op_layernorm_fwd(int dtype, int sum_f32, int rows, int d, float eps, const void* x, int ldx, const void* residual, int ldr, float p,
                        const uint64_t* rng, uint32_t site, uint32_t first_row, const void* gamma, const void* beta, void* sum, int lds, void* y, int ldy,
                        float* mean, float* rstd, void* hip_stream) {
  const char* who = "dp_op_layernorm_fwd";
  if (dtype != DP_F32 && dtype != DP_BF16) return set_error(DP_EINVAL, "unknown dtype");
  if (rows < 0 || d <= 0) return set_errorf(DP_EINVAL, "%s: bad size", who);
  if (d > NORM_MAX_D) return set_errorf(DP_EUNSUPPORTED, "%s: rows of at most %d columns", who, NORM_MAX_D);
  if (norm_too_many(rows, d)) return set_errorf(DP_EUNSUPPORTED, "%s: too many rows", who);
  if (!(eps > 0.f) || !(eps < INFINITY)) return set_errorf(DP_EINVAL, "%s: eps must be positive and finite", who);
  if ((gamma == nullptr) != (beta == nullptr)) return set_errorf(DP_EINVAL, "%s: gamma and beta come together", who);
  NormK k{rows, d, eps, x, ldx, residual, ldr, gamma, beta, sum, lds, y, ldy, mean, rstd, {}};
  DP_TRY(make_drop(p, rng, site, first_row, who, k.drop));
  if (rows == 0) return DP_OK;
  DP_TRY(check_rows(x, ldx, d, who, "x"));
  DP_TRY(check_rows(y, ldy, d, who, "y"));
  if (residual) DP_TRY(check_rows(residual, ldr, d, who, "residual"));
  if (sum) DP_TRY(check_rows(sum, lds, d, who, "sum"));
  DP_TRY(check_vec(gamma, who, "gamma")); DP_TRY(check_vec(beta, who, "beta")); DP_TRY(check_vec(mean, who, "mean")); DP_TRY(check_vec(rstd, who, "rstd"));
  hipStream_t s = (hipStream_t)hip_stream;
  const int es = dtype == DP_BF16 ? 2 : 4, ss = dtype == DP_F32 || sum_f32 ? 4 : 2;
  KScope ks(KK_LN_FWD, 0.0, (double)rows * d * (2 * es + (residual ? ss : 0) + (sum ? ss : 0)) + 8.0 * rows, s, rows, d);
  if (dtype == DP_F32) return norm_fwd_t<float, float>(k, s);
  return sum_f32 ? norm_fwd_t<bf16, float>(k, s) : norm_fwd_t<bf16, bf16>(k, s);
}

size_t dp_op_layernorm_bwd_workspace_bytes(int rows, int d) {
  if (rows <= 0 || d <= 0 || d > NORM_MAX_D) return 0;
  return align_up((size_t)norm_bwd_workgroups(rows, d, true) * 2 * d * sizeof(float), 256);
}

int dp_op_layernorm_bwd(int dtype, int sum_f32, int rows, int d, const void* dy, int lddy, const void* sum, int lds, const float* mean,
                        const float* rstd, const void* gamma, const void* dsum_in, int ldi, float p, const uint64_t* rng, uint32_t site,
                        uint32_t first_row, void* dsum, int ldds, void* dx, int lddx, float* dgamma, float* dbeta, int accumulate, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  const char* who = "dp_op_layernorm_bwd";
  if (dtype != DP_F32 && dtype != DP_BF16) return set_error(DP_EINVAL, "unknown dtype");
  if (rows < 0 || d <= 0) return set_errorf(DP_EINVAL, "%s: bad size", who);
  if (d > NORM_MAX_D) return set_errorf(DP_EUNSUPPORTED, "%s: rows of at most %d columns", who, NORM_MAX_D);
  if (norm_too_many(rows, d)) return set_errorf(DP_EUNSUPPORTED, "%s: too many rows", who);
  NormBwdK k{rows, d, dy, lddy, sum, lds, mean, rstd, gamma, dsum_in, ldi, dsum, ldds, dx, lddx, nullptr, {}};
  DP_TRY(make_drop(p, rng, site, first_row, who, k.drop));
  if (rows > 0) {
    DP_TRY(check_rows(dy, lddy, d, who, "dy"));
    DP_TRY(check_rows(sum, lds, d, who, "sum"));
    DP_TRY(check_ptr(mean, "mean")); DP_TRY(check_ptr(rstd, "rstd"));
    if (dsum_in) DP_TRY(check_rows(dsum_in, ldi, d, who, "dsum_in"));
    if (dsum) DP_TRY(check_rows(dsum, ldds, d, who, "dsum"));
    if (dx) DP_TRY(check_rows(dx, lddx, d, who, "dx"));
    if (!dsum && !dx) return set_errorf(DP_EINVAL, "%s: neither dsum nor dx is wanted", who);
  }
  DP_TRY(check_vec(gamma, who, "gamma")); DP_TRY(check_vec(dgamma, who, "dgamma")); DP_TRY(check_vec(dbeta, who, "dbeta"));
  hipStream_t s = (hipStream_t)hip_stream;
  const int workgroups = rows > 0 ? norm_bwd_workgroups(rows, d) : 0, es = dtype == DP_BF16 ? 2 : 4, ss = dtype == DP_F32 || sum_f32 ? 4 : 2;
  if (rows > 0 && (dgamma || dbeta)) {
    const size_t need = dp_op_layernorm_bwd_workspace_bytes(rows, d);
    DP_TRY(check_ptr(workspace, "workspace", 256));
    if (workspace_bytes < need) return set_errorf(DP_EWORKSPACE, "%s: workspace too small (%zu bytes, needs %zu)", who, workspace_bytes, need);
    k.partial = (float*)workspace;
  }
  if (rows > 0) {
    KScope ks(KK_LN_BWD, 0.0, (double)rows * d * (es + ss + (dsum_in ? ss : 0) + (dsum ? ss : 0) + (dx ? es : 0)) + 8.0 * rows, s, rows, d);
    if (dtype == DP_F32) DP_TRY((norm_bwd_t<float, float>(k, workgroups, s)));
    else if (sum_f32) DP_TRY((norm_bwd_t<bf16, float>(k, workgroups, s)));
    else DP_TRY((norm_bwd_t<bf16, bf16>(k, workgroups, s)));
  }
  if (!dgamma && !dbeta) return DP_OK;
  KScope ks(KK_REDUCE, 0.0, (double)workgroups * 2 * d * 4, s, workgroups, d);
  hipLaunchKernelGGL(norm_bwd_reduce_kernel, dim3((2 * d + 31) / 32), dim3(1024), 0, s, k.partial, workgroups, d, dgamma, dbeta, accumulate != 0);
  return launched(who);
}

}  // extern "C"
