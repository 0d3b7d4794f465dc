// Attention with a learned relative position bias, forward and backward: S = scale Q K^T + table[bucket(key - query), head] under key lengths and an
// optional causal mask, O = softmax(S) V, and the gradients of Q, K, V and of the table.
//
// bf16: the tiles, operand layouts and splits of the kernels without a bias (dp_attention_tile.h): a wave owns 32 queries (forward, dQ) or 32 keys
// (dK / dV), scores come out of the matrix instruction with one query (key) a lane, and the other side streams through LDS in tiles of 64.
// P and dS are rounded to bf16 as operands of the second products (the instruction for fp32 has a sixteenth of the rate): each is off by up to 2^-8 of itself, at random, so that outputs are some 0.0022 of their size
// from 64 bits, of which their own rounding is 0.0017; sums, references, lse and the table's gradient are fp32.
// The bias costs these loops no vector instruction.  What the accumulators of the scores are cleared with otherwise is the bias over the scale:
//   - bias over distance lies in LDS (fp32) from the last distance at which the bucket still changes to the other one, and 96 distances
//     of the end buckets beyond either, as far as a tile that touches the middle reaches; four neighbouring accumulator registers are four neighbouring entries;
//   - a tile of 64 keys and 32 queries outside of the middle lies in one bucket: one number is its bias, for the accumulators or for the exponent.
// The table's gradient, the sum of dS over the pairs of a bucket: in the middle a wave adds its blocks of dS along their diagonals in registers (rel_diagonals),
// two vector additions an element, and keeps one sum a distance in LDS; beyond the middle each lane adds to one sum per side.  The sums over distances become
// sums over buckets at the end of the workgroup, and the first workgroups of the next launch add those of all samples and query tiles; every sum in a fixed order, so
// that the result is the same bits every time.  8 x 10 heads of 1024, dQ with this, causal: 134 us with an atomic addition in LDS for each element of dS
// (about 150 cycles an instruction), 44 laid down in LDS and added along the diagonals from there, 38 in registers (without the mask 58 and 47), 36 without turns of priority.
#include "dp_attention_tile.h"
#include "dp_device.h"
#include "dp_errors.h"
#include "dp_host.h"
#include "dp_kernels.h"
#include "dp_ktime.h"
#include "dp_relbias_buckets.h"

#include <math.h>
#include <string.h>
#include <algorithm>
#include <atomic>
#include <iterator>
#include <type_traits>

namespace dp {

constexpr int REL_MARGIN = 96;

struct RelAttnK {
  int B, H, Nq, Nk, dh, causal, query0;
  float scale, scale_log2, inv_scale;
  const void* q; int ldq;
  const void* k; int ldk;
  const void* v; int ldv;
  const void* table;
  const int* key_len;
  void* o; int ldo;
  float* lse;
  const void* dout; int lddo;
  float* delta;
  void* dq; int lddq;
  void* dk; int lddk;
  void* dv; int lddv;
  float* dtable_partial;      // [head][sample and query tile][bucket]
  float* dtable; int dtable_parts, dtable_add, table_items;      // the gradient, of how many parts a head, and whether it is added to
  int even;
  int qsplits; float* dkv_partial;      // shares of the queries, and what they leave of dK and dV, [dK, dV][share][key row][column]
  int ksplits; float* dq_partial;       // shares of the keys, and what they leave of dQ, [share][query row][column]
  int shares; float* part;      // few queries: shares of the keys, and what they leave: outputs [share][row][column], references and sums [share][row][2]
  RelBucketsK bk;
};

// Least distance of each bucket of a direction, and behind the last one more than any in the sums' reach: in LDS from a kernel's beginning, for its end.
constexpr int REL_STARTS = REL_MAX_BUCKETS + 8;
__device__ __forceinline__ void rel_fill_starts(const RelBucketsK& r, const RelStarts& st, uint16_t* starts, int threads) {
  for (int k = threadIdx.x; k <= r.per_side; k += threads) starts[k] = (uint16_t)rel_start(r, st, k);
}
__host__ __device__ __forceinline__ int rel_entries(const RelBucketsK& r) { return r.hi - r.lo + 1 + 2 * REL_MARGIN; }
__host__ __device__ __forceinline__ int rel_table_floats(const RelBucketsK& r) { return (rel_entries(r) + 3) / 4 * 4; }
// Keys of a sample that any query of the call sees: what lies behind is not read, so that a cache may be longer than what it holds.
__device__ __forceinline__ int rel_keys(const RelAttnK& p, int b) {
  const int seen = p.causal ? max(0, min(p.Nk, p.query0 + p.Nq)) : p.Nk;
  return p.key_len ? max(0, min(p.key_len[b], seen)) : seen;
}
// An entry of the table, times a factor.  At -65536 fp32 sums of score and entry are 1/256 apart; from there on an entry masks, as -infinity does, where a
// sum would have kept little of the score (and lse, from which the backward forms the probabilities again, little of the logarithm).
__device__ __forceinline__ float rel_entry(float v, float factor) { return v <= -65536.f ? -INFINITY : v * factor; }

// Bias of head h by distance, times a factor.  Entry e is distance lo - margin + e, or, REVERSED, hi + margin - e.  In two steps, so that the table's
// loads are on their way beside the first tiles': what a thread has of the first two rounds is requested first and stored behind the tiles' copies.  Distances less than any of
// the call's have the bias of the least: only queries of the last tile that do not exist meet them, whose probabilities (0 times the bias's exponential) would be NaN if the
// table held NaN or infinity there.
template <typename T, bool REVERSED, int THREADS> struct RelFill {
  T v[2];
  __device__ __forceinline__ T entry(const RelAttnK& p, const RelStarts& st, int h, int e) const {
    const int dist = max(REVERSED ? p.bk.hi + REL_MARGIN - e : p.bk.lo - REL_MARGIN + e, 1 - p.Nq - p.query0);
    return ((const T*)p.table)[(size_t)rel_bucket(p.bk, st, dist) * p.H + h];
  }
  __device__ __forceinline__ void request(const RelAttnK& p, const RelStarts& st, int h) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = threadIdx.x + i * THREADS;
      if (e < rel_entries(p.bk)) v[i] = entry(p, st, h, e);
    }
  }
  __device__ __forceinline__ void store(const RelAttnK& p, const RelStarts& st, int h, float* tab, float factor) const {
    const int n = rel_entries(p.bk);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = threadIdx.x + i * THREADS;
      if (e < n) tab[e] = rel_entry(to_f<T>(v[i]), factor);
    }
    for (int e = threadIdx.x + 2 * THREADS; e < n; e += THREADS) tab[e] = rel_entry(to_f<T>(entry(p, st, h, e)), factor);
  }
};
// The same in all lanes, hence in a scalar register
__device__ __forceinline__ float rel_uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }
// Four neighbouring entries
__device__ __forceinline__ f32x4 rel_read4(const float* t) { return f32x4{t[0], t[1], t[2], t[3]}; }

// Workgroup -> (tile, batch * head).  Without the causal mask that of the other attention kernels.  Under it tiles differ in length (the last tiles of
// queries and the first tiles of keys are the longest): they go by length over all heads, the longest first, so that the launch does not end with
// few workgroups on their longest tiles; and every second 256, which meet the first 256 on the same CUs, the other way round, in steps of eight, so that all tiles of a
// head still go to one XCD.
__device__ __forceinline__ void rel_block_map(const RelAttnK& p, int id, int ntiles, bool last_longest, int& tile, int& bh) {
  const int BH = p.B * p.H, full = BH / 8 * 8;
  if (!p.causal || id >= full * ntiles) {
    attn_block_map(id, ntiles, BH, tile, bh);
    return;
  }
  if ((id & 256) && (id | 255) < full * ntiles) id ^= 248;
  tile = id / full;
  bh = id % full;
  if (last_longest) tile = ntiles - 1 - tile;
}

// byte extent of n rows, which may be none
__device__ __forceinline__ uint32_t rel_slice_bytes(int n, int ld, int dh) { return (uint32_t)__builtin_amdgcn_readfirstlane(n > 0 ? (int)attn_slice_bytes(n, ld, dh) : 0); }

// Four columns of a query's output, unscaled, and (first column) the logarithm of its sum; m: reference of its exponentials (log2 domain).
template <typename T> __device__ __forceinline__ void rel_store_o(const RelAttnK& p, const f32x4& o, float sum, float m, int b, int h, int row, int col) {
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  typedef __attribute__((ext_vector_type(4))) T Four;
  Four v;
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = (T)(o[u] * inv);
  *reinterpret_cast<Four*>((T*)p.o + ((size_t)b * p.Nq + row) * p.ldo + h * p.dh + col) = v;
  if (p.lse && col == 0) p.lse[((size_t)b * p.H + h) * p.Nq + row] = sum == 0.f ? -INFINITY : fmaf(m, LN2, logf(sum));
}
// The same of a share of the keys: unscaled columns, and (first column) reference and sum, for rel_join_kernel.
__device__ __forceinline__ void rel_store_share(const RelAttnK& p, const f32x4& o, float sum, float m, int share, int bh, int row, int col) {
  const size_t rows = (size_t)p.B * p.H * p.Nq, at = share * rows + (size_t)bh * p.Nq + row;
  *reinterpret_cast<f32x4*>(p.part + at * p.dh + col) = o;
  if (col == 0) *reinterpret_cast<u32x2*>(p.part + p.shares * rows * p.dh + 2 * at) = u32x2{__builtin_bit_cast(uint32_t, m), __builtin_bit_cast(uint32_t, sum)};
}

// ------------------------------------------------------------------ forward (bf16)
// 128 queries a workgroup, keys in tiles of 64, two LDS stages; online softmax with a reference point that moves when the sum outgrows it (see
// attn_fwd_bf16_kernel).  8 x 5 heads of 4096 tokens 192 us, 8 x 10 of 1024 31 (without a bias 188 and 29); with the bias of the far tiles in the accumulators, sixteen moves a
// block, 203 and 33.  Bound by the vector work of the softmax between the products (the products of the former alone are 153 us at the rate of a large one).  A query that sees no key keeps the reference -inf and the sum 0: zeros, and lse = -inf.
template <int DHP, int KC, int MINW, bool SHARES>
__global__ void __launch_bounds__(256, MINW) rel_fwd_bf16_kernel(const RelAttnK p, const RelStarts st) {
  constexpr int DT = DHP / 32, BQ = 128, TILE = 64 * DHP;
  __shared__ __attribute__((aligned(1024))) bf16 Ks[2][TILE];
  __shared__ __attribute__((aligned(1024))) bf16 Vs[2][TILE];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int qtiles = (p.Nq + BQ - 1) / BQ, all = qtiles * p.B * p.H, share = SHARES ? (int)blockIdx.x / all : 0;
  int qtile, bh;
  rel_block_map(p, SHARES ? (int)blockIdx.x % all : (int)blockIdx.x, qtiles, true, qtile, bh);
  const int b = bh / p.H, h = bh % p.H;
  RelFill<bf16, false, 256> fill;
  fill.request(p, st, h);
  const int q0 = qtile * BQ + wave * 32, qi = q0 + l32, pos0 = p.query0 + q0, pos = pos0 + l32;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys;                                   // keys that this lane's query sees
  const int lim_all = p.causal ? min(keys, pos0 + 1) : keys;                              // ... that all queries of the wave see
  const int lim_wave = p.causal ? min(keys, pos0 + 32) : keys;                            // ... that some query of the wave sees
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * BQ + BQ)) : keys;  // ... of the workgroup
  const int tiles = __builtin_amdgcn_readfirstlane(lim_any > 0 ? (lim_any + 63) / 64 : 0);
  const int kt0 = SHARES ? (int)((long)tiles * share / p.shares) : 0, nkt = SHARES ? (int)((long)tiles * (share + 1) / p.shares) : tiles;
  const bf16* qb = (const bf16*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh;
  const u32x4 kr = make_raw_rsrc((const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, rel_slice_bytes(keys, p.ldk, p.dh));
  const u32x4 vr = make_raw_rsrc((const bf16*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh, rel_slice_bytes(keys, p.ldv, p.dh));

  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> ck, cv;
  ck.init(wave, lane, p.ldk, p.dh);
  cv.init(wave, lane, p.ldv, p.dh);
  if (kt0 < nkt) {
    ck.issue(kr, kt0 * 64, p.ldk, Ks[0], wave);
    cv.issue(vr, kt0 * 64, p.ldv, Vs[0], wave);
  }
  const int tab = 4 * g - pos - (bk_lo - REL_MARGIN);      // entry of this lane's first key

  bf16x8 qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qf[c] = ld8(qb + (size_t)qi * p.ldq + 16 * c + 8 * g, qi < p.Nq && 16 * c + 8 * g < p.dh);
  fill.store(p, st, h, rel_lds, p.inv_scale);
  f32x16 oacc[DT];
  float m = -INFINITY, lsum = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  wait_vmcnt<0>();
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);

  for (int kt = kt0; kt < nkt; ++kt) {
    const int buf = (kt - kt0) & 1;
    take_turns(p.even, kt);
    if (kt + 1 < nkt) {      // every wave left stage buf ^ 1 at the barrier that ended the previous iteration
      ck.issue(kr, (kt + 1) * 64, p.ldk, Ks[buf ^ 1], wave);
      cv.issue(vr, (kt + 1) * 64, p.ldv, Vs[buf ^ 1], wave);
    }
    f32x16 s[2];
    // Beyond the middle the products begin with zero, which the instruction has as a constant, and the bias goes into the exponent, one addition for all (not for a
    // tile that is masked throughout: there it may be anything).
    const bool middle = kt * 64 + 63 - pos0 > bk_lo && kt * 64 - pos0 - 31 < bk_hi;
    const float shift = middle || kt * 64 >= lim_wave ? 0.f : (kt * 64 - pos0 - 31 < bk_hi ? far_lo : far_hi) * p.scale_log2;
    auto scores = [&]() __attribute__((always_inline)) {      // S^T = K Q^T + bias, over the scale
      if (middle) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 v = rel_read4(rel_lds + (tab + kt * 64) + 32 * t + 8 * r4);
#pragma unroll
            for (int u = 0; u < 4; ++u) s[t][4 * r4 + u] = v[u];
          }
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mfma32(fo.row_frag(Ks[buf], t, 0), qf[0], s[t]);
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mfma32(fo.row_frag(Ks[buf], t, 0), qf[0], f32x16{});
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 1; c < KC; ++c) s[t] = mfma32(fo.row_frag(Ks[buf], t, c), qf[c], s[t]);
      if (kt * 64 + 64 > lim_all) {      // (one wave-uniform branch around a block of selects)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] = kt * 64 + 32 * t + acc_row(r, g) < lim ? s[t][r] : -INFINITY;
      }
    };
    float rs;
    auto probabilities = [&]() __attribute__((always_inline)) {
      const float mref = shift - (m == -INFINITY ? 0.f : m);
      rs = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[t][r], p.scale_log2, mref));
          s[t][r] = e;
          rs += e;
        }
    };
    auto move_reference = [&]() __attribute__((always_inline)) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
      mx = fmaxf(m, fmaf(reduce_halves(mx, MaxOp()), p.scale_log2, shift + 8.0f));
      if (kt > kt0) {
        const float alpha = __builtin_amdgcn_exp2f(m - (mx == -INFINITY ? 0.f : mx));
        lsum *= alpha;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
      }
      m = mx;
    };
    scores();
    if (kt == kt0) move_reference();
    probabilities();
    if (__any(!(rs <= 256.f) || m == -INFINITY)) {
      if (kt > kt0) {
        scores();
        move_reference();
        probabilities();
      }
    }
    lsum += rs;
#pragma unroll
    for (int t = 0; t < 2; ++t)      // O^T += V^T P^T
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const bf16x8 pf = pack8(s[t], 8 * cc);
#pragma unroll
        for (int i = 0; i < DT; ++i) oacc[i] = mfma32(fo.tr_frag(Vs[buf], 32 * t + 16 * cc, i), pf, oacc[i]);
      }
    wait_vmcnt<0>();
    __syncthreads();
  }

  lsum = reduce_halves(lsum, AddOp());      // (each lane summed its own keys)
  if (qi >= p.Nq) return;
  if (SHARES) {
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int col = 32 * i + 8 * r4 + 4 * g;
        if (col < p.dh) rel_store_share(p, f32x4{oacc[i][4 * r4], oacc[i][4 * r4 + 1], oacc[i][4 * r4 + 2], oacc[i][4 * r4 + 3]}, lsum, m, share, bh, qi, col);
      }
    return;
  }
  const float inv = lsum > 0.f ? 1.0f / lsum : (lsum == 0.f ? 0.f : lsum);      // (NaN stays)
  bf16* ob = (bf16*)p.o + ((size_t)b * p.Nq + qi) * p.ldo + h * p.dh;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int col = 32 * i + 8 * r4 + 4 * g;
      if (col < p.dh) {
        bf16x4 o;
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] = (bf16)(oacc[i][4 * r4 + u] * inv);
        *reinterpret_cast<bf16x4*>(ob + col) = o;
      }
    }
  if (p.lse && g == 0) p.lse[((size_t)b * p.H + h) * p.Nq + qi] = lsum == 0.f ? -INFINITY : fmaf(m, LN2, logf(lsum));
}

// ------------------------------------------------------------------ forward of few queries (bf16)
// A workgroup has 32 queries of a head and one share of its tiles of 64 keys, each wave every fourth tile of them: K straight from memory into the
// operand's registers, V through an LDS tile of the wave's own, both requested a tile ahead; nothing waits at a barrier before the waves' sums meet at the end.
// Bound by reading K and V, of which a wave keeps a tile each in flight: 16 x 12 heads, one query, 4000 keys 36 us (5.5 TB/s), keys of different lengths up to
// that 24 (4.1, the longest ends last), and 4 to 5 for joining.  Shares that go to as many tiles each, whatever the sample's length, 30.  With several shares each leaves its unscaled output, reference and sum,
// and rel_join_kernel adds them in their order.
template <int DHP, int KC>
__global__ void __launch_bounds__(256, DHP == 64 ? 2 : 1) rel_fwd_few_bf16_kernel(const RelAttnK p, const RelStarts st) {
  constexpr int DT = DHP / 32, TILE = 64 * DHP;
  __shared__ __attribute__((aligned(1024))) bf16 Vs[4][2][TILE];
  __shared__ float stat[4][2][32];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi, qtiles = (p.Nq + 31) / 32;
  // the shares and query tiles of a head next to each other in turns of eight: on one XCD
  int part, bh;
  attn_block_map(blockIdx.x, qtiles * p.shares, p.B * p.H, part, bh);
  const int qtile = part / p.shares, share = part % p.shares, b = bh / p.H, h = bh % p.H;
  RelFill<bf16, false, 256> fill;
  fill.request(p, st, h);
  const int qi = qtile * 32 + l32, pos0 = p.query0 + qtile * 32, pos = pos0 + l32;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys, lim_all = p.causal ? min(keys, pos0 + 1) : keys;
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * 32 + 32)) : keys;
  const int nkt = __builtin_amdgcn_readfirstlane(lim_any > 0 ? (lim_any + 63) / 64 : 0);
  const int first = (int)((long)nkt * share / p.shares) + wave, last = (int)((long)nkt * (share + 1) / p.shares);
  const bf16* kb = (const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh;
  const u32x4 vr = make_raw_rsrc((const bf16*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh, rel_slice_bytes(keys, p.ldv, p.dh));

  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> cv[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) cv[w].init(w, lane, p.ldv, p.dh);
  bf16x8 kn[2][KC];
  auto request = [&](int kt, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int key = kt * 64 + 32 * t + l32;
        kn[t][c] = ld8(kb + (size_t)key * p.ldk + 16 * c + 8 * g, key < keys && 16 * c + 8 * g < p.dh);
      }
#pragma unroll
    for (int w = 0; w < 4; ++w) cv[w].issue(vr, kt * 64, p.ldv, Vs[wave][buf], w);
  };
  if (first < last) request(first, 0);
  const int tab = 4 * g - pos - (bk_lo - REL_MARGIN);
  bf16x8 qf[KC];
  const bf16* qrow = (const bf16*)p.q + ((size_t)b * p.Nq + qi) * p.ldq + h * p.dh;
#pragma unroll
  for (int c = 0; c < KC; ++c) qf[c] = ld8(qrow + 16 * c + 8 * g, qi < p.Nq && 16 * c + 8 * g < p.dh);
  fill.store(p, st, h, rel_lds, p.inv_scale);
  f32x16 oacc[DT];
  float m = -INFINITY, lsum = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);

  auto tile = [&](int kt, auto bc) __attribute__((always_inline)) {
    constexpr int buf = bc();
    wait_vmcnt<0>();      // this wave's own tile has landed
    asm volatile("" ::: "memory");
    f32x16 s[2];
    if (kt * 64 + 63 - pos0 > bk_lo && kt * 64 - pos0 - 31 < bk_hi) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 v = rel_read4(rel_lds + (tab + kt * 64) + 32 * t + 8 * r4);
#pragma unroll
          for (int u = 0; u < 4; ++u) s[t][4 * r4 + u] = v[u];
        }
    } else {
      const float below = far_lo, above = far_hi, far = kt * 64 - pos0 - 31 < bk_hi ? below : above;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = far;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) s[t] = mfma32(kn[t][c], qf[c], s[t]);
    if (kt + 4 < last) request(kt + 4, buf ^ 1);
    if (kt * 64 + 64 > lim_all) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = kt * 64 + 32 * t + acc_row(r, g) < lim ? s[t][r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    mx = fmaxf(m, reduce_halves(mx, MaxOp()) * p.scale_log2);
    const float ref = mx == -INFINITY ? 0.f : mx, alpha = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    lsum *= alpha;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], p.scale_log2, -ref));
        lsum += s[t][r];
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const bf16x8 pf = pack8(s[t], 8 * cc);
#pragma unroll
        for (int i = 0; i < DT; ++i) oacc[i] = mfma32(fo.tr_frag(Vs[wave][buf], 32 * t + 16 * cc, i), pf, oacc[i]);
      }
    }
  };
  for (int kt = first; kt < last; kt += 8) {
    tile(kt, std::integral_constant<int, 0>());
    if (kt + 4 < last) tile(kt + 4, std::integral_constant<int, 1>());
  }

  // the four waves' outputs, over their common reference, in their order: [query][column] of each in its own V tiles
  lsum = reduce_halves(lsum, AddOp());
  if (g == 0) { stat[wave][0][l32] = m; stat[wave][1][l32] = lsum; }
  constexpr int OLD = DHP + 4;      // floats from query to query
  static_assert(32 * OLD * 4 <= 2 * TILE * 2, "a wave's output lies in its V tiles");
  float* mine = reinterpret_cast<float*>(Vs[wave][0]);
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *reinterpret_cast<f32x4*>(mine + l32 * OLD + 32 * i + 8 * r4 + 4 * g) = f32x4{oacc[i][4 * r4], oacc[i][4 * r4 + 1], oacc[i][4 * r4 + 2], oacc[i][4 * r4 + 3]};
  __syncthreads();
  for (int at = tid; at < 32 * (DHP / 4); at += 256) {
    const int q = at / (DHP / 4), col = at % (DHP / 4) * 4, row = qtile * 32 + q;
    if (row >= p.Nq || col >= p.dh) continue;
    float top = fmaxf(fmaxf(stat[0][0][q], stat[1][0][q]), fmaxf(stat[2][0][q], stat[3][0][q])), sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = __builtin_amdgcn_exp2f(stat[w][0][q] - (top == -INFINITY ? 0.f : top));
      sum = fmaf(a, stat[w][1][q], sum);
      const f32x4 v = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(Vs[w][0]) + q * OLD + col);
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = fmaf(a, v[u], o[u]);
    }
    if (p.shares > 1) rel_store_share(p, o, sum, top, share, bh, row, col);
    else rel_store_o<bf16>(p, o, sum, top, b, h, row, col);
  }
}

// The shares of few queries, over their common reference, in their order; four columns a thread.
template <typename T> __global__ void __launch_bounds__(256) rel_join_kernel(const RelAttnK p) {
  const int per_row = p.dh / 4;
  const size_t rows = (size_t)p.B * p.H * p.Nq, at = blockIdx.x * 256ul + threadIdx.x, srow = at / per_row;
  if (srow >= rows) return;
  const int col = (int)(at % per_row) * 4, bh = (int)(srow / p.Nq), row = (int)(srow % p.Nq);
  const float* stat = p.part + p.shares * rows * p.dh;
  float top = -INFINITY, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int first = 0; first < p.shares; first += 8) {      // eight shares' values at once, behind what there is already
    float m[8], l[8], most = top;
    f32x4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const size_t i = min(first + u, p.shares - 1) * rows + srow;
      m[u] = stat[2 * i];
      l[u] = stat[2 * i + 1];
      v[u] = *reinterpret_cast<const f32x4*>(p.part + i * p.dh + col);
      if (first + u >= p.shares) m[u] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) most = fmaxf(most, m[u]);
    const float ref = most == -INFINITY ? 0.f : most, keep = __builtin_amdgcn_exp2f(top - ref);
    top = most;
    sum *= keep;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= keep;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float a = __builtin_amdgcn_exp2f(m[u] - ref);
      if (first + u >= p.shares) continue;
      sum = fmaf(a, l[u], sum);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = fmaf(a, v[u][c], o[c]);
    }
  }
  rel_store_o<T>(p, o, sum, top, bh / p.H, bh % p.H, row, col);
}

// ------------------------------------------------------------------ dQ and the table's gradient (bf16)
// 128 queries a workgroup, keys in tiles of 64, two LDS stages; S and dP = dO V^T with a query a lane, dS = P (dP - delta), dQ += dS K; delta = rowsum(dO O) goes
// to the workspace for dK / dV.  8 x 10 heads of 1024 47 us, 8 x 5 of 4096 272, 8 x 10 of 1024 causal 36: three products a block (8 x 5 of 4096: 258 GF, 229 us at a
// large product's rate) and some ten vector instructions an element between them, of which the diagonals are two.  SHARES: a workgroup has one of ksplits shares of
// its key tiles and leaves an fp32 sum (rel_grad_shares has what it gives).
__device__ __forceinline__ bf16x8 rel_turned(bf16x8 v, bool turn) {      // -v
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] ^= turn ? 0x80008000u : 0u;
  return __builtin_bit_cast(bf16x8, w);
}
// Sums of dS over distances: [wave][half of the wave][entry].
__host__ __device__ __forceinline__ int rel_sum_stride(const RelBucketsK& r) { return (rel_entries(r) + 3) / 4 * 4; }
__host__ __device__ __forceinline__ int rel_sum_floats(const RelBucketsK& r, int waves) { return rel_table_floats(r) + 2 * waves * rel_sum_stride(r); }
// The sums of a block of dS (a lane: one query; register r: key 8 (r / 4) + r % 4, in the other half of the wave 4 more) along its diagonals, without leaving the
// registers.  In a row of 16 lanes key k of lane j lies on diagonal k - j = 16 c - m with m = (j - k) mod 16 and c one of three: a register, moved by k mod 16
// lanes inside the row, adds to the c of the lanes that stay inside, and moved the other way to the next c of those that left it, two additions with a lane shift
// each.  Then the rows of queries 0 .. 15 and 16 .. 31 exchange what belongs together: lane l has in `near` the sum of key - query = 4 g - l, in `next` that of 32
// more.  TURNED: queries 16 .. 31 have the other sign.  (With keys for lanes and queries for registers: of query - key.)
struct RelDiagonals { float near, next; };
template <bool TURNED> __device__ __forceinline__ RelDiagonals rel_diagonals(const f32x16& s, int lane) {
  float acc[3] = {0.f, 0.f, 0.f};
  static_for<16>([&](auto rc) {
    constexpr int r = rc(), key = 8 * (r / 4) + r % 4, c = key / 16, n = key % 16;
    if constexpr (n == 0) {
      acc[c] += s[r];
    } else {
      acc[c] += lane_dpp<0x100 + n>(s[r]);              // row_shl: from lane m + n
      acc[c + 1] += lane_dpp<0x110 + 16 - n>(s[r]);     // row_shr: from lane m + n - 16
    }
  });
  const bool second = lane & 16;
  const auto rows = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, acc[1]), __builtin_bit_cast(uint32_t, acc[1]), false, false);
  const uint32_t r0 = rows[0], r1 = rows[1];
  const float first1 = __builtin_bit_cast(float, r0), second1 = __builtin_bit_cast(float, r1);      // of either row, in both
  if constexpr (TURNED) return second ? RelDiagonals{-acc[0], first1 - acc[2]} : RelDiagonals{acc[0] - second1, acc[2]};
  return second ? RelDiagonals{acc[0], first1 + acc[2]} : RelDiagonals{acc[0] + second1, acc[2]};
}

// The end of a workgroup that summed dS (REVERSED: entry e is distance hi + margin - e): the waves' sums of a distance, then the distances of a bucket (eight lanes each), then what lay beyond the middle.
template <int NW, bool REVERSED>
__device__ __forceinline__ void rel_bucket_sums(const RelAttnK& p, const uint16_t* starts, float* sums, int sum_stride, float (*far_sums)[NW], float far_sum_lo,
                                                float far_sum_hi, float* out) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, entries = rel_entries(p.bk);
  far_sum_lo = wave_sum(far_sum_lo);
  far_sum_hi = wave_sum(far_sum_hi);
  if (lane == 0) { far_sums[0][wave] = far_sum_lo; far_sums[1][wave] = far_sum_hi; }
  __syncthreads();
  for (int e = tid; e < entries; e += 64 * NW) {
    float v = sums[e];
#pragma unroll
    for (int w = 1; w < 2 * NW; ++w) v += sums[w * sum_stride + e];
    sums[e] = v;
  }
  __syncthreads();
  const int first = p.bk.lo - REL_MARGIN, last = p.bk.hi + REL_MARGIN;
  for (int bucket = tid / 8; bucket < (p.bk.n_buckets + 8 * NW - 1) / (8 * NW) * (8 * NW); bucket += 8 * NW) {
    const bool on = bucket < p.bk.n_buckets;
    const int side = on && p.bk.bidirectional && bucket >= p.bk.per_side, k = on ? bucket - side * p.bk.per_side : 0;
    const int n0 = starts[k], n1 = starts[k + 1] - 1;      // distances n0 .. n1 of this direction
    int d0, d1;
    if (side) d0 = max(n0, 1), d1 = min(n1, last);
    else d0 = max(-n1, first), d1 = -n0;
    if (!p.bk.bidirectional && k == 0) d1 = last;        // keys behind the query
    float v = 0.f;
    if (on)
      for (int d = d0 + tid % 8; d <= d1; d += 8) v += sums[REVERSED ? last - d : d - first];
    v += lane_dpp<0xB1>(v);       // lanes i ^ 1, i ^ 2, i ^ 7 (by then equal within four): the eight of a bucket
    v += lane_dpp<0x4E>(v);
    v += lane_dpp<0x141>(v);      // row_half_mirror
    if (on && tid % 8 == 0) {
      const int lo_bucket = p.bk.per_side - 1, hi_bucket = p.bk.bidirectional ? 2 * p.bk.per_side - 1 : 0;
      float far[2] = {0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) far[0] += far_sums[0][w], far[1] += far_sums[1][w];
      if (bucket == lo_bucket) v += far[0];
      if (bucket == hi_bucket) v += far[1];
      out[bucket] = v;
    }
  }
}

template <int DHP, int KC, bool SHARES>
__global__ void __launch_bounds__(256, DHP == 64 ? 3 : 2) rel_bwd_dq_bf16_kernel(const RelAttnK p, const RelStarts st) {
  constexpr int DT = DHP / 32, TILE = 64 * DHP;
  __shared__ __attribute__((aligned(1024))) bf16 Ks[2][TILE];
  __shared__ __attribute__((aligned(1024))) bf16 Vs[2][TILE];
  __shared__ float far_sums[2][4];
  __shared__ uint16_t starts[REL_STARTS];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int qtiles = (p.Nq + 127) / 128, entries = rel_entries(p.bk), bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int all = qtiles * p.B * p.H, share = SHARES ? (int)blockIdx.x / all : 0;
  int qtile, bh;
  rel_block_map(p, SHARES ? (int)blockIdx.x % all : (int)blockIdx.x, qtiles, true, qtile, bh);
  const int b = bh / p.H, h = bh % p.H;
  RelFill<bf16, false, 256> fill;
  rel_fill_starts(p.bk, st, starts, 256);
  const int q0 = qtile * 128 + wave * 32, qi = q0 + l32, pos0 = p.query0 + q0, pos = pos0 + l32;
  const bool qok = qi < p.Nq;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys, lim_all = p.causal ? min(keys, pos0 + 1) : keys, lim_wave = p.causal ? min(keys, pos0 + 32) : keys;
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * 128 + 128)) : keys;
  const int tiles = __builtin_amdgcn_readfirstlane(lim_any > 0 ? (lim_any + 63) / 64 : 0);
  const int kt0 = SHARES ? (int)((long)tiles * share / p.ksplits) : 0, nkt = SHARES ? (int)((long)tiles * (share + 1) / p.ksplits) : tiles;
  const u32x4 kr = make_raw_rsrc((const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, rel_slice_bytes(keys, p.ldk, p.dh));
  const u32x4 vr = make_raw_rsrc((const bf16*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh, rel_slice_bytes(keys, p.ldv, p.dh));
  const bf16* qrow = (const bf16*)p.q + ((size_t)b * p.Nq + qi) * p.ldq + h * p.dh;
  const bf16* dorow = (const bf16*)p.dout + ((size_t)b * p.Nq + qi) * p.lddo + h * p.dh;

  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> ck, cv;
  ck.init(wave, lane, p.ldk, p.dh);
  cv.init(wave, lane, p.ldv, p.dh);
  if (kt0 < nkt) {
    ck.issue(kr, kt0 * 64, p.ldk, Ks[0], wave);
    cv.issue(vr, kt0 * 64, p.ldv, Vs[0], wave);
  }
  fill.request(p, st, h);
  fill.store(p, st, h, rel_lds, p.inv_scale);
  float* sums = rel_lds + rel_table_floats(p.bk);
  const int sum_stride = rel_sum_stride(p.bk);
  for (int e = tid; e < 8 * sum_stride; e += 256) sums[e] = 0.f;
  const int tab = 4 * g - pos - (p.bk.lo - REL_MARGIN);      // entry of this lane's first key
  float* const mine = sums + (2 * wave + g) * sum_stride;
  float carry = 0.f;      // sums of the block behind in the distances of the one ahead
  int carry_at = -1;
  float far_sum_lo = 0.f, far_sum_hi = 0.f;

  // The matrix instruction rounds downwards when it adds products to an accumulator, by some 1e-9 of dP's size: nothing for dQ, but the table's gradient
  // adds up millions of pairs whose signs cancel (8 x 10^-6 of it at 3 x 1620 x 1620).  The second sixteen queries therefore work with -dO, hence -delta
  // and -dS, and the errors cancel; the sign is put right where a query's results leave the lane.
  const bool second = lane & 16;
  bf16x8 qf[KC], dof[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const bool ok = qok && 16 * c + 8 * g < p.dh;
    qf[c] = ld8(qrow + 16 * c + 8 * g, ok);
    dof[c] = rel_turned(ld8(dorow + 16 * c + 8 * g, ok), second);
  }
  const size_t sidx = ((size_t)b * p.H + h) * p.Nq + qi;
  float lse2 = INFINITY;      // of no query, and of one that sees no key: its probabilities are zero
  if (qok) {
    const float l = p.lse[sidx];
    if (l != -INFINITY) lse2 = l * LOG2E;
  }
  float dlt = 0.f;      // delta = rowsum(dO * O), see attn_bwd_dq_bf16_kernel
  {
    const bf16* orow = (const bf16*)p.o + ((size_t)b * p.Nq + qi) * p.ldo + h * p.dh;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8 of = ld8(orow + 16 * c + 8 * g, qok && 16 * c + 8 * g < p.dh);
#pragma unroll
      for (int u = 0; u < 8; ++u) dlt = fmaf((float)of[u], (float)dof[c][u], dlt);
    }
    dlt = reduce_halves(dlt, AddOp());
    if (qok && g == 0 && share == 0) p.delta[sidx] = second ? -dlt : dlt;
  }
  f32x16 ndelta;
#pragma unroll
  for (int r = 0; r < 16; ++r) ndelta[r] = -dlt;
  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
  wait_vmcnt<0>();
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[entries - 1]);

  auto tile = [&](int kt, auto bc) {
    take_turns(p.even, kt);
    constexpr int buf = bc();
    if (kt + 1 < nkt) {
      ck.issue(kr, (kt + 1) * 64, p.ldk, Ks[buf ^ 1], wave);
      cv.issue(vr, (kt + 1) * 64, p.ldv, Vs[buf ^ 1], wave);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (kt * 64 + 32 * t >= lim_wave) continue;      // (masked throughout)
      const bool below = kt * 64 + 32 * t + 31 - pos0 <= bk_lo, above = kt * 64 + 32 * t - pos0 - 31 >= bk_hi;
      f32x16 s, dp;
      float minus = -lse2;
      if (below || above) {
        minus += (below ? far_lo : far_hi) * p.scale_log2;
        s = mfma32(fo.row_frag(Ks[buf], t, 0), qf[0], f32x16{});
      } else {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 v = rel_read4(rel_lds + (tab + kt * 64) + 32 * t + 8 * r4);
#pragma unroll
          for (int u = 0; u < 4; ++u) s[4 * r4 + u] = v[u];
        }
        s = mfma32(fo.row_frag(Ks[buf], t, 0), qf[0], s);
      }
      dp = mfma32(fo.row_frag(Vs[buf], t, 0), dof[0], ndelta);      // dP - delta: the products accumulate onto -delta
#pragma unroll
      for (int c = 1; c < KC; ++c) {
        s = mfma32(fo.row_frag(Ks[buf], t, c), qf[c], s);
        dp = mfma32(fo.row_frag(Vs[buf], t, c), dof[c], dp);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, minus)) * dp[r];
      if (kt * 64 + 32 * t + 32 > lim_all) {      // (here and not before the exponential: what is masked counts for nothing whatever it is)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = kt * 64 + 32 * t + acc_row(r, g) < lim ? s[r] : 0.f;
      }
      if (below || above) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += s[r];
        if (below) far_sum_lo += sum;
        else far_sum_hi += sum;
      } else {
        // blocks of the middle follow each other: every distance of this half of the wave is written once
        const RelDiagonals d = rel_diagonals<true>(s, lane);
        mine[tab + kt * 64 + 32 * t] = d.near + carry;
        carry = d.next;
        carry_at = kt * 64 + 32 * t + 32;
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const bf16x8 dsf = pack8(s, 8 * cc);
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = mfma32(fo.tr_frag(Ks[buf], 32 * t + 16 * cc, i), dsf, acc[i]);
      }
    }
    wait_vmcnt<0>();
    __syncthreads();
  };
  two_stages(kt0, nkt, tile);
  if (carry_at >= 0) mine[tab + carry_at] = carry;
  if (qok) {
    bf16* ob = (bf16*)p.dq + ((size_t)b * p.Nq + qi) * p.lddq + h * p.dh;
    float* of = SHARES ? p.dq_partial + (((size_t)share * p.B + b) * p.Nq + qi) * ((size_t)p.H * p.dh) + h * p.dh : nullptr;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int col = 32 * i + 8 * r4 + 4 * g;
        if (col < p.dh) {
          f32x4 v;
          bf16x4 o;
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] = acc[i][4 * r4 + u] * (second ? -p.scale : p.scale);
          if (SHARES) {
            *reinterpret_cast<f32x4*>(of + col) = v;
            continue;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) o[u] = (bf16)v[u];
          *reinterpret_cast<bf16x4*>(ob + col) = o;
        }
      }
  }
  if (p.dtable_partial) rel_bucket_sums<4, false>(p, starts, sums, sum_stride, far_sums, second ? -far_sum_lo : far_sum_lo, second ? -far_sum_hi : far_sum_hi, p.dtable_partial + ((((size_t)h * p.B + b) * (SHARES ? p.ksplits : 1) + share) * qtiles + qtile) * p.bk.n_buckets);
}

// dtable[bucket][head] = sum over the parts, in their order: 32 buckets of a head a workgroup (item: head, then which 32), eight shares of the parts.  Where a
// launch for dK and dV follows, its first workgroups do this beside the others; meet: 256 floats of LDS.
__device__ __forceinline__ void rel_table_sums(const RelAttnK& p, int item, float* meet) {
  const int n_buckets = p.bk.n_buckets, turns = (n_buckets + 31) / 32, h = item / turns, parts = p.dtable_parts;
  const int lane = threadIdx.x % 32, share = threadIdx.x / 32, bucket = item % turns * 32 + lane;
  if (h >= p.H) return;
  float s = 0.f;
  if (bucket < n_buckets) {
#pragma unroll 8
    for (int i = share; i < parts; i += 8) s += p.dtable_partial[((size_t)h * parts + i) * n_buckets + bucket];
  }
  meet[threadIdx.x] = s;
  __syncthreads();
  if (share || bucket >= n_buckets) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) s += meet[32 * w + lane];
  float* out = p.dtable + (size_t)bucket * p.H + h;
  *out = p.dtable_add ? *out + s : s;
}
__global__ void __launch_bounds__(256) rel_dtable_kernel(const RelAttnK p) {
  __shared__ float meet[256];
  rel_table_sums(p, blockIdx.x, meet);
}

// A wave's dK and dV (lane: key ki): fp32 parts of a query share, or the result; zeros for keys past the sample's length.
template <int DT>
__device__ __forceinline__ void rel_store_dkv(const RelAttnK& p, const f32x16 (&dkacc)[DT], const f32x16 (&dvacc)[DT], float dk_scale, int qs, int b, int h, int ki, bool kok, int g) {
  if (ki >= p.Nk) return;
  const size_t hd = (size_t)p.H * p.dh, rows = (size_t)p.B * p.Nk, row = (size_t)b * p.Nk + ki;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int col = 32 * i + 8 * r4 + 4 * g;
      if (col >= p.dh) continue;
      f32x4 k, v;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        k[u] = kok ? dkacc[i][4 * r4 + u] * dk_scale : 0.f;
        v[u] = kok ? dvacc[i][4 * r4 + u] : 0.f;
      }
      if (p.qsplits > 1) {
        float* pk = p.dkv_partial + (qs * rows + row) * hd + h * p.dh + col;
        *reinterpret_cast<f32x4*>(pk) = k;
        *reinterpret_cast<f32x4*>(pk + p.qsplits * rows * hd) = v;
      } else {
        bf16x4 k4, v4;
#pragma unroll
        for (int u = 0; u < 4; ++u) { k4[u] = (bf16)k[u]; v4[u] = (bf16)v[u]; }
        *reinterpret_cast<bf16x4*>((bf16*)p.dk + row * p.lddk + h * p.dh + col) = k4;
        *reinterpret_cast<bf16x4*>((bf16*)p.dv + row * p.lddv + h * p.dh + col) = v4;
      }
    }
}

// ------------------------------------------------------------------ dK, dV (bf16)
// Each wave owns 32 keys and walks the queries in tiles of 64, from the first that sees one of the workgroup's keys (see attn_bwd_dkv_bf16_kernel).  The
// bias is the addend of the exponent here, and lse what the scores begin with.  MINW: waves per SIMD, exactly; three have no registers for K, which they read from
// LDS again for every tile, nor for the causal mask, and leave 5 of width 64 (2 of 48) in scratch, of which 3 (none) are read again every second tile: 8 x 10 heads of 1024 72 -> 55 us, 8 x 5 of 4096 372 -> 343, 16 x 16 of 300 33 -> 27.  Four products a block bound
// it: 8 x 5 of 4096 are 344 GF, 305 us at a large product's rate.  SHARES: one of qsplits shares of the query tiles, as above.
template <int DHP, int KC, int MINW, bool SHARES>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(MINW, MINW))) rel_bwd_dkv_bf16_kernel(const RelAttnK p, const RelStarts st) {
  constexpr int DT = DHP / 32, TILE = 64 * DHP;
  __shared__ __attribute__((aligned(1024))) bf16 Qs[2][TILE];
  __shared__ __attribute__((aligned(1024))) bf16 Ds[2][TILE];
  constexpr bool KEPT = MINW == 2;
  __shared__ __attribute__((aligned(1024))) bf16 Kt[KEPT ? 8 : 2 * TILE];
  __shared__ __attribute__((aligned(16))) float lse_s[2][64];
  __shared__ __attribute__((aligned(16))) float dlt_s[2][64];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int ktiles = (p.Nk + 127) / 128, id = (int)blockIdx.x - p.table_items;
  if (id < 0) return rel_table_sums(p, (int)blockIdx.x, reinterpret_cast<float*>(Qs[0]));
  const bool causal = MINW == 2 && p.causal;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int all = ktiles * p.B * p.H, share = SHARES ? id / all : 0;
  int ktile, bh;
  rel_block_map(p, SHARES ? id % all : id, ktiles, false, ktile, bh);
  const int b = bh / p.H, h = bh % p.H;
  RelFill<bf16, true, 256> fill;
  const int k0 = ktile * 128 + wave * 32, ki = k0 + l32;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const bool kok = ki < keys;
  const u32x4 qr = make_raw_rsrc((const bf16*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh, attn_slice_bytes(p.Nq, p.ldq, p.dh));
  const u32x4 dr = make_raw_rsrc((const bf16*)p.dout + (size_t)b * p.Nq * p.lddo + h * p.dh, attn_slice_bytes(p.Nq, p.lddo, p.dh));
  const bf16* krow = (const bf16*)p.k + ((size_t)b * p.Nk + ki) * p.ldk + h * p.dh;
  const bf16* vrow = (const bf16*)p.v + ((size_t)b * p.Nk + ki) * p.ldv + h * p.dh;
  const float* lse_b = p.lse + ((size_t)b * p.H + h) * p.Nq;
  const float* dlt_b = p.delta + ((size_t)b * p.H + h) * p.Nq;

  const int tiles = __builtin_amdgcn_readfirstlane(ktile * 128 < keys ? (p.Nq + 63) / 64 : 0);      // (no query sees keys past the sample's length)
  const int seen = causal ? max(0, ktile * 128 - p.query0) / 64 : 0, ahead = max(0, tiles - seen);
  const int qt0 = SHARES ? seen + (int)((long)ahead * share / p.qsplits) : seen, nqt = SHARES ? seen + (int)((long)ahead * (share + 1) / p.qsplits) : tiles;
  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> cq, cd;
  cq.init(wave, lane, p.ldq, p.dh);
  cd.init(wave, lane, p.lddo, p.dh);
  if (qt0 < nqt) {
    cq.issue(qr, qt0 * 64, p.ldq, Qs[0], wave);
    cd.issue(dr, qt0 * 64, p.lddo, Ds[0], wave);
  }
  float stat = 0.f;      // of a query tile: wave 0 lse, wave 1 delta; as loaded until the end of the tile before
  const float* stat_b = wave == 0 ? lse_b : dlt_b;
  auto load_stats = [&](int qt) {
    if (wave < 2) stat = stat_b[min((uint32_t)(qt * 64 + lane), (uint32_t)p.Nq - 1u)];
  };
  auto store_stats = [&](int qt, int buf) {
    const bool ok = qt * 64 + lane < p.Nq;
    if (wave == 0) lse_s[buf][lane] = ok && stat != -INFINITY ? -stat * p.inv_scale : -INFINITY;      // (a query that sees no key has no probabilities)
    if (wave == 1) dlt_s[buf][lane] = ok ? -stat : 0.f;
  };
  load_stats(qt0);
  fill.request(p, st, h);
  fill.store(p, st, h, rel_lds, LOG2E);
  const int tab = 4 * g + p.query0 - ki + p.bk.hi + REL_MARGIN;      // entry of this lane's first query

  if constexpr (!KEPT) {
    const u32x4 kr = make_raw_rsrc((const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, rel_slice_bytes(keys, p.ldk, p.dh));
    AttnTileCopy<DHP> ck;
    ck.init(wave, lane, p.ldk, p.dh);
    ck.issue(kr, ktile * 128, p.ldk, Kt, wave);
    ck.issue(kr, ktile * 128 + 64, p.ldk, Kt + TILE, wave);
  }
  bf16x8 kf[KC], vf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const bool ok = kok && 16 * c + 8 * g < p.dh;
    if (KEPT) kf[c] = ld8(krow + 16 * c + 8 * g, ok);
    vf[c] = ld8(vrow + 16 * c + 8 * g, ok);
  }
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) { dkacc[i][r] = 0.f; dvacc[i][r] = 0.f; }
  store_stats(qt0, 0);
  wait_vmcnt<0>();
  __syncthreads();
  const float far_hi = rel_uniform(rel_lds[0]), far_lo = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);

  auto tile = [&](int qt, auto bc) {
    take_turns(p.even, qt);
    constexpr int buf = bc();
    const bool more = qt + 1 < nqt;
    if (more) {
      cq.issue(qr, (qt + 1) * 64, p.ldq, Qs[buf ^ 1], wave);
      cd.issue(dr, (qt + 1) * 64, p.lddo, Ds[buf ^ 1], wave);
      load_stats(qt + 1);
    }
    const int pos = p.query0 + qt * 64;      // of the tile's first query; distances k0 - pos - 63 .. k0 + 31 - pos
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (MINW > 2) __builtin_amdgcn_sched_barrier(0);      // (the halves' fragments would overlap in registers)
      if (causal && k0 > pos + 32 * t + 31) continue;
      const bool below = k0 + 31 - pos - 32 * t <= bk_lo, above = k0 - pos - 32 * t - 31 >= bk_hi;
      f32x16 s, dp;      // S less lse, over the scale, and dP less delta: the products accumulate onto them.  The bias is the addend of the exponent
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(&lse_s[buf][32 * t + 8 * r4 + 4 * g]), d4 = *reinterpret_cast<const f32x4*>(&dlt_s[buf][32 * t + 8 * r4 + 4 * g]);
#pragma unroll
        for (int u = 0; u < 4; ++u) { s[4 * r4 + u] = l4[u]; dp[4 * r4 + u] = d4[u]; }
      }
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        s = mfma32(fo.row_frag(Qs[buf], t, c), KEPT ? kf[c] : fo.row_frag(Kt + 32 * wave * DHP, 0, c), s);
        dp = mfma32(fo.row_frag(Ds[buf], t, c), vf[c], dp);
      }
      // a lane whose key is past the sample's length computes garbage that stays in its own accumulator columns, which are not stored
      if (below || above) {
        const float far = below ? far_lo : far_hi;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, far));
      } else {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 v = rel_read4(rel_lds + (tab + qt * 64) + 32 * t + 8 * r4);
#pragma unroll
          for (int u = 0; u < 4; ++u) s[4 * r4 + u] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + u], p.scale_log2, v[u]));
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= s[r];
      if (causal && k0 + 31 > pos + 32 * t) {      // (here and not before the exponential: what is masked counts for nothing whatever it is)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool seen = ki <= pos + 32 * t + acc_row(r, g);
          s[r] = seen ? s[r] : 0.f;
          dp[r] = seen ? dp[r] : 0.f;
        }
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const bf16x8 pf = pack8(s, 8 * cc);
        const bf16x8 dsf = pack8(dp, 8 * cc);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          dvacc[i] = mfma32(fo.tr_frag(Ds[buf], 32 * t + 16 * cc, i), pf, dvacc[i]);
          dkacc[i] = mfma32(fo.tr_frag(Qs[buf], 32 * t + 16 * cc, i), dsf, dkacc[i]);
        }
      }
    }
    if (MINW > 2) __builtin_amdgcn_sched_barrier(0);
    if (more) store_stats(qt + 1, buf ^ 1);
    wait_vmcnt<0>();
    __syncthreads();
  };
  two_stages(qt0, nqt, tile);
  rel_store_dkv<DT>(p, dkacc, dvacc, p.scale, share, b, h, ki, kok, g);
}

// ------------------------------------------------------------------ dQ, dK, dV of few heads (bf16)
// A workgroup has 32 queries (keys) of a head, and each of its waves every fourth tile of the other side, on LDS tiles of its own that it requests a tile ahead:
// nothing waits at a barrier before the waves' sums meet at the end (see rel_fwd_few_bf16_kernel).  With 128 queries (keys) a workgroup the chain is sixteen tiles of 1.2 us for
// 1024 of the other side, whatever few CUs have work (8 heads: 64); here it is four, on all: 8 heads of 1024 dQ 27 -> 16 us, dK / dV 27 -> 13 (chains bound both).
// A wave's result [32 rows][columns] in LDS, and four columns of the sum over the waves
template <int DHP> __device__ __forceinline__ void rel_few_leave(float* mine, const f32x16 (&acc)[DHP / 32], float factor, bool ok, int g, int l32) {
#pragma unroll
  for (int i = 0; i < DHP / 32; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 v;
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = ok ? acc[i][4 * r4 + u] * factor : 0.f;
      *reinterpret_cast<f32x4*>(mine + l32 * (DHP + 4) + 32 * i + 8 * r4 + 4 * g) = v;
    }
}
template <int DHP, int STRIDE> __device__ __forceinline__ void rel_few_meet(const float* first, int row, int col, bool share, float* partial, bf16* out) {      // STRIDE: floats from wave to wave
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(first + w * STRIDE + row * (DHP + 4) + col);
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] += v[u];
  }
  if (share) {
    *reinterpret_cast<f32x4*>(partial) = s;
    return;
  }
  bf16x4 o;
#pragma unroll
  for (int u = 0; u < 4; ++u) o[u] = (bf16)s[u];
  *reinterpret_cast<bf16x4*>(out) = o;
}

// Tiles of 64 keys: K through LDS, V by rows straight into registers.
template <int DHP, int KC>
__device__ __forceinline__ void rel_few_dq(const RelAttnK& p, const RelStarts& st, int block, bf16 (*Ks)[2][64 * DHP], float (*far_sums)[4], uint16_t* starts, float* rel_lds) {
  constexpr int DT = DHP / 32, TILE = 64 * DHP;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int qtiles = (p.Nq + 31) / 32, entries = rel_entries(p.bk), bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int all = qtiles * p.B * p.H, share = p.ksplits > 1 ? block / all : 0;
  int qtile, bh;
  rel_block_map(p, block - share * all, qtiles, true, qtile, bh);
  const int b = bh / p.H, h = bh % p.H;
  RelFill<bf16, false, 256> fill;
  fill.request(p, st, h);
  rel_fill_starts(p.bk, st, starts, 256);
  const int qi = qtile * 32 + l32, pos0 = p.query0 + qtile * 32, pos = pos0 + l32;
  const bool qok = qi < p.Nq;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys, lim_all = p.causal ? min(keys, pos0 + 1) : keys;
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * 32 + 32)) : keys;
  const int tiles = __builtin_amdgcn_readfirstlane(lim_any > 0 ? (lim_any + 63) / 64 : 0);
  const int first = (int)((long)tiles * share / p.ksplits) + wave, nkt = (int)((long)tiles * (share + 1) / p.ksplits);
  const u32x4 kr = make_raw_rsrc((const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, rel_slice_bytes(keys, p.ldk, p.dh));
  const bf16* vb = (const bf16*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh;
  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> ck[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) ck[w].init(w, lane, p.ldk, p.dh);
  bf16x8 vn[2][KC];
  auto request = [&](int kt, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int key = kt * 64 + 32 * t + l32;
        vn[t][c] = ld8(vb + (size_t)key * p.ldv + 16 * c + 8 * g, key < keys && 16 * c + 8 * g < p.dh);
      }
#pragma unroll
    for (int w = 0; w < 4; ++w) ck[w].issue(kr, kt * 64, p.ldk, Ks[wave][buf], w);
  };
  if (first < nkt) request(first, 0);
  const bool second = lane & 16;      // (see rel_bwd_dq_bf16_kernel)
  const size_t row = (size_t)b * p.Nq + qi, head = h * p.dh;
  bf16x8 qf[KC], dof[KC];
  float dlt = 0.f;
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const bool ok = qok && 16 * c + 8 * g < p.dh;
    qf[c] = ld8((const bf16*)p.q + row * p.ldq + head + 16 * c + 8 * g, ok);
    dof[c] = rel_turned(ld8((const bf16*)p.dout + row * p.lddo + head + 16 * c + 8 * g, ok), second);
    const bf16x8 of = ld8((const bf16*)p.o + row * p.ldo + head + 16 * c + 8 * g, ok);
#pragma unroll
    for (int u = 0; u < 8; ++u) dlt = fmaf((float)of[u], (float)dof[c][u], dlt);
  }
  dlt = reduce_halves(dlt, AddOp());
  const size_t sidx = ((size_t)b * p.H + h) * p.Nq + qi;
  float lse2 = INFINITY;      // of no query, and of one that sees no key: its probabilities are zero
  if (qok) {
    const float l = p.lse[sidx];
    if (l != -INFINITY) lse2 = l * LOG2E;
    if (tid < 32 && share == 0) p.delta[sidx] = second ? -dlt : dlt;
  }
  fill.store(p, st, h, rel_lds, p.inv_scale);
  float* sums = rel_lds + rel_table_floats(p.bk);
  const int sum_stride = rel_sum_stride(p.bk);
  for (int e = tid; e < 8 * sum_stride; e += 256) sums[e] = 0.f;
  const int tab = 4 * g - pos - (bk_lo - REL_MARGIN);      // entry of this lane's first key
  float* const mine = sums + (2 * wave + g) * sum_stride;
  float far_sum_lo = 0.f, far_sum_hi = 0.f;
  f32x16 ndelta, acc[DT];
#pragma unroll
  for (int r = 0; r < 16; ++r) ndelta[r] = -dlt;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[entries - 1]);

  auto tile = [&](int kt, auto bc) __attribute__((always_inline)) {
    constexpr int buf = bc();
    wait_vmcnt<0>();      // this wave's own tile has landed
    asm volatile("" ::: "memory");
    f32x16 s[2], dp[2];
    bool below[2], above[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int d0 = kt * 64 + 32 * t - pos0;
      below[t] = d0 + 31 <= bk_lo;
      above[t] = d0 - 31 >= bk_hi;
      if (below[t] || above[t]) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = below[t] ? far_lo : far_hi;
      } else {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 v = rel_read4(rel_lds + (tab + kt * 64) + 32 * t + 8 * r4);
#pragma unroll
          for (int u = 0; u < 4; ++u) s[t][4 * r4 + u] = v[u];
        }
      }
      dp[t] = mfma32(vn[t][0], dof[0], ndelta);
      s[t] = mfma32(fo.row_frag(Ks[wave][buf], t, 0), qf[0], s[t]);
#pragma unroll
      for (int c = 1; c < KC; ++c) {
        dp[t] = mfma32(vn[t][c], dof[c], dp[t]);
        s[t] = mfma32(fo.row_frag(Ks[wave][buf], t, c), qf[c], s[t]);
      }
    }
    if (kt + 4 < nkt) request(kt + 4, buf ^ 1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int k0 = kt * 64 + 32 * t;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], p.scale_log2, -lse2)) * dp[t][r];
      if (k0 + 32 > lim_all) {      // (here and not before the exponential: what is masked counts for nothing whatever it is)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = k0 + acc_row(r, g) < lim ? s[t][r] : 0.f;
      }
      if (below[t] || above[t]) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += s[t][r];
        if (below[t]) far_sum_lo += sum;
        else far_sum_hi += sum;
      } else {      // this wave's tiles lie 256 keys apart, and the two blocks of one share 32 distances
        const RelDiagonals d = rel_diagonals<true>(s[t], lane);
        mine[tab + k0] += d.near;
        mine[tab + k0 + 32] = d.next;
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const bf16x8 dsf = pack8(s[t], 8 * cc);
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = mfma32(fo.tr_frag(Ks[wave][buf], 32 * t + 16 * cc, i), dsf, acc[i]);
      }
    }
  };
  for (int kt = first; kt < nkt; kt += 8) {
    tile(kt, std::integral_constant<int, 0>());
    if (kt + 4 < nkt) tile(kt + 4, std::integral_constant<int, 1>());
  }
  static_assert(32 * (DHP + 4) * 4 <= 2 * TILE * 2, "a wave's result lies in its K tiles");
  asm volatile("" ::: "memory");
  rel_few_leave<DHP>(reinterpret_cast<float*>(Ks[wave][0]), acc, second ? -p.scale : p.scale, true, g, l32);
  __syncthreads();
  for (int at = tid; at < 32 * (DHP / 4); at += 256) {
    const int q = qtile * 32 + at / (DHP / 4), col = at % (DHP / 4) * 4;
    if (q >= p.Nq || col >= p.dh) continue;
    const size_t r = (size_t)b * p.Nq + q;
    rel_few_meet<DHP, TILE>(reinterpret_cast<const float*>(Ks[0][0]), at / (DHP / 4), col, p.ksplits > 1, p.dq_partial + ((size_t)share * p.B * p.Nq + r) * (p.H * p.dh) + head + col,
                            (bf16*)p.dq + r * p.lddq + head + col);
  }
  if (p.dtable_partial) rel_bucket_sums<4, false>(p, starts, sums, sum_stride, far_sums, second ? -far_sum_lo : far_sum_lo, second ? -far_sum_hi : far_sum_hi, p.dtable_partial + ((((size_t)h * p.B + b) * p.ksplits + share) * qtiles + qtile) * p.bk.n_buckets);
}

// Tiles of 32 queries: Q and dO through LDS, lse and delta a lane each.  OWN: delta = rowsum(dO O) formed here, not read.  QD: [wave][stage][Q, dO]; stats: -lse over the scale, -delta.
template <int DHP, int KC, bool OWN>
__device__ __forceinline__ void rel_few_dkv(const RelAttnK& p, const RelStarts& st, int id, bf16 (*QD)[2][2][32 * DHP], float (*stats)[64], float* rel_lds) {
  constexpr int DT = DHP / 32, TILE = 32 * DHP;
  const int ktiles = (p.Nk + 31) / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int all = ktiles * p.B * p.H, share = p.qsplits > 1 ? id / all : 0;
  int ktile, bh;
  rel_block_map(p, id - share * all, ktiles, false, ktile, bh);
  const int b = bh / p.H, h = bh % p.H, k0 = ktile * 32, ki = k0 + l32;
  RelFill<bf16, true, 256> fill;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const bool kok = ki < keys;
  const u32x4 qr = make_raw_rsrc((const bf16*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh, attn_slice_bytes(p.Nq, p.ldq, p.dh));
  const u32x4 dr = make_raw_rsrc((const bf16*)p.dout + (size_t)b * p.Nq * p.lddo + h * p.dh, attn_slice_bytes(p.Nq, p.lddo, p.dh));
  const float* stat_b = (g && !OWN ? p.delta : p.lse) + ((size_t)b * p.H + h) * p.Nq;
  const int seen = p.causal ? max(0, k0 - p.query0) / 32 : 0;
  const int tiles = __builtin_amdgcn_readfirstlane(k0 < keys ? max(0, (p.Nq + 31) / 32 - seen) : 0);      // (no query sees keys past the sample's length)
  const int first = seen + (int)((long)tiles * share / p.qsplits) + wave, nqt = seen + (int)((long)tiles * (share + 1) / p.qsplits);
  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  AttnTileCopy<DHP> cq[2], cd[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    cq[w].init(w, lane, p.ldq, p.dh);
    cd[w].init(w, lane, p.lddo, p.dh);
  }
  float stat = 0.f;
  bf16x8 on[KC];
  auto request = [&](int qt, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      cq[w].issue(qr, qt * 32, p.ldq, QD[wave][buf][0], w);
      cd[w].issue(dr, qt * 32, p.lddo, QD[wave][buf][1], w);
    }
    stat = stat_b[min(qt * 32 + l32, p.Nq - 1)];
    if (OWN) {
      const int q = qt * 32 + l32;
#pragma unroll
      for (int c = 0; c < KC; ++c) on[c] = ld8((const bf16*)p.o + ((size_t)b * p.Nq + q) * p.ldo + h * p.dh + 16 * c + 8 * g, q < p.Nq && 16 * c + 8 * g < p.dh);
    }
  };
  if (first < nqt) request(first, 0);
  bf16x8 kf[KC], vf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const bool ok = kok && 16 * c + 8 * g < p.dh;
    kf[c] = ld8((const bf16*)p.k + ((size_t)b * p.Nk + ki) * p.ldk + h * p.dh + 16 * c + 8 * g, ok);
    vf[c] = ld8((const bf16*)p.v + ((size_t)b * p.Nk + ki) * p.ldv + h * p.dh + 16 * c + 8 * g, ok);
  }
  fill.request(p, st, h);
  fill.store(p, st, h, rel_lds, LOG2E);
  const int tab = 4 * g + p.query0 - ki + bk_hi + REL_MARGIN;      // entry of this lane's first query
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) { dkacc[i][r] = 0.f; dvacc[i][r] = 0.f; }
  __syncthreads();
  const float far_hi = rel_uniform(rel_lds[0]), far_lo = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);

  auto tile = [&](int qt, auto bc) __attribute__((always_inline)) {
    constexpr int buf = bc();
    const bf16 *Q = QD[wave][buf][0], *D = QD[wave][buf][1];
    wait_vmcnt<0>();      // this wave's own tile has landed
    asm volatile("" ::: "memory");
    {
      const bool ok = qt * 32 + l32 < p.Nq;
      if (OWN) {
        float d = 0.f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const bf16x8 v = fo.row_frag(D, 0, c);
#pragma unroll
          for (int u = 0; u < 8; ++u) d = fmaf((float)on[c][u], (float)v[u], d);
        }
        d = reduce_halves(d, AddOp());
        stat = g ? d : stat;
      }
      if (g) stats[wave][lane] = ok ? -stat : 0.f;
      else stats[wave][lane] = ok && stat != -INFINITY ? -stat * p.inv_scale : -INFINITY;      // (a query that sees no key has no probabilities)
    }
    if (qt + 4 < nqt) request(qt + 4, buf ^ 1);
    const int pos = p.query0 + qt * 32;
    const bool below = k0 + 31 - pos <= bk_lo, above = k0 - pos - 31 >= bk_hi;
    f32x16 s, dp;
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(&stats[wave][8 * r4 + 4 * g]), d4 = *reinterpret_cast<const f32x4*>(&stats[wave][32 + 8 * r4 + 4 * g]);
#pragma unroll
      for (int u = 0; u < 4; ++u) { s[4 * r4 + u] = l4[u]; dp[4 * r4 + u] = d4[u]; }
    }
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      s = mfma32(fo.row_frag(Q, 0, c), kf[c], s);
      dp = mfma32(fo.row_frag(D, 0, c), vf[c], dp);
    }
    if (below || above) {
      const float far = below ? far_lo : far_hi;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, far));
    } else {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 v = rel_read4(rel_lds + (tab + qt * 32) + 8 * r4);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[4 * r4 + u] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + u], p.scale_log2, v[u]));
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] *= s[r];
    if (p.causal && k0 + 31 > pos) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool seen = ki <= pos + acc_row(r, g);
        s[r] = seen ? s[r] : 0.f;
        dp[r] = seen ? dp[r] : 0.f;
      }
    }
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      const bf16x8 pf = pack8(s, 8 * cc), dsf = pack8(dp, 8 * cc);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        dvacc[i] = mfma32(fo.tr_frag(D, 16 * cc, i), pf, dvacc[i]);
        dkacc[i] = mfma32(fo.tr_frag(Q, 16 * cc, i), dsf, dkacc[i]);
      }
    }
  };
  for (int qt = first; qt < nqt; qt += 8) {
    tile(qt, std::integral_constant<int, 0>());
    if (qt + 4 < nqt) tile(qt + 4, std::integral_constant<int, 1>());
  }
  static_assert(32 * (DHP + 4) * 4 <= 4 * TILE * 2, "a wave's result lies in its tiles");
  asm volatile("" ::: "memory");
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();
    rel_few_leave<DHP>(reinterpret_cast<float*>(QD[wave][0][0]), which ? dvacc : dkacc, which ? 1.0f : p.scale, kok, g, l32);
    __syncthreads();
    for (int at = tid; at < 32 * (DHP / 4); at += 256) {
      const int j = k0 + at / (DHP / 4), col = at % (DHP / 4) * 4;
      if (j >= p.Nk || col >= p.dh) continue;
      const size_t r = (size_t)b * p.Nk + j, c = h * p.dh + col;
      rel_few_meet<DHP, 2 * TILE>(reinterpret_cast<const float*>(QD[0][0][0]), at / (DHP / 4), col, p.qsplits > 1, p.dkv_partial + ((size_t)(which * p.qsplits + share) * p.B * p.Nk + r) * (p.H * p.dh) + c,
                                  (bf16*)(which ? p.dv : p.dk) + r * (which ? p.lddv : p.lddk) + c);
    }
  }
}

template <int DHP, int KC>
__global__ void __launch_bounds__(256, DHP == 64 ? 2 : 1) rel_bwd_few_dq_bf16_kernel(const RelAttnK p, const RelStarts st) {
  __shared__ __attribute__((aligned(1024))) bf16 Ks[4][2][64 * DHP];
  __shared__ float far_sums[2][4];
  __shared__ uint16_t starts[REL_STARTS];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  rel_few_dq<DHP, KC>(p, st, (int)blockIdx.x, Ks, far_sums, starts, rel_lds);
}
template <int DHP, int KC>
__global__ void __launch_bounds__(256, DHP == 64 ? 2 : 1) rel_bwd_few_dkv_bf16_kernel(const RelAttnK p, const RelStarts st) {
  __shared__ __attribute__((aligned(1024))) bf16 QD[4][2][2][32 * DHP];
  __shared__ __attribute__((aligned(16))) float stats[4][64];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int id = (int)blockIdx.x - p.table_items;
  if (id < 0) return rel_table_sums(p, (int)blockIdx.x, stats[0]);
  rel_few_dkv<DHP, KC, false>(p, st, id, QD, stats, rel_lds);
}
// Both at once, of so few workgroups that they all run beside each other: first those for dQ.
template <int DHP, int KC>
__global__ void __launch_bounds__(256, DHP == 64 ? 2 : 1) rel_bwd_few_both_bf16_kernel(const RelAttnK p, const RelStarts st, int dq_workgroups) {
  __shared__ __attribute__((aligned(1024))) bf16 tiles[4][2][64 * DHP];
  __shared__ __attribute__((aligned(16))) float stats[4][64];
  __shared__ float far_sums[2][4];
  __shared__ uint16_t starts[REL_STARTS];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  if ((int)blockIdx.x < dq_workgroups) rel_few_dq<DHP, KC>(p, st, (int)blockIdx.x, tiles, far_sums, starts, rel_lds);
  else rel_few_dkv<DHP, KC, true>(p, st, (int)blockIdx.x - dq_workgroups, reinterpret_cast<bf16 (*)[2][2][32 * DHP]>(tiles), stats, rel_lds);
}

// ------------------------------------------------------------------ dQ, dK, dV and the table's gradient at once (bf16, at most 32 NW keys)
// A workgroup has all keys of its (sample, head), 32 per wave, and walks the queries of its share in tiles of 64 (see attn_bwd_short_bf16_kernel): scores, dP and
// exponentials once instead of twice.  Per tile every wave adds to its keys' dK and dV, adds its dS along the diagonals and leaves it in LDS; behind a barrier the
// dQ of the tile is formed from it and the keys, while the next tile's delta is.  64 x 12 heads of 77 tokens 31 us (42 by the two kernels above), 32 x 16 of 256 and
// width 72 75 (101); the chain of a tile, two barriers long, bounds it.  The second sixteen keys of a wave work with -V, hence -delta and
// -dS (see rel_bwd_dq_bf16_kernel).  Wide heads leave 11 to 23 registers in scratch, fragments and offsets that every tile reads again.
template <int DHP, int NW> struct RelShort {
  static constexpr int TILE = 64 * DHP, K = 32 * NW * DHP, DS = 32 * NW * 64;                            // elements
  static_assert(K <= 2 * TILE + DS, "V passes through the second stage and dS");
  static constexpr int BYTES = (K + 4 * TILE + DS) * (int)sizeof(bf16) + (3 * 64 + 2 * NW + REL_STARTS / 2) * (int)sizeof(float);
};

template <int DHP, int KC, int NW>
__global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) rel_bwd_short_bf16_kernel(const RelAttnK p, const RelStarts st) {
  using S = RelShort<DHP, NW>;
  constexpr int DT = DHP / 32, TILE = S::TILE;
  constexpr int LPR = DHP == 64 ? 8 : 16, RPP = 64 / LPR, PASSES = 64 / (NW * RPP);      // delta: lanes a row, rows a pass of a wave
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  // what the products of every tile read comes first: an LDS instruction reaches 64 KB past its base register
  bf16* const QD = reinterpret_cast<bf16*>(smem);      // two stages of Q and dO
  bf16* const dS = QD + 4 * TILE;
  bf16* const Vt = QD + 2 * TILE;                      // V on its way to the registers: where the second stage and dS will be
  bf16* const Kt = dS + S::DS;
  float* const lse_s = reinterpret_cast<float*>(Kt + S::K);
  float* const dlt_s = lse_s + 64;                     // -delta, delta
  float (*const far_sums)[NW] = reinterpret_cast<float (*)[NW]>(dlt_s + 128);
  uint16_t* const starts = reinterpret_cast<uint16_t*>(dlt_s + 128 + 2 * NW);
  float* const rel_lds = dlt_s + 128 + 2 * NW + REL_STARTS / 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  int qs, bh;
  attn_block_map(blockIdx.x, p.qsplits, p.B * p.H, qs, bh);
  const int b = bh / p.H, h = bh % p.H, k0 = 32 * wave, ki = k0 + l32;
  RelFill<bf16, true, 64 * NW> fill;
  rel_fill_starts(p.bk, st, starts, 64 * NW);
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b)), groups = (keys + 31) / 32;      // (a wave past the last group has copies, dQ and delta)
  const bool kok = ki < keys, second = lane & 16;
  const bf16* ob = (const bf16*)p.o + (size_t)b * p.Nq * p.ldo + h * p.dh;
  const float* lse_b = p.lse + ((size_t)b * p.H + h) * p.Nq;
  const u32x4 qr = make_raw_rsrc((const bf16*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh, attn_slice_bytes(p.Nq, p.ldq, p.dh));
  const u32x4 dr = make_raw_rsrc((const bf16*)p.dout + (size_t)b * p.Nq * p.lddo + h * p.dh, attn_slice_bytes(p.Nq, p.lddo, p.dh));
  const u32x4 kr = make_raw_rsrc((const bf16*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, rel_slice_bytes(keys, p.ldk, p.dh));
  const u32x4 vr = make_raw_rsrc((const bf16*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh, rel_slice_bytes(keys, p.ldv, p.dh));
  const int nqt_all = (p.Nq + 63) / 64, tps = (nqt_all + p.qsplits - 1) / p.qsplits;
  const int qt0 = qs * tps, nqt = min(nqt_all, qt0 + tps);      // no share is empty

  AttnFragOff<DHP, KC> fo;
  fo.init(lane);
  // four waves copy a query tile of both kinds, eight one kind each
  AttnTileCopy<DHP> ck, cv, cq, cd;
  ck.init(wave, lane, p.ldk, p.dh);
  cv.init(wave, lane, p.ldv, p.dh);
  cq.init(wave & 3, lane, p.ldq, p.dh);
  cd.init(wave & 3, lane, p.lddo, p.dh);
  auto issue = [&](int qt) __attribute__((always_inline)) {
    const int at = (qt - qt0) & 1;
    if (NW == 4 || wave < 4) cq.issue(qr, qt * 64, p.ldq, QD + at * 2 * TILE, wave & 3);
    if (NW == 4 || wave >= 4) cd.issue(dr, qt * 64, p.lddo, QD + (at * 2 + 1) * TILE, wave & 3);
  };
  // O and the logarithms of the sums of a tile, kept as loaded until delta is due
  bf16x8 of[PASSES];
  float stat = 0.f;
  const int drow = wave * RPP + lane / LPR, dchunk = lane % LPR;
  auto load_o = [&](int qt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int q = qt * 64 + i * NW * RPP + drow;
      of[i] = ld8(ob + (size_t)q * p.ldo + 8 * dchunk, q < p.Nq && 8 * dchunk < p.dh);
    }
    if (wave == 0) stat = lse_b[min((uint32_t)(qt * 64 + lane), (uint32_t)p.Nq - 1u)];
  };
  auto statistics = [&](int qt) __attribute__((always_inline)) {
    const bf16* tile = QD + (((qt - qt0) & 1) * 2 + 1) * TILE;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int row = i * NW * RPP + drow;
      float v = 0.f;
      if (dchunk < DHP / 8) {
        const bf16x8 df = *reinterpret_cast<const bf16x8*>(tile + row * DHP + 8 * (dchunk ^ AttnTile<DHP>::key(row)));
#pragma unroll
        for (int u = 0; u < 8; ++u) v = fmaf((float)of[i][u], (float)df[u], v);
      }
      v += lane_dpp<0xB1>(v);       // quad_perm:[1,0,3,2]
      v += lane_dpp<0x4E>(v);       // quad_perm:[2,3,0,1]
      v += lane_dpp<0x141>(v);      // row_half_mirror: the other quad of eight
      if (LPR == 16) v += lane_dpp<0x128>(v);      // row_ror:8
      if (dchunk == 0) { dlt_s[row] = -v; dlt_s[64 + row] = v; }
    }
    if (wave == 0) lse_s[lane] = qt * 64 + lane < p.Nq && stat != -INFINITY ? stat * LOG2E : INFINITY;      // (a query that sees no key has no probabilities)
  };

  ck.issue(kr, 0, p.ldk, Kt, wave);
  cv.issue(vr, 0, p.ldv, Vt, wave);
  ck.issue(kr, 16 * NW, p.ldk, Kt + 16 * NW * DHP, wave);
  cv.issue(vr, 16 * NW, p.ldv, Vt + 16 * NW * DHP, wave);
  issue(qt0);
  load_o(qt0);
  fill.request(p, st, h);
  fill.store(p, st, h, rel_lds, p.inv_scale);
  float* const sums = rel_lds + rel_table_floats(p.bk);
  const int sum_stride = rel_sum_stride(p.bk);
  for (int e = tid; e < 2 * NW * sum_stride; e += 64 * NW) sums[e] = 0.f;
  const int tab = 4 * g + p.query0 - ki + bk_hi + REL_MARGIN;                                                 // entry of this lane's first query
  float* const mine = sums + (2 * wave + g) * sum_stride;
  float carry = 0.f;      // sums of the block behind in the distances of the one ahead
  int carry_at = -1;
  float far_sum_lo = 0.f, far_sum_hi = 0.f;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) { dkacc[i][r] = 0.f; dvacc[i][r] = 0.f; }
  wait_vmcnt<0>();
  __syncthreads();
  const float far_hi = rel_uniform(rel_lds[0]), far_lo = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);
  constexpr bool KEPT = DHP == 64;      // (wide heads have no registers for K as well, and read it again for every tile)
  bf16x8 kf[KC], vf[KC];      // rows past the last key are zero
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    if (KEPT) kf[c] = fo.row_frag(Kt + 32 * wave * DHP, 0, c);
    vf[c] = rel_turned(fo.row_frag(Vt + 32 * wave * DHP, 0, c), second);
  }
  statistics(qt0);
  lds_barrier();
  if (wave >= groups) {      // keys that are not there: the products for dQ run over all of them
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(dS + 32 * wave * 64 + 512 * i + 8 * lane) = u32x4{0u, 0u, 0u, 0u};
  }
  if (qt0 + 1 < nqt) {
    issue(qt0 + 1);
    load_o(qt0 + 1);
  }

  auto frag = [](const bf16* lo, const bf16* hi) {
    const bf16x4 a = lds_read_tr(lo), c = lds_read_tr(hi);
    return __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto tile = [&](int qt, auto bc) __attribute__((always_inline)) {
    const bf16* Q = QD + bc() * 2 * TILE;
    const bf16* D = Q + TILE;
    if (wave < groups) {
      const int pos = p.query0 + qt * 64;      // of the tile's first query
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool below = k0 + 31 - pos - 32 * t <= bk_lo, above = k0 - pos - 32 * t - 31 >= bk_hi;
        f32x16 s, dp;      // S over the scale; dP less delta, of the other sign for the second sixteen keys
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(dlt_s + (second ? 64 : 0) + 32 * t + 8 * r4 + 4 * g);
#pragma unroll
          for (int u = 0; u < 4; ++u) dp[4 * r4 + u] = d4[u];
        }
        if (below || above) {
          const float far = below ? far_lo : far_hi;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = far;
        } else {
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 v = rel_read4(rel_lds + (tab + qt * 64) + 32 * t + 8 * r4);
#pragma unroll
            for (int u = 0; u < 4; ++u) s[4 * r4 + u] = v[u];
          }
        }
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          s = mfma32(fo.row_frag(Q, t, c), KEPT ? kf[c] : fo.row_frag(Kt + 32 * wave * DHP, 0, c), s);
          dp = mfma32(fo.row_frag(D, t, c), vf[c], dp);
        }
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse_s + 32 * t + 8 * r4 + 4 * g);
#pragma unroll
          for (int u = 0; u < 4; ++u) s[4 * r4 + u] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + u], p.scale_log2, -l4[u]));
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] *= s[r];
        if (k0 + 32 > keys || (p.causal && k0 + 31 > pos + 32 * t)) {      // what is masked counts for nothing whatever it is
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool seen = kok && (!p.causal || ki <= pos + 32 * t + acc_row(r, g));
            s[r] = seen ? s[r] : 0.f;
            dp[r] = seen ? dp[r] : 0.f;
          }
        }
        if (below || above) {
          float sum = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += dp[r];
          if (below) far_sum_lo += sum;
          else far_sum_hi += sum;
        } else {
          const RelDiagonals d = rel_diagonals<true>(dp, lane);
          mine[tab + qt * 64 + 32 * t] = d.near + carry;
          carry = d.next;
          carry_at = qt * 64 + 32 * t + 32;
        }
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const bf16x8 pf = pack8(s, 8 * cc), dsf = pack8(dp, 8 * cc);
          const bf16x8 out = rel_turned(dsf, second);
#pragma unroll
          for (int q4 = 0; q4 < 2; ++q4) {
            const bf16x4 v = q4 ? __builtin_shufflevector(out, out, 4, 5, 6, 7) : __builtin_shufflevector(out, out, 0, 1, 2, 3);
            *reinterpret_cast<u32x2*>(dS + ki * 64 + 8 * ((4 * t + 2 * cc + q4) ^ AttnTile<64>::key(l32)) + 4 * g) = __builtin_bit_cast(u32x2, v);
          }
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            dvacc[i] = mfma32(fo.tr_frag(D, 32 * t + 16 * cc, i), pf, dvacc[i]);
            dkacc[i] = mfma32(fo.tr_frag(Q, 32 * t + 16 * cc, i), dsf, dkacc[i]);
          }
        }
      }
    }
    wait_vmcnt<0>();
    __syncthreads();      // dS is there, and the next tile
    const bool more = qt + 1 < nqt;
    if (more) statistics(qt + 1);
    if (qt + 2 < nqt) {
      issue(qt + 2);
      load_o(qt + 2);
    }
    // dQ of the tile: blocks of 32 columns (di) x 32 queries (dt)
    for (int n = wave; n < 2 * DT; n += NW) {
      const int di = n % DT, dt = n / DT;
      int kt_lo, kt_hi, ds_lo, ds_hi;
      AttnFragOff<DHP, KC>::transposed(lane, di, kt_lo, kt_hi);
      AttnFragOff<64, KC>::transposed(lane, dt, ds_lo, ds_hi);
      f32x16 acc;
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
      for (int r = 0; r < 32 * NW; r += 16) acc = mfma32(frag(Kt + kt_lo + r * DHP, Kt + kt_hi + r * DHP), frag(dS + ds_lo + r * 64, dS + ds_hi + r * 64), acc);
      const int q = qt * 64 + 32 * dt + l32;
      if (q < p.Nq) {
        bf16* o = (bf16*)p.dq + ((size_t)b * p.Nq + q) * p.lddq + h * p.dh;
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int col = 32 * di + 8 * r4 + 4 * g;
          if (col < p.dh) {
            bf16x4 v;
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = (bf16)(acc[4 * r4 + u] * p.scale);
            *reinterpret_cast<bf16x4*>(o + col) = v;
          }
        }
      }
    }
    lds_barrier();      // dS has been read, the statistics of the next tile are there
  };
  two_stages(qt0, nqt, tile);
  if (carry_at >= 0) mine[tab + carry_at] = carry;
  rel_store_dkv<DT>(p, dkacc, dvacc, second ? -p.scale : p.scale, qs, b, h, ki, kok, g);
  if (p.dtable_partial)
    rel_bucket_sums<NW, true>(p, starts, sums, sum_stride, far_sums, second ? -far_sum_lo : far_sum_lo, second ? -far_sum_hi : far_sum_hi,
                              p.dtable_partial + ((size_t)h * p.B * p.qsplits + (size_t)b * p.qsplits + qs) * p.bk.n_buckets);
}

// What the shares leave of dQ, and of dK and dV, added in their order; four columns a thread.
template <typename T> __device__ __forceinline__ void rel_join_rows(const float* part, int shares, size_t rows, int cols, size_t at, T* out, int ld) {
  const size_t row = at / cols, col = at % cols;
  f32x4 s = *reinterpret_cast<const f32x4*>(part + at);
#pragma unroll 4
  for (int q = 1; q < shares; ++q) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(part + q * rows * cols + at);
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] += v[u];
  }
  typedef __attribute__((ext_vector_type(4))) T Four;
  Four o;
#pragma unroll
  for (int u = 0; u < 4; ++u) o[u] = (T)s[u];
  *reinterpret_cast<Four*>(out + row * ld + col) = o;
}
static size_t rel_join_workgroups(int B, int N, int H, int d_head) { return ((size_t)B * N * H * d_head / 4 + 255) / 256; }
template <typename T> __global__ void __launch_bounds__(256) rel_join_grads_kernel(const RelAttnK p, unsigned dq_workgroups) {
  __shared__ float meet[256];
  if ((int)blockIdx.x < p.table_items) return rel_table_sums(p, (int)blockIdx.x, meet);
  const unsigned id = blockIdx.x - p.table_items;
  const int hd = p.H * p.dh;
  const size_t at = ((id < dq_workgroups ? id : id - dq_workgroups) * 256ul + threadIdx.x) * 4;
  if (id < dq_workgroups) {
    const size_t rows = (size_t)p.B * p.Nq;
    if (at < rows * hd) rel_join_rows(p.dq_partial, p.ksplits, rows, hd, at, (T*)p.dq, p.lddq);
    return;
  }
  const size_t rows = (size_t)p.B * p.Nk;
  if (at >= rows * hd) return;
  rel_join_rows(p.dkv_partial, p.qsplits, rows, hd, at, (T*)p.dk, p.lddk);
  rel_join_rows(p.dkv_partial + p.qsplits * rows * hd, p.qsplits, rows, hd, at, (T*)p.dv, p.lddv);
}

// ------------------------------------------------------------------ fp32
// v_mfma_f32_32x32x2_f32: A row l % 32, k = l / 32; B column l % 32, k = l / 32; D as in bf16.  Any order of the contraction does as long as both operands
// follow it: over the head's columns step 4 c + u is column 8 c + 4 g + u (a lane's operands are 16 bytes of a row), over keys or queries step r is row acc_row(r, g),
// which makes register r of the scores the B operand as it stands and the A operand a row of which 32 lanes read neighbouring columns.  So nothing goes
// through LDS on its way in: an instruction takes 64 cycles, several loads' time.
// A workgroup has 32 queries (forward, dQ) or 32 keys (dK / dV) of a head; its four waves take every fourth tile of 32 of the other side and
// add what they have in LDS at the end, in their order.  Bound by the matrix instruction where there is work for all CUs, else by the chain of tiles: 2 x 8 heads of
// 1024, width 64, forward 59 us (73 TF/s of 153), dQ 83, dK / dV 109.  Few heads go in shares (rel_shares_f32).  Rows a tile ahead in registers, where there are any
// (widths to 64): 102 -> 90 and 127 -> 118 us.
__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <int KC> struct RelRows {      // a lane's 16-byte pieces of one row
  f32x4 v[KC];
  __device__ __forceinline__ void load(const float* base, int row, int ld, int dh, int g) {
    const float* r = base + (size_t)row * ld + 4 * g;
#pragma unroll
    for (int c = 0; c < KC; ++c) v[c] = 8 * c + 4 * g < dh ? *reinterpret_cast<const f32x4*>(r + 8 * c) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
};
// D += rows of a (A) times rows of b (B), over the head's columns
template <int KC> __device__ __forceinline__ f32x16 rel_rows_product(const RelRows<KC>& a, const RelRows<KC>& b, f32x16 acc) {
#pragma unroll
  for (int c = 0; c < KC; ++c)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc = mfma_f32(a.v[c][u], b.v[c][u], acc);
  return acc;
}
template <int DT> struct RelColumns {      // columns 32 i + l32 of the rows acc_row(r, g) of a tile
  float v[DT][16];
  __device__ __forceinline__ void load(const float* base, int row0, int last_row, int ld, int dh, int g, int l32) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float* row = base + (size_t)min(row0 + acc_row(r, g), last_row) * ld;
#pragma unroll
      for (int i = 0; i < DT; ++i) v[i][r] = row[min(32 * i + l32, dh - 1)];      // (rows of the result past the head are not stored)
    }
  }
};
template <int DT> __device__ __forceinline__ void rel_columns_product(const RelColumns<DT>& a, const f32x16& b, f32x16 (&acc)[DT]) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = mfma_f32(a.v[i][r], b[r], acc[i]);
}
// A wave's result [32 rows][columns] in LDS, and four columns of the sum over the waves, each times its weight
template <int DT> constexpr int REL_F32_LD = 32 * DT + 4;
template <int DT> constexpr int REL_F32_MEET = 4 * 32 * REL_F32_LD<DT>;      // floats
template <int DT> __device__ __forceinline__ void rel_leave(float* meet, const f32x16 (&acc)[DT], int wave, int g, int l32) {
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *reinterpret_cast<f32x4*>(meet + (32 * wave + l32) * REL_F32_LD<DT> + 32 * i + 8 * r4 + 4 * g) = f32x4{acc[i][4 * r4], acc[i][4 * r4 + 1], acc[i][4 * r4 + 2], acc[i][4 * r4 + 3]};
}
template <int DT> __device__ __forceinline__ f32x4 rel_meet(const float* meet, int row, int col, const float (&weight)[4]) {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(meet + (32 * w + row) * REL_F32_LD<DT> + col);
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] = fmaf(weight[w], v[u], o[u]);
  }
  return o;
}
// Scores of a tile begin with the bias over the scale
__device__ __forceinline__ f32x16 rel_bias16(const float* lds, int entry) {
  f32x16 s;
#pragma unroll
  for (int r4 = 0; r4 < 4; ++r4) {
    const f32x4 v = rel_read4(lds + entry + 8 * r4);
#pragma unroll
    for (int u = 0; u < 4; ++u) s[4 * r4 + u] = v[u];
  }
  return s;
}
__device__ __forceinline__ f32x16 rel_all16(float v) {
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = v;
  return s;
}

template <int DT, int KC>
__global__ void __launch_bounds__(256) rel_fwd_f32_kernel(const RelAttnK p, const RelStarts st) {
  __shared__ __attribute__((aligned(16))) float meet[REL_F32_MEET<DT>];
  __shared__ float stat[4][2][32];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int qtiles = (p.Nq + 31) / 32, all = qtiles * p.B * p.H, share = p.shares > 1 ? (int)blockIdx.x / all : 0;
  int qtile, bh;
  rel_block_map(p, (int)blockIdx.x - share * all, qtiles, true, qtile, bh);
  const int b = bh / p.H, h = bh % p.H, qi = qtile * 32 + l32, pos0 = p.query0 + qtile * 32, pos = pos0 + l32;
  RelFill<float, false, 256> fill;
  fill.request(p, st, h);
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys, lim_all = p.causal ? min(keys, pos0 + 1) : keys;
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * 32 + 32)) : keys, tiles = lim_any > 0 ? (lim_any + 31) / 32 : 0;
  const int first = (int)((long)tiles * share / p.shares) + wave, nkt = (int)((long)tiles * (share + 1) / p.shares);
  const float* kb = (const float*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh;
  const float* vb = (const float*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh;
  RelRows<KC> q, k;
  q.load((const float*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh, min(qi, p.Nq - 1), p.ldq, p.dh, g);
  if (first < nkt) k.load(kb, min(32 * first + l32, keys - 1), p.ldk, p.dh, g);
  fill.store(p, st, h, rel_lds, p.inv_scale);
  const int tab = 4 * g - pos - (bk_lo - REL_MARGIN);      // entry of this lane's first key
  f32x16 oacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) oacc[i] = rel_all16(0.f);
  float m = -INFINITY, lsum = 0.f;
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);
  for (int kt = first; kt < nkt; kt += 4) {
    const int k0 = 32 * kt;
    RelColumns<DT> v;
    v.load(vb, k0, keys - 1, p.ldv, p.dh, g, l32);
    const bool below = k0 + 31 - pos0 <= bk_lo, above = k0 - pos0 - 31 >= bk_hi;
    f32x16 s = below ? rel_all16(far_lo) : (above ? rel_all16(far_hi) : rel_bias16(rel_lds, tab + k0));
    s = rel_rows_product(k, q, s);
    if (kt + 4 < nkt) k.load(kb, min(k0 + 128 + l32, keys - 1), p.ldk, p.dh, g);
    if (k0 + 32 > lim_all) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = k0 + acc_row(r, g) < lim ? s[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = fmaxf(m, reduce_halves(mx, MaxOp()) * p.scale_log2);
    const float ref = mx == -INFINITY ? 0.f : mx, alpha = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    lsum *= alpha;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -ref));
      lsum += s[r];
    }
    rel_columns_product(v, s, oacc);
  }
  lsum = reduce_halves(lsum, AddOp());
  if (g == 0) { stat[wave][0][l32] = m; stat[wave][1][l32] = lsum; }
  rel_leave(meet, oacc, wave, g, l32);
  __syncthreads();
  for (int at = tid; at < 32 * 8 * DT; at += 256) {
    const int row = at / (8 * DT), col = at % (8 * DT) * 4, i = qtile * 32 + row;
    if (i >= p.Nq || col >= p.dh) continue;
    const float top = fmaxf(fmaxf(stat[0][0][row], stat[1][0][row]), fmaxf(stat[2][0][row], stat[3][0][row])), ref = top == -INFINITY ? 0.f : top;
    float a[4], sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      a[w] = __builtin_amdgcn_exp2f(stat[w][0][row] - ref);
      sum = fmaf(a[w], stat[w][1][row], sum);
    }
    const f32x4 o = rel_meet<DT>(meet, row, col, a);
    if (p.shares > 1) rel_store_share(p, o, sum, top, share, bh, i, col);
    else rel_store_o<float>(p, o, sum, top, b, h, i, col);
  }
}

// (block: the workgroup among those for dQ; meet: REL_F32_MEET floats)
template <int DT, int KC>
__device__ __forceinline__ void rel_dq_f32(const RelAttnK& p, const RelStarts& st, int block, float* meet, float (*far_sums)[4], uint16_t* starts, float* rel_lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi, qtiles = (p.Nq + 31) / 32, entries = rel_entries(p.bk);
  const int all = qtiles * p.B * p.H, share = p.ksplits > 1 ? block / all : 0;
  int qtile, bh;
  rel_block_map(p, block - share * all, qtiles, true, qtile, bh);
  const int b = bh / p.H, h = bh % p.H, qi = qtile * 32 + l32, pos0 = p.query0 + qtile * 32, pos = pos0 + l32;
  RelFill<float, false, 256> fill;
  fill.request(p, st, h);
  rel_fill_starts(p.bk, st, starts, 256);
  const bool qok = qi < p.Nq;
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int lim = p.causal ? min(keys, pos + 1) : keys, lim_all = p.causal ? min(keys, pos0 + 1) : keys;
  const int lim_any = p.causal ? min(keys, p.query0 + min(p.Nq, qtile * 32 + 32)) : keys, tiles = lim_any > 0 ? (lim_any + 31) / 32 : 0;
  const int first = (int)((long)tiles * share / p.ksplits) + wave, nkt = (int)((long)tiles * (share + 1) / p.ksplits);
  const float* kb = (const float*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh;
  const float* vb = (const float*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh;
  const int qrow = min(qi, p.Nq - 1);
  RelRows<KC> q, dout, k;
  q.load((const float*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh, qrow, p.ldq, p.dh, g);
  dout.load((const float*)p.dout + (size_t)b * p.Nq * p.lddo + h * p.dh, qrow, p.lddo, p.dh, g);
  k.load((const float*)p.o + (size_t)b * p.Nq * p.ldo + h * p.dh, qrow, p.ldo, p.dh, g);
  const size_t sidx = ((size_t)b * p.H + h) * p.Nq + qrow;
  const float l = p.lse[sidx], lse2 = qok && l != -INFINITY ? l * LOG2E : INFINITY;      // (of no query, and of one that sees no key: its probabilities are zero)
  float dlt = 0.f;
#pragma unroll
  for (int c = 0; c < KC; ++c)
#pragma unroll
    for (int u = 0; u < 4; ++u) dlt = fmaf(k.v[c][u], dout.v[c][u], dlt);
  dlt = reduce_halves(dlt, AddOp());
  if (qok && tid < 32 && share == 0) p.delta[sidx] = dlt;
  fill.store(p, st, h, rel_lds, p.inv_scale);
  float* sums = rel_lds + rel_table_floats(p.bk);
  const int sum_stride = rel_sum_stride(p.bk);
  for (int e = tid; e < 8 * sum_stride; e += 256) sums[e] = 0.f;
  const int tab = 4 * g - pos - (bk_lo - REL_MARGIN);      // entry of this lane's first key
  float* const mine = sums + (2 * wave + g) * sum_stride;
  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = rel_all16(0.f);
  float far_sum_lo = 0.f, far_sum_hi = 0.f;
  __syncthreads();
  const float far_lo = rel_uniform(rel_lds[0]), far_hi = rel_uniform(rel_lds[entries - 1]);
  constexpr bool AHEAD = DT < 3;      // the rows of the next tile requested behind this one's products (wide heads have no registers for them)
  RelRows<KC> v;
  if (AHEAD && first < nkt) {
    k.load(kb, min(32 * first + l32, keys - 1), p.ldk, p.dh, g);
    v.load(vb, min(32 * first + l32, keys - 1), p.ldv, p.dh, g);
  }
  for (int kt = first; kt < nkt; kt += 4) {
    const int k0 = 32 * kt, row = min(k0 + l32, keys - 1);
    RelColumns<DT> kc;
    if (!AHEAD) {
      k.load(kb, row, p.ldk, p.dh, g);
      v.load(vb, row, p.ldv, p.dh, g);
    }
    kc.load(kb, k0, keys - 1, p.ldk, p.dh, g, l32);
    const bool below = k0 + 31 - pos0 <= bk_lo, above = k0 - pos0 - 31 >= bk_hi;
    f32x16 s = below ? rel_all16(far_lo) : (above ? rel_all16(far_hi) : rel_bias16(rel_lds, tab + k0));
    s = rel_rows_product(k, q, s);
    const f32x16 dp = rel_rows_product(v, dout, rel_all16(-dlt));
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -lse2)) * dp[r];
    if (AHEAD && kt + 4 < nkt) {
      const int next = min(k0 + 128 + l32, keys - 1);
      k.load(kb, next, p.ldk, p.dh, g);
      v.load(vb, next, p.ldv, p.dh, g);
    }
    if (k0 + 32 > lim_all) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = k0 + acc_row(r, g) < lim ? s[r] : 0.f;
    }
    if (below || above) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += s[r];
      if (below) far_sum_lo += sum;
      else far_sum_hi += sum;
    } else {
      // this wave's blocks lie 128 keys apart: every distance of this half of the wave is written once
      const RelDiagonals d = rel_diagonals<false>(s, lane);
      mine[tab + k0] = d.near;
      mine[tab + k0 + 32] = d.next;
    }
    rel_columns_product(kc, s, acc);
  }
  rel_leave(meet, acc, wave, g, l32);
  __syncthreads();
  for (int at = tid; at < 32 * 8 * DT; at += 256) {
    const int row = at / (8 * DT), col = at % (8 * DT) * 4, i = qtile * 32 + row;
    if (i >= p.Nq || col >= p.dh) continue;
    const float each[4] = {p.scale, p.scale, p.scale, p.scale};
    float* out = p.ksplits > 1 ? p.dq_partial + (((size_t)share * p.B + b) * p.Nq + i) * ((size_t)p.H * p.dh) : (float*)p.dq + ((size_t)b * p.Nq + i) * p.lddq;
    *reinterpret_cast<f32x4*>(out + h * p.dh + col) = rel_meet<DT>(meet, row, col, each);
  }
  if (p.dtable_partial) rel_bucket_sums<4, false>(p, starts, sums, sum_stride, far_sums, far_sum_lo, far_sum_hi, p.dtable_partial + ((((size_t)h * p.B + b) * p.ksplits + share) * qtiles + qtile) * p.bk.n_buckets);
}

// OWN: delta = rowsum(dO O) formed here, not read (deltas: 32 floats a wave).
template <int DT, int KC, bool OWN>
__device__ __forceinline__ void rel_dkv_f32(const RelAttnK& p, const RelStarts& st, int id, float* meet, float (*deltas)[32], float* rel_lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, l32 = lane & 31;
  const int ktiles = (p.Nk + 31) / 32;
  const int bk_lo = p.bk.lo, bk_hi = p.bk.hi;
  const int all = ktiles * p.B * p.H, share = p.qsplits > 1 ? id / all : 0;
  int ktile, bh;
  rel_block_map(p, id - share * all, ktiles, false, ktile, bh);
  const int b = bh / p.H, h = bh % p.H, k0 = ktile * 32, ki = k0 + l32;
  RelFill<float, true, 256> fill;
  fill.request(p, st, h);
  const int keys = __builtin_amdgcn_readfirstlane(rel_keys(p, b));
  const int seen = p.causal ? max(0, k0 - p.query0) / 32 : 0, tiles = k0 < keys ? max(0, (p.Nq + 31) / 32 - seen) : 0;
  const int first = seen + (int)((long)tiles * share / p.qsplits), nqt = seen + (int)((long)tiles * (share + 1) / p.qsplits);
  const float* qb = (const float*)p.q + (size_t)b * p.Nq * p.ldq + h * p.dh;
  const float* dob = (const float*)p.dout + (size_t)b * p.Nq * p.lddo + h * p.dh;
  const float* lse_b = p.lse + ((size_t)b * p.H + h) * p.Nq;
  const float* dlt_b = p.delta + ((size_t)b * p.H + h) * p.Nq;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) dkacc[i] = dvacc[i] = rel_all16(0.f);
  constexpr bool AHEAD = DT < 3;
  RelRows<KC> k, v, q, dout;      // (a lane whose key is past the sample's length computes what is not stored)
  if (first + wave < nqt) {
    k.load((const float*)p.k + (size_t)b * p.Nk * p.ldk + h * p.dh, min(ki, keys - 1), p.ldk, p.dh, g);
    v.load((const float*)p.v + (size_t)b * p.Nk * p.ldv + h * p.dh, min(ki, keys - 1), p.ldv, p.dh, g);
    if (AHEAD) {
      q.load(qb, min(32 * (first + wave) + l32, p.Nq - 1), p.ldq, p.dh, g);
      dout.load(dob, min(32 * (first + wave) + l32, p.Nq - 1), p.lddo, p.dh, g);
    }
  }
  fill.store(p, st, h, rel_lds, p.inv_scale);
  const int tab = 4 * g + p.query0 - ki + bk_hi + REL_MARGIN;      // entry of this lane's first query
  __syncthreads();
  const float far_hi = rel_uniform(rel_lds[0]), far_lo = rel_uniform(rel_lds[rel_entries(p.bk) - 1]);
  for (int qt = first + wave; qt < nqt; qt += 4) {
    const int q0 = 32 * qt, row = min(q0 + l32, p.Nq - 1), pos0 = p.query0 + q0;
    RelColumns<DT> qc, dc;
    if (!AHEAD) {
      q.load(qb, row, p.ldq, p.dh, g);
      dout.load(dob, row, p.lddo, p.dh, g);
    }
    qc.load(qb, q0, p.Nq - 1, p.ldq, p.dh, g, l32);
    dc.load(dob, q0, p.Nq - 1, p.lddo, p.dh, g, l32);
    float lse2[16];
    f32x16 dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i = q0 + acc_row(r, g), at = min(i, p.Nq - 1);
      const float l = lse_b[at];
      lse2[r] = i < p.Nq && l != -INFINITY ? l * LOG2E : INFINITY;
      if (!OWN) dp[r] = -dlt_b[at];
    }
    if (OWN) {
      RelRows<KC> o;
      o.load((const float*)p.o + (size_t)b * p.Nq * p.ldo + h * p.dh, row, p.ldo, p.dh, g);
      float d = 0.f;
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) d = fmaf(o.v[c][u], dout.v[c][u], d);
      d = reduce_halves(d, AddOp());
      if (g == 0) deltas[wave][l32] = -d;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(&deltas[wave][8 * r4 + 4 * g]);
#pragma unroll
        for (int u = 0; u < 4; ++u) dp[4 * r4 + u] = v[u];
      }
    }
    const bool below = k0 + 31 - pos0 <= bk_lo, above = k0 - pos0 - 31 >= bk_hi;
    f32x16 s = below ? rel_all16(far_lo) : (above ? rel_all16(far_hi) : rel_bias16(rel_lds, tab + q0));
    s = rel_rows_product(q, k, s);
    dp = rel_rows_product(dout, v, dp);
    if (AHEAD && qt + 4 < nqt) {
      const int next = min(q0 + 128 + l32, p.Nq - 1);
      q.load(qb, next, p.ldq, p.dh, g);
      dout.load(dob, next, p.lddo, p.dh, g);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -lse2[r]));
      dp[r] *= s[r];
    }
    if (p.causal && k0 + 31 > pos0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool seen = ki <= pos0 + acc_row(r, g);
        s[r] = seen ? s[r] : 0.f;
        dp[r] = seen ? dp[r] : 0.f;
      }
    }
    rel_columns_product(dc, s, dvacc);
    rel_columns_product(qc, dp, dkacc);
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float f = which ? 1.0f : p.scale, each[4] = {f, f, f, f};
    const size_t hd = (size_t)p.H * p.dh;
    float* out = p.qsplits > 1 ? p.dkv_partial + (which * p.qsplits + share) * ((size_t)p.B * p.Nk * hd) : which ? (float*)p.dv : (float*)p.dk;
    const size_t ld = p.qsplits > 1 ? hd : which ? p.lddv : p.lddk;
    if (which) __syncthreads();
    rel_leave(meet, which ? dvacc : dkacc, wave, g, l32);
    __syncthreads();
    for (int at = tid; at < 32 * 8 * DT; at += 256) {
      const int row = at / (8 * DT), col = at % (8 * DT) * 4, j = k0 + row;
      if (j >= p.Nk || col >= p.dh) continue;
      f32x4 o = rel_meet<DT>(meet, row, col, each);
      if (j >= keys) o = f32x4{0.f, 0.f, 0.f, 0.f};
      *reinterpret_cast<f32x4*>(out + ((size_t)b * p.Nk + j) * ld + h * p.dh + col) = o;
    }
  }
}

template <int DT, int KC>
__global__ void __launch_bounds__(256) rel_bwd_dq_f32_kernel(const RelAttnK p, const RelStarts st) {
  __shared__ __attribute__((aligned(16))) float meet[REL_F32_MEET<DT>];
  __shared__ float far_sums[2][4];
  __shared__ uint16_t starts[REL_STARTS];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  rel_dq_f32<DT, KC>(p, st, (int)blockIdx.x, meet, far_sums, starts, rel_lds);
}
template <int DT, int KC>
__global__ void __launch_bounds__(256) rel_bwd_dkv_f32_kernel(const RelAttnK p, const RelStarts st) {
  __shared__ __attribute__((aligned(16))) float meet[REL_F32_MEET<DT>];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  const int id = (int)blockIdx.x - p.table_items;
  if (id < 0) return rel_table_sums(p, (int)blockIdx.x, meet);
  rel_dkv_f32<DT, KC, false>(p, st, id, meet, nullptr, rel_lds);
}
// Both at once, of so few workgroups that they all find a CU: first those for dQ.
template <int DT, int KC>
__global__ void __launch_bounds__(256) rel_bwd_both_f32_kernel(const RelAttnK p, const RelStarts st, int dq_workgroups) {
  __shared__ __attribute__((aligned(16))) float meet[REL_F32_MEET<DT>];
  __shared__ __attribute__((aligned(16))) float deltas[4][32];
  __shared__ float far_sums[2][4];
  __shared__ uint16_t starts[REL_STARTS];
  extern __shared__ __attribute__((aligned(16))) float rel_lds[];
  if ((int)blockIdx.x < dq_workgroups) rel_dq_f32<DT, KC>(p, st, (int)blockIdx.x, meet, far_sums, starts, rel_lds);
  else rel_dkv_f32<DT, KC, true>(p, st, (int)blockIdx.x - dq_workgroups, meet, deltas, rel_lds);
}

// ------------------------------------------------------------------ host side
// base^e other^f in words of 32 bits, the least first: at most 1024^255 256^256, 4598 bits.  (No allocation: nothing may be thrown here.)
struct RelPower { int n; uint32_t w[160]; };
static RelPower rel_power(uint32_t base, int e, uint32_t other, int f) {
  RelPower p;
  p.n = 1;
  p.w[0] = 1;
  for (int i = 0; i < e + f; ++i) {
    uint64_t carry = 0;
    for (int j = 0; j < p.n; ++j) {
      carry += (uint64_t)p.w[j] * (i < e ? base : other);
      p.w[j] = (uint32_t)carry;
      carry >>= 32;
    }
    if (carry) p.w[p.n++] = (uint32_t)carry;
  }
  return p;
}
static bool rel_less(const RelPower& a, const RelPower& b) {
  if (a.n != b.n) return a.n < b.n;
  return std::lexicographical_compare(std::reverse_iterator<const uint32_t*>(a.w + a.n), std::reverse_iterator<const uint32_t*>(a.w),
                                      std::reverse_iterator<const uint32_t*>(b.w + b.n), std::reverse_iterator<const uint32_t*>(b.w));
}

// Bucket half + k begins with the least whole n for which n >= half (far / half)^(k / rest).  Where that border is a whole number or next to one, as it is for
// the usual powers of two, n^rest half^k and far^k half^rest are compared as whole numbers.
static int rel_buckets(const char* who, int n_buckets, int max_distance, int bidirectional, RelBucketsK& r, RelStarts& st) {
  if (n_buckets < 2 || max_distance < 1) return set_errorf(DP_EINVAL, "%s: bad number of buckets or distance", who);
  if (n_buckets > REL_MAX_BUCKETS || max_distance > REL_MAX_DISTANCE)
    return set_errorf(DP_EUNSUPPORTED, "%s: at most %d buckets and a distance of %d", who, REL_MAX_BUCKETS, REL_MAX_DISTANCE);
  if (bidirectional && n_buckets % 2) return set_errorf(DP_EINVAL, "%s: buckets of two directions must be even in number", who);
  r.n_buckets = n_buckets;
  r.bidirectional = bidirectional != 0;
  r.per_side = bidirectional ? n_buckets / 2 : n_buckets;
  r.half = r.per_side / 2;
  if (r.per_side < 2) return set_errorf(DP_EINVAL, "%s: a direction needs two buckets", who);
  if (max_distance <= r.half) return set_errorf(DP_EINVAL, "%s: the largest distance must exceed %d, the buckets of one distance each", who, r.half);
  const int rest = r.per_side - r.half;
  memset(&st, 0xFF, sizeof(st));
  int last = r.half;
  for (int k = 0; k < rest; ++k) {
    const double border = r.half * pow((double)max_distance / r.half, (double)k / rest), near = nearbyint(border);
    int n = (int)ceil(border);
    if (fabs(border - near) < 1e-6) {
      n = (int)near;
      if (rel_less(rel_power((uint32_t)n, rest, (uint32_t)r.half, k), rel_power((uint32_t)max_distance, k, (uint32_t)r.half, rest))) ++n;
    }
    ((uint16_t*)st.of)[k] = (uint16_t)n;
    last = n;
  }
  r.lo = -last;
  r.hi = bidirectional ? last : 0;
  return DP_OK;
}

static size_t rel_align(size_t n) { return align_up(n, 256); }
// Shares of the queries where a workgroup has all keys of a head: as many as run beside each other (per_cu of them a CU: two of up to 128 keys and width 64 beside a small table, else one),
// of two tiles at least.  us a pass with as many as 512 workgroups, rounded up, / with what runs at once: 8 x 30 heads of 1024 x 77 63 / 46, 8 x 10 of 4096 x 77, width 40, 71 / 54, 4 x 20
// of 2048 x 77 48 / 38, width 96, 109 / 89, 8 x 20 of 1024 x 256 88 / 65, 4 x 20 of 1024 x 250, width 72, 68 / 54.
constexpr long REL_QUERY_SHARES = 16, REL_QUERY_BLOCKS = 512;
static int rel_query_shares(int B, int H, int Nq, int per_cu) {
  const long blocks = (long)B * H, tiles = (Nq + 63) / 64;
  if (blocks >= 256) return 1;
  const long shares = std::max<long>(1, std::min(std::min(REL_QUERY_SHARES, tiles / 2), std::min(REL_QUERY_BLOCKS, 256l * per_cu) / blocks)), each = (tiles + shares - 1) / shares;
  return (int)((tiles + each - 1) / each);
}
// Shares of the keys (dQ), or of the queries (dK / dV), where workgroups of 128 of the others are too few for the CUs: four tiles at least, two workgroups a CU at most,
// and one only where half of the CUs would have none or the way is long, as the shares' fp32 sums pass through memory.  dQ and dK / dV, us a pass with 1 / 2 / 3 / 4 / 8
// shares: width 96, 16 heads of 1024 67 / 58 / 64 / 62 / 92; 4 of 4096 175 / 105 / 99 / 90 / 107; 8 of 4096 176 / 146 / 166 / 164 / 191; but 32 of 1024 56 / 63, 48 of 512 37 / 47.
constexpr long REL_GRAD_SHARES = 8, REL_GRAD_BLOCKS = 512;
static long rel_grad_shares_most(int along) { return std::min(REL_GRAD_SHARES, (long)((along + 63) / 64) / 4); }
static int rel_grad_shares(int B, int H, int N, int along) {
  const long blocks = (long)B * H * ((N + 127) / 128);
  if (blocks > (along >= 2048 ? 256 : 128)) return 1;
  return (int)std::max<long>(1, std::min(rel_grad_shares_most(along), REL_GRAD_BLOCKS / blocks));
}
// Shares in fp32, where a workgroup has 32 of one side, its four waves every fourth tile of 32 of the other, and mostly a CU to itself: until each CU has one, or
// each wave one tile; the forward, which has less to do for a tile, where waves would have three.  Forward and backward, us a pass with 1 / 2 / 4 / 16 shares at most:
// 2 x 4 heads of 257, width 40, 12 + 38 / 14 + 33 / 11 + 26 / 11 + 26; 4 of 1024 causal 28 + 95 / 21 + 63 / 21 + 62 / 21 + 62; 16 of 256 11 + 38 / 13 + 33 (forward left whole); 12 of
// one query and 4000 keys, forward 88 / 50 / 29 / 15; 8 of 100 x 1000, width 96, 39 + 86 / 27 + 60 / 19 + 46 / 16 + 40.
static long rel_shares_most_f32(int along) { return std::min(16l, ((along + 31) / 32 + 3l) / 4); }
static int rel_shares_f32(int B, int H, int N, int along, bool backward) {
  const long blocks = (long)B * H * ((N + 31) / 32);
  return backward || along > 256 ? (int)std::max<long>(1, std::min(rel_shares_most_f32(along), 256 / blocks)) : 1;
}
// Whether the backward takes workgroups of 32 queries (keys) whose waves share the other side out: where those of 128 leave CUs without one, and these all run at once
// (per_cu of them a CU: two, wide heads and large tables one), or, where the causal mask leaves half of the tiles, in two rounds of a long way.  Both kernels, us a pass by 128 (shares where rel_grad_shares
// gives some) and by 32: 8 heads of 300 27 / 19, 8 of 512 30 / 20, 50 of 300 28 / 25, 8 of 1024 40 / 27, 16 of 1024 50 / 38 and causal 48 / 30, 8 of 2048 64 / 57, width 80, 16
// of 512 39 / 27, width 96, 8 of 1024 47 / 39; causal 24 of 1024 55 / 47, 32 56 / 52, 16 of 2048 83 / 71; but 48 of 512 37 / 42 and causal 36 / 40, 32 of 1024 56 / 68, width 96, 12 of 1024 57 / 63;
// 4 of 4096 89 / 97: each K and V read four times as often.  With 64 buckets to 256, by two a CU, of which the second had no LDS, / by the one that has: 50 of 300 35 / 26, 16 of 1024 49 / 45, 12 of
// 1024 49 / 42, 32 of 512 37 / 33, 8 of 2048 72 / 59, causal 24 of 1024 56 / 48, 32 of 1024 70 / 50, 16 of 2048 94 / 73, but 64 of 250 27.9 / 29.0.
static bool rel_few_grads(int B, int H, int N, int along, int d_head, bool causal, int per_cu) {
  return (long)B * H * ((N + 31) / 32) <= 256 * per_cu * (d_head <= 64 && causal && along >= 1024 ? 2 : 1);
}
// Their shares, until each CU has one, of eight tiles at least: 16 heads of 128 x 2048 in 1 / 2 / 4 shares (of dQ) 30 / 28 / 25, but 8 of 512 in 1 / 2 20 / 23.
static int rel_few_grad_shares(int B, int H, int N, int along) {
  return (int)std::max<long>(1, std::min(REL_GRAD_SHARES, std::min<long>((along + 63) / 64 / 8, 256 / ((long)B * H * ((N + 31) / 32)))));
}
// Shares of the keys and of the queries for q and k workgroups a head, each up to its most, as long as each CU has one workgroup at most: the longer of the two chains first.
static void rel_share_out(long heads, long q, long k, long k_most, long q_most, int& ksplits, int& qsplits) {
  for (;;) {
    const bool keys = ksplits < k_most && (qsplits >= q_most || k * qsplits >= q * ksplits);
    if ((!keys && qsplits >= q_most) || heads * (q * (ksplits + keys) + k * (qsplits + !keys)) > 256) return;
    (keys ? ksplits : qsplits)++;
  }
}
// Whether one launch takes the workgroups for dQ and those for dK / dV (which then form delta themselves), and the shares of the keys and of the queries: where all find a
// CU, the longer of the two chains shared out first; under the causal mask, where half of them end early, also in two rounds, unless there are shares to be had one after the
// other.  us a pass in two launches / in one: 4 heads of 128 27 / 17, 2 of 41, width 40, 19 / 12, 75 of 22, width 16, 15 / 11, 8 of 257, width 40, 25.5 / 24.2, 2 of 500 32 / 20, 4 of 512
// causal 32 / 25, 16 of 256 33 / 24, 24 of 206 causal 37 / 28, 6 of 790, width 40, causal 66 / 51, 16 of 512 causal 57 / 47; but 16 of 512 59 / 61, 60 of 128 28 / 31.
static bool rel_both_f32(int B, int H, int Nq, int Nk, int d_head, bool causal, int& ksplits, int& qsplits) {
  const long heads = (long)B * H, q = (Nq + 31) / 32, k = (Nk + 31) / 32, blocks = heads * (q + k);
  ksplits = qsplits = 1;
  if (d_head > 64 || blocks > (causal && heads * std::min(q, k) > 128 ? 512 : 256)) return false;
  rel_share_out(heads, q, k, rel_shares_most_f32(Nk), rel_shares_most_f32(Nq), ksplits, qsplits);
  return true;
}
// Whether the few heads' workgroups for dQ and those for dK / dV go in one launch (as in fp32, see there): where all run beside each other.  us a pass in two launches / in
// one: 8 heads of 300 18.6 / 14.2, 8 of 512 19.9 / 14.8, 8 of 1024 27.3 / 24.4, 16 of 512 causal 20.0 / 17.9, width 80, 8 of 512 25.8 / 17.7; but 16 of 1024 37.5 / 41, width 80, 16 of 512 27 / 31.
// One workgroup a CU (64 buckets to 256) where 512 were launched / are not: 16 of 512 26.3 / 22.5, causal 22.8 / 20.9, 8 of 1024 35 / 29, 20 of 300 x 250 23.4 / 20.0.
static bool rel_few_both(int B, int H, int Nq, int Nk, int per_cu, int& ksplits, int& qsplits) {
  const long heads = (long)B * H, q = (Nq + 31) / 32, k = (Nk + 31) / 32;
  ksplits = qsplits = 1;
  if (heads * (q + k) > 256 * per_cu) return false;
  if (heads * (q + k) > 256 && (rel_few_grad_shares(B, H, Nq, Nk) > 1 || rel_few_grad_shares(B, H, Nk, Nq) > 1)) return false;      // (no room for shares that the way calls for)
  rel_share_out(heads, q, k, std::min<long>(REL_GRAD_SHARES, (Nk + 63) / 64 / 8), std::min<long>(REL_GRAD_SHARES, (Nq + 63) / 64 / 8), ksplits, qsplits);
  return true;
}
// The backward's: the same for both types and any bias.  Fewer samples may have more shares, but never more workgroups than REL_*_BLOCKS where there are
// shares at all: what these leave is the bound, so that no size needs more than a greater one.
struct RelWorkspace { size_t delta, partial, dq, dkv, bytes; };
static RelWorkspace rel_workspace(int B, int H, int Nq, int Nk, int d_head, int n_buckets) {
  RelWorkspace w;
  const size_t heads = (size_t)B * H, row = d_head * sizeof(float);
  const size_t few_keys = REL_QUERY_BLOCKS, parts = std::max(heads * ((Nq + 31) / 32), std::min(heads * ((Nq + 31) / 32) * REL_QUERY_SHARES, few_keys));
  auto left = [&](int N, int along) {
    const long most = rel_shares_most_f32(along);      // (no less than the other type's)
    return most > 1 ? std::min(most * heads * N, (size_t)REL_GRAD_BLOCKS * 128) : 0;
  };
  w.delta = 0;
  w.partial = rel_align(heads * Nq * sizeof(float));
  w.dq = w.partial + rel_align(parts * n_buckets * sizeof(float));
  w.dkv = w.dq + rel_align(left(Nq, Nk) * row);
  const size_t short_keys = Nq > 192 ? std::min(heads * REL_QUERY_SHARES, few_keys) * std::min(Nk, 256) : 0;
  w.bytes = w.dkv + rel_align(2 * std::max(left(Nk, Nq), short_keys) * row);
  return w;
}

// Workgroups that a CU holds beside each other: as many as its registers allow (most), and as its LDS does, which is handed out in steps of 1280 bytes.  The bias takes its part of
// that: with 64 buckets to 256 distances the few heads' kernels for dQ take 90 KB each instead of 81 (32 to 128).
static int rel_per_cu(int lds, int most) { return std::max(1, std::min(most, 160 * 1024 / (int)align_up(lds, 1280))); }
constexpr int rel_few_lds(int dhp) { return 1024 * dhp + 4 * 64 * 4 + 2 * 4 * 4 + REL_STARTS * 2; }      // of the few heads' kernels, without the bias: tiles, statistics, far sums, bucket starts

// LDS beyond 64 KB in all has to be allowed, once per kernel and device (allowing it twice is harmless; the bits only save the call).
constexpr int REL_LDS_REST = 4096;
template <auto KERNEL> static int rel_allow_lds(int own, int dynamic) {
  static std::atomic<uint64_t> devices{0};
  if (own + REL_LDS_REST + dynamic <= 64 * 1024) return DP_OK;      // (own: of the tiles; a few rows of statistics come on top)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return set_error(DP_EHIP, "attention with a relative position bias: hipGetDevice failed");
  const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (bit && (devices.load(std::memory_order_acquire) & bit)) return DP_OK;
  if (hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - own - (own ? REL_LDS_REST : 0)) != hipSuccess)
    return set_error(DP_EHIP, "attention with a relative position bias: hipFuncSetAttribute failed");
  devices.fetch_or(bit, std::memory_order_release);
  return DP_OK;
}
// Width of the tiles and steps of 16 over the head.  us with the steps of the next line instead: width 40, 8 x 5 heads of 4096 forward 170 / 181, 8 x 10 of 1024 forward and backward 28.9 + 86.9 / 30.0 + 92.6; width 72
// and 80, 8 x 10 of 1024 39.3 + 148 / 40.4 + 154, 32 x 16 of 256 backward 76 / 85.
template <class F> static int rel_dispatch(int d_head, F f) {
  using std::integral_constant;
  if (d_head <= 48) return f(integral_constant<int, 64>(), integral_constant<int, 3>());
  if (d_head <= 64) return f(integral_constant<int, 64>(), integral_constant<int, 4>());
  if (d_head <= 80) return f(integral_constant<int, 96>(), integral_constant<int, 5>());
  return f(integral_constant<int, 96>(), integral_constant<int, 6>());
}
// Blocks of 32 columns and steps of 8 over the head.  us with the line behind instead: width 16, 8 x 16 heads of 1000 forward 153 / 185, backward 546 / 668, 4 x 8 of 300 11.5 / 12.9 and 37 / 42; width 40, 8 x 8 of 1000
// 161 / 184 and 598 / 699.
template <class F> static int rel_dispatch_f32(int d_head, F f) {
  using std::integral_constant;
  if (d_head <= 16) return f(integral_constant<int, 1>(), integral_constant<int, 2>());
  if (d_head <= 32) return f(integral_constant<int, 1>(), integral_constant<int, 4>());
  if (d_head <= 40) return f(integral_constant<int, 2>(), integral_constant<int, 5>());
  if (d_head <= 64) return f(integral_constant<int, 2>(), integral_constant<int, 8>());
  return f(integral_constant<int, 3>(), integral_constant<int, 12>());
}
template <class F> static int rel_short_dispatch(int d_head, int Nk, F f) {      // and waves: 32 keys each
  using std::integral_constant;
  return rel_dispatch(d_head, [&](auto dhp, auto kc) { return Nk <= 128 ? f(dhp, kc, integral_constant<int, 4>()) : f(dhp, kc, integral_constant<int, 8>()); });
}
// (take_turns keeps workgroups of equal length together; under the causal mask the long ones, which come first, had better stay ahead: dQ of 8 x 10 heads of 1024 39 -> 36 us,
// of 4 x 12 of 2048 65 -> 60)
static int rel_takes_turns(long blocks, int per_cu, bool causal) { return !causal && blocks > 256 && blocks <= 256L * per_cu; }
static int rel_launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DP_OK : set_errorf(DP_EHIP, "attention with a relative position bias: launch failed (%s)", hipGetErrorString(e));
}

// Shares of the keys for workgroups of 32 queries, none with less than two tiles for each of its waves.  Where a head is read for its few queries alone, and two
// workgroups fit a CU, until three a CU are there: 16 x 12 heads, one query, 4000 keys: 1 / 2 / 3 / 4 / 5 / 8 shares 44 / 40 / 41 / 36 / 37 / 38 us, keys of different lengths
// 37 / 33 / 30 / 26 / 27 / 28; 12 heads 31 / 19 / 15 / 12 / 11 / 9.  Else until each CU has one: 4 heads of 2000 in 1 / 2 / 4 shares 15 / 18 / 23, 8 of 1024 12 / 16, 8 of 256 x 4096
// 29 / 22 / 16 (8: 16), width 72, 16 of 300 x 1000 16 / 24, width 96, 192 and 64 of one query and 4000 keys 75 / 87 / 77 and 52 / 36 / 29 (8: 31).
constexpr long REL_SHARE_BLOCKS = 768;
static long rel_shares_most(int Nk) { return ((Nk + 63) / 64 + 7) / 8; }
static int rel_shares(int B, int H, int Nq, int Nk, int d_head) {
  const long blocks = (long)B * H * ((Nq + 31) / 32);
  return (int)std::max<long>(1, std::min(rel_shares_most(Nk), Nq <= 32 && d_head <= 64 ? (REL_SHARE_BLOCKS + blocks - 1) / blocks : 256 / blocks));
}
// Whether the forward takes 32 queries a workgroup and shares the keys out, instead of 128 queries that read each key once: where those are too few for
// the CUs and these all run at once.  Heads, queries x keys, width, us by 32 (with what joins the shares) and by 128: 8, 256 x 4096, 64 16 / 54 (one share); 8, 1024 x 1024, 64 12 / 17; 16
// 16 / 17; 8, 2048 x 2048, 64 27 / 30; 4, 2000 x 2000, 40 15 / 27; 32, 512 x 512, 64 11.0 / 11.2; 64, 128 x 256, 64 6.8 / 8.0; 24, 300 x 1000, 72 16 / 19; 12, 512 x 512, 96 11 / 13;
// but 64, 256 x 256, 64 8.9 / 8.2; 32, 300 x 1000, 72 29 / 20; beyond 2048 keys see rel_shares_128; 24, 512 x 512, 96 21 / 14; 144, 77 x 77, 64 7.3 / 6.4.
// Up to 32 queries either has a workgroup a head, this one more of them in flight (for shares) and that one four a CU: 512 heads of one query, width 64, 256 keys 7.7 / 9.2, 500 15.4 / 15.0, 1000 30 / 24, 320 of
// 500 13.4 / 13.6, 1000 24 / 22, 256 of 1000 18.5 / 17.3, 2000 29 / 30, 4000 51 / 56; keys of different lengths 512 of 1000 21 / 20, 384 of 4000 42 / 53, 800 of 4000 101 / 88; 600 of 32 x 32 10.9 / 6.5; width 96, 256 of
// 200 7.7 / 8.8, 1000 24 / 23, 288 of 200 13.5 / 10.8, 1000 38 / 29, 2040 of 32 x 500 119 / 85.
static bool rel_few(int B, int H, int Nq, int Nk, int d_head, bool lengths) {
  if (Nq <= 32) return (long)B * H <= (d_head <= 64 && (Nk <= 512 || lengths) ? 512 : 256);
  const long blocks = (long)B * H * ((Nq + 31) / 32);
  return blocks <= (Nk > 2048 ? 64 : d_head <= 64 && Nk > 256 ? 512 : 256);
}
// Shares of the keys for workgroups of 128 queries: where CUs would have none and the way is long, eight tiles at least, two workgroups a CU at most, and not in two.  Heads of as many
// queries as keys, us with 1 / 2 / 4 / 8 shares: 4 of 3044, width 88, causal 51 / 36 / 29 / 28; 3 of 4096, width 96, 67 / 46 / 37 / 37; 4 of 4096 54 / 38 / 32 / 32; 6 of 3000 41 / - / 31 (three); 8 of 2048, width 80, 33 / 30 / 30; but 12
// of 1024, width 96, 21.5 / 23.6, 8 of 4096 (256 workgroups) 54.6 / 55.9.  By 32 queries a workgroup instead: 4 of 4096 46, 2 of 3000 24 (21), 4 of 1024 x 8192 34 (24), but 4 of 2048 18.4 (19.4),
// 8 of 2048 causal 22 (26) and 4 of 300 x 8000 19 (22).
static int rel_shares_128(int B, int H, int Nq, int Nk) {
  const long blocks = (long)B * H * ((Nq + 127) / 128);
  return blocks > 170 || Nk < 2048 ? 1 : (int)std::max<long>(1, std::min(rel_shares_most(Nk), 512 / blocks));
}
// (no size needs more than a greater one, as in rel_workspace)
static size_t rel_share_bytes(int B, int H, int Nq, int Nk, int d_head) {
  const size_t most = std::max(rel_shares_most(Nk), rel_shares_most_f32(Nk));
  return most > 1 ? align_up(std::min(most * B * H * Nq, (size_t)512 * 128) * (d_head + 2) * sizeof(float), 256) : 0;
}

static int check_rel(const char* who, int dtype, const RelAttnK& k, const dp_relbias* bias, bool bwd) {
  if (dtype != DP_F32 && dtype != DP_BF16) return set_error(DP_EINVAL, "unknown dtype");
  if (k.B <= 0 || k.H <= 0 || k.Nq <= 0 || k.Nk <= 0 || k.dh <= 0) return set_errorf(DP_EINVAL, "%s: non-positive size", who);
  if (!(k.scale > 0.f) || !(k.scale < INFINITY)) return set_errorf(DP_EINVAL, "%s: the scale must be positive and finite", who);
  if (k.scale < 1e-6f || k.scale > 1e6f) return set_errorf(DP_EUNSUPPORTED, "%s: a scale between 1e-6 and 1e6", who);      // (the bias is held over the scale)
  if ((size_t)k.B * k.H > 65535) return set_errorf(DP_EUNSUPPORTED, "%s: batch * heads exceeds 65535", who);
  const int grid = dtype == DP_BF16 ? 8 : 4, es = dtype == DP_BF16 ? 2 : 4;
  if (k.dh % grid || k.dh > 96) return set_errorf(DP_EUNSUPPORTED, "%s: d_head must be a multiple of %d, at most 96", who, grid);
  if (k.query0 > (1 << 29) || k.query0 < -(1 << 29) || k.Nq > (1 << 29) || k.Nk > (1 << 29)) return set_errorf(DP_EUNSUPPORTED, "%s: positions beyond 2^29", who);
  const size_t rows = dtype == DP_BF16 ? 128 : 32, tiles = ((size_t)std::max(k.Nq, k.Nk) + rows - 1) / rows * k.B * k.H;
  if (tiles + (size_t)k.H * (REL_MAX_BUCKETS / 32) + 8 >= (1u << 24)) return set_errorf(DP_EUNSUPPORTED, "%s: too many tiles for one launch", who);      // (2^32 threads)
  const int span = k.H * k.dh;
  struct Op { const void* p; int ld, n; const char* name; };
  const Op ops[] = {{k.q, k.ldq, k.Nq, "q"}, {k.k, k.ldk, k.Nk, "k"}, {k.v, k.ldv, k.Nk, "v"}, {k.o, k.ldo, k.Nq, "o"},
                    {k.dout, k.lddo, k.Nq, "d_o"}, {k.dq, k.lddq, k.Nq, "dq"}, {k.dk, k.lddk, k.Nk, "dk"}, {k.dv, k.lddv, k.Nk, "dv"}};
  for (int i = 0; i < (bwd ? 8 : 4); ++i) {
    DP_TRY(check_ptr(ops[i].p, ops[i].name));
    if (ops[i].ld < span) return set_errorf(DP_EINVAL, "%s: the row stride of %s is less than heads * d_head", who, ops[i].name);
    if (ops[i].ld % grid) return set_errorf(DP_EUNSUPPORTED, "%s: the row stride of %s must be a multiple of %d", who, ops[i].name, grid);
    // (a tile's copies count up to 128 rows, whether they exist or not, by 32-bit byte offsets: beyond 2^32 those of missing rows would come round to others)
    if (dtype == DP_BF16 && ops[i].ld >= 1 << 24) return set_errorf(DP_EUNSUPPORTED, "%s: the row stride of %s must be below 2^24 elements", who, ops[i].name);
    // one (sample, head) is addressed with 32-bit byte offsets, of which bit 31 means "no data"
    if ((size_t)ops[i].n * ops[i].ld * es >= (1ull << 31)) return set_errorf(DP_EUNSUPPORTED, "%s: the rows of one sample of %s must span less than 2 GiB", who, ops[i].name);
  }
  if (!bias) return set_errorf(DP_EINVAL, "%s: bias is NULL", who);
  DP_TRY(check_ptr(bias->table, "the bias table"));
  if (k.key_len && (uintptr_t)k.key_len % 4) return set_errorf(DP_EALIGN, "%s: key_len must be 4-byte aligned", who);
  if (bwd && !k.lse) return set_errorf(DP_EINVAL, "%s: lse is NULL", who);
  if (k.lse && (uintptr_t)k.lse % 16) return set_errorf(DP_EALIGN, "%s: lse is not 16-byte aligned", who);
  return DP_OK;
}

}  // namespace dp

using namespace dp;

extern "C" {

int dp_relative_bucket(int n_buckets, int max_distance, int bidirectional, int distance) {
  RelBucketsK r;
  RelStarts st;
  DP_TRY(rel_buckets("dp_relative_bucket", n_buckets, max_distance, bidirectional, r, st));
  const int n = bidirectional ? (distance < 0 ? -(int64_t)distance > INT32_MAX ? INT32_MAX : -distance : distance) : (distance < 0 ? (distance == INT32_MIN ? INT32_MAX : -distance) : 0);
  const int side = bidirectional && distance > 0 ? r.per_side : 0;
  if (n < r.half) return side + n;
  const int k = (int)(std::upper_bound((const uint16_t*)st.of, (const uint16_t*)st.of + (r.per_side - r.half), n) - (const uint16_t*)st.of) - 1;
  return side + r.half + k;
}

size_t dp_op_attention_relbias_workspace_bytes(int B, int H, int Nq, int Nk, int d_head, int n_buckets, int backward) {
  if (B <= 0 || H <= 0 || Nq <= 0 || Nk <= 0 || d_head <= 0 || n_buckets <= 0) return 0;
  if (backward) return rel_workspace(B, H, Nq, Nk, d_head, n_buckets).bytes;
  return rel_share_bytes(B, H, Nq, Nk, d_head);
}

int dp_op_attention_relbias_fwd(int dtype, int B, int H, int Nq, int Nk, int d_head, int causal, float scale, const void* q, int ldq, const void* k,
                                int ldk, const void* v, int ldv, const dp_relbias* bias, const int32_t* key_len, void* o, int ldo, float* lse,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "dp_op_attention_relbias_fwd";
  RelAttnK a{};
  RelStarts st;
  a.B = B; a.H = H; a.Nq = Nq; a.Nk = Nk; a.dh = d_head; a.causal = causal != 0; a.query0 = bias ? bias->query0 : 0;
  a.scale = scale; a.scale_log2 = scale * LOG2E; a.inv_scale = 1.0f / scale; a.shares = 1;
  a.q = q; a.ldq = ldq; a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.table = bias ? bias->table : nullptr; a.key_len = key_len; a.o = o; a.ldo = ldo; a.lse = lse;
  DP_TRY(check_rel(who, dtype, a, bias, false));
  DP_TRY(rel_buckets(who, bias->n_buckets, bias->max_distance, bias->bidirectional, a.bk, st));
  hipStream_t s = (hipStream_t)hip_stream;
  KScope ks(dtype == DP_BF16 ? KK_ATTN_FWD : KK_ATTN_F32, 4.0 * B * H * (double)Nq * Nk * d_head, (dtype == DP_BF16 ? 2.0 : 4.0) * B * H * d_head * (2.0 * Nq + 2.0 * Nk), s, Nq, Nk, d_head);
  const size_t need = rel_share_bytes(B, H, Nq, Nk, d_head), joins = ((size_t)B * H * Nq * (d_head / 4) + 255) / 256;
  auto shares = [&](int n) -> int {      // as many, if there is a workspace for what they leave
    if (!workspace) return DP_OK;
    if ((uintptr_t)workspace % 256) return set_errorf(DP_EALIGN, "%s: workspace is not 256-byte aligned", who);
    if (workspace_bytes < need) return set_errorf(DP_EWORKSPACE, "%s: workspace too small (%zu bytes, needs %zu)", who, workspace_bytes, need);
    a.shares = n;
    a.part = (float*)workspace;
    return DP_OK;
  };
  if (dtype == DP_F32) {
    DP_TRY(shares(rel_shares_f32(B, H, Nq, Nk, false)));
    const int table = rel_table_floats(a.bk) * 4;
    DP_TRY(rel_dispatch_f32(d_head, [&](auto dt, auto kc) {
      DP_TRY((rel_allow_lds<rel_fwd_f32_kernel<dt, kc>>(REL_F32_MEET<dt> * 4, table)));
      hipLaunchKernelGGL((rel_fwd_f32_kernel<dt, kc>), dim3((unsigned)((Nq + 31) / 32 * B * H * a.shares)), dim3(256), table, s, a, st);
      return rel_launched();
    }));
    if (a.shares == 1) return DP_OK;
    hipLaunchKernelGGL((rel_join_kernel<float>), dim3((unsigned)joins), dim3(256), 0, s, a);
    return rel_launched();
  }
  const int lds = rel_table_floats(a.bk) * 4;
  if (rel_few(B, H, Nq, Nk, d_head, key_len != nullptr)) {
    DP_TRY(shares(rel_shares(B, H, Nq, Nk, d_head)));
    DP_TRY(rel_dispatch(d_head, [&](auto dhp, auto kc) {
      DP_TRY((rel_allow_lds<rel_fwd_few_bf16_kernel<dhp, kc>>(1024 * dhp, lds)));
      hipLaunchKernelGGL((rel_fwd_few_bf16_kernel<dhp, kc>), dim3((unsigned)((Nq + 31) / 32 * B * H * a.shares)), dim3(256), lds, s, a, st);
      return rel_launched();
    }));
    if (a.shares == 1) return DP_OK;
    hipLaunchKernelGGL((rel_join_kernel<bf16>), dim3((unsigned)joins), dim3(256), 0, s, a);
    return rel_launched();
  }
  DP_TRY(shares(rel_shares_128(B, H, Nq, Nk)));
  const long blocks = (long)((Nq + 127) / 128) * B * H * a.shares;
  a.even = rel_takes_turns(blocks, d_head <= 64 ? rel_per_cu(512 * 64 + lds, 4) : rel_per_cu(512 * 96 + lds, 3), causal);
  DP_TRY(rel_dispatch(d_head, [&](auto dhp, auto kc) {
    constexpr int W = dhp == 64 ? 4 : 3;
    auto run = [&](auto shares) {
      DP_TRY((rel_allow_lds<rel_fwd_bf16_kernel<dhp, kc, W, shares>>(512 * dhp, lds)));
      hipLaunchKernelGGL((rel_fwd_bf16_kernel<dhp, kc, W, shares>), dim3((unsigned)blocks), dim3(256), lds, s, a, st);
      return rel_launched();
    };
    return a.shares > 1 ? run(std::true_type()) : run(std::false_type());
  }));
  if (a.shares == 1) return DP_OK;
  hipLaunchKernelGGL((rel_join_kernel<bf16>), dim3((unsigned)joins), dim3(256), 0, s, a);
  return rel_launched();
}

int dp_op_attention_relbias_bwd(int dtype, int B, int H, int Nq, int Nk, int d_head, int causal, float scale, const void* q, int ldq, const void* k,
                                int ldk, const void* v, int ldv, const dp_relbias* bias, const int32_t* key_len, const void* o, int ldo,
                                const float* lse, const void* d_o, int lddo, void* dq, int lddq, void* dk, int lddk, void* dv, int lddv, float* dtable,
                                int accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "dp_op_attention_relbias_bwd";
  RelAttnK a{};
  RelStarts st;
  a.B = B; a.H = H; a.Nq = Nq; a.Nk = Nk; a.dh = d_head; a.causal = causal != 0; a.query0 = bias ? bias->query0 : 0;
  a.scale = scale; a.scale_log2 = scale * LOG2E; a.inv_scale = 1.0f / scale;
  a.q = q; a.ldq = ldq; a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.table = bias ? bias->table : nullptr; a.key_len = key_len;
  a.o = const_cast<void*>(o); a.ldo = ldo; a.lse = const_cast<float*>(lse); a.dout = d_o; a.lddo = lddo;
  a.dq = dq; a.lddq = lddq; a.dk = dk; a.lddk = lddk; a.dv = dv; a.lddv = lddv;
  DP_TRY(check_rel(who, dtype, a, bias, true));
  DP_TRY(rel_buckets(who, bias->n_buckets, bias->max_distance, bias->bidirectional, a.bk, st));
  if (dtable && (uintptr_t)dtable % 16) return set_errorf(DP_EALIGN, "%s: dtable is not 16-byte aligned", who);
  const RelWorkspace w = rel_workspace(B, H, Nq, Nk, d_head, bias->n_buckets);
  DP_TRY(check_ptr(workspace, "workspace", 256));
  if (workspace_bytes < w.bytes) return set_errorf(DP_EWORKSPACE, "%s: workspace too small (%zu bytes, needs %zu)", who, workspace_bytes, w.bytes);
  a.delta = (float*)((char*)workspace + w.delta);
  a.dq_partial = (float*)((char*)workspace + w.dq);
  a.dkv_partial = (float*)((char*)workspace + w.dkv);
  a.qsplits = a.ksplits = 1;
  a.dtable_partial = dtable ? (float*)((char*)workspace + w.partial) : nullptr;
  hipStream_t s = (hipStream_t)hip_stream;
  a.dtable = dtable;
  const int table = rel_table_floats(a.bk) * 4, both = rel_sum_floats(a.bk, 4) * 4;      // bytes of LDS: bias, and sums by distance with it
  const int dhp = d_head <= 64 ? 64 : 96;
  const bool few_fit = 1024 * dhp + REL_LDS_REST + both <= 160 * 1024;
  const int few_per_cu = rel_per_cu(rel_few_lds(dhp) + both, dhp == 64 ? 2 : 1), few_k_per_cu = rel_per_cu(rel_few_lds(dhp) + table, dhp == 64 ? 2 : 1);
  const bool at_once = dtype == DP_F32 ? rel_both_f32(B, H, Nq, Nk, d_head, causal, a.ksplits, a.qsplits) : few_fit && rel_few_both(B, H, Nq, Nk, few_per_cu, a.ksplits, a.qsplits);
  const bool few_q = few_fit && rel_few_grads(B, H, Nq, Nk, d_head, causal, few_per_cu), few_k = rel_few_grads(B, H, Nk, Nq, d_head, causal, few_k_per_cu);
  // One kernel whose workgroups hold all keys, where its LDS suffices for the bias; few heads go by 32 queries and keys, but up to 128 keys only in one launch: 8 heads of 200 20.6 /
  // 12.7 us, 8 of 128 15.4 / 12.1, 64 of 77 16.5 / 13.0, 20 of 300 x 250 27 / 16, 60 of 171, width 40, causal 22 / 18, 72 of 200 28 / 22; but 100 of 128 16.4 / 20.5, 144 of 41, width 40, 13 / 17.
  bool all_keys = false;
  int short_per_cu = 1;
  if (dtype == DP_BF16 && Nk <= 256 && !at_once && !(Nk > 128 && few_q && few_k))
    DP_TRY(rel_short_dispatch(d_head, Nk, [&](auto dhp, auto, auto nw) {
      const int lds = RelShort<dhp, nw>::BYTES + rel_sum_floats(a.bk, nw) * 4;
      all_keys = lds <= 160 * 1024;
      short_per_cu = rel_per_cu(lds, nw == 4 ? 2 : 1);
      return DP_OK;
    }));
  a.dtable_add = accumulate != 0;
  a.table_items = dtable ? (H * ((bias->n_buckets + 31) / 32) + 7) / 8 * 8 : 0;      // workgroups that add the parts of the table's gradient (eights: the others stay on their XCDs)
  const double fl = 4.0 * B * H * (double)Nq * Nk * d_head, by = (dtype == DP_BF16 ? 2.0 : 4.0) * B * H * d_head * (3.0 * Nq + 2.0 * Nk);
  if (dtype == DP_F32) {
    KScope ks(KK_ATTN_F32, 2 * fl, 2 * by, s, Nq, Nk, d_head);
    if (!at_once) {
      a.ksplits = rel_shares_f32(B, H, Nq, Nk, true);
      a.qsplits = rel_shares_f32(B, H, Nk, Nq, true);
    }
    const int dq = (Nq + 31) / 32 * B * H * a.ksplits, dkv = (Nk + 31) / 32 * B * H * a.qsplits;
    a.dtable_parts = B * ((Nq + 31) / 32) * a.ksplits;
    DP_TRY(rel_dispatch_f32(d_head, [&](auto dt, auto kc) {
      if constexpr (dt < 3)
        if (at_once) {
          DP_TRY((rel_allow_lds<rel_bwd_both_f32_kernel<dt, kc>>(REL_F32_MEET<dt> * 4, both)));
          hipLaunchKernelGGL((rel_bwd_both_f32_kernel<dt, kc>), dim3((unsigned)(dq + dkv)), dim3(256), both, s, a, st, dq);
          return rel_launched();
        }
      DP_TRY((rel_allow_lds<rel_bwd_dq_f32_kernel<dt, kc>>(REL_F32_MEET<dt> * 4, both)));
      hipLaunchKernelGGL((rel_bwd_dq_f32_kernel<dt, kc>), dim3((unsigned)dq), dim3(256), both, s, a, st);
      DP_TRY(rel_launched());
      DP_TRY((rel_allow_lds<rel_bwd_dkv_f32_kernel<dt, kc>>(REL_F32_MEET<dt> * 4, table)));
      hipLaunchKernelGGL((rel_bwd_dkv_f32_kernel<dt, kc>), dim3((unsigned)dkv + a.table_items), dim3(256), table, s, a, st);
      return rel_launched();
    }));
  } else if (all_keys) {
    a.qsplits = rel_query_shares(B, H, Nq, short_per_cu);
    a.dtable_parts = B * a.qsplits;
    KScope ks(KK_ATTN_BWD_DKV, 2 * fl, 2 * by, s, Nq, Nk, d_head);
    DP_TRY(rel_short_dispatch(d_head, Nk, [&](auto dhp, auto kc, auto nw) {
      const int lds = RelShort<dhp, nw>::BYTES + rel_sum_floats(a.bk, nw) * 4;
      DP_TRY((rel_allow_lds<rel_bwd_short_bf16_kernel<dhp, kc, nw>>(0, lds)));
      hipLaunchKernelGGL((rel_bwd_short_bf16_kernel<dhp, kc, nw>), dim3((unsigned)(B * H * a.qsplits)), dim3(64 * nw), lds, s, a, st);
      return rel_launched();
    }));
  } else if (at_once) {
    KScope ks(KK_ATTN_BWD_DKV, 2 * fl, 2 * by, s, Nq, Nk, d_head);
    const int dq = (Nq + 31) / 32 * B * H * a.ksplits, dkv = (Nk + 31) / 32 * B * H * a.qsplits;
    a.dtable_parts = B * ((Nq + 31) / 32) * a.ksplits;
    DP_TRY(rel_dispatch(d_head, [&](auto dhp, auto kc) {
      DP_TRY((rel_allow_lds<rel_bwd_few_both_bf16_kernel<dhp, kc>>(1024 * dhp, both)));
      hipLaunchKernelGGL((rel_bwd_few_both_bf16_kernel<dhp, kc>), dim3((unsigned)(dq + dkv)), dim3(256), both, s, a, st, dq);
      return rel_launched();
    }));
  } else {
    a.ksplits = few_q ? rel_few_grad_shares(B, H, Nq, Nk) : rel_grad_shares(B, H, Nq, Nk);
    a.qsplits = few_k ? rel_few_grad_shares(B, H, Nk, Nq) : rel_grad_shares(B, H, Nk, Nq);
    a.dtable_parts = B * ((Nq + (few_q ? 31 : 127)) / (few_q ? 32 : 128)) * a.ksplits;
    const int qrows = few_q ? 32 : 128, krows = few_k ? 32 : 128;
    const long qblocks = (long)((Nq + qrows - 1) / qrows) * B * H * a.ksplits, kblocks = (long)((Nk + krows - 1) / krows) * B * H * a.qsplits;
    {
      KScope ks(KK_ATTN_BWD_DQ, fl, by, s, Nq, Nk, d_head);
      a.even = rel_takes_turns(qblocks, rel_per_cu(512 * dhp + 2 * 4 * 4 + REL_STARTS * 2 + both, dhp == 64 ? 3 : 2), causal);
      DP_TRY(rel_dispatch(d_head, [&](auto dhp, auto kc) {
        if (few_q) {
          DP_TRY((rel_allow_lds<rel_bwd_few_dq_bf16_kernel<dhp, kc>>(1024 * dhp, both)));
          hipLaunchKernelGGL((rel_bwd_few_dq_bf16_kernel<dhp, kc>), dim3((unsigned)qblocks), dim3(256), both, s, a, st);
          return rel_launched();
        }
        auto run = [&](auto shares) {
          DP_TRY((rel_allow_lds<rel_bwd_dq_bf16_kernel<dhp, kc, shares>>(512 * dhp, both)));
          hipLaunchKernelGGL((rel_bwd_dq_bf16_kernel<dhp, kc, shares>), dim3((unsigned)qblocks), dim3(256), both, s, a, st);
          return rel_launched();
        };
        return a.ksplits > 1 ? run(std::true_type()) : run(std::false_type());
      }));
    }
    KScope ks(KK_ATTN_BWD_DKV, fl, by, s, Nq, Nk, d_head);
    // Three waves per SIMD where two would begin a second round; under the causal mask tiles end at different times anyway, and its selects have no registers
    // left (8 x 10 heads of 1024 40 and 46 us)
    const bool many = d_head <= 64 && !causal && kblocks > 2 * 256 && rel_per_cu(768 * dhp + 4 * 64 * 4 + table, 3) == 3;      // (with 512 buckets to 1024 LDS holds two: 263 -> 241 us)
    a.even = rel_takes_turns(kblocks, many ? 3 : 2, causal);
    DP_TRY(rel_dispatch(d_head, [&](auto dhp, auto kc) {
      if (few_k) {
        DP_TRY((rel_allow_lds<rel_bwd_few_dkv_bf16_kernel<dhp, kc>>(1024 * dhp, table)));
        hipLaunchKernelGGL((rel_bwd_few_dkv_bf16_kernel<dhp, kc>), dim3((unsigned)kblocks + a.table_items), dim3(256), table, s, a, st);
        return rel_launched();
      }
      auto run = [&](auto minw, auto shares) {
        DP_TRY((rel_allow_lds<rel_bwd_dkv_bf16_kernel<dhp, kc, minw, shares>>((minw == 3 ? 768 : 512) * dhp, table)));
        hipLaunchKernelGGL((rel_bwd_dkv_bf16_kernel<dhp, kc, minw, shares>), dim3((unsigned)kblocks + a.table_items), dim3(256), table, s, a, st);
        return rel_launched();
      };
      using std::integral_constant;
      if (a.qsplits > 1) return run(integral_constant<int, 2>(), std::true_type());
      return many ? run(integral_constant<int, dhp == 64 ? 3 : 2>(), std::false_type()) : run(integral_constant<int, 2>(), std::false_type());
    }));
  }
  if (!at_once && !all_keys) a.table_items = 0;      // (they were there already)
  if (a.ksplits == 1 && a.qsplits == 1 && a.table_items == 0) return DP_OK;
  const double parts = 4.0 * a.dtable_parts * H * bias->n_buckets, es = dtype == DP_BF16 ? 2.0 : 4.0, hd = (double)H * d_head;
  KScope ks(KK_REDUCE, 0.0, (a.table_items ? parts : 0.0) + (a.ksplits > 1 ? (4.0 * a.ksplits + es) * B * Nq * hd : 0.0) + (a.qsplits > 1 ? 2 * (4.0 * a.qsplits + es) * B * Nk * hd : 0.0), s,
            H * d_head, a.ksplits, a.qsplits);
  if (a.ksplits == 1 && a.qsplits == 1) {
    hipLaunchKernelGGL(rel_dtable_kernel, dim3(a.table_items), dim3(256), 0, s, a);
    return rel_launched();
  }
  const size_t dq_joins = a.ksplits > 1 ? rel_join_workgroups(B, Nq, H, d_head) : 0, dkv_joins = a.qsplits > 1 ? rel_join_workgroups(B, Nk, H, d_head) : 0;
  if (dtype == DP_F32) hipLaunchKernelGGL((rel_join_grads_kernel<float>), dim3((unsigned)(dq_joins + dkv_joins + a.table_items)), dim3(256), 0, s, a, (unsigned)dq_joins);
  else hipLaunchKernelGGL((rel_join_grads_kernel<bf16>), dim3((unsigned)(dq_joins + dkv_joins + a.table_items)), dim3(256), 0, s, a, (unsigned)dq_joins);
  return rel_launched();
}

}  // extern "C"
