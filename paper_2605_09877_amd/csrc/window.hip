// Sliding-window attention whose first tokens stay visible: the query at position t sees key j if j <= t and
// (t - j < W or j < S).
//
// Prompt: a workgroup's four waves own 32 queries each: of four heads that share a KV head where the group allows it,
// of consecutive positions otherwise.  Keys come in tiles, the sinks in front of the window first, then the window of
// the workgroup's first query up to its last query, under one online softmax (seq_tiles.h for the operands):
//   S^T[key, query] = K Q^T,  P^T = 2^(S^T scale log2 e - m),  O^T[channel, query] += V^T P^T
// Gradients, with D = dout . out and dP = dout V^T:  dS = P (dP - D),  dq = scale dS K  (one kernel, a workgroup's queries again),
// dk = scale dS^T q,  dv = P^T dout  (another, a workgroup's keys): seven products for the five there are, and no atomics.
// Single token: one pass over the rows that its sequence sees of a ring cache.
//
// What they reach (bf16, 128 channels): prompt, 2 sequences of 16k tokens, 32 heads on 8, window 2048: 1070 us, 0.97 PFLOP/s, where a
// large matrix product of a library takes 1.24.  Matrix instructions are 46 % of the cycles; the vector instructions of a tile (a
// quarter-rate exponential for every pair) take about as many cycles again, LDS reads and the tiles' direct loads the rest (without
// either, in a copy made to measure: -10 and -14 %).  Two sequences of 8k tokens, window 1024, of both passes: 402 us forward, 549 dq,
// 770 dk and dv: 1.16 TFLOP done in 1.5 ms.  Single token, 64 sequences, 8 KV heads, 4100 rows: 178 us, 5.7 TB/s, the card's read rate.
#include <math.h>

#include <type_traits>

#include "../../include/kvm.h"
#include "kvm_internal.h"
#include "seq_tiles.h"

namespace kvm {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kXcds = 8;
constexpr int kWaves = 4;
constexpr int kMaxSink = 128;

struct WinArgs {
  const char *q, *k, *v;
  char *out, *rest;   // rest (nullable): what rounding out left, for the backward pass; strides of out
  float *lse;         // nullable
  int64_t q_b, q_t, q_h, k_b, k_t, k_h, v_b, v_t, v_h, o_b, o_t, o_h;   // bytes
  int64_t l_b, l_t, l_h;                                                // elements
  const int32_t *lens;   // nullable
  float scale;
  int32_t B, Hq, Hkv, Tq, Tk, W, S;
  int32_t by_head, span, tiles, per_block, blocks;   // position tiles, of which per_block make a block; blocks of a unit
  // backward
  const char *dout;
  char *dq, *dk, *dv;
  float *delta;    // [B, Hq, Tq]
  float *part;     // [units, parts, 2, sink_rows, D]: shares of the sinks' dk and dv, the last from the queries of their window
  int32_t n_split, split_q;   // ranges that the queries beyond a sink's window are cut into, and their length
  int32_t sink_rows, parts;   // S up to 32, 64 or 128; shares
  float *sums;     // n_part > 1: [units, n_part, 2, Tk, D]: dk and dv of every part of a key tile's queries
  int32_t n_part;
  int32_t key_tiles, far_wgs;   // tiles of 128 keys; workgroups that have sinks' far queries
};

// Keys of a tile.  With 32 the prompt kernel has registers for three workgroups to a compute unit, in whose turns the exponentials of one
// run beside the products of another: 2 sequences of 16k tokens, 32 heads of 128 on 8, window 2048: 1094 us, 1147 with 64 and two
// workgroups.  Rows of 64 channels, us, 32 / 64: 4 x 4k tokens, 16 heads on 4, 70 / 77; 2k, 16 heads, 15 / 20; 8 x 1000, 8 heads, 28 /
// 26, the one kind that loses.  dq: 4 x 4k, 16 heads of 64 on 4, with dk and dv 207 / 216.
constexpr int kTileRows = 32;

__device__ __forceinline__ int tokens_of(const WinArgs &a, int b) {
  int n = a.Tk;
  if (a.lens) {
    n = a.lens[b];
    n = n < 0 ? 0 : n < a.Tk ? n : a.Tk;
  }
  return __builtin_amdgcn_readfirstlane(n);
}

// The keys of 32 * kWaves queries at most, first those at positions t0 .. t1 - 1: tiles of the sinks in front of the window, then
// of the window.
struct KeyTiles {
  int lo, n_sink_tiles, n_tiles, sinks, t1;
  __device__ __forceinline__ KeyTiles(const WinArgs &a, int t0, int t1_, int rows) : t1(t1_) {
    lo = t0 - a.W + 1 > 0 ? t0 - a.W + 1 : 0;
    sinks = a.S < lo ? a.S : lo;
    n_sink_tiles = (sinks + rows - 1) / rows;
    n_tiles = n_sink_tiles + (t1 - lo + rows - 1) / rows;
  }
  __device__ __forceinline__ int first(int it, int rows) const { return it < n_sink_tiles ? it * rows : lo + (it - n_sink_tiles) * rows; }
  __device__ __forceinline__ int end(int it) const { return it < n_sink_tiles ? sinks : t1; }
};

// Workgroup -> work item.  Consecutive workgroup ids go round-robin over the 8 XCDs: the workgroups of a block of
// position tiles of one unit, which read much the same keys, are given to one of them.
struct Item {
  int b, hkv, head, tile;   // head: first of the group's that the workgroup has
  bool none;
  __device__ __forceinline__ explicit Item(const WinArgs &a) {
    const int G = a.Hq / a.Hkv, heads = a.by_head ? G / kWaves : G;
    const int members = a.per_block * heads;
    const int xcd = blockIdx.x % kXcds, seq = blockIdx.x / kXcds;
    const int group = seq / members * kXcds + xcd, member = seq % members;
    const int u = group / a.blocks;
    tile = group % a.blocks * a.per_block + member / heads;
    head = member % heads * (a.by_head ? kWaves : 1);
    b = u / a.Hkv;
    hkv = u % a.Hkv;
    none = b >= a.B || tile >= a.tiles;
  }
};

template <typename T, int D>
__device__ __forceinline__ void load_row(const char *row, int g, Operand<T> (&f)[D / 16]) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const uint4 *p = reinterpret_cast<const uint4 *>(row + (16 * ks + 8 * g) * (int)sizeof(T));
    if constexpr (sizeof(T) == 2) {
      f[ks].f.q = p[0];
    } else {
      float x[4], y[4];
      unpack16<float>(p[0], x);
      unpack16<float>(p[1], y);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[ks].f[e] = x[e];
        f[ks].f[4 + e] = y[e];
      }
    }
  }
}

// Four channels (8 * vq + 4 * g .. + 3 of block blk) of an accumulator's column to memory.
template <typename T>
__device__ __forceinline__ void store4(char *row, int blk, int vq, int g, float x, float y, float z, float w) {
  char *p = row + (32 * blk + 8 * vq + 4 * g) * (int)sizeof(T);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x, y), pack_bf16(z, w));
  else *reinterpret_cast<float4 *>(p) = make_float4(x, y, z, w);
}
template <typename T>
__device__ __forceinline__ void load4(const char *row, int blk, int vq, int g, float (&x)[4]) {
  const char *p = row + (32 * blk + 8 * vq + 4 * g) * (int)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    x[0] = __uint_as_float(u.x << 16);
    x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16);
    x[3] = __uint_as_float(u.y & 0xffff0000u);
  } else {
    const float4 u = *reinterpret_cast<const float4 *>(p);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
  }
}

__device__ __forceinline__ float add_operand(const Operand<bf16_t> &x, float sum) {
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x.f.w[e]), ones, sum, false);
  return sum;
}
__device__ __forceinline__ float add_operand(const Operand<float> &x, float sum) {
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += x.f[e];
  return sum;
}

// A query done again, one visible key after the other in fp32 (a lane has half of its channels): a key that it does not see
// enters the second product of the tile kernels with p = 0, and a value of it that is not finite makes that NaN.  Every visible
// key has its part, whatever its place: a NaN logit, which fmaxf passes over, makes p and l NaN, a NaN value a NaN channel also
// where p is 0.  Nothing but logits of -infinity: zeros.
template <typename T, int D>
__device__ __forceinline__ void attend_one_by_one(const WinArgs &a, const char *qrow, const char *kb, const char *vb, int t, float c,
                                                  int g, f32x16 (&o)[D / 32], float &m, float &l) {
  constexpr int DB = D / 32;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
  m = -INFINITY;
  l = 0.f;
#pragma unroll 1
  for (int j = 0; j <= t; ++j) {
    if (j >= a.S && t - j >= a.W) {
      j = t - a.W;   // (the next one is the window's first)
      continue;
    }
    const char *kr = kb + (int64_t)j * a.k_t, *vr = vb + (int64_t)j * a.v_t;
    float dot = 0.f;
#pragma unroll 4
    for (int i = 0; i < 4 * DB; ++i) {
      float x[4], y[4];
      load4<T>(qrow, i >> 2, i & 3, g, x);
      load4<T>(kr, i >> 2, i & 3, g, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) dot = fmaf(x[e], y[e], dot);
    }
    const float x = xhalf_sum(dot) * c, m_new = fmaxf(m, x), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - ref), p = __builtin_amdgcn_exp2f(x - ref);
    m = m_new;
    l = fmaf(l, alpha, p);
    if (l != l) break;   // (NaN stays, and makes out and lse NaN whatever follows)
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      float y[4];
      load4<T>(vr, i >> 2, i & 3, g, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i >> 2][4 * (i & 3) + e] = fmaf(p, y[e], o[i >> 2][4 * (i & 3) + e] * alpha);
    }
  }
  if (l == 0.f)
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
}

// What a query's lane pair has in the end: o / l to out, what its rounding leaves to rest, the logarithm of the sum to lse.
template <typename T, int D>
__device__ __forceinline__ void write_query(const WinArgs &a, char *orow, float *lse, const f32x16 (&o)[D / 32], float m, float l, int g) {
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;   // (l = 0: every logit is -infinity)
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = o[i >> 2][4 * (i & 3) + e] * inv;
    store4<T>(orow, i >> 2, i & 3, g, x[0], x[1], x[2], x[3]);
    if constexpr (sizeof(T) == 2) {
      if (a.rest) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] -= __uint_as_float((uint32_t)float_to_bf16_bits(x[e]) << 16);
        store4<T>(a.rest + (orow - a.out), i >> 2, i & 3, g, x[0], x[1], x[2], x[3]);
      }
    }
  }
  if (lse && g == 0) *lse = (m + log2f(l)) * kLn2;
}
template <typename T, int D>
__device__ __forceinline__ bool all_finite(const f32x16 (&o)[D / 32], float l) {
  float bad = 0.f * l;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) bad = fmaf(o[i][v], 0.f, bad);
  return xhalf_sum(bad) == 0.f;
}

// Operands of two tiles, one read along its rows (K) and one across (V), whose addresses stay in registers: the step's and the
// buffer's parts are constants that fold into the instructions.
template <typename T, int D>
struct Fragments {
  using Tl = Tile<T, D>;
  static constexpr int kAlong = D / 16, kAcross = D / 32, kN = sizeof(T) == 2 ? 2 : 8;
  uint32_t al[kAlong], ac[kAcross][sizeof(T) == 2 ? 2 : 1];
  __device__ __forceinline__ Fragments(uint32_t at_k, uint32_t at_v, int lane) {
#pragma unroll
    for (int ks = 0; ks < kAlong; ++ks) al[ks] = (at_k + Tl::along0(lane)) ^ (uint32_t)(16 * (int)sizeof(T) * ks);
#pragma unroll
    for (int blk = 0; blk < kAcross; ++blk)
#pragma unroll
      for (int hi = 0; hi < (sizeof(T) == 2 ? 2 : 1); ++hi)
        ac[blk][hi] = (at_v + Tl::template across0<true>(lane)) ^ (uint32_t)(32 * (int)sizeof(T) * blk + 32 * hi);
  }
  __device__ __forceinline__ Operand<T> along(int blk, int ks, uint32_t buf) const {
    return Tl::along(al[ks] + buf, blk, 0);
  }
  __device__ __forceinline__ Operand<T> across(int blk, int ks, uint32_t buf) const {
    if constexpr (sizeof(T) == 2) {
      Operand<T> o;
#pragma unroll
      for (int hi = 0; hi < 2; ++hi)
        o.f.d[hi] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                  (__attribute__((address_space(3))) v4i16 *)(uintptr_t)(ac[blk][hi] + buf + (uint32_t)((16 * ks + 8 * hi) * Tl::kRowB))));
      return o;
    } else {
      return Tl::across(ac[blk][0] + buf, 0, ks);
    }
  }
};

// kFine (bf16): P enters the second product as two operands, with errors of 2^-16, where gradients will be asked for and rows are short
// (fine_rows).  What P's rounding moves, lse and D = dout . out, moves every dS of a row: dq and dk of rows of n keys would have
// the variance of 2 + 2 / n roundings instead of 2.
// (fp32 rows of 128 channels: with two workgroups to a CU registers spill; 2 sequences of 4096 tokens of 16 heads, window 512,
// take 385 us with one and 432 with two.)
template <typename T, int D, bool kFine>
__global__ __launch_bounds__(256, sizeof(T) * D > 256 ? 1 : kFine ? 2 : 3) void window_prefill_kernel(WinArgs a) {
  using Tl = Tile<T, D>;
  constexpr int kPlanes = kFine ? 2 : 1;
  constexpr int KT = kTileRows, NB = KT / 32, KS = D / 16, DB = D / 32;
  constexpr uint32_t kTileB = KT * Tl::kRowB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t at_k = lds_addr_of(lds), at_v = at_k + 2 * kTileB;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const Item w(a);
  if (w.none) return;
  const int G = a.Hq / a.Hkv, off = a.Tk - a.Tq;
  const int n = tokens_of(a, w.b);
  const int nq = n - off < 0 ? 0 : n - off;                           // queries of the sequence (n <= Tk: at most Tq)
  const int Q0 = w.tile * a.span, Q1 = Q0 + a.span < nq ? Q0 + a.span : nq;  // the workgroup's
  const int hq = w.hkv * G + w.head + (a.by_head ? wave : 0);
  const int myq = Q0 + (a.by_head ? 0 : 32 * wave) + l32;
  char *orow = a.out + w.b * a.o_b + (int64_t)myq * a.o_t + (int64_t)hq * a.o_h;
  float *lse = a.lse ? a.lse + w.b * a.l_b + (int64_t)myq * a.l_t + (int64_t)hq * a.l_h : nullptr;
  if (myq >= nq && myq < a.Tq) {   // behind the sequence
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) store4<T>(orow, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
    if (lse && g == 0) *lse = -INFINITY;
  }
  if (Q0 >= nq) return;
  const int t = myq + off;   // position of the lane's query
  const KeyTiles keys(a, Q0 + off, Q1 + off, KT);

  Operand<T> qf[KS];
  {
    const int qc = myq < nq ? myq : nq - 1;
    load_row<T, D>(a.q + w.b * a.q_b + (int64_t)qc * a.q_t + (int64_t)hq * a.q_h, g, qf);
  }
  const char *kb = uniform_ptr(a.k + w.b * a.k_b + (int64_t)w.hkv * a.k_h);
  const char *vb = uniform_ptr(a.v + w.b * a.v_b + (int64_t)w.hkv * a.v_h);
  auto load_tile = [&](int it) {
    const int j0 = keys.first(it, KT), nv = keys.end(it) - j0;
    const uint32_t buf = (uint32_t)(it & 1) * kTileB;
    Tl::template fill<KT, kWaves, false>(kb + (int64_t)j0 * a.k_t, (uint32_t)a.k_t, nv, at_k + buf, wave, lane);
    Tl::template fill<KT, kWaves, false>(vb + (int64_t)j0 * a.v_t, (uint32_t)a.v_t, nv, at_v + buf, wave, lane);
  };
  const float c = a.scale * kLog2e;
  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int wt0 = off + Q0 + (a.by_head ? 0 : 32 * wave);   // position of the wave's first query
  // LDS addresses of the lane's fragments, but for constants
  const Fragments<T, D> fr(at_k, at_v, lane);
  const int n_tiles = __builtin_amdgcn_readfirstlane(keys.n_tiles);
  auto tile_step = [&](int it, auto parity) {
    constexpr uint32_t kBuf = decltype(parity)::value * kTileB;
    wait_vmem<0>();
    publish();
    if (it + 1 < n_tiles) load_tile(it + 1);
    const int j0 = keys.first(it, KT), j1 = keys.end(it);
    if (j0 > wt0 + 31) return;   // all behind the wave's queries
    f32x16 s[NB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) s[blk] = mma(fr.along(blk, ks, kBuf), qf[ks], ks == 0 ? f32x16{0.f} : s[blk]);
    // every pair is visible: keys j0 .. j0 + KT - 1 up to the first query's position and inside the last one's window
    if (!(j0 + KT <= j1 && j0 + KT - 1 <= wt0 && (wt0 + 31 - j0 < a.W || j0 + KT <= a.S))) {
      // of the lane's tile rows, those up to `last` are visible, and of them those from `first` on or below `sink`
      const int last = (t < j1 - 1 ? t : j1 - 1) - j0 - 4 * g, first = t - a.W + 1 - j0 - 4 * g, sink = a.S - j0 - 4 * g;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * blk + mfma_row(v, 0);
          s[blk][v] = r <= last && (r >= first || r < sink) ? s[blk][v] : -INFINITY;
        }
    }
    // P enters the second product in the I/O dtype; the sum is taken over the rounded values, so that numerator and
    // denominator see the same ones
    Operand<T> pf[2 * NB][kPlanes];
    auto exponentials = [&]() {
      const float ref = m == -INFINITY ? 0.f : m;   // (nothing seen yet)
      float sum = 0.f;
#pragma unroll
      for (int ks = 0; ks < 2 * NB; ++ks) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[ks >> 1][8 * (ks & 1) + e], c, -ref));
        split_operand<kPlanes>(p, pf[ks]);
#pragma unroll
        for (int n = 0; n < kPlanes; ++n) sum = add_operand(pf[ks][n], sum);
      }
      return sum;
    };
    // m is the reference of the exponentials: it moves to the maximum when a lane's sum of them passes 2^12 (in fp32 and bf16 a p of up
    // to 2^12 is as exact as one of up to 1), so that most tiles need no maximum (2 sequences of 16k tokens, 32 heads on 8, window 2048:
    // 1065 us, 1100 with one in every tile)
    float sum = exponentials();
    if (__builtin_amdgcn_ballot_w64(!(sum <= 4096.f) || m == -INFINITY) != 0) {
      float top = s[0][0];
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, s[blk][v]);
      top = xhalf_max(top) * c;
      const float m_new = fmaxf(m, top);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
      sum = exponentials();
    }
    l += sum;
#pragma unroll
    for (int ks = 0; ks < 2 * NB; ++ks)
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const Operand<T> vt = fr.across(i, ks, kBuf);
#pragma unroll
        for (int n = 0; n < kPlanes; ++n) o[i] = mma(vt, pf[ks][n], o[i]);
      }
  };
  __builtin_amdgcn_s_waitcnt(0);
  load_tile(0);
  for (int it = 0; it < n_tiles; it += 2) {
    tile_step(it, std::integral_constant<uint32_t, 0>{});
    if (it + 1 < n_tiles) tile_step(it + 1, std::integral_constant<uint32_t, 1>{});
  }
  l = xhalf_sum(l);
  if (myq >= nq) return;
  if (!all_finite<T, D>(o, l))
    attend_one_by_one<T, D>(a, a.q + w.b * a.q_b + (int64_t)myq * a.q_t + (int64_t)hq * a.q_h, kb, vb, t, c, g, o, m, l);
  write_query<T, D>(a, orow, lse, o, m, l, g);
}

// The same where there are few queries: the four waves of a workgroup take the same 32 queries of one head and a quarter of the key tiles
// each, in LDS of their own and without a barrier, and their results are joined in the end.  What bounds such calls is the time of one
// workgroup's loop, which is a quarter as long.
template <typename T, int D>
constexpr size_t split_lds() {
  return kWaves * (2 * (size_t)kTileRows * D * sizeof(T) + 2 * 64 * sizeof(float)) + 32 * sizeof(int);
}
template <typename T, int D, bool kFine>
__global__ __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) void window_prefill_split_kernel(WinArgs a) {
  using Tl = Tile<T, D>;
  constexpr int kPlanes = kFine ? 2 : 1;
  constexpr int KT = kTileRows, NB = KT / 32, KS = D / 16, DB = D / 32;
  constexpr uint32_t kTileB = KT * Tl::kRowB;
  constexpr int kLoads = (int)(kTileB / 1024);   // of a wave for a tile
  static_assert(2 * kTileB >= 64 * 16 * DB * sizeof(float), "a wave's result fits its tiles");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const uint32_t at_k = lds_addr_of(lds) + (uint32_t)wave * (2 * kTileB), at_v = at_k + kTileB;
  float *stats = reinterpret_cast<float *>(lds + kWaves * 2 * kTileB);   // [wave][m | l][lane]
  int *redo = reinterpret_cast<int *>(stats + kWaves * 128);             // [query]
  const Item w(a);
  if (w.none) return;
  const int G = a.Hq / a.Hkv, off = a.Tk - a.Tq;
  const int n = tokens_of(a, w.b);
  const int nq = n - off < 0 ? 0 : n - off;
  const int Q0 = w.tile * 32, Q1 = Q0 + 32 < nq ? Q0 + 32 : nq;
  const int hq = w.hkv * G + w.head, myq = Q0 + l32, t = myq + off;
  char *orow = a.out + w.b * a.o_b + (int64_t)myq * a.o_t + (int64_t)hq * a.o_h;
  float *lse = a.lse ? a.lse + w.b * a.l_b + (int64_t)myq * a.l_t + (int64_t)hq * a.l_h : nullptr;
  if (wave == 0 && myq >= nq && myq < a.Tq) {   // behind the sequence
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) store4<T>(orow, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
    if (lse && g == 0) *lse = -INFINITY;
  }
  if (Q0 >= nq) return;
  if (tid < 32) redo[tid] = 0;
  const KeyTiles keys(a, Q0 + off, Q1 + off, KT);
  const int n_tiles = __builtin_amdgcn_readfirstlane(keys.n_tiles);
  const char *kb = uniform_ptr(a.k + w.b * a.k_b + (int64_t)w.hkv * a.k_h);
  const char *vb = uniform_ptr(a.v + w.b * a.v_b + (int64_t)w.hkv * a.v_h);
  auto load_k = [&](int it) {
    const int j0 = keys.first(it, KT);
    Tl::template fill<KT, 1, false>(kb + (int64_t)j0 * a.k_t, (uint32_t)a.k_t, keys.end(it) - j0, at_k, 0, lane);
  };
  auto load_v = [&](int it) {
    const int j0 = keys.first(it, KT);
    Tl::template fill<KT, 1, false>(vb + (int64_t)j0 * a.v_t, (uint32_t)a.v_t, keys.end(it) - j0, at_v, 0, lane);
  };
  Operand<T> qf[KS];
  const char *qrow = a.q + w.b * a.q_b + (int64_t)(myq < nq ? myq : nq - 1) * a.q_t + (int64_t)hq * a.q_h;
  load_row<T, D>(qrow, g, qf);
  const float c = a.scale * kLog2e;
  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) o[i] = f32x16{0.f};
  float m = -INFINITY, l = 0.f;
  const Fragments<T, D> fr(at_k, at_v, lane);
  __builtin_amdgcn_s_waitcnt(0);
  if (wave < n_tiles) {
    load_k(wave);
    load_v(wave);
  }
  for (int it = wave; it < n_tiles; it += kWaves) {
    const bool more = it + kWaves < n_tiles;
    const int j0 = keys.first(it, KT), j1 = keys.end(it);
    wait_vmem<kLoads>();   // k (v was asked for behind it)
    f32x16 s[NB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) s[blk] = mma(fr.along(blk, ks, 0), qf[ks], ks == 0 ? f32x16{0.f} : s[blk]);
    if (!(j0 + KT <= j1 && j0 + KT - 1 <= off + Q0 && (off + Q0 + 31 - j0 < a.W || j0 + KT <= a.S))) {
      const int last = (t < j1 - 1 ? t : j1 - 1) - j0 - 4 * g, first = t - a.W + 1 - j0 - 4 * g, sink = a.S - j0 - 4 * g;
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * blk + mfma_row(v, 0);
          s[blk][v] = r <= last && (r >= first || r < sink) ? s[blk][v] : -INFINITY;
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the k tile has been read
    if (more) load_k(it + kWaves);
    float top = s[0][0];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[blk][v]);
    const float m_new = fmaxf(m, xhalf_max(top) * c);
    const float ref = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m - ref);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
    if (more) wait_vmem<kLoads>();   // v (the next k was asked for behind it)
    else wait_vmem<0>();
#pragma unroll
    for (int ks = 0; ks < 2 * NB; ++ks) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[ks >> 1][8 * (ks & 1) + e], c, -ref));
      Operand<T> pf[kPlanes];
      split_operand<kPlanes>(p, pf);
#pragma unroll
      for (int n = 0; n < kPlanes; ++n) l = add_operand(pf[n], l);
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const Operand<T> vt = fr.across(i, ks, 0);
#pragma unroll
        for (int n = 0; n < kPlanes; ++n) o[i] = mma(vt, pf[n], o[i]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the v tile has been read
    if (more) load_v(it + kWaves);
  }
  // every wave's result, then a block of channels by each of them
  float *mine = reinterpret_cast<float *>(lds + wave * 2 * kTileB);
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) mine[(16 * i + v) * 64 + lane] = o[i][v];
  stats[wave * 128 + lane] = m;
  stats[wave * 128 + 64 + lane] = xhalf_sum(l);
  __syncthreads();
  m = -INFINITY;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) m = fmaxf(m, stats[x * 128 + lane]);
  l = 0.f;
  float f[kWaves];
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    f[x] = stats[x * 128 + lane] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stats[x * 128 + lane] - m);
    l = fmaf(f[x], stats[x * 128 + 64 + lane], l);
  }
  f32x16 sum = {0.f};
  if (wave < DB) {
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float *theirs = reinterpret_cast<const float *>(lds + x * 2 * kTileB) + 16 * wave * 64 + lane;
#pragma unroll
      for (int v = 0; v < 16; ++v) sum[v] = fmaf(f[x], theirs[v * 64], sum[v]);
    }
    float bad = 0.f * l;
#pragma unroll
    for (int v = 0; v < 16; ++v) bad = fmaf(sum[v], 0.f, bad);
    if (!(xhalf_sum(bad) == 0.f)) redo[l32] = 1;
  }
  __syncthreads();
  if (myq >= nq) return;
  if (redo[l32]) {
    if (wave == 0) {
      attend_one_by_one<T, D>(a, qrow, kb, vb, t, c, g, o, m, l);
      write_query<T, D>(a, orow, lse, o, m, l, g);
    }
    return;
  }
  if (wave < DB) {
    o[0] = sum;
    write_query<T, 32>(a, orow + 32 * wave * (int)sizeof(T), wave == 0 ? lse : nullptr, reinterpret_cast<const f32x16(&)[1]>(o[0]), m, l, g);
  }
}

// ------------------------------------------------------------------------------------------------
// Gradients.  P = 2^(S scale log2 e - lse log2 e) is formed again; D = dout . out of a query, out with what its rounding left;
//   dS = P (dP - D),  dq = scale dS K (queries stay, keys stream),  dk = scale dS^T q, dv = P^T dout (keys stay, queries stream).
// P and dS enter their products in the I/O dtype.
// (a query all of whose logits are -infinity has nothing of any key: P = 0)
__device__ __forceinline__ float lse_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// The lane's query for the dq kernels: q and dout, lse in powers of two, D = dout . out.
template <typename T, int D>
__device__ __forceinline__ void load_query(const WinArgs &a, int b, int hq, int myq, int nq, int g, Operand<T> (&qf)[D / 16],
                                           Operand<T> (&df)[D / 16], float &lse2, float &delta) {
  const int qc = myq < nq ? myq : nq - 1;
  const int64_t at = b * a.o_b + (int64_t)qc * a.o_t + (int64_t)hq * a.o_h;
  load_row<T, D>(a.q + at, g, qf);
  load_row<T, D>(a.dout + at, g, df);
  lse2 = lse_log2(a.lse[b * a.l_b + (int64_t)qc * a.l_t + (int64_t)hq * a.l_h]);
  delta = 0.f;
  auto add = [&](const char *row) {
    Operand<T> of[D / 16];
    load_row<T, D>(row, g, of);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      float x[8], y[8];
      from_operand(of[ks], x);
      from_operand(df[ks], y);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(x[e], y[e], delta);
    }
  };
  add(a.out + at);
  if (sizeof(T) == 2 && a.rest) add(a.rest + at);
  delta = xhalf_sum(delta);
}

template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) void window_dq_kernel(WinArgs a) {
  using Tl = Tile<T, D>;
  constexpr int KT = kTileRows, NB = KT / 32, KS = D / 16, DB = D / 32;
  constexpr uint32_t kTileB = KT * Tl::kRowB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t at_k = lds_addr_of(lds), at_v = at_k + 2 * kTileB;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const Item w(a);
  if (w.none) return;
  const int G = a.Hq / a.Hkv, off = a.Tk - a.Tq;
  const int n = tokens_of(a, w.b);
  const int nq = n - off < 0 ? 0 : n - off;
  const int Q0 = w.tile * a.span, Q1 = Q0 + a.span < nq ? Q0 + a.span : nq;
  const int hq = w.hkv * G + w.head + (a.by_head ? wave : 0);
  const int myq = Q0 + (a.by_head ? 0 : 32 * wave) + l32;
  const int64_t at_row = w.b * a.o_b + (int64_t)myq * a.o_t + (int64_t)hq * a.o_h;
  if (myq >= nq && myq < a.Tq) {
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) store4<T>(a.dq + at_row, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
  }
  if (Q0 >= nq) return;
  const int t = myq + off;
  const KeyTiles keys(a, Q0 + off, Q1 + off, KT);
  const char *kb = uniform_ptr(a.k + w.b * a.k_b + (int64_t)w.hkv * a.k_h);
  const char *vb = uniform_ptr(a.v + w.b * a.v_b + (int64_t)w.hkv * a.v_h);
  auto load_tile = [&](int it) {
    const int j0 = keys.first(it, KT), nv = keys.end(it) - j0;
    const uint32_t buf = (uint32_t)(it & 1) * kTileB;
    Tl::template fill<KT, kWaves, false>(kb + (int64_t)j0 * a.k_t, (uint32_t)a.k_t, nv, at_k + buf, wave, lane);
    Tl::template fill<KT, kWaves, false>(vb + (int64_t)j0 * a.v_t, (uint32_t)a.v_t, nv, at_v + buf, wave, lane);
  };
  load_tile(0);
  Operand<T> qf[KS], df[KS];
  float lse2, delta;
  load_query<T, D>(a, w.b, hq, myq, nq, g, qf, df, lse2, delta);
  if (myq < nq && g == 0) a.delta[((int64_t)w.b * a.Hq + hq) * a.Tq + myq] = delta;
  const float c = a.scale * kLog2e;
  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
  const int wt0 = off + Q0 + (a.by_head ? 0 : 32 * wave);
  const Fragments<T, D> fr(at_k, at_k, lane);
  const int n_tiles = __builtin_amdgcn_readfirstlane(keys.n_tiles);
  auto tile_step = [&](int it, auto parity) {
    constexpr uint32_t kBuf = decltype(parity)::value * kTileB;
    wait_vmem<0>();
    publish();
    if (it + 1 < n_tiles) load_tile(it + 1);
    const int j0 = keys.first(it, KT), j1 = keys.end(it);
    if (j0 > wt0 + 31) return;
    const bool masked = !(j0 + KT <= j1 && j0 + KT - 1 <= wt0 && (wt0 + 31 - j0 < a.W || j0 + KT <= a.S));
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      f32x16 s, dp;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = mma(fr.along(blk, ks, kBuf), qf[ks], ks == 0 ? f32x16{0.f} : s);
        dp = mma(fr.along(blk, ks, kBuf + 2 * kTileB), df[ks], ks == 0 ? f32x16{0.f} : dp);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse2)) * (dp[v] - delta);
      if (masked) {
        const int last = (t < j1 - 1 ? t : j1 - 1) - j0 - 4 * g, first = t - a.W + 1 - j0 - 4 * g, sink = a.S - j0 - 4 * g;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * blk + mfma_row(v, 0);
          s[v] = r <= last && (r >= first || r < sink) ? s[v] : 0.f;
        }
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[8 * hf + e];
        Operand<T> ds;
        to_operand(x, ds);
#pragma unroll
        for (int i = 0; i < DB; ++i) o[i] = mma(fr.across(i, 2 * blk + hf, kBuf), ds, o[i]);
      }
    }
  };
  __builtin_amdgcn_s_waitcnt(0);
  for (int it = 0; it < n_tiles; it += 2) {
    tile_step(it, std::integral_constant<uint32_t, 0>{});
    if (it + 1 < n_tiles) tile_step(it + 1, std::integral_constant<uint32_t, 1>{});
  }
  if (myq >= nq) return;
#pragma unroll
  for (int i = 0; i < 4 * DB; ++i)
    store4<T>(a.dq + at_row, i >> 2, i & 3, g, a.scale * o[i >> 2][4 * (i & 3)], a.scale * o[i >> 2][4 * (i & 3) + 1],
              a.scale * o[i >> 2][4 * (i & 3) + 2], a.scale * o[i >> 2][4 * (i & 3) + 3]);
}

// dq where there are few queries: waves share the key tiles of 32 queries, as in window_prefill_split_kernel.
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) void window_dq_split_kernel(WinArgs a) {
  using Tl = Tile<T, D>;
  constexpr int KT = kTileRows, NB = KT / 32, KS = D / 16, DB = D / 32;
  constexpr uint32_t kTileB = KT * Tl::kRowB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const uint32_t at_k = lds_addr_of(lds) + (uint32_t)wave * (2 * kTileB), at_v = at_k + kTileB;
  const Item w(a);
  if (w.none) return;
  const int G = a.Hq / a.Hkv, off = a.Tk - a.Tq;
  const int n = tokens_of(a, w.b);
  const int nq = n - off < 0 ? 0 : n - off;
  const int Q0 = w.tile * 32, Q1 = Q0 + 32 < nq ? Q0 + 32 : nq;
  const int hq = w.hkv * G + w.head, myq = Q0 + l32, t = myq + off;
  char *row = a.dq + w.b * a.o_b + (int64_t)myq * a.o_t + (int64_t)hq * a.o_h;
  if (wave == 0 && myq >= nq && myq < a.Tq) {
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) store4<T>(row, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
  }
  if (Q0 >= nq) return;
  const KeyTiles keys(a, Q0 + off, Q1 + off, KT);
  const int n_tiles = __builtin_amdgcn_readfirstlane(keys.n_tiles);
  const char *kb = uniform_ptr(a.k + w.b * a.k_b + (int64_t)w.hkv * a.k_h);
  const char *vb = uniform_ptr(a.v + w.b * a.v_b + (int64_t)w.hkv * a.v_h);
  auto load_tile = [&](int it) {
    const int j0 = keys.first(it, KT), nv = keys.end(it) - j0;
    Tl::template fill<KT, 1, false>(kb + (int64_t)j0 * a.k_t, (uint32_t)a.k_t, nv, at_k, 0, lane);
    Tl::template fill<KT, 1, false>(vb + (int64_t)j0 * a.v_t, (uint32_t)a.v_t, nv, at_v, 0, lane);
  };
  if (wave < n_tiles) load_tile(wave);
  Operand<T> qf[KS], df[KS];
  float lse2, delta;
  load_query<T, D>(a, w.b, hq, myq, nq, g, qf, df, lse2, delta);
  if (wave == 0 && myq < nq && g == 0) a.delta[((int64_t)w.b * a.Hq + hq) * a.Tq + myq] = delta;
  const float c = a.scale * kLog2e;
  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) o[i] = f32x16{0.f};
  const Fragments<T, D> fr(at_k, at_k, lane);
  for (int it = wave; it < n_tiles; it += kWaves) {
    wait_vmem<0>();
    const int j0 = keys.first(it, KT), j1 = keys.end(it);
    const bool masked = !(j0 + KT <= j1 && j0 + KT - 1 <= off + Q0 && (off + Q0 + 31 - j0 < a.W || j0 + KT <= a.S));
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      f32x16 s, dp;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = mma(fr.along(blk, ks, 0), qf[ks], ks == 0 ? f32x16{0.f} : s);
        dp = mma(fr.along(blk, ks, kTileB), df[ks], ks == 0 ? f32x16{0.f} : dp);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse2)) * (dp[v] - delta);
      if (masked) {
        const int last = (t < j1 - 1 ? t : j1 - 1) - j0 - 4 * g, first = t - a.W + 1 - j0 - 4 * g, sink = a.S - j0 - 4 * g;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * blk + mfma_row(v, 0);
          s[v] = r <= last && (r >= first || r < sink) ? s[v] : 0.f;
        }
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[8 * hf + e];
        Operand<T> ds;
        to_operand(x, ds);
#pragma unroll
        for (int i = 0; i < DB; ++i) o[i] = mma(fr.across(i, 2 * blk + hf, 0), ds, o[i]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
    if (it + kWaves < n_tiles) load_tile(it + kWaves);
  }
  float *mine = reinterpret_cast<float *>(lds + wave * 2 * kTileB);
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) mine[(16 * i + v) * 64 + lane] = o[i][v];
  __syncthreads();
  if (myq >= nq || wave >= DB) return;
  float sum[16];
#pragma unroll
  for (int v = 0; v < 16; ++v) sum[v] = 0.f;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    const float *theirs = reinterpret_cast<const float *>(lds + x * 2 * kTileB) + 16 * wave * 64 + lane;
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[v] += theirs[v * 64];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    store4<T>(row, wave, i, g, a.scale * sum[4 * i], a.scale * sum[4 * i + 1], a.scale * sum[4 * i + 2], a.scale * sum[4 * i + 3]);
}

// dk and dv of 128 keys, 32 to a wave (K in registers, V in LDS); the queries that see them, head after head of the group, stream
// in tiles of 32.  Sinks (keys below S) are also seen by every query beyond their window: by workgroups of their own (far), the first of
// the launch, which cut those into n_split ranges; a workgroup's waves share its range's tiles among them (or the sinks, 32 to a wave),
// each with tiles of its own and no barrier.  What ranges and window give for sinks is added up by window_sinks_kernel.  (All gradients,
// us, far in the same launch / in one of its own: fp32, 3 x 777 tokens, 6 heads on 2, 75 / 94; bf16, 2k, 16 heads of 64, 54 / 58;
// fp32, 2 x 4k, 16 heads of 128 on 4, 1210 / 1237; bf16, 2 x 8k, 16 heads of 128 on 2, 852 / 844.)
template <typename T, int D>
constexpr size_t kv_lds() {
  return (4 * 32 + 128) * (size_t)D * sizeof(T) + 4 * 64 * sizeof(float);
}
template <typename T, int D, bool far>
__device__ __forceinline__ void key_gradients(const WinArgs &a, int block) {
  using Tl = Tile<T, D>;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr uint32_t kTileB = 32 * Tl::kRowB;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t at_s = lds_addr_of(lds), at_v = at_s + 4 * kTileB;   // stage: q tile, dout tile; then 128 rows of v
  float *rows = reinterpret_cast<float *>(lds + 8 * kTileB);           // [stage or wave][lse, in powers of two | D][32]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const int G = a.Hq / a.Hkv, off = a.Tk - a.Tq, units = a.B * a.Hkv;
  // a unit's workgroups go to one XCD
  const int per_unit = far ? a.n_split : a.key_tiles * a.n_part;
  const int u = block / kXcds / per_unit * kXcds + block % kXcds;
  const int member = block / kXcds % per_unit / (far ? 1 : a.n_part), queries = block / kXcds % (far ? 1 : a.n_part);
  if (u >= units) return;
  const int b = u / a.Hkv, hkv = u % a.Hkv;
  const int n = tokens_of(a, b);
  const int n_kb = a.sink_rows / 32, tw = wave / n_kb;   // far: blocks of sinks, the wave's part of the tiles
  const int K0 = far ? 0 : 128 * member;
  const int kend = far ? (a.S < n ? a.S : n) : (K0 + 128 < n ? K0 + 128 : n);
  const int wk0 = K0 + 32 * (far ? wave % n_kb : wave), key = wk0 + l32;
  // positions of the queries streamed
  int t0, t1;
  if (far) {
    t0 = a.W + member * a.split_q;
    t1 = t0 + a.split_q;
  } else {
    t0 = K0;
    t1 = K0 + 127 + a.W;
  }
  t0 = t0 > off ? t0 : off;
  t1 = t1 < n ? t1 : n;
  const int n_rows = kend > K0 && t1 > t0 ? t1 - t0 : 0;
  // this workgroup's tiles, of 32 queries of a head: those from it0 on of all
  const int all_tiles = (n_rows + 31) / 32 * G, per_part = far ? all_tiles : (all_tiles + a.n_part - 1) / a.n_part;
  const int it0 = far ? 0 : queries * per_part;
  const int n_tiles = all_tiles - it0 < per_part ? all_tiles - it0 : per_part;

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[i][v] = dv[i][v] = 0.f;
  if (n_tiles > 0) {
    const char *kb = uniform_ptr(a.k + b * a.k_b + (int64_t)hkv * a.k_h);
    const char *vb = uniform_ptr(a.v + b * a.v_b + (int64_t)hkv * a.v_h);
    const char *qb = uniform_ptr(a.q + b * a.o_b + (int64_t)(hkv * G) * a.o_h + (int64_t)(t0 - off) * a.o_t);
    const char *db = uniform_ptr(a.dout + b * a.o_b + (int64_t)(hkv * G) * a.o_h + (int64_t)(t0 - off) * a.o_t);
    // the tile asked for last: 32 queries from t0 + str_row on, of one head
    int str_row = it0 / G * 32, str_head = it0 % G;
    // lse (the lower half of the wave) or D of its rows
    auto row_value = [&]() {
      int r = str_row + l32;
      r = (r < n_rows ? r : n_rows - 1) + t0 - off;
      return g == 0 ? a.lse[b * a.l_b + (int64_t)r * a.l_t + (int64_t)(hkv * G + str_head) * a.l_h]
                    : a.delta[((int64_t)b * a.Hq + hkv * G + str_head) * a.Tq + r];
    };
    const float c = a.scale * kLog2e;
    Operand<T> kf[KS];
    load_row<T, D>(kb + (int64_t)(key < kend ? key : kend - 1) * a.k_t, g, kf);
    // P and dS of a tile whose logits are in s and dP in dp, lse and D of its rows at rl
    auto weights = [&](f32x16 &s, f32x16 &dp, const float *rl) {
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const float4 x = *reinterpret_cast<const float4 *>(rl + 4 * g + 8 * v4);
        const float4 y = *reinterpret_cast<const float4 *>(rl + 4 * g + 32 + 8 * v4);
        const float lse4[4] = {x.x, x.y, x.z, x.w}, d4[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int v = 4 * v4 + e;
          s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse4[e]));
          dp[v] = s[v] * (dp[v] - d4[e]);
        }
      }
    };
    // rows first .. last of the tile see the lane's key
    auto mask = [&](f32x16 &s, f32x16 &dp, int first, int last) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = mfma_row(v, 0) + 4 * g;
        const bool sees = r >= first && r <= last;
        s[v] = sees ? s[v] : 0.f;
        dp[v] = sees ? dp[v] : 0.f;
      }
    };
    // dv += dout^T P, dk += q^T dS
    auto add_up = [&](const f32x16 &s, const f32x16 &dp, const Fragments<T, D> &fr, uint32_t buf) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float p[8], ds[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = s[8 * hf + e];
          ds[e] = dp[8 * hf + e];
        }
        Operand<T> pf, sf;
        to_operand(p, pf);
        to_operand(ds, sf);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          dv[i] = mma(fr.across(i, hf, buf + kTileB), pf, dv[i]);
          dk[i] = mma(fr.across(i, hf, buf), sf, dk[i]);
        }
      }
    };
    if constexpr (far) {
      const int step = kWaves / n_kb;   // tiles of this wave: tw, tw + step, ..
      const uint32_t at = at_s + (uint32_t)wave * (2 * kTileB);
      const Fragments<T, D> fr(at, at, lane);
      Operand<T> vf[KS];
      load_row<T, D>(vb + (int64_t)(key < kend ? key : kend - 1) * a.v_t, g, vf);
      for (int it = tw; it < n_tiles; it += step) {
        str_head = it % G;
        str_row = it / G * 32;
        const int64_t o = (int64_t)str_row * a.o_t + (int64_t)str_head * a.o_h;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile before has been read
        Tl::template fill<32, 1, false>(qb + o, (uint32_t)a.o_t, n_rows - str_row, at, 0, lane);
        Tl::template fill<32, 1, false>(db + o, (uint32_t)a.o_t, n_rows - str_row, at + kTileB, 0, lane);
        const float row = row_value();
        rows[wave * 64 + lane] = g == 0 ? lse_log2(row) : row;
        wait_vmem<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        f32x16 s, dp;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mma(fr.along(0, ks, 0), kf[ks], ks == 0 ? f32x16{0.f} : s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mma(fr.along(0, ks, kTileB), vf[ks], ks == 0 ? f32x16{0.f} : dp);
        weights(s, dp, rows + wave * 64);
        const int p0 = t0 + str_row;
        mask(s, dp, key + a.W - p0, key < kend ? t1 - 1 - p0 : -1);
        add_up(s, dp, fr, 0);
      }
    } else {
      float row = 0.f;
      auto load_tile = [&](uint32_t buf) {
        const int nv = n_rows - str_row;
        const int64_t o = (int64_t)str_row * a.o_t + (int64_t)str_head * a.o_h;
        Tl::template fill<32, kWaves, false>(qb + o, (uint32_t)a.o_t, nv, at_s + buf, wave, lane);
        Tl::template fill<32, kWaves, false>(db + o, (uint32_t)a.o_t, nv, at_s + buf + kTileB, wave, lane);
        if (wave == 0) row = row_value();
      };
      load_tile(0);
      Tl::template fill<128, kWaves, false>(vb + (int64_t)K0 * a.v_t, (uint32_t)a.v_t, kend - K0, at_v, wave, lane);
      const Fragments<T, D> fr(at_s, at_s, lane);
      const uint32_t at_rows = at_v + (uint32_t)(32 * wave * Tl::kRowB) + Tl::along0(lane);   // of the wave's rows of v
      auto tile_step = [&](int it, auto parity) {
        constexpr uint32_t kBuf = decltype(parity)::value * (2 * kTileB);
        if (wave == 0) rows[decltype(parity)::value * 64 + lane] = g == 0 ? lse_log2(row) : row;
        wait_vmem<0>();
        publish();
        const int p0 = t0 + str_row;   // position of the tile's first query
        if (it + 1 < n_tiles) {
          if (++str_head == G) {
            str_head = 0;
            str_row += 32;
          }
          load_tile(2 * kTileB - kBuf);
        }
        if (wk0 >= kend || p0 + 31 < wk0 || p0 - (wk0 + 31) >= a.W) return;
        const uint32_t v0 = here(at_rows);
        // (ahead of the other workgroup's wave while this one feeds the matrix cores: 752 us of the 2 x 8k shape, 708 with it)
        __builtin_amdgcn_s_setprio(1);
        f32x16 s, dp;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mma(fr.along(0, ks, kBuf), kf[ks], ks == 0 ? f32x16{0.f} : s);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mma(fr.along(0, ks, kBuf + kTileB), Tl::along(v0, 0, ks), ks == 0 ? f32x16{0.f} : dp);
        __builtin_amdgcn_s_setprio(0);
        weights(s, dp, rows + decltype(parity)::value * 64);
        if (!(p0 >= wk0 + 31 && p0 + 31 - wk0 < a.W && p0 + 32 <= t1))
          mask(s, dp, key - p0, (key + a.W < t1 ? key + a.W : t1) - 1 - p0);
        add_up(s, dp, fr, kBuf);
      };
      for (int it = 0; it < n_tiles; it += 2) {
        tile_step(it, std::integral_constant<uint32_t, 0>{});
        if (it + 1 < n_tiles) tile_step(it + 1, std::integral_constant<uint32_t, 1>{});
      }
    }
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) dk[i][v] *= a.scale;
  }
  if (!far && a.n_part > 1) {   // added up by window_sum_kernel
    if (key < a.Tk) {
      float *pk = a.sums + (((int64_t)u * a.n_part + queries) * 2 * a.Tk + key) * D;
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
        const f32x16 &x = dk[i >> 2], &y = dv[i >> 2];
        const int v = 4 * (i & 3);
        store4<float>((char *)pk, i >> 2, i & 3, g, x[v], x[v + 1], x[v + 2], x[v + 3]);
        store4<float>((char *)(pk + (int64_t)a.Tk * D), i >> 2, i & 3, g, y[v], y[v + 1], y[v + 2], y[v + 3]);
      }
    }
    return;
  }
  if (far || key < a.S) {   // a sink's share
    if (key < a.S) {
      const int share = far ? member * (kWaves / n_kb) + tw : a.parts - 1;
      float *pk = a.part + ((((int64_t)u * a.parts + share) * 2) * a.sink_rows + key) * D;
      float *pv = pk + (int64_t)a.sink_rows * D;
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ch = 32 * (i >> 2) + 8 * (i & 3) + 4 * g + e;
          pk[ch] = dk[i >> 2][4 * (i & 3) + e];
          pv[ch] = dv[i >> 2][4 * (i & 3) + e];
        }
    }
    return;
  }
  if (key < a.Tk) {
    char *pk = a.dk + b * a.k_b + (int64_t)key * a.k_t + (int64_t)hkv * a.k_h;
    char *pv = a.dv + b * a.v_b + (int64_t)key * a.v_t + (int64_t)hkv * a.v_h;
    const float z = key < n ? 1.f : 0.f;   // (a wave's last keys may be behind the sequence)
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      const f32x16 &x = dk[i >> 2], &y = dv[i >> 2];
      const int v = 4 * (i & 3);
      if (z != 0.f) {
        store4<T>(pk, i >> 2, i & 3, g, x[v], x[v + 1], x[v + 2], x[v + 3]);
        store4<T>(pv, i >> 2, i & 3, g, y[v], y[v + 1], y[v + 2], y[v + 3]);
      } else {
        store4<T>(pk, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
        store4<T>(pv, i >> 2, i & 3, g, 0.f, 0.f, 0.f, 0.f);
      }
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D <= 256 ? 2 : 1) void window_dkv_kernel(WinArgs a) {
  if ((int)blockIdx.x < a.far_wgs) key_gradients<T, D, true>(a, blockIdx.x);
  else key_gradients<T, D, false>(a, blockIdx.x - a.far_wgs);
}

// dk and dv where a key tile's queries are shared among workgroups: the sums of the parts, and of a sink's far shares.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_sum_kernel(WinArgs a) {
  const int u = blockIdx.y, b = u / a.Hkv, hkv = u % a.Hkv;
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x), n = (int64_t)a.Tk * D;
  if (i >= 2 * n) return;
  const int which = i >= n, key = (int)((i - which * n) / D), ch = (int)(i % D);
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const float *p) {
    const float4 y = *reinterpret_cast<const float4 *>(p);
    x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
  };
  if (key < tokens_of(a, b)) {
#pragma unroll 4
    for (int s = 0; s < a.n_part; ++s) add(a.sums + ((int64_t)u * a.n_part + s) * 2 * n + i);
    if (key < a.S)
#pragma unroll 4
      for (int s = 0; s + 1 < a.parts; ++s) add(a.part + ((((int64_t)u * a.parts + s) * 2 + which) * a.sink_rows + key) * D + ch);
  }
  char *row = which ? a.dv + b * a.v_b + (int64_t)key * a.v_t + (int64_t)hkv * a.v_h
                    : a.dk + b * a.k_b + (int64_t)key * a.k_t + (int64_t)hkv * a.k_h;
  store4<T>(row + ch * (int)sizeof(T), 0, 0, 0, x[0], x[1], x[2], x[3]);
}

// dk and dv of the sinks: the sums of their shares, four of them for every value, and these added.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_sinks_kernel(WinArgs a) {
  __shared__ float sums[4][64];
  const int u = blockIdx.x / (2 * a.S * D / 64), b = u / a.Hkv, hkv = u % a.Hkv, quarter = threadIdx.x / 64;
  const int i = blockIdx.x % (2 * a.S * D / 64) * 64 + threadIdx.x % 64;   // (2 S D is a multiple of 64)
  const int which = i / (a.S * D), key = i / D % a.S, ch = i % D;
  const float *p = a.part + (((int64_t)u * a.parts * 2 + which) * a.sink_rows + key) * D + ch;
  float sum = 0.f;
#pragma unroll 4
  for (int s = quarter; s < a.parts; s += 4) sum += p[(int64_t)s * 2 * a.sink_rows * D];
  sums[quarter][threadIdx.x % 64] = sum;
  __syncthreads();
  if (quarter != 0 || key >= a.Tk) return;
  sum = key < tokens_of(a, b) ? (sum + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]) : 0.f;
  char *dst = which ? a.dv + b * a.v_b + (int64_t)key * a.v_t + (int64_t)hkv * a.v_h
                    : a.dk + b * a.k_b + (int64_t)key * a.k_t + (int64_t)hkv * a.k_h;
  Io<T>::store((T *)dst + ch, sum);
}

// ------------------------------------------------------------------------------------------------
// The ring cache: sinks in rows 0 .. S - 1, position p >= S in row S + (p - S) % W.
struct CacheArgs {
  char *ck, *cv;   // [B, Hkv, S + W, D]
  const char *q, *k, *v;
  char *out;
  int64_t k_b, k_t, k_h, v_b, v_t, v_h;   // bytes (fill)
  const int32_t *at;                       // fill: lens or null; token: positions
  float *part;                             // [B * Hq, n_split, D + 2]
  float scale;
  int64_t W;
  int32_t B, Hq, Hkv, T, S, n_split, split_rows;
};

__global__ __launch_bounds__(256) void window_fill_kernel(CacheArgs a, int row_b) {
  const int64_t rows = a.S + a.W;
  const int parts = row_b / 16;
  const uint32_t wgs = (uint32_t)((rows * parts + 255) / 256);   // of a unit
  const int64_t i = (int64_t)(blockIdx.x % wgs) * 256 + threadIdx.x;
  if (i >= rows * parts) return;
  const int u = blockIdx.x / wgs, b = u / a.Hkv, h = u % a.Hkv, part = (int)(i % parts);
  const int64_t r = i / parts;
  int64_t n = a.T;
  if (a.at) n = a.at[b] < a.T ? a.at[b] : a.T;
  int64_t p = r;
  if (r >= a.S && n > a.S) p = r + (n - 1 - r >= 0 ? (n - 1 - r) / a.W * a.W : 0);   // the last position of the row's
  if (p >= n) return;   // nothing for this row: left as it is
  const int64_t to = ((int64_t)u * rows + r) * row_b + 16 * part;
  *reinterpret_cast<uint4 *>(a.ck + to) = *reinterpret_cast<const uint4 *>(a.k + b * a.k_b + p * a.k_t + h * a.k_h + 16 * part);
  *reinterpret_cast<uint4 *>(a.cv + to) = *reinterpret_cast<const uint4 *>(a.v + b * a.v_b + p * a.v_t + h * a.v_h + 16 * part);
}

// 16 bytes that nothing reads again before the next token: not kept in the caches (64 sequences, 4100 rows each: 198 us without, 177 with).
__device__ __forceinline__ uint4 load_once(const char *p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)));
}

// One token per sequence.  A workgroup has a range of the cache rows of one unit and up to kHeads of its query heads; lanes of a
// row hold 16 bytes of it each, a wave 1 KiB of consecutive rows at a time.  Every group of lanes keeps a softmax of its
// own rows; they are joined at the end, those of the ranges by window_join_kernel.
constexpr int kHeads = 4;
template <typename T, int D>
__global__ __launch_bounds__(256) void window_token_kernel(CacheArgs a) {
  constexpr int kVec = Vec16<T>::kN, kLanes = D / kVec, kRowsWave = 64 / kLanes, kRowsWg = 4 * kRowsWave;
  constexpr int kUnroll = 2;
  __shared__ float part[4][kHeads][D + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int G = a.Hq / a.Hkv, batches = (G + kHeads - 1) / kHeads;
  const int split = blockIdx.x % a.n_split, bu = blockIdx.x / a.n_split;
  const int u = bu / batches, g0 = bu % batches * kHeads, b = u / a.Hkv;
  const int ng = G - g0 < kHeads ? G - g0 : kHeads;
  const uint32_t rows = (uint32_t)a.S + (uint32_t)a.W;
  const int c = lane % kLanes, sub = wave * kRowsWave + lane / kLanes;
  const int64_t head0 = (int64_t)u * G + g0;   // of [B, Hq]
  float *po = a.n_split > 1 ? a.part + (head0 * a.n_split + split) * (D + 2) : nullptr;
  const uint32_t r0 = (uint32_t)split * (uint32_t)a.split_rows;
  const uint32_t r_end = r0 + (uint32_t)a.split_rows < rows ? r0 + (uint32_t)a.split_rows : rows;
  const char *ck = a.ck + (int64_t)u * rows * (D * sizeof(T)), *cv = a.cv + (int64_t)u * rows * (D * sizeof(T));
  // The rows of a step are asked for a step ahead, the first ones before the position is known: what of them holds no token, or
  // the token before this one, is not looked at.
  uint4 kx[2][kUnroll], vx[2][kUnroll];
  auto load = [&](uint32_t r, uint4 (&kd)[kUnroll], uint4 (&vd)[kUnroll]) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      uint32_t ri = r + i * kRowsWg;
      ri = ri < r_end ? ri : r_end - 1;
      kd[i] = load_once(ck + (uint64_t)ri * (D * sizeof(T)) + 16 * c);
      vd[i] = load_once(cv + (uint64_t)ri * (D * sizeof(T)) + 16 * c);
    }
  };
  load(r0 + (uint32_t)sub, kx[0], vx[0]);
  const uint4 fresh_k = reinterpret_cast<const uint4 *>(a.k + (int64_t)u * D * sizeof(T))[c];
  const uint4 fresh_v = reinterpret_cast<const uint4 *>(a.v + (int64_t)u * D * sizeof(T))[c];
  float q[kHeads][kVec], o[kHeads][kVec], m[kHeads], l[kHeads];
  const float sc = a.scale * kLog2e;
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    Vec16<T>::load((const T *)a.q + (head0 + (h < ng ? h : 0)) * D + c * kVec, q[h]);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      q[h][e] *= sc;
      o[h][e] = 0.f;
    }
    m[h] = -INFINITY;
    l[h] = 0.f;
  }
  const int pos = a.at[b];
  if (pos < 0) {   // no token for this sequence
    if (split == 0)
      for (int i = tid; i < ng * D; i += 256) Io<T>::store((T *)a.out + head0 * D + i, 0.f);
    return;
  }
  const uint32_t fresh = pos < a.S ? (uint32_t)pos : (uint32_t)a.S + (uint32_t)(pos - a.S) % (uint32_t)a.W;   // the token's own row
  const uint32_t r1 = r_end <= (uint32_t)pos ? r_end : (uint32_t)pos + 1;   // rows that hold a token
  if (g0 == 0 && fresh >= r0 && fresh < r1 && tid < kLanes) {
    reinterpret_cast<uint4 *>(a.ck + ((int64_t)u * rows + fresh) * (D * sizeof(T)))[tid] = fresh_k;
    reinterpret_cast<uint4 *>(a.cv + ((int64_t)u * rows + fresh) * (D * sizeof(T)))[tid] = fresh_v;
  }
  auto step = [&](uint32_t r, const uint4 (&kd)[kUnroll], const uint4 (&vd)[kUnroll]) {
    float s[kHeads][kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      float x[kVec];
      unpack16<T>(r + i * kRowsWg == fresh ? fresh_k : kd[i], x);
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) dot = fmaf(q[h][e], x[e], dot);
        dot = group_sum<kLanes>(dot);
        s[h][i] = r + i * kRowsWg < r1 ? dot : -INFINITY;
      }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      float top = m[h];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) top = fmaxf(top, s[h][i]);
      const float ref = top == -INFINITY ? 0.f : top;
      const float alpha = __builtin_amdgcn_exp2f(m[h] - ref);
      m[h] = top;
      l[h] *= alpha;
#pragma unroll
      for (int e = 0; e < kVec; ++e) o[h][e] *= alpha;
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        s[h][i] = __builtin_amdgcn_exp2f(s[h][i] - ref);
        l[h] += s[h][i];
      }
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      if (r + i * kRowsWg < r1) {
        float x[kVec];
        unpack16<T>(r + i * kRowsWg == fresh ? fresh_v : vd[i], x);
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
#pragma unroll
          for (int e = 0; e < kVec; ++e) o[h][e] = fmaf(s[h][i], x[e], o[h][e]);
      }
    }
  };
  constexpr uint32_t kStep = kRowsWg * kUnroll;
  for (uint32_t r = r0 + (uint32_t)sub; r < r1; r += 2 * kStep) {
    if (r + kStep < r1) load(r + kStep, kx[1], vx[1]);
    step(r, kx[0], vx[0]);
    if (r + kStep >= r1) break;
    if (r + 2 * kStep < r1) load(r + 2 * kStep, kx[0], vx[0]);
    step(r + kStep, kx[1], vx[1]);
  }
  // join the lane groups of a wave, then the waves
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const float top = strided_max<kLanes>(m[h]);
    const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[h] - top);
    l[h] = strided_sum<kLanes>(l[h] * f);
#pragma unroll
    for (int e = 0; e < kVec; ++e) o[h][e] = strided_sum<kLanes>(o[h][e] * f);
    if (lane < kLanes) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) part[wave][h][c * kVec + e] = o[h][e];
      if (lane == 0) {
        part[wave][h][D] = top;
        part[wave][h][D + 1] = l[h];
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < ng * D; i += 256) {
    const int h = i / D, ch = i % D;
    float top = part[0][h][D];
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, part[w][h][D]);
    float sum = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = part[w][h][D] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(part[w][h][D] - top);
      sum = fmaf(f, part[w][h][D + 1], sum);
      x = fmaf(f, part[w][h][ch], x);
    }
    if (po) {
      float *p = po + (int64_t)h * a.n_split * (D + 2);
      p[ch] = x;
      if (ch == 0) {
        p[D] = top;
        p[D + 1] = sum;
      }
    } else {
      Io<T>::store((T *)a.out + (head0 + h) * D + ch, sum == 0.f ? 0.f : x / sum);
    }
  }
}

// The ranges of a query head joined: a lane has a range's maximum and sum, a thread a channel of every kParts-th range.  A range without
// a token has factor, sum and channels of 0; one whose sum or channel is not a number makes the result that, whatever its factor.
constexpr int kMostSplits = 64;
template <typename T, int D>
__global__ __launch_bounds__(256) void window_join_kernel(CacheArgs a) {
  constexpr int kParts = 256 / D;
  __shared__ float factor[kMostSplits], acc[kParts][D];
  const int head = blockIdx.x, lane = threadIdx.x & 63;
  if (a.at[head / a.Hq] < 0) return;
  const float *p = a.part + (int64_t)head * a.n_split * (D + 2);
  const int ch = threadIdx.x % D, part = threadIdx.x / D;
  const float *own = p + (lane < a.n_split ? lane : 0) * (D + 2) + D;
  const float m = lane < a.n_split ? own[0] : -INFINITY, l = own[1];
  const float top = wave_max(m), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
  const float sum = wave_sum(lane < a.n_split ? f * l : 0.f);
  if (threadIdx.x < 64) factor[lane] = f;
  __syncthreads();
  float x = 0.f;
#pragma unroll 16
  for (int s = part; s < a.n_split; s += kParts) x = fmaf(factor[s], p[s * (D + 2) + ch], x);
  acc[part][ch] = x;
  __syncthreads();
  if (part != 0) return;
#pragma unroll
  for (int k = 1; k < kParts; ++k) x += acc[k][ch];
  Io<T>::store((T *)a.out + (int64_t)head * D + ch, sum == 0.f ? 0.f : x / sum);
}

// ---- host side

constexpr int64_t kMostWgs = 1ll << 24;   // workgroups of 256 threads: a launch has fewer than 2^32

bool valid(const kvm_window_config *c) {
  if (!c || c->batch <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->io_dtype != KVM_F32 && c->io_dtype != KVM_BF16) return false;
  if (!(c->scale >= 0.f) || isinf(c->scale)) return false;
  if (c->window < 1 || c->window >= (1ll << 30) || c->n_sink < 0 || c->n_sink > kMaxSink) return false;
  return (int64_t)c->batch * c->n_q_heads < (1 << 24);
}
float scale_of(const kvm_window_config *c) { return c->scale > 0.f ? c->scale : 1.f / sqrtf((float)c->head_dim); }
bool lengths_ok(int64_t Tq, int64_t Tk) { return Tq > 0 && Tk >= Tq && Tk < (1ll << 30); }
bool al16(const void *p) { return ((uintptr_t)p & 15) == 0; }

bool strides_ok(int64_t b, int64_t t, int64_t h, const kvm_window_config *c) {
  const int vec = c->io_dtype == KVM_BF16 ? 8 : 4;
  if (b < 0 || t < c->head_dim || h < c->head_dim) return false;
  if (b % vec || t % vec || h % vec) return false;
  return t <= (1 << 23);
}

// Position tiles of `span` queries, of four heads of a group together (by_head) or of one.
void tile_queries(WinArgs &a, bool by_head, int span) {
  a.by_head = by_head;
  a.span = span;
  a.tiles = (a.Tq + a.span - 1) / a.span;
  // blocks of position tiles: 2048 positions, fewer where there would not be eight blocks for every XCD; of equal sizes, and no larger
  // than there are tiles, since a block's workgroups are launched whether there are tiles for them or not (512 prompts of one token, 32
  // heads on 8: 30 us, 313 with blocks of 2048 positions)
  int64_t per = 2048 / a.span;
  const int64_t units = (int64_t)a.B * a.Hkv;
  while (per > 1 && units * ((a.tiles + per - 1) / per) < 8 * kXcds) per /= 2;
  a.blocks = (int32_t)((a.tiles + per - 1) / per);
  a.per_block = (a.tiles + a.blocks - 1) / a.blocks;
}
WinArgs base_args(const kvm_window_config *c, int64_t Tq, int64_t Tk, const int32_t *lens) {
  WinArgs a = {};
  a.lens = lens;
  a.scale = scale_of(c);
  a.B = c->batch; a.Hq = c->n_q_heads; a.Hkv = c->n_kv_heads;
  a.Tq = (int32_t)Tq; a.Tk = (int32_t)Tk;
  a.W = (int32_t)(c->window < Tk ? c->window : Tk);
  a.S = a.W >= Tk ? 0 : (int32_t)(c->n_sink < Tk ? c->n_sink : Tk);   // (nothing is beyond the window: no sinks needed)
  const bool by_head = a.Hq / a.Hkv % kWaves == 0;
  tile_queries(a, by_head, by_head ? 32 : 32 * kWaves);
  return a;
}
// Workgroups of the query kernels, all blocks full and a multiple of eight of them; 0: more than a grid holds.
unsigned query_grid(const WinArgs &a) {
  const int64_t G = a.Hq / a.Hkv, groups = ((int64_t)a.B * a.Hkv * a.blocks + kXcds - 1) / kXcds * kXcds;
  const int64_t n = groups * a.per_block * (a.by_head ? G / kWaves : G);
  return n < kMostWgs ? (unsigned)n : 0;
}
// The queries beyond a sink's window: ranges of one tile of each head for every wave at least, as many as fill the device (two
// workgroups to a compute unit) and 64 at most.
void cut_far(WinArgs &a) {
  a.key_tiles = (a.Tk + 127) / 128;
  // Few key tiles: the queries of each are shared among as many workgroups as give the device two to a compute unit, four tiles at
  // least to each.  (3 sequences of 777 tokens, 2 KV heads, fp32: 150 us
  // with 42 workgroups, 44 in 8 parts and 6 for their sum.)
  const int64_t units = (int64_t)a.B * a.Hkv, wgs = units * a.key_tiles;
  const int64_t stream = (int64_t)((a.W + 127 < a.Tk ? a.W + 127 : a.Tk) + 31) / 32 * (a.Hq / a.Hkv);
  a.n_part = 1;
  if (wgs < 256) a.n_part = (int32_t)(512 / wgs < stream / 4 ? 512 / wgs : stream / 4);
  if (a.n_part < 1) a.n_part = 1;
  a.sink_rows = 32;
  if (a.S == 0) return;
  a.sink_rows = a.S <= 32 ? 32 : a.S <= 64 ? 64 : 128;
  const int step = kWaves / (a.sink_rows / 32), far = a.Tk - a.W;
  const int64_t most = units < 8 ? 64 : units < 512 ? 512 / units : 1;
  a.split_q = (int32_t)((far + most - 1) / most + 32 * step - 1) / (32 * step) * (32 * step);
  a.n_split = (far + a.split_q - 1) / a.split_q;
  a.parts = a.n_split * step + 1;
}
size_t delta_bytes(const WinArgs &a) { return ((size_t)a.B * a.Hq * a.Tq * sizeof(float) + 255) & ~(size_t)255; }
size_t part_bytes(const WinArgs &a, int d) {
  return (size_t)a.B * a.Hkv * a.parts * 2 * a.sink_rows * d * sizeof(float);
}
size_t sums_bytes(const WinArgs &a, int d) {
  return a.n_part > 1 ? (size_t)a.B * a.Hkv * a.n_part * 2 * a.Tk * d * sizeof(float) : 0;
}

// Few workgroups for the device: 32 queries of one head in each instead, its waves sharing the key tiles.  Prompts, us, tiles shared / not
// (workgroups not shared): 512 tokens, 8 heads 9 / 20 (32); 1000, 8 on 2 heads 13 / 33 (64); fp32, 777, 6 on 2 heads 12 / 35 (42);
// 2048, 16 heads 55 / 66 (256); 1000, 32 on 8 heads, four to a workgroup, 28 / 26 (256); 4096, 16 on 4 heads 73 / 50 (512).
// Of 64 units (sequence, KV head) and more, a grid as small has short rows: there only where the smaller workgroups run at once, two to a
// compute unit, and had no tiles of a group's heads to share.  Shared / not (workgroups if shared): 64 x 128 tokens, one head, 6.8 /
// 9.6 (256); 64 x 256, 10.1 / 13.5 (512); 100 x 160, 13.0 / 10.7 (520); 64 x 500, fp32, 76 / 67 (1024); 200 x 32 tokens, four heads on
// one, 13.9 / 8.0 (800); 64 x 32, 6.6 / 7.2 (256).
bool split_tiles(WinArgs &a) {
  const unsigned grid = query_grid(a);
  if (grid == 0 || grid >= (a.by_head ? 256u : 512u)) return false;
  WinArgs b = a;
  tile_queries(b, false, 32);
  if ((int64_t)a.B * a.Hkv >= 64 && (a.by_head || query_grid(b) > 512)) return false;
  a = b;
  return true;
}
// Prompts of a training step (lse is asked for) whose rows have few keys: the errors of dq and dk against a single rounding's are 1.43 to
// 1.49 with P as one operand there (up to 1.56 for 16 tokens), 1.42 to 1.45 as two (1.49).  Beyond, the difference goes, and the second operand
// costs: us, two / one, 64 x 256 tokens, 16 heads, 77 / 67; 4 x 4k, 16 heads of 64 on 4, window 128, 39 / 34; 2 x 256, 8 heads, 8.0 / 7.6.
bool fine_rows(const WinArgs &a) { return a.lse && (a.Tk <= 256 || a.W + a.S <= 64); }

template <typename T, int D, bool kFine>
hipError_t run_prefill_as(const WinArgs &a, unsigned grid, bool split, hipStream_t st) {
  static OncePerDevice<hipError_t> once, once_split;
  if (split) {
    const hipError_t e = allow_lds(once_split, (const void *)window_prefill_split_kernel<T, D, kFine>, split_lds<T, D>());
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_prefill_split_kernel<T, D, kFine>), dim3(grid), dim3(256), (split_lds<T, D>()), st, a);
    return hipGetLastError();
  }
  constexpr size_t bytes = 4 * (size_t)kTileRows * D * sizeof(T);
  hipError_t e = allow_lds(once, (const void *)window_prefill_kernel<T, D, kFine>, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((window_prefill_kernel<T, D, kFine>), dim3(grid), dim3(256), bytes, st, a);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t run_prefill(const WinArgs &a, unsigned grid, bool split, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (fine_rows(a)) return run_prefill_as<T, D, true>(a, grid, split, st);
  }
  return run_prefill_as<T, D, false>(a, grid, split, st);
}
template <typename T, int D>
hipError_t run_backward_as(const WinArgs &a, unsigned grid, bool split, unsigned units8, hipStream_t st) {
  static OncePerDevice<hipError_t> once_q, once_split, once_kv;
  constexpr size_t bytes = 4 * (size_t)kTileRows * D * sizeof(T), bytes_kv = kv_lds<T, D>();
  hipError_t e = split ? allow_lds(once_split, (const void *)window_dq_split_kernel<T, D>, split_lds<T, D>())
                       : allow_lds(once_q, (const void *)window_dq_kernel<T, D>, bytes);
  if (e == hipSuccess) e = allow_lds(once_kv, (const void *)window_dkv_kernel<T, D>, bytes_kv);
  if (e != hipSuccess) return e;
  if (split) hipLaunchKernelGGL((window_dq_split_kernel<T, D>), dim3(grid), dim3(256), (split_lds<T, D>()), st, a);
  else hipLaunchKernelGGL((window_dq_kernel<T, D>), dim3(grid), dim3(256), bytes, st, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((window_dkv_kernel<T, D>), dim3(a.far_wgs + units8 * a.key_tiles * a.n_part), dim3(256), bytes_kv, st, a);
  e = hipGetLastError();
  if (e != hipSuccess || (a.n_split == 0 && a.n_part == 1)) return e;
  if (a.n_part > 1) {
    const unsigned wgs = (unsigned)((2 * (int64_t)a.Tk * D / 4 + 255) / 256);
    hipLaunchKernelGGL((window_sum_kernel<T, D>), dim3(wgs, (unsigned)(a.B * a.Hkv)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((window_sinks_kernel<T, D>), dim3((unsigned)(2 * a.S * D / 64) * (a.B * a.Hkv)), dim3(256), 0, st, a);
  return hipGetLastError();
}

// Ranges a unit's cache rows are cut into: workgroups enough to fill the device, 256 rows at least in each.  (64 sequences, 8 KV heads,
// 4100 rows: 199 us with 1024 workgroups, 177 with 1536, 182 with 2048; one sequence: 17 us with 128 or 256 rows at least, 21 with 512.)
constexpr int64_t kTokenWgs = 1536;
void cut_rows(CacheArgs &a, const kvm_window_config *c) {
  const int64_t rows = c->n_sink + c->window, G = c->n_q_heads / c->n_kv_heads;
  const int64_t wgs = (int64_t)c->batch * c->n_kv_heads * ((G + kHeads - 1) / kHeads);
  int64_t n = (kTokenWgs + wgs - 1) / wgs, most = (rows + 256 - 1) / 256;
  if (n > most) n = most;
  if (n > kMostSplits) n = kMostSplits;
  const int64_t per = ((rows + n - 1) / n + 15) / 16 * 16;
  a.split_rows = (int32_t)per;
  a.n_split = (int32_t)((rows + per - 1) / per);
}
template <typename T, int D>
hipError_t run_token(const CacheArgs &a, unsigned grid, hipStream_t st) {
  hipLaunchKernelGGL((window_token_kernel<T, D>), dim3(grid), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL((window_join_kernel<T, D>), dim3((unsigned)(a.B * a.Hq)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace kvm

#define KVM_BY_TYPE(cfg, fn, ...)                                                                    \
  ((cfg)->io_dtype == KVM_BF16 ? ((cfg)->head_dim == 128 ? fn<bf16_t, 128>(__VA_ARGS__) : fn<bf16_t, 64>(__VA_ARGS__)) \
                               : ((cfg)->head_dim == 128 ? fn<float, 128>(__VA_ARGS__) : fn<float, 64>(__VA_ARGS__)))

extern "C" int kvm_window_prefill(const kvm_window_config *cfg, const void *q, const void *k, const void *v,
                                  const int32_t *lens, void *out, void *out_rest, float *lse, int64_t Tq, int64_t Tk,
                                  const kvm_strides *strides, void *stream) {
  using namespace kvm;
  if (!valid(cfg) || !lengths_ok(Tq, Tk) || !q || !k || !v || !out) return KVM_ERR_ARG;
  if (!al16(q) || !al16(k) || !al16(v) || !al16(out) || !al16(out_rest)) return KVM_ERR_ARG;
  const int64_t d = cfg->head_dim, hq = cfg->n_q_heads, hk = cfg->n_kv_heads, es = cfg->io_dtype == KVM_BF16 ? 2 : 4;
  kvm_strides s;
  if (strides) s = *strides;
  else {
    s.q_b = s.o_b = Tq * hq * d; s.q_t = s.o_t = hq * d; s.q_h = s.o_h = d;
    s.k_b = s.v_b = Tk * hk * d; s.k_t = s.v_t = hk * d; s.k_h = s.v_h = d;
    s.lse_b = Tq * hq; s.lse_t = hq; s.lse_h = 1;
  }
  if (!strides_ok(s.q_b, s.q_t, s.q_h, cfg) || !strides_ok(s.k_b, s.k_t, s.k_h, cfg) || !strides_ok(s.v_b, s.v_t, s.v_h, cfg) ||
      !strides_ok(s.o_b, s.o_t, s.o_h, cfg) || !rows_apart({cfg->batch, Tq, hq}, {s.o_b, s.o_t, s.o_h}, d))
    return KVM_ERR_ARG;
  if (lse && (s.lse_b < 0 || s.lse_t < 1 || s.lse_h < 1 || !rows_apart({cfg->batch, Tq, hq}, {s.lse_b, s.lse_t, s.lse_h}, 1)))
    return KVM_ERR_ARG;
  WinArgs a = base_args(cfg, Tq, Tk, lens);
  a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v; a.out = (char *)out; a.lse = lse;
  a.rest = es == 2 ? (char *)out_rest : nullptr;
  a.q_b = s.q_b * es; a.q_t = s.q_t * es; a.q_h = s.q_h * es;
  a.k_b = s.k_b * es; a.k_t = s.k_t * es; a.k_h = s.k_h * es;
  a.v_b = s.v_b * es; a.v_t = s.v_t * es; a.v_h = s.v_h * es;
  a.o_b = s.o_b * es; a.o_t = s.o_t * es; a.o_h = s.o_h * es;
  a.l_b = s.lse_b; a.l_t = s.lse_t; a.l_h = s.lse_h;
  const bool split = split_tiles(a);
  const unsigned grid = query_grid(a);
  if (grid == 0) return KVM_ERR_ARG;
  const hipError_t e = KVM_BY_TYPE(cfg, run_prefill, a, grid, split, (hipStream_t)stream);
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_window_prefill");
}

extern "C" size_t kvm_window_backward_workspace_bytes(const kvm_window_config *cfg, int64_t Tq, int64_t Tk) {
  using namespace kvm;
  if (!valid(cfg) || !lengths_ok(Tq, Tk)) return 0;
  WinArgs a = base_args(cfg, Tq, Tk, nullptr);
  cut_far(a);
  return delta_bytes(a) + part_bytes(a, cfg->head_dim) + sums_bytes(a, cfg->head_dim);
}

extern "C" int kvm_window_backward(const kvm_window_config *cfg, const void *q, const void *k, const void *v, const int32_t *lens,
                                   const void *out, const void *out_rest, const float *lse, const void *dout, void *dq,
                                   void *dk, void *dv, int64_t Tq, int64_t Tk, void *workspace, size_t workspace_bytes,
                                   void *stream) {
  using namespace kvm;
  if (!valid(cfg) || !lengths_ok(Tq, Tk)) return KVM_ERR_ARG;
  const void *ptrs[] = {q, k, v, out, dout, dq, dk, dv, workspace};
  for (const void *p : ptrs)
    if (!p || !al16(p)) return KVM_ERR_ARG;
  if (!lse || !al16(out_rest)) return KVM_ERR_ARG;
  const int64_t d = cfg->head_dim, hq = cfg->n_q_heads, hk = cfg->n_kv_heads, es = cfg->io_dtype == KVM_BF16 ? 2 : 4;
  if (hq * d > (1 << 23)) return KVM_ERR_ARG;
  if (workspace_bytes < kvm_window_backward_workspace_bytes(cfg, Tq, Tk)) return KVM_ERR_CAPACITY;
  WinArgs a = base_args(cfg, Tq, Tk, lens);
  cut_far(a);
  a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v; a.out = (char *)const_cast<void *>(out);
  a.rest = es == 2 ? (char *)const_cast<void *>(out_rest) : nullptr;
  a.lse = const_cast<float *>(lse);
  a.dout = (const char *)dout; a.dq = (char *)dq; a.dk = (char *)dk; a.dv = (char *)dv;
  a.q_b = a.o_b = Tq * hq * d * es; a.q_t = a.o_t = hq * d * es; a.q_h = a.o_h = d * es;
  a.k_b = a.v_b = Tk * hk * d * es; a.k_t = a.v_t = hk * d * es; a.k_h = a.v_h = d * es;
  a.l_b = Tq * hq; a.l_t = hq; a.l_h = 1;
  a.delta = (float *)workspace;
  a.part = (float *)((char *)workspace + delta_bytes(a));
  a.sums = (float *)((char *)a.part + part_bytes(a, (int)d));
  const bool split = split_tiles(a);
  const unsigned grid = query_grid(a);
  const int64_t units8 = ((int64_t)a.B * a.Hkv + kXcds - 1) / kXcds * kXcds;
  a.far_wgs = (int32_t)(units8 * a.n_split);
  if (grid == 0 || units8 * (a.key_tiles + a.n_split) >= kMostWgs || (int64_t)a.B * a.Hkv * 2 * a.S * d / 64 >= kMostWgs) return KVM_ERR_ARG;
  const hipError_t e = KVM_BY_TYPE(cfg, run_backward_as, a, grid, split, (unsigned)units8, (hipStream_t)stream);
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_window_backward");
}

extern "C" int kvm_window_fill(const kvm_window_config *cfg, void *cache_k, void *cache_v, const void *k, const void *v,
                               const int32_t *lens, int64_t T, const kvm_strides *strides, void *stream) {
  using namespace kvm;
  if (!valid(cfg) || !lengths_ok(T, T) || !cache_k || !cache_v || !k || !v) return KVM_ERR_ARG;
  if (!al16(cache_k) || !al16(cache_v) || !al16(k) || !al16(v)) return KVM_ERR_ARG;
  const int64_t d = cfg->head_dim, hk = cfg->n_kv_heads, es = cfg->io_dtype == KVM_BF16 ? 2 : 4;
  kvm_strides s;
  if (strides) s = *strides;
  else {
    s.k_b = s.v_b = T * hk * d; s.k_t = s.v_t = hk * d; s.k_h = s.v_h = d;
  }
  if (!strides_ok(s.k_b, s.k_t, s.k_h, cfg) || !strides_ok(s.v_b, s.v_t, s.v_h, cfg)) return KVM_ERR_ARG;
  const int64_t units = (int64_t)cfg->batch * hk, parts = d * es / 16;
  CacheArgs a = {};
  a.ck = (char *)cache_k; a.cv = (char *)cache_v; a.k = (const char *)k; a.v = (const char *)v;
  a.k_b = s.k_b * es; a.k_t = s.k_t * es; a.k_h = s.k_h * es;
  a.v_b = s.v_b * es; a.v_t = s.v_t * es; a.v_h = s.v_h * es;
  a.at = lens; a.W = cfg->window; a.S = cfg->n_sink; a.T = (int32_t)T; a.B = cfg->batch; a.Hkv = (int32_t)hk;
  const int64_t wgs = ((a.S + a.W) * parts + 255) / 256;
  if (wgs * units >= kMostWgs) return KVM_ERR_ARG;
  hipLaunchKernelGGL(window_fill_kernel, dim3((unsigned)(wgs * units)), dim3(256), 0, (hipStream_t)stream, a, (int)(d * es));
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_window_fill");
}

extern "C" size_t kvm_window_decode_workspace_bytes(const kvm_window_config *cfg) {
  using namespace kvm;
  if (!valid(cfg)) return 0;
  CacheArgs a = {};
  cut_rows(a, cfg);
  return a.n_split > 1 ? (size_t)cfg->batch * cfg->n_q_heads * a.n_split * (cfg->head_dim + 2) * sizeof(float) : 256;
}

extern "C" int kvm_window_decode(const kvm_window_config *cfg, void *cache_k, void *cache_v, const void *q, const void *k,
                                 const void *v, const int32_t *pos, void *out, void *workspace, size_t workspace_bytes,
                                 void *stream) {
  using namespace kvm;
  if (!valid(cfg)) return KVM_ERR_ARG;
  const void *ptrs[] = {cache_k, cache_v, q, k, v, out, workspace};
  for (const void *p : ptrs)
    if (!p || !al16(p)) return KVM_ERR_ARG;
  if (!pos) return KVM_ERR_ARG;
  if (workspace_bytes < kvm_window_decode_workspace_bytes(cfg)) return KVM_ERR_CAPACITY;
  CacheArgs a = {};
  a.ck = (char *)cache_k; a.cv = (char *)cache_v; a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v;
  a.out = (char *)out; a.at = pos; a.part = (float *)workspace; a.scale = scale_of(cfg);
  a.W = cfg->window; a.S = cfg->n_sink; a.B = cfg->batch; a.Hq = cfg->n_q_heads; a.Hkv = cfg->n_kv_heads;
  cut_rows(a, cfg);
  const int64_t G = a.Hq / a.Hkv, grid = (int64_t)a.B * a.Hkv * ((G + kHeads - 1) / kHeads) * a.n_split;
  if (grid >= kMostWgs) return KVM_ERR_ARG;
  const hipError_t e = KVM_BY_TYPE(cfg, run_token, a, (unsigned)grid, (hipStream_t)stream);
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_window_decode");
}
