// Linear attention with a constant decay for each KV head.
//
//   S_t = e^a S_{t-1} + k_t v_t^T,   o_t = scale q_t S_t                       (a <= 0, S fp32 [d, d])
// A chunk of C tokens with start state S, token i of the chunk:
//   o_i = scale (sum_{s <= i} e^{a (i - s)} (q_i . k_s) v_s + e^{a (i + 1)} q_i S)
//   S'  = e^{a C} S + sum_i e^{a (C - 1 - i)} k_i v_i^T
// Gradients are the same walk in other roles, x the rows asked with, y and z the two factors of the state:
//   forward  x q   y k   z v    -> out        dq   x dout  y v     z k  (state transposed)
//   backwards in time, state R = sum over later tokens of e^{a (t - c0 + 1)} q_t dout_t^T (+ the end state's gradient):
//   dv       x k   y q   z dout               dk   x v     y dout  z q  (state transposed)
// where x is decayed by e^{a i} and y, z by e^{a (C - i)}, i counted from the chunk's later end (the exponents are one off
// against the forward walk: kShift).  In the backward walks y and z have the heads of the group, which add up.
//
// A workgroup walks one segment of one unit (sequence, KV head); a wave owns 32 channels of z, with S[:, those] in its
// registers.  S is an operand of x S as it lies there (seq_tiles.h), so it never passes through LDS.
// Few units: the sequence is cut into segments.  A first pass computes what each adds to the state (y and z alone are
// read), a second adds those up, and the walk starts every segment from its state.
//
// What it reaches (bf16, 128 channels): rows are read and written once in the walk, and y and z once more in the first pass.  8 sequences
// of 32k tokens, 32 heads on 8: 1.45 ms for 6.44 GB, 4.4 TB/s (a copy of one GiB: 5.1); matrix instructions take 29 % of the walk's
// cycles.  Gradients and prompt of 4 x 8k tokens, 16 heads: 637 us for 2.4 GB.  Neither memory nor the matrix units are full
// there: a workgroup has one chain of dependent steps for each chunk (pairs, their product, the state).  Single token, 128 sequences of 32 heads:
// states at 5.2 TB/s, read and written, where a copy takes 5.1.
#include <math.h>

#include <type_traits>

#include "../../include/kvm.h"
#include "kvm_internal.h"
#include "seq_tiles.h"

namespace kvm {

namespace {

struct LinArgs {
  const char *x, *y, *z;
  char *out;
  const char *x2;        // a pair's second walk: its x and out (strides of the first's)
  char *out2;
  int64_t x_b, x_t, x_h, y_b, y_t, y_h, z_b, z_t, z_h, o_b, o_t, o_h;   // bytes
  const float *log_decay;
  const int32_t *lens;   // nullable
  const float *start;    // nullable: the state before the first token walked
  float *seg;            // [units, seg_of_unit, D, D]: start states of segments (what each adds to the state, after the first pass);
                         // a walk's segment is seg_step of them
  float *end;            // nullable: the state behind the last token walked
  float start_scale, end_scale, scale;
  int32_t transposed;    // start and seg are [z channel][y channel]
  int32_t fine_state;    // the state is a result
  int32_t T, H, G, units, n_seg, seg_tokens, seg_of_unit, seg_step;
  int32_t head_parts;    // workgroups that share the heads of x, each with the state of its own
};

template <typename T>
constexpr int kChunk = sizeof(T) == 2 ? 64 : 32;   // tokens of a chunk: a tile of either type is C * D * sizeof = 16 KiB at D = 128

// Blocks of 32 x 32 pairs of a chunk, row block tb and column block sb <= tb: 0: (0, 0), 1: (1, 0), 2: (1, 1).
template <typename T>
constexpr int kBlocks = kChunk<T> == 64 ? 3 : 1;

// Two y tiles, z, x; pairs of a chunk as operands (bf16); the powers of the decay.
template <typename T, int D, bool kPair, bool kFine>
constexpr size_t linear_lds() {
  return (kPair ? 8 : 4) * (size_t)kChunk<T> * D * sizeof(T) +
         (sizeof(T) == 2 ? (kPair ? 2 : 1) * kBlocks<T> * (kFine ? 4096 : 2048) : 0) + (32 + 2 * kChunk<T>) * sizeof(float);
}

// kRev: from the last token to the first; kMany: y and z have the heads of the group (otherwise x has); kOut: rows are
// written, otherwise the state alone is advanced.
// kPair: two walks of one workgroup, half of its waves each, over the same two streams of tiles: y of the one is z of the other, the
// other's state the transpose.  dk and dv read q and dout once that way (4 x 8k tokens, 16 heads: 375 us apart, 260 together).
// Roundings in bf16 (sums and states are fp32 throughout): the state enters x S, and the decayed pairs of a chunk the product
// with z, as one operand each, which leaves an output twice the variance of its own rounding; kFine: as two, with
// errors of 2^-16, for prompts so short that an output rests on a few pairs.  The decayed z enters the state as three
// operands, all 24 bits, where the state is a result, as two elsewhere (a.fine_state).
template <typename T, int D, bool kRev, bool kMany, bool kOut, bool kPair, bool kFine>
__global__ __launch_bounds__(kPair ? 4 * D : 2 * D, 2) void linear_walk_kernel(LinArgs a) {
  using Tl = Tile<T, D>;
  constexpr int NW = D / 32, C = kChunk<T>, TB = C / 32, KS = D / 16, NB = D / 32, SK = C / 16;
  constexpr uint32_t kTileB = C * Tl::kRowB;
  constexpr int kShift = kRev ? 0 : 1;
  constexpr int kPlanes = Tl::kBf16 && kFine ? 2 : 1, kPlanesZ = Tl::kBf16 ? 3 : 1;
  constexpr bool kShare = Tl::kBf16;   // each pair block by one wave, passed on through LDS (fp32 has one block: every wave makes it)
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  constexpr int kWaves = kPair ? 2 * NW : NW;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool second = kPair && wave_all >= NW;          // of the pair's walks
  const int wave = second ? wave_all - NW : wave_all;
  // tiles: y twice, z, x (a pair, whose workgroup has its compute unit to itself: all of them twice)
  const uint32_t at0 = lds_addr_of(lds), at_y = second ? at0 + 2 * kTileB : at0;
  const uint32_t at_z = second ? at0 : at0 + 2 * kTileB, at_x = at0 + (kPair ? (second ? 6 : 4) : 3) * kTileB;
  char *pairs = lds + (kPair ? 8 : 4) * kTileB + (second ? kBlocks<T> * kPlanes * 2048 : 0);
  float *rel = reinterpret_cast<float *>(lds + (kPair ? 8 : 4) * kTileB + (kShare ? (kPair ? 2 : 1) * kBlocks<T> * kPlanes * 2048 : 0));   // [32 + n]: scale e^{a n}, n = -32 .. C - 1
  float *wt = rel + 32 + C;   // [i]: the decay of a chunk's token i in the state behind it
  const int g = lane >> 5, l32 = lane & 31;
  const bool transposed = kPair ? second : a.transposed != 0;
  // the lane's z channel of its wave's 32: such that results, which have z channels as rows, are in natural order
  const int zl = 16 * (l32 >> 4) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
  const int u = blockIdx.x % a.units, seg_part = blockIdx.x / a.units;
  const int seg = kMany ? seg_part : seg_part / a.head_parts, part = kMany ? 0 : seg_part % a.head_parts;
  const int b = u / a.H, h = u % a.H;
  int n = a.T;
  if (a.lens) {
    n = a.lens[b];
    n = n < 0 ? 0 : n < a.T ? n : a.T;
  }
  n = __builtin_amdgcn_readfirstlane(n);
  const int s0 = seg * a.seg_tokens;
  const int s1 = s0 + a.seg_tokens < n ? s0 + a.seg_tokens : n;   // positions s0 .. s1 - 1 of the walk
  const int heads_x = kMany ? 1 : a.G / a.head_parts, heads_y = kMany ? a.G : 1;
  const int head0 = kMany ? h : h * a.G + part * heads_x;   // first head of x
  const int steps = kMany ? heads_y : kOut ? heads_x : 1;   // of a chunk
  if constexpr (kOut) {   // rows behind the sequence
    const int z0 = s0 > n ? s0 : n, z1 = s0 + a.seg_tokens < a.T ? s0 + a.seg_tokens : a.T;
    constexpr int kParts = Tl::kRowB / 16;
    for (int t = z0 + (64 * wave + lane) / kParts; t < z1; t += 64 * NW / kParts)
      for (int hx = 0; hx < heads_x; ++hx)
        *reinterpret_cast<uint4 *>((second ? a.out2 : a.out) + b * a.o_b + (int64_t)t * a.o_t + (int64_t)(head0 + hx) * a.o_h +
                                   16 * (lane % kParts)) = make_uint4(0, 0, 0, 0);
  }
  const bool ends = kOut && a.end && !second && part == 0 && (n > 0 ? s0 < n && n <= s0 + a.seg_tokens : seg == 0);
  if (s0 >= n && !(ends && n == 0)) return;   // (an empty sequence's state is passed on)
  if (!kOut && s1 - s0 < a.seg_tokens) return;   // (a segment that another one follows is full)

  // ---- powers of the decay
  const float a_h = a.log_decay[h], al = a_h < -1e4f ? -1e4f : a_h;   // (-infinity too: its powers are 0, and 1 for no step at all)
  for (int i = tid; i < 32 + C; i += 64 * kWaves) rel[i] = i < 32 ? 0.f : a.scale * expf(al * (float)(i - 32));
  if (tid < C) wt[tid] = expf(al * (float)(C - kShift - tid));
  float dec[TB];
#pragma unroll
  for (int tb = 0; tb < TB; ++tb) dec[tb] = expf(al * (float)(32 * tb + l32 + kShift)) * a.scale;
  // e^{a C} as a float, and what that leaves.  Hundreds of chunks multiply a slowly decaying state by it, and the rounding of a
  // single float would be the same one every time: the rest is carried from chunk to chunk.
  const double lam = exp((double)al * C);
  const float lam_hi = (float)lam, lam_lo = (float)(lam - (double)lam_hi);
  float carry = 0.f;

  // ---- the state: element v of block blk is (y channel 32 blk + 16 (v / 8) + 8 g + v % 8, z channel 32 wave + zl)
  f32x16 S[NB];
  {
    // (of a sequence that is cut, the first segment's too is in seg: `start` may be `end`, which another workgroup writes)
    const bool cut = a.seg_of_unit > 1 && n > 0;
    const float *src = cut ? a.seg + ((int64_t)u * a.seg_of_unit + seg * a.seg_step) * (D * D)
                           : a.start ? a.start + (int64_t)u * (D * D) : nullptr;
    const float f = cut ? 1.f : a.start_scale;
    if (!kOut) src = nullptr;
    const int zc = 32 * wave + zl;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int yc = 32 * blk + 16 * (v >> 3) + 8 * g + (v & 7);
        S[blk][v] = src ? f * src[transposed ? zc * D + yc : yc * D + zc] : 0.f;
      }
  }

  const char *xb = uniform_ptr((second ? a.x2 : a.x) + b * a.x_b + (int64_t)head0 * a.x_h);
  const char *yb = uniform_ptr(a.y + b * a.y_b + (int64_t)(h * heads_y) * a.y_h);
  const char *zb = uniform_ptr(a.z + b * a.z_b + (int64_t)(h * heads_y) * a.z_h);
  char *ob = (second ? a.out2 : a.out) + b * a.o_b + (int64_t)head0 * a.o_h;
  // first row in memory of the chunk at position c0 with nv tokens
  auto first_row = [&](int c0, int nv) { return kRev ? n - c0 - nv : c0; };
  auto load_yz = [&](int c0, int hd, uint32_t buf) {
    const int nv = s1 - c0 < C ? s1 - c0 : C;
    const int64_t r = first_row(c0, nv);
    const int ln = (int)here((uint32_t)lane);
    Tl::template fill<C, kWaves, kRev>(yb + r * a.y_t + hd * a.y_h, (uint32_t)a.y_t, nv, at0 + buf * kTileB, wave_all, ln);
    Tl::template fill<C, kWaves, kRev>(zb + r * a.z_t + hd * a.z_h, (uint32_t)a.z_t, nv, at0 + (2 + (kPair ? buf : 0)) * kTileB, wave_all, ln);
  };
  auto load_x = [&](int c0, int hd, [[maybe_unused]] uint32_t buf) {
    const int nv = s1 - c0 < C ? s1 - c0 : C;
    Tl::template fill<C, NW, kRev>(xb + (int64_t)first_row(c0, nv) * a.x_t + hd * a.x_h, (uint32_t)a.x_t, nv, at_x + (kPair ? buf * kTileB : 0),
                                   wave, (int)here((uint32_t)lane));
  };

  Operand<T> xf[kPair ? 1 : TB][kPair ? 1 : KS], zf[SK];
  f32x16 o[TB];
  uint32_t buf = 0, xbuf = 0;
  bool stored = false;   // full rows have been stored behind the latest loads
  const uint32_t lane_along = Tl::along0(lane), lane_across = Tl::template across0<false>(lane);
  // the decayed pairs of block (tb, sb) as operands of the second product: z^T . pairs
  auto pairs_of = [&](auto tb_, auto sb_, uint32_t y_along, [[maybe_unused]] uint32_t x_along, Operand<T> (&pw)[2][kPlanes]) {
    constexpr int tb = decltype(tb_)::value, sb = decltype(sb_)::value;
    f32x16 sc = {0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (kPair) sc = mma(Tl::along(y_along, sb, ks), Tl::along(x_along, tb, ks), sc);
      else sc = mma(Tl::along(y_along, sb, ks), xf[tb][ks], sc);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int v = 8 * hf + e, gap = 32 * (tb - sb) + l32 - mfma_row(v, g);
        const float r = sc[v] * rel[32 + gap];
        w[e] = tb > sb || gap >= 0 ? r : 0.f;
      }
      split_operand<kPlanes>(w, pw[hf]);
    }
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, TB - 1>;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (s0 < s1) {
    load_yz(s0, 0, 0);
    if constexpr (kOut) load_x(s0, 0, 0);
  }
  for (int c0 = s0; c0 < s1; c0 += C) {
    const int nv = s1 - c0 < C ? s1 - c0 : C;
    for (int hd = 0; hd < steps; ++hd) {
      const bool new_x = kMany ? hd == 0 : true, new_yz = kMany ? true : hd == 0;
      const bool last = hd == steps - 1;
      const uint32_t y_along = here(at_y + buf * kTileB + lane_along), y_across = here(at_y + buf * kTileB + lane_across);
      // this step's tiles: asked for ahead of the stores of the step before, which need not have ended (a lane stores
      // kStores times for a full chunk)
      constexpr int kStores = TB * 32 * (int)sizeof(T) / 32;
      if (stored) wait_vmem<kStores>();
      else wait_vmem<0>();
      publish();
      stored = false;
      auto load_next = [&]() {
        const int nc0 = last ? c0 + C : c0, nhd = last ? 0 : hd + 1;
        if (nc0 < s1) {
          if (kMany || nhd == 0) load_yz(nc0, nhd, buf ^ 1);
          if (kOut && (!kMany || nhd == 0)) load_x(nc0, nhd, xbuf ^ 1);
        }
      };
      if constexpr (kPair) load_next();
      const uint32_t x_along = here(at_x + (kPair ? xbuf * kTileB : 0) + lane_along);
      if constexpr (kOut && !kPair) {
        if (new_x) {
#pragma unroll
          for (int tb = 0; tb < TB; ++tb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) xf[tb][ks] = Tl::along(x_along, tb, ks);
        }
      }
      // o = x S, decayed
      auto ask_state = [&]() {
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) o[tb] = f32x16{0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          float s[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] = S[ks >> 1][8 * (ks & 1) + e];
          Operand<T> pl[kPlanes], x[TB];
          split_operand<kPlanes>(s, pl);
#pragma unroll
          for (int tb = 0; tb < TB; ++tb) {
            if constexpr (kPair) x[tb] = Tl::along(x_along, tb, ks);
            else x[tb] = xf[tb][ks];
          }
#pragma unroll
          for (int i = 0; i < kPlanes; ++i)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) o[tb] = mma(pl[i], x[tb], o[tb]);
        }
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[tb][v] *= dec[tb];
      };
      if constexpr (kPair) {
        if (new_x) ask_state();
      }
      if (new_yz) {
        const uint32_t z = here((at_z + (kPair ? buf * kTileB : 0) + lane_across) ^ (uint32_t)(32 * wave * (int)sizeof(T)));
#pragma unroll
        for (int ks = 0; ks < SK; ++ks) zf[ks] = Tl::across(z, 0, ks);
      }
      if (nv < C && hd == 0 && tid < C) wt[tid] = tid < nv ? expf(al * (float)(nv - kShift - tid)) : 0.f;   // (decay to the end)
      if constexpr (kOut && kShare) {
        auto pass_on = [&](int i, auto tb, auto sb) {
          Operand<T> pw[2][kPlanes];
          pairs_of(tb, sb, y_along, x_along, pw);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl)
              *reinterpret_cast<Operand<T> *>(pairs + ((2 * i + hf) * kPlanes + pl) * 1024 + 16 * lane) = pw[hf][pl];
        };
        if (wave == 1) pass_on(0, I0{}, I0{});
        if (wave == 0) pass_on(1, I1{}, I0{});
        if (wave == (NW > 2 ? 2 : 1)) pass_on(2, I1{}, I1{});
      }
      publish();   // the step's pairs are in LDS, and where there is one tile of them, x and z in registers
      if constexpr (!kPair) load_next();
      if constexpr (kOut) {
        if constexpr (!kPair) {
          if (new_x) ask_state();
        }
        // the chunk's own tokens
        if constexpr (kShare) {
#pragma unroll
          for (int i = 0; i < kBlocks<T>; ++i)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
              for (int pl = 0; pl < kPlanes; ++pl)
                o[i > 0] = mma(zf[(i == 2 ? 2 : 0) + hf], *reinterpret_cast<const Operand<T> *>(pairs + ((2 * i + hf) * kPlanes + pl) * 1024 + 16 * lane), o[i > 0]);
        } else {
          Operand<T> pw[2][kPlanes];
          pairs_of(I0{}, I0{}, y_along, x_along, pw);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) o[0] = mma(zf[hf], pw[hf][0], o[0]);
        }
        if (kMany ? last : true) {
          constexpr int es = (int)sizeof(T);
          stored = nv == C;
#pragma unroll
          for (int tb = 0; tb < TB; ++tb) {
            const int i = 32 * tb + l32;
            if (i < nv) {
              const int64_t row = kRev ? n - 1 - (c0 + i) : c0 + i;
              char *dst = ob + row * a.o_t + (kMany ? 0 : hd * a.o_h) + (32 * wave + 8 * g) * es;
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const f32x16 &x = o[tb];
                const int v = 8 * hf;
                if constexpr (Tl::kBf16) {
                  *reinterpret_cast<uint4 *>(dst + 16 * hf * es) = make_uint4(pack_bf16(x[v], x[v + 1]), pack_bf16(x[v + 2], x[v + 3]),
                                                                              pack_bf16(x[v + 4], x[v + 5]), pack_bf16(x[v + 6], x[v + 7]));
                } else {
                  *reinterpret_cast<float4 *>(dst + 16 * hf * es) = make_float4(x[v], x[v + 1], x[v + 2], x[v + 3]);
                  *reinterpret_cast<float4 *>(dst + 16 * hf * es + 16) = make_float4(x[v + 4], x[v + 5], x[v + 6], x[v + 7]);
                }
              }
            }
          }
        }
      }
      if (kMany || last) {   // the state behind the chunk
        if (kMany ? hd == 0 : true) {
          carry += lam_lo;
          float f = lam_hi + carry;
          carry -= f - lam_hi;
          if (nv < C) f = (float)exp((double)al * nv);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk)
#pragma unroll
            for (int v = 0; v < 16; ++v) S[blk][v] *= f;
        }
#pragma unroll
        for (int ks = 0; ks < SK; ++ks) {
          __builtin_amdgcn_sched_barrier(0);
          float zs[8];
          from_operand(zf[ks], zs);
          const float4 w0 = *reinterpret_cast<const float4 *>(wt + 16 * ks + 4 * g);
          const float4 w1 = *reinterpret_cast<const float4 *>(wt + 16 * ks + 8 + 4 * g);
          const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) zs[e] *= w[e];
          Operand<T> pl[kPlanesZ], yt[NB];
          split_operand<kPlanesZ>(zs, pl);
#pragma unroll
          for (int blk = 0; blk < NB; ++blk) {
            yt[blk] = Tl::across(y_across, blk, ks);
            S[blk] = mma(yt[blk], pl[0], S[blk]);
            if constexpr (kPlanesZ > 1) S[blk] = mma(yt[blk], pl[1], S[blk]);
          }
          if constexpr (kPlanesZ > 2) {
            if (a.fine_state) {
#pragma unroll
              for (int blk = 0; blk < NB; ++blk) S[blk] = mma(yt[blk], pl[2], S[blk]);
            }
          }
        }
      }
      if (kMany || last) buf ^= 1;
      if (last) xbuf ^= 1;
    }
  }
  float *dst = nullptr;
  float f = 1.f;
  if constexpr (kOut) {
    if (ends) {
      dst = a.end + (int64_t)u * (D * D);
      f = a.end_scale;
    }
  } else {
    dst = a.seg + ((int64_t)u * a.seg_of_unit + seg) * (D * D);
  }
  if (dst) {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        dst[(32 * blk + 16 * (v >> 3) + 8 * g + (v & 7)) * D + 32 * wave + zl] = f * S[blk][v];
  }
}

// What each segment adds to the state becomes the state it starts from (fp32; as many steps as there are segments).
__global__ __launch_bounds__(256) void linear_segments_kernel(LinArgs a, int dd) {
  const int u = blockIdx.y, i = 4 * (blockIdx.x * 256 + threadIdx.x);
  if (i >= dd) return;
  int n = a.T;
  if (a.lens) n = a.lens[u / a.H] < a.T ? a.lens[u / a.H] : a.T;
  // (the factor as a float and what that leaves: the rounding of one, the same for up to 1024 segments, would add up to 3e-5 of the
  // state's oldest part where it decays by 1e-5 a token)
  const double factor = exp((double)a.log_decay[u % a.H] * a.seg_tokens);
  const float lam = (float)factor, rest = (float)(factor - (double)lam);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.start) {
    s = *reinterpret_cast<const float4 *>(a.start + (int64_t)u * dd + i);
    s.x *= a.start_scale; s.y *= a.start_scale; s.z *= a.start_scale; s.w *= a.start_scale;
  }
  // segments that another one follows are full; sixteen of them are asked for at a time
  const int n_full = n > 0 ? (n - 1) / a.seg_tokens : -1;
  float *at = a.seg + (int64_t)u * a.seg_of_unit * dd + i;
  constexpr int kAhead = 16;
  for (int seg0 = 0; seg0 <= n_full; seg0 += kAhead) {
    float4 add[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (seg0 + k < n_full) add[k] = *reinterpret_cast<const float4 *>(at + (int64_t)(seg0 + k) * dd);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (seg0 + k <= n_full) *reinterpret_cast<float4 *>(at + (int64_t)(seg0 + k) * dd) = s;
      if (seg0 + k < n_full) {
        s.x = fmaf(s.x, lam, fmaf(s.x, rest, add[k].x));
        s.y = fmaf(s.y, lam, fmaf(s.y, rest, add[k].y));
        s.z = fmaf(s.z, lam, fmaf(s.z, rest, add[k].z));
        s.w = fmaf(s.w, lam, fmaf(s.w, rest, add[k].w));
      }
    }
  }
}

// One token per sequence: the state is read, advanced, written and asked, once.  A workgroup has kCols value channels of one
// unit; a thread has four of them and D / (256 / (kCols / 4)) key channels.
struct LinTokenArgs {
  float *state;
  const char *q, *k, *v;
  char *out;
  const float *log_decay;
  const int32_t *active;   // nullable
  float scale;
  int32_t H, G;
};
constexpr int kTokenHeads = 8;   // query heads whose partial sums are in LDS together
template <typename T, int D, int kCols>
__global__ __launch_bounds__(256) void linear_token_kernel(LinTokenArgs a) {
  constexpr int kLanes = kCols / 4, kGroups = 256 / kLanes, kRows = D / kGroups, kParts = D / kCols;
  __shared__ float qs[kTokenHeads * D], part[kTokenHeads][4][kCols];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int u = blockIdx.x / kParts, col0 = (blockIdx.x % kParts) * kCols;
  const int b = u / a.H, h = u % a.H, G = a.G;
  const int c = col0 + 4 * (tid % kLanes), r0 = (tid / kLanes) * kRows;
  const T *k = (const T *)a.k + (int64_t)u * D, *v = (const T *)a.v + (int64_t)u * D;
  const T *q = (const T *)a.q + (int64_t)u * G * D;
  T *out = (T *)a.out + (int64_t)u * G * D;
  if (a.active && a.active[b] == 0) {
    for (int i = tid; i < G * kCols; i += 256) Io<T>::store(out + (i / kCols) * D + col0 + i % kCols, 0.f);
    return;
  }
  float *st = a.state + (int64_t)u * (D * D) + (int64_t)r0 * D + c;
  float4 s[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) s[r] = *reinterpret_cast<const float4 *>(st + r * D);
  // (the decay as a float and what that leaves: the rounding of one, the same in every call, would be 3e-8 of a slowly decaying state a
  // token, 7e-5 of it after 2000)
  const double decay = exp((double)a.log_decay[h]);
  const float lam = (float)decay, rest = lam == INFINITY ? 0.f : (float)(decay - (double)lam);
  float vv[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) vv[e] = Io<T>::load(v + c + e);
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const float kr = Io<T>::load(k + r0 + r);
    s[r].x = fmaf(s[r].x, lam, fmaf(s[r].x, rest, kr * vv[0]));
    s[r].y = fmaf(s[r].y, lam, fmaf(s[r].y, rest, kr * vv[1]));
    s[r].z = fmaf(s[r].z, lam, fmaf(s[r].z, rest, kr * vv[2]));
    s[r].w = fmaf(s[r].w, lam, fmaf(s[r].w, rest, kr * vv[3]));
    *reinterpret_cast<float4 *>(st + r * D) = s[r];
  }
  for (int g0 = 0; g0 < G; g0 += kTokenHeads) {
    const int ng = G - g0 < kTokenHeads ? G - g0 : kTokenHeads;
    __syncthreads();
    for (int i = tid; i < ng * D; i += 256) qs[i] = Io<T>::load(q + g0 * D + i);
    __syncthreads();
    for (int hd = 0; hd < ng; ++hd) {
      float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float x = qs[hd * D + r0 + r];
        o[0] = fmaf(x, s[r].x, o[0]);
        o[1] = fmaf(x, s[r].y, o[1]);
        o[2] = fmaf(x, s[r].z, o[2]);
        o[3] = fmaf(x, s[r].w, o[3]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = strided_sum<kLanes>(o[e]);
      if (lane < kLanes)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[hd][wave][4 * lane + e] = o[e];
    }
    __syncthreads();
    for (int i = tid; i < ng * kCols; i += 256) {
      const int hd = i / kCols, x = i % kCols;
      const float o = (part[hd][0][x] + part[hd][1][x]) + (part[hd][2][x] + part[hd][3][x]);
      Io<T>::store(out + (g0 + hd) * D + col0 + x, o * a.scale);
    }
  }
}

// ---- host side

bool valid(const kvm_linear_config *c) {
  if (!c || c->batch <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->io_dtype != KVM_F32 && c->io_dtype != KVM_BF16) return false;
  if (!(c->scale >= 0.f) || isinf(c->scale)) return false;
  return (int64_t)c->batch * c->n_q_heads < (1 << 24);
}
float scale_of(const kvm_linear_config *c) { return c->scale > 0.f ? c->scale : 1.f / sqrtf((float)c->head_dim); }

constexpr int64_t kMaxTokens = 1ll << 29;   // the end of twice a segment is a 32-bit position

// Segments a sequence is cut into: one workgroup has one segment of one unit, and the device holds `fill` of them at once.  The
// first pass reads y and z once more, so there are no more than it takes to fill the device.  Up to 32 segments may be a chunk each,
// more have two chunks at least (every segment is one more state to add up), and short sequences are not cut: two more launches cost
// more than the chunks walked less.  Prompts of 8 heads of 128 channels (in brackets their gradients), us, by the chunks of a segment:
//             one         two         four        not cut
//   bf16  5   32 (57)     36 (57)     38 (63)     23 (45)
//         8   34 (60)     37 (71)     47 (86)     33 (68)
//        16   40 (70)     40 (75)     48 (101)    62 (129)
//        32   46 (84)     45 (87)     50 (106)    120 (251)
//        64   55 (105)    48 (92)     53 (111)    235 (496)
//   fp32  5   37 (81)     46 (105)    49 (123)    42 (110)
//         8   39 (85)     47 (119)    66 (182)    65 (172)
//        32   50 (107)    55 (136)    70 (203)    245 (665)
struct Cut {
  int n_seg, seg_tokens;
};
Cut cut_of(const kvm_linear_config *c, int64_t T) {
  const int chunk = c->io_dtype == KVM_BF16 ? kChunk<bf16_t> : kChunk<float>;
  const int64_t units = (int64_t)c->batch * c->n_kv_heads, chunks = (T + chunk - 1) / chunk;
  const int64_t fill = c->head_dim == 128 ? 512 : 1024;
  int64_t n = (fill + units - 1) / units;
  const int64_t most = chunks <= 32 ? chunks : chunks / 2 > 32 ? chunks / 2 : 32;
  if (n > most) n = most;
  if (n < 1 || chunks < (c->io_dtype == KVM_BF16 ? 8 : 5)) n = 1;
  const int64_t per = (chunks + n - 1) / n;
  return Cut{(int)((chunks + per - 1) / per), (int)(per * chunk)};
}
size_t state_bytes(const kvm_linear_config *c) {
  return (size_t)c->batch * c->n_kv_heads * c->head_dim * c->head_dim * sizeof(float);
}

template <typename T, int D, bool kRev, bool kMany, bool kOut, bool kPair, bool kFine>
hipError_t launch_walk_as(const LinArgs &a, int n_wg, hipStream_t st) {
  static OncePerDevice<hipError_t> once;
  constexpr size_t bytes = linear_lds<T, D, kPair, kFine>();
  hipError_t e = allow_lds(once, (const void *)linear_walk_kernel<T, D, kRev, kMany, kOut, kPair, kFine>, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((linear_walk_kernel<T, D, kRev, kMany, kOut, kPair, kFine>), dim3((unsigned)n_wg), dim3(kPair ? 4 * D : 2 * D), bytes, st, a);
  return hipGetLastError();
}
// Few workgroups for the device: the query heads of a group are shared among several, up to one each, that walk the same state
// (1000 tokens of 32 heads on 8: 43 us, 50 with the heads of a group in one workgroup).
int head_parts_of(const kvm_linear_config *c, int n_wg) {
  const int G = c->n_q_heads / c->n_kv_heads, most = (c->head_dim == 128 ? 512 : 1024) / n_wg;
  int parts = 1;
  for (int k = 2; k <= G && k <= most; ++k)
    if (G % k == 0) parts = k;
  return parts;
}
// Prompts of up to kFineTokens tokens are a few chunks long and wait for latencies: two more operands for each product cost
// them nothing that shows.  Longer ones have many pairs behind most outputs, and the roundings of these average out.
constexpr int kFineTokens = 128;
template <bool kRev, bool kMany, bool kOut, bool kPair>
hipError_t launch_walk(const kvm_linear_config *c, LinArgs a, int n_wg, hipStream_t st) {
  a.head_parts = kOut && !kMany ? head_parts_of(c, n_wg) : 1;
  if (a.n_seg == 1 && a.start && a.start == a.end) a.head_parts = 1;   // (one workgroup reads the state before it writes it)
  n_wg *= kMany ? 1 : a.head_parts;
  if (c->io_dtype == KVM_F32)
    return c->head_dim == 128 ? launch_walk_as<float, 128, kRev, kMany, kOut, kPair, false>(a, n_wg, st)
                              : launch_walk_as<float, 64, kRev, kMany, kOut, kPair, false>(a, n_wg, st);
  if constexpr (kOut) {
    if (a.T <= kFineTokens)
      return c->head_dim == 128 ? launch_walk_as<bf16_t, 128, kRev, kMany, kOut, kPair, true>(a, n_wg, st)
                                : launch_walk_as<bf16_t, 64, kRev, kMany, kOut, kPair, true>(a, n_wg, st);
  }
  return c->head_dim == 128 ? launch_walk_as<bf16_t, 128, kRev, kMany, kOut, kPair, false>(a, n_wg, st)
                            : launch_walk_as<bf16_t, 64, kRev, kMany, kOut, kPair, false>(a, n_wg, st);
}
hipError_t launch_segments(const kvm_linear_config *c, const LinArgs &a, hipStream_t st) {
  const int dd = c->head_dim * c->head_dim;
  hipLaunchKernelGGL(linear_segments_kernel, dim3((unsigned)((dd / 4 + 255) / 256), (unsigned)a.units), dim3(256), 0, st, a, dd);
  return hipGetLastError();
}

bool al16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Strides of one operand, in elements: multiples of 16 bytes, rows whole and apart, 32-bit tile offsets.
bool strides_ok(int64_t b, int64_t t, int64_t h, const kvm_linear_config *c) {
  const int vec = c->io_dtype == KVM_BF16 ? 8 : 4;
  if (b < 0 || t < c->head_dim || h < c->head_dim) return false;
  if (b % vec || t % vec || h % vec) return false;
  return t <= (1 << 23);
}

template <typename T, int D>
void launch_token_as(const LinTokenArgs &a, int units, hipStream_t st) {
  if (units < 512)
    hipLaunchKernelGGL((linear_token_kernel<T, D, 32>), dim3((unsigned)(units * (D / 32))), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((linear_token_kernel<T, D, D>), dim3((unsigned)units), dim3(256), 0, st, a);
}

}  // namespace
}  // namespace kvm

extern "C" size_t kvm_linear_workspace_bytes(const kvm_linear_config *cfg, int64_t T) {
  if (!kvm::valid(cfg) || T <= 0 || T >= kvm::kMaxTokens) return 0;
  const kvm::Cut cut = kvm::cut_of(cfg, T);
  return cut.n_seg > 1 ? cut.n_seg * kvm::state_bytes(cfg) : 256;
}

extern "C" int kvm_linear_prefill(const kvm_linear_config *cfg, const void *q, const void *k, const void *v,
                                  const float *log_decay, const float *state_in, const int32_t *lens, void *out,
                                  float *state_out, int64_t T, const kvm_strides *strides, void *workspace,
                                  size_t workspace_bytes, void *stream) {
  using namespace kvm;
  if (!valid(cfg) || T <= 0 || T >= kMaxTokens || !q || !k || !v || !log_decay || !out || !workspace) return KVM_ERR_ARG;
  if (!al16(q) || !al16(k) || !al16(v) || !al16(out) || !al16(state_in) || !al16(state_out) || !al16(workspace)) return KVM_ERR_ARG;
  if (workspace_bytes < kvm_linear_workspace_bytes(cfg, T)) return KVM_ERR_CAPACITY;
  const int64_t d = cfg->head_dim, hq = cfg->n_q_heads, hk = cfg->n_kv_heads, es = cfg->io_dtype == KVM_BF16 ? 2 : 4;
  kvm_strides s;
  if (strides) s = *strides;
  else {
    s.q_b = s.o_b = T * hq * d; s.q_t = s.o_t = hq * d; s.q_h = s.o_h = d;
    s.k_b = s.v_b = T * hk * d; s.k_t = s.v_t = hk * d; s.k_h = s.v_h = d;
  }
  if (!strides_ok(s.q_b, s.q_t, s.q_h, cfg) || !strides_ok(s.k_b, s.k_t, s.k_h, cfg) || !strides_ok(s.v_b, s.v_t, s.v_h, cfg) ||
      !strides_ok(s.o_b, s.o_t, s.o_h, cfg) || !rows_apart({cfg->batch, T, hq}, {s.o_b, s.o_t, s.o_h}, d))
    return KVM_ERR_ARG;
  const Cut cut = cut_of(cfg, T);
  LinArgs a = {};
  a.x = (const char *)q; a.y = (const char *)k; a.z = (const char *)v; a.out = (char *)out;
  a.x_b = s.q_b * es; a.x_t = s.q_t * es; a.x_h = s.q_h * es;
  a.y_b = s.k_b * es; a.y_t = s.k_t * es; a.y_h = s.k_h * es;
  a.z_b = s.v_b * es; a.z_t = s.v_t * es; a.z_h = s.v_h * es;
  a.o_b = s.o_b * es; a.o_t = s.o_t * es; a.o_h = s.o_h * es;
  a.log_decay = log_decay; a.lens = lens; a.start = state_in; a.seg = (float *)workspace; a.end = state_out; a.fine_state = state_out != nullptr;
  a.start_scale = a.end_scale = 1.f; a.scale = scale_of(cfg);
  a.T = (int32_t)T; a.H = (int32_t)hk; a.G = (int32_t)(hq / hk); a.units = cfg->batch * cfg->n_kv_heads;
  a.n_seg = a.seg_of_unit = cut.n_seg; a.seg_tokens = cut.seg_tokens; a.seg_step = 1;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (cut.n_seg > 1) {
    e = launch_walk<false, false, false, false>(cfg, a, a.units * (a.n_seg - 1), st);
    if (e == hipSuccess) e = launch_segments(cfg, a, st);
  }
  if (e == hipSuccess) e = launch_walk<false, false, true, false>(cfg, a, a.units * a.n_seg, st);
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_linear_prefill");
}

extern "C" int kvm_linear_backward(const kvm_linear_config *cfg, const void *q, const void *k, const void *v,
                                   const float *log_decay, const float *state_in, const int32_t *lens, const void *dout,
                                   const float *dstate_out, void *dq, void *dk, void *dv, float *dstate_in, int64_t T,
                                   const void *kept, void *workspace, size_t workspace_bytes, void *stream) {
  using namespace kvm;
  if (!valid(cfg) || T <= 0 || T >= kMaxTokens || !q || !k || !v || !log_decay || !dout || !dq || !dk || !dv || !workspace)
    return KVM_ERR_ARG;
  const void *ptrs[] = {q, k, v, state_in, dout, dstate_out, dq, dk, dv, dstate_in, kept, workspace};
  for (const void *x : ptrs)
    if (!al16(x)) return KVM_ERR_ARG;
  if (workspace_bytes < kvm_linear_workspace_bytes(cfg, T)) return KVM_ERR_CAPACITY;
  const int64_t d = cfg->head_dim, hq = cfg->n_q_heads, hk = cfg->n_kv_heads, es = cfg->io_dtype == KVM_BF16 ? 2 : 4;
  const Cut cut = cut_of(cfg, T);
  const float scale = scale_of(cfg);
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (hq * d > (1 << 23)) return KVM_ERR_ARG;
  if (cfg->batch * hk * 4 * d >= 1ll << 32) return KVM_ERR_ARG;   // more threads than a launch has
  LinArgs c = {};
  c.log_decay = log_decay; c.lens = lens; c.seg = (float *)workspace; c.scale = scale;
  c.T = (int32_t)T; c.H = (int32_t)hk; c.G = (int32_t)(hq / hk); c.units = cfg->batch * cfg->n_kv_heads;
  c.n_seg = c.seg_of_unit = cut.n_seg; c.seg_tokens = cut.seg_tokens; c.seg_step = 1;
  auto roles = [&](const void *x, bool xq, const void *y, bool yq, const void *z, bool zq, void *o) {
    LinArgs a = c;
    auto put = [&](bool is_q, int64_t &sb, int64_t &s_t, int64_t &sh) {
      const int64_t hh = is_q ? hq : hk;
      sb = T * hh * d * es; s_t = hh * d * es; sh = d * es;
    };
    a.x = (const char *)x; a.y = (const char *)y; a.z = (const char *)z; a.out = (char *)o;
    put(xq, a.x_b, a.x_t, a.x_h);
    put(yq, a.y_b, a.y_t, a.y_h);
    put(zq, a.z_b, a.z_t, a.z_h);
    put(xq, a.o_b, a.o_t, a.o_h);
    return a;
  };
  // dq: the forward walk's states, transposed
  LinArgs f = roles(q, true, k, false, v, false, dq);
  f.start = state_in; f.start_scale = f.end_scale = 1.f;
  if (cut.n_seg > 1 && !kept) {
    e = launch_walk<false, false, false, false>(cfg, f, f.units * (f.n_seg - 1), st);
    if (e == hipSuccess) e = launch_segments(cfg, f, st);
  }
  LinArgs a = roles(dout, true, v, false, k, false, dq);
  a.start = state_in; a.start_scale = 1.f; a.transposed = 1;
  if (kept) a.seg = (float *)const_cast<void *>(kept);   // (read alone)
  if (e == hipSuccess) e = launch_walk<false, false, true, false>(cfg, a, a.units * a.n_seg, st);
  // dv and dk: backwards; the state there is that of the products q dout, without the scale
  LinArgs r = roles(k, false, q, true, dout, true, dv);
  r.x2 = (const char *)v; r.out2 = (char *)dk;
  r.start = dstate_out; r.start_scale = 1.f / scale; r.end = dstate_in; r.end_scale = scale; r.fine_state = dstate_in != nullptr;
  if (cut.n_seg > 1) {
    if (e == hipSuccess) e = launch_walk<true, true, false, false>(cfg, r, r.units * (r.n_seg - 1), st);
    if (e == hipSuccess) e = launch_segments(cfg, r, st);
  }
  // (a pair of walks has twice the waves of one: half as many segments fill the device)
  r.n_seg = (r.n_seg + 1) / 2; r.seg_tokens *= 2; r.seg_step = 2;
  if (e == hipSuccess) e = launch_walk<true, true, true, true>(cfg, r, r.units * r.n_seg, st);
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_linear_backward");
}

extern "C" int kvm_linear_decode(const kvm_linear_config *cfg, float *state, const void *q, const void *k, const void *v,
                                 const float *log_decay, const int32_t *active, void *out, void *stream) {
  using namespace kvm;
  if (!valid(cfg) || !state || !q || !k || !v || !log_decay || !out) return KVM_ERR_ARG;
  if (!al16(state) || !al16(q) || !al16(k) || !al16(v) || !al16(out)) return KVM_ERR_ARG;
  LinTokenArgs a;
  a.state = state; a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v; a.out = (char *)out;
  a.log_decay = log_decay; a.active = active; a.scale = scale_of(cfg);
  a.H = cfg->n_kv_heads; a.G = cfg->n_q_heads / cfg->n_kv_heads;
  const int units = cfg->batch * cfg->n_kv_heads;
  hipStream_t st = (hipStream_t)stream;
  if (cfg->io_dtype == KVM_BF16) {
    if (cfg->head_dim == 128) launch_token_as<bf16_t, 128>(a, units, st);
    else launch_token_as<bf16_t, 64>(a, units, st);
  } else {
    if (cfg->head_dim == 128) launch_token_as<float, 128>(a, units, st);
    else launch_token_as<float, 64>(a, units, st);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KVM_OK : report_hip(e, "kvm_linear_decode");
}
