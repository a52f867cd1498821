// Tiles and operand fragments of the window and linear kernels, for bf16 and fp32 I/O and head_dim 64 and 128.
//
// Both types are written against one 32x32 matrix step over 16 k's: a lane holds eight k's of its half g = lane / 32,
// of row (A) or column (B) lane % 32.  bf16: one v_mfma_f32_32x32x16_bf16.  fp32: eight v_mfma_f32_32x32x2_f32, the
// e-th of which takes the e-th value of either half; nothing is rounded there.  Which k a slot stands for is free as
// long as A and B agree, so the result of one product (lane: column; element v: row 8 * (v / 4) + 4 * g + v % 4)
// is an operand of the next as it lies in registers:
//   "accumulator order": slots of step s are k = 16 s + 4 g + {0..3}, 16 s + 8 + 4 g + {0..3}  (elements 8 s .. 8 s + 7)
//   "natural order":     slots of step s are k = 16 s + 8 g + {0..7}
//
// A tile is rows of D channels in LDS, unpadded, its 16-byte chunks permuted: chunk q of row r sits in slot q ^ swz(r),
// which keeps reads along rows and across rows apart in the banks (as in kvm_mfma.h, whose direct loads fill it).
#pragma once

#include "kvm_device.h"
#include "kvm_mfma.h"

namespace kvm {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct Operand;   // eight k's of a lane
template <>
struct Operand<bf16_t> {
  Frag8 f;
};
template <>
struct Operand<float> {
  float f[8];
};

__device__ __forceinline__ f32x16 mma(const Operand<bf16_t> &a, const Operand<bf16_t> &b, f32x16 c) {
  return mfma32(a.f.v, b.f.v, c);
}
__device__ __forceinline__ f32x16 mma(const Operand<float> &a, const Operand<float> &b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.f[e], b.f[e], c, 0, 0, 0);
  return c;
}

// Eight floats as an operand: rounded to nearest (bf16) or as they are (fp32).
__device__ __forceinline__ void to_operand(const float (&x)[8], Operand<bf16_t> &o) {
#pragma unroll
  for (int e = 0; e < 4; ++e) o.f.w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
}
__device__ __forceinline__ void to_operand(const float (&x)[8], Operand<float> &o) {
#pragma unroll
  for (int e = 0; e < 8; ++e) o.f[e] = x[e];
}
__device__ __forceinline__ void from_operand(const Operand<bf16_t> &o, float (&x)[8]) { unpack16<bf16_t>(o.f.q, x); }
__device__ __forceinline__ void from_operand(const Operand<float> &o, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = o.f[e];
}
// Eight floats as the sum of N operands, the largest first, each the rounding of what the ones before it left: 8 bits of the
// significand each in bf16 (three hold all 24), one in fp32.
template <int N>
__device__ __forceinline__ void split_operand(float (&x)[8], Operand<bf16_t> (&o)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    to_operand(x, o[n]);
    if (n + 1 < N) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] -= __uint_as_float(o[n].f.w[e] << 16);
        x[2 * e + 1] -= __uint_as_float(o[n].f.w[e] & 0xffff0000u);
      }
    }
  }
}
template <int N>
__device__ __forceinline__ void split_operand(float (&x)[8], Operand<float> (&o)[N]) {
  static_assert(N == 1, "fp32 is one operand");
  to_operand(x, o[0]);
}

__device__ __forceinline__ const char *uniform_ptr(const void *p) {
  const uint64_t x = (uint64_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32));
  return (const char *)(((uint64_t)hi << 32) | (uint64_t)lo);
}

template <typename T, int D>
struct Tile {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kRowB = D * (int)sizeof(T);      // bytes of a row: 128, 256 or 512
  static constexpr int kPieceRows = 1024 / kRowB;       // rows that one direct load of a wave fills
  static_assert(kRowB == 128 || kRowB == 256 || kRowB == 512, "row size");

  __device__ static __forceinline__ uint32_t swz(uint32_t r) {
    return kRowB == 128 ? 4 * ((r >> 1) & 1) + ((r >> 2) & 3) : 4 * (r & 3) + ((r >> 2) & 3);
  }

  // Rows 0 .. kRows - 1 of the tile at LDS address `at`, by kNW waves.  base (wave-uniform): the first of nv >= 1 rows in
  // memory, `stride` bytes apart; kRev: tile row r is memory row nv - 1 - r.  Tile rows beyond the last repeat it.
  // (swz is linear in the bits of a row: a lane's chunk is its own of the first piece, exclusive or the piece's)
  template <int kRows, int kNW, bool kRev>
  __device__ static __forceinline__ void fill(const char *base, uint32_t stride, int nv, uint32_t at, int wave, int lane) {
    constexpr int kPer = kRows / kPieceRows / kNW;
    static_assert(kPer * kNW * kPieceRows == kRows, "waves share a tile evenly");
    const uint32_t rl = (uint32_t)(16 * lane) / kRowB, col = 16 * (((uint32_t)lane % (kRowB / 16)) ^ swz(rl));
    const uint32_t piece0 = (uint32_t)(wave * kPer);
    if (nv >= kRows) {
      const uint32_t row = (kRev ? kPieceRows - 1 - rl : rl) * stride;
      base += (kRev ? kRows - (piece0 + 1) * kPieceRows : piece0 * kPieceRows) * stride;
#pragma unroll
      for (int n = 0; n < kPer; ++n) {
        const uint32_t piece = piece0 + n;
        dma16(base, row + (col ^ (16 * swz(piece * kPieceRows))), at + piece * 1024u);
        base = kRev ? base - kPieceRows * stride : base + kPieceRows * stride;
      }
    } else {
#pragma unroll
      for (int n = 0; n < kPer; ++n) {
        const uint32_t piece = piece0 + n;
        const int r = (int)(piece * kPieceRows + rl);
        int m = kRev ? nv - 1 - r : r;
        m = m < 0 ? 0 : m < nv ? m : nv - 1;
        dma16(base, (uint32_t)m * stride + (col ^ (16 * swz(piece * kPieceRows))), at + piece * 1024u);
      }
    }
  }

  // Operand along a row: tile row 32 * blk + lane % 32, channels 16 * ks + 8 * g .. + 7 (natural order).  base: the tile's LDS
  // address + along0(lane).  Swizzles repeat every 16 rows and tiles start on 1-KiB borders, so what a step changes of the chunk
  // is an exclusive or on the address.
  __device__ static __forceinline__ uint32_t along0(int lane) {
    const uint32_t l = (uint32_t)lane & 31, g = (uint32_t)lane >> 5;
    return l * kRowB + 16 * ((kBf16 ? g : 2 * g) ^ swz(l));
  }
  __device__ static __forceinline__ Operand<T> along(uint32_t base, int blk, int ks) {
    Operand<T> o;
    if constexpr (kBf16) {
      o.f.q = __builtin_bit_cast(uint4, *(const __attribute__((address_space(3))) u32x4_t *)(uintptr_t)((base ^ (uint32_t)(32 * ks)) + (uint32_t)(32 * blk * kRowB)));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4_t x = *(const __attribute__((address_space(3))) u32x4_t *)(uintptr_t)((base ^ (uint32_t)(64 * ks + 16 * i)) + (uint32_t)(32 * blk * kRowB));
#pragma unroll
        for (int e = 0; e < 4; ++e) o.f[4 * i + e] = __uint_as_float(x[e]);
      }
    }
    return o;
  }

  // Operand across rows: one channel of block `blk` (32 channels), tile rows 16 * ks + {4 g + 0..3, 8 + 4 g + 0..3}
  // (accumulator order).  base: the tile's LDS address + across0.  kNatural: the lane's channel is lane % 32; otherwise the one with which a product's
  // accumulator, its rows being these channels, is in natural order: element v of it is channel 16 * (v / 8) + 8 * g + v % 8.
  template <bool kNatural>
  __device__ static __forceinline__ uint32_t across0(int lane) {
    const uint32_t g = (uint32_t)lane >> 5;
    if constexpr (kBf16) {   // the transposing read: lane 4 t + c of 16 addresses row t, piece c of 4 channels
      const uint32_t j = (uint32_t)lane & 15, t = j >> 2, c = j & 3, half = ((uint32_t)lane >> 4) & 1;
      const uint32_t q = 2 * half + (kNatural ? c >> 1 : c & 1), sub = 8 * (kNatural ? c & 1 : c >> 1);
      return (4 * g + t) * kRowB + 16 * (q ^ swz(4 * g + t)) + sub;
    } else {
      const uint32_t l = (uint32_t)lane & 31;
      const uint32_t ch = kNatural ? l : 16 * (l >> 4) + 8 * ((l >> 2) & 1) + 4 * ((l >> 3) & 1) + (l & 3);
      return 4 * g * kRowB + 16 * ((ch >> 2) ^ g) + 4 * (ch & 3);
    }
  }
  __device__ static __forceinline__ Operand<T> across(uint32_t base, int blk, int ks) {
    Operand<T> o;
    if constexpr (kBf16) {
#pragma unroll
      for (int hi = 0; hi < 2; ++hi) {
        const uint32_t p = (base ^ (uint32_t)(64 * blk + 32 * hi)) + (uint32_t)((16 * ks + 8 * hi) * kRowB);
        o.f.d[hi] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(uintptr_t)p));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t p = (base ^ (uint32_t)((128 * blk) ^ (16 * (4 * (e % 4) + 2 * (e / 4))))) + (uint32_t)((16 * ks + 8 * (e / 4) + e % 4) * kRowB);
        o.f[e] = *(const __attribute__((address_space(3))) float *)(uintptr_t)p;
      }
    }
    return o;
  }
};

// Waits of loops that fill tiles with direct loads while stores of earlier results are under way.  wait_vmem<N>: until N of the
// wave's vector memory operations are left (they end in order).  publish: a barrier that waits for LDS operations alone.
template <int N>
__device__ __forceinline__ void wait_vmem() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void publish() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// An address computed where it is used: kept out of registers between uses (loops short of registers).
__device__ __forceinline__ uint32_t here(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

}  // namespace kvm
