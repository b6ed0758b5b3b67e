// Main loop of a block tile for products whose operands are not bf16: 16-bit floats (fp16), and 8-bit codes with a scale for every 128 of the
// contraction.  A row of a k-tile is 128 bytes in both, so that the operand tiles, their LDS layout and the ring of stages are those of gemm_dma.h; only
// the matrix instruction and the bytes that a lane feeds to it differ.
#pragma once
#include "gemm_dma.h"

namespace {

typedef _Float16 f16;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// fp16: a slice of a k-tile is 16 deep, a lane holds the 8 elements at 8 (lane / 32) of it
struct MmaF16 {
  typedef f16x8 Frag;                // as it is read from LDS
  typedef f16x8 Op;                  // as it is multiplied
  static constexpr int KS = 4;       // slices of a k-tile
  template <class T>
  static __device__ __forceinline__ Frag frag(const bf16* __restrict__ s, int rbase, int ks, int lane) {
    union { bf16x8 b; f16x8 h; } u;
    u.b = T::frag(s, rbase, ks, lane);
    return u.h;
  }
  static constexpr bool SCALED = false;
  template <int>
  static __device__ __forceinline__ Op op(const Frag& f, int) { return f; }
  template <int>
  static __device__ __forceinline__ void mma(const Op& a, const Op& b, f32x16& c, int, int) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
// 8-bit codes at the 8-bit rate: a slice is 64 deep, a lane holds 32 codes of its row and the instruction multiplies them by 2^(byte SEL of the scale word -
// 127).  Which of the 64 it holds does not matter as long as both operands agree, since the whole k-tile has one scale: it takes the two 16-byte chunks
// that a lane takes in two slices of 16-bit elements.
// The instruction adds products in groups of 8 neighbours that it aligns to the largest of them and cuts 13 bits below its leading one (measured: 448 * 448 - 448 * 448 + 2
// is 0 within 8 neighbours and 2 otherwise), in 32 bits from there on: 1.4e-5 relative to a Gaussian product, up to 4e-5 with rows of different size.
// That is a hundredth of the rounding of a bf16 result, but not what a 32-bit one may lose: see MmaE4M3Wide.
struct MmaE4M3 {
  typedef i32x8 Frag;
  typedef i32x8 Op;
  static constexpr int KS = 2;
  template <class T>
  static __device__ __forceinline__ Frag frag(const bf16* __restrict__ s, int rbase, int ks, int lane) {
    union { bf16x8 b[2]; i32x8 v; } u;
    u.b[0] = T::frag(s, rbase, 2 * ks, lane);
    u.b[1] = T::frag(s, rbase, 2 * ks + 1, lane);
    return u.v;
  }
  static constexpr bool SCALED = true;      // sa, sb: words of four scales, of which byte SEL is meant
  template <int>
  static __device__ __forceinline__ Op op(const Frag& f, int) { return f; }
  template <int SEL>
  static __device__ __forceinline__ void mma(const Op& a, const Op& b, f32x16& c, int sa, int sb) {
    c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, SEL, sa, SEL, sb);
  }
};
// 8-bit codes for 32-bit results: a lane's 16 codes of a 32-deep slice become bf16 with their scale (both exact: 4 significant bits, 8 of exponent) and
// go through two bf16 instructions, whose sums are 32 bits throughout.  Half the rate of MmaE4M3.
struct MmaE4M3Wide {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  typedef i32x4 Frag;
  struct Op { bf16x8 v[2]; };
  static constexpr int KS = 4;
  template <class T>
  static __device__ __forceinline__ Frag frag(const bf16* __restrict__ s, int rbase, int ks, int lane) {
    union { bf16x8 b; i32x4 v; } u;
    u.b = T::frag(s, rbase, ks, lane);
    return u.v;
  }
  static constexpr bool SCALED = true;
  template <int SEL>
  static __device__ __forceinline__ Op op(const Frag& f, int s) {
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    union { bf16x2 p[8]; Op o; } u;
    const float x = __uint_as_float(((uint32_t)s >> (8 * SEL) & 0xffu) << 23);      // 2^(byte - 127)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u.p[2 * k] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[k], x, false);
      u.p[2 * k + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[k], x, true);
    }
    return u.o;
  }
  template <int>
  static __device__ __forceinline__ void mma(const Op& a, const Op& b, f32x16& c, int, int) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[0], b.v[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[1], b.v[1], c, 0, 0, 0);
  }
};

// all products of a slice
template <class MMA, int SEL, int TI, int TJ>
__device__ __forceinline__ void mma_slice(const typename MMA::Frag (&fa)[TI], const typename MMA::Frag (&fb)[TJ], f32x16 (&acc)[TI][TJ], const int (&sa)[TI],
                                          const int (&sb)[TJ]) {
  typename MMA::Op oa[TI], ob[TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i) oa[i] = MMA::template op<SEL>(fa[i], sa[i]);
#pragma unroll
  for (int j = 0; j < TJ; ++j) ob[j] = MMA::template op<SEL>(fb[j], sb[j]);
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) MMA::template mma<SEL>(oa[i], ob[j], acc[i][j], sa[i], sb[j]);
}

// The pipeline of ahead_step over `nk` k-tiles: fragments are read one slice ahead, the barrier sits before the last slice of a k-tile.
// next(dst): requests the next k-tile into the stage at dst; it is called S times more than there are k-tiles to be used, and what it requests beyond
// them has to be harmless (an offset behind the operand, where a load returns zeros).  scales(t): called for t = 0, 4, 8, ... when k-tiles t to t + 3 are about to be
// used and what was requested before k-tile t - 1 has landed; sa and sb are the scale words of the tile's rows for these four (unused by fp16).
template <class C, class MMA, class TA, class TB, class Next, class Scales>
__device__ __forceinline__ void mma_loop(int nk, unsigned char* lds_raw, f32x16 (&acc)[C::TI][C::TJ], int (&sa)[C::TI], int (&sb)[C::TJ], int wm, int wn,
                                         int lane, Next&& next, Scales&& scales) {
  constexpr int TI = C::TI, TJ = C::TJ, S = C::S, KS = MMA::KS, NM = TI * TJ, NL = TA::NI + TB::NI;
  constexpr int NF = TI + TJ, FPM = (NF + NM - 1) / NM, RPS = sizeof(typename MMA::Frag) / 16;      // LDS reads per k-major fragment
  constexpr int UN = MMA::SCALED ? 4 : S;
  static_assert(KS % 2 == 0, "fragment sets alternate");
  static_assert(UN % S == 0, "the ring comes round with the scale words");
  typename MMA::Frag fa[2][TI], fb[2][TJ];
  // Where a lane's first chunk of a slice is (k-major, as in DmaTile::frag): chunk c of the row is at this XOR 32 times the slice.  The compiler would keep an
  // address for every slice and stage, which the 256 x 256 tile of 8-bit codes has no registers for (27 spilled, 8192^3 930 us instead of 435): LEAN, it sees
  // one, and makes the others.  Where they fit, keeping them is better (128 x 128 tiles 512 us, lean 533).
  constexpr bool LEAN = RPS == 2 && NM >= 8;
  static_assert(!LEAN || TB::RPF == 1, "both operands k-major");
  const int at = (lane & 31) * 128 + (((lane >> 5) ^ ((lane >> 1) & 7)) << 4);
  int atA = at + wm * TI * 4096, atB = at + wn * TJ * 4096 + TA::BYTES;
  auto lean = [&](typename MMA::Frag& f, const unsigned char* p, int a, int ks) __attribute__((always_inline)) {
    union { uint4 c[RPS]; typename MMA::Frag f; } u;
#pragma unroll
    for (int c = 0; c < RPS; ++c) u.c[c] = *(const uint4*)(p + (a ^ ((ks * RPS + c) << 5)));
    f = u.f;
  };
  auto read = [&](int set, const unsigned char* st, int ks) __attribute__((always_inline)) {
    if constexpr (LEAN) {
      asm volatile("" : "+v"(atA), "+v"(atB));
#pragma unroll
      for (int i = 0; i < TI; ++i) lean(fa[set][i], st + i * 4096, atA, ks);
#pragma unroll
      for (int j = 0; j < TJ; ++j) lean(fb[set][j], st + j * 4096, atB, ks);
    } else {
#pragma unroll
      for (int i = 0; i < TI; ++i) fa[set][i] = MMA::template frag<TA>((const bf16*)st, (wm * TI + i) * 32, ks, lane);
#pragma unroll
      for (int j = 0; j < TJ; ++j) fb[set][j] = MMA::template frag<TB>((const bf16*)(st + TA::BYTES), (wn * TJ + j) * 32, ks, lane);
    }
  };
#pragma unroll
  for (int s = 0; s < S; ++s) next(lds_raw + s * C::STAGE);
  asm volatile("" ::: "memory");
  wait_loads<(S - 1) * NL>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read(0, lds_raw, 0);
  for (int t0 = 0; t0 < nk; t0 += UN) {
    scales(t0);
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int t = t0 + u;
      if (t >= nk) break;
      unsigned char* const cur = lds_raw + (u % S) * C::STAGE;
      const unsigned char* const nxt = lds_raw + ((u + 1) % S) * C::STAGE;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int fc = s & 1, fn = fc ^ 1;
        const bool last = s == KS - 1;
        if (last) {
          asm volatile("" ::: "memory");
          wait_loads<(S - 2) * NL>();
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
        read(fn, last ? nxt : (const unsigned char*)cur, last ? 0 : s + 1);
        if (last) next(cur);
        if (!MMA::SCALED || (u & 3) == 0) mma_slice<MMA, 0>(fa[fc], fb[fc], acc, sa, sb);
        else if ((u & 3) == 1) mma_slice<MMA, 1>(fa[fc], fb[fc], acc, sa, sb);
        else if ((u & 3) == 2) mma_slice<MMA, 2>(fa[fc], fb[fc], acc, sa, sb);
        else mma_slice<MMA, 3>(fa[fc], fb[fc], acc, sa, sb);
#pragma unroll
        for (int q = 0; q < NM; ++q) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                       // MFMA
#pragma unroll
          for (int f = q * FPM; f < (q + 1) * FPM && f < NF; ++f) {                                // fragment reads of the next slice
            if (f < TI) __builtin_amdgcn_sched_group_barrier(0x100, TA::RPF * RPS, 0);
            else __builtin_amdgcn_sched_group_barrier(0x100, TB::RPF * RPS, 0);
          }
          if (last) __builtin_amdgcn_sched_group_barrier(0x020, (NL + NM - 1) / NM, 0);            // loads
        }
      }
    }
  }
  asm volatile("" ::: "memory");
  wait_loads<0>();
  __builtin_amdgcn_s_barrier();      // every wave is done with the stages, and nothing is in flight to them
  asm volatile("" ::: "memory");
}

// For products of few tiles, where the chain of latencies through the contraction is what counts: every wave of the block forms the whole 32 x 32 tile over the
// k-tiles w, w + NW, ..., from a ring of S stages of its own at `ring` and without a barrier; the tiles are added in wave order.  What comes back in acc is the sum,
// in wave 0.  next(dst) requests the wave's next k-tile (or, once they are used up, something harmless).
template <class MMA, class TA, class TB, int NW, int S, class Next>
__device__ __forceinline__ void ks_loop(int nk, unsigned char* lds_raw, f32x16& acc, int lane, int wave, Next&& next) {
  static_assert(!MMA::SCALED, "no scales");
  constexpr int KS = MMA::KS, STAGE = TA::BYTES + TB::BYTES, NL = TA::NI + TB::NI;
  unsigned char* const ring = lds_raw + wave * S * STAGE;
#pragma unroll
  for (int s = 0; s < S - 1; ++s) next(ring + s * STAGE);
  for (int t0 = 0; t0 < nk; t0 += S) {
#pragma unroll
    for (int u = 0; u < S; ++u) {
      const int t = t0 + u;
      if (t >= nk) break;
      asm volatile("" ::: "memory");
      wait_loads<(S - 2) * NL>();
      asm volatile("" ::: "memory");
      next(ring + ((u + S - 1) % S) * STAGE);      // its last reads are done: their results went into the last matrix instructions
      const bf16* sA = (const bf16*)(ring + u * STAGE);
      const bf16* sB = (const bf16*)(ring + u * STAGE + TA::BYTES);
      typename MMA::Frag fa[KS], fb[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) { fa[k] = MMA::template frag<TA>(sA, 0, k, lane); fb[k] = MMA::template frag<TB>(sB, 0, k, lane); }
#pragma unroll
      for (int k = 0; k < KS; ++k) MMA::template mma<0>(fa[k], fb[k], acc, 0, 0);
    }
  }
  asm volatile("" ::: "memory");
  wait_loads<0>();
  __syncthreads();               // the rings become the waves' tiles
  float4* const red = (float4*)lds_raw;
  if (wave > 0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) red[((wave - 1) * 4 + q) * 64 + lane] = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < NW - 1; ++w)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 v = red[(w * 4 + q) * 64 + lane];
        acc[4 * q] += v.x; acc[4 * q + 1] += v.y; acc[4 * q + 2] += v.z; acc[4 * q + 3] += v.w;
      }
  }
}

template <int TI, int TJ>
__device__ __forceinline__ void clear_tiles(f32x16 (&acc)[TI][TJ]) {
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
}

}  // namespace
