// Products in 8-bit floating point (e4m3) with a power-of-two scale for every 128 of the contraction, and the quantiser that writes their operands.
#include <algorithm>

#include "mma_tile.h"

namespace {

// ------------------------------------------------------------------------------------------
// quantiser
// ------------------------------------------------------------------------------------------
// One block per 128 x 128 elements, 256 threads with 8 x 8 elements each: the elements are read once and stay in registers until both forms are
// written.  The largest value of 128 in a row is the maximum over 16 lanes; of 128 in a column, over the 8 rows of a thread, the four row groups of a
// wave and, through LDS, the four waves.  A thread's 8 codes of a row go out as they are (16 lanes write a 128-byte line); its 8 codes of a column
// are put together in LDS, from where whole lines of the transposed codes go out.
// Scale: the least power of two 2^e with amax <= 448 2^e, held as the byte e + 127 (clamped to 0): a power of two changes no significand, so the only rounding is
// that of the code (nearest even, 4 significant bits), and the matrix instruction can apply it.  Values that are not finite become the code of NaN
// and do not enter the maximum.
constexpr int kQuantThreads = 256;
constexpr int kQuantLd = 128 + 16;      // bytes of a row of transposed codes in LDS

__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);      // 448 = 1.75 2^8
  return amax_bits == 0 ? 127u : (uint32_t)max(e, 0);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}
// a value times the inverse scale; infinities go on as NaN
__device__ __forceinline__ float scaled(float v, float inv) {
  const float y = v * inv;
  return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : y;
}

struct QuantDev {
  const void* x; int64_t ldx;
  int R, C, tile;
  uint8_t *q, *qs, *qt, *qts;      // a pair may be null
  int64_t ldq, ldqs, ldqt, ldqts;
  int nbx;                         // blocks along the columns
};

// A thread's 8 columns of the block's 128: neighbours in bf16, two times four in fp32, so that 16 lanes read whole lines with 16 bytes each.
template <class T>
__device__ __forceinline__ int quant_col(int cg, int t) { return sizeof(T) == 2 ? cg * 8 + t : (t >> 2) * 64 + cg * 4 + (t & 3); }
// half h of them (bf16: all, half 0), from their first
// (rows may start anywhere: 16 bytes are loaded at once at any element)
__device__ __forceinline__ void load_half(const float* __restrict__ p, int h, float (&v)[8]) {
  typedef f32x4 anywhere __attribute__((aligned(4)));
  const f32x4 a = *(const anywhere*)p;
#pragma unroll
  for (int t = 0; t < 4; ++t) v[4 * h + t] = a[t];
}
__device__ __forceinline__ void load_half(const bf16* __restrict__ p, int, float (&v)[8]) {
  typedef bf16x8 anywhere __attribute__((aligned(2)));
  const bf16x8 a = *(const anywhere*)p;
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = (float)a[t];
}

template <class T>
__global__ __launch_bounds__(kQuantThreads) void quantize_fp8_kernel(QuantDev p) {
  __shared__ uint32_t colmax[4][128];
  __shared__ uint32_t wavemax[4];
  __shared__ __attribute__((aligned(16))) uint8_t tq[128 * kQuantLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.x;
  const int bc = (int)(b % p.nbx), br = (int)(b / p.nbx);
  const int cg = tid & 15, rg = tid >> 4;                // column group, row group (8 each)
  const int r0 = br * 128 + rg * 8;
  // All loads of a thread are under way before the first is used: rows behind the matrix read its last one and become zeros afterwards.  (With a branch
  // per row instead, 8192 x 4096 took 43 us in place of 32.)
  constexpr int HALVES = sizeof(T) / 2, HALF = 8 / HALVES;
  float v[8][8];
  const T* const src = (const T*)p.x;
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    const int c = bc * 128 + quant_col<T>(cg, h * HALF);
    if (c + HALF <= p.C) {
#pragma unroll
      for (int i = 0; i < 8; ++i) load_half(src + (int64_t)min(r0 + i, p.R - 1) * p.ldx + c, h, v[i]);
    } else if (c < p.C) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int t = 0; t < HALF; ++t) v[i][h * HALF + t] = (float)src[(int64_t)min(r0 + i, p.R - 1) * p.ldx + min(c + t, p.C - 1)];
    }
    if (r0 + 8 > p.R || c + HALF > p.C) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int t = 0; t < HALF; ++t) if (r0 + i >= p.R || c + t >= p.C) v[i][h * HALF + t] = 0.0f;
    }
  }
  uint32_t rmax[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) m = max(m, finite_bits(v[i][t]));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    rmax[i] = m;
  }
  if (p.tile) {      // one scale for all: the maximum of the row maxima
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, rmax[i]);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if (lane == 0) wavemax[wave] = m;
    __syncthreads();
    m = max(max(wavemax[0], wavemax[1]), max(wavemax[2], wavemax[3]));
#pragma unroll
    for (int i = 0; i < 8; ++i) rmax[i] = m;
  }
  if (p.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + i;
      if (r >= p.R) break;
      const uint32_t byte = scale_byte(rmax[i]);
      const float inv = inverse_scale(byte);
      uint2 o;
      o.x = codes4(scaled(v[i][0], inv), scaled(v[i][1], inv), scaled(v[i][2], inv), scaled(v[i][3], inv));
      o.y = codes4(scaled(v[i][4], inv), scaled(v[i][5], inv), scaled(v[i][6], inv), scaled(v[i][7], inv));
      uint8_t* const at = p.q + (int64_t)r * p.ldq + bc * 128;
      if (sizeof(T) == 2) {
        *(uint2*)(at + cg * 8) = o;
      } else {
        *(uint32_t*)(at + cg * 4) = o.x;
        *(uint32_t*)(at + 64 + cg * 4) = o.y;
      }
      if (cg == 0) p.qs[(int64_t)r * p.ldqs + bc] = (uint8_t)byte;
    }
  }
  if (!p.qt) return;
  uint32_t cbyte[8];
  if (p.tile) {
#pragma unroll
    for (int t = 0; t < 8; ++t) cbyte[t] = scale_byte(rmax[0]);
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, finite_bits(v[i][t]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      if (lane < 16) colmax[wave][quant_col<T>(cg, t)] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int c = quant_col<T>(cg, t);
      cbyte[t] = scale_byte(max(max(colmax[0][c], colmax[1][c]), max(colmax[2][c], colmax[3][c])));
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float inv = inverse_scale(cbyte[t]);
    uint2 o;
    o.x = codes4(scaled(v[0][t], inv), scaled(v[1][t], inv), scaled(v[2][t], inv), scaled(v[3][t], inv));
    o.y = codes4(scaled(v[4][t], inv), scaled(v[5][t], inv), scaled(v[6][t], inv), scaled(v[7][t], inv));
    const int c = quant_col<T>(cg, t);
    *(uint2*)(tq + c * kQuantLd + rg * 8) = o;
    if (rg == 0 && bc * 128 + c < p.C) p.qts[(int64_t)(bc * 128 + c) * p.ldqts + br] = (uint8_t)cbyte[t];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {      // 8 lanes write a row's 128 bytes
    const int id = tid + k * kQuantThreads, c = id >> 3, at = (id & 7) * 16;
    if (bc * 128 + c < p.C) *(uint4*)(p.qt + (int64_t)(bc * 128 + c) * p.ldqt + br * 128 + at) = *(const uint4*)(tq + c * kQuantLd + at);
  }
}

// ------------------------------------------------------------------------------------------
// product
// ------------------------------------------------------------------------------------------
struct ScaleDev { const uint8_t *as, *bs; int64_t ldas, ldbs; };

// C = sum over blocks kb of 2^(as[m, kb] - 127) 2^(bs[n, kb] - 127) sum over k in kb of A[m, k] B[n, k].  A k-tile is one block of 128 codes, so that a
// row's scales of four k-tiles are one word; the words of the block's rows go into LDS like the operands, four k-tiles ahead, and from there into
// registers (held there two groups ahead they would cost the 256 x 256 tile 18 registers that it does not have).  Both operands k-major, rows of whole k-tiles (zeros
// behind K): nothing is masked.
template <class C>
constexpr size_t fp8_lds() { return std::max(C::PIPE, C::EPI_BYTES) + 2 * (C::BM + C::BN) * 4; }

template <class C, class MMA>
__device__ __forceinline__ void fp8_tile(const GemmDev& p, const ScaleDev& q, int m0, int n0, int split, unsigned char* lds_raw) {
  constexpr int TI = C::TI, TJ = C::TJ;
  typedef DmaTile<true, C::BK, C::BM, C::NS> TA;
  typedef DmaTile<true, C::BK, C::BN, C::NS> TB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  const int kbeg = split * p.k_per_split, kend = min(p.K, kbeg + p.k_per_split);
  const int nk = (kend - kbeg + 127) / 128;
  const int kbytes = (p.K + 127) / 128 * 128;
  const int mrows = min(C::BM, p.M - m0), nrows = min(C::BN, p.N - n0);
  typename TA::Cursor ca;
  typename TB::Cursor cb;
  // in units of two bytes, from the tile's first row on: offsets of 32 bits reach over 256 rows
  TA::init(ca, (const bf16*)p.A + (int64_t)m0 * (p.lda / 2), p.lda / 2, 0, mrows, kbeg / 2, kbytes / 2, lane, wave);
  TB::init(cb, (const bf16*)p.B + (int64_t)n0 * (p.ldb / 2), p.ldb / 2, 0, nrows, kbeg / 2, kbytes / 2, lane, wave);
  f32x16 acc[TI][TJ];
  clear_tiles(acc);
  const int words = (kbytes / 128 + 3) / 4;      // of a row of scales
  int sa[TI], sb[TJ];
  // the words of 64 rows per load instruction, A's rows first
  constexpr int NB = (C::BM + C::BN) / 64, PER = (NB + C::NW - 1) / C::NW;
  uint32_t* const store = (uint32_t*)(lds_raw + std::max(C::PIPE, C::EPI_BYTES));
  const int64_t spanA = (int64_t)(mrows - 1) * q.ldas + 4 * words, spanB = (int64_t)(nrows - 1) * q.ldbs + 4 * words;
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)(q.as + (int64_t)m0 * q.ldas), 0, (int)spanA, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)(q.bs + (int64_t)n0 * q.ldbs), 0, (int)spanB, 0x00020000);
  auto words_of = [&](int g) __attribute__((always_inline)) {      // group g of the split's k-tiles, into its half of the store
    if (nk <= 0) return;
    const int at = 4 * min(kbeg / 512 + g, words - 1);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int b = wave + k * C::NW;
      uint32_t* const dst = store + (g & 1) * (C::BM + C::BN) + b * 64;
      if (b < C::BM / 64) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void_ptr)dst, 4, (int)(min(b * 64 + lane, mrows - 1) * (int)q.ldas), at, 0, 0);
      else if (b < NB) __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void_ptr)dst, 4, (int)(min(b * 64 + lane - C::BM, nrows - 1) * (int)q.ldbs), at, 0, 0);
    }
  };
  words_of(0);
  int requested = 0;
  auto next = [&](unsigned char* dst) __attribute__((always_inline)) {
    if (requested >= nk) ca.soff = cb.soff = 0x80000000u;      // behind the operand: zeros
    ++requested;
    TA::issue(ca, dst, wave);
    TB::issue(cb, dst + TA::BYTES, wave);
  };
  auto scales = [&](int t) __attribute__((always_inline)) {
    const uint32_t* const src = store + ((t >> 2) & 1) * (C::BM + C::BN) + (lane & 31);
#pragma unroll
    for (int i = 0; i < TI; ++i) sa[i] = (int)src[(wm * TI + i) * 32];
#pragma unroll
    for (int j = 0; j < TJ; ++j) sb[j] = (int)src[C::BM + (wn * TJ + j) * 32];
    words_of((t >> 2) + 1);
  };
  mma_loop<C, MMA, TA, TB>(nk, lds_raw, acc, sa, sb, wm, wn, lane, next, scales);

  const int rbase = m0 + wm * TI * 32, cbase = n0 + wn * TJ * 32;
  float* stage = (float*)lds_raw + wave * C::EPI_FLOATS;
  // rows of the result that do not start on 16 bytes go out as they lie in the registers, with a column's bias loaded once (1237 x 2603 x 1000 with bias: 22 us element
  // by element through LDS)
  auto finish = [&](auto mode_tag, int sp) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_tag)::value;
    if (octet_aligned<MODE>(p)) tile_epilogue_pipe<MODE, TI, TJ>(p, acc, rbase, cbase, lane, sp, stage, nullptr);
    else tile_epilogue<MODE, TI, TJ>(p, acc, rbase, cbase, lane, sp);
  };
  if (p.partial) finish(std::integral_constant<int, EPI_PARTIAL>{}, split);
  else if (p.c_f32) finish(std::integral_constant<int, EPI_F32>{}, 0);
  else finish(std::integral_constant<int, EPI_ACT>{}, 0);
}

template <class C, class MMA>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(C::WPE, C::WPE)))
void gemm_fp8_kernel(GemmDev p, ScaleDev q, int nbx, int nby) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  // tile order as in gemm_bf16_wide
  const int nb = nbx * nby;
  int v = blockIdx.x;
  const int per_xcd = (int)gridDim.x >> 3;
  if (v < 8 * per_xcd) v = (v & 7) * per_xcd + (v >> 3);
  const int split = v / nb;
  int tm, tn;
  tile_of_block<(C::BM >= 256) ? 4 : 8>(v - split * nb, nbx, nby, tm, tn);
  fp8_tile<C, MMA>(p, q, tm * C::BM, tn * C::BN, split, lds_raw);
}

template <class C, class MMA>
hipError_t launch_fp8_one(const GemmDev& p, const ScaleDev& q, int splits, hipStream_t s) {
  auto kern = gemm_fp8_kernel<C, MMA>;
  constexpr size_t lds = fp8_lds<C>();
  static_assert(C::OCC * lds <= 160 * 1024, "the blocks of a CU do not fit its LDS");
  static bool configured = false;      // per instantiation, as in gemm_wide.h
  if (!configured && lds > 48 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  configured = true;
  const int nbx = (int)((p.N + (int64_t)C::BN - 1) / C::BN), nby = (int)((p.M + (int64_t)C::BM - 1) / C::BM);
  hipLaunchKernelGGL(kern, dim3((unsigned)(nbx * nby * splits)), dim3(C::NT), lds, s, p, q, nbx, nby);
  return hipGetLastError();
}
template <class C>
hipError_t launch_fp8(const GemmDev& p, const ScaleDev& q, int splits, hipStream_t s) {
  return p.c_f32 ? launch_fp8_one<C, MmaE4M3Wide>(p, q, splits, s) : launch_fp8_one<C, MmaE4M3>(p, q, splits, s);
}

typedef DmaCfg<1, 1, 2, 2, 1, 64, 4, 2, true> F8_64x64;      // TI TJ WGM WGN KW BK S OCC AHEAD
typedef DmaCfg<2, 2, 2, 2, 1, 64, 2, 2, true> F8_128x128;
typedef DmaCfg<4, 2, 2, 4, 1, 64, 2, 1, true> F8_256x256;

// Sum of a split contraction's parts in their order, bias, beta; four columns per thread.  Memory bound.
__global__ __launch_bounds__(256) void fp8_reduce_kernel(GemmDev p, int splits) {
  const int64_t per_row = (p.N + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= per_row * p.M) return;
  const int row = (int)(id / per_row), col = (int)(id % per_row) * 4;
  const int have = min(4, p.N - col);
  const float* src = p.partial + (int64_t)row * p.N + col;
  const int64_t stride = (int64_t)p.M * p.N;
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if ((p.N & 3) == 0) {
    for (int s = 0; s < splits; ++s) {
      const float4 x = *(const float4*)(src + s * stride);
      v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
  } else {
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k) if (k < have) v[k] += src[s * stride + k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k >= have) break;
    const int64_t o = (int64_t)row * p.ldc + col + k;
    const float x = v[k] + (p.bias ? (float)((const bf16*)p.bias)[col + k] : 0.0f);
    if (p.c_f32) { float* C = (float*)p.C + o; *C = p.beta != 0.0f ? p.beta * *C + x : x; }
    else ((bf16*)p.C)[o] = (bf16)x;
  }
}

// The time of a product with each tile, in us: rounds of the chip times (w per k-tile + e), with blocks that have a CU to themselves w1 per k-tile; fitted to 8192^3,
// 16384 x 4096 x 1024, 16384 x 1024 x 4096, 4096^3, 2048 x 1024 x 1024 and 512 x 1024 x 1024 (bf16 results: us with 64, 128, 256 tiles 836, 522, 432; 150, 90, 80; 109, 71,
// 61; 112, 70, 60; 6.6, 7.6, 15; 4.6, 7.1, 15) and 8192^3, 1024 x 4096 x 16384, 768 x 768 x 8192 (fp32: 1293, 926, 814; 167, 130, 257; 26, 51, 130).  A split contraction pays a second launch and its partial sums' way through memory, as in gemm.hip.
constexpr int kCUs = 256;
struct Fp8Cfg { int b, occ; float w, w1, e; };
const Fp8Cfg kFp8Cfg[2][3] = {{{64, 2, 0.39f, 0.17f, 1.4f}, {128, 2, 0.95f, 0.5f, 3.2f}, {256, 1, 1.58f, 1.58f, 7.3f}},
                              {{64, 2, 0.62f, 0.36f, 2.0f}, {128, 2, 1.75f, 0.85f, 5.0f}, {256, 1, 3.2f, 3.2f, 10.0f}}};

void choose_fp8(int M, int N, int K, int c_f32, size_t scratch_bytes, int* cfg, int* splits) {
  const int kb = (K + 127) / 128;
  float best = 3.0e38f;
  *cfg = 0; *splits = 1;
  for (int c = 0; c < 3; ++c) {
    const Fp8Cfg& f = kFp8Cfg[c_f32 ? 1 : 0][c];
    const int64_t tiles = ((M + (int64_t)f.b - 1) / f.b) * ((N + (int64_t)f.b - 1) / f.b);
    for (int sp = 1; sp <= 32; sp *= 2) {
      const int steps = ((kb + sp - 1) / sp + 3) / 4 * 4;      // whole scale words
      if (sp > 1 && (steps * (sp - 1) >= kb || (double)sp * M * N * sizeof(float) > (double)scratch_bytes || (double)M * N > 4e9)) break;
      const int64_t n = tiles * sp, slots = (int64_t)f.occ * kCUs, rest = n % slots;
      const float nk = (float)std::min(kb, steps);
      float t = (float)(n / slots) * (f.w * nk + f.e) + (rest == 0 ? 0.0f : (rest <= kCUs ? f.w1 : f.w) * nk + f.e);
      if (sp > 1) t += 3.0f + 8e-6f * sp * (float)M * (float)N / 3.5f;
      if (t < best) { best = t; *cfg = c; *splits = sp; }
    }
  }
}

// The tile (its place in kFp8Cfg), the contraction of a part in whole scale words, and the parts that have some of it.
void plan_fp8(int M, int N, int K, int c_f32, size_t scratch_bytes, int* cfg, int* k_per_split, int* splits) {
  const int64_t kb = (K + (int64_t)127) / 128;
  choose_fp8(M, N, K, c_f32, scratch_bytes, cfg, splits);
  *k_per_split = std::max<int>(1, (int)((kb + *splits - 1) / *splits + 3) / 4) * 512;
  *splits = std::max(1, (K + *k_per_split - 1) / *k_per_split);
}

}  // namespace

extern "C" {

hs_status hs_op_quantize_fp8(int32_t dtype, const void* x, int64_t ldx, int32_t R, int32_t C, int32_t tile, void* q, int64_t ldq, uint8_t* qs,
                             int64_t ldqs, void* qt, int64_t ldqt, uint8_t* qts, int64_t ldqts, void* stream) {
  if (dtype != HS_FP32 && dtype != HS_BF16) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_quantize_fp8: bad dtype");
  if (R < 0 || C < 0 || tile < 0 || tile > 1) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_quantize_fp8: negative size or bad tile flag");
  if ((q == nullptr) != (qs == nullptr) || (qt == nullptr) != (qts == nullptr) || (!q && !qt))
    return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_quantize_fp8: codes and scales come in pairs, one pair at least");
  if (R == 0 || C == 0) return HS_OK;
  if (!x) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_quantize_fp8: NULL input");
  if (ldx < C) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: rows of the input overlap");
  if ((uintptr_t)x % esize(dtype)) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: the input is not aligned to its type");
  const int64_t cb = (C + (int64_t)127) / 128, rb = (R + (int64_t)127) / 128;
  if (q && (ldq % 128 || ldq < 128 * cb || ldqs < cb || ((uintptr_t)q & 15)))
    return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: q needs rows of whole blocks of 128 and 16-byte alignment, qs a byte per block");
  if (qt && (ldqt % 128 || ldqt < 128 * rb || ldqts < rb || ((uintptr_t)qt & 15)))
    return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: qt needs rows of whole blocks of 128 and 16-byte alignment, qts a byte per block");
  if (cb * rb >= ((int64_t)1 << 32) / kQuantThreads) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: too many blocks");      // threads of one launch
  QuantDev p{x, ldx, R, C, tile, (uint8_t*)q, qs, (uint8_t*)qt, qts, ldq, ldqs, ldqt, ldqts, (int)cb};
  hipLaunchKernelGGL(dtype == HS_BF16 ? quantize_fp8_kernel<bf16> : quantize_fp8_kernel<float>, dim3((unsigned)(cb * rb)), dim3(kQuantThreads), 0,
                     (hipStream_t)stream, p);
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, std::string("hs_op_quantize_fp8: ") + hipGetErrorString(e));
}

hs_status hs_gemm_fp8_choice(int32_t M, int32_t N, int32_t K, int32_t c_f32, size_t scratch_bytes, int32_t* tile, int32_t* splits) {
  if (M < 1 || N < 1 || K < 1 || K > 1 << 22 || !tile || !splits) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_gemm_fp8_choice: bad argument");
  int cfg, per, n;
  plan_fp8(M, N, K, c_f32 ? 1 : 0, scratch_bytes, &cfg, &per, &n);
  *tile = kFp8Cfg[0][cfg].b; *splits = n;
  return HS_OK;
}

hs_status hs_op_gemm_fp8(int32_t M, int32_t N, int32_t K, const void* A, int64_t lda, const uint8_t* as, int64_t ldas, const void* B, int64_t ldb,
                         const uint8_t* bs, int64_t ldbs, void* C, int64_t ldc, int32_t c_f32, float beta, const void* bias, void* scratch,
                         size_t scratch_bytes, void* stream) {
  if (M < 0 || N < 0 || K < 0) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_gemm_fp8: negative size");
  if (M == 0 || N == 0) return HS_OK;
  if (!C || (K > 0 && (!A || !as || !B || !bs))) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_gemm_fp8: NULL operand");
  if (ldc < N) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: rows of C overlap");
  const int64_t kb = (K + (int64_t)127) / 128, most = (int64_t)1 << 22;
  if (lda % 128 || ldb % 128 || lda < 128 * kb || ldb < 128 * kb || lda > most || ldb > most || ((uintptr_t)A & 15) || ((uintptr_t)B & 15))
    return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: codes need rows of whole blocks of 128 (at most 4 MiB) and 16-byte alignment");
  if (ldas % 4 || ldbs % 4 || ldas < kb || ldbs < kb || ldas > most || ldbs > most || ((uintptr_t)as & 3) || ((uintptr_t)bs & 3))
    return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: scales need a byte per block, in rows of whole aligned 4-byte words");
  if (((uintptr_t)C % (c_f32 ? 4 : 2)) || ((uintptr_t)bias & 1)) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: C or bias is not aligned");
  if ((uintptr_t)scratch & 15) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: scratch must be 16-byte aligned");
  GemmDev p{};
  p.A = A; p.B = B; p.C = C; p.bias = bias;
  p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  p.M = M; p.N = N; p.K = K; p.c_f32 = c_f32 ? 1 : 0; p.beta = beta;
  int cfg, splits;
  plan_fp8(M, N, K, p.c_f32, scratch ? scratch_bytes : 0, &cfg, &p.k_per_split, &splits);
  const int64_t bt = kFp8Cfg[0][cfg].b, blocks = ((M + bt - 1) / bt) * ((N + bt - 1) / bt) * splits;
  if (blocks >= ((int64_t)1 << 32) / 512) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: too many tiles");      // threads of one launch
  p.partial = splits > 1 ? (float*)scratch : nullptr;
  const ScaleDev q{as, bs, ldas, ldbs};
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = cfg == 2 ? launch_fp8<F8_256x256>(p, q, splits, s) : cfg == 1 ? launch_fp8<F8_128x128>(p, q, splits, s) : launch_fp8<F8_64x64>(p, q, splits, s);
  if (e == hipSuccess && splits > 1) {
    hipLaunchKernelGGL(fp8_reduce_kernel, dim3((unsigned)(((int64_t)M * ((N + 3) / 4) + 255) / 256)), dim3(256), 0, s, p, splits);
    e = hipGetLastError();
  }
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, std::string("hs_op_gemm_fp8: ") + hipGetErrorString(e));
}

}  // extern "C"
