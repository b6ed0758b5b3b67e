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

template <class T>
__device__ __forceinline__ void load8(const T* __restrict__ p, int n, bool vec, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* __restrict__ p, int n, bool vec, float (&v)[8]) {
  if (vec && n >= 8) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = t < n ? p[t] : 0.0f;
  }
}
template <>
__device__ __forceinline__ void load8<bf16>(const bf16* __restrict__ p, int n, bool vec, float (&v)[8]) {
  if (vec && n >= 8) {
    const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = (float)a[t];
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = t < n ? (float)p[t] : 0.0f;
  }
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
  const int c0 = bc * 128 + cg * 8, r0 = br * 128 + rg * 8;
  const bool vec = (p.ldx % (16 / sizeof(T))) == 0 && ((uintptr_t)p.x & 15) == 0;
  float v[8][8];
  const T* const src = (const T*)p.x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + i;
    load8<T>(src + (int64_t)r * p.ldx + c0, r < p.R ? p.C - c0 : 0, vec, v[i]);
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
      *(uint2*)(p.q + (int64_t)r * p.ldq + c0) = o;
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
      if (lane < 16) colmax[wave][cg * 8 + t] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int c = cg * 8 + t;
      cbyte[t] = scale_byte(max(max(colmax[0][c], colmax[1][c]), max(colmax[2][c], colmax[3][c])));
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float inv = inverse_scale(cbyte[t]);
    uint2 o;
    o.x = codes4(scaled(v[0][t], inv), scaled(v[1][t], inv), scaled(v[2][t], inv), scaled(v[3][t], inv));
    o.y = codes4(scaled(v[4][t], inv), scaled(v[5][t], inv), scaled(v[6][t], inv), scaled(v[7][t], inv));
    *(uint2*)(tq + (cg * 8 + t) * kQuantLd + rg * 8) = o;
    if (rg == 0 && c0 + t < p.C) p.qts[(int64_t)(c0 + t) * p.ldqts + br] = (uint8_t)cbyte[t];
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
// lane's scales change with the k-tile: a row's bytes of four k-tiles are one word, read two groups ahead.  Both operands k-major, rows of whole k-tiles (zeros
// behind K): nothing is masked.
template <class C, class MMA>
__device__ __forceinline__ void fp8_tile(const GemmDev& p, const ScaleDev& q, int m0, int n0, int split, unsigned char* lds_raw) {
  constexpr int TI = C::TI, TJ = C::TJ;
  typedef DmaTile<true, C::BK, C::BM, C::NW> TA;
  typedef DmaTile<true, C::BK, C::BN, C::NW> TB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  const int kbeg = split * p.k_per_split, kend = min(p.K, kbeg + p.k_per_split);
  const int nk = (kend - kbeg + 127) / 128;
  const int kbytes = (p.K + 127) / 128 * 128;
  typename TA::Cursor ca;
  typename TB::Cursor cb;
  // in units of two bytes, from the tile's first row on: offsets of 32 bits reach over 256 rows
  TA::init(ca, (const bf16*)p.A + (int64_t)m0 * (p.lda / 2), p.lda / 2, 0, min(C::BM, p.M - m0), kbeg / 2, kbytes / 2, lane, wave);
  TB::init(cb, (const bf16*)p.B + (int64_t)n0 * (p.ldb / 2), p.ldb / 2, 0, min(C::BN, p.N - n0), kbeg / 2, kbytes / 2, lane, wave);
  f32x16 acc[TI][TJ];
  clear_tiles(acc);
  int requested = 0;
  auto next = [&](unsigned char* dst) __attribute__((always_inline)) {
    if (requested >= nk) ca.soff = cb.soff = 0x80000000u;      // behind the operand: zeros
    ++requested;
    TA::issue(ca, dst, wave);
    TB::issue(cb, dst + TA::BYTES, wave);
  };
  const uint8_t *pa[TI], *pb[TJ];
  uint32_t cura[TI], curb[TJ], nxta[TI], nxtb[TJ];
  int sa[TI], sb[TJ];
  const int first = kbeg / 512, lastg = (kbytes / 128 - 1) / 4;
  auto word = [&](const uint8_t* row, int g) __attribute__((always_inline)) { return nk > 0 ? *(const uint32_t*)(row + 4 * g) : 0u; };      // none where K == 0
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    pa[i] = q.as + (int64_t)min(m0 + (wm * TI + i) * 32 + (lane & 31), p.M - 1) * q.ldas;
    cura[i] = word(pa[i], first);
    nxta[i] = word(pa[i], min(first + 1, lastg));
  }
#pragma unroll
  for (int j = 0; j < TJ; ++j) {
    pb[j] = q.bs + (int64_t)min(n0 + (wn * TJ + j) * 32 + (lane & 31), p.N - 1) * q.ldbs;
    curb[j] = word(pb[j], first);
    nxtb[j] = word(pb[j], min(first + 1, lastg));
  }
  auto scales = [&](int t) __attribute__((always_inline)) {
    if (t && (t & 3) == 0) {
      const int g = min(first + (t >> 2) + 1, lastg);
#pragma unroll
      for (int i = 0; i < TI; ++i) { cura[i] = nxta[i]; nxta[i] = word(pa[i], g); }
#pragma unroll
      for (int j = 0; j < TJ; ++j) { curb[j] = nxtb[j]; nxtb[j] = word(pb[j], g); }
    }
#pragma unroll
    for (int i = 0; i < TI; ++i) sa[i] = MMA::scale(cura[i], t);
#pragma unroll
    for (int j = 0; j < TJ; ++j) sb[j] = MMA::scale(curb[j], t);
  };
  mma_loop<C, MMA, TA, TB>(nk, lds_raw, acc, sa, sb, wm, wn, lane, next, scales);

  const int rbase = m0 + wm * TI * 32, cbase = n0 + wn * TJ * 32;
  float* stage = (float*)lds_raw + wave * C::EPI_FLOATS;
  if (p.partial) tile_epilogue_pipe<EPI_PARTIAL, TI, TJ>(p, acc, rbase, cbase, lane, split, stage, nullptr);
  else if (p.c_f32) tile_epilogue_pipe<EPI_F32, TI, TJ>(p, acc, rbase, cbase, lane, 0, stage, nullptr);
  else tile_epilogue_pipe<EPI_ACT, TI, TJ>(p, acc, rbase, cbase, lane, 0, stage, nullptr);
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

template <class C>
hipError_t launch_fp8(const GemmDev& p, const ScaleDev& q, int splits, hipStream_t s) {
  auto kern = p.c_f32 ? gemm_fp8_kernel<C, MmaE4M3Wide> : gemm_fp8_kernel<C, MmaE4M3>;
  if (C::LDS > 48 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS);
    if (e != hipSuccess) return e;
  }
  const int nbx = (p.N + C::BN - 1) / C::BN, nby = (p.M + C::BM - 1) / C::BM;
  hipLaunchKernelGGL(kern, dim3((unsigned)(nbx * nby * splits)), dim3(C::NT), C::LDS, s, p, q, nbx, nby);
  return hipGetLastError();
}

typedef DmaCfg<1, 1, 2, 2, 1, 64, 3, 3, true> F8_64x64;      // TI TJ WGM WGN KW BK S OCC AHEAD
typedef DmaCfg<2, 2, 2, 2, 1, 64, 2, 2, true> F8_128x128;

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
  if (cb * rb > INT32_MAX) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_quantize_fp8: too many blocks");
  QuantDev p{x, ldx, R, C, tile, (uint8_t*)q, qs, (uint8_t*)qt, qts, ldq, ldqs, ldqt, ldqts, (int)cb};
  hipLaunchKernelGGL(dtype == HS_BF16 ? quantize_fp8_kernel<bf16> : quantize_fp8_kernel<float>, dim3((unsigned)(cb * rb)), dim3(kQuantThreads), 0,
                     (hipStream_t)stream, p);
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, std::string("hs_op_quantize_fp8: ") + hipGetErrorString(e));
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
  if (ldas % 4 || ldbs % 4 || ldas < kb || ldbs < kb || ((uintptr_t)as & 3) || ((uintptr_t)bs & 3))
    return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: scales need a byte per block, in rows of whole aligned 4-byte words");
  if (((uintptr_t)C % (c_f32 ? 4 : 2)) || ((uintptr_t)bias & 1)) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: C or bias is not aligned");
  (void)scratch; (void)scratch_bytes;
  GemmDev p{};
  p.A = A; p.B = B; p.C = C; p.bias = bias;
  p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  p.M = M; p.N = N; p.K = K; p.c_f32 = c_f32 ? 1 : 0; p.beta = beta;
  p.k_per_split = std::max<int>(1, (int)(kb + 3) / 4) * 512;
  const ScaleDev q{as, bs, ldas, ldbs};
  if (((M + (int64_t)63) / 64) * ((N + (int64_t)63) / 64) > INT32_MAX) return hs_fail(nullptr, HS_ERR_SHAPE, "hs_op_gemm_fp8: too many tiles");
  const int64_t mid = (int64_t)((M + 127) / 128) * ((N + 127) / 128);
  hipError_t e = mid >= 192 ? launch_fp8<F8_128x128>(p, q, 1, (hipStream_t)stream) : launch_fp8<F8_64x64>(p, q, 1, (hipStream_t)stream);
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, std::string("hs_op_gemm_fp8: ") + hipGetErrorString(e));
}

}  // extern "C"
