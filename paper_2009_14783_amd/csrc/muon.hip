// Update of weight matrices by their orthogonalised momentum: Newton-Schulz products on lists of matrices of different shapes.
//
// A matrix U is divided by its Frobenius norm and sent `steps` times through X <- a X + (b A + c A A) X with A = X X^T: an odd polynomial of the singular
// values that takes them towards 1 and leaves the singular vectors.  X is held with its shorter side as rows (a tall matrix is transposed on its
// way in and out), so that A is as small as it can be, in a workspace whose sides are padded with zeros to multiples of 64 (zeros stay zeros): no product
// masks anything.  A and A A are symmetric: only the tiles on and above the diagonal are computed, the others are their mirror images.
//
// Numbers.  The matrix instructions take fp16: as fast as bf16 with three more bits, and the range is no matter here, since every value is bounded by the
// largest singular value (X is held times 2^8, A times 2^12, S times 2^10, which keeps small entries above the subnormals).  What the roundings do is
// decided by what the polynomial amplifies: a direction with a small singular value grows by a = 3.4 in every step, and the rounding of the large ones
// would grow with it.  So X is kept as the sum of two fp16 numbers (22 bits) and a X is formed from both, in 32 bits; only the product with S reads the
// first alone, and S vanishes on the small directions.  The diagonal of S, whose rounding is of one sign in a whole row of X, is taken out
// of it and applied in 32 bits too.  Relative error of the result (2-norm, CPU emulation): Gaussian 768 x 768 8e-4, 512 x 512 of rank 32 with 2 % noise 8e-4; with
// X in one fp16 number and the diagonal left in 1.4e-3 and 2.4e-2; all in bf16 1.1e-2 and 1.9e-1.  32-bit products (HS_FP32) take the second numbers of both operands
// along: three products hi hi + hi lo + lo hi as one contraction three times as long, error as in fp32.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "mma_tile.h"

namespace {

constexpr int kGroups = 16;           // shapes of one launch
constexpr int kParts = 256;           // partial sums of a matrix' norm, at most
constexpr int kPartElems = 16384;     // ... of so many elements at least
constexpr float kSx = 256.0f, kSa = 4096.0f, kSs = 1024.0f;

// Matrices of one shape; `first` is the place of the first one in the table of offsets.
struct NsGroup {
  int rows, cols, m, n, tall, count, first, parts;
  int64_t ws, stride;      // bytes: first matrix' part of the workspace, and from one matrix to the next
};
struct NsPlace { int64_t offset, ld; };      // a matrix in the flat buffers
struct NsDev {
  int ng, split;           // split: 32-bit products
  int first_block[kGroups + 1];
  NsGroup g[kGroups];
  char* ws;
  const NsPlace* table;
  double* partial;         // [matrices][kParts]
  int from;                // which of the two X is read
  float a, b, c;
};
static_assert(sizeof(NsDev) < 2048, "kernel arguments");

// parts of a matrix' workspace
struct NsParts { size_t x, a, s, diag, total; };      // x: bytes of one X (both its numbers); the other one is behind it
__host__ __device__ inline NsParts ns_parts(int m, int n, int split) {
  NsParts p;
  const size_t x = (size_t)m * n * 2, a = (size_t)m * m * 2;
  p.x = 2 * x; p.a = 4 * x; p.s = p.a + (split ? 2 : 1) * a; p.diag = p.s + (split ? 2 : 1) * a;
  p.total = (p.diag + (size_t)m * 4 + 255) & ~(size_t)255;
  return p;
}

// the group, matrix and block within the matrix of this thread block, whose matrices have `per` blocks each
__device__ __forceinline__ int ns_group(const NsDev& d, int v) {
  int i = 0;
  while (i + 1 < d.ng && v >= d.first_block[i + 1]) ++i;
  return i;
}

struct TableArg { NsPlace place[200]; int first, n; };
__global__ void ns_table_kernel(TableArg t, NsPlace* __restrict__ table) {
  const int i = threadIdx.x;
  if (i < t.n) table[t.first + i] = t.place[i];
}

// ---- where the matrices come from and go to ---------------------------------------------------------
// update: momentum and weights; otherwise a flat buffer of matrices in, another out
struct MuonIO {
  float *w, *m; const float* G; bf16* wl;
  float denom, mu, decay, lr, rms;      // denom 0: G as it is; decay = 1 - lr wd
  int nesterov, scale;
};
struct PlainIO { const void* x; void* y; int bf; };

__device__ __forceinline__ float plain_at(const PlainIO& io, int64_t i) { return io.bf ? (float)((const bf16*)io.x)[i] : ((const float*)io.x)[i]; }

// First pass: the momentum is updated, and the sum of squares of what is going to be orthogonalised is formed in 64 bits (gradients of 1e-25 have squares
// that 32 bits do not hold), a part of a matrix per block, added in a fixed order.  Memory bound: 12 bytes per element.
template <class IO>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsDev d, IO io) {
  const int gi = ns_group(d, blockIdx.x);
  const NsGroup& g = d.g[gi];
  const int local = blockIdx.x - d.first_block[gi], mat = local / g.parts, part = local % g.parts;
  const NsPlace at = d.table[g.first + mat];
  const int64_t total = (int64_t)g.rows * g.cols, chunk = (total + g.parts - 1) / g.parts;
  const int64_t end = min(total, (part + 1) * chunk);
  double sum = 0.0;
  for (int64_t e = part * chunk + threadIdx.x; e < end; e += 256) {
    const int64_t r = e / g.cols, i = at.offset + r * at.ld + (e - r * g.cols);
    float u;
    if constexpr (std::is_same<IO, MuonIO>::value) {
      float gr = io.G[i];
      if (io.denom > 0.0f) gr /= io.denom;
      const float m = io.mu * io.m[i] + gr;
      io.m[i] = m;
      u = io.nesterov ? gr + io.mu * m : m;
    } else {
      u = plain_at(io, i);
    }
    sum += (double)u * (double)u;
  }
  __shared__ double red[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) d.partial[(int64_t)(g.first + mat) * kParts + part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// Second pass: X = U / (|U| + eps) in two fp16 numbers, the shorter side as rows, zeros in the padding.  64 x 64 elements per block.
template <class IO>
__global__ __launch_bounds__(256) void ns_start_kernel(NsDev d, IO io, double eps) {
  const int gi = ns_group(d, blockIdx.x);
  const NsGroup& g = d.g[gi];
  const int nbn = g.n / 64, per = g.m / 64 * nbn, local = blockIdx.x - d.first_block[gi], mat = local / per, t = local % per;
  const int i0 = t / nbn * 64, j0 = t % nbn * 64;
  const NsPlace at = d.table[g.first + mat];
  __shared__ float tile[64][65];
  __shared__ double inv_s;
  if (threadIdx.x < 64) {
    double s = 0.0;
    for (int k = threadIdx.x; k < g.parts; k += 64) s += d.partial[(int64_t)(g.first + mat) * kParts + k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (threadIdx.x == 0) inv_s = s == 0.0 ? 0.0 : (double)kSx / (sqrt(s) + eps);      // a matrix of zeros stays one
  }
  __syncthreads();
  const double inv = inv_s;
  const int r0 = g.tall ? j0 : i0, c0 = g.tall ? i0 : j0;
  for (int e = threadIdx.x; e < 4096; e += 256) {
    const int lr = e >> 6, lc = e & 63, r = r0 + lr, c = c0 + lc;
    float u = 0.0f;
    if (r < g.rows && c < g.cols) {
      const int64_t i = at.offset + r * at.ld + c;
      if constexpr (std::is_same<IO, MuonIO>::value) {
        u = io.m[i];
        if (io.nesterov) { float gr = io.G[i]; if (io.denom > 0.0f) gr /= io.denom; u = gr + io.mu * u; }
      } else {
        u = plain_at(io, i);
      }
      u = (float)((double)u * inv);
    }
    if (g.tall) tile[lc][lr] = u; else tile[lr][lc] = u;
  }
  __syncthreads();
  f16* const hi = (f16*)(d.ws + g.ws + mat * g.stride);
  f16* const lo = hi + (int64_t)g.m * g.n;
  for (int e = threadIdx.x; e < 512; e += 256) {
    const int r = e >> 3, c = (e & 7) * 8;
    f16x8 h, l;
#pragma unroll
    for (int k = 0; k < 8; ++k) { const float x = tile[r][c + k]; h[k] = (f16)x; l[k] = (f16)(x - (float)h[k]); }
    const int64_t o = (int64_t)(i0 + r) * g.n + j0 + c;
    *(f16x8*)(hi + o) = h;
    *(f16x8*)(lo + o) = l;
  }
}

// ---- the products ---------------------------------------------------------------------------------
enum { NS_GRAM = 0, NS_SQUARE, NS_APPLY, NS_LAST };

// the tile (row, column >= row) of number t of a symmetric matrix of nb x nb tiles
__device__ __forceinline__ void upper_tile(int t, int nb, int& ti, int& tj) {
  int r = (int)((2.0f * nb + 1.0f - sqrtf((2.0f * nb + 1.0f) * (2.0f * nb + 1.0f) - 8.0f * t)) * 0.5f);
  r = max(0, min(r, nb - 1));
  while (r > 0 && r * nb - r * (r - 1) / 2 > t) --r;
  while ((r + 1) * nb - (r + 1) * r / 2 <= t) ++r;
  ti = r; tj = r + t - (r * nb - r * (r - 1) / 2);
}

template <class C, int OP, class IO>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(C::WPE, C::WPE)))
void ns_product_kernel(NsDev d, IO io) {
  constexpr int TI = C::TI, TJ = C::TJ, WN = 32 * TJ, LDW = WN + 4;
  constexpr bool SYM = OP == NS_GRAM || OP == NS_SQUARE;
  typedef DmaTile<true, C::BK, C::BM, C::NW> TA;
  typedef DmaTile<SYM, C::BK, C::BN, C::NW> TB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  int v = blockIdx.x;      // a contiguous range of tiles per XCD
  const int per_xcd = (int)gridDim.x >> 3;
  if (v < 8 * per_xcd) v = (v & 7) * per_xcd + (v >> 3);
  const int gi = ns_group(d, v);
  const NsGroup& g = d.g[gi];
  const int m = g.m, n = g.n, nbm = (m + C::BM - 1) / C::BM, nbn = (n + C::BN - 1) / C::BN;
  const int per = SYM ? nbm * (nbm + 1) / 2 : nbm * nbn, local = v - d.first_block[gi], mat = local / per, t = local % per;
  int ti, tj;
  if (SYM) upper_tile(t, nbm, ti, tj);
  else tile_of_block<4>(t, nbn, nbm, ti, tj);
  const int m0 = ti * C::BM, n0 = tj * C::BN;
  const NsParts parts = ns_parts(m, n, d.split);
  char* const base = d.ws + g.ws + mat * g.stride;
  f16* const X = (f16*)(base + d.from * parts.x);
  f16* const Xn = (f16*)(base + (d.from ^ 1) * parts.x);
  f16* const A = (f16*)(base + parts.a);
  f16* const Sm = (f16*)(base + parts.s);
  float* const diag = (float*)(base + parts.diag);

  // operands, and how far behind the first numbers the second ones are (bytes)
  const f16* const opA = OP == NS_GRAM ? X : OP == NS_SQUARE ? A : Sm;
  const f16* const opB = OP == NS_SQUARE ? A : X;
  const int K = OP == NS_GRAM ? n : m;
  const int64_t sizeA = (int64_t)m * K * 2, sizeB = OP == NS_SQUARE ? sizeA : (int64_t)m * n * 2;
  const int nk1 = K / 64, nseg = d.split ? 3 : 1;
  typename TA::Cursor ca;
  typename TB::Cursor cb;
  TA::init(ca, (const bf16*)opA, K, m0, m, 0, K, lane, wave);
  if (SYM) TB::init(cb, (const bf16*)opB, K, n0, m, 0, K, lane, wave);
  else TB::init(cb, (const bf16*)opB, n, n0, n, 0, K, lane, wave);
  ca.rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)opA, 0, (int)(d.split ? 2 * sizeA : sizeA), 0x00020000);
  cb.rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)opB, 0, (int)(d.split ? 2 * sizeB : sizeB), 0x00020000);
  int kt = 0, seg = 0;
  auto next = [&](unsigned char* dst) __attribute__((always_inline)) {
    if (kt == nk1) {      // hi hi, hi lo, lo hi; then behind the operands
      kt = 0; ++seg;
      ca.soff = seg >= nseg ? 0x80000000u : seg == 2 ? (unsigned)sizeA : 0u;
      cb.soff = seg >= nseg ? 0x80000000u : seg == 1 ? (unsigned)sizeB : 0u;
    }
    ++kt;
    TA::issue(ca, dst, wave);
    TB::issue(cb, dst + TA::BYTES, wave);
  };
  f32x16 acc[TI][TJ];
  clear_tiles(acc);
  int sa[TI] = {}, sb[TJ] = {};
  mma_loop<C, MmaF16, TA, TB>(nk1 * nseg, lds_raw, acc, sa, sb, wm, wn, lane, next, [](int) {});

  const int rbase = m0 + wm * TI * 32, cbase = n0 + wn * TJ * 32;
  float* const stage = (float*)lds_raw + wave * C::EPI_FLOATS;
  const NsPlace at = OP == NS_LAST ? d.table[g.first + mat] : NsPlace{0, 0};
  float step = 0.0f;
  if constexpr (OP == NS_LAST && std::is_same<IO, MuonIO>::value)
    step = io.lr * (io.rms > 0.0f ? io.rms * sqrtf((float)max(g.rows, g.cols)) : sqrtf(fmaxf(1.0f, (float)g.rows / (float)g.cols)));
  // a result that leaves
  auto emit = [&](int r, int c, float y) __attribute__((always_inline)) {
    const int64_t i = at.offset + r * at.ld + c;
    if constexpr (std::is_same<IO, MuonIO>::value) {
      const float w = io.decay * io.w[i] - step * y;
      io.w[i] = w;
      if (io.wl) io.wl[i] = (bf16)w;
    } else {
      if (io.bf) ((bf16*)io.y)[i] = (bf16)y; else ((float*)io.y)[i] = y;
    }
  };
#pragma unroll
  for (int i = 0; i < TI; ++i) {
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) stage[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * LDW + j * 32 + (lane & 31)] = acc[i][j][r];
#pragma unroll
    for (int it = 0; it < 32 * WN / 8 / 64; ++it) {      // 8 columns of a row per lane
      const int piece = it * 64 + lane, lr = piece / (WN / 8), lc = (piece % (WN / 8)) * 8;
      const int row = rbase + i * 32 + lr, col = cbase + lc;
      if (row >= m || col >= (SYM ? m : n)) continue;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = stage[lr * LDW + lc + k];
      f16x8 h, l;
      if (OP == NS_GRAM) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= kSa / (kSx * kSx);
      } else if (OP == NS_SQUARE) {
        const f16x8 ah = *(const f16x8*)(A + (int64_t)row * m + col);
        f16x8 al = {};
        if (d.split) al = *(const f16x8*)(A + (int64_t)m * m + (int64_t)row * m + col);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float s = d.b * (((float)ah[k] + (float)al[k]) * (1.0f / kSa)) + d.c * (x[k] * (1.0f / (kSa * kSa)));
          if (row == col + k) { diag[row] = s; x[k] = 0.0f; } else x[k] = s * kSs;
        }
      } else {
        const int64_t o = (int64_t)row * n + col;
        const f16x8 xh = *(const f16x8*)(X + o), xl = *(const f16x8*)(X + (int64_t)m * n + o);
        const float f = d.a + diag[row];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = f * ((float)xh[k] + (float)xl[k]) + x[k] * (1.0f / kSs);
      }
      if (OP == NS_LAST) {
        if (!g.tall) {
#pragma unroll
          for (int k = 0; k < 8; ++k) if (row < g.rows && col + k < g.cols) emit(row, col + k, x[k] * (1.0f / kSx));
        }
      } else {
        f16* const out = OP == NS_GRAM ? A : OP == NS_SQUARE ? Sm : Xn;
        const int ld = SYM ? m : n;
#pragma unroll
        for (int k = 0; k < 8; ++k) { h[k] = (f16)x[k]; l[k] = (f16)(x[k] - (float)h[k]); }
        *(f16x8*)(out + (int64_t)row * ld + col) = h;
        if (!SYM || d.split) *(f16x8*)(out + (int64_t)m * ld + (int64_t)row * ld + col) = l;
      }
      if (OP == NS_SQUARE || OP == NS_LAST) {      // what the transposed way out reads
#pragma unroll
        for (int k = 0; k < 8; ++k) stage[lr * LDW + lc + k] = x[k];
      }
    }
    if (SYM && ti != tj) {      // the mirror image: 8 rows of a column per lane
      f16* const out = OP == NS_GRAM ? A : Sm;
#pragma unroll
      for (int it = 0; it < 32 * WN / 8 / 64; ++it) {
        const int piece = it * 64 + lane, lc = piece % WN, lr = piece / WN * 8;
        const int row = rbase + i * 32 + lr, col = cbase + lc;
        if (row >= m || col >= m) continue;
        f16x8 h, l;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float x = stage[(lr + k) * LDW + lc];
          if (OP == NS_GRAM) x *= kSa / (kSx * kSx);
          h[k] = (f16)x; l[k] = (f16)(x - (float)h[k]);
        }
        *(f16x8*)(out + (int64_t)col * m + row) = h;
        if (d.split) *(f16x8*)(out + (int64_t)m * m + (int64_t)col * m + row) = l;
      }
    }
    if (OP == NS_LAST && g.tall) {
#pragma unroll
      for (int it = 0; it < 32 * WN / 8 / 64; ++it) {
        const int piece = it * 64 + lane, lc = piece % WN, lr = piece / WN * 8;
        const int row = rbase + i * 32 + lr, col = cbase + lc;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (row + k < g.cols && col < g.rows) emit(col, row + k, stage[(lr + k) * LDW + lc] * (1.0f / kSx));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

typedef DmaCfg<1, 1, 2, 2, 1, 64, 3, 3, true> Ns64;
typedef DmaCfg<2, 2, 2, 2, 1, 64, 2, 2, true> Ns128;

int64_t ns_tiles(const NsGroup& g, int op, int bm, int bn) {
  const int64_t nbm = (g.m + bm - 1) / bm, nbn = (g.n + bn - 1) / bn;
  return g.count * (op == NS_GRAM || op == NS_SQUARE ? nbm * (nbm + 1) / 2 : nbm * nbn);
}

template <class C, int OP, class IO>
hipError_t launch_product(NsDev d, const IO& io, hipStream_t s) {
  int64_t blocks = 0;
  for (int i = 0; i < d.ng; ++i) { d.first_block[i] = (int)blocks; blocks += ns_tiles(d.g[i], OP, C::BM, C::BN); }
  d.first_block[d.ng] = (int)blocks;
  auto kern = ns_product_kernel<C, OP, IO>;
  if (C::LDS > 48 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(C::NT), C::LDS, s, d, io);
  return hipGetLastError();
}
template <int OP, class IO>
hipError_t product(const NsDev& d, const IO& io, hipStream_t s) {
  int64_t t128 = 0;
  for (int i = 0; i < d.ng; ++i) t128 += ns_tiles(d.g[i], OP, 128, 128);
  return t128 >= 192 ? launch_product<Ns128, OP, IO>(d, io, s) : launch_product<Ns64, OP, IO>(d, io, s);
}

// The shapes of a list and the order of its matrices, shape by shape; the workspace is laid out as [table][partial sums][matrices].
struct NsPlan {
  std::vector<NsGroup> groups;
  std::vector<int> order;
  size_t table, partial, total;
};
NsPlan ns_plan(const hs_matrix* mats, int n, int split) {
  NsPlan p;
  p.order.resize(n);
  std::iota(p.order.begin(), p.order.end(), 0);
  std::stable_sort(p.order.begin(), p.order.end(), [&](int i, int j) {
    return mats[i].rows != mats[j].rows ? mats[i].rows > mats[j].rows : mats[i].cols > mats[j].cols;
  });
  p.table = 0;
  p.partial = align_up((size_t)n * sizeof(NsPlace), 256);
  size_t off = align_up(p.partial + (size_t)n * kParts * sizeof(double), 256);
  for (int i = 0; i < n;) {
    const hs_matrix& a = mats[p.order[i]];
    int j = i;
    while (j < n && mats[p.order[j]].rows == a.rows && mats[p.order[j]].cols == a.cols) ++j;
    NsGroup g;
    g.rows = a.rows; g.cols = a.cols; g.tall = a.rows > a.cols;
    g.m = (std::min(a.rows, a.cols) + 63) / 64 * 64; g.n = (std::max(a.rows, a.cols) + 63) / 64 * 64;
    g.count = j - i; g.first = i;
    g.parts = (int)std::min<int64_t>(kParts, ((int64_t)a.rows * a.cols + kPartElems - 1) / kPartElems);
    g.ws = (int64_t)off; g.stride = (int64_t)ns_parts(g.m, g.n, split).total;
    off += (size_t)g.stride * g.count;
    p.groups.push_back(g);
    i = j;
  }
  p.total = off;
  return p;
}

bool ns_list_ok(const hs_matrix* mats, int32_t n, std::string* why) {
  if (n < 0 || (n > 0 && !mats)) { *why = "negative number of matrices or no list"; return false; }
  for (int i = 0; i < n; ++i) {
    const hs_matrix& a = mats[i];
    if (a.rows < 1 || a.cols < 1 || a.offset < 0 || a.ld < a.cols || a.ld > ((int64_t)1 << 40) || a.offset > ((int64_t)1 << 60)) { *why = "a matrix without elements, with a negative offset or with rows that overlap"; return false; }
    const int64_t m = (std::min(a.rows, a.cols) + (int64_t)63) / 64 * 64, l = (std::max(a.rows, a.cols) + (int64_t)63) / 64 * 64;
    if (m * l > (int64_t)1 << 28) { *why = "a matrix of more than 2^28 elements (sides rounded up to 64)"; return false; }
  }
  return true;
}

// Whether two matrices of the list share an element: neighbours in the order of their offsets whose ranges meet may only be columns of one wider
// matrix (the same row stride, other columns).
bool ns_disjoint(const hs_matrix* mats, int n) {
  std::vector<int> order(n);
  std::iota(order.begin(), order.end(), 0);
  std::sort(order.begin(), order.end(), [&](int i, int j) { return mats[i].offset < mats[j].offset; });
  auto end = [&](const hs_matrix& a) { return a.offset + (a.rows - 1) * a.ld + a.cols; };
  std::vector<int> open;      // matrices that reach beyond the present offset
  for (int i : order) {
    const hs_matrix& b = mats[i];
    open.erase(std::remove_if(open.begin(), open.end(), [&](int k) { return end(mats[k]) <= b.offset; }), open.end());
    for (int k : open) {
      const hs_matrix& a = mats[k];
      if (a.ld != b.ld) return false;
      const int64_t shift = (b.offset - a.offset) % a.ld;      // b's first column, counted from a's
      if (shift < a.cols || shift + b.cols > a.ld) return false;
    }
    open.push_back(i);
  }
  return true;
}

const double kDefaultCoeff[3] = {3.4445, -4.7750, 2.0315};

template <class IO>
hs_status orthogonalize(const char* who, const IO& io, size_t size, const hs_matrix* mats, int32_t n, int32_t products, int32_t steps,
                        const double* coeff, double eps, void* workspace, size_t workspace_bytes, hipStream_t s) {
  const std::string name = std::string(who) + ": ";
  std::string why;
  if (products != HS_FP32 && products != HS_BF16) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "products must be HS_FP32 or HS_BF16");
  if (!ns_list_ok(mats, n, &why)) return hs_fail(nullptr, HS_ERR_SHAPE, name + why);
  if (steps < 1 || steps > 64) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "steps must be 1 .. 64");
  if (!(eps >= 0.0) || std::isinf(eps)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "eps must be finite and >= 0");
  for (int i = 0; coeff && i < 3 * steps; ++i)
    if (!std::isfinite(coeff[i])) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "a coefficient is not finite");
  if (n == 0) return HS_OK;
  for (int i = 0; i < n; ++i) {
    const hs_matrix& a = mats[i];
    if ((uint64_t)a.offset + (uint64_t)(a.rows - 1) * (uint64_t)a.ld + (uint64_t)a.cols > (uint64_t)size)
      return hs_fail(nullptr, HS_ERR_SHAPE, name + "a matrix reaches beyond the buffers");
  }
  if (!ns_disjoint(mats, n)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "two matrices share elements");
  const int split = products == HS_FP32;
  const NsPlan plan = ns_plan(mats, n, split);
  if (!workspace || workspace_bytes < plan.total) return hs_fail(nullptr, HS_ERR_WORKSPACE, name + "workspace smaller than hs_orthogonalize_workspace_bytes()");
  if ((uintptr_t)workspace % 256) return hs_fail(nullptr, HS_ERR_INVALID_ARG, name + "workspace must be 256-byte aligned");
  char* const ws = (char*)workspace;
  NsPlace* const table = (NsPlace*)(ws + plan.table);
  hipError_t e = hipSuccess;
  for (int done = 0; done < n && e == hipSuccess; done += 200) {
    TableArg t;
    t.first = done; t.n = std::min(200, n - done);
    for (int i = 0; i < t.n; ++i) t.place[i] = NsPlace{mats[plan.order[done + i]].offset, mats[plan.order[done + i]].ld};
    hipLaunchKernelGGL(ns_table_kernel, dim3(1), dim3(256), 0, s, t, table);
    e = hipGetLastError();
  }
  for (size_t g0 = 0; g0 < plan.groups.size() && e == hipSuccess; g0 += kGroups) {
    NsDev d{};
    d.ng = (int)std::min<size_t>(kGroups, plan.groups.size() - g0);
    for (int i = 0; i < d.ng; ++i) d.g[i] = plan.groups[g0 + i];
    d.split = split; d.ws = ws; d.table = table; d.partial = (double*)(ws + plan.partial); d.from = 0;
    auto blocks_of = [&](auto per) {
      int64_t blocks = 0;
      for (int i = 0; i < d.ng; ++i) { d.first_block[i] = (int)blocks; blocks += (int64_t)d.g[i].count * per(d.g[i]); }
      d.first_block[d.ng] = (int)blocks;
      return (unsigned)blocks;
    };
    unsigned blocks = blocks_of([](const NsGroup& g) { return g.parts; });
    hipLaunchKernelGGL(ns_norm_kernel<IO>, dim3(blocks), dim3(256), 0, s, d, io);
    blocks = blocks_of([](const NsGroup& g) { return (g.m / 64) * (g.n / 64); });
    hipLaunchKernelGGL(ns_start_kernel<IO>, dim3(blocks), dim3(256), 0, s, d, io, eps);
    e = hipGetLastError();
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
      const double* const c = coeff ? coeff + 3 * k : kDefaultCoeff;
      d.a = (float)c[0]; d.b = (float)c[1]; d.c = (float)c[2];
      e = product<NS_GRAM>(d, io, s);
      if (e == hipSuccess) e = product<NS_SQUARE>(d, io, s);
      if (e == hipSuccess) e = k + 1 < steps ? product<NS_APPLY>(d, io, s) : product<NS_LAST>(d, io, s);
      d.from ^= 1;
    }
  }
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, name + hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t hs_orthogonalize_workspace_bytes(const hs_matrix* mats, int32_t n, int32_t products) {
  std::string why;
  if ((products != HS_FP32 && products != HS_BF16) || !ns_list_ok(mats, n, &why)) {
    hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_orthogonalize_workspace_bytes: " + (why.empty() ? "products must be HS_FP32 or HS_BF16" : why));
    return 0;
  }
  return ns_plan(mats, n, products == HS_FP32).total;
}

hs_status hs_op_orthogonalize(int32_t dtype, const void* x, void* y, size_t size, const hs_matrix* mats, int32_t n, int32_t products, int32_t steps,
                              const double* coeff, double eps, void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != HS_FP32 && dtype != HS_BF16) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_orthogonalize: bad dtype");
  if (n > 0 && (!x || !y)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_orthogonalize: NULL buffer");
  if ((uintptr_t)x % 16 || (uintptr_t)y % 16) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_op_orthogonalize: buffers must be 16-byte aligned");
  return orthogonalize("hs_op_orthogonalize", PlainIO{x, y, dtype == HS_BF16}, size, mats, n, products, steps, coeff, eps, workspace, workspace_bytes,
                       (hipStream_t)stream);
}

hs_status hs_muon_step(float* w, float* m, const float* G, void* w_lowp_out, size_t size, const hs_matrix* mats, int32_t n, int32_t products,
                       double denom, double lr, double momentum, int32_t nesterov, double weight_decay, double rms, int32_t steps, const double* coeff,
                       double eps, void* workspace, size_t workspace_bytes, void* stream) {
  if (n > 0 && (!w || !m || !G)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_muon_step: NULL buffer");
  if ((uintptr_t)w % 16 || (uintptr_t)m % 16 || (uintptr_t)G % 16 || (uintptr_t)w_lowp_out % 8)
    return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_muon_step: buffers must be 16-byte aligned");
  if (!(denom >= 0.0) || std::isinf(denom)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_muon_step: denom must be finite and >= 0");
  if (!(momentum >= 0.0 && momentum < 1.0)) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_muon_step: momentum must be in [0, 1)");
  if (!std::isfinite(lr) || !std::isfinite(weight_decay) || !(rms >= 0.0) || std::isinf(rms))
    return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_muon_step: lr and weight_decay must be finite, rms finite and >= 0");
  const MuonIO io{w, m, G, (bf16*)w_lowp_out, (float)denom, (float)momentum, (float)(1.0 - lr * weight_decay), (float)lr, (float)rms, nesterov ? 1 : 0, 0};
  return orthogonalize("hs_muon_step", io, size, mats, n, products, steps, coeff, eps, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
