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
// of it and applied in 32 bits too.  Relative error of the result (2-norm, CPU emulation), step by step: Gaussian 768 x 768 8e-4, 512 x 512 of rank 32 with 2 % noise 8e-4; with
// X in one fp16 number and the diagonal left in 1.4e-3 and 2.4e-2; all in bf16 1.1e-2 and 1.9e-1.  Step by step and through polynomials of A: 256 x 1024 Gaussian 7e-4, 8e-4; of rank 64 with
// 5 % noise 1.9e-3, 3.1e-3; rank 1 with 2 % 2e-4, 2.6e-3 (why the second only goes with many rows: see kGramAlone).  32-bit products (HS_FP32) take the second numbers of both operands
// along: three products hi hi + hi lo + lo hi as one contraction three times as long, error as in fp32.
#include <algorithm>
#include <cmath>
#include <new>
#include <numeric>
#include <tuple>

#include "mma_tile.h"

namespace {

constexpr int kJobs = 16;             // jobs of one launch
constexpr int kParts = 256;           // partial sums of a matrix' norm, at most
constexpr int kPartElems = 4096;      // ... of so many elements at least (but the last)
constexpr float kSx = 256.0f;         // X is held times this

// The square matrices that a matrix has beside its X, each in fp16 with its diagonal apart in 32 bits, times the factor of its kind.
enum { BUF_A = 0, BUF_S, BUF_T, BUF_Q, BUF_Q2, BUFS };
__host__ __device__ constexpr float buf_scale(int b) { return b == BUF_A || b == BUF_T ? 4096.0f : b == BUF_S ? 1024.0f : 64.0f; }

// The ways of a matrix: products with X in every step; polynomials of A, X in every third (see kGramAlone); a launch per step for small ones (see
// ns_panel).
enum NsKind { NS_BY_STEP = 0, NS_BY_GRAM, NS_BY_PANEL };
// Matrices of one shape; `first` is the place of the first one in the table of offsets.
struct NsGroup {
  int rows, cols, m, n, tall, count, first, parts, bufs;
  int kind;                // NsKind: the way it goes
  int64_t ws, stride;      // bytes: first matrix' part of the workspace, and from one matrix to the next
};
// What a launch does to the matrices of a group.  Symmetric products: out = ident I + alpha P + beta P Q.
struct NsJob { NsGroup g; int p, q, out; float ident, alpha, beta; };
struct NsPlace { int64_t offset, ld; };      // a matrix in the flat buffers
struct NsDev {
  int n, split;            // jobs; split: 32-bit products
  int first_block[kJobs + 1];
  NsJob job[kJobs];
  char* ws;
  NsPlace* table;
  double* partial;         // [matrices][kParts]
  int from;                // which of the two X is read
};

// parts of a matrix' workspace: two X of two numbers each, the square matrices (of two numbers each for 32-bit products), their diagonals
__host__ __device__ inline size_t x_bytes(const NsGroup& g) { return (size_t)g.m * g.n * 4; }
__host__ __device__ inline size_t buf_bytes(const NsGroup& g, int split) { return (size_t)g.m * g.m * (split ? 4 : 2); }
__device__ __forceinline__ f16* buf_ptr(char* base, const NsGroup& g, int split, int b) { return (f16*)(base + 2 * x_bytes(g) + b * buf_bytes(g, split)); }
__device__ __forceinline__ float* diag_ptr(char* base, const NsGroup& g, int split, int b) {
  return (float*)(base + 2 * x_bytes(g) + g.bufs * buf_bytes(g, split)) + (int64_t)b * g.m;
}
constexpr int kPanel = 64;            // columns of X that a block of the panel kernel works on
__host__ __device__ inline size_t gram_floats(const NsGroup& g) { return (size_t)(g.n / kPanel) * g.m * g.m; }      // a step's partial A
size_t matrix_bytes(const NsGroup& g, int split) {
  if (g.kind == NS_BY_PANEL) return align_up(x_bytes(g) + 2 * gram_floats(g) * sizeof(float), 256);
  return align_up(2 * x_bytes(g) + g.bufs * (buf_bytes(g, split) + (size_t)g.m * sizeof(float)), 256);
}

// the job that thread block v works on
__device__ __forceinline__ int ns_job(const NsDev& d, int v) {
  int i = 0;
  while (i + 1 < d.n && v >= d.first_block[i + 1]) ++i;
  return i;
}

// The places travel as kernel arguments: those of short lists with the first pass, which writes them into the table for the launches behind it (a launch less: one
// matrix 130 x 67 71.1 -> 69.6 us, toy model 114.5 -> 113.1); those of longer ones with launches of their own.
template <int N>
struct Places { NsPlace place[N]; int first, n; };
typedef Places<200> TableArg;
typedef Places<100> ShortTable;
__global__ void ns_table_kernel(TableArg t, NsPlace* __restrict__ table) {
  const int i = threadIdx.x;
  if (i < t.n) table[t.first + i] = t.place[i];
}

// ---- where the matrices come from and go to ---------------------------------------------------------
// update: momentum and weights; otherwise a flat buffer of matrices in, another out
struct MuonIO {
  float *w, *m; const float* G; bf16* wl;
  float denom, mu, decay, lr, rms;      // denom 0: G as it is; decay = 1 - lr wd
  int nesterov;
};
struct PlainIO { const void* x; void* y; int bf; };

// Four neighbours of a row from element i on, `have` of which exist (whole: all, and i is a multiple of 4).
__device__ __forceinline__ float4 load4(const float* __restrict__ p, int64_t i, int have, bool whole) {
  if (whole) return *(const float4*)(p + i);
  return make_float4(have > 0 ? p[i] : 0.0f, have > 1 ? p[i + 1] : 0.0f, have > 2 ? p[i + 2] : 0.0f, have > 3 ? p[i + 3] : 0.0f);
}
__device__ __forceinline__ float4 gradient4(const MuonIO& io, int64_t i, int have, bool whole) {
  float4 g = load4(io.G, i, have, whole);
  if (io.denom > 0.0f) { g.x /= io.denom; g.y /= io.denom; g.z /= io.denom; g.w /= io.denom; }
  return g;
}
__device__ __forceinline__ float4 plain4(const PlainIO& io, int64_t i, int have, bool whole) {
  if (!io.bf) return load4((const float*)io.x, i, have, whole);
  const bf16* const p = (const bf16*)io.x;
  if (whole) {
    const bf16x4 v = *(const bf16x4*)(p + i);
    return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
  }
  return make_float4(have > 0 ? (float)p[i] : 0.0f, have > 1 ? (float)p[i + 1] : 0.0f, have > 2 ? (float)p[i + 2] : 0.0f, have > 3 ? (float)p[i + 3] : 0.0f);
}
__device__ __forceinline__ float axpy1(const MuonIO& io, float m, float g) { return io.nesterov ? g + io.mu * m : m; }

// what is orthogonalised, once the momentum is updated
__device__ __forceinline__ float4 source4(const MuonIO& io, int64_t i, int have, bool quads) {
  const bool whole = quads && have >= 4;
  const float4 m = load4(io.m, i, have, whole);
  if (!io.nesterov) return m;
  const float4 g = gradient4(io, i, have, whole);
  return make_float4(axpy1(io, m.x, g.x), axpy1(io, m.y, g.y), axpy1(io, m.z, g.z), axpy1(io, m.w, g.w));
}
__device__ __forceinline__ float4 source4(const PlainIO& io, int64_t i, int have, bool quads) { return plain4(io, i, have, quads && have >= 4); }

// lr s of the update
__device__ __forceinline__ float update_scale(const MuonIO& io, const NsGroup& g) {
  return io.lr * (io.rms > 0.0f ? io.rms * sqrtf((float)max(g.rows, g.cols)) : sqrtf(fmaxf(1.0f, (float)g.rows / (float)g.cols)));
}
__device__ __forceinline__ float update_scale(const PlainIO&, const NsGroup&) { return 0.0f; }
__device__ __forceinline__ void emit1(const MuonIO& io, int64_t i, float step, float y) {
  const float w = io.decay * io.w[i] - step * y;
  io.w[i] = w;
  if (io.wl) io.wl[i] = (bf16)w;
}
__device__ __forceinline__ void emit1(const PlainIO& io, int64_t i, float, float y) { if (io.bf) ((bf16*)io.y)[i] = (bf16)y; else ((float*)io.y)[i] = y; }
// four neighbours, `have` of which exist
__device__ __forceinline__ void emit4(const MuonIO& io, int64_t i, int have, bool quads, float step, const float (&y)[4]) {
  if (quads && have >= 4) {
    float4 w = *(const float4*)(io.w + i);
    w.x = io.decay * w.x - step * y[0]; w.y = io.decay * w.y - step * y[1]; w.z = io.decay * w.z - step * y[2]; w.w = io.decay * w.w - step * y[3];
    *(float4*)(io.w + i) = w;
    if (io.wl) *(bf16x4*)(io.wl + i) = bf16x4{(bf16)w.x, (bf16)w.y, (bf16)w.z, (bf16)w.w};
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < have) emit1(io, i + k, step, y[k]);
  }
}
__device__ __forceinline__ void emit4(const PlainIO& io, int64_t i, int have, bool quads, float, const float (&y)[4]) {
  if (quads && have >= 4) {
    if (io.bf) *(bf16x4*)((bf16*)io.y + i) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    else *(float4*)((float*)io.y + i) = make_float4(y[0], y[1], y[2], y[3]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < have) emit1(io, i + k, 0.0f, y[k]);
  }
}

// First pass: the momentum is updated, and the sum of squares of what is going to be orthogonalised is formed in 64 bits (gradients of 1e-25 have squares
// that 32 bits do not hold), a part of a matrix per block, added in a fixed order.  Memory bound: 12 bytes per element.
template <class IO>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsDev d, IO io, ShortTable t) {
  const int ji = ns_job(d, blockIdx.x);
  const NsGroup& g = d.job[ji].g;
  const int local = blockIdx.x - d.first_block[ji], mat = local / g.parts, part = local % g.parts;
  const NsPlace at = t.n > 0 ? t.place[g.first + mat] : d.table[g.first + mat];
  if (t.n > 0 && part == 0 && threadIdx.x == 0) d.table[g.first + mat] = at;
  // a matrix without gaps is one long row
  const bool flat = at.ld == g.cols;
  const int cols = flat ? g.rows * g.cols : g.cols, per_row = (cols + 3) / 4, total = (flat ? 1 : g.rows) * per_row;
  const int chunk = (total + g.parts - 1) / g.parts, end = min(total, (part + 1) * chunk);
  const bool quads = ((at.offset | (flat ? 0 : at.ld)) & 3) == 0;
  double sum = 0.0;
#pragma unroll 4
  for (int e = part * chunk + threadIdx.x; e < end; e += 256) {
    const int r = flat ? 0 : e / per_row, c = (e - r * per_row) * 4, have = cols - c;
    const int64_t i = at.offset + r * at.ld + c;
    const bool whole = quads && have >= 4;
    float4 u;
    if constexpr (std::is_same<IO, MuonIO>::value) {
      const float4 gr = gradient4(io, i, have, whole);
      float4 m = load4(io.m, i, have, whole);
      m.x = io.mu * m.x + gr.x; m.y = io.mu * m.y + gr.y; m.z = io.mu * m.z + gr.z; m.w = io.mu * m.w + gr.w;
      if (whole) {
        *(float4*)(io.m + i) = m;
      } else {
        io.m[i] = m.x;
        if (have > 1) io.m[i + 1] = m.y;
        if (have > 2) io.m[i + 2] = m.z;
        if (have > 3) io.m[i + 3] = m.w;
      }
      u = make_float4(axpy1(io, m.x, gr.x), axpy1(io, m.y, gr.y), axpy1(io, m.z, gr.z), axpy1(io, m.w, gr.w));
    } else {
      u = plain4(io, i, have, whole);
    }
    sum += ((double)u.x * (double)u.x + (double)u.y * (double)u.y) + ((double)u.z * (double)u.z + (double)u.w * (double)u.w);
  }
  __shared__ double red[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) d.partial[(int64_t)(g.first + mat) * kParts + part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// Second pass: X = U / (|U| + eps) in two fp16 numbers, the shorter side as rows, zeros in the padding.  64 x 64 elements per block, turned in LDS if the
// matrix is tall.  Memory bound: 12 bytes per element.
template <class IO>
__global__ __launch_bounds__(256) void ns_start_kernel(NsDev d, IO io, double eps) {
  const int ji = ns_job(d, blockIdx.x);
  const NsGroup& g = d.job[ji].g;
  const int nbn = g.n / 64, per = g.m / 64 * nbn, local = blockIdx.x - d.first_block[ji], mat = local / per, t = local % per;
  const int i0 = t / nbn * 64, j0 = t % nbn * 64;
  const NsPlace at = d.table[g.first + mat];
  __shared__ float tile[64][65];
  __shared__ double inv_s;
  const bool quads = ((at.offset | at.ld) & 3) == 0;
  const int r0 = g.tall ? j0 : i0, c0 = (g.tall ? i0 : j0) + (threadIdx.x & 15) * 4;
  float4 u[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + k * 16 + (threadIdx.x >> 4), have = r < g.rows ? g.cols - c0 : 0;
    const int64_t i = at.offset + r * at.ld + c0;
    u[k] = source4(io, i, have, quads);
  }
  if (threadIdx.x < 64) {
    double s = 0.0;
    for (int k = threadIdx.x; k < g.parts; k += 64) s += d.partial[(int64_t)(g.first + mat) * kParts + k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (threadIdx.x == 0) inv_s = s == 0.0 ? 0.0 : (double)kSx / (sqrt(s) + eps);      // a matrix of zeros stays one
  }
  __syncthreads();
  const double inv = inv_s;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int lr = k * 16 + (threadIdx.x >> 4), lc = (threadIdx.x & 15) * 4;
    const float x[4] = {(float)((double)u[k].x * inv), (float)((double)u[k].y * inv), (float)((double)u[k].z * inv), (float)((double)u[k].w * inv)};
#pragma unroll
    for (int c = 0; c < 4; ++c) if (g.tall) tile[lc + c][lr] = x[c]; else tile[lr][lc + c] = x[c];
  }
  __syncthreads();
  f16* const hi = (f16*)(d.ws + g.ws + mat * g.stride);
  f16* const lo = hi + (int64_t)g.m * g.n;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int e = k * 256 + threadIdx.x, r = e >> 3, c = (e & 7) * 8;
    f16x8 h, l;
#pragma unroll
    for (int q = 0; q < 8; ++q) { const float x = tile[r][c + q]; h[q] = (f16)x; l[q] = (f16)(x - (float)h[q]); }
    const int64_t o = (int64_t)(i0 + r) * g.n + j0 + c;
    *(f16x8*)(hi + o) = h;
    *(f16x8*)(lo + o) = l;
  }
}

// ---- the products ---------------------------------------------------------------------------------
enum { NS_GRAM = 0, NS_SYM, NS_APPLY, NS_LAST };

// the tile (row, column >= row) of number t of a symmetric matrix of nb x nb tiles
__device__ __forceinline__ void upper_tile(int t, int nb, int& ti, int& tj) {
  int r = (int)((2.0f * nb + 1.0f - sqrtf((2.0f * nb + 1.0f) * (2.0f * nb + 1.0f) - 8.0f * t)) * 0.5f);
  r = max(0, min(r, nb - 1));
  while (r > 0 && r * nb - r * (r - 1) / 2 > t) --r;
  while ((r + 1) * nb - (r + 1) * r / 2 <= t) ++r;
  ti = r; tj = r + t - (r * nb - r * (r - 1) / 2);
}

__device__ __forceinline__ void to_f8(const f16x8& h, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = (float)h[k];
}

// GRAM: A = X X^T.  SYM: products of square matrices that commute (polynomials of A), whose diagonals are kept apart: with P = D + E and Q = D' + E' the
// matrix instruction forms E E', and D E' + E D' + D D' are added on the way out.  Both are symmetric: tiles on and above the diagonal only, each
// written in its place and mirrored.  APPLY: X <- (D + E) X, where X is read in 16 bits by the product with E and in full by D X.  LAST: the same on its way out.
// LDS in bytes: a wave's on the way out, and a block's.
template <class C, int OP, bool SPLIT>
constexpr int ns_wave_bytes() { return C::EPI_FLOATS * 4 + (OP == NS_GRAM || OP == NS_SYM ? (SPLIT ? 2 : 1) * 32 * (32 * C::TJ + 8) * 2 : 0); }
template <class C, int OP, bool SPLIT>
constexpr size_t ns_lds() { return std::max(C::KW * C::PIPE, (size_t)C::NS * ns_wave_bytes<C, OP, SPLIT>()); }      // KW > 1: a ring per wave

template <class C, int OP, bool SPLIT, class IO>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(C::WPE, C::WPE)))
void ns_product_kernel(NsDev d, IO io) {
  constexpr int TI = C::TI, TJ = C::TJ, WN = 32 * TJ, LDW = WN + 4, NIT = 32 * WN / 8 / 64;
  constexpr bool SYMM = OP == NS_GRAM || OP == NS_SYM;
  constexpr bool UPDATE = OP == NS_LAST && std::is_same<IO, MuonIO>::value;
  constexpr bool KSPLIT = C::KW > 1;      // the waves split the contraction (ks_loop)
  typedef DmaTile<true, C::BK, C::BM, C::NS> TA;
  typedef DmaTile<SYMM, C::BK, C::BN, C::NS> TB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = KSPLIT ? 0 : wave / C::WGN, wn = KSPLIT ? 0 : wave % C::WGN, lw = KSPLIT ? 0 : wave;
  const int ji = ns_job(d, blockIdx.x);
  const NsJob& job = d.job[ji];
  const NsGroup& g = job.g;
  const int m = g.m, n = g.n, nbm = (m + C::BM - 1) / C::BM, nbn = (n + C::BN - 1) / C::BN;
  // An XCD gets a contiguous range of the tiles of every job: of all of them together, the long contractions of one job would all be on a few XCDs.
  int local = blockIdx.x - d.first_block[ji];
  const int per_xcd = (d.first_block[ji + 1] - d.first_block[ji]) >> 3;
  if (local < 8 * per_xcd) local = (local & 7) * per_xcd + (local >> 3);
  const int per = SYMM ? nbm * (nbm + 1) / 2 : nbm * nbn, mat = local / per, t = local % per;
  int ti, tj;
  if (SYMM) upper_tile(t, nbm, ti, tj);
  else tile_of_block<4>(t, nbn, nbm, ti, tj);
  ti = __builtin_amdgcn_readfirstlane(ti); tj = __builtin_amdgcn_readfirstlane(tj);
  const int m0 = ti * C::BM, n0 = tj * C::BN;
  constexpr int split = SPLIT ? 1 : 0;
  char* const base = d.ws + g.ws + mat * g.stride;
  f16* const X = (f16*)(base + d.from * x_bytes(g));
  f16* const Xn = (f16*)(base + (d.from ^ 1) * x_bytes(g));

  // operands, and how far behind the first numbers the second ones are (bytes)
  const f16* const opA = OP == NS_GRAM ? X : buf_ptr(base, g, split, job.p);
  const f16* const opB = OP == NS_SYM ? buf_ptr(base, g, split, job.q) : X;
  const int K = OP == NS_GRAM ? n : m;
  const int64_t sizeA = (int64_t)m * K * 2, sizeB = OP == NS_SYM ? sizeA : (int64_t)m * n * 2;
  const int nk1 = K / 64, nseg = split ? 3 : 1;
  typename TA::Cursor ca;
  typename TB::Cursor cb;
  TA::init(ca, (const bf16*)opA, K, m0, m, 0, K, lane, lw);
  if (SYMM) TB::init(cb, (const bf16*)opB, K, n0, m, 0, K, lane, lw);
  else TB::init(cb, (const bf16*)opB, n, n0, n, 0, K, lane, lw);
  ca.rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)opA, 0, (int)(split ? 2 * sizeA : sizeA), 0x00020000);
  cb.rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)opB, 0, (int)(split ? 2 * sizeB : sizeB), 0x00020000);
  // k-tiles of the products hi hi, hi lo, lo hi one behind the other; then behind the operands
  auto from = [&](int seg, int kt) __attribute__((always_inline)) {
    ca.soff = seg >= nseg ? 0x80000000u : (seg == 2 ? (unsigned)sizeA : 0u) + kt * ca.step;
    cb.soff = seg >= nseg ? 0x80000000u : (seg == 1 ? (unsigned)sizeB : 0u) + kt * cb.step;
  };
  // Way out: a wave's 32-row slabs go through LDS, from where a lane takes 8 columns of a row (the same columns in every slab).  What a slab needs from memory is
  // requested while the one before it is worked on.  The mirror image comes out of a second copy of the slab, of the fp16 numbers that were
  // written, by transposing reads: 16 lanes get 16 columns, each 8 rows of one (and the four groups of 16 lanes the 32 rows).
  const int rbase = m0 + wm * TI * 32, cbase = n0 + wn * TJ * 32;
  const int ldo = SYMM ? m : n;                                     // of what is written, and of what it is added to
  const bool inside = rbase + 32 * TI <= m && cbase + WN <= ldo;    // sides are multiples of 64, so a slab of 8 is in or out as a whole
  constexpr int LDH = WN + 8;                                       // of the copy, in fp16 numbers
  float* const stage = (float*)(lds_raw + lw * ns_wave_bytes<C, OP, SPLIT>());
  f16* const half = (f16*)(stage + C::EPI_FLOATS);
  const bool mirror = SYMM && ti != tj;
  f16* const out = SYMM ? buf_ptr(base, g, split, job.out) : Xn;
  const int64_t lo_at = (int64_t)m * ldo;                           // second numbers
  float* const dout = SYMM ? diag_ptr(base, g, split, job.out) : nullptr;
  const float* const dp = OP == NS_GRAM ? nullptr : diag_ptr(base, g, split, job.p);
  const f16* const auxp = OP == NS_SYM ? opA : X;
  const f16* const auxq = opB;
  const bool same = OP == NS_SYM && job.p == job.q;
  const float f_out = SYMM ? buf_scale(job.out) : OP == NS_LAST ? 1.0f / kSx : 1.0f;
  const float f_acc = f_out * (OP == NS_GRAM ? 1.0f / (kSx * kSx) : OP == NS_SYM ? job.beta / (buf_scale(job.p) * buf_scale(job.q)) : 1.0f / buf_scale(job.p));
  // SYM, off the diagonal: out = f_acc acc + (rp + cp[column]) E_P + rq(row) E_Q, where for P = Q both go to E_P
  const float f_p = OP == NS_SYM ? f_out / buf_scale(job.p) : 0.0f, f_q = OP == NS_SYM ? f_out / buf_scale(job.q) : 0.0f;
  const int lane_col = cbase + (lane % (WN / 8)) * 8;
  float cp[8];
  if (OP == NS_SYM) {
    const float* const dq = diag_ptr(base, g, split, job.q);
#pragma unroll
    for (int k = 0; k < 8; ++k) cp[k] = lane_col < m ? f_p * (job.alpha + job.beta * dq[lane_col + k]) : 0.0f;
  }
  const NsPlace at = OP == NS_LAST ? d.table[g.first + mat] : NsPlace{0, 0};
  const bool quads = ((at.offset | at.ld) & 3) == 0;                // rows of the flat buffers start on 16 bytes
  float step = 0.0f;
  if constexpr (UPDATE) step = update_scale(io, g);

  // 8 neighbours of a row of the flat buffers, `have` of which exist; w: their weights, loaded before
  auto load_w = [&](int64_t i, bool whole, float (&w)[8]) __attribute__((always_inline)) {
    if constexpr (UPDATE) {
      if (whole) {
        const float4 a = *(const float4*)(io.w + i), b = *(const float4*)(io.w + i + 4);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
      }
    }
  };
  auto emit = [&](int64_t i, int have, bool whole, float (&w)[8], const float (&y)[8]) __attribute__((always_inline)) {
    if constexpr (UPDATE) {
      if (whole) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = io.decay * w[k] - step * y[k];
        *(float4*)(io.w + i) = make_float4(w[0], w[1], w[2], w[3]);
        *(float4*)(io.w + i + 4) = make_float4(w[4], w[5], w[6], w[7]);
        if (io.wl) {
          bf16x4 a, b;
#pragma unroll
          for (int k = 0; k < 4; ++k) { a[k] = (bf16)w[k]; b[k] = (bf16)w[k + 4]; }
          *(bf16x4*)(io.wl + i) = a;
          *(bf16x4*)(io.wl + i + 4) = b;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (k < have) emit1(io, i + k, step, y[k]);
      }
    } else if constexpr (OP == NS_LAST) {
      const float a[4] = {y[0], y[1], y[2], y[3]}, b[4] = {y[4], y[5], y[6], y[7]};
      emit4(io, i, have, whole, 0.0f, a);
      emit4(io, i + 4, have - 4, whole, 0.0f, b);
    }
  };

  auto place = [&](int it, int& lr, int& lc) __attribute__((always_inline)) {
    const int piece = it * 64 + lane;
    lr = piece / (WN / 8); lc = (piece % (WN / 8)) * 8;
  };
  auto place_t = [&](int it, int& lr, int& lc) __attribute__((always_inline)) {      // a tall matrix' way out: row group, column
    const int piece = it * 64 + lane;
    lr = (piece & 3) * 8; lc = piece >> 2;
  };
  // where 8 values go in the flat buffers, and how many of them there are
  auto target = [&](int i, int lr, int lc, int64_t& o, int& have) __attribute__((always_inline)) {
    const int row = rbase + i * 32 + lr, col = cbase + lc;
    if (g.tall) { o = at.offset + (int64_t)col * at.ld + row; have = col < g.rows ? g.cols - row : 0; }
    else { o = at.offset + (int64_t)row * at.ld + col; have = row < g.rows ? g.cols - col : 0; }
  };
  struct Aux { f16x8 p[NIT], pl[NIT], q[NIT], ql[NIT]; float d[NIT], dq[NIT], w[OP == NS_LAST ? NIT : 1][8]; };
  auto request = [&](auto all_tag, Aux& a, int i) __attribute__((always_inline)) {
    constexpr bool ALL = decltype(all_tag)::value;      // no piece is outside
    if (OP != NS_GRAM) {
#pragma unroll
      for (int it = 0; it < NIT; ++it) {
        int lr, lc;
        place(it, lr, lc);
        const int row = rbase + i * 32 + lr, col = cbase + lc;
        if (!ALL && (row >= m || col >= ldo)) continue;
        const int64_t o = (int64_t)row * ldo + col;
        a.p[it] = *(const f16x8*)(auxp + o);
        if (!SYMM || SPLIT) a.pl[it] = *(const f16x8*)(auxp + lo_at + o);
        if (OP == NS_SYM && !same) {
          a.q[it] = *(const f16x8*)(auxq + o);
          if (SPLIT) a.ql[it] = *(const f16x8*)(auxq + lo_at + o);
        }
        a.d[it] = dp[row];
        if (OP == NS_SYM) a.dq[it] = diag_ptr(base, g, split, job.q)[row];
      }
    }
    if constexpr (OP == NS_LAST) {
#pragma unroll
      for (int it = 0; it < NIT; ++it) {
        int lr, lc, have;
        int64_t o;
        if (g.tall) place_t(it, lr, lc); else place(it, lr, lc);
        target(i, lr, lc, o, have);
        load_w(o, quads && have >= 8, a.w[it]);
      }
    }
  };
  constexpr bool EARLY = !(UPDATE && TI > 2) && !(OP == NS_SYM && SPLIT);      // room in registers for two slabs' requests
  Aux aux[EARLY ? 2 : 1];

  f32x16 acc[TI][TJ];
  clear_tiles(acc);
  int seg = 0;
  if constexpr (KSPLIT) {
    int kt = wave;
    auto next = [&](unsigned char* dst) __attribute__((always_inline)) {
      while (kt >= nk1 && seg < nseg) { kt -= nk1; ++seg; }
      from(seg, kt);
      kt += C::KW;
      TA::issue(ca, dst, 0);
      TB::issue(cb, dst + TA::BYTES, 0);
    };
    const int nk = nk1 * nseg;
    ks_loop<MmaF16, TA, TB, C::KW, C::S>(nk > wave ? (nk - wave + C::KW - 1) / C::KW : 0, lds_raw, acc[0][0], lane, wave, next);
    if (wave > 0) return;
  } else {
    int kt = 0;
    auto next = [&](unsigned char* dst) __attribute__((always_inline)) {
      if (kt == nk1) { kt = 0; from(++seg, 0); }
      ++kt;
      TA::issue(ca, dst, wave);
      TB::issue(cb, dst + TA::BYTES, wave);
    };
    int sa[TI] = {}, sb[TJ] = {};      // no scales
    mma_loop<C, MmaF16, TA, TB>(nk1 * nseg, lds_raw, acc, sa, sb, wm, wn, lane, next, [](int) {});
  }

  auto flow = [&](auto all_tag) __attribute__((always_inline)) {
    constexpr bool ALL = decltype(all_tag)::value;
    auto slab = [&](Aux& a, int i) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) stage[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * LDW + j * 32 + (lane & 31)] = acc[i][j][r];
#pragma unroll
      for (int it = 0; it < NIT; ++it) {
        int lr, lc;
        place(it, lr, lc);
        const int row = rbase + i * 32 + lr, col = cbase + lc;
        if (!ALL && (row >= m || col >= ldo)) continue;
        const int64_t o = (int64_t)row * ldo + col;
        float* const st = stage + lr * LDW + lc;
        const float4 s0 = *(const float4*)st, s1 = *(const float4*)(st + 4);
        const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
        float x[8];
        if (OP == NS_GRAM) {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = s[k] * f_acc;
        } else if (OP == NS_SYM) {
          const float rq = job.beta * a.d[it];
          const float rp = same ? rq * f_p : 0.0f;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float e = (float)a.p[it][k];
            if (SPLIT) e += (float)a.pl[it][k];
            x[k] = s[k] * f_acc + (cp[k] + rp) * e;
          }
          if (!same) {
            const float f = rq * f_q;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float e = (float)a.q[it][k];
              if (SPLIT) e += (float)a.ql[it][k];
              x[k] += f * e;
            }
          }
        } else {
          const float f = a.d[it] * f_out;
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = f * ((float)a.p[it][k] + (float)a.pl[it][k]) + s[k] * f_acc;
        }
        if (SYMM && row / 8 == col / 8) {      // the diagonal goes apart
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (row == col + k) {
              if (OP == NS_GRAM) dout[row] = x[k] * (1.0f / f_out);
              else dout[row] = job.ident + job.alpha * a.d[it] + job.beta * a.d[it] * a.dq[it] + s[k] * (f_acc / f_out);
              x[k] = 0.0f;
            }
        }
        if (OP == NS_LAST) {
          if (!g.tall) {
            int64_t to;
            int have;
            target(i, lr, lc, to, have);
            emit(to, have, quads && have >= 8, a.w[OP == NS_LAST ? it : 0], x);
          } else {
            *(float4*)st = make_float4(x[0], x[1], x[2], x[3]);
            *(float4*)(st + 4) = make_float4(x[4], x[5], x[6], x[7]);
          }
        } else {
          f16x8 h;
#pragma unroll
          for (int k = 0; k < 8; ++k) h[k] = (f16)x[k];
          *(f16x8*)(out + o) = h;
          if (mirror) *(f16x8*)(half + lr * LDH + lc) = h;
          if (!SYMM || SPLIT) {
            f16x8 l;
#pragma unroll
            for (int k = 0; k < 8; ++k) l[k] = (f16)(x[k] - (float)h[k]);
            *(f16x8*)(out + lo_at + o) = l;
            if (mirror) *(f16x8*)(half + (32 + lr) * LDH + lc) = l;
          }
        }
      }
      if (mirror) {
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          const int lr = (lane >> 4) * 8, row = rbase + i * 32 + lr, col = cbase + it * 16 + (lane & 15);
          if (!ALL && (row >= m || cbase + it * 16 >= m)) continue;
          typedef s16x4 __attribute__((address_space(3))) * lds_v4;
          const f16* const src = half + (lr + ((lane & 15) >> 2)) * LDH + it * 16 + 4 * (lane & 3);
#pragma unroll
          for (int part = 0; part < (SPLIT ? 2 : 1); ++part) {
            union { struct { s16x4 a, b; } p; f16x8 v; } u;
            u.p.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(src + part * 32 * LDH));
            u.p.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(src + part * 32 * LDH + 4 * LDH));
            *(f16x8*)(out + part * lo_at + (int64_t)col * m + row) = u.v;
          }
        }
      }
      if constexpr (OP == NS_LAST) {
        if (g.tall) {
#pragma unroll
          for (int it = 0; it < NIT; ++it) {
            int lr, lc, have;
            int64_t o;
            place_t(it, lr, lc);
            target(i, lr, lc, o, have);
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = stage[(lr + k) * LDW + lc];
            emit(o, have, quads && have >= 8, a.w[it], x);
          }
        }
      }
    };
    if (EARLY) request(all_tag, aux[0], 0);
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if (EARLY) { if (i + 1 < TI) request(all_tag, aux[EARLY ? (i + 1) & 1 : 0], i + 1); }
      else request(all_tag, aux[0], i);
      slab(aux[EARLY ? i & 1 : 0], i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (inside) flow(std::true_type{}); else flow(std::false_type{});
}

// ---- small matrices ---------------------------------------------------------------------------------
// With up to 128 rows all of A and S fits the LDS of a CU, and S takes it less time than a launch: every block forms S for itself and applies it to 64 columns
// of X, which it then multiplies with themselves for its part of the next A.  One launch per step instead of three, rows padded to multiples of 32; the
// blocks of a matrix add up each other's parts of A in their order.  What bounds it is latency, 7 us a step with 64 rows, 10 with 96 and 13 to 18 with 128: one block of 512 threads
// per CU.  Which lists go this way: ns_small.
enum { PANEL_FIRST = 0, PANEL_STEP, PANEL_LAST };
constexpr int kPanelThreads = 512, kPanelM = 128;
constexpr int kLdS = kPanelM + 8, kLdX = kPanel + 8;      // of S and X in LDS, in fp16 numbers
template <bool SPLIT>
constexpr size_t panel_lds() { return (size_t)(SPLIT ? 2 : 1) * kPanelM * kLdS * 2 + 2 * (size_t)kPanelM * kLdX * 2 + 2 * kPanelM * sizeof(float); }

// 32 x 32 of the sum over k < K of P[row, k] Q[k, column]: P at its row, k contiguous; Q at its column, k contiguous (KMAJ) or columns contiguous
template <bool SPLIT, bool KMAJ, int K>
__device__ __forceinline__ void panel_product(f32x16& acc, const f16* p, int ldp, int lop, const f16* q, int ldq, int loq, int lane) {
  typedef s16x4 __attribute__((address_space(3))) * lds_v4;
  const int h = lane >> 5;
  auto rows = [&](const f16* b, int ld, int k) __attribute__((always_inline)) { return *(const f16x8*)(b + (lane & 31) * ld + k + 8 * h); };
  auto cols = [&](const f16* b, int ld, int k) __attribute__((always_inline)) {      // the transposing read of DmaTile::frag
    const f16* const at = b + (k + 8 * h + ((lane & 15) >> 2)) * ld + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    union { struct { s16x4 lo, hi; } v; f16x8 f; } u;
    u.v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)at);
    u.v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(at + 4 * ld));
    return u.f;
  };
#pragma unroll
  for (int k = 0; k < K; k += 16) {
    const f16x8 ph = rows(p, ldp, k), qh = KMAJ ? rows(q, ldq, k) : cols(q, ldq, k);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
    if (SPLIT) {
      const f16x8 pl = rows(p + lop, ldp, k), ql = KMAJ ? rows(q + loq, ldq, k) : cols(q + loq, ldq, k);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
    }
  }
}

template <bool SPLIT, int MODE, int M, class IO>
__device__ __forceinline__ void ns_panel(const NsDev& d, const IO& io, double eps, const NsJob& job, int local, unsigned char* lds_raw, double* inv_s) {
  constexpr int kLoS = kPanelM * kLdS, kLoX = kPanelM * kLdX;      // second numbers
  f16* const sS = (f16*)lds_raw;                                   // E of A, then of S
  f16* const sX = sS + (SPLIT ? 2 : 1) * kLoS;
  float* const sD = (float*)(sX + 2 * kLoX);                       // diagonal of A; of S behind it
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const NsGroup& g = job.g;
  constexpr int m = M, mt = M / 32, TILES = mt * mt, TPW = (TILES + 7) / 8;      // 32 x 32 tiles of a square matrix, and per wave
  const int n = g.n, panels = n / kPanel, mat = local / panels, j0 = local % panels * kPanel;
  char* const base = d.ws + g.ws + mat * g.stride;
  f16* const X = (f16*)base;
  const int64_t lo_at = (int64_t)m * n;
  float* const gram = (float*)(base + x_bytes(g));
  const float* const old = gram + d.from * gram_floats(g);
  float* const now = gram + (d.from ^ 1) * gram_floats(g) + (int64_t)(j0 / kPanel) * m * m;
  const NsPlace at = MODE == PANEL_STEP ? NsPlace{0, 0} : d.table[g.first + mat];
  const bool quads = ((at.offset | at.ld) & 3) == 0;
  // rows and columns of a result tile that a lane holds: 4 rows from row(r) on in register 4 r .. 4 r + 3, one column
  auto row = [&](int r) __attribute__((always_inline)) { return 8 * r + 4 * (lane >> 5); };
  const int col = lane & 31;

  if constexpr (MODE == PANEL_FIRST) {
    if (tid < 64) {
      double s = 0.0;
      for (int k = tid; k < g.parts; k += 64) s += d.partial[(int64_t)(g.first + mat) * kParts + k];
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
      if (tid == 0) *inv_s = s == 0.0 ? 0.0 : (double)kSx / (sqrt(s) + eps);      // a matrix of zeros stays one
    }
    // four neighbours of a row of the matrix: of X's row, or of its column where the matrix is tall
    const int per_row = (g.tall ? m : kPanel) / 4, total = m * kPanel / 4;
    float4 u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = tid + k * kPanelThreads, lr = e / per_row, lc = (e % per_row) * 4;
      const int r = g.tall ? j0 + lr : lr, c = g.tall ? lc : j0 + lc;
      u[k] = source4(io, at.offset + (int64_t)r * at.ld + c, e < total && r < g.rows ? g.cols - c : 0, quads);
    }
    __syncthreads();
    const double inv = *inv_s;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = tid + k * kPanelThreads, lr = e / per_row, lc = (e % per_row) * 4;
      if (e >= total) break;
      const float x[4] = {(float)((double)u[k].x * inv), (float)((double)u[k].y * inv), (float)((double)u[k].z * inv), (float)((double)u[k].w * inv)};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        f16* const o = g.tall ? sX + (lc + c) * kLdX + lr : sX + lr * kLdX + lc + c;
        const f16 h = (f16)x[c];
        o[0] = h; o[kLoX] = (f16)(x[c] - (float)h);
      }
    }
  } else {
    // X of the panel, and A: the sum of the blocks' parts
    for (int e = tid; e < m * kPanel / 8; e += kPanelThreads) {
      const int r = e / (kPanel / 8), c = (e % (kPanel / 8)) * 8;
      const f16* const src = X + (int64_t)r * n + j0 + c;
      *(f16x8*)(sX + r * kLdX + c) = *(const f16x8*)src;
      *(f16x8*)(sX + kLoX + r * kLdX + c) = *(const f16x8*)(src + lo_at);
    }
    // (several parts in flight at once: read one after the other they cost 2 us each)
    constexpr int QUADS = M * M / 4, NQ = (QUADS + kPanelThreads - 1) / kPanelThreads, AHEAD = 32 / NQ > 8 ? 8 : 32 / NQ;      // of a thread; parts in flight
    float4 a[NQ];
#pragma unroll
    for (int k = 0; k < NQ; ++k) a[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4* const src = (const float4*)old;
    for (int p = 0; p < panels; p += AHEAD) {
      float4 v[AHEAD][NQ];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
#pragma unroll
        for (int k = 0; k < NQ; ++k) v[q][k] = src[(int64_t)min(p + q, panels - 1) * QUADS + min(tid + k * kPanelThreads, QUADS - 1)];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        if (p + q < panels) {
#pragma unroll
          for (int k = 0; k < NQ; ++k) { a[k].x += v[q][k].x; a[k].y += v[q][k].y; a[k].z += v[q][k].z; a[k].w += v[q][k].w; }
        }
    }
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      const int e = tid + k * kPanelThreads, r = e / (M / 4), c = (e % (M / 4)) * 4;
      if (e >= QUADS) break;
      const float x[4] = {a[k].x, a[k].y, a[k].z, a[k].w};
      f16x4 h, l;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (r == c + t) sD[r] = x[t] * (1.0f / buf_scale(BUF_A));
        const float v = r == c + t ? 0.0f : x[t];
        h[t] = (f16)v; l[t] = (f16)(v - (float)h[t]);
      }
      *(f16x4*)(sS + r * kLdS + c) = h;
      if (SPLIT) *(f16x4*)(sS + kLoS + r * kLdS + c) = l;
    }
    __syncthreads();

    // S = a I + b A + c A A with the diagonals apart, as in ns_product_kernel; up to two tiles per wave
    f32x16 s[TPW];
    float sd[TPW];      // a diagonal element that this lane has
#pragma unroll
    for (int q = 0; q < TPW; ++q) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[q][r] = 0.0f;
      const int id = wave + 8 * q;
      if (id >= TILES) continue;
      const int ti = id / mt * 32, tj = id % mt * 32;
      panel_product<SPLIT, true, M>(s[q], sS + ti * kLdS, kLdS, kLoS, sS + tj * kLdS, kLdS, kLoS, lane);
      const float dc = sD[tj + col];
#pragma unroll
      for (int r = 0; r < 4; ++r) {      // A is symmetric: four elements of a column are read as four of a row
        const int i0 = ti + row(r), j = tj + col;
        const f16x4 eh = *(const f16x4*)(sS + j * kLdS + i0);
        f16x4 el = {};
        if (SPLIT) el = *(const f16x4*)(sS + kLoS + j * kLdS + i0);
        const float4 d4 = *(const float4*)(sD + i0);
        const float dr[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float e = ((float)eh[t] + (float)el[t]) * (1.0f / buf_scale(BUF_A)), prod = s[q][4 * r + t] * (1.0f / (buf_scale(BUF_A) * buf_scale(BUF_A)));
          if (i0 + t == j) { sd[q] = job.ident + job.alpha * dr[t] + job.beta * (prod + dr[t] * dr[t]); s[q][4 * r + t] = 0.0f; }
          else s[q][4 * r + t] = (job.alpha * e + job.beta * (prod + (dr[t] + dc) * e)) * buf_scale(BUF_S);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TPW; ++q) {
      const int id = wave + 8 * q;
      if (id >= TILES) continue;
      const int ti = id / mt * 32, tj = id % mt * 32;
#pragma unroll
      for (int r = 0; r < 4; ++r) {      // symmetric: written as column tj + col's four neighbours
        f16x4 h, l;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float v = s[q][4 * r + t];
          h[t] = (f16)v; l[t] = (f16)(v - (float)h[t]);
          if (ti + row(r) + t == tj + col) sD[kPanelM + tj + col] = sd[q];
        }
        f16* const o = sS + (tj + col) * kLdS + ti + row(r);
        *(f16x4*)o = h;
        if (SPLIT) *(f16x4*)(o + kLoS) = l;
      }
    }
    __syncthreads();

    // X <- (D + E) X; a tile per wave
    f32x16 x;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.0f;
    const int ti = wave / 2 * 32, tj = wave % 2 * 32;
    if (ti < m) {
      panel_product<SPLIT, false, M>(x, sS + ti * kLdS, kLdS, kLoS, sX + tj, kLdX, kLoX, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = ti + row(r >> 2) + (r & 3);
        const f16* const o = sX + i * kLdX + tj + col;
        x[r] = sD[kPanelM + i] * ((float)o[0] + (float)o[kLoX]) + x[r] * (1.0f / buf_scale(BUF_S));
      }
    }
    if constexpr (MODE == PANEL_LAST) {
      if (ti < m) {
        const float step = update_scale(io, g);
        const int j = j0 + tj + col;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = ti + row(r);
          const float y[4] = {x[4 * r] * (1.0f / kSx), x[4 * r + 1] * (1.0f / kSx), x[4 * r + 2] * (1.0f / kSx), x[4 * r + 3] * (1.0f / kSx)};
          if (g.tall) {
            if (j < g.rows) emit4(io, at.offset + (int64_t)j * at.ld + i, g.cols - i, quads, step, y);
          } else if (j < g.cols) {
#pragma unroll
            for (int t = 0; t < 4; ++t) if (i + t < g.rows) emit1(io, at.offset + (int64_t)(i + t) * at.ld + j, step, y[t]);
          }
        }
      }
      return;
    }
    __syncthreads();
    if (ti < m) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        f16* const o = sX + (ti + row(r >> 2) + (r & 3)) * kLdX + tj + col;
        const f16 h = (f16)x[r];
        o[0] = h; o[kLoX] = (f16)(x[r] - (float)h);
      }
    }
  }
  if constexpr (MODE != PANEL_LAST) {
    __syncthreads();
    for (int e = tid; e < m * kPanel / 8; e += kPanelThreads) {
      const int r = e / (kPanel / 8), c = (e % (kPanel / 8)) * 8;
      f16* const o = X + (int64_t)r * n + j0 + c;
      *(f16x8*)o = *(const f16x8*)(sX + r * kLdX + c);
      *(f16x8*)(o + lo_at) = *(const f16x8*)(sX + kLoX + r * kLdX + c);
    }
    // this panel's part of the next A
#pragma unroll
    for (int q = 0; q < TPW; ++q) {
      const int id = wave + 8 * q;
      if (id >= TILES) continue;
      const int ti = id / mt * 32, tj = id % mt * 32;
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.0f;
      panel_product<SPLIT, true, kPanel>(s, sX + ti * kLdX, kLdX, kLoX, sX + tj * kLdX, kLdX, kLoX, lane);
      constexpr float f = buf_scale(BUF_A) / (kSx * kSx);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(float4*)(now + (int64_t)(tj + col) * m + ti + row(r)) = make_float4(s[4 * r] * f, s[4 * r + 1] * f, s[4 * r + 2] * f, s[4 * r + 3] * f);
    }
  }
}

template <bool SPLIT, int MODE, class IO>
__global__ __launch_bounds__(kPanelThreads) void ns_panel_kernel(NsDev d, IO io, double eps) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  __shared__ double inv_s;
  const int ji = ns_job(d, blockIdx.x), local = blockIdx.x - d.first_block[ji];
  const NsJob& job = d.job[ji];
  switch (job.g.m) {
    case 32: ns_panel<SPLIT, MODE, 32>(d, io, eps, job, local, lds_raw, &inv_s); break;
    case 64: ns_panel<SPLIT, MODE, 64>(d, io, eps, job, local, lds_raw, &inv_s); break;
    case 96: ns_panel<SPLIT, MODE, 96>(d, io, eps, job, local, lds_raw, &inv_s); break;
    default: ns_panel<SPLIT, MODE, 128>(d, io, eps, job, local, lds_raw, &inv_s); break;
  }
}

typedef DmaCfg<1, 1, 1, 1, 4, 64, 4, 1, false> Ns32;      // TI TJ WGM WGN KW BK S OCC AHEAD
typedef DmaCfg<1, 1, 2, 2, 1, 64, 3, 3, true> Ns64;
typedef DmaCfg<2, 2, 2, 2, 1, 64, 2, 2, true> Ns128;
typedef DmaCfg<4, 2, 2, 4, 1, 64, 2, 1, true> Ns256;

int64_t ns_tiles(const NsGroup& g, int op, int bm, int bn) {
  const int64_t nbm = (g.m + bm - 1) / bm, nbn = (g.n + bn - 1) / bn;
  return g.count * (op == NS_GRAM || op == NS_SYM ? nbm * (nbm + 1) / 2 : nbm * nbn);
}

constexpr int kCUs = 256;
struct NoIO {};      // products that stay in the workspace
template <class C, int OP, bool SPLIT, class IO>
hipError_t launch_product(NsDev& d, const IO& io, hipStream_t s) {
  int64_t blocks = 0;
  for (int i = 0; i < d.n; ++i) { d.first_block[i] = (int)blocks; blocks += ns_tiles(d.job[i].g, OP, C::BM, C::BN); }
  d.first_block[d.n] = (int)blocks;
  auto kern = ns_product_kernel<C, OP, SPLIT, IO>;
  constexpr size_t lds = ns_lds<C, OP, SPLIT>();
  static_assert(C::OCC * lds <= 160 * 1024, "the blocks of a CU do not fit its LDS");
  static bool configured = false;      // per instantiation, as in gemm_wide.h
  if (!configured && lds > 48 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  configured = true;
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(C::NT), lds, s, d, io);
  return hipGetLastError();
}
// The side of the tiles that a launch takes.
template <int OP>
int product_tile(const NsDev& d) {
  // Rounds that the tiles of a size take on the chip (one 256 x 256 tile per CU, two of 128 x 128, three of 64 x 64) times what a round takes, as a share of one
  // of 256 x 256 tiles, from lists of 48 and 96 matrices of 1024 x 1024 and 1024 x 4096 (us with 256, 128, 64: GRAM 171, 189, 219; SYM 216, 211, 242; APPLY
  // 303, 335, 466).  256 x 256 tiles are not built for 32-bit products, nor taken by SYM.  A launch whose 32 x 32 tiles all have a CU takes
  // those, whose waves split the contraction (toy model 133 -> 117 us, one matrix 256 x 2048 135 -> 113).
  constexpr float kRound128 = OP == NS_SYM ? 0.48f : OP == NS_GRAM ? 0.60f : 0.55f, kRound64 = OP == NS_SYM ? 0.25f : 0.29f;
  auto rounds = [&](int b, int slots) {
    int64_t tiles = 0;
    for (int i = 0; i < d.n; ++i) tiles += ns_tiles(d.job[i].g, OP, b, b);
    return (float)((tiles + slots - 1) / slots);
  };
  if (rounds(32, kCUs) <= 1.0f) return 32;
  const float t256 = rounds(256, kCUs), t128 = rounds(128, 2 * kCUs) * kRound128, t64 = rounds(64, 3 * kCUs) * kRound64;
  if (!d.split && OP != NS_SYM && t256 <= std::min(t128, t64)) return 256;
  return t128 <= t64 ? 128 : 64;
}
template <int OP, class IO>
hipError_t product(NsDev& d, const IO& io, hipStream_t s) {
  switch (product_tile<OP>(d)) {
    case 32: return d.split ? launch_product<Ns32, OP, true, IO>(d, io, s) : launch_product<Ns32, OP, false, IO>(d, io, s);
    case 64: return d.split ? launch_product<Ns64, OP, true, IO>(d, io, s) : launch_product<Ns64, OP, false, IO>(d, io, s);
    case 128: return d.split ? launch_product<Ns128, OP, true, IO>(d, io, s) : launch_product<Ns128, OP, false, IO>(d, io, s);
    default: break;
  }
  if constexpr (OP != NS_SYM) return launch_product<Ns256, OP, false, IO>(d, io, s);
  return hipErrorInvalidValue;
}

// A large matrix whose longer side is at least twice the shorter is better served by polynomials of A than by products with X: over up to three steps
// X <- S_3 S_2 S_1 X with S_i = a I + b A_i + c A_i A_i and A_(i+1) = S_i A_i S_i, all symmetric m x m matrices that commute, and X itself is read
// and written once.  Five steps are 6 m m n + 14 m m m operations instead of 15 m m n + 5 m m m, in 17 launches instead of 15, beside those of the matrices that stay with the
// other form.  Where that pays (us, with and without, over 60 lists): of a list by itself from 1.5e10 operations saved on (2 of 640 x 2560, 1.4e10: 212, 228; 4 of 768 x 1536, 1.6e10: 251, 247;
// 12 of 1024 x 4096: 1169, 1586), in a stack of layers with square matrices from 8e10 on (12 layers of hidden 512, 8.7e10: 1048, 1204; 3 of 768, 7.3e10: 766, 743; 8 of 1024 with matrices 1 : 2,
// 1.5e11, the worst: 2581, 2442; 24 of 1024: 8.3 ms, 9.6 ms).
// From 512 rows on: A is not formed from X again in between, so that the rounding that its strong directions make stays in its weak ones, which grow by a in every step; it is the
// smaller the more rows it is spread over.  The worst of 80 spectra, one strong direction and a flat rest, came out 3.1e-2 off with 64 rows, 2.2e-2 with 128, 1.3e-2 with 256, 7e-3 with 512 and 5e-3 with
// 1024; step by step 7.5e-3, 4.0e-3, 2.8e-3, 1.7e-3 and 1.4e-3.
constexpr double kGramAlone = 1.5e10, kGramBeside = 8e10;
constexpr int kGramRows = 512;
bool ns_long(const NsGroup& g) { return g.m >= kGramRows && g.n >= 2 * g.m; }

// Whether a list goes through the panel kernel: up to 128 rows in every matrix, blocks for about one round of the chip, and not too much to read of each other's
// parts of A (a matrix of P panels: P P m m floats in a step).  The borders are the largest lists that measured better; nothing between them and the next ones was.  Whole list in us, with and without: 130 x 67 in 32 bits 70, 107; 64 x 64 42, 94; 16 of
// 64 x 1024 (64 MB) 77, 106, 64 of them 223, 142; 24 layers of hidden 64 (288 blocks) 89, 107, 48 of them 132, 122; of 128 rows, whose steps are longer: toy model
// 113, 121 (9 MB); 16 of 128 x 256 (17 MB) 94, 99; 16 of 128 x 512 (67 MB) 127, 103.
bool ns_small(const std::vector<NsGroup>& groups) {
  int64_t blocks = 0, bytes = 0;
  int rows = 0;
  for (const NsGroup& g : groups) {
    const int64_t m = (std::min(g.rows, g.cols) + 31) / 32 * 32, panels = g.n / kPanel;
    if (m > kPanelM) return false;
    rows = std::max(rows, (int)m);
    blocks += g.count * panels;
    bytes += g.count * panels * panels * m * m * 4;
  }
  return blocks <= 288 && bytes <= (rows > 96 ? (int64_t)17 << 20 : (int64_t)72 << 20);
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
    const int si = std::min(mats[i].rows, mats[i].cols), li = std::max(mats[i].rows, mats[i].cols);
    const int sj = std::min(mats[j].rows, mats[j].cols), lj = std::max(mats[j].rows, mats[j].cols);
    return std::make_tuple(lj, sj, mats[j].rows) < std::make_tuple(li, si, mats[i].rows);      // long contractions first
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
    p.groups.push_back(g);
    i = j;
  }
  const bool small = ns_small(p.groups);
  double saved = 0.0;
  bool others = false;
  for (const NsGroup& g : p.groups) {
    if (!split && ns_long(g)) saved += 9.0 * g.m * (double)g.m * (g.n - g.m) * g.count;
    else others = true;
  }
  const bool gram = saved >= (others ? kGramBeside : kGramAlone);
  for (NsGroup& g : p.groups) {
    g.kind = small ? NS_BY_PANEL : gram && ns_long(g) ? NS_BY_GRAM : NS_BY_STEP;
    if (small) g.m = (std::min(g.rows, g.cols) + 31) / 32 * 32;
    g.bufs = g.kind == NS_BY_GRAM ? BUFS : BUF_S + 1;
    g.ws = (int64_t)off; g.stride = (int64_t)matrix_bytes(g, split);
    off += (size_t)g.stride * g.count;
  }
  p.total = off;
  return p;
}

// Groups that go the same way, in runs of as many as the jobs of a launch.
std::vector<std::vector<NsGroup>> ns_runs(const NsPlan& plan, int kind) {
  const size_t most = kind == NS_BY_GRAM ? kJobs / 2 : kJobs;      // two products of a group in one launch
  std::vector<std::vector<NsGroup>> runs;
  for (const NsGroup& g : plan.groups) {
    if (g.kind != kind) continue;
    if (runs.empty() || runs.back().size() == most) runs.emplace_back();
    runs.back().push_back(g);
  }
  return runs;
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

// Whether two matrices share an element, a starting where b does or before and reaching beyond b's first.  With one row stride all rows of b lie alike
// between those of a; otherwise every row of the one with fewer rows is looked up among the other's.
bool ns_share(const hs_matrix& a, const hs_matrix& b) {
  if (a.ld == b.ld) {
    const int64_t shift = (b.offset - a.offset) % a.ld;      // b's first column, counted from a's
    return shift < a.cols || shift + b.cols > a.ld;
  }
  const hs_matrix& few = a.rows < b.rows ? a : b;
  const hs_matrix& many = a.rows < b.rows ? b : a;
  for (int64_t i = 0; i < few.rows; ++i) {
    const int64_t first = few.offset + i * few.ld - many.offset, last = first + few.cols;      // of this row, counted from the other matrix
    if (last <= 0) continue;
    if (first < 0) return true;
    const int64_t k = first / many.ld;                       // the other's row that starts here or before
    if (k >= many.rows) break;
    if (first - k * many.ld < many.cols || (k + 1 < many.rows && (k + 1) * many.ld < last)) return true;
  }
  return false;
}

// Whether no two matrices of the list share an element.
bool ns_disjoint(const hs_matrix* mats, int n) {
  std::vector<int> order(n);
  std::iota(order.begin(), order.end(), 0);
  std::sort(order.begin(), order.end(), [&](int i, int j) { return mats[i].offset < mats[j].offset; });
  auto end = [&](const hs_matrix& a) { return a.offset + (a.rows - 1) * a.ld + a.cols; };
  std::vector<int> open;      // matrices that reach beyond the present offset
  for (int i : order) {
    open.erase(std::remove_if(open.begin(), open.end(), [&](int k) { return end(mats[k]) <= mats[i].offset; }), open.end());
    for (int k : open) if (ns_share(mats[k], mats[i])) return false;
    open.push_back(i);
  }
  return true;
}

template <bool SPLIT, int MODE, class IO>
hipError_t launch_panel(const NsDev& d, const IO& io, double eps, unsigned blocks, hipStream_t s) {
  auto kern = ns_panel_kernel<SPLIT, MODE, IO>;
  constexpr size_t lds = panel_lds<SPLIT>();
  static bool configured = false;      // per instantiation, as in gemm_wide.h
  if (!configured) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  configured = true;
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(kPanelThreads), lds, s, d, io, eps);
  return hipGetLastError();
}

// The whole of it for groups that go the same way.
template <class IO>
hipError_t ns_run(const std::vector<NsGroup>& groups, int kind, int split, char* ws, NsPlace* table, const ShortTable& places, double* partial, const IO& io,
                  int steps, const double* c, double eps, hipStream_t s) {
  static_assert(sizeof(NsDev) + sizeof(ShortTable) + sizeof(IO) + 64 <= 4096, "kernel arguments");
  NsDev d{};
  d.split = split; d.ws = ws; d.table = table; d.partial = partial;
  auto add = [&](int p, int q, int out, double ident, double alpha, double beta) {
    for (const NsGroup& g : groups) d.job[d.n++] = NsJob{g, p, q, out, (float)ident, (float)alpha, (float)beta};
  };
  auto blocks_of = [&](auto per) {
    int64_t blocks = 0;
    for (int i = 0; i < d.n; ++i) { d.first_block[i] = (int)blocks; blocks += (int64_t)d.job[i].g.count * per(d.job[i].g); }
    d.first_block[d.n] = (int)blocks;
    return (unsigned)blocks;
  };
  add(0, 0, 0, 0.0, 0.0, 0.0);
  unsigned blocks = blocks_of([](const NsGroup& g) { return g.parts; });
  hipLaunchKernelGGL(ns_norm_kernel<IO>, dim3(blocks), dim3(256), 0, s, d, io, places);
  if (kind == NS_BY_PANEL) {
    blocks = blocks_of([](const NsGroup& g) { return g.n / kPanel; });
    hipError_t e = split ? launch_panel<true, PANEL_FIRST>(d, io, eps, blocks, s) : launch_panel<false, PANEL_FIRST>(d, io, eps, blocks, s);
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
      d.from ^= 1;
      for (int i = 0; i < d.n; ++i) { d.job[i].ident = (float)c[3 * k]; d.job[i].alpha = (float)c[3 * k + 1]; d.job[i].beta = (float)c[3 * k + 2]; }
      if (k + 1 < steps) e = split ? launch_panel<true, PANEL_STEP>(d, io, eps, blocks, s) : launch_panel<false, PANEL_STEP>(d, io, eps, blocks, s);
      else e = split ? launch_panel<true, PANEL_LAST>(d, io, eps, blocks, s) : launch_panel<false, PANEL_LAST>(d, io, eps, blocks, s);
    }
    return e;
  }
  const bool gram = kind == NS_BY_GRAM;
  blocks = blocks_of([](const NsGroup& g) { return (g.m / 64) * (g.n / 64); });
  hipLaunchKernelGGL(ns_start_kernel<IO>, dim3(blocks), dim3(256), 0, s, d, io, eps);
  hipError_t e = hipGetLastError();
  auto go = [&](auto op) {
    constexpr int OP = decltype(op)::value;
    if (e == hipSuccess && d.n > 0) {
      if constexpr (OP == NS_LAST) e = product<OP, IO>(d, io, s); else e = product<OP, NoIO>(d, NoIO{}, s);
    }
    d.n = 0;
  };
  typedef std::integral_constant<int, NS_GRAM> Gram;
  typedef std::integral_constant<int, NS_SYM> Sym;
  d.n = 0;
  for (int k = 0; k < steps && e == hipSuccess;) {
    // steps taken on A alone: their product must stay in range of its buffer
    int len = 1;
    double grown = std::fabs(c[3 * k]);
    while (gram && len < 3 && k + len < steps && (grown *= std::fabs(c[3 * (k + len)])) <= 64.0) ++len;
    add(0, 0, BUF_A, 0.0, 0.0, 1.0);
    go(Gram{});
    int q = BUF_S;      // the product of the steps so far
    for (int j = 0; j < len; ++j) {
      const int out = j == 0 && len > 1 ? BUF_Q : BUF_S;
      add(BUF_A, BUF_A, out, c[3 * (k + j)], c[3 * (k + j) + 1], c[3 * (k + j) + 2]);
      go(Sym{});
      if (j + 1 < len) add(out, BUF_A, BUF_T, 0.0, 0.0, 1.0);
      if (j == 0) {
        q = out;
      } else {
        const int to = q == BUF_Q ? BUF_Q2 : BUF_Q;
        add(BUF_S, q, to, 0.0, 0.0, 1.0);
        q = to;
      }
      go(Sym{});
      if (j + 1 < len) add(BUF_T, out, BUF_A, 0.0, 0.0, 1.0);
      go(Sym{});
    }
    k += len;
    add(q, 0, 0, 0.0, 0.0, 1.0);
    if (k < steps) go(std::integral_constant<int, NS_APPLY>{}); else go(std::integral_constant<int, NS_LAST>{});
    d.from ^= 1;
  }
  return e;
}

const double kDefaultCoeff[3] = {3.4445, -4.7750, 2.0315};

template <class IO>
hs_status orthogonalize_checked(const char* who, const IO& io, size_t size, const hs_matrix* mats, int32_t n, int32_t products, int32_t steps,
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
  auto place = [&](int i) { return NsPlace{mats[plan.order[i]].offset, mats[plan.order[i]].ld}; };
  hipError_t e = hipSuccess;
  ShortTable places{};
  places.first = 0; places.n = n <= 100 ? n : 0;
  for (int i = 0; i < places.n; ++i) places.place[i] = place(i);
  for (int done = 0; places.n == 0 && done < n && e == hipSuccess; done += 200) {
    TableArg t;
    t.first = done; t.n = std::min(200, n - done);
    for (int i = 0; i < t.n; ++i) t.place[i] = place(done + i);
    hipLaunchKernelGGL(ns_table_kernel, dim3(1), dim3(256), 0, s, t, table);
    e = hipGetLastError();
  }
  std::vector<double> c(3 * steps);
  for (int k = 0; k < 3 * steps; ++k) c[k] = coeff ? coeff[k] : kDefaultCoeff[k % 3];
  for (int kind : {NS_BY_STEP, NS_BY_GRAM, NS_BY_PANEL})
    for (const std::vector<NsGroup>& now : ns_runs(plan, kind))
      if (e == hipSuccess) e = ns_run(now, kind, split, ws, table, places, (double*)(ws + plan.partial), io, steps, c.data(), eps, s);
  return e == hipSuccess ? HS_OK : hs_fail(nullptr, HS_ERR_HIP, name + hipGetErrorString(e));
}

// no exception leaves a C entry
template <class IO>
hs_status orthogonalize(const char* who, const IO& io, size_t size, const hs_matrix* mats, int32_t n, int32_t products, int32_t steps,
                        const double* coeff, double eps, void* workspace, size_t workspace_bytes, hipStream_t s) {
  try {
    return orthogonalize_checked(who, io, size, mats, n, products, steps, coeff, eps, workspace, workspace_bytes, s);
  } catch (const std::bad_alloc&) {
    return hs_fail(nullptr, HS_ERR_STATE, "out of host memory");
  }
}

}  // namespace

extern "C" {

size_t hs_orthogonalize_workspace_bytes(const hs_matrix* mats, int32_t n, int32_t products) {
  std::string why;
  if ((products != HS_FP32 && products != HS_BF16) || !ns_list_ok(mats, n, &why)) {
    hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_orthogonalize_workspace_bytes: " + (why.empty() ? "products must be HS_FP32 or HS_BF16" : why));
    return 0;
  }
  try {
    return std::max<size_t>(ns_plan(mats, n, products == HS_FP32).total, 256);      // an empty list is no invalid one
  } catch (const std::bad_alloc&) {
    hs_fail(nullptr, HS_ERR_STATE, "hs_orthogonalize_workspace_bytes: out of host memory");
    return 0;
  }
}

hs_status hs_orthogonalize_choice(const hs_matrix* mats, int32_t n, int32_t products, int32_t matrix, int32_t* way, int32_t* tiles) {
  try {
    std::string why;
    if (products != HS_FP32 && products != HS_BF16) why = "products must be HS_FP32 or HS_BF16";
    else if (!ns_list_ok(mats, n, &why)) ;
    else if (matrix < 0 || matrix >= n || !way || !tiles) why = "no such matrix, or nowhere to write";
    if (!why.empty()) return hs_fail(nullptr, HS_ERR_INVALID_ARG, "hs_orthogonalize_choice: " + why);
    const NsPlan plan = ns_plan(mats, n, products == HS_FP32);
    const int at = (int)(std::find(plan.order.begin(), plan.order.end(), matrix) - plan.order.begin());
    for (int kind : {NS_BY_STEP, NS_BY_GRAM, NS_BY_PANEL})
      for (const std::vector<NsGroup>& now : ns_runs(plan, kind)) {
        if (std::none_of(now.begin(), now.end(), [&](const NsGroup& g) { return at >= g.first && at < g.first + g.count; })) continue;
        NsDev d{};
        d.split = products == HS_FP32;
        for (const NsGroup& g : now) d.job[d.n++].g = g;
        const bool panel = kind == NS_BY_PANEL;
        *way = kind;
        tiles[0] = panel ? 0 : product_tile<NS_GRAM>(d);
        tiles[1] = panel ? 0 : product_tile<NS_SYM>(d);
        tiles[2] = panel ? 0 : product_tile<NS_APPLY>(d);
      }
    return HS_OK;
  } catch (const std::bad_alloc&) {
    return hs_fail(nullptr, HS_ERR_STATE, "hs_orthogonalize_choice: out of host memory");
  }
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
  const MuonIO io{w, m, G, (bf16*)w_lowp_out, (float)denom, (float)momentum, (float)(1.0 - lr * weight_decay), (float)lr, (float)rms, nesterov ? 1 : 0};
  return orthogonalize("hs_muon_step", io, size, mats, n, products, steps, coeff, eps, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
