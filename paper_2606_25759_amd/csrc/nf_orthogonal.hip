// nf_orthogonal.hip - orthogonalisation by Newton-Schulz products and the
// matrix step around it.
//
//   k_norm     U's sum of squares (FP64 partials, fixed order); for the step
//              also M = mu M + g
//   k_scale    X = U / (||U|| + eps) as FP16 pairs, the short side as rows,
//              zero-padded to whole tiles, and X^T
//   k_prod     one product P Q^T on the matrix cores with an epilogue:
//                GRAM  A = X X^T
//                POLY  B = b A + c A A
//                MULT  alpha Y + Z Y of symmetric matrices that commute
//                BOTH  A and the product of a few steps' polynomials of it,
//                      where A is one tile (a short side of at most 64)
//                STEP  X = a X + B X
//                LAST  the same, into the caller's matrix or weights
//
// With m the short side and n the long one, a step is m^2 n + m^3 + 2 m^2 n
// flops: A and A A are symmetric, so tiles on and below the diagonal are
// computed and mirrored.
//
// Long sides take a few steps at once.  With q(A) = a + b A + c A A a step is
// X <- q(A) X, and A <- q(A) A q(A): after some steps X <- P X with P, the
// product of the q(A), from m x m matrices alone (MULT, BOTH), so that X is
// read and written once for all of them.
//
// Operands lie in panels of 32 k: element (row, k) of a matrix of R rows is
// at ((k / 32) R + row) 32 + k % 32.  A stage's BT rows are then one
// contiguous piece of memory, whole cache lines, whatever the tile.
//
// What is held in which precision.  Operands of products are FP16 (11 bits;
// in split mode a pair of FP16, 22 bits, and three products), sums FP32.  X
// times 2^10 lies well inside FP16's range, since no entry exceeds the
// largest singular value.  Three places would lose more than the rounding of
// the operands costs, and are kept apart:
//   - the linear term a X takes X as the pair (22 bits).  a > 1 is how small
//     singular values grow, by a^S = 485 over five steps: noise in every
//     direction, which rounding X is, would grow with them.  B X (X rounded)
//     only turns the large directions among themselves, which nothing
//     amplifies.
//   - the diagonals of A and B are FP32 vectors and their FP16 matrices have
//     a zero diagonal: near convergence A is close to a multiple of I, and
//     the rounding of its large diagonal would be the largest error left.
//   - B's diagonal multiplies the same rounded X as the rest of B does,
//     except in the last step, after which nothing is amplified any more.
// FP16 pairs keep 22 bits of what is well above their spacing of 2^-24.  Where
// ||G|| is far below eps, X is far below one, and held times another power of
// two a matrix and step (Steps); for all others that power is one.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "nf_internal.h"
#include "nf_types.h"

namespace nf {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));

constexpr float kScale = 1024.0f;         // X, A and B in FP16 are held times this
constexpr float kInvScale = 1.0f / kScale;
constexpr int kBK = 32;                   // k of one stage: a panel
constexpr int kStages = 4;                // LDS stages of k_prod
constexpr int kNormThreads = 256;
constexpr int kNormElems = 4096;          // elements of a norm partial, at least
constexpr int kMaxParts = 1024;           // of a matrix
constexpr int kBlock = 3;                 // steps that BOTH takes at once, at most

enum { GRAM, POLY, STEP, LAST, BOTH, MULT };

// One matrix of the caller's, seen as rows x cols.
struct View {
  void* p;
  int64_t ld, stride;
  int32_t type;
};

// A matrix's steps.  With X held times 2^e before a step and times 2^f after it, the same step has the coefficients
// a 2^(f - e), b 2^(f - 3 e) and c 2^(f - 5 e).
struct Steps {
  float coef[NF_ORTHOGONAL_MAX_STEPS][3];
  int32_t shift;  // the result is held times 2^shift
};

struct PrepArgs {
  View g;              // gradient or source
  float* mom;          // nullptr: U = g
  int64_t mom_ld, mom_stride;
  float mu;
  int32_t nesterov;
  int64_t rows, cols;
  int32_t tall;        // rows > cols: X is the transpose
  int64_t Mp, Np;      // padded short and long side
  double* part;        // [batch][nparts]
  int32_t nparts;
  int32_t lg_tx;       // k_norm: log2 of the threads across a row, four elements each
  float eps;
  int32_t steps;
  float coef[NF_ORTHOGONAL_MAX_STEPS][3];
  Steps* table;        // [batch]
  _Float16 *xh, *xl, *th, *tl;  // tl: split only
  int32_t* arrived;    // to be zeroed
  int64_t tiles;
};

struct ProdArgs {
  const _Float16 *ph, *pl, *qh, *ql;  // P: tm tiles of rows, Q: tn tiles
  int64_t ldk;                        // k of both
  int64_t pstride, qstride;           // a matrix of the batch
  int32_t tm, tn;                     // tiles
  const Steps* table;                 // [batch]
  int32_t k;                          // the step, or the first of them
  int32_t steps;                      // BOTH: at most kBlock of them
  int32_t whole;                      // STEP, LAST: Q is all that X is multiplied by (else a X is added)
  _Float16 *oh, *ol;                  // GRAM: A, POLY: B; STEP: X^T
  int64_t ostride;
  const _Float16 *ah, *al;            // POLY: A; MULT: Y (Z is P)
  float* dA;                          // diagonals, [batch][Mp]: of A or Y
  float* dB;                          // of B, of what MULT gives, of P where STEP takes that
  const float* dZ;                    // MULT: of Z
  float* dP;                          // POLY: if not nullptr, that of a + B
  _Float16 *xh, *xl;                  // STEP, LAST: X [Mp x Np]
  int64_t Mp, Np;
  View dst;                           // LAST
  int64_t m, n;                       // real short and long side
  int32_t tall;
  int32_t update;                     // 1: dst holds weights
  float keep, rate;                   // w = keep w - rate o
  int32_t shares;                     // GRAM: blocks that share a tile's k
  uint64_t* part;                     // their sums, [tile][share][BT x BT], two FP32 a word
  int32_t* arrived;                   // [tile], zero between launches
};

// The power of two that X of a norm of at most u is held times: to [1/2, 1), and never down.
__device__ __forceinline__ int shift_of(double u) {
  int e = 0;
  if (u > 0.0 && u < 0.5) frexp(u, &e);
  return -e;
}

// The steps of a matrix that begins with the norm u.  No singular value grows by more than |a| + |b| u^2 + |c| u^4, and
// neither does the norm.
__device__ void steps_of(const PrepArgs& a, double u, Steps* to) {
  int e = shift_of(u);
  for (int k = 0; k < a.steps; ++k) {
    const float* c = a.coef[k];
    const double uu = u * u;
    u = fmin(u * (fabs((double)c[0]) + uu * (fabs((double)c[1]) + uu * fabs((double)c[2]))), 0x1p100);
    const int f = shift_of(u);
    to->coef[k][0] = ldexpf(c[0], f - e);
    to->coef[k][1] = ldexpf(c[1], f - 3 * e);
    to->coef[k][2] = ldexpf(c[2], f - 5 * e);
    e = f;
  }
  to->shift = e;
}

// Elements c .. c + 3 of n of a row, the first at p + off; zeros past the row's end.
template <typename T>
__device__ __forceinline__ float4v load_four(const void* p, int64_t off, int64_t c, int64_t n) {
  const T* q = (const T*)p + off;
  float4v v = {};
  if (c + 3 < n) {
    const Near<T, 4> w = *(const Near<T, 4>*)q;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_f32(w.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < n) v[e] = to_f32(q[e]);
  }
  return v;
}

__device__ __forceinline__ float4v load_four(const View& g, int64_t off, int64_t c, int64_t n) {
  if (g.type == NF_TYPE_F32) return load_four<float>(g.p, off, c, n);
  if (g.type == NF_TYPE_BF16) return load_four<Bf16>(g.p, off, c, n);
  return load_four<_Float16>(g.p, off, c, n);
}

// The number that a pair of halves holds (as a product and sum: one instruction that takes both as FP16).
__device__ __forceinline__ float pair(_Float16 h, _Float16 l) { return fmaf((float)h, 1.0f, (float)l); }

// Where (row, k) of a matrix of R rows lies.
__device__ __forceinline__ int64_t panel_at(int64_t row, int64_t k, int64_t R) {
  return ((k / kBK) * R + row) * kBK + k % kBK;
}

// U at columns c .. c + 3 of row r, the momentum already stepped.
__device__ __forceinline__ float4v value_of(const PrepArgs& a, int64_t b, int64_t r, int64_t c) {
  float4v m = {};
  if (a.mom) {
    m = load_four<float>(a.mom, b * a.mom_stride + r * a.mom_ld + c, c, a.cols);
    if (!a.nesterov) return m;
  }
  float4v u = load_four(a.g, b * a.g.stride + r * a.g.ld + c, c, a.cols);
  if (a.mom)
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = fmaf(a.mu, m[e], u[e]);
  return u;
}

// The block's sum of x in a fixed order, in every thread.
__device__ double block_sum(double x, double* s) {
  for (int o = 32; o; o >>= 1) x += __shfl_down(x, o);
  if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = x;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kNormThreads / 64; ++i) t += s[i];
  return t;
}

// Block x of matrix y: every nparts-th group of rows, threads 2^lg_tx across
// a row.  Squares are FP64, so no gradient's scale overflows or vanishes.
// Bound by memory: 24 x (2048 x 2048) FP32 in 79 to 93 us (403 MB, 4.3 to 5.1
// TB/s); with the momentum, 4 x (8192 x 2048) in 142 us (805 MB, 5.7 TB/s).
__global__ __launch_bounds__(kNormThreads) void k_norm(PrepArgs a) {
  __shared__ double s[kNormThreads / 64];
  const int tx = 1 << a.lg_tx, ty = kNormThreads >> a.lg_tx;
  const int64_t b = blockIdx.y;
  if (b == 0) {
    const int64_t all = (int64_t)gridDim.x * kNormThreads;
    for (int64_t i = (int64_t)blockIdx.x * kNormThreads + threadIdx.x; i < a.tiles; i += all) a.arrived[i] = 0;
  }
  const int x = threadIdx.x & (tx - 1), y = threadIdx.x >> a.lg_tx;
  double sum = 0.0;
  for (int64_t r = (int64_t)blockIdx.x * ty + y; r < a.rows; r += (int64_t)gridDim.x * ty) {
    for (int64_t c = 4 * x; c < a.cols; c += 4 * tx) {
      float4v u = load_four(a.g, b * a.g.stride + r * a.g.ld + c, c, a.cols);
      if (a.mom) {
        const int64_t off = b * a.mom_stride + r * a.mom_ld + c;
        float4v m = load_four<float>(a.mom, off, c, a.cols);
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = fmaf(a.mu, m[e], u[e]);
        if (c + 3 < a.cols) {
          *(Near<float, 4>*)(a.mom + off) = Near<float, 4>{{m[0], m[1], m[2], m[3]}};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < a.cols) a.mom[off + e] = m[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = a.nesterov ? fmaf(a.mu, m[e], u[e]) : m[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += (double)u[e] * (double)u[e];
    }
  }
  sum = block_sum(sum, s);
  if (threadIdx.x == 0) a.part[b * a.nparts + blockIdx.x] = sum;
}

// A 64 x 64 tile of the caller's matrix, padding included: scaled, split in
// two FP16, stored as it lies and transposed.  Bound by memory: 24 x (2048 x
// 2048) in 177 us (403 MB read, 604 MB written: 5.7 TB/s).
__global__ __launch_bounds__(kNormThreads) void k_scale(PrepArgs a) {
  __shared__ double s[kNormThreads / 64];
  __shared__ float tile[64][65];
  const int64_t b = blockIdx.z;
  double part = 0.0;
  for (int i = threadIdx.x; i < a.nparts; i += kNormThreads) part += a.part[b * a.nparts + i];
  const double size_of_u = sqrt(block_sum(part, s)), norm = size_of_u + (double)a.eps;
  const double u = size_of_u / norm;  // of X
  const double inv = norm > 0.0 || norm != norm ? ldexp((double)kScale, shift_of(u)) / norm : 0.0;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) steps_of(a, u, a.table + b);
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  const int x = threadIdx.x % 16 * 4, y = threadIdx.x / 16;
  const int64_t size = a.Mp * a.Np;
  // rows x cols as it lies: X, or X^T where the caller's matrix is tall
  const int64_t R0 = a.tall ? a.Np : a.Mp, R1 = a.tall ? a.Mp : a.Np;
  _Float16* h0 = (a.tall ? a.th : a.xh) + b * size;
  _Float16* h1 = (a.tall ? a.xh : a.th) + b * size;
  _Float16* l0 = a.tall ? a.tl : a.xl;
  _Float16* l1 = a.tall ? a.xl : a.tl;
  auto store = [&](_Float16* hi, _Float16* lo, int64_t at, float4v v) {
    half4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[e] = (_Float16)v[e];
      l[e] = (_Float16)(v[e] - (float)h[e]);
    }
    *(half4*)(hi + at) = h;
    if (lo) *(half4*)(lo + b * size + at) = l;
  };
#pragma unroll
  for (int i = 0; i < 64; i += 16) {
    const int64_t r = r0 + y + i;
    float4v v = {};
    if (r < a.rows && c0 + x < a.cols) v = value_of(a, b, r, c0 + x);
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[y + i][x + e] = v[e] = (float)((double)v[e] * inv);
    store(h0, l0, panel_at(r, c0 + x, R0), v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 16) {
    const float4v v = {tile[x][y + i], tile[x + 1][y + i], tile[x + 2][y + i], tile[x + 3][y + i]};
    store(h1, l1, panel_at(c0 + y + i, r0 + x, R1), v);
  }
}

// ---------------------------------------------------------------- products

typedef const __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

// BT rows of a panel (contiguous in src) into an LDS tile: each wavefront
// moves sixteen rows (1 KiB) at a time straight into LDS, lane l the 16 bytes
// that belong in the l-th slot.
//
// A fragment is sixteen rows of thirty-two: rows 8 q + e and, in the odd
// fragment of a pair, 8 q + 4 + e (q, e in [0, 4)).  Of the products of two
// pairs a lane then holds eight adjacent rows of eight columns, 16 bytes of
// FP16 that belong together in memory, and four lanes a whole 64-byte row of
// a panel.
//
// Slot j of row r holds the row's 16-byte piece j ^ swizzle(r).  A 16-byte
// read of 64 lanes is served sixteen lanes at a time: lanes 0-3, 12-15, 20-23
// and 24-27 (q = 0 and 3 of one piece, 1 and 2 of the next) and so on; with
// this swizzle those, like lanes 0-15, touch sixteen different 16-byte
// columns of the 64 banks.  (With r / 8 % 4 for a swizzle, two of them
// collide: a conflict counted in every read.)
__device__ __forceinline__ int swizzle(int row) {
  const int q = row >> 3;
  return ((q >> 1) & 1) | (((q ^ (q >> 1)) & 1) << 1);
}

// A lane's place in the 1 KiB that its wavefront moves (row: the first of them), and in the rows of a fragment.
__device__ __forceinline__ int load_place(int row, int lane) {
  return lane / 4 * kBK + ((lane % 4) ^ swizzle(row + lane / 4)) * 8;
}
__device__ __forceinline__ int read_place(int lane) {
  const int row = lane % 16 / 4 * 8 + lane % 4;
  return row * kBK + ((lane / 16) ^ swizzle(row)) * 8;
}
// Where fragment i's rows begin.
__device__ __forceinline__ constexpr int fragment_at(int i) { return (i / 2 * 32 + i % 2 * 4) * kBK; }

template <int BT, int NW>
__device__ __forceinline__ void load_tile(const _Float16* src, _Float16* lds, int wave, int place) {
  static_assert(NW % 2 == 0, "a wavefront's rows begin at the same place of 32 each time");
#pragma unroll
  for (int i = 0; i < BT / 16 / NW; ++i) {
    const int rb = (i * NW + wave) * 16;
    __builtin_amdgcn_global_load_lds((gptr)(uintptr_t)(src + rb * kBK + place), (lptr)(lds + rb * kBK), 16, 0, 0);
  }
}

// Until at most N of this wavefront's loads into LDS, and R of its reads of LDS, are under way.
template <int N, int R>
__device__ __forceinline__ void wait_for() {
  static_assert(N >= 0 && N < 64 && R >= 0 && R < 16, "the counters' ranges");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)" ::"n"(N), "n"(R) : "memory");
}

__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Lanes 4q .. 4q + 3 hold a 4 x 4 block by columns (element e of lane i:
// row e, column i); after it by rows (element e of lane i: row i, column e).
__device__ __forceinline__ half4 transpose4(half4 v, int lane) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  const u2 x = __builtin_bit_cast(u2, v);
  // columns 2i, 2i + 1 of a row in one word: odd rows go to odd lanes
  const uint32_t ox = (uint32_t)__builtin_amdgcn_mov_dpp((int)x[0], 0xB1, 0xf, 0xf, true);  // lane ^ 1
  const uint32_t oy = (uint32_t)__builtin_amdgcn_mov_dpp((int)x[1], 0xB1, 0xf, 0xf, true);
  const bool odd = lane & 1;
  const uint32_t p = odd ? __builtin_amdgcn_perm(x[0], ox, 0x07060302) : __builtin_amdgcn_perm(ox, x[0], 0x05040100);
  const uint32_t q = odd ? __builtin_amdgcn_perm(x[1], oy, 0x07060302) : __builtin_amdgcn_perm(oy, x[1], 0x05040100);
  // p: row 0 or 1, q: row 2 or 3, of this lane's pair of columns; rows 2, 3 belong in lanes 2, 3
  const bool high = lane & 2;
  const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)(high ? p : q), 0x4E, 0xf, 0xf, true);  // lane ^ 2
  const u2 o = {high ? got : p, high ? q : got};
  return __builtin_bit_cast(half4, o);
}

// The same for FP32.
__device__ __forceinline__ float dpp_xor1(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true));
}
__device__ __forceinline__ float dpp_xor2(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, true));
}
__device__ __forceinline__ void transpose4(float (&v)[4], int lane) {
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    const float got = dpp_xor1(odd ? v[e] : v[e + 1]);
    if (odd)
      v[e] = got;
    else
      v[e + 1] = got;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float got = dpp_xor2(high ? v[e] : v[e + 2]);
    if (high)
      v[e] = got;
    else
      v[e + 2] = got;
  }
}

// Rows 4 x + (0 .. 3) of a pair of columns of four, after transposition: row 4 x + lane % 4, eight columns.
__device__ __forceinline__ half8 transpose8(half8 c0, half8 c1, int x, int lane) {
  const half4 a = {c0[4 * x], c0[4 * x + 1], c0[4 * x + 2], c0[4 * x + 3]};
  const half4 b = {c1[4 * x], c1[4 * x + 1], c1[4 * x + 2], c1[4 * x + 3]};
  const half4 p = transpose4(a, lane), q = transpose4(b, lane);
  return half8{p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
}

// Eight results of one row of the caller's matrix, columns c .. c + 7 of n.
template <typename T>
__device__ __forceinline__ void store_eight(const ProdArgs& a, int64_t off, int64_t c, int64_t n, const float (&o)[8]) {
  T* p = (T*)a.dst.p + off;
  if (c + 7 < n) {
    Near<T, 8> w;
    if (a.update) w = *(const Near<T, 8>*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      w.v[e] = from_f32<T>(a.update ? fmaf(a.keep, to_f32(w.v[e]), -a.rate * o[e]) : o[e]);
    *(Near<T, 8>*)p = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) p[e] = from_f32<T>(a.update ? fmaf(a.keep, to_f32(p[e]), -a.rate * o[e]) : o[e]);
  }
}

// The last step's results into the caller's matrix: rows (long side) r .. r + 7 of columns (short side)
// cq + 4 y + lane % 4, times the scale.  Eight adjacent elements of a row of it are rows here, or, where it is tall,
// columns.
__device__ __forceinline__ void store_last(const ProdArgs& a, int64_t b, int64_t r, int64_t rq, int64_t cq, int lane,
                                           float scale, float (&v)[2][8]) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    float o[8];
    if (a.tall) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float w[4] = {v[y][4 * x], v[y][4 * x + 1], v[y][4 * x + 2], v[y][4 * x + 3]};
        transpose4(w, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[4 * y + e] = w[e] * scale;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = v[x][e] * scale;
    }
    const int64_t row = a.tall ? rq + 4 * x : cq + 4 * x + lane % 4, col = a.tall ? cq : r;
    const int64_t rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
    const int64_t off = b * a.dst.stride + row * a.dst.ld + col;
    if (row < rows) {
      if (a.dst.type == NF_TYPE_F32)
        store_eight<float>(a, off, col, cols, o);
      else if (a.dst.type == NF_TYPE_BF16)
        store_eight<Bf16>(a, off, col, cols, o);
      else
        store_eight<_Float16>(a, off, col, cols, o);
    }
  }
}

// D = P Q^T over one BT x BT tile, WM x WN of it per wavefront.  Lane l of a
// 16 x 16 part holds rows 4 (l / 16) .. + 3 of column l % 16.
//
// Four stages of 32 k in LDS, filled three ahead of use; fragments are read
// from LDS one stage ahead of the products that use them.  One barrier a stage: a
// wavefront that passes it has its loads of stage s + 1 in LDS, and has read
// stage s - 1, whose place stage s + 3 takes.  In split mode a stage holds
// both halves of both operands, and feeds three products.
//
// What bounds it.  The loop by itself, with tiles of 256 on 4096 x 4096 x 4096,
// does 1.36 PFLOP/s, as a library product of that type does (1.38 to 1.41).
// Of 24 x (2048 x 2048), GRAM takes 243 us (0.95 PFLOP/s: 864 tiles are 3.4
// rounds of the card), POLY 266 us, STEP 481 us: 412 GFLOP are 300 us of that
// and the 1.0 GB that its epilogue reads and writes the rest, one after the
// other, since all blocks of a round end together.  (Two blocks a CU with
// tiles of 256 x 128 do not overlap them either: 488 us against 483 in a copy
// of the loop.)  Small matrices are bound by launches, 4 to 6 us each, most of
// it the way of the first operands from another XCD's writes.
template <int BT, int WM, int WN, bool SPLIT, int EPI, bool SHARED = false>
__global__ __launch_bounds__(BT / WM * (BT / WN) * 64) void k_prod(ProdArgs a) {
  constexpr int NW = BT / WM * (BT / WN);
  constexpr int OPS = SPLIT ? 4 : 2;         // tiles of a stage: P, Q (, their low halves)
  constexpr int LOADS = OPS * BT / 16 / NW;  // of a wavefront a stage
  constexpr int MI = WM / 16, NJ = WN / 16;
  constexpr bool SYM = EPI == GRAM || EPI == POLY || EPI == BOTH || EPI == MULT;
  __shared__ __align__(16) _Float16 lds[kStages][OPS][BT * kBK];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int lane = threadIdx.x % 64;
  // blocks go round the eight XCDs: each XCD takes a contiguous share of the tiles, matrix by matrix
  int id;
  {
    const int total = gridDim.x, x = blockIdx.x & 7, each = total >> 3, more = total & 7;
    id = x * each + min(x, more) + (blockIdx.x >> 3);
  }
  int share = 0;  // of the k
  if (SHARED) {
    share = id % a.shares;
    id /= a.shares;
  }
  const int per = SYM ? a.tm * (a.tm + 1) / 2 : a.tm * a.tn;
  const int64_t b = id / per;
  const int tile = id;
  id -= (int)b * per;
  int ti, tj;
  if (SYM) {  // tiles on and below the diagonal, row by row
    ti = (int)((sqrtf(8.0f * (float)id + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > id) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
    tj = id - ti * (ti + 1) / 2;
  } else {  // four rows of tiles at a time
    const int g = id / (4 * a.tn), rows = min(4, a.tm - 4 * g);
    const int in = id - g * 4 * a.tn;
    ti = 4 * g + in % rows;
    tj = in / rows;
  }
  const int wm = wave / (BT / WN) * WM, wn = wave % (BT / WN) * WN;
  float4v acc[MI][NJ] = {};

  // The matrix's coefficients, asked for before the products.
  constexpr int TAKEN = EPI == GRAM ? 0 : EPI == BOTH ? kBlock : 1;
  float coef[TAKEN ? TAKEN : 1][3] = {};
#pragma unroll
  for (int q = 0; q < TAKEN; ++q)
#pragma unroll
    for (int e = 0; e < 3; ++e) coef[q][e] = a.table[b].coef[min(a.k + q, NF_ORTHOGONAL_MAX_STEPS - 1)][e];
  const float ca = EPI == STEP || EPI == LAST ? (a.whole ? 0.0f : coef[0][0]) : coef[0][0];
  const float cb = coef[0][1], cc = coef[0][2];
  const float scale = EPI == LAST ? ldexpf(kInvScale, -a.table[b].shift) : 0.0f;

  // What the epilogue reads: of small tiles asked for now, before the products, else when it is needed.
  constexpr bool EARLY = BT == 64;
  constexpr int CI = MI / 2, CJ = NJ;  // eight rows of a column each
  half8 inh[EARLY ? CI : 1][EARLY ? CJ : 1], inl[EARLY ? CI : 1][EARLY ? CJ : 1];
  float dcol[EARLY ? CJ : 1];
  float4v drow[EARLY ? CI : 1][2];
  half8 inzh[EARLY && EPI == MULT ? CI : 1][EARLY && EPI == MULT ? CJ : 1];
  half8 inzl[EARLY && EPI == MULT ? CI : 1][EARLY && EPI == MULT ? CJ : 1];
  auto row_at = [&](int i) { return (int64_t)ti * BT + wm + 16 * i + lane / 16 * 8; };
  auto column_at = [&](int j) { return (int64_t)tj * BT + wn + j / 2 * 32 + j % 2 * 4 + lane % 16 / 4 * 8 + lane % 4; };
  auto ask = [&](int i, int j, half8& h, half8& l, float& dc, float4v (&dr)[2], half8& zh, half8& zl) {  // i even
    const int64_t r = row_at(i), c = column_at(j);
    l = half8{};
    if (EPI == POLY || EPI == MULT) {
      const int64_t at = b * a.ostride + panel_at(c, r, a.Mp);
      h = *(const half8*)(a.ah + at);
      if (SPLIT) l = *(const half8*)(a.al + at);
      dc = a.dA[b * a.Mp + c];
      const float* rows = EPI == MULT ? a.dZ : a.dA;
      dr[0] = *(const float4v*)(rows + b * a.Mp + r);
      dr[1] = *(const float4v*)(rows + b * a.Mp + r + 4);
      if (EPI == MULT) {
        zh = *(const half8*)(a.ph + at);
        zl = *(const half8*)(a.pl + at);
      }
    } else if (EPI == STEP || EPI == LAST) {
      const int64_t at = b * a.Mp * a.Np + panel_at(c, r, a.Mp);
      h = *(const half8*)(a.xh + at);
      l = *(const half8*)(a.xl + at);
      dc = a.dB[b * a.Mp + c];
    }
  };
  if constexpr (EARLY && (EPI == POLY || EPI == STEP || EPI == LAST || EPI == MULT)) {
#pragma unroll
    for (int i = 0; i < CI; ++i)
#pragma unroll
      for (int j = 0; j < CJ; ++j)
        ask(2 * i, j, inh[i][j], inl[i][j], dcol[j], drow[i], inzh[EPI == MULT ? i : 0][EPI == MULT ? j : 0],
            inzl[EPI == MULT ? i : 0][EPI == MULT ? j : 0]);
  }

  // stages [first, first + stages), an even number of them
  int first = 0, stages = (int)(a.ldk / kBK);
  if (SHARED) {
    const int pairs = stages / 2;
    first = (int)((int64_t)pairs * share / a.shares) * 2;
    stages = (int)((int64_t)pairs * (share + 1) / a.shares) * 2 - first;
  }
  const int64_t prow = (int64_t)a.tm * BT, qrow = SYM ? prow : (int64_t)a.tn * BT;
  const int load_at = load_place(wave * 16, lane), read_at = read_place(lane);
  const int64_t pat = b * a.pstride + (int64_t)ti * BT * kBK, qat = b * a.qstride + (int64_t)tj * BT * kBK;
  auto load = [&](int s) {
    const int64_t p = pat + (first + s) * prow * kBK, q = qat + (first + s) * qrow * kBK;
    auto& to = lds[s % kStages];
    load_tile<BT, NW>(a.ph + p, to[0], wave, load_at);
    load_tile<BT, NW>(a.qh + q, to[1], wave, load_at);
    if constexpr (SPLIT) {
      load_tile<BT, NW>(a.pl + p, to[2], wave, load_at);
      load_tile<BT, NW>(a.ql + q, to[3], wave, load_at);
    }
  };
  struct Frags {
    half8 p[OPS / 2][MI], q[OPS / 2][NJ];
  };
  auto read_from = [&](const _Float16* ph, const _Float16* qh, const _Float16* pl, const _Float16* ql, Frags& f) {
#pragma unroll
    for (int h = 0; h < OPS / 2; ++h) {
#pragma unroll
      for (int i = 0; i < MI; ++i) f.p[h][i] = *(const half8*)((h ? pl : ph) + wm * kBK + fragment_at(i) + read_at);
#pragma unroll
      for (int j = 0; j < NJ; ++j) f.q[h][j] = *(const half8*)((h ? ql : qh) + wn * kBK + fragment_at(j) + read_at);
    }
  };
  auto read = [&](int s, Frags& f) {
    const auto& from = lds[s % kStages];
    read_from(from[0], from[1], from[2 % OPS], from[3 % OPS], f);
  };
  auto multiply = [&](const Frags& f) {
    auto products = [&](const half8(&p)[MI], const half8(&q)[NJ]) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[i], q[j], acc[i][j], 0, 0, 0);
    };
    products(f.p[0], f.q[0]);
    if constexpr (SPLIT) {  // low by low is beyond the 22 bits
      products(f.p[0], f.q[1]);
      products(f.p[1], f.q[0]);
    }
  };
  // Stage s: at most `flying` loads stay under way (those of stage s + 2), and of the reads only this stage's own: the
  // products of stage s - 1, and with them the wait for its fragments, may be scheduled past the barrier, but its place
  // is given away behind it.  Without branches, so that the compiler knows which reads are outstanding and waits for
  // those of this stage only.
  constexpr int READS = OPS / 2 * (MI + NJ);
  auto step = [&](auto flying, auto loads, int s, Frags& now, Frags& next) {
    wait_for<decltype(flying)::value, READS>();
    block_barrier();
    if (decltype(loads)::value) load(s + 3);
    read(s + 1, next);
    multiply(now);
  };
  using std::integral_constant;
  const integral_constant<int, LOADS> two;
  const integral_constant<int, 0> none;
  const integral_constant<int, 1> more;
  Frags f0, f1;
  load(0);
  load(1);  // stages is even: sides are multiples of 64
  if (stages > 2) {
    load(2);
    wait_for<2 * LOADS, 0>();
  } else {
    wait_for<LOADS, 0>();
  }
  block_barrier();
  read(0, f0);
  if (stages > 2) {
    int s = 0;
    for (; s + 4 < stages; s += 2) {
      step(two, more, s, f0, f1);
      step(two, more, s + 1, f1, f0);
    }
    step(two, more, s, f0, f1);
    step(two, none, s + 1, f1, f0);
  }
  step(none, none, stages - 2, f0, f1);
  multiply(f1);
  asm volatile("" : "+v"(lane));  // what the epilogue derives from it is not worth registers during the products

  if constexpr (SHARED) {
    // Each share's sums go to memory; the block that is last to arrive adds them up, in the order of the shares.
    // They are written and read past the caches of the XCDs (relaxed atomics of the card's scope), so that no
    // block has to write back or drop a whole cache: with fences this launch took four times as long.
    constexpr int N = MI * NJ * 2 * NW * 64;    // 8-byte words of a tile
    constexpr int kAtOnce = BT == 64 ? 4 : 1;  // shares under way
    uint64_t* part = a.part + (int64_t)tile * a.shares * N;
    const int at = wave * MI * NJ * 128 + lane;
#pragma unroll
    for (int i = 0; i < MI * NJ * 2; ++i) {
      const float4v v = acc[i / 2 / NJ][i / 2 % NJ];
      const float2v w = {v[i % 2 * 2], v[i % 2 * 2 + 1]};
      __hip_atomic_store(part + (int64_t)share * N + at + i * 64, __builtin_bit_cast(uint64_t, w), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they have arrived
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
      last = __hip_atomic_fetch_add(a.arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.shares - 1;
      if (last) __hip_atomic_store(a.arrived + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
#pragma unroll
    for (int i = 0; i < MI * NJ; ++i) acc[i / NJ][i % NJ] = float4v{};
    for (int k = 0; k < a.shares; k += kAtOnce) {
      uint64_t u[kAtOnce][MI * NJ * 2];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q)
#pragma unroll
        for (int i = 0; i < MI * NJ * 2; ++i)
          u[q][i] = __hip_atomic_load(part + (int64_t)min(k + q, a.shares - 1) * N + at + i * 64, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        if (k + q >= a.shares) break;
#pragma unroll
        for (int i = 0; i < MI * NJ * 2; ++i) {
          const float2v w = __builtin_bit_cast(float2v, u[q][i]);
          acc[i / 2 / NJ][i / 2 % NJ][i % 2 * 2] += w[0];
          acc[i / 2 / NJ][i / 2 % NJ][i % 2 * 2 + 1] += w[1];
        }
      }
    }
  }

  // BOTH: the steps of A = X X^T in LDS.  With q(A) = a + b A + c A A a step is X <- q(A) X, so A <- q(A) A q(A), and
  // after some steps X <- P X with P the product of the q(A): all are polynomials of the first A, symmetric and
  // commuting.  P is formed here, and X read and written once for all of them.  A place in LDS holds a matrix as
  // operands (two panels, both halves, times the scale); of what a product gives, the lower triangle is kept and
  // mirrored (left unsymmetric, the rounding grows from step to step).  One block a matrix is slow at it, but nine
  // products are three steps, and those were a launch of 4 us for X and one of 8 us for A and B each: 3 x (64 x 576)
  // took 69 us step by step.
  if constexpr (EPI == BOTH) {
    static_assert(BT == 64 && SPLIT && kStages == 4, "a matrix takes the place of a stage");
    enum { kA, kZ, kP, kR };
    const int r = (int)row_at(0), cq = (int)column_at(0) - lane % 4;  // rows r .. r + 7 of columns cq .. cq + 7
    auto place = [&](int m, int half, int c, int row) {               // rows row .. row + 7 of column c
      return (half8*)&lds[m][2 * half + row / kBK][c * kBK + ((row % kBK / 8) ^ swizzle(c)) * 8];
    };
    auto put = [&](int m) {  // acc, which holds the matrix times the scale
      half8 h[2], l[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = acc[e / 4][y][e % 4];
          h[y][e] = (_Float16)v;
          l[y][e] = (_Float16)(v - (float)h[y][e]);
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const half8 th = transpose8(h[0], h[1], x, lane), tl = transpose8(l[0], l[1], x, lane);
        const int c = cq + 4 * x + lane % 4;  // of this lane, and, where r = cq, the row that th is of
        if (r > cq) {
          *place(m, 0, c, r) = h[x];
          *place(m, 1, c, r) = l[x];
          *place(m, 0, r + 4 * x + lane % 4, cq) = th;
          *place(m, 1, r + 4 * x + lane % 4, cq) = tl;
        } else if (r == cq) {
          half8 sh, sl;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sh[e] = r + e >= c ? h[x][e] : th[e];
            sl[e] = r + e >= c ? l[x][e] : tl[e];
          }
          *place(m, 0, c, r) = sh;
          *place(m, 1, c, r) = sl;
        }
      }
    };
    auto combine = [&](int z, int y, float alpha, float beta) {  // acc = alpha Y + beta Z Y
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[0][j] = acc[1][j] = float4v{};
#pragma unroll
      for (int s = 0; s < BT / kBK; ++s) {
        read_from(lds[z][s], lds[y][s], lds[z][2 + s], lds[y][2 + s], f0);
        multiply(f0);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const half8 yh = *place(y, 0, cq + 4 * j + lane % 4, r), yl = *place(y, 1, cq + 4 * j + lane % 4, r);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          acc[e / 4][j][e % 4] = fmaf(beta * kInvScale, acc[e / 4][j][e % 4], alpha * pair(yh[e], yl[e]));
      }
    };
#pragma unroll
    for (int i = 0; i < MI * NJ; ++i) acc[i / NJ][i % NJ] *= kInvScale;
    __syncthreads();  // the stages are read
    put(kA);
    __syncthreads();
    for (int k = 0; k < a.steps; ++k) {
      const float qa = k == 0 ? coef[0][0] : k == 1 ? coef[1][0] : coef[2][0];
      const float qb = k == 0 ? coef[0][1] : k == 1 ? coef[1][1] : coef[2][1];
      const float qc = k == 0 ? coef[0][2] : k == 1 ? coef[1][2] : coef[2][2];
      combine(kA, kA, qb, qc);  // Z = b A + c A A, q(A) = a + Z
      put(kZ);
      if (k == 0) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (r + e == cq + 4 * j + lane % 4) acc[e / 4][j][e % 4] += qa * kScale;
        put(kP);
      }
      __syncthreads();
      if (k) {
        combine(kZ, kP, qa, 1.0f);
        __syncthreads();  // P is read
        put(kP);
      }
      if (k + 1 < a.steps) {
        combine(kZ, kA, qa, 1.0f);
        put(kR);
        __syncthreads();
        combine(kZ, kR, qa, 1.0f);
        put(kA);  // (read by the product before the barrier, not by this one)
      }
      __syncthreads();
    }
    // P goes where B goes, its diagonal apart
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = cq + 4 * j + lane % 4;
      half8 h = *place(kP, 0, c, r), l = *place(kP, 1, c, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (r + e == c) {
          a.dB[b * a.Mp + c] = pair(h[e], l[e]) * kInvScale;
          h[e] = l[e] = (_Float16)0.0f;
        }
      }
      const int64_t at = b * a.ostride + panel_at(c, r, a.Mp);
      *(half8*)(a.oh + at) = h;
      *(half8*)(a.ol + at) = l;
    }
    return;
  }

  // Two pairs of fragments at a time: rows r .. r + 7 of columns c and c + 4; transposed, rows rq and rq + 4 of
  // columns cq .. cq + 7.
#pragma unroll
  for (int i = 0; i < MI; i += 2) {
#pragma unroll
    for (int j = 0; j < NJ; j += 2) {
      const int64_t r = row_at(i), rq = r + lane % 4;
      const int64_t cq = column_at(j) - lane % 4;
      float v[2][8];  // [column][row]
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int64_t c = column_at(j + y);
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = acc[i + e / 4][j + y][e % 4];
        if (EPI == GRAM) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[y][e] = d[e] * kInvScale;  // A times the scale
            if (r + e == c) {
              a.dA[b * a.Mp + c] = v[y][e] * kInvScale;
              v[y][e] = 0.0f;
            }
          }
          continue;
        }
        half8 h = {}, l = {}, zh = {}, zl = {};
        float dc = 0.0f;
        float4v dr[2] = {};
        if constexpr (EARLY) {
          h = inh[i / 2][j + y];
          l = inl[i / 2][j + y];
          dc = dcol[j + y];
          dr[0] = drow[i / 2][0];
          dr[1] = drow[i / 2][1];
          if (EPI == MULT) {
            zh = inzh[EPI == MULT ? i / 2 : 0][EPI == MULT ? j + y : 0];
            zl = inzl[EPI == MULT ? i / 2 : 0][EPI == MULT ? j + y : 0];
          }
        } else {
          ask(i, j + y, h, l, dc, dr, zh, zl);
        }
        if (EPI == POLY) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float o = pair(h[e], l[e]);
            // (D + O)^2 = D^2 + D O + O D + O O
            v[y][e] = fmaf(cc, fmaf(dr[e / 4][e % 4] + dc, o, d[e] * kInvScale), cb * o);
            if (r + e == c) {
              const float on = fmaf(cc, fmaf(dc, dc, d[e] * kInvScale * kInvScale), cb * dc);
              a.dB[b * a.Mp + c] = on;
              if (a.dP) a.dP[b * a.Mp + c] = ca + on;
              v[y][e] = 0.0f;
            }
          }
        } else if (EPI == MULT) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float o = pair(h[e], l[e]), z = pair(zh[e], zl[e]), dz = dr[e / 4][e % 4];
            v[y][e] = fmaf(dz, o, fmaf(z, dc, d[e] * kInvScale)) + ca * o;
            if (r + e == c) {
              a.dB[b * a.Mp + c] = fmaf(dz, dc, d[e] * kInvScale * kInvScale) + ca * dc;
              v[y][e] = 0.0f;
            }
          }
        } else {  // rows are the long side, columns the short one
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float hi = (float)h[e], x = pair(h[e], l[e]);
            v[y][e] = fmaf(ca, x, fmaf(dc, SPLIT || EPI == LAST ? x : hi, d[e] * kInvScale));
          }
        }
      }
      if (EPI == LAST) {
        store_last(a, b, r, rq, cq, lane, scale, v);
        continue;
      }
      half8 h[2], l[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[y][e] = (_Float16)v[y][e];
          l[y][e] = (_Float16)(v[y][e] - (float)h[y][e]);
        }
        const int64_t c = cq + 4 * y + lane % 4;
        if (!SYM) {
          const int64_t at = b * a.Mp * a.Np + panel_at(c, r, a.Mp);
          *(half8*)(a.xh + at) = h[y];
          *(half8*)(a.xl + at) = l[y];
        } else if (!SPLIT || ti != tj) {
          const int64_t at = b * a.ostride + panel_at(c, r, a.Mp);
          *(half8*)(a.oh + at) = h[y];
          if (SPLIT) *(half8*)(a.ol + at) = l[y];
        }
      }
      // Of a symmetric matrix a tile below the diagonal has its mirror image elsewhere.  A tile on it has both halves:
      // 11 bits do not show that they differ; of 22, what is below the diagonal is kept and mirrored.
      if (SYM && !SPLIT && ti == tj) continue;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const half8 th = transpose8(h[0], h[1], x, lane), tl = SPLIT ? transpose8(l[0], l[1], x, lane) : half8{};
        if (!SYM) {
          const int64_t to = b * a.ostride + panel_at(rq + 4 * x, cq, a.Np);
          *(half8*)(a.oh + to) = th;
          if (SPLIT) *(half8*)(a.ol + to) = tl;
          continue;
        }
        const int64_t c = cq + 4 * x + lane % 4;
        const int64_t at = b * a.ostride + panel_at(c, r, a.Mp), to = b * a.ostride + panel_at(rq + 4 * x, cq, a.Mp);
        if (ti != tj) {
          *(half8*)(a.oh + to) = th;
          if (SPLIT) *(half8*)(a.ol + to) = tl;
        } else if (SPLIT && r >= cq) {
          half8 sh = h[x], sl = l[x];
          if (r == cq) {  // th is of row c
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (r + e < c) sh[e] = th[e];
              if (r + e < c) sl[e] = tl[e];
            }
          } else {
            *(half8*)(a.oh + to) = th;
            *(half8*)(a.ol + to) = tl;
          }
          *(half8*)(a.oh + at) = sh;
          *(half8*)(a.ol + at) = sl;
        }
      }
    }
  }
}

// ------------------------------------------------------------------ layout

struct Plan {
  int64_t rows, cols, batch, m, n, Mp, Np;
  int tall, nparts, lg_tx;
  int tile, gram_tile, poly_tile;  // of STEP and LAST, GRAM and BOTH, POLY
  bool split;
  bool gram_space;  // a few steps at a time by their Gram matrix (m > 64: by MULT)
  int shares;      // of a GRAM tile's k
  int64_t tiles;   // GRAM's, if it has shares
  size_t gpart, arrived;
  size_t part, table, dA, dB, xh, xl, th[2], tl[2], ah, al, bh, bl, total;
  size_t sq[10], sqd[6];  // gram_space: R, two Z, two P, high and low; their diagonals and that of the first P
};

constexpr int64_t kCUs = 256;

// Microseconds that a launch's tiles take for one stage of 32 k, by how they fill the card: one block a CU with tiles
// of 256 (one of 128 in split mode), two of 128 (64 in split mode), four of 64.  Fitted to the time of whole calls, so
// a share of their epilogues and last rounds is in them: a full card comes to 1.23 PFLOP/s of products with tiles of
// 256, 0.90 with 128 and 0.67 with 64 (in split mode 1.30 with 128 and 0.89 with 64).  Smaller tiles fill it sooner:
// one matrix of 1000 x 1601 takes 184 us with tiles of 64, 279 with 128 and 528 with 256; four of 2048 x 2048 take
// 1,213, 1,029 and 933 us.  At 19 sizes of 1 to 24 matrices of 512 to 4,096, either products, what the rule takes is
// within 4% of the best of one tile for all.
double stage_us(int tile, bool split, int64_t tiles) {
  const int per = (tile == 64 ? 4 : tile == 128 ? 2 : 1) / (split ? 2 : 1);
  // of a card with 1, 2, .. `per` blocks a CU
  static const double k64[4] = {0.20, 0.25, 0.31, 0.40}, k128[2] = {0.36, 0.60}, k256[1] = {0.87};
  static const double s64[2] = {0.28, 0.45}, s128[1] = {0.62};
  const double* us = split ? (tile == 64 ? s64 : s128) : tile == 64 ? k64 : tile == 128 ? k128 : k256;
  const int64_t a_cu = ceil_div(tiles, kCUs), full = a_cu / per, rest = a_cu % per;
  return (double)full * us[per - 1] + (rest ? us[rest - 1] : 0.0);
}

// Blocks that share the k of a GRAM tile, as far as the tiles leave the card empty.  A stage takes about 0.25 us and
// adding up a share 0.35 us, so their sum is least at the square root of 0.7 of the stages.  Whole calls: 256 x 2304 in
// pairs 142 us with the 7 shares that this gives, 170 with one, 196 with 2, 135 at best (12); 3 x (65 x 3000) 137 with
// 8, 185 with one.  Where it gives two or three there is nothing to gain: 1000 x 1601 takes 183 us with 3 and 180 with
// one, in pairs 243 and 232, and 5 x (513 x 1100), tiles of 128, 212 and 178.
int shares_of(int64_t tiles, int64_t stages, int tile) {
  if (tile == 256) return 1;  // built without
  const int64_t free = (tile == 64 ? 2 : 1) * kCUs / (tiles > 0 ? tiles : 1);
  const int64_t best = (int64_t)sqrt(0.7 * (double)stages);
  const int64_t n = free < best ? free : best;
  return n < 1 ? 1 : (int)n;
}

int64_t below_diagonal(int64_t tm) { return tm * (tm + 1) / 2; }

// The tiles of each product: the cheapest for a STEP, whose tile the sides are padded to, then for the others the
// cheapest of those that divide it.  Returns the microseconds of a GRAM and a STEP, and of a product of m x m.
struct Cost {
  double x, square;
};
Cost choose_tiles(Plan* p) {
  const int most = p->split ? 128 : 256;
  p->tile = p->gram_tile = p->poly_tile = 64;
  if (p->m <= 64) return Cost{};  // A is one tile
  auto padded = [](int64_t x, int t) { return ceil_div(x, t) * t; };
  double best = 0.0;
  for (int t = 64; t <= most; t *= 2) {
    const int64_t M = padded(p->m, t), N = padded(p->n, t);
    const double us = stage_us(t, p->split, p->batch * (M / t) * (N / t)) * (double)(M / kBK);
    if (t == 64 || us < best) best = us, p->tile = t;
  }
  const int64_t M = padded(p->m, p->tile), N = padded(p->n, p->tile);
  double best_gram = 0.0, best_poly = 0.0;
  for (int t = 64; t <= p->tile; t *= 2) {
    const int64_t tiles = p->batch * below_diagonal(M / t);
    const int shares = shares_of(tiles, N / kBK, t);
    // (a share is added up in 0.35 us with tiles of 64, in four times that with 128)
    const double gram = stage_us(t, p->split, tiles * shares) * (double)(N / kBK) / shares +
                        (shares > 1 ? 0.35 * shares * (t / 64) * (t / 64) : 0.0);
    const double poly = stage_us(t, p->split, tiles) * (double)(M / kBK);
    if (t == 64 || gram < best_gram) best_gram = gram, p->gram_tile = t;
    if (t == 64 || poly < best_poly) best_poly = poly, p->poly_tile = t;
  }
  // a launch takes 4 us at least; what a STEP reads and writes of X, 5 TB/s, is not hidden behind its products
  const double moved = (p->split ? 16.0 : 10.0) * (double)p->batch * (double)M * (double)N / 5e6;
  return Cost{8.0 + best_gram + best + moved, 4.0 + best_poly};
}

// Steps from the k-th on that are taken at once by the Gram matrix.  What grows a small singular value grows the
// rounding of A, P and P X as well: as far as P, whose norm is at most the product of the largest |q|, stays within 48
// (three steps of 3.4445; FP16's range ends at 64).  The error is then up to 6e-6 (4e-6 step by step), which only a
// result in FP32 from split products shows: that one goes step by step.
int block_of(const nf_orthogonal_params& o, int k, bool coarse) {
  double top = 1.0, growth = 1.0;  // of the singular values: X is scaled to at most 1
  int n = 0;
  for (int i = 0; i < k + kBlock && i < o.steps; ++i) {
    const float* c = o.coef[i];
    double most = 0.0, next = 0.0;
    for (int j = 0; j <= 64; ++j) {
      const double sv = top * j / 64, q = fabs(c[0] + sv * sv * (c[1] + sv * sv * c[2]));
      most = fmax(most, q);
      next = fmax(next, sv * q);
    }
    top = next;
    if (i < k) continue;
    growth *= fmax(most, 1.0);
    if (n > 0 && (!coarse || !(growth <= 48.0))) break;
    ++n;
  }
  return n;
}

// What o's steps come to, taken at once as far as block_of goes: products with X, and products of m x m.
struct Schedule {
  int rounds, squares;
};
Schedule schedule_of(const nf_orthogonal_params& o, bool coarse) {
  Schedule s = {};
  for (int k = 0, taken; k < o.steps; k += taken, ++s.rounds) {
    taken = block_of(o, k, coarse);
    s.squares += 4 * taken - 3;
  }
  return s;
}

// Steps at a time by the Gram matrix, where that is sooner: of five steps (three and two), X is read and written for
// two, and there are fourteen products of m x m in place of five, all of split operands.  Both five such steps and
// the call's own have to be sooner: a workspace has room for what five take (o = nullptr), and so serves any steps.
// 8 x (300 x 16,384) takes 848 us, 1,114 step by step; 40 x (1024 x 2048) would take 4,448 in place of 2,456.
// At 38 sizes with five steps the rule took the sooner form at 31 and one at most 6% slower at five; 40 x (300 x 2048)
// (614 us, 487 step by step) and 8 x (1024 x 16,384) (4,193 and 3,705) go the slower way.
void choose_form(Plan* p, bool coarse, const nf_orthogonal_params* o) {
  Plan q = *p;
  q.split = true;
  const Cost by_step = choose_tiles(p);
  if (p->m <= 64 || !coarse) return;
  const Cost by_gram = choose_tiles(&q);
  auto sooner = [&](int steps, Schedule s) {
    return s.rounds * by_gram.x + s.squares * by_gram.square < steps * (by_step.x + by_step.square);
  };
  if (sooner(5, Schedule{2, 14}) && (!o || sooner(o->steps, schedule_of(*o, coarse)))) {
    *p = q;
    p->gram_space = true;
  }
}

// Sizes are checked by the caller.  o: the steps, or nullptr for the room that a workspace has.
Plan plan_of(int64_t rows, int64_t cols, int64_t batch, bool split, bool coarse, const nf_orthogonal_params* o) {
  Plan p = {};
  p.rows = rows;
  p.cols = cols;
  p.batch = batch;
  p.tall = rows > cols;
  p.m = p.tall ? cols : rows;
  p.n = p.tall ? rows : cols;
  // a short side of few rows has few roundings to average out (3.4e-3 measured at 1 x 7), and costs launches,
  // not products: always in pairs
  p.split = split || p.m <= 64;
  choose_form(&p, coarse, o);
  p.Mp = ceil_div(p.m, p.tile) * p.tile;
  p.Np = ceil_div(p.n, p.tile) * p.tile;
  p.nparts = (int)(ceil_div(rows * cols, kNormElems) < kMaxParts ? ceil_div(rows * cols, kNormElems) : kMaxParts);
  while (p.lg_tx < 8 && (4 << p.lg_tx) < cols) ++p.lg_tx;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  const size_t x = (size_t)(2 * batch * p.Mp * p.Np), a = (size_t)(2 * batch * p.Mp * p.Mp);
  p.part = take((size_t)(8 * batch * p.nparts));
  p.table = take(sizeof(Steps) * (size_t)batch);
  p.dA = take((size_t)(4 * batch * p.Mp));
  p.dB = take((size_t)(4 * batch * p.Mp));
  p.xh = take(x);
  p.xl = take(x);
  p.th[0] = take(x);
  p.th[1] = take(x);
  const bool one = p.m <= 64;  // A never leaves its block
  if (!one) p.ah = take(a);
  p.bh = take(a);
  if (p.gram_space) {
    for (size_t& o : p.sq) o = take(a);
    for (size_t& o : p.sqd) o = take((size_t)(4 * batch * p.Mp));
  }
  if (p.split) {
    p.tl[0] = take(x);
    p.tl[1] = take(x);
    if (!one) p.al = take(a);
    p.bl = take(a);
  }
  const int64_t tiles = batch * below_diagonal(p.Mp / p.gram_tile);
  p.shares = shares_of(tiles, p.Np / kBK, p.gram_tile);
  if (p.shares > 1) {
    p.gpart = take((size_t)(4 * tiles * p.shares * p.gram_tile * p.gram_tile));
    p.arrived = take((size_t)(4 * tiles));
    p.tiles = tiles;
  }
  p.total = at;
  return p;
}

template <int EPI, bool SPLIT>
hipError_t launch_prod(const Plan& p, const ProdArgs& a, int64_t tiles, hipStream_t s) {
  const unsigned grid = (unsigned)(tiles * p.batch);
  const int tile = EPI == GRAM || EPI == BOTH ? p.gram_tile : EPI == POLY || EPI == MULT ? p.poly_tile : p.tile;
  auto go = [&](auto shared, unsigned blocks) {
    constexpr bool S = decltype(shared)::value;
    if constexpr (EPI == BOTH) {
      k_prod<64, 32, 32, true, EPI, S><<<blocks, 256, 0, s>>>(a);
    } else if constexpr (SPLIT) {
      if (tile == 64)
        k_prod<64, 32, 32, true, EPI, S><<<blocks, 256, 0, s>>>(a);
      else
        k_prod<128, 64, 32, true, EPI, S><<<blocks, 512, 0, s>>>(a);
    } else {
      if (tile == 64)
        k_prod<64, 32, 32, false, EPI, S><<<blocks, 256, 0, s>>>(a);
      else if (tile == 128)
        k_prod<128, 64, 64, false, EPI, S><<<blocks, 256, 0, s>>>(a);
      else if constexpr (!S)
        k_prod<256, 128, 64, false, EPI><<<blocks, 512, 0, s>>>(a);
    }
  };
  if constexpr (EPI == GRAM || EPI == BOTH) {
    if (p.shares > 1) {
      go(std::true_type{}, grid * p.shares);
      return hipGetLastError();
    }
  }
  go(std::false_type{}, grid);
  return hipGetLastError();
}

template <int EPI>
hipError_t launch_prod(const Plan& p, const ProdArgs& a, int64_t tiles, hipStream_t s) {
  if constexpr (EPI == BOTH || EPI == MULT)
    return launch_prod<EPI, true>(p, a, tiles, s);
  else
    return p.split ? launch_prod<EPI, true>(p, a, tiles, s) : launch_prod<EPI, false>(p, a, tiles, s);
}

// coarse: the result need not be closer than about 1e-5.
hipError_t run(const Plan& p, PrepArgs pa, ProdArgs last, const nf_orthogonal_params& o, bool coarse, void* ws,
               hipStream_t s) {
  unsigned char* w = static_cast<unsigned char*>(ws);
  auto half = [&](size_t at) { return reinterpret_cast<_Float16*>(w + at); };
  pa.rows = p.rows;
  pa.cols = p.cols;
  pa.tall = p.tall;
  pa.Mp = p.Mp;
  pa.Np = p.Np;
  pa.part = reinterpret_cast<double*>(w + p.part);
  pa.nparts = p.nparts;
  pa.lg_tx = p.lg_tx;
  pa.eps = o.eps;
  pa.steps = o.steps;
  memcpy(pa.coef, o.coef, sizeof(pa.coef));
  pa.table = reinterpret_cast<Steps*>(w + p.table);
  pa.xh = half(p.xh);
  pa.xl = half(p.xl);
  pa.th = half(p.th[0]);
  pa.tl = p.split ? half(p.tl[0]) : nullptr;
  pa.arrived = reinterpret_cast<int32_t*>(w + p.arrived);
  pa.tiles = p.tiles;
  k_norm<<<dim3((unsigned)p.nparts, (unsigned)p.batch), kNormThreads, 0, s>>>(pa);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // the caller's matrix with both sides padded
  const int64_t rp = p.tall ? p.Np : p.Mp, cp = p.tall ? p.Mp : p.Np;
  k_scale<<<dim3((unsigned)(cp / 64), (unsigned)(rp / 64), (unsigned)p.batch), kNormThreads, 0, s>>>(pa);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  const int64_t tm = p.Mp / p.tile, tn = p.Np / p.tile;
  for (int k = 0, turn = 0, taken = 1; k < o.steps; k += taken, ++turn) {
    ProdArgs g = last;
    g.table = pa.table;
    g.k = k;
    g.dA = reinterpret_cast<float*>(w + p.dA);
    g.dB = reinterpret_cast<float*>(w + p.dB);
    g.Mp = p.Mp;
    g.Np = p.Np;
    g.m = p.m;
    g.n = p.n;
    g.tall = p.tall;
    g.shares = p.shares;
    g.part = reinterpret_cast<uint64_t*>(w + p.gpart);
    g.arrived = reinterpret_cast<int32_t*>(w + p.arrived);
    g.xh = half(p.xh);
    g.xl = half(p.xl);

    _Float16 *bh = half(p.bh), *bl = p.split ? half(p.bl) : nullptr;  // what STEP multiplies X by
    ProdArgs x = g;  // A = X X^T
    x.ph = x.qh = half(p.xh);
    x.pl = x.ql = half(p.xl);
    x.ldk = p.Np;
    x.pstride = x.qstride = p.Mp * p.Np;
    x.tm = x.tn = (int32_t)(p.Mp / p.gram_tile);
    x.oh = half(p.ah);
    x.ol = p.split ? half(p.al) : nullptr;
    x.ostride = p.Mp * p.Mp;
    if (p.m <= 64) {
      taken = block_of(o, k, coarse);
      x.steps = taken;
      x.oh = half(p.bh);
      x.ol = half(p.bl);
      if ((e = launch_prod<BOTH>(p, x, 1, s)) != hipSuccess) return e;
      g.whole = 1;
    } else if (p.gram_space) {
      taken = block_of(o, k, coarse);
      if ((e = launch_prod<GRAM>(p, x, below_diagonal(x.tm), s)) != hipSuccess) return e;
      // A <- q(A) A q(A) by R = q(A) A, and P, the product of the q(A) = a + Z so far
      struct Square {
        _Float16 *h, *l;
        float* d;
      };
      auto square = [&](int i, int d) {
        return Square{half(p.sq[2 * i]), half(p.sq[2 * i + 1]), reinterpret_cast<float*>(w + p.sqd[d])};
      };
      const Square A = {half(p.ah), half(p.al), g.dA}, R = square(0, 0), Z[2] = {square(1, 1), square(2, 2)},
                   Q[2] = {square(3, 3), square(4, 4)};
      ProdArgs y = x;
      y.ldk = p.Mp;
      y.pstride = y.qstride = p.Mp * p.Mp;
      y.tm = y.tn = (int32_t)(p.Mp / p.poly_tile);
      const int64_t tiles = below_diagonal(y.tm);
      auto multiply = [&](const Square& z, const Square& with, const Square& to) {
        y.ph = z.h;
        y.pl = z.l;
        y.dZ = z.d;
        y.qh = y.ah = with.h;
        y.ql = y.al = with.l;
        y.dA = with.d;
        y.oh = to.h;
        y.ol = to.l;
        y.dB = to.d;
        return launch_prod<MULT>(p, y, tiles, s);
      };
      Square P = {};
      for (int i = 0; i < taken; ++i) {
        y.k = k + i;
        const Square& z = Z[i & 1];
        y.ph = y.qh = y.ah = A.h;  // Z = b A + c A A
        y.pl = y.ql = y.al = A.l;
        y.dA = A.d;
        y.oh = z.h;
        y.ol = z.l;
        y.dB = z.d;
        y.dP = i == 0 ? reinterpret_cast<float*>(w + p.sqd[5]) : nullptr;
        if ((e = launch_prod<POLY>(p, y, tiles, s)) != hipSuccess) return e;
        if (i == 0) {
          P = Square{z.h, z.l, y.dP};  // differs from Z in its diagonal only
        } else {
          if ((e = multiply(z, P, Q[i & 1])) != hipSuccess) return e;
          P = Q[i & 1];
        }
        if (i + 1 < taken) {
          if ((e = multiply(z, A, R)) != hipSuccess) return e;
          if ((e = multiply(z, R, A)) != hipSuccess) return e;
        }
      }
      bh = P.h;
      bl = P.l;
      g.dB = P.d;
      g.whole = 1;
    } else {
      if ((e = launch_prod<GRAM>(p, x, below_diagonal(x.tm), s)) != hipSuccess) return e;
      x.ph = x.qh = x.ah = half(p.ah);  // B = b A + c A A
      x.pl = x.ql = x.al = p.split ? half(p.al) : nullptr;
      x.ldk = p.Mp;
      x.pstride = x.qstride = p.Mp * p.Mp;
      x.oh = half(p.bh);
      x.ol = p.split ? half(p.bl) : nullptr;
      x.tm = x.tn = (int32_t)(p.Mp / p.poly_tile);
      if ((e = launch_prod<POLY>(p, x, below_diagonal(x.tm), s)) != hipSuccess) return e;
    }

    const int from = turn & 1;  // X^T <- X^T B: rows of the long side
    x = g;
    x.ph = half(p.th[from]);
    x.pl = p.split ? half(p.tl[from]) : nullptr;
    x.qh = bh;
    x.ql = bl;
    x.ldk = p.Mp;
    x.pstride = p.Mp * p.Np;
    x.qstride = p.Mp * p.Mp;
    x.tm = (int32_t)tn;
    x.tn = (int32_t)tm;
    x.oh = half(p.th[from ^ 1]);
    x.ol = p.split ? half(p.tl[from ^ 1]) : nullptr;
    x.ostride = p.Mp * p.Np;
    e = k + taken < o.steps ? launch_prod<STEP>(p, x, tn * tm, s) : launch_prod<LAST>(p, x, tn * tm, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------ checks

constexpr int64_t kMaxSide = 1 << 17;

nf_status bad(const char* what) { return set_error(NF_ERR_INVALID_ARG, what); }
bool finite(float x) { return x - x == 0.0f; }

const char* check_params(const nf_orthogonal_params* o) {
  if (!o) return "params is NULL";
  if (o->products != NF_PRODUCTS_SINGLE && o->products != NF_PRODUCTS_SPLIT) return "unknown products";
  if (o->steps < 1 || o->steps > NF_ORTHOGONAL_MAX_STEPS) return "steps outside [1, NF_ORTHOGONAL_MAX_STEPS]";
  if (!(o->eps >= 0.0f) || !finite(o->eps)) return "eps must be finite and >= 0";
  for (int k = 0; k < o->steps; ++k)
    for (int i = 0; i < 3; ++i)
      if (!finite(o->coef[k][i])) return "coefficients must be finite";
  return nullptr;
}

const char* check_sizes(int64_t rows, int64_t cols, int64_t batch) {
  if (rows < 0 || cols < 0 || batch < 0) return "rows, cols and batch must be >= 0";
  return nullptr;
}

bool too_large(int64_t rows, int64_t cols, int64_t batch) {
  if (rows > kMaxSide || cols > kMaxSide || batch > 65535) return true;
  // a launch has under 2^32 threads
  return ceil_div(rows, 64) * ceil_div(cols, 64) > (1ll << 23) / (batch > 0 ? batch : 1);
}

nf_status check_view(const void* p, int32_t type, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int64_t batch,
                     const char* null, const char* shape, const char* align) {
  if (!known_type(type)) return bad("unknown element type");
  if (ld < cols || (batch > 1 && overlaps(stride, rows, ld, cols))) return bad(shape);
  if (!p) return bad(null);
  if ((uintptr_t)p % type_bytes(type)) return set_error(NF_ERR_ALIGNMENT, align);
  return NF_OK;
}

nf_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (ws_bytes < need) return set_error(NF_ERR_WORKSPACE, "workspace smaller than nf_orthogonal_workspace_bytes");
  if (!ws) return set_error(NF_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)ws % 256) return set_error(NF_ERR_ALIGNMENT, "workspace not 256-byte aligned");
  return NF_OK;
}

nf_status finish(hipError_t e) {
  if (e != hipSuccess) return set_error(NF_ERR_HIP, hipGetErrorString(e));
  return set_error(NF_OK, "");
}

}  // namespace
}  // namespace nf

extern "C" {

size_t nf_orthogonal_workspace_bytes(int64_t rows, int64_t cols, int64_t batch, const nf_orthogonal_params* params) {
  if (nf::check_params(params) || nf::check_sizes(rows, cols, batch) || nf::too_large(rows, cols, batch)) return 0;
  if (rows == 0 || cols == 0 || batch == 0) return 0;
  // (a caller's results may be of any type, and its steps any: the larger of the two forms)
  const bool split = params->products == NF_PRODUCTS_SPLIT;
  const size_t fine = nf::plan_of(rows, cols, batch, split, false, nullptr).total;
  const size_t coarse = nf::plan_of(rows, cols, batch, split, true, nullptr).total;
  return fine > coarse ? fine : coarse;
}

nf_status nf_orthogonal_path(int64_t rows, int64_t cols, int64_t batch, const nf_orthogonal_params* params,
                             int32_t dst_type, nf_orthogonal_path_info* info) {
  using namespace nf;
  if (!info) return bad("info is NULL");
  *info = nf_orthogonal_path_info{};
  if (const char* w = check_params(params)) return bad(w);
  if (const char* w = check_sizes(rows, cols, batch)) return bad(w);
  if (!known_type(dst_type)) return bad("unknown element type");
  if (too_large(rows, cols, batch)) return set_error(NF_ERR_UNSUPPORTED, "matrices too large");
  if (rows == 0 || cols == 0 || batch == 0) return set_error(NF_OK, "");
  const bool coarse = params->products == NF_PRODUCTS_SINGLE || dst_type != NF_TYPE_F32;
  const Plan p = plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT, coarse, params);
  info->split = p.split;
  info->step_tile = p.tile;
  info->gram_tile = p.gram_tile;
  info->poly_tile = p.poly_tile;
  info->shares = p.shares;
  const bool one = p.m <= 64;
  const Schedule s = one || p.gram_space ? schedule_of(*params, coarse) : Schedule{params->steps, params->steps};
  info->rounds = s.rounds;
  info->squares = one ? 0 : s.squares;
  return set_error(NF_OK, "");
}

nf_status nf_orthogonalize(const void* src, int32_t src_type, int64_t src_ld, int64_t src_stride, void* dst,
                           int32_t dst_type, int64_t dst_ld, int64_t dst_stride, int64_t rows, int64_t cols,
                           int64_t batch, const nf_orthogonal_params* params, void* ws, size_t ws_bytes,
                           void* stream) {
  using namespace nf;
  if (const char* w = check_params(params)) return bad(w);
  if (const char* w = check_sizes(rows, cols, batch)) return bad(w);
  if (too_large(rows, cols, batch)) return set_error(NF_ERR_UNSUPPORTED, "matrices too large");
  if (rows == 0 || cols == 0 || batch == 0) return set_error(NF_OK, "");
  nf_status st = check_view(src, src_type, src_ld, src_stride, rows, cols, batch, "src is NULL",
                            "src_ld < cols or src_stride too small", "src not aligned to its elements");
  if (st != NF_OK) return st;
  st = check_view(dst, dst_type, dst_ld, dst_stride, rows, cols, batch, "dst is NULL",
                  "dst_ld < cols or dst_stride too small", "dst not aligned to its elements");
  if (st != NF_OK) return st;
  const bool coarse = params->products == NF_PRODUCTS_SINGLE || dst_type != NF_TYPE_F32;
  const Plan p = plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT, coarse, params);
  if ((st = check_ws(ws, ws_bytes, nf_orthogonal_workspace_bytes(rows, cols, batch, params))) != NF_OK) return st;
  PrepArgs pa = {};
  pa.g = View{const_cast<void*>(src), src_ld, src_stride, src_type};
  ProdArgs last = {};
  last.dst = View{dst, dst_ld, dst_stride, dst_type};
  return finish(run(p, pa, last, *params, coarse, ws, static_cast<hipStream_t>(stream)));
}

nf_status nf_orthogonal_update(const void* grad, int32_t grad_type, int64_t grad_ld, int64_t grad_stride,
                               float* momentum, int64_t momentum_ld, int64_t momentum_stride, void* weight,
                               int32_t weight_type, int64_t weight_ld, int64_t weight_stride, int64_t rows,
                               int64_t cols, int64_t batch, const nf_matrix_step* step,
                               const nf_orthogonal_params* params, void* ws, size_t ws_bytes, void* stream) {
  using namespace nf;
  if (const char* w = check_params(params)) return bad(w);
  if (!step) return bad("step is NULL");
  if (!finite(step->lr) || !finite(step->momentum) || !finite(step->weight_decay) || !finite(step->scale))
    return bad("lr, momentum, weight_decay and scale must be finite");
  if (step->nesterov != 0 && step->nesterov != 1) return bad("nesterov must be 0 or 1");
  if (const char* w = check_sizes(rows, cols, batch)) return bad(w);
  if (too_large(rows, cols, batch)) return set_error(NF_ERR_UNSUPPORTED, "matrices too large");
  if (rows == 0 || cols == 0 || batch == 0) return set_error(NF_OK, "");
  nf_status st = check_view(grad, grad_type, grad_ld, grad_stride, rows, cols, batch, "grad is NULL",
                            "grad_ld < cols or grad_stride too small", "grad not aligned to its elements");
  if (st != NF_OK) return st;
  st = check_view(momentum, NF_TYPE_F32, momentum_ld, momentum_stride, rows, cols, batch, "momentum is NULL",
                  "momentum_ld < cols or momentum_stride too small", "momentum not 4-byte aligned");
  if (st != NF_OK) return st;
  st = check_view(weight, weight_type, weight_ld, weight_stride, rows, cols, batch, "weight is NULL",
                  "weight_ld < cols or weight_stride too small", "weight not aligned to its elements");
  if (st != NF_OK) return st;
  const Plan p = plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT, true, params);
  if ((st = check_ws(ws, ws_bytes, nf_orthogonal_workspace_bytes(rows, cols, batch, params))) != NF_OK) return st;
  PrepArgs pa = {};
  pa.g = View{const_cast<void*>(grad), grad_ld, grad_stride, grad_type};
  pa.mom = momentum;
  pa.mom_ld = momentum_ld;
  pa.mom_stride = momentum_stride;
  pa.mu = step->momentum;
  pa.nesterov = step->nesterov;
  ProdArgs last = {};
  last.dst = View{weight, weight_ld, weight_stride, weight_type};
  last.update = 1;
  last.keep = 1.0f - step->lr * step->weight_decay;
  last.rate = step->lr * step->scale;
  return finish(run(p, pa, last, *params, true, ws, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
