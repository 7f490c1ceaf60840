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
//                STEP  X = a X + B X
//                LAST  the same, into the caller's matrix or weights
//
// With m the short side and n the long one, a step is m^2 n + m^3 + 2 m^2 n
// flops: A and A A are symmetric, so tiles on and below the diagonal are
// computed and mirrored.
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
#include <math.h>

#include "nf_internal.h"
#include "nf_types.h"

namespace nf {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr float kScale = 1024.0f;         // X, A and B in FP16 are held times this
constexpr float kInvScale = 1.0f / kScale;
constexpr int kBK = 64;                   // k of one LDS tile
constexpr int kNormThreads = 256;
constexpr int kNormElems = 16384;         // elements of a norm partial, at least
constexpr int kMaxParts = 256;

enum { GRAM, POLY, STEP, LAST };

// One matrix of the caller's, seen as rows x cols.
struct View {
  void* p;
  int64_t ld, stride;
  int32_t type;
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
  int32_t lg_tx;       // k_norm: log2 of the threads across a row
  float eps;
  _Float16 *xh, *xl, *th, *tl;  // tl: split only
};

struct ProdArgs {
  const _Float16 *ph, *pl, *qh, *ql;  // P: [tm tiles x K], Q: [tn tiles x K], K adjacent
  int64_t ldk;                        // of both, = K
  int64_t pstride, qstride;           // a matrix of the batch
  int32_t tm, tn;                     // tiles
  float a, b, c;
  _Float16 *oh, *ol;                  // GRAM: A, POLY: B (ld = rows); STEP: X^T
  int64_t old, ostride;
  const _Float16 *ah, *al;            // POLY: A
  float* dA;                          // diagonals, [batch][Mp]
  float* dB;
  _Float16 *xh, *xl;                  // STEP, LAST: X [Mp x Np]
  int64_t Mp, Np;
  View dst;                           // LAST
  int64_t m, n;                       // real short and long side
  int32_t tall;
  int32_t update;                     // 1: dst holds weights
  float keep, rate;                   // w = keep w - rate o
};

__device__ __forceinline__ float load_elem(const View& v, int64_t off) {
  if (v.type == NF_TYPE_F32) return ((const float*)v.p)[off];
  if (v.type == NF_TYPE_BF16) return to_f32(((const Bf16*)v.p)[off]);
  return (float)((const _Float16*)v.p)[off];
}
__device__ __forceinline__ void store_elem(const View& v, int64_t off, float x) {
  if (v.type == NF_TYPE_F32)
    ((float*)v.p)[off] = x;
  else if (v.type == NF_TYPE_BF16)
    ((Bf16*)v.p)[off] = from_f32<Bf16>(x);
  else
    ((_Float16*)v.p)[off] = (_Float16)x;
}

// U at (r, c), the momentum already stepped.
__device__ __forceinline__ float value_of(const PrepArgs& a, int64_t b, int64_t r, int64_t c) {
  float m = 0.0f;
  if (a.mom) {
    m = a.mom[b * a.mom_stride + r * a.mom_ld + c];
    if (!a.nesterov) return m;
  }
  const float g = load_elem(a.g, b * a.g.stride + r * a.g.ld + c);
  return a.mom ? fmaf(a.mu, m, g) : g;
}

// The block's sum of x in a fixed order, in thread 0.
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
__global__ __launch_bounds__(kNormThreads) void k_norm(PrepArgs a) {
  __shared__ double s[kNormThreads / 64];
  const int tx = 1 << a.lg_tx, ty = kNormThreads >> a.lg_tx;
  const int64_t b = blockIdx.y;
  const int x = threadIdx.x & (tx - 1), y = threadIdx.x >> a.lg_tx;
  double sum = 0.0;
  for (int64_t r = (int64_t)blockIdx.x * ty + y; r < a.rows; r += (int64_t)gridDim.x * ty) {
    for (int64_t c = x; c < a.cols; c += tx) {
      float u = load_elem(a.g, b * a.g.stride + r * a.g.ld + c);
      if (a.mom) {
        float* mp = a.mom + b * a.mom_stride + r * a.mom_ld + c;
        const float m = fmaf(a.mu, *mp, u);
        *mp = m;
        u = a.nesterov ? fmaf(a.mu, m, u) : m;
      }
      sum += (double)u * (double)u;
    }
  }
  sum = block_sum(sum, s);
  if (threadIdx.x == 0) a.part[b * a.nparts + blockIdx.x] = sum;
}

// A 64 x 64 tile of the caller's matrix, padding included: scaled, split in
// two FP16, stored as it lies and transposed.
__global__ __launch_bounds__(kNormThreads) void k_scale(PrepArgs a) {
  __shared__ double s[kNormThreads / 64];
  __shared__ float tile[64][65];
  const int64_t b = blockIdx.z;
  const double ss = block_sum(threadIdx.x < a.nparts ? a.part[b * a.nparts + threadIdx.x] : 0.0, s);
  const double norm = sqrt(ss) + (double)a.eps;
  const double inv = norm > 0.0 || norm != norm ? (double)kScale / norm : 0.0;
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  const int x = threadIdx.x % 64, y = threadIdx.x / 64;
  for (int i = y; i < 64; i += 4) {
    float v = 0.0f;
    if (r0 + i < a.rows && c0 + x < a.cols) v = (float)((double)value_of(a, b, r0 + i, c0 + x) * inv);
    tile[i][x] = v;
  }
  __syncthreads();
  const int64_t size = a.Mp * a.Np;
  // as it lies: X, or X^T where the caller's matrix is tall
  const int64_t ld0 = a.tall ? a.Mp : a.Np, ld1 = a.tall ? a.Np : a.Mp;
  _Float16* h0 = (a.tall ? a.th : a.xh) + b * size;
  _Float16* h1 = (a.tall ? a.xh : a.th) + b * size;
  _Float16* l0 = a.tall ? a.tl : a.xl;
  _Float16* l1 = a.tall ? a.xl : a.tl;
  for (int i = y; i < 64; i += 4) {
    const float v = tile[i][x], w = tile[x][i];
    const _Float16 vh = (_Float16)v, wh = (_Float16)w;
    h0[(r0 + i) * ld0 + c0 + x] = vh;
    h1[(c0 + i) * ld1 + r0 + x] = wh;
    if (l0) l0[b * size + (r0 + i) * ld0 + c0 + x] = (_Float16)(v - (float)vh);
    if (l1) l1[b * size + (c0 + i) * ld1 + r0 + x] = (_Float16)(w - (float)wh);
  }
}

// ---------------------------------------------------------------- products

typedef const __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

// Rows row0 .. row0 + BT - 1, k in [k0, k0 + 64), of src into an LDS tile of
// BT rows of 64: each wavefront moves eight rows (1 KiB) at a time straight
// into LDS, lane l the 16 bytes that belong in the l-th slot.  Slot j of row
// r holds the row's 16-byte piece j ^ (r / 2 % 8): the sixteen rows that a
// fragment read touches then lie in sixteen different 16-byte columns of the
// 64 banks.
template <int BT, int NW>
__device__ __forceinline__ void load_tile(const _Float16* src, int64_t row0, int64_t k0, int64_t ld, _Float16* lds,
                                          int wave, int lane) {
#pragma unroll
  for (int i = 0; i < BT / 8 / NW; ++i) {
    const int rb = (i * NW + wave) * 8, r = rb + lane / 8;
    const int piece = (lane % 8) ^ ((r >> 1) & 7);
    __builtin_amdgcn_global_load_lds((gptr)(uintptr_t)(src + (row0 + r) * ld + k0 + piece * 8), (lptr)(lds + rb * kBK),
                                     16, 0, 0);
  }
}

__device__ __forceinline__ half8 fragment(const _Float16* lds, int row, int piece) {
  return *(const half8*)(lds + row * kBK + ((piece ^ ((row >> 1) & 7)) * 8));
}

// D = P Q^T over one BT x BT tile, WM x WN of it per wavefront.  Lane l of a
// 16 x 16 part holds rows 4 (l / 16) .. + 3 of column l % 16.
template <int BT, int WM, int WN, bool SPLIT, int EPI>
__global__ __launch_bounds__(BT / WM * (BT / WN) * 64) void k_prod(ProdArgs a) {
  constexpr int NW = BT / WM * (BT / WN);
  constexpr bool SYM = EPI == GRAM || EPI == POLY;
  __shared__ __align__(16) _Float16 lds[2][2][BT * kBK];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t b = blockIdx.y;
  int ti, tj;
  if (SYM) {  // tiles on and below the diagonal, row by row
    const int q = blockIdx.x;
    ti = (int)((sqrtf(8.0f * (float)q + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > q) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= q) ++ti;
    tj = q - ti * (ti + 1) / 2;
  } else {
    ti = blockIdx.x / a.tn;
    tj = blockIdx.x - ti * a.tn;
  }
  const int wm = wave / (BT / WN) * WM, wn = wave % (BT / WN) * WN;
  float4v acc[WM / 16][WN / 16] = {};

  const int nk = (int)(a.ldk / kBK);
  const int steps = SPLIT ? 3 * nk : nk;
  auto load = [&](int it, int buf) {
    const int seg = SPLIT ? (it >= nk) + (it >= 2 * nk) : 0;
    const int64_t k0 = (int64_t)(it - seg * nk) * kBK;
    const _Float16* p = (seg == 2 ? a.pl : a.ph) + b * a.pstride;
    const _Float16* q = (seg == 1 ? a.ql : a.qh) + b * a.qstride;
    load_tile<BT, NW>(p, (int64_t)ti * BT, k0, a.ldk, lds[buf][0], wave, lane);
    load_tile<BT, NW>(q, (int64_t)tj * BT, k0, a.ldk, lds[buf][1], wave, lane);
  };
  load(0, 0);
  for (int it = 0; it < steps; ++it) {
    // the loads of this tile have landed in every wavefront, and every
    // wavefront is done with the buffer that the next ones go to
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int buf = it & 1;
    if (it + 1 < steps) load(it + 1, buf ^ 1);
#pragma unroll
    for (int ks = 0; ks < kBK / 32; ++ks) {
      half8 pf[WM / 16], qf[WN / 16];
#pragma unroll
      for (int i = 0; i < WM / 16; ++i) pf[i] = fragment(lds[buf][0], wm + 16 * i + lane % 16, ks * 4 + lane / 16);
#pragma unroll
      for (int j = 0; j < WN / 16; ++j) qf[j] = fragment(lds[buf][1], wn + 16 * j + lane % 16, ks * 4 + lane / 16);
#pragma unroll
      for (int i = 0; i < WM / 16; ++i)
#pragma unroll
        for (int j = 0; j < WN / 16; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[i], qf[j], acc[i][j], 0, 0, 0);
    }
  }

#pragma unroll
  for (int i = 0; i < WM / 16; ++i) {
#pragma unroll
    for (int j = 0; j < WN / 16; ++j) {
      const int64_t r = (int64_t)ti * BT + wm + 16 * i + lane / 16 * 4;  // and the three after it
      const int64_t c = (int64_t)tj * BT + wn + 16 * j + lane % 16;
      const float4v d = acc[i][j];
      if (EPI == GRAM || EPI == POLY) {
        float v[4];
        if (EPI == GRAM) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = d[e] * kInvScale;  // A times the scale
            if (r + e == c) {
              a.dA[b * a.Mp + c] = v[e] * kInvScale;
              v[e] = 0.0f;
            }
          }
        } else {
          const half4 oh = *(const half4*)(a.ah + b * a.ostride + c * a.old + r);
          half4 ol = {};
          if (SPLIT) ol = *(const half4*)(a.al + b * a.ostride + c * a.old + r);
          const float dc = a.dA[b * a.Mp + c];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float dr = a.dA[b * a.Mp + r + e], o = (float)oh[e] + (float)ol[e];
            // (D + O)^2 = D^2 + D O + O D + O O
            v[e] = fmaf(a.c, fmaf(dr + dc, o, d[e] * kInvScale), a.b * o);
            if (r + e == c) {
              a.dB[b * a.Mp + c] = fmaf(a.c, fmaf(dc, dc, d[e] * kInvScale * kInvScale), a.b * dc);
              v[e] = 0.0f;
            }
          }
        }
        half4 h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          h[e] = (_Float16)v[e];
          l[e] = (_Float16)(v[e] - (float)h[e]);
        }
        *(half4*)(a.oh + b * a.ostride + c * a.old + r) = h;
        if (SPLIT) *(half4*)(a.ol + b * a.ostride + c * a.old + r) = l;
        if (ti != tj) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a.oh[b * a.ostride + (r + e) * a.old + c] = h[e];
            if (SPLIT) a.ol[b * a.ostride + (r + e) * a.old + c] = l[e];
          }
        }
      } else {  // rows are the long side, columns the short one
        const int64_t at = b * a.Mp * a.Np + c * a.Np + r;
        const half4 xh = *(const half4*)(a.xh + at), xl = *(const half4*)(a.xl + at);
        const float q = a.dB[b * a.Mp + c];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float h = (float)xh[e], x = h + (float)xl[e];
          v[e] = fmaf(a.a, x, fmaf(q, SPLIT || EPI == LAST ? x : h, d[e] * kInvScale));
        }
        if (EPI == STEP) {
          half4 h, l;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
          }
          *(half4*)(a.xh + at) = h;
          *(half4*)(a.xl + at) = l;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a.oh[b * a.ostride + (r + e) * a.old + c] = h[e];
            if (SPLIT) a.ol[b * a.ostride + (r + e) * a.old + c] = l[e];
          }
        } else if (c < a.m) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (r + e >= a.n) break;
            const float o = v[e] * kInvScale;
            const int64_t off = b * a.dst.stride + (a.tall ? (r + e) * a.dst.ld + c : c * a.dst.ld + r + e);
            store_elem(a.dst, off, a.update ? fmaf(a.keep, load_elem(a.dst, off), -a.rate * o) : o);
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------ layout

struct Plan {
  int64_t rows, cols, batch, m, n, Mp, Np;
  int tall, tile, nparts, lg_tx;
  bool split;
  size_t part, dA, dB, xh, xl, th[2], tl[2], ah, al, bh, bl, total;
};

// Sizes are checked by the caller.
Plan plan_of(int64_t rows, int64_t cols, int64_t batch, bool split) {
  Plan p = {};
  p.rows = rows;
  p.cols = cols;
  p.batch = batch;
  p.tall = rows > cols;
  p.m = p.tall ? cols : rows;
  p.n = p.tall ? rows : cols;
  p.tile = p.m <= 64 ? 64 : 128;
  p.Mp = ceil_div(p.m, p.tile) * p.tile;
  p.Np = ceil_div(p.n, p.tile) * p.tile;
  // a short side of few rows has few roundings to average out (3.4e-3 measured at 1 x 7), and costs launches,
  // not products: always in pairs
  p.split = split || p.m <= 64;
  p.nparts = (int)(ceil_div(rows * cols, kNormElems) < kMaxParts ? ceil_div(rows * cols, kNormElems) : kMaxParts);
  while (p.lg_tx < 8 && (1 << p.lg_tx) < cols) ++p.lg_tx;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  const size_t x = (size_t)(2 * batch * p.Mp * p.Np), a = (size_t)(2 * batch * p.Mp * p.Mp);
  p.part = take((size_t)(8 * batch * p.nparts));
  p.dA = take((size_t)(4 * batch * p.Mp));
  p.dB = take((size_t)(4 * batch * p.Mp));
  p.xh = take(x);
  p.xl = take(x);
  p.th[0] = take(x);
  p.th[1] = take(x);
  p.ah = take(a);
  p.bh = take(a);
  if (p.split) {
    p.tl[0] = take(x);
    p.tl[1] = take(x);
    p.al = take(a);
    p.bl = take(a);
  }
  p.total = at;
  return p;
}

template <int EPI, bool SPLIT>
hipError_t launch_prod(const Plan& p, const ProdArgs& a, int64_t tiles, hipStream_t s) {
  const dim3 grid((unsigned)tiles, (unsigned)p.batch);
  if (p.tile == 64)
    k_prod<64, 32, 32, true, EPI><<<grid, 256, 0, s>>>(a);
  else
    k_prod<128, 64, 64, SPLIT, EPI><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int EPI>
hipError_t launch_prod(const Plan& p, const ProdArgs& a, int64_t tiles, hipStream_t s) {
  return p.split ? launch_prod<EPI, true>(p, a, tiles, s) : launch_prod<EPI, false>(p, a, tiles, s);
}

hipError_t run(const Plan& p, PrepArgs pa, ProdArgs last, const nf_orthogonal_params& o, void* ws, hipStream_t s) {
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
  pa.xh = half(p.xh);
  pa.xl = half(p.xl);
  pa.th = half(p.th[0]);
  pa.tl = p.split ? half(p.tl[0]) : nullptr;
  k_norm<<<dim3((unsigned)p.nparts, (unsigned)p.batch), kNormThreads, 0, s>>>(pa);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // the caller's matrix with both sides padded
  const int64_t rp = p.tall ? p.Np : p.Mp, cp = p.tall ? p.Mp : p.Np;
  k_scale<<<dim3((unsigned)(cp / 64), (unsigned)(rp / 64), (unsigned)p.batch), kNormThreads, 0, s>>>(pa);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  const int64_t tm = p.Mp / p.tile, tn = p.Np / p.tile, sym = tm * (tm + 1) / 2;
  for (int k = 0; k < o.steps; ++k) {
    ProdArgs g = last;
    g.a = o.coef[k][0];
    g.b = o.coef[k][1];
    g.c = o.coef[k][2];
    g.dA = reinterpret_cast<float*>(w + p.dA);
    g.dB = reinterpret_cast<float*>(w + p.dB);
    g.Mp = p.Mp;
    g.Np = p.Np;
    g.m = p.m;
    g.n = p.n;
    g.tall = p.tall;
    g.xh = half(p.xh);
    g.xl = half(p.xl);

    ProdArgs x = g;  // A = X X^T
    x.ph = x.qh = half(p.xh);
    x.pl = x.ql = half(p.xl);
    x.ldk = p.Np;
    x.pstride = x.qstride = p.Mp * p.Np;
    x.oh = half(p.ah);
    x.ol = p.split ? half(p.al) : nullptr;
    x.old = p.Mp;
    x.ostride = p.Mp * p.Mp;
    if ((e = launch_prod<GRAM>(p, x, sym, s)) != hipSuccess) return e;

    x.ph = x.qh = x.ah = half(p.ah);  // B = b A + c A A
    x.pl = x.ql = x.al = p.split ? half(p.al) : nullptr;
    x.ldk = p.Mp;
    x.pstride = x.qstride = p.Mp * p.Mp;
    x.oh = half(p.bh);
    x.ol = p.split ? half(p.bl) : nullptr;
    if ((e = launch_prod<POLY>(p, x, sym, s)) != hipSuccess) return e;

    const int from = k & 1;  // X^T <- X^T B: rows of the long side
    x = g;
    x.ph = half(p.th[from]);
    x.pl = p.split ? half(p.tl[from]) : nullptr;
    x.qh = half(p.bh);
    x.ql = p.split ? half(p.bl) : nullptr;
    x.ldk = p.Mp;
    x.pstride = p.Mp * p.Np;
    x.qstride = p.Mp * p.Mp;
    x.tm = (int32_t)tn;
    x.tn = (int32_t)tm;
    x.oh = half(p.th[from ^ 1]);
    x.ol = p.split ? half(p.tl[from ^ 1]) : nullptr;
    x.old = p.Mp;
    x.ostride = p.Mp * p.Np;
    e = k + 1 < o.steps ? launch_prod<STEP>(p, x, tn * tm, s) : launch_prod<LAST>(p, x, tn * tm, s);
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
  return ceil_div(rows, 64) * ceil_div(cols, 64) > (1ll << 30) / (batch > 0 ? batch : 1);
}

nf_status check_view(const void* p, int32_t type, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int64_t batch,
                     const char* null, const char* shape, const char* align) {
  if (!known_type(type)) return bad("unknown element type");
  if (ld < cols || (batch > 1 && stride < (rows - 1) * ld + cols)) return bad(shape);
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
  return nf::plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT).total;
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
  const Plan p = plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT);
  if ((st = check_ws(ws, ws_bytes, p.total)) != NF_OK) return st;
  PrepArgs pa = {};
  pa.g = View{const_cast<void*>(src), src_ld, src_stride, src_type};
  ProdArgs last = {};
  last.dst = View{dst, dst_ld, dst_stride, dst_type};
  return finish(run(p, pa, last, *params, ws, static_cast<hipStream_t>(stream)));
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
  const Plan p = plan_of(rows, cols, batch, params->products == NF_PRODUCTS_SPLIT);
  if ((st = check_ws(ws, ws_bytes, p.total)) != NF_OK) return st;
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
  return finish(run(p, pa, last, *params, ws, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
