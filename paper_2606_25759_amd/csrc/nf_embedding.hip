// nf_embedding.hip - embedding lookup with scaling, and its gradient by
// sorted tokens.
//
//   k_lookup    out[t] = scale * table[ids[t]]
//   k_sort      tiles of a worker's tokens sorted by id in LDS (stable, so
//               tokens of one id stay in their order), while the launch's
//               other blocks zero the workers' segments
//   k_merge     pairs of sorted runs into one, until a worker has one run
//   k_partial   sums of the stretches of kChunk sorted tokens that are all of
//               one id: a frequent token's rows are summed by many wavefronts
//   k_rows_sum  a wavefront per kOwn sorted tokens and 256 columns: the rows
//               of every id that begins there
//
// All are bound by memory traffic: the gradient's floor is the dense FP32
// segment written once and dy read once.  The order in which a row's terms
// are added depends on the sorted tokens alone, so results are reproducible
// bit for bit.
#include "nf_internal.h"
#include "nf_types.h"

namespace nf {
namespace {

// ------------------------------------------------------------------ lookup

struct LookupArgs {
  const void* table;
  const void* ids;
  void* out;
  int64_t table_ld, out_ld, V, T;
  int32_t d, ids64;
  float scale;
  int32_t lg_tx;  // log2 of the threads across a row
};

__device__ __forceinline__ int64_t id_at(const void* ids, int32_t ids64, int64_t i) {
  return ids64 ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
}

template <typename T, int N>
struct alignas(sizeof(T) * N <= 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};

constexpr int kThreadsE = 256;

// N = 8: rows and bases aligned for 16-byte (FP32: two 16-byte) accesses.
template <typename A, typename B, int N>
__global__ __launch_bounds__(kThreadsE) void k_lookup(LookupArgs a) {
  const int tx = 1 << a.lg_tx, ty = kThreadsE >> a.lg_tx;
  const int x = threadIdx.x & (tx - 1);
  const int64_t t = (int64_t)blockIdx.x * ty + (threadIdx.x >> a.lg_tx);
  if (t >= a.T) return;
  const int64_t id = id_at(a.ids, a.ids64, t);
  const bool in = id >= 0 && id < a.V;
  const A* row = (const A*)a.table + (in ? id : 0) * a.table_ld;
  B* out = (B*)a.out + t * a.out_ld;
  for (int j = x * N; j < a.d; j += tx * N) {
    Pack<B, N> o;
    if (in) {
      const Pack<A, N> p = *(const Pack<A, N>*)(row + j);
#pragma unroll
      for (int e = 0; e < N; ++e) o.v[e] = from_f32<B>(to_f32(p.v[e]) * a.scale);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) o.v[e] = from_f32<B>(0.0f);
    }
    *(Pack<B, N>*)(out + j) = o;
  }
}

// -------------------------------------------------------------------- sort

constexpr int kChunk = 64;  // sorted tokens of a partial sum
constexpr int kOwn = 16;    // sorted tokens of a wavefront of k_rows_sum
constexpr int kCols = 256;  // columns of a wavefront

struct GradArgs {
  const void* dy;
  int64_t dy_ld, dy_stride;
  const void* ids;
  int64_t ids_stride;
  int32_t ids64;
  int32_t W, d;
  int64_t T, V, padding_id;
  float scale;
  int32_t accumulate;
  float* grads;
  int64_t worker_stride;
  uint32_t *key, *order;    // [W][T]: sorted runs; key V: a token that adds to no row
  uint32_t *key2, *order2;  // k_merge's result
  float* part;              // [W][T / kChunk][d]
  int64_t run;              // tokens of a sorted run
  int32_t tiles;            // k_sort: runs of a worker
  int32_t bits;             // of V
};

// Zeroes n floats at p with the blocks b of nb: whole 16-byte pieces, and
// what lies before the first and after the last one.
__device__ void fill_zero(float* p, int64_t n, int64_t b, int64_t nb) {
  const int64_t head = min((int64_t)((-(intptr_t)p) & 15) / 4, n);
  const int64_t n4 = (n - head) / 4, tail = n - head - 4 * n4;
  if (b == 0) {
    if (threadIdx.x < head) p[threadIdx.x] = 0.0f;
    if (threadIdx.x < tail) p[n - 1 - threadIdx.x] = 0.0f;
  }
  float4* q = (float4*)(p + head);
  for (int64_t i = b * blockDim.x + threadIdx.x; i < n4; i += nb * blockDim.x) q[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// Least-significant-digit radix sort of up to THREADS * ITEMS tokens, 8 bits
// a pass.  Item i of lane l of wavefront w is the (w * ITEMS + i) * 64 + l-th,
// so ranks taken wavefront by wavefront, item by item and lane by lane keep
// equal digits in order.
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void k_sort(GradArgs a) {
  constexpr int NW = THREADS / 64, CAP = THREADS * ITEMS;
  __shared__ uint32_t skey[CAP];
  __shared__ uint16_t spos[CAP];
  __shared__ uint32_t cnt[NW][256];
  __shared__ uint32_t wsum[4];
  const int64_t sorters = (int64_t)a.W * a.tiles;
  if (blockIdx.x >= sorters) {
    const int64_t nb = (gridDim.x - sorters) / a.W, f = blockIdx.x - sorters;
    fill_zero(a.grads + f / nb * a.worker_stride, a.V * a.d, f % nb, nb);
    return;
  }
  const int w = blockIdx.x / a.tiles;
  const int64_t t0 = (int64_t)(blockIdx.x % a.tiles) * CAP;
  const int count = (int)min((int64_t)CAP, a.T - t0);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint32_t key[ITEMS];
  uint16_t pos[ITEMS], rank[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int p = (wave * ITEMS + i) * 64 + lane;
    pos[i] = (uint16_t)p;
    key[i] = (uint32_t)a.V;
    if (p < count) {
      const int64_t id = id_at(a.ids, a.ids64, (int64_t)w * a.ids_stride + t0 + p);
      if (id >= 0 && id < a.V && id != a.padding_id) key[i] = (uint32_t)id;
    }
  }
  for (int shift = 0; shift < a.bits; shift += 8) {
    for (int i = threadIdx.x; i < NW * 256; i += THREADS) (&cnt[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t dg = (key[i] >> shift) & 255;
      uint64_t same = ~0ull;  // lanes with this digit
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint64_t set = __ballot((dg >> b) & 1);
        same &= (dg >> b) & 1 ? set : ~set;
      }
      const uint32_t below = (uint32_t)__popcll(same & ((1ull << lane) - 1));
      volatile uint32_t* mine = &cnt[wave][dg];  // other lanes' too
      const uint32_t before = *mine;
      rank[i] = (uint16_t)(before + below);
      __builtin_amdgcn_wave_barrier();  // every lane has read its counter
      if (same >> lane == 1) *mine = before + below + 1;  // the last of its digit
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // exclusive sums over (digit, wavefront)
    uint32_t total = 0;
    if (threadIdx.x < 256) {
      for (int v = 0; v < NW; ++v) {
        const uint32_t c = cnt[v][threadIdx.x];
        cnt[v][threadIdx.x] = total;
        total += c;
      }
    }
    uint32_t scan = total;
    if (threadIdx.x < 256) {
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(scan, o);
        if (lane >= o) scan += u;
      }
      if (lane == 63) wsum[wave] = scan;
    }
    __syncthreads();
    if (threadIdx.x < 256) {
      uint32_t base = scan - total;
      for (int v = 0; v < wave; ++v) base += wsum[v];
      for (int v = 0; v < NW; ++v) cnt[v][threadIdx.x] += base;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t p = cnt[wave][(key[i] >> shift) & 255] + rank[i];
      skey[p] = key[i];
      spos[p] = pos[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int p = (wave * ITEMS + i) * 64 + lane;
      key[i] = skey[p];
      pos[i] = spos[p];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int p = (wave * ITEMS + i) * 64 + lane;
    if (p < count) {
      a.key[(int64_t)w * a.T + t0 + p] = key[i];
      a.order[(int64_t)w * a.T + t0 + p] = (uint32_t)(t0 + pos[i]);
    }
  }
}

// Runs of a.run tokens, two and two: a token goes behind those of its own run
// before it and those of the other run with a smaller id (of the earlier run:
// or the same).
__global__ __launch_bounds__(kThreadsE) void k_merge(GradArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreadsE + threadIdx.x;
  if (i >= a.T) return;
  const uint32_t* key = a.key + (int64_t)blockIdx.y * a.T;
  const int64_t r = i / a.run, base = r / 2 * 2 * a.run;
  const int64_t o0 = min((r ^ 1) * a.run, a.T), o1 = min(o0 + a.run, a.T);
  const uint32_t k = key[i], limit = k + (r & 1);  // ids below it go first; k <= V < 2^31
  int64_t lo = o0, hi = o1;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (key[mid] < limit)
      lo = mid + 1;
    else
      hi = mid;
  }
  const int64_t to = base + (i - r * a.run) + (lo - o0);
  a.key2[(int64_t)blockIdx.y * a.T + to] = k;
  a.order2[(int64_t)blockIdx.y * a.T + to] = a.order[(int64_t)blockIdx.y * a.T + i];
}

// ---------------------------------------------------------------- the sums

// A lane's four columns of a wavefront's 256: adjacent where rows allow
// 4-element accesses, else 64 apart.
template <bool VEC>
__device__ __forceinline__ int column(int c0, int lane, int e) {
  return VEC ? c0 + 4 * lane + e : c0 + 64 * e + lane;
}

template <typename D, bool VEC>
__device__ __forceinline__ float4 load_row(const D* row, int c0, int lane, int d) {
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (VEC) {
    if (c0 + 4 * lane < d) {
      const Pack<D, 4> p = *(const Pack<D, 4>*)(row + c0 + 4 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = to_f32(p.v[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c0 + 64 * e + lane < d) v[e] = to_f32(row[c0 + 64 * e + lane]);
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void add4(float4& s, const float4& x) {
  s.x += x.x;
  s.y += x.y;
  s.z += x.z;
  s.w += x.w;
}

template <bool VEC>
__device__ __forceinline__ void store_row(float* row, int c0, int lane, int d, float4 s, float scale, bool add) {
  float v[4] = {s.x * scale, s.y * scale, s.z * scale, s.w * scale};
  if (VEC) {
    if (c0 + 4 * lane < d) {
      float4* p = (float4*)(row + c0 + 4 * lane);
      if (add) {
        const float4 o = *p;
        v[0] += o.x;
        v[1] += o.y;
        v[2] += o.z;
        v[3] += o.w;
      }
      *p = make_float4(v[0], v[1], v[2], v[3]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = c0 + 64 * e + lane;
      if (c < d) row[c] = add ? row[c] + v[e] : v[e];
    }
  }
}

constexpr int kDepth = 8;  // rows in flight

// s += the rows of sorted tokens [p, q) (q - p <= 64), in order.
template <typename D, bool VEC>
__device__ __forceinline__ void add_rows(const GradArgs& a, const D* dy, const uint32_t* order, int64_t p, int64_t q, int c0,
                                         int lane, float4& s) {
  const uint32_t mine = order[min(p + lane, q - 1)];
  const int n = (int)(q - p);
  for (int i = 0; i < n; i += kDepth) {
    float4 x[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i + k < n) x[k] = load_row<D, VEC>(dy + (int64_t)__builtin_amdgcn_readlane(mine, i + k) * a.dy_ld, c0, lane, a.d);
    }
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (i + k < n) add4(s, x[k]);
  }
}

// Chunk of kChunk sorted tokens of one id: their sum.
template <typename D, bool VEC>
__global__ __launch_bounds__(64) void k_partial(GradArgs a) {
  const int lane = threadIdx.x, w = blockIdx.z, c0 = blockIdx.y * kCols;
  const int64_t p = (int64_t)blockIdx.x * kChunk;  // p + kChunk <= T
  const uint32_t* key = a.key + (int64_t)w * a.T;
  const uint32_t k = key[p];
  if (k != key[p + kChunk - 1] || k >= (uint32_t)a.V) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  add_rows<D, VEC>(a, (const D*)a.dy + (int64_t)w * a.dy_stride, a.order + (int64_t)w * a.T, p, p + kChunk, c0, lane, s);
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * a.d;
  const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (column<VEC>(c0, lane, e) < a.d) out[column<VEC>(c0, lane, e)] = v[e];
}

// Sorted tokens [p0, p0 + kOwn): every id whose first token is one of them.
template <typename D, bool VEC>
__global__ __launch_bounds__(64) void k_rows_sum(GradArgs a) {
  const int lane = threadIdx.x, w = blockIdx.z, c0 = blockIdx.y * kCols;
  const int64_t p0 = (int64_t)blockIdx.x * kOwn, p1 = min(p0 + kOwn, a.T);
  const uint32_t* key = a.key + (int64_t)w * a.T;
  const uint32_t* order = a.order + (int64_t)w * a.T;
  const D* dy = (const D*)a.dy + (int64_t)w * a.dy_stride;
  const float* part = a.part + (int64_t)w * (a.T / kChunk) * a.d;
  float* grads = a.grads + (int64_t)w * a.worker_stride;
  // lane i < kOwn + 1: the id before position p0 + i, and at it
  const int64_t at = p0 + lane;
  const uint32_t none = 0xffffffffu;
  const uint32_t here = lane <= kOwn && at < a.T ? key[at] : none;
  const uint32_t prev = lane < kOwn && at > 0 && at - 1 < a.T ? key[at - 1] : none;
  // the positions where an id that belongs to a row begins
  uint64_t begins = __ballot(lane < kOwn && at < p1 && here != prev && here < (uint32_t)a.V);
  const uint64_t changes = __ballot(lane <= kOwn && lane > 0 && at <= p1 && here != prev) | 1ull << kOwn;
  while (begins) {
    const int i = __builtin_ctzll(begins);
    begins &= begins - 1;
    const uint32_t id = __builtin_amdgcn_readlane(here, i);
    int64_t p = p0 + i;
    // the first change after i, or the end of what this wavefront looked at
    int64_t q = p0 + __builtin_ctzll(changes >> (i + 1)) + i + 1;
    q = min(q, a.T);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (q < p1 || q == a.T || key[q] != id) {
      add_rows<D, VEC>(a, dy, order, p, q, c0, lane, s);
    } else {
      // it runs on: to the next multiple of kChunk, whole chunks by their sums, and what is left
      int64_t edge = min((p / kChunk + 1) * kChunk, a.T);
      q = p + __popcll(__ballot(p + lane < edge && key[min(p + lane, a.T - 1)] == id));
      add_rows<D, VEC>(a, dy, order, p, q, c0, lane, s);
      p = q;
      if (p == edge && p < a.T) {
        for (;;) {
          const int64_t last = p + (int64_t)lane * kChunk + kChunk - 1;
          const int n = __popcll(__ballot(last < a.T && key[min(last, a.T - 1)] == id));
          for (int c = 0; c < n; c += kDepth) {
            float4 x[kDepth];
#pragma unroll
            for (int e = 0; e < kDepth; ++e) {
              x[e] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (c + e < n) {
                const float* row = part + (p / kChunk + c + e) * a.d;
                float v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = column<VEC>(c0, lane, u) < a.d ? row[column<VEC>(c0, lane, u)] : 0.0f;
                x[e] = make_float4(v[0], v[1], v[2], v[3]);
              }
            }
#pragma unroll
            for (int e = 0; e < kDepth; ++e)
              if (c + e < n) add4(s, x[e]);
          }
          p += (int64_t)n * kChunk;
          if (n < 64) break;
        }
        q = p + __popcll(__ballot(p + lane < a.T && key[min(p + lane, a.T - 1)] == id));
        if (q > p) add_rows<D, VEC>(a, dy, order, p, q, c0, lane, s);
      }
    }
    store_row<VEC>(grads + (int64_t)id * a.d, c0, lane, a.d, s, a.scale, a.accumulate);
  }
}

// ------------------------------------------------------------------- hosts

struct GradPlan {
  int cap, tiles, passes;  // tokens of a tile, tiles and merge passes of a worker
  size_t key[2], order[2], part, total;
};

GradPlan plan_of(int32_t W, int64_t T, int64_t d) {
  GradPlan p = {};
  p.cap = T <= 1024 ? 1024 : T <= 4096 ? 4096 : 16384;
  p.tiles = (int)ceil_div(T, p.cap);
  for (int64_t run = p.cap; run < T; run *= 2) ++p.passes;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  const size_t n = (size_t)W * (size_t)T * 4;
  p.key[0] = take(n);
  p.order[0] = take(n);
  if (p.passes) {
    p.key[1] = take(n);
    p.order[1] = take(n);
  }
  p.part = take((size_t)W * (size_t)(T / kChunk) * (size_t)d * 4);
  p.total = at;
  return p;
}

nf_status bad(const char* what) { return set_error(NF_ERR_INVALID_ARG, what); }

nf_status finish(hipError_t e) {
  if (e != hipSuccess) return set_error(NF_ERR_HIP, hipGetErrorString(e));
  return set_error(NF_OK, "");
}

constexpr int64_t kMaxD = 1 << 24, kMaxT = 1 << 24, kMaxInt = 0x7fffffff;

const char* check_grad_sizes(int32_t W, int64_t T, int64_t V, int64_t d) {
  if (W < 1 || W > 255) return "W outside [1, 255]";
  if (T < 0 || T > kMaxT) return "T outside [0, 2^24]";
  if (V < 0 || V > kMaxInt) return "V outside [0, 2^31)";
  if (d < 0 || d > kMaxD) return "d outside [0, 2^24]";
  return nullptr;
}

template <typename D>
void launch_sums(const GradArgs& a, bool vec, hipStream_t s) {
  const unsigned slices = (unsigned)ceil_div(a.d, kCols);
  const int64_t chunks = a.T / kChunk;
  if (chunks) {
    const dim3 grid((unsigned)chunks, slices, (unsigned)a.W);
    if (vec)
      k_partial<D, true><<<grid, 64, 0, s>>>(a);
    else
      k_partial<D, false><<<grid, 64, 0, s>>>(a);
  }
  const dim3 grid((unsigned)ceil_div(a.T, kOwn), slices, (unsigned)a.W);
  if (vec)
    k_rows_sum<D, true><<<grid, 64, 0, s>>>(a);
  else
    k_rows_sum<D, false><<<grid, 64, 0, s>>>(a);
}

// Blocks that zero a worker's segment: 64 KiB each at least, 4,096 in all at most.
int64_t fill_blocks(const GradArgs& a) {
  if (a.accumulate) return 0;
  const int64_t want = ceil_div(a.V * a.d * 4, 65536), most = 4096 / a.W;
  return want < most ? want : most;
}

template <int THREADS, int ITEMS>
void launch_sort(const GradArgs& a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.W * (a.tiles + fill_blocks(a));
  if (blocks) k_sort<THREADS, ITEMS><<<(unsigned)blocks, THREADS, 0, s>>>(a);
}

}  // namespace
}  // namespace nf

extern "C" {

nf_status nf_embedding_lookup(const void* table, int32_t table_type, int64_t table_ld, int64_t V, int64_t d,
                              const void* ids, int32_t ids_bytes, int64_t T, float scale, void* out,
                              int32_t out_type, int64_t out_ld, void* stream) {
  using namespace nf;
  if (!known_type(table_type) || !known_type(out_type)) return bad("unknown element type");
  if (ids_bytes != 4 && ids_bytes != 8) return bad("ids_bytes must be 4 or 8");
  if (V < 0 || T < 0 || T > kMaxInt || d < 0 || d > kMaxD) return bad("V, T or d out of range");
  if (table_ld < d || out_ld < d) return bad("table_ld or out_ld < d");
  if (T == 0 || d == 0) return set_error(NF_OK, "");
  if (!ids || !out || (!table && V > 0)) return bad("table, ids or out is NULL");
  if ((uintptr_t)table % type_bytes(table_type) || (uintptr_t)out % type_bytes(out_type) || (uintptr_t)ids % ids_bytes)
    return set_error(NF_ERR_ALIGNMENT, "table, ids or out not aligned to its elements");
  LookupArgs a = {table, ids, out, table_ld, out_ld, V, T, (int32_t)d, ids_bytes == 8, scale, 0};
  auto wide = [&](const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; };
  const bool vec = d % 8 == 0 && wide(table, table_ld) && wide(out, out_ld);
  while (a.lg_tx < 8 && (1 << a.lg_tx) * (vec ? 8 : 1) < d) ++a.lg_tx;
  const unsigned blocks = (unsigned)ceil_div(T, kThreadsE >> a.lg_tx);
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_type(table_type, [&](auto* tp) {
    with_type(out_type, [&](auto* op) {
      using A = std::remove_pointer_t<decltype(tp)>;
      using B = std::remove_pointer_t<decltype(op)>;
      if (vec)
        k_lookup<A, B, 8><<<blocks, kThreadsE, 0, s>>>(a);
      else
        k_lookup<A, B, 1><<<blocks, kThreadsE, 0, s>>>(a);
    });
  });
  return finish(hipGetLastError());
}

size_t nf_embedding_workspace_bytes(int32_t W, int64_t T, int64_t V, int64_t d) {
  if (nf::check_grad_sizes(W, T, V, d)) return 0;
  return nf::plan_of(W, T, d).total;
}

nf_status nf_embedding_grad(const void* dy, int32_t dy_type, int64_t dy_ld, int64_t dy_stride, const void* ids,
                            int32_t ids_bytes, int64_t ids_stride, int32_t W, int64_t T, int64_t V, int64_t d,
                            float scale, int64_t padding_id, int32_t accumulate, float* grads,
                            int64_t worker_stride, void* ws, size_t ws_bytes, void* stream) {
  using namespace nf;
  if (!known_type(dy_type)) return bad("unknown element type");
  if (ids_bytes != 4 && ids_bytes != 8) return bad("ids_bytes must be 4 or 8");
  if (const char* why = check_grad_sizes(W, T, V, d)) return bad(why);
  if (dy_ld < d) return bad("dy_ld < d");
  if (W > 1 && T > 0 && (dy_stride < (T - 1) * dy_ld + d || ids_stride < T)) return bad("dy_stride or ids_stride too small");
  if (W > 1 && worker_stride < V * d) return bad("worker_stride < V * d");
  if (accumulate != 0 && accumulate != 1) return bad("accumulate must be 0 or 1");
  if (V == 0 || d == 0) return set_error(NF_OK, "");
  if (!grads) return bad("grads is NULL");
  if (T > 0 && (!dy || !ids)) return bad("dy or ids is NULL");
  if ((uintptr_t)grads % 4 || (uintptr_t)dy % type_bytes(dy_type) || (uintptr_t)ids % ids_bytes)
    return set_error(NF_ERR_ALIGNMENT, "dy, ids or grads not aligned to its elements");
  const GradPlan p = plan_of(W, T, d);
  if (ws_bytes < p.total) return set_error(NF_ERR_WORKSPACE, "workspace smaller than nf_embedding_workspace_bytes");
  if (p.total && !ws) return set_error(NF_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)ws % 256) return set_error(NF_ERR_ALIGNMENT, "workspace not 256-byte aligned");
  unsigned char* base = static_cast<unsigned char*>(ws);
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(base + at); };
  GradArgs a = {};
  a.dy = dy;
  a.dy_ld = dy_ld;
  a.dy_stride = dy_stride;
  a.ids = ids;
  a.ids_stride = ids_stride;
  a.ids64 = ids_bytes == 8;
  a.W = W;
  a.d = (int32_t)d;
  a.T = T;
  a.V = V;
  a.padding_id = padding_id;
  a.scale = scale;
  a.accumulate = accumulate;
  a.grads = grads;
  a.worker_stride = worker_stride;
  a.key = words(p.key[0]);
  a.order = words(p.order[0]);
  a.part = reinterpret_cast<float*>(base + p.part);
  a.tiles = p.tiles;
  while (a.bits < 32 && (V >> a.bits)) ++a.bits;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.cap == 1024)
    launch_sort<256, 4>(a, s);
  else if (p.cap == 4096)
    launch_sort<1024, 4>(a, s);
  else
    launch_sort<1024, 16>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || T == 0) return finish(e);
  a.run = p.cap;
  for (int k = 0; k < p.passes; ++k, a.run *= 2) {
    const int to = (k + 1) & 1;
    a.key = words(p.key[to ^ 1]);
    a.order = words(p.order[to ^ 1]);
    a.key2 = words(p.key[to]);
    a.order2 = words(p.order[to]);
    k_merge<<<dim3((unsigned)ceil_div(T, kThreadsE), (unsigned)W), kThreadsE, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return finish(e);
    a.key = a.key2;
    a.order = a.order2;
  }
  // four adjacent elements at a time where every row of dy and of the table allows it
  const size_t four = 4 * type_bytes(dy_type);
  const bool vec = d % 4 == 0 && dy_ld % 4 == 0 && (W == 1 || (dy_stride % 4 == 0 && worker_stride % 4 == 0)) &&
                   (uintptr_t)dy % four == 0 && (uintptr_t)grads % 16 == 0;
  with_type(dy_type, [&](auto* tp) { launch_sums<std::remove_pointer_t<decltype(tp)>>(a, vec, s); });
  return finish(hipGetLastError());
}

}  // extern "C"
