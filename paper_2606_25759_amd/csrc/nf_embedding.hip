// nf_embedding.hip - embedding lookup with scaling, and its gradient by
// sorted tokens.
//
//   k_lookup    out[t] = scale * table[ids[t]]
//   k_sort      tiles of a worker's tokens sorted by id in LDS (stable, so
//               tokens of one id stay in their order), while the launch's
//               other blocks zero the workers' segments
//   k_merge     up to kRuns sorted runs into one
//   k_rows_sum  a wavefront per kOwn sorted tokens and 256 columns: the rows
//               of every id that lies in them whole, and sums of those that
//               begin before or end after them
//   k_join      the rows of the latter: a frequent token's rows are read by
//               many wavefronts, and none reads more than kOwn
//
// All are bound by memory traffic, or, up to some thousand tokens, by the
// latency of one launch after the other.  The gradient's floor is the dense
// FP32 segment written once and dy read once.  The order in which a row's terms
// are added depends on the sorted tokens alone, so results are reproducible
// bit for bit.
#include <type_traits>

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

constexpr int kThreadsE = 256;

// Eight elements of a row a thread (one where rows have fewer), the last ones
// of a row where they are: the thread before may have some of them too.
// Bound by memory: 32,768 skewed tokens of width 2048, FP32 to BF16, in 43 us
// (about 12,500 different rows: 237 MB, 5.5 TB/s); 64 tokens in 2.7 us, under
// the 6 us that the call takes on the host.
template <typename A, typename B, int N>
__global__ __launch_bounds__(kThreadsE) void k_lookup(LookupArgs a) {
  const int tx = 1 << a.lg_tx, ty = kThreadsE >> a.lg_tx;
  const int x = threadIdx.x & (tx - 1);
  for (int64_t t = (int64_t)blockIdx.x * ty + (threadIdx.x >> a.lg_tx); t < a.T; t += (int64_t)gridDim.x * ty) {
    const int64_t id = id_at(a.ids, a.ids64, t);
    const bool in = id >= 0 && id < a.V;
    const A* row = (const A*)a.table + (in ? id : 0) * a.table_ld;
    B* out = (B*)a.out + t * a.out_ld;
    for (int j = x * N; j < a.d; j += tx * N) {
      const int at = min(j, a.d - N);
      Near<B, N> o;
      if (in) {
        const Near<A, N> p = *(const Near<A, N>*)(row + at);
#pragma unroll
        for (int e = 0; e < N; ++e) o.v[e] = from_f32<B>(to_f32(p.v[e]) * a.scale);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) o.v[e] = from_f32<B>(0.0f);
      }
      *(Near<B, N>*)(out + at) = o;
    }
  }
}

// -------------------------------------------------------------------- sort

constexpr int kOwn = 16;   // sorted tokens of a wavefront of k_rows_sum
constexpr int kRuns = 16;  // sorted runs of a merge
// Up to so many tokens of a worker, the wavefront that an id begins in adds all its rows itself (kOwn at a time), and
// there is no k_join: a launch less, 2.8 us of the 20 that 4 x 197 tokens take, against 16 rows after each other at
// most.
constexpr int64_t kAloneTokens = 256;

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
  float* part;              // [W][ceil(T / kOwn)][2][d]: sums of an id that began before, and of one that goes on
  int64_t run;              // tokens of a sorted run
  int32_t tiles;            // k_sort: runs of a worker
  int32_t bits;             // of V
};

// Zeroes n floats at p with the blocks b of nb: whole 16-byte pieces, four a
// thread and adjacent in the block (64 KiB of 1,024 threads: 5.6 TB/s; 4.7
// when all blocks write side by side), and what lies before the first and
// after the last one.
__device__ void fill_zero(float* p, int64_t n, int64_t b, int64_t nb) {
  const int64_t kPiece = 4 * blockDim.x;
  const int64_t head = min((int64_t)((-(intptr_t)p) & 15) / 4, n);
  const int64_t n4 = (n - head) / 4, tail = n - head - 4 * n4;
  if (b == 0) {
    if (threadIdx.x < head) p[threadIdx.x] = 0.0f;
    if (threadIdx.x < tail) p[n - 1 - threadIdx.x] = 0.0f;
  }
  float4* q = (float4*)(p + head);
  for (int64_t at = b * kPiece; at < n4; at += nb * kPiece) {
    const int64_t end = min(at + kPiece, n4);
    for (int64_t i = at + threadIdx.x; i < end; i += blockDim.x) q[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

// Least-significant-digit radix sort of up to THREADS * ITEMS tokens, 8 bits
// a pass: 12 us for runs of 4,096, hidden behind the zeroes where there are
// any (412 MB: 62 us, 6.6 TB/s; 3.3 GB: 570 us, 5.8 TB/s).  Runs of 16,384
// took 33 us: the ranks are VALU work of one CU.  Item i of lane l of wavefront w is the (w * ITEMS + i) * 64 + l-th,
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

// Groups of kRuns runs of a.run tokens: a token goes behind those of its own
// run before it and those of every other run with a smaller id (of the
// earlier runs: or the same).  Neighbours in a run have neighbouring ids, so
// a wavefront's searches touch the same few lines.  8,192 tokens in two runs
// 7.6 us, 2 x 30,011 in eight 12 us: the searches' latency.
__global__ __launch_bounds__(kThreadsE) void k_merge(GradArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreadsE + threadIdx.x;
  if (i >= a.T) return;
  const uint32_t* key = a.key + (int64_t)blockIdx.y * a.T;
  const int T = (int)a.T, len = (int)a.run;  // at most 2^24 and 2^28
  const int run = (int)(i / len), r = run % kRuns;
  const int64_t base = (int64_t)(run - r) * len;
  const int others = (int)min((int64_t)kRuns, (T - base + len - 1) / len) - 1;  // runs of the group but its own
  const uint32_t k = key[i];
  int64_t to = base + i - (int64_t)run * len;
  constexpr int kAtOnce = 4;
  for (int q0 = 0; q0 < others; q0 += kAtOnce) {
    int lo[kAtOnce], hi[kAtOnce];
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const int q = q0 + e < r ? q0 + e : q0 + e + 1;  // not its own
      lo[e] = (int)min(base + (int64_t)q * len, (int64_t)T);
      // past the group's runs (kRuns - 1 is no multiple of kAtOnce) there may be the next group's
      hi[e] = q0 + e < others ? (int)min((int64_t)lo[e] + len, (int64_t)T) : lo[e];
      to -= lo[e];
    }
    for (;;) {
      bool busy = false;
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const int mid = (lo[e] + hi[e]) / 2;
        const bool open = lo[e] < hi[e];
        const bool before = key[open ? mid : 0] < k + (q0 + e < r ? 1u : 0u);  // k <= V < 2^31
        if (open && before) lo[e] = mid + 1;
        if (open && !before) hi[e] = mid;
        busy |= open;
      }
      if (!__any(busy)) break;
    }
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) to += lo[e];
  }
  a.key2[(int64_t)blockIdx.y * a.T + to] = k;
  a.order2[(int64_t)blockIdx.y * a.T + to] = a.order[(int64_t)blockIdx.y * a.T + i];
}

// ---------------------------------------------------------------- the sums

// A block's columns are an even share of a row's groups of N (four; one where
// rows have fewer), a group a lane.  The row's last group is its last N
// columns, some of which its neighbour in the same wavefront may have too, and
// comes to the same values: no access needs a condition.  (A share has 32
// groups at least where there are several, so the neighbour is in it.)
struct Columns {
  int at;     // of this lane
  bool mine;  // false: `at` is another lane's too, and this one stores nothing
};
template <int N>
__device__ __forceinline__ Columns columns_of(int d, int lane) {
  const int64_t groups = (d + N - 1) / N;
  const int begin = (int)(groups * blockIdx.y / gridDim.y), end = (int)(groups * (blockIdx.y + 1) / gridDim.y);
  return {min(min(begin + lane, end - 1) * N, d - N), begin + lane < end};
}

template <typename D, int N>
__device__ __forceinline__ Near<D, N> load_row(const D* row, Columns c) {
  return *(const Near<D, N>*)(row + c.at);
}

template <typename D, int N>
__device__ __forceinline__ void add_to(float (&s)[N], const Near<D, N>& x) {
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] += to_f32(x.v[e]);
}

// Sorted tokens [p0, p0 + kOwn).  Their rows are asked for at once: an id
// does not wait for the one before it (8,192 tokens of width 2048: 73 us when
// it did, 23 us now, for 34 MB read and about 30 MB written).
template <typename D, int N, bool ADD, bool ALONE>
__global__ __launch_bounds__(64) void k_rows_sum(GradArgs a) {
  const int lane = threadIdx.x, w = blockIdx.z;
  const Columns c = columns_of<N>(a.d, lane);
  const int64_t p0 = (int64_t)blockIdx.x * kOwn;
  const int count = (int)min((int64_t)kOwn, a.T - p0);
  const uint32_t* key = a.key + (int64_t)w * a.T;
  const D* dy = (const D*)a.dy + (int64_t)w * a.dy_stride;
  float* grads = a.grads + (int64_t)w * a.worker_stride;
  const uint32_t none = 0xffffffffu, V = (uint32_t)a.V;
  // lane i <= kOwn: the id at position p0 + i, and before it
  const uint32_t token = a.order[(int64_t)w * a.T + p0 + min(lane, count - 1)];
  const uint32_t here = lane <= kOwn && p0 + lane < a.T ? key[p0 + lane] : none;
  uint32_t prev = __shfl_up(here, 1);
  if (lane == 0) prev = p0 > 0 ? key[p0 - 1] : none;
  const uint64_t begins = __ballot(lane < count && here != prev);
  const int end = __popcll(__ballot(lane < count && here < V));  // those of no row come last
  if (end == 0) return;
  if (ALONE && !(begins & ((1ull << end) - 1))) return;
  const bool goes_on =
      end == kOwn && __builtin_amdgcn_readlane(here, kOwn) == __builtin_amdgcn_readlane(here, kOwn - 1);
  auto row_of = [&](int i) {
    const uint32_t id = (uint32_t)__builtin_amdgcn_readlane(here, min(i, end - 1));
    return (Near<float, N>*)(grads + (int64_t)id * a.d + c.at);
  };
  Near<D, N> x[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i)
    x[i] = load_row<D, N>(dy + (int64_t)(uint32_t)__builtin_amdgcn_readlane(token, min(i, end - 1)) * a.dy_ld, c);
  // what the rows hold is asked for with the rest: a load behind a store would wait for it
  Near<float, N> old[ADD ? kOwn : 1] = {};
  if constexpr (ADD) {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) old[i] = *row_of(i);
  }
  float s[N] = {};
  bool whole = begins & 1;  // the id at hand began here
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    if (i >= end) continue;
    add_to(s, x[i]);
    const bool last = i == end - 1;
    if (!last && !(begins >> (i + 1) & 1)) continue;
    Near<float, N> v;
    if (ALONE && whole && last && goes_on) {
      const uint32_t id = __builtin_amdgcn_readlane(here, kOwn);
      for (int64_t p = p0 + kOwn;;) {
        const int n = __popcll(__ballot(lane < kOwn && p + lane < a.T && key[min(p + lane, a.T - 1)] == id));
        if (n == 0) break;
        const uint32_t more = a.order[(int64_t)w * a.T + min(p + lane, a.T - 1)];
        Near<D, N> y[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
          y[k] = load_row<D, N>(dy + (int64_t)(uint32_t)__builtin_amdgcn_readlane(more, min(k, n - 1)) * a.dy_ld, c);
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
          if (k < n) add_to(s, y[k]);
        p += n;
        if (n < kOwn) break;
      }
    }
    if (whole && (ALONE || !(last && goes_on))) {
#pragma unroll
      for (int e = 0; e < N; ++e) v.v[e] = s[e] * a.scale + (ADD ? old[ADD ? i : 0].v[e] : 0.0f);
      if (c.mine) *row_of(i) = v;
    } else if (!ALONE) {
#pragma unroll
      for (int e = 0; e < N; ++e) v.v[e] = s[e];
      float* part = a.part + (((int64_t)w * gridDim.x + blockIdx.x) * 2 + whole) * a.d;
      if (c.mine) *(Near<float, N>*)(part + c.at) = v;
    }
    whole = true;
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = 0.0f;
  }
}

// Ids that begin in kOwn tokens and go on after them, a wavefront each: their
// sums in order (5 us for 8,192 skewed tokens of width 2048).  One of more than
// kAlone sums is left to the whole block: an even share of them to each
// wavefront, and the shares in order.
constexpr int kDepth = 8;  // sums under way
constexpr int kAlone = 4 * kDepth;

template <int N>
__device__ __forceinline__ void add_sums(const float* sums, int from, int to, int64_t d, Columns c, float (&s)[N]) {
  for (int i = from; i < to; i += kDepth) {
    Near<float, N> x[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      const int q = min(i + k, to - 1);  // the first is of the id that goes on, the others of one that began before
      x[k] = *(const Near<float, N>*)(sums + (2 * (int64_t)q + (q == 0)) * d + c.at);
    }
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (i + k < to) add_to(s, x[k]);
  }
}

template <int N, bool ADD>
__global__ __launch_bounds__(kThreadsE) void k_join(GradArgs a) {
  constexpr int kWaves = kThreadsE / 64;
  __shared__ int left[kWaves];  // sums that are left to the block
  __shared__ float shares[kWaves][64][N];
  const int w = blockIdx.z, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t* key = a.key + (int64_t)w * a.T;
  const int64_t own = (a.T + kOwn - 1) / kOwn, own0 = (int64_t)blockIdx.x * kWaves;
  const Columns c = columns_of<N>(a.d, lane);
  float* grads = a.grads + (int64_t)w * a.worker_stride + c.at;
  const float* part = a.part + (int64_t)w * own * 2 * a.d;
  auto write = [&](uint32_t id, const float(&s)[N]) {
    if (!c.mine) return;
    Near<float, N>* row = (Near<float, N>*)(grads + (int64_t)id * a.d);
    Near<float, N> v = {};
    if (ADD) v = *row;
#pragma unroll
    for (int e = 0; e < N; ++e) v.v[e] = s[e] * a.scale + v.v[e];
    *row = v;
  };
  int pieces = 0;
  const int64_t p0 = (own0 + wave) * kOwn;
  if (p0 + kOwn < a.T) {
    // lane 0: the id before these tokens, 1: their last one, 2: the one after them
    const int64_t at = p0 + (lane == 0 ? -1 : kOwn - 2 + min(lane, 2));
    const uint32_t k = at >= 0 ? key[at] : 0xffffffffu;
    const uint32_t id = __builtin_amdgcn_readlane(k, 1);
    if (id == (uint32_t)__builtin_amdgcn_readlane(k, 2) && id < (uint32_t)a.V &&
        id != (uint32_t)__builtin_amdgcn_readlane(k, 0)) {
      for (pieces = 1;;) {  // and those after it that begin with it
        const int64_t p = p0 + (int64_t)(pieces + lane) * kOwn;
        const int n = __popcll(__ballot(p < a.T && key[min(p, a.T - 1)] == id));
        pieces += n;
        if (n < 64) break;
      }
      if (pieces <= kAlone) {
        float s[N] = {};
        add_sums<N>(part + (own0 + wave) * 2 * a.d, 0, pieces, a.d, c, s);
        write(id, s);
      }
    }
  }
  if (lane == 0) left[wave] = pieces > kAlone ? pieces : 0;
  __syncthreads();
  for (int q = 0; q < kWaves; ++q) {
    const int n = left[q];
    if (n == 0) continue;
    float s[N] = {};
    add_sums<N>(part + (own0 + q) * 2 * a.d, n * wave / kWaves, n * (wave + 1) / kWaves, a.d, c, s);
#pragma unroll
    for (int e = 0; e < N; ++e) shares[wave][lane][e] = s[e];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        for (int u = 1; u < kWaves; ++u) s[e] += shares[u][lane][e];
      write(key[(own0 + q) * kOwn + kOwn - 1], s);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------- hosts

struct GradPlan {
  int cap, tiles, passes;  // tokens of a tile, tiles and merge passes of a worker
  size_t key[2], order[2], part, total;
};

GradPlan plan_of(int32_t W, int64_t T, int64_t d) {
  GradPlan p = {};
  p.cap = T <= 1024 ? 1024 : 4096;
  p.tiles = (int)ceil_div(T, p.cap);
  for (int64_t run = p.cap; run < T; run *= kRuns) ++p.passes;
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
  if (T > kAloneTokens) p.part = take((size_t)W * (size_t)ceil_div(T, kOwn) * (size_t)d * 8);
  p.total = at;
  return p;
}

nf_status bad(const char* what) { return set_error(NF_ERR_INVALID_ARG, what); }

nf_status finish(hipError_t e) {
  if (e != hipSuccess) return set_error(NF_ERR_HIP, hipGetErrorString(e));
  return set_error(NF_OK, "");
}

constexpr int64_t kMaxD = 1 << 23, kMaxT = 1 << 24, kMaxInt = 0x7fffffff;

const char* check_grad_sizes(int32_t W, int64_t T, int64_t V, int64_t d) {
  if (W < 1 || W > 255) return "W outside [1, 255]";
  if (T < 0 || T > kMaxT) return "T outside [0, 2^24]";
  if (V < 0 || V > kMaxInt) return "V outside [0, 2^31)";
  if (d < 0 || d > kMaxD) return "d outside [0, 2^23]";
  return nullptr;
}

template <typename D, int N, bool ADD>
void launch_sums(const GradArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(a.T, kOwn), (unsigned)ceil_div(a.d, 64 * N), (unsigned)a.W);
  if (a.T <= kAloneTokens) {
    k_rows_sum<D, N, ADD, true><<<grid, 64, 0, s>>>(a);
    return;
  }
  k_rows_sum<D, N, ADD, false><<<grid, 64, 0, s>>>(a);
  k_join<N, ADD><<<dim3((grid.x + 3) / 4, grid.y, grid.z), kThreadsE, 0, s>>>(a);
}

template <typename D, int N>
void launch_sums(const GradArgs& a, hipStream_t s) {
  if (a.accumulate)
    launch_sums<D, N, true>(a, s);
  else
    launch_sums<D, N, false>(a, s);
}

// Blocks that zero a worker's segment: a piece each at least, 4,096 in all at most.
int64_t fill_blocks(const GradArgs& a, int threads) {
  if (a.accumulate) return 0;
  const int64_t want = ceil_div(a.V * a.d, 16 * threads), most = 4096 / a.W;
  return want < most ? want : most;
}

template <int THREADS, int ITEMS>
void launch_sort(const GradArgs& a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.W * (a.tiles + fill_blocks(a, THREADS));
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
  const int each = d < 8 ? 1 : 8;
  while (a.lg_tx < 8 && (each << a.lg_tx) < d) ++a.lg_tx;
  const int64_t most = 1 << 22, want = ceil_div(T, kThreadsE >> a.lg_tx);  // a launch has under 2^32 threads
  const unsigned blocks = (unsigned)(want < most ? want : most);
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_type(table_type, [&](auto* tp) {
    with_type(out_type, [&](auto* op) {
      using A = std::remove_pointer_t<decltype(tp)>;
      using B = std::remove_pointer_t<decltype(op)>;
      if (each == 8)
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
  if (W > 1 && T > 0 && (overlaps(dy_stride, T, dy_ld, d) || ids_stride < T))
    return bad("dy_stride or ids_stride too small");
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
  else
    launch_sort<1024, 4>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || T == 0) return finish(e);
  a.run = p.cap;
  for (int k = 0; k < p.passes; ++k, a.run *= kRuns) {
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
  with_type(dy_type, [&](auto* tp) {
    using D = std::remove_pointer_t<decltype(tp)>;
    if (d < 4)
      launch_sums<D, 1>(a, s);
    else
      launch_sums<D, 4>(a, s);
  });
  return finish(hipGetLastError());
}

}  // extern "C"
