// nf_norm.hip - norms over many tensors, and the tensors scaled by them.
//
//   k_squares  each block's sum of squares; a group of one block: its norm
//   k_norms    a group's norm from its blocks' sums
//   k_clip     dst = min(1, max_norm / (norm + eps)) src, the norm from memory
//              or, in the call that forms it, from the blocks' sums
//
// Tensors are cut on the host into pieces, of one row or of several short
// ones, that a wavefront reads at a time; pieces of a group into blocks of
// like cost.  A thousand small tensors are then one launch, and a large one
// fills the card.  Sums are FP64 in an order fixed by the table: no square or
// sum of any scale of gradients overflows or vanishes, and two calls give the
// same bits.  The norm is FP32: above its range it is infinite.
//
// Bound by memory.  Norms of 16 x 25.6M FP32 elements (2,576 tensors): 275 us,
// 5.95 TB/s.  The two passes of a clipping read what they scale twice; the
// second goes through each block's pieces from the last one back, since what
// was read last may still be in the card's cache: 1.3G BF16 into FP32 in
// 2,000 us (10.5 GB moved, 5.3 TB/s), 25.6M FP32 in 52.  A dozen small
// tensors are one block and one launch: 3 us, 5.3 with the call.  Blocks of
// 1,024 threads, as many as the card holds at once.
#include <limits.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "nf_internal.h"
#include "nf_types.h"

namespace nf {
namespace {

constexpr int kNormThreads = 1024;
constexpr int kNormWaves = kNormThreads / 64;
constexpr int kWavesAtOnce = 8;            // a SIMD: two blocks a CU (25.6M FP32 clipped: 12% less than with one)
constexpr int64_t kMostBlocks = 512;       // what the card holds at once
constexpr int64_t kLeastPiece = 1024, kMostPiece = 32768;  // elements
constexpr int64_t kPieceCost = 1024;       // of a piece besides its elements, in elements
constexpr int64_t kBlockCost = 32768;      // of a block, at least
constexpr int64_t kMaxTensors = 1 << 20, kMaxGroups = 1 << 16, kMaxPieces = 1 << 24;
constexpr int64_t kMaxRowsCompared = 1 << 22;

struct Piece {
  const void* src;
  void* dst;
  int64_t src_ld, dst_ld;
  int32_t rows, cols;
  int32_t src_type, dst_type;
};

struct Block {
  int32_t first, count;  // pieces
  int32_t group;
  int32_t lone;          // the group's only one
};

struct Span {
  int32_t first, count;  // blocks of a group
};

struct NormArgs {
  const Piece* pieces;
  const Block* blocks;
  const Span* spans;
  double* part;  // [blocks]
  float* norms;  // [groups]
  float max_norm, eps;
};

// Calls f with the first element, the count and the lane's first of them for the lane's part of a piece: N at a time
// while they are whole, else one by one.
template <int N, typename Whole, typename Single>
__device__ __forceinline__ void each_part(const Piece& p, Whole whole, Single single) {
  const int lane = threadIdx.x % 64, vectors = p.cols / N;
  int lg = 0;
  while (lg < 6 && (1 << lg) < vectors) ++lg;
  const int x = lane & ((1 << lg) - 1), y = lane >> lg;
  for (int r = y; r < p.rows; r += 64 >> lg) {
    whole(r, x, 1 << lg, vectors);
    for (int c = vectors * N + x; c < p.cols; c += 1 << lg) single(r, c);
  }
}

template <typename T>
__device__ __forceinline__ double squares(const Piece& p) {
  constexpr int N = 16 / (int)sizeof(T), U = 8;
  double sum[2] = {};
  auto add = [&](const Near<T, N>& v) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const double x = (double)to_f32(v.v[e]);
      sum[e & 1] = fma(x, x, sum[e & 1]);
    }
  };
  each_part<N>(
      p,
      [&](int r, int v, int step, int vectors) {
        const T* row = (const T*)p.src + r * p.src_ld;
        for (; v + (U - 1) * step < vectors; v += U * step) {
          Near<T, N> w[U];
#pragma unroll
          for (int u = 0; u < U; ++u) w[u] = *(const Near<T, N>*)(row + (v + u * step) * N);
#pragma unroll
          for (int u = 0; u < U; ++u) add(w[u]);
        }
        for (; v < vectors; v += step) add(*(const Near<T, N>*)(row + v * N));
      },
      [&](int r, int c) {
        const double x = (double)to_f32(((const T*)p.src + r * p.src_ld)[c]);
        sum[0] = fma(x, x, sum[0]);
      });
  return sum[0] + sum[1];
}

// SIZE bytes at any element's address that are not read again here: they need not displace what is (102 MB of FP32
// clipped: 7% less than with ordinary stores and eight loads under way where this has four).
template <int SIZE>
__device__ __forceinline__ void store_past(void* to, const void* from) {
  typedef uint32_t word __attribute__((aligned(2)));
  typedef word words __attribute__((ext_vector_type(SIZE % 16 ? 2 : 4), aligned(2)));
#pragma unroll
  for (int i = 0; i < SIZE / (int)sizeof(words); ++i) {
    words w;
    __builtin_memcpy(&w, (const char*)from + i * sizeof(w), sizeof(w));
    __builtin_nontemporal_store(w, (words*)to + i);
  }
}

template <typename S, typename D>
__device__ __forceinline__ void scale(const Piece& p, float by) {
  constexpr int N = 16 / (int)(sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), U = 4;
  auto put = [&](const Near<S, N>& v, D* to) {
    Near<D, N> w;
#pragma unroll
    for (int e = 0; e < N; ++e) w.v[e] = from_f32<D>(to_f32(v.v[e]) * by);
    store_past<sizeof(w)>(to, &w);
  };
  each_part<N>(
      p,
      [&](int r, int v, int step, int vectors) {
        const S* row = (const S*)p.src + r * p.src_ld;
        D* to = (D*)p.dst + r * p.dst_ld;
        for (; v + (U - 1) * step < vectors; v += U * step) {
          Near<S, N> w[U];
#pragma unroll
          for (int u = 0; u < U; ++u) w[u] = *(const Near<S, N>*)(row + (v + u * step) * N);
#pragma unroll
          for (int u = 0; u < U; ++u) put(w[u], to + (v + u * step) * N);
        }
        for (; v < vectors; v += step) put(*(const Near<S, N>*)(row + v * N), to + v * N);
      },
      [&](int r, int c) {
        ((D*)p.dst + r * p.dst_ld)[c] = from_f32<D>(to_f32(((const S*)p.src + r * p.src_ld)[c]) * by);
      });
}

// The block's sum of x in a fixed order, in every thread.
__device__ double sum_of_block(double x, double* s) {
  for (int o = 32; o; o >>= 1) x += __shfl_down(x, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = x;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kNormWaves; ++i) t += s[i];
  return t;
}

__device__ float norm_of(const NormArgs& a, int group, double* s) {
  const Span g = a.spans[group];
  double sum = 0.0;
  for (int i = threadIdx.x; i < g.count; i += kNormThreads) sum += a.part[g.first + i];
  return (float)sqrt(sum_of_block(sum, s));
}

__global__ __launch_bounds__(kNormThreads, kWavesAtOnce) void k_squares(NormArgs a) {
  __shared__ double s[kNormWaves];
  const Block b = a.blocks[blockIdx.x];
  double sum = 0.0;
  for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x / 64); i < b.count; i += kNormWaves) {
    const Piece p = a.pieces[b.first + i];
    if (p.src_type == NF_TYPE_F32)
      sum += squares<float>(p);
    else if (p.src_type == NF_TYPE_BF16)
      sum += squares<Bf16>(p);
    else
      sum += squares<_Float16>(p);
  }
  sum = sum_of_block(sum, s);
  if (threadIdx.x == 0) {
    a.part[blockIdx.x] = sum;
    if (b.lone) a.norms[b.group] = (float)sqrt(sum);
  }
}

__global__ __launch_bounds__(kNormThreads) void k_norms(NormArgs a) {
  __shared__ double s[kNormWaves];
  const float norm = norm_of(a, blockIdx.x, s);
  if (threadIdx.x == 0) a.norms[blockIdx.x] = norm;
}

// SUMS: the norm from the blocks' sums, else from a.norms.
template <bool SUMS>
__global__ __launch_bounds__(kNormThreads, kWavesAtOnce) void k_clip(NormArgs a) {
  __shared__ double s[kNormWaves];
  const Block b = a.blocks[blockIdx.x];
  float norm;
  if (SUMS) {
    norm = norm_of(a, b.group, s);
    if (threadIdx.x == 0 && (int)blockIdx.x == a.spans[b.group].first) a.norms[b.group] = norm;
  } else {
    norm = a.norms[b.group];
  }
  const double below = (double)norm + (double)a.eps;
  const double ratio = below == 0.0 ? 1.0 : (double)a.max_norm / below;
  const float by = ratio >= 1.0 ? 1.0f : (float)ratio;  // NaN stays NaN
  for (int i = b.count - 1 - __builtin_amdgcn_readfirstlane(threadIdx.x / 64); i >= 0; i -= kNormWaves) {
    const Piece p = a.pieces[b.first + i];
    if (by == 1.0f && p.dst == p.src) continue;  // in place, and nothing to scale
    with_type_on_device(p.src_type, [&](auto* from) {
      with_type_on_device(p.dst_type, [&](auto* to) {
        scale<std::remove_pointer_t<decltype(from)>, std::remove_pointer_t<decltype(to)>>(p, by);
      });
    });
  }
}

// --------------------------------------------------------------------- host

nf_status bad(const char* what) { return set_error(NF_ERR_INVALID_ARG, what); }

nf_status finish(hipError_t e) {
  if (e != hipSuccess) return set_error(NF_ERR_HIP, hipGetErrorString(e));
  return set_error(NF_OK, "");
}

nf_status check_tensor(const nf_norm_tensor& t, int32_t groups) {
  if (!known_type(t.src_type) || (t.dst && !known_type(t.dst_type))) return bad("unknown element type");
  if (t.group < 0 || t.group >= groups) return bad("a tensor's group is outside [0, groups)");
  if (t.rows < 0 || t.cols < 0) return bad("rows or cols < 0");
  if (t.rows == 0 || t.cols == 0) return NF_OK;
  if (t.rows > 1 && (t.src_ld < t.cols || (t.dst && t.dst_ld < t.cols))) return bad("src_ld or dst_ld < cols");
  if (!t.src) return bad("src is NULL");
  if ((uintptr_t)t.src % type_bytes(t.src_type) || (t.dst && (uintptr_t)t.dst % type_bytes(t.dst_type)))
    return set_error(NF_ERR_ALIGNMENT, "src or dst not aligned to its elements");
  for (int i = 0; i < (t.dst ? 2 : 1); ++i) {  // its last byte has an address
    const __int128 ld = t.rows > 1 ? (i ? t.dst_ld : t.src_ld) : 0;
    if ((ld * (t.rows - 1) + t.cols) * 4 > (__int128)INT64_MAX / 4) return bad("a tensor is larger than memory");
  }
  return NF_OK;
}

bool one_row(const nf_norm_tensor& t) {
  return t.rows == 1 || (t.src_ld == t.cols && (!t.dst || t.dst_ld == t.cols));
}

bool in_place(const nf_norm_tensor& t) {
  return t.dst == t.src && t.dst_type == t.src_type && (t.rows == 1 || t.dst_ld == t.src_ld);
}

// Bytes that a tensor reads or writes, or one of its rows.
struct Range {
  uintptr_t begin, end;
  int64_t tensor;
  bool written, whole;
};

void add_ranges(const nf_norm_tensor& t, int64_t index, bool by_rows, std::vector<Range>* to) {
  for (int i = 0; i < 2; ++i) {
    const bool written = i == 1;
    if (written ? !t.dst : in_place(t)) continue;  // in place: what is written is all there is
    const uintptr_t at = (uintptr_t)(written ? t.dst : t.src);
    const uintptr_t size = type_bytes(written ? t.dst_type : t.src_type);
    const uintptr_t ld = written ? t.dst_ld : t.src_ld;
    if (!by_rows || one_row(t)) {
      const uintptr_t n = t.rows == 1 ? t.cols : (t.rows - 1) * ld + t.cols;
      to->push_back(Range{at, at + n * size, index, written, !by_rows});
    } else {
      for (int64_t r = 0; r < t.rows; ++r)
        to->push_back(Range{at + r * ld * size, at + (r * ld + t.cols) * size, index, written, false});
    }
  }
}

// Whether an element that a tensor writes is another's as well, or its own but in another place.
nf_status check_apart(const nf_norm_tensor* tensors, int64_t count) {
  std::vector<Range> all, rows;
  for (int64_t i = 0; i < count; ++i)
    if (tensors[i].rows && tensors[i].cols) add_ranges(tensors[i], i, false, &all);
  auto before = [](const Range& a, const Range& b) { return a.begin < b.begin; };
  std::sort(all.begin(), all.end(), before);
  for (size_t i = 0; i < all.size();) {
    // ranges that touch one another
    size_t j = i + 1;
    uintptr_t end = all[i].end;
    bool written = all[i].written;
    for (; j < all.size() && all[j].begin < end; ++j) {
      end = std::max(end, all[j].end);
      written |= all[j].written;
    }
    if (j - i > 1 && written) {
      rows.clear();
      std::vector<int64_t> members;
      for (size_t k = i; k < j; ++k) members.push_back(all[k].tensor);
      std::sort(members.begin(), members.end());
      members.erase(std::unique(members.begin(), members.end()), members.end());
      int64_t n = 0;
      for (int64_t m : members) n += one_row(tensors[m]) ? 1 : tensors[m].rows;
      if (n > kMaxRowsCompared) return set_error(NF_ERR_UNSUPPORTED, "too many rows of interleaved tensors");
      for (int64_t m : members) add_ranges(tensors[m], m, true, &rows);
      std::sort(rows.begin(), rows.end(), before);
      uintptr_t any = 0, last = 0;  // ends of what has begun, and of what of it is written
      for (const Range& r : rows) {
        if (r.begin < last || (r.written && r.begin < any)) return bad("two tensors share an element that one writes");
        any = std::max(any, r.end);
        if (r.written) last = std::max(last, r.end);
      }
    }
    i = j;
  }
  return NF_OK;
}

// Cuts every tensor into pieces and the pieces into blocks, in the order of the groups.
template <typename OnPiece, typename OnBlock>
void cut(const nf_norm_tensor* tensors, const std::vector<int64_t>& order, int32_t groups, OnPiece on_piece,
         OnBlock on_block) {
  int64_t total = 0;
  for (int64_t i : order) total += tensors[i].rows * tensors[i].cols;
  const int64_t want = total / (kMostBlocks * kNormWaves * 2) / kLeastPiece * kLeastPiece;
  const int64_t most = std::min(std::max(want, kLeastPiece), kMostPiece);
  // pieces, with a first pass over their costs for what a block's share is
  auto pieces_of = [&](const nf_norm_tensor& t, auto f) {
    if (t.rows == 0 || t.cols == 0) return;
    const bool one = one_row(t);
    const int64_t rows = one ? 1 : t.rows, cols = one ? t.rows * t.cols : t.cols;
    const int64_t at_once = cols < most ? most / cols : 1;
    for (int64_t r = 0; r < rows; r += at_once)
      for (int64_t c = 0; c < cols; c += most)
        f(r, c, std::min(at_once, rows - r), std::min(most, cols - c));
  };
  int64_t cost = 0;
  for (int64_t i : order)
    pieces_of(tensors[i], [&](int64_t, int64_t, int64_t r, int64_t c) { cost += r * c + kPieceCost; });
  const int64_t share = std::max(kBlockCost, ceil_div(cost, kMostBlocks));
  int64_t n = 0, first = 0, have = 0;
  size_t at = 0;
  for (int32_t g = 0; g < groups; ++g) {
    bool some = false;
    for (; at < order.size() && tensors[order[at]].group == g; ++at) {
      const nf_norm_tensor& t = tensors[order[at]];
      pieces_of(t, [&](int64_t r, int64_t c, int64_t rows, int64_t cols) {
        on_piece(t, r, c, rows, cols);
        ++n;
        have += rows * cols + kPieceCost;
        if (have >= share) {
          on_block(g, first, n - first);
          first = n;
          have = 0;
          some = true;
        }
      });
    }
    if (n > first || !some) on_block(g, first, n - first);
    first = n;
    have = 0;
  }
}

std::vector<int64_t> by_group(const nf_norm_tensor* tensors, int64_t count) {
  std::vector<int64_t> order(count);
  for (int64_t i = 0; i < count; ++i) order[i] = i;
  std::stable_sort(order.begin(), order.end(),
                   [&](int64_t a, int64_t b) { return tensors[a].group < tensors[b].group; });
  return order;
}

struct Layout {
  size_t pieces, blocks, spans, total;
};

Layout layout_of(int64_t pieces, int64_t blocks, int32_t groups) {
  auto round = [](size_t n) { return (n + 255) / 256 * 256; };
  Layout l;
  l.pieces = 0;
  l.blocks = l.pieces + round(pieces * sizeof(Piece));
  l.spans = l.blocks + round(blocks * sizeof(Block));
  l.total = l.spans + round(groups * sizeof(Span));
  return l;
}

nf_status check_call(const void* table, const nf_norm_plan* plan, const float* norms, bool sums, const void* ws,
                     size_t ws_bytes, bool clips) {
  if (!plan) return bad("plan is NULL");
  if (plan->groups < 0 || plan->blocks < plan->groups || plan->pieces < 0) return bad("not a plan of nf_norm_plan_init");
  if (clips && !plan->writes) return bad("a tensor of the plan has no dst");
  if (plan->groups == 0) return NF_OK;
  if (!table) return bad("table is NULL");
  if (!norms) return bad("norms is NULL");
  if ((uintptr_t)table % 256 || (uintptr_t)norms % 4)
    return set_error(NF_ERR_ALIGNMENT, "table not 256-byte or norms not 4-byte aligned");
  if (sums) {
    if (ws_bytes < plan->workspace_bytes) return set_error(NF_ERR_WORKSPACE, "workspace smaller than the plan's");
    if (!ws) return set_error(NF_ERR_WORKSPACE, "workspace is NULL");
    if ((uintptr_t)ws % 256) return set_error(NF_ERR_ALIGNMENT, "workspace not 256-byte aligned");
  }
  return NF_OK;
}

NormArgs args_of(const void* table, const nf_norm_plan* plan, float* norms, void* ws) {
  const Layout l = layout_of(plan->pieces, plan->blocks, plan->groups);
  const unsigned char* base = static_cast<const unsigned char*>(table);
  NormArgs a = {};
  a.pieces = reinterpret_cast<const Piece*>(base + l.pieces);
  a.blocks = reinterpret_cast<const Block*>(base + l.blocks);
  a.spans = reinterpret_cast<const Span*>(base + l.spans);
  a.part = static_cast<double*>(ws);
  a.norms = norms;
  return a;
}

const char* check_limits(float max_norm, float eps) {
  if (!(max_norm >= 0.0f) || max_norm - max_norm != 0.0f) return "max_norm must be finite and >= 0";
  if (!(eps >= 0.0f) || eps - eps != 0.0f) return "eps must be finite and >= 0";
  return nullptr;
}

}  // namespace
}  // namespace nf

extern "C" {

nf_status nf_norm_plan_init(const nf_norm_tensor* tensors, int64_t count, int32_t groups, nf_norm_plan* plan) {
  using namespace nf;
  if (!plan) return bad("plan is NULL");
  *plan = nf_norm_plan{};
  if (count < 0 || count > kMaxTensors) return bad("count outside [0, 2^20]");
  if (groups < 0 || groups > kMaxGroups) return bad("groups outside [0, 2^16]");
  if (count && !tensors) return bad("tensors is NULL");
  bool writes = true;
  __int128 pieces_at_most = 0;
  for (int64_t i = 0; i < count; ++i) {
    const nf_status st = check_tensor(tensors[i], groups);
    if (st != NF_OK) return st;
    const nf_norm_tensor& t = tensors[i];
    if (t.rows == 0 || t.cols == 0) continue;
    writes &= t.dst != nullptr;
    pieces_at_most += one_row(t) ? 1 + (__int128)t.rows * t.cols / kMostPiece
                                 : t.cols < kMostPiece ? 1 + (__int128)t.rows / (kLeastPiece > t.cols ? kLeastPiece / t.cols : 1)
                                                       : (__int128)t.rows * (1 + t.cols / kMostPiece);
  }
  if (pieces_at_most > kMaxPieces) return set_error(NF_ERR_UNSUPPORTED, "tensors of more than 2^24 pieces");
  try {
    const nf_status st = check_apart(tensors, count);
    if (st != NF_OK) return st;
    int64_t pieces = 0, blocks = 0;
    cut(tensors, by_group(tensors, count), groups,
        [&](const nf_norm_tensor&, int64_t, int64_t, int64_t, int64_t) { ++pieces; },
        [&](int32_t, int64_t, int64_t) { ++blocks; });
    if (pieces > kMaxPieces) return set_error(NF_ERR_UNSUPPORTED, "tensors of more than 2^24 pieces");
    plan->pieces = pieces;
    plan->blocks = blocks;
    plan->groups = groups;
    plan->writes = writes;
    plan->table_bytes = layout_of(pieces, blocks, groups).total;
    plan->workspace_bytes = blocks * sizeof(double);
  } catch (...) {
    *plan = nf_norm_plan{};
    return set_error(NF_ERR_WORKSPACE, "no host memory for the plan");
  }
  return set_error(NF_OK, "");
}

nf_status nf_norm_table_init(const nf_norm_tensor* tensors, int64_t count, const nf_norm_plan* plan, void* table,
                             size_t table_bytes, void* stream) {
  using namespace nf;
  if (!plan) return bad("plan is NULL");
  if (table_bytes < plan->table_bytes) return set_error(NF_ERR_WORKSPACE, "table smaller than the plan's");
  nf_norm_plan again;
  nf_status st = nf_norm_plan_init(tensors, count, plan->groups, &again);
  if (st != NF_OK) return st;
  if (memcmp(&again, plan, sizeof(again))) return bad("plan is of other tensors");
  if (plan->groups == 0) return set_error(NF_OK, "");
  if (!table) return bad("table is NULL");
  if ((uintptr_t)table % 256) return set_error(NF_ERR_ALIGNMENT, "table not 256-byte aligned");
  std::vector<unsigned char> host;
  try {
    host.assign(plan->table_bytes, 0);
    const Layout l = layout_of(plan->pieces, plan->blocks, plan->groups);
    Piece* pieces = reinterpret_cast<Piece*>(host.data() + l.pieces);
    Block* blocks = reinterpret_cast<Block*>(host.data() + l.blocks);
    Span* spans = reinterpret_cast<Span*>(host.data() + l.spans);
    int32_t b = 0;
    cut(tensors, by_group(tensors, count), plan->groups,
        [&](const nf_norm_tensor& t, int64_t r, int64_t c, int64_t rows, int64_t cols) {
          Piece& p = *pieces++;
          const int64_t src = one_row(t) ? c : r * t.src_ld + c, dst = one_row(t) ? c : r * t.dst_ld + c;
          p.src = (const char*)t.src + src * (int64_t)type_bytes(t.src_type);
          p.dst = t.dst ? (char*)t.dst + dst * (int64_t)type_bytes(t.dst_type) : nullptr;
          p.src_ld = t.src_ld;
          p.dst_ld = t.dst_ld;
          p.rows = (int32_t)rows;
          p.cols = (int32_t)cols;
          p.src_type = t.src_type;
          p.dst_type = t.dst_type;
        },
        [&](int32_t g, int64_t first, int64_t n) {
          if (spans[g].count == 0) spans[g].first = b;
          ++spans[g].count;
          blocks[b++] = Block{(int32_t)first, (int32_t)n, g, 0};
        });
    for (int32_t g = 0; g < plan->groups; ++g)
      if (spans[g].count == 1) blocks[spans[g].first].lone = 1;
  } catch (...) {
    return set_error(NF_ERR_WORKSPACE, "no host memory for the table");
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipMemcpyAsync(table, host.data(), plan->table_bytes, hipMemcpyHostToDevice, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  return finish(e);
}

nf_status nf_grad_norm(const void* table, const nf_norm_plan* plan, float* norms, void* ws, size_t ws_bytes,
                       void* stream) {
  using namespace nf;
  const nf_status st = check_call(table, plan, norms, true, ws, ws_bytes, false);
  if (st != NF_OK) return st;
  if (plan->groups == 0) return set_error(NF_OK, "");
  const NormArgs a = args_of(table, plan, norms, ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  k_squares<<<(unsigned)plan->blocks, kNormThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan->blocks == plan->groups) return finish(e);  // a block each: it wrote the norm
  k_norms<<<(unsigned)plan->groups, kNormThreads, 0, s>>>(a);
  return finish(hipGetLastError());
}

nf_status nf_grad_clip(const void* table, const nf_norm_plan* plan, const float* norms, float max_norm, float eps,
                       void* stream) {
  using namespace nf;
  if (const char* why = check_limits(max_norm, eps)) return bad(why);
  const nf_status st = check_call(table, plan, norms, false, nullptr, 0, true);
  if (st != NF_OK) return st;
  if (plan->groups == 0) return set_error(NF_OK, "");
  NormArgs a = args_of(table, plan, const_cast<float*>(norms), nullptr);
  a.max_norm = max_norm;
  a.eps = eps;
  k_clip<false><<<(unsigned)plan->blocks, kNormThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  return finish(hipGetLastError());
}

nf_status nf_grad_norm_clip(const void* table, const nf_norm_plan* plan, float max_norm, float eps, float* norms,
                            void* ws, size_t ws_bytes, void* stream) {
  using namespace nf;
  if (const char* why = check_limits(max_norm, eps)) return bad(why);
  const nf_status st = check_call(table, plan, norms, true, ws, ws_bytes, true);
  if (st != NF_OK) return st;
  if (plan->groups == 0) return set_error(NF_OK, "");
  NormArgs a = args_of(table, plan, norms, ws);
  a.max_norm = max_norm;
  a.eps = eps;
  hipStream_t s = static_cast<hipStream_t>(stream);
  k_squares<<<(unsigned)plan->blocks, kNormThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return finish(e);
  k_clip<true><<<(unsigned)plan->blocks, kNormThreads, 0, s>>>(a);
  return finish(hipGetLastError());
}

}  // extern "C"
