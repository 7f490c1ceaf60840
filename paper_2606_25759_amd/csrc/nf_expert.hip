// nf_expert.hip - products of token rows with their expert's matrix, and the
// gradient of those matrices, for groups of rows of uneven sizes.
//
//   k_expert   D[q][p] = sum over r of Q[q][r] P[p][r] for one tile of one group:
//                FORWARD   y = W x:     P = W (n x k),    Q = x rows,   r over k
//                BACKWARD  y = W^T x:   P = W^T (k x n),  Q = x rows,   r over n
//                GRAD      dW = dy^T x: P = x^T (k x T),  Q = dy^T,     r over tokens
//   k_slim     FORWARD and BACKWARD for few rows: a tile's sum shared by the block's wavefronts
//   k_join     GRAD with tokens shared between blocks: the shares' sums, in order
//
// Group sizes are known on the device only, so the grid is the most that any
// sizes can need, and each wavefront finds its own tile by a scan over the
// offsets (a lane for every 1/64 of the experts); blocks past the last tile
// end at once.  Tiles never span groups: a group's last tile of rows is
// partly empty, which costs products but no memory traffic.
//
// P and Q lie in memory either with r adjacent (as the products take them) or
// with their own index adjacent (W for BACKWARD, both for GRAD); the latter
// are transposed on the way from LDS to registers, 16-bit elements by the
// LDS's own transposing read.
//
// FP16 and BF16 operands go to the matrix cores as they are, FP32 operands to
// its FP32 instruction; sums are FP32 in any case, each result rounded once.
#include <math.h>

#include <type_traits>

#include "nf_internal.h"
#include "nf_tile.h"
#include "nf_types.h"

namespace nf {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef int16_t short4v __attribute__((ext_vector_type(4)));

enum { FORWARD = NF_EXPERT_PRODUCT, BACKWARD = NF_EXPERT_TRANSPOSED, GRAD = NF_EXPERT_GRAD };

constexpr int kStageBytes = 128;  // of a row in LDS: 64 elements of 16 bits, 32 of FP32
constexpr int kMaxExperts = 4096;

struct ExpertArgs {
  const void *p, *q;
  int64_t p_ld, q_ld;              // elements between rows in memory
  int64_t p_worker, q_worker;      // between workers
  int64_t p_expert;                // between experts' matrices (FORWARD, BACKWARD)
  const void* offsets;             // [E + 1] of each worker
  int64_t offsets_stride;
  int64_t T;
  int32_t offsets64, E;
  int32_t P, Q, R;                 // lengths: of D's rows; GRAD: of its columns; FORWARD, BACKWARD: of r
  int32_t tp, tq;                  // tiles of P, and (GRAD) of Q
  int32_t rows;                    // of a group that a block takes: tile of Q, or (GRAD) tokens of a share
  void* out;
  int32_t out_type, accumulate;
  int64_t out_ld, out_worker, out_expert;
  float* part;                     // GRAD: sums of shares, [worker][unit][tile][elements]
  int32_t units;                   // most units of a worker: rounds up what any sizes need
  int32_t spread;                  // GRAD: see find()
};

// ------------------------------------------------------------ groups of rows

__device__ __forceinline__ int64_t offset_at(const ExpertArgs& a, int64_t worker, int e) {
  const int64_t at = worker * a.offsets_stride + e;
  int64_t v;
  if (a.offsets64)
    v = ((const int64_t*)a.offsets)[at];
  else
    v = ((const int32_t*)a.offsets)[at];
  return v < 0 ? 0 : v > a.T ? a.T : v;
}

struct Group {
  int32_t e, unit, units;  // expert, which of its units, how many it has
  int32_t base;            // units of the experts before it
  int64_t first, rows;     // its rows
};

// A group's units: a tile of rows each, or a share of its tokens (at least one: its gradient is written in any case).
template <int MODE>
__device__ __forceinline__ int units_of(const ExpertArgs& a, int64_t worker, int e, int64_t* first, int64_t* rows) {
  const int64_t lo = offset_at(a, worker, e), hi = offset_at(a, worker, e + 1);
  *first = lo;
  *rows = hi > lo ? hi - lo : 0;
  const int n = (int)(((uint32_t)*rows + (uint32_t)a.rows - 1) / (uint32_t)a.rows);
  return MODE == GRAD ? max(n, 1) : n;
}

// Sums of the lanes up to this one.
__device__ __forceinline__ int scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int w = __shfl_up(v, o);
    if (lane >= o) v += w;
  }
  return v;
}

// The group and unit of tile `block` of a worker, `per` tiles a unit; false past the last.  `id` becomes the tile's
// number in its group.  Blocks go round the eight XCDs: each takes a contiguous share of the tiles, whose operands its
// L2 then holds.
template <int MODE>
__device__ __forceinline__ bool find(const ExpertArgs& a, int64_t worker, int block, int per, Group* g, int* id) {
  const int lane = threadIdx.x % 64, each = (a.E + 63) / 64;
  int64_t first, rows;
  if (MODE == GRAD && a.spread) {
    // Tiles of long and short experts cost their tokens: every XCD takes an eighth of each expert's tiles, longest first
    // (32,768 tokens of 32 into 4096 x 2048: 692 us, 1,304 with a few experts an XCD).
    const int x = block & 7, j = block >> 3, lo = x * per >> 3, n = ((x + 1) * per >> 3) - lo, u = j / n;
    if (u >= a.E) return false;
    units_of<MODE>(a, worker, min(lane, a.E - 1), &first, &rows);
    const int mine = lane < a.E ? (int)rows : -1;
    int rank = 0;
    for (int m = 0; m < a.E; ++m) {
      const int other = __builtin_amdgcn_readlane(mine, m);
      rank += other > mine || (other == mine && m < lane);
    }
    const int at = __builtin_ctzll(__ballot(lane < a.E && rank == u));
    g->e = at;
    g->unit = g->base = 0;
    g->units = 1;
    g->first = __builtin_amdgcn_readlane((int)first, at);
    g->rows = __builtin_amdgcn_readlane(mine, at);
    *id = lo + j - u * n;
    return true;
  }
  int mine = 0;
  first = rows = 0;
  for (int j = 0; j < each; ++j)
    if (lane * each + j < a.E) mine += units_of<MODE>(a, worker, lane * each + j, &first, &rows);
  const int upto = scan(mine, lane);
  const int total = min(__builtin_amdgcn_readlane(upto, 63), a.units) * per;
  if (block >= total) return false;
  {
    const int x = block & 7, share = total >> 3, more = total & 7;
    block = x * share + min(x, more) + (block >> 3);
  }
  const int u = block / per;
  const int at = __builtin_ctzll(__ballot(upto > u));
  int base = __builtin_amdgcn_readlane(upto - mine, at), e = at * each, n = 0;
  if (each == 1) {
    n = __builtin_amdgcn_readlane(mine, at);
    first = __builtin_amdgcn_readlane((int)first, at);
    rows = __builtin_amdgcn_readlane((int)rows, at);
  } else {
    for (;; ++e) {
      n = units_of<MODE>(a, worker, e, &first, &rows);
      if (u < base + n || e + 1 >= a.E) break;
      base += n;
    }
  }
  g->e = __builtin_amdgcn_readfirstlane(e);
  g->units = __builtin_amdgcn_readfirstlane(n);
  g->base = __builtin_amdgcn_readfirstlane(base);
  g->unit = u - g->base;
  g->first = first;
  g->rows = rows;
  *id = block - g->base * per;
  return true;
}

// ----------------------------------------------------------------- operands

template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);  // elements of 16 bytes
template <typename T>
constexpr int kStageLen = kStageBytes / (int)sizeof(T);  // r of a stage

// Where BT x kStageLen elements lie in LDS, in pieces of 16 bytes.
//
// r adjacent: rows of 128 bytes, and slot j of row `row` holds its piece j ^ s(row).  A fragment is sixteen rows of
// thirty-two, 8 q + e and, in the odd fragment of a pair, 8 q + 4 + e (q, e in [0, 4)): of the products of a pair a
// lane then holds eight adjacent p.  A 16-byte read is served sixteen lanes at a time, which touch each of the 64
// banks once with this s.
//
// Own index adjacent: kStageLen rows of BT elements.  A fragment of 16-bit elements is sixteen adjacent columns, of
// which a transposing read gives each lane four rows of one, from 32 bytes of each of four rows; those go to slots
// that differ in the eight rows that are read at a time.  FP32 elements are read one by one, 64 bytes of four rows
// four apart.
template <typename T, int BT, int NW, bool TURNED, bool PAIRS = false>
struct Tile {
  static constexpr int kBytes = BT * kStageBytes;
  static constexpr int kLoads = BT / 8 / NW;  // of a wavefront, 1 KiB each
  static constexpr int kRow = TURNED ? BT * (int)sizeof(T) : kStageBytes;
  static constexpr int kRows = 1024 / kRow;  // of one load
  static constexpr int kReads = !TURNED ? 1 : sizeof(T) == 2 ? 2 : 4;  // of LDS, a fragment
  static_assert(BT % (8 * NW) == 0 && kRow <= 1024, "whole loads");

  static __device__ __forceinline__ int swizzle(int row) {
    if (!TURNED) {
      const int q = row >> 3;
      return PAIRS ? ((q >> 1) & 1) | (((q ^ (q >> 1)) & 1) << 1) | ((row & 2) << 1) : (row >> 1) & 7;
    }
    if (sizeof(T) == 2) return kRow >= 256 ? (row & 3) << 1 | (row & 8) : (row & 8) >> 2;
    return kRow >= 256 ? row & 12 : row & 4;
  }
  // The row and piece of it that lane `lane` of a wavefront loads in its i-th load.
  static __device__ __forceinline__ int load_row(int i, int wave, int lane) {
    return (i * NW + wave) * kRows + lane / (kRow / 16);
  }
  static __device__ __forceinline__ int load_piece(int row, int lane) { return (lane % (kRow / 16)) ^ swizzle(row); }

  // The bytes at which a lane reads fragment 0, first half, of the tile's part that begins at row or column w.
  static __device__ __forceinline__ uint32_t read_at(int w, int lane) {
    if (!TURNED) {
      const int row = w + (PAIRS ? lane % 16 / 4 * 8 + lane % 4 : lane % 16);
      return row * kStageBytes + ((lane / 16 ^ swizzle(row)) << 4);
    }
    if (sizeof(T) == 2) {
      const int row = lane / 16 * 8 + lane % 16 / 4;
      return row * kRow + ((w * 2 ^ swizzle(row) << 4) | (lane % 4 * 8));
    }
    const int row = lane / 16 * 4;
    return row * kRow + ((w * 4 ^ swizzle(row) << 4) | (lane % 16 * 4));
  }
  // Fragment i of half h; `at`: read_at's place in LDS.  What a fragment adds to it is a constant, or changes bits that
  // the rows' beginnings leave zero.
  static __device__ __forceinline__ uint4v read(uint32_t at, int i, int h) {
    if constexpr (!TURNED) {
      typedef const __attribute__((address_space(3))) uint4v* ptr;
      return *(ptr)(uintptr_t)((at ^ h * 64) + (PAIRS ? i / 2 * 32 + i % 2 * 4 : i * 16) * kStageBytes);
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) short4v* ptr;
      const uint32_t from = (at ^ i * 32) + h * 32 * kRow;
      const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)from));
      const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)(from + 4 * kRow)));
      return uint4v{x[0], x[1], y[0], y[1]};
    } else {
      typedef const __attribute__((address_space(3))) uint32_t* ptr;
      const uint32_t from = (at ^ i * 64) + h * 16 * kRow;
      uint4v v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *(ptr)(uintptr_t)(from + e * kRow);
      return v;
    }
  }
  // The place in the tile of a lane's column of fragment j of Q.
  static __device__ __forceinline__ int column_of(int j, int lane) { return 16 * j + lane % 16; }
};

__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (uint64_t)hi << 32 | lo;
}

// One operand's way from memory to LDS.
//
// PIECES: straight into LDS, 16 bytes a lane, for addresses and lengths in whole pieces.  ELEMENTS: the same by single
// elements of FP32, at any of their addresses and for any lengths.  What is past an end has an offset out of the buffer's
// range, for which the card writes zeros.  REGISTERS, a stage ahead: pieces at any element's address, and of one that its
// row ends in the last whole piece before that end, moved down when it goes to LDS; for 16 bits, FP32 gradients of narrow
// sides or few tokens (grad_plan), and rows so far apart that a tile's offsets would pass 32 bits.  Stages that exist as a whole are loaded without a branch, and in no
// stage does one load wait for another (3,001 FP16 rows of 515 by 7 of 515 x 1003: 37, 20 so).
enum { REGISTERS, ELEMENTS, PIECES };
constexpr uint32_t kNowhere = 0x80000000u;

// 16 bytes a lane (4: PIECE false) from base + off to LDS, lane after lane from `lds` on; zeros for off = kNowhere.
// Written out because the compiler, where it knows of such a load, waits for it before each transposing read of LDS (32,768 x
// 4096 x 2048 in 16 even experts: 580 us transposed, 490 without).  It has no result in registers, and who reads what it
// brings waits by wait_for().  The wait states are for a base that a vector instruction has just written; M0, which a clobber
// list cannot name, has no other use in these kernels.
template <bool PIECE>
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t lds, uint32_t off) {
  typedef uint32_t uint4s __attribute__((ext_vector_type(4)));
  const uint64_t at = (uint64_t)(uintptr_t)base;
  const uint4s buffer = {(uint32_t)at, (uint32_t)(at >> 32), 0x7fffffffu, 0x00020000u};
  if constexpr (PIECE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off),
                 "s"(buffer)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(buffer)
                 : "memory");
}

template <typename T, int BT, int NW, bool TURNED, bool PAIRS, int LOAD>
struct Operand {
  typedef Tile<T, BT, NW, TURNED, PAIRS> Lay;
  static constexpr bool DIRECT = LOAD != REGISTERS;
  static constexpr int kEach = LOAD == ELEMENTS ? 4 : 1;  // loads of 1 KiB
  static constexpr int kLoads = Lay::kLoads * kEach;
  static_assert(LOAD != ELEMENTS || sizeof(T) == 4, "elements of FP32");
  const char* at;   // of the tile at the next stage
  int64_t step;     // bytes of a stage
  int64_t row_bytes;
  int32_t left;     // r from there on
  int32_t extent;   // of the tile's own index
  int32_t length;   // of a row in memory
  bool held_whole;
  int32_t held_end; // what `left` or `extent` was when `held` was asked for
  uint32_t off[DIRECT ? kLoads : 1];
  uint4v held[DIRECT ? 1 : kLoads];
  int lane, wave;

  __device__ __forceinline__ void begin(const char* base, int64_t ld, int32_t extent_, int32_t r, int32_t length_,
                                        int wave_, int lane_) {
    length = length_;
    at = (const char*)uniform((uint64_t)(uintptr_t)base);
    row_bytes = ld * (int64_t)sizeof(T);
    step = TURNED ? row_bytes * kStageLen<T> : (int64_t)kStageBytes;
    left = __builtin_amdgcn_readfirstlane(r);
    extent = __builtin_amdgcn_readfirstlane(extent_);
    lane = lane_;
    wave = wave_;
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = row_of(i), c = element_of(i);
        off[i] = (TURNED ? c : row) < extent ? (uint32_t)(row * (int32_t)row_bytes + c * (int)sizeof(T)) : kNowhere;
      }
      if (left < kStageLen<T>) shorten();
    }
  }
  // The row and first element of it that this lane's i-th load brings: lanes take pieces, or four of them one.
  __device__ __forceinline__ int slot(int i) const { return LOAD == ELEMENTS ? i % kEach * 16 + lane / 4 : lane; }
  __device__ __forceinline__ int row_of(int i) const { return Lay::load_row(i / kEach, wave, slot(i)); }
  __device__ __forceinline__ int element_of(int i) const {
    return Lay::load_piece(row_of(i), slot(i)) * kPiece<T> + (LOAD == ELEMENTS ? lane % 4 : 0);
  }
  // The stage that is next ends before its place does.
  __device__ __forceinline__ void shorten() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if ((TURNED ? row_of(i) : element_of(i)) >= left) off[i] = kNowhere;
  }
  // Asks for the next stage: into LDS, or into registers.  In parts, for the loads to be placed one by one: load i of
  // the stage, and on to the next one.
  __device__ __forceinline__ void ask(uint32_t lds, int i) {
    if constexpr (DIRECT) {
      load_to_lds<LOAD == PIECES>(at, lds + (i / kEach * NW + wave) * 1024 + i % kEach * 256, off[i]);
    }
  }
  // Whether all of the next stage exists.
  __device__ __forceinline__ bool whole() const { return left >= kStageLen<T> && extent >= BT; }
  __device__ __forceinline__ void ask_held() {
    constexpr int N = kPiece<T>;
    const int end = TURNED ? extent : left;
    held_whole = whole();
    held_end = end;
    if (held_whole) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = Lay::load_row(i, wave, lane), c = Lay::load_piece(row, lane) * N;
        held[i] = __builtin_bit_cast(uint4v, *(const Near<T, N>*)(at + row * row_bytes + c * (int)sizeof(T)));
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = Lay::load_row(i, wave, lane), c = Lay::load_piece(row, lane) * N;
      const char* from = at + row * row_bytes;
      uint4v v = {};
      if ((TURNED ? row < left : row < extent) && c < end) {
        if (length >= N) {
          v = __builtin_bit_cast(uint4v, *(const Near<T, N>*)(from + min(c, end - N) * (int)sizeof(T)));
        } else {
          Near<T, N> x = {};
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (c + e < end) x.v[e] = ((const T*)from)[c + e];
          v = __builtin_bit_cast(uint4v, x);
        }
      }
      held[i] = v;
    }
  }
  __device__ __forceinline__ void on() {
    at += step;
    left -= kStageLen<T>;
    if constexpr (DIRECT)
      if (left < kStageLen<T>) shorten();
  }
  __device__ __forceinline__ void ask(uint32_t lds) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) ask(lds, i);
    } else {
      ask_held();
    }
    on();
  }
  // What was asked for into LDS, by registers.
  __device__ __forceinline__ void put(uint32_t lds) const {
    typedef __attribute__((address_space(3))) uint4v* ptr;
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        constexpr int N = kPiece<T>;
        const int c = Lay::load_piece(Lay::load_row(i, wave, lane), lane) * N;
        uint4v v = held[i];
        if (!held_whole && c + N > held_end && c < held_end && length >= N) {
          typedef unsigned __int128 wide;
          v = __builtin_bit_cast(uint4v, __builtin_bit_cast(wide, v) >> ((c + N - held_end) * 8 * (int)sizeof(T)));
        }
        *(ptr)(uintptr_t)(lds + (i * NW + wave) * 1024 + lane * 16) = v;
      }
    }
  }
};

// ----------------------------------------------------------------- products

template <typename T>
__device__ __forceinline__ float4v multiply(uint4v p, uint4v q, float4v c) {
  if constexpr (std::is_same<T, _Float16>::value) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, p), __builtin_bit_cast(half8, q), c, 0, 0,
                                                  0);
  } else if constexpr (std::is_same<T, Bf16>::value) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, p), __builtin_bit_cast(bhalf8, q), c, 0,
                                                   0, 0);
  } else {  // four r of each lane's group of lanes at a time
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(p[e]), __uint_as_float(q[e]), c, 0, 0, 0);
    return c;
  }
}

template <typename T>
constexpr int kMfmas = sizeof(T) == 2 ? 1 : 4;  // of multiply

// Asks the compiler to spread READS reads of LDS evenly between MFMAS matrix instructions, so that neither waits for a
// burst of the other.
template <int READS, int MFMAS>
__device__ __forceinline__ void spread() {
  constexpr int kEach = MFMAS / READS > 0 ? MFMAS / READS : 1;
#pragma unroll
  for (int i = 0; i < READS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
  }
}

// N results of one row of D, columns p .. of n.
template <typename T, int N>
__device__ __forceinline__ void store(T* to, int64_t p, int64_t n, int accumulate, const float (&v)[N]) {
  if (p + N <= n) {
    Near<T, N> w;
    if (accumulate) w = *(const Near<T, N>*)(to + p);
#pragma unroll
    for (int e = 0; e < N; ++e) w.v[e] = from_f32<T>(accumulate ? to_f32(w.v[e]) + v[e] : v[e]);
    *(Near<T, N>*)(to + p) = w;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (p + e < n) to[p + e] = from_f32<T>(accumulate ? to_f32(to[p + e]) + v[e] : v[e]);
  }
}

// Of a and b, which hold sixteen rows' (lane % 16) halves of 128 bytes, makes eight whole rows each: a the first eight, b
// the others, their first halves in the lanes below eight of sixteen.  Whole cache lines at a time: 4 x 2,048 tokens of 8
// added to 1024 x 512 take 38 us, 47 to 52 with two stores a line.
__device__ __forceinline__ void join_halves(uint4v& a, uint4v& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int x = (int)a[e], y = (int)b[e];
    a[e] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, 0x128, 0xf, 0xc, false);  // eight lanes round
    b[e] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xf, 0x3, false);
  }
}

// Eight results of 16 bits of one row from two fragments: of pairs they are adjacent, else of the first fragment in
// lanes 0 to 15 and 32 to 47 (its columns 0 to 7 and 8 to 15), of the second in the others.
template <typename T, bool PAIRS>
__device__ __forceinline__ uint4v eight(float4v a, float4v b) {
  struct Four {
    T v[4];
  };
  Four x, y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x.v[e] = from_f32<T>(a[e]);
    y.v[e] = from_f32<T>(b[e]);
  }
  const uint2v u = __builtin_bit_cast(uint2v, x), v = __builtin_bit_cast(uint2v, y);
  if (PAIRS) return uint4v{u[0], u[1], v[0], v[1]};
  const auto lo = __builtin_amdgcn_permlane16_swap(u[0], v[0], false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(u[1], v[1], false, false);
  return uint4v{lo[0], hi[0], lo[1], hi[1]};
}

template <typename T>
__device__ __forceinline__ void store_eight(T* to, int64_t p, int64_t n, uint4v v) {
  const Near<T, 8> w = __builtin_bit_cast(Near<T, 8>, v);
  if (p + 8 <= n) {
    *(Near<T, 8>*)(to + p) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (p + e < n) to[p + e] = w.v[e];
  }
}

// Part of a wavefront's tile: MI x NJ fragments at (wp, wq) of the tile at `out`, of which p < P and q < Q exist.
template <int MODE, typename LP, typename LQ, int MI, int NJ, typename T>
__device__ __forceinline__ void store_all(const ExpertArgs& a, T* out, int64_t P, int64_t Q, int wp, int wq, int lane,
                                          const float4v (&acc)[MI][NJ]) {
  constexpr bool PAIRS = MODE == FORWARD;  // two fragments' rows are adjacent
  const int accumulate = MODE == GRAD ? a.accumulate : 0;
  if constexpr (sizeof(T) == 4 && !PAIRS) {
    const int p = wp + lane / 16 * 4 + (lane & 8) * 2;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int q = wq + 16 * j + lane % 8;
#pragma unroll
      for (int i = 0; i < MI; i += 2) {
        uint4v x = __builtin_bit_cast(uint4v, acc[i][j]), y = __builtin_bit_cast(uint4v, acc[i + 1][j]);
        join_halves(x, y);
        const float4v u = __builtin_bit_cast(float4v, x), v = __builtin_bit_cast(float4v, y);
        const float first[4] = {u[0], u[1], u[2], u[3]}, second[4] = {v[0], v[1], v[2], v[3]};
        if (q < Q) store<T, 4>(out + q * a.out_ld, p + 16 * i, P, accumulate, first);
        if (q + 8 < Q) store<T, 4>(out + (q + 8) * a.out_ld, p + 16 * i, P, accumulate, second);
      }
    }
    return;
  }
  if constexpr (sizeof(T) == 2 && MI % 4 == 0) {
    const int g = lane / 16, p = wp + (PAIRS ? g * 8 : (g & 1) * 16 + (g >> 1) * 8) + (lane & 8) * 4;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int q = wq + 16 * j + lane % 8;
#pragma unroll
      for (int i = 0; i < MI; i += 4) {
        uint4v x = eight<T, PAIRS>(acc[i][j], acc[i + 1][j]), y = eight<T, PAIRS>(acc[i + 2][j], acc[i + 3][j]);
        join_halves(x, y);
        if (q < Q) store_eight(out + q * a.out_ld, p + 16 * i, P, x);
        if (q + 8 < Q) store_eight(out + (q + 8) * a.out_ld, p + 16 * i, P, y);
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int q = wq + LQ::column_of(j, lane);
    if (q >= Q) continue;
    T* to = out + q * a.out_ld;
    if constexpr (PAIRS) {
#pragma unroll
      for (int i = 0; i < MI; i += 2) {
        const float4v x = acc[i][j], y = acc[i + 1][j];
        const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        store<T, 8>(to, wp + 16 * i + lane / 16 * 8, P, accumulate, v);
      }
    } else {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const float4v x = acc[i][j];
        const float v[4] = {x[0], x[1], x[2], x[3]};
        store<T, 4>(to, wp + 16 * i + lane / 16 * 4, P, accumulate, v);
      }
    }
  }
}

// One BP x BQ tile, WP x WQ of it per wavefront; NS stages in LDS.
//
// One barrier a stage, in its middle: behind it the stage's place is free and the next one's loads have arrived.  The
// reads of the half stage that is next, and the loads of the stage after next, are placed between the products of the
// half that is in registers.
//
// What bounds it.  32,768 rows by 32 matrices of 4096 x 2048 in BF16, uneven: 528 to 555 us FORWARD (1.0 PFLOP/s), 522
// to 551 BACKWARD, 658 to 690 GRAD; rows spread evenly over 16: 500 to 545, 450 to 490, 507 to 555, where a library's
// one product of the sums' size takes 400, 436 and 525 (x W^T, x W, dy^T x).  Without loads the loop takes 379, with
// loads that all hit the L2 454, with its own 492 (FORWARD, even).  LDS has no bank conflicts; the matrix cores are at
// work 54% of the cycles, at 1.95 to 2.1 GHz (the library's product: 75% at 1.75: the card's power holds either).  What
// did not help: panels fetched into the L2 ahead (0 to 7% slower), a second barrier that lets loads go out half a stage
// earlier (0), four wavefronts of 128 x 128 (5 to 15% slower), 256 x 128 in two blocks a CU (0 to 15% slower), blocks
// that stay for several tiles and load the next one's before they store (0 to 4% slower), matrix instructions of 32 x 32
// (3 to 6% slower).  Small calls are bound by the launch and three waits for memory in a row: offsets, operands, stores;
// few rows by the matrices: 128 rows of 64 experts, 1024 x 2048: 29 us, 8 TB/s of what the last call left in the caches,
// 47 from memory.  FP32 is bound by its own matrix instruction: 32,768 rows by 32 of 4096 x 2048: 3,970 us, 0.138 of 0.15
// PFLOP/s; by what of tiles and rounds is empty in smaller calls.  By elements a stage of 128 x 128 is 128 loads, some 32
// cycles each: as long as its products, which hides them if barely (16,384 rows by 8 of 2047 x 1021: 575 us, 670 by
// registers; 8,192 of 8 into 1023 x 1021: 161, 190).
template <typename T, int MODE, int BP, int BQ, int WP, int WQ, int NS, int LOAD>
__global__ __launch_bounds__(BP / WP * (BQ / WQ) * 64, LOAD ? (BP / WP * (BQ / WQ) == 8 ? 1 : 2) : 4) void k_expert(
    ExpertArgs a) {
  constexpr int NW = BP / WP * (BQ / WQ);
  constexpr int MI = WP / 16, NJ = WQ / 16;
  constexpr bool DIRECT = LOAD != REGISTERS;
  typedef Operand<T, BP, NW, MODE != FORWARD, true, LOAD> OpP;
  typedef Operand<T, BQ, NW, MODE == GRAD, false, LOAD> OpQ;
  typedef typename OpP::Lay LP;
  typedef typename OpQ::Lay LQ;
  constexpr int kLoads = OpP::kLoads + OpQ::kLoads;
  __shared__ __align__(1024) char lds[NS * (LP::kBytes + LQ::kBytes)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int64_t worker = blockIdx.y;
  const int per = MODE == GRAD ? a.tp * a.tq : a.tp;
  Group g;
  int id;
  if (!find<MODE>(a, worker, blockIdx.x, per, &g, &id)) return;
  if (MODE == GRAD && a.accumulate && g.rows == 0) return;  // nothing to add
  int tp, tq;  // tile of P, and of Q or of the group's rows
  {            // four rows of tiles at a time
    const int across = MODE == GRAD ? a.tq : g.units;
    if (MODE == GRAD) id -= g.unit * per;
    const int four = id / (4 * a.tp), rows = min(4, across - 4 * four), in = id - four * 4 * a.tp;
    tq = 4 * four + in % rows;
    tp = in / rows;
  }
  OpP p;
  OpQ q;
  int32_t r;
  int64_t extent_q, q0;
  if (MODE == GRAD) {
    const int64_t from = (int64_t)g.unit * a.rows;
    const int64_t left = g.rows - from;
    r = (int32_t)(left < a.rows ? left : a.rows);
    const int64_t token = g.first + from;
    q0 = (int64_t)tq * BQ;
    extent_q = a.Q - q0;
    p.begin((const char*)a.p + (worker * a.p_worker + token * a.p_ld + (int64_t)tp * BP) * (int64_t)sizeof(T), a.p_ld,
            a.P - tp * BP, r, a.P, wave, lane);
    q.begin((const char*)a.q + (worker * a.q_worker + token * a.q_ld + q0) * (int64_t)sizeof(T), a.q_ld,
            (int32_t)extent_q, r, a.Q, wave, lane);
  } else {
    r = a.R;
    q0 = g.first + (int64_t)tq * BQ;
    extent_q = g.rows - (int64_t)tq * BQ;
    const int64_t at = g.e * a.p_expert + (int64_t)tp * BP * (MODE == FORWARD ? a.p_ld : 1);
    p.begin((const char*)a.p + at * (int64_t)sizeof(T), a.p_ld, a.P - tp * BP, r,
            MODE == FORWARD ? r : a.P, wave, lane);
    q.begin((const char*)a.q + (worker * a.q_worker + q0 * a.q_ld) * (int64_t)sizeof(T), a.q_ld,
            (int32_t)(extent_q < BQ ? extent_q : BQ), r, r, wave, lane);
  }
  const int wp = wave % (BP / WP) * WP, wq = wave / (BP / WP) * WQ;
  constexpr int kStage = LP::kBytes + LQ::kBytes;
  const uint32_t lds_at = (uint32_t)(uintptr_t)(lptr)lds;
  const uint32_t p_at = lds_at + LP::read_at(wp, lane), q_at = lds_at + LP::kBytes + LQ::read_at(wq, lane);
  float4v acc[MI][NJ] = {};
  struct Frags {
    uint4v p[MI], q[NJ];
  };
  auto read = [&](uint32_t stage, int h, Frags& f) {
#pragma unroll
    for (int i = 0; i < MI; ++i) f.p[i] = LP::read(p_at + stage, i, h);
#pragma unroll
    for (int j = 0; j < NJ; ++j) f.q[j] = LQ::read(q_at + stage, j, h);
  };
  constexpr int kAll = MI * NJ;
  auto products = [&](const Frags& f, int from, int to) {
#pragma unroll
    for (int m = from; m < to; ++m) acc[m / NJ][m % NJ] = multiply<T>(f.p[m / NJ], f.q[m % NJ], acc[m / NJ][m % NJ]);
  };
  auto ask = [&](uint32_t stage) {
    p.ask(lds_at + stage);
    q.ask(lds_at + stage + LP::kBytes);
  };
  auto put = [&](uint32_t stage) {
    p.put(lds_at + stage);
    q.put(lds_at + stage + LP::kBytes);
  };

  // Stage s: its first half is in registers.  Behind the barrier every wavefront has read all of it, and its loads of
  // stage s + 1 are in LDS; its place goes to stage s + NS.  Pieces of stages past the last are asked for as well, and are
  // zeros, so that the number of loads under way does not change; elements, whose loads take the most of a short sum's time,
  // are not.
  const int stages = __builtin_amdgcn_readfirstlane((r + kStageLen<T> - 1) / kStageLen<T>);
  Frags f0, f1;
  auto exists = [&](int s) { return LOAD != ELEMENTS || s < stages; };
  auto wait_below = [&](int s) {  // until stage s's loads are in LDS, with those of NS - 2 stages behind it under way
    if (exists(s + NS - 2))
      wait_for<DIRECT ? (NS - 2) * kLoads : 63, 0>();
    else
      wait_for<0, 0>();
  };
  if constexpr (DIRECT) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (exists(s)) ask(s * kStage);
    if (exists(NS - 1))
      wait_for<(NS - 1) * kLoads, 0>();
    else
      wait_for<0, 0>();
  } else {
    static_assert(DIRECT || NS == 2, "two stages");
    ask(0);
    put(0);
    ask(0);
    put(kStage);
    ask(0);
    wait_for<63, 0>();
  }
  block_barrier();
  uint32_t now = 0;
  if (wq >= extent_q) {  // none of this wavefront's rows exist: it only loads
    for (int s = 0; s < stages; ++s) {
      wait_below(s + 1);
      block_barrier();
      put(now);
      if (exists(s + NS)) ask(now);
      now = now + kStage == NS * kStage ? 0 : now + kStage;
    }
  } else if constexpr (!DIRECT) {  // by registers: more wavefronts a CU instead of fragments ahead of their use
    for (int s = 0; s < stages; ++s) {
      read(now, 0, f0);
      products(f0, 0, kAll);
      read(now, 1, f0);
      products(f0, 0, kAll);
      wait_for<63, 0>();
      block_barrier();
      put(now);
      ask(now);
      now ^= kStage;
    }
  } else {
    read(0, 0, f0);
    for (int s = 0; s < stages; ++s) {
      const uint32_t next = now + kStage == NS * kStage ? 0 : now + kStage;
      read(now, 1, f1);
      products(f0, 0, kAll);
      spread<(LP::kReads * MI + LQ::kReads * NJ), kAll * kMfmas<T>>();
      __builtin_amdgcn_sched_barrier(0);
      wait_below(s + 1);
      block_barrier();
      __builtin_amdgcn_sched_barrier(0);
      constexpr int kSome = LOAD == PIECES && kAll >= 2 * kLoads ? kLoads : 0;  // products between the loads
      if (exists(s + NS)) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
          if (n < OpP::kLoads)
            p.ask(lds_at + now, n);
          else
            q.ask(lds_at + now + LP::kBytes, n - OpP::kLoads);
          if (kSome) products(f1, n, n + 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        p.on();
        q.on();
      }
      read(next, 0, f0);
      products(f1, kSome, kAll);
      spread<(LP::kReads * MI + LQ::kReads * NJ), (kAll - kSome) * kMfmas<T>>();
      __builtin_amdgcn_sched_barrier(0);
      now = next;
    }
  }
  wait_for<0, 0>();  // what was asked for past the last stage

  if constexpr (MODE == GRAD) {
    if (g.units > 1) {
      float* to = a.part + (((int64_t)worker * a.units + g.base + g.unit) * per + id) * (BP * BQ);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i)
          *(float4v*)(to + (wq + LQ::column_of(j, lane)) * BP + wp + 16 * i + lane / 16 * 4) = acc[i][j];
      return;
    }
    float* out = (float*)a.out + worker * a.out_worker + g.e * a.out_expert + q0 * a.out_ld + (int64_t)tp * BP;
    store_all<MODE, LP, LQ>(a, out, a.P - tp * BP, extent_q, wp, wq, lane, acc);
  } else {
    const int64_t at = worker * a.out_worker + q0 * a.out_ld + (int64_t)tp * BP;
    with_type_on_device(a.out_type, [&](auto* t) {
      using O = std::remove_pointer_t<decltype(t)>;
      store_all<MODE, LP, LQ>(a, (O*)a.out + at, a.P - tp * BP, extent_q, wp, wq, lane, acc);
    });
  }
}

// A tile of 32 x 32 for few rows: its four wavefronts share the sum, a quarter of the stages each, from LDS of their own
// and without a barrier but for the last one, behind which they add up in their order.  More blocks, and a quarter of the
// way for each: 4096 x 4096 BF16 with one row takes 14.6 us, with tiles of 128 x 32 22.4.
template <typename T, int MODE, int LOAD>
__global__ __launch_bounds__(256) void k_slim(ExpertArgs a) {
  constexpr bool DIRECT = LOAD != REGISTERS;
  constexpr int B = 32, NW = 4, MI = 2, NJ = 2, NS = LOAD == PIECES ? 4 : 2;
  typedef Operand<T, B, 1, MODE != FORWARD, MODE == FORWARD, LOAD> OpP;
  typedef Operand<T, B, 1, false, false, LOAD> OpQ;
  typedef typename OpP::Lay LP;
  typedef typename OpQ::Lay LQ;
  constexpr int kLoads = OpP::kLoads + OpQ::kLoads, kStage = LP::kBytes + LQ::kBytes;
  __shared__ __align__(1024) char lds[NW][NS * kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int64_t worker = blockIdx.y;
  Group g;
  int id;
  if (!find<MODE>(a, worker, blockIdx.x, a.tp, &g, &id)) return;
  const int tq = id / a.tp, tp = id - tq * a.tp;
  const int64_t q0 = g.first + (int64_t)tq * B;
  const int rows = (int)(g.rows - (int64_t)tq * B < B ? g.rows - (int64_t)tq * B : B);
  const int all = (a.R + kStageLen<T> - 1) / kStageLen<T>;
  const int from = (int)((int64_t)all * wave / NW), to = (int)((int64_t)all * (wave + 1) / NW);
  const int begin = from * kStageLen<T>, end = min(a.R, to * kStageLen<T>);
  OpP p;
  OpQ q;
  const int64_t p_at = g.e * a.p_expert + (MODE == FORWARD ? (int64_t)tp * B * a.p_ld + begin
                                                          : (int64_t)begin * a.p_ld + (int64_t)tp * B);
  p.begin((const char*)a.p + p_at * (int64_t)sizeof(T), a.p_ld, a.P - tp * B, end - begin, MODE == FORWARD ? a.R : a.P,
          0, lane);
  q.begin((const char*)a.q + (worker * a.q_worker + q0 * a.q_ld + begin) * (int64_t)sizeof(T), a.q_ld, rows, end - begin,
          a.R, 0, lane);
  const uint32_t at = (uint32_t)(uintptr_t)(lptr)lds[wave];
  const uint32_t read_p = at + LP::read_at(0, lane), read_q = at + LP::kBytes + LQ::read_at(0, lane);
  float4v acc[MI][NJ] = {};
  auto ask = [&](uint32_t stage) {
    p.ask(at + stage);
    q.ask(at + stage + LP::kBytes);
  };
  auto put = [&](uint32_t stage) {
    p.put(at + stage);
    q.put(at + stage + LP::kBytes);
  };
  auto exists = [&](int s) { return LOAD != ELEMENTS || s < to; };
  if constexpr (DIRECT) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (exists(from + s)) ask(s * kStage);
  } else {
    ask(0);
    put(0);
    ask(0);
    put(kStage);
    ask(0);
  }
  uint32_t now = 0;
  for (int s = from; s < to; ++s) {
    if (exists(s + NS - 1))
      wait_for<DIRECT ? (NS - 1) * kLoads : 63, 0>();
    else
      wait_for<0, 0>();
    uint4v fp[2][MI], fq[2][NJ];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < MI; ++i) fp[h][i] = LP::read(read_p + now, i, h);
#pragma unroll
      for (int j = 0; j < NJ; ++j) fq[h][j] = LQ::read(read_q + now, j, h);
    }
    wait_for<63, 0>();  // they are read: their place is free
    put(now);
    if (exists(s + NS)) ask(now);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = multiply<T>(fp[h][i], fq[h][j], acc[i][j]);
    now = now + kStage == NS * kStage ? 0 : now + kStage;
  }
  wait_for<0, 0>();
  __syncthreads();
  float4v* sums = (float4v*)lds[0];
#pragma unroll
  for (int n = 0; n < NW; ++n) sums[(wave * NW + n) * 64 + lane] = acc[n / NJ][n % NJ];
  __syncthreads();
  float4v sum = {};
#pragma unroll
  for (int w = 0; w < NW; ++w) sum += sums[(w * NW + wave) * 64 + lane];
  const int i = wave / NJ, row = LQ::column_of(wave % NJ, lane);
  const int column = tp * B + (MODE == FORWARD ? lane / 16 * 8 + i * 4 : i * 16 + lane / 16 * 4);
  if (row >= rows) return;
  const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  with_type_on_device(a.out_type, [&](auto* t) {
    using O = std::remove_pointer_t<decltype(t)>;
    store<O, 4>((O*)a.out + worker * a.out_worker + (q0 + row) * a.out_ld, column, a.P, 0, v);
  });
}

// Elements of an expert's matrix whose tokens were shared: the shares' sums in order.  Block z of y of x: worker,
// expert, 1024 elements of a tile (30,011 tokens into 4 x (256 x 128) in 120 shares of two tiles:
// 6 us; 71 with a block a tile).
constexpr int kJoinThreads = 256;
constexpr int kJoinBlocks = 128 * 128 / 4 / kJoinThreads;  // of a tile

__global__ __launch_bounds__(kJoinThreads) void k_join(ExpertArgs a) {
  constexpr int B = 128, U = 8;
  const int lane = threadIdx.x % 64;
  const int64_t worker = blockIdx.z;
  const int e = blockIdx.y, per = a.tp * a.tq, tile = blockIdx.x / kJoinBlocks;
  int64_t first, rows;
  const int n = units_of<GRAD>(a, worker, e, &first, &rows);
  if (n == 1) return;
  int base = 0;
  for (int i = lane; i < e; i += 64) base += units_of<GRAD>(a, worker, i, &first, &rows);
  base = __builtin_amdgcn_readlane(scan(base, lane), 63);
  if (base + n > a.units) return;  // offsets that do not ascend
  const int at = (blockIdx.x % kJoinBlocks * kJoinThreads + threadIdx.x) * 4;
  const int64_t each = (int64_t)per * B * B;
  const float* from = a.part + ((int64_t)worker * a.units + base) * each + (int64_t)tile * B * B + at;
  float4v sum = {};
  for (int u = 0; u < n; u += U) {
    float4v v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = *(const float4v*)(from + min(u + i, n - 1) * each);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (u + i < n) sum += v[i];
  }
  const int four = tile / (4 * a.tp), trows = min(4, a.tq - 4 * four), in = tile - four * 4 * a.tp;
  const int64_t q = (int64_t)(4 * four + in % trows) * B + at / B, p = (int64_t)(in / trows) * B + at % B;
  if (q >= a.Q || p >= a.P) return;
  float* out = (float*)a.out + worker * a.out_worker + e * a.out_expert + q * a.out_ld + p;
  const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  store<float, 4>(out, 0, a.P - p, a.accumulate, v);
}

// --------------------------------------------------------------------- host

enum { SLIM, NARROW, MIDDLE, WIDE };  // tiles: 32 x 32, 128 x 32, 128 x 128, 256 x 256

struct Shape {
  int32_t W, E;
  int64_t T, n, k;
};

struct Plan {
  int tile, load;
  int32_t bp, bq, tp, tq, rows, units, spread;
  int64_t grid;        // blocks of a worker
  size_t part_bytes;
};

constexpr int64_t kCUs = 256;
constexpr int64_t kSlots = 2 * kCUs;  // blocks of tiles of 128 that the card holds at once
constexpr int64_t kMinShare = 256;       // tokens of a share, at least (128: 38 us where 30,011 of 4 take 34)

void finish_plan(Plan* p, const Shape& s, int mode) {
  p->bp = p->tile == WIDE ? 256 : p->tile == SLIM ? 32 : 128;
  p->bq = p->tile == WIDE ? 256 : p->tile == MIDDLE ? 128 : 32;
  p->tp = (int32_t)ceil_div(mode == FORWARD ? s.n : s.k, p->bp);
  const int64_t some = s.T < s.E ? s.T : s.E;  // experts with rows, at most
  int64_t units;
  if (mode == GRAD) {
    p->tq = (int32_t)ceil_div(s.n, p->bq);
    units = p->rows < s.T ? s.T / p->rows + s.E : s.E;
  } else {
    p->tq = 1;
    p->rows = p->bq;
    units = (s.T + some * (p->bq - 1)) / p->bq;
  }
  p->units = (int32_t)units;
  const int64_t per = (int64_t)p->tp * p->tq;
  p->spread = mode == GRAD && units == s.E && s.E <= 64 && per >= 16;
  p->grid = p->spread ? 8 * s.E * ceil_div(per, 8) : ceil_div(units * per, 8) * 8;  // workers begin on the same XCD
}

// FP32 takes six to eight times as long a stage as 16 bits, so that what of tiles and rounds is empty, or one after the
// other, counts for more than the rules for 16 bits allow.  The two functions below estimate a call's time and leave their
// choice where another's estimate is less by 15% and 4 us; experts' sizes, which the host does not know, move a call's
// time by as much as that.
bool pays(double other, double own) { return other < 0.85 * own && other < own - 4.0; }

// Tokens of a share, `rows` by the rule of grad_plan.
//
// In us: a tile's loop takes 0.075 a token, by registers 0.095; blocks beyond one a CU share its rate; the largest of N
// experts, of all workers, may have 1 + 0.4 log2 N times the average; a second launch costs 4, a share of a tile written and
// read again 0.024, and 0.08 in a row of them.  Over 1,588 sizes of 1 to 64 experts this takes 3% more than the best share,
// the rule for 16 bits 12%, and up to six times as long.  In us, not shared and shared: 32,768 tokens of 32 into 256 x 256:
// 213 and 67; 16,384 of 16 into 512 x 512: 226 and 119; 13,462 of 42 experts and 6 workers into 116 x 23: 176 and 70.
constexpr int64_t kMostShared = 1024;  // tiles' shares: 64 MiB of workspace
constexpr int64_t kShares[] = {64, 128, 192, 256, 384, 512, 768, 1024, 2048, 4096, 8192};

int64_t share_f32(const Shape& s, int64_t tiles, int load, int64_t rows) {
  const double even = (double)s.W * s.T * tiles / kCUs;  // tokens of a CU
  const int64_t some = s.T < s.E ? s.T : s.E;
  const double times = (1.0 + 0.4 * log2((double)s.W * s.E)) / s.E;
  const double largest = s.E == 1 || times > 1.0 ? s.T : times * s.T;
  auto time = [&](int64_t share) {
    const bool shared = share < s.T;
    const double shares = shared ? (double)s.T / share : 0.0, each = share < largest ? share : largest;
    double loop = each;
    if (s.E == 1)
      loop *= ceil_div(s.W * tiles * ceil_div(s.T, share), kCUs);
    else if (s.W * tiles * (shares + some) > kCUs && 1.05 * even > 0.55 * each)
      loop = 1.05 * even + 0.45 * each;
    return (load == REGISTERS ? 0.095 : 0.075) * loop + (shared ? 4.0 + 0.024 * s.W * (shares + s.E) * tiles + 0.08 * largest / share : 0.0);
  };
  int64_t best = s.T;
  double least = time(best);
  auto consider = [&](int64_t share) {
    if (share >= s.T || s.W * (s.T / share + s.E) * tiles > kMostShared) return;
    const double t = time(share);
    if (t >= least) return;
    least = t;
    best = share;
  };
  for (int64_t share : kShares) consider(share);
  if (s.E == 1) {  // whole rounds of blocks: 9,210 tokens into 704 x 2453: 350 us, 425
    for (int64_t blocks = kCUs; blocks <= kMostShared; blocks += kCUs)
      if (blocks >= 2 * s.W * tiles) consider(ceil_div(ceil_div(s.T, blocks / (s.W * tiles)), 64) * 64);
  }
  return pays(least, time(rows)) ? best : rows;
}

// The gradient in tiles of 128, with shared tokens where that saves more than it costs, in us.
//
// 16 bits: a tile's loop takes 0.012 a token, an expert may have twice the average, and what is above an even share of
// all tiles' tokens is saved; a second launch and its latency cost 8, a share of a tile written and read again 0.026.
// BF16, shared and not: 32,768 tokens of 16 experts into 512 x 512: 50 and 86; 2,048 of 4 into 1024 x 1024: 37 and 17;
// by registers, 3,001 of 7 into 515 x 1003: 41 and 24; the rule takes the slower form of 32,768 tokens of 20 into 512 x 512
// (48 and 60) and of 6 into 1024 x 1024 (115 and 91), where the experts' sizes decide, which the host does not know.  Over
// 1,473 sizes of 1 to 64 experts, a third of them by registers, BF16 takes 3% more than the best share.
//
// FP32 that is not read by pieces goes by elements where sides are above 64 and an expert or share has some 96 tokens, else by
// registers: of narrow sides most loads of elements are of none, and few tokens do not pay for them (elements / registers:
// 8,192 tokens of 8 into 1023 x 1021: 161 / 190; 14 x 71 into 17 x 2392: 25 / 20; one into 157 x 251: 17.6 / 13.6).
Plan grad_plan(const Shape& s, bool f32, int load) {
  Plan p = {};
  p.tile = MIDDLE;
  p.load = load == ELEMENTS && (s.n <= 64 || s.k <= 64) ? REGISTERS : load;
  const int64_t tiles = ceil_div(s.n, 128) * ceil_div(s.k, 128), all = s.W * s.E * tiles;
  int64_t rows = s.T > 0 ? s.T : 1;
  if (all < kSlots && s.T > 0) {
    int64_t share = ceil_div(ceil_div(s.W * s.T * tiles, kSlots), 64) * 64;
    share = share < kMinShare ? kMinShare : share;
    const double saved = 0.012 * (2.0 * s.T / s.E - (double)s.W * s.T * tiles / kSlots);
    const double cost = 8.0 + 0.026 * s.W * (double)(s.T / share + s.E) * tiles;
    if (saved > cost) rows = share;
  }
  if (f32 && s.T > 0) rows = share_f32(s, tiles, p.load, rows);
  if (p.load == ELEMENTS && (rows < 96 || s.T < 96 * (int64_t)s.E)) p.load = REGISTERS;
  p.rows = (int32_t)rows;
  finish_plan(&p, s, GRAD);
  if (rows < s.T) p.part_bytes = (size_t)(s.W * p.units * tiles) * 128 * 128 * sizeof(float);
  return p;
}

// The tile of an FP32 product, `tile` by the rule of plan_of.
//
// The estimate is
//   max(rounds x (4 + stages x alone), most blocks of a CU x stages x together) us,
// with the times of a stage of a block alone on its CU and of one that shares it, below; a wavefront of a tile of 32 has a
// quarter of the stages.  Over 2,404 sizes of 1 to 64 experts it takes 1.4% more than the best of the three, the rule of
// plan_of 6%, and up to three times as long where results are narrow or few and sums long (32 / 128 x 32 / 128): 22,635
// rows of 3 experts, 19 x 3000: 67 / 156 / 179; by elements, 8,192 of 8, 1023 x 1021: - / 181 / 203.
struct StageTime {
  int64_t blocks;  // that a CU holds
  double alone, together;
};
constexpr StageTime kStageF32[3][3] = {  // [load][tile]
    {{2, 1.51, 1.10}, {4, 1.32, 0.87}, {2, 2.55, 2.39}},
    {{2, 0.79, 0.87}, {2, 0.76, 0.56}, {2, 2.25, 1.99}},
    {{1, 0.61, 0.61}, {2, 0.57, 0.54}, {2, 1.56, 1.84}}};

int tile_f32(const Shape& s, int64_t len, int64_t r, int load, int tile) {
  const int64_t all = ceil_div(r, kStageBytes / 4);
  const double some = s.E * (1.0 - exp(-(double)s.T / s.E));  // experts with rows, if each row's is any of them
  auto time = [&](int t) {
    const int64_t bp = t == SLIM ? 32 : 128, bq = t == MIDDLE ? 128 : 32, stages = t == SLIM ? ceil_div(all, 4) : all;
    const double full = (double)s.T / bq + 0.5 * some;  // last tiles are half empty
    const bool one = s.E == 1 || s.T == 1;
    const double units = one ? ceil_div(s.T, bq) : some > full ? some : full;
    const StageTime& c = kStageF32[load][t];
    double sum = 0.0;
    for (double off : {0.9, 1.0, 1.1}) {  // a block more than there are CUs may be one less
      const double blocks = s.W * units * ceil_div(len, bp) * (one ? 1.0 : off);
      const double rounds = ceil(blocks / (kCUs * c.blocks)) * (4.0 + stages * c.alone);
      const double rate = ceil(blocks / kCUs) * stages * c.together;
      sum += rounds > rate ? rounds : rate;
    }
    return sum / 3.0;
  };
  int best = SLIM;
  for (int t : {NARROW, MIDDLE})
    if (time(t) < time(best)) best = t;
  return pays(time(best), time(tile)) ? best : tile;
}

// Which tiles a call takes, by how many there are of each if the experts' sizes are alike (measured in us, BF16 unless
// stated, with tiles of 32 / 128 x 32 / 128 / 256):
//   256    needs as many as there are CUs, and experts that fill them: 32,768 rows of 32 experts, 4096 x 2048: 1,604 with
//          128 through registers, 547; 4,096 rows of 16, 2048 x 2048 (192 tiles): - / 80 / 56 / 57; 1,024 rows of one,
//          4096 x 4096 (64): - / 68 / 48 / 90
//   128    8,192 rows of 8, 1024 x 1024 (576): 149 / 47 / 34 / 34; where there are too few, 128 x 32: 1,024 rows of one,
//          1024 x 1024 (64): 21 / 13 / 15 / 29.  FP32, whose products take long enough for a part of a tile and of a round
//          to count for more, needs two rounds and experts of 192 rows: 128 x 32 / 128: 32,768 rows of 32, 4096 x 2048:
//          4,676 / 4,064; of 128, 256 and 512, 2048 x 1024: 1,369 / 1,297, 1,475 / 1,536, 1,735 / 2,167; 16,384 of 8,
//          2047 x 1021: 869 / 769; 8,192 of 8, 2048 x 2048 (1,088 tiles): 692 / 663, 1024 x 1024 (544): 186 / 203; what
//          tile_f32 finds by its estimate goes before
//   128x32 for experts of few rows: 2,048 rows of 64, 1024 x 1024: 63 / 29 / 36 / 31
//   32     where there are few of those: one row, 4096 x 4096 (32 of 128 x 32): 15 / 22 / 39; 64 rows of 8, 2048 x 2048
//          (150): 19 / 15 / 25
Plan plan_of(const Shape& s, int mode, int32_t type, int load) {
  Plan p = {};
  p.load = load;
  const int64_t experts = s.E > 0 ? s.E : 1, some = s.T < experts ? s.T : experts;
  const int64_t rows = s.T / experts;  // of an expert, on average
  const int64_t len = mode == FORWARD ? s.n : s.k;
  const bool fits = load == PIECES && type != NF_TYPE_F32 && len >= 192;
  if (mode == GRAD) {
    if (!fits || s.n < 192 || s.W * s.E * ceil_div(s.n, 256) * ceil_div(s.k, 256) < kCUs)
      return grad_plan(s, type == NF_TYPE_F32, load);
    p.tile = WIDE;
    p.rows = (int32_t)(s.T > 0 ? s.T : 1);
  } else {
    auto tiles = [&](int64_t bp, int64_t bq) { return s.W * (s.T / bq + (some + 1) / 2) * ceil_div(len, bp); };
    if (fits && rows >= 192 && s.W * ceil_div(s.T, 256) * ceil_div(len, 256) >= kCUs)
      p.tile = WIDE;
    else if (type != NF_TYPE_F32 ? rows > 48 && tiles(128, 128) >= kCUs / 2 : rows >= 192 && tiles(128, 128) >= 2 * kSlots)
      p.tile = MIDDLE;
    else
      p.tile = tiles(128, 32) > kCUs * 3 / 8 ? NARROW : SLIM;
    if (type == NF_TYPE_F32) p.tile = tile_f32(s, len, mode == FORWARD ? s.k : s.n, load, p.tile);
  }
  finish_plan(&p, s, mode);
  return p;
}

template <typename T, int MODE, int LOAD>
void launch(const Plan& p, const Shape& s, const ExpertArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)p.grid, (unsigned)s.W);
  if constexpr (LOAD == PIECES && sizeof(T) == 2) {
    if (p.tile == WIDE) {
      k_expert<T, MODE, 256, 256, 128, 64, 2, PIECES><<<grid, 512, 0, stream>>>(a);
      return;
    }
  }
  if constexpr (MODE != GRAD) {
    if (p.tile == SLIM) {
      k_slim<T, MODE, LOAD><<<grid, 256, 0, stream>>>(a);
      return;
    }
    if (p.tile == NARROW) {
      k_expert<T, MODE, 128, 32, 32, 32, LOAD == PIECES ? 4 : LOAD == ELEMENTS ? 3 : 2, LOAD><<<grid, 256, 0, stream>>>(a);
      return;
    }
  }
  if constexpr (LOAD != REGISTERS)
    k_expert<T, MODE, 128, 128, 64, 64, 2, LOAD><<<grid, 256, 0, stream>>>(a);
  else
    k_expert<T, MODE, 128, 128, 64, 32, 2, LOAD><<<grid, 512, 0, stream>>>(a);
}

template <int MODE>
hipError_t run(const Plan& p, const Shape& s, ExpertArgs a, int32_t type, hipStream_t stream) {
  a.tp = p.tp;
  a.tq = p.tq;
  a.rows = p.rows;
  a.units = p.units;
  a.spread = p.spread;
  with_type(type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (p.load == PIECES) {
      launch<T, MODE, PIECES>(p, s, a, stream);
    } else if (p.load == REGISTERS) {
      launch<T, MODE, REGISTERS>(p, s, a, stream);
    } else {
      if constexpr (sizeof(T) == 4) launch<T, MODE, ELEMENTS>(p, s, a, stream);
    }
    if constexpr (MODE == GRAD) {
      if (p.part_bytes && hipPeekAtLastError() == hipSuccess)
        k_join<<<dim3((unsigned)(p.tp * p.tq * kJoinBlocks), (unsigned)s.E, (unsigned)s.W), kJoinThreads, 0, stream>>>(a);
    }
  });
  return hipGetLastError();
}

constexpr int64_t kMaxTokens = 1 << 24, kMaxSide = 1 << 20;

nf_status bad(const char* what) { return set_error(NF_ERR_INVALID_ARG, what); }

const char* check_sizes(int32_t W, int64_t T, int32_t E, int64_t n, int64_t k) {
  if (W < 1 || W > 255) return "W outside [1, 255]";
  if (T < 0 || T > kMaxTokens) return "T outside [0, 2^24]";
  if (E < 0 || E > kMaxExperts) return "E outside [0, 4096]";
  if (n < 0 || n > kMaxSide || k < 0 || k > kMaxSide) return "n or k outside [0, 2^20]";
  return nullptr;
}

// Whether W x rows x cols elements lie as a caller says.
bool misplaced(int32_t W, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
  return ld < cols || (W > 1 && rows > 0 && overlaps(stride, rows, ld, cols));
}

// W x rows runs of cols elements, as a caller lays them out, in bytes.
struct Runs {
  __int128 at, count, far, each;  // far: from one run's beginning to the next one's; each: a run's length
  bool even;                      // all runs lie `far` apart
};

Runs runs_of(const void* p, int32_t W, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int32_t type) {
  const __int128 size = (__int128)type_bytes(type);
  Runs r = {(__int128)(uintptr_t)p, rows, ld * size, cols * size, true};
  if (rows == 1) r.far = r.each;
  if (W > 1) {
    if (rows == 1) r.far = stride * size;
    r.even = stride * size == rows * r.far;
    if (r.even) r.count *= W;
  }
  if (r.even && (r.count == 1 || r.far == r.each)) {
    r.each *= r.count;
    r.far = r.each;
    r.count = 1;
  }
  return r;
}

// Whether two tensors share an element, as far as a few divisions tell: exactly where one is a single run or their runs
// lie equally far apart, and where they begin at the same place.
bool share(const Runs& a, const Runs& b) {
  if (a.count <= 0 || b.count <= 0 || a.each <= 0 || b.each <= 0) return false;
  if (a.at == b.at) return true;
  if (!a.even || !b.even || (a.count > 1 && b.count > 1 && a.far != b.far)) return false;
  // runs i of a and j of b meet where b.at - a.at + j b.far - i a.far is in (-b.each, a.each); with d the run of a less
  // that of b, of one far: the first d, rounded down, that brings b's beginning below a's end
  const __int128 far = a.count > 1 ? a.far : b.far, between = b.at - a.at - a.each;
  __int128 d = between / far + (between % far < 0 ? 0 : 1);
  if (d < 1 - b.count) d = 1 - b.count;
  return d <= a.count - 1 && b.at - a.at - d * far < a.each && b.at - a.at - d * far > -b.each;
}

bool whole(const void* p, int64_t ld, int64_t stride, int32_t type) {
  const int64_t bytes = (int64_t)type_bytes(type);
  return (uintptr_t)p % 16 == 0 && ld % (16 / bytes) == 0 && stride % (16 / bytes) == 0;
}

// How two operands are read: `pieces` says that their lengths and places are whole pieces of 16 bytes.
int load_of(int32_t type, bool pieces, int64_t p_ld, int64_t q_ld) {
  if (p_ld > kMaxSide || q_ld > kMaxSide) return REGISTERS;  // offsets of a tile's rows in 32 bits
  return pieces ? PIECES : type == NF_TYPE_F32 ? ELEMENTS : REGISTERS;
}

// A launch has under 2^32 threads, and every worker's tiles a number.
bool too_large(const Plan& p, int32_t W) { return p.grid > (1 << 22) || p.grid * W > (1 << 22); }

nf_status finish(hipError_t e) {
  if (e != hipSuccess) return set_error(NF_ERR_HIP, hipGetErrorString(e));
  return set_error(NF_OK, "");
}

}  // namespace
}  // namespace nf

extern "C" {

nf_status nf_expert_product(const void* x, int32_t type, int64_t x_ld, int64_t x_stride, const void* w, int64_t w_ld,
                            int64_t w_stride, int32_t transposed, const void* offsets, int32_t offsets_bytes,
                            int64_t offsets_stride, int32_t W, int64_t T, int32_t E, int64_t n, int64_t k, void* y,
                            int32_t y_type, int64_t y_ld, int64_t y_stride, void* stream) {
  using namespace nf;
  if (!known_type(type) || !known_type(y_type)) return bad("unknown element type");
  if (transposed != 0 && transposed != 1) return bad("transposed must be 0 or 1");
  if (offsets_bytes != 4 && offsets_bytes != 8) return bad("offsets_bytes must be 4 or 8");
  if (const char* why = check_sizes(W, T, E, n, k)) return bad(why);
  const int64_t in = transposed ? n : k, out = transposed ? k : n;
  if (misplaced(W, T, in, x_ld, x_stride)) return bad("x_ld or x_stride too small");
  if (misplaced(W, T, out, y_ld, y_stride)) return bad("y_ld or y_stride too small");
  if (w_ld < k || (E > 1 && n > 0 && overlaps(w_stride, n, w_ld, k))) return bad("w_ld or w_stride too small");
  if (W > 1 && offsets_stride < E + 1) return bad("offsets_stride < E + 1");
  if (T == 0 || E == 0 || out == 0) return set_error(NF_OK, "");
  if (!offsets || !y || (in > 0 && (!x || !w))) return bad("x, w, offsets or y is NULL");
  if (y == x || y == w) return bad("y must not be x or w");
  if ((uintptr_t)x % type_bytes(type) || (uintptr_t)w % type_bytes(type) || (uintptr_t)y % type_bytes(y_type) ||
      (uintptr_t)offsets % offsets_bytes)
    return set_error(NF_ERR_ALIGNMENT, "x, w, offsets or y not aligned to its elements");
  const Shape s = {W, E, T, n, k};
  const int64_t piece = 16 / (int64_t)type_bytes(type);
  const bool pieces = whole(x, x_ld, W > 1 ? x_stride : 0, type) && whole(w, w_ld, E > 1 ? w_stride : 0, type) &&
                      k % piece == 0 && (!transposed || n % piece == 0);
  const Plan p = plan_of(s, transposed ? BACKWARD : FORWARD, type, load_of(type, pieces, w_ld, x_ld));
  if (too_large(p, W)) return set_error(NF_ERR_UNSUPPORTED, "more tiles than a launch has");
  const Runs to = runs_of(y, W, T, out, y_ld, y_stride, y_type);
  if (share(to, runs_of(x, W, T, in, x_ld, x_stride, type)) || share(to, runs_of(w, E, n, k, w_ld, w_stride, type)))
    return bad("y shares an element with x or w");
  ExpertArgs a = {};
  a.p = w;
  a.p_ld = w_ld;
  a.p_expert = w_stride;
  a.q = x;
  a.q_ld = x_ld;
  a.q_worker = x_stride;
  a.offsets = offsets;
  a.offsets_stride = offsets_stride;
  a.offsets64 = offsets_bytes == 8;
  a.T = T;
  a.E = E;
  a.P = (int32_t)out;
  a.R = (int32_t)in;
  a.out = y;
  a.out_type = y_type;
  a.out_ld = y_ld;
  a.out_worker = y_stride;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return finish(transposed ? run<BACKWARD>(p, s, a, type, st) : run<FORWARD>(p, s, a, type, st));
}

size_t nf_expert_grad_workspace_bytes(int32_t W, int64_t T, int32_t E, int64_t n, int64_t k) {
  using namespace nf;
  if (check_sizes(W, T, E, n, k) || T == 0 || E == 0 || n == 0 || k == 0) return 0;
  const Shape s = {W, E, T, n, k};
  size_t most = 0;  // of any type and alignment
  // elements have the shares of pieces or of registers
  for (const Plan& p : {grad_plan(s, false, PIECES), grad_plan(s, true, PIECES), grad_plan(s, true, REGISTERS)})
    most = p.part_bytes > most ? p.part_bytes : most;
  return most;
}

nf_status nf_expert_path(int32_t op, int32_t type, int32_t W, int64_t T, int32_t E, int64_t n, int64_t k,
                         int32_t whole, nf_expert_path_info* info) {
  using namespace nf;
  if (!info) return bad("info is NULL");
  *info = nf_expert_path_info{};
  if (op < NF_EXPERT_PRODUCT || op > NF_EXPERT_GRAD) return bad("unknown op");
  if (!known_type(type)) return bad("unknown element type");
  if (whole != 0 && whole != 1) return bad("whole must be 0 or 1");
  if (const char* why = check_sizes(W, T, E, n, k)) return bad(why);
  if (E == 0 || (op == NF_EXPERT_GRAD ? n == 0 || k == 0 : T == 0 || (op == NF_EXPERT_PRODUCT ? n : k) == 0))
    return set_error(NF_OK, "");
  const Plan p = plan_of(Shape{W, E, T, n, k}, op, type, load_of(type, whole != 0, 0, 0));
  if (too_large(p, W)) return set_error(NF_ERR_UNSUPPORTED, "more tiles than a launch has");
  info->tile_columns = p.bp;
  info->tile_rows = p.bq;
  info->direct = whole;
  info->share = p.part_bytes ? p.rows : 0;
  return set_error(NF_OK, "");
}

nf_status nf_expert_grad(const void* dy, int64_t dy_ld, int64_t dy_stride, const void* x, int64_t x_ld,
                         int64_t x_stride, int32_t type, const void* offsets, int32_t offsets_bytes,
                         int64_t offsets_stride, int32_t W, int64_t T, int32_t E, int64_t n, int64_t k,
                         int32_t accumulate, float* grads, int64_t matrix_stride, int64_t worker_stride, void* ws,
                         size_t ws_bytes, void* stream) {
  using namespace nf;
  if (!known_type(type)) return bad("unknown element type");
  if (offsets_bytes != 4 && offsets_bytes != 8) return bad("offsets_bytes must be 4 or 8");
  if (const char* why = check_sizes(W, T, E, n, k)) return bad(why);
  if (misplaced(W, T, n, dy_ld, dy_stride)) return bad("dy_ld or dy_stride too small");
  if (misplaced(W, T, k, x_ld, x_stride)) return bad("x_ld or x_stride too small");
  if (accumulate != 0 && accumulate != 1) return bad("accumulate must be 0 or 1");
  if (E > 1 && matrix_stride < n * k) return bad("matrix_stride < n * k");
  if (W > 1 && E > 0 && overlaps(worker_stride, E, E > 1 ? matrix_stride : n * k, n * k))
    return bad("worker_stride too small");
  if (W > 1 && offsets_stride < E + 1) return bad("offsets_stride < E + 1");
  if (E == 0 || n == 0 || k == 0) return set_error(NF_OK, "");
  if (!offsets || !grads || (T > 0 && (!dy || !x))) return bad("dy, x, offsets or grads is NULL");
  if ((uintptr_t)dy % type_bytes(type) || (uintptr_t)x % type_bytes(type) || (uintptr_t)grads % 4 ||
      (uintptr_t)offsets % offsets_bytes)
    return set_error(NF_ERR_ALIGNMENT, "dy, x, offsets or grads not aligned to its elements");
  const Shape s = {W, E, T, n, k};
  const int64_t piece = 16 / (int64_t)type_bytes(type);
  const bool pieces = whole(dy, dy_ld, W > 1 ? dy_stride : 0, type) && whole(x, x_ld, W > 1 ? x_stride : 0, type) &&
                      n % piece == 0 && k % piece == 0;
  const Plan p = plan_of(s, GRAD, type, load_of(type, pieces, x_ld, dy_ld));
  if (too_large(p, W)) return set_error(NF_ERR_UNSUPPORTED, "more tiles than a launch has");
  const size_t need = nf_expert_grad_workspace_bytes(W, T, E, n, k);
  if (ws_bytes < need) return set_error(NF_ERR_WORKSPACE, "workspace smaller than nf_expert_grad_workspace_bytes");
  if (need && !ws) return set_error(NF_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)ws % 256) return set_error(NF_ERR_ALIGNMENT, "workspace not 256-byte aligned");
  const Runs to = runs_of(grads, W, E, n * k, matrix_stride, worker_stride, NF_TYPE_F32);
  if (share(to, runs_of(dy, W, T, n, dy_ld, dy_stride, type)) || share(to, runs_of(x, W, T, k, x_ld, x_stride, type)))
    return bad("grads shares an element with dy or x");
  ExpertArgs a = {};
  a.p = x;
  a.p_ld = x_ld;
  a.p_worker = x_stride;
  a.q = dy;
  a.q_ld = dy_ld;
  a.q_worker = dy_stride;
  a.offsets = offsets;
  a.offsets_stride = offsets_stride;
  a.offsets64 = offsets_bytes == 8;
  a.T = T;
  a.E = E;
  a.P = (int32_t)k;
  a.Q = (int32_t)n;
  a.out = grads;
  a.accumulate = accumulate;
  a.out_ld = k;
  a.out_worker = worker_stride;
  a.out_expert = matrix_stride;
  a.part = static_cast<float*>(ws);
  return finish(run<GRAD>(p, s, a, type, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
