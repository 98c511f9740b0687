// Shared by the kernels of the grouped operators (the matrix of a row is chosen by the row's group): descriptors,
// the search of a workgroup for its tile, and the tile product that they are built from.
#ifndef LQ_GROUPED_H_
#define LQ_GROUPED_H_

#include "lq_common.h"

namespace lq {

constexpr int64_t MOST_THREADS = 0xffffffffll;     // of a launch

// Everything a product needs, by value as the kernel argument.  The operator is Y[row(p)] = X[row(p)] * W_group(p).
struct GroupedArgs {
  const int32_t* off;     // [G + 1]; NULL: all positions use the first matrix
  const int32_t* order;   // [n] or NULL
  int32_t G, n;
  const void* X; int64_t ldx;
  const void* W; int64_t ldw, sw;       // sw: elements from one matrix to the next
  const void* bias; int64_t ldb;        // row g, or row 0 of a shared matrix
  const void* gate; int64_t ldg;
  void* Y; int64_t ldy;
  int32_t K, N;           // inner width and width of the result
  int32_t n_store;        // columns stored (>= N; those past N hold no result)
  int32_t slots;          // row r of Y reads row r / slots of X
  int32_t x_grouped, y_grouped;
  int32_t relu, y_bf16;
  int32_t y_vec;          // rows of Y, bias and gate are aligned to 16 bytes
  int32_t tiles_n, row_tiles;
  int32_t steps_per_split;   // K steps of one split; split z writes at Y + z * split_stride
  int64_t split_stride;
  int32_t* gpos;          // out: group of every position, -1 for none (or NULL)
  // adapters: U [n x rp] by position, fp32 or as two bf16 numbers (the second `u_rest` elements behind the first), B_g [rank x N]
  const void* U; int64_t u_rest; int32_t rp, rank;
  const void* B; int64_t ldB, sB;
  const int32_t* group_of;   // gpos of the product that made U
};

struct GradientArgs {
  const int32_t* off;
  const int32_t* order;
  int32_t G, n;
  const void* X; int64_t ldx; int32_t slots, x_grouped;
  const void* dY; int64_t ldy; int32_t y_grouped;
  void* dW; int64_t ldw, sw; int32_t w_bf16;
  void* db; int64_t ldb;
  int32_t k, l;
  int32_t tiles_m, tiles_n;
  int32_t most;          // rows of a chunk
  float* part;           // partial sums of the chunks of groups of more than one: [chunk][k + 1][l], the last row for db
};

int launch_group_rows(const int32_t* keys, int64_t n, int32_t G, int32_t* off, int32_t* order, void* ws, hipStream_t s);
size_t group_rows_ws_bytes(int64_t n, int32_t G);
int launch_check_groups(const lq_groups& g, int32_t* flag, hipStream_t s);
int launch_check_keys(const int32_t* keys, int64_t n, int32_t G, int32_t* flag, hipStream_t s);
// `copy`: rows of X and of the matrices may be read in pieces of 16 or 4 bytes, aligned to that, or only element by element (0).
size_t grouped_product_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t dtype);
int launch_grouped_product(const GroupedArgs& a, int32_t dtype, bool transposed, int copy, void* ws, size_t ws_bytes, hipStream_t s);
// `main`: everything but U, rp, u_rest and group_of, which the call puts into the workspace (256 bytes in).
size_t adapter_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t rank, int32_t dtype);
int launch_adapter_product(const GroupedArgs& main, const lq_stack& A, const float* scale, void* ws, int32_t dtype, int main_copy, int low_copy,
                           hipStream_t s);
size_t grouped_gradient_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t dtype);
int launch_grouped_gradient(const GradientArgs& a, int32_t dtype, int copy, void* ws, size_t ws_bytes, hipStream_t s);

#ifdef __HIPCC__

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));

// Sixteen bytes of zeros: what a lane reads where its operand has ended.
static __device__ const u32x4 g_zeros = {0, 0, 0, 0};

struct __attribute__((packed, aligned(2))) Bytes16 { unsigned int x, y, z, w; };

struct __attribute__((packed, aligned(2))) Bytes8 { unsigned int x, y; };

// The 16 bytes at p, any alignment.
template <typename T> __device__ __forceinline__ u32x4 load_whole(const T* p) {
  const Bytes16 t = *reinterpret_cast<const Bytes16*>(p);
  return u32x4{t.x, t.y, t.z, t.w};
}

// The same where only the first `valid` elements exist (the others read as zero).
template <typename T> __device__ __forceinline__ u32x4 load_piece(const T* p, int valid) {
  constexpr int PER = 16 / sizeof(T);
  if (valid >= PER) return load_whole(p);
  u32x4 r = {0, 0, 0, 0};
#pragma unroll
  for (int q = 0; q < PER; ++q)
    if (q < valid) {
      if constexpr (sizeof(T) == 4) r[q] = reinterpret_cast<const unsigned int*>(p)[q];
      else r[q >> 1] |= static_cast<unsigned int>(p[q]) << (16 * (q & 1));
    }
  return r;
}

// Four neighbouring results at p, of which the first `valid` exist; any alignment.
template <bool BF16> __device__ __forceinline__ void store_four(void* base, int64_t at, int valid, f32x4 v) {
  if constexpr (BF16) {
    bf16_t* p = static_cast<bf16_t*>(base) + at;
    const unsigned int lo = f32x2_to_bf16x2(v[0], v[1]), hi = f32x2_to_bf16x2(v[2], v[3]);
    if (valid >= 4) {
      *reinterpret_cast<Bytes8*>(p) = Bytes8{lo, hi};
      return;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < valid) p[q] = static_cast<bf16_t>((q < 2 ? lo : hi) >> (16 * (q & 1)));
  } else {
    float* p = static_cast<float*>(base) + at;
    if (valid >= 4) {
      *reinterpret_cast<Bytes16*>(p) = Bytes16{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      return;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < valid) p[q] = v[q];
  }
}

// Four neighbouring values at p, likewise.
template <typename T> __device__ __forceinline__ f32x4 load_four(const T* p, int valid) {
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  if (valid >= 4) {
    if constexpr (sizeof(T) == 4) {
      const u32x4 w = load_whole(p);
      r = __builtin_bit_cast(f32x4, w);
    } else {
      const Bytes8 w = *reinterpret_cast<const Bytes8*>(p);
      r = f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < valid) r[q] = Elem<T>::load(p + q);
  }
  return r;
}

// Workgroups go to the 8 dies in turn; each die gets a contiguous run of tiles, so that neighbouring tiles, which
// share rows or a matrix, share an L2.
__device__ __forceinline__ int die_order(int id, int total) {
  const int per = total >> 3, more = total & 7, die = id & 7, at = id >> 3;
  return die * per + min(die, more) + at;
}

struct RowTile { int group, first, rows, col; };
// Tile `local` of positions [begin, end): runs of 8 row tiles, the rows of a run fastest, so that neighbouring tiles share the rows of
// X and the columns of the matrix about evenly.  rows == 0: there is no such tile.
template <int TM> __device__ __forceinline__ RowTile tile_of_range(int group, int begin, int end, int local, int cols) {
  constexpr int RUN = 8;
  const int run = local / (RUN * cols), tiles = (end - begin + TM - 1) / TM;
  const int in_run = min(RUN, tiles - run * RUN), left = local - run * RUN * cols;
  if (in_run <= 0) return {group, begin, 0, 0};
  const int first = begin + (run * RUN + left % in_run) * TM;
  return {group, first, min(TM, end - first), left / in_run};
}
// The tile that workgroup `id` works on: TM rows of one group and one of `cols` column tiles.  Tiles are numbered group by
// group, then those of the rows without a group (group -1), and shared out evenly over the dies.  Called by a whole wavefront:
// lane l adds up the row tiles of groups l * per .. l * per + per - 1, the sums are scanned over the lanes, and the lane that holds
// the tile walks its groups again.
template <int TM> __device__ __forceinline__ RowTile find_tile(const int32_t* __restrict__ off, int G, int n, int id, int cols) {
  const int lane = threadIdx.x & 63;
  const int per = (G + 63) >> 6;
  const int g0 = min(lane * per, G), g1 = min(g0 + per, G);
  int own = 0;
  for (int g = g0; g < g1; ++g) own += (off[g + 1] - off[g] + TM - 1) / TM;
  int upto = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  const int total = __builtin_amdgcn_readlane(upto, 63);
  int group = -1, begin = __builtin_amdgcn_readfirstlane(off[G]), end = n, before = total;   // of the group: its positions, row tiles before it
  const int tiles = (total + (n - begin + TM - 1) / TM) * cols;
  if (id >= tiles) return {-1, 0, 0, 0};
  id = die_order(id, tiles);
  const int t = id / cols;
  if (t < total) {
    const unsigned long long holds = __ballot(upto > t);
    const int at = __ffsll(static_cast<long long>(holds)) - 1;
    if (lane == at) {
      before = upto - own;
      for (int g = g0; g < g1; ++g) {
        const int b = off[g], e = off[g + 1], more = (e - b + TM - 1) / TM;
        if (t < before + more) {
          group = g;
          begin = b;
          end = e;
          break;
        }
        before += more;
      }
    }
    group = __builtin_amdgcn_readlane(group, at);
    begin = __builtin_amdgcn_readlane(begin, at);
    end = __builtin_amdgcn_readlane(end, at);
    before = __builtin_amdgcn_readlane(before, at);
  }
  return tile_of_range<TM>(group, begin, end, id - before * cols, cols);
}
// The same where all positions use one matrix (group 0).
template <int TM> __device__ __forceinline__ RowTile all_rows(int n, int id, int cols) {
  return tile_of_range<TM>(0, 0, n, die_order(id, (n + TM - 1) / TM * cols), cols);
}

// Rows of a group are added up in chunks of about equal sizes, at most `most` rows each.
__host__ __device__ inline int chunks_of(int rows, int most) { return rows > most ? (rows + most - 1) / most : 1; }
__host__ __device__ inline int chunk_rows(int rows, int chunks) { return ((rows + chunks - 1) / chunks + 31) & ~31; }

// Chunk number t: group, rows, and among the chunks of the groups of more than one the place of this chunk's partial sums (-1: the only
// chunk of its group).  A group without rows has one empty chunk.  Up to 64 groups are taken by falling size of
// their chunks, so that the long ones do not start last.  group < 0: there is no such chunk.  Called by a whole wavefront, like find_tile.
struct Chunk { int group, first, rows, place; };
__device__ __forceinline__ Chunk find_chunk(const int32_t* __restrict__ off, int G, int most, int t) {
  const int lane = threadIdx.x & 63;
  const int per = (G + 63) >> 6;
  int g0 = min(lane * per, G), g1 = min(g0 + per, G);
  int own = 0, parts = 0, longest = 0;
  for (int g = g0; g < g1; ++g) {
    const int rows = off[g + 1] - off[g], c = chunks_of(rows, most);
    own += c;
    parts += c > 1 ? c : 0;
    longest = chunk_rows(rows, c);
  }
  int parts_upto = parts;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int w = __shfl_up(parts_upto, d);
    if (lane >= d) parts_upto += w;
  }
  int parts_before = parts_upto - parts;
  if (per == 1) {
    int rank = 0;
    for (int g = 0; g < G; ++g) {
      const int other = __builtin_amdgcn_readlane(longest, g);
      rank += other > longest || (other == longest && g < lane);
    }
    if (lane >= G) rank = lane;
    const int from = __builtin_amdgcn_ds_permute(rank * 4, lane);     // the group of this rank
    own = __shfl(own, from);
    parts_before = __shfl(parts_before, from);
    g0 = from < G ? from : G;
    g1 = from < G ? from + 1 : G;
  }
  int upto = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  const unsigned long long holds = __ballot(upto > t);
  if (!holds) return {-1, 0, 0, -1};
  const int at = __ffsll(static_cast<long long>(holds)) - 1;
  int group = 0, first = 0, rows = 0, place = -1;
  if (lane == at) {
    int before = upto - own;
    for (int g = g0; g < g1; ++g) {
      const int b = off[g], e = off[g + 1], c = chunks_of(e - b, most);
      if (t < before + c) {
        const int step = chunk_rows(e - b, c);
        group = g;
        first = min(b + (t - before) * step, e);
        rows = min(step, e - first);
        place = c > 1 ? parts_before + t - before : -1;
        break;
      }
      before += c;
      parts_before += c > 1 ? c : 0;
    }
  }
  return {__builtin_amdgcn_readlane(group, at), __builtin_amdgcn_readlane(first, at), __builtin_amdgcn_readlane(rows, at),
          __builtin_amdgcn_readlane(place, at)};
}

// One operand of the tile product in LDS: EXT rows of the result (or columns) by KSTEP of the inner dimension, as
// lines of 16-byte pieces.
//   KMAJ    a line per row, the inner dimension along it (KBYTES bytes): a lane's operand is one 16-byte read
//   !KMAJ   a line per inner index, the rows along it: bf16 operands come transposed out of LDS
//           (ds_read_b64_tr_b16: four inner indexes of a row a lane), fp32 ones a word at a time
// Piece c of a line lies at place c ^ spread(line), so that the lanes of a read use all banks.  Measured: no conflicts, but for KMAJ lines of
// 64 bytes (products in tiles of 256 x 256), whose reads take twice as long as without.
// COPY: bytes that a lane brings at a time (16, or 4 where rows are aligned to that only).
template <typename T, bool KMAJ, int EXT, int THREADS, int KBYTES = 128, int COPY = 16> struct Operand {
  static constexpr int EPC = 16 / sizeof(T);
  static constexpr int KSTEP = KBYTES / sizeof(T);
  static constexpr int LINES = KMAJ ? EXT : KSTEP;
  static constexpr int CPL = KMAJ ? KBYTES / 16 : EXT / EPC;
  static constexpr int PIECES = LINES * CPL;
  static constexpr int BYTES = PIECES * 16;
  static constexpr int PER = BYTES / COPY / THREADS;      // copies of a thread
  static constexpr int CPP = 16 / COPY;                   // of a piece
  static_assert(BYTES % (COPY * THREADS) == 0, "whole copies a thread");

  static __device__ __forceinline__ int spread(int line) {
    if constexpr (KMAJ) return CPL == 8 ? (line >> 1) & 7 : (line >> 2) & 3;
    else if constexpr (sizeof(T) == 4) return 4 * ((line >> 2) & 3);
    else if constexpr (CPL >= 16) return 2 * ((line & 3) | ((line >> 1) & 4));
    else return 2 * (((line >> 1) & 1) | ((line >> 2) & 2));
  }
  // The line of the thread's i-th copy, and the element of it that it begins with.
  static __device__ __forceinline__ int id_of(int i) { return i * THREADS + static_cast<int>(threadIdx.x % THREADS); }
  static __device__ __forceinline__ int line_of(int i) { return id_of(i) / (CPL * CPP); }
  static __device__ __forceinline__ int element_of(int i) {
    const int id = id_of(i), at = id % (CPL * CPP);
    return ((at / CPP) ^ spread(id / (CPL * CPP))) * EPC + at % CPP * (COPY / static_cast<int>(sizeof(T)));
  }
  static __device__ __forceinline__ int place(int line, int piece) { return (line * CPL + (piece ^ spread(line))) * 16; }

  // Rows r0 .. r0 + 15 and inner block kk (32 of bf16, 16 of fp32) as a matrix-instruction operand.
  static __device__ __forceinline__ u32x4 fragment(const char* lds, int r0, int kk) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    if constexpr (KMAJ) {
      return *reinterpret_cast<const u32x4*>(lds + place(r0 + i, 4 * kk + g));
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const int k = 32 * kk + 8 * g + (i >> 2), c = (r0 >> 3) + ((i & 3) >> 1);
      const char* p0 = lds + place(k, c) + 8 * (i & 1);
      const char* p1 = lds + place(k + 4, c) + 8 * (i & 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p0);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p1);
      const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
      return u32x4{a.x, a.y, b.x, b.y};
    } else {
      u32x4 r;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = 16 * kk + 4 * g + s, col = r0 + i;
        r[s] = *reinterpret_cast<const unsigned int*>(lds + place(k, col >> 2) + 4 * (col & 3));
      }
      return r;
    }
  }
};

// acc[n][m] += sum over the block of b[n] a[m]: lane l holds row m = l % 16 and four neighbouring columns n = 4 (l / 16) ..
// of the result.  fp32: the block of 16 in four instructions, each with the inner indexes 4 g + s.
template <typename T> __device__ __forceinline__ f32x4 multiply(const u32x4& b, const u32x4& a, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, b), __builtin_bit_cast(bf16x8v, a), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b[s]), __uint_as_float(a[s]), acc, 0, 0, 0);
    return acc;
  }
}

// A tile of TM x TN by WAVES_M x WAVES_N wavefronts; RING: steps that LDS holds.
template <int TM_, int TN_, int WAVES_M_, int WAVES_N_, int RING_ = 2> struct TileShape {
  static constexpr int TM = TM_, TN = TN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, RING = RING_;
  static constexpr int THREADS = 64 * WAVES_M * WAVES_N;
  static constexpr int MI = TM / WAVES_M / 16, NI = TN / WAVES_N / 16;
};

// One step of the product of a wavefront's part of the tile; with_b(b): called with its operands of B, twice.
template <typename T, class S, class A, class B, typename H>
__device__ __forceinline__ void multiply_step(const char* la, const char* lb, f32x4 (&acc)[S::MI][S::NI], H&& with_b) {
  const int wave = threadIdx.x >> 6;
  const int m0 = (wave / S::WAVES_N) * S::MI * 16, n0 = (wave % S::WAVES_N) * S::NI * 16;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    u32x4 a[S::MI], b[S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i) a[i] = A::fragment(la, m0 + 16 * i, kk);
#pragma unroll
    for (int j = 0; j < S::NI; ++j) b[j] = B::fragment(lb, n0 + 16 * j, kk);
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply<T>(b[j], a[i], acc[i][j]);
    with_b(b);
  }
}

// A point that no instruction is moved over.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// COPY (16 or 4) bytes a lane from memory straight into LDS: lane l's land at base + COPY l (`base`: LDS byte address, the same in all
// lanes).  Written as an instruction because the compiler, which sees LDS written by its own form of it, waits for all
// copies before the next transposed read of LDS, also where that reads another buffer.  It has no result in registers;
// the compiler does not count it: meet_after_copies() waits for it.  It writes m0, which nothing else in these kernels
// uses (the compiler takes no m0 in a list of what an instruction overwrites; a test reads the assembly for it).
template <int COPY> __device__ __forceinline__ void copy_to_lds(const void* p, unsigned int base) {
  base = __builtin_amdgcn_readfirstlane(base);
  if constexpr (COPY == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(base), "v"(p));
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(base), "v"(p));
}
__device__ __forceinline__ unsigned int lds_address(const char* p) {
  return static_cast<unsigned int>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}
// All but the N youngest copies of this wavefront and its reads and writes of LDS are done; then the workgroup meets.
template <int N> __device__ __forceinline__ void meet_after_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The product of a tile by four wavefronts over `steps` steps of 128 bytes of the inner dimension, with RING steps in LDS:
// issue(step, LDS address) copies a step's operands there, RING - 1 steps ahead of their product.
template <typename T, class S, class A, class B, int RING, typename F, typename H>
__device__ __forceinline__ void multiply_steps(char* lds, int steps, F&& issue, f32x4 (&acc)[S::MI][S::NI], H&& with_b) {
  constexpr int BUFFER = A::BYTES + B::BYTES, COPIES = A::PER + B::PER;
  const unsigned int at = lds_address(lds);
  int now = 0, then = 0;
  for (int step = 1 - RING; step < steps; ++step) {      // (from the first copies on: issue() is in the code once)
    // this step is in LDS, and the place of the one before is read to its end
    if (step >= 0) {
      if (step + RING - 1 <= steps) meet_after_copies<COPIES*(RING - 2)>();
      else meet_after_copies<0>();
    }
    if (step + RING - 1 < steps) issue(step + RING - 1, at + then * BUFFER);
    then = then + 1 == RING ? 0 : then + 1;
    if (step < 0) continue;
    multiply_step<T, S, A, B>(lds + now * BUFFER, lds + now * BUFFER + A::BYTES, acc, with_b);
    now = now + 1 == RING ? 0 : now + 1;
  }
}

// The product of a tile of 8 wavefronts, two on a SIMD, over `units` units of 64 inner indexes, each two blocks of 32: issue(block,
// LDS address) copies a block's operands to LDS, by four wavefronts.  The two wavefronts of a SIMD take turns: one multiplies a
// unit (64 matrix instructions, 1,024 clocks), reading the operands of the second block while it multiplies the first
// one; the other one meanwhile reads its operands of the first block of its next unit and issues copies, so that the matrix
// cores do not wait for LDS or for the way to it.  The second four wavefronts run one turn behind the first four, by one
// barrier more at the start.  In turns: the first four read unit w in turn 2 w and multiply it in turn 2 w + 1, the second
// four one later.  LDS holds four blocks.  The first blocks of units are copied by the first four, the second blocks by the
// second four: block 2 w + 2 in turn 2 w, when everyone has read block 2 w - 2, and block 2 w + 3 in turn 2 w + 1, when everyone
// has read block 2 w - 1; each is waited for at the end of the next turn, a turn before its first reader.
// (Turns of one block, 512 clocks: 1,296 TFLOP/s at 8,192^3; the copies, 64 bytes a clock for the whole compute unit, in front of
// the reads instead of behind them: 1,198.)
// with_b(b): called with the wavefront's operands of B beside the products.
template <typename T, class S, class A, class B, typename F, typename H>
__device__ __forceinline__ void multiply_in_turns(char* lds, int units, F&& issue, f32x4 (&acc)[S::MI][S::NI], H&& with_b) {
  static_assert(S::THREADS == 512 && S::WAVES_N == 4 && S::MI == 8 && S::NI == 4, "two wavefronts a SIMD");
  constexpr int BLOCK = A::BYTES + B::BYTES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool second = wave >= 4;
  const int m0 = (wave / S::WAVES_N) * S::MI * 16, n0 = (wave % S::WAVES_N) * S::NI * 16;
  const unsigned int at = lds_address(lds);
  auto turn = [&](bool copies) {
    fence();
    if (copies) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    fence();
  };
  issue(second ? 1 : 0, at + (second ? BLOCK : 0));
  turn(true);
  if (second) turn(false);
  for (int w = 0; w < units; ++w) {
    const char* from = lds + (w & 1) * 2 * BLOCK;
    u32x4 a[S::MI], b[2][S::NI];
#pragma unroll
    for (int j = 0; j < S::NI; ++j) b[0][j] = B::fragment(from + A::BYTES, n0 + 16 * j, 0);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) a[i] = A::fragment(from, m0 + 16 * i, 0);
    fence();
    if (w + 1 < units) issue(2 * w + (second ? 3 : 2), at + (((w + 1) & 1) * 2 + (second ? 1 : 0)) * BLOCK);
    turn(false);
    __builtin_amdgcn_s_setprio(1);
    from += BLOCK;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) b[1][j] = B::fragment(from + A::BYTES, n0 + 16 * j, 0);
    with_b(b[0]);
    fence();
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
#pragma unroll
      for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply<T>(b[0][j], a[i], acc[i][j]);
      a[i] = A::fragment(from, m0 + 16 * i, 0);
      fence();     // (the reads stay where they are)
    }
    with_b(b[1]);
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply<T>(b[1][j], a[i], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
    turn(true);
  }
  if (!second) turn(false);
}

// Four by four exchange of registers and groups of 16 lanes: register j of lanes 16 g .. 16 g + 15 and register g of lanes 16 j .. .
// A row's results, four neighbouring columns a lane and 16-column block, become 16 neighbouring columns a lane.
__device__ __forceinline__ void exchange(unsigned int& r0, unsigned int& r1, unsigned int& r2, unsigned int& r3) {
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  u32x2 p = __builtin_amdgcn_permlane32_swap(r0, r2, false, false), q = __builtin_amdgcn_permlane32_swap(r1, r3, false, false);
  u32x2 s = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false), t = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
  r0 = s[0];
  r1 = s[1];
  r2 = t[0];
  r3 = t[1];
}

#endif  // __HIPCC__
}  // namespace lq
#endif  // LQ_GROUPED_H_
