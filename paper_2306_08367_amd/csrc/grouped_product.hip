// Products with the matrix of the row's group, Y[r] = X[r] W_g, and with one shared matrix and a low-rank adapter per
// group, Y[r] = X[r] W + U[r] B_g with U[r] = scale_g X[r] A_g.
//
// A tile of the result takes TM positions of ONE group (positions are sorted by group, so its rows of X and Y are
// gathered and scattered through `order`) and TN columns.  How many tiles there are is known on the device only: the
// grid holds the most there can be (n / TM and one more per group), each workgroup looks its tile up in the offsets,
// and those past the last tile end at once.  The rows without a group get tiles too: zeros.
// Tiles of 256 x 256 (bf16, rows aligned to 16 bytes, where they fill the compute units), 128 x 128 (from one a compute unit on), 64 x 64 (below).
// Rows go to LDS without registers in pieces of 16 or 4 bytes; only bf16 rows of odd lengths pass through registers.
//
// An adapter product is ONE product over all positions with the shared W, whose inner dimension goes on: behind W's k
// come the adapters that occur in the tile, 8 ranks at a time, with U in the rows of that adapter and zeros in the
// others.  U is fp32; beside bf16 matrices it goes in as two bf16 numbers (two_halves), so that what is lost is at most 2^-16 of it and
// not 2^-8.  Few rows take another way (AdapterPlan), with the same infinities and NaNs: those of the formula with U as one number.
//
// What bounds them, measured: 8,192^3 in bf16 1,373 TFLOP/s, transposed 1,341 (the vendor's dense product 1,350 on the same card; on
// another 1,424 and 1,430), the matrix instructions' power and LDS; 32,768 rows in 32 groups, 2,048 -> 4,096, 545 us = 1,010, with parts of tiles at the groups' ends; fp32
// 8,192^3 136 (vendor 154); 128 rows over 64 matrices of 2,048 x 1,024 36 to 40 us, the 268 MB of the matrices;
// one row for two models, 1,024 -> 256, 8.4 us, 16 steps of a workgroup one after the other.
#include "grouped.h"

namespace lq {
namespace {

// Bias, ReLU and gate, and the rows m of the tile for which stored(m).
template <typename T, class S, typename F>
__device__ __forceinline__ void store_tile(const GroupedArgs& a, const RowTile& tile, int n0, int split, const int* yrow, f32x4 (&acc)[S::MI][S::NI], F&& stored) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / S::WAVES_N) * S::MI * 16, wn = n0 + (wave % S::WAVES_N) * S::NI * 16;
  const bool has_bias = a.bias && tile.group >= 0;
  const T* bias = static_cast<const T*>(a.bias) + (has_bias ? tile.group * a.ldb : 0);
  char* const Y = static_cast<char*>(a.Y) + split * a.split_stride * (a.y_bf16 ? 2 : 4);
  if (S::NI == 4 && a.y_vec && wn + 64 <= a.n_store && wn + 64 <= a.N) {
    // 16 neighbouring columns of a row a lane
    const int n = wn + 16 * (lane >> 4);
    f32x4 bv[4] = {};
    if (has_bias)
#pragma unroll
      for (int q = 0; q < 4; ++q) bv[q] = load_four(bias + n + 4 * q, 4);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      unsigned int v[4][4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j][q] = __float_as_uint(acc[i][j < S::NI ? j : 0][q]);
        exchange(v[0][q], v[1][q], v[2][q], v[3][q]);
      }
      const int m = wm + 16 * i + (lane & 15);
      if (m >= tile.rows || !stored(m)) continue;
      const int64_t r = yrow[m];
      f32x4 y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float x = __uint_as_float(v[j][q]) + bv[j][q];
          y[j][q] = a.relu && x < 0.f ? 0.f : x;
        }
        if (a.gate) {
          const f32x4 h = load_four(static_cast<const T*>(a.gate) + r * a.ldg + n + 4 * j, 4);
#pragma unroll
          for (int q = 0; q < 4; ++q) y[j][q] = h[q] > 0.f ? y[j][q] : 0.f;
        }
      }
      if (a.y_bf16) {
        uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(Y) + r * a.ldy + n);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          to[h] = uint4{f32x2_to_bf16x2(y[2 * h][0], y[2 * h][1]), f32x2_to_bf16x2(y[2 * h][2], y[2 * h][3]),
                        f32x2_to_bf16x2(y[2 * h + 1][0], y[2 * h + 1][1]), f32x2_to_bf16x2(y[2 * h + 1][2], y[2 * h + 1][3])};
      } else {
        f32x4* to = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(Y) + r * a.ldy + n);
#pragma unroll
        for (int h = 0; h < 4; ++h) to[h] = y[h];
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < S::NI; ++j) {
    const int n = wn + 16 * j + 4 * (lane >> 4), valid = a.n_store - n;
    if (valid <= 0) continue;
    f32x4 bv = {0.f, 0.f, 0.f, 0.f};
    if (has_bias) bv = load_four(bias + n, a.N - n);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int m = wm + 16 * i + (lane & 15);
      if (m >= tile.rows || !stored(m)) continue;
      const int64_t r = yrow[m];
      f32x4 v = acc[i][j] + bv;
      if (a.relu)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = v[q] < 0.f ? 0.f : v[q];
      if (a.gate) {
        const f32x4 h = load_four(static_cast<const T*>(a.gate) + r * a.ldg + n, valid);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = h[q] > 0.f ? v[q] : 0.f;
      }
      if (a.y_bf16) store_four<true>(Y, r * a.ldy + n, valid, v);
      else store_four<false>(Y, r * a.ldy + n, valid, v);
    }
  }
}

// Workgroup `block` of the product's grid, split `split` of its inner dimension.
template <typename T, class S, bool BT, int COPY, bool ADAPT>
__device__ __forceinline__ void tile_product(const GroupedArgs& a, int block, int split) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128, COPIERS = 256;     // threads that copy a step
  typedef Operand<T, true, S::TM, COPIERS, KBYTES, COPY ? COPY : 16> A;
  typedef Operand<T, BT, S::TN, COPIERS, KBYTES, COPY ? COPY : 16> B;
  constexpr bool DIRECT = COPY != 0;           // through LDS without registers
  constexpr int KSTEP = A::KSTEP, EPC = A::EPC, THREADS = S::THREADS;
  constexpr int E = DIRECT ? COPY / static_cast<int>(sizeof(T)) : 1;
  extern __shared__ __align__(1024) char lds[];
  __shared__ int xrow[S::TM], yrow[S::TM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  RowTile tile;
  if (ADAPT || !a.off) tile = all_rows<S::TM>(a.n, block, a.tiles_n);
  else tile = find_tile<S::TM>(a.off, a.G, a.n, block, a.tiles_n);
  const int n0 = tile.col * S::TN;
  if (tile.rows <= 0) return;

  for (int m = tid; m < S::TM; m += THREADS) {
    const bool in = m < tile.rows;
    const int p = tile.first + (in ? m : tile.rows - 1);     // (behind the last row: that row again, not stored)
    const int r = a.order ? a.order[p] : p;
    xrow[m] = a.x_grouped ? p : r / a.slots;
    yrow[m] = a.y_grouped ? p : r;
    if (!ADAPT && a.gpos && in && n0 == 0 && split == 0) a.gpos[p] = tile.group;
  }
  __syncthreads();

  // The adapters of the tile: positions are sorted by group, so a row starts one where its group differs from the one
  // before it.  which[m]: the row's adapter, counted from the tile's first one, -1 for none.
  __shared__ int which[ADAPT ? S::TM : 1], gid[ADAPT ? S::TM : 1], firsts[S::TM / 64];
  int adapters = 0;
  if constexpr (ADAPT) {
    bool starts = false;
    int g = -1, upto = 0;
    if (tid < S::TM) {
      const int p = tile.first + tid;
      g = tid < tile.rows ? a.group_of[p] : -1;
      starts = g >= 0 && (tid == 0 || a.group_of[p - 1] != g);
      const unsigned long long mask = __ballot(starts);
      upto = __popcll(mask & (~0ull >> (63 - lane)));
      if (lane == 0) firsts[tid >> 6] = __popcll(mask);
    }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < S::TM / 64; ++w) {
      before += w < wave ? firsts[w] : 0;
      adapters += firsts[w];
    }
    adapters = __builtin_amdgcn_readfirstlane(adapters);
    if (tid < S::TM) {
      which[tid] = g >= 0 ? before + upto - 1 : -1;
      if (starts) gid[before + upto - 1] = g;
    }
    __syncthreads();
  }

  const int k_first = split * a.steps_per_split * KSTEP;
  const int k_end = min(a.K, k_first + a.steps_per_split * KSTEP);
  const bool any = tile.group >= 0 && k_first < k_end;
  const T* X = static_cast<const T*>(a.X);
  const T* W = static_cast<const T*>(a.W) + (any ? tile.group * a.sw : 0);
  // Where this thread's pieces of either operand lie at inner index 0, and their first inner index.  Columns behind the
  // last one hold something else of the matrix or zeros; they are not stored.
  const T *pa[A::PER], *pb[B::PER];
  int va[A::PER], vb[B::PER];
#pragma unroll
  for (int i = 0; i < A::PER; ++i) {
    va[i] = A::element_of(i);
    pa[i] = X + xrow[A::line_of(i)] * a.ldx + va[i];
  }
#pragma unroll
  for (int i = 0; i < B::PER; ++i) {
    const int line = B::line_of(i), e = B::element_of(i);
    vb[i] = BT ? e : line;
    pb[i] = BT ? W + static_cast<int64_t>(min(n0 + line, a.N - 1)) * a.ldw + e : W + line * a.ldw + min(n0 + e, a.N - E);
  }
  const int64_t step_b = BT ? 1 : a.ldw;     // elements per inner index
  constexpr int BUFFER = A::BYTES + B::BYTES, SLOTS = KSTEP / EPC;
  const int own_steps = __builtin_amdgcn_readfirstlane(any ? (k_end - k_first + KSTEP - 1) / KSTEP : 0);
  // The adapters' steps: pieces of EPC inner indexes, two for every 8 ranks of every adapter: bf16: U's leading part and the
  // rest of it, times the same ranks of B; fp32: the two halves of the 8.
  const int per = ADAPT ? a.rp >> 3 : 1;
  const int steps = own_steps + (ADAPT ? (2 * adapters * per + SLOTS - 1) / SLOTS : 0);
  int only = -1;      // >= 0: of this adapter's pieces alone
  auto piece_of_u = [&](int step, int i) -> const void* {
    const int line = A::line_of(i), e = A::element_of(i);
    const int qq = (step - own_steps) * SLOTS + e / EPC, q = qq >> 1, ad = q / per;
    if (which[line] != ad || (only >= 0 && only != ad)) return &g_zeros;
    const int64_t at = static_cast<int64_t>(tile.first + line) * a.rp + (q - ad * per) * 8 + e % EPC;
    if constexpr (sizeof(T) == 2) return static_cast<const bf16_t*>(a.U) + ((qq & 1) ? a.u_rest : 0) + at;
    else return static_cast<const float*>(a.U) + at + 4 * (qq & 1);
  };
  // (the row of B that is line i of the step; NULL: zeros)
  auto row_of_b = [&](int step, int i) -> const T* {
    const int line = B::line_of(i), qq = (step - own_steps) * SLOTS + line / EPC, q = qq >> 1, ad = q / per;
    const int rank = (q - ad * per) * 8 + (sizeof(T) == 2 ? 0 : 4 * (qq & 1)) + line % EPC;
    if (ad >= adapters || rank >= a.rank || (only >= 0 && only != ad)) return nullptr;
    return static_cast<const T*>(a.B) + gid[ad] * a.sB + rank * a.ldB;
  };

  auto issue = [&](int step, unsigned int to) {
    const int k0 = k_first + step * KSTEP;
    to += (wave & 3) * 64 * COPY;
    if (ADAPT && step >= own_steps) {
      // (few steps with long addresses: not unrolled where there are many copies)
#pragma unroll COPY == 16 ? 4 : 1
      for (int i = 0; i < A::PER; ++i) copy_to_lds<COPY>(piece_of_u(step, i), to + i * COPIERS * COPY);
#pragma unroll COPY == 16 ? 4 : 1
      for (int i = 0; i < B::PER; ++i) {
        const T* row = row_of_b(step, i);
        copy_to_lds<COPY>(row ? static_cast<const void*>(row + min(n0 + B::element_of(i), a.N - E)) : &g_zeros, to + A::BYTES + i * COPIERS * COPY);
      }
    } else if (k0 + KSTEP <= k_end) {
#pragma unroll
      for (int i = 0; i < A::PER; ++i) copy_to_lds<COPY>(pa[i] + k0, to + i * COPIERS * COPY);
#pragma unroll
      for (int i = 0; i < B::PER; ++i) copy_to_lds<COPY>(pb[i] + k0 * step_b, to + A::BYTES + i * COPIERS * COPY);
    } else {
#pragma unroll
      for (int i = 0; i < A::PER; ++i)
        copy_to_lds<COPY>(k0 + va[i] < k_end ? static_cast<const void*>(pa[i] + k0) : &g_zeros, to + i * COPIERS * COPY);
#pragma unroll
      for (int i = 0; i < B::PER; ++i)
        copy_to_lds<COPY>(k0 + vb[i] < k_end ? static_cast<const void*>(pb[i] + k0 * step_b) : &g_zeros, to + A::BYTES + i * COPIERS * COPY);
    }
  };
  // Up to here all 16 bytes of a piece may be read: a row of X ends behind it; a row of W may end inside it, but another follows.
  const int whole_end = BT ? k_end : a.ldw >= EPC ? min(k_end, a.K - 1) : 0;
  auto whole = [&](int step) { return step < own_steps && k_first + (step + 1) * KSTEP <= whole_end; };
  u32x4 ra[DIRECT ? 1 : A::PER], rb[DIRECT ? 1 : B::PER];
  auto fetch = [&](int step) {
    const int k0 = k_first + step * KSTEP;
#pragma unroll
    for (int i = 0; i < A::PER; ++i) ra[i] = load_whole(pa[i] + k0);
#pragma unroll
    for (int i = 0; i < B::PER; ++i) rb[i] = load_whole(pb[i] + k0 * step_b);
  };
  auto put = [&](char* to) {
#pragma unroll
    for (int i = 0; i < A::PER; ++i) *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = ra[i];
#pragma unroll
    for (int i = 0; i < B::PER; ++i) *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = rb[i];
  };
  // A step that is not whole, from memory to LDS at once (its loads beside the products of the step before would meet those of
  // the other kind in the same registers, and the compiler would wait for both there).
  auto fill = [&](int step, char* to) {
    const int k0 = k_first + step * KSTEP;
    const bool of_adapters = ADAPT && step >= own_steps;
#pragma unroll
    for (int i = 0; i < A::PER; ++i) {
      u32x4 v;
      if (of_adapters) v = *static_cast<const u32x4*>(piece_of_u(step, i));
      else v = load_piece(pa[i] + k0, k_end - (k0 + va[i]));
      *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = v;
    }
#pragma unroll
    for (int i = 0; i < B::PER; ++i) {
      const int n = n0 + B::element_of(i);
      u32x4 v;
      if (of_adapters) {
        const T* row = row_of_b(step, i);
        v = load_piece(row + n, row ? a.N - n : 0);
      } else {
        v = load_piece(pb[i] + k0 * step_b, BT ? k_end - (k0 + vb[i]) : k0 + vb[i] < k_end ? a.N - n : 0);
      }
      *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = v;
    }
  };

  const auto nothing = [](const u32x4(&)[S::NI]) {};
  for (;;) {
    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (steps > 0) {
      if constexpr (DIRECT && THREADS == 512) {
        multiply_in_turns<T, S, A, B>(lds, (steps + 1) >> 1, issue, acc, nothing);     // (a block behind the last one is zeros)
      } else if constexpr (DIRECT) {
        multiply_steps<T, S, A, B, S::RING>(lds, steps, issue, acc, nothing);
      } else {
        fill(0, lds);
        for (int step = 0; step < steps; ++step) {
          const int at = (step & 1) * BUFFER;
          __syncthreads();         // this buffer is whole, the other one is read to its end
          const bool more = step + 1 < steps, ahead = more && whole(step + 1);
          if (ahead) fetch(step + 1);
          fence();                 // (the loads go ahead of the products)
          multiply_step<T, S, A, B>(lds + at, lds + at + A::BYTES, acc, nothing);
          if (ahead) put(lds + (at ^ BUFFER));
          else if (more) fill(step + 1, lds + (at ^ BUFFER));
        }
      }
    }
    if constexpr (!ADAPT) {
      store_tile<T, S>(a, tile, n0, split, yrow, acc, [](int) { return true; });
      return;
    } else {
      // An infinity or a NaN in one adapter's B, times the zeros in the rows of others, is a NaN there.  A tile with a NaN
      // is therefore computed again for one adapter at a time (the last time for the rows without one) and stored for its
      // rows only: the same sums, with zeros for the other adapters' terms.
      if (only < 0) {
        bool nan = false;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
          for (int j = 0; j < S::NI; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) nan |= acc[i][j][q] != acc[i][j][q];
        if (!__syncthreads_or(nan)) {
          store_tile<T, S>(a, tile, n0, split, yrow, acc, [](int) { return true; });
          return;
        }
      } else {
        store_tile<T, S>(a, tile, n0, split, yrow, acc, [&](int m) { return which[m] == (only < adapters ? only : -1); });
        __syncthreads();           // (LDS is read to its end)
      }
      if (++only > adapters) return;
    }
  }
}

template <typename T, class S, bool BT, int COPY, bool ADAPT>
__global__ __launch_bounds__(S::THREADS, 2) void grouped_product_kernel(GroupedArgs a) {
  tile_product<T, S, BT, COPY, ADAPT>(a, blockIdx.x, blockIdx.y);
}

// Two products in one launch: the first `blocks_a` workgroups work on a, `splits` after `splits`, the others on b.
template <typename T, class S, int COPY>
__global__ __launch_bounds__(S::THREADS, 2) void grouped_pair_kernel(GroupedArgs a, GroupedArgs b, int blocks_a) {
  const bool first = static_cast<int>(blockIdx.x) < blocks_a;
  const GroupedArgs& g = first ? a : b;
  const int at = blockIdx.x - (first ? 0 : blocks_a), tiles = g.tiles_n * g.row_tiles;
  tile_product<T, S, false, COPY, false>(g, at % tiles, at / tiles);
}

// `one`: all positions use one matrix (else there can be a part of a tile more for every group).
void set_tiles(GroupedArgs& a, int tm, int tn, int step, bool one, int splits) {
  a.tiles_n = (a.n_store + tn - 1) / tn;
  a.row_tiles = one ? (a.n + tm - 1) / tm : a.n / tm + std::min(a.n, a.G + 1);
  a.steps_per_split = ((a.K + step - 1) / step + splits - 1) / splits;
}

template <typename T, class S, bool BT, int COPY, bool ADAPT> int launch(GroupedArgs a, int splits, hipStream_t s) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128, COPIERS = 256;     // threads that copy a step
  typedef Operand<T, true, S::TM, COPIERS, KBYTES, COPY ? COPY : 16> A;
  typedef Operand<T, BT, S::TN, COPIERS, KBYTES, COPY ? COPY : 16> B;
  constexpr int LDS = (COPY ? S::RING : 2) * (A::BYTES + B::BYTES);
  set_tiles(a, S::TM, S::TN, A::KSTEP, ADAPT, splits);
  const int64_t blocks = static_cast<int64_t>(a.tiles_n) * a.row_tiles;
  if (blocks * S::THREADS > MOST_THREADS) return fail(LQ_ERR_UNSUPPORTED, "grouped product: %lld tiles are more than one launch takes", (long long)blocks);
  const auto kernel = grouped_product_kernel<T, S, BT, COPY, ADAPT>;
  if (LDS >= 64 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  kernel<<<dim3(static_cast<unsigned>(blocks), splits), S::THREADS, LDS, s>>>(a);
  LQ_LAUNCH_CHECK("grouped_product_kernel");
  return LQ_OK;
}

typedef TileShape<128, 128, 2, 2> Tile128;
typedef TileShape<64, 64, 2, 2> Tile64;
typedef TileShape<64, 64, 2, 2, 4> Tile64Ahead;
typedef TileShape<256, 256, 2, 4, 4> Tile256;

template <typename T, bool BT, int COPY, bool ADAPT> int by_size(const GroupedArgs& a, int splits, hipStream_t s) {
  const int64_t large = static_cast<int64_t>((a.n_store + 127) / 128) * ((a.n + 127) / 128);
  if constexpr (sizeof(T) == 2 && COPY == 16) {
    // One tile of 256 x 256 a compute unit at a time: where the last round of them would leave more than three in ten empty, smaller
    // ones (16,384 rows in 16 groups, 2,048 -> 1,024, 288 tiles: 133 us, in tiles of 128 119).
    const int64_t cus = num_cus(), half_a_tile = ADAPT ? 0 : std::min(a.n, a.G) / 2;
    const int64_t largest = static_cast<int64_t>((a.n_store + 255) / 256) * ((a.n + 255) / 256 + half_a_tile);
    if (largest >= cus && 10 * largest >= 7 * cus * ((largest + cus - 1) / cus)) return launch<T, Tile256, BT, COPY, ADAPT>(a, splits, s);
  }
  // (adapters in copies of 4 bytes: the addresses of the larger tile's copies do not fit in the registers beside the rest)
  if constexpr (!(ADAPT && COPY == 4))
    if (large >= num_cus()) return launch<T, Tile128, BT, COPY, ADAPT>(a, splits, s);
  // Few tiles: three steps ahead in each instead of several workgroups a compute unit (64 rows, 4,096 -> 4,096 with adapters: 59 -> 44 us;
  // 1,024 tiles of 64 experts' matrices, 2,048 -> 1,024: 45 us three steps ahead, 38 one).
  const int64_t small = static_cast<int64_t>((a.n_store + 63) / 64) * ((a.n + 63) / 64 + (ADAPT ? 0 : std::min(a.n, a.G) / 2)) * splits;
  if constexpr (COPY != 0)
    if (small <= 2 * num_cus()) return launch<T, Tile64Ahead, BT, COPY, ADAPT>(a, splits, s);
  return launch<T, Tile64, BT, COPY, ADAPT>(a, splits, s);
}

template <typename T, bool BT, bool ADAPT> int by_copy(const GroupedArgs& a, int copy, int splits, hipStream_t s) {
  if (copy == 16) return by_size<T, BT, 16, ADAPT>(a, splits, s);
  if constexpr (sizeof(T) == 2)
    if (copy == 0) return by_size<T, BT, 0, ADAPT>(a, splits, s);
  return by_size<T, BT, 4, ADAPT>(a, splits, s);
}

template <typename T> int product(const GroupedArgs& a, bool transposed, int copy, int splits, hipStream_t s) {
  return transposed ? by_copy<T, true, false>(a, copy, splits, s) : by_copy<T, false, false>(a, copy, splits, s);
}

// A number as two of bf16, `hi` its leading bits and `lo` the rest to eight bits, both of its sign and neither zero unless the number is:
// both meet the same row of B, and an infinity there times both is one infinity (hi rounded to nearest leaves a rest of the other
// sign or none, a NaN; it would lose half as much, 2^-17).  So hi is cut off, and where that leaves nothing it is the next number
// towards zero.  A number above the largest of bf16 stays finite, an infinity or a NaN is both.  (Of numbers below 2^-103
// the rest can be too small for bf16: an infinity times them is a NaN.)
__device__ __forceinline__ void two_halves(float u, float* hi, float* lo) {
  const unsigned int bits = __float_as_uint(u);
  const bool finite = __builtin_isfinite(u);
  const unsigned int back = (bits & 0xffffu) == 0 && u != 0.f ? 0x10000u : 0u;
  *hi = finite ? __uint_as_float((bits & 0xffff0000u) - back) : u;
  *lo = finite ? u - *hi : u;
}

// U from the partial sums of its product: scaled, zeros behind the last rank, as two bf16 numbers beside bf16 matrices.  Eight
// ranks of a position a thread.
template <bool HALVES>
__global__ __launch_bounds__(256) void adapter_scale_kernel(const float* __restrict__ part, int splits, int64_t stride, int64_t pieces, int per,
                                                            int rank, const float* __restrict__ scale, const int32_t* __restrict__ group_of,
                                                            void* __restrict__ out, int64_t rest) {
  const int64_t id = blockIdx.x * 256ll + threadIdx.x;
  if (id >= pieces) return;
  const int r0 = static_cast<int>(id % per) * 8, g = group_of[id / per];
  f32x4 u[2] = {};
  for (int z = 0; z < splits; ++z)
#pragma unroll
    for (int h = 0; h < 2; ++h) u[h] += *reinterpret_cast<const f32x4*>(part + z * stride + id * 8 + 4 * h);
  const float s = scale && g >= 0 ? scale[g] : 1.f;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) u[h][e] = g >= 0 && r0 + 4 * h + e < rank ? u[h][e] * s : 0.f;
  if constexpr (HALVES) {
    u32x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float h[2], l[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) two_halves(u[e >> 1][2 * (e & 1) + q], &h[q], &l[q]);
      hi[e] = f32x2_to_bf16x2(h[0], h[1]);
      lo[e] = f32x2_to_bf16x2(l[0], l[1]);
    }
    *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(out) + id * 8) = hi;
    *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(out) + rest + id * 8) = lo;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(static_cast<float*>(out) + id * 8 + 4 * h) = u[h];
  }
}

// Few rows: partial sums of X W [splits x n x l] and of U, added up here, with U B in fp32: one row and 1,024 columns a
// workgroup.
template <typename T>
__global__ __launch_bounds__(256) void adapter_finish_kernel(GroupedArgs a, const float* __restrict__ sums, int splits, const float* __restrict__ part,
                                                             int u_splits, const float* __restrict__ scale) {
  __shared__ float u[LQ_MAX_RANK];
  constexpr int AHEAD = 8;
  const int p = blockIdx.x, g = a.group_of[p], r = a.order ? a.order[p] : p;
  const int n = blockIdx.y * 1024 + 4 * threadIdx.x, valid = a.N - n, at = min(n, a.N - 1), there = min(max(valid, 1), 4);
  // the first partial sums and rows of B are under way while U is added up
  const float* sum = sums + static_cast<int64_t>(p) * a.n_store + at;
  const int64_t stride = static_cast<int64_t>(a.n) * a.n_store;
  const T* B = static_cast<const T*>(a.B) + max(g, 0) * a.sB + at;
  f32x4 part_y[AHEAD], row[AHEAD];
#pragma unroll
  for (int z = 0; z < AHEAD; ++z) part_y[z] = load_four(sum + min(z, splits - 1) * stride, there);
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) row[k] = load_four(B + min(k, a.rank - 1) * a.ldB, there);
  if (g >= 0 && static_cast<int>(threadIdx.x) < a.rank) {
    const float* of = part + static_cast<int64_t>(p) * a.rp + threadIdx.x;
    const int64_t step = static_cast<int64_t>(a.n) * a.rp;
    float v = 0.f;
#pragma unroll 8
    for (int z = 0; z < u_splits; ++z) v += of[z * step];
    u[threadIdx.x] = scale ? v * scale[g] : v;
  }
  __syncthreads();
  if (valid <= 0) return;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int z = 0; z < AHEAD; ++z)
    if (z < splits) y += part_y[z];
  for (int z = AHEAD; z < splits; ++z) y += load_four(sum + z * stride, valid);
  if (g >= 0) {
    f32x4 low = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (k < a.rank) low += u[k] * row[k];
#pragma unroll 8
    for (int k = AHEAD; k < a.rank; ++k) low += u[k] * load_four(B + k * a.ldB, valid);
    y += low;
  }
  if (a.bias) y += load_four(static_cast<const T*>(a.bias) + n, valid);
  if (a.y_bf16) store_four<true>(a.Y, static_cast<int64_t>(r) * a.ldy + n, valid, y);
  else store_four<false>(a.Y, static_cast<int64_t>(r) * a.ldy + n, valid, y);
}

// Adds up the partial sums of a product in splits: one position and 1,024 columns a workgroup.
template <typename T> __global__ __launch_bounds__(256) void grouped_finish_kernel(GroupedArgs a, const float* __restrict__ sums, int splits) {
  constexpr int AHEAD = 8;
  const int p = blockIdx.x, n = blockIdx.y * 1024 + 4 * threadIdx.x, valid = a.N - n;
  if (valid <= 0) return;
  const float* sum = sums + static_cast<int64_t>(p) * a.N + n;
  const int64_t stride = static_cast<int64_t>(a.n) * a.N;
  f32x4 part[AHEAD], y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int z = 0; z < AHEAD; ++z) part[z] = load_four(sum + min(z, splits - 1) * stride, valid);
  const int g = a.group_of[p];
  const int64_t r = a.y_grouped || !a.order ? p : a.order[p];
#pragma unroll
  for (int z = 0; z < AHEAD; ++z)
    if (z < splits) y += part[z];
  for (int z = AHEAD; z < splits; ++z) y += load_four(sum + z * stride, valid);
  if (a.bias && g >= 0) y += load_four(static_cast<const T*>(a.bias) + g * a.ldb + n, valid);
  if (a.relu)
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = y[q] < 0.f ? 0.f : y[q];
  if (a.gate) {
    const f32x4 h = load_four(static_cast<const T*>(a.gate) + r * a.ldg + n, valid);
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = h[q] > 0.f ? y[q] : 0.f;
  }
  if (a.y_bf16) store_four<true>(a.Y, r * a.ldy + n, valid, y);
  else store_four<false>(a.Y, r * a.ldy + n, valid, y);
}

// Splits of the inner dimension of a grouped product: where its tiles of 64 x 64 fill less than half of the compute units and have many
// steps, so that the second launch is worth it (320 rows in 10 groups, 3,509 -> 53 in bf16: 45 us in one split).  At least four steps each.
int product_splits(int64_t n, int32_t G, int32_t K, int32_t N, int32_t dtype) {
  const int64_t tiles = (n / 64 + std::min<int64_t>(n, G + 1)) * ((N + 63) / 64), steps = (K * static_cast<int64_t>(dtype_size(dtype)) + 127) / 128;
  if (n == 0 || tiles > 128 || steps < 32) return 1;
  return static_cast<int>(std::min<int64_t>({512 / tiles, steps / 4, 16}));
}
// (the group of every position, then the partial sums)
size_t split_bytes(int64_t n, int32_t N, int splits) {
  return splits < 2 ? 0 : round_up(static_cast<size_t>(n) * 4, 256) + round_up(static_cast<size_t>(splits) * n * N * 4, 256);
}

// How an adapter product runs, and what lies where in its workspace behind the first 256 bytes (kept for LQ_CHECK_FKS).  (For 256 compute units
// whatever the device, so that the workspace's size is the same on all.)
//   few rows    the products of X with W and with A in one launch of tiles of 64 x 64, both in splits of the inner dimension so that
//               there are two tiles a compute unit, then adapter_finish_kernel: where W alone has at most one tile a compute unit and
//               the rows' own reads of B (every row reads its adapter) stay small against the caches.  64 rows of 4,096 -> 4,096 with 48
//               adapters: 44 us in tiles
//   else        U first, then one product (tile_product, ADAPT)
struct AdapterPlan {
  bool few;
  int rp, splits, u_splits;
  size_t part, u, group_of, sums, bytes;
};
AdapterPlan adapter_plan(int64_t n, int32_t G, int32_t k, int32_t l, int32_t rank, int32_t dtype) {
  AdapterPlan p{};
  const int64_t size = static_cast<int64_t>(dtype_size(dtype)), steps = (k * size + 127) / 128, cus = 256;
  p.rp = (rank + 7) / 8 * 8;
  auto splits = [&](int64_t rows, int64_t columns, int64_t least) {      // two tiles a compute unit, `least` steps each
    const int64_t tiles = std::max<int64_t>(rows * ((columns + 63) / 64), 1);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({2 * cus / tiles, steps / least, 16})));
  };
  p.few = (n + 63) / 64 * ((l + 63) / 64) <= cus && n * rank * l * size <= (32ll << 20);
  p.u_splits = splits(n / 64 + (p.few ? std::min<int64_t>(n, G) : 1), p.rp, p.few ? 8 : 4);
  p.splits = p.few ? splits((n + 63) / 64, l, 4) : 1;
  p.part = 256;
  p.u = p.part + round_up(static_cast<size_t>(p.u_splits) * n * p.rp * 4, 256);
  p.group_of = p.u + (p.few ? 0 : round_up(static_cast<size_t>(n) * p.rp * 4, 256));
  p.sums = p.group_of + round_up(static_cast<size_t>(n) * 4, 256);
  p.bytes = p.sums + (p.few ? round_up(static_cast<size_t>(p.splits) * n * l * 4, 256) : 0);
  return p;
}

template <typename T, int COPY> int launch_pair(GroupedArgs a, GroupedArgs b, int splits_a, int splits_b, hipStream_t s) {
  typedef TileShape<64, 64, 2, 2, 3> S;
  typedef Operand<T, true, S::TM, S::THREADS, 128, COPY ? COPY : 16> A;
  constexpr int LDS = (COPY ? S::RING : 2) * 2 * A::BYTES;
  set_tiles(a, S::TM, S::TN, A::KSTEP, true, splits_a);
  set_tiles(b, S::TM, S::TN, A::KSTEP, false, splits_b);
  const int blocks_a = a.tiles_n * a.row_tiles * splits_a, blocks_b = b.tiles_n * b.row_tiles * splits_b;
  const auto kernel = grouped_pair_kernel<T, S, COPY>;
  if (LDS >= 64 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  kernel<<<blocks_a + blocks_b, S::THREADS, LDS, s>>>(a, b, blocks_a);
  LQ_LAUNCH_CHECK("grouped_pair_kernel");
  return LQ_OK;
}

template <typename T> int few_rows(const GroupedArgs& m, GroupedArgs low, const AdapterPlan& p, const float* scale, char* ws, int copy, hipStream_t s) {
  GroupedArgs a = m;
  a.off = nullptr;
  a.bias = nullptr;
  a.Y = ws + p.sums;
  a.ldy = a.n_store;
  a.split_stride = static_cast<int64_t>(a.n) * a.n_store;
  a.y_grouped = 1;
  a.y_bf16 = 0;
  a.y_vec = a.n_store % 4 == 0;
  int rc;
  if (copy == 16) rc = launch_pair<T, 16>(a, low, p.splits, p.u_splits, s);
  else if (sizeof(T) == 4 || copy == 4) rc = launch_pair<T, 4>(a, low, p.splits, p.u_splits, s);
  else rc = launch_pair<T, sizeof(T) == 4 ? 4 : 0>(a, low, p.splits, p.u_splits, s);
  if (rc) return rc;
  adapter_finish_kernel<T><<<dim3(m.n, (m.N + 1023) / 1024), 256, 0, s>>>(m, static_cast<const float*>(a.Y), p.splits, static_cast<const float*>(low.Y),
                                                                          p.u_splits, scale);
  LQ_LAUNCH_CHECK("adapter_finish_kernel");
  return LQ_OK;
}

}  // namespace

size_t grouped_product_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t dtype) {
  return std::max(split_bytes(n, l, product_splits(n, G, k, l, dtype)), split_bytes(n, k, product_splits(n, G, l, k, dtype)));
}

int launch_grouped_product(const GroupedArgs& args, int32_t dtype, bool transposed, int copy, void* ws, size_t ws_bytes, hipStream_t s) {
  GroupedArgs a = args;
  const int splits = product_splits(a.n, a.G, a.K, a.N, dtype);
  if (splits < 2 || !ws || ws_bytes < split_bytes(a.n, a.N, splits))
    return dtype == LQ_BF16 ? product<bf16_t>(a, transposed, copy, 1, s) : product<float>(a, transposed, copy, 1, s);
  a.gpos = static_cast<int32_t*>(ws);
  a.Y = static_cast<char*>(ws) + round_up(static_cast<size_t>(a.n) * 4, 256);
  a.ldy = a.N;
  a.split_stride = static_cast<int64_t>(a.n) * a.N;
  a.y_grouped = 1;
  a.y_bf16 = 0;
  a.y_vec = a.N % 4 == 0;
  a.bias = a.gate = nullptr;
  a.relu = 0;
  const int rc = dtype == LQ_BF16 ? product<bf16_t>(a, transposed, copy, splits, s) : product<float>(a, transposed, copy, splits, s);
  if (rc) return rc;
  GroupedArgs f = args;
  f.group_of = a.gpos;
  const dim3 grid(f.n, (f.N + 1023) / 1024);
  if (dtype == LQ_BF16) grouped_finish_kernel<bf16_t><<<grid, 256, 0, s>>>(f, static_cast<const float*>(a.Y), splits);
  else grouped_finish_kernel<float><<<grid, 256, 0, s>>>(f, static_cast<const float*>(a.Y), splits);
  LQ_LAUNCH_CHECK("grouped_finish_kernel");
  return LQ_OK;
}

size_t adapter_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t rank, int32_t dtype) { return adapter_plan(n, G, k, l, rank, dtype).bytes; }

int launch_adapter_product(const GroupedArgs& args, const lq_stack& A, const float* scale, void* ws, int32_t dtype, int main_copy, int low_copy,
                           hipStream_t s) {
  GroupedArgs m = args;
  const AdapterPlan p = adapter_plan(m.n, m.G, m.K, m.N, m.rank, dtype);
  char* const base = static_cast<char*>(ws);
  m.rp = p.rp;
  m.u_rest = static_cast<int64_t>(m.n) * p.rp;
  m.U = base + p.u;
  m.group_of = reinterpret_cast<const int32_t*>(base + p.group_of);
  GroupedArgs low{};
  low.off = m.off; low.order = m.order; low.G = m.G; low.n = m.n;
  low.X = m.X; low.ldx = m.ldx; low.K = m.K; low.slots = 1;
  low.W = A.data; low.ldw = A.ld; low.sw = A.stride;
  low.Y = base + p.part; low.ldy = p.rp; low.N = m.rank; low.n_store = p.rp; low.y_grouped = 1; low.y_vec = 1;
  low.split_stride = static_cast<int64_t>(m.n) * p.rp;
  low.gpos = reinterpret_cast<int32_t*>(base + p.group_of);
  const bool halves = dtype == LQ_BF16;
  if (p.few) {
    const int copy = std::min(main_copy, low_copy);
    return halves ? few_rows<bf16_t>(m, low, p, scale, base, copy, s) : few_rows<float>(m, low, p, scale, base, copy, s);
  }
  const int per = m.rp / 8;
  const int64_t pieces = static_cast<int64_t>(m.n) * per;
  if (pieces > MOST_THREADS - 255)
    return fail(LQ_ERR_UNSUPPORTED, "adapter product: %d rows of rank %d are more than one launch takes", m.n, m.rank);
  const int rc = halves ? product<bf16_t>(low, false, low_copy, p.u_splits, s) : product<float>(low, false, low_copy, p.u_splits, s);
  if (rc) return rc;
  const unsigned blocks = static_cast<unsigned>((pieces + 255) / 256);
  const float* part = static_cast<const float*>(low.Y);
  void* u = base + p.u;
  if (halves) adapter_scale_kernel<true><<<blocks, 256, 0, s>>>(part, p.u_splits, low.split_stride, pieces, per, m.rank, scale, low.gpos, u, m.u_rest);
  else adapter_scale_kernel<false><<<blocks, 256, 0, s>>>(part, p.u_splits, low.split_stride, pieces, per, m.rank, scale, low.gpos, u, 0);
  LQ_LAUNCH_CHECK("adapter_scale_kernel");
  return halves ? by_copy<bf16_t, false, true>(m, main_copy, 1, s) : by_copy<float, false, true>(m, main_copy, 1, s);
}

}  // namespace lq
