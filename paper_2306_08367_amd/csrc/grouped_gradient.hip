// Gradients of the grouped product's matrices: dW_g = sum over the rows r of group g of X[r]^T dY[r], db_g = sum of dY[r].
//
// A tile of dW_g is a product whose inner dimension is the group's rows: both operands are lines of the inner index
// (a row of X, a row of dY), so bf16 ones come transposed out of LDS.  The bias is the product of ones with dY, in the
// wavefronts of the first rows of the first tiles.
//
// Groups differ in size and only the device knows by how much, so a group's rows are added up in chunks of at most `most`
// rows, each by workgroups of its own.  A group of one chunk is written at once; the chunks of a larger one leave partial
// sums in the workspace, which a second launch adds up in their order: no atomics, the same bits every time.  `most` is
// what a workgroup gets if all rows are shared out evenly (half of that: 265 instead of 221 us below, for the partial sums' way through
// memory), but no fewer rows than are worth a workgroup.
//
// What bounds it, measured: 8,192^3 in bf16 1,052 TFLOP/s, both operands transposed on their way out of LDS; 32,768 rows in 16 groups,
// 2,048 x 1,024 into fp32, 196 to 203 us = 680 to 700, of which the launch that adds up partial sums takes 16, and 134 MB of results; fp32,
// 20,001 rows in 12 groups, 100 x 64, 20 us, two short launches.
#include "grouped.h"

namespace lq {
namespace {

constexpr int SEGMENT = 2048;     // rows whose numbers are held in LDS at a time
constexpr int RUN = 32;           // most tiles of a chunk that go to one die together

template <typename T, class S, int COPY>
__global__ __launch_bounds__(S::THREADS, 2) void grouped_gradient_kernel(GradientArgs a) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128, COPIERS = 256;     // threads that copy a step
  typedef Operand<T, false, S::TM, COPIERS, KBYTES, COPY ? COPY : 16> A;
  typedef Operand<T, false, S::TN, COPIERS, KBYTES, COPY ? COPY : 16> B;
  constexpr bool DIRECT = COPY != 0;           // through LDS without registers
  constexpr int E = DIRECT ? COPY / static_cast<int>(sizeof(T)) : 1;
  constexpr int KSTEP = A::KSTEP, EPC = A::EPC, THREADS = S::THREADS, BUFFER = A::BYTES + B::BYTES;
  extern __shared__ __align__(1024) char lds[];
  __shared__ int xrow[SEGMENT], yrow[SEGMENT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the 8 dies in turn.  The tiles of a chunk, which share its rows, go to one die in runs of up to 32 (a
  // die's compute units), the runs to the dies forth and back, so that each gets long and short ones.
  const int tiles = a.tiles_m * a.tiles_n, run_tiles = min(tiles, RUN), runs = (tiles + run_tiles - 1) / run_tiles;
  const int die = blockIdx.x & 7, turn = (blockIdx.x >> 3) / run_tiles;
  const int run = turn * 8 + ((turn & 1) ? 7 - die : die), tile = run % runs * run_tiles + (blockIdx.x >> 3) % run_tiles;
  if (tile >= tiles) return;
  const Chunk chunk = find_chunk(a.off, a.G, a.most, run / runs);
  if (chunk.group < 0) return;
  const int tm = tile / a.tiles_n, tn = tile % a.tiles_n;
  const int m0 = tm * S::TM, n0 = tn * S::TN;

  f32x4 acc[S::MI][S::NI], sum[S::NI];
#pragma unroll
  for (int j = 0; j < S::NI; ++j) {
    sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S::MI; ++i) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int wm = (wave / S::WAVES_N) * S::MI * 16, wn = (wave % S::WAVES_N) * S::NI * 16;
  const bool bias = a.db && tm == 0 && wm == 0;
  const unsigned int one = sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u;
  const u32x4 ones = {one, one, one, one};
  const auto add_up = [&](const u32x4(&b)[S::NI]) {
    if (bias)
#pragma unroll
      for (int j = 0; j < S::NI; ++j) sum[j] = multiply<T>(b[j], ones, sum[j]);
  };

  // (columns behind the last one hold something else of the matrix or zeros; they are not stored)
  const T *X = static_cast<const T*>(a.X), *dY = static_cast<const T*>(a.dY);
  int ca[A::PER], cb[B::PER];
#pragma unroll
  for (int i = 0; i < A::PER; ++i) ca[i] = min(m0 + A::element_of(i), a.k - E);
#pragma unroll
  for (int i = 0; i < B::PER; ++i) cb[i] = min(n0 + B::element_of(i), a.l - E);

  for (int s0 = 0; s0 < chunk.rows; s0 += SEGMENT) {
    const int first = chunk.first + s0, rows = min(SEGMENT, chunk.rows - s0), steps = (rows + KSTEP - 1) / KSTEP;
    __syncthreads();     // (the segment before is read to its end)
    for (int i = tid; i < rows; i += THREADS) {
      const int p = first + i, r = a.order ? a.order[p] : p;
      xrow[i] = a.x_grouped ? p : r / a.slots;
      yrow[i] = a.y_grouped ? p : r;
    }
    __syncthreads();
    // Copies of a step (rows behind the last one: zeros in both operands).  With turns, row numbers are read from LDS a turn ahead of
    // their copies.
    constexpr int COPIES = A::PER + B::PER;
    int number[COPIES], looked = -1;
    auto look_up = [&](int step) {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) {
        const int line = step * KSTEP + (c >= A::PER ? B::line_of(c - A::PER) : A::line_of(c));
        number[c] = line < rows ? (c >= A::PER ? yrow[line] : xrow[line]) : -1;
      }
      looked = step;
    };
    auto issue = [&](int step, unsigned int to) {
      if (THREADS != 512 || looked != step) look_up(step);
#pragma unroll
      for (int c = 0; c < COPIES; ++c) {
        const T* p = c >= A::PER ? dY + number[c] * a.ldy + cb[c - A::PER] : X + number[c] * a.ldx + ca[c];
        copy_to_lds<COPY>(number[c] >= 0 ? static_cast<const void*>(p) : &g_zeros,
                          to + (wave & 3) * 64 * COPY + (c >= A::PER ? A::BYTES + (c - A::PER) * COPIERS * COPY : c * COPIERS * COPY));
      }
      if constexpr (THREADS == 512) look_up(step + 2);     // (this wavefront's next block)
    };
    if constexpr (DIRECT && THREADS == 512) {
      // (a block behind the last one is zeros)
      multiply_in_turns<T, S, A, B>(lds, (steps + 1) >> 1, issue, acc, add_up);
    } else if constexpr (DIRECT) {
      multiply_steps<T, S, A, B, S::RING>(lds, steps, issue, acc, [&](const u32x4(&b)[S::NI]) { add_up(b); });
    } else {
      // A row may end inside a piece.  All 16 bytes may be read unless the row is the matrix's last one: there the 16 bytes end with
      // the row, and are moved to their places on the way to LDS.  (Rows shorter than a piece: element by element.)
      const bool narrow = a.k < EPC || a.l < EPC;
      const int last_x = a.n / a.slots - 1, last_y = a.n - 1;
      auto piece = [&](const T* base, int r, int64_t ld, int c, int cols, int last) -> const T* {
        if (r < 0) return reinterpret_cast<const T*>(&g_zeros);
        return base + r * ld + (r == last ? min(c, cols - EPC) : c);
      };
      auto in_place = [&](u32x4 v, int r, int c, int cols, int last) {
        const int by = c - (cols - EPC);      // elements that it starts early
        if (r == last && by > 0) {
          const T* e = reinterpret_cast<const T*>(&v);
          u32x4 w = {0, 0, 0, 0};
#pragma unroll
          for (int q = 0; q < EPC; ++q)
#pragma unroll
            for (int f = q + 1; f < EPC; ++f)
              if (f == q + by) reinterpret_cast<T*>(&w)[q] = e[f];
          return w;
        }
        return v;
      };
      auto x_at = [&](int line) { return line < rows ? xrow[line] : -1; };
      auto y_at = [&](int line) { return line < rows ? yrow[line] : -1; };
      u32x4 ra[A::PER], rb[B::PER];
      auto fetch = [&](int step) {
#pragma unroll
        for (int i = 0; i < A::PER; ++i) ra[i] = load_whole(piece(X, x_at(step * KSTEP + A::line_of(i)), a.ldx, ca[i], a.k, last_x));
#pragma unroll
        for (int i = 0; i < B::PER; ++i) rb[i] = load_whole(piece(dY, y_at(step * KSTEP + B::line_of(i)), a.ldy, cb[i], a.l, last_y));
      };
      auto put = [&](int step, char* to) {
#pragma unroll
        for (int i = 0; i < A::PER; ++i)
          *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = in_place(ra[i], x_at(step * KSTEP + A::line_of(i)), ca[i], a.k, last_x);
#pragma unroll
        for (int i = 0; i < B::PER; ++i)
          *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = in_place(rb[i], y_at(step * KSTEP + B::line_of(i)), cb[i], a.l, last_y);
      };
      auto fill = [&](int step, char* to) {
#pragma unroll
        for (int i = 0; i < A::PER; ++i) {
          const int r = x_at(step * KSTEP + A::line_of(i));
          *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = load_piece(X + r * a.ldx + ca[i], r >= 0 ? a.k - ca[i] : 0);
        }
#pragma unroll
        for (int i = 0; i < B::PER; ++i) {
          const int r = y_at(step * KSTEP + B::line_of(i));
          *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = load_piece(dY + r * a.ldy + cb[i], r >= 0 ? a.l - cb[i] : 0);
        }
      };
      fill(0, lds);
      for (int step = 0; step < steps; ++step) {
        const int at = (step & 1) * BUFFER;
        __syncthreads();         // this buffer is whole, the other one is read to its end
        const bool more = step + 1 < steps, ahead = more && !narrow;
        if (ahead) fetch(step + 1);
        fence();                 // (the loads go ahead of the products)
        multiply_step<T, S, A, B>(lds + at, lds + at + A::BYTES, acc, add_up);
        if (ahead) put(step + 1, lds + (at ^ BUFFER));
        else if (more) fill(step + 1, lds + (at ^ BUFFER));
      }
    }
  }

  const int64_t part = chunk.place >= 0 ? chunk.place * (static_cast<int64_t>(a.k) + 1) * a.l : 0;
  auto store = [&](void* base, int64_t at, int n, f32x4 v) {
    if (a.w_bf16) store_four<true>(base, at + n, a.l - n, v);
    else store_four<false>(base, at + n, a.l - n, v);
  };
#pragma unroll
  for (int j = 0; j < S::NI; ++j) {
    const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
    if (n >= a.l) continue;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int m = m0 + wm + 16 * i + (lane & 15);
      if (m >= a.k) continue;
      if (chunk.place >= 0) store_four<false>(a.part, part + static_cast<int64_t>(m) * a.l + n, a.l - n, acc[i][j]);
      else store(a.dW, chunk.group * a.sw + m * a.ldw, n, acc[i][j]);
    }
    if (bias && (lane & 15) == 0) {
      if (chunk.place >= 0) store_four<false>(a.part, part + static_cast<int64_t>(a.k) * a.l + n, a.l - n, sum[j]);
      else store(a.db, chunk.group * a.ldb, n, sum[j]);
    }
  }
}

// Adds up the partial sums of the blockIdx.y-th group of more than one chunk, four results of a row a thread.
template <bool BF16> __global__ __launch_bounds__(256) void gradient_sum_kernel(GradientArgs a) {
  const int lane = threadIdx.x & 63;
  // the group, and how many partial sums lie before its own
  const int per = (a.G + 63) >> 6, g0 = min(lane * per, a.G), g1 = min(g0 + per, a.G);
  int own = 0, parts = 0;
  for (int g = g0; g < g1; ++g) {
    const int c = chunks_of(a.off[g + 1] - a.off[g], a.most);
    own += c > 1;
    parts += c > 1 ? c : 0;
  }
  int upto = own, parts_upto = parts;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d), w = __shfl_up(parts_upto, d);
    if (lane >= d) {
      upto += v;
      parts_upto += w;
    }
  }
  const int which = blockIdx.y;
  const unsigned long long holds = __ballot(upto > which);
  if (!holds) return;
  const int at = __ffsll(static_cast<long long>(holds)) - 1;
  int group = 0, first = 0, count = 0;
  if (lane == at) {
    int left = which - (upto - own);
    first = parts_upto - parts;
    for (int g = g0; g < g1; ++g) {
      const int c = chunks_of(a.off[g + 1] - a.off[g], a.most);
      if (c <= 1) continue;
      if (left-- == 0) {
        group = g;
        count = c;
        break;
      }
      first += c;
    }
  }
  group = __builtin_amdgcn_readlane(group, at);
  first = __builtin_amdgcn_readlane(first, at);
  count = __builtin_amdgcn_readlane(count, at);

  const int fours = (a.l + 3) >> 2, rows = a.k + (a.db ? 1 : 0);
  const int64_t stride = (static_cast<int64_t>(a.k) + 1) * a.l;
  for (int64_t id = blockIdx.x * 256ll + threadIdx.x; id < static_cast<int64_t>(rows) * fours; id += gridDim.x * 256ll) {
    const int m = static_cast<int>(id / fours), n = static_cast<int>(id - static_cast<int64_t>(m) * fours) * 4;
    const float* p = a.part + first * stride + static_cast<int64_t>(m) * a.l + n;
    const int valid = min(4, a.l - n);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    int c = 0;
    for (; c + 4 <= count; c += 4) {      // (four loads under way together)
      f32x4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = load_four(p + (c + q) * stride, valid);
#pragma unroll
      for (int q = 0; q < 4; ++q) v += w[q];
    }
    for (; c < count; ++c) v += load_four(p + c * stride, valid);
    if (m < a.k) store_four<BF16>(a.dW, group * a.sw + m * a.ldw + n, valid, v);
    else store_four<BF16>(a.db, group * a.ldb + n, valid, v);
  }
}

// Side of the tiles and most rows of a chunk.  Large tiles read less from LDS for an instruction: 256 from where most of a tile
// is filled, in bf16 with aligned rows.  A workgroup's share of n rows is n * tiles / workgroups that run at once (one of 512
// threads a compute unit, else two).  At least 1,024 rows for a tile of 256 (its partial sums take as long as 800), else 256.
struct Plan { int side; int64_t most, places; };
// (the kernel holds it in 32 bits; tiles behind 2^32 make no difference to that)
constexpr int64_t most_rows(int64_t n, int64_t tiles, int64_t at_once, int64_t least) {
  const int64_t even = n * std::min(tiles, int64_t{1} << 32) / at_once;
  return std::min<int64_t>(std::max((even + 63) / 64 * 64, least), INT32_MAX);
}
static_assert(most_rows(1 << 25, 1 << 14, 256, 1024) == INT32_MAX && most_rows(1 << 30, int64_t{1} << 48, 512, 256) == INT32_MAX &&
              most_rows(32768, 32, 256, 1024) == 4096 && most_rows(0, 1, 512, 256) == 256, "rows of a chunk");
Plan plan_of(int64_t n, int32_t G, int32_t k, int32_t l, int32_t dtype, int copy) {
  Plan p;
  p.side = dtype == LQ_BF16 && copy == 16 && k > 192 && l > 192 ? 256 : k > 64 && l > 64 ? 128 : 64;
  const int64_t tiles = static_cast<int64_t>((k + p.side - 1) / p.side) * ((l + p.side - 1) / p.side);
  p.most = most_rows(n, tiles, num_cus() * (p.side == 256 ? 1 : 2), p.side == 256 ? 1024 : 256);
  // chunks of groups of more than one: fewer than two for every `most` rows, and fewer than one more a group
  p.places = n > p.most ? std::min<int64_t>(2 * n / p.most, n / p.most + G) : 0;
  return p;
}
size_t place_bytes(int64_t places, int32_t k, int32_t l) { return static_cast<size_t>(places) * (static_cast<size_t>(k) + 1) * l * 4; }

template <typename T, class S, int COPY> int launch(GradientArgs a, const Plan& p, hipStream_t s) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128, COPIERS = 256;     // threads that copy a step
  typedef Operand<T, false, S::TM, COPIERS, KBYTES, COPY ? COPY : 16> A;
  typedef Operand<T, false, S::TN, COPIERS, KBYTES, COPY ? COPY : 16> B;
  constexpr int LDS = (COPY ? S::RING : 2) * (A::BYTES + B::BYTES);
  a.tiles_m = (a.k + S::TM - 1) / S::TM;
  a.tiles_n = (a.l + S::TN - 1) / S::TN;
  const int64_t chunks = a.n / p.most + a.G, tiles = static_cast<int64_t>(a.tiles_m) * a.tiles_n;
  const int64_t run_tiles = std::min<int64_t>(tiles, RUN), runs = chunks * ((tiles + run_tiles - 1) / run_tiles);
  const int64_t blocks = (runs + 7) / 8 * 8 * run_tiles;
  if (blocks * S::THREADS > MOST_THREADS) return fail(LQ_ERR_UNSUPPORTED, "grouped gradient: %lld tiles are more than one launch takes", (long long)blocks);
  const auto kernel = grouped_gradient_kernel<T, S, COPY>;
  if (LDS + SEGMENT * 4 > 48 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  kernel<<<static_cast<unsigned>(blocks), S::THREADS, LDS, s>>>(a);
  LQ_LAUNCH_CHECK("grouped_gradient_kernel");
  return LQ_OK;
}

typedef TileShape<128, 128, 2, 2> Tile128;
typedef TileShape<64, 64, 2, 2, 4> Tile64;
typedef TileShape<256, 256, 2, 4, 4> Tile256;

template <typename T, int COPY> int by_size(const GradientArgs& a, const Plan& p, hipStream_t s) {
  if constexpr (sizeof(T) == 2 && COPY == 16)
    if (p.side == 256) return launch<T, Tile256, COPY>(a, p, s);
  return p.side == 128 ? launch<T, Tile128, COPY>(a, p, s) : launch<T, Tile64, COPY>(a, p, s);
}
template <typename T> int by_copy(const GradientArgs& a, int copy, const Plan& p, hipStream_t s) {
  if (copy == 16) return by_size<T, 16>(a, p, s);
  if constexpr (sizeof(T) == 2)
    if (copy == 0) return by_size<T, 0>(a, p, s);
  return by_size<T, 4>(a, p, s);
}

}  // namespace

size_t grouped_gradient_ws_bytes(int64_t n, int32_t G, int32_t k, int32_t l, int32_t dtype) {
  size_t most = 0;
  for (const int copy : {4, 16}) most = std::max(most, place_bytes(plan_of(n, G, k, l, dtype, copy).places, k, l));
  return round_up(most, 256);
}

int launch_grouped_gradient(const GradientArgs& args, int32_t dtype, int copy, void* ws, size_t ws_bytes, hipStream_t s) {
  GradientArgs a = args;
  Plan p = plan_of(a.n, a.G, a.k, a.l, dtype, copy);
  if (!ws || ws_bytes < place_bytes(p.places, a.k, a.l)) p.most = std::max<int64_t>(a.n, 1);     // without room: whole groups
  a.most = static_cast<int32_t>(p.most);
  a.part = static_cast<float*>(ws);
  const int rc = dtype == LQ_BF16 ? by_copy<bf16_t>(a, copy, p, s) : by_copy<float>(a, copy, p, s);
  if (rc) return rc;
  if (a.n > p.most) {
    const int64_t fours = static_cast<int64_t>(a.k + 1) * ((a.l + 3) / 4);
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>(a.G, a.n / p.most));    // more than `most` rows each
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((fours + 255) / 256, 1024)), groups);
    if (a.w_bf16) gradient_sum_kernel<true><<<grid, 256, 0, s>>>(a);
    else gradient_sum_kernel<false><<<grid, 256, 0, s>>>(a);
    LQ_LAUNCH_CHECK("gradient_sum_kernel");
  }
  return LQ_OK;
}

}  // namespace lq
