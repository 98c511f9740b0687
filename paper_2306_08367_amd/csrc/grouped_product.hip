// Products with the matrix of the row's group, Y[r] = X[r] W_g, and with one shared matrix and a low-rank adapter per
// group, Y[r] = X[r] W + U[r] B_g with U[r] = scale_g X[r] A_g.
//
// A tile of the result takes TM positions of ONE group (positions are sorted by group, so its rows of X and Y are
// gathered and scattered through `order`) and TN columns.  How many tiles there are is known on the device only: the
// grid holds the most there can be (n / TM and one more per group), each workgroup looks its tile up in the offsets,
// and those past the last tile end at once.  The rows without a group get tiles too: zeros.
//
// An adapter product is ONE product over all positions with the shared W, whose inner dimension goes on: behind W's k
// come the adapters that occur in the tile, 8 ranks at a time, with U in the rows of that adapter and zeros in the
// others.  U is fp32; beside bf16 matrices it goes in as two bf16 numbers (its value and what that leaves), so that
// what is lost is at most 2^-16 of it and not 2^-8.
#include "grouped.h"

namespace lq {
namespace {

// The four values of a row from column n on, by the type that the call gives: bias, gate.
template <typename T> __device__ __forceinline__ f32x4 load_four(const T* p, int valid, bool vec) {
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  if (vec) {
    if constexpr (sizeof(T) == 4) {
      r = *reinterpret_cast<const f32x4*>(p);
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      r = f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                __uint_as_float(w.y & 0xffff0000u)};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < valid) r[q] = Elem<T>::load(p + q);
  }
  return r;
}

__device__ __forceinline__ void store_four(void* row, int n, int valid, f32x4 v, bool bf16, bool vec) {
  if (vec) {
    if (bf16) *reinterpret_cast<uint2*>(static_cast<bf16_t*>(row) + n) = uint2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
    else *reinterpret_cast<f32x4*>(static_cast<float*>(row) + n) = v;
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < valid) {
      if (bf16) static_cast<bf16_t*>(row)[n + q] = f32_to_bf16(v[q]);
      else static_cast<float*>(row)[n + q] = v[q];
    }
}

template <typename T, class S, bool BT, bool DIRECT, bool ADAPT>
__global__ __launch_bounds__(S::THREADS) void grouped_product_kernel(GroupedArgs a) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128;
  typedef Operand<T, true, S::TM, S::THREADS, KBYTES> A;
  typedef Operand<T, BT, S::TN, S::THREADS, KBYTES> B;
  constexpr int KSTEP = A::KSTEP, EPC = A::EPC, THREADS = S::THREADS;
  extern __shared__ __align__(1024) char lds[];
  __shared__ int xrow[S::TM], yrow[S::TM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  RowTile tile;
  if constexpr (ADAPT) tile = all_rows<S::TM>(a.n, blockIdx.x, a.tiles_n);
  else tile = find_tile<S::TM>(a.off, a.G, a.n, blockIdx.x, a.tiles_n);
  const int n0 = tile.col * S::TN;
  if (tile.rows <= 0) return;

  for (int m = tid; m < S::TM; m += THREADS) {
    const bool in = m < tile.rows;
    const int p = tile.first + (in ? m : tile.rows - 1);     // (behind the last row: that row again, not stored)
    const int r = a.order ? a.order[p] : p;
    xrow[m] = a.x_grouped ? p : r / a.slots;
    yrow[m] = a.y_grouped ? p : r;
    if (!ADAPT && a.gpos && in && n0 == 0 && blockIdx.y == 0) a.gpos[p] = tile.group;
  }
  __syncthreads();

  f32x4 acc[S::MI][S::NI];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int k_first = blockIdx.y * a.steps_per_split * KSTEP;
  const int k_end = min(a.K, k_first + a.steps_per_split * KSTEP);
  if (tile.group >= 0 && k_first < k_end) {
    const T* X = static_cast<const T*>(a.X);
    const T* W = static_cast<const T*>(a.W) + tile.group * a.sw;
    // Where this thread's pieces of either operand lie at inner index 0, and their first inner index.  Columns behind the
    // last one repeat the last piece (direct copies) or are zeros; they are not stored.
    const T *pa[A::PER], *pb[B::PER];
    int va[A::PER], vb[B::PER];
#pragma unroll
    for (int i = 0; i < A::PER; ++i) {
      va[i] = A::piece_of(i) * EPC;
      pa[i] = X + xrow[A::line_of(i)] * a.ldx + va[i];
    }
#pragma unroll
    for (int i = 0; i < B::PER; ++i) {
      const int line = B::line_of(i), e = B::piece_of(i) * EPC;
      vb[i] = BT ? e : line;
      pb[i] = BT ? W + static_cast<int64_t>(min(n0 + line, a.N - 1)) * a.ldw + e : W + line * a.ldw + (DIRECT ? min(n0 + e, a.N - EPC) : n0 + e);
    }
    const int64_t step_b = BT ? 1 : a.ldw;     // elements per inner index
    constexpr int BUFFER = A::BYTES + B::BYTES;

    if constexpr (DIRECT) {
      auto issue = [&](int step, unsigned int to) {
        const int k0 = k_first + step * KSTEP;
        to += wave * 1024;
        if (k0 + KSTEP <= k_end) {
#pragma unroll
          for (int i = 0; i < A::PER; ++i) copy_to_lds(pa[i] + k0, to + i * THREADS * 16);
#pragma unroll
          for (int i = 0; i < B::PER; ++i) copy_to_lds(pb[i] + k0 * step_b, to + A::BYTES + i * THREADS * 16);
        } else {
#pragma unroll
          for (int i = 0; i < A::PER; ++i)
            copy_to_lds(k0 + va[i] < k_end ? static_cast<const void*>(pa[i] + k0) : &g_zeros, to + i * THREADS * 16);
#pragma unroll
          for (int i = 0; i < B::PER; ++i)
            copy_to_lds(k0 + vb[i] < k_end ? static_cast<const void*>(pb[i] + k0 * step_b) : &g_zeros, to + A::BYTES + i * THREADS * 16);
        }
      };
      const int steps = (k_end - k_first + KSTEP - 1) / KSTEP;
      if constexpr (THREADS == 512) {
        multiply_in_turns<T, S, A, B>(lds, steps, issue, acc);
      } else {
        issue(0, lds_address(lds));
        for (int step = 0; step < steps; ++step) {
          const int at = (step & 1) * BUFFER;
          meet_after_copies();     // this buffer is whole, the other one is read to its end
          if (step + 1 < steps) issue(step + 1, lds_address(lds) + (at ^ BUFFER));
          multiply_step<T, S, A, B>(lds + at, lds + at + A::BYTES, acc);
        }
      }
      __syncthreads();
    } else {
      u32x4 ra[A::PER], rb[B::PER];
      auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < A::PER; ++i) ra[i] = load_piece(pa[i] + k0, k_end - (k0 + va[i]));
#pragma unroll
        for (int i = 0; i < B::PER; ++i)
          rb[i] = load_piece(pb[i] + k0 * step_b, BT ? k_end - (k0 + vb[i]) : k0 + vb[i] < k_end ? a.N - n0 - B::piece_of(i) * EPC : 0);
      };
      auto put = [&](char* to) {
#pragma unroll
        for (int i = 0; i < A::PER; ++i) *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = ra[i];
#pragma unroll
        for (int i = 0; i < B::PER; ++i) *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = rb[i];
      };
      fetch(k_first);
      put(lds);
      int at = 0;
      for (int k0 = k_first; k0 < k_end; k0 += KSTEP, at ^= BUFFER) {
        __syncthreads();     // this buffer is whole, the other one is read to its end
        if (k0 + KSTEP < k_end) fetch(k0 + KSTEP);
        multiply_step<T, S, A, B>(lds + at, lds + at + A::BYTES, acc);
        if (k0 + KSTEP < k_end) put(lds + (at ^ BUFFER));
      }
      __syncthreads();
    }
  }

  if constexpr (ADAPT) {
    // The adapters of the tile: positions are sorted by group, so a row starts one where its group differs from the
    // row's before it.
    __shared__ int which[S::TM], gid[S::TM], firsts[S::TM / 64 + 1];
    bool starts = false;
    int g = -1;
    if (tid < S::TM) {
      const int p = tile.first + tid;
      g = tid < tile.rows ? a.group_of[p] : -1;
      starts = g >= 0 && (tid == 0 || a.group_of[p - 1] != g);
      const unsigned long long mask = __ballot(starts);
      which[tid] = __popcll(mask & (~0ull >> (63 - lane)));
      if (lane == 0) firsts[tid >> 6] = __popcll(mask);
    }
    __syncthreads();
    int count = 0, before = 0;
#pragma unroll
    for (int w = 0; w < S::TM / 64; ++w) {
      before += w < wave ? firsts[w] : 0;
      count += firsts[w];
    }
    if (tid < S::TM) {
      const int at = which[tid] + before - 1;
      which[tid] = g >= 0 ? at : -1;
      if (starts) gid[at] = g;
    }
    __syncthreads();
    // Four groups of 8 ranks a step: pieces 0..3 of a line of U's leading bf16 parts, 4..7 of the rest (fp32: 8 pieces).
    constexpr bool H = sizeof(T) == 2;
    const int per = a.rp >> 3, pieces = count * per;
    const T* Bm = static_cast<const T*>(a.B);
    // (only >= 0: of that adapter alone.)  True where B holds an infinity or a NaN.
    auto stage = [&](int q0, int only) {
      for (int id = tid; id < S::TM * (H ? 4 : 8); id += THREADS) {
        const int m = id / (H ? 4 : 8), c = id % (H ? 4 : 8);
        const int q = q0 + (H ? c : c >> 1), ad = q / per, r0 = (q % per) * 8 + (H ? 0 : 4 * (c & 1));
        float u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (q < pieces && which[m] == ad && (only < 0 || only == ad)) {
          const float* p = a.U + static_cast<int64_t>(tile.first + m) * a.rp + r0;
          for (int z = 0; z < a.u_splits; ++z)
#pragma unroll
            for (int e = 0; e < (H ? 8 : 4); ++e) u[e] += p[z * a.u_stride + e];
          const float s = a.scale ? a.scale[gid[ad]] : 1.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = r0 + e < a.rank ? u[e] * s : 0.f;    // (0 * infinity behind the last rank)
        }
        if constexpr (H) {
          u32x4 hi, lo;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            hi[e] = f32x2_to_bf16x2(u[2 * e], u[2 * e + 1]);
            const float h0 = __uint_as_float(hi[e] << 16), h1 = __uint_as_float(hi[e] & 0xffff0000u);
            // (an infinity leaves nothing)
            lo[e] = f32x2_to_bf16x2(__builtin_isfinite(h0) ? u[2 * e] - h0 : 0.f, __builtin_isfinite(h1) ? u[2 * e + 1] - h1 : 0.f);
          }
          *reinterpret_cast<u32x4*>(lds + A::place(m, c)) = hi;
          *reinterpret_cast<u32x4*>(lds + A::place(m, c + 4)) = lo;
        } else {
          *reinterpret_cast<u32x4*>(lds + A::place(m, c)) =
              u32x4{__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3])};
        }
      }
      bool bad = false;
      for (int id = tid; id < 32 * B::CPL; id += THREADS) {
        const int line = id / B::CPL, c = id % B::CPL;
        const int q = q0 + (line >> 3), ad = q / per, rank = (q % per) * 8 + (line & 7);
        u32x4 v = {0, 0, 0, 0};
        if (q < pieces && rank < a.rank && (only < 0 || only == ad))
          v = load_piece(Bm + gid[ad] * a.sB + rank * a.ldB + n0 + c * EPC, a.N - n0 - c * EPC);
        constexpr unsigned int ALL = H ? 0x7f80u : 0x7f800000u;
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (v[e] & ALL) == ALL || (H && (v[e] >> 16 & ALL) == ALL);
        *reinterpret_cast<u32x4*>(lds + A::BYTES + B::place(line, c)) = v;
      }
      return bad;
    };
    const int m0 = (wave / S::WAVES_N) * S::MI * 16, c0 = (wave % S::WAVES_N) * S::NI * 16;
    for (int q0 = 0; q0 < pieces; q0 += 4) {
      if (!__syncthreads_or(stage(q0, -1))) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int j = 0; j < S::NI; ++j) {
            const u32x4 b = B::fragment(lds + A::BYTES, c0 + 16 * j, H ? 0 : kk);
#pragma unroll
            for (int i = 0; i < S::MI; ++i) acc[i][j] = multiply<T>(b, A::fragment(lds, m0 + 16 * i, kk), acc[i][j]);
          }
      } else {
        // An infinity or a NaN times the zeros of another adapter's rows would be a NaN there: one adapter at a time,
        // added to its own rows only.
        for (int ad = q0 / per; ad <= min(q0 + 3, pieces - 1) / per; ++ad) {
          __syncthreads();
          stage(q0, ad);
          __syncthreads();
          for (int j = 0; j < S::NI; ++j)
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
              f32x4 part = {0.f, 0.f, 0.f, 0.f};
              for (int kk = 0; kk < 2; ++kk)
                part = multiply<T>(B::fragment(lds + A::BYTES, c0 + 16 * j, H ? 0 : kk), A::fragment(lds, m0 + 16 * i, kk), part);
              const bool mine = which[m0 + 16 * i + (lane & 15)] == ad;
#pragma unroll
              for (int jj = 0; jj < S::NI; ++jj)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i][jj][q] += mine && jj == j ? part[q] : 0.f;
            }
        }
      }
      __syncthreads();
    }
  }

  const int wm = (wave / S::WAVES_N) * S::MI * 16, wn = n0 + (wave % S::WAVES_N) * S::NI * 16;
  const bool has_bias = a.bias && tile.group >= 0;
  const T* bias = static_cast<const T*>(a.bias) + (has_bias ? tile.group * a.ldb : 0);
  char* const Y = static_cast<char*>(a.Y) + blockIdx.y * a.split_stride * (a.y_bf16 ? 2 : 4);
  if (S::NI == 4 && a.y_vec && wn + 64 <= a.n_store && wn + 64 <= a.N) {
    // 16 neighbouring columns of a row a lane
    const int n = wn + 16 * (lane >> 4);
    f32x4 bv[4] = {};
    if (has_bias)
#pragma unroll
      for (int q = 0; q < 4; ++q) bv[q] = load_four(bias + n + 4 * q, 4, true);
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
      if (m >= tile.rows) continue;
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
          const f32x4 h = load_four(static_cast<const T*>(a.gate) + r * a.ldg + n + 4 * j, 4, true);
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
    const bool vec = a.y_vec && valid >= 4;
    f32x4 bv = {0.f, 0.f, 0.f, 0.f};
    if (has_bias) bv = load_four(bias + n, a.N - n, vec);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int m = wm + 16 * i + (lane & 15);
      if (m >= tile.rows) continue;
      const int64_t r = yrow[m];
      f32x4 v = acc[i][j] + bv;
      if (a.relu)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = v[q] < 0.f ? 0.f : v[q];
      if (a.gate) {
        const f32x4 h = load_four(static_cast<const T*>(a.gate) + r * a.ldg + n, valid, vec);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = h[q] > 0.f ? v[q] : 0.f;
      }
      store_four(Y + r * a.ldy * (a.y_bf16 ? 2 : 4), n, valid, v, a.y_bf16, vec);
    }
  }
}

template <typename T, class S, bool BT, bool DIRECT, bool ADAPT> int launch(GroupedArgs a, int splits, hipStream_t s) {
  constexpr int KBYTES = S::THREADS == 512 ? 64 : 128;
  typedef Operand<T, true, S::TM, S::THREADS, KBYTES> A;
  typedef Operand<T, BT, S::TN, S::THREADS, KBYTES> B;
  constexpr int LDS = (S::THREADS == 512 ? 4 : 2) * (A::BYTES + B::BYTES);
  a.tiles_n = (a.n_store + S::TN - 1) / S::TN;
  a.row_tiles = ADAPT ? (a.n + S::TM - 1) / S::TM : a.n / S::TM + std::min(a.n, a.G + 1);
  const int steps = (a.K + A::KSTEP - 1) / A::KSTEP;
  a.steps_per_split = (steps + splits - 1) / splits;
  const int64_t blocks = static_cast<int64_t>(a.tiles_n) * a.row_tiles;
  if (blocks > 0x7fffffff) return fail(LQ_ERR_UNSUPPORTED, "grouped product: %lld tiles are more than one launch takes", (long long)blocks);
  const auto kernel = grouped_product_kernel<T, S, BT, DIRECT, ADAPT>;
  if (LDS >= 64 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  kernel<<<dim3(static_cast<unsigned>(blocks), splits), S::THREADS, LDS, s>>>(a);
  LQ_LAUNCH_CHECK("grouped_product_kernel");
  return LQ_OK;
}

typedef TileShape<128, 128, 2, 2> Tile128;
typedef TileShape<64, 64, 2, 2> Tile64;
typedef TileShape<256, 256, 2, 4> Tile256;

template <typename T, bool BT, bool DIRECT, bool ADAPT> int by_size(const GroupedArgs& a, int splits, hipStream_t s) {
  const int64_t large = static_cast<int64_t>((a.n_store + 127) / 128) * ((a.n + 127) / 128);
  if constexpr (sizeof(T) == 2 && DIRECT)
    if (large >= 4 * num_cus()) return launch<T, Tile256, BT, DIRECT, ADAPT>(a, splits, s);
  if (large >= num_cus()) return launch<T, Tile128, BT, DIRECT, ADAPT>(a, splits, s);
  return launch<T, Tile64, BT, DIRECT, ADAPT>(a, splits, s);
}

template <typename T> int product(const GroupedArgs& a, bool transposed, bool in_vec, int splits, hipStream_t s) {
  if (transposed) return in_vec ? by_size<T, true, true, false>(a, splits, s) : by_size<T, true, false, false>(a, splits, s);
  return in_vec ? by_size<T, false, true, false>(a, splits, s) : by_size<T, false, false, false>(a, splits, s);
}

}  // namespace

int launch_grouped_product(const GroupedArgs& a, int32_t dtype, bool transposed, bool in_vec, hipStream_t s) {
  return dtype == LQ_BF16 ? product<bf16_t>(a, transposed, in_vec, 1, s) : product<float>(a, transposed, in_vec, 1, s);
}

int launch_adapter_product(const GroupedArgs& m, const GroupedArgs& low, int32_t dtype, bool main_vec, bool low_vec, hipStream_t s) {
  const int rc = dtype == LQ_BF16 ? product<bf16_t>(low, false, low_vec, m.u_splits, s) : product<float>(low, false, low_vec, m.u_splits, s);
  if (rc) return rc;
  if (dtype == LQ_BF16) return main_vec ? by_size<bf16_t, false, true, true>(m, 1, s) : by_size<bf16_t, false, false, true>(m, 1, s);
  return main_vec ? by_size<float, false, true, true>(m, 1, s) : by_size<float, false, false, true>(m, 1, s);
}

}  // namespace lq
