// Gradients of the grouped product's matrices: dW_g = sum over the rows r of group g of X[r]^T dY[r], db_g = sum of dY[r].
//
// A tile of dW_g is a product whose inner dimension is the group's rows: both operands are lines of the inner index
// (a row of X, a row of dY), so bf16 ones come transposed out of LDS.  The bias is the product of ones with dY, in the
// workgroups of the first rows of the tiles.
#include "grouped.h"

namespace lq {
namespace {

template <typename T, class S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void grouped_gradient_kernel(GradientArgs a) {
  typedef Operand<T, false, S::TM, S::THREADS> A;
  typedef Operand<T, false, S::TN, S::THREADS> B;
  constexpr int KSTEP = A::KSTEP, EPC = A::EPC, THREADS = S::THREADS;
  extern __shared__ __align__(1024) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int id = die_order(blockIdx.x, gridDim.x);
  const int per_group = a.tiles_m * a.tiles_n;
  const int group = id / per_group, tm = id % per_group / a.tiles_n, tn = id % a.tiles_n;
  const int m0 = tm * S::TM, n0 = tn * S::TN;
  const int first = a.off[group], rows = a.off[group + 1] - first;

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

  const T *X = static_cast<const T*>(a.X), *dY = static_cast<const T*>(a.dY);
  // The rows of X and dY that hold this thread's pieces of the step from k0 on (-1: none).
  auto row_of = [&](int k, bool grouped, int slots) -> int {
    if (k >= rows) return -1;
    const int p = first + k;
    return grouped || !a.order ? (grouped ? p : p / slots) : a.order[p] / slots;
  };
  int xr[A::PER], yr[B::PER];
  auto look_up = [&](int k0) {
#pragma unroll
    for (int i = 0; i < A::PER; ++i) xr[i] = row_of(k0 + A::line_of(i), a.x_grouped, a.slots);
#pragma unroll
    for (int i = 0; i < B::PER; ++i) yr[i] = row_of(k0 + B::line_of(i), a.y_grouped, 1);
  };
  u32x4 ra[DIRECT ? 1 : A::PER], rb[DIRECT ? 1 : B::PER];
  auto fetch = [&](char* to) {
    const unsigned int at = DIRECT ? lds_address(to) : 0;
#pragma unroll
    for (int i = 0; i < A::PER; ++i) {
      const int c = m0 + A::piece_of(i) * EPC;
      const T* p = X + xr[i] * a.ldx + c;
      if constexpr (DIRECT) copy_to_lds(xr[i] >= 0 && c < a.k ? static_cast<const void*>(p) : &g_zeros, at + (i * THREADS + wave * 64) * 16);
      else ra[i] = load_piece(p, xr[i] >= 0 ? a.k - c : 0);
    }
#pragma unroll
    for (int i = 0; i < B::PER; ++i) {
      const int c = n0 + B::piece_of(i) * EPC;
      const T* p = dY + yr[i] * a.ldy + c;
      if constexpr (DIRECT) copy_to_lds(yr[i] >= 0 && c < a.l ? static_cast<const void*>(p) : &g_zeros, at + A::BYTES + (i * THREADS + wave * 64) * 16);
      else rb[i] = load_piece(p, yr[i] >= 0 ? a.l - c : 0);
    }
  };
  auto put = [&](char* to) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < A::PER; ++i) *reinterpret_cast<u32x4*>(to + (i * THREADS + tid) * 16) = ra[i];
#pragma unroll
      for (int i = 0; i < B::PER; ++i) *reinterpret_cast<u32x4*>(to + A::BYTES + (i * THREADS + tid) * 16) = rb[i];
    }
  };
  constexpr int BUFFER = A::BYTES + B::BYTES;
  if (rows > 0) {
    look_up(0);
    fetch(lds);
    put(lds);
    look_up(KSTEP);
    int at = 0;
    for (int k0 = 0; k0 < rows; k0 += KSTEP, at ^= 1) {
      if constexpr (DIRECT) meet_after_copies();
      else __syncthreads();     // this buffer is whole, the other one is read to its end
      const bool more = k0 + KSTEP < rows;
      if (more) {
        fetch(lds + (at ^ 1) * BUFFER);
        look_up(k0 + 2 * KSTEP);
      }
      multiply_step<T, S, A, B>(lds + at * BUFFER, lds + at * BUFFER + A::BYTES, acc);
      if (bias) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int j = 0; j < S::NI; ++j) sum[j] = multiply<T>(B::fragment(lds + at * BUFFER + A::BYTES, wn + 16 * j, kk), ones, sum[j]);
      }
      if (more) put(lds + (at ^ 1) * BUFFER);
    }
  }

  auto store = [&](void* base, int64_t row, int n, f32x4 v) {
    const int valid = a.l - n;
    if (a.w_vec && valid >= 4) {
      if (a.w_bf16) *reinterpret_cast<uint2*>(static_cast<bf16_t*>(base) + row + n) = uint2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
      else *reinterpret_cast<f32x4*>(static_cast<float*>(base) + row + n) = v;
      return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < valid) {
        if (a.w_bf16) static_cast<bf16_t*>(base)[row + n + q] = f32_to_bf16(v[q]);
        else static_cast<float*>(base)[row + n + q] = v[q];
      }
  };
#pragma unroll
  for (int j = 0; j < S::NI; ++j) {
    const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
    if (n >= a.l) continue;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int m = m0 + wm + 16 * i + (lane & 15);
      if (m < a.k) store(a.dW, group * a.sw + m * a.ldw, n, acc[i][j]);
    }
    if (bias && (lane & 15) == 0) store(a.db, group * a.ldb, n, sum[j]);
  }
}

template <typename T, class S, bool DIRECT> int launch(GradientArgs a, hipStream_t s) {
  typedef Operand<T, false, S::TM, S::THREADS> A;
  typedef Operand<T, false, S::TN, S::THREADS> B;
  constexpr int LDS = 2 * (A::BYTES + B::BYTES);
  a.tiles_m = (a.k + S::TM - 1) / S::TM;
  a.tiles_n = (a.l + S::TN - 1) / S::TN;
  const int64_t blocks = static_cast<int64_t>(a.G) * a.tiles_m * a.tiles_n;
  if (blocks > 0x7fffffff) return fail(LQ_ERR_UNSUPPORTED, "grouped gradient: %lld tiles are more than one launch takes", (long long)blocks);
  const auto kernel = grouped_gradient_kernel<T, S, DIRECT>;
  if (LDS >= 64 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  kernel<<<static_cast<unsigned>(blocks), S::THREADS, LDS, s>>>(a);
  LQ_LAUNCH_CHECK("grouped_gradient_kernel");
  return LQ_OK;
}

typedef TileShape<128, 128, 2, 2> Tile128;
typedef TileShape<64, 64, 2, 2> Tile64;

template <typename T, bool DIRECT> int by_size(const GradientArgs& a, hipStream_t s) {
  const int64_t large = static_cast<int64_t>((a.k + 127) / 128) * ((a.l + 127) / 128) * a.G;
  return large >= num_cus() ? launch<T, Tile128, DIRECT>(a, s) : launch<T, Tile64, DIRECT>(a, s);
}

}  // namespace

int launch_grouped_gradient(const GradientArgs& a, int32_t dtype, bool in_vec, hipStream_t s) {
  if (dtype == LQ_BF16) return in_vec ? by_size<bf16_t, true>(a, s) : by_size<bf16_t, false>(a, s);
  return in_vec ? by_size<float, true>(a, s) : by_size<float, false>(a, s);
}

}  // namespace lq
