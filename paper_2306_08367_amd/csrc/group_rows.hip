// Row numbers of every group from a column of keys: a stable counting sort by group.
//
// A workgroup takes a run of keys and each of its wavefronts a run of that.  Two passes over the keys: the first counts
// the keys of every group per wavefront (LDS), the second puts every row at
//   first place of the group + rows of earlier workgroups + of earlier wavefronts + of earlier steps + of earlier lanes,
// where the lanes of one step that share a group are told apart by ballots: no atomic decides a place, so the order is the rows'
// own.  Up to 10,240 keys are done by one workgroup in one launch; more take three launches: counts per workgroup, sums of those over
// the workgroups, places.  There a workgroup first sorts up to 8,192 rows in LDS and then writes them out in that order, so that
// neighbouring lanes write neighbouring places, as long as LDS holds that beside the counts (up to 3,173 groups).
// A key outside [0, G) counts as group G, whose rows come last.
// What bounds it: 64 keys 4.4 us, a launch; 200,000 keys in 64 groups 14 us, three; 6e6 keys in 2,000 groups 67 us, 50 of them in the last launch (the 48 MB that have to move take 9): the chain of LDS accesses and ballots of a step, four wavefronts a SIMD, and the barriers between the passes.
// (Rows written one by one: 75; ranks of the second pass kept in registers from the first: 67 to 71, small calls slower.)
#include "grouped.h"

namespace lq {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
// Most keys of the one-workgroup form (16 groups: 8,192 keys 11.0 us, in three launches 12.4; 12,000 15.4 and 12.5).
constexpr int64_t ONE_GROUP_KEYS = 10240;

__device__ __forceinline__ int group_of_key(int key, int G) { return static_cast<unsigned>(key) < static_cast<unsigned>(G) ? key : G; }

// Up to 15 groups over many keys: one lane of a group counts for all, which else wait for each other at its counter (2.3e6 keys in 7
// groups 54 -> 38 us; instantiations of their own, since the code of both ways took a call of 64 keys from 4.7 to 6.7 us).
constexpr int FEW_BITS = 4;

// The active lanes of this lane's group.
__device__ __forceinline__ unsigned long long same_group(int g, int bits, unsigned long long active) {
  unsigned long long same = active;
  for (int b = 0; b < bits; ++b) {
    const bool one = (g >> b) & 1;
    const unsigned long long v = __ballot(one);
    same &= one ? v : ~v;
  }
  return same;
}

// How many lanes below this one hold the same group, of those of `active`; `shared`: whether this lane's group is another active
// lane's as well.  A few such groups are gone through one by one; from many on, all lanes are compared bit by bit.
__device__ __forceinline__ int lanes_before(int g, int bits, bool shared, unsigned long long active) {
  const unsigned long long below = (1ull << (threadIdx.x & 63)) - 1;
  unsigned long long left = __ballot(shared);
  int before = 0;
  if (__popcll(left) <= 24) {
    while (left) {
      const int leader = __builtin_amdgcn_readlane(g, __ffsll(static_cast<long long>(left)) - 1);
      const unsigned long long same = __ballot(g == leader) & left;
      if (g == leader) before = __popcll(same & below);
      left &= ~same;
    }
    return before;
  }
  return __popcll(same_group(g, bits, active) & below);
}

// Sum over the workgroup's threads below this one; *total: over all.
__device__ __forceinline__ int scan_threads(int v, int* shared, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(upto, d);
    if (lane >= d) upto += u;
  }
  if (lane == 63) shared[wave] = upto;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? shared[w] : 0;
    all += shared[w];
  }
  __syncthreads();
  *total = all;
  return before + upto - v;
}

// LDS: base [G + 1] ints, then per wavefront [G + 1] 16-bit counts, two in a word.  sum_waves and place_rows make a count that of the
// rows of ALL wavefronts up to its own, so what a workgroup counts at a time has to stay below 65,536 rows: a round.
__host__ __device__ constexpr int count_words(int G) { return (G + 2) >> 1; }
constexpr size_t place_lds(int G) { return (static_cast<size_t>(G) + 1 + static_cast<size_t>(WAVES) * count_words(G)) * 4; }

// Keys [begin, end) of this workgroup, run [b, e) of a wavefront.
__device__ __forceinline__ void wave_run(int64_t begin, int64_t end, int64_t* b, int64_t* e) {
  const int64_t per = (end - begin + WAVES - 1) / WAVES;
  const int wave = threadIdx.x >> 6;
  *b = min(begin + wave * per, end);
  *e = min(*b + per, end);
}

constexpr int AHEAD = 8;      // keys of a lane whose loads are under way together

// add(group, how many) for the keys [b, e) of a wavefront.
template <bool FEW, typename F> __device__ __forceinline__ void count_groups(const int32_t* __restrict__ keys, int G, int bits, int64_t b, int64_t e, F&& add) {
  const int lane = threadIdx.x & 63;
  for (int64_t i0 = b; i0 < e; i0 += 64 * AHEAD) {
    int key[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) key[j] = i0 + 64 * j + lane < e ? keys[i0 + 64 * j + lane] : 0;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const bool in = i0 + 64 * j + lane < e;
      const int g = group_of_key(key[j], G);
      if constexpr (!FEW) {
        if (in) add(g, 1);
      } else {
        const unsigned long long same = same_group(g, bits, __ballot(in));
        if (in && (same & ((1ull << lane) - 1)) == 0) add(g, __popcll(same));
      }
    }
  }
}
template <bool FEW> __device__ __forceinline__ void count_keys(const int32_t* __restrict__ keys, int G, int bits, int64_t b, int64_t e, unsigned int* mine) {
  count_groups<FEW>(keys, G, bits, b, e, [&](int g, int n) { atomicAdd(&mine[g >> 1], static_cast<unsigned int>(n) << (16 * (g & 1))); });
}

// Turns counts per wavefront into counts of the earlier wavefronts and calls total(g, sum) for every group.  (Of a round: two groups' sums
// fit in one word and are added up together.)
template <typename F> __device__ __forceinline__ void sum_waves(int G, unsigned int* counts, F&& total) {
  const int words = count_words(G);
  for (int i = threadIdx.x; i < words; i += THREADS) {
    unsigned int v[WAVES], sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v[w] = counts[w * words + i];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      counts[w * words + i] = sum;
      sum += v[w];
    }
    total(2 * i, static_cast<int>(sum & 0xffffu));
    if (2 * i < G) total(2 * i + 1, static_cast<int>(sum >> 16));
  }
}

// Lanes of a wavefront read and change each other's counts: what stands before this point is seen behind it.  (LDS keeps a wavefront's
// order, so this is no instruction.)
__device__ __forceinline__ void wave_meets() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// put(row, group, place) for the rows of the wavefront's run, in their order; base: first places of the groups.
template <bool FEW, typename F>
__device__ __forceinline__ void place_rows(const int32_t* __restrict__ keys, int G, int bits, int64_t b, int64_t e, const int* base,
                                           unsigned int* mine, F&& put) {
  const int lane = threadIdx.x & 63;
  auto count = [&](int g) {
    return static_cast<int>(__hip_atomic_load(&mine[g >> 1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT) >> (16 * (g & 1)) & 0xffffu);
  };
  for (int64_t i0 = b; i0 < e; i0 += 64 * AHEAD) {
    int key[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) key[j] = i0 + 64 * j + lane < e ? keys[i0 + 64 * j + lane] : 0;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int64_t i = i0 + 64 * j + lane;
      const bool in = i < e;
      const unsigned long long some = __ballot(in);
      if (!some) break;
      const int g = in ? group_of_key(key[j], G) : -1;
      // (the counts before this step, with this step's rows, and then read again)
      int earlier = 0, after = 0, before;
      if (in) earlier = count(g);
      wave_meets();
      if constexpr (FEW) {
        const unsigned long long same = same_group(g, bits, some);
        before = __popcll(same & ((1ull << lane) - 1));
        if (in && before == 0) atomicAdd(&mine[g >> 1], static_cast<unsigned int>(__popcll(same)) << (16 * (g & 1)));
      } else {
        if (in) atomicAdd(&mine[g >> 1], 1u << (16 * (g & 1)));
        wave_meets();
        if (in) after = count(g);
        before = lanes_before(g, bits, in && after - earlier > 1, some);
      }
      if (in) put(i, g, base[g] + earlier + before);
      wave_meets();
    }
  }
}

__global__ __launch_bounds__(THREADS) void group_rows_kernel(const int32_t* __restrict__ keys, int n, int G, int bits,
                                                             int32_t* __restrict__ off, int32_t* __restrict__ order) {
  extern __shared__ int shared_base[];
  __shared__ int waves[WAVES];
  unsigned int* counts = reinterpret_cast<unsigned int*>(shared_base + G + 1);
  const int words = count_words(G);
  for (int i = threadIdx.x; i < WAVES * words; i += THREADS) counts[i] = 0;
  __syncthreads();
  int64_t b, e;
  wave_run(0, n, &b, &e);
  unsigned int* mine = counts + (threadIdx.x >> 6) * words;
  count_keys<false>(keys, G, bits, b, e, mine);
  __syncthreads();
  sum_waves(G, counts, [&](int g, int sum) { shared_base[g] = sum; });
  __syncthreads();
  int first = 0;
  for (int g0 = 0; g0 <= G; g0 += THREADS) {
    const int g = g0 + threadIdx.x;
    int total;
    const int before = scan_threads(g <= G ? shared_base[g] : 0, waves, &total);
    if (g <= G) {
      shared_base[g] = first + before;
      off[g] = first + before;
    }
    first += total;
  }
  __syncthreads();
  place_rows<false>(keys, G, bits, b, e, shared_base, mine,
             [&](int64_t row, int, int place) { order[place] = static_cast<int32_t>(row); });
}

template <bool FEW> __global__ __launch_bounds__(THREADS) void group_count_kernel(const int32_t* __restrict__ keys, int64_t n, int64_t per, int G, int bits,
                                                              int32_t* __restrict__ counts) {
  extern __shared__ int hist[];
  for (int g = threadIdx.x; g <= G; g += THREADS) hist[g] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * per, end = min(begin + per, n);
  int64_t b, e;
  wave_run(begin, max(begin, end), &b, &e);
  count_groups<FEW>(keys, G, bits, b, e, [&](int g, int n) { atomicAdd(&hist[g], n); });
  __syncthreads();
  for (int g = threadIdx.x; g <= G; g += THREADS) counts[static_cast<int64_t>(blockIdx.x) * (G + 1) + g] = hist[g];
}

// counts[b][g] becomes the rows of group g in workgroups before b; totals[g] all of them.  16 groups a workgroup, the
// workgroups' counts in 64 parts.
constexpr int SUM_GROUPS = 16, SUM_PARTS = THREADS / SUM_GROUPS;
__global__ __launch_bounds__(THREADS) void group_sum_kernel(int blocks, int G, int32_t* __restrict__ counts, int32_t* __restrict__ totals) {
  __shared__ int part[SUM_PARTS][SUM_GROUPS];
  const int lane = threadIdx.x % SUM_GROUPS, p = threadIdx.x / SUM_GROUPS, g = blockIdx.x * SUM_GROUPS + lane;
  const int per = (blocks + SUM_PARTS - 1) / SUM_PARTS, b0 = min(p * per, blocks), b1 = min(b0 + per, blocks);
  int sum = 0;
  if (g <= G)
    for (int b = b0; b < b1; ++b) sum += counts[static_cast<int64_t>(b) * (G + 1) + g];
  part[p][lane] = sum;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < p; ++w) before += part[w][lane];
  if (g > G) return;
  if (p == SUM_PARTS - 1) totals[g] = before + sum;
  for (int b = b0; b < b1; ++b) {
    const int64_t at = static_cast<int64_t>(b) * (G + 1) + g;
    const int v = counts[at];
    counts[at] = before;
    before += v;
  }
}

// LDS of the sorting form: next places [G + 1], counts per wavefront, and of SORTED rows at a time their numbers and groups in sorted
// order and the groups' first places among them.
constexpr int SORTED = THREADS * AHEAD;
constexpr size_t SORTED_LDS = 156 * 1024;
constexpr size_t sorted_lds(int G) { return place_lds(G) + (static_cast<size_t>(G) + 1) * 4 + SORTED * 4; }
static_assert(sorted_lds(3173) <= SORTED_LDS && sorted_lds(3174) > SORTED_LDS, "most groups of the sorting form");
// Rows of a round of the form that does not sort.
constexpr int UNSORTED = 7 * SORTED;
static_assert(ONE_GROUP_KEYS < 65536 && SORTED < 65536 && UNSORTED < 65536, "16-bit counts of a round");

template <bool SORT, bool FEW>
__global__ __launch_bounds__(THREADS) void group_place_kernel(const int32_t* __restrict__ keys, int64_t n, int64_t per, int G, int bits,
                                                              const int32_t* __restrict__ counts, const int32_t* __restrict__ totals,
                                                              int32_t* __restrict__ off, int32_t* __restrict__ order) {
  extern __shared__ int next[];         // where a group's next row goes
  __shared__ int waves[WAVES];
  const int words = count_words(G);
  unsigned int* own = reinterpret_cast<unsigned int*>(next + G + 1);
  unsigned int* mine = own + (threadIdx.x >> 6) * words;
  int* local = reinterpret_cast<int*>(own + WAVES * words);                       // SORT: first place of a group among the SORTED rows
  unsigned short* row = reinterpret_cast<unsigned short*>(local + G + 1);         // SORT: [SORTED] row - first row of them
  unsigned short* group = row + SORTED;                                           // SORT: [SORTED]
  const int64_t begin = blockIdx.x * per, end = min(begin + per, n);
  int first = 0;
  for (int g0 = 0; g0 <= G; g0 += THREADS) {
    const int g = g0 + threadIdx.x;
    int total;
    const int before = scan_threads(g <= G ? totals[g] : 0, waves, &total);
    if (g <= G) {
      next[g] = first + before + counts[static_cast<int64_t>(blockIdx.x) * (G + 1) + g];
      if (blockIdx.x == 0) off[g] = first + before;
    }
    first += total;
  }
  constexpr int ROUND = SORT ? SORTED : UNSORTED;
  for (int64_t at = begin; at < end; at += ROUND) {
    const int64_t to = min(at + ROUND, end);
    for (int i = threadIdx.x; i < WAVES * words; i += THREADS) own[i] = 0;
    __syncthreads();
    int64_t b, e;
    wave_run(at, to, &b, &e);
    count_keys<FEW>(keys, G, bits, b, e, mine);
    __syncthreads();
    if constexpr (SORT) {
      sum_waves(G, own, [&](int g, int sum) { local[g] = sum; });
      __syncthreads();
      int before_all = 0;
      for (int g0 = 0; g0 <= G; g0 += THREADS) {
        const int g = g0 + threadIdx.x;
        int total;
        const int before = scan_threads(g <= G ? local[g] : 0, waves, &total);
        if (g <= G) local[g] = before_all + before;
        before_all += total;
      }
      __syncthreads();
      place_rows<FEW>(keys, G, bits, b, e, local, mine, [&](int64_t r, int g, int place) {
        row[place] = static_cast<unsigned short>(r - at);
        group[place] = static_cast<unsigned short>(g);
      });
      __syncthreads();
      const int here = static_cast<int>(to - at);
      for (int i = threadIdx.x; i < here; i += THREADS) {
        const int g = group[i];
        order[next[g] + i - local[g]] = static_cast<int32_t>(at) + row[i];
      }
      __syncthreads();
      for (int g = threadIdx.x; g <= G; g += THREADS) next[g] += (g < G ? local[g + 1] : here) - local[g];
    } else {
      sum_waves(G, own, [](int, int) {});
      __syncthreads();
      place_rows<FEW>(keys, G, bits, b, e, next, mine,
                 [&](int64_t r, int, int place) { order[place] = static_cast<int32_t>(r); });
      __syncthreads();
      // (the last wavefront's counts are those of the whole round by now)
      for (int g = threadIdx.x; g <= G; g += THREADS) next[g] += (own[(WAVES - 1) * words + (g >> 1)] >> (16 * (g & 1))) & 0xffffu;
      __syncthreads();
    }
  }
}

// Keys and number of workgroups of the three-launch form: 256 workgroups (one a compute unit), of at least 1,024 keys (of 8,192:
// 200,000 keys in 64 groups 20.5 us instead of 14.3, 36,080 in 16 19.7 instead of 12.3), a whole number of rounds of SORTED where
// that is more than one, and at most 512K keys each.
constexpr int LEAST = 1024;
void split(int64_t n, int64_t* per, int* blocks) {
  int64_t p = (n + 255) / 256;
  const int64_t unit = p > SORTED ? SORTED : LEAST;
  p = std::min<int64_t>((p + unit - 1) / unit * unit, 1 << 19);
  *per = p;
  *blocks = static_cast<int>((n + p - 1) / p);
}

// Marks bit 0 where a key is G or more.
__global__ void check_keys_kernel(const int32_t* __restrict__ keys, int64_t n, int G, int32_t* flag) {
  bool bad = false;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x)
    bad |= keys[i] >= G;
  if (bad) atomicOr(flag, 1);
}

// Marks bit 0 where the offsets do not ascend from 0 to at most n, and bit 1 where an entry of order is outside [0, n).
__global__ void check_groups_kernel(lq_groups g, int32_t* flag) {
  const int64_t i0 = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * blockDim.x;
  int bad = 0;
  for (int64_t i = i0; i <= g.n_groups; i += step) {
    const int v = g.offsets[i];
    if (v > g.n || (i == 0 ? v != 0 : v < g.offsets[i - 1])) bad |= 1;
  }
  if (g.order)
    for (int64_t i = i0; i < g.n; i += step)
      if (static_cast<uint32_t>(g.order[i]) >= static_cast<uint64_t>(g.n)) bad |= 2;
  if (bad) atomicOr(flag, bad);
}
__global__ void clear_flag_kernel(int32_t* flag) { *flag = 0; }

}  // namespace

size_t group_rows_ws_bytes(int64_t n, int32_t G) {
  if (n <= ONE_GROUP_KEYS) return 0;
  int64_t per;
  int blocks;
  split(n, &per, &blocks);
  return round_up((static_cast<size_t>(blocks) + 1) * (G + 1) * 4, 256);
}

int launch_group_rows(const int32_t* keys, int64_t n, int32_t G, int32_t* off, int32_t* order, void* ws, hipStream_t s) {
  int bits = 0;
  while ((G >> bits) > 0) ++bits;
  const size_t lds = place_lds(G);
  if (n <= ONE_GROUP_KEYS) {
    if (lds > 64 * 1024)
      LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&group_rows_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(lds)));
    group_rows_kernel<<<1, THREADS, lds, s>>>(keys, static_cast<int>(n), G, bits, off, order);
    LQ_LAUNCH_CHECK("group_rows_kernel");
    return LQ_OK;
  }
  int64_t per;
  int blocks;
  split(n, &per, &blocks);
  int32_t* counts = static_cast<int32_t*>(ws);
  int32_t* totals = counts + static_cast<int64_t>(blocks) * (G + 1);
  const bool few = bits <= FEW_BITS;
  (few ? group_count_kernel<true> : group_count_kernel<false>)<<<blocks, THREADS, (G + 1) * 4, s>>>(keys, n, per, G, bits, counts);
  LQ_LAUNCH_CHECK("group_count_kernel");
  group_sum_kernel<<<G / SUM_GROUPS + 1, THREADS, 0, s>>>(blocks, G, counts, totals);
  LQ_LAUNCH_CHECK("group_sum_kernel");
  const bool sort = sorted_lds(G) <= SORTED_LDS;
  const size_t bytes = sort ? sorted_lds(G) : lds;
  const auto kernel = few ? group_place_kernel<true, true> : sort ? group_place_kernel<true, false> : group_place_kernel<false, false>;
  if (bytes > 64 * 1024)
    LQ_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
  kernel<<<blocks, THREADS, bytes, s>>>(keys, n, per, G, bits, counts, totals, off, order);
  LQ_LAUNCH_CHECK("group_place_kernel");
  return LQ_OK;
}

int launch_check_keys(const int32_t* keys, int64_t n, int32_t G, int32_t* flag, hipStream_t s) {
  clear_flag_kernel<<<1, 1, 0, s>>>(flag);
  LQ_LAUNCH_CHECK("clear_flag_kernel");
  const int blocks = static_cast<int>(std::min<int64_t>((n + 255) / 256, 2048));
  check_keys_kernel<<<std::max(blocks, 1), 256, 0, s>>>(keys, n, G, flag);
  LQ_LAUNCH_CHECK("check_keys_kernel");
  return LQ_OK;
}

int launch_check_groups(const lq_groups& g, int32_t* flag, hipStream_t s) {
  clear_flag_kernel<<<1, 1, 0, s>>>(flag);
  LQ_LAUNCH_CHECK("clear_flag_kernel");
  const int blocks = static_cast<int>(std::min<int64_t>((std::max<int64_t>(g.n, g.n_groups) + 256) / 256, 2048));
  check_groups_kernel<<<blocks, 256, 0, s>>>(g, flag);
  LQ_LAUNCH_CHECK("check_groups_kernel");
  return LQ_OK;
}

}  // namespace lq
