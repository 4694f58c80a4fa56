// Eviction by received weight: every (sequence, key head) whose cache is over the budget keeps `budget` tokens.
//
// select_kernel, one workgroup per (sequence, key head).  Weights become 32-bit keys in the same order (NaN below -infinity, tokens
// whose page is missing below that; protected tokens above everything), and the budget-th largest key is found digit by digit
// (11, 11 and 10 bits: 11 bits take sign, exponent and two bits of the mantissa, so that weights of a few orders of magnitude spread over
// dozens of counters).  Among equal keys the lower slots stay.  Then every wave walks a contiguous part of the slots: slots below the
// budget that lose their token and tokens behind it that stay are numbered in ascending order by ballots, and the i-th of the
// ones receives the i-th of the others.  Sources lie behind the budget and destinations before it, so the moves are free of
// order.
//
// move_kernel copies the rows.  A launch that can move few rows only has the selecting workgroup copy them itself.
#include "../../include/kvx.h"
#include "paged_types.h"

#include <type_traits>

namespace kvx {
namespace paged {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kLdsKeys = 32768;                 // longer caches read their keys again in every pass
constexpr uint32_t kProtected = 0xFFFFFFFFu;
constexpr int kFewMoves = 256;

// Index of slot j in weights and ids; -1: no page.
__device__ __forceinline__ int64_t meta_index(const Call& c, int b, int head, int j) {
  const int32_t page = page_of(c, b, j >> c.page_shift);
  return page < 0 ? -1 : (((int64_t)page * c.hkv + head) << c.page_shift) + (j & ((1 << c.page_shift) - 1));
}
__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, int64_t at, int seen) {
  if (at < 0) return 0u;
  const int32_t id = a.c.ids[at];
  if (id < a.sinks || id >= seen - a.recent) return kProtected;
  const float w = a.c.weights[at];
  if (w != w) return 1u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);            // the two zeros are one weight
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);                 // -infinity: 0x007FFFFF, +infinity: 0xFF800000
}

// A row of keys or values: lanes of a row copy 16 bytes each.
template <int ROW_BYTES>
__device__ __forceinline__ void move_rows(const EvictArgs& a, int b, int head, const int2* moves, int n, int first, int step) {
  constexpr int kLPR = ROW_BYTES / 16;
  const Call& c = a.c;
  const int mask = (1 << c.page_shift) - 1, chunk = threadIdx.x % kLPR;
  for (int i = first + (int)threadIdx.x / kLPR; i < n; i += step) {
    const int2 m = moves[i];
    const int32_t from = page_of(c, b, m.x >> c.page_shift), to = page_of(c, b, m.y >> c.page_shift);
    if (from < 0 || to < 0) continue;                                // (a token without a page never stays unless the budget asks for it)
    const int64_t src = from * c.page_stride + (m.x & mask) * c.slot_stride + head * c.head_stride + 16 * chunk;
    const int64_t dst = to * c.page_stride + (m.y & mask) * c.slot_stride + head * c.head_stride + 16 * chunk;
    const u32x4 k = *reinterpret_cast<const u32x4*>(c.k + src), v = *reinterpret_cast<const u32x4*>(c.v + src);
    *reinterpret_cast<u32x4*>(c.k + dst) = k;
    *reinterpret_cast<u32x4*>(c.v + dst) = v;
    if (chunk == 0) {
      const int64_t ws = (((int64_t)from * c.hkv + head) << c.page_shift) + (m.x & mask), wd = (((int64_t)to * c.hkv + head) << c.page_shift) + (m.y & mask);
      a.weights_out[wd] = c.weights[ws];
      a.ids_out[wd] = c.ids[ws];
    }
  }
}

// Sum over the waves of a workgroup in front of this one, and the total; every wave brings `mine`.
__device__ __forceinline__ int before_me(int mine, int wave, int* sums, int& total) {
  __syncthreads();                              // the last use of sums is over
  if ((threadIdx.x & 63) == 0) sums[wave] = mine;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < kWaves; ++i) {
    const int x = sums[i];
    before += i < wave ? x : 0;
    total += x;
  }
  return before;
}

template <int ROW_BYTES>
__global__ __launch_bounds__(kThreads) void select_kernel(const EvictArgs a, const int lds_keys, const bool move_here, int32_t* const arrived) {
  extern __shared__ uint32_t keys[];            // [lds_keys]
  __shared__ int hist[2048];
  __shared__ int sums[kWaves];
  __shared__ int found[2];
  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % c.hkv, b = blockIdx.x / c.hkv;
  const Seq s = sequence(c, b);
  const int len = s.len, budget = a.budget, seen = c.seen[b];
  const bool over = len > budget;
  // the new length is written by the sequence's last workgroup to get here: lens_out may be the lengths that all of them read
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&arrived[b], 1) == c.hkv - 1) {
      arrived[b] = 0;
      a.lens_out[b] = over ? budget : len;
    }
  }
  int2* const moves = a.moves + (int64_t)blockIdx.x * a.max_moves;
  if (!over) {
    for (int j = threadIdx.x; j < len; j += kThreads) {
      const int64_t at = meta_index(c, b, head, j);
      if (at < 0) {
        note_bad_page(c);
      } else {
        a.weights_out[at] = c.weights[at];
        a.ids_out[at] = c.ids[at];
      }
    }
    if (threadIdx.x == 0) a.n_moves[blockIdx.x] = 0;
    return;
  }
  const bool in_lds = len <= lds_keys;
  if (in_lds)
    for (int j = threadIdx.x; j < len; j += kThreads) keys[j] = key_of(a, meta_index(c, b, head, j), seen);
  auto key_at = [&](int j) { return in_lds ? keys[j] : key_of(a, meta_index(c, b, head, j), seen); };

  // the budget-th largest key, and how many of those equal to it stay
  uint32_t prefix = 0;
  int want = budget;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
    const uint32_t above = pass == 0 ? 0u : (pass == 1 ? 0xFFE00000u : 0xFFFFFC00u);
    for (int i = threadIdx.x; i < 2048; i += kThreads) hist[i] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < len; j += kThreads) {
      const uint32_t k = key_at(j);
      if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // from the largest digit down: thread t has digits bins - 1 - 2 t and the next one
    const int d0 = 2047 - 2 * (int)threadIdx.x, n0 = hist[d0], n1 = hist[d0 - 1];
    int upto = n0 + n1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    int total;
    const int before = before_me(__shfl(upto, 63), wave, sums, total) + upto - n0 - n1;
    if (before < want && before + n0 >= want) {
      found[0] = d0;
      found[1] = want - before;
    } else if (before + n0 < want && before + n0 + n1 >= want) {
      found[0] = d0 - 1;
      found[1] = want - before - n0;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    want = found[1];
    __syncthreads();
  }

  // contiguous parts of the slots, a multiple of 64 each
  const int part = ((len + kThreads - 1) / kThreads) * 64, j0 = min(len, wave * part), j1 = min(len, j0 + part);
  int ties = 0;
  for (int j = j0; j < j1; j += 64) ties += __popcll(__ballot(j + lane < j1 && key_at(j + lane) == prefix));
  int total;
  const int ties_before = before_me(ties, wave, sums, total);
  auto walk = [&](auto&& each) {
    int tie = ties_before;
    for (int j = j0; j < j1; j += 64) {
      const bool real = j + lane < j1;
      const uint32_t k = real ? key_at(j + lane) : 0u;
      const uint64_t same = __ballot(real && k == prefix);
      const int rank = tie + __popcll(same & ((1ull << lane) - 1));
      tie += __popcll(same);
      const bool stays = real && (k > prefix || (k == prefix && rank < want));
      each(j + lane, real, stays);
    }
  };
  int holes = 0, movers = 0;
  walk([&](int j, bool real, bool stays) {
    holes += __popcll(__ballot(real && !stays && j < budget));
    movers += __popcll(__ballot(stays && j >= budget));
  });
  int n_moves;
  int hole = before_me(holes, wave, sums, n_moves);
  int mover = before_me(movers, wave, sums, total);
  walk([&](int j, bool real, bool stays) {
    const bool is_hole = real && !stays && j < budget, is_mover = stays && j >= budget;
    const uint64_t hm = __ballot(is_hole), mm = __ballot(is_mover), below = (1ull << lane) - 1;
    if (is_hole) moves[hole + __popcll(hm & below)].y = j;
    if (is_mover) moves[mover + __popcll(mm & below)].x = j;
    hole += __popcll(hm);
    mover += __popcll(mm);
    if (real) {
      const int64_t at = meta_index(c, b, head, j);
      if (at < 0) {
        note_bad_page(c);
      } else if (stays && j < budget) {
        a.weights_out[at] = c.weights[at];
        a.ids_out[at] = c.ids[at];
      }
    }
  });
  if (threadIdx.x == 0) a.n_moves[blockIdx.x] = n_moves;
  if (!move_here) return;
  __syncthreads();                              // the moves are this workgroup's own
  move_rows<ROW_BYTES>(a, b, head, moves, n_moves, 0, kThreads / (ROW_BYTES / 16));
}

template <int ROW_BYTES>
__global__ __launch_bounds__(256) void move_kernel(const EvictArgs a, const int parts) {
  const int job = blockIdx.x / parts, part = blockIdx.x - job * parts;
  const int head = job % a.c.hkv, b = job / a.c.hkv;
  constexpr int kRows = 256 / (ROW_BYTES / 16);
  move_rows<ROW_BYTES>(a, b, head, a.moves + (int64_t)job * a.max_moves, a.n_moves[job], part * kRows, parts * kRows);
}

}  // namespace

void launch_evict(const EvictArgs& a, int d, bool e4m3, int32_t* arrived, hipStream_t st) {
  const int jobs = a.c.n_seqs * a.c.hkv;
  const int lds_keys = a.c.max_len < kLdsKeys ? a.c.max_len : kLdsKeys;
  const bool here = a.max_moves <= kFewMoves;
  auto go = [&](auto rb) {
    constexpr int kRB = decltype(rb)::value;
    select_kernel<kRB><<<dim3((unsigned)jobs), dim3(kThreads), (size_t)lds_keys * 4, st>>>(a, lds_keys, here, arrived);
    if (!here) {
      const int rows = 256 / (kRB / 16);
      int parts = (a.max_moves + 4 * rows - 1) / (4 * rows);          // four rows a lane group where every move happens
      if ((int64_t)parts * jobs > (1 << 20)) parts = (1 << 20) / jobs > 0 ? (1 << 20) / jobs : 1;
      move_kernel<kRB><<<dim3((unsigned)(parts * jobs)), dim3(256), 0, st>>>(a, parts);
    }
  };
  const int rb = d * (e4m3 ? 1 : 2);
  if (rb == 256) go(std::integral_constant<int, 256>{});
  else if (rb == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 64>{});
}

hipError_t prepare_evict() {
  // 128 KB of keys are more than a workgroup gets unasked
  for (const void* f : {(const void*)select_kernel<256>, (const void*)select_kernel<128>, (const void*)select_kernel<64>}) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsKeys * 4);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace paged
}  // namespace kvx
