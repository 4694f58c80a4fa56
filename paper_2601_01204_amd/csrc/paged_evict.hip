// Eviction by received weight: every (sequence, key head) whose cache is over the budget keeps `budget` tokens.
//
// select_kernel, one workgroup per (sequence, key head).  Weights become 32-bit keys in the same order (NaN below -infinity, tokens
// whose page is missing below that; protected tokens above everything), and the budget-th largest key is found digit by digit
// (11, 11 and 10 bits: 11 bits take sign, exponent and two bits of the mantissa, so that weights of a few orders of magnitude spread over
// dozens of counters).  Where a few tokens leave (decoding: one), they are found as the least keys instead.  Among equal keys the lower slots stay.  Then every wave walks a contiguous part of the slots: slots below the
// budget that lose their token and tokens behind it that stay are numbered in ascending order by ballots, and the i-th of the
// ones receives the i-th of the others.  Sources lie behind the budget and destinations before it, so the moves are free of
// order.
//
// Bound by latency: a chain of dependent loads (lengths, page, ids and weights) and the counting's barriers; 256 caches of 4097 tokens that give up one
// token each take 14 us, sixteen of 18432 that keep 8192 28 us and their moves (80 MB read and written) 18 us, 4.4 TB/s.
//
// move_kernel copies the rows.  A launch that can move few rows only has the selecting workgroup copy them itself.
#include "../../include/kvx.h"
#include "paged_types.h"

#include <type_traits>

namespace kvx {
namespace paged {

namespace {

constexpr int kThreads = kSelectThreads, kWaves = kThreads / 64;
constexpr uint32_t kProtected = 0xFFFFFFFFu;
constexpr int kFewLeave = 4;                    // tokens that leave by looking for the least: a pass each, where the digits take three longer ones

__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, int32_t id, float w, int seen) {
  if (id < a.sinks || id >= seen - a.recent) return kProtected;
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
    const uint64_t src = slot_offset(c, from, m.x & mask) + head_offset(c, head) + 16 * chunk;
    const uint64_t dst = slot_offset(c, to, m.y & mask) + head_offset(c, head) + 16 * chunk;
    const u32x4 k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(c.k + src)), v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(c.v + src));
    *reinterpret_cast<u32x4*>(c.k + dst) = k;
    *reinterpret_cast<u32x4*>(c.v + dst) = v;
    if (chunk == 0) {
      const int64_t ws = (((int64_t)from * c.hkv + head) << c.page_shift) + (m.x & mask), wd = (((int64_t)to * c.hkv + head) << c.page_shift) + (m.y & mask);
      a.weights_out[wd] = c.weights[ws];
      a.ids_out[wd] = c.ids[ws];
    }
  }
}

// Sums over the waves of a workgroup in front of this one, of two counts that every wave brings; totals too.
struct Counts {
  int x, y;
};
__device__ __forceinline__ Counts before_me(Counts mine, int wave, int2* sums, Counts* total = nullptr) {
  __syncthreads();                              // the last use of sums is over
  if ((threadIdx.x & 63) == 0) sums[wave] = make_int2(mine.x, mine.y);
  __syncthreads();
  int2 all[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) all[i] = sums[i];
  Counts before{0, 0}, sum{0, 0};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    before.x += i < wave ? all[i].x : 0;
    before.y += i < wave ? all[i].y : 0;
    sum.x += all[i].x;
    sum.y += all[i].y;
  }
  if (total) *total = sum;
  return before;
}

// A thread has groups of four neighbouring slots (pages begin on a multiple of eight).  NIT > 0: the keys of its NIT groups stay in its
// registers, up to kHold groups with the weights and ids they come from; NIT = 0: caches of any length, whose keys are formed again in
// every pass.
constexpr int kHold = 4;

template <int ROW_BYTES, int NIT>
__global__ __launch_bounds__(kThreads) void select_kernel(const EvictArgs a, const bool move_here, int32_t* const arrived) {
  constexpr bool kKeep = NIT > 0 && NIT <= kHold;
  constexpr int kRegs = NIT > 0 ? NIT : 1;
  __shared__ __align__(16) int hist[2048];
  __shared__ __align__(16) int2 sums[kWaves];
  __shared__ int found[3];
  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % c.hkv, b = blockIdx.x / c.hkv;
  const Seq s = sequence(c, b);
  const int len = s.len, budget = a.budget, seen = c.seen[b], mask = (1 << c.page_shift) - 1;
  const bool over = len > budget, in_place = a.weights_out == c.weights && a.ids_out == c.ids;
  int2* const moves = a.moves + (int64_t)blockIdx.x * a.max_moves;
  // a wave has a contiguous part of the slots, 256 at a time (short caches: of all that the launch provides for, so that the page table can be
  // read before the length is there)
  const int its = NIT == 1 || NIT == 2 ? NIT : (len + 4 * kThreads - 1) / (4 * kThreads), part = its * 256, j0 = wave * part, j1 = min(len, j0 + part);

  struct Group {
    int32_t page;
    int32_t id[4];
    float w[4];
  };
  auto slot_of = [&](int it) { return j0 + 256 * it + 4 * lane; };
  auto index_of = [&](int32_t page, int j) { return (((int64_t)page * c.hkv + head) << c.page_shift) + (j & mask); };
  auto load_page = [&](Group& g, int it) { g.page = slot_of(it) < c.max_len ? page_of(c, b, slot_of(it) >> c.page_shift) : -1; };
  auto load_rest = [&](Group& g, int it) {
    int4 i4 = make_int4(0, 0, 0, 0);
    float4 w4 = make_float4(0.f, 0.f, 0.f, 0.f);
    if (g.page >= 0 && slot_of(it) < j1) {
      const int64_t at = index_of(g.page, slot_of(it));
      i4 = *reinterpret_cast<const int4*>(c.ids + at);
      w4 = *reinterpret_cast<const float4*>(c.weights + at);
    }
    g.id[0] = i4.x; g.id[1] = i4.y; g.id[2] = i4.z; g.id[3] = i4.w;
    g.w[0] = w4.x; g.w[1] = w4.y; g.w[2] = w4.z; g.w[3] = w4.w;
  };
  auto form_keys = [&](const Group& g, int it, uint32_t (&k)[4]) {
    if (slot_of(it) < j1 && g.page < 0) note_bad_page(c);
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = g.page >= 0 ? key_of(a, g.id[e], g.w[e], seen) : 0u;
  };
  // the slots of `wanted` (a bit each of a group's four) go to weights_out and ids_out
  auto store = [&](const Group& g, int it, uint32_t wanted) {
    if (g.page < 0 || !wanted) return;
    const int64_t at = index_of(g.page, slot_of(it));
    if (wanted == 15u) {
      *reinterpret_cast<int4*>(a.ids_out + at) = make_int4(g.id[0], g.id[1], g.id[2], g.id[3]);
      *reinterpret_cast<float4*>(a.weights_out + at) = make_float4(g.w[0], g.w[1], g.w[2], g.w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((wanted >> e) & 1) {
          a.ids_out[at + e] = g.id[e];
          a.weights_out[at + e] = g.w[e];
        }
    }
  };

  uint32_t key[kRegs][4];
  Group held[kKeep ? kRegs : 1];
  if constexpr (kKeep) {
    // every load of a kind is on its way before the first is used
#pragma unroll
    for (int i = 0; i < NIT; ++i) load_page(held[i], i);
#pragma unroll
    for (int i = 0; i < NIT; ++i) load_rest(held[i], i);
#pragma unroll
    for (int i = 0; i < NIT; ++i) form_keys(held[i], i, key[i]);
  } else if constexpr (NIT > 0) {
#pragma unroll
    for (int base = 0; base < NIT; base += 4) {
      Group g[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) load_page(g[i], base + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) load_rest(g[i], base + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) form_keys(g[i], base + i, key[base + i]);
    }
  }
  // f(group number, first slot, keys); all lanes of a wave together, slots from j1 on are nobody's
  auto each = [&](auto&& f) {
    if constexpr (NIT > 0) {
#pragma unroll
      for (int i = 0; i < NIT; ++i)
        if (i < its) f(i, slot_of(i), key[i]);
    } else {
      for (int i = 0; i < its; ++i) {
        Group g;
        load_page(g, i);
        load_rest(g, i);
        uint32_t k[4];
        form_keys(g, i, k);
        f(i, slot_of(i), k);
      }
    }
  };
  // bit 4 i + e of `wanted`: slot e of group from + i
  auto carry = [&](uint32_t wanted, int from) {
    if constexpr (kKeep) {
#pragma unroll
      for (int i = 0; i < NIT; ++i) store(held[i], i, (wanted >> (4 * i)) & 15u);
    } else {
#pragma unroll
      for (int base = 0; base < 8; base += 4) {
        if (from + base >= its) break;
        Group g[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[i].page = -1;
          if ((wanted >> (4 * (base + i))) & 15u) load_page(g[i], from + base + i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) load_rest(g[i], from + base + i);
#pragma unroll
        for (int i = 0; i < 4; ++i) store(g[i], from + base + i, (wanted >> (4 * (base + i))) & 15u);
      }
    }
  };
  auto flush = [&](int i, uint32_t& wanted) {   // NIT = 0: after every eighth group and the last
    if constexpr (NIT == 0) {
      if ((i & 7) == 7 || i == its - 1) {
        carry(wanted, i & ~7);
        wanted = 0;
      }
    }
  };
  // The new length is written by the sequence's last workgroup to get here: lens_out may be the lengths that all of them have read.
  // Every wave's load of the length has returned before the barriers in front of this, so the count needs no fence of its own
  // (one of device scope writes the cache back: 256 workgroups took 25.8 us with it, 18.8 without).
  auto arrive = [&]() {
    if (threadIdx.x == 0) {
      if (atomicAdd(&arrived[b], 1) == c.hkv - 1) {
        arrived[b] = 0;
        a.lens_out[b] = over ? budget : len;
      }
    }
  };
  uint32_t wanted = 0;
  if (!over) {
    each([&](int i, int j, const uint32_t (&)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) wanted |= j + e < j1 && !in_place ? 1u << (4 * (i & 7) + e) : 0u;
      flush(i, wanted);
    });
    if constexpr (NIT > 0) carry(wanted, 0);
    if (threadIdx.x == 0) a.n_moves[blockIdx.x] = 0;
    __syncthreads();                            // every wave has read the length
    arrive();
    return;
  }

  // the key at which the staying ones end, and how many of those equal to it stay
  uint32_t prefix = 0;
  int want = budget;
  if (len - budget <= kFewLeave) {
    // few leave: the least keys one after the other, each with its count
    uint32_t least = 0;                         // keys below it have been counted
    for (int leave = len - budget;;) {
      uint32_t low = kProtected;
      int count = 0;
      each([&](int, int j, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < j1 && k[e] >= least) {
            count = k[e] < low ? 1 : count + (k[e] == low);
            low = min(low, k[e]);
          }
      });
      auto join = [&](uint32_t l, int n) {
        count = l < low ? n : count + (l == low ? n : 0);
        low = min(low, l);
      };
#pragma unroll
      for (int o = 32; o; o >>= 1) join((uint32_t)__shfl_xor((int)low, o), __shfl_xor(count, o));
      __syncthreads();                          // the last use of sums is over
      if (lane == 0) sums[wave] = make_int2((int)low, count);
      __syncthreads();
      low = kProtected;
      count = 0;
      int2 all[kWaves];
#pragma unroll
      for (int i = 0; i < kWaves; ++i) all[i] = sums[i];
#pragma unroll
      for (int i = 0; i < kWaves; ++i) join((uint32_t)all[i].x, all[i].y);
      if (count >= leave || low == kProtected) {
        prefix = low;
        want = max(0, count - leave);
        if (threadIdx.x == 0) found[2] = count;
        break;
      }
      leave -= count;
      least = low + 1;
    }
    __syncthreads();
  } else {
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
    const uint32_t above = pass == 0 ? 0u : (pass == 1 ? 0xFFE00000u : 0xFFFFFC00u);
    *reinterpret_cast<int2*>(&hist[2 * threadIdx.x]) = make_int2(0, 0);
    __syncthreads();
    each([&](int, int j, const uint32_t (&k)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < j1 && (k[e] & above) == prefix) atomicAdd(&hist[(k[e] >> shift) & (bins - 1)], 1);
    });
    __syncthreads();
    // from the largest digit down: thread t has digits 2047 - 2 t and the one below
    const int d0 = 2047 - 2 * (int)threadIdx.x;
    const int2 n = *reinterpret_cast<const int2*>(&hist[d0 - 1]);
    const int n0 = n.y, n1 = n.x;
    int upto = n0 + n1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const int before = before_me({__shfl(upto, 63), 0}, wave, sums).x + upto - n0 - n1;
    if (before < want && before + n0 >= want) {
      found[0] = d0;
      found[1] = want - before;
      found[2] = n0;
    } else if (before + n0 < want && before + n0 + n1 >= want) {
      found[0] = d0 - 1;
      found[1] = want - before - n0;
      found[2] = n1;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    want = found[1];                            // (read before the next pass's first barrier, written behind its second)
  }
  }
  const bool ranked = want < found[2];          // not all of the equal ones stay

  // of a count of 0..4 in every lane: the sum over the lanes below, and over all
  const uint64_t below = (1ull << lane) - 1;
  auto lanes_below = [&](int n, int& all) {
    const uint64_t b0 = __ballot(n & 1), b1 = __ballot(n & 2), b2 = __ballot(n & 4);
    all = __popcll(b0) + 2 * __popcll(b1) + 4 * __popcll(b2);
    return __popcll(b0 & below) + 2 * __popcll(b1 & below) + 4 * __popcll(b2 & below);
  };
  int ties_before = 0;
  if (ranked) {
    int ties = 0;
    each([&](int, int j, const uint32_t (&k)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) ties += __popcll(__ballot(j + e < j1 && k[e] == prefix));
    });
    ties_before = before_me({ties, 0}, wave, sums).x;
  }
  // f(group number, first slot, which of the four slots stay (a bit each))
  auto walk = [&](auto&& f) {
    int tie = ties_before;
    each([&](int i, int j, const uint32_t (&k)[4]) {
      uint32_t stay = 0, same = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        stay |= j + e < j1 && k[e] > prefix ? 1u << e : 0u;
        same |= j + e < j1 && k[e] == prefix ? 1u << e : 0u;
      }
      if (ranked) {
        int all;
        int rank = tie + lanes_below(__popc(same), all);
        tie += all;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((same >> e) & 1) stay |= rank++ < want ? 1u << e : 0u;
      } else {
        stay |= same;
      }
      f(i, j, stay);
    });
  };
  auto real_of = [&](int j) { return j >= j1 ? 0u : (j1 - j >= 4 ? 15u : (1u << (j1 - j)) - 1u); };
  auto in_budget = [&](int j) { return j >= budget ? 0u : (budget - j >= 4 ? 15u : (1u << (budget - j)) - 1u); };
  int holes = 0, movers = 0;                    // of this lane
  walk([&](int, int j, uint32_t stay) {
    holes += __popc(real_of(j) & ~stay & in_budget(j));
    movers += __popc(stay & ~in_budget(j));
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    holes += __shfl_xor(holes, o);
    movers += __shfl_xor(movers, o);
  }
  Counts total;
  const Counts first = before_me({holes, movers}, wave, sums, &total);
  const int n_moves = total.x;                  // as many tokens behind the budget stay as tokens before it leave
  int hole = first.x, mover = first.y;
  walk([&](int i, int j, uint32_t stay) {
    const uint32_t lose = real_of(j) & ~stay & in_budget(j), move = stay & ~in_budget(j);
    if (__ballot(lose != 0)) {
      int all;
      int at = hole + lanes_below(__popc(lose), all);
      hole += all;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((lose >> e) & 1) moves[at++].y = j + e;
    }
    if (__ballot(move != 0)) {
      int all;
      int at = mover + lanes_below(__popc(move), all);
      mover += all;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((move >> e) & 1) moves[at++].x = j + e;
    }
    wanted |= in_place ? 0u : (stay & in_budget(j)) << (4 * (i & 7));
    flush(i, wanted);
  });
  if constexpr (NIT > 0) carry(wanted, 0);
  if (threadIdx.x == 0) a.n_moves[blockIdx.x] = n_moves;
  arrive();
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
  const bool here = a.max_moves <= kFewMoves;
  auto go = [&](auto rb) {
    constexpr int kRB = decltype(rb)::value;
    const dim3 grid((unsigned)select_grid(a).x), block(kThreads);
    if (a.c.max_len <= 4 * kThreads) select_kernel<kRB, 1><<<grid, block, 0, st>>>(a, here, arrived);
    else if (a.c.max_len <= 8 * kThreads) select_kernel<kRB, 2><<<grid, block, 0, st>>>(a, here, arrived);
    else if (a.c.max_len <= 16 * kThreads) select_kernel<kRB, kHold><<<grid, block, 0, st>>>(a, here, arrived);
    else if (a.c.max_len <= 32 * kThreads) select_kernel<kRB, 8><<<grid, block, 0, st>>>(a, here, arrived);
    else select_kernel<kRB, 0><<<grid, block, 0, st>>>(a, here, arrived);
    if (!here) {
      const int rows = 256 / (kRB / 16);
      int parts = (a.max_moves + 2 * rows - 1) / (2 * rows);          // two rows a lane group where every move happens
      if ((int64_t)parts * jobs > (1 << 20)) parts = (1 << 20) / jobs > 0 ? (1 << 20) / jobs : 1;
      move_kernel<kRB><<<dim3((unsigned)(parts * jobs)), dim3(256), 0, st>>>(a, parts);
    }
  };
  const int rb = d * (e4m3 ? 1 : 2);
  if (rb == 256) go(std::integral_constant<int, 256>{});
  else if (rb == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 64>{});
}

}  // namespace paged
}  // namespace kvx
