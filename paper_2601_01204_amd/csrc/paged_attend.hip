// Attention of new tokens over a paged cache.
//
// Rows of one key head (new tokens x heads of the group) are cut into tiles, the keys of a tile into ranges; a workgroup takes one
// range of one tile.  Tiles of up to 32 rows (decoding) belong to attend_few_kernel, larger ones to attend_chunk_kernel.  With more than
// one range, workgroups leave partial results and merge_kernel joins them.
#include "../../include/kvx.h"
#include "paged_tile.h"

namespace kvx {
namespace paged {

namespace {

constexpr float kLn2 = 0.69314718055994531f;

// Result of a row: o channels (4 at `ch`), final or partial.
template <typename T>
__device__ __forceinline__ void store_out(const AttendArgs& a, int token, int head, int ch, const float (&x)[4]) {
  *reinterpret_cast<u32x2*>(a.out.p + (int64_t)token * a.out.tok + (int64_t)head * a.out.head + 2 * ch) =
      (u32x2){T::pack(x[0], x[1]), T::pack(x[2], x[3])};
}
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2; }

// ---- up to 32 rows: four waves, each with units of its own --------------------------------------------------------
// Bound by memory: every key and value is read once, past the caches.  A wave works on every fourth 32 keys, brings them through
// registers into its own part of LDS and holds the next loads in flight meanwhile (16 KB a wave, 8 waves a compute unit); no wave waits
// for another before the end, where the four waves' statistics and outputs are joined through the same LDS.
//
// A workgroup costs some 5 us besides its keys, so as many as the chip holds at a time (workers) share the keys of all columns evenly,
// whatever the sequences' lengths: a worker's share ends inside a column, and merge_kernel joins the pieces.  Against ranges of
// equal length, several to a slot, us: 64 sequences of up to 8192 tokens 207 -> 186, four of 131072 in 8 bits 215 -> 171 (1.07 GB
// each: 5.8 and 6.3 TB/s, where a loop that only reads reaches 6.2, and 7.0 past the caches).  128 keys of a wave's products and exponentials take
// 7 to 14 % of the matrix cores' time: nothing but the loads in flight counts.  Rows 17 to 32 of d = 128 in 16 bits need more registers than there are (140 bytes a
// lane go to memory): 32 sequences of 4096, 8 key heads: 101 us at 16 rows a key head, 124 at 32.
template <typename T, int D, bool E4M3, int ROWS>
__global__ __launch_bounds__(256, 2) void attend_few_kernel(const AttendArgs a) {
  typedef Shape<D, E4M3> S;
  typedef FewRows<T, D, E4M3, ROWS> W;
  constexpr int kRB = S::kRowBytes, kLPR = S::kLanesPerRow;
  constexpr int kLoads = 32 * kLPR / 64;                     // 16-byte loads of a lane for 32 rows
  constexpr int kWaveBytes = 64 * kRB;
  constexpr int kJoinBytes = ROWS * D * 4;
  __shared__ __align__(16) uint8_t lds[4 * (kWaveBytes > kJoinBytes ? kWaveBytes : kJoinBytes)];
  __shared__ float2 stats[4][ROWS];

  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), my_row = lane % ROWS, j = lane / ROWS;
  uint8_t* const lk = lds + wave * kWaveBytes;
  uint8_t* const lv = lk + 32 * kRB;
  const int ld_row = lane / kLPR * kLoads, ld_chunk = lane % kLPR;

  int unit = 0, unit_end = 1;                                // this workgroup's units; without workers: one column, whatever it holds
  Lanes lanes;
  if (a.workers) {
    lanes = load_lanes(a, 0, 0);
    int total = lanes.all;
    for (int base = 64; base < c.n_seqs; base += 64) total += load_lanes(a, base, 0).all;
    total *= c.hkv;
    const int share = share_of(a, total);
    unit = uniform(blockIdx.x * share);
    unit_end = uniform(min(total, unit + share));
  }
  while (unit < unit_end) {
    Column col;
    if (a.workers) {
      col = column_of(a, unit, lanes);
    } else {
      col.b = blockIdx.x / c.hkv;
      col.head = blockIdx.x - col.b * c.hkv;
      col.s = sequence(c, col.b);
      col.first = 0;
      col.units = 1;
    }
    const int b = uniform(col.b), head = uniform(col.head);
    const Seq s = uniform(col.s);
    const int n_rows = s.n * c.group;
    if (n_rows == 0) return;                                 // (a column of a worker has rows)
    const Range range = tile_range(a, s, 0, n_rows);
    const int upto = uniform(min(unit_end, col.first + col.units));
    const bool whole = unit == col.first && upto == col.first + col.units;
    const int k0 = uniform(a.workers ? range.lo + (unit - col.first) * kFewKeys : range.lo);
    const int k1 = uniform(a.workers ? min(range.hi, range.lo + (upto - col.first) * kFewKeys) : range.hi);

    W w;
    w.clear();
    const int row = min(my_row, n_rows - 1);                 // lanes without a row repeat the last one's
    const int i_row = row / c.group, g_row = row - i_row * c.group;
    const int place = s.len - s.n + i_row;
    w.hi = a.causal ? min(s.len, place + 1) : s.len;
    w.lo = a.window > 0 ? place + 1 - a.window : 0;
    w.load_queries(a.q.p + (int64_t)(s.first + i_row) * a.q.tok + (int64_t)(head * c.group + g_row) * a.q.head, j);
    // keys [all_lo, all_hi) are seen by every row
    const int all_hi = a.causal ? min(s.len, s.len - s.n + 1) : s.len;
    const int all_lo = a.window > 0 ? s.len - a.window : 0;
    auto mixed = [&](int u, uint64_t absent) { return u + 32 > all_hi || u < all_lo || absent != 0; };
    const float factor = a.factor * (E4M3 && c.k_scale ? c.k_scale[head] : 1.f);

    const uint8_t* const kp = c.k + head_offset(c, head) + 16 * ld_chunk;
    const uint8_t* const vp = c.v + head_offset(c, head) + 16 * ld_chunk;
    u32x4 rk[kLoads], rv[kLoads];
    uint32_t absent_next = 0;
    int32_t page = -1;
    auto fetch_page = [&](int u) { page = u < k1 ? page_of_key(c, b, u + (lane & 31), s.len) : 0; };
    auto fetch_rows = [&](int u) {                           // needs fetch_page(u)
      const uint64_t bad = __ballot(page < 0);
      absent_next = (uint32_t)bad;
      if (bad && lane == 0) note_bad_page(c);
      const uint64_t at = row_offset(c, __shfl(page, ld_row), u + ld_row), slot = (uint64_t)c.slot_stride << 4;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        rk[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + at + i * slot));
        rv[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + at + i * slot));
      }
    };
    // where this lane's row keeps its logits, four keys at a time
    float* const logits = a.logits && my_row < n_rows
                              ? a.logits + (((int64_t)b * c.hkv + head) * a.part_rows + my_row) * a.logit_stride + 4 * j : nullptr;

    bool odd = false;
    int u = k0 + 32 * wave;
    if (u < k1) {
      fetch_page(u);
      fetch_rows(u);
      fetch_page(u + kFewKeys);
    }
    for (; u < k1; u += kFewKeys) {
      const uint32_t absent = absent_next;
      // values behind the end and without a page are zero: a probability of zero times what lies there would not be
      const bool some = mixed(u, absent);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = ld_row + i;
        if (some) {
          if (u + r >= s.len || ((absent >> r) & 1)) rv[i] = (u32x4){0, 0, 0, 0};
          odd |= clean<T, E4M3>(rv[i]);
        }
        *reinterpret_cast<u32x4*>(lk + lds_offset<kRB>(r, ld_chunk)) = rk[i];
        *reinterpret_cast<u32x4*>(lv + lds_offset<kRB>(r, ld_chunk)) = rv[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // this wave's LDS only: its accesses are carried out in order
      __builtin_amdgcn_wave_barrier();
      if (u + kFewKeys < k1) {
        fetch_rows(u + kFewKeys);
        fetch_page(u + 2 * kFewKeys);
      }
      float x[W::kLogits];
      w.logits(lk, lane, x);
      if (mixed(u, absent)) w.mask(x, u, absent, j);
      if (logits)
#pragma unroll
        for (int g = 0; g < W::kLogits / 4; ++g)
          *reinterpret_cast<float4*>(logits + u + W::kSpan * g) =
              make_float4(x[4 * g] * factor, x[4 * g + 1] * factor, x[4 * g + 2] * factor, x[4 * g + 3] * factor);
      w.soften(x, factor);
      w.add_values(x, lv, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }

    // join the four waves
    w.l = W::over_row(w.l, [](float x, float y) { return x + y; });
    if (j == 0) stats[wave][my_row] = make_float2(w.m, w.l);
    __syncthreads();                                         // (also: no wave reads its K and V any more)
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, stats[i][my_row].x);
    const float mine = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(w.m - m);
    float* const jo = reinterpret_cast<float*>(lds) + (wave * ROWS + my_row) * D;
    if (my_row < n_rows)
#pragma unroll
      for (int i = 0; i < W::kQuads; ++i) {
        const float4 x = make_float4(w.quad(i, 0) * mine, w.quad(i, 1) * mine, w.quad(i, 2) * mine, w.quad(i, 3) * mine);
        odd |= w.l < kInf && !(fabsf(x.x) < kInf && fabsf(x.y) < kInf && fabsf(x.z) < kInf && fabsf(x.w) < kInf);
        *reinterpret_cast<float4*>(jo + ((W::kSpan * i + 4 * j) ^ (4 * (my_row & 7)))) = x;
      }
    if (__ballot(odd)) {                                     // (a row whose statistics are NaN stays NaN: they divide it below)
      float* const mend = my_row < n_rows ? jo : nullptr;
      auto at = [&](int i, int e) -> float& { return mend[(W::kSpan * i + 4 * j + e) ^ (4 * (my_row & 7))]; };
      set_odd_values<T, D, E4M3, 32>(
          c, b, head, s.len, k0 + 32 * wave, k1, kFewKeys, w.lo, w.hi, W::kSpan, j,
          [&](int i, int e) {
            if (mend) at(i, e) = 0.f;
          },
          [&](int i, int e, float x) {
            if (mend) at(i, e) += x;
          });
    }
    __syncthreads();
    const float v_scale = E4M3 && c.v_scale ? c.v_scale[head] : 1.f;
    const int64_t part = ((int64_t)blockIdx.x * 2 + (unit == col.first ? 1 : 0)) * a.part_rows;
    for (int at = threadIdx.x; at < n_rows * (D / 4); at += 256) {
      const int r = at / (D / 4), ch = at % (D / 4) * 4;
      float top = -kInf, sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, stats[i][r].x);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += top == -kInf ? 0.f : stats[i][r].y * __builtin_amdgcn_exp2f(stats[i][r].x - top);
      float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(lds) + (i * ROWS + r) * D + (ch ^ (4 * (r & 7))));
        o[0] += x.x;
        o[1] += x.y;
        o[2] += x.z;
        o[3] += x.w;
      }
      const int i_r = r / c.group, token = s.first + i_r, qh = head * c.group + r - i_r * c.group;
      if (whole) {
        const float f = sum == 0.f ? 0.f : v_scale / sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= f;
        store_out<T>(a, token, qh, ch, o);
        if (a.lse && ch == 0) a.lse[(int64_t)token * c.hq + qh] = log_sum(top, sum);
      } else {
        *reinterpret_cast<float4*>(a.part_o + (part + r) * D + ch) = make_float4(o[0], o[1], o[2], o[3]);
        if (ch == 0) a.part_ml[part + r] = make_float2(top, sum);
      }
    }
    unit = upto;
    if (unit < unit_end) __syncthreads();                    // the next column's keys go where the outputs were joined
  }
}

// ---- more rows: four waves of 32 rows share tiles of 64 keys ------------------------------------------------------
// Bound by the matrix cores and the vector units together: a unit (32 keys x 32 rows) is 6 d matrix cycles (768 for d = 128, a third of them the first
// product) and some 190 vector instructions, 16 of them exponentials.  So the work of a wave is a pipeline of units: the first product of one runs while
// the unit before it goes through its exponentials, then the second product of that one.  Three tiles of K
// and two of V lie in LDS, one barrier a tile.  K goes there from memory directly; V passes registers, where tiles that not every row sees are
// cleaned.  Both are asked for in the middle of a tile, for the tile after the next; but the compiler has them arrive before the running tile's last
// transposing reads of V, which it cannot tell from K's destination, so what they have in fact is the softmax of a unit.
// Two sequences of 20480 tokens, 4096 of them new, 32 heads on 8 of 128: 3.40 ms, 727 TFLOP/s of the formula's operations and 1090 of the matrix
// cores' own, which are busy 55 % of the time.  Before probabilities were pairs, 2717 us where K through registers took 2836; of 2865 there the
// staging was 22 %, the reads of LDS another 21 %, the exponentials 5 % after that.
// Two row blocks a wave, which would halve the reads, do not fit the registers.

template <typename T, int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void attend_chunk_kernel(const AttendArgs a) {
  typedef Shape<D, E4M3> S;
  constexpr int kRB = S::kRowBytes, kLPR = S::kLanesPerRow;
  constexpr int kLoads = 64 * kLPR / 256;
  constexpr int kTile = 64 * kRB;
  __shared__ __align__(16) uint8_t lds[5 * kTile];           // K, K, K, V, V

  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int columns = c.hkv * a.splits;
  const int column = blockIdx.x % columns, tile = a.tiles - 1 - blockIdx.x / columns;      // long causal tiles first
  const int head = column % c.hkv, split = column / c.hkv;
  int b, t;
  if (!find_tile(a, tile, kChunkRows, b, t)) return;
  b = uniform(b);
  t = uniform(t);
  const Seq s = uniform(sequence(c, b));
  const int rows = s.n * c.group, row0 = t * kChunkRows;
  if (row0 >= rows) return;
  const int n_rows = min(kChunkRows, rows - row0);
  const Range range = tile_range(a, s, row0, n_rows);
  const int n_splits = splits_of(a, range);
  if (split >= n_splits) return;
  const int k0 = uniform(range.lo + split * a.split_keys), k1 = uniform(split_end(a, range, split));

  RowBlock<T, D, E4M3> w;
  w.clear();
  const int first = row0 + 32 * wave, last = min(first + 31, row0 + n_rows - 1);           // of this wave; first > last: none
  const int row = min(first + (lane & 31), row0 + n_rows - 1);
  const int i_row = row / c.group, g_row = row - i_row * c.group;
  const int place = s.len - s.n + i_row;
  w.hi = a.causal ? min(s.len, place + 1) : s.len;
  w.lo = a.window > 0 ? place + 1 - a.window : 0;
  w.load_queries(a.q.p + (int64_t)(s.first + i_row) * a.q.tok + (int64_t)(head * c.group + g_row) * a.q.head, h);
  const int place_first = s.len - s.n + first / c.group, place_last = s.len - s.n + last / c.group;
  // keys [all_lo, all_hi) are seen by every row of the wave, keys outside [any_lo, any_hi) by none
  const int all_hi = uniform(a.causal ? min(s.len, place_first + 1) : s.len), any_hi = uniform(first > last ? 0 : (a.causal ? min(s.len, place_last + 1) : s.len));
  const int all_lo = uniform(a.window > 0 ? place_last + 1 - a.window : 0), any_lo = uniform(a.window > 0 ? place_first + 1 - a.window : 0);
  const float factor = a.factor * (E4M3 && c.k_scale ? c.k_scale[head] : 1.f);

  // A wave brings 16 neighbouring rows: eight of them and eight, whose places are scalars but for the lane's own part.
  const int ld_row = threadIdx.x / kLPR * kLoads, ld_chunk = threadIdx.x % kLPR, slot_mask = (1 << c.page_shift) - 1;
  const uint64_t slot_bytes = (uint64_t)c.slot_stride << 4, lane_part = (uint64_t)(ld_row & 7) * slot_bytes + 16 * ld_chunk;
  const uint8_t* const kp = c.k + head_offset(c, head);
  const uint8_t* const vp = c.v + head_offset(c, head);
  u32x4 rv[kLoads];                                          // rows of V on their way
  // Where a tile's rows lie, a key a lane: of the tiles of K and of V whose rows are loaded next, with the keys that have no page.
  struct Tile {
    uint64_t at, absent;
  };
  Tile tile_k{0, 0}, tile_v{0, 0};
  uint64_t absent_loaded = 0;                                // of the tile of V in the registers
  int32_t page = 0;                                          // of the tile after tile_k
  const int32_t* const entries = c.table + (int64_t)b * c.table_stride;
  auto page_at = [&](int u) { return u < k1 ? entries[min(u + lane, s.len - 1) >> c.page_shift] : 0; };      // (not looked at before it is needed: that would wait for it)
  auto tile_at = [&](int32_t entry, int u) {                 // (eight rows share a place)
    const int32_t pg = (uint32_t)entry < (uint32_t)c.n_pages ? entry : -1;
    return Tile{slot_offset(c, pg, (u + (lane & 56)) & slot_mask), __ballot(pg < 0)};
  };
  auto fetch = [&](u32x4 (&r)[kLoads], const uint8_t* p, const Tile& t) {
    auto of_row = [&](int row) {
      return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)t.at, row) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(t.at >> 32), row) << 32;
    };
    const uint64_t low = of_row(16 * wave), high = of_row(16 * wave + 8);
    const uint8_t* const q = p + (ld_row - 16 * wave < 8 ? low : high) + lane_part;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) r[i] = *reinterpret_cast<const u32x4*>(q + i * slot_bytes);
  };
  // K goes straight to LDS: 64 lanes fill 1 KB, whose pieces they ask for in the order that LDS has them
  constexpr int kRowsAtOnce = 64 / kLPR;
  const int dma_row = lane / kLPR;
  auto bring_k = [&](int buf, const Tile& t) {
    auto of_row = [&](int row) {
      return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)t.at, row) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(t.at >> 32), row) << 32;
    };
    const uint64_t low = of_row(16 * wave), high = of_row(16 * wave + 8);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = kRowsAtOnce * i + dma_row, chunk = (lane % kLPR) ^ swizzle<kRB>(row);      // (rows 16 apart swizzle alike)
      const uint8_t* const q = kp + (row < 8 ? low : high) + (uint64_t)(row & 7) * slot_bytes + 16 * chunk;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)q,
                                       (__attribute__((address_space(3))) void*)(lds + buf + (16 * wave + kRowsAtOnce * i) * kRB), 16, 0, 0);
    }
  };
  auto arrived = []() { __builtin_amdgcn_s_waitcnt(0x0F70); };      // vmcnt(0): the barrier does not wait for what is on its way to LDS
  auto fetch_v = [&]() {
    absent_loaded = tile_v.absent;
    if (absent_loaded && threadIdx.x == 0) note_bad_page(c);
    fetch(rv, vp, tile_v);
  };
  auto put = [&](const u32x4 (&r)[kLoads], int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(lds + buf + lds_offset<kRB>(ld_row + i, ld_chunk)) = r[i];
  };
  const int block_hi = uniform(a.causal ? min(s.len, s.len - s.n + row0 / c.group + 1) : s.len);
  const int block_lo = uniform(a.window > 0 ? s.len - s.n + (row0 + n_rows - 1) / c.group + 1 - a.window : 0);
  auto mixed = [&](int u, uint64_t missing) { return u + 64 > block_hi || u < block_lo || missing != 0; };
  bool odd = false;
  auto put_v = [&](int buf, int u) {                         // values behind the end and without a page are zero
    if (mixed(u, absent_loaded))
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if (u + ld_row + i >= s.len || ((absent_loaded >> (ld_row + i)) & 1)) rv[i] = (u32x4){0, 0, 0, 0};
        odd |= clean<T, E4M3>(rv[i]);
      }
    put(rv, buf);
  };
  // units [live_from, + live_keys) hold a key that one of the wave's rows sees, units [clear_from, + clear_keys) only keys that all of them see: one
  // comparison each, for scalar instructions count too (a unit took 69 of them, 124 vector ones and 8 matrix ones at d = 64)
  const int live_from = any_lo - 31, clear_from = all_lo;
  const uint32_t live_keys = (uint32_t)max(0, min(k1, any_hi) - live_from), clear_keys = (uint32_t)max(0, all_hi - 31 - all_lo);
  auto live = [&](int key0) { return (uint32_t)(key0 - live_from) < live_keys; };

  // in LDS before the first tile: its K and V and the next one's K; on the way: the next one's V and the third one's K
  uint64_t absent = 0;                                       // of the running tile
  f32x16 x, y;                                               // logits of the running unit, then its probabilities; of the next one
  if (k0 < k1) {
    tile_v = tile_at(page_at(k0), k0);
    bring_k(0, tile_v);
    fetch_v();
    tile_k = tile_at(page_at(k0 + 64), k0 + 64);
    put_v(3 * kTile, k0);
    absent = absent_loaded;
    if (k0 + 64 < k1) {
      bring_k(kTile, tile_k);
      tile_v = tile_k;
      fetch_v();
      tile_v = tile_at(page_at(k0 + 128), k0 + 128);
      tile_k = tile_at(page_at(k0 + 192), k0 + 192);
      page = page_at(k0 + 256);
    }
  }
  arrived();
  __syncthreads();
  int kb = 0, kb1 = kTile, kb2 = 2 * kTile, vb = 3 * kTile, vb1 = 4 * kTile;      // buffers: K of the running tile and the next two, V of it and the next
  bool now = live(k0);
  if (now) x = w.logits(lds, lane);
  for (int u = k0; u < k1; u += 64) {
    uint64_t absent_next = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int key0 = u + 32 * half;
      const uint8_t* const k_now = lds + kb + half * 32 * kRB;
      const uint8_t* const k_next = half == 0 ? lds + kb + 32 * kRB : lds + kb1;
      const uint8_t* const v_now = lds + vb + half * 32 * kRB;
      const bool next = live(key0 + 32);
      if (now) {
        const uint32_t missing = (uint32_t)(absent >> (32 * half));
        const bool masked = (uint32_t)(key0 - clear_from) >= clear_keys || missing;
        if (masked) w.mask(x, key0, missing, h);
        float sum = next ? w.template soften<true>(x, factor, k_next, lane, y) : w.template soften<false>(x, factor, k_next, lane, y);
        if (__ballot(sum > kMost || w.m == -kInf)) {         // rare: form the unit again and raise m to its largest
          x = w.logits(k_now, lane);
          if (masked) w.mask(x, key0, missing, h);
          w.raise(x, factor);
          sum = w.template soften<false>(x, factor, k_next, lane, y);
        }
        w.l += sum;
        __builtin_amdgcn_s_setprio(1);                       // (the matrix cores before the other wave's exponentials)
        w.add_values(x, v_now, lane);
        __builtin_amdgcn_s_setprio(0);
      } else if (next) {
        y = w.logits(k_next, lane);
      }
      x = y;
      now = next;
      // into buffers that were read last in the tile before this one, a barrier ago
      if (half == 0) {
        if (u + 64 < k1) {
          put_v(vb1, u + 64);
          absent_next = absent_loaded;
        }
        if (u + 128 < k1) {
          bring_k(kb2, tile_v);
          fetch_v();
        }
      } else if (u + 128 < k1) {
        tile_v = tile_k;
        tile_k = tile_at(page, u + 256);
        page = page_at(u + 320);
      }
    }
    arrived();
    __syncthreads();
    const int kb_free = kb, vb_free = vb;
    kb = kb1;
    kb1 = kb2;
    kb2 = kb_free;
    vb = vb1;
    vb1 = vb_free;
    absent = absent_next;
  }

  {
    const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(w.l), __float_as_uint(w.l), false, false);
    w.l = __uint_as_float(z[0]) + __uint_as_float(z[1]);
  }
  const bool mine = first + (lane & 31) <= last;
  const int token = s.first + i_row, qh = head * c.group + g_row;
  const bool whole = n_splits == 1;
  const int64_t part_row = (((int64_t)tile * c.hkv + head) * a.splits + split) * a.part_rows + (row - row0);
  const float f = whole ? (w.l == 0.f ? 0.f : (E4M3 && c.v_scale ? c.v_scale[head] : 1.f) / w.l) : 1.f;
  if (mine) {
#pragma unroll
    for (int cb = 0; cb < S::kBlocks; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ch = 32 * cb + 8 * g + 4 * h;
        const float o[4] = {w.o[cb][4 * g] * f, w.o[cb][4 * g + 1] * f, w.o[cb][4 * g + 2] * f, w.o[cb][4 * g + 3] * f};
        odd |= w.l < kInf && !(fabsf(o[0]) < kInf && fabsf(o[1]) < kInf && fabsf(o[2]) < kInf && fabsf(o[3]) < kInf);
        if (whole) store_out<T>(a, token, qh, ch, o);
        else *reinterpret_cast<float4*>(a.part_o + part_row * D + ch) = make_float4(o[0], o[1], o[2], o[3]);
      }
    if (h == 0) {
      if (!whole) a.part_ml[part_row] = make_float2(w.m, w.l);
      else if (a.lse) a.lse[(int64_t)token * c.hq + qh] = log_sum(w.m, w.l);
    }
  }
  // whether any thread met one: a word of the tiles, which are read no more (the kernel has no LDS to spare: 80 KB a workgroup, two of them)
  int* const any_odd = reinterpret_cast<int*>(lds);
  if (threadIdx.x == 0) *any_odd = 0;
  __syncthreads();
  if (odd) *any_odd = 1;
  __syncthreads();
  if (*any_odd) {                                            // (a lane changes what it has just written; a row whose statistics are NaN stays NaN)
    const bool mend = mine && w.l < kInf;
    uint16_t* const o16 = reinterpret_cast<uint16_t*>(a.out.p + (int64_t)token * a.out.tok + (int64_t)qh * a.out.head);
    set_odd_values<T, D, E4M3, 64>(
        c, b, head, s.len, k0, k1, 64, w.lo, w.hi, 8, h,
        [&](int i, int e) {
          if (!mend) return;
          if (whole) o16[8 * i + 4 * h + e] = 0;
          else a.part_o[part_row * D + 8 * i + 4 * h + e] = 0.f;
        },
        [&](int i, int e, float x) {
          if (!mend) return;
          uint16_t* const at = o16 + 8 * i + 4 * h + e;
          if (whole) *at = (uint16_t)T::pack(T::low(*at) + x, 0.f);
          else a.part_o[part_row * D + 8 * i + 4 * h + e] += x;
        });
  }
}

// ---- partial results ------------------------------------------------------------------------------------------------
// A piece's factor may be zero in fp32, but an infinity that a row sees is the row's whatever its weight.
__device__ __forceinline__ float weighed(float f, float x) { return fabsf(x) < kInf ? f * x : x; }

// Launches of few rows: WAVES waves join the pieces of one row (token, query head).  A lane has four channels, 256 / D lane groups of a wave
// take a piece each and the next ones after it, four loads ahead.  One wave is enough for a few pieces; 128 of them took one wave 58 us
// (128 rows, d = 128, two channels a lane, one piece after the other).
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(256) void merge_kernel(const AttendArgs a, const bool scaled) {
  constexpr int kLanes = D / 4, kGroups = 64 / kLanes * WAVES;      // lanes of a range, ranges at a time
  __shared__ float join[WAVES > 1 ? WAVES : 1][D + 1];
  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  const int token = (int)(job / (uint32_t)c.hq), qh = (int)(job - (uint32_t)token * (uint32_t)c.hq);
  if (token >= c.n_tokens) return;
  const int head = qh / c.group;
  int before = 0, units = -1, in_front = 0, row = 0;
  for (int base = 0; base < c.n_seqs; base += 64) {
    const Lanes x = load_lanes(a, base, before);
    const uint64_t mine = __ballot(token >= x.mine.first && token < x.mine.first + x.mine.n);
    if (units < 0 && mine) {
      const int at = __ffsll((unsigned long long)mine) - 1;
      units = __shfl(x.units, at);
      in_front = before + __shfl(x.upto, at) - units;
      row = (token - __shfl(x.mine.first, at)) * c.group + qh - head * c.group;
    }
    before += x.all;
  }
  if (units < 0) return;
  // A worker's places: 0 for a column that began before it, 1 for one that ends behind it, so the first piece lies in a 1, others in a 0.
  const int begin = in_front * c.hkv + head * units, share = share_of(a, before * c.hkv), w0 = begin / share;
  const int n = units ? (begin + units - 1) / share - w0 + 1 : 0;      // 0: the row sees nothing
  if (n == 1) return;                                        // written already
  auto piece = [&](int i) { return ((int64_t)(w0 + i) * 2 + (i == 0 ? 1 : 0)) * a.part_rows + row; };
  float m = -kInf;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, a.part_ml[piece(i)].x);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float ref = m == -kInf ? 0.f : m;
  const int ch = lane % kLanes * 4, group = (WAVES == 1 ? 0 : wave * (64 / kLanes)) + lane / kLanes;
  float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = group; i < n; i += kGroups) {
    const float2 w = a.part_ml[piece(i)];
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + piece(i) * D + ch);
    const float f = __builtin_amdgcn_exp2f(w.x - ref);
    l += f * w.y;
    x[0] += weighed(f, y.x);
    x[1] += weighed(f, y.y);
    x[2] += weighed(f, y.z);
    x[3] += weighed(f, y.w);
  }
#pragma unroll
  for (int o = kLanes; o < 64; o <<= 1) {
    l += __shfl_xor(l, o);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], o);
  }
  if constexpr (WAVES > 1) {
    if (lane < kLanes) {
#pragma unroll
      for (int e = 0; e < 4; ++e) join[wave][ch + e] = x[e];
      if (lane == 0) join[wave][D] = l;
    }
    __syncthreads();                                         // (a workgroup's waves have the same row: none has left)
    if (wave > 0) return;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      l += join[i][D];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += join[i][ch + e];
    }
  }
  if (lane >= kLanes) return;
  const float f = l == 0.f ? 0.f : (scaled && c.v_scale ? c.v_scale[head] : 1.f) / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= f;
  store_out<T>(a, token, qh, ch, x);
  if (a.lse && lane == 0) a.lse[(int64_t)token * c.hq + qh] = log_sum(m, l);
}

// Launches of more rows: D / 4 lanes a row of a row tile.
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_tile_kernel(const AttendArgs a, const int slices, const bool scaled) {
  constexpr int kLanes = D / 4, kRows = 256 / kLanes;
  const Call& c = a.c;
  const int job = blockIdx.x / slices, slice = blockIdx.x - job * slices, tile = job / c.hkv, head = job - tile * c.hkv;
  int b, t;
  if (!find_tile(a, tile, kChunkRows, b, t)) return;
  b = uniform(b);
  t = uniform(t);
  const Seq s = uniform(sequence(c, b));
  const int row0 = t * kChunkRows, n_rows = min(kChunkRows, s.n * c.group - row0), r = slice * kRows + (int)threadIdx.x / kLanes;
  if (n_rows <= 0) return;
  const int n = splits_of(a, tile_range(a, s, row0, n_rows));
  if (n == 1 || r >= n_rows) return;                         // (one range: written already)
  const int ch = threadIdx.x % kLanes * 4;
  const int64_t first = (int64_t)job * a.splits * a.part_rows + r;
  float m = -kInf;
#pragma unroll 4
  for (int i = 0; i < n; ++i) m = fmaxf(m, a.part_ml[first + (int64_t)i * a.part_rows].x);
  const float ref = m == -kInf ? 0.f : m;
  float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const int64_t at = first + (int64_t)i * a.part_rows;
    const float2 w = a.part_ml[at];
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + at * D + ch);
    const float f = __builtin_amdgcn_exp2f(w.x - ref);
    l += f * w.y;
    x[0] += weighed(f, y.x);
    x[1] += weighed(f, y.y);
    x[2] += weighed(f, y.z);
    x[3] += weighed(f, y.w);
  }
  const int row = row0 + r, i_row = row / c.group, token = s.first + i_row, qh = head * c.group + row - i_row * c.group;
  const float f = l == 0.f ? 0.f : (scaled && c.v_scale ? c.v_scale[head] : 1.f) / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= f;
  store_out<T>(a, token, qh, ch, x);
  if (a.lse && ch == 0) a.lse[(int64_t)token * c.hq + qh] = log_sum(m, l);
}

template <typename F>
void by_type(int d, int dtype, bool e4m3, F&& f) {
  auto by_d = [&](auto t, auto f8) {
    if (d == 128) f(t, std::integral_constant<int, 128>{}, f8);
    else f(t, std::integral_constant<int, 64>{}, f8);
  };
  auto by_cache = [&](auto t) {
    if (e4m3) by_d(t, std::true_type{});
    else by_d(t, std::false_type{});
  };
  if (dtype == KV_F16) by_cache(Half{});
  else by_cache(Brain{});
}

}  // namespace

void launch_attend(const AttendArgs& a, int d, int dtype, bool e4m3, int tile_rows, hipStream_t st) {
  const dim3 grid((unsigned)attend_grid(a).x);
  by_type(d, dtype, e4m3, [&](auto t, auto dd, auto f8) {
    if (tile_rows == kFewRows && a.part_rows <= 16) attend_few_kernel<decltype(t), decltype(dd)::value, decltype(f8)::value, 16><<<grid, dim3(256), 0, st>>>(a);
    else if (tile_rows == kFewRows) attend_few_kernel<decltype(t), decltype(dd)::value, decltype(f8)::value, 32><<<grid, dim3(256), 0, st>>>(a);
    else attend_chunk_kernel<decltype(t), decltype(dd)::value, decltype(f8)::value><<<grid, dim3(256), 0, st>>>(a);
  });
}

void launch_merge(const AttendArgs& a, int d, int dtype, bool e4m3, hipStream_t st) {
  const dim3 grid((unsigned)merge_grid(a, d).x);
  by_type(d, dtype, false, [&](auto t, auto dd, auto) {
    typedef decltype(t) Type;
    constexpr int kD = decltype(dd)::value;
    if (a.workers == 0) merge_tile_kernel<Type, kD><<<grid, dim3(256), 0, st>>>(a, merge_slices(a, kD), e4m3);
    else if (merge_waves(a) == 4) merge_kernel<Type, kD, 4><<<grid, dim3(256), 0, st>>>(a, e4m3);
    else merge_kernel<Type, kD, 1><<<grid, dim3(256), 0, st>>>(a, e4m3);
  });
}

}  // namespace paged
}  // namespace kvx
