// Weights that cached tokens receive in a call's attention: weights_out_j = weights_j + sum over the call's rows of the key head's group
// of softmax weight (row, j), from the rows' lse.
//
// weights_from_logits_kernel, behind attention launches of few rows, reads the logits that those kept: 8 bytes a row and key, written and
// read, where K would be another d elements.  weights_kernel forms them again.
//
// weights_kernel.  A workgroup owns 128 keys of one key head, a wave 32 of them, whose fragments stay in registers, and goes over all rows that see
// them, 64 at a time, brought into LDS for the four waves.  S = Q K^T with a key in a lane and its rows in that lane's registers: a key's
// weights are summed in its lane, in row order, in fp32 without a rounding between, and no two workgroups write the same
// token, so the sums do not depend on what ran when.  Where that makes too few workgroups for the chip the rows are
// cut into parts as well, whose sums weights_sum_kernel adds in order (4 us).  It is bound by its exponentials and the masks and sums around them,
// at about a third of the rate that the products alone would reach.
#include "../../include/kvx.h"
#include "paged_tile.h"

namespace kvx {
namespace paged {

namespace {

constexpr int kKeys = kWeightKeys, kRows = 64;

template <typename T, int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void weights_kernel(const AttendArgs a) {
  constexpr int kRB = 2 * D, kLPR = kRB / 16, kSteps = D / 16;     // rows of queries are 16-bit
  constexpr int kLoads = kRows * kLPR / 256;
  __shared__ __align__(16) uint8_t lq[2][kRows * kRB];
  __shared__ __align__(16) float l_lse[2][kRows];                  // log2 units; infinite: the row counts nothing
  __shared__ __align__(16) int l_place[2][kRows];

  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int head = blockIdx.x % c.hkv, block = blockIdx.x / c.hkv, column = blockIdx.y, b = column % c.n_seqs, split = column / c.n_seqs;
  const Seq s = uniform(sequence(c, b));
  const int kb = block * kKeys;
  if (kb >= s.len) return;
  const int key = kb + 32 * wave + (lane & 31);
  const int32_t page = key < s.len ? page_of_key(c, b, key, s.len) : -1;
  if (key < s.len && page < 0) note_bad_page(c);
  const float factor = a.factor * (E4M3 && c.k_scale ? c.k_scale[head] : 1.f);

  u32x4 kf[kSteps];
  {
    const uint8_t* kp = c.k + head_offset(c, head) + row_offset(c, page, key);
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < kSteps / 2; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(kp + 32 * i + 16 * h);
        kf[2 * i] = widen<T>((u32x2){x[0], x[1]});
        kf[2 * i + 1] = widen<T>((u32x2){x[2], x[3]});
      }
    } else {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) kf[i] = *reinterpret_cast<const u32x4*>(kp + 2 * step_channel<E4M3>(i, h));
    }
  }

  // rows that see one of the workgroup's keys: new tokens [i0, i1)
  const int base = s.len - s.n;
  const int i0 = a.causal ? min(s.n, max(0, kb - base)) : 0;
  const int i1 = a.window > 0 ? max(i0, min(s.n, kb + kKeys - 1 + a.window - base)) : s.n;
  const int rows = (i1 - i0) * c.group, part = a.weight_splits > 1 ? a.weight_rows : rows;
  const int r0 = uniform(i0 * c.group + min(rows, split * part)), r1 = uniform(i0 * c.group + min(rows, (split + 1) * part));
  // A thread brings the same rows of every kRows: their tokens and heads move on by the same steps (a division by the group would cost more
  // than a row's exponentials).
  struct Place {
    int it, g;
  };
  const int step_it = kRows / c.group, step_g = kRows - step_it * c.group;
  auto place_of = [&](int row) {
    const int it = row / c.group;
    return Place{it, row - it * c.group};
  };
  auto move_on = [&](Place& x) {
    x.it += step_it;
    x.g += step_g;
    if (x.g >= c.group) {
      x.g -= c.group;
      ++x.it;
    }
  };
  const int ld_row = threadIdx.x / kLPR, ld_chunk = threadIdx.x % kLPR;      // and every (256 / kLPR)-th row after it
  u32x4 rq[kLoads];
  float r_lse = 0.f;
  int r_place = 0;
  Place at[kLoads], mine = place_of(r0 + (int)(threadIdx.x & (kRows - 1)));
#pragma unroll
  for (int i = 0; i < kLoads; ++i) at[i] = place_of(r0 + ld_row + i * (256 / kLPR));
  auto fetch = [&]() {                                             // the next kRows rows; rows behind the last repeat it and count nothing
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool real = at[i].it < i1;
      const int it = real ? at[i].it : i1 - 1, g = real ? at[i].g : c.group - 1;
      rq[i] = *reinterpret_cast<const u32x4*>(a.q.p + (int64_t)(s.first + it) * a.q.tok + (int64_t)(head * c.group + g) * a.q.head + 16 * ld_chunk);
      move_on(at[i]);
    }
    if (threadIdx.x < kRows) {
      const bool real = mine.it < i1;
      const int it = real ? mine.it : i1 - 1, g = real ? mine.g : c.group - 1;
      const float x = a.lse[(int64_t)(s.first + it) * c.hq + head * c.group + g];
      r_lse = !real || x == -kInf ? kInf : x * 1.4426950408889634f;
      r_place = base + it;
      move_on(mine);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(lq[buf] + lds_offset<kRB>(ld_row + i * (256 / kLPR), ld_chunk)) = rq[i];
    if (threadIdx.x < kRows) {
      l_lse[buf][threadIdx.x] = r_lse;
      l_place[buf][threadIdx.x] = r_place;
    }
  };
  float sum = 0.f;
  if (r0 < r1) {
    fetch();
    put(0);
    if (r0 + kRows < r1) fetch();
  }
  __syncthreads();
  int buf = 0;
  // rows from here on see all of the workgroup's keys, and before there
  const int all_from = a.causal ? uniform(min(s.n, kb + kKeys - 1 - base) * c.group) : 0;
  const int all_to = a.window > 0 ? uniform(min(s.n, kb + a.window - base) * c.group) : r1 + kRows;
  for (int r = r0; r < r1; r += kRows, buf ^= 1) {
    const bool masked = r < all_from || min(r + kRows, r1) > all_to;
#pragma unroll
    for (int half = 0; half < kRows / 32; ++half) {
      f32x16 x{};
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        x = T::mfma(*reinterpret_cast<const u32x4*>(lq[buf] + 32 * half * kRB + lds_offset<kRB>(lane & 31, step_channel<E4M3>(i, h) / 8)), kf[i], x);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int first = 32 * half + 8 * g + 4 * h;
        const float4 l4 = *reinterpret_cast<const float4*>(&l_lse[buf][first]);
        const float ls[4] = {l4.x, l4.y, l4.z, l4.w};
        if (masked) {
          const int4 p4 = *reinterpret_cast<const int4*>(&l_place[buf][first]);
          const int place[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * g + e], factor, -ls[e]));
            sum += (!a.causal || key <= place[e]) && (a.window == 0 || key > place[e] - a.window) ? p : 0.f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * g + e], factor, -ls[e]));
        }
      }
    }
    if (r + kRows < r1) {
      put(buf ^ 1);
      if (r + 2 * kRows < r1) fetch();
    }
    __syncthreads();
  }
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
  sum = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  if (a.weight_splits > 1) {
    if (h == 0) a.weight_part[((int64_t)column * c.hkv + head) * a.weight_stride + key] = sum;
  } else if (h == 0 && page >= 0) {
    const int64_t at = (((int64_t)page * c.hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
    a.weights_out[at] = a.weights_in[at] + sum;
  }
}

// The sums over the parts of the rows, a key a thread.
__global__ __launch_bounds__(256) void weights_sum_kernel(const AttendArgs a) {
  const Call& c = a.c;
  const int head = blockIdx.x % c.hkv, b = blockIdx.y, key = blockIdx.x / c.hkv * 256 + threadIdx.x;
  const Seq s = sequence(c, b);
  if (key >= s.len) return;
  const int32_t page = page_of(c, b, key >> c.page_shift);
  if (page < 0) return;
  float sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < a.weight_splits; ++i) sum += a.weight_part[(((int64_t)i * c.n_seqs + b) * c.hkv + head) * a.weight_stride + key];
  const int64_t at = (((int64_t)page * c.hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
  a.weights_out[at] = a.weights_in[at] + sum;
}

// A thread has four neighbouring keys of one key head.  A row's range of keys (row tiles of decoding see them all but for masks) was
// written as far as its tile goes; keys that no row of the tile read (in front of a window) have no logits and gain nothing.
__global__ __launch_bounds__(256) void weights_from_logits_kernel(const AttendArgs a) {
  const Call& c = a.c;
  constexpr int kThreads = 256;
  __shared__ float lse[32];
  const int head = blockIdx.x % c.hkv, block = blockIdx.x / c.hkv, b = blockIdx.y;
  const Seq s = sequence(c, b);
  if (block * 4 * kThreads >= s.len) return;
  const int rows = s.n * c.group;                            // one tile of a sequence's rows
  if ((int)threadIdx.x < rows) {
    const int it = threadIdx.x / c.group, g = threadIdx.x - it * c.group;
    const float x = a.lse[(int64_t)(s.first + it) * c.hq + head * c.group + g];
    lse[threadIdx.x] = x == -kInf ? kInf : x * 1.4426950408889634f;
  }
  __syncthreads();
  const int key = (block * kThreads + threadIdx.x) * 4;
  if (key >= s.len) return;
  const int32_t page = page_of(c, b, key >> c.page_shift);
  if (page < 0) {
    note_bad_page(c);
    return;
  }
  const int64_t at = (((int64_t)page * c.hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
  const float4 before = *reinterpret_cast<const float4*>(a.weights_in + at);
  const Range range = rows ? tile_range(a, s, 0, rows) : Range{0, 0};
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if (key >= range.lo && key < range.hi) {
    const float* x = a.logits + ((int64_t)b * c.hkv + head) * a.part_rows * a.logit_stride + key;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
      const float4 y = *reinterpret_cast<const float4*>(x + r * a.logit_stride);
      sum[0] += __builtin_amdgcn_exp2f(y.x - lse[r]);
      sum[1] += __builtin_amdgcn_exp2f(y.y - lse[r]);
      sum[2] += __builtin_amdgcn_exp2f(y.z - lse[r]);
      sum[3] += __builtin_amdgcn_exp2f(y.w - lse[r]);
    }
  }
  float* out = a.weights_out + at;
  const float w[4] = {before.x + sum[0], before.y + sum[1], before.z + sum[2], before.w + sum[3]};
  if (key + 4 <= s.len) {
    *reinterpret_cast<float4*>(out) = make_float4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (key + e < s.len) out[e] = w[e];
  }
}

}  // namespace

void launch_weights_from_logits(const AttendArgs& a, hipStream_t st) {
  const Grid g = weights_from_logits_grid(a);
  weights_from_logits_kernel<<<dim3((unsigned)g.x, (unsigned)g.y), dim3(256), 0, st>>>(a);
}

void launch_weights(const AttendArgs& a, int d, int dtype, bool e4m3, hipStream_t st) {
  const Grid all = weights_grid(a), sum = weights_sum_grid(a);
  const dim3 grid((unsigned)all.x, (unsigned)all.y);
  auto go = [&](auto t, auto dd, auto f8) { weights_kernel<decltype(t), decltype(dd)::value, decltype(f8)::value><<<grid, dim3(256), 0, st>>>(a); };
  auto by_d = [&](auto t, auto f8) {
    if (d == 128) go(t, std::integral_constant<int, 128>{}, f8);
    else go(t, std::integral_constant<int, 64>{}, f8);
  };
  auto by_cache = [&](auto t) {
    if (e4m3) by_d(t, std::true_type{});
    else by_d(t, std::false_type{});
  };
  if (dtype == KV_F16) by_cache(Half{});
  else by_cache(Brain{});
  if (a.weight_splits > 1) weights_sum_kernel<<<dim3((unsigned)sum.x, (unsigned)sum.y), dim3(256), 0, st>>>(a);
}

}  // namespace paged
}  // namespace kvx
