// Weights that cached tokens receive in a call's attention: weights_out_j = weights_j + sum over the call's rows of the key head's group
// of softmax weight (row, j), from the rows' lse.
//
// weights_from_logits_kernel, behind attention launches of few rows, reads the logits that those kept: 8 bytes a row and key, written and
// read, where K would be another d elements.  weights_kernel forms them again.
//
// weights_kernel.  A workgroup owns 128 keys of one key head, a wave 32 of them, whose fragments stay in registers, and goes over all rows that see
// them, 32 at a time, brought into LDS for the four waves.  S = Q K^T with a key in a lane and its rows in that lane's registers: a key's
// weights are summed in its lane, in row order, in fp32 without a rounding between, and no two workgroups write the same
// token, so the sums do not depend on what ran when.
#include "../../include/kvx.h"
#include "paged_tile.h"

namespace kvx {
namespace paged {

namespace {

constexpr int kKeys = 128;

template <typename T, int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void weights_kernel(const AttendArgs a) {
  constexpr int kRB = 2 * D, kLPR = kRB / 16, kSteps = D / 16;     // rows of queries are 16-bit
  constexpr int kLoads = 32 * kLPR / 256;
  __shared__ __align__(16) uint8_t lq[2][32 * kRB];
  __shared__ __align__(16) float l_lse[2][32];                     // log2 units; infinite: the row counts nothing
  __shared__ __align__(16) int l_hi[2][32], l_lo[2][32];

  const Call& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int key_blocks = (c.max_len + kKeys - 1) / kKeys;
  const int head = blockIdx.x % c.hkv, rest = blockIdx.x / c.hkv;
  const int block = rest % key_blocks, b = rest / key_blocks;
  const Seq s = sequence(c, b);
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
  const int r0 = i0 * c.group, r1 = i1 * c.group;
  const int ld_row = threadIdx.x / kLPR * kLoads, ld_chunk = threadIdx.x % kLPR;
  u32x4 rq[kLoads];
  float r_lse = 0.f;
  int r_hi = 0, r_lo = 0;
  auto fetch = [&](int r) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = min(r + ld_row + i, r1 - 1), it = row / c.group, g = row - it * c.group;
      rq[i] = *reinterpret_cast<const u32x4*>(a.q.p + (int64_t)(s.first + it) * a.q.tok + (int64_t)(head * c.group + g) * a.q.head + 16 * ld_chunk);
    }
    if (threadIdx.x < 32) {
      const int row = min(r + (int)threadIdx.x, r1 - 1), it = row / c.group, g = row - it * c.group;
      const float x = a.lse[(int64_t)(s.first + it) * c.hq + head * c.group + g];
      r_lse = r + (int)threadIdx.x >= r1 || x == -kInf ? kInf : x * 1.4426950408889634f;
      r_hi = a.causal ? min(s.len, base + it + 1) : s.len;
      r_lo = a.window > 0 ? base + it + 1 - a.window : 0;
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(lq[buf] + lds_offset<kRB>(ld_row + i, ld_chunk)) = rq[i];
    if (threadIdx.x < 32) {
      l_lse[buf][threadIdx.x] = r_lse;
      l_hi[buf][threadIdx.x] = r_hi;
      l_lo[buf][threadIdx.x] = r_lo;
    }
  };
  float sum = 0.f;
  if (r0 < r1) {
    fetch(r0);
    put(0);
    if (r0 + 32 < r1) fetch(r0 + 32);
  }
  __syncthreads();
  int buf = 0;
  for (int r = r0; r < r1; r += 32, buf ^= 1) {
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      x = T::mfma(*reinterpret_cast<const u32x4*>(lq[buf] + lds_offset<kRB>(lane & 31, step_channel<E4M3>(i, h) / 8)), kf[i], x);
    const int first = r / c.group, last = (min(r + 32, r1) - 1) / c.group;
    const bool masked = (a.causal && kb + kKeys > base + first + 1) || (a.window > 0 && kb < base + last + 1 - a.window);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at = 8 * g + 4 * h;
      const float4 l4 = *reinterpret_cast<const float4*>(&l_lse[buf][at]);
      const float ls[4] = {l4.x, l4.y, l4.z, l4.w};
      if (masked) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * g + e], factor, -ls[e]));
          sum += key < l_hi[buf][at + e] && key >= l_lo[buf][at + e] ? p : 0.f;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * g + e], factor, -ls[e]));
      }
    }
    if (r + 32 < r1) {
      put(buf ^ 1);
      if (r + 64 < r1) fetch(r + 64);
    }
    __syncthreads();
  }
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
  sum = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  if (h == 0 && page >= 0) {
    const int64_t at = (((int64_t)page * c.hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
    a.weights_out[at] = a.weights_in[at] + sum;
  }
}

// A thread has four neighbouring keys of one key head.  A row's range of keys (row tiles of decoding see them all but for masks) was
// written as far as its tile goes; keys that no row of the tile read (in front of a window) have no logits and gain nothing.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void weights_from_logits_kernel(const AttendArgs a) {
  const Call& c = a.c;
  __shared__ float lse[32];
  const int key_blocks = (c.max_len + 4 * kThreads - 1) / (4 * kThreads);
  const int head = blockIdx.x % c.hkv, rest = blockIdx.x / c.hkv;
  const int block = rest % key_blocks, b = rest / key_blocks;
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
  constexpr int kThreads = 256;
  const dim3 grid((unsigned)((int64_t)((a.c.max_len + 4 * kThreads - 1) / (4 * kThreads)) * a.c.hkv * a.c.n_seqs));
  weights_from_logits_kernel<kThreads><<<grid, dim3(kThreads), 0, st>>>(a);
}

void launch_weights(const AttendArgs& a, int d, int dtype, bool e4m3, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)((a.c.max_len + kKeys - 1) / kKeys) * a.c.hkv * a.c.n_seqs));
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
}

}  // namespace paged
}  // namespace kvx
