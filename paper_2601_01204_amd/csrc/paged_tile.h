// Pieces of the attention kernels on a paged cache: tiles of keys and values in LDS, and one unit of work, 32 keys x 32 query rows.
//
// Products.  S^T = K Q^T and O^T += V^T P^T on the matrix cores (32 x 32 x 16), fp32 accumulators.  The transposed products put a
// query row in a lane (two lanes, l and l + 32, share one) and its keys in that lane's registers, so that softmax statistics are
// registers' business with one exchange between the halves, and the probabilities feed the second product without leaving
// them: register r of half h belongs to key 8 (r / 4) + 4 h + r % 4 of the unit, and V^T is read in that key order.
//
// LDS.  Rows of d channels as they lie in the page, in chunks of 16 bytes whose place within the row is exclusive-or'ed with
// swizzle(row), so that both the row reads of K (a lane a row) and the transposing reads of V (16 lanes four rows of 16 channels
// each, eight rows for 8-bit values) meet every bank equally often.
//
// 8-bit pages are widened as they leave LDS, which is exact; a head's key scale is part of the logit factor, its value scale of the
// final division.  A row of 8-bit keys is read 16 channels at a time, which serve two matrix instructions: their
// channels are 32 s + 16 h + 0..7 and 8..15, for the queries too.
//
// Softmax.  p = 2^(c s - m) in fp32.  Few rows: m lies kFewLift below the largest c s of the row so far, raised only where a key lies more than kFewGap
// above that one (O and l are rescaled in a rare, wave-uniform branch).  More rows, where vector instructions are dear: m lies kChunkLift below
// the largest of the row's first unit, and no maximum is taken after that; only where a unit's sum shows that some p is large (kMost,
// which fp16 still holds; sixteen equal keys reach half of it) is the unit formed again and m raised.  The second product takes a probability
// as two 16-bit values, the second what the first one's rounding leaves, so that nothing but the output is rounded to 16 bits.
// In fp16 an error of 2^-25 remains, half the type's least step: for every key 2^-39 of the row's largest weight (few rows) or 2^-35 (more), which is less
// than an output's half step of 2^-11 up to 2^28 and 2^24 keys.
#pragma once
#include "paged_types.h"

#include <type_traits>

namespace kvx {
namespace paged {

constexpr float kMost = 32768.0f;
constexpr float kInf = __builtin_inff();

template <int ROW_BYTES>
__device__ __forceinline__ int swizzle(int row) {
  if constexpr (ROW_BYTES == 256) return ((row & 3) << 2) | ((row >> 2) & 3);
  else if constexpr (ROW_BYTES == 128) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  else return (row >> 2) & 3;
}
template <int ROW_BYTES>
__device__ __forceinline__ int lds_offset(int row, int chunk) {
  return row * ROW_BYTES + ((chunk ^ swizzle<ROW_BYTES>(row)) << 4);
}

template <int D, bool E4M3>
struct Shape {
  static constexpr int kRowBytes = D * (E4M3 ? 1 : 2);
  static constexpr int kLanesPerRow = kRowBytes / 16;
  static constexpr int kSteps = D / 16;            // matrix instructions of a unit's first product
  static constexpr int kBlocks = D / 32;           // 32-channel blocks of the output
};

// First channel of the octet that half `h` of a wave brings to step s of the first product.
template <bool E4M3>
__device__ __forceinline__ int step_channel(int s, int h) {
  return E4M3 ? 32 * (s >> 1) + 16 * h + 8 * (s & 1) : 16 * s + 8 * h;
}

// 32 query rows of one wave.
template <typename T, int D, bool E4M3>
struct RowBlock {
  typedef Shape<D, E4M3> S;
  u32x4 q[S::kSteps];
  f32x16 o[S::kBlocks];
  float m, l;                  // m: the reference, in log2 units; l: this lane's half of the keys
  int lo, hi;                  // keys [lo, hi) are seen by this lane's row

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    m = -kInf;
    l = 0.f;
  }

  __device__ __forceinline__ void load_queries(const uint8_t* row, int h) {
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) q[s] = *reinterpret_cast<const u32x4*>(row + 2 * step_channel<E4M3>(s, h));
  }

  // S^T of the unit whose keys' rows begin at `k` in LDS.
  __device__ __forceinline__ f32x16 logits(const uint8_t* k, int lane) const {
    const int row = lane & 31, h = lane >> 5;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < S::kSteps / 2; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(k + lds_offset<S::kRowBytes>(row, 2 * i + h));
        s = T::mfma(widen<T>((u32x2){w[0], w[1]}), q[2 * i], s);
        s = T::mfma(widen<T>((u32x2){w[2], w[3]}), q[2 * i + 1], s);
      }
    } else {
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) s = T::mfma(*reinterpret_cast<const u32x4*>(k + lds_offset<S::kRowBytes>(row, 2 * i + h)), q[i], s);
    }
    return s;
  }

  // V^T fragment: channels 32 b + (lane & 31), keys of step t (16 keys) in the order of the probabilities' registers.
  static __device__ __forceinline__ u32x4 value_fragment(const uint8_t* v, int lane, int t, int b) {
    const int h = lane >> 5, j = (lane >> 4) & 1, i = lane & 15;
    if constexpr (E4M3) {
      const int row = 16 * t + 4 * h + ((i >> 1) & 3) + 8 * (i >> 3);
      const uint8_t* p = v + lds_offset<S::kRowBytes>(row, 2 * b + j) + 8 * (i & 1);
      return widen<T>(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p)));
    } else {
      const int row = 16 * t + 4 * h + (i >> 2), chunk = 4 * b + 2 * j + ((i & 3) >> 1);
      const uint8_t* p0 = v + lds_offset<S::kRowBytes>(row, chunk) + 8 * (i & 1);
      const uint8_t* p1 = v + lds_offset<S::kRowBytes>(row + 8, chunk) + 8 * (i & 1);
      const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p0));
      const u32x2 c = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p1));
      return (u32x4){a[0], a[1], c[0], c[1]};
    }
  }

  // What the row of this lane does not see becomes -infinity.  key0: first key of the unit; absent: keys without a page.
  __device__ __forceinline__ void mask(f32x16& s, int key0, uint32_t absent, int h) const {
    const int first = key0 + 4 * h;
    absent >>= 4 * h;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int off = 8 * (r >> 2) + (r & 3), key = first + off;
      s[r] = (key < hi && key >= lo && !((absent >> off) & 1)) ? s[r] : -kInf;
    }
  }

  // m rises to kChunkLift below the largest of the unit's logits.
  __device__ __forceinline__ void raise(const f32x16& s, float c) {
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
    {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = c * fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) - T::kChunkLift;
    }
    const float next = fmaxf(m, top), alpha = next == -kInf ? 1.f : __builtin_amdgcn_exp2f(m - next);
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[b][r] *= alpha;
    l *= alpha;
    m = next;
  }
  // Fragment i of the unit's keys as it lies in LDS: a step's, or for 8-bit keys those of steps 2 i and 2 i + 1.
  static __device__ __forceinline__ u32x4 key_fragment(const uint8_t* k, int lane, int i) {
    return *reinterpret_cast<const u32x4*>(k + lds_offset<S::kRowBytes>(lane & 31, 2 * i + (lane >> 5)));
  }
  // The unit's probabilities in place of its logits `s` (c: softmax scale * log2 e, m as it is), and their sum; with NEXT, the logits `y` of the
  // unit whose keys begin at `k`.  A matrix instruction (32 cycles) depends on the one before it and a wave issues in order, so the vector
  // instructions are put between them: 16 / kSteps logits behind each.
  template <bool NEXT>
  __device__ __forceinline__ float soften(f32x16& s, float c, const uint8_t* k, int lane, f32x16& y) const {
    constexpr int kPer = 16 / S::kSteps;
    const float ref = m == -kInf ? 0.f : m;
    u32x4 kf[2];
    if constexpr (NEXT) {
      kf[0] = key_fragment(k, lane, 0);
      kf[1] = key_fragment(k, lane, 1);
#pragma unroll
      for (int r = 0; r < 16; ++r) y[r] = 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < S::kSteps; ++i) {
      if constexpr (NEXT) {
        if constexpr (E4M3) {
          const u32x4 f = kf[(i >> 1) & 1];
          y = T::mfma(widen<T>((u32x2){f[2 * (i & 1)], f[2 * (i & 1) + 1]}), q[i], y);
          if ((i & 1) && i + 3 < S::kSteps) kf[(i >> 1) & 1] = key_fragment(k, lane, (i >> 1) + 2);
        } else {
          y = T::mfma(kf[i & 1], q[i], y);
          if (i + 2 < S::kSteps) kf[i & 1] = key_fragment(k, lane, i + 2);
        }
      }
#pragma unroll
      for (int r = i * kPer; r < (i + 1) * kPer; ++r) {
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -ref));
        sum += s[r];
      }
      if constexpr (NEXT) __builtin_amdgcn_sched_barrier(0);
    }
    return sum;
  }

  // O += P V, with probabilities as pairs of 16-bit values: rounded to one they would be off by as much as the output's own rounding (errors 1.4 times as
  // large).  The second values' products use the fragments of V that the first ones' have brought; they and the splitting make a call 1.13 to 1.3 times as long
  // (20480 keys, 2 x 4096 rows of 32 heads, d = 128: 2607 -> 3377 us).
  __device__ __forceinline__ void add_values(const f32x16& x, const uint8_t* v, int lane) {
    constexpr int kAll = 2 * S::kBlocks;
    u32x4 vf[2] = {value_fragment(v, lane, 0, 0), value_fragment(v, lane, 1 / S::kBlocks, 1 % S::kBlocks)}, p[2], p_low[2];
    auto split = [&](int t, int e) {
      const float x0 = x[8 * t + 2 * e], x1 = x[8 * t + 2 * e + 1];
      p[t][e] = T::pack(x0, x1);
      p_low[t][e] = T::pack(x0 - T::low(p[t][e]), x1 - T::high(p[t][e]));
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) split(0, e);
#pragma unroll
    for (int n = 0; n < kAll; ++n) {
      const int t = n / S::kBlocks, b = n % S::kBlocks;
      o[b] = T::mfma(vf[n & 1], p[t], o[b]);
      o[b] = T::mfma(vf[n & 1], p_low[t], o[b]);
      if (n + 2 < kAll) vf[n & 1] = value_fragment(v, lane, (n + 2) / S::kBlocks, (n + 2) % S::kBlocks);
      if (n < S::kBlocks) {
#pragma unroll
        for (int e = n * 4 / S::kBlocks; e < (n + 1) * 4 / S::kBlocks; ++e) split(1, e);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Up to ROWS (16 or 32) query rows of one wave, in launches of few rows: the same products from 16 x 16 x 32 instructions where 16 rows are
// enough, which halves the registers of queries and outputs.  A row has 64 / ROWS lanes; lane part `j` of them holds the logits of
// keys kSpan (r / 4) + 4 j + r % 4, and of the output the channels kSpan q + 4 j .. + 3, quad by quad.
template <typename T, int D, bool E4M3, int ROWS>
struct FewRows {
  typedef Shape<D, E4M3> S;
  static constexpr int kSpan = 256 / ROWS;             // 16 or 8
  static constexpr int kLogits = ROWS / 2;             // of a lane, for 32 keys
  static constexpr int kSteps = D * ROWS / 512;        // matrix instructions of 16 or 32 channels
  static constexpr int kQuads = D / kSpan;
  typedef float acc_t __attribute__((ext_vector_type(ROWS == 32 ? 16 : 4)));
  static constexpr int kBlocks = D / ROWS;             // accumulators of ROWS channels
  u32x4 q[kSteps];
  acc_t o[kBlocks];
  float m, l;                                          // m: the reference, in log2 units; l: this lane's part of the keys
  int lo, hi;                                          // keys [lo, hi) are seen by this lane's row

  static __device__ __forceinline__ acc_t mfma(u32x4 a, u32x4 b, acc_t c) {
    if constexpr (ROWS == 32) return T::mfma(a, b, c);
    else return T::mfma16(a, b, c);
  }
  // First channel of the octet that lane part j brings to step s of the first product.
  static __device__ __forceinline__ int channel(int s, int j) {
    constexpr int kPart = 64 / ROWS;
    return E4M3 ? 16 * kPart * (s >> 1) + 16 * j + 8 * (s & 1) : 8 * kPart * s + 8 * j;
  }
  __device__ __forceinline__ float quad(int i, int e) const { return o[ROWS == 32 ? i >> 2 : i][ROWS == 32 ? 4 * (i & 3) + e : e]; }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = acc_t{};
    m = -kInf;
    l = 0.f;
  }
  __device__ __forceinline__ void load_queries(const uint8_t* row, int j) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const u32x4*>(row + 2 * channel(s, j));
  }
  // A value per lane part joined over a row's lanes.
  template <typename F>
  static __device__ __forceinline__ float over_row(float x, F&& f) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    if constexpr (ROWS == 16) {
      const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      x = f(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return x;
  }

  // Logits of the 32 keys whose rows begin at `k` in LDS.
  __device__ __forceinline__ void logits(const uint8_t* k, int lane, float (&x)[kLogits]) const {
    const int row = lane % ROWS, j = lane / ROWS;
#pragma unroll
    for (int part = 0; part < 32 / ROWS; ++part) {
      acc_t s{};
      const int at = row + part * ROWS;
      if constexpr (E4M3) {
#pragma unroll
        for (int i = 0; i < kSteps / 2; ++i) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(k + lds_offset<S::kRowBytes>(at, channel(2 * i, j) / 16));
          s = mfma(widen<T>((u32x2){w[0], w[1]}), q[2 * i], s);
          s = mfma(widen<T>((u32x2){w[2], w[3]}), q[2 * i + 1], s);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = mfma(*reinterpret_cast<const u32x4*>(k + lds_offset<S::kRowBytes>(at, channel(i, j) / 8)), q[i], s);
      }
#pragma unroll
      for (int r = 0; r < (ROWS == 32 ? 16 : 4); ++r) x[4 * part + r] = s[r];
    }
  }

  // V^T fragment: ROWS channels from ROWS * b on, the keys of logits 8 t .. 8 t + 7 of every lane part.
  static __device__ __forceinline__ u32x4 value_fragment(const uint8_t* v, int lane, int t, int b) {
    const int j = lane / ROWS, i = lane & 15, c0 = ROWS * b + (ROWS == 32 ? 16 * ((lane >> 4) & 1) : 0);
    const int first = 2 * kSpan * t + 4 * j;           // key of the first four logits, the other four kSpan further
    if constexpr (E4M3) {
      const int row = first + ((i >> 1) & 3) + kSpan * (i >> 3);
      const uint8_t* p = v + lds_offset<S::kRowBytes>(row, c0 / 16) + 8 * (i & 1);
      return widen<T>(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p)));
    } else {
      const int row = first + (i >> 2), chunk = c0 / 8 + ((i & 3) >> 1);
      const uint8_t* p0 = v + lds_offset<S::kRowBytes>(row, chunk) + 8 * (i & 1);
      const uint8_t* p1 = v + lds_offset<S::kRowBytes>(row + kSpan, chunk) + 8 * (i & 1);
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p0));
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p1));
      return (u32x4){x[0], x[1], y[0], y[1]};
    }
  }

  // What the row of this lane does not see becomes -infinity.  key0: first of the 32 keys; absent: keys without a page.
  __device__ __forceinline__ void mask(float (&x)[kLogits], int key0, uint32_t absent, int j) const {
    const int first = key0 + 4 * j;
    absent >>= 4 * j;
#pragma unroll
    for (int r = 0; r < kLogits; ++r) {
      const int off = kSpan * (r >> 2) + (r & 3), key = first + off;
      x[r] = (key < hi && key >= lo && !((absent >> off) & 1)) ? x[r] : -kInf;
    }
  }

  // The probabilities in place of the logits (c: softmax scale * log2 e), and their sum; raises m where it has to.
  __device__ __forceinline__ void soften(float (&x)[kLogits], float c) {
    float top = fmaxf(x[0], x[1]);
#pragma unroll
    for (int r = 2; r < kLogits; ++r) top = fmaxf(top, x[r]);
    top = c * over_row(top, [](float a, float b) { return fmaxf(a, b); }) - T::kFewLift;
    if (__ballot(top > m + T::kFewGap)) {                    // (also the first key of a row, whose m is -infinity)
      const float next = fmaxf(m, top), alpha = next == -kInf ? 1.f : __builtin_amdgcn_exp2f(m - next);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < (ROWS == 32 ? 16 : 4); ++r) o[b][r] *= alpha;
      l *= alpha;
      m = next;
    }
    const float ref = m == -kInf ? 0.f : m;
#pragma unroll
    for (int r = 0; r < kLogits; ++r) {
      x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, -ref));
      l += x[r];
    }
  }

  // O += P V, with probabilities as a pair of 16-bit values, so that they are not rounded before the output is (the matrix cores have time).
  __device__ __forceinline__ void add_values(const float (&x)[kLogits], const uint8_t* v, int lane) {
#pragma unroll
    for (int t = 0; t < kLogits / 8; ++t) {
      u32x4 p, p_low;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x0 = x[8 * t + 2 * e], x1 = x[8 * t + 2 * e + 1];
        p[e] = T::pack(x0, x1);
        p_low[e] = T::pack(x0 - T::low(p[e]), x1 - T::high(p[e]));
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const u32x4 f = value_fragment(v, lane, t, b);
        o[b] = mfma(f, p, o[b]);
        o[b] = mfma(f, p_low, o[b]);
      }
    }
  }
};

// The page of key `key` of a sequence of `len` tokens (one lane a key): keys behind the end take the last one's.
__device__ __forceinline__ int32_t page_of_key(const Call& c, int b, int key, int len) {
  return page_of(c, b, min(key, len - 1) >> c.page_shift);
}
__device__ __forceinline__ uint64_t row_offset(const Call& c, int32_t page, int key) { return slot_offset(c, page, key & ((1 << c.page_shift) - 1)); }

// Infinite values and NaN among the values.  A row that sees such a value has it in that channel, whatever its weight (the sum of them, where there are
// several), and a row that does not see it has no part of it.  The products give neither: a probability that is zero in its type times an infinity is NaN, and
// so may be a pair's second value times one.  So the values of keys that some rows of a workgroup or wave see and others do not ("mixed" runs, see mixed() in
// the kernels) come into LDS without such (clean tells whether there were any).  Where there were, or where an output is not finite, set_odd_values
// looks all values through again and puts the outputs of the rows that see such values right, where those lie in memory.  Rare; all lanes of a
// wave together, KEYS keys at a time.  A lane has one row, which sees keys [lo, hi), and of its channels the quads span * q + 4 * part .. + 3;
// clear(q, e) makes the e-th of quad q zero, add(q, e, x) adds x to it.
template <typename T, bool E4M3>
__device__ __forceinline__ bool clean(u32x4& r) {
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = finite_part<T, E4M3>(r[e]);
    odd |= w != r[e];
    r[e] = w;
  }
  return odd;
}
template <typename T, int D, bool E4M3, int KEYS, typename CLEAR, typename ADD>
__device__ __forceinline__ void set_odd_values(const Call& c, int b, int head, int len, int k0, int k1, int step, int lo, int hi, int span, int part, CLEAR clear,
                                               ADD add) {
  constexpr int kPieces = D * (E4M3 ? 1 : 2) / 16;
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass)
#pragma unroll 1
    for (int u = k0; u < k1; u += step) {
      const int mine = u + lane % KEYS;
      const int32_t page = page_of_key(c, b, mine, len);
      bool odd = false;
      if (page >= 0 && mine < len) {
        const uint8_t* v = c.v + head_offset(c, head) + row_offset(c, page, mine);
#pragma unroll 4
        for (int i = 0; i < kPieces; ++i) {
          u32x4 w = *reinterpret_cast<const u32x4*>(v + 16 * i);
          odd |= clean<T, E4M3>(w);
        }
      }
      uint64_t keys = __ballot(odd);
      if (KEYS == 32) keys &= 0xFFFFFFFFull;                 // (two lanes had each key)
      for (; keys; keys &= keys - 1) {
        const int i = __ffsll((unsigned long long)keys) - 1;
        const uint8_t* v = c.v + head_offset(c, head) + row_offset(c, __shfl(page, i), u + i);
        const bool sees = u + i >= lo && u + i < hi;
#pragma unroll 1
        for (int q = 0; q * span < D; ++q) {
          const int ch = q * span + 4 * part;
          uint32_t w[2];
          if constexpr (E4M3) {
            const uint32_t x = *reinterpret_cast<const uint32_t*>(v + ch);
            w[0] = T::template from_e4m3<false>(x);
            w[1] = T::template from_e4m3<true>(x);
          } else {
            w[0] = *reinterpret_cast<const uint32_t*>(v + 2 * ch);
            w[1] = *reinterpret_cast<const uint32_t*>(v + 2 * ch + 4);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = e & 1 ? T::high(w[e >> 1]) : T::low(w[e >> 1]);
            if (sees && !(fabsf(x) < kInf)) {
              if (pass == 0) clear(q, e);
              else add(q, e, x);
            }
          }
        }
      }
    }
}

// Which rows a workgroup works on: row tile `t` of sequence `b`; false: none.
__device__ __forceinline__ bool find_tile(const AttendArgs& a, int tile, int tile_rows, int& b, int& t) {
  if (a.tiles_per_seq > 0) {
    b = tile / a.tiles_per_seq;
    t = tile - b * a.tiles_per_seq;
    return true;
  }
  const int lane = threadIdx.x & 63;
  int before = 0;                                        // tiles of the sequences passed
  for (int base = 0; base < a.c.n_seqs; base += 64) {
    const int s = base + lane;
    int mine = 0;
    if (s < a.c.n_seqs) mine = (sequence(a.c, s).n * a.c.group + tile_rows - 1) / tile_rows;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const int total = __shfl(upto, 63);
    if (tile < before + total) {
      const uint64_t behind = __ballot(before + upto <= tile);
      const int at = __popcll(behind);                   // ascending, so these are the lanes in front
      b = base + at;
      t = tile - before - (at ? __shfl(upto, at - 1) : 0);
      return true;
    }
    before += total;
  }
  return false;
}
// The keys that row tile t of a sequence reads: [lo, hi), lo on a multiple of 64.
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range tile_range(const AttendArgs& a, const Seq& s, int row0, int n_rows) {
  const int place0 = s.len - s.n + row0 / a.c.group, place1 = s.len - s.n + (row0 + n_rows - 1) / a.c.group;
  Range r;
  r.hi = a.causal ? min(s.len, place1 + 1) : s.len;
  r.lo = a.window > 0 ? max(0, place0 + 1 - a.window) & ~63 : 0;
  return r;
}
// How many key ranges that is; the last range of the launch ends where the tile's keys do.
__device__ __forceinline__ int splits_of(const AttendArgs& a, const Range& r) {
  return r.hi > r.lo ? min(a.splits, (r.hi - r.lo + a.split_keys - 1) / a.split_keys) : 1;
}
__device__ __forceinline__ int split_end(const AttendArgs& a, const Range& r, int split) {
  return split == a.splits - 1 ? r.hi : min(r.hi, r.lo + (split + 1) * a.split_keys);
}

// ---- launches of few rows: a column is a sequence's keys for one key head, a unit kFewKeys of them ----------------------
__device__ __forceinline__ int units_of(const AttendArgs& a, const Seq& s) {
  if (s.n == 0) return 0;
  const Range r = tile_range(a, s, 0, s.n * a.c.group);
  return r.hi > r.lo ? (r.hi - r.lo + kFewKeys - 1) / kFewKeys : 0;
}
// Sixty-four sequences, one a lane, with the units of one key head in front of and in them.
struct Lanes {
  int base;                     // sequence of lane 0
  Seq mine;
  int units, upto;              // of this lane's sequence; up to it within the sixty-four
  int before, all;              // in front of the sixty-four; in all of them
};
__device__ __forceinline__ Lanes load_lanes(const AttendArgs& a, int base, int before) {
  const int lane = threadIdx.x & 63, b = base + lane;
  Lanes x;
  x.base = base;
  x.before = before;
  x.mine = Seq{0, 0, 0};
  if (b < a.c.n_seqs) x.mine = sequence(a.c, b);
  x.units = units_of(a, x.mine);
  x.upto = x.units;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x.upto, o);
    if (lane >= o) x.upto += y;
  }
  x.all = __shfl(x.upto, 63);
  return x;
}
// Units of a worker's share: columns one after the other (sequence by sequence, head by head) are cut into even shares.
__device__ __forceinline__ int share_of(const AttendArgs& a, int total) { return max(1, (total + a.workers - 1) / a.workers); }

struct Column {
  int b, head;
  Seq s;
  int first, units;             // among all units
};
// The column of unit `unit`, which is one and no earlier than `x`'s sequences; x moves on to its sequences.
__device__ __forceinline__ Column column_of(const AttendArgs& a, int unit, Lanes& x) {
  const int hkv = a.c.hkv;
  while (unit >= (x.before + x.all) * hkv) x = load_lanes(a, x.base + 64, x.before + x.all);
  const int at = __popcll(__ballot((x.before + x.upto) * hkv <= unit));
  Column c;
  c.units = __shfl(x.units, at);
  const int first = x.before + __shfl(x.upto, at) - c.units;
  c.b = x.base + at;
  c.s = Seq{__shfl(x.mine.first, at), __shfl(x.mine.n, at), __shfl(x.mine.len, at)};
  c.head = (unit - first * hkv) / c.units;
  c.first = first * hkv + c.head * c.units;
  return c;
}

}  // namespace paged
}  // namespace kvx
