// What the paged cache's kernels share: the 16-bit input types (conversions and matrix instructions), and where a row, a token and a
// page are found.
#pragma once
#include "paged_dev.h"

namespace kvx {
namespace paged {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

struct Half {
  static constexpr uint32_t kExponent = 0x7C00u;
  // How softmax places probabilities in the type's range (paged_tile.h): fp16's least step is 2^-24 and its largest value 2^16, so references lie below
  // the largest logit.
  static constexpr float kFewLift = 14.0f, kFewGap = 1.0f, kChunkLift = 10.0f;
  // two floats rounded to nearest even, the first in the low half
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
  }
  static __device__ __forceinline__ float low(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
  static __device__ __forceinline__ float high(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  // two 8-bit floats (bytes 0, 1 or 2, 3 of a word): exact
  template <bool UPPER> static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, UPPER));
  }
};
struct Brain {
  static constexpr uint32_t kExponent = 0x7F80u;
  static constexpr float kFewLift = 0.0f, kFewGap = 8.0f, kChunkLift = 0.0f;      // (the range of fp32)
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
  }
  static __device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  template <bool UPPER> static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, UPPER));
  }
};

// A word without its infinities and NaN (two values of T, or four of 8 bits, which have no infinities).
template <typename T, bool E4M3>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  if constexpr (E4M3) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 32; i += 8) r |= ((w >> i) & 0x7Fu) == 0x7Fu ? 0u : w & (0xFFu << i);
    return r;
  } else {
    return ((w & T::kExponent) == T::kExponent ? 0u : w & 0xFFFFu) | (((w >> 16) & T::kExponent) == T::kExponent ? 0u : w & 0xFFFF0000u);
  }
}

// Eight 8-bit floats as eight values of T, in order.
template <typename T>
__device__ __forceinline__ u32x4 widen(u32x2 w) {
  return (u32x4){T::template from_e4m3<false>(w[0]), T::template from_e4m3<true>(w[0]), T::template from_e4m3<false>(w[1]),
                 T::template from_e4m3<true>(w[1])};
}

// ---- device helpers ----------------------------------------------------------------
// The sequence of a batch, with lengths cut to what the host promised.
struct Seq {
  int32_t first, n, len;        // first row, new rows, cached length
};
__device__ __forceinline__ Seq sequence(const Call& c, int b) {
  const int32_t a0 = c.start[b], a1 = c.start[b + 1], l0 = c.lens[b];
  Seq s;
  s.first = min(max(a0, 0), c.n_tokens);
  s.n = min(max(min(a1, c.n_tokens) - s.first, 0), c.max_new);
  s.len = min(max(l0, 0), c.max_len);
  if (s.first != a0 || s.first + s.n != a1 || s.len != l0) atomicOr(c.status, kStatusLength);
  return s;
}
// What is the same in all lanes, in scalar registers: branches on it are scalar too.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Seq uniform(const Seq& s) { return Seq{uniform(s.first), uniform(s.n), uniform(s.len)}; }
// Page number of entry `entry` of sequence b; -1 for one outside the pool.
__device__ __forceinline__ int32_t page_of(const Call& c, int b, int entry) {
  const int32_t page = c.table[(int64_t)b * c.table_stride + entry];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}
// Bytes from the pool's beginning to a slot of a page (0 for a page outside the pool) and a key head: 32 x 32-bit products, since 64-bit ones
// take a wave a hundred cycles.
__device__ __forceinline__ uint64_t slot_offset(const Call& c, int32_t page, int slot) {
  return ((uint64_t)(uint32_t)(page < 0 ? 0 : page) * c.page_stride + (uint64_t)(uint32_t)slot * c.slot_stride) << 4;
}
__device__ __forceinline__ uint64_t head_offset(const Call& c, int head) { return ((uint64_t)(uint32_t)head * c.head_stride) << 4; }
__device__ __forceinline__ void note_bad_page(const Call& c) { atomicOr(c.status, kStatusPage); }
// The sequence that row t belongs to (-1: none), found by all lanes of a wave together; t is the same in all of them.
// Sequences with no rows are passed over: the answer is the last one that begins at or before t.
__device__ __forceinline__ int sequence_of_row(const Call& c, int t) {
  const int lane = threadIdx.x & 63;
  int below = 0;
  for (int base = 0; base < c.n_seqs; base += 64) {
    const int s = base + lane;
    below += __popcll(__ballot(s < c.n_seqs && c.start[s] <= t));
    if (base + 64 < c.n_seqs && c.start[base + 64] > t) break;      // ascending: nothing further begins before t
  }
  const int b = below - 1;
  if (b < 0) return -1;
  return t < c.start[b + 1] ? b : -1;
}

}  // namespace paged
}  // namespace kvx
