// Rotary positions of a call's queries and keys, and the new tokens' keys and values into their pages.
//
// y1 = x1 cos a - x2 sin a, y2 = x2 cos a + x1 sin a for a pair of channels, a = position * w_i.  The angle is taken in turns:
// w_i / 2 pi is held as a fraction of 2^64, and the product with the position modulo 2^64 is the phase with an error below
// 2^-33 turns at any int32 position (in fp32 the angle of position 10^6 is off by 0.06 radians).  Sine and cosine, the products and the sum are fp32,
// rounded once to the type of the output.
//
// Bound by memory: a token is read and written once.  A wave works on one token; a lane moves 16 channels of a head at a time (two
// 16-byte loads): the two octets of a rotated pair range, or 16 neighbours.  A lane keeps the same channels in every head, so its
// eight sines and cosines are formed once: lane i forms pair i's, they cross lanes through LDS.  Where a token belongs takes three loads that
// wait for one another, so the token's own rows (up to UNITS pieces a lane) are requested before them.  6700 tokens of 32 query and 8 key heads into 8 bits:
// 35.4 us, 4.3 TB/s read and written; one token: the launch.
#include "../../include/kvx.h"
#include "paged_types.h"

namespace kvx {
namespace paged {

namespace {

constexpr int kWaves = 4;
constexpr int kMaxPairs = 64;

template <typename T>
__device__ __forceinline__ void floats(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = T::low(w[i]);
    x[2 * i + 1] = T::high(w[i]);
  }
}
template <typename T>
__device__ __forceinline__ void store8(uint8_t* p, const float (&x)[8]) {
  *reinterpret_cast<u32x4*>(p) = (u32x4){T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7])};
}
// x / scale to nearest even in 8 bits; beyond +-448 the largest value (the conversion saturates), NaN stays NaN
__device__ __forceinline__ void store8_e4m3(uint8_t* p, const float (&x)[8], float scale) {
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = x[4 * i + e] / scale;
      y[e] = y[e] > 448.f ? 448.f : (y[e] < -448.f ? -448.f : y[e]);
    }
    int b = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], b, true);
  }
  *reinterpret_cast<u32x2*>(p) = w;
}

template <typename T, bool E4M3, bool INTERLEAVED, int UNITS>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(const AppendArgs a, const int d, const int slabs) {
  __shared__ float2 trig[kWaves][kMaxPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Call& c = a.c;
  const int64_t job = (int64_t)blockIdx.x * kWaves + wave;
  const int t = (int)(job / slabs), slab = (int)(job - (int64_t)t * slabs);
  if (t >= c.n_tokens) return;                       // whole waves leave; nothing below waits for another wave

  // units of 16 channels: a head has d / 16; a multiple of them fits 64, so a lane's unit within its head is always the same
  const int pairs = a.rotary >> 1, per_head = d >> 4, u = lane & (per_head - 1);
  // The unit's two octets, so that neighbouring lanes have neighbouring octets: interleaved, octet u of each half of the head, pairs 4 c / 8 ..
  // of both; half layout, the octets of pairs 8 u .. 8 u + 7, or octet u of each half of the channels that pass.
  const int whole = a.rotary >> 4;                   // (half layout) units that turn
  const bool turned = INTERLEAVED ? 8 * u < a.rotary : u < whole;
  const int c0 = INTERLEAVED || turned ? 8 * u : a.rotary + 8 * (u - whole);
  const int c1 = INTERLEAVED ? c0 + 8 * per_head : turned ? c0 + pairs : c0 + 8 * (per_head - whole);
  const bool turned1 = INTERLEAVED ? c1 < a.rotary : turned;
  const int hq = a.q.p ? c.hq : 0, heads = hq + 2 * c.hkv, heads_at_once = 64 / per_head;
  const int h0 = heads_at_once * UNITS * slab + lane / per_head;
  u32x4 raw[UNITS][2];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int h = h0 + i * heads_at_once;
    if (h >= heads) break;
    const bool is_q = h < hq, is_v = h >= hq + c.hkv;
    const Rows& from = is_q ? a.q : (is_v ? a.v : a.k);
    const uint8_t* src = from.p + (int64_t)t * from.tok + (int64_t)(is_q ? h : is_v ? h - hq - c.hkv : h - hq) * from.head;
    raw[i][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 2 * c0));
    raw[i][1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 2 * c1));
  }

  const int b = sequence_of_row(c, t);
  if (b < 0) return;
  const Seq s = sequence(c, b);
  const int row = t - s.first;
  if (row < 0 || row >= s.n) return;
  const int place = s.len - s.n + row;               // negative: the sequence is shorter than its new tokens
  const int token = c.seen[b] - s.n + row;
  const int page = place >= 0 ? page_of(c, b, place >> c.page_shift) : -1;
  const int slot = place & ((1 << c.page_shift) - 1);
  if (page < 0 && lane == 0) atomicOr(c.status, place < 0 ? kStatusLength : kStatusPage);

  if (lane < pairs) {
    const int position = a.positions ? a.positions[t] : token;
    const uint64_t phase = (uint64_t)(int64_t)position * a.turns[lane];
    float sn, cs;
    sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &sn, &cs);      // half turns
    trig[wave][lane] = make_float2(cs * a.magnitude, sn * a.magnitude);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                // the table crosses lanes of this wave only
  __builtin_amdgcn_wave_barrier();

  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 w = trig[wave][INTERLEAVED ? (i < 4 ? (turned ? (c0 >> 1) + i : 0) : (turned1 ? (c1 >> 1) + i - 4 : 0)) : (turned ? 8 * u + i : 0)];
    cs[i] = w.x;
    sn[i] = w.y;
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int h = h0 + i * heads_at_once;
    if (h >= heads) break;
    const bool is_q = h < hq, is_v = h >= hq + c.hkv;
    const int kv = is_q ? 0 : (is_v ? h - hq - c.hkv : h - hq);
    float x0[8], x1[8];
    floats<T>(raw[i][0], x0);
    floats<T>(raw[i][1], x1);
    if (turned && !is_v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float& lo = INTERLEAVED ? (e < 4 ? x0[2 * e] : x1[2 * e - 8]) : x0[e];
        float& hi = INTERLEAVED ? (e < 4 ? x0[2 * e + 1] : x1[2 * e - 7]) : x1[e];
        const float y0 = lo * cs[e] - hi * sn[e], y1 = hi * cs[e] + lo * sn[e];
        if (!INTERLEAVED || e < 4 || turned1) {
          lo = y0;
          hi = y1;
        }
      }
    }
    if (is_q) {
      uint8_t* dst = a.q_out.p + (int64_t)t * a.q_out.tok + (int64_t)h * a.q_out.head;
      store8<T>(dst + 2 * c0, x0);
      store8<T>(dst + 2 * c1, x1);
    } else if (page >= 0) {
      uint8_t* dst = (is_v ? c.v : c.k) + slot_offset(c, page, slot) + head_offset(c, kv);
      if constexpr (E4M3) {
        const float* scales = is_v ? c.v_scale : c.k_scale;
        const float scale = scales ? scales[kv] : 1.0f;
        store8_e4m3(dst + c0, x0, scale);
        store8_e4m3(dst + c1, x1, scale);
      } else {
        store8<T>(dst + 2 * c0, x0);
        store8<T>(dst + 2 * c1, x1);
      }
      if (u == 0 && !is_v) {
        const int64_t at = (((int64_t)page * c.hkv + kv) << c.page_shift) + slot;
        if (c.ids) c.ids[at] = token;
        if (c.weights) c.weights[at] = 0.f;
      }
    }
  }
}

}  // namespace

void launch_append(const AppendArgs& a, int d, int dtype, bool e4m3, bool interleaved, hipStream_t st) {
  const dim3 grid((unsigned)append_grid(a, d).x);
  auto go = [&](auto t, auto f8, auto inter) {
    // a wave with six turns has all of up to 48 heads of 128 channels: 6700 tokens of 48 heads 38.5 us with four turns a wave, 36.4 with six
    auto with = [&](auto units) {
      constexpr int kUnits = decltype(units)::value;
      append_kernel<decltype(t), decltype(f8)::value, decltype(inter)::value, kUnits>
          <<<grid, dim3(64 * kWaves), 0, st>>>(a, d, (int)parts_of(append_turns(a, d), kUnits));
    };
    if (append_units(a, d) == 6) with(std::integral_constant<int, 6>{});
    else with(std::integral_constant<int, 1>{});
  };
  auto by_layout = [&](auto t, auto f8) {
    if (interleaved) go(t, f8, std::true_type{});
    else go(t, f8, std::false_type{});
  };
  auto by_cache = [&](auto t) {
    if (e4m3) by_layout(t, std::true_type{});
    else by_layout(t, std::false_type{});
  };
  if (dtype == KV_F16) by_cache(Half{});
  else by_cache(Brain{});
}

}  // namespace paged
}  // namespace kvx
