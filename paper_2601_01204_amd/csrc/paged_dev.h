// Shared declarations of the paged cache: what its host side (paged_api.hip) hands to its kernels (paged_*.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvx {
namespace paged {

struct Rows {                   // strides in bytes
  uint8_t* p;
  int64_t tok, head;
};

// One call's geometry.
struct Call {
  uint8_t* k;
  uint8_t* v;
  uint32_t page_stride, slot_stride, head_stride;      // of the pool, in pieces of 16 bytes
  const int32_t* table;
  int64_t table_stride;
  const float* k_scale;
  const float* v_scale;
  float* weights;               // [n_pages][Hkv][page_size]
  int32_t* ids;                 // [n_pages][Hkv][page_size]
  const int32_t* start;
  const int32_t* lens;
  const int32_t* seen;          // never NULL (kv_lens where the caller gave none)
  int32_t* status;              // sticky bits of kv_paged_status
  int32_t n_pages, n_seqs, n_tokens, max_new, max_len;
  int32_t hq, hkv, group;       // group = hq / hkv
  int32_t page_shift;
};

constexpr int kStatusPage = 1, kStatusLength = 2;

constexpr int kFewRows = 32, kChunkRows = 128;        // row tiles of the two attention kernels
constexpr int kFewKeys = 128;                         // a unit of keys in launches of few rows

struct AppendArgs {
  Call c;
  Rows q, q_out, k, v;
  const int32_t* positions;     // NULL: the ids
  const uint64_t* turns;        // [rotary / 2] turns per position, a fraction of 2^64
  float magnitude;
  int32_t rotary;
};

struct AttendArgs {
  Call c;
  Rows q, out;
  float* lse;                   // [n_tokens][hq] natural logarithm; NULL: not wanted
  float* part_o;                // partial results of a launch with splits: [block][row][d], and [block][row] (max, sum)
  float2* part_ml;
  const float* weights_in;
  float* weights_out;
  float* weight_part;           // [weight_splits][sequence][key head][weight_stride] sums over parts of the rows, where there is more than one
  int32_t weight_splits, weight_rows, weight_stride;            // weight_rows: of a part
  float* logits;                // launches of few rows that collect weights: [tile][key head][row][logit_stride], log2 units; NULL: not kept
  int64_t logit_stride;
  float factor;                 // softmax scale * log2(e)
  int32_t causal, window;
  int32_t tiles;                // row tiles of the launch (all sequences), per key head and split
  int32_t tiles_per_seq;        // > 0: tile t is tile t % tiles_per_seq of sequence t / tiles_per_seq; 0: tiles are counted out
  int32_t splits;               // key ranges per row tile
  int32_t split_keys;           // keys of a range, a multiple of 64
  int32_t part_rows;            // rows a block has in part_o
  int32_t workers;              // launches of few rows: workgroups that share the keys of all columns evenly, two places each in part_o;
                                // 0: a workgroup to each column
};

struct EvictArgs {
  Call c;
  float* weights_out;
  int32_t* ids_out;
  int32_t* lens_out;
  int2* moves;                  // [sequence][head][max_moves] (from, to) places
  int32_t* n_moves;             // [sequence][head]
  int32_t budget, sinks, recent, max_moves;
};

// ---- workgroups of each launch -------------------------------------------------------
// The runtime takes fewer than 2^32 threads in a dimension; calls that would need more are refused before anything is enqueued.
struct Grid {
  int64_t x = 0, y = 1;
  int32_t threads = 256;
  bool fits() const { return x * threads < (1ll << 32) && y <= 65536; }
};
constexpr int kSelectThreads = 1024;
constexpr int kFewMoves = 256;                        // as many rows of a (sequence, key head) are moved by the workgroup that selects
constexpr int kWeightKeys = 128;                      // keys of a workgroup of the launch that forms weights again
inline int64_t parts_of(int64_t n, int64_t size) { return (n + size - 1) / size; }
// All pieces (of 64 lanes, for a token) in one wave where that leaves four waves a SIMD on 256 units, one each for fewer tokens.
inline int append_turns(const AppendArgs& a, int d) { return (int)parts_of((int64_t)((a.q.p ? a.c.hq : 0) + 2 * a.c.hkv) * (d >> 4), 64); }
inline int append_units(const AppendArgs& a, int d) { return (int64_t)a.c.n_tokens * parts_of(append_turns(a, d), 6) >= 4096 ? 6 : 1; }
inline Grid append_grid(const AppendArgs& a, int d) { return Grid{parts_of(a.c.n_tokens * parts_of(append_turns(a, d), append_units(a, d)), 4)}; }
inline Grid attend_grid(const AttendArgs& a) { return Grid{a.workers ? a.workers : (int64_t)a.tiles * a.c.hkv * a.splits}; }
// Rows of new tokens that a workgroup of the join takes: of few rows one, or one a wave; of more, 1024 / d of a tile.
inline int merge_waves(const AttendArgs& a) { return (int64_t)a.c.n_tokens * a.c.hq * 8 < a.workers ? 4 : 1; }
inline int merge_slices(const AttendArgs& a, int d) { return (int)parts_of(a.part_rows, 1024 / d); }
inline Grid merge_grid(const AttendArgs& a, int d) {
  if (a.workers) return Grid{parts_of((int64_t)a.c.n_tokens * a.c.hq * merge_waves(a), 4)};
  return Grid{(int64_t)a.tiles * a.c.hkv * merge_slices(a, d)};
}
// Keys and heads in one dimension, sequences and parts of the rows in the other: max_len is a bound that may be generous.
inline Grid weights_grid(const AttendArgs& a) { return Grid{parts_of(a.c.max_len, kWeightKeys) * a.c.hkv, (int64_t)a.c.n_seqs * a.weight_splits}; }
inline Grid weights_sum_grid(const AttendArgs& a) { return Grid{parts_of(a.c.max_len, 256) * a.c.hkv, a.c.n_seqs}; }
inline Grid weights_from_logits_grid(const AttendArgs& a) { return Grid{parts_of(a.c.max_len, 4 * 256) * a.c.hkv, a.c.n_seqs}; }
inline Grid select_grid(const EvictArgs& a) { return Grid{(int64_t)a.c.n_seqs * a.c.hkv, 1, kSelectThreads}; }

// ---- launchers (each enqueues on `st`, never synchronises) --------------------------
// dtype: KV_BF16 or KV_F16; e4m3: the pages hold 8-bit floats.
void launch_append(const AppendArgs& a, int d, int dtype, bool e4m3, bool interleaved, hipStream_t st);
void launch_attend(const AttendArgs& a, int d, int dtype, bool e4m3, int tile_rows, hipStream_t st);
void launch_merge(const AttendArgs& a, int d, int dtype, bool e4m3, hipStream_t st);
void launch_weights_from_logits(const AttendArgs& a, hipStream_t st);
void launch_weights(const AttendArgs& a, int d, int dtype, bool e4m3, hipStream_t st);
// arrived: [n_seqs], zero before and after
void launch_evict(const EvictArgs& a, int d, bool e4m3, int32_t* arrived, hipStream_t st);

}  // namespace paged
}  // namespace kvx
