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
