// layer.h - host-side argument structures of the operators around the attention
// in a layer (cross attention, rotary positions).  Apart from internal.h, which
// the attention's and the composition's build ids cover: what profiles report for
// a build of theirs does not hinge on these.
#pragma once

#include "internal.h"
#include "kernel_lds.h"

namespace ditango {

// A launch has fewer than 2^31 workgroups and 2^32 threads.
inline bool launch_fits(int64_t workgroups, int threads) {
  return workgroups <= 0x7fffffff && workgroups * threads <= 0xffffffffLL;
}

// One launch of the cross attention.  The rows of a key/value head are those
// of the query heads that share it: row r is token r / G of head hk * G + r % G.
// Strides are in elements.
struct CrossArgs {
  const void* q;            // rows of D elements, as the strides say
  const void* k;
  const void* v;
  void* out;                // [B][q_len][H][D]
  float* lse;               // [B][H][q_len] or null
  int64_t q_batch, q_token, q_head;
  int64_t k_batch, k_token, k_head;
  int64_t v_batch, v_token, v_head;
  int64_t q_len;
  int B, H, Hk, G;
  int kv_len;               // keys of a sequence, at most
  int rows;                 // q_len * G
  int row_tiles;            // ceil(rows / rows per workgroup)
  int split;                // key ranges, each a workgroup's: equal shares of
  int chunk;                // a sequence's keys, or (> 0) this many each
  uint32_t g_inverse;       // 2^32 / G, rounded up (G > 1)
  int class_tasks;          // of the task kernel: the tasks of a class, and
  int classes;              // the classes
  uint32_t tiles_inverse, heads_inverse, batch_inverse;   // of its divisions
  float scale_log2;
  const int32_t* lens;      // [B] live keys of a sequence (a prefix), or null
  const uint8_t* mask;      // [B][kv_len] or null
  // the masked form, in the workspace: how many keys are live [B], and either
  // their places in order [B][kv_len] and a row of zeros, or their rows
  // [B][kv_len][Hk][D]
  int32_t* count;
  int32_t* list;
  float* zeros;
  void* packed_k;
  void* packed_v;
  // partial states of a split launch, in the workspace
  float* part_out;          // [split][B][H][q_len][D]
  float* part_lse;          // [split][B][H][q_len]
};

// Live keys of sequence b.
__device__ __forceinline__ int cross_keys(const CrossArgs& a, int b) {
  if (a.mask != nullptr) return a.count[b];
  return a.lens == nullptr ? a.kv_len : min(max(a.lens[b], 0), a.kv_len);
}

// How a launch of the cross attention runs on the current device, and the
// workspace it takes.
inline size_t align_up256(size_t x) { return (x + 255) & ~(size_t)255; }
struct CrossPlan {
  // kRows: 128 rows a workgroup, key ranges in others; kTask: 256 rows, one
  // after another (cross_task.hip; a masked call's live keys are packed for
  // it); kResident: the head's keys in LDS (cross_resident.hip); kFew: chunks
  // of keys (cross_few.hip)
  enum Form { kRows, kTask, kResident, kFew } form;
  int split, chunk;
  size_t need;              // bytes of a masked call
  size_t bytes;             // with the partial states: without room for them the launch is not split
};
hipError_t plan_cross(const CrossArgs& a, ditango_dtype dt, int D, CrossPlan* p);
hipError_t launch_cross(const CrossArgs& a, const CrossPlan& p, ditango_dtype dt, int D, void* ws, size_t ws_bytes,
                        hipStream_t s);
bool cross_task_fits(const CrossArgs& a, int D);
hipError_t launch_cross_task(const CrossArgs& a, int D, hipStream_t s);
int cross_resident_keys(int D);     // at most
int cross_resident_waves(int D);    // of a workgroup, one per compute unit
bool cross_resident_lists(const CrossArgs& a, int D);   // a masked call lists its live keys by itself
hipError_t launch_cross_resident(const CrossArgs& a, int D, hipStream_t s);
hipError_t launch_cross_few(const CrossArgs& a, int D, hipStream_t s);
hipError_t launch_cross_f32(const CrossArgs& a, int D, hipStream_t s);
int cross_f32_rows(const CrossArgs& a, int D, int cus);   // rows per workgroup

// One launch of the rotary positions.
struct RotaryArgs {
  ditango_rotary_tensor t[2];
  int n;                    // tensors
  int B;
  int64_t S;
  int rot;                  // rotated dims
  int axes;
  const int32_t* pos;       // [1 or B][S][axes]
  int64_t pos_batch;        // 0, or S * axes
  float factor;             // of cosine and sine
  float eps;
  // the launch: a team of threads per token
  int team;
  int tokens;               // of a workgroup
  int units[2];             // of a token of each tensor
  double turns[DITANGO_ROTARY_MAX_PAIRS];    // of a pair, per position
  uint8_t axis[DITANGO_ROTARY_MAX_PAIRS];
};
hipError_t launch_rotary(const RotaryArgs& a, ditango_dtype dt, int D, ditango_rotary_layout layout,
                         ditango_rotary_norm norm, hipStream_t s);

}  // namespace ditango
