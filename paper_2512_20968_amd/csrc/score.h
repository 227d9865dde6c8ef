// Internal interface of the tile attention under a score rule: what the host
// (score.cpp) passes to the kernels (score_fwd.hip, score_bwd.hip).  Not part of
// the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache.h"

namespace mesh_attn {

constexpr int kScoreRows = 128;   // query rows of a workgroup (dK/dV: keys)
constexpr int kScoreBlock = 64;   // rows of a tile staged in LDS
constexpr int kScoreMaxList = 256;

// The tile as all kernels read it.  The KV buffer is cut into segments: list
// entries, those merged that go on where the last one ended (contiguous
// partitions p, p + 1).  Row r of segment s is row seg_row[s] + r of the buffer
// and has position seg_pos[s] + r * step.
struct ScoreTile {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;  // elements from row to row
  const int32_t* key_begin;  // [rows_q] or null
  const int32_t* key_end;
  const float* slopes;  // [hq] or null
  int32_t rows_q, rows_kv;
  int32_t hq, hkv, group, head_dim;
  int32_t P, n, striped, step, causal, total;
  float scale;       // softmax scale
  float scale_log2;  // .. * log2(e)
  float cap;         // 0: none
  int32_t nseg, kv_blocks64, kv_blocks128;  // blocks of the segments
  int32_t seg_row[kScoreMaxList + 1], seg_pos[kScoreMaxList];
  int32_t q_idx[kScoreMaxList];
};

struct ScoreFwdParams {
  ScoreTile t;
  void* o;
  float* lse;
  // Partial results of keys that are cut into `splits` parts, in the layout that
  // the merge reads: [split][rows][hq][d], [split][hq][rows].
  float* part_o;
  float* part_lse;
  int32_t splits;
};
static_assert(sizeof(ScoreFwdParams) <= 4096, "kernel arguments");

// What the queries of a stage of 64 rows see, made by the first launch of the
// backward: least begin and largest end of rows that see something (begin = end
// = 0: there is none), and what all of them see.
struct ScoreStage {
  int32_t lo_min, hi_max, lo_max, hi_min;
  int32_t pos;   // its first row's position
  int32_t wide;  // rows of far partitions: pos_rel are integers
  int32_t pad[2];
};

struct ScoreBwdParams {
  ScoreTile t;
  const uint16_t* o;
  const uint16_t* d_o;
  const float* lse;
  void* dq;
  void* dk;
  void* dv;
  float* delta;   // [hq][rows_pad]: -<dO, O>
  float* lse2;    // [hq][rows_pad]: (LSE - cap) log2(e); +inf: sees no key
  int32_t* lo;    // [rows_pad]: a row's begin, end and position
  int32_t* hi;
  int32_t* pos;
  // Position less that of the stage's first row, as an integer's bits where one of
  // them is 2^23 or more.
  float* pos_rel;
  ScoreStage* stages;  // [rows_pad / 64]
  // Partial dK, dV of 128 keys whose stages are cut into parts of about
  // part_stages, at most kv_splits of them: [part][rows_kv][hkv][d]; how many there
  // are: [rows_kv][hkv].
  int32_t* kv_parts;
  float* part_dk;
  float* part_dv;
  // Partial dQ of keys cut into q_splits parts: [split][rows_q][hq][d].
  float* part_dq;
  int32_t rows_pad, kv_splits, q_splits;
  int32_t part_stages;
  int32_t kv_items;  // workgroups of dK/dV, those of dQ come behind
};
static_assert(sizeof(ScoreBwdParams) <= 4096, "kernel arguments");

// How many parts the keys of every Q block are cut into, from the sizes.
int score_fwd_splits(const ScoreTile& t);
hipError_t launch_score_fwd(const ScoreFwdParams& p, bool out_f32,
                            hipStream_t stream);
void score_bwd_splits(const ScoreTile& t, int* kv_splits, int* q_splits);
hipError_t launch_score_bwd(const ScoreBwdParams& p, bool out_f32,
                            hipStream_t stream);

// Rotation of Q and K and storage of K, V (rope_append.hip).
struct RopeAppendParams {
  RopeTable t;
  CacheDims c;
  const int32_t* positions;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const int64_t* slots;
  uint8_t* data;
  int64_t rows;
  int32_t hq, rot, interleaved;
  int32_t group_rows;  // rows of a workgroup
};
static_assert(sizeof(RopeAppendParams) <= 4096, "kernel arguments");
hipError_t launch_rope_append(const RopeAppendParams& p, hipStream_t stream);

}  // namespace mesh_attn
