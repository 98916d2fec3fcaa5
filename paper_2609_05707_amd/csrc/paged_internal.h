// The paged cache: sizes and parameter blocks shared by its host code and kernels.
//
// A decode step's attention is cut into pieces on the device.  Its work, per
// kv head, is two lines of 32-token tiles: the block line (contexts with more
// than 16 query rows, the rows in groups of whole questions) and the wave line
// (contexts with fewer rows, and segments).  Each line is cut into equal runs
// of tiles, whatever sequence they belong to: one workgroup takes a piece of
// the block line, one wave a piece of the wave line.  A task is a sequence (and
// row group) on a line; every (piece, task) pair leaves one partial softmax
// state per row.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ippd_internal.h"

namespace ippd {

constexpr int kPlanMagic = 0x49504450;    // first word of a plan
constexpr int kPlanHeader = 64;           // words of its header
constexpr int kPieceWords = 12;           // first task, first tile within it, tiles (block line: of that task; wave line: in all), 0;
                                          // that task's record
constexpr int kTaskWords = 8;             // sequence, tokens, rows, first active question; first state row, first piece, tiles,
                                          // tiles in the first piece (block line)
constexpr int kQuestionWords = 8;         // served, context state row, states, rows a state; segment state row, states; 0, 0
constexpr int kPromptWords = 4;           // kind (0 none, 1 block line, 2 wave line); first task and questions a
                                          // group, or first state row and states; rank of its first question

// Sizes of a batch's plan and of its partial states: functions of the batch's
// host fields only.
struct PagedShape {
  int G, page_shift;
  int W;                                  // workgroups per kv head
  int waves;                              // waves of a workgroup: 4, two workgroups on a compute unit, or 8
  int rb;                                 // 16-row blocks per wave of a block-line piece (0: no block line)
  int group_q;                            // questions of a block-line row group (0: no block line)
  int64_t rows;                           // partial states per kv head
  // word offsets of the plan's arrays
  int64_t piece1, piece2, task1, task2, quest, prompt, qlist, rank, where, words;
  int by_rows;                            // a block-line tile costs by its row blocks (fp32)
  int wave_shortest;                      // the shortest pieces of the wave line, in tiles
  size_t off_ml, workspace_bytes;
};

struct ReserveParams {
  const int32_t* new_tokens; const int32_t* token_start; const int32_t* q_start;
  int32_t* seq_len; int32_t* block_table; int32_t* free_pages; int32_t* free_count;
  int32_t* slot_map; int32_t* positions; int32_t* served; int32_t* err_flag;
  int B, Nt, page_shift, num_pages, table_pages, num_rows;
};

struct PagedAppendParams {
  const void* q; const void* k; const void* v; void* q_rot; void* k_pages; void* v_pages;
  const int32_t* slot_map; const int32_t* positions; int32_t* err_flag;
  int64_t q_stride, k_stride, v_stride;   // elements between rows
  int64_t slots;                          // num_pages * page_tokens
  int num_rows, Hq, Hkv, D, page_shift;
  alignas(16) double inv_freq[kMaxHalfDim];
};

struct PagedPlanParams {
  int32_t* plan;
  const int32_t* q_start; const int32_t* seq_len; const uint8_t* active; int32_t* err_flag;
  int B, Nt, G, W, waves, group_q, max_questions;
  int max_len;                            // table_pages * page_tokens
  int64_t piece1, piece2, task1, task2, quest, prompt, qlist, rank, where;
  int by_rows, wave_shortest;
};

struct PagedAttendParams {
  const int32_t* plan; const int32_t* block_table;
  const void* q_rot; const void* k_pages; const void* v_pages;
  void* out; float* lse; float* part_o; float* part_ml; int32_t* err_flag;
  int64_t rows;                           // partial states per kv head
  int64_t piece1, piece2, task1, task2, quest, qlist;
  int B, Nt, Hq, Hkv, G, W, waves, group_q, page_shift, num_pages, table_pages;
  float c;                                // scale * log2(e)
  float scale;
};

hipError_t launch_paged_reserve(const ReserveParams& p, hipStream_t s);
hipError_t launch_paged_append(int dtype, const PagedAppendParams& p, hipStream_t s);
hipError_t launch_paged_plan(const PagedPlanParams& p, hipStream_t s);
hipError_t launch_paged_attend(int dtype, int D, int waves, int rb, const PagedAttendParams& p, hipStream_t s);

}  // namespace ippd
