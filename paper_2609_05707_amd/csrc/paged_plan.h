// Argument checks and sizes of the paged cache's calls: host code only, a
// function of the batch fields, so that a size query and a launch agree.
#pragma once

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "ippd.h"
#include "paged_internal.h"

namespace ippd {

inline ippd_status_t check_paged(const ippd_paged_batch_t* bt) {
  if (bt == nullptr) return IPPD_ERR_NULL;
  if (bt->dtype != IPPD_DTYPE_F32 && bt->dtype != IPPD_DTYPE_BF16) return IPPD_ERR_DTYPE;
  if (bt->num_prompts < 1 || bt->num_questions < 0 || bt->num_q_heads < 1 || bt->num_kv_heads < 1)
    return IPPD_ERR_SHAPE;
  if (bt->num_prompts > IPPD_PAGED_MAX_SEQUENCES || bt->num_questions > IPPD_PAGED_MAX_SEQUENCES - bt->num_prompts)
    return IPPD_ERR_SHAPE;
  if (bt->num_q_heads % bt->num_kv_heads != 0) return IPPD_ERR_SHAPE;
  if (bt->num_q_heads / bt->num_kv_heads > kMaxGroup || bt->num_q_heads > 1024) return IPPD_ERR_SHAPE;
  // partial states of 2 x G rows a question and kv head: at 2^23, D = 128, over 8 GB for each query head of a kv head
  if (static_cast<int64_t>(bt->num_questions) * bt->num_kv_heads > (1 << 23)) return IPPD_ERR_SHAPE;
  if (bt->head_dim != 64 && bt->head_dim != 128) return IPPD_ERR_SHAPE;
  const int p = bt->page_tokens;
  if (p != 16 && p != 32 && p != 64 && p != 128 && p != 256) return IPPD_ERR_SHAPE;
  if (bt->num_pages < 1 || bt->table_pages < 1) return IPPD_ERR_SHAPE;
  if (static_cast<int64_t>(bt->num_pages) * p > INT32_MAX || static_cast<int64_t>(bt->table_pages) * p > INT32_MAX)
    return IPPD_ERR_SHAPE;
  if (bt->max_questions < 1 || bt->max_questions > kMaxQuestionsPerPrompt) return IPPD_ERR_SHAPE;
  if (!(bt->rope_base > 0.0) || !isfinite(bt->rope_base)) return IPPD_ERR_SHAPE;
  if (!isfinite(bt->scale)) return IPPD_ERR_SHAPE;
  if (!bt->q_start || !bt->seq_len || !bt->block_table || !bt->free_pages || !bt->free_count || !bt->active ||
      !bt->err_flag)
    return IPPD_ERR_NULL;
  return IPPD_OK;
}

inline int page_shift_of(int page_tokens) {
  int s = 0;
  while ((1 << s) < page_tokens) ++s;
  return s;
}

// (A constant of MI355X, not a device query: sizes then depend on the batch
// fields only.)
constexpr int kPagedComputeUnits = 256;

inline PagedShape paged_shape(const ippd_paged_batch_t* bt) {
  PagedShape s;
  s.G = bt->num_q_heads / bt->num_kv_heads;
  s.page_shift = page_shift_of(bt->page_tokens);
  const bool bf16 = bt->dtype == IPPD_DTYPE_BF16;
  const int most = bt->max_questions * s.G;
  // Eight waves, one workgroup on a compute unit, where a context has more rows than
  // four waves hold (a second row group would stream it again), and for fp32 at
  // head_dim 128, whose ring leaves no room for a second workgroup.  (bf16 at head_dim
  // 64: the nine stages are 72 of a unit's 160 KB.)
  s.waves = (bf16 ? most > 128 : bt->head_dim == 128) ? 8 : 4;
  s.rb = most <= 16 ? 0 : bf16 && most > 64 ? 2 : 1;
  s.by_rows = bf16 ? 0 : 1;
  // A piece's start against its states in the join: bf16, one request of 8192
  // tokens 150 us at 2, 131 at 4, 139 at 8 (eight layers), 4096 x 16 136, 133, 133;
  // an fp32 tile takes a wave longer than a piece's start (256 tokens, 4 questions
  // 16.0 us at 1, 17.0 at 2).
  s.wave_shortest = bf16 ? 4 : 1;
  s.W = std::max(2, kPagedComputeUnits * (s.waves == 8 ? 1 : 2) / bt->num_kv_heads);
  s.group_q = most > 16 ? 16 * s.waves * s.rb / s.G : 0;
  const int64_t nt = bt->num_questions, b = bt->num_prompts, w1 = s.W, w2 = w1 * s.waves;
  // every row of a task once, and again for each cut of a line that falls inside the task
  s.rows = 2 * nt * s.G + (s.group_q ? w1 * s.group_q * s.G : 0) + w2 * 16;
  int64_t at = kPlanHeader;
  s.piece1 = at; at += w1 * kPieceWords;
  s.piece2 = at; at += w2 * kPieceWords;
  s.task1 = at; at += nt * kTaskWords;                 // a row group holds a question at least
  s.task2 = at; at += 2 * nt * kTaskWords;             // contexts with questions, segments
  s.quest = at; at += nt * kQuestionWords;
  s.prompt = at; at += b * kPromptWords;
  s.qlist = at; at += nt;
  s.rank = at; at += nt + 1;
  at += at & 1;
  s.where = at; at += 2 * nt;
  s.words = at;
  const size_t states = static_cast<size_t>(s.rows) * bt->num_kv_heads;
  s.off_ml = (states * bt->head_dim * 4 + 255) & ~static_cast<size_t>(255);
  s.workspace_bytes = (s.off_ml + states * 8 + 255) & ~static_cast<size_t>(255);
  return s;
}

}  // namespace ippd
