// C ABI of the paged cache: argument validation and kernel launches.  As in
// ippd_api.hip, nothing here allocates, frees or synchronises; all work is
// enqueued on the caller's stream.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "ippd.h"
#include "paged_internal.h"
#include "paged_plan.h"

namespace {

using ippd::check_paged;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

float softmax_scale(const ippd_paged_batch_t* bt) {
  return bt->scale > 0.f ? bt->scale : 1.0f / sqrtf(static_cast<float>(bt->head_dim));
}

// theta_j = base^(-2j/D) in fp64, the rotation frequencies of pair j.  A thread
// keeps its last table with the base and size it is of: 64 powers cost 1 us.
void fill_inv_freq(const ippd_paged_batch_t* bt, double* out) {
  thread_local double base = 0.0, table[ippd::kMaxHalfDim];
  thread_local int dim = 0;
  if (base != bt->rope_base || dim != bt->head_dim) {
    const int half = bt->head_dim / 2;
    for (int j = 0; j < ippd::kMaxHalfDim; ++j)
      table[j] = j < half ? pow(bt->rope_base, -2.0 * j / bt->head_dim) : 0.0;
    base = bt->rope_base;
    dim = bt->head_dim;
  }
  memcpy(out, table, sizeof table);
}

ippd_status_t hip_status(hipError_t e) {
  if (e == hipSuccess) return IPPD_OK;
  ippd::keep_hip_error(e);
  return IPPD_ERR_HIP;
}

}  // namespace

extern "C" {

ippd_status_t ippd_paged_reserve(const ippd_paged_batch_t* bt, const int32_t* new_tokens, const int32_t* token_start,
                                 int32_t num_rows, int32_t* slot_map, int32_t* positions, int32_t* served,
                                 hipStream_t stream) {
  ippd_status_t st = check_paged(bt);
  if (st != IPPD_OK) return st;
  if (num_rows < 0 || num_rows > IPPD_PAGED_MAX_ROWS) return IPPD_ERR_SHAPE;
  if (!new_tokens || !token_start || !served || (num_rows > 0 && (!slot_map || !positions))) return IPPD_ERR_NULL;
  ippd::ReserveParams p;
  p.new_tokens = new_tokens; p.token_start = token_start; p.q_start = bt->q_start;
  p.seq_len = bt->seq_len; p.block_table = bt->block_table;
  p.free_pages = bt->free_pages; p.free_count = bt->free_count;
  p.slot_map = slot_map; p.positions = positions; p.served = served; p.err_flag = bt->err_flag;
  p.B = bt->num_prompts; p.Nt = bt->num_questions; p.page_shift = ippd::page_shift_of(bt->page_tokens);
  p.num_pages = bt->num_pages; p.table_pages = bt->table_pages; p.num_rows = num_rows;
  return hip_status(ippd::launch_paged_reserve(p, stream));
}

ippd_status_t ippd_paged_append(const ippd_paged_batch_t* bt, const ippd_pages_t* pages, int32_t num_rows,
                                const int32_t* slot_map, const int32_t* positions, const void* q, int64_t q_stride,
                                const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_rot,
                                hipStream_t stream) {
  ippd_status_t st = check_paged(bt);
  if (st != IPPD_OK) return st;
  if (num_rows < 0 || num_rows > IPPD_PAGED_MAX_ROWS) return IPPD_ERR_SHAPE;
  if (!pages || !pages->k || !pages->v || !slot_map || !positions || !k || !v || (q && !q_rot)) return IPPD_ERR_NULL;
  if (!aligned16(pages->k) || !aligned16(pages->v) || !aligned16(k) || !aligned16(v) ||
      (q && (!aligned16(q) || !aligned16(q_rot))))
    return IPPD_ERR_ALIGN;
  const int64_t ve = bt->dtype == IPPD_DTYPE_F32 ? 4 : 8, kv = static_cast<int64_t>(bt->num_kv_heads) * bt->head_dim;
  if (k_stride < kv || v_stride < kv || (q && q_stride < static_cast<int64_t>(bt->num_q_heads) * bt->head_dim) ||
      k_stride % ve || v_stride % ve || (q && q_stride % ve))
    return IPPD_ERR_SHAPE;
  if (num_rows == 0) return IPPD_OK;
  ippd::PagedAppendParams p;
  p.q = q; p.k = k; p.v = v; p.q_rot = q_rot; p.k_pages = pages->k; p.v_pages = pages->v;
  p.slot_map = slot_map; p.positions = positions; p.err_flag = bt->err_flag;
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.slots = static_cast<int64_t>(bt->num_pages) * bt->page_tokens;
  p.num_rows = num_rows; p.Hq = bt->num_q_heads; p.Hkv = bt->num_kv_heads; p.D = bt->head_dim;
  p.page_shift = ippd::page_shift_of(bt->page_tokens);
  fill_inv_freq(bt, p.inv_freq);
  return hip_status(ippd::launch_paged_append(bt->dtype, p, stream));
}

size_t ippd_paged_plan_bytes(const ippd_paged_batch_t* bt) {
  return check_paged(bt) == IPPD_OK ? static_cast<size_t>(ippd::paged_shape(bt).words) * 4 : 0;
}

ippd_status_t ippd_paged_plan(const ippd_paged_batch_t* bt, void* plan, size_t plan_bytes, hipStream_t stream) {
  ippd_status_t st = check_paged(bt);
  if (st != IPPD_OK) return st;
  const ippd::PagedShape s = ippd::paged_shape(bt);
  if (!plan || plan_bytes < static_cast<size_t>(s.words) * 4) return IPPD_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(plan) & 255u) return IPPD_ERR_ALIGN;
  ippd::PagedPlanParams p;
  p.plan = static_cast<int32_t*>(plan);
  p.q_start = bt->q_start; p.seq_len = bt->seq_len; p.active = bt->active; p.err_flag = bt->err_flag;
  p.B = bt->num_prompts; p.Nt = bt->num_questions; p.G = s.G; p.W = s.W; p.waves = s.waves; p.group_q = s.group_q;
  p.max_questions = bt->max_questions;
  p.max_len = bt->table_pages * bt->page_tokens;
  p.piece1 = s.piece1; p.piece2 = s.piece2; p.task1 = s.task1; p.task2 = s.task2; p.quest = s.quest;
  p.prompt = s.prompt; p.qlist = s.qlist; p.rank = s.rank; p.where = s.where;
  p.by_rows = s.by_rows; p.wave_shortest = s.wave_shortest;
  return hip_status(ippd::launch_paged_plan(p, stream));
}

size_t ippd_paged_workspace_bytes(const ippd_paged_batch_t* bt) {
  return check_paged(bt) == IPPD_OK ? ippd::paged_shape(bt).workspace_bytes : 0;
}

ippd_status_t ippd_paged_decode_attention(const ippd_paged_batch_t* bt, const ippd_pages_t* pages, const void* plan,
                                          size_t plan_bytes, const void* q_rot, void* out, float* lse,
                                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ippd_status_t st = check_paged(bt);
  if (st != IPPD_OK) return st;
  if (!pages || !pages->k || !pages->v || !q_rot || !out) return IPPD_ERR_NULL;
  if (!aligned16(pages->k) || !aligned16(pages->v) || !aligned16(q_rot) || !aligned16(out) ||
      (lse && (reinterpret_cast<uintptr_t>(lse) & 3)))
    return IPPD_ERR_ALIGN;
  if (bt->num_questions == 0) return IPPD_OK;
  const ippd::PagedShape s = ippd::paged_shape(bt);
  if (!plan || plan_bytes < static_cast<size_t>(s.words) * 4 || !workspace || workspace_bytes < s.workspace_bytes)
    return IPPD_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(plan) | reinterpret_cast<uintptr_t>(workspace)) & 255u) return IPPD_ERR_ALIGN;
  ippd::PagedAttendParams p;
  p.plan = static_cast<const int32_t*>(plan);
  p.block_table = bt->block_table; p.q_rot = q_rot; p.k_pages = pages->k; p.v_pages = pages->v;
  p.out = out; p.lse = lse; p.err_flag = bt->err_flag;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + s.off_ml);
  p.rows = s.rows;
  p.piece1 = s.piece1; p.piece2 = s.piece2; p.task1 = s.task1; p.task2 = s.task2; p.quest = s.quest; p.qlist = s.qlist;
  p.B = bt->num_prompts; p.Nt = bt->num_questions; p.Hq = bt->num_q_heads; p.Hkv = bt->num_kv_heads; p.G = s.G;
  p.W = s.W; p.waves = s.waves; p.group_q = s.group_q; p.page_shift = s.page_shift; p.num_pages = bt->num_pages;
  p.table_pages = bt->table_pages;
  p.scale = softmax_scale(bt);
  p.c = p.scale * 1.4426950408889634f;
  return hip_status(ippd::launch_paged_attend(bt->dtype, bt->head_dim, s.waves, s.rb, p, stream));
}

}  // extern "C"
