// Bookkeeping of the paged cache: block tables and slot maps from request
// lengths, and the attention's plan of a decode step.
//
// Both are a few thousand integers, so what bounds them is latency: the
// dependent round trips to memory and the barriers of a scan.  One workgroup
// of 1024 threads does a call; only a slot map of many rows gets a launch of
// its own.
#include "ippd_device.h"
#include "paged_internal.h"

namespace ippd {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
// reserve_kernel fills the slot map itself up to these sizes (one launch); its
// copies of the sequences' rows and lengths then fit the LDS
constexpr int kFusedSequences = 2048;
constexpr int kFusedRows = 8192;

constexpr int kFlagPagesExhausted = 4;

// Sum of v over the lanes below this one's and, in the last lane, over all.
template <typename V>
__device__ __forceinline__ V wave_inclusive(V v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V u = __shfl_up(v, d, 64);
    if (lane >= d) v += u;
  }
  return v;
}

// Exclusive prefix sum over the workgroup; total: the sum over all threads.
template <typename V>
__device__ __forceinline__ V block_exclusive(V v, V* lds, V& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const V inc = wave_inclusive(v);
  __syncthreads();                                   // the previous use of lds is over
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const V x = lds[w];
    before += w < wave ? x : 0;
    all += x;
  }
  total = all;
  return before + inc - v;
}

// The last index of a non-decreasing array of n entries that is <= x (0 if none).
template <typename A>
__device__ __forceinline__ int last_at_most(const A& a, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int pages_of(int tokens, int shift) { return static_cast<int>((static_cast<uint32_t>(tokens) + (1u << shift) - 1u) >> shift); }

// ---------------------------------------------------------------------------
// Reservation.  With len_s the tokens that sequence s holds and c_s the change
// asked for:
//   shrink (c_s < 0)  the sequence keeps max(0, len_s + c_s) tokens; of the R
//                     pages given back by all, in order of sequence and page,
//                     the k-th goes to free_pages[f + R - 1 - k];
//   grow (c_s > 0)    with f' = f + R pages free, the k-th page needed, in the
//                     same order, is free_pages[f' - 1 - k]; a sequence is
//                     served if the pages needed up to and including its own
//                     number f' at most (or it needs none).
// The orders make a shrink the inverse of the growth before it.  Each is a
// prefix sum over the sequences and then a flat loop over the pages, a thread
// per page, which finds its sequence by a search of the sums: 32 contexts of
// 256 pages cost as many rounds as 8192 sequences of one.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void write_row(const ReserveParams& p, int row, int s, int j, int got, int after, int base) {
  int slot = -1, pos = -1;
  if (j >= 0 && j < got) {
    const int tok = after - got + j;
    const int page = p.block_table[static_cast<int64_t>(s) * p.table_pages + (tok >> p.page_shift)];
    if (static_cast<uint32_t>(page) < static_cast<uint32_t>(p.num_pages)) {
      slot = (page << p.page_shift) + (tok & ((1 << p.page_shift) - 1));
      pos = base + tok;
    } else {
      raise_flag(p.err_flag, kFlagBadLayout);
    }
  }
  p.slot_map[row] = slot;
  p.positions[row] = pos;
}

template <bool ROWS>
__global__ __launch_bounds__(kThreads) void reserve_kernel(ReserveParams p) {
  __shared__ int64_t sums64[kWaves];
  __shared__ int sums[kWaves];
  __shared__ int first[kThreads];                    // pages before the sequence, in this window
  __shared__ int from[kThreads];                     // its first page moved
  __shared__ int taken;
  __shared__ int row0[ROWS ? kFusedSequences : 1], after[ROWS ? kFusedSequences : 1], got[ROWS ? kFusedSequences : 1];
  __shared__ int q0[ROWS ? kFusedSequences : 1];
  const int tid = threadIdx.x, S = p.B + p.Nt, sh = p.page_shift;
  const int64_t cap = static_cast<int64_t>(p.table_pages) << sh;
  const int f = *p.free_count;
  if (tid == 0) taken = 0;

  // checks, and the pages given back
  bool bad = f < 0 || f > p.num_pages;
  int64_t back = 0;
  for (int s = tid; s < S; s += kThreads) {
    const int len = p.seq_len[s], c = p.new_tokens[s], a = p.token_start[s], e = p.token_start[s + 1];
    bad = bad || len < 0 || len > cap || a < 0 || e < a || e > p.num_rows || c > e - a;
    if (c < 0 && len > 0) back += pages_of(len, sh) - pages_of(c < -len ? 0 : len + c, sh);
    if constexpr (ROWS) row0[s] = a;
  }
  for (int b = tid; b < p.B; b += kThreads) {
    const int qa = p.q_start[b], qb = p.q_start[b + 1];
    bad = bad || qb < qa || (b == 0 && qa != 0) || (b == p.B - 1 && qb != p.Nt);
    if constexpr (ROWS) q0[b] = qa;
  }
  int64_t total_back;
  block_exclusive<int64_t>(back, sums64, total_back);
  bad = __syncthreads_or(bad || total_back > p.num_pages - f);
  if (bad) {                                         // nothing is moved: no row of the call is served
    if (tid == 0) raise_flag(p.err_flag, kFlagBadLayout);
    for (int s = tid; s < S; s += kThreads) p.served[s] = 0;
    if constexpr (ROWS) {
      for (int r = tid; r < p.num_rows; r += kThreads) {
        p.slot_map[r] = -1;
        p.positions[r] = -1;
      }
    }
    return;
  }
  const int R = static_cast<int>(total_back), f1 = f + R;

  // shrink
  if (R > 0) {
    int carry = 0;
    for (int s0 = 0; s0 < S; s0 += kThreads) {
      const int s = s0 + tid;
      int n = 0, keep = 0;
      if (s < S) {
        const int len = p.seq_len[s], c = p.new_tokens[s];
        if (c < 0 && len > 0) {
          keep = pages_of(c < -len ? 0 : len + c, sh);
          n = pages_of(len, sh) - keep;
        }
      }
      int total;
      const int ex = block_exclusive<int>(n, sums, total);
      first[tid] = ex;
      from[tid] = keep;
      __syncthreads();
      for (int k = tid; k < total; k += kThreads) {
        const int w = last_at_most(first, min(kThreads, S - s0), k);
        const int64_t row = static_cast<int64_t>(s0 + w) * p.table_pages;
        p.free_pages[f1 - 1 - (carry + k)] = p.block_table[row + from[w] + (k - first[w])];
      }
      carry += total;
    }
  }
  __syncthreads();                                   // the pages given back are on the stack

  // grow
  int carry = 0;
  for (int s0 = 0; s0 < S; s0 += kThreads) {
    const int s = s0 + tid;
    int need = 0, len = 0, c = 0, have = 0;
    bool fits = false;
    if (s < S) {
      len = p.seq_len[s];
      c = p.new_tokens[s];
      if (c > 0) {
        fits = c <= cap - len;
        if (fits) {
          have = pages_of(len, sh);
          need = pages_of(len + c, sh) - have;
        } else {
          raise_flag(p.err_flag, kFlagSegmentFull);
        }
      }
    }
    int total;
    const int ex = block_exclusive<int>(need, sums, total);
    // (the sums need no 64 bits: the rows, and with them the new tokens, number
    // fewer than 2^31)
    const int upto = carry + ex + need;
    const bool ok = fits && (need == 0 || upto <= f1);
    first[tid] = ex;
    from[tid] = have;
    if (s < S) {
      int now = len, moved = 0;
      if (ok) {
        now = len + c;
        moved = c;
        if (need > 0) atomicMax(&taken, upto);
      } else if (c > 0 && fits) {
        raise_flag(p.err_flag, kFlagPagesExhausted);
      } else if (c < 0) {
        now = c < -len ? 0 : len + c;
        moved = now - len;
      }
      if (now != len) p.seq_len[s] = now;
      p.served[s] = moved;
      if constexpr (ROWS) {
        after[s] = now;
        got[s] = ok ? c : 0;
      }
    }
    __syncthreads();
    // the served sequences are those of a leading run of the pages needed
    const int run = min(total, taken - carry);
    for (int k = tid; k < run; k += kThreads) {
      const int w = last_at_most(first, min(kThreads, S - s0), k);
      const int64_t row = static_cast<int64_t>(s0 + w) * p.table_pages;
      p.block_table[row + from[w] + (k - first[w])] = p.free_pages[f1 - 1 - (carry + k)];
    }
    carry += total;
  }
  __syncthreads();                                   // tables, and the page count
  if (tid == 0) *p.free_count = f1 - taken;
  if constexpr (ROWS) {
    for (int r = tid; r < p.num_rows; r += kThreads) {
      const int s = last_at_most(row0, S, r);
      int base = 0;
      if (s >= p.B) base = after[last_at_most(q0, p.B, s - p.B)];
      write_row(p, r, s, r - row0[s], got[s], after[s], base);
    }
  }
}

// The slot map of many rows, a thread per row; the reservation's kernel has
// left the lengths after it and what each sequence was served.
__global__ __launch_bounds__(256) void rows_kernel(ReserveParams p) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= p.num_rows) return;
  const int s = last_at_most(p.token_start, p.B + p.Nt, r);
  const int got = max(p.served[s], 0);
  int base = 0;
  if (s >= p.B) base = p.seq_len[last_at_most(p.q_start, p.B, s - p.B)];
  write_row(p, r, s, r - p.token_start[s], got, p.seq_len[s], base);
}

// ---------------------------------------------------------------------------
// Plan of a decode step's attention: see paged_internal.h for the lines.
// ---------------------------------------------------------------------------
// A line of T tiles cut into n <= T pieces, the first T % n of them one tile longer.
struct Line {
  int64_t T, size, longer;                           // tiles; of a short piece; pieces that are longer
  int n;
  __device__ __forceinline__ Line(int64_t tiles, int pieces) : T(tiles), size(pieces ? tiles / pieces : 0), longer(pieces ? tiles % pieces : 0), n(pieces) {}
  __device__ __forceinline__ int64_t start(int p) const { return p * size + (p < longer ? p : longer); }
  __device__ __forceinline__ int piece_of(int64_t x) const {
    const int64_t edge = longer * (size + 1);
    return static_cast<int>(x < edge ? x / (size + 1) : longer + (x - edge) / size);
  }
};

// A task of `tiles` > 0 tiles from `at` on the line: its record, and the
// records of the pieces that begin inside it.
__device__ __forceinline__ void write_task(int32_t* plan, int64_t tasks, int64_t pieces, const Line& line, int index,
                                           int64_t at, int tiles, int seq, int len, int rows, int q, int row, int states) {
  const int first = line.piece_of(at);
  int4* t = reinterpret_cast<int4*>(plan + tasks + static_cast<int64_t>(index) * kTaskWords);
  t[0] = make_int4(seq, len, rows, q);
  t[1] = make_int4(row, first, tiles, states);
  for (int p = line.start(first) == at ? first : first + 1; p < line.n && line.start(p) < at + tiles; ++p)
    *reinterpret_cast<int4*>(plan + pieces + static_cast<int64_t>(p) * kPieceWords) =
        make_int4(index, static_cast<int>(line.start(p) - at), static_cast<int>(line.start(p + 1) - line.start(p)), 0);
}

__device__ __forceinline__ int tiles_of(int len) { return static_cast<int>((static_cast<uint32_t>(len) + 31u) >> 5); }

__global__ __launch_bounds__(kThreads) void plan_kernel(PagedPlanParams p) {
  __shared__ int64_t sums64[kWaves];
  __shared__ int sums[kWaves];
  const int tid = threadIdx.x, B = p.B, Nt = p.Nt, G = p.G;
  int32_t* plan = p.plan;
  int32_t* qlist = plan + p.qlist;
  int32_t* rank = plan + p.rank;
  int4* prompts = reinterpret_cast<int4*>(plan + p.prompt);

  // checks; the active questions in order
  bool bad = false;
  for (int b = tid; b < B; b += kThreads) {
    const int qa = p.q_start[b], qb = p.q_start[b + 1];
    bad = bad || qb < qa || qb - qa > p.max_questions || (b == 0 && qa != 0) || (b == B - 1 && qb != Nt);
  }
  for (int s = tid; s < B + Nt; s += kThreads) {
    const int len = p.seq_len[s];
    bad = bad || len < 0 || len > p.max_len;
  }
  bad = __syncthreads_or(bad);
  int nact = 0;
  for (int i0 = 0; i0 < Nt; i0 += kThreads) {
    const int i = i0 + tid;
    const int on = i < Nt && !bad && p.active[i] != 0;
    int total;
    const int ex = nact + block_exclusive<int>(on, sums, total);
    if (i < Nt) rank[i] = ex;
    if (on) qlist[ex] = i;
    nact += total;
  }
  if (tid == 0) rank[Nt] = nact;
  __syncthreads();

  // tiles of the two lines
  int64_t t1 = 0, t2 = 0, w1 = 0;
  if (!bad) {
    for (int b = tid; b < B; b += kThreads) {
      const int n = rank[p.q_start[b + 1]] - rank[p.q_start[b]], tiles = tiles_of(p.seq_len[b]);
      if (n == 0) continue;
      if (p.group_q > 0 && n * G > 16) {
        const int groups = (n + p.group_q - 1) / p.group_q;
        t1 += static_cast<int64_t>(groups) * tiles;
        w1 += static_cast<int64_t>(groups) * tiles;
      } else {
        t2 += tiles;
      }
    }
    for (int k = tid; k < nact; k += kThreads) t2 += tiles_of(p.seq_len[B + qlist[k]]);
  }
  int64_t T1, T2, W1;
  block_exclusive<int64_t>(t1, sums64, T1);
  block_exclusive<int64_t>(t2, sums64, T2);
  block_exclusive<int64_t>(w1, sums64, W1);
  // workgroups to the lines by their shares of the work, runs of four tiles
  // at least on the block line and of two on the wave line
  int n1 = 0, n2 = 0;
  if (T1 > 0) {
    const int64_t most = p.W - (T2 > 0 ? 1 : 0);
    const int64_t share = (W1 * p.W + (W1 + T2) / 2) / (W1 + T2);
    n1 = static_cast<int>(min(max(min(share, (T1 + 3) / 4), static_cast<int64_t>(1)), most));
  }
  if (T2 > 0) n2 = static_cast<int>(min(static_cast<int64_t>(p.waves) * (p.W - n1), (T2 + 1) / 2));
  const Line line1(T1, n1), line2(T2, n2);

  // block line: contexts, their active questions in even groups
  int tasks = 0, rows = 0;
  int64_t at = 0;
  for (int b0 = 0; b0 < B; b0 += kThreads) {
    const int b = b0 + tid;
    int groups = 0, per = 0, n = 0, r0 = 0, len = 0, kind = 0;
    if (b < B && !bad) {
      r0 = rank[p.q_start[b]];
      n = rank[p.q_start[b + 1]] - r0;
      len = p.seq_len[b];
      if (n > 0 && len > 0) {
        kind = p.group_q > 0 && n * G > 16 ? 1 : 2;
        if (kind == 1) {
          groups = (n + p.group_q - 1) / p.group_q;
          per = (n + groups - 1) / groups;           // (and ceil(n / per) is groups again)
        }
      }
    }
    const int tiles = tiles_of(len);
    int ntask;
    const int task0 = tasks + block_exclusive<int>(groups, sums, ntask);
    int64_t ntile;
    const int64_t at0 = at + block_exclusive<int64_t>(static_cast<int64_t>(groups) * tiles, sums64, ntile);
    int need = 0;
    for (int j = 0; j < groups; ++j) {
      const int64_t x = at0 + static_cast<int64_t>(j) * tiles;
      need += (line1.piece_of(x + tiles - 1) - line1.piece_of(x) + 1) * (min(per, n - j * per) * G);
    }
    int nrow;
    int row = rows + block_exclusive<int>(need, sums, nrow);
    for (int j = 0; j < groups; ++j) {
      const int64_t x = at0 + static_cast<int64_t>(j) * tiles;
      const int gr = min(per, n - j * per) * G, states = line1.piece_of(x + tiles - 1) - line1.piece_of(x) + 1;
      write_task(plan, p.task1, p.piece1, line1, task0 + j, x, tiles, b, len, gr, r0 + j * per, row, states);
      row += states * gr;
    }
    if (b < B) prompts[b] = make_int4(kind, task0, per, r0);
    tasks += ntask;
    rows += nrow;
    at += ntile;
  }
  __syncthreads();                                   // prompts

  // wave line: the other contexts, then the segments of the active questions
  tasks = 0;
  at = 0;
  for (int x0 = 0; x0 < B + nact; x0 += kThreads) {
    const int x = x0 + tid;
    int seq = -1, len = 0, q = 0, n = 0;
    if (x < B) {
      const int4 pr = prompts[x];
      if (pr.x == 2) {
        seq = x;
        q = pr.w;
        n = (rank[p.q_start[x + 1]] - q) * G;
        len = p.seq_len[x];
      }
    } else if (x < B + nact) {
      q = x - B;
      seq = B + qlist[q];
      n = G;
      len = p.seq_len[seq];
    }
    const int tiles = seq < 0 ? 0 : tiles_of(len);
    int ntask;
    const int task = tasks + block_exclusive<int>(tiles > 0, sums, ntask);
    int64_t ntile;
    const int64_t at0 = at + block_exclusive<int64_t>(tiles, sums64, ntile);
    const int np = tiles > 0 ? line2.piece_of(at0 + tiles - 1) - line2.piece_of(at0) + 1 : 0;
    int nrow;
    const int row = rows + block_exclusive<int>(np * n, sums, nrow);
    if (tiles > 0) write_task(plan, p.task2, p.piece2, line2, task, at0, tiles, seq, len, n, q, row, np);
    if (x < B) {
      if (seq >= 0) prompts[x].y = task;
    } else if (x < B + nact) {
      *reinterpret_cast<int4*>(plan + p.quest + static_cast<int64_t>(seq - B) * kQuestionWords + 4) = make_int4(row, np, 0, 0);
    }
    tasks += ntask;
    rows += nrow;
    at += ntile;
  }
  __syncthreads();                                   // tasks of contexts

  // where the states of each question's context are
  for (int i = tid; i < Nt; i += kThreads) {
    const int k = rank[i];
    int4 rec = make_int4(0, 0, 0, 0);
    if (rank[i + 1] > k) {
      const int b = last_at_most(p.q_start, B, i);
      const int4 pr = prompts[b];
      rec.x = 1;
      if (pr.x != 0) {
        const int local = k - pr.w, j = pr.x == 1 ? local / pr.z : 0;
        const int64_t rec0 = (pr.x == 1 ? p.task1 : p.task2) + static_cast<int64_t>(pr.y + j) * kTaskWords;
        const int4 ta = reinterpret_cast<const int4*>(plan + rec0)[0], tb = reinterpret_cast<const int4*>(plan + rec0)[1];
        rec.y = tb.x + (local - j * (pr.x == 1 ? pr.z : 0)) * G;
        rec.z = tb.w;
        rec.w = ta.z;
      }
    }
    *reinterpret_cast<int4*>(plan + p.quest + static_cast<int64_t>(i) * kQuestionWords) = rec;
  }
  if (tid < kPlanHeader) {
    const int head[9] = {kPlanMagic, B, Nt, p.W, p.group_q, G, n1, n2, p.max_len};
    plan[tid] = tid < 9 ? head[tid] : 0;
  }
  if (bad && tid == 0) raise_flag(p.err_flag, kFlagBadLayout);
}

}  // namespace

hipError_t launch_paged_reserve(const ReserveParams& p, hipStream_t s) {
  if (p.num_rows <= kFusedRows && p.B + p.Nt <= kFusedSequences) {
    reserve_kernel<true><<<1, kThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  reserve_kernel<false><<<1, kThreads, 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.num_rows == 0) return e;
  rows_kernel<<<static_cast<unsigned>((static_cast<int64_t>(p.num_rows) + 255) / 256), 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_paged_plan(const PagedPlanParams& p, hipStream_t s) {
  plan_kernel<<<1, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace ippd
