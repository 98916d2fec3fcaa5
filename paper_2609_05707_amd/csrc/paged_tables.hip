// Bookkeeping of the paged cache: block tables and slot maps from request
// lengths, and the attention's plan of a decode step.
//
// Both are a few thousand integers, so what bounds them is latency: the
// dependent round trips to memory and the barriers of a scan.  One workgroup
// does a call, with as many threads as it has sequences or rows (1024 at most);
// only a slot map of many rows gets a launch of its own.
#include "ippd_device.h"
#include "paged_internal.h"

namespace ippd {

namespace {

constexpr int kThreads = 1024;                       // at most; a launch has as many as its sequences (or rows) ask for
constexpr int kWaves = kThreads / 64;
// reserve_kernel fills the slot map itself up to these sizes (one launch); its
// copies of the sequences' rows and lengths then fit the LDS
constexpr int kFusedSequences = 2048;
constexpr int kFusedRows = 8192;

constexpr int kFlagPagesExhausted = 4;

// v of the lane that a DPP control names, 0 where there is none or row_mask leaves the row out.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t dpp(int64_t v) {
  const uint32_t lo = dpp<CTRL, ROWS>(static_cast<int>(v)), hi = dpp<CTRL, ROWS>(static_cast<int>(v >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// Sum over this lane and those below it: four shifts within rows of 16 lanes,
// then the rows' sums passed on (row_shr 1, 2, 4, 8, row_bcast 15 and 31).
template <typename V>
__device__ __forceinline__ V wave_inclusive(V v) {
  v += dpp<0x111, 0xF>(v);
  v += dpp<0x112, 0xF>(v);
  v += dpp<0x114, 0xF>(v);
  v += dpp<0x118, 0xF>(v);
  v += dpp<0x142, 0xA>(v);
  v += dpp<0x143, 0xC>(v);
  return v;
}

// Sum over this lane and those below it in its row of 16.
template <typename V>
__device__ __forceinline__ V row_inclusive(V v) {
  v += dpp<0x111, 0xF>(v);
  v += dpp<0x112, 0xF>(v);
  v += dpp<0x114, 0xF>(v);
  v += dpp<0x118, 0xF>(v);
  return v;
}
// The same with the largest value in place of the sum, none of them negative.
__device__ __forceinline__ int row_max(int v) {
  v = max(v, dpp<0x111, 0xF>(v));
  v = max(v, dpp<0x112, 0xF>(v));
  v = max(v, dpp<0x114, 0xF>(v));
  v = max(v, dpp<0x118, 0xF>(v));
  return v;
}
__device__ __forceinline__ int wave_max(int v) {
  v = row_max(v);
  v = max(v, dpp<0x142, 0xA>(v));
  v = max(v, dpp<0x143, 0xC>(v));
  return v;
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  const uint32_t lo = lane_value(static_cast<int>(v), lane), hi = lane_value(static_cast<int>(v >> 32), lane);
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// Exclusive prefix sums over the workgroup, and their totals.  The waves' sums
// meet in LDS and every wave adds them up in a row of lanes (kWaves is 16).  Two
// buffers are used in turn: one barrier a sum, and the next sum's barrier
// separates a buffer's readers from its next writers.
struct Scan {
  int64_t (*lds)[kWaves][2];
  int turn;
  // The places of waves that the launch does not have; a barrier follows.
  __device__ __forceinline__ void clear() const {
    if (threadIdx.x < 4 * kWaves) (&lds[0][0][0])[threadIdx.x] = 0;
  }
  template <typename V>
  __device__ __forceinline__ V place(V inc, int col, int64_t (*at)[2], V& total) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const V up = row_inclusive<V>(static_cast<V>(at[threadIdx.x & 15][col]));
    total = lane_value(up, 15);
    return (wave ? lane_value(up, wave - 1) : V(0)) + inc;
  }
  __device__ __forceinline__ void operator()(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb) {
    const int64_t ia = wave_inclusive(a), ib = wave_inclusive(b);
    int64_t (*at)[2] = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 63) {
      at[threadIdx.x >> 6][0] = ia;
      at[threadIdx.x >> 6][1] = ib;
    }
    __syncthreads();
    a = place(ia, 0, at, ta) - a;
    b = place(ib, 1, at, tb) - b;
  }
  __device__ __forceinline__ int operator()(int v, int& total) {
    const int inc = wave_inclusive(v);
    int64_t (*at)[2] = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 63) at[threadIdx.x >> 6][0] = inc;
    __syncthreads();
    return place(inc, 0, at, total) - v;
  }
  // The largest of the threads' values before this one's (none negative).
  __device__ __forceinline__ int latest(int v) {
    const int inc = wave_max(v), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t (*at)[2] = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 63) at[threadIdx.x >> 6][0] = inc;
    __syncthreads();
    const int up = row_max(static_cast<int>(at[threadIdx.x & 15][0]));
    return max(dpp<0x138, 0xF>(inc), wave ? lane_value(up, wave - 1) : 0);
  }
};
static_assert(kWaves == 16, "the waves' sums are added up in a row of lanes");

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

// put(k, w, get(k, w)) for every k < total, where w is the sequence of this window
// that page k falls to: thread t's has the pages ex .. ex + n - 1.  first: ex of
// each, in LDS (a barrier lies behind it).  Few pages find theirs by a search each;
// of more a thread takes kPer in a row, and the sequence of a page is the last that
// marked one up to it.  5679 pages of 671 sequences take
// 7.9 us a call, 1.4 more with a search and a round trip each (6 more with four
// searches at once: the searches' instructions are what costs).
constexpr int kPer = 4;
static_assert(kThreads <= 1 << 16, "a mark has 16 bits");
template <typename G, typename P>
__device__ __forceinline__ void move_pages(Scan& scan, uint16_t* marks, const int* first, int sequences, int ex, int n,
                                           int total, G get, P put) {
  const int tid = threadIdx.x, threads = blockDim.x;
  if (total <= threads) {
    if (tid < total) {
      const int w = last_at_most(first, sequences, tid);
      put(tid, w, get(tid, w));
    }
    return;
  }
  for (int k0 = 0; k0 < total; k0 += kPer * threads) {
    uint64_t mine = 0;
    __builtin_memcpy(marks + kPer * tid, &mine, sizeof mine);
    __syncthreads();
    if (n > 0 && ex < k0 + kPer * threads && ex + n > k0) marks[max(ex, k0) - k0] = static_cast<uint16_t>(tid);
    __syncthreads();
    __builtin_memcpy(&mine, marks + kPer * tid, sizeof mine);
    int w[kPer], v[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int x = static_cast<int>(mine >> (16 * u)) & 0xFFFF;
      w[u] = u ? max(w[u - 1], x) : x;
    }
    const int before = scan.latest(w[kPer - 1]), k = k0 + kPer * tid;
    if (k >= total) continue;                        // (uniform barriers: the loop's count is the workgroup's)
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      w[u] = max(w[u], before);
      v[u] = get(min(k + u, total - 1), w[u]);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (k + u < total) put(k + u, w[u], v[u]);
  }
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
// prefix sum over the sequences and then a flat loop over the pages
// (move_pages): 32 contexts of 256 pages cost as many rounds as 8192 sequences
// of one.
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
  __shared__ int64_t sums[2][kWaves][2];
  __shared__ int first[kThreads];                    // pages before the sequence, in this window
  __shared__ int from[kThreads];                     // its first page moved
  __shared__ __attribute__((aligned(8))) uint16_t marks[kPer * kThreads];   // the sequence whose pages begin at a page
  __shared__ int taken;
  __shared__ int row0[ROWS ? kFusedSequences : 1], after[ROWS ? kFusedSequences : 1], got[ROWS ? kFusedSequences : 1];
  __shared__ int q0[ROWS ? kFusedSequences : 1];
  const int tid = threadIdx.x, threads = blockDim.x, S = p.B + p.Nt, sh = p.page_shift;
  const int64_t cap = static_cast<int64_t>(p.table_pages) << sh;
  const int f = *p.free_count;
  Scan scan = {sums, 0};
  scan.clear();
  if (tid == 0) taken = 0;

  // checks, and the pages given back
  bool bad = f < 0 || f > p.num_pages;
  int64_t back = 0;
  for (int s = tid; s < S; s += threads) {
    const int len = p.seq_len[s], c = p.new_tokens[s], a = p.token_start[s], e = p.token_start[s + 1];
    bad = bad || len < 0 || len > cap || a < 0 || e < a || e > p.num_rows || c > e - a;
    if (c < 0 && len > 0) back += pages_of(len, sh) - pages_of(c < -len ? 0 : len + c, sh);
    if constexpr (ROWS) row0[s] = a;
  }
  for (int b = tid; b < p.B; b += threads) {
    const int qa = p.q_start[b], qb = p.q_start[b + 1];
    bad = bad || qb < qa || (b == 0 && qa != 0) || (b == p.B - 1 && qb != p.Nt);
    if constexpr (ROWS) q0[b] = qa;
  }
  __syncthreads();
  int64_t total_back, none = 0, zero;
  scan(back, none, total_back, zero);
  bad = __syncthreads_or(bad || total_back > p.num_pages - f);
  if (bad) {                                         // nothing is moved: no row of the call is served
    if (tid == 0) raise_flag(p.err_flag, kFlagBadLayout);
    for (int s = tid; s < S; s += threads) p.served[s] = 0;
    if constexpr (ROWS) {
      for (int r = tid; r < p.num_rows; r += threads) {
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
    for (int s0 = 0; s0 < S; s0 += threads) {
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
      const int ex = scan(n, total);
      first[tid] = ex;
      from[tid] = keep;
      __syncthreads();
      move_pages(scan, marks, first, min(threads, S - s0), ex, n, total,
                 [&](int k, int w) {
                   return p.block_table[static_cast<int64_t>(s0 + w) * p.table_pages + from[w] + (k - first[w])];
                 },
                 [&](int k, int, int page) {
                   // (an id outside the pool goes back too: the stack's count holds, and its next taker gets no slot)
                   if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.num_pages)) raise_flag(p.err_flag, kFlagBadLayout);
                   p.free_pages[f1 - 1 - (carry + k)] = page;
                 });
      carry += total;
    }
  }
  __syncthreads();                                   // the pages given back are on the stack

  // grow
  int carry = 0;
  for (int s0 = 0; s0 < S; s0 += threads) {
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
    const int ex = scan(need, total);
    // (the sums need no 64 bits: the rows, and with them the new tokens, number
    // fewer than 2^31)
    const int upto = carry + ex + need;
    const bool ok = fits && (need == 0 || upto <= f1);
    first[tid] = ex;
    from[tid] = have;
    const int most = wave_max(ok && need > 0 ? upto : 0);
    if ((tid & 63) == 63) atomicMax(&taken, most);
    if (s < S) {
      int now = len, moved = 0;
      if (ok) {
        now = len + c;
        moved = c;
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
    move_pages(scan, marks, first, min(threads, S - s0), ex, need, run,
               [&](int k, int) { return p.free_pages[f1 - 1 - (carry + k)]; },
               [&](int k, int w, int page) {
                 p.block_table[static_cast<int64_t>(s0 + w) * p.table_pages + from[w] + (k - first[w])] = page;
               });
    carry += total;
  }
  __syncthreads();                                   // tables, and the page count
  if (tid == 0) *p.free_count = f1 - taken;
  if constexpr (ROWS) {
    for (int r = tid; r < p.num_rows; r += threads) {
      const int s = last_at_most(row0, S, r);
      int base = 0;
      if (s >= p.B) base = after[last_at_most(q0, p.B, s - p.B)];
      write_row(p, r, s, r - row0[s], got[s], after[s], base);
    }
  }
}

// The slot map of many rows, a thread per row; the reservation's kernel has
// left the lengths after it and what each sequence was served.  Up to
// kFusedSequences the offsets are searched in LDS, a round trip to memory and not
// one a step.
template <bool LDS>
__global__ __launch_bounds__(256) void rows_kernel(ReserveParams p) {
  __shared__ int row_l[LDS ? kFusedSequences : 1], q_l[LDS ? kFusedSequences : 1];
  const int S = p.B + p.Nt, r = blockIdx.x * 256 + threadIdx.x;
  if constexpr (LDS) {
    for (int i = threadIdx.x; i < S; i += 256) row_l[i] = p.token_start[i];
    for (int i = threadIdx.x; i < p.B; i += 256) q_l[i] = p.q_start[i];
    __syncthreads();
  }
  if (r >= p.num_rows) return;
  const int* row0 = LDS ? row_l : p.token_start;
  const int* q0 = LDS ? q_l : p.q_start;
  const int s = last_at_most(row0, S, r);
  const int got = max(p.served[s], 0);
  int base = 0;
  if (s >= p.B) base = p.seq_len[last_at_most(q0, p.B, s - p.B)];
  write_row(p, r, s, r - row0[s], got, p.seq_len[s], base);
}

// ---------------------------------------------------------------------------
// Plan of a decode step's attention: see paged_internal.h for the lines.
//
// The two lines' tasks are numbered, placed and given their states by prefix
// sums over prompts and questions.  Up to kPlanLds sequences everything that is
// read twice (lengths, offsets, ranks, prompts) is in LDS and the call takes
// two round trips to memory, the inputs in and the plan out; larger batches
// keep it in the plan.
// ---------------------------------------------------------------------------
constexpr int kPlanLds = 1024;
// Tiles that the start of a task costs a piece of the block line (its rows' queries
// and the ring's first tiles, some 8 us): they count as length, so that a piece
// in which a task begins has fewer.  8 prompts of 8192 x 32, three layers: 258 us
// without, 248 with 4, 250 with 8.
constexpr int kSetup = 4;
// The shortest pieces of the block line, in tiles; longer than kSetup, so that
// every piece has a tile.  One prompt of 4096 tokens x 16 questions, eight layers:
// 150 us at 4 or 5, 145 at 6 and 8.
constexpr int kShortest = 6;
static_assert(kShortest > kSetup, "a piece may not lie between two tasks' tiles");

// a / b for 0 <= a < 2^52, 0 < b.  The double nearest a / b is on the quotient's side
// of the next integer: a / b lies 1 / b below it at least, which is 1 / a of it.
// (A line has fewer than 2^47 places.  The lines' shares may come from more, and are
// then near enough.)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return static_cast<int64_t>(static_cast<double>(a) / static_cast<double>(b));
}

// A line of T tiles cut into n <= T pieces, the first T % n of them one tile longer.
struct Line {
  int64_t size, longer, edge;                        // tiles of a short piece; pieces that are longer, and where they end
  double per, per1;                                  // 1 / size, 1 / (size + 1)
  int n;
  __device__ __forceinline__ Line(int64_t tiles, int pieces) : n(pieces) {
    size = quotient(tiles, max(pieces, 1));
    longer = tiles - size * pieces;
    edge = longer * (size + 1);
    per = 1.0 / static_cast<double>(size);
    per1 = 1.0 / static_cast<double>(size + 1);
  }
  __device__ __forceinline__ int64_t start(int p) const { return p * size + (p < longer ? p : longer); }
  // The piece that place x lies in: the product is within one of it.
  __device__ __forceinline__ int piece_of(int64_t x) const {
    const bool low = x < edge;
    const int64_t a = low ? x : x - edge, d = low ? size + 1 : size;
    const int q = static_cast<int>(static_cast<double>(a) * (low ? per1 : per));
    const int64_t r = a - q * d;
    return q + (r >= d) - (r < 0) + (low ? 0 : static_cast<int>(longer));
  }
};

// The records of the pieces p, p + by, .. < end whose first tile is one of a task's.
// A piece ends with its own places: its record counts its tiles on the block line
// within that task (the next task's record says how many of its tiles are still in
// the piece), on the wave line in all.
template <bool BLOCK>
__device__ __forceinline__ void write_pieces(int32_t* plan, int64_t pieces, const Line& line, int index, int64_t tile0,
                                             int tiles, const int4& t0, const int4& t1, int p, int end, int by) {
  for (; p < end; p += by) {
    // places from the task's first tile on (a piece that begins before the task: from less than its setup's)
    const int64_t from = line.start(p) - tile0, to = from + line.size + (p < line.longer);
    if (from < (BLOCK ? -kSetup : 0)) continue;
    const int tile = static_cast<int>(max(from, static_cast<int64_t>(0)));
    int4* rec = reinterpret_cast<int4*>(plan + pieces + static_cast<int64_t>(p) * kPieceWords);
    rec[0] = make_int4(index, tile, static_cast<int>(BLOCK ? min(to, static_cast<int64_t>(tiles)) - tile : to - from), 0);
    rec[1] = t0;
    rec[2] = t1;
  }
}

// A lane's task (has: it has one), whose `tiles` > 0 tiles follow `setup` places
// from `at` on the line, in pieces first .. first + states - 1: its record and its
// pieces'.  All lanes of a wave are here: one or two tasks of many pieces have theirs
// written by the whole wave, some 700 cycles each, where a lane takes 300 a record
// (one prompt of 4096 x 16, 22 pieces: 9300 cycles for the block line, 4900 so; 8
// tasks of 8 pieces 6200, 10000 so).
template <bool BLOCK>
__device__ __forceinline__ void write_task(int32_t* plan, int64_t tasks, int64_t pieces, const Line& line, bool has,
                                           int index, int64_t at, int tiles, int seq, int len, int rows, int q, int row,
                                           int first, int states) {
  constexpr int kWide = 6, kFew = 2;
  const int64_t tile0 = at + (BLOCK ? kSetup : 0);
  const int lead = BLOCK ? static_cast<int>(min(line.start(first + 1) - tile0, static_cast<int64_t>(tiles))) : 0;
  const int4 t0 = make_int4(seq, len, rows, q), t1 = make_int4(row, first, tiles, lead);
  if (has) {
    int4* t = reinterpret_cast<int4*>(plan + tasks + static_cast<int64_t>(index) * kTaskWords);
    t[0] = t0;
    t[1] = t1;
  }
  uint64_t wide = __ballot(has && states > kWide);
  if (__popcll(wide) > kFew) wide = 0;
  if (has && !(wide >> (threadIdx.x & 63) & 1))
    write_pieces<BLOCK>(plan, pieces, line, index, tile0, tiles, t0, t1, first, first + states, 1);
  while (wide) {
    const int l = __builtin_ctzll(wide);
    wide &= wide - 1;
    auto of = [&](auto v) { return lane_value(v, l); };
    const int p = of(first);
    write_pieces<BLOCK>(plan, pieces, line, of(index), of(tile0), of(tiles), make_int4(of(seq), of(len), of(rows), of(q)),
                        make_int4(of(row), p, of(tiles), of(lead)), p + static_cast<int>(threadIdx.x & 63), p + of(states), 64);
  }
}

__device__ __forceinline__ int tiles_of(int len) { return static_cast<int>((static_cast<uint32_t>(len) + 31u) >> 5); }

template <bool LDS>
__global__ __launch_bounds__(kThreads) void plan_kernel(PagedPlanParams p) {
  constexpr int N = LDS ? kPlanLds + 1 : 1;
  __shared__ int64_t sums[2][kWaves][2];
  __shared__ int len_l[N], start_l[N], rank_l[N], list_l[N];
  __shared__ int4 prompt_l[N];
  __shared__ int2 where_l[N];
  __shared__ int widest;                             // most states of a question
  const int tid = threadIdx.x, threads = blockDim.x, B = p.B, Nt = p.Nt, G = p.G;
  int32_t* plan = p.plan;
  int2* where = reinterpret_cast<int2*>(plan + p.where);   // first state row and states of the block line's tasks
  Scan scan = {sums, 0};
  scan.clear();
  if (tid == 0) widest = 0;
  auto len = [&](int s) { return LDS ? len_l[s] : p.seq_len[s]; };
  auto start = [&](int b) { return LDS ? start_l[b] : p.q_start[b]; };
  auto rank = [&](int i) -> int& { return LDS ? rank_l[i] : plan[p.rank + i]; };
  auto list = [&](int k) { return LDS ? list_l[k] : plan[p.qlist + k]; };
  auto prompt = [&](int b) -> int4& { return LDS ? prompt_l[b] : reinterpret_cast<int4*>(plan + p.prompt)[b]; };

  // checks; the active questions in order
  bool bad = false;
  for (int b = tid; b <= B; b += threads) {
    const int qa = p.q_start[b], qb = b < B ? p.q_start[b + 1] : qa;
    bad = bad || qb < qa || qb - qa > p.max_questions || (b == 0 && qa != 0) || (b == B && qa != Nt);
    if constexpr (LDS) start_l[b] = qa;
  }
  for (int s = tid; s < B + Nt; s += threads) {
    const int n = p.seq_len[s];
    bad = bad || n < 0 || n > p.max_len;
    if constexpr (LDS) len_l[s] = n;
  }
  int on0 = tid < Nt && p.active[tid] != 0;
  bad = __syncthreads_or(bad);
  int nact = 0;
  for (int i0 = 0; i0 < Nt; i0 += threads) {
    const int i = i0 + tid;
    const int on = !bad && (i0 == 0 ? on0 : i < Nt && p.active[i] != 0);
    int total;
    const int ex = nact + scan(on, total);
    if (i < Nt) rank(i) = ex;
    if (on) {
      plan[p.qlist + ex] = i;
      if constexpr (LDS) list_l[ex] = i;
    }
    nact += total;
  }
  if (tid == 0) rank(Nt) = nact;
  __syncthreads();

  // tiles of the two lines
  int64_t t1 = 0, t2 = 0, T1, T2, c1 = 0, none = 0, C1 = 0, zero;
  if (!bad) {
    for (int b = tid; b < B; b += threads) {
      const int n = rank(start(b + 1)) - rank(start(b)), tiles = tiles_of(len(b));
      if (p.group_q > 0 && n * G > 16) {
        const int groups = (n + p.group_q - 1) / p.group_q;
        const int64_t length = tiles > 0 ? static_cast<int64_t>(groups) * (tiles + kSetup) : 0;
        t1 += length;
        c1 += length * (p.by_rows ? max(2, ((n + groups - 1) / groups * G + 15) >> 4) : 2);
      } else if (n > 0) {
        t2 += tiles;
      }
    }
    for (int k = tid; k < nact; k += threads) t2 += tiles_of(len(B + list(k)));
  }
  scan(t1, t2, T1, T2);
  if (T1 > 0) scan(c1, none, C1, zero);
  // workgroups to the lines by their shares of the work, runs of
  // p.wave_shortest tiles at least on the wave line.  Bound by the stream (bf16) a
  // tile costs a workgroup the same on either line (twice as much on the block
  // line: 8 prompts of 8192 x 32 248 -> 269 us, three layers; three quarters
  // 235).  Bound by the products (fp32) it costs half as much as it has row
  // blocks: 8 prompts of 4096 tokens, 8 kv heads x 128, 64 rows 165 us at 4 and 105
  // at 2, 128 rows 181 at 4 and 201 at 2.
  int n1 = 0, n2 = 0;
  if (T1 > 0) {
    const int64_t most = p.W - (T2 > 0 ? 1 : 0), all = C1 + 2 * T2;
    const int64_t share = quotient(C1 * p.W + all / 2, all);
    n1 = static_cast<int>(min(max(min(share, T1 / kShortest), static_cast<int64_t>(1)), most));
  }
  if (T2 > 0) n2 = static_cast<int>(min(static_cast<int64_t>(p.waves) * (p.W - n1), (T2 + p.wave_shortest - 1) / p.wave_shortest));
  const Line line1(T1, n1), line2(T2, n2);

  // block line: contexts, their active questions in even groups
  int64_t tasks = 0, at = 0;
  int rows = 0;
  for (int b0 = 0; b0 < B; b0 += threads) {
    const int b = b0 + tid;
    int groups = 0, per = 0, n = 0, r0 = 0, tokens = 0, kind = 0;
    if (b < B && !bad) {
      r0 = rank(start(b));
      n = rank(start(b + 1)) - r0;
      tokens = len(b);
      if (n > 0 && tokens > 0) {
        kind = p.group_q > 0 && n * G > 16 ? 1 : 2;
        if (kind == 1) {
          groups = (n + p.group_q - 1) / p.group_q;
          per = (n + groups - 1) / groups;           // (and ceil(n / per) is groups again)
        }
      }
    }
    if (T1 == 0) {                                   // no block line
      if (b < B) prompt(b) = make_int4(kind, 0, 0, r0);
      continue;
    }
    const int tiles = tiles_of(tokens);
    int64_t task0 = groups, at0 = static_cast<int64_t>(groups) * (tiles + kSetup), ntask, ntile;
    scan(task0, at0, ntask, ntile);
    task0 += tasks;
    at0 += at;
    int need = 0;
    for (int j = 0; j < groups; ++j) {
      const int64_t x = at0 + static_cast<int64_t>(j) * (tiles + kSetup);
      need += (line1.piece_of(x + kSetup + tiles - 1) - line1.piece_of(x + kSetup) + 1) * (min(per, n - j * per) * G);
    }
    int nrow;
    int row = rows + scan(need, nrow);
    for (int j = 0; wave_any(j < groups); ++j) {
      const bool has = j < groups;
      const int64_t x = has ? at0 + static_cast<int64_t>(j) * (tiles + kSetup) : 0;
      const int gr = min(per, n - j * per) * G, first = line1.piece_of(x + kSetup);
      const int states = line1.piece_of(x + kSetup + tiles - 1) - first + 1;
      const int t = static_cast<int>(task0) + j;
      write_task<true>(plan, p.task1, p.piece1, line1, has, t, x, tiles, b, tokens, gr, r0 + j * per, row, first, states);
      if (has) {
        (LDS ? where_l[t] : where[t]) = make_int2(row, states);
        row += states * gr;
      }
    }
    if (b < B) prompt(b) = make_int4(kind, static_cast<int>(task0), per, r0);
    tasks += ntask;
    rows += nrow;
    at += ntile;
  }
  const int block_tasks = static_cast<int>(tasks);
  __syncthreads();                                   // prompts

  // wave line: the other contexts, then the segments of the active questions
  tasks = at = 0;
  for (int x0 = 0; x0 < B + nact; x0 += threads) {
    const int x = x0 + tid;
    int seq = -1, tokens = 0, q = 0, n = 0;
    if (x < B) {
      const int4 pr = prompt(x);
      if (pr.x == 2) {
        seq = x;
        q = pr.w;
        n = (rank(start(x + 1)) - q) * G;
        tokens = len(x);
      }
    } else if (x < B + nact) {
      q = x - B;
      seq = B + list(q);
      n = G;
      tokens = len(seq);
    }
    const int tiles = tiles_of(tokens);
    int64_t task = tiles > 0, at0 = tiles, ntask, ntile;
    scan(task, at0, ntask, ntile);
    task += tasks;
    at0 += at;
    const int first = tiles > 0 ? line2.piece_of(at0) : 0, np = tiles > 0 ? line2.piece_of(at0 + tiles - 1) - first + 1 : 0;
    int nrow;
    const int row = rows + scan(np * n, nrow);
    write_task<false>(plan, p.task2, p.piece2, line2, tiles > 0, static_cast<int>(task), at0, tiles, seq, tokens, n, q, row, first,
                      np);
    if (x < B) {
      if (seq >= 0) {
        prompt(x).y = row;
        prompt(x).z = np;
      }
    } else if (x < B + nact) {
      *reinterpret_cast<int4*>(plan + p.quest + static_cast<int64_t>(seq - B) * kQuestionWords + 4) = make_int4(row, np, 0, 0);
      if constexpr (LDS) list_l[q] = np;             // (read by this thread alone until here)
    }
    tasks += ntask;
    rows += nrow;
    at += ntile;
  }
  __syncthreads();                                   // states of contexts

  // where the states of each question's context are
  int most = 0;
  for (int i = tid; i < Nt; i += threads) {
    const int k = rank(i);
    int4 rec = make_int4(0, 0, 0, 0);
    if (rank(i + 1) > k) {
      int lo = 0, hi = B - 1;                        // the last prompt that starts at i at most
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start(mid) <= i) lo = mid; else hi = mid - 1;
      }
      const int4 pr = prompt(lo);
      rec.x = 1;
      if (pr.x == 1) {                               // (first task, questions a group)
        const int local = k - pr.w, j = local / pr.z;
        const int2 at1 = LDS ? where_l[pr.y + j] : where[pr.y + j];
        rec.y = at1.x + (local - j * pr.z) * G;
        rec.z = at1.y;
        rec.w = min(pr.z, rank(start(lo + 1)) - pr.w - j * pr.z) * G;
      } else if (pr.x == 2) {                        // (first state's row, states)
        rec.y = pr.y + (k - pr.w) * G;
        rec.z = pr.z;
        rec.w = (rank(start(lo + 1)) - pr.w) * G;
      }
      most = max(most, rec.z + (LDS ? list_l[k] : plan[p.quest + static_cast<int64_t>(i) * kQuestionWords + 5]));
    }
    *reinterpret_cast<int4*>(plan + p.quest + static_cast<int64_t>(i) * kQuestionWords) = rec;
  }
  most = wave_max(most);                             // (a lane's atomic each: 64 questions 5000 cycles)
  if ((tid & 63) == 63) atomicMax(&widest, most);
  __syncthreads();
  if (tid == 0) {
    int4* head = reinterpret_cast<int4*>(plan);
    head[0] = make_int4(kPlanMagic, B, Nt, p.W);
    head[1] = make_int4(p.group_q, G, n1, n2);
    head[2] = make_int4(p.max_len, widest, block_tasks, p.waves);
  }
  if (bad && tid == 0) raise_flag(p.err_flag, kFlagBadLayout);
}

}  // namespace

// Threads for n items: whole waves, kThreads at most.  These kernels are bound
// by latency and, where waves share a SIMD, by the instructions of all of them,
// so that idle waves cost: a plan of 5 to 264 sequences 3.5 to 4 us with 1024 threads.
static int threads_for(int64_t n) { return static_cast<int>(n >= kThreads ? kThreads : n <= 64 ? 64 : (n + 63) / 64 * 64); }

hipError_t launch_paged_reserve(const ReserveParams& p, hipStream_t s) {
  const int sequences = p.B + p.Nt;
  if (p.num_rows <= kFusedRows && sequences <= kFusedSequences) {
    reserve_kernel<true><<<1, threads_for(sequences > p.num_rows ? sequences : p.num_rows), 0, s>>>(p);
    return hipGetLastError();
  }
  reserve_kernel<false><<<1, kThreads, 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.num_rows == 0) return e;
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(p.num_rows) + 255) / 256);
  if (sequences <= kFusedSequences) rows_kernel<true><<<grid, 256, 0, s>>>(p);
  else rows_kernel<false><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_paged_plan(const PagedPlanParams& p, hipStream_t s) {
  const int sequences = p.B + p.Nt, threads = threads_for(sequences);
  if (sequences <= kPlanLds) plan_kernel<true><<<1, threads, 0, s>>>(p);
  else plan_kernel<false><<<1, threads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace ippd
