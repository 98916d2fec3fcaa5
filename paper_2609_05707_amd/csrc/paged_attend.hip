// Attention of one new token per question over the paged cache: the plan's
// pieces (paged_internal.h) in one launch, the join of their partial softmax
// states in a second.
//
// With x_k = scale * q . K_k over the keys of the prompt's context and of the
// question's own segment, out = sum_k e^(x_k) V_k / sum_k e^(x_k).  Any split of
// the keys gives partial states (m = max x, l = sum e^(x - m), o = sum e^(x - m) V)
// that join exactly: m = max m_i, l = sum e^(m_i - m) l_i, o likewise.
//
// A tile is 32 tokens, within one page (16-token pages: two).  Its page id is
// read through the scalar cache a tile ahead, apart from the vector loads that
// carry keys and values; an id outside the pool marks the piece's states as
// bad (l = -1), its tiles are read from page 0, and the question gets no output.
#include <algorithm>

#include "ippd_device.h"
#include "paged_internal.h"
#include "tile_attend.h"

namespace ippd {

namespace {

// Read-only words at a wave-uniform address, through the scalar cache.  (Their
// waits are lgkmcnt's, so they leave the counts of the ring's DMAs alone.)
typedef const int32_t __attribute__((address_space(4)))* scalar_words;
__device__ __forceinline__ scalar_words scalars(const int32_t* p) { return (scalar_words)(uintptr_t)p; }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Task {
  int seq, len, rows, q, row, first, tiles, lead;
  __device__ __forceinline__ void load(const int32_t* plan, int64_t at) {
    scalar_words w = scalars(plan + at);
    seq = w[0]; len = w[1]; rows = w[2]; q = w[3]; row = w[4]; first = w[5]; tiles = w[6]; lead = w[7];
  }
};

// One row block's running state.  l is the lane's own share of the row's sum of
// weights, in fp32 and before the weights are rounded for the value product;
// the four lanes of a row are summed at the end.
template <int D>
struct State {
  f32x4_t o[D / 16];
  float m, l;
};

template <int D>
__device__ __forceinline__ void clear(State<D>& st) {
#pragma unroll
  for (int db = 0; db < D / 16; ++db) st.o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  st.m = -INFINITY;
  st.l = 0.f;
}

// Folds a tile's scores (lane (lg, lr): tokens 8 lg + 4 kb + v of row lr) into
// the state and returns the weights as the value product's operand, rounded to
// the cache's type, since a matrix instruction takes both operands in one (bf16:
// off by 2^-8 of each at most; the sum keeps 32 bits).  A norm-wise error of
// 0.0023 in the outputs where their own rounding is 0.0017; a second product, with
// what the rounding left, ends at 0.0017 too, for 179 -> 226 us at 32768 tokens x
// 64 questions (three layers), 313 -> 325 on 32 ragged prompts (two), 118 -> 124 at
// 4096 x 16 (eight), and makes NaN of an infinite value (times 0).  The
// offset m moves only when a score exceeds it by 2^8 in the exponent.
template <typename T, int D>
__device__ __forceinline__ typename Mfma<T>::Frag fold(const f32x4_t (&sc)[2], State<D>& st, float c) {
  const float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                          fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
  if (wave_any((top - st.m) * c > kRescaleLog2)) {
    const float m = fmaxf(st.m, xor32_max(xor16_max(top)));
    const float alpha = fast_exp2((st.m - (m == -INFINITY ? 0.f : m)) * c);
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) st.o[db] *= alpha;
    st.m = m;
  }
  const float cm = (st.m == -INFINITY ? 0.f : st.m) * c;
  f32x8_t w;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int v = 0; v < 4; ++v) w[4 * kb + v] = fast_exp2(fmaf(sc[kb][v], c, -cm));
  st.l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
  return Mfma<T>::from_f32(w);
}

// The state of a row block's rows to their slots; bad: marked.
template <int D>
__device__ __forceinline__ void publish(const PagedAttendParams& p, const State<D>& st, int64_t row, bool live, bool bad,
                                        int lg) {
  const float l = xor32_sum(xor16_sum(st.l));
  if (!live) return;
  float* dst = p.part_o + row * D + 4 * lg;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4_t*>(dst + 16 * db) = st.o[db];
  if (lg == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * row) = make_float2(st.m, bad ? -1.f : l);
}

// Query fragments of a row: lane (lg, lr) holds dims 32 ds + 8 lg + u.
template <typename T, int D>
__device__ __forceinline__ void load_query(const PagedAttendParams& p, typename Mfma<T>::Frag (&qf)[D / 32], int q0, int r,
                                           int g, int lg) {
  const int i = p.plan[p.qlist + q0 + r / p.G];
  const T* src = static_cast<const T*>(p.q_rot) + (static_cast<int64_t>(i) * p.Hq + g * p.G + r % p.G) * D + 8 * lg;
#pragma unroll
  for (int ds = 0; ds < D / 32; ++ds) qf[ds] = Mfma<T>::load(src + 32 * ds);
}

// Where the tiles of one sequence lie, for kv head g.  A tile lies in one page, or
// at 16 tokens a page in two, of which the second may not exist: it then stands
// for the first.  (All of it in scalar registers: a step of the block line has
// few instructions besides its products.)
template <typename T, int D, bool SMALL>
struct Pages {
  scalar_words table;
  const char* k; const char* v;                      // head g's part of page 0
  uint32_t stride;                                   // bytes of a page, all heads
  int shift, most, last;                             // pages of the pool; the sequence's last page
  bool bad;
  __device__ __forceinline__ void init(const PagedAttendParams& p, int seq, int len, int g) {
    constexpr int ROW = D * static_cast<int>(sizeof(T));
    table = scalars(p.block_table + static_cast<int64_t>(seq) * p.table_pages);
    shift = SMALL ? 4 : p.page_shift;
    most = p.num_pages;
    last = (len - 1) >> shift;
    stride = (static_cast<uint32_t>(p.Hkv) << shift) * ROW;
    const uint64_t head = (static_cast<uint64_t>(g) << shift) * ROW;
    k = static_cast<const char*>(p.k_pages) + head;
    v = static_cast<const char*>(p.v_pages) + head;
    bad = false;
  }
  // Page ids of tile t of the sequence (the second is the first's unless SMALL).
  __device__ __forceinline__ int2 of(int t) const {
    if constexpr (!SMALL) {
      const int x = table[t >> (shift - 5)];
      return make_int2(x, x);
    } else {
      return make_int2(table[2 * t], table[min(2 * t + 1, last)]);
    }
  }
  __device__ __forceinline__ int2 checked(int2 id) {
    const bool no = static_cast<uint32_t>(id.x) >= static_cast<uint32_t>(most) ||
                    (SMALL && static_cast<uint32_t>(id.y) >= static_cast<uint32_t>(most));
    bad = bad || no;
    return no ? make_int2(0, 0) : id;
  }
  // Bytes from k (v) to page `id`, and to tile t's tokens in it.
  __device__ __forceinline__ uint64_t at(int id, int t) const {
    const uint64_t page = static_cast<uint64_t>(static_cast<uint32_t>(id)) * stride;
    if constexpr (SMALL) return page;
    const uint32_t t0 = (static_cast<uint32_t>(t) << 5) & ((1u << shift) - 1u);
    return page + t0 * static_cast<uint32_t>(D * sizeof(T));
  }
};

// Elements before page `id` of kv head g, and before its token t0 within the page.
template <bool SMALL, int D>
__device__ __forceinline__ int64_t page_at(const PagedAttendParams& p, int id, int g, int tile) {
  const int shift = SMALL ? 4 : p.page_shift;
  const int t0 = SMALL ? 0 : (tile << 5) & ((1 << shift) - 1);
  return (((static_cast<int64_t>(id) * p.Hkv + g) << shift) + t0) * D;
}

// ---------------------------------------------------------------------------
// Block line: a workgroup of NW waves, up to RB 16-row blocks each, streams the
// piece's tiles through the LDS ring of tile_attend.h, NS - 1 tiles ahead.
// Every fragment read from LDS serves the wave's row blocks.  Block j of wave w
// holds rows 16 (NW j + w) .., so that few rows spread over all four SIMDs.
// ---------------------------------------------------------------------------
// dma16s and dma16 with the non-temporal hint: a context's tiles are read once, and
// as ordinary lines they push each other and the partial states out of the caches
// (8 prompts of 8192 x 32, three layers: 250 us without it, 227 with).
__device__ __forceinline__ void stream16s(const void* sbase, uint32_t voff, uint32_t lds_block) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               :: "v"(voff), "s"(sbase), "{m0}"(__builtin_amdgcn_readfirstlane(lds_block)) : "memory");
}
__device__ __forceinline__ void stream16(const void* gptr, uint32_t lds_block) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
               :: "v"(gptr), "{m0}"(__builtin_amdgcn_readfirstlane(lds_block)) : "memory");
}

template <typename T, int D, int NW, int NS, bool SMALL>
__device__ __forceinline__ void fetch(uint32_t stage, const Pages<T, D, SMALL>& pages, int2 id, int tile, int wave,
                                      const TileOffsets<T, D, NW, NS>& to) {
  using R = Ring<T, D, NS>;
  constexpr int DPT = R::BLOCKS / NW;
  const uint64_t a = pages.at(id.x, tile);
  if constexpr (!SMALL) {
#pragma unroll
    for (int d = 0; d < DPT; ++d) {
      const int q = wave + NW * d;                   // wave-uniform
      stream16s((q < R::KBLOCKS ? pages.k : pages.v) + a, to.off[d], stage + static_cast<uint32_t>(q) * 1024u);
    }
  } else {
    // the offsets are those of a whole tile: tokens 16 .. 31 sit at the second page's start
    constexpr int HALF = 16 * D * R::E;
    const uint64_t b = pages.at(id.y, tile);
#pragma unroll
    for (int d = 0; d < DPT; ++d) {
      const int q = wave + NW * d;
      const bool second = to.off[d] >= HALF;
      stream16((q < R::KBLOCKS ? pages.k : pages.v) + (second ? b - HALF : a) + to.off[d],
               stage + static_cast<uint32_t>(q) * 1024u);
    }
  }
}

// Raw scores of a stage's keys.
template <typename T, int D, int NS, int RB>
__device__ __forceinline__ void scores(const unsigned char* stage, const typename Mfma<T>::Frag (&qf)[RB][D / 32],
                                       f32x4_t (&sc)[RB][2], int lr, int lg) {
  using R = Ring<T, D, NS>;
  using M = Mfma<T>;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int r = 16 * kb + lr, sw = (r >> R::KSH) & R::KMASK;
    const unsigned char* row = stage + r * (R::CPR * 16);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) sc[rb][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ds = 0; ds < D / 32; ++ds) {
      const int c0 = (8 * lg + 32 * ds) * R::E / 16;
      const typename M::Frag kf = M::lds2(row + ((c0 ^ sw) * 16), row + (((c0 + 1) ^ sw) * 16));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sc[rb][kb] = M::mma(kf, qf[rb][ds], sc[rb][kb]);
    }
  }
}

// Folds a tile's scores and adds the weights times its values (n valid tokens).
template <typename T, int D, int NS, int RB>
__device__ __forceinline__ void values(const unsigned char* stage, f32x4_t (&sc)[RB][2], State<D> (&st)[RB], int n, int lr,
                                       int lg, float c) {
  using R = Ring<T, D, NS>;
  using M = Mfma<T>;
  typename M::Frag pf[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (n < 32) mask_scores(sc[rb], n, lg);
    pf[rb] = fold<T, D>(sc[rb], st[rb], c);
  }
  const int keep = min(max(n - 8 * lg, 0), 8);
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
    const unsigned char* vp = stage + R::KBYTES + lg * R::VBLK + (16 * db + lr) * 8 * R::E;
    typename M::Frag vf = M::lds2(vp, vp + 16);
    if (n < 32) vf = M::keep_first(vf, keep);        // what lies past the end may be anything
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) st[rb].o[db] = M::mma(vf, pf[rb], st[rb].o[db]);
  }
}

// A step of the loop: the scores sn of the next tile (keys at stk) while this
// one's (sc, values at stv, all 32 tokens valid) are folded.  The key reads go
// out first and the softmax covers them, the score products cover the value
// reads; the wave's priority is up over its products, so that they issue back
// to back while the SIMD's other wave runs its softmax.
template <typename T, int D, int NS, int RB>
__device__ __forceinline__ void step(const unsigned char* stk, const unsigned char* stv,
                                     const typename Mfma<T>::Frag (&qf)[RB][D / 32], f32x4_t (&sc)[RB][2],
                                     f32x4_t (&sn)[RB][2], State<D> (&st)[RB], int lr, int lg, float c) {
  using R = Ring<T, D, NS>;
  using M = Mfma<T>;
  typename M::Frag kf[2][D / 32], vf[D / 16], pf[RB];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int r = 16 * kb + lr, sw = (r >> R::KSH) & R::KMASK;
    const unsigned char* row = stk + r * (R::CPR * 16);
#pragma unroll
    for (int ds = 0; ds < D / 32; ++ds) {
      const int c0 = (8 * lg + 32 * ds) * R::E / 16;
      kf[kb][ds] = M::lds2(row + ((c0 ^ sw) * 16), row + (((c0 + 1) ^ sw) * 16));
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) pf[rb] = fold<T, D>(sc[rb], st[rb], c);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) sn[rb][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ds = 0; ds < D / 32; ++ds)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sn[rb][kb] = M::mma(kf[kb][ds], qf[rb][ds], sn[rb][kb]);
  }
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
    const unsigned char* vp = stv + R::KBYTES + lg * R::VBLK + (16 * db + lr) * 8 * R::E;
    vf[db] = M::lds2(vp, vp + 16);
  }
#pragma unroll
  for (int db = 0; db < D / 16; ++db)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) st[rb].o[db] = M::mma(vf[db], pf[rb], st[rb].o[db]);
  __builtin_amdgcn_s_setprio(0);
}

// n tiles of a task from `tile` on, for a wave with RL row blocks (0: it only
// fetches).  Waves of a workgroup differ in RL and meet at the same barriers.
template <typename T, int D, int NW, int NS, int RL, bool SMALL>
__device__ __forceinline__ void stream(const PagedAttendParams& p, unsigned char* ring, const Task& task, int g, int tile,
                                       int n, int64_t row, Pages<T, D, SMALL>& pages, int wave, int lane,
                                       const TileOffsets<T, D, NW, NS>& to) {
  using R = Ring<T, D, NS>;
  using M = Mfma<T>;
  constexpr int DPT = R::BLOCKS / NW, RB = RL ? RL : 1, WRAP = NS * R::STAGE;
  const int lr = lane & 15, lg = lane >> 4, last = n - 1;
  const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring));
  typename M::Frag qf[RB][D / 32];
  State<D> st[RB];
  if constexpr (RL > 0) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      load_query<T, D>(p, qf[rb], task.q, min(16 * (NW * rb + wave) + lr, task.rows - 1), g, lg);
      clear(st[rb]);
    }
  }
  const int end = tile + last;
  int put = tile;                                    // the tile fetched next, and its pages
  int2 id = pages.of(tile);
  auto fetch_next = [&](int stage) {
    const int2 next = pages.of(min(put + 1, end));
    fetch<T, D, NW, NS, SMALL>(lds + stage, pages, pages.checked(id), put, wave, to);
    id = next;
    ++put;
  };
  for (int t = 0; t < NS - 1 && t < n; ++t) fetch_next(t * R::STAGE);
  // tile t is folded in step t, whose barrier also says that every wave is past
  // step t - 1; the stage of tile t - 1 then takes tile t + NS - 1.  Steps in
  // pairs, so that the two sets of scores swap places without copies; as long as
  // there are tiles to fetch the waits are constants.
  f32x4_t sa[RB][2], sb[RB][2];
  wait_tiles<DPT, NS - 2>(min(last, NS - 2));
  __syncthreads();
  if constexpr (RL > 0) scores<T, D, NS, RB>(ring, qf, sa, lr, lg);
  int free = (NS - 1) * R::STAGE, here = 0, then = R::STAGE;   // stages of tiles t - 1, t, t + 1
  auto rest = [&](f32x4_t (&now)[RB][2], f32x4_t (&next)[RB][2]) {
    if constexpr (RL > 0) step<T, D, NS, RB>(ring + then, ring + here, qf, now, next, st, lr, lg, p.c);
    free = here;
    here = then;
    then = then + R::STAGE == WRAP ? 0 : then + R::STAGE;
  };
  auto full = [&](f32x4_t (&now)[RB][2], f32x4_t (&next)[RB][2]) {
    wait_vmcnt<((NS - 3) * DPT < 63 ? (NS - 3) * DPT : 63)>();
    __syncthreads();
    fetch_next(free);
    rest(now, next);
  };
  auto drain = [&](int t, f32x4_t (&now)[RB][2], f32x4_t (&next)[RB][2]) {
    wait_tiles<DPT, NS - 3>(min(last - t - 1, NS - 3));
    __syncthreads();
    if (put <= end) fetch_next(free);
    rest(now, next);
  };
  int t = 0;
  while (put + 1 <= end) {                           // (a full step moves put)
    full(sa, sb);
    full(sb, sa);
    t += 2;
  }
  for (; t + 2 <= last; t += 2) {
    drain(t, sa, sb);
    drain(t + 1, sb, sa);
  }
  const int tail = min(32, task.len - 32 * end);
  if (t < last) {
    drain(t, sa, sb);
    if constexpr (RL > 0) values<T, D, NS, RB>(ring + here, sb, st, tail, lr, lg, p.c);
  } else {
    if constexpr (RL > 0) values<T, D, NS, RB>(ring + here, sa, st, tail, lr, lg, p.c);
  }
  if constexpr (RL > 0) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = 16 * (NW * rb + wave) + lr;
      publish<D>(p, st[rb], row + r, r < task.rows, pages.bad, lg);
    }
  }
}

template <typename T, int D, int NW, int NS, int RB, bool SMALL>
__device__ __forceinline__ void block_piece(const PagedAttendParams& p, unsigned char* ring, int piece, int index, int tile,
                                            int n, Task task, int g, int wave, int lane) {
  TileOffsets<T, D, NW, NS> to;
  to.init(wave, lane);
  const int tasks = scalars(p.plan)[10];
  while (true) {
    Pages<T, D, SMALL> pages;
    pages.init(p, task.seq, task.len, g);
    const int64_t row = static_cast<int64_t>(g) * p.rows + task.row + static_cast<int64_t>(piece - task.first) * task.rows;
    if (RB == 2 && 16 * (NW + wave) < task.rows)
      stream<T, D, NW, NS, RB, SMALL>(p, ring, task, g, tile, n, row, pages, wave, lane, to);
    else if (16 * wave < task.rows)
      stream<T, D, NW, NS, 1, SMALL>(p, ring, task, g, tile, n, row, pages, wave, lane, to);
    else
      stream<T, D, NW, NS, 0, SMALL>(p, ring, task, g, tile, n, row, pages, wave, lane, to);
    if (pages.bad && wave == 0 && lane == 0) raise_flag(p.err_flag, kFlagBadLayout);
    // the next task, if the piece goes on into it
    if (++index >= tasks) break;
    task.load(p.plan, p.task1 + static_cast<int64_t>(index) * kTaskWords);
    if (task.first != piece) break;
    tile = 0;
    n = task.lead;
    __syncthreads();                                 // every wave is past the last tile
  }
}

// ---------------------------------------------------------------------------
// Wave line: a wave streams its piece's tiles through its registers.  The keys
// and values of DEPTH further tiles are in flight while it computes one, across
// the ends of tasks too (a short segment is a tile or two): the page ids run a
// tile ahead of the loads, the record of the next task a task ahead, all by
// scalar loads.  Every tile issues the same loads, behind the piece's last tile
// a token's: the compiler counts them to know what is still in flight,
// and a load under a condition would make it wait for all.  Loads of a last
// tile stay within the sequence's tokens, so that a segment costs the bytes it has.
// ---------------------------------------------------------------------------
// A tile of a piece: its task's sequence, its tokens and tiles, and the tile within
// it.  (What else the task's record holds is read when it is needed, so that the
// places fit the scalar registers.)
struct Place {
  int seq, len, tiles, index, tile;
  __device__ __forceinline__ void load(const PagedAttendParams& p, int i) {
    scalar_words w = scalars(p.plan + p.task2 + static_cast<int64_t>(i) * kTaskWords);
    seq = w[0]; len = w[1]; tiles = w[6]; index = i; tile = 0;
  }
};

template <bool SMALL>
__device__ __forceinline__ int2 page_ids(const PagedAttendParams& p, const Place& at) {
  scalar_words table = scalars(p.block_table + static_cast<int64_t>(at.seq) * p.table_pages);
  const int shift = SMALL ? 4 : p.page_shift, a = (at.tile << 5) >> shift, last = (at.len - 1) >> shift;
  const int x = table[min(a, last)];
  return make_int2(x, SMALL ? table[min(a + 1, last)] : x);
}

// Eight elements, with the non-temporal hint or without.
template <typename T, bool NT>
__device__ __forceinline__ typename Mfma<T>::Frag load8(const T* p) {
  if constexpr (!NT) {
    return Mfma<T>::load(p);
  } else if constexpr (sizeof(T) == 2) {
    return __builtin_bit_cast(typename Mfma<T>::Frag, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
  } else {
    const f32x4_t a = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p));
    const f32x4_t b = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p) + 1);
    return typename Mfma<T>::Frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
}

template <typename T, int D, int DEPTH, bool NT, bool SMALL>
__device__ __forceinline__ void wave_piece(const PagedAttendParams& p, int piece, int g, int lane) {
  using M = Mfma<T>;
  const int lr = lane & 15, lg = lane >> 4;
  scalar_words pw = scalars(p.plan + p.piece2 + static_cast<int64_t>(piece) * kPieceWords);
  const int n = pw[2];
  Place at[DEPTH + 2];                               // of tiles t .. t + DEPTH + 1 (behind the last: that one's first token)
  Place after;                                       // the start of the task behind the furthest place's
  at[0] = {pw[4], pw[5], pw[10], pw[0], pw[1]};
  // (the record behind a line's last task is within the plan, and not used)
  after.load(p, at[0].index + 1);
  auto follow = [&](const Place& from, int t) {      // the place of tile t, behind `from`
    Place to = from;
    if (t >= n) {                                    // its loads are for nothing: one token's
      to.len = min(to.len, 32 * to.tile + 1);
      return to;
    }
    if (++to.tile < to.tiles) return to;
    to = after;
    after.load(p, to.index + 1);
    return to;
  };
  auto checked = [&](int2 id, bool& no) {
    no = static_cast<uint32_t>(id.x) >= static_cast<uint32_t>(p.num_pages) ||
         (SMALL && static_cast<uint32_t>(id.y) >= static_cast<uint32_t>(p.num_pages));
    return no ? make_int2(0, 0) : id;
  };
  // this lane's keys of a tile are those of tokens tile_token(kb, lr), its values
  // those of the eight tokens of block lg; at 16 tokens a page tokens 16 .. 31
  // are the second page's
  const int ktok = tile_token(0, lr);
  auto base_of = [&](const void* pages, int2 id, int tile, int& tok) {
    int64_t base = page_at<SMALL, D>(p, id.x, g, tile);
    if (SMALL && tok >= 16) {
      base = page_at<SMALL, D>(p, id.y, g, tile);
      tok -= 16;
    }
    return static_cast<const T*>(pages) + base;
  };
  struct Set {                                       // a tile in flight, with its rows' queries
    typename M::Frag q[D / 32], k[2][D / 32], v[D / 16];
    bool bad;                                        // its page lies outside the pool
  } set[DEPTH];
  auto load_keys = [&](Set& f, const Place& x, int2 id) {
    const int lim = x.len - 1 - 32 * x.tile;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      int tok = min(ktok + 4 * kb, lim);
      const T* src = base_of(p.k_pages, id, x.tile, tok) + tok * D + 8 * lg;
#pragma unroll
      for (int ds = 0; ds < D / 32; ++ds) f.k[kb][ds] = load8<T, NT>(src + 32 * ds);
    }
  };
  auto load_values = [&](Set& f, const Place& x, int2 id) {
    int tok = 8 * min(lg, (x.len - 1 - 32 * x.tile) >> 3);
    const T* src = base_of(p.v_pages, id, x.tile, tok) + tok * D + 8 * lr;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) f.v[db] = load8<T, NT>(src + 128 * db);
  };
  auto load_rows = [&](Set& f, const Place& x) {
    int i = x.seq - p.B, h = min(lr, p.G - 1);       // a segment's rows are its question's heads
    if (x.seq < p.B) {
      scalar_words w = scalars(p.plan + p.task2 + static_cast<int64_t>(x.index) * kTaskWords);
      const int r = min(lr, w[2] - 1);
      i = p.plan[p.qlist + w[3] + r / p.G];
      h = r % p.G;
      asm volatile("" : "+v"(i));                    // waited for here, not where a segment passes too
    }
    const T* src = static_cast<const T*>(p.q_rot) + (static_cast<int64_t>(i) * p.Hq + g * p.G + h) * D + 8 * lg;
#pragma unroll
    for (int ds = 0; ds < D / 32; ++ds) f.q[ds] = M::load(src + 32 * ds);
  };
  int2 id = page_ids<SMALL>(p, at[0]);
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) {
    at[d + 1] = follow(at[d], d + 1);
    const int2 ahead = page_ids<SMALL>(p, at[d + 1]);
    id = checked(id, set[d].bad);
    // in the loop's order: the waits there are for the worse of both
    load_rows(set[d], at[d]);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(set[d], at[d], id);
    __builtin_amdgcn_sched_barrier(0);
    load_values(set[d], at[d], id);
    __builtin_amdgcn_sched_barrier(0);
    id = ahead;
  }
  bool bad = false, any = false;
  State<D> st;
  clear(st);
  for (int t0 = 0; t0 < n; t0 += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int t = t0 + d;
      if (t >= n) break;
      Set& f = set[d];
      const bool ends = t + 1 >= n || at[1].index != at[0].index;   // the last tile of its task here
      bad = bad || f.bad;
      id = checked(id, f.bad);
      at[DEPTH + 1] = follow(at[DEPTH], t + DEPTH + 1);
      const int2 ahead = page_ids<SMALL>(p, at[DEPTH + 1]);
      f32x4_t sc[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        sc[kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ds = 0; ds < D / 32; ++ds) sc[kb] = M::mma(f.k[kb][ds], f.q[ds], sc[kb]);
      }
      if (at[DEPTH].index != at[0].index) load_rows(f, at[DEPTH]);
      load_keys(f, at[DEPTH], id);
      const int m = at[0].len - 32 * at[0].tile;
      if (m < 32) mask_scores(sc, m, lg);
      const typename M::Frag pf = fold<T, D>(sc, st, p.c);
      if (m < 32) {                                  // what lies past the end may be anything
        const int keep = min(max(m - 8 * lg, 0), 8);
#pragma unroll
        for (int db = 0; db < D / 16; ++db) f.v[db] = M::keep_first(f.v[db], keep);
      }
#pragma unroll
      for (int db = 0; db < D / 16; ++db) st.o[db] = M::mma(f.v[db], pf, st.o[db]);
      load_values(f, at[DEPTH], id);
      if (ends) {
        Task task;
        task.load(p.plan, p.task2 + static_cast<int64_t>(at[0].index) * kTaskWords);
        const int64_t row = static_cast<int64_t>(g) * p.rows + task.row + static_cast<int64_t>(piece - task.first) * task.rows;
        publish<D>(p, st, row + lr, lr < task.rows, bad, lg);
        any = any || bad;
        bad = false;
        clear(st);
      }
      id = ahead;
#pragma unroll
      for (int k = 0; k <= DEPTH; ++k) at[k] = at[k + 1];
    }
  }
  if (any && lane == 0) raise_flag(p.err_flag, kFlagBadLayout);
}

// Whether the buffer holds a plan of this batch's sizes, those that its arrays'
// places follow from (no branches: its loads go out together, and with others).
__device__ __forceinline__ bool plan_fits(const PagedAttendParams& p) {
  scalar_words h = scalars(p.plan);
  return (h[0] == kPlanMagic) & (h[1] == p.B) & (h[2] == p.Nt) & (h[3] == p.W) & (h[4] == p.group_q) & (h[5] == p.G) &
         (h[8] == p.table_pages << p.page_shift) & (h[11] == p.waves);
}

// RB = 0: a batch whose prompts have 16 rows at most, and so no block line.  Its
// contexts stream through the wave line with the non-temporal hint (64 requests
// of up to 16k tokens 376 -> 357 us); beside a block line the wave line holds
// segments mostly, and gains nothing by it (4096 x 16: 137 -> 141, eight layers).
template <typename T, int D, int NW, int NS, int RB, bool SMALL>
__global__ __launch_bounds__(64 * NW, 2) void paged_attend_kernel(PagedAttendParams p) {
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RB ? NS * Ring<T, D, NS>::STAGE : 16];
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = blockIdx.x % p.Hkv, b = blockIdx.x / p.Hkv;
  // a block-line piece's record is read with the header, not behind it
  int index = 0, tile = 0, n = 0;
  Task task = {};
  if constexpr (RB > 0) {
    scalar_words pw = scalars(p.plan + p.piece1 + static_cast<int64_t>(b) * kPieceWords);
    index = pw[0];
    tile = pw[1];
    n = pw[2];
    task.load(p.plan, p.piece1 + static_cast<int64_t>(b) * kPieceWords + 4);
    asm volatile("" : "+s"(index), "+s"(task.seq), "+s"(task.row));
  }
  const int n1 = scalars(p.plan)[6], n2 = scalars(p.plan)[7];
  if (!plan_fits(p)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(p.err_flag, kFlagBadLayout);
    return;
  }
  if constexpr (RB > 0) {
    if (b < n1) {
      block_piece<T, D, NW, NS, RB, SMALL>(p, ring, b, index, tile, n, task, g, wave, lane);
      return;
    }
  }
  const int piece = wave * (p.W - n1) + (b - n1);
  if (piece < n2) wave_piece<T, D, (sizeof(T) * D > 256 ? 1 : 2), RB == 0, SMALL>(p, piece, g, lane);
}

// ---------------------------------------------------------------------------
// Join: a wave takes a (question, head), or four do where some question has many
// states.  A lane folds every (64 / (D / 4) x waves)-th of the head's states for
// four dims; lanes of a wave are joined by swaps, waves in LDS.
//
// What bounds it is latency (a question's record, then its states) and, for many
// questions, the states' bytes.  One wave, its record read with the plan's header:
// 4096 x 16 (23 states) 134 -> 125 us for eight layers, where two or four waves a
// unit, known from the header first, took as long; ragged 317, 330 with two, 348
// with four.  One request of 8192 tokens (65 states) 150 us with one, 134 with four.
// ---------------------------------------------------------------------------
constexpr int kJoinWaves = 4;

struct Part {
  float m, l;
  f32x4_t o;
};
__device__ __forceinline__ void join(Part& a, float m, float l, const f32x4_t& o, float c) {
  const float top = fmaxf(a.m, m), base = top == -INFINITY ? 0.f : top;
  const float x = fast_exp2((a.m - base) * c), y = fast_exp2((m - base) * c);
  a.l = a.l * x + l * y;
  a.o = a.o * x + o * y;
  a.m = top;
}

// The value of the lane 16 (32) away.
__device__ __forceinline__ float far16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 16) ? r[0] : r[1]);
}
__device__ __forceinline__ float far32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// A question's record: whether it is served, and where its states are.
struct Record {
  int on, row0, n0, step0, row1, n1;
  __device__ __forceinline__ void load(const PagedAttendParams& p, int unit) {
    scalar_words w = scalars(p.plan + p.quest + static_cast<int64_t>(min(unit / p.Hq, p.Nt - 1)) * kQuestionWords);
    on = w[0]; row0 = w[1]; n0 = w[2]; step0 = w[3]; row1 = w[4]; n1 = w[5];
  }
};

// Units blockIdx.x * (kJoinWaves / WPU) + .. and on; rec: the first one's record.
template <typename T, int D, int WPU>
__device__ __forceinline__ void join_units(const PagedAttendParams& p, int units, Record rec, float (*part)[64][6], int wave,
                                           int lane) {
  constexpr int L = D / 4, IN = 64 / L, BATCH = 4, PER = kJoinWaves / WPU;   // lanes of a state; states a lane reads at once
  const int sub = wave % WPU, d = (lane % L) * 4, phase = sub * IN + lane / L, phases = WPU * IN;
  const int step = gridDim.x * PER;
  for (int u0 = blockIdx.x * PER; u0 < units; u0 += step) {
    const int u = u0 + wave / WPU;
    const int i = u / p.Hq, hq = u - i * p.Hq, g = hq / p.G, h = hq - g * p.G;
    const Record r = rec;
    if (u0 + step < units) rec.load(p, u + step);
    const bool served = (u < units) & (r.on != 0);
    const int n0 = r.n0, n = served ? n0 + r.n1 : 0;
    const int64_t base = static_cast<int64_t>(g) * p.rows + h;
    Part a = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    bool bad = false;
    for (int k0 = phase; k0 < n; k0 += phases * BATCH) {
      float2 ml[BATCH];
      f32x4_t o[BATCH];
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {              // all of them in flight; past the last, the last again
        const int k = min(k0 + x * phases, n - 1);
        const int64_t row = base + (k < n0 ? r.row0 + static_cast<int64_t>(k) * r.step0 : r.row1 + static_cast<int64_t>(k - n0) * p.G);
        ml[x] = *reinterpret_cast<const float2*>(p.part_ml + 2 * row);
        o[x] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p.part_o + row * D + d));
      }
#pragma unroll
      for (int x = 0; x < BATCH; ++x)
        if (k0 + x * phases < n) {
          bad = bad || ml[x].y < 0.f;
          join(a, ml[x].x, ml[x].y, o[x], p.c);
        }
    }
    // a page outside the pool in any state: no output
    float flag = bad ? 1.f : 0.f;
    flag = fmaxf(flag, far32(flag));
    if constexpr (IN == 4) {
      join(a, far16(a.m), far16(a.l), f32x4_t{far16(a.o[0]), far16(a.o[1]), far16(a.o[2]), far16(a.o[3])}, p.c);
      flag = fmaxf(flag, far16(flag));
    }
    join(a, far32(a.m), far32(a.l), f32x4_t{far32(a.o[0]), far32(a.o[1]), far32(a.o[2]), far32(a.o[3])}, p.c);
    if constexpr (WPU > 1) {
      __syncthreads();                               // the last unit's parts have been read
      float* mine = part[wave][lane];
      mine[0] = a.m; mine[1] = flag > 0.f ? -1.f : a.l;
#pragma unroll
      for (int v = 0; v < 4; ++v) mine[2 + v] = a.o[v];
      __syncthreads();
      if (sub == 0)
        for (int k = 1; k < WPU; ++k) {
          const float* x = part[wave + k][lane];
          flag = x[1] < 0.f ? 1.f : flag;
          join(a, x[0], x[1], f32x4_t{x[2], x[3], x[4], x[5]}, p.c);
        }
    }
    if (served && sub == 0 && lane < L && flag == 0.f) {
      const int64_t at = static_cast<int64_t>(i) * p.Hq + hq;
      const float inv = a.l == 0.f ? 0.f : 1.f / a.l;      // no keys at all: zeros, and lse -inf
      T* dst = static_cast<T*>(p.out) + at * D + d;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_t*>(dst) = a.o * inv;
      } else {
        typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
        u16x4_t y;
#pragma unroll
        for (int v = 0; v < 4; ++v) y[v] = f32_to_bf16(a.o[v] * inv);
        *reinterpret_cast<u16x4_t*>(dst) = y;
      }
      if (p.lse && d == 0) p.lse[at] = a.l == 0.f ? -INFINITY : a.m * p.scale + logf(a.l);
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kJoinWaves) void paged_join_kernel(PagedAttendParams p, int units) {
  __shared__ float part[kJoinWaves][64][6];
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int most = scalars(p.plan)[9];               // states of the widest question
  Record rec;
  rec.load(p, blockIdx.x * kJoinWaves + wave);
  asm volatile("" : "+s"(rec.on), "+s"(rec.row0));   // (read here, with the header, not where it is used)
  if (!plan_fits(p)) return;
  if (most <= 20 * (64 / (D / 4))) {
    join_units<T, D, 1>(p, units, rec, part, wave, lane);
  } else {
    rec.load(p, blockIdx.x);
    join_units<T, D, kJoinWaves>(p, units, rec, part, wave, lane);
  }
}

template <typename T, int D, int NW, int NS, int RB>
hipError_t launch(const PagedAttendParams& p, hipStream_t s) {
  const unsigned grid = static_cast<unsigned>(p.W) * p.Hkv;
  if (p.page_shift == 4) paged_attend_kernel<T, D, NW, NS, RB, true><<<grid, 64 * NW, 0, s>>>(p);
  else paged_attend_kernel<T, D, NW, NS, RB, false><<<grid, 64 * NW, 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // at most a chip full of workgroups, which then go on to further units
  const int units = p.Nt * p.Hq;
  paged_join_kernel<T, D><<<static_cast<unsigned>(std::min(units, 2048)), 64 * kJoinWaves, 0, s>>>(p, units);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attend(int dtype, int D, int waves, int rb, const PagedAttendParams& p, hipStream_t s) {
  if (dtype == 0) {
    if (D == 64) return rb == 0 ? launch<float, 64, 4, 5, 0>(p, s) : launch<float, 64, 4, 5, 1>(p, s);
    return rb == 0 ? launch<float, 128, 8, 4, 0>(p, s) : launch<float, 128, 8, 4, 1>(p, s);
  }
  if (D == 64) {
    if (waves == 8) return launch<uint16_t, 64, 8, 9, 2>(p, s);
    return rb == 0 ? launch<uint16_t, 64, 4, 9, 0>(p, s) : rb == 1 ? launch<uint16_t, 64, 4, 9, 1>(p, s) : launch<uint16_t, 64, 4, 9, 2>(p, s);
  }
  if (waves == 8) return launch<uint16_t, 128, 8, 9, 2>(p, s);
  return rb == 0 ? launch<uint16_t, 128, 4, 5, 0>(p, s) : rb == 1 ? launch<uint16_t, 128, 4, 5, 1>(p, s) : launch<uint16_t, 128, 4, 5, 2>(p, s);
}

}  // namespace ippd
