// Rotation of new tokens at their virtual positions (Sec. 4.1) and their write
// into pages through the slot map.
//
// A token's slot is page * page_tokens + offset.  Its key goes to row `offset`
// of the page's keys, its value to column offset % 8 of the page's 8-token
// block offset / 8.  Cos and sin come from the fp64-reduced angle
// (rope_cos_sin) and rotations round as in the contiguous cache's kernels, so
// both caches hold the same bits.
//
// What bounds it is the copy, every byte of q, k and v loaded and stored once;
// for a decode step's few tokens the latency of one load and one store (256
// tokens of 32 + 8 heads x 128: 5.0 us; 5.6 with a value head's elements in
// 16-byte pieces a lane, whose stores touch a line a lane).
#include <algorithm>

#include "ippd_device.h"
#include "paged_internal.h"

namespace ippd {

namespace {

// Up to so many rows a workgroup takes one row, above them eight.  32 + 8 heads x
// 128, bf16: 1500 rows without queries 11.2 us by one and 9.1 by eight, with them
// 14.4 and 18.4, 3000 rows 23.6 and 20.8.
constexpr int kStepRows = 1024, kStepRowsWithQueries = 2048;

template <typename T> struct Vec16 { static constexpr int N = 16 / static_cast<int>(sizeof(T)); typedef T type __attribute__((ext_vector_type(16 / sizeof(T)))); };
// (tensors and pages are promised at 16 bytes, eight floats by themselves would ask for 32)
template <typename T> struct Vec8 { typedef T type __attribute__((ext_vector_type(8), aligned(16))); };

// Element of the slot's key row, and of column 0 of its value block, for kv head g.
__device__ __forceinline__ int64_t key_at(const PagedAppendParams& p, int slot, int g) {
  const int off = slot & ((1 << p.page_shift) - 1);
  return ((((static_cast<int64_t>(slot >> p.page_shift) * p.Hkv + g) << p.page_shift) + off)) * p.D;
}
__device__ __forceinline__ int64_t value_at(const PagedAppendParams& p, int slot, int g) {
  const int off = slot & ((1 << p.page_shift) - 1) & ~7;
  return ((((static_cast<int64_t>(slot >> p.page_shift) * p.Hkv + g) << p.page_shift) + off)) * p.D;
}

// One row a workgroup.  An item is a 16-byte vector of each half of a query or key
// head, or two elements of a value head: a token's value goes to every 16th byte
// (fp32: 32nd) of its block, so neighbouring lanes take neighbouring dims and a
// store touches few lines.  Every load goes out before the row's slot is known;
// the row's D/2 angles are evaluated once, into LDS.
template <typename T>
__global__ __launch_bounds__(1024) void append_row_kernel(PagedAppendParams p) {
  constexpr int VE = Vec16<T>::N;
  typedef typename Vec16<T>::type vec_t;
  typedef T pair_t __attribute__((ext_vector_type(2)));
  const int row = blockIdx.x, half = p.D / 2;
  const int QP = half / VE;
  const int nq = p.q ? p.Hq * QP : 0, nk = p.Hkv * QP, turned = nq + nk, items = turned + p.Hkv * half;
  __shared__ float2 rot[kMaxHalfDim];
  const T* __restrict__ q = static_cast<const T*>(p.q) + row * p.q_stride;
  const T* __restrict__ k = static_cast<const T*>(p.k) + row * p.k_stride;
  const T* __restrict__ v = static_cast<const T*>(p.v) + row * p.v_stride;
  const int slot = p.slot_map[row], pos = p.positions[row];
  const double theta = threadIdx.x < static_cast<unsigned>(half) ? p.inv_freq[threadIdx.x] : 0.0;
  vec_t lo, hi;
  pair_t pr;
  auto load = [&](int e) {
    if (e < turned) {
      const int ee = e < nq ? e : e - nq;
      const T* src = (e < nq ? q : k) + (ee / QP) * p.D + (ee % QP) * VE;
      lo = *reinterpret_cast<const vec_t*>(src);
      hi = *reinterpret_cast<const vec_t*>(src + half);
    } else {
      pr = *reinterpret_cast<const pair_t*>(v + (e - turned) * 2);
    }
  };
  if (threadIdx.x < static_cast<unsigned>(items)) load(threadIdx.x);
  if (slot < 0) return;
  if (slot >= p.slots) {
    if (threadIdx.x == 0) raise_flag(p.err_flag, kFlagBadLayout);
    return;
  }
  if (threadIdx.x < static_cast<unsigned>(half)) {
    float c, sn;
    rope_cos_sin(pos, theta, c, sn);
    rot[threadIdx.x] = make_float2(c, sn);
  }
  __syncthreads();                                   // the slot is the row's: every thread is here
  for (int e = threadIdx.x; e < items; e += blockDim.x) {
    if (e >= static_cast<int>(blockDim.x)) load(e);
    if (e < turned) {
      const int ee = e < nq ? e : e - nq;
      const int h = ee / QP, j0 = (ee % QP) * VE;
      vec_t x, y;
#pragma unroll
      for (int u = 0; u < VE; ++u) {
        const float2 cs = rot[j0 + u];
        float xr, yr;
        rope_rotate(to_f32<T>(lo[u]), to_f32<T>(hi[u]), cs.x, cs.y, xr, yr);
        x[u] = from_f32<T>(xr);
        y[u] = from_f32<T>(yr);
      }
      T* dst = e < nq ? static_cast<T*>(p.q_rot) + (static_cast<int64_t>(row) * p.Hq + h) * p.D + j0
                      : static_cast<T*>(p.k_pages) + key_at(p, slot, h) + j0;
      *reinterpret_cast<vec_t*>(dst) = x;
      *reinterpret_cast<vec_t*>(dst + half) = y;
    } else {
      const int g = (e - turned) / half, d = (e - turned) % half * 2;
      T* dst = static_cast<T*>(p.v_pages) + value_at(p, slot, g) + d * 8 + (slot & 7);
      dst[0] = pr[0];
      dst[8] = pr[1];
    }
  }
}

// Eight rows a workgroup.  Waves 0 and 1 turn keys, 2 and 3 carry the values,
// then all turn the queries: lane (row, 8 pairs) holds its angles' cos and sin for
// all heads, evaluated once for the workgroup.  Values: eight rows in consecutive slots of one 8-token block are
// transposed in registers into pieces of a dim's eight tokens, put in order in
// LDS and written as whole lines, by the workgroup that holds the first of them,
// so that a fill whose rows do not start on a multiple of eight writes whole
// blocks too; other rows are written by themselves, element by element.
//
// The inputs and the values' lines go with the non-temporal hint, the keys without:
// 30.7k tokens of 8 heads x 128 (252 MB moved), bf16: 67 us with values in 16-byte
// pieces (129 with the hint, which then writes parts of lines), 63.5 by whole
// lines, 55.4 with the hint on them, 57.9 with it on the keys as well, 54.2 (4.6 TB/s)
// with angles evaluated once a workgroup and not once a wave.
template <typename T, int D>
__global__ __launch_bounds__(256) void append_rows_kernel(PagedAppendParams p) {
  typedef typename Vec8<T>::type vec_t;
  constexpr int half = D / 2, P = half / 8, HPW = 64 / (8 * P);   // pieces of 8 pairs a row; heads a wave holds
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r0 = blockIdx.x * 8;
  // slots of rows r0 - 7 .. r0 + 14: whether a block is whole takes its rows' all
  __shared__ int near[24];
  __shared__ vec_t turn_v[2][64 * 8];
  __shared__ __attribute__((aligned(16))) float2 rot[8][half];
  if (threadIdx.x < 22) {
    const int r = r0 - 7 + static_cast<int>(threadIdx.x);
    int slot = r >= 0 && r < p.num_rows ? p.slot_map[r] : -1;
    if (slot >= p.slots) {
      raise_flag(p.err_flag, kFlagBadLayout);
      slot = -1;
    }
    near[threadIdx.x] = slot;
  }
  const int t = lane / P % 8, j0 = (lane % P) * 8, hs = lane / (8 * P);
  const int row = min(r0 + t, p.num_rows - 1);
  const T* ksrc = static_cast<const T*>(p.k) + row * p.k_stride + j0;
  const T* qsrc = static_cast<const T*>(p.q) + row * p.q_stride + j0;
  struct Halves { vec_t lo, hi; } kf, qf;
  auto load = [&](const T* src) {
    return Halves{__builtin_nontemporal_load(reinterpret_cast<const vec_t*>(src)),
                  __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(src + half))};
  };
  // fp32: the first head of each goes out before the slots are known (12k rows of 6 +
  // 2 heads x 64 23.4 -> 20.2 us; bf16, whose registers then allow fewer waves,
  // 30.7k tokens 54.2 -> 58.2)
  constexpr bool EARLY = sizeof(T) == 4;
  const int h0 = wave * HPW + hs;
  if constexpr (EARLY) {
    if (wave < 2 && h0 < p.Hkv) kf = load(ksrc + h0 * D);
    if (p.q && h0 < p.Hq) qf = load(qsrc + h0 * D);
  }
  {
    const int mine = threadIdx.x / 32, pos = p.positions[min(r0 + mine, p.num_rows - 1)];
#pragma unroll
    for (int j = threadIdx.x % 32; j < half; j += 32) {
      float c, s;
      rope_cos_sin(pos, p.inv_freq[j], c, s);
      rot[mine][j] = make_float2(c, s);
    }
  }
  __syncthreads();
  float cs[8], sn[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float2 x = rot[t][j0 + u];
    cs[u] = x.x;
    sn[u] = x.y;
  }
  const int slot = r0 + t < p.num_rows ? near[7 + t] : -1;
  auto turn = [&](const Halves& f, T* dst) {
    const vec_t lo = f.lo, hi = f.hi;
    vec_t x, y;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      float xr, yr;
      rope_rotate(to_f32<T>(lo[u]), to_f32<T>(hi[u]), cs[u], sn[u], xr, yr);
      x[u] = from_f32<T>(xr);
      y[u] = from_f32<T>(yr);
    }
    *reinterpret_cast<vec_t*>(dst) = x;
    *reinterpret_cast<vec_t*>(dst + half) = y;
  };
  if (wave < 2) {
    if (slot >= 0) {
      T* dst = static_cast<T*>(p.k_pages) + key_at(p, slot, 0) + j0;
      const int64_t head = static_cast<int64_t>(D) << p.page_shift;
      if (EARLY && h0 < p.Hkv) turn(kf, dst + h0 * head);
#pragma unroll 4
      for (int g = h0 + (EARLY ? 2 * HPW : 0); g < p.Hkv; g += 2 * HPW) turn(load(ksrc + g * D), dst + g * head);
    }
  } else {
    const T* v = static_cast<const T*>(p.v);
    T* vp = static_cast<T*>(p.v_pages);
    for (int u = 0; u < 8; ++u) {
      const int s = near[7 + u];
      if (s < 0) continue;
      const int a = s & 7, l = 7 + u - a;            // the block's first row, as an index of near
      bool whole = true;
#pragma unroll
      for (int w = 0; w < 8; ++w) whole = whole && near[l + w] == s - a + w;
      if (whole && a != 0) continue;                 // its first row writes it
      const int items = p.Hkv * (D / 8);
      for (int e0 = (wave - 2) * 64; e0 < items; e0 += 128) {
        const int e = min(e0 + lane, items - 1);     // 8 dims of a head
        const int g = e / (D / 8), d0 = (e % (D / 8)) * 8;
        const T* src = v + static_cast<int64_t>(r0 + u) * p.v_stride + g * D + d0;
        if (whole) {
          vec_t x[8];
#pragma unroll
          for (int w = 0; w < 8; ++w) x[w] = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(src + w * p.v_stride));
          // dim d of item i is piece 8 i + d of the wave's; piece c is at c ^ (c / 8 % 8)
          vec_t* mine = turn_v[wave - 2];
          __builtin_amdgcn_wave_barrier();           // (a wave's LDS operations keep their order)
#pragma unroll
          for (int d = 0; d < 8; ++d) {
            vec_t y;
#pragma unroll
            for (int w = 0; w < 8; ++w) y[w] = x[w][d];
            mine[8 * lane + (d ^ (lane & 7))] = y;
          }
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int c = 64 * k + lane, item = e0 + c / 8;
            const vec_t y = mine[c ^ (c / 8 % 8)];
            const int gi = item / (D / 8), di = item % (D / 8) * 8 + c % 8;
            if (item < items) __builtin_nontemporal_store(y, reinterpret_cast<vec_t*>(vp + value_at(p, s, gi) + di * 8));
          }
        } else if (e0 + lane < items) {
          T* dst = vp + value_at(p, s, g) + d0 * 8;
          const vec_t x = *reinterpret_cast<const vec_t*>(src);
#pragma unroll
          for (int d = 0; d < 8; ++d) dst[d * 8 + a] = x[d];
        }
      }
    }
  }
  if (p.q && slot >= 0) {
    T* dst = static_cast<T*>(p.q_rot) + static_cast<int64_t>(row) * p.Hq * D + j0;
    if (EARLY && h0 < p.Hq) turn(qf, dst + h0 * D);
#pragma unroll 4
    for (int h = h0 + (EARLY ? 4 * HPW : 0); h < p.Hq; h += 4 * HPW) turn(load(qsrc + h * D), dst + h * D);
  }
}

template <typename T>
void launch_append(const PagedAppendParams& p, hipStream_t s) {
  if (p.num_rows <= (p.q ? kStepRowsWithQueries : kStepRows)) {
    constexpr int VE = Vec16<T>::N;
    const int items = ((p.q ? p.Hq : 0) + p.Hkv) * (p.D / 2 / VE) + p.Hkv * (p.D / 2);
    const int threads = std::min(1024, (items + 63) / 64 * 64);
    append_row_kernel<T><<<p.num_rows, threads, 0, s>>>(p);
    return;
  }
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(p.num_rows) + 7) / 8);
  if (p.D == 64) append_rows_kernel<T, 64><<<grid, 256, 0, s>>>(p);
  else append_rows_kernel<T, 128><<<grid, 256, 0, s>>>(p);
}

}  // namespace

hipError_t launch_paged_append(int dtype, const PagedAppendParams& p, hipStream_t s) {
  if (dtype == 0) launch_append<float>(p, s);
  else launch_append<uint16_t>(p, s);
  return hipGetLastError();
}

}  // namespace ippd
