// Attention of few query rows over the 8-bit cache (lv_kv_attend): one new token
// of a request, or some.
//
// The cache is read once, 2 D bytes a token and key/value head, and that bounds
// the kernel: a token of a head gets 11 clocks of an SM at the copy rate.  In
// them its 2 D codes become fp16 and meet G query heads twice, so both products
// go to the matrix unit, with the cache as the operand of 16 rows and the query
// rows as the one of 8 columns (an operand of 16 query rows would be three
// quarters empty at G = 4):
//     S^T [16 keys x 8 rows] = K Q^T,    O^T [D x 8 rows] += V^T P^T.
// A strip is 16 neighbouring keys, always of one block, and goes from global
// memory into the registers of one warp in the order in which the products want
// it: the sums over D and over keys may take their terms in any order, so lane
// (g, t) = (lane / 4, lane % 4) takes D/4 neighbouring codes of keys g and g + 8
// for K (16 and, 64 on, 16 more), and D/8 of keys 2t, 2t+1, 2t+8, 2t+9 for V,
// and no shared memory is passed.  e4m3 to fp16 is exact.  P^T is S^T's registers
// transposed (movmatrix).  The next keys are asked for once these have met the
// queries, the next values once these have met the weights.
//
// Weights are 2^(x - m + 12) with m the row's running maximum of x = log2(e)
// scale ks S; a strip whose scores are all at most m changes nothing (one vote),
// so m settles after a few strips.  The value scale vs of the strip's block goes
// to the weight, as vs / ref with ref the largest so far; the factor 2^12 keeps
// weights of 2^-26 of the largest normal in fp16, to which they are rounded (11
// bits); a segment whose value scales differ by more than 2^22 is done again row by
// row in fp32 (kDecThin).  bf16 queries are scaled by a power of two to a largest
// element of 2^14, where fp16 holds every one above 2^-28 of that exactly.  All sums
// are fp32.
//
// Work is cut evenly whatever the lengths: the strips of all (request, head, row
// tile) segments stand in one line, and each of W warps takes its W-th of it.  A
// segment that several warps share leaves a part (O, m, l) for each, two a warp
// at most, and k_attend_join adds them in the line's order.
//
// Measured: 256 requests of up to 32,768 tokens, 20/4 heads of 128, 950 MB of
// cache: 181 us with the join, 5.3 TB/s, 0.78 of the copy rate; 16 requests of up
// to 8,192 tokens, 32/8 heads: 41 us.  What is lost: the SMs are served by memory
// at different speeds (equal shares end between 113 and 189 us), and small calls
// wait for the scan, the first loads and the join.
#pragma once

#include "lv_attend.cuh"

namespace lv {

// CTAs of an SM, with one and two row tiles of 8: with four the registers of one
// row tile just spill (256 requests, as this was chosen: 183 us, three CTAs 196, five 263).
constexpr int kDecCtas1 = 4, kDecCtas2 = 2;
constexpr int kDecWarps = 4;       // warps of a CTA; they share only the scan
constexpr int kDecSegment = 4;     // strips' time that a segment's beginning and end cost (0: 6 % slower)
constexpr int kDecMinStrips = 8;   // strips a warp takes at least (5: no change)
constexpr int kDecRows = 16;       // rows of a request that go here: two row tiles of 8
constexpr int kJoinWarps = 8;      // rows of a CTA that joins, a warp each
constexpr float kWeightExp = 12.f;
constexpr float kDecThin = 0x1p-22f;  // least vs / ref under which fp16 holds 2^kWeightExp to 2^-15 of it (its least step is 2^-24)

struct DecodeArgs {
  AttendArgs a;
  int nt;               // row tiles of 8 nt rows
  int most_rows;        // requests of more rows are k_chunk's
  int64_t warps;        // warps launched
  int64_t *prefix;      // [n_req + 1] strips before each request
  bool given;           // prefix is there already, not formed here
  float *part;          // [warps][2][8 nt][D], then m and l [warps][2][8 nt][2]
  float *part_ml;
};

// A request's queries and keys.
struct Span {
  int64_t first;  // its first query
  int64_t n;      // keys of the last query
  int32_t p;      // queries
};

__device__ __forceinline__ Span request_span(const AttendArgs &a, int64_t i, bool *bad) {
  Span s;
  s.first = i;
  s.p = 1;
  if (a.offsets) {
    const int64_t x0 = a.offsets[i], x1 = a.offsets[i + 1];
    if (x0 < 0 || x1 < x0 || x1 > a.n_tok) {
      *bad = true;
      s.first = 0;
      s.p = 0;
    } else {
      s.first = x0;
      s.p = (int32_t)min(x1 - x0, (int64_t)INT32_MAX);
    }
  }
  const int32_t c = a.c[i];
  s.n = (int64_t)c + s.p;
  if (c < 0) {
    *bad = true;
    s.n = 0;
  } else if (s.p > 0 && s.n > (a.width << a.cache.log_b)) {
    *bad = true;
  }
  return s;
}

// Keys that query j of the request sees; the table may hold fewer.
__device__ __forceinline__ int64_t row_limit(const AttendArgs &a, const Span &s, int j) {
  if (s.n == 0) return 0;
  return min(s.n - s.p + j + 1, a.width << a.cache.log_b);
}

__device__ __forceinline__ int64_t span_strips(const AttendArgs &a, const Span &s) {
  return max((int64_t)1, (row_limit(a, s, s.p - 1) + 15) >> 4);  // one of none, so that its rows are written
}

// What a segment counts for in the line: its strips, and what its beginning and its
// end cost in strips' time, so that a warp of many short ones is given fewer.
__device__ __forceinline__ int64_t segment_units(int64_t strips) { return strips + kDecSegment; }

__device__ __forceinline__ int span_tiles(const AttendArgs &a, const Span &s, int rows) {
  return (int)quotient((int64_t)s.p * (a.hq / a.hkv) + rows - 1, rows);
}

__device__ __forceinline__ int64_t request_units(const DecodeArgs &d, int64_t i, bool *bad) {
  const Span s = request_span(d.a, i, bad);
  return s.p == 0 || (int64_t)s.p * (d.a.hq / d.a.hkv) > d.most_rows ? 0 : segment_units(span_strips(d.a, s)) * span_tiles(d.a, s, 8 * d.nt) * d.a.hkv;
}

// The running sums of more than kScan requests, by one CTA.
__global__ void __launch_bounds__(kScan) k_attend_prefix(DecodeArgs d) {
  bool bad = false;
  int64_t base = 0;
  for (int64_t i0 = 0; i0 < d.a.n_req; i0 += kScan) {
    const int n = (int)min((int64_t)kScan, d.a.n_req - i0);
    base = scan_units<kScan>(n, d.prefix + i0, base, [&](int k) { return request_units(d, i0 + k, &bad); });
  }
  if (bad) flag(d.a.status, kStatusData);
}

// Warps that take strips, and the first strip of warp w.
__device__ __forceinline__ int64_t busy_warps(int64_t warps, int64_t units) {
  return max((int64_t)1, min(warps, quotient(units, kDecMinStrips)));
}
__device__ __forceinline__ int64_t warp_start(int64_t w, int64_t W, int64_t units) {
  const int64_t q = quotient(units, W), r = units - q * W;  // the first r warps take one more
  return w * q + min(w, r);
}
__device__ __forceinline__ int64_t warp_of(int64_t u, int64_t W, int64_t units) {
  const int64_t q = quotient(units, W), r = units - q * W, cut = r * (q + 1);
  return u < cut ? quotient(u, q + 1) : r + quotient(u - cut, q);
}

__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The two codes of 16 bits as fp16 (exact).
__device__ __forceinline__ uint32_t lo_half2(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
  return r;
}
__device__ __forceinline__ uint32_t hi_half2(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)(w >> 16)));
  return r;
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

__device__ __forceinline__ uint4 load16(const uint8_t *p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 load8(const uint8_t *p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}

// The codes of a strip in one lane: K of keys g and g + 8, V of keys 2t, 2t+1,
// 2t+8, 2t+9.
template <int D>
struct Strip {
  uint32_t k[2][D / 16];
  uint32_t v[4][D / 32];

  __device__ __forceinline__ void load_keys(const uint8_t *p, int lane, int keys) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < D / 16; j += 4) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (g + 8 * r < keys) x = load16(p + (g + 8 * r) * D + 16 * j + t * 16);  // 64 bytes in a row
        k[r][j] = x.x, k[r][j + 1] = x.y, k[r][j + 2] = x.z, k[r][j + 3] = x.w;
      }
  }
  __device__ __forceinline__ void load_values(const uint8_t *p, int lane, int keys) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = 2 * t + (r & 1) + 8 * (r >> 1);
      if (D == 128) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (key < keys) x = load16(p + key * D + g * (D / 8));
        v[r][0] = x.x, v[r][1] = x.y, v[r][D / 32 - 2] = x.z, v[r][D / 32 - 1] = x.w;
      } else {
        uint2 x = make_uint2(0, 0);
        if (key < keys) x = load8(p + key * D + g * (D / 8));
        v[r][0] = x.x, v[r][1] = x.y;
      }
    }
  }
};

// All rows of a tile again, each alone.  A function of its own: inlined, its state takes
// registers from the loop over strips.
template <int D, bool F16>
__device__ __noinline__ void redo_tile(const AttendArgs &a, int64_t i, int h, int row0, int rows) {
  bool ignore = false;
  const Span sp = request_span(a, i, &ignore);
  const int G = a.hq / a.hkv;
  __syncwarp();
  for (int rr = row0; rr < row0 + rows && rr / G < sp.p; ++rr) {
    const int64_t n = row_limit(a, sp, rr / G);
    redo_row<D, F16, true>(a, sp.first, i, sp.first + rr / G, h * G + rr % G, n, n, true);
  }
}

template <int D, bool F16, int NT>
__global__ void __launch_bounds__(kDecWarps * 32, NT == 1 ? kDecCtas1 : kDecCtas2) k_attend_decode(DecodeArgs d) {
  constexpr int kRows = 8 * NT, kM = D / 16;  // row tile; tiles of 16 elements of the output
  __shared__ int64_t shared_sums[kScan + 1];
  __shared__ unsigned shared_least[kDecWarps];  // a segment's least value scale, lane 0's: there is no register left for it
  const AttendArgs &a = d.a;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  wait_previous();
  bool bad = false;
  const int64_t *sums = d.prefix;
  int64_t units;
  if (d.given) {
    units = sums[a.n_req];
  } else {
    units = scan_units<kDecWarps * 32>((int)a.n_req, shared_sums, 0, [&](int k) { return request_units(d, k, &bad); });
    sums = shared_sums;
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i <= a.n_req; i += kDecWarps * 32) d.prefix[i] = shared_sums[i];
  }
  let_next();
  const int64_t W = busy_warps(d.warps, units);
  const int64_t me = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x;  // neighbours on different SMs
  const int G = a.hq / a.hkv;
  const int64_t begin = me < W ? warp_start(me, W, units) : 0, end = me < W ? warp_start(me + 1, W, units) : 0;
  for (int64_t u = begin; u < end;) {
    // the segment that unit u is in
    const int64_t i = find_unit(sums, a.n_req, u);
    bool ignore = false;
    const Span sp = request_span(a, i, &ignore);
    const int64_t strips = span_strips(a, sp), all_units = segment_units(strips);
    const int tiles = span_tiles(a, sp, kRows);
    const int64_t seg = quotient(u - sums[i], all_units), s0 = u - sums[i] - seg * all_units, s1 = min(strips, s0 + end - u);
    if (s0 >= strips) {
      u += all_units - s0;
      continue;
    }
    const int h = (int)seg / tiles, row0 = ((int)seg - h * tiles) * kRows;
    // query rows: lane (g, t) holds D/4 elements of rows g + 8 nt
    uint32_t qf[NT][D / 8];
    float f[NT][2];       // x = f ks S, rows 2t and 2t + 1
    int lim[NT][2];       // keys these rows see, from the first strip on
    int least = INT32_MAX;
    const int64_t key0 = s0 << 4;
    auto from_key0 = [&](int64_t keys) { return (int)max((int64_t)0, min((int64_t)INT32_MAX, keys - key0)); };
    const int most = from_key0(row_limit(a, sp, sp.p - 1)), count = (int)(s1 - s0);
    // 32 strips at a time, a strip a lane: the blocks of these, of the next 32 and of
    // those after, the scales of these and of the next, so that no load is waited
    // for where it is issued
    int32_t id0, id1, id2;
    float ks, vs, next_ks, next_vs;
    const int32_t *const table_row = a.table + i * a.width;
    auto look_up = [&](int s) {
      const int mine = s + lane;
      return mine < count && (mine << 4) < most ? table_row[(key0 + (mine << 4)) >> a.cache.log_b] : -1;
    };
    auto checked = [&](int32_t id) {
      if (id >= -1 && id < a.cache.n_blocks) return id;
      bad = true;
      return -1;
    };
    auto scales_of = [&](int32_t id, float *k, float *v) {
      *k = *v = 0.f;
      if (id >= 0) {
        *k = a.cache.k_scale[(int64_t)id * a.cache.heads + h];
        *v = a.cache.v_scale[(int64_t)id * a.cache.heads + h];
      }
    };
    id0 = look_up(0);
    id1 = look_up(32);
    id2 = look_up(64);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = row0 + 8 * nt + g, j = row / G, hh = row % G;
      const bool in = j < sp.p;
      const uint16_t *qp = (const uint16_t *)a.q + (sp.first + j) * a.q_stride + ((int64_t)h * G + hh) * D + t * 16;
      float mine = a.scale;
#pragma unroll
      for (int k = 0; k < D / 8; k += 4) {  // 16 elements, and those 64 elements on
        uint4 x = make_uint4(0, 0, 0, 0);
        if (in) x = *reinterpret_cast<const uint4 *>(qp + k / 8 * 64 + k % 8 * 2);
        qf[nt][k] = x.x, qf[nt][k + 1] = x.y, qf[nt][k + 2] = x.z, qf[nt][k + 3] = x.w;
      }
      if (!F16) {
        uint32_t top = 0;  // the largest magnitude's bits
#pragma unroll
        for (int k = 0; k < D / 8; ++k)
          top = max(top, max((qf[nt][k] & 0x7fff0000u), (qf[nt][k] & 0x7fffu) << 16));
        top = max(top, __shfl_xor_sync(~0u, top, 1));
        top = max(top, __shfl_xor_sync(~0u, top, 2));
        const int e = top ? min(max((int)(top >> 23) - 127, -100), 127) : 14;  // 2^e <= largest < 2^(e+1)
        const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const float2 y = unpack2<false>(qf[nt][k]);
          qf[nt][k] = pack_half2(y.x * up, y.y * up);
        }
        mine = a.scale * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
      }
      // rows 2t and 2t + 1 are the lanes' of g = 2t and 2t + 1
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        f[nt][r] = __shfl_sync(~0u, mine, (2 * t + r) * 4);
        const int jr = (row0 + 8 * nt + 2 * t + r) / G;
        lim[nt][r] = jr < sp.p ? from_key0(row_limit(a, sp, jr)) : 0;
        if (jr < sp.p) least = min(least, lim[nt][r]);
      }
    }
    least = min(least, __shfl_xor_sync(~0u, least, 1));
    least = min(least, __shfl_xor_sync(~0u, least, 2));

    float o[NT][kM][4], m[NT][2], l[NT][2], ref = kLeastRef, inv_ref = 1.f / kLeastRef;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < kM; ++k) o[nt][k][0] = o[nt][k][1] = o[nt][k][2] = o[nt][k][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }
    // One strip's registers: the next keys are loaded once these have met the
    // queries, the next values once these have met the weights, each a whole strip's
    // time ahead.  (Two strips' registers and 12 warps an SM: 4.5 TB/s.)
    Strip<D> x;
    auto place = [&](int s) {  // of strip s, whose id the lanes hold; negative: hidden
      const int32_t b = __shfl_sync(~0u, id0, s & 31);
      return b < 0 ? (int64_t)-1
                   : ((((int64_t)b * a.cache.heads + h) << a.cache.log_b) +
                      ((key0 + (s << 4)) & ((1 << a.cache.log_b) - 1))) * D;
    };
    id0 = checked(id0);
    scales_of(id0, &ks, &vs);
    int64_t at = place(0);
    if (at >= 0) {
      x.load_keys(a.cache.k + at, lane, min(16, most));
      x.load_values(a.cache.v + at, lane, min(16, most));
    }
    id1 = checked(id1);
    scales_of(id1, &next_ks, &next_vs);
    unsigned *const least_vs = shared_least + (threadIdx.x >> 5);
    auto least_of = [&](float v) {
      return __reduce_min_sync(~0u, __float_as_uint(fabsf(v) > kLeastScale ? fabsf(v) : INFINITY));
    };
    {
      const unsigned v = least_of(vs);
      if (lane == 0) *least_vs = v;
    }
    for (int s = 0; s < count; ++s) {
      const float kss = __shfl_sync(~0u, ks, s & 31), vss = __shfl_sync(~0u, vs, s & 31);
      const bool here = at >= 0;
      if (((s + 1) & 31) == 0) {
        id0 = id1, ks = next_ks, vs = next_vs;
        const unsigned v = least_of(vs);
        if (lane == 0) *least_vs = min(*least_vs, v);
        id1 = checked(id2);
        scales_of(id1, &next_ks, &next_vs);
        id2 = look_up(s + 65);
      }
      at = s + 1 < count ? place(s + 1) : -1;
      const int keys = min(16, most - ((s + 1) << 4));
      float c[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t ka[4] = {lo_half2(x.k[0][k]), lo_half2(x.k[1][k]), hi_half2(x.k[0][k]), hi_half2(x.k[1][k])};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816(c[nt], ka, qf[nt][2 * k], qf[nt][2 * k + 1]);
      }
      if (at >= 0) x.load_keys(a.cache.k + at, lane, keys);
      if (!here) {
        if (at >= 0) x.load_values(a.cache.v + at, lane, keys);
        continue;
      }
      bool grow = !(fabsf(vss) <= ref);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          c[nt][r] *= f[nt][r] * kss;
          c[nt][2 + r] *= f[nt][r] * kss;
          if ((s << 4) + 16 > least) {
            if ((s << 4) + g >= lim[nt][r]) c[nt][r] = -INFINITY;
            if ((s << 4) + g + 8 >= lim[nt][r]) c[nt][2 + r] = -INFINITY;
          }
          grow |= fmaxf(c[nt][r], c[nt][2 + r]) > m[nt][r];
        }
      if (__any_sync(~0u, grow)) {
        const float nref = fmaxf(ref, fabsf(vss)), shrink = ref / nref;
        ref = nref;
        inv_ref = 1.f / nref;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float top = fmaxf(c[nt][r], c[nt][2 + r]);
#pragma unroll
            for (int x2 = 4; x2 < 32; x2 <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x2));
            const float nm = fmaxf(m[nt][r], top);
            const float up = m[nt][r] == nm ? 1.f : exp2_fast(m[nt][r] - nm);  // 0 from -inf
            m[nt][r] = nm;
            l[nt][r] *= up;
#pragma unroll
            for (int k = 0; k < kM; ++k) {
              o[nt][k][r] *= up * shrink;
              o[nt][k][2 + r] *= up * shrink;
            }
          }
      }
      uint32_t pb[NT][2];
      const float vr = vss * inv_ref;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float base = m[nt][r] == -INFINITY ? 0.f : m[nt][r] - kWeightExp;
          p[r] = exp2_fast(c[nt][r] - base);
          p[2 + r] = exp2_fast(c[nt][2 + r] - base);
          l[nt][r] += p[r] + p[2 + r];
        }
        pb[nt][0] = transpose8(pack_half2(p[0] * vr, p[1] * vr));
        pb[nt][1] = transpose8(pack_half2(p[2] * vr, p[3] * vr));
      }
#pragma unroll
      for (int q4 = 0; q4 < D / 32; ++q4) {
        // four elements of the lane's two pairs of keys, the pair side by side
        const uint32_t lo0 = __byte_perm(x.v[0][q4], x.v[1][q4], 0x5140), lo1 = __byte_perm(x.v[0][q4], x.v[1][q4], 0x7362);
        const uint32_t hi0 = __byte_perm(x.v[2][q4], x.v[3][q4], 0x5140), hi1 = __byte_perm(x.v[2][q4], x.v[3][q4], 0x7362);
        const uint32_t va[4] = {lo_half2(lo0), hi_half2(lo0), lo_half2(hi0), hi_half2(hi0)};
        const uint32_t vb[4] = {lo_half2(lo1), hi_half2(lo1), lo_half2(hi1), hi_half2(hi1)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma16816(o[nt][2 * q4], va, pb[nt][0], pb[nt][1]);
          mma16816(o[nt][2 * q4 + 1], vb, pb[nt][0], pb[nt][1]);
        }
      }
      if (at >= 0) x.load_values(a.cache.v + at, lane, keys);
    }
    // l over the keys' lanes; lane (g, t) has elements D/8 g .. of rows 2t, 2t + 1
    const bool whole = s0 == 0 && s1 == strips;
    const int64_t slot = (me * 2 + (u == begin ? 0 : 1)) * kRows;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nt][r] += __shfl_xor_sync(~0u, l[nt][r], x);
        const int row = row0 + 8 * nt + 2 * t + r, j = row / G, hh = h * G + row % G;
        if (j < sp.p) {
          if (whole) {
            const float inv = l[nt][r] == 0.f ? 0.f : 1.f / l[nt][r];
            const int64_t at = (sp.first + j) * a.hq + hh;
            uint32_t w[D / 16];
#pragma unroll
            for (int k = 0; k < kM; ++k) w[k] = pack_out<F16>(o[nt][k][r] * inv * ref, o[nt][k][2 + r] * inv * ref);
            uint4 *op = reinterpret_cast<uint4 *>((uint16_t *)a.o + at * D + g * (D / 8));
#pragma unroll
            for (int k = 0; k < kM / 4; ++k) op[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
            if (a.lse && g == 0)
              a.lse[at] = l[nt][r] == 0.f ? -INFINITY : (m[nt][r] - kWeightExp + log2f(l[nt][r])) * 0.6931471805599453f;
          } else {
            const int rr = 8 * nt + 2 * t + r;
            float4 *pp = reinterpret_cast<float4 *>(d.part + (slot + rr) * D + g * (D / 8));
#pragma unroll
            for (int k = 0; k < kM; k += 2)
              pp[k / 2] = make_float4(o[nt][k][r] * ref, o[nt][k][2 + r] * ref, o[nt][k + 1][r] * ref, o[nt][k + 1][2 + r] * ref);
            if (g == 0) {
              d.part_ml[2 * (slot + rr)] = m[nt][r];
              d.part_ml[2 * (slot + rr) + 1] = l[nt][r];
            }
          }
        }
      }
    if (whole && sp.p > 1) {
      __syncwarp();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        for (int row = 0; row < 8; ++row) {
          bool nan = false;
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if (2 * t + r == row) {
#pragma unroll
              for (int k = 0; k < kM; ++k) nan |= isnan(o[nt][k][r]) || isnan(o[nt][k][2 + r]);
            }
          const int rr = row0 + 8 * nt + row, j = rr / G;
          if (__any_sync(~0u, nan) && j < sp.p)
            redo_row<D, F16, true>(a, sp.first, i, sp.first + j, h * G + rr % G, row_limit(a, sp, j), row_limit(a, sp, sp.p - 1));
        }
    }
    // value scales so far apart that a weight, or the sums where ref grew, may have lost too much
    if (__shfl_sync(~0u, lane == 0 && __uint_as_float(*least_vs) < kDecThin * ref, 0)) {
      if (whole) {
        redo_tile<D, F16>(a, i, h, row0, kRows);
      } else {  // the join does it
        __syncwarp();
        if (lane < kRows) d.part_ml[2 * (slot + lane) + 1] *= -1.f;
      }
    }
    u += s1 == strips ? all_units - s0 : s1 - s0;
  }
  if (bad) flag(a.status, kStatusData);
}

// The segments that several warps shared: their parts are added in the line's
// order, eight at a time, by one warp a row (PER_ROW = 1; a CTA takes eight rows
// of a segment), or by PER_ROW warps a row, each its share of the parts, where
// there are few segments and so many parts in each.
template <int D, bool F16, int PER_ROW>
__global__ void __launch_bounds__((PER_ROW == 1 ? kJoinWarps : PER_ROW) * 32) k_attend_join(DecodeArgs d) {
  constexpr int per_row = PER_ROW;
  constexpr int E = D / 32, kBatch = 8;
  __shared__ float sm[PER_ROW][2], so[PER_ROW][D];
  const AttendArgs &a = d.a;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, G = a.hq / a.hkv, rows = 8 * d.nt;
  wait_previous();
  const int64_t units = d.prefix[a.n_req];
  const int64_t W = busy_warps(d.warps, units);
  const int64_t i = blockIdx.x;
  bool ignore = false;
  const Span sp = request_span(a, i, &ignore);
  if (d.prefix[i + 1] == d.prefix[i]) return;
  const int64_t strips = span_strips(a, sp);
  const int tiles = span_tiles(a, sp, rows), groups = per_row == 1 ? rows / kJoinWarps : min(rows, d.a.offsets ? rows : G);
  for (int64_t y = blockIdx.y; y < (int64_t)tiles * a.hkv * groups; y += gridDim.y) {
    const int64_t seg = (int)y / groups;
    const int64_t u0 = d.prefix[i] + seg * segment_units(strips), w0 = warp_of(u0, W, units), w1 = warp_of(u0 + strips - 1, W, units);
    if (w0 == w1) continue;
    const int64_t slot0 = w0 * 2 + (warp_start(w0, W, units) < u0 ? 1 : 0);
    const int h = (int)seg / tiles, r = ((int)y % groups) * (per_row == 1 ? kJoinWarps : 1) + (per_row == 1 ? w : 0);
    const int row = ((int)seg % tiles) * rows + r, j = row / G, hh = h * G + row % G;
    float top = -INFINITY, l = 0.f, o[E];
    bool thin = false;  // of a part whose weights lost bits l is negative
#pragma unroll
    for (int k = 0; k < E; ++k) o[k] = 0.f;
    if (j < sp.p)
      for (int64_t x0 = w0 + (per_row == 1 ? 0 : w); x0 <= w1; x0 += kBatch * per_row) {
        float pm[kBatch], pl[kBatch], po[kBatch][E], nm = top;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int64_t x = x0 + b * per_row;
          pm[b] = -INFINITY, pl[b] = 0.f;
#pragma unroll
          for (int k = 0; k < E; ++k) po[b][k] = 0.f;
          if (x <= w1) {
            const int64_t slot = (x == w0 ? slot0 : x * 2) * rows + r;
            const float2 ml = *reinterpret_cast<const float2 *>(d.part_ml + 2 * slot);
            pm[b] = ml.x, pl[b] = ml.y;
#pragma unroll
            for (int k = 0; k < E; k += 2) {
              const float2 v = *reinterpret_cast<const float2 *>(d.part + slot * D + lane * E + k);
              po[b][k] = v.x, po[b][k + 1] = v.y;
            }
          }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) nm = fmaxf(nm, pm[b]);
        const float base = nm == -INFINITY ? 0.f : nm, up = top == -INFINITY ? 1.f : exp2_fast(top - base);
        l *= up;
#pragma unroll
        for (int k = 0; k < E; ++k) o[k] *= up;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          // a part that saw nothing has zeros, one of a NaN score NaN
          const float f = pm[b] == -INFINITY ? 1.f : exp2_fast(pm[b] - base);
          l += fabsf(pl[b]) * f;
          thin |= pl[b] < 0.f;
#pragma unroll
          for (int k = 0; k < E; ++k) o[k] += po[b][k] * f;
        }
        top = nm;
      }
    if (per_row > 1) {
#pragma unroll
      for (int k = 0; k < E; ++k) so[w][lane * E + k] = o[k];
      if (lane == 0) sm[w % PER_ROW][0] = top, sm[w % PER_ROW][1] = thin ? -l : l;
      __syncthreads();
      if (w == 0) {
        for (int x = 1; x < PER_ROW; ++x) {
          const float nm = fmaxf(top, sm[x][0]), base = nm == -INFINITY ? 0.f : nm;
          const float f0 = top == -INFINITY ? 1.f : exp2_fast(top - base);
          const float f1 = sm[x][0] == -INFINITY ? 1.f : exp2_fast(sm[x][0] - base);
          l = l * f0 + fabsf(sm[x][1]) * f1;
          thin |= sm[x][1] < 0.f;
#pragma unroll
          for (int k = 0; k < E; ++k) o[k] = o[k] * f0 + so[x][lane * E + k] * f1;
          top = nm;
        }
      }
    }
    if (j < sp.p && (per_row == 1 || w == 0)) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t at = (sp.first + j) * a.hq + hh;
      bool nan = false;
#pragma unroll
      for (int k = 0; k < E; k += 2) {
        *reinterpret_cast<uint32_t *>((uint16_t *)a.o + at * D + lane * E + k) = pack_out<F16>(o[k] * inv, o[k + 1] * inv);
        nan |= isnan(o[k]) || isnan(o[k + 1]);
      }
      if (a.lse && lane == 0)
        a.lse[at] = l == 0.f ? -INFINITY : (top - kWeightExp + log2f(l)) * 0.6931471805599453f;
      if (__any_sync(~0u, thin || (nan && sp.p > 1)))
        redo_row<D, F16, true>(a, sp.first, i, sp.first + j, hh, row_limit(a, sp, j), row_limit(a, sp, sp.p - 1), thin);
    }
    if (per_row > 1) __syncthreads();
  }
}

}  // namespace lv
