// The boxes of a paged cache's keys, and the choice of pages by them, for sm_103a.
//
// page_bounds: for each (page, head) that new rows touch, the channel-wise minimum and
// maximum of its keys, rounded outward to whole numbers in [-127, 127] times the page's
// power of two.  Minima, maxima and products with powers of two are exact, so the box does
// not depend on the order of the rows or on how they came (one by one or as a prompt).
//
// select_pages: sum_j max(c_j lo_j, c_j hi_j) = sum_j max(c_j, 0) hi_j + min(c_j, 0) lo_j, two
// dot products of 8-bit numbers a query (dp4a, exact in int32); the powers of two of the
// query and of the page come last, exact too.  So the order of the scores, and the pages that
// are chosen, are those of the definition, whatever the kernel's order of summation.
#include <algorithm>
#include <atomic>

#include <cooperative_groups.h>

#include "tac_pages.cuh"

namespace tac {
namespace cg = cooperative_groups;

constexpr float kFltMax = 3.4028234663852886e38f;
constexpr int kPgThreads = 256, kPgWarps = kPgThreads / 32;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// Minimum and maximum that keep a NaN.
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// Exclusive prefix sums of one int a thread over the CTA, and the total; `s`: kPgWarps + 1 ints.
__device__ __forceinline__ int block_prefix(int v, int* s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s[warp] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPgWarps; ++w) {
    const int c = s[w];
    before += w < warp ? c : 0;
    all += c;
  }
  *total = all;
  return before + x - v;
}

// The rows of sequence s that land on its table: positions [a, b), position a from row r0.
struct Span { int64_t r0, a, b; };
__device__ __forceinline__ Span seq_span(const BoundsParams& p, int s) {
  int64_t r0 = s, r1 = s + 1;
  if (p.first) { r0 = p.first[s]; r1 = p.first[s + 1]; }
  Span v;
  v.a = p.start[s];
  int64_t skip = v.a < 0 ? -v.a : 0;               // rows before position 0 are left out
  if (r0 < 0) skip = max(skip, -r0);               // and rows outside k
  r1 = min(r1, p.rows);
  v.r0 = r0 + skip;
  v.a += skip;
  v.b = min(v.a + max(r1 - v.r0, (int64_t)0), (int64_t)p.pg.width * p.pg.page);
  if (v.b < v.a) v.b = v.a;
  return v;
}
__device__ __forceinline__ int span_pages(const BoundsParams& p, const Span& v) {
  return v.b > v.a ? (int)((v.b - 1) / p.pg.page - v.a / p.pg.page) + 1 : 0;
}

// A unit is one (touched page, head), taken by SPLIT warps of a CTA.
template <int D, typename T, int SPLIT>
__global__ void __launch_bounds__(kPgThreads) page_bounds_kernel(const __grid_constant__ BoundsParams p) {
  constexpr int EPL = 16 / (int)sizeof(T), LPR = D / EPL, RPW = 32 / LPR;   // channels a lane, lanes a row, rows a load
  constexpr int UPC = kPgWarps / SPLIT;                                     // units a CTA takes at a time
  __shared__ int pref[kPgThreads + 1], scan[kPgWarps + 1];
  __shared__ float part[SPLIT > 1 ? kPgWarps : 1][2][D];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int seqs = p.pg.seqs, heads = p.pg.heads, page = p.pg.page;
  const int chunk = (seqs + kPgThreads - 1) / kPgThreads;
  int items = seqs;                                // without `first`, item s is sequence s
  if (p.first) {
    int mine = 0;
    for (int s = tid * chunk; s < min(seqs, (tid + 1) * chunk); ++s) mine += span_pages(p, seq_span(p, s));
    pref[tid] = block_prefix(mine, scan, &items);
    if (tid == 0) pref[kPgThreads] = items;
    __syncthreads();
  }
  const int64_t units = (int64_t)items * heads;
  const int g = lane / LPR, ch = (lane % LPR) * EPL, sub = warp % SPLIT;
  for (int64_t u0 = (int64_t)blockIdx.x * UPC; u0 < units; u0 += (int64_t)gridDim.x * UPC) {
    const int64_t u = u0 + warp / SPLIT;
    int item = (int)(u / heads), h = (int)(u % heads), s = item, j = 0;
    Span v{0, 0, 0};
    bool live = u < units;
    if (live && p.first) {
      int lo = 0, hi = kPgThreads - 1;             // the thread whose sequences hold the item
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pref[mid] <= item) lo = mid; else hi = mid - 1;
      }
      item -= pref[lo];
      for (s = lo * chunk; ; ++s) {
        v = seq_span(p, s);
        const int c = span_pages(p, v);
        if (item < c) break;
        item -= c;
      }
      j = item;
    } else if (live) {
      v = seq_span(p, s);
      live = v.b > v.a;
    }
    int64_t phys = -1, pos0 = 0, row0 = 0;
    int rows = 0;
    if (live) {
      const int64_t col = v.a / page + j;
      pos0 = max(v.a, col * page);
      rows = (int)(min(v.b, (col + 1) * page) - pos0);
      row0 = v.r0 + (pos0 - v.a);
      phys = p.pg.table[(int64_t)s * p.pg.table_stride + col];
      live = phys >= 0 && phys < p.pg.pages;
    }
    const int64_t box = phys * heads + h;
    const bool fresh = pos0 % page == 0;
    float lo[EPL], hi[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
    float s_old = 0.f;
    int8_t old[2][EPL] = {};
    if (live) {
      if (!fresh) {                                // the box so far, asked for before the rows
        s_old = p.scales[box];
        const int8_t* c = p.codes + box * 2 * D + ch;
        if constexpr (EPL == 8) {
          *reinterpret_cast<uint2*>(old[0]) = *reinterpret_cast<const uint2*>(c);
          *reinterpret_cast<uint2*>(old[1]) = *reinterpret_cast<const uint2*>(c + D);
        } else {
          *reinterpret_cast<uint32_t*>(old[0]) = *reinterpret_cast<const uint32_t*>(c);
          *reinterpret_cast<uint32_t*>(old[1]) = *reinterpret_cast<const uint32_t*>(c + D);
        }
      }
      const T* base = reinterpret_cast<const T*>(p.k) + row0 * p.row_stride + (int64_t)h * p.head_stride + ch;
      // rows beyond the last repeat it: a minimum does not change by that
      for (int r = sub * RPW; r < rows; r += 8 * SPLIT * RPW) {
        uint4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = min(r + i * SPLIT * RPW + g, rows - 1);
          x[i] = __ldcs(reinterpret_cast<const uint4*>(base + row * p.row_stride));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            float f;
            if constexpr (EPL == 4) f = __uint_as_float(w[e]);
            else f = e & 1 ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
            lo[e] = min_nan(lo[e], f);
            hi[e] = max_nan(hi[e], f);
          }
        }
      }
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          lo[e] = min_nan(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], o));
          hi[e] = max_nan(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], o));
        }
    }
    if constexpr (SPLIT > 1) {
      if (g == 0) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) { part[warp][0][ch + e] = lo[e]; part[warp][1][ch + e] = hi[e]; }
      }
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int w = 1; w < SPLIT; ++w)
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            lo[e] = min_nan(lo[e], part[warp + w][0][ch + e]);
            hi[e] = max_nan(hi[e], part[warp + w][1][ch + e]);
          }
      }
      __syncthreads();
    }
    if (!live || sub != 0) continue;
    float a = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) a = max_nan(a, max_nan(fabsf(lo[e]), fabsf(hi[e])));
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    if (g != 0) continue;
    const bool bad = !(a < INFINITY) || !(s_old < INFINITY);
    int8_t c[2][EPL];
    float scale = INFINITY;
    if (bad) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) { c[0][e] = -127; c[1][e] = 127; }
    } else {
      const int e_old = s_old > 0.f ? (int)(__float_as_uint(s_old) >> 23) - 127 : -126;
      const int ex = max(box_exp(a), e_old), shift = min(ex - e_old, 31);
      const float inv = pow2i(-ex);                // ex <= 122
      scale = pow2i(ex);
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        // outward also where the product underflows
        int l = __float2int_rd(lo[e] * inv), m = __float2int_ru(hi[e] * inv);
        l = lo[e] < 0.f ? min(l, -1) : l;
        m = hi[e] > 0.f ? max(m, 1) : m;
        if (!fresh) {
          l = min(l, (int)old[0][e] >> shift);
          m = max(m, -((-(int)old[1][e]) >> shift));
        }
        c[0][e] = (int8_t)l;
        c[1][e] = (int8_t)m;
      }
    }
    int8_t* dst = p.codes + box * 2 * D + ch;
    if constexpr (EPL == 8) {
      *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(c[0]);
      *reinterpret_cast<uint2*>(dst + D) = *reinterpret_cast<const uint2*>(c[1]);
    } else {
      *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(c[0]);
      *reinterpret_cast<uint32_t*>(dst + D) = *reinterpret_cast<const uint32_t*>(c[1]);
    }
    if (lane == 0) p.scales[box] = scale;
  }
}

template <int D, typename T>
static cudaError_t launch_bounds_t(const BoundsParams& p, int sms, cudaStream_t st) {
  // at most this many (page, head)s are touched
  const int64_t items = p.first ? std::min(p.rows, p.rows / p.pg.page + 2 * (int64_t)p.pg.seqs) : p.pg.seqs;
  const int64_t units = items * p.pg.heads;
  if (units < 1) return cudaSuccess;
  auto grid = [&](int upc) { return (unsigned)std::min<int64_t>((units + upc - 1) / upc, (int64_t)sms * 6); };
  page_bounds_kernel<D, T, 1><<<grid(kPgWarps), kPgThreads, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_page_bounds(int d, int dtype, const BoundsParams& p, int sms, cudaStream_t st) {
  if (dtype == TAC_BF16) return d == 128 ? launch_bounds_t<128, __nv_bfloat16>(p, sms, st) : launch_bounds_t<64, __nv_bfloat16>(p, sms, st);
  return d == 128 ? launch_bounds_t<128, float>(p, sms, st) : launch_bounds_t<64, float>(p, sms, st);
}

// ---------------------------------------------------------------------------
// Choice of pages
// ---------------------------------------------------------------------------
// A cluster of CTAs takes one (sequence, head): each scores a contiguous part of the pages
// into shared memory, the largest `budget` are found by radix selection (8 bits a pass,
// the CTAs' histograms added through distributed shared memory), and every CTA writes its
// part of them in order.  A score becomes a whole number of the same order.
__device__ __forceinline__ uint32_t order_key(float s) {
  const uint32_t u = __float_as_uint(s + 0.f);     // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int D, typename T, int NQ>
__global__ void __launch_bounds__(kPgThreads) select_kernel(const __grid_constant__ SelectParams p) {
  constexpr int LP = D / 16, PW = 32 / LP;         // lanes a page (16 channels each), pages a warp takes at a time
  constexpr int R = NQ > LP ? NQ / LP : 1;         // queries a lane holds after the reduction
  extern __shared__ uint32_t keys[];               // of this CTA's pages
  __shared__ __align__(16) int qpos[NQ][D / 4], qneg[NQ][D / 4];
  __shared__ float qscale[NQ];
  __shared__ uint32_t hist[4][256];                // one for each pass: a CTA may lag behind a pass
  __shared__ uint32_t range[2];                    // smallest and largest key here
  __shared__ int counts[2];                        // pages above the threshold, at it
  __shared__ int wsum[kPgWarps][2], scan[kPgWarps + 1], found[2];
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int seg = blockIdx.x / cs, s = seg / p.pg.heads, h = seg % p.pg.heads;
  const int64_t len = min((int64_t)max(p.pg.lengths[s], 0), (int64_t)p.pg.width * p.pg.page);
  const int n = (int)((len + p.pg.page - 1) / p.pg.page);
  const int chunk = (n + cs - 1) / cs, first = min(rank * chunk, n), cnt = min(n - first, chunk);
  int32_t* const out = p.selected + (int64_t)seg * p.budget;
  const int take = min(n, p.budget);
  if (rank == 0) {
    if (tid == 0) p.counts[seg] = take;
    for (int i = take + tid; i < p.budget; i += kPgThreads) out[i] = -1;
  }
  if (n <= p.budget) {                             // no choice (the whole cluster leaves)
    for (int i = tid; i < cnt; i += kPgThreads) out[first + i] = first + i;
    return;
  }

  // ---- the queries in 8 bits, positive and negative parts apart ----
  if (warp < NQ) {
    constexpr int E = D / 32;
    float x[E];
    float a = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = 0.f;
      if (warp < p.group)
        x[e] = to_f<T>(reinterpret_cast<const T*>(p.q)[(int64_t)s * p.seq_stride + ((int64_t)h * p.group + warp) * p.row_stride + lane * E + e]);
      if (!(fabsf(x[e]) < INFINITY)) x[e] = 0.f;
      a = fmaxf(a, fabsf(x[e]));
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
    const int ex = box_exp(a);
    const float inv = pow2i(-ex);
    int pos = 0, neg = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = __float2int_rn(x[e] * inv);
      pos |= (max(c, 0) & 0xFF) << (8 * e);
      neg |= (min(c, 0) & 0xFF) << (8 * e);
    }
    if constexpr (E == 4) {
      qpos[warp][lane] = pos;
      qneg[warp][lane] = neg;
    } else {
      reinterpret_cast<uint16_t*>(qpos[warp])[lane] = (uint16_t)pos;
      reinterpret_cast<uint16_t*>(qneg[warp])[lane] = (uint16_t)neg;
    }
    if (lane == 0) qscale[warp] = pow2i(ex);
  }
  for (int i = tid; i < 4 * 256; i += kPgThreads) hist[0][i] = 0u;
  if (tid == 0) { range[0] = 0xFFFFFFFFu; range[1] = 0u; }
  __syncthreads();

  // ---- scores ----
  {
    const int sub = lane % LP, g = lane / LP;
    int qp[NQ][4], qn[NQ][4];
#pragma unroll
    for (int a = 0; a < NQ; ++a) {
      const int4 x = *reinterpret_cast<const int4*>(&qpos[a][4 * sub]), y = *reinterpret_cast<const int4*>(&qneg[a][4 * sub]);
      qp[a][0] = x.x; qp[a][1] = x.y; qp[a][2] = x.z; qp[a][3] = x.w;
      qn[a][0] = y.x; qn[a][1] = y.y; qn[a][2] = y.z; qn[a][3] = y.w;
    }
    // after the reduction over a page's lanes this one holds R queries from q0 on
    int q0 = 0;
    {
      int c = NQ;
#pragma unroll
      for (int o = LP / 2; o >= 1; o >>= 1)
        if (c > 1) { c /= 2; q0 += sub & o ? c : 0; }
    }
    float qs[R];
#pragma unroll
    for (int i = 0; i < R; ++i) qs[i] = qscale[q0 + i];
    uint32_t kmin = 0xFFFFFFFFu, kmax = 0u;
    const int32_t* row = p.pg.table + (int64_t)s * p.pg.table_stride + first;
    for (int base = warp * 32; base < cnt; base += kPgThreads) {
      int64_t at = -1;                             // box of page base + lane
      float sp = 0.f;
      if (base + lane < cnt) {
        const int ph = row[base + lane];
        if (ph >= 0 && ph < p.pg.pages) {
          at = (int64_t)ph * p.pg.heads + h;
          sp = p.scales[at];
        }
      }
#pragma unroll 4
      for (int it = 0; it < LP; ++it) {
        const int64_t box = __shfl_sync(0xffffffffu, at, it * PW + g);
        const float f = __shfl_sync(0xffffffffu, sp, it * PW + g);
        int4 lo = make_int4(0, 0, 0, 0), hi = lo;
        if (box >= 0) {
          const int4* b = reinterpret_cast<const int4*>(p.codes + box * 2 * D) + sub;
          lo = b[0];
          hi = b[D / 16];
        }
        int v[NQ];
#pragma unroll
        for (int a = 0; a < NQ; ++a) {
          int x = __dp4a(qp[a][0], hi.x, 0);
          x = __dp4a(qn[a][0], lo.x, x);
          x = __dp4a(qp[a][1], hi.y, x);
          x = __dp4a(qn[a][1], lo.y, x);
          x = __dp4a(qp[a][2], hi.z, x);
          x = __dp4a(qn[a][2], lo.z, x);
          x = __dp4a(qp[a][3], hi.w, x);
          v[a] = __dp4a(qn[a][3], lo.w, x);
        }
        int c = NQ;
#pragma unroll
        for (int o = LP / 2; o >= 1; o >>= 1) {
          if (c > 1) {
            c /= 2;
            const bool up = sub & o;
#pragma unroll
            for (int i = 0; i < c; ++i) {
              const int give = up ? v[i] : v[i + c], keep = up ? v[i + c] : v[i];
              v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
          }
        }
        float best = -INFINITY;
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (q0 + i < p.group) best = fmaxf(best, fmaxf(fminf(((float)v[i] * qs[i]) * f, kFltMax), -kFltMax));
#pragma unroll
        for (int o = LP / 2; o >= 1; o >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (box < 0) best = -INFINITY;
        else if (f == INFINITY) best = kFltMax;
        const int i = base + it * PW + g, page = first + i;
        if (sub == 0 && i < cnt) {
          uint32_t key = order_key(best);
          if (page < p.keep_first || page >= n - p.keep_last) {
            key = 0xFFFFFFFFu;                     // above every score: always taken
          } else {
            kmin = min(kmin, key);
            kmax = max(kmax, key);
          }
          keys[i] = key;
        }
      }
    }
    kmin = __reduce_min_sync(0xffffffffu, kmin);
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    if (lane == 0) {
      atomicMin(&range[0], kmin);
      atomicMax(&range[1], kmax);
    }
  }
  cluster.sync();

  // ---- the threshold: the need-th largest of the keys that are not always taken ----
  int need = p.budget - p.keep_first - p.keep_last;
  uint32_t thr = 0xFFFFFFFFu;
  if (need > 0) {
    uint32_t kmin = 0xFFFFFFFFu, kmax = 0u;
    for (int r = 0; r < cs; ++r) {
      const uint32_t* x = cluster.map_shared_rank(range, r);
      kmin = min(kmin, x[0]);
      kmax = max(kmax, x[1]);
    }
    // the bits above the first that differs are common to all
    int low = kmin == kmax ? 0 : 32 - __clz(kmin ^ kmax);
    uint32_t fixed = low == 32 ? 0u : kmax >> low << low;
    for (int pass = 0; low > 0; ++pass) {
      const int bits = min(low, 8), at = low - bits;
      const uint32_t above = low == 32 ? 0u : 0xFFFFFFFFu << low;
      for (int i = tid; i < cnt; i += kPgThreads) {
        const uint32_t k = keys[i];
        if (k != 0xFFFFFFFFu && (k & above) == fixed) atomicAdd(&hist[pass][(k >> at) & 255u & ((1u << bits) - 1u)], 1u);
      }
      cluster.sync();
      // digit 255 - tid: how many keys have a larger one
      int c = 0;
      for (int r = 0; r < cs; ++r) c += (int)cluster.map_shared_rank(hist[pass], r)[255 - tid];
      int total;
      const int before = block_prefix(c, scan, &total);
      if (before < need && need <= before + c) { found[0] = 255 - tid; found[1] = need - before; }
      __syncthreads();
      fixed |= (uint32_t)found[0] << at;
      need = found[1];
      low = at;
    }
    thr = fixed;
  }

  // ---- the pages above the threshold and the first `need` at it, in order ----
  const int per = (cnt + kPgThreads - 1) / kPgThreads * 32, lo = min(warp * per, cnt), hi = min(lo + per, cnt);
  int gt = 0, eq = 0;
  for (int i = lo + lane; i < hi; i += 32) {
    const uint32_t k = keys[i];
    const bool e = k == thr && thr != 0xFFFFFFFFu;
    gt += !e && k >= thr;
    eq += e;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) { wsum[warp][0] = gt; wsum[warp][1] = eq; }
  __syncthreads();
  if (tid == 0) {
    int a = 0, b = 0;
    for (int w = 0; w < kPgWarps; ++w) { a += wsum[w][0]; b += wsum[w][1]; }
    counts[0] = a;
    counts[1] = b;
  }
  cluster.sync();
  gt = eq = 0;                                     // before this warp's pages
  for (int r = 0; r < rank; ++r) {
    const int* x = cluster.map_shared_rank(counts, r);
    gt += x[0];
    eq += x[1];
  }
  for (int w = 0; w < warp; ++w) { gt += wsum[w][0]; eq += wsum[w][1]; }
  for (int i0 = lo; i0 < hi; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t k = i < hi ? keys[i] : 0u;
    const bool e = i < hi && k == thr && thr != 0xFFFFFFFFu, a = i < hi && !e && k >= thr;
    const uint32_t am = __ballot_sync(0xffffffffu, a), em = __ballot_sync(0xffffffffu, e), below = (1u << lane) - 1u;
    const int mg = gt + __popc(am & below), me = eq + __popc(em & below);
    if (a || (e && me < need)) out[mg + min(me, need)] = first + i;
    gt += __popc(am);
    eq += __popc(em);
  }
  cluster.sync();                                  // the others may still read this CTA's counts
}

template <int D, typename T, int NQ>
static cudaError_t launch_select_t(const SelectParams& p, int sms, cudaStream_t st) {
  auto kp = select_kernel<D, T, NQ>;
  static std::atomic<int> ready[64];               // per device: the shared-memory limit is set
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!ready[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(kp, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != cudaSuccess) return e;
    ready[dev].store(1, std::memory_order_release);
  }
  const int64_t segs = (int64_t)p.pg.seqs * p.pg.heads;
  if (segs < 1) return cudaSuccess;
  int cs = 1;
  while (cs < 8 && (segs * cs < 2 * sms || p.pg.width > cs * 32768) && p.pg.width > cs * 64) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(segs * cs));
  cfg.blockDim = dim3(kPgThreads);
  cfg.dynamicSmemBytes = (size_t)(4 * std::max(1, (p.pg.width + cs - 1) / cs));
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)cs;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kp, p);
}

cudaError_t launch_select_pages(int d, int dtype, const SelectParams& p, int sms, cudaStream_t st) {
#define TAC_SEL(DD, T) (p.group <= 4 ? launch_select_t<DD, T, 4>(p, sms, st) : launch_select_t<DD, T, 8>(p, sms, st))
  if (dtype == TAC_BF16) return d == 128 ? TAC_SEL(128, __nv_bfloat16) : TAC_SEL(64, __nv_bfloat16);
  return d == 128 ? TAC_SEL(128, float) : TAC_SEL(64, float);
#undef TAC_SEL
}

}  // namespace tac
