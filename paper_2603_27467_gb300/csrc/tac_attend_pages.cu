// Attention of new tokens over a paged record cache, for sm_103a.
//
// For a decoded key k^ = D H y^ (Sec. 3.1), q . k^ = (H D q) . y^ with y^_2i + i y^_2i+1 =
// r^_i exp(2 pi i k_i / n), and sum_t p_t v^_t = D H (sum_t p_t y^V_t): the queries are
// rotated once and the outputs back once, and a record is only looked up.
//
// Work: a tile is 16 tokens of one page.  The tiles of all (sequence, head)s, in order, are
// dealt evenly to the warps of a persistent grid; every CTA finds its place from the
// lengths on the device.  A warp walks its tiles two at a time (a batch) with the running
// maximum and sum of the softmax.  A (sequence, head) that lies within one warp is finished
// there; the parts of one that several warps of a CTA share are joined in shared memory in
// the order of the warps; the parts of several CTAs go to the workspace and a second
// kernel joins them in the order of the CTAs.
#include <algorithm>
#include <atomic>

#include "tac_pages.cuh"

namespace tac {

template <int V>
struct IC { static constexpr int value = V; };

constexpr float kPgLog2e = 1.4426950408889634f;
constexpr int kBatch = 2 * kTile;
constexpr int kMaxWarps = 16;
constexpr int kCopies = 16;                       // of each bin-centre table: a half-warp's lookups fall in distinct banks
constexpr int kTabShift = 7;                      // log2 of an entry's bytes, all copies

// Bin centres (cos, sin)(2 pi k / n) of every supported n, rounded from fp64 by the host compiler.
namespace cx {
struct PgCentreTable { float2 v[kTabEntries]; };
constexpr PgCentreTable make_pg_centre_table() {
  PgCentreTable t{};
  for (int idx = 0; idx < kTabEntries; ++idx) {
    const int n = tab_n_of(idx), k = idx - tab_offset_n(n);
    const CS cs = cos_sin_q8(8 * k, n);
    t.v[idx] = float2{(float)cs.c, (float)cs.s};
  }
  return t;
}
}  // namespace cx
static __device__ const cx::PgCentreTable g_pg_centre = cx::make_pg_centre_table();

// ---------------------------------------------------------------------------
// Small device helpers
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pg_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void pg_bar_init(uint32_t bar) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pg_bar_expect(uint32_t bar, int bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void pg_copy(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// Gives up after 2^16 tries (each suspends the warp for a while).
__device__ __forceinline__ bool pg_bar_wait(uint32_t bar, uint32_t parity) {
  for (int i = 0; i < (1 << 16); ++i) {
    uint32_t done;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ void pg_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint32_t pg_rotr(uint32_t x, int s) { return __funnelshift_r(x, x, s); }
__device__ __forceinline__ float2 ffma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// Unnormalized Walsh-Hadamard transform of a row of D floats over a warp: lane l holds
// elements E l .. E l + E - 1, E = D / 32.
template <int D>
__device__ __forceinline__ void pg_fwht(float (&y)[D / 32], int lane) {
  constexpr int E = D / 32;
#pragma unroll
  for (int h = 1; h < E; h <<= 1)
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (!(k & h)) {
        const float a = y[k], b = y[k + h];
        y[k] = a + b;
        y[k + h] = a - b;
      }
#pragma unroll
  for (int h = 1; h < 32; h <<= 1) {
    const float sg = lane & h ? -1.f : 1.f;
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] = __fmaf_rn(sg, y[k], __shfl_xor_sync(0xffffffffu, y[k], h));
  }
}

// Row a of a (sequence, head)'s queries, rotated and times scale * log2(e): elements E lane + k.
template <int D>
__device__ __forceinline__ void pg_load_query(const AttPagesParams& p, bool bf, int seq, int head, int a, int lane,
                                              float (&y)[D / 32]) {
  constexpr int E = D / 32;
  const int64_t at = (int64_t)seq * p.q_seq + ((int64_t)head * p.group + a) * p.q_row + E * lane;
  if (bf) {
    const uint32_t* x = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(p.q) + at);
#pragma unroll
    for (int k = 0; k < E / 2; ++k) {
      const uint32_t w = x[k];
      y[2 * k] = bf16lo(w);
      y[2 * k + 1] = bf16hi(w);
    }
  } else {
    const float2* x = reinterpret_cast<const float2*>(reinterpret_cast<const float*>(p.q) + at);
#pragma unroll
    for (int k = 0; k < E / 2; ++k) {
      const float2 w = x[k];
      y[2 * k] = w.x;
      y[2 * k + 1] = w.y;
    }
  }
  const uint32_t sg = p.k.signs[(E * lane) >> 5] >> ((E * lane) & 31);
#pragma unroll
  for (int k = 0; k < E; ++k)
    if ((sg >> k) & 1u) y[k] = -y[k];
  pg_fwht<D>(y, lane);
  const float qs = p.scale * kPgLog2e * rsqrtf((float)D);
#pragma unroll
  for (int k = 0; k < E; ++k) y[k] *= qs;
}

// Row a of the output from the accumulator in the rotated domain (elements E lane + k) and its sum.
template <int D>
__device__ __forceinline__ void pg_store_out(const AttPagesParams& p, bool bf, int seq, int head, int a, int lane,
                                             float (&y)[D / 32], float l) {
  constexpr int E = D / 32;
  pg_fwht<D>(y, lane);
  const float f = l == 0.f ? 0.f : rsqrtf((float)D) / l;      // no token: zeros
  const uint32_t sg = p.v.signs[(E * lane) >> 5] >> ((E * lane) & 31);
  const int64_t at = (int64_t)seq * p.o_seq + ((int64_t)head * p.group + a) * p.o_row + E * lane;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    y[k] = l == 0.f ? 0.f : y[k] * f;
    if ((sg >> k) & 1u) y[k] = -y[k];
  }
  if (bf) {
    uint32_t* o = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at);
#pragma unroll
    for (int k = 0; k < E / 2; ++k) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * k], y[2 * k + 1]);
      o[k] = *reinterpret_cast<const uint32_t*>(&v);
    }
  } else {
    float2* o = reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + at);
#pragma unroll
    for (int k = 0; k < E / 2; ++k) o[k] = make_float2(y[2 * k], y[2 * k + 1]);
  }
}

// ---------------------------------------------------------------------------
// Plan: tiles of each item (a sequence, or a (sequence, head) with a selection)
// ---------------------------------------------------------------------------
__device__ __forceinline__ int pg_len(const AttPagesParams& p, int seq) {
  return (int)min((int64_t)max(p.pg.lengths[seq], 0), (int64_t)p.pg.width * p.pg.page);
}
// Tiles of one (sequence, head) of item i.
__device__ __forceinline__ int pg_tiles(const AttPagesParams& p, int i) {
  if (!p.selected) return (pg_len(p, i) + kTile - 1) / kTile;
  return min(max(p.counts[i], 0), p.budget) * (p.pg.page / kTile);
}

// Walks a warp's tiles in order.
struct Cursor {
  int64_t left;          // tiles still to come
  int item, head;        // the (sequence, head) of the next tile
  int seq;
  int i, nt;             // next tile within it, its tiles
  int len;               // the sequence's tokens
  int ent, sub;          // page entry and tile within the page of tile i
  int base;              // first page entry held in the lanes' registers (a multiple of 32)
  int phys, logical;     // lane l: page and table column of entry base + l (page -1: none)
};

__device__ __forceinline__ void cursor_pages(const AttPagesParams& p, Cursor& c, int lane) {
  c.base = c.ent & ~31;
  const int e = c.base + lane;
  int col = -1;
  if (p.selected) {
    const int have = c.nt / (p.pg.page / kTile);
    if (e < have) col = p.selected[((int64_t)c.seq * p.pg.heads + c.head) * p.budget + e];
  } else if (e < p.pg.width) {
    col = e;
  }
  int ph = -1;
  if (col >= 0 && col < p.pg.width && (int64_t)col * p.pg.page < c.len) ph = p.pg.table[(int64_t)c.seq * p.pg.table_stride + col];
  c.phys = ph >= 0 && ph < p.pg.pages ? ph : -1;
  c.logical = col;
}

// The cursor at tile i of (item, head).
__device__ __forceinline__ void cursor_open(const AttPagesParams& p, Cursor& c, int lane) {
  c.seq = p.selected ? c.item / p.pg.heads : c.item;
  if (p.selected) c.head = c.item % p.pg.heads;
  c.len = pg_len(p, c.seq);
  const int per = p.pg.page / kTile;
  c.ent = c.i / per;
  c.sub = c.i - c.ent * per;
  cursor_pages(p, c, lane);
}

// A batch: two tiles (the second may be missing) of one (sequence, head).
struct Batch {
  int64_t slot0, slot1;  // first record slots
  int valid0, valid1;    // tokens of each tile that count (0: nothing is copied)
  int seq, head;
  bool begins, first;    // the warp's first batch of this (sequence, head); which starts with tile 0
  bool ends, last;       // the warp's last batch of it; which holds its last tile
};

__device__ __forceinline__ void cursor_tile(const AttPagesParams& p, Cursor& c, int lane, int64_t& slot, int& valid) {
  if (c.ent >= c.base + 32) cursor_pages(p, c, lane);
  const int ph = __shfl_sync(0xffffffffu, c.phys, c.ent - c.base), col = __shfl_sync(0xffffffffu, c.logical, c.ent - c.base);
  const int64_t pos = (int64_t)col * p.pg.page + c.sub * kTile;
  valid = ph < 0 ? 0 : (int)min(max(c.len - pos, (int64_t)0), (int64_t)kTile);
  slot = ((int64_t)ph * p.pg.heads + c.head) * p.pg.page + c.sub * kTile;
  ++c.i;
  if (++c.sub * kTile == p.pg.page) { c.sub = 0; ++c.ent; }
}

// The next batch; false when the warp's tiles are done.
__device__ __forceinline__ bool cursor_next(const AttPagesParams& p, Cursor& c, int lane, Batch& b) {
  if (c.left <= 0) return false;
  bool opened = false;
  while (c.i >= c.nt) {                            // to the next (sequence, head) that has tiles
    if (p.selected || ++c.head == p.pg.heads) {
      c.head = 0;
      ++c.item;
      c.nt = pg_tiles(p, c.item);
    }
    c.i = 0;
    opened = true;
  }
  if (opened) cursor_open(p, c, lane);
  b.seq = c.seq;
  b.head = c.head;
  b.first = c.i == 0;
  cursor_tile(p, c, lane, b.slot0, b.valid0);
  --c.left;
  b.slot1 = 0;
  b.valid1 = 0;
  if (c.i < c.nt && c.left > 0) {
    cursor_tile(p, c, lane, b.slot1, b.valid1);
    --c.left;
  }
  b.last = c.i == c.nt;
  b.ends = b.last || c.left == 0;
  return true;
}

// Shared memory of the fp32 kernel.
template <int D, int QT>
struct PgF {
  static constexpr int P = D / 2, NQ = 4 * QT, E = D / 32;
  static constexpr int KP = P / 4;                 // K: positions of a token a lane takes (4 lanes a token)
  static constexpr int VL = P / 4, VT = 32 / VL;   // V: lanes a token (4 positions each), tokens at a time
  static constexpr int QRUN = KP * 8 + 16;         // a lane's run of a query: padded, the four runs fall in distinct banks
  static constexpr int REC = NQ * pg_rec_floats(D) * 4;
  // per warp: rotated queries (and the record of a part that ends here) | record of a part
  // that began in an earlier warp | constants of the batch's tokens | softmax weights | staging
  static constexpr int W_Q = 0;
  static constexpr int W_REC = W_Q + NQ * 4 * QRUN;
  static constexpr int W_KC = W_REC + (REC + 15) / 16 * 16;
  static constexpr int W_VC = W_KC + kBatch * 8;
  static constexpr int W_P = W_VC + kBatch * 8;
  static constexpr int W_STG = W_P + kBatch * NQ * 4;
  static_assert(NQ * 4 * QRUN >= REC && W_KC % 16 == 0, "layout");
};
__host__ __device__ inline int pg_stage_bytes(const Book& b) { return kBatch * (b.ab + b.nb + b.hb) + 16; }

// CTA-wide bookkeeping, in front of the dynamic shared memory.
struct PgShared {
  int64_t bars[2 * kMaxWarps];                     // mbarriers: K, V of each warp
  int pref[kMaxWarps * 32 + 1];                    // first tile of each thread's items
  int scan[kMaxWarps];
  // parts: what each warp left.  0: one that began in an earlier warp, 1: one that begins
  // here and goes on.  -1: none; seq * heads + head otherwise.
  int part[kMaxWarps][2];
  int ends0[kMaxWarps];                            // part 0 ends in this warp
  int empty[kMaxWarps];                            // no tiles
};

// Joins of a CTA's parts: every (part that begins a chain, query) is one warp's task.
// rec(w, which): the record of a warp's part.
template <int D, typename Rec>
__device__ __forceinline__ void pg_join(const AttPagesParams& p, const PgShared& sh, bool bf, int nw, int warp, int lane,
                                        Rec rec) {
  constexpr int E = D / 32;
  int task = 0;
  for (int lead = 0; lead < 2 * nw; ++lead) {
    const int w0 = lead >> 1, which = lead & 1, id = sh.part[w0][which];
    if (id < 0) continue;
    if (which == 0) {                              // only the CTA's first part can have begun before it
      bool before = false;
      for (int w = 0; w < w0; ++w) before |= !sh.empty[w];
      if (before) continue;
    }
    int w1 = w0;                                   // the last warp of the chain
    bool ended = which == 0 && sh.ends0[w0];
    for (int w = w0 + 1; w < nw && !ended; ++w) {
      if (sh.empty[w]) continue;
      w1 = w;
      ended = sh.ends0[w];
    }
    const bool whole = which == 1 && ended;
    for (int a = 0; a < p.group; ++a, ++task) {
      if (task % nw != warp) continue;
      float M = -INFINITY;
      for (int w = w0; w <= w1; ++w)
        if (!sh.empty[w]) M = fmaxf(M, rec(w, w == w0 ? which : 0)[a * pg_rec_floats(D)]);
      float l = 0.f, y[E];
#pragma unroll
      for (int k = 0; k < E; ++k) y[k] = 0.f;
      for (int w = w0; w <= w1; ++w) {
        if (sh.empty[w]) continue;
        const float* r = rec(w, w == w0 ? which : 0) + a * pg_rec_floats(D);
        const float f = r[0] == -INFINITY ? 0.f : ex2_approx(r[0] - M);
        l = __fmaf_rn(r[1], f, l);
#pragma unroll
        for (int k = 0; k < E; ++k) y[k] = __fmaf_rn(r[2 + E * lane + k], f, y[k]);
      }
      if (whole) {
        pg_store_out<D>(p, bf, id / p.pg.heads, id % p.pg.heads, a, lane, y, l);
      } else {
        float* out = p.part + (((int64_t)blockIdx.x * 2 + which) * p.group + a) * pg_rec_floats(D);
        if (lane == 0) *reinterpret_cast<float2*>(out) = make_float2(M, l);
#pragma unroll
        for (int k = 0; k < E; k += 2) *reinterpret_cast<float2*>(out + 2 + E * lane + k) = make_float2(y[k], y[k + 1]);
      }
    }
  }
}

// The plan of a CTA: total tiles, and the warp's cursor.  All threads call it.
__device__ __forceinline__ int64_t pg_plan(const AttPagesParams& p, PgShared& sh, int nw, Cursor& c) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = nw * 32;
  const int items = p.items, mult = p.selected ? 1 : p.pg.heads;
  const int chunk = (items + nt - 1) / nt;
  int mine = 0;
  for (int i = tid * chunk; i < min(items, (tid + 1) * chunk); ++i) mine += pg_tiles(p, i) * mult;
  int x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh.scan[warp] = x;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += sh.scan[w];
  sh.pref[tid] = before + x - mine;
  if (tid == nt - 1) sh.pref[nt] = before + x;
  __syncthreads();
  const int64_t total = sh.pref[nt];
  // at least two tiles a warp
  const int64_t nc = min((int64_t)p.ctas, (total + 2 * nw - 1) / (2 * nw));
  if (blockIdx.x == 0) {                           // for the second kernel
    int at = sh.pref[tid];
    for (int i = tid * chunk; i < min(items, (tid + 1) * chunk); ++i) {
      p.plan[i] = at;
      at += pg_tiles(p, i) * mult;
    }
    if (tid == 0) {
      p.plan[items] = (int)total;
      p.plan[items + 1] = (int)nc;
    }
  }
  c.left = 0;
  if ((int64_t)blockIdx.x >= nc) return 0;
  const int64_t W = nc * nw, me = (int64_t)blockIdx.x * nw + warp;
  int64_t t0 = total * me / W;
  c.left = total * (me + 1) / W - t0;
  if (c.left <= 0) return total;
  int lo = 0, hi = nt - 1;                         // the thread whose items hold tile t0
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sh.pref[mid] <= t0) lo = mid; else hi = mid - 1;
  }
  t0 -= sh.pref[lo];
  int i = lo * chunk, n = pg_tiles(p, i);
  while (t0 >= (int64_t)n * mult) {
    t0 -= (int64_t)n * mult;
    n = pg_tiles(p, ++i);
  }
  c.item = i;
  c.nt = n;
  c.head = (int)(t0 / n);
  c.i = (int)(t0 - (int64_t)c.head * n);
  cursor_open(p, c, lane);
  return total;
}

// (A, B) of one token: r^ = A c + B for the norm code c (log: its log2).  fp32 norms: A tells
// whether the token counts.  A token that does not count gets r^ = 0 whatever its record holds.
__device__ __forceinline__ float2 pg_norm_consts(const uint8_t* hdr, int nc, int tok, bool live) {
  if (nc == 4) return make_float2(live ? 1.f : 0.f, 0.f);
  const bool lg = nc & 1;
  if (!live) return make_float2(0.f, lg ? -INFINITY : 0.f);
  const float2 h = reinterpret_cast<const float2*>(hdr)[tok];
  const float inv = nc >= 2 ? 1.f / 255.f : 1.f / 15.f;
  if (lg) {
    const float lo = lg2_approx(h.x);
    return make_float2(h.y > h.x ? (lg2_approx(h.y) - lo) * inv : 0.f, lo);
  }
  return make_float2(h.y > h.x ? (h.y - h.x) * inv : 0.f, h.x);
}

// r^ of position j of a run whose norm codes (or fp32 norms) are in w.
template <int NC>
__device__ __forceinline__ float pg_norm(const uint32_t* w, int j, float2 ab) {
  if constexpr (NC == 4) {
    return ab.x != 0.f ? __uint_as_float(w[j]) : 0.f;
  } else {
    float c;
    if constexpr (NC >= 2) c = __uint_as_float(__byte_perm(w[j >> 2], 0x4B000000u, 0x7540 | (j & 3))) - 8388608.f;
    else c = __uint_as_float(((w[j >> 3] >> (4 * (j & 7))) & 15u) | 0x4B000000u) - 8388608.f;
    const float r = __fmaf_rn(c, ab.x, ab.y);
    return NC & 1 ? ex2_ftz(r) : r;
  }
}

template <int D, int QT>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
    attend_pages_f32(const __grid_constant__ AttPagesParams p, int bf_, int tab_v, int warp_bytes) {
  using C = PgF<D, QT>;
  constexpr int P = C::P, NQ = C::NQ, E = C::E, KP = C::KP, VL = C::VL, VT = C::VT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ PgShared sh;
  const bool bf = bf_ != 0;
  const int tid = threadIdx.x, lane = tid & 31, nw = blockDim.x >> 5;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int g = lane >> 2, t = lane & 3;
  uint8_t* const tk = smem;
  uint8_t* const tv = smem + tab_v;                // the same table where K and V have the same bins
  uint8_t* const pool = smem + tab_v + ((1 << p.v.w) << kTabShift);
  uint8_t* const pw = pool + warp * warp_bytes;
  uint8_t* const st_k = pw + C::W_STG;
  uint8_t* const st_kn = st_k + kBatch * p.k.ab;
  uint8_t* const st_kh = st_kn + kBatch * p.k.nb;
  uint8_t* const st_v = st_k + pg_stage_bytes(p.k);
  uint8_t* const st_vn = st_v + kBatch * p.v.ab;
  uint8_t* const st_vh = st_vn + kBatch * p.v.nb;
  float2* const kc = reinterpret_cast<float2*>(pw + C::W_KC);
  float2* const vc = reinterpret_cast<float2*>(pw + C::W_VC);
  float* const wt = reinterpret_cast<float*>(pw + C::W_P);       // [token][query]
  auto rec_of = [&](int w, int which) {
    return reinterpret_cast<float*>(pool + w * warp_bytes + (which ? C::W_Q : C::W_REC));
  };

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t bar_k = pg_smem(&sh.bars[2 * warp]), bar_v = bar_k + 8;
  if (lane == 0) {
    pg_bar_init(bar_k);
    pg_bar_init(bar_v);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.part[warp][0] = sh.part[warp][1] = -1;
    sh.ends0[warp] = 0;
  }
  Cursor cur;
  const int64_t total = pg_plan(p, sh, nw, cur);
  if (total == 0) return;                          // no tile for this CTA
  if (lane == 0) sh.empty[warp] = cur.left <= 0;

  // ---- staging: lane x copies plane x % 3 (angle | norm | header) of tile (x / 3) % 2, of K
  // (x < 6) or V ----
  const bool c_v = lane >= 6;
  const int c_plane = lane % 3, c_half = (lane / 3) & 1;
  const Book& cb = c_v ? p.v : p.k;
  const int c_row = lane >= 12 ? 0 : c_plane == 0 ? cb.ab : c_plane == 1 ? cb.nb : cb.hb;
  const uint8_t* const c_src = c_plane == 0 ? cb.codes : c_plane == 1 ? cb.norms : cb.hdr;
  const uint32_t c_dst = pg_smem(c_plane == 0 ? (c_v ? st_v : st_k) : c_plane == 1 ? (c_v ? st_vn : st_kn) : (c_v ? st_vh : st_kh)) +
                         c_half * kTile * c_row;
  const int tile_k = kTile * (p.k.ab + p.k.nb + p.k.hb), tile_v = kTile * (p.v.ab + p.v.nb + p.v.hb);
  uint32_t phase_k = 0, phase_v = 0;
  bool dead = false;                               // a wait ran out
  auto issue = [&](bool v, const Batch& b) {
    if (dead || (b.valid0 | b.valid1) == 0) return;
    if (lane == 0) pg_bar_expect(v ? bar_v : bar_k, ((b.valid0 > 0) + (b.valid1 > 0)) * (v ? tile_v : tile_k));
    __syncwarp();
    if (c_v == v && c_row > 0 && (c_half ? b.valid1 : b.valid0) > 0)
      pg_copy(c_dst, c_src + (c_half ? b.slot1 : b.slot0) * c_row, kTile * c_row, v ? bar_v : bar_k);
  };
  auto landed = [&](const Batch& b, uint32_t bar, uint32_t& phase) {
    if ((b.valid0 | b.valid1) != 0 && !dead) {
      dead = !__all_sync(0xffffffffu, pg_bar_wait(bar, phase));
      phase ^= 1u;
    }
    __syncwarp();
  };
  Batch b, nx;
  bool more = cursor_next(p, cur, lane, nx);
  if (more) {
    nx.begins = true;
    issue(false, nx);
    issue(true, nx);
  }

  // ---- bin-centre tables: entry k, copy c at k 2^kTabShift + 8 c; entries n .. 2^w - 1 repeat
  // entry n - 1 (codes >= n count as that) ----
  for (int side = 0; side < (tab_v ? 2 : 1); ++side) {
    const Book& bk = tab_v && side == 0 ? p.k : p.v;
    float2* const tab = reinterpret_cast<float2*>(side ? tv : tk);
    for (int e = tid; e < (1 << bk.w) * kCopies; e += blockDim.x)
      tab[e] = g_pg_centre.v[tab_offset_n(bk.n) + min(e / kCopies, bk.n - 1)];
  }
  __syncthreads();

  const uint32_t lane_off = (uint32_t)(lane % kCopies) * 8;
  const uint32_t km = ((1u << p.k.w) - 1u) << kTabShift, vm = ((1u << p.v.w) - 1u) << kTabShift;
  bool begun = false;                              // this warp has the first tile of the current (sequence, head)
  float m_[QT], l_[QT];
  float2 acc[NQ][4];

  // Scores of the staged batch: lane (g, t) takes positions KP t .. KP t + KP - 1 of tokens g and
  // g + 8 of a tile.  sv[x][i]: token 16 (i / 2) + 8 (i & 1) + g, query 4 x + t.
  auto scores = [&](float (&sv)[QT][4], auto nc_) {
    constexpr int NC = decltype(nc_)::value;
    const int wk = p.k.w;
#pragma unroll
    for (int x = 0; x < QT; ++x) sv[x][2] = sv[x][3] = 0.f;
#pragma unroll 1
    for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
      for (int x = 0; x < QT; ++x) { sv[x][0] = sv[x][2]; sv[x][1] = sv[x][3]; }
      if ((hf ? b.valid1 : b.valid0) == 0) continue;
      float2 s[NQ][2];
#pragma unroll
      for (int a = 0; a < NQ; ++a) s[a][0] = s[a][1] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int q8 = 0; q8 < KP / 8; ++q8) {
        uint32_t ca[2][2], nr[2][NC == 4 ? 8 : 2];
        float2 ab[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int tok = kTile * hf + 8 * r + g;
          const int off = tok * p.k.ab + (t * (KP / 8) + q8) * wk;     // 8 codes: wk bytes
          const uint32_t* w = reinterpret_cast<const uint32_t*>(st_k + (off & ~3));
          const int sh_ = (off & 3) * 8;
          const uint32_t w0 = w[0], w1 = w[1], w2 = w[2];
          ca[r][0] = __funnelshift_r(w0, w1, sh_);
          ca[r][1] = __funnelshift_rc(ca[r][0], __funnelshift_r(w1, w2, sh_), 4 * wk);
          ab[r] = kc[tok];
          const uint8_t* nrow = st_kn + tok * p.k.nb;
          const int p0 = KP * t + 8 * q8;
          if constexpr (NC == 4) {
            const uint4 u = *reinterpret_cast<const uint4*>(nrow + 4 * p0), v = *reinterpret_cast<const uint4*>(nrow + 4 * p0 + 16);
            nr[r][0] = u.x; nr[r][1] = u.y; nr[r][2] = u.z; nr[r][3] = u.w;
            nr[r][4] = v.x; nr[r][5] = v.y; nr[r][6] = v.z; nr[r][7] = v.w;
          } else if constexpr (NC >= 2) {
            const uint2 u = *reinterpret_cast<const uint2*>(nrow + p0);
            nr[r][0] = u.x; nr[r][1] = u.y;
          } else {
            nr[r][0] = *reinterpret_cast<const uint32_t*>(nrow + p0 / 2);
          }
        }
        const float4* qr = reinterpret_cast<const float4*>(pw + C::W_Q + t * C::QRUN + q8 * 64);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          float2 y[2][2];
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t o = (pg_rotr(ca[r][(j + i) >> 2], (wk * ((j + i) & 3) - kTabShift) & 31) & km) | lane_off;
              const float2 cs = *reinterpret_cast<const float2*>(tk + o);
              const float rr = pg_norm<NC>(nr[r], j + i, ab[r]);
              y[r][i] = mul2(cs, make_float2(rr, rr));
            }
#pragma unroll
          for (int a = 0; a < NQ; ++a) {
            const float4 q = qr[a * (4 * C::QRUN / 16) + j / 2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              s[a][r] = ffma2(y[r][0], make_float2(q.x, q.y), s[a][r]);
              s[a][r] = ffma2(y[r][1], make_float2(q.z, q.w), s[a][r]);
            }
          }
        }
      }
      // sums over the four lanes of a token; lane t keeps query 4 x + t
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float v[4];
#pragma unroll
          for (int a = 0; a < 4; ++a) v[a] = s[4 * x + a][r].x + s[4 * x + a][r].y;
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const float give = t & 2 ? v[a] : v[a + 2], keep = t & 2 ? v[a + 2] : v[a];
            v[a] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
          }
          const float give = t & 1 ? v[0] : v[1], keep = t & 1 ? v[1] : v[0];
          sv[x][2 + r] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
        }
    }
  };

  // Values: lane (vt, vl) takes positions 4 vl .. 4 vl + 3 of tokens vt, vt + VT, ...
  const int vl = lane % VL, vt = lane / VL;
  auto values = [&](int tokens, auto nc_) {
    constexpr int NC = decltype(nc_)::value;
    const int wv = p.v.w, bit = 4 * vl * wv, woff = (bit >> 5) * 4, wsh = bit & 31;
#pragma unroll 1
    for (int tok = vt; tok < tokens; tok += VT) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(st_v + tok * p.v.ab + woff);
      const uint32_t ca = __funnelshift_r(w[0], w[1], wsh);
      const float2 ab = vc[tok];
      const uint8_t* nrow = st_vn + tok * p.v.nb;
      uint32_t nr[4];
      if constexpr (NC == 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(nrow + 16 * vl);
        nr[0] = u.x; nr[1] = u.y; nr[2] = u.z; nr[3] = u.w;
      } else if constexpr (NC >= 2) {
        nr[0] = *reinterpret_cast<const uint32_t*>(nrow + 4 * vl);
      } else {
        nr[0] = *reinterpret_cast<const uint16_t*>(nrow + 2 * vl);
      }
      float pr[NQ];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const float4 v = *reinterpret_cast<const float4*>(wt + tok * NQ + 4 * x);
        pr[4 * x] = v.x; pr[4 * x + 1] = v.y; pr[4 * x + 2] = v.z; pr[4 * x + 3] = v.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t o = (pg_rotr(ca, (wv * j - kTabShift) & 31) & vm) | lane_off;
        const float2 cs = *reinterpret_cast<const float2*>(tv + o);
        const float rr = pg_norm<NC>(nr, j, ab);
        const float2 y = mul2(cs, make_float2(rr, rr));
#pragma unroll
        for (int a = 0; a < NQ; ++a) acc[a][j] = ffma2(y, make_float2(pr[a], pr[a]), acc[a][j]);
      }
    }
  };

  while (more) {
    b = nx;
    if (b.begins) {                                // a new (sequence, head)
      begun = b.first;
      __syncwarp();
#pragma unroll 1
      for (int a = 0; a < NQ; ++a) {
        float y[E];
#pragma unroll
        for (int k = 0; k < E; ++k) y[k] = 0.f;
        if (a < p.group) pg_load_query<D>(p, bf, b.seq, b.head, a, lane, y);
#pragma unroll
        for (int k = 0; k < E; k += 2) {           // pair (E lane + k) / 2
          const int i = pair_slot<D>((E * lane + k) / 2);
          *reinterpret_cast<float2*>(pw + C::W_Q + (a * 4 + i / KP) * C::QRUN + (i % KP) * 8) = make_float2(y[k], y[k + 1]);
        }
      }
      __syncwarp();
#pragma unroll
      for (int x = 0; x < QT; ++x) { m_[x] = -INFINITY; l_[x] = 0.f; }
#pragma unroll
      for (int a = 0; a < NQ; ++a)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[a][j] = make_float2(0.f, 0.f);
    }
    more = cursor_next(p, cur, lane, nx);
    if (more) nx.begins = b.ends;
    const bool any = (b.valid0 | b.valid1) != 0;
    landed(b, bar_k, phase_k);
    float sv[QT][4];
    const bool alive = (lane < kTile ? lane < b.valid0 : lane - kTile < b.valid1);   // token `lane` counts
    if (any) {
      kc[lane] = pg_norm_consts(st_kh, p.k.nc, lane, alive);
      __syncwarp();
      switch (p.k.nc) {
        case 0: scores(sv, IC<0>{}); break;
        case 1: scores(sv, IC<1>{}); break;
        case 2: scores(sv, IC<2>{}); break;
        case 3: scores(sv, IC<3>{}); break;
        default: scores(sv, IC<4>{}); break;
      }
      __syncwarp();                                // every lane is done with the K rows
    }
    if (more) issue(false, nx);
    if (any) {
      bool moved = false;
      float fix[QT];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int o = 8 * (i & 1) + g;
          if (o >= (i >> 1 ? b.valid1 : b.valid0)) sv[x][i] = -INFINITY;
          mx = fmaxf(mx, sv[x][i]);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float mn = fmaxf(m_[x], mx), ref = mn == -INFINITY ? 0.f : mn;
        fix[x] = ex2_approx(m_[x] - ref);
        moved |= mn > m_[x];
        m_[x] = mn;
        l_[x] *= fix[x];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float pr = ex2_approx(sv[x][i] - ref);
          l_[x] += pr;
          wt[(16 * (i >> 1) + 8 * (i & 1) + g) * NQ + 4 * x + t] = pr;
        }
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int a = 0; a < NQ; ++a) {
          const float f = __shfl_sync(0xffffffffu, fix[a >> 2], a & 3);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[a][j] = mul2(acc[a][j], make_float2(f, f));
        }
      }
    }
    landed(b, bar_v, phase_v);
    if (any) {
      vc[lane] = pg_norm_consts(st_vh, p.v.nc, lane, alive);
      __syncwarp();
      const int tokens = b.valid1 > 0 ? kBatch : kTile;
      switch (p.v.nc) {
        case 0: values(tokens, IC<0>{}); break;
        case 1: values(tokens, IC<1>{}); break;
        case 2: values(tokens, IC<2>{}); break;
        case 3: values(tokens, IC<3>{}); break;
        default: values(tokens, IC<4>{}); break;
      }
      __syncwarp();                                // every lane is done with the V rows
    }
    if (more) issue(true, nx);
    if (b.ends) {
      // the part's record, elements in their order; in the place of the queries, unless the
      // part began in an earlier warp
      const bool whole = begun && b.last;
      float* const rec = rec_of(warp, begun);
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l_[x] += __shfl_xor_sync(0xffffffffu, l_[x], o);
#pragma unroll
      for (int a = 0; a < NQ; ++a)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int o = VL; o < 32; o <<= 1) {
            acc[a][j].x += __shfl_xor_sync(0xffffffffu, acc[a][j].x, o);
            acc[a][j].y += __shfl_xor_sync(0xffffffffu, acc[a][j].y, o);
          }
          if (vt == 0) *reinterpret_cast<float2*>(rec + a * pg_rec_floats(D) + 2 + 2 * slot_pair<D>(4 * vl + j)) = acc[a][j];
        }
      if (g == 0) {
#pragma unroll
        for (int x = 0; x < QT; ++x)
          *reinterpret_cast<float2*>(rec + (4 * x + t) * pg_rec_floats(D)) =
              make_float2(m_[x], dead ? __int_as_float(0x7FC00000) : l_[x]);
      }
      __syncwarp();
      if (whole) {
        for (int a = 0; a < p.group; ++a) {
          const float* r = rec + a * pg_rec_floats(D);
          float y[E];
#pragma unroll
          for (int k = 0; k < E; ++k) y[k] = r[2 + E * lane + k];
          pg_store_out<D>(p, bf, b.seq, b.head, a, lane, y, r[1]);
        }
      } else if (lane == 0) {
        sh.part[warp][begun] = b.seq * p.pg.heads + b.head;
        if (!begun) sh.ends0[warp] = b.last;
      }
    }
  }
  if (dead) {                                      // the copies issued and not waited for
    (void)pg_bar_wait(bar_k, phase_k);
    (void)pg_bar_wait(bar_v, phase_v);
  }
  __syncthreads();
  pg_join<D>(p, sh, bf, nw, warp, lane, rec_of);
}

// Joins the CTAs' parts of one (sequence, head) and query: warps take CTAs in turn, their
// sums are added in the order of the warps.  Also the zeros of a (sequence, head) without a token.
constexpr int kJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) attend_pages_join(const __grid_constant__ AttPagesParams p, int bf_) {
  constexpr int E = D / 32, RF = pg_rec_floats(D);
  __shared__ float part[kJoinWarps][D], red[kJoinWarps][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int a = blockIdx.x % p.group, seg = blockIdx.x / p.group;
  const int s = seg / p.pg.heads, h = seg % p.pg.heads;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t total = p.plan[p.items], nc = p.plan[p.items + 1];
  int64_t t0, t1;
  if (p.selected) {
    t0 = p.plan[seg];
    t1 = p.plan[seg + 1];
  } else {
    const int64_t x = p.plan[s], n = (p.plan[s + 1] - x) / p.pg.heads;
    t0 = x + n * h;
    t1 = t0 + n;
  }
  float y[E];
#pragma unroll
  for (int k = 0; k < E; ++k) y[k] = 0.f;
  if (t0 == t1) {
    if (warp == 0) pg_store_out<D>(p, bf_ != 0, s, h, a, lane, y, 0.f);
    return;
  }
  // CTA c starts at tile floor(total c / nc)
  const int c0 = (int)(((t0 + 1) * nc - 1) / total), c1 = (int)((t1 * nc - 1) / total);
  if (c0 == c1) return;                            // finished by that CTA
  auto rec = [&](int c) { return p.part + (((int64_t)c * 2 + (c == c0)) * p.group + a) * RF; };
  float M = -INFINITY;
  for (int c = c0 + (int)threadIdx.x; c <= c1; c += kJoinWarps * 32) M = fmaxf(M, rec(c)[0]);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) red[warp][0] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) M = fmaxf(M, red[w][0]);
  float l = 0.f;
#pragma unroll 4
  for (int c = c0 + warp; c <= c1; c += kJoinWarps) {
    const float* r = rec(c);
    const float f = r[0] == -INFINITY ? 0.f : ex2_approx(r[0] - M);
    l = __fmaf_rn(r[1], f, l);
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] = __fmaf_rn(r[2 + E * lane + k], f, y[k]);
  }
#pragma unroll
  for (int k = 0; k < E; ++k) part[warp][E * lane + k] = y[k];
  if (lane == 0) red[warp][1] = l;
  __syncthreads();
  if (warp != 0) return;
  l = 0.f;
#pragma unroll
  for (int k = 0; k < E; ++k) y[k] = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    l += red[w][1];
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] += part[w][E * lane + k];
  }
  pg_store_out<D>(p, bf_ != 0, s, h, a, lane, y, l);
}

template <typename K>
static cudaError_t set_smem_once(K kp, std::atomic<int>* ready) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (ready[dev].load(std::memory_order_acquire)) return cudaSuccess;
  // static shared memory counts towards the 227 KB
  const cudaError_t e = cudaFuncSetAttribute(kp, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)sizeof(PgShared) - 256);
  if (e == cudaSuccess) ready[dev].store(1, std::memory_order_release);
  return e;
}

template <int D>
static cudaError_t launch_join(const AttPagesParams& p, bool bf, cudaStream_t st) {
  // starts as the main kernel's CTAs leave and waits for its results on the device
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.pg.seqs * p.pg.heads * p.group));
  cfg.blockDim = dim3(kJoinWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, attend_pages_join<D>, p, (int)bf);
}

template <int D, int QT>
static cudaError_t launch_f32_t(const AttPagesParams& p, bool bf, cudaStream_t st) {
  using C = PgF<D, QT>;
  auto kp = attend_pages_f32<D, QT>;
  static std::atomic<int> ready[64];
  cudaError_t e = set_smem_once(kp, ready);
  if (e != cudaSuccess) return e;
  const int tab_v = p.k.n == p.v.n ? 0 : (1 << p.k.w) << kTabShift;
  const int tabs = tab_v + ((1 << p.v.w) << kTabShift);
  const int warp_bytes = (C::W_STG + pg_stage_bytes(p.k) + pg_stage_bytes(p.v) + 127) / 128 * 128;
  const int nw = std::min(kMaxWarps, (227 * 1024 - (int)sizeof(PgShared) - 256 - tabs) / warp_bytes);
  kp<<<p.ctas, nw * 32, tabs + nw * warp_bytes, st>>>(p, (int)bf, tab_v, warp_bytes);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_join<D>(p, bf, st);
}

// CTAs of the main kernel: one on every SM.
int attend_pages_ctas(int, int, int, int sms) { return std::min(sms, kAttPgMaxCtas); }

cudaError_t launch_attend_pages(int d, int dtype, const AttPagesParams& p, cudaStream_t st) {
  const bool bf = dtype == TAC_BF16;
  if (d == 128) return p.group <= 4 ? launch_f32_t<128, 1>(p, bf, st) : launch_f32_t<128, 2>(p, bf, st);
  return p.group <= 4 ? launch_f32_t<64, 1>(p, bf, st) : launch_f32_t<64, 2>(p, bf, st);
}

}  // namespace tac
