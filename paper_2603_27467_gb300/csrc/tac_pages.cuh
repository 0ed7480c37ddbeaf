// Parameters of the paged-cache kernels (tac_pages.cu, tac_attend_pages.cu), shared with the C ABI.
#pragma once
#include "tac_common.cuh"

namespace tac {

// Page table and lengths as the kernels take them.
struct Paging {
  const int32_t* table;
  const int32_t* lengths;
  int64_t table_stride;
  int64_t pages;
  int32_t width;       // table columns
  int32_t seqs;
  int32_t heads;       // KV heads
  int32_t page;        // tokens a page
};

struct BoundsParams {
  Paging pg;
  int8_t* codes;
  float* scales;
  const void* k;
  int64_t rows, row_stride, head_stride;   // elements
  const int32_t* first;                    // or nullptr: one row a sequence
  const int32_t* start;
};

struct SelectParams {
  Paging pg;
  const int8_t* codes;
  const float* scales;
  const void* q;
  int64_t seq_stride, row_stride;          // elements
  int32_t group, budget, keep_first, keep_last;
  int32_t* selected;
  int32_t* counts;
};

// 2^e', e' the smallest whole number >= -126 with a <= 127 * 2^e' (a >= 0, finite), as e'.
__device__ __forceinline__ int box_exp(float a) {
  const uint32_t u = __float_as_uint(a);
  // a = m 2^x, 1 <= m < 2: 127 * 2^e' = (127 / 64) 2^(e' + 6); subnormal a fall below the clamp
  const int x = (int)(u >> 23) - 127;
  return max(((u & 0x7FFFFFu) <= 0x7E0000u ? x - 6 : x - 5), -126);
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Codebook of one side (K or V) at run time.
struct Book {
  const uint8_t* codes;
  const uint8_t* norms;
  const uint8_t* hdr;
  int32_t n, w;        // bins, code bits
  int32_t nc;          // norm case: 0 / 1 = 4-bit linear / log, 2 / 3 = 8-bit linear / log, 4 = fp32
  int32_t ab, nb, hb;  // bytes of a record in each plane
  uint32_t signs[4];
};

struct AttPagesParams {
  Paging pg;
  Book k, v;
  const int32_t* selected;                 // or nullptr: every page
  const int32_t* counts;
  int32_t budget;
  int32_t group;
  float scale;
  const void* q;
  void* out;
  int64_t q_seq, q_row, o_seq, o_row;      // strides, elements
  int32_t ctas;                            // grid of the main kernel
  int32_t items;                           // spans of tiles: sequences, or (sequence, head)s with `selected`
  int32_t* plan;                           // workspace: items + 1 first tiles, then the CTAs in use and the warps of each
  float* part;                             // workspace: [ctas][2][group][d + 2]
};

// A tile is 16 tokens of one page.
constexpr int kTile = 16;
// Partial result of one (sequence, head) and query: maximum (log2 units), sum, accumulator.
__host__ __device__ constexpr int pg_rec_floats(int d) { return d + 2; }
constexpr int kAttPgMaxCtas = 1024;

// CTAs of the main kernel: one on every SM.
inline int attend_pages_ctas(int sms) { return sms < kAttPgMaxCtas ? sms : kAttPgMaxCtas; }
cudaError_t launch_attend_pages_128_bf16(const AttPagesParams& p, cudaStream_t st);
cudaError_t launch_attend_pages_128_f32(const AttPagesParams& p, bool bf, cudaStream_t st);
cudaError_t launch_attend_pages_64_bf16(const AttPagesParams& p, cudaStream_t st);
cudaError_t launch_attend_pages_64_f32(const AttPagesParams& p, bool bf, cudaStream_t st);

cudaError_t launch_page_bounds(int d, int dtype, const BoundsParams& p, int sms, cudaStream_t st);
cudaError_t launch_select_pages(int d, int dtype, const SelectParams& p, int sms, cudaStream_t st);

}  // namespace tac
