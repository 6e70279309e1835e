// The paged cache and the rotary positions as kernels see them, and the launchers the C-ABI layer dispatches to.
#pragma once
#include "common.h"

namespace mmsp {

struct CacheArgs {
  char* k; char* v;                                     // pool
  int64_t page_stride, tok_stride, head_stride;         // elements
  const int32_t* table; int64_t table_stride;
  const int32_t* lengths;
  const int32_t* cu_new;                                // nullptr: one new token per sequence
  int32_t n_pages, page_size, max_pages, n_seqs, n_rows;
  int32_t most_new;                                     // of a sequence, with cu_new; 0: not known
  FastDiv page_div;                                     // tokens / page_size
};

// A read of what no kernel of the call writes: a scalar load where the address is the same in all lanes.
template <class T>
__device__ __forceinline__ T load_const(const T* p, int64_t i) {
  return ((const __attribute__((address_space(4))) T*)(uintptr_t)p)[i];
}

// The new rows [first, first + count) of sequence s, the token of the first of them, and the tokens that the page table has room for.  Whatever the device arrays hold,
// rows stay inside the row buffers and tokens below `length` inside the page table.  Token numbers go by the length as given: new tokens behind the table's end are nowhere,
// they do not take the numbers of those before it.
struct SeqRows { int first, count, token, length; };
__device__ __forceinline__ SeqRows rows_of_seq(const CacheArgs& c, int s) {
  SeqRows r;
  const int length = max(load_const(c.lengths, s), 0);
  r.length = min(length, c.max_pages * c.page_size);
  if (c.cu_new == nullptr) {
    r.first = s;
    r.count = 1;
  } else {
    r.first = min(max(load_const(c.cu_new, s), 0), c.n_rows);
    r.count = min(max(load_const(c.cu_new, s + 1), r.first), c.n_rows) - r.first;
  }
  r.token = length - r.count;
  return r;
}
// The sequence of row r, -1 behind the last one: the first s with r < cu_new[s + 1].
__device__ __forceinline__ int seq_of_row(const CacheArgs& c, int r) {
  if (c.cu_new == nullptr) return r;
  if (r >= load_const(c.cu_new, c.n_seqs) || r < load_const(c.cu_new, 0)) return -1;
  int lo = 0, hi = c.n_seqs;                            // cu[lo] <= r < cu[hi]
  while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (load_const(c.cu_new, m) <= r) lo = m; else hi = m; }
  return lo;
}

constexpr int kMaxAxes = 4;
struct RotaryArgs {
  uint64_t turns[64];                                   // revolutions per position, in units of 2^-64
  uint8_t axis[64];
  const int32_t* positions; int64_t pos_stride;
  int32_t n_axes;
  int32_t inverse;
};
struct HeadsArgs { const char* x; char* y; int64_t x_ts, x_hs, y_ts, y_hs; int32_t n_heads; };

hipError_t launch_rotary(const RotaryArgs& rot, const HeadsArgs (&t)[2], int n_tensors, int n_rows, int d, int x_dtype, int y_dtype, hipStream_t stream);

struct AppendArgs {
  CacheArgs cache;
  const char* q; const char* k; const char* v; char* q_out;
  int64_t q_ts, q_hs, out_ts, out_hs, kv_ts, kv_hs;     // out: of q_out
  int32_t Hq, Hkv;                                      // Hq: 0 without q_out
};
hipError_t launch_append(const AppendArgs& a, const RotaryArgs* rot, int d, int io_dtype, hipStream_t stream);

struct CacheAttnArgs {
  CacheArgs cache;
  const void* q; void* o_final; float* o; float* lse;
  int64_t q_ts, q_hs, lse_hs;
  int32_t Hq, Hkv, group, d;
  FastDiv group_div;
  float scale;
  char* ws;
};
double cache_attn_tiles(const CacheAttnArgs& a, int io_dtype);   // tiles of work at most; more than 2^30 are for the caller to refuse
int64_t cache_attn_workspace_bytes(const CacheAttnArgs& a, int io_dtype);
hipError_t launch_cache_attn(const CacheAttnArgs& a, int io_dtype, hipStream_t stream);

hipError_t launch_copy_pages(const CacheArgs& c, int n_layers, int64_t layer_stride, int Hkv, int d, int elt_bytes, const int32_t* copies, int n_copies,
                             hipStream_t stream);

}  // namespace mmsp
