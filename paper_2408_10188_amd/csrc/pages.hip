// Copies of pages in the pools of a paged cache, over all layers in one launch (the partly filled last page of a forked
// sequence, or the moves that a compaction plan lists).  Memory-bound: 1 byte read and 1 written per byte.
#include <algorithm>

#include "paged.h"

namespace mmsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A workgroup takes 2 KiB, 128 pieces of 16 bytes, of one (copy, layer, K or V), one piece a thread, read and written past the caches.  Moving 301 pages of 64 tokens x 4
// heads in 28 layers (2.2 GB read and written): 372 us (5.9 TB/s; a copy of 1 GiB at its best 6.5); with the default cache policy and 16 KiB a
// workgroup 441, with 4 KiB 380, with 8 KiB or more 427 to 432.  Pieces of a page are numbered slot by slot inside a head or head by head
// inside a slot, whichever lies closer together, so that neighbouring threads have neighbouring addresses.
constexpr int kThreads = 128;
struct CopyArgs {
  char* base[2];
  int64_t layer_bytes, page_bytes, outer_bytes, inner_bytes;
  const int32_t* copies;
  int32_t n_pages, page_size, n_pieces, vec_bits;
  FastDiv inner, chunks, layers;
  int32_t slots_inside;                                 // the inner index is the slot
};
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyArgs a) {
  const uint32_t rest = blockIdx.x / a.chunks, chunk = blockIdx.x - rest * a.chunks.d;
  const uint32_t pair = rest >> 1, copy = pair / a.layers, layer = pair - copy * a.layers.d;
  const int src = a.copies[copy * 3], dst = a.copies[copy * 3 + 1], n = min(a.copies[copy * 3 + 2], a.page_size);
  if (src == dst || src < 0 || dst < 0 || src >= a.n_pages || dst >= a.n_pages || n <= 0) return;
  const uint32_t p = chunk * kThreads + threadIdx.x, r = p >> a.vec_bits;
  const uint32_t outer = r / a.inner, inner = r - outer * a.inner.d;
  if (p >= (uint32_t)a.n_pieces || (int)(a.slots_inside ? inner : outer) >= n) return;
  char* const at = a.base[rest & 1] + layer * a.layer_bytes + outer * a.outer_bytes + inner * a.inner_bytes + (p & ((1u << a.vec_bits) - 1)) * 16;
  const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + src * a.page_bytes));
  __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(at + dst * a.page_bytes));
}

}  // namespace

hipError_t launch_copy_pages(const CacheArgs& c, int n_layers, int64_t layer_stride, int Hkv, int d, int elt_bytes, const int32_t* copies, int n_copies,
                             hipStream_t stream) {
  if (n_copies == 0 || n_layers == 0) return hipSuccess;
  CopyArgs a;
  a.base[0] = c.k; a.base[1] = c.v;
  a.layer_bytes = layer_stride * elt_bytes; a.page_bytes = c.page_stride * elt_bytes;
  a.slots_inside = c.head_stride >= c.tok_stride;
  a.inner_bytes = (a.slots_inside ? c.tok_stride : c.head_stride) * elt_bytes;
  a.outer_bytes = (a.slots_inside ? c.head_stride : c.tok_stride) * elt_bytes;
  a.inner = fast_div(a.slots_inside ? c.page_size : Hkv);
  a.n_pages = c.n_pages; a.page_size = c.page_size;
  const int vec = d * elt_bytes / 16;
  a.vec_bits = __builtin_ctz(vec);
  a.n_pieces = c.page_size * Hkv * vec;
  const int chunks = (a.n_pieces + kThreads - 1) / kThreads;
  a.chunks = fast_div(chunks); a.layers = fast_div(n_layers);
  // a grid has fewer than 2^32 threads
  const int64_t per_copy = (int64_t)chunks * 2 * n_layers, most = std::max<int64_t>(1, ((int64_t)1 << 23) / per_copy);
  for (int64_t first = 0; first < n_copies; first += most) {
    a.copies = copies + 3 * first;
    copy_pages_kernel<<<dim3((unsigned)(per_copy * std::min<int64_t>(most, n_copies - first))), dim3(kThreads), 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mmsp
