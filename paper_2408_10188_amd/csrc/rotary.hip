// Rotary positions with several axes, alone (Q and K, or their gradients) and on the way of new tokens into a paged cache.
//
// Pair i of a head, (x[i], x[i + d/2]), is turned by a_i = position[axis(i)] * theta^(-2i/d).  The angle is kept as a fraction of a
// revolution in 64-bit fixed point: position * turns[i] modulo 2^64 is exact, where an fp32 product of a far position (2^18) and a
// frequency near 1 is off by up to 2^-7 rad.  Its upper 32 bits, as an fp32 number of half turns in [-1, 1), are off by at most 2^-25 half turns
// (10^-7 rad), and sine and cosine of a multiple of pi need no range reduction.
//
// The sines and cosines of a row are the same for all its heads: a workgroup computes those of its rows once, into LDS.  A thread then takes
// items of 8 pairs of one head, 16 bytes (bf16) of either half, and has several of them on their way before the first sine is known.
#include <algorithm>

#include "paged.h"

namespace mmsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));   // round to nearest even
}

// 8 consecutive elements, bf16 or f32, as they lie in memory and as fp32 numbers
template <bool kBf16> struct Eight { u32x4 w[kBf16 ? 1 : 2]; };
template <bool kBf16>
__device__ __forceinline__ Eight<kBf16> load8(const char* p) {
  Eight<kBf16> e;
#pragma unroll
  for (int i = 0; i < (kBf16 ? 1 : 2); ++i) e.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);   // read once
  return e;
}
// Results are written past the caches: 25.4 -> 23.1 us for 8192 rows of 28/4 heads (5.8 TB/s; a copy of that size reaches 6.0), 91.6 -> 84.4 us
// for 24 thousand prompt rows that go into a cache (452 MB).
template <bool kBf16>
__device__ __forceinline__ void store8(char* p, const Eight<kBf16>& e) {
#pragma unroll
  for (int i = 0; i < (kBf16 ? 1 : 2); ++i) __builtin_nontemporal_store(e.w[i], reinterpret_cast<u32x4*>(p) + i);
}
template <bool kBf16>
__device__ __forceinline__ void unpack8(const Eight<kBf16>& e, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (kBf16) f[i] = __uint_as_float(i & 1 ? e.w[0][i / 2] & 0xffff0000u : e.w[0][i / 2] << 16);
    else f[i] = __uint_as_float(e.w[i / 4][i % 4]);
  }
}
template <bool kBf16>
__device__ __forceinline__ Eight<kBf16> pack8(const float (&f)[8]) {
  Eight<kBf16> e;
#pragma unroll
  for (int i = 0; i < (kBf16 ? 4 : 8); ++i) {
    if constexpr (kBf16) e.w[0][i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    else e.w[i / 4][i % 4] = __float_as_uint(f[i]);
  }
  return e;
}

// Items of a thread in flight.  28/4 heads, 8192 rows, bf16 (134 MB): 27.1 us with one, 25.6 with two, 25.4 with four, 26.1 with six; the gradient, f32 to bf16 with
// twice the bytes an item: 34.9 with one, 36.0 with two, 37.0 with four.
template <bool kBf16> constexpr int items_of() { return kBf16 ? 4 : 1; }
constexpr int kMaxRows = 32;                            // rows of a workgroup

struct Angles {
  float cs[kMaxRows * 64], sn[kMaxRows * 64];           // [row][pair]
};
// Sines and cosines of rows [row0, row0 + rows), half = 2^half_bits pairs each.
__device__ __forceinline__ void angles_of(const RotaryArgs& r, int row0, int rows, int half_bits, Angles& to) {
  for (int i = threadIdx.x; i < rows << half_bits; i += 256) {
    const int pair = i & ((1 << half_bits) - 1);
    const int p = r.positions[r.axis[pair] * r.pos_stride + row0 + (i >> half_bits)];
    const uint64_t angle = (uint64_t)(int64_t)p * r.turns[pair];
    float sn, cs;
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &sn, &cs);
    to.cs[i] = cs;
    to.sn[i] = r.inverse ? -sn : sn;
  }
}

template <bool kIn, bool kOut>
__device__ __forceinline__ void turn8(const Eight<kIn>& a, const Eight<kIn>& b, const float* cs_at, const float* sn_at, Eight<kOut>& ya, Eight<kOut>& yb) {
  float x[8], z[8], u[8], w[8], cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    *reinterpret_cast<float4*>(cs + i) = *reinterpret_cast<const float4*>(cs_at + i);
    *reinterpret_cast<float4*>(sn + i) = *reinterpret_cast<const float4*>(sn_at + i);
  }
  unpack8(a, x);
  unpack8(b, z);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u[i] = x[i] * cs[i] - z[i] * sn[i];
    w[i] = z[i] * cs[i] + x[i] * sn[i];
  }
  ya = pack8<kOut>(u);
  yb = pack8<kOut>(w);
}

// Items of a workgroup: item i is piece i % vec of head (i / vec) % heads of row i / vec / heads.
struct Item { int row, h, piece; };
__device__ __forceinline__ Item item_of(uint32_t i, int vec_bits, const FastDiv& heads) {
  Item x;
  const uint32_t rh = i >> vec_bits, r = rh / heads;
  x.piece = (int)(i & ((1u << vec_bits) - 1));
  x.row = (int)r;
  x.h = (int)(rh - r * heads.d);
  return x;
}

template <bool kIn /* bf16 */, bool kOut>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs rot, HeadsArgs t0, HeadsArgs t1, int n_rows, int rows_each, int vec_bits, FastDiv heads) {
  __shared__ Angles angles;
  const int row0 = blockIdx.x * rows_each, rows = min(rows_each, n_rows - row0), half = 8 << vec_bits;
  constexpr int kInBytes = kIn ? 2 : 4, kOutBytes = kOut ? 2 : 4, kItems = items_of<kIn>();
  const int n = rows * (int)heads.d << vec_bits;
  for (int first = 0; first < n; first += 256 * kItems) {
    Eight<kIn> xa[kItems], xb[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = first + k * 256 + threadIdx.x;
      const Item it = item_of(min(i, n - 1), vec_bits, heads);
      const bool second = it.h >= t0.n_heads;
      const int64_t ts = second ? t1.x_ts : t0.x_ts, hs = second ? t1.x_hs : t0.x_hs;
      const char* x = (second ? t1.x : t0.x) + ((row0 + it.row) * ts + (second ? it.h - t0.n_heads : it.h) * hs + it.piece * 8) * kInBytes;
      if (i < n) {
        xa[k] = load8<kIn>(x);
        xb[k] = load8<kIn>(x + half * kInBytes);
      }
    }
    if (first == 0) {
      angles_of(rot, row0, rows, vec_bits + 3, angles);
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = first + k * 256 + threadIdx.x;
      if (i >= n) break;
      const Item it = item_of(i, vec_bits, heads);
      const bool second = it.h >= t0.n_heads;
      const int64_t ts = second ? t1.y_ts : t0.y_ts, hs = second ? t1.y_hs : t0.y_hs;
      char* y = (second ? t1.y : t0.y) + ((row0 + it.row) * ts + (second ? it.h - t0.n_heads : it.h) * hs + it.piece * 8) * kOutBytes;
      const int at = it.row * half + it.piece * 8;
      Eight<kOut> ya, yb;
      turn8<kIn, kOut>(xa[k], xb[k], angles.cs + at, angles.sn + at, ya, yb);
      store8<kOut>(y, ya);
      store8<kOut>(y + half * kOutBytes, yb);
    }
  }
}

// The same for new tokens.  Workgroups [0, q_blocks) turn rows of Q, the others rows of K and copy V's (heads [0, Hkv) are K's, then V's): apart, because the few heads
// of K and V then bring more consecutive tokens of a page to a workgroup (24 thousand prompt rows of 28/4 heads: 88.2 us together, 85.5 apart).
template <bool kBf16, bool kRotary>
__global__ __launch_bounds__(256) void append_kernel(RotaryArgs rot, AppendArgs a, int q_blocks, int q_rows, int kv_rows, int vec_bits, FastDiv q_heads, FastDiv kv_heads) {
  __shared__ Angles angles;
  __shared__ int64_t slot_at[kMaxRows];                 // where a row's K and V go, in elements; below 0: nowhere
  __shared__ int live[kMaxRows];
  const bool is_q = (int)blockIdx.x < q_blocks;
  const int rows_each = is_q ? q_rows : kv_rows, row0 = ((int)blockIdx.x - (is_q ? 0 : q_blocks)) * rows_each, rows = min(rows_each, a.cache.n_rows - row0), half = 8 << vec_bits;
  const FastDiv heads = is_q ? q_heads : kv_heads;
  constexpr int kBytes = kBf16 ? 2 : 4, kItems = items_of<kBf16>();
  const int n = rows * (int)heads.d << vec_bits;
  for (int first = 0; first < n; first += 256 * kItems) {
    Eight<kBf16> xa[kItems], xb[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = first + k * 256 + threadIdx.x;
      const Item it = item_of(min(i, n - 1), vec_bits, heads);
      const bool is_v = !is_q && it.h >= a.Hkv;
      const int hh = it.h - (is_v ? a.Hkv : 0);
      const int64_t ts = is_q ? a.q_ts : a.kv_ts, hs = is_q ? a.q_hs : a.kv_hs;
      const char* x = (is_q ? a.q : is_v ? a.v : a.k) + ((row0 + it.row) * ts + hh * hs + it.piece * 8) * kBytes;
      if (i < n) {
        xa[k] = load8<kBf16>(x);
        xb[k] = load8<kBf16>(x + half * kBytes);
      }
    }
    if (first == 0) {
      if ((int)threadIdx.x < rows) {
        const int row = row0 + threadIdx.x, seq = seq_of_row(a.cache, row);
        int64_t at = -1;
        if (seq >= 0) {
          const SeqRows s = rows_of_seq(a.cache, seq);
          const int token = s.token + row - s.first;
          if (token >= 0 && token < s.length) {          // behind the table's end: not written
            const int p = (int)((uint32_t)token / a.cache.page_div), page = a.cache.table[seq * a.cache.table_stride + p];
            if (page >= 0 && page < a.cache.n_pages) at = page * a.cache.page_stride + (token - p * a.cache.page_size) * a.cache.tok_stride;
          }
        }
        slot_at[threadIdx.x] = at;
        live[threadIdx.x] = seq >= 0;
      }
      if (kRotary) angles_of(rot, row0, rows, vec_bits + 3, angles);
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = first + k * 256 + threadIdx.x;
      if (i >= n) break;
      const Item it = item_of(i, vec_bits, heads);
      const bool is_v = !is_q && it.h >= a.Hkv;
      char* y;
      if (is_q) {
        if (!live[it.row]) continue;                    // padding behind the last sequence
        y = a.q_out + ((row0 + it.row) * a.out_ts + it.h * a.out_hs + it.piece * 8) * kBytes;
      } else {
        const int64_t at = slot_at[it.row];
        if (at < 0) continue;
        y = (is_v ? a.cache.v : a.cache.k) + (at + (it.h - (is_v ? a.Hkv : 0)) * a.cache.head_stride + it.piece * 8) * kBytes;
      }
      const int at = it.row * half + it.piece * 8;
      Eight<kBf16> ya = xa[k], yb = xb[k];
      if (kRotary && !is_v) turn8<kBf16, kBf16>(xa[k], xb[k], angles.cs + at, angles.sn + at, ya, yb);
      store8<kBf16>(y, ya);
      store8<kBf16>(y + half * kBytes, yb);
    }
  }
}

// Rows of a workgroup: enough for the items that a thread has in flight, but not so many that CUs stay idle, nor so few that a grid of two such parts has 2^32 threads.
int rows_of_group(int64_t n_rows, int heads, int vec, bool bf16) {
  const int64_t full = 256 * (bf16 ? items_of<true>() : items_of<false>()) / ((int64_t)heads * vec), spread = (n_rows + cu_count() - 1) / cu_count();
  const int64_t least = (n_rows + (1 << 22) - 1) >> 22;  // 2^26 rows at most: 16
  return (int)std::max<int64_t>({1, least, std::min<int64_t>({full, spread, kMaxRows})});
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& rot, const HeadsArgs (&t)[2], int n_tensors, int n_rows, int d, int x_dtype, int y_dtype, hipStream_t stream) {
  if (n_rows == 0) return hipSuccess;
  HeadsArgs t1 = t[n_tensors - 1];
  if (n_tensors == 1) t1.n_heads = 0;
  const int vec = d / 16, heads = t[0].n_heads + t1.n_heads, each = rows_of_group(n_rows, heads, vec, x_dtype == 0);
  const dim3 grid((unsigned)((n_rows + each - 1) / each)), block(256);
#define MMSP_ROTARY(I, O) rotary_kernel<I, O><<<grid, block, 0, stream>>>(rot, t[0], t1, n_rows, each, __builtin_ctz(vec), fast_div(heads))
  if (x_dtype == 0) MMSP_ROTARY(true, true);
  else if (y_dtype == 0) MMSP_ROTARY(false, true);
  else MMSP_ROTARY(false, false);
#undef MMSP_ROTARY
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, const RotaryArgs* rot, int d, int io_dtype, hipStream_t stream) {
  if (a.cache.n_rows == 0) return hipSuccess;
  const int vec = d / 16, n = a.cache.n_rows, q_rows = a.Hq > 0 ? rows_of_group(n, a.Hq, vec, io_dtype == 0) : 1, kv_rows = rows_of_group(n, 2 * a.Hkv, vec, io_dtype == 0);
  const int q_blocks = a.Hq > 0 ? (n + q_rows - 1) / q_rows : 0;
  const dim3 grid((unsigned)(q_blocks + (n + kv_rows - 1) / kv_rows)), block(256);
  const RotaryArgs none = {};
#define MMSP_APPEND(T, R) append_kernel<T, R><<<grid, block, 0, stream>>>(rot ? *rot : none, a, q_blocks, q_rows, kv_rows, __builtin_ctz(vec), fast_div(std::max(1, a.Hq)), fast_div(2 * a.Hkv))
  if (io_dtype == 0) { if (rot) MMSP_APPEND(true, true); else MMSP_APPEND(true, false); }
  else { if (rot) MMSP_APPEND(false, true); else MMSP_APPEND(false, false); }
#undef MMSP_APPEND
  return hipGetLastError();
}

}  // namespace mmsp
